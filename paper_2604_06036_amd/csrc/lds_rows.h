// Rows from memory to LDS without a stop in registers.  Internal to the library.
#pragma once

#include "common.h"

namespace cs {

// 16 bytes a lane from sbase + off to LDS.  Inline assembly, so that the compiler does not wait for all of them at the next read of LDS:
// the pipeline's own waits do.
__device__ __forceinline__ void to_lds(uint32_t off, const void* sbase, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(sbase), "s"(lds_addr) : "memory", "m0");
}
typedef __attribute__((address_space(3))) void lds_void;
__device__ __forceinline__ uint32_t lds_address(const void* at) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)at)); }

// This wave's requests are in LDS, and its reads of LDS are done; then the others' too.
__device__ __forceinline__ void rows_gate() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// The place in its row where row r holds 16-byte chunk c is c ^ row_place(r): lanes choose which chunk of a row they fetch, so that a read of
// one chunk of 16 rows spreads over the banks.  Rows of 2 * D bytes.
template <int D>
__device__ __forceinline__ int row_place(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }

}  // namespace cs
