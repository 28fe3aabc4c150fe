// Stores of an epilogue whose threads own one row each (as tcgen05.ld gives the accumulators). Not part of the C ABI.
#pragma once

#include <stdint.h>

namespace mcft {

// 32 bytes to global memory in one instruction (a whole sector a lane); 32-byte aligned.
__device__ __forceinline__ void store32(void* p, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// The same in two instructions; 16-byte aligned.
__device__ __forceinline__ void store32_by16(void* p, const uint32_t* v) {
  uint4* q = reinterpret_cast<uint4*>(p);
  q[0] = make_uint4(v[0], v[1], v[2], v[3]);
  q[1] = make_uint4(v[4], v[5], v[6], v[7]);
}

// 64 bytes u of each lane's own row to global memory, at `row` (NULL: none; ALIGN: bytes to which it is aligned, 32 or 16),
// by a whole warp. Two neighbouring lanes first exchange halves, so that an instruction writes 64 contiguous bytes of 16
// rows, not 32 of 32: each line that a store touches takes the way through L1 that the copies into shared memory take too
// (mx4 product of 4096 x 14336 x 4096: 16, 32, 64 and 128 bytes a row 109, 83.2, 82.2 and 83.8 us, the exchange of four
// lanes costing more than it gives).
template <int ALIGN = 32>
__device__ __forceinline__ void store_rows64(void* row, uint32_t* u) {
  static_assert(ALIGN == 32 || ALIGN == 16, "alignment of the rows");
  const uint32_t lane = threadIdx.x & 31u;
  const bool odd = lane & 1u;
#pragma unroll
  for (int e = 0; e < 8; ++e) {  // slot r: row r of the two, half `odd`
    const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? u[e] : u[8 + e], 1);
    if (odd) u[e] = got;
    else u[8 + e] = got;
  }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const unsigned long long at = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), (lane & ~1u) + r);
    char* to = reinterpret_cast<char*>(at) + odd * 32;
    if (at && ALIGN == 32) store32(to, u + 8 * r);
    if (at && ALIGN == 16) store32_by16(to, u + 8 * r);
  }
}

// u[i] of lane j <-> u[j] of lane i: the rows that 32 lanes own, turned so that lane j holds word j of each row, by halves
// of 16, 8, 4, 2 and 1.
__device__ __forceinline__ void transpose32(uint32_t* u) {
  const uint32_t lane = threadIdx.x & 31u;
#pragma unroll
  for (int h = 16; h > 0; h >>= 1) {
    const bool up = lane & uint32_t(h);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (i & h) continue;
      const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? u[i] : u[i | h], h);
      if (up) u[i] = got;
      else u[i | h] = got;
    }
  }
}

}  // namespace mcft
