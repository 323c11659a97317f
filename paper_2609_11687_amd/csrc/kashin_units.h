// How rows of x and of P x lie as operands of the products with the codes (kashin_matmul.hip), shared with the
// kernel that applies P and writes them so (kashin_layer_impl.h).
//
// A lane decodes codes 16 bytes (a chunk of 64) at a time, eight at a time (a unit) into an operand register block of
// a matrix instruction.  frags[factor][unit][part][row][8]: hi (part 0) and, where there are `parts` = 2, lo parts of
// scaled x (factor 0) and P x, eight entries of a row in the order of a unit's codes; rows innermost, so that the lanes of an
// operand read consecutive 16 bytes.  exps[row]: the exponent of the scale, for both factors.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace kashin {

using half8 = _Float16 __attribute__((ext_vector_type(8)));
using float4_t = float __attribute__((ext_vector_type(4)));

constexpr int kChunk = 64;  // codes of a 16-byte load
constexpr int kUnits = 8;   // units of a chunk
constexpr int kSlab = 4;    // chunks that the four quarters of a wave work on side by side

__host__ __device__ constexpr int chunks_per_group(int n) { return (n + kChunk - 1) / kChunk; }
// chunks of a factor, to a multiple of the slab (the last ones may be empty)
__host__ __device__ constexpr int64_t padded_chunks(int n, int groups) {
  return (static_cast<int64_t>(groups) * chunks_per_group(n) + kSlab - 1) / kSlab * kSlab;
}

// Entry k of a unit's eight: units 2d and 2d + 1 of a chunk come from its dword d, whose 16 codes leave four at a time, two
// bits of every byte.
__host__ __device__ constexpr int unit_entry(int unit, int k) {
  return 16 * (unit / 2) + 2 * (unit % 2) + k / 4 + 4 * (k % 4);
}

// Sixteen entries v of a row, times scale, as its units 2b and 2b + 1 of a factor (frags: that factor's), hi and lo parts.
__device__ __forceinline__ void put_units(_Float16* frags, int64_t b, int parts, int64_t t, int64_t row, const float (&v)[16],
                                          float scale) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    half8 h, l;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float w = v[unit_entry(u, j)] * scale;
      h[j] = static_cast<_Float16>(w);
      l[j] = static_cast<_Float16>(w - static_cast<float>(h[j]));
    }
    *reinterpret_cast<half8*>(frags + ((2 * b + u) * parts * t + row) * 8) = h;
    if (parts == 2) *reinterpret_cast<half8*>(frags + ((2 * b + u) * 2 * t + t + row) * 8) = l;
  }
}

}  // namespace kashin
