// Root-mean-square norm of rows with the residual's addition, and an output in 8 bits with scales:
//   s = x + r,  h = s,  y = s rsqrt(mean(s^2) + eps) weight,  scale_g = max|y_g| / 448,  y8 = e4m3(y / scale_g).
//
// A row is read once and stays in registers: NT threads hold it, eight consecutive entries each, C times
// over (entry (c NT + tid) 8 + j), so that a group of 32 .. 256 entries is 4 .. 32 neighbouring lanes and its
// maximum a few shuffles.  The sum of squares is fp32: eight entries in a thread, the wave by shuffles, the
// waves through LDS in a fixed order, so that results repeat bit for bit.
//
// Bound by memory: 8192 bf16 rows of 8192 with r and h (537 MB) take 102 to 104 us, 5.2 TB/s against 5.1 of a
// large copy; one row of 4096 is 4 us, the launch.  With e4m3 output and scales (472 MB) the vector ALU issues in 83 % of the
// cycles: 115 to 120 us.
#include "kashin_internal.h"
#include "kashin_rows.h"

namespace kashin {
namespace {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// The largest bit pattern over `lanes` neighbouring lanes (a power of two).  |v| as bits orders like |v|, with NaN above
// all numbers, so a NaN is not lost as fmaxf would lose it.
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int lanes) {
  for (int d = 1; d < lanes; d <<= 1) {
    const uint32_t o = __shfl_xor(v, d);
    v = o > v ? o : v;
  }
  return v;
}

// NT threads of a row: 64 (four rows a workgroup) to 1024.
template <class T, int NT, int C>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void rmsnorm_kernel(NormArgs a) {
  constexpr int RPW = NT < 256 ? 256 / NT : 1;  // rows a workgroup
  constexpr int NW = NT / 64;
  __shared__ float part[2][NW];
  __shared__ uint32_t peak[2][NW];
  const int tid = threadIdx.x % NT, n = a.n;
  const T* weight = static_cast<const T*>(a.weight);
  int slot = 0;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * RPW + threadIdx.x / NT; row < a.t;
       row += static_cast<int64_t>(gridDim.x) * RPW, slot ^= 1) {
    float s[C][8];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int i = (c * NT + tid) * 8;
      load8(static_cast<const T*>(a.x) + row * a.ldx + i, n - i, s[c]);
      if (a.r != nullptr) {
        float r[8];
        load8(static_cast<const T*>(a.r) + row * a.ldr + i, n - i, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[c][j] += r[j];
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fmaf(s[c][j], s[c][j], sum);
    }
    if (a.h != nullptr) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int i = (c * NT + tid) * 8;
        store8(static_cast<T*>(a.h) + row * a.ldh + i, n - i, s[c]);
      }
    }
    sum = wave_sum(sum);
    if constexpr (NW > 1) {
      if (tid % 64 == 0) part[slot][tid / 64] = sum;
      __syncthreads();
      sum = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) sum += part[slot][w];
    }
    const float inv = 1.f / sqrtf(sum / static_cast<float>(n) + a.eps);
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int i = (c * NT + tid) * 8;
      float w[8];
      if (weight != nullptr) {
        load8(weight + i, n - i, w);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[c][j] *= inv;
        if (weight != nullptr) s[c][j] *= w[j];
        if (i + j >= n) s[c][j] = 0.f;  // beyond the row (0 * inf would be NaN)
      }
    }
    if (a.y_dtype == KASHIN_F32) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int i = (c * NT + tid) * 8;
        store8(static_cast<float*>(a.y) + row * a.ldy + i, n - i, s[c]);
      }
      continue;
    }
    if (a.y_dtype == KASHIN_F16) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int i = (c * NT + tid) * 8;
        store8(static_cast<_Float16*>(a.y) + row * a.ldy + i, n - i, s[c]);
      }
      continue;
    }
    if (a.y_dtype == KASHIN_BF16) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int i = (c * NT + tid) * 8;
        store8(static_cast<__bf16*>(a.y) + row * a.ldy + i, n - i, s[c]);
      }
      continue;
    }
    uint32_t tops[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      tops[c] = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t b = __float_as_uint(s[c][j]) & 0x7fffffffu;
        tops[c] = b > tops[c] ? b : tops[c];
      }
      top = tops[c] > top ? tops[c] : top;
    }
    if (a.group == 0) {
      top = lanes_max(top, 64);
      if constexpr (NW > 1) {
        if (tid % 64 == 0) peak[slot][tid / 64] = top;
        __syncthreads();
        top = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) top = peak[slot][w] > top ? peak[slot][w] : top;
      }
#pragma unroll
      for (int c = 0; c < C; ++c) tops[c] = top;
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) tops[c] = lanes_max(tops[c], a.group / 8);
    }
    const int groups = a.group ? (n + a.group - 1) / a.group : 1;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int i = (c * NT + tid) * 8;
      // a group with an infinite entry has no more a scale than one with a NaN
      const float scale = tops[c] < 0x7f800000u ? __uint_as_float(tops[c]) / 448.f : __uint_as_float(0x7fc00000u);
      if (i < n && (a.group ? i % a.group == 0 : i == 0))
        a.scales[row * groups + (a.group ? i / a.group : 0)] = scale;
      // zeros for a group of zeros (scale 0) and for one that is not finite (scale NaN)
      float q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = scale > 0.f ? fminf(fmaxf(s[c][j] / scale, -448.f), 448.f) : 0.f;
      store8(static_cast<e4m3_t*>(a.y) + row * a.ldy + i, n - i, q);
    }
  }
}

template <class T, int NT, int C>
hipError_t launch_as(const NormArgs& a, hipStream_t stream) {
  constexpr int64_t rpw = NT < 256 ? 256 / NT : 1;
  const int64_t wgs = (a.t + rpw - 1) / rpw, most = int64_t(1) << 20;
  hipLaunchKernelGGL((rmsnorm_kernel<T, NT, C>), dim3(static_cast<unsigned>(wgs < most ? wgs : most)),
                     dim3(NT < 256 ? 256 : NT), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs& a, int dtype, hipStream_t stream) {
  // The fewest threads that hold the row in eight entries each, so that all its loads are under way at once, and short rows
  // four to a workgroup (16384 bf16 rows with e4m3 output, us: 512 wide 64 threads 16 and 256 threads 37; 2048 wide 256
  // threads 48 and 64 of 32 entries 56); from 4097 on two eights, which leave room for three rows a compute unit and more
  // (8192 wide 512 threads 216 and 1024 277; 16384 wide 1024 threads 538, 512 of 32 entries 517, but one pass over 64 rows 8.7
  // and 10.3).
  return with_float_type(dtype, [&](auto zero) {
    using T = decltype(zero);
    if (a.n <= 512) return launch_as<T, 64, 1>(a, stream);
    if (a.n <= 2048) return launch_as<T, 256, 1>(a, stream);
    if (a.n <= 4096) return launch_as<T, 512, 1>(a, stream);
    if (a.n <= 8192) return launch_as<T, 512, 2>(a, stream);
    return launch_as<T, 1024, 2>(a, stream);
  });
}

}  // namespace kashin
