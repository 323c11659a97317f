// P in front of the products with the codes (kashin_matmul.hip): rows of x (fp32, fp16, bf16) to operands of x and P x.
// Included by kashin_pair_impl.h, whose pairs of rows and transforms it runs.
//
// P is an orthonormal involution, so |P x| <= sqrt(N) max |x|: the row's exponent, known from the load, scales both
// factors, and no pass over P x is needed to find its largest entry.
//
// It is latency at few rows (one token 4096 wide: 10.3 us of P and 3.8 of a pass of its own over x and P x become one
// launch), hence: x's own operands are written by workgroups of their own, beside those that transform; the rows are
// asked for before the operator's constants (the plain P kernel loads its constants first, once for the many
// pairs that a workgroup walks); a row without a neighbour is loaded and written alone.
#pragma once

#include "kashin_rows.h"
#include "kashin_units.h"

namespace kashin {
namespace {

template <class IT>
struct RowType {
  using type = float;
};
template <>
struct RowType<__half> {
  using type = _Float16;
};
template <>
struct RowType<bf16_t> {
  using type = __bf16;
};

constexpr int half_log2(int n) {  // least h with 2^h >= sqrt(n)
  int h = 0;
  while ((int64_t(1) << (2 * h)) < n) ++h;
  return h;
}

// Workgroups 0 .. pairs - 1 transform a pair of rows each, as many again write the pairs' own operands.
template <class C, class IT>
__global__ __launch_bounds__(C::T) __attribute__((amdgpu_waves_per_eu(C::W))) void layer_rows_kernel(LayerArgs a) {
  __shared__ __align__(16) float2 lds[C::LDS + small_tw_total<C>()];
  __shared__ float red[2 * C::NW * 32];
  constexpr int N = C::N, H = 15 - half_log2(N);  // x below 2^H after scaling, P x below 2^15
  constexpr int BLOCKS = static_cast<int>(padded_chunks(N, 1)) * (kChunk / 16);
  constexpr bool RES = resident_ok<C>();
  const float qnan = __int_as_float(0x7fc00000), up = static_cast<float>(1 << H);
  const int64_t pairs = (a.rows + 1) / 2;
  const bool transform = blockIdx.x < pairs;
  const int64_t ra = 2 * (transform ? blockIdx.x : blockIdx.x - pairs), rb = ra + 1 < a.rows ? ra + 1 : -1;
  const int rows = rb < 0 ? 1 : 2, tid = opaque(threadIdx.x);
  _Float16* frags = a.frags + (transform ? static_cast<int64_t>(2 * BLOCKS) * a.parts * a.rows * 8 : 0);
  int slot = 0;
  if (!transform) {
    using T = typename RowType<IT>::type;
    auto load16 = [&](int b, int which, float (&v)[16]) {
      const T* x = static_cast<const T*>(a.x) + (ra + which) * a.ldx;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float u[8];
        const int i = 16 * b + 8 * h;
        load8(x + (i < N ? i : 0), i < N ? N - i : 0, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[8 * h + j] = u[j];
      }
    };
    // the scale as normalise_pair finds it: of the largest magnitude by its bits
    uint32_t top[2] = {0, 0};
    for (int b2 = tid; b2 < BLOCKS * rows; b2 += C::T) {
      const int which = rows == 2 ? b2 & 1 : 0;
      float v[16];
      load16(rows == 2 ? b2 >> 1 : b2, which, v);
      uint32_t t = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const uint32_t o = __float_as_uint(v[j]) & 0x7fffffffu;
        t = o > t ? o : t;
      }
      if (which) top[1] = t > top[1] ? t : top[1];
      else top[0] = t > top[0] ? t : top[0];
    }
    constexpr uint32_t kInf = 0x7f800000u;
    float most[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) most[w] = __uint_as_float(top[w] < kInf ? top[w] : kInf);
    block_max<C::T, 2>(most, red, slot);
    float scale[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      int e = 0;
      if (most[w] <= FLT_MAX && most[w] > 0.f) (void)frexpf(most[w], &e);
      e = e < -126 ? -126 : e;
      scale[w] = most[w] <= FLT_MAX ? ldexpf(1.f, -e) : qnan;
      if (tid == w && w < rows) a.exps[ra + w] = H - e;
    }
    for (int b2 = tid; b2 < BLOCKS * rows; b2 += C::T) {
      const int which = rows == 2 ? b2 & 1 : 0, b = rows == 2 ? b2 >> 1 : b2;
      const float s = which ? scale[1] : scale[0];
      float v[16];
      load16(b, which, v);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] *= s;
      put_units(frags, b, a.parts, a.rows, ra + which, v, up);
    }
    return;
  }
  float2 z[C::E];
#pragma unroll
  for (int e = 0; e < C::E; ++e) z[e] = make_float2(0.f, 0.f);
  if (rb >= 0) {
    load_pair_t<C>(z, static_cast<const IT*>(a.x), a.ldx, ra, rb, tid);
  } else {
    const IT* x = static_cast<const IT*>(a.x) + ra * a.ldx;
    for_each_elem<C>([&](int e, int i) { z[e].x = to_f32(x[i]); }, tid);
  }
  ResRegs<C> rr;
  if constexpr (RES) resident_load<C>(rr, lds, a.tw, a.mid4);
  float2 scale, unscale;
  bool bad_a, bad_b;
  normalise_pair<C>(z, red, slot, scale, unscale, bad_a, bad_b);
  if constexpr (RES) apply_P_res<C>(z, lds, rr);
  else apply_P<C>(z, lds, a.tw, a.mid4);
  lds_barrier();  // the last pass read the buffer
  float* lf = reinterpret_cast<float*>(lds);
  for_each_elem<C>([&](int e, int i) {
    lf[i] = bad_a ? qnan : z[e].x;
    if (rows == 2) lf[N + i] = bad_b ? qnan : z[e].y;
  }, tid);
  lds_barrier();
  for (int b2 = tid; b2 < BLOCKS * rows; b2 += C::T) {
    const int which = rows == 2 ? b2 & 1 : 0, b = rows == 2 ? b2 >> 1 : b2;
    float v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = 16 * b + j < N ? lf[which * N + 16 * b + j] : 0.f;
    put_units(frags, b, a.parts, a.rows, ra + which, v, up);
  }
}

template <class C>
hipError_t launch_layer_cfg(const LayerArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.rows + 1) / 2 * 2)), bd(C::T);
  if (a.x_dtype == KASHIN_F16) hipLaunchKernelGGL((layer_rows_kernel<C, __half>), grid, bd, 0, s, a);
  else if (a.x_dtype == KASHIN_BF16) hipLaunchKernelGGL((layer_rows_kernel<C, bf16_t>), grid, bd, 0, s, a);
  else hipLaunchKernelGGL((layer_rows_kernel<C, float>), grid, bd, 0, s, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace kashin
