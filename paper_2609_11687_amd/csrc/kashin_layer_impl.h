// P before and after the products with the codes (kashin_matmul.hip), on the pairs of rows and the transforms of
// kashin_pair_impl.h, which includes this file.
//
// Before: rows of x (fp32, fp16, bf16, e4m3 with scales) to operands of x and P x.  P is an orthonormal involution, so
// |P x| <= sqrt(N) max |x|: the row's exponent, known from the load, scales both factors, and no pass over P x is needed to
// find its largest entry.  After: y = zu + P zv, rounded to y's type.
//
// Few rows are latency: N = 4096 takes 11 us for one row of x or 32 (N = 11008 30 us), of which a transform's arithmetic is
// a small part; the operands of one row leave as 32-byte pieces of 32 KB.  Hence x's own operands are written by workgroups
// of their own, beside those that transform; the rows are asked for before the operator's constants (the plain P
// kernel loads its constants first, once for the many pairs that a workgroup walks); a row without a neighbour is loaded
// and written alone.  2048 bf16 rows of 4096 (50 MB in and out) take 33 us among other calls (39 after a pause, against
// 31 + 29 us of P x into memory and a pass over x and P x), of which the bytes would take 10: the vector ALU issues in
// 59 % of the cycles and LDS works in 44 %.
#pragma once

#include "kashin_rows.h"
#include "kashin_units.h"

namespace kashin {
namespace {

constexpr int half_log2(int n) {  // least h with 2^h >= sqrt(n)
  int h = 0;
  while ((int64_t(1) << (2 * h)) < n) ++h;
  return h;
}

// The rows' largest magnitudes by their bits, the scales from them, and the exponents of both.
template <class C>
__device__ __forceinline__ void layer_scales(const uint32_t (&top)[2], float* red, int& slot, float (&scale)[2], int (&exp)[2]) {
  constexpr uint32_t kInf = 0x7f800000u;
  float most[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) most[w] = __uint_as_float(top[w] < kInf ? top[w] : kInf);
  block_max<C::T, 2>(most, red, slot);
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const bool bad = most[w] > FLT_MAX;
    exp[w] = 0;
    if (!bad && most[w] > 0.f) (void)frexpf(most[w], &exp[w]);
    exp[w] = exp[w] < -126 ? -126 : exp[w];  // as normalise_pair
    scale[w] = bad ? __int_as_float(0x7fc00000) : ldexpf(1.f, -exp[w]);
  }
}

// A vector: group g of a row of x.
template <class T>
struct LayerVector {
  const T* x;
  const float* scales;  // of e4m3 entries: this row's
  int64_t row;
  int g, at;  // at: its first entry in the row
};

// Workgroups 0 .. pairs - 1 transform a pair of vectors each, as many again write the pairs' own operands.
template <class C, class T>
__global__ __launch_bounds__(C::T) __attribute__((amdgpu_waves_per_eu(C::W))) void layer_rows_kernel(LayerArgs a) {
  __shared__ __align__(16) float2 lds[C::LDS + small_tw_total<C>()];
  __shared__ float red[2 * C::NW * 32];
  constexpr bool E4M3 = std::is_same<T, e4m3_t>::value;
  constexpr int N = C::N, H = 15 - half_log2(N);  // x below 2^H after scaling, P x below 2^15
  constexpr int BLOCKS = chunks_per_group(N) * (kChunk / 16);
  constexpr bool RES = resident_ok<C>();
  const float qnan = __int_as_float(0x7fc00000), up = static_cast<float>(1 << H);
  const int64_t all = padded_chunks(N, a.groups) * (kChunk / 16), vectors = a.rows * a.groups, pairs = (vectors + 1) / 2;
  const int past = static_cast<int>(all - static_cast<int64_t>(a.groups) * BLOCKS);  // empty blocks behind a row's last group
  const bool transform = blockIdx.x < pairs;
  const int64_t va = 2 * (transform ? blockIdx.x : blockIdx.x - pairs);
  const int count = va + 1 < vectors ? 2 : 1, tid = opaque(threadIdx.x);
  LayerVector<T> vec[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int64_t v = va + (w < count ? w : 0);
    vec[w].row = a.groups == 1 ? v : v / a.groups;
    vec[w].g = static_cast<int>(v - vec[w].row * a.groups);
    vec[w].at = vec[w].g * N;
    vec[w].x = static_cast<const T*>(a.x) + vec[w].row * a.ldx + vec[w].at;
    if constexpr (E4M3)
      vec[w].scales = a.x_scales + vec[w].row * (a.x_group ? (static_cast<int64_t>(a.groups) * N + a.x_group - 1) / a.x_group : 1);
  }
  // entries i .. i + 7 of a vector's row (i from the vector's first), those from `left` on as zero
  auto load_eight = [&](const LayerVector<T>& v, int i, int left, float* to) {
    float u[8];
    load8(v.x + (left > 0 ? i : 0), left > 0 ? left : 0, u);
    if constexpr (E4M3) {  // a scale's entries begin at a multiple of 32 of the row, a vector at one of four or eight
      constexpr int S = N % 8 == 0 ? 8 : 4;
#pragma unroll
      for (int h = 0; h < 8; h += S) {
        const uint32_t at = static_cast<uint32_t>(v.at + i + h);
        const float s = left > h ? v.scales[a.x_group ? at / static_cast<uint32_t>(a.x_group) : 0] : 0.f;
#pragma unroll
        for (int j = 0; j < S; ++j) u[h + j] *= s;
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) to[j] = u[j];
  };
  auto top_of = [](const float* v, int n, uint32_t t) {
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const uint32_t o = __float_as_uint(v[j]) & 0x7fffffffu;
      t = o > t ? o : t;
    }
    return t;
  };
  // the largest of whole rows, where a row has several vectors
  auto row_tops = [&](uint32_t(&top)[2]) {
    constexpr int B = 4;  // loads on their way together; past the end the last eight again
    const int k = a.groups * N;
    const bool two = count == 2 && vec[1].row != vec[0].row;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if (w == 1 && !two) break;
      for (int i0 = 8 * tid; i0 < k; i0 += 8 * B * C::T) {
        float v[B][8];
#pragma unroll
        for (int b = 0; b < B; ++b) {
          const int i = i0 + 8 * b * C::T;
          load_eight(vec[w], (i < k - 8 ? i : k - 8) - vec[w].at, 8, v[b]);
        }
#pragma unroll
        for (int b = 0; b < B; ++b) top[w] = top_of(v[b], 8, top[w]);
      }
    }
    if (!two) top[1] = top[0];
  };
  _Float16* frags = a.frags + (transform ? 2 * all * a.parts * a.rows * 8 : 0);
  int slot = 0, exp[2];
  float scale[2];
  uint32_t top[2] = {0, 0};
  if (!transform) {
    auto load16 = [&](int b, int which, float (&v)[16]) {
      const LayerVector<T> from = which ? vec[1] : vec[0];
#pragma unroll
      for (int h = 0; h < 2; ++h) load_eight(from, 16 * b + 8 * h, N - 16 * b - 8 * h, v + 8 * h);
    };
    if (a.groups > 1) {
      row_tops(top);
    } else {
      for (int b2 = tid; b2 < BLOCKS * count; b2 += C::T) {
        const int which = count == 2 ? b2 & 1 : 0;
        float v[16];
        load16(count == 2 ? b2 >> 1 : b2, which, v);
        if (which) top[1] = top_of(v, 16, top[1]);
        else top[0] = top_of(v, 16, top[0]);
      }
    }
    layer_scales<C>(top, red, slot, scale, exp);
#pragma unroll
    for (int w = 0; w < 2; ++w)
      if (tid == w && w < count && vec[w].g == 0) a.exps[vec[w].row] = H - exp[w];
    for (int b2 = tid; b2 < (BLOCKS + past) * count; b2 += C::T) {
      const int which = count == 2 ? b2 & 1 : 0, b = count == 2 ? b2 >> 1 : b2;
      const int g = which ? vec[1].g : vec[0].g;
      if (b >= BLOCKS && g != a.groups - 1) continue;
      const float s = which ? scale[1] : scale[0];
      float v[16];
      load16(b, which, v);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] *= s;
      put_units(frags, static_cast<int64_t>(g) * BLOCKS + b, a.parts, a.rows, which ? vec[1].row : vec[0].row, v, up);
    }
    return;
  }
  float2 z[C::E];
#pragma unroll
  for (int e = 0; e < C::E; ++e) z[e] = make_float2(0.f, 0.f);
  float* lf = reinterpret_cast<float*>(lds);
  if constexpr (E4M3) {  // through LDS: a scale is looked up once for four entries
    for (int which = 0; which < count; ++which) {
      const LayerVector<T> from = which ? vec[1] : vec[0];
      for (int i = 8 * tid; i < N; i += 8 * C::T) {
        float v[8];
        load_eight(from, i, N - i, v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (i + j < N) lf[which * N + i + j] = v[j];
      }
    }
    lds_barrier();
    for_each_elem<C>([&](int e, int i) { z[e] = make_float2(lf[i], count == 2 ? lf[N + i] : 0.f); }, tid);
    lds_barrier();  // read out before the first pass writes
  } else {
    for_each_elem<C>([&](int e, int i) { z[e].x = widen(vec[0].x[i]); }, tid);
    if (count == 2) for_each_elem<C>([&](int e, int i) { z[e].y = widen(vec[1].x[i]); }, tid);
  }
  if (a.groups > 1) row_tops(top);
  ResRegs<C> rr;
  if constexpr (RES) resident_load<C>(rr, lds, a.tw, a.mid4);
  float2 by, unscale;
  bool bad[2];
  if (a.groups == 1) {
    normalise_pair<C>(z, red, slot, by, unscale, bad[0], bad[1]);
  } else {
    layer_scales<C>(top, red, slot, scale, exp);
    bad[0] = scale[0] != scale[0];
    bad[1] = scale[1] != scale[1];
#pragma unroll
    for (int e = 0; e < C::E; ++e) {  // a row that is not finite does not reach its neighbour
      z[e].x = bad[0] ? 0.f : z[e].x * scale[0];
      z[e].y = bad[1] ? 0.f : z[e].y * scale[1];
    }
  }
  if constexpr (RES) apply_P_res<C>(z, lds, rr);
  else apply_P<C>(z, lds, a.tw, a.mid4);
  lds_barrier();  // the last pass read the buffer
  for_each_elem<C>([&](int e, int i) {
    lf[i] = bad[0] ? qnan : z[e].x;
    if (count == 2) lf[N + i] = bad[1] ? qnan : z[e].y;
  }, tid);
  lds_barrier();
  for (int b2 = tid; b2 < (BLOCKS + past) * count; b2 += C::T) {
    const int which = count == 2 ? b2 & 1 : 0, b = count == 2 ? b2 >> 1 : b2;
    const int g = which ? vec[1].g : vec[0].g;
    if (b >= BLOCKS && g != a.groups - 1) continue;
    float v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = 16 * b + j < N ? lf[which * N + 16 * b + j] : 0.f;
    put_units(frags, static_cast<int64_t>(g) * BLOCKS + b, a.parts, a.rows, which ? vec[1].row : vec[0].row, v, up);
  }
}

// y = zu + P zv: the end of the transposed products (one row of 4096: 11 us, 509 rows 15; reading zu and zv and writing y would
// take 4 us there, the transform's latency of a pair a compute unit the rest).  A workgroup walks pairs of vectors; a vector passes through LDS into
// row order, where zu is added and y written in 16-byte pieces.
template <class C>
__global__ __launch_bounds__(C::T) __attribute__((amdgpu_waves_per_eu(C::W))) void layer_back_kernel(LayerBackArgs a) {
  __shared__ __align__(16) float2 lds[C::LDS + small_tw_total<C>()];
  __shared__ float red[2 * C::NW * 32];
  constexpr int N = C::N;
  constexpr bool RES = resident_ok<C>();
  const float qnan = __int_as_float(0x7fc00000);
  const int64_t vectors = a.t * a.groups, pairs = (vectors + 1) / 2;
  const int tid = opaque(threadIdx.x);
  const float4_t* lf4 = reinterpret_cast<const float4_t*>(lds);
  float* lf = reinterpret_cast<float*>(lds);
  int slot = 0;
  float2 z[C::E];
  auto load = [&](int64_t p) {
    const int64_t ra = 2 * p, rb = ra + 1 < vectors ? ra + 1 : -1;
    load_pair_t<C>(z, a.zv, N, ra, rb, tid);
  };
  load(blockIdx.x);  // gridDim.x <= pairs
  ResRegs<C> rr;
  if constexpr (RES) resident_load<C>(rr, lds, a.tw, a.mid4);
  for (int64_t p = blockIdx.x; p < pairs; p += gridDim.x) {
    float2 scale, unscale;
    bool bad[2];
    normalise_pair<C>(z, red, slot, scale, unscale, bad[0], bad[1]);
    unscale.x = bad[0] ? qnan : unscale.x;
    unscale.y = bad[1] ? qnan : unscale.y;
    if constexpr (RES) apply_P_res<C>(z, lds, rr);
    else apply_P<C>(z, lds, a.tw, a.mid4);
    lds_barrier();  // the last pass read the buffer
    for_each_elem<C>([&](int e, int i) {
      lf[i] = z[e].x * unscale.x;
      lf[N + i] = z[e].y * unscale.y;
    }, tid);
    if (p + gridDim.x < pairs) load(p + gridDim.x);
    lds_barrier();
    for (int which = 0; which < 2; ++which) {
      const int64_t v = 2 * p + which;
      if (v >= vectors) break;
      const int64_t row = a.groups == 1 ? v : v / a.groups, at = row * a.ldy + (v - row * a.groups) * N;
      if (a.offsets != nullptr && (row < a.offsets[0] || row >= a.offsets[a.experts])) continue;
      for (int i = tid; i < N / 4; i += C::T) {
        const float4_t o = lf4[which * (N / 4) + i] + *reinterpret_cast<const float4_t*>(a.zu + v * N + 4 * i);
        const float q[4] = {o[0], o[1], o[2], o[3]};
        put4(a.y, a.y_dtype, at + 4 * i, 4, q);
      }
    }
    lds_barrier();  // read out before the next pair's first pass writes
  }
}

template <class C>
hipError_t launch_layer_cfg(const LayerArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.rows * a.groups + 1) / 2 * 2)), bd(C::T);
  if (a.x_dtype == KASHIN_E4M3) {
    hipLaunchKernelGGL((layer_rows_kernel<C, e4m3_t>), grid, bd, 0, s, a);
  } else {
    with_float_type(a.x_dtype, [&](auto zero) {
      hipLaunchKernelGGL((layer_rows_kernel<C, decltype(zero)>), grid, bd, 0, s, a);
    });
  }
  return hipGetLastError();
}

template <class C>
hipError_t launch_layer_back_cfg(const LayerBackArgs& a, hipStream_t s) {
  const int64_t pairs = (a.t * a.groups + 1) / 2;
  hipLaunchKernelGGL((layer_back_kernel<C>), dim3(static_cast<unsigned>(std::min<int64_t>(pairs, kPmapGrid))), dim3(C::T), 0,
                     s, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace kashin
