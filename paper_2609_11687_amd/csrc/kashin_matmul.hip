// Products with the codes of a quantised matrix (App. C: X W^T = [X | X P] [U | V]^T): y = x W^T and y = x W for
// W = U + V P held as two 2-bit codes an entry and four centres a factor for each row and group, whole or
// grouped by expert.
#include "kashin_internal.h"
#include "kashin_rows.h"

namespace kashin {
namespace {

constexpr int64_t align256(int64_t v) { return (v + 255) & ~int64_t(255); }

// Rows lo .. hi - 1 of expert e, within [0, t] whatever the offsets hold.
__device__ __forceinline__ void expert_rows(const int64_t* offsets, int e, int64_t t, int64_t& lo, int64_t& hi) {
  lo = offsets[e];
  hi = offsets[e + 1];
  lo = lo < 0 ? 0 : lo > t ? t : lo;
  hi = hi < lo ? lo : hi > t ? t : hi;
}

// Tile number `tile` of at most TT rows that belong to one expert, tiles counted over the experts in turn; rows 0
// past the last tile.  Every lane of the wave calls it.
struct Tile {
  int expert;
  int64_t row0;
  int rows;
};
template <int TT>
__device__ Tile find_tile(const int64_t* offsets, int experts, int64_t t, int tile) {
  Tile r = {0, 0, 0};
  if (offsets == nullptr) {
    r.row0 = static_cast<int64_t>(tile) * TT;
    const int64_t left = t - r.row0;
    r.rows = left > TT ? TT : left > 0 ? static_cast<int>(left) : 0;
    return r;
  }
  const int lane = threadIdx.x % 64;
  int before = 0;
  for (int e0 = 0; e0 < experts; e0 += 64) {
    int64_t lo = 0, hi = 0;
    if (e0 + lane < experts) expert_rows(offsets, e0 + lane, t, lo, hi);
    const int tiles = static_cast<int>((hi - lo + TT - 1) / TT);
    int upto = tiles;  // tiles of this block's experts up to and with this lane's
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    const uint64_t past = __ballot(before + upto > tile);
    if (past != 0) {
      const int f = __ffsll(static_cast<unsigned long long>(past)) - 1;
      const int first = before + __shfl(upto - tiles, f);
      const int64_t l = __shfl(static_cast<long long>(lo), f), h = __shfl(static_cast<long long>(hi), f);
      r.expert = e0 + f;
      r.row0 = l + static_cast<int64_t>(tile - first) * TT;
      r.rows = static_cast<int>(h - r.row0 < TT ? h - r.row0 : TT);
      return r;
    }
    before += __shfl(upto, 63);
  }
  return r;
}
// The most tiles that offsets in order can give: whole ones, and a partial one for each expert with rows.
int64_t most_tiles(const ProductArgs& a, int64_t tt) {
  if (a.offsets == nullptr) return (a.t + tt - 1) / tt;
  return a.t / tt + (a.experts < a.t ? a.experts : a.t);
}

// x as contiguous fp32 rows.
template <class T>
__global__ __launch_bounds__(256) void widen_kernel(const T* x, int64_t ldx, const float* scales, int group, int64_t width,
                                                    float* out) {
  const int64_t row = blockIdx.x;
  const int64_t i = (static_cast<int64_t>(blockIdx.y) * 256 + threadIdx.x) * 8;
  if (i >= width) return;
  const int valid = width - i < 8 ? static_cast<int>(width - i) : 8;
  float v[8];
  load8(x + row * ldx + i, valid, v);
  if (scales != nullptr) {  // a group is a multiple of 32 entries: the eight share one
    const float s = group ? scales[row * ((width + group - 1) / group) + i / group] : scales[row];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= s;
  }
  store8(out + row * width + i, valid, v);
}

__device__ __forceinline__ float pick(const float* q, int c) { return c & 2 ? (c & 1 ? q[3] : q[2]) : (c & 1 ? q[1] : q[0]); }

__device__ __forceinline__ void put(void* y, int dtype, int64_t i, float v) {
  if (dtype == KASHIN_F32) static_cast<float*>(y)[i] = v;
  else if (dtype == KASHIN_F16) static_cast<_Float16*>(y)[i] = static_cast<_Float16>(v);
  else static_cast<__bf16*>(y)[i] = static_cast<__bf16>(v);
}

// y[t][i] = sum_k u[i][k] x[t][k] + v[i][k] px[t][k]: a wave for each matrix row and tile of four rows.
constexpr int kTT = 4;
__global__ __launch_bounds__(64) void rows_kernel(ProductArgs a, const float* x, const float* px) {
  const Tile tl = find_tile<kTT>(a.offsets, a.experts, a.t, blockIdx.y);
  if (tl.rows == 0) return;
  const int n = a.n, nby = n / 4, lane = threadIdx.x;
  const int64_t k = static_cast<int64_t>(a.groups) * n, i = blockIdx.x;
  float acc[kTT] = {};
  for (int g = 0; g < a.groups; ++g) {
    const int64_t row = (tl.expert * a.m + i) * a.groups + g;
    const float* q = a.centers + row * 8;
    for (int b = lane; b < nby; b += 64) {
      const int cu = a.codes_u[row * nby + b], cv = a.codes_v[row * nby + b];
#pragma unroll
      for (int s = 0; s < kTT; ++s) {
        if (s >= tl.rows) break;
        const int64_t at = (tl.row0 + s) * k + g * n + 4 * b;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[s] += pick(q, (cu >> (2 * j)) & 3) * x[at + j] + pick(q + 4, (cv >> (2 * j)) & 3) * px[at + j];
      }
    }
  }
#pragma unroll
  for (int s = 0; s < kTT; ++s) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) acc[s] += __shfl_xor(acc[s], d);
    if (lane == 0 && s < tl.rows) put(a.y, a.y_dtype, (tl.row0 + s) * a.ldy + i, acc[s]);
  }
}

// zu[t][j] = sum_i x[t][i] u[i][j], zv alike: a thread for each byte of codes (four columns).
__global__ __launch_bounds__(64) void columns_kernel(ProductArgs a, const float* x, float* zu, float* zv) {
  const Tile tl = find_tile<kTT>(a.offsets, a.experts, a.t, blockIdx.y);
  if (tl.rows == 0) return;
  const int n = a.n, nby = n / 4;
  const int64_t k = static_cast<int64_t>(a.groups) * n;
  const int64_t col = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x;  // byte of the row of all groups
  if (col >= k / 4) return;
  const int g = static_cast<int>(col / nby), b = static_cast<int>(col % nby);
  float au[kTT][4] = {}, av[kTT][4] = {};
  for (int64_t i = 0; i < a.m; ++i) {
    const int64_t row = (tl.expert * a.m + i) * a.groups + g;
    const float* q = a.centers + row * 8;
    const int cu = a.codes_u[row * nby + b], cv = a.codes_v[row * nby + b];
#pragma unroll
    for (int s = 0; s < kTT; ++s) {
      if (s >= tl.rows) break;
      const float xs = x[(tl.row0 + s) * a.m + i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        au[s][j] += pick(q, (cu >> (2 * j)) & 3) * xs;
        av[s][j] += pick(q + 4, (cv >> (2 * j)) & 3) * xs;
      }
    }
  }
#pragma unroll
  for (int s = 0; s < kTT; ++s) {
    if (s >= tl.rows) break;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      zu[(tl.row0 + s) * k + 4 * col + j] = au[s][j];
      zv[(tl.row0 + s) * k + 4 * col + j] = av[s][j];
    }
  }
}

// Whether a row belongs to an expert (all do without offsets).
__device__ __forceinline__ bool covered(const int64_t* offsets, int experts, int64_t row) {
  return offsets == nullptr || (row >= offsets[0] && row < offsets[experts]);
}

// Rows that no expert has, as zeros: P takes rows in pairs, and what lies in a row's neighbour may show in its last
// bits.
__global__ __launch_bounds__(256) void clear_spare_kernel(const int64_t* offsets, int experts, int64_t width, float* z) {
  if (covered(offsets, experts, blockIdx.x)) return;
  const int64_t i = static_cast<int64_t>(blockIdx.y) * 256 + threadIdx.x;
  if (i < width) z[blockIdx.x * width + i] = 0.f;
}

// z += pz (fp32 rows)
__global__ __launch_bounds__(256) void add_kernel(float* z, const float* pz, int64_t count) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i < count) z[i] += pz[i];
}

// y = z in y's type, covered rows only.
__global__ __launch_bounds__(256) void narrow_kernel(ProductArgs a, const float* z, int64_t width) {
  if (!covered(a.offsets, a.experts, blockIdx.x)) return;
  const int64_t i = static_cast<int64_t>(blockIdx.y) * 256 + threadIdx.x;
  if (i < width) put(a.y, a.y_dtype, blockIdx.x * a.ldy + i, z[blockIdx.x * width + i]);
}

hipError_t widen(const ProductArgs& a, int64_t width, float* out, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.t), static_cast<unsigned>((width + 2047) / 2048));
  if (a.x_dtype == KASHIN_E4M3) {
    hipLaunchKernelGGL((widen_kernel<e4m3_t>), grid, dim3(256), 0, s, static_cast<const e4m3_t*>(a.x), a.ldx, a.x_scales,
                       a.x_group, width, out);
  } else {
    with_float_type(a.x_dtype, [&](auto zero) {
      using T = decltype(zero);
      hipLaunchKernelGGL((widen_kernel<T>), grid, dim3(256), 0, s, static_cast<const T*>(a.x), a.ldx, nullptr, 0, width,
                         out);
    });
  }
  return hipGetLastError();
}

// out = P in, t rows of `groups` vectors
hipError_t apply_p(const ProductArgs& a, const float* in, float* out, hipStream_t s) {
  KArgs p = a.p;
  p.w = in;
  p.ldw = a.n;
  p.m = a.t * a.groups;
  p.y = out;
  p.ldy = a.n;
  return launch_pair(a.n, p, (p.m + 1) / 2, s);
}

hipError_t rotate(const ProductArgs& a, bool inverse, float* z, hipStream_t s) {
  return launch_rotate(a.n, a.rot_seed, inverse, z, KASHIN_F32, a.n, z, a.n, a.t * a.groups, s);
}

}  // namespace

int64_t product_workspace_bytes(int n, int64_t m, int groups, int64_t t, int experts, bool back) {
  (void)experts;
  const int64_t k = static_cast<int64_t>(groups) * n;
  return align256(t * (back ? m : k) * 4) + (back ? 3 : 1) * align256(t * k * 4);
}

hipError_t launch_product(const ProductArgs& a, hipStream_t s) {
  const int64_t k = static_cast<int64_t>(a.groups) * a.n, wx = a.back ? a.m : k;
  float* x = reinterpret_cast<float*>(a.work);
  float* z[3];
  for (int i = 0; i < 3; ++i) z[i] = reinterpret_cast<float*>(a.work + align256(a.t * wx * 4) + i * align256(a.t * k * 4));
  const unsigned tiles = static_cast<unsigned>(most_tiles(a, kTT)), t = static_cast<unsigned>(a.t);
  hipError_t e = widen(a, wx, x, s);
  if (e != hipSuccess) return e;
  if (!a.back) {
    if (a.rot) e = rotate(a, false, x, s);
    if (e == hipSuccess) e = apply_p(a, x, z[0], s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(rows_kernel, dim3(static_cast<unsigned>(a.m), tiles), dim3(64), 0, s, a, x, z[0]);
    return hipGetLastError();
  }
  const dim3 whole(t, static_cast<unsigned>((k + 255) / 256));
  if (a.offsets != nullptr) {
    hipLaunchKernelGGL(clear_spare_kernel, whole, dim3(256), 0, s, a.offsets, a.experts, k, z[1]);
    hipLaunchKernelGGL(clear_spare_kernel, whole, dim3(256), 0, s, a.offsets, a.experts, k, z[0]);
  }
  hipLaunchKernelGGL(columns_kernel, dim3(static_cast<unsigned>((k / 4 + 63) / 64), tiles), dim3(64), 0, s, a, x, z[0], z[1]);
  e = hipGetLastError();
  if (e == hipSuccess) e = apply_p(a, z[1], z[2], s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(add_kernel, dim3(static_cast<unsigned>((a.t * k + 255) / 256)), dim3(256), 0, s, z[0], z[2], a.t * k);
  e = hipGetLastError();
  if (e == hipSuccess && a.rot) e = rotate(a, true, z[0], s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(narrow_kernel, whole, dim3(256), 0, s, a, z[0], k);
  return hipGetLastError();
}

}  // namespace kashin
