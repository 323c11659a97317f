// Products with the codes of a quantised matrix (App. C: X W^T = [X | X P] [U | V]^T): y = x W^T and y = x W for
// W = U + V P held as two 2-bit codes an entry and four centres a factor for each row and group, whole or
// grouped by expert.
#include "kashin_internal.h"
#include "kashin_rows.h"
#include "kashin_units.h"

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

// A value that is the same in all lanes, as the compiler can use it for scalar addresses and branches.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<int>(v >> 32));
  return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// The largest value of a wave, the same in all lanes (an atomic maximum of 64 lanes on one address would go through them
// one by one).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t max_with(uint32_t v) {
  const uint32_t o = static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(static_cast<int>(v), static_cast<int>(v), CTRL, ROWS, 0xf, false));
  return o > v ? o : v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max_with<0xb1, 0xf>(v);   // lanes 1 apart in fours
  v = max_with<0x4e, 0xf>(v);   // 2 apart
  v = max_with<0x141, 0xf>(v);  // halves of a row of 16 mirrored
  v = max_with<0x140, 0xf>(v);  // rows mirrored
  v = max_with<0x142, 0xa>(v);  // row 0 into 1, 2 into 3
  v = max_with<0x143, 0xc>(v);  // rows 0, 1 into 2, 3
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63));
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
      r.expert = uniform(e0 + f);
      r.row0 = uniform(l + static_cast<int64_t>(tile - first) * TT);
      r.rows = uniform(static_cast<int>(h - r.row0 < TT ? h - r.row0 : TT));
      return r;
    }
    before += uniform(__shfl(upto, 63));
  }
  return r;
}
// The most tiles that offsets in order can give: whole ones, and a partial one for each expert with rows.
int64_t most_tiles(bool grouped, int64_t t, int experts, int64_t tt) {
  if (!grouped) return (t + tt - 1) / tt;
  return t / tt + (experts < t ? experts : t);
}

// Rows of x as a kernel reads them: the caller's (fp32, fp16, bf16) or fp32 ones in the workspace.
struct XRows {
  const void* p;
  int64_t ld;
  int dtype;
};
__device__ __forceinline__ void load_row8(const XRows& x, int64_t at, int valid, float (&v)[8]) {
  if (x.dtype == KASHIN_F32) load8(static_cast<const float*>(x.p) + at, valid, v);
  else if (x.dtype == KASHIN_F16) load8(static_cast<const _Float16*>(x.p) + at, valid, v);
  else load8(static_cast<const __bf16*>(x.p) + at, valid, v);
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

__device__ __forceinline__ void put(void* y, int dtype, int64_t i, float v) {
  if (dtype == KASHIN_F32) static_cast<float*>(y)[i] = v;
  else if (dtype == KASHIN_F16) static_cast<_Float16*>(y)[i] = static_cast<_Float16>(v);
  else static_cast<__bf16*>(y)[i] = static_cast<__bf16>(v);
}

// ------------------------------------------------------------------ operands of the matrix instructions
// Products run on fp16 matrix instructions with fp32 sums.  fp32 operands are two fp16 parts, hi + lo, which hold 22
// bits: x y = hi hi + hi lo + lo hi to 2^-21.  Both operands are scaled by powers of two first, a row of x with P x and a
// matrix row's centres each by its largest magnitude, into fp16's range.
using uint4_t = uint32_t __attribute__((ext_vector_type(4)));

constexpr int kRowsT = 512;

// Exponent s that takes a largest magnitude (as bits) into [2^13, 2^14) when multiplied by 2^s; NaN or infinity: none.
__device__ __forceinline__ int scale_exponent(uint32_t top) {
  const int e = 267 - static_cast<int>(top >> 23);
  return (e > 253 ? 253 : e) - 127;
}
__device__ __forceinline__ float power_of_two(int s) { return __uint_as_float(static_cast<uint32_t>(s + 127) << 23); }
constexpr uint32_t kInfBits = 0x7f800000u;

// The four centres of a factor as fp16 hi and lo parts, split into their low and high bytes: an entry of a table of
// four 16-bit values is two byte selections.
struct Table {
  uint32_t hi0, hi1, lo0, lo1;
};
__device__ __forceinline__ uint32_t pair_bits(_Float16 a, _Float16 b) {
  return static_cast<uint32_t>(__builtin_bit_cast(uint16_t, a)) |
         (static_cast<uint32_t>(__builtin_bit_cast(uint16_t, b)) << 16);
}
__device__ __forceinline__ Table make_table(float4_t q, float scale) {
  _Float16 h[4], l[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float v = q[c] * scale;
    h[c] = static_cast<_Float16>(v);
    l[c] = static_cast<_Float16>(v - static_cast<float>(h[c]));
  }
  const uint32_t a = pair_bits(h[0], h[1]), b = pair_bits(h[2], h[3]), c = pair_bits(l[0], l[1]), d = pair_bits(l[2], l[3]);
  return {__builtin_amdgcn_perm(b, a, 0x06040200u), __builtin_amdgcn_perm(b, a, 0x07050301u),
          __builtin_amdgcn_perm(d, c, 0x06040200u), __builtin_amdgcn_perm(d, c, 0x07050301u)};
}

// Eight values of unit `h` (0, 1) of a dword of 16 codes, hi and (LO) lo parts.
template <bool LO>
__device__ __forceinline__ void decode8(uint32_t w, int h, const Table& tb, half8& hi, half8& lo) {
  uint4_t a, b;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t c = (w >> (4 * h + 2 * k)) & 0x03030303u;
    uint32_t l = __builtin_amdgcn_perm(0, tb.hi0, c), u = __builtin_amdgcn_perm(0, tb.hi1, c);
    a[2 * k] = __builtin_amdgcn_perm(u, l, 0x05010400u);
    a[2 * k + 1] = __builtin_amdgcn_perm(u, l, 0x07030602u);
    if constexpr (LO) {
      l = __builtin_amdgcn_perm(0, tb.lo0, c);
      u = __builtin_amdgcn_perm(0, tb.lo1, c);
      b[2 * k] = __builtin_amdgcn_perm(u, l, 0x05010400u);
      b[2 * k + 1] = __builtin_amdgcn_perm(u, l, 0x07030602u);
    }
  }
  hi = __builtin_bit_cast(half8, a);
  if constexpr (LO) lo = __builtin_bit_cast(half8, b);
}

// A chunk's 16 bytes of codes.  The last chunk of a group may be short (n no multiple of 64): then the group's
// last 16 bytes are read (n >= 64) and moved down; what follows its codes meets zeros of x.
__device__ __forceinline__ uint4_t load_codes(const uint8_t* group, int nby, int off) {
  const int left = nby - off;
  uint4_t v;
  if (left >= 16) {
    __builtin_memcpy(&v, group + off, 16);
    return v;
  }
  uint64_t q[2];
  __builtin_memcpy(q, group + nby - 16, 16);
  const int bits = 8 * (16 - left);  // 8 .. 120
  if (bits >= 64) {
    q[0] = q[1] >> (bits - 64);
    q[1] = 0;
  } else {
    q[0] = (q[0] >> bits) | (q[1] << (64 - bits));
    q[1] >>= bits;
  }
  __builtin_memcpy(&v, q, 16);
  return v;
}

// ------------------------------------------------------------------ x W^T: x and P x as operands
// For rows of many groups (kashin_layer_impl.h writes the operands of others).  A workgroup takes ROWS rows (8: the lanes
// of eight rows write 128 consecutive bytes; 2 below kManyRows, to spread them over the chip: 4096 matrix rows, 16 groups of
// 256, 128 rows of x 43.8 -> 33.9 us, 1024 rows 172.7 -> 167.7, 1536 rows 186.4 -> 187.8), a thread 16 entries of a row at a
// time: two units.
constexpr int kSplitT = 512;
constexpr int kManyRows = 1536;
template <int ROWS>
__global__ __launch_bounds__(kSplitT) void split_rows_kernel(XRows x, const float* px, int n, int groups, int64_t t, int parts,
                                                             _Float16* frags, int32_t* exps) {
  __shared__ uint32_t tops[ROWS];
  const int tid = threadIdx.x, mine = tid % ROWS;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + mine, k = static_cast<int64_t>(groups) * n;
  const bool real = row < t;
  const XRows src[2] = {x, {px, k, KASHIN_F32}};
  const int per_group = chunks_per_group(n) * (kChunk / 16);
  const int64_t blocks = padded_chunks(n, groups) * (kChunk / 16), used = static_cast<int64_t>(groups) * per_group;
  auto load16 = [&](int f, int64_t b, float (&v)[16]) {  // block b of a factor, zeros past its group
    int left = 0;
    int64_t at = 0;
    if (real && b < used) {
      const int64_t g = b / per_group;
      const int in_group = static_cast<int>(b - g * per_group) * 16;
      at = row * src[f].ld + g * n + in_group;
      left = n - in_group;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float u[8];
      load_row8(src[f], at + 8 * h, left - 8 * h, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[8 * h + j] = u[j];
    }
  };
  if (tid < ROWS) tops[tid] = 0;
  __syncthreads();
  uint32_t top = 0;
  for (int64_t b = tid / ROWS; b < 2 * used; b += kSplitT / ROWS) {
    float v[16];
    if (b < used) load16(0, b, v);
    else load16(1, b - used, v);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const uint32_t o = __float_as_uint(v[j]) & 0x7fffffffu;
      top = o > top ? o : top;
    }
  }
#pragma unroll
  for (int d = ROWS; d < 64; d <<= 1) {
    const uint32_t o = __shfl_xor(top, d);
    top = o > top ? o : top;
  }
  if (tid % 64 < ROWS) atomicMax(&tops[mine], top);  // a maximum: the same in any order
  __syncthreads();
  top = tops[mine];
  const bool bad = top >= kInfBits;
  const int e = bad ? 0 : scale_exponent(top);
  const float scale = bad ? __int_as_float(0x7fc00000) : power_of_two(e);
  if (tid < ROWS && real) exps[row] = e;
  if (!real) return;
  for (int64_t b = tid / ROWS; b < 2 * blocks; b += kSplitT / ROWS) {
    float v[16];
    if (b < blocks) load16(0, b, v);
    else load16(1, b - blocks, v);
    put_units(frags, b, parts, t, row, v, scale);
  }
}

// y = x W^T for few rows of x: a workgroup computes 16 R matrix rows for a tile of rows of x, its eight waves taking an
// eighth of the codes each and their sums joined through LDS in a fixed order.  Operand A: lane (r, q) decodes chunk
// 4 s + q of matrix row r, operand B: the same chunk's entries of x's rows.  J tiles of 16 rows of x, or J = 0: 8
// rows, whose hi parts are B's columns 0 .. 7 and lo parts columns 8 .. 15, so that two instructions give all four products
// (against three for 16 rows).  LO: both operands in two parts; without it (J > 0) in one.  ALIGNED: n is a multiple of 256, so
// that a slab lies in one group and no chunk is short: addresses and branches are scalar then.
// One row of x, 11008 x 4096: 22.5 MB of codes in 12.0 us (1.9 TB/s; 4.4 us at the rate of a copy).  No unit is full: the
// vector ALU issues in 44 % of the cycles (mostly the decoding: four byte selections for eight values), the matrix units work in
// 11 %; the rest is waiting for codes and for what a launch of eight waves a workgroup needs first and last, the
// centres' scale and the joining of the waves' sums.
template <int J>
constexpr int tile_rows() { return J == 0 ? 8 : 16 * J; }

template <int J, int R, bool LO, bool ALIGNED>
__global__ __launch_bounds__(kRowsT, 2) void rows_kernel(ProductArgs a, const _Float16* frags, const int32_t* exps) {
  constexpr int TT = tile_rows<J>(), JJ = J == 0 ? 1 : J, NW = kRowsT / 64, RP = 16 * R + 4;
  constexpr int PARTS = J != 0 && LO ? 2 : 1;    // operands B for a unit and tile
  constexpr int STORED = LO ? 2 : 1;             // parts in frags
  constexpr int PF = JJ * PARTS <= 2 ? 4 : JJ * PARTS <= 4 ? 2 : 1;  // units whose x is loaded ahead: 16 .. 32 registers
  __shared__ float sums[NW][16 * JJ][RP];
  __shared__ uint32_t tops[16 * R];
  const Tile tl = find_tile<TT>(a.offsets, a.experts, a.t, blockIdx.y);
  if (tl.rows == 0) return;
  const int n = a.n, nby = n / 4, tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64);
  const int r = lane % 16, q = lane / 16, cpg = chunks_per_group(n), groups = a.groups;
  const int chunks = groups * cpg;
  const int slabs = static_cast<int>(padded_chunks(n, groups) / kSlab), per_group = slabs / groups;  // per_group: ALIGNED
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * (16 * R), matrix0 = (tl.expert * a.m + row0) * groups;
  // this lane's matrix rows (past the last repeat it), as offsets from the workgroup's first
  uint32_t crow[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t left = a.m - 1 - row0;
    crow[i] = static_cast<uint32_t>((16 * i + r < left ? 16 * i + r : left) * groups);
  }
  const uint8_t* cu = a.codes_u + matrix0 * nby;
  const uint8_t* cv = a.codes_v + matrix0 * nby;
  const float* ce = a.centers + matrix0 * 8;
  // this wave's items: item = factor * slabs + slab
  const int items = 2 * slabs, i0 = items * wave / NW, i1 = items * (wave + 1) / NW;
  constexpr int AHEAD = 3;
  uint4_t codes[AHEAD][R];
  auto load_item = [&](int it, uint4_t (&c)[R]) {
    const int f = it >= slabs, slab = it - f * slabs;
    const uint8_t* base = f ? cv : cu;
    if constexpr (ALIGNED) {
      base += slab * 64;
#pragma unroll
      for (int i = 0; i < R; ++i)
        __builtin_memcpy(&c[i], base + static_cast<uint32_t>(crow[i] * static_cast<uint32_t>(nby) + 16 * q), 16);
    } else {
      const int chunk = slab * kSlab + q, at = chunk < chunks ? chunk : chunks - 1, g = at / cpg;
#pragma unroll
      for (int i = 0; i < R; ++i)
        c[i] = load_codes(base + static_cast<uint32_t>((crow[i] + g) * static_cast<uint32_t>(nby)), nby, (at - g * cpg) * 16);
    }
  };
#pragma unroll
  for (int d = 0; d < AHEAD; ++d)
    if (i0 + d < i1) load_item(i0 + d, codes[d]);
  // B: column c of tile j is row 16 j + c of the tile (J = 0: row c % 8, hi or lo part); columns past the last repeat it
  const uint32_t t = static_cast<uint32_t>(a.t);
  uint32_t col[JJ];
#pragma unroll
  for (int j = 0; j < JJ; ++j) {
    int c = J == 0 ? r % 8 : 16 * j + r;
    c = c < tl.rows ? c : tl.rows - 1;
    col[j] = (q * kUnits * STORED * t + (J == 0 && r >= 8 ? t : 0) + c) * 16;
  }
  const char* x0 = reinterpret_cast<const char*>(frags + tl.row0 * 8);
  half8 ahead[PF][JJ][PARTS];
  auto load_x = [&](int it, int s0) {
    // a buffer of its own for each item: the lanes' 32-bit offsets stay in registers, the units' are scalars
    const auto units = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(x0) + static_cast<int64_t>(it) * (kSlab * kUnits) * STORED * t * 16, 0, -1, 0x00027000);
#pragma unroll
    for (int s = 0; s < PF; ++s)
#pragma unroll
      for (int j = 0; j < JJ; ++j)
#pragma unroll
        for (int pt = 0; pt < PARTS; ++pt)
          ahead[s][j][pt] = __builtin_bit_cast(
              half8, __builtin_amdgcn_raw_buffer_load_b128(units, col[j], ((s0 + s) * STORED + pt) * t * 16, 0));
  };
  if (i0 < i1) load_x(i0, 0);
  // the scale of every matrix row: its largest centre over all groups.  With one group a lane holds its rows' centres
  // from the start, and nothing waits for the other waves.
  float scale[R];
  constexpr bool OWN = R == 1;  // where registers allow
  float4_t own[R][2];
  if (OWN && groups == 1) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      uint32_t top = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        own[i][h] = *reinterpret_cast<const float4_t*>(ce + 4 * h + static_cast<uint32_t>(crow[i] * 8));
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t b = __float_as_uint(own[i][h][c]) & 0x7fffffffu;
          top = b > top ? b : top;
        }
      }
      scale[i] = top >= kInfBits ? __int_as_float(0x7fc00000) : power_of_two(scale_exponent(top));
      if (wave == 0 && q == 0) tops[16 * i + r] = top;  // for the sums, behind a barrier
    }
  } else {
    if (tid < 16 * R) tops[tid] = 0;
    __syncthreads();
    uint32_t top = 0;
    const int mine = tid % (16 * R);
    const int64_t left = a.m - 1 - row0;
    const float* mc = ce + static_cast<uint32_t>((mine < left ? mine : left) * groups) * 8u;
    for (int j = tid / (16 * R); j < groups * 2; j += kRowsT / (16 * R)) {
      const float4_t v = *reinterpret_cast<const float4_t*>(mc + 4 * j);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t b = __float_as_uint(v[c]) & 0x7fffffffu;
        top = b > top ? b : top;
      }
    }
    if (top) atomicMax(&tops[mine], top);  // a maximum: the same in any order
    __syncthreads();
#pragma unroll
    for (int i = 0; i < R; ++i) {
      top = tops[16 * i + r];
      scale[i] = top >= kInfBits ? __int_as_float(0x7fc00000) : power_of_two(scale_exponent(top));
    }
  }
  // this thread's first sum's exponent of x, loaded early
  const int xexp = exps[tl.row0 + (tid / (16 * R) < tl.rows ? tid / (16 * R) : 0)];
  float4_t acc[JJ][R];
#pragma unroll
  for (int j = 0; j < JJ; ++j)
#pragma unroll
    for (int i = 0; i < R; ++i) acc[j][i] = float4_t{0.f, 0.f, 0.f, 0.f};
  Table tb[R];
  int held = -1;  // the (factor, group) whose tables tb holds
  for (int b0 = i0; b0 < i1; b0 += AHEAD) {
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) {
      const int it = b0 + d;
      if (it >= i1) break;
      const int f = it >= slabs, slab = it - f * slabs;
      int g;
      if constexpr (ALIGNED) {
        g = groups == 1 ? 0 : slab / per_group;
      } else {
        const int chunk = slab * kSlab + q;
        g = (chunk < chunks ? chunk : chunks - 1) / cpg;
      }
      if (f * groups + g != held) {
        held = f * groups + g;
#pragma unroll
        for (int i = 0; i < R; ++i) {
          if (OWN && groups == 1) tb[i] = make_table(f ? own[i][1] : own[i][0], scale[i]);
          else tb[i] = make_table(*reinterpret_cast<const float4_t*>(ce + 8 * g + 4 * f + static_cast<uint32_t>(crow[i] * 8)), scale[i]);
        }
      }
      uint4_t now[R];
#pragma unroll
      for (int i = 0; i < R; ++i) now[i] = codes[d][i];
      if (it + AHEAD < i1) load_item(it + AHEAD, codes[d]);
#pragma unroll
      for (int s0 = 0; s0 < kUnits; s0 += PF) {
        half8 x[PF][JJ][PARTS];
#pragma unroll
        for (int s = 0; s < PF; ++s)
#pragma unroll
          for (int j = 0; j < JJ; ++j)
#pragma unroll
            for (int pt = 0; pt < PARTS; ++pt) x[s][j][pt] = ahead[s][j][pt];
        // the next units' rows of x, while these are multiplied
        if (s0 + PF < kUnits) load_x(it, s0 + PF);
        else if (it + 1 < i1) load_x(it + 1, 0);
#pragma unroll
        for (int s = 0; s < PF; ++s) {
          half8 hi[R], lo[R];
#pragma unroll
          for (int i = 0; i < R; ++i) decode8<LO>(now[i][(s0 + s) / 2], (s0 + s) % 2, tb[i], hi[i], lo[i]);
#pragma unroll
          for (int j = 0; j < JJ; ++j)
#pragma unroll
            for (int i = 0; i < R; ++i) {
              if constexpr (LO) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo[i], x[s][j][0], acc[j][i], 0, 0, 0);
              if constexpr (PARTS == 2)
                acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[i], x[s][j][PARTS - 1], acc[j][i], 0, 0, 0);
              acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[i], x[s][j][0], acc[j][i], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);  // loads of later units moved up here would spill
      }
    }
  }
#pragma unroll
  for (int j = 0; j < JJ; ++j)
#pragma unroll
    for (int i = 0; i < R; ++i) *reinterpret_cast<float4_t*>(&sums[wave][16 * j + r][16 * i + 4 * q]) = acc[j][i];
  __syncthreads();
  for (int o = tid; o < TT * 16 * R; o += kRowsT) {
    const int c = o / (16 * R), i = o % (16 * R);
    if (c >= tl.rows || row0 + i >= a.m) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += J == 0 ? sums[w][c][i] + sums[w][c + 8][i] : sums[w][c][i];
    const uint32_t top = tops[i];
    const int e = top >= kInfBits ? 0 : scale_exponent(top);
    put(a.y, a.y_dtype, (tl.row0 + c) * a.ldy + row0 + i, ldexpf(v, -(e + (o == tid ? xexp : exps[tl.row0 + c]))));
  }
}

// y = x W^T for many rows of x: a workgroup computes 256 matrix rows by TT rows of x in 32 x 32 tiles: 128 rows of x, wave
// (rw, cw) 64 by 64 of them, or 64, a wave 32 by 64.  The rows of x pass through LDS (128 entries of K of one factor at a
// time, two buffers, filled by loads that go to LDS directly); a wave decodes its matrix rows' codes in registers, each code
// once for 64 rows of x.
using float16_t = float __attribute__((ext_vector_type(16)));
constexpr int kTileM = 256;

// 16 bytes a lane from memory to LDS, lane by lane behind `lds`; `from` and `lds` are the same in all lanes, `off` is the lane's
// offset in bytes.  Written as an instruction: the
// compiler would let every later LDS read wait for it, also of the other buffer.  It has no register output; who reads the
// data waits with wait_loads first, then at a barrier (which alone does not wait).
__device__ __forceinline__ void load_to_lds(const void* from, uint32_t off, const void* lds) {
  const int at = uniform(static_cast<int>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)lds)));
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(from), "s"(at)
               : "memory", "m0");
}
// Until at most N of this wave's loads are under way (they arrive in order).
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// Two workgroups a unit where hi parts alone leave room for it (65 KB of LDS, 128 registers).  2048 rows of x, 11008 x 4096, bf16
// result: 369 GFLOP of [x | P x] [U | V]^T in 359 us among other calls, 1.03 PFLOP/s, 95 % of what a large fp16 product
// reaches here (after a pause 393 us, and 455 with one workgroup a unit and addresses of 64 bits for x); the matrix units work in
// 67 % of the cycles, the vector ALU issues in 55 %.  fp16 result, three products each: 865 us, 1.28 PFLOP/s.  K in groups of 10000 (no
// multiple of 256: all loads are waited for each step, one workgroup a unit), 4096 matrix rows, bf16: 394 us, 0.85 PFLOP/s.
template <int TT, bool LO, bool ALIGNED>
__global__ __launch_bounds__(512, LO || !ALIGNED ? 2 : 4) void rows_tile_kernel(ProductArgs a, const _Float16* frags, const int32_t* exps) {
  constexpr int PARTS = LO ? 2 : 1, SU = 2 * kUnits;  // units of a slab: two chunks
  constexpr int RT = TT / 64;                         // tiles of matrix rows of a wave; two of rows of x
  __shared__ __align__(16) _Float16 xs[2][PARTS][SU][TT][8];
  __shared__ uint32_t tops[kTileM];
  const Tile tl = find_tile<TT>(a.offsets, a.experts, a.t, blockIdx.y);
  if (tl.rows == 0) return;
  const int n = a.n, nby = n / 4, tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64);
  const int r = lane % 32, q = lane / 32, rw = wave / RT, cw = wave % RT, cpg = chunks_per_group(n), groups = a.groups;
  const int chunks = groups * cpg;
  const int64_t units = padded_chunks(n, groups) * kUnits;
  const int slabs = (chunks + 1) / 2, items = 2 * slabs, per_group = cpg / 2;  // per_group: ALIGNED
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kTileM, matrix0 = (tl.expert * a.m + row0) * groups;
  uint32_t crow[RT];  // this lane's matrix rows (past the last repeat it), as offsets from the workgroup's first
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int64_t left = a.m - 1 - row0;
    const int at = 32 * (RT * rw + i) + r;
    crow[i] = static_cast<uint32_t>((at < left ? at : left) * groups);
  }
  const uint8_t* cu = a.codes_u + matrix0 * nby;
  const uint8_t* cv = a.codes_v + matrix0 * nby;
  const float* ce = a.centers + matrix0 * 8;
  auto load_item = [&](int it, uint4_t (&c)[RT]) {
    const int f = it >= slabs, slab = it - f * slabs;
    const uint8_t* base = f ? cv : cu;
    if constexpr (ALIGNED) {
      base += slab * 32;
#pragma unroll
      for (int i = 0; i < RT; ++i)
        __builtin_memcpy(&c[i], base + static_cast<uint32_t>(crow[i] * static_cast<uint32_t>(nby) + 16 * q), 16);
    } else {
      const int chunk = slab * 2 + q, at = chunk < chunks ? chunk : chunks - 1, g = at / cpg;
#pragma unroll
      for (int i = 0; i < RT; ++i)
        c[i] = load_codes(base + static_cast<uint32_t>((crow[i] + g) * static_cast<uint32_t>(nby)), nby, (at - g * cpg) * 16);
    }
  };
  const int mine_x = (wave % RT) * 64 + lane;  // this lane's row of x in a load (past the last repeats it)
  const uint32_t x_off = static_cast<uint32_t>(tl.row0 + (mine_x < tl.rows ? mine_x : tl.rows - 1)) * 16u;
  auto fill = [&](int it, int buf) {  // a wave's load takes 64 rows of x of a unit
    const int f = it >= slabs;
    const int64_t u0 = f * units + static_cast<int64_t>(it - f * slabs) * SU;
#pragma unroll
    for (int pt = 0; pt < PARTS; ++pt)
#pragma unroll
      for (int k = 0; k < SU * RT / 8; ++k) {
        const int u = 8 / RT * k + wave / RT;
        load_to_lds(frags + ((u0 + u) * PARTS + pt) * a.t * 8, x_off, &xs[buf][pt][u][(wave % RT) * 64][0]);
      }
  };
  // codes are loaded two items ahead: an item takes less time than memory does
  uint4_t next[2][RT];
  load_item(0, next[0]);
  fill(0, 0);
  load_item(1, next[1]);  // items is even
  if (tid < kTileM) tops[tid] = 0;
  __syncthreads();
  {
    uint32_t top = 0;
    const int mine = tid % kTileM;
    const int64_t left = a.m - 1 - row0;
    const float* mc = ce + static_cast<uint32_t>((mine < left ? mine : left) * groups) * 8u;
    for (int j = tid / kTileM; j < groups * 2; j += 512 / kTileM) {
      const float4_t v = *reinterpret_cast<const float4_t*>(mc + 4 * j);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t b = __float_as_uint(v[k]) & 0x7fffffffu;
        top = b > top ? b : top;
      }
    }
    if (top) atomicMax(&tops[mine], top);  // a maximum: the same in any order
  }
  wait_loads<0>();
  __syncthreads();
  float scale[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const uint32_t top = tops[32 * (RT * rw + i) + r];
    scale[i] = top >= kInfBits ? __int_as_float(0x7fc00000) : power_of_two(scale_exponent(top));
  }
  float16_t acc[RT][2];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.f;
  Table tb[RT];
  int held = -1;
  for (int b0 = 0; b0 < items; b0 += 2) {
#pragma unroll
    for (int buf = 0; buf < 2; ++buf) {  // items is even
      const int it = b0 + buf, f = it >= slabs, slab = it - f * slabs;
      int g;
      if constexpr (ALIGNED) {
        g = groups == 1 ? 0 : slab / per_group;
      } else {
        const int chunk = slab * 2 + q;
        g = (chunk < chunks ? chunk : chunks - 1) / cpg;
      }
      uint4_t now[RT];
#pragma unroll
      for (int i = 0; i < RT; ++i) now[i] = next[buf][i];
      // taken before the loads to LDS are issued: the compiler counts its own loads only, and would wait for those too
#pragma unroll
      for (int i = 0; i < RT; ++i) asm volatile("" : "+v"(now[i]));
      fill(it + 1 < items ? it + 1 : it, buf ^ 1);  // past the last item: what nobody reads
      if (f * groups + g != held) {
        held = f * groups + g;
#pragma unroll
        for (int i = 0; i < RT; ++i)
          tb[i] = make_table(*reinterpret_cast<const float4_t*>(ce + 8 * g + 4 * f + static_cast<uint32_t>(crow[i] * 8)), scale[i]);
      }
      load_item(it + 2 < items ? it + 2 : items - 1, next[buf]);
      __builtin_amdgcn_sched_barrier(0);  // issued here, not behind the products
#pragma unroll
      for (int s = 0; s < kUnits; ++s) {
        half8 hi[RT], lo[RT], xh[2], xl[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          xh[j] = *reinterpret_cast<const half8*>(&xs[buf][0][q * kUnits + s][64 * cw + 32 * j + r][0]);
          if constexpr (LO) xl[j] = *reinterpret_cast<const half8*>(&xs[buf][1][q * kUnits + s][64 * cw + 32 * j + r][0]);
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) decode8<LO>(now[i][s / 2], s % 2, tb[i], hi[i], lo[i]);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if constexpr (LO) {
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lo[i], xh[j], acc[i][j], 0, 0, 0);
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi[i], xl[j], acc[i][j], 0, 0, 0);
            }
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi[i], xh[j], acc[i][j], 0, 0, 0);
          }
      }
      // x of the next item has arrived when at most the loads of codes behind it are under way
      wait_loads<ALIGNED ? RT : 0>();
      __syncthreads();
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int c = 64 * cw + 32 * j + r;
    if (c >= tl.rows) continue;
    const int ex = exps[tl.row0 + c];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int in_tile = 32 * (RT * rw + i) + 8 * b + 4 * q;
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t top = tops[in_tile + k];
          v[k] = ldexpf(acc[i][j][4 * b + k], -((top >= kInfBits ? 0 : scale_exponent(top)) + ex));
        }
        put4(a.y, a.y_dtype, (tl.row0 + c) * a.ldy + row0 + in_tile, a.m - row0 - in_tile, v);
      }
  }
}

// ------------------------------------------------------------------ x W: the columns of the codes
// y[t][c] = sum_i x[t][i] w[i][c]: the sum runs over matrix rows, whose centres differ, while a lane of operand A holds
// one column of eight rows.  A row's four centres q are therefore taken apart into functions of the code that
// A can hold without a table,
//   q[code] = a + p0 b0 + p1 b1 + d f,   b0 = {0,1,0,1}, b1 = {0,0,2,2}, f = {0,1,2,4},
//   a = q0, d = q3 - q2 - q1 + q0, p0 = q1 - q0 - d, p1 = (q2 - q0) / 2 - d,
// and the coefficients times x go into operand B (two fp16 parts).  With a code's two bits at bits 10 and 11 of a
// 16-bit half, the halves masked by 0x0400, 0x0800 and 0x0c00 are the fp16 numbers b0, b1 and f times 2^-14: two codes
// take a shift and three ands.
//
// A workgroup scales by what it meets: max |x| of a row of x into [2^6, 2^7), the largest finite centre into [2^4, 2^5), so
// that a coefficient times x stays below 1.5 * 2^14.  Both parts of it are taken whatever y's type: for up to 8 rows they cost
// nothing (hi and lo parts are columns of one operand), and 33 max|centre| |x| rounded to fp16 once would leave a bf16
// result little better than its own rounding.
// One row of x, 4096 x 4096: 8.4 MB of codes and 0.3 of centres in 10.5 us, and 3.5 us to join the splits; bound by the loads'
// latency over the steps of a workgroup, of which three are under way (vector ALU 40 % of the cycles, matrix units 14 %).
// The tiled kernel's partial maxima of the centres: of each expert's groups and factors (a key: group * 2 + factor), over this
// many slices of its matrix rows.
constexpr int kTopSlices = 16;
__host__ __device__ constexpr int top_slices(int64_t m) { return m < 512 ? static_cast<int>((m + 31) / 32) : kTopSlices; }

// The caller's rows of x.
template <class T>
struct XIn {
  const T* p;
  int64_t ld;
  const float* scales;  // e4m3
  int group, per_row;   // scales of a row
};
// Entry i of a row that starts `at` entries into p.
template <class T>
__device__ __forceinline__ float load1(const XIn<T>& x, int64_t at, int64_t row, uint32_t i) {
  float v = widen(x.p[at + i]);
  if constexpr (sizeof(T) == 1) v *= x.scales[row * x.per_row + (x.group ? i / static_cast<uint32_t>(x.group) : 0u)];
  return v;
}

// The split of a transposed product: a workgroup of `waves` waves takes as many blocks of columns of one group, over
// `rows` matrix rows (a multiple of 32), of which there are `splits` per matrix; their sums are joined afterwards.
struct ColumnsPlan {
  int tile;  // columns_tile_kernel's rows of x (a workgroup takes 256 columns of a group), or 0
  int j, waves, per_group, splits;
  int64_t rows, tiles, part_rows;
};

template <int J, class T>
__global__ __launch_bounds__(512, 2) void columns_kernel(ProductArgs a, ColumnsPlan pl, XIn<T> x, float* out) {
  constexpr int STEPS = 16;  // columns of a lane's dword
  constexpr int TT = tile_rows<J>(), JJ = J == 0 ? 1 : J, PARTS = J != 0 ? 2 : 1, CP = 16 * JJ;
  __shared__ __align__(16) _Float16 xs[2][4][PARTS][4][CP][8];  // [buffer][function][part][quarter][column of B][row]
  __shared__ uint32_t tops[TT + 1];  // of the rows of x, of the centres
  const Tile tl = find_tile<TT>(a.offsets, a.experts, a.t, blockIdx.y);
  if (tl.rows == 0) return;
  const int n = a.n, nby = n / 4, tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64), r = lane % 16, q = lane / 16;
  int id = blockIdx.x;
  const int wblk = id % pl.per_group;
  id /= pl.per_group;
  const int g = id % a.groups;
  id /= a.groups;
  const int f = id % 2, split = id / 2;
  const int block = wblk * pl.waves + wave;
  const bool busy = block * 256 < n;
  const int64_t i0 = split * pl.rows, i1 = i0 + pl.rows < a.m ? i0 + pl.rows : a.m;
  const float* ce0 = a.centers + (tl.expert * a.m * a.groups + g) * 8 + 4 * f;  // of matrix row i: 8 groups i further
  const uint8_t* codes = f ? a.codes_v : a.codes_u;
  // the lane's dword of codes; at a group's end (n no multiple of 16, or past the last column) the last four bytes
  // are read and moved down
  int off = block * 64 + 4 * r, shift = 0;
  if (off > nby - 4) {
    shift = 8 * (off - (nby - 4));
    shift = shift < 24 ? shift : 24;
    off = nby - 4;
  }
  // A step's codes through a buffer that ends with the expert's matrix (rows past the last come back as zeros): the lane's
  // offsets stay in registers, a step moves the base.
  const uint32_t stride = static_cast<uint32_t>(a.groups) * static_cast<uint32_t>(nby);  // of a matrix row
  const uint8_t* codes0 = codes + (tl.expert * a.m * a.groups + g) * static_cast<int64_t>(nby);
  uint32_t at[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) at[e] = (8 * q + e) * stride + off;
  auto load_codes8 = [&](int64_t k0, uint32_t (&w)[8]) {
    const int64_t left = a.m > k0 ? (a.m - k0) * stride - static_cast<int64_t>(g) * nby : 0;
    const auto rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(codes0) + k0 * stride, 0,
                                                        left < 0x7fffffff ? static_cast<int>(left) : 0x7fffffff, 0x00027000);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_raw_buffer_load_b32(rows, at[e], 0, 0);
  };
  // Codes, and a thread's first item of operand B, are loaded AHEAD steps ahead: a step takes less time than memory does.
  // Loads past the last matrix row take that row again.
  // Item it = (it % 16, it / 16) = (pair of matrix rows, row of x).
  constexpr int AHEAD = 3;
  struct Item {
    float x[2];
    float4_t ce[2];
  };
  const uint32_t last = static_cast<uint32_t>(a.m - 1), cstride = static_cast<uint32_t>(a.groups) * 32u;
  auto fetch = [&](int it, int64_t k0) {
    Item v;
    const int pair = it % 16, c = it / 16 < tl.rows ? it / 16 : tl.rows - 1;
    const int64_t row = (tl.row0 + c) * x.ld;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint32_t i = static_cast<uint32_t>(k0) + 2 * pair + e;
      i = i < last ? i : last;
      v.x[e] = load1(x, row, tl.row0 + c, i);
      v.ce[e] = *reinterpret_cast<const float4_t*>(reinterpret_cast<const char*>(ce0) + static_cast<uint64_t>(i) * cstride);
    }
    return v;
  };
  for (int c = tid; c <= TT; c += blockDim.x) tops[c] = 0;
  __syncthreads();
  uint32_t next[AHEAD][8];
  Item ahead[AHEAD];
#pragma unroll
  for (int e = 0; e < AHEAD; ++e) {
    load_codes8(i0 + 32 * e, next[e]);
    ahead[e] = fetch(tid, i0 + 32 * e);
  }
  {
    const int range = static_cast<int>(i1 - i0);
    uint32_t top = 0;
    for (int i = tid; i < range; i += blockDim.x) {
      const float4_t v = *reinterpret_cast<const float4_t*>(ce0 + (i0 + i) * a.groups * 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t b = __float_as_uint(v[j]) & 0x7fffffffu;
        top = b > top && b < kInfBits ? b : top;  // a row that is not finite gives NaN by itself
      }
    }
    top = wave_max(top);
    if (lane == 0) atomicMax(&tops[TT], top);  // a maximum: the same in any order
    // a wave for each row of x in turn
    for (int c = wave; c < tl.rows; c += blockDim.x / 64) {
      top = 0;
      for (int i = lane; i < range; i += 64) {
        const uint32_t b = __float_as_uint(load1(x, (tl.row0 + c) * x.ld, tl.row0 + c, static_cast<uint32_t>(i0) + i)) & 0x7fffffffu;
        top = b > top ? b : top;
      }
      top = wave_max(top);
      if (lane == 0) tops[c] = top;
    }
  }
  __syncthreads();
  const int ec = scale_exponent(tops[TT]) - 9;
  const float cscale = power_of_two(ec);
  auto store = [&](int it, const Item& v, int64_t k0, int buf) {
    const int pair = it % 16, c = it / 16;
    const uint32_t top = tops[c];
    const float xscale = top >= kInfBits ? __int_as_float(0x7fc00000) : power_of_two(scale_exponent(top) - 7);
    _Float16 h[2][4], l[2][4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float4_t ce = v.ce[e] * cscale;
      const bool real = c < tl.rows && k0 + 2 * pair + e < i1;
      const float xv = real ? v.x[e] * xscale : 0.f;
      const float d = (ce[3] - ce[2]) - (ce[1] - ce[0]);
      const float p[4] = {xv * ce[0], xv * ((ce[1] - ce[0]) - d), xv * (0.5f * (ce[2] - ce[0]) - d), xv * d};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        h[e][k] = static_cast<_Float16>(p[k]);
        l[e][k] = static_cast<_Float16>(p[k] - static_cast<float>(h[e][k]));
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      *reinterpret_cast<uint32_t*>(&xs[buf][k][0][pair / 4][c][2 * (pair % 4)]) = pair_bits(h[0][k], h[1][k]);
      if constexpr (J == 0) *reinterpret_cast<uint32_t*>(&xs[buf][k][0][pair / 4][c + 8][2 * (pair % 4)]) = pair_bits(l[0][k], l[1][k]);
      else *reinterpret_cast<uint32_t*>(&xs[buf][k][1][pair / 4][c][2 * (pair % 4)]) = pair_bits(l[0][k], l[1][k]);
    }
  };
  auto build = [&](const Item& first, int64_t k0, int buf) {
    if (tid < 16 * TT) store(tid, first, k0, buf);
    for (int it = tid + blockDim.x; it < 16 * TT; it += blockDim.x) store(it, fetch(it, k0), k0, buf);
  };

  float4_t acc[JJ][STEPS], flat[JJ];
#pragma unroll
  for (int j = 0; j < JJ; ++j) {
    flat[j] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < STEPS; ++s) acc[j][s] = float4_t{0.f, 0.f, 0.f, 0.f};
  }
  build(ahead[0], i0, 0);
  __syncthreads();
  const int steps = static_cast<int>((i1 - i0 + 31) / 32);
  for (int s0 = 0; s0 < steps; s0 += AHEAD) {
#pragma unroll
   for (int e0 = 0; e0 < AHEAD; ++e0) {
    const int st = s0 + e0, buf = st & 1;
    if (st >= steps) break;
    const int64_t k0 = i0 + static_cast<int64_t>(st) * 32;
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = next[e0][e] >> shift;
    load_codes8(k0 + 32 * AHEAD, next[e0]);
    ahead[e0] = fetch(tid, k0 + 32 * AHEAD);
    if (busy) {
      half8 b[JJ][4][PARTS];
#pragma unroll
      for (int j = 0; j < JJ; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int pt = 0; pt < PARTS; ++pt) b[j][k][pt] = *reinterpret_cast<const half8*>(&xs[buf][k][pt][q][16 * j + r][0]);
      uint4_t ones = {0x04000400u, 0x04000400u, 0x04000400u, 0x04000400u};
#pragma unroll
      for (int j = 0; j < JJ; ++j)
#pragma unroll
        for (int pt = 0; pt < PARTS; ++pt)
          flat[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, ones), b[j][0][pt], flat[j], 0, 0, 0);
      uint32_t p[2][4];  // low and high halves of the dwords, two rows side by side
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[0][e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x05040100u);
        p[1][e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x07060302u);
      }
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        uint4_t fn[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t v = p[s / 8][e];
          const int at = 2 * (s % 8);
          const uint32_t c = at <= 10 ? v << (10 - at) : v >> (at - 10);
          fn[0][e] = c & 0x04000400u;
          fn[1][e] = c & 0x08000800u;
          fn[2][e] = c & 0x0c000c00u;
        }
#pragma unroll
        for (int j = 0; j < JJ; ++j)
#pragma unroll
          for (int pt = PARTS - 1; pt >= 0; --pt)
#pragma unroll
            for (int k = 0; k < 3; ++k)
              acc[j][s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, fn[k]), b[j][k + 1][pt], acc[j][s], 0, 0, 0);
      }
    }
    build(ahead[(e0 + 1) % AHEAD], k0 + 32, buf ^ 1);  // past the last row: zeros that nobody reads
    __syncthreads();
   }
  }
  if (!busy) return;
  const int64_t k = static_cast<int64_t>(a.groups) * n;
#pragma unroll
  for (int j = 0; j < JJ; ++j) {
    const int c = J == 0 ? r : 16 * j + r;
    const bool mine = c < tl.rows;
    const int64_t row = tl.row0 + (mine ? c : 0);
    const uint32_t top = tops[mine ? c : 0];
    const int unscale = 14 - ec - (top >= kInfBits ? 0 : scale_exponent(top) - 7);
    float* o = out + ((static_cast<int64_t>(split) * 2 + f) * a.t + row) * k + static_cast<int64_t>(g) * n;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = block * 256 + (4 * q + i) * 16;
#pragma unroll
      for (int s0 = 0; s0 < STEPS; s0 += 4) {
        float4_t v;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          float z = acc[j][s0 + s][i] + flat[j][i];
          if constexpr (J == 0)  // the lo part's column
            z += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(z), 0x128, 0xf, 0xf, true));
          v[s] = ldexpf(z, unscale);
        }
        if (mine && (J != 0 || r < 8) && col + s0 < n) *reinterpret_cast<float4_t*>(o + col + s0) = v;
      }
    }
  }
}

// y = x W for many rows of x: a workgroup computes TT rows of x (128 or 64) by 256 columns of a factor over a range of
// matrix rows, wave (cw, tw) TT / 2 by 64 of them in 32 x 32 tiles, 32 matrix rows at a time.  The workgroup decodes the 32 x 256 codes once,
// a dword a thread, into LDS as fp16 rows; operand B takes them with loads that transpose (a lane wants one column of
// eight matrix rows).  A dword's codes lie in LDS in the order they come out of the tables, 0 4 8 12 1 5 9 13 ..: column
// 16 d + p / 4 + 4 (p % 4) at place p, which the stores undo.
// x comes as units of eight matrix rows: units[part][unit][row of x][8], scaled as for x W^T.
// 509 rows of x, 11008 x 4096, bf16 result, among other calls: 92 GFLOP in 115 us, 800 TFLOP/s (128-row tiles, two workgroups
// a unit; 142 us where 122 were measured with the two registers more that leave room for one).  No unit is full: matrix units 42 %
// of the cycles, LDS 43 % (a quarter of that on bank conflicts), vector ALU 48 %; what the waves wait for is each other, at the
// barrier of every step.  fp16 result, three products each: 252 us, 1.09 PFLOP/s.
constexpr int kColsM = 32, kColsN = 256, kColsLd = kColsN + 32;  // 576-byte rows: four of them on 64 banks
using short4_t = short __attribute__((ext_vector_type(4)));

__host__ __device__ inline int64_t column_units(int64_t m) { return (m + kColsM - 1) / kColsM * (kColsM / 8); }

// x as such units: a workgroup takes ROWS rows (as split_rows_kernel: 509 bf16 rows of 11008, 24.3 us with 8 and 11.7 with
// 2), and behind those workgroups each looks through a slice of an expert's matrix rows for the largest finite centre of
// up to kSplitT keys, which lie behind each other in a matrix row's centres.
template <int ROWS, class T>
__global__ __launch_bounds__(kSplitT) void split_columns_kernel(const T* x, int64_t ldx, const float* scales, int group, int64_t m,
                                                                int64_t t, int parts, const float* centers, int keys,
                                                                _Float16* units, int32_t* exps, uint32_t* tops) {
  __shared__ uint32_t top_of[kSplitT];
  const int tid = threadIdx.x, mine = tid % ROWS;
  const int64_t row_blocks = (t + ROWS - 1) / ROWS;
  top_of[tid] = 0;
  __syncthreads();
  uint32_t top = 0;
  if (blockIdx.x >= row_blocks) {
    const int slices = top_slices(m), key_blocks = (keys + kSplitT - 1) / kSplitT;
    int64_t id = blockIdx.x - row_blocks;
    const int first = static_cast<int>(id % key_blocks) * kSplitT, here = keys - first < kSplitT ? keys - first : kSplitT;
    id /= key_blocks;
    const int64_t e = id / slices, slice = id % slices;
    const int rows = kSplitT / here, key = tid % here;  // matrix rows side by side; threads past the last whole one idle
    if (tid < rows * here) {
      const float* ce = centers + (e * m * keys + first + key) * 4;
#pragma unroll 4
      for (int64_t i = slice * rows + tid / here; i < m; i += static_cast<int64_t>(slices) * rows) {
        const float4_t v = *reinterpret_cast<const float4_t*>(ce + i * keys * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t b = __float_as_uint(v[j]) & 0x7fffffffu;
          top = b > top && b < kInfBits ? b : top;
        }
      }
    }
    const bool fold = here < 64 && (here & (here - 1)) == 0;  // 64 lanes hold whole matrix rows: no two lanes on one address
    if (fold) {
      for (int d = here; d < 64; d <<= 1) {
        const uint32_t o = __shfl_xor(top, d);
        top = o > top ? o : top;
      }
    }
    if (tid < rows * here && (!fold || tid % 64 < here)) atomicMax(&top_of[key], top);  // a maximum: the same in any order
    __syncthreads();
    if (tid < here) tops[(e * keys + first + tid) * slices + slice] = top_of[tid];
    return;
  }
  const int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + mine;
  const bool real = row < t;
  auto load_unit = [&](int64_t u, float (&v)[8]) {
    const int64_t i = 8 * u, left = m - i;
    load8(x + (real ? row * ldx + i : 0), real ? (left < 8 ? static_cast<int>(left < 0 ? 0 : left) : 8) : 0, v);
    if (scales != nullptr && real && left > 0) {
      const float s = group ? scales[row * ((m + group - 1) / group) + i / group] : scales[row];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < left ? v[j] * s : 0.f;
    }
  };
  const int64_t all = column_units(m);
  for (int64_t u = tid / ROWS; u < all; u += kSplitT / ROWS) {
    float v[8];
    load_unit(u, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t o = __float_as_uint(v[j]) & 0x7fffffffu;
      top = o > top ? o : top;
    }
  }
  if (top) atomicMax(&top_of[mine], top);
  __syncthreads();
  top = top_of[mine];
  const bool bad = top >= kInfBits;
  const int e = bad ? 0 : scale_exponent(top);
  const float scale = bad ? __int_as_float(0x7fc00000) : power_of_two(e);
  if (!real) return;
  if (tid < ROWS) exps[row] = e;
  for (int64_t u = tid / ROWS; u < all; u += kSplitT / ROWS) {
    float v[8];
    load_unit(u, v);
    half8 h, l;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float w = v[j] * scale;
      h[j] = static_cast<_Float16>(w);
      l[j] = static_cast<_Float16>(w - static_cast<float>(h[j]));
    }
    *reinterpret_cast<half8*>(units + (u * t + row) * 8) = h;
    if (parts == 2) *reinterpret_cast<half8*>(units + ((all + u) * t + row) * 8) = l;
  }
}

template <int TT, bool LO>
__global__ __launch_bounds__(512, LO ? 2 : 4) void columns_tile_kernel(ProductArgs a, ColumnsPlan pl, const _Float16* units,
                                                              const int32_t* exps, const uint32_t* tops, float* out) {
  constexpr int PARTS = LO ? 2 : 1, I = TT / 64;
  __shared__ __align__(16) _Float16 ws[2][PARTS][kColsM][kColsLd];
  __shared__ __align__(16) _Float16 xs[2][PARTS][kColsM / 8][TT][8];
  __shared__ int32_t ex[TT];
  const Tile tl = find_tile<TT>(a.offsets, a.experts, a.t, blockIdx.y);
  if (tl.rows == 0) return;
  const int n = a.n, nby = n / 4, tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64);
  const int r = lane % 32, q = lane / 32, cw = wave / 2, tw = wave % 2;
  int id = blockIdx.x;
  const int block = id % pl.per_group;
  id /= pl.per_group;
  const int g = id % a.groups;
  id /= a.groups;
  const int f = id % 2, split = id / 2;
  const int64_t i0 = split * pl.rows, i1 = i0 + pl.rows < a.m ? i0 + pl.rows : a.m;
  // scaled by the largest centre of this group and factor, so that other groups' magnitudes do not matter
  uint32_t top = 0;
  const int slices = top_slices(a.m);
  const uint32_t* key_tops = tops + ((static_cast<int64_t>(tl.expert) * a.groups + g) * 2 + f) * slices;
#pragma unroll
  for (int s = 0; s < kTopSlices; ++s) {
    const uint32_t o = key_tops[s < slices ? s : 0];
    top = o > top ? o : top;
  }
  const int ec = scale_exponent(top);
  const float cscale = power_of_two(ec);
  if (tid < TT) ex[tid] = tid < tl.rows ? exps[tl.row0 + tid] : 0;
  // this thread's dword of codes: matrix row `mine` of a step, columns 16 d ..; past a group's last byte its last four
  // are read and moved down
  const int mine = tid / 16, d = tid % 16;
  int off = block * 64 + 4 * d, shift = 0;
  if (off > nby - 4) {
    shift = 8 * (off - (nby - 4));
    shift = shift < 24 ? shift : 24;
    off = nby - 4;
  }
  const uint8_t* codes = f ? a.codes_v : a.codes_u;
  // codes and centres are loaded three steps ahead: a step takes less time than memory does
  constexpr int AHEAD = 3;
  uint32_t w[AHEAD];
  float4_t ce[AHEAD];
  auto load_codes_of = [&](int64_t k0, int at) {
    const int64_t i = k0 + mine, row = (tl.expert * a.m + (i < a.m ? i : a.m - 1)) * a.groups + g;
    __builtin_memcpy(&w[at], codes + row * nby + off, 4);
    ce[at] = *reinterpret_cast<const float4_t*>(a.centers + row * 8 + 4 * f);
  };
  auto decode = [&](int buf, uint32_t codes_of, float4_t centers_of) {
    // 0, or NaN where one of the four is not finite: then all are, whichever the codes take
    const float lost = fmaf(centers_of[0], 0.f, centers_of[1] * 0.f) + fmaf(centers_of[2], 0.f, centers_of[3] * 0.f);
    const Table tb = make_table(centers_of, cscale + lost);
    const uint32_t word = codes_of >> shift;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      half8 hi, lo;
      decode8<LO>(word, h, tb, hi, lo);
      *reinterpret_cast<half8*>(&ws[buf][0][mine][16 * d + 8 * h]) = hi;
      if constexpr (LO) *reinterpret_cast<half8*>(&ws[buf][PARTS - 1][mine][16 * d + 8 * h]) = lo;
    }
  };
  const int64_t all = column_units(a.m);
  const int mine_x = 64 * (wave % I) + lane;  // this lane's row of x in a load (past the last repeats it)
  const uint32_t x_off = static_cast<uint32_t>(tl.row0 + (mine_x < tl.rows ? mine_x : tl.rows - 1)) * 16u;
  auto fill = [&](int64_t k0, int buf) {
    constexpr int PIECES = PARTS * (kColsM / 8) * I;  // of 64 rows: a wave's load
#pragma unroll
    for (int p0 = 0; p0 < PIECES; p0 += 8) {
      const int p = p0 + wave, u = p / I % (kColsM / 8), pt = p / I / (kColsM / 8);
      if (PIECES < 8 && p >= PIECES) break;
      load_to_lds(units + (pt * all + k0 / 8 + u) * a.t * 8, x_off, &xs[buf][pt][u][64 * (wave % I)][0]);
    }
  };
  float16_t acc[I][2];
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.f;
  const int steps = static_cast<int>((i1 - i0 + kColsM - 1) / kColsM);
  fill(i0, 0);
#pragma unroll
  for (int e = 0; e < AHEAD; ++e) load_codes_of(i0 + e * kColsM, e);  // past the last row: that row again
  decode(0, w[0], ce[0]);
  wait_loads<0>();
  __syncthreads();
  // the lane's place in a transposing load: matrix row (lane / 32) 8 + lane % 16 / 4 of sixteen, four columns
  const int tr_row = (lane / 32) * 8 + (lane % 16) / 4, tr_col = 64 * cw + (lane / 16 % 2) * 16 + 4 * (lane % 4);
  for (int s0 = 0; s0 < steps; s0 += AHEAD) {
#pragma unroll
   for (int e = 0; e < AHEAD; ++e) {
    const int st = s0 + e, buf = st & 1;
    if (st >= steps) break;
    const int64_t k0 = i0 + static_cast<int64_t>(st) * kColsM;
    // the next step's codes, taken before the loads to LDS are issued: the compiler counts its own loads only, and would
    // wait for those too
    uint32_t codes_of = w[(e + 1) % AHEAD];
    float4_t centers_of = ce[(e + 1) % AHEAD];
    asm volatile("" : "+v"(codes_of), "+v"(centers_of));
    fill(st + 1 < steps ? k0 + kColsM : k0, buf ^ 1);  // past the last step: what nobody reads
    load_codes_of(k0 + AHEAD * kColsM, e);
    __builtin_amdgcn_sched_barrier(0);  // issued here, not behind the products
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      half8 x[I][PARTS], b[2][PARTS];
#pragma unroll
      for (int pt = 0; pt < PARTS; ++pt) {
#pragma unroll
        for (int i = 0; i < I; ++i)
          x[i][pt] = *reinterpret_cast<const half8*>(&xs[buf][pt][2 * ks + q][32 * (I * tw + i) + r][0]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          union {
            short4_t s[2];
            half8 h;
          } v;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            v.s[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) short4_t*)&ws[buf][pt][16 * ks + 4 * h + tr_row][tr_col + 32 * j]);
          b[j][pt] = v.h;
        }
      }
#pragma unroll
      for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if constexpr (LO) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][0], b[j][PARTS - 1], acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][PARTS - 1], b[j][0], acc[i][j], 0, 0, 0);
          }
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][0], b[j][0], acc[i][j], 0, 0, 0);
        }
    }
    decode(buf ^ 1, codes_of, centers_of);
    // x of the next step has arrived when at most the loads behind it, of codes and of centres, are under way
    wait_loads<2>();
    __syncthreads();
   }
  }
  const int64_t k = static_cast<int64_t>(a.groups) * n;
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int c = 32 * (I * tw + i) + 8 * (v / 4) + 4 * q + v % 4;
      if (c >= tl.rows) continue;
      float* o = out + ((static_cast<int64_t>(split) * 2 + f) * a.t + tl.row0 + c) * k + static_cast<int64_t>(g) * n;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int place = 64 * cw + 32 * j + r, col = block * kColsN + place / 16 * 16 + place % 16 / 4 + 4 * (place % 4);
        if (col < n) o[col] = ldexpf(acc[i][j][v], -(ec + ex[c]));
      }
    }
}

// Whether a row belongs to an expert (all do without offsets).
__device__ __forceinline__ bool covered(const int64_t* offsets, int experts, int64_t row) {
  return offsets == nullptr || (row >= offsets[0] && row < offsets[experts]);
}

// The sum of a row's parts at four columns (this factor's of part 0 at p, `stride` floats from part to part), by four
// threads a quarter of the parts each; the sum is thread `sub` 0's.
__device__ __forceinline__ float4_t sum_parts(const float* p, int64_t stride, int splits, int sub, float4_t (&lds)[4][64],
                                              int at) {
  float4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = sub; s < splits; s += 4) v += *reinterpret_cast<const float4_t*>(p + s * stride);
  lds[sub][at] = v;
  __syncthreads();
  return lds[0][at] + lds[1][at] + lds[2][at] + lds[3][at];
}

// zu and zv, each the sum of its parts (z: zu of all rows, then zv); zeros for rows that no expert has (P takes rows in
// pairs, and what lies in a row's neighbour may show in its last bits).  256 columns of one of them a workgroup.
__global__ __launch_bounds__(256) void join_kernel(ProductArgs a, int splits, const float* parts, int64_t k, float* z) {
  __shared__ float4_t lds[4][64];
  const int at = threadIdx.x % 64, sub = threadIdx.x / 64;
  const int64_t row = blockIdx.x, i = (static_cast<int64_t>(blockIdx.y) * 64 + at) * 4;
  const bool has = covered(a.offsets, a.experts, row) && i < k;
  const int64_t mine = (blockIdx.z * a.t + row) * k + (i < k ? i : 0);
  const float4_t v = sum_parts(parts + mine, 2 * a.t * k, has ? splits : 0, sub, lds, at);
  if (sub == 0 && i < k) *reinterpret_cast<float4_t*>(z + mine) = v;
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

// out = P in, t rows of `groups` vectors (of a row behind each other; rows apart only for one group)
hipError_t apply_p(const ProductArgs& a, const XRows& in, float* out, hipStream_t s) {
  KArgs p = a.p;
  p.w = in.p;
  p.dtype = in.dtype;
  p.ldw = a.groups == 1 ? in.ld : a.n;
  p.m = a.t * a.groups;
  p.y = out;
  p.ldy = a.n;
  return launch_pair(a.n, p, (p.m + 1) / 2, s);
}

hipError_t rotate(const ProductArgs& a, bool inverse, float* z, hipStream_t s) {
  return launch_rotate(a.n, a.rot_seed, inverse, z, KASHIN_F32, a.n, z, a.n, a.t * a.groups, s);
}

template <int J, int R, bool LO>
hipError_t launch_rows(const ProductArgs& a, const _Float16* frags, const int32_t* exps, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.m + 16 * R - 1) / (16 * R)),
                  static_cast<unsigned>(most_tiles(a.offsets != nullptr, a.t, a.experts, tile_rows<J>())));
  if (a.n % (kChunk * kSlab) == 0) hipLaunchKernelGGL((rows_kernel<J, R, LO, true>), grid, dim3(kRowsT), 0, s, a, frags, exps);
  else hipLaunchKernelGGL((rows_kernel<J, R, LO, false>), grid, dim3(kRowsT), 0, s, a, frags, exps);
  return hipGetLastError();
}

template <int TT, bool LO>
hipError_t launch_rows_tile(const ProductArgs& a, const _Float16* frags, const int32_t* exps, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.m + kTileM - 1) / kTileM),
                  static_cast<unsigned>(most_tiles(a.offsets != nullptr, a.t, a.experts, TT)));
  if (a.n % (kChunk * kSlab) == 0)
    hipLaunchKernelGGL((rows_tile_kernel<TT, LO, true>), grid, dim3(512), 0, s, a, frags, exps);
  else
    hipLaunchKernelGGL((rows_tile_kernel<TT, LO, false>), grid, dim3(512), 0, s, a, frags, exps);
  return hipGetLastError();
}

// Rows of x that a matrix (an expert's, on average) meets.
int64_t rows_each(int64_t t, int experts) { return t / (experts < t ? experts : t > 0 ? t : 1); }

// The number of splits goes by the sizes alone (the workspace does not know y's type); the tile by both.
ColumnsPlan plan_columns(int n, int64_t m, int groups, int64_t t, int experts, bool grouped, bool lo) {
  ColumnsPlan p;
  const int64_t each = rows_each(t, experts);
  const int blocks = (n + 255) / 256;
  for (p.waves = 8; p.waves > 1; p.waves /= 2)  // at most an eighth of the waves idle
    if (((blocks + p.waves - 1) / p.waves * p.waves - blocks) * 8 <= blocks) break;
  p.per_group = (blocks + p.waves - 1) / p.waves;
  p.j = each <= 8 ? 0 : 1;  // 8 rows of x: 36 us against 42 of the 16-row form, one row 25 and 27 (4096 x 4096, fp32)
  p.tiles = most_tiles(grouped, t, experts, p.j == 0 ? 8 : 16);
  // enough workgroups of eight waves to fill the chip twice over, of at least 64 rows each
  const int64_t fill = 512 * 8 / p.waves, one = static_cast<int64_t>(p.per_group) * groups * 2;
  const int64_t tiles = p.tiles > 0 ? p.tiles : 1, most = (m + 63) / 64;
  const int64_t want = (fill + one * tiles - 1) / (one * tiles), splits = want < most ? want : most;
  p.rows = ((m + splits - 1) / splits + 31) / 32 * 32;
  p.splits = static_cast<int>((m + p.rows - 1) / p.rows);
  // splits * t of this and of every smaller t (a workspace for t rows serves fewer): at most one split a 64 rows, and
  // tiles of at most 16 rows each want their share of `fill`
  const int64_t bound = (fill / one + 1) * 16 + t;
  p.part_rows = most * t < bound ? most * t : bound;
  // Tiles from 16 rows of x a matrix on, with hi parts alone from 8, by expert from 6, whose tiles of eight rows are partly
  // empty (us with and without: 4096 x 4096, fp32 results, 16 rows of x 45 and 59, 12 rows 44 and 39, 47 rows 50 and 83; bf16
  // results, 7 rows 33.0 and 34.5, 4 rows 31.9 and 30.2; 1024 x 1024 bf16 7 rows 22.3 and 20.2; 8 experts, 2048 x 4096: fp32
  // 16 rows each 88 and 83, 32 rows 90 and 124, bf16 7 rows 52 and 61, 5 rows 51 and 58; 64 experts, 1000 x 2048: bf16 7
  // rows 83 and 98, 5 rows 81 and 74).  Of 64 rows where 128
  // would be half empty; where experts' rows end in a tile's middle 64 also pay up to 128 rows a matrix with hi and lo parts,
  // whose products hide the codes' decoding (8 experts, 2048 x 4096, fp32 results, us with 64 and 128: 400 rows 131 and
  // 152, 700 rows 156 and 191, 1500 rows 288 and 248; bf16: 400 rows 81 and 84, 700 rows 96 and 92).
  p.tile = each < (lo ? 16 : grouped ? 6 : 8) ? 0 : (grouped ? each < (lo ? 128 : 64) : t <= 64) ? 64 : 128;
  if (p.tile) {
    p.per_group = (n + kColsN - 1) / kColsN;
    p.tiles = most_tiles(grouped, t, experts, p.tile);
    // two workgroups a compute unit, of at least 256 matrix rows each; never more than the bound above, whose tiles
    // are half of these or less and whose workgroups take 2048 columns
    const int64_t others = static_cast<int64_t>(p.per_group) * groups * 2 * p.tiles;
    const int64_t wanted = (512 + others - 1) / others, top = (m + 255) / 256, cut = wanted < top ? wanted : top;
    p.rows = ((m + cut - 1) / cut + 31) / 32 * 32;
    p.splits = static_cast<int>((m + p.rows - 1) / p.rows);
  }
  return p;
}

struct ColumnsWork {
  int64_t x, exps, tops, z, rz, parts, end;
};
ColumnsWork columns_work(const ColumnsPlan& p, int n, int64_t m, int groups, int64_t t, int experts) {
  const int64_t k = static_cast<int64_t>(groups) * n;
  ColumnsWork w;
  w.x = 0;
  w.exps = w.x + align256(t * column_units(m) * 32);  // units in two parts
  w.tops = w.exps + align256(t * 4);
  w.z = w.tops + align256(static_cast<int64_t>(experts) * groups * 2 * top_slices(m) * 4);
  w.rz = w.z + align256(2 * t * k * 4);
  w.parts = w.rz + align256(t * k * 4);
  w.end = w.parts + p.part_rows * 2 * k * 4;
  return w;
}

template <int J>
hipError_t launch_columns(const ProductArgs& a, const ColumnsPlan& p, float* parts, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(p.per_group) * a.groups * 2 * p.splits),
                  static_cast<unsigned>(p.tiles));
  auto launch = [&](auto zero) {
    using T = decltype(zero);
    const XIn<T> x = {static_cast<const T*>(a.x), a.ldx, a.x_scales, a.x_group,
                      a.x_group ? static_cast<int>((a.m + a.x_group - 1) / a.x_group) : 1};
    hipLaunchKernelGGL((columns_kernel<J, T>), grid, dim3(64 * p.waves), 0, s, a, p, x, parts);
  };
  if (a.x_dtype == KASHIN_E4M3) launch(e4m3_t());
  else with_float_type(a.x_dtype, launch);
  return hipGetLastError();
}

template <int TT, bool LO>
hipError_t launch_columns_tile(const ProductArgs& a, const ColumnsPlan& p, const _Float16* units, const int32_t* exps,
                               const uint32_t* tops, float* parts, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(p.per_group) * a.groups * 2 * p.splits),
                  static_cast<unsigned>(p.tiles));
  hipLaunchKernelGGL((columns_tile_kernel<TT, LO>), grid, dim3(512), 0, s, a, p, units, exps, tops, parts);
  return hipGetLastError();
}

hipError_t product_back(const ProductArgs& a, hipStream_t s) {
  const int64_t k = static_cast<int64_t>(a.groups) * a.n;
  const bool lo = a.y_dtype != KASHIN_BF16;  // as the rows' product
  const ColumnsPlan p = plan_columns(a.n, a.m, a.groups, a.t, a.experts, a.offsets != nullptr, lo);
  if (p.splits * a.t > p.part_rows) return hipErrorInvalidValue;  // the bound holds: never
  const ColumnsWork at = columns_work(p, a.n, a.m, a.groups, a.t, a.experts);
  int32_t* exps = reinterpret_cast<int32_t*>(a.work + at.exps);
  uint32_t* tops = reinterpret_cast<uint32_t*>(a.work + at.tops);
  float* z = reinterpret_cast<float*>(a.work + at.z);
  float* rz = reinterpret_cast<float*>(a.work + at.rz);
  float* parts = reinterpret_cast<float*>(a.work + at.parts);
  _Float16* units = reinterpret_cast<_Float16*>(a.work + at.x);
  const int keys = a.groups * 2;
  const int64_t slices = static_cast<int64_t>(a.experts) * top_slices(a.m) * ((keys + kSplitT - 1) / kSplitT);
  hipError_t e = hipSuccess;
  if (p.tile) {
    auto split = [&](auto zero) {
      using T = decltype(zero);
      auto launch = [&](auto rows) {
        constexpr int ROWS = decltype(rows)::value;
        hipLaunchKernelGGL((split_columns_kernel<ROWS, T>), dim3(static_cast<unsigned>((a.t + ROWS - 1) / ROWS + slices)),
                           dim3(kSplitT), 0, s, static_cast<const T*>(a.x), a.ldx, a.x_scales, a.x_group, a.m, a.t, lo ? 2 : 1,
                           a.centers, keys, units, exps, tops);
      };
      if (a.t < kManyRows) launch(std::integral_constant<int, 2>());
      else launch(std::integral_constant<int, 8>());
      return hipGetLastError();
    };
    e = a.x_dtype == KASHIN_E4M3 ? split(e4m3_t()) : with_float_type(a.x_dtype, split);
    if (e != hipSuccess) return e;
    e = p.tile == 64 ? (lo ? launch_columns_tile<64, true>(a, p, units, exps, tops, parts, s)
                           : launch_columns_tile<64, false>(a, p, units, exps, tops, parts, s))
                     : (lo ? launch_columns_tile<128, true>(a, p, units, exps, tops, parts, s)
                           : launch_columns_tile<128, false>(a, p, units, exps, tops, parts, s));
  } else {
    e = p.j == 0 ? launch_columns<0>(a, p, parts, s) : launch_columns<1>(a, p, parts, s);
  }
  if (e != hipSuccess) return e;
  const unsigned rows = static_cast<unsigned>(a.t), strips = static_cast<unsigned>((k + 255) / 256);
  const float* sums = parts;  // one part of each is its sum
  if (p.splits > 1 || a.offsets != nullptr) {
    hipLaunchKernelGGL(join_kernel, dim3(rows, strips, 2), dim3(256), 0, s, a, p.splits, parts, k, z);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    sums = z;
  }
  LayerBackArgs back = {a.p.tw, a.p.mid4, a.t, a.groups, sums, sums + a.t * k, a.offsets, a.experts, a.y, a.y_dtype, a.ldy};
  if (a.rot) {  // fp32 rows of all, which R^T follows
    back.offsets = nullptr;
    back.y = rz;
    back.y_dtype = KASHIN_F32;
    back.ldy = k;
  }
  e = launch_layer_back(a.n, back, s);
  if (e != hipSuccess || !a.rot) return e;
  e = rotate(a, true, rz, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(narrow_kernel, dim3(rows, strips), dim3(256), 0, s, a, rz, k);
  return hipGetLastError();
}

// The product itself, by the rows that a matrix meets.
hipError_t launch_product_rows(const ProductArgs& a, const _Float16* frags, const int32_t* exps, int64_t each, bool lo,
                               hipStream_t s) {
  // 4096 x 4096, fp32: 8 rows of x 21.2 us against 22.3 of the 16-row form
  if (each <= 8 && lo) return launch_rows<0, 1, true>(a, frags, exps, s);
  // Few workgroups: smaller tiles.  16 x 16 up to 384 workgroups of them, 32 x 32 up to 256 (k = 4096, fp16 results, us with
  // 16 x 16, 32 x 32 and 32 x 64: m = 72 with 300 rows of x, 95 workgroups, 29 36 46; with 1255, 395, 87 75 82; with 4000, 375 of
  // 32 x 32, 238 206 204; m = 2000 with 40 rows, 375, 26 29 36; with 100, 875 and 252, 44 36 42).
  const int64_t small = (a.m + 15) / 16 * ((a.t + 15) / 16), middle = (a.m + 31) / 32 * ((a.t + 31) / 32);
  if (each <= 16 || small <= 384) return lo ? launch_rows<1, 1, true>(a, frags, exps, s) : launch_rows<1, 1, false>(a, frags, exps, s);
  // Enough tiles of 256 x 128, or 256 x 64, to fill half the chip; the whole chip up to 48 rows of x a matrix, which leave
  // much of a tile empty.  Experts' rows end inside a tile, so theirs are of 64 rows up to 192 a matrix (bf16 results, us with these
  // tiles and with the next smaller: 32 experts, 2048 x 4096, 256 tiles: 30 rows each 94 and 138, 18 rows 90 and 103;
  // 8 experts, 4096 x 4096, 128 tiles: 60 rows each 83 and 109, 40 rows 81 and 75; 64 and 128 rows: 32 experts, 130 rows each
  // 246 and 278, 190 rows 351 and 354).
  const int64_t row_tiles = (a.m + kTileM - 1) / kTileM;
  const bool grouped = a.offsets != nullptr;
  const int64_t tiles = grouped ? a.t / each * ((each + 63) / 64) : a.t / 64;
  if (each >= (grouped ? 192 : 96) && row_tiles * (a.t / 128) >= 128)
    return lo ? launch_rows_tile<128, true>(a, frags, exps, s) : launch_rows_tile<128, false>(a, frags, exps, s);
  if (row_tiles * tiles >= (each > 48 ? 128 : 256))
    return lo ? launch_rows_tile<64, true>(a, frags, exps, s) : launch_rows_tile<64, false>(a, frags, exps, s);
  if (each <= 32 || middle <= 256)
    return lo ? launch_rows<2, 2, true>(a, frags, exps, s) : launch_rows<2, 2, false>(a, frags, exps, s);
  return lo ? launch_rows<4, 2, true>(a, frags, exps, s) : launch_rows<4, 2, false>(a, frags, exps, s);
}

// Whether P's kernel writes the operands itself: one launch and no P x in memory (4096 x 4096, bf16, 16 rows of x 22.9 -> 19.5
// us against a pass of its own over x and P x, 2048 rows 198 -> 178; 64 experts 1000 x 2048, 4000 rows 119 -> 102).  Where a
// row has several groups each pair of them looks for the row's largest entry: up to 2^28 entries looked at in all (4096
// matrix rows; 16 groups of 256: one row of x 18.0 -> 13.8 us, 1000 rows 125 -> 122; 64 groups of 256: 100 rows, 2^27, 84 -> 76,
// 1000 rows, 2^30, 453 -> 478).
bool direct_operands(int n, int groups, int64_t t) { return groups == 1 || t * groups * groups * n <= int64_t(1) << 28; }

struct RowsWork {
  int64_t wide, px, exps, frags, end;  // px: only where P x passes through memory
};
RowsWork rows_work(int n, int groups, int64_t t) {
  const int64_t rows = align256(t * groups * n * 4);
  RowsWork w;
  w.wide = 0;
  w.px = w.wide + rows;
  w.exps = w.px + (direct_operands(n, groups, t) ? 0 : rows);
  w.frags = w.exps + align256(t * 4);
  w.end = w.frags + 4 * padded_chunks(n, groups) * kUnits * t * 16;
  return w;
}

}  // namespace

int64_t product_workspace_bytes(int n, int64_t m, int groups, int64_t t, int experts, bool back) {
  if (t == 0) return 0;
  if (back) return columns_work(plan_columns(n, m, groups, t, experts, experts > 1, true), n, m, groups, t, experts).end;
  return rows_work(n, groups, t).end;
}

hipError_t launch_product(const ProductArgs& a, hipStream_t s) {
  if (a.back) return product_back(a, s);
  const int64_t k = static_cast<int64_t>(a.groups) * a.n;
  const RowsWork at = rows_work(a.n, a.groups, a.t);
  float* wide = reinterpret_cast<float*>(a.work + at.wide);
  float* px = reinterpret_cast<float*>(a.work + at.px);
  int32_t* exps = reinterpret_cast<int32_t*>(a.work + at.exps);
  _Float16* frags = reinterpret_cast<_Float16*>(a.work + at.frags);
  // bf16 results are rounded by up to 2^-8 each; operands rounded to fp16 (2^-11 each) add little to that
  const int64_t each = rows_each(a.t, a.experts);
  const bool lo = a.y_dtype != KASHIN_BF16;
  const int parts = lo ? 2 : 1;
  const bool direct = direct_operands(a.n, a.groups, a.t);
  // the caller's rows where the next kernel can read them, else fp32 ones
  XRows x = {a.x, a.ldx, a.x_dtype};
  hipError_t e = hipSuccess;
  if ((a.rot || !direct) && (a.x_dtype == KASHIN_E4M3 || (a.groups > 1 && a.ldx != k))) {
    e = widen(a, k, wide, s);
    x = {wide, k, KASHIN_F32};
  }
  if (e == hipSuccess && a.rot) {
    // rows of one group may lie apart, groups of a row lie behind each other
    e = launch_rotate(a.n, a.rot_seed, false, x.p, x.dtype, a.groups == 1 ? x.ld : a.n, wide, a.n, a.t * a.groups, s);
    x = {wide, k, KASHIN_F32};
  }
  if (e != hipSuccess) return e;
  if (direct) {
    const LayerArgs l = {a.p.tw, a.p.mid4, a.t, a.groups, x.p, x.dtype, x.ld, a.x_scales, a.x_group, frags, exps, parts};
    e = launch_layer(a.n, l, s);
    return e != hipSuccess ? e : launch_product_rows(a, frags, exps, each, lo, s);
  }
  e = apply_p(a, x, px, s);
  if (e != hipSuccess) return e;

  if (a.t >= kManyRows)
    hipLaunchKernelGGL((split_rows_kernel<8>), dim3(static_cast<unsigned>((a.t + 7) / 8)), dim3(kSplitT), 0, s, x, px, a.n,
                       a.groups, a.t, parts, frags, exps);
  else
    hipLaunchKernelGGL((split_rows_kernel<2>), dim3(static_cast<unsigned>((a.t + 1) / 2)), dim3(kSplitT), 0, s, x, px, a.n,
                       a.groups, a.t, parts, frags, exps);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_product_rows(a, frags, exps, each, lo, s);
}

}  // namespace kashin
