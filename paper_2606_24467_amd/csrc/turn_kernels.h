// New tokens' rows: rotated by their positions, and written out or into the pages of a
// cache.
//
//   pair (x0, x1) of a token at position m  ->  (x0 c - x1 s, x1 c + x0 s),
//   c, s = amplitude cos, sin (2 pi (m t mod 1)),  t the pair's turns per position
//
// t is a 64-bit fraction, so that m t modulo one turn is the low word of an integer
// product, exact at every position.  Its nearest quarter turn is taken off, and the rest, at
// most pi / 4, goes through the Taylor series of sine and cosine in fp64 (to x^15 and x^16,
// which leaves 2^-54).
//
// Bound by memory: each row is read and written once, and a token's cosines and sines are computed by
// the lanes of its wave, so that no table of them is read.  32768 tokens of 32 + 8 heads of 128 bf16
// values: 128 us, 671 MB at 5.2 TB/s (a large read reaches 5.8); 64 tokens: 4.0 us, a launch; 5001
// tokens of 8 + 2 heads of 64 fp32 values: 8.3 us, 26 MB at 3.1 TB/s, the start and the angles'
// chain; 2048 tokens of 32 + 8 heads into bf16 pages 12.9 us, into fp32 ones 18.7, fp32 rows into 8-bit ones
// 19.8.  (In the form for 8-bit pages the first rows were loaded before the angles too: more registers, 4931
// tokens in and read back 69 -> 79 us.  The other forms were not measured so.)
#pragma once

#include <type_traits>

#include "paged_device.h"

namespace ckv {

struct TurnArgs {
  const char *q, *k, *v;         // input rows (v: pages only)
  char *q_out, *k_out;           // (k_out: without pages)
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;   // byte strides
  int64_t qo_tok, qo_head, ko_tok, ko_head;
  const int32_t *pos;            // [tokens] (without pages)
  const int32_t *cu_q;           // pages: the chunk
  const uint64_t *turns;         // NULL: no rotation
  PagedView c;
  int32_t Hq, Hk, tokens;
  int32_t rotary_dim, pairs, transposed;
  float amplitude;
  int32_t share;                 // waves per token: 1 or 4
};

// Cosine and sine of a part of a turn.
__device__ __forceinline__ void turn_of(uint64_t part, double &c, double &s) {
  const uint64_t quarter = (part + (1ull << 61)) >> 62;            // 0 .. 3, and 0 again past the top
  const double x = (double)(int64_t)(part - (quarter << 62)) * (0x1.921fb54442d18p+2 * 0x1p-64);
  const double y = x * x;
  double a = 0x1p0, b = 0x1p0;                                     // sin x / x, cos x
  constexpr double kSin[] = {-1. / 210, -1. / 156, -1. / 110, -1. / 72, -1. / 42, -1. / 20, -1. / 6};
  constexpr double kCos[] = {-1. / 240, -1. / 182, -1. / 132, -1. / 90, -1. / 56, -1. / 30, -1. / 12, -1. / 2};
#pragma unroll
  for (int i = 0; i < 7; ++i) a = __builtin_fma(y * kSin[i], a, 1.);
#pragma unroll
  for (int i = 0; i < 8; ++i) b = __builtin_fma(y * kCos[i], b, 1.);
  a *= x;
  c = quarter & 1 ? a : b;
  s = quarter & 1 ? b : a;
  c = quarter == 1 || quarter == 2 ? -c : c;
  s = quarter >= 2 ? -s : s;
}

// x in fp32 with the last bit set where it is not exact: rounding that to fewer bits is then
// rounding x.
__device__ __forceinline__ float to_odd(double x) {
  const float f = (float)x;
  if ((double)f == x) return f;
  uint32_t u = __float_as_uint(f);
  if (fabs((double)f) > fabs(x)) u -= 1;         // towards zero, from an infinity too
  return __uint_as_float(u | 1u);
}

// Eight consecutive values of a row: as they lie there, and in fp32.
template <typename T>
struct RowRun {
  uint4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ RowRun<T> load_run(gptr<const char> p) {
  RowRun<T> r;
  r.w[0] = load16(p);
  if constexpr (sizeof(T) == 4) r.w[sizeof(T) / 2 - 1] = load16(p + 16);
  return r;
}
template <typename T>
__device__ __forceinline__ void values_of(const RowRun<T> &r, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    const f32x4 a = __builtin_bit_cast(f32x4, r.w[0]), b = __builtin_bit_cast(f32x4, r.w[sizeof(T) / 2 - 1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  } else {
    const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}

template <typename T>
__device__ __forceinline__ void store_values(gptr<char> p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    store16(p, __builtin_bit_cast(uint4, f32x4{x[0], x[1], x[2], x[3]}));
    store16(p + 16, __builtin_bit_cast(uint4, f32x4{x[4], x[5], x[6], x[7]}));
  } else {
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)x[i];
    store16(p, __builtin_bit_cast(uint4, r));
  }
}

// A row's run of eight values turned.  x: the run, p: the values that it turns with (the layout
// in halves: those half a rotation's dimensions away; the first half of a pair where
// `first`), or in pairs x alone.
template <typename W, bool WIDE>
__device__ __forceinline__ void turn8(const float (&x)[8], const float (&p)[8], const W (&c)[8], const W (&s)[8],
                                      bool pairs, bool first, float (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const W mate = pairs ? (W)x[i ^ 1] : (W)p[i];
    const bool minus = pairs ? (i & 1) == 0 : first;
    const W cc = pairs ? c[i >> 1] : c[i], ss = pairs ? s[i >> 1] : s[i];
    const W b = mate * (minus ? -ss : ss);
    if constexpr (WIDE) y[i] = to_odd(__builtin_fma((W)x[i], cc, b));
    else y[i] = __builtin_fmaf(x[i], cc, b);
  }
}

// Grid (tokens or a fourth of them), 256 threads: a wave per token, or all four for one
// token where there are few (`share`).  The wave's lanes compute the token's cosines and sines
// once, for all heads; then D / 8 lanes take a head, eight values each, and load
// with them the eight that they turn with.  Those lie with other lanes of the same wave, so
// that an output may be its input.  8-bit rows: a block is four lanes.
template <typename T, int D, CacheType CT, bool PAGED>
__global__ __launch_bounds__(256) void turn_kernel(const TurnArgs a) {
  constexpr bool F8 = PAGED && CT == kCacheFp8;
  constexpr int U = D / 8, HW = 64 / U;          // lanes per head, heads per wave
  // K's arithmetic.  (fp64 for fp32 rows too, which would then be rounded once: 5001 tokens of 10 heads of
  // 64 values 8.3 -> 11.0 us, 40000 37.7 -> 53.8; 110 registers instead of 78.)
  typedef std::conditional_t<F8, double, float> W;
  __shared__ W c_s[4][D / 2], s_s[4][D / 2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t_mine = a.share == 4 ? flat_block() : flat_block() * 4 + wave;
  const int t = min(t_mine, a.tokens - 1);
  const bool mine = t_mine < a.tokens;

  int pos, page = -1, slot = 0;
  if constexpr (PAGED) {
    const int b = sequence_of(a.cu_q, a.c.batch, t);
    const int most = a.c.max_pages << a.c.shift;
    pos = paged_len(a.c, b, most) - (a.cu_q[b + 1] - t);
    if (pos >= 0) {
      page = a.c.table[(int64_t)b * a.c.max_pages + (pos >> a.c.shift)];
      slot = pos & ((1 << a.c.shift) - 1);
      if ((uint32_t)page >= (uint32_t)a.c.n_pages) page = -1;
    }
  } else {
    pos = a.pos[t];
  }
  const int u = lane % U, h0 = lane / U;
  const bool turns = a.turns && 8 * u < a.rotary_dim;
  const int half = a.rotary_dim / 2;
  const bool first = 8 * u < half;
  const int mate = a.pairs || !turns ? u : first ? u + half / 8 : u - half / 8;
  W c[8] = {}, s[8] = {};
  if (a.turns) {                                 // uniform
    if (lane < half) {
      double x, y;
      turn_of((uint64_t)(int64_t)pos * a.turns[lane], x, y);
      c_s[wave][lane] = (W)(x * a.amplitude);
      s_s[wave][lane] = (W)((a.transposed ? -y : y) * a.amplitude);
    }
    __syncthreads();
    const int f0 = a.pairs ? 4 * u : 8 * u % half;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int f = min(f0 + i, half - 1);       // (in pairs four are used; of the rest none)
      c[i] = c_s[wave][f];
      s[i] = s_s[wave][f];
    }
  }
  if (!mine) return;
  float cf[8], sf[8];                            // Q's
#pragma unroll
  for (int i = 0; i < 8; ++i) cf[i] = (float)c[i], sf[i] = (float)s[i];
  const int step = HW * a.share;
  const int from = h0 + (a.share == 4 ? HW * wave : 0);

  // A row's loads are under way while the one before is turned (5000 tokens of 40 heads 22.4 -> 21.4 us,
  // 2048 into bf16 pages 14.0 -> 13.6; 4931 into 8-bit pages and back 68.3 -> 69.3).
  auto q_at = [&](int h) { return to_global(a.q) + t * a.q_tok + h * a.q_head; };
  auto kv_at = [&](int r) {
    return PAGED && r >= a.Hk ? to_global(a.v) + t * a.v_tok + (r - a.Hk) * a.v_head
                              : to_global(a.k) + t * a.k_tok + r * a.k_head;
  };
  RowRun<T> own, other;                          // the lane's values, and those that they turn with
  auto load_q = [&](int h) __attribute__((always_inline)) {
    own = load_run<T>(q_at(h) + 8 * u * sizeof(T));
    other = load_run<T>(q_at(h) + 8 * mate * sizeof(T));
  };
  if (from < a.Hq) load_q(from);
  for (int h = from; h < a.Hq; h += step) {
    float x[8], p[8], y[8];
    values_of<T>(own, x);
    values_of<T>(other, p);
    if (h + step < a.Hq) load_q(h + step);
    turn8<float, false>(x, p, cf, sf, a.pairs, first, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = turns ? y[i] : x[i];
    store_values<T>(to_global(a.q_out) + t * a.qo_tok + h * a.qo_head + 8 * u * sizeof(T), y);
  }
  // K, then (pages) V
  const int rows = PAGED ? 2 * a.Hk : a.Hk;
  auto load_kv = [&](int r) __attribute__((always_inline)) {
    own = load_run<T>(kv_at(r) + 8 * u * sizeof(T));
    other = load_run<T>(kv_at(r) + 8 * (PAGED && r >= a.Hk ? u : mate) * sizeof(T));
  };
  if (from < rows) load_kv(from);
  for (int r = from; r < rows; r += step) {
    const bool is_v = PAGED && r >= a.Hk;
    const int h = is_v ? r - a.Hk : r;
    float x[8], p[8], y[8];
    values_of<T>(own, x);
    values_of<T>(other, p);
    if (r + step < rows) load_kv(r + step);
    const bool turned = turns && !is_v;
    if (a.turns) turn8<W, F8>(x, p, c, s, a.pairs, first, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = turned ? y[i] : x[i];
    if constexpr (!PAGED) {
      store_values<T>(to_global(a.k_out) + t * a.ko_tok + h * a.ko_head + 8 * u * sizeof(T), y);
    } else {
      const int64_t row = paged_row(a.c, max(page, 0), h, slot);
      char *rows_to = is_v ? a.c.v : a.c.k;
      if constexpr (!F8) {
        if (page >= 0) store_values<T>(to_global(rows_to) + (row * D + 8 * u) * (int64_t)sizeof(T), y);
      } else {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[i]) & 0x7FFFFFFFu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2));
        const uint32_t byte = fp8_scale_byte(top);
        const uint2 codes = fp8_codes(y, byte);
        if (page >= 0) {
          *reinterpret_cast<gptr<uint64_t>>(to_global(rows_to) + row * D + 8 * u) =
              (uint64_t)codes.y << 32 | codes.x;
          if ((u & 3) == 0) to_global(is_v ? a.c.v_scale : a.c.k_scale)[row * (D / 32) + (u >> 2)] = (uint8_t)byte;
        }
      }
    }
  }
}

// Tokens up to which all four waves of a workgroup share one (4096: 2000 tokens of 40 heads 11.0 -> 11.9 us;
// 16384: 5001 fp32 tokens of 10 heads 9.0 -> 13.3 us; with one wave each 64 tokens leave most CUs idle).
constexpr int kShareTokens = 1024;

template <typename T, int D, CacheType CT, bool PAGED>
void launch_turn(TurnArgs a, hipStream_t stream) {
  a.share = a.tokens <= kShareTokens ? 4 : 1;
  const dim3 grid = flat_grid(a.share == 4 ? a.tokens : ((int64_t)a.tokens + 3) / 4);
  hipLaunchKernelGGL((turn_kernel<T, D, CT, PAGED>), grid, dim3(256), 0, stream, a);
}

}  // namespace ckv
