// Tokens drawn from the mixture readout (Sec. 4.2, Eqs. (17)-(18)) with
// temperature, top-k, top-p and min-p, from given random numbers.
//
// A token's weight is w_v = (m_v / max m)^(1/T), m = alpha p + (1 - alpha) q,
// evaluated in float64 and held as the integer W_v = rint(w_v 2^s) (2^s times the
// vocabulary fits 63 bits).  Every sum is then exact in any order, so tokens
// depend on no schedule: float32 weights are 2^-24 off each, which in a flat
// distribution of 128256 tokens (2^-17 apart in the running sum) would turn a few
// draws in a hundred.
//
// top-k, top-p and min-p all keep a run from the front of the order by falling
// weight (equal weights by index), so what stays is everything above one cut.
// The cut is found without sorting.  Every part of a row leaves a histogram of
// its mass (and number) by 254 classes of W, eight an octave; the classes in which
// the cuts can fall are known from it, and only their tokens are listed; one
// workgroup per row places the cut among them exactly.  The histograms give
// each part's mass above the cut, so the draw finds its part from those and reads
// that part alone again.
//
// Six kernels, for 64 rows of 128256 tokens with one branch and requests of every
// kind: statistics of the tiles 20 us, row constants 9 (without branches the
// weights' kernel finds the maximum itself), weights and histograms 33, cut
// classes 7, list 6, cut and draw 21 (a call whose rows have no cut skips the list
// and the cut classes); 500 rows of 50257 without branches: 16, none, 43, 6, 17, 20.
// The floor is the logits read once, 13 and 20 us; the kernels read them twice.  The
// weights are bound by vector instructions, some 44 a token of which half are float64;
// the statistics by memory without branches and by the exponentials
// with one; the list by the lines of logits around its tokens; the row kernels by
// their chains of dependent steps, a workgroup a row (64 rows leave three quarters
// of the compute units idle, and a flat row's candidate tiles are all its workgroup's).
#include <cmath>

#include "../../include/dbt.h"
#include "common.h"
#include "host_internal.h"

// A token's weight is evaluated by three kernels, which have to agree on its
// bits: fused operations are the ones written here, no others.
#pragma clang fp contract(off)

namespace dbt {
namespace {

typedef unsigned long long u64;

constexpr int kTile = 2048;         // tokens of one statistics tile
constexpr int kMaxVocab = 1 << 20;
constexpr int kParamSets = 96, kParamRows = 2048;  // different parameters, and rows, of one launch of the first kernel
constexpr int kClasses = 256;       // weight classes: 0..253 by octave eighths, 254 everything lower, 255 weight zero
constexpr int kLow = 254, kNone = 255;
constexpr int kMaxScale = 46;       // s at most: the largest mixture value, within some 2^-52 of max m, has weight 2^s
constexpr int kRankCap = 64;        // tokens that are ranked against each other
constexpr int kFinal = 512;         // threads of the row kernels
constexpr int kMaxParts = kMaxVocab / kTile;
constexpr int kMaxPart = 4 * kTile;  // tokens of a part, at most

struct RowParams {
  float t, top_p, min_p;
  int top_k;  // 0: no cut
};
struct ParamBlock {  // (kernel arguments: below 4 KB)
  RowParams set[kParamSets];
  uint8_t of[kParamRows];  // each row's set
};

struct RowState {
  double scale[4];  // several paths: m / max m = sum_j scale[j] exp(z_j - zmax[j])
  double inv_t;
  u64 least;        // weights below stay out (min-p; 1: nothing but zeros)
  u64 k_mass;       // mass of the classes before kc
  float zmax[4];
  float top_p;
  float u;
  int top_k;
  int valid, greedy, cut;  // cut: top-k or top-p can remove something
  int kc, k_need;   // class in which top-k cuts and how many of it stay (kc = -1: nothing is cut)
  int k_whole;      // that class stays whole
  int pl, ph;       // classes in which top-p can cut (pl > ph: none)
  int lc;           // class of `least` if min-p can be the lowest cut (else -1)
  int l0, l1;       // those classes lie in l0 .. l1 (l0 > l1: none)
  unsigned listed;
};

struct Work {
  RowState *state;   // [rows]
  double2 *stats;    // [rows][tiles][4]: max, sum exp(z - max) of path j
  u64 *tmass;        // [rows][parts][256]: mass by class (rows without a cut: [0] the kept mass)
  unsigned *tcount;  // [rows][parts][256] (rows with top-k)
  u64 *upto;         // [rows][256]: mass of classes 0..c
  uint8_t *cls;      // [rows][vocab up to 16]
  u64 *lw;           // [rows][vocab] listed weights
  int *li;           // [rows][vocab] listed tokens
};

struct Args {
  const float *z1, *z2, *alpha, *u;
  int rows, V, Vp, s;
  int tiles;         // statistics tiles per row
  int parts, part;   // workgroups per row of the weighing kernels, tokens of each
  int *token;
  float *prob;
  Work w;
};

__device__ __forceinline__ const float *path_row(const Args &a, int j, int row) {
  return j == 0 ? a.z1 + (size_t)row * a.V : a.z2 + ((size_t)(j - 1) * a.rows + row) * a.V;
}

constexpr double kLog2eD = 1.4426950408889634074;

// a b + c with c in scalar registers (the compiler copies such a constant into
// the result's registers first, one more instruction each).
__device__ __forceinline__ double fma_s(double a, double b, double c) {
  double r;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(c));
  return r;
}

// 2^t for t <= 0 (and small t above), within 1e-14: t = n + f, |f| <= 1/2, and the
// Taylor series of 2^f = e^(f ln 2) to the eleventh power (its remainder is below
// (ln 2 / 2)^12 / 12! = 6.3e-15).  Sixteen instructions; the library's exp takes
// about three times as many, and these kernels are bound by them.
__device__ __forceinline__ double pow2(double t) {
  constexpr double L = 0.69314718055994530942;
  constexpr double c1 = L, c2 = c1 * L / 2, c3 = c2 * L / 3, c4 = c3 * L / 4, c5 = c4 * L / 5, c6 = c5 * L / 6, c7 = c6 * L / 7,
                   c8 = c7 * L / 8, c9 = c8 * L / 9, c10 = c9 * L / 10, c11 = c10 * L / 11;
  t = fmax(t, -1200.0);
  const double n = rint(t), f = t - n;
  double p = fma(f, c11, c10);
  p = fma_s(p, f, c9);
  p = fma_s(p, f, c8);
  p = fma_s(p, f, c7);
  p = fma_s(p, f, c6);
  p = fma_s(p, f, c5);
  p = fma_s(p, f, c4);
  p = fma_s(p, f, c3);
  p = fma_s(p, f, c2);
  p = fma_s(p, f, c1);
  p = fma(p, f, 1.0);
  return __builtin_amdgcn_ldexp(p, (int)n);
}

// log2(r), r > 0: the hardware's float32 logarithm y of the mantissa m, and the
// rest from m 2^-y = 1 + d with |d| below 2^-20.
__device__ __forceinline__ double log2_of(double r) {
  const double m = __builtin_amdgcn_frexp_mant(r);
  const double y = (double)__builtin_amdgcn_logf((float)m);
  const double d = fma(m, pow2(-y), -1.0);
  return (double)__builtin_amdgcn_frexp_exp(r) + y + d * fma(d, fma(d, 1.0 / 3, -0.5), 1.0) * kLog2eD;
}

// Logits i .. i + 3 of a row (rows start at any multiple of four bytes); from
// `hi` on those of tokens without weight.
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ float4u load4(const float *z, int i, int hi) {
  if (i + 4 <= hi) return *(const float4u *)(z + i);
  float4u v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = i + e < hi ? z[i + e] : -INFINITY;
  return v;
}

// scale_0 exp(z_0 - zmax_0) + ...: the same operations wherever it is evaluated
template <int NP> __device__ __forceinline__ double mixture(const RowState &r, const float (&z)[NP]) {
  double m = r.scale[0] * pow2(((double)z[0] - (double)r.zmax[0]) * kLog2eD);
#pragma unroll
  for (int j = 1; j < NP; ++j) m = fma(r.scale[j], pow2(((double)z[j] - (double)r.zmax[j]) * kLog2eD), m);
  return m;
}

// rint(w 2^s) as an integer and as a double
struct Weight {
  u64 w;
  double d;
};
template <int NP> __device__ __forceinline__ Weight weight(const RowState &r, const float (&z)[NP], int s) {
  double w;
  if constexpr (NP == 1) {
    w = pow2(((double)z[0] - (double)r.zmax[0]) * (r.inv_t * kLog2eD));
  } else {
    // the largest m is off 1 by its few roundings, 2^-51, which a small
    // temperature would blow up
    w = mixture<NP>(r, z);
    if (r.inv_t != 1.0) w = w > 1.0 - 0x1p-50 ? 1.0 : w > 0.0 ? pow2(log2_of(w) * r.inv_t) : 0.0;
  }
  // (w 2^s < 2^52: the sum's last mantissa bit is worth 1, so the addition rounds to an integer)
  constexpr double kBig = 4503599627370496.0;  // 2^52
  const double x = fma(w, __builtin_amdgcn_ldexp(1.0, s), kBig);
  return {(u64)__double_as_longlong(x) & 0xfffffffffffffull, x - kBig};
}

// Class of a weight, from the exponent and first three mantissa bits of the
// integer as a double.
__device__ __forceinline__ int weight_class(double d, int s) {
  const int c = ((1023 + s) << 3) + 7 - (__double2hiint(d) >> 17);
  return d == 0.0 ? kNone : min(kLow, c);
}
// Weights of class c: [lo, hi).
__device__ __forceinline__ void class_range(int c, int s, u64 &lo, u64 &hi) {
  const int sh = s - (c >> 3) - 3, f = 7 - (c & 7);  // (s >= 42: sh >= 8 for every class)
  lo = c == kLow ? 1 : (u64)(8 + f) << sh;
  hi = (u64)(9 + f) << sh;
}

// f x rounded down, and up where UP, for 0 <= f <= 1: f is a 24-bit integer
// times a power of two, the product fits 128 bits.  (A float64 product drops up to
// ten bits of a sum, and a border that it moves is another token.)
template <bool UP> __device__ __forceinline__ u64 times(float f, u64 x) {
  const unsigned b = __float_as_uint(f), e = b >> 23;
  const u64 m = (b & 0x7fffff) | (e ? 0x800000u : 0u);
  const int sh = 150 - (int)max(e, 1u);  // f = m 2^-sh, 23 <= sh <= 149
  const u64 hi = __umul64hi(m, x), lo = m * x;
  u64 q = 0, rest = hi | lo;
  if (sh < 64) {
    q = hi << (64 - sh) | lo >> sh;
    rest = lo << (64 - sh);
  } else if (sh < 88) {  // (the product is below 2^87)
    q = hi >> (sh - 64);
    rest = (hi & ((1ull << (sh - 64)) - 1)) | lo;
  }
  return q + (UP && rest != 0);
}

// Inclusive running sum over the wave's lanes (all of them active) without
// LDS: shifts within each row of 16, then the rows' sums handed on.
__device__ __forceinline__ u64 wave_scan64(u64 v) {
  auto add = [](u64 x, auto ctrl, auto rows) {
    const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, true);
    const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xf, true);
    return x + ((u64)hi << 32 | lo);
  };
  const std::integral_constant<int, 0xf> all{};
  v = add(v, std::integral_constant<int, 0x111>{}, all);  // row_shr:1, 2, 4, 8
  v = add(v, std::integral_constant<int, 0x112>{}, all);
  v = add(v, std::integral_constant<int, 0x114>{}, all);
  v = add(v, std::integral_constant<int, 0x118>{}, all);
  v = add(v, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});  // row_bcast:15 to rows 1 and 3
  return add(v, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});  // row_bcast:31 to rows 2 and 3
}
__device__ __forceinline__ u64 lane64(u64 v, int lane) {  // lane: the same in every lane
  return (u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ u64 wave_sum64(u64 v) { return lane64(wave_scan64(v), 63); }
// Sums (MAX: maxima) of the wave's N values, in lane 63, by the same steps in
// their fixed order.
template <bool MAX, int N> __device__ __forceinline__ void wave_reduce_d(double (&v)[N]) {
  auto step = [&](auto ctrl, auto rows) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      // (a lane without a partner: 0, or its own value)
      const int lo = __double2loint(v[k]), hi = __double2hiint(v[k]);
      const double o = __hiloint2double(
          __builtin_amdgcn_update_dpp(MAX ? hi : 0, hi, decltype(ctrl)::value, decltype(rows)::value, 0xf, false),
          __builtin_amdgcn_update_dpp(MAX ? lo : 0, lo, decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
      v[k] = MAX ? fmax(v[k], o) : v[k] + o;
    }
  };
  const std::integral_constant<int, 0xf> all{};
  step(std::integral_constant<int, 0x111>{}, all);
  step(std::integral_constant<int, 0x112>{}, all);
  step(std::integral_constant<int, 0x114>{}, all);
  step(std::integral_constant<int, 0x118>{}, all);
  step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
  step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
}
// The same over a row kernel's block, for every thread.
template <bool MAX, int N> __device__ __forceinline__ void block_reduce_d(double (&v)[N], double (*red)[4]) {
  wave_reduce_d<MAX>(v);
  __syncthreads();  // (the last call's readers)
  if ((threadIdx.x & 63) == 63)
#pragma unroll
    for (int k = 0; k < N; ++k) red[threadIdx.x >> 6][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = red[0][k];
#pragma unroll
    for (int w = 1; w < kFinal / 64; ++w) v[k] = MAX ? fmax(v[k], red[w][k]) : v[k] + red[w][k];
  }
}

// A row's parameters.  The greedy token is the first of the largest weight:
// a draw with u = 0 among those of weight 2^s.
__device__ __forceinline__ void set_params(const Args &a, const RowParams &p, int row) {
  RowState &r = a.w.state[row];
  const bool greedy = p.t == 0.f;
  r.greedy = greedy;
  r.inv_t = greedy ? 1.0 : 1.0 / (double)p.t;
  r.top_p = p.top_p;
  r.top_k = p.top_k >= a.V ? 0 : p.top_k;
  r.cut = !greedy && (r.top_k > 0 || p.top_p < 1.f);
  const u64 least = greedy ? 1ull << a.s : (u64)__double2ull_rn(ldexp((double)p.min_p, a.s));
  r.least = least > 1 ? least : 1;
  const float u = a.u[row];
  r.u = !greedy && u > 0.f ? fminf(u, 0.99999994f) : 0.f;
  r.listed = 0;
}

// Statistics of a tile of path blockIdx.z by one wave: its maximum and, with
// several paths (SUM), the sum of exponentials; NaN for a tile that holds a NaN or
// +infinity.  Each lane has its 32 values in flight together.
template <bool SUM>
__global__ __launch_bounds__(256) void k_sample_stats(Args a, ParamBlock pb, int row0) {
  const int lane = threadIdx.x & 63, row = row0 + blockIdx.y, j = blockIdx.z;
  const int tile = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x == 0 && j == 0 && threadIdx.x == 0) set_params(a, pb.set[pb.of[blockIdx.y]], row);
  if (tile >= a.tiles) return;
  constexpr int N = kTile / 64;
  const float *z = path_row(a, j, row) + tile * kTile;
  const int n = a.V - tile * kTile;
  float v[N];
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = z[min(k * 64 + lane, n - 1)];
  float mx = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    mx = fmaxf(mx, v[k]);
    bad |= !(v[k] < INFINITY);
  }
  mx = wave_max_dpp(mx);
  double sum[1] = {0.0};
  if constexpr (SUM) {
    if (mx > -INFINITY) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const double e = pow2(((double)v[k] - (double)mx) * kLog2eD);
        sum[0] += k * 64 + lane < n ? e : 0.0;  // (values past the row repeat its last)
      }
    }
    wave_reduce_d<false>(sum);
  }
  if (__any(bad)) sum[0] = __longlong_as_double(0x7ff8000000000000ll);
  if (lane == 63) a.w.stats[((size_t)row * a.tiles + tile) * 4 + j] = make_double2(mx, sum[0]);
}

// Row constants of several paths: each one's maximum and normaliser, and the
// largest mixture value.  A tile holds none above ub = sum_j scale_j exp(max_j - zmax_j), while
// the token of a tile's maximum proves lb = max_j of the terms: only tiles with
// ub >= lb (less a margin over both sides' rounding) are evaluated.
template <int NP>
__global__ __launch_bounds__(kFinal) void k_sample_rows(Args a) {
  __shared__ double red[kFinal / 64][4];
  __shared__ int list[kMaxVocab / kTile];
  __shared__ int nlist;
  const int row = blockIdx.x, t = threadIdx.x;
  static_assert(kMaxVocab / kTile <= kFinal, "one tile per thread");
  RowState &r = a.w.state[row];
  double2 st[NP];  // this thread's tile
#pragma unroll
  for (int j = 0; j < NP; ++j)
    st[j] = t < a.tiles ? a.w.stats[((size_t)row * a.tiles + t) * 4 + j] : make_double2(-INFINITY, 0.0);
  double M[NP], S[NP], term[NP];
  bool ok = true;
#pragma unroll
  for (int j = 0; j < NP; ++j) M[j] = st[j].x;
  block_reduce_d<true>(M, red);
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    term[j] = t < a.tiles ? pow2((st[j].x - M[j]) * kLog2eD) : 0.0;
    S[j] = st[j].y > 0.0 ? st[j].y * term[j] : st[j].y;
  }
  block_reduce_d<false>(S, red);
#pragma unroll
  for (int j = 0; j < NP; ++j) ok = ok && M[j] > -INFINITY && S[j] == S[j];
  RowState rs;
  const double al = a.alpha[row];
  ok = ok && al >= 0.0 && al <= 1.0;
  rs.scale[0] = al / S[0];
#pragma unroll
  for (int j = 1; j < NP; ++j) rs.scale[j] = (1.0 - al) / (NP - 1) / S[j];
#pragma unroll
  for (int j = 0; j < NP; ++j) rs.zmax[j] = (float)M[j];
  double mmax = 1.0;
  if (ok) {
    double lb[1] = {0.0}, ub = 0.0;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      term[j] *= rs.scale[j];
      lb[0] = fmax(lb[0], term[j]);
      ub += term[j];
    }
    if (t == 0) nlist = 0;
    block_reduce_d<true>(lb, red);  // (its barriers come after the clearing)
    if (t < a.tiles && ub >= lb[0] * (1.0 - 1e-9)) list[atomicAdd(&nlist, 1)] = t;  // (a maximum has no order)
    __syncthreads();
    double mx[1] = {0.0};
    // G tiles at a time, their loads in flight together (a last one again)
    constexpr int N = kTile / kFinal, G = 4;
    const int tiles = __builtin_amdgcn_readfirstlane(nlist);
    for (int n = 0; n < tiles; n += G) {
      float z[G * N][NP];
#pragma unroll
      for (int k = 0; k < G * N; ++k)
#pragma unroll
        for (int j = 0; j < NP; ++j)
          z[k][j] = path_row(a, j, row)[min(a.V - 1, list[min(n + k / N, tiles - 1)] * kTile + k % N * kFinal + t)];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if (n + g >= tiles) break;
#pragma unroll
        for (int k = g * N; k < g * N + N; ++k) mx[0] = fmax(mx[0], mixture<NP>(rs, z[k]));
      }
    }
    block_reduce_d<true>(mx, red);
    mmax = mx[0];
  }
  if (t == 0) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      r.scale[j] = rs.scale[j] / mmax;
      r.zmax[j] = rs.zmax[j];
    }
    r.valid = ok;
  }
}

// Weights of one part of a row: histogram by class and the tokens' classes, or,
// for a row without a cut, the mass that stays.
template <int NP>
__global__ __launch_bounds__(256) void k_sample_weigh(Args a) {
  __shared__ u64 mass[kClasses];
  __shared__ unsigned count[kClasses];
  const int part = blockIdx.x, row = blockIdx.y, t = threadIdx.x;
  RowState r = a.w.state[row];
  const int lo = part * a.part, hi = min(a.V, lo + a.part);
  mass[t] = 0;
  count[t] = 0;
  if constexpr (NP == 1) {
    // the path's maximum straight from the tiles' statistics (+infinity: the row has no answer)
    __shared__ float top[4];
    float m = -INFINITY;
    for (int i = t; i < a.tiles; i += 256) {
      const double2 st = a.w.stats[((size_t)row * a.tiles + i) * 4];
      m = st.y == st.y ? fmaxf(m, (float)st.x) : INFINITY;
    }
    m = wave_max_dpp(m);
    if ((t & 63) == 0) top[t >> 6] = m;
    __syncthreads();
    r.zmax[0] = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    r.valid = r.zmax[0] > -INFINITY && r.zmax[0] < INFINITY;
    if (part == 0 && t == 0) {
      a.w.state[row].zmax[0] = r.zmax[0];
      a.w.state[row].valid = r.valid;
    }
  } else {
    __syncthreads();
  }
  if (!r.valid) return;
  u64 kept = 0;  // no cut: kept mass; cut: mass of the low class
  unsigned low = 0;
  // four neighbours a thread (their classes are one store), the next round's
  // logits on their way while these are weighed
  constexpr int Q = NP <= 2 ? 2 : 1;
  float4u z[Q][NP], zn[Q][NP];
  auto fetch = [&](int i0, float4u (&v)[Q][NP]) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int j = 0; j < NP; ++j) v[q][j] = load4(path_row(a, j, row), i0 + q * 1024 + t * 4, hi);
  };
  fetch(lo, zn);
  for (int i0 = lo; i0 < hi; i0 += Q * 1024) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int j = 0; j < NP; ++j) z[q][j] = zn[q][j];
    if (i0 + Q * 1024 < hi) fetch(i0 + Q * 1024, zn);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int i = i0 + q * 1024 + t * 4;
      if (i >= hi) continue;
      Weight w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float ze[NP];
#pragma unroll
        for (int j = 0; j < NP; ++j) ze[j] = z[q][j][e];
        w[e] = weight<NP>(r, ze, a.s);
      }
      if (!r.cut) {
#pragma unroll
        for (int e = 0; e < 4; ++e) kept += w[e].w >= r.least ? w[e].w : 0;
        continue;
      }
      uint32_t cls = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = weight_class(w[e].d, a.s);
        cls |= (uint32_t)c << (8 * e);
        kept += c == kLow ? w[e].w : 0;
        low += c == kLow;
        if (c < kLow) {
          atomicAdd(&mass[c], w[e].w);
          if (r.top_k > 0) atomicAdd(&count[c], 1u);
        }
      }
      *(uint32_t *)(a.w.cls + (size_t)row * a.Vp + i) = cls;
    }
  }
  const int slot = r.cut ? kLow : 0;
  kept = wave_sum64(kept);
  const u64 lows = wave_sum64(low);
  if ((t & 63) == 0) {
    atomicAdd(&mass[slot], kept);
    atomicAdd(&count[slot], (unsigned)lows);
  }
  __syncthreads();
  const size_t o = ((size_t)row * a.parts + part) * kClasses + t;
  if (r.cut) {
    a.w.tmass[o] = mass[t];
    if (r.top_k > 0) a.w.tcount[o] = count[t];
  } else if (t == 0) {
    a.w.tmass[o] = mass[0];
  }
}

// Where the cuts can fall: the class in which top-k is reached, and those in
// which top-p can be, whose target follows from what top-k keeps of its class.
__global__ __launch_bounds__(256) void k_sample_cut(Args a) {
  __shared__ u64 ms[kClasses], red[4];
  __shared__ unsigned cs[kClasses], wred[4];
  __shared__ int kc_s, pl_s, ph_s;
  const int row = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
  RowState &r = a.w.state[row];
  if (!r.valid || !r.cut) return;
  const int top_k = r.top_k;
  u64 m = 0;
  unsigned c = 0;
  const size_t o = (size_t)row * a.parts * kClasses + t;
#pragma unroll 8
  for (int p = 0; p < a.parts; ++p) m += a.w.tmass[o + (size_t)p * kClasses];
  if (top_k > 0)
#pragma unroll 8
    for (int p = 0; p < a.parts; ++p) c += a.w.tcount[o + (size_t)p * kClasses];
  const u64 mi = wave_scan64(m), ci = wave_scan64(c);
  if (lane == 63) {
    red[wave] = mi;
    wred[wave] = (unsigned)ci;
  }
  if (t == 0) kc_s = pl_s = ph_s = -1;
  __syncthreads();
  u64 mo = 0, total = 0;
  unsigned co = 0;
  for (int w = 0; w < 4; ++w) {
    if (w < wave) {
      mo += red[w];
      co += wred[w];
    }
    total += red[w];
  }
  ms[t] = mo + mi;
  cs[t] = co + (unsigned)ci;
  a.w.upto[(size_t)row * kClasses + t] = ms[t];
  __syncthreads();
  const u64 m0 = t ? ms[t - 1] : 0;
  const unsigned c0 = t ? cs[t - 1] : 0;
  if (top_k > 0 && cs[t] >= (unsigned)top_k && c0 < (unsigned)top_k) kc_s = t;
  __syncthreads();
  const int kc = kc_s;
  // least and largest mass that top-k can keep
  u64 wl = total, wh = total;
  unsigned need = 0;
  bool whole = false;
  if (kc >= 0) {
    need = (unsigned)top_k - (kc ? cs[kc - 1] : 0);
    const u64 before = kc ? ms[kc - 1] : 0, in = ms[kc] - before;
    whole = cs[kc] == (unsigned)top_k;
    u64 lo, hi;
    class_range(kc, a.s, lo, hi);
    wl = whole ? ms[kc] : before + need * lo;
    wh = whole ? ms[kc] : before + min(in, need * (hi - 1));
  }
  const float top_p = r.top_p;
  if (top_p < 1.f) {
    const u64 nl = times<true>(top_p, wl), nh = times<true>(top_p, wh);
    if (ms[t] >= nl && m0 < nl) pl_s = t;
    if (ms[t] >= nh && m0 < nh) ph_s = t;
  }
  __syncthreads();
  if (t == 0) {
    r.kc = kc;
    r.k_need = (int)need;
    r.k_whole = whole;
    r.k_mass = kc > 0 ? ms[kc - 1] : 0;
    r.pl = top_p < 1.f ? pl_s : 0;
    r.ph = top_p < 1.f ? ph_s : -1;
    int l0 = kClasses, l1 = -1;
    if (kc >= 0 && !whole) l0 = l1 = kc;
    if (top_p < 1.f) {
      l0 = min(l0, pl_s);
      l1 = max(l1, ph_s);
    }
    int lc = r.least > 1 ? weight_class((double)r.least, a.s) : -1;
    if (lc > (l1 >= 0 ? l1 : kc >= 0 ? kc : kLow)) lc = -1;  // the other cuts have removed what it would
    if (lc >= 0) {
      l1 = lc < l0 ? lc : l1;  // above every other cut: those do not matter
      l0 = min(l0, lc);
    }
    r.lc = lc;
    r.l0 = l0;
    r.l1 = l1;
  }
}

// Tokens of those classes, with their weights, in any order.  (One test a token
// for nearly all of them; the exact one for those that pass it: between the
// classes of top-p and of top-k may lie almost top_k tokens.)
template <int NP>
__global__ __launch_bounds__(256) void k_sample_list(Args a) {
  __shared__ uint16_t idx[kMaxPart];
  __shared__ unsigned n_s, at_s;
  const int part = blockIdx.x, row = blockIdx.y, t = threadIdx.x;
  const RowState r = a.w.state[row];
  if (!r.valid || !r.cut || r.l0 > r.l1) return;
  const int kc = r.k_whole ? -1 : r.kc;
  const int lo = part * a.part, hi = min(a.V, lo + a.part);
  const uint8_t *cls = a.w.cls + (size_t)row * a.Vp;
  if (t == 0) n_s = 0;
  __syncthreads();
  for (int i = lo + t * 16; i < hi; i += 256 * 16) {
    const u32x4 v = *(const u32x4 *)(cls + i);
    const u64 half[2] = {(u64)v[1] << 32 | v[0], (u64)v[3] << 32 | v[2]};
    unsigned m = 0;
#pragma unroll
    for (int b = 0; b < 16; ++b) {
      const int c = (v[b >> 2] >> (8 * (b & 3))) & 0xff;
      m |= (unsigned)(c - r.l0) <= (unsigned)(r.l1 - r.l0) ? 1u << b : 0u;
    }
    if (hi - i < 16) m &= (1u << (hi - i)) - 1;
    for (unsigned k = m; k; k &= k - 1) {
      const int b = __ffs(k) - 1, c = (half[b >> 3] >> (8 * (b & 7))) & 0xff;
      if (!((c >= r.pl && c <= r.ph) || c == kc || c == r.lc)) m &= ~(1u << b);
    }
    if (m) {
      unsigned at = atomicAdd(&n_s, (unsigned)__popc(m));
      for (; m; m &= m - 1) idx[at++] = (uint16_t)(i + __ffs(m) - 1 - lo);
    }
  }
  __syncthreads();
  // (the first token of every thread is on its way before the list's place is known)
  const int n = (int)n_s;
  float z[NP];
  auto fetch = [&](int k) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NP; ++j) z[j] = path_row(a, j, row)[lo + idx[k]];
  };
  if (t < n) fetch(t);
  if (t == 0 && n) at_s = atomicAdd(&a.w.state[row].listed, (unsigned)n);
  __syncthreads();
  for (int k = t; k < n; k += 256) {
    if (k != t) fetch(k);
    const size_t o = (size_t)row * a.V + at_s + k;
    a.w.lw[o] = weight<NP>(r, z, a.s).w;
    a.w.li[o] = lo + idx[k];
  }
}

struct FinalShared {
  u64 mass[256];
  unsigned count[256];
  u64 rw[kRankCap];
  int ri[kRankCap];
  u64 pmass[kMaxParts], runs[kMaxPart / kTile * (kFinal / 64)];
  u64 red[kFinal / 64];
  u64 cut_w, sum, need;
  int cut_i, n, bin, token;
  unsigned inside;
};

// One step of narrowing: of 256 bins (filled in sh.mass, sh.count), taken from
// the first in `descending` or ascending order, the one in which `need` (of mass or
// number) is reached: sh.bin, sh.inside, what is left of need in sh.need, the
// mass of the bins before it in sh.sum.  By the first wave.
__device__ __forceinline__ void pick_bin(FinalShared &sh, u64 need, bool by_mass, bool descending) {
  const int lane = threadIdx.x & 63;
  u64 v[4], m[4], vs = 0, msum = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int b = descending ? 255 - (lane * 4 + k) : lane * 4 + k;
    m[k] = sh.mass[b];
    v[k] = by_mass ? m[k] : sh.count[b];
    vs += v[k];
    msum += m[k];
  }
  u64 before = wave_scan64(vs), mb = wave_scan64(msum) - msum;
  need = min(need, lane64(before, 63));
  before -= vs;
  if (before < need && before + vs >= need) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (before < need && before + v[k] >= need) {
        const int b = descending ? 255 - (lane * 4 + k) : lane * 4 + k;
        sh.bin = b;
        sh.inside = sh.count[b];
        sh.need = need - before;
        sh.sum = mb;
      }
      before += v[k];
      mb += m[k];
    }
  }
}

// A row's listed tokens as its workgroup goes over them: a list that fits sits
// in registers, loaded once with every load in flight; others are read again.
struct Listed {
  static constexpr int N = 8;
  const u64 *lw;
  const int *li;
  int n;
  u64 w[N];
  int i[N];
  __device__ __forceinline__ void load() {
    if (n > N * kFinal) return;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int e = k * kFinal + (int)threadIdx.x;
      w[k] = e < n ? lw[e] : 0;  // (weight zero: in no range)
      i[k] = e < n ? li[e] : 0;
    }
  }
  template <typename F> __device__ __forceinline__ void each(F f) const {
    if (n <= N * kFinal) {
#pragma unroll
      for (int k = 0; k < N; ++k) f(w[k], i[k]);
    } else {
      for (int e = threadIdx.x; e < n; e += kFinal) f(lw[e], li[e]);
    }
  }
};

// Where the order by (weight falling, index) is cut among the listed weights of
// [lo, hi), `inside` of them, after `need` tokens (by_mass: after the shortest run
// whose mass reaches need; the range holds as much): the last token that stays
// in sh.cut_w, sh.cut_i, the mass that stays of the range in sh.sum.  Ranges of
// more than kRankCap tokens are narrowed 256-fold by histograms of the weight and, once all
// weights are equal, of the index.
__device__ __forceinline__ void cut_range(FinalShared &sh, const Listed &list, int V, u64 lo, u64 hi, u64 need, bool by_mass) {
  const int t = threadIdx.x;
  u64 above = 0;  // mass that stays above the narrowed range
  int ilo = 0, ihi = V;
  unsigned inside = 0;
  {
    unsigned mine = 0;
    list.each([&](u64 w, int) { mine += w >= lo && w < hi; });
    const u64 w = wave_sum64(mine);
    __syncthreads();
    if ((t & 63) == 0) sh.red[t >> 6] = w;
    __syncthreads();
    for (int k = 0; k < kFinal / 64; ++k) inside += (unsigned)sh.red[k];
  }
  while (inside > kRankCap && (hi - lo > 1 || ihi - ilo > 1)) {
    const bool by_index = hi - lo <= 1;
    const u64 width = by_index ? ihi - ilo : hi - lo;
    const int bits = 64 - __clzll(width - 1), shift = bits > 8 ? bits - 8 : 0;
    if (by_index && by_mass) {  // (equal weights: so many of them)
      need = (need + lo - 1) / lo;
      by_mass = false;
    }
    __syncthreads();
    if (t < 256) {
      sh.mass[t] = 0;
      sh.count[t] = 0;
    }
    __syncthreads();
    list.each([&](u64 w, int ix) {
      if (w < lo || w >= hi || ix < ilo || ix >= ihi) return;
      const int b = by_index ? (ix - ilo) >> shift : (int)((w - lo) >> shift);
      atomicAdd(&sh.mass[b], w);
      atomicAdd(&sh.count[b], 1u);
    });
    __syncthreads();
    if (t < 64) pick_bin(sh, need, by_mass, !by_index);
    __syncthreads();
    if (by_index) {
      ilo += sh.bin << shift;
      ihi = min(ihi, ilo + (1 << shift));
    } else {
      lo += (u64)sh.bin << shift;
      hi = min(hi, lo + (1ull << shift));
    }
    need = sh.need;
    above += sh.sum;
    inside = sh.inside;
  }
  __syncthreads();
  if (t == 0) sh.n = 0;
  __syncthreads();
  list.each([&](u64 w, int ix) {
    if (w < lo || w >= hi || ix < ilo || ix >= ihi) return;
    const int k = atomicAdd(&sh.n, 1);  // (any order: ranks come from weight and index)
    if (k < kRankCap) {
      sh.rw[k] = w;
      sh.ri[k] = ix;
    }
  });
  if (t == 0) {
    sh.cut_w = lo;
    sh.cut_i = V;
    sh.sum = above;
  }
  __syncthreads();
  // eight threads a token, each comparing it with an eighth of the others
  const int k = min(sh.n, kRankCap), e = t >> 3;
  static_assert(kRankCap * 8 == kFinal, "every token's eight threads");
  u64 mass = 0, w = 0;
  unsigned rank = 0;
  int ix = 0;
  if (e < k) {
    w = sh.rw[e];
    ix = sh.ri[e];
    for (int o = t & 7; o < k; o += 8)
      if (sh.rw[o] > w || (sh.rw[o] == w && sh.ri[o] < ix)) {
        mass += sh.rw[o];
        ++rank;
      }
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    mass += __shfl_xor(mass, o, 64);
    rank += __shfl_xor(rank, o, 64);
  }
  if (e < k && (t & 7) == 0) {
    // the token before which less than need has come, and with which it is reached
    const u64 before = by_mass ? mass : rank, with = by_mass ? mass + w : rank + 1;
    if (before < need && with >= need) {
      sh.cut_w = w;
      sh.cut_i = ix;
      sh.sum = above + mass + w;
    }
  }
  __syncthreads();
}

// One workgroup per row: the exact cut among the listed tokens, every part's
// mass above it, the part in which the draw falls, its token.
template <int NP>
__global__ __launch_bounds__(kFinal) void k_sample_final(Args a) {
  constexpr int NW = kFinal / 64;
  __shared__ FinalShared sh;
  const int row = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const RowState r = a.w.state[row];
  if (!r.valid) {
    if (t == 0) {
      a.token[row] = -1;
      if (a.prob) a.prob[row] = 0.f;
    }
    return;
  }
  const u64 *tm = a.w.tmass + (size_t)row * a.parts * kClasses;
  // stays: W > cut_w, or W == cut_w and the index at most cut_i
  u64 cut_w = 1;
  int cut_i = a.V;
  Listed list{a.w.lw + (size_t)row * a.V, a.w.li + (size_t)row * a.V, r.cut ? (int)r.listed : 0};
  list.load();
  if (r.cut) {
    const u64 *upto = a.w.upto + (size_t)row * kClasses;
    u64 total = upto[kLow], lo, hi;
    if (r.kc >= 0) {
      class_range(r.kc, a.s, lo, hi);
      if (r.k_whole) {
        total = upto[r.kc];
        cut_w = lo;
      } else {
        cut_range(sh, list, a.V, lo, hi, r.k_need, false);
        total = r.k_mass + sh.sum;
        cut_w = sh.cut_w;
        cut_i = sh.cut_i;
      }
    }
    if (r.top_p < 1.f) {
      const u64 need = times<true>(r.top_p, total);
      int c = r.pl;
      while (c < r.ph && upto[c] < need) ++c;
      class_range(c, a.s, lo, hi);
      __syncthreads();
      cut_range(sh, list, a.V, lo, hi, need - (c ? upto[c - 1] : 0), true);
      cut_w = sh.cut_w;
      cut_i = sh.cut_i;
    }
  }
  if (r.least > cut_w) {
    cut_w = r.least;
    cut_i = a.V;
  }
  // the parts' masses: the classes above the cut's from their histograms, and
  // what stays of that class from the list
  if (r.cut) {
    const int ce = weight_class((double)cut_w, a.s);
    u64 lo, hi;
    class_range(ce, a.s, lo, hi);
    const bool whole = cut_w <= lo && cut_i >= a.V - 1;
    const int last = whole ? ce : ce - 1;
    for (int p = wave; p < a.parts; p += NW) {
      u64 m = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = k * 64 + lane;
        const u64 x = tm[(size_t)p * kClasses + c];
        m += c <= last ? x : 0;
      }
      m = wave_sum64(m);
      if (lane == 0) sh.pmass[p] = m;
    }
    __syncthreads();
    if (!whole)
      list.each([&](u64 w, int ix) {
        if (w < hi && (w > cut_w || (w == cut_w && ix <= cut_i))) atomicAdd(&sh.pmass[ix / a.part], w);
      });
  } else {
    for (int p = t; p < a.parts; p += kFinal) sh.pmass[p] = tm[(size_t)p * kClasses];
  }
  __syncthreads();
  static_assert(kMaxParts <= kFinal, "one part per thread");
  u64 m = t < a.parts ? sh.pmass[t] : 0;
  u64 incl = wave_scan64(m);
  if (lane == 63) sh.red[wave] = incl;
  __syncthreads();
  u64 total = 0, before = 0;
  for (int k = 0; k < NW; ++k) {
    if (k < wave) before += sh.red[k];
    total += sh.red[k];
  }
  if (total == 0) {  // (not reached: the largest weight stays)
    if (t == 0) {
      a.token[row] = -1;
      if (a.prob) a.prob[row] = 0.f;
    }
    return;
  }
  incl += before;
  const u64 target = times<false>(r.u, total);  // (u < 1: below total)
  if (target < incl && target >= incl - m) {
    sh.bin = t;
    sh.sum = incl - m;
  }
  __syncthreads();
  // the token: sums of every 256 neighbours by the waves, then the wave that
  // holds the target weighs its 256 again and finds the token
  constexpr int PER = 4, RUN = PER * 64;
  static_assert(RUN * NW == kTile, "a run per wave");
  const int p0 = sh.bin * a.part, n = min(a.V, p0 + a.part) - p0;
  before = sh.sum;
  auto run = [&](int s0, u64 (&w)[PER]) __attribute__((always_inline)) {  // this lane's four of the run's weights that stay
    const int i = p0 + s0 + lane * PER;
    float4u z[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) z[j] = load4(path_row(a, j, row), i, p0 + n);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      float zk[NP];
#pragma unroll
      for (int j = 0; j < NP; ++j) zk[j] = z[j][k];
      const u64 x = weight<NP>(r, zk, a.s).w;
      w[k] = x > cut_w || (x == cut_w && i + k <= cut_i) ? x : 0;
    }
  };
#pragma unroll 2
  for (int c = 0; c < kMaxPart / kTile; ++c) {
    u64 w[PER], sum = 0;
    if (c * kTile + wave * RUN < n) {
      run(c * kTile + wave * RUN, w);
#pragma unroll
      for (int k = 0; k < PER; ++k) sum += w[k];
      sum = wave_sum64(sum);
    }
    if (lane == 0) sh.runs[c * NW + wave] = sum;
  }
  __syncthreads();
  static_assert(kMaxPart / kTile * NW <= 64, "one run per lane");
  u64 mine = lane < kMaxPart / kTile * NW ? sh.runs[lane] : 0, runs = before + wave_scan64(mine);
  const u64 at = __ballot(target < runs);
  const int pick = __ffsll(at) - 1;  // (every wave agrees)
  if (pick >= 0 && pick % NW == wave) {
    before = lane64(runs - mine, pick);
    const int s0 = pick / NW * kTile + wave * RUN;
    u64 w[PER], own = 0;
    run(s0, w);
#pragma unroll
    for (int k = 0; k < PER; ++k) own += w[k];
    before += wave_scan64(own) - own;
    if (before <= target && target < before + own) {
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        if (before <= target && target < before + w[k]) {
          a.token[row] = p0 + s0 + lane * PER + k;
          if (a.prob) a.prob[row] = r.greedy ? 1.f : (float)((double)w[k] / (double)total);
        }
        before += w[k];
      }
    }
  }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Parts of a row: statistics tiles, up to four of them together where the rows
// alone fill the chip (a part's histogram is written and read again: 3 KB).
void partition(int rows, int vocab, int *tiles, int *parts, int *part) {
  *tiles = (vocab + kTile - 1) / kTile;
  int f = 1;
  while (f < kMaxPart / kTile && (long long)rows * ((*tiles + f) / (f + 1)) >= 2048) ++f;
  *part = f * kTile;
  *parts = (vocab + *part - 1) / *part;
}

int round16(int x) { return (x + 15) / 16 * 16; }

size_t layout(int rows, int vocab, char *base, Work *w) {
  int tiles, parts, part;
  partition(rows, vocab, &tiles, &parts, &part);
  size_t o = 0;
  auto take = [&](size_t bytes) {
    char *p = base + o;
    o += align256(bytes);
    return p;
  };
  const size_t R = rows, V = vocab;
  Work x;
  x.state = (RowState *)take(R * sizeof(RowState));
  x.stats = (double2 *)take(R * tiles * 4 * sizeof(double2));
  x.tmass = (u64 *)take(R * parts * kClasses * 8);
  x.tcount = (unsigned *)take(R * parts * kClasses * 4);
  x.upto = (u64 *)take(R * kClasses * 8);
  x.cls = (uint8_t *)take(R * round16(vocab));
  x.lw = (u64 *)take(R * V * 8);
  x.li = (int *)take(R * V * 4);
  if (w) *w = x;
  return o;
}

dbt_status fail(dbt_status s, const char *msg) { return set_error(s, msg); }

template <int NP> hipError_t launch(const Args &a, const dbt_sampling *p, bool cuts, hipStream_t st) {
  for (int r0 = 0; r0 < a.rows;) {
    // rows while their parameters fit (the requests of a batch, or the nodes of
    // a request's tree, share them)
    ParamBlock pb;
    int n = 0, sets = 0, last = -1;
    for (; r0 + n < a.rows && n < kParamRows; ++n) {
      const dbt_sampling &q = p[r0 + n];
      auto same = [&](int k) {
        return pb.set[k].t == q.temperature && pb.set[k].top_p == q.top_p && pb.set[k].min_p == q.min_p && pb.set[k].top_k == q.top_k;
      };
      int k = last >= 0 && same(last) ? last : 0;
      while (k < sets && !same(k)) ++k;
      if (k == kParamSets) break;
      if (k == sets) pb.set[sets++] = RowParams{q.temperature, q.top_p, q.min_p, q.top_k};
      pb.of[n] = (uint8_t)(last = k);
    }
    hipLaunchKernelGGL(k_sample_stats<(NP > 1)>, dim3((a.tiles + 3) / 4, n, NP), dim3(256), 0, st, a, pb, r0);
    if (const hipError_t e = hipGetLastError()) return e;
    r0 += n;
  }
  if constexpr (NP > 1) {
    hipLaunchKernelGGL(k_sample_rows<NP>, dim3(a.rows), dim3(kFinal), 0, st, a);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  hipLaunchKernelGGL(k_sample_weigh<NP>, dim3(a.parts, a.rows), dim3(256), 0, st, a);
  if (const hipError_t e = hipGetLastError()) return e;
  if (cuts) {
    hipLaunchKernelGGL(k_sample_cut, dim3(a.rows), dim3(256), 0, st, a);
    if (const hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL(k_sample_list<NP>, dim3(a.parts, a.rows), dim3(256), 0, st, a);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  hipLaunchKernelGGL(k_sample_final<NP>, dim3(a.rows), dim3(kFinal), 0, st, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace dbt

using namespace dbt;

extern "C" size_t dbt_sample_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 1 || rows > 65535 || vocab < 1 || vocab > kMaxVocab) {
    fail(DBT_ERR_ARG, "rows must be in [1, 65535], vocab in [1, 2^20]");
    return 0;
  }
  return layout(rows, vocab, nullptr, nullptr);
}

extern "C" dbt_status dbt_sample(const dbt_sample_in *in, int32_t *token, float *prob, void *workspace,
                                 dbt_stream stream) {
  if (!in || !in->logits1 || !in->u || !in->h_params || !token) return fail(DBT_ERR_ARG, "NULL argument");
  if (in->rows < 1 || in->rows > 65535) return fail(DBT_ERR_ARG, "rows out of [1, 65535]");
  if (in->vocab < 1 || in->vocab > kMaxVocab) return fail(DBT_ERR_ARG, "vocab out of [1, 2^20]");
  if (in->n_branches < 0 || in->n_branches > 3) return fail(DBT_ERR_ARG, "n_branches must be in [0, 3]");
  if (in->n_branches > 0 && (!in->logits2 || !in->alpha)) return fail(DBT_ERR_ARG, "logits2 or alpha is NULL");
  if (!workspace || ((uintptr_t)workspace & 255)) return fail(DBT_ERR_ARG, "workspace NULL or not 256-byte aligned");
  bool cuts = false;
  for (int r = 0; r < in->rows; ++r) {
    const dbt_sampling &p = in->h_params[r];
    if (!(p.temperature >= 0.f) || !std::isfinite(p.temperature) || !(p.top_p > 0.f && p.top_p <= 1.f) ||
        !(p.min_p >= 0.f && p.min_p <= 1.f) || p.top_k < 0)
      return fail(DBT_ERR_ARG, "temperature must be >= 0, top_p in (0, 1], min_p in [0, 1], top_k >= 0");
    cuts = cuts || (p.temperature > 0.f && (p.top_p < 1.f || (p.top_k > 0 && p.top_k < in->vocab)));
  }
  Args a{};
  a.z1 = in->logits1;
  a.z2 = in->logits2;
  a.alpha = in->alpha;
  a.u = in->u;
  a.rows = in->rows;
  a.V = in->vocab;
  a.Vp = round16(in->vocab);
  a.s = 62;
  for (int v = 1; v < in->vocab; v *= 2) --a.s;  // 2^s * vocab <= 2^62
  if (a.s > kMaxScale) a.s = kMaxScale;
  partition(a.rows, a.V, &a.tiles, &a.parts, &a.part);
  a.token = token;
  a.prob = prob;
  layout(a.rows, a.V, (char *)workspace, &a.w);
  const hipStream_t st = (hipStream_t)stream;
  hipError_t e;
  switch (in->n_branches) {
    case 0: e = launch<1>(a, in->h_params, cuts, st); break;
    case 1: e = launch<2>(a, in->h_params, cuts, st); break;
    case 2: e = launch<3>(a, in->h_params, cuts, st); break;
    default: e = launch<4>(a, in->h_params, cuts, st); break;
  }
  if (e != hipSuccess) return fail(DBT_ERR_HIP, hipGetErrorString(e));
  return DBT_OK;
}
