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
// The cut is found without sorting: a histogram over 254 classes of
// W (eight per octave) by count and mass gives the class in which it falls;
// the tokens up to that class are listed in index order; a workgroup per row
// ranks the class's own tokens exactly.  The draw is a prefix search over the list
// (rows without a cut: over tile sums, then inside one tile).
#include <cmath>

#include "../../include/dbt.h"
#include "common.h"
#include "host_internal.h"

namespace {

using namespace dbt;
typedef unsigned long long u64;

constexpr int kTile = 2048;         // tokens of one statistics tile
constexpr int kMaxVocab = 1 << 20;
constexpr int kRowsPerCall = 128;   // rows of one launch of the first kernel (parameters travel as arguments)
constexpr int kClasses = 256;       // weight classes: 0..253 by octave eighths, 254 everything lower, 255 weight zero
constexpr int kLow = 254, kNone = 255;
constexpr int kRankCap = 2048;      // tokens of the cut's class that are ranked in LDS
constexpr int kFinal = 512;         // threads of the row kernel

struct RowParams {
  float t, top_p, min_p;
  int top_k;  // 0: no cut
};
struct ParamBlock {
  RowParams r[kRowsPerCall];
};

struct RowState {
  double scale[4];  // m = sum_j scale[j] exp(z_j - zmax[j])
  double inv_t, mmax;
  u64 least;        // weights below stay out (min-p; 1: nothing but zeros)
  float zmax[4];
  float top_p;
  float u;
  int top_k;
  int valid, greedy, cut;  // cut: top-k or top-p remove something
  int last;         // class of the cut: tokens of classes 0..last are listed
  int listed;
};

struct Work {
  RowState *state;   // [rows]
  double2 *stats;    // [rows][tiles][4]: max, sum exp(z - max) of path j
  u64 *tmass;        // [rows][parts][256]: mass by class (rows without a cut: [0] the kept mass)
  unsigned *tcount;  // [rows][parts][256]
  u64 *mass;         // [rows][256]
  unsigned *count;   // [rows][256]
  unsigned *toff;    // [rows][parts]: place in the list of a part's first listed token
  uint8_t *cls;      // [rows][vocab]
  u64 *lw;           // [rows][vocab] listed weights
  int *li;           // [rows][vocab] listed tokens
};

struct Args {
  const float *z1, *z2, *alpha, *u;
  int rows, V, nb, s;
  int tiles;         // statistics tiles per row
  int parts, part;   // workgroups per row of the weighing kernels, tokens of each
  int *token;
  float *prob;
  Work w;
};

template <int NP> __device__ __forceinline__ const float *path_row(const Args &a, int j, int row) {
  return j == 0 ? a.z1 + (size_t)row * a.V : a.z2 + ((size_t)(j - 1) * a.rows + row) * a.V;
}

// Mixture value of one token: the same operations wherever it is evaluated, so
// that the largest one divides to exactly 1.
template <int NP> __device__ __forceinline__ double mixture(const RowState &r, const float (&z)[NP]) {
  double m = r.scale[0] * exp((double)z[0] - (double)r.zmax[0]);
#pragma unroll
  for (int j = 1; j < NP; ++j) m = fma(r.scale[j], exp((double)z[j] - (double)r.zmax[j]), m);
  return m;
}

template <int NP> __device__ __forceinline__ u64 weight(const RowState &r, const float (&z)[NP], int s) {
  double w;
  if constexpr (NP == 1) {
    w = r.greedy ? (z[0] == r.zmax[0] ? 1.0 : 0.0) : exp(((double)z[0] - (double)r.zmax[0]) * r.inv_t);
  } else {
    w = mixture<NP>(r, z) / r.mmax;
    if (r.greedy) w = w == 1.0 ? 1.0 : 0.0;
    else if (r.inv_t != 1.0) w = exp(log(w) * r.inv_t);
  }
  return (u64)__double2ull_rn(ldexp(w, s));
}

__device__ __forceinline__ int weight_class(u64 w, int s) {
  if (w == 0) return kNone;
  const int msb = 63 - __clzll(w);
  const int f = msb >= 3 ? (int)(w >> (msb - 3)) & 7 : (int)(w << (3 - msb)) & 7;
  return min(kLow, (s - msb) * 8 + 7 - f);
}
// Weights of class c: [lo, hi).
__device__ __forceinline__ void class_range(int c, int s, u64 &lo, u64 &hi) {
  const int sh = s - (c >> 3) - 3, f = 7 - (c & 7);  // (s >= 42: sh >= 8 for every class)
  lo = c == kLow ? 1 : (u64)(8 + f) << sh;
  hi = (u64)(9 + f) << sh;
}

__device__ __forceinline__ u64 shfl_up64(u64 v, int d) { return __shfl_up(v, d, 64); }
__device__ __forceinline__ u64 wave_sum64(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ u64 wave_scan64(u64 v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 x = shfl_up64(v, o);
    if (lane >= o) v += x;
  }
  return v;
}
__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// (red: 16 doubles; every thread gets the result; fixed order)
__device__ __forceinline__ double block_sum_d(double v, double *red) {
  v = wave_sum_d(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0;
  for (int i = 0; i < (int)blockDim.x >> 6; ++i) t += red[i];
  return t;
}
__device__ __forceinline__ double block_max_d(double v, double *red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = red[0];
  for (int i = 1; i < (int)blockDim.x >> 6; ++i) t = fmax(t, red[i]);
  return t;
}

// Statistics of one tile: each path's maximum and, with several paths, the sum
// of exponentials; NaN for a tile that holds a NaN or +infinity.
template <int NP>
__global__ __launch_bounds__(256) void k_sample_stats(Args a, ParamBlock pb, int row0) {
  __shared__ float red[16];
  __shared__ double redd[16];
  const int tile = blockIdx.x, row = row0 + blockIdx.y, t = threadIdx.x;
  if (tile == 0 && t == 0) {
    const RowParams p = pb.r[blockIdx.y];
    RowState &r = a.w.state[row];
    r.greedy = p.t == 0.f;
    r.inv_t = p.t == 0.f ? 1.0 : 1.0 / (double)p.t;
    r.top_p = p.top_p;
    r.top_k = p.top_k >= a.V ? 0 : p.top_k;
    r.cut = !r.greedy && (r.top_k > 0 || p.top_p < 1.f);
    const u64 least = r.greedy ? 1 : __double2ull_rn(ldexp((double)p.min_p, a.s));
    r.least = least > 1 ? least : 1;
  }
  float v[NP][8];
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    const float *z = path_row<NP>(a, j, row);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = tile * kTile + k * 256 + t;
      v[j][k] = i < a.V ? z[i] : -INFINITY;
    }
  }
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    float mx = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      mx = fmaxf(mx, v[j][k]);
      bad |= !(v[j][k] < INFINITY);
    }
    mx = block_max(mx, red);
    double sum = 0.0;
    if (NP > 1 && mx > -INFINITY) {
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += exp((double)v[j][k] - (double)mx);
    }
    if (bad) sum = __longlong_as_double(0x7ff8000000000000ll);
    sum = block_sum_d(sum, redd);
    if (t == 0) a.w.stats[((size_t)row * a.tiles + tile) * 4 + j] = make_double2(mx, sum);
  }
}

// Row constants: every path's maximum and normaliser, and the largest mixture
// value.  A tile holds none above ub = sum_j scale_j exp(max_j - zmax_j), while
// the token of a tile's maximum proves lb = max_j of the terms: only tiles with
// ub >= lb (less a margin over both sides' rounding) are evaluated.
template <int NP>
__global__ __launch_bounds__(256) void k_sample_rows(Args a) {
  __shared__ float red[16];
  __shared__ double redd[16];
  __shared__ int list[kMaxVocab / kTile];
  __shared__ int nlist;
  const int row = blockIdx.x, t = threadIdx.x;
  const double2 *st = a.w.stats + (size_t)row * a.tiles * 4;
  RowState &r = a.w.state[row];
  float M[NP];
  double S[NP];
  bool ok = true;
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    float mx = -INFINITY;
    for (int i = t; i < a.tiles; i += 256) mx = fmaxf(mx, (float)st[i * 4 + j].x);
    M[j] = block_max(mx, red);
    double s = 0.0;
    if (NP == 1)  // (the sums only say whether the row is sound)
      for (int i = t; i < a.tiles; i += 256) s += st[i * 4 + j].y;
    else
      for (int i = t; i < a.tiles; i += 256)
        if (!(st[i * 4 + j].y == 0.0)) s += st[i * 4 + j].y * exp(st[i * 4 + j].x - (double)M[j]);
    S[j] = block_sum_d(s, redd);
    ok = ok && M[j] > -INFINITY && S[j] == S[j];
  }
  double scale[NP];
  scale[0] = 1.0;
  if (NP > 1) {
    const double al = a.alpha[row];
    ok = ok && al >= 0.0 && al <= 1.0;
    scale[0] = al / S[0];
#pragma unroll
    for (int j = 1; j < NP; ++j) scale[j] = (1.0 - al) / (NP - 1) / S[j];
  }
  if (t == 0) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      r.scale[j] = scale[j];
      r.zmax[j] = M[j];
    }
    const float u = a.u[row];
    r.u = u > 0.f ? fminf(u, 0.99999994f) : 0.f;
    r.valid = ok;
    r.mmax = 1.0;
    nlist = 0;
  }
  if (NP == 1 || !ok) return;
  auto term = [&](int i, int j) { return scale[j] * exp(st[i * 4 + j].x - (double)M[j]); };
  double lb = 0.0;
  for (int i = t; i < a.tiles; i += 256)
#pragma unroll
    for (int j = 0; j < NP; ++j) lb = fmax(lb, term(i, j));
  lb = block_max_d(lb, redd) * (1.0 - 1e-9);  // (nlist is cleared by this barrier)
  for (int i = t; i < a.tiles; i += 256) {
    double ub = 0.0;
#pragma unroll
    for (int j = 0; j < NP; ++j) ub += term(i, j);
    if (ub >= lb) list[atomicAdd(&nlist, 1)] = i;  // (the order does not matter to a maximum)
  }
  __syncthreads();
  RowState rs;
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    rs.scale[j] = scale[j];
    rs.zmax[j] = M[j];
  }
  double mx = 0.0;
  for (int n = 0; n < nlist; ++n)
    for (int i = list[n] * kTile + t; i < min(a.V, (list[n] + 1) * kTile); i += 256) {
      float z[NP];
#pragma unroll
      for (int j = 0; j < NP; ++j) z[j] = path_row<NP>(a, j, row)[i];
      mx = fmax(mx, mixture<NP>(rs, z));
    }
  mx = block_max_d(mx, redd);
  if (t == 0) r.mmax = mx;
}

// Weights of one part of a row: histogram by class and the tokens' classes, or,
// for a row without a cut, the mass that stays.
template <int NP>
__global__ __launch_bounds__(256) void k_sample_weigh(Args a) {
  __shared__ u64 mass[kClasses];
  __shared__ unsigned count[kClasses];
  const int part = blockIdx.x, row = blockIdx.y, t = threadIdx.x;
  const RowState r = a.w.state[row];
  if (!r.valid) return;
  const int lo = part * a.part, hi = min(a.V, lo + a.part);
  mass[t] = 0;
  count[t] = 0;
  __syncthreads();
  u64 kept = 0;  // no cut: kept mass; cut: mass of the low class
  unsigned low = 0;
  for (int i = lo + t; i < hi; i += 256) {
    float z[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) z[j] = path_row<NP>(a, j, row)[i];
    const u64 w = weight<NP>(r, z, a.s);
    if (!r.cut) {
      if (w >= r.least) kept += w;
      continue;
    }
    const int c = weight_class(w, a.s);
    a.w.cls[(size_t)row * a.V + i] = (uint8_t)c;
    if (c == kLow) {
      kept += w;
      ++low;
    } else if (c < kLow) {
      atomicAdd(&mass[c], w);
      atomicAdd(&count[c], 1u);
    }
  }
  const int slot = r.cut ? kLow : 0;
  kept = wave_sum64(kept);
  if ((t & 63) == 0) atomicAdd(&mass[slot], kept);
  const u64 lows = wave_sum64(low);
  if ((t & 63) == 0) atomicAdd(&count[slot], (unsigned)lows);
  __syncthreads();
  const size_t o = ((size_t)row * a.parts + part) * kClasses + t;
  if (r.cut) {
    a.w.tmass[o] = mass[t];
    a.w.tcount[o] = count[t];
  } else if (t == 0) {
    a.w.tmass[o] = mass[0];
  }
}

// The class in which the cut falls, and where each part's tokens go in the list.
__global__ __launch_bounds__(256) void k_sample_cut(Args a) {
  __shared__ u64 ms[kClasses], red[4];
  __shared__ unsigned cs[kClasses], wred[4];
  __shared__ int last_s;
  const int row = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
  RowState &r = a.w.state[row];
  if (!r.valid || !r.cut) return;
  u64 m = 0;
  unsigned c = 0;
  for (int p = 0; p < a.parts; ++p) {
    const size_t o = ((size_t)row * a.parts + p) * kClasses + t;
    m += a.w.tmass[o];
    c += a.w.tcount[o];
  }
  a.w.mass[(size_t)row * kClasses + t] = m;
  a.w.count[(size_t)row * kClasses + t] = c;
  const u64 mi = wave_scan64(m), ci = wave_scan64(c);
  if (lane == 63) {
    red[wave] = mi;
    wred[wave] = (unsigned)ci;
  }
  if (t == 0) last_s = kLow;
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
  __syncthreads();
  // the first class at which top-k, or without it top-p, is reached
  bool at;
  if (r.top_k > 0) {
    at = cs[t] >= (unsigned)r.top_k && (t == 0 || cs[t - 1] < (unsigned)r.top_k);
  } else {
    const u64 need = (u64)ceil((double)r.top_p * (double)total);
    at = ms[t] >= need && (t == 0 || ms[t - 1] < need);
  }
  if (at) last_s = min(t, kLow);
  __syncthreads();
  const int last = last_s;
  if (t == 0) {
    r.last = last;
    r.listed = (int)cs[last];
  }
  // tokens each part lists, then the exclusive sums over the parts
  unsigned *toff = a.w.toff + (size_t)row * a.parts;
  for (int p = wave; p < a.parts; p += 4) {
    const unsigned *tc = a.w.tcount + ((size_t)row * a.parts + p) * kClasses;
    u64 n = 0;
    for (int k = lane; k <= last; k += 64) n += tc[k];
    n = wave_sum64(n);
    if (lane == 0) toff[p] = (unsigned)n;
  }
  __syncthreads();
  if (wave == 0) {
    unsigned before = 0;
    for (int p0 = 0; p0 < a.parts; p0 += 64) {
      const unsigned n = p0 + lane < a.parts ? toff[p0 + lane] : 0;
      const unsigned incl = (unsigned)wave_scan64(n);
      if (p0 + lane < a.parts) toff[p0 + lane] = before + incl - n;
      before += __shfl(incl, 63, 64);
    }
  }
}

// Tokens of the classes up to the cut's, in index order, with their weights.
template <int NP>
__global__ __launch_bounds__(256) void k_sample_list(Args a) {
  __shared__ unsigned wn[4];
  const int part = blockIdx.x, row = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const RowState r = a.w.state[row];
  if (!r.valid || !r.cut) return;
  const int lo = part * a.part, hi = min(a.V, lo + a.part);
  const int q = (a.part + 3) / 4, w0 = lo + wave * q, w1 = min(hi, w0 + q);  // a wave's tokens
  const uint8_t *cls = a.w.cls + (size_t)row * a.V;
  unsigned n = 0;
  for (int i = w0; i < w1; i += 64) n += __popcll(__ballot(i + lane < w1 && cls[min(i + lane, w1 - 1)] <= r.last));
  if (lane == 0) wn[wave] = n;
  __syncthreads();
  if (n == 0) return;
  size_t at = (size_t)row * a.V + a.w.toff[(size_t)row * a.parts + part];
  for (int w = 0; w < wave; ++w) at += wn[w];
  for (int i = w0; i < w1; i += 64) {
    const bool in = i + lane < w1 && cls[min(i + lane, w1 - 1)] <= r.last;
    const u64 all = __ballot(in);
    if (in) {
      float z[NP];
#pragma unroll
      for (int j = 0; j < NP; ++j) z[j] = path_row<NP>(a, j, row)[i + lane];
      const size_t o = at + __popcll(all & ((1ull << lane) - 1));
      a.w.lw[o] = weight<NP>(r, z, a.s);
      a.w.li[o] = i + lane;
    }
    at += __popcll(all);
  }
}

struct FinalShared {
  u64 mass[256];
  unsigned count[256];
  u64 rw[kRankCap];
  int ri[kRankCap];
  u64 red[kFinal / 64];
  u64 cut_w, sum, lo, hi, need;
  int cut_i, n, found;
  unsigned inside;
};

// The index of the n-th (from 0) entry with lw == w of a list in index order.
__device__ int nth_equal(FinalShared &sh, const u64 *lw, const int *li, int n, u64 w, unsigned nth) {
  constexpr int NW = kFinal / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int seg = (n + NW - 1) / NW, s0 = wave * seg, s1 = min(n, s0 + seg);
  unsigned c = 0;
  for (int i = s0; i < s1; i += 64) c += __popcll(__ballot(i + lane < s1 && lw[min(i + lane, n - 1)] == w));
  __syncthreads();
  if (lane == 0) sh.red[wave] = c;
  __syncthreads();
  u64 before = 0;
  for (int k = 0; k < wave; ++k) before += sh.red[k];
  if (before <= nth && nth < before + c) {
    for (int i = s0; i < s1; i += 64) {
      const u64 all = __ballot(i + lane < s1 && lw[min(i + lane, n - 1)] == w);
      const int k = __popcll(all);
      if (before + k > nth) {
        const int mine = __popcll(all & ((1ull << lane) - 1));
        if (((all >> lane) & 1) && before + mine == nth) sh.cut_i = li[i + lane];
        break;
      }
      before += k;
    }
  }
  __syncthreads();
  return sh.cut_i;
}

// Where the order by (weight falling, index) is cut inside the class [lo, hi)
// of the list, after `need` of its tokens (by_mass: after the shortest run
// whose mass reaches need; the class holds as much): the last token that stays
// in sh.cut_w, sh.cut_i, the mass that stays of the class in sh.sum.  Classes of
// more than kRankCap tokens are narrowed 256-fold, by the same histogram,
// until few are left or all are equal.
__device__ void cut_class(FinalShared &sh, const u64 *lw, const int *li, int n, u64 lo, u64 hi, unsigned inside,
                          u64 need, bool by_mass) {
  const int t = threadIdx.x;
  u64 above = 0;  // mass of the class above the narrowed range
  while (inside > kRankCap && hi - lo > 1) {
    const int bits = 64 - __clzll(hi - lo - 1), shift = bits > 8 ? bits - 8 : 0;
    __syncthreads();
    if (t < 256) {
      sh.mass[t] = 0;
      sh.count[t] = 0;
    }
    __syncthreads();
    for (int i = t; i < n; i += kFinal) {
      const u64 w = lw[i];
      if (w >= lo && w < hi) {
        const int b = (int)((w - lo) >> shift);
        atomicAdd(&sh.mass[b], w);
        atomicAdd(&sh.count[b], 1u);
      }
    }
    __syncthreads();
    if (t == 0) {
      u64 left = need, ab = 0;
      int b = 255;
      for (;; --b) {
        const u64 have = by_mass ? sh.mass[b] : sh.count[b];
        if (have >= left || b == 0) break;
        left -= have;
        ab += sh.mass[b];
      }
      sh.lo = lo + ((u64)b << shift);
      sh.hi = sh.lo + (1ull << shift);
      sh.need = left;
      sh.sum = ab;
      sh.inside = sh.count[b];
    }
    __syncthreads();
    lo = sh.lo;
    hi = sh.hi < hi ? sh.hi : hi;
    need = sh.need;
    above += sh.sum;
    inside = sh.inside;
  }
  __syncthreads();
  if (inside > kRankCap) {  // equal weights: by index
    const u64 nth = by_mass ? (need + lo - 1) / lo : need;
    nth_equal(sh, lw, li, n, lo, (unsigned)nth - 1);
    if (t == 0) {
      sh.cut_w = lo;
      sh.sum = above + nth * lo;
    }
    __syncthreads();
    return;
  }
  if (t == 0) sh.n = 0;
  __syncthreads();
  for (int i = t; i < n; i += kFinal) {
    const u64 w = lw[i];
    if (w >= lo && w < hi) {
      const int k = atomicAdd(&sh.n, 1);  // (any order: ranks come from weight and index)
      if (k < kRankCap) {
        sh.rw[k] = w;
        sh.ri[k] = li[i];
      }
    }
  }
  __syncthreads();
  const int k = min(sh.n, kRankCap);
  for (int e = t; e < k; e += kFinal) {
    const u64 w = sh.rw[e];
    const int ix = sh.ri[e];
    u64 mass = 0;
    unsigned rank = 0;
    for (int o = 0; o < k; ++o)
      if (sh.rw[o] > w || (sh.rw[o] == w && sh.ri[o] < ix)) {
        mass += sh.rw[o];
        ++rank;
      }
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

// The first of n entries, in order, whose running sum of `get` exceeds u times
// their whole sum, and its share of it.  get(i): the entry's weight, 0 where
// it does not stay.
template <typename F>
__device__ void draw(FinalShared &sh, int n, float u, F get, int &found, double &share) {
  constexpr int NW = kFinal / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int seg = ((n + NW - 1) / NW + 63) / 64 * 64, s0 = min(n, wave * seg), s1 = min(n, s0 + seg);
  u64 sum = 0;
  for (int i = s0 + lane; i < s1; i += 64) sum += get(i);
  sum = wave_sum64(sum);
  __syncthreads();
  if (lane == 0) sh.red[wave] = sum;
  if (threadIdx.x == 0) sh.found = -1;
  __syncthreads();
  u64 total = 0, before = 0;
  for (int k = 0; k < NW; ++k) {
    if (k < wave) before += sh.red[k];
    total += sh.red[k];
  }
  u64 target = (u64)((double)u * (double)total);
  if (total && target >= total) target = total - 1;
  if (sum && before <= target && target < before + sum) {
    for (int i = s0; i < s1; i += 64) {
      const u64 w = i + lane < s1 ? get(i + lane) : 0;
      const u64 incl = before + wave_scan64(w);
      const u64 hit = __ballot(incl > target);
      if (hit) {
        if (lane == __ffsll(hit) - 1) {
          sh.found = i + lane;
          sh.sum = w;
        }
        break;
      }
      before = __shfl(incl, 63, 64);
    }
  }
  __syncthreads();
  found = sh.found;
  share = found < 0 ? 0.0 : (double)sh.sum / (double)total;
}

// One workgroup per row: the exact cut in its class, then the draw.
template <int NP>
__global__ __launch_bounds__(kFinal) void k_sample_final(Args a) {
  __shared__ FinalShared sh;
  const int row = blockIdx.x, t = threadIdx.x;
  const RowState r = a.w.state[row];
  int token = -1;
  double share = 0.0;
  if (r.valid && !r.cut) {
    // the part in which the draw falls, then its token
    const u64 *tm = a.w.tmass + (size_t)row * a.parts * kClasses;
    int part;
    u64 total = 0, before = 0;
    for (int p = 0; p < a.parts; ++p) total += tm[(size_t)p * kClasses];
    const float u = r.greedy ? 0.f : r.u;
    u64 target = (u64)((double)u * (double)total);
    if (target >= total) target = total - 1;
    for (part = 0; part < a.parts - 1; ++part) {
      const u64 m = tm[(size_t)part * kClasses];
      if (target < before + m) break;
      before += m;
    }
    const int lo = part * a.part, hi = min(a.V, lo + a.part);
    auto get = [&](int i) {
      float z[NP];
#pragma unroll
      for (int j = 0; j < NP; ++j) z[j] = path_row<NP>(a, j, row)[lo + i];
      const u64 w = weight<NP>(r, z, a.s);
      return w >= r.least ? w : 0;
    };
    constexpr int NW = kFinal / 64;
    const int lane = t & 63, wave = t >> 6, n = hi - lo;
    const int seg = ((n + NW - 1) / NW + 63) / 64 * 64, s0 = min(n, wave * seg), s1 = min(n, s0 + seg);
    u64 sum = 0;
    for (int i = s0 + lane; i < s1; i += 64) sum += get(i);
    sum = wave_sum64(sum);
    if (lane == 0) sh.red[wave] = sum;
    __syncthreads();
    for (int k = 0; k < wave; ++k) before += sh.red[k];
    if (before <= target && target < before + sum)
      for (int i = s0; i < s1; i += 64) {
        const u64 w = i + lane < s1 ? get(i + lane) : 0;
        const u64 incl = before + wave_scan64(w);
        const u64 hit = __ballot(incl > target);
        if (hit) {
          if (lane == __ffsll(hit) - 1) {
            a.token[row] = lo + i + lane;
            if (a.prob) a.prob[row] = r.greedy ? 1.f : (float)((double)w / (double)total);
          }
          break;
        }
        before = __shfl(incl, 63, 64);
      }
    return;
  }
  if (r.valid) {
    const u64 *lw = a.w.lw + (size_t)row * a.V;
    const int *li = a.w.li + (size_t)row * a.V;
    const u64 *mass = a.w.mass + (size_t)row * kClasses;
    const unsigned *count = a.w.count + (size_t)row * kClasses;
    u64 total = 0;           // mass of the tokens that top-k keeps
    u64 cut_w = 0;
    int cut_i = a.V;         // stays: (W > cut_w) or (W == cut_w and index <= cut_i)
    u64 lo, hi;
    if (r.top_k > 0 && (unsigned)r.listed > (unsigned)r.top_k) {
      unsigned before = 0;
      for (int c = 0; c < r.last; ++c) {
        before += count[c];
        total += mass[c];
      }
      class_range(r.last, a.s, lo, hi);
      cut_class(sh, lw, li, r.listed, lo, hi, count[r.last], (u64)r.top_k - before, false);
      total += sh.sum;
      cut_w = sh.cut_w;
      cut_i = sh.cut_i;
    } else {
      for (int c = 0; c <= (r.top_k > 0 ? r.last : kLow); ++c) total += mass[c];
    }
    if (r.top_p < 1.f) {
      u64 need = (u64)ceil((double)r.top_p * (double)total), before = 0;
      need = need < 1 ? 1 : need > total ? total : need;
      int c = 0;
      for (; c < r.last && before + mass[c] < need; ++c) before += mass[c];
      class_range(c, a.s, lo, hi);
      __syncthreads();
      cut_class(sh, lw, li, r.listed, lo, hi, count[c], need - before, true);
      cut_w = sh.cut_w;
      cut_i = sh.cut_i;
    }
    int at;
    draw(sh, r.listed, r.u, [&](int i) {
      const u64 w = lw[i];
      return w >= r.least && (w > cut_w || (w == cut_w && li[i] <= cut_i)) ? w : 0;
    }, at, share);
    token = at < 0 ? -1 : li[at];
  }
  if (t == 0) {
    a.token[row] = token;
    if (a.prob) a.prob[row] = (float)share;
  }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Parts of a row: statistics tiles, several of them together where the rows
// alone fill the chip (a part writes 3 KB of histogram, which the next kernel
// reads).
void partition(int rows, int vocab, int *tiles, int *parts, int *part) {
  *tiles = (vocab + kTile - 1) / kTile;
  int f = 1;
  while (f < 8 && (long long)rows * ((*tiles + f) / (f + 1)) >= 1024) ++f;
  *part = f * kTile;
  *parts = (vocab + *part - 1) / *part;
}

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
  x.mass = (u64 *)take(R * kClasses * 8);
  x.count = (unsigned *)take(R * kClasses * 4);
  x.toff = (unsigned *)take(R * parts * 4);
  x.cls = (uint8_t *)take(R * V);
  x.lw = (u64 *)take(R * V * 8);
  x.li = (int *)take(R * V * 4);
  if (w) *w = x;
  return o;
}

dbt_status fail(dbt_status s, const char *msg) { return set_error(s, msg); }

template <int NP> hipError_t launch(const Args &a, const dbt_sampling *p, bool cuts, hipStream_t st) {
  for (int r0 = 0; r0 < a.rows; r0 += kRowsPerCall) {
    ParamBlock pb;
    const int n = a.rows - r0 < kRowsPerCall ? a.rows - r0 : kRowsPerCall;
    for (int i = 0; i < n; ++i)
      pb.r[i] = RowParams{p[r0 + i].temperature, p[r0 + i].top_p, p[r0 + i].min_p, p[r0 + i].top_k};
    hipLaunchKernelGGL(k_sample_stats<NP>, dim3(a.tiles, n), dim3(256), 0, st, a, pb, r0);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  hipLaunchKernelGGL(k_sample_rows<NP>, dim3(a.rows), dim3(256), 0, st, a);
  if (const hipError_t e = hipGetLastError()) return e;
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
  a.nb = in->n_branches;
  a.s = 62;
  for (int v = 1; v < in->vocab; v *= 2) --a.s;  // 2^s * vocab <= 2^62
  if (a.s > 60) a.s = 60;
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
