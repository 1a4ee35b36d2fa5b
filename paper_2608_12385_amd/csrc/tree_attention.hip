// Attention of drafted nodes over the paged cache, the nodes' row map, and the
// cache keeping one path of a tree.
//
// Node i of a sequence with `base` cached positions sees positions 0 .. base - 1
// and the slots base + a of its line: itself and its ancestors a.  A line is 64
// bits, one per node; a wave finds all of them with one lane per node by
// pointer doubling: line |= line of the node pointed at, pointer = its pointer,
// six times for lines of up to 64 nodes.
#include "common.h"
#include "kernels.h"

namespace dbt {

namespace {

// Lines of the n nodes of a sequence, by a whole wave: lane i's bit set of node
// i and its ancestors (0 for lanes past the nodes).
__device__ __forceinline__ uint64_t node_line(const int *parents, int n) {
  const int lane = threadIdx.x & 63;
  int up = lane < n ? parents[lane] : -1;
  if (up < 0 || up >= lane) up = lane;  // a root points at itself
  uint64_t line = lane < n ? 1ull << lane : 0;
#pragma unroll
  for (int k = 0; k < 6; ++k) {
    line |= __shfl(line, up, 64);
    up = __shfl(up, up, 64);
  }
  return line;
}

__global__ __launch_bounds__(64) void k_tree_rows(TreeSeqs s, const int *parents, PromptRow *rows) {
  const int i = blockIdx.x, lane = threadIdx.x, first = s.off[i], n = s.off[i + 1] - first;
  const uint64_t line = node_line(parents + first, n);
  if (lane < n)
    ((int4 *)rows)[first + lane] = make_int4(s.base[i] + __popcll(line) - 1, s.seq[i], -1, s.base[i] + lane);
}

// One workgroup per (query row, query head): scores of 256 keys at a time, one
// per thread, online softmax over the groups, values summed by dimension.
template <typename T, typename QT>
__global__ __launch_bounds__(256) void k_tree_attn_simple(TreeAttn a) {
  const int i = blockIdx.z, head = blockIdx.y, t = threadIdx.x;
  const int first = a.s.off[i], n = a.s.off[i + 1] - first;
  const int node = blockIdx.x / a.np, path = blockIdx.x % a.np;
  if (node >= n) return;
  const int DH = a.kv.d_h, base = a.s.base[i], len = base + n, g = head / (a.n_q / a.kv.n_kv);
  __shared__ float q_s[128], p_s[256], red[16];
  __shared__ uint64_t line_s;
  const uint64_t line = t < 64 ? node_line(a.parents + first, n) : 0;
  if (t == node) line_s = line;
  const size_t row = ((size_t)path * a.path_rows + first + node) * a.n_q + head;
  if (t < DH) q_s[t] = ld<QT>((const QT *)a.Q, row * DH + t) * (kLog2e / sqrtf((float)DH));
  __syncthreads();
  const int *ptab = a.kv.page_table + (size_t)a.s.seq[i] * a.kv.mpps;
  auto sees = [&](int pos) { return pos < base || (pos < len && ((line_s >> (pos - base)) & 1)); };
  float m = kNoScore, l = 0.f, o = 0.f;
  for (int p0 = 0; p0 < len; p0 += 256) {
    const int pos = p0 + t;
    float s = -INFINITY;
    if (pos < len && sees(pos)) {
      const T *k = (const T *)a.kv.k + (((size_t)ptab[pos >> 4] * a.kv.n_kv + g) * 16 + (pos & 15)) * DH;
      s = 0.f;
      for (int d = 0; d < DH; ++d) s = fmaf(q_s[d], ld<T>(k, d), s);
    }
    const float mn = fmaxf(m, block_max(s, red)), f = exp2f(m - mn), p = exp2f(s - mn);
    p_s[t] = p;
    l = l * f + block_sum(p, red);
    o *= f;
    m = mn;
    if (t < DH)
      for (int j = 0; j < min(256, len - p0); ++j)
        if (sees(p0 + j))
          o += p_s[j] * ld<T>((const T *)a.kv.v, (((size_t)ptab[(p0 + j) >> 4] * a.kv.n_kv + g) * DH + t) * 16 + ((p0 + j) & 15));
    __syncthreads();
  }
  if (t < DH) st<T>((T *)a.O, row * DH + t, o / l);
}

// The kept nodes' keys and values of one (layer, KV head, sequence): all read
// into LDS, then all written, since one node's new slot can be another's old
// one.  K rows move as 16-byte pieces; a value dimension's 16 slots are
// adjacent, so neighbouring threads take neighbouring nodes of one dimension.
template <typename T>
__global__ __launch_bounds__(256) void k_tree_keep(KeepSeqs s, KVRef kv, size_t layer_elems) {
  constexpr int EP = 16 / sizeof(T);
  __shared__ __attribute__((aligned(16))) T ks[kTreeNodes * 128], vs[kTreeNodes * 128];
  const int g = blockIdx.x, i = blockIdx.z, t = threadIdx.x, DH = kv.d_h, pr = DH / EP;
  const int j0 = s.first[i], n = s.count[i] - j0, base = s.base[i];
  const int *ptab = kv.page_table + (size_t)s.seq[i] * kv.mpps;
  T *k = (T *)kv.k + blockIdx.y * layer_elems, *v = (T *)kv.v + blockIdx.y * layer_elems;
  auto krow = [&](int pos) { return k + (((size_t)ptab[pos >> 4] * kv.n_kv + g) * 16 + (pos & 15)) * DH; };
  auto vcol = [&](int pos) { return v + ((size_t)ptab[pos >> 4] * kv.n_kv + g) * DH * 16 + (pos & 15); };
  for (int e = t; e < n * pr; e += 256)
    ((u32x4 *)ks)[e] = ((const u32x4 *)krow(base + s.path[i][j0 + e / pr]))[e % pr];
  for (int e = t; e < n * DH; e += 256) vs[e] = vcol(base + s.path[i][j0 + e % n])[(e / n) * 16];
  __syncthreads();
  for (int e = t; e < n * pr; e += 256) ((u32x4 *)krow(base + j0 + e / pr))[e % pr] = ((const u32x4 *)ks)[e];
  for (int e = t; e < n * DH; e += 256) vcol(base + j0 + e % n)[(e / n) * 16] = vs[e];
}

}  // namespace

hipError_t launch_tree_rows(const TreeSeqs &s, const int *parents, PromptRow *rows, hipStream_t st) {
  hipLaunchKernelGGL(k_tree_rows, dim3(s.n), dim3(64), 0, st, s, parents, rows);
  return hipGetLastError();
}

hipError_t launch_tree_attn(const TreeAttn &a, hipStream_t st) {
  if (a.kv.d_h > 128 || a.s.n < 1) return hipErrorInvalidValue;
  const dim3 grid(a.max_nodes * a.np, a.n_q, a.s.n);
  if (a.dtype == 1 && a.q32)
    hipLaunchKernelGGL((k_tree_attn_simple<uint16_t, float>), grid, dim3(256), 0, st, a);
  else if (a.dtype == 1)
    hipLaunchKernelGGL((k_tree_attn_simple<uint16_t, uint16_t>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_tree_attn_simple<float, float>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_tree_keep(const KeepSeqs &s, const KVRef &kv, int n_layers, size_t layer_elems, int dtype,
                            hipStream_t st) {
  if (s.n < 1) return hipSuccess;
  if (kv.d_h > 128 || (dtype == 1 && kv.d_h % 8)) return hipErrorInvalidValue;
  const dim3 grid(kv.n_kv, n_layers, s.n);
  if (dtype == 1)
    hipLaunchKernelGGL(k_tree_keep<uint16_t>, grid, dim3(256), 0, st, s, kv, layer_elems);
  else
    hipLaunchKernelGGL(k_tree_keep<float>, grid, dim3(256), 0, st, s, kv, layer_elems);
  return hipGetLastError();
}

}  // namespace dbt
