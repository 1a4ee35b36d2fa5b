// Attention of drafted nodes over the paged cache, the nodes' row map, and the
// cache keeping one path of a tree.
//
// Node i of a sequence with `base` cached positions sees positions 0 .. base - 1
// and the slots base + a of its line: itself and its ancestors a.  A line is 64
// bits, one per node; a wave finds all of them with one lane per node by
// pointer doubling: line |= line of the node pointed at, pointer = its pointer,
// six times for lines of up to 64 nodes.
#include "attn_f32.h"
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
  const int i = blockIdx.x, lane = threadIdx.x, first = s.row[i], n = s.nodes[i];
  const uint64_t line = node_line(parents + first, n);
  if (lane < n)
    ((int4 *)rows)[first + lane] = make_int4(s.base[i] + __popcll(line) - 1, s.seq[i], -1, s.base[i] + lane);
}

// The place of query row `rho` of a sequence's nodes (node-major, then path,
// then head of the KV head) in Q and O.
struct RowPlace {
  int G, np, first, g, n_q;
  size_t path_rows;
  __device__ __forceinline__ size_t operator()(int rho) const {
    const int t = rho / G;
    return ((size_t)(t % np) * path_rows + first + t / np) * n_q + g * G + rho % G;
  }
};

// The next piece of work of run w at position s of the schedule (TreeSeqs):
// stages st0 .. st1 - 1 of the `stages` of KV head g of a sequence (seq, whose
// n nodes, rows first .., come after `base` positions).
struct Piece {
  int seq, base, first, n, g, st0, st1, stages, next;  // next: position of the next piece
  __device__ __forceinline__ bool is_whole() const { return st0 == 0 && st1 == stages; }
  // A run has at most one piece that begins inside a unit (its first) and one
  // that begins a unit without ending it (its last).
  __device__ __forceinline__ int slot(int w) const { return 2 * w + (st0 == 0); }
};
__device__ __forceinline__ int seq_rows(const TreeAttn &a, int i) { return a.s.nodes[i] * a.np * (a.n_q / a.kv.n_kv); }
__device__ __forceinline__ int stages_of(int len) { return (((len + 15) >> 4) + kTreeStagePages - 1) / kTreeStagePages; }
__device__ __forceinline__ int padded(const TreeSeqs &s, int stages) { return (stages + s.pad - 1) / s.pad * s.pad; }
__device__ __forceinline__ Piece piece_at(const TreeAttn &a, int s, int end) {
  // as many of first[0 .. n) as are at most s lie before the sequence's end,
  // counted by the wave: every lane brings one sequence's arguments (a search
  // would wait for one argument after the other)
  const int lane = threadIdx.x & 63;
  int lo = -1, first[kTreeSeqs / 64], seq[kTreeSeqs / 64], base[kTreeSeqs / 64], row[kTreeSeqs / 64], nodes[kTreeSeqs / 64];
#pragma unroll
  for (int k = 0; k < kTreeSeqs / 64; ++k) {
    first[k] = a.s.first[k * 64 + lane];
    seq[k] = a.s.seq[k * 64 + lane];
    base[k] = a.s.base[k * 64 + lane];
    row[k] = a.s.row[k * 64 + lane];
    nodes[k] = a.s.nodes[k * 64 + lane];
  }
#pragma unroll
  for (int k = 0; k < kTreeSeqs / 64; ++k) lo += __popcll(__ballot(k * 64 + lane < a.s.n && first[k] <= s));
  auto its = [&](const int (&v)[kTreeSeqs / 64]) {
    static_assert(kTreeSeqs == 128, "two sequences a lane");
    return __builtin_amdgcn_readlane(lo >= 64 ? v[1] : v[0], lo & 63);
  };
  Piece p;
  p.seq = its(seq);
  p.base = its(base);
  p.first = its(row);
  p.n = its(nodes);
  p.stages = stages_of(p.base + p.n);
  const int len = a.s.whole ? 1 : padded(a.s, p.stages), rem = s - its(first), unit = rem / len;
  p.g = unit;
  p.st0 = a.s.whole ? 0 : rem % len;
  p.st1 = a.s.whole ? p.stages : min(p.stages, p.st0 + end - s);
  p.next = s + (a.s.whole ? 1 : padded(a.s, p.st1 - p.st0));
  return p;
}
// Workgroups are dealt to the eight XCDs in turn: workgroup b takes a place that
// keeps neighbours on one XCD.  Those are the blocks of one run, which read the
// same pages at the same time: all but the first of them from the XCD's L2
// (8 x 16k-32k positions, two blocks: counters show 0.90 GB read, the cache is 0.83).
__device__ __forceinline__ int schedule_place(int b, int n) {
  const int x = b & 7, q = n >> 3, r = n & 7;
  return x * q + min(x, r) + (b >> 3);
}

typedef __attribute__((address_space(3))) void lds_void;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
constexpr int kWindow = 1024;  // pages whose ids are in LDS together

// Growth of a row's score maximum (base 2) that moves its softmax base.
constexpr float kLazyMargin = 8.f;

// bf16 cache, d_h = 128.  A workgroup of four waves, two of them a compute
// unit, owns 64 RT query rows of one (sequence, KV head) and a piece of its pages.
// Four pages a stage (32 KB) go straight into LDS, one stage ahead of the
// multiplies, so every key and value is fetched once for all rows of the
// workgroup; wave w multiplies its RT row tiles of 16 with all of them.  The
// arithmetic of a pair of pages is that of the decode kernel: scores S = K Q^T
// with permuted rows, so that lane (row r, group gq) ends up with eight
// consecutive positions of one page, which is the operand of O^T = V^T P^T; one
// running maximum and sum a row.  Rows see different keys only in pages from
// position `base` on; those pairs take a masked path.
//
// Up to 64 rows RT is 1, so that all four SIMDs have a part of them, and one
// workgroup alone reads each page: the loads' non-temporal hint takes 97 us to 91
// with 8 rows (32 x 4096 positions, eight KV heads), 112 to 103 with 64 and 109 to
// 99 over 48 x 200-4000 (whole calls, the merge with them, by events).  With RT = 2,
// which leaves two SIMDs idle, the three take 100, 112 and 115.  More rows are faster
// with two tiles a wave, whose softmax steps run side by side and which read LDS half
// as often; the hint gains nothing there (8 x 16k-32k with 128 rows: 176 and 178), and
// where several blocks share the pages in an L2 it costs 2-5 % (256 rows: 285 against
// 280, 16 x 300-1500 with 1024 rows 56 against 54).  Eight waves that also share a
// stage's pairs (merged at the end) took 107 against 111 for the 64 rows, both without
// the hint, but 142 against 111 for 48 x 200-4000, since nothing runs while the compute
// unit's one workgroup begins its next piece.
//
// Bound: up to 64 rows the memory (32 x 4096 with 64 rows: 0.54 GB read in 94 us of
// the kernel, 5.8 TB/s).  From 128 rows the matrix unit beside the softmax, whose
// steps for a pair follow each other: 16 x 300-1500 with 1024 rows 54 us for 3.1e10
// operations, 8 x 16k-32k with 256 rows 280 us for 2.1e11.
template <int RT, typename QT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_tree_attn_bf16(TreeAttn a) {
  constexpr int DH = 128, NW = 4, SP = 4, PB = 16 * DH;  // waves; pages of a stage; elements of a page
  constexpr int kOnce = RT == 1 ? 2 : 0;  // the loads' non-temporal hint
  static_assert(SP == NW && kTreeStagePages % SP == 0, "a page per wave, whole stages");
  // two sets of stage buffers, separate arrays so that the loads filling one
  // set are told apart from the reads of the other
  __shared__ __attribute__((aligned(16))) uint16_t kl0[SP * PB], vl0[SP * PB], kl1[SP * PB], vl1[SP * PB];
  __shared__ int pid_s[kWindow];
  __shared__ uint64_t line_s[kTreeNodes];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int r = lane & 15, gq = lane >> 4;
  const int n_kv = a.kv.n_kv, G = a.n_q / n_kv;
  const float scale = kLog2e / sqrtf((float)DH);
  const int place_w = schedule_place(blockIdx.x, gridDim.x), w = place_w / a.blocks, blk = place_w % a.blocks;
  const int end = min(a.s.first[a.s.n], (w + 1) * a.s.per);
  for (int at = w * a.s.per; at < end;) {
    const Piece pc = piece_at(a, at, end);
    at = pc.next;
    const int g = pc.g, first = pc.first, n = pc.n, base = pc.base, len = base + n;
    const int rows = n * a.np * G, row0 = blk * (16 * RT * NW);
    if (row0 >= rows) continue;
    const RowPlace place{G, a.np, first, g, a.n_q, a.path_rows};
    const int *ptab = a.kv.page_table + (size_t)pc.seq * a.kv.mpps;
    const int pages0 = pc.st0 * kTreeStagePages, pages1 = min((len + 15) >> 4, pc.st1 * kTreeStagePages);  // the piece's pages
    int pb = pages0, npg = min(pages1 - pb, kWindow);  // the window's first page, its pages
    __syncthreads();  // (the last piece's readers)

    // K row j of a page holds its 16-byte chunk c at c ^ kswz(j): the score operand
    // reads rows {0..3, 8..11} (or {4..7, 12..15}) of both pages at one chunk
    // without bank conflicts.  V rows (one dimension, 32 bytes) need no swizzle.
    auto kswz = [](int row) { return ((row & 3) | ((row >> 3) << 2)) << 1; };
    const uint16_t *kbase = (const uint16_t *)a.kv.k, *vbase = (const uint16_t *)a.kv.v;
    // A stage is eight loads of 1 KB a page, four of K and four of V: each wave
    // takes one page.  Pages past the piece's last re-read it (never used unmasked).
    auto dma = [&](int id, uint16_t *kb, uint16_t *vb) __attribute__((always_inline)) {
      const size_t at = ((size_t)__builtin_amdgcn_readfirstlane(id) * n_kv + g) * PB;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = 4 * j + (lane >> 4);
        __builtin_amdgcn_global_load_lds((const void *)(kbase + at + row * DH + ((lane & 15) ^ kswz(row)) * 8),
                                         (lds_void *)(kb + wave * PB + 4 * j * DH), 16, 0, kOnce);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        __builtin_amdgcn_global_load_lds((const void *)(vbase + at + 32 * j * 16 + lane * 8),
                                         (lds_void *)(vb + wave * PB + 32 * j * 16), 16, 0, kOnce);
    };
    auto next = [&](int st, uint16_t *kb, uint16_t *vb) __attribute__((always_inline)) {
      dma(pid_s[min(st * SP + wave, npg - 1)], kb, vb);
    };
    // Start: each wave finds its first stages' pages by itself and sends for them
    // (for two stages where the piece is so short that the wait for each is a large
    // part of its time); the other page ids, the lines and the queries come in
    // meanwhile.  The first stage's barrier shows all of them.
    const int wrow = row0 + wave * RT * 16;  // the wave's first row
    const int id0 = ptab[pb + min(wave, npg - 1)], id1 = ptab[pb + min(SP + wave, npg - 1)];
    dma(id0, kl0, vl0);
    const int sent = npg > SP && npg <= 4 * SP ? 2 : 1;  // stages sent for
    if (sent == 2) dma(id1, kl1, vl1);
    for (int k = t; k < npg; k += 64 * NW) pid_s[k] = ptab[pb + k];
    if (wave == 0) line_s[lane] = node_line(a.parents + first, n);
    constexpr int QW = sizeof(QT) / 2;
    int node[RT];
    u32x4 raw[RT][4][QW];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int rho = wrow + rt * 16 + r, own = rho < rows ? rho : 0;
      node[rt] = own / (G * a.np);
      const u32x4 *qp = (const u32x4 *)((const QT *)a.Q + place(own) * DH + gq * 8);
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int h = 0; h < QW; ++h) raw[rt][s][h] = qp[s * 4 * QW + h];
    }
    u32x4 qf[RT][4];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if constexpr (QW == 1) {
          qf[rt][s] = raw[rt][s][0];
        } else {  // the projections' queries, rounded once to the cache's type as in a step
          const float4 x = __builtin_bit_cast(float4, raw[rt][s][0]), y = __builtin_bit_cast(float4, raw[rt][s][1]);
          qf[rt][s] = u32x4{pack2(x.x, x.y), pack2(x.z, x.w), pack2(y.x, y.y), pack2(y.z, y.w)};
        }
      }

    float m_run[RT];
    floatx4 acc[RT][8], acc_l[RT];  // acc_l: the sums of the rounded probabilities, by one more value multiply with V = 1
    const u32x4 ones = u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m_run[rt] = kNoScore;
      acc_l[rt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[rt][c] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const int kpage = r >> 3, kpos = 8 * ((r >> 2) & 1) + (r & 3);
    const int vpage = gq >> 1, vpos = 8 * (gq & 1);
    const bool active = wrow < rows;
    bool odd = false;  // some node's value is not finite

    auto pair = [&](int pg0, const uint16_t *kb, const uint16_t *vb, auto masked) __attribute__((always_inline)) {
      constexpr bool MASKED = decltype(masked)::value;
      u32x4 ka[4], kc[4], vf[8];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        ka[s] = *(const u32x4 *)&kb[(kpage * 16 + kpos) * DH + ((s * 4 + gq) ^ kswz(kpos)) * 8];
        kc[s] = *(const u32x4 *)&kb[(kpage * 16 + kpos + 4) * DH + ((s * 4 + gq) ^ kswz(kpos + 4)) * 8];
      }
      floatx4 sc[RT][2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        sc[rt][0] = sc[rt][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          sc[rt][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ka[s]),
                                                              __builtin_bit_cast(bf16x8, qf[rt][s]), sc[rt][0], 0, 0, 0);
          sc[rt][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kc[s]),
                                                              __builtin_bit_cast(bf16x8, qf[rt][s]), sc[rt][1], 0, 0, 0);
        }
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) vf[c] = *(const u32x4 *)&vb[(vpage * DH + c * 16 + r) * 16 + vpos];
      const int kp0 = (pb + pg0 + vpage) * 16 + vpos;  // position of this lane's first score
      const bool page_ok = pg0 + vpage < npg;
      if (MASKED) {
        if ((pb + pg0 + 2) * 16 > len) {  // slots past the sequence may hold anything
#pragma unroll
          for (int c = 0; c < 8; ++c) vf[c] = mask8(vf[c], kp0, page_ok ? len : kp0);
        }
        // a node's values that are not finite would reach the rows that do not
        // see it as 0 * infinity, so they are taken out here and added at the end
        u16x2 top = {0, 0};
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int w = 0; w < 4; ++w) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[c][w] & 0x7fff7fffu));
        if (__any(top.x >= 0x7f80 || top.y >= 0x7f80)) {
#pragma unroll
          for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const uint32_t x = vf[c][w];
              const bool lo = (x & 0x7f80u) == 0x7f80u && kp0 + 2 * w >= base;
              const bool hi = (x & 0x7f800000u) == 0x7f800000u && kp0 + 2 * w + 1 >= base;
              odd |= lo | hi;
              vf[c][w] = x & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
            }
        }
      }
      // (the row tiles' steps side by side: one tile alone leaves the units waiting
      // for its chain of maximum, exponentials and conversion)
      float s[RT][8], m_new[RT];
      bool grow = false;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[rt][e] = sc[rt][0][e];
          s[rt][4 + e] = sc[rt][1][e];
        }
        if (MASKED) {  // the row's eight positions: before `base`, or on its line
          const int rel = kp0 - base;
          const uint64_t line = line_s[node[rt]];
          const uint32_t seen = !page_ok || rel >= 64 ? 0u
                                : rel >= 0            ? (uint32_t)(line >> rel) & 0xff
                                : rel > -8            ? (uint32_t)((line << -rel) | ((1u << -rel) - 1)) & 0xff
                                                      : 0xffu;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!((seen >> e) & 1)) s[rt][e] = -INFINITY;
        }
        float mt = s[rt][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mt = fmaxf(mt, s[rt][e]);
        // lazy rescaling: a row's base moves only when the pair's maximum exceeds it
        // by more than kLazyMargin, so exponentials stay <= 2^kLazyMargin
        const float mt_s = rows4_max(mt) * scale;
        const bool up = mt_s > m_run[rt] + kLazyMargin;
        m_new[rt] = up ? mt_s : m_run[rt];
        grow |= up;
      }
      if (__any(grow)) {  // (a factor of exactly 1 where the base stays)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const float corr = __builtin_amdgcn_exp2f(m_run[rt] - m_new[rt]);
          acc_l[rt] = acc_l[rt] * corr;
#pragma unroll
          for (int c = 0; c < 8; ++c) acc[rt][c] = acc[rt][c] * corr;
          m_run[rt] = m_new[rt];
        }
      }
      u32x4 pf[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(s[rt][e], scale, -m_new[rt]));
        // (probabilities are rounded to bf16 for the matrix unit; their sum is of the rounded ones)
        pf[rt] = u32x4{pack2(p[0], p[1]), pack2(p[2], p[3]), pack2(p[4], p[5]), pack2(p[6], p[7])};
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        acc_l[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones),
                                                            __builtin_bit_cast(bf16x8, pf[rt]), acc_l[rt], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < 8; ++c)
          acc[rt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[c]),
                                                               __builtin_bit_cast(bf16x8, pf[rt]), acc[rt][c], 0, 0, 0);
      }
    };
    auto stage = [&](int st, const uint16_t *kb, const uint16_t *vb, auto masked) __attribute__((always_inline)) {
      if (!active) return;
#pragma unroll 1
      for (int j = 0; j < SP / 2; ++j) {
        const int pg0 = st * SP + 2 * j;
        if (decltype(masked)::value && pg0 >= npg) break;
        pair(pg0, kb + 2 * j * PB, vb + 2 * j * PB, masked);
      }
    };
    // The barrier in front of a stage waits for its loads and for the readers of
    // the other set, which the next stage's loads then fill.  Stages of which
    // every row sees every key first, in pairs so that each set is known; then
    // the last ones, those from the page of position `base` on.
    for (;;) {
      const int nst = (npg + SP - 1) / SP, nfull = max(0, min(npg, (base >> 4) - pb)) / SP;
      for (int st = 0; st < nfull; st += 2) {
        stage_barrier();
        if (st + 1 >= sent && st + 1 < nst) next(st + 1, kl1, vl1);
        __builtin_amdgcn_sched_barrier(0);
        stage(st, kl0, vl0, std::false_type{});
        if (st + 1 < nfull) {
          stage_barrier();
          if (st + 2 < nst) next(st + 2, kl0, vl0);
          __builtin_amdgcn_sched_barrier(0);
          stage(st + 1, kl1, vl1, std::false_type{});
        }
      }
#pragma unroll 1
      for (int st = nfull; st < nst; ++st) {
        stage_barrier();
        const bool set1 = st & 1;
        if (st + 1 >= sent && st + 1 < nst) next(st + 1, set1 ? kl0 : kl1, set1 ? vl0 : vl1);
        stage(st, set1 ? kl1 : kl0, set1 ? vl1 : vl0, std::true_type{});
      }
      pb += kWindow;
      if (pb >= pages1) break;
      npg = min(pages1 - pb, kWindow);
      __syncthreads();
      for (int k = t; k < npg; k += 64 * NW) pid_s[k] = ptab[pb + k];
      __syncthreads();
      next(0, kl0, vl0);
    }

    if (__any(odd)) {
      // such values make the sums of the rows that see them infinite or NaN,
      // whatever their weights
      for (int pos = max(base, pages0 * 16); pos < min(len, pages1 * 16); ++pos) {
        const uint16_t *v = vbase + ((size_t)ptab[pos >> 4] * n_kv + g) * PB + (pos & 15);
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint16_t x = v[(16 * c + 4 * gq + d) * 16];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              if ((x & 0x7f80) == 0x7f80 && ((line_s[node[rt]] >> (pos - base)) & 1)) acc[rt][c][d] += bf2f(x);
          }
      }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int rho = wrow + rt * 16 + r;
      if (rho >= rows) continue;
      if (pc.is_whole()) {
        const float inv = 1.f / acc_l[rt][0];
        uint16_t *o = (uint16_t *)a.O + place(rho) * DH + 4 * gq;
#pragma unroll
        for (int c = 0; c < 8; ++c)
          *(u32x2 *)(o + 16 * c) = u32x2{pack2(acc[rt][c][0] * inv, acc[rt][c][1] * inv), pack2(acc[rt][c][2] * inv, acc[rt][c][3] * inv)};
      } else {
        const size_t to = ((size_t)pc.slot(w) * a.blocks + blk) * a.block + rho - row0;
#pragma unroll
        for (int c = 0; c < 8; ++c)
          *(float4 *)(a.opart + to * DH + 16 * c + 4 * gq) = make_float4(acc[rt][c][0], acc[rt][c][1], acc[rt][c][2], acc[rt][c][3]);
        if (gq == 0) *(float2 *)(a.ostat + to * 2) = make_float2(m_run[rt], acc_l[rt][0]);
      }
    }
  }
}

// fp32 cache: blocks of sixteen query rows, on the fp32 matrix instruction
// (attn_f32.h).
template <int NC>
__global__ __launch_bounds__(64 * kWavesF32Attn) void k_tree_attn_f32(TreeAttn a) {
  __shared__ F32Merge<NC> mg;
  __shared__ uint64_t line_s[kTreeNodes];
  const int G = a.n_q / a.kv.n_kv, DH = a.kv.d_h;
  const int place_w = schedule_place(blockIdx.x, gridDim.x), w = place_w / a.blocks, blk = place_w % a.blocks;
  const int end = min(a.s.first[a.s.n], (w + 1) * a.s.per);
  for (int s = w * a.s.per; s < end;) {
    const Piece pc = piece_at(a, s, end);
    s = pc.next;
    const int g = pc.g, first = pc.first, n = pc.n, base = pc.base, len = base + n;
    const int rows = n * a.np * G, row0 = blk * 16;
    if (row0 >= rows) continue;
    const RowPlace place{G, a.np, first, g, a.n_q, a.path_rows};
    __syncthreads();  // (the last piece's readers)
    if (threadIdx.x < 64) line_s[threadIdx.x] = node_line(a.parents + first, n);
    __syncthreads();
    const int rho = row0 + (threadIdx.x & 15);
    const bool live = rho < rows;
    const SeesLine sees{base, live ? line_s[rho / (G * a.np)] : 0};
    attn_f32<NC>(mg, (const float *)a.Q + place(live ? rho : 0) * DH, live, sees, base >> 4, len, (const float *)a.kv.k,
                 (const float *)a.kv.v, a.kv.page_table + (size_t)pc.seq * a.kv.mpps, pc.st0 * kTreeStagePages,
                 min((len + 15) >> 4, pc.st1 * kTreeStagePages), a.kv.n_kv, g, DH);
    for (int e = threadIdx.x; e < min(16, rows - row0) * DH; e += 64 * kWavesF32Attn) {
      const int qr = e / DH, dh = e % DH;
      float o, l, mx;
      mg.merged(qr, dh, o, l, mx);
      if (pc.is_whole()) {
        ((float *)a.O)[place(row0 + qr) * DH + dh] = o / l;
      } else {
        const size_t at = ((size_t)pc.slot(w) * a.blocks + blk) * 16 + qr;
        a.opart[at * DH + dh] = o;
        if (dh == 0) *(float2 *)(a.ostat + at * 2) = make_float2(mx, l);
      }
    }
  }
}

// The pieces of every cut unit merged in order: one thread per (query row, four
// dimensions).
template <typename T>
__global__ __launch_bounds__(256) void k_tree_combine(TreeAttn a) {
  const int i = blockIdx.z, g = blockIdx.y, DH = a.kv.d_h, Q4 = DH / 4;
  const int first = a.s.row[i], rows = seq_rows(a, i), stages = stages_of(a.s.base[i] + a.s.nodes[i]);
  const int e = blockIdx.x * 256 + threadIdx.x, rho = e / Q4, d4 = e % Q4;
  if (rho >= rows) return;
  const int s0 = a.s.first[i] + g * padded(a.s, stages);
  const int w0 = s0 / a.s.per, w1 = (s0 + stages - 1) / a.s.per;
  if (w0 == w1) return;  // written whole
  const RowPlace place{a.n_q / a.kv.n_kv, a.np, first, g, a.n_q, a.path_rows};
  // run w's piece begins the unit only for w0
  auto row = [&](int w) { return (size_t)(2 * w + (w == w0)) * a.blocks * a.block + rho; };
  // eight pieces at a time, all of their loads in flight together
  float mx = kNoScore, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int w = w0; w <= w1; w += 8) {
    float2 ml[8];
    float4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const size_t at = row(min(w + k, w1));
      ml[k] = *(const float2 *)(a.ostat + at * 2);
      v[k] = ((const float4 *)(a.opart + at * DH))[d4];
    }
    float mn = mx;
#pragma unroll
    for (int k = 0; k < 8; ++k) mn = fmaxf(mn, ml[k].x);
    const float f0 = exp2f(mx - mn);
    o = make_float4(o.x * f0, o.y * f0, o.z * f0, o.w * f0);
    l *= f0;
    mx = mn;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (w + k > w1) break;
      const float f = exp2f(ml[k].x - mx);
      o.x += v[k].x * f;
      o.y += v[k].y * f;
      o.z += v[k].z * f;
      o.w += v[k].w * f;
      l += ml[k].y * f;
    }
  }
  T *out = (T *)a.O + place(rho) * DH + d4 * 4;
  st<T>(out, 0, o.x / l);
  st<T>(out, 1, o.y / l);
  st<T>(out, 2, o.z / l);
  st<T>(out, 3, o.w / l);
}

// The kept nodes' keys and values of one (layer, KV head, sequence): all read
// into LDS, then all written, since one node's new slot can be another's old
// one.  K rows move as 16-byte pieces; a value dimension's 16 slots are
// adjacent, so neighbouring threads take neighbouring nodes of one dimension.
template <typename T>
__global__ __launch_bounds__(256) void k_tree_keep(KeepSeqs s, KVRef kv, size_t layer_elems) {
  constexpr int EP = 16 / sizeof(T);
  __shared__ __attribute__((aligned(16))) T ks[kTreeNodes * 128], vs[kTreeNodes * 128];
  __shared__ size_t block[2 * kTreeNodes];
  __shared__ int slot[2 * kTreeNodes];
  const int g = blockIdx.x, i = blockIdx.z, t = threadIdx.x, DH = kv.d_h, pr = DH / EP;
  const int j0 = s.first[i], n = s.count[i] - j0, base = s.base[i];
  T *k = (T *)kv.k + blockIdx.y * layer_elems, *v = (T *)kv.v + blockIdx.y * layer_elems;
  if (t < 2 * n) {  // the nodes' places: old ones, then new ones
    const int j = t < n ? t : t - n, pos = base + (t < n ? s.path[i][j0 + j] : j0 + j);
    const int page = kv.page_table[(size_t)s.seq[i] * kv.mpps + (pos >> 4)];
    block[t] = ((size_t)page * kv.n_kv + g) * 16 * DH;
    slot[t] = pos & 15;
  }
  __syncthreads();
  auto krow = [&](int j) { return (u32x4 *)(k + block[j] + slot[j] * DH); };
  auto vcol = [&](int j) { return v + block[j] + slot[j]; };
#pragma unroll 4
  for (int e = t; e < n * pr; e += 256) ((u32x4 *)ks)[e] = krow(e / pr)[e % pr];
#pragma unroll 4
  for (int e = t; e < n * DH; e += 256) vs[e] = vcol(e % n)[(e / n) * 16];
  __syncthreads();
#pragma unroll 4
  for (int e = t; e < n * pr; e += 256) krow(n + e / pr)[e % pr] = ((const u32x4 *)ks)[e];
#pragma unroll 4
  for (int e = t; e < n * DH; e += 256) vcol(n + e % n)[(e / n) * 16] = vs[e];
}

}  // namespace

hipError_t launch_tree_rows(const TreeSeqs &s, const int *parents, PromptRow *rows, hipStream_t st) {
  hipLaunchKernelGGL(k_tree_rows, dim3(s.n), dim3(64), 0, st, s, parents, rows);
  return hipGetLastError();
}

hipError_t launch_tree_attn(const TreeAttn &a, hipStream_t st) {
  const int rows = a.max_nodes * a.np * (a.n_q / a.kv.n_kv);
  if (a.s.n < 1 || a.s.n > kTreeSeqs || a.max_nodes < 1 || a.max_nodes > kTreeNodes || a.s.per < 1 || a.s.pad < 1 ||
      a.block != tree_block_rows(rows, a.dtype) || a.blocks != (rows + a.block - 1) / a.block || (!a.s.whole && (!a.opart || !a.ostat)))
    return hipErrorInvalidValue;
  const dim3 grid((a.s.first[a.s.n] + a.s.per - 1) / a.s.per * a.blocks);
  if (a.dtype == 1) {
    if (a.kv.d_h != 128) return hipErrorInvalidValue;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
    if (a.q32)
      a.block == 64 ? go(k_tree_attn_bf16<1, float>) : go(k_tree_attn_bf16<2, float>);
    else
      a.block == 64 ? go(k_tree_attn_bf16<1, uint16_t>) : go(k_tree_attn_bf16<2, uint16_t>);
  } else {
    if (a.kv.d_h > 128) return hipErrorInvalidValue;
    const dim3 block(64 * kWavesF32Attn);
    switch ((a.kv.d_h + 15) / 16) {
      case 1: hipLaunchKernelGGL(k_tree_attn_f32<1>, grid, block, 0, st, a); break;
      case 2: hipLaunchKernelGGL(k_tree_attn_f32<2>, grid, block, 0, st, a); break;
      case 3: hipLaunchKernelGGL(k_tree_attn_f32<3>, grid, block, 0, st, a); break;
      case 4: hipLaunchKernelGGL(k_tree_attn_f32<4>, grid, block, 0, st, a); break;
      case 5: hipLaunchKernelGGL(k_tree_attn_f32<5>, grid, block, 0, st, a); break;
      case 6: hipLaunchKernelGGL(k_tree_attn_f32<6>, grid, block, 0, st, a); break;
      case 7: hipLaunchKernelGGL(k_tree_attn_f32<7>, grid, block, 0, st, a); break;
      default: hipLaunchKernelGGL(k_tree_attn_f32<8>, grid, block, 0, st, a); break;
    }
  }
  if (const hipError_t e = hipGetLastError()) return e;
  if (!a.s.whole) {
    const dim3 cgrid((rows * (a.kv.d_h / 4) + 255) / 256, a.kv.n_kv, a.s.n);
    if (a.dtype == 1)
      hipLaunchKernelGGL(k_tree_combine<uint16_t>, cgrid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(k_tree_combine<float>, cgrid, dim3(256), 0, st, a);
  }
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
