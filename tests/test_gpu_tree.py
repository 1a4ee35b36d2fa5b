"""Drafted tokens on the GPU: attention of a tree over the paged cache against
float64, the grouped step over a tree against the oracle run along every line of
it, and the cache keeping a path."""
import dataclasses

import numpy as np
import pytest

import synth
from oracle import Oracle
from tests.gpu_util import check_readout, fill_cache, make_session, row_err, to_np
from tests.tiny import tiny_shape

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32_TOL, BF16_TOL = 1e-5, 2e-2  # whole steps, as for the ordinary step


def lines(parents):
    """Every node's line, itself first."""
    out = []
    for i, p in enumerate(parents):
        out.append([i] + (out[p] if 0 <= p < i else []))
    return out


def random_tree(rng, n):
    return [int(rng.integers(-1, i)) if rng.random() < 0.9 else i - 1 for i in range(n)]


class Cache:
    """A one-layer model's cache filled with given K/V, sequences grown in turns."""

    def __init__(self, dtype, nq, nkv, dh, totals, branches=1, seed=0, layers=1, spread=1.0):
        from paper_2608_12385_amd import binding
        self.B = binding
        rng = np.random.default_rng(seed)
        f32 = dtype == "f32"
        self.shape = synth.ModelShape(n_layers=layers, d_model=128, n_q_heads=nq, n_kv_heads=nkv, head_dim=dh, d_ff=128,
                                      vocab=0, dtype=dtype, has_embeddings=False, n_branches=branches)
        self.W = synth.make_weights(self.shape, seed=0)
        self.sess = make_session(self.shape, self.W, max_batch=len(totals), max_pos=max(max(totals), 1) + 80)
        self.tt = torch.float32 if f32 else torch.bfloat16
        self.totals = totals
        kv = self.sess.kv
        for b, n in enumerate(totals):
            if n // 2:
                binding.dbt_kv_reserve(kv, b, n // 2)
        for b, n in reversed(list(enumerate(totals))):
            if n:
                binding.dbt_kv_reserve(kv, b, n)
        # whatever lies past the ends must not matter
        for p in (self.sess.k_pages, self.sess.v_pages):
            p.view(self.tt).fill_(float("nan"))
        self.K = [[torch.from_numpy((spread * rng.standard_normal((n, nkv, dh))).astype(np.float32)).to(self.tt)
                   for n in totals] for _ in range(layers)]
        self.V = [[torch.from_numpy(rng.standard_normal((n, nkv, dh)).astype(np.float32)).to(self.tt) for n in totals]
                  for _ in range(layers)]

    def fill(self):
        for l in range(len(self.K)):
            for b, n in enumerate(self.totals):
                if n:
                    k, v = self.K[l][b].cuda(), self.V[l][b].cuda()
                    self.B.dbt_kv_fill(self.sess.kv, l, b, 0, n, k.data_ptr(), v.data_ptr(), self.sess.stream)
                    torch.cuda.synchronize()

    def attend(self, nodes, parents, q, layer=0, stream=None):
        up = torch.tensor(parents, dtype=torch.int32, device="cuda")
        qd, n = q.cuda(), sum(nodes)
        out = torch.full_like(qd, 7.0)
        ws = torch.full((self.B.dbt_tree_workspace_bytes(self.sess.cfg, n),), 0xff, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        self.B.dbt_tree_attention(self.sess.kv, layer, self.B.make_tree(nodes, up.data_ptr()), q.shape[0],
                                  qd.data_ptr(), out.data_ptr(), ws.data_ptr(), stream or self.sess.stream)
        torch.cuda.synchronize()
        return out.cpu()


def reference(c, nodes, parents, q, layer=0):
    """Outputs in float64 and what a correct kernel may be off by: bf16 rounds
    every probability (2^-8, also where they are summed) and the output (2^-8),
    fp32 the scores (d + 2 products' roundings) and the sums."""
    s = c.shape
    G, dh = s.n_q_heads // s.n_kv_heads, s.head_dim
    P, _, nq, _ = q.shape
    qd = q.double()
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    first = 0
    for b, n in enumerate(nodes):
        L = c.totals[b] - n
        for i, line in enumerate(lines(parents[first:first + n])):
            pos = list(range(L)) + sorted(L + j for j in line)
            k, v = c.K[layer][b][pos].double(), c.V[layer][b][pos].double()
            for h in range(nq):
                kh, vh = k[:, h // G], v[:, h // G]
                z = qd[:, first + i, h] @ kh.T / dh ** 0.5
                w = torch.softmax(z, -1)
                o, a = w @ vh, w @ vh.abs()
                out[:, first + i, h] = o
                if s.dtype == "bf16":
                    t = 2.0 ** -8 * o.abs() + 2.02 * 2.0 ** -8 * a
                else:
                    zs = (qd[:, first + i, h].abs() @ kh.T.abs() / dh ** 0.5).amax(-1, keepdim=True)
                    t = (2 * (dh + 2) * zs + len(pos) + 16) * 2.0 ** -24 * a
                tol[:, first + i, h] = t + 1e-30
        first += n
    return out, tol


def check(c, nodes, parents, paths, seed=1, layer=0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((paths, sum(nodes), c.shape.n_q_heads, c.shape.head_dim), generator=g).to(c.tt)
    got = c.attend(nodes, parents, q, layer)
    ref, tol = reference(c, nodes, parents, q, layer)
    off = (got.double() - ref).abs() / tol
    assert bool((off <= 1).all()), float(off.max())
    assert torch.equal(got, c.attend(nodes, parents, q, layer))
    return q, got


CASES = [
    # dtype, query heads, KV heads, d, branches, paths, positions before the nodes, nodes
    ("bf16", 32, 8, 128, 1, 2, [777], [12]),
    ("bf16", 4, 1, 128, 1, 1, [0, 1, 15, 16, 17, 33], [1, 64, 3, 0, 16, 5]),
    ("bf16", 16, 4, 128, 3, 4, [100, 31, 32, 5], [64, 63, 17, 2]),
    ("bf16", 8, 1, 128, 1, 2, [250, 1000], [33, 40]),
    ("bf16", 1, 1, 128, 1, 2, [2, 500], [1, 9]),
    ("bf16", 3, 1, 128, 2, 3, [47, 300], [7, 20]),
    ("bf16", 5, 5, 128, 1, 1, [129], [30]),
    ("bf16", 4, 2, 128, 1, 2, [5000, 700, 64], [4, 30, 1]),
    ("f32", 4, 4, 64, 1, 2, [33, 137, 0], [3, 20, 64]),
    ("f32", 8, 2, 16, 3, 4, [15, 16, 300], [1, 0, 33]),
    ("f32", 2, 1, 20, 1, 2, [70, 1], [5, 2]),
    ("f32", 4, 1, 128, 1, 1, [2100], [9]),
    ("f32", 16, 2, 4, 1, 2, [31], [64]),
]


@pytest.mark.parametrize("dtype,nq,nkv,dh,branches,paths,lens,nodes", CASES)
def test_attention_of_trees(dtype, nq, nkv, dh, branches, paths, lens, nodes):
    rng = np.random.default_rng(5)
    c = Cache(dtype, nq, nkv, dh, [a + b for a, b in zip(lens, nodes)], branches, spread=2.0)
    c.fill()
    check(c, nodes, [p for n in nodes for p in random_tree(rng, n)], paths)
    # a chain, and nodes that all follow the cache
    check(c, nodes, [i - 1 for n in nodes for i in range(n)], paths, seed=2)
    check(c, nodes, [-1] * sum(nodes), paths, seed=3)
    c.sess.close()


@pytest.mark.parametrize("dtype,nq,nkv,dh", [("bf16", 4, 1, 128), ("f32", 2, 2, 16)])
def test_cache_beyond_one_splits_page_ids(dtype, nq, nkv, dh):
    """More than 1024 pages in one sequence, a short one beside it."""
    nodes, lens = [5, 2], [20011, 40]
    c = Cache(dtype, nq, nkv, dh, [a + b for a, b in zip(lens, nodes)])
    c.fill()
    check(c, nodes, [-1, 0, 0, 2, 1, -1, 0], 2)
    c.sess.close()


@pytest.mark.parametrize("dtype,nq,nkv,dh,branches,paths,long", [("bf16", 16, 4, 128, 3, 4, 6000), ("bf16", 8, 2, 128, 1, 1, 3333),
                                                                 ("f32", 16, 4, 16, 3, 4, 2500)])
def test_runs_over_many_short_sequences(dtype, nq, nkv, dh, branches, paths, long):
    """More (sequence, KV head) pairs than workgroups, one of them long: runs of
    pages begin and end inside sequences and go over several."""
    rng = np.random.default_rng(11)
    n = 40 if paths > 1 else 300
    nodes = [64] + [int(x) for x in rng.integers(1, 4, n)]
    lens = [long] + [int(x) for x in rng.integers(0, 300, n)]
    order = rng.permutation(n + 1)
    nodes, lens = [nodes[i] for i in order], [lens[i] for i in order]
    c = Cache(dtype, nq, nkv, dh, [a + b for a, b in zip(lens, nodes)], branches=branches)
    c.fill()
    check(c, nodes, [p for m in nodes for p in random_tree(rng, m)], paths)
    c.sess.close()


@pytest.mark.parametrize("paths,nodes", [(4, [64, 50]), (1, [4, 1])])
def test_more_than_1024_pages_in_one_workgroup(paths, nodes):
    """A sequence so long that the sixteen workgroups it is cut for have more
    pages than they keep the numbers of.  A few rows in float64; the sums of n
    keys take up to n more roundings in fp32."""
    lens = [270000, 100]
    c = Cache("bf16", 4, 1, 128, [a + b for a, b in zip(lens, nodes)], branches=3)
    c.fill()
    rng = np.random.default_rng(3)
    parents = [p for n in nodes for p in random_tree(rng, n)]
    q = torch.randn((paths, sum(nodes), 4, 128), generator=torch.Generator().manual_seed(4)).to(c.tt)
    got = c.attend(nodes, parents, q)
    assert torch.equal(got, c.attend(nodes, parents, q))
    first = 0
    for b, n in enumerate(nodes):
        for i, line in enumerate(lines(parents[first:first + n])):
            if i not in (0, 17, n - 1):
                continue
            pos = list(range(lens[b])) + sorted(lens[b] + j for j in line)
            k, v = c.K[0][b][pos, 0].double(), c.V[0][b][pos, 0].double()
            rows = [(p, h) for p in range(paths) for h in range(4)]
            w = torch.softmax(torch.stack([q[p, first + i, h] for p, h in rows]).double() @ k.T / 128 ** 0.5, -1)
            o, a = w @ v, w @ v.abs()
            tol = 2.0 ** -8 * o.abs() + (2.02 * 2.0 ** -8 + len(pos) * 2.0 ** -24) * a
            off = (torch.stack([got[p, first + i, h] for p, h in rows]).double() - o).abs() / tol
            assert bool((off <= 1).all()), (b, i, float(off.max()))
        first += n
    c.sess.close()


@pytest.mark.parametrize("batch", [130, 300])
def test_more_sequences_than_one_launch_takes(batch):
    rng = np.random.default_rng(batch)
    nodes = [int(x) for x in rng.integers(0, 4, batch)]
    nodes[0] = 2
    c = Cache("bf16", 2, 1, 128, [int(x) + n for x, n in zip(rng.integers(0, 60, batch), nodes)])
    c.fill()
    check(c, nodes, [p for n in nodes for p in random_tree(rng, n)], 1)
    c.sess.close()


def test_layers_and_bad_parents():
    """The layer asked for; parents that are no earlier node read as none."""
    nodes = [6, 4]
    c = Cache("bf16", 4, 2, 128, [40, 20], layers=3)
    c.fill()
    bad = [0, 5, 1, -7, 1 << 30, 4, 3, 0, -1, 2]  # per sequence: own, later, earlier, ...
    good = [-1, -1, 1, -1, -1, 4, -1, 0, -1, 2]
    for layer in (2, 0):
        q, got = check(c, nodes, good, 2, layer=layer)
        assert torch.equal(c.attend(nodes, bad, q, layer), got)
    c.sess.close()


@pytest.mark.parametrize("dtype,nq,nkv,dh,base", [("bf16", 8, 2, 128, 0), ("bf16", 8, 2, 128, 27), ("bf16", 8, 2, 128, 4090),
                                                  ("f32", 4, 2, 64, 0), ("f32", 4, 2, 64, 27), ("f32", 4, 2, 64, 1500)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3.3e38])
def test_what_a_node_does_not_see_leaves_no_trace(dtype, nq, nkv, dh, base, bad):
    """Values that are not finite (or the type's largest) in nodes of other
    lines; the rows that see them show it where they are not finite."""
    n = 40
    up = [-1, 0] + [i - 2 for i in range(2, n)]  # two lines from node 0: odd and even nodes
    c = Cache(dtype, nq, nkv, dh, [base + n])
    c.fill()
    g = torch.Generator().manual_seed(0)
    q = torch.randn((2, n, nq, dh), generator=g).to(c.tt)
    clean = c.attend([n], up, q)
    for what, at in ((c.V, 7), (c.K, 7), (c.V, 39), (c.V, 20)):
        keep = what[0][0][base + at].clone()
        what[0][0][base + at, :, ::3] = bad
        c.fill()
        got = c.attend([n], up, q)
        sees = [at in line for line in lines(up)]
        for i in range(n):
            if not sees[i]:
                assert torch.equal(got[:, i], clean[:, i]), (i, at)
            elif what is c.V and not np.isfinite(bad):
                assert not torch.isfinite(got[:, i][..., ::3]).any(), (i, at)
                rest = torch.ones(dh, dtype=torch.bool)
                rest[::3] = False
                assert torch.equal(got[:, i][..., rest], clean[:, i][..., rest])
        what[0][0][base + at] = keep
    # a value before the nodes is every row's
    if base and not np.isfinite(bad):
        c.V[0][0][base - 1, :, 5] = bad
        c.fill()
        got = c.attend([n], up, q)
        assert not torch.isfinite(got[..., 5]).any() and torch.equal(got[..., :5], clean[..., :5])
    c.sess.close()


@pytest.mark.parametrize("dtype,dh,base", [("bf16", 128, 90), ("bf16", 128, 6000), ("f32", 20, 700)])
def test_outputs_in_place_of_the_queries(dtype, dh, base):
    rng = np.random.default_rng(2)
    nodes = [30, 41, 3]
    c = Cache(dtype, 8, 2, dh, [base + 30, 17 + 41, 300 + 3])
    c.fill()
    parents = [p for n in nodes for p in random_tree(rng, n)]
    q = torch.randn((2, 74, 8, dh), generator=torch.Generator().manual_seed(5)).to(c.tt)
    want = c.attend(nodes, parents, q)
    up, qd = torch.tensor(parents, dtype=torch.int32, device="cuda"), q.cuda()
    ws = torch.empty(c.B.dbt_tree_workspace_bytes(c.sess.cfg, 74), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    c.B.dbt_tree_attention(c.sess.kv, 0, c.B.make_tree(nodes, up.data_ptr()), 2, qd.data_ptr(), qd.data_ptr(),
                           ws.data_ptr(), c.sess.stream)
    torch.cuda.synchronize()
    assert torch.equal(qd.cpu(), want)
    c.sess.close()


def test_only_the_calls_rows_are_written():
    c = Cache("bf16", 4, 2, 128, [40, 20])
    c.fill()
    up = torch.tensor([-1, 0, 0, -1, 0], dtype=torch.int32, device="cuda")
    q = torch.randn((2, 5, 4, 128), device="cuda").to(torch.bfloat16)
    out = torch.full((2 * 5 + 6, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(c.B.dbt_tree_workspace_bytes(c.sess.cfg, 5), dtype=torch.uint8, device="cuda")
    c.B.dbt_tree_attention(c.sess.kv, 0, c.B.make_tree([3, 2], up.data_ptr()), 2, q.data_ptr(), out[3:].data_ptr(),
                           ws.data_ptr(), c.sess.stream)
    torch.cuda.synchronize()
    assert bool((out[:3] == 3).all()) and bool((out[13:] == 3).all()) and not bool((out[3:13] == 3).any())
    c.sess.close()


def test_attention_captured_on_a_stream_of_its_own():
    """Replays of a captured call (after eager ones) give the eager bits, with the
    program's own work and synchronizations between them."""
    nodes = [9, 30]
    c = Cache("bf16", 8, 2, 128, [4000, 300])
    c.fill()
    rng = np.random.default_rng(1)
    up = torch.tensor([p for n in nodes for p in random_tree(rng, n)], dtype=torch.int32, device="cuda")
    q = torch.randn((2, 39, 8, 128), device="cuda").to(torch.bfloat16)
    out, ws = torch.empty_like(q), torch.empty(c.B.dbt_tree_workspace_bytes(c.sess.cfg, 39), dtype=torch.uint8, device="cuda")
    tree = c.B.make_tree(nodes, up.data_ptr())

    def call(stream):
        c.B.dbt_tree_attention(c.sess.kv, 0, tree, 2, q.data_ptr(), out.data_ptr(), ws.data_ptr(), stream.cuda_stream)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(s)
    s.synchronize()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(s)
    for k in range(3):
        qk = torch.randn((2, 39, 8, 128), device="cuda").to(torch.bfloat16)
        keep = q.clone()
        q.copy_(qk)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            call(s)
        s.synchronize()
        eager = out.clone()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), k
        q.copy_(keep)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first), k
    c.sess.close()


# --------------------------------------------------------------------------
# The cache keeps a path
# --------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,nkv,dh,layers", [("bf16", 2, 128, 3), ("f32", 3, 20, 2), ("f32", 1, 128, 1)])
def test_kept_nodes_move_together(dtype, nkv, dh, layers):
    rng = np.random.default_rng(3)
    batch = 40  # more sequences than one launch moves
    nodes = [int(x) for x in rng.integers(1, 65, batch)]
    lens = [int(x) for x in rng.integers(0, 70, batch)]
    nodes[:6], lens[:6] = [64, 64, 5, 0, 7, 1], [0, 31, 16, 30, 15, 3]
    paths = [sorted(rng.choice(n, size=int(rng.integers(0, n + 1)), replace=False).tolist()) if n else [] for n in nodes]
    paths[0], paths[1], paths[2] = list(range(64)), list(range(1, 64)), []
    c = Cache(dtype, nkv, nkv, dh, [a + b for a, b in zip(lens, nodes)], layers=layers)
    c.fill()
    sess, B = c.sess, c.B
    free = sess.num_pages - sum(len(B.dbt_kv_pages(sess.kv, b)) for b in range(batch))
    before = [B.dbt_kv_pages(sess.kv, b) for b in range(batch)]
    k0, v0 = sess.k_pages.clone(), sess.v_pages.clone()
    sess.keep(nodes, paths)
    kp, k0 = (x.view(c.tt).view(layers, sess.num_pages, nkv, 16, dh).cpu() for x in (sess.k_pages, k0))
    vp, v0 = (x.view(c.tt).view(layers, sess.num_pages, nkv, dh, 16).cpu() for x in (sess.v_pages, v0))
    touched = set()
    for b in range(batch):
        want = lens[b] + len(paths[b])
        assert B.dbt_kv_length(sess.kv, b) == want
        pages = B.dbt_kv_pages(sess.kv, b)
        assert pages == before[b][:(want + 15) // 16]
        free += len(before[b]) - len(pages)
        src = list(range(lens[b])) + [lens[b] + i for i in paths[b]]
        for pos, of in enumerate(src):
            page, slot = pages[pos // 16], pos % 16
            if pos >= lens[b]:
                touched.add((page, slot))
            for l in range(layers):
                assert torch.equal(kp[l, page, :, slot], c.K[l][b][of]) and torch.equal(vp[l, page, :, :, slot], c.V[l][b][of])
    # nothing else was written
    same_k, same_v = (kp == k0) | (kp.isnan() & k0.isnan()), (vp == v0) | (vp.isnan() & v0.isnan())
    changed = {(int(p), int(j)) for p, j in (~same_k).any(4).any(2).any(0).nonzero()}
    changed |= {(int(p), int(j)) for p, j in (~same_v).any(3).any(2).any(0).nonzero()}
    assert changed <= touched
    # the pages given back are there to be taken
    B.dbt_kv_reserve(sess.kv, 3, lens[3] + 16)
    assert free >= 1
    sess.close()


# --------------------------------------------------------------------------
# The step over a tree
# --------------------------------------------------------------------------

def oracle_nodes(orc, lens, nodes, parents, tokens=None, h1=None, h2=None, on=True):
    outs, first = [], 0
    for b, n in enumerate(nodes):
        for line in lines(parents[first:first + n]):
            for i in reversed(line):
                o = orc.step_one(b, token=None if tokens is None else int(tokens[first + i]),
                                 h1=None if h1 is None else h1[first + i],
                                 h2=None if h2 is None else h2[first + i] if orc.s.n_branches == 1 else h2[:, first + i],
                                 branch_on=on, readout=False)
            orc.truncate(b, lens[b])
            outs.append(o)
        first += n
    orc._readout(outs)
    return outs


def bf16_shape(**kw):
    base = dict(n_layers=2, d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=128, d_ff=384, vocab=512, dtype="bf16",
                has_embeddings=True, std=0.05, coupling_std=0.5)
    base.update(kw)
    return synth.ModelShape(**base)


MOE = dict(n_layers=1, d_model=512, n_q_heads=8, n_kv_heads=2, d_ff=0, vocab=0, has_embeddings=False, n_experts=8,
           d_ff_expert=128, n_shared_experts=1, d_ff_shared=128, top_k1=2)
SHAPES = {
    "f32": tiny_shape(),
    "f32_branches": tiny_shape(n_branches=3),
    "bf16": bf16_shape(),
    "bf16_states": bf16_shape(has_embeddings=False, vocab=0),
    "bf16_branches": bf16_shape(n_branches=3, n_layers=1),
    "moe": bf16_shape(**MOE, top_k2=4),
    "moe_replay": bf16_shape(**MOE, top_k2=2, replay=True),
    "moe_matched": bf16_shape(**MOE, top_k2=2, compute_matched=True),
}


def same_experts(t, outs, path, k, replay=False):
    """Rows of an MoE layer whose experts are the oracle's.  Another selection
    needs a near-tie: with every router logit within e of the oracle's, an expert
    that takes another's place is within 2 e of it."""
    idx, lg = to_np(t[f"route_idx{path}"])[0], to_np(t[f"route_logits{path}"])[0].astype(np.float64)
    rows = []
    for i, o in enumerate(outs):
        rec = o["layers"][0]
        if np.array_equal(idx[i], rec[f"idx{path}"]):
            rows.append(i)
            continue
        if replay:  # the primary's selection, whatever the branch's logits say
            assert np.array_equal(idx[i], to_np(t["route_idx1"])[0][i])
            continue
        r = np.asarray(rec[f"r{path}"], np.float64)
        e, order = np.abs(lg[i] - r).max(), np.sort(r)[::-1]
        assert e <= BF16_TOL * np.abs(r).max()
        assert all(abs(r[idx[i][j]] - order[j]) <= 2 * e for j in range(k)), (i, path)
    assert len(rows) >= len(outs) - max(1, len(outs) // 8)
    return rows


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("on", [True, False])
def test_step_over_a_tree(name, on):
    shape = SHAPES[name]
    tol = F32_TOL if shape.dtype == "f32" else BF16_TOL
    rng = np.random.default_rng(7)
    lens, nodes = [37, 0, 16, 100], [9, 3, 0, 20]
    parents = [p for n in nodes for p in random_tree(rng, n)]
    R = sum(nodes)
    W = synth.make_weights(shape, seed=0)
    sess = make_session(shape, W, max_batch=40, max_pos=200)
    orc = Oracle(shape, W.values)
    fill_cache(sess, orc, shape, lens)
    for b, n in enumerate(lens):
        if n == 0:
            orc.kv_fill(b, 0, [np.zeros((0, shape.n_kv_heads, shape.head_dim))] * shape.n_layers,
                        [np.zeros((0, shape.n_kv_heads, shape.head_dim))] * shape.n_layers)
    kw = {}
    if shape.has_embeddings:
        kw["tokens"] = synth.make_tokens(1, 0, (R,), shape.vocab)
    else:
        h = synth.make_hidden(shape, R, paths=1 + shape.n_branches)
        kw["h1"], kw["h2"] = h[0], h[1] if shape.n_branches == 1 else h[1:]
    outs = oracle_nodes(orc, lens, nodes, parents, on=on, **kw)
    t = sess.decode_tree(nodes, parents, branch_on=on, **kw)
    print(f"tree step {name} on={on}", flush=True)
    every = same = list(range(R))
    if shape.n_experts:  # (an expert exchanged at a near-tie of two router logits is not the tree's)
        every = same_experts(t, outs, 1, shape.top_k1)
        same = sorted(set(every) & set(same_experts(t, outs, 2, shape.top_k2, shape.replay))) if on else []
    assert row_err(to_np(t["h1_out"])[every], np.stack([o["h1"] for o in outs])[every]).max() <= tol
    if on:
        h2 = to_np(t["h2_out"])
        for j in range(shape.n_branches):
            ref = np.stack([o["hb"][j] if shape.n_branches > 1 else o["h2"] for o in outs])
            assert row_err((h2 if shape.n_branches == 1 else h2[j])[same], ref[same]).max() <= tol
    if shape.vocab:
        check_readout(t, outs, tol, name, branch=on)
    from paper_2608_12385_amd import binding
    assert [binding.dbt_kv_length(sess.kv, b) for b in range(4)] == [a + b for a, b in zip(lens, nodes)]
    sess.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_drafting_gives_the_sequences_of_ordinary_steps(dtype):
    """Greedy generation by whole rounds of drafts (right ones, wrong ones and
    branches at once): the tokens are those of ordinary steps, wherever two of them do
    not nearly tie, and the cache ends up with the accepted lines."""
    shape = SHAPES[dtype]
    tol = F32_TOL if dtype == "f32" else BF16_TOL
    W = synth.make_weights(shape, seed=0)
    prompts = [synth.make_tokens(1, i, (n,), shape.vocab) for i, n in enumerate((19, 33))]
    from paper_2608_12385_amd import binding

    def fresh():
        s = make_session(shape, W, max_batch=32, max_pos=120, max_prompt=40)
        return s, s.prefill(prompts)["next_token"].cpu().tolist()

    plain, nxt = fresh()
    want = [[x] for x in nxt]
    margins = [[1.0] for _ in nxt]  # of each token over the next best, in mixture values
    for _ in range(12):
        t = plain.decode(tokens=[w[-1] for w in want])
        z1, z2, a = (to_np(t[k]).astype(np.float64) for k in ("logits1", "logits2", "alpha"))
        for b in range(2):
            p, q = (np.exp(z[b] - z[b].max()) / np.exp(z[b] - z[b].max()).sum() for z in (z1, z2))
            m = np.sort(a[b] * p + (1 - a[b]) * q)
            margins[b].append((m[-1] - m[-2]) / m[-1])
            want[b].append(int(t["next_token"][b]))
    sess, nxt = fresh()
    got = [[x] for x in nxt]
    lens = [len(p) for p in prompts]
    rounds = 0
    while min(len(g) for g in got) < 10:
        nodes, parents, tokens, guesses, clear = [], [], [], [], []
        for b in range(2):
            k = len(got[b])
            clear.append(got[b] == want[b][:k] and min(margins[b][:k + 4]) > 8 * tol)
            line = want[b][k - 1:k + 3]  # the last answer, then three right guesses
            if rounds % 3 == 1:
                line[2] = (line[2] + 1) % shape.vocab  # the second guess is wrong
            wrong = [(x + 7) % shape.vocab for x in line[1:]]
            toks, up = [line[0]], [-1]
            at = 0
            for i, x in enumerate(line[1:]):  # a wrong sibling before every guess
                toks += [wrong[i], x]
                up += [at, at]
                at = len(toks) - 1
            guesses.append(len(line))
            nodes.append(len(toks))
            parents += up
            tokens += toks
        t = sess.decode_tree(nodes, parents, tokens=tokens)
        token, _ = sess.sample(t, [0.5] * sum(nodes), [(0.0, 0, 1.0, 0.0)] * sum(nodes))
        drawn = token.cpu().tolist()
        # (the greedy draw evaluates the mixture in float64, the readout in float32)
        paths, after = binding.dbt_tree_accept(nodes, parents, tokens, drawn)
        sess.keep(nodes, paths)
        first = 0
        for b in range(2):
            assert paths[b][0] == 0
            got[b] += [tokens[first + i] for i in paths[b][1:]] + [after[b]]
            lens[b] += len(paths[b])
            assert binding.dbt_kv_length(sess.kv, b) == lens[b] == len(prompts[b]) + len(got[b]) - 1
            if clear[b]:  # every right guess is kept, and nothing after the wrong one
                assert len(paths[b]) == (2 if rounds % 3 == 1 else guesses[b])
            first += nodes[b]
        rounds += 1
    for b in range(2):
        for i, (x, y) in enumerate(zip(got[b], want[b])):
            if x != y:
                assert margins[b][i] <= 8 * tol, (b, i)
                break
    # the kept keys are those of a cache that took the tokens one by one
    again, _ = fresh()
    for i in range(min(len(g) for g in got) - 1):
        again.decode(tokens=[g[i] for g in got])
    for b in range(2):
        n = min(binding.dbt_kv_length(again.kv, b), lens[b])
        ka, kb = (torch.cat([s.k_pages.view(torch.float32 if dtype == "f32" else torch.bfloat16)
                             .view(shape.n_layers, s.num_pages, shape.n_kv_heads, 16, shape.head_dim)[:, p]
                             for p in binding.dbt_kv_pages(s.kv, b)[:(n + 15) // 16]], dim=2)[:, :, :n].float().cpu()
                  for s in (again, sess))
        assert row_err(ka.transpose(1, 2).reshape(-1, ka.shape[1] * shape.head_dim).numpy(),
                       kb.transpose(1, 2).reshape(-1, ka.shape[1] * shape.head_dim).numpy()).max() <= tol
    for s in (plain, sess, again):
        s.close()


def test_steps_around_a_tree_keep_their_bits():
    """A tree that is dropped leaves nothing behind: the next step and its cache
    are those of a session that never saw it."""
    shape = SHAPES["bf16"]
    W = synth.make_weights(shape, seed=0)
    from paper_2608_12385_amd import binding
    lens = [30, 47]

    def fresh():
        s = make_session(shape, W, max_batch=24, max_pos=150)
        s.k_pages.zero_(), s.v_pages.zero_()
        fill_cache(s, None, shape, lens)
        return s

    a, b = fresh(), fresh()
    b.decode_tree([12, 12], [i - 1 for _ in range(2) for i in range(12)], tokens=list(range(24)))
    for i, n in enumerate(lens):
        binding.dbt_kv_truncate(b.kv, i, n)
    for _ in range(2):
        x, y = a.decode(tokens=[3, 4]), b.decode(tokens=[3, 4])
        for k in x:
            assert torch.equal(x[k], y[k]), k
    a.close(), b.close()
