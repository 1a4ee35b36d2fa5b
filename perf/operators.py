"""Measured operators of drafted-token decoding: attention for a tree of
drafted tokens over the paged cache, the cache keeping one path of the tree,
and tokens drawn from the mixture of the two paths.

A case is one call as a serving program makes it.  Head layouts and
vocabularies are those of the repository's workloads (one 8B-shape layer, its
eight-way tensor-parallel share, the 24-layer model, the small fp32 model).
listed() and draw() give cases, prepare() makes what a program has in hand,
run() is one call (`own`: through the library; else in elementary torch
operations), work() the bytes and operations it cannot do without and exact()
its outputs in float64.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
MOST_NODES = 64  # drafted tokens of one sequence

# Head layouts: query heads, KV heads, head dimension.
HEADS = {
    "8b": (32, 8, 128, "bf16"),
    "shard": (4, 1, 128, "bf16"),
    "base": (16, 4, 128, "bf16"),
    "tiny": (4, 4, 64, "f32"),
}

# Request kinds of the draw: temperature, top_k, top_p, min_p.
REQUESTS = {
    "chat": (0.7, 50, 0.95, 0.0),
    "nucleus": (1.0, 0, 0.9, 0.0),
    "minp": (1.3, 0, 1.0, 0.05),
    "plain": (1.0, 0, 1.0, 0.0),
    "greedy": (0.0, 0, 1.0, 0.0),
    "wide": (0.9, 1000, 0.99, 0.0),
}


def listed():
    return [
        # one interactive sequence with a small draft: latency
        dict(name="tree_8b_b1", op="tree", heads="8b", batch=1, lo=777, hi=777, nlo=12, nhi=12, paths=2),
        # the serving batch, short drafts: bound by reading the cache once
        dict(name="tree_8b_b32", op="tree", heads="8b", batch=32, lo=4096, hi=4096, nlo=8, nhi=8, paths=2),
        # few users with long ragged contexts and wide trees: 256 query rows for each key
        dict(name="tree_8b_long", op="tree", heads="8b", batch=8, lo=16384, hi=32768, nlo=32, nhi=32, paths=2),
        # a tensor-parallel share, one-flow model, ragged lengths and drafts, sequences without a draft among them
        dict(name="tree_shard_b13", op="tree", heads="shard", batch=13, lo=150, hi=4096, nlo=0, nhi=9, paths=1),
        # full trees over an ordinary batch, three decode branches
        dict(name="tree_base_b16", op="tree", heads="base", batch=16, lo=300, hi=1500, nlo=64, nhi=64, paths=4),
        # the fp32 model
        dict(name="tree_f32_b4", op="tree", heads="tiny", batch=4, lo=33, hi=900, nlo=3, nhi=20, paths=2),
        # one request's next token: latency
        dict(name="sample_b1", op="sample", rows=1, vocab=32000, branches=1, kind="chat"),
        # a batch of requests of every kind over the large vocabulary
        dict(name="sample_b64", op="sample", rows=64, vocab=128256, branches=1, kind="mixed"),
        # every node of the drafts of a batch, one-flow model, odd vocabulary
        dict(name="sample_nodes", op="sample", rows=500, vocab=50257, branches=0, kind="nucleus"),
        # the whole distribution of two branches, nothing cut off
        dict(name="sample_full", op="sample", rows=16, vocab=32000, branches=2, kind="plain"),
        # accepted paths of the 24-layer model's batch
        dict(name="keep_24l_b16", op="keep", heads="base", layers=24, batch=16, lo=40, hi=300, nlo=16, nhi=16),
        # one sequence of the fp32 model
        dict(name="keep_f32_b1", op="keep", heads="tiny", layers=2, batch=1, lo=137, hi=137, nlo=6, nhi=6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = [work(c) for c in listed()]
    most = {k: max(w[k] for w in top) for k in ("bytes", "flops")}
    while True:
        c = _draw(rng)
        w = work(c)
        if all(w[k] <= most[k] for k in most):
            return c


def _draw(rng):
    op = rng.choice(["tree"] * 3 + ["sample"] * 3 + ["keep"])
    if op == "sample":
        vocab = rng.choice([16064, 32000, 50257, 128256, _log(rng, 64, 131072)])
        return dict(op="sample", rows=_log(rng, 1, 512), vocab=vocab, branches=rng.choice([0, 1, 1, 2, 3]),
                    kind=rng.choice(["mixed", "mixed"] + list(REQUESTS)))
    heads = rng.choice(["8b", "shard", "base", "tiny"])
    nq, nkv = HEADS[heads][:2]
    nhi = _log(rng, 1, MOST_NODES)
    nlo = rng.randint(0, nhi)
    if op == "keep":
        hi = _log(rng, 2, 400)
        return dict(op="keep", heads=heads, layers=_log(rng, 1, 24), batch=_log(rng, 1, 24), lo=rng.randint(0, hi), hi=hi,
                    nlo=nlo, nhi=nhi)
    hi = _log(rng, 2, {"8b": 32768, "shard": 32768, "base": 16384, "tiny": 2048}[heads])
    return dict(op="tree", heads=heads, batch=_log(rng, 1, 40 if heads != "tiny" else 8), lo=rng.randint(hi // 8, hi), hi=hi,
                nlo=nlo, nhi=nhi, paths=rng.randint(1, min(4, 16 // (nq // nkv))))


def _spread(lo, hi, n):
    """n values over [lo, hi], the same for every seed (low-discrepancy order)."""
    return [lo + int((hi - lo) * ((b + 1) * 0.6180339887498949 % 1.0) + 0.5) for b in range(n)]


def _lengths(c):
    return _spread(c["lo"], c["hi"], c["batch"])


def _nodes(c):
    n = _spread(c["nlo"], c["nhi"], c["batch"])
    n[0] = max(n[0], 1)  # (a call without a drafted token computes nothing)
    return n


def _kept(c):
    """Indices of the accepted nodes of each sequence: a third of the draft, ascending."""
    out = []
    for b, n in enumerate(_nodes(c)):
        k = (n + 2) // 3 if b % 7 != 3 else 0  # (some drafts are turned down whole)
        out.append(sorted({min(n - 1, (j * 3 + (b + j) % 3)) for j in range(k)}))
    return out


def work(c):
    if c["op"] == "sample":
        paths = 1 + c["branches"]
        return {"bytes": c["rows"] * (c["vocab"] * paths * 4 + 12), "flops": c["rows"] * c["vocab"] * paths * 4}
    nq, nkv, dh, dtype = HEADS[c["heads"]]
    es = 2 if dtype == "bf16" else 4
    if c["op"] == "keep":
        moved = sum(sum(1 for j, i in enumerate(p) if i != j) for p in _kept(c))
        return {"bytes": max(1, 2 * 2 * moved * c["layers"] * nkv * dh * es), "flops": 0}
    lens, nodes = _lengths(c), _nodes(c)
    kv = sum(n + t for n, t in zip(lens, nodes) if t) * 2 * nkv * dh * es
    rows = sum(nodes) * c["paths"]
    pairs = sum((n + (t + 1) / 2) * t for n, t in zip(lens, nodes)) * c["paths"]
    return {"bytes": kv + 2 * rows * nq * dh * es + 4 * sum(nodes), "flops": 4 * pairs * nq * dh}


# --------------------------------------------------------------------------
# What a program has in hand
# --------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=g)


class _Cache:
    """Pages of a cache whose sequences grew in turns, so that the pages of one
    are not all in a row, and (own) the library's handles on them."""

    def __init__(self, c, seed, layers):
        self.c = c
        g = _generator(seed)
        self.heads = nq, nkv, dh, dtype = HEADS[c["heads"]]
        wt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.lens, self.nodes = _lengths(c), _nodes(c)
        total = [n + t for n, t in zip(self.lens, self.nodes)]
        pages = [(n + PAGE - 1) // PAGE for n in total]
        self.mpps = max(1, max(pages))
        self.num_pages = max(1, sum(pages))
        # K: [layer][page][KV head][slot][d]; V: [layer][page][KV head][d][slot]
        self.k = _normal(g, (layers, self.num_pages, nkv, PAGE, dh), wt)
        self.v = _normal(g, (layers, self.num_pages, nkv, dh, PAGE), wt)
        half = [p // 2 for p in pages]
        grow = [(b, half[b]) for b in range(c["batch"])] + [(b, pages[b] - half[b]) for b in reversed(range(c["batch"]))]
        table, free = [[] for _ in pages], 0
        for b, n in grow:
            table[b] += range(free, free + n)
            free += n
        self.table = torch.tensor([t + [0] * (self.mpps - len(t)) for t in table], dtype=torch.int32, device="cuda")
        # every node's parent: an earlier node of its sequence, or none (-1)
        cpu = torch.Generator().manual_seed(seed)
        up = [torch.zeros(0, dtype=torch.int64)]
        for n in self.nodes:
            back = (torch.rand(n, generator=cpu) ** 2 * torch.arange(n)).long()
            p = torch.arange(n) - 1 - back
            p[1:] = torch.where(torch.rand(max(0, n - 1), generator=cpu) < 0.05, -1, p[1:])
            up.append(p)
        self.parents = torch.cat(up).to(torch.int32).cuda()
        if own:
            self._open(layers, pages, half, total)
            if c["op"] == "keep":
                _grow_again(self, pages, half, total)

    def _open(self, layers, pages, half, total):
        from paper_2608_12385_amd import binding
        self.lib = binding
        c, (nq, nkv, dh, dtype) = self.c, self.heads
        wt = torch.bfloat16 if dtype == "bf16" else torch.float32
        d = 128
        cfg = binding.dbt_config(
            n_layers=layers, d_model=d, n_q_heads=nq, n_kv_heads=nkv, head_dim=dh, d_ff=d, n_branches=max(1, c.get("paths", 2) - 1),
            dtype=binding.DBT_BF16 if dtype == "bf16" else binding.DBT_F32, max_batch=c["batch"],
            max_pos=self.mpps * PAGE, rms_eps=1e-5, rope_theta=10000.0)
        shapes = dict(wq=(nq * dh, d), wk=(nkv * dh, d), wv=(nkv * dh, d), wo=(d, nq * dh), w_gate=(d, d), w_up=(d, d), w_down=(d, d))
        vectors = dict(attn_norm=d, mlp_norm=d, a=nq * dh, b=d, c=d)
        w = {n: torch.zeros(s, dtype=wt, device="cuda") for n, s in shapes.items()}
        w.update({n: torch.zeros(s, dtype=torch.float32, device="cuda") for n, s in vectors.items()})
        hl = (binding.dbt_layer_weights * layers)(*[binding.dbt_layer_weights(**{n: t.data_ptr() for n, t in w.items()})] * layers)
        self.keep = w, hl
        self.workspace = torch.empty(binding.dbt_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        self.model = binding.dbt_create(cfg, binding.dbt_weights(h_layers=hl), self.workspace.data_ptr())
        self.page_table = torch.full((c["batch"], self.mpps), -1, dtype=torch.int32, device="cuda")
        self.kv = binding.dbt_kv_create(self.model, self.k.data_ptr(), self.v.data_ptr(), self.num_pages,
                                        self.page_table.data_ptr(), self.mpps)
        for b in range(c["batch"]):
            if half[b]:
                binding.dbt_kv_reserve(self.kv, b, half[b] * PAGE)
        for b in reversed(range(c["batch"])):
            binding.dbt_kv_reserve(self.kv, b, total[b])
        self.tree = binding.make_tree(self.nodes, self.parents.data_ptr())
        if c["op"] == "tree":
            self.tree_workspace = torch.empty(binding.dbt_tree_workspace_bytes(cfg, sum(self.nodes)), dtype=torch.uint8,
                                              device="cuda")
        else:
            self.paths = binding.make_paths(_kept(c))
            for b in range(c["batch"]):
                binding.dbt_kv_truncate(self.kv, b, self.lens[b])

    def __del__(self):
        if getattr(self, "kv", None):
            self.lib.dbt_kv_destroy(self.kv)
        if getattr(self, "model", None):
            self.lib.dbt_destroy(self.model)


def _grow_again(s, pages, half, total):
    """Lets a pass over kept paths run again on the same cache: it grows the
    nodes that the last one dropped, on the pages they had.  The library hands
    out the lowest free page first, so the sequences stand in reverse, in which
    order growing them takes the pages of the table again."""
    B = s.c["batch"]
    kept = _kept(s.c)
    at = [B - 1 - b for b in range(B)]
    for b in range(B):
        s.lib.dbt_kv_truncate(s.kv, b, 0)
    for b in range(B):
        if half[b]:
            s.lib.dbt_kv_reserve(s.kv, at[b], half[b] * PAGE)
    for b in reversed(range(B)):
        s.lib.dbt_kv_reserve(s.kv, at[b], total[b])
    s.tree = s.lib.make_tree(s.nodes[::-1])
    s.paths = s.lib.make_paths(kept[::-1])
    now = [n + len(p) for n, p in zip(s.lens, kept)]
    for b in range(B):
        s.lib.dbt_kv_truncate(s.kv, at[b], now[b])
    # one call, unless sequences are so short that they drop most of their pages:
    # then calls whose pages are handed out in ascending order each
    table = s.table.tolist()
    lost = sorted((table[b][j], at[b], b, j) for b in range(B) for j in range((now[b] + PAGE - 1) // PAGE, pages[b]))
    last, s.grow, grown = -1, [], [0] * B
    for b in range(B):
        if pages[b] == (now[b] + PAGE - 1) // PAGE:
            grown[at[b]], now[b] = total[b] - now[b], total[b]
    for _, a, b, j in lost:
        if a < last:
            s.grow.append(s.lib.make_tree(grown))
            grown = [0] * B
        last, end = a, min(total[b], (j + 1) * PAGE)
        grown[a] += end - now[b]
        now[b] = end
    s.grow.append(s.lib.make_tree(grown))


class _Tree(_Cache):
    def __init__(self, c, seed):
        super().__init__(c, seed, 1)
        nq, _, dh, _ = self.heads
        self.q = _normal(_generator(seed + 1), (c["paths"], sum(self.nodes), nq, dh), self.k.dtype)
        self.out = torch.empty_like(self.q)


class _Keep(_Cache):
    def __init__(self, c, seed):
        super().__init__(c, seed, c["layers"])
        self.kept = _kept(c)


class _Sample:
    """Logits as a language model gives them (weights that fall off with the
    rank, the branch near the primary), the step's alpha, random numbers and
    what each request asked for."""

    def __init__(self, c, seed):
        self.c = c
        g = _generator(seed)
        R, V, nb = c["rows"], c["vocab"], c["branches"]
        rank = torch.rand((R, V), device="cuda", generator=g) * V
        steep = 0.8 + 0.7 * torch.rand((R, 1), device="cuda", generator=g)
        self.logits1 = 8.0 - steep * torch.log1p(rank) + 0.5 * _normal(g, (R, V), torch.float32)
        self.logits2 = self.alpha = None
        if nb:
            self.logits2 = torch.stack([self.logits1 + _normal(g, (R, V), torch.float32) for _ in range(nb)])
            self.alpha = torch.softmax(self.logits1, 1).square().sum(1).clamp(0.5, 1.0)
        self.u = torch.rand(R, device="cuda", generator=g)
        kinds = list(REQUESTS) if c["kind"] == "mixed" else [c["kind"]]
        self.requests = [REQUESTS[kinds[r % len(kinds)]] for r in range(R)]
        if own:
            from paper_2608_12385_amd import binding
            self.lib = binding
            self.token = torch.empty(R, dtype=torch.int32, device="cuda")
            self.prob = torch.empty(R, dtype=torch.float32, device="cuda")
            self.params = binding.make_sampling(self.requests)
            self.input = binding.dbt_sample_in(
                logits1=self.logits1.data_ptr(), logits2=self.logits2.data_ptr() if nb else None,
                alpha=self.alpha.data_ptr() if nb else None, u=self.u.data_ptr(), h_params=self.params, rows=R, vocab=V,
                n_branches=nb)
            self.workspace = torch.empty(binding.dbt_sample_workspace_bytes(R, V), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    return {"tree": _Tree, "sample": _Sample, "keep": _Keep}[case["op"]](case, seed)


# --------------------------------------------------------------------------
# One call
# --------------------------------------------------------------------------

def run(s):
    op = s.c["op"]
    if own:
        stream = torch.cuda.current_stream().cuda_stream
        if op == "tree":
            s.lib.dbt_tree_attention(s.kv, 0, s.tree, s.c["paths"], s.q.data_ptr(), s.out.data_ptr(),
                                     s.tree_workspace.data_ptr(), stream)
            return s.out
        if op == "keep":
            for tree in s.grow:
                s.lib.dbt_tree_reserve(s.kv, tree)
            s.lib.dbt_kv_keep(s.kv, s.tree, s.paths, stream)
            return {"k": s.k, "v": s.v}
        s.lib.dbt_sample(s.input, s.token.data_ptr(), s.prob.data_ptr(), s.workspace.data_ptr(), stream)
        return {"token": s.token, "prob": s.prob}
    return {"tree": _plain_tree, "sample": _plain_sample, "keep": _plain_keep}[op](s)


def _plain_tree(s):
    """softmax(q k^T / sqrt(d)) v over the cached positions and the node's own
    line of the tree, in float32, for the whole batch padded to its longest."""
    nq, nkv, dh, _ = s.heads
    B, N, P = s.c["batch"], max(s.nodes), s.c["paths"]
    base, count = torch.tensor([s.lens, s.nodes], device="cuda")
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), count)
    node = torch.arange(len(seq), device="cuda") - (torch.cumsum(count, 0) - count)[seq]
    # line[b, i, j]: node j is node i or an ancestor of it
    up = s.parents.long()
    inner = up >= 0
    line = torch.zeros(B, N, N, device="cuda")
    line[seq[inner], node[inner], up[inner]] = 1.0
    line = line + torch.eye(N, device="cuda")
    line = torch.clamp(line @ line, max=1.0)  # (lines of up to 2, 4, ... 64 nodes)
    line = torch.clamp(line @ line, max=1.0)
    line = torch.clamp(line @ line, max=1.0)
    line = torch.clamp(line @ line, max=1.0)
    line = torch.clamp(line @ line, max=1.0)
    line = torch.clamp(line @ line, max=1.0)
    pos = torch.arange(s.mpps * PAGE, device="cuda")
    at = (pos - base[:, None]).clamp(0, N - 1)  # [B, L] index of the position's node
    drafted = (pos >= base[:, None]) & (pos < (base + count)[:, None])
    sees = torch.gather(line, 2, at[:, None, :].expand(B, N, -1)) > 0
    sees = (sees & drafted[:, None, :]) | (pos < base[:, None])[:, None, :]  # [B, N, L]
    ids = s.table.long()
    k = s.k[0][ids].permute(0, 2, 1, 3, 4).reshape(B, nkv, -1, dh).float()
    v = s.v[0][ids].permute(0, 2, 1, 4, 3).reshape(B, nkv, -1, dh).float()
    v = v * (pos < (base + count)[:, None])[:, None, :, None]
    q = torch.zeros(P, B, N, nq, dh, device="cuda")
    q[:, seq, node] = s.q.float()
    q = q.reshape(P, B, N, nkv, nq // nkv, dh).permute(1, 3, 2, 0, 4, 5).reshape(B, nkv, -1, dh)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(dh)
    score = score.reshape(B, nkv, N, -1, score.shape[-1]).masked_fill(~sees[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.reshape(B, nkv, -1, weight.shape[-1]), v).reshape(B, nkv, N, -1, dh) / total
    out = out.reshape(B, nkv, N, P, nq // nkv, dh).permute(3, 0, 2, 1, 4, 5).reshape(P, B, N, nq, dh)
    return out[:, seq, node].to(s.q.dtype)


def _plain_sample(s):
    """The draw from the definition, in float64: every comparison is between
    sums whose distance can be a millionth of the largest."""
    t, k, top_p, min_p = torch.tensor(s.requests, dtype=torch.float32).cuda().double().unbind(1)
    V = s.c["vocab"]

    def softmax(z):
        e = torch.exp(z.double() - z.double().amax(-1, keepdim=True))
        return e / e.sum(-1, keepdim=True)

    mix = softmax(s.logits1)
    if s.alpha is not None:
        a = s.alpha.double()[:, None]
        mix = a * mix + (1.0 - a) * softmax(s.logits2).mean(0)
    ratio = mix / mix.amax(1, keepdim=True)
    greedy = (t == 0)[:, None]
    weight = torch.where(greedy, (ratio == 1.0).double(), ratio ** (1.0 / torch.where(t == 0, 1.0, t))[:, None])
    k = torch.where(greedy[:, 0], 1.0, torch.where(k == 0, float(V), k))
    order = torch.sort(ratio, dim=1, descending=True, stable=True).indices
    sorted_w = torch.gather(weight, 1, order)
    sorted_w = sorted_w * (torch.arange(V, device="cuda") < k[:, None])
    before = torch.cumsum(sorted_w, 1) - sorted_w
    sorted_w = sorted_w * (before < top_p[:, None] * sorted_w.sum(1, keepdim=True)) * (sorted_w >= min_p[:, None])
    weight = torch.zeros_like(weight).scatter_(1, order, sorted_w)
    total = torch.cumsum(weight, 1)
    token = (total <= s.u.double()[:, None] * total[:, -1:]).sum(1).clamp(max=V - 1)
    prob = torch.gather(weight, 1, token[:, None])[:, 0] / total[:, -1]
    return {"token": token.to(torch.int32), "prob": prob.float()}


def _plain_keep(s):
    """The kept nodes' keys and values, in order, to the positions after the cached ones."""
    lens = torch.tensor(s.lens, device="cuda")
    count = torch.tensor([len(p) for p in s.kept], device="cuda")
    seq = torch.repeat_interleave(torch.arange(s.c["batch"], device="cuda"), count)
    to = torch.arange(len(seq), device="cuda") - (torch.cumsum(count, 0) - count)[seq] + lens[seq]
    of = torch.tensor(sum(s.kept, []), dtype=torch.int64, device="cuda") + lens[seq]
    table = s.table.long()
    k = s.k[:, table[seq, of // PAGE], :, of % PAGE]
    v = s.v[:, table[seq, of // PAGE], :, :, of % PAGE]
    s.k[:, table[seq, to // PAGE], :, to % PAGE] = k
    s.v[:, table[seq, to // PAGE], :, :, to % PAGE] = v
    return {"k": s.k, "v": s.v}


# --------------------------------------------------------------------------
# Float64 reference
# --------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "sample":
        # (a large drawn batch would take the CPU too long)
        return _exact_sample(prepare(case, seed)) if case["rows"] * case["vocab"] <= 30_000_000 else None
    s = prepare(case, seed)
    if case["op"] == "keep":
        return _exact_keep(s)
    nq, nkv, dh, _ = s.heads
    G, q, up = nq // nkv, s.q.double(), s.parents.tolist()
    out = torch.empty_like(q)
    first = 0
    for b, n in enumerate(s.nodes):
        L = s.lens[b]
        ids = s.table[b, :(L + n + PAGE - 1) // PAGE].long()
        for h in range(nq):
            k = s.k[0, ids, h // G].reshape(-1, dh).double()[:L + n]
            v = s.v[0, ids, h // G].transpose(1, 2).reshape(-1, dh).double()[:L + n]
            z = q[:, first:first + n, h] @ k.t() / dh ** 0.5  # [paths, n, L + n]
            mask = torch.full((n, L + n), -math.inf, dtype=torch.float64)
            mask[:, :L] = 0.0
            for i in range(n):
                j = i
                while j >= 0:
                    mask[i, L + j] = 0.0
                    j = up[first + j]
            if n:
                out[:, first:first + n, h] = torch.softmax(z + mask.cuda(), -1) @ v
        first += n
    return out


def _exact_sample(s):
    token, prob = [], []
    z1 = s.logits1.cpu().numpy().astype(np.float64)
    z2 = None if s.logits2 is None else s.logits2.cpu().numpy().astype(np.float64)
    u = s.u.cpu().numpy().astype(np.float64)
    for r, (t, k, top_p, min_p) in enumerate(s.requests):
        t, top_p, min_p = (float(np.float32(x)) for x in (t, top_p, min_p))
        e = np.exp(z1[r] - z1[r].max())
        m = e / e.sum()
        if z2 is not None:
            a = float(s.alpha[r])
            e = np.exp(z2[:, r] - z2[:, r].max(1, keepdims=True))
            m = a * m + (1 - a) * (e / e.sum(1, keepdims=True)).mean(0)
        order = np.argsort(-m, kind="stable")
        if t == 0:
            token.append(order[0])
            prob.append(1.0)
            continue
        order = order[:k] if k else order
        w = np.exp(np.log(m[order] / m[order[0]]) / t)
        keep = np.searchsorted(np.cumsum(w), top_p * w.sum()) + 1
        order, w = order[:keep], w[:keep]
        order, w = order[w >= min_p], w[w >= min_p]
        by = np.argsort(order)
        order, w = order[by], w[by]
        c = np.cumsum(w)
        i = min(int(np.searchsorted(c, u[r] * c[-1], side="right")), len(w) - 1)
        token.append(order[i])
        prob.append(w[i] / c[-1])
    return {"token": torch.tensor(np.array(token), dtype=torch.int32), "prob": torch.tensor(prob, dtype=torch.float64)}


def _exact_keep(s):
    k, v = s.k.double(), s.v.double()
    for b, path in enumerate(s.kept):
        row = s.table[b].tolist()
        for j, i in enumerate(path):  # (ascending: no source is overwritten before it is read)
            to, of = s.lens[b] + j, s.lens[b] + i
            k[:, row[to // PAGE], :, to % PAGE] = k[:, row[of // PAGE], :, of % PAGE]
            v[:, row[to // PAGE], :, :, to % PAGE] = v[:, row[of // PAGE], :, :, of % PAGE]
    return {"k": k, "v": v}
