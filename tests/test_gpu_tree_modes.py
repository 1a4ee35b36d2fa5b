"""The step over drafted tokens with the branch on and off: the primary's
outputs, its routes and the keys and values it appends are the same bits, also
where the two calls' query rows would cut a long cache differently."""
import numpy as np
import pytest

import synth
from tests.gpu_util import make_session

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def shape_of(kv, group, dtype="bf16", **kw):
    base = dict(n_layers=2, d_model=256, n_q_heads=kv * group, n_kv_heads=kv, head_dim=128, d_ff=384, vocab=512, dtype=dtype,
                has_embeddings=True, std=0.05, coupling_std=0.5)
    return synth.ModelShape(**dict(base, **kw))


MOE = dict(d_model=512, d_ff=0, vocab=0, has_embeddings=False, n_experts=8, d_ff_expert=128, n_shared_experts=1,
           d_ff_shared=128, top_k1=2, top_k2=2)
CASES = {
    # units cut into stages of their own, or into two together
    "few": (shape_of(8, 4), [2000] * 4, [20] * 4),
    # cut once, or whole
    "batch": (shape_of(8, 4), [4096] * 32, [20] * 32),
    "branches": (shape_of(8, 4, n_branches=3), [2000] * 4, [20] * 4),
    "f32": (shape_of(8, 4, "f32", head_dim=16, d_model=48, d_ff=96, vocab=64, std=0.2), [2000] * 4, [20] * 4),
    "ragged": (shape_of(8, 4), [1000, 2000, 0, 700], [16, 20, 3, 0]),
    "states": (shape_of(8, 4, vocab=0, has_embeddings=False), [2000] * 4, [20] * 4),
    "moe": (shape_of(8, 4, **MOE), [2000] * 4, [20] * 4),
    "moe_matched": (shape_of(8, 4, **dict(MOE, compute_matched=True)), [2000] * 4, [20] * 4),
    "short": (shape_of(2, 2), [37, 5, 16], [9, 3, 20]),
}


@pytest.mark.parametrize("name", list(CASES))
def test_primary_does_not_depend_on_the_branch(name):
    from paper_2608_12385_amd import binding as B
    shape, lens, nodes = CASES[name]
    print(name, flush=True)
    rng = np.random.default_rng(5)
    R, pos = sum(nodes), max(lens) + max(nodes)
    parents = [int(rng.integers(-1, i)) if i else -1 for n in nodes for i in range(n)]
    sess = make_session(shape, synth.make_weights(shape, seed=0), max_batch=R, max_pos=pos, num_pages=sum((a + b + 15) // 16 for a, b in zip(lens, nodes)))
    tt = torch.float32 if shape.dtype == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(3)
    for p in (sess.k_pages, sess.v_pages):
        p.view(tt).normal_(0.0, 1.0, generator=g)
    for b, n in enumerate(lens):
        B.dbt_kv_reserve(sess.kv, b, n)
    kw = {}
    if shape.has_embeddings:
        kw["tokens"] = synth.make_tokens(1, 0, (R,), shape.vocab)
    else:
        h = synth.make_hidden(shape, R, paths=2)
        kw["h1"], kw["h2"] = h[0], h[1]
    full = sess.k_pages.clone(), sess.v_pages.clone()
    seen = []
    for on in (True, False):
        sess.k_pages.copy_(full[0]), sess.v_pages.copy_(full[1])
        for b, n in enumerate(lens):
            B.dbt_kv_truncate(sess.kv, b, n)
        t = sess.decode_tree(nodes, parents, branch_on=on, **kw)
        got = {k: t[k].clone() for k in ("h1_out", "logits1", "route_idx1", "route_w1", "route_logits1") if k in t}
        got["k"], got["v"] = sess.k_pages.clone(), sess.v_pages.clone()  # (the sequences take the same pages again)
        seen.append((got, [B.dbt_kv_pages(sess.kv, b) for b in range(len(lens))]))
    assert seen[0][1] == seen[1][1]
    assert not torch.equal(seen[0][0]["k"], full[0])
    for k in seen[0][0]:
        assert torch.equal(seen[0][0][k], seen[1][0][k]), k
    sess.close()
