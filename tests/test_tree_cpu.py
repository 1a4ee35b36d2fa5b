"""Drafted tokens and drawn tokens on the CPU: what the calls refuse, the
accepted path, and the pages of sequences that grow by a tree, keep a path or
fail on the way (on the stand-in for the HIP runtime)."""
import ctypes
import os
import random
import subprocess
import sys

import pytest

from tests.test_launches_cpu import FAKE, ROOT, Program, fake  # noqa: F401

ARG, SHAPE, NO_PAGES, HIP = 1, 2, 3, 6


def program(**kw):
    from paper_2608_12385_amd import binding as B
    p = Program("f32", **kw)
    kv, table = p.cache(pages=24)
    return B, p, kv, table


def config(B, **kw):
    return B.dbt_config(dtype=B.DBT_F32, **dict(dict(n_layers=2, d_model=48, n_q_heads=4, n_kv_heads=2, head_dim=16, d_ff=96, vocab=64,
                                                     has_embeddings=1, max_batch=4, max_pos=256, rope_theta=1e4), **kw))


def status(B, fn, *a):
    try:
        fn(*a)
    except B.DbtError as e:
        return e.status
    return 0


def test_trees_refused():
    B, p, kv, _t = program(max_batch=4, n_branches=2)
    tree = B.make_tree
    for b in range(4):
        B.dbt_kv_reserve(kv, b, 20)

    def attend(t, layer=0, paths=1, q=FAKE, out=FAKE, ws=FAKE, cache=kv):
        return status(B, B.dbt_tree_attention, cache, layer, t, paths, q, out, ws, 0)

    ok = tree([1, 2], FAKE)
    for bad in (tree([65], FAKE), tree([-1, 2], FAKE), tree([0, 0], FAKE), tree([], FAKE), tree([1] * 5, FAKE), tree([1, 2]),
                tree([21], FAKE), B.dbt_tree(batch=1, h_nodes=None, parents=FAKE)):
        assert attend(bad) == ARG
    for kw in (dict(layer=-1), dict(layer=2), dict(paths=0), dict(paths=4), dict(q=0), dict(out=0), dict(ws=0), dict(cache=None),
               dict(ws=FAKE + 16), dict(q=FAKE + 8), dict(out=FAKE + 4)):
        assert attend(ok, **kw) == ARG, kw

    def step(t, batch, cache=kv, ws=FAKE, **kw):
        return status(B, B.dbt_decode_tree, p.model, cache, B.dbt_step_in(batch=batch, **dict(dict(tokens=FAKE), **kw)), t, 1, p.out,
                      ws, 0)

    assert step(ok, 2) == ARG and step(ok, 3, tokens=None) == ARG and step(ok, 3, ws=FAKE + 8) == ARG and step(ok, 3, ws=0) == ARG
    assert step(tree([3, 2], FAKE), 5) == ARG  # more nodes than the model's buffers hold
    assert step(tree([1, 2]), 3) == ARG and step(tree([66], FAKE), 66) == ARG
    # neither lengths nor pages changed
    assert [B.dbt_kv_length(kv, b) for b in range(4)] == [20] * 4 and all(len(B.dbt_kv_pages(kv, b)) == 2 for b in range(4))
    # growth: max_pos (256), the pool (24 pages, 8 taken), the caller's array
    assert status(B, B.dbt_tree_reserve, kv, tree([64] * 4)) == 0
    assert [B.dbt_kv_length(kv, b) for b in range(4)] == [84] * 4 and all(len(B.dbt_kv_pages(kv, b)) == 6 for b in range(4))
    assert status(B, B.dbt_tree_reserve, kv, tree([0, 0, 0, 64])) == NO_PAGES
    for b in range(3):
        B.dbt_kv_truncate(kv, b, 0)
    B.dbt_kv_reserve(kv, 3, 230)
    assert status(B, B.dbt_tree_reserve, kv, tree([1, 0, 0, 27])) == SHAPE and B.dbt_kv_length(kv, 0) == 0
    assert status(B, B.dbt_tree_reserve, kv, tree([1, 0, 0, 26])) == 0 and B.dbt_kv_length(kv, 3) == 256

    def keep(nodes, kept, path):
        n = (ctypes.c_int32 * max(1, len(path)))(*path), (ctypes.c_int32 * len(kept))(*kept)
        return status(B, B.dbt_kv_keep, kv, tree(nodes), (n[1], n[0], len(nodes)), 0)

    assert keep([0, 0, 0, 4], [0, 0, 0, 5], [0, 1, 2, 3, 3]) == ARG
    assert keep([0, 0, 0, 4], [0, 0, 0, -1], []) == ARG
    for path in ([0, 4], [-1, 0], [2, 2], [3, 1]):
        assert keep([0, 0, 0, 4], [0, 0, 0, 2], path) == ARG, path
    assert keep([2, 0, 0, 0], [0, 0, 0, 0], []) == ARG  # more nodes than positions
    assert B.dbt_kv_length(kv, 3) == 256
    for bad in (0, -3):
        assert B.dbt_tree_workspace_bytes(config(B), bad) == 0
    assert 0 < B.dbt_tree_workspace_bytes(config(B), 1) <= B.dbt_tree_workspace_bytes(config(B), 64)
    assert B.dbt_tree_workspace_bytes(config(B, n_q_heads=3), 4) == 0


def test_steps_over_states_need_them():
    from paper_2608_12385_amd import binding as B
    p = Program("f32", max_batch=4, has_embeddings=0, max_prompt=0)
    kv, _t = p.cache()
    t = B.make_tree([2], FAKE)
    for on, kw in ((1, dict(h1_in=FAKE)), (1, dict(h2_in=FAKE)), (0, dict())):
        assert status(B, B.dbt_decode_tree, p.model, kv, B.dbt_step_in(batch=2, **kw), t, on, p.out, FAKE, 0) == ARG


def test_draws_refused():
    from paper_2608_12385_amd import binding as B
    good = dict(logits1=FAKE, logits2=FAKE, alpha=FAKE, u=FAKE, rows=2, vocab=100, n_branches=1)

    def draw(params=((1.0, 0, 1.0, 0.0),) * 2, token=FAKE, ws=FAKE, **kw):
        return status(B, B.dbt_sample, B.dbt_sample_in(h_params=B.make_sampling(list(params)), **dict(good, **kw)), token, 0, ws, 0)

    for kw in (dict(logits1=None), dict(u=None), dict(logits2=None), dict(alpha=None), dict(rows=0), dict(rows=65536), dict(vocab=0),
               dict(vocab=(1 << 20) + 1), dict(n_branches=4), dict(n_branches=-1), dict(token=0), dict(ws=0), dict(ws=FAKE + 64)):
        assert draw(**kw) == ARG, kw
    nan, inf = float("nan"), float("inf")
    for bad in ((-0.5, 0, 1, 0), (nan, 0, 1, 0), (inf, 0, 1, 0), (1, -1, 1, 0), (1, 0, 0, 0), (1, 0, 1.5, 0), (1, 0, nan, 0),
                (1, 0, 1, -0.1), (1, 0, 1, 1.1), (1, 0, 1, nan)):
        assert draw(params=((1.0, 0, 1.0, 0.0), bad)) == ARG, bad
    assert status(B, B.dbt_sample, B.dbt_sample_in(h_params=None, **good), FAKE, 0, FAKE, 0) == ARG
    for rows, vocab in ((0, 5), (5, 0), (65536, 5), (5, (1 << 20) + 1)):
        assert B.dbt_sample_workspace_bytes(rows, vocab) == 0
    assert B.dbt_sample_workspace_bytes(1, 1) > 0


def test_accepted_paths():
    from paper_2608_12385_amd import binding as B
    # (parents, tokens, drawn) -> path, next
    hand = [([], [], [], [], -1), ([-1], [5], [9], [0], 9), ([-1, 0, 1], [5, 6, 7], [6, 7, 8], [0, 1, 2], 8),
            ([-1, 0, 1], [5, 6, 7], [6, 9, 8], [0, 1], 9), ([-1, 0, 0, 2], [5, 6, 7, 8], [7, 1, 8, 3], [0, 2, 3], 3),
            ([-1, 0, 0], [5, 6, 6], [6, 1, 2], [0, 1], 1),      # the first of two equal children
            ([-1, -1, 1], [5, 5, 6], [5, 6, 7], [0], 5),        # another root is never reached
            ([-1, 0, 0, 1], [5, 6, 6, 2], [6, 3, 2, 4], [0, 1], 3)]
    nodes = [len(h[0]) for h in hand]
    paths, after = B.dbt_tree_accept(nodes, *[sum((h[i] for h in hand), []) for i in range(3)])
    assert paths == [h[3] for h in hand] and after == [h[4] for h in hand]
    rng = random.Random(0)
    for _ in range(200):
        n = rng.randint(1, 64)
        up = [-1] + [rng.randrange(0, i) for i in range(1, n)]
        tok, drawn = ([rng.randrange(3) for _ in range(n)] for _ in range(2))
        at, want = 0, [0]
        while True:
            kids = [j for j in range(n) if up[j] == at and j > at and tok[j] == drawn[at]]
            if not kids:
                break
            at = kids[0]
            want.append(at)
        (path,), (nxt,) = B.dbt_tree_accept([n], up, tok, drawn)
        assert path == want and nxt == drawn[at]
    with pytest.raises(B.DbtError):
        B.dbt_tree_accept([65], [-1] * 65, [0] * 65, [0] * 65)
    with pytest.raises(B.DbtError):
        B.dbt_tree_accept([], [], [], [])
    with pytest.raises(ValueError):
        B.dbt_tree_accept([2], [-1], [0, 0], [0, 0])
    with pytest.raises(ValueError):
        B.dbt_kv_keep(None, B.make_tree([1, 1]), B.make_paths([[0]]), 0)


def run_child(fake, name):  # noqa: F811
    pre = " ".join(x for x in (fake, os.environ.get("LD_PRELOAD", "")) if x)
    r = subprocess.run([sys.executable, __file__, name, fake], capture_output=True, text=True, cwd=ROOT, timeout=300,
                       env=dict(os.environ, LD_PRELOAD=pre, PYTHONPATH=ROOT))
    assert r.returncode == 0 and "done" in r.stdout, (r.stdout + r.stderr)[-3000:]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_trees_that_fail_give_their_pages_back(fake, dtype):  # noqa: F811
    run_child(fake, "failing_" + dtype)


def test_page_tables_of_trees(fake):  # noqa: F811
    run_child(fake, "tables")


# ---------------------------------------------------------------------------
# in the child
# ---------------------------------------------------------------------------

def failing(fk, dtype):
    p = Program(dtype, max_batch=40)
    B = p.B
    kv, table = p.cache(pages=64, nseq=40)
    for b, n in enumerate((20, 0, 31)):
        B.dbt_kv_reserve(kv, b, n)
    t = B.make_tree([12, 3, 20], FAKE)
    sin = B.dbt_step_in(tokens=FAKE, batch=35)

    def held():
        return [(B.dbt_kv_length(kv, b), B.dbt_kv_pages(kv, b)) for b in range(3)]

    before = held()
    fk.fake_reset(-1)
    assert p.status(B.dbt_decode_tree, p.model, kv, sin, t, 1, p.out, FAKE, 0) == 0
    n = fk.fake_launches()
    after = held()
    assert n > 10 and [x[0] for x in after] == [32, 3, 51]
    for b, m in enumerate((20, 0, 31)):
        B.dbt_kv_truncate(kv, b, m)
    for at in range(n):
        fk.fake_reset(at)
        assert p.status(B.dbt_decode_tree, p.model, kv, sin, t, 1, p.out, FAKE, 0) == 6, at
        assert held() == before, at
    fk.fake_reset(-1)
    assert p.status(B.dbt_decode_tree, p.model, kv, sin, t, 1, p.out, FAKE, 0) == 0 and held() == after
    for b in range(3):
        assert list(table[b * p.mpps:][:len(after[b][1])]) == after[b][1]
    # a keep whose launch fails leaves the lengths
    fk.fake_reset(0)
    assert p.status(B.dbt_kv_keep, kv, t, B.make_paths([[0, 3], [1], []]), 0) == 6 and held() == after
    fk.fake_reset(-1)
    assert p.status(B.dbt_kv_keep, kv, t, B.make_paths([[0, 3], [1], []]), 0) == 0
    assert [x[0] for x in held()] == [22, 1, 31] and [len(x[1]) for x in held()] == [2, 1, 2]
    assert fk.fake_launches() == 1


def tables(fk):
    """Growth, keeps and drops at random: every sequence's device table
    holds its pages, no page has two owners, none is lost."""
    rng = random.Random(1)
    p = Program("f32", max_batch=40)
    B = p.B
    kv, table = p.cache(pages=60, nseq=40)
    fk.fake_reset(-1)
    for _ in range(400):
        nodes = [rng.choice([0, 0, 1, 5, 16, 40]) for _ in range(rng.randint(1, 6))]
        t = B.make_tree(nodes, FAKE)
        lens = [B.dbt_kv_length(kv, b) for b in range(6)]
        if rng.random() < 0.5 or sum(nodes) > 40:
            s = p.status(B.dbt_tree_reserve, kv, t)
            p.status(B.dbt_tree_attention, kv, 1, t, 2, FAKE, FAKE, FAKE, 0)
        else:
            s = p.status(B.dbt_decode_tree, p.model, kv, B.dbt_step_in(tokens=FAKE, batch=sum(nodes)), t, 1, p.out, FAKE, 0)
        grown = [n + (nodes[b] if s == 0 and b < len(nodes) else 0) for b, n in enumerate(lens)]
        assert s in ((0, 1) if sum(nodes) == 0 else (0, 2, 3)) and [B.dbt_kv_length(kv, b) for b in range(6)] == grown
        if s == 0:
            for b in range(len(nodes)):
                held = B.dbt_kv_pages(kv, b)
                assert list(table[b * p.mpps:][:len(held)]) == held
            paths = [sorted(rng.sample(range(n), rng.randint(0, n))) for n in nodes]
            assert p.status(B.dbt_kv_keep, kv, t, B.make_paths(paths), 0) == 0
            for b, q in enumerate(paths):
                assert B.dbt_kv_length(kv, b) == lens[b] + len(q)
        owners = [x for b in range(6) for x in B.dbt_kv_pages(kv, b)]
        assert len(owners) == len(set(owners)) == sum((B.dbt_kv_length(kv, b) + 15) // 16 for b in range(6))
        if rng.random() < 0.3:
            b = rng.randrange(6)
            B.dbt_kv_truncate(kv, b, rng.randint(0, B.dbt_kv_length(kv, b)))


if __name__ == "__main__":
    sys.path.insert(0, ROOT)
    fk = ctypes.CDLL(sys.argv[2])
    name = sys.argv[1]
    if name.startswith("failing_"):
        failing(fk, name[8:])
    else:
        tables(fk)
    print("done")
