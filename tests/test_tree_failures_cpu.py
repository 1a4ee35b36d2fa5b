"""Kept paths on the stand-in for the HIP runtime: a call of several launches that
fails in between, and the pages that come back."""
import ctypes
import os
import subprocess
import sys

import pytest

from tests.test_launches_cpu import FAKE, ROOT, Program, fake  # noqa: F401

NO_PAGES, HIP = 3, 6


def run_child(fake, name):  # noqa: F811
    pre = " ".join(x for x in (fake, os.environ.get("LD_PRELOAD", "")) if x)
    r = subprocess.run([sys.executable, __file__, name, fake], capture_output=True, text=True, cwd=ROOT, timeout=300,
                       env=dict(os.environ, LD_PRELOAD=pre, PYTHONPATH=ROOT))
    assert r.returncode == 0 and "done" in r.stdout, (r.stdout + r.stderr)[-3000:]


@pytest.mark.parametrize("name", ["launches", "pages"])
def test_kept_paths(fake, name):  # noqa: F811
    run_child(fake, name)


# ---------------------------------------------------------------------------
# in the child
# ---------------------------------------------------------------------------

def launches(fk):
    """70 sequences whose nodes move, 32 a launch, among some whose nodes stay in
    place: wherever a launch fails, the sequences whose nodes were moved by an
    earlier one have ended at their paths and the others are as they were, and
    the rest of them can be kept by another call."""
    B_, moved = 80, [b for b in range(80) if b % 8 != 5]
    p = Program("f32", max_batch=B_)
    B = p.B
    kv, _table = p.cache(pages=200, nseq=B_)
    nodes = [20] * B_
    paths = [[1, 3] if b in moved else [0, 1] for b in range(B_)]
    t = B.make_tree(nodes)

    def held():
        return [(B.dbt_kv_length(kv, b), B.dbt_kv_pages(kv, b)) for b in range(B_)]

    def grow():
        for b in range(B_):
            B.dbt_kv_truncate(kv, b, 0)
        for b in range(B_):
            B.dbt_kv_reserve(kv, b, 25)

    fk.fake_reset(-1)
    grow()
    before = held()
    assert p.status(B.dbt_kv_keep, kv, t, B.make_paths(paths), 0) == 0
    names = [fk.fake_kernel(i).decode() for i in range(fk.fake_launches())]
    keeps = [i for i, n in enumerate(names) if "k_tree_keep" in n]
    assert len(keeps) == 3 and keeps[-1] == len(names) - 1
    after = held()
    assert all(n == 7 and len(pages) == 1 for n, pages in after)
    for at in range(len(names)):
        fk.fake_reset(-1)
        grow()
        assert held() == before
        fk.fake_reset(at)
        assert p.status(B.dbt_kv_keep, kv, t, B.make_paths(paths), 0) == HIP
        n = 32 * sum(i < at for i in keeps)  # sequences moved by the launches before
        end = moved[n - 1] + 1 if n else 0
        now = held()
        assert now == after[:end] + before[end:], at
        fk.fake_reset(-1)
        rest = [0] * end + nodes[end:]
        assert p.status(B.dbt_kv_keep, kv, B.make_tree(rest), B.make_paths([[]] * end + paths[end:]), 0) == 0
        assert held() == after


def pages(fk):
    """A pool of exactly the pages that the sequences hold: what a keep gives back,
    and no page more, can be taken again."""
    p = Program("f32", max_batch=4)
    B = p.B
    kv, _table = p.cache(pages=9, nseq=4)
    fk.fake_reset(-1)
    for b, n in enumerate((40, 33, 48)):
        B.dbt_kv_reserve(kv, b, n)
    assert p.status(B.dbt_kv_reserve, kv, 3, 1) == NO_PAGES
    held = [B.dbt_kv_pages(kv, b) for b in range(3)]
    t = B.make_tree([30, 2, 40])  # positions 10, 31 and 8 before the nodes
    assert p.status(B.dbt_kv_keep, kv, t, B.make_paths([[0, 4, 20], [1], []]), 0) == 0
    assert [B.dbt_kv_length(kv, b) for b in range(3)] == [13, 32, 8]
    assert [B.dbt_kv_pages(kv, b) for b in range(3)] == [held[0][:1], held[1][:2], held[2][:1]]
    back = sorted(held[0][1:] + held[1][2:] + held[2][1:])
    assert len(back) == 5
    assert p.status(B.dbt_kv_reserve, kv, 3, 6 * 16) == NO_PAGES
    assert B.dbt_kv_reserve(kv, 3, 5 * 16) == back
    assert p.status(B.dbt_kv_reserve, kv, 3, 5 * 16 + 1) == NO_PAGES


if __name__ == "__main__":
    sys.path.insert(0, ROOT)
    fk = ctypes.CDLL(sys.argv[2])
    fk.fake_kernel.restype = ctypes.c_char_p
    {"launches": launches, "pages": pages}[sys.argv[1]](fk)
    print("done")
