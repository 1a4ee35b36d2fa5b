"""Measured operators (perf/operators.py): passes over kept paths can follow each
other on one cache and leave what the plain form's passes leave."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def cases():
    from perf import operators as o
    rng = random.Random(11)
    found = [c for c in o.listed() if c["op"] == "keep"]
    while len(found) < 8:
        c = o.draw(rng)
        if c["op"] == "keep":
            found.append(c)
    # sequences that drop most of their pages, one without a node among them
    found.append(dict(op="keep", heads="shard", layers=2, batch=5, lo=0, hi=20, nlo=0, nhi=64))
    return found


@pytest.mark.parametrize("i", range(9))
def test_passes_over_kept_paths_repeat(i, monkeypatch):
    from perf import operators as o
    case = cases()[i]
    print(case, flush=True)
    plain = o.prepare(case, 5)
    monkeypatch.setattr(o, "own", True)
    lib = o.prepare(case, 5)
    assert torch.equal(plain.k, lib.k) and torch.equal(plain.v, lib.v)
    for _ in range(3):
        got = o.run(lib)
        monkeypatch.setattr(o, "own", False)
        want = o.run(plain)
        monkeypatch.setattr(o, "own", True)
        torch.cuda.synchronize()
        assert torch.equal(got["k"], want["k"]) and torch.equal(got["v"], want["v"])
