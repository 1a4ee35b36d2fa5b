"""Draws whose random number falls exactly between two tokens: the running sum
has to exceed u times the sum, so the token behind the border is the one."""
import numpy as np
import pytest

from tests.test_gpu_sample import call

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nb", [0, 1])
@pytest.mark.parametrize("params", [(1.0, 0, 1.0, 0.0), (0.7, 0, 1.0, 0.0), (3.0, 0, 1.0, 0.85)])
@pytest.mark.parametrize("V,copies,at", [(4096, 2, 1), (50000, 2, 1), (8192, 4, 1), (8192, 4, 3), (131072, 16, 5), (1 << 20, 8, 7)])
def test_sums_that_meet_the_random_number(V, copies, at, params, nb):
    """Rows of equal stretches of tokens, u = at / copies: the sum of the first `at`
    stretches is u times the whole, whatever the weights, and its sum has more bits
    than a float64's fraction."""
    rng = np.random.default_rng(V + at)
    R = 8 if V > 100000 else 48

    def rows():
        return np.tile(rng.uniform(-0.5, 0.5, (R, V // copies)).astype(np.float32), (1, copies))

    z1 = rows()
    zb = rows()[None] if nb else None
    alpha = rng.uniform(0.5, 1.0, R).astype(np.float32) if nb else None
    token, _ = call(z1, zb, alpha, np.full(R, at / copies, np.float32), [params] * R)
    m = np.exp(z1[:, :V // copies].astype(np.float64))
    m /= m.sum(1, keepdims=True)
    if nb:
        q = np.exp(zb[0, :, :V // copies].astype(np.float64))
        m = alpha[:, None] * m + (1.0 - alpha[:, None]) * q / q.sum(1, keepdims=True)
    w = (m / m.max(1, keepdims=True)) ** (1.0 / params[0])
    # the first token of the stretch that min-p leaves (no weight is near it)
    assert np.abs(w - params[3]).min() > 1e-9
    first = (w >= params[3]).argmax(1)
    assert (token == V // copies * at + first).all(), token
