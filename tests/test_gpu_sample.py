"""Tokens drawn from the mixture against the definition in float64: tokens
equal, probabilities within their float32 rounding."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NONE = (1.0, 0, 1.0, 0.0)


def softmax(z):
    e = np.exp(z - z.max())
    return e / e.sum()


def definition(z1, zb, alpha, u, params):
    """Token and probability of one row; weights relative to the largest."""
    t, k, top_p, min_p = params
    t, top_p, min_p = (float(np.float32(x)) for x in (t, top_p, min_p))
    z1 = z1.astype(np.float64)
    if len(zb):
        m = float(alpha) * softmax(z1) + (1 - float(alpha)) * np.mean([softmax(z.astype(np.float64)) for z in zb], axis=0)
    else:
        m = np.exp(z1 - z1.max())
    r = m / m.max()
    if t == 0:
        return int(np.argmax(r)), 1.0
    with np.errstate(divide="ignore"):
        w = r if t == 1 else np.exp(np.log(r) / t)
    order = np.argsort(-r, kind="stable")
    if 0 < k < len(order):
        order = order[:k]
    c = np.cumsum(w[order])
    if top_p < 1:
        order = order[:int(np.searchsorted(c, top_p * c[-1])) + 1]
    stay = np.zeros(len(r), bool)
    stay[order] = True
    stay &= w >= min_p
    w = np.where(stay, w, 0.0)
    c = np.cumsum(w)
    i = int(np.searchsorted(c, float(u) * c[-1], side="right"))
    return i, w[i] / c[-1]


def call(z1, zb, alpha, u, params, stream=None):
    from paper_2608_12385_amd import binding as B
    R, V = z1.shape
    z1d, ud = torch.from_numpy(z1).cuda(), torch.from_numpy(u).cuda()
    zd = torch.from_numpy(zb).cuda() if zb is not None else None
    ad = torch.from_numpy(alpha).cuda() if zb is not None else None
    token = torch.full((R + 2,), -9, dtype=torch.int32, device="cuda")
    prob = torch.full((R + 2,), -9.0, device="cuda")
    ws = torch.full((B.dbt_sample_workspace_bytes(R, V),), 0xff, dtype=torch.uint8, device="cuda")
    sin = B.dbt_sample_in(logits1=z1d.data_ptr(), logits2=zd.data_ptr() if zb is not None else None,
                          alpha=ad.data_ptr() if zb is not None else None, u=ud.data_ptr(),
                          h_params=B.make_sampling(params), rows=R, vocab=V, n_branches=0 if zb is None else zb.shape[0])
    torch.cuda.synchronize()
    B.dbt_sample(sin, token.data_ptr(), prob.data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    token, prob = token.cpu().numpy(), prob.cpu().numpy()
    assert (token[R:] == -9).all() and (prob[R:] == -9).all()
    return token[:R], prob[:R]


def check(z1, zb, alpha, u, params):
    token, prob = call(z1, zb, alpha, u, params)
    for r in range(len(u)):
        t, p = definition(z1[r], [] if zb is None else zb[:, r], None if zb is None else alpha[r], u[r], params[r])
        assert token[r] == t, (r, params[r], int(token[r]), t)
        # float32 rounding, and the weights' step (2^-42 of the largest) in each of the two
        assert abs(prob[r] - p) <= p * 2.0 ** -24 + 2.0 ** -40, (r, prob[r], p)
    return token


def logits(rng, R, V, nb, std=3.0):
    z1 = (std * rng.standard_normal((R, V))).astype(np.float32)
    z1 -= 2.0 * np.log1p(rng.random((R, V)).astype(np.float32) * V) * rng.random((R, 1)).astype(np.float32)
    zb = (z1 + rng.standard_normal((nb, R, V))).astype(np.float32) if nb else None
    alpha = rng.uniform(0.5, 1.0, R).astype(np.float32) if nb else None
    return z1, zb, alpha


KINDS = [NONE, (0.0, 0, 1.0, 0.0), (0.7, 50, 0.95, 0.0), (1.0, 0, 0.9, 0.0), (1.3, 0, 1.0, 0.05), (1.0, 1, 1.0, 0.0),
         (0.3, 1000, 0.99, 1e-3), (2.5, 7, 0.5, 0.2), (1.0, 0, 1e-6, 0.0), (1.0, 0, 1.0, 1.0), (0.05, 0, 0.999, 0.0),
         (1.0, 3, 1.0, 0.0), (5.0, 0, 0.97, 0.0), (1.7, 40, 1.0, 0.0)]


@pytest.mark.parametrize("nb", [0, 1, 2, 3])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 1024, 2047, 2048, 2049, 16064, 50257])
def test_draws(V, nb):
    rng = np.random.default_rng(V + nb)
    R = 2 * len(KINDS)
    z1, zb, alpha = logits(rng, R, V, nb)
    u = rng.random(R).astype(np.float32)
    u[:4] = [0.0, 0.99999994, 0.5, 1e-30]
    check(z1, zb, alpha, u, KINDS * 2)


@pytest.mark.parametrize("R,V,nb", [(1, 128256, 1), (130, 4000, 1), (300, 1000, 0), (9, 128256, 0), (1, 1 << 20, 0)])
def test_rows_and_large_vocabularies(R, V, nb):
    rng = np.random.default_rng(R)
    z1, zb, alpha = logits(rng, R, V, nb)
    check(z1, zb, alpha, rng.random(R).astype(np.float32), [KINDS[r % len(KINDS)] for r in range(R)])
    if R == 1:
        for k in KINDS:
            check(z1, zb, alpha, rng.random(R).astype(np.float32), [k])


@pytest.mark.parametrize("R,V,nb", [(2100, 5000, 1), (700, 9000, 0), (520, 16385, 0)])
def test_parts_of_several_tiles_and_many_requests(R, V, nb):
    """Rows enough to fill the chip (parts of two to four tiles), over 2048 of
    them, over 96 different parameters."""
    rng = np.random.default_rng(R)
    z1, zb, alpha = logits(rng, R, V, nb)
    kinds = KINDS + [(0.5 + 0.01 * i, 5 + i, 0.8, 0.0) for i in range(150)]
    check(z1, zb, alpha, rng.random(R).astype(np.float32), [kinds[int(i)] for i in rng.integers(0, len(kinds), R)])


@pytest.mark.parametrize("V", [5, 3000, 40000])
@pytest.mark.parametrize("nb", [0, 1])
def test_ties(V, nb):
    """Equal weights go by index: all of them, a few levels, and a level that
    fills the class of the cut."""
    rng = np.random.default_rng(V)
    rows = [np.zeros(V), rng.integers(0, 3, V), np.where(np.arange(V) % 7 == 0, 2.0, 1.0), -np.arange(V) // 4 * 0.25]
    kinds = [(1.0, max(1, V // 2), 1.0, 0.0), (1.0, 0, 0.5, 0.0), (1.0, max(1, V - 1), 0.25, 0.0), NONE, (0.0, 0, 1.0, 0.0),
             (1.0, V + 10, 0.875, 0.0), (1.0, 0, 1.0, 1.0), (0.5, 2, 0.5, 0.0), (1.0, min(V, 2500), 1.0, 0.0)]
    z = np.stack([r for r in rows for _ in kinds]).astype(np.float32)
    R = len(z)
    zb = np.stack([z]) if nb else None
    check(z, zb, np.full(R, 0.5, np.float32) if nb else None, rng.random(R).astype(np.float32), kinds * len(rows))


@pytest.mark.parametrize("spread", [1e-3, 1e-5, 0.05])
def test_nearly_flat_rows(spread):
    """Every weight in one class of the histogram, tens of thousands of them."""
    rng = np.random.default_rng(2)
    V, kinds = 60000, [(1.0, 30000, 1.0, 0.0), (1.0, 0, 0.4, 0.0), (1.0, 20000, 0.7, 0.0), (0.8, 0, 0.6, 0.99), NONE]
    z = (spread * rng.standard_normal((len(kinds) * 2, V))).astype(np.float32)
    check(z, None, None, rng.random(len(z)).astype(np.float32), kinds * 2)


@pytest.mark.parametrize("nb", [0, 1])
@pytest.mark.parametrize("min_p", [1e-6, 0.02, 0.3, 0.7, 1.0])
def test_min_p_before_between_and_behind_the_other_cuts(min_p, nb):
    rng = np.random.default_rng(12)
    V, kinds = 20000, [(1.0, 700, 1.0, min_p), (1.0, 700, 0.5, min_p), (1.0, 0, 0.6, min_p), (1.5, 9000, 0.05, min_p),
                       (1.0, 1, 1.0, min_p), (0.7, 12000, 0.99, min_p), (1.0, 0, 1.0, min_p)]
    z1, zb, alpha = logits(rng, 2 * len(kinds), V, nb)
    check(z1, zb, alpha, rng.random(len(z1)).astype(np.float32), kinds * 2)


@pytest.mark.parametrize("nb", [0, 1, 2, 3])
@pytest.mark.parametrize("t", [1e-3, 1e-7, 1e-13, 1e-30, 1e-45])
def test_the_smallest_temperatures(t, nb):
    """The largest weight stays one, whatever its logarithm is multiplied with:
    those of the rows' seconds are below 2^-46 from 1e-3 on."""
    rng = np.random.default_rng(13)
    z1, zb, alpha = logits(rng, 12, 3000, nb)
    z1[:, 100] += 60
    if nb:
        zb[:, :, 100] += 60
    u = rng.random(12).astype(np.float32)
    token, prob = call(z1, zb, alpha, u, [(t, 0, 1.0, 0.0), (t, 5, 0.9, 0.1)] * 6)
    assert (token == 100).all() and (prob == 1).all()


def test_masked_tokens_are_never_drawn():
    rng = np.random.default_rng(4)
    V, R = 5000, 3 * len(KINDS)
    z1, zb, alpha = logits(rng, R, V, 1)
    hide = rng.random((R, V)) < 0.9
    hide[:, 17] = False
    hide[:5] = True
    hide[:5, 4999] = False  # one token left
    z1[hide] = -np.inf
    zb[0][hide] = -np.inf
    low = np.float32(np.finfo(np.float32).min)
    z1[5:9][hide[5:9]] = low  # masked by the type's lowest value
    zb[0][5:9][hide[5:9]] = low
    token = check(z1, zb, alpha, rng.random(R).astype(np.float32), KINDS * 3)
    assert not hide[np.arange(R), token].any() and (token[:5] == 4999).all()


@pytest.mark.parametrize("nb", [0, 1, 3])
def test_rows_without_an_answer(nb):
    """A NaN, +infinity, nothing above -infinity, alpha outside [0, 1]: -1 and 0,
    the other rows as without them."""
    rng = np.random.default_rng(6)
    V, R = 3000, 12
    z1, zb, alpha = logits(rng, R, V, nb)
    u = rng.random(R).astype(np.float32)
    params = [KINDS[2 + r % 3] if r % 2 else NONE for r in range(R)]
    want = check(z1, zb, alpha, u, params)
    bad = {1: np.nan, 2: np.inf, 4: -np.inf, 7: np.nan}
    for r, x in bad.items():
        if np.isneginf(x):
            z1[r] = x
        else:
            z1[r, 2999 if r == 7 else 5] = x
    if nb:
        zb[nb - 1, 8, 1] = np.nan
        zb[0, 9] = -np.inf
        alpha[10], alpha[11], alpha[0] = np.nan, 1.5, -0.1
        bad.update({8: 0, 9: 0, 10: 0, 11: 0, 0: 0})
    token, prob = call(z1, zb, alpha, u, params)
    for r in range(R):
        assert (token[r], prob[r]) == (-1, 0.0) if r in bad else token[r] == want[r], r


def test_random_numbers_at_the_edges():
    rng = np.random.default_rng(8)
    z1, _, _ = logits(rng, 8, 500, 0)
    z1[:] = z1[0]
    lo, _ = definition(z1[0], [], None, 0.0, NONE)
    hi, _ = definition(z1[0], [], None, 0.99999994, NONE)
    for params in (NONE, (1.0, 100, 1.0, 0.0)):
        u = np.array([-1.0, np.nan, -np.inf, 0.0, 1.0, 2.0, np.inf, 0.99999994], np.float32)
        token, _ = call(z1, None, None, u, [params] * 8)
        assert (token[:4] == token[3]).all() and (token[4:] == token[7]).all()
        if params == NONE:
            assert token[0] == lo and token[7] == hi


@pytest.mark.parametrize("alpha", [0.0, 1.0])
def test_one_path_alone(alpha):
    rng = np.random.default_rng(9)
    z1, zb, a = logits(rng, len(KINDS), 7000, 1)
    check(z1, zb, np.full_like(a, alpha), rng.random(len(KINDS)).astype(np.float32), KINDS)


def test_a_rows_token_depends_on_its_row_only():
    rng = np.random.default_rng(10)
    z1, zb, alpha = logits(rng, 70, 9000, 1)
    u = rng.random(70).astype(np.float32)
    params = [KINDS[r % len(KINDS)] for r in range(70)]
    token, prob = call(z1, zb, alpha, u, params)
    for r in (0, 13, 69):
        t, p = call(z1[r:r + 1], zb[:, r:r + 1], alpha[r:r + 1], u[r:r + 1], params[r:r + 1])
        assert t[0] == token[r] and p[0] == prob[r]


def test_captured_draws():
    """Replays give the eager tokens, with eager work between them."""
    from paper_2608_12385_amd import binding as B
    R, V = 28, 20000
    rng = np.random.default_rng(11)
    z1, zb, alpha = (torch.from_numpy(x).cuda() for x in logits(rng, R, V, 1))
    u = torch.rand(R, device="cuda")
    token, prob = torch.empty(R, dtype=torch.int32, device="cuda"), torch.empty(R, device="cuda")
    ws = torch.empty(B.dbt_sample_workspace_bytes(R, V), dtype=torch.uint8, device="cuda")
    params = B.make_sampling([KINDS[r % len(KINDS)] for r in range(R)])
    sin = B.dbt_sample_in(logits1=z1.data_ptr(), logits2=zb.data_ptr(), alpha=alpha.data_ptr(), u=u.data_ptr(),
                          h_params=params, rows=R, vocab=V, n_branches=1)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()

    def run():
        B.dbt_sample(sin, token.data_ptr(), prob.data_ptr(), ws.data_ptr(), s.cuda_stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run()
    for k in range(4):
        u.uniform_()
        z1.add_(0.1 * torch.randn_like(z1))
        torch.cuda.synchronize()
        run()
        s.synchronize()
        eager = token.clone(), prob.clone()
        token.fill_(-5), prob.fill_(-5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(token, eager[0]) and torch.equal(prob, eager[1]), k


def test_a_step_answers_drawn_tokens():
    """Session.sample on a step's outputs, both paths and one."""
    import synth
    from tests.gpu_util import fill_cache, make_session, to_np
    from tests.tiny import tiny_shape
    shape = tiny_shape(vocab=300)
    W = synth.make_weights(shape, seed=0)
    sess = make_session(shape, W, max_batch=3, max_pos=64)
    fill_cache(sess, None, shape, [5, 20, 33])
    params, u = [KINDS[2], NONE, KINDS[1]], [0.3, 0.8, 0.1]
    for on in (True, False):
        t = sess.decode(tokens=[1, 2, 3], branch_on=on)
        token, prob = sess.sample(t, u, params, branch_on=on)
        for r in range(3):
            want = definition(to_np(t["logits1"])[r], [to_np(t["logits2"])[r]] if on else [], float(t["alpha"][r]), np.float32(u[r]), params[r])
            assert int(token[r]) == want[0]
            if r == 2 and on:
                assert abs(float(prob[r]) - 1.0) == 0
    sess.close()
