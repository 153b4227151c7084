"""Token scores on the GPU (log probability of given tokens, entropy, top alternatives, gradient) against the fp64
definitions.

Tolerances, from the arithmetic of one pass in fp32 with V logits per row.  Differences to the maximum are rounded once
(2^-24), each exponential carries the rounding of its argument (2^-24 of it, twice) and the two units of the exponential
itself; a thread adds V / 512 of them and the partial sums meet in a dozen more steps.  With A = E |u - max u| under p,
    e_sum = 2^-21 + (V / 512 + 32) 2^-24 + 2^-22 A
bounds the relative error of the sum S, hence the absolute one of its logarithm, and of T = E (u - max u) relative to A:
    log probability:  e_sum + 2^-22 (|u_t - max u| + ln S + 1)
    entropy:          e_sum (1 + 2 A) + 2^-22 (ln S + A)
A gradient is a product of p (relative error e_sum + 2^-22 (|log p| + 1)) with sums of the given gradients:
    scale p (|g_lp| + |g_H| (|log p| + H)) (2 e_sum + 2^-21 (|log p| + 2)) + scale p |g_H| tol(H) + 2^-22 scale |g_lp| at the target
and, for bf16 logits, one rounding to bf16 (2^-8 of the value)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2505_11204_b200 import build, randes    # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def definition(z, targets, scale):
    """(u, log p, p, H, max, lnS) in fp64 for rows that have something left."""
    u = z.astype(np.float64) * float(np.float32(scale))
    m = u.max(1, keepdims=True)
    e = np.exp(u - m)
    s = e.sum(1, keepdims=True)
    lp = u - m - np.log(s)
    p = e / s
    h = -(p * np.where(p > 0, lp, 0)).sum(1)
    return u, lp, p, h, m[:, 0], np.log(s[:, 0])


def e_sum(u, p, m):
    a = (p * np.where(p > 0, m[:, None] - u, 0)).sum(1)
    return 2.0 ** -21 + (u.shape[1] / 512 + 32) * 2.0 ** -24 + 2.0 ** -22 * a, a


def tol_entropy(u, p, m, ln):
    e, a = e_sum(u, p, m)
    return e * (1 + 2 * a) + 2.0 ** -22 * (ln + a)


def make(rng, n, vocab, dtype, sharp=True):
    z = (rng.standard_normal((n, vocab)) * 2.5).astype(np.float32)
    t = rng.integers(0, vocab, size=n)
    if sharp:
        z[np.arange(0, n, 2), t[::2]] += 9
    z = torch.from_numpy(z).to(TYPES[dtype])
    return z.float().numpy(), z.cuda(), t, torch.from_numpy(t).cuda()


def check_scores(z, t, r, scale, top_k):
    n, vocab = z.shape
    u, lp, p, h, m, ln = definition(z, t, scale)
    e, _ = e_sum(u, p, m)
    rows = np.arange(n)
    if r.logprob is not None:
        err, tol = np.abs(r.logprob.cpu().numpy() - lp[rows, t]), e + 2.0 ** -22 * (m - u[rows, t] + ln + 1)
        assert (err <= tol).all(), "log probability: worst %.3g x tolerance" % float((err / tol).max())
    err, tol = np.abs(r.entropy.cpu().numpy() - h), tol_entropy(u, p, m, ln)
    assert (err <= tol).all(), "entropy: worst %.3g x tolerance" % float((err / tol).max())
    if top_k:
        k = min(top_k, vocab)
        order = np.argsort(-z, axis=1, kind="stable")[:, :k]
        ids, tops = r.top_ids.cpu().numpy(), r.top_logprobs.cpu().numpy()
        assert np.array_equal(ids[:, :k], order)
        want = np.take_along_axis(lp, order, 1)
        tol = e[:, None] + 2.0 ** -22 * (np.take_along_axis(m[:, None] - u, order, 1) + ln[:, None] + 1)
        assert (np.abs(tops[:, :k] - want) <= tol).all()
        assert (ids[:, k:] == -1).all() and (tops[:, k:] == -np.inf).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(1, 1), (3, 2), (2, 7), (5, 64), (1, 513), (4, 1000), (3, 4099), (1, 50257), (7, 32128), (200, 777), (2, 131072), (1, 100003)])
def test_scores_against_the_definition(n, vocab, dtype):
    rng = np.random.default_rng(n * 1000003 + vocab)
    z, zd, t, td = make(rng, n, vocab, dtype)
    for scale, top_k in ((1.0, 5), (0.7, 64), (2.5, 0), (1.0, 1)):
        check_scores(z, t, randes.token_scores(zd, td, top_k=top_k, scale=scale), scale, top_k)
    r = randes.token_scores(zd, top_k=3)
    assert r.logprob is None
    check_scores(z, t, r, 1.0, 3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_and_misaligned_rows(dtype):
    rng = np.random.default_rng(1)
    n, vocab = 6, 5003
    z, zd, t, td = make(rng, n, vocab, dtype)
    for off, pad in ((0, 1), (1, 0), (3, 5), (5, 8), (0, 13)):
        store = torch.full((off + n * (vocab + pad),), float("nan"), device="cuda", dtype=TYPES[dtype])
        v = store[off:].view(n, vocab + pad)[:, :vocab]
        v.copy_(zd)
        r = randes.token_scores(v, td, top_k=9, scale=0.9)
        check_scores(z, t, r, 0.9, 9)
        g = torch.randn(n, device="cuda")
        out = torch.full((n, vocab + 3), -7.0, device="cuda", dtype=TYPES[dtype])
        randes.token_scores_backward(v, td, r, g, g, scale=0.9, out=out[:, 2:2 + vocab])
        assert torch.equal(out[:, 2:2 + vocab], randes.token_scores_backward(zd, td, r, g, g, scale=0.9))
        assert (out[:, :2] == -7).all() and (out[:, 2 + vocab:] == -7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(1, 32128), (40, 20000)])
def test_equal_logits_are_ordered_by_index(n, vocab, dtype):
    rng = np.random.default_rng(2)
    flat = np.zeros((n, vocab), dtype=np.float32)                                   # every logit the same
    few = rng.integers(0, 4, size=(n, vocab)).astype(np.float32)                    # thousands of equals at the top
    late = np.where(np.arange(vocab) >= vocab - 70, 3.0, -1.0).astype(np.float32) * np.ones((n, 1), dtype=np.float32)
    signed = np.where(rng.random((n, vocab)) < 0.5, 0.0, -0.0).astype(np.float32)   # both zeros are equal
    for z in (flat, few, late, signed):
        t = rng.integers(0, vocab, size=n)
        zd = torch.from_numpy(z).to(TYPES[dtype]).cuda()
        for k in (1, 8, 64):
            check_scores(z, t, randes.token_scores(zd, torch.from_numpy(t).cuda(), top_k=k), 1.0, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [50, 3000, 40001])
def test_masked_logits_and_rows_with_nothing_left(vocab, dtype):
    rng = np.random.default_rng(3)
    n = 6
    z, _, t, td = make(rng, n, vocab, dtype, sharp=False)
    low = float(torch.finfo(TYPES[dtype]).min)
    z[0, rng.permutation(vocab)[: vocab - 3]] = -np.inf      # three tokens left
    z[1, :] = -np.inf                                        # none
    z[2, :] = low                                            # all of the type's lowest value: uniform
    z[3, rng.permutation(vocab)[: vocab // 2]] = low         # half of it masked by that value
    z[4, :] = -np.inf
    z[4, vocab - 1] = 1.5                                    # one
    z[0, t[0]], z[3, t[3]] = 2.0, 1.0
    zd = torch.from_numpy(z).to(TYPES[dtype]).cuda()
    z = zd.float().cpu().numpy()
    r = randes.token_scores(zd, td, top_k=7)
    keep = [0, 2, 3, 5]
    with np.errstate(all="ignore"):
        sub = randes.TokenScores(r.logprob[keep], r.entropy[keep], r.stats[:, keep], r.top_ids[keep], r.top_logprobs[keep])
        u, lp, p, h, m, ln = definition(z[keep], t[keep], 1.0)
        lp = np.where(np.isnan(lp), -np.inf, lp)
        e, _ = e_sum(np.where(np.isinf(u), m[:, None] - 1, u), p, m)
        got = sub.logprob.cpu().numpy()
        assert (np.abs(got - lp[np.arange(4), t[keep]]) <= e + 2.0 ** -20 * (np.abs(lp[np.arange(4), t[keep]]) + ln + 1)).all()
        assert (np.abs(sub.entropy.cpu().numpy() - h) <= 2.0 ** -19 * (h + 1) + 2.0 ** -24 * vocab / 512).all()
    ids, tops = r.top_ids.cpu().numpy(), r.top_logprobs.cpu().numpy()
    left = np.flatnonzero(z[0] > -np.inf)
    want = left[np.argsort(-z[0, left], kind="stable")][:7]
    assert list(ids[0][: len(want)]) == list(want) and (ids[0][len(want):] == -1).all() and (tops[0][len(want):] == -np.inf).all()
    assert list(ids[2]) == list(range(min(7, vocab)))
    assert r.logprob[1].item() == -np.inf and r.entropy[1].item() == 0 and (ids[1] == -1).all() and (tops[1] == -np.inf).all()
    assert ids[4][0] == vocab - 1 and tops[4][0] == 0 and (ids[4][1:] == -1).all() and r.entropy[4].item() == 0
    g = torch.ones(n, device="cuda")
    grad = randes.token_scores_backward(zd, td, r, g, g)
    assert torch.isfinite(grad).all()
    assert (grad[1] == 0).all() and (grad[0][torch.from_numpy(z[0]).cuda() == -np.inf] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(5, 900), (5, 33000)])
def test_nan_infinity_and_bad_targets_stay_in_their_row(n, vocab, dtype):
    rng = np.random.default_rng(4)
    z, zd, t, td = make(rng, n, vocab, dtype)
    zd[1, vocab // 2] = float("nan")
    zd[2, vocab - 1] = float("inf")
    td[3] = -100
    td[4] = vocab
    r = randes.token_scores(zd, td, top_k=4)
    for row in (1, 2):
        assert torch.isnan(r.logprob[row]) and torch.isnan(r.entropy[row]) and (r.top_ids[row] == -1).all() and torch.isnan(r.top_logprobs[row]).all()
    assert r.logprob[3].item() == 0 and torch.isnan(r.logprob[4])
    zs, ts = z[[0, 3, 4]], t[[0, 3, 4]]
    check_scores(zs, ts, randes.TokenScores(None, r.entropy[[0, 3, 4]], None, r.top_ids[[0, 3, 4]], r.top_logprobs[[0, 3, 4]]), 1.0, 4)
    g = torch.ones(n, device="cuda")
    grad = randes.token_scores_backward(zd, td, r, g, None)
    assert torch.isfinite(grad[0]).all() and (grad[3] == 0).all() and torch.isnan(grad[4]).all()


def grad_definition(z, t, scale, g_lp, g_h):
    u, lp, p, h, m, ln = definition(z, t, scale)
    one = np.zeros_like(u)
    one[np.arange(len(t)), t] = 1
    s = float(np.float32(scale))
    lpz = np.where(p > 0, lp, 0)
    return s * (g_lp[:, None] * (one - p) - g_h[:, None] * p * (lpz + h[:, None]))


def grad_tolerance(z, t, scale, g_lp, g_h, dtype):
    u, lp, p, h, m, ln = definition(z, t, scale)
    e, _ = e_sum(u, p, m)
    s = float(np.float32(scale))
    a = np.abs(np.where(p > 0, lp, 0))
    tol = s * p * (np.abs(g_lp)[:, None] + np.abs(g_h)[:, None] * (a + h[:, None])) * (2 * e[:, None] + 2.0 ** -21 * (a + 2))
    tol += s * p * np.abs(g_h)[:, None] * tol_entropy(u, p, m, ln)[:, None]
    tol[np.arange(len(t)), t] += 2.0 ** -22 * s * np.abs(g_lp)
    tol += 2.0 ** -126
    return tol + (2.0 ** -8 * np.abs(grad_definition(z, t, scale, g_lp, g_h)) if dtype == "bf16" else 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(1, 1), (2, 7), (3, 1000), (5, 4099), (2, 50257), (300, 129)])
def test_gradient_against_the_formula(n, vocab, dtype):
    rng = np.random.default_rng(vocab)
    z, zd, t, td = make(rng, n, vocab, dtype)
    for scale, use in ((1.0, "both"), (0.6, "lp"), (1.7, "h")):
        g_lp, g_h = (rng.standard_normal(n).astype(np.float32) for _ in range(2))
        r = randes.token_scores(zd, td, scale=scale)
        gl, gh = (torch.from_numpy(g).cuda() for g in (g_lp, g_h))
        got = randes.token_scores_backward(zd, td, r, gl if use != "h" else None, gh if use != "lp" else None, scale=scale)
        a, b = (g_lp if use != "h" else 0 * g_lp).astype(np.float64), (g_h if use != "lp" else 0 * g_h).astype(np.float64)
        err, tol = np.abs(got.float().cpu().numpy() - grad_definition(z, t, scale, a, b)), grad_tolerance(z, t, scale, a, b, dtype)
        assert (err <= tol).all(), "%s: worst %.3g x tolerance" % (use, float((err / tol).max()))
        inplace = zd.clone()
        assert randes.token_scores_backward(inplace, td, r, gl, gh, scale=scale, out=inplace) is inplace
        assert torch.equal(inplace, randes.token_scores_backward(zd, td, r, gl, gh, scale=scale))


def test_gradient_against_differences():
    rng = np.random.default_rng(6)
    n, vocab, scale, step = 3, 11, 0.8, 1e-4
    z, zd, t, td = make(rng, n, vocab, "f32", sharp=False)
    g_lp, g_h = (rng.standard_normal(n).astype(np.float32) for _ in range(2))
    r = randes.token_scores(zd, td, scale=scale)
    got = randes.token_scores_backward(zd, td, r, torch.from_numpy(g_lp).cuda(), torch.from_numpy(g_h).cuda(), scale=scale).cpu().numpy()

    def loss(v):
        _, lp, _, h, _, _ = definition(v, t, scale)
        return float((g_lp * lp[np.arange(n), t]).sum() + (g_h * h).sum())

    tol = grad_tolerance(z, t, scale, g_lp.astype(np.float64), g_h.astype(np.float64), "f32") + 1e-6     # central differences: step^2 times a third derivative of a few units
    for i in range(n):
        for j in range(vocab):
            hi, lo = z.astype(np.float64), z.astype(np.float64)
            hi[i, j] += step
            lo[i, j] -= step
            d = (loss(hi) - loss(lo)) / (2 * step)
            assert abs(d - got[i, j]) <= tol[i, j], (i, j, d, got[i, j])


def test_empty_calls():
    r = randes.token_scores(torch.zeros(0, 10, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), top_k=2)
    assert r.logprob.shape == (0,) and r.top_ids.shape == (0, 2)
    r = randes.token_scores(torch.zeros(3, 0, device="cuda"), top_k=2)
    assert (r.entropy == 0).all() and (r.top_ids == -1).all()


def test_refusals():
    inv, mis = randes.INVALID_ARGUMENT, randes.MISALIGNED

    def refused(code, fn):
        with pytest.raises(randes.RandesError) as e:
            fn()
        assert e.value.code == code, (e.value.code, str(e.value))

    z = torch.randn(4, 100, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    r = randes.token_scores(z, t)
    g = torch.ones(4, device="cuda")
    before = randes.randes_launch_count()
    refused(randes.UNSUPPORTED_DTYPE, lambda: randes.token_scores(z.half(), t))
    refused(inv, lambda: randes.token_scores(z.t(), t))
    refused(inv, lambda: randes.token_scores(z, t[:3]))
    refused(inv, lambda: randes.token_scores(z, t.int()))
    refused(inv, lambda: randes.token_scores(z, t, top_k=65))
    refused(inv, lambda: randes.token_scores(z, t, scale=0.0))
    refused(inv, lambda: randes.token_scores(z, t, scale=float("nan")))
    refused(inv, lambda: randes.token_scores(z, t, scale=-1.0))
    refused(inv, lambda: randes.token_scores(z[:1].expand(4, 100), t))
    refused(inv, lambda: randes.token_scores_backward(z, t, r, g[:1].expand(4), None))
    refused(inv, lambda: randes.token_scores_backward(z, t, r, g.double(), None))
    refused(inv, lambda: randes.token_scores_backward(z, None, r, g, None))
    refused(inv, lambda: randes.token_scores_backward(z, t, r, g, None, out=torch.empty(4, 99, device="cuda")))
    refused(inv, lambda: randes.token_scores_backward(z[:3], t[:3], r, g[:3], None))
    s = torch.cuda.current_stream().cuda_stream
    st = r.stats.data_ptr()
    refused(inv, lambda: randes.randes_token_scores(z, 0, 4, 100, 99, t, 1.0, 0, g, g, st, None, None, s))
    refused(inv, lambda: randes.randes_token_scores(z, 0, 4, 100, 100, t, 1.0, 0, None, g, st, None, None, s))
    refused(inv, lambda: randes.randes_token_scores(z, 0, 4, 100, 100, t, 1.0, 3, g, g, st, None, None, s))
    refused(inv, lambda: randes.randes_token_scores(None, 0, 4, 100, 100, t, 1.0, 0, g, g, st, None, None, s))
    refused(mis, lambda: randes.randes_token_scores(z.data_ptr() + 2, 0, 4, 100, 100, t, 1.0, 0, g, g, st, None, None, s))
    refused(mis, lambda: randes.randes_token_scores(z, 0, 4, 100, 100, t.data_ptr() + 4, 1.0, 0, g, g, st, None, None, s))
    # a gradient shifted into the logits' memory would be read after it is written
    big = torch.randn(5, 100, device="cuda")
    refused(inv, lambda: randes.randes_token_scores_backward(big, 0, 4, 100, 100, t, 1.0, st, g, g, None, big.data_ptr() + 400, 100, s))
    assert randes.randes_launch_count() == before


def range_tolerance(z, t, scale, g_lp, g_h, dtype):
    """grad_tolerance where u spans more than fp32's exponentials: a p below 2^-126 may come out as 0, and what multiplies it
    is the bracket of the formula."""
    u, lp, p, h, m, ln = definition(z, t, scale)
    a = np.abs(np.where(p > 0, lp, 0))
    flushed = float(np.float32(scale)) * 2.0 ** -126 * (np.abs(g_lp)[:, None] + np.abs(g_h)[:, None] * (a + h[:, None]))
    return grad_tolerance(z, t, scale, g_lp, g_h, dtype) + flushed


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-6, 1.0, 2e4, 1e6])
@pytest.mark.parametrize("mask", ["-inf", "lowest"])
def test_gradient_at_masked_logits_for_every_scale(mask, scale, dtype):
    rng = np.random.default_rng(7)
    n, vocab = 5, 3001
    z, _, t, td = make(rng, n, vocab, dtype)
    value = -np.inf if mask == "-inf" else float(torch.finfo(TYPES[dtype]).min)
    masked = rng.random((n, vocab)) < 0.3
    masked[np.arange(n), t] = False
    masked[4] = True                                       # one token left
    masked[4, t[4]] = False
    z[masked] = value
    zd = torch.from_numpy(z).to(TYPES[dtype]).cuda()
    z = zd.float().cpu().numpy()
    r = randes.token_scores(zd, td, scale=scale)
    zero = torch.from_numpy(masked).cuda()
    with np.errstate(invalid="ignore"):
        for loss_scale in (1.0, 65536.0):
            g_lp, g_h = (loss_scale * rng.standard_normal(n).astype(np.float32) for _ in range(2))
            got = randes.token_scores_backward(zd, td, r, torch.from_numpy(g_lp).cuda(), torch.from_numpy(g_h).cuda(), scale=scale).float()
            assert torch.isfinite(got).all(), "%d of %d elements are no numbers" % (int((~torch.isfinite(got)).sum()), got.numel())
            a, b = g_lp.astype(np.float64), g_h.astype(np.float64)
            err, tol = np.abs(got.cpu().numpy() - grad_definition(z, t, scale, a, b)), range_tolerance(z, t, scale, a, b, dtype)
            assert (err <= tol).all(), "worst %.3g x tolerance" % float((err / tol).max())
            if mask == "-inf" or scale * -value > 1e9:     # (lowest value times 1e-6 is masked as well)
                assert (got[zero] == 0).all()
    # whatever the gradients: nothing comes back through a token of probability 0
    for big in (3e38, -3e38):
        g = torch.full((n,), big, device="cuda")
        for pair in ((g, g), (g, None), (None, g)):
            got = randes.token_scores_backward(zd, td, r, *pair, scale=scale)
            assert (got[zero] == 0).all(), "%d of %d masked elements are not 0" % (int((got[zero] != 0).sum()), int(zero.sum()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-6, 0.5, 1.0, 3.0, 1e6])
@pytest.mark.parametrize("vocab", [37, 5000, 40001])
def test_one_logit_near_the_greatest_number(vocab, scale, dtype):
    rng = np.random.default_rng(8)
    n = 6
    z, _, t, _ = make(rng, n, vocab, dtype, sharp=False)
    top = rng.integers(0, vocab, size=n)
    z[np.arange(n), top] = [3e38, 2.5e38, float(torch.finfo(TYPES[dtype]).max), 1e38, 1e33, 2e30]      # (a token that is forced)
    t[::2] = top[::2]
    zd, td = torch.from_numpy(z).to(TYPES[dtype]).cuda(), torch.from_numpy(t).cuda()
    z = zd.float().cpu().numpy()
    r = randes.token_scores(zd, td, top_k=3, scale=scale)
    u, lp, p, h, m, ln = definition(z, t, scale)
    assert (p[np.arange(n), top] == 1).all()
    assert (r.entropy == 0).all(), r.entropy
    want = lp[np.arange(n), t]
    with np.errstate(over="ignore"):
        want32 = want.astype(np.float32)                   # -inf where fp32 has no such number
    got, tol = r.logprob.cpu().numpy(), 2.0 ** -21 * (np.abs(want) + 1)
    assert ((np.abs(got - want) <= tol) | (np.isinf(want32) & (got == want32))).all(), (got, want)
    assert np.array_equal(r.top_ids.cpu().numpy(), np.argsort(-z, axis=1, kind="stable")[:, :3]) and (r.top_logprobs[:, 0] == 0).all()
    g_lp, g_h = (rng.standard_normal(n).astype(np.float32) for _ in range(2))
    gl, gh = torch.from_numpy(g_lp).cuda(), torch.from_numpy(g_h).cuda()
    for a, b in ((gl, gh), (gl, None), (None, gh)):
        x, y = (np.zeros(n) if g is None else g.double().cpu().numpy() for g in (a, b))
        grad = randes.token_scores_backward(zd, td, r, a, b, scale=scale).float().cpu().numpy()
        err, tol = np.abs(grad - grad_definition(z, t, scale, x, y)), range_tolerance(z, t, scale, x, y, dtype)
        assert (err <= tol).all(), "worst %.3g x tolerance" % float(np.nanmax(err / tol))


def test_the_entropy_is_not_read_without_its_gradient():
    rng = np.random.default_rng(9)
    z, zd, t, td = make(rng, 4, 300, "f32")
    r = randes.token_scores(zd, td)
    g = torch.ones(4, device="cuda")
    want = randes.token_scores_backward(zd, td, r, g, None)
    stats = r.stats.clone()
    stats[1] = float("nan")
    spoilt = randes.TokenScores(stats[0], stats[1], stats, None, None)
    assert torch.equal(randes.token_scores_backward(zd, td, spoilt, g, None), want) and torch.isfinite(want).all()
