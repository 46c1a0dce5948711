"""GPU checks of kq_token_logprobs and its gradient against 64-bit numpy.

Bounds. e^(x - m) of an fp32 difference is off by at most 2^-21 (range below 2^7 in the exponent, two
roundings), the sums of V terms by (log2 V + 32) 2^-24 with partial sums a thread and a tree over them; with
V <= 2^18 both logs are within 2^-19 of the sum of their terms in absolute value, taken as
tol = 2^-18 (1 + |m| + |value|). A gradient is a sum of at most three products, each within 2^-18, rounded once
more to the output's type (2^-9 in bf16)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_07964_gb300 import build
    build.build()


def K():
    from paper_2607_07964_gb300 import kronq
    return kronq


def _logits(T, V, dtype, kind, rng):
    x = rng.standard_normal((T, V)) * 3
    if kind == "peaked":
        x[np.arange(T), rng.integers(0, V, T)] += 30
    if kind == "masked":
        x[rng.random((T, V)) < 0.5] = -np.inf
        x[:, V // 2] = 0.5
    if kind == "ties":
        x = np.round(x)
    if kind == "flat":
        x[:] = 1.25
    if kind == "far":
        x = x * 40 + 3000
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])


def _reference(x, target, top):
    x = x.float().numpy().astype(np.float64)
    with np.errstate(all="ignore"):
        m = x.max(1, keepdims=True)
        z = np.exp(x - m).sum(1, keepdims=True)
        lp = x - m - np.log(z)
        p = np.exp(lp)
        h = -np.where(p > 0, p * np.where(p > 0, lp, 0), 0).sum(1)
    lse = (m + np.log(z))[:, 0]
    got = np.where(target >= 0, lp[np.arange(len(x)), np.maximum(target, 0)], 0.0)
    ids = np.argsort(-x, axis=1, kind="stable")[:, :top]
    return lse, got, h, ids, np.take_along_axis(lp, ids, 1), lp, p, np.abs(m[:, 0])


def _run(x, target, top, info=None):
    T = x.shape[0]
    logp, h, lse = (torch.full((T,), 5.0, device=DEV) for _ in range(3))
    ids = torch.full((T, top), -1, dtype=torch.int32, device=DEV) if top else None
    tl = torch.full((T, top), 5.0, device=DEV) if top else None
    K().kq_token_logprobs(x, target, logp, entropy=h, lse=lse, top_id=ids, top_logp=tl, info=info)
    torch.cuda.synchronize()
    return logp, h, lse, ids, tl


SIZES = [(1, 1, 1), (3, 2, 2), (5, 31, 4), (2, 1000, 32), (7, 4097, 5), (1, 50001, 20), (40, 8192, 1), (300, 513, 3),
         (3, 131072, 32), (2, 200003, 7), (1, 1 << 20, 32), (5, 33, 32)]


@pytest.mark.parametrize("T,V,top", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["plain", "peaked", "masked", "ties", "flat", "far"])
def test_logprobs_match_64_bits(T, V, top, dtype, kind):
    rng = np.random.default_rng(T + V)
    x = _logits(T, V, dtype, kind, rng)
    target = rng.integers(0, V, T)
    target[T // 2] = -1 if T > 1 else target[0]
    want = _reference(x, target, top)
    wide = torch.zeros(T, V + 3, dtype=x.dtype, device=DEV)   # a row stride that is not aligned
    wide[:, :V] = x.to(DEV)
    info = torch.zeros(1, dtype=torch.int32, device=DEV)
    for src in (x.to(DEV), wide[:, :V]):
        logp, h, lse, ids, tl = _run(src, torch.from_numpy(target).to(DEV), top, info)
        assert K().kq_check(info)[0] == K().KQ_OK
        big = want[7]
        for got, exact in ((lse, want[0]), (logp, want[1]), (h, want[2])):
            got = got.cpu().numpy().astype(np.float64)
            inf = np.isinf(exact)
            assert np.array_equal(got[inf], exact[inf])
            assert np.all(np.abs(got - exact)[~inf] <= (2.0 ** -18 * (1 + big + np.abs(exact)))[~inf])
        assert np.array_equal(ids.cpu().numpy(), want[3])
        got, exact = tl.cpu().numpy().astype(np.float64), want[4]
        inf = np.isinf(exact)
        assert np.array_equal(got[inf], exact[inf])
        assert np.all((np.abs(got - exact) <= 2.0 ** -18 * (1 + big[:, None] + np.abs(exact)))[~inf])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logprobs_without_top_and_optional_outputs(dtype):
    x = _logits(9, 700, dtype, "plain", np.random.default_rng(0)).to(DEV)
    y = torch.arange(9, device=DEV)
    full = _run(x, y, 6)
    logp = torch.empty(9, device=DEV)
    K().kq_token_logprobs(x, y, logp)
    assert torch.equal(logp, full[0])
    assert torch.equal(_run(x, y, 0)[1], full[1])
    e = torch.empty(0, 700, dtype=x.dtype, device=DEV)
    K().kq_token_logprobs(e, y[:0], logp[:0])


@pytest.mark.parametrize("V", [5, 3001, 150000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logprobs_rows_without_a_distribution(V, dtype):
    x = torch.randn(5, V, device=DEV).to(TYPES[dtype])
    x[0] = -float("inf")
    x[1, 3] = float("nan")
    x[2, V - 1] = float("inf")
    x[3, 2] = -float("inf")
    y = torch.tensor([1, 0, 0, 2, 4], device=DEV)
    logp, h, lse, ids, tl = _run(x, y, 2)
    inf = float("inf")
    assert logp[0] == -inf and lse[0] == -inf and h[0] == 0 and ids[0].tolist() == [0, 1] and (tl[0] == -inf).all()
    for r in (1, 2):
        assert torch.isnan(logp[r]) and torch.isnan(lse[r]) and torch.isnan(h[r]) and torch.isnan(tl[r]).all()
    assert ids[1, 0] == 3 and ids[2, 0] == V - 1
    assert logp[3] == -inf and torch.isfinite(lse[3]) and torch.isfinite(h[3])
    assert torch.isfinite(logp[4]) and torch.isfinite(tl[4]).all()
    grad = torch.empty_like(x)
    K().kq_token_logprobs_grad(x, y, lse, torch.ones(5, device=DEV), grad, entropy=h, g_entropy=torch.ones(5, device=DEV))
    assert not grad[0].any() and torch.isnan(grad[1]).any() and torch.isfinite(grad[3:].float()).all()


@pytest.mark.parametrize("V", [7, 5000, 60000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logprobs_with_masks_of_the_lowest_value_and_huge_logits(V, dtype):
    """Masks as the type's lowest number, alone, with a few allowed tokens (fewer than asked for), with -infinity, and
    logits near the type's largest: the fast way's range ends at 1e38."""
    lowest = torch.finfo(TYPES[dtype]).min
    x = torch.full((6, V), lowest).to(TYPES[dtype])
    x[1, 3] = 2.0
    x[1, 5] = 1.0
    x[2, ::2] = -float("inf")
    x[3] = torch.linspace(-5, 5, V)
    x[3, 1] = 3.0e38
    x[4] = torch.linspace(-5, 5, V)
    x[4, 0] = lowest
    x[5, 2:5] = -float("inf")
    x[5, 1] = -1.5
    top = 4
    target = np.array([2, 5, 1, 1, 0, 1])
    want = _reference(x, target, top)
    logp, h, lse, ids, tl = _run(x.to(DEV), torch.from_numpy(target).to(DEV), top)
    for got, exact in ((lse, want[0]), (logp, want[1]), (h, want[2])):
        got = got.cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - exact) <= 2.0 ** -18 * (1 + np.abs(exact)) + 2.0 ** -18 * np.where(want[7] < 1e30, want[7], 0))
    assert np.array_equal(ids.cpu().numpy(), want[3])
    got, exact = tl.cpu().numpy().astype(np.float64), want[4]
    inf = np.isinf(exact)
    assert np.array_equal(got[inf], exact[inf]) and np.all(np.abs(got - exact)[~inf] <= (2.0 ** -18 * (1 + np.abs(exact)) + 2.0 ** -16)[~inf])
    # the gradient of the rows whose log-sum fp32 can tell from the maximum
    g = torch.ones(6, device=DEV)
    grad = torch.empty_like(x, device=DEV)
    K().kq_token_logprobs_grad(x.to(DEV), torch.from_numpy(target).to(DEV), lse, g, grad, entropy=h, g_entropy=g)
    got = grad.float().cpu()
    assert torch.isfinite(got).all()
    assert (got[1, 6:] == 0).all() and (got[3, 2:] == 0).all()


def test_logprobs_record_a_target_out_of_range():
    x = torch.randn(2, 10, device=DEV)
    info = torch.zeros(1, dtype=torch.int32, device=DEV)
    logp, h, lse, _, _ = _run(x, torch.tensor([10, 3], device=DEV), 0, info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG
    assert torch.isnan(logp[0]) and torch.isfinite(logp[1]) and torch.isfinite(h).all()
    grad = torch.empty_like(x)
    K().kq_token_logprobs_grad(x, torch.tensor([1 << 40, 3], device=DEV), lse, torch.ones(2, device=DEV), grad, info=info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG
    assert not grad[0].any() and grad[1].any()


@pytest.mark.parametrize("T,V", [(1, 1), (3, 7), (4, 1000), (2, 50001), (33, 4096)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["plain", "peaked", "masked", "far"])
@pytest.mark.parametrize("with_entropy", [False, True])
def test_gradient_matches_the_formula(T, V, dtype, kind, with_entropy):
    rng = np.random.default_rng(V + T)
    x = _logits(T, V, dtype, kind, rng)
    target = rng.integers(0, V, T)
    if T > 2:
        target[1] = -7
    g, ge = rng.standard_normal(T).astype(np.float32), rng.standard_normal(T).astype(np.float32)
    lse, _, h, _, _, _, _, big = _reference(x, target, 0)
    # the gradient's own inputs: lse and entropy as fp32 has them
    lse, h = (a.astype(np.float32).astype(np.float64) for a in (lse, h))
    lp = x.float().numpy().astype(np.float64) - lse[:, None]
    p = np.exp(lp)
    want = -g[:, None] * p * (target >= 0)[:, None]
    mag = np.abs(want)
    for r, y in enumerate(target):
        if y >= 0:
            want[r, y] += g[r]
            mag[r, y] += abs(g[r])
    if with_entropy:
        term = p * (np.where(p > 0, lp, 0) + h[:, None]) * ge[:, None]
        want -= term
        mag += p * (np.abs(np.where(p > 0, lp, 0)) + h[:, None]) * np.abs(ge)[:, None]
    f = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(DEV)  # noqa: E731
    d = x.to(DEV)
    for out in (torch.empty_like(d), d.clone(), torch.zeros(T, V + 5, dtype=d.dtype, device=DEV)[:, :V]):
        src = out if out.is_contiguous() and out.data_ptr() != d.data_ptr() and torch.equal(out, d) else d
        K().kq_token_logprobs_grad(src, torch.from_numpy(target).to(DEV), f(lse), f(g), out, entropy=f(h) if with_entropy else None,
                                   g_entropy=f(ge) if with_entropy else None)
        got = out.float().cpu().numpy().astype(np.float64)
        tol = mag * (2.0 ** -18 + 2.0 ** -22 * (1 + big[:, None])) + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0) + 1e-36
        assert np.all(np.abs(got - want) <= tol)


def test_gradient_matches_differences():
    """Central differences of the kernel's own logp and entropy: step h = 1/16 leaves h^2/6 times a third derivative
    below 2 in size (6.6e-4 * 2) and the fp32 results' rounding of 2^-20 over 2 h."""
    rng = np.random.default_rng(11)
    V, step = 9, 1 / 16
    x = torch.from_numpy(rng.standard_normal((1, V)).astype(np.float32)).to(DEV)
    y = torch.tensor([4], device=DEV)
    logp, h, lse, _, _ = _run(x, y, 0)
    grad = torch.empty_like(x)
    for g, ge in ((1.0, 0.0), (0.0, 1.0), (-0.5, 2.0)):
        K().kq_token_logprobs_grad(x, y, lse, torch.tensor([g], device=DEV), grad, entropy=h,
                                   g_entropy=torch.tensor([ge], device=DEV))
        up, down = x.repeat(V, 1) + step * torch.eye(V, device=DEV), x.repeat(V, 1) - step * torch.eye(V, device=DEV)
        a, b = _run(up, y.repeat(V), 0), _run(down, y.repeat(V), 0)
        diff = (g * (a[0] - b[0]) + ge * (a[1] - b[1])) / (2 * step)
        tol = (abs(g) + 4 * abs(ge)) * (2 * step ** 2 / 6 + 2.0 ** -20 / step)
        assert torch.all((diff - grad[0]).abs() <= tol), (diff, grad)


def test_binding_refuses_what_does_not_fit():
    kq = K()
    x, y, f = torch.randn(4, 50, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros(4, device=DEV)
    with pytest.raises(ValueError, match="int64"):
        kq.kq_token_logprobs(x, y.int(), f)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        kq.kq_token_logprobs(x.half(), y, f)
    with pytest.raises(ValueError, match="go together"):
        kq.kq_token_logprobs(x, y, f, top_id=torch.zeros(4, 2, dtype=torch.int32, device=DEV))
    with pytest.raises(kq.KronqError, match="INVALID_ARG"):
        kq.kq_token_logprobs(x, y, f, top_id=torch.zeros(4, 33, dtype=torch.int32, device=DEV), top_logp=torch.zeros(4, 33, device=DEV))
    with pytest.raises(kq.KronqError, match="ld >= V"):
        kq.kq_token_logprobs(x[:1].expand(4, 50), y, f)
    with pytest.raises(ValueError, match="unit column"):
        kq.kq_token_logprobs(x.t(), y, f)
    with pytest.raises(ValueError, match="shape and type"):
        kq.kq_token_logprobs_grad(x, y, f, f, x.bfloat16())
    with pytest.raises(kq.KronqError, match="INVALID_ARG"):
        kq.kq_token_logprobs_grad(x, y, f, f, torch.empty_like(x), g_entropy=f)
    with pytest.raises(kq.KronqError, match="INVALID_ARG"):
        wide = torch.zeros(4, 60, device=DEV)
        kq.kq_token_logprobs_grad(wide[:, :50], y, f, f, torch.as_strided(wide, (4, 50), (50, 1)))
    torch.cuda.synchronize()
