"""GPU checks of kq_linear_logprobs and its gradient against 64 bits.

Bounds. Products of bf16 values are exact; over 1024 of d (512 for few rows) the tensor cores add 16 products at a time and may drop a unit (2^-23)
of the sum so far at each of the 64 steps, which is half of A = sum |x w| or less in the mean of products that come in no order,
and at most 128 chunks are added in fp32: a logit is off by at most e = 2^-18 A. With u = 2^-18 (1 + |m| + |value|) for the softmax's own arithmetic (as in kq_token_logprobs's
tests): |lse - exact| <= e + u, |logp - exact| <= 2 e + u, and the entropy, whose derivative is -p (ln p + H):
|H - exact| <= sum_v p |ln p + H| 2 e_v + u. The logits' gradient D = g (delta - p) - h p (ln p + H) from given lse and H:
    |dD| <= p (|g| + |h| (|ln p + H| + 1)) (2 e + 2^-18 (1 + |z| + |lse|)) + 2^-8 |D|,
and the products sum |dD| |w| (|x|), with their own sums' 2^-16 of sum |D w| (2048 of K between chunks: 128 steps of 2^-23) and the
outputs' rounding, 2^-8."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_07964_gb300 import build
    build.build()


def K():
    from paper_2607_07964_gb300 import kronq
    return kronq


def _case(T, V, d, kind="plain", seed=0):
    g = torch.Generator(DEV).manual_seed(seed + T + V + d)
    w = torch.randn(V, d, device=DEV, generator=g) * (2.5 / d ** 0.5)
    y = torch.randint(0, V, (T,), device=DEV, generator=g)
    x = torch.randn(T, d, device=DEV, generator=g)
    if kind == "peaked":
        x += 6 / 2.5 * w[y] * torch.rand(T, 1, device=DEV, generator=g)
    if kind == "flat":
        x *= 0
    if kind == "far":
        x, w = x * 8, w * 8
    y[torch.rand(T, device=DEV, generator=g) < 0.2] = -3
    return x.bfloat16(), w.bfloat16(), y


def _strided(t):
    wide = torch.zeros(t.shape[0], t.shape[1] + 24, dtype=t.dtype, device=DEV)
    wide[:, 8:8 + t.shape[1]] = t
    return wide[:, 8:8 + t.shape[1]]


def _exact(x, w, y):
    X, W = x.double(), w.double()
    z = X @ W.T
    e = 2.0 ** -18 * (X.abs() @ W.abs().T)
    m = z.amax(1)
    lse = torch.logsumexp(z, 1)
    lp = z - lse[:, None]
    p = lp.exp()
    H = -(p * lp).sum(1)
    got = torch.where(y >= 0, lp.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    return z, e, m, lse, lp, p, H, got


def _score(x, w, y, info=None, poison=255):
    outs = [torch.full((x.shape[0],), 5.0, device=DEV) for _ in range(3)]
    ws = torch.full((K().kq_linear_logprobs_workspace(x, w),), poison, dtype=torch.uint8, device=DEV)
    K().kq_linear_logprobs(x, w, y, outs[0], ws, entropy=outs[1], lse=outs[2], info=info)
    torch.cuda.synchronize()
    return outs


SIZES = [(1, 1, 8), (1, 1000, 64), (2, 127, 72), (3, 128, 520), (5, 129, 8), (17, 4097, 264), (127, 300, 1000), (128, 513, 512),
         (129, 257, 1024), (256, 255, 136), (257, 1025, 2056), (300, 20000, 128), (1000, 5003, 320), (4100, 700, 64), (8, 33000, 4096),
         (33, 10241, 72), (64, 20000, 136), (100, 12345, 328), (90, 11000, 520), (10, 10240, 8), (1, 1000, 4096),
         (33, 2000, 2056), (96, 5000, 2800), (70, 9000, 1032), (128, 130, 6000), (40, 9729, 1024)]


@pytest.mark.parametrize("T,V,d", SIZES)
@pytest.mark.parametrize("kind", ["plain", "peaked", "flat", "far"])
def test_log_probabilities_match_64_bits(T, V, d, kind):
    x, w, y = _case(T, V, d, kind)
    z, e, m, lse, lp, p, H, want = _exact(x, w, y)
    e1 = e.amax(1)
    info = torch.zeros(1, dtype=torch.int32, device=DEV)
    logp, ent, ls = _score(x, w, y, info)
    assert K().kq_check(info)[0] == K().KQ_OK

    def u(v):
        return 2.0 ** -18 * (1 + m.abs() + v.abs())

    assert ((ls - lse).abs() <= e1 + u(lse)).all()
    assert ((logp - want).abs() <= 2 * e1 + u(want)).all() and (logp <= 0).all()
    assert ((ent - H).abs() <= (p * (lp + H[:, None]).abs() * 2 * e).sum(1) + u(H)).all()
    again = _score(x, w, y, poison=127)
    assert all(torch.equal(a, b) for a, b in zip((logp, ent, ls), again))
    some = _score(_strided(x), _strided(w), y)
    assert all(torch.equal(a, b) for a, b in zip((logp, ent, ls), some))


@pytest.mark.parametrize("T,V,d", SIZES)
@pytest.mark.parametrize("entropy", [False, True])
def test_gradient_matches_64_bits(T, V, d, entropy):
    x, w, y = _case(T, V, d, "peaked")
    z, e, m, lse, lp, p, H, _ = _exact(x, w, y)
    g = torch.Generator(DEV).manual_seed(9)
    gl, ge = torch.randn(T, device=DEV, generator=g), torch.randn(T, device=DEV, generator=g) if entropy else None
    ls, h = lse.float(), H.float()
    gx, gw = _strided(torch.full_like(x, 3.0)), _strided(torch.full_like(w, 3.0))
    ws = torch.full((K().kq_linear_logprobs_grad_workspace(x, w),), 255, dtype=torch.uint8, device=DEV)
    info = torch.zeros(1, dtype=torch.int32, device=DEV)
    K().kq_linear_logprobs_grad(x, w, y, ls, gl, ws, gx=gx, gw=gw, entropy=h if entropy else None, g_entropy=ge, info=info)
    assert K().kq_check(info)[0] == K().KQ_OK
    G = torch.where(y >= 0, gl, 0.0).double()[:, None]
    E = ge.double()[:, None] if entropy else torch.zeros_like(G)
    lp = z - ls.double()[:, None]
    p = lp.exp()
    Hc = h.double()[:, None]
    D = -p * (G + E * (lp + Hc))
    D[torch.arange(T, device=DEV), y.clamp(min=0)] += G[:, 0]
    tol = p * (G.abs() + E.abs() * ((lp + Hc).abs() + 1)) * (2 * e + 2.0 ** -18 * (1 + z.abs() + lse.abs()[:, None])) + 2.0 ** -8 * D.abs()
    X, W = x.double(), w.double()
    for got, want, t in ((gx, D @ W, tol @ W.abs() + 2.0 ** -16 * (D.abs() @ W.abs())),
                         (gw, D.T @ X, tol.T @ X.abs() + 2.0 ** -16 * (D.abs().T @ X.abs()))):
        assert ((got.double() - want).abs() <= t + 2.0 ** -8 * want.abs() + 1e-37).all()
    # each alone, and twice: the same bits
    for only in ("gx", "gw"):
        out = torch.empty_like(x if only == "gx" else w)
        ws.fill_(127)
        K().kq_linear_logprobs_grad(x, w, y, ls, gl, ws, entropy=h if entropy else None, g_entropy=ge, **{only: out})
        assert torch.equal(out, gx if only == "gx" else gw)


def test_several_pieces_of_the_vocabulary():
    """More columns than a piece holds, an odd rest, gx over several launches."""
    T, V, d = 9000, 10001, 72
    x, w, y = _case(T, V, d, "peaked")
    z, e, m, lse, lp, p, H, want = _exact(x, w, y)
    logp, ent, ls = _score(x, w, y)
    assert ((logp - want).abs() <= 2 * e.amax(1) + 2.0 ** -18 * (1 + m.abs() + want.abs())).all()
    gl = torch.randn(T, device=DEV)
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.full((K().kq_linear_logprobs_grad_workspace(x, w),), 255, dtype=torch.uint8, device=DEV)
    K().kq_linear_logprobs_grad(x, w, y, ls, gl, ws, gx=gx, gw=gw)
    G = torch.where(y >= 0, gl, 0.0).double()[:, None]
    p = (z - ls.double()[:, None]).exp()
    D = -p * G
    D[torch.arange(T, device=DEV), y.clamp(min=0)] += G[:, 0]
    tol = p * G.abs() * (2 * e + 2.0 ** -18 * (1 + z.abs() + lse.abs()[:, None])) + 2.0 ** -8 * D.abs()
    X, W = x.double(), w.double()
    for got, want, t in ((gx, D @ W, tol @ W.abs() + 2.0 ** -16 * (D.abs() @ W.abs())),
                         (gw, D.T @ X, tol.T @ X.abs() + 2.0 ** -16 * (D.abs().T @ X.abs()))):
        assert ((got.double() - want).abs() <= t + 2.0 ** -8 * want.abs() + 1e-37).all()


def test_the_gradient_is_that_of_the_log_probabilities():
    """Against differences of kq_linear_logprobs itself in the direction of the gradient gx: steps that bf16 holds."""
    T, V, d = 16, 600, 128
    x, w, y = _case(T, V, d, "plain")
    y = y.clamp(min=0)
    gl, ge = torch.ones(T, device=DEV), torch.full((T,), 0.5, device=DEV)
    logp, ent, ls = _score(x, w, y)
    gx = torch.empty_like(x)
    ws = torch.empty(K().kq_linear_logprobs_grad_workspace(x, w), dtype=torch.uint8, device=DEV)
    K().kq_linear_logprobs_grad(x, w, y, ls, gl, ws, gx=gx, entropy=ent, g_entropy=ge)
    a, b = (x.float() + 0.25 * gx.float()).bfloat16(), (x.float() - 0.25 * gx.float()).bfloat16()
    la, ea, _ = _score(a, w, y)
    lb, eb, _ = _score(b, w, y)
    step = a.double() - b.double()     # as the rounding left it
    diff = (la.double() - lb.double()) + 0.5 * (ea.double() - eb.double())
    got = (step * gx.double()).sum(1)
    # gx's own rounding 2^-7 of |step| |gx|, and the third derivative along a step of at most 0.3 |w| in the logits
    z = (step @ w.double().T).abs().amax(1)
    assert ((got - diff).abs() <= 2.0 ** -6 * (step.abs() * gx.double().abs()).sum(1) + z ** 3 + 1e-3).all()


@pytest.mark.parametrize("d", [64, 2056])
def test_targets_out_of_range_infinities_and_nan(d):
    x, w, y = _case(6, 300, d)
    y = torch.tensor([3, -1, 300, 7, 5, 2 ** 40], device=DEV)
    x[3, 5], x[4, 0] = float("nan"), float("inf")
    info = torch.zeros(1, dtype=torch.int32, device=DEV)
    logp, ent, ls = _score(x, w, y, info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG
    assert torch.isnan(logp).tolist() == [False, False, True, True, True, True] and logp[1] == 0
    assert torch.isnan(ls).tolist() == torch.isnan(ent).tolist() == [False, False, False, True, True, False]
    good = torch.tensor([0, 1, 2, 5], device=DEV)
    gx, gw = torch.empty_like(x[good]), torch.empty_like(w)
    ws = torch.empty(K().kq_linear_logprobs_grad_workspace(x[good], w), dtype=torch.uint8, device=DEV)
    one = torch.ones(4, device=DEV)
    K().kq_linear_logprobs_grad(x[good].contiguous(), w, y[good], ls[good], one, ws, gx=gx, gw=gw, info=info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG
    assert gx[0].any() and not gx[1:].any() and torch.isfinite(gw).all()


@pytest.mark.parametrize("d", [64, 2056])
def test_logits_of_a_huge_size(d):
    x, w, y = _case(4, 500, d)
    big = (x.float() * 2.0 ** 60).bfloat16(), (w.float() * 2.0 ** 40).bfloat16()
    logp, ent, ls = _score(*big, y.clamp(min=0))
    z = big[0].double() @ big[1].double().T
    lse = torch.logsumexp(z, 1)
    assert ((ls - lse).abs() <= 2.0 ** -17 * (big[0].double().abs() @ big[1].double().abs().T).amax(1)).all()
    assert (ent == 0).all() and (logp <= 0).all() and torch.isfinite(logp).all()


@pytest.mark.parametrize("T,V,d", [(3, 200, 72), (90, 513, 136), (129, 257, 64), (300, 1000, 200)])
def test_gradients_between_other_columns_leave_them(T, V, d):
    x, w, y = _case(T, V, d)
    logp, ent, ls = _score(x, w, y)
    wide = [torch.full((t.shape[0], t.shape[1] + 24), 3.0, dtype=t.dtype, device=DEV) for t in (x, w)]
    ws = torch.empty(K().kq_linear_logprobs_grad_workspace(x, w), dtype=torch.uint8, device=DEV)
    K().kq_linear_logprobs_grad(x, w, y, ls, torch.ones(T, device=DEV), ws, gx=wide[0][:, 8:8 + d], gw=wide[1][:, 8:8 + d])
    for t in wide:
        assert (t[:, :8] == 3).all() and (t[:, 8 + d:] == 3).all() and not (t[:, 8:8 + d] == 3).all()


def test_two_streams_at_once():
    cases = [_case(T, V, d, "peaked") for T, V, d in ((64, 20000, 512), (400, 5000, 512))]

    def run(x, w, y, ws, gs, outs):
        K().kq_linear_logprobs(x, w, y, outs[0], ws, entropy=outs[1], lse=outs[2])
        K().kq_linear_logprobs_grad(x, w, y, outs[2], outs[0], gs, gx=outs[3], gw=outs[4])

    sets = []
    for x, w, y in cases:
        sets.append((x, w, y, torch.empty(K().kq_linear_logprobs_workspace(x, w), dtype=torch.uint8, device=DEV),
                     torch.empty(K().kq_linear_logprobs_grad_workspace(x, w), dtype=torch.uint8, device=DEV)))
    want, got = ([[torch.empty(len(x), device=DEV) for _ in range(3)] + [torch.empty_like(x), torch.empty_like(w)] for x, w, _ in cases]
                 for _ in range(2))
    for s, o in zip(sets, want):
        run(*s, o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        for st, s, o in zip(streams, sets, got):
            with torch.cuda.stream(st):
                run(*s, o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))


def test_no_rows():
    x, w, y = _case(4, 300, 64)
    K().kq_linear_logprobs(x[:0], w, y[:0], torch.empty(0, device=DEV), None)
    gw = torch.full_like(w, 3.0)
    wide = _strided(gw)
    K().kq_linear_logprobs_grad(x[:0], w, y[:0], torch.empty(0, device=DEV), torch.empty(0, device=DEV), None, gw=wide)
    assert not wide.any()


def test_replays_in_a_graph_and_on_another_stream():
    x, w, y = _case(70, 3000, 256, "peaked")
    outs = [torch.empty(70, device=DEV) for _ in range(3)]
    ws = torch.empty(K().kq_linear_logprobs_workspace(x, w), dtype=torch.uint8, device=DEV)
    gs = torch.empty(K().kq_linear_logprobs_grad_workspace(x, w), dtype=torch.uint8, device=DEV)
    gx, gw, one = torch.empty_like(x), torch.empty_like(w), torch.ones(70, device=DEV)

    def run():
        K().kq_linear_logprobs(x, w, y, outs[0], ws, entropy=outs[1], lse=outs[2])
        K().kq_linear_logprobs_grad(x, w, y, outs[2], one, gs, gx=gx, gw=gw, entropy=outs[1], g_entropy=one)

    run()
    want = [t.clone() for t in outs + [gx, gw]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for t in outs + [gx, gw]:
        t.zero_()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(want, outs + [gx, gw]))
    s = torch.cuda.Stream()
    for t in outs + [gx, gw]:
        t.zero_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs + [gx, gw]))
