"""kq_linear_logprobs_grad, from kq_linear_logprobs's own log-sums and entropies, against differences of the log probabilities and
entropies in 64 bits, entry by entry.

f(x, W) = sum_t (g_t logp_t + h_t entropy_t) is taken at an entry's value plus and minus s = 2^-17 and 2 s. The quotient of the first pair is off
by a third of what the two differ by (the next order is s^2 of that), and by rounding: f is at most 2^12, its sums off by
2^-53 2^12 16 = 2^-37, over 2 s 2^-21. The gradient's own bounds are those of test_gpu_linear_logprobs.py, with what the log-sums (e1 + u)
and entropies that it is given are off by."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
STEP = 2.0 ** -17


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_07964_gb300 import build
    build.build()


def K():
    from paper_2607_07964_gb300 import kronq
    return kronq


def _terms(z, y, g, h):
    """g logp + h entropy of each row of logits in 64 bits."""
    lp = torch.log_softmax(z, -1)
    logp = torch.where(y >= 0, lp.gather(-1, y.clamp(min=0)[..., None])[..., 0], 0.0)
    return g * logp - h * (lp.exp() * lp).sum(-1)


def _differences(f):
    """(quotient, what it may be off by) of a function of an entry's change."""
    near, far = ((f(s) - f(-s)) / (2 * s) for s in (STEP, 2 * STEP))
    return near, (far - near).abs() + 2.0 ** -20


# few rows, gW by tiles; few rows, gW in the same pass; tiles
@pytest.mark.parametrize("T,V,d", [(16, 600, 128), (9, 10300, 64), (150, 777, 72)])
@pytest.mark.parametrize("share", [0.0, 0.5, -2.0])
def test_entries_are_the_quotients_of_differences(T, V, d, share):
    g = torch.Generator(DEV).manual_seed(T)
    w = (torch.randn(V, d, device=DEV, generator=g) * (2.5 / d ** 0.5)).bfloat16()
    x = torch.randn(T, d, device=DEV, generator=g).bfloat16()
    y = torch.randint(-V // 10, V, (T,), device=DEV, generator=g)
    gl, ge = 1 + torch.rand(T, device=DEV, generator=g), share * (1 + torch.rand(T, device=DEV, generator=g))
    logp, ent, lse = (torch.empty(T, device=DEV) for _ in range(3))
    ws = torch.empty(K().kq_linear_logprobs_workspace(x, w), dtype=torch.uint8, device=DEV)
    K().kq_linear_logprobs(x, w, y, logp, ws, entropy=ent, lse=lse)
    ws = torch.empty(K().kq_linear_logprobs_grad_workspace(x, w), dtype=torch.uint8, device=DEV)

    def grads(ge):
        gx, gw = torch.empty_like(x), torch.empty_like(w)
        K().kq_linear_logprobs_grad(x, w, y, lse, gl, ws, gx=gx, gw=gw, entropy=None if ge is None else ent, g_entropy=ge)
        return gx.double(), gw.double()

    gx, gw = grads(ge if share else None)
    X, W, G, E = x.double(), w.double(), torch.where(y >= 0, gl, 0.0).double()[:, None], ge.double()[:, None]
    z = X @ W.T
    e = 2.0 ** -18 * (X.abs() @ W.abs().T)
    lp = torch.log_softmax(z, 1)
    p, exact = lp.exp(), torch.logsumexp(z, 1)[:, None]
    H = -(p * lp).sum(1, keepdim=True)
    slope = (lp + H).abs()
    m = z.amax(1, keepdim=True).abs()
    e_lse = e.amax(1, keepdim=True) + 2.0 ** -18 * (1 + m + exact.abs())
    e_ent = (p * slope * 2 * e).sum(1, keepdim=True) + 2.0 ** -18 * (1 + m + H)
    D = -p * (G + E * (lp + H))
    D[torch.arange(T, device=DEV), y.clamp(min=0)] += G[:, 0]
    dD = p * ((G.abs() + E.abs() * (slope + 1)) * (2 * e + e_lse + 2.0 ** -18 * (1 + z.abs() + exact.abs())) + E.abs() * e_ent) + 2.0 ** -8 * D.abs()
    # of x: every entry; a column's change moves a row's logits by it times the column of W
    want, off = (torch.stack(t, 1) for t in zip(*(
        _differences(lambda s: _terms(z + s * W[:, i], y, gl.double(), ge.double())) for i in range(d))))
    tol = dD @ W.abs() + 2.0 ** -16 * (D.abs() @ W.abs()) + 2.0 ** -8 * want.abs() + off
    # of W: entries of the targets' rows, of the likeliest tokens' and of others
    v = torch.cat([y.clamp(min=0)[:40], z.argmax(1)[:40], torch.randint(0, V, (60,), device=DEV, generator=g)])
    i = torch.randint(0, d, (len(v),), device=DEV, generator=g)

    def moved(at, col):
        def f(s):
            q = z.clone()
            q[:, at] += s * X[:, col]
            return _terms(q, y, gl.double(), ge.double()).sum()
        return f

    want_w, off_w = (torch.stack(t) for t in zip(*(_differences(moved(a, b)) for a, b in zip(v.tolist(), i.tolist()))))
    tol_w = ((dD + 2.0 ** -16 * D.abs()).T @ X.abs())[v, i] + 2.0 ** -8 * want_w.abs() + off_w

    def within(gx, gw):
        return bool(((gx - want).abs() <= tol).all()), bool(((gw[v, i] - want_w).abs() <= tol_w).all())

    assert within(gx, gw) == (True, True)
    # and the bounds tell these from it
    wrong = [(-gx, -gw), (2 * gx, 2 * gw), (0 * gx, 0 * gw), (1.05 * gx, 1.05 * gw)]
    if share:
        wrong += [grads(None), grads(-ge)]
    for a, b in wrong:
        assert within(a, b) == (False, False)
