"""kq_linear_logprobs_grad where the vocabulary goes in three pieces and more: gx carried from piece to piece in fp32 and finished
by the last, D's two buffers written again, columns of W and targets at an offset, and from 65536 rows on pieces of 1024 columns. Bounds
as derived in test_gpu_linear_logprobs.py."""
import json
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, GUARD = "cuda", 4096
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_07964_gb300 import build
    build.build()


def K():
    from paper_2607_07964_gb300 import kronq
    return kronq


def _case(T, V, d):
    g = torch.Generator(DEV).manual_seed(T + V + d)
    w = (torch.randn(V, d, device=DEV, generator=g) * (2.5 / d ** 0.5)).bfloat16()
    y = torch.randint(-V // 8, V, (T,), device=DEV, generator=g)
    x = torch.randn(T, d, device=DEV, generator=g) + 2.4 * w.float()[y.clamp(min=0)] * torch.rand(T, 1, device=DEV, generator=g)
    return x.bfloat16(), w, y, torch.randn(T, device=DEV, generator=g), torch.randn(T, device=DEV, generator=g)


# pieces of 8192 columns, four of them, gx by one launch after the other, three tiles of d, an odd rest of rows and columns; of 1024
# columns, the last of them 52, more than 65536 rows
@pytest.mark.parametrize("T,V,d", [(8190, 25001, 768), (70001, 2100, 136)])
@pytest.mark.parametrize("entropy", [False, True])
def test_gradients_of_three_pieces_and_more_match_64_bits(T, V, d, entropy):
    x, w, y, gl, ge = _case(T, V, d)
    X, W = x.double(), w.double()
    z = X @ W.T
    e = 2.0 ** -18 * (X.abs() @ W.abs().T)
    lse = torch.logsumexp(z, 1)
    lp = z - lse[:, None]
    h = -(lp.exp() * lp).sum(1).float()
    ls = lse.float()
    kw = dict(entropy=h, g_entropy=ge) if entropy else {}
    n = K().kq_linear_logprobs_grad_workspace(x, w)

    def run(poison, **out):
        ws = torch.full((n,), poison, dtype=torch.uint8, device=DEV)
        info = torch.zeros(1, dtype=torch.int32, device=DEV)
        K().kq_linear_logprobs_grad(x, w, y, ls, gl, ws, info=info, **out, **kw)
        assert K().kq_check(info)[0] == K().KQ_OK

    gx, gw = torch.full_like(x, 3.0), torch.full_like(w, 3.0)
    run(255, gx=gx, gw=gw)
    G = torch.where(y >= 0, gl, 0.0).double()[:, None]
    E = ge.double()[:, None] if entropy else torch.zeros_like(G)
    lp = z - ls.double()[:, None]
    p = lp.exp()
    slope = lp + h.double()[:, None]
    D = -p * (G + E * slope)
    D[torch.arange(T, device=DEV), y.clamp(min=0)] += G[:, 0]
    tol = p * (G.abs() + E.abs() * (slope.abs() + 1)) * (2 * e + 2.0 ** -18 * (1 + z.abs() + lse.abs()[:, None])) + 2.0 ** -8 * D.abs()
    del z, e, lp, p, slope
    tol += 2.0 ** -16 * D.abs()
    want = D @ W
    assert ((gx.double() - want).abs() <= tol @ W.abs() + 2.0 ** -8 * want.abs() + 1e-37).all()
    want = D.T @ X
    assert ((gw.double() - want).abs() <= tol.T @ X.abs() + 2.0 ** -8 * want.abs() + 1e-37).all()
    # each alone, and again: the same bits
    for only, got in (("gx", gx), ("gw", gw)):
        for poison in (127, 255):
            out = torch.full_like(got, 3.0)
            run(poison, **{only: out})
            assert torch.equal(out, got)


def _small():
    """Three pieces with the least work: 5376 columns of 12001 rows."""
    return _case(12001, 11001, 72)


def test_nothing_outside_the_outputs_and_the_workspace():
    x, w, y, gl, ge = _small()
    made = []

    def new(n):
        raw = torch.full((GUARD + n + GUARD + (-n) % 256,), 0x5A, dtype=torch.uint8, device=DEV)
        made.append((raw, n))
        return raw[GUARD:GUARD + n]

    logp, ent, lse = (torch.empty(len(x), device=DEV) for _ in range(3))
    gx, gw = (new(2 * t.numel()).view(torch.bfloat16).view(t.shape) for t in (x, w))
    ws, gs = new(K().kq_linear_logprobs_workspace(x, w)), new(K().kq_linear_logprobs_grad_workspace(x, w))
    K().kq_linear_logprobs(x, w, y, logp, ws, entropy=ent, lse=lse)
    K().kq_linear_logprobs_grad(x, w, y, lse, gl, gs, gx=gx, gw=gw, entropy=ent, g_entropy=ge)
    for raw, n in made:
        assert (raw[:GUARD] == 0x5A).all() and (raw[GUARD + n:] == 0x5A).all()
    assert torch.isfinite(gx).all() and torch.isfinite(gw).all()


def test_pieces_replay_in_a_graph():
    x, w, y, gl, ge = _small()
    logp, ent, lse = (torch.empty(len(x), device=DEV) for _ in range(3))
    ws = torch.empty(K().kq_linear_logprobs_workspace(x, w), dtype=torch.uint8, device=DEV)
    gs = torch.empty(K().kq_linear_logprobs_grad_workspace(x, w), dtype=torch.uint8, device=DEV)
    gx, gw = torch.empty_like(x), torch.empty_like(w)

    def run():
        K().kq_linear_logprobs(x, w, y, logp, ws, entropy=ent, lse=lse)
        K().kq_linear_logprobs_grad(x, w, y, lse, gl, gs, gx=gx, gw=gw, entropy=ent, g_entropy=ge)

    run()
    outs = [logp, ent, lse, gx, gw]
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(2):
        for t in outs:
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


CHILD = r'''
import hashlib, json, os, sys
sys.path[:0] = [os.environ["KQ_ROOT"], os.path.join(os.environ["KQ_ROOT"], "tests")]
import torch
import test_gpu_linear_logprobs_pieces as t
from paper_2607_07964_gb300 import kronq as K
from paper_2607_07964_gb300.serving import score_hidden, score_hidden_grad
x, w, y, gl, ge = t._small()
logp, h, lse = score_hidden(x, w, y)
gx, gw = score_hidden_grad(x, w, y, lse, gl, h, ge)
digest = lambda t: hashlib.sha256(t.cpu().contiguous().view(torch.uint8).numpy().tobytes()).hexdigest()
print(json.dumps({"debug": K.kq_debug_build(), "res": [digest(t) for t in (logp, h, lse, gx, gw)], "after": K.kq_debug_status()}))
'''


def test_debug_build_finds_no_store_out_of_bounds_and_agrees():
    from paper_2607_07964_gb300 import build
    build.build(debug=True)

    def child(debug):
        env = dict(os.environ, KQ_ROOT=ROOT, KQ_DEBUG="1" if debug else "0")
        r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, r.stderr[-3000:]
        return json.loads(r.stdout.strip().splitlines()[-1])

    dbg, rel = child(True), child(False)
    assert dbg["debug"] == 1 and rel["debug"] == 0
    assert dbg["after"] == [None, 0], dbg["after"]
    assert dbg["res"] == rel["res"]
