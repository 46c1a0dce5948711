"""GPU checks of kq_qk_rotate and its gradient against 64-bit numpy.

Bounds. The fraction of a turn is cut to 2^-32 and rounded by at most 2^-25 of a half turn: 1e-7 rad; sincospif is within 2
units (2^-23 of values up to 1), the scale rounds once and the two products and their sum three times: 6 2^-24 of
(|a| + |b|) s with the angle's 1.7 2^-24 makes 2^-21. A norm's r has the sum of D squares (13 roundings of its
terms, halved by the root), a division, the root and two products: 11 2^-24. Together below 2^-19 of (|a| + |b|) s.
Backwards the mean of u h adds 15 roundings and twice r's error to its terms: below 2^-18 of r (|u| + |h| mean |u h|). The sums
over rows are of at most 128 terms one after the other (a slot's, 32 slots, a block's sixteenth of 512, 32 warps): 2^-17 of the sum of
|g h| with the terms' 2^-18 in it twice. Each output is rounded once: eps / 2 of the value."""
import numpy as np
import pytest
import torch

import rotate_reference as ref

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


def np64(t):
    return t.detach().double().cpu().numpy()


def _theta(n):
    return [10000.0 ** (-j / max(1, n)) for j in range(n)]


def _rows(rng, T, heads, dim, dtype, where):
    x = rng.standard_normal((T, heads, dim)) * np.exp(rng.standard_normal((T, heads, 1)))
    if where == "part":     # rows with strides of their own
        wide = torch.zeros(T, heads + 3, dim + 8, dtype=dtype, device=DEV)
        wide[:, 1:1 + heads, :dim] = torch.from_numpy(x).to(DEV).to(dtype)
        return wide[:, 1:1 + heads, :dim]
    if where == "odd":      # rows that begin anywhere
        wide = torch.zeros(T, heads, dim + 3, dtype=dtype, device=DEV)
        wide[..., 1:1 + dim] = torch.from_numpy(x).to(DEV).to(dtype)
        return wide[..., 1:1 + dim]
    if where == "across":   # heads first
        return torch.from_numpy(x).to(DEV).to(dtype).transpose(0, 1).contiguous().transpose(0, 1)
    return torch.from_numpy(x).to(DEV).to(dtype)


def _close(got, want, size, dtype, share):
    tol = share * size + torch.finfo(dtype).eps / 2 * np.abs(want) * (1 + 2.0 ** -9) + 1e-38
    bad = np.abs(np64(got) - want) / tol
    assert np.all(bad <= 1), float(np.nanmax(bad))


CASES = [(1, 1, 1, 128, 128, False, True), (5, 4, 1, 64, 64, False, True), (3, 2, 2, 80, 80, False, True),
         (7, 3, 1, 96, 24, True, True), (130, 8, 2, 128, 64, False, False), (9, 7, 1, 256, 256, False, True),
         (9, 7, 1, 256, 34, False, True), (4, 5, 5, 65, 64, False, True), (4, 2, 1, 33, 22, True, False),
         (6, 3, 0, 128, 128, True, True), (2, 2, 1, 2, 2, False, True), (3, 2, 1, 100, 0, False, True),
         (1, 70, 9, 128, 128, False, True), (1000, 8, 4, 128, 128, False, True), (700, 3, 1, 112, 66, False, True),
         (20001, 1, 1, 64, 16, True, True), (10003, 4, 2, 64, 64, False, True), (20003, 1, 0, 128, 34, False, False),
         (19999, 1, 1, 256, 256, False, True)]


@pytest.mark.parametrize("T,hq,hk,dim,rot,interleaved,norm", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("where", ["whole", "part", "odd", "across"])
def test_forward_and_gradient(T, hq, hk, dim, rot, interleaved, norm, dtype, where):
    rng = np.random.default_rng(T + dim + rot)
    dt = TYPES[dtype]
    q, gq = (_rows(rng, T, hq, dim, dt, where) for _ in range(2))
    k, gk = (_rows(rng, T, hk, dim, dt, where) if hk else None for _ in range(2))
    wq, wk = (torch.from_numpy(1 + 0.3 * rng.standard_normal(dim)).to(DEV).to(dt) if norm else None for _ in range(2))
    pos = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, T).astype(np.int32)).to(DEV)
    theta, scale, eps = _theta(rot // 2), 1.25, 1e-5
    freq = K().kq_rotation_freq(theta)
    angle = ref.angles(pos.cpu().numpy(), ref.fractions(theta))
    out = [None if t is None else torch.full(t.shape, 7.0, dtype=dt, device=DEV) for t in (q, k)]
    K().kq_qk_rotate(q, k, out[0], out[1], freq, pos=pos, interleaved=interleaved, scale=scale, q_weight=wq,
                     k_weight=wk if hk else None, eps=eps)
    back = [None if t is None else torch.full_like(t, 7.0) for t in (q, k)]
    sums = [torch.full((dim,), 7.0, device=DEV) if norm and t is not None else None for t in (q, k)]
    ws = torch.empty(K().kq_qk_rotate_grad_workspace(gq), dtype=torch.uint8, device=DEV)
    args = dict(pos=pos, interleaved=interleaved, scale=scale, q_weight=wq, k_weight=wk if hk else None, eps=eps)
    K().kq_qk_rotate_grad(q if norm else None, k if norm else None, gq, gk, back[0], back[1], freq, gq_weight=sums[0],
                          gk_weight=sums[1], ws=ws, **args)
    for x, g, w, o, b, s in ((q, gq, wq, out[0], back[0], sums[0]), (k, gk, wk, out[1], back[1], sums[1])):
        if x is None:
            continue
        w = None if w is None else np64(w)
        y, size = ref.forward(np64(x), w, eps, angle, rot, interleaved, scale)
        _close(o, y, size, dt, 2.0 ** -19)
        gx, size, gw, wsize = ref.backward(np64(x), w, eps, np64(g), angle, rot, interleaved, scale)
        _close(b, gx, size, dt, 2.0 ** -18)
        if norm:
            _close(s, gw, wsize, torch.float32, 2.0 ** -16)


def test_in_place_and_positions_of_sequences_and_tokens_of_none():
    rng = np.random.default_rng(0)
    T, hq, hk, dim = 11, 3, 1, 64
    start = torch.tensor([0, 4, 4, 9], dtype=torch.int32, device=DEV)
    first = torch.tensor([100, 7, 0], dtype=torch.int32, device=DEV)
    pos = torch.tensor([100, 101, 102, 103, 0, 1, 2, 3, 4, 0, 0], dtype=torch.int32, device=DEV)
    q, k = (_rows(rng, T, h, dim, torch.float32, "part") for h in (hq, hk))
    w = torch.rand(dim, device=DEV)
    freq = K().kq_rotation_freq(_theta(32))
    want = [torch.empty(t.shape, device=DEV) for t in (q, k)]
    K().kq_qk_rotate(q, k, want[0], want[1], freq, pos=pos, q_weight=w)
    a, b = q.clone(), k.clone()
    K().kq_qk_rotate(q, k, q, k, freq, start=start, first=first, q_weight=w)
    for got, was, new in ((q, a, want[0]), (k, b, want[1])):
        assert torch.equal(got[:9], new[:9]) and torch.equal(got[9:], was[9:])
    # the same backwards, tokens of no sequence without a share in the weight's gradient
    sums = [torch.empty(dim, device=DEV) for _ in range(2)]
    ws = torch.empty(K().kq_qk_rotate_grad_workspace(a), dtype=torch.uint8, device=DEV)
    gq, gk = torch.randn(T, hq, dim, device=DEV), torch.randn(T, hk, dim, device=DEV)
    outs = [[torch.full(t.shape, 3.0, device=DEV) for t in (gq, gk)] for _ in range(2)]
    K().kq_qk_rotate_grad(a, None, gq, gk, outs[0][0], outs[0][1], freq, start=start, first=first, q_weight=w, gq_weight=sums[0], ws=ws)
    K().kq_qk_rotate_grad(a[:9], None, gq[:9], gk[:9], outs[1][0][:9], outs[1][1][:9], freq, pos=pos[:9], q_weight=w,
                          gq_weight=sums[1], ws=ws)
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    assert torch.allclose(sums[0], sums[1], rtol=1e-5, atol=1e-5)   # 2^-17 of at most 27 terms of size 10, in another split


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sequences_over_many_tokens_of_few_heads(dtype):
    """Several tokens to a warp, the last of them of no sequence: as by positions, and not written."""
    dt = TYPES[dtype]
    g = torch.Generator(DEV).manual_seed(2)
    counts = [7000, 0, 1, 9001, 4000]
    T, end = 20011, sum(counts)
    start = torch.tensor([0] + counts, device=DEV).cumsum(0).to(torch.int32)
    first = torch.tensor([5, 1, 100000, 0, 77], dtype=torch.int32, device=DEV)
    pos = torch.cat([torch.arange(f, f + n) for f, n in zip(first.tolist(), counts)] + [torch.zeros(T - end)]).to(DEV).to(torch.int32)
    q, k, gq, gk = (torch.randn(T, h, 64, device=DEV, generator=g).to(dt) for h in (1, 1, 1, 1))
    w = torch.rand(64, device=DEV, generator=g).to(dt)
    freq = K().kq_rotation_freq(_theta(32))
    ws = torch.empty(K().kq_qk_rotate_grad_workspace(q), dtype=torch.uint8, device=DEV)
    got = []
    for how in (dict(pos=pos[:end]), dict(start=start, first=first)):
        n = end if "pos" in how else T
        outs = [torch.full((T, 1, 64), 7.0, dtype=dt, device=DEV) for _ in range(4)] + [torch.empty(64, device=DEV) for _ in range(2)]
        K().kq_qk_rotate(q[:n], k[:n], outs[0][:n], outs[1][:n], freq, q_weight=w, k_weight=w, **how)
        K().kq_qk_rotate_grad(q[:n], k[:n], gq[:n], gk[:n], outs[2][:n], outs[3][:n], freq, q_weight=w, k_weight=w, gq_weight=outs[4],
                              gk_weight=outs[5], ws=ws, **how)
        got.append(outs)
    assert all(torch.equal(a, b) for a, b in zip(got[0][:4], got[1][:4])) and (got[1][0][end:] == 7).all()
    assert all(torch.allclose(a, b, rtol=0, atol=2.0 ** -17 * 20000) for a, b in zip(got[0][4:], got[1][4:]))   # of about 16000 in all


def test_no_positions_means_the_index():
    q = torch.randn(6, 2, 64, device=DEV)
    freq = K().kq_rotation_freq(_theta(16))
    a, b = torch.empty_like(q), torch.empty_like(q)
    K().kq_qk_rotate(q, None, a, None, freq)
    K().kq_qk_rotate(q, None, b, None, freq, pos=torch.arange(6, dtype=torch.int32, device=DEV))
    assert torch.equal(a, b)


def test_infinities_stay_in_their_pair_and_nan_in_its_row():
    q = torch.ones(1, 2, 64, device=DEV)
    q[0, 0, 3] = float("inf")     # pair (3, 19) of 32 rotated values
    q[0, 1, 50] = float("nan")    # not rotated
    out = torch.empty_like(q)
    K().kq_qk_rotate(q, None, out, None, K().kq_rotation_freq(_theta(16)))
    bad = ~torch.isfinite(out)
    assert bad[0, 0].nonzero().flatten().tolist() == [3, 19] and bad[0, 1].nonzero().flatten().tolist() == [50]
    K().kq_qk_rotate(q, None, out, None, K().kq_rotation_freq(_theta(16)), q_weight=torch.ones(64, device=DEV))
    assert torch.isnan(out[0, 1]).all()


def test_rows_of_zeros_and_no_tokens():
    q, w = torch.zeros(3, 2, 128, device=DEV), torch.ones(128, device=DEV)
    out, g = torch.empty_like(q), torch.empty(128, device=DEV)
    freq = K().kq_rotation_freq(_theta(64))
    K().kq_qk_rotate(q, None, out, None, freq, q_weight=w, eps=1e-6)
    assert torch.equal(out, q)
    ws = torch.empty(K().kq_qk_rotate_grad_workspace(q), dtype=torch.uint8, device=DEV)
    K().kq_qk_rotate_grad(q, None, q, None, out, None, freq, q_weight=w, gq_weight=g, ws=ws)
    assert torch.equal(out, q) and not g.any()
    g.fill_(5.0)
    K().kq_qk_rotate_grad(q[:0], None, q[:0], None, out[:0], None, freq, q_weight=w, gq_weight=g, ws=ws)
    assert not g.any()


@pytest.mark.parametrize("T,hq,hk", [(5, 3, 1), (3, 9, 5), (9001, 1, 1), (700, 33, 4)])
@pytest.mark.parametrize("dim", [64, 128, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_without_eps(T, hq, hk, dim, dtype):
    """Heads that fill no whole number of a warp's rows: what is not there adds nothing, though its norm would be infinite."""
    rng = np.random.default_rng(T + dim)
    dt = TYPES[dtype]
    q, gq = (_rows(rng, T, hq, dim, dt, "whole") for _ in range(2))
    k, gk = (_rows(rng, T, hk, dim, dt, "whole") for _ in range(2))
    w = torch.from_numpy(1 + 0.3 * rng.standard_normal(dim)).to(DEV).to(dt)
    theta = _theta(dim // 2)
    freq, angle = K().kq_rotation_freq(theta), ref.angles(np.arange(T), ref.fractions(theta))
    out, back = ([torch.empty_like(t) for t in (q, k)] for _ in range(2))
    sums = [torch.empty(dim, device=DEV) for _ in range(2)]
    ws = torch.empty(K().kq_qk_rotate_grad_workspace(gq), dtype=torch.uint8, device=DEV)
    K().kq_qk_rotate(q, k, *out, freq, q_weight=w, k_weight=w, eps=0.0)
    K().kq_qk_rotate_grad(q, k, gq, gk, *back, freq, q_weight=w, k_weight=w, eps=0.0, gq_weight=sums[0], gk_weight=sums[1], ws=ws)
    for x, g, o, b, s in ((q, gq, out[0], back[0], sums[0]), (k, gk, out[1], back[1], sums[1])):
        y, size = ref.forward(np64(x), np64(w), 0.0, angle, dim, False, 1.0)
        _close(o, y, size, dt, 2.0 ** -19)
        gx, size, gw, wsize = ref.backward(np64(x), np64(w), 0.0, np64(g), angle, dim, False, 1.0)
        _close(b, gx, size, dt, 2.0 ** -18)
        _close(s, gw, wsize, torch.float32, 2.0 ** -16)


def test_gradient_matches_differences_of_the_kernel():
    """In float32 along a direction v of size 1 an element: forward errors of 2^-19 of about 2 a value, over 2 e = 2^-4, summed
    over n values with signs of their own, against the difference's e^2 / 6 times the third derivative (below 20)."""
    g = torch.Generator(DEV).manual_seed(0)
    T, h, dim, e = 4, 2, 64, 2.0 ** -5
    x, gy, v = (torch.randn(T, h, dim, device=DEV, generator=g) for _ in range(3))
    w = torch.rand(dim, device=DEV, generator=g) + 0.5
    freq = K().kq_rotation_freq(_theta(32))

    def loss(x):
        out = torch.empty_like(x)
        K().kq_qk_rotate(x, None, out, None, freq, q_weight=w)
        return (out.double() * gy).sum().item()

    gx = torch.empty_like(x)
    K().kq_qk_rotate_grad(x, None, gy, None, gx, None, freq, q_weight=w)
    n = T * h * dim
    got = (gx.double() * v).sum().item()
    diff = (loss(x + e * v) - loss(x - e * v)) / (2 * e)
    assert abs(got - diff) <= n ** 0.5 * (2.0 ** -18 / (2 * e) + 20 * e * e / 6)


def test_results_do_not_depend_on_the_run_and_replay_in_a_graph():
    g = torch.Generator(DEV).manual_seed(1)
    q, k = (torch.randn(3000, h, 128, device=DEV, generator=g).bfloat16() for h in (8, 2))
    w = torch.rand(128, device=DEV, generator=g).bfloat16()
    pos = torch.arange(3000, dtype=torch.int32, device=DEV)
    freq = K().kq_rotation_freq(_theta(64))
    ws = torch.empty(K().kq_qk_rotate_grad_workspace(q), dtype=torch.uint8, device=DEV)

    def run():
        outs = [torch.empty_like(t) for t in (q, k, q, k)] + [torch.empty(128, device=DEV) for _ in range(2)]
        K().kq_qk_rotate(q, k, outs[0], outs[1], freq, pos=pos, q_weight=w, k_weight=w)
        K().kq_qk_rotate_grad(q, k, q, k, outs[2], outs[3], freq, pos=pos, q_weight=w, k_weight=w, gq_weight=outs[4],
                              gk_weight=outs[5], ws=ws)
        return outs

    a, b = run(), run()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = run()
    q.neg_()
    graph.replay()
    d = run()
    assert all(torch.equal(x, y) for x, y in zip(c, d)) and not torch.equal(a[0], c[0])
