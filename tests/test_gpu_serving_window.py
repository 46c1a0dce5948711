"""Rotation, window and scoring of hidden states as a model strings them together: projections, norm and rotation, append,
attention with a window, the head's log probabilities and the gradient that goes back through them."""
import math

import numpy as np
import pytest
import torch

import rotate_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_07964_gb300 import build
    build.build()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_block_is_dense_attention_with_window_and_rotation_over_the_cached_values():
    """Against 64 bits: keys and values as the cache holds them, queries rotated by the reference. The cached keys are also
    within half a step of the rotated ones. Bounds as in the tests of the parts: a query is off by 2^-19 of its pair's size, which a
    score's 2^-18 of its terms takes in twice."""
    from paper_2607_07964_gb300.serving import AttentionBlock, KvCache, Rotation, rotation_theta
    g = torch.Generator(DEV).manual_seed(0)
    d, heads, kv, dim, window, sink = 96, 4, 2, 64, 7, 2
    W = {n: torch.randn(s, d, device=DEV, generator=g) / math.sqrt(d) for n, s in (("q", heads * dim), ("k", kv * dim), ("v", kv * dim))}
    O = torch.randn(d, heads * dim, device=DEV, generator=g) / 16
    made = {}

    def proj(n):
        def f(x):
            made.setdefault(n, []).append((x @ (O if n == "o" else W[n]).T).clone())
            return made[n][-1].clone()
        return f

    theta, scale = rotation_theta(32, stretch=4.0, original=16)
    wq, wk = (torch.rand(dim, device=DEV, generator=g) + 0.5 for _ in range(2))
    cache = KvCache(2, kv, dim, 64, page=16)
    block = AttentionBlock({n: proj(n) for n in "qkvo"}, heads, cache, Rotation(theta, scale, q_weight=wq, k_weight=wk), window, sink)
    have, attended = [0, 0], []
    f = ref.fractions(theta)
    for most, counts in ((9, [9, 4]), (1, [1, 1]), ([0, 3], [0, 3]), (20, [20, 1]), (1, [1, 1])):
        x = torch.randn(sum(counts), d, device=DEV, generator=g)
        y = block(x, _i32([0, counts[0], sum(counts)]), most)
        assert torch.equal(y, x + made["o"][-1])
        attended.append((counts, list(have)))
        have = [a + b for a, b in zip(have, counts)]
    cache.check()
    ck, cv = (t.double().cpu().numpy() for t in cache.read())
    for step, (counts, before) in enumerate(attended):
        k = made["k"][step].double().cpu().numpy().reshape(-1, kv, dim)
        pos = np.concatenate([before[b] + np.arange(n) for b, n in enumerate(counts)])
        angle = ref.angles(pos, f)
        kr, _ = ref.forward(k, wk.double().cpu().numpy(), 1e-6, angle, 32, False, scale)
        i = 0
        for b, n in enumerate(counts):
            for j in range(n):
                at = before[b] + j
                span = kr[i].max(-1) - kr[i].min(-1)
                assert np.all(np.abs(ck[b, at] - kr[i]).max(-1) <= span / 15 * 1.02 / 2 + 1e-5)
                i += 1
    # the attention itself, on the last step's queries
    counts, before = attended[-1]
    q = made["q"][-1].view(-1, heads, dim).clone()
    k = made["k"][-1].view(-1, kv, dim).clone()
    block.rotation(q, k, pos=_i32(before))
    got = cache.attend(q, _i32([0, 1, 2]), window=window, sink=sink).double().cpu().numpy()
    qd = q.double().cpu().numpy()
    for b in range(2):
        n = have[b]
        j = [t for t in range(n) if t >= n - window or t < sink]
        for h in range(heads):
            kk, vv = ck[b, j, h // 2], cv[b, j, h // 2]
            s = kk @ qd[b, h] / math.sqrt(dim)
            p = np.exp(s - s.max())
            want = (p / p.sum()) @ vv
            terms = (np.abs(kk) @ np.abs(qd[b, h])).max() / math.sqrt(dim)
            assert np.abs(got[b, h] - want).max() <= 2.0 ** -17 * np.abs(vv).max() * (1 + terms)


def test_a_cache_that_evicts_has_no_window():
    from paper_2607_07964_gb300.serving import KvCache
    c = KvCache(1, 1, 64, 32, page=16, budget=16)
    with pytest.raises(ValueError, match="window"):
        c.attend(torch.zeros(1, 1, 64, device=DEV), _i32([0, 1]), window=4)


def test_a_captured_step_with_rotation_and_window_replays_as_a_plain_one():
    from paper_2607_07964_gb300.serving import AttentionBlock, KvCache, Rotation, rotation_theta
    g = torch.Generator(DEV).manual_seed(3)
    d = 64
    W = {n: torch.randn(128 if n == "q" else 64, d, device=DEV, generator=g) / 8 for n in "qkv"}
    W["o"] = torch.randn(d, 128, device=DEV, generator=g) / 8
    theta, scale = rotation_theta(64)
    plain, made = (AttentionBlock({n: (lambda w: lambda x: x @ w.T)(W[n]) for n in "qkvo"}, 2, KvCache(2, 1, 64, 40, page=16),
                                  Rotation(theta, scale), 5, 1) for _ in range(2))
    start = _i32([0, 1, 2])
    xs = torch.randn(12, 2, d, device=DEV, generator=g)
    want = [plain(x, start, 1).clone() for x in xs]
    got = [made(x, start, 1).clone() for x in xs[:3]]
    static = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = made(static, start, 1)
    for x in xs[3:]:
        static.copy_(x)
        graph.replay()
        got.append(out.clone())
    made.cache.check()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_hidden_states_score_as_their_logits_do():
    """Against score on the logits in fp32: both within the bounds of their tests."""
    from paper_2607_07964_gb300.serving import score, score_hidden, score_hidden_grad
    g = torch.Generator(DEV).manual_seed(5)
    T, V, d = 130, 3001, 256
    x, w = torch.randn(T, d, device=DEV, generator=g).bfloat16(), (torch.randn(V, d, device=DEV, generator=g) / 8).bfloat16()
    y = torch.randint(0, V, (T,), device=DEV, generator=g)
    z = (x.double() @ w.double().T).float()
    logp, entropy, lse = score_hidden(x, w, y)
    want, h, _, _ = score(z, y)
    tol = 2 * 2.0 ** -18 * (x.double().abs() @ w.double().abs().T).amax(1) + 2.0 ** -16 * (1 + z.abs().amax(1) + want.abs())
    assert ((logp - want).abs() <= tol).all() and ((entropy - h).abs() <= tol * (1 + h)).all()
    gx, gw = score_hidden_grad(x, w, y, lse, torch.full((T,), -1.0 / T, device=DEV))
    p = torch.softmax(z.double(), 1)
    p[torch.arange(T, device=DEV), y] -= 1
    # 2^-8 for the logits' gradient in bf16, 2^-8 for the outputs, twice
    for got, exact, size in ((gx, p @ w.double() / T, p.abs() @ w.double().abs() / T), (gw, p.T @ x.double() / T, p.abs().T @ x.double().abs() / T)):
        assert ((got.double() - exact).abs() <= 2.0 ** -7 * size + 2.0 ** -7 * exact.abs()).all()
    assert score_hidden_grad(x, w, y, lse, torch.ones(T, device=DEV), of_head=False)[1] is None


def test_rotation_gradient_in_place():
    from paper_2607_07964_gb300.serving import Rotation, rotation_theta
    g = torch.Generator(DEV).manual_seed(7)
    theta, scale = rotation_theta(64)
    w = torch.rand(64, device=DEV, generator=g) + 0.5
    r = Rotation(theta, scale, interleaved=True, q_weight=w, k_weight=w)
    q, k, gq, gk = (torch.randn(5, h, 64, device=DEV, generator=g) for h in (4, 1, 4, 1))
    pos = _i32([0, 3, 100, 7, 7])
    angle = ref.angles(pos.cpu().numpy(), ref.fractions(theta))
    want = [ref.backward(t.double().cpu().numpy(), w.double().cpu().numpy(), 1e-6, u.double().cpu().numpy(), angle, 64, True, scale)
            for t, u in ((q, gq), (k, gk))]
    sums = r.grad(q, k, gq, gk, pos=pos)
    for got, s, (gx, size, gw, wsize) in zip((gq, gk), sums, want):
        assert np.all(np.abs(got.double().cpu().numpy() - gx) <= 2.0 ** -18 * size + 2.0 ** -24 * np.abs(gx) + 1e-30)
        assert np.all(np.abs(s.double().cpu().numpy() - gw) <= 2.0 ** -16 * wsize)
    r = Rotation(theta, scale)
    assert r.grad(None, None, gq, gk, pos=pos) == (None, None)
    # queries alone, where the keys have a norm too
    r = Rotation(theta, scale, q_weight=w, k_weight=w)
    a, b = q.clone(), torch.empty_like(q)
    r(a, None, pos=pos)
    r(b.copy_(q), k.clone(), pos=pos)
    assert torch.equal(a, b)
    one, two = gq.clone(), gq.clone()
    sums, both = r.grad(q, None, one, None, pos=pos), r.grad(q, k, two, gk, pos=pos)
    assert sums[1] is None and torch.equal(one, two) and torch.allclose(sums[0], both[0], rtol=1e-5, atol=1e-5)   # 20 terms, another split


def test_example_with_a_window_decodes_and_scores():
    from paper_2607_07964_gb300.serving import example
    ids, logps, block = example(steps=12, budget=None, window=16)
    again = example(steps=12, budget=None, window=16)
    assert torch.equal(ids, again[0]) and torch.equal(logps, again[1])
    assert ids.shape == (12, 3) and torch.isfinite(logps).all() and (logps <= 0).all()
    assert block.cache.lens.tolist() == [52, 19, 35]
