"""kq_linear_logprobs of more rows than are scored at once: a row's results are the bits that it has in a call of its own
block, and within the bounds of 64 bits (those of test_gpu_linear_logprobs.py, whose derivation they share)."""
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


def _score(x, w, y, poison, info=None, all_of=True):
    outs = [torch.full((x.shape[0],), 5.0, device=DEV) for _ in range(3 if all_of else 1)]
    n = K().kq_linear_logprobs_workspace(x, w)
    raw = torch.full((n + 4096,), poison, dtype=torch.uint8, device=DEV)
    K().kq_linear_logprobs(x, w, y, outs[0], raw[:n], *(outs[1:] if all_of else ()), info=info)
    assert (raw[n:] == poison).all()
    return outs


# two blocks of 2304 and 1793 rows, two of 2560 and 2440, two of 4352 and 3969, three of 4096, 4096 and 3906
@pytest.mark.parametrize("T,V,d", [(4097, 200001, 64), (5000, 262144, 72), (8321, 100003, 136), (12098, 200001, 8)])
def test_rows_in_blocks(T, V, d):
    g = torch.Generator(DEV).manual_seed(T)
    w = (torch.randn(V, d, device=DEV, generator=g) * (2.5 / d ** 0.5)).bfloat16()
    y = torch.randint(-V // 8, V, (T,), device=DEV, generator=g)
    wide = torch.randn(T, d + 24, device=DEV, generator=g).bfloat16()
    x = wide[:, 8:8 + d]
    room = max(4096, (1 << 24) // -(-V // 64) // 4096 * 4096)
    block = -(-(-(-T // -(-T // room))) // 256) * 256
    assert block < T
    got = _score(x, w, y, 255)
    logp, ent, lse = got
    assert torch.equal(_score(x, w, y, 127, all_of=False)[0], logp)
    for r in range(0, T, block):
        for a, b in zip(got, _score(x[r:r + block], w, y[r:r + block], 127)):
            assert torch.equal(a[r:r + block], b)
    # 64 bits, rows beside the border and the last ones
    rows = torch.tensor([0, 1, block - 2, block - 1, block, min(block + 1, T - 1), T - 2, T - 1], device=DEV)
    X, W = x[rows].double(), w.double()
    z = X @ W.T
    e = (2.0 ** -18 * (X.abs() @ W.abs().T)).amax(1)
    m, exact = z.amax(1), torch.logsumexp(z, 1)
    lp = z - exact[:, None]
    H = -(lp.exp() * lp).sum(1)
    want = torch.where(y[rows] >= 0, lp.gather(1, y[rows].clamp(min=0)[:, None])[:, 0], 0.0)

    def u(v):
        return 2.0 ** -18 * (1 + m.abs() + v.abs())

    assert ((lse[rows] - exact).abs() <= e + u(exact)).all()
    assert ((logp[rows] - want).abs() <= 2 * e + u(want)).all()
    assert ((ent[rows] - H).abs() <= (lp.exp() * (lp + H[:, None]).abs()).sum(1) * 2 * e + u(H)).all()


def test_a_target_past_the_vocabulary_in_a_later_block():
    T, V, d = 4200, 200000, 8
    x, w = torch.randn(T, d, device=DEV).bfloat16(), torch.randn(V, d, device=DEV).bfloat16()
    y = torch.zeros(T, dtype=torch.int64, device=DEV)
    info = torch.zeros(1, dtype=torch.int32, device=DEV)
    _score(x, w, y, 0, info)
    assert K().kq_check(info)[0] == K().KQ_OK
    y[4150] = V
    logp, _, _ = _score(x, w, y, 0, info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG
    assert torch.isnan(logp).nonzero().flatten().tolist() == [4150]


def test_blocks_replay_in_a_graph():
    T, V, d = 4200, 200000, 64
    g = torch.Generator(DEV).manual_seed(1)
    x, w = torch.randn(T, d, device=DEV, generator=g).bfloat16(), torch.randn(V, d, device=DEV, generator=g).bfloat16()
    y = torch.randint(0, V, (T,), device=DEV, generator=g)
    outs = [torch.empty(T, device=DEV) for _ in range(3)]
    ws = torch.empty(K().kq_linear_logprobs_workspace(x, w), dtype=torch.uint8, device=DEV)

    def run():
        K().kq_linear_logprobs(x, w, y, outs[0], ws, entropy=outs[1], lse=outs[2])

    run()
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(2):
        for t in outs:
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
