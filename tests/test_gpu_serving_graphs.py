"""KvCache through captured graphs and on several streams."""
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


def _step(c, x, start):
    c.append(x[0], x[1], start, 1)
    return c.attend(x[2], start)


@pytest.mark.parametrize("budget", [None, 20])
def test_a_captured_step_replays_as_a_plain_one(budget):
    from paper_2607_07964_gb300.serving import KvCache
    g = torch.Generator(DEV).manual_seed(0)
    start = torch.arange(3, dtype=torch.int32, device=DEV)
    xs = [[torch.randn(2, h, 64, device=DEV, generator=g) for h in (1, 1, 4)] for _ in range(12)]
    plain, made = (KvCache(2, 1, 64, 40, page=16, budget=budget, recent=0 if budget is None else 4) for _ in range(2))
    want = [_step(plain, x, start).clone() for x in xs]
    got = [_step(made, x, start).clone() for x in xs[:3]]   # an odd number of steps before the capture
    static = [t.clone() for t in xs[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(made, static, start)
    for i, x in enumerate(xs[3:]):
        if i % 4 == 1:   # plain steps between the replays
            got.append(_step(made, x, start).clone())
            continue
        for a, b in zip(static, x):
            a.copy_(b)
        graph.replay()
        got.append(out.clone())
    made.check()
    assert made.lens.tolist() == [12, 12] and made.seen.tolist() == [12, 12]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a, b) for a, b in zip(made.read(), plain.read()))


@pytest.mark.parametrize("budget", [None, 20])
def test_replays_count_for_what_fits_afterwards(budget):
    from paper_2607_07964_gb300.serving import KvCache
    start = torch.arange(2, dtype=torch.int32, device=DEV)
    x = [torch.randn(1, h, 64, device=DEV) for h in (1, 1, 4)]
    c = KvCache(1, 1, 64, 32, page=16, budget=budget, recent=0 if budget is None else 4)
    _step(c, x, start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(c, x, start)
    for _ in range(31):
        graph.replay()
    assert c.lens.tolist() == [32]
    if budget is None:
        with pytest.raises(ValueError, match="do not fit"):
            _step(c, x, start)
    else:
        _step(c, x, start)
        assert c.lens.tolist() == [21] and c.seen.tolist() == [33]
    c.check()


def test_a_captured_attention_sees_what_plain_calls_append():
    from paper_2607_07964_gb300.serving import KvCache
    start = torch.arange(2, dtype=torch.int32, device=DEV)
    c = KvCache(1, 1, 64, 32, page=16)
    x = [torch.randn(1, h, 64, device=DEV) for h in (1, 1, 4)]
    _step(c, x, start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.attend(x[2], start)
    for _ in range(3):
        y = torch.randn(2, 1, 1, 64, device=DEV)
        c.append(y[0], y[1], start, 1)
        graph.replay()
        assert torch.equal(out, c.attend(x[2], start))
    c.check()
    assert c.lens.tolist() == [4]


def test_a_workspace_that_a_graph_writes_to_is_kept():
    from paper_2607_07964_gb300.serving import KvCache
    c = KvCache(1, 1, 64, 64, page=16)
    x = [torch.randn(1, h, 64, device=DEV) for h in (1, 1, 4)]
    start, big = (torch.tensor([0, n], dtype=torch.int32, device=DEV) for n in (1, 40))
    _step(c, x, start)
    at, size = c._ws.data_ptr(), c._ws.numel()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(x[2], start)
    torch.cuda.synchronize()
    c.attend(torch.randn(40, 64, 64, device=DEV), big)   # a larger one; the first 39 tokens see nothing
    assert c._ws.data_ptr() != at
    others = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(3)]
    assert all(t.data_ptr() != at for t in others)
