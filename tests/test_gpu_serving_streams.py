"""KvCache used on several streams."""
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


def test_a_workspace_that_another_stream_uses_is_not_given_away():
    """The workspace of a first stream, used on a second one and replaced there while its kernels are still to run: the
    allocator may not hand its memory to the first stream."""
    from paper_2607_07964_gb300.serving import KvCache
    c = KvCache(1, 1, 64, 64, page=16)
    k, q = torch.randn(1, 1, 64, device=DEV), torch.randn(1, 4, 64, device=DEV)
    start = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    big = torch.tensor([0, 40], dtype=torch.int32, device=DEV)
    q40 = torch.randn(40, 64, 64, device=DEV)
    torch.cuda.synchronize()
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(first):
        c.append(k, k, start, 1)
        c.attend(q, start)
    at, size = c._ws.data_ptr(), c._ws.numel()
    second.wait_stream(first)
    with torch.cuda.stream(second):
        torch.cuda._sleep(200_000_000)   # a tenth of a second: what follows waits its turn
        c.attend(q, start)
        c.attend(q40, big)               # a larger workspace; the first 39 tokens see nothing
        assert c._ws.data_ptr() != at
        with torch.cuda.stream(first):
            other = torch.empty(size, dtype=torch.uint8, device=DEV)
        assert other.data_ptr() != at
    torch.cuda.synchronize()
    c.check()
