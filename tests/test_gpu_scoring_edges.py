"""GPU checks of kq_token_logprobs where float32 logits lie close together: the top values' order is that of
all 32 bits, whatever the block sizes."""
import math

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


def _run(x, target, top):
    T = x.shape[0]
    logp, h, lse = (torch.full((T,), 5.0, device=DEV) for _ in range(3))
    ids = torch.full((T, top), -1, dtype=torch.int32, device=DEV)
    tl = torch.full((T, top), 5.0, device=DEV)
    K().kq_token_logprobs(x, target, logp, entropy=h, lse=lse, top_id=ids, top_logp=tl)
    torch.cuda.synchronize()
    return logp, h, lse, ids, tl


# rows for a cluster a row, blocks of 1024, of 512 and smaller ones (the last by the row's length)
@pytest.mark.parametrize("T,V", [(200, 2000), (1, 8000), (100, 8000), (200, 8000), (330, 8000), (3, 32000), (100, 32000),
                                 (330, 32000), (2, 128000), (40, 128000), (100, 128000), (200, 128000), (330, 128000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,top", [("close", 5), ("close", 32), ("shifted", 5), ("shifted", 20), ("equal", 7), ("rising", 9),
                                      ("falling", 9)])
def test_top_values_that_share_their_leading_bits(T, V, dtype, kind, top):
    """close: logits near 100, thousands of them in one bf16 value. shifted: forbidden tokens moved by -1e4, fewer
    allowed ones than asked for. rising, falling: a step of one unit in the last place from token to token.
    Bound of the log probabilities: 2^-18 (1 + |m| + |value|), as e^(x - m) is off by 2^-21 and the sums by less."""
    g = torch.Generator(DEV).manual_seed(V + T + top)
    x = torch.randn(T, V, device=DEV, generator=g)
    if kind == "close":
        x = 100.25 + 0.03 * x
    elif kind == "shifted":
        allowed = torch.randint(0, V, (T, 3), device=DEV, generator=g)
        x = (x - 1e4).scatter_(1, allowed, x.gather(1, allowed))
    elif kind == "equal":
        x = torch.full_like(x, -3.1415)
    else:
        step = torch.arange(V, dtype=torch.int32, device=DEV)
        x = ((step if kind == "rising" else V - step) + 0x42C80000).expand(T, V).contiguous().view(torch.float32)   # from 100
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    target = torch.randint(0, V, (T,), device=DEV, generator=g)
    logp, h, lse, ids, tl = _run(x, target, top)
    want = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(ids.long(), want), f"{int((ids != want).any(1).sum())} of {T} rows"
    lp = torch.log_softmax(x.double(), 1)
    exact = lp.gather(1, want)
    assert ((tl - exact).abs() <= 2.0 ** -18 * (1 + x.double().amax(1, keepdim=True).abs() + exact.abs())).all()
