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


@pytest.mark.parametrize("V", [50, 9001, 60000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["infinite", "lowest"])
@pytest.mark.parametrize("rows", [8, 200, 400])
def test_entropy_of_rows_with_a_huge_maximum_and_masked_tokens(V, dtype, mask, rows):
    """Row i: i % 4 + 1 tokens share a maximum between 1e37 and 3e38, most others are masked, some 0. The maximum's
    tokens have differences of exactly 0 and the others probability 0, so logp is -ln k and the entropy ln k, each one
    logarithm of a small whole number: within 2^-19 (1 + the value)."""
    ty = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.full((rows, V), -math.inf if mask == "infinite" else torch.finfo(ty).min, dtype=ty, device=DEV)
    x[:, 1::7] = 0
    tops = [1e37, 2.9e37, 3.1e37, 3.7e37, 5e37, 9.9e37, 1.01e38, 3e38]
    k = [1 + i % 4 for i in range(rows)]
    for i in range(rows):
        x[i, 5:5 + 3 * k[i]:3] = tops[i % 8]
    logp, h, lse, ids, tl = _run(x, torch.full((rows,), 5, device=DEV), 2)
    want = torch.tensor(k, dtype=torch.float64, device=DEV).log()
    tol = 2.0 ** -19 * (1 + want)
    assert ((logp + want).abs() <= tol).all() and ((h - want).abs() <= tol).all()
    assert ((lse - x[:, 5].double()).abs() <= 2.0 ** -22 * x[:, 5].double()).all()
    assert (ids[:, 0] == 5).all() and ((tl[:, 0] + want).abs() <= tol).all()


@pytest.mark.parametrize("V", [50, 9001, 60000])
@pytest.mark.parametrize("rows", [14, 210, 420])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_whose_logits_are_all_large(V, rows, dtype):
    """Row i: i % 4 + 1 tokens share a maximum of either sign, the others lie at least 2^-7 of it lower, which is more than
    a thousand: probability 0. Up to 2^30 the reference is off by up to 64 powers of two, so terms of that size are
    rounded (2^-18 each, three of them) where they cancel; beyond, differences are exact: within 2^-16 (1 + the value)."""
    ty = torch.bfloat16 if dtype == "bf16" else torch.float32
    tops = torch.tensor([2e5, -3e7, 2e8, -1e9, 1.05e9, 1.2e9, -3e9, 7e9, 1e10, -1e12, 1e15, 1e20, -1e30, 2.5e37], device=DEV)
    k = [1 + i % 4 for i in range(rows)]
    m = tops.repeat(rows // 14)[:, None]
    x = (m - m.abs() * (0.01 + torch.rand(rows, V, device=DEV, generator=torch.Generator(DEV).manual_seed(V)))).to(ty)
    m = m.to(ty)
    for i in range(rows):
        x[i, 5:5 + 3 * k[i]:3] = m[i, 0]
    logp, h, lse, ids, tl = _run(x, torch.full((rows,), 5, device=DEV), 1)
    want = torch.tensor(k, dtype=torch.float64, device=DEV).log()
    tol = 2.0 ** -16 * (1 + want)
    assert ((logp + want).abs() <= tol).all() and ((h - want).abs() <= tol).all()
    exact = m[:, 0].double() + want
    assert ((lse - exact).abs() <= 2.0 ** -22 * exact.abs()).all()
    assert (ids[:, 0] == 5).all() and ((tl[:, 0] + want).abs() <= tol).all()


@pytest.mark.parametrize("T,V,top", [(1, 900, 3), (200, 5003, 3), (400, 28505, 5), (3, 60000, 2), (40, 128000, 0), (400, 128000, 20)])
@pytest.mark.parametrize("shift", [0, 3e3, -3e5, 3e6, -1.5e7, -2e7, 1e8, -9e8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_shift_of_all_logits_costs_no_precision(T, V, top, shift, dtype):
    """Logits spread by some 30 about a common value: differences within a row are exact, so the bound does not grow
    with the shift. A term is off by 2^-24 of its own size and a power of two by 2^-21: 2^-18 (1 + |value|) in all up to 2^24, and
    up to 2^30, where the reference is off by up to 64 powers of two (2^-18 of rounding, three times), 2^-16 (1 + |value|).
    Rounding the difference of a log-sum costs 2^-24 of it twice."""
    g = torch.Generator(DEV).manual_seed(V)
    x = (torch.randn(T, V, device=DEV, generator=g) * 30 + shift).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    target = torch.randint(0, V, (T,), device=DEV, generator=g)
    logp, h, lse, ids, tl = _run(x, target, max(top, 1))
    lp = torch.log_softmax(x.double(), 1)
    eps = 2.0 ** -18 if abs(shift) < 2 ** 24 else 2.0 ** -16
    want = lp.gather(1, target[:, None])[:, 0]
    entropy = -(lp.exp() * lp).sum(1)
    tops = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :max(top, 1)]
    assert torch.equal(ids.long(), tops)
    for got, exact in ((logp, want), (h, entropy), (tl, lp.gather(1, tops))):
        assert ((got - exact).abs() <= eps * (1 + exact.abs())).all(), float(((got - exact).abs() / (1 + exact.abs())).max())
    exact = torch.logsumexp(x.double(), 1)
    assert ((lse - exact).abs() <= 2.0 ** -18 + 2.0 ** -22 * exact.abs()).all()
