"""Rotation, attention with a window and scoring of hidden states write nothing outside their outputs and workspaces: each
lies between guard regions that hold a pattern before and after."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, GUARD = "cuda", 4096


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_07964_gb300 import build
    build.build()


def K():
    from paper_2607_07964_gb300 import kronq
    return kronq


class Guarded:
    def __init__(self):
        self.all = []

    def __call__(self, *shape, dtype=torch.float32):
        n = torch.empty(0, dtype=dtype).element_size()
        for s in shape:
            n *= s
        raw = torch.full((GUARD + n + GUARD + (-n) % 256,), 0x5A, dtype=torch.uint8, device=DEV)
        self.all.append((raw, n))
        return raw[GUARD:GUARD + n].view(dtype).view(*shape)

    def check(self):
        for raw, n in self.all:
            assert (raw[:GUARD] == 0x5A).all() and (raw[GUARD + n:] == 0x5A).all()


@pytest.mark.parametrize("T,dim,rot,dtype", [(1, 128, 128, torch.bfloat16), (37, 80, 34, torch.float32), (1000, 64, 64, torch.bfloat16),
                                             (3, 33, 22, torch.bfloat16), (5, 256, 100, torch.float32)])
def test_rotation(T, dim, rot, dtype):
    new = Guarded()
    q, k = (torch.randn(T, h, dim, device=DEV).to(dtype) for h in (5, 1))
    w = torch.ones(dim, device=DEV).to(dtype)
    freq = K().kq_rotation_freq([0.5 ** j for j in range(rot // 2)])
    qo, ko, gq, gk = (new(T, h, dim, dtype=dtype) for h in (5, 1, 5, 1))
    sq, sk = new(dim), new(dim)
    ws = new(K().kq_qk_rotate_grad_workspace(q), dtype=torch.uint8)
    K().kq_qk_rotate(q, k, qo, ko, freq, q_weight=w, k_weight=w)
    K().kq_qk_rotate_grad(q, k, q, k, gq, gk, freq, q_weight=w, k_weight=w, gq_weight=sq, gk_weight=sk, ws=ws)
    new.check()


@pytest.mark.parametrize("heads,group,dim,page,window,sink", [(1, 1, 64, 16, 1, 0), (2, 8, 128, 64, 50, 4), (3, 5, 64, 48, 33, 40)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_window(heads, group, dim, page, window, sink, dtype):
    new = Guarded()
    lens = torch.tensor([300, 0, 31, 299], dtype=torch.int32, device=DEV)
    start = torch.tensor([0, 2, 2, 3, 12], dtype=torch.int32, device=DEV)
    per = -(-300 // page)
    cache = torch.randint(0, 60, (4 * per, heads, page * (dim + 8)), dtype=torch.uint8, device=DEV)
    table = torch.randperm(4 * per, device=DEV).to(torch.int32).view(4, per)
    q = torch.randn(12, heads * group, dim, device=DEV).to(dtype)
    out, lse = new(12, heads * group, dim, dtype=dtype), new(12, heads * group)
    ws = new(K().kq_kv_attend_workspace(q, cache, table), dtype=torch.uint8)
    before = cache.clone()
    K().kq_kv_attend_window(q, start, lens, cache, table, out, ws, 0.1, window, sink, lse=lse)
    new.check()
    assert torch.equal(cache, before)


@pytest.mark.parametrize("T,V,d", [(1, 1, 8), (2, 200, 72), (33, 1000, 264), (96, 4097, 136), (128, 129, 1000), (129, 257, 64), (700, 3001, 520),
                                   (1, 10241, 8), (96, 12001, 136), (128, 20000, 264),
                                   (1, 1000, 4096), (40, 2001, 2056), (100, 4000, 1032)])
def test_linear(T, V, d):
    new = Guarded()
    x, w = torch.randn(T, d, device=DEV).bfloat16(), (torch.randn(V, d, device=DEV) / d ** 0.5).bfloat16()
    y = torch.randint(-1, V, (T,), device=DEV)
    logp, h, lse = new(T), new(T), new(T)
    gx, gw = new(T, d, dtype=torch.bfloat16), new(V, d, dtype=torch.bfloat16)
    ws = new(K().kq_linear_logprobs_workspace(x, w), dtype=torch.uint8)
    gs = new(K().kq_linear_logprobs_grad_workspace(x, w), dtype=torch.uint8)
    K().kq_linear_logprobs(x, w, y, logp, ws, entropy=h, lse=lse)
    K().kq_linear_logprobs_grad(x, w, y, lse, logp, gs, gx=gx, gw=gw, entropy=h, g_entropy=h)
    new.check()
    assert torch.isfinite(gx).all() and torch.isfinite(gw).all()
