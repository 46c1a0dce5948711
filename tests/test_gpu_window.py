"""GPU checks of kq_kv_attend_window against 64 bits, with the bounds of kq_kv_attend's tests: a score is off by at most
e = 2^-18 |scale| sum |q| max (15 |s| + |o|), and with M = sum_j p_j (15 |s_j| + |o_j|) of the values
    |out - exact| <= (2 e + 2^-18) M                      fp32
    |out - exact| <= (2 e + 2^-9) M + 2^-8 |exact|        bf16
    |lse - exact| <= 2 e + 2^-20 (1 + |exact|)."""
import numpy as np
import pytest
import torch

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


def _pool(rng, batch, per, heads, dim, page):
    """Pages in an order of their own; values [pages, 2, heads, page, dim] and the size 15 |s| + |o| of each row, in 64 bits."""
    pages, g = batch * per + 2, page // 16
    codes = rng.integers(0, 256, (pages, heads, g, 2, 16, dim // 2), dtype=np.uint8)
    size = 0.2 * np.exp(0.3 * rng.standard_normal((pages, heads, g, 2, 16)))
    grid = np.stack([size, -7.5 * size * (1 + 0.1 * rng.standard_normal(size.shape))], -1).astype(np.float32)
    bits = torch.from_numpy(grid).bfloat16()
    so = bits.double().numpy()
    raw = bits.view(torch.int16).numpy().view(np.uint8).reshape(pages, heads, g, -1)
    data = np.concatenate([codes.reshape(pages, heads, g, -1), raw], -1).reshape(pages, heads, page * (dim + 8))
    val = np.stack([codes & 15, codes >> 4], -1).reshape(pages, heads, g, 2, 16, dim) * so[..., :1] + so[..., 1:]
    mag = 15 * np.abs(so[..., 0]) + np.abs(so[..., 1])
    val = val.transpose(0, 3, 1, 2, 4, 5).reshape(pages, 2, heads, page, dim)
    mag = mag.transpose(0, 3, 1, 2, 4).reshape(pages, 2, heads, page)
    table = rng.permutation(pages)[: batch * per].reshape(batch, per).astype(np.int32)
    return data, table, val, mag


def _reference(q, start, lens, table, val, mag, page, scale, window, sink):
    T, Hq, D = q.shape
    heads = val.shape[2]
    G = Hq // heads
    out, lse = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf)
    es, ev = np.zeros((T, Hq)), np.zeros((T, Hq))
    for b, n in enumerate(lens):
        for i in range(start[b], start[b + 1]):
            m = n - (start[b + 1] - 1 - i)
            j = np.array([t for t in range(max(m, 0)) if t >= m - window or t < sink], int)
            if len(j) == 0:
                continue
            pg, at = table[b][j // page], j % page
            for h in range(heads):
                k, v = val[pg, 0, h, at], val[pg, 1, h, at]
                for g in range(G):
                    x = q[i, h * G + g]
                    s = scale * (k @ x)
                    top = s.max()
                    e = np.exp(s - top)
                    p = e / e.sum()
                    out[i, h * G + g], lse[i, h * G + g] = p @ v, top + np.log(e.sum())
                    es[i, h * G + g] = abs(scale) * np.abs(x).sum() * mag[pg, 0, h, at].max()
                    ev[i, h * G + g] = p @ mag[pg, 1, h, at]
    return out, lse, es, ev


def _run(q, start, lens, data, table, scale, window, sink, info=None):
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV)
    lse = torch.full(q.shape[:2], 9.0, device=DEV)
    ws = torch.full((K().kq_kv_attend_workspace(q, data, table),), 255, dtype=torch.uint8, device=DEV)
    K().kq_kv_attend_window(q, start, lens, data, table, out, ws, scale, window, sink, lse=lse, info=info)
    torch.cuda.synchronize()
    return out, lse


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).to(DEV)


# lens, counts, kv heads, group, dim, page, window, sink
CASES = [([1], [1], 1, 1, 128, 16, 1, 0), ([1, 200], [1, 1], 2, 4, 64, 32, 7, 3), ([300, 17, 0], [1, 1, 0], 2, 8, 128, 64, 40, 4),
         ([300, 17, 0], [1, 1, 2], 1, 5, 64, 16, 33, 20), ([500], [40], 1, 3, 128, 48, 50, 0), ([77, 500, 3], [30, 100, 5], 2, 2, 64, 16, 1, 1),
         ([900, 31], [8, 8], 1, 8, 128, 16, 100, 64), ([640], [1], 1, 16, 64, 256, 256, 32), ([640], [1], 1, 8, 128, 32, 255, 31),
         ([640], [3], 1, 8, 128, 32, 639, 1), ([640], [3], 1, 8, 128, 32, 5000, 2), ([333, 90], [1, 1], 1, 1, 64, 16, 64, 500),
         ([3000, 1500, 2999], [1, 2, 1], 1, 7, 128, 64, 1024, 17), ([40], [90], 1, 4, 64, 16, 12, 2), ([700], [700], 1, 1, 64, 64, 90, 5)]


@pytest.mark.parametrize("lens,counts,heads,group,dim,page,window,sink", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matches_64_bits(lens, counts, heads, group, dim, page, window, sink, dtype):
    rng = np.random.default_rng(sum(lens) + window)
    per = -(-max(max(lens), 1) // page) + 1
    data, table, val, mag = _pool(rng, len(lens), per, heads, dim, page)
    T = sum(counts)
    start = np.concatenate([[0], np.cumsum(counts)])
    wide = torch.from_numpy(rng.standard_normal((T, heads * group + 2, dim))).to(DEV).to(TYPES[dtype])
    q = wide[:, 1:1 + heads * group]
    scale = 1 / np.sqrt(dim)
    want, lse_want, es, ev = _reference(q.double().cpu().numpy(), start, lens, table, val, mag, page, scale, window, sink)
    # pages that no token sees may be gone: their entries in the table are none
    seen = np.zeros((len(lens), per * page), bool)
    for b, n in enumerate(lens):
        for i in range(counts[b]):
            m = n - (counts[b] - 1 - i)
            for j in range(max(m, 0)):
                seen[b, j] |= j >= m - window or j < sink
    gone = table.copy()
    gone[~seen.reshape(len(lens), per, page).any(-1)] = -77
    info = torch.zeros(1, dtype=torch.int32, device=DEV)
    if window < per * page:
        out, lse = _run(q, _i32(start), _i32(lens), torch.from_numpy(data).to(DEV), _i32(gone), scale, window, sink, info)
    else:   # no window: every page is looked up
        out, lse = _run(q, _i32(start), _i32(lens), torch.from_numpy(data).to(DEV), _i32(table), scale, window, sink, info)
    assert K().kq_check(info)[0] == K().KQ_OK
    e = 2.0 ** -18 * es
    tol = ((2 * e + (2.0 ** -18 if dtype == "f32" else 2.0 ** -9)) * ev)[..., None]
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * np.abs(want)
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol + 1e-30), np.max(np.abs(got - want) / (tol + 1e-30))
    got = lse.double().cpu().numpy()
    none = np.isinf(lse_want)
    assert np.array_equal(np.isinf(got), none)
    with np.errstate(invalid="ignore"):
        assert np.all((np.abs(got - lse_want) <= 2 * e + 2.0 ** -20 * (1 + np.abs(lse_want))) | none)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sink", [(9, 0), (40, 3), (64, 33)])
def test_unseen_slots_may_hold_anything(dtype, window, sink):
    """NaN grids in every slot outside the window change no bit."""
    rng = np.random.default_rng(3)
    heads, dim, page, n = 2, 128, 16, 150
    data, table, val, mag = _pool(rng, 1, 10, heads, dim, page)
    q = torch.from_numpy(rng.standard_normal((1, 8, dim))).to(DEV).to(TYPES[dtype])
    start, lens = _i32([0, 1]), _i32([n])
    a = _run(q, start, lens, torch.from_numpy(data).to(DEV), _i32(table), 0.1, window, sink)
    bad = data.copy()
    for j in range(160):
        if (n - window <= j < n) or j < min(sink, n):
            continue
        block = bad[table[0, j // page]]
        for which in range(2):
            at = 16 * dim + (which * 16 + j % 16) * 4
            block[:, at:at + 4] = np.array([0x80, 0x7F, 0xC0, 0x7F], np.uint8)   # scale infinite, offset NaN
    b = _run(q, start, lens, torch.from_numpy(bad).to(DEV), _i32(table), 0.1, window, sink)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # and a NaN inside is seen
    bad[table[0, (n - 1) // page], :, 16 * dim + 64 + (n - 1) % 16 * 4 + 3] = 0x7F
    bad[table[0, (n - 1) // page], :, 16 * dim + 64 + (n - 1) % 16 * 4 + 2] = 0xC0
    assert torch.isnan(_run(q, start, lens, torch.from_numpy(bad).to(DEV), _i32(table), 0.1, window, sink)[0]).all()


def test_a_window_that_holds_everything_is_none():
    rng = np.random.default_rng(4)
    data, table, _, _ = _pool(rng, 2, 9, 2, 64, 32)
    q = torch.from_numpy(rng.standard_normal((6, 6, 64))).to(DEV).float()
    start, lens, data, table = _i32([0, 4, 6]), _i32([270, 33]), torch.from_numpy(data).to(DEV), _i32(table)
    out, lse = torch.empty_like(q), torch.empty(6, 6, device=DEV)
    ws = torch.empty(K().kq_kv_attend_workspace(q, data, table), dtype=torch.uint8, device=DEV)
    K().kq_kv_attend(q, start, lens, data, table, out, ws, 0.2, lse=lse)
    for window in (288, 1 << 40):
        a, b = _run(q, start, lens, data, table, 0.2, window, 0)
        assert torch.equal(a, out) and torch.equal(b, lse)
    a, b = _run(q, start, lens, data, table, 0.2, 1, 1 << 40)   # and so are first slots that do
    assert torch.allclose(a, out, rtol=0, atol=1e-4) and torch.allclose(b, lse, rtol=0, atol=1e-4)


def test_many_sequences_and_a_replayed_graph():
    rng = np.random.default_rng(5)
    batch = 300
    data, table, val, mag = _pool(rng, batch, 4, 1, 64, 32)
    lens, start = rng.integers(0, 129, batch), np.arange(batch + 1)
    q = torch.from_numpy(rng.standard_normal((batch, 4, 64))).to(DEV).float()
    args = (_i32(start), _i32(lens), torch.from_numpy(data).to(DEV), _i32(table))
    want, _, es, ev = _reference(q.double().cpu().numpy(), start, lens, table, val, mag, 32, 0.1, 50, 2)
    ws = torch.empty(K().kq_kv_attend_workspace(q, args[2], args[3]), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K().kq_kv_attend_window(q, args[0], args[1], args[2], args[3], out, ws, 0.1, 50, 2)
    for _ in range(3):
        out.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        got = out.double().cpu().numpy()
        assert np.all(np.abs(got - want) <= ((2 * 2.0 ** -18 * es + 2.0 ** -18) * ev)[..., None] + 1e-30)
    first = out.clone()
    graph.replay()
    assert torch.equal(first, out)


def test_pages_out_of_range_inside_the_window_are_reported():
    rng = np.random.default_rng(6)
    data, table, _, _ = _pool(rng, 1, 8, 1, 64, 16)
    table[0, 7] = 99
    info = torch.zeros(1, dtype=torch.int32, device=DEV)
    q = torch.ones(1, 2, 64, device=DEV)
    _run(q, _i32([0, 1]), _i32([128]), torch.from_numpy(data).to(DEV), _i32(table), 0.1, 4, 0, info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG
