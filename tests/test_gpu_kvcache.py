"""GPU checks of the 4-bit key/value cache against numpy: append is bit for bit, read is exact,
attention is within bounds derived from the formats, eviction is exact.

Bounds of attention. A score is scale (s sum_d q_d c_d + o sum_d q_d): the codes are exact, a
bf16 q is exact, an fp32 q enters to 2^-22, and the sums over d keep 2^-22 of the terms' sum at each of the
up to 16 partial sums, so a score is off by at most e = 2^-18 A with A = |scale| sum |q| max (15 |s| + |o|).
A weight is then off by at most a factor e^(2 e) and its own rounding: 2^-20 with fp32 outputs, 2^-10 with
bf16 ones (fp16 weights). With M = sum_j p_j (15 |s_j| + |o_j|) of the values:
    |out - exact| <= (2 e + 2^-18) M                              fp32
    |out - exact| <= (2 e + 2^-9) M + 2^-8 |exact|                bf16
    |lse - exact| <= 2 e + 2^-20 (1 + |exact|),   |weight - exact| <= sum p (2 e + 2^-18) + 2^-22 |acc|.
"""
import numpy as np
import pytest
import torch

import kv_reference as ref

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


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _starts(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)


def _pool(batch, slots, page, heads, dim, rng, stale=True):
    """(numpy cache, device cache, device table) of random pages in random order; unused bytes are 0xFF (NaN parameters)."""
    per = max(1, -(-slots // page))
    pages = batch * per + 2
    data = np.full((pages, heads, page * (dim + 8)), 0xFF, np.uint8) if stale else np.zeros((pages, heads, page * (dim + 8)), np.uint8)
    table = rng.permutation(pages)[: batch * per].reshape(batch, per).astype(np.int32)
    return ref.Cache(data, table, page, dim)


def _to_dev(cache):
    return torch.from_numpy(cache.data.copy()).to(DEV), torch.from_numpy(cache.table).to(DEV)


def _rounded(x, dtype):
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])


def _fill(cache, lens, heads, rng, gain=1.0):
    for b, n in enumerate(lens):
        for h in range(heads):
            chan = np.exp(0.7 * rng.standard_normal(cache.dim))
            for j in range(n):
                for which in range(2):
                    cache.put(b, h, j, which, (gain * chan * rng.standard_normal(cache.dim)).astype(np.float32))


# ------------------------------------------------------------------------- append, read
@pytest.mark.parametrize("dim,page,heads,dtype,counts,lens", [
    (128, 64, 8, "bf16", [1, 1, 1], [0, 63, 64]), (128, 16, 1, "f32", [5, 0, 40], [3, 7, 15]),
    (64, 48, 3, "bf16", [100, 1], [0, 47]), (64, 256, 2, "f32", [0, 0, 17, 1, 0], [9, 0, 0, 255, 2]),
    (128, 32, 2, "bf16", [0, 0], [4, 0])])
@pytest.mark.parametrize("layout", ["plain", "strided", "shifted"])
def test_append_writes_the_defined_bytes(dim, page, heads, dtype, counts, lens, layout):
    rng = np.random.default_rng(dim + page + len(counts))
    B, T, slots = len(counts), sum(counts), max(np.add(counts, lens)) + 3
    cache = _pool(B, slots, page, heads, dim, rng)
    dc, dt = _to_dev(cache)
    start = _starts(counts)
    k, v = (_rounded(rng.standard_normal((T, heads, dim)) * 3 + 0.3, dtype) for _ in range(2))

    def place(x):
        if layout == "plain":
            return x.to(DEV)
        extra = 8 if layout == "strided" else 3
        wide = torch.zeros(T, heads + 1, dim + extra, dtype=x.dtype, device=DEV)
        wide[:, :heads, extra:] = x.to(DEV)
        return wide[:, :heads, extra:]

    S = slots + 1
    acc = torch.full((B, heads, S), 9.0, device=DEV)
    pos = torch.full((B, heads, S), -5, dtype=torch.int32, device=DEV)
    lens_out, seen_out, info = _i32(np.zeros(B)), _i32(np.zeros(B)), _i32([0])
    seen = np.add(lens, 11)
    K().kq_kv_append(place(k), place(v), _i32(start), _i32(lens), dc, dt, lens_out=lens_out, acc=acc, pos=pos,
                     seen=_i32(seen), seen_out=seen_out, info=info)
    want_acc, want_pos = np.full((B, heads, S), 9.0, np.float32), np.full((B, heads, S), -5, np.int32)
    for b in range(B):
        for i in range(start[b], start[b + 1]):
            j = lens[b] + i - start[b]
            want_acc[b, :, j], want_pos[b, :, j] = 0, seen[b] + i - start[b]
            for h in range(heads):
                cache.put(b, h, j, 0, k[i, h].float().numpy())
                cache.put(b, h, j, 1, v[i, h].float().numpy())
    assert K().kq_check(info)[0] == K().KQ_OK
    assert np.array_equal(dc.cpu().numpy(), cache.data)
    assert np.array_equal(acc.cpu().numpy(), want_acc) and np.array_equal(pos.cpu().numpy(), want_pos)
    assert np.array_equal(lens_out.cpu().numpy(), np.add(lens, counts))
    assert np.array_equal(seen_out.cpu().numpy(), np.add(seen, counts))
    # read back: exactly scale * code + offset in the asked type, zeros past the length
    first = [max(0, n - 2) for n in lens]
    many = [c + 2 + 3 for c in counts]
    for name in ("bf16", "f32"):
        ko, vo = (torch.full((sum(many), heads, dim), 7.0, dtype=TYPES[name], device=DEV) for _ in range(2))
        K().kq_kv_read(dc, dt, _i32(_starts(many)), _i32(first), lens_out, ko, vo, info=info)
        assert K().kq_check(info)[0] == K().KQ_OK
        for which, got in enumerate((ko, vo)):
            got = got.cpu()
            for b in range(B):
                n = lens[b] + counts[b]
                for h in range(heads):
                    vals = cache.rows(b, h, n, which)[0]
                    w = np.zeros((many[b], dim))
                    w[:max(0, min(many[b], n - first[b]))] = vals[first[b]:first[b] + many[b]]
                    at = _starts(many)[b]
                    assert torch.equal(torch.nan_to_num(got[at:at + many[b], h].float(), nan=77.0),
                                       torch.nan_to_num(_rounded(w, name).float(), nan=77.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_rows_at_the_edges_of_the_grid(dtype):
    dim = 128
    rows = np.zeros((12, dim), np.float32)
    rows[1] = 0.7109375                         # constant, held by bf16: scale 0
    rows[2] = 1.001                             # constant, not held by bf16 in fp32
    rows[3, 5] = np.nan
    rows[4, 9] = np.inf
    rows[5, 9] = -np.inf
    rows[6] = np.linspace(-3e38, 3e38, dim)     # the range overflows
    rows[7] = np.linspace(0, 1e-40, dim)        # subnormal
    rows[8] = np.linspace(100, 101, dim)
    rows[9, ::2] = -0.0
    rows[10] = np.arange(dim) % 16              # every code, exactly
    rows[11] = (np.arange(dim) % 31) / 2        # ties
    x = _rounded(rows, dtype)[:, None]
    rng = np.random.default_rng(0)
    cache = _pool(1, 16, 16, 1, dim, rng)
    dc, dt = _to_dev(cache)
    K().kq_kv_append(x.to(DEV), x.to(DEV), _i32([0, 12]), _i32([0]), dc, dt)
    for j in range(12):
        for which in range(2):
            cache.put(0, 0, j, which, x[j, 0].float().numpy())
    assert np.array_equal(dc.cpu().numpy(), cache.data)
    got = cache.rows(0, 0, 12, 0)[0]
    fine = [0, 1, 2, 8, 9, 10, 11]
    step = np.array([quant[0] for quant in ref.quantize(x[:, 0].float().numpy())[1]])
    assert np.all(np.abs(got - x[:, 0].double().numpy())[fine] <= 0.5001 * step[fine, None])
    assert np.array_equal(got[10], rows[10]) and np.isnan(got[3:7]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [-126, -110, -70, -66, -30, 0, 40, 63, 67, 100, 120])
def test_append_codes_near_ties_at_every_scale(dtype, power):
    """Quotients on ties, a float to either side of them and anywhere, from the smallest scales to the largest: the
    bytes are those of the defining operations."""
    dim, n = 128, 96
    rng = np.random.default_rng(power + 200)
    x = np.zeros((n, dim), np.float32)
    for i in range(n):
        m = 1 if i % 3 == 0 else rng.integers(128, 256) / 128     # of the scale: 8 bits, or a power of two
        codes = rng.integers(0, 31, dim) / 2
        codes[:2] = 0, 15
        row = (codes * m * 2.0**power).astype(np.float32)
        side = np.where(rng.random(dim) < 0.5, np.float32(np.inf), np.float32(0))
        near = np.nextafter(row, side).astype(np.float32)
        far = (rng.random(dim) * 15 * m * 2.0**power).astype(np.float32)
        x[i] = np.where(codes == 15, row, np.choose(rng.integers(0, 3, dim), [row, near, far]))
        x[i, :2] = 0, row[1]
        if i % 4 == 1:   # an offset of about the range: values lose bits to it
            x[i] += np.float32(-7.37 * 2.0**power)
    x = _rounded(x, dtype)[:, None]
    cache = _pool(1, n, 16, 1, dim, rng)
    dc, dt = _to_dev(cache)
    K().kq_kv_append(x.to(DEV), x.to(DEV), _i32([0, n]), _i32([0]), dc, dt)
    for j in range(n):
        for which in range(2):
            cache.put(0, 0, j, which, x[j, 0].float().numpy())
    assert np.array_equal(dc.cpu().numpy(), cache.data)


def test_append_and_read_record_what_has_no_slot():
    rng = np.random.default_rng(1)
    cache = _pool(2, 32, 16, 2, 64, rng)
    dc, dt = _to_dev(cache)
    before = dc.clone()
    x = torch.randn(4, 2, 64, device=DEV)
    out, info = _i32([0, 0]), _i32([0])
    K().kq_kv_append(x, x, _i32([0, 2, 4]), _i32([31, 0]), dc, dt, lens_out=out, info=info)   # the second token of 0 has none
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG
    assert out.tolist() == [32, 2]
    for i, (b, j) in enumerate([(0, 31), (None, 0), (1, 0), (1, 1)]):
        if b is not None:
            for h in range(2):
                for which in range(2):
                    cache.put(b, h, j, which, x[i, h].cpu().numpy())
    assert np.array_equal(dc.cpu().numpy(), cache.data)
    dc.copy_(before)
    bad = dt.clone()
    bad[1, 0], bad[0, 0] = 99, -1
    K().kq_kv_append(x, x, _i32([0, 2, 4]), _i32([0, 0]), dc, bad, info=info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG and torch.equal(dc, before)
    K().kq_kv_append(x, x, _i32([0, 2, 3]), _i32([0, 0]), dc, dt, info=info)   # the fourth token is nobody's
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG
    ko, vo = torch.ones(4, 2, 64, device=DEV), torch.ones(4, 2, 64, device=DEV)
    K().kq_kv_read(dc, bad, _i32([0, 2, 4]), None, None, ko, vo, info=info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG and not ko.any() and not vo.any()


# ------------------------------------------------------------------------------ attention
def _run_attend(cache, q, counts, lens, heads, scale, track, dtype, acc0=None, S=None, want_lse=True):
    B, T, Hq = len(counts), q.shape[0], q.shape[1]
    dc, dt = _to_dev(cache)
    S = S or int(cache.table.shape[1] * cache.page)
    acc = None
    if track:
        acc = torch.from_numpy(acc0).to(DEV)
    out = torch.full((T, Hq, cache.dim), 5.0, dtype=TYPES[dtype], device=DEV)
    lse = torch.full((T, Hq), 5.0, device=DEV) if want_lse else None
    info = _i32([0])
    ws = torch.full((max(256, K().kq_kv_attend_workspace(q, dc, dt, acc)),), 0xFF, dtype=torch.uint8, device=DEV)
    K().kq_kv_attend(q, _i32(_starts(counts)), _i32(lens), dc, dt, out, ws, scale, lse=lse, acc=acc, info=info)
    assert K().kq_check(info)[0] == K().KQ_OK
    return out, lse, acc


def _check_attend(cache, q, counts, lens, heads, scale, dtype, out, lse, acc, acc0):
    o, l, w, es, ev, werr = ref.attend(cache, q.cpu().float().numpy(), _starts(counts), lens, heads, scale)
    e = 2.0 ** -18 * es
    tol = (2 * e + (2.0 ** -18 if dtype == "f32" else 2.0 ** -9)) * ev
    tol = tol[..., None] + (2.0 ** -8 * np.abs(o) if dtype == "bf16" else 0)
    got = out.float().cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - o) <= tol + 1e-30), np.max(np.abs(got - o) / (tol + 1e-30))
    if lse is not None:
        g = lse.cpu().numpy().astype(np.float64)
        empty = np.isinf(l)
        assert np.array_equal(np.isinf(g), empty) and np.all(g[empty] < 0)
        assert np.all(np.abs(g - l)[~empty] <= (2 * e + 2.0 ** -20 * (1 + np.abs(l)))[~empty])
    if acc is not None:
        S = acc0.shape[-1]
        w, werr = w[..., :S], werr[..., :S]
        got = acc.cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - acc0 - w) <= 2.0 ** -17 * werr + 2.0 ** -18 * w + 2.0 ** -22 * np.abs(acc0 + w) + 1e-30)


CASES = [
    # dim, page, kv heads, group, lens, queries a sequence
    (128, 64, 2, 4, [1, 17, 130], [1, 1, 1]),
    (128, 16, 1, 8, [0, 1, 15, 16, 33], [1, 1, 1, 1, 1]),
    (64, 48, 3, 1, [97, 200], [1, 1]),
    (64, 16, 2, 7, [63, 64, 65], [3, 1, 2]),
    (128, 128, 1, 16, [257], [1]),
    (128, 32, 2, 5, [2, 40, 0, 300], [4, 3, 2, 5]),     # more queries than slots: empty rows
    (64, 64, 1, 4, [500, 3], [9, 0]),                   # a sequence without queries
    (128, 256, 1, 2, [1000], [40]),                     # many rows for one head
]


@pytest.mark.parametrize("dim,page,heads,group,lens,counts", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("track", [False, True])
def test_attend_matches_64_bits(dim, page, heads, group, lens, counts, dtype, track):
    rng = np.random.default_rng(dim + page + sum(lens))
    cache = _pool(len(lens), max(lens) + 5, page, heads, dim, rng)
    _fill(cache, lens, heads, rng)
    T = sum(counts)
    q = _rounded(rng.standard_normal((T, heads * group, dim)) * 1.5, dtype)
    wide = torch.zeros(T, heads * group + 2, dim, dtype=q.dtype, device=DEV)
    wide[:, 1:-1] = q.to(DEV)
    scale = 1 / np.sqrt(dim)
    S = max(lens) + 1
    acc0 = rng.random((len(lens), heads, S)).astype(np.float32)
    out, lse, acc = _run_attend(cache, wide[:, 1:-1], counts, lens, heads, scale, track, dtype, acc0, S)
    _check_attend(cache, q, counts, lens, heads, scale, dtype, out, lse, acc, acc0)


@pytest.mark.parametrize("dim,heads,group,n,counts", [(128, 1, 8, 6000, 1), (64, 1, 3, 5011, 2), (128, 2, 12, 3100, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_splits_few_rows_over_many_warps(dim, heads, group, n, counts, dtype):
    """Long sequences of few heads: a row's result is joined from more parts than a warp has lanes."""
    rng = np.random.default_rng(n)
    cache = _pool(1, n, 64, heads, dim, rng)
    _fill(cache, [n], heads, rng)
    q = _rounded(rng.standard_normal((counts, heads * group, dim)) * 2, dtype)
    acc0 = np.zeros((1, heads, n), np.float32)
    out, lse, acc = _run_attend(cache, q.to(DEV), [counts], [n], heads, 1 / np.sqrt(dim), True, dtype, acc0, n)
    _check_attend(cache, q, [counts], [n], heads, 1 / np.sqrt(dim), dtype, out, lse, acc, acc0)


@pytest.mark.parametrize("batch", [129, 400])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_short_sequences(batch, dtype):
    """More sequences than a block has threads, some without tokens and some without queries: append, read, attend."""
    rng = np.random.default_rng(batch)
    dim, heads, group = 64, 2, 3
    lens = rng.integers(0, 40, batch)
    counts = rng.integers(0, 3, batch)
    lens = np.maximum(lens, counts)
    lens[5] = 0
    cache = _pool(batch, 40, 16, heads, dim, rng)
    dc, dt = _to_dev(cache)
    T = int(lens.sum())
    k, v = (_rounded(rng.standard_normal((T, heads, dim)), dtype) for _ in range(2))
    at = _starts(lens)
    K().kq_kv_append(k.to(DEV), v.to(DEV), _i32(at), _i32(np.zeros(batch)), dc, dt)
    for b in range(batch):
        for j in range(lens[b]):
            for h in range(heads):
                cache.put(b, h, j, 0, k[at[b] + j, h].float().numpy())
                cache.put(b, h, j, 1, v[at[b] + j, h].float().numpy())
    assert np.array_equal(dc.cpu().numpy(), cache.data)
    ko, vo = torch.empty(T, heads, dim, device=DEV), torch.empty(T, heads, dim, device=DEV)
    K().kq_kv_read(dc, dt, _i32(at), None, _i32(lens), ko, vo)
    want = np.concatenate([cache.rows(b, 1, lens[b], 1)[0] for b in range(batch)])
    assert np.array_equal(vo[:, 1].cpu().numpy().astype(np.float64), want)
    q = _rounded(rng.standard_normal((int(counts.sum()), heads * group, dim)), dtype)
    acc0 = rng.random((batch, heads, 40)).astype(np.float32)
    lens, counts = lens.tolist(), counts.tolist()
    out, lse, acc = _run_attend(cache, q.to(DEV), counts, lens, heads, 0.2, True, dtype, acc0, 40)
    _check_attend(cache, q, counts, lens, heads, 0.2, dtype, out, lse, acc, acc0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_of_unaligned_and_strided_queries(dtype):
    rng = np.random.default_rng(3)
    cache = _pool(1, 70, 16, 1, 64, rng)
    _fill(cache, [70], 1, rng)
    q = _rounded(rng.standard_normal((3, 2, 64)), dtype)
    wide = torch.zeros(3, 5, 67, dtype=q.dtype, device=DEV)
    wide[:, 1::2][:, :2, 1:65] = q.to(DEV)
    out, lse, _ = _run_attend(cache, wide[:, 1::2][:, :2, 1:65], [3], [70], 1, 0.125, False, dtype)
    _check_attend(cache, q, [3], [70], 1, 0.125, dtype, out, lse, None, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("track", [False, True])
def test_attend_over_extreme_values(dtype, track):
    """Scores of thousands (one slot takes all), values whose scale spans ten decades, a sink whose value is
    tiny, an all-zero query, rows of zeros."""
    rng = np.random.default_rng(4)
    dim, n = 128, 150
    cache = _pool(1, n, 64, 1, dim, rng)
    for j in range(n):
        cache.put(0, 0, j, 0, (rng.standard_normal(dim) * (100 if j % 7 == 0 else 0.1)).astype(np.float32))
        cache.put(0, 0, j, 1, (rng.standard_normal(dim) * 10.0 ** ((j % 11) - 6)).astype(np.float32))
    cache.put(0, 0, 0, 0, np.full(dim, 5.0, np.float32))
    cache.put(0, 0, 0, 1, (rng.standard_normal(dim) * 1e-7).astype(np.float32))
    cache.put(0, 0, 40, 0, np.zeros(dim, np.float32))
    cache.put(0, 0, 41, 1, np.zeros(dim, np.float32))
    q = rng.standard_normal((1, 4, dim))
    q[0, 0] *= 40
    q[0, 1] = 0
    q[0, 2] = 1.0
    q[0, 3] *= 1e-4
    q = _rounded(q, dtype)
    acc0 = np.zeros((1, 1, n), np.float32)
    out, lse, acc = _run_attend(cache, q.to(DEV), [1], [n], 1, 0.25, track, dtype, acc0, n)
    _check_attend(cache, q, [1], [n], 1, 0.25, dtype, out, lse, acc, acc0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_nan_reaches_only_those_who_see_it(dtype):
    rng = np.random.default_rng(5)
    dim, lens, counts = 128, [40, 40, 70], [1, 3, 1]
    cache = _pool(3, 70, 16, 2, dim, rng)
    _fill(cache, lens, 2, rng)
    bad = np.full(dim, np.nan, np.float32)
    cache.put(0, 0, 7, 0, bad)      # a key of sequence 0, head 0
    cache.put(1, 1, 39, 1, bad)     # the last value of sequence 1, head 1: only the last query sees it
    q = _rounded(rng.standard_normal((5, 4, dim)), dtype)
    out, lse, _ = _run_attend(cache, q.to(DEV), counts, lens, 2, 0.1, False, dtype)
    nan = torch.isnan(out).all(-1).cpu()
    assert torch.equal(nan, torch.isnan(out).any(-1).cpu())
    want = torch.zeros(5, 4, dtype=torch.bool)
    want[0, :2] = True
    want[3, 2:] = True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_nonfinite_query_touches_its_own_row_only(value, dtype):
    rng = np.random.default_rng(6)
    cache = _pool(1, 90, 32, 1, 64, rng)
    _fill(cache, [90], 1, rng)
    q = _rounded(rng.standard_normal((2, 8, 64)), dtype)
    clean, _, _ = _run_attend(cache, q.to(DEV), [2], [90], 1, 0.1, False, dtype)
    dirty = q.clone()
    dirty[1, 3, 5] = value
    out, _, _ = _run_attend(cache, dirty.to(DEV), [2], [90], 1, 0.1, False, dtype)
    assert torch.isnan(out[1, 3]).all()
    keep = torch.ones(2, 8, dtype=torch.bool)
    keep[1, 3] = False
    assert torch.equal(out.cpu()[keep], clean.cpu()[keep])


def test_attend_is_deterministic_and_runs_on_its_stream_and_in_graphs():
    rng = np.random.default_rng(7)
    dim, lens, counts = 128, [700, 30, 411], [1, 1, 1]
    cache = _pool(3, 700, 64, 2, dim, rng)
    _fill(cache, lens, 2, rng)
    dc, dt = _to_dev(cache)
    q = torch.from_numpy(rng.standard_normal((3, 16, dim)).astype(np.float32)).to(DEV).to(torch.bfloat16)
    start, ln = _i32([0, 1, 2, 3]), _i32(lens)
    acc = torch.zeros(3, 2, 700, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(3, 16, device=DEV)
    ws = torch.empty(K().kq_kv_attend_workspace(q, dc, dt, acc), dtype=torch.uint8, device=DEV)

    def step(stream=None):
        K().kq_kv_attend(q, start, ln, dc, dt, out, ws, 0.1, lse=lse, acc=acc, stream=stream)

    step()
    torch.cuda.synchronize()
    first = (out.clone(), lse.clone(), acc.clone())
    for _ in range(3):
        acc.zero_()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (out, lse, acc)))
    side = torch.cuda.Stream()
    acc.zero_(), out.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (out, lse, acc)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step(side)
    acc.zero_(), out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (out, lse, acc)))


def test_attend_and_append_beyond_four_gibibytes():
    """Pages past the 2^32nd byte of a pool: append, attend, evict and read address them in 64 bits."""
    rng = np.random.default_rng(8)
    dim, page, heads, n = 128, 64, 8, 200
    per = (1 << 32) // (heads * page * (dim + 8)) + 8
    small = _pool(1, n, page, heads, dim, rng)
    dc = torch.empty(per, heads, page * (dim + 8), dtype=torch.uint8, device=DEV)
    order = np.array([[per - 1, per - 3, per - 2, per - 5]], np.int32)
    x = [torch.from_numpy(rng.standard_normal((n, heads, dim)).astype(np.float32)).to(DEV) for _ in range(2)]
    q = torch.from_numpy(rng.standard_normal((1, heads, dim)).astype(np.float32)).to(DEV)
    got = []
    for c, t in ((dc, torch.from_numpy(order).to(DEV)), _to_dev(small)):
        K().kq_kv_append(x[0], x[1], _i32([0, n]), _i32([0]), c, t)
        acc, pos = torch.rand(1, heads, n, generator=torch.Generator(DEV).manual_seed(1), device=DEV), torch.arange(
            n, dtype=torch.int32, device=DEV).expand(1, heads, n).contiguous()
        out = torch.empty_like(q)
        ws = torch.empty(K().kq_kv_attend_workspace(q, c, t, acc) + 256, dtype=torch.uint8, device=DEV)
        K().kq_kv_attend(q, _i32([0, 1]), _i32([n]), c, t, out, ws, 0.1, acc=acc)
        ln = _i32([0])
        ew = torch.empty(K().kq_kv_evict_workspace(acc, 70), dtype=torch.uint8, device=DEV)
        K().kq_kv_evict(c, t, _i32([n]), acc, pos, _i32([n]), dim, 70, 10, 2, ln, acc, pos, ew)
        k, v = torch.empty(70, heads, dim, device=DEV), torch.empty(70, heads, dim, device=DEV)
        K().kq_kv_read(c, t, _i32([0, 70]), None, ln, k, v)
        got.append((out, acc, pos, k, v))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_attend_records_bad_lengths_pages_and_tokens():
    rng = np.random.default_rng(9)
    cache = _pool(2, 32, 16, 1, 64, rng)
    _fill(cache, [20, 32], 1, rng)
    dc, dt = _to_dev(cache)
    q = torch.randn(2, 2, 64, device=DEV)
    out, info = torch.zeros_like(q), _i32([0])
    ws = torch.empty(K().kq_kv_attend_workspace(q, dc, dt, torch.empty(2, 1, 32)), dtype=torch.uint8, device=DEV)

    def status(start, lens, table, acc=None):
        K().kq_kv_attend(q, _i32(start), _i32(lens), dc, table, out, ws, 0.1, acc=acc, info=info)
        return K().kq_check(info)[0]

    assert status([0, 1, 2], [20, 32], dt) == K().KQ_OK
    good = out.clone()
    bad = dt.clone()
    bad[0, 0] = 1 << 20
    for start, lens, table, acc in (([0, 1, 2], [20, 33], dt, None), ([0, 1, 2], [-1, 32], dt, None),
                                    ([0, 1, 2], [20, 32], bad, None), ([0, 1, 1], [20, 32], dt, None),
                                    ([0, 1, 3], [20, 32], dt, None), ([0, 2, 1], [20, 32], dt, None),
                                    ([0, 1, 2], [20, 32], dt, torch.zeros(2, 1, 31, device=DEV))):
        assert status(start, lens, table, acc) == K().KQ_ERR_INVALID_ARG, (start, lens)
    assert status([0, 1, 2], [20, 32], dt) == K().KQ_OK and torch.equal(out, good)


def test_attend_of_overlapping_sequences_stays_in_its_workspace():
    """start goes back and forth: more rows than tokens, reported, with nothing written past the workspace or out."""
    rng = np.random.default_rng(10)
    batch, T = 64, 9
    cache = _pool(batch, 16, 16, 1, 64, rng)
    _fill(cache, [16] * batch, 1, rng)
    dc, dt = _to_dev(cache)
    q = torch.randn(T, 1, 64, device=DEV)
    out = torch.full((T + 64, 1, 64), 3.0, device=DEV)
    need = K().kq_kv_attend_workspace(q, dc, dt, None)
    ws = torch.full((need + 65536,), 0xAB, dtype=torch.uint8, device=DEV)
    info = _i32([0])
    start = _i32([0, T] * (batch // 2) + [0])
    K().kq_kv_attend(q, start, _i32([16] * batch), dc, dt, out[:T], ws[:need], 0.1, info=info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG
    assert (ws[need:] == 0xAB).all() and (out[T:] == 3.0).all()


# ------------------------------------------------------------------------------- eviction
@pytest.mark.parametrize("dim,page,heads,lens,budget,recent,sink,kind", [
    (128, 64, 2, [300, 90, 0], 100, 10, 4, "random"), (64, 16, 1, [1000], 999, 0, 0, "random"),
    (64, 32, 3, [257, 256], 1, 0, 1, "random"), (128, 16, 1, [500], 200, 200, 0, "random"),
    (64, 48, 2, [3000], 1500, 100, 3, "ties"), (64, 16, 1, [700], 64, 20, 2, "flat"),
    (128, 64, 1, [400], 100, 40, 4, "odd"), (64, 16, 1, [200], 50, 50, 0, "crowd"),
    (64, 128, 1, [40000], 20011, 100, 4, "ties"), (64, 16, 2, [90], 200, 100, 4, "random"),
    (64, 1024, 1, [420001], 900, 100, 4, "ties"), (128, 64, 1, [4096, 4097, 9000], 4095, 64, 4, "random")])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_keeps_and_moves_the_right_slots(dim, page, heads, lens, budget, recent, sink, kind, in_place):
    rng = np.random.default_rng(len(kind) + budget)
    B, S = len(lens), max(lens) + 2
    cache = _pool(B, S, page, heads, dim, rng)
    cache.data[:] = rng.integers(0, 256, cache.data.shape, dtype=np.uint8)
    acc = rng.random((B, heads, S)).astype(np.float32)
    if kind == "ties":
        acc = (acc * 8).round() / 8
    if kind == "flat":
        acc[:] = 0.25
    if kind == "odd":
        acc[..., ::5] = np.nan
        acc[..., 1::5] = np.inf
        acc[..., 2::5] = -1.0
        acc[..., 3::5] = 0.0
        acc[..., 4::10] = -0.0
    seen = np.array([n + 50 for n in lens])
    pos = np.stack([np.stack([rng.permutation(S) + 50 - (S - max(n, 1)) for _ in range(heads)]) for n in lens])
    if kind == "crowd":
        pos[:] = seen[0] - 1
    pos = pos.astype(np.int32)
    dc, dt = _to_dev(cache)
    da, dp = torch.from_numpy(acc).to(DEV), torch.from_numpy(pos).to(DEV)
    oa, op = (da, dp) if in_place else (torch.full_like(da, -3.0), torch.full_like(dp, -3))
    want_a, want_p = oa.cpu().numpy().copy(), op.cpu().numpy().copy()
    lo, info = _i32(np.zeros(B)), _i32([0])
    ws = torch.full((max(1, K().kq_kv_evict_workspace(da, budget)),), 0xFF, dtype=torch.uint8, device=DEV)
    K().kq_kv_evict(dc, dt, _i32(lens), da, dp, _i32(seen), dim, budget, recent, sink, lo, oa, op, ws, info=info)
    assert K().kq_check(info)[0] == K().KQ_OK
    assert lo.tolist() == [min(n, budget) for n in lens]
    for b, n in enumerate(lens):
        for h in range(heads):
            src = ref.evict(acc[b, h], pos[b, h], n, seen[b], budget, recent, sink)
            want_a[b, h, :len(src)], want_p[b, h, :len(src)] = acc[b, h, src], pos[b, h, src]
            for d, s in enumerate(src):
                if d != s:
                    cache.move(b, h, s, d)
    assert np.array_equal(oa.cpu().numpy(), want_a, equal_nan=True) and np.array_equal(op.cpu().numpy(), want_p)
    assert np.array_equal(dc.cpu().numpy(), cache.data)


def test_evict_records_bad_lengths_and_pages():
    rng = np.random.default_rng(2)
    cache = _pool(1, 64, 16, 1, 64, rng)
    dc, dt = _to_dev(cache)
    acc, pos = torch.rand(1, 1, 64, device=DEV), torch.arange(64, dtype=torch.int32, device=DEV).view(1, 1, 64)
    lo, info, ws = _i32([0]), _i32([0]), torch.empty(4096, dtype=torch.uint8, device=DEV)
    before = dc.clone()
    K().kq_kv_evict(dc, torch.full_like(dt, 1 << 30), _i32([64]), acc, pos, _i32([64]), 64, 32, 0, 0, lo, acc.clone(),
                    pos.clone(), ws, info=info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG and torch.equal(dc, before)
    K().kq_kv_evict(dc, dt, _i32([65]), acc, pos, _i32([64]), 64, 64, 0, 0, lo, acc, pos, ws, info=info)
    assert K().kq_check(info)[0] == K().KQ_ERR_INVALID_ARG and lo.tolist() == [64]


# ------------------------------------------------------------------------------ refusals
def test_binding_refuses_what_does_not_fit():
    kq = K()
    cache = torch.zeros(4, 2, 16 * 72, dtype=torch.uint8, device=DEV)
    table = torch.zeros(1, 4, dtype=torch.int32, device=DEV)
    start, lens = _i32([0, 1]), _i32([0])
    k = torch.zeros(1, 2, 64, device=DEV)
    with pytest.raises(ValueError, match="heads"):
        kq.kq_kv_append(torch.zeros(1, 3, 64, device=DEV), k, start, lens, cache, table)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        kq.kq_kv_append(k.half(), k.half(), start, lens, cache, table)
    with pytest.raises(ValueError, match="shape"):
        kq.kq_kv_append(k, k, _i32([0, 1, 1]), lens, cache, table)
    with pytest.raises(ValueError, match="one shape"):
        kq.kq_kv_append(k, k.bfloat16(), start, lens, cache, table)
    with pytest.raises(ValueError, match="last dimension"):
        kq.kq_kv_append(k, k, start, lens, torch.zeros(4, 2, 1000, dtype=torch.uint8, device=DEV), table)
    with pytest.raises(kq.KronqError, match="KQ_ERR_INVALID_ARG"):
        kq.kq_kv_append(k, k, start, lens, cache, table, lens_out=lens)
    q, out = torch.zeros(1, 4, 64, device=DEV), torch.zeros(1, 4, 64, device=DEV)
    ws = torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError, match="out must"):
        kq.kq_kv_attend(q, start, lens, cache, table, out.bfloat16(), ws, 1.0)
    with pytest.raises(kq.KronqError, match="multiple of kv_heads"):
        kq.kq_kv_attend(q[:, :3], start, lens, cache, table, out[:, :3].contiguous(), ws, 1.0)
    with pytest.raises(kq.KronqError, match="WORKSPACE"):
        kq.kq_kv_attend(q, start, lens, cache, table, out, ws[:4], 1.0, acc=torch.zeros(1, 2, 64, device=DEV))
    with pytest.raises(kq.KronqError, match="scale finite"):
        kq.kq_kv_attend(q, start, lens, cache, table, out, ws, float("inf"))
    with pytest.raises(ValueError, match="unit stride"):
        kq.kq_kv_attend(torch.zeros(1, 64, 4, device=DEV).transpose(1, 2), start, lens, cache, table, out, ws, 1.0)
    acc, pos = torch.zeros(1, 2, 64, device=DEV), torch.zeros(1, 2, 64, dtype=torch.int32, device=DEV)
    with pytest.raises(kq.KronqError, match="recent"):
        kq.kq_kv_evict(cache, table, lens, acc, pos, lens, 64, 8, 7, 2, _i32([0]), acc, pos, ws)
    with pytest.raises(kq.KronqError, match="WORKSPACE"):
        kq.kq_kv_evict(cache, table, lens, acc, pos, lens, 64, 8, 7, 1, _i32([0]), acc, pos, ws[:16])
    torch.cuda.synchronize()
