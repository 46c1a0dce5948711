"""Host-side checks of the decoding and scoring entry points (no GPU): arguments are refused before any
CUDA call, workspace queries, and the numpy quantizer that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest

import kv_reference as ref


@pytest.fixture(scope="module")
def K():
    from paper_2607_07964_gb300 import build, kronq
    build.build()
    kronq.lib()
    return kronq


P = ctypes.c_void_p
FAKE = P(256)   # never dereferenced: validation fails first


def _cache(K, **over):
    f = dict(data=256, table=256, pages=4, page=64, kv_heads=2, dim=128, batch=1, table_ld=2)
    f.update(over)
    return ctypes.byref(K._KvCache(*f.values()))


@pytest.mark.parametrize("over,status", [
    ({"dim": 96}, 2), ({"page": 8}, 1), ({"page": 24}, 1), ({"page": 2048}, 1), ({"pages": 0}, 1), ({"kv_heads": 0}, 1),
    ({"batch": 0}, 1), ({"batch": 70000}, 1), ({"table_ld": 0}, 1), ({"table_ld": 1 << 30}, 1), ({"data": 264}, 1),
    ({"data": None}, 1), ({"table": None}, 1)])
def test_cache_descriptions_are_checked_by_every_call(K, over, status):
    c, lib = _cache(K, **over), K.lib()
    assert lib.kq_kv_append(c, FAKE, FAKE, 0, 1, 256, 128, 256, 128, FAKE, FAKE, None, None, None, 0, None, None, None,
                            None) == status
    assert lib.kq_kv_read(c, FAKE, None, None, 0, 1, FAKE, FAKE, None, None) == status
    assert lib.kq_kv_attend(c, FAKE, 0, 1, 4, 512, 128, FAKE, FAKE, 1.0, FAKE, None, None, 0, None, FAKE, 1 << 30,
                            None) == status
    assert lib.kq_kv_evict(c, FAKE, FAKE, FAKE, FAKE, 64, 8, 0, 0, P(512), FAKE, FAKE, None, FAKE, 1 << 30, None) == status


def test_arguments_are_refused_on_the_host(K):
    lib, c = K.lib(), _cache(K)
    assert lib.kq_kv_append(None, FAKE, FAKE, 0, 1, 256, 128, 256, 128, FAKE, FAKE, None, None, None, 0, None, None, None,
                            None) == K.KQ_ERR_INVALID_ARG
    assert lib.kq_kv_append(c, FAKE, FAKE, 7, 1, 256, 128, 256, 128, FAKE, FAKE, None, None, None, 0, None, None, None,
                            None) == K.KQ_ERR_UNSUPPORTED
    assert lib.kq_kv_append(c, FAKE, None, 0, 1, 256, 128, 256, 128, FAKE, FAKE, None, None, None, 0, None, None, None,
                            None) == K.KQ_ERR_INVALID_ARG
    assert lib.kq_kv_append(c, P(257), FAKE, 0, 1, 256, 128, 256, 128, FAKE, FAKE, None, None, None, 0, None, None, None,
                            None) == K.KQ_ERR_INVALID_ARG
    assert lib.kq_kv_append(c, FAKE, FAKE, 0, 1, 256, 128, 256, 128, FAKE, FAKE, None, FAKE, None, 0, None, None, None,
                            None) == K.KQ_ERR_INVALID_ARG     # acc without S
    assert lib.kq_kv_read(c, FAKE, None, None, 0, 1, P(264), FAKE, None, None) == K.KQ_ERR_INVALID_ARG
    att = [c, FAKE, 0, 1, 4, 512, 128, FAKE, FAKE, 1.0, FAKE, None, FAKE, 64, None, FAKE, 1 << 30, None]
    for at, value, status in ((4, 3, 1), (9, float("nan"), 1), (13, 0, 1), (15, None, 6), (16, 8, 6), (15, P(264), 6),
                              (2, 2, 2), (1, None, 1), (3, -1, 1)):
        args = list(att)
        args[at] = value
        assert lib.kq_kv_attend(*args) == status, (at, value)
    ev = [c, FAKE, FAKE, FAKE, FAKE, 64, 8, 4, 2, P(512), FAKE, FAKE, None, FAKE, 1 << 20, None]
    for at, value, status in ((6, 0, 1), (7, 7, 1), (8, -1, 1), (9, FAKE, 1), (2, None, 1), (14, 4, 6), (13, P(260), 6)):
        args = list(ev)
        args[at] = value
        assert lib.kq_kv_evict(*args) == status, (at, value)
    lp = [FAKE, 0, 2, 100, 100, FAKE, 5, FAKE, None, None, FAKE, FAKE, None, None]
    for at, value, status in ((1, 3, 2), (3, (1 << 20) + 1, 2), (4, 99, 1), (6, 33, 1), (6, -1, 1), (10, None, 1), (5, None, 1),
                              (0, P(257), 1), (2, -1, 1), (3, 0, 1)):
        args = list(lp)
        args[at] = value
        assert lib.kq_token_logprobs(*args) == status, (at, value)
    gr = [FAKE, 0, 2, 100, 100, FAKE, FAKE, None, FAKE, None, P(1 << 20), 100, None, None]
    for at, value, status in ((9, FAKE, 1), (11, 99, 1), (10, None, 1), (6, None, 1), (10, P(257), 1)):
        args = list(gr)
        args[at] = value
        assert lib.kq_token_logprobs_grad(*args) == status, (at, value)


def test_workspace_queries(K):
    lib = K.lib()
    assert lib.kq_kv_attend_workspace(0, 8, 2, 128, 0) == 0 and lib.kq_kv_attend_workspace(1, 7, 2, 128, 0) == 0
    assert lib.kq_kv_attend_workspace(3, 8, 2, 128, 1000) >= 3 * 8 * 1000 * 4
    assert lib.kq_kv_evict_workspace(2, 3, 100, 40) >= 2 * 3 * 40 * 4


def test_numpy_quantizer_bounds_its_error_and_never_clamps():
    rng = np.random.default_rng(0)
    for x in (rng.standard_normal((200, 128)), rng.random((50, 64)) + 100, 1e-30 * rng.standard_normal((20, 64)),
              1e30 * rng.standard_normal((20, 128))):
        x = x.astype(np.float32)
        c, so = ref.quantize(x)
        s, o = so[..., :1].astype(np.float64), so[..., 1:].astype(np.float64)
        assert np.all(np.abs(c * s + o - x) <= 0.50001 * s)
        assert np.all(o <= x.min(-1, keepdims=True)) and np.all(o + 15 * s >= x.max(-1, keepdims=True))


def test_numpy_eviction_by_hand():
    acc = np.array([.5, .1, .1, .9, .2, .1], np.float32)
    pos = np.arange(6)
    assert ref.evict(acc, pos, 6, 6, 4, 1, 1) == [0, 4, 5, 3]       # 0 (sink), 5 (recent), .9, .2: slots 4 and 5 move into 1 and 2
    assert ref.evict(acc, pos, 6, 6, 3, 0, 0) == [0, 3, 4]          # .5, .9, .2: slots 3 and 4 move into 1 and 2, in order


def test_append_refuses_outputs_that_its_blocks_still_read(K):
    """lens, seen and start are read by every block while the first one writes lens_out and seen_out."""
    lib, c = K.lib(), _cache(K)
    start, lens, seen, out, out2 = (P(256 * i) for i in range(1, 6))
    arg = [c, FAKE, FAKE, 0, 1, 256, 128, 256, 128, start, lens, None, None, None, 0, seen, None, None, None]
    for lens_out, seen_out in ((lens, None), (seen, None), (start, None), (None, lens), (None, seen), (None, start),
                               (out, out), (out, lens), (seen, out2)):
        arg[11], arg[16] = lens_out, seen_out
        assert lib.kq_kv_append(*arg) == K.KQ_ERR_INVALID_ARG, (lens_out, seen_out)
        assert "apart" in K.last_error()
    arg[11], arg[15], arg[16] = None, None, lens   # seen = NULL counts from lens
    assert lib.kq_kv_append(*arg) == K.KQ_ERR_INVALID_ARG
    many = _cache(K, batch=8)
    arg[0], arg[15], arg[16] = many, seen, None
    for near in (lens, seen, start):   # parts of one array
        for off in (-28, 4, 28):
            arg[11] = P(near.value + off)
            assert lib.kq_kv_append(*arg) == K.KQ_ERR_INVALID_ARG, off


def test_evict_refuses_a_length_output_that_its_blocks_still_read(K):
    """A sequence's lens and seen are read by the blocks of all its heads while one of them writes lens_out."""
    lens, acc, pos, seen, lib = *(P(256 * i) for i in range(1, 5)), K.lib()
    c = _cache(K, batch=8)
    for lens_out in (lens, seen, P(lens.value + 4), P(seen.value - 28)):
        assert lib.kq_kv_evict(c, lens, acc, pos, seen, 64, 8, 4, 2, lens_out, acc, pos, None, FAKE, 1 << 20,
                               None) == K.KQ_ERR_INVALID_ARG
        assert "apart" in K.last_error()
