"""kq_qk_rotate and its gradient on the CPU: outputs that would be written over one another, or over what the other side still
reads, are refused before any CUDA call."""
import ctypes

import pytest

P, I64 = ctypes.c_void_p, ctypes.c_int64


class Heads(ctypes.Structure):   # as include/kronq.h has them
    _fields_ = [("data", P), ("heads", I64), ("token_stride", I64), ("head_stride", I64)]


class Rotation(ctypes.Structure):
    _fields_ = [("freq", P), ("rot", I64), ("pos", P), ("start", P), ("first", P), ("batch", I64), ("interleaved", ctypes.c_int),
                ("scale", ctypes.c_float)]


@pytest.fixture(scope="module")
def K():
    from paper_2607_07964_gb300 import build, kronq
    build.build()
    kronq.lib()
    return kronq


def _at(data):
    return ctypes.byref(Heads(data, 2, 256, 128))


ROTATION = ctypes.byref(Rotation(256, 64, 256, None, None, 0, 0, 1.0))
Q, KEY, GQ, GK, QO, KO = (4096 * i for i in range(1, 7))


@pytest.mark.parametrize("q,k,q_out,k_out", [(Q, KEY, QO, QO), (Q, Q, Q, Q), (Q, KEY, KEY, KO), (Q, KEY, QO, Q), (Q, KEY, KEY, Q)])
def test_forward(K, q, k, q_out, k_out):
    r = K.lib().kq_qk_rotate(ROTATION, 0, 4, 128, _at(q), _at(k), _at(q_out), _at(k_out), P(256), P(256), 1e-6, None)
    assert r == K.KQ_ERR_INVALID_ARG and "each other" in K.last_error()


@pytest.mark.parametrize("q_out,k_out,gq_weight,gk_weight", [(QO, QO, 256, 512), (GK, KO, 256, 512), (QO, GQ, 256, 512), (KEY, KO, 256, 512),
                                                             (QO, Q, 256, 512), (QO, KO, 256, 256)])
def test_gradient(K, q_out, k_out, gq_weight, gk_weight):
    r = K.lib().kq_qk_rotate_grad(ROTATION, 1, 4, 128, _at(Q), _at(KEY), _at(GQ), _at(GK), _at(q_out), _at(k_out), P(256), P(256), 1e-6,
                                  P(gq_weight), P(gk_weight), P(256), 1 << 30, None)
    assert r == K.KQ_ERR_INVALID_ARG and "each other" in K.last_error()
