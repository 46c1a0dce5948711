"""kq_kv_attend_window, kq_linear_logprobs and its gradient on the CPU: arguments that are refused before any CUDA call."""
import ctypes

import pytest

P = ctypes.c_void_p
A = P(256)


@pytest.fixture(scope="module")
def K():
    from paper_2607_07964_gb300 import build, kronq
    build.build()
    kronq.lib()
    return kronq


def _refused(call, good, cases):
    for at, value, status in cases:
        args = list(good)
        args[at] = value
        assert call(*args) == status, (at, value)


def test_scoring_refuses(K):
    # x, T, d, ldx, w, V, ldw, target, logp, entropy, lse, info, ws, bytes, stream
    good = [A, 4, 64, 64, A, 100, 64, A, A, A, A, None, A, 1 << 30, None]
    _refused(K.lib().kq_linear_logprobs, good, [
        (0, None, 1), (0, P(264), 1), (1, -1, 1), (1, (1 << 24) + 1, 1), (2, 60, 2), (2, 0, 1), (2, 65544, 2), (3, 56, 1), (3, 68, 1),
        (4, None, 1), (4, P(258), 1), (5, 0, 1), (5, (1 << 20) + 1, 2), (6, 56, 1), (6, 66, 1), (7, None, 1), (8, None, 1),
        (12, None, 6), (12, P(264), 6), (13, 64, 6)])


def test_gradient_refuses(K):
    # x, T, d, ldx, w, V, ldw, target, lse, entropy, g_logp, g_entropy, gx, ldgx, gw, ldgw, info, ws, bytes, stream
    B, C, D = P(512), P(1024), P(2048)
    good = [A, 4, 64, 64, B, 100, 64, A, A, A, A, A, C, 64, D, 64, None, A, 1 << 40, None]
    _refused(K.lib().kq_linear_logprobs_grad, good, [
        (0, None, 1), (1, -1, 1), (2, 4, 2), (7, None, 1), (8, None, 1), (9, None, 1), (10, None, 1), (12, P(264), 1), (13, 56, 1),
        (13, 66, 1), (14, P(264), 1), (15, 56, 1), (15, 68, 1), (12, A, 1), (12, B, 1), (12, D, 1), (14, A, 1), (14, B, 1), (17, None, 6),
        (17, P(264), 6), (18, 64, 6)])
    args = list(good)
    args[12] = args[14] = None
    assert K.lib().kq_linear_logprobs_grad(*args) == K.KQ_ERR_INVALID_ARG


def test_workspaces_do_not_grow_with_the_logits(K):
    lib = K.lib()
    assert lib.kq_linear_logprobs_workspace(0, 10, 8) == lib.kq_linear_logprobs_grad_workspace(0, 10, 8) == 0
    for T, V, d in ((1, 1, 8), (4096, 128000, 4096), (100000, 200000, 64), (1, 1 << 20, 8), (128, 1 << 20, 64)):
        assert lib.kq_linear_logprobs_workspace(T, V, d) <= 16 * T * max(V / 64 + 1, 8 * (min(V, 16384) / 128 + 1)) + 4 * T + 1024
        # two pieces of 2^26 values in bf16, or of 1024 columns; all columns of up to 128 rows; gx in fp32, split where it is small
        piece = max(1 << 26, 1024 * T) if T > 128 else 128 * (V + 256) // 2
        split = max(1, 76 // (-(-T // 256) * -(-d // 256)))
        assert lib.kq_linear_logprobs_grad_workspace(T, V, d) <= 2 * 2 * piece + split * T * d * 4 + 4096


def test_window_refuses(K):
    c = ctypes.byref(K._KvCache(256, 256, 4, 64, 2, 128, 1, 2))
    # cache, q, dtype, T, q_heads, strides, start, lens, scale, window, sink, out, lse, info, ws, bytes, stream
    good = [c, A, 0, 1, 4, 512, 128, A, A, 1.0, 16, 4, A, None, None, A, 1 << 30, None]
    _refused(K.lib().kq_kv_attend_window, good, [
        (0, None, 1), (1, None, 1), (2, 5, 2), (3, -1, 1), (4, 3, 1), (7, None, 1), (8, None, 1), (9, float("nan"), 1), (10, 0, 1),
        (10, -5, 1), (11, -1, 1), (12, None, 1), (15, None, 6), (16, 8, 6), (15, P(264), 6)])
    assert "window" in (K.lib().kq_kv_attend_window(*good[:10], 0, *good[11:]), K.last_error())[1]
