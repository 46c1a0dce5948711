"""Norm and rotation on the CPU: the reference's gradient against differences, and arguments that are refused before any
CUDA call."""
import ctypes

import numpy as np
import pytest

import rotate_reference as ref

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


@pytest.mark.parametrize("rot,interleaved,norm", [(8, False, True), (6, True, True), (2, False, False), (0, True, True)])
def test_reference_gradient_matches_differences(rot, interleaved, norm):
    rng = np.random.default_rng(rot)
    T, H, D, eps, scale = 3, 2, 8, 1e-3, 1.3
    x, gy = rng.standard_normal((T, H, D)), rng.standard_normal((T, H, D))
    w = rng.standard_normal(D) if norm else None
    angle = ref.angles([0, 5, -7], ref.fractions(rng.random(rot // 2)))

    def loss(x, w):
        return (ref.forward(x, w, eps, angle, rot, interleaved, scale)[0] * gy).sum()

    gx, _, gw, _ = ref.backward(x, w, eps, gy, angle, rot, interleaved, scale)
    e = 1e-5   # the differences' own error: e^2 times the third derivative, and 1e-16 / e
    for _ in range(4):
        v = rng.standard_normal(x.shape)
        assert abs((loss(x + e * v, w) - loss(x - e * v, w)) / (2 * e) - (gx * v).sum()) < 1e-7
        if norm:
            v = rng.standard_normal(D)
            assert abs((loss(x, w + e * v) - loss(x, w - e * v)) / (2 * e) - (gw * v).sum()) < 1e-7


def test_angles_of_far_positions():
    theta = [1.0, 0.123, 1e-4]
    got = ref.angles([2 ** 31 - 1, -3], ref.fractions(theta))
    from fractions import Fraction
    for i, p in enumerate((2 ** 31 - 1, -3)):
        for j, t in enumerate(theta):
            exact = Fraction(p) * Fraction(t) / Fraction(2 * np.pi)
            turn = float(exact - round(exact))
            d = got[i, j] / (2 * np.pi) - turn
            # theta / (2 pi) is rounded once (2^-53 of it) before it is counted in 2^-64, which loses nothing more of
            # a number from 2^-11 up and 2^-65 of a smaller one; the angle itself is a float of at most half a turn, as
            # is its quotient by 2 pi: 3 roundings of 2^-54
            assert abs(d - round(d)) <= 2.0 ** 31 * (t / (2 * np.pi) * 2.0 ** -53 + 2.0 ** -65) + 3 * 2.0 ** -54


def _heads(K, **over):
    f = dict(data=256, heads=2, token_stride=256, head_stride=128)
    f.update(over)
    return ctypes.byref(Heads(*f.values()))


def _rotation(K, **over):
    f = dict(freq=256, rot=64, pos=256, start=None, first=None, batch=0, interleaved=0, scale=1.0)
    f.update(over)
    return ctypes.byref(Rotation(*f.values()))


def test_arguments_are_refused_on_the_host(K):
    lib, h, r = K.lib(), _heads(K), _rotation(K)
    good = [r, 0, 4, 128, h, h, h, h, P(256), P(256), 1e-6, None]
    cases = [(0, None, 1), (1, 2, 2), (2, -1, 1), (3, 0, 1), (3, 257, 2), (3, 32, 1), (4, None, 1), (5, None, 1), (6, None, 1),
             (7, None, 1), (8, P(257), 1), (10, -1.0, 1), (10, float("nan"), 1), (10, float("inf"), 1)]
    cases += [(0, _rotation(K, **o), 1) for o in (dict(rot=63), dict(rot=-2), dict(rot=130), dict(freq=None), dict(freq=260),
                                                  dict(scale=float("inf")), dict(start=256), dict(first=256),
                                                  dict(start=256, first=256, batch=1), dict(pos=None, start=256, first=256, batch=0))]
    cases += [(i, _heads(K, **o), 1) for i in (4, 6) for o in (dict(data=None), dict(data=257), dict(heads=3), dict(heads=0))]
    cases += [(i, _heads(K, **o), 1) for i in (6, 7) for o in (dict(token_stride=0), dict(head_stride=0))]   # rows in one place
    for at, value, status in cases:
        args = list(good)
        args[at] = value
        assert lib.kq_qk_rotate(*args) == status, (at, value)
    assert lib.kq_qk_rotate(r, 0, 0, 128, h, h, h, h, None, None, 0.0, None) == 0   # no tokens
    back = [r, 1, 4, 128, h, h, h, h, h, h, P(256), P(256), 1e-6, P(256), P(256), P(256), 1 << 30, None]
    for at, value, status in ((4, None, 1), (6, None, 1), (7, None, 1), (8, None, 1), (10, None, 1), (15, None, 6), (15, P(264), 6),
                              (16, 8, 6), (4, _heads(K, heads=3), 1), (1, 9, 2)):
        args = list(back)
        args[at] = value
        assert lib.kq_qk_rotate_grad(*args) == status, (at, value)
    assert lib.kq_qk_rotate_grad_workspace(0, 128) == 0 and lib.kq_qk_rotate_grad_workspace(3, 128) == 3 * 2 * 128 * 4


def test_the_binding_packs_the_structures_of_the_header(K):
    assert len(K._HEADS(0, 0, 0, 0)) == ctypes.sizeof(Heads)
    r = Rotation.from_buffer_copy(K._ROTATION(8, 64, 16, 24, 32, 5, True, 1.5))
    assert [getattr(r, n) for n, _ in Rotation._fields_] == [8, 64, 16, 24, 32, 5, 1, 1.5]


def test_binding_refuses_host_tensors_and_wrong_shapes(K):
    import torch
    x = torch.zeros(2, 3, 64)
    with pytest.raises(ValueError, match="CUDA"):
        K.kq_qk_rotate(x, None, x, None, torch.zeros(32, dtype=torch.int64))


def test_frequencies_are_fractions_of_a_turn(K):
    theta = [1.0, 0.5, 3.2, 6.0, -1.0, 1e-6]
    got = K.kq_rotation_freq(theta, device="cpu").numpy().view(np.uint64)
    assert np.array_equal(got, ref.fractions(theta))
