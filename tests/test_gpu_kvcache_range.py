"""GPU checks of attention over values near the end of float32's range. Bounds as derived in test_gpu_kvcache.py; the
sizes keep a value times the weights' sum (at most e^2 a slot here, the scores being within 1 of each other's
middle) below 2^127."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import test_gpu_kvcache as kv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_07964_gb300 import build
    build.build()


@pytest.mark.parametrize("n,power", [(1, 108), (1, 109), (1, 113), (1, 121), (20, 109), (20, 112), (20, 115), (300, 109)])
@pytest.mark.parametrize("dim,group", [(64, 4), (128, 4), (64, 16), (128, 16)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_over_values_of_huge_scales(n, power, dim, group, dtype):
    """Value rows whose scale is about 2^power, every third one 2^-40 of it."""
    rng = np.random.default_rng(power + n)
    cache = kv._pool(1, n, 16, 1, dim, rng)
    for j in range(n):
        cache.put(0, 0, j, 0, rng.standard_normal(dim).astype(np.float32))
        codes = rng.integers(0, 16, dim)
        codes[:2] = 0, 15
        cache.put(0, 0, j, 1, ((codes - 5) * 1.25 * 2.0 ** (power - 40 * (j % 3 == 2))).astype(np.float32))
    q = kv._rounded(0.02 * rng.standard_normal((1, group, dim)), dtype)
    acc0 = np.zeros((1, 1, n), np.float32)
    out, lse, acc = kv._run_attend(cache, q.to(kv.DEV), [1], [n], 1, 0.25, True, dtype, acc0, n)
    kv._check_attend(cache, q, [1], [n], 1, 0.25, dtype, out, lse, acc, acc0)


def test_numpy_values_are_those_of_their_codes():
    """The reference's rows for such values: scale 1.25 2^109, code 12, offset -5 scales is 8.75 2^109."""
    cache = kv._pool(1, 1, 16, 1, 64, np.random.default_rng(0))
    row = np.full(64, 7.0, np.float32)
    row[:2] = -5, 10
    cache.put(0, 0, 0, 1, row * np.float32(1.25 * 2.0 ** 109))
    assert ref.quantize(row[None])[0][0, 2] == 12 and cache.rows(0, 0, 1, 1)[0][0, 2] == 8.75 * 2.0 ** 109


@pytest.mark.parametrize("n", [9, 70, 333])
@pytest.mark.parametrize("dim,group", [(64, 4), (128, 5), (64, 12), (128, 16)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
def test_attend_over_values_whose_sizes_the_weights_even_out(n, dim, group, dtype, order):
    """Value rows from 2^-50 to 2^50, and keys that give the larger ones the smaller weights: query 0 weighs them so that all
    count alike, the next ones lean to the large or to the small, the last sees the keys reversed. A row's result is what its own
    weights make of it, whatever lies beside."""
    rng = np.random.default_rng(n + dim)
    cache = kv._pool(1, n, 16, 1, dim, rng)
    power = np.linspace(-50, 50, n)
    power = power[::-1] if order == "falling" else rng.permutation(power) if order == "mixed" else power
    for j in range(n):
        key = 0.01 * rng.standard_normal(dim)
        key[0] = -power[j] * np.log(2)
        cache.put(0, 0, j, 0, key.astype(np.float32))
        cache.put(0, 0, j, 1, (rng.standard_normal(dim) * 2.0 ** power[j]).astype(np.float32))
    q = 0.01 * rng.standard_normal((1, group, dim))
    q[0, :, 0] = np.resize([1, 1.5, 0.5, -1, 0.02, 2.5], group)
    q = kv._rounded(q, dtype)
    acc0 = np.zeros((1, 1, n), np.float32)
    out, lse, acc = kv._run_attend(cache, q.to(kv.DEV), [1], [n], 1, 1.0, True, dtype, acc0, n)
    kv._check_attend(cache, q, [1], [n], 1, 1.0, dtype, out, lse, acc, acc0)
