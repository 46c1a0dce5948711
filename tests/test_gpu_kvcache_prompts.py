"""GPU checks of attention with weights over whole prompts and without a log-sum output. Bounds as derived in
test_gpu_kvcache.py."""
import numpy as np
import pytest
import torch

import test_gpu_kvcache as kv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_07964_gb300 import build
    build.build()


@pytest.mark.parametrize("dim,heads,group,lens,counts", [(128, 2, 4, [130, 33, 0], [1, 3, 1]), (64, 1, 5, [40, 700], [2, 1])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_from_the_workspaces_own_log_sums(dim, heads, group, lens, counts, dtype):
    """acc without lse: the log-sums that the weights need stay in the workspace."""
    rng = np.random.default_rng(dim + sum(lens))
    cache = kv._pool(len(lens), max(lens), 16, heads, dim, rng)
    kv._fill(cache, lens, heads, rng)
    q = kv._rounded(rng.standard_normal((sum(counts), heads * group, dim)), dtype)
    acc0 = rng.random((len(lens), heads, max(lens))).astype(np.float32)
    out, lse, acc = kv._run_attend(cache, q.to(kv.DEV), counts, lens, heads, 0.1, True, dtype, acc0, max(lens), want_lse=False)
    assert lse is None
    kv._check_attend(cache, q, counts, lens, heads, 0.1, dtype, out, lse, acc, acc0)


@pytest.mark.parametrize("dim,heads,group,lens,counts", [(64, 1, 4, [300, 171], [300, 170]), (128, 1, 2, [260], [230])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_whole_prompts_with_weights(dim, heads, group, lens, counts, dtype):
    """Hundreds of queries a sequence, each seeing what came before it, their weights summed over all of them."""
    rng = np.random.default_rng(dim + sum(counts))
    cache = kv._pool(len(lens), max(lens), 64, heads, dim, rng)
    kv._fill(cache, lens, heads, rng)
    q = kv._rounded(rng.standard_normal((sum(counts), heads * group, dim)), dtype)
    acc0 = np.zeros((len(lens), heads, max(lens)), np.float32)
    scale = 1 / np.sqrt(dim)
    out, lse, acc = kv._run_attend(cache, q.to(kv.DEV), counts, lens, heads, scale, True, dtype, acc0, max(lens))
    kv._check_attend(cache, q, counts, lens, heads, scale, dtype, out, lse, acc, acc0)
