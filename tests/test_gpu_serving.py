"""The serving path end to end: a cache that evicts keeps what its positions say, and one that does not
reproduces dense attention over the values that were cached."""
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


def test_cache_without_a_budget_is_dense_attention_over_the_cached_values():
    from paper_2607_07964_gb300.serving import KvCache
    g = torch.Generator(DEV).manual_seed(0)
    c = KvCache(2, 2, 64, 50, page=16)
    outs, qs = [], []
    for most, counts in ((9, [9, 4]), (1, [1, 1]), (3, [0, 3])):
        start = torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32, device=DEV)
        k, v = (torch.randn(sum(counts), 2, 64, device=DEV, generator=g) for _ in range(2))
        q = torch.randn(sum(counts), 6, 64, device=DEV, generator=g)
        c.append(k, v, start, most)
        outs.append(c.attend(q, start))
        qs.append((q, counts))
    c.check()
    assert c.lens.tolist() == [10, 8] and c.seen.tolist() == [10, 8]
    k, v = (t.double() for t in c.read())
    have = [0, 0]
    for out, (q, counts) in zip(outs, qs):
        i = 0
        for b, n in enumerate(counts):
            for j in range(n):
                see = have[b] + j + 1
                for h in range(6):
                    s = k[b, :see, h // 3] @ q[i, h].double() / math.sqrt(64)
                    want = torch.softmax(s, 0) @ v[b, :see, h // 3]
                    # 2^-18 of the values' size, and 2^-18 of the scores' terms (sums of |q| |k| over 64 dimensions)
                    size = v[b, :see, h // 3].abs().max()
                    terms = (k[b, :see, h // 3].abs() @ q[i, h].double().abs()).max() / math.sqrt(64)
                    assert (out[i, h].double() - want).abs().max() <= 2.0 ** -17 * size * (1 + terms)
                i += 1
            have[b] += n


def test_cache_with_a_budget_evicts_when_it_is_full():
    from paper_2607_07964_gb300.serving import KvCache
    g = torch.Generator(DEV).manual_seed(1)
    c = KvCache(1, 1, 64, 24, page=16, budget=16, recent=6, sink=2)
    start = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    keys = []
    for t in range(60):
        k = torch.randn(1, 1, 64, device=DEV, generator=g)
        keys.append(k[0, 0])
        c.append(k, -k, start, 1)
        c.attend(torch.randn(1, 4, 64, device=DEV, generator=g), start)
    c.check()
    n = int(c.lens[0])
    pos = c.pos[0, 0, :n].tolist()
    assert int(c.seen[0]) == 60 and n <= 24 and len(set(pos)) == n
    assert {0, 1} <= set(pos) and set(range(54, 60)) <= set(pos)     # the sink and the last ones
    k, v = c.read()
    for j, p in enumerate(pos):   # every slot holds the row of its position: within half a step of it, and a rounding of the scale
        step = (keys[p].max() - keys[p].min()) / 15 * 1.02
        assert (k[0, j, 0] - keys[p]).abs().max() <= step / 2 and (v[0, j, 0] + keys[p]).abs().max() <= step / 2
    assert torch.isfinite(c.acc).all() and abs(float(c.acc[0, 0, :n].sum())) <= 4 * 60
    with pytest.raises(ValueError, match="do not fit"):
        c.append(torch.zeros(9, 1, 64, device=DEV), torch.zeros(9, 1, 64, device=DEV),
                 torch.tensor([0, 9], dtype=torch.int32, device=DEV), 9)


def test_example_decodes_and_scores():
    from paper_2607_07964_gb300.serving import example
    ids, logps, block = example(steps=12)
    again = example(steps=12)
    assert torch.equal(ids, again[0]) and torch.equal(logps, again[1])
    assert ids.shape == (12, 3) and torch.isfinite(logps).all() and (logps <= 0).all()
    c = block.cache
    assert c.seen.tolist() == [52, 19, 35] and max(c.lens.tolist()) <= c.slots
