"""KvCache's own account of its sequences, on the CPU with a stand-in for the kernels' calls: what fits is
taken, without an eviction that nothing asks for, and what does not is refused."""
import pytest
import torch


@pytest.fixture
def serving(monkeypatch):
    from paper_2607_07964_gb300 import serving

    class Calls:
        evictions = 0

        @staticmethod
        def kq_kv_append(k, v, start, lens, data, table, lens_out, acc, pos, seen, seen_out, info):
            lens_out.copy_(lens + start[1:] - start[:-1])
            seen_out.copy_(seen + start[1:] - start[:-1])

        @classmethod
        def kq_kv_evict(cls, data, table, lens, acc, pos, seen, dim, budget, recent, sink, lens_out, acc_out, pos_out, ws, info):
            cls.evictions += 1
            lens_out.copy_(lens.clamp(max=budget))

        @staticmethod
        def kq_kv_evict_workspace(acc, budget):
            return 256

        @staticmethod
        def kq_kv_cache_bytes(page, dim):
            return page * (dim + 8)

    monkeypatch.setattr(serving, "kq", Calls)
    return serving


def _append(c, counts, most=None):
    start = torch.tensor([0] + counts, dtype=torch.int32).cumsum(0).to(torch.int32)
    x = torch.zeros(sum(counts), c.kv_heads, c.dim)
    c.append(x, x, start, max(counts) if most is None else most)


@pytest.mark.parametrize("by_sequence", [False, True])
def test_sequences_that_take_turns_fill_their_own_slots(serving, by_sequence):
    c = serving.KvCache(2, 1, 64, 16, page=16, device="cpu")
    for counts in ([6, 0], [0, 9], [10, 0], [0, 7]):
        _append(c, counts, counts if by_sequence else None)
    assert c.lens.tolist() == [16, 16] and c.seen.tolist() == [16, 16] and c.most == 16
    with pytest.raises(ValueError, match="do not fit"):
        _append(c, [0, 1], [0, 1] if by_sequence else None)
    assert c.lens.tolist() == [16, 16]


@pytest.mark.parametrize("by_sequence", [False, True])
def test_a_budget_cuts_only_when_a_sequence_is_full(serving, by_sequence):
    c = serving.KvCache(2, 1, 64, 16, page=16, budget=8, device="cpu")
    for counts in ([8, 1], [1, 9], [7, 1]):
        _append(c, counts, counts if by_sequence else None)
    assert c.lens.tolist() == [16, 11] and serving.kq.evictions == 0
    _append(c, [0, 5], [0, 5] if by_sequence else None)
    assert c.lens.tolist() == [16, 16] and serving.kq.evictions == 0
    _append(c, [1, 0], [1, 0] if by_sequence else None)
    assert c.lens.tolist() == [9, 8] and serving.kq.evictions == 1 and c.most == 9
    with pytest.raises(ValueError, match="do not fit"):
        _append(c, [0, 9], [0, 9] if by_sequence else None)


def test_steps_of_all_sequences_do_not_wait_for_the_device(serving):
    """Prompts of known lengths and steps that every sequence takes part in leave nothing to read back."""
    c = serving.KvCache(3, 1, 64, 24, page=16, budget=16, device="cpu")
    c.measure = None   # not callable
    _append(c, [9, 2, 5], [9, 2, 5])
    for _ in range(40):
        _append(c, [1, 1, 1], 1)
    assert c.seen.tolist() == [49, 42, 45] and max(c.lens.tolist()) == c.most
    with pytest.raises(ValueError, match="3 counts"):
        _append(c, [1, 1, 1], [1, 2])
    with pytest.raises(ValueError, match="tokens of k"):
        _append(c, [1, 1, 1], [1, 1, 2])


def test_eviction_without_a_budget_is_refused(serving):
    with pytest.raises(ValueError, match="without a budget"):
        serving.KvCache(1, 1, 64, 16, page=16, device="cpu").evict()
