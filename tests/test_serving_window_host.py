"""AttentionBlock on the CPU with a stand-in for the kernels' calls: a window that its cache cannot have, or that is none, is
refused when the block is made, not after a step has appended its tokens."""
import pytest
import torch


@pytest.fixture
def serving(monkeypatch):
    from paper_2607_07964_gb300 import serving

    class Calls:
        @staticmethod
        def kq_kv_append(k, v, start, lens, data, table, lens_out, acc, pos, seen, seen_out, info):
            lens_out.copy_(lens + start[1:] - start[:-1])
            seen_out.copy_(seen + start[1:] - start[:-1])

        @staticmethod
        def kq_kv_attend_workspace(q, data, table, acc):
            return 256

        @staticmethod
        def kq_kv_attend(q, start, lens, data, table, out, ws, scale, lse, acc, info):
            out.copy_(q)

        @staticmethod
        def kq_kv_attend_window(q, start, lens, data, table, out, ws, scale, window, sink, lse, info):
            assert window >= 1 and sink >= 0
            out.copy_(q)

        @staticmethod
        def kq_kv_evict_workspace(acc, budget):
            return 256

        @staticmethod
        def kq_kv_cache_bytes(page, dim):
            return page * (dim + 8)

    monkeypatch.setattr(serving, "kq", Calls)
    return serving


def _proj():
    return {n: torch.clone for n in "qkvo"}


@pytest.mark.parametrize("budget,window,sink,word", [(8, 4, 0, "evicts"), (8, 4, 2, "evicts"), (None, 0, 0, "window"),
                                                     (None, -3, 0, "window"), (None, 4, -1, "sink")])
def test_windows_that_no_step_could_use_are_refused_before_any(serving, budget, window, sink, word):
    cache = serving.KvCache(1, 1, 64, 16, page=16, budget=budget, device="cpu")
    with pytest.raises(ValueError, match=word):
        serving.AttentionBlock(_proj(), 1, cache, window=window, sink=sink)(torch.zeros(3, 64), torch.tensor([0, 3], dtype=torch.int32), 3)
    assert cache.lens.tolist() == cache.seen.tolist() == [0] and cache.most == 0


@pytest.mark.parametrize("budget,window,sink", [(8, None, 0), (None, None, 0), (None, None, 2), (None, 1, 0), (None, 5, 3)])
def test_a_block_that_can_step_does(serving, budget, window, sink):
    """Without a window every position is seen, the first ones among them."""
    cache = serving.KvCache(1, 1, 64, 16, page=16, budget=budget, device="cpu")
    x = torch.ones(3, 64)
    y = serving.AttentionBlock(_proj(), 1, cache, window=window, sink=sink)(x, torch.tensor([0, 3], dtype=torch.int32), 3)
    assert torch.equal(y, 2 * x) and cache.seen.tolist() == [3]
