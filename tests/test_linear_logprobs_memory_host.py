"""Workspaces of scoring from hidden states on the CPU: bounded whatever the number of rows."""
import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2607_07964_gb300 import build, kronq
    build.build()
    return kronq.lib()


@pytest.mark.parametrize("V", [1, 64, 1000, 32001, 128000, 200000, 1 << 20])
def test_scoring_holds_sums_of_a_bounded_number_of_rows(lib, V):
    """16 bytes for each of 2^24 sums, or of 4096 rows', and 4 a row, however many rows there are."""
    parts = -(-V // 64)
    rows = max(4096, (1 << 24) // parts)
    for T in (129, 4096, 4097, 16384, 262144, 1 << 24):
        assert lib.kq_linear_logprobs_workspace(T, V, 4096) <= 16 * min(T, rows) * parts + 4 * min(T, rows) + 512
    assert lib.kq_linear_logprobs_workspace(262144, 128000, 4096) <= (1 << 28) + 65536 + 512
