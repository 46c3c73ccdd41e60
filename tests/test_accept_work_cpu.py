"""The size of kvb_accept's workspace (no GPU)."""
import pytest

from paper_2605_19049_amd import kvb

BATCHES = list(range(0, 300)) + [511, 512, 600, 1023, 1024, 1025, 4096, 1 << 20]
VOCABS = [1, 1000, 8191, 8192, 32767, 32768, 32769, 40000, 40960, 65535, 65536, 65537, 131071, 131072, 150001, 1 << 20, 1 << 24]


def size(B, V, dtype):
    return kvb.accept_work(kvb.vocab(B, 4, V, dtype))


@pytest.mark.parametrize("dtype", [kvb.F32, kvb.BF16, kvb.F16])
def test_a_workspace_for_the_largest_batch_serves_smaller_ones(dtype):
    """It never falls as B or V rises: a loop that sizes it once may call with fewer requests, whose rows may be split where
    those of the whole batch are not."""
    table = [[size(B, V, dtype) for V in VOCABS] for B in BATCHES]
    for i, row in enumerate(table):
        assert row == sorted(row), BATCHES[i]
    for j, V in enumerate(VOCABS):
        column = [row[j] for row in table]
        assert column == sorted(column), V


def test_it_holds_the_sums_and_walks_of_a_split_batch():
    """Rows of 150001 tokens are split into eight segments at 128 requests, 16 at 64: eight bytes each, and 12 a request's walk."""
    assert size(128, 150001, kvb.F32) >= 128 * (8 * 8 + 12) and size(64, 150001, kvb.F32) >= 64 * (16 * 8 + 12)
    assert all(size(B, 150001, kvb.F32) >= 128 * (8 * 8 + 12) for B in (129, 160, 600))
