"""What moa_kv_reserve says of entries that name no page, where the batch has too few rows: the same by one launch and by three.

Only entries that rows of the batch lie in count: those of a refused sequence do, those of tokens beyond the batch's rows do not."""
import pytest

from test_gpu_kv_pages import Pages, i32

pytestmark = pytest.mark.gpu

PAGE, MP = 16, 8


def bad_entries(s, at):
    for b, p in at:
        s.table[b, p] = s.n_pages + 3 + b
    s.t_table.copy_(i32(s.table))


@pytest.mark.parametrize("B", [4, 1024, 1025, 2300])           # one launch up to 1024 sequences, then three
@pytest.mark.parametrize("where", ["behind the cut", "on both sides of it", "in front of it", "in a sequence without rows", "nowhere"])
def test_entries_behind_the_last_row(B, where):
    """The last but one sequence wants five pages' worth and has rows for two."""
    s = Pages(B, 3 * B + 40, PAGE, MP, seed=B)
    n = s.rng.integers(0, 3, B)
    n[B - 2:] = 5 * PAGE, 3
    T = int(n[:B - 2].sum()) + 2 * PAGE
    bad_entries(s, {"behind the cut": [(B - 2, 2), (B - 2, 4)], "on both sides of it": [(B - 2, 1), (B - 2, 3)], "in front of it": [(B - 2, 0)],
                    "in a sequence without rows": [(B - 1, 0)], "nowhere": []}[where])
    for alias in (False, True):
        got = s.reserve(n, T, alias=alias)                     # (compares the status with the host's)
        assert got[B - 2:] == [2 * PAGE, 0]


@pytest.mark.parametrize("rows", [20, 9000])                   # one launch; three, where nothing is cut
def test_entries_of_a_refused_sequence(rows):
    s = Pages(3, 12, PAGE, MP, seed=1, free=1)
    bad_entries(s, [(1, 0)])
    assert s.reserve([0, 3 * PAGE, 4], 3 * PAGE + rows) == [0, 0, 0]
    assert s.reserve([0, 0, 4], rows) == [0, 0, 4]


@pytest.mark.parametrize("first", [4, 6000])                   # 3004 rows, one launch; 9000, three
def test_a_long_prompt_s_entries(first):
    """More entries than a workgroup looks at in one go, one of them no page: in the rows that there are, or behind them."""
    for p in (2999, 3000, 5999):
        s = Pages(2, 12000, 1, 6000, seed=2)
        bad_entries(s, [(1, p)])
        assert s.reserve([first, 6000], first + 3000) == [first, 3000]
