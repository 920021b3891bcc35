"""si_attend with heads of 96, 192 and 256 over sequences that are cut into slices: unfinished sums, joined by the last block or by the second kernel, rings that
go round many times.  Comparison and tolerances are those of test_gpu_attend.py."""
import pytest

from test_gpu_attend import BF, F8, attend_case

pytestmark = pytest.mark.gpu
DIMS = [(BF, 96), (BF, 192), (BF, 256), (F8, 192), (F8, 256), (F8, 128)]


@pytest.mark.parametrize("kind,d", DIMS)
@pytest.mark.parametrize("per,n_new", [(1, 1), (4, 5), (9, 8), (13, 10)])
def test_long_sequences(kind, d, per, n_new):
    """Rows: 1 (joined by the last block), 20, 72 and 130 (sums of more than 64 KB for a sequence: the second kernel)."""
    attend_case(kind, [5000], n_new, 2 * per, 2, d, 64, seed=d)
    attend_case(kind, [3000, 0, 5, 1900, 64], n_new, per, 1, d, 128, seed=per)


@pytest.mark.parametrize("kind,d", DIMS)
@pytest.mark.parametrize("per,n_new", [(2, 1), (5, 4), (12, 6)])
def test_windows_over_long_sequences(kind, d, per, n_new):
    attend_case(kind, [4500, 800], n_new, 2 * per, 2, d, 64, window=2100, seed=d)
    attend_case(kind, [2500], n_new, per, 1, d, 64, window=37, max_len=30000, seed=d + 1)


@pytest.mark.parametrize("kind,d", DIMS)
@pytest.mark.parametrize("per,n_new", [(4, 1), (4, 5), (12, 6)])
def test_many_sequences_of_all_lengths(kind, d, per, n_new):
    """Slices that hold ends, whole sequences and beginnings."""
    attend_case(kind, [(i * 379) % 2900 for i in range(23)], n_new, 2 * per, 2, d, 64, seed=d)
