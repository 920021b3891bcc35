"""si_attend_shared where a window is longer than sequences, up to the longest that there is, and where a window hides positions of a head whose scores are all 0."""
import numpy as np
import pytest
import torch

from test_gpu_attend import BF, F8, compare
from test_gpu_attend import call as call_alone
from test_gpu_attend_shared import call, shared_cache, small_calls_by_pieces_too  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("n_new", [1, 8, 70])
@pytest.mark.parametrize("window", [0x7fffffff, 0x7fffffff - 3, 1 << 30])
def test_windows_longer_than_any_sequence(kind, n_new, window):
    """sequences of fewer tokens than are asked for among them: what comes before their first token sees nothing"""
    c, lens, rows = shared_cache(kind, [(128, [3, 90, 0]), (0, [4, 2, 0]), (64, [5])], 64, 2, 64)
    q = torch.randn((len(rows) * n_new, 4 * 64), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    out, lse = call(c, q, lens, rows, n_new, 4, window)
    assert int(c.status.item()) == 0
    compare(c, q, lens, n_new, 4, 0, 0, 0.0, rows, out, lse)
    want = call(c, q, lens, rows, n_new, 4, 0)
    assert np.array_equal(out, want[0]) and np.array_equal(lse, want[1])


@pytest.mark.parametrize("window", [0, 100, 300])
def test_a_head_whose_scale_is_zero(window):
    """all of its scores are 0: the mean of what a row sees, under a window too"""
    c, lens, rows = shared_cache(F8, [(400, [3, 90, 10]), (130, [40, 4])], 64, 2, 64, scales=([0.0, 1.0], [1.0, 0.5]))
    q = torch.randn((len(rows) * 2, 4 * 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    out, lse = call(c, q, lens, rows, 2, 4, window)
    compare(c, q, lens, 2, 4, window, 0, 0.0, rows, out, lse)
    want = call_alone(c, q, lens, 2, 4, window=window, seqs=rows)
    assert np.max(np.abs(out - want[0])) < 0.02 and np.max(np.abs(lse - want[1])) < 1e-4
