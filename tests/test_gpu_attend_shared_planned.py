"""si_attend_shared at sizes that it plans by itself, against 64 bits (tolerances of test_gpu_attend.py), and the same bits from every call."""
import numpy as np
import pytest
import torch

from test_gpu_attend import BF, F8, compare
from test_gpu_attend import call as call_alone
from test_gpu_attend_shared import call, shared_cache

pytestmark = pytest.mark.gpu

CASES = {  # type, groups, new tokens, heads, kv heads, head_dim, page, window
    "64 answers to a prompt of 4000": (BF, [(4000, [1 + 7 * i % 100 for i in range(64)])], 1, 32, 8, 128, 64, 0),
    "32 answers to each of two prompts": (BF, [(5000, [3 + i for i in range(32)]), (3000, [40] * 32)], 2, 16, 8, 128, 128, 0),
    "beams over windows": (F8, [(9100, [5 * i + 1 for i in range(8)]) for _ in range(6)], 3, 24, 8, 128, 64, 8000),
    "windows that begin in own pages for some": (BF, [(6000, [4 + 200 * i for i in range(30)])], 1, 16, 8, 128, 64, 5500),
    "e4m3 heads of 256": (F8, [(5000, [9 * i for i in range(40)])], 1, 16, 8, 256, 64, 0),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_planned_calls(name, monkeypatch):
    monkeypatch.delenv("SI_ATTEND_PIECES", raising=False)
    kind, groups, n_new, heads, kv_heads, d, page, window = CASES[name]
    scales = (list(np.linspace(0.5, 1.5, kv_heads)), list(np.linspace(1.25, 0.75, kv_heads))) if kind == F8 else None
    c, lens, rows = shared_cache(kind, groups, page, kv_heads, d, scales=scales)
    q = (2 * torch.randn((len(rows) * n_new, heads * d), generator=torch.Generator().manual_seed(8))).to(torch.bfloat16).cuda()
    out, lse = call(c, q, lens, rows, n_new, heads, window)
    assert int(c.status.item()) == 0
    for i in (0, len(rows) // 2 + 1, len(rows) - 1):
        compare(c, q[i * n_new:(i + 1) * n_new], lens, n_new, heads, window, 0, 0.0, [rows[i]], out[i:i + 1], lse[i:i + 1])
    alone = call_alone(c, q, lens, n_new, heads, window=window, seqs=rows)
    assert not np.array_equal(lse, alone[1])  # (planned: the order of its sums tells)
    for _ in range(4):
        again = call(c, q, lens, rows, n_new, heads, window)
        assert np.array_equal(out, again[0]) and np.array_equal(lse, again[1])
        torch.randn(1 << 22, device="cuda").sum().item()
