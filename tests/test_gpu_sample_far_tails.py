"""si_sample where the border of top_p lies far below the largest logit: right, and in a time that does not depend on how far.

Expected numbers and their distance from the next as in test_gpu_sample_plateaus.py."""
import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
from test_gpu_sample_plateaus import around, check_rows

pytestmark = pytest.mark.gpu
V = 131072


def far_tail(offset, top, spread, seed=0):
    l = (offset + spread * np.random.default_rng(seed).uniform(-1, 1, V)).astype(np.float32)
    l[77] = offset + top
    return l


ROWS = {  # logits, temperature, top_p
    "dense values far from 0 below one peak": (far_tail(1000.0, 23.0, 0.05), 1.0, 0.99999),
    "the same next to 0": (far_tail(0.0, 23.0, 0.05), 1.0, 0.9999933242797852),
    "a flat tail": (far_tail(-20.0, 20.0, 0.5), 1.0, 0.9999),
    "two peaks": (np.where(np.arange(V) % 5000 == 9, 12.0, far_tail(-40.0, 60.0, 2.0)).astype(np.float32), 2.6, 0.9999980330467224),
}


def call_of(l, t, p):
    x, out = torch.from_numpy(l).cuda(), torch.empty(1, dtype=torch.int32, device="cuda")
    par = [torch.tensor([v], device="cuda") for v in (t, p, 0.5)]
    d = si.si_sample_t(logits=x.data_ptr(), temperature=par[0].data_ptr(), top_p=par[1].data_ptr(), u=par[2].data_ptr(), token=out.data_ptr(), stride=V, rows=1, vocab=V, type=si.SI_F32)
    d.scratch_bytes = si.si_sample_scratch_bytes(d)
    scratch = torch.zeros(d.scratch_bytes, dtype=torch.uint8, device="cuda")
    d.scratch = scratch.data_ptr()
    return d, (x, out, par, scratch)


def time_of(l, t, p):
    """us of a call on a GPU that has nothing else to do"""
    d, keep = call_of(l, t, p)
    best = 1e9
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        a.record()
        for _ in range(4):
            si.si_sample(d, torch.cuda.current_stream().cuda_stream)
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) * 250)
    return best


@pytest.mark.parametrize("name", sorted(ROWS))
def test_tokens_of_a_far_tail(name):
    l, t, p = ROWS[name]
    check_rows(l, t, [p, 1 - (1 - p) / 3, 1 - 3 * (1 - p)])
    n = int(np.sum(l >= np.median(l)))
    check_rows(l, t, around(l, t, n, 3))


@pytest.mark.parametrize("name", sorted(ROWS))
def test_a_far_tail_takes_a_few_times_an_ordinary_row(name):
    """a few turns of the search instead of one; with bins that are passed one by one these rows took up to four hundred"""
    rng = np.random.default_rng(1)
    usual = time_of((2 * rng.standard_normal(V)).astype(np.float32), 1.0, 0.9)
    t = time_of(*ROWS[name])
    print("far tail %s: %.0f us, an ordinary row %.0f" % (name, t, usual), flush=True)
    assert t < 8 * usual
