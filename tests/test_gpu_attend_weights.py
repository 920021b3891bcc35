"""The weights of si_attend between the softmax and the values: how many bits they keep, and what becomes of values that are not finite.

Tolerances are those of test_gpu_attend.py but for the weights: two bf16 roundings one after the other, half a step (2^-8) of half a step, so 2^-16 of
sum p |v|.  Values of alternating sign make sum p v small beside it, and small q the errors of the scores small beside both."""
import math

import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
from attention_reference import attend64
from test_gpu_attend import BF, F8, call, filled

pytestmark = pytest.mark.gpu


def set_value(c, seq, pos, dim, bits, which=1, head=0, layer=0):
    """one element of K (which = 0) or V (1); dim None: all of them"""
    page = int(c.table[seq, pos // c.page])
    place = c.places([pos % c.page])[which][0]
    flat = c.pages.view(torch.uint8 if c.kind == F8 else torch.int16)
    flat[page, layer, which, head, torch.from_numpy(place if dim is None else place[[dim]]).cuda()] = bits


def alternating(c, lens):
    """V of position t: +1 or -1 in turn"""
    one, minus = (0x38, 0xb8) if c.kind == F8 else (0x3f80, 0xbf80 - 0x10000)
    for s, x in enumerate(lens):
        for t in range(x):
            for h in range(c.kv_heads):
                set_value(c, s, t, None, one if t % 2 == 0 else minus, head=h)


@pytest.mark.parametrize("kind,d", [(BF, 64), (BF, 96), (BF, 128), (BF, 192), (BF, 256), (F8, 64), (F8, 128), (F8, 192), (F8, 256)])
@pytest.mark.parametrize("per,n_new", [(4, 1), (5, 4), (12, 5)])
def test_values_that_cancel(kind, d, per, n_new):
    """Rows of 16, 32 and 64 a block."""
    lens = [40, 61]
    c = filled(kind, lens, 64, 1, d, seed=d + per)
    alternating(c, lens)
    check(c, lens, per, n_new)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_cancel_for_128_rows(kind, d):
    """The last 50 of 3000 positions, under a window."""
    lens = [3000]
    c = filled(kind, lens, 128, 1, d, seed=d)
    one, minus = (0x38, 0xb8) if kind == F8 else (0x3f80, 0xbf80 - 0x10000)
    for t in range(2900, 3000):
        set_value(c, 0, t, None, one if t % 2 == 0 else minus)
    check(c, lens, 16, 6, window=50, max_len=20000)


def check(c, lens, per, n_new, window=0, max_len=None):
    heads, d = per * c.kv_heads, c.d
    q = (torch.randn((len(lens) * n_new, heads * d), generator=torch.Generator().manual_seed(d)) * 0.05).to(torch.bfloat16).cuda()
    out, lse = call(c, q, lens, n_new, heads, window, max_len=max_len)
    qq = q.double().cpu().numpy().reshape(-1, n_new, heads, d)
    for i, x in enumerate(lens):
        k, v = c.gather(0, i, x)
        lo = max(0, x - n_new + 1 - window) if window else 0
        o, l, mag_s, mag_o = attend64(qq[i], k[:, lo:], v[:, lo:], n_new, window, 1 / math.sqrt(d))
        ds = (d * 2.0 ** -23 + 2.0 ** -22) * mag_s
        sums = (x / 16 + 64) * 2.0 ** -23
        tol = 2.0 ** -8 * np.abs(o) + 1.01 * (2.0 ** -16 + 2 * ds[..., None] + 2 * sums) * mag_o
        err = np.abs(out[i] - o)
        assert np.all(err <= tol), "sequence %d: worst %.3g of its tolerance" % (i, np.max(err / tol))
        assert np.all(np.abs(lse[i] - l) <= ds + sums + 2.0 ** -22 * np.abs(l))


@pytest.mark.parametrize("kind,bits,want", [(BF, 0x7f80, math.inf), (BF, 0xff80 - 0x10000, -math.inf), (BF, 0x7fc0, math.nan), (F8, 0x7f, math.nan)])
@pytest.mark.parametrize("per,n_new,L", [(4, 1, 700), (8, 2, 203), (6, 5, 700), (16, 4, 2500), (16, 6, 2500)])
def test_a_value_that_is_not_finite(kind, bits, want, per, n_new, L):
    """Seen by all rows, in the middle of a sequence and beside its end: its element of the output is the value, whatever the weights' rests are; every other
    element has the bits that it has without."""
    for at in (L // 2, L - n_new):
        c = filled(kind, [L, 90], 128, 2, 64, seed=3)
        q = (torch.randn((2 * n_new, 2 * per * 64), generator=torch.Generator().manual_seed(1)) * 0.3).to(torch.bfloat16).cuda()
        clean_out, clean_lse = call(c, q, [L, 90], n_new, 2 * per)
        set_value(c, 0, at, 5, bits, head=1)
        out, lse = call(c, q, [L, 90], n_new, 2 * per)
        assert np.array_equal(out[0, :, per:, 5], np.full((n_new, per), want), equal_nan=True)
        out[0, :, per:, 5] = clean_out[0, :, per:, 5]
        assert np.array_equal(out, clean_out) and np.array_equal(lse, clean_lse)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("per,n_new", [(2, 3), (6, 5), (16, 6)])
def test_values_that_are_not_finite_seen_by_some(kind, per, n_new):
    """NaN in each of the new tokens' values: token j has it in elements 0 .. j, and all else as without."""
    L = 1900
    c = filled(kind, [L], 128, 1, 128, seed=5)
    q = (torch.randn((n_new, per * 128), generator=torch.Generator().manual_seed(2)) * 0.3).to(torch.bfloat16).cuda()
    clean_out, clean_lse = call(c, q, [L], n_new, per, max_len=6000)
    for j in range(n_new):
        set_value(c, 0, L - n_new + j, j, 0x7f if kind == F8 else 0x7fc0)
    out, lse = call(c, q, [L], n_new, per, max_len=6000)
    assert np.array_equal(lse, clean_lse)
    for j in range(n_new):
        assert np.isnan(out[0, j, :, :j + 1]).all() and np.array_equal(out[0, j, :, j + 1:], clean_out[0, j, :, j + 1:])


def test_values_that_overflow_the_sum():
    """Finite values, a sum beyond fp32: infinite, as the sum is."""
    c = filled(BF, [64], 64, 1, 64, seed=1)
    for t in range(64):
        set_value(c, 0, t, 9, 0x7f7f)
    q = torch.zeros((1, 64), dtype=torch.bfloat16, device="cuda")
    out, _ = call(c, q, [64], 1, 1)
    assert np.isposinf(out[0, 0, 0, 9]) and np.isfinite(np.delete(out[0, 0, 0], 9)).all()


@pytest.mark.parametrize("per,n_new,L", [(4, 1, 300), (4, 1, 9000), (6, 4, 700), (6, 5, 9000), (16, 5, 2500)])
def test_scores_of_plus_infinity(per, n_new, L):
    """A key of +infinity against positive queries: ln sum exp is +infinity, the output inf / inf; against negative ones the weight is 0.  The other sequence
    and the tokens before keep their bits, and NaN beside +infinity is NaN."""
    c = filled(BF, [L, 90], 128, 2, 64, seed=4)
    q = (torch.randn((2 * n_new, 2 * per * 64), generator=torch.Generator().manual_seed(3)) * 0.3).to(torch.bfloat16).cuda()
    q.view(2, n_new, 2, per, 64)[0, :, 0, :, 7] = torch.tensor([1.0, -1.0] * (per // 2), dtype=torch.bfloat16)
    clean_out, clean_lse = call(c, q, [L, 90], n_new, 2 * per)
    pages = c.pages.clone()
    for at, seen in ((L // 2, 0), (L - 1, n_new - 1)):
        set_value(c, 0, at, 7, 0x7f80, which=0)
        out, lse = call(c, q, [L, 90], n_new, 2 * per)
        rows = lse[0, seen:, :per]
        assert np.isposinf(rows[:, ::2]).all() and np.isfinite(rows[:, 1::2]).all()
        assert np.isnan(out[0, seen:, :per:2]).all() and np.isfinite(out[0, seen:, 1:per:2]).all()
        for a, b in ((out, clean_out), (lse, clean_lse)):
            assert np.array_equal(a[1], b[1]) and np.array_equal(a[0, :, per:], b[0, :, per:]) and np.array_equal(a[0, :seen], b[0, :seen])
        c.pages.copy_(pages)
    set_value(c, 0, L // 2, 7, 0x7f80, which=0)
    set_value(c, 0, 3, 7, 0x7fc0, which=0)
    out, lse = call(c, q, [L, 90], n_new, 2 * per)
    assert np.isnan(lse[0, :, :per]).all() and np.isnan(out[0, :, :per]).all() and np.isfinite(out[1]).all()


@pytest.mark.parametrize("kind,d", [(BF, 96), (BF, 128), (BF, 192), (BF, 256), (F8, 128), (F8, 192), (F8, 256)])
@pytest.mark.parametrize("per,n_new", [(4, 1), (5, 4), (9, 6), (16, 6)])
def test_values_that_are_not_finite_in_heads_of_other_sizes(kind, d, per, n_new):
    """One that all rows see, one that only the last token sees."""
    lens = [1500, 90]
    c = filled(kind, lens, 128, 2, d, seed=d)
    q = (torch.randn((2 * n_new, 2 * per * d), generator=torch.Generator().manual_seed(d)) * 0.3).to(torch.bfloat16).cuda()
    clean_out, clean_lse = call(c, q, lens, n_new, 2 * per)
    nan = 0x7f if kind == F8 else 0x7fc0
    set_value(c, 0, 700, d - 1, nan if kind == F8 else 0x7f80, head=0)
    set_value(c, 0, lens[0] - 1, 3, nan, head=1)
    out, lse = call(c, q, lens, n_new, 2 * per)
    first = out[0, :, :per, d - 1]
    assert np.isnan(first).all() if kind == F8 else np.isposinf(first).all()
    assert np.isnan(out[0, n_new - 1, per:, 3]).all()
    out[0, :, :per, d - 1] = clean_out[0, :, :per, d - 1]
    out[0, n_new - 1, per:, 3] = clean_out[0, n_new - 1, per:, 3]
    assert np.array_equal(out, clean_out) and np.array_equal(lse, clean_lse)
