"""si_attend against its formula in 64 bits, over a cache whose pages lie in random order and hold NaN wherever no token may look.

Tolerances.  Products of bf16 (e4m3 widens exactly) are exact in fp32; a score is a sum of d of them, so it is off by at most
  ds = d 2^-23 sum |q k| scale + 2^-22 |s|   (the largest over the positions seen),
a weight by the factor e^ds, the two sums over the positions by (len / 16 + 64) 2^-23 (a lane adds one position in 16, then the joins).
  lse: ds + (len / 16 + 64) 2^-23 + 2^-22 |lse|
  out: half a bf16 step (2^-8) for the rounding of the weights and (2 ds + the sums) of sum p |v|, and half a bf16 step of the value."""
import math

import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
from attention_reference import Cache, attend64

pytestmark = pytest.mark.gpu
BF, F8 = si.SI_KV_BF16, si.SI_KV_E4M3
SCRATCH = {}


def scratch(n):
    """one piece of memory for all calls of this file: every call has to leave it fit for the next, whatever its shape"""
    if "t" not in SCRATCH or SCRATCH["t"].numel() < n:
        SCRATCH["t"] = torch.zeros(max(n, 1 << 24), dtype=torch.uint8, device="cuda")
    return SCRATCH["t"]


def filled(kind, lens, page, kv_heads, d, n_layers=1, layer=0, seed=0, scales=None, spare=3, max_pages=0, nan=True):
    """A cache with these sequences; in `layer`, what no token owns is NaN"""
    rng = np.random.default_rng(seed)
    need = [-(-x // page) for x in lens]
    n_pages = sum(need) + spare
    c = Cache(kind, n_pages, page, len(lens), max(max_pages, max(need + [1])), n_layers, kv_heads, d, scales, seed)
    order = rng.permutation(n_pages)
    at = 0
    bits = c.pages.view(torch.uint8 if kind == F8 else torch.int16)
    bad = 0x7f if kind == F8 else 0x7fc0
    if nan:
        bits[torch.from_numpy(order[sum(need):]).cuda()] = bad
    for s, x in enumerate(lens):
        pages = order[at:at + need[s]]
        at += need[s]
        c.give(s, [int(p) for p in pages], x)
        if nan and x % page:
            ik, iv = c.places(np.arange(x % page, page))
            last = bits[int(pages[-1]), layer]
            for h in range(kv_heads):
                last[0, h][torch.from_numpy(ik.ravel()).cuda()] = bad
                last[1, h][torch.from_numpy(iv.ravel()).cuda()] = bad
    return c


def call(c, q, lens, n_new, heads, window=0, layer=0, scale=0.0, seqs=None, pad=0, max_len=None, with_lse=True):
    """q: [n * n_new][heads * d + pad] bf16 on the GPU; returns out, lse as float64"""
    n = len(lens) if seqs is None else len(seqs)
    d = c.d
    out = torch.full((n * n_new, heads * d + pad), 99.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n * n_new, heads), 99.0, device="cuda")
    sq = torch.tensor(seqs, dtype=torch.int32, device="cuda") if seqs is not None else None
    desc = si.si_attend_t(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr() if with_lse else None, seqs=sq.data_ptr() if sq is not None else None,
                          q_stride=q.shape[1], out_stride=heads * d + pad, n=n, n_new=n_new, n_heads=heads, window=window,
                          max_len=max(lens + [0]) if max_len is None else max_len, scale=scale)
    desc.scratch_bytes = si.si_attend_scratch_bytes(c.desc, desc)
    if desc.scratch_bytes:
        desc.scratch = scratch(desc.scratch_bytes).data_ptr()
    print("attend", dict(kind=c.kind, lens=lens[:6], n=n, n_new=n_new, heads=heads, kv=c.kv_heads, d=d, page=c.page, window=window, scratch=desc.scratch_bytes), flush=True)
    si.si_attend(c.desc, layer, desc, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert pad == 0 or bool((out[:, heads * d:] == 99.0).all())
    return out[:, :heads * d].double().cpu().numpy().reshape(n, n_new, heads, d), lse.double().cpu().numpy().reshape(n, n_new, heads)


def compare(c, q, lens, n_new, heads, window, layer, scale, seqs, out, lse):
    d = c.d
    qq = q[:, :heads * d].double().cpu().numpy().reshape(-1, n_new, heads, d)
    sc = float(np.float32(scale)) if scale else 1.0 / math.sqrt(d)
    for i, s in enumerate(seqs if seqs is not None else range(len(lens))):
        k, v = c.gather(layer, s, lens[s])
        o, l, mag_s, mag_o = attend64(qq[i], k, v, n_new, window, sc)
        nothing = np.isneginf(l)
        assert np.array_equal(np.isneginf(lse[i]), nothing), "rows that see nothing"
        assert np.all(out[i][nothing] == 0)
        ds = d * 2.0 ** -23 * mag_s + 2.0 ** -22 * mag_s
        sums = (lens[s] / 16 + 64) * 2.0 ** -23
        ll = np.where(nothing, 0, l)
        assert np.all(np.abs(np.where(nothing, 0, lse[i]) - ll) <= ds + sums + 2.0 ** -22 * np.abs(ll)), np.max(np.abs(np.where(nothing, 0, lse[i]) - ll))
        tol = 2.0 ** -8 * np.abs(o) + 1.01 * (2.0 ** -8 + 2 * ds[..., None] + 2 * sums) * mag_o
        err = np.abs(out[i] - o)
        assert np.all(err <= tol), "sequence %d: worst %.3g of its tolerance" % (s, np.max(err / np.maximum(tol, 1e-30)))


def attend_case(kind, lens, n_new, heads, kv_heads, d, page, window=0, n_layers=1, layer=0, scale=0.0, seqs=None, pad=0, max_len=None, seed=0, spread=2.0):
    scales = (list(np.linspace(0.5, 1.5, kv_heads)), list(np.linspace(1.25, 0.75, kv_heads))) if kind == F8 else None
    c = filled(kind, lens, page, kv_heads, d, n_layers, layer, seed, scales)
    n = len(lens) if seqs is None else len(seqs)
    q = (torch.randn((n * n_new, heads * d + pad), generator=torch.Generator().manual_seed(seed + 7)) * spread).to(torch.bfloat16).cuda()
    out, lse = call(c, q, lens, n_new, heads, window, layer, scale, seqs, pad, max_len)
    assert int(c.status.item()) == 0
    compare(c, q, lens, n_new, heads, window, layer, scale, seqs, out, lse)
    return c


@pytest.mark.parametrize("kind,d", [(BF, 64), (BF, 96), (BF, 128), (BF, 192), (BF, 256), (F8, 64), (F8, 128), (F8, 192), (F8, 256)])
@pytest.mark.parametrize("rows", [(1, 1), (8, 1), (3, 5), (12, 2), (4, 8), (12, 5), (12, 8)])
def test_dims_and_rows(kind, d, rows):
    per, n_new = rows
    attend_case(kind, [0, 1, 5, 70, 300], n_new, 2 * per, 2, d, 64, seed=d + per)


@pytest.mark.parametrize("kind", [BF, F8])
def test_lengths_around_the_blocks(kind):
    B = 32 if kind == BF else 64
    lens = [0, 1, 2, B - 1, B, B + 1, 2 * B - 1, 2 * B, 4 * B + 1, 5 * B, 8 * B - 1, 8 * B + 1]
    for n_new in (1, 3):
        attend_case(kind, lens, n_new, 4, 1, 64, 2 * B, pad=5)
        attend_case(kind, lens, n_new, 4, 2, 128, 3 * B)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 65, 200, 5000])
@pytest.mark.parametrize("n_new", [1, 4])
def test_windows(kind, window, n_new):
    attend_case(kind, [0, 1, 3, 64, 65, 130, 700], n_new, 6, 2, 64, 64, window=window)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("n_new", [1, 6])
def test_long_sequences_split_over_blocks(kind, n_new):
    attend_case(kind, [9000], n_new, 8, 1, 128, 256)
    attend_case(kind, [4097, 0, 12, 2500, 1], n_new, 6, 2, 64, 64)
    attend_case(kind, [6000, 700], n_new, 4, 4, 128, 128, window=3000)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("n_new,heads", [(9, 16), (13, 20), (17, 16)])
def test_many_rows_over_long_sequences(kind, n_new, heads):
    """72, 130 and 136 rows a kv head: one block, and more, of 128 rows; pieces of a sequence from several blocks."""
    attend_case(kind, [3001], n_new, heads, 2, 128, 128)
    attend_case(kind, [2100, 0, 7, 1500, 1], n_new, heads, 2, 64, 64, window=1100)


@pytest.mark.parametrize("kind", [BF, F8])
def test_many_sequences_of_all_lengths(kind):
    lens = [(i * 379) % 1700 for i in range(41)]
    attend_case(kind, lens, 1, 8, 2, 64, 64)
    attend_case(kind, lens, 5, 8, 2, 128, 128)


def test_many_new_tokens():
    attend_case(BF, [100, 37, 400], 50, 8, 2, 64, 32)
    attend_case(F8, [300, 64], 65, 4, 2, 128, 64, window=40)


def test_short_sequences_with_more_new_tokens_than_they_hold():
    attend_case(BF, [0, 1, 2, 3, 4, 5], 5, 4, 2, 64, 32)
    attend_case(F8, [0, 1, 2, 3, 4, 5], 5, 4, 2, 64, 64, window=2)


def test_listed_sequences_layers_strides_and_scale():
    attend_case(BF, [40, 500, 77, 1200], 2, 4, 2, 64, 32, n_layers=3, layer=1, seqs=[3, 0, 3], pad=3, scale=0.25)
    attend_case(F8, [40, 500, 77], 1, 4, 2, 64, 64, n_layers=2, layer=1, seqs=[1, 2], pad=8, scale=-0.1)


def test_sequences_longer_than_max_len_are_still_whole():
    for max_len in (0, 1, 300):
        attend_case(BF, [3000, 10], 2, 4, 2, 64, 64, max_len=max_len)


def test_large_scores():
    attend_case(BF, [200, 1000], 1, 4, 2, 128, 64, spread=200.0)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_what_only_later_tokens_see_stays_out_of_earlier_ones(kind, what):
    """A drafted token with a value that is not finite: the tokens before it keep their results, it and those after it do not.  The same for a
    key, and for a token that only the first rows' windows reach."""
    if kind == F8 and what == "inf":
        pytest.skip("e4m3 has no infinity")
    n_new, heads, L = 4, 4, 203
    for which in (0, 1):
        for window, at, seen in ((0, L - 2, [2, 3]), (100, L - n_new + 1 - 100 + 1, [0, 1])):
            c = filled(kind, [L], 64, 1, 64, seed=3)
            q = (torch.randn((n_new, heads * 64), generator=torch.Generator().manual_seed(1)) * 2).to(torch.bfloat16).cuda()
            clean_out, clean_lse = call(c, q, [L], n_new, heads, window)
            page = int(c.table[0, at // 64])
            place = c.places([at % 64])[which][0][5]
            flat = c.pages.view(torch.uint8 if kind == F8 else torch.int16)
            flat[page, 0, which, 0, int(place)] = 0x7f if kind == F8 else (0x7f80 if what == "inf" else 0x7fc0)
            out, lse = call(c, q, [L], n_new, heads, window)
            others = [j for j in range(n_new) if j not in seen]
            assert np.array_equal(out[0, others], clean_out[0, others]) and np.array_equal(lse[0, others], clean_lse[0, others])
            if which == 1:
                bad = np.zeros(out[0].shape, bool)
                bad[seen, :, 5] = True
                assert np.array_equal(~np.isfinite(out[0]), bad)


def test_scores_of_minus_infinity_everywhere():
    """A key of -infinity against a positive query: the weight is 0; where that is all a row sees, so is the output."""
    c = filled(BF, [1, 40], 32, 1, 64)
    q = torch.ones((2, 64), dtype=torch.bfloat16, device="cuda")
    ik, _ = c.places([0])
    flat = c.pages.view(torch.int16)
    for s in (0, 1):
        flat[int(c.table[s, 0]), 0, 0, 0, int(ik[0][3])] = -128  # 0xff80
    out, lse = call(c, q, [1, 40], 1, 1)
    assert np.all(out[0] == 0) and np.isneginf(lse[0]).all()
    assert np.isfinite(out[1]).all() and np.isfinite(lse[1]).all()


@pytest.mark.parametrize("kind", [BF, F8])
def test_pages_outside_the_pool_are_not_seen(kind):
    lens, page = [256, 640], 64
    c = filled(kind, lens, page, 2, 64, nan=False)
    q = torch.randn((2, 4 * 64), device="cuda").to(torch.bfloat16)
    for entry in (-1, c.desc.n_pages, 0x7fffffff, -0x80000000):
        c.status.zero_()
        keep = int(c.table[1, 3])
        c.table[1, 3] = entry
        out, lse = call(c, q, lens, 1, 4)
        assert int(c.status.item()) == si.SI_CACHE_BAD_PAGE
        c.table[1, 3] = keep
        qq = q.double().cpu().numpy().reshape(2, 4, 64)
        k, v = c.gather(0, 1, 640)
        k, v = (np.delete(a, np.arange(192, 256), axis=1) for a in (k, v))
        o, l, _, _ = attend64(qq[1:2], k, v, 1, 0, 1 / 8.0)
        assert np.max(np.abs(lse[1] - l)) < 1e-3 and np.max(np.abs(out[1] - o)) < 0.05
        assert np.isfinite(out[0]).all()


def test_bad_sequences_and_lengths():
    c = filled(BF, [64, 64], 32, 1, 64, nan=False)
    q = torch.randn((3, 64), device="cuda").to(torch.bfloat16)
    for seqs in ([0, -1, 1], [0, 2, 1], [0, 0x7fffffff, 1]):
        c.status.zero_()
        out, lse = call(c, q, [64, 64], 1, 1, seqs=seqs)
        assert int(c.status.item()) == si.SI_CACHE_BAD_SEQ
        assert np.all(out[1] == 0) and np.isneginf(lse[1]).all() and np.isfinite(lse[[0, 2]]).all()
    for length in (-5, -0x80000000, 65, 0x7fffffff):
        c.status.zero_()
        c.lens[1] = length
        out, lse = call(c, q[:2], [64, 64], 1, 1)
        assert int(c.status.item()) == si.SI_CACHE_BAD_LEN
        assert np.isfinite(lse[0]).all() and np.isneginf(lse[1]).all() == (length < 0)


def test_a_recorded_call_follows_the_tables():
    """Replays of one recorded call as a sequence grows, eager calls between them."""
    c = filled(BF, [3000, 900], 64, 2, 64, max_pages=60)
    q = torch.randn((2, 8 * 64), device="cuda").to(torch.bfloat16)
    out, lse = torch.empty((2, 512), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 8), device="cuda")
    desc = si.si_attend_t(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), q_stride=512, out_stride=512, n=2, n_new=1, n_heads=8, max_len=3840)
    desc.scratch_bytes = si.si_attend_scratch_bytes(c.desc, desc)
    assert desc.scratch_bytes > 0
    desc.scratch = scratch(desc.scratch_bytes).data_ptr()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        si.si_attend(c.desc, 0, desc, torch.cuda.current_stream().cuda_stream)
    for step in range(4):
        lens = [3000 - 700 * step, 900 - step]
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got_out, got_lse = out.double().cpu().numpy().reshape(2, 1, 8, 64), lse.double().cpu().numpy().reshape(2, 1, 8)
        compare(c, q, lens, 1, 8, 0, 0, 0.0, None, got_out, got_lse)
        eager_out, eager_lse = call(c, q, lens, 1, 8, max_len=3840)
        assert np.array_equal(eager_out, got_out) and np.array_equal(eager_lse, got_lse)
        q.copy_(torch.randn((2, 512), device="cuda"))


def test_the_same_bits_every_time():
    c = filled(BF, [20000, 5000, 1], 64, 2, 128)
    q = torch.randn((3, 16 * 128), device="cuda").to(torch.bfloat16)
    first = call(c, q, [20000, 5000, 1], 1, 16)
    for _ in range(5):
        again = call(c, q, [20000, 5000, 1], 1, 16)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


def test_a_pool_beyond_32_bit_offsets():
    """Pages whose elements lie more than 2^32 bytes, and 2^31 elements, into the pool."""
    page, kv, d = 256, 8, 128
    n_pages = (5 << 30) // (2 * kv * page * d * 2) + 3
    c = Cache(BF, 1, page, 1, 2, 1, kv, d)
    c.pages = torch.zeros((n_pages, 1, 2, kv, page * d), dtype=torch.bfloat16, device="cuda")
    c.pages[-2:] = torch.randn(c.pages[-2:].shape, device="cuda").to(torch.bfloat16)
    c.desc.pages, c.desc.n_pages = c.pages.data_ptr(), n_pages
    c.table[0] = torch.tensor([n_pages - 1, n_pages - 2], dtype=torch.int32)
    c.lens[0] = 500
    q = torch.randn((1, 8 * 128), device="cuda").to(torch.bfloat16)
    out, lse = call(c, q, [500], 1, 8)
    small = Cache(BF, 2, page, 1, 2, 1, kv, d)
    small.pages = c.pages[-2:].clone()
    small.table[0] = torch.tensor([1, 0], dtype=torch.int32)
    compare(small, q, [500], 1, 8, 0, 0, 0.0, None, out, lse)


def test_no_sequences():
    c = filled(BF, [3], 32, 1, 64)
    q = torch.zeros((1, 64), dtype=torch.bfloat16, device="cuda")
    si.si_attend(c.desc, 0, si.si_attend_t(q=q.data_ptr(), out=q.data_ptr(), q_stride=64, out_stride=64, n=0, n_new=1, n_heads=1, max_len=3))
