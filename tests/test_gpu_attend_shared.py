"""si_attend_shared against the formula in 64 bits, over caches whose sequences share leading pages and hold NaN wherever no token may look.

Tolerances are those of test_gpu_attend.py: the sums over shared and own positions are joined once more, which its 64 additions beside the positions' cover."""
import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
from attention_reference import Cache
from test_gpu_attend import BF, F8, compare
from test_gpu_attend import call as call_alone
from test_gpu_attend_weights import set_value

pytestmark = pytest.mark.gpu
SCRATCH = {}


@pytest.fixture(autouse=True)
def small_calls_by_pieces_too(monkeypatch):
    monkeypatch.setenv("SI_ATTEND_PIECES", "1")


def scratch(n):
    """one piece of memory for all calls of this file: every call has to leave it fit for the next, whatever its shape"""
    if "t" not in SCRATCH or SCRATCH["t"].numel() < n:
        SCRATCH["t"] = torch.zeros(max(n, 1 << 27), dtype=torch.uint8, device="cuda")
    return SCRATCH["t"]


def shared_cache(kind, groups, page, kv_heads, d, n_layers=1, layer=0, seed=0, scales=None, spare=3, shuffled=True):
    """groups: [(tokens that all share, [own tokens of each])].  Returns the cache, lens, and the rows of the table in list order"""
    rng = np.random.default_rng(seed)
    lens = [share + own for share, owns in groups for own in owns]
    common = [(share // page if len(owns) > 1 else 0) for share, owns in groups]
    need = sum(common) + sum(-(-(share + own) // page) - c for (share, owns), c in zip(groups, common) for own in owns)
    c = Cache(kind, need + spare, page, len(lens), max(1, max(-(-x // page) for x in lens)), n_layers, kv_heads, d, scales, seed)
    order = [int(p) for p in rng.permutation(need + spare)]
    rows = [int(r) for r in (rng.permutation(len(lens)) if shuffled else range(len(lens)))]
    bits = c.pages.view(torch.uint8 if kind == F8 else torch.int16)
    bad = 0x7f if kind == F8 else 0x7fc0
    at, i = 0, 0
    for (share, owns), m in zip(groups, common):
        first = order[at:at + m]
        at += m
        for own in owns:
            x = share + own
            more = -(-x // page) - m
            pages = first + order[at:at + more]
            at += more
            c.give(rows[i], pages, x)
            if x % page:
                ik, iv = c.places(np.arange(x % page, page))
                for h in range(kv_heads):
                    bits[pages[-1], layer, 0, h][torch.from_numpy(ik.ravel()).cuda()] = bad
                    bits[pages[-1], layer, 1, h][torch.from_numpy(iv.ravel()).cuda()] = bad
            i += 1
    bits[torch.tensor(order[at:], device="cuda")] = bad
    by_row = [0] * len(lens)
    for r, x in zip(rows, lens):
        by_row[r] = x
    return c, by_row, rows


def call(c, q, lens, seqs, n_new, heads, window=0, layer=0, scale=0.0, pad=0, max_len=None):
    n, d = len(seqs), c.d
    out = torch.full((n * n_new, heads * d + pad), 99.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n * n_new, heads), 99.0, device="cuda")
    sq = torch.tensor(seqs, dtype=torch.int32, device="cuda")
    desc = si.si_attend_t(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), seqs=sq.data_ptr(), q_stride=q.shape[1], out_stride=heads * d + pad, n=n, n_new=n_new, n_heads=heads,
                          window=window, max_len=max(lens + [0]) if max_len is None else max_len, scale=scale)
    desc.scratch_bytes = si.si_attend_shared_scratch_bytes(c.desc, desc)
    desc.scratch = scratch(desc.scratch_bytes).data_ptr()
    print("attend_shared", dict(kind=c.kind, n=n, n_new=n_new, heads=heads, kv=c.kv_heads, d=d, page=c.page, window=window, scratch=desc.scratch_bytes), flush=True)
    si.si_attend_shared(c.desc, layer, desc, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert pad == 0 or bool((out[:, heads * d:] == 99.0).all())
    return out[:, :heads * d].double().cpu().numpy().reshape(n, n_new, heads, d), lse.double().cpu().numpy().reshape(n, n_new, heads)


def run_case(kind, groups, n_new, heads, kv_heads, d, page, window=0, n_layers=1, layer=0, scale=0.0, pad=0, seed=0, spread=2.0, only=None, max_len=None, seqs=None):
    scales = (list(np.linspace(0.5, 1.5, kv_heads)), list(np.linspace(1.25, 0.75, kv_heads))) if kind == F8 else None
    c, lens, rows = shared_cache(kind, groups, page, kv_heads, d, n_layers, layer, seed, scales)
    rows = rows if seqs is None else [rows[i] for i in seqs]
    q = (torch.randn((len(rows) * n_new, heads * d + pad), generator=torch.Generator().manual_seed(seed + 7)) * spread).to(torch.bfloat16).cuda()
    out, lse = call(c, q, lens, rows, n_new, heads, window, layer, scale, pad, max_len)
    assert int(c.status.item()) == 0
    some = range(len(rows)) if only is None else [i for i in only if i < len(rows)]
    for i in some:
        compare(c, q[i * n_new:(i + 1) * n_new], lens, n_new, heads, window, layer, scale, [rows[i]], out[i:i + 1], lse[i:i + 1])
    return c


@pytest.mark.parametrize("kind,d", [(BF, 64), (BF, 96), (BF, 128), (BF, 192), (BF, 256), (F8, 64), (F8, 128), (F8, 192), (F8, 256)])
@pytest.mark.parametrize("rows", [(1, 1), (4, 1), (3, 5), (12, 2), (8, 8)])
def test_dims_and_rows(kind, d, rows):
    per, n_new = rows
    run_case(kind, [(200, [9, 70, 33]), (64, [20, 8]), (130, [150])], n_new, 2 * per, 2, d, 64, seed=d + per)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("n_new", [1, 4])
def test_groups_of_all_shapes(kind, n_new):
    page = 64
    run_case(kind, [(0, [0, 1, 3])], n_new, 4, 2, 64, page)
    run_case(kind, [(63, [5, 7]), (64, [4, 4]), (65, [6, 300]), (500, [4]), (0, [200, 17])], n_new, 4, 2, 64, page, pad=5)
    run_case(kind, [(128, [4] * 17), (256, [130] * 3), (0, [0]), (192, [4, 5, 0, 9])], n_new, 6, 2, 128, page)
    run_case(kind, [(1000, [0, 0, 64, 1])], n_new, 4, 1, 64, page)
    run_case(kind, [(700, [5])], n_new, 4, 1, 64, page)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("window", [1, 5, 64, 100, 333, 5000])
@pytest.mark.parametrize("n_new", [1, 3])
def test_windows_that_begin_in_shared_and_in_own_pages(kind, window, n_new):
    run_case(kind, [(400, [3, 90, 10, 200]), (130, [40, 4]), (64, [3, 500])], n_new, 6, 2, 64, 64, window=window)


@pytest.mark.parametrize("kind", [BF, F8])
def test_fewer_own_tokens_than_new_ones(kind):
    """the first of the new tokens does not see all of the common pages: fewer are attended to together"""
    run_case(kind, [(256, [0, 3, 64]), (128, [1, 2])], 70, 2, 1, 64, 64)
    run_case(kind, [(64, [0, 3, 1]), (0, [0, 2])], 5, 4, 2, 64, 64)


@pytest.mark.parametrize("kind,d", [(BF, 64), (BF, 128), (F8, 64), (F8, 128), (BF, 256)])
def test_long_shared_pages_split_over_blocks(kind, d):
    run_case(kind, [(6000, [5, 900, 33] * 5)], 1, 8, 2, d, 128, only=[0, 1, 7, 14])
    run_case(kind, [(2500, [5, 90] * 9), (3500, [40] * 7), (30, [2000])], 2, 12, 2, d, 64, only=[0, 17, 18, 24, 25])


@pytest.mark.parametrize("kind", [BF, F8])
def test_many_rows(kind):
    """more than 128 rows of a kv head in a group, and groups that end inside a block of rows"""
    run_case(kind, [(800, [3] * 50), (700, [9] * 13)], 1, 16, 2, 64, 64, only=[0, 15, 16, 31, 49, 50, 62])
    run_case(kind, [(800, [30] * 20)], 5, 18, 1, 128, 64, only=[0, 1, 2, 13, 19])


def test_many_sequences():
    """lists longer than a round of the plan, groups across its borders"""
    groups = [(64 * (1 + i % 3), [1 + (i * j) % 70 for j in range(1 + i % 7)]) for i in range(160)]
    run_case(BF, groups, 1, 2, 1, 64, 64, only=list(range(0, 640, 29)) + [255, 256, 257, 511, 512, 513])
    run_case(BF, [(128, [1 + i % 50 for i in range(700)])], 1, 2, 1, 64, 64, only=list(range(0, 700, 97)) + [255, 256, 511, 512, 699])


def test_more_sequences_than_the_plan_notes_in_shared_memory():
    groups = [(64 * (1 + i % 2), [1 + (i * j) % 70 for j in range(1 + i % 7)]) for i in range(240)] + [(64, [5] * 300)]
    run_case(BF, groups, 1, 2, 1, 64, 64, only=list(range(0, 1200, 61)) + [255, 256, 767, 768, 1023, 1024])


def test_the_same_sequence_several_times_and_prompts_within_prompts():
    run_case(BF, [(300, [5, 9]), (100, [3])], 2, 4, 2, 64, 64, seqs=[0, 0, 1, 1, 1, 2, 2, 0])
    # two long prompts that begin alike, forked: cut between them
    c, lens, rows = shared_cache(BF, [(1000, [3, 5, 9]), (900, [4, 8])], 64, 2, 64)
    for j in range(4):
        c.table[rows[3]:rows[3] + 1, j] = c.table[rows[0], j]
        c.table[rows[4]:rows[4] + 1, j] = c.table[rows[0], j]
    q = torch.randn((5, 4 * 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    out, lse = call(c, q, lens, rows, 1, 4)
    compare(c, q, lens, 1, 4, 0, 0, 0.0, rows, out, lse)


def test_layers_strides_scale_and_max_len():
    groups = [(200, [40, 5, 77]), (64, [1200, 1])]
    run_case(BF, groups, 2, 4, 2, 64, 32, n_layers=3, layer=1, pad=3, scale=0.25, seqs=[3, 0, 1, 3])
    run_case(F8, groups, 1, 4, 2, 64, 64, n_layers=2, layer=1, pad=8, scale=-0.1)
    for max_len in (0, 1, 300, 100000):
        run_case(BF, groups, 2, 4, 2, 64, 64, max_len=max_len)
    run_case(BF, groups, 1, 4, 2, 128, 64, spread=200.0)


@pytest.mark.parametrize("kind", [BF, F8])
def test_nothing_shared(kind):
    run_case(kind, [(0, [500]), (0, [3]), (0, [0]), (0, [1200])], 2, 8, 2, 64, 64)
    run_case(kind, [(0, [77]), (0, [4000])], 1, 4, 1, 128, 64)


def test_pages_outside_the_pool_and_bad_sequences():
    groups = [(256, [5, 70, 9])]
    for entry in (-1, 1 << 20, 0x7fffffff, -0x80000000):
        c, lens, rows = shared_cache(BF, groups, 64, 2, 64, shuffled=False)
        c.table[:, 2] = entry
        q = torch.randn((3, 4 * 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
        got, want = call(c, q, lens, rows, 1, 4), call_alone(c, q, lens, 1, 4, seqs=rows)
        assert int(c.status.item()) == si.SI_CACHE_BAD_PAGE
        assert np.max(np.abs(got[0] - want[0])) < 0.03 and np.max(np.abs(got[1] - want[1])) < 1e-4
    for seqs, bit in (([0, -1, 1, 2], si.SI_CACHE_BAD_SEQ), ([0, 1, 9, 2], si.SI_CACHE_BAD_SEQ), ([0x7fffffff, 0, 1, 2], si.SI_CACHE_BAD_SEQ)):
        c, lens, rows = shared_cache(BF, groups, 64, 2, 64, shuffled=False)
        q = torch.randn((4, 4 * 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
        out, lse = call(c, q, lens, seqs, 1, 4)
        assert int(c.status.item()) == bit
        for i, s in enumerate(seqs):
            if 0 <= s < 3:
                compare(c, q[i:i + 1], lens, 1, 4, 0, 0, 0.0, [s], out[i:i + 1], lse[i:i + 1])
            else:
                assert np.all(out[i] == 0) and np.isneginf(lse[i]).all()
    for length in (-5, -0x80000000, 100000, 0x7fffffff):
        c, lens, rows = shared_cache(BF, groups, 64, 2, 64, shuffled=False)
        c.lens[1] = length
        q = torch.randn((3, 4 * 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
        out, lse = call(c, q, lens, rows, 1, 4)
        assert int(c.status.item()) & si.SI_CACHE_BAD_LEN
        for s in (0, 2):
            compare(c, q[s:s + 1], lens, 1, 4, 0, 0, 0.0, [s], out[s:s + 1], lse[s:s + 1])


@pytest.mark.parametrize("length", [321, 100000, 0x7fffffff])
def test_lengths_beyond_the_table_are_cut_under_windows_too(length):
    c, lens, rows = shared_cache(BF, [(256, [5, 64, 9])], 64, 2, 64, shuffled=False)
    c.lens[1] = length  # (its 320 tokens fill the table)
    q = torch.randn((3, 4 * 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    out, lse = call(c, q, lens, rows, 1, 4, window=100)
    assert int(c.status.item()) == si.SI_CACHE_BAD_LEN
    compare(c, q, lens, 1, 4, 100, 0, 0.0, rows, out, lse)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("per,n_new", [(4, 1), (6, 2), (8, 6)])
def test_values_that_are_not_finite(kind, per, n_new):
    """In a shared page: in the element of every row that sees it and nowhere else, under a window in the rows of those tokens only."""
    groups = [(640, [100, 20, 60, 9]), (300, [50, 40])]
    nan = 0x7f if kind == F8 else 0x7fc0
    for window, at in ((0, 333), (300, 400), (150, 600)):
        c, lens, rows = shared_cache(kind, groups, 64, 2, 64)
        q = (torch.randn((6 * n_new, 2 * per * 64), generator=torch.Generator().manual_seed(1)) * 0.3).to(torch.bfloat16).cuda()
        clean_out, clean_lse = call(c, q, lens, rows, n_new, 2 * per, window)
        set_value(c, rows[0], at, 5, nan, head=1)
        out, lse = call(c, q, lens, rows, n_new, 2 * per, window)
        sees = np.array([[i < 4 and (window == 0 or at > lens[r] - n_new + j - window) for j in range(n_new)] for i, r in enumerate(rows)])
        assert sees.any()
        assert np.array_equal(np.isnan(out[:, :, per:, 5]), np.broadcast_to(sees[:, :, None], (6, n_new, per)))
        out[:, :, per:, 5] = clean_out[:, :, per:, 5]
        assert np.array_equal(out, clean_out) and np.array_equal(lse, clean_lse)


def test_scores_of_plus_and_minus_infinity_in_shared_pages():
    c, lens, rows = shared_cache(BF, [(640, [10, 70, 9])], 64, 1, 64)
    q = (torch.randn((3, 2 * 64), generator=torch.Generator().manual_seed(3)) * 0.3).to(torch.bfloat16).cuda()
    q.view(3, 2, 64)[:, 0, 7], q.view(3, 2, 64)[:, 1, 7] = 1.0, -1.0
    set_value(c, rows[0], 100, 7, 0x7f80, which=0)
    out, lse = call(c, q, lens, rows, 1, 2)
    assert np.isposinf(lse[:, 0, 0]).all() and np.isnan(out[:, 0, 0]).all()
    assert np.isfinite(lse[:, 0, 1]).all() and np.isfinite(out[:, 0, 1]).all()
    # every shared score -infinity: what is left are the own tokens
    c, lens, rows = shared_cache(BF, [(64, [10, 70, 9])], 64, 1, 64)
    q = torch.ones((3, 64), dtype=torch.bfloat16, device="cuda")
    for t in range(64):
        set_value(c, rows[0], t, 3, -128, which=0)
    out, lse = call(c, q, lens, rows, 1, 1)
    want_out, want_lse = call_alone(c, q, lens, 1, 1, seqs=rows)
    assert np.max(np.abs(out - want_out)) < 0.03 and np.max(np.abs(lse - want_lse)) < 1e-4


def test_the_same_bits_every_time_and_one_scratch_with_si_attend():
    c, lens, rows = shared_cache(BF, [(5000, [40] * 9), (900, [7, 3000])], 64, 2, 128)
    q = torch.randn((11, 16 * 128), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    first = call(c, q, lens, rows, 1, 16)
    for i in range(5):
        desc = si.si_attend_t(q=q.data_ptr(), out=torch.empty_like(q).data_ptr(), q_stride=2048, out_stride=2048, n=11, n_new=1, n_heads=16, max_len=max(lens))
        out = torch.empty_like(q)
        desc.out, desc.scratch_bytes = out.data_ptr(), scratch(0).numel()
        desc.scratch = scratch(0).data_ptr()
        si.si_attend(c.desc, 0, desc, torch.cuda.current_stream().cuda_stream)
        again = call(c, q, lens, rows, 1, 16)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


def test_which_calls_are_si_attend(monkeypatch):
    """small ones by max_len are, to the bit; larger ones plan their pieces, which the order of their sums tells"""
    c, lens, rows = shared_cache(BF, [(900, [7, 300, 40, 5, 20])], 64, 2, 64)
    q = torch.randn((5, 8 * 64), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    pieces = call(c, q, lens, rows, 1, 8)
    monkeypatch.delenv("SI_ATTEND_PIECES")
    small, large = call(c, q, lens, rows, 1, 8), call(c, q, lens, rows, 1, 8, max_len=1 << 20)
    alone = call_alone(c, q, lens, 1, 8, seqs=rows)
    assert np.array_equal(small[0], alone[0]) and np.array_equal(small[1], alone[1])
    assert not np.array_equal(pieces[1], alone[1]) and not np.array_equal(large[1], alone[1])
    for out, lse in (small, large, pieces):
        compare(c, q, lens, 1, 8, 0, 0, 0.0, rows, out, lse)
    windowed = call(c, q, lens, rows, 1, 8, window=100, max_len=1 << 20)
    alone = call_alone(c, q, lens, 1, 8, window=100, seqs=rows, max_len=1 << 20)
    assert np.array_equal(windowed[0], alone[0]) and np.array_equal(windowed[1], alone[1])


def test_a_recorded_call_follows_forks():
    """Replays of one recorded call as sequences are forked anew and grow, eager calls between them."""
    c = Cache(BF, 80, 64, 6, 20, 1, 2, 64)
    c.scratch = torch.zeros(si.si_cache_scratch_bytes(c.desc), dtype=torch.uint8, device="cuda")
    c.desc.scratch = c.scratch.data_ptr()
    stream = torch.cuda.current_stream().cuda_stream
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.randn((4, 8 * 64), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    out, lse, seqs = torch.empty((4, 512), dtype=torch.bfloat16, device="cuda"), torch.empty((4, 8), device="cuda"), dev([2, 3, 4, 5])
    desc = si.si_attend_t(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), seqs=seqs.data_ptr(), q_stride=512, out_stride=512, n=4, n_new=1, n_heads=8, max_len=1280)
    desc.scratch_bytes = si.si_attend_shared_scratch_bytes(c.desc, desc)
    mine = torch.zeros(desc.scratch_bytes, dtype=torch.uint8, device="cuda")
    desc.scratch = mine.data_ptr()
    roots, first = dev([0, 1]), dev([700, 333])
    si.si_cache_extend(c.desc, roots.data_ptr(), 2, first.data_ptr(), 0, None, None, 0, stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        si.si_attend_shared(c.desc, 0, desc, torch.cuda.current_stream().cuda_stream)
    for parents, grow in (([0, 0, 0, 0], 1), ([0, 0, 1, 1], 40), ([0, 1, 0, 1], 3), ([1, 1, 1, 0], 70)):
        par, counts = dev(parents), dev([grow] * 4)
        si.si_cache_trim(c.desc, seqs.data_ptr(), 4, None, stream)
        si.si_cache_fork(c.desc, par.data_ptr(), seqs.data_ptr(), 4, stream)
        si.si_cache_extend(c.desc, seqs.data_ptr(), 4, counts.data_ptr(), 0, None, None, 0, stream)
        graph.replay()
        torch.cuda.synchronize()
        assert int(c.status.item()) == 0
        lens = c.lens.tolist()
        got = out.double().cpu().numpy().reshape(4, 1, 8, 64), lse.double().cpu().numpy().reshape(4, 1, 8)
        compare(c, q, lens, 1, 8, 0, 0, 0.0, [2, 3, 4, 5], *got)
        eager = call(c, q, lens, [2, 3, 4, 5], 1, 8, max_len=1280)
        assert all(np.array_equal(a, b) for a, b in zip(got, eager))
        q.copy_(torch.randn((4, 512), device="cuda"))


def test_no_sequences_and_no_list():
    c, lens, rows = shared_cache(BF, [(128, [3, 9])], 64, 1, 64, shuffled=False)
    q = torch.randn((2, 64), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
    si.si_attend_shared(c.desc, 0, si.si_attend_t(q_stride=64, out_stride=64, n=0, n_new=1, n_heads=1, max_len=3))
    want = call(c, q, lens, [0, 1], 1, 1)
    out = torch.empty_like(q)
    desc = si.si_attend_t(q=q.data_ptr(), out=out.data_ptr(), q_stride=64, out_stride=64, n=2, n_new=1, n_heads=1, max_len=200)
    desc.scratch_bytes = si.si_attend_shared_scratch_bytes(c.desc, desc)
    desc.scratch = scratch(desc.scratch_bytes).data_ptr()
    si.si_attend_shared(c.desc, 0, desc, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert np.array_equal(out.double().cpu().numpy().reshape(2, 1, 1, 64), want[0])
