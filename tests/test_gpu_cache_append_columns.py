"""si_cache_append where a token's heads are shared by several blocks, and where a block has one to four tokens and runs of blocks go to one die: the
shapes of ordinary models.  Comparison and tolerances are those of test_gpu_cache_append.py.

A head has head_dim / 16 units (more where rot_dim is no multiple of 16); a block has 256 units, or 1024 from 256 tokens on."""
import pytest

import paper_2411_15715_amd as si
from test_gpu_cache_append import BF, F8, append_case, prompt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pairs", [False, True])
def test_few_tokens_of_320_units(kind, in_place, pairs):
    """8 single tokens of 32 + 8 heads of 128: two blocks a token."""
    scales = ([0.5 + 0.1 * i for i in range(8)], [1.5 - 0.1 * i for i in range(8)]) if kind == F8 else None
    append_case(kind, [(i, 300 * i + 7) for i in range(8)], 32, 8, 128, 64, 128, pairs, in_place=in_place, pad=16 * in_place, scales=scales)


@pytest.mark.parametrize("heads,kv_heads,d,rot,kind", [(33, 11, 96, 96, BF), (33, 11, 96, 32, BF), (24, 8, 64, 56, BF), (24, 8, 64, 56, F8), (48, 16, 64, 2, BF), (64, 1, 256, 256, F8),
                                                       (96, 8, 128, 120, BF), (16, 16, 192, 0, F8)])
@pytest.mark.parametrize("n", [3, 21])
def test_units_that_the_blocks_do_not_divide(heads, kv_heads, d, rot, kind, n):
    append_case(kind, prompt((0, 50, n), (1, 3, 2)), heads, kv_heads, d, 64, rot, in_place=n == 3, seed=rot)


@pytest.mark.parametrize("heads,kv_heads,d,rot,kind", [(6, 2, 128, 128, F8), (64, 8, 128, 128, F8), (128, 8, 128, 128, BF), (24, 8, 64, 56, BF), (36, 12, 128, 64, F8), (30, 10, 96, 96, BF),
                                                       (40, 8, 64, 64, F8), (15, 5, 256, 256, BF)])
def test_prompts(heads, kv_heads, d, rot, kind):
    """64 units a token (four a block), 576 (one), 1088 and 1152 (two blocks a token), 384 and 320 (two, three): several runs of blocks on each die."""
    append_case(kind, prompt((0, 9, 180), (1, 0, 130)), heads, kv_heads, d, 64, rot, seed=heads)


@pytest.mark.parametrize("kind", [BF, F8])
@pytest.mark.parametrize("n", [12, 300])
def test_a_token_without_a_place_among_many_blocks(kind, n):
    """Reported once, its queries 0 in every block, the others as ever."""
    toks = prompt((0, 0, n))
    toks[n // 2] = (1000, 0)
    toks[n // 3] = (-1, -1)
    append_case(kind, toks, 64, 8, 128, 64, 128, left_out=(n // 2, n // 3), want_status=si.SI_CACHE_BAD_SEQ)


def test_keys_and_values_only_of_many_heads():
    append_case(BF, prompt((0, 3, 20)), 32, 32, 128, 64, 128, with_q=False)
    append_case(F8, prompt((0, 3, 300)), 32, 32, 256, 64, 128, with_q=False)
