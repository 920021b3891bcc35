"""si_cache_append_normed where a block has several tokens (long prompts) and where a token's heads are several blocks' (many heads), against 64 bits; tolerances as in
test_gpu_cache_append_normed.py."""
import pytest

from test_gpu_cache_append_normed import BF, F8, MEAN, RMS, prompt, run_case

pytestmark = pytest.mark.gpu
ONE, TWO = ([0.5], [0.25]), ([0.07, 0.13], [1.1, 0.25])


@pytest.mark.parametrize("n", [1919, 1920, 1921, 2885, 3843])
@pytest.mark.parametrize("per_head", [False, True])
def test_blocks_of_one_to_four_tokens(n, per_head):
    """the last block of a call has fewer"""
    run_case(BF, prompt((0, 7, n)), 2, 1, 64, 64, 64, per_head=per_head, bias=per_head, seed=n)
    run_case(F8, prompt((0, 0, n)), 3, 1, 128, 64, 32, norm=MEAN, per_head=per_head, weights="f32", seed=n, scales=ONE)


@pytest.mark.parametrize("n", [1930, 3843])
@pytest.mark.parametrize("rot, pairs", [(0, False), (10, False), (34, False), (96, False), (96, True), (50, True)])
def test_rotated_parts(n, rot, pairs):
    run_case(BF, prompt((0, 1000, n - 500), (1, 3, 500)), 2, 2, 96, 32, rot, pairs, in_place=True, pad=3, seed=rot)


@pytest.mark.parametrize("kind, d", [(BF, 192), (BF, 256), (F8, 64), (F8, 192), (F8, 256)])
def test_dims(kind, d):
    run_case(kind, prompt((0, 0, 2000), (1, 64, 900)), 2, 2, d, 64, d // 2, norm=RMS, bias=True, scales=TWO if kind == F8 else None, seed=d)


def test_tokens_left_out_inside_blocks_and_no_q():
    tokens = prompt((0, 0, 3000))
    gone = tuple(i for i in range(3000) if i % 7 == 3 or 1500 <= i < 1530)
    run_case(BF, [(-1, p) if i in gone else (s, p) for i, (s, p) in enumerate(tokens)], 2, 1, 64, 32, 64, left_out=gone)
    run_case(F8, prompt((0, 20, 3000)), 4, 2, 64, 64, 32, n_layers=2, layer=1, with_q=False)


@pytest.mark.parametrize("heads, kv_heads, d", [(140, 7, 256), (290, 10, 256), (280, 8, 128), (600, 24, 64)])
@pytest.mark.parametrize("n", [5, 255, 256, 301])
def test_heads_of_a_token_over_several_blocks(heads, kv_heads, d, n):
    run_case(BF, prompt((0, 0, n)), heads, kv_heads, d, 32, d, seed=n)
    if n in (5, 256):
        run_case(F8, prompt((0, 3, n)), heads, kv_heads, d, 64, 20, norm=MEAN, per_head=True, bias=True, seed=n, scales=([0.5] * kv_heads, [0.25] * kv_heads))
