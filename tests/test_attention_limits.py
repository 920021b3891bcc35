"""How large a call of the attention's operators may be, on the CPU."""
import pytest

import paper_2411_15715_amd as si
from test_attention_host import BASE, append, attend, cache, refused


def big_cache(**kw):
    return cache(**{**dict(n_pages=1 << 20, max_pages=1 << 12, n_seqs=65535, n_kv_heads=8, head_dim=128), **kw})


@pytest.mark.parametrize("n,n_new,n_heads", [(64, 4096, 64), (32, 8192, 64), (4, 65536, 64), (1, 65536, 256), (16384, 5, 128), (65535, 1, 64)])
@pytest.mark.parametrize("max_len", [600, 70000])
def test_prompts_and_batches_are_not_too_large(n, n_new, n_heads, max_len):
    """No launch holds a joining block for each of these rows, and none is needed."""
    row = n_heads * 128
    assert si.si_attend_scratch_bytes(big_cache(), attend(n=n, n_new=n_new, n_heads=n_heads, max_len=max_len, q_stride=row, out_stride=row)) >= 0


@pytest.mark.parametrize("kw", [dict(n=65535, n_new=65536, n_heads=64, max_len=600), dict(n=65535, n_new=1024, n_heads=64, max_len=70000), dict(n=32768, n_new=512, n_heads=64),
                                dict(n=32768, n_new=8, n_heads=4096, max_len=5)])
def test_more_blocks_than_a_launch_holds(kw):
    assert "too large" in refused(si.si_attend_scratch_bytes, big_cache(), attend(**kw))


@pytest.mark.parametrize("kw", [dict(n_tokens=2_000_000, n_heads=64, rot_dim=254), dict(n_tokens=1 << 22, n_heads=1024, rot_dim=256), dict(n_tokens=1 << 21, n_heads=4096, rot_dim=0)])
def test_tokens_and_heads_for_more_blocks_than_a_launch_holds(kw):
    row = kw["n_heads"] * 256
    c = big_cache(n_kv_heads=1, head_dim=256)
    assert "too many tokens and heads" in refused(si.si_cache_append, c, 0, append(q_stride=row, q_out_stride=row, k_stride=256, v_stride=256, **kw))
