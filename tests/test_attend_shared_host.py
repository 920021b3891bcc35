"""si_attend_shared on the CPU: what it refuses before any GPU call, and the size of its scratch."""
import ctypes

import numpy as np
import pytest

import paper_2411_15715_amd as si

BUF = np.zeros(1 << 16, np.uint8)
BASE = (BUF.ctypes.data + 255) // 256 * 256


def cache(**kw):
    d = dict(pages=BASE, table=BASE, lens=BASE, refs=BASE, status=BASE, n_pages=4, page_tokens=64, n_layers=2, n_kv_heads=2, head_dim=64, type=si.SI_KV_BF16, n_seqs=2, max_pages=2)
    d.update(kw)
    return si.si_cache_t(**d)


def attend(**kw):
    d = dict(q=BASE, out=BASE, lse=BASE, seqs=BASE, scratch=BASE, scratch_bytes=1 << 50, q_stride=256, out_stride=256, n=2, n_new=1, n_heads=4, max_len=100)
    d.update(kw)
    return si.si_attend_t(**d)


def refused(f, *args):
    with pytest.raises(si.ScheInferError) as e:
        f(*args)
    assert e.value.code == si.SI_EINVAL and "si_attend_shared" in str(e.value)


@pytest.mark.parametrize("kw", [dict(n=-1), dict(n=65536), dict(n_new=0), dict(n_new=65537), dict(n_heads=3), dict(n_heads=0), dict(n_heads=4098), dict(window=-1), dict(max_len=-1),
                                dict(scale=float("nan")), dict(n=65535, n_new=65536), dict(n=60000, n_new=9, n_heads=4096)])
def test_bad_shapes_are_refused(kw):
    refused(si.si_attend_shared, cache(), 0, attend(**kw))
    refused(si.si_attend_shared_scratch_bytes, cache(), attend(**kw))


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(q=BASE + 1), dict(out=BASE + 1), dict(lse=BASE + 2), dict(seqs=BASE + 2), dict(q_stride=255), dict(out_stride=255),
                                dict(seqs=None, n=3), dict(scratch=None), dict(scratch=BASE + 8), dict(scratch_bytes=1000)])
def test_bad_pointers_strides_and_scratch_are_refused(kw):
    refused(si.si_attend_shared, cache(), 0, attend(**kw))


def test_bad_caches_layers_and_missing_descriptors_are_refused():
    refused(si.si_attend_shared, cache(page_tokens=48), 0, attend())
    refused(si.si_attend_shared, cache(), 2, attend())
    L = si.lib()
    assert L.si_attend_shared(None, 0, ctypes.byref(attend()), None) == si.SI_EINVAL
    assert L.si_attend_shared(ctypes.byref(cache()), 0, None, None) == si.SI_EINVAL


def test_calls_that_are_never_in_pieces_need_no_scratch_for_them():
    """one sequence, and rows beyond what a plan takes; but what serves a list serves the shorter ones that are planned"""
    c = cache(head_dim=128, n_kv_heads=8, n_seqs=4096, max_pages=4096)
    one = attend(n=1, n_new=65536, n_heads=1024, max_len=100000)
    assert si.si_attend_shared_scratch_bytes(c, one) == si.si_attend_scratch_bytes(c, one)
    most = si.si_attend_shared_scratch_bytes(c, attend(n=4000, n_new=100, n_heads=64, max_len=5000))
    assert most < 2 << 30
    many = cache(head_dim=128, n_kv_heads=1024, n_seqs=4096, max_pages=4096)
    assert si.si_attend_shared_scratch_bytes(many, attend(n=4000, n_new=16, n_heads=1024, max_len=5000)) < 3 << 30
    for n in (2, 50, 81, 82, 1000, 3999):
        a = attend(n=n, n_new=100, n_heads=64, max_len=5000)
        assert si.si_attend_scratch_bytes(c, a) <= si.si_attend_shared_scratch_bytes(c, a) <= most


def test_no_sequences_is_a_no_op():
    si.si_attend_shared(cache(), 0, attend(n=0, q=None, out=None, scratch=None, scratch_bytes=0))


@pytest.mark.parametrize("kind,d", [(si.SI_KV_BF16, 64), (si.SI_KV_BF16, 128), (si.SI_KV_BF16, 256), (si.SI_KV_E4M3, 64), (si.SI_KV_E4M3, 128)])
def test_scratch_serves_smaller_calls_and_si_attend(kind, d):
    c = cache(type=kind, head_dim=d, n_kv_heads=8, n_seqs=4096, max_pages=4096)
    for n_new, heads, window in ((1, 32, 0), (5, 64, 9000), (3, 8, 0)):
        most = si.si_attend_shared_scratch_bytes(c, attend(n=200, n_new=n_new, n_heads=heads, window=window, max_len=100000))
        for n in (0, 1, 2, 7, 33, 100, 200):
            for max_len in (0, 1, 500, 640, 641, 5000, 100000):
                a = attend(n=n, n_new=n_new, n_heads=heads, window=window, max_len=max_len)
                assert si.si_attend_scratch_bytes(c, a) <= si.si_attend_shared_scratch_bytes(c, a) <= most
