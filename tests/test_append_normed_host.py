"""si_cache_append_normed on the CPU: what it refuses before any GPU call."""
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


def append(**kw):
    d = dict(q=BASE, k=BASE, v=BASE, q_out=BASE, seq=BASE, pos=BASE, inv_freq=BASE, q_stride=256, k_stride=256, v_stride=256, q_out_stride=256, n_tokens=3, n_heads=4, rot_dim=64)
    d.update(kw)
    return si.si_append_t(**d)


def norm(**kw):
    d = dict(w_q=BASE, b_q=BASE, w_k=BASE, b_k=BASE, w_type=si.SI_BF16, kind=si.SI_NORM_RMS, eps=1e-6)
    d.update(kw)
    return si.si_head_norm_t(**d)


def refused(c, layer, a, n):
    with pytest.raises(si.ScheInferError) as e:
        si.si_cache_append_normed(c, layer, a, n)
    assert e.value.code == si.SI_EINVAL and "si_cache_append_normed" in str(e.value)


@pytest.mark.parametrize("kw", [dict(kind=3), dict(kind=-1), dict(w_type=2), dict(w_type=-1), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(w_q=BASE + 1),
                                dict(b_k=BASE + 1), dict(w_type=si.SI_F32, w_k=BASE + 2), dict(w_type=si.SI_F32, b_q=BASE + 2)])
def test_bad_norms_are_refused(kw):
    refused(cache(), 0, append(), norm(**kw))


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(seq=None), dict(q_out=None), dict(n_heads=3), dict(n_heads=0), dict(rot_dim=63), dict(rot_dim=66), dict(rot_dim=-2),
                                dict(inv_freq=None), dict(q=BASE + 1), dict(pos=BASE + 2), dict(q_stride=255), dict(k_stride=127), dict(q_out_stride=0), dict(q_out_stride=512),
                                dict(n_tokens=-1), dict(n_tokens=(1 << 22) + 1)])
def test_bad_appends_are_refused(kw):
    refused(cache(), 0, append(**kw), norm())


def test_bad_caches_layers_and_missing_descriptors_are_refused():
    refused(cache(head_dim=80), 0, append(), norm())
    refused(cache(), 2, append(), norm())
    L = si.lib()
    assert L.si_cache_append_normed(None, 0, ctypes.byref(append()), ctypes.byref(norm()), None) == si.SI_EINVAL
    assert L.si_cache_append_normed(ctypes.byref(cache()), 0, None, ctypes.byref(norm()), None) == si.SI_EINVAL
    assert L.si_cache_append_normed(ctypes.byref(cache()), 0, ctypes.byref(append()), None, None) == si.SI_EINVAL


def test_no_tokens_is_a_no_op():
    si.si_cache_append_normed(cache(), 0, si.si_append_t(), norm())
