"""The operators around the feed-forward layer, on the CPU: what their entry points refuse before any GPU call."""
import ctypes

import numpy as np
import pytest

import paper_2411_15715_amd as si

BUF = np.zeros(1 << 16, np.uint8)
BASE = (BUF.ctypes.data + 255) // 256 * 256


def refused(f, *args):
    with pytest.raises(si.ScheInferError) as e:
        f(*args)
    assert e.value.code == si.SI_EINVAL and len(str(e.value)) > 25
    return str(e.value)


def norm(**kw):
    d = dict(r=BASE, y=BASE, w_pre=BASE, r_out=BASE, out=BASE, r_stride=64, y_stride=64, r_out_stride=64, out_stride=64, rows=2, d=64, eps=1e-5,
             r_type=si.SI_BF16, y_type=si.SI_F32, w_type=si.SI_BF16, r_out_type=si.SI_BF16, out_type=si.SI_BF16, pre=si.SI_NORM_RMS, res_scale=1.0,
             y_scale=1.0)
    d.update(kw)
    return si.si_norm_t(**d)


@pytest.mark.parametrize("kw", [dict(r=None, y=None), dict(r_out=None, out=None), dict(rows=-1), dict(d=0), dict(d=si.SI_NORM_MAX_D + 1, r_stride=1 << 20),
                                dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(pre=3), dict(post=-1), dict(post=1, y=None),
                                dict(r_type=2), dict(w_type=-1), dict(y=BASE + 2), dict(r=BASE + 1), dict(r_stride=-64), dict(out_stride=63), dict(r_out_stride=0),
                                dict(gate=BASE, gate_stride=-1), dict(gate=BASE, gate_type=9)])
def test_norm_refuses(kw):
    assert "si_norm" in refused(si.si_norm, norm(**kw))


def test_norm_refuses_no_descriptor_and_takes_no_rows():
    assert si.lib().si_norm(None, None) == si.SI_EINVAL
    si.si_norm(norm(rows=0))
