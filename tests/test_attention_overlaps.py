"""Outputs in the place of an input with another type or stride, on the CPU: refused, as rows would be written that others have still to read."""
import pytest

import paper_2411_15715_amd as si
from test_attention_host import BASE, append, cache, norm, refused

R, Y, G, W, O = (BASE + 4096 * i for i in range(5))


def base(**kw):
    return norm(**{**dict(r=R, y=Y, gate=G, gate_stride=64, gate_type=si.SI_BF16, w_pre=W, r_out=O, out=O + 2048, y_type=si.SI_F32), **kw})


@pytest.mark.parametrize("kw", [dict(out=Y), dict(r_out=Y), dict(out=R, out_type=si.SI_F32), dict(r_out=R, r_out_stride=65), dict(r_out=G, gate_stride=0), dict(out=G, gate_type=si.SI_F32),
                                dict(out=W), dict(out=Y, rows=1)])
def test_norm(kw):
    assert "address" in refused(si.si_norm, base(**kw))


def test_append():
    assert "q_out" in refused(si.si_cache_append, cache(), 0, append(q=R, k=Y, v=G, q_out=R, q_out_stride=260))
    assert "q_out" in refused(si.si_cache_append, cache(), 0, append(q=R, k=Y, v=G, q_out=R, q_stride=512))
