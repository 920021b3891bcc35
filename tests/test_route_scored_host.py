"""si_route_scored and si_layer_set_scores on the CPU: what they refuse before any GPU call, and calls with nothing to do."""
import ctypes

import numpy as np
import pytest

import paper_2411_15715_amd as si

BUF = np.zeros(1 << 12, np.uint8)
BASE = (BUF.ctypes.data + 255) // 256 * 256
ALL = {"idx": BASE, "w": BASE, "count": BASE, "off": BASE, "perm": BASE, "inv": BASE}


def refused(f, *args):
    with pytest.raises(si.ScheInferError) as e:
        f(*args)
    assert e.value.code == si.SI_EINVAL and len(str(e.value)) > 25
    return str(e.value)


GROUPS = dict(n_groups=4, top_groups=2, group_best=2)


@pytest.mark.parametrize("kw", [dict(score=2), dict(score=-1), dict(bias=BASE + 2), dict(scale=float("nan")), dict(scale=float("inf")), dict(n_groups=-1), dict(GROUPS, n_groups=3),
                                dict(GROUPS, n_groups=32), dict(GROUPS, top_groups=0), dict(GROUPS, top_groups=5), dict(GROUPS, group_best=0), dict(GROUPS, group_best=5),
                                dict(GROUPS, top_groups=1)])
def test_bad_scores_are_refused(kw):
    assert "si_route_scored" in refused(si.si_route_scored, BASE, 3, 16, 5, si.si_score_t(**kw), ALL)


@pytest.mark.parametrize("T, E, k", [(-1, 16, 2), ((1 << 24) + 1, 16, 2), (1 << 24, 256, 128), (14221746, 151, 151), (1 << 23, 256, 129), (3, 0, 1), (3, 257, 2), (3, 16, 0), (3, 16, 17)])
def test_bad_sizes_are_refused(T, E, k):
    refused(si.si_route_scored, BASE, T, E, k, si.si_score_t(), ALL)


@pytest.mark.parametrize("name", ["idx", "w", "count", "off", "perm", "inv"])
def test_bad_outputs_are_refused(name):
    refused(si.si_route_scored, BASE, 3, 16, 2, si.si_score_t(), dict(ALL, **{name: BASE + 2}))
    if name in ("idx", "w"):
        refused(si.si_route_scored, BASE, 3, 16, 2, si.si_score_t(), dict(ALL, **{name: None}))


def test_null_pointers_are_refused():
    L, rout = si.lib(), si.si_routing_out_t(*[BASE] * 6)
    refused(si.si_route_scored, None, 3, 16, 2, si.si_score_t(), ALL)
    refused(si.si_route_scored, BASE + 1, 3, 16, 2, si.si_score_t(), ALL)
    assert L.si_route_scored(BASE, 3, 16, 2, None, ctypes.byref(rout), None) == si.SI_EINVAL
    assert L.si_route_scored(BASE, 3, 16, 2, ctypes.byref(si.si_score_t()), None, None) == si.SI_EINVAL
    assert L.si_layer_set_scores(None, ctypes.byref(si.si_score_t())) == si.SI_EINVAL


def test_no_tokens_is_a_no_op():
    si.si_route_scored(None, 0, 16, 2, si.si_score_t(), {})
    si.si_route_scored(None, 0, 16, 2, si.si_score_t(**GROUPS), ALL)
