"""si_route_scored and layers that choose by scores, against the formulas in 64 bits.

Choices and tables have to be equal: both sides compare scores of 64 bits, whose errors (a few 2^-53 of a score) are some 10^8 times smaller than
the gaps between random fp32 logits.  Weights: one rounding to fp32, 2^-24 of the weight, and 2^-40 for the few of 64 bits before it."""
import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
import synth
from gpu_helpers import GpuLayer, assert_parity

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -24 + 2.0 ** -40
SIG, SOFT = si.SI_SCORE_SIGMOID, si.SI_SCORE_SOFTMAX


def scores64(x, score):
    x = x.astype(np.float64)
    with np.errstate(all="ignore"):
        if score == SIG:
            return 1 / (1 + np.exp(-x))
        top = x.max(1, keepdims=True)
        e = np.where(x == top, 1.0, np.exp(x - top))
        e = np.where(x == -np.inf, 0.0, e)
        total = e.sum(1, keepdims=True)
        return e / np.where(total == 0, 1.0, total)


def choose64(x, k, score=SOFT, bias=None, n_groups=0, top_groups=0, group_best=0, renorm=0, scale=0.0):
    """idx, w of every token, one at a time on Python floats"""
    s = scores64(x, score)
    T, E = x.shape
    c = s + (0.0 if bias is None else bias.astype(np.float64))
    key = np.where(np.isnan(c), -np.inf, c)
    nan = np.isnan(c)
    idx, w = np.zeros((T, k), np.int32), np.zeros((T, k))
    for t in range(T):
        worst_first = lambda e: (nan[t, e], -key[t, e], e)  # noqa: E731
        left = list(range(E))
        if n_groups > 1:
            n = E // n_groups
            worth = []
            for g in range(n_groups):
                best = sorted(range(g * n, g * n + n), key=worst_first)[:group_best]
                worth.append(sum(c[t, e] for e in best))
            order = sorted(range(n_groups), key=lambda g: (np.isnan(worth[g]), -worth[g] if not np.isnan(worth[g]) else 0, g))
            left = [e for g in order[:top_groups] for e in range(g * n, g * n + n)]
        chosen = sorted(left, key=worst_first)[:k]
        v = np.array([s[t, e] for e in chosen])
        total = v.sum()
        with np.errstate(all="ignore"):
            w[t] = (scale or 1.0) * (v if not renorm else v * 0 if total == 0 else v / total)
        idx[t] = chosen
    return idx, w


def route(x, k, bias=None, stream=None, **rule):
    T, E = x.shape
    lg = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    b = torch.from_numpy(bias).cuda() if bias is not None else None
    n = T * k
    out = {name: torch.full((m,), -7, dtype=torch.float32 if name == "w" else torch.int32, device="cuda")
           for name, m in (("idx", n), ("w", n), ("count", E), ("off", E + 1), ("perm", n), ("inv", n))}
    desc = si.si_score_t(bias=b.data_ptr() if b is not None else None, **rule)
    si.si_route_scored(lg.data_ptr(), T, E, k, desc, {name: t.data_ptr() for name, t in out.items()}, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return {name: t.cpu().numpy() for name, t in out.items()}


def check(x, k, bias=None, **rule):
    T, E = x.shape
    got = route(x, k, bias, **rule)
    idx, w = choose64(x, k, bias=bias, **rule)
    assert np.array_equal(got["idx"].reshape(T, k), idx)
    gw = got["w"].reshape(T, k).astype(np.float64)
    assert np.array_equal(np.isnan(gw), np.isnan(w))
    fine = ~np.isnan(w)
    assert np.all(np.abs(gw - w)[fine] <= HALF * np.abs(w[fine]) + 2.0 ** -149)
    flat = idx.reshape(-1)
    perm = np.argsort(flat, kind="stable")
    count = np.bincount(flat, minlength=E)
    assert np.array_equal(got["count"], count)
    assert np.array_equal(got["off"], np.concatenate(([0], np.cumsum(count))))
    assert np.array_equal(got["perm"], perm)
    assert np.array_equal(got["inv"], np.argsort(perm, kind="stable"))


RULES = {
    "softmax": dict(score=SOFT),
    "softmax_renorm": dict(score=SOFT, renorm=1, scale=2.5),
    "sigmoid": dict(score=SIG, scale=0.5),
    "sigmoid_bias": dict(score=SIG, renorm=1, scale=2.5),
}


@pytest.mark.parametrize("rule", sorted(RULES))
@pytest.mark.parametrize("T, E, k", [(1, 2, 1), (1, 8, 2), (1, 64, 8), (1, 256, 8), (5, 60, 4), (7, 65, 9), (8, 8, 8), (9, 128, 8), (64, 1, 1), (64, 17, 3), (65, 16, 2), (65, 256, 256), (129, 72, 6),
                                     (1500, 64, 8), (1031, 255, 12)])
def test_choices_and_weights(rule, T, E, k):
    rng = np.random.default_rng(T * 1009 + E * 31 + k)
    x = (1.5 * rng.standard_normal((T, E))).astype(np.float32)
    check(x, k, (0.1 * rng.standard_normal(E)).astype(np.float32) if rule == "sigmoid_bias" else None, **RULES[rule])


@pytest.mark.parametrize("T, E, k, n_groups, top_groups, group_best", [(1, 8, 2, 2, 1, 1), (3, 256, 8, 8, 4, 2), (70, 256, 8, 8, 4, 2), (33, 60, 4, 5, 2, 3), (66, 64, 6, 32, 3, 2), (9, 256, 3, 256, 3, 1),
                                                                       (9, 256, 5, 128, 100, 2), (65, 96, 32, 3, 1, 32), (6, 12, 12, 4, 4, 3), (2, 200, 7, 2, 2, 100)])
@pytest.mark.parametrize("score", [SOFT, SIG])
def test_groups(T, E, k, n_groups, top_groups, group_best, score):
    rng = np.random.default_rng(T + E + n_groups)
    x = (2.0 * rng.standard_normal((T, E))).astype(np.float32)
    rule = dict(score=score, n_groups=n_groups, top_groups=top_groups, group_best=group_best, renorm=1)
    check(x, k, (0.2 * rng.standard_normal(E)).astype(np.float32), **rule)
    check(x, k, None, **rule)


@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("E", [16, 256])
def test_ties_go_to_the_lower_expert_and_group(E, score):
    rng = np.random.default_rng(E)
    x = rng.integers(-2, 3, (67, E)).astype(np.float32)
    x[0] = 1.0
    x[1] = 80.0   # sigmoids of 1
    x[2] = -200.0  # and as good as 0
    check(x, 6, None, score=score, renorm=1)
    check(x, 6, None, score=score, n_groups=4, top_groups=2, group_best=2)
    # the bias alone decides, and brings scores that differ to the same sum
    bias = rng.integers(-1, 2, E).astype(np.float32)
    check(np.zeros((3, E), np.float32), 5, bias, score=score)


@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("groups", [dict(), dict(n_groups=4, top_groups=2, group_best=2)])
def test_masked_infinite_and_nan_logits(score, groups):
    rng = np.random.default_rng(5)
    E, k = 32, 6
    x = rng.standard_normal((70, E)).astype(np.float32)
    x[0] = -np.inf
    x[1, 4:] = -np.inf
    x[2, 7] = np.inf
    x[3, [5, 9]] = np.inf
    x[4, 3] = np.nan
    x[5] = np.nan
    x[6, 8] = np.finfo(np.float32).min
    x[7] = np.finfo(np.float32).min
    x[8, :30] = np.finfo(np.float32).max
    x[9, 0], x[9, 1] = -np.nan, np.inf
    for renorm in (0, 1):
        check(x, k, None, score=score, renorm=renorm, **groups)
        bias = np.zeros(E, np.float32)
        bias[20] = -np.inf
        check(x[10:], k, bias, score=score, renorm=renorm, **groups)
        check(x[:10], 1, bias, score=score, renorm=renorm, **groups)


def test_scores_closer_than_fp32_are_told_apart():
    """sums of a score and a bias that round to the same fp32"""
    x = np.zeros((1, 8), np.float32)
    x[0, 3] = 1e-6
    bias = np.full(8, 1000.0, np.float32)
    got = route(x, 1, bias, score=SIG)
    assert got["idx"].tolist() == [3]


def test_optional_outputs_may_be_left_out():
    x = np.random.default_rng(1).standard_normal((90, 16)).astype(np.float32)
    want = route(x, 3, None, score=SIG)
    lg = torch.from_numpy(x).cuda()
    idx, w = torch.empty(270, dtype=torch.int32, device="cuda"), torch.empty(270, device="cuda")
    si.si_route_scored(lg.data_ptr(), 90, 16, 3, si.si_score_t(score=SIG), {"idx": idx.data_ptr(), "w": w.data_ptr()}, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert np.array_equal(idx.cpu().numpy(), want["idx"]) and np.array_equal(w.cpu().numpy(), want["w"])


def test_another_stream_and_replays_of_a_graph():
    T, E, k = 130, 64, 6
    rng = np.random.default_rng(3)
    xs = [rng.standard_normal((T, E)).astype(np.float32) for _ in range(4)]
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
    rule = dict(score=SIG, n_groups=8, top_groups=3, group_best=2, renorm=1)
    want = [route(x, k, bias, **rule) for x in xs]
    lg, b = torch.from_numpy(xs[0]).cuda(), torch.from_numpy(bias).cuda()
    out = {name: torch.zeros(m, dtype=torch.float32 if name == "w" else torch.int32, device="cuda")
           for name, m in (("idx", T * k), ("w", T * k), ("count", E), ("off", E + 1), ("perm", T * k), ("inv", T * k))}
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        si.si_route_scored(lg.data_ptr(), T, E, k, si.si_score_t(bias=b.data_ptr(), **rule), {name: t.data_ptr() for name, t in out.items()}, torch.cuda.current_stream().cuda_stream)
    for i in (0, 1, 2, 3, 1):
        lg.copy_(torch.from_numpy(xs[i]))
        graph.replay()
        torch.cuda.synchronize()
        for name, t in out.items():
            assert np.array_equal(t.cpu().numpy(), want[i][name]), name


# ---------------------------------------------------------------- layers
def mlp64(x, g, u, d):
    a = x @ g.T
    return (a / (1 + np.exp(-a)) * (x @ u.T)) @ d


def layer64(x_bits, w, idx, wt, shared):
    f = synth.bf16_bits_to_f64
    x = f(x_bits)
    y = np.zeros_like(x)
    for e in np.unique(idx):
        t, s = np.nonzero(idx == e)
        y[t] += wt[t, s, None] * mlp64(x[t], f(w["w_gate"][e]), f(w["w_up"][e]), f(w["w_down"][e]))
    return y + mlp64(x, f(w["s_gate"]), f(w["s_up"]), f(w["s_down"])) if shared else y


CFG = synth.scaled(synth.CONFIGS["qwen_moe"], n_experts=16, top_k=4, d_model=256, d_ff=128, d_ff_shared=192)
RULE = dict(score=SIG, n_groups=4, top_groups=2, group_best=2, renorm=1, scale=1.5)


@pytest.fixture(scope="module")
def weights():
    return synth.make_weights(CFG)


@pytest.mark.parametrize("split", [(1.0, 0.0, 0.0), (0.5, 0.5, 0.0), (0.4, 0.2, 0.4)])
@pytest.mark.parametrize("T", [1, 2, 13, 90])
def test_a_layer_chooses_by_scores(weights, split, T):
    bias = (0.2 * np.random.default_rng(8).standard_normal(16)).astype(np.float32)
    b = torch.from_numpy(bias).cuda()
    x = synth.make_tokens(CFG, T)
    lg = synth.make_router_logits(CFG, x)
    L = GpuLayer(CFG, weights, split, max_tokens=96)
    try:
        before = L.forward(x, lg)
        si.si_layer_set_scores(L.h, si.si_score_t(bias=b.data_ptr(), **RULE))
        y, r = L.forward(x, lg, routing=True)
        idx, wt = choose64(lg, CFG.top_k, bias=bias, **RULE)
        assert np.array_equal(r["idx"], idx)
        assert np.all(np.abs(r["w"] - wt) <= HALF * wt)
        assert_parity(y, layer64(x, weights, idx, wt, True))
        # without asking for the tables, and back to the raw logits
        assert np.array_equal(L.forward(x, lg), y)
        si.si_layer_set_scores(L.h, None)
        assert np.array_equal(L.forward(x, lg), before)
    finally:
        L.close()


def test_layers_of_a_stack_choose_by_scores(weights):
    T = 6
    x = synth.make_tokens(CFG, T)
    lg = [synth.make_router_logits(CFG, synth.make_tokens(CFG, T, stream=s)) for s in (1, 2)]
    layers = [GpuLayer(CFG, weights, (0.5, 0.5, 0.0), max_tokens=8) for _ in range(2)]
    try:
        si.si_layer_set_scores(layers[1].h, si.si_score_t(**RULE))
        f = synth.bf16_bits_to_f32
        h = f(x) + layers[0].forward(x, lg[0])
        want = f(synth.f32_to_bf16_bits(h)) + layers[1].forward(synth.f32_to_bf16_bits(h), lg[1])
        stack = si.si_stack_create([m.h for m in layers])
        try:
            xd = torch.from_numpy(x.view(np.int16)).cuda()
            lgd = [torch.from_numpy(v).cuda() for v in lg]
            out = torch.empty((T, CFG.d_model), device="cuda")
            si.si_stack_forward(stack, xd.data_ptr(), [v.data_ptr() for v in lgd], T, 0, si.SI_AUTO, out.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            assert_parity(out.cpu().numpy(), want.astype(np.float64), tol=1e-5)
        finally:
            si.si_stack_destroy(stack)
    finally:
        for m in layers:
            m.close()


def test_layers_refuse_bad_scores(weights):
    L = GpuLayer(CFG, weights, (1.0, 0.0, 0.0), max_tokens=8)
    try:
        with pytest.raises(si.ScheInferError) as e:
            si.si_layer_set_scores(L.h, si.si_score_t(n_groups=8, top_groups=1, group_best=1))  # two experts for four choices
        assert e.value.code == si.SI_EINVAL
        x = synth.make_tokens(CFG, 3)
        lg = synth.make_router_logits(CFG, x)
        before = L.forward(x, lg)
        assert np.array_equal(L.forward(x, lg), before)
    finally:
        L.close()
    dense = synth.CONFIGS["tiny_dense"]
    L = GpuLayer(dense, synth.make_weights(dense), (1.0, 0.0, 0.0), max_tokens=8)
    try:
        with pytest.raises(si.ScheInferError) as e:
            si.si_layer_set_scores(L.h, si.si_score_t())
        assert e.value.code == si.SI_ESTATE
    finally:
        L.close()
