"""Expert scores, head norms, shared attention and sampling together, as examples/many_answers.py uses them: a two-layer model against its definition in 64 bits.

Tolerance: the largest error of the logits against their RMS.  A layer takes the feed-forward layer's own bound (2e-2) and, on the way from one residual
to the next, six roundings to bf16 (norm, projection, rotation, weights, attention, output) and two more for the experts' weights, whose scores come of a rounded
input, 2^-8 each, counted as if they all added up: 2 layers of 2e-2 + 8 / 256, the last norm and the logits' own product 2 / 256, in all 0.11.
Which experts are chosen can hang on a rounding: the definition takes the choice that was made, which has to be within 0.06 of the best
scores (the logits of the router have an RMS of 1 and an error of 0.11 at most, a sigmoid's slope is 1 / 4, and two scores are compared)."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
from test_gpu_sample import one_row

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("many_answers", os.path.join(ROOT, "examples", "many_answers.py"))
ex = importlib.util.module_from_spec(spec)
spec.loader.exec_module(ex)


@pytest.fixture(scope="module")
def model():
    m = ex.Model()
    yield m
    m.close()


def plain(m, tokens, experts):
    """logits of a whole text, float64; experts: of each layer [T][top_k]"""
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    rms = lambda x, w: x / np.sqrt((x * x).mean(-1, keepdims=True) + ex.EPS) * w  # noqa: E731
    T, H, K, hd = len(tokens), m.heads, m.kv_heads, m.head_dim
    r = f(m.emb)[tokens]
    ang = np.arange(T)[:, None] * f(m.inv_freq)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]

    def turn(x):
        a, b = x[..., :hd // 2], x[..., hd // 2:]
        return np.concatenate((a * c - b * s, b * c + a * s), -1)

    for l in range(m.n_layers):
        qkv = (rms(r, f(m.w_norm[l][0])) @ f(m.w_qkv[l]).T).reshape(T, H + 2 * K, hd)
        q, k, v = turn(rms(qkv[:, :H], f(m.w_head[l][0]))), turn(rms(qkv[:, H:H + K], f(m.w_head[l][1]))), qkv[:, H + K:]
        o = np.zeros((T, H, hd))
        for h in range(H):
            x = q[:, h] @ k[:, h // (H // K)].T / math.sqrt(hd)
            x[np.triu_indices(T, 1)] = -np.inf
            p = np.exp(x - x.max(-1, keepdims=True))
            o[:, h] = p / p.sum(-1, keepdims=True) @ v[:, h // (H // K)]
        r = r + o.reshape(T, -1) @ f(m.w_o[l]).T
        x = rms(r, f(m.w_norm[l][1]))
        score = 1 / (1 + np.exp(-(x @ f(m.w_router[l]).T)))
        by = score + f(m.bias[l])
        chosen = experts[l]
        assert all(len(set(row)) == m.top_k for row in chosen.tolist())
        assert np.all(np.take_along_axis(by, chosen, 1).min(-1) >= np.sort(by, -1)[:, -m.top_k] - 0.06)
        w = np.take_along_axis(score, chosen, 1)
        w = m.scale * w / w.sum(-1, keepdims=True)
        gate, up, down = (f(t) for t in m.host_mlp[l])
        y = np.zeros_like(r)
        for t in range(T):
            for j in range(m.top_k):
                e = chosen[t, j]
                a = gate[e] @ x[t]
                y[t] += w[t, j] * ((a / (1 + np.exp(-a)) * (up[e] @ x[t])) @ down[e])
        r = r + y
    return rms(r, f(m.w_last)) @ f(m.emb).T


def close(got, want):
    err = np.max(np.abs(got.double().cpu().numpy() - want)) / np.sqrt(np.mean(want ** 2))
    print("error %.3g of the logits' RMS" % err, flush=True)
    assert err <= 0.11


@pytest.mark.parametrize("n, length, max_pages", [(24, 130, 1024), (24, 130, 4), (3, 64, 4), (1, 1, 4)])
def test_answers_hold_what_their_text_says(model, n, length, max_pages):
    """with a table that is long enough for a plan of shared pieces, and short calls"""
    cache = ex.Cache(model, n_pages=80, n_seqs=n + 1, max_pages=max_pages)
    prompt = torch.randint(0, 512, (length,), generator=torch.Generator().manual_seed(4)).cuda()
    steps, trace = 8, []
    if length > 64:  # (the prompt in two parts: the layers are made for 64 tokens)
        first = []
        for i in range(0, length - length % 64, 64):
            ex.forward(model, cache, [0], prompt[None, i:i + 64], first)
        rest = prompt[length - length % 64:]
    else:
        first, rest = [], prompt
    text, limits, last = ex.answers(model, cache, rest, n, steps, trace=trace)
    assert trace[1][0].shape == (n, 512)
    t, k, p = (x.double().cpu().numpy() for x in limits)
    for logits, u, token, _ in trace[1:]:
        l = logits.cpu().numpy()
        for i in range(n):
            ok = {one_row(l[i], float(np.float32(t[i])), int(k[i]), float(np.float32(p[i])), 0.0, float(u[i].item()) + e)[0] for e in (-1e-7, 0.0, 1e-7)}
            assert int(token[i]) in ok
    for i in {0, n // 2, n - 1}:
        parts = [[first[j][0] for j in range(l, len(first), 2)] + [trace[0][3][l][0]] + [s[3][l][i] for s in trace[1:]] for l in range(2)]
        experts = [torch.cat(q).long().cpu().numpy() for q in parts]
        want = plain(model, prompt.tolist() + text[i].tolist(), experts)
        close(last[i], want[-1])
        close(trace[1][0][i], want[length - 1])
    cache.check()


def test_a_recorded_step_is_replayed(model):
    """append, attention and sampling in one graph, replayed as the sequences grow, with eager calls between; every replay equals the eager calls"""
    n, H, K, hd, V = 6, model.heads, model.kv_heads, model.head_dim, 5000
    caches = [ex.Cache(model, n_pages=40, n_seqs=n + 1, max_pages=2048) for _ in range(2)]
    g = torch.Generator().manual_seed(9)
    prompt = torch.randint(0, 512, (64,), generator=g).cuda()
    root, kids = ex._list([0] * n), ex._list(range(1, n + 1))
    for c in caches:
        ex.forward(model, c, [0], prompt[None])
        si.si_cache_fork(c.desc, root.data_ptr(), kids.data_ptr(), n, ex._stream())
    qkv, u, w_out = torch.empty((n, (H + 2 * K) * hd), dtype=ex.BF16, device="cuda"), torch.empty(n, device="cuda"), torch.randn((H * hd, V), generator=g).cuda()
    t, k, p = torch.full((n,), 0.9, device="cuda"), ex._list([0, 1, 40, 0, 3000, 7]), torch.tensor([0.9, 1.0, 0.8, 0.99, 0.5, 1.0], device="cuda")

    def make(c):
        s = dict(q=torch.empty((n, H * hd), dtype=ex.BF16, device="cuda"), att=torch.empty((n, H * hd), dtype=ex.BF16, device="cuda"), logits=torch.empty((n, V), device="cuda"),
                 seq=torch.empty(n, dtype=torch.int32, device="cuda"), pos=torch.empty(n, dtype=torch.int32, device="cuda"), token=torch.empty(n, dtype=torch.int32, device="cuda"),
                 prob=torch.empty(n, device="cuda"))
        row, a = qkv.shape[1], qkv.data_ptr()
        s["append"] = si.si_append_t(q=a, k=a + 2 * H * hd, v=a + 2 * (H + K) * hd, q_out=s["q"].data_ptr(), seq=s["seq"].data_ptr(), pos=s["pos"].data_ptr(),
                                     inv_freq=model.inv_freq.data_ptr(), q_stride=row, k_stride=row, v_stride=row, q_out_stride=H * hd, n_tokens=n, n_heads=H, rot_dim=hd)
        s["norm"] = si.si_head_norm_t(w_q=model.w_head[0][0].data_ptr(), w_k=model.w_head[0][1].data_ptr(), w_type=si.SI_BF16, kind=si.SI_NORM_RMS, eps=ex.EPS)
        s["attend"] = si.si_attend_t(q=s["q"].data_ptr(), out=s["att"].data_ptr(), seqs=kids.data_ptr(), q_stride=H * hd, out_stride=H * hd, n=n, n_new=1, n_heads=H,
                                     max_len=c.desc.max_pages * 64 * 8)
        s["sample"] = si.si_sample_t(logits=s["logits"].data_ptr(), temperature=t.data_ptr(), top_k=k.data_ptr(), top_p=p.data_ptr(), u=u.data_ptr(), token=s["token"].data_ptr(),
                                     prob=s["prob"].data_ptr(), stride=V, rows=n, vocab=V, type=si.SI_F32)
        for d, size in ((s["attend"], si.si_attend_shared_scratch_bytes(c.desc, s["attend"])), (s["sample"], si.si_sample_scratch_bytes(s["sample"]))):
            s["scratch%d" % size] = torch.zeros(size, dtype=torch.uint8, device="cuda")
            d.scratch, d.scratch_bytes = s["scratch%d" % size].data_ptr(), size
        return s

    def step(c, s):
        st = torch.cuda.current_stream().cuda_stream
        si.si_cache_extend(c.desc, kids.data_ptr(), n, None, 1, s["seq"].data_ptr(), s["pos"].data_ptr(), n, st)
        si.si_cache_append_normed(c.desc, 0, s["append"], s["norm"], st)
        si.si_attend_shared(c.desc, 0, s["attend"], st)
        torch.mul(s["att"].float()[:, :1], w_out[:1], out=s["logits"])
        for i in range(1, 40):
            s["logits"].addcmul_(s["att"].float()[:, i:i + 1], w_out[i:i + 1])
        si.si_sample(s["sample"], st)

    states = [make(c) for c in caches]
    qkv.normal_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step(caches[0], states[0])
    for i in range(70):
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        u.copy_(torch.rand(n, generator=g))
        graph.replay()
        step(caches[1], states[1])
        if i % 7 == 0 or i > 60:
            torch.cuda.synchronize()
            assert all(torch.equal(states[0][x], states[1][x]) for x in ("q", "att", "logits", "token", "prob"))
    for c in caches:
        c.check()
        assert c.lens.tolist() == [64] + [134] * n


def test_the_script_runs():
    ex.main()
