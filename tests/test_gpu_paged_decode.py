"""The operators together, as examples/paged_decode.py uses them: a two-layer model against its definition in 64 bits.

Tolerance: the largest error of the logits against their RMS.  A layer takes the feed-forward layer's own bound (2e-2) and, on the way from
one residual to the next, six roundings to bf16 (norm, projection, rotation, weights, attention, output), 2^-8 each, which are counted as if they all
added up: 2 layers of 2e-2 + 6 / 256, the last norm and the logits' own product 2 / 256, in all 0.1."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("paged_decode", os.path.join(ROOT, "examples", "paged_decode.py"))
ex = importlib.util.module_from_spec(spec)
spec.loader.exec_module(ex)


@pytest.fixture(scope="module")
def model():
    m = ex.Model()
    yield m
    m.close()


def plain(m, tokens):
    """logits of a whole text, float64"""
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    rms = lambda x, w: x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-5) * w  # noqa: E731
    T, H, K, hd = len(tokens), m.heads, m.kv_heads, m.head_dim
    r = f(m.emb)[tokens]
    ang = np.arange(T)[:, None] * f(m.inv_freq)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]

    def turn(x):
        a, b = x[..., :hd // 2], x[..., hd // 2:]
        return np.concatenate((a * c - b * s, b * c + a * s), -1)

    for l in range(m.n_layers):
        qkv = (rms(r, f(m.w_norm[l][0])) @ f(m.w_qkv[l]).T).reshape(T, H + 2 * K, hd)
        q, k, v = turn(qkv[:, :H]), turn(qkv[:, H:H + K]), qkv[:, H + K:]
        o = np.zeros((T, H, hd))
        for h in range(H):
            x = q[:, h] @ k[:, h // (H // K)].T / math.sqrt(hd)
            x[np.triu_indices(T, 1)] = -np.inf
            p = np.exp(x - x.max(-1, keepdims=True))
            o[:, h] = p / p.sum(-1, keepdims=True) @ v[:, h // (H // K)]
        r = r + o.reshape(T, -1) @ f(m.w_o[l]).T
        g, u, d = (f(t)[0] for t in m.host_mlp[l])
        x = rms(r, f(m.w_norm[l][1]))
        a = x @ g.T
        r = r + (a / (1 + np.exp(-a)) * (x @ u.T)) @ d
    return rms(r, f(m.w_last)) @ f(m.emb).T


def close(got, want):
    err = np.max(np.abs(got.double().cpu().numpy() - want)) / np.sqrt(np.mean(want ** 2))
    print("error %.3g of the logits' RMS" % err, flush=True)
    assert err <= 0.1


def test_prompt_and_single_tokens(model):
    cache = ex.Cache(model, n_pages=16, n_seqs=3, max_pages=4)
    text = torch.randint(0, 512, (75,), generator=torch.Generator().manual_seed(3)).tolist()
    want = plain(model, text)
    got = ex.forward(model, cache, [1], torch.tensor([text[:60]], device="cuda"))
    close(got[0], want[:60])
    for i in range(60, 75):
        close(ex.forward(model, cache, [1], torch.tensor([[text[i]]], device="cuda"))[0], want[i:i + 1])
    cache.check()


def test_beams_hold_what_their_text_says(model):
    cache = ex.Cache(model, n_pages=48, n_seqs=9, max_pages=4)
    prompt = torch.randint(0, 512, (40,), generator=torch.Generator().manual_seed(4)).cuda()
    text, live = ex.beams(model, cache, prompt, n_beams=4, steps=30)
    got = ex.forward(model, cache, live, torch.tensor([t[-1:] for t in text], device="cuda"))
    for b in range(4):
        close(got[b], plain(model, prompt.tolist() + text[b])[-1:])
    cache.check()


def test_rejected_drafts_leave_no_trace(model):
    cache = ex.Cache(model, n_pages=16, n_seqs=2, max_pages=4)
    text = torch.randint(0, 512, (62,), generator=torch.Generator().manual_seed(5)).tolist()
    ex.forward(model, cache, [0], torch.tensor([text[:-1]], device="cuda"))
    want = plain(model, text)[-1]
    accepted, token = ex.speculate(model, cache, 0, text[-1], [int(want.argmax()), 7, 7, 7])
    full = text + accepted
    assert int(cache.lens[0].item()) == len(full)
    got = ex.forward(model, cache, [0], torch.tensor([[token]], device="cuda"))
    close(got[0], plain(model, full + [token])[-1:])


def test_the_script_runs():
    ex.main()
