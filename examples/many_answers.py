"""A small Transformer of experts answers one prompt many times: the prompt is read once, its pages are shared, every answer is drawn for itself.

    python examples/many_answers.py

Between two layers of experts, chosen by sigmoid scores with a correcting bias (si_layer_set_scores), run si_norm, si_cache_append_normed (each head of q and k
has a norm) and si_attend_shared; si_sample draws the tokens, each answer with a temperature of its own.  The projections are plain matrix
products.  Weights are random, so the text is noise."""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2411_15715_amd as si  # noqa: E402
from paged_decode import BF16, Cache, _list, _norm, _stream  # noqa: E402

EPS = 1e-5


class Model:
    def __init__(self, vocab=512, d_model=256, d_ff=128, n_layers=2, heads=8, kv_heads=2, head_dim=64, experts=8, top_k=2, max_tokens=64, split=(0.5, 0.5, 0.0), seed=0):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *shape: (torch.randn(shape, generator=g) * shape[-1] ** -0.5).to(BF16)  # noqa: E731
        gain = lambda n: (1 + 0.1 * torch.randn(n, generator=g)).to(BF16).cuda()  # noqa: E731
        self.d, self.heads, self.kv_heads, self.head_dim, self.n_layers, self.experts, self.top_k = d_model, heads, kv_heads, head_dim, n_layers, experts, top_k
        self.emb = rand(vocab, d_model).cuda()
        self.w_qkv = [rand((heads + 2 * kv_heads) * head_dim, d_model).cuda() for _ in range(n_layers)]
        self.w_o = [rand(d_model, heads * head_dim).cuda() for _ in range(n_layers)]
        self.w_norm = [[gain(d_model) for _ in range(2)] for _ in range(n_layers)]
        self.w_head = [[gain(head_dim) for _ in range(2)] for _ in range(n_layers)]  # of q and of k
        self.w_last = gain(d_model)
        self.w_router = [(torch.randn((experts, d_model), generator=g) * d_model ** -0.5).cuda() for _ in range(n_layers)]
        self.bias = [(0.1 * torch.randn(experts, generator=g)).cuda() for _ in range(n_layers)]  # evens the experts' load: chooses, but does not weigh
        self.inv_freq = (10000.0 ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)).float().cuda()
        self.scale = 1.5
        self.host_mlp = [[rand(experts, d_ff, d_model) for _ in range(3)] for _ in range(n_layers)]
        bits = lambda t: t.view(torch.int16).numpy().view(np.uint16)  # noqa: E731
        self.mlp = [si.si_layer_create(d_model, d_ff, experts, top_k, *(bits(t) for t in w), *split, max_tokens) for w in self.host_mlp]
        for h, b in zip(self.mlp, self.bias):
            si.si_layer_set_scores(h, si.si_score_t(bias=b.data_ptr(), score=si.SI_SCORE_SIGMOID, renorm=1, scale=self.scale))

    def close(self):
        for h in self.mlp:
            si.si_layer_destroy(h)
        self.mlp = []


def forward(model, cache, seqs, tokens, experts=None):
    """Appends tokens [n][n_new] to sequences and returns the logits after each of them, [n][n_new][vocab]; experts: a list that gets each layer's choice."""
    n, n_new = tokens.shape
    T, H, K, hd = n * n_new, model.heads, model.kv_heads, model.head_dim
    who, (seq, pos) = _list(seqs), (torch.empty(T, dtype=torch.int32, device="cuda") for _ in range(2))
    si.si_cache_extend(cache.desc, who.data_ptr(), n, None, n_new, seq.data_ptr(), pos.data_ptr(), T, _stream())
    r = model.emb[tokens.reshape(-1)]
    h, q, att = torch.empty_like(r), torch.empty((T, H * hd), dtype=BF16, device="cuda"), torch.empty((T, H * hd), dtype=BF16, device="cuda")
    y = torch.empty((T, model.d), dtype=torch.float32, device="cuda")
    at = si.si_attend_t(q=q.data_ptr(), out=att.data_ptr(), seqs=who.data_ptr(), q_stride=H * hd, out_stride=H * hd, n=n, n_new=n_new, n_heads=H,
                        max_len=cache.desc.max_pages * cache.desc.page_tokens)
    at.scratch_bytes = si.si_attend_shared_scratch_bytes(cache.desc, at)
    scratch = torch.zeros(max(1, at.scratch_bytes), dtype=torch.uint8, device="cuda")
    at.scratch = scratch.data_ptr()
    for l in range(model.n_layers):
        _norm(model, r, y if l else None, model.w_norm[l][0], h, si.SI_F32)
        qkv = h @ model.w_qkv[l].T
        row, p = qkv.shape[1], qkv.data_ptr()
        w_q, w_k = model.w_head[l]
        si.si_cache_append_normed(cache.desc, l, si.si_append_t(
            q=p, k=p + 2 * H * hd, v=p + 2 * (H + K) * hd, q_out=q.data_ptr(), seq=seq.data_ptr(), pos=pos.data_ptr(), inv_freq=model.inv_freq.data_ptr(),
            q_stride=row, k_stride=row, v_stride=row, q_out_stride=H * hd, n_tokens=T, n_heads=H, rot_dim=hd),
            si.si_head_norm_t(w_q=w_q.data_ptr(), w_k=w_k.data_ptr(), w_type=si.SI_BF16, kind=si.SI_NORM_RMS, eps=EPS), _stream())
        si.si_attend_shared(cache.desc, l, at, _stream())
        o = att @ model.w_o[l].T
        _norm(model, r, o, model.w_norm[l][1], h, si.SI_BF16)
        scores = h.float() @ model.w_router[l].T
        chosen = torch.empty((T, model.top_k), dtype=torch.int32, device="cuda")
        si.si_layer_forward(model.mlp[l], h.data_ptr(), scores.data_ptr(), T, 0, si.SI_AUTO, y.data_ptr(), {"idx": chosen.data_ptr()}, _stream())
        if experts is not None:
            experts.append(chosen.view(n, n_new, -1))
    _norm(model, r, y, model.w_last, h, si.SI_F32)
    return (h @ model.emb.T).float().view(n, n_new, -1)


def draw(logits, u, temperature, top_k, top_p):
    """A token for each row of logits, with what each row is limited to; returns tokens and their probabilities, on the GPU."""
    rows, vocab = logits.shape
    token, prob = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    d = si.si_sample_t(logits=logits.data_ptr(), temperature=temperature.data_ptr(), top_k=top_k.data_ptr(), top_p=top_p.data_ptr(), u=u.data_ptr(),
                       token=token.data_ptr(), prob=prob.data_ptr(), stride=logits.stride(0), rows=rows, vocab=vocab, type=si.SI_F32)
    d.scratch_bytes = si.si_sample_scratch_bytes(d)
    scratch = torch.zeros(d.scratch_bytes, dtype=torch.uint8, device="cuda")
    d.scratch = scratch.data_ptr()
    si.si_sample(d, _stream())
    return token, prob


def answers(model, cache, prompt, n, steps, seed=0, log=print, trace=None):
    """n answers of `steps` tokens to the prompt, which sequence 0 holds; sequences 1 .. n share its pages.  Returns tokens [n][steps].
    trace: a list that gets (logits, u, tokens, experts of each layer) of the prompt and of every step."""
    u = torch.rand((steps, n), generator=torch.Generator().manual_seed(seed)).cuda()
    temperature = torch.linspace(0.0, 1.5, n, device="cuda")
    top_k, top_p = _list([50 if i % 3 else 0 for i in range(n)]), torch.tensor([0.9 if i % 2 else 1.0 for i in range(n)], device="cuda")
    limits = (temperature, top_k, top_p)
    experts = []
    last = forward(model, cache, [0], prompt[None], experts)[0, -1:].expand(n, -1).contiguous()
    if trace is not None:
        trace.append((None, None, None, experts))
    live = list(range(1, n + 1))
    root, kids = _list([0] * n), _list(live)
    si.si_cache_fork(cache.desc, root.data_ptr(), kids.data_ptr(), n, _stream())
    text = []
    for step in range(steps):
        token, _ = draw(last, u[step], *limits)
        text.append(token)
        experts = []
        logits = forward(model, cache, live, token[:, None].long(), experts)[:, 0].contiguous()
        if trace is not None:
            trace.append((last, u[step], token, experts))
        last = logits
    cache.check()
    log("%d answers of %d tokens to a prompt of %d: %d pages in use" % (n, steps, prompt.numel(), cache.used()))
    return torch.stack(text, 1), limits, last


def main():
    model = Model()
    try:
        cache = Cache(model, n_pages=64, n_seqs=25, max_pages=1024)
        prompt = torch.randint(0, 512, (60,), generator=torch.Generator().manual_seed(1)).cuda()
        text, limits, _ = answers(model, cache, prompt, n=24, steps=12)
        different = len({tuple(t) for t in text.tolist()})
        print("%d of them differ; the first, of temperature 0: %s" % (different, text[0].tolist()))
        gone = _list(list(range(25)))
        si.si_cache_trim(cache.desc, gone.data_ptr(), 25, None, _stream())
        cache.check()
        assert cache.used() == 0
    finally:
        model.close()


if __name__ == "__main__":
    main()
