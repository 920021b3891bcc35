"""A small Transformer generates text with the library: prompts, beams, drafted tokens, pages that come and go.

    python examples/paged_decode.py

Between two feed-forward layers (si_layer_forward, split over GPU and host link) run si_norm, si_cache_append and si_attend; the projections
are plain matrix products.  Weights are random, so the text is noise; what the script prints is what the cache does."""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2411_15715_amd as si  # noqa: E402

BF16 = torch.bfloat16


class Model:
    def __init__(self, vocab=512, d_model=256, d_ff=512, n_layers=2, heads=8, kv_heads=2, head_dim=64, max_tokens=64, split=(0.5, 0.5, 0.0), seed=0):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *shape: (torch.randn(shape, generator=g) * shape[-1] ** -0.5).to(BF16)  # noqa: E731
        self.d, self.heads, self.kv_heads, self.head_dim, self.n_layers = d_model, heads, kv_heads, head_dim, n_layers
        self.emb = rand(vocab, d_model).cuda()
        self.w_qkv = [rand((heads + 2 * kv_heads) * head_dim, d_model).cuda() for _ in range(n_layers)]
        self.w_o = [rand(d_model, heads * head_dim).cuda() for _ in range(n_layers)]
        self.w_norm = [[(1 + 0.1 * torch.randn(d_model, generator=g)).to(BF16).cuda() for _ in range(2)] for _ in range(n_layers)]
        self.w_last = (1 + 0.1 * torch.randn(d_model, generator=g)).to(BF16).cuda()
        self.inv_freq = (10000.0 ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)).float().cuda()
        self.host_mlp = [[rand(1, d_ff, d_model) for _ in range(3)] for _ in range(n_layers)]
        bits = lambda t: t.view(torch.int16).numpy().view(np.uint16)  # noqa: E731
        self.mlp = [si.si_layer_create(d_model, d_ff, 1, 1, *(bits(t) for t in w), *split, max_tokens) for w in self.host_mlp]

    def close(self):
        for h in self.mlp:
            si.si_layer_destroy(h)
        self.mlp = []


class Cache:
    """The pool with its tables, and the descriptor of it."""

    def __init__(self, model, n_pages, n_seqs, max_pages, page=64, kind=si.SI_KV_BF16):
        zeros = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
        dtype = BF16 if kind == si.SI_KV_BF16 else torch.float8_e4m3fn
        self.pages = torch.zeros((n_pages, model.n_layers * 2 * model.kv_heads * page * model.head_dim), dtype=BF16, device="cuda").to(dtype)
        self.table, self.lens, self.refs, self.status = zeros(n_seqs, max_pages) - 1, zeros(n_seqs), zeros(n_pages), zeros(1)
        self.desc = si.si_cache_t(pages=self.pages.data_ptr(), table=self.table.data_ptr(), lens=self.lens.data_ptr(), refs=self.refs.data_ptr(),
                                  status=self.status.data_ptr(), n_pages=n_pages, page_tokens=page, n_layers=model.n_layers, n_kv_heads=model.kv_heads,
                                  head_dim=model.head_dim, type=kind, n_seqs=n_seqs, max_pages=max_pages)
        self.scratch = torch.zeros(si.si_cache_scratch_bytes(self.desc), dtype=torch.uint8, device="cuda")
        self.desc.scratch = self.scratch.data_ptr()

    def check(self):
        assert int(self.status.item()) == 0, "the cache reports %d" % int(self.status.item())

    def used(self):
        return int((self.refs > 0).sum().item())


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _list(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _norm(model, r, y, w, out, y_type):
    """r += y (where there is a y), out = its norm"""
    n = r.shape[0]
    si.si_norm(si.si_norm_t(r=r.data_ptr(), y=y.data_ptr() if y is not None else None, w_pre=w.data_ptr(), r_out=r.data_ptr(), out=out.data_ptr(), r_stride=model.d,
                            y_stride=model.d, r_out_stride=model.d, out_stride=model.d, rows=n, d=model.d, r_type=si.SI_BF16, y_type=y_type, w_type=si.SI_BF16,
                            r_out_type=si.SI_BF16, out_type=si.SI_BF16, pre=si.SI_NORM_RMS, eps=1e-5, res_scale=1.0, y_scale=1.0), _stream())


def forward(model, cache, seqs, tokens):
    """Appends tokens [n][n_new] to sequences and returns the logits after each of them, [n][n_new][vocab]."""
    n, n_new = tokens.shape
    T, H, K, hd = n * n_new, model.heads, model.kv_heads, model.head_dim
    who, (seq, pos) = _list(seqs), (torch.empty(T, dtype=torch.int32, device="cuda") for _ in range(2))
    si.si_cache_extend(cache.desc, who.data_ptr(), n, None, n_new, seq.data_ptr(), pos.data_ptr(), T, _stream())
    r = model.emb[tokens.reshape(-1)]
    h, q, att = torch.empty_like(r), torch.empty((T, H * hd), dtype=BF16, device="cuda"), torch.empty((T, H * hd), dtype=BF16, device="cuda")
    y = torch.empty((T, model.d), dtype=torch.float32, device="cuda")
    at = si.si_attend_t(q=q.data_ptr(), out=att.data_ptr(), seqs=who.data_ptr(), q_stride=H * hd, out_stride=H * hd, n=n, n_new=n_new, n_heads=H,
                        max_len=cache.desc.max_pages * cache.desc.page_tokens)
    at.scratch_bytes = si.si_attend_scratch_bytes(cache.desc, at)
    scratch = torch.zeros(max(1, at.scratch_bytes), dtype=torch.uint8, device="cuda")
    at.scratch = scratch.data_ptr()
    for l in range(model.n_layers):
        _norm(model, r, y if l else None, model.w_norm[l][0], h, si.SI_F32)
        qkv = h @ model.w_qkv[l].T
        row, p = qkv.shape[1], qkv.data_ptr()
        si.si_cache_append(cache.desc, l, si.si_append_t(
            q=p, k=p + 2 * H * hd, v=p + 2 * (H + K) * hd, q_out=q.data_ptr(), seq=seq.data_ptr(), pos=pos.data_ptr(), inv_freq=model.inv_freq.data_ptr(),
            q_stride=row, k_stride=row, v_stride=row, q_out_stride=H * hd, n_tokens=T, n_heads=H, rot_dim=hd), _stream())
        si.si_attend(cache.desc, l, at, _stream())
        o = att @ model.w_o[l].T
        _norm(model, r, o, model.w_norm[l][1], h, si.SI_BF16)
        si.si_layer_forward(model.mlp[l], h.data_ptr(), None, T, 0, si.SI_AUTO, y.data_ptr(), stream=_stream())
    _norm(model, r, y, model.w_last, h, si.SI_F32)
    return (h @ model.emb.T).float().view(n, n_new, -1)


def beams(model, cache, prompt, n_beams, steps, log=print):
    """Beam search over sequences 1 .. n_beams, sequence 0 holding the prompt; returns the tokens of each beam and its sequence."""
    logits = forward(model, cache, [0], prompt[None])[0, -1]
    score, token = logits.log_softmax(-1).topk(n_beams)
    live = list(range(1, n_beams + 1))
    root, kids = _list([0] * n_beams), _list(live)
    si.si_cache_fork(cache.desc, root.data_ptr(), kids.data_ptr(), n_beams, _stream())
    text = [[int(t)] for t in token]
    spare = list(range(n_beams + 1, 2 * n_beams + 1))
    for step in range(steps):
        logits = forward(model, cache, live, torch.tensor([t[-1:] for t in text], device="cuda"))[:, -1].log_softmax(-1)
        score, flat = (score[:, None] + logits).view(-1).topk(n_beams)
        parent, token = (flat // logits.shape[1]).tolist(), (flat % logits.shape[1]).tolist()
        # every beam starts from its parent's pages: full ones are shared, the last one is copied
        old, new = _list([live[p] for p in parent]), _list(spare)
        si.si_cache_fork(cache.desc, old.data_ptr(), new.data_ptr(), n_beams, _stream())
        gone = _list(live)
        si.si_cache_trim(cache.desc, gone.data_ptr(), n_beams, None, _stream())
        live, spare = spare, live
        text = [text[p] + [t] for p, t in zip(parent, token)]
    cache.check()
    log("%d beams after %d steps: %d pages in use, %d tokens each" % (n_beams, steps, cache.used(), int(cache.lens[live[0]].item())))
    return text, live


def speculate(model, cache, seq, last, drafts, log=print):
    """Checks drafted tokens at once: `last` (not in the cache yet) and the drafts go in together, the greedy choices say how many stay.
    Returns the accepted drafts and the next token."""
    before = int(cache.lens[seq].item())
    choice = forward(model, cache, [seq], torch.tensor([[last] + drafts], device="cuda"))[0].argmax(-1).tolist()
    good = 0
    while good < len(drafts) and drafts[good] == choice[good]:
        good += 1
    keep, who = _list([before + 1 + good]), _list([seq])
    si.si_cache_trim(cache.desc, who.data_ptr(), 1, keep.data_ptr(), _stream())
    cache.check()
    log("%d of %d drafted tokens accepted, %d tokens in the cache" % (good, len(drafts), before + 1 + good))
    return drafts[:good], choice[good]


def main():
    model = Model()
    try:
        cache = Cache(model, n_pages=64, n_seqs=12, max_pages=8)
        prompt = torch.randint(0, 512, (50,), generator=torch.Generator().manual_seed(1)).cuda()
        text, live = beams(model, cache, prompt, n_beams=4, steps=20)
        best = live[0]
        rest = _list([0] + live[1:])
        si.si_cache_trim(cache.desc, rest.data_ptr(), rest.numel(), None, _stream())
        accepted, token = speculate(model, cache, best, text[0][-1], [3, 1, 4])
        small = Cache(model, n_pages=cache.used() + 2, n_seqs=12, max_pages=8)
        si.si_cache_compact(cache.desc, small.desc, None, _stream())
        print("packed from a pool of %d pages into one of %d" % (cache.desc.n_pages, small.desc.n_pages))
        before = forward(model, cache, [best], torch.tensor([[token]], device="cuda"))
        after = forward(model, small, [best], torch.tensor([[token]], device="cuda"))
        cache.check()
        small.check()
        assert torch.equal(before, after), "the packed cache gives another answer"
        print("next token %d, the same from both pools" % int(after[0, -1].argmax()))
    finally:
        model.close()


if __name__ == "__main__":
    main()
