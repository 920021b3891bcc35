"""Performance cases of the operators that draw several answers to one prompt from a sparse model.

A step of a batch of such sequences norms its queries and keys head by head before it rotates them into the cache, lets sequences that share
leading pages (si_cache_fork) attend to these once for all of them, gives its tokens to experts by scores with a bias, and draws each sequence's
next token from the logits.  prepare() makes one call's inputs, run() is one such call, as elementary torch operations (own = False) or as
the library's calls (own = True).

A case is a dict; "op" is one of
  route    tokens to experts: T tokens, E experts, k of them, score ("softmax", "sigmoid"), bias, n_groups / top_groups / group_best
           (1 / 1 / 1: no groups), renorm, scale of the weights
  append   tokens, heads, kv_heads, d, type of the cache, page, rot (rotated dimensions), pairs (neighbours instead of halves), far (first position),
           norm ("rms", "mean"), bias, per_head (weights of each head), w (their type)
  shared   n sequences, neighbours in groups of `group` that share the first share_lo .. share_hi tokens (whole pages of them), own_lo .. own_hi tokens of their
           own after these, n_new query tokens each, heads, kv_heads, d, type, page, window (0: none)
  sample   rows of `vocab` logits of a type, temperature, top_k, top_p, min_p (0, 1 and 0: no such limit; mixed: each row has its own)

The cache's layout (pages of `page` tokens): pages [n_pages][2: K, V][kv_heads][page / B blocks], a block holds B = 4 E tokens,
E = 16 bytes / element size
  K block [d / E][B slots][E], token t of the block in slot (t % E / 4) * 16 + 4 * (t / E) + t % 4
  V block [4][d][E], token t in chunk t / E at t % E
A stored e4m3 code stands for code * scale of its head; bf16 values stand for themselves.
"""
import math
import random

import numpy as np
import torch

own = False

EPS = 1e-6
MAX_CACHE = 560_000_000       # elements of K in the largest shared case, every sequence padded to the longest
MAX_PRODUCTS = 7_000_000_000  # these elements times the rows of a kv head
MAX_SCORES = 8192 * 256       # of a route case
MAX_LOGITS = 256 * 131072


def listed():
    return [
        # one token of one sequence, probabilities of the chosen experts as they are
        dict(name="route_token", op="route", T=1, E=64, k=8, score="softmax", bias=False, n_groups=1, top_groups=1, group_best=1, renorm=False, scale=1.0),
        # a batch in the generation phase, an expert count that fills no wave evenly
        dict(name="route_batch_60", op="route", T=97, E=60, k=4, score="softmax", bias=False, n_groups=1, top_groups=1, group_best=1, renorm=True, scale=1.0),
        # a long prompt on many small experts whose load a bias balances, half of the groups open to a token
        dict(name="route_prompt_groups", op="route", T=8192, E=256, k=8, score="sigmoid", bias=True, n_groups=8, top_groups=4, group_best=2, renorm=True, scale=2.5),
        # a step of a small batch: a token for each of eight sequences
        dict(name="append_batch_8", op="append", tokens=8, heads=32, kv_heads=8, d=128, type="bf16", page=64, rot=128, pairs=False, far=20000, norm="rms",
             bias=False, per_head=False, w="bf16"),
        # prompts of three sequences, 8-bit cache
        dict(name="append_prompt_e4m3", op="append", tokens=4099, heads=64, kv_heads=8, d=128, type="e4m3", page=128, rot=128, pairs=False, far=0, norm="rms",
             bias=False, per_head=False, w="bf16"),
        # heads that fill no power of two, a rotated quarter of them, weights and biases of each head
        dict(name="append_odd_96", op="append", tokens=1931, heads=24, kv_heads=8, d=96, type="bf16", page=96, rot=24, pairs=True, far=100, norm="mean",
             bias=True, per_head=True, w="f32"),
        # four answers to one question, a few tokens into them
        dict(name="shared_few", op="shared", n=4, group=4, share_lo=611, share_hi=611, own_lo=1, own_hi=90, n_new=1, heads=32, kv_heads=8, d=128, type="bf16",
             page=64, window=0),
        # many answers to one long prompt
        dict(name="shared_answers_64", op="shared", n=64, group=64, share_lo=8000, share_hi=8000, own_lo=1, own_hi=500, n_new=1, heads=32, kv_heads=8, d=128,
             type="bf16", page=64, window=0),
        # beams of several prompts with drafted tokens, 8-bit cache, a sliding window over part of the text
        dict(name="shared_beams_e4m3", op="shared", n=45, group=8, share_lo=900, share_hi=11000, own_lo=3, own_hi=700, n_new=3, heads=48, kv_heads=8, d=128, type="e4m3",
             page=128, window=9000),
        # the next token of one sequence
        dict(name="sample_one", op="sample", rows=1, vocab=32000, type="bf16", temperature=0.8, top_k=50, top_p=0.95, min_p=0.0, mixed=False),
        # a batch whose rows each have their own limits, an odd vocabulary
        dict(name="sample_mixed_61", op="sample", rows=61, vocab=100003, type="f32", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=True),
        # the largest batch, nucleus only
        dict(name="sample_nucleus_256", op="sample", rows=256, vocab=131072, type="f32", temperature=1.0, top_k=0, top_p=0.9, min_p=0.0, mixed=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "append", "shared", "shared", "sample"])
    if op == "route":
        E = rng.choice([8, 16, 60, 64, 72, 128, 160, 192, 256, rng.randint(2, 256)])
        k = rng.randint(1, min(E, 12))
        n_groups, top_groups, group_best = 1, 1, 1
        splits = [g for g in (2, 3, 4, 5, 8, 10, 12, 16) if E % g == 0 and E // g >= 2]
        if splits and rng.random() < 0.5:
            n_groups = rng.choice(splits)
            top_groups = rng.randint(_ceil(k, E // n_groups), n_groups)
            group_best = rng.randint(1, min(3, E // n_groups))
        return dict(op=op, T=_log_int(rng, 1, MAX_SCORES // max(E, 64)), E=E, k=k, score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.6, n_groups=n_groups,
                    top_groups=top_groups, group_best=group_best, renorm=rng.random() < 0.6, scale=rng.choice([1.0, 1.0, 2.5, 16.0]))
    if op == "sample":
        vocab = rng.choice([_log_int(rng, 100, 200_000), _log_int(rng, 16_000, 200_000), 64 * _log_int(rng, 16, 3000)])
        return dict(op=op, rows=_log_int(rng, 1, min(256, MAX_LOGITS // vocab)), vocab=vocab, type=rng.choice(["bf16", "f32"]), temperature=rng.choice([1.0, 0.7, 0.3, 1.3]),
                    top_k=rng.choice([0, 0, 1, 20, 50, 300, _log_int(rng, 1, 5000)]), top_p=rng.choice([1.0, 0.95, 0.9, 0.5]), min_p=rng.choice([0.0, 0.0, 0.05]),
                    mixed=rng.random() < 0.4)
    d = rng.choice([64, 96, 128, 128, 128, 192, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 6, 8, 12])
    kind = "bf16" if d == 96 else rng.choice(["bf16", "bf16", "e4m3"])
    page = rng.choice([32, 64, 64, 96, 128, 256] if kind == "bf16" else [64, 128, 128, 192, 256])
    if op == "append":
        most = max(1, 4096 * 72 * 128 // ((heads + kv_heads) * d))
        return dict(op=op, tokens=_log_int(rng, 1, most), heads=heads, kv_heads=kv_heads, d=d, type=kind, page=page, rot=rng.choice([0, 24, d // 2, d, d, d]),
                    pairs=rng.random() < 0.3, far=rng.choice([0, 0, _log_int(rng, 100, 1_000_000)]), norm=rng.choice(["rms", "rms", "mean"]), bias=rng.random() < 0.3,
                    per_head=rng.random() < 0.3, w=rng.choice(["bf16", "f32"]))
    n = _log_int(rng, 2, 128)
    n_new = rng.choice([1, 1, 1, 2, 3, 5, 8])
    hi = _log_int(rng, n_new, max(n_new, min(60000, MAX_CACHE // (n * kv_heads * d), MAX_PRODUCTS // (n * heads * d * n_new))))
    share = min(int(hi * rng.choice([0.0, 0.3, 0.7, 0.95, 0.99])), hi - n_new)
    own_hi = hi - share
    return dict(op=op, n=n, group=rng.choice([1, 2, 4, 8, _ceil(n, 2), n, n]), share_lo=rng.choice([share, share // 2]), share_hi=share, own_lo=rng.choice([n_new, own_hi]),
                own_hi=own_hi, n_new=n_new, heads=heads, kv_heads=kv_heads, d=d, type=kind, page=page, window=rng.choice([0, 0, 0, _log_int(rng, 1, max(1, hi))]))


# ------------------------------------------------------------------------------------------------ sizes and inputs
def _ceil(a, b):
    return -(-a // b)


def _esize(kind):
    return {"e4m3": 1, "bf16": 2, "f32": 4}[kind]


def _lengths(case):
    """What each group shares and how long each sequence is; the same for every seed, as the work goes by them."""
    r = random.Random(case["n"] * 1000003 + case["share_hi"] * 31 + case["own_hi"])
    shares = [r.randint(case["share_lo"], case["share_hi"]) for _ in range(_ceil(case["n"], case["group"]))]
    shares[r.randrange(len(shares))] = case["share_hi"]
    return shares, [shares[i // case["group"]] + r.randint(case["own_lo"], case["own_hi"]) for i in range(case["n"])]


def work(case):
    op = case["op"]
    if op == "route":
        n, pairs = case["T"] * case["E"], case["T"] * case["k"]
        return {"bytes": 4 * (n + 4 * pairs + 2 * case["E"]), "flops": 8 * n}
    if op == "append":
        q, kv = case["tokens"] * case["heads"] * case["d"], case["tokens"] * case["kv_heads"] * case["d"]
        return {"bytes": 4 * q + 2 * kv * (2 + _esize(case["type"])), "flops": 8 * (q + kv)}
    if op == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * _esize(case["type"]) + 32 * case["rows"], "flops": 4 * n}
    shares, lens = _lengths(case)
    page, group, m, window = case["page"], case["group"], case["n_new"], case["window"]
    tokens = seen = 0
    for g, share in enumerate(shares):
        mine = lens[g * group:(g + 1) * group]
        common = share // page * page if len(mine) > 1 else 0  # tokens in pages that all of them name
        first = [max(0, x - m + 1 - window) if window else 0 for x in mine]
        tokens += max(0, common - min(first)) + sum(x - max(common, a) for x, a in zip(mine, first))
        seen += sum(min(x - i, window or x) for x in mine for i in range(m))
    rows = case["n"] * m * case["heads"]
    return {"bytes": 2 * tokens * case["kv_heads"] * case["d"] * _esize(case["type"]) + rows * (4 * case["d"] + 4), "flops": 4 * seen * case["heads"] * case["d"]}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 2654435761 % (1 << 62))


def _randn(g, shape, dtype, scale=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    return x.mul_(scale).to(dtype)


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}


def _pool(g, case, n_pages):
    """Random pages: N(0, 1) values as they come out of a projection, in the cache's type."""
    shape = (n_pages, 2 * case["kv_heads"] * case["page"] * case["d"])
    if case["type"] == "bf16":
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    pool = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    step = max(1, (1 << 28) // shape[1])
    for at in range(0, n_pages, step):
        pool[at:at + step] = torch.randn((min(step, n_pages - at), shape[1]), generator=g, device="cuda").to(torch.float8_e4m3fn)
    return pool


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = {"case": case}
    if op == "route":
        T, E = case["T"], case["E"]
        # experts differ in how often they are wanted, as without a bias they do
        s["logits"] = _randn(g, (T, E), torch.float32, 1.5) + 0.5 * torch.randn(E, generator=g, device="cuda")
        s["bias"] = 0.1 * torch.randn(E, generator=g, device="cuda") if case["bias"] else None
        s["out"] = {name: torch.empty(n, dtype=torch.float32 if name == "w" else torch.int32, device="cuda")
                    for name, n in (("idx", T * case["k"]), ("w", T * case["k"]), ("count", E), ("off", E + 1), ("perm", T * case["k"]), ("inv", T * case["k"]))}
        return s
    if op == "sample":
        R, V = case["rows"], case["vocab"]
        x = 2.2 * torch.randn((R, V), generator=g, device="cuda")
        peaks = torch.randint(0, V, (R, 64), generator=g, device="cuda")  # what the model has in mind
        x.scatter_add_(1, peaks, 12 * torch.rand((R, 64), generator=g, device="cuda") ** 2)
        s["logits"] = x.to(_TYPES[case["type"]])
        fill = lambda v, t: torch.full((R,), v, dtype=t, device="cuda")  # noqa: E731
        s["temperature"], s["top_k"] = fill(case["temperature"], torch.float32), fill(case["top_k"], torch.int32)
        s["top_p"], s["min_p"] = fill(case["top_p"], torch.float32), fill(case["min_p"], torch.float32)
        if case["mixed"]:
            pick = lambda values, t: torch.tensor(values, dtype=t, device="cuda")[torch.randint(0, len(values), (R,), generator=g, device="cuda")]  # noqa: E731
            s["temperature"] = pick([0.0, 0.3, 0.7, 1.0, 1.0, 1.5], torch.float32)
            s["top_k"] = pick([0, 0, 1, 20, 50, 1000], torch.int32)
            s["top_p"] = pick([1.0, 0.95, 0.8, 0.5], torch.float32)
            s["min_p"] = pick([0.0, 0.0, 0.02, 0.1], torch.float32)
        s["u"] = torch.rand(R, generator=g, device="cuda")
        s["token"], s["kept"] = (torch.empty(R, dtype=torch.int32, device="cuda") for _ in range(2))
        s["prob"] = torch.empty(R, dtype=torch.float32, device="cuda")
        return s
    H, K, d, page = case["heads"], case["kv_heads"], case["d"], case["page"]
    s["scale_k"] = 0.5 + torch.rand(K, generator=g, device="cuda") if case["type"] == "e4m3" else None
    s["scale_v"] = 0.5 + torch.rand(K, generator=g, device="cuda") if case["type"] == "e4m3" else None
    if op == "append":
        T = case["tokens"]
        if T <= 64:  # a token for each sequence, at the ends of texts of different lengths
            first, count = [case["far"] + 3 * i + 1 for i in range(T)], [1] * T
        else:        # prompts of three sequences
            a, b = T // 2, T // 3
            first, count = [case["far"], case["far"] + 7, case["far"]], [a, b, T - a - b]
        # only the pages that the call writes exist; the table names page 0 for the others, which nothing reads here
        table = np.zeros((len(first), _ceil(max(f + c for f, c in zip(first, count)), page)), np.int32)
        spots = [(i, j) for i, (f, c) in enumerate(zip(first, count)) for j in range(f // page, _ceil(f + c, page))]
        for spot, p in zip(spots, torch.randperm(len(spots), generator=g, device="cuda").cpu().tolist()):
            table[spot] = p
        s["pages"] = _pool(g, case, len(spots))
        s["table"] = torch.from_numpy(table).cuda()
        s["lens"] = torch.tensor([f + c for f, c in zip(first, count)], dtype=torch.int32, device="cuda")
        s["seq"] = torch.tensor([i for i, c in enumerate(count) for _ in range(c)], dtype=torch.int32, device="cuda")
        s["pos"] = torch.tensor([f + j for f, c in zip(first, count) for j in range(c)], dtype=torch.int32, device="cuda")
        s["qkv"] = _randn(g, (T, (H + 2 * K) * d), torch.bfloat16, 1.5)  # one projection makes all three
        rot = case["rot"]
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda() if rot else None
        for x, n in (("q", H), ("k", K)):
            shape = (n if case["per_head"] else 1, d)
            s["w_" + x] = (1 + 0.2 * torch.randn(shape, generator=g, device="cuda")).to(_TYPES[case["w"]])
            s["b_" + x] = _randn(g, shape, _TYPES[case["w"]], 0.1) if case["bias"] else None
        s["q_out"] = torch.empty((T, H, d), dtype=torch.bfloat16, device="cuda")
        return s
    shares, lens = _lengths(case)
    n, group, m = case["n"], case["group"], case["n_new"]
    rows = torch.randperm(n, generator=g, device="cuda").cpu().tolist()  # where in the table the list's sequences are
    common = [x // page if min(group, n - i * group) > 1 else 0 for i, x in enumerate(shares)]
    used = sum(common) + sum(_ceil(x, page) - common[i // group] for i, x in enumerate(lens))
    n_pages = used + used // 16 + 1
    order = iter(torch.randperm(n_pages, generator=g, device="cuda").cpu().tolist())
    table, refs = np.full((n, max(1, _ceil(max(lens), page))), -1, np.int32), np.zeros(n_pages, np.int32)
    first = [[next(order) for _ in range(c)] for c in common]
    for i, x in enumerate(lens):
        pages = first[i // group] + [next(order) for _ in range(_ceil(x, page) - common[i // group])]
        table[rows[i], :len(pages)] = pages
        refs[pages] += 1
    s["pages"] = _pool(g, case, n_pages)
    s["table"], s["refs"] = torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda()
    s["seqs"] = torch.tensor(rows, dtype=torch.int32, device="cuda")
    s["lens"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["lens"][s["seqs"].long()] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["q"] = _randn(g, (n * m, H, d), torch.bfloat16, 2.0)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((n * m, H), dtype=torch.float32, device="cuda")
    s["max_len"] = max(lens)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_route(s):
    """Scores in 64 bits, as the choice goes by their order."""
    c = s["case"]
    T, E, k = c["T"], c["E"], c["k"]
    x = s["logits"].double()
    if c["score"] == "softmax":
        x = torch.exp(x - x.amax(1, keepdim=True))
        p = x / x.sum(1, keepdim=True)
    else:
        p = 1 / (1 + torch.exp(-x))
    choice = p if s["bias"] is None else p + s["bias"].double()
    if c["n_groups"] > 1:
        runs = choice.view(T, c["n_groups"], -1)
        worth = runs.sort(dim=-1, descending=True).values[..., :c["group_best"]].sum(-1)
        best = worth.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        open_ = torch.zeros_like(worth, dtype=torch.bool)
        open_[torch.arange(T, device="cuda")[:, None], best] = True
        choice = torch.where(open_[:, :, None], runs, -math.inf).view(T, E)
    idx = choice.sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = p.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    flat = idx.reshape(-1)
    perm = flat.sort(stable=True).indices
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(T * k, device="cuda")
    count = torch.zeros(E, dtype=torch.int64, device="cuda").index_add_(0, flat, torch.ones_like(flat))
    off = torch.cat((count[:1] * 0, count.cumsum(0)))
    return {"idx": flat.int(), "w": (w * c["scale"]).float().view(-1), "count": count.int(), "off": off.int(), "perm": perm.int(), "inv": inv.int()}


def _plain_rotate(x, ang, rot, pairs):
    """x [T, heads, d] float32, ang [T, rot / 2] float64"""
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if pairs else (r[..., :rot // 2], r[..., rot // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack((a, b), -1).flatten(-2) if pairs else torch.cat((a, b), -1)
    return torch.cat((r, x[..., rot:]), -1)


def _plain_append(s):
    c = s["case"]
    T, H, K, d, page, rot = c["tokens"], c["heads"], c["kv_heads"], c["d"], c["page"], c["rot"]

    def norm(x, w, b):
        if c["norm"] == "mean":
            x = x - x.mean(-1, keepdim=True)
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        return x if b is None else x + b.float()

    q, k, v = s["qkv"].float().view(T, H + 2 * K, d).split((H, K, K), 1)
    q, k = norm(q, s["w_q"], s["b_q"]), norm(k, s["w_k"], s["b_k"])
    if rot:
        ang = s["pos"].double()[:, None] * s["inv_freq"].double()
        q, k = _plain_rotate(q, ang, rot, c["pairs"]), _plain_rotate(k, ang, rot, c["pairs"])
    if c["type"] == "e4m3":
        k, v = ((x / w[:, None]).clamp(-448.0, 448.0) for x, w in ((k, s["scale_k"]), (v, s["scale_v"])))
    E = 16 // _esize(c["type"])
    B = 4 * E
    pos = s["pos"].long()
    at = s["table"].long()[s["seq"].long(), pos // page] * (2 * K * page * d)  # element where the token's page begins
    t = pos % page
    block, t = t // B * (B * d), t % B
    dim, head = torch.arange(d, device="cuda"), torch.arange(K, device="cuda") * (page * d)
    slot = t % E // 4 * 16 + 4 * (t // E) + t % 4
    at = (at + block)[:, None, None] + head[:, None]
    to_k = at + (dim // E * (B * E) + dim % E) + (slot * E)[:, None, None]
    to_v = at + K * page * d + dim * E + (t // E * (d * E) + t % E)[:, None, None]
    pool = s["pages"].view(-1)
    pool = pool.view(torch.uint8) if c["type"] == "e4m3" else pool
    for to, x in ((to_k, k), (to_v, v)):
        x = x.to(s["pages"].dtype)
        pool[to.view(-1)] = (x.view(torch.uint8) if c["type"] == "e4m3" else x).reshape(-1)
    return {"q": q.to(torch.bfloat16), "pages": s["pages"]}


def _plain_shared(s):
    c = s["case"]
    n, m, H, K, d, page = c["n"], c["n_new"], c["heads"], c["kv_heads"], c["d"], c["page"]
    E = 16 // _esize(c["type"])
    table, lens = s["table"].long()[s["seqs"].long()], s["lens"].long()[s["seqs"].long()]
    width = table.shape[1]
    kv = s["pages"].view(-1, 2, K * page * d)[table.clamp(min=0)]  # [n, width, 2, ...]
    k = kv[:, :, 0].float().view(n, width, K, page // (4 * E), d // E, E // 4, 4, 4, E)
    k = k.permute(0, 2, 1, 3, 6, 5, 7, 4, 8).reshape(n, K, width * page, d)
    v = kv[:, :, 1].float().view(n, width, K, page // (4 * E), 4, d, E)
    v = v.permute(0, 2, 1, 3, 4, 6, 5).reshape(n, K, width * page, d)
    del kv
    q = s["q"].float().view(n, m, K, H // K, d).transpose(1, 2).reshape(n, K, m * (H // K), d)
    x = torch.matmul(q, k.transpose(-1, -2)) * d ** -0.5
    if c["type"] == "e4m3":
        x = x * s["scale_k"][:, None, None]
    end = lens[:, None] - m + 1 + torch.arange(m, device="cuda")  # [n, m]: the first position that a token does not see
    t = torch.arange(width * page, device="cuda")
    see = t < end[..., None]
    if c["window"]:
        see &= t >= end[..., None] - c["window"]
    see = see[:, None, :, None]
    x = x.view(n, K, m, H // K, -1).masked_fill(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    v = torch.where((t < lens[:, None])[:, None, :, None], v, torch.zeros_like(v))
    o = torch.matmul(p.view(n, K, m * (H // K), -1), v).view(n, K, m, H // K, d)
    if c["type"] == "e4m3":
        o = o * s["scale_v"][:, None, None, None]
    lse = (top + total.log())[..., 0]
    return {"out": o.transpose(1, 2).reshape(n * m, H, d).to(torch.bfloat16), "lse": lse.transpose(1, 2).reshape(n * m, H)}


def _plain_sample(s):
    """Probabilities and their sums in 64 bits: what is drawn, and how many are kept, goes by the borders between them."""
    x = s["logits"].double()
    R, V = x.shape
    t, u = s["temperature"].double()[:, None], s["u"].double()[:, None]
    greedy = t <= 0
    x, at = x.sort(dim=1, descending=True, stable=True)
    w = torch.exp((x - x[:, :1]) / torch.where(greedy, 1.0, t))
    rank = torch.arange(V, device="cuda")
    k = s["top_k"].long()[:, None]
    w = torch.where((rank < torch.where(k > 0, k, V)) & (~greedy | (rank == 0)), w, 0.0)
    total, p = w.cumsum(1), s["top_p"].double()[:, None]
    keep = (w > 0) & ((p >= 1) | (total - w < p * total[:, -1:]) | (rank == 0)) & (w >= s["min_p"].double()[:, None].clamp(max=1.0))
    w = torch.where(keep, w, 0.0)
    in_order = torch.zeros_like(w).scatter_(1, at, w)
    total = in_order.cumsum(1)
    token = (total <= u * total[:, -1:]).sum(1).clamp(max=V - 1)
    prob = in_order.gather(1, token[:, None]) / total[:, -1:]
    return {"token": token.int(), "prob": prob[:, 0].float(), "kept": keep.sum(1).int()}


# ------------------------------------------------------------------------------------------------ the library's calls
def _plan(s):
    """The descriptors that a program makes once, with its buffers: addresses and sizes only."""
    import paper_2411_15715_amd as si
    c = s["case"]
    ptr = lambda x: None if x is None else x.data_ptr()  # noqa: E731
    if c["op"] == "route":
        return si, si.si_score_t(bias=ptr(s["bias"]), score=si.SI_SCORE_SIGMOID if c["score"] == "sigmoid" else si.SI_SCORE_SOFTMAX, n_groups=c["n_groups"],
                                 top_groups=c["top_groups"], group_best=c["group_best"], renorm=int(c["renorm"]), scale=c["scale"]), {
            name: t.data_ptr() for name, t in s["out"].items()}
    if c["op"] == "sample":
        t = si.si_sample_t(logits=ptr(s["logits"]), temperature=ptr(s["temperature"]), top_k=ptr(s["top_k"]), top_p=ptr(s["top_p"]), min_p=ptr(s["min_p"]),
                           u=ptr(s["u"]), token=ptr(s["token"]), prob=ptr(s["prob"]), kept=ptr(s["kept"]), scratch=None, scratch_bytes=0, stride=c["vocab"],
                           rows=c["rows"], vocab=c["vocab"], type=si.SI_BF16 if c["type"] == "bf16" else si.SI_F32)
        t.scratch_bytes = si.si_sample_scratch_bytes(t)
        s["scratch"] = torch.zeros(t.scratch_bytes, dtype=torch.uint8, device="cuda")
        t.scratch = s["scratch"].data_ptr()
        return si, t
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    H, K, d = c["heads"], c["kv_heads"], c["d"]
    a = si.si_cache_t(
        pages=ptr(s["pages"]), scale_k=ptr(s["scale_k"]), scale_v=ptr(s["scale_v"]), table=ptr(s["table"]), lens=ptr(s["lens"]), refs=ptr(s.get("refs")),
        status=ptr(s["status"]), scratch=None, n_pages=s["pages"].shape[0], page_tokens=c["page"], n_layers=1, n_kv_heads=K, head_dim=d,
        type=si.SI_KV_E4M3 if c["type"] == "e4m3" else si.SI_KV_BF16, n_seqs=s["table"].shape[0], max_pages=s["table"].shape[1])
    if c["op"] == "append":
        q = s["qkv"].data_ptr()
        row = (H + 2 * K) * d
        return si, a, si.si_append_t(
            q=q, k=q + 2 * H * d, v=q + 2 * (H + K) * d, q_out=ptr(s["q_out"]), seq=ptr(s["seq"]), pos=ptr(s["pos"]), inv_freq=ptr(s["inv_freq"]),
            q_stride=row, k_stride=row, v_stride=row, q_out_stride=H * d, n_tokens=c["tokens"], n_heads=H, rot_dim=c["rot"], rot_pairs=int(c["pairs"])), si.si_head_norm_t(
            w_q=ptr(s["w_q"]), b_q=ptr(s["b_q"]), w_k=ptr(s["w_k"]), b_k=ptr(s["b_k"]), w_type=si.SI_F32 if c["w"] == "f32" else si.SI_BF16,
            kind=si.SI_NORM_MEAN if c["norm"] == "mean" else si.SI_NORM_RMS, per_head=int(c["per_head"]), eps=EPS)
    t = si.si_attend_t(q=ptr(s["q"]), out=ptr(s["out"]), lse=ptr(s["lse"]), seqs=ptr(s["seqs"]), scratch=None, scratch_bytes=0, q_stride=H * d, out_stride=H * d,
                       n=c["n"], n_new=c["n_new"], n_heads=H, window=c["window"], max_len=s["max_len"], scale=0.0)
    t.scratch_bytes = si.si_attend_shared_scratch_bytes(a, t)
    s["scratch"] = torch.zeros(t.scratch_bytes, dtype=torch.uint8, device="cuda")
    t.scratch = s["scratch"].data_ptr()
    return si, a, t


def _own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    c, (si, *a) = s["case"], s["plan"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "route":
        si.si_route_scored(s["logits"].data_ptr(), c["T"], c["E"], c["k"], a[0], a[1], stream)
        return dict(s["out"])
    if c["op"] == "append":
        si.si_cache_append_normed(a[0], 0, a[1], a[2], stream)
        return {"q": s["q_out"], "pages": s["pages"]}
    if c["op"] == "shared":
        si.si_attend_shared(a[0], 0, a[1], stream)
        return {"out": s["out"], "lse": s["lse"]}
    si.si_sample(a[0], stream)
    return {"token": s["token"], "prob": s["prob"], "kept": s["kept"]}


def run(state):
    if own:
        return _own(state)
    return {"route": _plain_route, "append": _plain_append, "shared": _plain_shared, "sample": _plain_sample}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_route(s):
    c = s["case"]
    T, E, k = c["T"], c["E"], c["k"]
    x = s["logits"].double().cpu().numpy()
    if c["score"] == "softmax":
        p = np.exp(x - np.log(np.exp(x - x.max(1, keepdims=True)).sum(1, keepdims=True)) - x.max(1, keepdims=True))
    else:
        p = np.where(x >= 0, 1 / (1 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1 + np.exp(-np.abs(x))))
    choice = p + (0.0 if s["bias"] is None else s["bias"].double().cpu().numpy())
    if c["n_groups"] > 1:
        runs = choice.reshape(T, c["n_groups"], E // c["n_groups"])
        worth = np.sort(runs, -1)[..., ::-1][..., :c["group_best"]].sum(-1)
        rank = np.argsort(np.argsort(-worth, 1, kind="stable"), 1)
        choice = np.where((rank < c["top_groups"]).repeat(E // c["n_groups"], 1), choice, -np.inf)
    idx = np.argsort(-choice, 1, kind="stable")[:, :k]
    w = np.take_along_axis(p, idx, 1)
    w = c["scale"] * (w / w.sum(1, keepdims=True) if c["renorm"] else w)
    flat = idx.reshape(-1)
    perm = np.argsort(flat, kind="stable")
    inv = np.argsort(perm, kind="stable")
    count = np.bincount(flat, minlength=E)
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    return {"idx": cuda(flat), "w": torch.from_numpy(np.ascontiguousarray(w.reshape(-1))).cuda(), "count": cuda(count),
            "off": cuda(np.concatenate(([0], np.cumsum(count)))), "perm": cuda(perm), "inv": cuda(inv)}


def _exact_append(s):
    c = s["case"]
    T, H, K, d, page, rot = c["tokens"], c["heads"], c["kv_heads"], c["d"], c["page"], c["rot"]
    x = s["qkv"].double().view(T, H + 2 * K, d).clone()
    for a, b, w, bias in ((0, H, s["w_q"], s["b_q"]), (H, H + K, s["w_k"], s["b_k"])):
        y = x[:, a:b]
        mu = y.sum(-1, keepdim=True) / d if c["norm"] == "mean" else 0.0
        var = ((y - mu) ** 2).sum(-1, keepdim=True) / d
        x[:, a:b] = (y - mu) / (var + EPS).sqrt() * w.double() + (0 if bias is None else bias.double())
    if rot:
        # the rotation as a product of complex numbers
        i = np.arange(rot // 2)
        re, im = (2 * i, 2 * i + 1) if c["pairs"] else (i, i + rot // 2)
        ang = s["pos"].double()[:, None] * s["inv_freq"].double()
        z = torch.complex(x[:, :H + K, re], x[:, :H + K, im]) * torch.polar(torch.ones_like(ang), ang)[:, None]
        x[:, :H + K, re], x[:, :H + K, im] = z.real, z.imag
    E = 16 // _esize(c["type"])
    blocks = page // (4 * E)
    pages = s["pages"].double()
    k = pages.view(-1, 2, K, blocks, d // E, E // 4, 4, 4, E)  # page, K / V, head, block, d / E, j, g, i, e of d: token g E + 4 j + i
    v = pages.view(-1, 2, K, blocks, 4, d, E)                  # page, K / V, head, block, g, d, token % E
    p = s["pos"].long()
    at = s["table"].long()[s["seq"].long(), p // page]
    p = p % page
    b, t = p // (4 * E), p % (4 * E)
    scale = lambda a, w: a if w is None else (a / w.double()[:, None]).clamp(-448, 448)  # noqa: E731
    k[at, 0, :, b, :, t % E // 4, t // E, t % 4, :] = scale(x[:, H:H + K], s["scale_k"]).reshape(T, K, d // E, E)
    v[at, 1, :, b, t // E, :, t % E] = scale(x[:, H + K:], s["scale_v"])
    return {"q": x[:, :H], "pages": pages}


def _exact_shared(s):
    """One sequence and kv head at a time, its pages gathered element by element."""
    c = s["case"]
    n, m, H, K, d, page = c["n"], c["n_new"], c["heads"], c["kv_heads"], c["d"], c["page"]
    E = 16 // _esize(c["type"])
    rows, table = s["seqs"].tolist(), s["table"].cpu()
    lens = s["lens"].cpu()[rows].tolist()
    if max(lens) * n * K * d * m > 2e9:
        return None
    out = torch.zeros((n, m, H, d), dtype=torch.float64, device="cuda")
    lse = torch.full((n, m, H), -math.inf, dtype=torch.float64, device="cuda")
    dim = torch.arange(d, device="cuda")
    flat = s["pages"].view(-1)
    flat = flat.view(torch.uint8) if c["type"] == "e4m3" else flat
    for i in range(n):
        lo = max(0, lens[i] - m + 1 - c["window"]) if c["window"] else 0
        t = torch.arange(lo, lens[i], device="cuda")
        at = table[rows[i]].cuda().long()[t // page] * (2 * K * page * d) + t % page // (4 * E) * (4 * E * d)
        u = t % (4 * E)
        at_k = at[:, None] + dim // E * (4 * E * E) + ((u % E // 4 * 16 + u // E * 4 + u % 4) * E)[:, None] + dim % E
        at_v = at[:, None] + K * page * d + (u // E * (d * E) + u % E)[:, None] + dim * E
        for h in range(K):
            k, v = flat[at_k + h * page * d], flat[at_v + h * page * d]
            k, v = (x.view(s["pages"].dtype).double() for x in (k, v))
            if s["scale_k"] is not None:
                k, v = k * s["scale_k"][h].double(), v * s["scale_v"][h].double()
            heads = slice(h * (H // K), (h + 1) * (H // K))
            for j in range(m):
                end = lens[i] - m + 1 + j
                a, b = max(0, end - c["window"]) - lo if c["window"] else 0, end - lo
                if b <= a:
                    continue
                x = (s["q"][i * m + j, heads].double() @ k[a:b].T) / math.sqrt(d)
                lse[i, j, heads] = torch.logsumexp(x, 1)
                out[i, j, heads] = torch.softmax(x, 1) @ v[a:b]
    return {"out": out.view(n * m, H, d), "lse": lse.view(n * m, H)}


def _exact_sample(s):
    x, u = s["logits"].double().cpu().numpy(), s["u"].double().tolist()
    limits = [s[name].double().tolist() for name in ("temperature", "top_k", "top_p", "min_p")]
    tokens, probs, counts = [], [], []
    for r in range(x.shape[0]):
        t, k, p, least = (a[r] for a in limits)
        if t <= 0:
            tokens.append(int(np.argmax(x[r])))
            probs.append(1.0)
            counts.append(1)
            continue
        w = np.exp((x[r] - x[r].max()) / t)
        order = np.argsort(-x[r], kind="stable")[:int(k) if k > 0 else x.shape[1]]  # the kept ones, best first
        if p < 1:
            sums = np.cumsum(w[order])
            order = order[:1 + int(np.searchsorted(sums, p * sums[-1]))]  # the first whose sum reaches the share is the last kept
        order = order[w[order] >= min(least, 1.0)]
        order = np.sort(order[w[order] > 0])
        sums = np.cumsum(w[order])
        i = min(int(np.searchsorted(sums, u[r] * sums[-1], side="right")), len(order) - 1)
        tokens.append(int(order[i]))
        probs.append(w[order[i]] / sums[-1])
        counts.append(len(order))
    as_int = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"token": as_int(tokens), "prob": torch.tensor(probs, dtype=torch.float64, device="cuda"), "kept": as_int(counts)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "append": _exact_append, "shared": _exact_shared, "sample": _exact_sample}[case["op"]](s)
