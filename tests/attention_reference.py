"""Plain implementations in 64 bits of the operators around the feed-forward layer, for the tests; written from the description in the header."""
import math

import numpy as np
import torch

import paper_2411_15715_amd as si

TORCH = {si.SI_KV_BF16: torch.bfloat16, si.SI_KV_E4M3: torch.float8_e4m3fn}


class Cache:
    """A pool on the GPU (or host: device="cpu") with its tables, and the descriptor of it."""

    def __init__(self, kind, n_pages, page, n_seqs, max_pages, n_layers=1, kv_heads=2, d=64, scales=None, seed=0, device="cuda", fill=1.0):
        self.kind, self.E = kind, 8 if kind == si.SI_KV_BF16 else 16
        self.page, self.n_layers, self.kv_heads, self.d = page, n_layers, kv_heads, d
        g = torch.Generator().manual_seed(seed)
        self.shape = (n_pages, n_layers, 2, kv_heads, page * d)
        pool = (torch.randn(self.shape, generator=g) * fill).to(TORCH[kind])
        self.pages = pool.to(device)
        self.table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(n_seqs, dtype=torch.int32, device=device)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.scale_k = self.scale_v = None
        if scales is not None:
            self.scale_k, self.scale_v = (torch.tensor(s, dtype=torch.float32, device=device) for s in scales)
        self.desc = si.si_cache_t(
            pages=self.pages.data_ptr(), table=self.table.data_ptr(), lens=self.lens.data_ptr(), refs=self.refs.data_ptr(), status=self.status.data_ptr(),
            scale_k=None if scales is None else self.scale_k.data_ptr(), scale_v=None if scales is None else self.scale_v.data_ptr(),
            n_pages=n_pages, page_tokens=page, n_layers=n_layers, n_kv_heads=kv_heads, head_dim=d, type=kind, n_seqs=n_seqs, max_pages=max_pages)

    def bits(self):
        """the pool as unsigned integers on the host, [n_pages][n_layers][2][kv_heads][page * d]"""
        t = self.pages.view(torch.uint8 if self.kind == si.SI_KV_E4M3 else torch.int16)
        a = t.cpu().numpy()
        return a if a.dtype == np.uint8 else a.view(np.uint16)

    def values(self):
        """what the pool's bits stand for without the scales, float64"""
        return self.pages.cpu().to(torch.float64).numpy()

    def places(self, tokens):
        """index [n][d] inside a head's page * d elements, of K and of V, for positions inside a page"""
        E, B, d = self.E, 4 * self.E, self.d
        t = np.asarray(tokens)[:, None]
        dim = np.arange(d)[None]
        block, u = t // B * (B * d), t % B
        slot = u % E // 4 * 16 + 4 * (u // E) + u % 4
        return block + dim // E * (B * E) + slot * E + dim % E, block + u // E * (d * E) + dim * E + u % E

    def give(self, seq, pages, length):
        self.table[seq, :len(pages)] = torch.tensor(pages, dtype=torch.int32, device=self.table.device)
        self.lens[seq] = length
        for p in pages:
            self.refs[p] += 1

    def gather(self, layer, seq, length):
        """K and V of a sequence, [kv_heads][length][d] float64, scales applied"""
        val, table = self.values(), self.table.cpu().numpy()
        k, v = np.zeros((2, self.kv_heads, length, self.d))
        for j in range(-(-length // self.page)):
            n = min(self.page, length - j * self.page)
            ik, iv = self.places(np.arange(n))
            for h in range(self.kv_heads):
                k[h, j * self.page:j * self.page + n] = val[table[seq, j], layer, 0, h][ik]
                v[h, j * self.page:j * self.page + n] = val[table[seq, j], layer, 1, h][iv]
        if self.scale_k is not None:
            k = k * self.scale_k.cpu().double().numpy()[:, None, None]
            v = v * self.scale_v.cpu().double().numpy()[:, None, None]
        return k, v


def rotate64(x, pos, inv_freq, pairs):
    """x [T][heads][d] float64; returns the rotated values and the magnitude of the terms that form them"""
    rot = 2 * len(inv_freq)
    out, mag = x.copy(), np.abs(x)
    if rot:
        ang = np.asarray(pos, np.float64)[:, None] * np.asarray(inv_freq, np.float64)
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
        i, j = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if pairs else (np.arange(rot // 2), np.arange(rot // 2, rot))
        a, b = x[..., i], x[..., j]
        out[..., i], out[..., j] = a * c - b * s, b * c + a * s
        mag[..., i] = mag[..., j] = np.abs(a) + np.abs(b)
    return out, mag


def attend64(q, k, v, n_new, window, scale):
    """q [n_new][heads][d], k / v [kv_heads][len][d]; returns out, lse, and the largest |k|-weighted magnitudes for tolerances:
    sum |q k| scale per score (its maximum over the positions seen) and sum p |v|"""
    m, H, d = q.shape
    K, L = k.shape[0], k.shape[1]
    out, lse = np.zeros((m, H, d)), np.full((m, H), -math.inf)
    mag_s, mag_o = np.zeros((m, H)), np.zeros((m, H, d))
    for j in range(m):
        end = L - m + 1 + j
        start = max(0, end - window) if window else 0
        if end <= start:
            continue
        for h in range(H):
            kk, vv = k[h // (H // K), start:end], v[h // (H // K), start:end]
            x = kk @ q[j, h] * scale
            mag_s[j, h] = np.max(np.abs(kk) @ np.abs(q[j, h])) * abs(scale)
            top = x.max()
            p = np.exp(x - top)
            lse[j, h] = top + math.log(p.sum())
            p /= p.sum()
            out[j, h] = p @ vv
            mag_o[j, h] = p @ np.abs(vv)
    return out, lse, mag_s, mag_o


class Books:
    """The page calls on Python integers.  content[p]: which page's original content page p holds."""

    def __init__(self, cache):
        self.page = cache.page
        self.table, self.lens, self.refs = (t.cpu().numpy().astype(np.int64) for t in (cache.table, cache.lens, cache.refs))
        self.content = np.arange(len(self.refs))

    def pages_of(self, length):
        return -(-length // self.page)

    def _try(self, f):
        """all or nothing"""
        keep = [a.copy() for a in (self.table, self.lens, self.refs, self.content)]
        try:
            return f(), 0
        except _Refused as e:
            self.table, self.lens, self.refs, self.content = keep
            return None, e.bit

    def _take(self):
        free = np.flatnonzero(self.refs <= 0)
        if len(free) == 0:
            raise _Refused(si.SI_CACHE_NO_PAGES)
        self.refs[free[0]] = 1
        return int(free[0])

    def trim(self, seqs, keep=None):
        status = 0
        for i, s in enumerate(seqs):
            k = 0 if keep is None else keep[i]
            if k < 0:
                status |= si.SI_CACHE_BAD_LEN
            elif not 0 <= s < len(self.lens):
                status |= si.SI_CACHE_BAD_SEQ
            elif k > self.lens[s]:
                status |= si.SI_CACHE_BAD_LEN
            else:
                for j in range(self.pages_of(k), self.pages_of(self.lens[s])):
                    self.refs[self.table[s, j]] -= 1
                    self.table[s, j] = -1
                self.lens[s] = k
        return status

    def extend(self, seqs, counts, capacity):
        def f():
            out, seen = [], set()
            for s, m in zip(seqs, counts):
                if not 0 <= s < len(self.lens) or s in seen:
                    raise _Refused(si.SI_CACHE_BAD_SEQ)
                seen.add(s)
                if m < 0 or self.lens[s] + m > self.table.shape[1] * self.page:
                    raise _Refused(si.SI_CACHE_BAD_LEN)
            if sum(counts) > capacity:
                raise _Refused(si.SI_CACHE_NO_ROOM)
            for s, m in zip(seqs, counts):
                for p in range(self.lens[s], self.lens[s] + m):
                    j = p // self.page
                    old = self.table[s, j]
                    if p % self.page == 0:
                        self.table[s, j] = self._take()
                    elif self.refs[old] > 1:
                        new = self._take()
                        self.content[new] = self.content[old]
                        self.refs[old] -= 1
                        self.table[s, j] = new
                    out.append((s, p))
                self.lens[s] += m
            return out
        out, status = self._try(f)
        out = out or []
        return out + [(-1, -1)] * (capacity - len(out)), status

    def fork(self, parents, children):
        def f():
            if len(set(children)) < len(children) or set(children) & set(parents):
                raise _Refused(si.SI_CACHE_BAD_SEQ)
            for a, b in zip(parents, children):
                if not (0 <= a < len(self.lens) and 0 <= b < len(self.lens)):
                    raise _Refused(si.SI_CACHE_BAD_SEQ)
                if self.lens[b] != 0:
                    raise _Refused(si.SI_CACHE_BAD_LEN)
            for a, b in zip(parents, children):
                for j in range(self.pages_of(self.lens[a])):
                    p = self.table[a, j]
                    if (j + 1) * self.page > self.lens[a]:
                        new = self._take()
                        self.content[new] = self.content[p]
                        p = new
                    else:
                        self.refs[p] += 1
                    self.table[b, j] = p
                self.lens[b] = self.lens[a]
        return self._try(f)[1]

    def compact(self):
        """(new number of each page or -1, number in use)"""
        used = self.refs > 0
        m = int(used.sum())
        place = np.full(len(self.refs), -1)
        holes = [p for p in range(m) if not used[p]]
        for p in np.flatnonzero(used):
            place[p] = p if p < m else holes.pop(0)
        return place, m


class _Refused(Exception):
    def __init__(self, bit):
        self.bit = bit
