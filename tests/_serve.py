"""Plain definitions of the serving-step operators in 64 bits (numpy, CPU), and
the cache's page layout written out element by element: what the GPU tests
compare with."""
import numpy as np
import torch

E4M3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()


def bf16(x):
    """To bf16 and back, to nearest even, in float64."""
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(torch.float32).to(torch.bfloat16).double().numpy()


def key_at(t, d, D, elem):
    c = 16 // elem
    return (t // 16 * (D // c) + d // c) * 16 * c + t % 16 * c + d % c


def value_at(t, d, D, elem):
    c = 16 // elem
    return ((t // (4 * c) * (D // 16) + d // 16) * 4 + t % 16 // 4) * 16 * c + d % 16 * c + t % (4 * c) // 16 * 4 + t % 4


def key_exp_at(t):
    return t // 64 * 64 + t % 16 * 4 + t % 64 // 16


def value_exp_at(t):
    return t // 64 * 64 + t % 16 // 4 * 16 + t % 64 // 16 * 4 + t % 4


def quantise(x):
    """E4M3 bytes and the exponent of each row's scale (last axis: a head): the nearest value, ties to the even byte."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.where(np.isfinite(x), np.abs(x), 0.0)
    amax = np.where(np.isinf(x).any(-1), np.finfo(np.float32).max, finite.max(-1))
    e = np.full(amax.shape, -126, dtype=np.int64)
    for n in range(-126, 121):
        e = np.where(amax > 448.0 * 2.0 ** n, n + 1, e)
    e = np.where(amax == 0, 0, e)
    y = np.clip(x / np.exp2(e.astype(np.float64))[..., None], -448, 448)
    grid = E4M3[:127]                                     # 0 .. 448
    mag = np.where(np.isnan(y), 0, np.abs(y))
    hi = np.searchsorted(grid, mag, side="left").clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = mag - grid[lo], grid[hi] - mag
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(y), 127, code) | np.where(np.signbit(y), 128, 0)
    return code.astype(np.uint8), e


class Cache:
    """A cache as values, in slots, and as the bytes of its pages."""

    def __init__(self, pages, heads, D, page, elem, fill=0xFF):
        self.pages, self.heads, self.D, self.page, self.elem = pages, heads, D, page, elem
        self.k = np.full((pages * page, heads, D), np.nan)
        self.v = np.full((pages * page, heads, D), np.nan)
        dt = np.uint8 if elem == 1 else np.uint16
        self.kb, self.vb = (np.full((pages, heads, page * D), fill * (1 if elem == 1 else 0x101), dtype=dt) for _ in range(2))
        self.ke, self.ve = (np.full((pages, heads, page), fill, dtype=np.uint8) for _ in range(2))

    def put(self, slot, k, v):
        """Float64 [heads, D] entries, stored as the library stores them."""
        if not 0 <= slot < self.pages * self.page:
            return
        p, t, d = slot // self.page, slot % self.page, np.arange(self.D)
        for x, vals, data, at, exps, e_at in ((k, self.k, self.kb, key_at, self.ke, key_exp_at),
                                              (v, self.v, self.vb, value_at, self.ve, value_exp_at)):
            where = at(t, d, self.D, self.elem)
            if self.elem == 1:
                code, e = quantise(x)
                data[p][:, where] = code
                exps[p][:, e_at(t)] = e + 127
                vals[slot] = E4M3[code] * np.exp2(e.astype(np.float64))[:, None]
            else:
                b = torch.from_numpy(np.asarray(x)).to(torch.float32).to(torch.bfloat16)
                data[p][:, where] = b.view(torch.int16).numpy().view(np.uint16)
                vals[slot] = b.double().numpy()

    def device(self):
        import paper_2607_04031_amd as tl

        def up(x):
            return torch.from_numpy(x.view(np.int16) if x.dtype == np.uint16 else x.copy()).cuda()

        k, v = up(self.kb), up(self.vb)
        if self.elem == 2:
            return tl.KVCache(k.view(torch.bfloat16), v.view(torch.bfloat16), None, None, self.page, self.heads, self.D)
        return tl.KVCache(k, v, up(self.ke), up(self.ve), self.page, self.heads, self.D)

    def bytes(self):
        return [self.kb, self.vb] + ([self.ke, self.ve] if self.elem == 1 else [])


def device_bytes(c):
    """The bytes of a tl.KVCache as numpy arrays."""
    out = []
    for x in (c.k, c.v, c.k_exp, c.v_exp):
        if x is not None:
            x = x.cpu()
            out.append(x.view(torch.int16).numpy().view(np.uint16) if x.dtype == torch.bfloat16 else x.numpy())
    return out


def rotate(x, positions, inv_freq, sections, interleaved):
    """x [n, heads, D], positions [axes, n]: angles in 64 bits."""
    x = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = positions[axis].astype(np.float64).T * inv_freq.astype(np.float64)       # [n, half]
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    xa, xb = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    return x


def attention(q, cache, table, lens, offsets, scale, mask=None):
    """(outputs, sum of p |v| / sum of p) in 64 bits; q [total, heads, D] float64.  Rows that see nothing: zeros."""
    total, Hq, D = q.shape
    out, size = np.zeros((total, Hq, D)), np.zeros((total, Hq, D))
    G = Hq // cache.heads
    for b in range(len(lens)):
        L = int(lens[b])
        n = int(offsets[b + 1] - offsets[b])
        at = np.array([table[b][t // cache.page] * cache.page + t % cache.page if 0 <= table[b][t // cache.page] < cache.pages else -1
                       for t in range(L)], dtype=np.int64)
        for i in range(n):
            j = np.arange(L) - (L - n)
            if mask is None:
                sees = j <= i
            else:
                row = mask[offsets[b] + i]
                bits = np.array([x < 32 * len(row) and bool(int(row[x // 32]) >> (x % 32) & 1) if x >= 0 else True for x in j], dtype=bool)
                sees = bits
            sees = sees & (at >= 0)
            if not sees.any():
                continue
            k, v = cache.k[at[sees]], cache.v[at[sees]]
            for h in range(Hq):
                s = k[:, h // G] @ q[offsets[b] + i, h] * scale
                p = np.exp(s - s.max())
                out[offsets[b] + i, h] = p @ v[:, h // G] / p.sum()
                size[offsets[b] + i, h] = p @ np.abs(v[:, h // G]) / p.sum()
    return out, size


def verify(logits, offsets, parents, tokens, temperature, uniform, noise, max_nodes, draft=None):
    """(path, counts, next, margin): the walk as it is defined, in 64 bits; margin: how far (relative) the nearest decision
    was from going the other way."""
    B, V = noise.shape
    path, counts, nxt = np.full((B, max_nodes), -1), np.zeros(B, dtype=int), np.full(B, -1)
    margin = np.inf
    for s in range(B):
        first, n = offsets[s], offsets[s + 1] - offsets[s]
        if n == 0:
            continue
        at = 0
        while True:
            path[s, counts[s]] = at
            counts[s] += 1
            z = logits[first + at]
            if temperature[s] > 0:
                p = np.exp((z - z.max()) / temperature[s])
                p /= p.sum()
            else:
                p = np.zeros(V)
                p[np.argmax(z)] = 1.0
            w, m, accepted = p.copy(), 1.0, -1
            for c in range(at + 1, n):
                x = tokens[first + c]
                if parents[first + c] != at or not 0 <= x < V:
                    continue
                q = 1.0 if draft is None else draft[first + at, x]
                lhs = uniform[first + c] * q * m
                if max(lhs, w[x]) > 0 and temperature[s] > 0:
                    margin = min(margin, abs(lhs - w[x]) / max(lhs, w[x]))
                if lhs < w[x]:
                    accepted = c
                    break
                if draft is None:
                    m -= w[x]
                    w[x] = 0.0
                else:
                    w = np.maximum(w / max(m, 1e-30) - draft[first + at], 0.0)
                    m = w.sum()
            if accepted < 0:
                break
            at = accepted
        race = (w if (w > 0).any() else p) / noise[s]
        nxt[s] = np.argmax(race)
        second = np.partition(race, -2)[-2] if V > 1 else 0.0
        if race[nxt[s]] > 0:
            margin = min(margin, 1 - second / race[nxt[s]])
    return path, counts, nxt, margin
