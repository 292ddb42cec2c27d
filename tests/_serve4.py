"""The 4-bit cache's format and page layout in 64 bits (numpy, CPU), written out element by element: what the GPU tests of
the 4-bit cache compare with.  A Cache4 takes the place of a _serve.Cache in _serve.attention."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E2M1 = np.concatenate([GRID, -GRID])


def quantise(x):
    """Codes and the exponent (biased, 255: NaN) of each 32 elements of the last axis: the nearest value, ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    x = x.reshape(x.shape[:-1] + (-1, 32))
    nan = np.isnan(x).any(-1)
    x = np.where(nan[..., None], 0.0, x)
    amax = np.abs(x).max(-1)
    e = np.full(amax.shape, -126, dtype=np.int64)
    for n in range(-126, 125):
        e = np.where(amax > 6.0 * 2.0 ** n, n + 1, e)
    e = np.where(amax == 0, 0, e)
    y = np.clip(x, -1e300, 1e300) / np.exp2(e.astype(np.float64))[..., None]
    mag = np.minimum(np.abs(y), 6.0)
    hi = np.searchsorted(GRID, mag, side="left").clip(0, 7)
    lo = np.maximum(hi - 1, 0)
    dl, dh = mag - GRID[lo], GRID[hi] - mag
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi) + np.where(np.signbit(y) & ~nan[..., None], 8, 0)
    return code.reshape(code.shape[:-2] + (-1,)), np.where(nan, 255, e + 127)


def values(code, exps):
    """float64 of codes [..., D] and biased exponents [..., D / 32]."""
    scale = np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127))
    return E2M1[code] * np.repeat(scale, 32, axis=-1)


class Cache4:
    """A cache as values, in slots, and as the bytes of its pages; 'fill' is what the bytes hold before anything is stored."""
    elem = 4

    def __init__(self, pages, heads, D, page, fill=0xFF):
        self.pages, self.heads, self.D, self.page = pages, heads, D, page
        self.k = np.full((pages * page, heads, D), np.nan)
        self.v = np.full((pages * page, heads, D), np.nan)
        self.kb, self.vb = (np.full((pages, heads, page * D // 2), fill, dtype=np.uint8) for _ in range(2))
        self.ke, self.ve = (np.full((pages, heads, page * D // 32), fill, dtype=np.uint8) for _ in range(2))

    def put(self, slot, k, v):
        if not 0 <= slot < self.pages * self.page:
            return
        p, t, B = slot // self.page, slot % self.page, self.D // 32
        for is_value, x, vals, data, exps in ((False, k, self.k, self.kb, self.ke), (True, v, self.v, self.vb, self.ve)):
            code, e = quantise(x)
            for d in range(self.D):
                b, r = d // 32, d % 32
                if is_value:
                    at = ((t // 64 * B + b) * 4 + t % 16 // 4) * 256 + r % 16 * 16 + t % 64 // 16 * 4 + t % 4
                    shift = r // 16 * 4
                else:
                    at, shift = (t // 16 * B + b) * 256 + t % 16 * 16 + r // 2, r % 2 * 4
                data[p][:, at] = data[p][:, at] & (0xF0 >> shift) | (code[:, d] << shift).astype(np.uint8)
            for b in range(B):
                at = (t // 64 * B + b) * 64 + (t % 16 // 4 * 16 + t % 64 // 16 * 4 + t % 4 if is_value else t % 16 * 4 + t % 64 // 16)
                exps[p][:, at] = e[:, b]
            vals[slot] = values(code, e)

    def device(self):
        import paper_2607_04031_amd as tl
        return tl.KVCache(*(torch.from_numpy(x.copy()).cuda() for x in self.bytes()), self.page, self.heads, self.D,
                          elem_bytes=tl.TL_KV_E2M1)

    def bytes(self):
        return [self.kb, self.vb, self.ke, self.ve]
