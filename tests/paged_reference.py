"""Plain 64-bit implementations of the 4-bit cache's operators, written from the format's definition: what the device is
compared with."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def decode(codes, scales):
    """uint8 codes [..., dh / 2] and exponents [..., dh / 32] as the values they stand for."""
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = GRID[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    e = np.repeat(scales.astype(np.int64), 32, -1)
    return np.where(e == 255, np.nan, np.ldexp(v, np.minimum(e, 254) - 127))


def encode(x):
    """float32 x [..., dh] to codes and exponents."""
    b = x.astype(np.float32).reshape(*x.shape[:-1], -1, 32)
    bad = ~np.isfinite(b).all(-1)
    a = np.where(np.isfinite(b), np.abs(b), 0).astype(np.float64)
    top = a.max(-1)
    m, p = np.frexp(np.where(top > 0, top, 1.0))            # top = m 2^p, m in [1/2, 1)
    e = np.where(top > 0, p - 1 + (m > 0.875) - 2, -1000)
    e = np.maximum(e, -100)
    y = np.ldexp(a, -e[..., None])
    d = np.abs(y[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    code = np.where(d == best, np.where(np.arange(8) % 2 == 0, 0, 100) + np.arange(8), 1000).argmin(-1)   # ties: the even code
    code = code + 8 * np.signbit(b)
    code = np.where(bad[..., None], 0, code).reshape(*x.shape[:-1], -1).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), np.where(bad, 255, e + 127).astype(np.uint8)


def rotate(x, cos, sin):
    """float32, product by product (the device rounds each of them)."""
    h = x.shape[-1] // 2
    a, b = x[..., :h].astype(np.float32), x[..., h:].astype(np.float32)
    return np.concatenate([a * cos - b * sin, b * cos + a * sin], -1)


class Cache:
    """Pools, page table and lengths as numpy arrays."""

    def __init__(self, rng, layers, batch, kv_heads, page, dh, lengths, room, spare=2, shuffle=True):
        per = [-(-(int(c) + room) // page) for c in lengths]
        n = sum(per) + spare
        order = rng.permutation(n) if shuffle else np.arange(n)
        self.page, self.dh, self.kv = page, dh, kv_heads
        self.table = np.full((batch, max(per)), 0, np.int32)
        at = 0
        for b in range(batch):
            self.table[b, :per[b]] = order[at:at + per[b]]
            at += per[b]
        self.len = np.array(lengths, np.int32)
        shp = (layers, n, kv_heads, page)
        self.pool = {}
        for name in ("k", "v"):
            self.pool[name] = rng.integers(0, 256, shp + (dh // 2,), dtype=np.uint8)
            self.pool[name + "_scale"] = rng.integers(123, 129, shp + (dh // 32,), dtype=np.uint8)

    def rows(self, name, layer, b, first, n):
        """Copies of n slots of a sequence: [n, kv, ...]."""
        s = np.arange(first, first + n)
        return self.pool[name][layer][self.table[b][s // self.page], :, s % self.page]

    def put(self, name, layer, b, slot, x):
        self.pool[name][layer][self.table[b][slot // self.page], :, slot % self.page] = x

    def values(self, name, layer, b, first, n):
        return decode(self.rows(name, layer, b, first, n), self.rows(name + "_scale", layer, b, first, n))

    def device(self):
        import torch
        from paper_2408_08146_amd import PagedCache
        t = {k: torch.from_numpy(v.copy()).cuda() for k, v in self.pool.items()}
        table, length = torch.from_numpy(self.table).cuda(), torch.from_numpy(self.len).cuda()
        return PagedCache(t["k"], t["v"], t["k_scale"], t["v_scale"], table, length), t, length

    def append(self, layer, k, v, cos, sin, depth=None, n_new=None):
        """k, v float32 [batch, rows, kv, dh]."""
        for b in range(k.shape[0]):
            for i in range(k.shape[1] if n_new is None else min(k.shape[1], n_new[b])):
                pos = self.len[b] + (i if depth is None else depth[i])
                for name, x in (("k", rotate(k[b, i], cos[pos], sin[pos])), ("v", v[b, i])):
                    c, s = encode(x)
                    self.put(name, layer, b, self.len[b] + i, c)
                    self.put(name + "_scale", layer, b, self.len[b] + i, s)

    def commit(self, accept_len, path):
        for b, a in enumerate(accept_len):
            for i in range(1, a + 1):
                for name in self.pool:
                    for layer in range(self.pool[name].shape[0]):
                        self.put(name, layer, b, self.len[b] + i, self.rows(name, layer, b, self.len[b] + path[b][i], 1)[0])
        self.len = self.len + np.array(accept_len, np.int32) + 1

    def attend(self, layer, q, seen, scale, max_len=None):
        """q float64 [batch, rows, heads, dh]; seen [batch][rows][rows] truth values over the new rows -> [batch, rows, heads, dh]."""
        B, T, H, D = q.shape
        out = np.zeros(q.shape)
        for b in range(B):
            C = int(self.len[b])
            n = C + T if max_len is None else min(C + T, max_len)
            k, v = self.values("k", layer, b, 0, n), self.values("v", layer, b, 0, n)
            for t in range(T):
                vis = np.concatenate([np.ones(C, bool), np.asarray(seen[b][t], bool)])[:n]
                if not vis.any():
                    continue
                for h in range(H):
                    kh, vh = k[vis, h // (H // self.kv)], v[vis, h // (H // self.kv)]
                    s = kh @ q[b, t, h] * scale
                    p = np.exp(s - s.max())
                    out[b, t, h] = (p / p.sum()) @ vh
        return out
