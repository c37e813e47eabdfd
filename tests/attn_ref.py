"""Plain 64-bit forms of the 8-bit cache operators (numpy), and the random caches
their tests run on."""
import numpy as np
import torch

SMALLEST = 2.0 ** -64

# The e4m3 numbers by code: sign, 4 exponent bits (bias 7), 3 fraction bits.
_MAG = np.array([(8 + c % 8) * 2.0 ** (c // 8 - 10) if c >= 8 else c * 2.0 ** -9
                 for c in range(127)])
VALUE = np.concatenate([_MAG, [np.nan], -_MAG, [np.nan]])


def encode(x):
    """Codes of the nearest e4m3 numbers, ties to the even code; NaN keeps its
    sign bit clear."""
    a = np.abs(x)
    hi = np.searchsorted(_MAG, np.where(np.isnan(a), 0, a)).clip(0, 126)
    lo = (hi - 1).clip(0)
    below, above = a - _MAG[lo], _MAG[hi] - a
    with np.errstate(invalid="ignore"):
        take_lo = (below < above) | ((below == above) & (lo % 2 == 0))
    c = np.where(take_lo, lo, hi)
    c = np.where(np.signbit(x), c + 128, c)
    return np.where(np.isnan(x), 127, c).astype(np.uint8)


def same_codes(a, b):
    """Equal codes, where the two NaNs count as one."""
    return bool(np.all((a == b) | (((a & 127) == 127) & ((b & 127) == 127))))


def power_for(x):
    """The smallest power of two, at least SMALLEST, whose 448-fold holds all of x
    (NaN counts for nothing)."""
    m = np.nanmax(np.abs(x), initial=0.0) if x.size else 0.0
    p = SMALLEST
    while 448 * p < m:
        p *= 2
    return p


LIMIT = {"f16": 0.9375 * 2.0 ** 16, "bf16": 0.9375 * 2.0 ** 128}
TDTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}


class Cache8:
    """An 8-bit cache on the host: codes, scales, table and companions."""

    def __init__(self, kind, L, H, D, B, cap, bs, rng, *, spare=3, companions=False, holes=()):
        self.kind, self.L, self.H, self.D, self.B, self.bs = kind, L, H, D, B, bs
        self.table = None
        if kind == "paged":
            self.mb = -(-cap // bs)
            self.cap = self.mb * bs
            self.nblocks = B * self.mb + spare
            self.table = rng.permutation(self.nblocks)[:B * self.mb].reshape(B, self.mb).astype(
                np.int32)
            for b, j, v in holes:
                self.table[b, j] = v
            shape, scales = (L, 2, self.nblocks, H, bs, D), (L, 2, self.nblocks, H)
        else:
            self.cap = cap
            shape, scales = (L, 2, B, H, cap, D), (L, 2, B, H, -(-cap // bs))
        self.codes = encode(np.clip(rng.normal(size=shape) * 90, -448, 448))
        self.scale = np.ldexp(1.0, rng.integers(-8, -5, size=scales)).astype(np.float32)
        slots = (L, B, H, self.cap)
        self.weight = rng.random(slots).astype(np.float32) if companions else None
        self.position = np.cumsum(rng.integers(1, 4, size=slots), -1).astype(np.int32) \
            if companions else None

    def place(self, b, j):
        """(index into codes and scale for a block of a sequence) or None."""
        if self.kind == "paged":
            at = int(self.table[b, j])
            return at if 0 <= at < self.nblocks else None
        return j

    def block(self, l, kv, b, h, j):
        """Views of one block's codes [slots, D] and its scale's array and index."""
        at = self.place(b, j)
        if at is None:
            return None
        if self.kind == "paged":
            return self.codes[l, kv, at, h], (self.scale, (l, kv, at, h))
        return (self.codes[l, kv, b, h, j * self.bs:(j + 1) * self.bs],
                (self.scale, (l, kv, b, h, j)))

    def values(self, l, kv, b, h, n):
        """Values [n, D] in 64 bits, and which of the slots are mapped."""
        x, ok = np.zeros((n, self.D)), np.ones(n, bool)
        for j in range(-(-n // self.bs)):
            lo, hi = j * self.bs, min(n, (j + 1) * self.bs)
            blk = self.block(l, kv, b, h, j)
            if blk is None:
                ok[lo:hi] = False
                continue
            arr, at = blk[1]
            x[lo:hi] = VALUE[blk[0][:hi - lo]] * float(arr[at])
        return x, ok

    def device(self, dv, attn):
        """The descriptor on the GPU, and its tensors."""
        t = {"codes": torch.from_numpy(self.codes).cuda(),
             "scale": torch.from_numpy(self.scale).cuda()}
        for name in ("table", "weight", "position"):
            x = getattr(self, name)
            t[name] = None if x is None else torch.from_numpy(x).cuda()
        paged = self.kind == "paged"
        c = dv.Cache(dv.DV_PAGED if paged else dv.DV_DENSE, self.L, self.H, self.D, self.B,
                     [t["codes"]], elem_bytes=1, max_seq=0 if paged else self.cap,
                     block_size=self.bs if paged else 0,
                     num_blocks=self.nblocks if paged else 0, max_blocks=self.mb if paged else 0,
                     block_tables=[t["table"]] if paged else None)
        q = attn.QuantCache(c, [t["scale"]], scale_block=self.bs,
                            weights=None if t["weight"] is None else [t["weight"]],
                            positions=None if t["position"] is None else [t["position"]])
        return q, t


def quant_in(c, l0, l1, t0, t1, wire, dtype):
    """Appends to the host cache; wire: float64 [l1 - l0, 2, heads * tokens, D]."""
    first = 0
    for b in range(c.B):
        a, e = int(t0[b]), int(t1[b])
        n = e - a
        if n == 0:
            continue
        x = wire[:, :, first * c.H:(first + n) * c.H].reshape(l1 - l0, 2, c.H, n, c.D)
        first += n
        x = np.clip(x, -LIMIT[dtype], LIMIT[dtype])
        for l in range(l0, l1):
            for h in range(c.H):
                if c.position is not None:
                    p = c.position[l, b, h]
                    p[a:e] = (p[a - 1] + 1 if a else 0) + np.arange(n)
                if c.weight is not None:
                    c.weight[l, b, h, a:e] = 0
                for kv in range(2):
                    for j in range(a // c.bs, -(-e // c.bs)):
                        blk = c.block(l, kv, b, h, j)
                        if blk is None:
                            continue
                        codes, (arr, at) = blk
                        lo, hi = max(a, j * c.bs), min(e, (j + 1) * c.bs)
                        new = x[l - l0, kv, h, lo - a:hi - a]
                        p, held = power_for(new), lo - j * c.bs
                        if held:
                            old = float(arr[at])
                            p = max(p, old)
                            if p > old:
                                codes[:held] = encode(VALUE[codes[:held]] * (old / p))
                        arr[at] = p
                        codes[held:hi - j * c.bs] = encode(new / p)


def attend(c, layer, q_len, kv_len, q, scale, slopes=None):
    """q: float64 [tokens, q_heads, D].  Returns out, the sum of p |v| (what errors
    of the probabilities scale with), lse and the weights received."""
    hq = q.shape[1]
    G = hq // c.H
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    got = np.zeros((c.B, c.H, c.cap))
    first = 0
    with np.errstate(invalid="ignore"):
        for b in range(c.B):
            n, m = int(kv_len[b]), int(q_len[b])
            for h in range(c.H):
                if m == 0:
                    continue
                K, ok = c.values(layer, 0, b, h, n)
                V, _ = c.values(layer, 1, b, h, n)
                pos = np.arange(n) if c.position is None else c.position[layer, b, h, :n]
                for i in range(m):
                    a = n - m + i
                    sees = (np.arange(n) <= a) & ok
                    if not sees.any():
                        continue
                    for g in range(h * G, (h + 1) * G):
                        s = K[sees] @ q[first + i, g] * scale
                        if slopes is not None:
                            s = s + slopes[g] * (pos[sees] - pos[a])
                        top = s.max()
                        p = np.exp(s - top)
                        lse[first + i, g] = top + np.log(p.sum())
                        p = p / p.sum()
                        out[first + i, g] = p @ V[sees]
                        mass[first + i, g] = p @ np.abs(V[sees])
                        got[b, h, :n][sees] += p
            first += m
    return out, mass, lse, got


def evict(c, d, l0, l1, length, keep, recent, stride):
    """Evicts from host cache c into d (which may be c); returns the slots kept."""
    kept = np.full((l1 - l0, c.B, c.H, stride), -1, np.int32)
    for l in range(l0, l1):
        for b in range(c.B):
            n = int(length[b])
            k = min(n, int(keep[b]))
            r = min(recent, k)
            for h in range(c.H):
                w = c.weight[l, b, h, :n - r].astype(np.float64)
                w = np.where(np.isnan(w), -np.inf, w)
                # NaN below every number, -infinity included
                rank = np.lexsort((np.arange(n - r), -w,
                                   np.isnan(c.weight[l, b, h, :n - r])))
                rows = np.concatenate([np.sort(rank[:k - r]), np.arange(n - r, n)]).astype(int)
                kept[l - l0, b, h, :k] = rows
                kv = [c.values(l, half, b, h, n)[0][rows] for half in (0, 1)]
                weights = c.weight[l, b, h, rows].copy()
                pos = rows if c.position is None else c.position[l, b, h, rows].copy()
                if d.weight is not None:
                    d.weight[l, b, h, :k] = weights
                if d.position is not None:
                    d.position[l, b, h, :k] = pos
                for half in (0, 1):
                    for j in range(-(-k // d.bs)):
                        blk = d.block(l, half, b, h, j)
                        if blk is None:
                            continue
                        x = kv[half][j * d.bs:(j + 1) * d.bs]
                        codes, (arr, at) = blk
                        arr[at] = power_for(x)
                        codes[:len(x)] = encode(x / float(arr[at]))
    return kept
