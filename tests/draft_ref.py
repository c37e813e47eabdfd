"""Plain 64-bit forms of the operators over drafted tokens (numpy), and the trees and
distributions their tests run on."""
import numpy as np

from tests import attn_ref as ref


def lines(parent):
    """For each draft the list of itself and its ancestors, or None where it is not there."""
    out = []
    for i, p in enumerate(parent):
        up = [] if p == -1 else out[p] if 0 <= p < i else None
        out.append(None if up is None else up + [i])
    return out


def trees(q_len, rng, shape="tree", broken=0.0):
    """Parents of every sequence's drafts, one after another."""
    parts = []
    for n in q_len:
        i = np.arange(n)
        if shape == "chain":
            p = i - 1
        elif shape == "star":
            p = np.minimum(i - 1, 0)
        elif shape == "roots":
            p = np.where(rng.random(n) < 0.4, -1, (rng.random(n) * i).astype(int))
            p[:1] = -1
        else:
            low = np.maximum(i - 1, 0) // 3
            p = np.where(i == 0, -1, low + (rng.random(n) * np.minimum(i - low, 8)).astype(int))
        if broken:
            bad = rng.random(n) < broken
            p = np.where(bad, rng.choice([-2, 1 << 30, -(1 << 31), 128, 64]), p)
            p = np.where(bad & (rng.random(n) < 0.5), i, p)  # itself
        parts.append(p)
    return np.concatenate(parts + [np.zeros(0)]).astype(np.int32)


def attend_tree(c, layer, q_len, kv_len, parent, q, scale, slopes=None):
    """q: float64 [tokens, q_heads, D].  Returns out, the sum of p |v| and lse."""
    hq = q.shape[1]
    G = hq // c.H
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    first = 0
    with np.errstate(invalid="ignore"):
        for b in range(c.B):
            n, m = int(kv_len[b]), int(q_len[b])
            base = n - m
            family = lines(parent[first:first + m])
            for h in range(c.H):
                if m == 0:
                    continue
                K, ok = c.values(layer, 0, b, h, n)
                V, _ = c.values(layer, 1, b, h, n)
                at = np.arange(n) if c.position is None else c.position[layer, b, h, :n].astype(int)
                before = at[base - 1] if base > 0 else -1
                for i, line in enumerate(family):
                    if line is None:
                        continue
                    sees = np.zeros(n, bool)
                    sees[:base] = True
                    sees[[base + x for x in line]] = True
                    sees &= ok
                    if not sees.any():
                        continue
                    pos = at.astype(np.int64).copy()
                    for depth, x in enumerate(line):
                        pos[base + x] = before + 1 + depth
                    here = before + len(line)
                    for g in range(h * G, (h + 1) * G):
                        s = K[sees] @ q[first + i, g] * scale
                        if slopes is not None:
                            s = s + slopes[g] * (pos[sees] - here)
                        top = s.max()
                        p = np.exp(s - top)
                        lse[first + i, g] = top + np.log(p.sum())
                        p = p / p.sum()
                        out[first + i, g] = p @ V[sees]
                        mass[first + i, g] = p @ np.abs(V[sees])
            first += m
    return out, mass, lse


def target(x, T):
    """The distribution of a row of logits (None: nothing has any probability)."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    top = x.max()
    if top == -np.inf:
        return None
    if T == 0:
        return np.eye(1, len(x), int(np.argmax(x)))[0]
    with np.errstate(invalid="ignore", over="ignore"):
        e = np.where(x == top, 1.0, np.exp((x - top) / T))
    return e / e.sum()


def verify(q_len, parent, token, logits, uniform, temperature=None, drawn=None):
    """The walk as it is defined.  Returns path (-1 past a sequence's count), count, next
    (-2 where a sequence has no drafts), and how near a decision came to its border: the
    smallest distance over what decided it."""
    path, count, follow = np.full(len(parent), -1), [], []
    near = np.inf
    first = 0
    for b, m in enumerate(q_len):
        if m == 0:
            count.append(0)
            follow.append(-2)
            continue
        T = 1.0 if temperature is None else float(temperature[b])
        u = np.asarray(uniform[first:first + m], np.float64)
        u = np.where(u < 1, np.maximum(u, 0), 1.0)  # NaN: 1
        here, line, r = 0, [0], target(logits[first], T)
        for i in range(1, m):
            x = int(token[first + i])
            if parent[first + i] != here or not 0 <= x < logits.shape[1] or r is None:
                continue
            q = None if drawn is None else \
                np.where(drawn[first + here] > 0, drawn[first + here], 0).astype(np.float64)
            side = u[i] * (1.0 if q is None else q[x])
            if side != r[x] and max(side, r[x]) > 0:
                near = min(near, abs(side - r[x]) / max(side, r[x]))
            if side < r[x]:
                here, r = i, target(logits[first + i], T)
                line.append(i)
                continue
            left = np.maximum(r - q, 0) if q is not None else np.where(np.arange(len(r)) == x, 0, r)
            if left.sum() > 0:
                r = left / left.sum()
        if r is None:
            follow.append(-1)
        else:
            sums = np.cumsum(r)
            goal = u[0] * sums[-1]
            past = np.nonzero((sums > goal) & (r > 0))[0]
            follow.append(int(past[0]) if len(past) else int(np.nonzero(r > 0)[0][-1]))
            if 0 < u[0] < 1:
                near = min(near, float(np.abs(sums - goal).min()))
        path[first:first + len(line)] = line
        count.append(len(line))
        first += m
    return path, np.array(count), np.array(follow), near


def kept(path, count, n):
    """The part of a path that counts."""
    out = []
    for x in path[:max(0, min(int(count), n))]:
        if not (out[-1] if out else -1) < x < n:
            break
        out.append(int(x))
    return out


def keep_path(c, l0, l1, q_len, kv_len, path, count):
    """Keeps drafts of the host cache, in place."""
    first = 0
    for b in range(c.B):
        m, base = int(q_len[b]), int(kv_len[b]) - int(q_len[b])
        line = kept(path[first:first + m], count[b], m)
        first += m
        if not line:
            continue
        end = base + len(line)
        for l in range(l0, l1):
            for h in range(c.H):
                if c.weight is not None:
                    w = c.weight[l, b, h]
                    w[base:end] = w[[base + x for x in line]]
                for kv in range(2):
                    fresh = c.values(l, kv, b, h, base + m)[0][[base + x for x in line]]
                    for j in range(base // c.bs, -(-end // c.bs)):
                        blk = c.block(l, kv, b, h, j)
                        if blk is None:
                            continue
                        codes, (arr, at) = blk
                        lo, hi = max(base, j * c.bs), min(end, (j + 1) * c.bs)
                        new, held = fresh[lo - base:hi - base], lo - j * c.bs
                        p = ref.power_for(new)
                        if held:
                            old = float(arr[at])
                            p = max(p, old)
                            if p > old:
                                codes[:held] = ref.encode(ref.VALUE[codes[:held]] * (old / p))
                        arr[at] = p
                        codes[held:hi - j * c.bs] = ref.encode(new / p)


LARGEST = {"f16": 65504.0, "bf16": float(2.0 ** 127 * (2 - 2.0 ** -7))}


def quant_out(c, l0, l1, t0, t1):
    """The wire's values in 64 bits, [l1 - l0, 2, rows, D], and which rows are there."""
    parts, there = [], []
    for b in range(c.B):
        a, e = int(t0[b]), int(t1[b])
        if a == e:
            continue
        x = np.zeros((l1 - l0, 2, c.H, e - a, c.D))
        ok = np.zeros((c.H, e - a), bool)
        for l in range(l0, l1):
            for kv in range(2):
                for h in range(c.H):
                    v, o = c.values(l, kv, b, h, e)
                    x[l - l0, kv, h], ok[h] = v[a:], o[a:]
        parts.append(x.reshape(l1 - l0, 2, -1, c.D))
        there.append(ok.reshape(-1))
    if not parts:
        return np.zeros((l1 - l0, 2, 0, c.D)), np.zeros(0, bool)
    return np.concatenate(parts, 2), np.concatenate(there)
