"""Plain 64-bit implementations of the 4-bit cache's operators and of sampled
acceptance, written from their definitions in include/ppd.h (numpy; the codes
are defined by float32 operations, which numpy's are).  They share no code with
the library."""
import numpy as np
import torch

BLOCK, BYTES = 32, 4608


def bf16(x):
    """float32 array -> the float32 values of its bfloat16 rounding."""
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).bfloat16().float().numpy()


def _word(x):
    return np.ascontiguousarray(x, np.float32).view(np.uint32) >> 16


def quantize(rows):
    """rows float32 [n][128] (bfloat16 values) -> codes uint32 [n][128], scale
    and zero float32 [n][2] (bfloat16 values)."""
    g = np.asarray(rows, np.float32).reshape(-1, 2, 64)
    with np.errstate(all="ignore"):
        lo, hi = g.min(-1), g.max(-1)
        r = hi - lo
        bad = ~np.isfinite(g).all(-1) | ~np.isfinite(r)
        s = np.where(bad, np.float32("nan"), bf16(r / np.float32(15)))
        z = np.where(bad, np.float32(0), lo)
        q = np.rint((g - z[..., None]) / s[..., None])
        c = np.where(s[..., None] > 0, np.minimum(q, 15), 0)
        c = np.where(np.isnan(c), 0, c)
    return c.astype(np.uint32).reshape(-1, 128), s, z


def held(c, s, z, dtype=np.float64):
    j = np.arange(128) // 64
    with np.errstate(all="ignore"):
        return c.astype(dtype) * s.astype(dtype)[:, j] + z.astype(dtype)[:, j]


def _key_word(p, d):
    """(word of a block, bit) of dim d of the key at position p (of 32)."""
    lane = 4 * (p // 8) + p % 4 + 16 * (d % 32 // 8)
    e = d % 8
    return (p // 4 % 2 * 64 + lane) * 4 + d // 32, 4 * (e // 2) + 16 * (e % 2)


def _value_word(p, d):
    lane = d % 16 + 16 * (p // 8)
    e = p % 8
    return 512 + (d // 64 * 64 + lane) * 4 + d // 16 % 4, 4 * (e // 2) + 16 * (e % 2)


def store(words, pos, key_rows, value_rows):
    """Rows float32 [n][128] to positions pos.. of one head's blocks (uint32
    [nb][1152], changed in place)."""
    d = np.arange(128)
    for which, rows in ((0, key_rows), (1, value_rows)):
        c, s, z = quantize(rows)
        sz = _word(s) | (_word(z) << 16)
        sz = np.where(np.isnan(s), np.uint32(0x7fc0), sz)
        for i in range(len(c)):
            b, p = divmod(pos + i, BLOCK)
            w, bit = np.broadcast_arrays(*(_key_word if which == 0 else _value_word)(p, d))
            for k in range(128):
                x = int(words[b, w[k]])
                words[b, w[k]] = (x & ~(15 << int(bit[k])) & 0xffffffff) | int(c[i, k]) << int(bit[k])
            words[b, 1024 + 64 * which + 2 * p:1024 + 64 * which + 2 * p + 2] = sz[i]


def load(words, n, dtype=np.float64):
    """The held keys and values [n][128] of one head's blocks."""
    pos = np.arange(n)
    b, p = (pos // BLOCK)[:, None], (pos % BLOCK)[:, None]
    d = np.arange(128)[None]
    out = []
    for which, at in ((0, _key_word), (1, _value_word)):
        w, bit = at(p, d)
        c = (words[b, w] >> np.asarray(bit, np.uint32)) & 15
        sz = words[b, 1024 + 64 * which + 2 * p + np.arange(2)[None]]
        s = (sz << np.uint32(16)).view(np.float32)
        z = (sz & np.uint32(0xffff0000)).view(np.float32)
        out.append(held(c, s, z, dtype))
    return out


def heads_of(blocks):
    """Device blocks [layers][heads][nb][4608] -> uint32 [layers][heads][nb][1152]."""
    return np.ascontiguousarray(blocks.cpu().numpy()).view(np.uint32)


def mask_bits(mask, T):
    m = np.asarray(mask).view(np.uint64)
    j = np.arange(T)
    return ((m[:, j // 64] >> (j % 64).astype(np.uint64)) & np.uint64(1)).astype(bool)


def attention(q, k, v, kt, vt, vis):
    """One head: q [T][128], prefix k, v [L][128], tree rows kt, vt [T][128], vis
    [T][T] -> out [T][128], lse [T]; rows that see nothing: 0, -inf."""
    T, L = len(q), len(k)
    s = q @ np.concatenate((k, kt)).T / np.sqrt(128.0)
    s[:, L:][~vis] = -np.inf
    out, lse = np.zeros((T, 128)), np.full(T, -np.inf)
    vv = np.concatenate((v, vt))
    for t in range(T):
        on = s[t] > -np.inf
        if on.any():
            m = s[t][on].max()
            p = np.exp(s[t][on] - m)
            out[t] = p @ vv[on] / p.sum()
            lse[t] = m + np.log(p.sum())
    return out, lse


def score(q, lse, k, kt, path, base):
    """One kv head: q [T][G][128], lse [T][G], prefix k [L][128], tree keys kt
    [T][128] -> sums of the L + len(path) positions."""
    L, n = len(k), len(path)
    keys = np.concatenate((k, kt[path])) if n else k
    out = np.concatenate((np.asarray(base[:L], np.float64), np.zeros(n)))
    for i, node in enumerate(path):
        w = np.exp(q[node] @ keys[:L + i + 1].T / np.sqrt(128.0) - lse[node][:, None])
        out[:L + i + 1] += w.sum(0)
    return out


def keep(score, L, budget, n_sink, n_recent):
    """Kept positions, rising: first, last and, of the others, the largest
    (equal: the smaller position; NaN last)."""
    n = min(L, budget)
    first = set(range(min(n_sink, L))) | set(range(max(0, L - n_recent), L))
    rest = [i for i in range(L) if i not in first]
    rest.sort(key=lambda i: (np.isnan(score[i]), -score[i] if not np.isnan(score[i]) else 0.0, i))
    return sorted(first | set(rest[:max(0, n - len(first))]))


def weights(row, temperature):
    x = np.asarray(row, np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    m = x.max()
    if m == -np.inf:
        return np.zeros(len(x))
    with np.errstate(invalid="ignore"):
        return np.where(x == m, 1.0, np.exp((x - m) / np.float64(np.float32(temperature))))


def accept_sample(parent, ids, vocab, logits, temperature, draft, u):
    """-> path, bonus token, flagged (a NaN, or a row without weight, on the path)."""
    T = len(parent)
    node, path, flagged = 0, [0], False
    while True:
        w = weights(logits[node], temperature)
        flagged |= bool(np.isnan(logits[node]).any()) or not w.any()
        r, took = w.copy(), -1
        for c in range(node + 1, T):
            if parent[c] != node or not 0 <= ids[c] < vocab or not w.any():
                continue
            x = ids[c]
            q = np.zeros(vocab)
            if draft is None:
                q[x] = 1.0
            else:
                q = np.where(draft[node] > 0, draft[node], 0).astype(np.float64)
            if float(u[c]) * q[x] * r.sum() < r[x]:
                took = c
                break
            r = np.where(q == 1.0, 0.0, r) if draft is None else np.maximum(r - r.sum() * q, 0.0)
        if took < 0:
            break
        node = took
        path.append(node)
    if not r.sum() > 0:
        r = w
    if not r.any():
        return path, 0, flagged
    over = np.cumsum(r) > float(u[0]) * r.sum()
    return path, int(np.argmax(over)) if over.any() else int(np.flatnonzero(r)[-1]), flagged
