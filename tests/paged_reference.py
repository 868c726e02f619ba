"""Plain 64-bit forms of the paged cache's calls, on the CPU, written from
include/ppd.h: element addresses, page tables, rows into pages, attention over
pages and the choice of pages."""
import math

import numpy as np
import torch

D = 128


def key_at(u, d):
    return (((u // 4 % 2) * 4 + d // 32) * 64 + 16 * (d // 8 % 4) + 4 * (u // 8) + u % 4) * 8 + d % 8


def value_at(u, d):
    return ((d // 16) * 64 + 16 * (u // 8) + d % 16) * 8 + u % 8


_U, _D = np.meshgrid(np.arange(32), np.arange(D), indexing="ij")
KEY, VALUE = key_at(_U, _D), value_at(_U, _D)  # [32][128]


def rows_of(pages, pt, s, layer, head, n, page):
    """Keys and values [n][128] (the pages' type) of sequence s, from the pages
    [layers][n_pages][heads][page / 32][2][4096] (CPU) by its table's row."""
    if n == 0:
        return (torch.empty((0, D), dtype=pages.dtype),) * 2
    m = -(-n // page)
    b = pages[layer, pt[s, :m].long(), head].reshape(m * (page // 32), 2, 4096)
    return b[:, 0][:, torch.from_numpy(KEY)].reshape(-1, D)[:n], b[:, 1][:, torch.from_numpy(VALUE)].reshape(-1, D)[:n]


def put(pages, layer, page_no, head, off, k, v):
    """One position's key and value [128] into the pages."""
    b = pages[layer, page_no, head, off // 32]
    b[0, torch.from_numpy(KEY[off % 32])] = k
    b[1, torch.from_numpy(VALUE[off % 32])] = v


def tables(table, length, add, ring, state, page, n_slots, slots):
    """What ppd_paged_tables leaves: (table, len, ring, state, start, slots,
    refused), from numpy int32 arrays, which stay as they are."""
    table, ring, slots = table.copy(), ring.copy(), slots.copy()
    n_pages, width = len(ring), table.shape[1]
    first, count = int(state[0]), int(state[1])
    out, start, back, asked, popped, refused = [], [0], [], 0, 0, False
    for s, (n, a) in enumerate(zip(length.tolist(), add.tolist())):
        old = -(-n // page)
        start.append(start[-1] + max(a, 0))
        if a < 0:
            back += table[s, :old].tolist()
            out.append(0)
            continue
        new = -(-(n + a) // page)
        ok = new <= width and start[-1] <= n_slots
        if ok:
            asked += new - old
            ok = new == old or asked <= count
        if not ok:
            refused = True
            slots[start[-2]:min(start[-1], n_slots)] = -1
            out.append(n)
            continue
        for j in range(old, new):
            table[s, j] = ring[(first + popped) % n_pages]
            popped += 1
        for t in range(a):
            p = n + t
            slots[start[-2] + t] = table[s, p // page] * page + p % page
        out.append(n + a)
    for i, x in enumerate(back):
        ring[(first + count + i) % n_pages] = x
    state = np.array([(first + popped) % n_pages, count - popped + len(back)], np.int32)
    return table, np.array(out, np.int32), ring, state, np.minimum(start, 2 ** 31 - 1).astype(np.int32), slots, refused


def store(pages, bounds, k, v, start, row_start, path, slots, page):
    """Rows of k [layers][heads][cap][128], v [layers][heads][128][cap] into pages
    and bounds, in place (CPU tensors)."""
    for s in range(len(start) - 1):
        for i in range(start[s], min(start[s + 1], len(slots))):
            slot = int(slots[i])
            if slot < 0 or slot // page >= pages.shape[1]:
                continue
            r = row_start[s] + i - start[s]
            if path is not None:
                r = row_start[s] + path[r]
            at, off = divmod(slot, page)
            for l in range(pages.shape[0]):
                for h in range(pages.shape[2]):
                    put(pages, l, at, h, off, k[l, h, r], v[l, h, :, r])
            if bounds is None:
                continue
            key = k[:, :, r].float()                      # [layers][heads][128]
            lo, hi = bounds[:, at, :, 0].float(), bounds[:, at, :, 1].float()
            # (a NaN has no part, be it a key or what the bounds held)
            lo, hi = torch.where(lo.isnan(), math.inf, lo), torch.where(hi.isnan(), -math.inf, hi)
            if off == 0:
                lo, hi = torch.full_like(key, math.inf), torch.full_like(key, -math.inf)
            bounds[:, at, :, 0] = torch.fmin(lo, key).to(bounds.dtype)
            bounds[:, at, :, 1] = torch.fmax(hi, key).to(bounds.dtype)


def sees(mask, row0, T):
    """[T][T] booleans; mask None: the rows up to itself."""
    if mask is None:
        return torch.tril(torch.ones((T, T))).bool()
    w = [[int(x) & (1 << 64) - 1 for x in m] for m in mask[row0:row0 + T].tolist()]
    return torch.tensor([[w[i][j // 64] >> (j % 64) & 1 for j in range(T)] for i in range(T)]).bool().reshape(T, T)


class Attention:
    """out, lse in float64 of every row, what each may be off by, and which rows
    belong to a sequence."""

    def __init__(self, pages, table, length, tk, tv, layer, row_start, q, mask, page, sel=None, n_sel=None):
        n_rows, nh, _ = q.shape
        nkv = pages.shape[2]
        G = nh // nkv
        self.out = torch.full((n_rows, nh, D), math.nan, dtype=torch.float64)
        self.lse = torch.full((n_rows, nh), math.nan, dtype=torch.float64)
        self.tol, self.tol_lse = torch.zeros_like(self.out), torch.zeros_like(self.lse)
        self.mine = torch.zeros(n_rows, dtype=torch.bool)
        small = q.dtype == torch.bfloat16
        for s in range(len(length)):
            t0, T, n = int(row_start[s]), int(row_start[s + 1] - row_start[s]), int(length[s])
            self.mine[t0:t0 + T] = True
            see = sees(mask, t0, T)
            for h in range(nkv):
                k, v = rows_of(pages, table, s, layer, h, n, page)
                if sel is not None:
                    at = torch.tensor([p * page + i for p in sel[s, h, : int(n_sel[s])].tolist() for i in range(page)], dtype=torch.long)
                    at = at[at < n]
                    k, v = k[at], v[at]
                k = torch.cat((k, tk[layer, h, t0:t0 + T])).double()
                v = torch.cat((v, tv[layer, h, :, t0:t0 + T].t())).double()
                m = len(k) - T
                for t in range(T):
                    on = torch.cat((torch.ones(m, dtype=torch.bool), see[t]))
                    kk, vv = k[on], v[on]
                    for a in range(G):
                        x = q[t0 + t, h * G + a].double()
                        y = kk @ x / math.sqrt(D)
                        lse = torch.logsumexp(y, 0) if len(y) else torch.tensor(-math.inf, dtype=torch.float64)
                        w = torch.exp(y - lse)
                        o = w @ vv if len(y) else torch.zeros(D, dtype=torch.float64)
                        self.out[t0 + t, h * G + a], self.lse[t0 + t, h * G + a] = o, lse
                        if not len(y):
                            continue
                        # a score: 128 products added in float32 (and a query's parts), its
                        # exponent and exp2: an error ds; a weight is off by twice that
                        # (its sum too), its parts, and the sums over n terms
                        mag = float((kk.abs() @ x.abs()).max()) / math.sqrt(D)
                        ds = 132 * 2.0 ** -24 * mag + (float(y.abs().max()) + 8) * 2.0 ** -23 + 2.0 ** -22
                        if not small:
                            ds += mag * 2.0 ** -24
                        dw = 2 * ds + 2.0 ** (-16 if small else -24) + 2 * (len(y) + 64) * 2.0 ** -24
                        half = 2.0 ** (-8 if small else -24)
                        self.tol[t0 + t, h * G + a] = half * o.abs() + dw * (w @ vv.abs()) + 1e-30
                        self.tol_lse[t0 + t, h * G + a] = ds + (len(y) + 64) * 2.0 ** -24 + abs(float(lse)) * 2.0 ** -22

    def check(self, out, lse=None, untouched=None):
        """Rows of sequences within tolerance (NaN and infinities alike); others
        as `untouched` = (out, lse) before the call."""
        got = out.cpu()
        for want, tol, g in ((self.out, self.tol, got.double()), (self.lse, self.tol_lse, None if lse is None else lse.cpu().double())):
            if g is None:
                continue
            w, t, x = want[self.mine], tol[self.mine], g[self.mine]
            odd = ~torch.isfinite(w)
            assert torch.equal(torch.isnan(x), torch.isnan(w))
            assert torch.equal(x[odd & ~torch.isnan(w)], w[odd & ~torch.isnan(w)])
            err = (x - w).abs()[~odd]
            assert bool((err <= t[~odd]).all()), float((err - t[~odd]).max())
        if untouched is not None:
            for a, b in zip((out, lse), untouched):
                if a is not None:
                    assert torch.equal(a.cpu()[~self.mine].view(torch.uint8), b.cpu()[~self.mine].view(torch.uint8))


def select(bounds, table, length, row_start, q, layer, page, budget, n_first, n_last):
    """Lists of pages [seqs][kv heads] by the definition, in 64 bits."""
    nkv, G = bounds.shape[2], q.shape[1] // bounds.shape[2]
    out = []
    for s, n in enumerate(length.tolist()):
        m = -(-n // page)
        x = q[int(row_start[s]):int(row_start[s + 1])].double()
        heads = []
        for h in range(nkv):
            y = x[:, h * G:(h + 1) * G].reshape(-1, D)
            pos, neg = y.clamp(min=0).sum(0), y.clamp(max=0).sum(0)
            b = bounds[layer, table[s, :m].long(), h].double()
            score = ((b[:, 1] * pos).sum(1) + (b[:, 0] * neg).sum(1)).tolist()
            rank = sorted(range(m), key=lambda p: (not (p < n_first or p >= m - n_last), math.isnan(score[p]),
                                                   0.0 if math.isnan(score[p]) else -score[p], p))
            heads.append(sorted(rank[:budget]))
        out.append(heads)
    return out
