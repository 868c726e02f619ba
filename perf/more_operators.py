"""Operators of a decode loop whose sequences share a paged cache, as cases with
inputs, one pass each in plain torch operations or through the library, and a
64-bit value.

  tables   page tables and slot maps from the sequences' lengths and the tokens
           that each adds or gives back (ppd_paged_tables)
  store    accepted or prompt rows into the pages by the slot map, with the
           pages' key bounds (ppd_paged_store)
  attend   attention of one layer: new tokens -- one of each sequence, or a
           tree's -- over the paged prefixes and their own rows
           (ppd_paged_attention)
  sparse   the same over pages that a score of their key bounds selects
           (ppd_paged_select, ppd_paged_attention)

A page holds 32, 64, 128 or 256 positions of every kv head in blocks of 32:
8 KB of keys and 8 KB of values in the operand order of the matrix instructions.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128            # head dim
BLOCK = 32         # positions of a block
SCALE = 1.0 / math.sqrt(D)
FREE_SLACK = 7     # pages free beyond those needed


# ---------------------------------------------------------------------------
# cases


def _named(name, c):
    return dict(c, name=name) if name else c


def _tables(name, B, page, L, add, ended, scarce):
    """L, add: the longest cached length and the most added tokens; every
    ended-th sequence gives its pages back; scarce: too few free pages."""
    return _named(name, dict(kind="tables", B=B, page=page, L=L, add=add, ended=ended, scarce=scarce))


def _store(name, layers, nkv, page, B, L, add, T):
    """T: tree rows a sequence, of which up to `add` are accepted; 0: prompts of
    `add` rows as they lie in the source."""
    return _named(name, dict(kind="store", layers=layers, nkv=nkv, page=page, B=B, L=L, add=add, T=T))


def _attend(name, nh, nkv, page, B, T, L, ragged, dtype):
    return _named(name, dict(kind="attend", nh=nh, nkv=nkv, page=page, B=B, T=T, L=L, ragged=ragged, dtype=dtype))


def _sparse(name, nh, nkv, page, B, T, L, ragged, dtype, budget, first, last):
    return _named(name, dict(kind="sparse", nh=nh, nkv=nkv, page=page, B=B, T=T, L=L, ragged=ragged, dtype=dtype,
                             budget=budget, first=first, last=last))


def listed():
    return [
        # after a decode step: a few accepted tokens of each of 16 sequences
        _tables("tables_decode_B16", 16, 64, 4096, 6, 0, False),
        # requests that come and go in a large batch, their prompts of up to 4k tokens
        _tables("tables_prompts_B512", 512, 32, 20000, 4096, 5, False),
        # after a decode step: the accepted paths of four 16-node trees, all layers of the 7B shape
        _store("store_7b_B4", 32, 32, 64, 4, 2048, 5, 16),
        # prompts of up to 2k tokens into pages, grouped-query heads
        _store("store_prompts_gqa", 24, 8, 32, 4, 0, 2048, 0),
        # the smallest call: one token of an edge-size model, short context
        _attend("attend_1b4_T1_L200", 16, 16, 32, 1, 1, 200, False, "bf16"),
        # one new token of each of 64 users, prefixes of any length
        _attend("attend_gqa_B64", 32, 8, 64, 64, 1, 8192, True, "bf16"),
        # the 64-node tree of the 7B shape over its 2k prefix
        _attend("attend_7b_T64_L2048", 32, 32, 64, 1, 64, 2048, False, "bf16"),
        # one token over a long prefix, float32 queries
        _attend("attend_gqa_L131072", 32, 8, 128, 1, 1, 131072, False, "f32"),
        # the same prefix length, a small tree, 2048 positions of it
        _sparse("sparse_gqa_L131072", 32, 8, 32, 1, 16, 131072, False, "bf16", 64, 1, 4),
        # eight users with long prefixes, one token each
        _sparse("sparse_7b_B8", 32, 32, 64, 8, 1, 32768, True, "bf16", 48, 1, 2),
        # a short prefix of an edge-size model: where selection costs more than it reads
        _sparse("sparse_1b4_L4000", 16, 16, 32, 1, 1, 4000, False, "f32", 31, 1, 1),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(("tables", "store", "attend", "attend", "attend", "sparse", "sparse"))
    page = rng.choice((32, 32, 64, 64, 128, 256))
    if kind == "tables":
        B = _log(rng, 1, 1024)
        return _tables(None, B, page, _log(rng, 1, 40000), _log(rng, 1, max(1, 2000000 // B) if B > 64 else 4096),
                       rng.choice((0, 0, 2, 3, 7)), rng.random() < 0.25)
    nkv = rng.choice((2, 4, 8, 16, 32, 40))
    if kind == "store":
        layers = rng.randint(1, 32)
        B = _log(rng, 1, 16)
        layers = max(1, min(layers, 4000000 // ((2 * B + 3) * page * nkv)))
        if rng.random() < 0.5:
            T = _log(rng, 1, 128 // B)
            return _store(None, layers, nkv, page, B, min(_log(rng, 1, 2048), 600000 // (layers * nkv * B)),
                          rng.randint(1, min(T, 16)), T)
        add = _log(rng, 1, max(1, 1500000 // (layers * nkv * B)))
        return _store(None, layers, nkv, page, B, rng.randint(0, 100), add, 0)
    nh = nkv * rng.choice([g for g in (1, 2, 4, 8) if g * nkv <= 40])
    B = _log(rng, 1, 64)
    T = _log(rng, 1, max(1, 128 // B)) if rng.random() < 0.5 else 1
    dtype = rng.choice(("bf16", "bf16", "f32"))
    ragged = B > 1 and rng.random() < 0.8
    most = 1048576 // (nkv * B)
    if kind == "attend":
        L = _log(rng, 1, min(131072, most if T * B <= 16 else most // 4))
        return _attend(None, nh, nkv, page, B, T, L, ragged, dtype)
    L = _log(rng, page, max(page, min(131072, most)))
    budget = _log(rng, 2, max(2, 4096 // page))
    first = rng.randint(0, 1)
    return _sparse(None, nh, nkv, page, B, T, L, ragged, dtype, budget, first, rng.randint(0, min(4, budget - first)))


# ---------------------------------------------------------------------------
# what a case fixes: lengths, added tokens (page numbers and values are the seed's)


def _counts(case):
    """Cached lengths, and for `tables` and `store` the tokens added (-1: ended)."""
    c = case
    r = random.Random("%s %s" % (c["kind"], sorted((k, v) for k, v in c.items() if k != "name")))
    B, L = c["B"], c["L"]
    if c["kind"] in ("attend", "sparse"):
        if not c["ragged"]:
            return [L] * B, None
        lens = [_log(r, max(1, L // 64), L) for _ in range(B)]
        lens[r.randrange(B)] = L
        return lens, None
    lens = [_log(r, 1, L) if L > 0 else 0 for _ in range(B)]
    add = [r.randint(1, c["add"]) for _ in range(B)]
    add[r.randrange(B)] = c["add"]
    if c["kind"] == "tables":
        for s in range(B):
            if c["ended"] and s % c["ended"] == c["ended"] - 1:
                add[s] = -1
            elif s % 11 == 10:
                add[s] = 0
    return lens, add


def _ceil(a, b):
    return -(-a // b)


def _needs(c, lens, add):
    return [0 if a < 0 else _ceil(n + a, c["page"]) - _ceil(n, c["page"]) for n, a in zip(lens, add)]


# ---------------------------------------------------------------------------
# pages: [layers][n_pages][kv heads][page / 32][2][4096] bf16.  Keys of a block:
# fragment (tile t, step k), lane l, element e: position 8 (l % 16 / 4) + 4 t +
# l % 4, dim 32 k + 8 (l / 16) + e; values: fragment w, lane l, element e: dim
# 16 w + l % 16, position 8 (l / 16) + e


def _pack(k, v):
    """Rows [.., n, 128] (n % 32 == 0) -> blocks [.., n / 32, 2, 4096]."""
    lead, nb = k.shape[:-2], k.shape[-2] // BLOCK
    i = len(lead) + 1
    own_dims = list(range(i))
    kb = k.reshape(*lead, nb, 4, 2, 4, 4, 4, 8)   # a t b | k g e
    kb = kb.permute(*own_dims, i + 1, i + 3, i + 4, i, i + 2, i + 5).reshape(*lead, nb, 4096)
    vb = v.reshape(*lead, nb, 4, 8, 8, 16)        # g e | w r
    vb = vb.permute(*own_dims, i + 2, i, i + 3, i + 1).reshape(*lead, nb, 4096)
    return torch.stack((kb, vb), -2)


def _unpack(blocks):
    """Blocks [.., nb, 2, 4096] -> keys and values [.., 32 nb, 128]."""
    lead, nb = blocks.shape[:-3], blocks.shape[-3]
    i = len(lead) + 1
    own_dims = list(range(i))
    kb = blocks[..., 0, :].reshape(*lead, nb, 2, 4, 4, 4, 4, 8)   # t k g a b e
    kb = kb.permute(*own_dims, i + 3, i, i + 4, i + 1, i + 2, i + 5).reshape(*lead, nb * BLOCK, D)
    vb = blocks[..., 1, :].reshape(*lead, nb, 8, 4, 16, 8)        # w g r e
    vb = vb.permute(*own_dims, i + 1, i + 3, i, i + 2).reshape(*lead, nb * BLOCK, D)
    return kb, vb


# ---------------------------------------------------------------------------
# inputs


def _gen(seed, *salt):
    h = 0
    for x in salt:
        h = (h * 1000003 + int(x)) % (1 << 31)
    g = torch.Generator("cuda")
    g.manual_seed((seed * 7919 + h) % (1 << 40))
    return g


def _dev(a, dtype=torch.int32):
    return torch.tensor(a, dtype=dtype, device="cuda")


def _offsets(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _mask(r, T):
    """Ancestor bits of a tree of T nodes: small ones grow anywhere, from 16 on
    three of four nodes hang in chains of three."""
    n_cand = max(1, T // 4) if T >= 16 else T
    parent = [-1] + [r.randrange(max(0, i - 6), i) for i in range(1, n_cand)]
    at = 0
    while len(parent) < T:
        up = at % n_cand
        for _ in range(3):
            if len(parent) < T:
                parent.append(up)
                up = len(parent) - 1
        at += 1
    m = np.zeros((T, 2), np.uint64)
    for i in range(T):
        j = i
        while j >= 0:
            m[i, j // 64] |= np.uint64(1 << (j % 64))
            j = parent[j]
    return m


def _tables_of(g, lens, page, n_pages, width):
    """A table of physical pages, dealt in no order, and what is left over."""
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.zeros((len(lens), width), dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(lens):
        k = _ceil(n, page)
        table[s, :k] = order[at:at + k]
        at += k
    return table, order[at:]


def _cap8(n):
    return (n + 7) // 8 * 8


def _pack_heads(k, v, page):
    """Rows [nkv, n, 128], n a multiple of page -> [n / page][nkv][page / 32][2][4096]."""
    nkv, n, _ = k.shape
    b = _pack(k, v)
    return b.reshape(nkv, n // page, page // BLOCK, 2, 4096).transpose(0, 1)


def _prefixes(g, c, lens, table, n_pages):
    """Pages and bounds of one layer.  Keys wander slowly, as neighbouring
    tokens' keys are alike, with some dims larger than others; the rest of the
    pool holds anything."""
    nkv, page = c["nkv"], c["page"]
    pages = torch.randn((1, n_pages, nkv, page // BLOCK, 2, 4096), generator=g, device="cuda").to(torch.bfloat16)
    bounds = torch.zeros((1, n_pages, nkv, 2, D), dtype=torch.bfloat16, device="cuda")
    spread = 0.5 + torch.rand((nkv, 1, D), generator=g, device="cuda")
    for s, n in enumerate(lens):
        if n == 0:
            continue
        full = _ceil(n, page) * page
        drift = torch.randn((nkv, _ceil(full, 16), D), generator=g, device="cuda").repeat_interleave(16, 1)[:, :full]
        k = ((torch.randn((nkv, full, D), generator=g, device="cuda") * 0.7 + drift * 0.7) * spread).to(torch.bfloat16)
        v = torch.randn((nkv, full, D), generator=g, device="cuda").to(torch.bfloat16)
        at = table[s, : full // page].long()
        pages[0, at] = _pack_heads(k, v, page)
        live = k.float()
        lo, hi = live.clone(), live
        lo[:, n:], hi[:, n:] = float("inf"), float("-inf")
        for i, x in enumerate((lo.view(nkv, -1, page, D).amin(2), hi.view(nkv, -1, page, D).amax(2))):
            bounds[0, at, :, i] = x.transpose(0, 1).to(torch.bfloat16)
    return pages, bounds


def prepare(case, seed):
    c = dict(case)
    kind, B, page = c["kind"], c["B"], c["page"]
    lens, add = _counts(c)
    r = random.Random("%s %d" % (kind, seed))
    g = _gen(seed, *[x for x in c.values() if isinstance(x, (int, bool))])
    s = dict(case=c)
    if kind == "tables":
        need = sum(_needs(c, lens, add))
        used = sum(_ceil(n, page) for n in lens)
        free = need // 2 if c["scarce"] else need + FREE_SLACK
        n_pages = used + free
        width = max(_ceil(n + max(a, 0), page) for n, a in zip(lens, add)) + 2
        table, left = _tables_of(g, lens, page, n_pages, width)
        first = r.randrange(n_pages)
        ring = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        ring[(first + torch.arange(free, device="cuda")) % n_pages] = left
        s.update(table=table, ring=ring, state=_dev([first, free]), len=_dev(lens), add=_dev(add),
                 len_out=_dev([0] * B), state_out=_dev([0, 0]), start=_dev([0] * (B + 1)),
                 slots=torch.full((sum(max(a, 0) for a in add) + 5,), -7, dtype=torch.int32, device="cuda"))
    elif kind == "store":
        layers, nkv = c["layers"], c["nkv"]
        # the pages of the rows' sequences alone: those before are not touched
        touched = [_ceil(n + a, page) - n // page for n, a in zip(lens, add)]
        n_pages = sum(touched) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").tolist()
        slots, at = [], 0
        for n, a, k in zip(lens, add, touched):
            slots += [order[at + (n % page + t) // page] * page + (n + t) % page for t in range(a)]
            at += k
        T = c["T"]
        rows = [T] * B if T else add
        total = _cap8(sum(rows))
        s["k"] = torch.randn((layers, nkv, total, D), generator=g, device="cuda").to(torch.bfloat16)
        s["v"] = torch.randn((layers, nkv, D, total), generator=g, device="cuda").to(torch.bfloat16)
        s["pages"] = torch.randn((layers, n_pages, nkv, page // BLOCK, 2, 4096), generator=g, device="cuda").to(torch.bfloat16)
        b = torch.randn((layers, n_pages, nkv, 2, D), generator=g, device="cuda")
        s["bounds"] = torch.stack((b.amin(3), b.amax(3)), 3).to(torch.bfloat16).contiguous()
        s["slots"], s["start"], s["row_start"] = _dev(slots), _dev(_offsets(add)), _dev(_offsets(rows))
        s["path"] = None
        if T:
            path = []
            for a in add:
                p = [0] + sorted(r.sample(range(1, T), a - 1))
                path += p + [-1] * (T - a)
            s["path"] = _dev(path)
    else:
        nh, T = c["nh"], c["T"]
        n_pages = sum(_ceil(n, page) for n in lens) + 2
        width = max(_ceil(n, page) for n in lens) + 1
        table, left = _tables_of(g, lens, page, n_pages, width)
        s["pages"], s["bounds"] = _prefixes(g, c, lens, table, n_pages)
        rows = B * T
        s["tk"] = torch.randn((1, c["nkv"], _cap8(rows), D), generator=g, device="cuda").to(torch.bfloat16)
        s["tv"] = torch.randn((1, c["nkv"], D, _cap8(rows)), generator=g, device="cuda").to(torch.bfloat16)
        q = torch.randn((rows, nh, D), generator=g, device="cuda")
        dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        s["q"] = q.to(dt)
        mask = np.concatenate([_mask(r, T) for _ in range(B)])
        s["mask"] = torch.from_numpy(mask.view(np.int64)).cuda()
        s.update(table=table, len=_dev(lens), row_start=_dev(_offsets([T] * B)), out=torch.zeros((rows, nh, D), dtype=dt, device="cuda"),
                 lse=torch.zeros((rows, nh), device="cuda"), ring=torch.zeros(n_pages, dtype=torch.int32, device="cuda"),
                 state=_dev([0, 0]))
        if kind == "sparse":
            s["sel"] = torch.full((B, c["nkv"], c["budget"]), -1, dtype=torch.int32, device="cuda")
            s["n_sel"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    if own:
        _handles(s)
    return s


def _handles(s):
    import paper_2405_18628_amd as ppd
    c = s["case"]
    kind, B, page = c["kind"], c["B"], c["page"]
    s["ppd"] = ppd

    def workspace(n):
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        ppd.ppd_workspace_init(ws)
        return ws
    if kind == "store":
        s["cache"] = ppd.PagedCache(s["pages"], s["bounds"])
        s["src"] = ppd.KVCache(s["k"], s["v"])
        return
    s["pt"] = ppd.PageTables(s["table"], s["len"], s["ring"], s["state"], page)
    if kind == "tables":
        s["ws"] = workspace(ppd.ppd_paged_tables_workspace_bytes(B))
        return
    s["cache"] = ppd.PagedCache(s["pages"], s["bounds"], ppd.KVCache(s["tk"], s["tv"]))
    s["ws"] = workspace(ppd.ppd_paged_attention_workspace_bytes(c["nh"], c["nkv"], B, B * c["T"]))
    if kind == "sparse":
        s["ws_sel"] = workspace(ppd.ppd_paged_select_workspace_bytes(c["nkv"], B, s["table"].shape[1]))


# ---------------------------------------------------------------------------
# one pass through the library


def _run_own(s):
    c, ppd = s["case"], s["ppd"]
    kind = c["kind"]
    if kind == "tables":
        ppd.ppd_paged_tables(s["pt"], s["add"], s["start"], s["slots"], s["ws"], len_out=s["len_out"],
                             free_state_out=s["state_out"])
        return _tables_out(s, s["table"], s["ring"], s["len_out"], s["state_out"], s["start"], s["slots"])
    if kind == "store":
        ppd.ppd_paged_store(s["cache"], s["src"], s["start"], s["row_start"], s["path"], s["slots"])
        return dict(pages=s["pages"], bounds=s["bounds"])
    if kind == "attend":
        ppd.ppd_paged_attention(s["cache"], 0, s["pt"], s["row_start"], s["q"], s["mask"], s["out"], s["ws"], lse=s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    ppd.ppd_paged_select(s["cache"], 0, s["pt"], s["row_start"], s["q"], c["budget"], c["first"], c["last"], s["sel"],
                         s["n_sel"], s["ws_sel"])
    ppd.ppd_paged_attention(s["cache"], 0, s["pt"], s["row_start"], s["q"], s["mask"], s["out"], s["ws"], lse=s["lse"],
                            sel=s["sel"], n_sel=s["n_sel"])
    return dict(sel=s["sel"], n_sel=s["n_sel"], out=s["out"], lse=s["lse"])


def _tables_out(s, table, ring, len_out, state_out, start, slots):
    return dict(table=table, ring=ring, len=len_out, state=state_out, start=start, slots=slots)


# ---------------------------------------------------------------------------
# the plain form


def _run_tables(s):
    page, table, ring = s["case"]["page"], s["table"].clone(), s["ring"].clone()
    B, width = table.shape
    n_pages, n_slots = ring.numel(), s["slots"].numel()
    n, add = s["len"].long(), s["add"].long()
    first, count = s["state"][0].long(), s["state"][1].long()
    ended = add < 0
    grow = add.clamp(min=0)
    start = torch.cat((torch.zeros(1, dtype=torch.long, device=n.device), grow.cumsum(0)))
    old, new = (n + page - 1) // page, (n + grow + page - 1) // page
    fits = (new <= width) & (start[1:] <= n_slots)
    need = torch.where(fits, new - old, torch.zeros_like(new))
    upto = need.cumsum(0)
    served = fits & ((need == 0) | (upto <= count)) & ~ended
    take = torch.where(served, need, torch.zeros_like(need))
    before = upto - need
    # entries of the tables: column j of sequence s, old <= j < new
    j = torch.arange(width, device=n.device)[None]
    popped = ring[((first + before[:, None] + j - old[:, None]) % n_pages).clamp(min=0)]
    table = torch.where(served[:, None] & (j >= old[:, None]) & (j < new[:, None]), popped, table)
    # rows: the sequence and the token of each, by its place
    at = torch.arange(n_slots, device=n.device)
    total = start[-1]
    sq = torch.searchsorted(start[1:].contiguous(), at, right=True).clamp(max=B - 1)
    pos = (n[sq] + at - start[sq])
    slot = table[sq, (pos // page).clamp(0, width - 1)].long() * page + pos % page
    slots = torch.where(at < total, torch.where(served[sq], slot, torch.full_like(slot, -1)), s["slots"].long())
    # pages given back, behind the free ones, in order
    given = torch.where(ended, old, torch.zeros_like(old))
    g0 = given.cumsum(0) - given
    back = (j < given[:, None])
    place = (first + count + g0[:, None] + j) % n_pages
    ring[place[back]] = table[back]
    taken = take.sum()
    state = torch.stack(((first + taken) % n_pages, count - taken + given.sum())).int()
    length = torch.where(ended, torch.zeros_like(n), n + torch.where(served, grow, torch.zeros_like(grow)))
    return _tables_out(s, table, ring, length.int(), state, start.int(), slots.int())


def _source_rows(s):
    """Row of the source of each stored row."""
    start, row_start = s["start"].long(), s["row_start"].long()
    i = torch.arange(s["slots"].numel(), device=start.device)
    sq = torch.searchsorted(start[1:].contiguous(), i, right=True)
    k = row_start[sq] + i - start[sq]
    return k if s["path"] is None else row_start[sq] + s["path"].long()[k]


def _run_store(s):
    page = s["case"]["page"]
    pages, bounds = s["pages"], s["bounds"].float()
    layers, n_pages, nkv = pages.shape[:3]
    rows = _source_rows(s)
    k, v = s["k"][:, :, rows], s["v"][:, :, :, rows].transpose(2, 3)
    slots = s["slots"].long()
    pg, off = slots // page, slots % page
    hk, hv = _unpack(pages)                                  # [layers][pages][heads][page][128]
    hk, hv = hk.clone(), hv.clone()
    hk[:, pg, :, off] = k.permute(2, 0, 1, 3)
    hv[:, pg, :, off] = v.permute(2, 0, 1, 3)
    # bounds: from nothing where a page's first position is among the rows
    begun = torch.zeros(n_pages, dtype=torch.bool, device=pg.device)
    begun[pg[off == 0]] = True
    x = k.float().permute(2, 0, 1, 3).reshape(len(slots), -1)   # [rows][layers x heads x 128]
    lo = torch.where(begun[:, None], torch.full_like(x[:1], float("inf")), bounds[:, :, :, 0].transpose(0, 1).reshape(n_pages, -1))
    hi = torch.where(begun[:, None], torch.full_like(x[:1], float("-inf")), bounds[:, :, :, 1].transpose(0, 1).reshape(n_pages, -1))
    at = pg[:, None].expand_as(x)
    lo, hi = lo.scatter_reduce(0, at, x, "amin"), hi.scatter_reduce(0, at, x, "amax")
    b = torch.stack([t.view(n_pages, layers, nkv, D).transpose(0, 1) for t in (lo, hi)], 3)
    return dict(pages=_pack(hk, hv), bounds=b.to(torch.bfloat16))


def _bits(mask, T):
    """[rows][T]: whether a row sees node j of its tree."""
    j = torch.arange(T, device=mask.device)
    return (mask[:, j // 64] >> (j % 64) & 1).bool()


def _attention(q, k, v, see, dt):
    """Rows q [nkv][R][128] over keys [nkv][n][128]; see [R][n] or [nkv][R][n]."""
    x = torch.matmul(q, k.transpose(1, 2).contiguous()) * SCALE
    x = torch.where(see, x, torch.full_like(x, float("-inf")))
    m = x.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    e = torch.exp(x - m)
    l = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(l == 0, torch.ones_like(l), l)
    return o.to(dt), (m + torch.log(l))[..., 0].float()


def _select(s):
    """Selected pages of every sequence and kv head, and how many."""
    c = s["case"]
    B, T, nkv, page, budget = c["B"], c["T"], c["nkv"], c["page"], c["budget"]
    q = s["q"].double().view(B, T, nkv, -1, D)
    qp, qm = q.clamp(min=0).sum((1, 3)), q.clamp(max=0).sum((1, 3))          # [B][nkv][128]
    np_ = (s["len"].long() + page - 1) // page
    most = _ceil(c["L"], page)
    bd = s["bounds"][0, s["table"][:, :most].long()].double()               # [B][pages][nkv][2][128]
    score = (bd[:, :, :, 1] * qp[:, None] + bd[:, :, :, 0] * qm[:, None]).sum(-1).transpose(1, 2)
    at, inf = torch.arange(most, device=q.device), float("inf")
    kept = (at < c["first"]) | (at >= np_[:, None] - c["last"])
    score = torch.where(kept[:, None], torch.full_like(score, inf), score)
    score = torch.where((at < np_[:, None])[:, None], score, torch.full_like(score, -inf))
    best = torch.sort(score, dim=2, descending=True, stable=True)[1][:, :, :budget]
    n_sel = np_.clamp(max=budget)
    m = torch.arange(best.shape[2], device=q.device)
    live = (m < n_sel[:, None])[:, None]
    best = torch.sort(torch.where(live, best, torch.full_like(best, most)), dim=2)[0]
    sel = s["sel"].clone()
    sel[:, :, : best.shape[2]] = torch.where(live, best.int(), sel[:, :, : best.shape[2]])
    return sel, n_sel.int()


def _run_attention(s, sel=None, n_sel=None):
    c = s["case"]
    B, T, nkv, nh, page = c["B"], c["T"], c["nkv"], c["nh"], c["page"]
    G = nh // nkv
    dev = s["q"].device
    q = s["q"].float().view(B, T, nkv, G, D).permute(0, 2, 1, 3, 4).reshape(B * nkv, T * G, D)
    most = _ceil(c["L"], page)
    # logical pages [B][nkv or 1][m] and whether they count
    if sel is None:
        pick = torch.arange(most, device=dev).expand(B, 1, most)
        counts = torch.ones_like(pick, dtype=torch.bool)
        blocks = s["pages"][0, s["table"][:, :most].long()].transpose(1, 2)
    else:
        counts = (torch.arange(sel.shape[2], device=dev) < n_sel[:, None])[:, None].expand_as(sel)
        pick = torch.where(counts, sel, torch.zeros_like(sel)).long()
        phys = s["table"].long()[torch.arange(B, device=dev)[:, None, None], pick]
        blocks = s["pages"][0, phys, torch.arange(nkv, device=dev)[:, None]]
    k, v = _unpack(blocks.reshape(B, nkv, -1, 2, 4096))
    pos = pick[..., None] * page + torch.arange(page, device=dev)
    seen = ((pos < s["len"][:, None, None, None]) & counts[..., None]).reshape(B, -1, 1, k.shape[2]).expand(B, nkv, T * G, -1)
    rows = B * T
    tk = s["tk"][0, :, :rows].view(nkv, B, T, D).transpose(0, 1)
    tv = s["tv"][0, :, :, :rows].view(nkv, D, B, T).permute(2, 0, 3, 1)
    k, v = torch.cat((k, tk), 2).float(), torch.cat((v, tv), 2).float()
    tree = _bits(s["mask"], T).view(B, 1, T, 1, T).expand(B, nkv, T, G, T).reshape(B, nkv, T * G, T)
    see = torch.cat((seen, tree), 3).reshape(B * nkv, T * G, -1)
    o, l = _attention(q, k.reshape(B * nkv, -1, D), v.reshape(B * nkv, -1, D), see, s["q"].dtype)
    out = o.view(B, nkv, T, G, D).permute(0, 2, 1, 3, 4).reshape(rows, nh, D)
    return out, l.view(B, nkv, T, G).permute(0, 2, 1, 3).reshape(rows, nh)


def run(state):
    kind = state["case"]["kind"]
    if own:
        return _run_own(state)
    if kind == "tables":
        return _run_tables(state)
    if kind == "store":
        return _run_store(state)
    if kind == "attend":
        out, lse = _run_attention(state)
        return dict(out=out, lse=lse)
    sel, n_sel = _select(state)
    out, lse = _run_attention(state, sel, n_sel)
    return dict(sel=sel, n_sel=n_sel, out=out, lse=lse)


# ---------------------------------------------------------------------------
# 64 bits, from the definitions


def _held(s, phys, head, pos):
    """Keys and values [n][128] at `pos` (inside pages phys, [n]) of a head, by
    the layout's address of every element."""
    flat = s["pages"][0, :, head].reshape(s["pages"].shape[1], -1, 4096)     # [pages][2 blocks][4096]
    d = torch.arange(D, device=pos.device)
    p = pos % BLOCK
    lane = 16 * (d % 32 // 8)[None] + 4 * (p // 8)[:, None] + (p % 4)[:, None]
    ki = (((p % 8 // 4)[:, None] * 4 + (d // 32)[None]) * 64 + lane) * 8 + (d % 8)[None]
    vi = ((d // 16)[None] * 64 + 16 * (p // 8)[:, None] + (d % 16)[None]) * 8 + (p % 8)[:, None]
    blk = (2 * (pos // BLOCK))[:, None]
    return flat[phys[:, None], blk, ki].double(), flat[phys[:, None], blk + 1, vi].double()


def _exact_tables(s):
    page = s["case"]["page"]
    table, ring = s["table"].cpu().numpy().copy(), s["ring"].cpu().numpy().copy()
    n, add = s["len"].tolist(), s["add"].tolist()
    first, count = s["state"].tolist()
    slots = s["slots"].cpu().numpy().copy()
    n_pages, length, start = len(ring), [], [0]
    popped, asked, back = 0, 0, []
    for q, (have, more) in enumerate(zip(n, add)):
        old = _ceil(have, page)
        if more < 0:
            back += table[q, :old].tolist()
            length.append(0)
            start.append(start[-1])
            continue
        start.append(start[-1] + more)
        new = _ceil(have + more, page)
        ok = new <= table.shape[1] and start[-1] <= len(slots)
        if ok:
            asked += new - old
            ok = new == old or asked <= count
        if not ok:
            slots[start[-2]:min(start[-1], len(slots))] = -1
            length.append(have)
            continue
        for i in range(old, new):
            table[q, i] = ring[(first + popped) % n_pages]
            popped += 1
        pos = np.arange(have, have + more)
        slots[start[-2]:start[-1]] = table[q, pos // page] * page + pos % page
        length.append(have + more)
    for i, x in enumerate(back):
        ring[(first + count + i) % n_pages] = x
    state = [(first + popped) % n_pages, count - popped + len(back)]
    t = torch.from_numpy
    return _tables_out(s, t(table), t(ring), torch.tensor(length), torch.tensor(state), torch.tensor(start), t(slots))


def _exact_store(s):
    page = s["case"]["page"]
    pages, bounds = s["pages"].double(), s["bounds"].double()
    start, row_start, slots = s["start"].tolist(), s["row_start"].tolist(), s["slots"].tolist()
    path = None if s["path"] is None else s["path"].tolist()
    d = torch.arange(D, device=pages.device)
    dk = d // 32 * 512 + d % 32 // 8 * 128 + d % 8      # address of a key's dims, beside its position's
    dv = d // 16 * 512 + d % 16 * 8
    for q in range(len(start) - 1):
        i = start[q]
        while i < start[q + 1]:
            at, off = divmod(slots[i], page)
            m = min(page - off, start[q + 1] - i)       # the rows of one page
            rows = [row_start[q] + (k if path is None else path[row_start[q] + k]) for k in range(i - start[q], i - start[q] + m)]
            k, v = s["k"][:, :, rows].double(), s["v"][:, :, :, rows].transpose(2, 3).double()   # [layers][heads][m][128]
            pos = torch.arange(off, off + m, device=d.device)
            p = pos % BLOCK
            ka = (p % 8 // 4 * 2048 + p // 8 * 32 + p % 4 * 8)[:, None] + dk
            va = (p // 8 * 128 + p % 8)[:, None] + dv
            blk = (pos // BLOCK)[:, None]
            pages[:, at][:, :, blk, 0, ka] = k
            pages[:, at][:, :, blk, 1, va] = v
            lo, hi = k.amin(2), k.amax(2)
            if off:
                lo, hi = torch.minimum(lo, bounds[:, at, :, 0]), torch.maximum(hi, bounds[:, at, :, 1])
            bounds[:, at, :, 0], bounds[:, at, :, 1] = lo, hi
            i += m
    return dict(pages=pages, bounds=bounds)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] == "tables":
        return _exact_tables(s)
    if c["kind"] == "store":
        return _exact_store(s)
    nkv, nh, T, page = c["nkv"], c["nh"], c["T"], c["page"]
    G = nh // nkv
    dev = s["q"].device
    out = torch.zeros((c["B"] * T, nh, D), dtype=torch.float64, device=dev)
    lse = torch.zeros((c["B"] * T, nh), dtype=torch.float64, device=dev)
    sel, n_sel = [], []
    for b, n in enumerate(_counts(c)[0]):
        r0, np_ = b * T, _ceil(n, page)
        words = s["mask"][r0:r0 + T].tolist()
        sees = torch.tensor([[w[j // 64] >> (j % 64) & 1 for j in range(T)] for w in words], device=dev).bool()
        rows = []
        for h in range(nkv):
            q = s["q"][r0:r0 + T, h * G:(h + 1) * G].double()                # [T][G][128]
            if c["kind"] == "attend":
                pos = torch.arange(n, device=dev)
            else:
                lo, hi = (s["bounds"][0, s["table"][b, :np_].long(), h, i].double() for i in (0, 1))
                up = (torch.where(q > 0, q, 0.0 * q).sum((0, 1)) * hi).sum(1) + (torch.where(q < 0, q, 0.0 * q).sum((0, 1)) * lo).sum(1)
                keep = set(range(min(c["first"], np_))) | set(range(max(0, np_ - c["last"]), np_))
                m = min(np_, c["budget"])
                order = sorted(range(np_), key=lambda p, u=up.tolist(): (p not in keep, -u[p], p))[:m]
                rows.append(sorted(order) + [-1] * (c["budget"] - m))
                pos = (torch.tensor(sorted(order), device=dev)[:, None] * page + torch.arange(page, device=dev)).reshape(-1)
                pos = pos[pos < n]
            k, v = _held(s, s["table"][b].long()[pos // page], h, pos % page)
            k = torch.cat((k, s["tk"][0, h, r0:r0 + T].double()))
            v = torch.cat((v, s["tv"][0, h, :, r0:r0 + T].double().t()))
            x = (q.reshape(T * G, D) @ k.t()).view(T, G, -1) / math.sqrt(D)
            x[:, :, len(pos):].masked_fill_(~sees[:, None], float("-inf"))
            lse[r0:r0 + T, h * G:(h + 1) * G] = torch.logsumexp(x, -1)
            w = torch.exp(x - lse[r0:r0 + T, h * G:(h + 1) * G, None])
            out[r0:r0 + T, h * G:(h + 1) * G] = (w.view(T * G, -1) @ v).view(T, G, D)
        if rows:
            sel.append(rows)
            n_sel.append(min(np_, c["budget"]))
    if c["kind"] == "attend":
        return dict(out=out, lse=lse)
    return dict(sel=torch.tensor(sel, device=dev), n_sel=torch.tensor(n_sel, device=dev), out=out, lse=lse)


# ---------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    c = dict(case)
    kind, B, page = c["kind"], c["B"], c["page"]
    lens, add = _counts(c)
    if kind == "tables":
        rows, need = sum(max(a, 0) for a in add), sum(_needs(c, lens, add))
        back = sum(_ceil(n, page) for n, a in zip(lens, add) if a < 0)
        if c["scarce"]:
            need //= 2
        # lengths and counts in, lengths and offsets out, the slots, each page's number read and written
        return {"bytes": 4 * (4 * B + rows + 2 * (need + back)), "flops": 0}
    nkv = c["nkv"]
    if kind == "store":
        rows = sum(add)
        touched = sum(_ceil(n + a, page) - n // page for n, a in zip(lens, add))
        # rows in and out, bounds out
        return {"bytes": c["layers"] * nkv * (rows * 2 * 512 + touched * 512), "flops": 0}
    nh, T = c["nh"], c["T"]
    size = 2 if c["dtype"] == "bf16" else 4
    # queries and outputs, the new tokens' rows, their masks and log-sums
    total = B * T * (nh * D * 2 * size + nkv * 512 + 16 + 4 * nh)
    flops = 0
    for n in lens:
        np_ = _ceil(n, page)
        if kind == "sparse":
            total += np_ * nkv * 512
            flops += np_ * nkv * 512
            np_ = min(np_, c["budget"])
            n = min(n, np_ * page)
        total += n * nkv * 512 + 4 * np_
        flops += 4 * D * nh * T * (n + T)
    return {"bytes": total, "flops": flops}
