"""Operators of a decode loop at a temperature on a bounded 4-bit cache, as
cases with inputs, one pass each in plain torch operations or through the
library, and a 64-bit value.

  attend   tree attention of one layer over 4-bit prefixes and the trees' own
           bf16 rows (ppd_kvq_attention)
  fill     bf16 cache rows to 4 bits and back (ppd_kvq_quantize,
           ppd_kvq_dequantize)
  commit   the accepted path's rows into the 4-bit cache, read back
           (ppd_kvq_commit, ppd_kvq_dequantize)
  score    the accepted nodes' attention weights added to every cached
           position's sum, all layers (ppd_kvq_score)
  evict    the positions of largest sums kept, with the first and the last
           ones, read back (ppd_kvq_evict, ppd_kvq_dequantize)
  sample   drafted tokens verified against the target's probabilities from
           given random numbers (ppd_accept_sample)

A 4-bit row holds 128 dims in two groups of 64: a code c of 0 .. 15 stands for
s c + z, z the group's minimum, s = (maximum - minimum) / 15 in float32 rounded
to bfloat16, c the float32 quotient (x - z) / s rounded to even.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128            # head dim
BLOCK, BLOCK_BYTES = 32, 4608
SCALE = 1.0 / math.sqrt(D)


# ---------------------------------------------------------------------------
# cases


def _attend(name, nh, nkv, T, L):
    c = dict(kind="attend", nh=nh, nkv=nkv, T="/".join(map(str, T)), L="/".join(map(str, L)))
    return dict(c, name=name) if name else c


def _fill(name, layers, nkv, n, src_pos, dst_pos):
    c = dict(kind="fill", layers=layers, nkv=nkv, n=n, src_pos=src_pos, dst_pos=dst_pos)
    return dict(c, name=name) if name else c


def _commit(name, layers, nkv, T, L, accepted):
    c = dict(kind="commit", layers=layers, nkv=nkv, T=T, L=L, accepted=accepted)
    return dict(c, name=name) if name else c


def _score(name, layers, nh, nkv, T, L, accepted, dtype):
    c = dict(kind="score", layers=layers, nh=nh, nkv=nkv, T=T, L=L, accepted=accepted, dtype=dtype)
    return dict(c, name=name) if name else c


def _evict(name, layers, nkv, L, budget, sink, recent):
    c = dict(kind="evict", layers=layers, nkv=nkv, L=L, budget=budget, sink=sink, recent=recent)
    return dict(c, name=name) if name else c


def _sample(name, T, vocab, draft, temperature):
    c = dict(kind="sample", T=T, vocab=vocab, draft=draft, temperature=temperature)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: one token of an edge-size model, short context
        _attend("attend_1b4_T1_L200", 16, 16, [1], [200]),
        # the 64-node tree of the 7B shape over its 2k prefix
        _attend("attend_7b_T64_L2048", 32, 32, [64], [2048]),
        # grouped-query heads, four users with trees and prefixes of any size
        _attend("attend_gqa_batch4", 32, 8, [41, 16, 1, 7], [777, 4096, 6001, 32]),
        # long context, a small tree: the cache is all that counts
        _attend("attend_7b_T16_L32768", 32, 32, [16], [32768]),
        # a prompt's bf16 prefix handed over to the 4-bit cache
        _fill("fill_7b_2048", 8, 32, 2048, 0, 0),
        # after every step: the accepted path of a 64-node tree, all layers
        _commit("commit_7b_T64", 32, 32, 64, 2048, 5),
        # after every step: the weights of three accepted nodes, all layers
        _score("score_7b_L2048", 32, 32, 32, 64, 2048, 3, "f32"),
        # the same with grouped-query heads and a longer, odd prefix
        _score("score_gqa_L8191", 32, 32, 8, 41, 8191, 5, "bf16"),
        # a cache at its limit cut to half
        _evict("evict_7b_4096", 8, 32, 4096, 2048, 4, 256),
        # the rolling form: a few positions go, an odd number stays
        _evict("evict_gqa_1100", 24, 8, 1100, 1021, 0, 64),
        # candidates that are the drafter's best tokens: no draft probabilities
        _sample("sample_T64_V32000", 64, 32000, False, 0.7),
        # candidates drawn from draft probabilities, an odd vocabulary
        _sample("sample_draft_T25_V32001", 25, 32001, True, 1.0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "fill", "commit", "score", "evict", "sample", "sample"))
    nkv = rng.choice((2, 4, 8, 16, 32, 40))
    if kind == "attend":
        nh = nkv * rng.choice([g for g in (1, 2, 4, 8) if g * nkv <= 40])
        B = rng.choice((1, 1, 1, 2, 3, 5))
        T = [_log(rng, 1, 128 // B) for _ in range(B)]
        L = [min(_log(rng, 1, 32768), 32768 * 32 // (nkv * B)) for _ in range(B)]
        if sum(T) > 16:
            L = [min(x, 8192 // B) for x in L]
        return _attend(None, nh, nkv, T, L)
    layers = rng.randint(1, 32)
    if kind == "fill":
        n = _log(rng, 1, 524288 // (layers * nkv))
        return _fill(None, layers, nkv, n, rng.randint(0, 70), rng.randint(0, 70))
    if kind == "commit":
        T = _log(rng, 1, 128)
        return _commit(None, layers, nkv, T, _log(rng, 1, 2048), rng.randint(1, min(T, 16)))
    if kind == "score":
        nh = nkv * rng.choice([g for g in (1, 2, 4) if g * nkv <= 40])
        T = _log(rng, 1, 128)
        return _score(None, layers, nh, nkv, T, _log(rng, 1, 2000000 // (layers * nkv)),
                      rng.randint(1, min(T, 8)), rng.choice(("f32", "bf16")))
    if kind == "evict":
        L = max(8, _log(rng, 8, 1048576 // (layers * nkv)))
        budget = rng.randint(max(1, L // 8), L)
        sink = rng.randint(0, min(4, budget))
        return _evict(None, layers, nkv, L, budget, sink, rng.randint(0, (budget - sink) // 2))
    return _sample(None, _log(rng, 1, 64), rng.choice((1000, 8191, 32000, 32001, 50257)) + rng.randint(0, 8),
                   rng.random() < 0.5, rng.choice((0.3, 0.7, 1.0, 1.7)))


def _ints(s):
    return [int(x) for x in str(s).split("/")]


# ---------------------------------------------------------------------------
# the 4-bit layout: one block of 32 positions is 4608 bytes -- the keys' codes
# (2048), the values' codes (2048), and per position 8 bytes of (scale, zero)
# bfloat16 pairs of its two groups, keys then values

_SHIFT = [4 * (e // 2) + 16 * (e % 2) for e in range(8)]  # element e of a 32-bit word


def _quantize(x):
    """codes (int32) [.., 128], scale and zero (bf16) [.., 2] of float32 rows."""
    g = x.reshape(*x.shape[:-1], 2, 64)
    z = g.amin(-1)
    s = ((g.amax(-1) - z) / 15.0).to(torch.bfloat16)
    sf = s.float()[..., None]
    q = torch.where(sf > 0, (g - z[..., None]) / torch.where(sf > 0, sf, torch.ones_like(sf)), torch.zeros_like(g))
    c = torch.clamp(torch.round(q), 0, 15).to(torch.int32)
    return c.reshape(x.shape), s, z.to(torch.bfloat16)


def _words(c):
    """int64 codes [.., 8] -> int32 words."""
    sh = torch.tensor(_SHIFT, device=c.device)
    w = (c.long() << sh).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _pairs(s, z):
    """(scale, zero) bf16 -> int32 words, the scale in the low half."""
    return torch.stack((s, z), -1).contiguous().view(torch.int32).squeeze(-1)


def pack(k, v):
    """blocks uint8 [H][nb][4608] of float32 rows k, v [H][32 nb][128]."""
    H, n, _ = k.shape
    nb = n // BLOCK
    kc, ks, kz = _quantize(k)
    vc, vs, vz = _quantize(v)
    # keys: position 8 a + 4 t + b of the block, dims 32 d + 8 g + e -> word [t][lane 16 g + 4 a + b][d]
    kw = _words(kc.view(H, nb, 4, 2, 4, 4, 4, 8)).permute(0, 1, 3, 6, 2, 4, 5)
    # values: position 8 g + e, dims 64 h + 16 i + r -> word [h][lane 16 g + r][i]
    vw = _words(vc.view(H, nb, 4, 8, 2, 4, 16).permute(0, 1, 4, 2, 6, 5, 3))
    parts = (kw, vw, _pairs(ks, kz), _pairs(vs, vz))
    return torch.cat([p.reshape(H, nb, -1).contiguous().view(torch.uint8) for p in parts], -1)


def _codes(blocks):
    """Codes and (scale, zero) of blocks [H][nb][4608]: kc, ks, kz, vc, vs, vz,
    codes [H][32 nb][128], the others float32 [H][32 nb][2]."""
    H, nb, _ = blocks.shape
    sh = torch.tensor(_SHIFT, device=blocks.device, dtype=torch.int32)

    def words(lo, hi):
        return blocks[:, :, lo:hi].contiguous().view(torch.int32)
    kw = words(0, 2048).view(H, nb, 2, 4, 4, 4, 4)              # t g a b d
    kc = ((kw[..., None] >> sh) & 15).permute(0, 1, 4, 2, 5, 6, 3, 7).reshape(H, nb * BLOCK, D)
    vw = words(2048, 4096).view(H, nb, 2, 4, 16, 4)             # h g r i
    vc = ((vw[..., None] >> sh) & 15).permute(0, 1, 3, 6, 2, 5, 4).reshape(H, nb * BLOCK, D)

    def pairs(lo, hi):
        p = words(lo, hi).view(H, nb * BLOCK, 2, 1).view(torch.bfloat16)
        return p[..., 0], p[..., 1]
    ks, kz = pairs(4096, 4352)
    vs, vz = pairs(4352, 4608)
    return kc, ks, kz, vc, vs, vz


def _values(c, s, z, dtype=torch.float32):
    g = c.to(dtype).view(*c.shape[:-1], 2, 64)
    return (g * s.to(dtype)[..., None] + z.to(dtype)[..., None]).view(c.shape)


def _unpack(blocks, n):
    """float32 keys and values [H][n][128] of the first n positions."""
    kc, ks, kz, vc, vs, vz = _codes(blocks[:, : (n + BLOCK - 1) // BLOCK])
    return _values(kc, ks, kz)[:, :n], _values(vc, vs, vz)[:, :n]


# ---------------------------------------------------------------------------
# inputs


def _gen(seed, *salt):
    h = 0
    for x in salt:
        h = (h * 1000003 + x) % (1 << 31)
    g = torch.Generator("cuda")
    g.manual_seed((seed * 7919 + h) % (1 << 40))
    return g


def _rows(g, H, n, spread=1.0):
    """Cache rows: N(0, 1), some dims larger than others, as trained keys are."""
    x = torch.randn((H, n, D), generator=g, device="cuda")
    w = 1.0 + spread * torch.rand((H, 1, D), generator=g, device="cuda")
    return (x * w * 0.75).to(torch.bfloat16).float()


def _cap(n):
    return (n + BLOCK - 1) // BLOCK * BLOCK


def _blocks(g, layers, nkv, capacity, L, spread=1.0):
    """A 4-bit cache [layers][nkv][capacity / 32][4608] with L positions; the
    rest holds anything."""
    out = torch.randint(0, 256, (layers, nkv, capacity // BLOCK, BLOCK_BYTES), generator=g, device="cuda",
                        dtype=torch.uint8)
    n = _cap(L)
    for l in range(layers):
        if L == 0:
            break
        b = pack(_rows(g, nkv, n, spread), _rows(g, nkv, n, spread))
        if L < n:  # positions past the last: their scale words hold anything
            b[:, -1, 4096 + 8 * (L % BLOCK):4352] = 255
            b[:, -1, 4352 + 8 * (L % BLOCK):] = 255
        out[l, :, : n // BLOCK] = b
    return out


def _tail(g, layers, nkv, capacity):
    k = torch.randn((layers, nkv, capacity, D), generator=g, device="cuda").to(torch.bfloat16)
    v = torch.randn((layers, nkv, D, capacity), generator=g, device="cuda").to(torch.bfloat16)
    return k, v


def _tree(r, T, chains):
    """parent array of a tree of T nodes; chains: of the candidates' share of a
    tree with prompt tokens, the rest hangs under the candidates in chains of
    three.  Returns (parent, is_prompt)."""
    n_cand = max(1, T // 4) if chains else T
    parent = [-1] + [r.randrange(max(0, i - 6), i) for i in range(1, n_cand)]
    prompt = [False] * n_cand
    at = 0
    while len(parent) < T:
        up = at % n_cand
        for _ in range(3):
            if len(parent) < T:
                parent.append(up)
                prompt.append(True)
                up = len(parent) - 1
        at += 1
    return parent, prompt


def _mask(parent):
    T = len(parent)
    m = np.zeros((T, 2), np.uint64)
    for i in range(T):
        j = i
        while j >= 0:
            m[i, j // 64] |= np.uint64(1 << (j % 64))
            j = parent[j]
    return m


def _path(r, T, accepted):
    """A path of `accepted` nodes: root, then growing node indices."""
    return [0] + sorted(r.sample(range(1, T), accepted - 1))


def _dev(a, dtype=torch.int32):
    return torch.tensor(a, dtype=dtype, device="cuda")


def _seq(c):
    return list(zip(_ints(c["T"]), _ints(c["L"])))


def prepare(case, seed):
    c = dict(case)
    kind = c["kind"]
    r = random.Random("%s %d" % (kind, seed))
    g = _gen(seed, *[int(x) for x in c.values() if isinstance(x, (int, bool))])
    s = dict(case=c)
    if kind == "attend":
        seqs = _seq(c)
        n_tok = sum(T for T, _ in seqs)
        s["q"] = torch.randn((n_tok, c["nh"], D), generator=g, device="cuda").to(torch.bfloat16)
        s["seqs"] = []
        masks = []
        for T, L in seqs:
            cap = max(BLOCK, _cap(L))
            tail_cap = (T + 7) // 8 * 8
            s["seqs"].append(dict(T=T, L=L, blocks=_blocks(g, 1, c["nkv"], cap, L),
                                  tail=_tail(g, 1, c["nkv"], tail_cap)))
            masks.append(_mask(_tree(r, T, T >= 16)[0]))
        mask = np.concatenate(masks)
        s["mask"] = torch.from_numpy(mask.view(np.int64)).cuda()
        s["out"] = torch.zeros((n_tok, c["nh"], D), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((n_tok, c["nh"]), device="cuda")
    elif kind == "fill":
        layers, nkv, n = c["layers"], c["nkv"], c["n"]
        cap = (c["src_pos"] + n + 7) // 8 * 8
        s["k"] = torch.empty((layers, nkv, cap, D), dtype=torch.bfloat16, device="cuda")
        s["v"] = torch.empty((layers, nkv, D, cap), dtype=torch.bfloat16, device="cuda")
        for l in range(layers):
            s["k"][l] = _rows(g, nkv, cap)
            s["v"][l] = _rows(g, nkv, cap).transpose(1, 2)
        s["blocks"] = _blocks(g, layers, nkv, _cap(c["dst_pos"] + n), 0)
        s.update(_out(layers, nkv, n))
    elif kind == "commit":
        layers, nkv, T, L, n = c["layers"], c["nkv"], c["T"], c["L"], c["accepted"]
        s["blocks"] = _blocks(g, layers, nkv, _cap(L + n), 0)  # what the prefix holds is not read
        s["tail"] = _tail(g, layers, nkv, (T + 7) // 8 * 8)
        path = _path(r, T, n)
        s["path"], s["n_path"] = _dev(path + [0] * (T - n)), _dev([n])
        s.update(_out(layers, nkv, n))
    elif kind == "score":
        layers, nh, nkv, T, L, n = c["layers"], c["nh"], c["nkv"], c["T"], c["L"], c["accepted"]
        s["blocks"] = _blocks(g, layers, nkv, _cap(L + n), L)
        s["tail"] = _tail(g, layers, nkv, (T + 7) // 8 * 8)
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        s["q"] = torch.randn((layers, T, nh, D), generator=g, device="cuda").to(dt)
        # the log-sum-exp of L scores N(0, 1), near enough
        s["lse"] = math.log(L + 1) + 0.5 + 0.1 * torch.randn((layers, T, nh), generator=g, device="cuda")
        path = _path(r, T, n)
        s["path"], s["n_path"], s["nodes"] = _dev(path + [0] * (T - n)), _dev([n]), path
        cap = _cap(L + n)
        s["score"] = torch.rand((layers, nkv, cap), generator=g, device="cuda")
        s["score_out"] = torch.zeros((layers, nkv, cap), device="cuda")
    elif kind == "evict":
        layers, nkv, L, n = c["layers"], c["nkv"], c["L"], min(c["L"], c["budget"])
        s["blocks"] = _blocks(g, layers, nkv, _cap(L), L)
        s["dst"] = _blocks(g, layers, nkv, _cap(n), 0)
        # sums of weights: many small ones, some equal, a few large
        u = torch.rand((layers, nkv, _cap(L)), generator=g, device="cuda")
        s["score"] = torch.where(u < 0.02, torch.floor(u * 500) / 500, (4 * u) ** 6 / 4096)
        s["score_out"] = torch.zeros((layers, nkv, _cap(n)), device="cuda")
        s["kept"] = torch.zeros((layers, nkv, c["budget"]), dtype=torch.int32, device="cuda")
        s.update(_out(layers, nkv, n))
    else:
        T, V = c["T"], c["vocab"]
        parent, prompt = _tree(r, T, T >= 16 and not c["draft"])
        logits = 2.0 * torch.randn((T, V), generator=g, device="cuda")
        s["draft"] = None
        kids = [[j for j in range(T) if parent[j] == i and not prompt[j]] for i in range(T)]
        ids = [0] * T
        if c["draft"]:  # children drawn from draft rows that are near the target's
            d = torch.softmax(logits / c["temperature"] + torch.randn((T, V), generator=g, device="cuda"), -1)
            s["draft"] = d
            drawn = torch.multinomial(d, max([1] + [len(x) for x in kids]), True, generator=g).cpu().tolist()
            for i in range(T):
                for j, x in enumerate(kids[i]):
                    ids[x] = drawn[i][j]
        else:           # children that are likely tokens: the target gives the first about a half
            for i in range(T):
                for j, x in enumerate(kids[i]):
                    ids[x] = r.randrange(V)
                    top = math.log(V) + 2.0 / c["temperature"] ** 2 + 0.4 - 0.7 * j
                    logits[i, ids[x]] = c["temperature"] * top
        for i in range(T):
            if prompt[i]:
                ids[i] = V + r.randrange(3)
        s["logits"] = logits
        s["parent"], s["ids"] = _dev(parent), _dev(ids)
        s["u"] = torch.rand(T, generator=g, device="cuda")
        # the tree's shape, known on the host as its template is
        s["kids"] = kids
        s["depth"] = max(_depths(parent, prompt))
        s["path"] = torch.zeros(T, dtype=torch.int32, device="cuda")
        s["n_path"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        s["next"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        # per rank j: the nodes that have a j-th child, and these children
        s["ranks"] = []
        for j in range(max(len(x) for x in kids)):
            at = [i for i in range(T) if len(kids[i]) > j]
            ch = [kids[i][j] for i in at]
            s["ranks"].append((_dev(at, torch.int64), _dev(ch, torch.int64), _dev([ids[x] for x in ch], torch.int64)))
    if own:
        _handles(s)
    return s


def _depths(parent, prompt):
    d = []
    for i, p in enumerate(parent):
        d.append(0 if p < 0 or prompt[i] else d[p] + 1)
    return d


def _out(layers, nkv, n):
    cap = (n + 7) // 8 * 8
    return dict(n=n, k_out=torch.zeros((layers, nkv, cap, D), dtype=torch.bfloat16, device="cuda"),
                v_out=torch.zeros((layers, nkv, D, cap), dtype=torch.bfloat16, device="cuda"))


def _handles(s):
    """The library's descriptions of the buffers, and a workspace."""
    import paper_2405_18628_amd as ppd
    s["ppd"] = ppd
    c, kind = s["case"], s["case"]["kind"]
    if "k_out" in s:
        s["back"] = ppd.KVCache(s["k_out"], s["v_out"])
    if kind == "attend":
        s["kvs"] = [ppd.KVQCache(q["blocks"], ppd.KVCache(*q["tail"])) for q in s["seqs"]]
        s["Ls"] = np.array([q["L"] for q in s["seqs"]], np.int32)
        s["Ts"] = np.array([q["T"] for q in s["seqs"]], np.int32)
        n = ppd.ppd_kvq_attention_workspace_bytes(c["nh"], c["nkv"], int(s["Ts"].sum()))
    elif kind == "sample":
        n = ppd.ppd_accept_sample_workspace_bytes(c["T"], c["vocab"])
    else:
        tail = ppd.KVCache(*s["tail"]) if "tail" in s else None
        s["kv"] = ppd.KVQCache(s["blocks"], tail)
        if kind == "fill":
            s["src"] = ppd.KVCache(s["k"], s["v"])
        if kind == "evict":
            s["to"] = ppd.KVQCache(s["dst"])
        n = 0
    if n:
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        ppd.ppd_workspace_init(s["ws"])


# ---------------------------------------------------------------------------
# one pass


def run(s):
    return (_run_own if own else _run_plain)[s["case"]["kind"]](s)


# ---- through the library


def _own_attend(s):
    s["ppd"].ppd_kvq_attention(s["kvs"], 0, s["Ls"], s["Ts"], s["q"], s["mask"], s["out"], s["ws"], lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"])


def _own_fill(s):
    c, ppd = s["case"], s["ppd"]
    ppd.ppd_kvq_quantize(s["kv"], c["dst_pos"], s["src"], c["src_pos"], c["n"])
    ppd.ppd_kvq_dequantize(s["kv"], c["dst_pos"], s["back"], 0, c["n"])
    return dict(k=s["k_out"], v=s["v_out"])


def _own_commit(s):
    c, ppd = s["case"], s["ppd"]
    ppd.ppd_kvq_commit(s["kv"], c["L"], s["path"], s["n_path"])
    ppd.ppd_kvq_dequantize(s["kv"], c["L"], s["back"], 0, c["accepted"])
    return dict(k=s["k_out"], v=s["v_out"])


def _own_score(s):
    s["ppd"].ppd_kvq_score(s["kv"], s["case"]["L"], s["q"], s["lse"], s["path"], s["n_path"], s["score"],
                           s["score_out"])
    return dict(score=s["score_out"])


def _own_evict(s):
    c, ppd = s["case"], s["ppd"]
    ppd.ppd_kvq_evict(s["kv"], s["to"], c["L"], c["budget"], c["sink"], c["recent"], s["score"], s["score_out"],
                      s["kept"])
    ppd.ppd_kvq_dequantize(s["to"], 0, s["back"], 0, s["n"])
    return dict(kept=s["kept"], score=s["score_out"], k=s["k_out"], v=s["v_out"])


def _own_sample(s):
    c = s["case"]
    s["ppd"].ppd_accept_sample(c["T"], s["parent"], s["ids"], c["vocab"], s["logits"], c["temperature"], s["draft"],
                               s["u"], s["path"], s["n_path"], s["next"], s["ws"])
    return dict(path=s["path"], n_path=s["n_path"], next=s["next"])


# ---- plain operations


def _plain_attend(s):
    c = s["case"]
    nh, nkv = c["nh"], c["nkv"]
    out, lse, t0 = [], [], 0
    for q in s["seqs"]:
        T, L = q["T"], q["L"]
        k, v = _unpack(q["blocks"][0], L)                                   # [nkv][L][128]
        kt = q["tail"][0][0][:, :T].float()
        vt = q["tail"][1][0][:, :, :T].float().transpose(1, 2)
        k, v = torch.cat((k, kt), 1), torch.cat((v, vt), 1)
        qs = s["q"][t0:t0 + T].float().view(T, nkv, nh // nkv, D).permute(1, 2, 0, 3).reshape(nkv, -1, D)
        sc = torch.matmul(qs, k.transpose(1, 2).contiguous()) * SCALE       # [nkv][G T][L + T]
        bits = (s["mask"][t0:t0 + T, torch.arange(T, device="cuda") // 64] >> (torch.arange(T, device="cuda") % 64)) & 1
        sc = sc.view(nkv, -1, T, L + T)
        sc[..., L:] = torch.where(bits.bool(), sc[..., L:], -math.inf)
        sc = sc.view(nkv, -1, L + T)
        m = sc.amax(-1, keepdim=True)
        p = torch.exp(sc - m)
        l = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v.contiguous()) / l
        out.append(o.view(nkv, -1, T, D).permute(2, 0, 1, 3).reshape(T, nh, D).to(torch.bfloat16))
        lse.append((m + torch.log(l)).view(nkv, -1, T).permute(2, 0, 1).reshape(T, nh))
        t0 += T
    return dict(out=torch.cat(out), lse=torch.cat(lse))


def _plain_fill(s):
    c = s["case"]
    n, sp = c["n"], c["src_pos"]
    for l in range(c["layers"]):
        for src, dst, tr in ((s["k"], s["k_out"], False), (s["v"], s["v_out"], True)):
            x = src[l][:, :, sp:sp + n].transpose(1, 2) if tr else src[l][:, sp:sp + n]
            _put(dst, l, n, _values(*_quantize(x.float())), tr)
    return dict(k=s["k_out"], v=s["v_out"])


def _put(dst, l, n, x, tr):
    if tr:
        dst[l][:, :, :n] = x.transpose(1, 2)
    else:
        dst[l][:, :n] = x


def _plain_commit(s):
    c = s["case"]
    n = c["accepted"]
    at = s["path"][:n].long()
    for l in range(c["layers"]):
        _put(s["k_out"], l, n, _values(*_quantize(s["tail"][0][l][:, at].float())), False)
        _put(s["v_out"], l, n, _values(*_quantize(s["tail"][1][l][:, :, at].transpose(1, 2).float())), True)
    return dict(k=s["k_out"], v=s["v_out"])


def _plain_score(s):
    c = s["case"]
    nh, nkv, L, n = c["nh"], c["nkv"], c["L"], c["accepted"]
    at = s["path"][:n].long()
    seen = torch.ones((n, L + n), dtype=torch.bool, device="cuda")
    seen[:, L:] = torch.tril(seen[:, L:])
    for l in range(c["layers"]):
        k = torch.cat((_unpack(s["blocks"][l], L)[0], s["tail"][0][l][:, at].float()), 1)
        q = s["q"][l][at].float().view(n, nkv, -1, D).permute(1, 2, 0, 3).reshape(nkv, -1, D)   # [nkv][G n][128]
        lse = s["lse"][l][at].view(n, nkv, -1).permute(1, 2, 0).reshape(nkv, -1, 1)
        w = torch.exp(torch.matmul(q, k.transpose(1, 2).contiguous()) * SCALE - lse).view(nkv, -1, n, L + n)
        w = torch.where(seen, w, 0.0).sum((1, 2))
        s["score_out"][l][:, :L] = s["score"][l][:, :L] + w[:, :L]
        s["score_out"][l][:, L:L + n] = w[:, L:]
    return dict(score=s["score_out"])


def _keep(score, L, n, sink, recent):
    """Kept positions [.., n] of score [.., capacity], ascending."""
    lead = score.shape[:-1]
    mid = score[..., sink:L - recent]
    best = torch.sort(mid, dim=-1, descending=True, stable=True)[1][..., :n - sink - recent] + sink
    first = torch.arange(sink, device="cuda").expand(*lead, sink)
    last = torch.arange(L - recent, L, device="cuda").expand(*lead, recent)
    return torch.cat((first, torch.sort(best, -1)[0], last), -1)


def _plain_evict(s):
    c = s["case"]
    L, n = c["L"], s["n"]
    kept = _keep(s["score"], L, n, c["sink"], c["recent"])
    s["kept"][..., :n] = kept.int()
    s["score_out"][..., :n] = torch.gather(s["score"], -1, kept)
    for l in range(c["layers"]):
        k, v = _unpack(s["blocks"][l], L)
        at = kept[l][..., None].expand(-1, -1, D)
        _put(s["k_out"], l, n, torch.gather(k, 1, at), False)
        _put(s["v_out"], l, n, torch.gather(v, 1, at), True)
    return dict(kept=s["kept"], score=s["score_out"], k=s["k_out"], v=s["v_out"])


def _plain_sample(s):
    c = s["case"]
    T = c["T"]
    x = s["logits"].double() / c["temperature"]
    r = torch.exp(x - x.amax(-1, keepdim=True))
    Z = r.sum(-1)
    u = s["u"].double()
    go = torch.full((T,), -1, dtype=torch.int64, device="cuda")     # the accepted child
    for at, ch, tok in s["ranks"]:
        open_ = go[at] < 0
        w = r[at, tok]
        q = s["draft"][at, tok].double() if c["draft"] else 1.0
        ok = open_ & (u[ch] * q * Z[at] < w)
        go[at] = torch.where(ok, ch, go[at])
        no = (open_ & ~ok)[:, None]
        if c["draft"]:
            rest = torch.clamp(r[at] - Z[at][:, None] * s["draft"][at].double(), min=0.0)
        else:
            rest = r[at].scatter(1, tok[:, None], 0.0)
        rest = torch.where(no, rest, r[at])
        r[at] = rest
        Z[at] = rest.sum(-1)
    cum = torch.cumsum(r, -1)
    bonus = (cum <= (u[0] * cum[:, -1])[:, None]).sum(-1)
    path = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    node = torch.zeros((), dtype=torch.int64, device="cuda")
    n = torch.ones((), dtype=torch.int64, device="cuda")
    path[0] = 0
    for d in range(1, s["depth"] + 1):
        nxt = go[node]
        on = nxt >= 0
        node = torch.where(on, nxt, node)
        path[d] = torch.where(on & (n == d), nxt, path[d])
        n = n + (on & (n == d)).long()
    s["path"].copy_(path)
    s["n_path"].copy_(n.view(1))
    s["next"].copy_(bonus[node].view(1))
    return dict(path=s["path"], n_path=s["n_path"], next=s["next"])


_run_own = dict(attend=_own_attend, fill=_own_fill, commit=_own_commit, score=_own_score, evict=_own_evict,
                sample=_own_sample)
_run_plain = dict(attend=_plain_attend, fill=_plain_fill, commit=_plain_commit, score=_plain_score,
                  evict=_plain_evict, sample=_plain_sample)


# ---------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    c = case
    kind = c["kind"]
    if kind == "attend":
        b = f = 0
        for T, L in _seq(c):
            b += c["nkv"] * (144 * L + 512 * T) + T * c["nh"] * (4 * D + 4) + 16 * T
            f += 4 * T * c["nh"] * D * (L + T)
        return dict(bytes=b, flops=f)
    rows = c.get("layers", 0) * c.get("nkv", 0)
    if kind == "fill":   # bf16 rows in, 4-bit rows out, bf16 rows out
        return dict(bytes=rows * c["n"] * (512 + 144 + 512), flops=rows * c["n"] * 256 * 6)
    if kind == "commit":
        return dict(bytes=rows * c["accepted"] * (512 + 144 + 512), flops=rows * c["accepted"] * 256 * 6)
    if kind == "score":
        n, L = c["accepted"], c["L"]
        q = c["layers"] * n * c["nh"] * (D * (4 if c["dtype"] == "f32" else 2) + 4)
        return dict(bytes=rows * (L * (72 + 8) + n * (256 + 4)) + q,
                    flops=2 * D * c["layers"] * c["nh"] * n * (L + n))
    if kind == "evict":  # sums in, kept rows moved, their positions, sums and bf16 values out
        n = min(c["L"], c["budget"])
        return dict(bytes=rows * (4 * c["L"] + n * (144 + 144 + 4 + 4 + 512)), flops=rows * n * 256 * 2)
    # the root's row and one accepted child's: which rows a pass needs depends on the draws
    n = min(2, c["T"]) * c["vocab"]
    return dict(bytes=4 * n * (2 if c["draft"] else 1), flops=20 * n)


# ---------------------------------------------------------------------------
# 64-bit values, one head or node at a time


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return dict(attend=_exact_attend, fill=_exact_fill, commit=_exact_commit, score=_exact_score,
                evict=_exact_evict, sample=_exact_sample)[case["kind"]](s)


def _row_values(words, scale, zero):
    """[n][16][..8 codes] words of whole rows -> float64 [n][128]: group j of a
    row is words 8 j .. 8 j + 7."""
    e = torch.arange(8, device=words.device)
    c = (words[..., None] >> (4 * (e // 2) + 16 * (e % 2))) & 15
    c = c.reshape(words.shape[0], D).double()
    j = torch.arange(D, device=words.device) // 64
    return c * scale.double()[:, j] + zero.double()[:, j]


def _head64(blocks, n):
    """float64 keys and values [n][128] of one head's blocks, position by
    position from the layout's definition."""
    pos = torch.arange(n, device="cuda")
    b, p = pos // BLOCK, pos % BLOCK
    w = blocks.view(torch.int32).long() & 0xffffffff                          # [nb][1152]
    dim8 = torch.arange(16, device="cuda")                                    # dims 8 j .. 8 j + 7
    lane = (4 * (p // 8) + p % 4)[:, None] + 16 * (dim8 % 4)[None]
    at = ((p // 4 % 2)[:, None] * 64 + lane) * 4 + (dim8 // 4)[None]
    kw = w[b[:, None], at]
    dim = torch.arange(D, device="cuda")
    lane = 16 * (p // 8)[:, None] + (dim % 16)[None]
    at = 512 + ((dim // 64)[None] * 64 + lane) * 4 + (dim // 16 % 4)[None]
    e = (p % 8)[:, None]
    vc = (w[b[:, None], at] >> (4 * (e // 2) + 16 * (e % 2))) & 15

    def pairs(base):
        x = w[b[:, None], base + 2 * p[:, None] + torch.arange(2, device="cuda")[None]]
        low, high = ((x & 0xffff) << 16).int(), (x >> 16 << 16)
        high = torch.where(high >= 1 << 31, high - (1 << 32), high).int()
        low = torch.where((x & 0xffff) >= 1 << 15, ((x & 0xffff) << 16) - (1 << 32), (x & 0xffff) << 16).int()
        return low.view(torch.float32), high.view(torch.float32)
    j = dim // 64
    vs, vz = pairs(1088)
    v = vc.double() * vs.double()[:, j] + vz.double()[:, j]
    return _row_values(kw, *pairs(1024)), v


def _exact_attend(s):
    c = s["case"]
    G = c["nh"] // c["nkv"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    t0 = 0
    for x in s["seqs"]:
        T, L = x["T"], x["L"]
        m = s["mask"][t0:t0 + T].cpu().numpy().view(np.uint64)
        vis = np.array([[bool(int(m[i, j // 64]) >> (j % 64) & 1) for j in range(T)] for i in range(T)])
        hide = torch.from_numpy(~vis).cuda()
        for h in range(c["nkv"]):
            k, v = _head64(x["blocks"][0, h], L)
            k = torch.cat((k, x["tail"][0][0, h, :T].double()))
            v = torch.cat((v, x["tail"][1][0, h, :, :T].double().t()))
            for a in range(h * G, h * G + G):
                sc = s["q"][t0:t0 + T, a].double() @ k.t() / math.sqrt(D)
                sc[:, L:].masked_fill_(hide, -math.inf)
                out[t0:t0 + T, a] = torch.softmax(sc, -1) @ v
                lse[t0:t0 + T, a] = torch.logsumexp(sc, -1)
        t0 += T
    return dict(out=out, lse=lse)


def _quant64(x):
    """The values that bf16 rows [n][128] are held as.  The scale and the codes
    are defined by float32 operations on bfloat16 numbers; numpy's are."""
    f = x.float().cpu().numpy().reshape(-1, 2, 64)
    z = f.min(-1)
    s = torch.from_numpy((f.max(-1) - z) / np.float32(15)).bfloat16().float().numpy()
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(s[..., None] > 0, np.minimum(np.rint((f - z[..., None]) / s[..., None]), 15), 0)
    return torch.from_numpy((c.astype(np.float64) * s[..., None] + z[..., None]).reshape(-1, D)).cuda()


def _exact_rows(s, rows):
    """k, v outputs (float64) of rows(layer, head) -> (keys, values) [n][128]."""
    c, n = s["case"], s["n"]
    k = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
    v = torch.zeros(s["v_out"].shape, dtype=torch.float64, device="cuda")
    for l in range(c["layers"]):
        for h in range(c["nkv"]):
            a, b = rows(l, h)
            k[l, h, :n] = a
            v[l, h, :, :n] = b.t()
    return dict(k=k, v=v)


def _exact_fill(s):
    sp, n = s["case"]["src_pos"], s["n"]
    return _exact_rows(s, lambda l, h: (_quant64(s["k"][l, h, sp:sp + n]), _quant64(s["v"][l, h, :, sp:sp + n].t())))


def _exact_commit(s):
    at = s["path"][:s["n"]].long()
    return _exact_rows(s, lambda l, h: (_quant64(s["tail"][0][l, h, at]), _quant64(s["tail"][1][l, h].t()[at])))


def _exact_score(s):
    c = s["case"]
    L, n = c["L"], c["accepted"]
    G = c["nh"] // c["nkv"]
    out = torch.zeros(s["score_out"].shape, dtype=torch.float64, device="cuda")
    for l in range(c["layers"]):
        for h in range(c["nkv"]):
            k = torch.cat((_head64(s["blocks"][l, h], L)[0], s["tail"][0][l, h][s["path"][:n].long()].double()))
            out[l, h, :L] = s["score"][l, h, :L].double()
            for i, node in enumerate(s["nodes"]):
                for a in range(h * G, h * G + G):
                    x = k[:L + i + 1] @ s["q"][l, node, a].double() / math.sqrt(D) - s["lse"][l, node, a].double()
                    out[l, h, :L + i + 1] += torch.exp(x)
    return dict(score=out)


def _exact_evict(s):
    c = s["case"]
    L, n, sink, recent = c["L"], s["n"], c["sink"], c["recent"]
    kept = np.zeros(tuple(s["kept"].shape), np.int64)
    score = s["score"].double().cpu().numpy()
    out = np.zeros(tuple(s["score_out"].shape))
    for l in range(c["layers"]):
        for h in range(c["nkv"]):
            mid = np.arange(sink, L - recent)
            order = np.lexsort((mid, -score[l, h, mid]))[:n - sink - recent]
            at = np.concatenate((np.arange(sink), np.sort(mid[order]), np.arange(L - recent, L)))
            kept[l, h, :n] = at
            out[l, h, :n] = score[l, h, at]
    at = torch.from_numpy(kept).cuda()

    def rows(l, h):
        k, v = _head64(s["blocks"][l, h], L)
        return k[at[l, h, :n]], v[at[l, h, :n]]
    return dict(kept=at, score=torch.from_numpy(out).cuda(), **_exact_rows(s, rows))


def _exact_sample(s):
    c = s["case"]
    T, V = c["T"], c["vocab"]
    u = s["u"].cpu().numpy().astype(np.float64)
    ids = s["ids"].cpu().numpy()
    node, path = 0, [0]
    while True:
        x = s["logits"][node].cpu().numpy().astype(np.float64)
        r = np.exp((x - x.max()) / c["temperature"])
        q = s["draft"][node].cpu().numpy().astype(np.float64) if c["draft"] else None
        took = -1
        for ch in s["kids"][node]:
            t = ids[ch]
            if u[ch] * (q[t] if c["draft"] else 1.0) * r.sum() < r[t]:
                took = ch
                break
            r = np.maximum(r - r.sum() * q, 0.0) if c["draft"] else np.where(np.arange(V) == t, 0.0, r)
        if took < 0:
            break
        node = took
        path.append(node)
    bonus = int(np.argmax(np.cumsum(r) > u[0] * r.sum()))
    return dict(path=torch.tensor(path + [-1] * (T - len(path)), device="cuda"),
                n_path=torch.tensor([len(path)], device="cuda"), next=torch.tensor([bonus], device="cuda"))
