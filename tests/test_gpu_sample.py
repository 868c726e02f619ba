"""Sampled acceptance on the GPU against the plain 64-bit walk
(kvq_reference.accept_sample): the same path, count and bonus token.  Both
compute in float64, so a decision differs only where a draw falls within about
1e-13 of a border, which no seed here does."""
import numpy as np
import pytest
import torch

import kvq_reference as R
import paper_2405_18628_amd as ppd
from gpu_cases import say

pytestmark = pytest.mark.gpu


def _dev(a, dt=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dt, device="cuda")


def _call(parent, ids, V, logits, temperature, draft, u, stream=None, bufs=None):
    T = len(parent)
    ws = torch.empty(ppd.ppd_accept_sample_workspace_bytes(T, V), dtype=torch.uint8, device="cuda").fill_(255)
    ppd.ppd_workspace_init(ws)
    path, n, nxt = (torch.full((k,), -9, dtype=torch.int32, device="cuda") for k in (T, 1, 1))
    lg = torch.from_numpy(logits).cuda()
    dr = None if draft is None else torch.from_numpy(draft).cuda()
    ud = torch.from_numpy(u).cuda()
    p, i = _dev(parent), _dev(ids)
    torch.cuda.synchronize()
    ppd.ppd_accept_sample(T, p, i, V, lg, temperature, dr, ud, path, n, nxt, ws, stream=stream)
    torch.cuda.synchronize()
    n = int(n.item())
    assert path[n:].cpu().tolist() == [-1] * (T - n)
    return path[:n].cpu().tolist(), int(nxt.item()), ppd.ppd_device_status(ws)


def _tree(rng, T, style):
    parent = [-1]
    for i in range(1, T):
        parent.append(0 if style == "flat" else i - 1 if style == "chain" else int(rng.integers(max(0, i - 9), i)))
    return parent


def _check(parent, ids, V, logits, temperature, draft, u, status=0, **kw):
    path, bonus, flagged = R.accept_sample(parent, ids, V, logits, temperature, draft, u)
    got = _call(parent, ids, V, logits, temperature, draft, u, **kw)
    assert got[0] == path and got[1] == bonus, (got, path, bonus)
    assert got[2] == (status | (ppd.PPD_DEV_NAN_LOGIT if flagged else 0))
    return path


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("T,V,style", [(1, 1, "tree"), (1, 1000, "tree"), (2, 2, "chain"), (20, 7, "tree"), (16, 1025, "flat"),
                                       (64, 4096, "tree"), (128, 333, "tree"), (128, 60, "chain"), (33, 32001, "tree"),
                                       (9, 50257, "flat"), (5, 131075, "tree"), (3, 300000, "tree")])
def test_accept_sample(T, V, style, with_draft):
    say(f"[sample] T={T} V={V} {style} draft={with_draft}")
    rng = np.random.default_rng(T * 31 + V)
    lengths = set()
    for trial in range(6 if V < 60000 else 2):
        parent = _tree(rng, T, style)
        temperature = float(rng.choice([0.25, 0.7, 1.0, 2.0]))
        logits = (rng.standard_normal((T, V)) * 2).astype(np.float32)
        draft = None
        ids = rng.integers(0, V, T).astype(np.int32)
        if with_draft:
            z = logits / temperature + rng.standard_normal((T, V)).astype(np.float32)
            draft = np.exp(z - z.max(-1, keepdims=True))
            draft = (draft / draft.sum(-1, keepdims=True)).astype(np.float32)
            for i in range(1, T):
                ids[i] = rng.choice(V, p=draft[parent[i]] / draft[parent[i]].sum(dtype=np.float64))
        else:
            for i in range(1, T):  # likely children, as a drafter's best tokens are
                logits[parent[i], ids[i]] += temperature * (np.log(V) + rng.uniform(-1, 3))
        for i in range(1, T):
            if style == "tree" and rng.random() < 0.2:
                ids[i] = V + rng.integers(0, 3)      # a prompt token
            if rng.random() < 0.1:
                ids[i] = ids[max(0, i - 1)]          # a sibling's token again
        lengths.add(len(_check(parent, ids, V, logits, temperature, draft, rng.random(T).astype(np.float32))))
    if T >= 16 and V < 60000:
        assert max(lengths) > 1                      # some children were accepted


@pytest.mark.parametrize("with_draft", [False, True])
def test_a_vocabulary_of_millions(with_draft):
    """More parts of a row than the walk has threads, more chunks than one pass sums."""
    rng = np.random.default_rng(8)
    T, V = 3, 4300001
    parent, ids = [-1, 0, 1], np.array([0, 4299999, 17], np.int32)
    logits = rng.standard_normal((T, V)).astype(np.float32)
    logits[0, 4299999] = logits[1, 17] = np.log(V) + 2.0
    draft = np.full((T, V), 1 / V, np.float32) if with_draft else None
    for u0 in (0.001, 0.5, 0.9999):
        for u1 in (0.0, 0.99):
            _check(parent, ids, V, logits, 1.0, draft, np.array([u0, u1, u1], np.float32))


@pytest.mark.parametrize("with_draft", [False, True])
def test_rows_with_infinities_and_nan(with_draft):
    rng = np.random.default_rng(3)
    T, V = 6, 50
    parent, ids = [-1, 0, 0, 1, 1, 2], np.array([0, 3, 4, 3, 9, 7], np.int32)
    draft = np.full((T, V), 1 / V, np.float32) if with_draft else None
    base = rng.standard_normal((T, V)).astype(np.float32)
    kinds = {"banned": lambda x: np.where(np.arange(V) % 3 == 0, x, -np.inf), "nan": lambda x: np.where(np.arange(V) == 20, np.nan, x),
             "empty": lambda x: np.full(V, -np.inf), "all nan": lambda x: np.full(V, np.nan),
             "infinite": lambda x: np.where(np.isin(np.arange(V), [3, 8]), np.inf, x),
             "lowest": lambda x: np.where(np.arange(V) % 2 == 0, np.finfo(np.float32).min, x),
             "one": lambda x: np.where(np.arange(V) == 3, 0.0, -np.inf)}
    for name, f in kinds.items():
        for trial in range(4):
            logits = base.copy()
            logits[:] = np.stack([f(r) for r in base]).astype(np.float32)
            say(f"[sample] {name} {trial}")
            _check(parent, ids, V, logits, 1.0, draft, rng.random(T).astype(np.float32))


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("scale,temperature", [(3e9, 4.0), (1e30, 1.0), (1e-3, 1e-30), (700.0, 1.0), (2e3, 2.8), (1.0, 1e30),
                                               (3e38, 1e36), (50.0, 0.07)])
def test_far_logits_and_temperatures(scale, temperature, with_draft):
    """Logits whose neighbours lie further apart than any weight reaches, and
    weights down to the smallest number."""
    rng = np.random.default_rng(7)
    T, V = 9, 5000
    parent, ids = _tree(rng, T, "tree"), rng.integers(0, V, T).astype(np.int32)
    draft = np.full((T, V), 1 / V, np.float32) if with_draft else None
    for trial in range(3):
        logits = (rng.uniform(-1, 1, (T, V)) * scale).astype(np.float32)
        u = rng.random(T).astype(np.float32)
        _check(parent, ids, V, logits, temperature, draft, u)


def test_borders_of_the_draws():
    """Draws of 0 take the first token that has weight, draws of 1 (out of
    range) the last; a draw of 0 accepts every child that has weight."""
    V = 40
    logits = np.full((2, V), -np.inf, np.float32)
    logits[:, 5:30] = 0.0
    for u0, bonus in ((0.0, 5), (1.0, 29), (7.0, 29), (0.5, 17)):
        got = _call([-1, 0], [0, 31], V, logits, 1.0, None, np.array([u0, 0.5], np.float32))
        assert got == ([0], bonus, 0), (u0, got)
    assert _call([-1, 0], [0, 31], V, logits, 1.0, None, np.array([0.0, 0.0], np.float32))[0] == [0]      # no weight
    assert _call([-1, 0], [0, 29], V, logits, 1.0, None, np.array([0.0, 0.0], np.float32))[0] == [0, 1]
    # all weight on a token that is rejected by a draw of 1: the residual is empty, the bonus token drawn from the weights
    logits[:] = -np.inf
    logits[:, 7] = 1.0
    for draft in (None, np.eye(V, dtype=np.float32)[[7, 7]]):
        got = _call([-1, 0, 0], [0, 7, 7], V, np.concatenate((logits, logits[:1])), 1.0,
                    draft if draft is None else np.concatenate((draft, draft[:1])), np.array([0.5, 1.0, 1.0], np.float32))
        assert got == ([0], 7, 0)


def test_draft_rows_of_any_kind():
    """Rows that do not add up to 1, negative and NaN entries, no probability for the drafted token."""
    rng = np.random.default_rng(11)
    T, V = 12, 200
    for trial in range(8):
        parent = _tree(rng, T, "tree")
        draft = (rng.random((T, V)) * rng.choice([0.001, 0.01, 1.0])).astype(np.float32)
        draft[:, ::5] = 0.0
        draft[:, 1::7] = -1.0
        draft[:, 2::11] = np.nan
        ids = rng.integers(0, V, T).astype(np.int32)
        _check(parent, ids, V, rng.standard_normal((T, V)).astype(np.float32), 0.9, draft, rng.random(T).astype(np.float32))


def test_bad_parents_are_clamped():
    rng = np.random.default_rng(2)
    logits = rng.standard_normal((5, 64)).astype(np.float32)
    u = rng.random(5).astype(np.float32)
    bad, fixed = [-1, 0, 5, -3, 3], [-1, 0, 0, 0, 3]
    _check_ids = np.array([1, 2, 3, 4, 5], np.int32)
    got = _call(bad, _check_ids, 64, logits, 1.0, None, u)
    path, bonus, _ = R.accept_sample(fixed, _check_ids, 64, logits, 1.0, None, u)
    assert got == (path, bonus, ppd.PPD_DEV_BAD_PARENT)


def test_unaligned_rows_and_another_stream():
    """An odd vocabulary in a buffer that starts 4 bytes past a 16-byte border."""
    rng = np.random.default_rng(4)
    T, V = 7, 1003
    parent = _tree(rng, T, "tree")
    ids = rng.integers(0, V, T).astype(np.int32)
    logits = rng.standard_normal((T, V)).astype(np.float32)
    u = rng.random(T).astype(np.float32)
    buf = torch.zeros(T * V + 1, device="cuda")
    lg = buf[1:].view(T, V)
    lg.copy_(torch.from_numpy(logits))
    ws = torch.zeros(ppd.ppd_accept_sample_workspace_bytes(T, V), dtype=torch.uint8, device="cuda")
    path, n, nxt = (torch.zeros(k, dtype=torch.int32, device="cuda") for k in (T, 1, 1))
    args = (T, _dev(parent), _dev(ids), V, lg, 1.0, None, torch.from_numpy(u).cuda(), path, n, nxt, ws)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    ppd.ppd_accept_sample(*args, stream=s)
    s.synchronize()
    want = R.accept_sample(parent, ids, V, logits, 1.0, None, u)
    assert path[:int(n)].cpu().tolist() == want[0] and int(nxt) == want[1]
    # captured; the draws change between replays, as they do in a loop
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ppd.ppd_accept_sample(*args)
    for r in range(4):
        u = rng.random(T).astype(np.float32)
        args[7].copy_(torch.from_numpy(u))
        g.replay()
        torch.cuda.synchronize()
        want = R.accept_sample(parent, ids, V, logits, 1.0, None, u)
        assert path[:int(n)].cpu().tolist() == want[0] and int(nxt) == want[1], r
