"""Calls on pages with numbers on the device that are out of range or do not fit
together: what they leave behind, and the bits that name them."""
import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2405_18628_amd as ppd
from gpu_cases import make_case, tree_for
from synth import workload
from test_gpu_paged import BF, Pool, attend, dev, new_rows, workspace
from test_gpu_paged_step import Paged, joined

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,rows,wide", [(64, 64, False), (64, 640, True), (100, 100, False), (100, 1000, True)])
def test_offsets_that_fall_leave_the_workspace_as_it_was(B, rows, wide):
    """Every second sequence with all rows of the call: 64 sequences of 64 rows, 23 of
    them long, would be 880 workgroups on a grid of 464.  No row is written, and the
    next call on the workspace is right.  All sequences read the same pages."""
    nh, L = 4, 4000
    pool = Pool([L], 1, 32, seed=B)
    pool.table = np.repeat(pool.table, B, 0)
    pool.lens = np.where(np.arange(B) % 2 == 0, L, 0).astype(np.int32)
    pool.lens[46:64] = 0
    tk, tv = new_rows(1, (rows + 15) // 8 * 8, rows)
    kv, pt = pool.on_gpu(tk, tv, (1 << 19) // 32 if wide else 0)
    q = torch.randn((rows, nh, 128), generator=torch.Generator().manual_seed(B)).to(BF)
    ws = workspace(ppd.ppd_paged_attention_workspace_bytes(nh, 1, B, rows))
    counts = np.zeros(B, int)
    counts[[0, 1, 2, B - 1]] = 3, 2, 5, 1
    good = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    ref = R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, good, q, None, 32)
    kept = torch.full((rows, nh, 128), 7.0, dtype=BF), torch.full((rows, nh), 7.0)
    falling = np.where(np.arange(B + 1) % 2, rows, 0)
    for bad in (falling, np.where(np.arange(B + 1) == B, 0, good)):
        out, lse, _ = attend(kv, pt, dev(bad), q.cuda(), None, ws=ws)
        assert ppd.ppd_device_status(ws, clear=True) & ppd.PPD_DEV_BAD_LENGTH
        assert torch.equal(out.cpu(), kept[0]) and torch.equal(lse.cpu(), kept[1])
        for _ in range(2):
            out, lse, _ = attend(kv, pt, dev(good), q.cuda(), None, ws=ws)
            assert ppd.ppd_device_status(ws) == 0
            ref.check(out, lse, kept)


@pytest.mark.parametrize("budget", [1, 3, 5, 9])
def test_selection_reports_bad_numbers(budget):
    """Tables of five pages, budgets below and above them (above: no scores are formed)."""
    pool = Pool([150, 50], 2, 32)
    pool.table = np.abs(pool.table[:, :5]) % pool.n_pages
    tk, tv = new_rows(2, 8, 8)
    kv, pt = pool.on_gpu(tk, tv)
    assert pt.max_pages == 5
    q = torch.randn((8, 2, 128), device="cuda").to(BF)
    ws = workspace(ppd.ppd_paged_select_workspace_bytes(2, 2, 5))
    sel, n_sel = torch.full((2, 2, budget), -8, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for length, rows in (([150, 50], [0, 4, 8]), ([-1, 50], [0, 4, 8]), ([150, 161], [0, 4, 8]), ([10 ** 9, 50], [0, 4, 8]),
                         ([150, 50], [0, 4, 9]), ([150, 50], [-2 ** 31, 4, 2 ** 31 - 1]), ([150, 50], [6, 2, 8])):
        pt.len.copy_(dev(length))
        ppd.ppd_paged_select(kv, 0, pt, dev(rows), q, budget, 0, 1, sel, n_sel, ws)
        bad = length != [150, 50] or rows != [0, 4, 8]
        assert ppd.ppd_device_status(ws, clear=True) == (ppd.PPD_DEV_BAD_LENGTH if bad else 0), (length, rows)
        want = [min(budget, -(-min(max(n, 0), 160) // 32)) for n in length]
        assert n_sel.tolist() == want
        for s, m in enumerate(want):
            picked = sel[s, :, :m]
            assert bool(((picked >= 0) & (picked < 5)).all()) and bool((picked[:, 1:] > picked[:, :-1]).all())


@pytest.mark.parametrize("budget", [0, 3])
def test_a_step_reports_rows_that_no_sequence_has(budget):
    case = make_case(workload("small-gqa", cache_len=150))
    trees = [tree_for(case, spec=s, seed_offset=i) for i, s in enumerate(("total:16", "chain:7"))]
    T0, n = trees[0].T, sum(t.T for t in trees)
    p = Paged(case, 2, 32, 20, 8, n, budget)
    p.prompts(case.k, case.v, [150, 70])
    tt = joined(trees)

    def step(offsets):
        p.logits.fill_(7.0)
        p.verify(dev(offsets), tt, budget=budget, n_last=min(1, budget))
        return p.logits.clone(), ppd.ppd_device_status(p.ws, clear=True)

    right, status = step([0, T0, n])
    assert status == 0
    for offsets, rows in (([0, T0, n - 2], slice(0, n - 2)), ([0, T0, T0], slice(0, T0)), ([2, T0, n], slice(T0, n)),
                          ([0, T0, n + 5], slice(0, n)), ([0, n, T0], slice(0, 0))):
        logits, status = step(offsets)
        assert status & ppd.PPD_DEV_BAD_LENGTH, offsets
        assert not len(logits[rows]) or float((logits[rows] - right[rows]).abs().max()) < 1e-3, offsets
    again, status = step([0, T0, n])
    assert status == 0 and torch.equal(again, right)
    again, status = step([0, 0, n])      # a sequence that sits out: every row is the other's
    assert status == 0


@pytest.mark.parametrize("B", [1, 2, 70])
def test_offsets_at_the_ends_of_32_bits_stay_inside(B):
    """A difference of offsets that passes 32 bits is no number of rows: what lies
    behind the call's rows stays as it was."""
    n, nh, low, high = 8, 2, -2 ** 31, 2 ** 31 - 1
    pool = Pool([100], 1, 32)
    pool.table, pool.lens = np.repeat(pool.table, B, 0), np.full(B, 100, np.int32)
    tk, tv = new_rows(1, 8, n)
    kv, pt = pool.on_gpu(tk, tv)
    q = torch.randn((n + 256, nh, 128), generator=torch.Generator().manual_seed(B)).to(BF).cuda()
    ws = workspace(max(ppd.ppd_paged_attention_workspace_bytes(nh, 1, B, n), ppd.ppd_paged_select_workspace_bytes(1, B, pt.max_pages)))
    out, lse = torch.full_like(q, 7.0), torch.full((n + 256, nh), 7.0, device="cuda")
    sel, n_sel = dev(np.zeros((B, 1, 2))), dev(np.zeros(B))
    for ends in ((5, low), (low, high), (high, low), (low, 5), (3, high), (n, low), (0, low), (low, low), (high, high)):
        offsets = np.concatenate((np.full(B, ends[0]), [ends[1]])) if B < 3 else np.concatenate((np.full(B // 2, ends[0]), np.full(B // 2 + 1, ends[1])))
        rows = dev(offsets.astype(np.int64))
        for listed in (False, True):
            if listed:
                ppd.ppd_paged_select(kv, 0, pt, rows, q[:n], 2, 0, 1, sel, n_sel, ws)
                assert ppd.ppd_device_status(ws, clear=True) == ppd.PPD_DEV_BAD_LENGTH, ends
            ppd.ppd_paged_attention(kv, 0, pt, rows, q[:n], None, out[:n], ws, lse[:n], *((sel, n_sel) if listed else ()))
            assert ppd.ppd_device_status(ws, clear=True) == ppd.PPD_DEV_BAD_LENGTH, ends
            assert bool((out[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all()), ends
    good = dev(np.minimum(np.arange(B + 1) * 4, n))
    ppd.ppd_paged_attention(kv, 0, pt, good, q[:n], None, out[:n], ws, lse[:n])
    assert ppd.ppd_device_status(ws) == 0
    ref = R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, good.tolist(), q[:n].cpu(), None, 32)
    ref.check(out[:n], lse[:n])


def test_any_calls_in_turn_share_a_workspace():
    """Split attention on a workspace whose scratch holds what other calls left there:
    bytes of ones, a step's, a selection's, another batch's.  The header keeps nothing."""
    case = make_case(workload("small-gqa", cache_len=150))
    tree = tree_for(case, spec="total:16")
    p = Paged(case, 1, 32, 20, 8, tree.T, 3)
    p.prompts(case.k, case.v, [150])
    runs = []
    for i, (lens, nkv, nh, T) in enumerate((([3000, 900], 2, 4, [5, 1]), ([700] * 40, 1, 2, [1] * 40), ([5000], 3, 3, [20]))):
        pool = Pool(lens, nkv, 64, seed=i)
        tk, tv = new_rows(nkv, 40, sum(T), seed=i)
        kv, pt = pool.on_gpu(tk, tv)
        q = torch.randn((sum(T), nh, 128), generator=torch.Generator().manual_seed(i)).to(BF).cuda()
        rows = dev(np.concatenate(([0], np.cumsum(T))))
        out, lse, ws = attend(kv, pt, rows, q, None)
        runs.append((kv, pt, rows, q, out, lse, ws.numel(), dev(np.zeros((len(lens), nkv, 2))), dev([0] * len(lens))))
    size = max([r[6] for r in runs] + [p.ws.numel(), ppd.ppd_workspace_bytes(case.model, 16, case.k.shape[2])])
    ws = workspace(size)
    ws[256:] = 255
    steps = (lambda r: None, lambda r: ppd.ppd_verify_batch_paged(case.model, p.kv, p.pt, dev([0, tree.T]), tt["ids"], tt["depth"],
                                                                  tt["mask"], ws, p.logits, p.pred, budget=3, n_last=1),
             lambda r: ppd.ppd_paged_select(r[0], 0, r[1], r[2], r[3], 2, 0, 1, r[7], r[8], ws),
             lambda r: ppd.ppd_paged_tables(p.pt, dev([0]), p.start, dev([0]), ws),
             lambda r: ppd.ppd_verify_step(case.model, ppd.KVCache(case.k, case.v), 150, tree.T, tt["ids"], tt["depth"], tt["mask"], ws,
                                           p.logits, p.pred), lambda r: ws[256:].fill_(3))
    tt = joined([tree])
    for between in steps:
        for r in runs:
            between(r)
            out, lse, _ = attend(*r[:4], None, ws=ws)
            assert ppd.ppd_device_status(ws) == 0 and not ws[:256].any()
            assert torch.equal(out, r[4]) and torch.equal(lse, r[5])


@pytest.mark.parametrize("B", [1, 3, 400])
def test_pages_given_back_stay_in_the_ring(B):
    """Tables wider than the pool, and lengths on the device of more pages than it has."""
    n, width = 6, 20
    ring = torch.full((n + 64,), -9, dtype=torch.int32, device="cuda")
    ring[:n] = torch.arange(n, dtype=torch.int32)
    pt = ppd.PageTables(torch.zeros((B, width), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"),
                        ring[:n], dev([4, 3]), 32)
    start, slots = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    ws = workspace(ppd.ppd_paged_tables_workspace_bytes(B))
    for length in (width * 32, 10 ** 9, 7 * 32):
        pt.len.fill_(length)
        ppd.ppd_paged_tables(pt, dev(np.full(B, -1)), start, slots, ws)
        assert ppd.ppd_device_status(ws, clear=True) == ppd.PPD_DEV_BAD_LENGTH
        assert bool((ring[n:] == -9).all()) and not pt.len.any() and 0 <= int(pt.free_state[1]) <= n
