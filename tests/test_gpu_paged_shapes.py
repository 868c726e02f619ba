"""Every shape of the paged attention's workgroups -- 1, 2, 4 and 8 tiles of 16 rows,
with and without splits -- with bfloat16 and float32 queries, and in the step, whose
queries are operand planes.  The shape follows the tables' width, so wide tables with
short lengths reach them all."""
import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2405_18628_amd as ppd
from gpu_cases import check_logits, check_pred, make_case, oracle_step, tree_for
from synth import workload
from test_gpu_paged import BF, Pool, attend, dev, new_rows, offsets, tree_masks
from test_gpu_paged_step import Paged, joined

pytestmark = pytest.mark.gpu

# lens, T, heads, kv heads, page, positions of the tables, tiles of a workgroup
SHAPES = [([900], [16], 2, 2, 32, 900, 1), ([40], [30], 2, 2, 32, 40, 1),
          ([3000], [20], 2, 2, 32, 1 << 19, 2), ([700, 0, 260], [30, 20, 25], 3, 3, 64, 1 << 19, 2), ([100], [17], 1, 1, 32, 1 << 19, 2),
          ([2500], [6], 8, 2, 128, 1 << 19, 2), ([5000], [32], 1, 1, 64, 1 << 19, 2),
          ([2000], [60], 2, 2, 32, 4096 * 16, 2), ([300] * 70, [9] * 70, 2, 1, 32, 1 << 19, 2),
          ([1500], [40], 2, 2, 32, 1 << 19, 4), ([50], [64], 1, 1, 32, 1 << 19, 4), ([600, 333], [40, 45], 2, 1, 64, 1 << 19, 8),
          ([4000], [128], 1, 1, 32, 1 << 19, 8), ([100], [100], 2, 2, 256, 1 << 19, 8)]


def tiles_of(heads, kv_heads, seqs, rows, positions, page):
    """The rule by which a call chooses them, from what the host knows."""
    tiles = min(64, -(-min(-(-rows // seqs), 128) * (heads // kv_heads) // 16))
    blocks = (positions // page * (page // 32) + 1) * kv_heads * min(seqs, rows)
    if tiles == 1 or blocks * tiles <= 48 * 256:
        return 1
    if tiles == 2 or blocks * ((tiles + 1) // 2) <= 96 * 256:
        return 2
    return 4 if tiles <= 4 else 8


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_attention_in_every_shape(case, dtype):
    lens, T, nh, nkv, page, width, tiles = SHAPES[case]
    rows = sum(T)
    pool = Pool(lens, nkv, page, seed=case)
    tk, tv = new_rows(nkv, (rows + 15) // 8 * 8, rows)
    kv, pt = pool.on_gpu(tk, tv, -(-width // page))
    assert tiles_of(nh, nkv, len(T), rows, pt.max_pages * page, page) == tiles
    q = torch.randn((rows, nh, 128), generator=torch.Generator().manual_seed(case)).to(dtype)
    m = tree_masks(np.random.default_rng(case), T)
    m[rows // 2] = 0
    row_start = offsets(T)
    out, lse, ws = attend(kv, pt, dev(row_start), q.cuda(), torch.from_numpy(m.view(np.int64)).cuda())
    assert ppd.ppd_device_status(ws) == 0
    R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, row_start, q, m, page).check(out, lse)
    again = attend(kv, pt, dev(row_start), q.cuda(), torch.from_numpy(m.view(np.int64)).cuda(), ws=ws)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("T,tiles", [(16, 1), (30, 2), (50, 4), (100, 8)])
def test_attention_over_listed_pages_in_every_shape(T, tiles, dtype):
    """The budget takes the tables' place in the choice of the shape."""
    L, page, nkv, nh, budget = 4000, 32, 1, 1, 16384
    pool = Pool([L], nkv, page, seed=T)
    tk, tv = new_rows(nkv, 128, T)
    kv, pt = pool.on_gpu(tk, tv, budget)
    assert tiles_of(nh, nkv, 1, T, budget * page, page) == tiles
    sel = np.full((1, nkv, budget), -3, np.int32)
    listed = np.sort(np.random.default_rng(T).permutation(L // page)[:61])
    sel[0, 0, :61] = listed
    q = torch.randn((T, nh, 128), generator=torch.Generator().manual_seed(T)).to(dtype)
    out, lse, ws = attend(kv, pt, dev([0, T]), q.cuda(), None, sel=dev(sel), n_sel=dev([61]))
    assert ppd.ppd_device_status(ws) == 0
    R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, [0, T], q, None, page, torch.from_numpy(sel),
                np.array([61])).check(out, lse)


# the model's heads a kv head make rows of tokens
STEPS = [("small", [700], ["total:16"], 700, 1), ("small", [700], ["total:29"], 1 << 19, 2), ("small-gqa", [700], ["total:13"], 1 << 19, 2),
         ("small", [900], ["total:50"], 1 << 19, 4), ("small", [200, 640], ["total:40", "total:60"], 1 << 19, 4),
         ("small", [900], ["total:128"], 1 << 19, 8), ("small", [30], ["total:100"], 1 << 19, 8)]


@pytest.mark.parametrize("budget", [0, 5, 16384])
@pytest.mark.parametrize("case", range(len(STEPS)))
def test_step_in_every_shape(case, budget):
    """Logits against the oracle's and the contiguous step's, with all pages; with a
    budget those of a step that selects as much in tight tables (a budget of more than
    the tables hold leaves the shape to their width)."""
    name, lens, specs, width, tiles = STEPS[case]
    page = 32
    c = make_case(workload(name, cache_len=max(lens)))
    sh = c.shape
    trees = [tree_for(c, spec=s, seed_offset=i) for i, s in enumerate(specs)]
    T = [t.T for t in trees]
    B, rows, n_pages = len(T), sum(T), sum(-(-n // page) for n in lens) + 2
    cols = max(width, max(lens)) // page + 1
    tt, row_start = joined(trees), dev(offsets(T))
    p = Paged(c, B, page, n_pages, cols, rows, budget)
    p.prompts(c.k, c.v, lens)
    if budget:
        tight = Paged(c, B, page, n_pages, max(lens) // page + 1, rows, budget)
        tight.prompts(c.k, c.v, lens)
        for q in (p, tight):
            q.verify(row_start, tt, budget=budget, n_first=1, n_last=2)
            assert q.clean()
        assert float((p.logits - tight.logits).abs().max()) < 1e-3
        return
    assert tiles_of(sh.n_heads, sh.n_kv_heads, B, rows, cols * page, page) == tiles
    p.verify(row_start, tt)
    torch.cuda.synchronize()
    assert p.clean()
    ws = p.new_ws(ppd.ppd_workspace_bytes(c.model, rows, c.k.shape[2]))
    logits, pred = torch.empty((rows, sh.vocab), device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
    kvs = [ppd.KVCache(c.k.clone(), c.v.clone()) for _ in range(B)]
    ppd.ppd_verify_batch(c.model, kvs, lens, T, tt["ids"], tt["depth"], tt["mask"], ws, logits, pred)
    assert float((p.logits - logits).abs().max()) < 1e-3
    i = int(np.argmax(T))
    c.kc_host.L = c.vc_host.L = lens[i]
    ref = oracle_step(c, trees[i], L=lens[i])
    a = slice(int(offsets(T)[i]), int(offsets(T)[i]) + T[i])
    check_logits(p.logits[a].cpu().numpy().astype(np.float64), ref["logits"], "bf16")
    check_pred(p.pred[a].cpu().numpy(), ref["logits"], "bf16")
