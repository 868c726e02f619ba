"""Page tables, rows into pages, attention over pages and the choice of pages on
the GPU, against the plain forms of paged_reference (whole numbers and moved
rows equal; attention within bounds that count its roundings)."""
import math

import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2405_18628_amd as ppd

pytestmark = pytest.mark.gpu
I32, BF = torch.int32, torch.bfloat16
NAN = float("nan")


def dev(a, dtype=I32):
    return torch.as_tensor(np.asarray(a), dtype=dtype).cuda()


def offsets(counts):
    return np.concatenate(([0], np.cumsum(counts))).astype(np.int32)


def workspace(n):
    ws = torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
    ppd.ppd_workspace_init(ws)
    return ws


# ---------------------------------------------------------------------------
# tables


def run_tables(pt, add, n_slots, ws, inplace=True):
    """One call beside the reference; returns start, slots (numpy)."""
    before = [t.cpu().numpy() for t in (pt.table, pt.len, pt.free_pages, pt.free_state)]
    slots0 = np.full(n_slots, -9, np.int32)
    start, slots = torch.full((pt.n_seqs + 1,), -5, dtype=I32, device="cuda"), dev(slots0)
    len_out = state_out = None
    if not inplace:
        len_out, state_out = torch.full_like(pt.len, -3), torch.full_like(pt.free_state, -3)
    ppd.ppd_paged_tables(pt, dev(add), start, slots, ws, len_out, state_out)
    status = ppd.ppd_device_status(ws, clear=True)
    want = R.tables(before[0], before[1], np.asarray(add), before[2], before[3], pt.page, n_slots, slots0)
    got = [t.cpu().numpy() for t in (pt.table, pt.len if inplace else len_out, pt.free_pages,
                                     pt.free_state if inplace else state_out, start, slots)]
    for name, a, b in zip(("table", "len", "ring", "state", "start", "slots"), got, want):
        assert np.array_equal(a, b), name
    assert status == (ppd.PPD_DEV_NO_PAGES if want[6] else 0)
    if not inplace:
        assert np.array_equal(pt.len.cpu().numpy(), before[1]) and np.array_equal(pt.free_state.cpu().numpy(), before[3])
    return got[4], got[5]


@pytest.mark.parametrize("B,page,n_pages,width,most,steps", [(1, 32, 9, 9, 40, 12), (6, 32, 40, 12, 90, 25), (16, 64, 90, 20, 7, 25),
                                                             (65, 128, 130, 5, 200, 8), (300, 32, 2000, 30, 400, 6),
                                                             (1025, 256, 1500, 3, 3, 5), (4096, 32, 9000, 4, 60, 3)])
def test_tables_over_many_steps(B, page, n_pages, width, most, steps):
    r = np.random.default_rng(B)
    pt = ppd.PageTables.empty(B, width, n_pages, page)
    pt.free_pages.copy_(dev(r.permutation(n_pages)))
    pt.free_state.copy_(dev([n_pages - 3, n_pages]))
    ws = workspace(ppd.ppd_paged_tables_workspace_bytes(B))
    for i in range(steps):
        add = np.where(r.random(B) < 0.12, -int(r.integers(1, 9)), r.integers(0, most + 1, B)).astype(np.int32)
        rows = int(np.maximum(add, 0).sum())
        run_tables(pt, add, max(1, rows + [4, 0, -rows // 5][i % 3]), ws, inplace=i % 2 == 0)
        if i % 2:
            run_tables(pt, np.zeros(B, np.int32), 1, ws)
        length = pt.len.cpu().numpy()
        held = [p for s in range(B) for p in pt.table[s, :-(-int(length[s]) // page)].tolist()] if i % 2 == 0 else []
        if held:
            first, count = pt.free_state.tolist()
            ring = pt.free_pages.cpu().numpy()
            assert sorted(held + [int(ring[(first + j) % n_pages]) for j in range(count)]) == list(range(n_pages))


def test_tables_of_one_long_prompt():
    pt = ppd.PageTables.empty(3, 4000, 4100, 64)
    ws = workspace(ppd.ppd_paged_tables_workspace_bytes(3))
    run_tables(pt, np.array([1, 200001, 0], np.int32), 200002, ws)
    run_tables(pt, np.array([7, 0, 100], np.int32), 200, ws)
    run_tables(pt, np.array([-1, -1, -1], np.int32), 5, ws)
    assert pt.free_state[1].item() == 4100


def test_tables_refuse_in_order():
    ws = workspace(ppd.ppd_paged_tables_workspace_bytes(5))
    pt = ppd.PageTables.empty(5, 3, 6, 32)
    # the second passes its table, the third takes what is left but one, the fourth needs two
    run_tables(pt, np.array([64, 97, 96, 33, 1], np.int32), 400, ws)
    assert pt.len.tolist() == [64, 0, 96, 0, 0]
    run_tables(pt, np.array([-1, 32, 0, 32, 32], np.int32), 400, ws)   # pages given back serve the next call
    assert pt.len.tolist() == [0, 32, 96, 0, 0]
    run_tables(pt, np.array([1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 1], np.int32), 4, ws)  # sums past 32 bits
    assert pt.len.tolist() == [1, 32, 96, 0, 0]


def test_tables_with_bad_numbers_stay_inside():
    ws = workspace(ppd.ppd_paged_tables_workspace_bytes(2))
    pt = ppd.PageTables.empty(2, 3, 6, 32)
    start, slots = torch.zeros(3, dtype=I32, device="cuda"), torch.zeros(8, dtype=I32, device="cuda")
    for length, state in (([-5, 7], [0, 6]), ([7, 1000000], [0, 6]), ([7, 7], [9, 4]), ([7, 7], [-1, 4]), ([7, 7], [0, 99])):
        pt.len.copy_(dev(length))
        pt.free_state.copy_(dev(state))
        ppd.ppd_paged_tables(pt, dev([1, 1]), start, slots, ws)
        assert ppd.ppd_device_status(ws, clear=True) & ppd.PPD_DEV_BAD_LENGTH


# ---------------------------------------------------------------------------
# store


@pytest.mark.parametrize("page,layers,nkv,B,tree,off,bounds", [(32, 2, 3, 3, True, 0, True), (64, 1, 2, 5, True, 3, True),
                                                               (32, 2, 2, 2, False, 8, True), (64, 1, 3, 3, False, 5, True),
                                                               (128, 1, 2, 2, False, 0, False), (256, 2, 1, 3, False, 1, True)])
def test_store(page, layers, nkv, B, tree, off, bounds):
    r = np.random.default_rng(page + B)
    width, n_pages = 6, 6 * B + 2
    pt = ppd.PageTables.empty(B, width, n_pages, page)
    pt.free_pages.copy_(dev(r.permutation(n_pages)))
    kv = ppd.PagedCache.empty(layers, nkv, n_pages, page, 8, bounds)
    kv.pages.copy_(torch.randn(kv.pages.shape, device="cuda"))
    if bounds:
        kv.bounds.fill_(NAN)
    ws = workspace(ppd.ppd_paged_tables_workspace_bytes(B))
    pages, bd = kv.pages.cpu(), kv.bounds.cpu() if bounds else None
    for step in range(4):
        add = r.integers(0, 9 if tree else 2 * page, B).astype(np.int32)
        add[r.integers(B)] = 0
        rows = int(add.sum())
        start, slots = run_tables(pt, add, max(rows + 2, 1), ws)
        if step == 2 and rows:
            slots[start[1]:start[2]] = -1           # a refused sequence's
        T = 12
        cap = (int(off + (B * T if tree else rows)) + 15) // 8 * 8
        k = torch.randn((layers, nkv, cap, 128), device="cuda").to(BF)
        v = torch.randn((layers, nkv, 128, cap), device="cuda").to(BF)
        k[..., 7], k[:, :, 1::3, 9] = NAN, NAN
        path = None
        if tree:
            row_start = offsets([T] * B) + off
            path = np.full(int(row_start[-1]), -1, np.int32)
            for s in range(B):
                path[row_start[s]:row_start[s] + add[s]] = np.sort(r.choice(T, add[s], replace=False))
        else:
            row_start = offsets(add) + off
        ppd.ppd_paged_store(kv, ppd.KVCache(k, v), dev(start), dev(row_start), None if path is None else dev(path), dev(slots))
        R.store(pages, bd, k.cpu(), v.cpu(), start.tolist(), row_start.tolist(), path, slots[:rows], page)
        assert torch.equal(kv.pages.cpu().view(torch.int16), pages.view(torch.int16)), step
        if bounds:
            assert torch.equal(kv.bounds.cpu().nan_to_num(77.0), bd.nan_to_num(77.0)), step


@pytest.mark.parametrize("tree", [False, True])
def test_store_of_many_sequences(tree):
    """300 sequences, some without rows; slots that are not 16-byte aligned."""
    r = np.random.default_rng(3)
    B, page, T = 300, 32, 3
    pt = ppd.PageTables.empty(B, 3, 700, page)
    pt.free_pages.copy_(dev(r.permutation(700)))
    kv = ppd.PagedCache.empty(1, 2, 700, page, 8)
    kv.pages.zero_(), kv.bounds.zero_()
    ws = workspace(ppd.ppd_paged_tables_workspace_bytes(B))
    pages, bd = kv.pages.cpu(), kv.bounds.cpu()
    for step in range(3):
        add = r.integers(0, T + 1 if tree else 30, B).astype(np.int32)
        rows, start = int(add.sum()), torch.zeros(B + 1, dtype=I32, device="cuda")
        slots = torch.full((rows + 5,), -9, dtype=I32, device="cuda")[1:]
        before = [t.cpu().numpy() for t in (pt.table, pt.len, pt.free_pages, pt.free_state)]
        ppd.ppd_paged_tables(pt, dev(add), start, slots, ws)
        want = R.tables(before[0], before[1], add, before[2], before[3], page, rows + 4, np.full(rows + 4, -9, np.int32))
        assert np.array_equal(slots.cpu().numpy(), want[5]) and np.array_equal(start.cpu().numpy(), want[4])
        assert np.array_equal(pt.table.cpu().numpy(), want[0]) and ppd.ppd_device_status(ws) == 0
        row_start = offsets([T] * B) if tree else offsets(add)
        path = np.tile(np.arange(T, dtype=np.int32)[::-1], B) if tree else None
        cap = (int(row_start[-1]) + 7) // 8 * 8 + 8
        k, v = torch.randn((1, 2, cap, 128), device="cuda").to(BF), torch.randn((1, 2, 128, cap), device="cuda").to(BF)
        ppd.ppd_paged_store(kv, ppd.KVCache(k, v), start, dev(row_start), None if path is None else dev(path), slots)
        R.store(pages, bd, k.cpu(), v.cpu(), want[4].tolist(), row_start.tolist(), path, want[5][:rows], page)
        assert torch.equal(kv.pages.cpu(), pages) and torch.equal(kv.bounds.cpu(), bd), step


def test_store_leaves_out_what_lies_outside():
    kv = ppd.PagedCache.empty(1, 1, 2, 32, 8)
    kv.pages.zero_(), kv.bounds.zero_()
    k, v = torch.ones((1, 1, 8, 128), dtype=BF, device="cuda"), torch.ones((1, 1, 128, 8), dtype=BF, device="cuda")
    src = ppd.KVCache(k, v)
    for slots in ([-1, -1, -1], [64, 65, 66], [2 ** 31 - 1] * 3):
        ppd.ppd_paged_store(kv, src, dev([0, 3]), dev([0]), None, dev(slots))
    ppd.ppd_paged_store(kv, src, dev([0, 0]), dev([0]), None, dev([0, 1]))
    assert not kv.pages.any() and not kv.bounds.any()
    ppd.ppd_paged_store(kv, src, dev([0, 30]), dev([10 ** 9]), dev([5]), dev([0, 1, 2, 3]))  # source rows are clamped
    assert kv.pages.float().sum() == 4 * 256


# ---------------------------------------------------------------------------
# attention


class Pool:
    """A pool of pages for sequences of given lengths; what lies behind a length
    is NaN, as are the pages that nobody holds."""

    def __init__(self, lens, nkv, page, layers=1, spare=2, seed=0, scale=1.0):
        r = np.random.default_rng(seed)
        need = [-(-n // page) for n in lens]
        self.n_pages, self.page, self.nkv = sum(need) + spare, page, nkv
        order, at = r.permutation(self.n_pages), 0
        self.table = np.full((len(lens), max(need) + 1), 10 ** 9, np.int32)   # unused entries are never followed
        for s, m in enumerate(need):
            self.table[s, :m] = order[at:at + m]
            at += m
        g = torch.Generator().manual_seed(seed)
        self.pages = torch.full((layers, self.n_pages, nkv, page // 32, 2, 4096), NAN, dtype=BF)
        self.bounds = torch.full((layers, self.n_pages, nkv, 2, 128), NAN, dtype=BF)
        for s, n in enumerate(lens):
            for l in range(layers):
                for h in range(nkv):
                    k, v = (torch.randn((n, 128), generator=g) * scale).to(BF), torch.randn((n, 128), generator=g).to(BF)
                    for j in range(need[s]):
                        p, m = self.table[s, j], min(page, n - j * page)
                        b = self.pages[l, p, h].view(-1)
                        u = np.arange(m)
                        b[torch.from_numpy((u // 32 * 8192)[:, None] + R.KEY[u % 32])] = k[j * page:j * page + m]
                        b[torch.from_numpy((u // 32 * 8192 + 4096)[:, None] + R.VALUE[u % 32])] = v[j * page:j * page + m]
                        x = k[j * page:j * page + m].float()
                        self.bounds[l, p, h, 0], self.bounds[l, p, h, 1] = x.amin(0).to(BF), x.amax(0).to(BF)
        self.lens = np.asarray(lens, np.int32)

    def on_gpu(self, tk, tv, width=0):
        """width: columns of the tables at least (by it a call chooses its kernel)."""
        t = torch.zeros(self.n_pages, dtype=I32, device="cuda")
        table = np.pad(self.table, ((0, 0), (0, max(0, width - self.table.shape[1]))), constant_values=-7)
        pt = ppd.PageTables(dev(table), dev(self.lens), t, t[:2].clone(), self.page)
        return ppd.PagedCache(self.pages.cuda(), self.bounds.cuda(), ppd.KVCache(tk.cuda(), tv.cuda())), pt


def tree_masks(r, T):
    m = np.zeros((sum(T), 2), np.uint64)
    at = 0
    for n in T:
        for i in range(n):
            m[at + i] = m[at + r.integers(0, i)] if i else 0
            m[at + i, i // 64] |= np.uint64(1 << (i % 64))
        at += n
    return m


def new_rows(nkv, cap, rows, layers=1, seed=1):
    g = torch.Generator().manual_seed(seed)
    tk = torch.randn((layers, nkv, cap, 128), generator=g).to(BF)
    tv = torch.randn((layers, nkv, 128, cap), generator=g).to(BF)
    tk[:, :, rows:], tv[..., rows:] = NAN, NAN
    return tk, tv


def attend(kv, pt, row_start, q, mask, layer=0, sel=None, n_sel=None, ws=None, lse=True):
    n, nh, _ = q.shape
    ws = workspace(ppd.ppd_paged_attention_workspace_bytes(nh, kv.n_kv_heads, pt.n_seqs, n)) if ws is None else ws
    out, ls = torch.full_like(q, 7.0), torch.full((n, nh), 7.0, device="cuda") if lse else None
    ppd.ppd_paged_attention(kv, layer, pt, row_start, q, mask, out, ws, ls, sel, n_sel)
    return out, ls, ws


CASES = [  # lens, T, heads, kv heads, page, rows behind the last sequence
    ([0], [1], 2, 2, 32, 0), ([1], [1], 4, 1, 64, 3), ([31, 32, 33], [1, 1, 1], 2, 2, 32, 0), ([200], [1], 16, 16, 32, 0),
    ([95, 0, 500, 64], [3, 0, 17, 1], 4, 2, 64, 5), ([700], [40], 4, 4, 128, 0), ([2000, 1], [1, 1], 8, 1, 32, 1),
    ([1300], [16], 8, 2, 256, 0), ([257], [128], 2, 1, 32, 0), ([40] * 9, [1, 5, 0, 9, 2, 1, 1, 1, 13], 6, 3, 32, 2),
    ([3000], [5], 3, 1, 64, 0), ([77], [100], 16, 2, 32, 0), ([10] * 70, [1] * 70, 2, 1, 32, 0)]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, dtype, wide):
    """wide: tables of 2^19 positions, with which several tiles share a workgroup."""
    lens, T, nh, nkv, page, extra = CASES[case]
    r = np.random.default_rng(case)
    pool = Pool(lens, nkv, page, layers=2, seed=case)
    rows = sum(T) + extra
    tk, tv = new_rows(nkv, (rows + 15) // 8 * 8, sum(T), layers=2)
    kv, pt = pool.on_gpu(tk, tv, (1 << 19) // page if wide else 0)
    g = torch.Generator().manual_seed(case)
    q = torch.randn((rows, nh, 128), generator=g).to(dtype)
    m = np.concatenate((tree_masks(r, T), np.full((extra, 2), 2 ** 64 - 1, np.uint64)))
    if case % 3 == 1:
        m[r.integers(sum(T))] = 0                       # a row that sees the prefix alone (or nothing)
    row_start = offsets(T)
    for mask in (m, None):
        gm = None if mask is None else torch.from_numpy(mask.view(np.int64)).cuda()
        out, lse, ws = attend(kv, pt, dev(row_start), q.cuda(), gm, layer=1)
        assert ppd.ppd_device_status(ws) == 0
        ref = R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 1, row_start, q, mask, page)
        ref.check(out, lse, (torch.full_like(out, 7.0), torch.full_like(lse, 7.0)))
        again = attend(kv, pt, dev(row_start), q.cuda(), gm, layer=1, ws=ws, lse=False)
        assert torch.equal(again[0], out)


@pytest.mark.parametrize("wide", [False, True])
def test_attention_of_a_row_that_sees_nothing_and_of_odd_values(wide):
    """Infinities and NaN in new rows reach the rows that see them and no others;
    queries and keys of large and tiny magnitude."""
    T, nkv, nh = [6, 6], 1, 8
    pool = Pool([0, 70], nkv, 32)
    tk, tv = new_rows(nkv, 16, 12)
    tv[0, 0, 5, 2], tv[0, 0, 6, 3], tk[0, 0, 4, 0] = math.inf, NAN, NAN
    tv[0, 0, 0, 11] = -math.inf
    kv, pt = pool.on_gpu(tk, tv, 1 << 19 if wide else 0)
    m = np.zeros((12, 2), np.uint64)
    for i in range(6):
        m[i, 0] = 1 << i        # itself alone
        m[6 + i, 0] = 1
    m[5] = 0                    # nothing at all
    m[11, 0] = 1 | 1 << 5
    g = torch.Generator().manual_seed(5)
    for scale, dtype in ((1.0, BF), (30.0, torch.float32), (1e-3, BF)):
        q = (torch.randn((12, nh, 128), generator=g) * scale).to(dtype)
        out, lse, _ = attend(kv, pt, dev([0, 6, 12]), q.cuda(), torch.from_numpy(m.view(np.int64)).cuda())
        assert not out[5].any() and bool((lse[5] == -math.inf).all())
        assert bool(torch.isnan(out[2, :, 5]).all()) and bool(torch.isnan(out[3, :, 6]).all()) and bool(torch.isnan(out[4]).all())
        assert bool(torch.isnan(out[11, :, 0]).all())
        keep = torch.ones(out.shape, dtype=torch.bool)
        keep[2, :, 5] = keep[11, :, 0] = False          # (an infinity seen is NaN here, an infinity in 64 bits)
        ref = R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, [0, 6, 12], q, m, 32)
        got = out.cpu().double()
        ref.out[~keep] = got[~keep] = 0.0
        ref.check(got, lse)


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("L", [200, 3000])
def test_attention_at_the_limits_of_magnitude(L, dtype):
    """Values of up to 2^95; then scores of up to 2^125 too, whole multiples of 2^119
    before the scale (exact in float32), so that a row is the mean of its best
    keys' values: those weights are equal and the others zero."""
    T, nkv, nh = 5, 1, 4
    pool = Pool([L], nkv, 64, seed=L)
    tk, tv = new_rows(nkv, 8, T)
    pool.pages[:, :, :, :, 1] = (pool.pages[:, :, :, :, 1] * 2.0 ** 93).clamp(-2.0 ** 95, 2.0 ** 95)
    tv = (tv * 2.0 ** 93).clamp(-2.0 ** 95, 2.0 ** 95)
    q = torch.randn((T, nh, 128), generator=torch.Generator().manual_seed(L)).to(dtype)
    kv, pt = pool.on_gpu(tk, tv)
    out, lse, _ = attend(kv, pt, dev([0, T]), q.cuda(), None)
    assert bool(torch.isfinite(out).all())
    R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, [0, T], q, None, 64).check(out, lse)

    pool.pages[:, :, :, :, 0] = torch.sign(pool.pages[:, :, :, :, 0]) * 2.0 ** 59
    tk, q = torch.sign(tk) * 2.0 ** 59, torch.sign(q) * 2.0 ** 59
    kv, pt = pool.on_gpu(tk, tv)
    out, lse, _ = attend(kv, pt, dev([0, T]), q.cuda(), None)
    k, v = R.rows_of(pool.pages, torch.from_numpy(pool.table), 0, 0, 0, L, 64)
    k, v = torch.cat((k, tk[0, 0, :T])).double(), torch.cat((v, tv[0, 0, :, :T].t())).double()
    half, part = (2.0 ** -8, 2.0 ** -16) if dtype == BF else (2.0 ** -24, 2.0 ** -24)
    for t in range(T):
        y = q[t].double() @ k[:L + t + 1].t()                    # whole multiples of 2^119
        for h in range(nh):
            best = v[:L + t + 1][y[h] == y[h].max()]
            want, mag = best.mean(0), best.abs().mean(0)
            err = (out[t, h].cpu().double() - want).abs()
            assert bool((err <= half * want.abs() + (part + 2 * (L + 64) * 2.0 ** -24) * mag).all())
            top = float(y[h].max()) / math.sqrt(128)
            assert abs(float(lse[t, h]) - top) <= abs(top) * 2.0 ** -21


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("B,nkv,long", [(64, 5, 700), (65, 1, 3000), (100, 3, 2100), (600, 1, 1500)])
def test_attention_of_many_lengths(B, nkv, long, wide):
    """More groups of rows than compute units, or more sequences than a wave's lanes: a
    few long ones that are cut among short and empty ones, in any order."""
    r = np.random.default_rng(B)
    lens = np.where(r.random(B) < 0.2, 0, (30 * np.exp(r.random(B) * 2.5)).astype(int))
    lens[r.integers(0, B, 3)] = [long, long // 2, long - 31]
    T = r.integers(0, 3, B)
    T[[0, B - 1]] = 1
    T[r.integers(B)] = 40
    nh, n = 2 * nkv, int(T.sum())
    pool = Pool(lens.tolist(), nkv, 32, seed=B)
    tk, tv = new_rows(nkv, (n + 15) // 8 * 8, n)
    kv, pt = pool.on_gpu(tk, tv, 1 << 19 if wide else 0)
    q = torch.randn((n, nh, 128), generator=torch.Generator().manual_seed(B)).to(BF)
    row_start = offsets(T.tolist())
    out, lse, ws = attend(kv, pt, dev(row_start), q.cuda(), None)
    assert ppd.ppd_device_status(ws) == 0
    ref = R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, row_start, q, None, 32)
    ref.check(out, lse)
    again = attend(kv, pt, dev(row_start), q.cuda(), None, ws=ws)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("nkv", [1, 2])
def test_attention_and_selection_of_many_sequences(nkv):
    """300 sequences, most without rows or without a prefix, some that share all pages."""
    r = np.random.default_rng(nkv)
    lens = np.where(r.random(300) < 0.4, 0, r.integers(1, 200, 300)).tolist()
    lens[123] = 3000
    T = np.where(r.random(300) < 0.7, 0, r.integers(1, 4, 300))
    T[123], T[7], lens[7] = 2, 1, 150
    for s in range(200, 220):
        lens[s], T[s] = 0, 1
    pool = Pool(lens, nkv, 32, seed=nkv)
    for s in range(200, 220):                           # these read sequence 7's pages
        pool.table[s], pool.lens[s] = pool.table[7], 150 - (s - 200)
    rows = int(T.sum())
    tk, tv = new_rows(nkv, (rows + 15) // 8 * 8, rows)
    kv, pt = pool.on_gpu(tk, tv)
    q = torch.randn((rows, 2 * nkv, 128), generator=torch.Generator().manual_seed(1)).to(BF)
    row_start = offsets(T)
    out, lse, ws = attend(kv, pt, dev(row_start), q.cuda(), None)
    assert ppd.ppd_device_status(ws) == 0
    table = torch.from_numpy(pool.table)
    R.Attention(pool.pages, table, pool.lens, tk, tv, 0, row_start, q, None, 32).check(out, lse)
    sel, n_sel = run_select(pool, kv, pt, row_start, q, 3, 1, 1)
    out, lse, _ = attend(kv, pt, dev(row_start), q.cuda(), None, sel=sel, n_sel=n_sel)
    R.Attention(pool.pages, table, pool.lens, tk, tv, 0, row_start, q, None, 32, sel.cpu(), n_sel.cpu()).check(out, lse)


@pytest.mark.parametrize("page,lens,T,nh,nkv,budget", [(32, [500, 90, 20], [1, 4, 2], 4, 2, 5), (64, [3000], [20], 4, 1, 17),
                                                       (128, [1000, 0], [1, 1], 2, 2, 1)])
def test_attention_over_listed_pages(page, lens, T, nh, nkv, budget):
    r = np.random.default_rng(page)
    pool = Pool(lens, nkv, page)
    rows = sum(T)
    tk, tv = new_rows(nkv, (rows + 15) // 8 * 8, rows)
    kv, pt = pool.on_gpu(tk, tv)
    row_start = offsets(T)
    q = torch.randn((rows, nh, 128), generator=torch.Generator().manual_seed(1)).to(BF)
    sel = np.full((len(lens), nkv, budget), 10 ** 9, np.int32)
    n_sel = np.zeros(len(lens), np.int32)
    for s, n in enumerate(lens):
        m = -(-n // page)
        n_sel[s] = min(budget, m) if s else max(0, min(budget, m) - 1)
        for h in range(nkv):
            pick = r.permutation(m)[: n_sel[s]]
            sel[s, h, : n_sel[s]] = pick if h else np.sort(pick)    # any order
    out, lse, ws = attend(kv, pt, dev(row_start), q.cuda(), None, sel=dev(sel), n_sel=dev(n_sel))
    assert ppd.ppd_device_status(ws) == 0
    R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, row_start, q, None, page, torch.from_numpy(sel),
                n_sel).check(out, lse)


def test_attention_with_bad_numbers_stays_inside():
    pool = Pool([100, 50], 2, 32)
    tk, tv = new_rows(2, 8, 8)
    kv, pt = pool.on_gpu(tk, tv)
    kv.pages.nan_to_num_()
    q = torch.randn((8, 2, 128), device="cuda").to(BF)
    ws = workspace(ppd.ppd_paged_attention_workspace_bytes(2, 2, 2, 8))
    pt.table.copy_(dev(np.array([[-5, 10 ** 9, 3, 2 ** 31 - 1, -1], [0, 1, 2, 3, 4]])))
    for length, rows in (([100, 50], [0, 4, 8]), ([-1, 50], [0, 4, 8]), ([10 ** 9, 50], [0, 4, 8]), ([100, 50], [0, 4, 2000]),
                         ([100, 50], [-9, 4, 8]), ([100, 50], [6, 2, 8])):
        pt.len.copy_(dev(length))
        sel, n_sel = dev(np.full((2, 2, 2), 10 ** 9)), dev([2, 2])
        for s in (None, sel):
            out, _, _ = attend(kv, pt, dev(rows), q, None, sel=s, n_sel=None if s is None else n_sel, ws=ws)
            bad = length != [100, 50] or rows != [0, 4, 8]
            assert bool(ppd.ppd_device_status(ws, clear=True) & ppd.PPD_DEV_BAD_LENGTH) == bad
    n_sel.fill_(9)
    pt.len.copy_(dev([100, 50]))
    attend(kv, pt, dev([0, 4, 8]), q, None, sel=sel, n_sel=n_sel, ws=ws)
    assert ppd.ppd_device_status(ws, clear=True) & ppd.PPD_DEV_BAD_LENGTH


def test_attention_past_32_bits():
    """Pages behind 4 GB of the pool, and a prefix of many splits."""
    nkv, page, n_pages = 1, 256, 40000          # 5.2 GB a layer
    lens = [9000]
    pool = Pool(lens, nkv, page, spare=1)
    big = torch.zeros((1, n_pages, nkv, 8, 2, 4096), dtype=BF, device="cuda")
    at = np.arange(36) * 1100 + 900             # spread over all of it
    far = torch.from_numpy(at)
    big[0, far.cuda()] = pool.pages[0, torch.from_numpy(pool.table[0, :36]).long()].cuda()
    tk, tv = new_rows(nkv, 8, 3)
    t = torch.zeros(n_pages, dtype=I32, device="cuda")
    pt = ppd.PageTables(dev(np.concatenate((at, [0]))[None]), dev(lens), t, t[:2].clone(), page)
    kv = ppd.PagedCache(big, None, ppd.KVCache(tk.cuda(), tv.cuda()))
    q = torch.randn((3, 2, 128), generator=torch.Generator().manual_seed(1))
    out, lse, _ = attend(kv, pt, dev([0, 3]), q.cuda(), None)
    R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, [0, 3], q, None, page).check(out, lse)
    # and a store there
    k, v = torch.randn((1, 1, 8, 128), device="cuda").to(BF), torch.randn((1, 1, 128, 8), device="cuda").to(BF)
    kv = ppd.PagedCache(big, torch.zeros((1, n_pages, 1, 2, 128), dtype=BF, device="cuda"))
    ppd.ppd_paged_store(kv, ppd.KVCache(k, v), dev([0, 2]), dev([0]), None, dev([39990 * 256 + 255, 39991 * 256]))
    flat = big[0, 39990, 0, 7, 0].cpu()
    assert torch.equal(flat[torch.from_numpy(R.KEY[31])], k[0, 0, 0].cpu()) and not big[0, 39991, 0, 1:].any()


# ---------------------------------------------------------------------------
# select


def run_select(pool, kv, pt, row_start, q, budget, first, last):
    B = pt.n_seqs
    ws = workspace(ppd.ppd_paged_select_workspace_bytes(kv.n_kv_heads, B, pt.max_pages))
    sel, n_sel = torch.full((B, kv.n_kv_heads, budget), -8, dtype=I32, device="cuda"), torch.full((B,), -8, dtype=I32, device="cuda")
    ppd.ppd_paged_select(kv, 0, pt, dev(row_start), q.cuda(), budget, first, last, sel, n_sel, ws)
    assert ppd.ppd_device_status(ws) == 0
    want = R.select(kv.bounds.cpu(), torch.from_numpy(pool.table), pool.lens, row_start, q, 0, pool.page, budget, first, last)
    for s, heads in enumerate(want):
        m = min(budget, -(-int(pool.lens[s]) // pool.page))
        assert int(n_sel[s]) == m
        for h, pages in enumerate(heads):
            assert sel[s, h, :m].tolist() == pages, (s, h)
            assert bool((sel[s, h, m:] == -8).all())
    return sel, n_sel


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("page,lens,T,nh,nkv,budget,first,last", [
    (32, [3000, 5, 0, 64], [1, 1, 1, 1], 4, 2, 9, 1, 2), (64, [700], [17], 8, 1, 4, 0, 0), (32, [2100, 2100], [0, 5], 2, 2, 30, 0, 1),
    (128, [4000], [128], 8, 2, 31, 2, 29), (32, [990], [3], 2, 1, 1, 0, 0), (256, [300, 1000], [2, 2], 2, 1, 5, 1, 1)])
def test_select(page, lens, T, nh, nkv, budget, first, last, dtype):
    pool = Pool(lens, nkv, page, seed=7)
    rows = sum(T)
    tk, tv = new_rows(nkv, (rows + 15) // 8 * 8, rows)
    kv, pt = pool.on_gpu(tk, tv)
    q = torch.randn((rows, nh, 128), generator=torch.Generator().manual_seed(2)).to(dtype)
    sel, n_sel = run_select(pool, kv, pt, offsets(T), q, budget, first, last)
    out, lse, _ = attend(kv, pt, dev(offsets(T)), q.cuda(), None, sel=sel, n_sel=n_sel)
    R.Attention(pool.pages, torch.from_numpy(pool.table), pool.lens, tk, tv, 0, offsets(T), q, None, page, sel.cpu(),
                n_sel.cpu()).check(out, lse)


@pytest.mark.parametrize("m,budget", [(1, 1), (2, 1), (63, 62), (64, 5), (1024, 1000), (1500, 37), (8192, 4096), (8193, 8192),
                                      (20000, 3), (20000, 19999)])
def test_select_by_crafted_bounds(m, budget):
    """Ties (the smaller page), runs of equal scores across the threshold, NaN and
    infinities, zeros of both signs."""
    r = np.random.default_rng(m)
    nkv, page = 2, 32
    pool = Pool([1], nkv, page)
    pool.table = np.arange(m, dtype=np.int32)[None]
    pool.lens = np.array([m * page - 5], np.int32)
    values = np.array([0.0, -0.0, 1.0, 1.0, 2.0, -3.0, 1e30, -1e30, np.inf, -np.inf, np.nan, 0.5])
    for kind in range(3):
        b = torch.zeros((1, m, nkv, 2, 128))
        x = torch.from_numpy(values[r.integers(0, (4, 8, 12)[kind], (m, nkv))])
        b[0, :, :, 1, 3] = x
        if kind == 1:
            b[0, :, :, 0, 4] = torch.from_numpy(r.normal(size=(m, nkv))).float()
        kv = ppd.PagedCache(torch.zeros((1, m, nkv, 1, 2, 4096), dtype=BF, device="cuda"), b.to(BF).cuda())
        t = torch.zeros(m, dtype=I32, device="cuda")
        pt = ppd.PageTables(dev(pool.table), dev(pool.lens), t, torch.zeros(2, dtype=I32, device="cuda"), page)
        q = torch.zeros((1, nkv, 128))
        q[0, :, 3], q[0, :, 4] = 1.5, -0.25
        run_select(pool, kv, pt, [0, 1], q, budget, 0, min(1, budget - 1))


# ---------------------------------------------------------------------------
# streams and graphs


def test_calls_on_another_stream():
    pool = Pool([900, 40], 2, 64)
    tk, tv = new_rows(2, 8, 5)
    kv, pt = pool.on_gpu(tk, tv)
    q = torch.randn((5, 4, 128), device="cuda").to(BF)
    rows = dev([0, 3, 5])
    want = attend(kv, pt, rows, q, None)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = workspace(ppd.ppd_paged_attention_workspace_bytes(4, 2, 2, 5))
    torch.cuda.synchronize()
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    ppd.ppd_paged_attention(kv, 0, pt, rows, q, None, out, ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    with torch.cuda.stream(side):
        assert torch.equal(attend(kv, pt, rows, q, None)[0], want)
    side.synchronize()


def test_two_streams_at_once():
    """Chains of selection and attention of two batches side by side, each stream with
    a workspace that its calls share, beside the same calls one after another."""
    nh, nkv, T, budget = 8, 2, 3, 9
    runs = []
    for i, lens in enumerate(([5000, 40, 0], [777, 3000, 1200])):
        pool = Pool(lens, nkv, 64, seed=i)
        tk, tv = new_rows(nkv, 16, 3 * T, seed=i)
        kv, pt = pool.on_gpu(tk, tv)
        q = torch.randn((3 * T, nh, 128), generator=torch.Generator().manual_seed(i)).to(BF).cuda()
        width = pt.table.shape[1]
        need = max(ppd.ppd_paged_attention_workspace_bytes(nh, nkv, 3, 3 * T), ppd.ppd_paged_select_workspace_bytes(nkv, 3, width))
        sel = torch.zeros((3, nkv, budget), dtype=I32, device="cuda")
        runs.append(dict(kv=kv, pt=pt, q=q, rows=dev(offsets([T] * 3)), ws=workspace(need), sel=sel, n=torch.zeros(3, dtype=I32, device="cuda"),
                         out=[torch.zeros_like(q) for _ in range(2)], stream=torch.cuda.Stream()))

    def chain(r, stream):
        ppd.ppd_paged_select(r["kv"], 0, r["pt"], r["rows"], r["q"], budget, 1, 2, r["sel"], r["n"], r["ws"], stream=stream)
        ppd.ppd_paged_attention(r["kv"], 0, r["pt"], r["rows"], r["q"], None, r["out"][0], r["ws"], None, r["sel"], r["n"], stream=stream)
        ppd.ppd_paged_attention(r["kv"], 0, r["pt"], r["rows"], r["q"], None, r["out"][1], r["ws"], stream=stream)

    torch.cuda.synchronize()
    want = []
    for r in runs:
        chain(r, None)
        torch.cuda.synchronize()
        want.append([x.clone() for x in (*r["out"], r["sel"], r["n"])])
    for _ in range(20):
        for r in runs:
            for x in r["out"]:
                x.zero_()
        torch.cuda.synchronize()
        for r in runs:
            chain(r, r["stream"])
        torch.cuda.synchronize()
        for r, w in zip(runs, want):
            assert all(torch.equal(a, b) for a, b in zip((*r["out"], r["sel"], r["n"]), w))
            assert ppd.ppd_device_status(r["ws"]) == 0


def test_a_captured_chain_follows_the_lengths():
    """Select, attention, tables and store captured once and replayed while the
    sequences grow, end and start again, beside eager calls; two graphs share the
    workspaces."""
    B, nkv, nh, page, n_pages, T = 3, 2, 4, 32, 60, 4
    kv = ppd.PagedCache.empty(1, nkv, n_pages, page, 16)
    kv.pages.fill_(NAN), kv.bounds.fill_(NAN)
    pt = ppd.PageTables.empty(B, 20, n_pages, page)
    row_start, add = dev(offsets([T] * B)), dev([1] * B)
    path = dev([0, 1, 2, 3] * B)
    start, slots = torch.zeros(B + 1, dtype=I32, device="cuda"), torch.zeros(B * 40, dtype=I32, device="cuda")
    q, out = torch.zeros((B * T, nh, 128), dtype=BF, device="cuda"), torch.zeros((B * T, nh, 128), dtype=BF, device="cuda")
    sel, n_sel = torch.zeros((B, nkv, 3), dtype=I32, device="cuda"), torch.zeros(B, dtype=I32, device="cuda")
    ws = workspace(ppd.ppd_paged_attention_workspace_bytes(nh, nkv, B, B * T))
    wt, wl = workspace(ppd.ppd_paged_tables_workspace_bytes(B)), workspace(ppd.ppd_paged_select_workspace_bytes(nkv, B, 20))

    def chain(sparse):
        if sparse:
            ppd.ppd_paged_select(kv, 0, pt, row_start, q, 3, 1, 1, sel, n_sel, wl)
        ppd.ppd_paged_attention(kv, 0, pt, row_start, q, None, out, ws, None, *((sel, n_sel) if sparse else ()))
        ppd.ppd_paged_tables(pt, add, start, slots, wt)
        ppd.ppd_paged_store(kv, kv.tail, start, row_start, path, slots)

    graphs = []
    kv.tail.k.zero_(), kv.tail.v.zero_()
    for sparse in (False, True):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            chain(sparse)
        graphs.append(graph)
    r = np.random.default_rng(0)
    keep = ("pages", "bounds")
    for step in range(40):
        sparse = step % 3 == 2
        torch.cuda.synchronize()
        kv.tail.k.copy_(torch.randn(kv.tail.k.shape, device="cuda"))
        kv.tail.v.copy_(torch.randn(kv.tail.v.shape, device="cuda"))
        q.copy_(torch.randn(q.shape, device="cuda"))
        a = r.integers(0, T + 1, B)
        if step % 13 == 12:
            a[r.integers(B)] = -1
        add.copy_(dev(a))
        state = [t.clone() for t in (kv.pages, kv.bounds, pt.table, pt.len, pt.free_pages, pt.free_state)]
        torch.cuda.synchronize()
        chain(sparse)
        torch.cuda.synchronize()
        eager = [t.clone() for t in (kv.pages, kv.bounds, pt.table, pt.len, pt.free_pages, pt.free_state, out, start)]
        for t, x in zip((kv.pages, kv.bounds, pt.table, pt.len, pt.free_pages, pt.free_state), state):
            t.copy_(x)
        out.zero_()
        torch.cuda.synchronize()
        graphs[sparse].replay()
        torch.cuda.synchronize()
        for t, x in zip((kv.pages, kv.bounds, pt.table, pt.len, pt.free_pages, pt.free_state, out, start), eager):
            assert torch.equal(t.view(torch.uint8), x.view(torch.uint8)), step
        assert not torch.isnan(out).any()
    assert int(pt.len.max()) > 64 and ppd.ppd_device_status(ws) == ppd.ppd_device_status(wt) == ppd.ppd_device_status(wl) == 0
