"""The paged cache without a GPU: refusals of the C ABI and of the binding, sizes,
and the reference forms against their definitions."""
import ctypes as C
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2405_18628_amd as ppd
from test_kernel_resources_cpu import _kernels

F = 0x10000  # a pointer that is never followed
L = ppd.lib()
BIG = 1 << 40


def _cache(pages=F, bounds=F, layers=2, heads=4, n=16, page=64, tail=(F, F, 128)):
    return ppd.ppd_paged(pages, bounds, layers, heads, n, page, ppd.ppd_kv(tail[0], tail[1], tail[2], None))


def _tables(table=F, length=F, ring=F, state=F, seqs=3, width=8, n=16, page=64):
    return ppd.ppd_page_tables(table, length, ring, state, seqs, width, n, page)


def test_sizes():
    assert ppd.ppd_paged_bytes(2, 4, 16, 64) == 2 * 4 * 16 * 64 * 512
    assert ppd.ppd_paged_bounds_bytes(2, 4, 16) == 2 * 4 * 16 * 512
    assert ppd.ppd_paged_bytes(32, 32, 1 << 17, 32) == 32 * 32 * (1 << 17) * 32 * 512
    for bad in ((0, 4, 16, 64), (2, 0, 16, 64), (2, 4, 0, 64), (2, 4, 16, 16), (2, 4, 16, 48), (2, 4, 16, 512),
                (2, 4, 1 << 26, 32), (1 << 13, 1 << 13, 1, 32)):
        assert L.ppd_paged_bytes(*bad) == 0 and ppd.ppd_last_error()
    small, big = (ppd.ppd_paged_attention_workspace_bytes(32, 8, 1, n) for n in (1, 128))
    assert 0 < small < big
    for bad in ((0, 1, 1, 1), (4, 3, 1, 1), (4, 4, 0, 1), (4, 4, 4097, 1), (4, 4, 1, 0), (1024, 8, 1, 4097)):
        assert L.ppd_paged_attention_workspace_bytes(*bad) == 0 and ppd.ppd_last_error()
    assert 0 < ppd.ppd_paged_tables_workspace_bytes(1) <= ppd.ppd_paged_tables_workspace_bytes(4096)
    for bad in (0, -1, 4097):
        assert L.ppd_paged_tables_workspace_bytes(bad) == 0
    assert ppd.ppd_paged_select_workspace_bytes(8, 4, 100) >= 8 * 4 * 100 * 8
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 4097, 1), (1, 1, (1 << 19) + 1), (8192, 4096, 1), (64, 64, 1 << 18)):
        assert L.ppd_paged_select_workspace_bytes(*bad) == 0


def test_layout_holds_every_element_once():
    assert sorted(R.KEY.reshape(-1)) == list(range(4096)) == sorted(R.VALUE.reshape(-1))


BAD_TABLES = [(dict(table=None), ppd.PPD_EINVAL), (dict(length=None), ppd.PPD_EINVAL), (dict(seqs=0), ppd.PPD_EINVAL),
              (dict(seqs=4097), ppd.PPD_EINVAL), (dict(width=0), ppd.PPD_EINVAL), (dict(n=0), ppd.PPD_EINVAL),
              (dict(page=40), ppd.PPD_EUNSUPPORTED), (dict(width=(1 << 18) + 1), ppd.PPD_EUNSUPPORTED)]
BAD_CACHES = [(dict(pages=None), ppd.PPD_EINVAL), (dict(pages=F + 8), ppd.PPD_EINVAL), (dict(bounds=F + 4), ppd.PPD_EINVAL),
              (dict(layers=0), ppd.PPD_EINVAL), (dict(heads=0), ppd.PPD_EINVAL), (dict(n=0), ppd.PPD_EINVAL),
              (dict(page=100), ppd.PPD_EUNSUPPORTED), (dict(n=1 << 26), ppd.PPD_EUNSUPPORTED)]
BAD_TAILS = [((None, F, 64), ppd.PPD_EINVAL), ((F, F + 2, 64), ppd.PPD_EINVAL), ((F, F, 0), ppd.PPD_EINVAL),
             ((F, F, 60), ppd.PPD_EUNSUPPORTED), ((F, F, (1 << 24) + 8), ppd.PPD_EUNSUPPORTED)]


def test_tables_refuse():
    def call(pt=None, add=F, len_out=F, state=F, start=F, slots=F, n=8, ws=F, size=BIG):
        return L.ppd_paged_tables(C.byref(pt or _tables()), add, len_out, state, start, slots, n, ws, size, None)
    for kw, code in BAD_TABLES + [(dict(ring=None), ppd.PPD_EINVAL), (dict(state=None), ppd.PPD_EINVAL)]:
        assert call(_tables(**kw)) == code, kw
    for kw in (dict(add=None), dict(len_out=None), dict(state=None), dict(start=None), dict(slots=None), dict(n=0),
               dict(n=-1), dict(ws=F + 4)):
        assert call(**kw) == ppd.PPD_EINVAL, kw
    assert call(ws=None) == call(size=ppd.ppd_paged_tables_workspace_bytes(3) - 1) == ppd.PPD_EWORKSPACE


def test_store_refuses():
    def call(kv=None, src=(F, F, 64), seqs=2, start=F, row_start=F, path=None, n_path=0, slots=F, n=4):
        return L.ppd_paged_store(C.byref(kv or _cache()), C.byref(ppd.ppd_kv(*src, None)), seqs, start, row_start, path, n_path,
                                 slots, n, None)
    for kw, code in BAD_CACHES:
        assert call(_cache(**kw)) == code, kw
    for src, code in BAD_TAILS:
        assert call(src=src) == code, src
    for kw in (dict(seqs=0), dict(seqs=4097), dict(start=None), dict(row_start=None), dict(slots=None), dict(n=0),
               dict(path=F, n_path=0)):
        assert call(**kw) == ppd.PPD_EINVAL, kw


def _attend(nh=8, kv=None, layer=0, pt=None, row_start=F, n=4, q=F, dt=ppd.PPD_BF16, mask=None, out=2 * F, sel=None, n_sel=None,
            budget=0, ws=F, size=BIG):
    return L.ppd_paged_attention(nh, C.byref(kv or _cache()), layer, C.byref(pt or _tables()), row_start, n, q, dt, mask, out, None,
                                 sel, n_sel, budget, ws, size, None)


def _select(nh=8, kv=None, layer=0, pt=None, row_start=F, n=4, q=F, dt=ppd.PPD_F32, budget=4, first=1, last=1, sel=F, n_sel=F,
            ws=F, size=BIG):
    return L.ppd_paged_select(nh, C.byref(kv or _cache()), layer, C.byref(pt or _tables()), row_start, n, q, dt, budget, first, last,
                              sel, n_sel, ws, size, None)


def test_attention_and_select_refuse():
    for f in (_attend, _select):
        for kw, code in BAD_CACHES:
            assert f(kv=_cache(**kw)) == code, kw
        for kw, code in BAD_TABLES:
            assert f(pt=_tables(**kw)) == code, kw
        for kw in (dict(nh=6), dict(nh=0), dict(layer=-1), dict(layer=2), dict(row_start=None), dict(n=0), dict(n=1 << 20),
                   dict(q=None), dict(q=F + 8), dict(dt=2), dict(ws=F + 8)):
            assert f(**kw) == ppd.PPD_EINVAL, kw
        # tables of another pool than the cache's
        assert f(pt=_tables(n=17)) == f(pt=_tables(page=32)) == ppd.PPD_EINVAL
        assert f(ws=None) == f(size=256) == ppd.PPD_EWORKSPACE
    for tail, code in BAD_TAILS:
        assert _attend(kv=_cache(tail=tail)) == code, tail
    assert _attend(n=129) == ppd.PPD_ECAPACITY
    # (four rows of eight heads are 8192 bytes, in float32 16384)
    for kw in (dict(out=None), dict(out=2 * F + 4), dict(out=F), dict(out=F + 8176), dict(out=F - 8176),
               dict(out=F + 8192, dt=ppd.PPD_F32), dict(sel=F), dict(n_sel=F), dict(sel=F, n_sel=F, budget=0)):
        assert _attend(**kw) == ppd.PPD_EINVAL, kw
    assert _select(kv=_cache(bounds=None)) == ppd.PPD_EINVAL
    for kw in (dict(budget=0), dict(first=-1), dict(last=-1), dict(first=3, last=2), dict(sel=None), dict(n_sel=None)):
        assert _select(**kw) == ppd.PPD_EINVAL, kw


def test_step_refuses():
    def model(**kw):
        d = dict(n_layers=2, hidden=256, n_heads=8, n_kv_heads=4, head_dim=128, ffn=512, vocab=100, n_prompt=3, rms_eps=1e-6,
                 rope_base=1e4, dtype=ppd.PPD_BF16)
        d.update(kw)
        ptr = (C.c_void_p * 2)(F, F)
        arr = C.cast(ptr, C.POINTER(C.c_void_p))
        m = ppd.ppd_model(tok_emb=F, prompt_emb=F, attn_norm=arr, w_qkv=arr, w_o=arr, mlp_norm=arr, w_gate_up=arr, w_down=arr,
                          final_norm=F, lm_head=F, **d)
        m._keep = ptr
        return m

    def call(m=None, kv=None, pt=None, row_start=F, n=4, ids=F, mask=F, pred=F, budget=0, first=0, last=0, ws=F, size=BIG):
        return L.ppd_verify_batch_paged(C.byref(m or model()), C.byref(kv or _cache()), C.byref(pt or _tables()), row_start, n, ids, F,
                                        mask, budget, first, last, ws, size, None, pred, None)
    for kw, code in BAD_CACHES:
        assert call(kv=_cache(**kw)) == code, kw
    for kw, code in BAD_TABLES:
        assert call(pt=_tables(**kw)) == code, kw
    for tail, code in BAD_TAILS:
        assert call(kv=_cache(tail=tail)) == code, tail
    assert call(model(dtype=ppd.PPD_F32)) == ppd.PPD_EUNSUPPORTED
    assert call(kv=_cache(layers=3)) == call(kv=_cache(heads=8)) == ppd.PPD_EINVAL
    for kw in (dict(n=0), dict(n=129), dict(row_start=None), dict(ids=None), dict(mask=None), dict(pred=None), dict(budget=-1),
               dict(budget=2, first=2, last=1), dict(budget=2, kv=_cache(bounds=None))):
        assert call(**kw) == ppd.PPD_EINVAL, kw
    assert call(n=72, kv=_cache(tail=(F, F, 64))) == ppd.PPD_ECAPACITY
    assert call(ws=None) == call(size=1000) == ppd.PPD_EWORKSPACE
    m = model()
    sizes = [L.ppd_paged_workspace_bytes(C.byref(m), 3, 8, 4, b) for b in (0, 4)]
    assert 0 < sizes[0] < sizes[1]
    for bad in ((0, 8, 4, 0), (3, 0, 4, 0), (3, 8, 0, 0), (3, 8, 129, 0), (3, 8, 4, -1)):
        assert L.ppd_paged_workspace_bytes(C.byref(m), *bad) == 0


def test_binding_refuses():
    bf = torch.bfloat16
    pages, bounds = torch.zeros((2, 3, 4, 2, 2, 4096), dtype=bf), torch.zeros((2, 3, 4, 2, 128), dtype=bf)
    kv = ppd.PagedCache(pages, bounds)
    assert (kv.n_layers, kv.n_pages, kv.n_kv_heads, kv.page) == (2, 3, 4, 64)
    for bad in (pages.float(), pages[:, :, :, :, :1], pages.transpose(1, 2), pages[0]):
        with pytest.raises(ValueError):
            ppd.PagedCache(bad, bounds)
    for bad in (bounds[:1], bounds.float(), bounds.transpose(1, 2)):
        with pytest.raises(ValueError):
            ppd.PagedCache(pages, bad)
    with pytest.raises(ValueError):
        ppd.PagedCache(pages, bounds, ppd.KVCache(torch.zeros((2, 3, 8, 128), dtype=bf), torch.zeros((2, 3, 128, 8), dtype=bf)))
    with pytest.raises(ValueError):
        ppd.PagedCache.empty(1, 1, 1, 48, device="cpu")
    pt = ppd.PageTables.empty(3, 5, 7, 64, device="cpu")
    assert (pt.n_seqs, pt.max_pages, pt.n_pages, pt.page) == (3, 5, 7, 64)
    assert pt.free_pages.tolist() == list(range(7)) and pt.free_state.tolist() == [0, 7]
    for i, bad in ((0, pt.table[:, 1:]), (0, pt.table.long()), (1, pt.len[:2]), (2, pt.table), (3, pt.len)):
        args = [pt.table, pt.len, pt.free_pages, pt.free_state]
        args[i] = bad
        with pytest.raises(ValueError):
            ppd.PageTables(*args, 64)
    # a call's tensors have to be on the device
    i32 = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        ppd.ppd_paged_tables(pt, i32[:3], i32, i32, i32)
    with pytest.raises(ValueError):
        ppd.ppd_paged_select(kv, 0, pt, i32, torch.zeros((4, 8, 128)), 2, 0, 0, i32, i32, i32)


@pytest.mark.parametrize("seed", range(5))
def test_reference_tables_keep_every_page_in_one_place(seed):
    r = np.random.default_rng(seed)
    B, page, n_pages, width = 6, 32, 40, 12
    table, length = np.zeros((B, width), np.int32), np.zeros(B, np.int32)
    ring, state = r.permutation(n_pages).astype(np.int32), np.array([0, n_pages], np.int32)
    refusals = 0
    for _ in range(60):
        add = np.where(r.random(B) < 0.15, -1, r.integers(0, 90, B)).astype(np.int32)
        n = int(np.maximum(add, 0).sum()) + 3
        table, length, ring, state, start, slots, refused = R.tables(table, length, add, ring, state, page, n, np.full(n, -9, np.int32))
        refusals += refused
        held = [p for s in range(B) for p in table[s, :-(-int(length[s]) // page)]]
        free = [ring[(state[0] + i) % n_pages] for i in range(state[1])]
        assert sorted(held + free) == list(range(n_pages))
        assert (slots[start[B]:] == -9).all()
    assert refusals


def test_a_pages_score_bounds_its_keys():
    g = torch.Generator().manual_seed(3)
    k, q = torch.randn((64, 128), generator=g).double(), torch.randn((5, 128), generator=g).double()
    lo, hi = k.amin(0), k.amax(0)
    up = q.clamp(min=0).sum(0) @ hi + q.clamp(max=0).sum(0) @ lo
    assert bool(((q @ k.t()).sum(0) <= up).all())


class On:
    """A contiguous device tensor of device d, as far as the checks look."""
    is_cuda = True

    def __init__(self, d, dtype=torch.int32):
        self.d, self.dtype = d, dtype

    def get_device(self):
        return self.d

    def is_contiguous(self):
        return True

    def numel(self):
        return 4


def test_calls_refuse_another_device(monkeypatch):
    """Tensors, tables or caches of device 1 with device 0 current, and the other way round."""
    monkeypatch.setattr(ppd, "_torch", SimpleNamespace(
        _C=SimpleNamespace(_cuda_getDevice=lambda: 0), bfloat16=torch.bfloat16, float32=torch.float32, int32=torch.int32))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    bf = torch.bfloat16
    kv = ppd.PagedCache(torch.zeros((1, 3, 4, 2, 2, 4096), dtype=bf), torch.zeros((1, 3, 4, 2, 128), dtype=bf))
    pt = ppd.PageTables.empty(3, 5, 3, 64, device="cpu")
    kv.pages, pt.table = On(0, bf), On(0)
    for cache, table, tensor in ((1, 1, 1), (0, 1, 0), (1, 0, 0), (0, 0, 1)):
        kv.device, pt.device, kv.pages.d, pt.table.d = cache, table, cache, table
        t, f = On(tensor), On(tensor, torch.float32)
        f.shape = (4, 8, 128)
        with pytest.raises(ValueError):
            ppd.ppd_paged_select(kv, 0, pt, t, f, 2, 0, 0, t, t, t)
        with pytest.raises(ValueError):
            ppd.ppd_paged_attention(kv, 0, pt, t, f, None, f, t)
        if (cache, table, tensor) != (1, 0, 0):
            with pytest.raises(ValueError):
                ppd.ppd_paged_tables(pt, t, t, t, t, t, t)


def test_kernels_use_no_scratch_memory():
    mine = [k for k in _kernels() if "paged_" in k[".name"]]
    for part in ("paged_tables_kernel", "paged_put_kernel", "paged_fill_rows_kernel", "paged_attention_kernel", "paged_merge_kernel",
                 "paged_score_kernel", "paged_pick_kernel"):
        assert any(part in k[".name"] for k in mine), part
    assert not [k[".name"] for k in mine if k[".private_segment_fixed_size"]]
