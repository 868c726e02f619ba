"""The 4-bit cache and sampled acceptance without a GPU: refusals on the host,
the reference implementations against their definitions, and that sampled
acceptance emits the target's distribution."""
import ctypes as C
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import kvq_reference as R
import paper_2405_18628_amd as ppd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F = 0x10000  # a pointer that is never followed
OK_TAIL = dict(k=F, v=F, capacity=128)


def _kvq(blocks=F, layers=2, heads=4, cap=256, tail=None):
    t = OK_TAIL if tail is None else tail
    return ppd.ppd_kvq(blocks, layers, heads, cap, ppd.ppd_kv(t.get("k"), t.get("v"), t.get("capacity", 0), None))


def _i32(*v):
    return np.asarray(v, np.int32)


def test_sizes():
    assert ppd.ppd_kvq_bytes(2, 4, 256) == 2 * 4 * 8 * 4608
    assert ppd.ppd_kvq_bytes(32, 32, 1 << 24) == 32 * 32 * (1 << 19) * 4608
    L = ppd.lib()
    for bad in ((0, 4, 256), (2, 0, 256), (2, 4, 0), (2, 4, 255), (2, 4, (1 << 24) + 32), (1 << 13, 1 << 13, 32), (1 << 20, 2, 32)):
        assert L.ppd_kvq_bytes(*bad) == 0 and ppd.ppd_last_error()
    small, big = (ppd.ppd_kvq_attention_workspace_bytes(32, 8, t) for t in (1, 128))
    assert 0 < small < big
    for bad in ((0, 1, 1), (4, 3, 1), (4, 4, 0), (4, 4, 129), (4, 0, 4), (1 << 17, 1, 4)):
        assert L.ppd_kvq_attention_workspace_bytes(*bad) == 0 and ppd.ppd_last_error()
    assert ppd.ppd_accept_sample_workspace_bytes(64, 32000) > 0
    for bad in ((0, 10), (129, 10), (4, 0), (4, (1 << 30) + 1)):
        assert L.ppd_accept_sample_workspace_bytes(*bad) == 0 and ppd.ppd_last_error()


BAD_CACHES = [(dict(blocks=None), ppd.PPD_EINVAL), (dict(blocks=F + 4), ppd.PPD_EINVAL),
              (dict(layers=0), ppd.PPD_EINVAL), (dict(heads=-1), ppd.PPD_EINVAL),
              (dict(cap=250), ppd.PPD_EUNSUPPORTED), (dict(cap=(1 << 24) + 32), ppd.PPD_EUNSUPPORTED)]
BAD_ROWS = [(dict(k=None, v=F, capacity=64), ppd.PPD_EINVAL), (dict(k=F, v=F + 2, capacity=64), ppd.PPD_EINVAL),
            (dict(k=F, v=F, capacity=0), ppd.PPD_EINVAL), (dict(k=F, v=F, capacity=60), ppd.PPD_EUNSUPPORTED)]


def test_quantize_and_dequantize_refuse():
    L = ppd.lib()
    src = ppd.ppd_kv(F, F, 512, None)
    for f in (L.ppd_kvq_quantize, L.ppd_kvq_dequantize):
        for kw, code in BAD_CACHES:
            assert f(C.byref(_kvq(**kw)), 0, C.byref(src), 0, 4, None) == code, kw
        for kw, code in BAD_ROWS:
            bad = ppd.ppd_kv(kw["k"], kw["v"], kw["capacity"], None)
            assert f(C.byref(_kvq()), 0, C.byref(bad), 0, 4, None) == code, kw
        assert f(None, 0, C.byref(src), 0, 4, None) == ppd.PPD_EINVAL
        assert f(C.byref(_kvq()), 0, None, 0, 4, None) == ppd.PPD_EINVAL
        for a, b, n, code in ((-1, 0, 4, ppd.PPD_EINVAL), (0, -1, 4, ppd.PPD_EINVAL), (0, 0, -1, ppd.PPD_EINVAL),
                              (0, 0, 257, ppd.PPD_ECAPACITY), (253, 0, 4, ppd.PPD_ECAPACITY),
                              (0, 509, 4, ppd.PPD_ECAPACITY), (2147483647, 0, 2147483647, ppd.PPD_ECAPACITY)):
            assert f(C.byref(_kvq()), a, C.byref(src), b, n, None) == code, (a, b, n)
        assert f(C.byref(_kvq(tail={})), 256, C.byref(src), 512, 0, None) == ppd.PPD_OK  # nothing to do


def test_commit_refuses():
    L = ppd.lib()

    def call(kv, Lc=10, path=F, n=4, cnt=F):
        return L.ppd_kvq_commit(C.byref(kv), Lc, path, n, cnt, None)
    for kw, code in BAD_CACHES:
        assert call(_kvq(**kw)) == code, kw
    for kw, code in BAD_ROWS:
        assert call(_kvq(tail=kw)) == code, kw
    assert call(_kvq(tail={})) == ppd.PPD_EINVAL
    assert call(_kvq(), Lc=-1) == ppd.PPD_ECAPACITY and call(_kvq(), Lc=256) == ppd.PPD_ECAPACITY
    assert call(_kvq(), path=None) == ppd.PPD_EINVAL and call(_kvq(), cnt=None) == ppd.PPD_EINVAL
    assert call(_kvq(), n=0) == ppd.PPD_EINVAL and call(_kvq(), n=129) == ppd.PPD_EINVAL


def test_attention_refuses():
    L = ppd.lib()
    need = ppd.ppd_kvq_attention_workspace_bytes(8, 4, 20)

    def call(kvs, Ls=(5, 6), Ts=(10, 10), B=None, nh=8, layer=0, q=F, mask=F, out=F, ws=F, n=need):
        arr = (ppd.ppd_kvq * len(kvs))(*kvs)
        a, b = _i32(*Ls), _i32(*Ts)
        return L.ppd_kvq_attention(nh, len(kvs) if B is None else B, C.cast(arr, C.c_void_p), layer, a.ctypes.data,
                                   b.ctypes.data, q, mask, out, None, ws, n, None)
    two = [_kvq(), _kvq()]
    for kw, code in BAD_CACHES:
        assert call([_kvq(), _kvq(**kw)]) == code, kw
    for kw, code in BAD_ROWS:
        assert call([_kvq(), _kvq(tail=kw)]) == code, kw
    assert call(two, B=0) == ppd.PPD_EINVAL and call([_kvq()] * 17, (0,) * 17, (1,) * 17) == ppd.PPD_EINVAL
    assert call(two, Ts=(10, 0)) == ppd.PPD_EINVAL and call(two, Ls=(5, -1)) == ppd.PPD_EINVAL
    assert call(two, Ls=(5, 257)) == ppd.PPD_ECAPACITY
    assert call([_kvq(), _kvq(tail=dict(k=F, v=F, capacity=8))]) == ppd.PPD_ECAPACITY
    assert call(two, Ts=(65, 64)) == ppd.PPD_EINVAL
    assert call(two, nh=0) == ppd.PPD_EINVAL and call(two, nh=6) == ppd.PPD_EINVAL
    assert call([_kvq(), _kvq(heads=2)]) == ppd.PPD_EINVAL
    assert call(two, layer=2) == ppd.PPD_EINVAL and call(two, layer=-1) == ppd.PPD_EINVAL
    for null in ("q", "mask", "out"):
        assert call(two, **{null: None}) == ppd.PPD_EINVAL
    assert call(two, q=F + 2) == ppd.PPD_EINVAL and call(two, out=F + 8) == ppd.PPD_EINVAL
    assert call(two, ws=None) == ppd.PPD_EWORKSPACE and call(two, n=need - 1) == ppd.PPD_EWORKSPACE
    assert call(two, ws=F + 4) == ppd.PPD_EINVAL


def _fake_model(dtype=ppd.PPD_BF16, **kw):
    n = kw.get("n_layers", 2)
    arr = (C.c_void_p * n)(*([F] * n))
    f = C.c_void_p(F)
    return ppd.ppd_model(n, kw.get("hidden", 512), kw.get("n_heads", 4), kw.get("n_kv_heads", 4),
                         kw.get("head_dim", 128), kw.get("ffn", 1344), 1000, 3, 1e-6, 10000.0, dtype, f, f,
                         *[C.cast(arr, C.POINTER(C.c_void_p)) for _ in range(6)], f, f), arr


def test_verify_refuses():
    L = ppd.lib()
    m, keep = _fake_model()
    need = L.ppd_kvq_workspace_bytes(C.byref(m), 16)
    assert need > L.ppd_workspace_bytes(C.byref(m), 16, 256)
    assert L.ppd_kvq_workspace_bytes(C.byref(m), 129) == 0
    mf, kf = _fake_model(ppd.PPD_F32, head_dim=64, hidden=256, ffn=688)
    assert L.ppd_kvq_workspace_bytes(C.byref(mf), 16) == 0

    def call(kv=None, model=m, Lc=3, pos=3, T=16, ids=F, ws=F, n=need, q=None):
        kv = _kvq() if kv is None else kv
        return L.ppd_verify_step_kvq(C.byref(model), C.byref(kv), Lc, pos, T, ids, F, F, ws, n, None, F, q, None, None)
    for kw, code in BAD_CACHES:
        assert call(_kvq(**kw)) == code, kw
    for kw, code in BAD_ROWS:
        assert call(_kvq(tail=kw)) == code, kw
    assert call(model=mf) == ppd.PPD_EUNSUPPORTED
    assert call(_kvq(layers=3)) == ppd.PPD_EINVAL and call(_kvq(heads=2)) == ppd.PPD_EINVAL
    assert call(T=0) == ppd.PPD_EINVAL and call(T=129) != ppd.PPD_OK
    assert call(Lc=-1) == ppd.PPD_EINVAL and call(Lc=257) == ppd.PPD_ECAPACITY and call(pos=-1) == ppd.PPD_EINVAL
    assert call(_kvq(tail=dict(k=F, v=F, capacity=8))) == ppd.PPD_ECAPACITY
    assert call(ids=None) == ppd.PPD_EINVAL and call(q=F + 4) == ppd.PPD_EINVAL
    assert call(ws=None) == ppd.PPD_EWORKSPACE and call(n=need - 1) == ppd.PPD_EWORKSPACE


def test_batch_refuses_a_shared_tail():
    """Two sequences' trees in one staging cache would overwrite each other."""
    L = ppd.lib()
    m, keep = _fake_model()
    far = dict(k=F + (1 << 20), v=F + (2 << 20), capacity=128)
    need = L.ppd_kvq_workspace_bytes(C.byref(m), 32)

    def call(second, n=need):
        arr = (ppd.ppd_kvq * 2)(_kvq(), _kvq(tail=second))
        v = _i32(16, 16)
        return L.ppd_verify_batch_kvq(C.byref(m), 2, C.cast(arr, C.c_void_p), v.ctypes.data, v.ctypes.data, v.ctypes.data, F,
                                      F, F, F, n, None, F, None, None, None)
    assert call(OK_TAIL) == ppd.PPD_EINVAL and call(dict(far, v=F)) == ppd.PPD_EINVAL
    assert call(far, need - 1) == ppd.PPD_EWORKSPACE


def test_another_device_refuses(monkeypatch):
    """A tensor of another device than the current one is named."""
    class On:
        def __init__(self, d):
            self.d = d

        def get_device(self):
            return self.d
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    ppd._here(a=On(1), b=None)
    with pytest.raises(ValueError, match="q is on device 0"):
        ppd._here(a=On(1), q=On(0))


def test_score_refuses():
    L = ppd.lib()

    def call(kv=None, Lc=5, nh=8, T=4, q=F, dt=ppd.PPD_F32, lse=F, rows=4, path=F, n=4, cnt=F, out=F):
        kv = _kvq() if kv is None else kv
        return L.ppd_kvq_score(C.byref(kv), Lc, nh, T, q, dt, lse, rows, path, n, cnt, None, out, None)
    for kw, code in BAD_CACHES:
        assert call(_kvq(**kw)) == code, kw
    for kw, code in BAD_ROWS:
        assert call(_kvq(tail=kw)) == code, kw
    assert call(Lc=-1) == ppd.PPD_ECAPACITY and call(Lc=257) == ppd.PPD_ECAPACITY
    assert call(nh=6) == ppd.PPD_EINVAL and call(nh=0) == ppd.PPD_EINVAL and call(nh=1 << 17) == ppd.PPD_EINVAL
    assert call(T=0) == ppd.PPD_EINVAL and call(T=129, rows=200) == ppd.PPD_EINVAL and call(rows=3) == ppd.PPD_EINVAL
    assert call(_kvq(tail=dict(k=F, v=F, capacity=8)), T=9, rows=9) == ppd.PPD_ECAPACITY
    assert call(dt=7) == ppd.PPD_EINVAL and call(q=F + 4) == ppd.PPD_EINVAL
    for null in ("q", "lse", "path", "cnt", "out"):
        assert call(**{null: None}) == ppd.PPD_EINVAL
    assert call(n=0) == ppd.PPD_EINVAL and call(n=129) == ppd.PPD_EINVAL


def test_evict_refuses():
    L = ppd.lib()
    far = F + (1 << 30)

    def call(src=None, dst=None, Lc=100, budget=50, sink=2, recent=8, score=F, out=None, kept=F):
        src = _kvq() if src is None else src
        dst = _kvq(blocks=far) if dst is None else dst
        return L.ppd_kvq_evict(C.byref(src), C.byref(dst), Lc, budget, sink, recent, score, far if out is None else out,
                               kept, None)
    for kw, code in BAD_CACHES:
        assert call(_kvq(**kw)) == code and call(dst=_kvq(**kw)) == code, kw
    assert call(dst=_kvq(blocks=far, layers=3)) == ppd.PPD_EINVAL and call(dst=_kvq(blocks=far, heads=2)) == ppd.PPD_EINVAL
    assert call(Lc=-1) == ppd.PPD_ECAPACITY and call(Lc=257) == ppd.PPD_ECAPACITY
    assert call(budget=0) == ppd.PPD_EINVAL and call(budget=257) == ppd.PPD_ECAPACITY
    assert call(sink=-1) == ppd.PPD_EINVAL and call(recent=-1) == ppd.PPD_EINVAL
    assert call(sink=40, recent=11) == ppd.PPD_EINVAL and call(sink=2147483647, recent=2147483647) == ppd.PPD_EINVAL
    assert call(score=None) == ppd.PPD_EINVAL and call(kept=None) == ppd.PPD_EINVAL
    # caches or scores that lie over one another without being the same
    assert call(dst=_kvq(blocks=F + 4608)) == ppd.PPD_EINVAL
    assert call(dst=_kvq(cap=128)) == ppd.PPD_EINVAL
    assert call(out=F + 16) == ppd.PPD_EINVAL and call(out=F) == ppd.PPD_EINVAL
    assert call(dst=_kvq(tail={}), out=F, Lc=0) == ppd.PPD_OK  # in place, nothing cached


def test_accept_sample_refuses():
    L = ppd.lib()
    need = ppd.ppd_accept_sample_workspace_bytes(4, 10)

    def call(T=4, vocab=10, t=1.0, ws=F, n=need, **kw):
        p = dict(parent=F, ids=F, logits=F, u=F, path=F, n_path=F, nxt=F)
        p.update(kw)
        return L.ppd_accept_sample(T, p["parent"], p["ids"], vocab, p["logits"], t, None, p["u"], p["path"], p["n_path"],
                                   p["nxt"], ws, n, None)
    assert call(T=0) == ppd.PPD_EINVAL and call(T=129) == ppd.PPD_EINVAL and call(vocab=0) == ppd.PPD_EINVAL
    for t in (0.0, -1.0, float("inf"), float("nan")):
        assert call(t=t) == ppd.PPD_EINVAL
    for null in ("parent", "ids", "logits", "u", "path", "n_path", "nxt"):
        assert call(**{null: None}) == ppd.PPD_EINVAL
    assert call(ws=None) == ppd.PPD_EWORKSPACE and call(n=need - 1) == ppd.PPD_EWORKSPACE
    assert call(ws=F + 8) == ppd.PPD_EINVAL


def test_python_refusals():
    """What only the binding sees: shapes, types, devices."""
    ok = torch.zeros((2, 4, 8, 4608), dtype=torch.uint8)
    rows = ppd.KVCache(torch.zeros((2, 4, 16, 128), dtype=torch.bfloat16), torch.zeros((2, 4, 128, 16), dtype=torch.bfloat16))
    kv = ppd.KVQCache(ok, rows)
    assert (kv.n_layers, kv.n_kv_heads, kv.capacity) == (2, 4, 256)
    for bad in (ok[..., :4600], ok[0], ok.float(), torch.zeros((2, 4, 4608, 8), dtype=torch.uint8).transpose(2, 3)):
        with pytest.raises(ValueError):
            ppd.KVQCache(bad)
    for k, v in (((2, 4, 16, 64), (2, 4, 64, 16)), ((2, 2, 16, 128), (2, 2, 128, 16)), ((2, 4, 16, 128), (2, 4, 16, 128))):
        with pytest.raises(ValueError):
            ppd.KVQCache(ok, ppd.KVCache(torch.zeros(k, dtype=torch.bfloat16), torch.zeros(v, dtype=torch.bfloat16)))
    with pytest.raises(ValueError):
        ppd.KVQCache(ok, ppd.KVCache(rows.k.float(), rows.v.float()))
    with pytest.raises(ValueError):
        ppd.KVQCache.empty(2, 4, 100, device="cpu")
    with pytest.raises(ValueError, match="device"):
        ppd.ppd_kvq_quantize(kv, 0, rows, 0, 4)
    z = torch.zeros(4)
    with pytest.raises(ValueError, match="device"):
        ppd.ppd_accept_sample(1, z.int(), z.int(), 4, z, 1.0, None, z, z.int(), z.int(), z.int(), z)
    with pytest.raises(ValueError, match="device"):
        ppd.ppd_kvq_commit(kv, 0, torch.zeros(4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))


@pytest.mark.parametrize("seed", range(3))
def test_reference_blocks_round_trip(seed):
    """store and load agree, leave other positions alone, and a held value is
    within half a scale step of its row (a bf16 scale rounds by 2^-9, so the
    largest code's value by 15 x 2^-9 of a step more)."""
    rng = np.random.default_rng(seed)
    words = rng.integers(0, 1 << 32, (2, 1152), dtype=np.uint32)
    k, v = (R.bf16(rng.standard_normal((19, 128))) for _ in range(2))
    R.store(words, 20, k, v)
    before = words.copy()
    R.store(words, 25, k[5:8], v[5:8])  # the same rows again
    assert np.array_equal(words, before)
    for got, rows in zip(R.load(words, 39), (k, v)):
        g = rows.reshape(-1, 2, 64)
        step = ((g.max(-1) - g.min(-1)) / 15).repeat(64, -1).reshape(-1, 128)
        assert (np.abs(got[20:] - rows) <= step * (0.5 + 15 * 2.0 ** -8)).all()


@pytest.mark.parametrize("with_draft", [False, True])
def test_sampled_acceptance_follows_the_target(with_draft):
    """Over random draws the first emitted token (the accepted child's, or the
    bonus) has the target's distribution: chi-square of 5 classes, 4 degrees
    of freedom, below 30 (probability 5e-6 by chance, and the seed is fixed)."""
    rng = np.random.default_rng(5)
    V, N = 5, 20000
    logits = rng.standard_normal((4, V)).astype(np.float32)
    target = R.weights(logits[0], 0.8)
    target /= target.sum()
    q = rng.random(V).astype(np.float32)
    q /= q.sum()
    draft = np.tile(q, (4, 1)) if with_draft else None
    parent = np.array([-1, 0, 0, 0])
    count = np.zeros(V)
    for _ in range(N):
        kids = rng.choice(V, 3, p=q / q.sum(dtype=np.float64)) if with_draft else np.array([3, 1, 1])
        ids = np.concatenate(([0], kids))
        path, bonus, bad = R.accept_sample(parent, ids, V, logits, 0.8, draft, rng.random(4).astype(np.float32))
        assert not bad
        count[ids[path[1]] if len(path) > 1 else bonus] += 1
    assert ((count - N * target) ** 2 / (N * target)).sum() < 30


def test_host_code_clean_under_asan_and_ubsan():
    """The refusals above again, against the host sources built with both
    sanitizers (a child process; torch's checks of it are not repeated)."""
    if os.environ.get("PPD_LIBRARY"):
        pytest.skip("already the sanitized build")
    from paper_2405_18628_amd.build import build_host_sanitized, sanitizer_runtime
    env = dict(os.environ, LD_PRELOAD=sanitizer_runtime(), PPD_LIBRARY=build_host_sanitized(),
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "-k", "refuse or sizes", __file__],
                       env=env, cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "passed" in r.stdout
