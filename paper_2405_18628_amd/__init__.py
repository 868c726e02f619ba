"""Python binding of libppd, the MI355X (gfx950) PPD tree-verification step.

Argument marshalling only: every step of the computation runs in the HIP
kernels of libppd.so.  Functions carry the names of the C ABI (include/ppd.h);
tensors are torch tensors used as device memory, streams are torch streams.
Importing works without a GPU (the host-side tree builder and the argument
checks run anywhere); device calls need the built library and a GPU, and
fail loudly otherwise -- there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# PPD_LIBRARY selects another build of the same library (the host-sanitizer
# build that the CPU tests load); by default the one next to this file
LIB_PATH = os.environ.get("PPD_LIBRARY") or os.path.join(_HERE, "libppd.so")

PPD_OK, PPD_EINVAL, PPD_ETREE, PPD_ECAPACITY, PPD_EDEVICE, PPD_EUNSUPPORTED, PPD_EWORKSPACE = range(7)
PPD_F32, PPD_BF16 = 0, 1
PPD_T_MAX = 128
PPD_MASK_WORDS = 2
PPD_DEV_BAD_TOKEN, PPD_DEV_BAD_PARENT, PPD_DEV_NAN_LOGIT = 1, 2, 4
PPD_KVQ_BLOCK, PPD_KVQ_BLOCK_BYTES = 32, 4608
PPD_W_QKV, PPD_W_O, PPD_W_GATE_UP, PPD_W_DOWN, PPD_W_LM_HEAD = range(5)

_STATUS_NAMES = {0: "PPD_OK", 1: "PPD_EINVAL", 2: "PPD_ETREE", 3: "PPD_ECAPACITY",
                 4: "PPD_EDEVICE", 5: "PPD_EUNSUPPORTED", 6: "PPD_EWORKSPACE"}


class PPDError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class ppd_model(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hidden", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn", C.c_int32),
                ("vocab", C.c_int32), ("n_prompt", C.c_int32), ("rms_eps", C.c_float),
                ("rope_base", C.c_float), ("dtype", C.c_int32),
                ("tok_emb", C.c_void_p), ("prompt_emb", C.c_void_p),
                ("attn_norm", C.POINTER(C.c_void_p)), ("w_qkv", C.POINTER(C.c_void_p)),
                ("w_o", C.POINTER(C.c_void_p)), ("mlp_norm", C.POINTER(C.c_void_p)),
                ("w_gate_up", C.POINTER(C.c_void_p)), ("w_down", C.POINTER(C.c_void_p)),
                ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)]


class ppd_kv(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("capacity", C.c_int32),
                ("len_dev", C.c_void_p)]


class ppd_kvq(C.Structure):
    _fields_ = [("blocks", C.c_void_p), ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32),
                ("capacity", C.c_int32), ("tail", ppd_kv)]


_lib = None


def lib() -> C.CDLL:
    """The loaded libppd.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run paper_2405_18628_amd.build.build()")
        L = C.CDLL(LIB_PATH)
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        P = C.POINTER
        L.ppd_workspace_bytes.argtypes = [P(ppd_model), i32, i32]
        L.ppd_workspace_bytes.restype = sz
        L.ppd_workspace_init.argtypes = [vp, sz, vp]
        L.ppd_build_tree_mask.argtypes = [i32, vp, vp, vp]
        L.ppd_verify_step.argtypes = [P(ppd_model), P(ppd_kv), i32, i32, vp, vp, vp, vp, sz, vp,
                                      vp, vp]
        L.ppd_verify_batch.argtypes = [P(ppd_model), i32, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp,
                                       vp]
        L.ppd_verify_step_static.argtypes = [P(ppd_model), P(ppd_kv), i32, i32, vp, vp, vp, vp, vp,
                                             vp, vp]
        L.ppd_accept.argtypes = [i32, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.ppd_kv_compact.argtypes = [P(ppd_model), P(ppd_kv), i32, vp, i32, vp, vp]
        L.ppd_device_status.argtypes = [vp, sz, P(C.c_uint32), i32, vp]
        L.ppd_set_kernel_timer.argtypes = [i32, vp, vp, i32]
        L.ppd_last_error.restype = C.c_char_p
        L.ppd_next_tree.argtypes = [i32, vp, vp, i32, i32, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp,
                                    sz, vp]
        L.ppd_sparse_template.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, P(C.c_int32),
                                          P(C.c_double)]
        L.ppd_packed_weight_bytes.argtypes = [i32, i32, i32]
        L.ppd_packed_weight_bytes.restype = sz
        L.ppd_pack_weight.argtypes = [i32, i32, i32, vp, vp, vp]
        L.ppd_read_probe.argtypes = [vp, sz, vp, vp]
        L.ppd_kvq_bytes.argtypes = [i32, i32, i32]
        L.ppd_kvq_attention_workspace_bytes.argtypes = [i32, i32, i32]
        L.ppd_kvq_workspace_bytes.argtypes = [P(ppd_model), i32]
        L.ppd_accept_sample_workspace_bytes.argtypes = [i32, i32]
        for f in ("ppd_kvq_bytes", "ppd_kvq_attention_workspace_bytes", "ppd_kvq_workspace_bytes",
                  "ppd_accept_sample_workspace_bytes"):
            getattr(L, f).restype = sz
        L.ppd_kvq_quantize.argtypes = [P(ppd_kvq), i32, P(ppd_kv), i32, i32, vp]
        L.ppd_kvq_dequantize.argtypes = [P(ppd_kvq), i32, P(ppd_kv), i32, i32, vp]
        L.ppd_kvq_commit.argtypes = [P(ppd_kvq), i32, vp, i32, vp, vp]
        L.ppd_kvq_attention.argtypes = [i32, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.ppd_verify_batch_kvq.argtypes = [P(ppd_model), i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp, vp, vp, vp]
        L.ppd_verify_step_kvq.argtypes = [P(ppd_model), P(ppd_kvq), i32, i32, i32, vp, vp, vp, vp, sz, vp, vp, vp, vp,
                                          vp]
        L.ppd_kvq_score.argtypes = [P(ppd_kvq), i32, i32, i32, vp, i32, vp, i32, vp, i32, vp, vp, vp, vp]
        L.ppd_kvq_evict.argtypes = [P(ppd_kvq), P(ppd_kvq), i32, i32, i32, i32, vp, vp, vp, vp]
        L.ppd_accept_sample.argtypes = [i32, vp, vp, i32, vp, C.c_float, vp, vp, vp, vp, vp, vp, sz, vp]
        for f in ("ppd_kvq_quantize", "ppd_kvq_dequantize", "ppd_kvq_commit", "ppd_kvq_attention",
                  "ppd_verify_batch_kvq", "ppd_verify_step_kvq", "ppd_kvq_score", "ppd_kvq_evict", "ppd_accept_sample"):
            getattr(L, f).restype = C.c_int
        for f in ("ppd_verify_step_static", "ppd_next_tree", "ppd_sparse_template", "ppd_verify_batch", "ppd_pack_weight", "ppd_workspace_init", "ppd_build_tree_mask", "ppd_verify_step", "ppd_accept",
                  "ppd_kv_compact", "ppd_device_status", "ppd_set_kernel_timer", "ppd_read_probe"):
            getattr(L, f).restype = C.c_int
        _lib = L
    return _lib


def ppd_last_error() -> str:
    return lib().ppd_last_error().decode()


def _check(status: int):
    if status != PPD_OK:
        raise PPDError(status, ppd_last_error())


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


# The small calls after a forward pass are bound by this module's host time
# (accept, compact and next tree: 34 us of Python for 20 us of kernels), so
# what every call does is kept short: the current stream's handle comes from
# torch's raw getters (0.2 us; building a torch.cuda.Stream takes 2.5), and
# the tensor checks take one pass (_i32_ok), with _dev naming the fault.
_torch = None


def _forget_torch():
    global _torch
    _torch = None


# a forked child goes through torch.cuda.init() again, which refuses a child of
# a process that uses the GPU (the raw getters would hand out its stream)
os.register_at_fork(after_in_child=_forget_torch)


def _stream(stream) -> Optional[int]:
    if stream is None:
        global _torch
        if _torch is None:
            import torch
            torch.cuda.init()
            _torch = torch
        c = _torch._C
        return c._cuda_getCurrentRawStream(c._cuda_getDevice())
    return getattr(stream, "cuda_stream", stream)


def _i32_ok(tensors) -> bool:
    """Every tensor is a contiguous int32 device tensor."""
    try:
        for t in tensors:
            if not (t.is_cuda and t.dtype is _torch.int32 and t.is_contiguous()):
                return False
        return True
    except AttributeError:  # None, or torch not loaded yet: the full check decides
        return False


def _i32(**tensors):
    if not _i32_ok(tensors.values()):
        import torch
        for name, t in tensors.items():
            _dev(t, torch.int32, name)


def _host_i32(v):
    """`v` as a contiguous int32 numpy array (no copy if it is one; a scalar
    becomes an array of one)."""
    if type(v) is np.ndarray and v.ndim and v.dtype == np.int32 and v.flags.c_contiguous:
        return v
    return np.ascontiguousarray(np.asarray(v, dtype=np.int32))


def _np_ptr(a) -> int:
    return a.__array_interface__["data"][0]


def _dev(t, dtype=None, name="tensor"):
    if t is None:
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")


def _here(**tensors):
    """Refuse tensors of another device than the current one, on whose stream
    a call is enqueued."""
    import torch
    now = torch.cuda.current_device()
    for name, t in tensors.items():
        if t is not None and t.get_device() != now:
            raise ValueError(f"{name} is on device {t.get_device()}, the current device is {now}")


def _tensors(dev, *checks):
    """Every (tensor or None, dtype or None, name) is contiguous, of its type and
    on device `dev`, which is the current one; _dev and _here name a fault.  One
    pass of a few lookups a tensor, as _i32_ok: the short calls are bound by it."""
    if dev >= 0 and _torch is None:
        _stream(None)  # sets _torch
    ok = dev >= 0 and _torch._C._cuda_getDevice() == dev
    for t, dtype, name in checks:
        if t is not None and not (ok and t.get_device() == dev and t.is_contiguous() and (dtype is None or t.dtype is dtype)):
            _dev(t, dtype, name)
            _here(**{name: t})


# ---------------------------------------------------------------------------


class Model:
    """A ppd_model description over device tensors (kept alive by this object).

    `w` follows the row-major layout of include/ppd.h (see
    synth.model.make_weights).  For bf16 models the five projection matrices
    are packed once here (ppd_pack_weight) and the description points at the
    packed copies; `w` itself is left unchanged."""

    _PACKED = {"w_qkv": PPD_W_QKV, "w_o": PPD_W_O, "w_gate_up": PPD_W_GATE_UP,
               "w_down": PPD_W_DOWN}

    def __init__(self, shape, w, stream=None):
        import torch
        dt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        self.shape = shape
        self.w = w
        layers = w["layers"]
        n = shape.n_layers
        bf16 = shape.dtype == "bf16"
        self.packed = {k: [] for k in self._PACKED}

        def arr(key):
            ptrs = []
            for lay in layers:
                _dev(lay[key], dt, key)
                if bf16 and key in self._PACKED:
                    pk = ppd_pack_weight(self._PACKED[key], lay[key], stream)
                    self.packed[key].append(pk)
                    ptrs.append(_ptr(pk))
                else:
                    ptrs.append(_ptr(lay[key]))
            return (C.c_void_p * n)(*ptrs)

        for key in ("tok_emb", "prompt_emb", "final_norm", "lm_head"):
            _dev(w[key], dt, key)
        self._arrays = {k: arr(k) for k in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up",
                                            "w_down")}
        self.lm_head = ppd_pack_weight(PPD_W_LM_HEAD, w["lm_head"], stream) if bf16 else w["lm_head"]
        a = self._arrays
        self.desc = ppd_model(
            shape.n_layers, shape.hidden, shape.n_heads, shape.n_kv_heads, shape.head_dim,
            shape.ffn, shape.vocab, shape.n_prompt, shape.rms_eps, shape.rope_base,
            PPD_BF16 if bf16 else PPD_F32,
            _ptr(w["tok_emb"]), _ptr(w["prompt_emb"]),
            C.cast(a["attn_norm"], C.POINTER(C.c_void_p)), C.cast(a["w_qkv"], C.POINTER(C.c_void_p)),
            C.cast(a["w_o"], C.POINTER(C.c_void_p)), C.cast(a["mlp_norm"], C.POINTER(C.c_void_p)),
            C.cast(a["w_gate_up"], C.POINTER(C.c_void_p)), C.cast(a["w_down"], C.POINTER(C.c_void_p)),
            _ptr(w["final_norm"]), _ptr(self.lm_head))


    def first_layers(self, n: int) -> "Model":
        """The same model cut to its first n decoder layers (final norm and
        LM head unchanged), sharing this object's packed weights: no copy."""
        import copy
        if not 1 <= n <= self.shape.n_layers:
            raise ValueError(f"n={n} outside [1, {self.shape.n_layers}]")
        m = copy.copy(self)
        m.shape = self.shape.with_layers(n)
        m.desc = ppd_model.from_buffer_copy(self.desc)
        m.desc.n_layers = n
        m._parent = self
        return m


class KVCache:
    """K [layers][kv_heads][capacity][head_dim], V [layers][kv_heads][head_dim][capacity]."""

    def __init__(self, k, v, len_dev=None):
        self.k, self.v, self.len_dev = k, v, len_dev
        self.capacity = int(k.shape[2])
        self.desc = ppd_kv(_ptr(k), _ptr(v), self.capacity, _ptr(len_dev) or None)


class KVQCache:
    """4-bit cache: blocks uint8 [layers][kv_heads][capacity / 32][4608] (layout
    in include/ppd.h) and, for the calls that read or write tree rows, their
    bf16 staging cache `tail` (a KVCache of the same layers and heads)."""

    def __init__(self, blocks, tail: Optional[KVCache] = None):
        if blocks.dim() != 4 or blocks.shape[3] != PPD_KVQ_BLOCK_BYTES or blocks.element_size() != 1:
            raise ValueError(f"blocks must be bytes [layers][kv_heads][capacity / 32][{PPD_KVQ_BLOCK_BYTES}]")
        if not blocks.is_contiguous():
            raise ValueError("blocks must be contiguous")
        if tail is not None:
            self._check_rows(tail, blocks.shape[:2], "tail")
        self.blocks, self.tail = blocks, tail
        self.device = blocks.get_device()
        self.n_layers, self.n_kv_heads = int(blocks.shape[0]), int(blocks.shape[1])
        self.capacity = int(blocks.shape[2]) * PPD_KVQ_BLOCK
        self.desc = ppd_kvq(_ptr(blocks), self.n_layers, self.n_kv_heads, self.capacity,
                            tail.desc if tail is not None else ppd_kv())

    @classmethod
    def empty(cls, n_layers: int, n_kv_heads: int, capacity: int, tail_capacity: int = PPD_T_MAX, device="cuda"):
        """A cache of `capacity` positions and its staging cache, uninitialised."""
        import torch
        if capacity < 1 or capacity % PPD_KVQ_BLOCK:
            raise ValueError(f"capacity must be a positive multiple of {PPD_KVQ_BLOCK}")
        k = torch.empty((n_layers, n_kv_heads, tail_capacity, 128), dtype=torch.bfloat16, device=device)
        v = torch.empty((n_layers, n_kv_heads, 128, tail_capacity), dtype=torch.bfloat16, device=device)
        blocks = torch.empty((n_layers, n_kv_heads, capacity // PPD_KVQ_BLOCK, PPD_KVQ_BLOCK_BYTES),
                             dtype=torch.uint8, device=device)
        return cls(blocks, KVCache(k, v))

    @staticmethod
    def _check_rows(kv: KVCache, heads, name):
        """kv is a bf16 cache of [layers][kv_heads] = heads, head_dim 128 (looked at
        once: a KVCache describes its tensors as they were given)."""
        import torch
        want = (int(heads[0]), int(heads[1]))
        if getattr(kv, "_rows", None) == want:
            return
        if (tuple(kv.k.shape) != (*want, kv.capacity, 128) or tuple(kv.v.shape) != (*want, 128, kv.capacity) or
                kv.k.dtype != torch.bfloat16 or kv.v.dtype != torch.bfloat16):
            raise ValueError(f"{name} must be a bf16 cache of {want[0]} layers, {want[1]} heads and 128 dims")
        if not (kv.k.is_contiguous() and kv.v.is_contiguous()):
            raise ValueError(f"{name} must be contiguous")
        if kv.k.get_device() != kv.v.get_device():
            raise ValueError(f"{name} lies on two devices")
        n = kv.len_dev
        if n is not None and (n.dtype != torch.int32 or n.numel() < 1 or n.get_device() != kv.k.get_device()):
            raise ValueError(f"{name}: len_dev must be an int32 on its device")
        kv._rows = want

    def _on_device(self, *checks):
        """The cache, and the call's other tensors, are on the current device."""
        tail = self.tail
        _tensors(self.device, (self.blocks, None, "blocks"), (tail.k if tail is not None else None, None, "tail"), *checks)


# ---------------------------------------------------------------------------
# the C ABI, one Python function per entry point


def ppd_workspace_bytes(model: Model, t_max: int, max_len: int) -> int:
    n = lib().ppd_workspace_bytes(C.byref(model.desc), t_max, max_len)
    if n == 0:
        raise PPDError(PPD_EINVAL, ppd_last_error())
    return int(n)


def ppd_packed_weight_bytes(kind: int, rows: int, cols: int) -> int:
    n = lib().ppd_packed_weight_bytes(int(kind), int(rows), int(cols))
    if n == 0:
        raise PPDError(PPD_EINVAL, ppd_last_error())
    return int(n)


def ppd_pack_weight(kind: int, src, stream=None):
    """Packed copy (a new uint8 device tensor) of the row-major bf16 matrix
    `src` [rows][cols], in the layout the bf16 GEMMs read."""
    import torch
    _dev(src, torch.bfloat16, "weight")
    rows, cols = (int(x) for x in src.shape)
    dst = torch.empty(ppd_packed_weight_bytes(kind, rows, cols), dtype=torch.uint8,
                      device=src.device)
    _check(lib().ppd_pack_weight(int(kind), rows, cols, _ptr(src), _ptr(dst), _stream(stream)))
    return dst


def ppd_workspace_init(ws, stream=None):
    _dev(ws, None, "ws")
    _check(lib().ppd_workspace_init(_ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def ppd_build_tree_mask(parent: Sequence[int]):
    """Host: (depth int32[T], mask uint64[T][2]) of a topological parent array."""
    p = np.ascontiguousarray(np.asarray(parent, dtype=np.int32))
    T = int(p.shape[0])
    depth = np.zeros(T, np.int32)
    mask = np.zeros((T, PPD_MASK_WORDS), np.uint64)
    _check(lib().ppd_build_tree_mask(T, p.ctypes.data, depth.ctypes.data, mask.ctypes.data))
    return depth, mask


def ppd_verify_step(model: Model, kv: KVCache, L: int, T: int, ids, depth, mask, ws, logits,
                    pred, stream=None):
    import torch
    _i32(ids=ids, depth=depth, pred=pred)
    _dev(mask, None, "mask")
    _dev(ws, None, "ws")
    _dev(logits, torch.float32, "logits")
    _check(lib().ppd_verify_step(C.byref(model.desc), C.byref(kv.desc), int(L), int(T), _ptr(ids),
                                 _ptr(depth), _ptr(mask), _ptr(ws),
                                 ws.numel() * ws.element_size(), _ptr(logits) or None,
                                 _ptr(pred), _stream(stream)))


def ppd_verify_step_static(model: Model, kv: KVCache, L: int, T: int, ids, depth, mask, logits,
                           pred, status_out=None, stream=None):
    """ppd_verify_step with the library's static workspace (no allocation)."""
    import torch
    for t, n in ((ids, "ids"), (depth, "depth"), (pred, "pred")):
        _dev(t, torch.int32, n)
    _dev(mask, None, "mask")
    _dev(logits, torch.float32, "logits")
    _dev(status_out, torch.int32, "status_out")
    _check(lib().ppd_verify_step_static(C.byref(model.desc), C.byref(kv.desc), int(L), int(T),
                                        _ptr(ids), _ptr(depth), _ptr(mask), _ptr(logits) or None,
                                        _ptr(pred), _ptr(status_out) or None, _stream(stream)))


def ppd_verify_batch(model: Model, kvs: Sequence[KVCache], L: Sequence[int], T: Sequence[int],
                     ids, depth, mask, ws, logits, pred, stream=None):
    """One step over len(kvs) sequences whose trees are packed in sequence
    order (device ids / depth / mask / logits / pred rows)."""
    import torch
    for t, n in ((ids, "ids"), (depth, "depth"), (pred, "pred")):
        _dev(t, torch.int32, n)
    _dev(mask, None, "mask")
    _dev(ws, None, "ws")
    _dev(logits, torch.float32, "logits")
    B = len(kvs)
    if len(L) != B or len(T) != B:
        raise ValueError("kvs, L and T differ in length")
    descs = (ppd_kv * max(B, 1))(*[kv.desc for kv in kvs])
    Ls = np.ascontiguousarray(np.asarray(L, dtype=np.int32))
    Ts = np.ascontiguousarray(np.asarray(T, dtype=np.int32))
    _check(lib().ppd_verify_batch(C.byref(model.desc), B, C.cast(descs, C.c_void_p),
                                  Ls.ctypes.data, Ts.ctypes.data, _ptr(ids), _ptr(depth),
                                  _ptr(mask), _ptr(ws), ws.numel() * ws.element_size(),
                                  _ptr(logits) or None, _ptr(pred), _stream(stream)))


def ppd_accept(T: int, parent, ids, pred, vocab: int, path, n_path, next_tok, ws, stream=None):
    _i32(parent=parent, ids=ids, pred=pred, path=path, n_path=n_path, next_tok=next_tok)
    _check(lib().ppd_accept(int(T), _ptr(parent), _ptr(ids), _ptr(pred), int(vocab), _ptr(path),
                            _ptr(n_path), _ptr(next_tok), _ptr(ws), ws.numel() * ws.element_size(),
                            _stream(stream)))


def ppd_next_tree(T: int, parent, ids, vocab: int, n_prompt: int, logits, path, n_path,
                  next_tok, tpl_parent: Sequence[int], tpl_kind: Sequence[int], next_ids, ws,
                  stream=None, n_ept: int = 1):
    """Token ids of the next step's tree (template tpl_parent / tpl_kind, host
    sequences) into the device tensor next_ids."""
    import torch
    _i32(parent=parent, ids=ids, path=path, n_path=n_path, next_tok=next_tok, next_ids=next_ids)
    _dev(logits, torch.float32, "logits")
    tp = _host_i32(tpl_parent)
    tk = _host_i32(tpl_kind)
    if tp.shape != tk.shape:
        raise ValueError("tpl_parent and tpl_kind differ in length")
    _check(lib().ppd_next_tree(int(T), _ptr(parent), _ptr(ids), int(vocab), int(n_prompt),
                               int(n_ept), _ptr(logits), _ptr(path), _ptr(n_path), _ptr(next_tok),
                               int(tp.shape[0]), _np_ptr(tp), _np_ptr(tk), _ptr(next_ids),
                               _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def ppd_sparse_template(p_table, n_cand: int, n_prompt: int, n_ept: int = 1):
    """Template of the n_cand candidates that maximise Proposition 1's expected
    accepted length under the host table p_table[depth - 1][rank].  Returns
    (tpl_parent, tpl_kind, expected accepted candidates)."""
    p = np.ascontiguousarray(np.asarray(p_table, dtype=np.float64))
    if p.ndim != 2:
        raise ValueError("p_table must be 2-D [depth][rank]")
    par = np.zeros(PPD_T_MAX, np.int32)
    kind = np.zeros(PPD_T_MAX, np.int32)
    T = C.c_int32(0)
    f = C.c_double(0.0)
    _check(lib().ppd_sparse_template(p.ctypes.data, p.shape[0], p.shape[1], int(n_cand),
                                     int(n_prompt), int(n_ept), par.ctypes.data, kind.ctypes.data,
                                     C.byref(T), C.byref(f)))
    return par[:T.value].copy(), kind[:T.value].copy(), float(f.value)


def ppd_kv_compact(model: Model, kv: KVCache, L: int, path, n_path, stream=None,
                   path_len: Optional[int] = None):
    """path: device int32 tensor (its length is passed as path_len unless
    given); n_path: device int32 count, clamped on the device."""
    _i32(path=path, n_path=n_path)
    n = int(path.numel()) if path_len is None else int(path_len)
    _check(lib().ppd_kv_compact(C.byref(model.desc), C.byref(kv.desc), int(L), _ptr(path), n,
                                _ptr(n_path), _stream(stream)))


def _bytes(n: int) -> int:
    if n == 0:
        raise PPDError(PPD_EINVAL, ppd_last_error())
    return int(n)


def ppd_kvq_bytes(n_layers: int, n_kv_heads: int, capacity: int) -> int:
    return _bytes(lib().ppd_kvq_bytes(int(n_layers), int(n_kv_heads), int(capacity)))


def _rows_of(kv: KVQCache, other: KVCache, name: str):
    KVQCache._check_rows(other, (kv.n_layers, kv.n_kv_heads), name)
    kv._on_device((other.k, None, name))


def ppd_kvq_quantize(kv: KVQCache, dst_pos: int, src: KVCache, src_pos: int, n: int, stream=None):
    """n bf16 positions of src, from src_pos on, into kv from dst_pos on."""
    _rows_of(kv, src, "src")
    _check(lib().ppd_kvq_quantize(C.byref(kv.desc), int(dst_pos), C.byref(src.desc), int(src_pos), int(n),
                                  _stream(stream)))


def ppd_kvq_dequantize(kv: KVQCache, src_pos: int, dst: KVCache, dst_pos: int, n: int, stream=None):
    """n positions of kv, from src_pos on, as bf16 into dst from dst_pos on."""
    _rows_of(kv, dst, "dst")
    _check(lib().ppd_kvq_dequantize(C.byref(kv.desc), int(src_pos), C.byref(dst.desc), int(dst_pos), int(n),
                                    _stream(stream)))


def _path_len(path, path_len) -> int:
    """Entries of the path that the kernels may read, at most the tensor's."""
    n = path.numel()
    if path_len is None:
        return n
    if path_len > n:
        raise ValueError(f"path holds {n} entries, not {path_len}")
    return int(path_len)


def ppd_kvq_commit(kv: KVQCache, L: int, path, n_path, stream=None, path_len: Optional[int] = None):
    """Rows path[0], .., path[*n_path - 1] of kv.tail to positions L, L + 1, .. of kv."""
    import torch
    n = _path_len(path, path_len)
    kv._on_device((path, torch.int32, "path"), (n_path, torch.int32, "n_path"))
    _check(lib().ppd_kvq_commit(C.byref(kv.desc), int(L), _ptr(path), n, _ptr(n_path), _stream(stream)))


def ppd_kvq_attention_workspace_bytes(n_heads: int, n_kv_heads: int, t_max: int) -> int:
    return _bytes(lib().ppd_kvq_attention_workspace_bytes(int(n_heads), int(n_kv_heads), int(t_max)))


def _dtypes():
    t = _torch
    if t is None:
        import torch as t
    return t.bfloat16, t.float32


def _kvq_batch(kvs, counts, checks=()):
    """The sequences' descriptions and host int32 arrays of one entry each; the
    caches and the call's tensors (`checks`) are on the current device."""
    B = len(kvs)
    arrays = [_host_i32(a) for a in counts]
    for a in arrays:
        if a.shape != (B,):
            raise ValueError("kvs and the sequences' counts differ in length")
    for i, kv in enumerate(kvs):
        kv._on_device(*(() if i else checks))
    descs = C.byref(kvs[0].desc) if B == 1 else (ppd_kvq * max(B, 1))(*[kv.desc for kv in kvs])
    return (B, descs, *arrays)


def ppd_kvq_attention(kvs: Sequence[KVQCache], layer: int, L: Sequence[int], T: Sequence[int], q, mask, out, ws,
                      lse=None, stream=None):
    """Tree attention of one layer: q, out bf16 [tokens][heads][128], lse float32
    [tokens][heads] (optional), mask int64 / uint64 [tokens][2]."""
    bf16, f32 = _dtypes()
    B, descs, Ls, Ts = _kvq_batch(kvs, (L, T), ((q, bf16, "q"), (out, bf16, "out"), (lse, f32, "lse"), (mask, None, "mask"),
                                                (ws, None, "ws")))
    n = int(Ts[0]) if B == 1 else int(Ts.sum())
    shape = q.shape
    if len(shape) != 3 or shape[0] != n or shape[2] != 128 or out.shape != shape:
        raise ValueError(f"q and out must be [{n}][heads][128]")
    nh = shape[1]
    if lse is not None and lse.shape != (n, nh):
        raise ValueError(f"lse must be [{n}][{nh}]")
    if mask.numel() * mask.element_size() < 16 * n:
        raise ValueError(f"mask must be [{n}][2] words of 64 bits")
    _check(lib().ppd_kvq_attention(nh, B, descs, int(layer), _np_ptr(Ls), _np_ptr(Ts), _ptr(q), _ptr(mask), _ptr(out),
                                   _ptr(lse) or None, _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def ppd_kvq_workspace_bytes(model: Model, t_max: int) -> int:
    return _bytes(lib().ppd_kvq_workspace_bytes(C.byref(model.desc), int(t_max)))


def _trace(model, n, q_out, lse_out):
    sh = model.shape
    if q_out is not None and tuple(q_out.shape) != (sh.n_layers, n, sh.n_heads, 128):
        raise ValueError(f"q_out must be [{sh.n_layers}][{n}][{sh.n_heads}][128]")
    if lse_out is not None and tuple(lse_out.shape) != (sh.n_layers, n, sh.n_heads):
        raise ValueError(f"lse_out must be [{sh.n_layers}][{n}][{sh.n_heads}]")


def _step_tensors(dev, ids, depth, mask, ws, logits, pred, q_out, lse_out):
    import torch
    i32, f32 = torch.int32, torch.float32
    _tensors(dev, (ids, i32, "ids"), (depth, i32, "depth"), (pred, i32, "pred"), (mask, None, "mask"), (ws, None, "ws"),
             (logits, f32, "logits"), (q_out, f32, "q_out"), (lse_out, f32, "lse_out"))


def ppd_verify_batch_kvq(model: Model, kvs: Sequence[KVQCache], L: Sequence[int], pos: Sequence[int], T: Sequence[int],
                         ids, depth, mask, ws, logits, pred, q_out=None, lse_out=None, stream=None):
    """ppd_verify_batch on 4-bit caches; pos: the roots' positions."""
    B, descs, Ls, ps, Ts = _kvq_batch(kvs, (L, pos, T))
    _step_tensors(kvs[0].device if B else -1, ids, depth, mask, ws, logits, pred, q_out, lse_out)
    _trace(model, int(Ts.sum()), q_out, lse_out)
    _check(lib().ppd_verify_batch_kvq(C.byref(model.desc), B, descs, _np_ptr(Ls), _np_ptr(ps),
                                      _np_ptr(Ts), _ptr(ids), _ptr(depth), _ptr(mask), _ptr(ws),
                                      ws.numel() * ws.element_size(), _ptr(logits) or None, _ptr(pred),
                                      _ptr(q_out) or None, _ptr(lse_out) or None, _stream(stream)))


def ppd_verify_step_kvq(model: Model, kv: KVQCache, L: int, pos: int, T: int, ids, depth, mask, ws, logits, pred,
                        q_out=None, lse_out=None, stream=None):
    """ppd_verify_step on a 4-bit cache; pos: the root's position."""
    kv._on_device()
    _step_tensors(kv.device, ids, depth, mask, ws, logits, pred, q_out, lse_out)
    _trace(model, int(T), q_out, lse_out)
    _check(lib().ppd_verify_step_kvq(C.byref(model.desc), C.byref(kv.desc), int(L), int(pos), int(T), _ptr(ids),
                                     _ptr(depth), _ptr(mask), _ptr(ws), ws.numel() * ws.element_size(),
                                     _ptr(logits) or None, _ptr(pred), _ptr(q_out) or None, _ptr(lse_out) or None,
                                     _stream(stream)))


def ppd_kvq_score(kv: KVQCache, L: int, q, lse, path, n_path, score_in, score_out, stream=None,
                  path_len: Optional[int] = None):
    """Attention weights of the accepted nodes added to score_in (None: zeros).
    q float32 or bf16 [layers][T][heads][128], lse float32 [layers][T][heads]:
    a tree's rows, which may be a slice [:, t0:t0 + T] of a batch's."""
    import torch
    i32, f32 = torch.int32, torch.float32
    n = _path_len(path, path_len)
    kv._on_device((path, i32, "path"), (n_path, i32, "n_path"), (score_in, f32, "score_in"), (score_out, f32, "score_out"))
    layers, T, nh, d = q.shape if q.dim() == 4 else (0, 0, 0, 0)
    if layers != kv.n_layers or d != 128 or lse.shape != q.shape[:3]:
        raise ValueError("q must be [layers][T][heads][128], lse [layers][T][heads]")
    if q.dtype not in (f32, torch.bfloat16) or lse.dtype is not f32:
        raise ValueError("q must be float32 or bfloat16, lse float32")
    rows = T if layers == 1 else q.stride(0) // (nh * 128)
    for t, name, row in ((q, "q", nh * 128), (lse, "lse", nh)):
        if t.get_device() != kv.device:
            raise ValueError(f"{name} must be a device tensor, on the cache's device")
        if not t[0].is_contiguous() or (layers > 1 and t.stride(0) != rows * row):
            raise ValueError(f"{name} must be contiguous, or a slice of the rows of a contiguous tensor")
    want = (layers, kv.n_kv_heads, kv.capacity)
    if score_out.shape != want or (score_in is not None and score_in.shape != want):
        raise ValueError(f"score_in and score_out must be [{want[0]}][{want[1]}][{want[2]}]")
    _check(lib().ppd_kvq_score(C.byref(kv.desc), int(L), nh, T, _ptr(q), PPD_F32 if q.dtype is f32 else PPD_BF16,
                               _ptr(lse), rows, _ptr(path), n, _ptr(n_path), _ptr(score_in) or None, _ptr(score_out),
                               _stream(stream)))


def ppd_kvq_evict(src: KVQCache, dst: KVQCache, L: int, budget: int, n_sink: int, n_recent: int, score, score_out, kept,
                  stream=None) -> int:
    """The kept positions of src moved up into dst (which may be src); returns
    how many stay, min(L, budget)."""
    import torch
    f32 = torch.float32
    src._on_device((score, f32, "score"), (score_out, f32, "score_out"), (kept, torch.int32, "kept"))
    if dst is not src:
        dst._on_device()
    for t, name, kv in ((score, "score", src), (score_out, "score_out", dst)):
        if t.shape != (kv.n_layers, kv.n_kv_heads, kv.capacity):
            raise ValueError(f"{name} must be [{kv.n_layers}][{kv.n_kv_heads}][{kv.capacity}]")
    if kept.shape != (src.n_layers, src.n_kv_heads, budget):
        raise ValueError(f"kept must be [{src.n_layers}][{src.n_kv_heads}][{budget}]")
    _check(lib().ppd_kvq_evict(C.byref(src.desc), C.byref(dst.desc), int(L), int(budget), int(n_sink), int(n_recent),
                               _ptr(score), _ptr(score_out), _ptr(kept), _stream(stream)))
    return min(int(L), int(budget))


def ppd_accept_sample_workspace_bytes(T: int, vocab: int) -> int:
    return _bytes(lib().ppd_accept_sample_workspace_bytes(int(T), int(vocab)))


def ppd_accept_sample(T: int, parent, ids, vocab: int, logits, temperature: float, draft, u, path, n_path, next_tok, ws,
                      stream=None):
    """ppd_accept's place at a temperature: children verified against the
    target's probabilities with the draws u [T]; draft float32 [T][vocab] or
    None (children chosen without chance)."""
    import torch
    i32, f32 = torch.int32, torch.float32
    _tensors(logits.get_device(), (logits, f32, "logits"), (parent, i32, "parent"), (ids, i32, "ids"), (u, f32, "u"),
             (path, i32, "path"), (n_path, i32, "n_path"), (next_tok, i32, "next_tok"), (draft, f32, "draft"), (ws, None, "ws"))
    n = int(T)
    for t, name, least in ((parent, "parent", n), (ids, "ids", n), (u, "u", n), (path, "path", n),
                           (logits, "logits", n * vocab), (draft, "draft", n * vocab)):
        if t is not None and t.numel() < least:
            raise ValueError(f"{name} holds {t.numel()} elements, not {least}")
    _check(lib().ppd_accept_sample(int(T), _ptr(parent), _ptr(ids), int(vocab), _ptr(logits), float(temperature),
                                   _ptr(draft) or None, _ptr(u), _ptr(path), _ptr(n_path), _ptr(next_tok), _ptr(ws),
                                   ws.numel() * ws.element_size(), _stream(stream)))


def ppd_device_status(ws, clear: bool = False, stream=None) -> int:
    out = C.c_uint32(0)
    _check(lib().ppd_device_status(_ptr(ws), ws.numel() * ws.element_size(), C.byref(out),
                                   int(bool(clear)), _stream(stream)))
    return int(out.value)


def ppd_read_probe(buf, sink, stream=None):
    """One read of the whole device tensor buf by the HBM read probe; the XOR
    of what it read lands in the device uint32 tensor sink."""
    _dev(buf, None, "buf")
    _dev(sink, None, "sink")
    _check(lib().ppd_read_probe(_ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), _stream(stream)))


KERNEL_KINDS = {"qkv": 0, "attention": 1, "o_proj": 2, "gate_up": 3, "down": 4, "lm_head": 5,
                "next_tree": 6}


def ppd_set_kernel_timer(kind, start_events=(), stop_events=()):
    """Record HIP events around every launch of one kernel kind in later
    ppd_verify_step calls of this thread (torch.cuda.Event objects);
    call with no events to disable.  Returns the ctypes arrays (keep them)."""
    n = len(start_events)
    if n == 0:
        _check(lib().ppd_set_kernel_timer(0, None, None, 0))
        return None
    k = KERNEL_KINDS.get(kind, kind)
    for e in list(start_events) + list(stop_events):
        if not e.cuda_event:      # torch creates the HIP event on first record
            e.record()
    st = (C.c_void_p * n)(*[e.cuda_event for e in start_events])
    sp = (C.c_void_p * n)(*[e.cuda_event for e in stop_events])
    _check(lib().ppd_set_kernel_timer(int(k), st, sp, n))
    return st, sp


__all__ = ["ppd_verify_step_static", "ppd_verify_batch", "ppd_next_tree", "ppd_sparse_template", "ppd_packed_weight_bytes", "ppd_pack_weight", "ppd_set_kernel_timer", "Model", "KVCache", "PPDError", "lib", "ppd_workspace_bytes", "ppd_workspace_init",
           "ppd_build_tree_mask", "ppd_verify_step", "ppd_accept", "ppd_kv_compact",
           "ppd_device_status", "ppd_last_error", "ppd_read_probe", "KVQCache", "ppd_kvq_bytes", "ppd_kvq_quantize",
           "ppd_kvq_dequantize", "ppd_kvq_commit", "ppd_kvq_attention_workspace_bytes", "ppd_kvq_attention",
           "ppd_kvq_workspace_bytes", "ppd_verify_batch_kvq", "ppd_verify_step_kvq", "ppd_kvq_score", "ppd_kvq_evict",
           "ppd_accept_sample_workspace_bytes", "ppd_accept_sample"]
