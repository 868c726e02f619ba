"""Limits of the calls on pages, without a GPU."""
import ctypes as C

import paper_2405_18628_amd as ppd

F = 0x10000  # a pointer that is never followed
L = ppd.lib()


def _model(heads):
    ptr = (C.c_void_p * 2)(F, F)
    arr = C.cast(ptr, C.POINTER(C.c_void_p))
    m = ppd.ppd_model(tok_emb=F, prompt_emb=F, attn_norm=arr, w_qkv=arr, w_o=arr, mlp_norm=arr, w_gate_up=arr, w_down=arr,
                      final_norm=F, lm_head=F, n_layers=2, hidden=256, n_heads=heads, n_kv_heads=heads, head_dim=128, ffn=512,
                      vocab=100, n_prompt=3, rms_eps=1e-6, rope_base=1e4, dtype=ppd.PPD_BF16)
    m._keep = ptr
    return m


def test_a_step_over_all_pages_has_no_limit_of_ranked_pages():
    """40 heads x 4096 sequences x 4096 pages are more than selection ranks."""
    m = _model(40)
    size = lambda *a: L.ppd_paged_workspace_bytes(C.byref(m), *a)
    assert L.ppd_paged_select_workspace_bytes(40, 4096, 4096) == 0
    assert size(4096, 4096, 128, 0) > 0 and size(4096, 4096, 128, 64) == 0
    # tables no wider: the same memory
    assert size(4096, 4096, 128, 0) == size(4096, 8, 128, 0)
    for bad in ((0, 8, 4, 0), (4097, 8, 4, 0), (3, 0, 4, 0), (3, -1, 4, 0), (3, (1 << 19) + 1, 4, 0)):
        assert size(*bad) == 0 and ppd.ppd_last_error()
    # the step itself (refused here for its small workspace, not for its sizes)
    kv = ppd.ppd_paged(F, F, 2, 40, 1 << 20, 64, ppd.ppd_kv(F, F, 128, None))
    pt = ppd.ppd_page_tables(F, F, F, F, 4096, 4096, 1 << 20, 64)
    for budget, code in ((0, ppd.PPD_EWORKSPACE), (64, ppd.PPD_EINVAL)):
        assert L.ppd_verify_batch_paged(C.byref(m), C.byref(kv), C.byref(pt), F, 128, F, F, F, budget, 0, 0, F, 1000, None, F,
                                        None) == code
