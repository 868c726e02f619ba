"""More of the 4-bit cache on the GPU: magnitudes up to the documented limit,
and captured attention with eager attention between its replays.  The bounds
are those of test_gpu_kvq."""
import numpy as np
import pytest
import torch

import kvq_reference as R
import paper_2405_18628_amd as ppd
from gpu_cases import say
from test_gpu_kvq import _bf16, _cache, _f32, _gen, _score_bound, _tree_mask

pytestmark = pytest.mark.gpu


def _scaled(src, tail, scale):
    """The same rows times a power of two (exact in bfloat16)."""
    for t in (src.k, src.v, tail.k, tail.v):
        t.mul_(scale)


@pytest.mark.parametrize("T,L", [(1, 200), (20, 777), (70, 40)])
@pytest.mark.parametrize("power", [86, -60])
def test_attention_and_weights_at_far_magnitudes(T, L, power):
    """Keys and values of up to 2^90 (16 times 2^86): held, read back, attended to and
    weighed as finite numbers.  (Queries are scaled the other way, so that the
    scores are ordinary ones.)"""
    nh, nkv, cap = 4, 2, (L + 64) // 32 * 32
    say(f"[far] T={T} L={L} 2^{power}")
    kv, src = _cache(1, nkv, L, cap, T, (T + 7) // 8 * 8, T)
    _scaled(src, kv.tail, 2.0 ** power)
    ppd.ppd_kvq_quantize(kv, 0, src, 0, L)
    mask = _tree_mask(T, np.random.default_rng(T), "tree")
    q = _bf16((T, nh, 128), _gen(3)) * 2.0 ** -power
    out, lse = torch.empty_like(q), torch.empty((T, nh), device="cuda")
    ws = torch.empty(ppd.ppd_kvq_attention_workspace_bytes(nh, nkv, T), dtype=torch.uint8, device="cuda")
    ppd.ppd_workspace_init(ws)
    ppd.ppd_kvq_attention([kv], 0, [L], [T], q, torch.from_numpy(mask.view(np.int64)).cuda(), out, ws, lse=lse)
    score = torch.zeros((1, nkv, cap), device="cuda")
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    ppd.ppd_kvq_score(kv, L, q[None], lse[None], torch.zeros(1, dtype=torch.int32, device="cuda"), one, None, score)
    torch.cuda.synchronize()
    words, vis = R.heads_of(kv.blocks)[0], R.mask_bits(mask, T)
    qf = _f32(q).astype(np.float64)
    for a in range(nh):
        h = a // (nh // nkv)
        k, v = R.load(words[h], L)
        kt, vt = _f32(kv.tail.k[0, h, :T]).astype(np.float64), _f32(kv.tail.v[0, h, :, :T]).T.astype(np.float64)
        ref, rl = R.attention(qf[:, a], k, v, kt, vt, vis)
        ds = _score_bound(qf[:, a], words[h], L, kt).max(1)
        tol = 2.0 ** -8 * np.abs(ref) + (2 * (2 * ds + 2.0 ** -16) * max(np.abs(v).max(), np.abs(vt).max()))[:, None]
        assert (np.abs(_f32(out[:, a]) - ref) <= tol).all()
        assert (np.abs(lse[:, a].cpu().numpy() - rl) <= ds + 2.0 ** -22 * (1 + np.abs(rl))).all()
    # the root's weights add up to the heads of a kv head
    assert float((score[..., :L + 1].double().sum(-1) / (nh // nkv) - 1).abs().max()) < 5e-5


def test_attention_captured_between_eager_calls():
    """Two graphs with a workspace each; between the replays eager calls of
    other shapes, on a workspace of their own: all give what they gave alone."""
    cases = []
    for seed, (T, L) in enumerate(((7, 900), (40, 3000), (100, 5000), (3, 20))):
        kv, _ = _cache(1, 4, L, (L + 31) // 32 * 32, T, (T + 7) // 8 * 8, seed)
        m = torch.from_numpy(_tree_mask(T, np.random.default_rng(seed), "tree").view(np.int64)).cuda()
        q = _bf16((T, 8, 128), _gen(seed))
        out = torch.empty_like(q)
        ws = torch.empty(ppd.ppd_kvq_attention_workspace_bytes(8, 4, T), dtype=torch.uint8, device="cuda")
        ppd.ppd_workspace_init(ws)
        run = lambda kv=kv, m=m, q=q, out=out, ws=ws, T=T, L=L: ppd.ppd_kvq_attention([kv], 0, [L], [T], q, m, out, ws)
        run()
        torch.cuda.synchronize()
        cases.append([run, out, out.clone()])
    for c in cases[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c[0]()
        c.append(graph)
    for _ in range(4):
        for graph_case, eager_case in zip(cases[:2], cases[2:]):
            graph_case[1].zero_()
            eager_case[1].zero_()
            graph_case[3].replay()
            eager_case[0]()
            torch.cuda.synchronize()
            assert torch.equal(graph_case[1], graph_case[2]) and torch.equal(eager_case[1], eager_case[2])
