"""Calls on pages with numbers on the device that are out of range or do not fit
together: what they leave behind, and the bits that name them."""
import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2405_18628_amd as ppd
from test_gpu_paged import BF, Pool, attend, dev, new_rows, workspace

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
