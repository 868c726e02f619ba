"""What the binding of the 4-bit cache refuses before a call is enqueued,
without a GPU: tensors of another device, counts past a path's tensor."""
from types import SimpleNamespace

import pytest
import torch

import paper_2405_18628_amd as ppd


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


def _cache(len_dev=None):
    rows = ppd.KVCache(torch.zeros((2, 4, 16, 128), dtype=torch.bfloat16),
                       torch.zeros((2, 4, 128, 16), dtype=torch.bfloat16), len_dev)
    return ppd.KVQCache(torch.zeros((2, 4, 8, 4608), dtype=torch.uint8), rows)


def _moved(d):
    kv = _cache()
    kv.blocks, kv.tail.k, kv.device = On(d, torch.uint8), On(d, torch.bfloat16), d
    return kv


def test_calls_refuse_another_device(monkeypatch):
    """The current device is 1: a cache, or another tensor of the call, on 0 is
    named, and nothing reaches the library."""
    monkeypatch.setattr(ppd, "_torch", SimpleNamespace(_C=SimpleNamespace(_cuda_getDevice=lambda: 1)))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(ppd, "lib", lambda: pytest.fail("enqueued"))
    ppd._tensors(1, (On(1), torch.int32, "path"), (None, torch.int32, "kept"))
    with pytest.raises(ValueError, match="blocks is on device 0, the current device is 1"):
        ppd.ppd_kvq_commit(_moved(0), 0, On(0), On(0))
    with pytest.raises(ValueError, match="path is on device 0"):
        ppd.ppd_kvq_commit(_moved(1), 0, On(0), On(1))
    with pytest.raises(ValueError, match="n_path is on device 2"):
        ppd.ppd_kvq_commit(_moved(1), 0, On(1), On(2))
    with pytest.raises(ValueError, match="path must be torch.int32"):
        ppd.ppd_kvq_commit(_moved(1), 0, On(1, torch.int64), On(1))
    with pytest.raises(ValueError, match="score is on device 0"):
        ppd.ppd_kvq_evict(_moved(1), _moved(1), 4, 4, 0, 0, On(0, torch.float32), On(1, torch.float32), On(1))
    with pytest.raises(ValueError, match="u is on device 0"):
        ppd.ppd_accept_sample(4, On(1), On(1), 1, On(1, torch.float32), 1.0, None, On(0, torch.float32), On(1), On(1), On(1),
                              On(1))


def test_a_count_past_the_path_is_refused():
    """path_len entries are read on the device: more than the tensor holds would
    be read past its end."""
    kv, path, n = _cache(), torch.zeros(4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q, lse = torch.zeros((2, 4, 8, 128)), torch.zeros((2, 4, 8))
    score = torch.zeros((2, 4, 256))
    with pytest.raises(ValueError, match="path holds 4 entries, not 5"):
        ppd.ppd_kvq_commit(kv, 0, path, n, path_len=5)
    with pytest.raises(ValueError, match="path holds 4 entries, not 128"):
        ppd.ppd_kvq_score(kv, 0, q, lse, path, n, None, score, path_len=128)
    for ok in (None, 1, 4):  # on to the next check
        with pytest.raises(ValueError, match="device"):
            ppd.ppd_kvq_commit(kv, 0, path, n, path_len=ok)


def test_a_count_of_another_kind_or_device_is_refused():
    """len_dev is written as an int32 by the commit's kernel."""
    assert _cache(torch.zeros(1, dtype=torch.int32)).tail.len_dev is not None
    for bad in (torch.zeros(1, dtype=torch.int64), torch.zeros(0, dtype=torch.int32), torch.zeros(1)):
        with pytest.raises(ValueError, match="tail: len_dev"):
            _cache(bad)
    with pytest.raises(ValueError, match="tail: len_dev"):
        far = _cache().tail
        far.len_dev, far._rows = On(0), None
        ppd.KVQCache(torch.zeros((2, 4, 8, 4608), dtype=torch.uint8), far)
