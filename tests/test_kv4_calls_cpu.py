"""What the binding's calls of the cache in 4 bits take and refuse, on the host: tensors that only say where they are, and no launch."""
import ctypes as ct

import pytest
import torch

from paper_2512_16483_b200 import binding as fv


class OnDevice:
    """A host tensor that says it is on the first device.  Its memory is never used."""
    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def __getitem__(self, which):
        return OnDevice(self.t[which])


def _arrays(B, H, L_cap, D):
    return [torch.zeros((B, H, L_cap, d), dtype=torch.uint8) for d in (D // 2, D // 2, D // 32, D // 32)]


def _cache(arrays):
    return fv.Kv4(*(OnDevice(t) for t in arrays))


@pytest.mark.parametrize("D", [64, 128])
def test_elements_that_share_memory_are_refused(D):
    """An element's distance of 0 is the C structure's word for the default: kernels would step n_heads * L_cap rows, out of the arrays."""
    one = _arrays(1, 2, 16, D)
    for B in (2, 5):
        with pytest.raises(AssertionError):
            _cache([t.expand(B, -1, -1, -1) for t in one])
    with pytest.raises(AssertionError):                  # half of an element apart
        _cache([t.view(-1).as_strided((3, 2, 16, t.shape[3]), (16 * t.shape[3], 16 * t.shape[3], t.shape[3], 1)) for t in _arrays(3, 2, 16, D)])
    assert _cache([t.expand(1, -1, -1, -1) for t in one])._c.elem_stride == 32


def test_elements_apart_are_taken():
    all_ = _arrays(6, 2, 16, 64)
    for which, B, stride in ((slice(None), 6, 32), (slice(1, None, 2), 3, 64), (slice(0, 1), 1, 32), (slice(0, None, 5), 2, 160)):
        kv = _cache([t[which] for t in all_])
        assert (kv.B, kv._c.elem_stride) == (B, stride) and kv._c.k_codes == all_[0][which].data_ptr()
