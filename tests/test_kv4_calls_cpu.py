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


FAR = (2 ** 32, 2 ** 32 + 3, 2 ** 31, -2 ** 32 + 1, 2 ** 63, -2 ** 70)


class Recorder:
    """The library's functions, which take their arguments as ctypes converts them and launch nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        real = getattr(fv_lib, name)

        def call(*args):
            self.calls.append((name, [a if t is not ct.c_int else ct.c_int(a).value for t, a in zip(real.argtypes, args)]))
            return 0
        return call


fv_lib = fv.load_library()


@pytest.fixture
def recorded(monkeypatch):
    """The general way of every call, with the library's functions recorded."""
    rec = Recorder()
    monkeypatch.setattr(fv, "load_library", lambda: rec)
    monkeypatch.setattr(fv, "_native", lambda: type("None_", (), {n: staticmethod(lambda *a: None) for n in ("kv4_write", "kv4_read", "attention_kv4")}))
    monkeypatch.setattr(fv, "_current", lambda device: None)
    monkeypatch.setattr(fv, "_stream", lambda: 0)
    return rec


def _bf16(*shape):
    return OnDevice(torch.zeros(shape, dtype=torch.bfloat16))


@pytest.mark.parametrize("far", FAR)
def test_numbers_beyond_32_bits_are_not_cut(recorded, far):
    """What reaches the library is outside every cache, as the number that was given is."""
    kv, rows = _cache(_arrays(2, 2, 16, 64)), _bf16(2, 3, 128)
    fv.fvar_kv4_write(kv, rows, rows, far)
    fv.fvar_kv4_read(kv, 3, far, out=(rows, rows))
    fv.fvar_attention_kv4(rows, kv, far, out=_bf16(2, 3, 128))
    L0s = [recorded.calls[0][1][5], recorded.calls[1][1][2]]
    Ls = [a[5] for n, a in recorded.calls if n == "fvar_attention_kv4"] + [a[3] for n, a in recorded.calls if n == "fvar_attention_kv4_workspace"]
    assert [n for n, _ in recorded.calls] == ["fvar_kv4_write", "fvar_kv4_read", "fvar_attention_kv4_workspace", "fvar_attention_kv4"]
    for v in L0s + Ls:
        assert (v > 2 ** 30) if far > 0 else (v < 0), v
    # and the library refuses them (no rows: nothing would be launched)
    for L0 in L0s:
        assert fv_lib.fvar_kv4_write(ct.byref(fv._Kv4(4096, 4096, 4096, 4096, 2, 2, 64, 16, 0)), None, None, 128, 0, L0, None, None, None) == fv.EINVAL


def test_positions_are_whole_numbers(recorded):
    kv, rows = _cache(_arrays(2, 2, 16, 64)), _bf16(2, 3, 128)
    for bad in (3.7, "3", None):
        for call in (lambda: fv.fvar_kv4_write(kv, rows, rows, bad), lambda: fv.fvar_kv4_read(kv, 3, bad, out=(rows, rows)),
                     lambda: fv.fvar_attention_kv4(rows, kv, bad, out=_bf16(2, 3, 128))):
            with pytest.raises(TypeError):
                call()
    assert not recorded.calls
    import numpy as np
    fv.fvar_kv4_write(kv, rows, rows, np.int64(5))
    assert recorded.calls[0][1][5] == 5


def test_elements_are_never_copied():
    """A list of elements would index copies, and rows written to them would be lost."""
    kv = _cache(_arrays(4, 2, 16, 64))
    for which in ([0, 2], (0, 2), torch.tensor([0, 2]), torch.tensor([True, False, True, False]), 1, None):
        with pytest.raises(TypeError):
            kv.elements(which)
    some = kv.elements(slice(1, None, 2))
    assert some.B == 2 and some.v_scales.data_ptr() == kv.v_scales[1].data_ptr()


def test_no_elements_or_heads_are_refused():
    for shape in ((0, 2, 16, 64), (2, 0, 16, 64), (2, 2, 0, 64)):
        with pytest.raises(AssertionError):
            _cache(_arrays(*shape))
    with pytest.raises(AssertionError):
        _cache(_arrays(4, 2, 16, 64)).elements(slice(4, None))
    for D in (16, 32, 96, 256):
        with pytest.raises(AssertionError):
            _cache(_arrays(2, 2, 16, D))


class Wants(Recorder):
    """A library that would like a workspace."""

    def __getattr__(self, name):
        call = super().__getattr__(name)
        return call if name != "fvar_attention_kv4_workspace" else lambda *a: (call(*a), 4096)[1]


def _attend_where_no_workspace_is_to_be_had(monkeypatch, **how):
    rec, asked, real = Wants(), [], torch.empty
    monkeypatch.setattr(fv, "load_library", lambda: rec)

    def empty(*shape, dtype=None, device=None):
        asked.append((shape, dtype))
        if dtype == torch.uint8:
            raise torch.OutOfMemoryError("CUDA out of memory")
        return OnDevice(real(*shape, dtype=dtype))
    monkeypatch.setattr(torch, "empty", empty)
    kv, q = _cache(_arrays(2, 2, 16, 64)), _bf16(2, 3, 128)
    out = fv.fvar_attention_kv4(q, kv, 16, **how)
    assert tuple(out.shape) == (2, 3, 128)
    (name, args), = [c for c in rec.calls if c[0] == "fvar_attention_kv4"]
    assert args[8] is None and args[9] == 0              # no address, no bytes
    return [shape for shape, dtype in asked if dtype == torch.uint8]


def test_attention_without_memory_for_a_workspace(recorded, monkeypatch):
    """The workspace makes a call faster and is not needed for it."""
    assert _attend_where_no_workspace_is_to_be_had(monkeypatch) == [(4096,)]


def test_a_workspace_can_be_declined(recorded, monkeypatch):
    assert _attend_where_no_workspace_is_to_be_had(monkeypatch, workspace=False) == []
