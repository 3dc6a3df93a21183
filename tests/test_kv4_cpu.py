"""The cache in 4 bits without a GPU: the format's definition, and the calls that are refused before anything is launched."""
import ctypes as ct

import numpy as np
import pytest

import kv4_plain as kp
import synth_inputs as si


def test_format_is_within_half_a_step_and_exact_in_bf16():
    rng = np.random.default_rng(1)
    x = si.round_to_bf16((rng.standard_normal((200, 128)) * np.exp(4 * rng.standard_normal((200, 1)))).astype(np.float32))
    u, byte = kp.quantise(x)
    v = kp.values(u, byte)
    step = np.repeat(kp.SCALES[byte], kp.GROUP, -1)
    top = np.abs(x.reshape(200, 4, 32)).max(-1)
    inside = top <= 28800                                # the format's range; what is beyond takes 7 at the greatest scale
    assert np.all((np.abs(v - x) <= step / 2)[np.repeat(inside, 32, -1)]) and u.min() >= 1 and u.max() <= 15
    assert np.all((7.5 * kp.SCALES[byte] >= top)[inside]) and np.all((7.5 * kp.SCALES[np.maximum(byte, 1) - 1] < top)[byte > 0])
    assert np.array_equal(kp.unpack(kp.pack(u)), u)
    every = kp.values(np.tile(np.arange(16, dtype=np.uint8), (256, 2)), np.arange(256, dtype=np.uint8)[:, None])
    assert np.array_equal(si.round_to_bf16(every.astype(np.float32)).astype(np.float64), every)


def test_zero_nan_and_infinity():
    x = np.zeros((4, 64))
    x[1, 3], x[1, 40] = np.nan, -2.0
    x[2, 5], x[2, 6] = -np.inf, 1.0
    x[3, 7] = 1e30
    u, byte = kp.quantise(x)
    v = kp.values(u, byte)
    assert np.all(v[0] == 0) and np.all(byte[0] == 0)
    assert v[1, 3] == 0 and abs(v[1, 40] + 2.0) <= 0.15
    assert v[2, 5] == -7 * 3840.0 and v[2, 6] == 0 and v[3, 7] == 7 * 3840.0


P = 4096                                              # an address that is never used: only refused calls are made


def _cache(**over):
    from paper_2512_16483_b200 import binding
    f = {"k_codes": P, "v_codes": P, "k_scales": P, "v_scales": P, "B": 2, "n_heads": 4, "head_dim": 64, "L_cap": 40, "elem_stride": 0}
    f.update(over)
    return ct.byref(binding._Kv4(**f))


BAD_CACHES = [{"k_codes": None}, {"v_codes": None}, {"k_scales": None}, {"v_scales": None}, {"k_codes": P + 8}, {"v_codes": P + 4},
              {"k_scales": P + 2}, {"v_scales": P + 1}, {"B": 0}, {"n_heads": 0}, {"head_dim": 32}, {"head_dim": 96}, {"L_cap": 36}, {"L_cap": 0},
              {"elem_stride": 152}, {"elem_stride": 161}, {"elem_stride": -160}]
GOOD = {"fvar_kv4_write": (P, P, 256, 3, 0, None, None, None), "fvar_kv4_read": (3, 0, None, None, P, P, None),
        "fvar_attention_kv4": (P, 512, None, 8, 3, 40, None, P, P, 0, None)}


def _call(name, args, cache):
    from paper_2512_16483_b200 import binding
    args = list(args)
    if name == "fvar_attention_kv4":
        args[2] = cache
    else:
        args.insert(0, cache)
    return getattr(binding.load_library(), name)(*args)


@pytest.mark.parametrize("name", sorted(GOOD))
def test_bad_caches_are_refused(name):
    from paper_2512_16483_b200 import binding
    for over in BAD_CACHES:
        assert _call(name, GOOD[name], _cache(**over)) == binding.EINVAL, over
        assert b"kv4" in binding.load_library().fvar_last_error(None)
    assert _call(name, GOOD[name], None) == binding.EINVAL


@pytest.mark.parametrize("name,vary", [
    ("fvar_kv4_write", {0: (None, P + 8), 1: (None, P + 4), 2: (248, 260, 0), 3: (-1, 41), 4: (-1, 38)}),
    ("fvar_kv4_read", {0: (-1, 41), 1: (-1, 38), 4: (None, P + 8), 5: (None, P + 2)}),
    ("fvar_attention_kv4", {0: (None, P + 8), 1: (504, 516), 3: (0, -4, 6), 4: (0, -1), 5: (-1, 41), 7: (None, P + 8), 8: (P + 8,)}),
])
def test_bad_arguments_are_refused(name, vary):
    from paper_2512_16483_b200 import binding
    for pos, bad in vary.items():
        for v in bad:
            args = list(GOOD[name])
            args[pos] = v
            assert _call(name, args, _cache()) == binding.EINVAL, (pos, v)


def test_no_rows_is_no_work():
    from paper_2512_16483_b200 import binding
    assert _call("fvar_kv4_write", (P, P, 256, 0, 40, None, None, None), _cache()) == binding.OK
    assert _call("fvar_kv4_read", (0, 0, None, None, P, P, None), _cache()) == binding.OK


def test_binding_refuses_host_tensors():
    import torch
    from paper_2512_16483_b200 import binding as fv
    t = [torch.zeros((1, 2, 8, d), dtype=torch.uint8) for d in (32, 32, 2, 2)]
    with pytest.raises(AssertionError):
        fv.Kv4(*t)


def test_no_rows_are_nothing():
    """Tensors without elements have no address."""
    from paper_2512_16483_b200 import binding
    lib = binding.load_library()
    for L0 in (0, 7, 40):
        assert lib.fvar_kv4_write(_cache(), None, None, 256, 0, L0, None, None, None) == binding.OK
        assert lib.fvar_kv4_read(_cache(), 0, L0, None, None, None, None, None) == binding.OK
    assert lib.fvar_kv4_write(_cache(), None, None, 256, 0, 41, None, None, None) == binding.EINVAL
    assert lib.fvar_kv4_read(_cache(), 0, -1, None, None, None, None, None) == binding.EINVAL


def test_more_elements_or_heads_than_a_grid_has():
    from paper_2512_16483_b200 import binding
    lib = binding.load_library()
    assert lib.fvar_attention_kv4(P, 512, _cache(B=65536), 8, 1, 40, None, P, None, 0, None) == binding.EUNSUPPORTED
    assert lib.fvar_attention_kv4(P, 64 * 65536, _cache(n_heads=65536), 65536, 1, 40, None, P, None, 0, None) == binding.EUNSUPPORTED
