"""Attention over a cache in 4 bits, every form of launch that this device's rule picks: no key is left out or counted twice, results are within
what each form's own roundings allow, element by element and on average."""
import ctypes as ct

import numpy as np
import pytest
import torch

import kv4_plain as kp
import synth_inputs as si
from helpers import bf16_to_numpy, to_bf16_cuda
from test_gpu_kv4_forms import B200_CLUSTERS, B200_SMS, CASES, FEW, MANY

# Pairs of tiles in six ranges, which have a layout of their own where the ranges meet: 6 x (22 + 22) rows
PAIRS_IN_SIX = [((MANY, 2, 6), shape) for shape in [(1, 17, 1, 129, 10521, 64), (1, 17, 1, 129, 10521, 128), (1, 17, 1, 200, 10521, 128)]]
ONCE = [((MANY, tiles, 0), shape) for tiles, shape in [(2, (2, 2, 1, 9500, 515, 64)), (2, (1, 2, 3, 6340, 390, 128)), (2, (4, 8, 1, 3500, 260, 128))]]
EVERY = CASES + PAIRS_IN_SIX + ONCE                      # key ranges 0: decoded once


class _Plan(ct.Structure):
    _fields_ = [("form", ct.c_int), ("tiles", ct.c_int), ("splits", ct.c_int), ("us", ct.c_float)]


def _plan(B, Hkv, G, r, D, L, sms, clusters):
    from paper_2512_16483_b200 import binding
    fn = binding.load_library()._ZN4fvar18attention_kv4_planEiiiiiiiPKi
    fn.restype, fn.argtypes = _Plan, [ct.c_int] * 7 + [ct.POINTER(ct.c_int)]
    return fn(B, Hkv, G, r, D, L, sms, clusters)


def test_pairs_in_six_ranges_are_what_the_rule_picks():
    for form, (B, Hkv, G, r, L, D) in PAIRS_IN_SIX:
        p = _plan(B, Hkv, G, r, D, L, B200_SMS, (ct.c_int * 7)(*B200_CLUSTERS))
        assert (p.form, p.tiles, p.splits) == form and 5.0 < p.us < 100.0


@pytest.fixture(scope="module")
def fv():
    from paper_2512_16483_b200 import binding
    binding.load_library()
    return binding


@pytest.mark.gpu
def test_this_device_is_launched_as_these_tests_say(fv):
    """The rule with this device's own processors and resident clusters."""
    fn = fv.load_library()._ZN4fvar26attention_kv4_max_clustersEv
    fn.restype, fn.argtypes = ct.POINTER(ct.c_int), []
    clusters, sms = fn(), torch.cuda.get_device_properties(0).multi_processor_count
    here = (sms, tuple(clusters[s] for s in range(7)))
    other = [(form, (p.form, p.tiles, p.splits), shape) for form, shape in CASES + PAIRS_IN_SIX
             for p in [_plan(shape[0], shape[1], shape[2], shape[3], shape[5], shape[4], sms, clusters)] if (p.form, p.tiles, p.splits) != form]
    if other and here != (B200_SMS, B200_CLUSTERS):       # a part with other processors switched off: the results are tested all the same
        pytest.skip("%s processors and clusters: %d shapes are launched in other forms, %s" % (here, len(other), other[:3]))
    assert not other, other[:3]
    for form, (B, Hkv, G, r, L, D) in EVERY:
        kv = fv._Kv4(4096, 4096, 4096, 4096, B, Hkv, D, (L + 7) // 8 * 8, 0)      # asked, not called
        n = fv.load_library().fvar_attention_kv4_workspace(ct.byref(kv), Hkv * G, r, L)
        assert n == (4 * B * Hkv * L * D if form[2] == 0 else 0)


def _cache(fv, x, y):
    """Keys x and values y [B][H][L][D] packed on the host, garbage behind them, and the values it stands for."""
    L, cap, arrays, vals = x.shape[2], (x.shape[2] + 7) // 8 * 8, [], []
    for t in (x, y):
        u, byte = kp.quantise(si.round_to_bf16(t.astype(np.float32)))
        codes, scales = (np.full(t.shape[:2] + (cap, d), 0xFF, np.uint8) for d in (t.shape[3] // 2, t.shape[3] // 32))
        codes[:, :, :L], scales[:, :, :L] = kp.pack(u), byte
        arrays.append((torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()))
        vals.append(kp.values(u, byte))
    return fv.Kv4(arrays[0][0], arrays[1][0], arrays[0][1], arrays[1][1]), vals[0], vals[1]


def _keys_in_places(heads, L, D):
    """Numbers [heads][L][D / 32][32], one 1 in each group of each key and zeros: at place key mod 31 in the groups whose turn it is, at place 31
    in the others.  Places 0 to 30 have few keys each: L / 31, shared out over the groups of all heads."""
    keys, groups = np.arange(L), heads * (D // 32)
    turns = min(groups, max(1, L // 31))
    x = np.zeros((groups, L, 32))
    for g in range(groups):
        x[g, keys, np.where((keys // 31) % turns == g % turns, keys % 31, 31)] = 1.0
    return x.reshape(heads, D // 32, L, 32).transpose(0, 2, 1, 3)


def test_places_hold_few_keys():
    """A key more or less changes a result of places 0 to 30 by more than twice what its rounding may."""
    for _, (B, Hkv, G, r, L, D) in EVERY:
        assert _keys_in_places(B * Hkv, L, D)[..., :31].sum(1).max() < 128


@pytest.mark.gpu
@pytest.mark.parametrize("form,shape", EVERY)
def test_every_key_counts_once(fv, form, shape):
    """Queries of zero: all weights are 1.  Every group of a key has one value v and the scale s = v / 7 of four bits, so that all products and
    sums are whole numbers of s / 16 below 2^24 of them and exact in fp32, in any order.  A result is v x (keys of its place) / (keys seen): off by
    the reciprocal and two products (2^-20 covers them) and by its rounding to bf16, 2^-8."""
    B, Hkv, G, r, L, D = shape
    places = _keys_in_places(B * Hkv, L, D).reshape(B, Hkv, L, D)
    rng = np.random.default_rng(L)
    kv, _, V = _cache(fv, rng.standard_normal(places.shape), 6.5625 * places)
    v = V.max()
    assert np.array_equal(V, v * places) and 15 * 16 * L < 2 ** 24
    q = torch.zeros((B, r, Hkv * G * D), dtype=torch.bfloat16, device="cuda")
    limits = rng.integers(1, L + 1, (B, r))
    limits[:, -1] = L
    counts = np.concatenate([np.zeros((B, Hkv, 1, D)), np.cumsum(places, 2)], 2)
    rows = np.unique(np.concatenate([np.arange(0, r, 1 + r // 400), [r - 1]]))
    for lim in (None, limits):
        n = np.full((B, len(rows)), L) if lim is None else lim[:, rows]
        ref = np.stack([np.repeat(counts[b][:, n[b]].transpose(1, 0, 2), G, 1) for b in range(B)]) * v / n[..., None, None]       # [B][rows][H][D]
        got = fv.fvar_attention_kv4(q, kv, L, None if lim is None else torch.tensor(lim, dtype=torch.int32, device="cuda"))
        got = bf16_to_numpy(got[:, rows]).reshape(ref.shape)
        over = np.abs(got - ref) - (2.0 ** -8 + 2.0 ** -20) * (1 + 2.0 ** -8) * ref
        assert over.max() <= 0, (float(over.max()), np.unravel_index(over.argmax(), over.shape))
    assert fv.kernel_poll_status() == fv.OK


@pytest.mark.gpu
@pytest.mark.parametrize("form,shape", [c for c in EVERY if c[1][0] * c[1][1] * c[1][2] * min(c[1][3], 400) * c[1][4] < 4e7])
def test_errors_are_those_of_the_form(fv, form, shape):
    """Against 64 bits.  Queries are -1, 0 and 1 and keys whole numbers, so that products are exact; a score has the product with log2(e) / sqrt(D)
    and the subtraction of the maximum, 2^-22 of the greatest score in all, and the weight an exp2 of 2^-22.  What is left are the roundings to
    bf16: of the result, and of a weight two in the kernel of few rows and one in that of many, 2^-8 each at most.  Element by element they
    add up.  On average they do not: a rounding is spread evenly over its step or a smaller one, a mean square of at most (2^-8)^2 / 3, and those
    of different weights are independent: mean square at most (2^-16 / 3) (result^2 + roundings x sum (weight x value)^2), to which the
    others come as a whole.  That is asked where there are 60 rows and more to average over."""
    B, Hkv, G, r, L, D = shape
    k = 2 if form[0] == FEW else 1
    rng = np.random.default_rng(7 * r + L)
    keys = rng.integers(-3, 4, (B, Hkv, L, D)).astype(float)
    keys[..., :: 32] = 7.25                              # makes the scale 1, and becomes 7
    kv, K, V = _cache(fv, keys, rng.standard_normal((B, Hkv, L, D)) * np.exp(0.7 * rng.standard_normal(D)))
    assert np.array_equal(K, np.where(keys == 7.25, 7.0, keys))
    q = rng.integers(-1, 2, (B, r, Hkv * G * D)).astype(np.float32)
    rows = np.unique(np.concatenate([np.arange(0, r, 1 + r // 400), [r - 1]]))
    got = bf16_to_numpy(fv.fvar_attention_kv4(to_bf16_cuda(q), kv, L)[:, rows]).astype(np.float64)
    ref, (mag, wide), _ = kp.attention(q[:, rows], K, V, L)
    square, top = np.zeros_like(ref), 0.0
    for b in range(B):
        for h in range(Hkv * G):
            s = q[b, rows, h * D : (h + 1) * D].astype(np.float64) @ K[b, h // G].T / np.sqrt(D)
            top = max(top, np.abs(s).max())
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            square[b, :, h * D : (h + 1) * D] = (w ** 2) @ (V[b, h // G] ** 2)
    one = 2.0 ** -22 * top + 2.0 ** -22                  # relative error of a weight but for the roundings to bf16, and of their sum
    fine = (2.0 ** -16 + 2 * one) * mag + 2 * (L / 8 + 64) * 2.0 ** -23 * wide        # products of two roundings; the weighted sum's steps, see kp.bound
    off = k * 2.0 ** -8 * mag + fine
    over = np.abs(got - ref) / (off + 2.0 ** -8 * (np.abs(ref) + off) + 1e-30)
    main = np.sqrt(2.0 ** -16 / 3 * np.mean(ref ** 2 + k * square))
    allowed = main + np.sqrt(np.mean(fine ** 2))
    rms = np.sqrt(np.mean((got - ref) ** 2))
    print("%s %s: %.3f of the element bound, %.3f of the mean one (%.3f of its roundings), %.4f %% of the results" % (
        form, shape, over.max(), rms / allowed, rms / main, 100 * rms / np.sqrt(np.mean(ref ** 2))))
    assert over.max() <= 1, (float(over.max()), np.unravel_index(over.argmax(), over.shape))
    assert rms <= allowed or B * Hkv * G * len(rows) < 60, (rms, allowed)


@pytest.mark.gpu
@pytest.mark.parametrize("form,shape", PAIRS_IN_SIX)
def test_pairs_in_six_ranges(fv, form, shape):
    """With limits of each row's own, beyond both ends, and rows that see nothing; the same from call to call."""
    B, Hkv, G, r, L, D = shape
    rng = np.random.default_rng(r + D)
    kv, K, V = _cache(fv, rng.standard_normal((B, Hkv, L, D)), rng.standard_normal((B, Hkv, L, D)))
    q = si.round_to_bf16(1.5 * rng.standard_normal((B, r, Hkv * G * D)).astype(np.float32))
    q[:, ::3] *= 4.0
    dev, limits = to_bf16_cuda(q), rng.integers(-5, L + 20, (B, r))
    limits[:, 1::3] = 0
    lim = torch.tensor(limits, dtype=torch.int32, device="cuda")
    got, rows = fv.fvar_attention_kv4(dev, kv, L, lim), np.arange(0, r, 3)
    assert bool((got[torch.tensor(limits <= 0)] == 0).all())
    for _ in range(3):
        assert torch.equal(fv.fvar_attention_kv4(dev, kv, L, lim), got)
    rows = np.unique(np.concatenate([np.arange(0, r, 5), [127, 128, r - 1]]))
    ref, mags, err = kp.attention(q[:, rows], K, V, L, limits[:, rows])
    over = np.abs(bf16_to_numpy(got[:, rows]) - ref) - kp.bound(ref, mags, err, L, D)
    assert not np.isnan(over).any() and over.max() <= 0, float(over.max())
    assert fv.kernel_poll_status() == fv.OK


@pytest.mark.gpu
def test_no_query_rows_are_refused(fv):
    kv = fv.Kv4.empty(2, 3, 40, 64)
    with pytest.raises(fv.FvarError) as e:
        fv.fvar_attention_kv4(torch.empty((2, 0, 192), dtype=torch.bfloat16, device="cuda"), kv, 8)
    assert e.value.status == fv.EINVAL
