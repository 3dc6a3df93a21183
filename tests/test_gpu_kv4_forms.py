"""Attention over a cache in 4 bits in every form that its launch rule has: 8 or 16 rows at a time, lone tiles and pairs of tiles, each in
every number of key ranges, units walked by fewer blocks, and the cache decoded once for many query tiles."""
import ctypes as ct

import numpy as np
import pytest
import torch

import kv4_plain as kp
import synth_inputs as si
from helpers import bf16_to_numpy, to_bf16_cuda

FEW, MANY = 0, 1
B200_SMS, B200_CLUSTERS = 148, (0, 148, 74, 45, 33, 26, 22)


class _Plan(ct.Structure):
    _fields_ = [("form", ct.c_int), ("tiles", ct.c_int), ("splits", ct.c_int)]


def _plan(B, Hkv, G, r, D, L):
    """(form, tiles, key ranges) that the library picks on a B200 (fvar::attention_kv4_plan)."""
    from paper_2512_16483_b200 import binding
    fn = binding.load_library()._ZN4fvar18attention_kv4_planEiiiiiiiPKi
    fn.restype, fn.argtypes = _Plan, [ct.c_int] * 7 + [ct.POINTER(ct.c_int)]
    p = fn(B, Hkv, G, r, D, L, B200_SMS, (ct.c_int * 7)(*B200_CLUSTERS))
    return p.form, p.tiles, p.splits


SHAPES = {  # B, Hkv, G, r, L, for both head widths where the rule picks the same
    (FEW, 1, 1): [(1, 1, 1, 1, 77, 64), (1, 1, 1, 1, 77, 128), (40, 8, 1, 3, 200, 128)],
    (FEW, 1, 2): [(1, 1, 1, 1, 512, 64), (1, 20, 1, 1, 512, 128)],
    (FEW, 1, 3): [(1, 1, 1, 1, 300, 64), (1, 1, 1, 1, 300, 128)],
    (FEW, 1, 4): [(1, 1, 1, 1, 1000, 64), (1, 1, 1, 1, 512, 128)],
    (FEW, 1, 5): [(5, 5, 1, 1, 2100, 64), (5, 5, 1, 1, 2100, 128)],
    (FEW, 1, 6): [(1, 1, 1, 1, 2100, 64), (1, 1, 1, 1, 1500, 128)],
    (FEW, 1, 7): [(2, 5, 1, 1, 6441, 64), (2, 5, 1, 1, 6441, 128)],
    (FEW, 1, 8): [(1, 1, 1, 1, 6441, 64), (1, 1, 1, 1, 3000, 128)],
    (FEW, 2, 1): [(1, 1, 1, 9, 77, 64), (1, 1, 1, 9, 77, 128)],
    (FEW, 2, 2): [(1, 1, 1, 9, 512, 64), (5, 5, 1, 17, 300, 128)],
    (FEW, 2, 3): [(1, 1, 1, 9, 300, 64), (1, 1, 1, 9, 300, 128)],
    (FEW, 2, 4): [(1, 1, 1, 9, 1000, 64), (1, 1, 1, 9, 512, 128)],
    (FEW, 2, 5): [(5, 5, 1, 9, 2100, 64), (5, 5, 1, 9, 2100, 128)],
    (FEW, 2, 6): [(1, 1, 1, 9, 2100, 64), (1, 1, 1, 9, 700, 128)],
    (FEW, 2, 7): [(2, 5, 1, 17, 6441, 64), (2, 5, 1, 17, 6441, 128)],
    (FEW, 2, 8): [(1, 1, 1, 9, 6441, 64), (1, 1, 1, 9, 3000, 128)],
    (MANY, 1, 1): [(1, 1, 1, 65, 77, 64), (1, 1, 1, 65, 77, 128), (12, 30, 1, 70, 260, 64)],
    (MANY, 1, 2): [(2, 30, 1, 33, 1000, 64), (2, 30, 1, 33, 700, 128)],
    (MANY, 1, 3): [(2, 20, 3, 17, 1000, 64), (1, 1, 1, 65, 700, 128)],
    (MANY, 1, 4): [(1, 1, 1, 65, 1000, 64), (1, 1, 1, 65, 1000, 128)],
    (MANY, 1, 5): [(3, 8, 1, 65, 2100, 64), (5, 5, 1, 33, 2100, 128)],
    (MANY, 1, 6): [(1, 1, 1, 65, 2100, 64), (1, 1, 1, 65, 2100, 128)],
    (MANY, 2, 1): [(5, 16, 1, 129, 77, 64), (5, 16, 1, 129, 77, 128), (7, 9, 1, 700, 400, 64), (20, 5, 3, 43, 130, 128)],
    (MANY, 2, 2): [(2, 30, 1, 129, 6441, 64), (2, 30, 1, 129, 6441, 128)],
    (MANY, 2, 3): [(2, 20, 1, 129, 2100, 64), (2, 20, 1, 129, 2100, 128)],
    (MANY, 2, 4): [(1, 30, 1, 129, 6441, 64), (1, 30, 1, 129, 6441, 128)],
    (MANY, 2, 5): [(3, 8, 1, 129, 3000, 64), (3, 8, 1, 129, 3000, 128)],
}
CASES = [(form, shape) for form, shapes in SHAPES.items() for shape in shapes]


def test_the_rule_picks_what_these_tests_say():
    for form, (B, Hkv, G, r, L, D) in CASES:
        assert _plan(B, Hkv, G, r, D, L) == form, (B, Hkv, G, r, D, L)


def test_the_rule_stays_within_what_the_kernels_have():
    for D in (64, 128):
        for groups in (1, 7, 20, 64, 300, 2048):
            for rows in (1, 8, 9, 16, 17, 64, 65, 128, 129, 1000, 5000):
                for L in (0, 1, 100, 128, 129, 1000, 10521, 200000):
                    form, tiles, splits = _plan(groups, 1, 1, rows, D, L)
                    blocks = max(1, -(-L // 128))
                    assert form in (FEW, MANY) and tiles in (1, 2) and 1 <= splits <= (8 if form == FEW else 6)
                    assert splits == 1 or (splits - 1) * -(-blocks // splits) < blocks               # no range without keys
                    assert (form == FEW) if rows <= 8 else (form == MANY or rows <= 64)
                    assert form == MANY or (tiles == 1) == (rows <= 8)


@pytest.fixture(scope="module")
def fv():
    from paper_2512_16483_b200 import binding
    binding.load_library()
    return binding


def _stored(fv, rng, B, H, L, D):
    """A cache with L rows packed on the host, garbage behind them, and the values it stands for."""
    cap, vals, parts = (L + 7) // 8 * 8, [], []
    for _ in range(2):
        x = (rng.standard_normal((B, H, L, D)) * np.exp(0.7 * rng.standard_normal(D))).astype(np.float32)
        u, byte = kp.quantise(si.round_to_bf16(x))
        codes, scales = np.full((B, H, cap, D // 2), 0xFF, np.uint8), np.full((B, H, cap, D // 32), 0xFF, np.uint8)
        codes[:, :, :L], scales[:, :, :L] = kp.pack(u), byte
        parts += [torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()]
        vals.append(kp.values(u, byte))
    return fv.Kv4(parts[0], parts[2], parts[1], parts[3]), vals[0], vals[1]


def _queries(rng, B, r, C):
    q = (1.5 * rng.standard_normal((B, r, C))).astype(np.float32)
    q[:, ::3] *= 4.0                                     # rows whose maximum moves
    return si.round_to_bf16(q)


def _compare(got, q, K, V, L, limits=None):
    ref, mag, err = kp.attention(q, K, V, L, limits)
    over = np.abs(bf16_to_numpy(got) - ref) - kp.bound(ref, mag, err, L, K.shape[3])
    assert not np.isnan(over).any() and over.max() <= 0, (float(over.max()), np.unravel_index(over.argmax(), over.shape))


@pytest.mark.gpu
@pytest.mark.parametrize("form,shape", CASES)
def test_every_form(fv, form, shape):
    """Without limits, then with limits of each row's own, beyond both ends too, and elements whose rows see nothing among the others."""
    B, Hkv, G, r, L, D = shape
    rng = np.random.default_rng(B + 10 * Hkv + 100 * r + L)
    kv, K, V = _stored(fv, rng, B, Hkv, L, D)
    q = _queries(rng, B, r, Hkv * G * D)
    dev = to_bf16_cuda(q)
    rows = np.arange(r) if B * Hkv * G * r * L < 2e7 else np.unique(np.concatenate([np.arange(0, r, 9), np.arange(r - 3, r)]))
    _compare(fv.fvar_attention_kv4(dev, kv, L)[:, rows], q[:, rows], K, V, L)
    limits = rng.integers(-5, L + 20, (B, r))
    limits[1::3] = 0
    lim = torch.tensor(limits, dtype=torch.int32, device="cuda")
    got = fv.fvar_attention_kv4(dev, kv, L, lim)
    _compare(got[:, rows], q[:, rows], K, V, L, limits[:, rows])
    assert bool((got[torch.tensor(limits <= 0)] == 0).all())
    for _ in range(3):                                   # no order of additions depends on timing
        assert torch.equal(fv.fvar_attention_kv4(dev, kv, L, lim), got)
    assert fv.kernel_poll_status() == fv.OK


def _call(fv, q, kv, L, lim, work, nbytes):
    lib, out = fv.load_library(), torch.full_like(q, 7.0)
    D = kv.head_dim
    st = lib.fvar_attention_kv4(q.data_ptr(), q.shape[2], kv._ref, q.shape[2] // D, q.shape[1], L, None if lim is None else lim.data_ptr(),
                                out.data_ptr(), None if work is None else work.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)
    assert st == fv.OK
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hkv,G,r,L,D", [(128, 2, 1, 65, 150, 64), (129, 2, 1, 65, 150, 64), (33, 5, 1, 70, 300, 128), (3, 60, 1, 130, 140, 64), (2, 30, 3, 100, 400, 128)])
@pytest.mark.parametrize("kind", ["shuffled", "equal", "last row sees least", "nothing but one"])
def test_ragged_batches(fv, B, Hkv, G, r, L, D, kind):
    """More units than there are processors: elements are walked by length, each gets its own rows."""
    rng = np.random.default_rng(B + r)
    kv, K, V = _stored(fv, rng, B, Hkv, L, D)
    q = _queries(rng, B, r, Hkv * G * D)
    limits = np.broadcast_to((L * rng.permutation(B) // max(B - 1, 1))[:, None], (B, r)).copy()
    if kind == "equal":
        limits[:] = L - 3
    elif kind == "last row sees least":
        limits[:, -1] = -7
    elif kind == "nothing but one":
        limits[:] = 0
        limits[B // 2] = 2 ** 31 - 1
    got = fv.fvar_attention_kv4(to_bf16_cuda(q), kv, L, torch.tensor(limits, dtype=torch.int32, device="cuda"))
    _compare(got, q, K, V, L, limits)
    assert bool((got[torch.tensor(limits <= 0)] == 0).all())
    assert fv.kernel_poll_status() == fv.OK


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hkv,G,r,L,D", [(2, 2, 1, 9500, 515, 64), (1, 2, 3, 6340, 390, 128), (4, 8, 1, 3500, 260, 128), (4, 8, 1, 8200, 260, 64)])
def test_the_cache_decoded_once(fv, B, Hkv, G, r, L, D):
    """Lone tiles and pairs: with the workspace that the library asks for, with one that is too small (left alone) and without any.  Every
    seventh row is compared, and the last ones; all of them between the calls."""
    rng = np.random.default_rng(r)
    kv, K, V = _stored(fv, rng, B, Hkv, L, D)
    q = _queries(rng, B, r, Hkv * G * D)
    dev = to_bf16_cuda(q)
    n = fv.load_library().fvar_attention_kv4_workspace(kv._ref, Hkv * G, r, L)
    assert n == 4 * B * Hkv * L * D
    rows = np.unique(np.concatenate([np.arange(0, r, 7), np.arange(r - 3, r)]))
    limits = rng.integers(-5, L + 20, (B, r))
    limits[:, 200:1400:3] = 0
    for lim in (None, limits):
        t = None if lim is None else torch.tensor(lim, dtype=torch.int32, device="cuda")
        ref, mag, err = kp.attention(q[:, rows], K, V, L, None if lim is None else lim[:, rows])
        bound = kp.bound(ref, mag, err, L, D)
        work = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        outs = [_call(fv, dev, kv, L, t, work, n - 1)]
        assert bool((work == 0x5A).all())
        outs += [_call(fv, dev, kv, L, t, None, n), _call(fv, dev, kv, L, t, work, n), fv.fvar_attention_kv4(dev, kv, L, t)]
        assert bool((work[n:] == 0x5A).all()) and not bool((work[:n] == 0x5A).all())
        for out in outs:
            over = np.abs(bf16_to_numpy(out[:, rows]) - ref) - bound
            assert not np.isnan(over).any() and over.max() <= 0, float(over.max())
            assert not bool(torch.isnan(out).any()) and (lim is None or bool((out[t <= 0] == 0).all()))
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[2], outs[3])
    assert fv.kernel_poll_status() == fv.OK
    assert fv.load_library().fvar_attention_kv4_workspace(kv._ref, Hkv * G, 64 // G, L) == 0


@pytest.mark.gpu
def test_graphs_and_streams_side_by_side(fv):
    """Two captured graphs, each with a call that takes a workspace, one with ranges and one of a single row, replayed on two streams at
    once, with eager calls between: each gives what it gives alone."""
    rng = np.random.default_rng(9)
    sides, graphs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(2):
        kv, _, _ = _stored(fv, rng, 1, 2, 515, 64)
        qs = [to_bf16_cuda(_queries(rng, 1, r, 128)) for r in (19000, 90, 1)]
        assert fv.load_library().fvar_attention_kv4_workspace(kv._ref, 2, 19000, 515) > 0
        alone = [fv.fvar_attention_kv4(q, kv, 515) for q in qs]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=sides[i]):
            outs = [fv.fvar_attention_kv4(q, kv, 515) for q in qs]
        graphs.append((g, outs, alone, qs, kv))
    torch.cuda.synchronize()
    for _ in range(20):
        for (g, *_), s in zip(graphs, sides):
            with torch.cuda.stream(s):
                g.replay()
        for _, _, alone, qs, kv in graphs:
            assert torch.equal(fv.fvar_attention_kv4(qs[1], kv, 515), alone[1])
    torch.cuda.synchronize()
    for _, outs, alone, _, _ in graphs:
        for a, b in zip(outs, alone):
            assert torch.equal(a, b)
    assert fv.kernel_poll_status() == fv.OK


@pytest.mark.gpu
@pytest.mark.parametrize("r", [1, 12, 70, 300])
def test_queries_of_any_magnitude(fv, r):
    """Rows from 2^-100 to 2^60: powers of two that the kernel multiplies by cancel."""
    rng = np.random.default_rng(r)
    B, H, D, L = 1, 2, 128, 300
    kv, K, V = _stored(fv, rng, B, H, L, D)
    q = si.round_to_bf16(rng.standard_normal((B, r, H * D)).astype(np.float32))
    base = bf16_to_numpy(fv.fvar_attention_kv4(to_bf16_cuda(q), kv, L))
    for e in (-100, -40, 60):
        got = fv.fvar_attention_kv4(to_bf16_cuda((q * np.float32(2.0 ** e)).astype(np.float32)), kv, L)
        assert not bool(torch.isnan(got).any())
        ref, mag, err = kp.attention(q.astype(np.float64) * 2.0 ** e, K, V, L)
        if e < 0:
            _compare(got, q.astype(np.float64) * 2.0 ** e, K, V, L)
        else:                                            # one weight is 1, the others 0: which one is beyond doubt unless two scores are close
            s = np.abs(bf16_to_numpy(got) - ref) - 2.0 ** -8 * np.abs(ref) - 1e-30
            assert (s <= 0).mean() > 0.999
    assert np.isfinite(base).all()


@pytest.mark.gpu
def test_calls_without_rows(fv):
    kv = fv.Kv4.empty(2, 3, 40, 64)
    none = torch.empty((2, 0, 192), dtype=torch.bfloat16, device="cuda")
    fv.fvar_kv4_write(kv, none, none, 40)
    K, V = fv.fvar_kv4_read(kv, 0, 40)
    assert K.shape == V.shape == (2, 0, 192)
    assert fv.fvar_kv4_read(kv, 0, 3, out=(none, none))[0] is none
    with pytest.raises(Exception):
        fv.fvar_attention_kv4(none, kv, 8)
