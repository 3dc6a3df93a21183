"""The cache in 4 bits on the GPU: rows written, read back and attended to, against plain numpy in 64 bits (kv4_plain.py)."""
import numpy as np
import pytest
import torch

import kv4_plain as kp
import synth_inputs as si
from helpers import bf16_to_numpy, to_bf16_cuda, weights_to_cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fv():
    from paper_2512_16483_b200 import binding
    binding.load_library()
    return binding


def _rows(rng, *shape):
    return si.round_to_bf16((rng.standard_normal(shape) * np.exp(0.7 * rng.standard_normal(shape[-1]))).astype(np.float32))


def _kv4(fv, B, H, L_cap, D, fill=0xA5):
    return fv.Kv4(*(torch.full((B, H, L_cap, d), fill, dtype=torch.uint8, device="cuda") for d in (D // 2, D // 2, D // 32, D // 32)))


def _stored(fv, rng, B, H, L, L_cap, D, fill=0xFF):
    """A cache with L rows packed on the host, garbage behind them, and the values it stands for."""
    kv, vals = _kv4(fv, B, H, L_cap, D, fill), []
    for codes, scales in ((kv.k_codes, kv.k_scales), (kv.v_codes, kv.v_scales)):
        u, byte = kp.quantise(_rows(rng, B, H, L, D))
        codes[:, :, :L] = torch.from_numpy(kp.pack(u)).cuda()
        scales[:, :, :L] = torch.from_numpy(byte).cuda()
        vals.append(kp.values(u, byte))
    return kv, vals[0], vals[1]


def _heads(x, H):
    """[B][n][H * D] -> [B][H][n][D]."""
    B, n, C = x.shape
    return x.reshape(B, n, H, C // H).transpose(0, 2, 1, 3)


# ----------------------------------------------------------------------------- rows

@pytest.mark.parametrize("B,H,D,n,cap,at", [
    (1, 1, 64, 1, 8, 7), (2, 16, 128, 1, 24, 0), (3, 5, 64, 17, 40, 3), (2, 3, 128, 100, 104, 4), (1, 30, 64, 257, 680, 423), (4, 2, 128, 9, 16, 0)])
@pytest.mark.parametrize("fused", [False, True])
def test_rows_written_and_read_back(fv, B, H, D, n, cap, at, fused):
    rng = np.random.default_rng(n + D)
    C = H * D
    qkv = _rows(rng, B, n, 3 * C)
    dev = to_bf16_cuda(qkv)
    K, V = dev[..., C : 2 * C], dev[..., 2 * C :]
    if not fused:
        K, V = K.contiguous(), V.contiguous()
    kv = _kv4(fv, B, H, cap, D)
    fv.fvar_kv4_write(kv, K, V, at)
    Ko, Vo = fv.fvar_kv4_read(kv, n, at)
    assert fv.kernel_poll_status() == fv.OK
    for codes, scales, got, x in ((kv.k_codes, kv.k_scales, Ko, qkv[..., C : 2 * C]), (kv.v_codes, kv.v_scales, Vo, qkv[..., 2 * C :])):
        u, byte = kp.quantise(_heads(x, H))
        assert np.array_equal(codes[:, :, at : at + n].cpu().numpy(), kp.pack(u))
        assert np.array_equal(scales[:, :, at : at + n].cpu().numpy(), byte)
        assert np.array_equal(_heads(bf16_to_numpy(got), H), kp.values(u, byte))
        for t in (codes, scales):                            # rows before and behind stay
            assert bool((t[:, :, :at] == 0xA5).all()) and bool((t[:, :, at + n :] == 0xA5).all())


def test_every_bf16_number(fv):
    """All 65536 patterns: once beside numbers like themselves, once shuffled (infinities and NaN among the rest)."""
    bits = np.arange(65536, dtype=np.uint32)
    for seed in (None, 3):
        b = bits if seed is None else np.random.default_rng(seed).permutation(bits)
        x = (b << 16).astype(np.uint32).view(np.float32).reshape(1, 512, 128)
        t = torch.from_numpy(b.astype(np.uint16).view(np.int16).reshape(1, 512, 128)).view(torch.bfloat16).cuda()
        kv = _kv4(fv, 1, 1, 512, 128)
        fv.fvar_kv4_write(kv, t, t, 0)
        u, byte = kp.quantise(x)
        assert np.array_equal(kv.k_scales[0, 0].cpu().numpy(), byte[0])
        assert np.array_equal(kp.unpack(kv.v_codes[0, 0].cpu().numpy()), u[0])


def test_every_step_of_every_scale(fv):
    """Each bf16 number within a factor of 100 of one as the maximum of a group, with smaller ones at and around the halves."""
    tops = np.arange(0x3C80, 0x42C8, dtype=np.uint32)
    top = (tops << 16).view(np.float32).astype(np.float64)
    g = np.zeros((len(top), 32))
    byte = np.searchsorted(7.5 * kp.SCALES, top)
    for j in range(15):
        g[:, 2 * j] = kp.SCALES[byte] * (j // 2 + 0.5) * (-1) ** j                      # halves (exact in bf16 up to 7.5)
        g[:, 2 * j + 1] = g[:, 2 * j] * (1 + (0.0078125 if j % 3 else -0.0078125))
    g = np.where(np.abs(g) > top[:, None], 0.0, g)
    g[:, 31] = top
    x = si.round_to_bf16(g.astype(np.float32))
    x = np.concatenate([x, np.zeros((-len(x) % 4, 32), np.float32)]).reshape(1, -1, 128)
    n = x.shape[1]
    kv = _kv4(fv, 1, 1, (n + 7) // 8 * 8, 128)
    fv.fvar_kv4_write(kv, to_bf16_cuda(x), to_bf16_cuda(-x), 0)
    for codes, scales, y in ((kv.k_codes, kv.k_scales, x), (kv.v_codes, kv.v_scales, -x)):
        u, b = kp.quantise(y)
        assert np.array_equal(scales[0, 0, :n].cpu().numpy(), b[0])
        assert np.array_equal(kp.unpack(codes[0, 0, :n].cpu().numpy()), u[0])


def test_ragged_rows_leave_the_others_alone(fv):
    B, H, D, n, cap = 6, 2, 64, 37, 64
    rng = np.random.default_rng(11)
    K, V = _rows(rng, B, n, H * D), _rows(rng, B, n, H * D)
    start, count = [0, 5, 27, 63, 1, 20], [0, 37, 37, 1, -3, 99]              # counts beyond [0, n] are its ends
    real = np.clip(count, 0, n)
    kv = _kv4(fv, B, H, cap, D)
    st, cn = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (start, count))
    fv.fvar_kv4_write(kv, to_bf16_cuda(K), to_bf16_cuda(V), st, cn)
    Ko, Vo = (torch.full((B, n, H * D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fv.fvar_kv4_read(kv, n, st, cn, out=(Ko, Vo))
    assert fv.kernel_poll_status() == fv.OK
    zeros = fv.fvar_kv4_read(kv, n, st, cn)[0]
    for b in range(B):
        s, c = start[b], real[b]
        for codes, got, x in ((kv.k_codes, Ko, K), (kv.v_codes, Vo, V)):
            u, byte = kp.quantise(_heads(x[b : b + 1, :c], H)) if c else (None, None)
            if c:
                assert np.array_equal(codes[b, :, s : s + c].cpu().numpy(), kp.pack(u)[0])
                assert np.array_equal(_heads(bf16_to_numpy(got[b : b + 1, :c]), H), kp.values(u, byte))
            rest = torch.ones(cap, dtype=torch.bool)
            rest[s : s + c] = False
            assert bool((codes[b, :, rest.cuda()] == 0xA5).all()) and bool((got[b, c:] == 7.0).all())
        assert bool((zeros[b, c:] == 0).all())


def test_rows_outside_the_cache_are_skipped_and_reported(fv):
    B, H, D, n, cap = 3, 2, 128, 10, 16
    rng = np.random.default_rng(12)
    K, V = _rows(rng, B, n, H * D), _rows(rng, B, n, H * D)
    start = [-4, 12, 2 ** 31 - 3]
    st = torch.tensor(start, dtype=torch.int32, device="cuda")
    kv = _kv4(fv, B, H, cap, D)
    fv.fvar_kv4_write(kv, to_bf16_cuda(K), to_bf16_cuda(V), st)
    assert fv.kernel_poll_status() == fv.EINVAL and fv.kernel_poll_status() == fv.OK
    Ko, Vo = (torch.full((B, n, H * D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fv.fvar_kv4_read(kv, n, st, out=(Ko, Vo))
    assert fv.kernel_poll_status() == fv.EINVAL and fv.kernel_poll_status() == fv.OK
    for b in range(B):
        for i in range(n):
            there = 0 <= start[b] + i < cap
            for codes, got, x in ((kv.k_codes, Ko, K), (kv.v_codes, Vo, V)):
                if there:
                    u, byte = kp.quantise(_heads(x[b : b + 1, i : i + 1], H))
                    assert np.array_equal(codes[b, :, start[b] + i].cpu().numpy(), kp.pack(u)[0, :, 0])
                    assert np.array_equal(_heads(bf16_to_numpy(got[b : b + 1, i : i + 1]), H), kp.values(u, byte))
                else:
                    assert bool((got[b, i] == 7.0).all())
        rest = [p for p in range(cap) if not 0 <= p - start[b] < n]
        assert bool((kv.k_codes[b, :, rest] == 0xA5).all())


# ----------------------------------------------------------------------------- attention

def _check(fv, q, kv, K, V, L, limits=None, q_dev=None, out=None):
    got = fv.fvar_attention_kv4(to_bf16_cuda(q) if q_dev is None else q_dev, kv, L,
                                None if limits is None else torch.tensor(np.asarray(limits), dtype=torch.int32, device="cuda"), out=out)
    assert fv.kernel_poll_status() == fv.OK
    ref, mag, err = kp.attention(q, K, V, L, limits)
    over = np.abs(bf16_to_numpy(got) - ref) - kp.bound(ref, mag, err, L, K.shape[3])
    assert not np.isnan(over).any() and over.max() <= 0, (float(over.max()), np.unravel_index(over.argmax(), over.shape))
    return got


@pytest.mark.parametrize("B,Hkv,G,D,r,L", [
    (1, 1, 1, 64, 1, 1), (1, 1, 1, 128, 1, 1), (2, 16, 1, 128, 1, 300), (1, 2, 1, 64, 1, 10521), (3, 2, 4, 128, 1, 1000), (2, 1, 7, 64, 2, 129),
    (1, 3, 1, 128, 16, 640), (2, 2, 1, 64, 17, 127), (1, 2, 3, 128, 5, 513), (1, 1, 8, 64, 33, 255), (5, 30, 1, 64, 85, 509), (2, 3, 1, 128, 128, 128),
    (1, 2, 1, 128, 129, 1031), (1, 4, 1, 64, 256, 680), (3, 2, 2, 128, 200, 391), (1, 2, 1, 128, 410, 2931), (40, 8, 1, 64, 3, 77), (12, 16, 1, 64, 169, 424),
    (1, 1, 32, 128, 40, 384), (2, 1, 3, 64, 100, 1500), (1, 2, 1, 128, 1600, 300), (2, 16, 1, 128, 26, 2547), (1, 40, 1, 64, 257, 1030)])
def test_attention(fv, B, Hkv, G, D, r, L):
    rng = np.random.default_rng(B * 1000 + r * 10 + L)
    kv, K, V = _stored(fv, rng, B, Hkv, L, (L + 7) // 8 * 8, D)
    q = si.round_to_bf16((1.5 * rng.standard_normal((B, r, Hkv * G * D))).astype(np.float32))
    q[:, ::3] *= 4.0                                     # rows whose maximum moves
    first = _check(fv, q, kv, K, V, L)
    again = fv.fvar_attention_kv4(to_bf16_cuda(q), kv, L)
    assert torch.equal(first, again)                     # no order of additions depends on timing


@pytest.mark.parametrize("B,Hkv,G,D,r,L,mask", [
    (4, 2, 1, 128, 1, 900, "lengths"), (6, 3, 4, 64, 1, 3000, "lengths"), (3, 2, 2, 64, 40, 700, "lengths"), (2, 2, 1, 128, 300, 600, "causal"),
    (2, 4, 1, 64, 385, 385, "scales"), (1, 2, 1, 128, 260, 1300, "random"), (2, 2, 1, 64, 13, 200, "random"), (1, 1, 5, 128, 30, 4000, "random"),
    (2, 2, 1, 128, 5, 300, "none_seen"), (2, 2, 1, 64, 300, 300, "none_seen"), (1, 1, 1, 64, 150, 5000, "first_key"), (2, 2, 1, 128, 70, 6000, "late_rows")])
def test_attention_masks(fv, B, Hkv, G, D, r, L, mask):
    rng = np.random.default_rng(r + L)
    kv, K, V = _stored(fv, rng, B, Hkv, L, (L + 7) // 8 * 8, D)
    q = si.round_to_bf16((1.5 * rng.standard_normal((B, r, Hkv * G * D))).astype(np.float32))
    if mask == "lengths":
        limits = np.repeat(np.linspace(0, L, B).astype(int)[:, None], r, 1)
    elif mask == "causal":
        limits = np.tile(L - r + 1 + np.arange(r), (B, 1))
    elif mask == "scales":
        ends = np.cumsum([s * s for s in (1, 2, 3, 4, 5, 6, 8, 10, 13)])
        limits = np.tile([ends[np.searchsorted(ends, i, side="right")] if i < ends[-1] else L for i in range(r)], (B, 1))
    elif mask == "random":
        limits = rng.integers(-5, L + 20, (B, r))                        # beyond both ends too
    elif mask == "none_seen":
        limits = np.zeros((B, r), int)
    elif mask == "first_key":
        limits = np.ones((B, r), int)
    else:                                                # rows that end in the first keys beside rows that see them all
        limits = np.where(np.arange(r) % 5 == 0, L, 3)[None].repeat(B, 0)
    got = _check(fv, q, kv, K, V, L, limits)
    assert bool((got[torch.tensor(limits <= 0)] == 0).all())


def test_attention_over_nothing(fv):
    kv = _kv4(fv, 2, 2, 16, 64, 0xFF)
    q = torch.full((2, 3, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    for r in (1, 3):
        assert bool((fv.fvar_attention_kv4(q[:, :r].contiguous(), kv, 0) == 0).all())
    long = torch.full((2, 300, 128), 1.0, dtype=torch.bfloat16, device="cuda")
    assert bool((fv.fvar_attention_kv4(long, kv, 0) == 0).all())
    assert fv.kernel_poll_status() == fv.OK


@pytest.mark.parametrize("r,L", [(1, 500), (20, 500), (200, 500)])
def test_rows_of_a_wider_matrix_elements_of_a_larger_cache_and_an_output_given(fv, r, L):
    B, Hkv, G, D = 3, 2, 2, 64
    rng = np.random.default_rng(r)
    C = Hkv * G * D
    both, K, V = _stored(fv, rng, 2 * B, Hkv, L, 504, D)
    wide = si.round_to_bf16(rng.standard_normal((B, r, C + 2 * Hkv * D)).astype(np.float32))
    out = torch.full((B + 2, r, C), 7.0, dtype=torch.bfloat16, device="cuda")
    _check(fv, np.ascontiguousarray(wide[..., :C]), both.elements(slice(1, None, 2)), K[1::2], V[1::2], L, q_dev=to_bf16_cuda(wide)[..., :C], out=out[1:-1])
    assert bool((out[0] == 7.0).all()) and bool((out[-1] == 7.0).all())         # nothing in front of it or behind it


@pytest.mark.parametrize("r", [3, 40, 300])
def test_a_row_of_nan_or_infinity_is_alone(fv, r):
    B, H, D, L = 1, 2, 128, 700
    rng = np.random.default_rng(r)
    kv, K, V = _stored(fv, rng, B, H, L, 704, D)
    q = si.round_to_bf16(rng.standard_normal((B, r, H * D)).astype(np.float32))
    want = fv.fvar_attention_kv4(to_bf16_cuda(q), kv, L)
    t = to_bf16_cuda(q)
    t[0, 1, 5] = float("nan")
    t[0, r - 1, D + 3] = float("inf")
    got = fv.fvar_attention_kv4(t, kv, L)
    assert fv.kernel_poll_status() == fv.OK
    same = torch.ones((r, H), dtype=torch.bool)
    same[1, 0] = same[r - 1, 1] = False
    a, b = got.view(r, H, D).cpu(), want.view(r, H, D).cpu()
    assert torch.equal(a[same], b[same]) and bool(torch.isnan(a[1, 0]).all()) and bool(torch.isnan(a[r - 1, 1]).all())


@pytest.mark.parametrize("r", [1, 100])
def test_scores_far_apart(fv, r):
    """Scores of several hundreds, the greatest one last and first: every weight but a few is zero, sums stay finite."""
    B, H, D, L = 2, 2, 64, 1000
    rng = np.random.default_rng(r)
    kv, K, V = _stored(fv, rng, B, H, L, 1000, D)
    q = si.round_to_bf16((60.0 * rng.standard_normal((B, r, H * D))).astype(np.float32))
    _check(fv, q, kv, K, V, L)


def test_a_cache_of_more_than_4_gb(fv):
    """Element 1 begins 2^26 + 8 rows behind element 0: its codes are beyond 32 bits of bytes."""
    B, H, D, L, cap, gap = 2, 2, 128, 130, 136, 2 ** 26 + 8
    rng = np.random.default_rng(5)
    small, K, V = _stored(fv, rng, B, H, L, cap, D, 0)
    arrays = []
    for t in (small.k_codes, small.v_codes, small.k_scales, small.v_scales):
        d = t.shape[3]
        base = torch.empty((gap + H * cap) * d, dtype=torch.uint8, device="cuda")
        view = base.as_strided((B, H, cap, d), (gap * d, cap * d, d, 1))
        view.copy_(t)
        arrays.append(view)
    big = fv.Kv4(*arrays)
    for r in (1, 40, 200):
        q = to_bf16_cuda(si.round_to_bf16(rng.standard_normal((B, r, H * D)).astype(np.float32)))
        assert torch.equal(fv.fvar_attention_kv4(q, big, L), fv.fvar_attention_kv4(q, small, L))
    for a, b in zip(fv.fvar_kv4_read(big, L, 0), fv.fvar_kv4_read(small, L, 0)):
        assert torch.equal(a, b)
    rows = to_bf16_cuda(_rows(rng, B, 3, H * D))
    for c in (big, small):
        fv.fvar_kv4_write(c, rows, rows, 131)
    assert torch.equal(big.k_codes, small.k_codes) and torch.equal(big.v_scales, small.v_scales)
    assert fv.kernel_poll_status() == fv.OK


# ----------------------------------------------------------------------------- together

def test_scales_written_one_after_the_other_and_attended_to(fv):
    """A generation's use: every scale's rows quantised behind the earlier ones, then its queries over all of them; a last step
    of the null-prompt branches alone.  The same on another stream, and captured into a graph that is replayed on new inputs."""
    B, H, D, sides = 4, 3, 64, (1, 2, 3, 5, 8, 13)
    rng = np.random.default_rng(21)
    C, total = H * D, sum(s * s for s in sides)
    qkv = [si.round_to_bf16(rng.standard_normal((B, s * s, 3 * C)).astype(np.float32)) for s in sides]

    def generate(cache, inputs):
        outs, at = [], 0
        for x in inputs:
            n = x.shape[1]
            fv.fvar_kv4_write(cache, x[..., C : 2 * C], x[..., 2 * C :], at)
            at += n
            outs.append(fv.fvar_attention_kv4(x[..., :C], cache, at))
        null = cache.elements(slice(1, None, 2))
        outs.append(fv.fvar_attention_kv4(inputs[-1][1::2, :, :C].contiguous(), null, at))
        return outs

    dev = [to_bf16_cuda(x) for x in qkv]
    cache = fv.Kv4.empty(B, H, total, D)
    outs = generate(cache, dev)
    assert fv.kernel_poll_status() == fv.OK
    K, V = (np.concatenate([kp.values(*kp.quantise(_heads(x[..., i * C : (i + 1) * C], H))) for x in qkv], 2) for i in (1, 2))
    at = 0
    for x, got in zip(qkv, outs):
        at += x.shape[1]
        ref, mag, err = kp.attention(x[..., :C], K, V, at)
        assert np.all(np.abs(bf16_to_numpy(got) - ref) <= kp.bound(ref, mag, err, at, D))
    assert torch.equal(outs[-1], outs[-2][1::2])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = generate(fv.Kv4.empty(B, H, total, D), dev)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(other, outs):
        assert torch.equal(a, b)

    held = [torch.zeros_like(x) for x in dev]
    graph_cache = fv.Kv4.empty(B, H, total, D)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = generate(graph_cache, held)
    for scale in (1.0, 0.5, 1.0):
        for h, x in zip(held, dev):
            h.copy_(x * scale)
        graph.replay()
        want = outs if scale == 1.0 else generate(cache, [x * scale for x in dev])
        for a, b in zip(captured, want):
            assert torch.equal(a, b)
    assert fv.kernel_poll_status() == fv.OK


def test_one_token_at_a_time(fv):
    """Rows appended at places of their own (a batch of sequences of different lengths), one token each, then attended to."""
    B, Hkv, G, D, cap = 5, 2, 4, 128, 208
    rng = np.random.default_rng(31)
    lens = np.array([0, 1, 63, 127, 200])
    kv = _kv4(fv, B, Hkv, cap, D, 0xFF)
    K, V = _rows(rng, B, cap, Hkv * D), _rows(rng, B, cap, Hkv * D)
    fv.fvar_kv4_write(kv, to_bf16_cuda(K), to_bf16_cuda(V), 0, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    Kq, Vq = (kp.values(*kp.quantise(_heads(x, Hkv))) for x in (K, V))
    for step in range(4):
        at = torch.tensor(lens + step, dtype=torch.int32, device="cuda")
        k, v = (np.stack([x[b, lens[b] + step] for b in range(B)])[:, None] for x in (K, V))
        fv.fvar_kv4_write(kv, to_bf16_cuda(k), to_bf16_cuda(v), at)
        q = si.round_to_bf16(rng.standard_normal((B, 1, Hkv * G * D)).astype(np.float32))
        _check(fv, q, kv, Kq, Vq, cap, (lens + step + 1)[:, None])


def test_rows_read_back_are_what_the_step_takes(fv):
    """A prefix kept in 4 bits is loaded into a context (fvar_load_kv) and a step runs over it: the same as from the values."""
    shp, B = si.shape_tiny(n_blocks=2, scales=(1, 2, 3, 4)), 2
    Ms, H, D = shp.tokens_per_scale(), shp.n_heads, shp.head_dim
    L = sum(Ms[:3])
    weights = weights_to_cuda(si.make_weights(5, shp))
    K, V = si.make_kv_prefill(5, 2, B, L, shp.width)
    results = []
    for packed in (True, False):
        ctx = fv.Fvar(weights, blocks_per_group=1, n_heads=H, head_dim=D, ffn_dim=shp.ffn_dim, scale_hw=shp.hw(), max_batch=B)
        ctx.set_cond(to_bf16_cuda(si.make_cond(5, B, shp.width)))
        if packed:
            rows = []
            for blk in range(2):
                kv = fv.Kv4.empty(B, H, L, D)
                fv.fvar_kv4_write(kv, to_bf16_cuda(K[blk]), to_bf16_cuda(V[blk]), 0)
                rows.append(fv.fvar_kv4_read(kv, L, 0))
            k, v = (torch.stack([x[i] for x in rows]) for i in (0, 1))
        else:
            k, v = (to_bf16_cuda(np.stack([kp.values(*kp.quantise(_heads(x[blk], H))).transpose(0, 2, 1, 3).reshape(B, L, shp.width)
                                           for blk in range(2)]).astype(np.float32)) for x in (K, V))
        ctx.load_kv(k, v)
        results.append(ctx.scale_step(to_bf16_cuda(si.make_tokens(6, B, Ms[3], shp.width)), 3))
        assert ctx.poll_status() == fv.OK
    assert torch.equal(results[0], results[1])


def test_binding_refuses(fv):
    kv = _kv4(fv, 2, 2, 16, 64)
    q = torch.zeros((2, 3, 128), dtype=torch.bfloat16, device="cuda")
    lim = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    rows = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device="cuda")
    good = torch.zeros(2, dtype=torch.int32, device="cuda")
    for call in (lambda: fv.fvar_attention_kv4(q.float(), kv, 4), lambda: fv.fvar_attention_kv4(q[:1], kv, 4), lambda: fv.fvar_attention_kv4(q, kv, 4, lim.long()),
                 lambda: fv.fvar_attention_kv4(q, kv, 4, lim[:, :2]), lambda: fv.fvar_attention_kv4(q.cpu(), kv, 4), lambda: fv.fvar_attention_kv4(q, kv, 4, out=q.float()),
                 lambda: fv.fvar_attention_kv4(q.transpose(0, 1).contiguous().transpose(0, 1), kv, 4),
                 lambda: fv.fvar_kv4_write(kv, rows, rows[:, :3], 0), lambda: fv.fvar_kv4_write(kv, rows[..., :64], rows[..., :64], 0),
                 lambda: fv.fvar_kv4_write(kv, rows, rows, good.long()), lambda: fv.fvar_kv4_write(kv, rows, rows, 0, good[:1]),
                 lambda: fv.fvar_kv4_read(kv, 4, 0, out=(rows, rows[:, :3])),
                 lambda: fv.Kv4(kv.k_codes, kv.v_codes, kv.k_scales, kv.v_scales[:, :, :8]), lambda: fv.Kv4(kv.k_codes, kv.v_codes, kv.k_scales.int(), kv.v_scales)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: fv.fvar_attention_kv4(q, kv, 17), lambda: fv.fvar_attention_kv4(q, kv, -1), lambda: fv.fvar_kv4_write(kv, rows, rows, 13),
                 lambda: fv.fvar_kv4_read(kv, 4, -1), lambda: fv.fvar_attention_kv4(torch.zeros((2, 3, 192), dtype=torch.bfloat16, device="cuda"), kv, 4)):
        with pytest.raises(fv.FvarError) as e:
            call()
        assert e.value.status == fv.EINVAL
