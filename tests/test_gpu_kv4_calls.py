"""Calls of the cache in 4 bits at the edges of what they allow, in every kind of launch."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import kv4_plain as kp
import synth_inputs as si
from helpers import bf16_to_numpy, to_bf16_cuda

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# r, L and whether the cache is decoded once for them: few rows on one range and several, lone tiles and pairs, alone and in ranges
LAUNCHES = [(1, 77), (3, 3000), (12, 77), (12, 3000), (70, 77), (70, 2100), (300, 140), (129, 6441), (9500, 515)]


@pytest.fixture(scope="module")
def fv():
    from paper_2512_16483_b200 import binding
    binding.load_library()
    return binding


def _stored(fv, x, y):
    """A cache of keys x and values y [B][H][L][D] packed on the host, garbage behind them, and the values it stands for."""
    B, H, L, D = x.shape
    cap, arrays, vals = (L + 7) // 8 * 8, [], []
    for t in (x, y):
        u, byte = kp.quantise(si.round_to_bf16(t.astype(np.float32)))
        codes, scales = np.full((B, H, cap, D // 2), 0xFF, np.uint8), np.full((B, H, cap, D // 32), 0xFF, np.uint8)
        codes[:, :, :L], scales[:, :, :L] = kp.pack(u), byte
        arrays.append((torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()))
        vals.append(kp.values(u, byte))
    return fv.Kv4(arrays[0][0], arrays[1][0], arrays[0][1], arrays[1][1]), vals[0], vals[1]


@pytest.mark.parametrize("r,L", LAUNCHES)
@pytest.mark.parametrize("D", [64, 128])
def test_a_row_whose_scores_are_all_minus_infinity_is_nan(fv, r, L, D):
    """Keys of one sign and a query element of the other that is infinite: softmax of nothing but minus infinity is NaN, as for every other
    row with an infinity.  Finite elements whose products pass fp32: NaN, or an average of the values seen where the kernel has scaled the
    row, but never 0.  A row that sees no key stays 0, its neighbours what they are."""
    B, H = 1, 2
    rng = np.random.default_rng(r + L)
    kv, _, V = _stored(fv, 0.5 + rng.random((B, H, L, D)), rng.standard_normal((B, H, L, D)))
    q = to_bf16_cuda(si.round_to_bf16(rng.standard_normal((B, r, H * D)).astype(np.float32)))
    limits = torch.full((B, r), L, dtype=torch.int32, device="cuda")
    limits[0, r // 2 + 1 :] = 1
    if r > 2:
        limits[0, 1] = 0
    want = fv.fvar_attention_kv4(q, kv, L, limits)
    bad = q.clone()
    bad[0, r // 2, 5] = float("-inf")                    # head 0
    bad[0, r - 1, D : 2 * D] = -3.0e38                   # head 1
    if r > 2:
        bad[0, 1, 3] = float("-inf")                     # sees nothing
    got = fv.fvar_attention_kv4(bad, kv, L, limits).view(r, H, D)
    assert fv.kernel_poll_status() == fv.OK
    nan = torch.isnan(got).all(-1).cpu()
    expect = torch.zeros((r, H), dtype=torch.bool)
    expect[r // 2, 0] = int(limits[0, r // 2]) > 0
    others = torch.ones((r, H), dtype=torch.bool)
    others[r - 1, 1] = False
    assert torch.equal(nan[others], expect[others]), torch.nonzero((nan != expect) & others)[:8]
    others &= ~expect
    assert torch.equal(got.cpu()[others], want.view(r, H, D).cpu()[others])
    seen, far = V[0, 1, : int(limits[0, r - 1])], bf16_to_numpy(got[r - 1, 1])
    off = 2.0 ** -7 * np.abs(seen).max(0)                # weights and the result rounded to bf16
    assert bool(nan[r - 1, 1]) or np.all((far >= seen.min(0) - off) & (far <= seen.max(0) + off))


@pytest.mark.parametrize("r,L", [c for c in LAUNCHES if c[0] <= 12])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [100, 112, 125])
def test_few_rows_of_the_largest_queries(fv, r, L, D, power):
    """Queries up to the end of bf16: one weight is 1, the others are 0, also where a product in fp32 would be infinite.  Keys with the greatest
    scales and the least ones.  Rows whose two greatest scores are within 2^-9 of the greatest sum of magnitudes are left out: twice what a score
    may be off by, 2^-14 of 16 / 7 x such a sum for the sums of queries and (D + 8) 2^-23 of it for the rest."""
    B, H = 2, 2
    rng = np.random.default_rng(r + L + power)
    keys = rng.standard_normal((B, H, L, D)) * np.where(np.arange(L) % 2, 8000.0, 2.0 ** -19)[:, None]
    kv, K, V = _stored(fv, keys, rng.standard_normal((B, H, L, D)))
    q = si.round_to_bf16((np.clip(rng.standard_normal((B, r, H * D)), -3, 3) * 2.0 ** power).astype(np.float32))
    got = bf16_to_numpy(fv.fvar_attention_kv4(to_bf16_cuda(q), kv, L)).reshape(B, r, H, D)
    assert fv.kernel_poll_status() == fv.OK and np.isfinite(got).all()
    looked = 0
    for b in range(B):
        for h in range(H):
            x = q[b, :, h * D : (h + 1) * D].astype(np.float64)
            s, far = x @ K[b, h].T, (np.abs(x) @ np.abs(K[b, h]).T).max(-1)
            best = np.sort(s, -1)
            for i in np.nonzero(best[:, -1] - best[:, -2] > 2.0 ** -9 * far)[0]:
                want = V[b, h, s[i].argmax()]
                assert np.all(np.abs(got[b, i, h] - want) <= 2.0 ** -7 * np.abs(want))        # the weight and the result, a rounding each at most
                looked += 1
    assert looked >= B * H * r // 2


@pytest.mark.parametrize("native", [True, False])
def test_attention_where_memory_for_a_workspace_is_short_or_declined(fv, monkeypatch, native):
    """98 MB of workspace that the allocator may not take, or is not asked for: the call runs as the library does without one."""
    B, H, D, L, r = 4, 16, 128, 3000, 3500
    kv = fv.Kv4.empty(B, H, L, D)
    rows = torch.randn((B, L, H * D), device="cuda").bfloat16()
    fv.fvar_kv4_write(kv, rows, rows.flip(1), 0)
    q = torch.randn((B, r, H * D), device="cuda").bfloat16()
    lib = fv.load_library()
    n = lib.fvar_attention_kv4_workspace(kv._ref, H, r, L)
    assert n == 4 * B * H * L * D
    without = torch.empty_like(q)
    assert lib.fvar_attention_kv4(q.data_ptr(), H * D, kv._ref, H, r, L, None, without.data_ptr(), None, 0, torch.cuda.current_stream().cuda_stream) == fv.OK
    out = torch.zeros_like(q)
    del rows
    if not native:
        monkeypatch.setattr(fv, "_native", lambda: type("None_", (), {"attention_kv4": staticmethod(lambda *a: None)}))
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = torch.cuda.memory_allocated()

    def peak():                                          # since the last look at it (a comparison takes memory too)
        top = torch.cuda.max_memory_allocated()
        same = torch.equal(out, without)
        out.zero_()
        torch.cuda.empty_cache()
        torch.cuda.reset_peak_memory_stats()
        return top - before, same

    torch.cuda.reset_peak_memory_stats()
    assert fv.fvar_attention_kv4(q, kv, L, out=out, workspace=False) is out
    assert peak() == (0, True)
    free, total = torch.cuda.mem_get_info()
    torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + n // 2) / total)
    try:
        assert fv.fvar_attention_kv4(q, kv, L, out=out) is out
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert peak() == (0, True)
    fv.fvar_attention_kv4(q, kv, L, out=out)
    assert peak()[0] >= n
    assert fv.kernel_poll_status() == fv.OK


FIRST_CALLS = """
import threading
import torch
from paper_2512_16483_b200 import binding as fv
fv.load_library(), fv._native()
torch.manual_seed(0)
kv = fv.Kv4.empty(2, 4, 515, 64)
rows = torch.randn(2, 515, 256, device="cuda").bfloat16()
fv.fvar_kv4_write(kv, rows, rows.flip(1), 0)
qs = [torch.randn(2, r, 256, device="cuda").bfloat16() for r in (1, 12, 70, 130, 9500, 1, 12, 70)]
torch.cuda.synchronize()
gate, outs = threading.Barrier(len(qs)), [None] * len(qs)
def work(i):
    with torch.cuda.stream(torch.cuda.Stream()):
        gate.wait()
        outs[i] = [fv.fvar_attention_kv4(qs[i], kv, 515) for _ in range(20)]
threads = [threading.Thread(target=work, args=(i,)) for i in range(len(qs))]
[t.start() for t in threads], [t.join() for t in threads]
torch.cuda.synchronize()
for q, several in zip(qs, outs):
    alone = fv.fvar_attention_kv4(q, kv, 515)
    assert all(torch.equal(o, alone) for o in several)
assert fv.kernel_poll_status() == fv.OK
print("same")
"""


def test_first_calls_from_several_threads():
    """A fresh process, whose first calls of every form come at once, each on a stream of its own: each gives what it gives alone."""
    p = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout == "same\n", (p.stdout, p.stderr[-3000:])


FIRST_CALLS_CAPTURED = """
import torch
from paper_2512_16483_b200 import binding as fv
torch.manual_seed(0)
D, H, L = %d, 2, 515
rows = torch.randn(1, L, H * D, device="cuda").bfloat16()
kv, at, lim = fv.Kv4.empty(1, H, 520, D), torch.tensor([3], dtype=torch.int32, device="cuda"), None
qs = [torch.randn(1, r, H * D, device="cuda").bfloat16() for r in (1, 12, 70, 300, 19000)]
back = tuple(torch.zeros_like(rows) for _ in range(2))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    fv.fvar_kv4_write(kv, rows, rows, at)
    fv.fvar_kv4_read(kv, L, at, out=back)
    outs = [fv.fvar_attention_kv4(q, kv, L + 3) for q in qs]
for _ in range(2):
    rows.normal_()
    for t in (kv.k_codes, kv.v_codes, kv.k_scales, kv.v_scales):
        t.zero_()
    graph.replay()
    eager = fv.Kv4.empty(1, H, 520, D)
    for t in (eager.k_codes, eager.v_codes, eager.k_scales, eager.v_scales):
        t.zero_()
    fv.fvar_kv4_write(eager, rows, rows, 3)
    assert torch.equal(fv.fvar_kv4_read(eager, L, 3)[1], back[1])
    for q, o in zip(qs, outs):
        assert torch.equal(fv.fvar_attention_kv4(q, eager, L + 3), o)
assert fv.kernel_poll_status() == fv.OK
print("same")
"""


@pytest.mark.parametrize("D", [64, 128])
def test_first_calls_are_captured(D):
    """A fresh process whose first calls of every form come inside a capture: nothing that they set up belongs to a stream."""
    p = subprocess.run([sys.executable, "-c", FIRST_CALLS_CAPTURED % D], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout == "same\n", (p.stdout, p.stderr[-3000:])
