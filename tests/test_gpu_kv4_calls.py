"""Calls of the cache in 4 bits at the edges of what they allow, in every kind of launch."""
import numpy as np
import pytest
import torch

import kv4_plain as kp
import synth_inputs as si
from helpers import bf16_to_numpy, to_bf16_cuda

pytestmark = pytest.mark.gpu

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
