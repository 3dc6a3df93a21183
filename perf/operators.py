"""The cache in 4 bits, as cases that can be timed and compared: rows quantised as they are written, read back, attended to.

Three kinds:
  store   rows of keys and values written into the cache and read back (fvar_kv4_write, fvar_kv4_read)
  load    rows of a cache that is there read back as bf16 (fvar_kv4_read)
  attend  query rows over the cache (fvar_attention_kv4)

The plain form below is the definition of the format and of the three operators in elementary torch operations.

Format: a row of a head has D values in groups of 32.  A group has a scale s = (1 + m / 8) 2^(e - 20), kept as the byte
8 e + m, and 32 numbers u of 4 bits, 1 to 15; the values are (u - 8) s.  s is the least scale with 7.5 s >= max |x|.  Eight
values are a 32-bit word: value 2p at bits 4p, value 2p + 1 at bits 16 + 4p.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32
INFINITY_SIDES = (1, 2, 4, 6, 8, 12, 16, 20, 24, 32, 40, 48, 64)
VAR_SIDES = (1, 2, 3, 4, 5, 6, 8, 10, 13, 16)


def listed():
    return [
        # the first token of a generation: one row for each branch of a CFG pair, launches only
        {"name": "store_first_token_b2", "kind": "store", "B": 2, "H": 16, "D": 128, "n": 1, "cap": 10521, "ragged": False, "fused": True},
        # the rows of the 40 x 40 scale, cut out of the fused QKV product, behind the 2521 rows of the scales before
        {"name": "store_40x40_b2", "kind": "store", "B": 2, "H": 16, "D": 128, "n": 1600, "cap": 10521, "ragged": False, "fused": True},
        # a padded batch whose elements stand at different places: VAR-d30, up to 256 rows each
        {"name": "store_ragged_d30_b32", "kind": "store", "B": 32, "H": 30, "D": 64, "n": 256, "cap": 680, "ragged": True, "fused": False},
        # a generation that was put away before its last scale, taken up again
        {"name": "load_infinity_b2", "kind": "load", "B": 2, "H": 16, "D": 128, "n": 6425, "cap": 10521, "ragged": False},
        # the finished caches of 64 images, of different lengths, zero among them
        {"name": "load_ragged_d16_b64", "kind": "load", "B": 64, "H": 16, "D": 64, "n": 680, "cap": 680, "ragged": True},
        # a single row over the whole cache of every scale: nothing but reading it
        {"name": "attend_row_b2", "kind": "attend", "B": 2, "H": 16, "kv": 16, "D": 128, "r": 1, "L": 10521, "mask": "none", "halves": False},
        # the smallest rank of the last scale's table, null-prompt branches alone out of a cache of both
        {"name": "attend_r16_null_b4", "kind": "attend", "B": 4, "H": 16, "kv": 16, "D": 128, "r": 16, "L": 6441, "mask": "none", "halves": True},
        # 64 sequences of lengths from nothing to 8191, four query heads to a head of the cache, a token each
        {"name": "attend_token_grouped_b64", "kind": "attend", "B": 64, "H": 32, "kv": 8, "D": 128, "r": 1, "L": 8191, "mask": "ragged", "halves": False},
        # half of the rows of the 13 x 13 scale of VAR-d30 over what was there and themselves
        {"name": "attend_r85_d30_b32", "kind": "attend", "B": 32, "H": 30, "kv": 30, "D": 64, "r": 85, "L": 509, "mask": "none", "halves": False},
        # the largest rank of the 40 x 40 scale's table
        {"name": "attend_r410_b2", "kind": "attend", "B": 2, "H": 16, "kv": 16, "D": 128, "r": 410, "L": 2931, "mask": "none", "halves": False},
        # every scale of VAR-d16 in one call, each row up to the end of its own scale
        {"name": "attend_scales_d16_b16", "kind": "attend", "B": 16, "H": 16, "kv": 16, "D": 64, "r": 680, "L": 680, "mask": "scales", "halves": False},
        # the last scale without approximation: the largest attention there is
        {"name": "attend_64x64_b2", "kind": "attend", "B": 2, "H": 16, "kv": 16, "D": 128, "r": 4096, "L": 10521, "mask": "none", "halves": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    kind = rng.choice(("store", "load", "attend", "attend", "attend", "attend"))
    D = rng.choice((64, 128))
    if kind != "attend":
        n = _log(rng, 1, 10521)
        case = {"kind": kind, "B": _log(rng, 1, 64), "H": _log(rng, 1, 32), "D": D, "n": n, "cap": max(n, _log(rng, 1, 10521)),
                "ragged": rng.random() < 0.4}
        if kind == "store":
            case["fused"] = rng.random() < 0.5
        return case
    kv = _log(rng, 1, 32)
    group = rng.choice((1, 1, 1, 2, 3, 4, 7, 8))
    mask = rng.choice(("none", "none", "ragged", "scales"))
    r, L = _log(rng, 1, 4096), _log(rng, 1, 10521)
    if mask == "scales":
        L = max(L, r)                             # the rows are those of the last scales, earlier ones stand before them
    return {"kind": kind, "B": _log(rng, 1, 64), "H": kv * group, "kv": kv, "D": D, "r": r, "L": L, "mask": mask, "halves": rng.random() < 0.2}


def draw(rng):
    top = {}
    for c in listed():
        w, t = work(c), top.setdefault(c["kind"] == "attend", {"bytes": 0.0, "flops": 0.0})
        t.update({k: max(t[k], w[k]) for k in t})
    while True:
        case = _draw_once(rng)
        w, t = work(case), top[case["kind"] == "attend"]
        if w["flops"] <= t["flops"] and w["bytes"] <= t["bytes"]:
            return case


# ------------------------------------------------------------------------------------------------ sizes of a case

def _spans(case):
    """Per element: the first cache row and how many of the n rows there are."""
    B, n, cap = case["B"], case["n"], case["cap"]
    if not case["ragged"]:
        return [cap - n if case["kind"] == "store" and n < cap - n else 0] * B, [n] * B
    counts = [n * b // max(B - 1, 1) for b in range(B)]            # from none to all of them
    return [(cap - c) * (B - b) // (2 * B) for b, c in enumerate(counts)], counts


def _limits(case):
    """Per element: the keys that each row sees, or None."""
    B, r, L = case["B"], case["r"], case["L"]
    if case["mask"] == "ragged":
        return [[L * b // max(B - 1, 1)] * r for b in range(B)]
    if case["mask"] == "scales":
        rows, end, i = [], L - r, 0                              # whole scales in order, the last one cut at r rows
        while len(rows) < r:
            take = min(VAR_SIDES[min(i, len(VAR_SIDES) - 1)] ** 2, r - len(rows))
            end, i = end + take, i + 1
            rows += [end] * take
        return [rows] * B
    return None


def work(case):
    B, D = case["B"], case["D"]
    if case["kind"] != "attend":
        values = 2.0 * sum(_spans(case)[1]) * case["H"] * D
        packed = values * (0.5 + 1.0 / GROUP)
        # written: rows read, codes and scales written; read back: those read, rows written
        return {"bytes": (2.0 * values + 2.0 * packed + 2.0 * values) if case["kind"] == "store" else packed + 2.0 * values,
                "flops": (8.0 if case["kind"] == "store" else 2.0) * values}
    limits = _limits(case)
    seen = [max(x) for x in limits] if limits else [case["L"]] * B
    pairs = sum(sum(x) for x in limits) if limits else B * case["r"] * case["L"]
    return {"bytes": 4.0 * B * case["r"] * case["H"] * D + 2.0 * sum(seen) * case["kv"] * D * (0.5 + 1.0 / GROUP)
            + (4.0 * B * case["r"] if limits else 0.0), "flops": 4.0 * pairs * case["H"] * D}


# ------------------------------------------------------------------------------------------------ the format, in plain torch

def _quantise(x):
    """x fp32 [..., D] -> codes uint8 [..., D / 2], scales uint8 [..., D / 32]."""
    g = x.unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    m, e = torch.frexp(top / torch.full_like(top, 7.5))          # a division (by a number it would be a product with 1 / 7.5)
    scale = ((e + 19) * 8 + torch.ceil(m * 16).int() - 8).clamp(0, 255)       # m in [1/2, 1): 16 m rounded up has four bits
    scale = torch.where(top > 0, scale, torch.zeros_like(scale))
    q = torch.floor(g.abs() / _scale(scale).unsqueeze(-1) + 0.5).clamp_(max=7.0)
    u = (torch.where(g < 0, -q, q) + 8.0).to(torch.uint8).flatten(-2).unflatten(-1, (-1, 8))
    word = torch.stack((u[..., 0] | u[..., 2] << 4, u[..., 4] | u[..., 6] << 4, u[..., 1] | u[..., 3] << 4, u[..., 5] | u[..., 7] << 4), -1)
    return word.flatten(-2), scale.to(torch.uint8)


def _scale(byte):
    # 2^(e - 20) (1 + m / 8) as the bits of an fp32 number
    return ((byte.int() + (107 << 3)) << 20).view(torch.float32)


def _values(codes, scales):
    """codes uint8 [..., D / 2], scales uint8 [..., D / 32] -> fp32 [..., D]."""
    b = codes.unflatten(-1, (-1, 4))
    lo, hi = b & 15, b >> 4
    u = torch.stack((lo[..., 0], lo[..., 2], hi[..., 0], hi[..., 2], lo[..., 1], lo[..., 3], hi[..., 1], hi[..., 3]), -1)
    v = (u.flatten(-2).float() - 8.0).unflatten(-1, (-1, GROUP))
    return (v * _scale(scales).unsqueeze(-1)).flatten(-2)


# ------------------------------------------------------------------------------------------------ inputs

def _randn(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)


def _rows(g, *shape):
    """Rows of keys or values: some channels much larger than the rest, as projections of normalised rows have them."""
    size = torch.exp(0.7 * torch.randn(shape[-1], generator=g, device="cuda"))
    return (torch.randn(shape, generator=g, device="cuda") * size).to(torch.bfloat16)


def _filled(g, B, H, cap, D):
    """A cache whose rows are all there: (k_codes, v_codes, k_scales, v_scales)."""
    parts = {k: [] for k in ("kc", "vc", "ks", "vs")}
    for _ in range(B):
        for name in "kv":
            c, s = _quantise(_rows(g, H, cap, D).float())
            parts[name + "c"].append(c)
            parts[name + "s"].append(s)
    return tuple(torch.stack(parts[k]) for k in ("kc", "vc", "ks", "vs"))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, B, D = case["kind"], case["B"], case["D"]
    state = {"kind": kind}
    if kind == "attend":
        L, kv, r, H = case["L"], case["kv"], case["r"], case["H"]
        limits = _limits(case)
        cap = (L + 127) // 128 * 128
        state.update(L=L, heads=H, q=_randn(g, B, r, H * D, std=1.5),
                     limits=None if limits is None else torch.tensor(limits, dtype=torch.int32, device="cuda"))
        cache = _filled(g, 2 * B if case["halves"] else B, kv, cap, D)
        state["cache"] = tuple(t[1::2] for t in cache) if case["halves"] else cache     # elements 2p + 1: the null prompts
        return state
    n, H = case["n"], case["H"]
    cap = (case["cap"] + 7) // 8 * 8
    start, count = _spans(case)
    state.update(n=n, K_out=torch.zeros((B, n, H * D), dtype=torch.bfloat16, device="cuda"),
                 V_out=torch.zeros((B, n, H * D), dtype=torch.bfloat16, device="cuda"))
    if case["ragged"]:
        state["start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
        state["count"] = torch.tensor(count, dtype=torch.int32, device="cuda")
    else:
        state["start"], state["count"] = start[0], None
    if kind == "load":
        state["cache"] = _filled(g, B, H, cap, D)
        return state
    state["cache"] = tuple(torch.zeros((B, H, cap, d), dtype=torch.uint8, device="cuda") for d in (D // 2, D // 2, D // GROUP, D // GROUP))
    if case["fused"]:
        state["K"], state["V"] = _rows(g, B, n, 3 * H * D).split(H * D, -1)[1:]
    else:
        state["K"], state["V"] = _rows(g, B, n, H * D), _rows(g, B, n, H * D)
    return state


# ------------------------------------------------------------------------------------------------ passes

def _places(state):
    """(element, row of the n, cache row) of every row that is there."""
    n, B = state["n"], state["K_out"].shape[0]
    i = torch.arange(n, device="cuda").expand(B, n)
    b = torch.arange(B, device="cuda").unsqueeze(1).expand(B, n)
    if state["count"] is None:
        return b.reshape(-1), i.reshape(-1), (i + state["start"]).reshape(-1)
    there = i < state["count"].unsqueeze(1)
    return b[there], i[there], (i + state["start"].unsqueeze(1))[there]


def _plain_store(state):
    kc, vc, ks, vs = state["cache"]
    H, D = kc.shape[1], 2 * kc.shape[3]
    b, i, at = _places(state)
    for rows, codes, scales in ((state["K"], kc, ks), (state["V"], vc, vs)):
        c, s = _quantise(rows[b, i].float().unflatten(-1, (H, D)))
        codes[b, :, at], scales[b, :, at] = c, s


def _plain_load(state):
    kc, vc, ks, vs = state["cache"]
    b, i, at = _places(state)
    for out, codes, scales in ((state["K_out"], kc, ks), (state["V_out"], vc, vs)):
        out[b, i] = _values(codes[b, :, at], scales[b, :, at]).flatten(1).to(torch.bfloat16)


def _plain_attend(state):
    kc, vc, ks, vs = state["cache"]
    q, L, H, limits = state["q"], state["L"], state["heads"], state["limits"]
    B, r, _ = q.shape
    kv, D = kc.shape[1], 2 * kc.shape[3]
    G = H // kv
    out = torch.empty_like(q)
    rows = max(1, (1 << 28) // max(1, H * L))                    # scores of at most 1 GB at a time
    for b in range(B):
        K, V = _values(kc[b, :, :L], ks[b, :, :L]), _values(vc[b, :, :L], vs[b, :, :L])
        for i in range(0, r, rows):
            x = q[b, i : i + rows].float().unflatten(-1, (kv, G, D)).permute(1, 2, 0, 3)
            s = torch.matmul(x.flatten(1, 2), K.transpose(1, 2)).unflatten(1, (G, -1)) / math.sqrt(D)
            if limits is not None:
                seen = torch.arange(L, device="cuda") < limits[b, i : i + rows].unsqueeze(1)
                s = s.masked_fill(~seen, -math.inf)
            top = s.amax(-1, keepdim=True).clamp_min(-1e30)      # a row that sees nothing: every weight is 0
            p = torch.exp(s - top)
            o = torch.matmul(p.flatten(1, 2), V).unflatten(1, (G, -1)) / p.sum(-1, keepdim=True).clamp_min(1e-30)
            out[b, i : i + rows] = o.permute(2, 0, 1, 3).flatten(1).to(torch.bfloat16)
    return out


def run(state):
    kind = state["kind"]
    if own:
        from paper_2512_16483_b200 import binding as fv
        if "kv4" not in state:
            state["kv4"] = fv.Kv4(*state["cache"])               # the handle that a program keeps beside its cache
        kv4 = state["kv4"]
        if kind == "attend":
            return fv.fvar_attention_kv4(state["q"], kv4, state["L"], state["limits"])
        if kind == "store":
            fv.fvar_kv4_write(kv4, state["K"], state["V"], state["start"], state["count"])
        return fv.fvar_kv4_read(kv4, state["n"], state["start"], state["count"], out=(state["K_out"], state["V_out"]))
    if kind == "attend":
        return _plain_attend(state)
    if kind == "store":
        _plain_store(state)
    _plain_load(state)
    return state["K_out"], state["V_out"]


# ------------------------------------------------------------------------------------------------ from the definition, in 64 bits

def _grid():
    """Every scale that there is, in order."""
    return torch.tensor([(8 + c % 8) * 2.0 ** (c // 8 - 23) for c in range(256)], dtype=torch.float64, device="cuda")


def _exact_round_trip(x):
    """What the cache gives back for rows x [..., D]."""
    v = x.double().reshape(*x.shape[:-1], -1, GROUP)
    grid = _grid()
    at = torch.searchsorted(7.5 * grid, v.abs().max(-1).values).clamp(max=255)
    s = grid[at][..., None]
    return (torch.sign(v) * torch.minimum(torch.floor(v.abs() / s + 0.5), torch.full_like(s, 7.0)) * s).reshape(x.shape)


def _exact_values(codes, scales):
    """The values that codes [..., D / 2] and scales [..., D / 32] stand for."""
    byte = codes.long().reshape(*codes.shape[:-1], -1, 4)
    word = byte[..., 0] + byte[..., 1] * 256 + byte[..., 2] * 65536 + byte[..., 3] * 16777216
    v = torch.stack([(word // 2 ** (4 * (j // 2) + 16 * (j % 2))) % 16 - 8 for j in range(8)], -1)
    v = v.reshape(*codes.shape[:-1], -1, GROUP).double()
    return (v * _grid()[scales.long()][..., None]).reshape(*codes.shape[:-1], -1)


def _exact_attend(case, state):
    q, L, limits = state["q"], state["L"], _limits(case)
    B, r = q.shape[:2]
    H, kv, D = case["H"], case["kv"], case["D"]
    kc, vc, ks, vs = state["cache"]
    out = torch.zeros((B, r, H, D), dtype=torch.float64, device="cuda")
    key = torch.arange(L, device="cuda")
    for b in range(B):
        lim = None if limits is None else torch.tensor(limits[b], device="cuda")
        for h in range(kv):
            K, V = _exact_values(kc[b, h, :L], ks[b, h, :L]), _exact_values(vc[b, h, :L], vs[b, h, :L])
            for head in range(h * (H // kv), (h + 1) * (H // kv)):
                s = q[b, :, head * D : (head + 1) * D].double() @ K.T * D ** -0.5
                if lim is not None:
                    s[key[None, :] >= lim[:, None]] = -math.inf
                w = torch.exp(s - s.max(-1, keepdim=True).values)
                w = w / w.sum(-1, keepdim=True)
                if lim is not None:
                    w[lim <= 0] = 0.0
                out[b, :, head] = w @ V
    return out.reshape(B, r, H * D)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "attend":
        return None if work(case)["flops"] > 4e12 else _exact_attend(case, state)
    B, n, H, D = case["B"], case["n"], case["H"], case["D"]
    start, count = _spans(case)
    outs = []
    for i, name in enumerate("KV"):
        out = torch.zeros((B, n, H * D), dtype=torch.float64, device="cuda")
        for b in range(B):
            c = count[b]
            if c == 0:
                continue
            if case["kind"] == "store":
                out[b, :c] = _exact_round_trip(state[name][b, :c])
            else:
                codes, scales = state["cache"][i][b, :, start[b] : start[b] + c], state["cache"][2 + i][b, :, start[b] : start[b] + c]
                out[b, :c] = _exact_values(codes, scales).transpose(0, 1).reshape(c, H * D)
        outs.append(out)
    return tuple(outs)
