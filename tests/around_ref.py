"""Plain 64-bit forms of the operators around the projection (norm, rotation, paged cache, attention), and the tolerances of their tests."""
import math

import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11, "e4m3": 2.0 ** -4}     # of a rounding, relative to the value


def values(cache):
    """A cache's entries in 64 bits (codes as what they stand for)."""
    return (cache.contiguous().view(torch.float8_e4m3fn) if cache.dtype == torch.uint8 else cache).double()


def bits(t):
    """What is stored, comparable where it is NaN."""
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def to_e4m3(x):
    """Nearest E4M3 value, ties to even, saturating at 448; steps of 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def norm(x, r, w, eps):
    h = x.double() + (r.double() if r is not None else 0.0)
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, y * w.double() if w is not None else y


def turns(rot, base=10000.0, factor=1.0, original=0.0, low=1.0, high=32.0):
    out = []
    for i in range(rot // 2):
        t = base ** (-2.0 * i / rot) / (2.0 * math.pi)
        g = min(max((original * t - low) / (high - low), 0.0), 1.0) if original > 0 else 0.0
        out.append(t * (g + (1.0 - g) / factor))
    return torch.tensor(out, dtype=torch.float64)


def rotate(x, heads, dh, pos, t, interleaved, magnitude=1.0):
    """x: n x (heads * dh) in 64 bits; pair by pair.  Also the sum of the magnitudes that enter each component."""
    n, rot = x.shape[0], 2 * t.numel()
    x = x.double().reshape(n, heads, dh)
    out, size = x.clone(), x.abs()
    frac = torch.remainder(pos.double()[:, None] * t.to(x.device)[None], 1.0)
    c, s = magnitude * torch.cos(2 * math.pi * frac), magnitude * torch.sin(2 * math.pi * frac)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        u, v = x[:, :, a], x[:, :, b]
        out[:, :, a] = u * c[:, i, None] - v * s[:, i, None]
        out[:, :, b] = v * c[:, i, None] + u * s[:, i, None]
        size[:, :, a] = size[:, :, b] = magnitude * (u.abs() + v.abs())
    return out, size


# The rotation's arithmetic: the angle is rounded to fp32 within half a circle (2^-25 of a circle, 2^-22.3 radians), sincospif is good to two
# units in the last place (2^-23), its result times the magnitude and the two products and the sum are rounded (2^-24 each, five at most).
ROTATED = 2.0 ** -22.3 + 2.0 ** -23 + 5 * 2.0 ** -24


def attend(q, k, v, table, lengths, scale, window=0, k_scale=1.0, v_scale=1.0):
    """q: seqs x hq x dh; k, v: (page, token, head, component).  Returns o, lse, sum p |v| and the bound on a logit's error, in 64 bits."""
    seqs, hq, dh = q.shape
    hk, ps = k.shape[2], k.shape[1]
    o = torch.zeros((seqs, hq, dh), dtype=torch.float64, device=q.device)
    weight = torch.zeros_like(o)
    lse = torch.full((seqs, hq), -math.inf, dtype=torch.float64, device=q.device)
    slack = torch.zeros_like(lse)
    pages = table.tolist()
    for s in range(seqs):
        n = min(int(lengths[s]), table.shape[1] * ps)
        at = [t for t in range(max(0, n - window) if window else 0, n) if 0 <= pages[s][t // ps] < k.shape[0]]
        if not at:
            continue
        at = torch.tensor(at, device=q.device)
        page = table[s].long()[at // ps]
        ks, vs = (values(x[page, at % ps]).repeat_interleave(hq // hk, 1) * f for x, f in ((k, k_scale), (v, v_scale)))
        z = scale * torch.einsum("hd,nhd->hn", q[s].double(), ks)
        top = z.max(1, keepdim=True).values
        p = torch.exp(z - top)
        lse[s] = top[:, 0] + torch.log(p.sum(1))
        p = p / p.sum(1, keepdim=True)
        o[s] = torch.einsum("hn,nhd->hd", p, vs)
        weight[s] = torch.einsum("hn,nhd->hd", p, vs.abs())
        # dh products summed in fp32, and q held to 2^-24 of its largest component
        slack[s] = abs(scale) * (dh + 8) * 2.0 ** -24 * q[s].double().abs().amax(1) * ks.abs().sum(2).amax(0)
    return o, lse, weight, slack


def attend_tolerance(o, lse, weight, slack, lengths, vmax, dtype, cache):
    """|o - o_64| and |lse - lse_64|: the stored result's rounding; each p off by its logit's error twice (its own and the sum's), by exp (2^-21
    with the scaling of its argument) and by its rounding for the second product: 16-bit caches hold p as a pair (2^-16), E4M3 ones as
    one half (2^-11, and 2^-25 absolute next to zero); sums of n terms in fp32."""
    n = torch.as_tensor(lengths, device=o.device).clamp_min(1).double()[:, None, None]
    rel = 2 * slack[..., None] + 2.0 ** -21 * (1 + lse.abs().nan_to_num(posinf=0, neginf=0))[..., None] + (n + 16) * 2.0 ** -24
    rel = rel + (2.0 ** -11 if cache == "e4m3" else 2.0 ** -16 if dtype != "f32" else 0.0)
    tol_o = HALF_STEP[dtype] * o.abs() + rel * weight + (n * 2.0 ** -24 * vmax if cache == "e4m3" else 0.0) + 2.0 ** -25
    tol_l = slack + (n[..., 0] + 16) * 2.0 ** -24 + 2.0 ** -21 * (1 + lse.abs().nan_to_num(posinf=0, neginf=0))
    return tol_o, tol_l
