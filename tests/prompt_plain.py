"""What a prompt and a row of logits go through, in plain form and 64 bits: rotary positions, attention of packed prompts, cut rows."""
from __future__ import annotations

import math

import torch


# ---- rotary positions ----

def rotate(x, positions, freq, interleaved, mscale):
    """(y float64, bound on |kernel - y|) for x [..., heads, D] and positions [...] (integers of any size).

    The bound, with u = 2^-24: an angle of p freq radians is formed in 64 bits, by four roundings: 2^-51 of it.  What is left of a turn is rounded to
    32 bits (2^-26 of a turn, 2^-23 radians at most), sine and cosine of that are off by 2 u and mscale rounds them once more: 6 u in all (2 pi 2^-26 is 1.6 u).  A
    result is two products of them, added, with a rounding each: 3 u more; all relative to mscale (|x| + |y|), and rounded once to its type."""
    half = freq.numel()
    rot, D = 2 * half, x.shape[-1]
    z = x.double()
    angle = positions.double()[..., None] * freq.double()
    c, s = (f(angle)[..., None, :] * mscale for f in (torch.cos, torch.sin))
    a, b = (z[..., 0:rot:2], z[..., 1:rot:2]) if interleaved else (z[..., :half], z[..., half:rot])
    p, q = a * c - b * s, b * c + a * s
    size = abs(mscale) * (a.abs() + b.abs()) * (9 * 2.0 ** -24 + 2.0 ** -51 * angle.abs()[..., None, :])
    eps = torch.finfo(x.dtype).eps / 2
    y, bound = z.clone(), torch.zeros_like(z)
    places = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    for at, value in zip(places, (p, q)):
        y[..., at] = value
        bound[..., at] = size + eps * (value.abs() + size)
    return y, bound


# ---- attention of packed prompts ----

def attend(q, k, v, offsets, scale=None, window=0, sinks=0, weight_bits=24):
    """(out float64, bound, written [tokens]) of bv_prompt_attend.

    As in cache_plain.attend, with u = 2^-24: scores, references and exponentials make a weight off by e = 2 ((2 D + 24) u (max |score| + 1) + 2^-22) at
    most, its normaliser included, which moves a row by e sum_j w_j |v_j - out|; weights rounded to `weight_bits` bits (their sum is of the rounded
    ones) by 2^-weight_bits of the same; sums of L terms and the rescalings around them (L + 64) 2^-23 of their magnitudes; the result is rounded once."""
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    group = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    u, r, half = 2.0 ** -24, 2.0 ** -weight_bits, torch.finfo(q.dtype).eps / 2
    dev = q.device
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device=dev)
    bound = torch.zeros_like(out)
    written = torch.zeros((T,), dtype=torch.bool, device=dev)
    off = offsets.cpu().tolist()
    for first, end in zip(off[:-1], off[1:]):
        if not 0 <= first < end <= T:
            continue
        L = end - first
        # (rows of two sequences, where offsets do not ascend, get either's result: nothing is known of them)
        twice = written[first:end].clone()
        written[first:end] = True
        i = torch.arange(L, device=dev)
        see = i[None, :] <= i[:, None]
        if window > 0:
            see &= (i[:, None] - i[None, :] < window) | (i[None, :] < sinks)
        for h in range(Hq):
            qq, kk, vv = q[first:end, h].double(), k[first:end, h // group].double(), v[first:end, h // group].double()
            s = (qq @ kk.t()) * scale
            S = ((qq.abs() @ kk.abs().t()) * abs(scale)).nan_to_num(0.0, 0.0, 0.0).masked_fill(~see, 0.0).amax(1, keepdim=True)
            w = torch.softmax(s.masked_fill(~see, -math.inf), -1)
            o = torch.empty((L, D), dtype=torch.float64, device=dev)
            A, mag = torch.empty_like(o), torch.empty_like(o)
            # (what is not seen does not count, infinities and NaN among it)
            for t in range(0, L, 64):
                ww, vs = w[t:t + 64, :, None], torch.where(see[t:t + 64, :, None], vv[None], 0.0)
                o[t:t + 64] = (ww * vs).sum(1)
                A[t:t + 64] = (ww * (vs - o[t:t + 64, None])).abs().sum(1)
                mag[t:t + 64] = (ww * vs).abs().sum(1)
            e = 2 * ((2 * D + 24) * u * (S + 1) + 2.0 ** -22)
            err = (e + r * (1 + 2 * r)) * A + (L + 64) * 2.0 ** -23 * (mag + o.abs())
            out[first:end, h] = o
            bound[first:end, h] = (err + half * (o.abs() + err)).masked_fill(twice[:, None], math.inf)
    return out, bound, written


# ---- cut rows ----

def cut(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Which tokens of one row (a 1-d tensor) are kept, by sorting in 64 bits: (kept bool [V], weights float64 [V], zero where not kept); None where the
    row cannot be read."""
    z = z.detach().cpu().double()
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))
    temperature, top_p, min_p = f32(temperature), f32(top_p), f32(min_p)
    if torch.isnan(z).any() or (z == math.inf).any() or (z == -math.inf).all():
        return None
    order = sorted(range(z.numel()), key=lambda i: (-z[i].item(), i)) if z.numel() < 64 else z.sort(descending=True, stable=True).indices.tolist()
    s = z[order]
    w = ((s - s[0]) / temperature).exp()
    n = z.numel() if top_k <= 0 else min(top_k, z.numel())
    w[n:] = 0
    upto = w.cumsum(0)
    if top_p < 1:
        n = min(n, max(1, int((upto - w < top_p * upto[-1]).sum())))
    if min_p > 0:
        n = min(n, int(((s - s[0]) / temperature >= math.log(min_p)).sum()))
    kept = torch.zeros(z.shape, dtype=torch.bool)
    weights = torch.zeros_like(z)
    kept[order[:n]] = True
    kept &= z > -math.inf
    weights[kept] = ((z[kept] - s[0]) / temperature).exp()
    return kept, weights


def drawn(weights, u):
    """The token that u selects, and whether u is clear of the borders of its cell (by 10^-11 of the mass)."""
    c = weights.cumsum(0)
    t = u * c[-1]
    i = int(((c > t) & (weights > 0)).to(torch.int32).argmax()) if bool(((c > t) & (weights > 0)).any()) else int(weights.nonzero()[-1])
    return i, bool((c - t).abs().min() > 1e-11 * c[-1])
