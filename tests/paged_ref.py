"""Plain 64-bit forms of the cache of pages and of the rows on their way into it, on the CPU, and bounds on how far fp32 arithmetic may be from them."""
import math

import torch

from tests import operators_ref as ref

EPS = ref.EPS
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}     # half a step, relative to the value
QMAX = ref.QMAX


def axis_of(half, sections, in_turn):
    axes = len(sections)
    if in_turn:
        return [i % axes if i % axes and i < axes * sections[i % axes] else 0 for i in range(half)]
    return [a for a in range(axes) for _ in range(sections[a])]


def turn(x, weight, eps, inv_freq, positions, sections, in_turn, pairing, gain):
    """x [B,H,n,d] -> (64-bit result, bound of the fp32 arithmetic's error before it is rounded to a type).

    The norm: a sum of d squares (d roundings, of which the root halves the effect) and six more (mean, eps, root, quotient, two
    products).  A turned pair: the angle, in half turns, is rounded to fp32 (an error of pi 2^-24 at most), sine and cosine by at most four half steps
    more, gain one, products and sum three: 12 half steps of |u| + |v|."""
    d = x.shape[-1]
    y = x.double()
    err = torch.zeros_like(y)
    if weight is not None:
        y = y / torch.sqrt(y.pow(2).mean(-1, keepdim=True) + eps) * weight.double()
        err = y.abs() * ((d / 2 + 6) * EPS)
    out, bound = y.clone(), err.clone()
    half = 0 if inv_freq is None else inv_freq.numel()
    for i, ax in enumerate(axis_of(half, sections, in_turn)):
        a, b = (i, i + half) if pairing == "halves" else (2 * i, 2 * i + 1)
        angle = positions[ax].double().unsqueeze(1) * float(inv_freq[i])      # [B,1,n]
        c, s = torch.cos(angle), torch.sin(angle)
        out[..., a] = gain * (y[..., a] * c - y[..., b] * s)
        out[..., b] = gain * (y[..., b] * c + y[..., a] * s)
        e = abs(gain) * (err[..., a] + err[..., b] + 12 * EPS * (y[..., a].abs() + y[..., b].abs()))
        bound[..., a], bound[..., b] = e, e
    return out, bound


def quantise_rows(x, code):
    """x [.., d] -> codes (as the numbers they are, fp32) and scales [..], by the documented fp32 steps."""
    x = x.float()
    amax = x.abs().amax(-1)
    top = torch.full_like(amax, QMAX[code])
    some = amax >= 2.0 ** -100
    y = x * torch.where(some, top / amax, torch.zeros_like(amax)).unsqueeze(-1)
    codes = y.round().clamp(-127, 127) if code == "i8" else y.to(torch.float8_e4m3fn).float()
    return codes, torch.where(some, amax / top, torch.zeros_like(amax))


def attend(q, K, V, sm):
    return ref.attention(q, K, V, sm)[0]


def attend_error(q, K, V, sm):
    return ref.out_error(q, K, V, sm)


def sm_of(d):
    return 1.0 / math.sqrt(d)


def weighted_error(q, K, V, sm):
    """Bound [G,d] of the output's error where every logit is ONE product (queries of one channel), relative to what the channel's sum is made of,
    sum p |v|, so that nothing hides behind the largest value of another row or channel.

    A logit: a product (two steps at most, an fp32 query over codes in three parts), the scale (root, quotient, log2 e, its product, itself: five
    halves), the row's scale (one): 10 EPS of it, of the maximum as much, their difference 2: 22 EPS of the largest; the exponential a step (2 EPS).
    Both sums have that.  A sum of n weights, each in three parts: 4 n + 16 additions and products, a step (2 EPS) each if they are cut off."""
    n = K.shape[0]
    if n == 0:
        return torch.zeros_like(q)
    p = ref.attention(q, K, V, sm)[1]
    a = float((q.abs() @ K.abs().t()).max()) * sm
    return (2 * (22 * a + 2) + 2 * (4 * n + 16)) * EPS * (p @ V.abs())


def in_parts(x, parts):
    """fp32 numbers as so many bf16, each cut off, added up again"""
    left, out = x.float(), torch.zeros_like(x, dtype=torch.float64)
    for _ in range(parts):
        hi = (left.view(torch.int32) & -65536).view(torch.float32)
        out += hi.double()
        left = left - hi
    return out


def attend_in_parts(q, K, V, sm, parts, scale=None):
    """Attention whose weights (times the rows' scales: V are codes then) are held in so many bf16 parts."""
    s = q @ K.t() * sm
    p = torch.exp(s - s.amax(-1, keepdim=True))
    w = p.float() if scale is None else p.float() * scale.float()
    return in_parts(w, parts) @ V / p.sum(-1, keepdim=True)
