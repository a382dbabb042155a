"""Plain 64-bit forms of the operators that bound a decode step's reads (the 8-bit cache, chosen blocks, attention weights), on the
CPU, and bounds on how far fp32 arithmetic may be from them."""
import math

import torch

BLK = 64
EPS = 2.0 ** -24          # half a step of fp32, relative to the value
QMAX = {"i8": 127.0, "e4m3": 448.0}


def lens_of(B, Hkv, P, kind):
    """Slots in use per unit: "full", or lengths of every awkward kind up to P."""
    if kind == "full":
        return torch.full((B, Hkv), P, dtype=torch.int32)
    odd = [0, 1, 63, 64, 65, 127, 128, P // 2, P - 1, P]
    flat = [min(P, max(0, odd[(3 * u) % len(odd)])) for u in range(B * Hkv)]
    return torch.tensor(flat, dtype=torch.int32).view(B, Hkv)


def quantise(x, code):
    """x [64, d] -> codes (as the numbers they are, fp32) and scale, by the documented fp32 steps."""
    x = x.float()
    amax = x.abs().max()
    if amax < 2.0 ** -100:
        return torch.zeros_like(x), torch.tensor(0.0)
    top = torch.tensor(QMAX[code])
    y = x * (top / amax)
    return (y.round().clamp(-127, 127) if code == "i8" else y.to(torch.float8_e4m3fn).float()), amax / top


class Cache8:
    """The 8-bit cache of one unit, row by row."""

    def __init__(self, d, code):
        self.d, self.code = d, code
        self.codes, self.scales, self.tail = [[], []], [[], []], [[], []]
        self.n = 0

    def append(self, k, v):
        for j, row in enumerate((k, v)):
            self.tail[j].append(row.float())
            if len(self.tail[j]) == BLK:
                c, s = quantise(torch.stack(self.tail[j]), self.code)
                self.codes[j].append(c)
                self.scales[j].append(s)
                self.tail[j] = []
        self.n += 1

    def rows(self, j):
        full = [c.double() * s.double() for c, s in zip(self.codes[j], self.scales[j])]
        return torch.cat(full + [torch.stack(self.tail[j]).double()] if self.tail[j] else full) if self.n else torch.zeros(0, self.d).double()


def attention(q, K, V, sm):
    """q [G,d], K and V [n,d], 64 bits: (out [G,d], weights [G,n])"""
    if K.shape[0] == 0:
        return torch.zeros_like(q), torch.zeros(q.shape[0], 0).double()
    s = q @ K.t() * sm
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    return p @ V, p


def weight_error(q, K, sm):
    """Bound on the relative error of a normalized score in fp32: a logit is a sum of d products (d + 16 roundings, those of
    the scales, of the log2 domain and of q held in 22 bits among them, each of at most the sum of the magnitudes); the exponential adds 2 steps and a
    rounding to 22 bits, the normalisation doubles what every score has."""
    if K.shape[0] == 0:
        return 0.0
    a = float((q.abs() @ K.abs().t()).max()) * sm
    return 2 * ((q.shape[1] + 16) * EPS * a + 12 * EPS)


def out_error(q, K, V, sm):
    """... and of the output, absolute: the scores' errors, and one rounding for each of the n keys in both sums."""
    if K.shape[0] == 0:
        return 0.0
    return float(V.abs().max()) * (weight_error(q, K, sm) + 2 * (K.shape[0] + 8) * EPS)


def bounds_of(K):
    """K [n,d] -> [blocks, 2, d]"""
    return torch.stack([torch.stack([x.amin(0), x.amax(0)]) for x in K.split(BLK)]) if K.shape[0] else K.new_zeros(0, 2, K.shape[1])


def choose(q, bounds, nsel, nlast):
    """q [G,d], bounds [blocks,2,d] -> the chosen blocks, ascending"""
    m = bounds.shape[0]
    q, lo, hi = q.double(), bounds[:, 0].double(), bounds[:, 1].double()
    up = torch.maximum(q[:, None] * lo, q[:, None] * hi).sum(-1).amax(0).float().tolist() if m else []
    first = max(0, m - nlast)
    best = sorted(range(first), key=lambda i: (-up[i], i))[:max(0, nsel - (m - first))]
    return sorted(best) + list(range(first, m))


def kept(weight, L, r, budget):
    """weight [Lcap] -> keep of the slots < L"""
    if L <= budget:
        return [1] * L
    w = weight[:L - r].tolist()
    best = set(sorted(range(L - r), key=lambda i: (-(w[i] if w[i] == w[i] else -math.inf), i))[:budget - r])
    return [int(i >= L - r or i in best) for i in range(L)]
