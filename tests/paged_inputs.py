"""Inputs of attention over pages whose outputs have tight bounds, on the CPU."""
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}

# A weight of 1 on one row: its scale, in three parts, times a code: three products that are exact, added up with a step (2 EPS) each if they are cut off:
# 6 EPS.  All other weights, and what waves and parts add, are 0; the quotient is by 1.  Twice that is allowed.
ONE_ROW = 12 * 2.0 ** -24


def one_channel(g, dtype, B, Hq, Hkv, n, d):
    """q [B,Hq,d], k, v [B,Hkv,n,d]: queries and keys of one channel, logits (log2) up to 4 apart; values of one sign, so that what a weight loses adds up."""
    q, k = torch.zeros(B, Hq, d), torch.zeros(B, Hkv, n, d)
    q[..., 0] = 1 + torch.rand(B, Hq, generator=g)
    k[..., 0] = torch.rand(B, Hkv, n, generator=g) * (d ** 0.5 * 0.6931 * 2)
    return q.to(DT[dtype]), k.to(DT[dtype]), (0.1 + torch.randn(B, Hkv, n, d, generator=g).abs()).to(DT[dtype])


def one_row(g, dtype, Hq, n, d, decades=25.0):
    """q [1,Hq,d], k, v [1,1,n,d] (n <= 256) and, for each head, the row that it looks at: keys are the bits of their slots as +1 and -1, so that any other
    row is at least 2 x d / 8 x 80 / sqrt(d) x 1.44 > 300 (d 128) or 230 (d 64) below in the log2 domain, a weight of 0; the rows of v differ by so many powers of ten."""
    bits = torch.arange(n).unsqueeze(-1) >> torch.arange(8) & 1
    k = (2.0 * bits - 1).repeat(1, d // 8)
    size = 10.0 ** (-decades * torch.rand(n, generator=g))
    v = torch.randn(n, d, generator=g) * size.unsqueeze(-1)
    target = size.argsort()[:: max(1, n // Hq)][:Hq]           # the smallest among them, and others up to the largest
    return (80 * k[target]).to(DT[dtype])[None], k.to(DT[dtype])[None, None], v.to(DT[dtype])[None, None], target
