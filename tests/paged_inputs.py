"""Inputs of attention over pages whose outputs have tight bounds, on the CPU."""
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def one_channel(g, dtype, B, Hq, Hkv, n, d):
    """q [B,Hq,d], k, v [B,Hkv,n,d]: queries and keys of one channel, logits (log2) up to 4 apart; values of one sign, so that what a weight loses adds up."""
    q, k = torch.zeros(B, Hq, d), torch.zeros(B, Hkv, n, d)
    q[..., 0] = 1 + torch.rand(B, Hq, generator=g)
    k[..., 0] = torch.rand(B, Hkv, n, generator=g) * (d ** 0.5 * 0.6931 * 2)
    return q.to(DT[dtype]), k.to(DT[dtype]), (0.1 + torch.randn(B, Hkv, n, d, generator=g).abs()).to(DT[dtype])
