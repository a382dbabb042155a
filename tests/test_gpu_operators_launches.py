"""The launches that many units and long units select by their number: a sample of units, those of every length among them, against the plain 64-bit forms."""
import math

import pytest
import torch

from paper_2404_15949_amd import corm
from tests import operators_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _normal(g, *shape, dtype="f32", scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale).to(DT[dtype])


def _lens(units, cap, odd):
    """The awkward lengths over and over, and every third unit a length of its own."""
    odd = [min(x, cap) for x in odd]
    return torch.tensor([odd[u % len(odd)] if u % 3 else (u * 7919) % (cap + 1) for u in range(units)], dtype=torch.int32)


def _sample(lens, n=24):
    """Units of every length kind, the first and the last."""
    units = len(lens)
    at = sorted({0, units - 1} | {(i * 37 + 1) % units for i in range(n)})
    return at


def _check(got, q, K, V, sm, where):
    want, p = ref.attention(q, K, V, sm)
    err = float((got - want).abs().max()) if K.shape[0] else float(got.abs().max())
    assert err <= ref.out_error(q, K, V, sm), (where, K.shape[0], err, ref.out_error(q, K, V, sm))
    return p


@pytest.mark.parametrize("path", [0, 1, 2, 3])
@pytest.mark.parametrize("G,d,dtype,cap", [(1, 64, "f32", 2500), (1, 128, "bf16", 2500), (2, 64, "bf16", 2500), (2, 128, "f32", 1500), (4, 128, "bf16", 2500),
                                           (4, 64, "f32", 1500), (8, 128, "bf16", 2500), (8, 64, "f32", 2500)])
def test_weigh_of_many_units(G, d, dtype, cap, path):
    """More units than twice the compute units: the small stages of one workgroup a unit, and two rounds of keys a workgroup behind the split launch."""
    units = 1040
    g = torch.Generator(device=DEV).manual_seed(G * 1000 + cap + d)
    lens = _lens(units, cap, [0, 1, 511, 512, 513, 1023, 1024, 1025, 2047, 2048, 2049, cap - 1, cap])
    desc = corm.make_desc(units // 8, 8 * G, 8, d, cap, cap, 1, 1, dtype)
    if path == 2 and G < 8:
        assert corm.corm_selected_path(desc, corm.make_opts(2)) == 2
    K, V = _normal(g, units, cap, d, dtype=dtype, scale=1.3), _normal(g, units, cap, d, dtype=dtype, scale=2.0)
    q = _normal(g, units * G, d, dtype=dtype, scale=1.5)
    w0 = torch.rand(units, cap, generator=g, device=DEV)
    weight, out = torch.full((units, cap), 5.0, device=DEV), torch.full((units * G, d), float("nan"), device=DEV)
    ws = torch.full((corm.corm_workspace_bytes(desc),), 0xA5, dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    corm.corm_decode_attend_weigh(desc, q, K, V, lens.to(DEV), w0, weight, out, ws, status=status, opts=corm.make_opts(path))
    assert int(status) == 0
    sm = 1.0 / math.sqrt(d)
    behind = torch.arange(cap, device=DEV) >= lens.to(DEV).unsqueeze(1)
    assert bool((weight[behind] == 5.0).all()) and not bool(out.isnan().any())
    for u in _sample(lens):
        L = int(lens[u])
        x, Kr, Vr = q[u * G:(u + 1) * G].cpu().double(), K[u, :L].cpu().double(), V[u, :L].cpu().double()
        p = _check(out[u * G:(u + 1) * G].cpu().double(), x, Kr, Vr, sm, u)
        e = ref.weight_error(x, Kr, sm) + (L + 8) * ref.EPS
        total = w0[u, :L].cpu().double() + p.sum(0)
        assert bool(((weight[u, :L].cpu().double() - total).abs() <= p.sum(0) * e + (G + 1) * ref.EPS * total).all()), (u, L)


def _codes(g, code, *shape):
    if code == "i8":
        return torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int8)
    x = torch.randint(0, 127, shape, generator=g, device=DEV, dtype=torch.uint8)      # (127 is not a number)
    x ^= torch.randint(0, 2, shape, generator=g, device=DEV, dtype=torch.uint8) << 7
    return x.view(torch.float8_e4m3fn)


class Cache8:
    """An 8-bit cache of any codes: scales that make rows of magnitude 1."""

    def __init__(self, g, units, G, d, nblk, dtype, code, lens):
        top = ref.QMAX[code]
        self.G, self.d, self.lens, self.code = G, d, lens, code
        self.desc = corm.make_desc(units, G, 1, d, nblk * 64, nblk * 64, 1, 1, dtype)
        self.Kc, self.Vc = _codes(g, code, units, 1, nblk, d // 64, 64, 64), _codes(g, code, units, 1, nblk, d, 64)
        self.ks, self.vs = (torch.rand(units, 1, nblk, generator=g, device=DEV).add_(0.5).mul_(s / top) for s in (1.5, 4.0))
        self.Kt, self.Vt = _normal(g, units, 1, 64, d, dtype=dtype), _normal(g, units, 1, 64, d, dtype=dtype)
        self.q = _normal(g, units, G, d, dtype=dtype, scale=1.5)
        self.out = torch.full((units, G, d), float("nan"), device=DEV)
        self.ws = torch.full((corm.corm_blocks_workspace_bytes(self.desc),), 0xA5, dtype=torch.uint8, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def attend(self, blocks=None):
        corm.corm_q8_attend(self.desc, self.code, self.q, self.Kc, self.Vc, self.ks, self.vs, self.Kt, self.Vt, self.lens.to(DEV), self.out, self.ws,
                            blocks=None if blocks is None else blocks.to(DEV), nsel=0 if blocks is None else blocks.shape[-1], status=self.status)
        assert int(self.status) == 0

    def check(self, u, blocks=None):
        L, d = int(self.lens[u]), self.d
        full, rest = L // 64, L % 64
        ids = list(range(full + (rest > 0))) if blocks is None else [i for i in blocks[u].tolist() if i >= 0]
        K, V = [torch.zeros(0, d).double()], [torch.zeros(0, d).double()]
        for i in ids:
            if i < full:
                K.append(self.Kc[u, 0, i].cpu().float().double().permute(1, 0, 2).reshape(64, d) * self.ks[u, 0, i].cpu().double())
                V.append(self.Vc[u, 0, i].cpu().float().double().t() * self.vs[u, 0, i].cpu().double())
            else:
                K.append(self.Kt[u, 0, :rest].cpu().double())
                V.append(self.Vt[u, 0, :rest].cpu().double())
        _check(self.out[u].cpu().double(), self.q[u].cpu().double(), torch.cat(K), torch.cat(V), 1.0 / math.sqrt(d), u)


@pytest.mark.parametrize("units,nblk", [(520, 70), (520, 23), (1300, 9), (300, 70), (16, 700), (100, 150)])
@pytest.mark.parametrize("G,d,dtype,code", [(1, 128, "bf16", "i8"), (4, 128, "bf16", "e4m3"), (8, 64, "f32", "i8"), (2, 128, "f32", "e4m3")])
def test_q8_attend_of_many_and_of_long_units(units, nblk, G, d, dtype, code):
    """A workgroup a unit with many rounds of blocks, and parts of two and more rounds; every block, and lists of them in no order."""
    g = torch.Generator(device=DEV).manual_seed(units + nblk + G)
    cap = nblk * 64
    lens = _lens(units, cap, [0, 1, 63, 64, 65, 64 * 4 + 1, 64 * 8, 64 * 9 - 1, cap // 2 + 5, cap - 64, cap - 1, cap])
    c = Cache8(g, units, G, d, nblk, dtype, code, lens.view(units, 1))
    c.attend()
    assert not bool(c.out.isnan().any())
    for u in _sample(lens):
        c.check(u)
    h = torch.Generator().manual_seed(nblk)
    for nsel in (nblk, 40):
        used = (lens + 63) // 64
        blocks = torch.randint(-1, nblk, (units, nsel), generator=h, dtype=torch.int32)
        blocks = torch.where(blocks < used.unsqueeze(1), blocks, torch.full_like(blocks, -1))
        c.out.fill_(float("nan"))
        c.attend(blocks.view(units, 1, nsel))
        assert not bool(c.out.isnan().any())
        for u in _sample(lens, 12):
            c.check(u, blocks)


def test_q8_attend_in_the_longest_parts():
    """Parts of 256 blocks, and the last one shorter: 500 units of up to 2400 blocks."""
    g = torch.Generator(device=DEV).manual_seed(3)
    units, nblk = 500, 2400
    cap = nblk * 64
    odd = [0, 64 * 256, 64 * 256 + 1, 64 * 256 - 1, 64 * 512 + 63, 64 * 2304, 64 * 2305 - 1, cap - 1, cap]
    lens = torch.tensor([odd[u % len(odd)] for u in range(units)], dtype=torch.int32)
    c = Cache8(g, units, 1, 64, nblk, "bf16", "i8", lens.view(units, 1))
    c.attend()
    assert not bool(c.out.isnan().any())
    for u in list(range(len(odd))) + [units - 1]:
        c.check(u)


@pytest.mark.parametrize("nsel", [9, 33, 64, 100])
@pytest.mark.parametrize("units,G,d,dtype", [(130, 1, 128, "bf16"), (130, 2, 64, "bf16"), (130, 4, 128, "bf16"), (130, 8, 128, "bf16"), (300, 8, 64, "bf16"),
                                             (260, 2, 128, "f32"), (130, 8, 128, "f32"), (260, 4, 64, "f32")])
def test_block_attend_of_many_units(units, G, d, dtype, nsel):
    """Parts of up to eight listed blocks: empty places between them, the unfinished block anywhere, blocks twice."""
    nblk = 80
    g = torch.Generator(device=DEV).manual_seed(units + G + nsel)
    cap = nblk * 64 - 5
    lens = _lens(units, cap, [0, 1, 64, 65, 64 * 8, 64 * 8 + 1, 64 * 40 - 1, cap - 60, cap])
    K, V = _normal(g, units, cap, d, dtype=dtype, scale=1.3), _normal(g, units, cap, d, dtype=dtype, scale=2.0)
    q = _normal(g, units, G, d, dtype=dtype, scale=1.5)
    desc = corm.make_desc(units, G, 1, d, cap, cap, 1, 1, dtype)
    h = torch.Generator().manual_seed(nsel)
    used = (lens + 63) // 64
    blocks = torch.randint(-1, nblk, (units, nsel), generator=h, dtype=torch.int32)
    blocks = torch.where(blocks < used.unsqueeze(1), blocks, torch.full_like(blocks, -1))
    for u in range(0, units, 5):       # ascending and whole, as a choice leaves them
        n = min(nsel, int(used[u]))
        blocks[u] = -1
        blocks[u, :n] = torch.arange(int(used[u]) - n, int(used[u]), dtype=torch.int32)
    out = torch.full((units, G, d), float("nan"), device=DEV)
    ws = torch.full((corm.corm_blocks_workspace_bytes(desc),), 0xA5, dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    corm.corm_block_attend(desc, q, K, V, lens.to(DEV).view(units, 1), blocks.to(DEV).view(units, 1, nsel), nsel, out, ws, status=status)
    assert int(status) == 0 and not bool(out.isnan().any())
    for u in _sample(lens) + [5, 10, 20]:
        L = int(lens[u])
        slots = [s for i in blocks[u].tolist() if i >= 0 for s in range(64 * i, min(64 * i + 64, L))]
        _check(out[u].cpu().double(), q[u].cpu().double(), K[u, slots].cpu().double(), V[u, slots].cpu().double(), 1.0 / math.sqrt(d), u)


@pytest.mark.parametrize("units,cap", [(3, 1 << 20), (20, 131072), (300, 60000)])
@pytest.mark.parametrize("sigma", [2.0, 0.5, 0.25, 0.1])
def test_evict_mask_weight_of_close_accounts(units, cap, sigma):
    """Long units with more accounts in the digit of the cut than a workgroup holds, few and many of all there are; a part of them equal."""
    g = torch.Generator(device=DEV).manual_seed(cap)
    w = torch.exp(sigma * torch.randn(units, cap, generator=g, device=DEV)) / 1024
    w[1] = (w[1] * 2 ** 14).round() / 2 ** 14
    lens = torch.full((units, 1), cap, dtype=torch.int32)
    lens[1::3] = cap - 17
    r = 33
    desc = corm.make_desc(units, 1, 1, 64, cap, cap, 1, r, "f32")
    ws = torch.full((corm.corm_blocks_workspace_bytes(desc),), 0xA5, dtype=torch.uint8, device=DEV)
    for budget in (cap // 16, cap // 2):
        keep = torch.full((units, cap), 9, dtype=torch.uint8, device=DEV)
        corm.corm_evict_mask_weight(desc, w, lens.to(DEV), budget, keep, ws)
        at = torch.arange(cap, device=DEV)
        for u in sorted({0, 1, 2, units - 1, units // 2}):
            L = int(lens[u])
            order = torch.sort(w[u, :L - r], descending=True, stable=True)[1][:budget - r]      # (equal ones: the lower slot first)
            want = (at >= L - r).to(torch.uint8)
            want[order] = 1
            want[L:] = 9
            assert torch.equal(keep[u], want), (u, L, budget)
