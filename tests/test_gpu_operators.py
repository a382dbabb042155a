"""The 8-bit cache, attention over chosen blocks and eviction by attention weight against plain 64-bit forms, on the device."""
import math

import pytest
import torch

from paper_2404_15949_amd import corm
from tests import operators_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rows(g, dtype, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(DT[dtype])


def _ws(desc):
    return torch.full((corm.corm_blocks_workspace_bytes(desc),), 0xA5, dtype=torch.uint8, device=DEV)   # nothing prepared


class Q8:
    """Device arrays of an 8-bit cache, filled with junk where nothing is to be read, and the plain form beside it."""

    def __init__(self, B, Hq, Hkv, d, cap, dtype, code, bounds=False):
        self.B, self.Hq, self.Hkv, self.d, self.cap, self.dtype, self.code = B, Hq, Hkv, d, cap, dtype, code
        self.desc = corm.make_desc(B, Hq, Hkv, d, cap, cap, 1, 1, dtype)
        n = (cap + 63) // 64
        cdt = torch.int8 if code == "i8" else torch.float8_e4m3fn
        junk = lambda *s: torch.full(s, float("nan"), device=DEV)  # noqa: E731
        self.Kc = torch.full((B, Hkv, n, d // 64, 64, 64), 0x7F, dtype=torch.int8, device=DEV).view(cdt)
        self.Vc = torch.full((B, Hkv, n, d, 64), 0x7F, dtype=torch.int8, device=DEV).view(cdt)
        self.ks, self.vs = junk(B, Hkv, n), junk(B, Hkv, n)
        self.Kt, self.Vt = junk(B, Hkv, 64, d).to(DT[dtype]), junk(B, Hkv, 64, d).to(DT[dtype])
        self.bounds = junk(B, Hkv, n, 2, d).to(DT[dtype]) if bounds else None
        self.lens = torch.zeros(B, Hkv, dtype=torch.int32, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.out = torch.full((B, Hq, d), float("nan"), device=DEV)
        self.plain = [[ref.Cache8(d, code) for _ in range(Hkv)] for _ in range(B)]
        self.seen = [[[] for _ in range(Hkv)] for _ in range(B)]
        self.ws = _ws(self.desc)

    def append(self, k, v, n_new=None):
        n = k.shape[2]
        dev_n = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device=DEV)
        corm.corm_q8_append(self.desc, self.code, k.to(DEV), v.to(DEV), n, dev_n, self.Kc, self.Vc, self.ks, self.vs, self.Kt, self.Vt,
                            self.lens, self.lens, self.bounds, self.status)
        for b in range(self.B):
            take = n if n_new is None else min(max(n_new[b], 0), n)
            for h in range(self.Hkv):
                if self.plain[b][h].n + take > self.cap:
                    continue
                for i in range(take):
                    self.plain[b][h].append(k[b, h, i], v[b, h, i])
                    self.seen[b][h].append(k[b, h, i].float())

    def check_state(self):
        Kc, Vc = self.Kc.cpu().float(), self.Vc.cpu().float()
        ks, vs, Kt, Vt, lens = (x.cpu() for x in (self.ks, self.vs, self.Kt.float(), self.Vt.float(), self.lens))
        for b in range(self.B):
            for h in range(self.Hkv):
                c = self.plain[b][h]
                where = (b, h, c.n)
                assert int(lens[b, h]) == c.n, where
                for i in range(len(c.codes[0])):
                    assert torch.equal(Kc[b, h, i].permute(1, 0, 2).reshape(64, self.d), c.codes[0][i]), where
                    assert torch.equal(Vc[b, h, i].t(), c.codes[1][i]), where
                    assert float(ks[b, h, i]) == float(c.scales[0][i]) and float(vs[b, h, i]) == float(c.scales[1][i]), where
                full = len(c.codes[0])                    # blocks that are not full are left as they were
                assert bool((self.Kc.view(torch.int8)[b, h, full:] == 0x7F).all()) and bool((self.Vc.view(torch.int8)[b, h, full:] == 0x7F).all()), where
                assert bool(ks[b, h, full:].isnan().all()) and bool(vs[b, h, full:].isnan().all()), where
                m = c.n % 64
                if m:
                    assert torch.equal(Kt[b, h, :m], torch.stack(c.tail[0])) and torch.equal(Vt[b, h, :m], torch.stack(c.tail[1])), where
                if self.bounds is not None and c.n:
                    want = ref.bounds_of(torch.stack(self.seen[b][h]))
                    assert torch.equal(self.bounds[b, h, :want.shape[0]].cpu().float(), want), where

    def check_out(self, q, blocks=None):
        G, sm, got = self.Hq // self.Hkv, 1.0 / math.sqrt(self.d), self.out.cpu().double()
        for b in range(self.B):
            for h in range(self.Hkv):
                c = self.plain[b][h]
                K, V = c.rows(0), c.rows(1)
                if blocks is not None:
                    slots = [s for i in blocks[b][h] if 0 <= i for s in range(64 * i, min(64 * i + 64, c.n))]
                    K, V = K[slots], V[slots]
                x = q[b, h * G:(h + 1) * G].double()
                want, _ = ref.attention(x, K, V, sm)
                err = float((got[b, h * G:(h + 1) * G] - want).abs().max())
                assert err <= ref.out_error(x, K, V, sm), (b, h, c.n, err, ref.out_error(x, K, V, sm))

    def attend(self, q, blocks=None):
        self.out.fill_(float("nan"))
        bl = None if blocks is None else torch.tensor(blocks, dtype=torch.int32, device=DEV)
        corm.corm_q8_attend(self.desc, self.code, q.to(DEV), self.Kc, self.Vc, self.ks, self.vs, self.Kt, self.Vt, self.lens, self.out,
                            self.ws, blocks=bl, nsel=0 if bl is None else bl.shape[2], status=self.status)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_q8_append_in_pieces(dtype, d, code):
    """Rows in pieces of every awkward length, ragged over the batch: codes, scales, tails, lengths and bounds to the bit."""
    g = _gen(1)
    c = Q8(3, 2, 2, d, 64 * 6 + 17, dtype, code, bounds=True)
    for n, n_new in ((1, None), (62, None), (1, [1, 0, 1]), (1, None), (64, [64, 63, 1]), (65, [65, 0, 64]), (130, [3, 130, 129]), (1, None),
                     (63, [63, 62, 0]), (5, [-3, 99, 2])):
        c.append(_rows(g, dtype, 3, 2, n, d), _rows(g, dtype, 3, 2, n, d, scale=30.0), n_new)
        c.check_state()
    assert int(c.status) == 0


def test_q8_append_refuses_what_does_not_fit():
    """A unit without room gets none of the rows and keeps its state; the others get theirs.  Lengths that are none are clamped for reading and
    nothing is written."""
    g = _gen(2)
    c = Q8(2, 1, 1, 64, 100, "bf16", "i8", bounds=True)
    c.append(_rows(g, "bf16", 2, 1, 90, 64), _rows(g, "bf16", 2, 1, 90, 64), [90, 20])
    before = [x.clone() for x in (c.Kt, c.Vt, c.Kc.view(torch.int8), c.Vc.view(torch.int8))]
    c.append(_rows(g, "bf16", 2, 1, 11, 64), _rows(g, "bf16", 2, 1, 11, 64))
    c.check_state()
    assert int(c.status) == corm.CORM_DEV_UNIT_FULL
    for x, y in zip((c.Kt, c.Vt, c.Kc.view(torch.int8), c.Vc.view(torch.int8)), before):
        assert torch.equal(x[0], y[0]) or (x[0].isnan() == y[0].isnan()).all() and torch.equal(x[0].nan_to_num(), y[0].nan_to_num())
    c.append(_rows(g, "bf16", 2, 1, 10, 64), _rows(g, "bf16", 2, 1, 10, 64))      # to the last slot
    c.check_state()
    c.append(_rows(g, "bf16", 2, 1, 1, 64), _rows(g, "bf16", 2, 1, 1, 64))
    c.check_state()
    c.status.zero_()
    bad = torch.tensor([[-5], [101]], dtype=torch.int32, device=DEV)
    out = torch.zeros_like(bad)
    state = [x.clone() for x in (c.Kt, c.Vt)]
    one = torch.zeros(2, 1, 1, 64, dtype=torch.bfloat16, device=DEV)
    corm.corm_q8_append(c.desc, "i8", one, one, 1, None, c.Kc, c.Vc, c.ks, c.vs, c.Kt, c.Vt, bad, out, None, c.status)
    assert int(c.status) == corm.CORM_DEV_BAD_LENS and torch.equal(out, bad)
    assert all(torch.equal(x.nan_to_num(), y.nan_to_num()) for x, y in zip((c.Kt, c.Vt), state))


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_q8_blocks_of_zeros_tiny_and_large_rows(code):
    g = _gen(3)
    c = Q8(1, 1, 1, 128, 64 * 5, "f32", code)
    scale = torch.tensor([0.0, 1e-33, 1e-20, 1e25, 1.0]).repeat_interleave(64).view(1, 1, -1, 1)
    c.append(_rows(g, "f32", 1, 1, 320, 128) * scale, _rows(g, "f32", 1, 1, 320, 128) * scale)
    c.check_state()
    assert float(c.ks[0, 0, 0]) == 0.0 and float(c.ks[0, 0, 1]) == 0.0 and float(c.ks[0, 0, 2]) > 0.0


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("B,Hq,Hkv,d,P,dtype", [
    (2, 4, 4, 128, 300, "bf16"), (3, 24, 3, 64, 705, "f32"), (2, 16, 4, 128, 1000, "f32"), (1, 2, 1, 64, 191, "bf16"),
    (5, 16, 2, 128, 129, "bf16"), (1, 1, 1, 128, 64 * 67 + 1, "bf16"), (2, 10, 5, 64, 640, "bf16")])
def test_q8_attend(B, Hq, Hkv, d, P, dtype, code):
    g = _gen(P)
    c = Q8(B, Hq, Hkv, d, P + 3, dtype, code)
    c.append(_rows(g, dtype, B, Hkv, P, d, scale=1.3), _rows(g, dtype, B, Hkv, P, d, scale=2.0), [max(0, P - 97 * b) for b in range(B)])
    q = _rows(g, dtype, B, Hq, d, scale=1.5)
    c.attend(q)
    c.check_out(q)
    assert int(c.status) == 0


@pytest.mark.parametrize("dtype,code", [("bf16", "i8"), ("f32", "e4m3")])
def test_q8_attend_lengths_one_by_one(dtype, code):
    """Every unit another length, from none to two blocks and a row; queries of very different magnitude."""
    g = _gen(5)
    lens = [0, 1, 2, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129]
    c = Q8(len(lens), 4, 1, 128, 130, dtype, code)
    c.append(_rows(g, dtype, len(lens), 1, 130, 128), _rows(g, dtype, len(lens), 1, 130, 128), lens)
    for scale in (1e-30, 1e-4, 1.0, 12.0):
        q = _rows(g, dtype, len(lens), 4, 128, scale=scale)
        q[:, 1] *= 1e-3
        q[:, 2] = 0
        q[:, 3, 1:] *= 1e-6
        c.attend(q)
        c.check_out(q)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_q8_attend_over_rows_of_very_different_magnitude(code):
    """Blocks whose keys and values are of magnitude 0, 1e-33, 1e-6, 1 and (values) 1e30: scales of every size."""
    g, d = _gen(8), 128
    c = Q8(1, 4, 1, d, 64 * 6, "f32", code)
    mag = lambda *m: torch.tensor(m).repeat_interleave(64)[:350].view(1, 1, -1, 1)  # noqa: E731
    c.append(_rows(g, "f32", 1, 1, 350, d) * mag(0.0, 1e-33, 1.0, 1e-6, 1.0, 1.0), _rows(g, "f32", 1, 1, 350, d) * mag(1.0, 0.0, 1e30, 1e-33, 1e30, 1.0))
    q = _rows(g, "f32", 1, 4, d)
    c.attend(q)
    c.check_out(q)


def test_q8_attend_over_listed_blocks():
    """Any order, -1 between, blocks beyond the unit's (skipped and flagged), the unfinished block, blocks listed twice, an empty list."""
    g = _gen(7)
    c = Q8(4, 8, 1, 64, 64 * 40, "bf16", "i8")
    c.append(_rows(g, "bf16", 4, 1, 64 * 39 + 5, 64), _rows(g, "bf16", 4, 1, 64 * 39 + 5, 64), [64 * 39 + 5, 64 * 20, 30, 64 * 39 + 5])
    q = _rows(g, "bf16", 4, 8, 64)
    n = 21
    lists = [[39, 3, -1, 0, 17, 4] + list(range(18, 33)), [19, 19, 0, 1] + [-1] * 17, [0, 0] + [-1] * 19, [-1] * 21]
    c.attend(q, [[x] for x in lists])
    c.check_out(q, [[x] for x in lists])
    assert int(c.status) == 0
    lists = [[39, 40, 5, -2] + [-1] * (n - 4), [20, 19] + [-1] * (n - 2), [1, 0, 1 << 30] + [-1] * (n - 3), [-(1 << 31)] * n]
    c.attend(q, [[x] for x in lists])
    ok = [[[39, 5]], [[19]], [[0]], [[]]]
    c.check_out(q, ok)
    assert int(c.status) == corm.CORM_DEV_BAD_BLOCK


def _state(g, B, Hq, Hkv, d, cap, dtype, lens):
    K, V = _rows(g, dtype, B, Hkv, cap, d, scale=1.3), _rows(g, dtype, B, Hkv, cap, d, scale=2.0)
    for b in range(B):
        for h in range(Hkv):   # (what lies behind a unit's rows is never used)
            K[b, h, int(lens[b, h]):], V[b, h, int(lens[b, h]):] = float("nan"), float("nan")
    return K, V, _rows(g, dtype, B, Hq, d, scale=1.5)


SHAPES = [(2, 4, 4, 128, 333, "bf16"), (3, 24, 3, 64, 705, "f32"), (2, 16, 4, 128, 1000, "f32"), (1, 2, 1, 64, 191, "bf16"),
          (5, 16, 2, 128, 130, "bf16"), (1, 4, 1, 128, 64 * 70 + 9, "bf16"), (10, 2, 2, 64, 650, "f32"), (2, 8, 4, 128, 64 * 300, "bf16"),
          (1, 8, 1, 128, 2000, "f32"), (2, 8, 4, 64, 900, "bf16"), (1, 2, 1, 128, 640, "f32"), (1, 2, 2, 128, 640, "f32")]


@pytest.mark.parametrize("B,Hq,Hkv,d,cap,dtype", SHAPES)
def test_block_bounds(B, Hq, Hkv, d, cap, dtype):
    g = _gen(cap)
    lens = ref.lens_of(B, Hkv, cap, "odd")
    K, _, _ = _state(g, B, Hq, Hkv, d, cap, dtype, lens)
    desc = corm.make_desc(B, Hq, Hkv, d, cap, cap, 1, 1, dtype)
    nblk = (cap + 63) // 64
    for newest in (0, 1, 2, 64, 65, 200, 1 << 30):
        bounds = torch.full((B, Hkv, nblk, 2, d), 7.0, dtype=DT[dtype], device=DEV)
        corm.corm_block_bounds(desc, K.to(DEV), lens.to(DEV), bounds, newest)
        got = bounds.cpu().float()
        for b in range(B):
            for h in range(Hkv):
                L = int(lens[b, h])
                want = torch.full((nblk, 2, d), 7.0)
                first = 0 if newest == 0 else max(L - newest, 0) // 64
                real = ref.bounds_of(K[b, h, :L].float())
                want[first:real.shape[0]] = real[first:]
                assert torch.equal(got[b, h], want), (b, h, L, newest)


@pytest.mark.parametrize("B,Hq,Hkv,d,cap,dtype", SHAPES)
@pytest.mark.parametrize("nsel,nlast", [(1, 1), (5, 2), (32, 1), (300, 7)])
def test_block_select(B, Hq, Hkv, d, cap, dtype, nsel, nlast):
    g = _gen(cap + nsel)
    lens = ref.lens_of(B, Hkv, cap, "odd" if nsel != 5 else "full")
    K, _, q = _state(g, B, Hq, Hkv, d, cap, dtype, lens)
    desc = corm.make_desc(B, Hq, Hkv, d, cap, cap, 1, 1, dtype)
    nblk, G = (cap + 63) // 64, Hq // Hkv
    bounds = torch.full((B, Hkv, nblk, 2, d), float("nan"), dtype=DT[dtype])
    for b in range(B):
        for h in range(Hkv):
            if lens[b, h] > 640 and h % 2 == 0:   # equal blocks: the lower one first
                K[b, h, 128:192], K[b, h, 512:576] = K[b, h, 0:64], K[b, h, 0:64]
            x = ref.bounds_of(K[b, h, :int(lens[b, h])])
            bounds[b, h, :x.shape[0]] = x
    blocks = torch.full((B, Hkv, nsel), -77, dtype=torch.int32, device=DEV)
    corm.corm_block_select(desc, q.to(DEV), bounds.to(DEV), lens.to(DEV), nsel, nlast, blocks, _ws(desc))
    for b in range(B):
        for h in range(Hkv):
            m = (int(lens[b, h]) + 63) // 64
            want = ref.choose(q[b, h * G:(h + 1) * G], bounds[b, h, :m], nsel, nlast)
            assert blocks[b, h].tolist() == want + [-1] * (nsel - len(want)), (b, h, m)


@pytest.mark.parametrize("nblk", [100, 129, 700, 5000])
def test_block_select_among_equal_and_many_blocks(nblk):
    """Every block the same: the lowest are chosen.  Then all but a few, and numbers on both sides of what one launch and LDS hold."""
    g, d, G = _gen(nblk), 64, 2
    desc = corm.make_desc(3, G, 1, d, nblk * 64, nblk * 64, 1, 1, "f32")
    lens = torch.tensor([[nblk * 64], [nblk * 64 - 70], [nblk * 32 + 1]], dtype=torch.int32)
    q = _rows(g, "f32", 3, G, d)
    bounds = torch.zeros(3, 1, nblk, 2, d)
    bounds[:, :, :, 0], bounds[:, :, :, 1] = -1.0, 2.0
    bounds[1, 0, ::17] = torch.randn(len(range(0, nblk, 17)), 2, d, generator=g)
    bounds[2] = torch.randn(1, nblk, 2, d, generator=g)
    for nsel, nlast in ((60, 3), (5, 1), (90, 90)):
        blocks = torch.full((3, 1, nsel), -77, dtype=torch.int32, device=DEV)
        corm.corm_block_select(desc, q.to(DEV), bounds.to(DEV), lens.to(DEV), nsel, nlast, blocks, _ws(desc))
        for b in range(3):
            m = (int(lens[b]) + 63) // 64
            want = ref.choose(q[b], bounds[b, 0, :m], nsel, nlast)
            assert blocks[b, 0].tolist() == want + [-1] * (nsel - len(want)), (b, nsel)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_block_select_with_keys_of_the_lowest_value(dtype):
    """Keys overwritten with the type's lowest value, as a mask: the bounds' other side still decides among blocks where queries are positive, nothing is lost to
    the large numbers (q >= 0, so the lowest values never enter a score)."""
    g, d, n = _gen(21), 64, 40
    K = _rows(g, dtype, 1, 1, n * 64, d)
    K[0, 0, 5::64] = torch.finfo(DT[dtype]).min
    q = _rows(g, dtype, 1, 2, d).abs()
    desc = corm.make_desc(1, 2, 1, d, n * 64, n * 64, 1, 1, dtype)
    lens = torch.tensor([[n * 64]], dtype=torch.int32, device=DEV)
    bounds, blocks = torch.empty(1, 1, n, 2, d, dtype=DT[dtype], device=DEV), torch.empty(1, 1, 9, dtype=torch.int32, device=DEV)
    corm.corm_block_bounds(desc, K.to(DEV), lens, bounds)
    corm.corm_block_select(desc, q.to(DEV), bounds, lens, 9, 1, blocks, _ws(desc))
    assert blocks[0, 0].tolist() == ref.choose(q[0], ref.bounds_of(K[0, 0]), 9, 1)


@pytest.mark.parametrize("B,Hq,Hkv,d,cap,dtype", SHAPES)
@pytest.mark.parametrize("nsel", [1, 2, 11, 70])
def test_block_attend(B, Hq, Hkv, d, cap, dtype, nsel):
    g = _gen(cap + nsel)
    lens = ref.lens_of(B, Hkv, cap, "odd")
    K, V, q = _state(g, B, Hq, Hkv, d, cap, dtype, lens)
    desc = corm.make_desc(B, Hq, Hkv, d, cap, cap, 1, 1, dtype)
    nblk, G, sm = (cap + 63) // 64, Hq // Hkv, 1.0 / math.sqrt(d)
    blocks = torch.randint(-1, nblk, (B, Hkv, nsel), generator=g, dtype=torch.int32)   # any order, some twice, some beyond
    if nsel > 2:
        blocks[0, 0, 0], blocks[0, 0, 1] = 1 << 30, -(1 << 31)
    out = torch.full((B, Hq, d), float("nan"), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    corm.corm_block_attend(desc, q.to(DEV), K.to(DEV), V.to(DEV), lens.to(DEV), blocks.to(DEV), nsel, out, _ws(desc), status=status)
    got, bad = out.cpu().double(), False
    for b in range(B):
        for h in range(Hkv):
            L = int(lens[b, h])
            bad |= any(i != -1 and not 0 <= i < (L + 63) // 64 for i in blocks[b, h].tolist())
            slots = [s for i in blocks[b, h].tolist() if i >= 0 for s in range(64 * i, min(64 * i + 64, L))]
            x = q[b, h * G:(h + 1) * G].double()
            Ks, Vs = K[b, h, slots].double(), V[b, h, slots].double()
            want, _ = ref.attention(x, Ks, Vs, sm)
            err = float((got[b, h * G:(h + 1) * G] - want).abs().max())
            assert err <= ref.out_error(x, Ks, Vs, sm), (b, h, L, err)
    assert int(status) == (corm.CORM_DEV_BAD_BLOCK if bad else 0)


@pytest.mark.parametrize("B,Hq,Hkv,d,cap,dtype", SHAPES)
@pytest.mark.parametrize("path", [0, 1, 2, 3])
def test_attend_weigh(B, Hq, Hkv, d, cap, dtype, path):
    g = _gen(cap)
    lens = ref.lens_of(B, Hkv, cap, "odd")
    K, V, q = _state(g, B, Hq, Hkv, d, cap, dtype, lens)
    desc = corm.make_desc(B, Hq, Hkv, d, cap, cap, 1, 1, dtype)
    G, sm = Hq // Hkv, 1.0 / math.sqrt(d)
    ws = torch.full((corm.corm_workspace_bytes(desc),), 0xA5, dtype=torch.uint8, device=DEV)
    w0 = torch.rand(B, Hkv, cap, generator=g)
    dev = [x.to(DEV) for x in (q, K, V, lens)]
    weight, out = torch.full((B, Hkv, cap), 5.0, device=DEV), torch.full((B, Hq, d), float("nan"), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    corm.corm_decode_attend_weigh(desc, *dev, w0.to(DEV), weight, out, ws, status=status, opts=corm.make_opts(path))
    same = w0.to(DEV)
    corm.corm_decode_attend_weigh(desc, *dev, same, same, torch.empty_like(out), ws, opts=corm.make_opts(path))
    got, acc = out.cpu().double(), weight.cpu()
    for b in range(B):
        for h in range(Hkv):
            L, x = int(lens[b, h]), q[b, h * G:(h + 1) * G].double()
            want, p = ref.attention(x, K[b, h, :L].double(), V[b, h, :L].double(), sm)
            assert float((got[b, h * G:(h + 1) * G] - want).abs().max()) <= ref.out_error(x, K[b, h, :L].double(), V[b, h, :L].double(), sm)
            if L:
                e = ref.weight_error(x, K[b, h, :L].double(), sm) + (L + 8) * ref.EPS     # (the sum that normalizes)
                total = w0[b, h, :L].double() + p.sum(0)
                assert bool(((acc[b, h, :L].double() - total).abs() <= p.sum(0) * e + (G + 1) * ref.EPS * total).all()), (b, h, L)
            assert bool((acc[b, h, L:] == 5.0).all()) and torch.equal(same[b, h, L:].cpu(), w0[b, h, L:])
            assert torch.equal(same[b, h, :L], weight[b, h, :L])
    assert int(status) == 0


def test_weigh_with_accounts_at_odd_addresses():
    """Accounts whose rows begin at no multiple of 16 bytes: the bits of the aligned ones."""
    g, B, Hq, Hkv, d, cap = _gen(4), 2, 4, 2, 64, 900
    lens = torch.tensor([[900, 77], [4, 899]], dtype=torch.int32)
    K, V, q = (x.to(DEV) for x in _state(g, B, Hq, Hkv, d, cap, "f32", lens))
    desc = corm.make_desc(B, Hq, Hkv, d, cap, cap, 1, 1, "f32")
    ws = torch.empty(corm.corm_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    w0 = torch.rand(B, Hkv, cap, generator=g).to(DEV)
    out, want = torch.empty(B, Hq, d, device=DEV), torch.zeros_like(w0)
    corm.corm_decode_attend_weigh(desc, q, K, V, lens.to(DEV), w0, want, out, ws)
    for off in (1, 2, 3):
        a, b = (torch.zeros(w0.numel() + 4, device=DEV)[off:off + w0.numel()].view_as(w0) for _ in range(2))
        a.copy_(w0)
        corm.corm_decode_attend_weigh(desc, q, K, V, lens.to(DEV), a, b, out, ws)
        assert torch.equal(b, want)


@pytest.mark.parametrize("units,cap,r,budget", [(3, 50, 1, 1), (4, 700, 16, 200), (2, 1024, 1, 1023), (5, 1500, 100, 100), (13, 4100, 64, 1000),
                                                (1, 9000, 3, 5000), (2, 16384, 10, 3000), (2, 16385, 50, 50), (2, 40000, 500, 2000), (3, 30001, 7, 9000),
                                                (1, 200000, 5, 70000)])
def test_evict_mask_weight(units, cap, r, budget):
    """Heavy-tailed accounts with zeros and many equal ones; lengths on both sides of the budget."""
    g = _gen(cap)
    w = torch.exp(3 * torch.randn(units, 1, cap, generator=g)) * (torch.rand(units, 1, cap, generator=g) > 0.2)
    w[0] = (w[0] * 4).round() / 4                                   # ties everywhere
    if units > 1:
        w[1] = 0.25
    if units > 2:
        w[2, 0, ::7], w[2, 0, 1::7], w[2, 0, 2::7], w[2, 0, 3::7] = float("nan"), float("inf"), -1.0, -0.0
    odd = [cap, budget, budget + 1, cap - 1, 0, 1, r, cap // 2]
    lens = torch.tensor([min(cap, odd[u % len(odd)]) for u in range(units)], dtype=torch.int32).view(units, 1)
    desc = corm.make_desc(units, 1, 1, 64, cap, cap, 1, r, "f32")
    keep = torch.full((units, 1, cap), 9, dtype=torch.uint8, device=DEV)
    corm.corm_evict_mask_weight(desc, w.to(DEV), lens.to(DEV), budget, keep, _ws(desc))
    for u in range(units):
        L = int(lens[u])
        assert keep[u, 0].tolist() == ref.kept(w[u, 0], L, r, budget) + [9] * (cap - L), (u, L)


def test_evict_mask_weight_of_many_long_units():
    """Many units of more slots than a workgroup holds: eight of them, over and over."""
    kinds, units, cap, r, budget = 8, 704, 20001, 9, 6000
    g = _gen(17)
    w = torch.exp(3 * torch.randn(kinds, 1, cap, generator=g)) * (torch.rand(kinds, 1, cap, generator=g) > 0.2)
    w[1] = 0.25
    w[2] = (w[2] * 4).round() / 4
    lens = torch.tensor([cap, cap, cap - 1, 12345, budget, budget + 1, 0, r], dtype=torch.int32)
    desc = corm.make_desc(units, 1, 1, 64, cap, cap, 1, r, "f32")
    keep = torch.full((units, 1, cap), 9, dtype=torch.uint8, device=DEV)
    corm.corm_evict_mask_weight(desc, w.repeat(units // kinds, 1, 1).to(DEV), lens.repeat(units // kinds).to(DEV), budget, keep, _ws(desc))
    for u in range(kinds):
        L = int(lens[u])
        want = torch.tensor(ref.kept(w[u, 0], L, r, budget) + [9] * (cap - L), dtype=torch.uint8)
        assert (keep[u::kinds, 0].cpu() == want).all(), (u, L)


# ---------------------------------------------------------------- together, as they would be used

def _layer(B, Hq, Hkv, d, cap, dtype, P, g, r=8):
    st = corm.LayerState(B, Hq, Hkv, d, cap, cap, 4, r, dtype, device=DEV, want_ring=False, want_bounds=True, want_weight=True)
    K, V = _rows(g, dtype, B, Hkv, P, d), _rows(g, dtype, B, Hkv, P, d)
    st.preload(K.to(DEV), V.to(DEV))
    return st, K, V


def test_weigh_steps_evict_and_go_on():
    """Twenty steps of eviction by attention weight, cut to the budget at every third: accounts, survivors, rows and outputs of a unit follow the plain form (slaved
    to the device's accounts, which decide)."""
    g, B, Hq, Hkv, d, P, r, budget = _gen(11), 2, 4, 2, 64, 90, 8, 60
    st, K, V = _layer(B, Hq, Hkv, d, 160, "f32", P, g, r)
    sm, G = 1.0 / math.sqrt(d), Hq // Hkv
    units = {(b, h): [[K[b, h, i] for i in range(P)], [V[b, h, i] for i in range(P)], list(range(P))] for b in range(B) for h in range(Hkv)}
    evicted = 0
    for s in range(20):
        q, k, v = _rows(g, "f32", B, Hq, d, scale=2.0), _rows(g, "f32", B, Hkv, d), _rows(g, "f32", B, Hkv, d)
        t = torch.full((B,), P + 1 + s, dtype=torch.int32, device=DEV)
        cut = s % 3 == 2
        before = st.weight.cpu().clone()
        lens0 = st.lens.cpu().clone()
        st.step_weigh(q.to(DEV), k.to(DEV), v.to(DEV), t, budget if cut else None)
        out, acc, lens, pos, Kd, Vd = (x.cpu() for x in (st.out, st.weight, st.lens, st.pos, st.K, st.V))
        for (b, h), (ks, vs, ps) in units.items():
            L0 = int(lens0[b, h])
            assert L0 == len(ks)
            ks.append(k[b, h])
            vs.append(v[b, h])
            ps.append(P + s)
            Kr, Vr, x = torch.stack(ks).double(), torch.stack(vs).double(), q[b, h * G:(h + 1) * G].double()
            want, p = ref.attention(x, Kr, Vr, sm)
            assert float((out[b, h * G:(h + 1) * G].double() - want).abs().max()) <= ref.out_error(x, Kr, Vr, sm)
            e = ref.weight_error(x, Kr, sm) + (L0 + 9) * ref.EPS
            total = torch.cat([before[b, h, :L0], torch.zeros(1)]).double() + p.sum(0)
            if cut and L0 + 1 > budget:
                keep = st.weight_keep[b, h, :L0 + 1].cpu().bool()
                idx = keep.nonzero().flatten().tolist()
                assert len(idx) == budget and all(i in idx for i in range(L0 + 1 - r, L0 + 1))
                # no key that went had clearly more than one that stayed (accounts are within e of the plain ones)
                old = total[:L0 + 1 - r]
                went, stayed = old[~keep[:L0 + 1 - r]], old[keep[:L0 + 1 - r]]
                assert float(went.max()) <= float(stayed.min()) * (1 + 4 * e)
                evicted += L0 + 1 - budget
                ks[:], vs[:], ps[:] = [ks[i] for i in idx], [vs[i] for i in idx], [ps[i] for i in idx]
                total, p = total[idx], p[:, idx]
            L = int(lens[b, h])
            assert L == len(ks) and pos[b, h, :L].tolist() == ps
            assert torch.equal(Kd[b, h, :L], torch.stack(ks)) and torch.equal(Vd[b, h, :L], torch.stack(vs))
            assert bool(((acc[b, h, :L].double() - total).abs() <= p.sum(0) * e + (G + 1) * ref.EPS * total).all())
    assert evicted > 0 and int(st.status) == 0
    bare = corm.LayerState(1, 1, 1, 64, 64, 64, 4, 4, "f32", device=DEV, want_ring=False)
    for step in (lambda: bare.step_weigh(None, None, None, None), lambda: bare.step_blocks(None, None, None, None, 1), bare.renew_bounds):
        with pytest.raises(RuntimeError):
            step()


def test_block_steps_follow_the_chosen_blocks():
    g, B, Hq, Hkv, d, P, nsel, nlast = _gen(12), 2, 8, 2, 128, 64 * 9 - 3, 4, 2
    st, K, V = _layer(B, Hq, Hkv, d, 64 * 11, "bf16", P, g)
    sm, G = 1.0 / math.sqrt(d), Hq // Hkv
    st.renew_bounds()
    for s in range(8):
        q, k, v = _rows(g, "bf16", B, Hq, d, scale=2.0), _rows(g, "bf16", B, Hkv, d), _rows(g, "bf16", B, Hkv, d)
        K, V = torch.cat([K, k.unsqueeze(2)], 2), torch.cat([V, v.unsqueeze(2)], 2)
        st.step_blocks(q.to(DEV), k.to(DEV), v.to(DEV), torch.full((B,), P + 1 + s, dtype=torch.int32, device=DEV), nsel, nlast)
        for b in range(B):
            for h in range(Hkv):
                x, n = q[b, h * G:(h + 1) * G], P + 1 + s
                want = ref.choose(x, ref.bounds_of(K[b, h]), nsel, nlast)
                assert st.blocks[b, h].tolist() == want
                slots = [i for w in want for i in range(64 * w, min(64 * w + 64, n))]
                Ks, Vs = K[b, h, slots].double(), V[b, h, slots].double()
                o, _ = ref.attention(x.double(), Ks, Vs, sm)
                assert float((st.out[b, h * G:(h + 1) * G].cpu().double() - o).abs().max()) <= ref.out_error(x.double(), Ks, Vs, sm)
    assert int(st.status) == 0


@pytest.mark.parametrize("code,dtype,nsel", [("i8", "bf16", 0), ("e4m3", "f32", 0), ("i8", "f32", 3), ("e4m3", "bf16", 3)])
def test_q8_state_prompt_and_steps(code, dtype, nsel):
    """A ragged prompt and then single tokens across block borders, over every block or the chosen ones."""
    g, B, Hq, Hkv, d, P = _gen(13), 2, 4, 2, 128, 64 * 5 + 60
    st = corm.Q8State(B, Hq, Hkv, d, 64 * 8, dtype, code, device=DEV, want_bounds=nsel > 0)
    plain = [[ref.Cache8(d, code) for _ in range(Hkv)] for _ in range(B)]
    rows = [[[] for _ in range(Hkv)] for _ in range(B)]
    n_new = [P, 64 * 2 + 62]

    def put(b, h, k, v):
        plain[b][h].append(k, v)
        rows[b][h].append(k.float())

    k, v = _rows(g, dtype, B, Hkv, P, d), _rows(g, dtype, B, Hkv, P, d)
    st.append(k.to(DEV), v.to(DEV), torch.tensor(n_new, dtype=torch.int32, device=DEV))
    for b in range(B):
        for h in range(Hkv):
            for i in range(n_new[b]):
                put(b, h, k[b, h, i], v[b, h, i])
    sm, G = 1.0 / math.sqrt(d), Hq // Hkv
    for s in range(7):
        q, k, v = _rows(g, dtype, B, Hq, d, scale=2.0), _rows(g, dtype, B, Hkv, d), _rows(g, dtype, B, Hkv, d)
        st.step(q.to(DEV), k.to(DEV), v.to(DEV), nsel, 1)
        for b in range(B):
            for h in range(Hkv):
                put(b, h, k[b, h], v[b, h])
                c, x = plain[b][h], q[b, h * G:(h + 1) * G]
                K, V = c.rows(0), c.rows(1)
                if nsel:
                    want = ref.choose(x, ref.bounds_of(torch.stack(rows[b][h])), nsel, 1)
                    assert st.blocks[b, h].tolist() == want
                    slots = [i for w in want for i in range(64 * w, min(64 * w + 64, c.n))]
                    K, V = K[slots], V[slots]
                o, _ = ref.attention(x.double(), K, V, sm)
                assert int(st.lens[b, h]) == c.n
                assert float((st.out[b, h * G:(h + 1) * G].cpu().double() - o).abs().max()) <= ref.out_error(x.double(), K, V, sm)
    assert int(st.status) == 0


def test_captured_steps_on_another_stream_repeat_the_eager_ones():
    """Two graphs that share a workspace, captured on a stream of their own and replayed in turn between eager work: the eager bits every time."""
    g, B, Hq, Hkv, d, P = _gen(14), 2, 8, 2, 128, 64 * 12 + 5
    lens = ref.lens_of(B, Hkv, P, "odd")
    K, V, q = (x.to(DEV) for x in _state(g, B, Hq, Hkv, d, P, "bf16", lens))
    lens = lens.to(DEV)
    desc = corm.make_desc(B, Hq, Hkv, d, P, P, 1, 8, "bf16")
    nblk = (P + 63) // 64
    ws, full = _ws(desc), torch.empty(corm.corm_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    c = corm.Q8State(B, Hq, Hkv, d, P, "bf16", "i8", device=DEV, want_bounds=True, workspace=ws)
    c.append(K.nan_to_num(), V.nan_to_num(), None)
    bounds = torch.zeros(B, Hkv, nblk, 2, d, dtype=torch.bfloat16, device=DEV)
    blocks = torch.zeros(B, Hkv, 3, dtype=torch.int32, device=DEV)
    w0 = torch.rand(B, Hkv, P, device=DEV)
    w1, keep = torch.zeros_like(w0), torch.zeros(B, Hkv, P, dtype=torch.uint8, device=DEV)
    outs = [torch.zeros(B, Hq, d, device=DEV) for _ in range(2)]

    def first():
        corm.corm_block_bounds(desc, K, lens, bounds)
        corm.corm_block_select(desc, q, bounds, lens, 3, 1, blocks, ws)
        corm.corm_block_attend(desc, q, K, V, lens, blocks, 3, outs[0], ws)
        corm.corm_decode_attend_weigh(desc, q, K, V, lens, w0, w1, outs[1], full)

    def second():
        c.attend(q, 4, 1)
        corm.corm_evict_mask_weight(desc, w1, lens, 100, keep, ws)

    watched = [bounds, blocks, w1, keep, c.out, *outs]
    first()
    second()
    torch.cuda.synchronize()
    want = [x.clone() for x in watched]
    s = torch.cuda.Stream()
    graphs = []
    for f in (first, second):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            f()
        graphs.append(gr)
    for _ in range(3):
        for x in watched:
            x.zero_()
        graphs[0].replay()
        torch.randn(1000, device=DEV).sum().item()
        graphs[1].replay()
        torch.cuda.synchronize()
        for x, y in zip(watched, want):
            assert torch.equal(x, y)
    for x in watched:                      # given a stream that is not the current one
        x.zero_()
    torch.cuda.synchronize()
    corm.corm_block_bounds(desc, K, lens, bounds, stream=s)
    corm.corm_block_select(desc, q, bounds, lens, 3, 1, blocks, ws, stream=s)
    corm.corm_block_attend(desc, q, K, V, lens, blocks, 3, outs[0], ws, stream=s)
    s.synchronize()
    for x, y in zip((bounds, blocks, outs[0]), (want[0], want[1], want[5])):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_that_are_none_are_clamped_and_flagged(dtype):
    """-3 and Lcap + 5: what 0 and Lcap give, in every call that reads lengths, and the flag where the call has one."""
    g, B, Hq, Hkv, d, cap = _gen(31), 2, 4, 1, 64, 64 * 9 + 7
    good, bad = torch.tensor([[0], [cap]], dtype=torch.int32, device=DEV), torch.tensor([[-3], [cap + 5]], dtype=torch.int32, device=DEV)
    K, V, q = (x.to(DEV) for x in _state(g, B, Hq, Hkv, d, cap, dtype, torch.full((B, Hkv), cap)))
    desc = corm.make_desc(B, Hq, Hkv, d, cap, cap, 1, 4, dtype)
    full = torch.empty(corm.corm_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    c = Q8(B, Hq, Hkv, d, cap, dtype, "i8")
    c.append(K.cpu(), V.cpu())
    w0 = torch.rand(B, Hkv, cap, device=DEV)
    blocks = torch.arange(10, dtype=torch.int32, device=DEV).view(1, 1, 10).repeat(B, 1, 1)
    blocks[0] = -1
    got = []
    for lens in (good, bad):
        status = torch.zeros(3, dtype=torch.int32, device=DEV)
        outs = [torch.full((B, Hq, d), 3.0, device=DEV) for _ in range(3)]
        bounds = torch.zeros(B, Hkv, 10, 2, d, dtype=DT[dtype], device=DEV)
        picked, weight = torch.zeros(B, Hkv, 4, dtype=torch.int32, device=DEV), torch.zeros(B, Hkv, cap, device=DEV)
        keep = torch.zeros(B, Hkv, cap, dtype=torch.uint8, device=DEV)
        corm.corm_q8_attend(desc, "i8", q, c.Kc, c.Vc, c.ks, c.vs, c.Kt, c.Vt, lens, outs[0], c.ws, status=status[0:1])
        corm.corm_block_attend(desc, q, K, V, lens, blocks, 10, outs[1], c.ws, status=status[1:2])
        corm.corm_decode_attend_weigh(desc, q, K, V, lens, w0, weight, outs[2], full, status=status[2:3])
        corm.corm_block_bounds(desc, K, lens, bounds)
        corm.corm_block_select(desc, q, bounds, lens, 4, 1, picked, c.ws)
        corm.corm_evict_mask_weight(desc, w0, lens, 100, keep, c.ws)
        got.append([*outs, weight, bounds, picked, keep])
        assert status.tolist() == ([0] * 3 if lens is good else [corm.CORM_DEV_BAD_LENS] * 3)
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert not got[0][0][0].any() and bool(got[0][0][1].any())


@pytest.mark.parametrize("dtype,G", [("bf16", 4), ("bf16", 1), ("f32", 2)])
def test_lists_of_the_most_blocks(dtype, G):
    """512 places for a unit of nine blocks, most of them empty, some blocks several times."""
    g, d, cap, n = _gen(33), 128, 64 * 9, 512
    lens = torch.tensor([[cap - 10], [200]], dtype=torch.int32)
    K, V, q = _state(g, 2, G, 1, d, cap, dtype, lens)
    desc = corm.make_desc(2, G, 1, d, cap, cap, 1, 1, dtype)
    blocks = torch.full((2, 1, n), -1, dtype=torch.int32)
    for b, many in ((0, 9), (1, 4)):
        at = torch.randperm(n, generator=g)[:40]
        blocks[b, 0, at] = torch.randint(0, many, (40,), generator=g, dtype=torch.int32)
    sm, ws = 1.0 / math.sqrt(d), _ws(desc)
    out = torch.full((2, G, d), float("nan"), device=DEV)
    corm.corm_block_attend(desc, q.to(DEV), K.to(DEV), V.to(DEV), lens.to(DEV), blocks.to(DEV), n, out, ws)
    c = Q8(2, G, 1, d, cap, dtype, "e4m3")
    c.append(K.nan_to_num(), V.nan_to_num(), lens.flatten().tolist())
    c.attend(q, blocks.tolist())
    c.check_out(q, blocks.tolist())
    for b in range(2):
        slots = [s for i in blocks[b, 0].tolist() if i >= 0 for s in range(64 * i, min(64 * i + 64, int(lens[b])))]
        x, Ks, Vs = q[b].double(), K[b, 0, slots].double(), V[b, 0, slots].double()
        want, _ = ref.attention(x, Ks, Vs, sm)
        assert float((out[b].cpu().double() - want).abs().max()) <= ref.out_error(x, Ks, Vs, sm)


def test_what_is_not_a_number_stays_none():
    """A query that is not a number gives outputs that are none, of its head alone, also where partials are joined."""
    g, d = _gen(22), 64
    for P in (40, 64 * 3, 64 * 30 + 7):
        c = Q8(1, 2, 1, d, 64 * 31, "bf16", "i8")
        c.append(_rows(g, "bf16", 1, 1, P, d), _rows(g, "bf16", 1, 1, P, d))
        q = _rows(g, "bf16", 1, 2, d)
        q[0, 1, 3] = float("nan")
        c.attend(q)
        assert bool(c.out[0, 1].isnan().all()) and not bool(c.out[0, 0].isnan().any()), P
        K, V = (_rows(g, "bf16", 1, 1, 64 * 31, d).to(DEV) for _ in range(2))
        out = torch.zeros(1, 2, d, device=DEV)
        blocks = torch.arange(31, dtype=torch.int32, device=DEV).view(1, 1, 31)
        corm.corm_block_attend(c.desc, q.to(DEV), K, V, torch.tensor([[64 * 31]], dtype=torch.int32, device=DEV), blocks, 31, out, c.ws)
        assert bool(out[0, 1].isnan().all()) and not bool(out[0, 0].isnan().any())


def test_tensors_that_do_not_fit_the_call_are_refused():
    desc = corm.make_desc(1, 2, 1, 64, 128, 128, 1, 1, "bf16")
    ws = _ws(desc)
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device=DEV)
    K = torch.zeros(1, 1, 128, 64, dtype=torch.bfloat16, device=DEV)
    lens = torch.ones(1, 1, dtype=torch.int32, device=DEV)
    blocks = torch.zeros(1, 1, 2, dtype=torch.int32, device=DEV)
    out = torch.zeros(1, 2, 64, device=DEV)
    good = dict(q=q, K=K, V=K, lens=lens, blocks=blocks, nsel=2, out=out, workspace=ws)
    corm.corm_block_attend(desc, **good)
    for name, bad in (("q", q.float()), ("K", K[:, :, ::2]), ("K", K[:, :, :64].contiguous()), ("K", K.repeat(1, 1, 2, 1)), ("lens", lens.long()), ("out", out.cpu()),
                      ("blocks", blocks[:, :, :1]), ("workspace", ws[::2]), ("workspace", ws.cpu())):
        with pytest.raises(ValueError):
            corm.corm_block_attend(desc, **{**good, name: bad})


def test_units_beyond_four_gigabytes():
    """Forty units of a million slots: the last one lies 5 GB (codes) and 10 GB (rows) into its array, its keys at the end of a unit."""
    g, units, cap, d, G = _gen(15), 40, 1 << 20, 128, 2
    desc = corm.make_desc(units, G, 1, d, cap, cap, 1, 1, "bf16")
    n, u, sm = cap // 64, units - 1, 1.0 / math.sqrt(d)
    lens = torch.zeros(units, 1, dtype=torch.int32, device=DEV)
    lens[u] = cap - 3
    last = [n - 1, n - 2, 5]
    k, v, q = _rows(g, "bf16", 64 * 3, d), _rows(g, "bf16", 64 * 3, d), _rows(g, "bf16", units, G, d)
    ws, out = _ws(desc), torch.full((units, G, d), float("nan"), device=DEV)
    blocks = torch.full((units, 1, 4), -1, dtype=torch.int32, device=DEV)
    blocks[u, 0, :3] = torch.tensor(last, dtype=torch.int32)
    K = torch.empty(units, 1, n, 64, d, dtype=torch.bfloat16, device=DEV)
    V = torch.empty_like(K)
    for i, blk in enumerate(last):
        K[u, 0, blk], V[u, 0, blk] = k[64 * i:64 * i + 64].to(DEV), v[64 * i:64 * i + 64].to(DEV)
    corm.corm_block_attend(desc, q.to(DEV), K, V, lens, blocks, 4, out, ws)
    live = [i for i in range(192) if not 61 <= i < 64]          # (three slots of the last block are not in use)
    x, Kr, Vr = q[u].double(), k[live].double(), v[live].double()
    want, _ = ref.attention(x, Kr, Vr, sm)
    assert float((out[u].cpu().double() - want).abs().max()) <= ref.out_error(x, Kr, Vr, sm) and not out[:u].any()
    bounds = torch.empty(units, 1, n, 2, d, dtype=torch.bfloat16, device=DEV)
    corm.corm_block_bounds(desc, K, lens, bounds, newest=1)
    assert torch.equal(bounds[u, 0, n - 1].cpu().float(), ref.bounds_of(k[:61].float())[0])
    del K, V, bounds
    Kc = torch.empty(units, 1, n, 2, 64, 64, dtype=torch.int8, device=DEV)
    Vc = torch.empty(units, 1, n, d, 64, dtype=torch.int8, device=DEV)
    ks, vs = torch.zeros(units, 1, n, device=DEV), torch.zeros(units, 1, n, device=DEV)
    Kt, Vt = torch.zeros(units, 1, 64, d, dtype=torch.bfloat16, device=DEV), torch.zeros(units, 1, 64, d, dtype=torch.bfloat16, device=DEV)
    for i, blk in enumerate((n - 2, 5)):                        # the append that fills block n - 2, and block 5 by hand
        lens[u] = blk * 64
        rows = [torch.zeros(units, 1, 64, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        rows[0][u, 0], rows[1][u, 0] = k[64 * i:64 * i + 64].to(DEV), v[64 * i:64 * i + 64].to(DEV)
        only = torch.zeros(units, dtype=torch.int32, device=DEV)
        only[u] = 64
        corm.corm_q8_append(desc, "i8", *rows, 64, only, Kc, Vc, ks, vs, Kt, Vt, lens, lens)
    lens[u] = (n - 1) * 64
    blocks[u, 0, :3] = torch.tensor([n - 2, 5, -1], dtype=torch.int32)
    corm.corm_q8_attend(desc, "i8", q.to(DEV), Kc, Vc, ks, vs, Kt, Vt, lens, out, ws, blocks=blocks, nsel=4)
    c = ref.Cache8(d, "i8")
    for i in range(128):
        c.append(k[i], v[i])
    want, _ = ref.attention(x, c.rows(0), c.rows(1), sm)
    assert float((out[u].cpu().double() - want).abs().max()) <= ref.out_error(x, c.rows(0), c.rows(1), sm) and not out[:u].any()
