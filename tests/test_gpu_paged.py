"""Rows normed and rotated, the cache of pages and attention over it against plain 64-bit forms, on the device."""
import pytest
import torch

from paper_2404_15949_amd import corm
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(g, dtype, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(DT[dtype])


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _nan(*shape, dtype="f32"):
    return torch.full(shape, float("nan"), dtype=DT[dtype], device=DEV)


def _same(a, b):
    """equal, what is not a number taken for equal to itself"""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())


def _freq(rot, base=10000.0):
    return (base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float() if rot else None


class Turn:
    """A rotation, on the device and as the plain form takes it."""

    def __init__(self, g, dtype, d, rot=None, pairing="halves", sections=None, in_turn=False, norm=True, gain=1.0, eps=1e-5):
        rot = d if rot is None else rot
        self.freq, self.pairing, self.in_turn, self.gain, self.eps = _freq(rot), pairing, in_turn, gain, eps
        self.sections = [rot // 2] if sections is None else sections
        self.w = [(1 + 0.3 * torch.randn(d, generator=g)).to(DT[dtype]) if norm else None for _ in range(2)]
        dev = [None if x is None else x.to(DEV) for x in [self.freq] + self.w]
        self.c = corm.Rotation(dev[0], q_norm=dev[1], k_norm=dev[2], eps=eps, pairing=pairing, sections=self.sections, in_turn=in_turn, gain=gain)

    def plain(self, x, which, pos):
        eps = torch.tensor(self.eps, dtype=torch.float32).double().item()
        return ref.turn(x, self.w[which], eps, self.freq, pos, self.sections, self.in_turn, self.pairing, torch.tensor(self.gain).double().item())


def _packed(g, dtype, B, Hq, Hkv, n, d, pad=0):
    """q, k, v as views of a projection's rows (pad more elements between the tokens), on the device, and the same on the CPU"""
    x = _normal(g, dtype, B, n, (Hq + 2 * Hkv) * d + pad, scale=2.0)
    def cut(y):
        return y[:, :, :(Hq + 2 * Hkv) * d].unflatten(2, (Hq + 2 * Hkv, d)).transpose(1, 2).split([Hq, Hkv, Hkv], 1)
    return cut(x.to(DEV)), cut(x)


def _close(got, want, bound, dtype, where):
    """`bound` before the rounding to the type, half a step (of what is rounded) in it"""
    got = got.cpu().double()
    slack = bound + ref.HALF[dtype] * (want.abs() + bound)
    worst = ((got - want).abs() - slack).max()
    assert not got.isnan().any() and float(worst) <= 0, (where, float(worst))


TURNS = [
    dict(), dict(pairing="neighbours"), dict(rot=16), dict(rot=48, pairing="neighbours", norm=False), dict(norm=False, gain=1.25),
    dict(sections=[16, 8, 8], rot=64), dict(sections=[12, 10, 10], rot=64, in_turn=True), dict(sections=[8, 0, 16, 8], rot=64, pairing="neighbours"),
    dict(sections=[20, 12], rot=64, in_turn=True, norm=False), dict(rot=0),
]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("kind", range(len(TURNS)))
def test_rotate(dtype, d, kind):
    g = _gen(100 * kind + d)
    for B, Hq, Hkv, n, n_new in ((1, 1, 1, 1, None), (3, 8, 2, 7, None), (2, 6, 3, 19, [19, 4]), (2, 32, 4, 1, [0, 5]), (1, 5, 5, 600, None)):
        t = Turn(g, dtype, d, **TURNS[kind])
        (q, k, v), (cq, ck, cv) = _packed(g, dtype, B, Hq, Hkv, n, d, pad=8 * (n % 3))
        pos = torch.randint(-5, 4000, (len(t.sections), B, n), generator=g, dtype=torch.int32)
        desc = corm.make_desc(B, Hq, Hkv, d, n, n, 1, 1, dtype)
        outs = _nan(B, Hq, n, d, dtype=dtype), _nan(B, Hkv, n, d, dtype=dtype), _nan(B, Hkv, n, d, dtype=dtype)
        corm.corm_rotate(desc, q, k, v, t.c, pos.to(DEV), *outs, n_new=None if n_new is None else _i32(n_new))
        want = t.plain(cq, 0, pos), t.plain(ck, 1, pos), (cv.double(), torch.zeros(cv.shape).double())
        for b in range(B):
            take = n if n_new is None else min(max(n_new[b], 0), n)
            for i, (o, (w, e)) in enumerate(zip(outs, want)):
                if take:
                    if i == 2:
                        assert torch.equal(o[b, :, :take].cpu(), cv[b, :, :take])
                    else:
                        _close(o[b, :, :take], w[b, :, :take], e[b, :, :take], dtype, (B, Hq, n, b, i))
                assert bool(o[b, :, take:].isnan().all())
        only = _nan(B, Hkv, n, d, dtype=dtype), _nan(B, Hkv, n, d, dtype=dtype)      # without queries: the same keys
        corm.corm_rotate(desc, None, k, v, t.c, pos.to(DEV), None, *only, n_new=None if n_new is None else _i32(n_new))
        assert _same(only[0], outs[1]) and _same(only[1], outs[2])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("kind", [0, 1, 2, 6, 9])
def test_rotate_long_prompts(dtype, d, kind):
    """As many tokens as are taken in groups: odd numbers of them, a ragged batch, sequences without any."""
    g = _gen(200 + kind)
    for B, Hq, Hkv, n, n_new in ((6, 4, 2, 701, [701, 0, 700, 5, 698, 1]), (1, 3, 3, 4099, None)):
        t = Turn(g, dtype, d, **TURNS[kind])
        (q, k, v), (cq, ck, cv) = _packed(g, dtype, B, Hq, Hkv, n, d)
        pos = torch.randint(0, 200000, (len(t.sections), B, n), generator=g, dtype=torch.int32)
        outs = _nan(B, Hq, n, d, dtype=dtype), _nan(B, Hkv, n, d, dtype=dtype), _nan(B, Hkv, n, d, dtype=dtype)
        corm.corm_rotate(corm.make_desc(B, Hq, Hkv, d, n, n, 1, 1, dtype), q, k, v, t.c, pos.to(DEV), *outs, n_new=None if n_new is None else _i32(n_new))
        want = t.plain(cq, 0, pos), t.plain(ck, 1, pos)
        for b in range(B):
            take = n if n_new is None else n_new[b]
            assert all(bool(o[b, :, take:].isnan().all()) for o in outs) and torch.equal(outs[2][b, :, :take].cpu(), cv[b, :, :take])
            for i in range(2 if take else 0):
                _close(outs[i][b, :, :take], want[i][0][b, :, :take], want[i][1][b, :, :take], dtype, (B, n, b, i))


@pytest.mark.parametrize("dtype,code", [("bf16", None), ("f32", None), ("bf16", "i8"), ("bf16", "e4m3"), ("f32", "i8"), ("f32", "e4m3")])
@pytest.mark.parametrize("d,per_head", [(128, False), (64, True)])
def test_append_long_prompts(dtype, code, d, per_head):
    """Groups of tokens into pages, the lengths replaced in place: ragged, behind rows that are there, without room, without a page."""
    g = _gen(24)
    B, n = 6, 701
    c = Cache(g, B, 2, 2, d, 1500, dtype, code, 32, per_head)
    c.append(_normal(g, dtype, B, 2, 7, d), _normal(g, dtype, B, 2, 7, d), [7, 0, 1, 3, 7, 2])
    for n_new in ([701, 0, 700, 5, 698, 1], [701, 701, 701, 701, 701, 0]):
        c.append(_normal(g, dtype, B, 2, n, d), _normal(g, dtype, B, 2, n, d, scale=9.0), n_new)
        c.check()
    assert int(c.status) == 0
    c.append(_normal(g, dtype, B, 2, n, d), _normal(g, dtype, B, 2, n, d), [701, 701, 701, 0, 90, 701])       # no room in the first, the third
    c.check()
    assert int(c.status) == corm.CORM_DEV_UNIT_FULL
    q = _normal(g, dtype, B, 2, d, scale=2.0)
    c.attend(q)
    c.check_out(q)
    c = Cache(g, B, 2, 2, d, 704, dtype, code, 32, per_head)
    c.dev_table[2, 0, 3] = -1
    c.append(_normal(g, dtype, B, 2, n, d), _normal(g, dtype, B, 2, n, d), None)
    assert int(c.status) == corm.CORM_DEV_BAD_PAGE and bool((c.lens == n).all())
    c.attend(q)
    c.check_out(q, lambda b, h: range(96, 128) if b == 2 and (h == 0 or not per_head) else ())


def test_rows_of_any_strides():
    """Rows shared by heads and sequences (stride 0), tokens apart by more than a row, every layout the same rows."""
    g = _gen(25)
    t = Turn(g, "bf16", 128)
    B, n = 2, 33
    desc = corm.make_desc(B, 4, 2, 128, n, n, 1, 1, "bf16")
    pos = torch.arange(B * n, dtype=torch.int32, device=DEV).view(1, B, n)
    one = _normal(g, "bf16", 1, 1, n, 128).to(DEV)
    q, k = one.expand(B, 4, n, 128), one.expand(B, 2, n, 128)
    v = _normal(g, "bf16", n, 2, 3, B, 128).to(DEV)[:, :, 1].permute(2, 1, 0, 3)
    outs = []
    for x in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
        o = [_nan(B, h, n, 128, dtype="bf16") for h in (4, 2, 2)]
        corm.corm_rotate(desc, *x, t.c, pos, *o)
        outs.append(o)
    assert all(torch.equal(a, b) for a, b in zip(*outs)) and torch.equal(outs[0][2], v.contiguous())
    bad = _normal(g, "bf16", B, 4, n, 132).to(DEV)[..., :128]           # rows that are not 16 bytes apart
    with pytest.raises(corm.CormError):
        corm.corm_rotate(desc, bad, k, v, t.c, pos, *outs[0])
    with pytest.raises(ValueError):                                     # channels that do not lie together
        corm.corm_rotate(desc, q, k, v.transpose(2, 3).contiguous().transpose(2, 3), t.c, pos, *outs[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rotate_far_positions(dtype):
    """Angles of positions up to the largest int32 are as exact as near ones."""
    g = _gen(7)
    pos = torch.tensor([[[0, 1, 131071, 1000003, 16777217, 2147483647, -2147483648, -77]]], dtype=torch.int32)
    t = Turn(g, dtype, 128, norm=False)
    (q, k, v), (cq, ck, _) = _packed(g, dtype, 1, 4, 2, 8, 128)
    outs = _nan(1, 4, 8, 128, dtype=dtype), _nan(1, 2, 8, 128, dtype=dtype), _nan(1, 2, 8, 128, dtype=dtype)
    corm.corm_rotate(corm.make_desc(1, 4, 2, 128, 8, 8, 1, 1, dtype), q, k, v, t.c, pos.to(DEV), *outs)
    for o, x, i in ((outs[0], cq, 0), (outs[1], ck, 1)):
        w, e = t.plain(x, i, pos)
        # (an angle of 2^31 rad is off by 2^-53 of itself in 64 bits, twice: 5e-7 rad; beside that the bound of near ones)
        pair = x.double().abs()
        pair = pair + torch.cat([pair[..., 64:], pair[..., :64]], -1)
        _close(o, w, e + 2.0 ** -52 * pos[0, 0].double().abs().view(1, 1, 8, 1) * pair * 1.1, dtype, i)


def test_rotate_rows_that_are_not_numbers_stay_apart():
    """A row with an infinite element does not reach another; rows of zeros stay zeros."""
    g = _gen(8)
    t = Turn(g, "bf16", 128)
    (q, k, v), _ = _packed(g, "bf16", 2, 4, 2, 5, 128)
    clean = [x.clone() for x in (q, k, v)]
    bad = [x.clone() for x in clean]
    bad[0][1, 2, 3, 17] = float("inf")
    bad[1][0, 1, 2] = float("nan")
    bad[0][0, 0, 0], clean[0][0, 0, 0] = 0, 0
    pos = torch.arange(10, dtype=torch.int32, device=DEV).view(1, 2, 5)
    outs = []
    for x in (clean, bad):
        o = [torch.zeros(2, h, 5, 128, dtype=torch.bfloat16, device=DEV) for h in (4, 2, 2)]
        corm.corm_rotate(corm.make_desc(2, 4, 2, 128, 5, 5, 1, 1, "bf16"), *x, t.c, pos, *o)
        outs.append(o)
    outs[1][0][1, 2, 3] = outs[0][0][1, 2, 3]
    outs[1][1][0, 1, 2] = outs[0][1][0, 1, 2]
    assert all(torch.equal(a, b) for a, b in zip(*outs)) and not outs[0][0][0, 0, 0].any()


# ---------------------------------------------------------------- pages

class Cache:
    """A pool full of junk, tables with junk behind their last page, and the rows that units hold, beside it."""

    def __init__(self, g, B, Hq, Hkv, d, most, dtype, code=None, page=16, per_head=False, spare=3):
        self.B, self.Hq, self.Hkv, self.d, self.dtype, self.code, self.page, self.per_head = B, Hq, Hkv, d, dtype, code, page, per_head
        self.TH = Hkv if per_head else 1
        self.max_pages = (most + page - 1) // page
        self.desc = corm.make_desc(B, Hq, Hkv, d, most, most, 1, 1, dtype)
        self.npages = B * self.TH * self.max_pages + spare
        order = torch.randperm(self.npages, generator=g)[:B * self.TH * self.max_pages]
        self.table = order.to(torch.int32).view(B, self.TH, self.max_pages)
        shape = (self.npages,) + (() if per_head else (Hkv,)) + (page, d)
        if code:
            self.K, self.V = (torch.full(shape, 0x7F, dtype=torch.int8, device=DEV).view(CODE[code]) for _ in range(2))
            self.ks, self.vs = _nan(*shape[:-1]), _nan(*shape[:-1])
        else:
            self.K, self.V, self.ks, self.vs = _nan(*shape, dtype=dtype), _nan(*shape, dtype=dtype), None, None
        self.dev_table = self.table.to(DEV)
        self.pages = corm.Pages(self.desc, self.K, self.V, self.dev_table, self.ks, self.vs)
        self.lens = torch.zeros(B, self.TH, dtype=torch.int32, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.rows = [[[[], []] for _ in range(Hkv)] for _ in range(B)]     # of a unit: lists of keys and values, as they came
        self.out = _nan(B, Hq, d)
        self.ws = torch.full((corm.corm_paged_workspace_bytes(self.desc),), 0xA5, dtype=torch.uint8, device=DEV)

    def length(self, b, h):
        return len(self.rows[b][h][0])

    def append(self, k, v, n_new=None, **kw):
        """k, v [B,Hkv,n,d] on the CPU"""
        corm.corm_paged_append(self.desc, self.pages, k.to(DEV), v.to(DEV), self.lens, self.lens,
                               n_new=None if n_new is None else _i32(n_new), status=self.status, **kw)
        for b in range(self.B):
            take = k.shape[2] if n_new is None else min(max(n_new[b], 0), k.shape[2])
            for h in range(self.Hkv):
                if self.length(b, h) + take <= self.desc.Lcap:
                    for j, x in enumerate((k, v)):
                        self.rows[b][h][j] += list(x[b, h, :take])

    def fill(self, g, lens, scale=(1.0, 1.0)):
        """Units of the given lengths [B][TH], by one append of so many rows each (per table, since a call brings a sequence's heads as many)."""
        top = max(max(r) for r in lens)
        if not top:
            return
        k = _normal(g, self.dtype, self.B, self.Hkv, top, self.d, scale=scale[0])
        v = _normal(g, self.dtype, self.B, self.Hkv, top, self.d, scale=scale[1])
        corm.corm_paged_append(self.desc, self.pages, k.to(DEV), v.to(DEV), self.lens, self.lens, status=self.status)
        self.lens.copy_(_i32(lens))       # shorter ones: what lies behind is junk to them
        for b in range(self.B):
            for h in range(self.Hkv):
                n = lens[b][h if self.per_head else 0]
                self.rows[b][h] = [list(k[b, h, :n]), list(v[b, h, :n])]

    def unit(self, b, h, j):
        """The rows that a unit's slots stand for, 64 bits"""
        x = self.rows[b][h][j]
        if not x:
            return torch.zeros(0, self.d).double()
        x = torch.stack(x)
        if not self.code:
            return x.double()
        c, s = ref.quantise_rows(x, self.code)
        return c.double() * s.double().unsqueeze(-1)

    def where(self, b, h, n):
        """Index into the pool of slots 0 .. n-1 of a unit"""
        at = torch.arange(n)
        ids = self.table[b, h if self.per_head else 0].long()[at // self.page]
        return (ids, at % self.page) if self.per_head else (ids, torch.full_like(ids, h), at % self.page)

    def check(self):
        """Every row, code and scale to the bit; what no unit holds is as it was."""
        K, V = self.K.cpu().float(), self.V.cpu().float()
        ks, vs = (None, None) if not self.code else (self.ks.cpu(), self.vs.cpu())
        used = torch.zeros(K.shape[:-1], dtype=torch.bool)
        lens = self.lens.cpu()
        for b in range(self.B):
            for h in range(self.Hkv):
                n = self.length(b, h)
                assert int(lens[b, h if self.per_head else 0]) == n, (b, h, n)
                if not n:
                    continue
                at = self.where(b, h, n)
                used[at] = True
                for j, (pool, sc) in enumerate(((K, ks), (V, vs))):
                    want = torch.stack(self.rows[b][h][j])
                    if self.code:
                        c, s = ref.quantise_rows(want, self.code)
                        assert torch.equal(pool[at], c), (b, h, n, j)
                        assert torch.equal(sc[at], s), (b, h, n, j)
                    else:
                        assert torch.equal(pool[at], want.float()), (b, h, n, j)
        if self.code:
            assert bool((self.K.view(torch.int8).cpu()[~used] == 0x7F).all()) and bool((self.V.view(torch.int8).cpu()[~used] == 0x7F).all())
            assert bool(ks[~used].isnan().all()) and bool(vs[~used].isnan().all())
        else:
            assert bool(K[~used].isnan().all()) and bool(V[~used].isnan().all())

    def attend(self, q):
        self.out.fill_(float("nan"))
        corm.corm_paged_attend(self.desc, self.pages, q.to(DEV), self.lens, self.out, self.ws, status=self.status)

    def check_out(self, q, skip=None):
        """skip(b, h): slots of a unit that are not to be seen"""
        G, got, sm = self.Hq // self.Hkv, self.out.cpu().double(), ref.sm_of(self.d)
        for b in range(self.B):
            for h in range(self.Hkv):
                K, V = self.unit(b, h, 0), self.unit(b, h, 1)
                if skip is not None:
                    keep = torch.ones(K.shape[0], dtype=torch.bool)
                    keep[[s for s in skip(b, h) if s < K.shape[0]]] = False
                    K, V = K[keep], V[keep]
                x = q[b, h * G:(h + 1) * G].double()
                err = (got[b, h * G:(h + 1) * G] - ref.attend(x, K, V, sm)).abs().max()
                assert float(err) <= ref.attend_error(x, K, V, sm), (b, h, K.shape[0], float(err), ref.attend_error(x, K, V, sm))


FORMS = [("bf16", None), ("f32", None), ("bf16", "i8"), ("bf16", "e4m3"), ("f32", "i8"), ("f32", "e4m3")]


@pytest.mark.parametrize("dtype,code", FORMS)
@pytest.mark.parametrize("d,page,per_head", [(128, 16, False), (64, 64, True), (128, 256, True), (64, 32, False), (128, 128, False)])
def test_append_in_pieces(dtype, code, d, page, per_head):
    g = _gen(11)
    c = Cache(g, 3, 4, 2, d, 300, dtype, code, page, per_head)
    for n, n_new in ((1, None), (15, None), (1, [1, 0, 1]), (1, None), (64, [64, 63, 1]), (130, [3, 130, 129]), (1, None), (5, [-3, 99, 2])):
        c.append(_normal(g, dtype, 3, 2, n, d), _normal(g, dtype, 3, 2, n, d, scale=30.0), n_new)
        c.check()
    assert int(c.status) == 0
    # to the last slot, and one too many: a sequence without room gets none, the others theirs
    left = 300 - c.length(1, 0)
    c.append(_normal(g, dtype, 3, 2, left, d), _normal(g, dtype, 3, 2, left, d), [0, left, 1])
    c.check()
    assert int(c.status) == 0
    c.append(_normal(g, dtype, 3, 2, 2, d), _normal(g, dtype, 3, 2, 2, d), [2, 1, 0])
    c.check()
    assert int(c.status) == corm.CORM_DEV_UNIT_FULL


@pytest.mark.parametrize("dtype,code", FORMS)
def test_append_special_rows(dtype, code):
    """Rows of zeros, tiny and huge ones, single large elements, borders of the codes' steps; rows with an element that is none have a scale that is none."""
    g = _gen(12)
    d = 128
    k = _normal(g, dtype, 1, 2, 10, d)
    k[0, 0, 0] = 0
    k[0, 0, 1] *= 1e-32
    k[0, 0, 2] *= 1e-30
    k[0, 0, 3] *= 1e30
    k[0, 0, 4] = 0
    k[0, 0, 4, 77] = -3.0
    k[0, 0, 5] = (torch.arange(d) - 63.5).to(DT[dtype])
    k[0, 0, 6] = torch.arange(d).sub(64).mul(7).to(DT[dtype])
    k[0, 0, 6, 0] = 448
    c = Cache(g, 1, 2, 2, d, 32, dtype, code, 16, True)
    c.append(k, k.flip(2))
    c.check()
    if code:
        k[0, 1, 3, 5], k[0, 1, 4, 9] = float("inf"), float("nan")
        c = Cache(g, 1, 2, 2, d, 32, dtype, code, 16, True)
        corm.corm_paged_append(c.desc, c.pages, k.to(DEV), k.to(DEV), c.lens, c.lens)
        at = c.where(0, 1, 10)
        assert c.ks.cpu()[at].isnan().tolist() == [i in (3, 4) for i in range(10)]


def test_append_lengths_that_are_none_and_lens_out():
    g = _gen(13)
    c = Cache(g, 3, 2, 2, 64, 40, "bf16", None, 16, True)
    lens, out = _i32([[-1, 3], [41, 40], [0, 39]]), _i32([[9, 9]] * 3)
    before = lens.clone()
    one = torch.ones(3, 2, 64, dtype=torch.bfloat16, device=DEV)
    corm.corm_paged_append(c.desc, c.pages, one, one, lens, out, status=c.status)
    assert torch.equal(lens, before) and out.tolist() == [[-1, 4], [41, 40], [1, 40]]
    assert int(c.status) == corm.CORM_DEV_BAD_LENS | corm.CORM_DEV_UNIT_FULL
    K = c.K.cpu().float()
    written = ~K.isnan().any(-1)
    want = torch.zeros_like(written)
    for b, h, s in ((0, 1, 3), (2, 0, 0), (2, 1, 39)):
        want[int(c.table[b, h, s // 16]), s % 16] = True
    assert torch.equal(written, want)


def test_pages_that_are_none():
    """Slots whose table entry is no page are neither written nor read; the others of the call are."""
    g = _gen(14)
    for bad_id in (-1, -2147483648, 2147483647, None):
        for code in (None, "e4m3"):
            c = Cache(g, 2, 4, 2, 128, 100, "bf16", code, 16, False)
            bad = c.npages if bad_id is None else bad_id
            c.dev_table[0, 0, 1], c.dev_table[1, 0, 6] = bad, bad
            k, v = _normal(g, "bf16", 2, 2, 100, 128), _normal(g, "bf16", 2, 2, 100, 128)
            c.append(k, v)
            assert int(c.status) == corm.CORM_DEV_BAD_PAGE and c.lens.tolist() == [[100], [100]]
            gone = lambda b, h: range(16, 32) if b == 0 else range(96, 112)  # noqa: E731
            c.status.zero_()
            q = _normal(g, "bf16", 2, 4, 128, scale=2.0)
            c.attend(q)
            c.check_out(q, gone)
            assert int(c.status) == corm.CORM_DEV_BAD_PAGE
            c.status.zero_()
            K, V = _nan(2, 2, 100, 128, dtype="bf16"), _nan(2, 2, 100, 128, dtype="bf16")
            corm.corm_paged_read(c.desc, c.pages, c.lens, K, V, status=c.status)
            assert int(c.status) == corm.CORM_DEV_BAD_PAGE
            for b in range(2):
                miss = [s in gone(b, 0) for s in range(100)]
                assert K[b, 0].isnan().all(-1).tolist() == miss and V[b, 1].isnan().any(-1).tolist() == miss
            # without any page: nothing to attend to
            c.dev_table.fill_(bad)
            c.attend(q)
            assert not c.out.any()


@pytest.mark.parametrize("dtype,code", FORMS)
@pytest.mark.parametrize("d,page,per_head", [(128, 16, True), (64, 256, False)])
def test_read(dtype, code, d, page, per_head):
    g = _gen(15)
    lens = [[0, 1], [17, 300], [299, 64]] if per_head else [[0], [301], [63]]
    c = Cache(g, 3, 8, 2, d, 301, dtype, code, page, per_head)
    c.fill(g, lens, (1.0, 5.0))
    for n in (301, 350, 64, 1):
        K, V = _nan(3, 2, n, d, dtype=dtype), _nan(3, 2, n, d, dtype=dtype)
        corm.corm_paged_read(c.desc, c.pages, c.lens, K, V, status=c.status)
        for b in range(3):
            for h in range(2):
                m = min(c.length(b, h), n)
                for j, x in enumerate((K, V)):
                    assert bool(x[b, h, m:].isnan().all())
                    if m:
                        want = torch.stack(c.rows[b][h][j][:m])
                        if code:
                            q, s = ref.quantise_rows(want, code)
                            want = (q * s.unsqueeze(-1)).to(DT[dtype])
                        assert torch.equal(x[b, h, :m].cpu(), want), (n, b, h, j)
    assert int(c.status) == 0
    bad = c.lens.clone()
    bad[0], bad[1] = -4, 302            # read as 0 and as all slots
    K, V = _nan(3, 2, 301, d, dtype=dtype), _nan(3, 2, 301, d, dtype=dtype)
    corm.corm_paged_read(c.desc, c.pages, bad, K, V, status=c.status)
    assert int(c.status) == corm.CORM_DEV_BAD_LENS and bool(K[0].isnan().all())


@pytest.mark.parametrize("dtype,code", FORMS)
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_attend_awkward_lengths(dtype, code, d, G):
    """Units of no slot, of one, around tiles' and pages' ends; whatever lies behind a unit's length (not a number, or another's rows) is not seen."""
    g = _gen(16)
    for page, per_head in ((16, True), (64, False), (256, True)):
        c = Cache(g, 5, 2 * G, 2, d, 417, dtype, code, page, per_head)
        odd = [0, 1, 15, 16, 17, 63, 64, 65, 255, 417]
        lens = [[odd[(2 * b + h) % 10] for h in range(2)] if per_head else [odd[2 * b + (page == 64)]] for b in range(5)]
        for j, pool in enumerate((c.K, c.V)):
            if code is None:
                pool.copy_(torch.full_like(pool, float("inf" if j else "nan")))
        top = max(max(r) for r in lens)
        k, v = _normal(g, dtype, 5, 2, top, d, scale=2.0), _normal(g, dtype, 5, 2, top, d, scale=3.0)
        # (rows behind a unit's length stay junk: one call per table)
        for b in range(5):
            for h in range(c.TH):
                n = lens[b][h]
                for kh in ([h] if per_head else [0, 1]):
                    c.rows[b][kh] = [list(k[b, kh, :n]), list(v[b, kh, :n])]
                    if n:
                        at = tuple(x.to(DEV) for x in c.where(b, kh, n))
                        for x, pool, sc in ((k, c.K, c.ks), (v, c.V, c.vs)):
                            rows = x[b, kh, :n]
                            if code:
                                q, s = ref.quantise_rows(rows, code)
                                pool.view(torch.int8)[at] = (q.to(torch.int8) if code == "i8" else q.to(torch.float8_e4m3fn).view(torch.int8)).to(DEV)
                                sc[at] = s.to(DEV)
                            else:
                                pool[at] = rows.to(DEV)
        c.lens.copy_(_i32(lens))
        for b in range(5):                                           # entries behind the last page: anything
            for h in range(c.TH):
                c.dev_table[b, h, (lens[b][h] + page - 1) // page:] = -1 if b % 2 else 2147483647
        q = _normal(g, dtype, 5, 2 * G, d, scale=2.0)
        c.attend(q)
        c.check_out(q)
        assert int(c.status) == 0


@pytest.mark.parametrize("dtype,code", FORMS)
def test_attend_many_units_and_long_ones(dtype, code):
    """Units in one part, in few, in many; queries that look at one key, and scores that lie far apart."""
    g = _gen(17)
    for B, Hq, Hkv, d, P, page, per_head in ((70, 16, 8, 64, 130, 16, True), (1, 8, 1, 128, 9000, 64, False), (2, 8, 4, 128, 3001, 32, True),
                                             (40, 8, 2, 64, 600, 128, False)):
        c = Cache(g, B, Hq, Hkv, d, P, dtype, code, page, per_head)
        n = Hkv if per_head else 1
        c.fill(g, [[P - (37 * (b * n + h)) % max(P // 2, 1) for h in range(n)] for b in range(B)], (3.0, 2.0))
        q = _normal(g, dtype, B, Hq, d, scale=4.0)
        c.attend(q)
        c.check_out(q)
        again = c.out.clone()
        c.attend(q)
        assert torch.equal(c.out, again) and int(c.status) == 0


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("dtype,code", [("bf16", None), ("f32", None), ("bf16", "e4m3")])
def test_attend_units_of_every_length(dtype, code, per_head):
    """Hundreds of units, and few long ones, of any lengths: none, one slot, fewer tiles than waves and workgroups, more."""
    g = _gen(21)
    for B, Hkv, most in ((130, 2, 200), (3, 2, 20000), (1, 1, 40), (400, 2, 33)):
        c = Cache(g, B, 2 * Hkv, Hkv, 64, most, dtype, code, 16, per_head, spare=1)
        n = Hkv if per_head else 1
        lens = torch.randint(0, most + 1, (B, n), generator=g)
        lens = torch.where(torch.rand(B, n, generator=g) < 0.25, torch.randint(0, 2, (B, n), generator=g) * most, lens)
        c.fill(g, lens.tolist(), (2.0, 2.0))
        q = _normal(g, dtype, B, 2 * Hkv, 64, scale=3.0)
        c.attend(q)
        c.check_out(q)


@pytest.mark.parametrize("B,Hkv,most,per_head", [(60, 2, 1100, True), (100, 1, 900, False), (170, 3, 2100, True), (255, 2, 2070, False), (2, 1, 70000, False),
                                                 (512, 1, 2100, False)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_attend_shares_of_all_units(dtype, d, B, Hkv, most, per_head):
    """Units whose tiles are shared out: of every length, runs that begin and end inside them, empty ones between, long ones over many runs."""
    g = _gen(23)
    TH, G, page = (Hkv if per_head else 1), 2, 64
    maxp = (most + page - 1) // page
    lens = torch.randint(0, most + 1, (B, TH), generator=g, dtype=torch.int32)
    lens[torch.rand(B, TH, generator=g) < 0.2] = 0
    lens[torch.rand(B, TH, generator=g) < 0.1] = most
    lens[-1] = most if B < 100 else 0                       # (the last run ends with the last unit, or with empty ones)
    npages = B * TH * maxp // 2 + 1                         # pages are shared by tables: they are only read
    table = torch.randint(0, npages, (B, TH, maxp), generator=g, dtype=torch.int32)
    shape = (npages,) + (() if per_head else (Hkv,)) + (page, d)
    gd = torch.Generator(device=DEV).manual_seed(23)
    K, V = ((torch.randn(shape, generator=gd, device=DEV) * 2).to(DT[dtype]) for _ in range(2))
    q = _normal(g, dtype, B, Hkv * G, d, scale=2.0).to(DEV)
    desc = corm.make_desc(B, Hkv * G, Hkv, d, most, most, 1, 1, dtype)
    out, ws = _nan(B, Hkv * G, d), torch.full((corm.corm_paged_workspace_bytes(desc),), 0xA5, dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    td, ld = table.to(DEV), lens.to(DEV)
    corm.corm_paged_attend(desc, corm.Pages(desc, K, V, td), q, ld, out, ws, status=status)
    assert int(status) == 0 and not bool(out.isnan().any())
    for b in range(B):
        for h in range(Hkv):
            n = int(lens[b, h if per_head else 0])
            x, got = q[b, h * G:(h + 1) * G].double(), out[b, h * G:(h + 1) * G].double()
            if not n:
                assert not got.any()
                continue
            ids = td[b, h if per_head else 0, :(n + page - 1) // page].long()
            k, v = ((p if per_head else p[:, h])[ids].reshape(-1, d)[:n].double() for p in (K, V))
            s = torch.mm(x, k.t()) * ref.sm_of(d)
            want = torch.mm(torch.softmax(s, -1), v)
            bound = ref.attend_error(x, k, v, ref.sm_of(d))
            assert float((got - want).abs().max()) <= bound, (b, h, n)


@pytest.mark.parametrize("B,Hkv,most", [(3, 2, 20000), (90, 6, 300), (2, 2, 300)])
def test_attend_bad_lengths_and_pages_in_every_launch(B, Hkv, most):
    """Shared tiles, whole units, a workgroup a round: lengths that are none are held to the bounds, pages that are none are not seen, both are reported."""
    g = _gen(26)
    d, G, page = 64, 2, 32
    maxp = (most + page - 1) // page
    lens = torch.randint(0, most + 1, (B, 1), generator=g, dtype=torch.int32)
    lens[0], lens[1] = -5, most + 9
    held = lens.clamp(0, most)
    npages = 50
    table = torch.randint(0, npages, (B, 1, maxp), generator=g, dtype=torch.int32)
    K, V = ((torch.randn(npages, Hkv, page, d, generator=g) * 2).to(torch.bfloat16).to(DEV) for _ in range(2))
    q = _normal(g, "bf16", B, Hkv * G, d, scale=2.0).to(DEV)
    desc = corm.make_desc(B, Hkv * G, Hkv, d, most, most, 1, 1, "bf16")
    ws, status = torch.empty(corm.corm_paged_workspace_bytes(desc), dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    outs = []
    for x in (held, lens):
        status.zero_()
        outs.append(_nan(B, Hkv * G, d))
        corm.corm_paged_attend(desc, corm.Pages(desc, K, V, table.to(DEV)), q, x.to(DEV), outs[-1], ws, status=status)
        assert int(status) == (0 if x is held else corm.CORM_DEV_BAD_LENS)
    assert torch.equal(*outs)
    gone = torch.rand(B, 1, maxp, generator=g) < 0.3
    gone[1, 0, 0] = True
    td = torch.where(gone, torch.where(torch.rand(B, 1, maxp, generator=g) < 0.5, -1, npages), table).to(torch.int32).to(DEV)
    out = _nan(B, Hkv * G, d)
    status.zero_()
    corm.corm_paged_attend(desc, corm.Pages(desc, K, V, td), q, held.to(DEV), out, ws, status=status)
    assert int(status) == corm.CORM_DEV_BAD_PAGE
    for b in range(0, B, 1 if B < 10 else 7):
        n = int(held[b])
        seen = ~gone[b, 0, torch.arange(n) // page].to(DEV)
        for h in range(Hkv):
            k, v = (p[table[b, 0].long().to(DEV), h].reshape(-1, d)[:n][seen].double() for p in (K, V))
            x, got = q[b, h * G:(h + 1) * G].double(), out[b, h * G:(h + 1) * G].double()
            if not k.shape[0]:
                assert not got.any()
                continue
            want = torch.mm(torch.softmax(torch.mm(x, k.t()) * ref.sm_of(d), -1), v)
            assert float((got - want).abs().max()) <= ref.attend_error(x, k, v, ref.sm_of(d)), (b, h, n)


def test_attend_thousands_of_units():
    g = _gen(22)
    B, d = 4100, 64
    lens = torch.randint(0, 65, (B, 1), generator=g, dtype=torch.int32)
    K, V = _normal(g, "bf16", B, 1, 64, d).to(DEV), _normal(g, "bf16", B, 1, 64, d).to(DEV)
    q = _normal(g, "bf16", B, 2, d, scale=2.0)
    desc = corm.make_desc(B, 2, 1, d, 64, 64, 1, 1, "bf16")
    table = torch.randperm(B * 4, generator=g).to(torch.int32).view(B, 1, 4)
    at = table.view(B, 4).long().to(DEV)
    pool = [torch.zeros(B * 4, 1, 16, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for p, x in zip(pool, (K, V)):
        p[at.view(-1), 0] = x.view(B * 4, 16, d)
    out, ws = _nan(B, 2, d), torch.empty(corm.corm_paged_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    corm.corm_paged_attend(desc, corm.Pages(desc, *pool, table.to(DEV)), q.to(DEV), lens.to(DEV), out, ws)
    got = out.cpu().double()
    for b in range(0, B, 17):
        k, v, x = K[b, 0, :lens[b]].cpu().double(), V[b, 0, :lens[b]].cpu().double(), q[b].double()
        assert float((got[b] - ref.attend(x, k, v, ref.sm_of(d))).abs().max()) <= ref.attend_error(x, k, v, ref.sm_of(d)), b
    live = (torch.arange(64, device=DEV) < lens.to(DEV)).unsqueeze(1)
    s = torch.matmul(q.to(DEV).float(), K[:, 0].float().transpose(1, 2).contiguous()) * ref.sm_of(d)
    p = torch.softmax(s.masked_fill(~live, float("-inf")), -1).nan_to_num()
    assert float((torch.matmul(p, V[:, 0].float()) - out).abs().max()) < 1e-4


def test_attend_lengths_that_are_none_and_scale():
    g = _gen(18)
    c = Cache(g, 3, 4, 2, 128, 200, "bf16", None, 16, False)
    c.fill(g, [[200], [200], [50]])
    q = _normal(g, "bf16", 3, 4, 128)
    c.lens.copy_(_i32([[-7], [201], [50]]))       # as 0 and as all slots
    c.attend(q)
    assert int(c.status) == corm.CORM_DEV_BAD_LENS and not c.out[0].any()
    c.rows[0][0], c.rows[0][1] = [[], []], [[], []]
    c.check_out(q)
    c.desc.sm_scale = 0.5
    c.lens.copy_(_i32([[200], [200], [50]]))
    c.attend(q)
    for b, h in ((1, 0), (2, 1)):
        K, V, x = c.unit(b, h, 0), c.unit(b, h, 1), q[b, 2 * h:2 * h + 2].double()
        assert float((c.out[b, 2 * h:2 * h + 2].cpu().double() - ref.attend(x, K, V, 0.5)).abs().max()) <= ref.attend_error(x, K, V, 0.5)


def test_attend_codes_with_scales_far_apart():
    """Rows whose scales differ by twenty powers of ten: the smallest still counts where its probability does."""
    g = _gen(19)
    for code in ("i8", "e4m3"):
        c = Cache(g, 1, 8, 1, 128, 256, "bf16", code, 16, False)
        k, v = _normal(g, "bf16", 1, 1, 256, 128), _normal(g, "bf16", 1, 1, 256, 128)
        v = v * (10.0 ** (-20 * torch.rand(256, generator=g))).view(1, 1, 256, 1)
        v = v.to(torch.bfloat16)
        c.append(k, v)
        q = _normal(g, "bf16", 1, 8, 128, scale=3.0)
        c.attend(q)
        c.check_out(q)


def test_pool_beyond_32_bits():
    """Pages whose rows lie more than 4 GiB (and 2^32 elements) into the pool."""
    g = _gen(20)
    d, page, B = 128, 256, 2
    npages = (1 << 32) // (page * d) + 40          # 2^32 elements and some: 8.6 GB a pool in bf16
    for code in (None, "i8"):
        shape = (npages, page, d)
        K = torch.empty(shape, dtype=torch.int8 if code else torch.bfloat16, device=DEV)
        V = torch.empty(shape, dtype=torch.int8 if code else torch.bfloat16, device=DEV)
        sc = [torch.empty(shape[:-1], device=DEV) for _ in range(2)] if code else [None, None]
        desc = corm.make_desc(B, 4, 1, d, 600, 600, 1, 1, "bf16")
        table = torch.tensor([[[npages - 1, 3, npages - 7]], [[npages - 3, npages - 20, 5]]], dtype=torch.int32)
        pages = corm.Pages(desc, K, V, table.to(DEV), *sc)
        lens, status = torch.zeros(B, 1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        k, v = _normal(g, "bf16", B, 1, 600, d), _normal(g, "bf16", B, 1, 600, d)
        corm.corm_paged_append(desc, pages, k.to(DEV), v.to(DEV), lens, lens, status=status)
        out, ws = _nan(B, 4, d), torch.empty(corm.corm_paged_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
        q = _normal(g, "bf16", B, 4, d, scale=2.0)
        corm.corm_paged_attend(desc, pages, q.to(DEV), lens, out, ws, status=status)
        back = [_nan(B, 1, 600, d, dtype="bf16") for _ in range(2)]
        corm.corm_paged_read(desc, pages, lens, *back, status=status)
        assert int(status) == 0
        for b in range(B):
            rows = []
            for x, y in zip((k, v), back):
                r = x[b, 0]
                if code:
                    cc, s = ref.quantise_rows(r, code)
                    assert torch.equal(y[b, 0].cpu(), (cc * s.unsqueeze(-1)).to(torch.bfloat16))
                    rows.append(cc.double() * s.double().unsqueeze(-1))
                else:
                    assert torch.equal(y[b, 0].cpu(), r)
                    rows.append(r.double())
            sm = ref.sm_of(d)
            err = float((out[b].cpu().double() - ref.attend(q[b].double(), *rows, sm)).abs().max())
            assert err <= ref.attend_error(q[b].double(), *rows, sm)
        del K, V, sc, pages
        torch.cuda.empty_cache()


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("dtype,code,per_head", [("bf16", None, False), ("f32", None, True), ("bf16", "i8", True), ("bf16", "e4m3", False), ("f32", "e4m3", True)])
@pytest.mark.parametrize("kind", [0, 1, 6])
def test_append_rotates(dtype, code, per_head, kind):
    """Rotated on the way into the pages: queries and, in the KV type, keys have the bits of corm_rotate's; codes stand for the fp32 values."""
    g = _gen(30 + kind)
    d = 128
    for B, Hq, Hkv, n, n_new in ((3, 8, 2, 1, None), (2, 8, 4, 45, [45, 31]), (2, 4, 2, 1, [1, 0])):
        t = Turn(g, dtype, d, **TURNS[kind])
        (q, k, v), (_, ck, cv) = _packed(g, dtype, B, Hq, Hkv, n, d)
        pos = torch.randint(0, 100000, (len(t.sections), B, n), generator=g, dtype=torch.int32)
        c = Cache(g, B, Hq, Hkv, d, 64, dtype, code, 16, per_head)
        q_out, dense = _nan(B, Hq, n, d, dtype=dtype), [_nan(B, h, n, d, dtype=dtype) for h in (Hq, Hkv, Hkv)]
        dn = None if n_new is None else _i32(n_new)
        corm.corm_paged_append(c.desc, c.pages, k, v, c.lens, c.lens, n_new=dn, q=q, q_out=q_out, rotation=t.c, positions=pos.to(DEV), status=c.status)
        corm.corm_rotate(c.desc, q, k, v, t.c, pos.to(DEV), *dense, n_new=dn)
        assert _same(q_out, dense[0])
        want, bound = t.plain(ck, 1, pos)
        for b in range(B):
            take = n if n_new is None else n_new[b]
            assert c.lens[b].tolist() == [take] * c.TH
            for h in range(Hkv):
                at = tuple(x.to(DEV) for x in c.where(b, h, take))
                if not take:
                    continue
                if code is None:
                    assert torch.equal(c.K[at], dense[1][b, h, :take]) and torch.equal(c.V[at].cpu(), cv[b, h, :take])
                    continue
                codes = c.K.view(torch.int8)[at].cpu().view(CODE[code]).double()
                scale = c.ks[at].cpu().double().unsqueeze(-1)
                w, e = want[b, h, :take], bound[b, h, :take]
                # the scale: that of the largest value, off by its error and a rounding; a code: half a step, and the roundings of factor and product
                amax, slack = w.abs().amax(-1, keepdim=True), e.amax(-1, keepdim=True)
                assert bool(((scale * ref.QMAX[code] - amax).abs() <= slack + 2 * ref.EPS * amax).all())
                half = 0.5 * scale if code == "i8" else torch.maximum(2.0 ** -4 * w.abs(), 2.0 ** -10 * scale)
                assert bool(((codes * scale - w).abs() <= 1.001 * half + 2 * (e + slack) + 6 * ref.EPS * amax).all())
        assert int(c.status) == 0


@pytest.mark.parametrize("dtype,code,per_head", [("bf16", None, False), ("f32", None, True), ("bf16", "i8", True), ("f32", "e4m3", False)])
def test_a_conversation(dtype, code, per_head):
    """A padded batch of prompts goes into the pages, then steps: every step's output is attention over what the pages hold."""
    g = _gen(40)
    B, Hq, Hkv, d, n, steps = 3, 8, 2, 128, 70, 5
    st = corm.PagedState(B, Hq, Hkv, d, 3 * (2 if per_head else 1) * 6, 6, dtype, 16, code, per_head, device=DEV)
    st.deal()
    t = Turn(g, dtype, d, rot=64, sections=[16, 8, 8])
    lens = [70, 1, 33]
    (q, k, v), _ = _packed(g, dtype, B, Hq, Hkv, n, d)
    pos = torch.arange(n, dtype=torch.int32).expand(3, B, n).contiguous()
    q_rows = _nan(B, Hq, n, d, dtype=dtype)
    st.append(k, v, n_new=_i32(lens), q=q, q_out=q_rows, rotation=t.c, positions=pos.to(DEV))
    assert st.lens.tolist() == [[x] * st.lens.shape[1] for x in lens]
    for i in range(steps):
        (q, k, v), (cq, _, _) = _packed(g, dtype, B, Hq, Hkv, 1, d)
        at = torch.tensor([x + i for x in lens], dtype=torch.int32).view(1, B, 1).expand(3, B, 1).contiguous()
        st.step(q, k, v, rotation=t.c, positions=at.to(DEV))
        K, V = (_nan(B, Hkv, 80, d, dtype="f32") for _ in range(2))
        for b in range(B):       # what the pages hold, in full precision
            for h in range(Hkv):
                m = lens[b] + i + 1
                ids = st.table[b, h if per_head else 0].long().repeat_interleave(16)[:m]
                slots = torch.arange(m, device=DEV) % 16
                idx = (ids, slots) if per_head else (ids, torch.full_like(ids, h), slots)
                rows = []
                for pool, sc in ((st.K, st.k_scale), (st.V, st.v_scale)):
                    x = pool.view(torch.int8)[idx].view(pool.dtype).cpu().double() * sc[idx].cpu().double().unsqueeze(-1) if code else pool[idx].cpu().double()
                    rows.append(x)
                x = st.q[b, 4 * h:4 * h + 4].cpu().double()
                err = float((st.out[b, 4 * h:4 * h + 4].cpu().double() - ref.attend(x, *rows, ref.sm_of(d))).abs().max())
                assert err <= ref.attend_error(x, *rows, ref.sm_of(d)), (i, b, h)
        w, e = t.plain(cq, 0, at)
        _close(st.q.unsqueeze(2), w, e, dtype, i)
    assert int(st.status) == 0


def test_pages_beside_a_layer_state():
    """Rows that go through corm_rotate into a LayerState and through pages: the same attention while nothing is evicted, and the pages' rows read back
    preload another state."""
    g = _gen(41)
    B, Hq, Hkv, d, n = 2, 8, 2, 128, 100
    t = Turn(g, "bf16", d)
    st = corm.LayerState(B, Hq, Hkv, d, 128, 128, 64, 64, "bf16", device=DEV)
    pg = corm.PagedState(B, Hq, Hkv, d, 2 * 8, 8, "bf16", device=DEV)
    pg.deal()
    (q, k, v), _ = _packed(g, "bf16", B, Hq, Hkv, n, d)
    pos = torch.arange(n, dtype=torch.int32, device=DEV).expand(1, B, n).contiguous()
    o = [_nan(B, h, n, d, dtype="bf16") for h in (Hq, Hkv, Hkv)]
    corm.corm_rotate(st.desc, q, k, v, t.c, pos, *o)
    st.preload(o[1], o[2])
    pg.append(k, v, rotation=t.c, positions=pos)
    K, V = _nan(B, Hkv, n, d, dtype="bf16"), _nan(B, Hkv, n, d, dtype="bf16")
    pg.read(K, V)
    assert torch.equal(K, o[1]) and torch.equal(V, o[2])
    t_first = _i32([n + 1] * B)
    for i in range(4):
        (q, k, v), _ = _packed(g, "bf16", B, Hq, Hkv, 1, d)
        at = torch.full((1, B, 1), n + i, dtype=torch.int32, device=DEV)
        s = [_nan(B, h, d, dtype="bf16") for h in (Hq, Hkv, Hkv)]
        corm.corm_rotate(st.desc, q, k, v, t.c, at, *s)
        st.step(*s, _i32([n + i + 1] * B), t_first)
        pg.step(q, k, v, rotation=t.c, positions=at)
        assert torch.equal(pg.q, s[0])
        for b in range(B):
            for h in range(Hkv):
                K, V = st.K[b, h, :n + i + 1].cpu().double(), st.V[b, h, :n + i + 1].cpu().double()
                err = 2 * ref.attend_error(s[0][b, 4 * h:4 * h + 4].cpu().double(), K, V, ref.sm_of(d))
                assert float((pg.out - st.out)[b, 4 * h:4 * h + 4].abs().max()) <= err
    assert int(pg.status) == 0 and int(st.status) == 0


def test_two_graphs_share_a_workspace():
    """Attention over two caches of other shapes, captured with one workspace and replayed in turns, with eager calls between."""
    g = _gen(43)
    caches = [Cache(g, 3, 8, 2, 128, 9000, "bf16", "i8", 64, False), Cache(g, 40, 4, 2, 64, 1100, "f32", None, 16, True), Cache(g, 2, 4, 4, 128, 50, "bf16")]
    ws = torch.empty(max(corm.corm_paged_workspace_bytes(c.desc) for c in caches), dtype=torch.uint8, device=DEV)
    qs, want = [], []
    for c in caches:
        n = c.Hkv if c.per_head else 1
        c.fill(g, [[(997 * (b * n + h) + 331) % (c.desc.Lcap + 1) for h in range(n)] for b in range(c.B)])
        c.ws = ws
        qs.append(_normal(g, c.dtype, c.B, c.Hq, c.d).to(DEV))
        c.attend(qs[-1])
        c.check_out(qs[-1].cpu())
        want.append(c.out.clone())
    graphs = []
    for c, q in zip(caches, qs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            corm.corm_paged_attend(c.desc, c.pages, q, c.lens, c.out, ws)
    for i in (0, 1, 2, 1, 0, 2, 2, 0, 1):
        caches[i].out.zero_()
        graphs[i].replay()
        assert torch.equal(caches[i].out, want[i])
        caches[(i + 1) % 3].attend(qs[(i + 1) % 3])
        torch.cuda.synchronize()
        assert torch.equal(caches[(i + 1) % 3].out, want[(i + 1) % 3])


@pytest.mark.parametrize("code", [None, "i8"])
def test_captured_steps_and_other_streams(code):
    """Steps captured once and replayed with other inputs and pages, eager work between the replays; the same on a stream of its own."""
    g = _gen(42)
    B, Hq, Hkv, d = 2, 8, 2, 128
    t = Turn(g, "bf16", d)
    x = [_packed(g, "bf16", B, Hq, Hkv, 1, d)[0] for _ in range(8)]
    pos = [torch.full((1, B, 1), 7 * i, dtype=torch.int32, device=DEV) for i in range(8)]

    def fresh():
        s = corm.PagedState(B, Hq, Hkv, d, 40, 4, "bf16", 16, code, device=DEV)
        s.table.copy_(torch.arange(8, dtype=torch.int32).mul(5).view(B, 1, 4))
        return s
    want, st = [], fresh()
    for i in range(8):
        st.step(*x[i], rotation=t.c, positions=pos[i])
        want.append(st.out.clone())
    end = [st.K.clone().view(torch.int8 if code else torch.bfloat16), st.lens.clone()]
    # captured
    st = fresh()
    buf, at = [torch.zeros_like(y) for y in x[0]], torch.zeros_like(pos[0])
    st.step(*buf, rotation=t.c, positions=at)           # (the first call asks the device for its size)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.step(*buf, rotation=t.c, positions=at)
    st.lens.zero_()
    st.K.view(torch.int8).zero_()
    st.V.view(torch.int8).zero_()
    for i in range(8):
        for y, z in zip(buf, x[i]):
            y.copy_(z)
        at.copy_(pos[i])
        graph.replay()
        assert torch.equal(st.out, want[i]), i
        torch.cuda.synchronize()
        torch.randn(1000, device=DEV).sum()
    assert torch.equal(st.K.view(end[0].dtype), end[0]) and torch.equal(st.lens, end[1])
    # a stream of its own
    st = fresh()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for i in range(8):
        st.step(*x[i], rotation=t.c, positions=pos[i], stream=side)
        side.synchronize()
        assert torch.equal(st.out, want[i]), i
