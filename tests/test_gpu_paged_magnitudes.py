"""Attention over pages where magnitudes matter: values near the largest that the type has, infinite ones, rows whose scales lie far apart, and outputs
held to what each channel's sum is made of."""
import pytest
import torch

from paper_2404_15949_amd import corm
from tests import paged_inputs as inp
from tests import paged_ref as ref
from tests.test_gpu_paged import DEV, FORMS, Cache, _gen

pytestmark = pytest.mark.gpu

# B, Hkv, the bound of a length, lengths: whole units by one workgroup, a workgroup a round and a merge, shares of all units' tiles
LAUNCHES = {"whole": (2, 1, 190, [190, 150]), "parts": (2, 1, 2000, [190, 1999]), "shares": (8, 2, 9000, [190, 8999, 1, 33, 700, 0, 128, 2500])}


def _cache(g, launch, dtype, code, d, G=4, page=64):
    B, Hkv, most, lens = LAUNCHES[launch]
    return Cache(g, B, G * Hkv, Hkv, d, most, dtype, code, page, False), lens


def _hold(c, k, v, lens):
    """Units of `lens` rows of k and v [B,Hkv,n,d]"""
    corm.corm_paged_append(c.desc, c.pages, k.to(DEV), v.to(DEV), c.lens, c.lens, n_new=torch.tensor(lens, dtype=torch.int32, device=DEV), status=c.status)
    for b in range(c.B):
        for h in range(c.Hkv):
            c.rows[b][h] = [list(k[b, h, :lens[b]]), list(v[b, h, :lens[b]])]


def _check(c, q):
    """... against 64 bits, channel by channel; infinities and what is not a number where the definition has them"""
    G, sm, got = c.Hq // c.Hkv, ref.sm_of(c.d), c.out.cpu().double()
    assert int(c.status) == 0
    for b in range(c.B):
        for h in range(c.Hkv):
            K, V = c.unit(b, h, 0), c.unit(b, h, 1)
            x, o = q[b, h * G:(h + 1) * G].double(), got[b, h * G:(h + 1) * G]
            if not K.shape[0]:
                assert not o.any()
                continue
            odd = ~V.isfinite()
            F = V.masked_fill(odd, 0.0)
            want, bound = ref.attend(x, K, F, sm), ref.weighted_error(x, K, F, sm)
            plus, minus, none = ((V == float("inf")).any(0), (V == -float("inf")).any(0), V.isnan().any(0))
            none = none | (plus & minus)
            plus, minus = plus & ~none, minus & ~none
            assert torch.equal(o.isnan(), none.expand_as(o)), (b, h)
            assert torch.equal(o == float("inf"), plus.expand_as(o)) and torch.equal(o == -float("inf"), minus.expand_as(o)), (b, h)
            fine = ~odd.any(0)
            err = ((o - want).abs() - bound)[:, fine].max()
            assert float(err) <= 0, (b, h, K.shape[0], float(((o - want).abs() / bound)[:, fine].max()))


@pytest.mark.parametrize("launch", LAUNCHES)
@pytest.mark.parametrize("dtype,code", FORMS)
@pytest.mark.parametrize("d", [128, 64])
def test_every_channel_by_what_its_sum_is_made_of(launch, dtype, code, d):
    g = _gen(60)
    c, lens = _cache(g, launch, dtype, code, d)
    q, k, v = inp.one_channel(g, dtype, c.B, c.Hq, c.Hkv, max(lens), d)
    _hold(c, k, v, lens)
    c.attend(q)
    _check(c, q)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,most", [(128, 256), (64, 256), (128, 9000), (64, 60000)])
def test_rows_with_tiny_scales_count_whole(dtype, code, d, most):
    """A head whose weight lies on one row has that row, to the last bits, whatever the scales of the others: in one workgroup, in parts, in shares."""
    for G in (1, 8):
        g = _gen(61)
        q, k, v, target = inp.one_row(g, dtype, G, 256, d)
        c = Cache(g, 1, G, 1, d, most, dtype, code, 64, False)
        c.append(k, v)
        c.attend(q)
        want = c.unit(0, 0, 1)[target]
        assert int(c.status) == 0 and float(want.abs().amax(-1).min()) < 1e-22
        got = c.out[0].cpu().double()
        assert bool(((got - want).abs() <= inp.ONE_ROW * want.abs()).all()), (G, float(((got - want).abs() / want.abs().clamp(min=1e-99)).max()))


@pytest.mark.parametrize("dtype,code", FORMS)
@pytest.mark.parametrize("d", [128, 64])
def test_values_near_the_largest(dtype, code, d):
    """The sum of all magnitudes is within fp32, so is every output: also where the maximum of the scores rises from tile to tile by less than would
    matter for smaller values, in steps of 7.8 (log2), and where one value alone is nearly the largest."""
    g = _gen(62)
    c, lens = _cache(g, "whole", dtype, code, d)
    q, k, _ = inp.one_channel(g, dtype, c.B, c.Hq, c.Hkv, max(lens), d)
    q[..., 0], k[..., 0] = 1.0, 0.0
    at = 64 if dtype == "f32" and code is None else 128            # slots that the waves take at a time
    k[:, :, at:, 0] = 7.8 * 0.6931 * d ** 0.5
    v = (1 + torch.rand(c.B, c.Hkv, max(lens), d, generator=g)) * 2.0 ** 118 * (1 - 2 * torch.randint(0, 2, (c.B, c.Hkv, max(lens), d), generator=g))
    v[0, 0, at + 1] = 0
    v[0, 0, at + 1, ::3] = 2.0 ** 126
    _hold(c, k, v.to(k.dtype), lens)
    c.attend(q)
    _check(c, q)


@pytest.mark.parametrize("launch", LAUNCHES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64])
def test_infinite_values_stay_in_their_channel(launch, dtype, d):
    """A value that is infinite makes its channel's output so, the largest weight's and small ones'; one of each sign, or one that is no number, none; others are not touched."""
    g = _gen(63)
    c, lens = _cache(g, launch, dtype, None, d)
    q, k, v = inp.one_channel(g, dtype, c.B, c.Hq, c.Hkv, max(lens), d)
    k[:, :, 5, 0] = k[:, :, :, 0].max() + 1                        # the largest weight, of 1 where one wave has all slots
    k[:, :, 6, 0] = -30.0
    inf = float("inf")
    v[:, :, 5, 1], v[:, :, 6, 2], v[:, :, 7, 3], v[:, :, 20, d - 1] = inf, -inf, inf, -inf
    v[:, :, 8, 9], v[:, :, 9, 9] = inf, -inf
    v[:, :, 10, 11] = float("nan")
    for b, n in enumerate(lens):
        if n > 100:
            v[b, :, n - 1, 20], v[b, :, n // 2, 21] = inf, -inf
    _hold(c, k, v, lens)
    c.attend(q)
    _check(c, q)
