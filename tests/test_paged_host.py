"""Refusals of the cache of pages and of the rows on their way into it, on the host, before anything is launched; and the plain forms that the GPU tests
compare with."""
import ctypes
import math

import pytest
import torch

from paper_2404_15949_amd import corm
from tests import paged_ref as ref

A = 4096   # a plausible aligned address; never dereferenced because validation fails first


def _desc(**kw):
    base = dict(B=2, Hq=8, Hkv=2, d=128, Lcap=1024, Tcap=1024, w=16, r=16, kv_dtype="bf16")
    base.update(kw)
    return corm.make_desc(**base)


def _rows(**kw):
    r = corm.corm_rows(A, A, A, *([1536, 768, 128] * 3))
    for k, v in kw.items():
        if k.endswith("_stride"):
            for of, x in zip(("seq", "token", "head"), v):
                setattr(r, k.replace("stride", of), x)
        else:
            setattr(r, k, v)
    return r


def _rot(**kw):
    r = corm.corm_rotation(128, corm.CORM_HALVES, 1, 0, (ctypes.c_int32 * 4)(64, 0, 0, 0), 1e-6, 1.0, A, A, A)
    for k, v in kw.items():
        setattr(r, k, v if not isinstance(v, tuple) else (ctypes.c_int32 * 4)(*v))
    return r


def _pages(**kw):
    p = corm.corm_pages(corm.CORM_BF16, 16, 100, 64, 1, 0, A, A, None, None, A)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


CALLS = {   # arguments behind the descriptor, in order; those that may be NULL
    "corm_rotate": ("rows rotation positions n n_new q_out k_out v_out stream", ("n_new", "q_out", "stream")),
    "corm_paged_append": ("pages rows rotation positions n n_new q_out lens lens_out status stream",
                          ("n_new", "q_out", "status", "stream", "rotation")),
    "corm_paged_read": ("pages lens n K_out V_out status stream", ("status", "stream")),
    "corm_paged_attend": ("pages q lens out workspace workspace_bytes status stream", ("status", "stream")),
}
STRUCTS = {"rows": _rows, "rotation": _rot, "pages": _pages}
NUMBERS = {"n": 4, "workspace_bytes": 16, "stream": None}
BYTES16 = ("q_out", "k_out", "v_out", "K_out", "V_out", "q")


def _call(name, desc=None, **change):
    """A call that some check refuses: attention by its workspace of 16 bytes, the others by what the test changes."""
    args = []
    for k in CALLS[name][0].split():
        x = change[k] if k in change else STRUCTS[k]() if k in STRUCTS else NUMBERS.get(k, A)
        args.append(ctypes.byref(x) if isinstance(x, ctypes.Structure) else x)
    return getattr(corm.lib(), name)(ctypes.byref(_desc() if desc is None else desc), *args)


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned_pointers(name):
    names, optional = CALLS[name]
    for k in names.split():
        if k in NUMBERS:
            continue
        if k not in optional:
            assert _call(name, **{k: None}) == corm.CORM_EINVAL, k
        if k not in STRUCTS:
            assert _call(name, **{k: A + 2}) == corm.CORM_EINVAL, k
        if k in BYTES16:
            assert _call(name, **{k: A + 8}) == corm.CORM_EINVAL, k


@pytest.mark.parametrize("name", CALLS)
def test_descriptors(name):
    for bad, code in ((dict(d=96), corm.CORM_EUNSUPPORTED), (dict(Hq=6), corm.CORM_EUNSUPPORTED), (dict(B=0), corm.CORM_EINVAL),
                      (dict(B=40000), corm.CORM_EUNSUPPORTED), (dict(Lcap=1 << 22), corm.CORM_EUNSUPPORTED)):
        assert _call(name, _desc(**bad)) == code, bad


@pytest.mark.parametrize("name", [n for n in CALLS if "pages" in CALLS[n][0]])
def test_pages(name):
    E, U = corm.CORM_EINVAL, corm.CORM_EUNSUPPORTED
    for change, code in ((dict(dtype=corm.CORM_F32), U), (dict(dtype=corm.CORM_BIT), U), (dict(dtype=9), U), (dict(K=None), E), (dict(V=None), E),
                         (dict(table=None), E), (dict(K=A + 8), E), (dict(V=A + 8), E), (dict(table=A + 2), E), (dict(page=8), U), (dict(page=48), U),
                         (dict(page=0), U), (dict(page=512), U), (dict(page=-16), U), (dict(npages=0), E), (dict(max_pages=0), E), (dict(max_pages=63), E),
                         (dict(table_heads=0), E), (dict(table_heads=3), E), (dict(dtype=corm.CORM_I8), E),
                         (dict(dtype=corm.CORM_I8, k_scale=A), E), (dict(dtype=corm.CORM_E4M3, v_scale=A), E),
                         (dict(dtype=corm.CORM_I8, k_scale=A + 4, v_scale=A), E), (dict(dtype=corm.CORM_E4M3, k_scale=A, v_scale=A + 8), E)):
        assert _call(name, pages=_pages(**change)) == code, change


def test_numbers():
    E = corm.CORM_EINVAL
    for n in (0, -1, 1025):
        assert _call("corm_paged_append", n=n) == E
    for n in (0, -1):
        assert _call("corm_rotate", n=n) == E and _call("corm_paged_read", n=n) == E
    assert _call("corm_paged_attend") == corm.CORM_ECAPACITY                    # 16 bytes of workspace
    assert _call("corm_paged_attend", workspace=A + 128) == E
    for kw in (dict(pages=_pages(dtype=corm.CORM_I8, k_scale=A, v_scale=A)), dict(pages=_pages(table_heads=2, page=256, max_pages=4))):
        assert _call("corm_paged_attend", **kw) == corm.CORM_ECAPACITY          # fine but for that


@pytest.mark.parametrize("name", ["corm_rotate", "corm_paged_append"])
def test_rows(name):
    E = corm.CORM_EINVAL
    for change in (dict(k=None), dict(v=None), dict(q=None), dict(k=A + 8), dict(q=A + 2), dict(k_stride=(1536, 768, 4)), dict(v_stride=(4, 768, 128)),
                   dict(q_stride=(1536, -768, 128)), dict(k_stride=(-8, 768, 128))):
        assert _call(name, rows=_rows(**change)) == E, change
    # without queries theirs are not looked at: refused for the other reason alone
    assert _call(name, rows=_rows(q=None, q_stride=(1, 1, 1)), q_out=None, n=0) == E


@pytest.mark.parametrize("name", ["corm_rotate", "corm_paged_append"])
def test_rotations(name):
    bad = [dict(rot=-16), dict(rot=8), dict(rot=144), dict(rot=100), dict(pairing=2), dict(axes=0), dict(axes=5), dict(eps=-1.0),
           dict(eps=math.nan), dict(eps=math.inf), dict(gain=math.nan), dict(q_norm=A + 8), dict(k_norm=A + 4), dict(inv_freq=None), dict(inv_freq=A + 2),
           dict(section=(63, 0, 0, 0)), dict(section=(65, 0, 0, 0)), dict(section=(32, 32, 0, 0)), dict(axes=2, section=(65, -1, 0, 0)),
           dict(axes=3, section=(20, 22, 22, 0), in_turn=1), dict(axes=2, section=(31, 33, 0, 0), in_turn=1), dict(axes=4, section=(16, 16, 16, 15))]
    for change in bad:
        assert _call(name, rotation=_rot(**change)) == corm.CORM_EINVAL, change
    assert _call(name, positions=None) == corm.CORM_EINVAL and _call(name, positions=A + 2) == corm.CORM_EINVAL


def test_workspace():
    """Two partials of each of 1024 workgroups, and eight bytes a unit: no more for longer caches."""
    for kw in (dict(), dict(Lcap=1), dict(Lcap=131072), dict(Hq=1, Hkv=1, B=1, Lcap=4194303), dict(B=64, Hq=64, Hkv=64), dict(B=8191, Hq=64, Hkv=8)):
        d = _desc(**kw)
        partials = 1024 * 2 * (d.Hq // d.Hkv) * 130 * 4
        assert partials % 256 == 0 and corm.corm_paged_workspace_bytes(d) == (partials + d.B * d.Hkv * 8 + 255) // 256 * 256
    assert corm.corm_paged_workspace_bytes(_desc(d=96), check=False) == corm.CORM_EUNSUPPORTED
    assert corm.lib().corm_paged_workspace_bytes(ctypes.byref(_desc()), None) == corm.CORM_EINVAL


def test_structures_have_the_headers_layout():
    assert ctypes.sizeof(corm.corm_rows) == 96 and corm.corm_rows.q_seq.offset == 24 and corm.corm_rows.v_head.offset == 88
    assert ctypes.sizeof(corm.corm_rotation) == 64 and corm.corm_rotation.eps.offset == 32 and corm.corm_rotation.inv_freq.offset == 40
    assert ctypes.sizeof(corm.corm_pages) == 64 and corm.corm_pages.K.offset == 24 and corm.corm_pages.table.offset == 56


def test_wrappers_refuse_what_does_not_fit():
    d = _desc()
    K, table = torch.zeros(10, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(2, 1, 64, dtype=torch.int32)
    corm.Pages(d, K, K, table)
    for kw in (dict(V=K[:5]), dict(V=K.float()), dict(K=K[:, :1], V=K[:, :1]), dict(table=table[0]), dict(table=table.expand(2, 2, 64)), dict(K=K[0], V=K[0]),
               dict(K=K[..., :64], V=K[..., :64])):
        with pytest.raises(ValueError):
            corm.Pages(d, **{**dict(K=K, V=K, table=table), **kw})
    p = corm.Pages(d, K, K, table)
    with pytest.raises(ValueError):                                 # on the host
        corm.corm_paged_attend(d, p, A, A, A, A, workspace_bytes=1 << 30)
    with pytest.raises(ValueError):                                 # another descriptor's pages
        corm.corm_paged_attend(_desc(Hq=16, Hkv=4), p, A, A, A, A, workspace_bytes=1 << 30)
    rows = torch.zeros(2, 2, 3, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        corm.corm_paged_append(d, p, rows, rows, A, A)
    with pytest.raises(ValueError):
        corm.Rotation(torch.zeros(64), sections=[])
    with pytest.raises(ValueError):
        corm.Rotation(torch.zeros(64), sections=[16, 16, 16, 8, 8])
    with pytest.raises(KeyError):
        corm.Rotation(torch.zeros(64), pairing="thirds")


def test_states_refuse_before_a_row_goes_in():
    st = corm.PagedState(2, 8, 2, 128, 7, 4, "bf16", device="cpu")
    assert bool((st.table == -1).all()) and tuple(st.K.shape) == (7, 2, 16, 128) and tuple(st.lens.shape) == (2, 1)
    with pytest.raises(corm.CormError):
        st.deal()                                                   # eight pages
    rows = torch.zeros(2, 2, 3, 128, dtype=torch.bfloat16)
    for rotation in (None, corm.Rotation(torch.zeros(64))):
        with pytest.raises(ValueError):
            st.step(torch.zeros(2, 8, 128, dtype=torch.bfloat16), rows, rows, rotation=rotation)
    st = corm.PagedState(1, 4, 4, 64, 8, 2, "f32", page=32, code="e4m3", per_head=True, device="cpu")
    st.deal()
    assert st.table.flatten().tolist() == list(range(8)) and tuple(st.k_scale.shape) == (8, 32) and st.K.dtype == torch.float8_e4m3fn
    with pytest.raises(corm.CormError):
        corm.PagedState(1, 4, 4, 64, 8, 2, "f32", device="cpu", workspace=torch.zeros(16))


def test_the_plain_rotation_keeps_lengths_and_turns_by_differences():
    """Norms stay; the product of a query and a key depends on the difference of their positions alone."""
    g = torch.Generator().manual_seed(3)
    freq = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float()
    x, y = torch.randn(1, 1, 1, 64, generator=g), torch.randn(1, 1, 1, 64, generator=g)
    for pairing in ("halves", "neighbours"):
        def at(v, p):
            return ref.turn(v, None, 0.0, freq, torch.tensor([[[p]]]), [32], False, pairing, 1.0)[0]
        assert abs(float(at(x, 12345).norm() - x.double().norm())) < 1e-12
        assert abs(float((at(x, 5) * at(y, 9)).sum() - (at(x, 1005) * at(y, 1009)).sum())) < 1e-9
    assert ref.axis_of(8, [4, 2, 2], False) == [0, 0, 0, 0, 1, 1, 2, 2] and ref.axis_of(8, [4, 2, 2], True) == [0, 1, 2, 0, 1, 2, 0, 0]
