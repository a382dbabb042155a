"""What Rotation, Pages and PagedState keep of the tensors that they are given: nothing that another call's tensors could be taken for.  On CPU memory
(device -1), which is looked at as device memory is; nothing is launched."""
import pytest
import torch

from paper_2404_15949_amd import corm


def _desc(**kw):
    base = dict(B=2, Hq=8, Hkv=2, d=128, Lcap=1024, Tcap=1024, w=16, r=16, kv_dtype="bf16")
    base.update(kw)
    return corm.make_desc(**base)


def _rotation(**kw):
    base = dict(inv_freq=torch.ones(64), q_norm=torch.ones(128, dtype=torch.bfloat16), k_norm=torch.ones(128, dtype=torch.bfloat16))
    base.update(kw)
    return corm.Rotation(**base)


def _bound(x, desc=None):
    """Addresses as the call gets them"""
    x._bind(_desc() if desc is None else desc, -1)
    return {k: getattr(x.c, k) for k in (("inv_freq", "q_norm", "k_norm") if isinstance(x, corm.Rotation) else ("K", "V", "table", "k_scale", "v_scale"))}


@pytest.mark.parametrize("name", ["q_norm", "k_norm"])
def test_weights_that_became_another_type_in_the_same_memory(name):
    r = _rotation()
    _bound(r)
    w = getattr(r, name)
    w.data = w.data.view(torch.float16)
    with pytest.raises(ValueError):
        _bound(r)
    with pytest.raises(ValueError):                                  # nor by the second call
        _bound(r)
    w.data = w.data.view(torch.bfloat16)
    assert _bound(r)[name] == w.data_ptr()


@pytest.mark.parametrize("name", ["inv_freq", "q_norm", "k_norm"])
def test_other_weights_at_the_same_address(name):
    r = _rotation()
    _bound(r)
    w = getattr(r, name)
    wide = torch.ones(2 * w.numel(), dtype=w.dtype)
    setattr(r, name, wide[:w.numel()])
    assert _bound(r)[name] == wide.data_ptr()
    for bad in (wide[::2], wide[:w.numel() // 2], wide):
        assert bad.data_ptr() == wide.data_ptr()
        setattr(r, name, bad)
        with pytest.raises(ValueError):
            _bound(r)
    setattr(r, name, None)
    if name == "inv_freq":
        assert _bound(r)[name] is None                               # (the library refuses the call)
    else:
        assert _bound(r)[name] is None
        new = torch.ones(128, dtype=torch.bfloat16)
        setattr(r, name, new)
        assert _bound(r)[name] == new.data_ptr()


def test_weights_that_moved():
    """Other memory of the same parameter is looked at and taken; the old memory is nobody else's before that."""
    r = _rotation()
    w = torch.nn.Parameter(torch.ones(128, dtype=torch.bfloat16))
    r.q_norm = w
    at = _bound(r)["q_norm"]
    w.data = w.data.float()
    others = [torch.zeros(128, dtype=torch.bfloat16) for _ in range(200)]
    assert at not in [x.data_ptr() for x in others]
    with pytest.raises(ValueError):                                  # float32 now
        _bound(r)
    w.data = w.data.to(torch.bfloat16)
    assert _bound(r)["q_norm"] == w.data_ptr()


def _pages(code=None, pool=12, desc=None, per_head=False):
    d = _desc() if desc is None else desc
    shape = (pool,) + (() if per_head else (d.Hkv,)) + (16, d.d)
    K, V = (torch.zeros(shape, dtype=torch.int8 if code else torch.bfloat16) for _ in range(2))
    sc = [torch.zeros(shape[:-1]) for _ in range(2)] if code else [None, None]
    return corm.Pages(d, K, V, torch.zeros(d.B, d.Hkv if per_head else 1, 64, dtype=torch.int32), *sc)


def test_pools_of_another_type_or_layout_at_the_same_address():
    for name in ("K", "V"):
        p = _pages()
        _bound(p)
        x = getattr(p, name)
        x.data = x.data.view(torch.float16)
        with pytest.raises(ValueError):
            _bound(p)
        p = _pages()
        _bound(p)
        setattr(p, name, getattr(p, name).transpose(1, 2))
        with pytest.raises(ValueError):
            _bound(p)
    for name in ("k_scale", "v_scale"):
        p = _pages("i8")
        _bound(p)
        x = getattr(p, name)
        x.data = x.data.view(torch.int32)
        with pytest.raises(ValueError):
            _bound(p)
        setattr(p, name, torch.zeros(12, 2, 32)[..., ::2])
        with pytest.raises(ValueError):
            _bound(p)


def test_a_table_that_became_a_view_of_a_wider_one():
    big = torch.zeros(2, 1, 200, dtype=torch.int32)
    p = _pages()
    p.table = big[:, :, :64].contiguous()
    _bound(p)
    p.table = big[:, :, :64]
    with pytest.raises(ValueError):
        _bound(p)
    p = corm.Pages(_desc(), p.K, p.V, big)
    _bound(p)
    p.table = big[:, :, :64]                                         # the same address
    with pytest.raises(ValueError):
        _bound(p)


def _sizes(p):
    _bound(p)
    return p.c.npages, p.c.page, p.c.max_pages, p.c.table_heads, p.tables


def test_pools_and_tables_of_other_sizes():
    """The sizes that a call goes by are those of the tensors that it reads: page numbers beyond a smaller pool are none."""
    p = _pages()
    assert _sizes(p) == (12, 16, 64, 1, 2)
    p.K, p.V = (torch.zeros(5, 2, 16, 128, dtype=torch.bfloat16) for _ in range(2))
    assert _sizes(p) == (5, 16, 64, 1, 2)
    p.K, p.V = (torch.zeros(5, 2, 32, 128, dtype=torch.bfloat16) for _ in range(2))
    assert _sizes(p) == (5, 32, 64, 1, 2)
    p.table = torch.zeros(2, 1, 200, dtype=torch.int32)
    assert _sizes(p) == (5, 32, 200, 1, 2)
    p.K.data, p.V.data = (torch.zeros(3, 2, 16, 128, dtype=torch.bfloat16) for _ in range(2))      # the same tensors, moved
    assert _sizes(p) == (3, 16, 200, 1, 2)
    p.table = torch.zeros(2, 2, 64, dtype=torch.int32)                                              # a table for each head of a pool shared by them
    with pytest.raises(ValueError):
        _bound(p)
    p.K, p.V = (torch.zeros(7, 16, 128, dtype=torch.bfloat16) for _ in range(2))
    assert _sizes(p) == (7, 16, 64, 2, 4)
    p.K = torch.zeros(8, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        _bound(p)
    with pytest.raises(ValueError):                                                                 # nor by the second call
        _bound(p)
    p.K, p.V = (torch.zeros(7, 16, 128, dtype=torch.int8) for _ in range(2))                        # codes, once there are scales for them
    assert p._bind(_desc(), -1) and (p.c.dtype, p.c.k_scale) == (corm.CORM_I8, None)                # (the library refuses the call)
    p.k_scale, p.v_scale = (torch.zeros(7, 16) for _ in range(2))
    assert _bound(p)["v_scale"] == p.v_scale.data_ptr()
    p.k_scale = torch.zeros(6, 16)
    with pytest.raises(ValueError):
        _bound(p)


@pytest.mark.parametrize("code", [None, "i8"])
def test_a_state_whose_tensors_are_set_anew(code):
    """They are the ones that the calls take, whether they are set on the state or on its pages."""
    st = corm.PagedState(2, 8, 2, 128, 7, 4, "bf16", code=code, device="cpu")
    st.table = torch.arange(8, dtype=torch.int32).view(2, 1, 4)
    st.K, st.V = (torch.zeros(9, 2, 16, 128, dtype=st.K.dtype) for _ in range(2))
    if code:
        st.k_scale, st.v_scale = (torch.ones(9, 2, 16) for _ in range(2))
    for _ in range(2):
        at = _bound(st.pages, st.desc)
        for name, x in at.items():
            assert x == (None if getattr(st, name) is None else getattr(st, name).data_ptr()), name
        assert st.pages.c.npages == 9 and st.table.data_ptr() == st.pages.table.data_ptr()
    st.deal()                                                        # nine pages: into the table that is there now
    assert st.table.flatten().tolist() == list(range(8))
    st.pages.table = torch.full((2, 1, 4), 3, dtype=torch.int32)
    assert st.table is st.pages.table and _bound(st.pages, st.desc)["table"] == st.table.data_ptr()
    st.table[0, 0, 1] = 5
    assert st.pages.table[0, 0, 1] == 5


def test_sections_that_no_structure_holds():
    for bad in ([2 ** 32 + 64], [64 - 2 ** 32, 0], [2 ** 31, 64], [65], [-1, 65]):
        with pytest.raises(ValueError):
            corm.Rotation(torch.ones(64), sections=bad)
    with pytest.raises(ValueError):
        corm.Rotation(None, sections=[2 ** 32])
    assert list(corm.Rotation(torch.ones(64), sections=[40, 0, 24]).c.section) == [40, 0, 24, 0]
