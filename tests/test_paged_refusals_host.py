"""More refusals of the calls over pages, on the host: strides of rows whose offsets leave 64 bits, fields that have to be 0."""
import pytest

from paper_2404_15949_amd import corm
from tests import test_paged_host as host

A = host.A


def _refused_for_the_strides(n, B=2, **strides):
    """What corm_rotate says to a call whose only fault is in the strides; one without it is refused too, as its launch has more threads than there are."""
    return host._call("corm_rotate", host._desc(B=B), rows=host._rows(**strides), n=n)


def test_strides_whose_offsets_leave_64_bits():
    """Every stride by itself is one that is taken, the last row is not in 64 bits: 2^40 elements a token, 2^31 - 1 tokens."""
    E, U, n, most = corm.CORM_EINVAL, corm.CORM_EUNSUPPORTED, 2147483647, 1 << 40
    assert _refused_for_the_strides(n) == U and _refused_for_the_strides(n, k_stride=(most, 8, most)) == U
    for x in ("q", "k", "v"):
        assert _refused_for_the_strides(n, **{x + "_stride": (768, most, 128)}) == E, x
        assert _refused_for_the_strides(n, **{x + "_stride": (768, 1 << 32, 128)}) == E, x          # 2^31 x 2^32 x 2 bytes
        assert _refused_for_the_strides(n, **{x + "_stride": (768, 1 << 29, 128)}) == U, x          # 2^61: in range
    assert _refused_for_the_strides(n, B=1, k_stride=(most, 1 << 29, most)) == U                      # (2^60 and little more)
    # without queries theirs are not looked at
    assert host._call("corm_rotate", rows=host._rows(q_stride=(768, most, 128)), n=n, q_out=None) == U


def test_strides_of_a_prompt_in_pages():
    """The same check on the way into pages, where n is a length at most: 2^21 tokens of 2^40 fp32 elements."""
    d = host._desc(Lcap=1 << 21, kv_dtype="f32")
    pages = host._pages(dtype=corm.CORM_F32, max_pages=1 << 17)
    assert host._call("corm_paged_append", d, pages=pages, n=1 << 21, rows=host._rows(k_stride=(768, 1 << 40, 128))) == corm.CORM_EINVAL


@pytest.mark.parametrize("name", [n for n in host.CALLS if "pages" in host.CALLS[n][0]])
def test_reserved_fields_are_zero(name):
    for x in (1, -1, 1 << 30):
        assert host._call(name, pages=host._pages(reserved=x)) == corm.CORM_EINVAL, x
    assert host._call("corm_paged_attend", pages=host._pages()) == corm.CORM_ECAPACITY       # 16 bytes of workspace: fine but for that
