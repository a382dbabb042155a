"""What the bounds of the attention tests notice: weights held in fewer bits than they have, and small rows that are dropped, as mistakes planted in the
plain form, on the CPU."""
import pytest
import torch

from tests import paged_inputs as inp
from tests import paged_ref as ref


@pytest.mark.parametrize("n", [2, 5, 20, 300])
def test_the_bound_notices_a_lost_part_of_the_weights(n):
    q, k, v = inp.one_channel(torch.Generator().manual_seed(n), "f32", 1, 8, 1, n, 128)
    q, k, v = q[0].double(), k[0, 0].double(), v[0, 0].double()
    want, bound = ref.attend(q, k, v, ref.sm_of(128)), ref.weighted_error(q, k, v, ref.sm_of(128))
    assert bool(((ref.attend_in_parts(q, k, v, ref.sm_of(128), 3) - want).abs() <= bound).all())
    assert bool(((ref.attend_in_parts(q, k, v, ref.sm_of(128), 1) - want).abs() > bound).any())


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_the_bound_of_a_single_row_notices_lost_parts_and_dropped_rows(code):
    """A head's weight lies on one row, whose scale may be tiny: the weight's parts are those of the scale."""
    q, k, v, target = inp.one_row(torch.Generator().manual_seed(5), "bf16", 8, 256, 128)
    q, k = q[0].double(), k[0, 0].double()
    codes, scale = ref.quantise_rows(v[0, 0], code)
    rows = codes.double() * scale.double().unsqueeze(-1)
    want = rows[target]
    for parts, fine in ((3, True), (2, False), (1, False)):
        got = ref.attend_in_parts(q, k, codes.double(), ref.sm_of(128), parts, scale)
        assert bool(((got - want).abs() <= inp.ONE_ROW * want.abs()).all()) == fine, parts
    dropped = torch.where(rows.abs().amax(-1, keepdim=True) < 1e-2 * rows.abs().max(), torch.zeros_like(rows), rows)
    assert bool(((ref.attend(q, k, dropped, ref.sm_of(128)) - want).abs() > inp.ONE_ROW * want.abs()).any())
