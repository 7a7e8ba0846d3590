"""What the binding does around the training operators and the layer's training settings, without a GPU."""
import pytest
import torch

from paper_2312_07987_b200 import binding as b


@pytest.mark.parametrize("shape,strides", [((2, 3, 2, 8), (100, 1, 40, 1)), ((3, 4, 2, 16), (4, 12, 1, 1)), ((2, 3, 2, 8), (0, 1, 0, 1)), ((2, 3, 2, 8), (1, 1, 1, 1)),
                                           ((2, 3, 2, 8), (48, 8, 24, 1)), ((2, 3, 2, 1), (6, 2, 1, 5)), ((2, 0, 2, 8), (0, 1, 0, 1)), ((1, 1, 1, 2), (7, 7, 7, 1))])
def test_outputs_of_heads_have_dense_rows_of_their_own(shape, strides):
    t = torch.zeros(1000).as_strided(shape, strides)
    out, (at, *_, ) = b._heads_like(t)
    assert out.shape == t.shape and out.dtype == t.dtype and at == out.data_ptr()
    assert out.stride(3) == 1 or shape[3] == 1
    if out.numel():
        places = torch.zeros(out.untyped_storage().nbytes() // 4, dtype=torch.int32)
        places.as_strided(out.shape, out.stride()).fill_(1)
        assert int(places.sum()) == out.numel()              # no two elements at one address


def test_outputs_of_heads_keep_the_order_of_dimensions():
    for t in (torch.zeros(2, 5, 3, 8), torch.zeros(2, 3, 5, 8).transpose(1, 2)):
        out, fields = b._heads_like(t)
        assert out.stride() == t.stride() and fields == (out.data_ptr(), *t.stride()[:3])
