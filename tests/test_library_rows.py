"""CPU-only: the row strides that tensor arguments are passed on with."""
import pytest
import torch

BF = torch.bfloat16


@pytest.fixture(scope="module")
def api():
    from paper_2608_00938_b200 import build
    build()
    from paper_2608_00938_b200 import api as _api
    return _api


@pytest.mark.parametrize("stride", [0, 1, 511, 512, 513, 100000])
def test_a_single_row_counts_as_its_width(api, stride):
    t = torch.zeros(100513, dtype=BF).as_strided((1, 512), (stride, 1))
    assert api._rows(t, "call", "x", BF, -1) == (t.data_ptr(), 512)


def test_rows_keep_their_stride(api):
    t = torch.zeros(4000, dtype=BF)
    assert api._rows(t.as_strided((3, 512), (513, 1)), "call", "x", BF, -1)[1] == 513
    assert api._rows(t.as_strided((3, 512), (0, 1)), "call", "x", BF, -1)[1] == 0         # (refused by the entries: below the width)
    assert api._rows(t.as_strided((3, 1), (7, 5)), "call", "x", BF, -1)[1] == 7
    assert api._rows(None, "call", "x", BF, -1) == (None, 0)
    for bad in (t.as_strided((3, 4), (1, 3)), t.as_strided((1, 4), (1, 2)), t[:4], t.float()[:4].view(2, 2)):
        with pytest.raises(ValueError):
            api._rows(bad, "call", "x", BF, -1)
