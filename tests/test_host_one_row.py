"""A single row is passed on with its own length as the stride, whatever its tensor's stride is."""

import pytest

torch = pytest.importorskip("torch")

import paper_2512_04013_amd as aug  # noqa: E402


def test_strides_of_rows():
    x = torch.zeros(8, 1, 128)
    for t in (x.transpose(0, 1), torch.zeros(1, 8, 128), torch.zeros(1, 8, 128).as_strided((1, 8, 128), (7, 128, 1)),
              torch.zeros(1, 8, 128).expand(1, 8, 128), torch.zeros(9, 1024)[3:4].view(1, 8, 128)):
        assert aug._rows_arg(t) == (t.data_ptr(), 1024)
    assert aug._rows_arg(torch.zeros(5, 2000)[:, :1024].view(5, 8, 128))[1] == 2000
    assert aug._rows_arg(None) == (None, 0)
