"""Which tensors the autograd functions of the encoder operators hand on as they are, and which they copy."""
import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2607_03574_amd")


def test_rows_that_the_kernels_take():
    from paper_2607_03574_amd import torch_api
    x = torch.arange(60.0).view(3, 4, 5)
    for same in (x, x[:, :, 1:4], x[:, :1], x[1:, :, :1], torch.empty(0, 5), torch.empty(3, 0), x[0, 0]):
        assert torch_api._rows(same) is same
    one = torch.arange(5.0)
    for copied in (one.expand(4, 5), one.expand(2, 3, 5), one.as_strided((3, 4), (0, 1)), one.as_strided((2, 4), (1, 1)), x.transpose(1, 2),
                   x.transpose(0, 1), one[:1].expand(5)):
        rows = torch_api._rows(copied)
        assert rows.is_contiguous() and rows.data_ptr() != copied.data_ptr() and torch.equal(rows, copied)
