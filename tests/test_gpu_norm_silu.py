"""silu value by value: with a scale of zero the activation is that of the shift itself."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [(1, 3, 2), (1, 300, 211)], ids=str)
def test_silu_and_its_slope_keep_the_bits_of_fp32(size):
    """An exponential and a quotient of 2 * 2^-24 each, two products and a sum: 8 * 2^-24 of the value; of the slope, whose two terms may cancel, of both."""
    from paper_2210_09887_amd import ops
    C = 1024
    beta = torch.linspace(-60, 60, C)
    x = torch.randn((*size, C), generator=torch.Generator().manual_seed(1))
    gamma = torch.zeros(C)
    y, m, r = ops.group_norm(x.cuda(), 8, gamma.cuda(), beta.cuda(), act="silu")
    u = beta.double()
    s = torch.sigmoid(u)
    assert float(((y.double().cpu() - u * s).abs() / (u * s).abs()).max()) < 8 * 2.0 ** -24
    dy = torch.zeros_like(x)
    dy[:, 0, 0] = 1                                      # one pixel: its slope is the gradient of the shift
    db = ops.group_norm_backward(x.cuda(), dy.cuda(), m, r, 8, gamma.cuda(), beta.cuda(), "silu")[2]
    off = (db.double().cpu() - (s + u * s * (1 - s))).abs() / (s + (u * s * (1 - s)).abs())
    assert float(off.max()) < 8 * 2.0 ** -24, float(off.max()) * 2 ** 24
