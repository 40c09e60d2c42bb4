"""Normalisation's backward pass where its rows are very many or very small: rings of rows that are filled many times over, and rows whose spread is so small
that the cube of 1 / spread leaves fp32's range."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B
from test_layer_gpu import HALF, close, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("W", [24, 1000, 4112, 333, 8200])
@pytest.mark.parametrize("center", [True, False])
def test_rows_whose_spread_is_tiny(W, dtype, center):
    """eps = 0 and a spread of 4e-20: 1 / spread is 2.5e19, its cube no fp32 number, the gradients (some 1e20) are."""
    T = 37
    g = gen(W)
    x = (torch.randn((T, W), generator=g, device="cuda") * 4e-20).to(dtype)
    w = (1 + 0.3 * torch.randn(W, generator=g, device="cuda")).to(dtype)
    dy = torch.randn((T, W), generator=g, device="cuda").to(dtype)
    got = B.qless_layer_norm(x, w, eps=0.0, center=center)
    X, Wt, DY = x.double(), w.double(), dy.double()
    mu = X.mean(dim=1, keepdim=True) if center else 0.0
    r = 1 / torch.sqrt(((X - mu) ** 2).mean(dim=1, keepdim=True))
    # squares of 1.6e-39 and their mean are subnormal: each is off by at most 2^-150, half of their last place (relative to 1.6e-39: 2^-20.1); small squares of a
    # row count by what they add. With the mean's own error (2^-19 of the mean size, and size r < 1) below 2^-18 in all.
    close(got["rstd"], r[:, 0], 2.0 ** -18 * r[:, 0])
    back = B.qless_layer_norm_backward(dy, x, w, got["mean"], got["rstd"], want_weight=True)
    # from the statistics as given, as wherever rows are larger
    m0 = got["mean"].double()[:, None] if center else 0.0
    r0 = got["rstd"].double()[:, None]
    xh, gw = (X - m0) * r0, DY * Wt
    dx = r0 * (gw - (gw.mean(dim=1, keepdim=True) if center else 0.0) - xh * (gw * xh).mean(dim=1, keepdim=True))
    # fp32 sums and products: 2^-19, as in the tests of larger rows. The products of a row's second mean are g d, some 4e-20, far above what is subnormal.
    room = r0 * 2.0 ** -19 * (gw.abs() + gw.abs().mean(dim=1, keepdim=True) + xh.abs() * (gw * xh).abs().mean(dim=1, keepdim=True))
    step = HALF if dtype == torch.bfloat16 else 0.0
    close(back["grad_x"], dx, room + step * dx.abs())
    close(back["grad_weight"], (DY * xh).sum(dim=0), 2.0 ** -19 * (DY * xh).abs().sum(dim=0) + step * (DY * xh).sum(dim=0).abs())
    alone = B.qless_layer_norm_backward(dy, x, w, got["mean"], got["rstd"])
    assert torch.equal(alone["grad_x"], back["grad_x"])


@pytest.mark.parametrize("dtype,pdtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T,W", [(40000, 64), (20001, 512), (20000, 1032), (3001, 4112), (2999, 8192), (5003, 16384), (70003, 8)])
def test_more_rows_than_a_ring_holds(T, W, dtype, pdtype):
    """Values and statistics are small whole numbers and halves, so that the parameters' gradients are exact in fp32 whatever the order of the sums: a row that is
    left out, taken twice, or overwritten before it is read shows."""
    g = gen(T + W)
    draw = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, generator=g, device="cuda")  # noqa: E731
    x, dy = draw(-2, 2, T, W).to(dtype), draw(-3, 3, T, W).to(dtype)
    w = (draw(1, 4, W) * 0.5).to(pdtype)
    mean, rstd = draw(-1, 1, T).float(), torch.exp2(draw(-1, 1, T).float())
    for center in (True, False):
        back = B.qless_layer_norm_backward(dy, x, w, mean if center else None, rstd, want_weight=True, want_bias=True)
        DY, R = dy.double(), rstd.double()[:, None]
        xh = (x.double() - (mean.double()[:, None] if center else 0.0)) * R
        # sums of halves: at most 70003 x 18 x 2 < 2^24 halves
        assert torch.equal(back["grad_weight"], (DY * xh).sum(dim=0).float().to(pdtype))
        assert torch.equal(back["grad_bias"], DY.sum(dim=0).float().to(pdtype))
        gw = DY * w.double()
        m, a = gw.mean(dim=1, keepdim=True) if center else 0.0, (gw * xh).mean(dim=1, keepdim=True)
        dx = R * (gw - m - xh * a)
        # fp32: g, xh and their sums are exact; the two means and the three products of a value are off by less than 2^-21 of what they add
        room = R * 2.0 ** -21 * (gw.abs() + abs(m) + (xh * a).abs())
        close(back["grad_x"], dx, room + (HALF if dtype == torch.bfloat16 else 0.0) * dx.abs())
        alone = B.qless_layer_norm_backward(dy, x, w, mean if center else None, rstd)
        assert torch.equal(alone["grad_x"], back["grad_x"])
    B.qless_check()
