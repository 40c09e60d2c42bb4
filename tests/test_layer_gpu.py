"""Normalisation, packed causal attention and the gated feed-forward block, forward and backward, against plain 64-bit implementations of the formulas.

Tolerances are bounds, element by element, from the roundings that lie between the exact value and the kernel's: a result rounded to bf16 is off by at most
HALF = 2^-8 of itself; an operand rounded to bf16 inside (probabilities, ds, hidden, grad_gate, grad_up) moves a product's sum by at most HALF times the sum of
the products' absolute values; fp32 arithmetic (accumulators that cut instead of rounding, exponentials, sums) by at most SUMS = 2^-13 of that sum, where
a contraction has at most 2^14 terms in steps of 16: 2^10 additions of 2^-23 each."""
import math

import pytest
import torch

from paper_2502_01703_b200 import binding as B

pytestmark = pytest.mark.gpu

HALF, SUMS = 2.0 ** -8, 2.0 ** -13


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def close(have, want, room):
    have = have.double()
    assert have.shape == want.shape
    assert torch.isfinite(have).all()
    off = (have - want).abs() - room
    assert float(off.max() if off.numel() else -1.0) <= 0.0, (float(((have - want).abs() / (room + 1e-300)).max()), float((have - want).norm() / want.norm()))


# ---- normalisation -----------------------------------------------------------------------------------------------------

NORMS = [(1, 1), (1, 8), (3, 1024), (37, 512), (130, 1025), (64, 4096), (65, 4112), (9, 8200), (5, 16384), (3, 16383), (1000, 72), (513, 24), (2000, 1032)]


def norm_inputs(T, W, dtype, pdtype, pad, seed=3):
    g = gen(seed + T * 7 + W)
    x = torch.randn((T, W + pad), generator=g, device="cuda")[:, :W] * 2 + 0.5
    full = torch.zeros((T, W + pad), dtype=dtype, device="cuda")
    full[:, :W] = x.to(dtype)
    w = (1 + 0.3 * torch.randn(W, generator=g, device="cuda")).to(pdtype)
    b = (0.2 * torch.randn(W, generator=g, device="cuda")).to(pdtype)
    dy = torch.randn((T, W), generator=g, device="cuda").to(dtype)
    return full[:, :W], w, b, dy


@pytest.mark.parametrize("dtype,pdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T,W", NORMS)
def test_layer_norm(T, W, dtype, pdtype):
    for center, bias, pad in ((True, True, 0), (False, False, 8), (True, False, 3)):
        x, w, b, dy = norm_inputs(T, W, dtype, pdtype, pad)
        got = B.qless_layer_norm(x, w, b if bias else None, eps=1e-5, center=center)
        X, Wt, DY = x.double(), w.double(), dy.double()
        mu = X.mean(dim=1, keepdim=True) if center else torch.zeros((T, 1), dtype=torch.float64, device="cuda")
        r = 1 / torch.sqrt(((X - mu) ** 2).mean(dim=1, keepdim=True) + 1e-5)
        xh = (X - mu) * r
        want = xh * Wt + (b.double() if bias else 0.0)
        # fp32: the mean is off by at most 2^-19 of the mean size (sums of at most 37 additions after one another), xh by that and 2^-20 of itself
        unit, step = 2.0 ** -19, HALF if dtype == torch.bfloat16 else 0.0
        size = X.abs().mean(dim=1, keepdim=True)
        dxh = unit * (xh.abs() + size * r)
        if center:
            close(got["mean"], mu[:, 0], unit * size[:, 0])
        # where a row is nearly constant (one column), its spread is made of eps alone
        close(got["rstd"], r[:, 0], (unit + 2 * unit * (size * r) ** 2)[:, 0] * r[:, 0])
        drift = unit * (size * r) ** 2 * 2
        close(got["out"], want, (dxh + drift * xh.abs()) * Wt.abs() + (step + 2.0 ** -22) * want.abs())
        back = B.qless_layer_norm_backward(dy, x, w, got["mean"], got["rstd"], want_weight=True, want_bias=bias)
        # from the statistics as given
        m0 = got["mean"].double()[:, None] if center else 0.0
        r0 = got["rstd"].double()[:, None]
        xh = (X - m0) * r0
        gw = DY * Wt
        dx = r0 * (gw - (gw.mean(dim=1, keepdim=True) if center else 0.0) - xh * (gw * xh).mean(dim=1, keepdim=True))
        room = r0 * unit * (gw.abs() + gw.abs().mean(dim=1, keepdim=True) + xh.abs() * (gw * xh).abs().mean(dim=1, keepdim=True))
        close(back["grad_x"], dx, room + step * dx.abs())
        pstep = HALF if pdtype == torch.bfloat16 else 0.0
        dw, db = (DY * xh).sum(dim=0), DY.sum(dim=0)
        close(back["grad_weight"], dw, unit * (DY * xh).abs().sum(dim=0) + pstep * dw.abs())
        if bias:
            close(back["grad_bias"], db, unit * DY.abs().sum(dim=0) + pstep * db.abs())
        else:
            assert back["grad_bias"] is None
        alone = B.qless_layer_norm_backward(dy, x, w, got["mean"], got["rstd"])
        assert alone["grad_weight"] is None and torch.equal(alone["grad_x"], back["grad_x"])


# ---- attention ---------------------------------------------------------------------------------------------------------

def attention_exact(q, k, v, off, scale, dout=None, out=None):
    """Results and their rooms: out, lse and, with dout, the gradients. `out` as given to the backward pass counts for roundings only: ds is rounded as it is
    with delta taken from it, and put right by rho = <dout, exact out - out> times the mean of the keys, whose probabilities are rounded."""
    T, H, D = q.shape
    K = k.shape[1]
    f = dict(dtype=torch.float64, device="cuda")
    got = {n: torch.zeros(s, **f) for n, s in (("out", q.shape), ("lse", (T, H)), ("grad_q", q.shape), ("grad_k", k.shape), ("grad_v", k.shape))}
    room = {n: torch.zeros_like(t) for n, t in got.items()}
    for lo, hi in zip(off, off[1:]):
        if lo == hi:
            continue
        mask = torch.ones((hi - lo, hi - lo), dtype=torch.bool, device="cuda").triu(1)
        for h in range(H):
            c = h // (H // K)
            Q, Kk, V = q[lo:hi, h].double(), k[lo:hi, c].double(), v[lo:hi, c].double()
            s = (scale * Q @ Kk.T).masked_fill(mask, -math.inf)
            lse = torch.logsumexp(s, dim=1)
            p = torch.exp(s - lse[:, None])
            o = p @ V
            got["out"][lo:hi, h], got["lse"][lo:hi, h] = o, lse
            room["out"][lo:hi, h] = HALF * o.abs() + (HALF * (1 + HALF) + SUMS) * (p @ V.abs())
            room["lse"][lo:hi, h] = 2.0 ** -20 * (1 + lse.abs() + scale * (Q.abs() @ Kk.abs().T).amax(dim=1))
            if dout is None:
                continue
            dO, O = dout[lo:hi, h].double(), out[lo:hi, h].double()
            dp = dO @ V.T
            ds = p * (dp - (dO * o).sum(dim=1, keepdim=True))
            rho = (dO * (o - O)).sum(dim=1, keepdim=True)
            rough = (ds + p * rho).abs()
            # dp, delta and rho are fp32 sums of products
            eds = p * SUMS * 2 * (dO.abs() @ V.abs().T + (dO * O).abs().sum(dim=1, keepdim=True))
            got["grad_q"][lo:hi, h] = scale * ds @ Kk
            room["grad_q"][lo:hi, h] = scale * (eds + (HALF + SUMS) * (rough + p * rho.abs())) @ Kk.abs()
            got["grad_k"][lo:hi, c] += scale * ds.T @ Q
            room["grad_k"][lo:hi, c] += scale * (eds + (HALF + SUMS) * ds.abs()).T @ Q.abs()
            got["grad_v"][lo:hi, c] += p.T @ dO
            room["grad_v"][lo:hi, c] += (HALF + SUMS) * p.T @ dO.abs()
    for n in ("grad_q", "grad_k", "grad_v"):
        room[n] = room[n] * (1 + HALF) + HALF * got[n].abs()
    return got, room


def attention_inputs(T, H, K, D, seed, sharp=1.5, fused=False):
    g = gen(seed)
    if fused:                                # slices of one matrix
        m = torch.randn((T, (H + 2 * K) * D + 8), generator=g, device="cuda").to(torch.bfloat16)
        q, k, v = m[:, :H * D].view(T, H, D), m[:, H * D:(H + K) * D].unflatten(1, (K, D)), m[:, (H + K) * D:(H + 2 * K) * D].unflatten(1, (K, D))
    else:
        q, k, v = [torch.randn((T, n, D), generator=g, device="cuda").to(torch.bfloat16) for n in (H, K, K)]
        k = (k.float() * sharp).to(torch.bfloat16)
    return q, k, v, (torch.randn((T, H, D), generator=g, device="cuda") * 0.1).to(torch.bfloat16)


ATTN = [
    ([0, 1], 1, 1, 8), ([0, 1], 8, 2, 128), ([0, 2, 3], 4, 4, 64), ([0, 127], 2, 1, 64), ([0, 128], 4, 1, 128), ([0, 129], 4, 2, 128), ([0, 257], 2, 2, 80),
    ([0, 0, 5, 5, 300, 301, 700, 700], 8, 2, 128), ([0, 31, 62, 95, 96, 130], 16, 1, 64), ([0, 640], 7, 1, 96), ([0, 515], 28, 4, 64),
    ([0, 1000, 1333], 6, 2, 40), ([0, 383, 384, 1500], 32, 2, 128), ([0, 2049], 2, 1, 128), ([0] + list(range(1, 200)), 4, 2, 64),
    ([0, 200, 333], 48, 3, 56), ([0, 96], 64, 1, 120), ([0, 1100], 12, 12, 16),
]


@pytest.mark.parametrize("off,H,K,D", ATTN)
def test_attention(off, H, K, D):
    T = off[-1]
    for fused in (False, True):
        q, k, v, dout = attention_inputs(T, H, K, D, seed=T + H + D, fused=fused)
        got = B.qless_attention(q, k, v, off)
        want, room = attention_exact(q, k, v, off, D ** -0.5, dout, got["out"])
        close(got["lse"], want["lse"], room["lse"])
        close(got["out"], want["out"], room["out"])
        back = B.qless_attention_backward(dout, q, k, v, got["out"], got["lse"], off)
        for n in ("grad_v", "grad_q", "grad_k"):
            close(back[n], want[n], room[n])
    B.qless_check()


# ---- feed-forward block ------------------------------------------------------------------------------------------------

def act64(name, g):
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    F = 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * F, F + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


FFNS = [(1, 8, 8), (1, 512, 1376), (5, 64, 72), (16, 256, 640), (17, 520, 1000), (61, 1024, 2752), (200, 264, 696), (256, 512, 1376), (257, 512, 1376),
        (300, 136, 264), (513, 1000, 2048), (1500, 768, 1112),
        # tiles beyond whole rounds of the pairs, which are shared: 12 of 16 columns' tiles; more than a round; a contraction of one stage that is not shared
        (700, 2048, 4096), (2500, 2304, 2816), (5000, 128, 1400)]


def check_ffn_forward(got, x, wg, wu, wd, act):
    X, G, U, D = x.double(), wg.double(), wu.double(), wd.double()
    gate, up = X @ G.T, X @ U.T
    eg, eu = SUMS * (X.abs() @ G.abs().T), SUMS * (X.abs() @ U.abs().T)
    close(got["gate"], gate, eg + HALF * gate.abs())
    close(got["up"], up, eu + HALF * up.abs())
    a, da = act64(act, gate)
    h = a * up
    # the slope of both activations is at most 1.13; exponential and quotient cost 2^-18 of the value
    eh = 1.13 * eg * (up.abs() + eu) + (a.abs() + 2.0 ** -18 * a.abs()) * eu + 2.0 ** -18 * h.abs() + HALF * h.abs() + 1e-7
    close(got["hidden"], h, eh * (1 + HALF))
    y = h @ D.T
    close(got["out"], y, (eh * (1 + HALF) + SUMS * h.abs()) @ D.abs().T * (1 + HALF) + HALF * y.abs())


def check_ffn_backward(back, dy, x, gate, up, wg, wu, wd, act):
    """From gate and up as given; the weights' gradients where there are any."""
    X, G, U, D, DY, gate, up = [t.double() if t is not None else None for t in (x, wg, wu, wd, dy, gate, up)]
    a, da = act64(act, gate)
    dh, edh = DY @ D, SUMS * (DY.abs() @ D.abs())
    dg, du, h = dh * up * da, dh * a, a * up
    edg = (edh * da.abs() + 2.0 ** -17 * dh.abs()) * up.abs() + HALF * dg.abs() + 1e-7
    edu = edh * a.abs() + 2.0 ** -17 * du.abs() + HALF * du.abs() + 1e-7
    edg, edu, eh = edg * (1 + HALF), edu * (1 + HALF), (HALF + 2.0 ** -17) * h.abs() + 1e-7
    close(back["grad_gate"], dg, edg)
    close(back["grad_up"], du, edu)
    want = dict(grad_x=(dg @ G + du @ U, (edg + SUMS * dg.abs()) @ G.abs() + (edu + SUMS * du.abs()) @ U.abs()))
    if back["grad_w_gate"] is not None:
        want.update(grad_w_gate=(dg.T @ X, (edg + SUMS * dg.abs()).T @ X.abs()), grad_w_up=(du.T @ X, (edu + SUMS * du.abs()).T @ X.abs()),
                    grad_w_down=(DY.T @ h, DY.abs().T @ (eh + SUMS * h.abs())))
    for name, (exact, room) in want.items():
        close(back[name], exact, room * (1 + HALF) + HALF * exact.abs())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,W,F", FFNS)
def test_gated_ffn(T, W, F, act):
    g = gen(T + W + F)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = torch.cat([rand(T, W), rand(T, 8)], dim=1).to(torch.bfloat16)[:, :W]
    wg, wu, wd = [(rand(*s) * 1.3 * s[1] ** -0.5).to(torch.bfloat16) for s in ((F, W), (F, W), (W, F))]
    dy = rand(T, W).to(torch.bfloat16)
    got = B.qless_gated_ffn(x, wg, wu, wd, activation=act, want_saved=True)
    check_ffn_forward(got, x, wg, wu, wd, act)
    alone = B.qless_gated_ffn(x, wg, wu, wd, activation=act)
    assert alone["gate"] is None and torch.equal(alone["out"], got["out"]) and torch.equal(alone["hidden"], got["hidden"])
    back = B.qless_gated_ffn_backward(dy, x, got["gate"], got["up"], wg, wu, wd, activation=act, want_weight=True)
    check_ffn_backward(back, dy, x, got["gate"], got["up"], wg, wu, wd, act)
    alone = B.qless_gated_ffn_backward(dy, None, got["gate"], got["up"], wg, wu, wd, activation=act)
    assert alone["grad_w_up"] is None and all(torch.equal(alone[n], back[n]) for n in ("grad_x", "grad_gate", "grad_up"))
    B.qless_check()
