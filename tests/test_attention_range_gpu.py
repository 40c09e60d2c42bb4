"""Attention at the ends of its range: very many heads, and an example so long that it is held to the 64-bit form in strips of queries."""
import math

import pytest
import torch

from paper_2502_01703_b200 import binding as B
from test_layer_gpu import HALF, attention_exact, attention_inputs, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("off,H,K,D", [([0, 37, 60], 4096, 1, 8), ([0, 1, 20], 4096, 4096, 8), ([0, 150], 2048, 128, 16)])
def test_very_many_heads(off, H, K, D):
    T = off[-1]
    q, k, v, dout = attention_inputs(T, H, K, D, seed=H + K)
    got = B.qless_attention(q, k, v, off)
    back = B.qless_attention_backward(dout, q, k, v, got["out"], got["lse"], off)
    want, room = attention_exact(q, k, v, off, D ** -0.5, dout, got["out"])
    # a key's gradient sums T H / K terms: with 4096 heads to a key head more than the 2^14 that a tolerance of 2^-13 stands for, T H / K / 16 additions of 2^-23
    more = max(0.0, T * H / K / 16 * 2.0 ** -23 - 2.0 ** -13)
    for n in ("grad_k", "grad_v"):
        room[n] = room[n] * (1 + more / HALF)                # (each room is at least HALF times the sum of absolute values that the additions' error counts by)
    for n in ("lse", "out", "grad_v", "grad_q", "grad_k"):
        close({**got, **back}[n], want[n], room[n])
    B.qless_check()


@pytest.mark.parametrize("T,H,K,D", [(70001, 2, 1, 64), (40003, 3, 3, 128)])
def test_a_very_long_example(T, H, K, D):
    q, k, v, dout = attention_inputs(T, H, K, D, seed=T, sharp=2.0)
    got = B.qless_attention(q, k, v, [0, T])
    back = B.qless_attention_backward(dout, q, k, v, got["out"], got["lse"], [0, T])
    B.qless_check()
    # as in attention_exact, with T H / K / 16 additions of 2^-23 in the longest sums
    sums, scale = T * H / K / 16 * 2.0 ** -23, D ** -0.5
    f = dict(dtype=torch.float64, device="cuda")
    for c in range(K):
        Kk, V = k[:, c].double(), v[:, c].double()
        gk, gv, rk, rv = [torch.zeros((T, D), **f) for _ in range(4)]
        for h in range(c * (H // K), (c + 1) * (H // K)):
            for lo in range(0, T, 2000):
                hi = min(T, lo + 2000)
                Q, dO, O, keys = q[lo:hi, h].double(), dout[lo:hi, h].double(), got["out"][lo:hi, h].double(), slice(0, hi)
                s = scale * Q @ Kk[keys].T
                s.masked_fill_(torch.arange(hi, device="cuda")[None, :] > torch.arange(lo, hi, device="cuda")[:, None], -math.inf)
                lse = torch.logsumexp(s, dim=1)
                p = torch.exp(s - lse[:, None])
                o = p @ V[keys]
                close(got["lse"][lo:hi, h], lse, 2.0 ** -20 * (1 + lse.abs() + scale * (Q.abs() @ Kk[keys].abs().T).amax(dim=1)) + sums)
                close(got["out"][lo:hi, h], o, HALF * o.abs() + (HALF * (1 + HALF) + sums) * (p @ V[keys].abs()))
                dp = dO @ V[keys].T
                ds = p * (dp - (dO * o).sum(dim=1, keepdim=True))
                rho = (dO * (o - O)).sum(dim=1, keepdim=True)
                eds = p * sums * 2 * (dO.abs() @ V[keys].abs().T + (dO * O).abs().sum(dim=1, keepdim=True))
                gq = scale * ds @ Kk[keys]
                rq = scale * (eds + (HALF + sums) * ((ds + p * rho).abs() + p * rho.abs())) @ Kk[keys].abs()
                close(back["grad_q"][lo:hi, h], gq, rq * (1 + HALF) + HALF * gq.abs())
                gk[keys] += scale * ds.T @ Q
                rk[keys] += scale * (eds + (HALF + sums) * ds.abs()).T @ Q.abs()
                gv[keys] += p.T @ dO
                rv[keys] += (HALF + sums) * p.T @ dO.abs()
        close(back["grad_k"][:, c], gk, rk * (1 + HALF) + HALF * gk.abs())
        close(back["grad_v"][:, c], gv, rv * (1 + HALF) + HALF * gv.abs())
