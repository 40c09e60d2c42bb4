"""Refusals of the calls that carry a gradient through a decoder layer, checked without a GPU: every bad argument returns its status before anything is launched,
and the binding refuses tensors that it cannot pass on."""
import ctypes as C

import pytest
import torch

from paper_2502_01703_b200 import binding as B

FAKE, ODD = C.c_void_p(4096), C.c_void_p(4096 + 8)


@pytest.fixture(scope="module")
def L():
    from paper_2502_01703_b200 import build
    build.build()
    return B.lib()


def test_layer_norm_refusals(L):
    def norm(x=FAKE, dtype=B.BF16, tokens=4, width=64, ld=64, w=FAKE, b=FAKE, pd=B.BF16, eps=1e-5, center=1, out=FAKE, ldo=64, mean=FAKE, rstd=FAKE):
        return L.qless_layer_norm(x, dtype, tokens, width, ld, w, b, pd, eps, center, out, ldo, mean, rstd, None)

    assert norm(tokens=-1) == B.ERR_INVALID_ARG and norm(width=0) == B.ERR_INVALID_ARG
    assert norm(dtype=7) == B.ERR_INVALID_ARG and norm(pd=-1) == B.ERR_INVALID_ARG
    assert norm(width=16385, ld=16385, ldo=16385) == B.ERR_UNSUPPORTED and b"16384" in L.qless_last_error()
    assert norm(tokens=1 << 31) == B.ERR_UNSUPPORTED
    assert norm(eps=-1e-5) == B.ERR_INVALID_ARG and norm(eps=float("nan")) == B.ERR_INVALID_ARG and norm(eps=float("inf")) == B.ERR_INVALID_ARG
    assert norm(x=None) == B.ERR_INVALID_ARG and norm(w=None) == B.ERR_INVALID_ARG and norm(out=None) == B.ERR_INVALID_ARG
    assert norm(ld=63) == B.ERR_INVALID_ARG and norm(ldo=63) == B.ERR_INVALID_ARG
    assert norm(x=C.c_void_p(4097)) == B.ERR_INVALID_ARG and norm(mean=C.c_void_p(4098)) == B.ERR_INVALID_ARG
    assert norm(tokens=0, x=None, w=None, out=None) == B.QLESS_OK

    def back(dy=FAKE, ldy=64, x=FAKE, dtype=B.BF16, tokens=4, width=64, ld=64, w=FAKE, pd=B.F32, center=1, mean=FAKE, rstd=FAKE, dx=FAKE, ldx=64, dw=None, db=None,
             ws=None, wsb=0):
        return L.qless_layer_norm_backward(dy, ldy, x, dtype, tokens, width, ld, w, pd, center, mean, rstd, dx, ldx, dw, db, ws, wsb, None)

    assert back(dy=None) == B.ERR_INVALID_ARG and back(rstd=None) == B.ERR_INVALID_ARG and back(dx=None) == B.ERR_INVALID_ARG
    assert back(mean=None) == B.ERR_INVALID_ARG and b"mean" in L.qless_last_error()
    assert back(ldy=60) == B.ERR_INVALID_ARG and back(ldx=60) == B.ERR_INVALID_ARG
    assert back(dw=FAKE) == B.ERR_WORKSPACE and back(db=FAKE, ws=FAKE, wsb=16) == B.ERR_WORKSPACE
    assert back(dw=C.c_void_p(4098)) == B.ERR_INVALID_ARG


def test_attention_refusals(L):
    many = tuple(range(0, 4001, 10))                         # so many tiles that a table is needed

    def attn(q=FAKE, ldq=512, k=FAKE, ldk=128, v=FAKE, ldv=128, off=many, tokens=4000, n=400, heads=8, kv=2, d=64, scale=0.125, out=FAKE, ldo=512, lse=FAKE,
             ws=FAKE, wsb=0):
        o = (C.c_int64 * len(off))(*off) if off is not None else None
        return L.qless_attention(q, ldq, k, ldk, v, ldv, o, tokens, n, heads, kv, d, scale, out, ldo, lse, ws, wsb, None)

    def back(dout=FAKE, lddo=512, q=FAKE, ldq=512, k=FAKE, ldk=128, v=FAKE, ldv=128, out=FAKE, ldo=512, lse=FAKE, off=many, tokens=4000, n=400, heads=8, kv=2, d=64,
             scale=0.125, dq=FAKE, lddq=512, dk=FAKE, lddk=128, dv=FAKE, lddv=128, ws=FAKE, wsb=0):
        o = (C.c_int64 * len(off))(*off) if off is not None else None
        return L.qless_attention_backward(dout, lddo, q, ldq, k, ldk, v, ldv, out, ldo, lse, o, tokens, n, heads, kv, d, scale, dq, lddq, dk, lddk, dv, lddv, ws, wsb, None)

    for call in (attn, back):
        assert call() == B.ERR_WORKSPACE and b"too small" in L.qless_last_error()      # valid but for the workspace
        assert call(ws=None, wsb=1 << 30) == B.ERR_WORKSPACE and call(ws=ODD, wsb=1 << 30) == B.ERR_WORKSPACE
        assert call(tokens=-1) == B.ERR_INVALID_ARG and call(n=-1) == B.ERR_INVALID_ARG and call(heads=0) == B.ERR_INVALID_ARG and call(kv=0) == B.ERR_INVALID_ARG
        assert call(heads=9, ldq=576, ldo=576) == B.ERR_UNSUPPORTED and b"multiple of kv_heads" in L.qless_last_error()
        assert call(d=68) == B.ERR_UNSUPPORTED and call(d=136) == B.ERR_UNSUPPORTED and call(d=0) == B.ERR_INVALID_ARG
        assert call(tokens=1 << 31) == B.ERR_UNSUPPORTED
        for bad in (0.0, -1.0, float("nan"), float("inf")):
            assert call(scale=bad) == B.ERR_INVALID_ARG
        assert call(off=(0, 3, 5), n=2, tokens=4) == B.ERR_INVALID_ARG and call(off=(-1, 3, 4), n=2) == B.ERR_INVALID_ARG and call(off=None) == B.ERR_INVALID_ARG
        assert call(off=(0, 4, 3), n=2) == B.ERR_INVALID_ARG and b"decrease" in L.qless_last_error()
        assert call(q=None) == B.ERR_INVALID_ARG and call(k=ODD) == B.ERR_INVALID_ARG and call(v=None) == B.ERR_INVALID_ARG and call(out=ODD) == B.ERR_INVALID_ARG
        assert call(ldq=504) == B.ERR_INVALID_ARG and call(ldk=132) == B.ERR_INVALID_ARG
        assert call(n=0, off=None, q=None) == B.QLESS_OK and call(tokens=0, n=2, off=(0, 0, 0), q=None, ws=None) == B.QLESS_OK
    long = dict(heads=4096, kv=1, d=8, tokens=20000, n=2)     # 4096 heads share a key head: 2^13 tokens are the most
    for call, wide in ((attn, dict(ldq=32768, ldo=32768)), (back, dict(ldq=32768, ldo=32768, lddo=32768, lddq=32768))):
        assert call(**long, **wide, off=(3, 3, 8196)) == B.ERR_UNSUPPORTED and b"2^25" in L.qless_last_error()
        assert call(**long, **wide, off=(3, 4, 8196)) == B.ERR_WORKSPACE
    assert attn(lse=C.c_void_p(4098)) == B.ERR_INVALID_ARG
    assert back(lse=None) == B.ERR_INVALID_ARG and back(dq=None) == B.ERR_INVALID_ARG and back(lddk=120) == B.ERR_INVALID_ARG and back(dout=ODD) == B.ERR_INVALID_ARG


def test_gated_ffn_refusals(L):
    def ffn(x=FAKE, ldx=2048, wg=FAKE, ldg=2048, wu=FAKE, ldu=2048, wd=FAKE, ldd=8192, tokens=4, width=2048, inner=8192, act=B.SILU, out=FAKE, ldo=2048, h=FAKE, ldh=8192, gate=None,
            up=None, ws=FAKE, wsb=0):
        return L.qless_gated_ffn(x, ldx, wg, ldg, wu, ldu, wd, ldd, tokens, width, inner, act, out, ldo, h, ldh, gate, 8192, up, 8192, ws, wsb, None)

    def back(dy=FAKE, ldy=2048, x=None, ldx=0, gate=FAKE, ldgt=8192, up=FAKE, ldup=8192, wg=FAKE, wu=FAKE, wd=FAKE, tokens=4, width=2048, inner=8192, act=B.GELU, dx=FAKE, lddx=2048,
             dg=FAKE, du=FAKE, dwg=None, dwu=None, dwd=None, ws=FAKE, wsb=0):
        return L.qless_gated_ffn_backward(dy, ldy, x, ldx, gate, ldgt, up, ldup, wg, 2048, wu, 2048, wd, 8192, tokens, width, inner, act, dx, lddx, dg, 8192, du, 8192, dwg, 2048,
                                          dwu, 2048, dwd, 8192, ws, wsb, None)

    for call in (ffn, back):
        assert call() == B.ERR_WORKSPACE and call(ws=ODD, wsb=1 << 30) == B.ERR_WORKSPACE and call(ws=None, wsb=1 << 30) == B.ERR_WORKSPACE
        assert call(tokens=-1) == B.ERR_INVALID_ARG and call(width=0) == B.ERR_INVALID_ARG and call(inner=0) == B.ERR_INVALID_ARG and call(act=2) == B.ERR_INVALID_ARG
        assert call(width=60) == B.ERR_UNSUPPORTED and call(inner=100) == B.ERR_UNSUPPORTED and call(inner=(1 << 20) + 8) == B.ERR_UNSUPPORTED
        assert call(tokens=(1 << 31) - 256) == B.ERR_UNSUPPORTED
        assert call(wg=None) == B.ERR_INVALID_ARG and call(wu=ODD) == B.ERR_INVALID_ARG and call(wd=None) == B.ERR_INVALID_ARG
        assert call(tokens=0, wg=None, wd=None) == B.QLESS_OK
    assert ffn(x=None) == B.ERR_INVALID_ARG and ffn(h=None) == B.ERR_INVALID_ARG and ffn(ldx=2040) == B.ERR_INVALID_ARG and ffn(ldh=8196) == B.ERR_INVALID_ARG
    assert ffn(gate=FAKE) == B.ERR_INVALID_ARG and b"together" in L.qless_last_error() and ffn(up=FAKE) == B.ERR_INVALID_ARG
    assert back(gate=None) == B.ERR_INVALID_ARG and back(dg=None) == B.ERR_INVALID_ARG and back(dx=ODD) == B.ERR_INVALID_ARG and back(dy=None) == B.ERR_INVALID_ARG
    assert back(dwu=FAKE) == B.ERR_INVALID_ARG and b"x is required" in L.qless_last_error()
    assert back(dwd=ODD) == B.ERR_INVALID_ARG
    assert back(dwd=FAKE, tokens=(1 << 27) + 1) == B.ERR_UNSUPPORTED and b"2^27" in L.qless_last_error()
    assert back(dwd=FAKE, tokens=1 << 27) == B.ERR_WORKSPACE


def test_binding_refusals():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    q, k = bf(5, 4, 64), bf(5, 2, 64)
    for off in (torch.tensor([0, 5], dtype=torch.int32), torch.tensor([[0, 5]]), torch.tensor([], dtype=torch.int64)):
        with pytest.raises(TypeError):
            B.qless_attention(q, k, k, off)
    with pytest.raises(TypeError):
        B.qless_attention(q.float(), k, k, [0, 5])
    with pytest.raises(ValueError):
        B.qless_attention(q, k, bf(5, 2, 32), [0, 5])
    with pytest.raises(ValueError):
        B.qless_attention(bf(5, 64, 4).transpose(1, 2), k, k, [0, 5])
    with pytest.raises(ValueError):                          # in host memory
        B.qless_attention(q, k, k, [0, 5])
    with pytest.raises(ValueError):
        B.qless_attention_backward(q, q, k, k, q, torch.zeros(5, 2), [0, 5])
    with pytest.raises(ValueError):
        B.qless_gated_ffn(bf(5, 64), bf(128, 64), bf(120, 64), bf(64, 128))
    with pytest.raises(ValueError):
        B.qless_gated_ffn(bf(5, 64), bf(128, 64), bf(128, 64), bf(64, 128), activation="relu")
    with pytest.raises(ValueError):
        B.qless_gated_ffn_backward(bf(5, 64), None, bf(5, 120), bf(5, 128), bf(128, 64), bf(128, 64), bf(64, 128))
    with pytest.raises(ValueError):
        B.qless_layer_norm(bf(5, 64), bf(32))
    with pytest.raises(TypeError):
        B.qless_layer_norm(bf(5, 64), bf(64), torch.zeros(64))
    with pytest.raises(ValueError):
        B.qless_layer_norm_backward(bf(5, 64), bf(5, 64), bf(64), None, torch.zeros(4))
    with pytest.raises(ValueError):
        B.qless_layer_norm_backward(bf(5, 64).float(), bf(5, 64), bf(64), None, torch.zeros(5))


def test_workspaces():
    assert B.qless_attention_workspace(-1, 1, 8, 2) == 0 and B.qless_gated_ffn_workspace(4, 60, 128) == 0 and B.qless_layer_norm_backward_workspace(4, 20000) == 0
    assert B.qless_layer_norm_backward_workspace(4, 64, False) == 0 and B.qless_layer_norm_backward_workspace(4, 64) >= 4 * 2 * 64 * 4
    # tables of tiles: 32 tokens to a tile of four heads, one more for every example; lse and delta's rows
    assert B.qless_attention_workspace(1 << 20, 100, 32, 8) >= ((1 << 15) + 100) * 16
    assert B.qless_attention_backward_workspace(1 << 20, 100, 32, 8) >= (1 << 20) * 32 * 4
    assert B.qless_attention_workspace(10, 1 << 20, 32, 8) == 0                  # examples without tokens need none, few tiles travel in the launch
    assert B.qless_gated_ffn_workspace(0, 4096, 11008) == 0 and B.qless_gated_ffn_workspace(64, 4096, 11008) >= 64 * 11008 * 4
    assert B.qless_gated_ffn_workspace(5, 512, 1376) == 0
    assert B.qless_gated_ffn_backward_workspace(4096, 2048, 5632, True) >= 4096 * 5632 * 2
