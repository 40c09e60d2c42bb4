"""Refusals of the gradient-row calls, checked without a GPU: every bad argument returns its status before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2502_01703_b200 import binding as B

FAKE = C.c_void_p(4096)
ODD = C.c_void_p(4096 + 8)


@pytest.fixture(scope="module")
def L():
    from paper_2502_01703_b200 import build
    build.build()
    return B.lib()


def test_activation_refusals(L):
    def quant(x=FAKE, dtype=B.BF16, tokens=4, width=64, ld_x=64, group=32, codes=FAKE, ld_codes=64, scales=FAKE, ld_scales=2):
        return L.qless_activation_quantize(x, dtype, tokens, width, ld_x, group, codes, ld_codes, scales, ld_scales, None)

    def back(x=FAKE, dtype=B.BF16, tokens=4, width=64, ld_x=64, group=32, codes=FAKE, ld_codes=64, scales=FAKE, ld_scales=2):
        return L.qless_activation_dequantize(codes, ld_codes, scales, ld_scales, tokens, width, group, x, dtype, ld_x, None)

    for call in (quant, back):
        assert call(tokens=-1) == B.ERR_INVALID_ARG
        assert call(width=0) == B.ERR_INVALID_ARG
        assert call(dtype=5) == B.ERR_INVALID_ARG
        assert call(group=16) == B.ERR_UNSUPPORTED and b"group" in L.qless_last_error()
        assert call(ld_x=63) == B.ERR_INVALID_ARG
        assert call(ld_codes=63) == B.ERR_INVALID_ARG
        assert call(ld_scales=1) == B.ERR_INVALID_ARG
        assert call(width=(1 << 24) + 1, ld_x=1 << 25, ld_codes=1 << 25, ld_scales=1 << 20) == B.ERR_UNSUPPORTED
        assert call(x=None) == B.ERR_INVALID_ARG and call(codes=None) == B.ERR_INVALID_ARG and call(scales=None) == B.ERR_INVALID_ARG
        assert call(x=C.c_void_p(4097)) == B.ERR_INVALID_ARG
        assert call(tokens=0, x=None, codes=None, scales=None) == B.QLESS_OK


def test_lora_refusals(L):
    def lora(codes=FAKE, ld_codes=64, scales=FAKE, ld_scales=2, group=32, dy=FAKE, ld_dy=32, a=FAKE, b=FAKE, off=(0, 3, 4), tokens=4, n=2,
             wi=64, wo=32, rank=8, grads=FAKE, dtype=B.BF16, ld_grads=768, ws=None, wsb=0):
        o = (C.c_int64 * len(off))(*off) if off is not None else None
        return L.qless_lora_gradients(codes, ld_codes, scales, ld_scales, group, dy, ld_dy, a, b, o, tokens, n, wi, wo, rank, 1.0, grads, dtype,
                                      ld_grads, ws, wsb, None)

    assert lora() == B.ERR_WORKSPACE                                  # valid but for the workspace
    assert lora(ws=FAKE, wsb=64) == B.ERR_WORKSPACE and b"too small" in L.qless_last_error()
    assert lora(ws=ODD, wsb=1 << 30) == B.ERR_WORKSPACE
    assert lora(tokens=-1) == B.ERR_INVALID_ARG and lora(n=-1) == B.ERR_INVALID_ARG
    assert lora(wi=0) == B.ERR_INVALID_ARG and lora(rank=0) == B.ERR_INVALID_ARG and lora(dtype=3) == B.ERR_INVALID_ARG
    assert lora(wi=72, ld_codes=80, ld_scales=3) == B.ERR_UNSUPPORTED and lora(wo=40) == B.ERR_UNSUPPORTED
    assert lora(rank=12) == B.ERR_UNSUPPORTED and lora(rank=136) == B.ERR_UNSUPPORTED and b"rank" in L.qless_last_error()
    assert lora(group=48) == B.ERR_UNSUPPORTED
    assert lora(tokens=1 << 31) == B.ERR_UNSUPPORTED
    assert lora(off=(0, 3, 5)) == B.ERR_INVALID_ARG                   # beyond the tokens
    assert lora(off=(-1, 3, 4)) == B.ERR_INVALID_ARG
    assert lora(off=(0, 4, 3)) == B.ERR_INVALID_ARG and b"decrease" in L.qless_last_error()
    assert lora(off=None) == B.ERR_INVALID_ARG
    for name in ("codes", "scales", "dy", "a", "b", "grads"):
        assert lora(**{name: None}) == B.ERR_INVALID_ARG, name
    for name in ("codes", "dy", "a", "b", "grads"):
        assert lora(**{name: ODD}) == B.ERR_INVALID_ARG, name
    assert lora(ld_codes=72) == B.ERR_INVALID_ARG and lora(ld_codes=48) == B.ERR_INVALID_ARG
    assert lora(ld_dy=36) == B.ERR_INVALID_ARG and lora(ld_dy=24) == B.ERR_INVALID_ARG
    assert lora(ld_grads=760) == B.ERR_INVALID_ARG and lora(ld_grads=772) == B.ERR_INVALID_ARG
    assert lora(n=0, off=(0,), grads=None) == B.QLESS_OK              # no examples: nothing to write


def test_lm_loss_refusals(L):
    def loss(h=FAKE, ld_h=64, w=FAKE, ld_w=64, labels=FAKE, tw=None, tokens=5, width=64, vocab=100, out=FAKE, gh=FAKE, ld_gh=64, gw=FAKE, ld_gw=64,
             ws=None, wsb=0):
        return L.qless_lm_loss(h, ld_h, w, ld_w, labels, tw, tokens, width, vocab, out, gh, ld_gh, gw, ld_gw, ws, wsb, None)

    assert loss() == B.ERR_WORKSPACE
    assert loss(ws=FAKE, wsb=1024) == B.ERR_WORKSPACE and b"too small" in L.qless_last_error()
    assert loss(ws=ODD, wsb=1 << 40) == B.ERR_WORKSPACE
    assert loss(tokens=-1) == B.ERR_INVALID_ARG and loss(width=0) == B.ERR_INVALID_ARG and loss(vocab=0) == B.ERR_INVALID_ARG
    assert loss(width=60) == B.ERR_UNSUPPORTED and loss(width=65544, ld_h=65544, ld_w=65544) == B.ERR_UNSUPPORTED
    assert loss(tokens=(1 << 31) - 1) == B.ERR_UNSUPPORTED
    assert loss(vocab=(1 << 31) - 1) == B.ERR_UNSUPPORTED
    for name in ("h", "w", "labels", "out"):
        assert loss(**{name: None}) == B.ERR_INVALID_ARG, name
    for name in ("h", "w", "gh", "gw"):
        assert loss(**{name: ODD}) == B.ERR_INVALID_ARG, name
    for name in ("ld_h", "ld_w", "ld_gh", "ld_gw"):
        assert loss(**{name: 56}) == B.ERR_INVALID_ARG and loss(**{name: 68}) == B.ERR_INVALID_ARG, name
    assert loss(tokens=0, h=None, w=None, labels=None, out=None, gh=None, gw=None) == B.QLESS_OK


def test_workspace_queries_grow_with_what_is_asked_for():
    assert B.qless_lora_gradients_workspace(1000, 8, 512, 256, 16, torch.float32) > B.qless_lora_gradients_workspace(100, 8, 512, 256, 16) >= 256
    assert B.qless_lora_gradients_workspace(-1, 8, 512, 256, 16) == 256
    loss, grad = (B.qless_lm_loss_workspace(1000, 512, 32000, want_hidden=h) for h in (False, True))
    assert grad > loss and B.qless_lm_loss_workspace(1000, 512, 32000, want_hidden=False, want_weight=True) > loss
    # no room for the logits of all tokens: 65 536 tokens against 131 072 columns would be 16 GiB of bf16
    assert B.qless_lm_loss_workspace(65536, 1024, 131072) < (4 << 30)


def test_binding_checks_types_and_shapes():
    h, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((10, 64), dtype=torch.bfloat16)
    y = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError):
        B.qless_lm_loss(h.float(), w, y)
    with pytest.raises(TypeError):
        B.qless_lm_loss(h, w, y.int())
    with pytest.raises(ValueError):
        B.qless_lm_loss(h, w[:, :32], y)
    with pytest.raises(ValueError):
        B.qless_lm_loss(h, w, y, token_weight=torch.zeros(3))
    codes, scales = torch.zeros((4, 64), dtype=torch.int8), torch.zeros((4, 2), dtype=torch.uint8)
    dy, a, b = torch.zeros((4, 32), dtype=torch.bfloat16), torch.zeros((8, 64), dtype=torch.bfloat16), torch.zeros((32, 8), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        B.qless_lora_gradients(codes, scales, dy.float(), a, b, [0, 4])
    with pytest.raises(TypeError):
        B.qless_lora_gradients(codes, scales, dy, a, b, torch.tensor([0, 4], dtype=torch.int32))
    with pytest.raises(ValueError):
        B.qless_lora_gradients(codes, scales, dy[:3], a, b, [0, 4])
    with pytest.raises(ValueError):
        B.qless_lora_gradients(codes, scales, dy, a, b, [0, 4], grads=torch.zeros((2, 768), dtype=torch.bfloat16))
