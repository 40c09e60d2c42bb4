"""Edges of the gradient-row calls: single rows of wider buffers, infinite logits, step bytes of groups that held no finite value,
gradients of the hidden states beside those of the weights, calls in a row on one stream and in a graph."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _rand(shape, seed, scale=1.0, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def test_single_rows_of_wider_buffers():
    width, vocab, rank = 144, 900, 8
    wide = _rand((2, width + 5), 1)
    one, copy = wide[:1, :width], wide[:1, :width].clone()
    weight, labels = _rand((vocab, width), 2, 0.1), torch.tensor([17], device=DEV)
    for a, b in zip(B.qless_lm_loss(one, weight, labels, want_weight=True).values(), B.qless_lm_loss(copy, weight, labels, want_weight=True).values()):
        assert torch.equal(a, b)
    codes, scales = B.qless_activation_quantize(one)
    want_codes, want_scales = B.qless_activation_quantize(copy)
    assert torch.equal(codes, want_codes) and torch.equal(scales, want_scales)
    c2, s2 = torch.zeros((2, width + 3), dtype=torch.int8, device=DEV), torch.zeros((2, 9), dtype=torch.uint8, device=DEV)
    c2[0, :width], s2[0, :5] = codes[0], scales[0]
    dy, a, b = _rand((1, 64), 3), _rand((rank, width), 4), _rand((64, rank), 5)
    got = B.qless_lora_gradients(c2[:1, :width], s2[:1, :5], dy, a, b, [0, 1])
    assert torch.equal(got, B.qless_lora_gradients(codes, scales, dy, a, b, [0, 1]))


def test_calls_in_a_row_without_a_wait_between_them():
    # the loss with the weights' gradient alone ends in a kernel on CTA pairs; the checkpoint and LoRA kernels behind it are launched ahead
    T, width, vocab, rank = 40, 256, 3000, 8
    hidden, weight = _rand((T, width), 11), _rand((vocab, width), 12, 0.05)
    labels = torch.randint(0, vocab, (T,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(13))
    dy, a, b = _rand((T, 128), 14), _rand((rank, width), 15), _rand((128, rank), 16)

    def calls():
        w = B.qless_lm_loss(hidden, weight, labels, want_hidden=False, want_weight=True)
        c = B.qless_activation_quantize(hidden)
        g = B.qless_lora_gradients(*c, dy, a, b, [0, 13, 40])
        h = B.qless_lm_loss(hidden, weight, labels)
        return w["loss"], w["grad_weight"], c[0], c[1], g, h["loss"], h["grad_hidden"]

    want = calls()
    torch.cuda.synchronize()
    for _ in range(150):
        got = calls()
    torch.cuda.synchronize()
    B.qless_check()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
