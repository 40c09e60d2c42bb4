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
