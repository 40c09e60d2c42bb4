"""Edges of the gradient-row calls: single rows of wider buffers, infinite logits, step bytes of groups that held no finite value,
gradients of the hidden states beside those of the weights, calls in a row on one stream and in a graph."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B
from test_lm_loss_gpu import _case, check, reference

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

def test_the_hidden_states_gradient_does_not_lose_the_labels_digits_beside_the_weights():
    # Row t's gradient is w sigma (sum_v q_v W_v - W_label): its length shows how the label's factor w sigma came through. Rounding the row's
    # 1024 entries to bf16 moves the length by a weighted mean of as many errors of at most 2^-8 each (spread over +-2^-8 their deviation is
    # 2^-8 / sqrt(3)), with weights as the squares of normal numbers: deviation 2^-8 / sqrt(3) * sqrt(3 / 1024) = 1.2e-4, six of them 7.4e-4; the
    # other probabilities' errors come in through 600 independent terms and are smaller still. A factor rounded to 8 bits would move single rows by up to 3.9e-3.
    T, width, vocab = 64, 1024, 600
    weight = _rand((vocab, width), 21, 0.05)
    labels = torch.arange(0, 9 * T, 9, device=DEV)
    gap = torch.linspace(2.0, 14.0, T, device=DEV)
    w = weight[labels].float()
    hidden = (w * (gap / w.square().sum(dim=1))[:, None]).to(torch.bfloat16)
    tw = torch.rand(T, device=DEV, generator=torch.Generator(device=DEV).manual_seed(22)) + 0.5
    for T_all in (T, 300):                      # both orientations of the products: up to 256 tokens, and more
        pad = T_all - T
        h = torch.cat([hidden, _rand((pad, width), 23)])
        y = torch.cat([labels, torch.full((pad,), 1, device=DEV)])
        f = torch.cat([tw, torch.ones(pad, device=DEV)])
        hd, wd = h.double(), weight.double()
        p = torch.softmax(hd @ wd.T, dim=1)
        at = torch.arange(T_all, device=DEV)
        p[at, y] = 0.0
        p[at, y] = -p.sum(dim=1)
        ref = (p * f.double()[:, None]) @ wd
        for want_weight in (False, True):
            got = B.qless_lm_loss(h, weight, y, f, want_weight=want_weight)["grad_hidden"].double()
            off = ((got * ref).sum(dim=1) / ref.square().sum(dim=1) - 1.0)[:T]
            assert off.abs().max() <= 1e-3, (T_all, want_weight, float(off.abs().max()))


@pytest.mark.parametrize("T", [6, 300])
@pytest.mark.parametrize("wants", [(False, False), (True, False), (True, True)])
def test_rows_whose_logits_are_infinite_have_no_loss(T, wants):
    # logsumexp(l) - l_label with the label's logit +infinity, or with every logit -infinity, is not a number
    width, vocab = 64, 500
    hidden, weight = _rand((T, width), 31), _rand((vocab, width), 32, 0.05)
    labels = torch.randint(0, vocab, (T,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(33))
    weight[:, 0], weight[:, 1] = -1.0, -1.0
    weight[7, 0] = 1.0
    hidden[:, :2] = 0.25
    clean = B.qless_lm_loss(hidden, weight, labels, want_hidden=wants[0], want_weight=wants[1])
    hidden[2, 0], labels[2] = float("inf"), 7
    hidden[4, 1] = float("inf")
    got = B.qless_lm_loss(hidden, weight, labels, want_hidden=wants[0], want_weight=wants[1])
    B.qless_check()
    rest = torch.ones(T, dtype=torch.bool, device=DEV)
    rest[2] = rest[4] = False
    assert torch.isnan(got["loss"][~rest]).all() and torch.equal(got["loss"][rest], clean["loss"][rest])
    if wants[0]:
        assert torch.isnan(got["grad_hidden"][~rest].float()).all() and torch.isfinite(got["grad_hidden"][rest].float()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_group_marked_as_not_finite_is_nan_whatever_its_codes(dtype):
    # byte 0xFF says NaN; codes other than the 0 that quantising leaves there must not make an infinity of it
    offsets, wi, wo, rank = [0, 40, 100], 256, 128, 16
    x, dy, a, b = _rand((100, wi), 41), _rand((100, wo), 42, 0.1), _rand((rank, wi), 43, 0.06), _rand((wo, rank), 44, 0.1)
    codes, scales = B.qless_activation_quantize(x)
    clean = B.qless_lora_gradients(codes, scales, dy, a, b, offsets, dtype=dtype)
    codes, scales = codes.clone(), scales.clone()
    codes[55, 32:64], scales[55, 1] = 3, 255
    assert torch.isnan(B.qless_activation_dequantize(codes, scales, dtype=dtype)[55, 32:64].float()).all()
    got = B.qless_lora_gradients(codes, scales, dy, a, b, offsets, dtype=dtype)
    B.qless_check()
    assert torch.equal(got[0], clean[0])
    da, db = got[1, :rank * wi].view(rank, wi).float(), got[1, rank * wi:].float()
    want = clean[1, :rank * wi].view(rank, wi).float()
    assert torch.isnan(da[:, 32:64]).all() and torch.isnan(db).all()
    assert torch.equal(da[:, :32], want[:, :32]) and torch.equal(da[:, 64:], want[:, 64:])


def test_the_calls_in_a_graph():
    # more examples than travel in the launch (tables go up first), one example longer than a piece; the graph reads what its inputs hold when it runs
    lengths = [int(v) for v in torch.randint(0, 9, (90,), generator=torch.Generator().manual_seed(51))] + [1100]
    offsets = [0]
    for v in lengths:
        offsets.append(offsets[-1] + v)
    T, width, vocab, rank = offsets[-1], 128, 2000, 8
    x, w, a, b = _rand((T, width), 52), _rand((vocab, width), 53, 0.05), _rand((rank, width), 54), _rand((width, rank), 55)
    labels = torch.randint(0, vocab, (T,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(56))

    def calls():
        c = B.qless_activation_quantize(x)
        loss = B.qless_lm_loss(x, w, labels, want_weight=True)
        few = B.qless_lm_loss(x[:50], w, labels[:50])
        g = B.qless_lora_gradients(*c, loss["grad_hidden"], a, b, offsets)
        g32 = B.qless_lora_gradients(*c, loss["grad_hidden"], a, b, offsets, dtype=torch.float32)
        back = B.qless_activation_dequantize(*c)
        return [c[0], c[1], loss["loss"], loss["grad_hidden"], loss["grad_weight"], few["loss"], few["grad_hidden"], g, g32, back]

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    for seed in (52, 57):
        x.copy_(_rand((T, width), seed))
        graph.replay()
        torch.cuda.synchronize()
        B.qless_check()
        for have, want in zip(got, calls()):
            assert torch.equal(have, want)


@pytest.mark.parametrize("wants", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("T,width,vocab", [(161, 136, 2500), (192, 264, 1024), (193, 264, 1025), (255, 72, 4099)])
def test_the_loss_around_the_change_of_orientation(T, width, vocab, wants):
    case = _case(T, width, vocab, 61, 0.9, pad=8)
    got = B.qless_lm_loss(*case, want_hidden=wants[0], want_weight=wants[1])
    B.qless_check()
    check(got, reference(*case), T, vocab)
