"""Calls on another stream with nothing but `stream=`: outputs and workspaces of the binding's own, inputs dropped at once, and the
current stream allocating and overwriting memory while the kernels still wait for their turn."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _rand(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


def _churn(sizes):
    """Takes and overwrites blocks of these sizes on the current stream."""
    for _ in range(3):
        keep = [torch.full((max(s, 1),), 0x5A, dtype=torch.uint8, device=DEV) for s in sizes]
        del keep


def _busy(stream):
    """Some milliseconds of work in front of the call, behind all that the current stream has been given."""
    a = _rand((8192, 8192), 99)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(6):
            a = a @ a
    a.record_stream(stream)


@pytest.mark.parametrize("wants", [(True, False), (True, True), (False, True)])
def test_lm_loss_with_a_stream_alone(wants):
    T, width, vocab = 300, 256, 5000
    hidden, weight = _rand((T, width), 1), _rand((vocab, width), 2, 0.05)
    labels = torch.randint(0, vocab, (T,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
    want = B.qless_lm_loss(hidden, weight, labels, want_hidden=wants[0], want_weight=wants[1])
    size = B.qless_lm_loss_workspace(T, width, vocab, *wants)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    mine = [hidden.clone(), weight.clone(), labels.clone()]
    _busy(st)
    got = B.qless_lm_loss(*mine, want_hidden=wants[0], want_weight=wants[1], stream=st)
    del mine
    _churn([size, hidden.nbytes, weight.nbytes, labels.nbytes, T * 4])
    st.synchronize()
    B.qless_check()
    for k, v in want.items():
        assert v is None or torch.equal(got[k], v), k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_checkpoint_and_lora_gradients_with_a_stream_alone(dtype):
    T, wi, wo, rank, offsets = 2000, 256, 512, 16, [0, 700, 703, 2000]
    x, dy, a, b = _rand((T, wi), 4), _rand((T, wo), 5, 0.1), _rand((rank, wi), 6, 0.06), _rand((wo, rank), 7, 0.1)
    codes, scales = B.qless_activation_quantize(x)
    want = B.qless_lora_gradients(codes, scales, dy, a, b, offsets, dtype=dtype)
    back = B.qless_activation_dequantize(codes, scales, dtype=dtype)
    size = B.qless_lora_gradients_workspace(T, 3, wi, wo, rank, dtype)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    x2, dy2, a2, b2 = x.clone(), dy.clone(), a.clone(), b.clone()
    _busy(st)
    c2, s2 = B.qless_activation_quantize(x2, stream=st)
    values = B.qless_activation_dequantize(c2, s2, dtype=dtype, stream=st)
    got = B.qless_lora_gradients(c2, s2, dy2, a2, b2, offsets, dtype=dtype, stream=st)
    del x2, dy2, a2, b2
    _churn([size, x.nbytes, dy.nbytes, a.nbytes, b.nbytes, codes.nbytes, scales.nbytes, want.nbytes])
    st.synchronize()
    B.qless_check()
    assert torch.equal(c2, codes) and torch.equal(s2, scales) and torch.equal(values, back) and torch.equal(got, want)


def test_projection_and_selection_with_a_stream_alone():
    g = _rand((64, 4096), 8)
    want = B.qless_project_quantize(g, 512, 7, 8)
    scores = torch.randn(200_000, device=DEV, generator=torch.Generator(device=DEV).manual_seed(9))
    top = B.qless_select_topk(scores, 0.05)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    g2, scores2 = g.clone(), scores.clone()
    _busy(st)
    got = B.qless_project_quantize(g2, 512, 7, 8, stream=st)
    chosen = B.qless_select_topk(scores2, 0.05, stream=st)
    del g2, scores2
    _churn([B.qless_project_quantize_workspace(64, 4096, 512, 8), B.qless_select_topk_workspace(200_000), g.nbytes, scores.nbytes, top.nbytes])
    st.synchronize()
    B.qless_check()
    for k, v in want.items():
        assert v is None or torch.equal(got[k], v), k
    assert torch.equal(chosen, top)
