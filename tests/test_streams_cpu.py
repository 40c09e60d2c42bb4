"""Memory of calls on another stream than the current one, without a GPU: the library, the streams and the allocator are stood in for, and
what is looked at is on which stream's pool every output and workspace is allocated and which tensors are recorded as used where."""
import contextlib
import types

import pytest
import torch

from paper_2502_01703_b200 import binding as B

HERE, SIDE = types.SimpleNamespace(cuda_stream=0), types.SimpleNamespace(cuda_stream=77)


class FakeLibrary:
    """Every workspace query asks for 1000 bytes, every call succeeds."""
    def __getattr__(self, name):
        return (lambda *a: 1000) if name.endswith("_workspace") else (lambda *a: B.QLESS_OK)


@pytest.fixture
def world(monkeypatch):
    log = types.SimpleNamespace(current=HERE, made=[], recorded=[])

    @contextlib.contextmanager
    def use(stream):
        before, log.current = log.current, stream
        yield
        log.current = before

    def watch(make):
        def made(*a, **k):
            t = make(*a, **{**k, "device": "cpu"})
            log.made.append((t, log.current))
            return t
        return made

    monkeypatch.setattr(B, "lib", lambda: FakeLibrary())
    monkeypatch.setattr(B, "_stream", lambda stream=None, device=None: (log.current if stream is None else stream).cuda_stream)
    monkeypatch.setattr(B, "_on_gpu", lambda *a: None, raising=False)
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: log.current)
    monkeypatch.setattr(torch, "empty", watch(torch.empty))
    monkeypatch.setattr(torch, "empty_strided", watch(torch.empty_strided))
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log.recorded.append((t.data_ptr(), s)))
    return log


def _calls():
    bf, u8, i8 = torch.bfloat16, torch.uint8, torch.int8
    x, w, y = torch.zeros((4, 64), dtype=bf), torch.zeros((10, 64), dtype=bf), torch.zeros(4, dtype=torch.int64)
    codes, scales = torch.zeros((4, 64), dtype=i8), torch.zeros((4, 2), dtype=u8)
    a, b, dy = torch.zeros((8, 64), dtype=bf), torch.zeros((32, 8), dtype=bf), torch.zeros((4, 32), dtype=bf)
    g, f, rows = torch.zeros((3, 128)), torch.zeros((4, 512)), torch.zeros((1, 4, 512), dtype=bf)
    tc, vc, ts, vs = (torch.zeros(s, dtype=t) for s, t in (((1, 6, 512), u8), ((1, 5, 512), u8), ((1, 6), torch.float32), ((1, 5), torch.float32)))
    return [
        ("activation_quantize", [x], lambda s: B.qless_activation_quantize(x, stream=s)),
        ("activation_dequantize", [codes, scales], lambda s: B.qless_activation_dequantize(codes, scales, stream=s)),
        ("lora_gradients", [codes, scales, dy, a, b], lambda s: B.qless_lora_gradients(codes, scales, dy, a, b, [0, 4], stream=s)),
        ("lm_loss", [x, w, y], lambda s: B.qless_lm_loss(x, w, y, want_weight=True, stream=s)),
        ("project_quantize", [g], lambda s: B.qless_project_quantize(g, 512, 1, 8, stream=s, want_proj=True)),
        ("quantize", [f], lambda s: B.qless_quantize(f, 8, stream=s)),
        ("quantize_absmean", [f], lambda s: B.qless_quantize_absmean(f, 8, stream=s)),
        ("adam_gamma", [g], lambda s: B.qless_adam_gamma(g, stream=s)),
        ("score", [tc, vc, ts, vs], lambda s: B.qless_score(tc, vc, ts, vs, [1.0], [0, 5], 512, 8, stream=s)),
        ("score_16bit", [rows], lambda s: B.qless_score_16bit(rows, rows, [1.0], [0, 4], stream=s)),
        ("inv_norms_16bit", [rows], lambda s: B.qless_inv_norms_16bit(rows, stream=s)),
        ("score_dots", [tc, vc], lambda s: B.qless_score_dots(tc[0], vc[0], 512, 8, stream=s)),
        ("select_topk", [ts], lambda s: B.qless_select_topk(ts[0], 0.5, stream=s)),
    ]


@pytest.mark.parametrize("which", range(13))
def test_a_call_on_another_stream_takes_its_memory_from_that_streams_pool(which, world):
    name, inputs, call = _calls()[which]
    world.made.clear()
    out = call(SIDE)
    assert world.made and all(on is SIDE for _, on in world.made), name
    for t in inputs:
        assert (t.data_ptr(), SIDE) in world.recorded, name
    # what the caller gets is likely to be read on the stream that was current
    results = list(out.values()) if isinstance(out, dict) else list(out) if isinstance(out, (tuple, list)) else [out]
    for t in results:
        assert t is None or t.numel() == 0 or (t.data_ptr(), HERE) in world.recorded, name      # (no index is selected here)


@pytest.mark.parametrize("which", range(13))
def test_a_call_on_the_current_stream_records_nothing(which, world):
    _, _, call = _calls()[which]
    world.made.clear()
    call(None)
    call(HERE)
    assert world.made and all(on is HERE for _, on in world.made) and not world.recorded
