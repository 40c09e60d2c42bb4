"""What the binding itself decides for the gradient-row calls, with nothing launched: refusals that no status of the library stands
behind, the stride it passes, the stream it finds."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B


def _loss_inputs(T=4, width=64, vocab=10):
    return torch.zeros((T, width), dtype=torch.bfloat16), torch.zeros((vocab, width), dtype=torch.bfloat16), torch.zeros(T, dtype=torch.int64)


def test_a_strided_loss_is_refused():
    # the kernels write it as consecutive numbers
    with pytest.raises(ValueError, match="contiguous"):
        B.qless_lm_loss(*_loss_inputs(), out=dict(loss=torch.zeros(8)[::2]))


def test_tensors_in_host_memory_are_refused():
    # the kernels would read them through their host addresses
    bf = torch.bfloat16
    with pytest.raises(ValueError, match="GPU"):
        B.qless_lm_loss(*_loss_inputs())
    with pytest.raises(ValueError, match="GPU"):
        B.qless_activation_quantize(torch.zeros((4, 64)))
    codes, scales = torch.zeros((4, 64), dtype=torch.int8), torch.zeros((4, 2), dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        B.qless_activation_dequantize(codes, scales)
    with pytest.raises(ValueError, match="GPU"):
        B.qless_lora_gradients(codes, scales, torch.zeros((4, 32), dtype=bf), torch.zeros((8, 64), dtype=bf), torch.zeros((32, 8), dtype=bf), [0, 4])


class OnGpu:
    """Stands in for a tensor on GPU `index` (-1: in host memory)."""
    def __init__(self, index):
        self.index = index

    def get_device(self):
        return self.index


def test_one_tensor_elsewhere_is_enough(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    B._on_gpu(None, OnGpu(0), None, OnGpu(0))
    for others in ((OnGpu(0), OnGpu(-1)), (OnGpu(0), None, OnGpu(1)), (OnGpu(-1), OnGpu(0)), (OnGpu(1), OnGpu(1))):
        with pytest.raises(ValueError, match="GPU"):
            B._on_gpu(None, *others)
    stream = type("Stream", (), dict(device_index=1))()
    B._on_gpu(stream, OnGpu(1), OnGpu(1))
    with pytest.raises(ValueError, match="GPU"):
        B._on_gpu(stream, OnGpu(0), OnGpu(0))


@pytest.mark.parametrize("width,pad", [(72, 3), (64, 0), (8, 1), (4096, 5)])
def test_a_single_row_is_taken_whatever_its_stride_says(width, pad):
    # a row cut out of a wider buffer is contiguous to torch; its stride of width + 3 would be refused for rows that have neighbours
    one = torch.zeros((2, width + pad), dtype=torch.bfloat16)[:1, :width]
    assert one.is_contiguous()
    assert B._row_stride(one) >= width and B._row_stride(one) % 16 == 0
    two = torch.zeros((2, width + pad), dtype=torch.bfloat16)[:, :width]
    assert B._row_stride(two) == width + pad


def test_the_current_stream_is_found_without_the_private_call(monkeypatch):
    monkeypatch.setattr(B, "_raw_current", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: type("Stream", (), dict(cuda_stream=5))())
    assert B._stream() == 5
    monkeypatch.setattr(B, "_raw_current", lambda device: 7 + device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert B._stream() == 7
