"""The calls in the order a user makes them: 8-bit checkpoint -> loss and its gradient -> per-example LoRA gradients -> datastore
codes (the `extract` stage of run_case), against 64-bit automatic differentiation of the same model.

Tolerance, on the 2-norm of an example's gradient: three roundings to bf16 lie between the exact gradient and the kernels' one (the
probabilities that enter the head's second product, the gradient at the layer's output, the gradient itself), each at most 2^-8
of what it rounds; sums are fp32. The reference takes the restored checkpoint as the layer's input where the kernels do."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B
from paper_2502_01703_b200.run_case import extract

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,tokens,width,vocab,rank", [(6, 300, 256, 1000, 8), (5, 700, 512, 5003, 16)])
def test_extract_against_automatic_differentiation(n, tokens, width, vocab, rank):
    got = extract(n, tokens, width, vocab, rank, d=256, bits=8)
    assert got["grads"].shape == (n, 2 * rank * width) and got["store"]["codes"].shape == (n, 256)
    x = B.qless_activation_dequantize(*got["checkpoint"], group=got["group"], dtype=torch.float32).double()
    head, hidden, labels = got["head"].double(), got["hidden"].double(), got["labels"]
    for e in range(n):
        lo, hi = int(got["offsets"][e]), int(got["offsets"][e + 1])
        a, b = got["a"].double().requires_grad_(), got["b"].double().requires_grad_()
        live = labels[lo:hi] >= 0
        # the adapter's output enters as hidden + (its value - its value): the loss is taken at the hidden states the kernels were given,
        # and its derivative reaches A and B
        ada = got["scaling"] * (x[lo:hi] @ a.T) @ b.T
        h = hidden[lo:hi] + ada - ada.detach()
        nll = torch.nn.functional.cross_entropy(h[live] @ head.T, labels[lo:hi][live], reduction="none")
        (nll * got["weight"][lo:hi][live].double()).sum().backward()
        want = torch.cat([a.grad.flatten(), b.grad.flatten()])
        have = got["grads"][e].double()
        assert (have - want).norm() <= 3 * 2.0 ** -8 * want.norm() + 1e-30, (e, float((have - want).norm() / want.norm()))
        assert torch.allclose(got["loss"]["loss"][lo:hi][live].double(), nll.detach(), rtol=1e-5, atol=1e-5)
    want_codes = B.qless_project_quantize(got["grads"], 256, 7, 8)
    assert torch.equal(got["store"]["codes"], want_codes["codes"])
