"""A whole decoder layer and the head (the `layer` stage of run_case): the gradient rows of every adapted projection against 64-bit automatic differentiation
of the same model.

Tolerance, on the 2-norm of an example's gradient of one projection: the activations and gradients that the calls hand on are bf16, each rounding at
most 2^-8 of what it rounds. On the longest way (to the query, key and value projections) a gradient passes some twelve of them: probabilities and gradient of the
head, three normalisations, grad_gate and grad_up with their product, the residual sums, the products in front of and behind attention, ds, the
gradient row; and the activations that the products meet carry up to ten of their own (normalisations, q k v, out, the residual stream, gate, up, hidden, out,
checkpoints' inputs). Independent of each other, 22 of them add up to sqrt(22) 2^-8 = 4.7 2^-8 of the gradient's length where each changes it by its own
size; the bound is twice that."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B
from paper_2502_01703_b200.run_case import layer

pytestmark = pytest.mark.gpu
BOUND = 2 * 22 ** 0.5 * 2.0 ** -8


def rms(t, w):
    return t / torch.sqrt(t.square().mean(dim=1, keepdim=True) + 1e-5) * w


@pytest.mark.parametrize("n,tokens,width,heads,kv,inner,vocab,rank", [(5, 300, 256, 4, 2, 688, 1000, 8), (7, 900, 512, 8, 2, 1376, 5003, 16)])
def test_layer_against_automatic_differentiation(n, tokens, width, heads, kv, inner, vocab, rank):
    got = layer(n, tokens, width, heads, kv, inner, vocab, rank, d=256, bits=8)
    head_dim, scaling = width // heads, got["scaling"]
    w = {k: t.double() for k, t in got["w"].items()}
    norms = [t.double() for t in got["norms"]]
    head, labels, x = got["head"].double(), got["labels"], got["x"].double().requires_grad_()
    total = got["grads"].shape[1]
    assert total == sum(s.stop - s.start for s in got["places"].values())
    dx = torch.zeros_like(x)
    for e in range(n):
        lo, hi = int(got["offsets"][e]), int(got["offsets"][e + 1])
        if lo == hi:
            assert not got["grads"][e].any()
            continue
        a = {k: t.double().requires_grad_() for k, t in got["a"].items()}
        b = {k: t.double().requires_grad_() for k, t in got["b"].items()}

        def project(t, name):                # the adapter's value is in the weights: it enters as its value minus its value, for its derivative
            ada = scaling * (t.detach() @ a[name].T) @ b[name].T
            return t @ w[name].T + ada - ada.detach()

        xe = x[lo:hi]
        qkv = project(rms(xe, norms[0]), "qkv")
        q, k, v = [t.unflatten(1, (-1, head_dim)).transpose(0, 1) for t in qkv.split([width, kv * head_dim, kv * head_dim], dim=1)]
        k, v = [t.repeat_interleave(heads // kv, dim=0) for t in (k, v)]
        s = (q @ k.transpose(1, 2)) * head_dim ** -0.5
        s = s.masked_fill(torch.ones(hi - lo, hi - lo, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        y = xe + project((torch.softmax(s, dim=2) @ v).transpose(0, 1).flatten(1), "o")
        m = rms(y, norms[1])
        z = y + project(torch.nn.functional.silu(project(m, "gate")) * project(m, "up"), "down")
        nll = torch.nn.functional.cross_entropy(rms(z, norms[2]) @ head.T, labels[lo:hi].clamp(min=0), reduction="none")
        ((nll * got["token_weight"][lo:hi].double())[labels[lo:hi] >= 0]).sum().backward()
        for name, at in got["places"].items():
            want = torch.cat([a[name].grad.flatten(), b[name].grad.flatten()])
            have = got["grads"][e, at].double()
            assert (have - want).norm() <= BOUND * want.norm() + 1e-30, (e, name, float((have - want).norm() / want.norm()))
    assert (got["grad_x"].double() - x.grad).norm() <= BOUND * x.grad.norm(), float((got["grad_x"].double() - x.grad).norm() / x.grad.norm())
    assert torch.equal(got["store"]["codes"], B.qless_project_quantize(got["grads"], 256, 7, 8)["codes"])
