"""What the bits of attention depend on: the list of the examples' lengths (with the head counts and the GPU), which decides how tiles are dealt out, and
an example's own rows; not where the examples lie, nor what the other examples hold."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B
from test_layer_gpu import attention_exact, attention_inputs, close

pytestmark = pytest.mark.gpu

NAMES = ("out", "lse", "grad_q", "grad_k", "grad_v")


def both_ways(q, k, v, dout, off):
    got = B.qless_attention(q, k, v, off)
    return {**got, **B.qless_attention_backward(dout, q, k, v, got["out"], got["lse"], off)}


# many short examples; few long ones, whose loops are dealt out (forward and backward, backward alone)
@pytest.mark.parametrize("lens,H,K,D", [([171, 40, 0, 300], 8, 2, 64), ([2900, 150], 2, 1, 128), ([700, 5, 90], 32, 1, 64)])
def test_the_same_list_of_lengths_gives_the_same_bits(lens, H, K, D):
    T = sum(lens)
    off = torch.tensor([0] + lens).cumsum(0)
    q, k, v, dout = attention_inputs(T, H, K, D, seed=T)
    first = both_ways(q, k, v, dout, off)
    # elsewhere, between rows of nobody
    before, after = 77, 4321
    place = lambda t: torch.cat([torch.ones_like(t[:1]).expand(before, -1, -1), t, torch.ones_like(t[:1]).expand(after, -1, -1)])  # noqa: E731
    there = both_ways(*(place(t) for t in (q, k, v, dout)), off + before)
    assert all(torch.equal(there[n][before:before + T], first[n]) for n in NAMES)
    # beside other contents of the other examples
    lo, hi = int(off[0]), int(off[1])
    others = [t.flip(0) for t in (q, k, v, dout)]
    for t, mine in zip(others, (q, k, v, dout)):
        t[lo:hi] = mine[lo:hi]
    beside = both_ways(*others, off)
    assert all(torch.equal(beside[n][lo:hi], first[n][lo:hi]) for n in NAMES)
    B.qless_check()


@pytest.mark.parametrize("H,K,D", [(2, 1, 128), (32, 1, 64)])
def test_beside_other_examples_the_results_are_as_exact(H, K, D):
    """With more examples in the call the first one's loop may be dealt out otherwise or not at all: its bits may change, its bounds do not."""
    T = 1500
    q, k, v, dout = attention_inputs(4 * T, H, K, D, seed=H)
    for off in ([0, T], [0, T, 2 * T], [0, T, 2 * T, 3 * T, 4 * T]):
        n = off[-1]
        got = both_ways(q[:n], k[:n], v[:n], dout[:n], off)
        want, room = attention_exact(q[:n], k[:n], v[:n], off, D ** -0.5, dout[:n], got["out"])
        for name in ("lse", "out", "grad_v", "grad_q", "grad_k"):
            close(got[name], want[name], room[name])
    B.qless_check()
