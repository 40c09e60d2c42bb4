"""The feed-forward block with few tokens where tiles of the weights' features are shared by several blocks (partial sums, joined by a kernel of their own) and
where a block has several whole tiles. Which way a product goes shows in the number of launches."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B
from test_layer_gpu import check_ffn_backward, check_ffn_forward, gen

pytestmark = pytest.mark.gpu

# (width, inner) and, for 148 SMs, which products are shared: gate and up, down; backward: dh (beyond 8 tokens), dx
SIZES = {
    (2600, 264): (True, False, True, False),        # few tiles and a long contraction: a block has a piece of one tile
    (264, 5000): (False, True, True, True),
    (3000, 5000): (True, True, True, True),         # pieces that reach over a tile's end
    (256, 19200): (False, True, True, True),        # gate and up: two whole tiles to a block
    (8, 19208): (False, True, True, True),
}


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [1, 5, 9, 33, 61, 130, 256])
@pytest.mark.parametrize("W,F", list(SIZES))
def test_shared_tiles(W, F, T, act):
    g = gen(T + W + F)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, dy = rand(T, W).to(torch.bfloat16), rand(T, W).to(torch.bfloat16)
    wg, wu, wd = [(rand(*s) * 1.3 * s[1] ** -0.5).to(torch.bfloat16) for s in ((F, W), (F, W), (W, F))]
    counts = [B.qless_kernel_launches()]
    got = B.qless_gated_ffn(x, wg, wu, wd, activation=act, want_saved=True)
    counts.append(B.qless_kernel_launches())
    back = B.qless_gated_ffn_backward(dy, None, got["gate"], got["up"], wg, wu, wd, activation=act)
    counts.append(B.qless_kernel_launches())
    if torch.cuda.get_device_properties(0).multi_processor_count == 148:
        glu, down, dh, dx = SIZES[W, F]
        assert counts[1] - counts[0] == 2 + glu + down and counts[2] - counts[1] == 2 + (dh and T > 8) + dx
    # (the roundings of test_gated_ffn: no sum of a block has more than 2^10 additions here, the longest contractions being dealt out in pieces of a few stages)
    check_ffn_forward(got, x, wg, wu, wd, act)
    check_ffn_backward(back, dy, None, got["gate"], got["up"], wg, wu, wd, act)
    again = B.qless_gated_ffn(x, wg, wu, wd, activation=act)
    assert torch.equal(again["out"], got["out"]) and torch.equal(again["hidden"], got["hidden"])
    full = B.qless_gated_ffn_backward(dy, x, got["gate"], got["up"], wg, wu, wd, activation=act, want_weight=True)
    check_ffn_backward(full, dy, x, got["gate"], got["up"], wg, wu, wd, act)
    assert all(torch.equal(full[n], back[n]) for n in ("grad_x", "grad_gate", "grad_up"))
    B.qless_check()


def one_pass(s, **kw):
    got = B.qless_gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], want_saved=True, **kw)
    back = B.qless_gated_ffn_backward(s["dy"], s["x"], got["gate"], got["up"], s["wg"], s["wu"], s["wd"], want_weight=True, **kw)
    return [*got.values(), *back.values()]


def inputs(seed, T, W, F):
    g = gen(seed)
    rand = lambda *s: (torch.randn(s, generator=g, device="cuda") / 4).to(torch.bfloat16)  # noqa: E731
    return dict(x=rand(T, W), dy=rand(T, W), wg=rand(F, W), wu=rand(F, W), wd=rand(W, F))


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("T,W,F", [(5, 264, 5000), (61, 3000, 5000), (130, 2600, 264), (200, 256, 1000)])
def test_in_a_long_row_on_streams_and_in_graphs(T, W, F):
    s = [inputs(T + i, T, W, F) for i in range(2)]
    want = [[t.clone() for t in one_pass(x)] for x in s]
    for _ in range(200):
        last = one_pass(s[0])
    assert same(last, want[0])
    graphs, outs, pool = [], [], None
    for x in s:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            outs.append(one_pass(x))
        pool = pool or graph.pool()
        graphs.append(graph)
    for _ in range(3):
        for graph, out, w in zip(graphs, outs, want):        # one behind the other: they share workspaces
            graph.replay()
            torch.cuda.synchronize()
            assert same(out, w)
    for k, t in inputs(T + 1, T, W, F).items():
        s[0][k].copy_(t)
    graphs[0].replay()                                       # new contents at the captured addresses
    torch.cuda.synchronize()
    assert same(outs[0], want[1])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    got = [one_pass(s[1], stream=st) for _ in range(5) for st in streams]
    torch.cuda.synchronize()
    assert all(same(x, want[1]) for x in got)
    B.qless_check()
