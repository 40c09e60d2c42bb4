"""Edges of normalisation, packed attention and the feed-forward block: rows that belong to nobody, infinities and NaN beside other examples, maxima that keep growing,
nothing to do, matrices beyond 2^31 elements, calls in a row, on other streams and in captured graphs."""
import math

import pytest
import torch

from paper_2502_01703_b200 import binding as B
from test_layer_gpu import act64, attention_exact, attention_inputs, check_ffn_backward, check_ffn_forward, close, gen

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def run_attention(q, k, v, dout, off, **kw):
    got = B.qless_attention(q, k, v, off, **kw)
    return {**got, **B.qless_attention_backward(dout, q, k, v, got["out"], got["lse"], off, **kw)}


# ---- attention ---------------------------------------------------------------------------------------------------------

def test_rows_outside_the_examples():
    T, H, K, D = 700, 8, 2, 64
    off = torch.tensor([37, 37, 180, 431], dtype=torch.int64)
    q, k, v, dout = attention_inputs(T, H, K, D, 1)
    inside = torch.zeros(T, dtype=torch.bool, device="cuda")
    inside[37:431] = True
    fresh = run_attention(q, k, v, dout, off)
    for name in ("out", "lse", "grad_q", "grad_k", "grad_v"):
        assert not fresh[name][~inside].any() and fresh[name][inside].any(), name
    given = {n: torch.full_like(t, 7.0) for n, t in fresh.items()}
    out = B.qless_attention(q, k, v, off, out=given["out"])["out"]
    assert out.data_ptr() == given["out"].data_ptr()
    B.qless_attention_backward(dout, q, k, v, out, fresh["lse"], off, grads={n: given[n] for n in ("grad_q", "grad_k", "grad_v")})
    for name in ("out", "grad_q", "grad_k", "grad_v"):
        assert (given[name][~inside] == 7.0).all() and torch.equal(given[name][inside], fresh[name][inside]), name


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("H,K,D", [(8, 2, 128), (3, 3, 40)])
def test_what_one_example_holds_reaches_no_other(bad, H, K, D):
    off, T = [5, 150, 290, 291, 500], 520
    q, k, v, dout = attention_inputs(T, H, K, D, 2)
    clean = run_attention(q, k, v, dout, off)
    spoiled = [t.clone() for t in (q, k, v, dout)]
    for t in spoiled:
        t[:5], t[150:290], t[500:] = bad, bad, bad           # an example in the middle, and the rows of nobody
    out, lse = clean["out"].clone(), clean["lse"].clone()
    got = run_attention(*spoiled, off)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[150:290] = False
    for name in ("out", "lse", "grad_q", "grad_k", "grad_v"):
        assert torch.equal(got[name][keep], clean[name][keep]), name
        assert not torch.isfinite(got[name][150:290].float()).any() or name == "lse", name
    # only the backward pass's own inputs spoiled
    out[150:290], lse[150:290] = bad, bad
    back = B.qless_attention_backward(spoiled[3], q, k, v, out, lse, off)
    for name in ("grad_q", "grad_k", "grad_v"):
        assert torch.equal(back[name][keep], clean[name][keep]), name
    B.qless_check()


def test_a_nan_reaches_every_row_that_sees_it():
    T, H, K, D = 400, 4, 2, 64
    for tensor, at in (("k", 130), ("v", 257), ("q", 301)):
        q, k, v, _ = attention_inputs(T, H, K, D, 3)
        dict(q=q, k=k, v=v)[tensor][at] = float("nan")
        out = B.qless_attention(q, k, v, [0, T])["out"].float()
        seen = out[at:at + 1] if tensor == "q" else out[at:]
        assert torch.isnan(seen).all()
        before = out[:at // 128 * 128] if tensor != "q" else torch.cat([out[:at], out[at + 1:]])
        assert torch.isfinite(before).all()


@pytest.mark.parametrize("H,K,D,T", [(4, 1, 128, 1500), (2, 2, 64, 1100)])
def test_maxima_that_keep_growing(H, K, D, T):
    # keys that point along the queries more and more: every tile of keys raises the maximum by some 40 powers of two; and the other way round
    g = gen(4)
    line = torch.nn.functional.normalize(torch.randn(D, generator=g, device="cuda"), dim=0)
    q = (line * 8 + 0.05 * torch.randn((T, H, D), generator=g, device="cuda")).to(torch.bfloat16)
    steps = torch.arange(T, device="cuda", dtype=torch.float32)[:, None, None] / 128 * 28 * D ** 0.5 / 8
    v = torch.randn((T, K, D), generator=g, device="cuda").to(torch.bfloat16)
    dout = torch.randn((T, H, D), generator=g, device="cuda").to(torch.bfloat16)
    for sign in (1.0, -1.0):
        k = (line * steps * sign + torch.randn((T, K, D), generator=g, device="cuda")).to(torch.bfloat16)
        got = run_attention(q, k, v, dout, [0, T])
        want, room = attention_exact(q, k, v, [0, T], D ** -0.5, dout, got["out"])
        # scores of some hundreds: fp32 holds their exponents to 2^-23 of the score's size, which counts for every probability
        wide = 1.0 + 2.0 ** -23 * 1000 * 2 / 2.0 ** -13
        # a probability below fp32's and bf16's smallest normal number, 2^-126, may come out as 0: that moves each of the up to T H terms of a sum by
        # 2^-126 times what it meets (ds: dp - delta, at most 2 D |dout| |v|, times q or k)
        top = lambda t: float(t.abs().max())  # noqa: E731
        lost = T * H * 2.0 ** -126 * max(top(dout), top(v), 2 * D * top(dout) * top(v) * max(top(q), top(k)))
        for name in ("out", "grad_v", "grad_q", "grad_k"):
            close(got[name], want[name], room[name] * wide + lost)
        close(got["lse"], want["lse"], room["lse"])


def test_scale_and_single_tokens():
    T, H, K, D = 260, 6, 2, 96
    q, k, v, dout = attention_inputs(T, H, K, D, 5)
    off = [0, 1, 2, 130, 131, 260]
    for scale in (1e-4, 0.5):
        got = run_attention(q, k, v, dout, off, scale=scale)
        want, room = attention_exact(q, k, v, off, scale, dout, got["out"])
        for name in ("out", "lse", "grad_v", "grad_q", "grad_k"):
            close(got[name], want[name], room[name])
    assert torch.equal(got["out"][0], v[0].repeat_interleave(H // K, dim=0))         # a token alone sees its own value


def test_nothing_to_do():
    q, k = [torch.zeros((0, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2)]
    assert B.qless_attention(q, k, k, [0])["out"].shape == (0, 4, 64) and B.qless_attention(q, k, k, [0, 0, 0])["lse"].shape == (0, 4)
    q, k, v, dout = attention_inputs(50, 4, 2, 64, 6)
    for off in ([0], [10, 10, 10]):
        got = run_attention(q, k, v, dout, off)
        assert all(not t.any() for t in got.values())
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda")
    got = B.qless_layer_norm(x, w)
    back = B.qless_layer_norm_backward(x, x, w, got["mean"], got["rstd"], want_weight=True, want_bias=True)
    assert got["out"].shape == (0, 64) and not back["grad_weight"].any() and not back["grad_bias"].any()
    w1, w2 = torch.ones((128, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((64, 128), dtype=torch.bfloat16, device="cuda")
    got = B.qless_gated_ffn(x, w1, w1, w2, want_saved=True)
    back = B.qless_gated_ffn_backward(x, x, got["gate"], got["up"], w1, w1, w2, want_weight=True)
    assert got["out"].shape == (0, 64) and not back["grad_w_gate"].any() and not back["grad_w_down"].any() and back["grad_gate"].shape == (0, 128)
    B.qless_check()


def test_beyond_32_bits():
    T, H, K, D = 270_000, 64, 1, 128                         # q, out, and the gradients: more than 2^31 elements each
    q = torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda")
    assert q.numel() > 1 << 31
    kv, dout = torch.zeros((T, 2, D), dtype=torch.bfloat16, device="cuda"), torch.zeros_like(q)
    small = attention_inputs(300, H, K, D, 7)
    q[-300:], kv[-300:, :1], kv[-300:, 1:], dout[-300:] = small
    got = run_attention(q, kv[:, :1], kv[:, 1:], dout, [T - 300, T - 100, T])
    here = run_attention(*small, [0, 200, 300])
    for name in ("out", "lse", "grad_q", "grad_k", "grad_v"):
        assert torch.equal(got[name][-300:], here[name]) and not got[name][:-300].any(), name
    del q, kv, dout, got
    T, W, F = 200_000, 64, 11008
    g = gen(8)
    wg, wu, wd = [(torch.randn(s, generator=g, device="cuda") / 8).to(torch.bfloat16) for s in ((F, W), (F, W), (W, F))]
    x = torch.zeros((T, W), dtype=torch.bfloat16, device="cuda")
    x[-512:] = torch.randn((512, W), generator=g, device="cuda").to(torch.bfloat16)
    dy = torch.zeros_like(x)
    dy[-512:] = torch.randn((512, W), generator=g, device="cuda").to(torch.bfloat16)
    big = B.qless_gated_ffn(x, wg, wu, wd, want_saved=True)
    last = {n: t[-512:] for n, t in big.items()}
    assert big["hidden"].numel() > 1 << 31 and not big["out"][:-512].any()
    check_ffn_forward(last, x[-512:], wg, wu, wd, "silu")
    back = B.qless_gated_ffn_backward(dy, None, big["gate"], big["up"], wg, wu, wd)
    check_ffn_backward({n: t[-512:] if t is not None else None for n, t in back.items()}, dy[-512:], None, last["gate"], last["up"], wg, wu, wd, "silu")
    del dy, last
    del big, back, x
    x = torch.zeros((140_000, 16384), dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn((3, 16384), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.ones(16384, device="cuda")
    got, here = B.qless_layer_norm(x, w), B.qless_layer_norm(x[-3:], w)
    assert x.numel() > 1 << 31 and torch.equal(got["out"][-3:], here["out"]) and not got["out"][:-3].any()
    back = B.qless_layer_norm_backward(x, x, w, got["mean"], got["rstd"], want_weight=True)
    want = B.qless_layer_norm_backward(x[-3:], x[-3:], w, here["mean"], here["rstd"], want_weight=True)
    assert torch.equal(back["grad_x"][-3:], want["grad_x"]) and torch.allclose(back["grad_weight"], want["grad_weight"], rtol=1e-5, atol=1e-6)
    B.qless_check()


# ---- feed-forward block ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [40, 300])
def test_activations_over_their_whole_range(act, T):
    # the gate's weights pick single inputs, so that it takes given values; the other projections are plain
    W, F = 64, 64
    eye = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    values = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3, 0.5, -0.5, 1.0, -1.0, 3.0, -3.0, 6.0, -6.0, 10.0, -10.0, 20.0, -20.0, 60.0, -60.0, 88.0, -88.0, 100.0, -100.0,
                           1e4, -1e4, 1e30, -1e30], device="cuda")
    x = values[torch.randint(0, len(values), (T, W), generator=gen(9), device="cuda")].to(torch.bfloat16)
    up = torch.full((F, W), 0.0, dtype=torch.bfloat16, device="cuda")
    ones = torch.ones((T, F), dtype=torch.bfloat16, device="cuda")
    got = B.qless_gated_ffn(x, eye, up, eye, activation=act, want_saved=True)
    assert torch.equal(got["gate"], x) and not got["up"].any() and not got["out"].any()
    dy = torch.randn((T, W), generator=gen(10), device="cuda").to(torch.bfloat16)
    back = B.qless_gated_ffn_backward(dy, None, got["gate"], ones, eye, up, eye, activation=act)
    a, da = act64(act, x.double())
    close(back["grad_gate"], dy.double() * da, (HALF + 2.0 ** -16) * (dy.double() * da).abs() + 1e-30 + 2.0 ** -20 * dy.double().abs())
    close(back["grad_up"], dy.double() * a, (HALF + 2.0 ** -16) * (dy.double() * a).abs() + 2.0 ** -20 * dy.double().abs())


@pytest.mark.parametrize("T", [50, 300])
def test_an_infinite_token_reaches_its_own_row_only(T):
    W, F = 128, 264
    g = gen(11)
    wg, wu, wd = [(torch.randn(s, generator=g, device="cuda") / 8).to(torch.bfloat16) for s in ((F, W), (F, W), (W, F))]
    x, dy = [torch.randn((T, W), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    clean = B.qless_gated_ffn(x, wg, wu, wd, want_saved=True)
    back = B.qless_gated_ffn_backward(dy, None, clean["gate"], clean["up"], wg, wu, wd)
    rows = torch.arange(T, device="cuda") != T // 2
    for bad in (float("inf"), float("nan")):
        x2, dy2 = x.clone(), dy.clone()
        x2[T // 2, 3], dy2[T // 2, 5] = bad, bad
        got = B.qless_gated_ffn(x2, wg, wu, wd, want_saved=True)
        assert all(torch.equal(got[n][rows], clean[n][rows]) for n in clean) and not torch.isfinite(got["out"][T // 2].float()).any()
        got = B.qless_gated_ffn_backward(dy2, None, clean["gate"], clean["up"], wg, wu, wd)
        assert all(torch.equal(got[n][rows], back[n][rows]) for n in ("grad_x", "grad_gate", "grad_up"))


def test_each_weights_gradient_alone():
    T, W, F = 300, 136, 264
    g = gen(12)
    wg, wu, wd = [(torch.randn(s, generator=g, device="cuda") / 8).to(torch.bfloat16) for s in ((F, W), (F, W), (W, F))]
    x, dy = [torch.randn((T, W), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    saved = B.qless_gated_ffn(x, wg, wu, wd, want_saved=True)
    full = B.qless_gated_ffn_backward(dy, x, saved["gate"], saved["up"], wg, wu, wd, want_weight=True)
    for name in ("grad_w_gate", "grad_w_up", "grad_w_down"):
        mine = torch.full_like(full[name], 3.0)
        got = B.qless_gated_ffn_backward(dy, x if name != "grad_w_down" else None, saved["gate"], saved["up"], wg, wu, wd, want_x=False, grads={name: mine})
        assert torch.equal(mine, full[name]) and got["grad_x"] is None and torch.equal(got["grad_up"], full["grad_up"])
        assert all(got[o] is None for o in ("grad_w_gate", "grad_w_up", "grad_w_down") if o != name)


# ---- normalisation -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,W", [(torch.float32, 1000), (torch.bfloat16, 4112), (torch.float32, 333)])
def test_a_mean_far_from_zero_and_rows_without_spread(dtype, W):
    g = gen(13)
    base = torch.randn((6, W), generator=g, device="cuda", dtype=torch.float64)
    x = (base + 1000.0).to(dtype)
    x[4] = 5.0                                               # no spread at all: eps decides
    x[5] = 0.0
    w = torch.ones(W, device="cuda", dtype=dtype)
    got = B.qless_layer_norm(x, w, eps=1e-5)
    X = x.double()
    d = X - X.mean(dim=1, keepdim=True)
    r = 1 / torch.sqrt(d.square().mean(dim=1, keepdim=True) + 1e-5)
    # the mean of numbers near 1000 is off by at most 2^-23 of it for every of the ten or so additions in a row
    room = 12 * 2.0 ** -23 * 1000 * r + 2.0 ** -18 * (d * r).abs() + (HALF if dtype == torch.bfloat16 else 0.0) * (d * r).abs()
    close(got["out"][:4], (d * r)[:4], room[:4])
    assert not got["out"][4:].any() and torch.allclose(got["rstd"][4:].double(), r[4:, 0], rtol=1e-6)
    for bad in (float("nan"), float("inf")):
        x[2, W // 2] = bad
        again = B.qless_layer_norm(x, w, eps=1e-5)
        keep = torch.tensor([0, 1, 3, 4, 5], device="cuda")
        assert torch.equal(again["out"][keep], got["out"][keep]) and torch.isnan(again["out"][2].float()).any()


# ---- calls in a row, streams, graphs -------------------------------------------------------------------------------------

def everything(seed, T=333, scale=1.0):
    """One pass through all of them, on fresh tensors."""
    g = gen(seed)
    rand = lambda *s: (torch.randn(s, generator=g, device="cuda") * scale).to(torch.bfloat16)  # noqa: E731
    return dict(x=rand(T, 256), dy=rand(T, 256), w=rand(256), wg=rand(512, 256), wu=rand(512, 256), wd=rand(256, 512), qkv=rand(T, 512))


OFFSETS = torch.tensor([0, 100, 100, 101, 333], dtype=torch.int64)


def chain(s, **kw):
    n = B.qless_layer_norm(s["x"], s["w"], s["w"], **kw)
    q, k, v = s["qkv"].split([256, 128, 128], dim=1)
    q, k, v = q.unflatten(1, (4, 64)), k.unflatten(1, (2, 64)), v.unflatten(1, (2, 64))
    a = B.qless_attention(q, k, v, OFFSETS, **kw)
    f = B.qless_gated_ffn(n["out"], s["wg"], s["wu"], s["wd"], want_saved=True, **kw)
    fb = B.qless_gated_ffn_backward(s["dy"], n["out"], f["gate"], f["up"], s["wg"], s["wu"], s["wd"], want_weight=True, **kw)
    nb = B.qless_layer_norm_backward(fb["grad_x"], s["x"], s["w"], n["mean"], n["rstd"], want_weight=True, want_bias=True, **kw)
    ab = B.qless_attention_backward(f["out"].unflatten(1, (4, 64)), q, k, v, a["out"], a["lse"], OFFSETS, **kw)
    out = {}
    for name, d in dict(n=n, a=a, f=f, fb=fb, nb=nb, ab=ab).items():
        out.update({f"{name}.{k}": t for k, t in d.items()})
    return out


def same(a, b):
    return all(torch.equal(a[k], b[k]) for k in a)


def test_the_same_inputs_give_the_same_bits_in_a_long_row_of_calls():
    s = everything(20)
    first = {k: t.clone() for k, t in chain(s).items()}
    for _ in range(200):
        last = chain(s)
    assert same(first, last)
    B.qless_check()


def test_on_another_stream():
    s = everything(21)
    want = chain(s)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = chain(s, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert same(want, got)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()          # two at a time
    for t in (a, b):
        t.wait_stream(torch.cuda.current_stream())
    both = [chain(s, stream=t) for t in (a, b) for _ in range(5)]
    torch.cuda.synchronize()
    assert all(same(want, g) for g in both)
    B.qless_check()


def test_in_captured_graphs_that_share_a_pool():
    s = [everything(22), everything(23)]
    want = [{k: t.clone() for k, t in chain(x).items()} for x in s]
    torch.cuda.synchronize()
    graphs, outs = [], []
    pool = None
    for x in s:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            outs.append(chain(x))
        pool = pool or graph.pool()
        graphs.append(graph)
    for _ in range(3):
        for graph, out, w in zip(graphs, outs, want):        # one behind the other: they share workspaces
            graph.replay()
            torch.cuda.synchronize()
            assert same(w, out)
    other = everything(24)
    fresh = {k: t.clone() for k, t in chain(other).items()}
    for k, t in other.items():
        s[0][k].copy_(t)
    graphs[0].replay()                                       # new contents at the captured addresses
    torch.cuda.synchronize()
    assert same(fresh, outs[0])
    B.qless_check()


def test_tables_of_work_in_captured_graphs_and_on_two_streams():
    """So many examples that the tables of tiles lie in the workspace, put there by two launches each; two lists of examples take turns."""
    H, K, D, n = 4, 1, 64, 300
    lens = [[(7 * e + s) % 41 for e in range(n)] for s in (0, 13)]
    off = [torch.tensor([sum(x[:e]) for e in range(n + 1)], dtype=torch.int64) for x in lens]
    ins = [attention_inputs(int(o[-1]), H, K, D, 30 + i) for i, o in enumerate(off)]
    want = [{k: t.clone() for k, t in run_attention(*x, o).items()} for x, o in zip(ins, off)]
    torch.cuda.synchronize()
    graphs, outs, pool = [], [], None
    for x, o in zip(ins, off):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            outs.append(run_attention(*x, o))
        pool = pool or graph.pool()
        graphs.append(graph)
    for _ in range(3):
        for graph, out, w in zip(graphs, outs, want):
            graph.replay()
            torch.cuda.synchronize()
            assert same(w, out)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for st, x, o in zip(streams, ins, off):
            with torch.cuda.stream(st):
                got.append(run_attention(*x, o))
    torch.cuda.synchronize()
    assert all(same(want[i % 2], g) for i, g in enumerate(got))
    B.qless_check()


@pytest.mark.parametrize("off,H,K,D", [([0, 3001], 2, 1, 128), ([0, 900, 900, 2304, 2305], 1, 1, 64), ([0, 1025, 1200], 4, 4, 8), ([0, 4000], 1, 1, 96), ([0, 1700], 7, 1, 40)])
def test_few_long_examples(off, H, K, D):
    """So few tiles of queries that their keys are dealt out over several blocks and joined."""
    T = off[-1]
    q, k, v, dout = attention_inputs(T + 9, H, K, D, seed=T + D)
    got = run_attention(q, k, v, dout, off)
    assert not got["out"][T:].any()
    want, room = attention_exact(q[:T], k[:T], v[:T], off, D ** -0.5, dout[:T], got["out"][:T])
    for name in ("lse", "out", "grad_v", "grad_q", "grad_k"):
        close(got[name][:T], want[name], room[name])
    assert same(got, run_attention(q, k, v, dout, off))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run_attention(q, k, v, dout, off)
    graph.replay()
    torch.cuda.synchronize()
    assert same(got, captured)
    B.qless_check()


def test_maxima_that_grow_from_piece_to_piece():
    """Keys whose scores grow by powers of two along a long example: the last pieces outweigh all before them; and an infinite value at its end reaches
    the rows that see it and those that share its tile of keys, no other."""
    T, D = 2500, 64
    q, k, v, dout = attention_inputs(T, 1, 1, D, seed=5)
    k = (k.float() * (1 + torch.arange(T, device="cuda")[:, None, None] / 64)).to(torch.bfloat16)
    got = B.qless_attention(q, k, v, [0, T])
    want, room = attention_exact(q, k, v, [0, T], D ** -0.5, dout, got["out"])
    # (as in test_maxima_that_keep_growing: scores of some hundreds; probabilities below 2^-126 may come out as 0)
    wide = 1.0 + 2.0 ** -23 * 1000 * 2 / 2.0 ** -13
    close(got["lse"], want["lse"], room["lse"])
    close(got["out"], want["out"], room["out"] * wide + T * 2.0 ** -126 * float(v.abs().max()))
    v = v.clone()
    v[2490] = float("inf")
    again = B.qless_attention(q, k, v, [0, T])
    start = 2490 // 128 * 128
    assert torch.equal(again["out"][:start], got["out"][:start]) and not torch.isfinite(again["out"][2490:].float()).all(dim=(1, 2)).any()
    B.qless_check()


@pytest.mark.parametrize("T,H,K,D", [(700, 32, 1, 128), (413, 24, 1, 64), (1003, 7, 1, 40)])
def test_many_heads_that_share_a_key_head(T, H, K, D):
    """So many query rows to so few tiles of keys that these rows are dealt out, over the passes of the group's heads too; an example without tokens between."""
    off = [0, 5, 5, T]
    q, k, v, dout = attention_inputs(T, H, K, D, seed=T + H)
    got = run_attention(q, k, v, dout, off)
    want, room = attention_exact(q, k, v, off, D ** -0.5, dout, got["out"])
    for name in ("lse", "out", "grad_v", "grad_q", "grad_k"):
        close(got[name], want[name], room[name])
    assert same(got, run_attention(q, k, v, dout, off))
    B.qless_check()
