"""Cases that time the operators which carry a loss's gradient through a decoder layer, down to the projections whose LoRA
gradients are wanted: causal attention over packed examples, the normalisation of a layer's input, and the gated feed-forward
block, each forward and backward. Each case can be computed in a plain form (elementary torch operations in 32 bits) or by
the library."""
import math
import random

import torch

own = False

DEV = "cuda"


def listed():
    return [
        # Latency: the input of one layer for a short prompt in fp32.
        dict(name="norm_small", op="norm", way="forward", tokens=37, width=512, dtype="f32", center=True, bias=True, wants="hidden"),
        # A layer's input for a batch of instruction examples, scale only.
        dict(name="norm_batch", op="norm", way="forward", tokens=16381, width=4096, dtype="bf16", center=False, bias=False, wants="hidden"),
        # The same on the way back, parameters trained too; a long packed batch, a width that is no multiple of 128.
        dict(name="norm_back_large", op="norm", way="backward", tokens=65521, width=4112, dtype="bf16", center=True, bias=True, wants="both"),
        # Latency: eight examples of some twenty tokens through a small layer.
        dict(name="attn_small", op="attn", way="forward", examples=8, tokens=171, heads=8, kv_heads=2, head_dim=64),
        # One layer for a batch of 32 ragged instruction examples, four query heads to a key head.
        dict(name="attn_batch", op="attn", way="forward", examples=32, tokens=16381, heads=32, kv_heads=8, head_dim=128),
        # The same batch on the way back.
        dict(name="attn_back_batch", op="attn", way="backward", examples=32, tokens=16381, heads=32, kv_heads=8, head_dim=128),
        # Two long documents.
        dict(name="attn_long", op="attn", way="forward", examples=2, tokens=16383, heads=32, kv_heads=8, head_dim=128),
        # A document on the way back, a key head to every query head, narrow heads.
        dict(name="attn_back_narrow", op="attn", way="backward", examples=1, tokens=8191, heads=16, kv_heads=16, head_dim=64),
        # Latency: the last tokens of one short prompt through a small block.
        dict(name="ffn_small", op="ffn", way="forward", tokens=5, width=512, inner=1376, wants="hidden"),
        # A few answer tokens through a full block: the weights' bytes count.
        dict(name="ffn_few", op="ffn", way="forward", tokens=61, width=4096, inner=11008, wants="hidden"),
        # A batch of instruction examples on the way back to the block's input, its weights frozen.
        dict(name="ffn_back_batch", op="ffn", way="backward", tokens=4095, width=4096, inner=11008, wants="hidden"),
        # The block's weights trained too.
        dict(name="ffn_back_trained", op="ffn", way="backward", tokens=8192, width=2048, inner=5632, wants="both"),
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["norm", "attn", "attn", "ffn", "ffn"])
    way = rng.choice(["forward", "backward"])
    if op == "norm":
        width = _log(rng, 64, 8192, rng.choice([1, 8, 8]))
        return dict(op=op, way=way, tokens=_log(rng, 1, min(65536, 260_000_000 // width)), width=width, dtype=rng.choice(["f32", "bf16", "bf16"]),
                    center=rng.choice([True, False]), bias=rng.choice([True, False]), wants=rng.choice(["hidden", "both"]))
    if op == "attn":
        head_dim = rng.choice([40, 64, 64, 80, 96, 128, 128])
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 4, 4, 7, 8])
        tokens = _log(rng, 2, min(16384, 70_000_000 // (heads * head_dim)))
        # the plain form holds every score of the padded batch
        fewest = max(1, math.ceil(heads * (1.75 * tokens) ** 2 / 7.0e9))
        examples = max(fewest, _log(rng, 1, max(1, min(64, tokens // 2))))
        return dict(op=op, way=way, examples=examples, tokens=tokens, heads=heads, kv_heads=kv, head_dim=head_dim)
    width = _log(rng, 256, 5120, 8)
    inner = max(256, int(width * rng.uniform(2.0, 4.0)) // 8 * 8)
    wants = rng.choice(["hidden", "hidden", "both"]) if way == "backward" else "hidden"
    return dict(op=op, way=way, tokens=_log(rng, 1, max(2, min(8192, 94_000_000_000 // (width * inner)))), width=width, inner=inner, wants=wants)


def _lengths(case):
    """Example lengths that add up to the case's tokens: some long, some short, one empty where there are four examples or more."""
    n, total = case["examples"], case["tokens"]
    rng = random.Random(1000003 * n + total)
    w = [rng.uniform(0.25, 1.75) for _ in range(n)]
    if n >= 4:
        w[rng.randrange(n)] = 0.0
    ends = [0]
    at = 0.0
    for x in w:
        at += x
        ends.append(min(total, int(round(total * at / sum(w)))))
    ends[-1] = total
    return ends


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    return g


def _torch_type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _stream(g, tokens, width):
    """A residual stream: entries around one, a few channels that are some twenty times larger, a mean that is not zero."""
    gain = torch.exp(0.4 * torch.randn(width, generator=g, device=DEV))
    gain[torch.rand(width, generator=g, device=DEV) < 0.004] *= 20.0
    return torch.randn((tokens, width), generator=g, device=DEV) * gain + 0.1


def _grads(g, tokens, width):
    """Gradients: tokens differ in the size of theirs."""
    row = torch.exp(torch.randn((tokens, 1), generator=g, device=DEV))
    return torch.randn((tokens, width), generator=g, device=DEV) * row * 1e-3


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    if case["op"] == "norm":
        t, w, dt = case["tokens"], case["width"], _torch_type(case["dtype"])
        s["x"] = _stream(g, t, w).to(dt)
        s["weight"] = (1.0 + 0.2 * torch.randn(w, generator=g, device=DEV)).to(dt)
        s["bias"] = (0.1 * torch.randn(w, generator=g, device=DEV)).to(dt) if case["bias"] else None
        if case["way"] == "backward":
            s["grad_out"] = _grads(g, t, w).to(dt)
            s["mean"], s["rstd"] = _plain_moments(s["x"].float(), case["center"])
    elif case["op"] == "attn":
        t, h, kv, d = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
        # heads differ in how sharply they look: scores with a spread of 0.5 to 4
        sharp = torch.exp(torch.rand((1, kv, 1), generator=g, device=DEV) * math.log(8.0)) * 0.5
        s["q"] = torch.randn((t, h, d), generator=g, device=DEV).to(torch.bfloat16)
        s["k"] = (torch.randn((t, kv, d), generator=g, device=DEV) * sharp).to(torch.bfloat16)
        s["v"] = torch.randn((t, kv, d), generator=g, device=DEV).to(torch.bfloat16)
        s["offsets"] = torch.tensor(_lengths(case), dtype=torch.int64)
        if case["way"] == "backward":
            out, lse = _plain_attention(s)
            s["out"], s["lse"] = out.to(torch.bfloat16), lse
            s["grad_out"] = _grads(g, t, h * d).view(t, h, d).to(torch.bfloat16)
    else:
        t, w, f = case["tokens"], case["width"], case["inner"]
        # behind a normalisation: unit entries
        s["x"] = torch.randn((t, w), generator=g, device=DEV).to(torch.bfloat16)
        s["w_gate"], s["w_up"] = [(torch.randn((f, w), generator=g, device=DEV) * 1.5 / math.sqrt(w)).to(torch.bfloat16) for _ in range(2)]
        s["w_down"] = (torch.randn((w, f), generator=g, device=DEV) / math.sqrt(f)).to(torch.bfloat16)
        if case["way"] == "backward":
            x = s["x"].float()
            s["gate"], s["up"] = (x @ s["w_gate"].float().T).to(torch.bfloat16), (x @ s["w_up"].float().T).to(torch.bfloat16)
            s["grad_out"] = _grads(g, t, w).to(torch.bfloat16)
    return s


EPS = 1e-5


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def _plain_moments(x, center):
    mean = x.mean(dim=1) if center else torch.zeros(x.shape[0], device=x.device)
    y = x - mean[:, None]
    return mean, torch.rsqrt((y * y).mean(dim=1) + EPS)


def _plain_norm(s):
    case, dt = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["weight"].float()
    if case["way"] == "forward":
        mean, rstd = _plain_moments(x, case["center"])
        out = (x - mean[:, None]) * rstd[:, None] * w
        return dict(out=(out + s["bias"].float() if s["bias"] is not None else out).to(dt), rstd=rstd)
    dy = s["grad_out"].float()
    xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
    wdy = dy * w
    along = (wdy * xhat).mean(dim=1, keepdim=True)
    dx = wdy - xhat * along
    if case["center"]:
        dx = dx - wdy.mean(dim=1, keepdim=True)
    out = dict(grad_x=(dx * s["rstd"][:, None]).to(dt))
    if case["wants"] == "both":
        out["grad_weight"] = (dy * xhat).double().sum(dim=0).to(dt)        # long sums with a small result
        if s["bias"] is not None:
            out["grad_bias"] = dy.double().sum(dim=0).to(dt)
    return out


def _plain_scores(s):
    """The padded batch: places of the tokens [examples, longest], which of them are there, queries, keys, values [examples, heads, longest,
    head_dim] in 32 bits, scores with -infinity where a query does not look."""
    case = s["case"]
    lo = s["offsets"][:-1].to(DEV)
    count = s["offsets"][1:].to(DEV) - lo
    longest = int((s["offsets"][1:] - s["offsets"][:-1]).max())
    at = torch.arange(longest, device=DEV)
    live = at[None, :] < count[:, None]
    place = (lo[:, None] + at[None, :]).clamp(max=case["tokens"] - 1)
    group = case["heads"] // case["kv_heads"]
    q = s["q"].float()[place].transpose(1, 2)
    k, v = [s[name].float()[place].transpose(1, 2).repeat_interleave(group, dim=1) for name in ("k", "v")]
    scores = q @ k.transpose(2, 3)
    scores *= 1.0 / math.sqrt(case["head_dim"])
    scores.masked_fill_((at[:, None] < at[None, :])[None, None], -math.inf)
    return place, live, q, k, v, scores


def _plain_softmax(scores):
    """In the scores' place; also the logarithm of the sum of exponentials."""
    top = scores.amax(dim=3, keepdim=True)
    p = scores.sub_(top).exp_()
    total = p.sum(dim=3, keepdim=True)
    p /= total
    return p, (top + total.log())[..., 0]


def _packed(y, live):
    """[examples, heads, longest, ...] -> [tokens, heads, ...]"""
    return y.transpose(1, 2)[live]


def _plain_attention(s):
    place, live, q, k, v, scores = _plain_scores(s)
    p, lse = _plain_softmax(scores)
    return _packed(p @ v, live), _packed(lse, live)


def _plain_attention_backward(s):
    case = s["case"]
    place, live, q, k, v, scores = _plain_scores(s)
    p, _ = _plain_softmax(scores)
    do = s["grad_out"].float()[place]
    do = torch.where(live[:, :, None, None], do, 0.0).transpose(1, 2)
    dv = p.transpose(2, 3) @ do
    ds = do @ v.transpose(2, 3)
    ds -= (do * (p @ v)).sum(dim=3, keepdim=True)
    ds *= p
    ds *= 1.0 / math.sqrt(case["head_dim"])
    dq, dk = ds @ k, ds.transpose(2, 3) @ q
    shape = (case["tokens"], case["kv_heads"], case["heads"] // case["kv_heads"], case["head_dim"])
    return dict(grad_q=_packed(dq, live).to(torch.bfloat16), grad_k=_packed(dk, live).view(shape).sum(dim=2).to(torch.bfloat16),
                grad_v=_packed(dv, live).view(shape).sum(dim=2).to(torch.bfloat16))


def _plain_ffn(s):
    case, b16 = s["case"], torch.bfloat16
    x, wg, wu, wd = s["x"].float(), s["w_gate"].float(), s["w_up"].float(), s["w_down"].float()
    if case["way"] == "forward":
        gate = x @ wg.T
        return dict(out=(((gate / (1.0 + torch.exp(-gate))) * (x @ wu.T)) @ wd.T).to(b16))
    gate, up, dy = s["gate"].float(), s["up"].float(), s["grad_out"].float()
    sig = 1.0 / (1.0 + torch.exp(-gate))
    dh = dy @ wd
    dgate, dup = dh * up * sig * (1.0 + gate * (1.0 - sig)), dh * gate * sig
    out = dict(grad_x=(dgate @ wg + dup @ wu).to(b16), grad_gate=dgate.to(b16), grad_up=dup.to(b16))
    if case["wants"] == "both":
        out.update(grad_w_gate=(dgate.T @ x).to(b16), grad_w_up=(dup.T @ x).to(b16), grad_w_down=(dy.T @ (gate * sig * up)).to(b16))
    return out


# ---- one pass ----------------------------------------------------------------------------------------------------------

def _there(d):
    return {k: v for k, v in d.items() if v is not None}


def run(state):
    s, case = state, state["case"]
    if own:
        from paper_2502_01703_b200 import binding as B
        if case["op"] == "norm":
            if case["way"] == "forward":
                got = B.qless_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, center=case["center"])
                return dict(out=got["out"], rstd=got["rstd"])
            return _there(B.qless_layer_norm_backward(s["grad_out"], s["x"], s["weight"], s["mean"] if case["center"] else None, s["rstd"],
                                                      want_weight=case["wants"] == "both", want_bias=case["wants"] == "both" and case["bias"]))
        if case["op"] == "attn":
            if case["way"] == "forward":
                return B.qless_attention(s["q"], s["k"], s["v"], s["offsets"])
            return B.qless_attention_backward(s["grad_out"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["offsets"])
        if case["way"] == "forward":
            return dict(out=B.qless_gated_ffn(s["x"], s["w_gate"], s["w_up"], s["w_down"])["out"])
        return _there(B.qless_gated_ffn_backward(s["grad_out"], s["x"], s["gate"], s["up"], s["w_gate"], s["w_up"], s["w_down"],
                                                 want_weight=case["wants"] == "both"))
    if case["op"] == "norm":
        return _plain_norm(s)
    if case["op"] == "attn":
        if case["way"] == "backward":
            return _plain_attention_backward(s)
        out, lse = _plain_attention(s)
        return dict(out=out.to(torch.bfloat16), lse=lse)
    return _plain_ffn(s)


def work(case):
    t = case["tokens"]
    if case["op"] == "norm":
        n, size = t * case["width"], 4 if case["dtype"] == "f32" else 2
        if case["way"] == "forward":
            return dict(bytes=2 * n * size + 4 * t, flops=7 * n)
        return dict(bytes=3 * n * size + 8 * t, flops=(14 if case["wants"] == "both" else 10) * n)
    if case["op"] == "attn":
        h, kv, d = case["heads"], case["kv_heads"], case["head_dim"]
        ends = _lengths(case)
        pairs = sum((b - a) * (b - a + 1) // 2 for a, b in zip(ends, ends[1:]))
        if case["way"] == "forward":
            return dict(bytes=2 * t * d * (2 * h + 2 * kv) + 4 * t * h, flops=4 * d * h * pairs)
        return dict(bytes=2 * t * d * (4 * h + 4 * kv) + 4 * t * h, flops=10 * d * h * pairs)
    w, f = case["width"], case["inner"]
    if case["way"] == "forward":
        return dict(bytes=2 * (2 * t * w + 3 * w * f), flops=6 * t * w * f)
    both = case["wants"] == "both"
    return dict(bytes=2 * ((3 if both else 2) * t * w + 4 * t * f + (6 if both else 3) * w * f), flops=(12 if both else 6) * t * w * f)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _exact_norm(s):
    case = s["case"]
    x = s["x"].double().requires_grad_()
    w = s["weight"].double().requires_grad_()
    b = (s["bias"].double() if s["bias"] is not None else torch.zeros_like(w)).requires_grad_()
    var = x.var(dim=1, unbiased=False, keepdim=True) if case["center"] else x.square().mean(dim=1, keepdim=True)
    y = (x - x.mean(dim=1, keepdim=True) if case["center"] else x) / torch.sqrt(var + EPS) * w + b
    if case["way"] == "forward":
        return dict(out=y.detach(), rstd=(var.detach() + EPS).pow(-0.5)[:, 0])
    gx, gw, gb = torch.autograd.grad(y, (x, w, b), s["grad_out"].double())
    out = dict(grad_x=gx)
    if case["wants"] == "both":
        out["grad_weight"] = gw
        if s["bias"] is not None:
            out["grad_bias"] = gb
    return out


def _exact_attention(s):
    case = s["case"]
    t, h, kv, d = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
    back = case["way"] == "backward"
    zero = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)  # noqa: E731
    out, lse, dq, dk, dv = zero(t, h, d), zero(t, h), zero(t, h, d), zero(t, kv, d), zero(t, kv, d)
    ends = s["offsets"].tolist()
    for lo, hi in zip(ends, ends[1:]):
        if lo == hi:
            continue
        sees = torch.ones((hi - lo, hi - lo), dtype=torch.bool, device=DEV).tril()
        for j in range(h):
            c = j * kv // h
            q, k, v = [s[n][lo:hi, i].double().requires_grad_(back) for n, i in (("q", j), ("k", c), ("v", c))]
            logits = torch.where(sees, torch.einsum("id,jd->ij", q, k) / d ** 0.5, -math.inf)
            y = torch.einsum("ij,jd->id", torch.softmax(logits, dim=1), v)
            if back:
                a, b, e = torch.autograd.grad(y, (q, k, v), s["grad_out"][lo:hi, j].double())
                dq[lo:hi, j] = a
                dk[lo:hi, c] += b
                dv[lo:hi, c] += e
            else:
                out[lo:hi, j], lse[lo:hi, j] = y, torch.logsumexp(logits, dim=1)
    return dict(grad_q=dq, grad_k=dk, grad_v=dv) if back else dict(out=out, lse=lse)


def _exact_ffn(s):
    case = s["case"]
    x, wg, wu, wd = [s[n].double() for n in ("x", "w_gate", "w_up", "w_down")]
    if case["way"] == "forward":
        h = torch.nn.functional.silu(torch.einsum("tw,fw->tf", x, wg)) * torch.einsum("tw,fw->tf", x, wu)
        return dict(out=torch.einsum("tf,wf->tw", h, wd))
    gate, up = s["gate"].double().requires_grad_(), s["up"].double().requires_grad_()
    dy = s["grad_out"].double()
    h = torch.nn.functional.silu(gate) * up
    dgate, dup = torch.autograd.grad(h, (gate, up), torch.einsum("tw,wf->tf", dy, wd))
    out = dict(grad_x=torch.einsum("tf,fw->tw", dgate, wg) + torch.einsum("tf,fw->tw", dup, wu), grad_gate=dgate, grad_up=dup)
    if case["wants"] == "both":
        out.update(grad_w_gate=torch.einsum("tf,tw->fw", dgate, x), grad_w_up=torch.einsum("tf,tw->fw", dup, x),
                   grad_w_down=torch.einsum("tw,tf->wf", dy, h.detach()))
    return out


def exact(case, seed):
    return dict(norm=_exact_norm, attn=_exact_attention, ffn=_exact_ffn)[case["op"]](prepare(case, seed))
