"""Cases that time the operators which turn a language model's backward pass into gradient rows: 8-bit activation
checkpoints, per-example LoRA gradients from them, and the softmax cross entropy over a large vocabulary with its
gradient. Each case can be computed in a plain form (elementary torch operations in 32 bits) or by the library."""
import math
import random

import torch

own = False

DEV = "cuda"
HIDDEN_WANTED = ("hidden", "both")


def listed():
    return [
        # Latency: the last layer's input of one short prompt in fp32.
        dict(name="checkpoint_small", op="checkpoint", tokens=37, width=512, group=32, dtype="f32"),
        # One layer's input for a batch of instruction examples.
        dict(name="checkpoint_batch", op="checkpoint", tokens=8192, width=4096, group=64, dtype="bf16"),
        # Layer inputs of a whole gradient-extraction batch kept at once; a width that is no multiple of the group.
        dict(name="checkpoint_large", op="checkpoint", tokens=65521, width=4112, group=128, dtype="bf16"),
        # Latency: eight examples of a few answer tokens, a small adapter, gradients in fp32.
        dict(name="lora_small", op="lora", examples=8, tokens=19, width_in=512, width_out=512, rank=8, group=32, dtype="f32"),
        # One adapted projection for a batch of 32 ragged instruction examples, rank 64.
        dict(name="lora_batch", op="lora", examples=32, tokens=16381, width_in=4096, width_out=4096, rank=64, group=32, dtype="bf16"),
        # Two long documents through a narrow output projection: few examples, a long axis to sum over.
        dict(name="lora_long", op="lora", examples=2, tokens=16383, width_in=4096, width_out=1024, rank=16, group=64, dtype="f32"),
        # The largest batch: 128 examples, gradients in the type the projection reads.
        dict(name="lora_large", op="lora", examples=128, tokens=65536, width_in=4096, width_out=4096, rank=64, group=128, dtype="bf16"),
        # Latency: the answer tokens of one short example, a small odd vocabulary.
        dict(name="loss_small", op="loss", tokens=33, kept=21, width=512, vocab=4099, wants="hidden"),
        # Per-token losses alone (ranking candidates by their loss).
        dict(name="loss_only", op="loss", tokens=2048, kept=2048, width=4096, vocab=32000, wants="none"),
        # A few answer tokens against a full head: the weights' bytes count.
        dict(name="loss_few", op="loss", tokens=127, kept=64, width=4096, vocab=32001, wants="hidden"),
        # A head that is trained too: gradients of hidden states and weights.
        dict(name="loss_trained", op="loss", tokens=4095, kept=3001, width=2048, vocab=50021, wants="both"),
        # Instruction tuning over a large vocabulary: half of the tokens are prompt and carry no loss.
        dict(name="loss_large", op="loss", tokens=8192, kept=4096, width=4096, vocab=131072, wants="hidden"),
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["checkpoint", "lora", "lora", "loss", "loss"])
    if op == "checkpoint":
        width = _log(rng, 256, 8192, 8)
        return dict(op=op, tokens=_log(rng, 1, min(65536, 260_000_000 // width)), width=width, group=rng.choice([32, 64, 128]),
                    dtype=rng.choice(["f32", "bf16"]))
    if op == "lora":
        wi, wo = _log(rng, 256, 8192, 16), _log(rng, 256, 8192, 16)
        tokens = _log(rng, 1, 500_000_000 // (wi + wo))
        rank = rng.choice([8, 16, 24, 32, 64, 128])
        examples = _log(rng, 1, max(1, min(128, 4 * tokens, 60_000_000 // (rank * (wi + wo)))))
        return dict(op=op, examples=examples, tokens=tokens, width_in=wi, width_out=wo, rank=rank, group=rng.choice([32, 64, 128]),
                    dtype=rng.choice(["f32", "bf16"]))
    width, vocab = _log(rng, 256, 5120, 8), _log(rng, 1000, 131072)
    wants = rng.choice(["none", "hidden", "hidden", "both"])
    tokens = _log(rng, 1, max(2, min(8192, int(8192 * 4096 * 131072 / 2 / (width * vocab)))))
    return dict(op=op, tokens=tokens, kept=max(1, int(tokens * rng.choice([1.0, 0.7, 0.4]))), width=width, vocab=vocab, wants=wants)


def _lengths(case, seed):
    """Example lengths that add up to the case's tokens: some long, some short, one empty and one of a single token where
    there are four examples or more."""
    rng = random.Random(seed)
    n, total = case["examples"], case["tokens"]
    w = [rng.uniform(0.25, 1.75) for _ in range(n)]
    if n >= 4:
        w[rng.randrange(n)] = 0.0
    whole = sum(w)
    ends = [0]
    at = 0.0
    for x in w:
        at += x
        ends.append(min(total, int(round(total * at / whole))))
    ends[-1] = total
    return ends


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    return g


def _torch_type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _activations(g, tokens, width, dtype):
    """Inputs of a layer behind a normalisation: unit entries, a few channels that are some twenty times larger."""
    gain = torch.exp(0.4 * torch.randn(width, generator=g, device=DEV))
    gain[torch.rand(width, generator=g, device=DEV) < 0.004] *= 20.0
    return (torch.randn((tokens, width), generator=g, device=DEV) * gain).to(dtype)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    if case["op"] == "checkpoint":
        s["x"] = _activations(g, case["tokens"], case["width"], _torch_type(case["dtype"]))
    elif case["op"] == "lora":
        t, wi, wo, r = case["tokens"], case["width_in"], case["width_out"], case["rank"]
        x = _activations(g, t, wi, torch.float32)
        codes, scales = _plain_quantize(x, case["group"])
        s["codes"], s["scales"] = codes.to(torch.int8), scales
        row = torch.exp(torch.randn((t, 1), generator=g, device=DEV))                  # tokens differ in the size of their gradient
        s["grad_out"] = (torch.randn((t, wo), generator=g, device=DEV) * row * 1e-3).to(torch.bfloat16)
        s["lora_a"] = ((torch.rand((r, wi), generator=g, device=DEV) * 2 - 1) / math.sqrt(wi)).to(torch.bfloat16)
        s["lora_b"] = (torch.randn((wo, r), generator=g, device=DEV) * 0.02).to(torch.bfloat16)
        s["offsets"] = torch.tensor(_lengths(case, seed), dtype=torch.int64)
        s["scaling"] = 4.0
    else:
        t, h, v = case["tokens"], case["width"], case["vocab"]
        s["weight"] = (torch.randn((v, h), generator=g, device=DEV) * 0.02).to(torch.bfloat16)
        truth = torch.randint(0, v, (t,), generator=g, device=DEV)
        # tokens from hopeless to all but certain: the label's logit is moved by up to 14
        pull = torch.rand((t, 1), generator=g, device=DEV) * 14.0 / (0.0004 * h)
        s["hidden"] = (torch.randn((t, h), generator=g, device=DEV) + pull * s["weight"][truth].float()).to(torch.bfloat16)
        order = torch.randperm(t, generator=g, device=DEV)
        labels = truth.clone()
        labels[order[case["kept"]:]] = -100                                            # prompt tokens
        s["labels"] = labels
        s["token_weight"] = torch.rand(t, generator=g, device=DEV) / case["kept"] + 1e-6
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def _plain_quantize(x, group):
    """Codes (whole numbers in fp32) [tokens, width] and biased exponents (uint8) [tokens, groups]."""
    t, w = x.shape
    groups = -(-w // group)
    y = torch.nn.functional.pad(x.float(), (0, groups * group - w)).view(t, groups, group)
    top = y.abs().amax(dim=2)
    mant, exp = torch.frexp(top)                                                       # top = mant * 2^exp, mant in [1/2, 1)
    e = exp - 7 + (mant > 127.0 / 128.0).to(exp.dtype)
    e = torch.where(top > 0, e, torch.full_like(e, -120)).clamp(-120, 121)
    codes = torch.round(torch.ldexp(y, -e.unsqueeze(2))).reshape(t, groups * group)[:, :w]
    return codes, (e + 127).to(torch.uint8)


def _plain_dequantize(codes, scales, group):
    w = codes.shape[1]
    step = torch.ldexp(torch.ones(scales.shape, device=scales.device), scales.to(torch.int32) - 127)
    return codes.float() * step.repeat_interleave(group, dim=1)[:, :w]


def _plain_lora(s):
    case = s["case"]
    x = _plain_dequantize(s["codes"], s["scales"], case["group"])
    dy, a, b = s["grad_out"].float(), s["lora_a"].float(), s["lora_b"].float()
    lo = s["offsets"][:-1].to(DEV)
    count = s["offsets"][1:].to(DEV) - lo
    longest = int((s["offsets"][1:] - s["offsets"][:-1]).max())
    at = torch.arange(longest, device=DEV)
    live = (at[None, :] < count[:, None]).unsqueeze(2)
    place = (lo[:, None] + at[None, :]).clamp(max=case["tokens"] - 1)
    xe, de = torch.where(live, x[place], 0.0), torch.where(live, dy[place], 0.0)       # [examples, longest, width]
    u = s["scaling"] * (de @ b)
    h = s["scaling"] * (xe @ a.T)
    da, db = u.transpose(1, 2) @ xe, de.transpose(1, 2) @ h
    return torch.cat([da.flatten(1), db.flatten(1)], dim=1).to(_torch_type(case["dtype"]))


def _plain_loss(s):
    case = s["case"]
    live = s["labels"] >= 0
    y = s["labels"].clamp(min=0)
    x, w = s["hidden"].float(), s["weight"].float()
    logits = x @ w.T
    top = logits.amax(dim=1, keepdim=True)
    p = (logits - top).exp_()
    total = p.sum(dim=1, keepdim=True)
    loss = torch.where(live, (top + total.log() - logits.gather(1, y[:, None]))[:, 0], 0.0)
    out = dict(loss=loss)
    del logits
    if case["wants"] in HIDDEN_WANTED:
        p /= total
        p.scatter_add_(1, y[:, None], torch.full((len(y), 1), -1.0, device=DEV))
        p *= torch.where(live, s["token_weight"], 0.0)[:, None]
        out["grad_hidden"] = (p @ w).to(torch.bfloat16)
        if case["wants"] == "both":
            out["grad_weight"] = (p.T @ x).to(torch.bfloat16)
    return out


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        from paper_2502_01703_b200 import binding as B
        if case["op"] == "checkpoint":
            codes, scales = B.qless_activation_quantize(state["x"], group=case["group"])
            return dict(exponents=scales, values=B.qless_activation_dequantize(codes, scales, group=case["group"], dtype=state["x"].dtype))
        if case["op"] == "lora":
            return B.qless_lora_gradients(state["codes"], state["scales"], state["grad_out"], state["lora_a"], state["lora_b"],
                                          state["offsets"], scaling=state["scaling"], group=case["group"], dtype=_torch_type(case["dtype"]))
        got = B.qless_lm_loss(state["hidden"], state["weight"], state["labels"], token_weight=state["token_weight"],
                              want_hidden=case["wants"] in HIDDEN_WANTED, want_weight=case["wants"] == "both")
        return {k: v for k, v in got.items() if v is not None}
    if case["op"] == "checkpoint":
        codes, scales = _plain_quantize(state["x"], case["group"])
        return dict(exponents=scales, values=_plain_dequantize(codes.to(torch.int8), scales, case["group"]).to(state["x"].dtype))
    if case["op"] == "lora":
        return _plain_lora(state)
    return _plain_loss(state)


def work(case):
    if case["op"] == "checkpoint":
        n, size = case["tokens"] * case["width"], 4 if case["dtype"] == "f32" else 2
        scales = case["tokens"] * -(-case["width"] // case["group"])
        return dict(bytes=2 * n * size + 2 * n + 2 * scales, flops=4 * n)
    if case["op"] == "lora":
        t, wi, wo, r = case["tokens"], case["width_in"], case["width_out"], case["rank"]
        size = 4 if case["dtype"] == "f32" else 2
        return dict(bytes=t * (wi + -(-wi // case["group"])) + 2 * t * wo + 2 * r * (wi + wo) + case["examples"] * r * (wi + wo) * size,
                    flops=4 * t * r * (wi + wo))
    t, m, h, v = case["tokens"], case["kept"], case["width"], case["vocab"]
    products = dict(none=1, hidden=2, both=3)[case["wants"]]
    size = 2 * m * h + 2 * v * h + 16 * t
    size += 2 * t * h if products > 1 else 0
    size += 2 * v * h if products > 2 else 0
    return dict(bytes=size, flops=2 * m * h * v * products)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _exact_values(x, group):
    """The values that 8-bit codes with a power of two per group stand for: the smallest step whose 127-fold covers the group."""
    t, w = x.shape
    out = torch.empty_like(x)
    for c in range(0, w, group):
        y = x[:, c:c + group]
        top = y.abs().max(dim=1, keepdim=True).values
        step = torch.exp2(torch.ceil(torch.log2(top / 127.0)).clamp(-120.0, 121.0))
        step = torch.where(top > 127.0 * step, 2.0 * step, step)
        step = torch.where((top <= 63.5 * step) & (step > 2.0 ** -120), 0.5 * step, step)
        out[:, c:c + group] = torch.round(y / step) * step
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "checkpoint":
        return dict(exponents=None, values=_exact_values(s["x"].double(), case["group"]))
    if case["op"] == "lora":
        r, wi, wo = case["rank"], case["width_in"], case["width_out"]
        groups = -(-wi // case["group"])
        rows = torch.zeros((case["examples"], r * (wi + wo)), dtype=torch.float64, device=DEV)
        a, b = s["lora_a"].double(), s["lora_b"].double()
        for e in range(case["examples"]):
            lo, hi = int(s["offsets"][e]), int(s["offsets"][e + 1])
            if lo == hi:
                continue
            channel = torch.arange(wi, device=DEV) // case["group"]
            step = torch.pow(2.0, s["scales"][lo:hi].double() - 127.0)[:, :groups]
            x = s["codes"][lo:hi].double() * step[:, channel]
            dy = s["grad_out"][lo:hi].double()
            rows[e, :r * wi] = torch.einsum("tr,tc->rc", s["scaling"] * (dy @ b), x).reshape(-1)
            rows[e, r * wi:] = s["scaling"] * torch.einsum("to,tr->or", dy, torch.einsum("tc,rc->tr", x, a)).reshape(-1)
        return rows
    t, h, v = case["tokens"], case["width"], case["vocab"]
    keep = torch.nonzero(s["labels"] >= 0)[:, 0]
    y = s["labels"][keep]
    x, w = s["hidden"][keep].double(), s["weight"].double()
    logits = torch.einsum("th,vh->tv", x, w)
    lse = torch.logsumexp(logits, dim=1)
    at = torch.arange(len(y), device=DEV)
    loss = torch.zeros(t, dtype=torch.float64, device=DEV)
    loss[keep] = lse - logits[at, y]
    out = dict(loss=loss)
    if case["wants"] in HIDDEN_WANTED:
        grad = torch.exp(logits.sub_(lse[:, None]))
        # the label's entry, 1 less than its probability, as minus the sum of the others
        grad[at, y] = 0.0
        grad[at, y] = -grad.sum(dim=1)
        grad *= s["token_weight"].double()[keep, None]
        out["grad_hidden"] = torch.zeros((t, h), dtype=torch.float64, device=DEV)
        out["grad_hidden"][keep] = grad @ w
        if case["wants"] == "both":
            out["grad_weight"] = grad.T @ x
    return out
