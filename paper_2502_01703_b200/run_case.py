"""Run one stage of the hot path at a chosen shape on synthetic inputs (for profiling a small case).

    python -m paper_2502_01703_b200.run_case project  --n 256 --P 1048576 --d 8192 --bits 4 --iters 3   (--matrix gaussian)
    python -m paper_2502_01703_b200.run_case quantize --n 32768 --d 8192 --bits 4
    python -m paper_2502_01703_b200.run_case score    --N 20000 --V 448 --C 4 --d 8192 --bits 8     (16: the bf16 baseline)
    python -m paper_2502_01703_b200.run_case select   --N 67108864 --frac 0.05
    python -m paper_2502_01703_b200.run_case extract  --n 32 --tokens 16384 --width 2048 --vocab 32000 --rank 16 --d 1024 --bits 4
    python -m paper_2502_01703_b200.run_case layer    --n 32 --tokens 16384 --width 2048 --heads 16 --kv-heads 4 --inner 5632 --rank 16 --d 1024 --bits 4

Prints the CUDA-event time per iteration of the library call (extract, layer: of each call; the products of layer's attention projections, forward and backward, are
torch's and not among the printed times).
"""
import argparse

import torch

from . import binding as B
from . import workloads as W


def extract(n, tokens, width, vocab, rank, d, bits, seed=1, group=32, scaling=2.0, device="cuda"):
    """From packed tokens to datastore rows: the last adapted layer y = W x + scaling * B (A x) of a language model (random weights)
    feeds its head. The layer's input is kept as an 8-bit checkpoint, the loss of the second half of every example's tokens (the
    answer; mean per example) gives the gradient at y, that and the checkpoint the example's LoRA gradient, and the gradient its
    projected code. Returns the inputs, every intermediate result and the milliseconds of each library call."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    def rand(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device=device) * scale).to(torch.bfloat16)
    cuts = torch.randint(1, max(tokens, 2), (n - 1,), generator=g, device=device).sort().values.cpu()
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([tokens])])
    x, w = rand(tokens, width), rand(width, width, scale=width ** -0.5)
    a, b = rand(rank, width, scale=width ** -0.5), rand(width, rank, scale=0.05)
    head = rand(vocab, width, scale=2.0 * width ** -0.5)
    labels = torch.randint(0, vocab, (tokens,), generator=g, device=device)
    weight = torch.zeros(tokens, device=device)
    for e in range(n):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        answer = lo + (hi - lo) // 2
        labels[lo:answer] = -100
        weight[answer:hi] = 1.0 / max(hi - answer, 1)
    hidden = x @ w.T + (scaling * (x @ a.T) @ b.T).to(torch.bfloat16)

    ms = {}
    def timed(name, fn):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        out = fn()
        end.record()
        end.synchronize()
        ms[name] = start.elapsed_time(end)
        return out
    codes, scales = timed("qless_activation_quantize", lambda: B.qless_activation_quantize(x, group=group))
    loss = timed("qless_lm_loss", lambda: B.qless_lm_loss(hidden, head, labels, token_weight=weight))
    grads = timed("qless_lora_gradients", lambda: B.qless_lora_gradients(codes, scales, loss["grad_hidden"], a, b, offsets, scaling=scaling, group=group))
    store = timed("qless_project_quantize", lambda: B.qless_project_quantize(grads, d, 7, bits))
    B.qless_check()
    return dict(offsets=offsets, x=x, a=a, b=b, head=head, labels=labels, weight=weight, hidden=hidden, scaling=scaling, group=group,
                checkpoint=(codes, scales), loss=loss, grads=grads, store=store, ms=ms)


def layer(n, tokens, width, heads, kv_heads, inner, vocab, rank, d, bits, seed=1, group=32, scaling=2.0, device="cuda"):
    """`extract` through a whole decoder layer (random weights, adapters merged into them): every one of its projections is adapted.

        y = x + attention(q, k, v) Wo^T,  [q k v] = norm(x) Wqkv^T;   z = y + ffn(norm(y));   logits = norm(z) head^T

    The loss's gradient goes back through the head, the normalisations, the feed-forward block and attention; at each projection it meets the
    8-bit checkpoint of the projection's input, and the rows of all adapters side by side are projected and quantised. Returns the inputs, every
    intermediate result and the milliseconds of each library call."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    def rand(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device=device) * scale).to(torch.bfloat16)
    head_dim = width // heads
    cuts = torch.randint(0, tokens + 1, (n - 1,), generator=g, device=device).sort().values.cpu()
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([tokens])])
    sizes = dict(qkv=(width, (heads + 2 * kv_heads) * head_dim), o=(width, width), gate=(width, inner), up=(width, inner), down=(inner, width))
    w = {k: rand(o, i, scale=i ** -0.5) for k, (i, o) in sizes.items()}
    a = {k: rand(rank, i, scale=i ** -0.5) for k, (i, o) in sizes.items()}
    b = {k: rand(o, rank, scale=0.05) for k, (i, o) in sizes.items()}
    norms = [(1.0 + 0.1 * torch.randn(width, generator=g, device=device)).to(torch.bfloat16) for _ in range(3)]
    head = rand(vocab, width, scale=2.0 * width ** -0.5)
    x = rand(tokens, width)
    labels = torch.randint(0, vocab, (tokens,), generator=g, device=device)
    token_weight = torch.zeros(tokens, device=device)
    for e in range(n):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        answer = lo + (hi - lo) // 2
        labels[lo:answer] = -100
        token_weight[answer:hi] = 1.0 / max(hi - answer, 1)

    ms = {}
    def timed(name, fn):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        out = fn()
        end.record()
        end.synchronize()
        ms[name] = ms.get(name, 0.0) + start.elapsed_time(end)
        return out
    def keep(t):
        return timed("qless_activation_quantize", lambda: B.qless_activation_quantize(t, group=group))
    def norm(t, i):
        return timed("qless_layer_norm", lambda: B.qless_layer_norm(t, norms[i], center=False))
    def norm_back(dy, t, i, kept):
        return timed("qless_layer_norm_backward", lambda: B.qless_layer_norm_backward(dy, t, norms[i], None, kept["rstd"]))["grad_x"]
    saved = {}
    n1 = norm(x, 0)
    saved["qkv"] = keep(n1["out"])
    qkv = n1["out"] @ w["qkv"].T
    q, k, v = qkv.split([heads * head_dim, kv_heads * head_dim, kv_heads * head_dim], dim=1)
    q, k, v = q.unflatten(1, (heads, head_dim)), k.unflatten(1, (kv_heads, head_dim)), v.unflatten(1, (kv_heads, head_dim))
    att = timed("qless_attention", lambda: B.qless_attention(q, k, v, offsets))
    mixed = att["out"].flatten(1)
    saved["o"] = keep(mixed)
    y = x + mixed @ w["o"].T
    n2 = norm(y, 1)
    saved["gate"] = saved["up"] = keep(n2["out"])
    ffn = timed("qless_gated_ffn", lambda: B.qless_gated_ffn(n2["out"], w["gate"], w["up"], w["down"], want_saved=True))
    saved["down"] = keep(ffn["hidden"])
    z = y + ffn["out"]
    n3 = norm(z, 2)
    loss = timed("qless_lm_loss", lambda: B.qless_lm_loss(n3["out"], head, labels, token_weight=token_weight))

    at = {}                                                  # gradients at the projections' outputs
    dz = norm_back(loss["grad_hidden"], z, 2, n3)
    at["down"] = dz
    back = timed("qless_gated_ffn_backward", lambda: B.qless_gated_ffn_backward(dz, None, ffn["gate"], ffn["up"], w["gate"], w["up"], w["down"]))
    at["gate"], at["up"] = back["grad_gate"], back["grad_up"]
    dy = dz + norm_back(back["grad_x"], y, 1, n2)
    at["o"] = dy
    dmixed = (dy @ w["o"]).unflatten(1, (heads, head_dim))
    at["qkv"] = torch.empty_like(qkv)
    dq, dk, dv = at["qkv"].split([heads * head_dim, kv_heads * head_dim, kv_heads * head_dim], dim=1)
    timed("qless_attention_backward", lambda: B.qless_attention_backward(
        dmixed, q, k, v, att["out"], att["lse"], offsets,
        grads=dict(grad_q=dq.unflatten(1, (heads, head_dim)), grad_k=dk.unflatten(1, (kv_heads, head_dim)), grad_v=dv.unflatten(1, (kv_heads, head_dim)))))
    dx = dy + norm_back(at["qkv"] @ w["qkv"], x, 0, n1)

    grads = torch.empty((n, sum(rank * (i + o) for i, o in sizes.values())), dtype=torch.bfloat16, device=device)
    column = 0
    places = {}
    for name, (i, o) in sizes.items():
        places[name] = slice(column, column + rank * (i + o))
        column += rank * (i + o)
        timed("qless_lora_gradients", lambda: B.qless_lora_gradients(*saved[name], at[name], a[name], b[name], offsets, scaling=scaling, group=group,
                                                                    grads=grads[:, places[name]]))
    store = timed("qless_project_quantize", lambda: B.qless_project_quantize(grads, d, 7, bits))
    B.qless_check()
    return dict(offsets=offsets, x=x, w=w, a=a, b=b, norms=norms, head=head, labels=labels, token_weight=token_weight, scaling=scaling, group=group, heads=heads,
                kv_heads=kv_heads, checkpoints=saved, loss=loss, at=at, grad_x=dx, grads=grads, places=places, store=store, ms=ms)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("stage", choices=["project", "quantize", "score", "select", "extract", "layer"])
    ap.add_argument("--tokens", type=int, default=16384)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--rank", type=int, default=16)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--inner", type=int, default=5632)
    ap.add_argument("--n", type=int, default=256)
    ap.add_argument("--N", type=int, default=20000)
    ap.add_argument("--V", type=int, default=448)
    ap.add_argument("--C", type=int, default=4)
    ap.add_argument("--P", type=int, default=1 << 20)
    ap.add_argument("--d", type=int, default=8192)
    ap.add_argument("--bits", type=int, default=4)
    ap.add_argument("--frac", type=float, default=0.05)
    ap.add_argument("--iters", type=int, default=3)
    ap.add_argument("--no-adam", action="store_true")
    ap.add_argument("--matrix", choices=["rademacher", "gaussian"], default="rademacher", help="random matrix of the projection")
    a = ap.parse_args()
    dev = "cuda"
    if a.stage in ("extract", "layer"):
        for _ in range(a.iters):
            got = extract(a.n, a.tokens, a.width, a.vocab, a.rank, a.d, a.bits) if a.stage == "extract" else layer(
                a.n, a.tokens, a.width, a.heads, a.kv_heads, a.inner, a.vocab, a.rank, a.d, a.bits)
        kept = int((got["labels"] >= 0).sum())
        print(f"{a.stage}: {a.n} examples, {a.tokens} tokens ({kept} with a loss), mean loss {got['loss']['loss'].sum().item() / max(kept, 1):.4f}, "
              f"{got['grads'].shape[1]} gradient entries each; " + ", ".join(f"{k} {v:.3f} ms" for k, v in got["ms"].items()))
        return
    if a.stage == "project":
        matrix = B.GAUSSIAN if a.matrix == "gaussian" else B.RADEMACHER
        g = W.student_t_gradients(a.n, a.P, seed=1, device=dev, dtype=torch.bfloat16)
        m, v = (None, None) if a.no_adam else W.adam_moments(a.P, seed=2, device=dev)
        ws = torch.empty(B.qless_project_quantize_workspace(a.n, a.P, a.d, a.bits), dtype=torch.uint8, device=dev)
        fn = lambda: B.qless_project_quantize(g, a.d, 7, a.bits, m, v, workspace=ws, matrix=matrix)
    elif a.stage == "quantize":
        x = torch.randn((a.n, a.d), device=dev)
        fn = lambda: B.qless_quantize(x, a.bits)
    elif a.stage == "score":
        sizes = [64, 128, 256] if a.V == 448 else [a.V]
        off = W.task_offsets(sizes).tolist()
        eta = [1.0, 0.75, 0.5, 0.25, 0.2, 0.1, 0.05, 0.01][:a.C]
        sc = torch.empty(a.N, device=dev)
        if a.bits == 16:
            t16 = torch.empty((a.C, a.N, a.d), dtype=torch.bfloat16, device=dev)
            v16 = torch.empty((a.C, a.V, a.d), dtype=torch.bfloat16, device=dev)
            for i in range(a.C):
                for r0 in range(0, a.N, 8192):
                    r1 = min(a.N, r0 + 8192)
                    t16[i, r0:r1] = W.lowrank_gaussian_features(r1 - r0, a.d, 1, seed=100 + i * 1000 + r0, device=dev)[0].to(torch.bfloat16)
                v16[i] = W.lowrank_gaussian_features(a.V, a.d, 1, seed=5 + i, device=dev)[0].to(torch.bfloat16)
            ws = torch.empty(B.qless_score_16bit_workspace(a.N, a.V, a.C, len(sizes)), dtype=torch.uint8, device=dev)
            tn, vn = B.qless_inv_norms_16bit(t16), B.qless_inv_norms_16bit(v16)
            fn = lambda: B.qless_score_16bit(t16, v16, eta, off, scores=sc, workspace=ws, train_inv_norms=tn, val_inv_norms=vn)
        rb = a.d * min(a.bits, 8) // 8
        tc = torch.empty((a.C, a.N if a.bits != 16 else 1, rb), dtype=torch.uint8, device=dev)
        vc = torch.empty((a.C, a.V, rb), dtype=torch.uint8, device=dev)
        ts = torch.empty((a.C, a.N), device=dev); vs = torch.empty((a.C, a.V), device=dev)
        tss = torch.empty((a.C, a.N), dtype=torch.int32, device=dev); vss = torch.empty((a.C, a.V), dtype=torch.int32, device=dev)
        chunk = 8192
        for i in range(a.C if a.bits != 16 else 0):
            for r0 in range(0, a.N, chunk):
                r1 = min(a.N, r0 + chunk)
                x = W.lowrank_gaussian_features(r1 - r0, a.d, 1, seed=100 + i * 1000 + r0, device=dev)[0]
                tc[i, r0:r1], ts[i, r0:r1], tss[i, r0:r1] = B.qless_quantize(x, a.bits)
            x = W.lowrank_gaussian_features(a.V, a.d, 1, seed=5 + i, device=dev)[0]
            vc[i], vs[i], vss[i] = B.qless_quantize(x, a.bits)
        if a.bits != 16:
            ws = torch.empty(B.qless_score_workspace(a.N, a.V, a.C, len(sizes), a.d, a.bits), dtype=torch.uint8, device=dev)
            fn = lambda: B.qless_score(tc, vc, ts, vs, eta, off, a.d, a.bits, train_sumsq=tss, val_sumsq=vss, scores=sc, workspace=ws)
    else:
        s = torch.randn(a.N, device=dev)
        idx = torch.empty(a.N, dtype=torch.int64, device=dev)
        ws = torch.empty(B.qless_select_topk_workspace(a.N), dtype=torch.uint8, device=dev)
        fn = lambda: B.qless_select_topk(s, a.frac, indices=idx, workspace=ws)
    fn()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(a.iters):
        fn()
    e1.record()
    torch.cuda.synchronize()
    B.qless_check()
    print(f"{a.stage}: {e0.elapsed_time(e1) / a.iters:.4f} ms per call")


if __name__ == "__main__":
    main()
