"""8-bit activation checkpoints and the per-example LoRA gradients taken from them, against plain 64-bit implementations.

Tolerances. Codes, step bytes and restored values are exact. A gradient entry is a sum of products that the kernels add in
fp32 on the tensor cores, 16 products per instruction; each instruction may leave an error of two units in the last place
(2^-22) of the largest partial sum, which the sum of the terms' absolute values bounds: STEP * (K / 16 + 4) of that sum for a
contraction of K terms. A bf16 value has 8 significant bits, so rounding to bf16 leaves up to 2^-8 of the value. The factors U and
H enter the second product as sums of bf16 terms: two (bf16 gradients) leave 2^-16 of the factor, three (fp32 gradients) 2^-24;
the result is rounded once to its type."""
import numpy as np
import pytest
import torch

from paper_2502_01703_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
STEP = 2.0 ** -22


def _rand(shape, seed, scale=1.0, dtype=torch.float32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def reference_quantize(x, group):
    """64-bit numpy: codes, step bytes, values."""
    x = x.double().cpu().numpy()
    T, w = x.shape
    G = -(-w // group)
    codes, steps = np.zeros((T, w), np.int8), np.zeros((T, G), np.uint8)
    values = np.zeros((T, w))
    for g in range(G):
        y = x[:, g * group:(g + 1) * group]
        for t in range(T):
            row = y[t]
            if not np.isfinite(row).all():
                steps[t, g], values[t, g * group:(g + 1) * group] = 255, np.nan
                continue
            a, e = np.abs(row).max(), -120
            while a > 127 * 2.0 ** e and e < 121:
                e += 1
            q = np.clip(np.rint(row / 2.0 ** e), -127, 127)
            codes[t, g * group:(g + 1) * group] = q
            steps[t, g], values[t, g * group:(g + 1) * group] = e + 127, q * 2.0 ** e
    return codes, steps, values


@pytest.mark.parametrize("tokens,width,group,dtype,pad", [
    (1, 1, 32, torch.float32, 0), (1, 33, 32, torch.bfloat16, 0), (3, 256, 32, torch.float32, 0), (5, 257, 64, torch.bfloat16, 7),
    (4, 512, 128, torch.bfloat16, 8), (7, 1000, 64, torch.float32, 8), (130, 304, 128, torch.float32, 3), (9, 4112, 32, torch.bfloat16, 16),
])
def test_checkpoint_codes_and_values_are_exact(tokens, width, group, dtype, pad):
    big = _rand((tokens, width + pad), 3, dtype=dtype)
    x = big[:, :width]
    if tokens > 2:
        x[1] = 0.0                                  # a token of zeros
        x[2] *= 2.0 ** -100
    if tokens > 4:
        x[3, ::7] *= 1000.0
        x[4, 0] = 127.0                             # exactly 127 steps of size one
        x[4, 1] = 0.5                               # and a tie
    cbuf = torch.full((tokens, width + pad), 77, dtype=torch.int8, device=DEV)
    codes, scales = B.qless_activation_quantize(x, group=group, codes=cbuf[:, :width])
    want_c, want_s, want_v = reference_quantize(x, group)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert (cbuf[:, width:] == 77).all()
    for out_type in (torch.float32, torch.bfloat16):
        out = torch.full((tokens, width + pad), 5.0, dtype=out_type, device=DEV)
        B.qless_activation_dequantize(codes, scales, group=group, out=out[:, :width])
        assert np.array_equal(out[:, :width].double().cpu().numpy(), want_v)      # bf16 holds the values exactly
        assert (out[:, width:] == 5.0).all()


def test_checkpoint_of_extreme_and_non_finite_values():
    x = torch.zeros((6, 96), device=DEV)
    x[0, 5] = float("inf"); x[1, 40] = float("nan"); x[2, 95] = -float("inf")
    x[3, :32] = torch.finfo(torch.float32).max          # above 127 * 2^121: codes saturate at 127
    x[4, :32] = 2.0 ** -140                             # a denormal: below the smallest step
    x[5, 32:64] = 2.0 ** -120
    codes, scales = B.qless_activation_quantize(x, group=32)
    want_c, want_s, want_v = reference_quantize(x, 32)
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
    got = B.qless_activation_dequantize(codes, scales, group=32, dtype=torch.float32).double().cpu().numpy()
    assert np.array_equal(got, want_v, equal_nan=True)
    assert scales[0, 0] == 255 and scales[0, 1] == 7 and np.isnan(got[0, :32]).all() and (got[0, 32:] == 0).all()


def test_checkpoint_error_is_at_most_half_a_step():
    x = _rand((64, 512), 5)
    codes, scales = B.qless_activation_quantize(x, group=32)
    y = B.qless_activation_dequantize(codes, scales, group=32, dtype=torch.float32)
    step = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127).repeat_interleave(32, dim=1)
    assert ((x - y).abs() <= 0.5 * step).all()


def _lora_case(tokens, wi, wo, rank, group, seed, pad=0):
    x = _rand((tokens, wi), seed)
    codes, scales = B.qless_activation_quantize(x, group=group)
    wide_c = torch.zeros((tokens, wi + 2 * pad), dtype=torch.int8, device=DEV)
    wide_c[:, :wi] = codes
    dy = _rand((tokens, wo + pad), seed + 1, 0.1, torch.bfloat16)[:, :wo]
    a, b = _rand((rank, wi), seed + 2, wi ** -0.5, torch.bfloat16), _rand((wo, rank), seed + 3, 0.1, torch.bfloat16)
    return wide_c[:, :wi], scales, dy, a, b


def reference_lora(codes, scales, dy, a, b, offsets, scaling, group):
    """Gradients and, per entry, the sum of the absolute values of what is added up."""
    T, wi = codes.shape
    step = torch.ldexp(torch.ones(scales.shape, dtype=torch.float64, device=DEV), scales.int() - 127)
    step = torch.where(scales == 255, torch.full_like(step, float("nan")), step)
    x = codes.double() * step.repeat_interleave(group, dim=1)[:, :wi]
    dy, a, b = dy.double(), a.double(), b.double()
    rows, mags = [], []
    for e in range(len(offsets) - 1):
        s = slice(offsets[e], offsets[e + 1])
        u, h = scaling * dy[s] @ b, scaling * x[s] @ a.T
        um, hm = abs(scaling) * dy[s].abs() @ b.abs(), abs(scaling) * x[s].abs() @ a.abs().T
        rows.append(torch.cat([(u.T @ x[s]).flatten(), (dy[s].T @ h).flatten()]))
        mags.append(torch.cat([(um.T @ x[s].abs()).flatten(), (dy[s].abs().T @ hm).flatten()]))
    return torch.stack(rows), torch.stack(mags)


def _check_lora(got, want, mag, wi, wo, tokens, dtype):
    k = (max(wi, wo) + tokens) / 16 + 8
    tol = mag * (STEP * k + (2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -24))
    if dtype == torch.bfloat16:
        tol = tol + want.abs() * 2.0 ** -8 * (1 + 2.0 ** -6)
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / (mag + 1e-300)).max()))


LORA = [
    ([0, 1], 16, 16, 8, 32), ([0, 0], 64, 64, 16, 32), ([0, 1, 1, 3], 128, 256, 8, 64), ([0, 64, 128], 256, 128, 16, 128),
    ([0, 63, 64, 129], 272, 144, 24, 32), ([0, 5, 5, 70, 200], 512, 512, 64, 32), ([0, 130], 528, 1040, 40, 64),
    ([0, 17, 200], 384, 640, 128, 128), ([0, 90, 161], 192, 320, 32, 32), ([0, 90, 161], 192, 320, 48, 64), ([0, 71, 161], 256, 128, 96, 32), ([0, 300], 4096, 256, 64, 64), ([0, 0, 0, 0, 1], 1024, 16, 32, 128),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offsets,wi,wo,rank,group", LORA)
def test_lora_gradients(offsets, wi, wo, rank, group, dtype):
    T = max(offsets[-1], 1)
    case = _lora_case(T, wi, wo, rank, group, 11, pad=16)
    got = B.qless_lora_gradients(*case, offsets, scaling=1.75, group=group, dtype=dtype)
    want, mag = reference_lora(*case, offsets, 1.75, group)
    B.qless_check()
    _check_lora(got, want, mag, wi, wo, T, dtype)
    again = B.qless_lora_gradients(*case, offsets, scaling=1.75, group=group, dtype=dtype)
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lora_gradients_of_examples_longer_than_a_piece(dtype):
    # few channels: pieces of 512 tokens; examples of 1500 (three pieces), 3, 512 (one) and 600 tokens (two)
    offsets = [2, 1502, 1505, 2017, 2617]
    case = _lora_case(2700, 256, 512, 16, 32, 21)
    got = B.qless_lora_gradients(*case, offsets, scaling=2.0, group=32, dtype=dtype)
    want, mag = reference_lora(*case, offsets, 2.0, 32)
    B.qless_check()
    _check_lora(got, want, mag, 256, 512, 1500, dtype)


def test_lora_gradients_of_many_examples():
    # more table entries than one upload launch takes
    g = np.random.default_rng(3)
    offsets = np.concatenate([[0], np.cumsum(g.integers(0, 9, 700))]).tolist()
    case = _lora_case(offsets[-1], 64, 96, 8, 64, 31)
    got = B.qless_lora_gradients(*case, offsets, group=64, dtype=torch.float32)
    want, mag = reference_lora(*case, offsets, 1.0, 64)
    _check_lora(got, want, mag, 64, 96, 9, torch.float32)


def test_lora_gradients_of_more_tiles_than_multiprocessors():
    # every block of the grid works through several tiles of both kinds, with pieces of one to several 64-token blocks
    g = np.random.default_rng(5)
    offsets = np.concatenate([[0], np.cumsum(g.integers(1, 1200, 40))]).tolist()
    T, wi, wo, rank = offsets[-1], 528, 1296, 16
    case = _lora_case(T, wi, wo, rank, 32, 81)
    got = B.qless_lora_gradients(*case, offsets, group=32, dtype=torch.float32)
    want, mag = reference_lora(*case, offsets, 1.0, 32)
    B.qless_check()
    _check_lora(got, want, mag, wi, wo, 1200, torch.float32)


def test_lora_gradients_into_a_slice_of_the_gradient_matrix():
    offsets, wi, wo, rank = [0, 70, 71, 200], 128, 256, 16
    P = rank * (wi + wo)
    case = _lora_case(200, wi, wo, rank, 32, 41)
    wide = torch.full((3, 2 * P + 128), 9.0, dtype=torch.bfloat16, device=DEV)
    B.qless_lora_gradients(*case, offsets, group=32, grads=wide[:, 64:64 + P])
    assert torch.equal(wide[:, 64:64 + P], B.qless_lora_gradients(*case, offsets, group=32))
    assert (wide[:, :64] == 9.0).all() and (wide[:, 64 + P:] == 9.0).all()


@pytest.mark.parametrize("where", ["codes", "grad_out"])
def test_a_nan_stays_in_its_example(where):
    offsets, wi, wo, rank = [0, 37, 100, 230], 256, 384, 24
    codes, scales, dy, a, b = _lora_case(230, wi, wo, rank, 32, 51)
    clean = B.qless_lora_gradients(codes, scales, dy, a, b, offsets, group=32)
    if where == "codes":
        scales = scales.clone()
        scales[37:100] = 255
    else:
        dy = dy.clone()
        dy[37:100] = float("nan")
    got = B.qless_lora_gradients(codes, scales, dy, a, b, offsets, group=32)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2])
    assert torch.isnan(got[1].float()).all()


def test_lora_gradients_are_those_of_differences():
    # f(A, B) = sum_t <dY_t, s B A x_t> in 64 bits: central differences (f is bilinear, so they are exact up to rounding)
    T, wi, wo, rank, s = 50, 64, 48, 8, 0.5
    codes, scales, dy, a, b = _lora_case(T, wi, wo, rank, 32, 61)
    got = B.qless_lora_gradients(codes, scales, dy, a, b, [0, T], scaling=s, group=32, dtype=torch.float32)[0].double().cpu()
    x = B.qless_activation_dequantize(codes, scales, group=32, dtype=torch.float32).double().cpu()
    dy, a, b = dy.double().cpu(), a.double().cpu(), b.double().cpu()
    f = lambda a_, b_: (dy * (s * x @ a_.T @ b_.T)).sum()
    scale_a, scale_b = got[:rank * wi].abs().max(), got[rank * wi:].abs().max()
    for k in range(0, rank * wi, 37):
        d = torch.zeros(rank * wi, dtype=torch.float64)
        d[k] = 1e-3
        d = d.view(rank, wi)
        assert abs((f(a + d, b) - f(a - d, b)) / 2e-3 - got[k]) <= 1e-5 * scale_a
    for k in range(0, wo * rank, 29):
        d = torch.zeros(wo * rank, dtype=torch.float64)
        d[k] = 1e-3
        d = d.view(wo, rank)
        assert abs((f(a, b + d) - f(a, b - d)) / 2e-3 - got[rank * wi + k]) <= 1e-5 * scale_b


def test_lora_gradients_on_another_stream():
    offsets, wi, wo, rank = [0, 100, 333], 512, 256, 32
    case = _lora_case(333, wi, wo, rank, 64, 71)
    want = B.qless_lora_gradients(*case, offsets, group=64)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = torch.empty_like(want)
    ws = torch.empty(B.qless_lora_gradients_workspace(333, 2, wi, wo, rank), dtype=torch.uint8, device=DEV)
    B.qless_lora_gradients(*case, offsets, group=64, grads=got, workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(got, want)


# An fp32 sum is taken in accumulators of at most 512 channels or tokens: 32 steps of 16, each of which cuts the running sum's last bits by
# half a unit (2^-24 of it) on average, one way; a sum of random signs is on average at 2/3 of its end: 32 * 2^-24 * 2/3 = 1.3e-6 a product,
# two products in a row. Above 64 columns the three terms share accumulators of 256 tokens: 48 steps, 1.9e-6. Sums taken whole would
# have three to eight times as many steps here.
@pytest.mark.parametrize("offsets,wi,wo,rank,bound", [
    ([0, 7000, 7001, 14300], 4096, 2064, 16, 2.6e-6),            # one slice, eight accumulators a factor, pieces of 1216 tokens
    ([0, 2000, 6000], 4096, 4112, 48, 2.6e-6),                   # slices of the channels, terms of 64 columns
    ([0, 1100, 4100], 1040, 528, 128, 3.2e-6),
    ([3, 515, 516, 1029], 640, 512, 64, 2.6e-6),                 # one token behind an accumulator's last
])
def test_fp32_lora_gradients_do_not_lose_digits_with_length(offsets, wi, wo, rank, bound):
    case = _lora_case(offsets[-1] + 5, wi, wo, rank, 32, 91)
    got = B.qless_lora_gradients(*case, offsets, scaling=0.5, group=32, dtype=torch.float32)
    want, mag = reference_lora(*case, offsets, 0.5, 32)
    B.qless_check()
    _check_lora(got, want, mag, wi, wo, max(b - a for a, b in zip(offsets, offsets[1:])), torch.float32)
    for part in (slice(0, rank * wi), slice(rank * wi, None)):
        for e in range(len(offsets) - 1):
            w = want[e, part].double()
            assert (got[e, part].double() - w.to(got.device)).norm() <= bound * w.norm().to(got.device)
    assert torch.equal(got, B.qless_lora_gradients(*case, offsets, scaling=0.5, group=32, dtype=torch.float32))
