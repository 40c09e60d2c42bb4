"""The large-vocabulary softmax cross entropy and its gradient against a plain 64-bit implementation.

Tolerances. A logit is an fp32 sum of exact products, 16 per tensor-core instruction, each instruction leaving at most two units
in the last place (2^-22) of the sum of the terms' absolute values: E = 2^-22 (width / 16 + 4) max sum |h W|. The loss is a
difference of two such values and of a logarithm computed in fp32: 2 E + 2^-20 (1 + |logsumexp|). A probability then has the
relative error 3 E + 2^-18 and enters the second product rounded to bf16 (2^-8 of the value); that product is summed in fp32
(2^-22 per 16 terms); the result is rounded to bf16 once more. A gradient below 2^-126, the smallest normal number of bf16 and
fp32, may come out as zero."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
STEP = 2.0 ** -22


def _case(T, width, vocab, seed, keep=1.0, spread=0.05, pad=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    hidden = torch.randn((T, width + pad), generator=g, device=DEV).to(torch.bfloat16)[:, :width]
    weight = (torch.randn((vocab, width + pad), generator=g, device=DEV) * spread).to(torch.bfloat16)[:, :width]
    labels = torch.randint(0, vocab, (T,), generator=g, device=DEV)
    drop = torch.rand(T, generator=g, device=DEV) >= keep
    labels[drop] = -100
    tw = torch.rand(T, generator=g, device=DEV) + 0.1
    return hidden, weight, labels, tw


def reference(hidden, weight, labels, tw):
    vocab = weight.shape[0]
    live = (labels >= 0) & (labels < vocab)
    x, w = torch.where(live[:, None], hidden.double(), 0.0), weight.double()
    y = labels.clamp(0, vocab - 1)
    logits = x @ w.T
    lse = torch.logsumexp(logits, dim=1)
    at = torch.arange(len(y), device=DEV)
    p = torch.exp(logits - lse[:, None])
    others = p.clone()
    others[at, y] = 0.0
    apart = logits.clone()
    apart[at, y] = -float("inf")
    # log(1 + others / label): lse - l_y itself has no digits left for a token the model is sure of
    loss = torch.where(live, torch.nn.functional.softplus(torch.logsumexp(apart, dim=1) - logits[at, y], threshold=1e9), 0.0)
    g = others.clone()
    g[at, y] = -others.sum(dim=1)
    factor = torch.where(live, tw.double(), 0.0)[:, None]
    g = g * factor
    E = STEP * (hidden.shape[1] / 16 + 4) * (x.abs() @ w.abs().T).max().item()
    return dict(loss=loss, lse=lse, g=g, x=x, w=w, E=E, grad_hidden=g @ w, mag_h=g.abs() @ w.abs(), grad_weight=g.T @ x, mag_w=g.abs().T @ x.abs())


def check(got, ref, T, vocab, live_only=None):
    E = ref["E"]
    tol = 2 * E + 2.0 ** -20 * (1 + ref["lse"].abs())
    assert ((got["loss"].double() - ref["loss"]).abs() <= tol).all(), float(((got["loss"].double() - ref["loss"]).abs() / tol).max())
    p_err = 2.0 ** -8 + 3 * E + 2.0 ** -18
    for name, mag, k in (("grad_hidden", ref["mag_h"], vocab), ("grad_weight", ref["mag_w"], T)):
        if got[name] is None:
            continue
        tol = mag * (p_err + STEP * (k / 16 + 16)) + ref[name].abs() * 2.0 ** -8 * (1 + 2.0 ** -6) + 2.0 ** -126
        bad = (got[name].double() - ref[name]).abs() > tol
        assert not bad.any(), (name, int(bad.sum()), bad.numel())


SHAPES = [
    (1, 8, 1, 1.0), (1, 64, 2, 1.0), (1, 512, 1000, 1.0), (3, 72, 255, 1.0), (5, 128, 256, 1.0), (7, 136, 257, 0.6), (64, 512, 513, 1.0),
    (129, 264, 1024, 0.7), (257, 200, 4099, 1.0), (300, 1032, 2500, 0.5), (513, 256, 9000, 0.9), (600, 64, 33000, 0.8),
]


@pytest.mark.parametrize("wants", ["none", "hidden", "weight", "both"])
@pytest.mark.parametrize("T,width,vocab,keep", SHAPES)
def test_loss_and_gradients(T, width, vocab, keep, wants):
    case = _case(T, width, vocab, 5, keep, pad=8)
    got = B.qless_lm_loss(*case, want_hidden=wants in ("hidden", "both"), want_weight=wants in ("weight", "both"))
    B.qless_check()
    check(got, reference(*case), T, vocab)
    again = B.qless_lm_loss(*case, want_hidden=wants in ("hidden", "both"), want_weight=wants in ("weight", "both"))
    for k in ("loss", "grad_hidden", "grad_weight"):
        assert got[k] is None or torch.equal(got[k], again[k])


@pytest.mark.parametrize("T,width,vocab,keep", [(5, 2048, 40_000, 1.0), (300, 1024, 40_001, 0.8), (1300, 1024, 9000, 0.9)])
def test_gradient_of_the_hidden_states_in_two_products(T, width, vocab, keep):
    # more columns than one round of tiles, in both orientations of the products (up to 256 tokens the vocabulary's rows are the tile's)
    case = _case(T, width, vocab, 31, keep, spread=0.02)
    got = B.qless_lm_loss(*case)
    B.qless_check()
    check(got, reference(*case), T, vocab)
    again = B.qless_lm_loss(*case)
    assert torch.equal(got["loss"], again["loss"]) and torch.equal(got["grad_hidden"], again["grad_hidden"])


def test_two_products_with_a_row_far_above_its_reference():
    # row 7's largest logit lies more than 64 powers of two above its label's: the pass has to be redone from the true maximum; row 9's
    # label lies as far above everything else, and row 11 holds an infinity
    T, width, vocab = 40, 1024, 40_000
    hidden, weight, labels, tw = _case(T, width, vocab, 37, spread=0.02)
    weight = weight.clone()
    weight[39_000] = hidden[7] * 0.0625
    weight[25_000] = hidden[9] * 0.0625
    labels[7], labels[9] = 3, 25_000
    assert float((hidden[7].double() @ weight[39_000].double()) - (hidden[7].double() @ weight[3].double())) > 64 * 0.6932
    got = B.qless_lm_loss(hidden, weight, labels, tw)
    B.qless_check()
    check(got, reference(hidden, weight, labels, tw), T, vocab)
    bad = hidden.clone()
    bad[11, 0] = float("inf")
    dirty = B.qless_lm_loss(bad, weight, labels, tw)
    keep = torch.arange(T, device=DEV) != 11
    assert torch.equal(dirty["loss"][keep], got["loss"][keep]) and torch.equal(dirty["grad_hidden"][keep], got["grad_hidden"][keep])
    assert not torch.isfinite(dirty["loss"][11])


def test_several_pieces_of_the_vocabulary():
    # 140 000 tokens' capacity (almost all without a loss): a piece holds 7 column tiles, so 5000 columns take three
    T, width, vocab = 140_000, 64, 5000
    hidden, weight, labels, tw = _case(T, width, vocab, 7, 0.005)
    for wants in ((True, False), (True, True)):
        got = B.qless_lm_loss(hidden, weight, labels, tw, want_hidden=wants[0], want_weight=wants[1])
        B.qless_check()
        keep = (labels >= 0).nonzero()[:, 0]
        ref = reference(hidden[keep], weight, labels[keep], tw[keep])
        check(dict(loss=got["loss"][keep], grad_hidden=got["grad_hidden"][keep], grad_weight=got["grad_weight"]), ref, len(keep), vocab)
        rest = labels < 0
        assert (got["loss"][rest] == 0).all() and (got["grad_hidden"][rest] == 0).all()


def test_rows_far_above_their_first_columns():
    # columns 300 and 700 of some rows lie far more than 64 powers of two above the first 256 columns: the reference has to be redone
    T, width, vocab = 40, 128, 1000
    hidden, weight, labels, tw = _case(T, width, vocab, 9)
    weight = weight.clone()
    weight[300] = hidden[3] * 2
    weight[700] = hidden[17]
    labels[3], labels[17], labels[5] = 300, 2, 700
    ref = reference(hidden, weight, labels, tw)
    assert float((hidden[17].double() @ weight[700].double()) - (hidden[17].double() @ weight[:256].double().T).max()) > 64 * 0.6932
    for want_weight in (False, True):
        got = B.qless_lm_loss(hidden, weight, labels, tw, want_weight=want_weight)
        B.qless_check()
        check(got, ref, T, vocab)


def test_a_sure_token_keeps_its_small_gradient():
    # p of the label = 1 - 1e-5 and nearer to 1: the loss and the gradient keep their relative precision
    width, vocab = 64, 600
    hidden = torch.zeros((3, width), device=DEV, dtype=torch.bfloat16)
    weight = (torch.randn((vocab, width), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV) * 0.01).to(torch.bfloat16)
    labels = torch.tensor([10, 300, 599], device=DEV)
    for t, gap in enumerate((18.0, 24.0, 40.0)):
        hidden[t, t] = 1.0
        weight[labels[t], t] = gap
    got = B.qless_lm_loss(hidden, weight, labels)
    ref = reference(hidden, weight, labels, torch.ones(3, device=DEV))
    # (E is of no use here: the logits are sums of few products; each is exact to 2^-22 of 40)
    assert ((got["loss"].double() / ref["loss"] - 1).abs() < 1e-4).all()
    tol = ref["mag_h"] * (2.0 ** -8 + 1e-4) + ref["grad_hidden"].abs() * 2.0 ** -8 * 1.02
    assert ((got["grad_hidden"].double() - ref["grad_hidden"]).abs() <= tol).all()


def test_ignored_rows_may_hold_anything():
    T, width, vocab = 300, 128, 700
    hidden, weight, labels, tw = _case(T, width, vocab, 11, 0.5)
    clean = B.qless_lm_loss(hidden, weight, labels, tw, want_weight=True)
    dirty, twd = hidden.clone(), tw.clone()
    drop = labels < 0
    dirty[drop] = float("nan")
    dirty[drop.nonzero()[0]] = float("inf")
    twd[drop] = float("nan")
    lab = labels.clone()
    lab[drop.nonzero()[1]] = vocab                         # just outside
    lab[drop.nonzero()[2]] = 1 << 40
    got = B.qless_lm_loss(dirty, weight, lab, twd, want_weight=True)
    for k in ("loss", "grad_hidden", "grad_weight"):
        assert torch.equal(got[k], clean[k])
    assert (got["loss"][drop] == 0).all() and (got["grad_hidden"][drop] == 0).all()


def test_no_token_carries_a_loss():
    hidden, weight, labels, tw = _case(70, 64, 500, 13)
    labels[:] = -100
    got = B.qless_lm_loss(hidden, weight, labels, tw, want_weight=True)
    assert not got["loss"].any() and not got["grad_hidden"].any() and not got["grad_weight"].any()
    got = B.qless_lm_loss(hidden[:0], weight, labels[:0], tw[:0], want_weight=True)
    assert got["loss"].numel() == 0 and not got["grad_weight"].any()
    B.qless_check()


def test_a_nan_row_reaches_only_its_own_row():
    hidden, weight, labels, tw = _case(50, 64, 900, 17)
    clean = B.qless_lm_loss(hidden, weight, labels, tw)
    bad = hidden.clone()
    bad[20] = float("nan")
    got = B.qless_lm_loss(bad, weight, labels, tw)
    keep = torch.arange(50, device=DEV) != 20
    assert torch.equal(got["loss"][keep], clean["loss"][keep]) and torch.equal(got["grad_hidden"][keep], clean["grad_hidden"][keep])
    assert torch.isnan(got["loss"][20]) and torch.isnan(got["grad_hidden"][20].float()).all()
    for wants in (dict(want_hidden=False), dict(want_weight=True)):
        assert torch.isnan(B.qless_lm_loss(bad, weight, labels, tw, **wants)["loss"][20])


def test_default_weights_and_strided_outputs():
    T, width, vocab = 90, 72, 800
    hidden, weight, labels, _ = _case(T, width, vocab, 19, 0.8)
    ones = torch.ones(T, device=DEV)
    want = B.qless_lm_loss(hidden, weight, labels, ones, want_weight=True)
    gh = torch.full((T, width + 24), 3.0, dtype=torch.bfloat16, device=DEV)
    gw = torch.full((vocab, width + 8), 3.0, dtype=torch.bfloat16, device=DEV)
    got = B.qless_lm_loss(hidden, weight, labels, out=dict(grad_hidden=gh[:, 8:8 + width], grad_weight=gw[:, :width]))
    assert torch.equal(got["loss"], want["loss"])
    assert torch.equal(gh[:, 8:8 + width], want["grad_hidden"]) and torch.equal(gw[:, :width], want["grad_weight"])
    assert (gh[:, :8] == 3).all() and (gh[:, 8 + width:] == 3).all() and (gw[:, width:] == 3).all()


def test_gradients_are_those_of_differences():
    # f = sum_t w_t loss_t in 64 bits; central differences of single entries with step 1e-4 (third-order error about 1e-8)
    T, width, vocab = 12, 16, 300
    hidden, weight, labels, tw = _case(T, width, vocab, 23, 0.8, spread=0.3)
    got = B.qless_lm_loss(hidden, weight, labels, tw, want_weight=True)
    f = lambda h, w: (tw.double() * reference(h, w, labels, tw)["loss"]).sum().item()
    h, w = hidden.double(), weight.double()
    top_h, top_w = got["grad_hidden"].double().abs().max().item(), got["grad_weight"].double().abs().max().item()
    step = 1e-4
    for t, c in ((0, 0), (3, 5), (7, 15), (11, 8)):
        d = torch.zeros_like(h)
        d[t, c] = step
        assert abs((f(h + d, w) - f(h - d, w)) / (2 * step) - got["grad_hidden"][t, c].item()) <= 2.0 ** -6 * top_h
    for v, c in ((0, 0), (int(labels.max()), 3), (150, 7), (299, 15)):
        d = torch.zeros_like(w)
        d[v, c] = step
        assert abs((f(h, w + d) - f(h, w - d)) / (2 * step) - got["grad_weight"][v, c].item()) <= 2.0 ** -6 * top_w


def test_on_another_stream():
    case = _case(200, 256, 3000, 29, 0.7)
    want = B.qless_lm_loss(*case)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    out = dict(loss=torch.empty_like(want["loss"]), grad_hidden=torch.empty_like(want["grad_hidden"]))
    ws = torch.empty(B.qless_lm_loss_workspace(200, 256, 3000), dtype=torch.uint8, device=DEV)
    B.qless_lm_loss(*case, out=out, workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(out["loss"], want["loss"]) and torch.equal(out["grad_hidden"], want["grad_hidden"])


@pytest.mark.parametrize("T,keep", [(256, 1.0), (300, 1.0), (1100, 0.5), (140_000, 0.003)])
def test_a_second_pass_at_every_layout(T, keep):
    # a row far above its label, in either orientation of the products and with one or several pieces of the vocabulary (the last: three)
    width, vocab = 128, 5000
    hidden, weight, labels, tw = _case(T, width, vocab, 41, keep)
    live = (labels >= 0).nonzero()[:, 0]
    a, b, c = (int(live[i]) for i in (0, len(live) // 2, -1))
    weight = weight.clone()
    weight[4990] = hidden[a]
    weight[10] = hidden[c]
    labels[a], labels[b], labels[c] = 7, 4990, 4991
    assert float(hidden[a].double() @ (weight[4990] - weight[7]).double()) > 64 * 0.6932
    got = B.qless_lm_loss(hidden, weight, labels, tw)
    B.qless_check()
    ref = reference(hidden[live], weight, labels[live], tw[live])
    check(dict(loss=got["loss"][live], grad_hidden=got["grad_hidden"][live], grad_weight=None), ref, len(live), vocab)
    again = B.qless_lm_loss(hidden, weight, labels, tw)
    assert torch.equal(got["loss"], again["loss"]) and torch.equal(got["grad_hidden"], again["grad_hidden"])
    # and a call that needs none, after one that did
    plain = _case(T, width, vocab, 43, keep)
    live = (plain[2] >= 0).nonzero()[:, 0]
    got = B.qless_lm_loss(*plain)
    check(dict(loss=got["loss"][live], grad_hidden=got["grad_hidden"][live], grad_weight=None),
          reference(plain[0][live], plain[1], plain[2][live], plain[3][live]), len(live), vocab)


@pytest.mark.parametrize("T,wants", [(3, (True, True)), (40, (False, True)), (5, (True, False))])
def test_few_tokens_over_a_vocabulary_of_several_pieces(T, wants):
    # up to 256 tokens a piece holds 2^20 columns
    width, vocab = 16, (1 << 20) + 1000
    hidden, weight, labels, tw = _case(T, width, vocab, 47)
    labels[0], labels[1], labels[2] = vocab - 1, (1 << 20) - 1, 1 << 20
    got = B.qless_lm_loss(hidden, weight, labels, tw, want_hidden=wants[0], want_weight=wants[1])
    B.qless_check()
    check(got, reference(hidden, weight, labels, tw), T, vocab)
