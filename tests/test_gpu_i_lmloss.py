"""GPU tests of the language-model loss (softmax cross entropy over a vocabulary, logits never kept) and its
gradients against a plain fp64 implementation written here.

Tolerances, with A[t] = max_v sum_d |h_td w_vd| (what bounds a logit's rounding error):
* a logit is an fp32 sum of exact products: 1e-5 A (the class of the library's other fp32 sums); lse and loss carry
  one and two of those, and 1e-6 |lse| for the exponentials and the logarithm;
* G = dloss (p - onehot): relative error of p from the logits, e = 2e-5 A + 2e-6 (1 + |lse|), plus the rounding of the
  bf16 operand, 2^-8 |G| (half a unit at 8 significant bits);
* dH, dW: those errors through the product, 1e-5 of the sum of |terms| for the fp32 sums, 2^-8 of the result for its
  own rounding to bf16.
"""
import ctypes as C

import pytest
import torch

from paper_2411_11038_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return B.Context(0)


def make(T, V, D, seed, ignore=0.2, std=3.0):
    g = torch.Generator().manual_seed(seed)
    H = torch.randn((T, D), generator=g).to(torch.bfloat16).cuda()
    W = (torch.randn((V, D), generator=g) * (std / D ** 0.5)).to(torch.bfloat16).cuda()
    labels = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    labels[torch.rand((T,), generator=g) < ignore] = -1
    dloss = torch.randn((T,), generator=g)
    return H, W, labels.cuda(), dloss.cuda()


def reference(H, W, labels, dloss):
    """fp64 values and the bounds stated above."""
    h, w = H.double(), W.double()
    live = labels >= 0
    d = torch.where(live, dloss.double(), 0.0)[:, None]
    h = torch.where(live[:, None], h, 0.0)                  # a token without a target takes no part
    z = h @ w.t()
    a = (h.abs() @ w.abs().t()).amax(dim=1)
    lse = torch.logsumexp(z, dim=1)
    at = labels.long().clamp(min=0)[:, None]
    loss = torch.where(live, lse - z.gather(1, at)[:, 0], 0.0)
    p = torch.softmax(z, dim=1)
    G = p * d
    G.scatter_add_(1, at, -d)
    e = (2e-5 * a + 2e-6 * (1 + lse.abs()))[:, None]
    Gerr = e * p * d.abs() + 2.0 ** -8 * G.abs()
    dH, dW = G @ w, G.t() @ h
    tolH = Gerr @ w.abs() + 1e-5 * (G.abs() @ w.abs()) + 2.0 ** -8 * dH.abs()
    tolW = Gerr.t() @ h.abs() + 1e-5 * (G.abs().t() @ h.abs()) + 2.0 ** -8 * dW.abs()
    return dict(lse=lse, loss=loss, dH=dH, dW=dW, tol_lse=1e-5 * a + 1e-6 * lse.abs(),
                tol_loss=2e-5 * a + 1e-6 * lse.abs(), tolH=tolH, tolW=tolW)


def within(got, ref, tol):
    err = (got.double() - ref).abs()
    over = (err - tol).max()
    assert torch.isfinite(got.double()).all() and float(over) <= 0, (float(over), float(err.max()))


def check(ctx, T, V, D, seed, **kw):
    H, W, labels, dloss = make(T, V, D, seed, **kw)
    plan = B.LmLossPlan(ctx, T, V, D, "cuda")
    loss = plan.fwd(H, W, labels)
    r = reference(H, W, labels, dloss)
    live = labels >= 0
    within(loss, r["loss"], r["tol_loss"])
    within(plan.lse[live], r["lse"][live], r["tol_lse"][live])
    plan.dH.fill_(7), plan.dW.fill_(7)
    out = plan.bwd(H, W, labels, dloss)
    within(out["dH"], r["dH"], r["tolH"])
    within(out["dW"], r["dW"], r["tolW"])
    assert float(out["dH"][~live].abs().sum()) == 0
    again = [t.clone() for t in (loss, plan.lse, out["dH"], out["dW"])]
    plan.fwd(H, W, labels)
    plan.bwd(H, W, labels, dloss)
    for a, b in zip(again, (plan.loss, plan.lse, plan.dH, plan.dW)):
        assert torch.equal(a, b)                              # fixed order of every sum
    assert ctx.device_status() == 0


@pytest.mark.parametrize("T,V,D", [
    (1, 5, 8), (1, 1000, 256), (2, 33, 72), (3, 257, 64), (17, 300, 1000), (127, 513, 128), (128, 512, 64),
    (129, 1003, 264), (200, 2049, 1000), (256, 256, 256), (257, 7001, 768), (500, 4099, 136), (1024, 3001, 520),
    (64, 50259, 64)])
def test_loss_and_gradients(ctx, T, V, D):
    check(ctx, T, V, D, T + V + D)


@pytest.mark.parametrize("T,V,D", [(130, 700, 1032), (300, 999, 2056), (9, 33, 1096), (520, 3001, 4096), (64, 300, 9000)])
def test_long_contractions(ctx, T, V, D):
    """Logits that are summed in segments of at most 1024 columns: two to nine of them, the last one shorter."""
    check(ctx, T, V, D, T + D)


@pytest.mark.parametrize("V,D", [(1, 8), (3, 24), (4, 512), (31, 520), (32000, 1024), (50259, 1000), (9001, 16),
                                 (700, 20480), (700, 20488)])
def test_one_token(ctx, V, D):
    """A single token: rows of W shorter and longer than a warp's step, not a multiple of 32 bytes, and hidden states
    on both sides of the length that a block keeps in shared memory."""
    check(ctx, 1, V, D, V + D, ignore=0.0)


def test_one_token_offset_and_nan(ctx):
    """The same weights at an address that is a multiple of 16 but not of 32 bytes; a NaN in a row of W."""
    V, D = 5003, 256
    H, W, labels, _ = make(1, V, D, 4, ignore=0.0)
    flat = torch.zeros(V * D + 16, dtype=torch.bfloat16, device="cuda")
    odd = flat[8:8 + V * D].view(V, D)
    odd.copy_(W)
    assert odd.data_ptr() % 32 == 16
    plan = B.LmLossPlan(ctx, 1, V, D, "cuda", backward=False)
    want = plan.fwd(H, W, labels).clone()
    assert torch.equal(plan.fwd(H, odd, labels), want)
    W[4999, 17] = float("nan")
    assert torch.isnan(plan.fwd(H, W, labels)).all() and torch.isnan(plan.lse).all()
    assert ctx.device_status() == 0


@pytest.mark.parametrize("T,V,D", [(16, 9001, 1032), (260, 9001, 768), (580, 3001, 520), (1100, 5001, 200)])
def test_slabs_joined(ctx, T, V, D):
    """dH from many slabs of its contraction over the vocabulary, joined by 8, 4, 2 and 1 threads per column."""
    check(ctx, T, V, D, T + 1)


def test_several_pieces_of_the_vocabulary(ctx):
    """A vocabulary that takes three pieces of G (256 MiB each at most), the last one narrower."""
    T, V, D = 12288, 30001, 72
    assert B.lm_loss_workspace_bytes(T, V, D)[1] < T * V * 2
    check(ctx, T, V, D, 3)


def test_confident_and_flat_logits(ctx):
    """Logits spread over +-100 (one exponential dominates, others underflow) and all equal (lse = log V)."""
    check(ctx, 130, 1500, 128, 1, std=30.0)
    H, W, labels, dloss = make(130, 1500, 128, 2)
    W.zero_()
    plan = B.LmLossPlan(ctx, 130, 1500, 128, "cuda")
    loss = plan.fwd(H, W, labels)
    want = torch.where(labels >= 0, torch.log(torch.tensor(1500.0, dtype=torch.float64)).item(), 0.0)
    assert float((loss.double() - want).abs().max()) <= 1e-6 * 8


def test_tokens_without_a_target(ctx):
    """No target at all, one target only, and NaN or infinity in the hidden states that have none."""
    T, V, D = 300, 700, 136
    H, W, labels, dloss = make(T, V, D, 5)
    plan = B.LmLossPlan(ctx, T, V, D, "cuda")
    none = torch.full_like(labels, -100)
    assert float(plan.fwd(H, W, none).abs().max()) == 0 and torch.isfinite(plan.lse).all()
    plan.dH.fill_(7), plan.dW.fill_(7)
    out = plan.bwd(H, W, none, dloss)
    assert float(out["dH"].abs().max()) == 0 and float(out["dW"].abs().max()) == 0
    one = none.clone()
    one[211] = 699
    plan.fwd(H, W, one)
    out = plan.bwd(H, W, one, dloss)
    r = reference(H, W, one, dloss)
    within(out["dH"], r["dH"], r["tolH"])
    within(out["dW"], r["dW"], r["tolW"])
    bad = H.clone()
    skipped = torch.nonzero(labels < 0)[:, 0]
    bad[skipped[0]] = float("nan")
    bad[skipped[1]] = float("inf")
    loss = plan.fwd(bad, W, labels)
    r = reference(H, W, labels, dloss)
    within(loss, r["loss"], r["tol_loss"])
    out = plan.bwd(bad, W, labels, dloss)
    within(out["dH"], r["dH"], r["tolH"])
    within(out["dW"], r["dW"], r["tolW"])


def test_upstream_gradients(ctx):
    """dloss of zero, of one common value (the mean over the targets) and over many magnitudes."""
    T, V, D = 260, 900, 128
    H, W, labels, _ = make(T, V, D, 8)
    plan = B.LmLossPlan(ctx, T, V, D, "cuda")
    plan.fwd(H, W, labels)
    out = plan.bwd(H, W, labels, torch.zeros(T, device="cuda"))
    assert float(out["dH"].abs().max()) == 0 and float(out["dW"].abs().max()) == 0
    n = int((labels >= 0).sum())
    g = torch.Generator().manual_seed(3)
    spread = torch.exp(8 * torch.randn((T,), generator=g)).cuda()
    for d in (torch.full((T,), 1.0 / n, device="cuda"), torch.full((T,), 1e-30, device="cuda"), spread):
        out = plan.bwd(H, W, labels, d)
        r = reference(H, W, labels, d)
        within(out["dH"], r["dH"], r["tolH"])
        within(out["dW"], r["dW"], r["tolW"])


def test_non_finite_hidden_states_reach_their_own_loss_only(ctx):
    T, V, D = 140, 600, 64
    H, W, labels, dloss = make(T, V, D, 11, ignore=0.0)
    H[37, 5] = float("nan")
    plan = B.LmLossPlan(ctx, T, V, D, "cuda")
    loss = plan.fwd(H, W, labels)
    assert torch.isnan(loss[37]) and torch.isfinite(torch.cat([loss[:37], loss[38:]])).all()
    out = plan.bwd(H, W, labels, dloss)
    assert torch.isnan(out["dH"][37]).all() and torch.isfinite(out["dH"][:37]).all()
    assert torch.isnan(out["dW"]).any()


def test_gradients_against_differences(ctx):
    """Directional derivatives of sum(dloss * loss) by central differences of the forward.  H and W are multiples of
    the steps, so that H + h d is exact in bf16; curvature of the loss is below 1 / 4 of the squared logit change."""
    T, V, D, h = 96, 515, 64, 2.0 ** -6
    g = torch.Generator().manual_seed(21)
    H = (torch.randint(-64, 65, (T, D), generator=g).float() / 64).cuda()
    W = (torch.randint(-32, 33, (V, D), generator=g).float() / 64).cuda()
    dH = torch.randint(-1, 2, (T, D), generator=g).float().cuda()
    dW = torch.randint(-1, 2, (V, D), generator=g).float().cuda()
    labels = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda()
    up = torch.randn((T,), generator=g).cuda()
    plan = B.LmLossPlan(ctx, T, V, D, "cuda")
    bf = lambda t: t.to(torch.bfloat16)
    value = lambda a, b: float((plan.fwd(bf(a), bf(b), labels).double() * up.double()).sum())
    by_h = (value(H + h * dH, W) - value(H - h * dH, W)) / (2 * h)
    by_w = (value(H, W + h * dW) - value(H, W - h * dW)) / (2 * h)
    plan.fwd(bf(H), bf(W), labels)
    out = plan.bwd(bf(H), bf(W), labels, up)
    for diff, grad, direction in ((by_h, out["dH"], dH), (by_w, out["dW"], dW)):
        size = float((grad.double().abs() * direction.double().abs()).sum())
        assert abs(diff - float((grad.double() * direction.double()).sum())) <= 1e-2 * size


def test_zero_tokens_and_streams(ctx):
    plan = B.LmLossPlan(ctx, 0, 100, 64, "cuda")
    H, W = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((100, 64), dtype=torch.bfloat16, device="cuda")
    labels, d = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    plan.fwd(H, W, labels)
    plan.dW.fill_(3)
    assert float(plan.bwd(H, W, labels, d)["dW"].abs().max()) == 0
    H, W, labels, d = make(200, 900, 64, 4)
    plan = B.LmLossPlan(ctx, 200, 900, 64, "cuda")
    here = [plan.fwd(H, W, labels).clone(), *(t.clone() for t in plan.bwd(H, W, labels, d).values())]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = [plan.fwd(H, W, labels).clone(), *(t.clone() for t in plan.bwd(H, W, labels, d).values())]
    side.synchronize()
    for a, b in zip(here, there):
        assert torch.equal(a, b)


def test_labels_past_the_vocabulary_are_reported(ctx):
    H, W, labels, d = make(64, 200, 64, 6, ignore=0.0)
    plan = B.LmLossPlan(ctx, 64, 200, 64, "cuda")
    labels[5] = 200
    loss = plan.fwd(H, W, labels)
    assert float(loss[5]) == 0 and ctx.device_status() == 2
    out = plan.bwd(H, W, labels, d)
    assert float(out["dH"][5].abs().max()) == 0 and ctx.device_status() == 2
    labels[5] = -1
    r = reference(H, W, labels, d)
    within(out["dW"], r["dW"], r["tolW"])


def test_refusals(ctx):
    lib, h = B.load(), ctx.handle
    T, V, D = 8, 40, 64
    H, W, labels, d = make(T, V, D, 1)
    plan = B.LmLossPlan(ctx, T, V, D, "cuda")
    p = lambda t, off=0: C.c_void_p(t.data_ptr() + off)
    fwd = lambda *a: lib.efqat_lm_loss_fwd(h, *a, None)
    ws = (p(plan.ws), plan.ws.numel())
    assert lib.efqat_lm_loss_fwd(None, p(H), p(W), p(labels), T, V, D, p(plan.loss), p(plan.lse), *ws, None) == -1
    assert fwd(None, p(W), p(labels), T, V, D, p(plan.loss), p(plan.lse), *ws) == -1
    assert fwd(p(H), p(W), None, T, V, D, p(plan.loss), p(plan.lse), *ws) == -1
    assert fwd(p(H), p(W), p(labels), T, 0, D, p(plan.loss), p(plan.lse), *ws) == -2
    assert fwd(p(H), p(W), p(labels), T, V, 60, p(plan.loss), p(plan.lse), *ws) == -3
    assert fwd(p(H, 2), p(W), p(labels), T, V, D, p(plan.loss), p(plan.lse), *ws) == -3
    assert fwd(p(H), p(W), p(labels), T, 1 << 25, D, p(plan.loss), p(plan.lse), *ws) == -11
    assert fwd(p(H), p(W), p(labels), T, V, D, p(plan.loss), p(plan.lse), p(plan.ws), 16) == -7
    bwd = lambda *a: lib.efqat_lm_loss_bwd(h, *a, None)
    args = [p(H), p(W), p(labels), p(plan.lse), p(d), T, V, D, p(plan.dH), p(plan.dW)]
    for i in (0, 1, 2, 3, 4, 8, 9):
        bad = list(args)
        bad[i] = None
        assert bwd(*bad, *ws) == -1
    assert bwd(*args, None, 0) == -7
    with pytest.raises(ValueError):
        plan.fwd(H.float(), W, labels)
    with pytest.raises(ValueError):
        plan.fwd(H, W, labels.long())
    with pytest.raises(ValueError):
        plan.fwd(H, W[:, :32], labels)
    with pytest.raises(B.EfqatError):
        B.LmLossPlan(ctx, T, V, 60, "cuda")
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
