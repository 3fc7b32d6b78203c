"""GPU tests of the row operators around the quantized layers: 8-bit activation checkpoints, GELU and layer norm,
each against a plain fp64 implementation written here, with their edge values, their refusals and finite differences.

Tolerances (u = 2^-24, the relative rounding error of fp32):
* checkpoint codes, scales and decoded fp32 values: the definition fixes every rounding, so bit-exact;
* GELU: erf's approximation is within 1.5e-7 and its terms carry a few roundings: 6e-7 max(1, |x|) on y (16 u on
  Phi would be 9.5e-7), 1e-6 |dY| max(1, |x|) on dX;
* layer norm: sums of C terms by a tree of depth <= 64 sums per lane, i.e. at most 64 u of the sum of |terms|:
  4e-6 of the terms' magnitudes on y, 1e-5 on dX, 1e-5 of the sum of |terms| on dgamma and dbeta (the class of the
  library's other fp32 reductions);
* half a unit of bf16 (8 significant bits: 2^-8 |value|), on top wherever the output is bf16.
"""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2411_11038_b200 import binding as B

pytestmark = pytest.mark.gpu

DT = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def ctx():
    return B.Context(0)


def f64(t):
    return t.detach().double().cpu().numpy()


def out_ulp(dtype, ref):
    return (2.0 ** -8) * np.abs(ref) if dtype == torch.bfloat16 else 0.0


def within(got, ref, tol):
    err = np.abs(got - ref)
    assert np.all(err <= tol), (float(np.max(err - tol)), float(err.max()))


def draw(M, Cn, dtype, seed, mean=0.3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, Cn), generator=g) * torch.exp(0.5 * torch.randn((Cn,), generator=g)) + mean
    return x.to(dtype)


# ------------------------------------------------------------------------------------------------ definitions
def ckpt_ref(x64):
    """Codes, scales and decoded values of a checkpoint, group by group."""
    M, Cn = x64.shape
    G = -(-Cn // 128)
    codes, scales, vals = np.zeros((M, Cn), np.int8), np.zeros((M, G), np.float32), np.zeros((M, Cn), np.float32)
    for g in range(G):
        cols = slice(g * 128, (g + 1) * 128)
        v = x64[:, cols].astype(np.float32)
        a = np.abs(v).max(axis=1)                                     # NaN wins over every number
        bad, tiny = ~np.isfinite(a), a < np.float32(2.0 ** -100)
        a = np.where(bad | tiny, np.float32(1), a)
        s, f = a / np.float32(127), np.float32(127) / a
        q = np.rint(np.where((bad | tiny)[:, None], np.float32(0), v) * f[:, None])
        s = np.where(bad, np.float32(np.nan), np.where(tiny, np.float32(0), s))
        codes[:, cols], scales[:, g], vals[:, cols] = q.astype(np.int8), s, q.astype(np.float32) * s[:, None]
    return codes, scales, vals


def phi_cdf(x):
    return torch.special.ndtr(torch.from_numpy(x)).numpy()


def gelu_ref(x):
    return x * phi_cdf(x)


def gelu_slope(x):
    return phi_cdf(x) + x * np.exp(-x * x / 2) / np.sqrt(2 * np.pi)


def ln_ref(x, gamma, beta, eps):
    mean = x.mean(axis=1)
    var = ((x - mean[:, None]) ** 2).mean(axis=1)
    rstd = 1 / np.sqrt(var + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    return xh * gamma + (0 if beta is None else beta), mean, rstd, xh


def ln_bwd_ref(dy, xh, gamma, rstd):
    g = dy * gamma
    m1, m2 = g.mean(axis=1, keepdims=True), (g * xh).mean(axis=1, keepdims=True)
    dx = rstd[:, None] * (g - m1 - xh * m2)
    mag = rstd[:, None] * (np.abs(g) + np.abs(g).mean(axis=1, keepdims=True) +
                           np.abs(xh) * np.abs(g * xh).mean(axis=1, keepdims=True))
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0), mag, np.abs(dy * xh).sum(axis=0), np.abs(dy).sum(axis=0)


# ------------------------------------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,Cn", [(1, 16), (1, 128), (3, 144), (33, 1040), (257, 256), (5, 4112), (300, 48)])
def test_ckpt_is_bit_exact(ctx, dtype, M, Cn):
    x = draw(M, Cn, dtype, M * 31 + Cn)
    ck = B.Checkpoint(ctx, M, Cn, "cuda").store(x.cuda())
    codes, scales, vals = ckpt_ref(f64(x))
    assert np.array_equal(ck.codes.cpu().numpy(), codes)
    assert np.array_equal(ck.scales.cpu().numpy(), scales)
    back = ck.load(torch.float32).cpu().numpy()
    assert np.array_equal(back, vals)
    assert torch.equal(ck.load(torch.bfloat16).cpu(), torch.from_numpy(vals).to(torch.bfloat16))
    assert ck.nbytes == M * Cn + 4 * M * (-(-Cn // 128))
    # half a step of the group's scale, the method's own error
    step = np.repeat(scales, 128, axis=1)[:, :Cn]
    assert np.all(np.abs(vals - f64(x)) <= 0.5001 * step)


def test_ckpt_edge_values(ctx):
    """Zero and tiny groups read back as zeros, ties go to the even code, a non-finite value makes its group (and
    only its group) NaN, the largest and the smallest magnitudes survive."""
    x = torch.zeros((8, 256))
    x[1, :128] = 2.0 ** -120                       # tiny: stored as zeros
    x[1, 128:] = 2.0 ** -99                        # just above the limit
    x[2, 0], x[2, 1], x[2, 2], x[2, 3] = 127.0, 0.5, 1.5, -2.5      # scale 1: ties 0, 2, -2
    x[3, 5] = float("inf")
    x[4, 200] = float("nan")
    x[5, 0], x[5, 1] = -3.3e38, 3.3e38
    x[6, 77], x[6, 78] = -float("inf"), float("nan")
    x[7, :] = -1.0
    ck = B.Checkpoint(ctx, 8, 256, "cuda").store(x.cuda())
    codes, scales, vals = ckpt_ref(f64(x))
    assert np.array_equal(ck.codes.cpu().numpy(), codes)
    assert np.array_equal(ck.scales.cpu().numpy(), scales, equal_nan=True)
    got = ck.load(torch.float32).cpu().numpy()
    assert np.array_equal(got, vals, equal_nan=True)
    assert codes[2, :4].tolist() == [127, 0, 2, -2]
    assert np.all(got[1, :128] == 0) and np.all(got[1, 128:] == np.float32(2.0 ** -99))
    assert np.isnan(got[3, :128]).all() and not np.isnan(got[3, 128:]).any()
    assert not np.isnan(got[4, :128]).any() and np.isnan(got[4, 128:]).all()


# ------------------------------------------------------------------------------------------------ GELU
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,Cn", [(1, 8), (1, 16), (7, 136), (61, 1504), (1000, 128), (2, 16400)])
def test_gelu_forward_and_backward(ctx, dtype, M, Cn):
    x, dy = draw(M, Cn, dtype, 5 + M + Cn) * 2, draw(M, Cn, dtype, 6 + M + Cn)
    plan = B.GeluPlan(ctx, M, Cn, dtype, "cuda")
    x64, d64 = f64(x), f64(dy)
    mag = np.maximum(1, np.abs(x64))
    ref = gelu_ref(x64)
    within(f64(plan.fwd(x.cuda())), ref, 6e-7 * mag + out_ulp(dtype, ref))
    ref = d64 * gelu_slope(x64)
    within(f64(plan.bwd(dy.cuda(), x=x.cuda())), ref, 1e-6 * np.abs(d64) * mag + out_ulp(dtype, ref))
    if Cn % 16:
        return
    ck = B.Checkpoint(ctx, M, Cn, "cuda")
    y = plan.fwd(x.cuda(), save=ck).clone()
    assert torch.equal(y, plan.fwd(x.cuda()))                     # saving does not change y
    codes, scales, vals = ckpt_ref(x64)
    assert np.array_equal(ck.codes.cpu().numpy(), codes) and np.array_equal(ck.scales.cpu().numpy(), scales)
    v64 = vals.astype(np.float64)
    mag = np.maximum(1, np.abs(v64))
    ref = d64 * gelu_slope(v64)
    within(f64(plan.bwd(dy.cuda(), saved=ck)), ref, 1e-6 * np.abs(d64) * mag + out_ulp(dtype, ref))
    ref = gelu_ref(v64)
    within(f64(plan.recompute(ck)), ref, 6e-7 * mag + out_ulp(dtype, ref))
    assert ctx.device_status() == 0


def test_gelu_extremes_and_differences(ctx):
    """Far tails, zero, non-finite inputs; and the slope against central differences of the forward."""
    x = torch.tensor([[0.0, -0.0, 40.0, -40.0, 1e30, -1e30, float("inf"), float("nan")]], device="cuda")
    plan = B.GeluPlan(ctx, 1, 8, torch.float32, "cuda")
    y = plan.fwd(x)[0].cpu().numpy()
    assert y[0] == 0 and y[2] == 40 and y[4] == np.float32(1e30) and y[6] == np.inf and np.isnan(y[7])
    assert abs(y[3]) <= 6e-7 * 40 and abs(y[5]) <= 6e-7 * 1e30
    one = torch.ones_like(x)
    d = plan.bwd(one, x=x)[0].cpu().numpy()
    assert abs(d[0] - 0.5) <= 1e-6 and d[2] == 1 and abs(d[3]) <= 1e-6 * 40
    # differences: step 2^-6, curvature |gelu'''| <= 1.5 gives 1.5 h^2 / 6 = 6.1e-5; noise 2 * 3.6e-6 / (2 h) = 2.3e-4
    h = 2.0 ** -6
    t = torch.linspace(-6, 6, 4096, device="cuda").reshape(1, 4096)
    p = B.GeluPlan(ctx, 1, 4096, torch.float32, "cuda")
    up, down = p.fwd(t + h).double().clone(), p.fwd(t - h).double().clone()
    slope = p.bwd(torch.ones_like(t), x=t).double()
    width = (t + h).double() - (t - h).double()
    assert float(((up - down) / width - slope).abs().max()) <= 3e-4


# ------------------------------------------------------------------------------------------------ layer norm
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,Cn", [(1, 8), (1, 768), (2, 256), (3, 264), (333, 520), (37, 1000), (1021, 1024),
                                  (9, 1032), (130, 2056), (64, 4096), (5, 8200), (3, 16384), (700, 64),
                                  (7001, 264), (5000, 1000), (2601, 4096), (1200, 8192), (900, 16384)])
def test_layer_norm_forward_and_backward(ctx, dtype, M, Cn):
    x, dy = draw(M, Cn, dtype, M + Cn, mean=3.0), draw(M, Cn, dtype, 1 + M + Cn)
    g = torch.Generator().manual_seed(M + 7)
    gamma, beta = 1 + 0.2 * torch.randn((Cn,), generator=g), torch.randn((Cn,), generator=g)
    plan = B.LayerNormPlan(ctx, M, Cn, dtype, "cuda", eps=1e-5)
    x64, d64, g64, b64 = f64(x), f64(dy), f64(gamma), f64(beta)
    ref, mean, rstd, xh = ln_ref(x64, g64, b64, 1e-5)
    y = plan.fwd(x.cuda(), gamma.cuda(), beta.cuda())
    reach = np.abs(x64).max(axis=1, keepdims=True) * rstd[:, None]        # magnitude of the terms behind xh
    within(f64(y), ref, 4e-6 * ((reach + np.abs(xh)) * np.abs(g64) + np.abs(b64)) + out_ulp(dtype, ref))
    within(f64(plan.mean), mean, 4e-6 * np.abs(x64).mean(axis=1))
    within(f64(plan.rstd), rstd, 1e-5 * rstd)
    no_beta = f64(plan.fwd(x.cuda(), gamma.cuda()))
    within(no_beta, ref - b64, 4e-6 * (reach + np.abs(xh)) * np.abs(g64) + out_ulp(dtype, ref - b64))
    out = plan.bwd(dy.cuda(), gamma.cuda(), x=x.cuda())
    dx, dg, db, mag, dga, dba = ln_bwd_ref(d64, xh, g64, rstd)
    within(f64(out["dx"]), dx, 1e-5 * mag * (1 + reach) + out_ulp(dtype, dx))
    # xh carries 4e-6 of the row's reach, summed over the rows
    within(f64(out["dgamma"]), dg, 1e-5 * dga + 4e-6 * (np.abs(d64) * reach).sum(axis=0))
    within(f64(out["dbeta"]), db, 1e-5 * dba)
    again = [t.clone() for t in out.values()]
    for t, u in zip(plan.bwd(dy.cuda(), gamma.cuda(), x=x.cuda()).values(), again):
        assert torch.equal(t, u)                                            # fixed order of every sum
    assert ctx.device_status() == 0


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,Cn", [(1, 16), (3, 272), (257, 1024), (31, 1040), (12, 4096), (2, 16384), (9001, 80),
                                  (2601, 4096), (900, 16384)])
def test_layer_norm_from_its_checkpoint(ctx, dtype, M, Cn):
    x, dy = draw(M, Cn, dtype, 3 * M + Cn), draw(M, Cn, dtype, 1 + 3 * M + Cn)
    g = torch.Generator().manual_seed(M + 7)
    gamma, beta = 1 + 0.2 * torch.randn((Cn,), generator=g), torch.randn((Cn,), generator=g)
    plan = B.LayerNormPlan(ctx, M, Cn, dtype, "cuda")
    ck = B.Checkpoint(ctx, M, Cn, "cuda")
    plain = plan.fwd(x.cuda(), gamma.cuda(), beta.cuda()).clone()
    assert torch.equal(plain, plan.fwd(x.cuda(), gamma.cuda(), beta.cuda(), save=ck))
    codes, scales, vals = ckpt_ref(f64(x))
    assert np.array_equal(ck.codes.cpu().numpy(), codes) and np.array_equal(ck.scales.cpu().numpy(), scales)
    g64, b64, d64 = f64(gamma), f64(beta), f64(dy)
    _, mean, rstd, _ = ln_ref(f64(x), g64, b64, 1e-5)
    xh = (vals.astype(np.float64) - mean[:, None]) * rstd[:, None]
    reach = np.abs(f64(x)).max(axis=1, keepdims=True) * rstd[:, None]
    out = plan.bwd(dy.cuda(), gamma.cuda(), saved=ck)
    dx, dg, db, mag, dga, dba = ln_bwd_ref(d64, xh, g64, rstd)
    within(f64(out["dx"]), dx, 1e-5 * mag * (1 + reach) + out_ulp(dtype, dx))
    within(f64(out["dgamma"]), dg, 1e-5 * dga + 4e-6 * (np.abs(d64) * reach).sum(axis=0))
    within(f64(out["dbeta"]), db, 1e-5 * dba)
    ref = xh * g64 + b64
    within(f64(plan.recompute(ck, gamma.cuda(), beta.cuda())), ref,
           4e-6 * ((reach + np.abs(xh)) * np.abs(g64) + np.abs(b64)) + out_ulp(dtype, ref))


def test_layer_norm_backward_against_differences(ctx):
    """Directional derivatives of sum(w * y) in x, gamma and beta by central differences of the forward (fp32 in,
    sums in fp64).  Step 2^-7 on unit-variance rows: truncation about h^2 = 6e-5 relative, noise 4e-6 / h = 5e-4."""
    M, Cn, h = 64, 520, 2.0 ** -7
    x, w = draw(M, Cn, torch.float32, 1).cuda(), draw(M, Cn, torch.float32, 2).cuda()
    dirx = draw(M, Cn, torch.float32, 3, mean=0.0).cuda()
    gamma, beta = draw(1, Cn, torch.float32, 4, mean=1.0)[0].cuda(), draw(1, Cn, torch.float32, 5)[0].cuda()
    dirp = draw(1, Cn, torch.float32, 6)[0].cuda()
    plan = B.LayerNormPlan(ctx, M, Cn, torch.float32, "cuda")

    def value(xx, gg, bb):
        return float((plan.fwd(xx, gg, bb).double() * w.double()).sum())

    by_x = (value(x + h * dirx, gamma, beta) - value(x - h * dirx, gamma, beta)) / (2 * h)
    by_g = (value(x, gamma + h * dirp, beta) - value(x, gamma - h * dirp, beta)) / (2 * h)
    by_b = (value(x, gamma, beta + h * dirp) - value(x, gamma, beta - h * dirp)) / (2 * h)
    plan.fwd(x, gamma, beta)
    out = plan.bwd(w, gamma, x=x)
    for diff, grad, direction in ((by_x, out["dx"], dirx), (by_g, out["dgamma"], dirp), (by_b, out["dbeta"], dirp)):
        size = float((grad.double().abs() * direction.double().abs()).sum())
        assert abs(diff - float((grad.double() * direction.double()).sum())) <= 1e-3 * size


def test_layer_norm_special_rows(ctx):
    """A constant row (variance zero: only eps stands under the root), and a row with a NaN or an infinity, which
    spoils its own row and the columns' sums but no other row."""
    M, Cn = 6, 512
    x = draw(M, Cn, torch.float32, 9)
    x[1] = 7.0
    x[3, 100] = float("nan")
    x[4, 7] = float("inf")
    gamma, beta = torch.ones(Cn).cuda(), torch.zeros(Cn).cuda()
    plan = B.LayerNormPlan(ctx, M, Cn, torch.float32, "cuda", eps=1e-5)
    y = plan.fwd(x.cuda(), gamma, beta).cpu().numpy()
    assert np.all(np.abs(y[1]) <= 4e-6 * 7 / np.sqrt(1e-5))
    assert abs(plan.rstd[1].item() * np.sqrt(1e-5) - 1) <= 1e-5
    assert np.isnan(y[3]).all() and np.isnan(y[4]).any()
    keep = [0, 1, 2, 5]
    ref = ln_ref(f64(x[keep]), 1.0, 0.0, 1e-5)[0]
    assert np.all(np.isfinite(y[keep])) and np.abs(y[keep][[0, 2, 3]] - ref[[0, 2, 3]]).max() <= 1e-4
    out = plan.bwd(torch.ones((M, Cn), device="cuda"), gamma, x=x.cuda())
    assert torch.isfinite(out["dx"][keep]).all() and torch.isfinite(out["dbeta"]).all()


# ------------------------------------------------------------------------------------------------ all of them
def test_zero_rows(ctx):
    """A batch without rows: nothing to do, and the parameters' gradients are zero."""
    plan = B.LayerNormPlan(ctx, 0, 128, torch.bfloat16, "cuda")
    x, gamma = torch.empty((0, 128), dtype=torch.bfloat16, device="cuda"), torch.ones(128, device="cuda")
    ck = B.Checkpoint(ctx, 0, 128, "cuda").store(x)
    assert plan.fwd(x, gamma, save=ck).shape == (0, 128)
    plan.dgamma.fill_(5), plan.dbeta.fill_(5)
    out = plan.bwd(x, gamma, saved=ck)
    assert float(out["dgamma"].abs().sum()) == 0 and float(out["dbeta"].abs().sum()) == 0
    gelu = B.GeluPlan(ctx, 0, 128, torch.bfloat16, "cuda")
    assert gelu.fwd(x, save=ck).shape == (0, 128) and gelu.bwd(x, saved=ck).shape == (0, 128)
    assert ck.load().shape == (0, 128) and ck.nbytes == 0


def test_on_another_stream(ctx):
    """Work goes to torch's current stream: a chain on a side stream gives what the default stream gives."""
    M, Cn = 515, 1040
    x, dy = draw(M, Cn, torch.bfloat16, 1).cuda(), draw(M, Cn, torch.bfloat16, 2).cuda()
    gamma = torch.ones(Cn, device="cuda")
    norm, gelu = B.LayerNormPlan(ctx, M, Cn, torch.bfloat16, "cuda"), B.GeluPlan(ctx, M, Cn, torch.bfloat16, "cuda")
    c1, c2 = B.Checkpoint(ctx, M, Cn, "cuda"), B.Checkpoint(ctx, M, Cn, "cuda")

    def chain():
        y = gelu.fwd(norm.fwd(x, gamma, save=c1), save=c2)
        out = norm.bwd(gelu.bwd(dy, saved=c2), gamma, saved=c1)
        return [t.clone() for t in (y, out["dx"], out["dgamma"], out["dbeta"])]

    here = chain()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = chain()
    side.synchronize()
    for a, b in zip(here, there):
        assert torch.equal(a, b)


def test_refusals(ctx):
    """Status codes of arguments the row operators do not take, found before any launch."""
    lib, h, st = B.load(), ctx.handle, None
    M, Cn = 4, 128
    x = torch.zeros((M, Cn), dtype=torch.bfloat16, device="cuda")
    y, g = torch.zeros_like(x), torch.zeros(Cn, device="cuda")
    r = torch.zeros(M, device="cuda")
    ck = B.Checkpoint(ctx, M, Cn, "cuda")
    p = lambda t, off=0: C.c_void_p(t.data_ptr() + off)
    none = B.CkptArrays(None, None)
    ws = torch.zeros(B.layer_norm_workspace_bytes(M, Cn), dtype=torch.uint8, device="cuda")
    assert lib.efqat_ckpt_store(None, 1, p(x), M, Cn, ck.ref, st) == -1
    assert lib.efqat_ckpt_store(h, 1, None, M, Cn, ck.ref, st) == -1
    assert lib.efqat_ckpt_store(h, 1, p(x), M, Cn, None, st) == -1
    assert lib.efqat_ckpt_store(h, 1, p(x), M, Cn, C.byref(none), st) == -1
    assert lib.efqat_ckpt_store(h, 7, p(x), M, Cn, ck.ref, st) == -4
    assert lib.efqat_ckpt_store(h, 1, p(x), -1, Cn, ck.ref, st) == -2
    assert lib.efqat_ckpt_store(h, 1, p(x), M, 120, ck.ref, st) == -3
    assert lib.efqat_ckpt_store(h, 1, p(x, 2), M, Cn, ck.ref, st) == -3
    assert lib.efqat_ckpt_load(h, 1, None, M, Cn, p(y), st) == -1
    assert lib.efqat_gelu_fwd(h, 1, p(x), M, 100, p(y), None, st) == -3
    assert lib.efqat_gelu_fwd(h, 1, p(x), M, 0, p(y), None, st) == -2
    assert lib.efqat_gelu_bwd(h, 1, p(x), p(x), ck.ref, M, Cn, p(y), st) == -6
    assert lib.efqat_gelu_bwd(h, 1, p(x), None, None, M, Cn, p(y), st) == -1
    assert lib.efqat_layer_norm_fwd(h, 1, p(x), M, 16392, p(g), None, 1e-5, p(y), p(r), p(r), None, st) == -11
    assert lib.efqat_layer_norm_fwd(h, 1, p(x), M, Cn, None, None, 1e-5, p(y), p(r), p(r), None, st) == -1
    assert lib.efqat_layer_norm_fwd(h, 1, p(x), M, Cn, p(g), None, -1.0, p(y), p(r), p(r), None, st) == -2
    assert lib.efqat_layer_norm_fwd(h, 1, p(x), M, Cn, p(g), None, float("nan"), p(y), p(r), p(r), None, st) == -2
    assert lib.efqat_layer_norm_fwd(h, 1, p(x), M, Cn, p(g), None, 1e-5, p(y), None, p(r), None, st) == -1
    bwd = lambda *a: lib.efqat_layer_norm_bwd(h, 1, *a, st)
    assert bwd(p(x), p(x), ck.ref, M, Cn, p(g), p(r), p(r), p(y), p(g), p(g), p(ws), ws.numel()) == -6
    assert bwd(p(x), None, None, M, Cn, p(g), p(r), p(r), p(y), p(g), p(g), p(ws), ws.numel()) == -1
    assert bwd(p(x), p(x), None, M, Cn, p(g), p(r), p(r), p(y), None, p(g), p(ws), ws.numel()) == -1
    assert bwd(p(x), p(x), None, M, Cn, p(g), p(r), p(r), p(y), p(g), p(g), p(ws), 64) == -7
    assert bwd(p(x), p(x), None, M, Cn, p(g), p(r), p(r), p(y), p(g), p(g), None, ws.numel()) == -7
    plan = B.GeluPlan(ctx, M, Cn, torch.bfloat16, "cuda")
    for bad in (x.float(), x[:2], x.t().contiguous().t(), x.cpu()):
        with pytest.raises(ValueError):
            plan.fwd(bad)
    with pytest.raises(ValueError):
        plan.bwd(x, x=x, saved=ck)
    with pytest.raises(ValueError):
        plan.bwd(x)
    with pytest.raises(ValueError):
        plan.fwd(x, save=B.Checkpoint(ctx, M, 256, "cuda"))
    with pytest.raises(TypeError):
        B.GeluPlan(ctx, M, Cn, torch.float16, "cuda")
    with pytest.raises(B.EfqatError):
        B.Checkpoint(ctx, M, 24, "cuda")
    torch.cuda.synchronize()
    assert ctx.device_status() == 0


def test_a_checkpoint_past_4_gib_of_elements(ctx):
    """Element offsets beyond 32 bits: the last rows of a [262208, 16384] bf16 tensor (4.3e9 elements, 8.6 GB)."""
    M, Cn = 262208, 16384
    x = torch.zeros((M, Cn), dtype=torch.bfloat16, device="cuda")
    tail = draw(3, Cn, torch.bfloat16, 4).cuda()
    x[-3:] = tail
    ck = B.Checkpoint(ctx, M, Cn, "cuda").store(x)
    codes, scales, vals = ckpt_ref(f64(tail))
    assert np.array_equal(ck.codes[-3:].cpu().numpy(), codes) and np.array_equal(ck.scales[-3:].cpu().numpy(), scales)
    assert int(ck.codes[:-3].max()) == 0
    x[-3:] = 1
    ck.load(out=x)
    assert torch.equal(x[-3:].cpu(), torch.from_numpy(vals).to(torch.bfloat16)) and float(x[-4].abs().max()) == 0
