"""Layer norm on the GPU against float64, forward and backward: layouts, types, widths from one channel on, alignments."""
import numpy as np
import pytest
import torch

import paper_1803_07289_amd as fx
from oracle import operators as ref
from gpu_util import say
from operator_util import TYPES, U, chain, half_step, laid_out, smallest_half, to_positions, within

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 1), (1, 1, 4096), (2, 3, 2), (1, 65, 3), (3, 41, 9), (1, 1000, 13), (2, 129, 16), (1, 64, 63), (1, 300, 64), (2, 70, 65),
          (1, 513, 100), (1, 33, 128), (1, 5, 255), (2, 17, 257), (1, 40, 513), (1, 21, 1000), (1, 9, 2049), (2, 5, 5120), (1, 3, 8191),
          (1, 7, 16000), (1, 2, 33000), (1, 4100, 48), (1, 20011, 4), (1, 19, 130), (1, 70, 300), (3, 23, 385), (3, 11, 700), (1, 9, 1400),
          (2, 7, 2500), (1, 6001, 1030), (1, 1301, 4500)]


def make(seed, B, N, C, dtype, shift=0.5):
    rng = np.random.default_rng(seed)
    rnd = lambda a, d=dtype: torch.from_numpy(a).to(d).double().numpy()
    return rng, rnd(rng.standard_normal((B * N, C)) * 1.5 + shift), rnd(rng.standard_normal((B * N, C)) * 0.5)


def check_fwd(x, w, b, eps, got, dtype, layout):
    y, mean, rstd = got
    C = x.shape[1]
    wy, wmean, wrstd = ref.norm_fwd(x, w, b, eps)
    k, size = chain(C), np.abs(x).mean(1)
    # the mean: k of the mean magnitude; its error shifts the squares' mean in second order; a root halves a relative error
    within(mean.cpu().numpy().reshape(-1), wmean, k * size, "mean")
    within(rstd.cpu().numpy().reshape(-1), wrstd, (k + (k * size * wrstd) ** 2) * wrstd, "rstd")
    ww = 1.0 if w is None else np.abs(w)
    bound = k * (ww * ((size * wrstd)[:, None] + 2 * np.abs((x - wmean[:, None]) * wrstd[:, None])) + np.abs(wy) + (0 if b is None else np.abs(b)))
    within(to_positions(y, layout), wy, bound + half_step(dtype) * np.abs(wy) + smallest_half(dtype), "y")


def check_bwd(x, w, g, mean, rstd, got, dtype, wdtype, layout):
    gx, gw, gb = got
    wx, ww, wb = ref.norm_bwd(x, w, g, mean, rstd)
    rows, C = x.shape
    r = rstd[:, None]
    xh = (x - mean[:, None]) * r
    h = g * (1.0 if w is None else w)
    k = chain(C)
    # xh itself is (x - mean) rstd of two roundings, the rest k of the magnitudes that meet
    part = np.abs(h) + np.abs(h).mean(1, keepdims=True) + np.abs(xh) * np.abs(h * xh).mean(1, keepdims=True) * 2
    within(to_positions(gx, layout), wx, k * r * part + half_step(dtype) * np.abs(wx) + smallest_half(dtype), "grad_x")
    if w is not None:
        kr = chain(rows)
        within(gw.double().cpu().numpy(), ww, kr * np.abs(g * xh).sum(0) + half_step(wdtype) * np.abs(ww) + smallest_half(wdtype), "grad_weight")
        within(gb.double().cpu().numpy(), wb, kr * np.abs(g).sum(0) + half_step(wdtype) * np.abs(wb) + smallest_half(wdtype), "grad_bias")


@pytest.mark.parametrize("layout", [fx.BNC, fx.BCN], ids=["bnc", "bcn"])
@pytest.mark.parametrize("dtype, wdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norm(shape, dtype, wdtype, layout):
    B, N, C = shape
    say(f"norm {shape} {dtype} {wdtype} {layout}")
    td, wd = TYPES[dtype], TYPES[wdtype]
    rng, x, g = make(sum(shape), B, N, C, td)
    w = torch.from_numpy(rng.standard_normal(C) + 1).to(wd).double().numpy()
    b = torch.from_numpy(rng.standard_normal(C)).to(wd).double().numpy()
    put = lambda a: torch.from_numpy(a).to(wd).cuda()
    offset = sum(shape) % 3                                        # storage that begins at any element
    dx, dg = laid_out(x, B, layout, td, offset), laid_out(g, B, layout, td, offset * 2)
    got = fx.flexnorm_fwd(dx, put(w), put(b), layout=layout)
    check_fwd(x, w, b, 1e-5, got, td, layout)
    mean, rstd = got[1].double().cpu().numpy().reshape(-1), got[2].double().cpu().numpy().reshape(-1)
    need = fx.lib().flexnorm_bwd_workspace_bytes(B, N, C, fx._DTYPES[td], layout)
    guarded = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    back = fx.flexnorm_bwd(dx, put(w), dg, got[1], got[2], layout=layout, workspace=guarded[:need])
    check_bwd(x, w, g, mean, rstd, back, td, wd, layout)
    assert bool((guarded[need:] == 0xA5).all()), "wrote past the workspace"
    again = fx.flexnorm_bwd(dx, put(w), dg, got[1], got[2], layout=layout)
    for one, two in zip(back, again):
        assert torch.equal(one, two), "another result for the same inputs"
    only_x = fx.flexnorm_bwd(dx, put(w), dg, got[1], got[2], layout=layout, need_params=False)
    only_w = fx.flexnorm_bwd(dx, put(w), dg, got[1], got[2], layout=layout, need_x=False)
    assert only_x[1] is None and only_w[0] is None
    # (a call for one of them may add in another order)
    check_bwd(x, w, g, mean, rstd, (only_x[0], only_w[1], only_w[2]), td, wd, layout)


@pytest.mark.parametrize("layout", [fx.BNC, fx.BCN], ids=["bnc", "bcn"])
def test_norm_without_parameters_and_rows_without_variance(layout):
    x = np.random.default_rng(5).standard_normal((40, 24))
    x[7] = 3.25                                                     # exact mean: rstd = 1 / sqrt(eps), y = 0
    x = x.astype(np.float32).astype(np.float64)
    dx = laid_out(x, 2, layout, torch.float32)
    y, mean, rstd = fx.flexnorm_fwd(dx, eps=1e-3, layout=layout)
    check_fwd(x, None, None, 1e-3, (y, mean, rstd), torch.float32, layout)
    assert np.all(to_positions(y, layout)[7] == 0)
    gx, gw, gb = fx.flexnorm_bwd(dx, None, dx, mean, rstd, layout=layout)
    assert gw is None and gb is None
    check_bwd(x, None, x, mean.double().cpu().numpy().reshape(-1), rstd.double().cpu().numpy().reshape(-1), (gx, None, None), torch.float32,
              torch.float32, layout)


@pytest.mark.parametrize("layout", [fx.BNC, fx.BCN], ids=["bnc", "bcn"])
@pytest.mark.parametrize("C", [9, 64, 1000, 9000])
def test_a_mean_far_from_zero_costs_no_more_than_its_own_rounding(layout, C):
    rng, x, _ = make(9, 1, 30, C, torch.float32, shift=1000.0)
    got = fx.flexnorm_fwd(laid_out(x, 1, layout, torch.float32), layout=layout)
    check_fwd(x, None, None, 1e-5, got, torch.float32, layout)


@pytest.mark.parametrize("layout", [fx.BNC, fx.BCN], ids=["bnc", "bcn"])
@pytest.mark.parametrize("C", [5, 64, 700, 20000])
def test_a_row_with_nan_or_infinity_spoils_its_own_outputs_only(layout, C):
    rng, x, g = make(11, 1, 20, C, torch.float32)
    clean = fx.flexnorm_fwd(laid_out(x, 1, layout, torch.float32), layout=layout)
    bad = x.copy()
    bad[3, C // 2], bad[12, C - 1] = np.nan, np.inf
    got = fx.flexnorm_fwd(laid_out(bad, 1, layout, torch.float32), layout=layout)
    keep = np.setdiff1d(np.arange(20), [3, 12])
    assert np.array_equal(to_positions(got[0], layout)[keep], to_positions(clean[0], layout)[keep])
    assert np.all(np.isnan(to_positions(got[0], layout)[3])) and np.isnan(got[2][0, 12].item())


def test_large_sums_over_positions():
    """Many positions, so that partial sums are many; the reference on the GPU in float64."""
    for layout, C, N in ((fx.BNC, 64, 300_007), (fx.BCN, 13, 200_003)):
        g = torch.Generator(device="cuda").manual_seed(3)
        shape = (1, C, N) if layout == fx.BCN else (1, N, C)
        x, go = torch.randn(shape, device="cuda", generator=g), torch.randn(shape, device="cuda", generator=g)
        w = torch.ones(C, device="cuda")
        y, mean, rstd = fx.flexnorm_fwd(x, w, w, layout=layout)
        gx, gw, gb = fx.flexnorm_bwd(x, w, go, mean, rstd, layout=layout)
        d = 1 if layout == fx.BCN else 2
        xh = (x.double() - mean.double().unsqueeze(d)) * rstd.double().unsqueeze(d)
        rows = (0, 3 - d)
        kr = chain(N, 256)
        for got, terms in ((gw, go.double() * xh), (gb, go.double())):
            off = (got.double() - terms.sum(rows)).abs()
            assert bool((off <= kr * terms.abs().sum(rows)).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout, C, N", [(fx.BCN, 100, 90_001), (fx.BCN, 20, 300_002), (fx.BCN, 250, 30_003), (fx.BNC, 600, 20_005),
                                          (fx.BNC, 40, 150_001)])
def test_workgroups_that_walk_over_many_positions(layout, C, N, dtype):
    """Every turn of the backward kernels' loops; the reference on the GPU in float64 from the same statistics."""
    g = torch.Generator(device="cuda").manual_seed(C)
    shape = (1, C, N) if layout == fx.BCN else (1, N, C)
    d = 1 if layout == fx.BCN else 2
    x, go = (torch.randn(shape, device="cuda", generator=g).to(TYPES[dtype]) for _ in range(2))
    w = torch.rand(C, device="cuda", generator=g) + 0.5
    _, mean, rstd = fx.flexnorm_fwd(x, w, w, layout=layout)
    gx, gw, gb = fx.flexnorm_bwd(x, w, go, mean, rstd, layout=layout)
    r = rstd.double().unsqueeze(d)
    xh = (x.double() - mean.double().unsqueeze(d)) * r
    rows = (0, 3 - d)
    for got, terms in ((gw, go.double() * xh), (gb, go.double())):
        assert bool(((got.double() - terms.sum(rows)).abs() <= chain(N, 256) * terms.abs().sum(rows)).all())
    h = go.double() * (w.double()[:, None] if layout == fx.BCN else w.double())
    m1, m2 = h.mean(d, keepdim=True), (h * xh).mean(d, keepdim=True)
    want = r * (h - m1 - xh * m2)
    part = h.abs() + h.abs().mean(d, keepdim=True) + 2 * xh.abs() * (h * xh).abs().mean(d, keepdim=True)
    bound = chain(C) * r * part + half_step(TYPES[dtype]) * want.abs() + smallest_half(TYPES[dtype])
    assert bool(((gx.double() - want).abs() <= bound).all())
    only = fx.flexnorm_bwd(x, w, go, mean, rstd, layout=layout, need_params=False)[0]
    assert bool(((only.double() - want).abs() <= bound).all())


def test_refusals_of_the_binding():
    x, w = torch.zeros(2, 5, 8, device="cuda"), torch.zeros(5, device="cuda")
    y, mean, rstd = fx.flexnorm_fwd(x, w, w)
    for call, error in ((lambda: fx.flexnorm_fwd(x[0], w, w), ValueError), (lambda: fx.flexnorm_fwd(x, w[:4], w[:4]), ValueError),
                        (lambda: fx.flexnorm_fwd(x, w, None), ValueError), (lambda: fx.flexnorm_fwd(x.transpose(1, 2), w, w), ValueError),
                        (lambda: fx.flexnorm_fwd(x.double(), w, w), TypeError), (lambda: fx.flexnorm_fwd(x, w.half(), w.half()), TypeError),
                        (lambda: fx.flexnorm_fwd(x, w, w, out=x), fx.FlexError), (lambda: fx.flexnorm_fwd(x, w, w, eps=-1.0), fx.FlexError),
                        (lambda: fx.flexnorm_fwd(x[:, :, :0], w, w), fx.FlexError), (lambda: fx.flexnorm_bwd(x, w, y[:1], mean, rstd), ValueError),
                        (lambda: fx.flexnorm_bwd(x, w, y, mean[:, :4], rstd), ValueError),
                        (lambda: fx.flexnorm_bwd(x, w, y, mean, rstd, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), fx.FlexError)):
        with pytest.raises(error):
            call()
