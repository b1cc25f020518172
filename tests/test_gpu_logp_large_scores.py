"""Log probabilities do not depend on the size of the scores: rows far from zero, rows of one value, masks of finite values, scores
divided by a small temperature, and rows whose maximum grows by orders of magnitude on the way."""
import numpy as np
import pytest
import torch

import paper_1803_07289_amd as fx
from gpu_util import say
from operator_util import TYPES, U, chain, half_step, laid_out, smallest_half, to_positions, within

pytestmark = pytest.mark.gpu

OFFSETS = (100.3, -100.3, 1000.7, -1000.7, 1e4, -1e4, 65000.0, -65000.0, 1e6, -1e6, 1.23e7, 1e9, -1e9, 1.7e10, -1e12, 1e20, -1e30, 1e37, -3e38)


def rows_of_all_sizes(C, dtype):
    """Rows of C scores with values of the type, as float64, and a target for each."""
    rng = np.random.default_rng(C)
    f = torch.finfo(dtype)
    rows, targets = [], []

    def row(x, t):
        rows.append(np.where(np.isneginf(x), x, np.clip(x, f.min, f.max)))
        targets.append(t)
    noise = lambda s=3.0: rng.standard_normal(C) * s
    for o in (o for o in OFFSETS if abs(o) <= f.max):
        row(noise() + o, int(rng.integers(C)))
        row(np.full(C, o), C - 1)                                     # (a position masked by a finite value altogether)
        one = np.zeros(C)
        one[C // 3] = o                                               # one class far from the others, which are alike
        row(one, C // 3 if o > 0 else 0)
        row(np.where(np.arange(C) % 3 == 1, noise(), -abs(o)), 1)       # others masked by a finite value
        left = np.full(C, -np.inf)
        left[C // 2] = o
        row(left, C // 2)
        for far_first in (True, False):                               # ordinary scores behind or before far ones
            x = noise()
            half = slice(None, C // 2) if far_first else slice(C // 2, None)
            x[half] += o
            row(x, int(np.argmax(x)))
    for s in (1e3, 3e5, 3e8):
        if s * 8 < f.max:
            row(noise(s), int(rng.integers(C)))
    row(np.arange(C) * (300.0 / C), C - 1)                            # each lane has a maximum of its own
    row(-np.arange(C) * (3e4 / C), 0)
    row(np.where(np.arange(C) % 64 < 32, -1.0, 1.0) * 5e4 + noise(), 40 % C)
    x = torch.from_numpy(np.stack(rows)).to(dtype).double().numpy()
    return x, np.array(targets)


def check(x, t, got, top, layout):
    logp, h, lse, top_logp, top_class = got
    flat = lambda v: v.double().cpu().numpy().reshape(-1)
    m = x.max(1)
    z = x - m[:, None]
    with np.errstate(all="ignore"):
        e = np.exp(z)
        s = e.sum(1)
        zs = np.where(np.isneginf(z), 0.0, np.abs(z))
    p, log_s = e / s[:, None], np.log(s)
    rows = np.arange(len(x))
    want = z[rows, t] - log_s
    want_h = log_s + (p * zs).sum(1)
    # the exponent of a term: a difference and a product, or a fused one, each rounded, and log2(e) itself: 3 U |z| of the term; the
    # power 2 U, and those of the sum.  No part of this knows the size of the scores.
    k = (p * (3 * zs + 4)).sum(1) * U + chain(x.shape[1], 64)
    b_log = k + 4 * U * log_s
    b_logp = b_log + U * np.abs(z[rows, t]) + U * np.abs(want)
    within(flat(logp), want, np.where(np.isfinite(b_logp), b_logp, 0), "logp")
    assert np.all(flat(logp) <= 0), "positive log probabilities"
    within(flat(lse), m + log_s, b_log + U * np.abs(m + log_s), "lse")
    within(flat(h), want_h, 2 * k * (1 + (p * zs).sum(1)) + (p * zs * (3 * zs + 8)).sum(1) * U + 4 * U * log_s, "entropy")
    assert np.all(flat(h) >= 0), "negative entropies"
    order = np.argsort(-x, axis=1, kind="stable")[:, :top]
    best = np.take_along_axis(z, order, 1)
    none = np.isneginf(best)
    assert np.array_equal(to_positions(top_class, layout).astype(int), np.where(none, -1, order)), "classes"
    w = best - log_s[:, None]
    b_top = b_log[:, None] + 2 * U * np.where(none, 0, np.abs(best) + np.abs(w))
    within(to_positions(top_logp, layout), w, b_top, "top_logp")
    assert np.all(to_positions(top_logp, layout) <= 0), "positive log probabilities of alternatives"


@pytest.mark.parametrize("layout", [fx.BNC, fx.BCN], ids=["bnc", "bcn"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", [20, 40, 64, 300, 700, 1500, 2048])
def test_scores_of_any_size(C, dtype, layout):
    say(f"logp large scores {C} {dtype} {layout}")
    x, t = rows_of_all_sizes(C, TYPES[dtype])
    dx, dt = laid_out(x, 1, layout, TYPES[dtype]), torch.from_numpy(t.astype(np.int32))[None].cuda()
    for top in (3, min(C, 9)):
        check(x, t, fx.flexlogp_fwd(dx, dt, top=top, layout=layout), top, layout)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C, times", [(5000, 1), (9000, 1), (9000, 20), (20000, 1), (70000, 1), (70000, 20), (131072, 1)])
def test_scores_of_any_size_in_long_rows(C, times, dtype):
    """Rows in parts; many times over, a workgroup to each."""
    say(f"logp large scores {C} {times} {dtype}")
    x, t = rows_of_all_sizes(C, TYPES[dtype])
    dx, dt = laid_out(x, 1, fx.BNC, TYPES[dtype]), torch.from_numpy(t.astype(np.int32))[None].cuda()
    if times > 1:
        dx, dt = dx.repeat(1, times, 1), dt.repeat(1, times)
    got = fx.flexlogp_fwd(dx, dt, top=5, layout=fx.BNC)
    check(x, t, [v[:, :len(x)] for v in got], 5, fx.BNC)
    for v in got:
        assert all(torch.equal(v[:, i * len(x):(i + 1) * len(x)], v[:, :len(x)]) for i in range(times))


@pytest.mark.parametrize("layout", [fx.BNC, fx.BCN], ids=["bnc", "bcn"])
@pytest.mark.parametrize("C", [13, 40, 1000, 3000, 70000])
def test_a_shift_of_all_scores_changes_nothing(C, layout):
    """Scores in steps of 1/8, to which whole numbers are added without rounding: the same logp, entropy and alternatives."""
    rng = np.random.default_rng(C + 1)
    x = np.round(rng.standard_normal((4, C)) * 24) / 8
    t = torch.from_numpy(rng.integers(0, C, (1, 4)).astype(np.int32)).cuda()
    m, e = x.max(1), np.exp(x - x.max(1, keepdims=True))
    zs = (m[:, None] - x) * e / e.sum(1, keepdims=True)
    k = float((chain(C, 64) + (3 * zs.sum(1) + 4 + 4 * np.log(e.sum(1))) * U).max())
    base = fx.flexlogp_fwd(laid_out(x, 1, layout, torch.float32), t, top=4, layout=layout)
    for o in (99.0, -4097.0, 65537.0, -200001.0, 1000003.0):
        got = fx.flexlogp_fwd(laid_out(x + o, 1, layout, torch.float32), t, top=4, layout=layout)
        # both sides within k of the exact value, and of the differences' own rounding none
        assert float((got[0] - base[0]).abs().max()) <= 2 * k + 2 * U * float(base[0].abs().max())
        assert float((got[1] - base[1]).abs().max()) <= 4 * k * (1 + float(base[1].abs().max()))
        assert float((got[3] - base[3]).abs().max()) <= 2 * k + 2 * U * float(base[3].abs().max())
        assert torch.equal(got[4], base[4])


def check_bwd(x, t, h, gl, gh, got, dtype, layout):
    """From p as it is, not from an lse rounded to fp32."""
    m = x.max(1)
    z = x - m[:, None]
    with np.errstate(all="ignore"):
        log_s = np.log(np.exp(z).sum(1))
        lp = z - log_s[:, None]
        p = np.exp(lp)
        lp = np.where(np.isneginf(lp), 0.0, lp)
    want = -gh[:, None] * p * (lp + h[:, None]) - gl[:, None] * p
    want[np.arange(len(x)), t] += gl
    part = np.abs(gl)[:, None] + np.abs(gh)[:, None] * (np.abs(lp) + np.abs(h)[:, None] + 1)
    # the exponent's roundings 3 U |lp|, the power's 2 U, those of the products; half a step of an lse up to 128, or those of a sum
    off = (3 * np.abs(lp) + 10 + np.minimum(np.abs(m + log_s), 128)[:, None]) * U + chain(x.shape[1], 64)
    within(to_positions(got, layout), want, p * part * off + 2 * U * np.abs(gl)[:, None] + half_step(dtype) * np.abs(want) +
           smallest_half(dtype), "grad_logits")


@pytest.mark.parametrize("layout", [fx.BNC, fx.BCN], ids=["bnc", "bcn"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", [6, 13, 20, 40, 100, 300, 700, 1500, 2500, 9001, 70000])
def test_gradients_of_scores_of_any_size(C, dtype, layout):
    say(f"logp large scores, gradient {C} {dtype} {layout}")
    td = TYPES[dtype]
    x, t = rows_of_all_sizes(C, td)
    rng = np.random.default_rng(C + 5)
    gl, gh = (rng.standard_normal(len(x)).astype(np.float32) for _ in range(2))
    d = lambda a: torch.from_numpy(a)[None].cuda()
    dx, dt = laid_out(x, 1, layout, td, 1, (len(x) if layout == fx.BCN else C) + 3), d(t.astype(np.int32))
    _, h, lse, _, _ = fx.flexlogp_fwd(dx, dt, layout=layout)
    hh = h.double().cpu().numpy().reshape(-1)
    got = fx.flexlogp_bwd(dx, dt, lse, h, d(gl), d(gh), layout=layout)
    check_bwd(x, t, hh, gl, gh, got, td, layout)
    back = fx.flexlogp_bwd(dx, dt, lse, None, d(gl), layout=layout, out=dx)           # in place
    check_bwd(x, t, hh, gl, np.zeros_like(gh), back, td, layout)
