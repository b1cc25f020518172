"""The AdamW step on the GPU against float64, and its 8-bit states bit for bit against the same formulas in float32."""
import numpy as np
import pytest
import torch

import paper_1803_07289_amd as fx
from oracle import operators as ref
from gpu_util import say
from operator_util import TYPES, U, half_step, smallest_half, within

pytestmark = pytest.mark.gpu

SIZES = [1, 7, 8, 31, 32, 33, 100, 0, 2047, 2048, 2049, 4096, 5000, 65537]
F32 = np.float32
LR, BETAS, EPS = 0.01, (0.9, 0.99), 1e-6


def tensors(seed, sizes, dtype, scale=1.0, offset=0):
    """float64 values of the type, and device tensors whose storage begins `offset` elements in."""
    rng = np.random.default_rng(seed)
    values = [torch.from_numpy(rng.standard_normal(n) * scale).to(dtype).double().numpy() for n in sizes]
    placed = [torch.empty(n + offset, dtype=dtype, device="cuda")[offset:] for n in sizes]
    for t, v in zip(placed, values):
        t.copy_(torch.from_numpy(v))
    return values, placed


def numpy_of(ts):
    return [t.double().cpu().numpy() for t in ts]


def codes_of(ts):
    return [t.view(torch.uint8).cpu().numpy() for t in ts]


def check_p(got, p, m, v, g, t, decay, dtype, what):
    """p after step t from the float64 state before it."""
    want, wm, wv = ref.adamw(p, m, v, g, t, LR, *BETAS, EPS, decay)
    size, second = np.abs(BETAS[0] * m) + np.abs((1 - BETAS[0]) * g), wv
    step = LR / (1 - BETAS[0] ** t)
    under = np.sqrt(second / (1 - BETAS[1] ** t)) + EPS
    # the first moment: 4 roundings of its parts; the update another 12, v's among them
    update = step * (4 * U * size + 12 * U * np.abs(wm)) / under
    within(got, want, 3 * U * np.abs(p) + update + U * np.abs(want) + half_step(dtype) * np.abs(want) + smallest_half(dtype), what)
    return want, wm, wv


@pytest.mark.parametrize("ptype, gtype, ctype", [("f32", "f32", None), ("f32", "bf16", "bf16"), ("f32", "f16", "f16"), ("bf16", "bf16", None),
                                                ("f16", "f32", None), ("bf16", "f32", "f16")])
@pytest.mark.parametrize("offset", [0, 1])
def test_states_in_32_bits(ptype, gtype, ctype, offset):
    say(f"adamw 32 {ptype} {gtype} {ctype} {offset}")
    pt, gt = TYPES[ptype], TYPES[gtype]
    _, params = tensors(1, SIZES, pt, 1.0, offset)
    _, copies = tensors(1, SIZES, TYPES[ctype], 1.0, offset) if ctype else (None, None)
    m, v, _, _ = fx.flexadamw_state(params)
    decay = [0.1 * (i % 3) for i in range(len(SIZES))]
    plan = fx.flexadamw_plan_build(params, m, v, copies=copies, weight_decay=decay, betas=BETAS, eps=EPS)
    clip = torch.tensor([0.5], device="cuda")
    for t in range(1, 4):
        gv, grads = tensors(10 + t, SIZES, gt, 0.1, offset)
        was = [numpy_of(x) for x in (params, m, v)]
        fx.flexadamw_step(plan, grads, LR, grad_scale=clip)
        for i in range(len(SIZES)):
            p0, m0, v0 = (x[i] for x in was)
            g = gv[i] * 0.5                                            # exact
            got = params[i].double().cpu().numpy()
            want, wm, wv = check_p(got, p0, m0, v0, g, t, decay[i], pt, f"p {i}")
            within(m[i].double().cpu().numpy(), wm, 4 * U * (np.abs(m0) + np.abs(g)), f"m {i}")
            within(v[i].double().cpu().numpy(), wv, 6 * U * wv + 2.0 ** -149, f"v {i}")
            if copies:
                check_p(copies[i].double().cpu().numpy(), p0, m0, v0, g, t, decay[i], TYPES[ctype], f"copy {i}")
    assert plan.steps() == 3


@pytest.mark.parametrize("ptype, gtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("offset", [0, 1])
def test_states_in_8_bits(ptype, gtype, offset):
    say(f"adamw 8 {ptype} {gtype} {offset}")
    pt, gt = TYPES[ptype], TYPES[gtype]
    _, params = tensors(2, SIZES, pt, 1.0, offset)
    m, v, ms, vs = fx.flexadamw_state(params, 8)
    if offset:                                                         # 8-bit states that begin at odd bytes
        shift = lambda ts: [torch.zeros(t.numel() + 3, dtype=torch.uint8, device="cuda")[3:].view(t.dtype) for t in ts]
        m, v, ms, vs = shift(m), shift(v), shift(ms), shift(vs)
    plan = fx.flexadamw_plan_build(params, m, v, ms, vs, weight_decay=0.1, betas=BETAS, eps=EPS, seed=77)
    for t in range(1, 5):
        # gradients over many powers of ten, so that blocks hold large and small values and some of them zeros
        gv, grads = tensors(20 + t, SIZES, gt, 0.1, offset)
        for x, y in zip(gv, grads):
            x *= 10.0 ** (-6 * np.random.default_rng(t).random(len(x)))
            x[::5] = 0
            y.copy_(torch.from_numpy(x))
            x[:] = y.double().cpu().numpy()
        was = [codes_of(x) for x in (m, ms, v, vs)]
        p0 = numpy_of(params)
        fx.flexadamw_step(plan, grads, LR)
        now = [codes_of(x) for x in (m, ms, v, vs)]
        for i in range(len(SIZES)):
            m0, ms0, v0, vs0 = (x[i] for x in was)
            p, *want = ref.adamw_8bit(p0[i], m0, ms0, v0, vs0, gv[i], t, LR, *BETAS, EPS, 0.1, 77, i) if SIZES[i] else (p0[i],) + tuple(x[i] for x in was)
            for got, w, name in zip((x[i] for x in now), want, ("m", "m scale", "v", "v scale")):
                assert np.array_equal(got, w), (name, i, t, int(np.sum(got != w)))
            check_p(params[i].double().cpu().numpy(), p0[i], ref.widen(m0, ms0).astype(np.float64), ref.widen(v0, vs0).astype(np.float64) ** 2,
                    gv[i], t, 0.1, pt, f"p {i}")


def test_every_8_bit_state_is_read_as_what_it_is():
    """All finite e4m3 bytes under several powers of two, with beta = 0.5 and no gradient: the states are halved exactly."""
    codes = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    n = len(codes)
    for power in (127, 100, 140):
        p = torch.zeros(n, device="cuda")
        m, v, ms, vs = fx.flexadamw_state([p], 8)
        m[0].view(torch.uint8).copy_(torch.from_numpy(codes))
        ms[0].view(torch.uint8).fill_(power)
        plan = fx.flexadamw_plan_build([p], m, v, ms, vs, betas=(0.5, 0.5), eps=1.0)
        before = ref.widen(codes, np.full((n + 31) // 32, power, np.uint8))
        fx.flexadamw_step(plan, [torch.zeros(n, device="cuda")], 1.0)
        # p = - lr (m / 2) / (1 - 1/2) / (0 + 1) = -m
        assert np.array_equal(p.cpu().numpy(), -before)


def test_a_long_run_in_8_bits_follows_one_in_32():
    """Constant second moments: the mean of the 8-bit states over many elements stays at the exact ones."""
    n, steps = 1 << 15, 300
    rng = torch.Generator(device="cuda").manual_seed(1)
    p = [torch.zeros(n, device="cuda")]
    m, v, ms, vs = fx.flexadamw_state(p, 8)
    plan = fx.flexadamw_plan_build(p, m, v, ms, vs, betas=(0.9, 0.99), eps=1e-8)
    m1, v1 = torch.zeros(n, device="cuda", dtype=torch.float64), torch.zeros(n, device="cuda", dtype=torch.float64)
    for _ in range(steps):
        g = torch.randn(n, device="cuda", generator=rng) + 0.5
        fx.flexadamw_step(plan, [g], 1e-3)
        m1, v1 = 0.9 * m1 + 0.1 * g.double(), 0.99 * v1 + 0.01 * g.double() ** 2
    wide = lambda x, s: x[0].double() * s[0].double().repeat_interleave(32)
    m8, v8 = wide(m, ms), wide(v, vs) ** 2
    # The states' error is a sum of the steps' roundings, each at most one step of e4m3 (an eighth of the value; of v a quarter of it and
    # a little) and zero in the mean, faded by beta: for n elements the mean's standard deviation is below
    # 0.3 / sqrt(1 - beta2^2) / sqrt(n) = 0.012 of the value; five of them
    assert abs(float(v8.mean() / v1.mean()) - 1) < 0.06
    assert abs(float(m8.mean() / m1.mean()) - 1) < 0.06


@pytest.mark.parametrize("size", [1e-18, 1e-20, 1e-21])
@pytest.mark.parametrize("eps", [1e-8, 1e-13, 1e-25, 1e-36])
def test_second_moments_of_the_smallest_gradients(size, eps):
    """v = 0.01 g^2 below fp32's normal numbers: its root stands above eps all the same."""
    n = 5000
    rng = np.random.default_rng(6)
    g = torch.from_numpy(rng.choice([-1.0, 1.0], n) * (1 + rng.random(n)) * size).float().cuda()
    p = torch.zeros(n, device="cuda")
    m, v, _, _ = fx.flexadamw_state([p])
    plan = fx.flexadamw_plan_build([p], m, v, betas=BETAS, eps=eps)
    fx.flexadamw_step(plan, [g], LR)
    m, v = m[0].double().cpu().numpy(), v[0].double().cpu().numpy()
    assert np.all(v > 0)
    # from the moments as they were stored: root, correction, sum, quotient, two products, of an ulp (2 U) each at most
    want = -LR * (m / (1 - BETAS[0])) / (np.sqrt(v / (1 - BETAS[1])) + eps)
    within(p.double().cpu().numpy(), want, 12 * U * np.abs(want) + 2.0 ** -149, "p")


@pytest.mark.parametrize("eps", [1e-6, 1e-30])
def test_8_bit_states_of_the_smallest_gradients(eps):
    """Second moments below fp32's normal numbers, in blocks of their own and beside large ones: above zero they are stored above zero."""
    n = 4096
    rng = np.random.default_rng(7)
    g = (rng.choice([-1.0, 1.0], n) * 10.0 ** -(17 + 4.2 * rng.random(n))).astype(np.float32)
    g[:1024:32] = 0.5                                                  # (the first blocks have a large one each)
    g[1024:2048] = (g[1024:2048].astype(np.float64) * 1e4).astype(np.float32)
    g[::7] = 0
    p = torch.zeros(n, device="cuda")
    m, v, ms, vs = fx.flexadamw_state([p], 8)
    plan = fx.flexadamw_plan_build([p], m, v, ms, vs, betas=BETAS, eps=eps, seed=9)
    for t in (1, 2):
        was = [codes_of(x)[0] for x in (m, ms, v, vs)]
        before = p.cpu().numpy()
        fx.flexadamw_step(plan, [torch.from_numpy(g).cuda()], LR)
        want_p, *want = ref.adamw_8bit(before, *was, g, t, LR, *BETAS, eps, 0.0, 9, 0)
        for got, w, name in zip((codes_of(x)[0] for x in (m, ms, v, vs)), want, ("m", "m scale", "v", "v scale")):
            assert np.array_equal(got, w), (name, t, int(np.sum(got != w)))
        live = (F32(1 - BETAS[1]) * g * g) > 0
        assert np.all(codes_of(v)[0][live] > 0)
        # the formula in fp32, a handful of roundings on either side
        within(p.double().cpu().numpy(), want_p, 24 * U * np.maximum(np.abs(want_p), np.abs(want_p - before)) + 4 * U * np.abs(before), "p")


def test_exponents_of_blocks_at_their_borders():
    """Blocks of one value each, whose second moments step through the places where the root's exponent changes."""
    a2 = F32(1 - BETAS[1])
    g = []
    for k in range(-30, 30, 3):
        for square in (3.0625, 1.0):
            x = F32(np.sqrt(square * 2.0 ** (2 * k) / a2))
            g.append((x.view(np.int32) + np.arange(-40, 41, dtype=np.int32)).view(F32))
    g = np.repeat(np.concatenate(g), 32)
    p = torch.zeros(len(g), device="cuda")
    m, v, ms, vs = fx.flexadamw_state([p], 8)
    plan = fx.flexadamw_plan_build([p], m, v, ms, vs, betas=BETAS, eps=EPS, seed=3)
    was = [codes_of(x)[0] for x in (m, ms, v, vs)]
    _, *want = ref.adamw_8bit(p.cpu().numpy(), *was, g, 1, LR, *BETAS, EPS, 0.0, 3, 0)
    assert len(np.unique(want[3])) >= 40
    fx.flexadamw_step(plan, [torch.from_numpy(g).cuda()], LR)
    for got, w, name in zip((codes_of(x)[0] for x in (m, ms, v, vs)), want, ("m", "m scale", "v", "v scale")):
        assert np.array_equal(got, w), (name, int(np.sum(got != w)))


def test_no_gradient_and_no_step():
    _, params = tensors(3, [100, 3000, 50], torch.float32)
    m, v, ms, vs = fx.flexadamw_state(params, 8)
    plan = fx.flexadamw_plan_build(params, m, v, ms, vs, weight_decay=0.5)
    before = [p.clone() for p in params]
    grads = [torch.ones_like(p) for p in params]
    for bad in (float("nan"), float("inf")):
        fx.flexadamw_step(plan, grads, 0.1, grad_scale=torch.tensor([bad], device="cuda"))
    assert plan.steps() == 0 and all(torch.equal(a, b) for a, b in zip(params, before))
    fx.flexadamw_step(plan, [grads[0], None, grads[2]], torch.tensor([0.1], device="cuda"))
    assert plan.steps() == 1 and torch.equal(params[1], before[1]) and not m[1].view(torch.uint8).any()
    # the first step is lr * sign(g) beside the decay: 0.1 rounded to fp32, and a few roundings more
    for i in (0, 2):
        want = before[i].double() * (1 - 0.1 * 0.5) - 0.1
        assert float((params[i].double() - want).abs().max()) < 1e-6
    fx.flexadamw_step(plan, [None] * 3, 0.1)
    assert plan.steps() == 2


def test_many_tensors_and_resuming():
    """More tensors than one launch takes gradients of; a run continued by a new plan is the run that was not interrupted."""
    sizes = [1 + 37 * i % 300 for i in range(1000)]
    _, one = tensors(4, sizes, torch.float32)
    two = [p.clone() for p in one]
    a, b = fx.flexadamw_state(one, 8), fx.flexadamw_state(two, 8)
    grads = [torch.randn_like(p) for p in one]
    plan = fx.flexadamw_plan_build(one, *a, seed=5)
    for _ in range(3):
        fx.flexadamw_step(plan, grads, 0.01)
    first = fx.flexadamw_plan_build(two, *b, seed=5)
    fx.flexadamw_step(first, grads, 0.01)
    then = fx.flexadamw_plan_build(two, *b, seed=5, steps=first.steps())
    for _ in range(2):
        fx.flexadamw_step(then, grads, 0.01)
    # (the powers of beta are a product in one run and a power in the other: the last bit of a double)
    for i in range(len(sizes)):
        assert float((one[i] - two[i]).abs().max()) <= 4 * 2.0 ** -23 * float(one[i].abs().max())
    assert plan.steps() == then.steps() == 3


def test_replayed_from_a_graph():
    _, params = tensors(6, [64, 5000, 33], torch.bfloat16)
    ours = [p.clone() for p in params]
    grads = [torch.randn_like(p) for p in params]
    lr, scale = torch.tensor([0.01], device="cuda"), torch.tensor([1.0], device="cuda")
    states = fx.flexadamw_state(params, 8), fx.flexadamw_state(ours, 8)
    plan, eager = fx.flexadamw_plan_build(params, *states[0]), fx.flexadamw_plan_build(ours, *states[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fx.flexadamw_step(plan, grads, lr, grad_scale=scale)
    torch.cuda.synchronize()
    for k in range(4):
        lr.fill_(0.01 * (k + 1))
        for g in grads:
            g.normal_()
        graph.replay()
        torch.cuda.synchronize()
        fx.flexadamw_step(eager, grads, 0.01 * (k + 1) if k == 0 else lr)
        torch.cuda.synchronize()
        for a, b in zip(params + states[0][0] + states[0][1], ours + states[1][0] + states[1][1]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), f"replay {k}"
    assert plan.steps() == eager.steps() == 4


def test_refusals_of_the_binding():
    p = torch.zeros(64, device="cuda")
    m, v, _, _ = fx.flexadamw_state([p])
    build = lambda **k: (lambda: fx.flexadamw_plan_build(**{**dict(params=[p], exp_avg=m, exp_avg_sq=v), **k}))
    e8 = fx.flexadamw_state([p], 8)
    half = p.half()
    for call, error in ((build(params=[p, p]), ValueError), (build(exp_avg=[m[0][:63]]), ValueError), (build(exp_avg=[m[0].double()]), TypeError),
                        (build(exp_avg_sq=m), ValueError), (build(params=[p[::2]]), ValueError), (build(avg_scales=e8[2]), ValueError),
                        (build(avg_scales=e8[2], avg_sq_scales=e8[3]), TypeError), (build(copies=[p]), ValueError), (build(copies=[half[:3]]), ValueError),
                        (build(weight_decay=[0.1, 0.2]), ValueError), (build(betas=(1.0, 0.9)), fx.FlexError), (build(eps=0.0), fx.FlexError),
                        (build(params=[p, torch.zeros(64, device="cuda")], exp_avg=m * 2, exp_avg_sq=v * 2), ValueError),
                        (build(params=[p, half], exp_avg=m * 2, exp_avg_sq=v * 2), TypeError), (build(steps=-1), fx.FlexError),
                        (lambda: fx.flexadamw_plan_build([p], e8[0], e8[1], e8[2], [e8[3][0][:1]]), ValueError)):
        with pytest.raises(error):
            call()
    plan = fx.flexadamw_plan_build([p], m, v)
    step = lambda *a, **k: (lambda: fx.flexadamw_step(plan, *a, **k))
    for call, error in ((step([], 0.1), ValueError), (step([p[:63]], 0.1), ValueError), (step([p.double()], 0.1), TypeError), (step([p.cpu()], 0.1), TypeError),
                        (step([p.view(8, 8).t()], 0.1), ValueError), (step([p], float("nan")), fx.FlexError), (step([p], p), ValueError),
                        (step([p], 0.1, grad_scale=p), ValueError), (step([p], 0.1, grad_scale=p[:1].half()), TypeError)):
        with pytest.raises(error):
            call()
    assert plan.steps() == 0
