"""Host-side checks of the operators around the layers (no GPU needed): what is refused, before anything is launched."""
import ctypes

import pytest
import torch

import paper_1803_07289_amd as fx

ONE, NONE = ctypes.c_void_p(256), None      # never dereferenced: validation fails first
BIG = 1 << 30


@pytest.fixture(scope="module")
def L():
    return fx.lib()


def norm_fwd(L, x=ONE, w=ONE, b=ONE, y=ctypes.c_void_p(512), B=1, N=8, C=4, eps=1e-5, dtype=0, pdtype=0, layout=1):
    return L.flexnorm_fwd(x, w, b, y, ONE, ONE, B, N, C, eps, dtype, pdtype, layout, None)


@pytest.mark.parametrize("change, status", [
    (dict(x=NONE), 1), (dict(y=NONE), 1), (dict(w=NONE), 1), (dict(b=NONE), 1), (dict(B=0), 2), (dict(N=0), 2), (dict(C=0), 2), (dict(C=-1), 2),
    (dict(B=1 << 12, N=1 << 20), 2), (dict(eps=-1.0), 2), (dict(eps=float("nan")), 2), (dict(dtype=3), 2), (dict(dtype=-1), 2),
    (dict(dtype=1, pdtype=2), 2), (dict(pdtype=1), 2), (dict(layout=2), 2), (dict(y=ONE), 2)])
def test_norm_forward_refuses(L, change, status):
    assert norm_fwd(L, **change) == status


def norm_bwd(L, x=ONE, g=ctypes.c_void_p(512), mean=ONE, rstd=ONE, gx=ctypes.c_void_p(768), gw=ONE, gb=ONE, B=1, N=8, C=4, dtype=0, pdtype=0,
             layout=1, ws=ONE, ws_bytes=BIG):
    return L.flexnorm_bwd(x, ONE, g, mean, rstd, gx, gw, gb, B, N, C, dtype, pdtype, layout, ws, ws_bytes, None)


@pytest.mark.parametrize("change, status", [
    (dict(x=NONE), 1), (dict(g=NONE), 1), (dict(mean=NONE), 1), (dict(rstd=NONE), 1), (dict(gw=NONE), 1), (dict(gb=NONE), 1),
    (dict(gx=NONE, gw=NONE, gb=NONE), 1), (dict(N=0), 2), (dict(dtype=7), 2), (dict(layout=5), 2), (dict(gx=ONE), 2),
    (dict(gx=ctypes.c_void_p(512)), 2), (dict(ws=NONE), 4), (dict(ws=ctypes.c_void_p(260)), 4), (dict(ws_bytes=16), 4)])
def test_norm_backward_refuses(L, change, status):
    assert norm_bwd(L, **change) == status


def test_workspace_sizes_of_refused_sizes_are_zero(L):
    assert L.flexnorm_bwd_workspace_bytes(1, 8, 4, 0, 1) > 0 and L.flexnorm_bwd_workspace_bytes(1, 8, 0, 0, 1) == 0
    assert L.flexlogp_fwd_workspace_bytes(1, 8, 4, 2, 0, 1) > 0
    for sizes in ((0, 8, 4, 2, 0, 1), (1, 8, 4, 5, 0, 1), (1, 8, 64, 33, 0, 1), (1, 8, 4, -1, 0, 1), (1, 8, (1 << 20) + 1, 0, 0, 1),
                  (1, 8, 4, 2, 9, 1), (1, 8, 4, 2, 0, 3)):
        assert L.flexlogp_fwd_workspace_bytes(*sizes) == 0


def test_sizes_that_one_launch_does_not_take_are_refused(L):
    """Positions whose number overflows in the last workgroup, launches of 2^32 threads; the sizes below them have workspaces."""
    most = (1 << 31) - 1024
    for layout in (0, 1):
        assert L.flexlogp_fwd_workspace_bytes(1, most, 1, 0, 0, layout) == (256 if layout == 0 else 0)
        assert L.flexlogp_fwd_workspace_bytes(1, most + 1, 1, 0, 0, layout) == 0
        assert L.flexnorm_bwd_workspace_bytes(1, most + 1, 1, 0, layout) == 0
        assert norm_fwd(L, N=most + 1, C=1, layout=layout) == 2
    assert L.flexnorm_bwd_workspace_bytes(1, most, 1, 0, 1) > 0 and L.flexnorm_bwd_workspace_bytes(1, most, 1, 0, 0) > 0
    for rows, C in ((1 << 24, 4000), (1 << 22, 8193)):                        # 256 and 1024 threads to a row
        assert norm_fwd(L, N=rows, C=C, dtype=1, pdtype=1) == 2 and norm_bwd(L, N=rows, C=C, dtype=1, pdtype=1, ws_bytes=1 << 40) == 2
        assert L.flexnorm_bwd_workspace_bytes(1, rows - 1, C, 1, 1) > 0
    assert norm_fwd(L, N=1 << 28, C=129, layout=0) == 2                        # 16 waves to 64 positions
    assert L.flexlogp_fwd_workspace_bytes(1, (1 << 23) - 1, 4097, 0, 1, 1) > 0
    assert logp_fwd(L, N=1 << 23, C=4097, row=4097, dtype=1) == 2 and logp_bwd(L, N=1 << 23, C=4097, row=4097, grow=4097, dtype=1) == 2
    assert logp_fwd(L, N=1 << 28, C=129, layout=0, row=1 << 28) == 2 and logp_bwd(L, N=1 << 28, C=129, layout=0, row=1 << 28, grow=1 << 28) == 2
    tensors = (fx._AdamwTensor * 17)(*(fx._AdamwTensor(count=(1 << 31) - 1) for _ in range(17)))
    assert L.flexadamw_plan_bytes(tensors, 15) > 0 and L.flexadamw_plan_bytes(tensors, 17) == 0


def logp_fwd(L, x=ONE, t=ONE, lp=ONE, h=ONE, lse=ONE, tl=ONE, tc=ONE, B=1, N=8, C=64, top=2, row=64, dtype=0, layout=1, ws=ONE, ws_bytes=BIG):
    return L.flexlogp_fwd(x, t, lp, h, lse, tl, tc, B, N, C, top, row, dtype, layout, ws, ws_bytes, None)


@pytest.mark.parametrize("change, status", [
    (dict(x=NONE), 1), (dict(h=NONE), 1), (dict(lse=NONE), 1), (dict(t=NONE), 1), (dict(lp=NONE), 1), (dict(tl=NONE), 1), (dict(tc=NONE), 1),
    (dict(B=0), 2), (dict(C=(1 << 20) + 1, row=BIG), 2), (dict(top=-1), 2), (dict(top=33), 2), (dict(C=1, top=2), 2), (dict(row=63), 2),
    (dict(row=1 << 31), 2), (dict(layout=0, row=7), 2), (dict(dtype=3), 2), (dict(layout=4), 2), (dict(C=100_000, row=100_000, ws=NONE), 4),
    (dict(C=100_000, row=100_000, ws=ctypes.c_void_p(8)), 4), (dict(C=100_000, row=100_000, ws_bytes=256), 4)])
def test_log_probabilities_refuse(L, change, status):
    assert logp_fwd(L, **change) == status


def logp_bwd(L, x=ONE, t=ONE, lse=ONE, h=ONE, gl=ONE, gh=ONE, gx=ctypes.c_void_p(512), B=1, N=8, C=64, row=64, grow=64, dtype=0, layout=1):
    return L.flexlogp_bwd(x, t, lse, h, gl, gh, gx, B, N, C, row, grow, dtype, layout, None)


@pytest.mark.parametrize("change, status", [
    (dict(x=NONE), 1), (dict(lse=NONE), 1), (dict(gx=NONE), 1), (dict(gl=NONE, gh=NONE), 1), (dict(t=NONE), 1), (dict(h=NONE), 1),
    (dict(N=-1), 2), (dict(row=63), 2), (dict(grow=10), 2), (dict(dtype=5), 2), (dict(layout=-1), 2), (dict(gx=ONE, grow=65), 2)])
def test_gradient_of_the_scores_refuses(L, change, status):
    assert logp_bwd(L, **change) == status


def adamw_list(L, **change):
    t = fx._AdamwTensor(256, 512, 768, 1024, 1280, None, 100, 0.0)
    for k, v in change.items():
        setattr(t, k, v)
    return (fx._AdamwTensor * 1)(t)


@pytest.mark.parametrize("entry, change, status", [
    ({}, dict(tensors=NONE), 1), ({}, dict(plan=NONE), 1), ({}, dict(out=NONE), 1), (dict(param=None), {}, 1), (dict(exp_avg=None), {}, 1),
    (dict(exp_avg_sq=None), {}, 1), (dict(avg_scale=None), dict(bits=8), 1), (dict(avg_sq_scale=None), dict(bits=8), 1), ({}, dict(n=0), 2),
    ({}, dict(n=(1 << 20) + 1), 2), (dict(count=-1), {}, 2), (dict(count=1 << 31), {}, 2), ({}, dict(dtype=3), 2), ({}, dict(bits=16), 2),
    ({}, dict(copy=0), 2), ({}, dict(beta1=1.0), 2), ({}, dict(beta2=-0.1), 2), ({}, dict(beta2=float("nan")), 2), ({}, dict(eps=0.0), 2),
    ({}, dict(steps=-1), 2), ({}, dict(plan=ctypes.c_void_p(264)), 4), ({}, dict(bytes=512), 4)])
def test_the_optimizers_plan_refuses(L, entry, change, status):
    tensors = adamw_list(L, **entry)
    handle = fx._Adamw()
    a = dict(tensors=tensors, n=1, dtype=0, bits=32, copy=1, beta1=0.9, beta2=0.99, eps=1e-8, steps=0, plan=ONE, bytes=BIG,
             out=ctypes.byref(handle))
    a.update(change)
    assert L.flexadamw_plan_build(a["tensors"], a["n"], a["dtype"], a["bits"], a["copy"], a["beta1"], a["beta2"], a["eps"], a["steps"], 0,
                                  a["plan"], a["bytes"], a["out"], None) == status
    assert status == 4 or handle.plan is None


def test_the_optimizers_step_refuses(L):
    handle = fx._Adamw(256, 1, 1, 0, 32, 1)
    grads = (ctypes.c_void_p * 1)(256)
    step = lambda handle, grads=grads, n=1, dtype=0, lr=0.1: L.flexadamw_step(handle, grads, n, dtype, lr, None, None, None)
    assert step(None) == 1 and step(ctypes.byref(handle), grads=None) == 1 and step(ctypes.byref(fx._Adamw())) == 1
    assert step(ctypes.byref(handle), n=2) == 2 and step(ctypes.byref(handle), dtype=3) == 2
    assert step(ctypes.byref(handle), lr=float("inf")) == 2
    for broken in (dict(tensors=0), dict(param_dtype=4), dict(state_bits=7), dict(chunks=-1)):
        h = fx._Adamw(256, 1, 1, 0, 32, 1)
        for k, v in broken.items():
            setattr(h, k, v)
        assert step(ctypes.byref(h), n=h.tensors) == 2


def test_the_plans_size(L):
    up = lambda x: (x + 255) // 256 * 256
    for counts in ((1,), (2048, 2049, 0), (1000,) * 100):
        t = (fx._AdamwTensor * len(counts))(*(fx._AdamwTensor(count=c) for c in counts))
        n, chunks = len(counts), sum((c + 2047) // 2048 for c in counts)
        assert L.flexadamw_plan_bytes(t, n) == 256 + up(64 * n) + up(8 * n) + up(4 * chunks)


def test_the_binding_refuses_tensors_of_the_cpu():
    x, t = torch.zeros(1, 4, 8), torch.zeros(1, 8, dtype=torch.int32)
    for call in (lambda: fx.flexnorm_fwd(x), lambda: fx.flexlogp_fwd(x, t), lambda: fx.flexlogp_bwd(x, t, x, x, x),
                 lambda: fx.flexnorm_bwd(x, None, x, x, x), lambda: fx.flexadamw_plan_build([x], [x], [x])):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        fx.flexnorm_fwd(x, layout="nbc")
    with pytest.raises(ValueError):
        fx.flexadamw_plan_build([], [], [])
    with pytest.raises(ValueError):
        fx.flexadamw_plan_build([x], [], [x])
    with pytest.raises(ValueError):
        fx.flexadamw_state([x], bits=16)


def at(address):
    return ctypes.c_void_p(address)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype, size", [(0, 4), (1, 2), (2, 2)])
def test_norm_refuses_results_that_share_memory_with_its_inputs(L, dtype, size, layout):
    """Tensors of 8 positions of 4 channels, an element, a position or all but an element apart, either way round."""
    x = 1 << 20
    for d in (size, 4 * size, 31 * size, 1, 32 * size - 1):
        for y in (x - d, x + d):
            assert norm_fwd(L, x=at(x), y=at(y), dtype=dtype, pdtype=dtype, layout=layout) == 2
            assert norm_bwd(L, x=at(x), g=at(2 * x), gx=at(y), dtype=dtype, pdtype=dtype, layout=layout) == 2
            assert norm_bwd(L, x=at(2 * x), g=at(x), gx=at(y), dtype=dtype, pdtype=dtype, layout=layout) == 2


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype, size", [(0, 4), (1, 2), (2, 2)])
def test_gradient_of_the_scores_refuses_rows_that_share_memory_with_others(L, dtype, size, layout):
    x, (N, C) = 1 << 20, (5, 7)
    rows, width = (7, 5) if layout == 0 else (5, 7)
    f = lambda gx, row, grow: logp_bwd(L, x=at(x), gx=at(gx), N=N, C=C, row=row, grow=grow, dtype=dtype, layout=layout)
    cases = [(d, row, row) for row in (width, 20) for d in (1, -1, width - 1, 1 - width, row + 1, row - 1, (rows - 1) * row + width - 1)]
    cases += [(d, row, grow) for row, grow in ((8, 16), (24, 16), (9, 7), (16, 41)) for d in (0, 1, -1, 2 * row)]
    held = 0
    for d, row, grow in cases:
        a = {i * row + j for i in range(rows) for j in range(width)}
        b = {d + i * grow + j for i in range(rows) for j in range(width)}
        if a & b:
            held += 1
            assert f(x + d * size, row, grow) == 2, (d, row, grow)
    assert held > 25
    assert f(x, 20, 21) == 2 and f(x + 1, width, width) == 2 and f(x - 1, width, width) == 2
