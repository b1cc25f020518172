"""The numpy reference of the operators around the layers: gradients against differences, closed forms, the 8-bit states'
format against torch's, their rounding's mean."""
import numpy as np
import pytest
import torch

from oracle import operators as ref


def differences(f, x, h=1e-6):
    """Gradient of the scalar f at x by central differences."""
    g = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        e = np.zeros(x.shape)
        e[i] = h
        g[i] = (f(x + e) - f(x - e)) / (2 * h)
    return g


def test_norm_gradients_are_the_differences():
    rng = np.random.default_rng(0)
    x, g, w, b = rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7)
    loss = lambda x, w, b: (ref.norm_fwd(x, w, b)[0] * g).sum()
    _, mean, rstd = ref.norm_fwd(x, w, b)
    gx, gw, gb = ref.norm_bwd(x, w, g, mean, rstd)
    # central differences at h = 1e-6: rounding 1e-16 / 1e-6, truncation h^2
    assert np.allclose(gx, differences(lambda v: loss(v, w, b), x), atol=1e-8)
    assert np.allclose(gw, differences(lambda v: loss(x, v, b), w), atol=1e-8)
    assert np.allclose(gb, differences(lambda v: loss(x, w, v), b), atol=1e-8)


def test_norm_of_two_values_is_plus_and_minus_one():
    y, mean, rstd = ref.norm_fwd([[1.0, 5.0]], eps=0.0)
    assert np.allclose(y, [[-1, 1]]) and np.allclose(mean, 3) and np.allclose(rstd, 0.5)


def test_log_probabilities_by_hand_and_gradients_by_differences():
    x = np.log(np.array([[1.0, 2.0, 1.0, 4.0], [3.0, 1.0, 0.0, 0.0], [1.0, 1.0, 1.0, 1.0], [0.0, 0.0, 0.0, 0.0]]) + 0.0,
               where=np.array([[1, 1, 1, 1], [1, 1, 0, 0], [1, 1, 1, 1], [0, 0, 0, 0]], bool), out=np.full((4, 4), -np.inf))
    logp, h, lse, top, which = ref.logp_fwd(x, [1, 0, -1, 2], top=3)
    assert np.allclose(np.exp(logp[:2]), [0.25, 0.75]) and np.allclose(np.exp(lse[:2]), [8, 4])
    assert np.allclose(h[0], -(2 / 8 * np.log(1 / 8) + 1 / 4 * np.log(1 / 4) + 1 / 2 * np.log(1 / 2)))
    assert which.tolist() == [[3, 1, 0], [0, 1, -1], [-1, -1, -1], [-1, -1, -1]]
    assert (logp[2], h[2], lse[2]) == (0, 0, 0) and (logp[3], h[3], lse[3]) == (-np.inf, 0, -np.inf)
    rng = np.random.default_rng(1)
    x, t, gl, gh = rng.standard_normal((3, 5)), [4, 0, -1], rng.standard_normal(3), rng.standard_normal(3)

    def loss(x):
        logp, h, _, _, _ = ref.logp_fwd(x, t)
        return (logp * gl + h * gh).sum()
    _, h, lse, _, _ = ref.logp_fwd(x, t)
    assert np.allclose(ref.logp_bwd(x, t, lse, h, gl, gh), differences(loss, x), atol=1e-8)


def test_adamw_is_torchs():
    rng = np.random.default_rng(2)
    p = torch.tensor(rng.standard_normal(50), dtype=torch.float64, requires_grad=True)
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    q, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.standard_normal(50)
        p.grad = torch.tensor(g)
        opt.step()
        q, m, v = ref.adamw(q, m, v, g, t, 0.01, 0.9, 0.99, 1e-6, 0.1)
    assert np.allclose(q, p.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_the_8_bit_values_are_torchs_e4m3_and_e8m0():
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(ref.e4m3(codes.numpy()), codes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    assert np.array_equal(2.0 ** (np.arange(255) - 127.0), codes[:255].view(torch.float8_e8m0fnu).double().numpy())


@pytest.mark.parametrize("spread", [0.0, 8.0, 25.0])
def test_stored_states_are_neighbours_of_the_value_and_right_in_the_mean(spread):
    rng = np.random.default_rng(3)
    n, rounds = 96, 4000
    x = (rng.standard_normal(n) * 10.0 ** (-spread * rng.random(n) - 3)).astype(np.float32)
    for second in (False, True):
        value = (x * x if second else x).astype(np.float32)
        mean = np.zeros(n)
        for k in range(rounds):
            r = ref.noise(n, 7, k, 3)[second]
            codes, scale = ref.store(value, r, np.sqrt(value) if second else None)
            got = ref.widen(codes, scale).astype(np.float64)
            mean += (got * got if second else got) / rounds
            unit = np.repeat(2.0 ** (scale.astype(np.float64) - 127), 32)[:n]
            root = np.sqrt(value.astype(np.float64)) if second else np.abs(value.astype(np.float64))
            # spacing of e4m3: 2^-3 of the power of two below, 2^-9 of the block's unit at least; one step up or down, and a v
            # above zero not at zero
            step = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(root, 1e-300))) - 3), unit * 2.0 ** -9)
            assert np.all(np.abs(np.abs(got) - root) <= step * (1 + 1e-6))
            assert not second or np.all((got > 0) == (value > 0))
        # the mean of `rounds` draws, each within one step: five standard deviations of at most half a step each, and 2^-16 of a step
        # for the 16 random bits; below the smallest code v is held up
        half = step / 2 * (2 * root + step if second else 1)
        fine = (root > unit * 2.0 ** -9) | (not second)
        assert np.all(np.abs(mean - value)[fine] <= (5 * half / np.sqrt(rounds) + 2.0 ** -15 * half)[fine])


def test_noise_is_even_and_its_halves_and_neighbours_do_not_go_together():
    n = 1 << 18
    a, b = ref.noise(n, 1, 1, 0)
    c, _ = ref.noise(n, 1, 2, 0)
    for u in (a, b, c):
        counts = np.bincount((u * 64).astype(int), minlength=64)
        assert np.all(np.abs(counts - n / 64) < 6 * np.sqrt(n / 64))
    for u, v in ((a, b), (a, c), (a[1:], a[:-1]), (a[32:], a[:-32])):
        assert abs(np.corrcoef(u, v)[0, 1]) < 5 / np.sqrt(n)
