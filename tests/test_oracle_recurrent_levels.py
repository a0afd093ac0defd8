"""Layer norm and its gradients at the lowest levels that their constants accept, where results have few primes left, decrypted from the CPU oracle: slots that differ and slots that are all alike
(whose polynomial has the value times the scale as one coefficient, the most that a modulus has to hold).

Tolerances as in test_oracle_recurrent.py, with gradients at the scale 2^40: an operation there is off by less than 2^20 / 2^40 = 1e-6, which 1 / sqrt below 2, gains up to 1.5 and the three terms of
dx, each at most (1 + the largest |norm|^2) times the gradient's, multiply by at most 30; the constants' ratio adds 2^-17 of a term below 8.  Both together are below 1e-4."""
import numpy as np
import pytest

from test_oracle_recurrent import BOUND, EPS, SCALE, World, layer_norm
from paper_2604_16834_amd.block import layer_norm_constants, layer_norm_grad_constants, norm_constants

GRAD_SCALE = 2.0 ** 40


@pytest.fixture(scope="module")
def world():
    return World()


def channels_of(rng, channels, n, alike):
    x = rng.uniform(0.4, 1.0, (channels, n)) * np.where(np.arange(channels) % 2, -1, 1)[:, None]
    return np.repeat(x[:, :1], n, 1) if alike else x


@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("affine", [False, True])
@pytest.mark.parametrize("above", [0, 1])
def test_layer_norm_gradients_at_the_lowest_levels(world, affine, alike, above):
    w, rng, channels, level = world, np.random.default_rng(5), 4, 3 + affine + above
    n = w.orc.n
    x, up, gain = channels_of(rng, channels, n, alike), channels_of(rng, channels, n, alike), rng.uniform(0.5, 1.5, channels)
    norm, inv, _ = layer_norm(x)
    assert inv.max() < 2
    k = layer_norm_constants(w.p.moduli, 15, channels, 2.0 ** 47, (0.3, 1.1), 3, EPS)  # the scales that a forward call leaves
    g = layer_norm_grad_constants(w.p.moduli, level, channels, GRAD_SCALE, k.norm_scale, k.inv_scale, SCALE if affine else None)
    ct_gain = w.encrypt(np.repeat(gain[:, None], n, 1), level, SCALE, 40) if affine else None
    ct_up, ct_norm = w.encrypt(up, level, GRAD_SCALE, 90), w.encrypt(norm, level, k.norm_scale, 20)
    dx, dgain, dbias = w.orc.layer_norm_backward(ct_up, ct_norm, w.encrypt(inv[None], level, k.inv_scale, 30)[0], level, g.k_grad, g.k_norm, w.rlk, ct_gain)
    gy = up * gain[:, None] if affine else up
    want = inv * (gy - gy.mean(0) - norm * (gy * norm).mean(0))
    assert g.dx_level == above
    assert np.abs(w.decrypt(dx, g.dx_level, g.dx_scale) - want).max() < BOUND
    assert np.abs(w.decrypt(dgain, level - 1, g.dgain_scale) - up * norm).max() < BOUND
    assert np.abs(w.decrypt(dbias, level - 1, g.dbias_scale) - up).max() < BOUND


def test_gradient_constants_where_there_is_room_and_where_not(world):
    q = world.p.moduli
    norm_scale, inv_scale = q[3] / 2.0 ** 0.5, 2.0 ** 50
    # far from the end: both constants at least 2^bits
    g = layer_norm_grad_constants(q, 6, 4, SCALE, norm_scale, inv_scale)
    assert min(g.k_grad, -g.k_norm) >= 1 << 16
    # the last prime holds values below 2^49 alone: smaller constants of the same ratio, and a refusal where these do not fit either
    ratio = -g.k_norm / g.k_grad
    small = layer_norm_grad_constants(q, 3, 4, GRAD_SCALE, norm_scale, inv_scale)
    assert small.dx_level == 0 and 2.0 * small.dx_scale < q[0]
    assert abs(-small.k_norm / small.k_grad / ratio - 1) < 2.0 ** -16
    for kw in (dict(grad_scale=SCALE), dict(grad_scale=GRAD_SCALE, largest=2.0 ** 8), dict(grad_scale=GRAD_SCALE, norm_scale=norm_scale * 1.2345678)):
        with pytest.raises(ValueError, match="room"):
            layer_norm_grad_constants(**{**dict(moduli=q, level=3, channels=4, norm_scale=norm_scale, inv_scale=inv_scale), **kw})
    # a ratio that no small constants meet, with fewer bits asked for
    g = layer_norm_grad_constants(q, 3, 4, 2.0 ** 36, norm_scale * 1.2345678, inv_scale, bits=6)
    ratio = float(q[3]) * q[2] / (norm_scale * 1.2345678) ** 2
    assert abs(-g.k_norm / g.k_grad / ratio - 1) <= 2.0 ** -7 and 2.0 * g.dx_scale < q[0]


@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("channels,iterations", [(2, 1), (4, 0), (9, 2), (17, 1)])
def test_layer_norm_that_ends_at_the_last_prime(world, channels, iterations, alike):
    """Without a gain, from the lowest level: norm at level 0, up to sqrt(channels - 1) in magnitude.  The error of 1 / sqrt is relative to the result; the rest as in test_oracle_recurrent.py."""
    w, rng, level = world, np.random.default_rng(channels), 3 + 2 * iterations
    x = channels_of(rng, channels, w.orc.n, alike)
    x[0] *= 1 if channels < 9 else 8  # one channel that holds nearly all of the variance
    var = x.var(0) + EPS
    k = layer_norm_constants(w.p.moduli, level, channels, 2.0 ** 46, (0.99 * var.min(), 1.01 * var.max()), iterations, EPS)
    norm, inv, _ = w.orc.layer_norm(w.encrypt(x, level, 2.0 ** 46), level, k.k_eps, k.k_slope, k.k_start, k.k_newton, w.rlk)
    want, want_inv, _ = layer_norm(x)
    assert k.norm_level == 0
    assert np.abs(w.decrypt(norm, 0, k.norm_scale) - want).max() < BOUND + k.relative_error * np.abs(want).max()
    assert np.abs(w.decrypt([inv], 1, k.inv_scale) - want_inv).max() < BOUND + k.relative_error * want_inv.max()


@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("channels,iterations", [(1, 1), (2, 1), (4, 0), (9, 2)])
def test_root_mean_square_norm_that_ends_at_the_last_prime(world, channels, iterations, alike):
    """The norm without a mean, which shares the chain: outputs at level 0, up to sqrt(channels) where one channel holds nearly everything.  Tolerance as above."""
    w, rng, level = world, np.random.default_rng(channels), 3 + 2 * iterations
    x = channels_of(rng, channels, w.orc.n, alike)
    x[1:] *= 0.05
    square = (x * x).mean(0) + EPS
    k = norm_constants(w.p.moduli, level, channels, 2.0 ** 47, (0.99 * square.min(), 1.01 * square.max()), iterations, EPS)
    out = w.orc.norm_gate(w.encrypt(x, level, 2.0 ** 47), level, k.k_eps, k.k_slope, k.k_start, k.k_newton, w.rlk)
    want = x / np.sqrt(square)
    assert k.out_level == 0
    assert np.abs(w.decrypt(out, 0, k.out_scale) - want).max() < BOUND + k.relative_error * np.abs(want).max()


@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("channels,iterations", [(2, 1), (4, 0), (9, 2)])
def test_layer_norm_with_gain_and_bias_that_ends_at_the_last_prime(world, channels, iterations, alike):
    """From the lowest level: out at level 0.  Its error is the norm's times gains up to 2."""
    w, rng, level = world, np.random.default_rng(channels), 4 + 2 * iterations
    n = w.orc.n
    x, gain, bias = channels_of(rng, channels, n, alike), rng.uniform(1, 2, channels), rng.uniform(-2, 2, channels)
    var = x.var(0) + EPS
    k = layer_norm_constants(w.p.moduli, level, channels, 2.0 ** 46, (0.99 * var.min(), 1.01 * var.max()), iterations, EPS, SCALE, SCALE)
    ct_gain, ct_bias = (w.encrypt(np.repeat(v[:, None], n, 1), 1, SCALE, s) for v, s in ((gain, 40), (bias, 50)))
    norm, inv, out = w.orc.layer_norm(w.encrypt(x, level, 2.0 ** 46), level, k.k_eps, k.k_slope, k.k_start, k.k_newton, w.rlk, ct_gain, ct_bias, k.k_bias)
    want, _, want_out = layer_norm(x, gain, bias)
    assert k.norm_level == 1
    assert np.abs(w.decrypt(norm, 1, k.norm_scale) - want).max() < BOUND + k.relative_error * np.abs(want).max()
    assert np.abs(w.decrypt(out, 0, k.out_scale) - want_out).max() < 2 * (BOUND + k.relative_error * np.abs(want).max())


@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("channels,iterations", [(1, 1), (4, 0), (9, 2)])
def test_root_mean_square_norm_with_gate_or_residual_that_ends_at_the_last_prime(world, channels, iterations, gated, alike):
    """Plaintext gates up to 2, residuals up to 3 with the factor -1.5: outputs at level 0.  A gate multiplies the error of 1 / sqrt, a residual leaves it."""
    w, rng, level = world, np.random.default_rng(channels), 3 + 2 * iterations
    n, gate, residual = w.orc.n, None, None
    x = channels_of(rng, channels, n, alike)
    square = (x * x).mean(0) + EPS
    args = (w.p.moduli, level, channels, 2.0 ** 47, (0.99 * square.min(), 1.01 * square.max()), iterations, EPS)
    want = x / np.sqrt(square)
    if gated:
        values = channels_of(rng, channels, n, alike) * 2
        gate = [w.orc.encode_ntt(row, 2.0 ** 49, level) for row in values]
        want = want * values
        k = norm_constants(*args, gate_scale=2.0 ** 49)
    else:
        values = channels_of(rng, channels, n, alike) * 3
        residual = w.encrypt(values, level, 2.0 ** 46, 70)
        want = want - 1.5 * values
        k = norm_constants(*args, residual=(-1.5, 2.0 ** 46))
    out = w.orc.norm_gate(w.encrypt(x, level, 2.0 ** 47), level, k.k_eps, k.k_slope, k.k_start, k.k_newton, w.rlk, gate, residual, k.k_residual)
    assert k.out_level == 0
    assert np.abs(w.decrypt(out, 0, k.out_scale) - want).max() < 2 * (BOUND + k.relative_error * channels ** 0.5)
