"""Pins of the oracle's transformer-block operators and of the host-side constants: decrypted results against float64 formulas, on a ring
of 2^8 points (128 slots) with 50-bit primes.

Tolerances: a fresh encryption's noise decodes to about sigma sqrt(N) * few / scale, a division by dropped primes rounds each
coefficient by a few units (times the secret's at most N ones), so a result at scale near 2^50 is off by less than 2^20 / 2^50 = 1e-9 per
operation here; the bounds below are a hundred times that, or what quantised weights or the Newton iteration leave by their formulas."""
import numpy as np
import pytest

from oracle import Oracle
from workloads import make_params
from paper_2604_16834_amd.block import (bias_residues, grid_positions, linear_scale, norm_constants, quantise_weights, rope_angles)

SCALE = 2.0 ** 49


@pytest.fixture(scope="module")
def world():
    p = make_params(8, 14, 5, 3)
    orc = Oracle(p)
    s, s_ntt = orc.gen_secret(3)
    return p, orc, s_ntt, orc.gen_relin_key(s_ntt, 4)


def encrypt(orc, s_ntt, z, level, seed, scale=SCALE):
    return [orc.encrypt(row, scale, level, s_ntt, seed + i) for i, row in enumerate(z)]


@pytest.mark.parametrize("bits", [8, 16, 32])
@pytest.mark.parametrize("rows", [(1,), (2, 0, 1)])
def test_grouped_product_is_the_matrix_product(world, bits, rows):
    p, orc, s_ntt, _ = world
    rng, level, c_in, c_out = np.random.default_rng(bits), 3, 5, 3
    w, b = rng.normal(0, 0.3, (len(rows), c_out, c_in)), rng.uniform(-1, 1, (len(rows), c_out))
    x = rng.uniform(-1, 1, (sum(rows), c_in, orc.n))
    qw = quantise_weights(w, p.moduli[level], bits)
    bias = bias_residues(b, qw, SCALE, p.moduli, level)
    got = orc.linear_grouped([encrypt(orc, s_ntt, x[t], level, 50 * t) for t in range(sum(rows))], level, rows, qw.w, qw.multiplier, bias)
    out_scale = linear_scale(SCALE, qw, p.moduli[level])
    for t, g in enumerate(np.repeat(np.arange(len(rows)), rows)):
        want = (qw.w[g] * qw.step) @ x[t] + b[g][:, None]
        dec = np.stack([orc.decrypt(ct, level - 1, s_ntt, out_scale) for ct in got[t]])
        assert np.abs(dec - want).max() < 1e-7
        assert np.abs(want - (w[g] @ x[t] + b[g][:, None])).max() <= c_in * qw.step / 2 + 1e-12  # half a step per weight


@pytest.mark.parametrize("shape,pairs,interleaved", [((64,), (2,), False), ((8, 8), (1, 2), True), ((2, 8, 8), (1, 1, 2), False)])
def test_rotary_positions_turn_pairs_by_their_axis(world, shape, pairs, interleaved):
    p, orc, s_ntt, _ = world
    rng, level, n_pairs = np.random.default_rng(len(shape)), 4, sum(pairs)
    x = rng.uniform(-1, 1, (2 * n_pairs + 1, orc.n))
    pos = grid_positions(shape, orc.n // int(np.prod(shape)), orc.n)
    ang = rope_angles(pos, pairs)
    assert ang.shape == (n_pairs, orc.n)
    side = int(np.prod(shape[1:]))
    assert np.array_equal(pos[0][:int(np.prod(shape))], np.arange(int(np.prod(shape))) // side)
    q = p.moduli[level]
    cos, sin = ([orc.encode_ntt(f(a), float(q), level) for a in ang] for f in (np.cos, np.sin))
    cts = encrypt(orc, s_ntt, x, level, 7)
    out = orc.rope_axes(cts, level, cos, sin, interleaved)
    dec = np.stack([orc.decrypt(ct, level - 1, s_ntt, SCALE) for ct in out])
    z = np.array(x, dtype=complex)
    for j in range(n_pairs):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + n_pairs)
        turned = (x[a] + 1j * x[b]) * np.exp(1j * ang[j])
        z[a], z[b] = turned.real, turned.imag
    assert np.abs(dec - z.real).max() < 1e-7
    # back again with the tables of the level below: the input
    q1 = p.moduli[level - 1]
    cos, sin = ([orc.encode_ntt(f(a), float(q1), level - 1) for a in ang] for f in (np.cos, np.sin))
    back = orc.rope_axes(out, level - 1, cos, sin, interleaved, inverse=True)
    dec = np.stack([orc.decrypt(ct, level - 2, s_ntt, SCALE) for ct in back])
    assert np.abs(dec - x).max() < 1e-7


@pytest.mark.parametrize("iterations", [0, 1, 3, 4])
@pytest.mark.parametrize("gate,residual", [(None, False), ("plain", True), ("cipher", True)])
def test_norm_is_the_root_mean_square_norm(world, iterations, gate, residual):
    p, orc, s_ntt, rlk = world
    rng, level, channels, eps = np.random.default_rng(iterations), 13, 6, 0.01
    x = rng.uniform(-1, 1, (channels, orc.n)) * rng.uniform(0.5, 1.0, orc.n)
    x[:, :3] = 0.0                                    # slots without a token: the norm of nothing is nothing, eps or not
    v = (x * x).mean(0) + eps
    interval = (0.01, 1.02)
    q = p.moduli[level]
    g, res = rng.uniform(-1, 1, (channels, orc.n)), rng.uniform(-1, 1, (channels, orc.n))
    res_scale, factor = 2.0 ** 45, 0.75
    k = norm_constants(p.moduli, level, channels, SCALE, interval, iterations, eps, gate_scale={None: None, "plain": float(q), "cipher": SCALE}[gate],
                       residual=(factor, res_scale) if residual else None)
    gates = {None: None, "plain": [orc.encode_ntt(r, float(q), level) for r in g], "cipher": encrypt(orc, s_ntt, g, level, 500)}[gate]
    out = orc.norm_gate(encrypt(orc, s_ntt, x, level, 100), level, k.k_eps, k.k_slope, k.k_start, k.k_newton, rlk, gates,
                        encrypt(orc, s_ntt, res, level, 700, res_scale) if residual else None, k.k_residual)
    assert k.out_level == level - 3 - 2 * iterations and out[0].shape[1] == k.out_level + 1
    dec = np.stack([orc.decrypt(ct, k.out_level, s_ntt, k.out_scale) for ct in out])
    want = x / np.sqrt(v) * (g if gate else 1.0)
    bound = np.abs(want) * k.relative_error + 1e-6 + (2.0 ** 25 / res_scale if residual else 0.0)
    if residual:
        want = want + factor * res
    assert (np.abs(dec - want) <= bound).all()


def test_the_norm_s_error_bound_holds_for_the_plain_iteration():
    """The line and the Newton steps in float64 over the interval: never above what norm_constants promises, and close to it."""
    p = make_params(8, 14, 5, 3)
    for lo, hi in ((0.5, 1.0), (0.01, 1.0), (1.0, 4000.0)):
        v = np.geomspace(lo, hi, 4001)
        b = (np.sqrt(hi) - np.sqrt(lo)) / (hi ** 1.5 - lo ** 1.5)
        r = 2.0 / (2.0 / 3.0 / np.sqrt(3.0 * b) + np.sqrt(lo) * (1 - b * lo)) * (1 - b * v)
        for iterations in range(6):
            promised = norm_constants(p.moduli, 13, 4, SCALE, (lo, hi), iterations).relative_error
            worst = np.abs(r * np.sqrt(v) - 1).max()
            assert promised / 1.01 - 1e-12 <= worst <= promised * (1 + 1e-6) + 1e-12
            r = r * (3 - v * r * r) / 2


def test_host_side_refusals():
    p = make_params(8, 14, 5, 3)
    with pytest.raises(ValueError):
        quantise_weights([[1.0, float("nan")]], p.moduli[1])
    with pytest.raises(ValueError):
        quantise_weights([[1.0]], p.moduli[1], bits=12)
    with pytest.raises(ValueError):
        grid_positions((16, 16), 2, 256)
    with pytest.raises(ValueError):
        rope_angles(np.zeros((2, 8)), (1,))
    with pytest.raises(ValueError):
        norm_constants(p.moduli, 6, 4, SCALE, (0.1, 1.0), 2)
    with pytest.raises(ValueError):
        norm_constants(p.moduli, 13, 4, 2.0 ** 30, (0.1, 1.0), 2)
    with pytest.raises(ValueError):
        norm_constants(p.moduli, 13, 4, SCALE, (0.0, 1.0), 2)
    assert quantise_weights(np.zeros((2, 2)), p.moduli[1], 8).w.tolist() == [[0, 0], [0, 0]]
