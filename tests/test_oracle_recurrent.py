"""Pins of the oracle's recurrent-block operators and of their host-side constants: decrypted results against float64 formulas and against differences of them, on a ring
of 2^8 points (128 slots) with 50-bit primes.

Tolerances: an operation at a scale near 2^49 is off by less than 2^20 / 2^49 = 2e-9 (fresh encryptions: sigma sqrt(N) times a few; divisions: a few units times the
secret's at most N ones); states and gradients here are at most 20 in magnitude, sums over 128 slots at most 128 of them, and a chain has at most 20 operations whose errors such factors
multiply, which the bound 1e-4 leaves room for; a constant rounded to an integer k adds 1 / (2 k)."""
import numpy as np
import pytest

from oracle import Oracle
from workloads import make_params
from paper_2604_16834_amd.block import (layer_norm_constants, layer_norm_grad_constants, scan_constants, scan_gate_mask, scan_steps, step_constant)

SCALE = 2.0 ** 49
BOUND = 1e-4


class World:
    def __init__(self):
        self.p = make_params(8, 16, 6, 3)
        self.orc = Oracle(self.p)
        self.s, self.s_ntt = self.orc.gen_secret(3)
        self.rlk = self.orc.gen_relin_key(self.s_ntt, 4)
        self.keys = {}

    def rot(self, off):
        if off not in self.keys:
            self.keys[off] = (self.orc.gen_rotation_key(self.s, self.s_ntt, off, 300 + off), self.orc.gen_cross_key(self.s_ntt, off, 600 + off))
        return self.keys[off]

    def encrypt(self, z, level, scale=SCALE, seed=10):
        return [self.orc.encrypt(row, scale, level, self.s_ntt, seed + i) for i, row in enumerate(z)]

    def decrypt(self, cts, level, scale):
        return np.stack([self.orc.decrypt(ct, level, self.s_ntt, scale) for ct in cts])


@pytest.fixture(scope="module")
def world():
    return World()


def recurrence(x, gate):
    """h_t = a_t h_{t-1} + x_t; gate [heads][slots] already zero at the first tokens."""
    h, per = np.zeros_like(x), len(x) // len(gate)
    for t in range(x.shape[1]):
        h[:, t] = x[:, t] + (np.repeat(gate[:, t], per) * h[:, t - 1] if t else 0)
    return h


LENGTHS = [[1, 5, 8, 0, 3, 8, 7, 1, 1, 6, 8], [2] * 60, [16, 16, 13, 1, 15]]


@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("reverse", [False, True])
def test_scan_is_the_recurrence(world, lengths, reverse):
    w, rng, level = world, np.random.default_rng(1), 7
    n, channels, heads = w.orc.n, 4, 2
    steps = scan_steps(max(lengths))
    mask = scan_gate_mask(lengths, n, reverse)
    gate = rng.uniform(-1, 1, (heads, n)) * mask
    x = rng.uniform(-1, 1, (channels, n))
    x[:, sum(lengths):] = 0
    k = scan_constants(w.p.moduli, level, SCALE, 2.0 ** 50, steps)
    sign = 1 if reverse else -1
    keys = [w.rot(sign << s) for s in range(steps)]
    out = w.orc.scan_gated(w.encrypt(x, level), w.encrypt(gate, level, 2.0 ** 50, 50), level, k.k, [a for a, _ in keys], [b for _, b in keys], sign)
    want = recurrence(x[:, ::-1], gate[:, ::-1])[:, ::-1] if reverse else recurrence(x, gate)
    got = w.decrypt(out, k.out_level, k.out_scale)
    assert np.abs(got - want).max() < BOUND
    assert np.abs(got[:, sum(lengths):]).max() < BOUND if sum(lengths) < n else True


@pytest.mark.parametrize("lengths", LENGTHS[:2])
def test_scan_gradients_are_those_of_the_recurrence(world, lengths):
    """The loss sum(upstream * h): its differences along x and along the raw gates, which a mask multiplies."""
    w, rng, level = world, np.random.default_rng(2), 9
    n, channels, heads, steps = w.orc.n, 4, 2, scan_steps(max(lengths))
    mask = scan_gate_mask(lengths, n)
    raw, x, up = rng.uniform(0.2, 1, (heads, n)), rng.uniform(-1, 1, (channels, n)), rng.uniform(-1, 1, (channels, n))
    k = scan_constants(w.p.moduli, level, SCALE, 2.0 ** 50, steps)
    fwd, bwd = [w.rot(-(1 << s)) for s in range(steps)], [w.rot(1 << s) for s in range(steps)]
    gates = w.encrypt(raw * mask, level, 2.0 ** 50, 50)
    states = w.orc.scan_gated(w.encrypt(x, level), gates, level, k.k, [a for a, _ in fwd], [b for _, b in fwd])
    dx, dgate = w.orc.scan_gated_backward(w.encrypt(up, level, seed=80), gates, states, level, k.k, [a for a, _ in bwd], [b for _, b in bwd], *w.rot(-1))
    got_x = w.decrypt(dx, k.out_level, k.out_scale)
    got_a = w.decrypt(dgate, k.out_level - 1, k.out_scale ** 2 / w.p.moduli[k.out_level]) * mask
    # the formulas
    d = recurrence(up[:, ::-1], np.roll(raw * mask, -1, 1)[:, ::-1])[:, ::-1]
    h = recurrence(x, raw * mask)
    da = (d * np.roll(h, 1, 1)).reshape(heads, channels // heads, n).sum(1) * mask
    assert np.abs(got_x - d).max() < BOUND and np.abs(got_a - da).max() < BOUND
    # differences: central ones of a loss that is linear in x and, one gate at a time, linear in a gate, so exact but for rounding
    loss = lambda x_, raw_: float((up * recurrence(x_, raw_ * mask)).sum())  # noqa: E731
    for _ in range(12):
        i, c, hd = int(rng.integers(n)), int(rng.integers(channels)), int(rng.integers(heads))
        e = np.zeros_like(x)
        e[c, i] = 0.5
        assert abs(loss(x + e, raw) - loss(x - e, raw) - got_x[c, i]) < BOUND
        e = np.zeros_like(raw)
        e[hd, i] = 0.5
        assert abs(loss(x, raw + e) - loss(x, raw - e) - got_a[hd, i]) < BOUND


@pytest.mark.parametrize("shift", [0, -1, 3])
def test_step_is_one_step_of_the_recurrence(world, shift):
    w, rng, level = world, np.random.default_rng(3), 2
    n = w.orc.n
    a, h, x = rng.uniform(-1, 1, (1, n)), rng.uniform(-1, 1, (1, n)), rng.uniform(-1, 1, (1, n))
    k, scale = step_constant(w.p.moduli, level, 2.0 ** 50, SCALE, 2.0 ** 47)
    ca, ch, cx = w.encrypt(a, level, 2.0 ** 50)[0], w.encrypt(h, level)[0], w.encrypt(x, level, 2.0 ** 47)[0]
    if shift:
        out = w.orc.turned_product(ca, ch, level, shift, *w.rot(shift), k, cx)
    else:
        out = w.orc.ctct_mul_relin_rescale(ca, ch, w.rlk, level, addend=w.orc.scalar_mul(cx, w.orc.scalar_residues(k, level), level))
    assert np.abs(w.decrypt([out], level - 1, scale) - (a * np.roll(h, -shift, 1) + x)).max() < BOUND


def test_a_rotated_product_is_the_product_with_the_rotation(world):
    """Same slots as a rotation followed by a product, one rounding less: other residues."""
    w, rng, level = world, np.random.default_rng(4), 5
    a, h = w.encrypt(rng.uniform(-1, 1, (2, w.orc.n)), level)
    rot, cross = w.rot(2)
    one = w.orc.turned_product(a, h, level, 2, rot, cross)
    two = w.orc.ctct_mul_relin_rescale(a, w.orc.rotate(h, level, 2, rot, hoisted=True), w.rlk, level)
    scale = SCALE * SCALE / w.p.moduli[level]
    assert np.abs(w.decrypt([one], level - 1, scale) - w.decrypt([two], level - 1, scale)).max() < BOUND
    assert not np.array_equal(one, two)


EPS = 0.01


def layer_norm(x, gain=None, bias=None):
    mu = x.mean(0)
    inv = 1.0 / np.sqrt(x.var(0) + EPS)
    norm = (x - mu) * inv
    return norm, inv, norm if gain is None else gain[:, None] * norm + bias[:, None]


@pytest.mark.parametrize("affine", [False, True])
@pytest.mark.parametrize("channels", [2, 5])
def test_layer_norm_and_its_gradients(world, channels, affine):
    w, rng, level, its = world, np.random.default_rng(channels), 15, 3
    n = w.orc.n
    x = rng.uniform(0.4, 1.0, (channels, n)) * np.where(np.arange(channels) % 2, -1, 1)[:, None] + rng.uniform(-0.5, 0.5, n)
    gain, bias, up = rng.uniform(0.5, 1.5, channels), rng.uniform(-1, 1, channels), rng.uniform(-1, 1, (channels, n))
    var = x.var(0) + EPS
    lo, hi = var.min(), var.max()
    k = layer_norm_constants(w.p.moduli, level, channels, 2.0 ** 47, (lo, hi), its, EPS, *((SCALE, SCALE) if affine else ()))
    spread = lambda v, lv, seed: w.encrypt(np.repeat(v[:, None], n, 1), lv, SCALE, seed)  # noqa: E731
    m = k.norm_level
    cg, cb = (spread(gain, m, 40), spread(bias, m, 50)) if affine else (None, None)
    norm, inv, out = w.orc.layer_norm(w.encrypt(x, level, 2.0 ** 47), level, k.k_eps, k.k_slope, k.k_start, k.k_newton, w.rlk, cg, cb, k.k_bias)
    want_norm, want_inv, want = layer_norm(x, gain, bias) if affine else layer_norm(x)
    slack = 4 * k.relative_error  # of values up to 2.1, gains up to 1.5
    assert k.relative_error < 1e-3
    assert np.abs(w.decrypt([inv], m + 1, k.inv_scale) - want_inv).max() < BOUND + slack * want_inv.max()
    assert np.abs(w.decrypt(norm, m, k.norm_scale) - want_norm).max() < BOUND + slack
    if affine:
        assert np.abs(w.decrypt(out, m - 1, k.out_scale) - want).max() < BOUND + slack
    # backward from the level of norm, sums over eight slots by 1 + 1, 2 + 2, 4 + 4 or 1 .. 7 at once
    g = layer_norm_grad_constants(w.p.moduli, m, channels, SCALE, k.norm_scale, k.inv_scale, SCALE if affine else None)
    stages = [((1,), [w.rot(1)[0]]), ((2, 4, 6), [w.rot(o)[0] for o in (2, 4, 6)])]
    dx, dgain, dbias = w.orc.layer_norm_backward(w.encrypt(up, m, seed=90), norm, inv, m, g.k_grad, g.k_norm, w.rlk, cg, stages)
    gy = up * gain[:, None] if affine else up
    want_dx = want_inv * (gy - gy.mean(0) - want_norm * (gy * want_norm).mean(0))
    got_dx = w.decrypt(dx, g.dx_level, g.dx_scale)
    # norm and inv enter three times; |dx| parts below 12
    assert np.abs(got_dx - want_dx).max() < BOUND + 12 * (slack + 2.0 ** -16) * want_inv.max()
    eight = lambda v: sum(np.roll(v, -i, 1) for i in range(8))  # noqa: E731
    assert np.abs(w.decrypt(dgain, m - 1, g.dgain_scale) - eight(up * want_norm)).max() < BOUND + 8 * slack
    assert np.abs(w.decrypt(dbias, m - 1, g.dbias_scale) - eight(up)).max() < BOUND
    # differences of the loss sum(upstream * out), central ones: off by the step squared times a third derivative below 6 * 20 * inv^3
    loss = lambda v: float((up * layer_norm(v, *((gain, bias) if affine else ()))[2]).sum())  # noqa: E731
    step = 1e-4
    for _ in range(8):
        e = np.zeros_like(x)
        at = int(rng.integers(channels)), int(rng.integers(n))
        e[at] = step
        slope = (loss(x + e) - loss(x - e)) / (2 * step)
        assert abs(slope - want_dx[at]) < 20 * step * step * want_inv.max() ** 3 + 1e-9


def test_layer_norm_of_one_channel_is_zero(world):
    w, rng, level = world, np.random.default_rng(9), 5
    x = rng.uniform(-1, 1, (1, w.orc.n))
    k = layer_norm_constants(w.p.moduli, level, 1, SCALE, (0.5, 1.5), 1, 1.0)
    norm, inv, _ = w.orc.layer_norm(w.encrypt(x, level), level, k.k_eps, k.k_slope, k.k_start, k.k_newton, w.rlk)
    assert np.abs(w.decrypt(norm, k.norm_level, k.norm_scale)).max() < BOUND
    assert np.abs(w.decrypt([inv], k.norm_level + 1, k.inv_scale) - 1.0).max() < BOUND + 4 * k.relative_error


def test_constants_refuse_what_they_cannot_serve():
    q = make_params(8, 8, 3, 3).moduli
    with pytest.raises(ValueError):
        scan_constants(q, 3, SCALE, 2.0 ** 50, 4)
    with pytest.raises(ValueError):
        scan_constants(q, 3, SCALE, 2.0 ** 50, 0)
    with pytest.raises(ValueError):
        scan_constants(q, 7, SCALE, 2.0 ** 20, 6)   # the gates' scale falls below one
    with pytest.raises(ValueError):
        scan_constants(q, 7, SCALE, 2.0 ** 63, 1)
    with pytest.raises(ValueError):
        step_constant(q, 2, 2.0 ** 60, 2.0 ** 60, 1.0)
    with pytest.raises(ValueError):
        layer_norm_constants(q, 4, 4, SCALE, (0.5, 1.0), 1)
    with pytest.raises(ValueError):
        layer_norm_constants(q, 5, 4, SCALE, (0.5, 1.0), 1, gain_scale=SCALE)
    with pytest.raises(ValueError):
        layer_norm_constants(q, 7, 4, SCALE, (1.0, 0.5), 1)
    with pytest.raises(ValueError):
        layer_norm_grad_constants(q, 3, 4, SCALE, SCALE, SCALE, gain_scale=SCALE)
    with pytest.raises(ValueError):
        scan_gate_mask([5, 4], 8)
    with pytest.raises(ValueError):
        scan_gate_mask([-1], 8)
    assert [scan_steps(n) for n in (1, 2, 3, 4, 5, 4096)] == [1, 1, 2, 2, 3, 12]
    with pytest.raises(ValueError):
        scan_steps(0)
    assert scan_gate_mask([1, 3, 0, 2], 8).tolist() == [0, 0, 1, 1, 0, 1, 0, 0] and scan_gate_mask([1, 3, 0, 2], 8, True).tolist() == [0, 1, 1, 0, 1, 0, 0, 0]


def test_the_examples_gradients_are_differences():
    """examples/encrypted_recurrence.py: its float64 gradients against central differences of its loss sum(upstream * states).  The loss is linear in gain and bias and in each gate alone
    (exact but for rounding); along the inputs a step of 1e-4 leaves its square times a third derivative, below 1e3 here (inv^3 up to 30, states' sums up to 30)."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "encrypted_recurrence.py")
    spec = importlib.util.spec_from_file_location("encrypted_recurrence", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    rng, n = np.random.default_rng(0), 24
    mask = scan_gate_mask([3, 8, 1, 5, 7], n)
    x = rng.uniform(0.4, 1.0, (ex.CHANNELS, n)) * np.array([1.0, -1.0, 1.0, -1.0])[:, None]
    gain, bias, up, gate = rng.uniform(0.5, 1.5, ex.CHANNELS), rng.uniform(-1, 1, ex.CHANNELS), rng.uniform(-1, 1, (ex.CHANNELS, n)), rng.uniform(0.3, 1.0, (ex.HEADS, n)) * mask
    _, dx, dgate, dgain, dbias = ex.reference(x, gain, bias, gate, up)
    loss = lambda x, gain, bias, gate: float((up * ex.recurrence(ex.layer_norm(x, gain, bias)[2], gate)).sum())  # noqa: E731

    def slope(which, at, step):
        args = [x, gain, bias, gate]
        ends = []
        for sign in (1, -1):
            moved = args[which].copy()
            moved[at] += sign * step
            ends.append(loss(*args[:which], moved, *args[which + 1:]))
        return (ends[0] - ends[1]) / (2 * step)

    for _ in range(20):
        c, t, h = int(rng.integers(ex.CHANNELS)), int(rng.integers(n)), int(rng.integers(ex.HEADS))
        assert abs(slope(0, (c, t), 1e-4) - dx[c, t]) < 1e-5
        assert abs(slope(1, c, 0.5) - dgain[c].sum()) < 1e-9
        assert abs(slope(2, c, 0.5) - dbias[c].sum()) < 1e-9
        if mask[t]:
            assert abs(slope(3, (h, t), 0.5) - dgate[h, t]) < 1e-9
