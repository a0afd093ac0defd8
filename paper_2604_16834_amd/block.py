"""Host-side constants of a transformer block's operators (``he_linear_grouped``, ``he_rope_axes``, ``he_norm_gate``) and of a recurrent
block's (``he_scan_gated``, ``he_layer_norm`` and their backward passes): integers and angles that a program computes once, with the
scales it has to track.  Nothing here touches ciphertexts or the GPU."""
from __future__ import annotations

import math
from fractions import Fraction
from typing import NamedTuple, Optional, Sequence, Tuple

import numpy as np


# ------------------------------------------------------------------------------------------ grouped products
class QuantisedWeights(NamedTuple):
    w: np.ndarray      # int8, int16 or int32, the shape of the weights
    multiplier: int    # what he_linear_grouped multiplies its sums by
    step: float        # a weight is w * step

    def bias_scale(self, scale: float) -> float:
        """The scale at which a bias joins the sums of inputs at ``scale`` (before the division by q_level)."""
        return scale * self.multiplier / self.step


def quantise_weights(weights, q_level: int, bits: int = 32, gain: float = 1.0) -> QuantisedWeights:
    """Weights rounded to integers of 8, 16 or 32 bits, and the multiplier round(step * q_level * gain): the product's outputs have `gain` times the scale of its
    inputs but for the rounding (the multiplier is one at least: where step * q_level * gain is below that, as with short moduli, the scale grows by more), exactly
    what ``linear_scale`` gives."""
    w = np.asarray(weights, dtype=np.float64)
    if bits not in (8, 16, 32):
        raise ValueError("bits must be 8, 16 or 32")
    if not 0.0 < gain < math.inf:
        raise ValueError("gain must be positive and finite")
    top = float(np.abs(w).max()) if w.size else 0.0
    if not math.isfinite(top):
        raise ValueError("weights must be finite")
    # below 2^-(bits - 1) of q the multiplier would lose the step's accuracy: steps are kept above 2^-40
    step = max(top / (2 ** (bits - 1) - 1), 2.0 ** -40)
    dtype = {8: np.int8, 16: np.int16, 32: np.int32}[bits]
    multiplier = max(1, round(step * q_level * gain))
    if multiplier >= 1 << 64:
        raise ValueError("the multiplier passes 64 bits")
    return QuantisedWeights(np.round(w / step).astype(dtype), multiplier, step)


def linear_scale(scale: float, weights: QuantisedWeights, q_level: int) -> float:
    """Scale of he_linear_grouped's outputs for inputs at ``scale``."""
    return scale * weights.multiplier / weights.step / q_level


def bias_residues(bias, weights: QuantisedWeights, scale: float, moduli: Sequence[int], level: int) -> np.ndarray:
    """uint64[..., level + 1]: residues of a bias at the scale of the sums."""
    b = np.asarray(bias, dtype=np.float64)
    big = [int(round(float(v) * weights.bias_scale(scale))) for v in b.reshape(-1)]
    return np.array([[v % int(moduli[i]) for i in range(level + 1)] for v in big], dtype=np.uint64).reshape(*b.shape, level + 1)


# ------------------------------------------------------------------------------------------ rotary positions
def grid_positions(shape: Sequence[int], batch: int, slots: int) -> np.ndarray:
    """[axes][slots]: the position on every axis of the token in each slot, for ``batch`` grids (images: height, width; videos: time,
    height, width) packed one after the other in row-major order, as channel-by-channel packing has them; 0 in unused slots."""
    size = math.prod(shape)
    if size * batch > slots:
        raise ValueError("the grids do not fit the slots")
    out = np.zeros((len(shape), slots), dtype=np.int64)
    one = np.stack([axis.reshape(-1) for axis in np.meshgrid(*[np.arange(n) for n in shape], indexing="ij")])
    out[:, :size * batch] = np.tile(one, batch)
    return out


def rope_angles(positions: np.ndarray, axis_pairs: Sequence[int], base: float = 10000.0) -> np.ndarray:
    """[pairs][slots]: pair i of the axis_pairs[a] pairs on axis a turns by positions[a] * base^(-i / axis_pairs[a]); the pairs of an axis
    follow each other.  Angles are products in double precision: exact to 2^-53 of the position."""
    positions = np.asarray(positions)
    if len(positions) != len(axis_pairs):
        raise ValueError("need the positions on every axis")
    rows = [positions[a].astype(np.float64) * base ** (-i / n) for a, n in enumerate(axis_pairs) for i in range(n)]
    return np.stack(rows) if rows else np.zeros((0, positions.shape[-1]))


# ------------------------------------------------------------------------------------------ norm
class NormConstants(NamedTuple):
    k_eps: int
    k_slope: int
    k_start: int
    k_newton: Tuple[int, ...]
    k_residual: int
    out_level: int           # level of the outputs
    out_scale: float
    relative_error: float    # of 1 / sqrt after the last iteration, at most, for mean squares inside the interval


class _InverseRoot(NamedTuple):
    k_eps: int
    k_slope: int
    k_start: int
    k_newton: Tuple[int, ...]
    level: int
    scale: float
    relative_error: float


def _check_chain(level: int, iterations: int) -> None:
    if iterations < 0 or level < 3 + 2 * iterations:
        raise ValueError("need level >= 3 + 2 * iterations")


def _inverse_root(q: Sequence[float], level: int, s_scale: float, interval: Tuple[float, float], iterations: int, eps: float, most: float = math.inf) -> _InverseRoot:
    """The guess and the Newton steps of 1 / sqrt(v) for v at ``s_scale``, level - 1 (see ``norm_constants``); most: a bound on the scale of the result."""
    lo, hi = interval
    if not 0 < lo < hi:
        raise ValueError("need 0 < lo < hi")
    sign = -1 if iterations % 2 else 1
    # the line
    b = (math.sqrt(hi) - math.sqrt(lo)) / (hi ** 1.5 - lo ** 1.5)
    top, end = 2.0 / 3.0 / math.sqrt(3.0 * b), math.sqrt(lo) * (1.0 - b * lo)
    a, error = 2.0 / (top + end), (top - end) / (top + end)
    m = level - 2
    r_scale = math.sqrt(q[m] * q[m] * q[max(m - 1, 0)] / (2.0 * s_scale))
    last = r_scale  # behind the steps
    for n in range(m, m - 2 * iterations, -2):
        last = 2.0 * (last * last / q[n]) * (s_scale * last / q[n]) / q[n - 1]
    if most < last < math.inf:  # every step cubes what the scale is below the one that stays
        r_scale *= (most / last) ** (3.0 ** -iterations)
    k_eps = round(eps * s_scale)
    k_slope, k_start = round(-sign * a * b * r_scale * q[level - 1] / s_scale), round(sign * a * r_scale)
    newton = []
    for i in range(iterations):
        error = (3.0 + (error if i == 0 else -error)) * error * error / 2.0
        product = 2.0 * (r_scale * r_scale / q[m]) * (s_scale * r_scale / q[m])  # scale of u * w taken as v r^3 / 2
        newton.append(round(-1.5 * product / r_scale))
        r_scale = product / q[m - 1]
        m -= 2
    return _InverseRoot(k_eps, k_slope, k_start, tuple(newton), m, r_scale, error)


def _check_int64(*values: int) -> None:
    if any(not -(1 << 63) < k < 1 << 63 for k in values):
        raise ValueError("a constant passes 63 bits: the inputs' scale is too far from the moduli")


def _room(q: Sequence[float], level: int) -> float:
    """What a value times its scale may be at ``level``: coefficients are at most that, below half the product q_0 .. q_level with a part left for noise."""
    return math.prod(q[:level + 1]) * (0.5 - 2.0 ** -7)


def norm_constants(moduli: Sequence[int], level: int, channels: int, scale: float, interval: Tuple[float, float], iterations: int, eps: float = 0.0,
                   gate_scale: Optional[float] = None, residual: Optional[Tuple[float, float]] = None, largest: Optional[float] = None) -> NormConstants:
    """The integers of ``he_norm_gate`` for inputs at ``scale`` (close to the moduli: the mean square has the scale channels * scale^2 /
    q_level) whose mean squares plus eps lie in ``interval``; gate_scale: the gate's scale; residual: (factor, scale) of the residual.

    The first guess is the line a (1 - b v) whose error against 1 / sqrt(v) is the same at both ends and in the middle; a Newton step turns
    r sqrt(v) = 1 + e into 1 - (3 + e) e^2 / 2, so the first step's worst error is at e > 0 and all later ones come from below.  The scale of r is the one that a step leaves as it is: twice the scale of
    u * w, r^2 and s r each divided by one modulus, the product by another.  Where outputs end at level 0 it is one at which they fit: without gate and residual they are at most
    sqrt(channels) in magnitude; largest: a bound on them with either, sixteen times that if not given."""
    q = [float(int(m)) for m in moduli]
    _check_chain(level, iterations)
    last = level - 2 - 2 * iterations
    t_scale = scale if gate_scale is None else scale * gate_scale / q[level]
    bound = math.sqrt(channels)
    if gate_scale is not None or residual is not None:
        bound = 16.0 * bound if largest is None else largest
    r = _inverse_root(q, level, channels * scale * scale / q[level], interval, iterations, eps, _room(q, last - 1) / bound * q[last] / t_scale)
    k_residual = round(residual[0] * t_scale * r.scale / residual[1]) if residual else 0
    _check_int64(r.k_eps, r.k_slope, r.k_start, k_residual, *r.k_newton)
    return NormConstants(r.k_eps, r.k_slope, r.k_start, r.k_newton, k_residual, r.level - 1, t_scale * r.scale / q[r.level], r.relative_error)


# ------------------------------------------------------------------------------------------ layer norm
class LayerNormConstants(NamedTuple):
    k_eps: int
    k_slope: int
    k_start: int
    k_newton: Tuple[int, ...]
    k_bias: int
    norm_level: int          # of the normalised channels; inv is one level above, the output with gain and bias one below
    norm_scale: float
    inv_scale: float
    out_scale: float         # with a gain; norm_scale without
    relative_error: float    # of 1 / sqrt after the last iteration, at most, for variances inside the interval


def layer_norm_constants(moduli: Sequence[int], level: int, channels: int, scale: float, interval: Tuple[float, float], iterations: int, eps: float = 0.0,
                         gain_scale: Optional[float] = None, bias_scale: Optional[float] = None, largest: Optional[float] = None) -> LayerNormConstants:
    """The integers of ``he_layer_norm`` for inputs at ``scale`` whose variances over the channels plus eps lie in ``interval``: what the Newton chain works on is channels^2
    times the variance, at the scale channels^2 scale^2 / q_level; the centred channels have channels times the inputs' scale.  norm, at most sqrt(channels - 1) in magnitude, has
    the scale that a Newton step leaves as it is, or one at which it, and with a gain out, fits where that ends at level 0; largest: a bound on |out| with a gain, sixteen times
    norm's if not given."""
    q = [float(int(m)) for m in moduli]
    _check_chain(level, iterations)
    if gain_scale is not None and level < 4 + 2 * iterations:
        raise ValueError("a gain needs one more level")
    last, bound = level - 2 - 2 * iterations, math.sqrt(max(channels - 1, 1))
    most = _room(q, last - 1) / bound  # norm's scale
    if gain_scale is not None:
        most = min(most, _room(q, last - 2) / (16.0 * bound if largest is None else largest) * q[last - 1] / gain_scale)
    r = _inverse_root(q, level, channels * channels * scale * scale / q[level], interval, iterations, eps, most * q[last] / (channels * scale))
    norm_scale, m = channels * scale * r.scale / q[r.level], r.level - 1
    k_bias = round(gain_scale * norm_scale / bias_scale) if gain_scale is not None and bias_scale is not None else 0
    _check_int64(r.k_eps, r.k_slope, r.k_start, k_bias, *r.k_newton)
    return LayerNormConstants(r.k_eps, r.k_slope, r.k_start, r.k_newton, k_bias, m, norm_scale, r.scale, norm_scale if gain_scale is None else gain_scale * norm_scale / q[m],
                              r.relative_error)


class LayerNormGradConstants(NamedTuple):
    k_grad: int
    k_norm: int
    dx_level: int
    dx_scale: float
    dgain_scale: float       # dgain and dbias are at level - 1
    dbias_scale: float


def layer_norm_grad_constants(moduli: Sequence[int], level: int, channels: int, grad_scale: float, norm_scale: float, inv_scale: float, gain_scale: Optional[float] = None,
                              bits: int = 16, largest: float = 1.0) -> LayerNormGradConstants:
    """The integers of ``he_layer_norm_backward`` for a gradient at ``grad_scale``: k_norm / k_grad is minus the ratio of the scales of the two terms of
    channels * dx, to within 2^-(bits + 1); dx's scale holds the factors channels and k_grad.  Both integers are at least 2^bits, or, where dx's modulus has no room for that
    (at level 3, with a gain 4, a single prime is left), the smallest found that meet the ratio as closely: small ones do where it is close to a simple fraction, as it is for a norm of
    ``layer_norm_constants``.  largest: a bound on |dx|.  Raises ValueError where dx does not fit: a smaller grad_scale, fewer bits or a level more are needed then."""
    q = [float(int(m)) for m in moduli]
    if level < (3 if gain_scale is None else 4):
        raise ValueError("need level >= 3, 4 with a gain")
    b = level if gain_scale is None else level - 1
    g_scale = grad_scale if gain_scale is None else gain_scale * grad_scale / q[level]
    t_scale = inv_scale * (g_scale * norm_scale / q[b]) / q[b - 1]
    ratio = inv_scale * g_scale / (t_scale * norm_scale)
    unit = channels * inv_scale * g_scale / q[b - 2]  # dx's scale for k_grad = 1
    most = _room(q, b - 3) / (unit * largest)
    k_grad = max(1, math.ceil(2.0 ** bits * max(1.0, 1.0 / ratio)))
    if k_grad > most:
        span, exact = 1, Fraction(ratio)
        while span < k_grad:
            near = exact.limit_denominator(span)
            if abs(near / exact - 1) <= Fraction(2.0 ** -(bits + 1)):
                k_grad = near.denominator
            span *= 2
        if k_grad > most:
            raise ValueError("no room for dx at its level: its scale times its largest value passes half of the modulus that is left")
    k_norm = -round(k_grad * ratio)
    _check_int64(k_grad, k_norm)
    return LayerNormGradConstants(k_grad, k_norm, b - 3, k_grad * unit, grad_scale * norm_scale / q[level], grad_scale)


# ------------------------------------------------------------------------------------------ gated recurrence
class ScanConstants(NamedTuple):
    k: Tuple[int, ...]       # one integer a step
    out_level: int
    out_scale: float


def scan_steps(longest: int) -> int:
    """Doublings of a scan over sequences of at most ``longest`` tokens (one at least: the call has no scan without a step)."""
    if longest < 1:
        raise ValueError("a sequence has at least one token")
    return max(1, (longest - 1).bit_length())


def scan_gate_mask(lengths: Sequence[int], slots: int, reverse: bool = False) -> np.ndarray:
    """[slots]: 0 where a gate has to be zero, the first token (reverse: the last) of every sequence and the padding behind the last one; 1 elsewhere."""
    lengths = [int(n) for n in lengths]
    if any(n < 0 for n in lengths) or sum(lengths) > slots:
        raise ValueError("the sequences do not fit the slots")
    mask, start = np.zeros(slots), 0
    for n in lengths:
        if reverse:
            mask[start:start + max(n - 1, 0)] = 1.0
        else:
            mask[start + 1:start + n] = 1.0
        start += n
    return mask


def scan_constants(moduli: Sequence[int], level: int, scale: float, gate_scale: float, steps: int) -> ScanConstants:
    """The integers of ``he_scan_gated`` (and of its backward pass) for inputs at ``scale`` and gates at ``gate_scale``: at every step the gates' scale, rounded, as what is
    carried on has to join a product with them.  Scales stay where gate_scale is close to the moduli: out_scale times the largest state or
    gradient has to stay below half of q_0 .. q_out_level, which at level 0 is the caller's to see to, by ``scale``."""
    if not 1 <= steps <= level:
        raise ValueError("need 1 <= steps <= level")
    q, k = [float(int(m)) for m in moduli], []
    for s in range(steps):
        k.append(round(gate_scale))
        scale, gate_scale = scale * gate_scale / q[level - s], gate_scale * gate_scale / q[level - s]
    _check_int64(*k)
    if min(k) < 1:
        raise ValueError("the gates' scale falls below one")
    return ScanConstants(tuple(k), level - steps, scale)


def step_constant(moduli: Sequence[int], level: int, gate_scale: float, state_scale: float, x_scale: float) -> Tuple[int, float]:
    """The integer of ``he_scan_step`` and the scale of its outputs."""
    k = round(gate_scale * state_scale / x_scale)
    _check_int64(k)
    return k, gate_scale * state_scale / float(int(moduli[level]))
