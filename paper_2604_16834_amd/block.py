"""Host-side constants of a transformer block's operators (``he_linear_grouped``, ``he_rope_axes``, ``he_norm_gate``): integers and
angles that a program computes once, with the scales it has to track.  Nothing here touches ciphertexts or the GPU."""
from __future__ import annotations

import math
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


def norm_constants(moduli: Sequence[int], level: int, channels: int, scale: float, interval: Tuple[float, float], iterations: int, eps: float = 0.0,
                   gate_scale: Optional[float] = None, residual: Optional[Tuple[float, float]] = None) -> NormConstants:
    """The integers of ``he_norm_gate`` for inputs at ``scale`` (close to the moduli: the mean square has the scale channels * scale^2 /
    q_level) whose mean squares plus eps lie in ``interval``; gate_scale: the gate's scale; residual: (factor, scale) of the residual.

    The first guess is the line a (1 - b v) whose error against 1 / sqrt(v) is the same at both ends and in the middle; a Newton step turns
    r sqrt(v) = 1 + e into 1 - (3 + e) e^2 / 2, so the first step's worst error is at e > 0 and all later ones come from below.  The scale of r is the one that a step leaves as it is: twice the scale of
    u * w, r^2 and s r each divided by one modulus, the product by another."""
    lo, hi = interval
    if not 0 < lo < hi:
        raise ValueError("need 0 < lo < hi")
    if iterations < 0 or level < 3 + 2 * iterations:
        raise ValueError("need level >= 3 + 2 * iterations")
    q = [float(int(m)) for m in moduli]
    s_scale = channels * scale * scale / q[level]
    sign = -1 if iterations % 2 else 1
    # the line
    b = (math.sqrt(hi) - math.sqrt(lo)) / (hi ** 1.5 - lo ** 1.5)
    top, end = 2.0 / 3.0 / math.sqrt(3.0 * b), math.sqrt(lo) * (1.0 - b * lo)
    a, error = 2.0 / (top + end), (top - end) / (top + end)
    m = level - 2
    r_scale = math.sqrt(q[m] * q[m] * q[max(m - 1, 0)] / (2.0 * s_scale))
    k_eps = round(eps * s_scale)
    k_slope, k_start = round(-sign * a * b * r_scale * q[level - 1] / s_scale), round(sign * a * r_scale)
    newton = []
    for i in range(iterations):
        error = (3.0 + (error if i == 0 else -error)) * error * error / 2.0
        product = 2.0 * (r_scale * r_scale / q[m]) * (s_scale * r_scale / q[m])  # scale of u * w taken as v r^3 / 2
        newton.append(round(-1.5 * product / r_scale))
        r_scale = product / q[m - 1]
        m -= 2
    t_scale = scale if gate_scale is None else scale * gate_scale / q[level]
    k_residual = round(residual[0] * t_scale * r_scale / residual[1]) if residual else 0
    for k in (k_eps, k_slope, k_start, k_residual, *newton):
        if abs(k) >= 1 << 63:
            raise ValueError("a constant passes 63 bits: the inputs' scale is too far from the moduli")
    return NormConstants(k_eps, k_slope, k_start, tuple(newton), k_residual, m - 1, t_scale * r_scale / q[m], error)
