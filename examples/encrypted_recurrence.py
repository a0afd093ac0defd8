"""Forward and backward pass of a recurrent block on encrypted sequences, one call after the other as a training server makes them:

    layer norm with encrypted gain and bias  ->  gated recurrence over ragged sequences  ->  the next token of every sequence
    upstream gradient  ->  gradients of the recurrence's inputs and gates  ->  gradients of the norm's inputs, and of gain and bias summed over all tokens

Four channels in two heads; the slots hold sequences of one to eight tokens, one after the other.  The client's side (keys, encryption, decryption) is the CPU oracle's, the
server's the library's calls and ``block.py`` for their constants.  Decrypted results are compared with the same block in float64.

    python examples/encrypted_recurrence.py            # needs an MI355X
"""
import argparse
import os
import sys
import time

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2604_16834_amd as hx  # noqa: E402
from paper_2604_16834_amd.block import (layer_norm_constants, layer_norm_grad_constants, scan_constants, scan_gate_mask, scan_steps, step_constant)  # noqa: E402
from oracle import Oracle  # noqa: E402
from workloads import make_params  # noqa: E402

CHANNELS, HEADS, EPS, ITERATIONS = 4, 2, 0.01, 3
SCALE, GATE_SCALE = 2.0 ** 48, 2.0 ** 50


def layer_norm(x, gain, bias):
    inv = 1.0 / np.sqrt(x.var(0) + EPS)
    norm = (x - x.mean(0)) * inv
    return norm, inv, gain[:, None] * norm + bias[:, None]


def recurrence(x, gate):
    """h_t = a_t h_{t-1} + x_t; x [channels][slots], gate [heads][slots], zero at every sequence's first token."""
    a, h = np.repeat(gate, len(x) // len(gate), 0), np.zeros_like(x)
    for t in range(x.shape[1]):
        h[:, t] = x[:, t] + (a[:, t] * h[:, t - 1] if t else 0.0)
    return h


def reference(x, gain, bias, gate, up):
    """The block and its gradients in float64: (states, d x, d gate, d gain, d bias), the last two per token."""
    norm, inv, y = layer_norm(x, gain, bias)
    h = recurrence(y, gate)
    dy = recurrence(up[:, ::-1], np.roll(gate, -1, 1)[:, ::-1])[:, ::-1]
    dgate = (dy * np.roll(h, 1, 1)).reshape(HEADS, -1, x.shape[1]).sum(1)
    g = gain[:, None] * dy
    return h, inv * (g - g.mean(0) - norm * (g * norm).mean(0)), dgate, dy * norm, dy


class Client:
    """Keys, encryption and decryption."""

    def __init__(self, ctx, params, seed):
        self.ctx, self.orc, self.seed = ctx, Oracle(params), seed
        self.s, self.s_ntt = self.orc.gen_secret(seed)
        self.rlk = hx.ckks_key_load(ctx, hx.from_host(self.orc.gen_relin_key(self.s_ntt, seed + 1)), 0)

    def rotation(self, offset, cross=True):
        """The rotation's key and its cross key."""
        g = self.orc.galois(offset)
        keys = [hx.ckks_key_load(self.ctx, hx.from_host(self.orc.gen_rotation_key(self.s, self.s_ntt, offset, self.seed + 7 + offset)), g)]
        if cross:
            keys.append(hx.ckks_key_load(self.ctx, hx.from_host(self.orc.gen_cross_key(self.s_ntt, offset, self.seed + 5007 + offset)), hx.CKKS_KEY_CROSS | g))
        return keys

    def encrypt(self, z, level, scale, seed):
        return hx.from_host(np.stack([self.orc.encrypt(row, scale, level, self.s_ntt, self.seed + seed + i) for i, row in enumerate(z)]))

    def decrypt(self, cts, level, scale):
        return np.stack([self.orc.decrypt(ct, level, self.s_ntt, scale) for ct in hx.to_host(cts)])


def run(log_n=12, seed=0, verbose=True):
    """Returns {result: (largest difference from float64 relative to its largest value, bound on it)}."""
    p = make_params(log_n, 24, 8, 3)
    ctx = hx.Context(p)
    client = Client(ctx, p, seed)
    n, rng = client.orc.n, np.random.default_rng(seed)
    lengths, left = [], n
    while left:
        lengths.append(min(left, int(rng.integers(1, 9))))
        left -= lengths[-1]
    steps, mask = scan_steps(8), scan_gate_mask(lengths, n)
    x = rng.uniform(0.4, 1.0, (CHANNELS, n)) * np.array([1.0, -1.0, 1.0, -1.0])[:, None] + rng.uniform(-0.5, 0.5, n)
    gain, bias, up = rng.uniform(0.5, 1.5, CHANNELS), rng.uniform(-1, 1, CHANNELS), rng.uniform(-1, 1, (CHANNELS, n))
    gate, token = rng.uniform(0.3, 1.0, (HEADS, n)) * mask, rng.uniform(-1, 1, (CHANNELS, n))
    want = reference(x, gain, bias, gate, up)

    # keys: rotations by 1, 2, 4 either way with their cross keys; for the sums over all slots rotations by 1, 2, 3, then 4, 8, 12, ...
    fwd, bwd = [client.rotation(-(1 << s)) for s in range(steps)], [client.rotation(1 << s) for s in range(steps)]
    sums, span = [], 1
    while span < n:
        sums.append([client.rotation(j * span, cross=False)[0] for j in range(1, min(4, n // span))])
        span *= len(sums[-1]) + 1

    # 1. layer norm
    top = p.num_q - 1
    var = x.var(0) + EPS
    k = layer_norm_constants(p.moduli, top, CHANNELS, SCALE, (var.min(), var.max()), ITERATIONS, EPS, SCALE, SCALE)
    ct_x = client.encrypt(x, top, SCALE, 100)
    ct_gain, ct_bias = (client.encrypt(np.repeat(v[:, None], n, 1), k.norm_level, SCALE, s) for v, s in ((gain, 200), (bias, 300)))
    ct_gate, ct_token = client.encrypt(gate, k.norm_level, GATE_SCALE, 400), client.encrypt(token, k.norm_level, SCALE, 500)
    start = time.perf_counter()
    norm, inv, y = hx.he_layer_norm(ctx, top, ct_x, k.k_eps, k.k_slope, k.k_start, k.k_newton, client.rlk, gain=ct_gain, bias=ct_bias, k_bias=k.k_bias)
    level = k.norm_level - 1

    # 2. the recurrence (the gates were encrypted a level above: their first limbs are read), and one more token: every stream's state in its last token's slot moves
    # to the next slot
    c = scan_constants(p.moduli, level, k.out_scale, GATE_SCALE, steps)
    h = hx.he_scan_gated(ctx, level, y, ct_gate, c.k, *map(list, zip(*fwd)))
    level, h_scale = c.out_level, c.out_scale
    k_step, step_scale = step_constant(p.moduli, level, GATE_SCALE, h_scale, SCALE)
    after = hx.he_scan_step(ctx, level, ct_gate, h, fwd[0][1], rot_key=fwd[0][0], x=ct_token, k=k_step)

    # 3. backward: the recurrence, then the norm, whose gradients of gain and bias are summed over all tokens
    ct_up = client.encrypt(up, level, SCALE, 600)
    c = scan_constants(p.moduli, level, SCALE, GATE_SCALE, steps)
    states = h[..., :level + 1 - steps, :]
    dy, dgate = hx.he_scan_gated_backward(ctx, level, ct_up, ct_gate, states, c.k, *map(list, zip(*bwd)), *fwd[0])
    b = c.out_level
    g = layer_norm_grad_constants(p.moduli, b, CHANNELS, c.out_scale, k.norm_scale, k.inv_scale, SCALE)
    dx, dgain, dbias = hx.he_layer_norm_backward(ctx, b, dy, norm, inv, g.k_grad, g.k_norm, client.rlk, gain=ct_gain, sum_keys=sums)
    hx.binding.torch.cuda.synchronize()
    seconds = time.perf_counter() - start

    total = [v.sum(1, keepdims=True).repeat(n, 1) for v in want[3:]]
    got = {
        "states": (client.decrypt(h, level, h_scale), want[0]),
        "next token": (client.decrypt(after, level - 1, step_scale), np.repeat(gate, CHANNELS // HEADS, 0) * np.roll(want[0], 1, 1) + token),
        "d input": (client.decrypt(dx, g.dx_level, g.dx_scale), want[1]),
        "d gate": (client.decrypt(dgate, b - 1, c.out_scale * h_scale / p.moduli[b]) * mask, want[2] * mask),
        "d gain": (client.decrypt(dgain, b - 1, g.dgain_scale), total[0]),
        "d bias": (client.decrypt(dbias, b - 1, g.dbias_scale), total[1]),
    }
    # 1 / sqrt enters the states and the gains' gradient once, the inputs' three times, each with the error of the Newton iterations relative to parts that may be a few times
    # the result; the backward pass' constants are rounded to 2^-17 of theirs; 1e-6 for encryption and divisions
    weight = {"states": 4, "next token": 4, "d input": 12, "d gate": 4, "d gain": 4, "d bias": 0}
    out = {}
    for name, (have, should) in got.items():
        out[name] = (float(np.abs(have - should).max() / np.abs(should).max()), weight[name] * (k.relative_error + 2.0 ** -17) + 1e-6)
    if verbose:
        print(f"N = 2^{log_n}, {CHANNELS} channels x {n} tokens in {len(lengths)} sequences, levels {top} -> {g.dx_level}: {seconds * 1e3:.1f} ms with the client's encryption of the gradient")
        for name, (diff, bound) in out.items():
            print(f"{name:10s}  largest difference from float64 {diff:.2e} of the largest value (bound {bound:.2e})")
    return out


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--log-n", type=int, default=12)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    sys.exit(0 if all(diff <= bound for diff, bound in run(a.log_n, a.seed).values()) else 1)
