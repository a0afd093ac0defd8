"""A transformer block's operators on encrypted tokens, one after the other as a server calls them:

    norm  ->  projection by expert  ->  rotary positions (height, width)  ->  norm with an encrypted gate and the residual

Three ciphertext vectors of 8 channels hold the tokens (8 x 8 images in channel-by-channel packing, one position per slot); the first goes to expert 0, the other
two to expert 1.  The client's side (keys, encryption, decryption) is the CPU oracle's, the server's the library's three calls and ``block.py`` for
their constants.  Decrypted results are compared with the same block in float64.

    python examples/encrypted_block.py            # needs an MI355X
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2604_16834_amd as hx  # noqa: E402
from paper_2604_16834_amd.block import grid_positions, linear_scale, norm_constants, quantise_weights, rope_angles  # noqa: E402
from oracle import Oracle  # noqa: E402
from workloads import make_params  # noqa: E402

CHANNELS, ROWS, SIDE, EPS = 8, (1, 2), 8, 0.01
SCALE = 2.0 ** 49


def rms(x, axis):
    return x / np.sqrt((x * x).mean(axis, keepdims=True) + EPS)


def reference(x, w, angles, gate):
    """The block in float64: x [rows][channels][slots]."""
    y = np.stack([w[g] @ rms(x[t], 0) for t, g in enumerate(np.repeat(np.arange(len(ROWS)), ROWS))])
    half = CHANNELS // 2
    turned = (y[:, :half] + 1j * y[:, half:]) * np.exp(1j * angles)
    y = np.concatenate((turned.real, turned.imag), 1)
    return gate * rms(y, 1) + x


def run(log_n=13, seed=0, verbose=True):
    """Returns the largest difference from the float64 block, relative to its largest value, and the bound on it."""
    p = make_params(log_n, 21, 7, 3)
    ctx, client = hx.Context(p), Oracle(p)
    secret, s_ntt = client.gen_secret(seed)
    rlk = hx.ckks_key_load(ctx, hx.from_host(client.gen_relin_key(s_ntt, seed + 1)), 0)
    rng = np.random.default_rng(seed)
    rows = sum(ROWS)
    x = rng.uniform(0.3, 1.0, (rows, CHANNELS, client.n)) * rng.choice((-1.0, 1.0), (rows, CHANNELS, client.n))
    gate = rng.uniform(-1, 1, (rows, CHANNELS, client.n))
    w = np.stack([np.linalg.qr(rng.normal(size=(CHANNELS, CHANNELS)))[0] for _ in ROWS])  # (orthogonal: the second norm's interval is narrow)

    def encrypt(z, level, scale=SCALE):
        flat = [client.encrypt(v, scale, level, s_ntt, 100 + i) for i, v in enumerate(z.reshape(-1, client.n))]
        return hx.from_host(np.stack(flat)).unflatten(0, z.shape[:-1])

    level = p.num_q - 1
    ct_x = encrypt(x, level)
    start = time.perf_counter()

    # 1. norm over the channels of every token (the mean square of x is between 0.09 and 1)
    k = norm_constants(p.moduli, level, CHANNELS, SCALE, (0.09, 1.02), 3, EPS)
    h = torch.stack([hx.he_norm_gate(ctx, level, ct_x[t], k.k_eps, k.k_slope, k.k_start, k.k_newton, rlk) for t in range(rows)])
    level, scale, error = k.out_level, k.out_scale, k.relative_error

    # 2. the experts' projections; the multiplier brings the scale back up for the second norm
    qw = quantise_weights(w, p.moduli[level], 32, gain=SCALE / scale)
    h = hx.he_linear_grouped(ctx, level, ROWS, h, torch.from_numpy(qw.w).cuda(), qw.multiplier)
    scale, level = linear_scale(scale, qw, p.moduli[level]), level - 1

    # 3. rotary positions, half of the pairs on the image's height and half on its width; the tables keep the scale
    angles = rope_angles(grid_positions((SIDE, SIDE), client.n // SIDE ** 2, client.n), (CHANNELS // 4, CHANNELS // 4))
    cos, sin = (hx.from_host(np.stack([client.encode_ntt(f(a), float(p.moduli[level]), level) for a in angles])) for f in (np.cos, np.sin))
    h = hx.he_rope_axes(ctx, level, h, cos, sin)
    level -= 1

    # 4. norm of the block's output, times an encrypted gate, plus the block's input
    want = reference(x, w, angles, gate)
    span = ((1 - 2 * error) * (1 - EPS / 0.09), 1 + 2 * error + EPS)  # mean squares behind an orthogonal projection of normed tokens, plus eps
    k = norm_constants(p.moduli, level, CHANNELS, scale, span, 2, EPS, gate_scale=SCALE, residual=(1.0, SCALE))
    ct_gate = encrypt(gate, level)
    out = torch.stack([hx.he_norm_gate(ctx, level, h[t], k.k_eps, k.k_slope, k.k_start, k.k_newton, rlk, gate=ct_gate[t], residual=ct_x[t], k_residual=k.k_residual)
                       for t in range(rows)])
    torch.cuda.synchronize()
    seconds = time.perf_counter() - start
    got = np.stack([[client.decrypt(ct, k.out_level, s_ntt, k.out_scale) for ct in row] for row in hx.to_host(out)])
    top = np.abs(want).max()
    diff, bound = float(np.abs(got - want).max() / top), 2 * error + k.relative_error + 1e-6
    if verbose:
        print(f"N = 2^{log_n}, {rows} vectors of {CHANNELS} channels x {client.n} tokens, levels {p.num_q - 1} -> {k.out_level}: {seconds * 1e3:.1f} ms with the client's encoding")
        print(f"largest difference from float64 {diff:.2e} of the largest value (bound from the Newton iterations {bound:.2e})")
    return diff, bound


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--log-n", type=int, default=13)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    diff, bound = run(a.log_n, a.seed)
    sys.exit(0 if diff <= bound else 1)
