"""A recurrent block's operators on the GPU, through the C boundary, against the CPU oracle on the same seeded inputs: every residue equal (results are integers: there is
no tolerance)."""
import ctypes as C
import gc

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2604_16834_amd as hx  # noqa: E402
from oracle import Oracle  # noqa: E402
from workloads import make_params  # noqa: E402
from workloads.params import CkksParams, make_params, ntt_primes, primitive_2n_root  # noqa: E402
from gpu_common import rand_ct  # noqa: E402

B = hx.binding
_worlds = {}
# log N, ciphertext primes, special primes, digits, bits: both sides of every rule on rings, digits and moduli
RINGS = [(12, 7, 3, 3, 50), (13, 7, 4, 2, 50), (12, 7, 1, 7, 50), (10, 7, 3, 3, 50), (4, 7, 3, 3, 20), (12, 7, 3, 3, 56), (11, 7, 3, 3, 56), (14, 7, 7, 1, 50)]


def world(log_n, num_q, num_p, dnum, bits=50):
    """bits: of all moduli, or a tuple with the length of each."""
    key = (log_n, num_q, num_p, dnum, bits)
    if key not in _worlds:
        if isinstance(bits, tuple):
            pools = {b: ntt_primes(log_n, len(bits), bits=b) for b in set(bits)}
            moduli = tuple(pools[b].pop() for b in bits)
            p = CkksParams(log_n, num_q, num_p, dnum, moduli, tuple(primitive_2n_root(q, log_n) for q in moduli))
        else:
            p = make_params(log_n, num_q, num_p, dnum, bits=bits)
        _worlds[key] = (p, Oracle(p), hx.Context(p))
    return _worlds[key]


@pytest.fixture(scope="module", autouse=True)
def leave_nothing():
    """Contexts, and tensors that refusals' tracebacks hold on to, go when this file is done: others watch the allocator."""
    yield
    _worlds.clear()
    gc.collect()


def ciphertexts(rng, p, level, n):
    """[n][2][level+1][N] uniform residues, some points of every limb at 0, 1, q/2 and q - 1."""
    out = np.stack([rand_ct(rng, p.moduli, level, p.n) for _ in range(n)])
    for i in range(level + 1):
        q = p.moduli[i]
        out[:, :, i, :4] = (0, 1, q // 2, q - 1)
        out[n // 2, :, i, 4:12] = q - 1
    return out


def spread(ct, extra_limbs=2, gap=1):
    """The same ciphertexts as a strided view: extra limbs behind each component, `gap` ciphertexts between neighbours."""
    n, _, limbs, N = ct.shape
    wide = torch.full((n, 1 + gap, 2, limbs + extra_limbs, N), -1, dtype=torch.int64, device="cuda")
    wide[:, 0, :, :limbs] = hx.from_host(ct)
    return wide[:, 0]


def place(ct, strided):
    return spread(ct) if strided else hx.from_host(ct)


def random_key(rng, p):
    return np.stack([rand_ct(rng, p.moduli, p.num_q + p.num_p - 1, p.n) for _ in range(p.dnum)])


class Turns:
    """Keys of rotations, made once per offset: uniform residues."""

    def __init__(self, ring, rng):
        self.p, self.orc, self.ctx = world(*ring)
        self.rng, self.known = rng, {}

    def __call__(self, off):
        if off not in self.known:
            g = self.orc.galois(off)
            host = random_key(self.rng, self.p), random_key(self.rng, self.p)
            self.known[off] = host, (hx.ckks_key_load(self.ctx, hx.from_host(host[0]), g), hx.ckks_key_load(self.ctx, hx.from_host(host[1]), hx.CKKS_KEY_CROSS | g))
        return self.known[off]

    def lists(self, offs):
        pairs = [self(o) for o in offs]
        return [h[0] for h, _ in pairs], [h[1] for h, _ in pairs], [d[0] for _, d in pairs], [d[1] for _, d in pairs]


def equal(got, want):
    assert np.array_equal(hx.to_host(got), np.array(want).reshape(tuple(got.shape)))


# ------------------------------------------------------------------------------------------ recurrence
def scan_case(ring, level, channels, heads, steps, reverse, seed, strided=False, backward=True):
    rng = np.random.default_rng(seed)
    turns = Turns(ring, rng)
    p, orc, ctx = turns.p, turns.orc, turns.ctx
    x, gate = ciphertexts(rng, p, level, channels), ciphertexts(rng, p, level, heads)
    k = [int(rng.integers(1, 1 << 62)) * (-1 if s == 1 else 1) for s in range(steps)]
    sign = 1 if reverse else -1
    hr, hc, dr, dc = turns.lists([sign << s for s in range(steps)])
    got = hx.he_scan_gated(ctx, level, place(x, strided), place(gate, strided), k, dr, dc, reverse)
    assert tuple(got.shape) == (channels, 2, level + 1 - steps, orc.N)
    equal(got, orc.scan_gated(x, gate, level, k, hr, hc, sign))
    if not backward:
        return
    hr, hc, dr, dc = turns.lists([-sign << s for s in range(steps)])
    want_gate = level > steps
    (hb, db) = turns(sign)
    states = ciphertexts(rng, p, level - steps, channels)
    dx, dgate = hx.he_scan_gated_backward(ctx, level, place(x, strided), hx.from_host(gate) if strided else place(gate, True), place(states, strided) if want_gate else None, k, dr, dc,
                                          *(db if want_gate else (None, None)), reverse=reverse, want_gate=want_gate)
    want_x, want_g = orc.scan_gated_backward(x, gate, states if want_gate else None, level, k, hr, hc, *hb, sign=-sign)
    equal(dx, want_x)
    if want_gate:
        equal(dgate, want_g)
    else:
        assert dgate is None


@pytest.mark.parametrize("ring", RINGS)
def test_scan_and_gradients_match_the_oracle(ring):
    scan_case(ring, ring[1] - 1, 4, 2, 3, False, 1)
    scan_case(ring, 2, 3, 1, 2, True, 2, strided=True)   # down to level 0: no gradient of the gates there


@pytest.mark.parametrize("channels,heads,steps", [(1, 1, 1), (5, 5, 2), (9, 1, 1), (7, 7, 1), (17, 1, 2), (8, 8, 2), (12, 4, 1), (20, 10, 1)])
def test_scan_in_batches(channels, heads, steps):
    """Batches that gates and channels share, that hold one of them only, and that are not full."""
    scan_case((12, 4, 2, 2, 50), 3, channels, heads, steps, False, channels, strided=channels % 2 == 0)
    scan_case((10, 4, 2, 2, 56), 3, channels, heads, steps, True, channels + 1, strided=channels % 2 == 1)


@pytest.mark.parametrize("level,steps", [(1, 1), (6, 5), (6, 6)])
def test_scan_uses_up_its_levels(level, steps):
    scan_case((12, 7, 3, 3, 50), level, 2, 1, steps, False, level + steps)


def test_scan_of_the_whole_ring():
    """log2(N/2) steps: every slot sees all others."""
    scan_case((4, 7, 3, 3, 20), 5, 2, 2, 3, False, 4)
    scan_case((5, 7, 3, 3, 20), 6, 2, 1, 4, True, 5)


def test_scan_of_a_large_ring():
    scan_case((16, 7, 3, 3, 50), 6, 2, 1, 1, False, 6)


def test_scan_with_one_gate_for_all_by_a_zero_stride():
    """A gate given once and expanded to every head, and one input in the place of all channels."""
    ring, level = (12, 4, 2, 2, 50), 3
    rng = np.random.default_rng(11)
    turns = Turns(ring, rng)
    x, gate = ciphertexts(rng, turns.p, level, 1), ciphertexts(rng, turns.p, level, 1)
    hr, hc, dr, dc = turns.lists([-1])
    got = hx.he_scan_gated(turns.ctx, level, hx.from_host(x).expand(6, -1, -1, -1), hx.from_host(gate).expand(3, -1, -1, -1), [1 << 50], dr, dc)
    want = turns.orc.scan_gated(x, gate, level, [1 << 50], hr, hc)[0]
    equal(got, [want] * 6)


@pytest.mark.parametrize("ring", RINGS)
@pytest.mark.parametrize("shift", [0, -1, 3])
def test_step_matches_the_oracle(ring, shift):
    rng = np.random.default_rng(shift + 9)
    turns = Turns(ring, rng)
    p, orc, ctx = turns.p, turns.orc, turns.ctx
    for level, channels, heads, k, strided in ((ring[1] - 1, 6, 3, 12345678901234567, False), (1, 2, 2, -(1 << 62), True), (2, 3, 1, None, True)):
        gate, state, x = (ciphertexts(rng, p, level, n) for n in (heads, channels, channels))
        if shift:
            host, dev = turns(shift)
            want = [orc.turned_product(gate[c // (channels // heads)], state[c], level, shift, *host, k or 0, x[c] if k else None) for c in range(channels)]
            keys = dict(cross_key=dev[1], rot_key=dev[0])
        else:
            rlk = random_key(rng, p)
            add = [orc.scalar_mul(x[c], orc.scalar_residues(k, level), level) if k else None for c in range(channels)]
            want = [orc.ctct_mul_relin_rescale(gate[c // (channels // heads)], state[c], rlk, level, addend=add[c]) for c in range(channels)]
            keys = dict(cross_key=hx.ckks_key_load(ctx, hx.from_host(rlk), 0))
        got = hx.he_scan_step(ctx, level, place(gate, strided), place(state, strided), x=place(x, not strided) if k else None, k=k or 0, **keys)
        equal(got, want)


# ------------------------------------------------------------------------------------------ layer norm
def norm_case(ring, level, channels, its, gain, bias, seed, strided=False):
    rng = np.random.default_rng(seed)
    p, orc, ctx = world(*ring)
    m = level - 2 - 2 * its
    x = ciphertexts(rng, p, level, channels)
    g = ciphertexts(rng, p, m - 1, channels) if gain else None
    b = ciphertexts(rng, p, m - 1, channels) if bias else None
    key = random_key(rng, p)
    k = [int(rng.integers(-(1 << 62), 1 << 62)) for _ in range(4)]
    newton = [int(rng.integers(-(1 << 62), 1 << 62)) for _ in range(its)]
    rlk = hx.ckks_key_load(ctx, hx.from_host(key), 0)
    norm, inv, out = hx.he_layer_norm(ctx, level, place(x, strided), k[0], k[1], k[2], newton, rlk, gain=place(g, strided) if gain else None,
                                      bias=place(b, not strided) if bias else None, k_bias=k[3])
    want_norm, want_inv, want_out = orc.layer_norm(x, level, k[0], k[1], k[2], newton, key, g, b, k[3])
    equal(norm, want_norm)
    equal(inv, want_inv)
    if gain:
        equal(out, want_out)
    else:
        assert out is None


@pytest.mark.parametrize("ring", RINGS)
def test_layer_norm_matches_the_oracle(ring):
    norm_case(ring, ring[1] - 1, 3, 1, True, True, 1)
    norm_case(ring, 3, 5, 0, False, False, 2, strided=True)
    norm_case(ring, 4, 2, 0, True, False, 3, strided=True)


@pytest.mark.parametrize("channels", [1, 2, 8, 9, 16, 17, 33, 130])
def test_layer_norm_in_batches(channels):
    norm_case((12, 7, 3, 3, 50), 6, channels, 1, True, channels % 2 == 0, channels)
    norm_case((10, 5, 2, 3, 56), 4, channels, 0, channels % 2 == 0, False, channels + 1, strided=True)


def test_layer_norm_of_a_large_ring():
    norm_case((16, 7, 3, 3, 50), 6, 3, 1, True, True, 5)


def grad_case(ring, level, channels, affine, stages, seed, strided=False, want_gain=True, want_bias=True):
    """stages: lists of offsets."""
    rng = np.random.default_rng(seed)
    turns = Turns(ring, rng)
    p, orc, ctx = turns.p, turns.orc, turns.ctx
    grad, norm, inv = ciphertexts(rng, p, level, channels), ciphertexts(rng, p, level, channels), ciphertexts(rng, p, level, 1)
    gain = ciphertexts(rng, p, level, channels) if affine else None
    key = random_key(rng, p)
    kg, kn = int(rng.integers(1, 1 << 62)), -int(rng.integers(1, 1 << 62))
    host = [(row, [turns(o)[0][0] for o in row]) for row in stages]
    dx, dgain, dbias = hx.he_layer_norm_backward(ctx, level, place(grad, strided), place(norm, not strided), place(inv, strided)[0], kg, kn, hx.ckks_key_load(ctx, hx.from_host(key), 0),
                                                 gain=place(gain, strided) if affine else None, sum_keys=[[turns(o)[1][0] for o in row] for row in stages],
                                                 want_gain=want_gain, want_bias=want_bias)
    want = orc.layer_norm_backward(grad, norm, inv[0], level, kg, kn, key, gain, host)
    equal(dx, want[0])
    for got, wanted, w in ((dgain, want_gain, want[1]), (dbias, want_bias, want[2])):
        if wanted:
            equal(got, w)
        else:
            assert got is None


@pytest.mark.parametrize("ring", RINGS)
def test_layer_norm_gradients_match_the_oracle(ring):
    grad_case(ring, ring[1] - 1, 3, True, [(1,), (2, 4, 6)], 1)
    grad_case(ring, 3, 2, False, [(1, 2, 3, 4, 5, 6, 7)], 2, strided=True)
    grad_case(ring, 4, 4, True, [(-1,)], 3, strided=True, want_bias=False)


@pytest.mark.parametrize("channels", [1, 7, 8, 9, 17, 33])
def test_layer_norm_gradients_in_batches(channels):
    grad_case((12, 5, 2, 3, 50), 4, channels, True, [(1, 2), (3,)], channels, strided=channels % 2 == 0)
    grad_case((10, 5, 2, 3, 56), 3, channels, False, [(1,)], channels + 1, want_gain=channels % 2 == 0)


@pytest.mark.parametrize("stages", [[], [(1,)], [(1,), (2,)], [(1,)] * 3, [(5, 5)], [tuple(range(1, 70))], [(1, 2, 3), (4, 8, 12), (16, 32)], [(1, 2), (3,), (1, 4), (5,), (-1,)], [(2,), (1, 2, 3), (7,)]])
def test_sums_over_slots(stages):
    """None, one rotation a stage an odd and an even number of times, the same again, one twice in a stage, more rotations than a launch holds, mixed."""
    grad_case((12, 4, 2, 2, 50), 3, 2, False, stages, len(stages))
    grad_case((11, 4, 2, 2, 56), 3, 2, False, stages, len(stages) + 1)


@pytest.mark.parametrize("dnum", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("channels", [1, 2, 3, 5, 9])
def test_sums_over_slots_by_digits_and_ciphertexts(dnum, channels):
    """Every number of digits that has a kernel of its own and more, with both counts of ciphertexts a thread takes."""
    ring = (12, 8, -(-8 // dnum), dnum, 50)
    grad_case(ring, 7, channels, False, [(1, 2, 3, 4, 5, 6, 7), (-1, 5)], dnum + channels)
    grad_case((11, 8, -(-8 // dnum), dnum, 50), 3, channels, False, [(3,), (1, 2, 3)], dnum + channels, want_gain=False)


def test_layer_norm_gradients_of_a_large_ring():
    grad_case((16, 6, 2, 3, 50), 5, 3, True, [(1, 2, 3)], 5)


# moduli of 43 to 50 bits (double precision) and of 53 to 55 (integers), ciphertext primes first
@pytest.mark.parametrize("log_n", [10, 12, 13])
@pytest.mark.parametrize("bits", [(50, 43, 47, 45, 50, 44, 50, 50), (55, 53, 54, 55, 53, 54, 55, 55)])
def test_moduli_of_unequal_lengths(log_n, bits):
    ring = (log_n, 6, 2, 3, bits)
    scan_case(ring, 5, 4, 2, 2, False, 1)
    norm_case(ring, 5, 3, 0, True, True, 2)
    grad_case(ring, 5, 3, True, [(1, 2, 3)], 3)


def test_extreme_residues():
    """Every residue of operands and keys at q - 1, and constants at the ends of their type."""
    ring, level = (12, 4, 2, 2, 50), 3
    p, orc, ctx = world(*ring)
    top = np.stack([np.stack([np.full(orc.N, p.moduli[i] - 1, np.uint64) for i in range(level + 1)])] * 2)
    key = np.stack([np.stack([np.stack([np.full(orc.N, q - 1, np.uint64) for q in p.moduli])] * 2)] * p.dnum)
    g = orc.galois(-1)
    rot, cross, rlk = (hx.ckks_key_load(ctx, hx.from_host(key), e) for e in (g, hx.CKKS_KEY_CROSS | g, 0))
    for k in ((1 << 63) - 1, -(1 << 63)):
        got = hx.he_scan_gated(ctx, level, hx.from_host(np.stack([top] * 4)), hx.from_host(top[None]), [k], [rot], [cross])
        equal(got, [orc.turned_product(top, top, level, -1, key, key, k, top)] * 4)
        got = hx.he_layer_norm_backward(ctx, level, hx.from_host(np.stack([top] * 3)), hx.from_host(np.stack([top] * 3)), hx.from_host(top), k, k, rlk, sum_keys=[[rot, rot]])
        want = orc.layer_norm_backward([top] * 3, [top] * 3, top, level, k, k, key, None, [((-1, -1), [key, key])])
        for a, b in zip(got, want):
            equal(a, b)


# ------------------------------------------------------------------------------------------ the calls' manner
def calls(ring=(12, 7, 3, 3, 50), seed=3):
    """Each operator as a function of (ws, outs), its workspace, its outputs' shapes: arguments that stay alive with it."""
    rng = np.random.default_rng(seed)
    turns = Turns(ring, rng)
    p, ctx, N = turns.p, turns.ctx, turns.orc.N
    level = ring[1] - 1
    ct = lambda n, limbs=level + 1: hx.from_host(ciphertexts(rng, p, limbs - 1, n))  # noqa: E731
    x, gate, states, rlk = ct(18), ct(2), ct(18, level - 1), hx.ckks_key_load(ctx, hx.from_host(random_key(rng, p)), 0)
    fwd, bwd, back = turns.lists((-1, -2))[2:], turns.lists((1, 2))[2:], turns(-1)[1]
    k, m = [1 << 50, 3 << 49], level - 4
    gain, bias, inv = ct(18), ct(18), ct(1)[0]
    sums = [[turns(o)[1][0] for o in (1, 2, 3)], [turns(4)[1][0]]]
    return ctx, {
        "scan": (lambda ws, o, st=None: hx.he_scan_gated(ctx, level, x, gate, k, *fwd, out=o[0], ws=ws, stream=st),
                 hx.he_scan_workspace_bytes(ctx, level, 18, 2, 2), [(18, 2, level - 1, N)]),
        "scan_backward": (lambda ws, o, st=None: hx.he_scan_gated_backward(ctx, level, x, gate, states, k, *bwd, *back, dx=o[0], dgate=o[1], ws=ws, stream=st),
                          hx.he_scan_backward_workspace_bytes(ctx, level, 18, 2, 2), [(18, 2, level - 1, N), (2, 2, level - 2, N)]),
        "step": (lambda ws, o, st=None: hx.he_scan_step(ctx, level, gate, x, back[1], back[0], bias, 1 << 50, out=o[0], ws=ws, stream=st),
                 hx.he_scan_step_workspace_bytes(ctx, level, 18, 2), [(18, 2, level, N)]),
        "step_in_place": (lambda ws, o, st=None: hx.he_scan_step(ctx, level, gate, x, rlk, None, bias, 1 << 50, out=o[0], ws=ws, stream=st),
                          hx.he_scan_step_workspace_bytes(ctx, level, 18, 2), [(18, 2, level, N)]),
        "norm": (lambda ws, o, st=None: hx.he_layer_norm(ctx, level, x, 1 << 40, -(3 << 47), 5 << 48, (3 << 49,), rlk, gain, bias, 1 << 49, norm=o[0], inv=o[1], out=o[2], ws=ws, stream=st),
                 hx.he_layer_norm_workspace_bytes(ctx, level, 18, 1, True), [(18, 2, m, N), (2, m + 1, N), (18, 2, m - 1, N)]),
        "norm_backward": (lambda ws, o, st=None: hx.he_layer_norm_backward(ctx, level, x, bias, inv, 1 << 20, -(1 << 20), rlk, gain, sums, dx=o[0], dgain=o[1], dbias=o[2], ws=ws, stream=st),
                          hx.he_layer_norm_backward_workspace_bytes(ctx, level, 18, True, 2), [(18, 2, level - 3, N), (18, 2, level, N), (18, 2, level, N)]),
    }


NAMES = ["scan", "scan_backward", "step", "step_in_place", "norm", "norm_backward"]


def outputs(shapes, pad=64):
    """Outputs inside larger buffers filled with -1: (buffers, views)."""
    bufs = [torch.full((int(np.prod(s)) + 2 * pad,), -1, dtype=torch.int64, device="cuda") for s in shapes]
    return bufs, [b[pad:-pad].view(s) for b, s in zip(bufs, shapes)]


def alone(bufs, ws=None, need=0, pad=64):
    for b in bufs:
        assert bool((b[:pad] == -1).all()) and bool((b[-pad:] == -1).all())
    if ws is not None:
        assert bool((ws[need:] == 0x5a).all())


@pytest.mark.parametrize("ring", [(12, 7, 3, 3, 50), (10, 7, 3, 3, 50), (12, 7, 3, 3, 56), (13, 7, 1, 7, 50), (14, 7, 3, 3, 50)])
@pytest.mark.parametrize("name", NAMES)
def test_nothing_is_written_beside_outputs_and_workspace(name, ring):
    ctx, ops = calls(ring)
    call, need, shapes = ops[name]
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    bufs, outs = outputs(shapes)
    call(ws[:need], outs)
    alone(bufs, ws, need)
    again = [o.clone() for o in outs]
    ws[:need] = 0xff  # what is in the workspace does not matter
    call(ws[:need], outs)
    assert all(torch.equal(a, b) for a, b in zip(again, outs))


@pytest.mark.parametrize("name", NAMES)
def test_a_workspace_of_a_byte_less_is_refused(name):
    ctx, ops = calls()
    call, need, shapes = ops[name]
    bufs, outs = outputs(shapes)
    with pytest.raises(hx.CkksError) as e:
        call(torch.empty(need - 1, dtype=torch.uint8, device="cuda"), outs)
    assert e.value.code == B.CKKS_ERR_WORKSPACE_TOO_SMALL
    torch.cuda.synchronize()
    assert all(bool((b == -1).all()) for b in bufs)


@pytest.mark.parametrize("name", NAMES)
def test_on_another_stream(name):
    ctx, ops = calls()
    call, need, shapes = ops[name]
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    _, ref = outputs(shapes)
    call(ws, ref)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    _, outs = outputs(shapes)
    torch.cuda.synchronize()
    call(ws, outs, side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, outs))
    with torch.cuda.stream(side):  # the current stream is taken where none is given
        _, outs = outputs(shapes)
        call(ws, outs)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, outs))


@pytest.mark.parametrize("ring", [(12, 7, 3, 3, 50), (14, 7, 3, 3, 50), (12, 7, 3, 3, 56)])
@pytest.mark.parametrize("name", NAMES)
def test_two_calls_at_once(name, ring):
    """One context, two streams, a workspace each: nothing waits on the host between the calls, and the context's second stream serves both."""
    ctx, ops = calls(ring)
    call, need, shapes = ops[name]
    first, second = ([torch.empty(need, dtype=torch.uint8, device="cuda"), torch.cuda.Stream(), outputs(shapes)[1]] for _ in range(2))
    _, ref = outputs(shapes)
    call(first[0], ref)
    torch.cuda.synchronize()
    for _ in range(3):
        for ws, stream, outs in (first, second):
            call(ws, outs, stream.cuda_stream)
    torch.cuda.synchronize()
    for _, _, outs in (first, second):
        assert all(torch.equal(a, b) for a, b in zip(ref, outs))


@pytest.mark.parametrize("bits", [50, 56])
def test_operands_far_apart(bits):
    """Ciphertexts 2^30 words (8 GiB) and their components more than 2^29 words from each other: offsets pass 32 bits in bytes and, at the fifth, in words."""
    ring, level, channels, far, comp = (12, 6, 2, 3, bits), 5, 5, 1 << 30, (1 << 29) + 4096
    rng = np.random.default_rng(5)
    turns = Turns(ring, rng)
    p, ctx, N = turns.p, turns.ctx, turns.orc.N
    pool = torch.empty((channels - 1) * far + comp + (level + 1) * N, dtype=torch.int64, device="cuda")
    apart = pool.as_strided((channels, 2, level + 1, N), (far, comp, N, 1))
    near, gate, rlk = hx.from_host(ciphertexts(rng, p, level, channels)), hx.from_host(ciphertexts(rng, p, level, 1)), hx.ckks_key_load(ctx, hx.from_host(random_key(rng, p)), 0)
    apart.copy_(near)
    fwd, bwd, back = turns.lists((-1, -2))[2:], turns.lists((1, 2))[2:], turns(-1)[1]
    k = [1 << 50, 3 << 49]
    for f in (lambda x: [hx.he_scan_gated(ctx, level, x, gate, k, *fwd)],
              lambda x: hx.he_scan_gated_backward(ctx, level, x, gate, x, k, *bwd, *back),
              lambda x: [hx.he_scan_step(ctx, level, x, x, back[1], back[0], x, 1 << 50)],
              lambda x: [hx.he_scan_step(ctx, level, x, x, rlk, None, x, 1 << 50)],
              lambda x: hx.he_layer_norm(ctx, level, x, 1 << 40, -(3 << 47), 5 << 48, (), rlk, x, x, 1 << 49),
              lambda x: hx.he_layer_norm_backward(ctx, level, x, x, gate[0], 1 << 20, -(1 << 20), rlk, x, [[back[0], fwd[0][1]]])):
        assert all(torch.equal(a, b) for a, b in zip(f(near), f(apart)))


@pytest.mark.parametrize("ring", [(13, 7, 3, 3, 50), (14, 7, 3, 3, 50), (12, 7, 3, 3, 56)])
@pytest.mark.parametrize("name", NAMES)
def test_one_stream_and_two_agree(name, ring):
    """The same workspace serves both; sizes on both sides of the rule that deals batches to the context's second stream."""
    ctx, ops = calls(ring)
    call, need, shapes = ops[name]
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    (b1, one), (b2, two) = outputs(shapes), outputs(shapes)
    call(ws[:need], two)
    try:
        hx.ckks_ctx_set_overlap(ctx, False)
        call(ws[:need], one)
    finally:
        hx.ckks_ctx_set_overlap(ctx, True)
    alone(b1 + b2, ws, need)
    assert all(torch.equal(a, b) for a, b in zip(one, two))


@pytest.mark.parametrize("ring", [(12, 7, 3, 3, 50), (14, 7, 3, 3, 50)])
@pytest.mark.parametrize("name", NAMES)
def test_captured_and_replayed(name, ring):
    """Two graphs that share a workspace, replayed in turn with eager calls between, every replay against the eager result."""
    ctx, ops = calls(ring)
    call, need, shapes = ops[name]
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    _, ref = outputs(shapes)
    call(ws, ref)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        _, outs = outputs(shapes)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            call(ws, outs)
        graphs.append((g, outs))
    for turn in range(3):
        for g, outs in graphs:
            for o in outs:
                o.fill_(-1)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(ref, outs)), turn
        _, eager = outputs(shapes)
        call(ws, eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, eager)), turn


def test_refusals_of_the_library():
    """Through the binding, which leaves levels, keys and counts to the library; nothing is launched."""
    ring, level = (12, 4, 2, 2, 50), 3
    rng = np.random.default_rng(5)
    turns = Turns(ring, rng)
    p, ctx, N = turns.p, turns.ctx, turns.orc.N
    key = hx.from_host(random_key(rng, p))
    ct = lambda n, limbs=4: hx.from_host(ciphertexts(rng, p, limbs - 1, n))  # noqa: E731
    x, gate, k = ct(4), ct(2), [1 << 50]
    rot, cross, rlk = turns(-1)[1][0], turns(-1)[1][1], hx.ckks_key_load(ctx, key, 0)
    fwd = turns(1)[1]

    def code(fn, *a, **kw):
        with pytest.raises(hx.CkksError) as e:
            fn(*a, **kw)
        return e.value.code

    for bad in (hx.CKKS_KEY_CROSS, hx.CKKS_KEY_CROSS | 2, hx.CKKS_KEY_CROSS | (2 * N + 1), 2 * N + 1):
        assert code(hx.ckks_key_load, ctx, key, bad) == B.CKKS_ERR_INVALID_ARG
    scan, step, back, norm, grad = hx.he_scan_gated, hx.he_scan_step, hx.he_scan_gated_backward, hx.he_layer_norm, hx.he_layer_norm_backward
    ok = (ctx, level, x, gate, k, [rot], [cross])
    scan(*ok)
    assert code(scan, ctx, level, x, gate, k, [cross], [rot]) == B.CKKS_ERR_NO_KEY
    assert code(scan, ctx, level, x, gate, k, [rot], [rlk]) == B.CKKS_ERR_NO_KEY
    assert code(scan, ctx, level, x, gate, k, [fwd[0]], [fwd[1]]) == B.CKKS_ERR_NO_KEY
    assert code(scan, *ok, reverse=True) == B.CKKS_ERR_NO_KEY
    assert code(scan, ctx, level, x[:3], gate, k, [rot], [cross]) == B.CKKS_ERR_INVALID_ARG       # channels not a multiple of the heads
    assert code(scan, ctx, level, x[:0], gate, k, [rot], [cross]) == B.CKKS_ERR_INVALID_ARG
    assert code(scan, ctx, level, x, gate, [], [], []) == B.CKKS_ERR_INVALID_ARG
    assert code(scan, ctx, 1, x, gate, k * 2, [rot] * 2, [cross] * 2) == B.CKKS_ERR_LEVEL_MISMATCH
    assert code(scan, ctx, 0, x, gate, k, [rot], [cross]) == B.CKKS_ERR_LEVEL_MISMATCH
    small = Turns((4, 7, 3, 3, 20), rng)
    sx = hx.from_host(ciphertexts(rng, small.p, 6, 1))
    pair = small(-1)[1]
    assert code(scan, small.ctx, 6, sx, sx, [1] * 4, [pair[0]] * 4, [pair[1]] * 4) == B.CKKS_ERR_INVALID_ARG  # 16 positions on 8 slots
    assert code(back, ctx, 1, x, gate, x, k, [fwd[0]], [fwd[1]], rot, cross) == B.CKKS_ERR_LEVEL_MISMATCH
    assert code(back, ctx, level, x, gate, x, k, [fwd[0]], [fwd[1]], fwd[0], fwd[1]) == B.CKKS_ERR_NO_KEY
    assert code(back, ctx, level, x, gate, x, k, [rot], [cross], rot, cross) == B.CKKS_ERR_NO_KEY
    assert code(step, ctx, level, gate, x, cross) == B.CKKS_ERR_NO_KEY
    assert code(step, ctx, level, gate, x, rlk, rot) == B.CKKS_ERR_NO_KEY
    assert code(step, ctx, level, gate, x, fwd[1], rot) == B.CKKS_ERR_NO_KEY
    assert code(step, ctx, level, gate, x, hx.ckks_key_load(ctx, key, hx.CKKS_KEY_CROSS | 1), hx.ckks_key_load(ctx, key, 1)) == B.CKKS_ERR_NO_KEY
    assert code(step, ctx, 0, gate, x, rlk) == B.CKKS_ERR_LEVEL_MISMATCH
    assert code(norm, ctx, level, x, 1, 1, 1, (), rot) == B.CKKS_ERR_NO_KEY
    assert code(norm, ctx, 2, x, 1, 1, 1, (), rlk) == B.CKKS_ERR_LEVEL_MISMATCH
    assert code(norm, ctx, level, x, 1, 1, 1, (1,), rlk) == B.CKKS_ERR_LEVEL_MISMATCH
    assert code(norm, ctx, level, x, 1, 1, 1, (), rlk, gain=x) == B.CKKS_ERR_LEVEL_MISMATCH
    inv = x[0]
    assert code(grad, ctx, 2, x, x, inv, 1, 1, rlk) == B.CKKS_ERR_LEVEL_MISMATCH
    assert code(grad, ctx, level, x, x, inv, 1, 1, rlk, gain=x) == B.CKKS_ERR_LEVEL_MISMATCH
    assert code(grad, ctx, level, x, x, inv, 1, 1, cross) == B.CKKS_ERR_NO_KEY
    assert code(grad, ctx, level, x, x, inv, 1, 1, rlk, sum_keys=[[rot], []]) == B.CKKS_ERR_INVALID_ARG
    assert code(grad, ctx, level, x, x, inv, 1, 1, rlk, sum_keys=[[rot, cross]]) == B.CKKS_ERR_NO_KEY
    assert code(grad, ctx, level, x, x, inv, 1, 1, rlk, sum_keys=[[rlk]]) == B.CKKS_ERR_NO_KEY
    assert code(grad, ctx, level, x, x, inv, 1, 1, rlk, sum_keys=[[rot]] * 65) == B.CKKS_ERR_INVALID_ARG
    # cross keys serve nothing else
    assert code(hx.ckks_rotate_hoisted, ctx, x[0], level, [-1], [cross]) == B.CKKS_ERR_NO_KEY
    assert code(hx.ckks_ctct_mul_relin, ctx, x[0], x[1], level, cross) == B.CKKS_ERR_NO_KEY
    for query in (hx.he_scan_workspace_bytes(ctx, level, 3, 2, 1), hx.he_scan_workspace_bytes(ctx, level, 2, 2, 4), hx.he_scan_step_workspace_bytes(ctx, 0, 1, 1),
                  hx.he_scan_backward_workspace_bytes(ctx, level, 1, 0, 1), hx.he_layer_norm_workspace_bytes(ctx, level, 1, 1), hx.he_layer_norm_backward_workspace_bytes(ctx, 2, 1)):
        assert query == 0


def test_a_stride_whose_offsets_wrap_is_refused():
    """2^44 words between 65536 ciphertexts: through the C boundary, as no tensor is that large.  No workspace is given either: nothing can be launched."""
    turns = Turns((12, 4, 2, 2, 50), np.random.default_rng(6))
    ctx, N = turns.ctx, turns.orc.N
    x = hx.empty(2, 4, N)
    rot, cross = turns(-1)[1]
    d, arr = B._ScanDesc(65536, 1, 3, 1, 0), B._CtArray(x.data_ptr(), 1 << 44, 4 * N)
    one = B._CtArray(x.data_ptr(), 0, 4 * N)
    rc = B._lib.he_scan_gated(ctx.handle, C.byref(d), (C.c_int64 * 1)(1), C.byref(arr), C.byref(one), B._key_handles([rot]), B._key_handles([cross]), x.data_ptr(), None, 0, None)
    assert rc == B.CKKS_ERR_INVALID_ARG and b"stride" in B._lib.ckks_last_error_string(ctx.handle)


def test_contexts_without_key_switching_refuse():
    p = make_params(12, 4, 0, 0)
    ctx = hx.Context(p)
    for need in (hx.he_scan_workspace_bytes(ctx, 3, 1, 1, 1), hx.he_layer_norm_workspace_bytes(ctx, 3, 1, 0), hx.he_layer_norm_backward_workspace_bytes(ctx, 3, 1)):
        assert need == 0


# ------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("log_n", [12, 13])
def test_the_example_agrees_with_float64(log_n):
    """examples/encrypted_recurrence.py: norm, recurrence, step and both backward passes one after the other, decrypted, within what the Newton iterations and the constants' rounding
    leave.  (That the float64 gradients are the differences of its loss is tested without a GPU.)"""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "encrypted_recurrence.py")
    spec = importlib.util.spec_from_file_location("encrypted_recurrence", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    for name, (diff, bound) in module.run(log_n, seed=log_n, verbose=False).items():
        assert diff <= bound, name
