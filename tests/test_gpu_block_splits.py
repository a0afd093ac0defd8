"""A transformer block's operators where a call goes in parts (outputs, groups and gated channels beyond what a part of the workspace holds), where sums are as long
as they get, and on contexts of other kinds (moduli of unequal lengths, no key switching), against the CPU oracle on the same seeded inputs: every residue equal."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2604_16834_amd as hx  # noqa: E402
from oracle import Oracle  # noqa: E402
from workloads.params import CkksParams, make_params, ntt_primes, primitive_2n_root  # noqa: E402
from gpu_common import rand_ct, rand_poly  # noqa: E402

B = hx.binding
_worlds = {}


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


def ciphertexts(rng, p, level, n):
    """[n][2][level+1][N] uniform residues, the first points of every limb at 0, 1, q/2 and q - 1."""
    out = np.stack([rand_ct(rng, p.moduli, level, p.n) for _ in range(n)])
    for i in range(level + 1):
        out[:, :, i, :4] = (0, 1, p.moduli[i] // 2, p.moduli[i] - 1)
    return out


def device_residues(seed, p, limbs, *lead):
    """[*lead][limbs][N] uniform residues made on the GPU."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.tensor(p.moduli[:limbs], dtype=torch.int64, device="cuda").unsqueeze(-1)
    return torch.randint(0, 1 << 62, (*lead, limbs, p.n), generator=gen, device="cuda").remainder_(q)


# ------------------------------------------------------------------------------------------ grouped products
# rings where the sums' part of the workspace (1 GiB) holds fewer outputs than a row has: 512 of one limb at N = 2^17; 102 of ten limbs at N = 2^16 where all limbs'
# sums are stored (no key switching; moduli of 56 bits), which is no multiple of a tile; 9 channels go to the matrix cores where the moduli allow, one to the vector units
@pytest.mark.parametrize("ring,level,c_in,c_out,seams", [
    ((17, 2, 1, 1, 50), 1, 9, 600, (0, 383, 384, 599)), ((17, 2, 1, 1, 50), 1, 1, 530, (0, 383, 384, 529)),
    ((16, 10, 0, 0, 50), 9, 9, 120, (0, 101, 102, 119)), ((16, 10, 5, 2, 56), 9, 3, 120, (0, 101, 102, 119))])
def test_grouped_product_with_rows_in_parts(ring, level, c_in, c_out, seams):
    p, orc, ctx = world(*ring)
    rng = np.random.default_rng(c_out)
    rows = (1, 0, 1)
    stored = 1 if ring[2] and ring[4] <= 50 else level + 1  # limbs of an output's sums in the workspace
    assert hx.he_linear_workspace_bytes(ctx, level, rows, c_in, c_out, torch.int16) < 16 * c_out * stored * orc.N  # a row does go in parts
    x = ciphertexts(rng, p, level, 2 * c_in)
    w = rng.integers(-32768, 32768, size=(3, c_out, c_in)).astype(np.int16)
    b = np.stack([rng.integers(0, q, size=(3, c_out), dtype=np.uint64) for q in p.moduli[:level + 1]], -1)
    got = hx.he_linear_grouped(ctx, level, rows, hx.from_host(x).unflatten(0, (2, c_in)), torch.from_numpy(w).cuda(), 3 << 30, hx.from_host(b))
    for t, g in ((0, 0), (1, 2)):
        for o in seams:
            want = orc.linear_grouped([x[t * c_in:(t + 1) * c_in]], level, (1,), w[g:g + 1, o:o + 1], 3 << 30, b[g:g + 1, o:o + 1])
            assert np.array_equal(hx.to_host(got[t, o]), want[0][0]), (t, o)
    # every output of a part against the same outputs computed alone
    for lo, hi in ((0, seams[1] + 1), (seams[2], c_out)):
        lo = max(lo, hi - 100)
        alone = hx.he_linear_grouped(ctx, level, rows, hx.from_host(x).unflatten(0, (2, c_in)), torch.from_numpy(w[:, lo:hi].copy()).cuda(), 3 << 30,
                                     hx.from_host(b[:, lo:hi]))
        assert torch.equal(alone, got[:, lo:hi])


def test_grouped_product_of_more_groups_than_the_digits_part_holds():
    """60 groups whose weights' digits take 8 MB each, of which 256 MB go together, and as many channels as a call may have.  One ciphertext stands in the place of all
    channels, so that the oracle's sum is that of the weights."""
    p, orc, ctx = world(12, 2, 1, 1)
    rng = np.random.default_rng(60)
    groups, c_in, c_out = 60, 65536, 17
    assert hx.he_linear_workspace_bytes(ctx, 1, (1,) * groups, c_in, c_out, torch.int32) < groups * 32 * c_in * 4  # the digits of all groups
    x = ciphertexts(rng, p, 1, 1)
    gen = torch.Generator(device="cuda").manual_seed(60)
    w = torch.randint(-(1 << 31), 1 << 31, (groups, c_out, c_in), generator=gen, device="cuda").to(torch.int32)
    got = hx.to_host(hx.he_linear_grouped(ctx, 1, (1,) * groups, hx.from_host(x[0]).expand(groups, c_in, 2, 2, orc.N), w, 12345))
    sums = w.sum(-1, dtype=torch.int64, keepdim=True).cpu().numpy()
    assert len(np.unique(sums)) > groups * c_out - 5
    want = orc.linear_grouped(np.broadcast_to(x, (groups, 1, 2, 2, orc.N)), 1, (1,) * groups, sums, 12345)
    for g in range(groups):
        assert np.array_equal(got[g], np.array(want[g])), g


def recoded(v):
    """The seven signed base-256 digits that the matrix-core kernel makes of a residue."""
    bias = 0x0080808080808080
    s = (v + bias) ^ bias
    return [((s >> 8 * i & 0xff) ^ 0x80) - 0x80 for i in range(7)]


@pytest.mark.parametrize("dtype", [np.int8, np.int16, np.int32])
@pytest.mark.parametrize("c_in", [64, 128, 256, 512])
def test_grouped_product_of_the_largest_diagonals(dtype, c_in):
    """Residues whose digits are -128 (or 127) six times in every channel, against weights whose digits are -128 (or 127) throughout, for as many channels as a launch
    takes: each diagonal at its bound."""
    assert recoded(0x7f7f7f7f7f80) == [-128] * 6 + [1] and recoded(0x7f7f7f7f7f7f) == [127] * 6 + [0]
    p, orc, ctx = world(12, 2, 1, 1)
    info = np.iinfo(dtype)
    c_out = 18
    x = ciphertexts(np.random.default_rng(c_in), p, 1, c_in)
    x[:, :, :, 100:200] = 0x7f7f7f7f7f80
    x[:, :, :, 200:300] = 0x7f7f7f7f7f7f
    x[:, 0, :, 300:400] = 0x7f7f7f7f7f80
    x[::2, :, :, 400:500] = 0x7f7f7f7f7f80
    x[:, :, 0, 500:600], x[:, :, 1, 500:600] = p.moduli[0] - 1, p.moduli[1] - 1
    w = np.empty((1, c_out, c_in), dtype=dtype)
    w[0, 0::2], w[0, 1::2] = info.min, info.max  # every digit of info.min is -128 and of info.max 127, once 128 is taken off the lower bytes
    w[0, 4, ::2] = 0
    got = hx.to_host(hx.he_linear_grouped(ctx, 1, (1,), hx.from_host(x)[None], torch.from_numpy(w).cuda(), (1 << 50) + 1))
    kinds = orc.linear_grouped([x], 1, (1,), w[:, (0, 1, 4)], (1 << 50) + 1)[0]
    for o in range(c_out):
        assert np.array_equal(got[0, o], kinds[2 if o == 4 else o % 2]), o


@pytest.mark.parametrize("bits", [50, 56])
def test_grouped_product_of_the_longest_sums(bits):
    """65536 channels at q - 1 times weights at the type's ends: the longest sums, in both arithmetics."""
    p, orc, ctx = world(12, 2, 1, 1, bits)
    x = np.empty((1, 2, 2, orc.N), dtype=np.uint64)
    for i in range(2):
        x[:, :, i] = p.moduli[i] - 1
    w = np.empty((1, 3, 65536), dtype=np.int32)
    w[0, 0], w[0, 1], w[0, 2] = -(1 << 31), (1 << 31) - 1, -1
    got = hx.to_host(hx.he_linear_grouped(ctx, 1, (1,), hx.from_host(x[0]).expand(1, 65536, 2, 2, orc.N), torch.from_numpy(w).cuda(), (1 << 64) - 1))
    want = orc.linear_grouped(x[None], 1, (1,), w.sum(-1, dtype=np.int64, keepdims=True), (1 << 64) - 1)
    assert np.array_equal(got, np.array(want))


def test_a_stride_whose_offsets_wrap_is_refused():
    """2^40 words between 2^32 ciphertexts: through the C boundary, as no tensor is that large.  No workspace is given either: nothing can be launched."""
    p, orc, ctx = world(12, 2, 1, 1)
    x = hx.empty(2, 2, orc.N)
    d = B._LinearDesc(65536, 1, 1, 1, B.HE_WEIGHT_INT8, 0, 1)
    arr = B._CtArray(x.data_ptr(), 1 << 40, 2 * orc.N)
    rc = B._lib.he_linear_grouped(ctx.handle, C.byref(d), (C.c_uint32 * 1)(65536), C.byref(arr), x.data_ptr(), None, x.data_ptr(), None, 0, None)
    assert rc == B.CKKS_ERR_INVALID_ARG and b"stride" in B._lib.ckks_last_error_string(ctx.handle)


# ------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("gate", ["cipher", "plain"])
def test_norm_with_gated_channels_in_two_parts(gate):
    """150 channels of which 16 limbs are kept behind the gate, at N = 2^17: 4 GB hold 128.  Single channels on both sides of the seam against the oracle; all of
    them against one stream, and against the channels in reverse order, where others go together (the sum of squares is the same)."""
    p, orc, ctx = world(17, 18, 9, 2)
    level, channels, last = 17, 150, 15
    need = [hx.he_norm_workspace_bytes(ctx, level, n, 0, B.HE_GATE_CIPHER if gate == "cipher" else B.HE_GATE_PLAIN) for n in (105, 120, 135, 150)]
    assert need[0] < need[1] == need[2] == need[3]  # (batches of 15 in all four)
    x, res = device_residues(1, p, level + 1, channels, 2), device_residues(2, p, last + 1, channels, 2)
    g = device_residues(3, p, level + 1, channels, 2) if gate == "cipher" else device_residues(3, p, level + 1, channels)
    rng = np.random.default_rng(4)
    key = np.stack([rand_ct(rng, p.moduli, p.num_q + p.num_p - 1, orc.N) for _ in range(p.dnum)])
    rlk, k = hx.ckks_key_load(ctx, hx.from_host(key), 0), (1 << 40, -(3 << 47), 5 << 48, 1 << 49)

    def call(order=slice(None)):
        a, b, c = (x, g, res) if order == slice(None) else (x.flip(0), g.flip(0), res.flip(0))
        return hx.he_norm_gate(ctx, level, a, k[0], k[1], k[2], (), rlk, b, c, k[3])
    two = call()
    try:
        hx.ckks_ctx_set_overlap(ctx, False)
        assert torch.equal(call(), two)
    finally:
        hx.ckks_ctx_set_overlap(ctx, True)
    assert torch.equal(call("reversed").flip(0), two)
    print("norm: parts, streams and orders agree", flush=True)
    only = (0, 119, 120, 149)
    pick = lambda t: {c: hx.to_host(t[c]) for c in only}  # noqa: E731
    want = orc.norm_gate(list(hx.to_host(x)), level, k[0], k[1], k[2], (), key, pick(g), pick(res), k[3], only=only)
    for c, ct in zip(only, want):
        assert np.array_equal(hx.to_host(two[c]), ct), c


# ------------------------------------------------------------------------------------------ contexts of other kinds
# moduli of 43 to 50 bits (double precision) and of 53 to 55 (integers), ciphertext primes first
MIXED = [(50, 43, 47, 45, 50, 44, 50, 50), (55, 53, 54, 55, 53, 54, 55, 55)]


@pytest.mark.parametrize("log_n", [10, 12, 13, 16])
@pytest.mark.parametrize("bits", MIXED)
def test_moduli_of_unequal_lengths(log_n, bits):
    p, orc, ctx = world(log_n, 6, 2, 3, bits)
    rng = np.random.default_rng(log_n)
    for level in (5, 4):
        x = ciphertexts(rng, p, level, 12)
        for dtype, c_out in ((np.int8, 2), (np.int32, 11)):
            info = np.iinfo(dtype)
            w = rng.integers(info.min, info.max, size=(1, c_out, 12), endpoint=True).astype(dtype)
            got = hx.he_linear_grouped(ctx, level, (1,), hx.from_host(x)[None], torch.from_numpy(w).cuda(), (1 << 40) + 77)
            assert np.array_equal(hx.to_host(got), np.array(orc.linear_grouped([x], level, (1,), w, (1 << 40) + 77))), (level, dtype)
        tab = np.stack([rand_poly(rng, p.moduli[:level + 1], orc.N) for _ in range(10)])
        got = hx.he_rope_axes(ctx, level, hx.from_host(x)[None], hx.from_host(tab[:5]), hx.from_host(tab[5:]), interleaved=True, inverse=level == 4)
        assert np.array_equal(hx.to_host(got[0]), np.array(orc.rope_axes(x, level, tab[:5], tab[5:], True, level == 4))), level
    level, channels = 5, 3
    x, g, res = ciphertexts(rng, p, level, channels), ciphertexts(rng, p, level, channels), ciphertexts(rng, p, 1, channels)
    gp = np.stack([rand_poly(rng, p.moduli[:level + 1], orc.N) for _ in range(channels)])
    key = np.stack([rand_ct(rng, p.moduli, p.num_q + p.num_p - 1, orc.N) for _ in range(p.dnum)])
    rlk, k = hx.ckks_key_load(ctx, hx.from_host(key), 0), (1 << 40, -(3 << 47), 5 << 48, 1 << 49, -(3 << 49))
    for gate in (None, g, gp):
        got = hx.he_norm_gate(ctx, level, hx.from_host(x), k[0], k[1], k[2], k[4:], rlk, None if gate is None else hx.from_host(gate), hx.from_host(res), k[3])
        assert np.array_equal(hx.to_host(got), np.array(orc.norm_gate(x, level, k[0], k[1], k[2], k[4:], key, gate, res, k[3])))


@pytest.mark.parametrize("log_n,bits", [(8, 50), (12, 50), (14, 50), (12, 56)])
def test_contexts_without_key_switching(log_n, bits):
    """Products and rotary positions need no key: their divisions go by the kernels that such a context has."""
    p, orc, ctx = world(log_n, 4, 0, 0, bits)
    rng = np.random.default_rng(log_n)
    x = ciphertexts(rng, p, 3, 18)
    for c_out in (2, 40):
        w = rng.integers(-32768, 32768, size=(2, c_out, 9)).astype(np.int16)
        got = hx.he_linear_grouped(ctx, 3, (1, 1), hx.from_host(x).unflatten(0, (2, 9)), torch.from_numpy(w).cuda(), 1 << 33)
        assert np.array_equal(hx.to_host(got), np.array(orc.linear_grouped(x.reshape(2, 9, 2, 4, orc.N), 3, (1, 1), w, 1 << 33)))
    tab = np.stack([rand_poly(rng, p.moduli[:4], orc.N) for _ in range(8)])
    got = hx.he_rope_axes(ctx, 3, hx.from_host(x).unflatten(0, (2, 9)), hx.from_host(tab[:4]), hx.from_host(tab[4:]))
    for h in range(2):
        assert np.array_equal(hx.to_host(got[h]), np.array(orc.rope_axes(x[9 * h:9 * h + 9], 3, tab[:4], tab[4:])))
