"""A transformer block's operators on the GPU, through the C boundary, against the CPU oracle on the same seeded inputs: every residue
equal (results are integers: there is no tolerance)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2604_16834_amd as hx  # noqa: E402
from oracle import Oracle  # noqa: E402
from workloads import make_params  # noqa: E402
from gpu_common import rand_poly, rand_ct  # noqa: E402

B = hx.binding
_worlds = {}


def world(log_n, num_q, num_p, dnum, bits=50):
    key = (log_n, num_q, num_p, dnum, bits)
    if key not in _worlds:
        p = make_params(log_n, num_q, num_p, dnum, bits=bits)
        _worlds[key] = (p, Oracle(p), hx.Context(p))
    return _worlds[key]


def ciphertexts(rng, p, level, n, edges=True):
    """[n][2][level+1][N] uniform residues, the first points of every limb at 0, 1, q/2 and q - 1."""
    out = np.stack([rand_ct(rng, p.moduli, level, p.n) for _ in range(n)]) if n else np.zeros((0, 2, level + 1, p.n), np.uint64)
    if edges and n:
        for i in range(level + 1):
            q = p.moduli[i]
            out[:, :, i, :4] = (0, 1, q // 2, q - 1)
            out[n // 2, :, i, 4:12] = q - 1
    return out


def spread(ct, level, extra_limbs, gap):
    """The same ciphertexts as a strided view: extra limbs behind each component, `gap` ciphertexts between neighbours."""
    n, _, limbs, N = ct.shape
    wide = torch.full((n, 1 + gap, 2, limbs + extra_limbs, N), -1, dtype=torch.int64, device="cuda")
    wide[:, 0, :, :limbs] = hx.from_host(ct)
    return wide[:, 0]


# ------------------------------------------------------------------------------------------ grouped products
RINGS = [(12, 4, 2, 2, 50), (13, 5, 2, 3, 50), (10, 4, 2, 2, 50), (4, 3, 2, 2, 20), (12, 4, 2, 2, 56), (14, 3, 1, 1, 50)]


def linear_case(ring, level, rows, c_in, c_out, dtype, bias, transposed, multiplier, seed, strided=False, extremes=False):
    p, orc, ctx = world(*ring)
    rng = np.random.default_rng(seed)
    info = np.iinfo(dtype)
    w = rng.integers(info.min, info.max, size=(len(rows), c_in, c_out) if transposed else (len(rows), c_out, c_in), endpoint=True).astype(dtype)
    if extremes:
        w = np.where(w < 0, info.min, info.max).astype(dtype)
        w[0] = info.min
    x = ciphertexts(rng, p, level, sum(rows) * c_in)
    if extremes:
        for i in range(level + 1):
            x[:, 0, i] = p.moduli[i] - 1
    b = np.stack([rng.integers(0, q, size=(len(rows), c_out), dtype=np.uint64) for q in p.moduli[:level + 1]], -1) if bias else None
    want = orc.linear_grouped(x.reshape(sum(rows), c_in, 2, level + 1, orc.N), level, rows, w.transpose(0, 2, 1) if transposed else w, multiplier, b)
    dx = spread(x, level, 2, 1) if strided else hx.from_host(x)
    dx = dx.unflatten(0, (sum(rows), c_in))
    got = hx.he_linear_grouped(ctx, level, rows, dx, torch.from_numpy(w).cuda(), multiplier, hx.from_host(b) if bias else None, transposed)
    assert tuple(got.shape) == (sum(rows), c_out, 2, level, orc.N)
    assert np.array_equal(hx.to_host(got), np.array(want).reshape(sum(rows), c_out, 2, level, orc.N))


@pytest.mark.parametrize("ring", RINGS)
@pytest.mark.parametrize("dtype", [np.int8, np.int16, np.int32])
def test_grouped_product_matches_the_oracle(ring, dtype):
    top = ring[1] - 1
    linear_case(ring, top, (2, 0, 1), 5, 3, dtype, True, False, (1 << 45) + 12345, 1)
    linear_case(ring, 1, (0, 1), 3, 7, dtype, False, True, 1, 2, strided=True)


@pytest.mark.parametrize("c_in,c_out", [(1, 1), (2, 65), (63, 2), (64, 33), (65, 31), (129, 4), (16, 64), (17, 96)])
def test_grouped_product_at_the_edges_of_its_tiles(c_in, c_out):
    linear_case((12, 4, 2, 2, 50), 2, (1, 2), c_in, c_out, np.int16, True, False, 3 << 40, c_in)
    linear_case((12, 4, 2, 2, 50), 2, (1,), c_in, c_out, np.int8, False, True, 3 << 40, c_in + 1)


@pytest.mark.parametrize("ring", [(12, 4, 2, 2, 50), (12, 4, 2, 2, 56), (4, 3, 2, 2, 20), (13, 4, 2, 2, 50)])
@pytest.mark.parametrize("dtype", [np.int8, np.int16, np.int32])
def test_grouped_product_of_extreme_values(ring, dtype):
    """Every weight at the type's ends, residues at q - 1, the largest multiplier: the sums are as long as they get."""
    linear_case(ring, ring[1] - 1, (1,), 70, 5, dtype, True, False, (1 << 64) - 1, 9, extremes=True)


@pytest.mark.parametrize("dtype", [np.int8, np.int32])
@pytest.mark.parametrize("c_in,c_out", [(9, 8), (16, 3), (16, 9), (17, 1), (17, 3), (32, 2), (33, 1), (8, 9), (48, 15), (64, 17), (192, 16), (193, 18)])
def test_grouped_product_where_the_kernels_change(c_in, c_out, dtype):
    """Both sides of the rule that names the kernel, and tiles of 16 outputs and 64 channels filled, by one short of and by one past."""
    linear_case((13, 3, 1, 2, 50), 2, (1, 0, 2), c_in, c_out, dtype, True, False, 5 << 41, 7 * c_in + c_out)
    linear_case((12, 3, 1, 2, 50), 1, (1,), c_in, c_out, dtype, True, True, (1 << 64) - 1, c_out, extremes=True)


@pytest.mark.parametrize("log_n", [5, 6, 7])
@pytest.mark.parametrize("c_in", [20, 100, 250])
def test_grouped_product_on_rings_of_about_one_workgroup(log_n, c_in):
    linear_case((log_n, 4, 2, 2, 20), 3, (1, 2), c_in, 18, np.int16, True, False, 12345, c_in)


def test_grouped_product_of_a_large_ring():
    linear_case((16, 3, 1, 1, 50), 2, (1, 1), 9, 10, np.int32, True, False, 1 << 20, 4, strided=True)


def test_grouped_product_in_chunks_of_rows_and_outputs():
    """More outputs than the workspace holds sums of (2 GiB at N = 2^17, 17 limbs: 60 ciphertexts), and more rows."""
    p, orc, ctx = world(17, 18, 1, 2)
    rng = np.random.default_rng(5)
    level, rows, c_in, c_out = 17, (3, 1), 1, 40
    x = ciphertexts(rng, p, level, 4)
    w = rng.integers(-100, 100, size=(2, c_out, c_in)).astype(np.int8)
    dx = hx.from_host(x).unflatten(0, (4, 1))
    got = hx.he_linear_grouped(ctx, level, rows, dx, torch.from_numpy(w).cuda(), 7)
    for t, g, o in ((0, 0, 0), (1, 0, 39), (2, 0, 17), (3, 1, 38)):
        want = orc.linear_grouped([x[t:t + 1]], level, (1,), w[g:g + 1, o:o + 1], 7)
        assert np.array_equal(hx.to_host(got[t, o]), want[0][0]), (t, o)
    many = hx.he_linear_grouped(ctx, level, (1,), dx[:1], torch.from_numpy(rng.integers(-100, 100, size=(1, 70, 1)).astype(np.int8)).cuda(), 7)
    one = hx.he_linear_grouped(ctx, level, (1,), dx[:1], torch.full((1, 1, 1), 1, dtype=torch.int8, device="cuda"), 7)
    assert tuple(many.shape) == (1, 70, 2, level, 1 << 17) and tuple(one.shape) == (1, 1, 2, level, 1 << 17)


def test_grouped_product_of_many_small_groups():
    """150 groups, every third without rows: more than one launch takes, each with its own weights and biases."""
    p, orc, ctx = world(12, 3, 1, 1)
    rng = np.random.default_rng(9)
    rows = [(0, 1, 2)[g % 3] for g in range(150)]
    for c_in in (3, 11):
        x = ciphertexts(rng, p, 1, sum(rows) * c_in)
        w = rng.integers(-128, 128, size=(150, 2, c_in)).astype(np.int8)
        b = np.stack([rng.integers(0, q, size=(150, 2), dtype=np.uint64) for q in p.moduli[:2]], -1)
        got = hx.he_linear_grouped(ctx, 1, rows, hx.from_host(x).unflatten(0, (sum(rows), c_in)), torch.from_numpy(w).cuda(), 1 << 42, hx.from_host(b))
        want = orc.linear_grouped(x.reshape(sum(rows), c_in, 2, 2, orc.N), 1, rows, w, 1 << 42, b)
        assert np.array_equal(hx.to_host(got), np.array(want))


def test_grouped_product_of_nothing():
    p, orc, ctx = world(12, 4, 2, 2)
    out = hx.he_linear_grouped(ctx, 3, (0, 0), hx.empty(0, 5, 2, 4, orc.N), torch.zeros(2, 3, 5, dtype=torch.int8, device="cuda"), 1)
    assert tuple(out.shape) == (0, 3, 2, 3, orc.N)


@pytest.mark.parametrize("dtype", [np.int8, np.int16, np.int32])
@pytest.mark.parametrize("c_in,c_out,transposed", [(128, 40, True), (256, 33, False), (300, 5, False), (520, 2, True)])
def test_grouped_product_over_many_channels(dtype, c_in, c_out, transposed):
    """Sums as long as one launch of the matrix cores takes and longer; residues whose digits are all -128 and weights at the type's ends in
    half of the products, so that every diagonal is as large as it gets."""
    p, orc, ctx = world(12, 2, 1, 1)
    rng = np.random.default_rng(c_in)
    info = np.iinfo(dtype)
    x = ciphertexts(rng, p, 1, c_in)
    x[:, 0, :, 100:200] = 0x0000808080808080 & ~0x0000800000000000 | 0x0000400000000000
    x[:, :, :, 200:300] = 0x0000008080808080
    w = rng.integers(info.min, info.max, size=(1, c_out, c_in), endpoint=True).astype(dtype)
    w[0, 0], w[0, -1] = info.min, info.max
    w[0, c_out // 2, ::2] = info.min
    dw = torch.from_numpy(np.ascontiguousarray(w.transpose(0, 2, 1)) if transposed else w).cuda()
    got = hx.to_host(hx.he_linear_grouped(ctx, 1, (1,), hx.from_host(x)[None], dw, 987654321, transposed=transposed))
    for o in {0, 1, c_out // 2, c_out - 1}:
        assert np.array_equal(got[0, o], orc.linear_grouped([x], 1, (1,), w[:, o:o + 1], 987654321)[0][0]), o


def test_one_ciphertext_in_the_place_of_all_channels():
    p, orc, ctx = world(12, 4, 2, 2)
    rng = np.random.default_rng(8)
    x, w = ciphertexts(rng, p, 3, 1), rng.integers(-128, 128, size=(1, 2, 5)).astype(np.int8)
    got = hx.he_linear_grouped(ctx, 3, (1,), hx.from_host(x).expand(5, 2, 4, orc.N)[None], torch.from_numpy(w).cuda(), 99)
    assert np.array_equal(hx.to_host(got), np.array(orc.linear_grouped([[x[0]] * 5], 3, (1,), w, 99)))


# ------------------------------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("ring", RINGS)
@pytest.mark.parametrize("heads,head_dim,n_pairs", [(1, 2, 1), (2, 5, 2), (3, 8, 4), (1, 7, 0), (5, 6, 1)])
def test_rotary_positions_match_the_oracle(ring, heads, head_dim, n_pairs):
    p, orc, ctx = world(*ring)
    rng = np.random.default_rng(head_dim)
    for level, interleaved, inverse in ((p.num_q - 1, False, False), (1, True, True), (p.num_q - 1, True, False), (1, False, True)):
        x = ciphertexts(rng, p, level, heads * head_dim)
        tab = np.stack([rand_poly(rng, p.moduli[:level + 1], orc.N) for _ in range(2 * n_pairs)]) if n_pairs else np.zeros((0, level + 1, orc.N), np.uint64)
        tab[:, :, :2] = 0
        for i in range(level + 1):
            tab[:, i, 2:5] = p.moduli[i] - 1
        cos, sin = tab[:n_pairs], tab[n_pairs:]
        want = [orc.rope_axes(x[h * head_dim:(h + 1) * head_dim], level, cos, sin, interleaved, inverse) for h in range(heads)]
        got = hx.he_rope_axes(ctx, level, spread(x, level, 1, 2).unflatten(0, (heads, head_dim)), hx.from_host(cos), hx.from_host(sin), interleaved, inverse)
        assert np.array_equal(hx.to_host(got), np.array(want)), (level, interleaved, inverse)


def test_rotary_positions_of_a_large_ring():
    p, orc, ctx = world(16, 3, 1, 1)
    rng = np.random.default_rng(6)
    x = ciphertexts(rng, p, 2, 18)
    tab = np.stack([rand_poly(rng, p.moduli[:3], orc.N) for _ in range(8)])
    want = [orc.rope_axes(x[9 * h:9 * h + 9], 2, tab[:4], tab[4:]) for h in range(2)]
    got = hx.he_rope_axes(ctx, 2, hx.from_host(x).unflatten(0, (2, 9)), hx.from_host(tab[:4]), hx.from_host(tab[4:]))
    assert np.array_equal(hx.to_host(got), np.array(want))


def test_turning_back_returns_the_input():
    """Encoded angles, forward at the top and back one level below: the decrypted input, through the GPU alone (the noise of two divisions at a
    scale of 2^49, a hundredfold)."""
    from paper_2604_16834_amd.block import grid_positions, rope_angles
    p, orc, ctx = world(12, 4, 2, 2)
    s, s_ntt = orc.gen_secret(1)
    rng = np.random.default_rng(3)
    scale = 2.0 ** 49
    z = rng.uniform(-1, 1, (6, orc.n))
    cts = hx.from_host(np.stack([orc.encrypt(r, scale, 3, s_ntt, 5 + i) for i, r in enumerate(z)]))[None]
    ang = rope_angles(grid_positions((4, 16, 16), 2, orc.n), (1, 1, 1))

    def tables(level):
        return [hx.from_host(np.stack([orc.encode_ntt(f(a), float(p.moduli[level]), level) for a in ang])) for f in (np.cos, np.sin)]
    turned = hx.he_rope_axes(ctx, 3, cts, *tables(3))
    back = hx.to_host(hx.he_rope_axes(ctx, 2, turned, *tables(2), inverse=True))
    dec = np.stack([orc.decrypt(ct, 1, s_ntt, scale) for ct in back[0]])
    assert np.abs(dec - z).max() < 1e-7


# ------------------------------------------------------------------------------------------ norm
NORM_RINGS = [(12, 8, 3, 3, 50), (13, 8, 3, 3, 50), (10, 8, 3, 3, 50), (6, 8, 3, 3, 20), (12, 8, 3, 3, 56), (12, 8, 2, 8, 50)]


def norm_case(ring, level, channels, iterations, gate, residual, seed, strided=False):
    p, orc, ctx = world(*ring)
    rng = np.random.default_rng(seed)
    last = level - 2 - 2 * iterations
    x = ciphertexts(rng, p, level, channels)
    x[0] = 0                                           # a channel of nothing
    key = np.stack([rand_ct(rng, p.moduli, p.num_q + p.num_p - 1, orc.N) for _ in range(p.dnum)])
    rlk = hx.ckks_key_load(ctx, hx.from_host(key), 0)
    k = [int(v) for v in rng.integers(-(1 << 62), 1 << 62, size=4 + iterations)]
    g = {None: None, "plain": np.stack([rand_poly(rng, p.moduli[:level + 1], orc.N) for _ in range(channels)]), "cipher": ciphertexts(rng, p, level, channels)}[gate]
    res = ciphertexts(rng, p, last, channels) if residual else None
    want = orc.norm_gate(x, level, k[0], k[1], k[2], k[4:], key, g, res, k[3])
    dx = spread(x, level, 1, 2) if strided else hx.from_host(x)
    dg = None if g is None else (spread(g, level, 2, 1) if strided and gate == "cipher" else hx.from_host(g))
    dr = None if res is None else (spread(res, last, 1, 1) if strided else hx.from_host(res))
    got = hx.he_norm_gate(ctx, level, dx, k[0], k[1], k[2], k[4:], rlk, dg, dr, k[3])
    assert np.array_equal(hx.to_host(got), np.array(want))


@pytest.mark.parametrize("ring", NORM_RINGS)
@pytest.mark.parametrize("iterations,gate,residual", [(0, None, False), (1, "plain", True), (2, "cipher", False), (2, None, True)])
def test_norm_matches_the_oracle(ring, iterations, gate, residual):
    norm_case(ring, 7, 3, iterations, gate, residual, iterations)
    norm_case(ring, 3 + 2 * iterations, 1, iterations, gate, residual, 50 + iterations, strided=True)


@pytest.mark.parametrize("channels", [2, 8, 9, 16, 17, 33])
def test_norm_of_many_channels(channels):
    norm_case((12, 8, 3, 3, 50), 6, channels, 1, "plain", True, channels)
    norm_case((12, 8, 3, 3, 50), 5, channels, 0, "cipher", True, channels, strided=True)


@pytest.mark.parametrize("ring,channels", [((13, 5, 2, 3, 50), 40), ((4, 5, 2, 3, 20), 300), ((12, 5, 2, 3, 56), 70)])
def test_norm_s_sum_of_squares_over_long_axes(ring, channels):
    norm_case(ring, 4, channels, 0, None, False, 3)


def test_norm_of_a_large_ring():
    norm_case((16, 6, 2, 3, 50), 5, 4, 1, "cipher", True, 8, strided=True)


@pytest.mark.parametrize("gate,residual", [("cipher", True), ("plain", False), (None, True)])
def test_norm_over_two_streams(gate, residual):
    """Sizes at which the gates run beside the chain and the last products in turn on two streams, with the inner products of the limbs that stay
    inside the division: the residues of one stream, of a workspace for one stream, and (three channels) of the oracle; then from a graph."""
    p, orc, ctx = world(16, 6, 2, 3)
    rng = np.random.default_rng(21)
    level, channels, its = 5, 40, 1
    last = level - 2 - 2 * its
    x = ciphertexts(rng, p, level, channels)
    g = {None: None, "plain": np.stack([rand_poly(rng, p.moduli[:level + 1], orc.N) for _ in range(channels)]), "cipher": ciphertexts(rng, p, level, channels)}[gate]
    res = ciphertexts(rng, p, last, channels) if residual else None
    key = np.stack([rand_ct(rng, p.moduli, p.num_q + p.num_p - 1, orc.N) for _ in range(p.dnum)])
    rlk, k = hx.ckks_key_load(ctx, hx.from_host(key), 0), (1 << 40, -(3 << 47), 5 << 48, 1 << 49, -(3 << 49))
    dx, dg, dr = (None if a is None else hx.from_host(a) for a in (x, g, res))

    def call(ws=None, out=None):
        return hx.he_norm_gate(ctx, level, dx, k[0], k[1], k[2], k[4:], rlk, dg, dr, k[3], ws=ws, out=out)
    two = hx.to_host(call())
    kind = {None: B.HE_GATE_NONE, "plain": B.HE_GATE_PLAIN, "cipher": B.HE_GATE_CIPHER}[gate]
    need = hx.he_norm_workspace_bytes(ctx, level, channels, its, kind)
    try:
        hx.ckks_ctx_set_overlap(ctx, False)
        assert np.array_equal(hx.to_host(call()), two)
    finally:
        hx.ckks_ctx_set_overlap(ctx, True)
    only = (0, 17, 39)
    want = orc.norm_gate(x, level, k[0], k[1], k[2], k[4:], key, g, res, k[3], only=only)
    for c, w in zip(only, want):
        assert np.array_equal(two[c], w), c
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), hx.empty(channels, 2, last, orc.N)
    call(ws, out)
    torch.cuda.synchronize()
    st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call(ws, out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(hx.to_host(out), two)
        assert np.array_equal(hx.to_host(call(torch.empty_like(ws))), two)


@pytest.mark.parametrize("bits", [50, 56])
def test_grouped_product_of_more_outputs_than_go_together(bits):
    """1100 outputs: two parts of a row, the second ragged (the transforms number 1024 outputs' components), in both arithmetics."""
    p, orc, ctx = world(12, 3, 1, 1, bits)
    rng = np.random.default_rng(bits)
    x = ciphertexts(rng, p, 1, 2 * 9)
    w = rng.integers(-32768, 32768, size=(1, 1100, 9)).astype(np.int16)
    b = np.stack([rng.integers(0, q, size=(1, 1100), dtype=np.uint64) for q in p.moduli[:2]], -1)
    got = hx.to_host(hx.he_linear_grouped(ctx, 1, (2,), hx.from_host(x).unflatten(0, (2, 9)), torch.from_numpy(w).cuda(), 77, hx.from_host(b)))
    for t, o in ((0, 0), (0, 639), (1, 640), (1, 1023), (0, 1024), (1, 1099)):
        want = orc.linear_grouped([x[9 * t:9 * t + 9]], 1, (1,), w[:, o:o + 1], 77, b[:, o:o + 1])
        assert np.array_equal(got[t, o], want[0][0]), (t, o)


def test_grouped_product_and_rotary_positions_in_several_batches():
    """More outputs and pairs than go through the transforms together (1024 components' limbs, 512 MB of converted limbs): one group of 600 rows on a small ring, and
    36 pairs of 2^16 points and 6 limbs, against the same calls in parts."""
    p, orc, ctx = world(12, 3, 1, 1)
    rng = np.random.default_rng(31)
    x = hx.from_host(ciphertexts(rng, p, 2, 600 * 3)).unflatten(0, (600, 3))
    w = torch.from_numpy(rng.integers(-128, 128, size=(1, 2, 3)).astype(np.int8)).cuda()
    whole = hx.he_linear_grouped(ctx, 2, (600,), x, w, 12345)
    for r in (0, 511, 512, 599):
        assert torch.equal(whole[r:r + 1], hx.he_linear_grouped(ctx, 2, (1,), x[r:r + 1], w, 12345)), r
    assert np.array_equal(hx.to_host(whole[599]), np.array(orc.linear_grouped([hx.to_host(x[599])], 2, (1,), w.cpu().numpy(), 12345)[0]))
    p, orc, ctx = world(16, 6, 2, 3)
    level, heads, n_pairs = 5, 9, 4
    x = hx.from_host(ciphertexts(rng, p, level, 9)).repeat(heads, 1, 1, 1).unflatten(0, (heads, 9))
    x[1:] = x[1:].flip(1)
    tab = [hx.from_host(np.stack([rand_poly(rng, p.moduli[:level + 1], orc.N) for _ in range(n_pairs)])) for _ in range(2)]
    whole = hx.he_rope_axes(ctx, level, x, *tab, interleaved=True)
    for h in (0, 1, 5, 8):
        assert torch.equal(whole[h:h + 1], hx.he_rope_axes(ctx, level, x[h:h + 1], *tab, interleaved=True)), h


def device_residues(seed, p, limbs, *lead):
    """[*lead][limbs][N] uniform residues made on the GPU."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.tensor(p.moduli[:limbs], dtype=torch.int64, device="cuda").unsqueeze(-1)
    return torch.randint(0, (1 << 62), (*lead, limbs, p.n), generator=gen, device="cuda").remainder_(q)


@pytest.mark.parametrize("ring,heads,n_pairs,rest", [((17, 18, 1, 2), 8, 4, 1), ((12, 3, 1, 1), 150, 4, 0)])
def test_rotary_positions_in_two_batches(ring, heads, n_pairs, rest):
    """More pairs than 2 GB of converted limbs (N = 2^17, 17 limbs: 30), and more than 512: single heads of the call against the same heads alone, a pair of the last against
    the oracle."""
    p, orc, ctx = world(*ring)
    level = p.num_q - 1
    x = device_residues(1, p, level + 1, heads, 2 * n_pairs + rest, 2)
    cos, sin = device_residues(2, p, level + 1, n_pairs), device_residues(3, p, level + 1, n_pairs)
    got = hx.he_rope_axes(ctx, level, x, cos, sin, inverse=True)
    for h in (0, heads // 2 - 1, heads // 2, heads - 2, heads - 1):
        assert torch.equal(got[h:h + 1], hx.he_rope_axes(ctx, level, x[h:h + 1], cos, sin, inverse=True)), h
    want = orc.rope_axes(hx.to_host(x[heads - 1, [0, n_pairs]]), level, hx.to_host(cos[:1]), hx.to_host(sin[:1]), inverse=True)
    assert np.array_equal(hx.to_host(got[heads - 1, [0, n_pairs]]), np.array(want))


# ------------------------------------------------------------------------------------------ together, streams, graphs, refusals
def block_calls(ctx, level, x, w, tab, rlk, k, ws):
    h = hx.he_norm_gate(ctx, level, x, k[0], k[1], k[2], k[3:], rlk, ws=ws)
    lv = level - 3 - 2 * len(k[3:])
    y = hx.he_linear_grouped(ctx, lv, (1,), h[None], w, 5 << 30, ws=ws)
    return hx.he_rope_axes(ctx, lv - 1, y, tab[0][:, :lv].contiguous(), tab[1][:, :lv].contiguous(), ws=ws)


@pytest.mark.parametrize("ring", [(12, 9, 3, 3, 50), (14, 9, 3, 3, 50), (12, 9, 3, 3, 56)])
def test_block_on_another_stream_and_from_a_graph(ring):
    """Norm, projection and rotary positions one after the other on a stream of their own, then captured and replayed with eager work in
    between: every replay gives the eager result, also of changed inputs."""
    p, orc, ctx = world(*ring)
    rng = np.random.default_rng(12)
    level, c = 8, 6
    xs = [hx.from_host(ciphertexts(rng, p, level, c)) for _ in range(2)]
    w = torch.from_numpy(rng.integers(-128, 128, size=(1, 4, c)).astype(np.int8)).cuda()
    tab = [hx.from_host(np.stack([rand_poly(rng, p.moduli[:level + 1], orc.N) for _ in range(2)])) for _ in range(2)]
    rlk = hx.ckks_key_load(ctx, hx.from_host(np.stack([rand_ct(rng, p.moduli, p.num_q + p.num_p - 1, orc.N) for _ in range(p.dnum)])), 0)
    k = [int(v) for v in rng.integers(-(1 << 50), 1 << 50, size=4)]
    need = max(hx.he_norm_workspace_bytes(ctx, level, c, 1), hx.he_linear_workspace_bytes(ctx, 3, (1,), c, 4, torch.int8),
               hx.he_rope_workspace_bytes(ctx, 2, 1, 4, 2))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    eager = [block_calls(ctx, level, x, w, tab, rlk, k, ws).clone() for x in xs]
    assert not torch.equal(eager[0], eager[1])
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        other = block_calls(ctx, level, xs[0], w, tab, rlk, k, ws)
    st.synchronize()
    assert torch.equal(other, eager[0])
    x = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = block_calls(ctx, level, x, w, tab, rlk, k, ws)
    for i in (0, 1, 0, 1):
        x.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i])
        assert torch.equal(block_calls(ctx, level, xs[i], w, tab, rlk, k, torch.empty_like(ws)), eager[i])  # eager work between replays


def test_the_block_of_the_example():
    """examples/encrypted_block.py: the three operators together, decrypted, against float64 within what the Newton iterations leave."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "encrypted_block.py")
    spec = importlib.util.spec_from_file_location("encrypted_block", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    diff, bound = example.run(12, verbose=False)
    assert diff <= bound


def raises(code, text, call):
    with pytest.raises(hx.CkksError) as e:
        call()
    assert e.value.code == code and text in str(e.value), str(e.value)


def test_refusals():
    p, orc, ctx = world(12, 8, 3, 3)
    N, key = orc.N, hx.ckks_key_load(ctx, hx.empty(3, 2, 11, 1 << 12), 0)
    rot = hx.ckks_key_load(ctx, key.tensor, 5)
    x, w = hx.empty(1, 3, 2, 8, N), torch.zeros(1, 2, 3, dtype=torch.int8, device="cuda")
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    lin = lambda **kw: hx.he_linear_grouped(**{**dict(ctx=ctx, level=7, group_rows=(1,), x=x, w=w, multiplier=3), **kw})  # noqa: E731
    raises(B.CKKS_ERR_LEVEL_MISMATCH, "level", lambda: lin(level=0))
    raises(B.CKKS_ERR_WORKSPACE_TOO_SMALL, "workspace", lambda: lin(ws=small))
    raises(B.CKKS_ERR_INVALID_ARG, "aligned", lambda: lin(out=hx.empty(2 * 2 * 7 * N + 1)[1:]))
    raises(B.CKKS_ERR_INVALID_ARG, "aligned", lambda: lin(x=hx.empty(3 * 2 * 8 * N + 1)[1:].view(1, 3, 2, 8, N)))
    raises(B.CKKS_ERR_INVALID_ARG, "overlap", lambda: lin(x=x.as_strided((1, 3, 2, 8, N), (0, 8 * N, 8 * N, N, 1))))
    for bad in (dict(multiplier=0), dict(multiplier=1 << 64), dict(group_rows=(2,)), dict(group_rows=(-1,)), dict(w=w.long()), dict(x=x[..., :-1]),
                dict(level=8), dict(x=x[:, :, :, ::2]), dict(bias=hx.empty(1, 2, 7)), dict(out=hx.empty(1, 2, 2, 8, N)), dict(x=x.cpu())):
        with pytest.raises(ValueError):
            lin(**bad)
    assert hx.he_linear_workspace_bytes(ctx, 0, (1,), 3, 2) == 0 and hx.he_linear_workspace_bytes(ctx, 7, (1,), 0, 2) == 0

    cos = hx.empty(1, 8, N)
    rope = lambda **kw: hx.he_rope_axes(**{**dict(ctx=ctx, level=7, x=x, cos=cos, sin=cos), **kw})  # noqa: E731
    raises(B.CKKS_ERR_INVALID_ARG, "pairs", lambda: rope(cos=hx.empty(2, 8, N), sin=hx.empty(2, 8, N)))
    raises(B.CKKS_ERR_WORKSPACE_TOO_SMALL, "workspace", lambda: rope(ws=small))
    raises(B.CKKS_ERR_LEVEL_MISMATCH, "level", lambda: rope(level=0, cos=hx.empty(1, 1, N), sin=hx.empty(1, 1, N)))
    for bad in (dict(sin=hx.empty(2, 8, N)), dict(level=6), dict(x=x[0]), dict(out=hx.empty(1, 3, 2, 8, N))):
        with pytest.raises(ValueError):
            rope(**bad)

    norm = lambda **kw: hx.he_norm_gate(**{**dict(ctx=ctx, level=7, x=x[0], k_eps=1, k_slope=1, k_start=1, k_newton=(1,), rlk=key), **kw})  # noqa: E731
    raises(B.CKKS_ERR_NO_KEY, "relinearisation", lambda: norm(rlk=None))
    raises(B.CKKS_ERR_NO_KEY, "rotation", lambda: norm(rlk=rot))
    raises(B.CKKS_ERR_LEVEL_MISMATCH, "iterations", lambda: norm(k_newton=(1, 1, 1)))
    raises(B.CKKS_ERR_INVALID_ARG, "iterations", lambda: norm(k_newton=(1,) * 17))
    raises(B.CKKS_ERR_WORKSPACE_TOO_SMALL, "workspace", lambda: norm(ws=small))
    for bad in (dict(k_eps=1 << 63), dict(gate=hx.empty(3, 7, N)), dict(residual=hx.empty(3, 2, 3, N)), dict(gate=hx.empty(2, 8, N)), dict(x=x), dict(out=hx.empty(3, 2, 4, N))):
        with pytest.raises(ValueError):
            norm(**bad)
    _, _, plain = world(12, 4, 0, 0)
    raises(B.CKKS_ERR_UNSUPPORTED_PARAMS, "digits", lambda: norm(ctx=plain, level=3, x=hx.empty(2, 2, 4, N), k_newton=()))
