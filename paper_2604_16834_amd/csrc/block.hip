// Kernels of a transformer block's operators on channel-by-channel packed ciphertexts (ciphertext c of a vector = channel c, the
// slots = the tokens or positions of a batch): sums of channels with integer weights per expert, the rotation of channel pairs by
// plaintext angles, the sum of squares over channels.  All of them are pointwise over evaluation points.
#include "ctx.h"

#define BK_THREADS 256

// ---- sums over channels with the weights of one expert ------------------------------------------------------
// acc[r][o][comp][e][x] = (sum_c W[o][c] * in[r][c][comp][e][x]) * mult[e] + (comp == 0 ? bias[o][e] : 0)   mod q_e
// The products are summed as signed 128-bit integers: a term is below 2^31 q in magnitude, 2^16 of them below 2^47 q, so with 2^48 q
// added the sum is positive and below 2^49 q, which barrett_reduce takes.
#define LG_OUT_TILE 4
template <class W>
__global__ __launch_bounds__(BK_THREADS) void linear_sum_kernel(const u64* __restrict__ in, size_t in_ct, size_t in_comp, const W* __restrict__ w,
                                                                size_t w_out, size_t w_in, const u64* __restrict__ bias, LimbScalars mult,
                                                                u64* __restrict__ acc, const ModConst* __restrict__ mc, u32 N, u32 limbs,
                                                                u32 c_in, u32 c_out, u32 o_tiles) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 e = blockIdx.y % limbs, comp = blockIdx.y / limbs, row = blockIdx.z / o_tiles, o0 = blockIdx.z % o_tiles * LG_OUT_TILE;
    const ModConst m = mc[e];
    const u64* src = in + (size_t)row * c_in * in_ct + comp * in_comp + (size_t)e * N + x;
    __int128 sum[LG_OUT_TILE];
#pragma unroll
    for (u32 t = 0; t < LG_OUT_TILE; t++) sum[t] = 0;
    for (u32 ch = 0; ch < c_in; ch++) {
        const long long v = (long long)src[ch * in_ct];
#pragma unroll
        for (u32 t = 0; t < LG_OUT_TILE; t++) {
            const u32 o = o0 + t < c_out ? o0 + t : c_out - 1;
            sum[t] += (__int128)v * (long long)w[o * w_out + ch * w_in];
        }
    }
#pragma unroll
    for (u32 t = 0; t < LG_OUT_TILE; t++) {
        if (o0 + t >= c_out) return;
        const unsigned __int128 s = (unsigned __int128)(sum[t] + ((__int128)m.q << 48));
        U128 r;
        r.lo = (u64)s;
        r.hi = (u64)(s >> 64);
        u64 v = mulmod_barrett(barrett_reduce(r, m), mult.v[e], m);
        if (bias && comp == 0) v = add_mod(v, bias[(size_t)(o0 + t) * limbs + e], m.q);
        acc[(((size_t)row * c_out + o0 + t) * 2 + comp) * limbs * N + (size_t)e * N + x] = v;
    }
}

// The same for moduli below 2^50 and few channels, in double precision (f64m_dot_w: chains of eight exact products of centred residues and
// weights): a thread reads a column's channels eight at a time and adds a chain to each of OT outputs.
template <class W, u32 OT>
__global__ __launch_bounds__(BK_THREADS) void linear_sum_f64_kernel(const u64* __restrict__ in, size_t in_ct, size_t in_comp, const W* __restrict__ w,
                                                                    size_t w_out, size_t w_in, const u64* __restrict__ bias, LimbScalars mult,
                                                                    u64* __restrict__ acc, const ModConstF* __restrict__ mcf, u32 N, u32 limbs,
                                                                    u32 c_in, u32 c_out, u32 o_tiles) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 e = blockIdx.y % limbs, comp = blockIdx.y / limbs, row = blockIdx.z / o_tiles, o0 = blockIdx.z % o_tiles * OT;
    const ModConstF m = mcf[e];
    const u64* src = in + (size_t)row * c_in * in_ct + comp * in_comp + (size_t)e * N + x;
    double sum[OT];
#pragma unroll
    for (u32 t = 0; t < OT; t++) sum[t] = 0.0;
    for (u32 c0 = 0; c0 < c_in; c0 += 8) {
        double y[8];
#pragma unroll
        for (u32 a = 0; a < 8; a++) y[a] = f64m_from_u64(src[(c0 + a < c_in ? c0 + a : c_in - 1) * in_ct]);
#pragma unroll
        for (u32 a = 0; a < 8; a++) y[a] = c0 + a < c_in ? f64m_centre(y[a], m.q) : 0.0;
#pragma unroll
        for (u32 t = 0; t < OT; t++) {
            const W* wr = w + (o0 + t < c_out ? o0 + t : c_out - 1) * w_out;
            double v[8];
#pragma unroll
            for (u32 a = 0; a < 8; a++) v[a] = (double)(int)wr[(c0 + a < c_in ? c0 + a : c_in - 1) * w_in];
            sum[t] = f64m_reduce(sum[t] + f64m_dot_w<8>(y, v, m.q, m.qinv), m.q, m.qinv);
        }
    }
    const double k = f64m_from_u64(mult.v[e]);
#pragma unroll
    for (u32 t = 0; t < OT; t++) {
        if (o0 + t >= c_out) return;
        double v = f64m_mulmod_any(sum[t], k, m.q, m.qinv);
        if (bias && comp == 0) v = f64m_reduce(v + f64m_from_u64(bias[(size_t)(o0 + t) * limbs + e]), m.q, m.qinv);
        acc[(((size_t)row * c_out + o0 + t) * 2 + comp) * limbs * N + (size_t)e * N + x] = f64m_canonical(v, m.q);
    }
}

// Up to this many channels on rings that the matrix-core kernel takes.
#define LINEAR_F64_CHANNELS 8

// scratch: linear_mfma_scratch_elems words where linear_mfma_applies
hipError_t launch_linear_sum(const ckks_ctx* c, u32 level, u32 rows, const u64* in, size_t in_ct, size_t in_comp, u32 c_in, u32 c_out,
                             const void* w, u32 weight_bytes, size_t w_out, size_t w_in, const u64* bias, u64 multiplier, u64* acc, u64* scratch,
                             hipStream_t st) {
    if (linear_mfma_applies(c) && c_in > LINEAR_F64_CHANNELS)
        return launch_linear_mfma(c, level, rows, in, in_ct, in_comp, c_in * in_ct, c_in, c_out, w, weight_bytes, w_out, w_in, bias, multiplier, acc, scratch, st);
    LimbScalars mult;
    for (u32 i = 0; i < CKKS_MAX_MODULI; i++) mult.v[i] = i <= level ? multiplier % c->mod[i] : 0;
    const u32 limbs = level + 1, tile = c->small_q ? (c_out <= 2 ? 2 : 8) : LG_OUT_TILE, o_tiles = (c_out + tile - 1) / tile;
    for (u32 r0 = 0; r0 < rows;) {  // the launch's third dimension holds 65535 workgroups
        const u32 most = 65535 / o_tiles, n = rows - r0 < most ? rows - r0 : most;
        const dim3 grid((c->N + BK_THREADS - 1) / BK_THREADS, 2 * limbs, n * o_tiles);
        const u64* src = in + (size_t)r0 * c_in * in_ct;
        u64* dst = acc + (size_t)r0 * c_out * 2 * limbs * c->N;
        ProfScope ps__(c, K_WEIGHTED_SUM, st, 16.0 * n * c->N * limbs * (c_in + c_out), 2.0 * n * c->N * limbs * c_in * c_out);
#define LINEAR_ARGS(W, TABLE) grid, dim3(BK_THREADS), 0, st, src, in_ct, in_comp, (const W*)w, w_out, w_in, bias, mult, dst, TABLE, c->N, limbs, c_in, c_out, o_tiles
#define LINEAR_SUM(W)                                                                               \
    {                                                                                               \
        if (!c->small_q) hipLaunchKernelGGL(linear_sum_kernel<W>, LINEAR_ARGS(W, c->d_mc));         \
        else if (tile == 2) hipLaunchKernelGGL((linear_sum_f64_kernel<W, 2>), LINEAR_ARGS(W, c->d_mcf)); \
        else hipLaunchKernelGGL((linear_sum_f64_kernel<W, 8>), LINEAR_ARGS(W, c->d_mcf));           \
    }
        if (weight_bytes == 1) LINEAR_SUM(int8_t)
        else if (weight_bytes == 2) LINEAR_SUM(int16_t)
        else LINEAR_SUM(int32_t)
#undef LINEAR_SUM
#undef LINEAR_ARGS
        r0 += n;
    }
    return hipGetLastError();
}

// ---- rotation of channel pairs ----------------------------------------------------------------------------
// pair z: y_a = a C - b S, y_b = a S + b C on limbs 0 .. level (S negated for the inverse); y [2 pairs][2][level + 1][N]: y_a, y_b of each
__global__ __launch_bounds__(BK_THREADS) void rope_turn_kernel(const u64* __restrict__ in, size_t in_ct, size_t in_comp, RopePairs P,
                                                               const u64* __restrict__ cs, const u64* __restrict__ sn, u64* __restrict__ y,
                                                               const ModConst* __restrict__ mc, u32 N, u32 limbs) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 e = blockIdx.y % limbs, comp = blockIdx.y / limbs, z = P.z0 + blockIdx.z;
    const u32 j = z % P.n_pairs;
    const size_t head = (size_t)(z / P.n_pairs) * P.head_dim, at = comp * in_comp + (size_t)e * N + x, table = ((size_t)j * limbs + e) * N + x;
    const ModConst m = mc[e];
    const u64 a = in[(head + P.first(j)) * in_ct + at], b = in[(head + P.second(j)) * in_ct + at];
    const u64 c0 = cs[table], sv = sn[table], s0 = P.inverse && sv ? m.q - sv : sv;
    const u64 ya = sub_mod(mulmod_barrett(a, c0, m), mulmod_barrett(b, s0, m), m.q);
    const u64 yb = add_mod(mulmod_barrett(a, s0, m), mulmod_barrett(b, c0, m), m.q);
    const size_t out = ((size_t)blockIdx.z * 2 * 2 + comp) * limbs * N + (size_t)e * N + x;
    y[out] = ya;
    y[out + (size_t)2 * limbs * N] = yb;
}

hipError_t launch_rope_turn(const ckks_ctx* c, u32 level, u32 n, const u64* in, size_t in_ct, size_t in_comp, const RopePairs& P, const u64* cs,
                            const u64* sn, u64* y, hipStream_t st) {
    const u32 limbs = level + 1;
    const dim3 grid((c->N + BK_THREADS - 1) / BK_THREADS, 2 * limbs, n);
    ProfScope ps__(c, K_PTCT_MAC, st, 8.0 * c->N * limbs * n * 10.0, 8.0 * c->N * limbs * n);
    hipLaunchKernelGGL(rope_turn_kernel, grid, dim3(BK_THREADS), 0, st, in, in_ct, in_comp, P, cs, sn, y, c->d_mc, c->N, limbs);
    return hipGetLastError();
}

// ---- limbs 0 .. level - 1 of ciphertexts that nothing is done to ---------------------------------------------
// channels 2 n_pairs .. head_dim of every head, compact at level - 1
__global__ __launch_bounds__(BK_THREADS) void rope_pass_kernel(const u64* __restrict__ in, size_t in_ct, size_t in_comp, RopePairs P,
                                                               u64* __restrict__ out, u32 N, u32 level) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 e = blockIdx.y % level, comp = blockIdx.y / level, rest = P.head_dim - 2 * P.n_pairs, z = P.z0 + blockIdx.z;
    const size_t ch = (size_t)(z / rest) * P.head_dim + 2 * P.n_pairs + z % rest;
    out[((ch * 2 + comp) * level + e) * N + x] = in[ch * in_ct + comp * in_comp + (size_t)e * N + x];
}

hipError_t launch_rope_pass(const ckks_ctx* c, u32 level, u32 n, const u64* in, size_t in_ct, size_t in_comp, const RopePairs& P, u64* out,
                            hipStream_t st) {
    const dim3 grid((c->N + BK_THREADS - 1) / BK_THREADS, 2 * level, n);
    ProfScope ps__(c, K_COPY, st, 32.0 * c->N * level * n, 0.0);
    hipLaunchKernelGGL(rope_pass_kernel, grid, dim3(BK_THREADS), 0, st, in, in_ct, in_comp, P, out, c->N, level);
    return hipGetLastError();
}

// ---- sum of squares over channels ----------------------------------------------------------------------------
// d[0] = sum x0 x0 + add[e], d[1] = 2 sum x0 x1, d[2] = sum x1 x1   mod q_e;  d [3][level + 1][N]
__global__ __launch_bounds__(BK_THREADS) void square_sum_kernel(const u64* __restrict__ in, size_t in_ct, size_t in_comp, u32 channels, LimbScalars add,
                                                                u64* __restrict__ d, const ModConst* __restrict__ mc, u32 N, u32 limbs, u32 lazy_terms) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 e = blockIdx.y;
    const ModConst m = mc[e];
    const u64* src = in + (size_t)e * N + x;
    u64 r0 = add.v[e], r1 = 0, r2 = 0;
    for (u32 c0 = 0; c0 < channels; c0 += lazy_terms) {
        const u32 c1 = channels - c0 < lazy_terms ? channels : c0 + lazy_terms;
        U128 s0 = {0, 0}, s1 = {0, 0}, s2 = {0, 0};
        for (u32 ch = c0; ch < c1; ch++) {
            const u64 a = src[ch * in_ct], b = src[ch * in_ct + in_comp];
            acc_wide(s0, a, a);
            acc_wide(s1, a, b);
            acc_wide(s2, b, b);
        }
        r0 = add_mod(r0, barrett_reduce(s0, m), m.q);
        r1 = add_mod(r1, barrett_reduce(s1, m), m.q);
        r2 = add_mod(r2, barrett_reduce(s2, m), m.q);
    }
    const size_t row = (size_t)e * N + x, poly = (size_t)limbs * N;
    d[row] = r0;
    d[poly + row] = add_mod(r1, r1, m.q);
    d[2 * poly + row] = r2;
}

hipError_t launch_square_sum(const ckks_ctx* c, u32 level, const u64* in, size_t in_ct, size_t in_comp, u32 channels, const LimbScalars& add, u64* d,
                             hipStream_t st) {
    const u32 limbs = level + 1;
    const dim3 grid((c->N + BK_THREADS - 1) / BK_THREADS, limbs);
    ProfScope ps__(c, K_TENSOR, st, 8.0 * c->N * limbs * (2.0 * channels + 3.0), 3.0 * c->N * limbs * channels);
    hipLaunchKernelGGL(square_sum_kernel, grid, dim3(BK_THREADS), 0, st, in, in_ct, in_comp, channels, add, d, c->d_mc, c->N, limbs, c->lazy_terms);
    return hipGetLastError();
}

// out = k ct + (add, 0) on limbs 0 .. level, one residue each per limb; ct with component stride ct_comp, out [2][level + 1][N]
__global__ __launch_bounds__(BK_THREADS) void affine_kernel(const u64* __restrict__ ct, size_t ct_comp, LimbScalars k, LimbScalars add, u64* __restrict__ out,
                                                            const ModConst* __restrict__ mc, u32 N, u32 limbs) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 e = blockIdx.y, comp = blockIdx.z;
    const ModConst m = mc[e];
    const size_t row = (size_t)e * N + x;
    const u64 v = mulmod_barrett(ct[comp * ct_comp + row], k.v[e], m);
    out[(size_t)comp * limbs * N + row] = comp == 0 ? add_mod(v, add.v[e], m.q) : v;
}

hipError_t launch_affine(const ckks_ctx* c, u32 level, const u64* ct, size_t ct_comp, const LimbScalars& k, const LimbScalars& add, u64* out,
                         hipStream_t st) {
    const dim3 grid((c->N + BK_THREADS - 1) / BK_THREADS, level + 1, 2);
    ProfScope ps__(c, K_LINCOMB2, st, 32.0 * c->N * (level + 1.0), 2.0 * c->N * (level + 1.0));
    hipLaunchKernelGGL(affine_kernel, grid, dim3(BK_THREADS), 0, st, ct, ct_comp, k, add, out, c->d_mc, c->N, level + 1);
    return hipGetLastError();
}

// out_z[comp][e] = gate_z[e] * ct_z[comp][e]; ciphertexts and plaintexts at equal distances, out compact
__global__ __launch_bounds__(BK_THREADS) void gate_mul_kernel(const u64* __restrict__ ct, size_t ct_stride, size_t ct_comp, const u64* __restrict__ gate,
                                                              size_t gate_stride, u64* __restrict__ out, const ModConst* __restrict__ mc, u32 N, u32 limbs) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 e = blockIdx.y, z = blockIdx.z;
    const ModConst m = mc[e];
    const size_t row = (size_t)e * N + x;
    const u64 g = gate[z * gate_stride + row];
#pragma unroll
    for (u32 comp = 0; comp < 2; comp++)
        out[((size_t)z * 2 + comp) * limbs * N + row] = mulmod_barrett(ct[z * ct_stride + comp * ct_comp + row], g, m);
}

hipError_t launch_gate_mul(const ckks_ctx* c, u32 level, u32 n, const u64* ct, size_t ct_stride, size_t ct_comp, const u64* gate, size_t gate_stride,
                           u64* out, hipStream_t st) {
    const dim3 grid((c->N + BK_THREADS - 1) / BK_THREADS, level + 1, n);
    ProfScope ps__(c, K_MASK_MUL, st, 40.0 * n * c->N * (level + 1.0), 2.0 * n * c->N * (level + 1.0));
    hipLaunchKernelGGL(gate_mul_kernel, grid, dim3(BK_THREADS), 0, st, ct, ct_stride, ct_comp, gate, gate_stride, out, c->d_mc, c->N, level + 1);
    return hipGetLastError();
}
