// Kernels of a transformer block's operators on channel-by-channel packed ciphertexts (ciphertext c of a vector = channel c, the
// slots = the tokens or positions of a batch): sums of channels with integer weights per expert, the rotation of channel pairs by
// plaintext angles, the sum of squares over channels.  All of them are pointwise over evaluation points.
#include "ctx.h"

#define BK_THREADS 256

// ---- sums over channels with the weights of one expert ------------------------------------------------------
struct LinearArgs {
    const u64* in;
    size_t in_ct, in_comp, in_row;
    const void* w;
    size_t w_out, w_in, w_group, bias_group;
    const u64* bias;
    u64* acc;
    size_t acc_ct, acc_comp, acc_row;
    u32 N, limb0, limbs, bias_limbs, c_in, c_out, o_tiles, add;
    LimbScalars mult, bias_mult;
    LinearGroups groups;
};
// Any modulus.  The products are summed as signed 128-bit integers: a term is below 2^31 q in magnitude, 2^16 of them below 2^47 q, so with 2^48 q
// added the sum is positive and below 2^49 q, which barrett_reduce takes.
#define LG_OUT_TILE 4
template <class W>
__global__ __launch_bounds__(BK_THREADS) void linear_sum_kernel(LinearArgs A, const ModConst* __restrict__ mc) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= A.N) return;
    const u32 er = blockIdx.y % A.limbs, e = A.limb0 + er, comp = blockIdx.y / A.limbs, row = blockIdx.z / A.o_tiles, o0 = blockIdx.z % A.o_tiles * LG_OUT_TILE;
    const ModConst m = mc[e];
    const u64* src = A.in + row * A.in_row + comp * A.in_comp + (size_t)e * A.N + x;
    const u32 group = A.groups.id[A.groups.of_row(row)];
    const W* w = (const W*)A.w + group * A.w_group;
    const u64* bias = A.bias ? A.bias + group * A.bias_group : nullptr;
    __int128 sum[LG_OUT_TILE];
#pragma unroll
    for (u32 t = 0; t < LG_OUT_TILE; t++) sum[t] = 0;
    for (u32 ch = 0; ch < A.c_in; ch++) {
        const long long v = (long long)src[ch * A.in_ct];
#pragma unroll
        for (u32 t = 0; t < LG_OUT_TILE; t++) {
            const u32 o = o0 + t < A.c_out ? o0 + t : A.c_out - 1;
            sum[t] += (__int128)v * (long long)w[o * A.w_out + ch * A.w_in];
        }
    }
#pragma unroll
    for (u32 t = 0; t < LG_OUT_TILE; t++) {
        const u32 o = o0 + t;
        if (o >= A.c_out) return;
        const unsigned __int128 s = (unsigned __int128)(sum[t] + ((__int128)m.q << 48));
        U128 r;
        r.lo = (u64)s;
        r.hi = (u64)(s >> 64);
        u64 v = mulmod_barrett(barrett_reduce(r, m), A.mult.v[e], m);
        if (bias && comp == 0) v = add_mod(v, mulmod_barrett(bias[(size_t)o * A.bias_limbs + e], A.bias_mult.v[e], m), m.q);
        u64* acc = A.acc + row * A.acc_row + o * A.acc_ct + comp * A.acc_comp + (size_t)er * A.N + x;
        *acc = A.add ? add_mod(v, *acc, m.q) : v;
    }
}

// Moduli below 2^50, few channels or outputs, in double precision (f64m_dot_w: chains of eight exact products of centred residues and weights): a thread reads a
// column's channels eight at a time and adds a chain to each of OT outputs, whose weights are in LDS.
template <class W, u32 OT>
__global__ __launch_bounds__(BK_THREADS) void linear_sum_f64_kernel(LinearArgs A, const ModConstF* __restrict__ mcf) {
    __shared__ double lw[8 * OT];
    const u32 tid = threadIdx.x, x = blockIdx.x * BK_THREADS + tid, xc = x < A.N ? x : A.N - 1;
    const u32 er = blockIdx.y % A.limbs, e = A.limb0 + er, comp = blockIdx.y / A.limbs, row = blockIdx.z / A.o_tiles, o0 = blockIdx.z % A.o_tiles * OT;
    const ModConstF m = mcf[e];
    const u32 group = A.groups.id[A.groups.of_row(row)];
    const W* w = (const W*)A.w + group * A.w_group;
    const u64* bias = A.bias ? A.bias + group * A.bias_group : nullptr;
    const u64* src = A.in + row * A.in_row + comp * A.in_comp + (size_t)e * A.N + xc;
    u64* acc = A.acc + row * A.acc_row + o0 * A.acc_ct + comp * A.acc_comp + (size_t)er * A.N + xc;
    const u32 n_out = A.c_out - o0 < OT ? A.c_out - o0 : OT;
    u64 old[OT];
    if (A.add) {
#pragma unroll
        for (u32 t = 0; t < OT; t++) old[t] = acc[(t < n_out ? t : 0) * A.acc_ct];
    }
    double sum[OT];
#pragma unroll
    for (u32 t = 0; t < OT; t++) sum[t] = 0.0;
    for (u32 c0 = 0; c0 < A.c_in; c0 += 8) {
        const u32 n = A.c_in - c0 < 8 ? A.c_in - c0 : 8;
        u64 raw[8];
#pragma unroll
        for (u32 a = 0; a < 8; a++)
            if (a < n) raw[a] = src[(c0 + a) * A.in_ct];  // (uniform)
        if (c0) __syncthreads();
        if (tid < 8 * OT) {
            const u32 a = tid / OT, t = tid % OT;
            lw[tid] = a < n && t < n_out ? (double)(int)w[(o0 + t) * A.w_out + (c0 + a) * A.w_in] : 0.0;
        }
        __syncthreads();
        double tt[OT], lo[OT];
#pragma unroll
        for (u32 t = 0; t < OT; t++) tt[t] = F64M_DOT_BASE, lo[t] = 0.0;
#pragma unroll
        for (u32 a = 0; a < 8; a++)
            if (a < n) {
                const double y = f64m_centre(f64m_from_u64(raw[a]), m.q);
#pragma unroll
                for (u32 t = 0; t < OT; t++) f64m_chain_add(tt[t], lo[t], y, lw[a * OT + t]);
            }
#pragma unroll
        for (u32 t = 0; t < OT; t++) sum[t] = f64m_reduce(sum[t] + f64m_chain_join(tt[t], lo[t], m.q, m.qinv), m.q, m.qinv);
    }
    if (x >= A.N) return;
    const double k = f64m_from_u64(A.mult.v[e]), kb = f64m_from_u64(A.bias_mult.v[e]);
#pragma unroll
    for (u32 t = 0; t < OT; t++) {
        if (t >= n_out) return;
        double v = f64m_mulmod_any(sum[t], k, m.q, m.qinv);
        if (bias && comp == 0)
            v = f64m_reduce(v + f64m_mulmod_any(f64m_from_u64(bias[(size_t)(o0 + t) * A.bias_limbs + e]), kb, m.q, m.qinv), m.q, m.qinv);
        if (A.add) v = f64m_reduce(v + f64m_from_u64(old[t]), m.q, m.qinv);
        acc[t * A.acc_ct] = f64m_canonical(v, m.q);
    }
}

hipError_t launch_linear_sum(const ckks_ctx* c, const LinearSum& S, u64* scratch, bool prepared, hipStream_t st) {
    if (linear_mfma_applies(c, S.c_in, S.c_out)) return launch_linear_mfma(c, S, scratch, prepared, st);
    const u32 tile = c->small_q ? (S.c_out <= 2 ? S.c_out : 8) : LG_OUT_TILE, o_tiles = (S.c_out + tile - 1) / tile;
    if (S.groups.n == 0 || S.groups.n > LINEAR_GROUPS || (u64)S.rows * S.c_out > 1024) return hipErrorInvalidValue;  // (the grid's third dimension)
    const dim3 grid((c->N + BK_THREADS - 1) / BK_THREADS, 2 * S.limbs, S.rows * o_tiles);
    const LinearArgs A = {S.in, S.in_ct, S.in_comp, S.in_row, S.w, S.w_out, S.w_in, S.w_group, S.bias_group, S.bias, S.acc, S.acc_ct, S.acc_comp, S.acc_row,
                          c->N, S.limb0, S.limbs, S.bias_limbs, S.c_in, S.c_out, o_tiles, S.add, S.mult, S.bias_mult, S.groups};
    ProfScope ps__(c, K_WEIGHTED_SUM, st, 16.0 * S.rows * c->N * S.limbs * (S.c_in + (1.0 + S.add) * S.c_out), 2.0 * S.rows * c->N * S.limbs * S.c_in * S.c_out);
#define LINEAR_F64(W, OT) hipLaunchKernelGGL((linear_sum_f64_kernel<W, OT>), grid, dim3(BK_THREADS), 0, st, A, c->d_mcf)
#define LINEAR_SUM(W)                                                                                            \
    {                                                                                                            \
        if (!c->small_q) hipLaunchKernelGGL(linear_sum_kernel<W>, grid, dim3(BK_THREADS), 0, st, A, c->d_mc);    \
        else if (tile == 1) LINEAR_F64(W, 1);                                                                    \
        else if (tile == 2) LINEAR_F64(W, 2);                                                                    \
        else LINEAR_F64(W, 8);                                                                                   \
    }
    if (S.weight_bytes == 1) LINEAR_SUM(int8_t)
    else if (S.weight_bytes == 2) LINEAR_SUM(int16_t)
    else LINEAR_SUM(int32_t)
#undef LINEAR_SUM
#undef LINEAR_F64
    return hipGetLastError();
}

// ---- rotation of channel pairs ----------------------------------------------------------------------------
// pair z: y_a = a C - b S, y_b = a S + b C on limbs limb0 .. level (S negated for the inverse); y [2 pairs][2][limbs][N]: y_a, y_b of each
__global__ __launch_bounds__(BK_THREADS) void rope_turn_kernel(const u64* __restrict__ in, size_t in_ct, size_t in_comp, RopePairs P,
                                                               const u64* __restrict__ cs, const u64* __restrict__ sn, u64* __restrict__ y,
                                                               const ModConst* __restrict__ mc, u32 N, u32 limb0, u32 limbs) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 er = blockIdx.y % limbs, e = limb0 + er, comp = blockIdx.y / limbs, z = P.z0 + blockIdx.z;
    const u32 j = z % P.n_pairs;
    const size_t head = (size_t)(z / P.n_pairs) * P.head_dim, at = comp * in_comp + (size_t)e * N + x, table = ((size_t)j * (limb0 + limbs) + e) * N + x;
    const ModConst m = mc[e];
    const u64 a = in[(head + P.first(j)) * in_ct + at], b = in[(head + P.second(j)) * in_ct + at];
    const u64 c0 = cs[table], sv = sn[table], s0 = P.inverse && sv ? m.q - sv : sv;
    const u64 ya = sub_mod(mulmod_barrett(a, c0, m), mulmod_barrett(b, s0, m), m.q);
    const u64 yb = add_mod(mulmod_barrett(a, s0, m), mulmod_barrett(b, c0, m), m.q);
    const size_t out = ((size_t)blockIdx.z * 2 * 2 + comp) * limbs * N + (size_t)er * N + x;
    y[out] = ya;
    y[out + (size_t)2 * limbs * N] = yb;
}

hipError_t launch_rope_turn(const ckks_ctx* c, u32 level, u32 limb0, u32 n, const u64* in, size_t in_ct, size_t in_comp, const RopePairs& P, const u64* cs,
                            const u64* sn, u64* y, hipStream_t st) {
    const u32 limbs = level + 1 - limb0;
    const dim3 grid((c->N + BK_THREADS - 1) / BK_THREADS, 2 * limbs, n);
    ProfScope ps__(c, K_PTCT_MAC, st, 8.0 * c->N * limbs * n * 10.0, 8.0 * c->N * limbs * n);
    hipLaunchKernelGGL(rope_turn_kernel, grid, dim3(BK_THREADS), 0, st, in, in_ct, in_comp, P, cs, sn, y, c->d_mc, c->N, limb0, limbs);
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
                                                              size_t gate_stride, u64* __restrict__ out, const ModConst* __restrict__ mc, u32 N, u32 limb0) {
    const u32 x = blockIdx.x * BK_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 limbs = gridDim.y, e = limb0 + blockIdx.y, z = blockIdx.z;
    const ModConst m = mc[e];
    const size_t row = (size_t)e * N + x;
    const u64 g = gate[z * gate_stride + row];
#pragma unroll
    for (u32 comp = 0; comp < 2; comp++)
        out[(((size_t)z * 2 + comp) * limbs + blockIdx.y) * N + x] = mulmod_barrett(ct[z * ct_stride + comp * ct_comp + row], g, m);
}

hipError_t launch_gate_mul(const ckks_ctx* c, u32 level, u32 limb0, u32 n, const u64* ct, size_t ct_stride, size_t ct_comp, const u64* gate, size_t gate_stride,
                           u64* out, hipStream_t st) {
    const dim3 grid((c->N + BK_THREADS - 1) / BK_THREADS, level + 1 - limb0, n);
    ProfScope ps__(c, K_MASK_MUL, st, 40.0 * n * c->N * (level + 1.0 - limb0), 2.0 * n * c->N * (level + 1.0 - limb0));
    hipLaunchKernelGGL(gate_mul_kernel, grid, dim3(BK_THREADS), 0, st, ct, ct_stride, ct_comp, gate, gate_stride, out, c->d_mc, c->N, limb0);
    return hipGetLastError();
}
