// Kernels of the gated recurrence's and the layer norm's operators on channel-by-channel packed ciphertexts (ciphertext c of a vector = channel c, the
// slots = the tokens of a batch of sequences): tensor products with a rotated operand, sums of products over channels, centred channels.  All of them
// are pointwise over evaluation points, but for the rotated operand, which is read through its automorphism: an aligned run of 64 points comes from
// an aligned run of 64 points.
#include "galois.h"

#define RC_THREADS 256

// ---- a sigma_g(h) --------------------------------------------------------------------------------------------
// Item b: the four products of components, by what they are to be multiplied by to decrypt, with k x added where no key switch follows:
//   e0 = a0 sigma(h0) + k x0 (1),  e1 = a1 sigma(h0) + k x1 (s),  u = a0 sigma(h1) (sigma(s)),  v = a1 sigma(h1) (s sigma(s));   each [n][level + 1][N]
__global__ __launch_bounds__(RC_THREADS) void turned_terms_kernel(PtrList8 a, size_t a_comp, PtrList8 h, size_t h_comp, PtrList8 x, size_t x_comp, LimbScalars k, u32 g,
                                                                  u64* __restrict__ out, const ModConst* __restrict__ mc, u32 log_n, u32 limbs, u32 n) {
    const u32 N = 1u << log_n, i = blockIdx.x * RC_THREADS + threadIdx.x;
    if (i >= N) return;
    const u32 e = blockIdx.y, b = blockIdx.z;
    const ModConst m = mc[e];
    const size_t row = (size_t)e * N, at = row + i, from = row + galois_gather_index(i, g, log_n);
    const u64 a0 = a.p[b][at], a1 = a.p[b][a_comp + at], h0 = h.p[b][from], h1 = h.p[b][h_comp + from];
    u64 e0 = mulmod_barrett(a0, h0, m), e1 = mulmod_barrett(a1, h0, m);
    if (x.p[b]) {
        e0 = add_mod(e0, mulmod_barrett(x.p[b][at], k.v[e], m), m.q);
        e1 = add_mod(e1, mulmod_barrett(x.p[b][x_comp + at], k.v[e], m), m.q);
    }
    const size_t poly = (size_t)limbs * N, o = b * poly + at;
    out[o] = e0;
    out[n * poly + o] = e1;
    out[2 * n * poly + o] = mulmod_barrett(a0, h1, m);
    out[3 * n * poly + o] = mulmod_barrett(a1, h1, m);
}

hipError_t launch_turned_terms(const ckks_ctx* c, u32 level, const PtrList8& a, size_t a_comp, const PtrList8& h, size_t h_comp, const PtrList8& x, size_t x_comp,
                               const LimbScalars& k, u32 g, u64* out, u32 n, hipStream_t st) {
    const dim3 grid((c->N + RC_THREADS - 1) / RC_THREADS, level + 1, n);
    ProfScope ps__(c, K_TENSOR, st, 8.0 * c->N * n * (level + 1.0) * 10.0, 6.0 * c->N * n * (level + 1.0));
    hipLaunchKernelGGL(turned_terms_kernel, grid, dim3(RC_THREADS), 0, st, a, a_comp, h, h_comp, x, x_comp, k, g, out, c->d_mc, c->log_n, level + 1, n);
    return hipGetLastError();
}

// Group z: the same products summed over its `per` channels.  g = 1 (closed): d0, d1 = a1 h0 + a0 h1, d2 = v: three terms; otherwise e0, e1, u, v.  out [terms][groups][level + 1][N].
// sum (or null, one group): sum_c a_c on limbs 0 .. sum_limbs - 1, [2][sum_limbs][N]
__global__ __launch_bounds__(RC_THREADS) void tensor_sum_kernel(TensorSum T, u64* __restrict__ out, const ModConst* __restrict__ mc, u32 log_n, u32 limbs, u32 lazy_terms) {
    const u32 N = 1u << log_n, i = blockIdx.x * RC_THREADS + threadIdx.x;
    if (i >= N) return;
    const u32 e = blockIdx.y, z = blockIdx.z;
    const ModConst m = mc[e];
    const size_t row = (size_t)e * N;
    const u64* a = T.a + (size_t)z * T.per * T.a_ct + row + i;
    const u64* b = T.b + (size_t)z * T.per * T.b_ct + row + galois_gather_index(i, T.g, log_n);
    u64 r00 = 0, r10 = 0, r01 = 0, r11 = 0, t0 = 0, t1 = 0;
    for (u32 c0 = 0; c0 < T.per; c0 += lazy_terms) {
        const u32 c1 = T.per - c0 < lazy_terms ? T.per : c0 + lazy_terms;
        U128 s00 = {0, 0}, s10 = {0, 0}, s01 = {0, 0}, s11 = {0, 0};
        for (u32 ch = c0; ch < c1; ch++) {
            const u64 a0 = a[ch * T.a_ct], a1 = a[ch * T.a_ct + T.a_comp], b0 = b[ch * T.b_ct], b1 = b[ch * T.b_ct + T.b_comp];
            acc_wide(s00, a0, b0);
            acc_wide(s10, a1, b0);
            acc_wide(s01, a0, b1);
            acc_wide(s11, a1, b1);
            t0 = add_mod(t0, a0, m.q);
            t1 = add_mod(t1, a1, m.q);
        }
        r00 = add_mod(r00, barrett_reduce(s00, m), m.q);
        r10 = add_mod(r10, barrett_reduce(s10, m), m.q);
        r01 = add_mod(r01, barrett_reduce(s01, m), m.q);
        r11 = add_mod(r11, barrett_reduce(s11, m), m.q);
    }
    const size_t poly = (size_t)limbs * N, term = T.groups * poly;
    u64* o = out + z * poly + row + i;
    o[0] = r00;
    o[term] = T.closed ? add_mod(r10, r01, m.q) : r10;
    o[2 * term] = T.closed ? r11 : r01;
    if (!T.closed) o[3 * term] = r11;
    if (T.sum && e < T.sum_limbs) {
        T.sum[row + i] = t0;
        T.sum[(size_t)T.sum_limbs * N + row + i] = t1;
    }
}

hipError_t launch_tensor_sum(const ckks_ctx* c, u32 level, const TensorSum& T, u64* out, hipStream_t st) {
    if (T.groups == 0 || T.groups > 65535 || (T.closed && T.g != 1) || (T.sum && T.groups != 1)) return hipErrorInvalidValue;
    const dim3 grid((c->N + RC_THREADS - 1) / RC_THREADS, level + 1, T.groups);
    ProfScope ps__(c, K_TENSOR, st, 8.0 * c->N * (level + 1.0) * T.groups * (4.0 * T.per + 4.0), 4.0 * c->N * (level + 1.0) * T.groups * T.per);
    hipLaunchKernelGGL(tensor_sum_kernel, grid, dim3(RC_THREADS), 0, st, T, out, c->d_mc, c->log_n, level + 1, c->lazy_terms);
    return hipGetLastError();
}

// ---- layer norm ----------------------------------------------------------------------------------------------
// d = C sum_c x_c x_c - S S + (add, 0), S = sum_c x_c: with the variance's C^2 var = C sum x^2 - (sum x)^2 one pass over the channels gives both.
// d [3][limbs][N], sum [2][limbs][N]
__global__ __launch_bounds__(RC_THREADS) void centred_squares_kernel(const u64* __restrict__ in, size_t in_ct, size_t in_comp, u32 channels, LimbScalars add, u64* __restrict__ d,
                                                                     u64* __restrict__ sum, const ModConst* __restrict__ mc, u32 N, u32 limbs, u32 lazy_terms) {
    const u32 i = blockIdx.x * RC_THREADS + threadIdx.x;
    if (i >= N) return;
    const u32 e = blockIdx.y;
    const ModConst m = mc[e];
    const size_t row = (size_t)e * N + i, poly = (size_t)limbs * N;
    const u64* src = in + row;
    u64 r0 = 0, r1 = 0, r2 = 0, t0 = 0, t1 = 0;
    for (u32 c0 = 0; c0 < channels; c0 += lazy_terms) {
        const u32 c1 = channels - c0 < lazy_terms ? channels : c0 + lazy_terms;
        U128 s0 = {0, 0}, s1 = {0, 0}, s2 = {0, 0};
        for (u32 ch = c0; ch < c1; ch++) {
            const u64 a = src[ch * in_ct], b = src[ch * in_ct + in_comp];
            acc_wide(s0, a, a);
            acc_wide(s1, a, b);
            acc_wide(s2, b, b);
            t0 = add_mod(t0, a, m.q);
            t1 = add_mod(t1, b, m.q);
        }
        r0 = add_mod(r0, barrett_reduce(s0, m), m.q);
        r1 = add_mod(r1, barrett_reduce(s1, m), m.q);
        r2 = add_mod(r2, barrett_reduce(s2, m), m.q);
    }
    const u64 C = reduce_word(channels, m);
    r0 = sub_mod(mulmod_barrett(r0, C, m), mulmod_barrett(t0, t0, m), m.q);
    r1 = sub_mod(mulmod_barrett(r1, C, m), mulmod_barrett(t0, t1, m), m.q);
    r2 = sub_mod(mulmod_barrett(r2, C, m), mulmod_barrett(t1, t1, m), m.q);
    d[row] = add_mod(r0, add.v[e], m.q);
    d[poly + row] = add_mod(r1, r1, m.q);
    d[2 * poly + row] = r2;
    sum[row] = t0;
    sum[poly + row] = t1;
}

hipError_t launch_centred_squares(const ckks_ctx* c, u32 level, const u64* in, size_t in_ct, size_t in_comp, u32 channels, const LimbScalars& add, u64* d, u64* sum,
                                  hipStream_t st) {
    const u32 limbs = level + 1;
    const dim3 grid((c->N + RC_THREADS - 1) / RC_THREADS, limbs);
    ProfScope ps__(c, K_TENSOR, st, 8.0 * c->N * limbs * (2.0 * channels + 5.0), 3.0 * c->N * limbs * channels);
    hipLaunchKernelGGL(centred_squares_kernel, grid, dim3(RC_THREADS), 0, st, in, in_ct, in_comp, channels, add, d, sum, c->d_mc, c->N, limbs, c->lazy_terms);
    return hipGetLastError();
}

// out_z = C x_z - S on limbs 0 .. limbs - 1, out [n][2][limbs][N]
__global__ __launch_bounds__(RC_THREADS) void centre_kernel(const u64* __restrict__ in, size_t in_ct, size_t in_comp, u32 channels, const u64* __restrict__ sum, size_t sum_comp,
                                                            u64* __restrict__ out, const ModConst* __restrict__ mc, u32 N) {
    const u32 i = blockIdx.x * RC_THREADS + threadIdx.x;
    if (i >= N) return;
    const u32 limbs = gridDim.y / 2, e = blockIdx.y % limbs, comp = blockIdx.y / limbs, z = blockIdx.z;
    const ModConst m = mc[e];
    const size_t row = (size_t)e * N + i;
    const u64 v = mulmod_barrett(in[z * in_ct + comp * in_comp + row], reduce_word(channels, m), m);
    out[((size_t)z * 2 + comp) * limbs * N + row] = sub_mod(v, sum[comp * sum_comp + row], m.q);
}

hipError_t launch_centre(const ckks_ctx* c, u32 limbs, u32 n, const u64* in, size_t in_ct, size_t in_comp, u32 channels, const u64* sum, size_t sum_comp, u64* out,
                         hipStream_t st) {
    const dim3 grid((c->N + RC_THREADS - 1) / RC_THREADS, 2 * limbs, n);
    ProfScope ps__(c, K_LINCOMB2, st, 32.0 * c->N * limbs * n, 2.0 * c->N * limbs * n);
    hipLaunchKernelGGL(centre_kernel, grid, dim3(RC_THREADS), 0, st, in, in_ct, in_comp, channels, sum, sum_comp, out, c->d_mc, c->N);
    return hipGetLastError();
}

// d_z = r (x) k_grad (C g_z - S) + (k_norm t) (x) xh_z on limbs 0 .. level: d0, d1, d2, each [n][level + 1][N]
__global__ __launch_bounds__(RC_THREADS) void norm_grad_terms_kernel(NormGradTerms T, u64* __restrict__ out, const ModConst* __restrict__ mc, u32 N, u32 limbs, u32 n) {
    const u32 i = blockIdx.x * RC_THREADS + threadIdx.x;
    if (i >= N) return;
    const u32 e = blockIdx.y, z = blockIdx.z;
    const ModConst m = mc[e];
    const size_t row = (size_t)e * N + i;
    const u64 C = reduce_word(T.channels, m), kg = T.k_grad.v[e], kn = T.k_norm.v[e];
    const u64 r0 = mulmod_barrett(T.inv[row], kg, m), r1 = mulmod_barrett(T.inv[T.inv_comp + row], kg, m);
    const u64 t0 = mulmod_barrett(T.t[row], kn, m), t1 = mulmod_barrett(T.t[T.t_comp + row], kn, m);
    const u64* g = T.g + z * T.g_ct + row;
    const u64* xh = T.norm + z * T.norm_ct + row;
    const u64 g0 = sub_mod(mulmod_barrett(g[0], C, m), T.sum[row], m.q), g1 = sub_mod(mulmod_barrett(g[T.g_comp], C, m), T.sum[T.sum_comp + row], m.q);
    const u64 x0 = xh[0], x1 = xh[T.norm_comp];
    const size_t poly = (size_t)limbs * N, o = z * poly + row;
    out[o] = add_mod(mulmod_barrett(r0, g0, m), mulmod_barrett(t0, x0, m), m.q);
    out[n * poly + o] = add_mod(add_mod(mulmod_barrett(r0, g1, m), mulmod_barrett(r1, g0, m), m.q), add_mod(mulmod_barrett(t0, x1, m), mulmod_barrett(t1, x0, m), m.q), m.q);
    out[2 * n * poly + o] = add_mod(mulmod_barrett(r1, g1, m), mulmod_barrett(t1, x1, m), m.q);
}

hipError_t launch_norm_grad_terms(const ckks_ctx* c, u32 level, const NormGradTerms& T, u64* out, u32 n, hipStream_t st) {
    const dim3 grid((c->N + RC_THREADS - 1) / RC_THREADS, level + 1, n);
    ProfScope ps__(c, K_TENSOR, st, 8.0 * c->N * (level + 1.0) * (7.0 * n + 6.0), 10.0 * c->N * (level + 1.0) * n);
    hipLaunchKernelGGL(norm_grad_terms_kernel, grid, dim3(RC_THREADS), 0, st, T, out, c->d_mc, c->N, level + 1, n);
    return hipGetLastError();
}

// ---- sums of rotations on the extended basis -------------------------------------------------------------------
// out_b = sum_r (P sigma_r(c0_b) + <sigma_r(digits_b), key_r>_0, <sigma_r(digits_b), key_r>_1), b < n: what one stage of a sum over slots divides by P once.  Moduli below 2^50: the
// sums as chains of eight fused multiply-adds on centred doubles (f64m_chain_add).  A thread holds both components of one destination point of NB ciphertexts, so that a
// key word is read once for them, and gathers their digits through each automorphism in turn (a wavefront's 64 points are one aligned run of 512 bytes); the operands of the next
// digit are requested before the present one's are used.  Workgroups are dealt to the eight dies in turn: each die takes a contiguous eighth of the (limb, points) list, so that what
// the rotations gather again comes from its own L2 cache.
struct RotSumKeys {
    const u64* key[ROT_SUM_KEYS];
    u32 g[ROT_SUM_KEYS];
    u32 n;
};
template <int NB>
__global__ __launch_bounds__(RC_THREADS) void rot_sum_kernel(DigitSrc digits, RotSumKeys K, PtrList8 c0s, OutList8 out, u32 add, const u64* __restrict__ negp,
                                                             const ModConstF* __restrict__ mcf, u32 log_n, u32 level, u32 num_q, u32 M, u32 E, u32 beta, u32 n) {
    const u32 N = 1u << log_n, nxb = (N + RC_THREADS - 1) / RC_THREADS;
    const u32 list = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3), e = list / nxb, b0 = blockIdx.y * NB;
    if (e >= E) return;  // whole workgroup
    const u32 x = list % nxb * RC_THREADS + threadIdx.x;
    if (x >= N) return;
    const u32 t = e <= level ? e : num_q + (e - level - 1), own = e <= level ? e / digits.alpha : 0xffffffffu;
    const double q = mcf[t].q, qinv = mcf[t].qinv;
    const u32 terms = beta + (e <= level ? 1 : 0);  // the digits, then c0 (P c0 is zero on the special primes)
    auto centred = [&](u64 v) {
        const double d = f64m_from_u64(v);
        return d > 0.5 * q ? d - q : d;
    };
    const double pres = e <= level ? centred((u64)q - negp[e]) : 0.0;
    const u64* rows[NB];  // digit 0's row of every ciphertext
#pragma unroll
    for (int i = 0; i < NB; i++) rows[i] = digits.digits + (b0 + i < n ? b0 + i : n - 1) * digits.bstride + (size_t)e * N;
    u64 dv[NB], k0 = 0, k1 = 0;
    u32 xs = 0;
    auto load = [&](u32 r, u32 j) {
        if (j == 0) xs = galois_gather_index(x, K.g[r], log_n);
        if (j < beta) {
            const u64* kp = K.key[r] + ((size_t)2 * j * M + t) * N + x;
            k0 = kp[0];
            k1 = kp[(size_t)M * N];
        }
#pragma unroll
        for (int i = 0; i < NB; i++) {
            const u32 b = b0 + i < n ? b0 + i : n - 1;
            const u64* row = j == beta ? c0s.p[b] + (size_t)e * N : (j == own ? digits.own.p[b] + (size_t)e * N : rows[i] + (size_t)j * E * N);
            dv[i] = row[xs];
        }
    };
    double ct[2][NB], cl[2][NB];  // a chain's running sum and remainders; a chain goes on from the last one's reduced sum as one more remainder, below 2^49 + 1: with the eight of a
                                  // chain below 9 2^49 + 1, and with the chain's high part (f64m_chain_join) below 2^53
    auto join = [&]() {
#pragma unroll
        for (int c = 0; c < 2; c++)
#pragma unroll
            for (int i = 0; i < NB; i++) cl[c][i] = f64m_chain_join(ct[c][i], cl[c][i], q, qinv), ct[c][i] = F64M_DOT_BASE;
    };
#pragma unroll
    for (int c = 0; c < 2; c++)
#pragma unroll
        for (int i = 0; i < NB; i++) ct[c][i] = F64M_DOT_BASE, cl[c][i] = 0.0;
    load(0, 0);
    u32 r = 0, j = 0, count = 0;
    while (r < K.n) {
        double y[NB];
        const bool key = j < beta;
        const double w0 = key ? centred(k0) : pres, w1 = centred(k1);
#pragma unroll
        for (int i = 0; i < NB; i++) y[i] = centred(dv[i]);
        if (++j == terms) j = 0, r++;
        if (r < K.n) load(r, j);
#pragma unroll
        for (int i = 0; i < NB; i++) f64m_chain_add(ct[0][i], cl[0][i], y[i], w0);
        if (key) {  // uniform
#pragma unroll
            for (int i = 0; i < NB; i++) f64m_chain_add(ct[1][i], cl[1][i], y[i], w1);
        }
        if (++count == 8) {  // uniform
            join();
            count = 0;
        }
    }
    join();
#pragma unroll
    for (int i = 0; i < NB; i++) {
        if (b0 + i >= n) break;
        u64* o = out.p[b0 + i] + (size_t)e * N + x;
#pragma unroll
        for (int c = 0; c < 2; c++) {
            u64* oc = o + (size_t)c * E * N;
            const double v = add ? f64m_reduce(cl[c][i] + f64m_from_u64(*oc), q, qinv) : cl[c][i];
            *oc = f64m_canonical(v, q);
        }
    }
}

hipError_t launch_rot_sum(const ckks_ctx* c, u32 level, const DigitSrc& digits, const u64* const* keys, const u32* gs, u32 n_keys, const u64* const* c0s, u64* const* outs, u32 n,
                          bool add, hipStream_t st) {
    if (!c->small_q || n == 0 || n > KS_MAX_BATCH || n_keys == 0 || n_keys > ROT_SUM_KEYS) return hipErrorInvalidValue;
    const u32 E = c->ext_limbs(level), beta = c->live_digits(level), nxb = (c->N + RC_THREADS - 1) / RC_THREADS;
    RotSumKeys K = {};
    K.n = n_keys;
    for (u32 r = 0; r < n_keys; r++) K.key[r] = keys[r], K.g[r] = gs[r];
    PtrList8 cl;
    OutList8 ol;
    for (u32 b = 0; b < KS_MAX_BATCH; b++) cl.p[b] = b < n ? c0s[b] : nullptr, ol.p[b] = b < n ? outs[b] : nullptr;
    const u64* negp = c->d_moddown + 2 * c->k_pad + (size_t)c->k_pad * c->num_q + 2 * c->num_q;
    u32 nb = 8;
    while (nb > 1 && (nb / 2 >= n || (u64)nxb * E * ((n + nb - 1) / nb) < 1024)) nb /= 2;
    const dim3 grid((nxb * E + 7) / 8 * 8, (n + nb - 1) / nb);
    ProfScope ps__(c, K_KEY_INNER, st, 8.0 * c->N * (E * (n * (beta + (add ? 4.0 : 2.0)) + n_keys * 2.0 * beta * grid.y) + n * (level + 1.0)), 2.0 * n_keys * n * c->N * E * beta);
#define ROT_SUM(NB_) hipLaunchKernelGGL(rot_sum_kernel<NB_>, grid, dim3(RC_THREADS), 0, st, digits, K, cl, ol, add ? 1u : 0u, negp, c->d_mcf, c->log_n, level, c->num_q, c->M, E, beta, n)
    if (nb == 8) ROT_SUM(8);
    else if (nb == 4) ROT_SUM(4);
    else if (nb == 2) ROT_SUM(2);
    else ROT_SUM(1);
#undef ROT_SUM
    return hipGetLastError();
}

// ---- sums on the extended basis, copies ------------------------------------------------------------------------
// v += w, n polynomials [E][N] each
__global__ __launch_bounds__(RC_THREADS) void add_ext_kernel(u64* __restrict__ v, const u64* __restrict__ w, const ModConst* __restrict__ mc, u32 N, u32 level, u32 num_q) {
    const u32 i = blockIdx.x * RC_THREADS + threadIdx.x;
    if (i >= N) return;
    const u32 e = blockIdx.y;
    const size_t at = ((size_t)blockIdx.z * gridDim.y + e) * N + i;
    v[at] = add_mod(v[at], w[at], mc[e <= level ? e : num_q + (e - level - 1)].q);
}

hipError_t launch_add_ext(const ckks_ctx* c, u32 level, u64* v, const u64* w, u32 n, hipStream_t st) {
    const u32 E = c->ext_limbs(level);
    const dim3 grid((c->N + RC_THREADS - 1) / RC_THREADS, E, n);
    ProfScope ps__(c, K_LINCOMB2, st, 24.0 * c->N * E * n, 0.0);
    hipLaunchKernelGGL(add_ext_kernel, grid, dim3(RC_THREADS), 0, st, v, w, c->d_mc, c->N, level, c->num_q);
    return hipGetLastError();
}

// the first `limbs` limbs of n ciphertexts, compact
__global__ __launch_bounds__(RC_THREADS) void copy_cts_kernel(const u64* __restrict__ in, size_t in_ct, size_t in_comp, u64* __restrict__ out, u32 N) {
    const u32 i = blockIdx.x * RC_THREADS + threadIdx.x;
    if (i >= N) return;
    const u32 limbs = gridDim.y / 2, e = blockIdx.y % limbs, comp = blockIdx.y / limbs, z = blockIdx.z;
    out[(((size_t)z * 2 + comp) * limbs + e) * N + i] = in[z * in_ct + comp * in_comp + (size_t)e * N + i];
}

hipError_t launch_copy_cts(const ckks_ctx* c, u32 limbs, u32 n, const u64* in, size_t in_ct, size_t in_comp, u64* out, hipStream_t st) {
    const dim3 grid((c->N + RC_THREADS - 1) / RC_THREADS, 2 * limbs, n);
    ProfScope ps__(c, K_COPY, st, 32.0 * c->N * limbs * n, 0.0);
    hipLaunchKernelGGL(copy_cts_kernel, grid, dim3(RC_THREADS), 0, st, in, in_ct, in_comp, out, c->N);
    return hipGetLastError();
}
