// Kernels of the gated recurrence's and the layer norm's operators on channel-by-channel packed ciphertexts (ciphertext c of a vector = channel c, the
// slots = the tokens of a batch of sequences): tensor products with a rotated operand, sums of products over channels, centred channels.  All of them
// are pointwise over evaluation points, but for the rotated operand, which is read through its automorphism: an aligned run of 64 points comes from
// an aligned run of 64 points.  A few products a word: the pointwise ones are bound by their traffic, so that each forms all it can from what it reads; their figures
// are at N = 2^16 on a card that copies at 5.1 TB/s.
#include "galois.h"

#define RC_THREADS 256

// ---- a sigma_g(h) --------------------------------------------------------------------------------------------
// Item b: the four products of components, with k x added where no key switch follows; in brackets what each is to be multiplied by to decrypt:
//   e0 = a0 sigma(h0) + k x0 (1),  e1 = a1 sigma(h0) + k x1 (s),  u = a0 sigma(h1) (sigma(s)),  v = a1 sigma(h1) (s sigma(s));   each [n][level + 1][N]
// For moduli of 2^50 and more and for small rings; elsewhere the transforms form the four where they use them.  Four items of 24 limbs: 89 us, 0.5 GB.
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
// A thread holds the terms' sums, so that every operand is read once: eight channels of 21 limbs in two groups 83 us, 0.44 GB, 5.3 TB/s.
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
// 32 channels of 24 limbs: 183 us, 0.8 GB read, 4.6 TB/s; centring first would read the channels three times and write them once.
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

// out_z = C x_z - S on limbs 0 .. limbs - 1, out [n][2][limbs][N].  16 channels of 14 limbs: 111 to 203 us, with the other stream's kernels beside it.
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

// d_z = r (x) k_grad (C g_z - S) + (k_norm t) (x) xh_z on limbs 0 .. level: d0, d1, d2, each [n][level + 1][N].  Both products
// are summed before they are decomposed, so that they share one key switch.  Eight channels of 10 limbs: 97 us; operands and results once are 0.33 GB (3.3 TB/s), but the L2 caches fetch 0.42
// and write 0.13 (5.6 TB/s), as the six words that all channels share come again for each, from the last-level cache.
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
// out_b = sum_r (P sigma_r(c0_b) + <sigma_r(digits_b), key_r>_0, <sigma_r(digits_b), key_r>_1), b < n: what one stage of a sum over slots divides by P once.  Moduli below 2^50,
// BETA digits: the sums as chains of fused multiply-adds on centred doubles (f64m_chain_add).  A thread holds both components of one destination point of NB ciphertexts, so that a
// key word is read once for them, and gathers their digits through each automorphism in turn (a wavefront's 64 points are one aligned run of 512 bytes).  Workgroups are dealt to the eight
// dies in turn: each die takes a contiguous eighth of the (limb, points, ciphertexts) list, so that what the rotations gather again, and the keys for the next ciphertexts, come from its own L2
// cache.  16 ciphertexts of 12 + 8 limbs at N = 2^16, seven rotations: 480 us; 1.0 GB have to be moved (196 us), the arithmetic alone takes 220.  An inner product and an addition for every
// rotation took 1160 us; with one term after the other behind branches 530; four ciphertexts a thread 517, two 570; four points of two ciphertexts 575.  It fetches 1.3 GB where the stage's rotations share runs of
// points and 2.5 where they do not; an order of the runs along the first rotation's orbits brought the latter to 1.1 and the kernel from 490 us to 482 on average, too little for its code: the
// waits for gathered words and the arithmetic bound it, not the traffic.
struct RotSumKeys {
    const u64* key[ROT_SUM_KEYS];
    u32 g[ROT_SUM_KEYS];
    u32 n;
};
__device__ __forceinline__ u64 word_at_byte(const u64* poly, u32 byte) { return *reinterpret_cast<const u64*>(reinterpret_cast<const char*>(poly) + byte); }

// LIVE: limb e is one of the ciphertexts' (nothing of c0 is added on the special primes)
template <int BETA, int NB, bool LIVE>
__device__ __forceinline__ void rot_sum_chains(const u64* const (&row)[BETA][NB], const u64* const (&c0)[NB], const RotSumKeys& K, u32 x, u32 log_n, size_t to_limb, size_t kstride,
                                               double q, double qinv, double pres, double (&sum)[2][NB]) {
    // A chain's running sum and remainders; a chain of at most eight terms goes on from the last one's reduced sum as one more remainder, below 2^49 + 1: with the eight of a
    // chain below 9 2^49 + 1, and with what is left of the chain's high part (f64m_chain_join) below 2^53.
    constexpr u32 PER = 8 / (BETA + 1);  // rotations a chain
    double ct[2][NB];
#pragma unroll
    for (int c = 0; c < 2; c++)
#pragma unroll
        for (int i = 0; i < NB; i++) ct[c][i] = F64M_DOT_BASE, sum[c][i] = 0.0;
    auto centred = [&](u64 v) {
        const double d = f64m_from_u64(v);
        return d > 0.5 * q ? d - q : d;
    };
    // The next rotation's operands are requested as the present one's are used, with no branch around a request: a wait is then for the operands that are needed alone.  Behind
    // the last rotation it is requested once more.
    u64 dv[BETA][NB], k0[BETA], k1[BETA], cv[NB];
    const u64* key = K.key[0] + to_limb;
    u32 xs = 8 * galois_gather_index(x, K.g[0], log_n);
    auto request = [&](int j) {
        k0[j] = word_at_byte(key + (size_t)(2 * j) * kstride, 8 * x);
        k1[j] = word_at_byte(key + (size_t)(2 * j + 1) * kstride, 8 * x);
#pragma unroll
        for (int i = 0; i < NB; i++) dv[j][i] = word_at_byte(row[j][i], xs);
    };
    auto request_c0 = [&]() {
#pragma unroll
        for (int i = 0; i < NB; i++) cv[i] = word_at_byte(c0[i], xs);
    };
#pragma unroll
    for (int j = 0; j < BETA; j++) request(j);
    if (LIVE) request_c0();
    for (u32 r = 0, count = 0; r < K.n; r++) {
        const u32 rn = r + 1 < K.n ? r + 1 : r;
        key = K.key[rn] + to_limb;
        xs = 8 * galois_gather_index(x, K.g[rn], log_n);
#pragma unroll
        for (int j = 0; j < BETA; j++) {
            const double w0 = centred(k0[j]), w1 = centred(k1[j]);
            double y[NB];
#pragma unroll
            for (int i = 0; i < NB; i++) y[i] = centred(dv[j][i]);
            request(j);
#pragma unroll
            for (int i = 0; i < NB; i++) {
                f64m_chain_add(ct[0][i], sum[0][i], y[i], w0);
                f64m_chain_add(ct[1][i], sum[1][i], y[i], w1);
            }
        }
        if (LIVE) {
            double y[NB];
#pragma unroll
            for (int i = 0; i < NB; i++) y[i] = centred(cv[i]);
            request_c0();
#pragma unroll
            for (int i = 0; i < NB; i++) f64m_chain_add(ct[0][i], sum[0][i], y[i], pres);
        }
        if (++count == PER || r + 1 == K.n) {  // uniform
            count = 0;
#pragma unroll
            for (int c = 0; c < 2; c++)
#pragma unroll
                for (int i = 0; i < NB; i++) sum[c][i] = f64m_chain_join(ct[c][i], sum[c][i], q, qinv), ct[c][i] = F64M_DOT_BASE;
        }
    }
}

template <int BETA, int NB>
__global__ __launch_bounds__(RC_THREADS) void rot_sum_kernel(const u64* __restrict__ digits, size_t bstride, u32 alpha, RotSumKeys K, PtrList8 cts, OutList8 out, u32 add,
                                                             const u64* __restrict__ negp, const ModConstF* __restrict__ mcf, u32 log_n, u32 level, u32 num_q, u32 M, u32 E, u32 n) {
    const u32 N = 1u << log_n, nxb = (N + RC_THREADS - 1) / RC_THREADS, groups = (n + NB - 1) / NB;
    const u32 list = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3), e = list / (nxb * groups), b0 = list % groups * NB;
    if (e >= E) return;  // whole workgroup
    const u32 x = list / groups % nxb * RC_THREADS + threadIdx.x;
    if (x >= N) return;
    const bool live = e <= level;
    const u32 t = live ? e : num_q + (e - level - 1), own = live ? e / alpha : 0xffffffffu;
    const double q = mcf[t].q, qinv = mcf[t].qinv;
    const u64 *row[BETA][NB], *c0[NB];
#pragma unroll
    for (int i = 0; i < NB; i++) {
        const u32 b = b0 + i < n ? b0 + i : n - 1;
        c0[i] = cts.p[b] + (size_t)(live ? e : 0) * N;
#pragma unroll
        for (int j = 0; j < BETA; j++) row[j][i] = own == (u32)j ? c0[i] + (size_t)(level + 1) * N : digits + b * bstride + ((size_t)j * E + e) * N;
    }
    double sum[2][NB];
    if (live) {
        const double p = q - f64m_from_u64(negp[e]);  // P mod q_e
        rot_sum_chains<BETA, NB, true>(row, c0, K, x, log_n, (size_t)t * N, (size_t)M * N, q, qinv, p > 0.5 * q ? p - q : p, sum);
    } else {
        rot_sum_chains<BETA, NB, false>(row, c0, K, x, log_n, (size_t)t * N, (size_t)M * N, q, qinv, 0.0, sum);
    }
#pragma unroll
    for (int i = 0; i < NB; i++) {
        if (b0 + i >= n) break;
        u64* o = out.p[b0 + i] + (size_t)e * N + x;
#pragma unroll
        for (int c = 0; c < 2; c++) {
            u64* oc = o + (size_t)c * E * N;
            const double v = add ? f64m_reduce(sum[c][i] + f64m_from_u64(*oc), q, qinv) : sum[c][i];
            *oc = f64m_canonical(v, q);
        }
    }
}

bool rot_sum_applies(const ckks_ctx* c, u32 level) { return c->small_q && c->live_digits(level) <= 4; }
hipError_t launch_rot_sum(const ckks_ctx* c, u32 level, const u64* digits, size_t bstride, const u64* const* keys, const u32* gs, u32 n_keys, const u64* const* cts, u64* const* outs, u32 n,
                          bool add, hipStream_t st) {
    if (!rot_sum_applies(c, level) || n == 0 || n > KS_MAX_BATCH || n_keys == 0 || n_keys > ROT_SUM_KEYS) return hipErrorInvalidValue;
    const u32 E = c->ext_limbs(level), beta = c->live_digits(level), nxb = (c->N + RC_THREADS - 1) / RC_THREADS;
    RotSumKeys K = {};
    K.n = n_keys;
    for (u32 r = 0; r < n_keys; r++) K.key[r] = keys[r], K.g[r] = gs[r];
    PtrList8 cl;
    OutList8 ol;
    for (u32 b = 0; b < KS_MAX_BATCH; b++) cl.p[b] = b < n ? cts[b] : nullptr, ol.p[b] = b < n ? outs[b] : nullptr;
    const u64* negp = c->d_moddown + 2 * c->k_pad + (size_t)c->k_pad * c->num_q + 2 * c->num_q;
    // ciphertexts a thread: as many as its registers hold, fewer where a launch would not give every CU four workgroups
    u32 nb = beta <= 2 ? 8 : 4;
    while (nb > 1 && (nb / 2 >= n || (u64)nxb * E * ((n + nb - 1) / nb) < 1024)) nb /= 2;
    const u32 groups = (n + nb - 1) / nb;
    const dim3 grid((nxb * E * groups + 7) / 8 * 8);
    ProfScope ps__(c, K_KEY_INNER, st, 8.0 * c->N * (E * (n * (beta + (add ? 4.0 : 2.0)) + n_keys * 2.0 * beta) + n * (level + 1.0)), 2.0 * n_keys * n * c->N * E * beta);
#define ROT_SUM(B_, NB_) hipLaunchKernelGGL((rot_sum_kernel<B_, NB_>), grid, dim3(RC_THREADS), 0, st, digits, bstride, c->alpha, K, cl, ol, add ? 1u : 0u, negp, c->d_mcf, c->log_n, level, c->num_q, c->M, E, n)
#define ROT_SUM_B(B_)                     \
    {                                     \
        if (nb == 4) ROT_SUM(B_, 4);      \
        else if (nb == 2) ROT_SUM(B_, 2); \
        else ROT_SUM(B_, 1);              \
    }
    if (nb == 8 && beta == 1) ROT_SUM(1, 8);
    else if (nb == 8) ROT_SUM(2, 8);
    else if (beta == 1) ROT_SUM_B(1)
    else if (beta == 2) ROT_SUM_B(2)
    else if (beta == 3) ROT_SUM_B(3)
    else ROT_SUM_B(4)
#undef ROT_SUM_B
#undef ROT_SUM
    return hipGetLastError();
}

// ---- sums on the extended basis, copies ------------------------------------------------------------------------
// v += w, n polynomials [E][N] each: sums of rotations, and of the two key switches of a rotated product, outside the fused passes.  16 polynomials of 21 limbs: 84 us, 0.53 GB.
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
