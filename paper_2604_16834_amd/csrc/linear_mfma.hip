// Matrix products grouped by expert on the matrix cores (he_linear_grouped, moduli below 2^50): for every limb e, component and row
//     acc[o][x] = K * sum_c W[o][c] * X[c][x] + bias[o]  mod q_e,      o < c_out, c < c_in, x < N,
// W small signed integers that are the same for all limbs.
//
// Residues are written in seven signed base-256 digits; W's two's complement bytes b_0 .. b_{DW-1}, b_0 .. b_{DW-2} less 128, are DW signed digits of
// W - 128 (1 + 256 + ...), which reaches the type's whole range (digits of W itself would not: 2^31 - 1 takes a fifth), and what that leaves out is the
// constant times the column's sum, one number for all outputs.  The digit products are exact 8-bit integer matrix products with 32-bit sums,
// added up by diagonal.
//
// Fold: a diagonal is below DW * 256 channels * 2^14 <= 2^24, so four of them in a row, D_0 + 2^8 D_1 + 2^16 D_2 + 2^24 D_3, are an exact double below
// 2^49; the two or three groups and the column's sum are then one chain of fused multiply-adds with the constants K 2^(32 g) mod q, centred
// (f64m_dot_w): 45 double-precision operations an output, the multiplier included.
//
// A workgroup owns 64 (CT = 2) or 32 columns of one row, component and limb: it reads them once, for all channels, turns them into digits in LDS, and its
// four waves take the 32-output tiles in turn, so X streams from HBM exactly once for any number of outputs.  Bound by HBM up to 64 x 64 channels (a column
// is 8 (c_in + c_out) bytes against c_in c_out 7 DW digit products); two workgroups per CU, so that one's matrix instructions run under
// the other's loads and folds.  More than 256 channels: launches that add to what the one before them left.
#include "ctx.h"

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

#define LM_THREADS 256
#define LM_DX 7                      // digits of a residue
#define LM_BIAS 0x0080808080808080ull
#define LM_CHUNK 256                 // channels of a launch

// ---- weights -> digit planes in A-operand layout: wa[((ot*KS + ks)*DW + dw)*64 + lane] = 16 bytes, digit dw of
//   W[32*ot + lane%32][32*ks + 16*(lane/32) + j], j < 16  (zero beyond c_out and c_in)
template <class W>
__global__ __launch_bounds__(LM_THREADS) void linear_prep_kernel(const W* __restrict__ w, size_t w_out, size_t w_in, uint4* __restrict__ wa, u32 c_out,
                                                                 u32 c_in, u32 KS, u32 OT) {
    constexpr u32 DW = sizeof(W);
    const u32 idx = blockIdx.x * LM_THREADS + threadIdx.x;
    if (idx >= OT * KS * DW * 64) return;
    const u32 lane = idx & 63, dw = (idx >> 6) % DW, ks = (idx >> 6) / DW % KS, ot = (idx >> 6) / DW / KS;
    const u32 o = 32 * ot + (lane & 31), c0 = 32 * ks + 16 * (lane >> 5);
    u32 words[4];
#pragma unroll
    for (u32 m = 0; m < 4; m++) {
        u32 v = 0;
#pragma unroll
        for (u32 j = 0; j < 4; j++) {
            const u32 ch = c0 + 4 * m + j;
            u32 d = 0;
            if (o < c_out && ch < c_in) {
                d = (u32)((int)w[o * w_out + ch * w_in] >> (8 * dw)) & 0xffu;
                if (dw + 1 < DW) d ^= 0x80u;  // less 128
            }
            v |= d << (8 * j);
        }
        words[m] = v;
    }
    wa[idx] = make_uint4(words[0], words[1], words[2], words[3]);
}

// {a.b[i], b.b[i], c.b[i], d.b[i]} for i = 0..3 from four dwords
__device__ __forceinline__ void lm_transpose(u32 a, u32 b, u32 c, u32 d, u32* o) {
    const u32 ab_lo = __builtin_amdgcn_perm(b, a, 0x05010400u), ab_hi = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const u32 cd_lo = __builtin_amdgcn_perm(d, c, 0x05010400u), cd_hi = __builtin_amdgcn_perm(d, c, 0x07030602u);
    o[0] = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x05040100u);
    o[1] = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x07060302u);
    o[2] = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x05040100u);
    o[3] = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x07060302u);
}

struct LinearMfmaArgs {
    const u64* in;
    size_t in_ct, in_comp, in_row;
    const uint4* wa;
    const u64* bias;  // [c_out][limbs] or null
    u64* acc;         // [row][c_out][2][limbs][N]
    const ModConstF* mcf;
    u32 N, limbs, c_in, c_out, KS, OT, ot_per_wg, add;
};
// per limb: K 2^(32 g) mod q, centred, g < 3, and the column sum's constant
struct LinearConsts {
    double c[4][CKKS_MAX_MODULI];
};

template <u32 DW, u32 CT>
__global__ __launch_bounds__(LM_THREADS, 2) void linear_mfma_kernel(LinearMfmaArgs A, LinearConsts K) {
    constexpr u32 DIAGS = LM_DX + DW - 1, GROUPS = (DIAGS + 3) / 4, COLS = 32 * CT, KG = LM_THREADS / COLS;  // KG groups of 16 channels at a time
    extern __shared__ uint4 lds[];  // [CT][KS][7][64], then the column sums
    const u32 tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const u32 KS = A.KS, N = A.N;
    u64* colsum = reinterpret_cast<u64*>(lds + CT * KS * LM_DX * 64);
    const u32 e = blockIdx.y % A.limbs, comp = blockIdx.y / A.limbs;
    const u32 n_split = (A.OT + A.ot_per_wg - 1) / A.ot_per_wg, row = blockIdx.z / n_split, ot_first = blockIdx.z % n_split * A.ot_per_wg;
    const u32 x0 = blockIdx.x * COLS;
    const u64* src = A.in + row * A.in_row + comp * A.in_comp + (size_t)e * N + x0;
    if (DW > 1 && tid < COLS) colsum[tid] = 0;
    if (DW > 1) __syncthreads();

    // the digits of all channels of the columns: thread (col, kg) takes 16 channels of a column
    {
        const u32 col = tid & (COLS - 1), kg = tid / COLS;
        u64 total = 0;
        for (u32 g0 = kg; g0 < 2 * KS; g0 += KG) {
            u64 v[16];
#pragma unroll
            for (u32 j = 0; j < 16; j++) {
                const u32 ch = 16 * g0 + j;
                v[j] = src[(ch < A.c_in ? ch : A.c_in - 1) * A.in_ct + col];
            }
#pragma unroll
            for (u32 j = 0; j < 16; j++)
                if (16 * g0 + j >= A.c_in) v[j] = 0;
            u32 w[8][4];
#pragma unroll
            for (u32 m = 0; m < 4; m++) {
                u64 s[4];
#pragma unroll
                for (u32 j = 0; j < 4; j++) {
                    if (DW > 1) total += v[4 * m + j];
                    s[j] = (v[4 * m + j] + LM_BIAS) ^ LM_BIAS;
                }
                u32 lo[4], hi[4];
                lm_transpose((u32)s[0], (u32)s[1], (u32)s[2], (u32)s[3], lo);
                lm_transpose((u32)(s[0] >> 32), (u32)(s[1] >> 32), (u32)(s[2] >> 32), (u32)(s[3] >> 32), hi);
#pragma unroll
                for (u32 i = 0; i < 4; i++) w[i][m] = lo[i], w[4 + i][m] = hi[i];
            }
            uint4* dst = lds + (((col >> 5) * KS + (g0 >> 1)) * LM_DX) * 64 + 32 * (g0 & 1) + (col & 31);
#pragma unroll
            for (u32 dx = 0; dx < LM_DX; dx++) dst[dx * 64] = make_uint4(w[dx][0], w[dx][1], w[dx][2], w[dx][3]);
        }
        if (DW > 1) atomicAdd(&colsum[col], total);  // whole numbers below 2^58: any order
    }
    __syncthreads();

    const u32 ct = wave % CT, x = x0 + 32 * ct + (lane & 31), half = lane >> 5;
    const ModConstF m = A.mcf[e];
    double cw[GROUPS + 1], part[GROUPS + 1];
#pragma unroll
    for (u32 g = 0; g < GROUPS; g++) cw[g] = K.c[g][e];
    cw[GROUPS] = K.c[3][e];
    if (DW > 1) {  // below 2^58: two halves joined modulo q
        const u64 s = colsum[32 * ct + (lane & 31)];
        const double hi = f64m_reduce((double)(u32)(s >> 32), m.q, m.qinv), lo = (double)(u32)s;
        const double two32 = f64m_reduce(4294967296.0, m.q, m.qinv);
        part[GROUPS] = f64m_reduce(f64m_mulmod_any(hi, two32, m.q, m.qinv) + lo, m.q, m.qinv);
    } else {
        part[GROUPS] = 0.0;
    }
    const uint4* lb = lds + (ct * KS) * LM_DX * 64 + lane;
    const u32 ot_last = min(ot_first + A.ot_per_wg, A.OT);
    for (u32 ot = ot_first + wave / CT; ot < ot_last; ot += 4 / CT) {
        v16i d[DIAGS];
#pragma unroll
        for (u32 s = 0; s < DIAGS; s++)
#pragma unroll
            for (u32 r = 0; r < 16; r++) d[s][r] = 0;
        const uint4* wa = A.wa + (size_t)ot * KS * DW * 64 + lane;
        uint4 an[DW];
#pragma unroll
        for (u32 dw = 0; dw < DW; dw++) an[dw] = wa[dw * 64];
        for (u32 ks = 0; ks < KS; ks++) {
            uint4 a[DW];
#pragma unroll
            for (u32 dw = 0; dw < DW; dw++) a[dw] = an[dw];
            const u32 nx = ks + 1 < KS ? ks + 1 : ks;  // the next step's weights are requested a step ahead
#pragma unroll
            for (u32 dw = 0; dw < DW; dw++) an[dw] = wa[(nx * DW + dw) * 64];
            v4i b[LM_DX];
#pragma unroll
            for (u32 dx = 0; dx < LM_DX; dx++) {
                const uint4 t = lb[(ks * LM_DX + dx) * 64];
                b[dx] = (v4i){(int)t.x, (int)t.y, (int)t.z, (int)t.w};
            }
#pragma unroll
            for (u32 dw = 0; dw < DW; dw++) {
                const v4i av = (v4i){(int)a[dw].x, (int)a[dw].y, (int)a[dw].z, (int)a[dw].w};
#pragma unroll
                for (u32 dx = 0; dx < LM_DX; dx++) d[dx + dw] = __builtin_amdgcn_mfma_i32_32x32x32_i8(av, b[dx], d[dx + dw], 0, 0, 0);
            }
        }
#pragma unroll
        for (u32 r = 0; r < 16; r++) {
            const u32 o = 32 * ot + 8 * (r >> 2) + 4 * half + (r & 3);
#pragma unroll
            for (u32 g = 0; g < GROUPS; g++) {
                const u32 top = 4 * g + 3 < DIAGS ? 4 * g + 3 : DIAGS - 1;
                double t = (double)d[top][r];
                for (u32 s = top; s > 4 * g; s--) t = __builtin_fma(t, 256.0, (double)d[s - 1][r]);
                part[g] = t;
            }
            if (o < A.c_out) {
                u64* out = A.acc + ((((size_t)row * A.c_out + o) * 2 + comp) * A.limbs + e) * N + x;
                double v = DW > 1 ? f64m_dot_w<GROUPS + 1>(part, cw, m.q, m.qinv) : f64m_dot_w<GROUPS>(part, cw, m.q, m.qinv);
                if (A.add) v = f64m_reduce(v + f64m_from_u64(*out), m.q, m.qinv);
                else if (A.bias && comp == 0) v = f64m_reduce(v + f64m_from_u64(A.bias[(size_t)o * A.limbs + e]), m.q, m.qinv);
                *out = f64m_canonical(v, m.q);
            }
        }
    }
}

// The matrix-core kernel takes moduli below 2^50 and whole column tiles.
bool linear_mfma_applies(const ckks_ctx* c) { return c->small_q && c->N >= 64; }

size_t linear_mfma_scratch_elems(u32 c_in, u32 c_out, u32 weight_bytes) {
    return (size_t)((c_out + 31) / 32) * ((c_in + 31) / 32) * weight_bytes * 64 * 2;
}

template <u32 DW>
static hipError_t launch_linear_dw(const LinearMfmaArgs& A, const LinearConsts& K, u32 rows, u32 n_split, hipStream_t st) {
    const u32 CT = A.KS <= 4 ? 2 : 1;
    const dim3 grid(A.N / (32 * CT), 2 * A.limbs, rows * n_split);
    const size_t lds = (size_t)CT * A.KS * LM_DX * 64 * 16 + 64 * 8;
    if (CT == 2) hipLaunchKernelGGL((linear_mfma_kernel<DW, 2>), grid, dim3(LM_THREADS), lds, st, A, K);
    else hipLaunchKernelGGL((linear_mfma_kernel<DW, 1>), grid, dim3(LM_THREADS), lds, st, A, K);
    return hipGetLastError();
}

// scratch: linear_mfma_scratch_elems words
hipError_t launch_linear_mfma(const ckks_ctx* c, u32 level, u32 rows, const u64* in, size_t in_ct, size_t in_comp, size_t in_row, u32 c_in, u32 c_out,
                              const void* w, u32 weight_bytes, size_t w_out, size_t w_in, const u64* bias, u64 multiplier, u64* acc, u64* scratch,
                              hipStream_t st) {
    const u32 limbs = level + 1;
    LinearConsts K;
    for (u32 i = 0; i < CKKS_MAX_MODULI; i++) {
        const u64 q = i < limbs ? c->mod[i] : 3;
        auto centred = [&](unsigned __int128 v) {
            const u64 r = (u64)(v % q);
            return r > q / 2 ? -(double)(q - r) : (double)r;
        };
        unsigned __int128 k = multiplier % q;
        u64 off = 0;  // what the digits leave out
        for (u32 b = 0; b + 1 < weight_bytes; b++) off = off * 256 + 128;
        K.c[3][i] = centred(k * (off % q));
        for (u32 g = 0; g < 3; g++) {
            K.c[g][i] = centred(k);
            k = k * (((u64)1 << 32) % q) % q;
        }
    }
    for (u32 c0 = 0; c0 < c_in; c0 += LM_CHUNK) {
        const u32 nc = c_in - c0 < LM_CHUNK ? c_in - c0 : LM_CHUNK;
        const char* wc = (const char*)w + c0 * w_in * weight_bytes;
        const u32 KS = (nc + 31) / 32, OT = (c_out + 31) / 32, prep = OT * KS * weight_bytes * 64;
        uint4* wa = (uint4*)(scratch + linear_mfma_scratch_elems(c0, c_out, weight_bytes));
        const dim3 pg((prep + LM_THREADS - 1) / LM_THREADS);
        if (weight_bytes == 1) hipLaunchKernelGGL(linear_prep_kernel<int8_t>, pg, dim3(LM_THREADS), 0, st, (const int8_t*)wc, w_out, w_in, wa, c_out, nc, KS, OT);
        else if (weight_bytes == 2) hipLaunchKernelGGL(linear_prep_kernel<int16_t>, pg, dim3(LM_THREADS), 0, st, (const int16_t*)wc, w_out, w_in, wa, c_out, nc, KS, OT);
        else hipLaunchKernelGGL(linear_prep_kernel<int32_t>, pg, dim3(LM_THREADS), 0, st, (const int32_t*)wc, w_out, w_in, wa, c_out, nc, KS, OT);
        // outputs of a workgroup: all, unless that leaves the chip short of workgroups
        const u32 ct = KS <= 4 ? 2 : 1, step = 4 / ct;
        const u64 wgs = (u64)(c->N / (32 * ct)) * 2 * limbs * rows;
        u32 n_split = wgs >= 1024 ? 1 : (u32)(1024 / wgs);
        u32 per = (OT + n_split - 1) / n_split;
        per = (per + step - 1) / step * step;
        n_split = (OT + per - 1) / per;
        for (u32 r0 = 0; r0 < rows;) {  // the launch's third dimension holds 65535 workgroups
            const u32 most = 65535 / n_split, n = rows - r0 < most ? rows - r0 : most;
            const LinearMfmaArgs A = {in + r0 * in_row + c0 * in_ct, in_ct, in_comp, in_row, wa, bias, acc + (size_t)r0 * c_out * 2 * limbs * c->N, c->d_mcf,
                                      c->N, limbs, nc, c_out, KS, OT, per, c0 ? 1u : 0u};
            ProfScope ps__(c, K_WEIGHTED_SUM, st, 16.0 * n * c->N * limbs * (nc + (c0 ? 2.0 : 1.0) * c_out), 2.0 * n * c->N * limbs * nc * c_out);
            hipError_t err = weight_bytes == 1 ? launch_linear_dw<1>(A, K, n, n_split, st)
                                               : (weight_bytes == 2 ? launch_linear_dw<2>(A, K, n, n_split, st) : launch_linear_dw<4>(A, K, n, n_split, st));
            if (err != hipSuccess) return err;
            r0 += n;
        }
    }
    return hipSuccess;
}
