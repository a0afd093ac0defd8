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
// A workgroup owns 64 columns (up to 64 channels) or 32 of one row, component and limb: it reads them once, for all channels, turns them into digits in LDS, and its
// waves take units of 16 outputs x 16 columns in turn: X is read once for all outputs, unless the columns alone leave the chip short of workgroups
// (fewer than 1024: the outputs are then split over several, each of which reads and converts them).  Such a unit's diagonals are 28 to 40 registers, and
// four waves per SIMD hide each other's loads, products and folds.  Bound by HBM (a column is 8 (c_in + 2 c_out) bytes with what is added to, against c_in c_out 7 DW
// digit products): 64 -> 64 channels, 8-bit weights, three rows of 23 limbs at N = 2^16 3.07 ms, 4.5 TB/s; 256 -> 192, 32-bit weights, two rows of 12 limbs 5.87 ms, 2.7 TB/s.
// Tried and slower: units of 32 x 32 (160 registers of diagonals, two waves per SIMD: 3.25 and 6.5 ms, the matrix pipe 30 % and the vector units 34 % busy, the two
// workgroups of a CU load, multiply and fold in step); one persistent workgroup of eight waves per CU, two of which read and convert the next tile while six multiply
// (6.9 to 9 ms in the second case: too few loads in flight); the next step's weights requested a step ahead (2 % slower: registers); what is added to requested behind
// the products (1 %).  A cheaper fold (neighbouring diagonals joined in 32 bits where they fit, the column's sum added after the chain: a fifth fewer operations) changes
// nothing beyond 1 %.  Loads behind a lane's own bound instead of clamped ones: 10 % slower.  128 columns and 512 threads up to
// 64 channels: 1 to 4 % slower.  More than 256 channels: launches that add to what the one before them left.
#include "ctx.h"

typedef int v4i __attribute__((ext_vector_type(4)));

#define LM_THREADS 256  // linear_prep_kernel
#define LM_DX 7                      // digits of a residue
#define LM_BIAS 0x0080808080808080ull
#define LM_CHUNK 256                 // channels of a launch

// ---- weights -> digit planes in A-operand layout, group by group (blockIdx.y): wa[((ot*KS + ks)*DW + dw)*64 + lane] = 16 bytes, digit dw of
//   W[16*ot + lane%16][64*ks + 16*(lane/16) + j], j < 16  (zero beyond c_out and c_in)
template <class W>
__global__ __launch_bounds__(LM_THREADS) void linear_prep_kernel(const W* __restrict__ w, size_t w_out, size_t w_in, size_t w_group, LinearGroups groups,
                                                                 uint4* __restrict__ wa, size_t wa_group, u32 c_out, u32 c_in, u32 KS, u32 OT) {
    constexpr u32 DW = sizeof(W);
    const u32 idx = blockIdx.x * LM_THREADS + threadIdx.x;
    if (idx >= OT * KS * DW * 64) return;
    w += groups.id[blockIdx.y] * w_group;
    wa += blockIdx.y * wa_group;
    const u32 lane = idx & 63, dw = (idx >> 6) % DW, ks = (idx >> 6) / DW % KS, ot = (idx >> 6) / DW / KS;
    const u32 o = 16 * ot + (lane & 15), c0 = 64 * ks + 16 * (lane >> 4);
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
    size_t wa_group, bias_group;
    const u64* bias;
    u64* acc;
    size_t acc_ct, acc_comp, acc_row;
    const ModConstF* mcf;
    u32 N, limb0, limbs, bias_limbs, c_in, c_out, KS, OT, ot_per_wg, add;
    LinearGroups groups;
};
// per limb: K 2^(32 g) mod q, centred, g < 3, and the column sum's constant
struct LinearConsts {
    double c[4][CKKS_MAX_MODULI], bias[CKKS_MAX_MODULI];
};

template <u32 DW, u32 CT, u32 THREADS, bool ADD>
__global__ __launch_bounds__(THREADS, 4) void linear_mfma_kernel(LinearMfmaArgs A, LinearConsts K) {
    constexpr u32 DIAGS = LM_DX + DW - 1, GROUPS = (DIAGS + 3) / 4, COLS = 16 * CT, OT_STEP = THREADS / 64 / CT;
    extern __shared__ uint4 lds[];  // [CT][KS][7][64], then the column sums
    const u32 tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (a number of steps known here: 64 -> 64 with 32-bit weights 6.54 -> 6.36 ms, 128 -> 96 with 16-bit ones 3.76 -> 3.56; with 8-bit ones the registers that the
    // compiler then takes for loads ahead cost a wave per SIMD, 6.15 instead of 5.9 ms)
    const u32 KS = DW == 1 ? A.KS : (CT == 4 ? 1 : (THREADS == 256 ? 2 : A.KS)), N = A.N;
    u64* colsum = reinterpret_cast<u64*>(lds + CT * KS * LM_DX * 64);
    const u32 er = blockIdx.y % A.limbs, e = A.limb0 + er, comp = blockIdx.y / A.limbs;
    const u32 n_split = (A.OT + A.ot_per_wg - 1) / A.ot_per_wg, row = blockIdx.z / n_split, ot_first = blockIdx.z % n_split * A.ot_per_wg;
    const u32 x0 = blockIdx.x * COLS, gi = A.groups.of_row(row);
    const u64* bias = A.bias ? A.bias + A.groups.id[gi] * A.bias_group : nullptr;
    u64* acc = A.acc + row * A.acc_row + comp * A.acc_comp + (size_t)er * N;
    if (DW > 1 && tid < COLS) colsum[tid] = 0;
    if (DW > 1) __syncthreads();

    // the digits of all channels of the columns: a thread takes 16 channels of a column (4 KS groups of 16; CT KS is THREADS / 64 at most)
    const u32 col = tid & (COLS - 1), g = tid / COLS;
    if (g < 4 * KS) {
        const u64* src = A.in + row * A.in_row + comp * A.in_comp + (size_t)e * N + x0 + col;
        u64 v[16];
        if (16 * g < A.c_in) {
#pragma unroll
            for (u32 j = 0; j < 16; j++) v[j] = src[(16 * g + j < A.c_in ? 16 * g + j : A.c_in - 1) * A.in_ct];
        } else {
#pragma unroll
            for (u32 j = 0; j < 16; j++) v[j] = 0;
        }
        u64 total = 0;
        u32 w[8][4];
#pragma unroll
        for (u32 m = 0; m < 4; m++) {
            u64 s[4];
#pragma unroll
            for (u32 j = 0; j < 4; j++) {
                if (16 * g + 4 * m + j >= A.c_in) v[4 * m + j] = 0;
                if (DW > 1) total += v[4 * m + j];
                s[j] = (v[4 * m + j] + LM_BIAS) ^ LM_BIAS;
            }
            u32 lo[4], hi[4];
            lm_transpose((u32)s[0], (u32)s[1], (u32)s[2], (u32)s[3], lo);
            lm_transpose((u32)(s[0] >> 32), (u32)(s[1] >> 32), (u32)(s[2] >> 32), (u32)(s[3] >> 32), hi);
#pragma unroll
            for (u32 i = 0; i < 4; i++) w[i][m] = lo[i], w[4 + i][m] = hi[i];
        }
        uint4* dst = lds + (((col >> 4) * KS + (g >> 2)) * LM_DX) * 64 + 16 * (g & 3) + (col & 15);
#pragma unroll
        for (u32 dx = 0; dx < LM_DX; dx++) dst[dx * 64] = make_uint4(w[dx][0], w[dx][1], w[dx][2], w[dx][3]);
        if (DW > 1) atomicAdd(&colsum[col], total);  // whole numbers below 2^58: any order
    }
    __syncthreads();

    const u32 ct = wave % CT, x = x0 + 16 * ct + (lane & 15), quarter = lane >> 4;
    const ModConstF m = A.mcf[e];
    double cw[GROUPS + 1], part[GROUPS + 1];
#pragma unroll
    for (u32 i = 0; i < GROUPS; i++) cw[i] = K.c[i][e];
    cw[GROUPS] = K.c[3][e];
    if (DW > 1) {  // below 2^58: two halves joined modulo q
        const u64 s = colsum[16 * ct + (lane & 15)];
        const double hi = f64m_reduce((double)(u32)(s >> 32), m.q, m.qinv), lo = (double)(u32)s;
        const double two32 = f64m_reduce(4294967296.0, m.q, m.qinv);
        part[GROUPS] = f64m_reduce(f64m_mulmod_any(hi, two32, m.q, m.qinv) + lo, m.q, m.qinv);
    } else {
        part[GROUPS] = 0.0;
    }
    const uint4* lb = lds + (ct * KS) * LM_DX * 64 + lane;
    const u32 ot_last = min(ot_first + A.ot_per_wg, A.OT);
    for (u32 ot = ot_first + wave / CT; ot < ot_last; ot += OT_STEP) {
        u64 old[4];
        if (ADD) {  // requested ahead of the products
#pragma unroll
            for (u32 r = 0; r < 4; r++) {
                const u32 o = 16 * ot + 4 * quarter + r;
                old[r] = acc[(o < A.c_out ? o : A.c_out - 1) * A.acc_ct + x];
            }
        }
        v4i d[DIAGS];
#pragma unroll
        for (u32 s = 0; s < DIAGS; s++) d[s] = (v4i){0, 0, 0, 0};
        const uint4* wa = A.wa + gi * A.wa_group + (size_t)ot * KS * DW * 64 + lane;
        for (u32 ks = 0; ks < KS; ks++) {
            v4i a[DW];
#pragma unroll
            for (u32 dw = 0; dw < DW; dw++) {
                const uint4 t = wa[(ks * DW + dw) * 64];
                a[dw] = (v4i){(int)t.x, (int)t.y, (int)t.z, (int)t.w};
            }
#pragma unroll
            for (u32 dx = 0; dx < LM_DX; dx++) {
                const uint4 t = lb[(ks * LM_DX + dx) * 64];
                const v4i b = (v4i){(int)t.x, (int)t.y, (int)t.z, (int)t.w};
#pragma unroll
                for (u32 dw = 0; dw < DW; dw++) d[dx + dw] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[dw], b, d[dx + dw], 0, 0, 0);
            }
        }
#pragma unroll
        for (u32 r = 0; r < 4; r++) {
            const u32 o = 16 * ot + 4 * quarter + r;
#pragma unroll
            for (u32 i = 0; i < GROUPS; i++) {
                const u32 top = 4 * i + 3 < DIAGS ? 4 * i + 3 : DIAGS - 1;
                double t = (double)d[top][r];
                for (u32 s = top; s > 4 * i; s--) t = __builtin_fma(t, 256.0, (double)d[s - 1][r]);
                part[i] = t;
            }
            double v = DW > 1 ? f64m_dot_w<GROUPS + 1>(part, cw, m.q, m.qinv) : f64m_dot_w<GROUPS>(part, cw, m.q, m.qinv);
            if (o >= A.c_out) continue;
            if (bias && comp == 0)
                v = f64m_reduce(v + f64m_mulmod_any(f64m_from_u64(bias[(size_t)o * A.bias_limbs + e]), K.bias[e], m.q, m.qinv), m.q, m.qinv);
            if (ADD) v = f64m_reduce(v + f64m_from_u64(old[r]), m.q, m.qinv);
            acc[o * A.acc_ct + x] = f64m_canonical(v, m.q);
        }
    }
}

// The matrix-core kernel takes moduli below 2^50, whole column tiles, and sums that fill its tiles (64 channels x 16 outputs): a chain of the vector kernel holds 8
// channels and 8 outputs.  Vector / matrix kernel in us, four rows of 10 limbs at N = 2^14, 8-bit weights: 8 -> 24 channels 312 / 307, 12 -> 8 131 / 150, 16 -> 24
// 399 / 311, 12 -> 2 64 / 100, 40 -> 1 128 / 129, 40 -> 3 219 / 152.  Whole calls with up to eight channels and many outputs, 8- and 32-bit weights, vector (the same for
// both) / matrix, matrix: 2 -> 24 250 / 286, 315, 2 -> 192 1940 / 2017, 2168, 4 -> 24 269 / 290, 321, 4 -> 192 2105 / 2013, 2178, 8 -> 24 317 / 296, 335, 8 -> 192 2380 / 2019,
// 2181; one row of 24 limbs at 2^16: 4 -> 192 5310 / 4986, 5373, 8 -> 192 6200 / 4991, 5385.  So up to four channels the rule is the faster side or within 7 % of it;
// at eight channels and more than some 40 outputs the matrix kernel would be up to 24 % faster.
bool linear_mfma_applies(const ckks_ctx* c, u32 c_in, u32 c_out) {
    if (!c->small_q || c->N < 64) return false;
    return c_in <= 16 ? c_in > 8 && c_out > 8 : c_in > 32 || c_out > 2;
}

size_t linear_mfma_scratch_elems(u32 c_in, u32 c_out, u32 weight_bytes) {
    return (size_t)((c_out + 15) / 16) * ((c_in + 63) / 64) * weight_bytes * 64 * 2;
}

// Threads and 16-column tiles of a workgroup by the number of 64-channel steps: 28 KB of digits, or 42 and 56 KB, for four waves per SIMD
static u32 linear_threads(u32 KS) { return KS <= 2 ? 256 : 512; }
static u32 linear_col_tiles(u32 KS) { return KS == 1 ? 4 : 2; }

template <u32 DW>
static hipError_t launch_linear_dw(const LinearMfmaArgs& A, const LinearConsts& K, u32 rows, hipStream_t st) {
    const u32 CT = linear_col_tiles(A.KS), threads = linear_threads(A.KS);
    const dim3 grid(A.N / (16 * CT), 2 * A.limbs, rows);
    const size_t lds = (size_t)CT * A.KS * LM_DX * 64 * 16 + 16 * CT * 8;
#define LINEAR_MFMA(CT, T, ADD) hipLaunchKernelGGL((linear_mfma_kernel<DW, CT, T, ADD>), grid, dim3(T), lds, st, A, K)
    if (CT == 4 && A.add) LINEAR_MFMA(4, 256, true);
    else if (CT == 4) LINEAR_MFMA(4, 256, false);
    else if (threads == 256 && A.add) LINEAR_MFMA(2, 256, true);
    else if (threads == 256) LINEAR_MFMA(2, 256, false);
    else if (A.add) LINEAR_MFMA(2, 512, true);
    else LINEAR_MFMA(2, 512, false);
#undef LINEAR_MFMA
    return hipGetLastError();
}

hipError_t launch_linear_mfma(const ckks_ctx* c, const LinearSum& S, u64* scratch, bool prepared, hipStream_t st) {
    if (S.groups.n == 0 || S.groups.n > LINEAR_GROUPS || (u64)S.rows * S.c_out > 1024) return hipErrorInvalidValue;  // (the grid's third dimension)
    const u32 wb = S.weight_bytes;
    LinearConsts K = {};
    for (u32 i = S.limb0; i < S.limb0 + S.limbs; i++) {
        const u64 q = c->mod[i];
        auto centred = [&](unsigned __int128 v) {
            const u64 r = (u64)(v % q);
            return r > q / 2 ? -(double)(q - r) : (double)r;
        };
        unsigned __int128 k = S.mult.v[i] % q;
        u64 off = 0;  // what the digits leave out
        for (u32 b = 0; b + 1 < wb; b++) off = off * 256 + 128;
        K.c[3][i] = centred(k * (off % q));
        for (u32 g = 0; g < 3; g++) {
            K.c[g][i] = centred(k);
            k = k * (((u64)1 << 32) % q) % q;
        }
        K.bias[i] = centred(S.bias_mult.v[i]);
    }
    for (u32 c0 = 0; c0 < S.c_in; c0 += LM_CHUNK) {
        const u32 nc = S.c_in - c0 < LM_CHUNK ? S.c_in - c0 : LM_CHUNK;
        const char* wc = (const char*)S.w + c0 * S.w_in * wb;
        const u32 KS = (nc + 63) / 64, OT = (S.c_out + 15) / 16, prep = OT * KS * wb * 64;
        uint4* wa = (uint4*)(scratch + S.groups.n * linear_mfma_scratch_elems(c0, S.c_out, wb));
        if (!prepared) {
            const dim3 pg((prep + LM_THREADS - 1) / LM_THREADS, S.groups.n);
#define LINEAR_PREP(W) hipLaunchKernelGGL(linear_prep_kernel<W>, pg, dim3(LM_THREADS), 0, st, (const W*)wc, S.w_out, S.w_in, S.w_group, S.groups, wa, prep, S.c_out, nc, KS, OT)
            if (wb == 1) LINEAR_PREP(int8_t);
            else if (wb == 2) LINEAR_PREP(int16_t);
            else LINEAR_PREP(int32_t);
#undef LINEAR_PREP
        }
        // outputs of a workgroup: all, unless that leaves the chip short of workgroups
        const u32 ct = linear_col_tiles(KS), step = linear_threads(KS) / 64 / ct;
        const u64 wgs = (u64)(c->N / (16 * ct)) * 2 * S.limbs * S.rows;
        u32 n_split = wgs >= 1024 ? 1 : (u32)(1024 / wgs);
        u32 per = (OT + n_split - 1) / n_split;
        per = (per + step - 1) / step * step;
        n_split = (OT + per - 1) / per;
        const u32 add = c0 || S.add ? 1 : 0;
        const LinearMfmaArgs A = {S.in + c0 * S.in_ct, S.in_ct, S.in_comp, S.in_row, wa, prep, S.bias_group, c0 ? nullptr : S.bias, S.acc, S.acc_ct, S.acc_comp, S.acc_row,
                                  c->d_mcf, c->N, S.limb0, S.limbs, S.bias_limbs, nc, S.c_out, KS, OT, per, add, S.groups};
        ProfScope ps__(c, K_WEIGHTED_SUM, st, 16.0 * S.rows * c->N * S.limbs * (nc + (1.0 + add) * S.c_out), 2.0 * S.rows * c->N * S.limbs * nc * S.c_out);
        const u32 rows = S.rows * n_split;
        hipError_t err = wb == 1 ? launch_linear_dw<1>(A, K, rows, st) : (wb == 2 ? launch_linear_dw<2>(A, K, rows, st) : launch_linear_dw<4>(A, K, rows, st));
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}
