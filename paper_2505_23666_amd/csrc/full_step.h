// Attention of few rows over the 8-bit cache: the generation step, and calls of a few tokens (up to 32 rows, a row being one query of one
// query head of the group).
//
// Bound by HBM: every code is read once for all rows of the group (256 bytes a slot at d = 128 against 2 x 4 x 128 x 2 flops for four heads).
// 64 sequences of 2048 to 4096 pairs (32 query, 8 kv heads, d = 128): 82 us a step, 4.9 TB/s, the rate of a large copy; one sequence of
// 128 Ki pairs 55 us with the join.  Short caches are bound by a chain of dependent loads: 8 streams of 1500 pairs at d = 64 6 + 3 us.
// A stream's blocks are dealt to `nsplit` workgroups and within one to its wavefronts (four, or eight where one workgroup has all of a short cache); each wavefront keeps a running maximum, sum
// and output of its own over the blocks it reads, nothing is exchanged before its last block.
//
// One block (64 slots) of a wavefront:
//   S^T = K Q^T   16x16x32 bf16: keys (codes times scale) are exact in bf16, so are bf16 queries; fp32 queries enter as three bf16 parts (24 bits).  A lane's
//                 operand is eight consecutive bytes of its key row, straight from global memory: the order of the contraction
//                 index is free as long as the queries are laid out the same.
//   p = 2^(s - m + 14) times the values' scale in units of 2^x, rounded to fp16 (fp32 outputs: two fp16 parts): the operand of the second product.
//                 m (the maximum rounded up) and x are whole numbers of the row's own, see RowRef.  The shift keeps products of weight and scale
//                 down to 2^-28 of the row's largest among fp16's normal numbers; the sum takes p before the rounding.
//   O^T += V^T P^T  16x16x32 fp16: V's codes, exact in fp16; they pass through LDS for the transposing 8-bit read, 16-byte pieces XOR-swizzled
//                 by row so that the 32 rows of a read meet all banks alike.  The C layout of the first product is the B layout of this one.
#pragma once
#include "full_cache.h"

namespace lola {
namespace full {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i2 __attribute__((ext_vector_type(2)));

constexpr float P_SHIFT = 14.f;    // probabilities are held times 2^14
constexpr int STEP_BLOCKS = 64;    // most blocks that one wavefront of the step kernel reads

// eight codes times their block's scale -> eight bf16 (exact: the keys themselves)
__device__ __forceinline__ bf8 codes_to_bf16(uint32_t a, uint32_t b, float scale) {
    union { bf8 v; bf2 p[4]; } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false); u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false); u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
    return u.v;
}
// eight codes -> eight fp16 (exact)
__device__ __forceinline__ h8 codes_to_f16(uint32_t a, uint32_t b) {
    union { h8 v; h2 p[4]; } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false); u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false); u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true);
    return u.v;
}
__device__ __forceinline__ i2 lds_read_tr8(const uint8_t *p) {
    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i2 *)(p));
}
// x as three bf16 parts whose sum it is: 8 of its 24 bits each, cut off rather than rounded, so that no part overflows.  What is not finite
// becomes NaN (see spoil_query).
__device__ __forceinline__ void split_bf16(const float *x, bf8 *part) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        float r = x[e];
#pragma unroll
        for (int p = 0; p < 3; p++) {
            const uint32_t u = finite(r) ? __float_as_uint(r) & 0xFFFF0000u : 0x7FC00000u;
            part[p][e] = __builtin_bit_cast(__bf16, (uint16_t)(u >> 16));
            r = finite(r) ? r - __uint_as_float(u) : 0.f;
        }
    }
}

// Two fp32 numbers as fp16 operand parts: rounded, and (where PP = 2) what the rounding left, rounded.  The difference is one mixed-precision
// fused operation per number; minus_one holds -1 where the compiler cannot see it (it would make a conversion and a subtraction).
template <int PP>
__device__ __forceinline__ void to_f16_parts(float x, float y, float minus_one, h2 *part) {
    part[0] = (h2){(_Float16)x, (_Float16)y};
    if (PP == 2) {      // (one packed conversion whose halves are read again, not two more)
        uint32_t u = __builtin_bit_cast(uint32_t, part[0]);
        asm("" : "+v"(u));
        part[0] = __builtin_bit_cast(h2, u);
    }
    if (PP == 2) part[PP - 1] = (h2){(_Float16)__builtin_fmaf((float)part[0][0], minus_one, x), (_Float16)__builtin_fmaf((float)part[0][1], minus_one, y)};
}
__device__ __forceinline__ float opaque_minus_one() {
    float x = -1.f;
    asm volatile("" : "+v"(x));
    return x;
}

// A row's references, whole numbers.  m: its sum of weights is held times 2^-m.  x: its output is held times 2^(-m - x), x being such that of the
// row's products of a weight and a block's scale (2^(s - m) 2^ev) the largest so far is about 2^x.  So the scales enter by the weights, row
// by row, and values of a block that the row does not see, or hardly, take no bits from the others.
struct RowRef {
    float m = -3.4028234663852886e38f, x = -200.f;     // (nothing seen: finite, so that differences are)
    __device__ __forceinline__ bool seen() const { return m != -3.4028234663852886e38f; }
    // Moves on to a block whose largest logit is mb (-inf: none) and whose values have the exponent ev; by what the sum and the output then shrink.
    __device__ __forceinline__ void move(float mb, float ev, float &fl, float &fo) {
        const float top = ceilf(mb), mn = fmaxf(m, top), xn = fmaxf(x + (m - mn), (top - mn) + ev);
        fl = __builtin_amdgcn_exp2f(m - mn);
        fo = __builtin_amdgcn_exp2f((m - mn) + (x - xn));
        m = mn; x = xn;
    }
    // The block's weights are to be held times 2^(shift - m - drop()).  From 2^64 below the row's largest products on they are nothing in fp16 anyway.
    __device__ __forceinline__ float drop(float ev) const { return fminf(x - ev, 64.f); }
    // m + drop - shift is no whole number any more: the logits are to be taken relative to m first
    __device__ __forceinline__ bool far() const { return fabsf(m) >= 4194304.f && seen(); }
};

struct StepArgs {
    Args a;
    int nsplit;
    float *part_o;     // [S][nsplit][R][d] outputs of the shares, normalised
    float *part_ml;    // [S][nsplit][R][2] RowRef::m and sum; sum 0: an empty share
    float *logit;      // [S][R][cap] logits (powers of two) where weights are gathered, else NULL
    int32_t *counts;   // [S] with a token appended by the same launch and weights gathered: the slots in use after it
    int append;        // the join moves the counters on (a.k, a.v hold the token)
};

// swizzle of the 16-byte pieces of an LDS row of DH bytes: rows whose addresses differ by a multiple of 256 bytes meet other banks
template <int DH>
__device__ __forceinline__ int vswz(int row) { return (row / (256 / DH)) & (DH / 16 - 1); }

__device__ __forceinline__ float half_max(float v) { const Two t = swap_halves(v); return fmaxf(t.a, t.b); }
__device__ __forceinline__ float half_sum(float v) { const Two t = swap_halves(v); return t.a + t.b; }
__device__ __forceinline__ float quad_max(float v) { const Two t = swap_rows16(v); return half_max(fmaxf(t.a, t.b)); }
__device__ __forceinline__ float quad_sum(float v) { const Two t = swap_rows16(v); return half_sum(t.a + t.b); }

// eight query elements as matrix operand parts
__device__ __forceinline__ void load_query(const bf16_t *p, bf8 *part) { part[0] = *reinterpret_cast<const bf8 *>(p); }
__device__ __forceinline__ void load_query(const float *p, bf8 *part) {
    float x[8];
    load8(p, x);
    split_bf16(x, part);
}
// A query with an element that is not finite has the output NaN wherever it sees a pair: an infinite element makes each of its logits infinite
// or NaN, and a softmax of infinities is NaN, also where all of them are negative and would pass for weights of zero.  So `sum`, the row's
// product with zeros (NaN for such a query, else 0), makes its first operand NaN, and with it every logit.  (A test of the elements would move
// all operands through vector registers: many rows at d = 256 took 14 % longer.)
__device__ __forceinline__ void spoil_query(bf8 *q, float sum) {
    if (__any(sum != 0.f) && sum != 0.f) q[0] = __builtin_bit_cast(bf8, make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u));
}
template <int QP>
__device__ __forceinline__ void zero_query(bf8 *part) {
#pragma unroll
    for (int p = 0; p < QP; p++) part[p] = __builtin_bit_cast(bf8, make_uint4(0, 0, 0, 0));
}

// Puts the stream's new token into slot c0, by one wavefront: lanes below DH / 8 take eight elements of the key each, as many behind them the value.
// The same codes, scales and rules as append_kernel.
template <int DH, typename TI>
__device__ __forceinline__ void append_token(const Args &a, int si, int b, int h, int c0, int lane) {
    constexpr int NL = DH / 8;
    const int J = c0 / BLK, off = c0 % BLK, part = lane % NL;
    const bool isk = lane < NL, mine = lane < 2 * NL;
    const int64_t told = a.mem.n_tokens[si];
    float *kss = a.mem.ks + (size_t)si * a.nblk + J, *vss = a.mem.vs + (size_t)si * a.nblk + J;
    const float oks = *kss, ovs = *vss;      // (of a block that held nothing: not looked at)
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = 0.f;
    if (mine) load8((const TI *)(isk ? a.k : a.v) + b * a.k_sb + h * a.k_sh + part * 8, x);
    float top = 0.f;
    bool nf = false;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        if (!finite(x[e])) { nf = true; x[e] = 0.f; }
        top = fmaxf(top, fabsf(x[e]));
    }
    const bool bad = __any(nf);
    const float ak = bad ? 0.f : max_of_wave(isk ? top : 0.f), av = max_of_wave(isk ? 0.f : top);
    int ek = fit_exponent(ak), ev = fit_exponent(av);
    uint8_t *kb = a.mem.k + ((size_t)si * a.cap + (size_t)J * BLK) * DH, *vb = a.mem.v + ((size_t)si * a.cap + (size_t)J * BLK) * DH;
    if (off > 0) {
        const int ok = exponent_of(oks), ov = exponent_of(ovs);
        ek = max(ek, ok); ev = max(ev, ov);
        if (ek > ok || ev > ov) {
            const float fk = pow2(max(ok - ek, -40)), fv = pow2(max(ov - ev, -40));
            for (int e = lane; e < off * NL; e += 64) {
                if (ek > ok) { uint2 u = reinterpret_cast<uint2 *>(kb)[e]; u.x = rescale_codes(u.x, fk); u.y = rescale_codes(u.y, fk); reinterpret_cast<uint2 *>(kb)[e] = u; }
                if (ev > ov) { uint2 u = reinterpret_cast<uint2 *>(vb)[e]; u.x = rescale_codes(u.x, fv); u.y = rescale_codes(u.y, fv); reinterpret_cast<uint2 *>(vb)[e] = u; }
            }
        }
    }
    if (mine) {
        const float f = pow2(isk ? -ek : -ev);
        uint2 u;
        u.x = to_codes(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
        u.y = to_codes(x[4] * f, x[5] * f, x[6] * f, x[7] * f);
        if (isk && bad) u.x = u.y = 0x7F7F7F7Fu;
        *reinterpret_cast<uint2 *>((isk ? kb : vb) + off * DH + part * 8) = u;
    }
    if (lane == 0) {
        *kss = pow2(ek); *vss = pow2(ev);
        a.mem.idx[(size_t)si * a.cap + c0] = (int32_t)told;
        if (a.mem.weight) a.mem.weight[(size_t)si * a.cap + c0] = 0.f;
    }
    __threadfence_block();      // this wavefront reads the block back
}

template <int DH, int CT, int NW, typename TI, typename TO, bool MASK, bool APPEND>
__global__ __launch_bounds__(64 * NW) void step_kernel(StepArgs sa) {
    constexpr int QP = sizeof(TI) == 4 ? 3 : 1, PP = sizeof(TO) == 4 ? 2 : 1;
    constexpr int NK = DH / 32;                     // contraction steps of the first product
    constexpr int ND = DH / 16;                     // tiles of 16 output columns
    constexpr int KB = DH / 4;                      // bytes of a key row per lane: quad q holds pieces c * 64 + q * 16 (DH = 32: q * 8)
    constexpr int VI = DH / 16;                     // 16-byte loads per lane of a block's values
    constexpr int PR = DH / 16;                     // pieces per row
    __shared__ __attribute__((aligned(16))) uint8_t stage[NW][BLK * DH];
    __shared__ float ml_l[NW][3][16 * CT];
    const Args &a = sa.a;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n16 = lane & 15, quad = lane >> 4;
    const int si = blockIdx.x, split = blockIdx.y, b = si / a.Hkv, h = si - b * a.Hkv;
    const int R = a.T * a.g, n = new_tokens(a, b), c0 = n ? held(a, si) : 0, count = APPEND ? min(c0 + 1, a.cap) : c0;
    const int nb = (count + BLK - 1) / BLK;
    const int J0 = (int)((int64_t)nb * split / sa.nsplit), J1 = (int)((int64_t)nb * (split + 1) / sa.nsplit);
    // a step's own token goes into the stream's last block, by the wavefront that reads it (nobody else does)
    if (APPEND && count > c0 && J1 == nb && J1 > J0 && (nb - 1 - J0) % NW == w) append_token<DH, TI>(a, si, b, h, c0, lane);
    const uint8_t *kc = a.mem.k + (size_t)si * a.cap * DH, *vc = a.mem.v + (size_t)si * a.cap * DH;
    const float *ks = a.mem.ks + (size_t)si * a.nblk, *vs = a.mem.vs + (size_t)si * a.nblk;
    const int32_t *idx = a.mem.idx + (size_t)si * a.cap;
    const int64_t pos0 = MASK ? a.mem.n_tokens[si] - n : 0;

    uint32_t kr[4][KB / 4], vr[VI * 4];
    float ksT = 0.f, vsT = 0.f;       // scales of this wavefront's blocks, 64 at most (STEP_BLOCKS), one per lane (a scalar load would make each LDS wait longer)
    auto scales = [&](int J) {
        const int x = min(J + NW * lane, a.nblk - 1);
        ksT = ks[x]; vsT = vs[x];
    };
    int4 id[4];
    auto load = [&](int J) {
        const uint8_t *kp = kc + (size_t)J * BLK * DH, *vp = vc + (size_t)J * BLK * DH;
#pragma unroll
        for (int t = 0; t < 4; t++) {
            const uint8_t *row = kp + (t * 16 + n16) * DH;
            if constexpr (DH == 32) {
                const uint2 u = *reinterpret_cast<const uint2 *>(row + quad * 8);
                kr[t][0] = u.x; kr[t][1] = u.y;
            } else {
#pragma unroll
                for (int c = 0; c < DH / 64; c++) {
                    const uint4 u = *reinterpret_cast<const uint4 *>(row + c * 64 + quad * 16);
                    kr[t][4 * c] = u.x; kr[t][4 * c + 1] = u.y; kr[t][4 * c + 2] = u.z; kr[t][4 * c + 3] = u.w;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < VI; i++) {
            const uint4 u = *reinterpret_cast<const uint4 *>(vp + i * 1024 + lane * 16);
            vr[4 * i] = u.x; vr[4 * i + 1] = u.y; vr[4 * i + 2] = u.z; vr[4 * i + 3] = u.w;
        }
        if (MASK)
#pragma unroll
            for (int t = 0; t < 4; t++) id[t] = *reinterpret_cast<const int4 *>(idx + (size_t)J * BLK + t * 16 + quad * 4);
    };
    if (J0 + w < J1) { scales(J0 + w); load(J0 + w); }

    // queries of row 16 ct + n16 in the keys' order of columns
    bf8 qf[CT][NK][QP];
    int64_t pos[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
        const int r = ct * 16 + n16, t = r / a.g, hq = h * a.g + (r - t * a.g);
        pos[ct] = pos0 + t;
        const TI *qp = (const TI *)a.q + b * a.q_sb + hq * a.q_sh + t * a.q_st;
#pragma unroll
        for (int s = 0; s < NK; s++) {
            if (t < n) load_query(qp + (DH == 32 ? quad * 8 : (s / 2) * 64 + quad * 16 + (s & 1) * 8), qf[ct][s]);
            else zero_query<QP>(qf[ct][s]);
        }
        if constexpr (QP == 1) {
            f4 sum = {0.f, 0.f, 0.f, 0.f};
            bf8 zero;
            zero_query<1>(&zero);
#pragma unroll
            for (int s = 0; s < NK; s++) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(zero, qf[ct][s][0], sum, 0, 0, 0);
            spoil_query(qf[ct][0], sum[0]);
        }
    }
    f4 o[CT][ND];
    RowRef ref[CT];
    float l[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
        l[ct] = 0.f;
#pragma unroll
        for (int c = 0; c < ND; c++) o[ct][c] = (f4){0.f, 0.f, 0.f, 0.f};
    }
    uint8_t *st = stage[w];
    const float minus_one = opaque_minus_one();
    for (int J = J0 + w, it = 0; J < J1; J += NW, it++) {
        const float ksJ = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ksT), it)), vsJ = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsT), it));
        const int live = count - J * BLK;          // slots of this block that hold pairs (64 and more: all)
        const float c = a.scale2, ev = (float)exponent_of(vsJ);
        // values to LDS; slots without a pair hold zeros there
#pragma unroll
        for (int i = 0; i < VI; i++) {
            const int row = i * (64 / PR) + lane / PR, piece = lane % PR;
            uint4 u = make_uint4(vr[4 * i], vr[4 * i + 1], vr[4 * i + 2], vr[4 * i + 3]);
            if (row >= live) u = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4 *>(st + row * DH + ((piece ^ vswz<DH>(row)) * 16)) = u;
        }
        f4 s[CT][4];
#pragma unroll
        for (int t = 0; t < 4; t++) {
#pragma unroll
            for (int ct = 0; ct < CT; ct++) s[ct][t] = (f4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NK; k++) {
                const bf8 kf = codes_to_bf16(kr[t][2 * k], kr[t][2 * k + 1], ksJ);
#pragma unroll
                for (int ct = 0; ct < CT; ct++)
#pragma unroll
                    for (int p = QP - 1; p >= 0; p--) s[ct][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[ct][k][p], s[ct][t], 0, 0, 0);
            }
        }
        const int4 idJ[4] = {id[0], id[1], id[2], id[3]};
        if (J + NW < J1) load(J + NW);
        h8 pf[CT][2][PP];
#pragma unroll
        for (int ct = 0; ct < CT; ct++) {
            float mb = -INFINITY;
#pragma unroll
            for (int t = 0; t < 4; t++) {
                const int ids[4] = {idJ[t].x, idJ[t].y, idJ[t].z, idJ[t].w};
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    float v = s[ct][t][e] * c;
                    if (t * 16 + quad * 4 + e >= live || (MASK && (int64_t)ids[e] > pos[ct])) v = -INFINITY;
                    s[ct][t][e] = v;
                    mb = fmaxf(mb, v);
                }
            }
            if (sa.logit && ct * 16 + n16 < R) {
                float *lp = sa.logit + ((size_t)si * R + ct * 16 + n16) * a.cap + (size_t)J * BLK + quad * 4;
#pragma unroll
                for (int t = 0; t < 4; t++) *reinterpret_cast<f4 *>(lp + t * 16) = s[ct][t];
            }
            float fl, fo;
            ref[ct].move(quad_max(mb), ev, fl, fo);
            const float t = ref[ct].drop(ev);
            float off = ref[ct].m + (t - P_SHIFT);
            if (__builtin_expect(__any(ref[ct].far()), 0)) {
                off = t - P_SHIFT;
#pragma unroll
                for (int k = 0; k < 4; k++)
#pragma unroll
                    for (int e = 0; e < 4; e++) s[ct][k][e] -= ref[ct].m;
            }
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 4; k++)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float x = __builtin_amdgcn_exp2f(s[ct][k][e] - off), y = __builtin_amdgcn_exp2f(s[ct][k][e + 1] - off);
                    sum += x + y;
                    h2 part[PP];
                    to_f16_parts<PP>(x, y, minus_one, part);
#pragma unroll
                    for (int p = 0; p < PP; p++) { pf[ct][k / 2][p][(k & 1) * 4 + e] = part[p][0]; pf[ct][k / 2][p][(k & 1) * 4 + e + 1] = part[p][1]; }
                }
            l[ct] = l[ct] * fl + quad_sum(sum) * __builtin_amdgcn_exp2f(t);
#pragma unroll
            for (int d = 0; d < ND; d++) o[ct][d] *= fo;
        }
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int i8 = n16 >> 1, row = k * 32 + (i8 & 4) * 4 + quad * 4 + (i8 & 3);
#pragma unroll
            for (int d = 0; d < ND; d++) {
                const i2 u = lds_read_tr8(st + row * DH + ((d ^ vswz<DH>(row)) * 16) + (n16 & 1) * 8);
                const h8 vf = codes_to_f16((uint32_t)u[0], (uint32_t)u[1]);
#pragma unroll
                for (int ct = 0; ct < CT; ct++)
#pragma unroll
                    for (int p = PP - 1; p >= 0; p--) o[ct][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[ct][k][p], o[ct][d], 0, 0, 0);
            }
        }
    }

    // the wavefronts' shares: O^T [column][row] in turn through the staging memory, weighted by their references
    if (quad == 0)
#pragma unroll
        for (int ct = 0; ct < CT; ct++) { ml_l[w][0][ct * 16 + n16] = ref[ct].m; ml_l[w][1][ct * 16 + n16] = l[ct]; ml_l[w][2][ct * 16 + n16] = ref[ct].x; }
    __syncthreads();
    if (APPEND && tid == 0) {
        if (!sa.part_ml) { a.mem.count[si] = count; a.mem.n_tokens[si] += 1; }       // (the stream's only workgroup)
        else if (sa.counts && split == 0) sa.counts[si] = count;
    }
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
        float *ol = reinterpret_cast<float *>(stage[0]);     // [wavefront][column][16 rows]
        if (ct) __syncthreads();
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
            for (int e = 0; e < 4; e++) ol[(w * DH + d * 16 + quad * 4 + e) * 16 + n16] = o[ct][d][e];
        __syncthreads();
        for (int e = tid; e < 16 * DH; e += 64 * NW) {
            const int r16 = e / DH, col = e - r16 * DH, r = ct * 16 + r16;
            if (r >= R) continue;
            float M = -INFINITY;
#pragma unroll
            for (int i = 0; i < NW; i++) M = fmaxf(M, ml_l[i][0][r]);
            float L = 0.f, y = 0.f;
#pragma unroll
            for (int i = 0; i < NW; i++) L += ml_l[i][1][r] * __builtin_amdgcn_exp2f(ml_l[i][0][r] - M);
            const int t = r / a.g, hq = h * a.g + (r - t * a.g);
            if (t >= n) L = 0.f;     // padding
            if (L != 0.f) {
                const float iL = 1.f / L;
#pragma unroll
                for (int i = 0; i < NW; i++) y += ol[(i * DH + col) * 16 + r16] * iL * __builtin_amdgcn_exp2f((ml_l[i][0][r] - M) + ml_l[i][2][r]);
            }
            if (sa.nsplit == 1) stf((TO *)a.out + b * a.q_sb + hq * a.q_sh + t * a.q_st, col, y);
            else sa.part_o[(((size_t)si * sa.nsplit + split) * R + r) * DH + col] = y;
            if (sa.part_ml && col == 0) {
                float *p = sa.part_ml + (((size_t)si * sa.nsplit + split) * R + r) * 2;
                p[0] = M; p[1] = L;
            }
        }
    }
}

// Joins the shares: workgroup y < jo of a stream one row of outputs (DH / 4 threads per share, the shares dealt to the groups of threads); the
// others, where weights are gathered, add sum over rows of 2^(logit - M) / L to the weights of 1024 slots at a time.
template <int DH, typename TO>
__global__ __launch_bounds__(256) void step_join_kernel(StepArgs sa, int jo) {
    const Args &a = sa.a;
    constexpr float SCALE = 1.f / 16384.f;           // sums hold p times 2^14
    constexpr int TPS = DH / 4, NG = 256 / TPS;
    __shared__ float M_l[32], L_l[32];
    __shared__ __attribute__((aligned(16))) float acc_l[NG][DH + 4];
    const int tid = threadIdx.x, si = blockIdx.x, b = si / a.Hkv, h = si - b * a.Hkv, R = a.T * a.g, ns = sa.nsplit;
    const float2 *ml = reinterpret_cast<const float2 *>(sa.part_ml) + (size_t)si * ns * R;
    const int y = blockIdx.y;
    if (sa.append && y == 0 && tid == 0) {    // (nobody else of this launch looks at them)
        a.mem.count[si] = min(held(a, si) + 1, a.cap);
        a.mem.n_tokens[si] += 1;
    }
    if (y < jo) {
        const int gr = tid / TPS, col = (tid % TPS) * 4;
        const int t = y / a.g, hq = h * a.g + (y - t * a.g);
        const float *po = sa.part_o + ((size_t)si * ns * R + y) * DH + col;
        // every group of threads a running maximum and sum over its shares (an empty share: maximum -inf, sum 0, outputs 0)
        float M = -INFINITY, L = 0.f;
        f4 acc = (f4){0.f, 0.f, 0.f, 0.f};
        for (int s0 = gr; s0 < ns; s0 += 4 * NG) {
            float2 p[4];
            f4 o[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int s = s0 + i * NG;
                p[i] = s < ns ? ml[s * R + y] : make_float2(-INFINITY, 0.f);
                o[i] = s < ns ? *reinterpret_cast<const f4 *>(po + (size_t)s * R * DH) : (f4){0.f, 0.f, 0.f, 0.f};
            }
            const float mn = fmaxf(fmaxf(fmaxf(p[0].x, p[1].x), fmaxf(p[2].x, p[3].x)), M), mu = mn == -INFINITY ? 0.f : mn;
            const float f = __builtin_amdgcn_exp2f(M - mu);
            M = mn; L *= f; acc *= f;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float x = p[i].y * __builtin_amdgcn_exp2f(p[i].x - mu);
                L += x; acc += o[i] * x;
            }
        }
        *reinterpret_cast<f4 *>(&acc_l[gr][col]) = acc;
        if (tid % TPS == 0) { M_l[gr] = M; L_l[gr] = L; }
        __syncthreads();
        if (tid < DH) {
            float Mx = -INFINITY, Ls = 0.f, v = 0.f;
            for (int i = 0; i < NG; i++) Mx = fmaxf(Mx, M_l[i]);
            const float mu = Mx == -INFINITY ? 0.f : Mx;
            for (int i = 0; i < NG; i++) {
                const float f = __builtin_amdgcn_exp2f(M_l[i] - mu);
                Ls += L_l[i] * f; v += acc_l[i][tid] * f;
            }
            stf((TO *)a.out + b * a.q_sb + hq * a.q_sh + t * a.q_st, tid, Ls == 0.f ? 0.f : v / Ls);
        }
        return;
    }
    const int n = new_tokens(a, b), count = sa.append ? sa.counts[si] : n ? held(a, si) : 0;
    if ((y - jo) * 1024 >= count) return;
    // eight lanes per row look at the shares
    const int r8 = tid >> 3, j = tid & 7;
    if (r8 < R) {
        float M = -INFINITY, L = 0.f;
        for (int s = j; s < ns; s += 8) M = fmaxf(M, ml[s * R + r8].x);
        M = fmaxf(M, __shfl_xor(M, 1)); M = fmaxf(M, __shfl_xor(M, 2)); M = fmaxf(M, __shfl_xor(M, 4));
        const float mu = M == -INFINITY ? 0.f : M;
        for (int s = j; s < ns; s += 8) { const float2 p = ml[s * R + r8]; L += p.y * __builtin_amdgcn_exp2f(p.x - mu); }
        L += __shfl_xor(L, 1); L += __shfl_xor(L, 2); L += __shfl_xor(L, 4);
        if (j == 0) { M_l[r8] = mu; L_l[r8] = L > 0.f && finite(L) ? 1.f / (L * SCALE) : 0.f; }
    }
    __syncthreads();
    // four slots per thread (the logits of slots without a pair are -inf or were never written: masked)
    for (int slot = ((y - jo) * 256 + tid) * 4; slot < count; slot += (gridDim.y - jo) * 1024) {
        f4 acc = (f4){0.f, 0.f, 0.f, 0.f};
        for (int r = 0; r < n * a.g; r++) {
            const float f = L_l[r], m = M_l[r];
            const f4 s = *reinterpret_cast<const f4 *>(sa.logit + ((size_t)si * R + r) * a.cap + slot);
            if (f != 0.f)
#pragma unroll
                for (int e = 0; e < 4; e++) acc[e] += __builtin_amdgcn_exp2f(s[e] - m) * f;
        }
        float *wp = a.mem.weight + (size_t)si * a.cap + slot;
        const f4 was = *reinterpret_cast<const f4 *>(wp);
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (slot + e < count) wp[e] = was[e] + acc[e];
    }
}

}  // namespace full
}  // namespace lola
