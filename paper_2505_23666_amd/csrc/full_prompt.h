// Attention of many rows over the 8-bit cache: prompts, further turns, pieces of long prompts.  Row r of a stream is query
// head r % g of token r / g: the heads of a group lie beside each other, so that a workgroup's rows cover few tokens and read one cache.
//
// One workgroup takes 32 NW rows of a stream, wavefront w the 32 from 32 w on, and goes over the blocks of 64 slots that any of them may
// see; where there are few rows, the blocks are dealt to several workgroups and their shares joined.  A block's codes are loaded
// into registers while the one before it is worked on, converted once for all rows and put into the other of two LDS buffers: keys as bf16 with their scale, values'
// codes as fp16 (both exact); the values' scales enter by the weights (RowRef).  Products are 32x32x16 and transposed: S^T = K Q^T has a query per
// lane pair, so the running maximum and sum live there, and its C layout is the B layout of O^T += V^T P^T, whose V^T comes from the
// transposing 16-bit LDS read.  Which blocks can be passed over and which need a comparison per element follows from the least and largest token
// index of each block (of long caches taken beforehand by a kernel of its own): slots need not be in the order of tokens (evictions fill holes).
//
// Bound by the sum of its matrix and vector instructions, of two wavefronts per SIMD, by LDS, as busy as the matrix cores (every wavefront reads all of a block for its
// 32 rows; a quarter of the active cycles are bank conflicts), and by power: four prompts of 4096 tokens (32 query, 8 kv heads, d = 128, bf16) 0.59 ms in a long row of
// passes, 930 TFLOP/s, 0.68 to 0.8 ms in the first twenty, where a large library product reaches 1330; the same with all elements equal is a fifth
// faster.  A block of a wavefront is 32 products of 32 cycles, 32 exponentials, about 200 other vector instructions and 32 KB from LDS.  At
// d = 64 the exponentials weigh as much as the products (two prompts of 2000 tokens, fp32 outputs: 72 us).
//
// The row's references (RowRef) are only moved when a logit exceeds them by more than `raise`: weights (times scales) then reach 2^raise, held times
// 2^shift in fp16 (Slack).
#pragma once
#include <type_traits>
#include "full_step.h"

namespace lola {
namespace full {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));

// The 15 powers of two that fp16 has above 1, dealt to raise and shift.  The fewer to raise, the more often the references move; the more to shift, the
// more bits small weights keep, which are all of an output where one pair takes nearly all the weight and has hardly a value (2^-17 beside such a
// pair, fp32 outputs: off by 7e-6 to 2e-5 at raise 8, 1e-6 to 2.5e-6 at 4, 5e-7 to 8e-7 at 2; 2^-26, bf16 outputs: 1e-2 at 8, the output's own rounding at 4).
// Four prompts of 4096 tokens (d = 128, bf16) 629, 628, 633 and 640 us at raise 8, 4, 2, 1; two of 2000 with weights (d = 64, fp32 outputs) 129, 129, 131, 132.
template <typename TO> struct Slack { static constexpr float raise = sizeof(TO) == 4 ? 2.f : 4.f, shift = 15.f - raise; };

struct PromptArgs {
    Args a;
    int nsplit, ntiles;
    int2 *span;        // [S][nblk] least and largest token index of each block; NULL: up to 16 blocks, each workgroup looks at the indices
    float *part_o;     // [S][nsplit][R][d] outputs of the shares, normalised
    float *part_ml;    // [S][nsplit][R][2] RowRef::m and sum
    float2 *stat;      // [S][R] weight_stat(), where weights are gathered
};

// least and largest token index of each block in use; slots without a pair count as later than all queries
__global__ __launch_bounds__(256) void span_kernel(PromptArgs pa) {
    const Args &a = pa.a;
    const int si = blockIdx.y, lane = threadIdx.x & 63, count = held(a, si);
    for (int J = blockIdx.x * 4 + (threadIdx.x >> 6); J * BLK < count; J += gridDim.x * 4) {
        const int v = J * BLK + lane < count ? a.mem.idx[(size_t)si * a.cap + (size_t)J * BLK + lane] : 0x7FFFFFFF;
        int lo = v, hi = v;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { lo = min(lo, __shfl_xor(lo, o)); hi = max(hi, __shfl_xor(hi, o)); }
        if (lane == 0) pa.span[(size_t)si * a.nblk + J] = make_int2(lo, hi);
    }
}

__device__ __forceinline__ h4 lds_read_tr16(const _Float16 *p) {
    typedef __fp16 v4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) v4 *)(p)));
}

// swizzles of the 16-byte pieces of the rows in LDS (DH 2-byte numbers): 32 rows, one piece each (keys), and 4 rows x 64 bytes (values)
template <int DH> __device__ __forceinline__ int kswz2(int row) { return DH >= 128 ? row & 15 : DH == 64 ? (row >> 1) & 7 : (row >> 2) & 3; }
template <int DH> __device__ __forceinline__ int vswz2(int row) { return DH >= 128 ? (row & 3) << 2 : DH == 64 ? (row & 2) << 1 : 0; }

// What the weights of a row are made of, p = 2^(logit - .x) .y: .x the next whole number above the sum's logarithm (no logit exceeds it), .y, from 1
// to 2, what is left of 1 / sum.  (As one number, m + log2 of the sum, the logarithm's error would be the same for all of the row's weights and lean to one
// side over the rows: 3.2e-7 of the weights' 2-norm, so 0.5e-7.)  m, l: reference and sum of the row, the latter held times 2^shift.  A row
// without pairs, or whose sum is not finite, adds no weight.
__device__ __forceinline__ float2 weight_stat(float m, float l, float shift) {
    const float n = m + ((float)exponent_of(l) + 1.f - shift);
    return l > 0.f && finite(l) ? make_float2(n, __builtin_amdgcn_exp2f((n - m) + shift) / l) : make_float2(INFINITY, 0.f);
}

// four values to consecutive elements of an output row
__device__ __forceinline__ void store4(float *p, f4 v) { *reinterpret_cast<f4 *>(p) = v; }
__device__ __forceinline__ void store4(bf16_t *p, f4 v) {
    typedef __bf16 b4 __attribute__((ext_vector_type(4)));
    b4 u;
#pragma unroll
    for (int e = 0; e < 4; e++) u[e] = (__bf16)v[e];
    *reinterpret_cast<b4 *>(p) = u;
}

template <int DH, int NW, typename TI, typename TO>
__global__ __launch_bounds__(64 * NW, (DH == 256 || sizeof(TI) == 4) ? 1 : 2) void prompt_kernel(PromptArgs pa) {
    constexpr int QP = sizeof(TI) == 4 ? 3 : 1, PP = sizeof(TO) == 4 ? 2 : 1;
    constexpr float RAISE = Slack<TO>::raise, SHIFT = Slack<TO>::shift;
    constexpr int NK = DH / 16, ND = DH / 32;           // contraction steps of S, tiles of 32 output columns
    constexpr int NTHR = 64 * NW, TPR = DH / 16;        // threads per row of codes (16 each)
    constexpr int NL = BLK * TPR / NTHR < 1 ? 1 : BLK * TPR / NTHR;   // 16-byte loads per thread
    constexpr bool ALL = BLK * TPR >= NTHR;             // every thread loads
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // two buffers of keys [64][DH] bf16, values [64][DH] fp16, indices [64]
    constexpr int HALF = BLK * DH * 2, BUF = 2 * HALF + BLK * 4;      // (and the pairs' token indices)
    const Args &a = pa.a;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
    const int S = a.B * a.Hkv;
    const int si = blockIdx.x % S, rest = blockIdx.x / S, split = rest % pa.nsplit, tile = pa.ntiles - 1 - rest / pa.nsplit;   // (long rows first)
    const int b = si / a.Hkv, h = si - b * a.Hkv, R = a.T * a.g, n = new_tokens(a, b);
    const int r0 = tile * 32 * NW, r = r0 + w * 32 + l32;
    const int count = r0 < n * a.g ? held(a, si) : 0;
    const int64_t pos0 = a.mem.n_tokens[si] - n;
    const int t = r / a.g, hq = h * a.g + (r - t * a.g);
    const int pos = (int)(pos0 + t);
    const int64_t wg_last = pos0 + min((r0 + 32 * NW - 1) / a.g, n - 1);        // the workgroup's latest query
    const int64_t w_first = pos0 + (r0 + w * 32) / a.g;                        // the wavefront's earliest
    const uint8_t *kc = a.mem.k + (size_t)si * a.cap * DH, *vc = a.mem.v + (size_t)si * a.cap * DH;
    const float *ks = a.mem.ks + (size_t)si * a.nblk, *vs = a.mem.vs + (size_t)si * a.nblk;
    const int32_t *idx = a.mem.idx + (size_t)si * a.cap;
    const int2 *span = pa.span ? pa.span + (size_t)si * a.nblk : nullptr;
    const int nb = (count + BLK - 1) / BLK;
    const int J0 = (int)((int64_t)nb * split / pa.nsplit), J1 = (int)((int64_t)nb * (split + 1) / pa.nsplit);
    // What is known of 64 blocks from `base` on, one per lane, and which of them any query of the workgroup sees.  (Read block by
    // block they would be scalar loads, which every wait for LDS then waits for too.)
    int base = J0;
    int2 spT;
    float ksT, vsT;
    uint64_t seen;
    auto table = [&](int J) {
        base = J;
        const int x = min(J + lane, a.nblk - 1);
        spT = span[x]; ksT = ks[x]; vsT = vs[x];
        seen = __ballot(J + lane < J1 && (int64_t)spT.x <= wg_last);
    };
    // the same from the indices themselves (short caches, a block per lane: one launch less)
    auto table_of_indices = [&]() {
        base = J0;
        const int x = min(J0 + lane, a.nblk - 1), live = count - x * BLK;
        int lo = 0x7FFFFFFF, hi2 = live < BLK ? 0x7FFFFFFF : 0;
        if (J0 + lane < J1) {
            const int4 *ip = reinterpret_cast<const int4 *>(idx + (size_t)x * BLK);
#pragma unroll
            for (int q = 0; q < BLK / 4; q++) {
                const int4 id = ip[q];
                if (q * 4 < live) lo = min(lo, id.x);
                if (q * 4 + 1 < live) lo = min(lo, id.y);
                if (q * 4 + 2 < live) lo = min(lo, id.z);
                if (q * 4 + 3 < live) lo = min(lo, id.w);
                hi2 = max(hi2, max(max(id.x, id.y), max(id.z, id.w)));
            }
        }
        spT = make_int2(lo, hi2); ksT = ks[x]; vsT = vs[x];
        seen = __ballot(J0 + lane < J1 && (int64_t)lo <= wg_last);
    };
    auto lane_of = [&](int v, int J) { return __builtin_amdgcn_readlane(v, J - base); };
    auto lane_of_f = [&](float v, int J) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), J - base)); };
    // the next block from J on that is seen; the table holds it afterwards
    auto next = [&](int J) {
        while (true) {
            if (J >= J1) return J1;
            if (J >= base + 64) table(J);
            const uint64_t rest = seen >> (J - base);
            if (rest) return J + __builtin_ctzll(rest);
            J = base + 64;
        }
    };

    bf8 qf[NK][QP];
#pragma unroll
    for (int s = 0; s < NK; s++) {
        if (t < n) load_query((const TI *)a.q + b * a.q_sb + hq * a.q_sh + t * a.q_st + s * 16 + hi * 8, qf[s]);
        else zero_query<QP>(qf[s]);
    }
    f16v o[ND];
#pragma unroll
    for (int d = 0; d < ND; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) o[d][e] = 0.f;
    RowRef ref;
    float l = 0.f;          // (this lane's half of the row)

    uint4 kr[NL], vr[NL];
    int idr = 0;
    auto load = [&](int J) {
        if (tid < BLK) idr = idx[(size_t)J * BLK + tid];
        const uint8_t *kp = kc + (size_t)J * BLK * DH, *vp = vc + (size_t)J * BLK * DH;
#pragma unroll
        for (int i = 0; i < NL; i++)
            if (ALL || tid < BLK * TPR) {
                kr[i] = *reinterpret_cast<const uint4 *>(kp + (i * NTHR + tid) * 16);
                vr[i] = *reinterpret_cast<const uint4 *>(vp + (i * NTHR + tid) * 16);
            }
    };
    auto store = [&](uint8_t *buf, int J, float kscale) {
        const int live = count - J * BLK;
        if (tid < BLK) reinterpret_cast<int *>(buf + 2 * HALF)[tid] = tid < live ? idr : 0x7FFFFFFF;    // (no pair: later than all queries)
#pragma unroll
        for (int i = 0; i < NL; i++)
            if (ALL || tid < BLK * TPR) {
                const int e = i * NTHR + tid, row = e / TPR, pc = (e % TPR) * 2;
                uint8_t *kp = buf + row * DH * 2, *vp = buf + HALF + row * DH * 2;
                *reinterpret_cast<bf8 *>(kp + ((pc ^ kswz2<DH>(row)) * 16)) = codes_to_bf16(kr[i].x, kr[i].y, kscale);
                *reinterpret_cast<bf8 *>(kp + (((pc + 1) ^ kswz2<DH>(row)) * 16)) = codes_to_bf16(kr[i].z, kr[i].w, kscale);
                if (row >= live) vr[i] = make_uint4(0, 0, 0, 0);      // slots without a pair hold zeros
                *reinterpret_cast<h8 *>(vp + ((pc ^ vswz2<DH>(row)) * 16)) = codes_to_f16(vr[i].x, vr[i].y);
                *reinterpret_cast<h8 *>(vp + (((pc + 1) ^ vswz2<DH>(row)) * 16)) = codes_to_f16(vr[i].z, vr[i].w);
            }
    };

    int J = J1;
    if (J0 < J1) {
        if (span) table(J0); else table_of_indices();
        J = next(J0);
    }
    const float c = a.scale2;
    const float minus_one = opaque_minus_one();
    float ev = 0.f;      // exponent of the staged block's values
    bool masked = false, far = false;      // far: of any row (references only change where they are moved)
    if (J < J1) {
        load(J);
        ev = (float)exponent_of(lane_of_f(vsT, J));
        masked = (int64_t)lane_of(spT.y, J) > w_first;
        store(lds, J, lane_of_f(ksT, J));
    }
    if constexpr (QP == 1) {
        f16v sum;
#pragma unroll
        for (int e = 0; e < 16; e++) sum[e] = 0.f;
        bf8 zero;
        zero_query<1>(&zero);
#pragma unroll
        for (int k = 0; k < NK; k++) sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(zero, qf[k][0], sum, 0, 0, 0);
        spoil_query(qf[0], sum[0]);
    }
    lds_barrier();
    auto block = [&](auto which) {
        constexpr int CUR = decltype(which)::value;
        const int Jn = next(J + 1);
        if (Jn < J1) load(Jn);
        const uint8_t *kb = lds + CUR * BUF;
        const _Float16 *vb = reinterpret_cast<const _Float16 *>(kb + HALF);
        f16v s[2];
#pragma unroll
        for (int kt = 0; kt < 2; kt++) {
#pragma unroll
            for (int e = 0; e < 16; e++) s[kt][e] = 0.f;
            const int row = kt * 32 + l32;
#pragma unroll
            for (int k = 0; k < NK; k++) {
                const bf8 kf = *reinterpret_cast<const bf8 *>(kb + row * DH * 2 + (((2 * k + hi) ^ kswz2<DH>(row)) * 16));
#pragma unroll
                for (int p = QP - 1; p >= 0; p--) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[k][p], s[kt], 0, 0, 0);
            }
        }
        if (masked) {
            const int *ids_l = reinterpret_cast<const int *>(kb + 2 * HALF);
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const int4 id = *reinterpret_cast<const int4 *>(ids_l + kt * 32 + q * 8 + hi * 4);
                    const int ids[4] = {id.x, id.y, id.z, id.w};
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (ids[e] > pos) s[kt][q * 4 + e] = -INFINITY;
                }
        }
        float mb = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int e = 0; e < 16; e++) mb = fmaxf(mb, s[kt][e]);
        mb *= c;
        if (__builtin_expect(__any(mb - ref.m > RAISE + fminf(ref.x - ev, 0.f)), 0)) {
            float fl, fo;
            ref.move(half_max(mb), ev, fl, fo);
            far = __any(ref.far());
            l *= fl;
#pragma unroll
            for (int d = 0; d < ND; d++) o[d] *= fo;
        }
        const float drop = ref.drop(ev);
        float off = ref.m + (drop - SHIFT);
        if (__builtin_expect(far, 0)) {
            off = drop - SHIFT;
            const float ic = 1.f / c;
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
                for (int e = 0; e < 16; e++) s[kt][e] = fmaf(s[kt][e], c, -ref.m) * ic;
        }
        h8 pf[4][PP];
        float sum = 0.f;
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[kt][e], c, -off)), y = __builtin_amdgcn_exp2f(fmaf(s[kt][e + 1], c, -off));
                sum += x; sum += y;
                h2 part[PP];
                to_f16_parts<PP>(x, y, minus_one, part);
#pragma unroll
                for (int p = 0; p < PP; p++) { pf[kt * 2 + e / 8][p][e & 7] = part[p][0]; pf[kt * 2 + e / 8][p][(e & 7) + 1] = part[p][1]; }
            }
        l = fmaf(sum, __builtin_amdgcn_exp2f(drop), l);
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int j = lane & 15, key = k * 16 + hi * 4 + (j >> 2);
#pragma unroll
            for (int d = 0; d < ND; d++) {
                const int col = d * 32 + ((lane >> 4) & 1) * 16 + (j & 3) * 4;
                h8 vf;
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    const int row = key + 8 * x;
                    const h4 u = lds_read_tr16(vb + row * DH + (((col >> 3) ^ vswz2<DH>(row)) << 3) + (col & 7));
                    vf[4 * x] = u[0]; vf[4 * x + 1] = u[1]; vf[4 * x + 2] = u[2]; vf[4 * x + 3] = u[3];
                }
#pragma unroll
                for (int p = PP - 1; p >= 0; p--) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pf[k][p], o[d], 0, 0, 0);
            }
        }
        if (Jn < J1) {
            ev = (float)exponent_of(lane_of_f(vsT, Jn));
            masked = (int64_t)lane_of(spT.y, Jn) > w_first;
            store(lds + (CUR ^ 1) * BUF, Jn, lane_of_f(ksT, Jn));
        }
        lds_barrier();
        J = Jn;
    };
    while (J < J1) {      // (twice, so that each buffer's addresses are constants)
        block(std::integral_constant<int, 0>());
        if (J >= J1) break;
        block(std::integral_constant<int, 1>());
    }
    l = half_sum(l);
    if (r < R) {
        const bool pad = t >= n;
        const float il = pad || l == 0.f ? 0.f : 1.f / l, unit = __builtin_amdgcn_exp2f(ref.x);
        auto put = [&](auto *op) {
#pragma unroll
            for (int d = 0; d < ND; d++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    f4 u;
#pragma unroll
                    for (int e = 0; e < 4; e++) u[e] = il == 0.f ? 0.f : o[d][q * 4 + e] * il * unit;
                    store4(op + d * 32 + q * 8 + hi * 4, u);
                }
        };
        if (pa.nsplit == 1) {
            put((TO *)a.out + b * a.q_sb + hq * a.q_sh + t * a.q_st);
            if (pa.stat && hi == 0) pa.stat[(size_t)si * R + r] = weight_stat(ref.m, pad ? 0.f : l, SHIFT);
        } else {
            const size_t at = ((size_t)si * pa.nsplit + split) * R + r;
            put(pa.part_o + at * DH);
            if (hi == 0) { pa.part_ml[at * 2] = ref.m; pa.part_ml[at * 2 + 1] = pad ? 0.f : l; }
        }
    }
}

// joins the shares of a row: DH / 4 threads each
template <int DH, typename TO>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs pa) {
    const Args &a = pa.a;
    constexpr int TPR = DH / 4;
    const int si = blockIdx.y, R = a.T * a.g, r = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, col = (threadIdx.x % TPR) * 4;
    if (r >= R) return;
    const int b = si / a.Hkv, h = si - b * a.Hkv, t = r / a.g, hq = h * a.g + (r - t * a.g);
    float M = -INFINITY, L = 0.f;
    for (int s = 0; s < pa.nsplit; s++) M = fmaxf(M, pa.part_ml[(((size_t)si * pa.nsplit + s) * R + r) * 2]);
    const float mu = M == -INFINITY ? 0.f : M;
    f4 acc = (f4){0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < pa.nsplit; s++) {
        const size_t at = ((size_t)si * pa.nsplit + s) * R + r;
        const float f = pa.part_ml[at * 2 + 1] * __builtin_amdgcn_exp2f(pa.part_ml[at * 2] - mu);
        L += f;
        acc += *reinterpret_cast<const f4 *>(pa.part_o + at * DH + col) * f;
    }
    TO *op = (TO *)a.out + b * a.q_sb + hq * a.q_sh + t * a.q_st;
#pragma unroll
    for (int e = 0; e < 4; e++) stf(op, col + e, L == 0.f ? 0.f : acc[e] / L);
    if (pa.stat && col == 0) pa.stat[(size_t)si * R + r] = weight_stat(mu, L, Slack<TO>::shift);
}

// sum over the 32 lanes of a half wavefront, in each of them
__device__ __forceinline__ float sum32(float v) {
    v += lane_perm<PERM_XOR1>(v); v += lane_perm<PERM_XOR2>(v); v += lane_perm<PERM_MIRROR8>(v); v += lane_perm<PERM_MIRROR16>(v);
    const Two t = swap_rows16(v);
    return t.a + t.b;
}

// weight[j] += sum over rows of their weight of pair j (weight_stat): one workgroup per block of slots, whose keys stay in registers as the first operand of
// S^T = K Q^T; the wavefronts take 32 rows in turn, straight from global memory, and join their sums at the end.  Bound by vector
// instructions, an exponential and three others per logit, and by unequal workgroups: the first block's has all rows, the last one's hardly any (two prompts of
// 2000 tokens at d = 64: 58 us, 16.4 GFLOP).
template <int DH, typename TI>
__global__ __launch_bounds__(256, (DH == 256 || sizeof(TI) == 4) ? 1 : 2) void prompt_gather_kernel(PromptArgs pa) {
    constexpr int QP = sizeof(TI) == 4 ? 3 : 1, NK = DH / 16;
    __shared__ float sum_l[4][64];
    const Args &a = pa.a;
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
    const int S = a.B * a.Hkv, si = blockIdx.x % S, b = si / a.Hkv, h = si - b * a.Hkv;
    const int R = a.T * a.g, n = new_tokens(a, b), count = n ? held(a, si) : 0;
    for (int J = blockIdx.x / S; J * BLK < count; J += gridDim.x / S) {
        const int2 sp = pa.span[(size_t)si * a.nblk + J];
        const int64_t pos0 = a.mem.n_tokens[si] - n;
        const int live = count - J * BLK;
        const float kscale = a.mem.ks[(size_t)si * a.nblk + J];
        bf8 kf[2][NK];
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int k = 0; k < NK; k++) {
                const uint2 u = *reinterpret_cast<const uint2 *>(a.mem.k + ((size_t)si * a.cap + (size_t)J * BLK + kt * 32 + l32) * DH + k * 16 + hi * 8);
                kf[kt][k] = codes_to_bf16(u.x, u.y, kscale);
            }
        const float c = a.scale2;
        float acc[2][16];
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[kt][e] = 0.f;
        // rows from the first token that sees any of the block's pairs
        const int64_t t0 = (int64_t)sp.x > pos0 ? (int64_t)sp.x - pos0 : 0;
        const int rows = n * a.g, first = t0 >= n ? rows : (int)t0 * a.g / 32 * 32;
        // this lane's row as token and head, moved on by 128 rows at a time; the next row's queries are under way while one is worked on
        int r = first + w * 32 + l32, t = r / a.g, hd = r - t * a.g;
        const int t_step = 128 / a.g, h_step = 128 - t_step * a.g;
        bf8 qf[NK][QP];
        float2 st;
        auto load = [&]() {
            const TI *qp = (const TI *)a.q + b * a.q_sb + (h * a.g + hd) * a.q_sh + t * a.q_st + hi * 8;
            st = r < rows ? pa.stat[(size_t)si * R + r] : make_float2(INFINITY, 0.f);
#pragma unroll
            for (int k = 0; k < NK; k++) {
                if (r < rows) load_query(qp + k * 16, qf[k]);
                else zero_query<QP>(qf[k]);
            }
        };
        load();
        for (int r0 = first + w * 32; r0 < rows; r0 += 128) {
            const int pos = (int)(pos0 + t);
            const float off = st.x, part = st.y;
            f16v s[2];
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
                for (int e = 0; e < 16; e++) s[kt][e] = 0.f;
#pragma unroll
            for (int k = 0; k < NK; k++)
#pragma unroll
                for (int kt = 0; kt < 2; kt++)
#pragma unroll
                    for (int p = QP - 1; p >= 0; p--) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kt][k], qf[k][p], s[kt], 0, 0, 0);
            const bool masked = (int64_t)sp.y > pos0 + r0 / a.g;      // (slots without a pair count as later than all queries)
            r += 128; t += t_step; hd += h_step;
            if (hd >= a.g) { hd -= a.g; t++; }
            load();
            // the power is in [0, 1]; the clamp, an output modifier of the exponential, makes 0 of what rows without weight (off infinite) make of a NaN key
            if (masked) {
#pragma unroll
                for (int kt = 0; kt < 2; kt++)
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        const int at = kt * 32 + q * 8 + hi * 4;
                        const int4 id = *reinterpret_cast<const int4 *>(a.mem.idx + (size_t)si * a.cap + (size_t)J * BLK + at);
                        const int ids[4] = {id.x, id.y, id.z, id.w};
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            if (ids[e] > pos || at + e >= live) s[kt][q * 4 + e] = -INFINITY;
                    }
            }
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
                for (int e = 0; e < 16; e++) acc[kt][e] = fmaf(__builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(fmaf(s[kt][e], c, -off)), 0.f, 1.f), part, acc[kt][e]);
        }
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int e = 0; e < 16; e++) {
                float v = acc[kt][e];
                v = sum32(v);
                if (l32 == 0) sum_l[w][kt * 32 + (e / 4) * 8 + hi * 4 + (e & 3)] = v;
            }
        __syncthreads();
        if (tid < 64 && tid < live) {
            float *wp = a.mem.weight + (size_t)si * a.cap + (size_t)J * BLK + tid;
            *wp += (sum_l[0][tid] + sum_l[1][tid]) + (sum_l[2][tid] + sum_l[3][tid]);
        }
        __syncthreads();   // the sums have been read
    }
}

}  // namespace full
}  // namespace lola
