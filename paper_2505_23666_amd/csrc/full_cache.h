// Kernels of the 8-bit full-context cache (include/lola.h, lola_full_*): append, attention, eviction.
//
// One stream = one (sequence, kv head).  Codes are OCP e4m3, row-major [slot][d] for keys and values alike; a block of 64 slots
// has one power-of-two scale for its keys and one for its values, so that quantising, rescaling and moving a code are exact up
// to the single rounding to the e4m3 grid, and dequantising is exact.
#pragma once
#include "lola_common.h"

namespace lola {
namespace full {

constexpr int BLK = 64;          // slots per block
constexpr int EXP_MIN = -100;    // least exponent of a block's scale
constexpr float LOG2E_F = 1.44269504088896340736f;

struct Mem {
    uint8_t *k, *v;
    float *ks, *vs;
    int32_t *idx;
    float *weight;
    int32_t *count;
    int64_t *n_tokens;
};

struct Args {
    Mem mem;
    int B, Hq, Hkv, g, d, cap, nblk, T;
    const int32_t *lens;
    // token matrices: element offset of (b, head, token) is b * sb + head * sh + token * st
    const void *q, *k, *v;
    void *out;
    int64_t q_sb, q_sh, q_st, k_sb, k_sh, k_st;
    float scale2;                // logit scale * log2(e): softmax in powers of two
};

__device__ __forceinline__ int exponent_of(float scale) { return (int)((__float_as_uint(scale) >> 23) & 255u) - 127; }
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// least e >= EXP_MIN with a <= 448 * 2^e, a >= 0 finite: 448 = 1.75 * 2^8, a = 1.f * 2^x (a below 2^-126 is below every bound)
__device__ __forceinline__ int fit_exponent(float a) {
    const uint32_t u = __float_as_uint(a);
    const int x = (int)(u >> 23) - 127;
    const int e = x - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < EXP_MIN ? EXP_MIN : e;
}
__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }

typedef float f32x2 __attribute__((ext_vector_type(2)));
// four floats -> four codes (round to nearest even; the callers' scales keep |x| <= 448)
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
__device__ __forceinline__ void from_codes(uint32_t c, float *x) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
}
// codes of one block's scale -> codes of another's (f = 2^(old - new)); NaN stays
__device__ __forceinline__ uint32_t rescale_codes(uint32_t c, float f) {
    float x[4];
    from_codes(c, x);
    return to_codes(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
}

// this lane's value and that of the lane 16 / 32 away (row swaps, no LDS round trip)
struct Two { float a, b; };
__device__ __forceinline__ Two swap_rows16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return Two{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ Two swap_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return Two{__uint_as_float(r[0]), __uint_as_float(r[1])};
}

// Permutations of lanes inside rows of 16, a vector instruction each (a shuffle goes through LDS, some 100 cycles)
enum { PERM_XOR1 = 0xB1, PERM_XOR2 = 0x4E, PERM_MIRROR8 = 0x141, PERM_MIRROR16 = 0x140 };
template <int PERM>
__device__ __forceinline__ float lane_perm(float v) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), PERM, 0xF, 0xF, true));
}
// maximum over N neighbouring lanes (N = 4, 8, 16, 32, aligned), in each of them
template <int N>
__device__ __forceinline__ float max_of(float v) {
    v = fmaxf(v, lane_perm<PERM_XOR1>(v));
    v = fmaxf(v, lane_perm<PERM_XOR2>(v));
    if (N >= 8) v = fmaxf(v, lane_perm<PERM_MIRROR8>(v));
    if (N >= 16) v = fmaxf(v, lane_perm<PERM_MIRROR16>(v));
    if (N >= 32) { const Two t = swap_rows16(v); v = fmaxf(t.a, t.b); }
    return v;
}
__device__ __forceinline__ float max_of_wave(float v) { const Two t = swap_halves(max_of<32>(v)); return fmaxf(t.a, t.b); }
// sums of the lanes up to and with this one
__device__ __forceinline__ int scan_wave(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);     // from 1, 2, 4, 8 lanes below in the row
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);     // the last lane of rows 0 and 2 to rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);     // lane 31 to rows 2 and 3
    return x;
}

__device__ __forceinline__ void load8(const float *p, float *x) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t *p, float *x) {
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; i++) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u); }
}

__device__ __forceinline__ int new_tokens(const Args &a, int b) {
    if (!a.lens) return a.T;
    const int n = a.lens[b];
    return n < 0 ? 0 : (n > a.T ? a.T : n);
}
__device__ __forceinline__ int held(const Args &a, int si) {
    const int c = a.mem.count[si];
    return c < 0 ? 0 : (c > a.cap ? a.cap : c);
}

// ---- append -------------------------------------------------------------------------------------------------
// A workgroup takes `per` consecutive blocks of the window of blocks that a stream's new tokens fall into, G at a time, 256 threads each: a
// block's new rows (8 elements of a row per thread) are held in registers, the largest magnitudes are joined over its threads,
// rows that the block held before are rescaled only if its exponent grows.  Bound by HBM: 2 T d elements read, 2 T d codes written (4 x 32 Ki
// tokens, 8 kv heads, d = 128: 158 us, 5.1 TB/s); a call of a few tokens is a chain of four dependent accesses, 6 us.
template <int DH, typename TI, int G>
__global__ __launch_bounds__(256 * G) void append_kernel(Args a, int per, int advance) {
    constexpr int TPR = DH / 8, RPP = 256 / TPR, NP = BLK / RPP < 1 ? 1 : BLK / RPP;   // threads per row, rows per pass, passes
    __shared__ float red_l[G][2][4];
    const int si = blockIdx.x, b = si / a.Hkv, h = si - b * a.Hkv, grp = threadIdx.x / 256, tid = threadIdx.x % 256, lane = tid & 63, w = tid >> 6;
    float (*red)[4] = red_l[grp];
    const int c0 = held(a, si), told = new_tokens(a, b), n = min(told, a.cap - c0);
    const int64_t first = a.mem.n_tokens[si];
    const TI *kp = (const TI *)a.k + b * a.k_sb + h * a.k_sh, *vp = (const TI *)a.v + b * a.k_sb + h * a.k_sh;
    const int col = (tid % TPR) * 8, row0 = tid / TPR;
    for (int i = 0; i < per; i += G) {
        const int Ji = c0 / BLK + blockIdx.y * per + i, J = Ji + grp, lo = max(c0, J * BLK), hi = min(c0 + n, J * BLK + BLK);
        if (Ji * BLK >= c0 + n) break;   // (the workgroup's; a group beyond the end goes along without rows)
        const bool work = G == 1 || lo < hi;
        uint8_t *kc = a.mem.k + ((size_t)si * a.cap + (size_t)J * BLK) * DH, *vc = a.mem.v + ((size_t)si * a.cap + (size_t)J * BLK) * DH;
        float x[NP][8], y[NP][8], ak = 0.f, av = 0.f;
        bool bad[NP];
#pragma unroll
        for (int p = 0; p < NP; p++) {
            const int slot = J * BLK + p * RPP + row0;
            const bool mine = slot >= lo && slot < hi;
#pragma unroll
            for (int e = 0; e < 8; e++) x[p][e] = y[p][e] = 0.f;
            if (mine) {
                load8(kp + (slot - c0) * a.k_st + col, x[p]);
                load8(vp + (slot - c0) * a.k_st + col, y[p]);
            }
        }
#pragma unroll
        for (int p = 0; p < NP; p++) {
            int nf = 0;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                if (!finite(x[p][e])) nf = 1;
                if (!finite(y[p][e])) { nf = 1; y[p][e] = 0.f; }
                av = fmaxf(av, fabsf(y[p][e]));
            }
            bad[p] = ((__ballot(nf) >> (lane & ~(TPR - 1))) & ((1ull << TPR) - 1)) != 0;     // any of the row's threads
            if (!bad[p])
#pragma unroll
                for (int e = 0; e < 8; e++) ak = fmaxf(ak, fabsf(x[p][e]));
        }
        ak = max_of_wave(ak); av = max_of_wave(av);
        __syncthreads();   // (the last block's readers are done)
        if (lane == 0) { red[0][w] = ak; red[1][w] = av; }
        __syncthreads();
        ak = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
        av = fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3]));
        int ek = fit_exponent(ak), ev = fit_exponent(av);
        const int nold = work ? max(0, c0 - J * BLK) : 0;   // rows held before
        if (nold > 0) {
            const int ok = exponent_of(a.mem.ks[(size_t)si * a.nblk + J]), ov = exponent_of(a.mem.vs[(size_t)si * a.nblk + J]);
            ek = max(ek, ok); ev = max(ev, ov);
            const float fk = pow2(max(ok - ek, -40)), fv = pow2(max(ov - ev, -40));   // (2^-40 takes every code to zero)
            for (int e = tid; e < nold * TPR; e += 256) {
                if (ek > ok) { uint2 u = reinterpret_cast<uint2 *>(kc)[e]; u.x = rescale_codes(u.x, fk); u.y = rescale_codes(u.y, fk); reinterpret_cast<uint2 *>(kc)[e] = u; }
                if (ev > ov) { uint2 u = reinterpret_cast<uint2 *>(vc)[e]; u.x = rescale_codes(u.x, fv); u.y = rescale_codes(u.y, fv); reinterpret_cast<uint2 *>(vc)[e] = u; }
            }
        }
        if (G > 1 || nold > 0) __syncthreads();   // every thread has read the old scales
        if (work && tid == 0) { a.mem.ks[(size_t)si * a.nblk + J] = pow2(ek); a.mem.vs[(size_t)si * a.nblk + J] = pow2(ev); }
        const float ik = pow2(-ek), iv = pow2(-ev);
#pragma unroll
        for (int p = 0; p < NP; p++) {
            const int row = p * RPP + row0, slot = J * BLK + row;
            if (slot < lo || slot >= hi) continue;
            uint2 u;
            u.x = to_codes(x[p][0] * ik, x[p][1] * ik, x[p][2] * ik, x[p][3] * ik);
            u.y = to_codes(x[p][4] * ik, x[p][5] * ik, x[p][6] * ik, x[p][7] * ik);
            if (bad[p]) u.x = u.y = 0x7F7F7F7Fu;
            *reinterpret_cast<uint2 *>(kc + row * DH + col) = u;
            u.x = to_codes(y[p][0] * iv, y[p][1] * iv, y[p][2] * iv, y[p][3] * iv);
            u.y = to_codes(y[p][4] * iv, y[p][5] * iv, y[p][6] * iv, y[p][7] * iv);
            *reinterpret_cast<uint2 *>(vc + row * DH + col) = u;
        }
        for (int s = lo + tid; s < hi; s += 256) {
            a.mem.idx[(size_t)si * a.cap + s] = (int32_t)(first + (s - c0));
            if (a.mem.weight) a.mem.weight[(size_t)si * a.cap + s] = 0.f;
        }
    }
    if (advance) {   // this workgroup has all of the stream's blocks
        __syncthreads();   // every thread has read count and n_tokens
        if (threadIdx.x == 0) { a.mem.count[si] = c0 + n; a.mem.n_tokens[si] = first + told; }
    }
}

// count and n_tokens after an append of several workgroups per stream
__global__ __launch_bounds__(256) void advance_kernel(Args a) {
    const int si = blockIdx.x * 256 + threadIdx.x;
    if (si >= a.B * a.Hkv) return;
    const int c0 = held(a, si), told = new_tokens(a, si / a.Hkv);
    a.mem.count[si] = c0 + min(told, a.cap - c0);
    a.mem.n_tokens[si] += told;
}

__global__ __launch_bounds__(256) void init_kernel(int32_t *count, int64_t *n_tokens, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) { count[i] = 0; n_tokens[i] = 0; }
}

// ---- eviction -------------------------------------------------------------------------------------------------
struct EvictArgs {
    Mem mem;
    int cap, nblk, keep, first, recent, d;
    // per stream: slots that become free, where their new pairs come from (ascending both), number of holes below each block,
    // scales of the block that the budget ends in, as they were
    int32_t *dst, *src, *before;
    float *edge;
    int most, nkb;               // entries per stream of dst and src; blocks that hold slots below keep
};

// larger rank = stays: pairs that always stay above all, then NaN, then by weight (any float, -0 = +0)
__device__ __forceinline__ uint32_t rank_of(int i, float w, int first, int64_t recent_from) {
    if (i < first || i >= recent_from) return 0xFFFFFFFFu;
    w += 0.f;
    if (w != w) return 0xFFFFFFFEu;
    const uint32_t u = __float_as_uint(w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// exclusive sum over the workgroup's threads; *total receives the sum
template <int NT>
__device__ __forceinline__ int scan_all(int v, int *wsum, int *total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int x = scan_wave(v);
    __syncthreads();
    if (lane == 63) wsum[w] = x;
    __syncthreads();
    int base = 0, all = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; i++) { if (i < w) base += wsum[i]; all += wsum[i]; }
    *total = all;
    return base + x - v;
}

constexpr int RANKS_LDS = 32768;   // ranks that the selection keeps in LDS; longer caches compute them again in each pass

constexpr int RANK_BINS = 2048;
struct SelectLds { int hist[RANK_BINS], wsum[16], found[3]; };

// The workgroup finds the stream's keep-th largest rank (0 < keep < count) in three passes over the ranks (11, 11 and 10 bits: a histogram in LDS
// and a scan over its bins), then writes the lists: dst, src, and before (may be NULL) without its last entry.  A thread takes four
// slots at a time.  Returns the number of pairs that move.
template <int NT>
__device__ __forceinline__ int select_pairs(const EvictArgs &a, int si, int count, uint32_t *rank_l, SelectLds &l, int32_t *dst, int32_t *src, int32_t *before) {
    constexpr int NB = RANK_BINS, BPT = NB / NT;
    int *hist = l.hist, *wsum = l.wsum, *found = l.found;
    const int tid = threadIdx.x;
    const size_t base = (size_t)si * a.cap;
    const int64_t recent_from = a.mem.n_tokens[si] - a.recent;
    const bool cached = a.cap <= RANKS_LDS;
    // ranks of slots s .. s + 3 (s a multiple of four; beyond count: nothing looks at them)
    auto ranks_of = [&](int4 i, float4 w) {
        return make_uint4(rank_of(i.x, w.x, a.first, recent_from), rank_of(i.y, w.y, a.first, recent_from),
                          rank_of(i.z, w.z, a.first, recent_from), rank_of(i.w, w.w, a.first, recent_from));
    };
    auto compute = [&](int s) {
        return ranks_of(*reinterpret_cast<const int4 *>(a.mem.idx + base + s), *reinterpret_cast<const float4 *>(a.mem.weight + base + s));
    };
    auto ranks = [&](int s) { return cached ? *reinterpret_cast<const uint4 *>(rank_l + s) : compute(s); };
    uint32_t prefix = 0, mask = 0;
    int want = a.keep, equal = 0;       // of the ranks that match the prefix, the want-th largest is looked for
#pragma unroll
    for (int pass = 0; pass < 3; pass++) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digit = pass == 2 ? 1023u : 2047u;
        for (int i = tid; i < NB; i += NT) hist[i] = 0;
        __syncthreads();
        auto count_in = [&](int s, uint4 u) {
            const uint32_t us[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (s + e < count && (us[e] & mask) == prefix) atomicAdd(&hist[(us[e] >> shift) & digit], 1);
        };
        if (pass == 0) {      // (sixteen slots' loads under way at a time)
            for (int s0 = tid * 4; s0 < count; s0 += NT * 16) {
                int4 i[4];
                float4 w[4];
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    const int s = s0 + x * NT * 4;
                    if (s < count) { i[x] = *reinterpret_cast<const int4 *>(a.mem.idx + base + s); w[x] = *reinterpret_cast<const float4 *>(a.mem.weight + base + s); }
                }
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    const int s = s0 + x * NT * 4;
                    if (s >= count) continue;
                    const uint4 u = ranks_of(i[x], w[x]);
                    if (cached) *reinterpret_cast<uint4 *>(rank_l + s) = u;
                    count_in(s, u);
                }
            }
        } else
            for (int s = tid * 4; s < count; s += NT * 4) count_in(s, ranks(s));
        __syncthreads();
        // bins from the largest down: thread t has BPT of them from NB - 1 - t BPT on
        int mine = 0, total;
#pragma unroll
        for (int i = 0; i < BPT; i++) mine += hist[NB - 1 - tid * BPT - i];
        int above = scan_all<NT>(mine, wsum, &total);
        if (above < want && above + mine >= want) {
            for (int i = 0; i < BPT; i++) {
                const int v = NB - 1 - tid * BPT - i, n = hist[v];
                if (above + n >= want) { found[0] = v; found[1] = want - above; found[2] = n; break; }
                above += n;
            }
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift; mask |= digit << shift; want = found[1]; equal = found[2];
        __syncthreads();
    }
    // kept: rank > prefix, and the `want` lowest slots of the `equal` ones with rank == prefix
    int ties = 0, holes = 0, moved = 0;
    for (int s0 = 0; s0 < count; s0 += NT * 4) {
        const int s = s0 + tid * 4;
        const uint4 u = s < count ? ranks(s) : make_uint4(0, 0, 0, 0);
        const uint32_t us[4] = {u.x, u.y, u.z, u.w};
        int t_at = ties;
        if (equal != want) {
            int n = 0, all;
#pragma unroll
            for (int e = 0; e < 4; e++) n += s + e < count && us[e] == prefix;
            t_at += scan_all<NT>(n, wsum, &all);
            ties += all;
        }
        int kinds = 0, hole[4], mover[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const bool in = s + e < count, tie = in && us[e] == prefix;
            const bool kept = in && (us[e] > prefix || (tie && t_at < want));
            if (tie && equal != want) t_at++;
            hole[e] = in && s + e < a.keep && !kept;
            mover[e] = s + e >= a.keep && kept;
            kinds += hole[e] + (mover[e] << 16);
        }
        int all;
        const int at = scan_all<NT>(kinds, wsum, &all);
        int h_at = holes + (at & 0xFFFF), m_at = moved + (at >> 16);
        if (before && s % BLK == 0 && s < a.keep) before[s / BLK] = h_at;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            if (hole[e] && h_at < a.most) dst[h_at++] = s + e;
            if (mover[e] && m_at < a.most) src[m_at++] = s + e;
        }
        holes += all & 0xFFFF; moved += all >> 16;
    }
    return holes;
}

// One workgroup per stream: the lists of evict_move_kernel.  Bound by latency: a handful of dependent passes over a few thousand ranks
// (32 Ki slots of 32 streams 26 us).
template <int NT>
__global__ __launch_bounds__(NT) void evict_select_kernel(EvictArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint32_t rank_l[];     // [min(cap, RANKS_LDS)] where they fit
    __shared__ SelectLds l;
    const int si = blockIdx.x, tid = threadIdx.x;
    int count = a.mem.count[si];
    count = count < 0 ? 0 : (count > a.cap ? a.cap : count);
    int32_t *before = a.before + (size_t)si * (a.nkb + 1);
    if (count <= a.keep) {
        for (int J = tid; J <= a.nkb; J += NT) before[J] = 0;
        return;
    }
    if (a.keep == 0) {      // nothing to rank
        if (tid == 0) a.mem.count[si] = 0;
        return;
    }
    const int holes = select_pairs<NT>(a, si, count, rank_l, l, a.dst + (size_t)si * a.most, a.src + (size_t)si * a.most, before);
    if (tid == 0) {
        before[a.nkb] = holes;
        if (a.keep % BLK) {
            a.edge[2 * si] = a.mem.ks[(size_t)si * a.nblk + a.keep / BLK];
            a.edge[2 * si + 1] = a.mem.vs[(size_t)si * a.nblk + a.keep / BLK];
        }
        a.mem.count[si] = a.keep;
    }
}

// The whole eviction of a stream by one workgroup, where few pairs can move: the lists stay in LDS, the pairs are moved side by side rather
// than block by block.  Each pair raises its block's exponents to what it needs (an LDS maximum), blocks whose exponent grew are
// rescaled, then the pairs are written; the scales themselves last, since a pair may come from the block that the budget ends in.
// Bound by latency: 64 of 2112 pairs, 128 streams, d = 128 14 us; 16 of 1127, 1024 streams, d = 64 17 us.
template <int DH>
__global__ __launch_bounds__(256) void evict_few_kernel(EvictArgs a) {
    constexpr int TPR = DH / 8, RPP = 256 / TPR, U = 4;      // threads per row, rows per pass, passes held in registers
    extern __shared__ __attribute__((aligned(16))) uint32_t rank_l[];     // ranks [cap], then dst, src [most], exponents of keys, values [nkb], grown [nkb]
    __shared__ SelectLds l;
    __shared__ int ngrown;
    const int si = blockIdx.x, tid = threadIdx.x;
    int count = a.mem.count[si];
    count = count < 0 ? 0 : (count > a.cap ? a.cap : count);
    if (count <= a.keep) return;
    if (a.keep == 0) {
        if (tid == 0) a.mem.count[si] = 0;
        return;
    }
    int *dst = (int *)rank_l + a.cap, *src = dst + a.most, *ek = src + a.most, *ev = ek + a.nkb, *grown = ev + a.nkb;
    float *ks = a.mem.ks + (size_t)si * a.nblk, *vs = a.mem.vs + (size_t)si * a.nblk;
    int ok = 0, ov = 0;      // of block tid (at most 128 blocks)
    if (tid < a.nkb) { ek[tid] = ok = exponent_of(ks[tid]); ev[tid] = ov = exponent_of(vs[tid]); }
    if (tid == 0) ngrown = 0;
    const int n = select_pairs<256>(a, si, count, rank_l, l, dst, src, nullptr);
    __syncthreads();
    const size_t base = (size_t)si * a.cap;
    const int col = (tid % TPR) * 8;
    uint2 kc[U], vc[U];
    float sk[U], sv[U], wt[U];
    int32_t id[U];
    auto load = [&](int p0) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int p = p0 + u * RPP + tid / TPR;
            kc[u] = vc[u] = make_uint2(0, 0); sk[u] = sv[u] = 0.f;
            if (p >= n) continue;
            const int s = src[p];
            kc[u] = *reinterpret_cast<const uint2 *>(a.mem.k + (base + s) * DH + col);
            vc[u] = *reinterpret_cast<const uint2 *>(a.mem.v + (base + s) * DH + col);
            sk[u] = ks[s / BLK]; sv[u] = vs[s / BLK];
            id[u] = a.mem.idx[base + s]; wt[u] = a.mem.weight[base + s];
        }
    };
    for (int p0 = 0; p0 < n; p0 += U * RPP) {
        load(p0);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int p = p0 + u * RPP + tid / TPR;
            float x[8], mk = 0.f, mv = 0.f;
            from_codes(kc[u].x, x); from_codes(kc[u].y, x + 4);
#pragma unroll
            for (int e = 0; e < 8; e++) mk = fmaxf(mk, fabsf(x[e]));   // (a NaN key counts as zero)
            from_codes(vc[u].x, x); from_codes(vc[u].y, x + 4);
#pragma unroll
            for (int e = 0; e < 8; e++) mv = fmaxf(mv, fabsf(x[e]));
            mk = max_of<TPR>(mk); mv = max_of<TPR>(mv);
            if (p < n && tid % TPR == 0) {
                atomicMax(&ek[dst[p] / BLK], fit_exponent(mk * sk[u]));
                atomicMax(&ev[dst[p] / BLK], fit_exponent(mv * sv[u]));
            }
        }
    }
    __syncthreads();
    if (tid < a.nkb && (ek[tid] > ok || ev[tid] > ov)) grown[atomicAdd(&ngrown, 1)] = tid;
    __syncthreads();
    for (int i = 0; i < ngrown; i++) {
        const int J = grown[i], dk = exponent_of(ks[J]) - ek[J], dv = exponent_of(vs[J]) - ev[J], rows = min(BLK, a.keep - J * BLK);
        const float fk = pow2(max(dk, -40)), fv = pow2(max(dv, -40));
        uint8_t *kb = a.mem.k + (base + (size_t)J * BLK) * DH, *vb = a.mem.v + (base + (size_t)J * BLK) * DH;
        for (int e = tid; e < rows * TPR; e += 256) {
            if (dk < 0) { uint2 u = reinterpret_cast<uint2 *>(kb)[e]; u.x = rescale_codes(u.x, fk); u.y = rescale_codes(u.y, fk); reinterpret_cast<uint2 *>(kb)[e] = u; }
            if (dv < 0) { uint2 u = reinterpret_cast<uint2 *>(vb)[e]; u.x = rescale_codes(u.x, fv); u.y = rescale_codes(u.y, fv); reinterpret_cast<uint2 *>(vb)[e] = u; }
        }
    }
    if (ngrown) __syncthreads();      // (rows that moved pairs replace were rescaled by other threads)
    for (int p0 = 0; p0 < n; p0 += U * RPP) {
        if (n > U * RPP) load(p0);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int p = p0 + u * RPP + tid / TPR;
            if (p >= n) continue;
            const int t = dst[p], J = t / BLK;
            const float fk = pow2(min(40, max(exponent_of(sk[u]) - ek[J], -40))), fv = pow2(min(40, max(exponent_of(sv[u]) - ev[J], -40)));
            uint2 c = kc[u];
            c.x = rescale_codes(c.x, fk); c.y = rescale_codes(c.y, fk);
            *reinterpret_cast<uint2 *>(a.mem.k + (base + t) * DH + col) = c;
            c = vc[u];
            c.x = rescale_codes(c.x, fv); c.y = rescale_codes(c.y, fv);
            *reinterpret_cast<uint2 *>(a.mem.v + (base + t) * DH + col) = c;
            if (tid % TPR == 0) { a.mem.idx[base + t] = id[u]; a.mem.weight[base + t] = wt[u]; }
        }
    }
    __syncthreads();      // every source's scale has been read
    for (int i = tid; i < ngrown; i += 256) { const int J = grown[i]; ks[J] = pow2(ek[J]); vs[J] = pow2(ev[J]); }
    if (tid == 0) a.mem.count[si] = a.keep;
}

// The pairs that move into a block below the budget come from slots at and beyond `keep`, which no workgroup writes.  (Of the block
// that the budget ends in only rows below it are rescaled; its scales, which others read as a source's, are read from the copy
// taken beforehand.)  One workgroup per block; up to four passes over the rows are held in registers between finding the exponent
// and writing.
template <int DH>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    constexpr int TPR = DH / 8, RPP = 256 / TPR, U = 4;      // threads per row, rows per pass, passes held
    __shared__ float red[2][4];
    const int si = blockIdx.y, w = threadIdx.x >> 6, lane = threadIdx.x & 63, tid = threadIdx.x, J = blockIdx.x;
    const int j0 = a.before[(size_t)si * (a.nkb + 1) + J], j1 = min(a.before[(size_t)si * (a.nkb + 1) + J + 1], a.most);
    if (j0 >= j1) return;
    const int32_t *dst = a.dst + (size_t)si * a.most, *src = a.src + (size_t)si * a.most;
    const size_t base = (size_t)si * a.cap;
    const int col = (tid % TPR) * 8;
    const float ok_s = a.mem.ks[(size_t)si * a.nblk + J], ov_s = a.mem.vs[(size_t)si * a.nblk + J];
    const float edge_k = a.edge[2 * si], edge_v = a.edge[2 * si + 1];
    uint2 kc[U], vc[U];
    float sk[U], sv[U];
    int from[U];
    auto load = [&](int jb) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int j = jb + u * RPP + tid / TPR;
            from[u] = j < j1 ? src[j] : -1;
            if (from[u] < a.keep || from[u] >= a.cap) from[u] = -1;      // (never, unless weights change while they are ranked)
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int s = from[u];
            kc[u] = vc[u] = make_uint2(0, 0); sk[u] = sv[u] = 0.f;
            if (s < 0) continue;
            kc[u] = *reinterpret_cast<const uint2 *>(a.mem.k + (base + s) * DH + col);
            vc[u] = *reinterpret_cast<const uint2 *>(a.mem.v + (base + s) * DH + col);
            const bool edge = a.keep % BLK && s / BLK == a.keep / BLK;
            sk[u] = edge ? edge_k : a.mem.ks[(size_t)si * a.nblk + s / BLK];
            sv[u] = edge ? edge_v : a.mem.vs[(size_t)si * a.nblk + s / BLK];
        }
    };
    float ak = 0.f, av = 0.f;
    for (int jb = j0; jb < j1; jb += U * RPP) {
        load(jb);
#pragma unroll
        for (int u = 0; u < U; u++) {
            float x[8], mk = 0.f, mv = 0.f;
            from_codes(kc[u].x, x); from_codes(kc[u].y, x + 4);
#pragma unroll
            for (int e = 0; e < 8; e++) mk = fmaxf(mk, fabsf(x[e]));   // (a NaN key counts as zero)
            from_codes(vc[u].x, x); from_codes(vc[u].y, x + 4);
#pragma unroll
            for (int e = 0; e < 8; e++) mv = fmaxf(mv, fabsf(x[e]));
            ak = fmaxf(ak, mk * sk[u]);
            av = fmaxf(av, mv * sv[u]);
        }
    }
    ak = max_of_wave(ak); av = max_of_wave(av);
    if (lane == 0) { red[0][w] = ak; red[1][w] = av; }
    __syncthreads();
    ak = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    av = fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3]));
    const int ok = exponent_of(ok_s), ov = exponent_of(ov_s), ek = max(ok, fit_exponent(ak)), ev = max(ov, fit_exponent(av));
    uint8_t *kb = a.mem.k + (base + (size_t)J * BLK) * DH, *vb = a.mem.v + (base + (size_t)J * BLK) * DH;
    if (ek > ok || ev > ov) {
        const float fk = pow2(max(ok - ek, -40)), fv = pow2(max(ov - ev, -40));
        const int rows = min(BLK, a.keep - J * BLK);
        for (int e = tid; e < rows * TPR; e += 256) {
            if (ek > ok) { uint2 u = reinterpret_cast<uint2 *>(kb)[e]; u.x = rescale_codes(u.x, fk); u.y = rescale_codes(u.y, fk); reinterpret_cast<uint2 *>(kb)[e] = u; }
            if (ev > ov) { uint2 u = reinterpret_cast<uint2 *>(vb)[e]; u.x = rescale_codes(u.x, fv); u.y = rescale_codes(u.y, fv); reinterpret_cast<uint2 *>(vb)[e] = u; }
        }
        if (tid == 0) { a.mem.ks[(size_t)si * a.nblk + J] = pow2(ek); a.mem.vs[(size_t)si * a.nblk + J] = pow2(ev); }
        __syncthreads();   // the rows that the moved pairs replace were rescaled by other threads
    }
    for (int jb = j0; jb < j1; jb += U * RPP) {
        if (j1 - j0 > U * RPP) load(jb);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int s = from[u];
            if (s < 0) continue;
            const int t = dst[jb + u * RPP + tid / TPR];
            if (t < 0 || t >= a.keep) continue;
            // (a source's exponent may be larger than the block's: its codes then grow, and fit by the choice of ek, ev)
            const float fk = pow2(min(40, max(exponent_of(sk[u]) - ek, -40))), fv = pow2(min(40, max(exponent_of(sv[u]) - ev, -40)));
            uint2 c = kc[u];
            c.x = rescale_codes(c.x, fk); c.y = rescale_codes(c.y, fk);
            *reinterpret_cast<uint2 *>(a.mem.k + (base + t) * DH + col) = c;
            c = vc[u];
            c.x = rescale_codes(c.x, fv); c.y = rescale_codes(c.y, fv);
            *reinterpret_cast<uint2 *>(a.mem.v + (base + t) * DH + col) = c;
            if (tid % TPR == 0) { a.mem.idx[base + t] = a.mem.idx[base + s]; a.mem.weight[base + t] = a.mem.weight[base + s]; }
        }
    }
}

}  // namespace full
}  // namespace lola
