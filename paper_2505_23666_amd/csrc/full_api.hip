// C ABI of the 8-bit full-context cache (include/lola.h, lola_full_*): host-side validation, workspace carving and kernel
// dispatch.  Nothing here allocates or synchronises.
#include "../../include/lola.h"
#include <algorithm>
#include <math.h>
#include "full_prompt.h"

using namespace lola;
using namespace lola::full;

namespace {

constexpr size_t ALIGN = 256;
inline size_t up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
inline int bytes_of(int32_t dtype) { return dtype == LOLA_F32 ? 4 : 2; }
inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
#define LAUNCH_CHECK() do { if (hipGetLastError() != hipSuccess) return LOLA_ERR_HIP; } while (0)

lola_status check_config(const lola_full_config *c) {
    if (!c) return LOLA_ERR_NULL;
    if (c->dtype != LOLA_F32 && c->dtype != LOLA_BF16) return LOLA_ERR_DTYPE;
    if (c->out_dtype != LOLA_F32 && c->out_dtype != LOLA_BF16) return LOLA_ERR_DTYPE;
    if (c->batch < 1 || c->n_kv_heads < 1 || c->n_q_heads < c->n_kv_heads || c->n_q_heads % c->n_kv_heads) return LOLA_ERR_SHAPE;
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return LOLA_ERR_SHAPE;
    if (c->capacity < LOLA_FULL_BLOCK || c->capacity % LOLA_FULL_BLOCK || c->capacity > (1 << 26)) return LOLA_ERR_SHAPE;
    // streams index the y dimension of some launch grids (limit 65535)
    if ((long long)c->batch * c->n_kv_heads > 65535 || c->n_q_heads > 65535) return LOLA_ERR_SHAPE;
    if (c->tokens_first != 0 && c->tokens_first != 1) return LOLA_ERR_SHAPE;
    return LOLA_OK;
}

lola_status check_state(const lola_full_state *st) {
    if (!st || !st->k || !st->v || !st->k_scale || !st->v_scale || !st->idx || !st->count || !st->n_tokens) return LOLA_ERR_NULL;
    const void *ps[] = {st->k, st->v, st->k_scale, st->v_scale, st->idx, st->weight, st->count, st->n_tokens};
    for (const void *p : ps) if (p && misaligned(p)) return LOLA_ERR_ALIGN;
    return LOLA_OK;
}

// (2^30 query rows in all are 2^23 workgroups of the prompt kernel and 2^31 threads of one grid dimension)
bool rows_ok(const lola_full_config *c, int32_t T) {
    return T >= 0 && (long long)T * (c->n_q_heads / c->n_kv_heads) <= (1 << 24) && (long long)T * c->batch * c->n_q_heads <= (1ll << 30);
}

Mem make_mem(const lola_full_state *st) {
    return Mem{st->k, st->v, st->k_scale, st->v_scale, st->idx, st->weight, st->count, st->n_tokens};
}

Args make_args(const lola_full_config *c, const lola_full_state *st, int32_t T, const int32_t *lens) {
    Args a = {};
    a.mem = make_mem(st);
    a.B = c->batch; a.Hq = c->n_q_heads; a.Hkv = c->n_kv_heads; a.g = a.Hq / a.Hkv;
    a.d = c->head_dim; a.cap = c->capacity; a.nblk = a.cap / BLK; a.T = T;
    a.lens = lens;
    const int64_t d = a.d;
    a.q_sb = (int64_t)a.Hq * T * d; a.k_sb = (int64_t)a.Hkv * T * d;
    a.q_sh = c->tokens_first ? d : T * d; a.q_st = c->tokens_first ? a.Hq * d : d;
    a.k_sh = a.q_sh; a.k_st = c->tokens_first ? a.Hkv * d : d;
    a.scale2 = (c->softmax_scale > 0.f ? c->softmax_scale : 1.0f / sqrtf((float)c->head_dim)) * LOG2E_F;
    return a;
}

constexpr int CHIP_CUS = 256;      // compute units of the MI355X
// rows (query heads of a group x tokens) that the step kernel takes: two column tiles of 16, one where the head is 256 wide (two
// would need more registers than there are)
inline size_t step_rows(int head_dim) { return head_dim == 256 ? 16 : 32; }

constexpr int PROMPT_NW = 4;       // wavefronts (of 32 rows) per workgroup of the prompt kernel

struct AttendPlan {
    bool step, wide, span;    // wide: one workgroup of eight wavefronts has all of a stream; span: the blocks' index ranges are taken beforehand
    int nsplit, ntiles;
    size_t off_stat, off_o, off_ml, off_logit, off_counts, off_span, bytes;
};
AttendPlan plan_attend(const lola_full_config *c, int32_t T, int32_t gather) {
    const size_t S = (size_t)c->batch * c->n_kv_heads, R = (size_t)T * (c->n_q_heads / c->n_kv_heads);
    AttendPlan p = {};
    p.step = R <= step_rows(c->head_dim);
    size_t off = 0;
    if (p.step) {
        // Two workgroups per compute unit (8 streams of 128 Ki pairs at d = 128 54.4 us a step with the join, 56.9 with four; 8 of 32 Ki 19.8 and 22.6; but 128
        // streams of unequal lengths up to 8192 with weights 61.7 and 60.3).  All run at once in the forms that these figures are of: one token, up to 16 rows,
        // d up to 128, bf16 storage or outputs.  The registers of others leave room for one (fp32 storage and outputs at d = 128, several tokens at d = 128,
        // more than 16 rows at d = 128 and, with several tokens or fp32 storage, at d = 64; d = 256): half of those shares wait for the others.  Shares have about 8192
        // slots (sequences of unequal lengths), 16320 at most: 255 blocks, STEP_BLOCKS for each of four wavefronts; each wavefront has a block at least when the cache is full.
        const size_t most = ((size_t)c->capacity / BLK + 3) / 4;
        p.nsplit = (int)std::max((size_t)1, std::min(most, std::max((2 * CHIP_CUS + S - 1) / S, (size_t)c->capacity / 8192)));
        static_assert(2 * 8192 / BLK <= 4 * STEP_BLOCKS, "a share of less than twice 8192 slots");
        // One workgroup of eight wavefronts per stream, and no join, where the streams fill the chip (256 streams of 4096 pairs at
        // d = 128 46 us a step, 50 in four shares each; 512 streams 105 and 108; but 128 streams of up to 8192 pairs 80 and 66) or the cache is
        // short (8 streams of 512 slots at d = 64 5.7 us, joined 7.0; but 1024 slots 7.1 and 6.8).
        p.wide = R <= 16 && c->head_dim < 256 && (c->capacity <= 512 || (S >= CHIP_CUS && c->capacity <= 8192));
        if (p.wide) p.nsplit = 1;
        p.off_o = off; if (p.nsplit > 1) off += up(S * p.nsplit * R * c->head_dim * 4);
        p.off_ml = off; if (p.nsplit > 1 || gather) off += up(S * p.nsplit * R * 2 * 4);
        p.off_logit = off; if (gather) off += up(S * R * c->capacity * 4);
        p.off_counts = off; if (gather) off += up(S * 4);
    } else {
        p.ntiles = (int)((R + 32 * PROMPT_NW - 1) / (32 * PROMPT_NW));
        // two workgroups fit a compute unit (one with fp32 queries at d = 128, and at d = 256); fewer are split over the blocks, four blocks each at least when the cache is full
        const size_t wgs = S * p.ntiles, most = std::max((size_t)1, (size_t)c->capacity / BLK / 4);
        p.nsplit = (int)(wgs >= 2 * CHIP_CUS ? 1 : std::min(most, (2 * CHIP_CUS + wgs - 1) / wgs));
        // (a launch of its own, 3 us, against 16 loads per lane in every workgroup: at 5 blocks a call of 27 us takes 23 without it, at 64
        // blocks and 4096 workgroups one of 649 us takes 659)
        p.span = gather || c->capacity / BLK > 16;
        p.off_span = off; if (p.span) off += up(S * (c->capacity / BLK) * 8);
        p.off_o = off; if (p.nsplit > 1) off += up(S * p.nsplit * R * c->head_dim * 4);
        p.off_ml = off; if (p.nsplit > 1) off += up(S * p.nsplit * R * 2 * 4);
        p.off_stat = off; if (gather) off += up(S * R * 8);
    }
    p.bytes = off;
    return p;
}

struct EvictPlan {
    size_t off_dst, off_src, off_before, off_edge, bytes;
    int most, nkb;
};
EvictPlan plan_evict(const lola_full_config *c, int32_t keep) {
    const size_t S = (size_t)c->batch * c->n_kv_heads;
    EvictPlan p;
    p.most = std::min(keep, c->capacity - keep);
    p.nkb = (keep + BLK - 1) / BLK;
    size_t off = 0;
    p.off_dst = off; off += up(S * p.most * 4);
    p.off_src = off; off += up(S * p.most * 4);
    p.off_before = off; off += up(S * ((size_t)p.nkb + 1) * 4);
    p.off_edge = off; off += up(S * 2 * 4);
    p.bytes = off;
    return p;
}
// an eviction to any budget: at most capacity / 2 pairs move, at most all blocks receive some
size_t evict_bytes(const lola_full_config *c) {
    const size_t S = (size_t)c->batch * c->n_kv_heads;
    return 2 * up(S * (c->capacity / 2) * 4) + up(S * ((size_t)c->capacity / BLK + 1) * 4) + up(S * 2 * 4);
}

template <typename TI>
lola_status run_append(const Args &a, hipStream_t stream) {
    // Blocks that T tokens may fall into.  One workgroup has all of a stream's, and moves the counters on itself, where they are at most two, or
    // eight of short rows, four at a time (a prompt of 257 tokens, append and attention, 4 streams of 32 fp32 columns 20.5 us, 24.3 with a workgroup per
    // block and a second launch; but 64 streams of 333 tokens of 128 bf16 columns 39.8 and 37.0).  (Grid y is limited to 65535.)
    const int w = (int)(((int64_t)a.T + 2 * BLK - 2) / BLK);
    const bool four = w > 2 && w <= 8 && a.d * sizeof(TI) <= 128;
    const int per = w <= 2 || four ? w : (w + 32767) / 32768, adv = per == w;
    const dim3 grid(a.B * a.Hkv, (w + per - 1) / per);
#define APPEND(DH, G) hipLaunchKernelGGL((append_kernel<DH, TI, G>), grid, dim3(256 * G), 0, stream, a, per, adv)
    if (four) {
        if (a.d == 32) APPEND(32, 4);
        else if constexpr (sizeof(TI) == 2) APPEND(64, 4);
    } else switch (a.d) {
        case 32: APPEND(32, 1); break;
        case 64: APPEND(64, 1); break;
        case 128: APPEND(128, 1); break;
        default: APPEND(256, 1); break;
    }
#undef APPEND
    LAUNCH_CHECK();
    if (!adv) {
        hipLaunchKernelGGL(advance_kernel, dim3((a.B * a.Hkv + 255) / 256), dim3(256), 0, stream, a);
        LAUNCH_CHECK();
    }
    return LOLA_OK;
}

template <int DH, typename TI, typename TO>
lola_status launch_attend(const Args &a, const AttendPlan &p, int gather, char *ws, hipStream_t stream) {
    const bool fused = a.k != nullptr;     // a generation step whose token the step kernel puts into the cache
    if (p.step) {
        StepArgs sa;
        sa.a = a; sa.nsplit = p.nsplit;
        sa.part_o = p.nsplit > 1 ? (float *)(ws + p.off_o) : nullptr;
        sa.part_ml = p.nsplit > 1 || gather ? (float *)(ws + p.off_ml) : nullptr;
        sa.logit = gather ? (float *)(ws + p.off_logit) : nullptr;
        sa.append = fused && sa.part_ml;
        sa.counts = fused && gather ? (int32_t *)(ws + p.off_counts) : nullptr;
        const int S = a.B * a.Hkv, R = a.T * a.g;
        const dim3 grid(S, p.nsplit);
#define STEP(CT, NW, M, AP) hipLaunchKernelGGL((step_kernel<DH, CT, NW, TI, TO, M, AP>), grid, dim3(64 * NW), 0, stream, sa)
#define STEP3(CT, NW) if (fused) STEP(CT, NW, false, true); else if (a.T > 1) STEP(CT, NW, true, false); else STEP(CT, NW, false, false)
        if constexpr (DH < 256) {
            if (p.wide) { STEP3(1, 8); }
            else if (R <= 16) { STEP3(1, 4); }
            else { STEP3(2, 4); }
        } else { STEP3(1, 4); }
#undef STEP3
#undef STEP
        LAUNCH_CHECK();
        const int jo = p.nsplit > 1 ? R : 0, jw = gather ? std::min((a.cap + 1023) / 1024, 4096) : 0;
        if (jo + jw) {
            hipLaunchKernelGGL((step_join_kernel<DH, TO>), dim3(S, jo + jw), dim3(256), 0, stream, sa, jo);
            LAUNCH_CHECK();
        }
        return LOLA_OK;
    }
    PromptArgs pa;
    pa.a = a; pa.nsplit = p.nsplit; pa.ntiles = p.ntiles;
    pa.span = p.span ? (int2 *)(ws + p.off_span) : nullptr;
    pa.part_o = p.nsplit > 1 ? (float *)(ws + p.off_o) : nullptr;
    pa.part_ml = p.nsplit > 1 ? (float *)(ws + p.off_ml) : nullptr;
    pa.stat = gather ? (float2 *)(ws + p.off_stat) : nullptr;
    const int S = a.B * a.Hkv, R = a.T * a.g;
    constexpr int LDS = 4 * BLK * DH * 2 + 2 * BLK * 4;
    if (p.span) {
        hipLaunchKernelGGL(span_kernel, dim3(std::min((a.nblk + 3) / 4, 256), S), dim3(256), 0, stream, pa);
        LAUNCH_CHECK();
    }
    hipLaunchKernelGGL((prompt_kernel<DH, PROMPT_NW, TI, TO>), dim3((unsigned)S * p.ntiles * p.nsplit), dim3(64 * PROMPT_NW), LDS, stream, pa);
    LAUNCH_CHECK();
    if (p.nsplit > 1) {
        constexpr int RPW = 1024 / DH;      // rows per workgroup
        hipLaunchKernelGGL((prompt_join_kernel<DH, TO>), dim3((R + RPW - 1) / RPW, S), dim3(256), 0, stream, pa);
        LAUNCH_CHECK();
    }
    if (gather) {
        // (a grid of 2^22 workgroups at most; each then takes several blocks)
        const int nj = std::min(a.nblk, std::max(1, (1 << 22) / S));
        hipLaunchKernelGGL((prompt_gather_kernel<DH, TI>), dim3((unsigned)S * nj), dim3(256), 0, stream, pa);
        LAUNCH_CHECK();
    }
    return LOLA_OK;
}

template <typename TI, typename TO>
lola_status run_attend(const Args &a, const AttendPlan &p, int gather, char *ws, hipStream_t stream) {
    switch (a.d) {
        case 32: return launch_attend<32, TI, TO>(a, p, gather, ws, stream);
        case 64: return launch_attend<64, TI, TO>(a, p, gather, ws, stream);
        case 128: return launch_attend<128, TI, TO>(a, p, gather, ws, stream);
        default: return launch_attend<256, TI, TO>(a, p, gather, ws, stream);
    }
}

// k, v: NULL, or a token per sequence that the step kernel puts into the cache first (plans with p.step, T = 1)
lola_status attend(const lola_full_config *c, const lola_full_state *st, const void *q, const void *k, const void *v, const int32_t *lens,
                   int32_t T, int32_t gather, void *out, void *workspace, hipStream_t stream) {
    Args a = make_args(c, st, T, lens);
    a.q = q; a.k = k; a.v = v; a.out = out;
    const AttendPlan p = plan_attend(c, T, gather);
    char *ws = (char *)workspace;
    const bool bo = c->out_dtype == LOLA_BF16;
    if (c->dtype == LOLA_F32) return bo ? run_attend<float, bf16_t>(a, p, gather, ws, stream) : run_attend<float, float>(a, p, gather, ws, stream);
    return bo ? run_attend<bf16_t, bf16_t>(a, p, gather, ws, stream) : run_attend<bf16_t, float>(a, p, gather, ws, stream);
}

lola_status append(const lola_full_config *c, const lola_full_state *st, const void *k, const void *v, const int32_t *lens, int32_t T,
                   hipStream_t stream) {
    Args a = make_args(c, st, T, lens);
    a.k = k; a.v = v;
    return c->dtype == LOLA_F32 ? run_append<float>(a, stream) : run_append<bf16_t>(a, stream);
}

lola_status check_attend(const lola_full_config *c, const lola_full_state *st, const void *q, int32_t T, int32_t gather, const void *out,
                         const void *workspace, size_t workspace_bytes) {
    if (!q || !out || (gather && !st->weight)) return LOLA_ERR_NULL;
    if (misaligned(q) || misaligned(out) || (workspace && misaligned(workspace))) return LOLA_ERR_ALIGN;
    const size_t need = plan_attend(c, T, gather).bytes;
    if (need && (!workspace || workspace_bytes < need)) return LOLA_ERR_WORKSPACE;
    return LOLA_OK;
}

// Every row's output is written by the workgroup that alone reads its query, after that, or by a later launch: outputs may lie in the queries' place.  Not so
// where the weights of many rows are gathered, whose kernel reads the queries again.  k, v: NULL, or a step's token.
lola_status check_overlap(const lola_full_config *c, const void *q, const void *k, const void *v, int32_t T, int32_t gather, const void *out) {
    auto overlap = [&](const void *x, int heads) {
        const uintptr_t a = (uintptr_t)x, o = (uintptr_t)out, row = (uintptr_t)c->batch * T * c->head_dim;
        return a < o + row * c->n_q_heads * bytes_of(c->out_dtype) && o < a + row * heads * bytes_of(c->dtype);
    };
    if (overlap(q, c->n_q_heads) && (q != out || c->dtype != c->out_dtype || (gather && !plan_attend(c, T, gather).step))) return LOLA_ERR_UNSUPPORTED;
    if (k && (overlap(k, c->n_kv_heads) || overlap(v, c->n_kv_heads))) return LOLA_ERR_UNSUPPORTED;
    return LOLA_OK;
}

}  // namespace

extern "C" {

size_t lola_full_state_bytes(const lola_full_config *c, size_t field_bytes[8]) {
    if (check_config(c) != LOLA_OK) { if (field_bytes) std::fill(field_bytes, field_bytes + 8, (size_t)0); return 0; }
    const size_t S = (size_t)c->batch * c->n_kv_heads, cap = c->capacity, codes = S * cap * c->head_dim, nb = S * (cap / BLK) * 4;
    const size_t fb[8] = {codes, codes, nb, nb, S * cap * 4, S * cap * 4, S * 4, S * 8};
    size_t total = 0;
    for (int i = 0; i < 8; i++) { total += fb[i]; if (field_bytes) field_bytes[i] = fb[i]; }
    return total;
}

size_t lola_full_workspace_bytes(const lola_full_config *c, int32_t T, int32_t gather) {
    if (check_config(c) != LOLA_OK || !rows_ok(c, T) || (gather != 0 && gather != 1)) return 0;
    return std::max(plan_attend(c, T, gather).bytes, evict_bytes(c));
}

lola_status lola_full_init(const lola_full_config *c, const lola_full_state *st, void *stream) {
    lola_status rc = check_config(c);
    if (rc != LOLA_OK) return rc;
    rc = check_state(st);
    if (rc != LOLA_OK) return rc;
    const int S = c->batch * c->n_kv_heads;
    hipLaunchKernelGGL(init_kernel, dim3((S + 255) / 256), dim3(256), 0, (hipStream_t)stream, st->count, st->n_tokens, S);
    LAUNCH_CHECK();
    return LOLA_OK;
}

lola_status lola_full_append(const lola_full_config *c, const lola_full_state *st, const void *k, const void *v,
                             const int32_t *lens, int32_t T, void *stream) {
    lola_status rc = check_config(c);
    if (rc != LOLA_OK) return rc;
    rc = check_state(st);
    if (rc != LOLA_OK) return rc;
    if (!rows_ok(c, T)) return LOLA_ERR_SHAPE;
    if (T == 0) return LOLA_OK;   // nothing to read or write: the token pointers are not looked at
    if (!k || !v) return LOLA_ERR_NULL;
    if (misaligned(k) || misaligned(v) || (lens && misaligned(lens))) return LOLA_ERR_ALIGN;
    return append(c, st, k, v, lens, T, (hipStream_t)stream);
}

lola_status lola_full_attend(const lola_full_config *c, const lola_full_state *st, const void *q, const int32_t *lens,
                             int32_t T, int32_t gather, void *out, void *workspace, size_t workspace_bytes, void *stream) {
    lola_status rc = check_config(c);
    if (rc != LOLA_OK) return rc;
    rc = check_state(st);
    if (rc != LOLA_OK) return rc;
    if (!rows_ok(c, T) || (gather != 0 && gather != 1)) return LOLA_ERR_SHAPE;
    if (T == 0) return LOLA_OK;
    rc = check_attend(c, st, q, T, gather, out, workspace, workspace_bytes);
    if (rc != LOLA_OK) return rc;
    if (lens && misaligned(lens)) return LOLA_ERR_ALIGN;
    rc = check_overlap(c, q, nullptr, nullptr, T, gather, out);
    if (rc != LOLA_OK) return rc;
    return attend(c, st, q, nullptr, nullptr, lens, T, gather, out, workspace, (hipStream_t)stream);
}

lola_status lola_full_step(const lola_full_config *c, const lola_full_state *st, const void *q, const void *k, const void *v,
                           int32_t gather, void *out, void *workspace, size_t workspace_bytes, void *stream) {
    lola_status rc = check_config(c);
    if (rc != LOLA_OK) return rc;
    rc = check_state(st);
    if (rc != LOLA_OK) return rc;
    if (!rows_ok(c, 1) || (gather != 0 && gather != 1)) return LOLA_ERR_SHAPE;
    if (!k || !v) return LOLA_ERR_NULL;
    rc = check_attend(c, st, q, 1, gather, out, workspace, workspace_bytes);
    if (rc != LOLA_OK) return rc;
    if (misaligned(k) || misaligned(v)) return LOLA_ERR_ALIGN;
    rc = check_overlap(c, q, k, v, 1, gather, out);
    if (rc != LOLA_OK) return rc;
    if (plan_attend(c, 1, gather).step) return attend(c, st, q, k, v, nullptr, 1, gather, out, workspace, (hipStream_t)stream);
    rc = append(c, st, k, v, nullptr, 1, (hipStream_t)stream);      // more query heads per kv head than the step kernel takes
    if (rc != LOLA_OK) return rc;
    return attend(c, st, q, nullptr, nullptr, nullptr, 1, gather, out, workspace, (hipStream_t)stream);
}

lola_status lola_full_evict(const lola_full_config *c, const lola_full_state *st, int32_t keep, int32_t first, int32_t recent,
                            void *workspace, size_t workspace_bytes, void *stream) {
    lola_status rc = check_config(c);
    if (rc != LOLA_OK) return rc;
    rc = check_state(st);
    if (rc != LOLA_OK) return rc;
    if (keep < 0 || keep > c->capacity || first < 0 || recent < 0 || (long long)first + recent > keep) return LOLA_ERR_SHAPE;
    if (!st->weight) return LOLA_ERR_NULL;
    if (workspace && misaligned(workspace)) return LOLA_ERR_ALIGN;
    if (keep == c->capacity) return LOLA_OK;   // no stream holds more
    const EvictPlan p = plan_evict(c, keep);
    if (!workspace || workspace_bytes < p.bytes) return LOLA_ERR_WORKSPACE;
    EvictArgs a = {};
    a.mem = make_mem(st);
    a.cap = c->capacity; a.nblk = a.cap / BLK; a.keep = keep; a.first = first; a.recent = recent; a.d = c->head_dim;
    char *ws = (char *)workspace;
    a.dst = (int32_t *)(ws + p.off_dst); a.src = (int32_t *)(ws + p.off_src); a.before = (int32_t *)(ws + p.off_before);
    a.edge = (float *)(ws + p.off_edge);
    a.most = p.most; a.nkb = p.nkb;
    const int S = c->batch * c->n_kv_heads;
    const int lds = a.cap <= RANKS_LDS ? a.cap * 4 : 0;
#define BY_DIM(K) (a.d == 32 ? K<32> : a.d == 64 ? K<64> : a.d == 128 ? K<128> : K<256>)
    // Short caches from which at most 512 pairs can move: the whole eviction of a stream in one workgroup (with the append of a
    // turn, 16 sequences of the 8B shape with a budget of 2048 pairs 22.7 us, 24.5 by the kernels below as both were then; 128 of the 1B shape with 1111 23.8 and 28.8).
    if (a.cap <= 8192 && a.most <= 512) {
        hipLaunchKernelGGL(BY_DIM(evict_few_kernel), dim3(S), dim3(256), lds + (2 * a.most + 3 * a.nkb) * 4, (hipStream_t)stream, a);
        LAUNCH_CHECK();
        return LOLA_OK;
    }
    // (up to 8192 slots in workgroups of 256, of which more fit a compute unit)
    if (a.cap <= 8192) hipLaunchKernelGGL((evict_select_kernel<256>), dim3(S), dim3(256), lds, (hipStream_t)stream, a);
    else hipLaunchKernelGGL((evict_select_kernel<1024>), dim3(S), dim3(1024), lds, (hipStream_t)stream, a);
    LAUNCH_CHECK();
    if (p.nkb == 0) return LOLA_OK;
    hipLaunchKernelGGL(BY_DIM(evict_move_kernel), dim3(p.nkb, S), dim3(256), 0, (hipStream_t)stream, a);
#undef BY_DIM
    LAUNCH_CHECK();
    return LOLA_OK;
}

}  // extern "C"
