// Sparse attention, device half of the C ABI (see include/ampd.h): the launches of each call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "api_host.h"
#include "sparse.h"

using namespace ampd;
using namespace ampd::host;

namespace {

// f(params' AppendParams, pages, most new tokens of a page) for every run of APPEND_MAX_REQS requests with new tokens
template <class F>
hipError_t for_page_rows(const ampd_kv_cache* c, const ampd_batch* b, AppendParams& a, F&& f) {
    std::memset(&a, 0, sizeof(a));
    a.k_pool = c->k_pool;
    a.v_pool = c->v_pool;
    a.k_scale = c->k_scale;
    a.v_scale = c->v_scale;
    a.block_table = b->d_block_table;
    a.Hkv = c->num_kv_heads;
    a.D = c->head_dim;
    a.P = c->page_size;
    a.logP = log2_exact(c->page_size);
    a.max_pages = b->max_pages_per_req;
    a.hn = c->num_kv_heads;
    int64_t row_off = 0;
    for (int r0 = 0; r0 < b->num_reqs; r0 += APPEND_MAX_REQS) {
        a.req0 = r0;
        a.n = std::min(APPEND_MAX_REQS, b->num_reqs - r0);
        int64_t pages = 0;
        int most = 0;
        for (int i = 0; i < a.n; ++i) {
            const int C = b->h_ctx_len[r0 + i], L = b->h_incr_len[r0 + i];
            a.rows[i] = AppendRow{C, L, (int32_t)row_off, (int32_t)pages};
            row_off += L;
            most = std::max(most, std::min(L, c->page_size));
            if (L > 0) pages += (C + L - 1) / c->page_size - C / c->page_size + 1;
        }
        if (pages == 0) continue;
        const hipError_t e = f(pages, most);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int kv_type(const ampd_kv_cache* c) { return c->kv_dtype == AMPD_KV_FP8_E4M3 ? KV_FP8 : KV_BF16; }

bool nothing_new(const ampd_batch* b) {
    for (int r = 0; r < b->num_reqs; ++r)
        if (b->h_incr_len[r] > 0) return false;
    return true;
}

bool aligned(const void* p, uintptr_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

extern "C" {

ampd_status ampd_rope_kv_append(const ampd_kv_cache* cache, const ampd_batch* batch, const ampd_rope* rope, const ampd_qkv_rows* rows,
                                void* q_out, const ampd_page_bounds* bounds, void* stream) {
    ampd_status vs = validate_rope(cache, batch, rope, rows, q_out);
    if (vs != AMPD_OK) return vs;
    if (bounds && (vs = validate_bounds(bounds)) != AMPD_OK) return vs;
    if (nothing_new(batch)) return AMPD_OK;
    RopeParams p;
    p.q = rows->q;
    p.q_out = q_out;
    p.q_stride = rows->q_stride * 2;
    p.k_stride = rows->k_stride * 2;
    p.v_stride = rows->v_stride * 2;
    p.inv_freq = rope->inv_freq;
    p.positions = rope->positions;
    p.codes = bounds ? bounds->codes : nullptr;
    p.bscale = bounds ? bounds->scale : nullptr;
    p.num_pages = cache->num_pages;
    p.Hq = cache->num_q_heads;
    p.rd = rope->rotary_dim;
    p.interleaved = rope->interleaved;
    p.scale = rope->scale;
    const hipError_t e = for_page_rows(cache, batch, p.a, [&](int64_t pages, int most) {
        p.a.k_new = rows->k;
        p.a.v_new = rows->v;
        return launch_rope(p, kv_type(cache), pages, most, static_cast<hipStream_t>(stream));
    });
    return e == hipSuccess ? AMPD_OK : AMPD_ERR_HIP;
}

ampd_status ampd_page_bounds_update(const ampd_kv_cache* cache, const ampd_batch* batch, const ampd_page_bounds* bounds, void* stream) {
    ampd_status vs = validate(cache, batch, true);
    if (vs != AMPD_OK) return vs;
    if ((vs = validate_bounds(bounds)) != AMPD_OK) return vs;
    BoundsParams p;
    p.codes = bounds->codes;
    p.bscale = bounds->scale;
    p.num_pages = cache->num_pages;
    const hipError_t e = for_page_rows(cache, batch, p.a, [&](int64_t pages, int) {
        return launch_bounds(p, kv_type(cache), pages, static_cast<hipStream_t>(stream));
    });
    return e == hipSuccess ? AMPD_OK : AMPD_ERR_HIP;
}

ampd_status ampd_select_pages(const ampd_kv_cache* cache, const ampd_batch* batch, const ampd_page_bounds* bounds, const ampd_page_selection* sel,
                              const void* q, int32_t* selected, void* workspace, size_t workspace_bytes, void* stream) {
    ampd_status vs = validate_select(cache, batch, sel);
    if (vs != AMPD_OK) return vs;
    if ((vs = validate_bounds(bounds)) != AMPD_OK) return vs;
    if (nothing_new(batch)) return AMPD_OK;
    if (!batch->d_block_table || !aligned(q, 16) || !aligned(selected, 4)) return AMPD_ERR_INVALID_ARG;
    SelectPlan plan;
    select_plan(cache, batch, sel, &plan);
    if (!aligned(workspace, 256) || workspace_bytes < (size_t)plan.bytes) return AMPD_ERR_WORKSPACE;
    SelectParams p;
    p.q = q;
    p.codes = bounds->codes;
    p.bscale = bounds->scale;
    p.block_table = batch->d_block_table;
    p.selected = selected;
    p.keys = static_cast<uint32_t*>(workspace);
    p.num_pages = cache->num_pages;
    p.Hq = cache->num_q_heads;
    p.Hkv = cache->num_kv_heads;
    p.P = cache->page_size;
    p.logP = log2_exact(cache->page_size);
    p.max_pages = batch->max_pages_per_req;
    p.budget = sel->budget;
    p.first = sel->first_pages;
    p.last = sel->last_pages;
    p.g = sel->group_tokens;
    auto launch = [&](const SelectLaunch& l) {
        p.qcodes = static_cast<int8_t*>(workspace) + l.code_offset();
        p.score_tiles = l.score_tiles;
        p.n = l.n;
        std::memcpy(p.rows, l.rows, l.n * sizeof(SelectRow));
        return launch_select(p, cache->head_dim, l.groups, l.score_blocks, l.codes, l.max_keys, static_cast<hipStream_t>(stream)) == hipSuccess ? AMPD_OK : AMPD_ERR_HIP;
    };
    return plan.launches == 1 ? launch(plan.only) : select_launches(cache, batch, sel, launch);
}

ampd_status ampd_sparse_attn(const ampd_kv_cache* cache, const ampd_batch* batch, const int32_t* selected, int32_t budget, int32_t group_tokens,
                             const void* q, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    ampd_status vs = validate(cache, batch, true);
    if (vs != AMPD_OK) return vs;
    if ((vs = validate_sparse(cache, batch, budget, group_tokens)) != AMPD_OK) return vs;
    if (nothing_new(batch)) return AMPD_OK;
    if (!aligned(selected, 4) || !aligned(q, 16) || !aligned(out, 16)) return AMPD_ERR_INVALID_ARG;
    SparsePlan plan;
    sparse_plan(cache, batch, budget, group_tokens, &plan);
    if (!aligned(workspace, 256) || workspace_bytes < (size_t)plan.bytes) return AMPD_ERR_WORKSPACE;
    SparseParams p;
    p.q = q;
    p.out = out;
    p.k_pool = cache->k_pool;
    p.v_pool = cache->v_pool;
    p.k_scale = cache->k_scale;
    p.v_scale = cache->v_scale;
    p.block_table = batch->d_block_table;
    p.partial = static_cast<float*>(workspace);
    p.num_pages = cache->num_pages;
    p.Hq = cache->num_q_heads;
    p.Hkv = cache->num_kv_heads;
    p.P = cache->page_size;
    p.logP = log2_exact(cache->page_size);
    p.max_pages = batch->max_pages_per_req;
    p.budget = budget;
    p.g = group_tokens;
    p.c_log2 = cache->softmax_scale * 1.44269504088896340736f;
    auto launch = [&](const SparseLaunch& l) {
        p.selected = selected + l.group0 * cache->num_kv_heads * budget;
        p.tiles = l.tiles;
        p.splits = l.splits;
        p.chunk = l.chunk;
        p.n = l.n;
        std::memcpy(p.rows, l.rows, l.n * sizeof(SparseRow));
        return launch_sparse(p, cache->head_dim, kv_type(cache), l.groups, l.waves, static_cast<hipStream_t>(stream)) == hipSuccess ? AMPD_OK : AMPD_ERR_HIP;
    };
    return plan.launches == 1 ? launch(plan.only) : sparse_launches(cache, batch, budget, group_tokens, launch);
}

}  // extern "C"
