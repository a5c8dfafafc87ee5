// Sparse attention, host half: argument validation, how a call is cut into launches, workspace sizes.  Nothing here includes or calls HIP.
#include "sparse.h"

#include <algorithm>
#include <cmath>

#include "api_host.h"

namespace ampd {
namespace host {

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

ampd_status validate_rope(const ampd_kv_cache* c, const ampd_batch* b, const ampd_rope* rope, const ampd_qkv_rows* rows, const void* q_out) {
    const ampd_status vs = validate(c, b, true);
    if (vs != AMPD_OK) return vs;
    if (!rope || !rows || rope->reserved != 0) return AMPD_ERR_INVALID_ARG;
    if (rope->interleaved != 0 && rope->interleaved != 1) return AMPD_ERR_INVALID_ARG;
    if (!(rope->scale > 0.0f) || !std::isfinite(rope->scale)) return AMPD_ERR_INVALID_ARG;
    if (rope->rotary_dim < 16 || rope->rotary_dim > c->head_dim || rope->rotary_dim % 16 != 0) return AMPD_ERR_UNSUPPORTED;
    int64_t sumL = 0;
    for (int r = 0; r < b->num_reqs; ++r) sumL += b->h_incr_len[r];
    if (sumL == 0) return AMPD_OK;
    if (!rope->inv_freq || !rows->k || !rows->v || (rows->q && !q_out)) return AMPD_ERR_INVALID_ARG;
    const int64_t q_row = (int64_t)c->num_q_heads * c->head_dim, kv_row = (int64_t)c->num_kv_heads * c->head_dim;
    const struct {
        const void* p;
        int64_t stride, row;
    } in[3] = {{rows->k, rows->k_stride, kv_row}, {rows->v, rows->v_stride, kv_row}, {rows->q, rows->q_stride, q_row}};
    for (const auto& x : in) {
        if (!x.p) continue;
        if (!aligned16(x.p) || x.stride < x.row || x.stride % 8 != 0 || x.stride > (int64_t)1 << 40) return AMPD_ERR_INVALID_ARG;
    }
    if (rows->q && !aligned16(q_out)) return AMPD_ERR_INVALID_ARG;
    if (rows->q && rows->q == q_out && rows->q_stride != q_row) return AMPD_ERR_INVALID_ARG;
    return AMPD_OK;
}

ampd_status validate_bounds(const ampd_page_bounds* bounds) {
    if (!bounds || !bounds->codes || !bounds->scale || !aligned16(bounds->codes)) return AMPD_ERR_INVALID_ARG;
    return AMPD_OK;
}

static ampd_status validate_group(const ampd_kv_cache* c, int32_t budget, int32_t group_tokens) {
    if (budget < 1 || group_tokens < 1) return AMPD_ERR_INVALID_ARG;
    if ((int64_t)group_tokens * (c->num_q_heads / c->num_kv_heads) > SPARSE_MAX_ROWS) return AMPD_ERR_UNSUPPORTED;
    if ((int64_t)budget * c->page_size > (int64_t)1 << 29) return AMPD_ERR_UNSUPPORTED;
    return AMPD_OK;
}

ampd_status validate_select(const ampd_kv_cache* c, const ampd_batch* b, const ampd_page_selection* s) {
    ampd_status vs = validate(c, b, false);
    if (vs != AMPD_OK) return vs;
    if (!s) return AMPD_ERR_INVALID_ARG;
    for (int i = 0; i < 4; ++i)
        if (s->reserved[i] != 0) return AMPD_ERR_INVALID_ARG;
    vs = validate_group(c, s->budget, s->group_tokens);
    if (vs != AMPD_OK) return vs;
    if (s->first_pages < 0 || s->last_pages < 1) return AMPD_ERR_INVALID_ARG;
    const int64_t always = (int64_t)s->first_pages + s->last_pages + (s->group_tokens - 1 + c->page_size - 1) / c->page_size;
    return s->budget < always ? AMPD_ERR_INVALID_ARG : AMPD_OK;
}

ampd_status validate_sparse(const ampd_kv_cache* c, const ampd_batch* b, int32_t budget, int32_t group_tokens) {
    const ampd_status vs = validate(c, b, false);
    return vs != AMPD_OK ? vs : validate_group(c, budget, group_tokens);
}

ampd_status select_launches(const ampd_kv_cache* c, const ampd_batch* b, const ampd_page_selection* s, LaunchFn<SelectLaunch> f) {
    const int P = c->page_size, logP = log2_exact(P), g = s->group_tokens, Hkv = c->num_kv_heads;
    const int64_t most_groups = std::max<int64_t>(1, (1 << 21) / Hkv);        // a grid holds fewer than 2^32 threads
    const int64_t code_words = (int64_t)Hkv * c->head_dim;                    // of a group
    SelectLaunch l;
    bool many = false;                                                        // some row of the launch has more than one group
    ampd_status st = AMPD_OK;
    // pages that the last group of a row may choose by score (its other groups: no more), or 0 if it takes all it has
    auto scored = [&](const SelectRow& x) -> int64_t {
        const int64_t tok0 = (groups_of(x.L, g) - 1) * g, lp0 = (x.C + tok0) >> logP, lp1 = ((int64_t)x.C + x.L - 1) >> logP, end = lp0 - s->last_pages + 1;
        return end > s->first_pages && lp1 + 1 > s->budget ? end : 0;
    };
    auto flush = [&]() {
        int64_t tiles = 0;
        l.codes = false;
        for (int i = 0; i < l.n; ++i) l.codes |= l.keys > 0 && l.rows[i].L > g;
        for (int i = 0; i < l.n; ++i) tiles += (groups_of(l.rows[i].L, g) + 15) / 16 * ((scored(l.rows[i]) + 15) / 16) * Hkv;
        l.score_tiles = score_tiles(tiles);
        const int per = score_pages(Hkv, l.score_tiles);
        for (int i = 0; i < l.n; ++i) {
            l.rows[i].tile0 = l.score_blocks;
            l.score_blocks += (int)((groups_of(l.rows[i].L, g) + 15) / 16 * ((scored(l.rows[i]) + per - 1) / per));
        }
        if (l.n > 0 && st == AMPD_OK) st = f(l);
        l.n = l.groups = l.score_blocks = 0;
        l.keys = l.max_keys = 0;
        many = false;
    };
    int64_t row_off = 0, out0 = 0;
    for (int r = 0; r < b->num_reqs && st == AMPD_OK; ++r) {
        const int64_t C = b->h_ctx_len[r], L = b->h_incr_len[r], groups = groups_of(L, g);
        for (int64_t at = 0; at < groups && st == AMPD_OK;) {
            SelectRow x;
            x.C = (int32_t)(C + at * g);
            x.L = (int32_t)(L - at * g);
            // words that the launch holds with this row in it, and that each of the row's groups adds
            const bool scores = scored(x) > 0, codes = (l.keys > 0 || scores) && (many || groups - at > 1);
            const int64_t per_group = (scores ? Hkv * key_stride(C + L, P) : 0) + (codes ? code_words : 0);
            const int64_t used = l.keys + (codes ? l.groups * code_words : 0);
            if (l.n == SELECT_MAX_REQS || l.groups == most_groups || (l.n > 0 && used + per_group > SELECT_WORDS)) {
                flush();
                if (st != AMPD_OK) break;
                continue;
            }
            const int64_t room = per_group > 0 ? std::max<int64_t>(1, (SELECT_WORDS - used) / per_group) : groups;
            const int64_t take = std::min({groups - at, most_groups - l.groups, room});
            x.L = (int32_t)std::min(L - at * g, take * g);
            x.row_off = (int32_t)(row_off + at * g);
            x.req = r;
            x.out0 = (int32_t)(out0 + at);
            x.item0 = l.groups;
            x.tile0 = 0;
            x.key0 = (uint32_t)(l.keys / 64);
            many |= take > 1;
            l.groups += (int)take;
            if (const int64_t end = scored(x)) {
                l.max_keys = std::max(l.max_keys, end - s->first_pages);
                l.keys += take * Hkv * key_stride((int64_t)x.C + x.L, P);
            }
            l.rows[l.n++] = x;
            at += take;
        }
        row_off += L;
        out0 += groups;
    }
    flush();
    return st;
}

void select_plan(const ampd_kv_cache* c, const ampd_batch* b, const ampd_page_selection* s, SelectPlan* out) {
    out->bytes = 256;
    select_launches(c, b, s, [&](const SelectLaunch& l) {
        // (a group's codes at least, also where no launch makes any)
        out->bytes = std::max(out->bytes, l.code_offset() + (l.codes ? l.groups : 1) * (int64_t)c->num_kv_heads * 4 * c->head_dim);
        if (out->launches++ == 0) out->only = l;
        return AMPD_OK;
    });
}

void sparse_plan(const ampd_kv_cache* c, const ampd_batch* b, int32_t budget, int32_t g, SparsePlan* out) {
    int64_t floats = 0;
    sparse_launches(c, b, budget, g, [&](const SparseLaunch& l) {
        floats = std::max(floats, l.partial_floats);
        if (out->launches++ == 0) out->only = l;
        return AMPD_OK;
    });
    out->bytes = std::max<int64_t>(256, floats * 4);
}

ampd_status sparse_launches(const ampd_kv_cache* c, const ampd_batch* b, int32_t budget, int32_t g, LaunchFn<SparseLaunch> f) {
    const int Hkv = c->num_kv_heads, rows = g * (c->num_q_heads / Hkv), tile = sparse_tile(rows), tiles = (rows + tile - 1) / tile;
    const int64_t most_groups = std::max<int64_t>(1, (1 << 22) / ((int64_t)Hkv * tiles));     // a grid holds fewer than 2^32 threads
    const int64_t keys = (int64_t)budget * c->page_size;
    SparseLaunch l;
    ampd_status st = AMPD_OK;
    auto flush = [&](int64_t next) {
        if (l.n > 0 && st == AMPD_OK) {
            l.tiles = tiles;
            // Two workgroups of 4 waves to a CU fill the chip.  Half as many items, down to one for every other CU, go as workgroups of 8 waves
            // (200 lists of 2 048 keys, 8 bits, d = 64: 16.0 us instead of 16.6 in two pieces and 4.0 for the join); fewer are cut into pieces, of a
            // block of 32 keys per wave at least.
            const int64_t items = (int64_t)l.groups * tiles * Hkv;
            l.waves = items >= 128 && items <= 256 ? 8 : 4;
            const int64_t want = l.waves == 8 ? 1 : std::max<int64_t>(1, 512 / items), least = l.waves * 32;
            const int64_t per = ((keys + want - 1) / want + least - 1) / least * least;
            l.chunk = (int)per;
            l.splits = (int)((keys + per - 1) / per);
            l.partial_floats = l.splits > 1 ? items * l.splits * tile * (c->head_dim + 2) : 0;
            st = f(l);
        }
        l = SparseLaunch();
        l.group0 = next;
    };
    int64_t row_off = 0, group = 0;
    for (int r = 0; r < b->num_reqs && st == AMPD_OK; ++r) {
        const int64_t L = b->h_incr_len[r], groups = groups_of(L, g);
        for (int64_t at = 0; at < groups && st == AMPD_OK;) {
            if (l.n == SPARSE_MAX_REQS || l.groups == most_groups) {
                flush(group + at);
                if (st != AMPD_OK) break;
            }
            const int64_t take = std::min(groups - at, most_groups - l.groups);
            SparseRow& x = l.rows[l.n++];
            x.C = (int32_t)(b->h_ctx_len[r] + at * g);
            x.L = (int32_t)std::min(L - at * g, take * g);
            x.row_off = (int32_t)(row_off + at * g);
            x.req = r;
            x.first = l.groups;
            l.groups += (int)take;
            at += take;
        }
        row_off += L;
        group += groups;
    }
    flush(group);
    return st;
}

}  // namespace host
}  // namespace ampd

using namespace ampd;
using namespace ampd::host;

extern "C" {

size_t ampd_select_pages_workspace_bytes(const ampd_kv_cache* cache, const ampd_batch* batch, const ampd_page_selection* sel) {
    if (validate_select(cache, batch, sel) != AMPD_OK) return 0;
    SelectPlan plan;
    select_plan(cache, batch, sel, &plan);
    return (size_t)plan.bytes;
}

size_t ampd_sparse_attn_workspace_bytes(const ampd_kv_cache* cache, const ampd_batch* batch, int32_t budget, int32_t group_tokens) {
    if (validate_sparse(cache, batch, budget, group_tokens) != AMPD_OK) return 0;
    SparsePlan plan;
    sparse_plan(cache, batch, budget, group_tokens, &plan);
    return (size_t)plan.bytes;
}

}  // extern "C"
