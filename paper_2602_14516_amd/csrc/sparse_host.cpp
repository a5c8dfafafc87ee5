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

// Waves of a workgroup, and pieces of a list, for `items` lists (of a group, row tile and KV head) of so many keys.  A CU holds as many waves either
// way: two workgroups of 4 waves or one of 8 at d = 128, by their LDS, twice as many at d = 64.  Cutting a list costs a second launch and the
// partial results' way through memory, about 4 us.  us per call, of rows whose histories are four times as long as their lists:
//                                            512 keys      2 048          8 192
//    32 items, bf16, d = 128: 8 waves           9.2         24.7          85         4 waves, 16 pieces   9.9   13.2   30
//    64                       8 waves          10.6         26.4          88         8 waves, 4 pieces   12.0   18.9   51      (4 waves, 8 pieces 18.7, 52)
//   128                       8 waves          11.6         29.8         101         8 waves, 2 pieces   13.2   29.7   93
//   128, 8 bits               8 waves           9.5         21.9          72         8 waves, 2 pieces   11.8   19.8   53
//   192                       8 waves          12.7         37.0         129         4 waves, 4 pieces   17.7   40.7  134      (4 waves 13.0, 39.5, 146)
//   264                       4 waves          19.7         62.5         238         4 waves, 3 pieces   23.4   57.0  192      (8 waves 23.1, 67.0, 239)
//   384                       4 waves          22.5         71.1         284         4 waves, 3 pieces   26.1   76.7  264
//   288, 32 rows              4 waves          13.8         33.3         112         4 waves, 3 pieces   24.6   40.2   98
//   320, 8 bits, d = 64       4 waves           9.4         26.0          86         8 waves              9.1   21.1   69
// Just above 256 items some CUs get two lists and most get one; thirds are spread more evenly.  What the rule does not take: 160 items over 8 192 keys are
// up to a quarter faster in three pieces, 640 as much by 8 waves or in pieces.
struct SparseCut {
    int waves;
    int64_t pieces;
};
static SparseCut sparse_cut(int64_t items, int64_t keys, int d, int tile) {
    const bool long_lists = keys * d > 96 << 10;      // 768 keys at d = 128: whole 10 to 11 us, in pieces 9.5 to 12
    if (items <= 32 && long_lists) return {4, std::min(512 / items, std::max<int64_t>(16, keys / 512))};     // (the join takes 16 pieces at once)
    if (items <= 256) return {8, long_lists ? 256 / items : 1};
    return {items <= 256 * 128 / d ? 8 : 4, items <= 341 && keys * d >= (int64_t)tile << 14 ? 3 : 1};
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
            const int64_t items = (int64_t)l.groups * tiles * Hkv;
            const SparseCut cut = sparse_cut(items, keys, c->head_dim, tile);
            const int64_t least = cut.waves * 32;
            const int64_t per = ((keys + cut.pieces - 1) / cut.pieces + least - 1) / least * least;
            l.waves = cut.waves;
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
