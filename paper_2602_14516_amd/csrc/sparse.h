// Kernel parameter blocks and launcher declarations of the sparse-attention operators, shared by sparse.hip and sparse_api.cpp, and the
// rules on sizes that the host half (sparse_host.cpp) needs too.
#pragma once
#include <stdint.h>

#include "ampd.h"
#include "plan.h"

namespace ampd {

// ---- sizes -------------------------------------------------------------------------------------

constexpr int SPARSE_MAX_ROWS = 128;          // query rows of a group (tokens x heads of a KV head)

inline int64_t groups_of(int64_t L, int g) { return (L + g - 1) / g; }

// Scores of a row's pages, for one group and KV head: this many 32-bit keys.
inline int64_t key_stride(int64_t T, int P) { return ((T + P - 1) / P + 63) / 64 * 64; }
// A launch writes at most this many 32-bit words, keys and query codes together, or those of a single group: the workspace stays at 64 MiB
// where rows are many or long, and what one launch writes the next one finds in the last-level cache.
constexpr int64_t SELECT_WORDS = 16 << 20;

// Row tile of a sparse-attention workgroup: 16 query rows, or 32 where a group has more.
inline int sparse_tile(int rows) { return rows <= 16 ? 16 : 32; }

// A wave of the score launch goes through score_tiles tiles of 16 pages, SCORE_BATCH at a time; a workgroup's waves are `score_heads`
// neighbouring heads of the same pages, then neighbouring pages.  Long launches give a wave more tiles, which spares it queries to quantise,
// until some 3 000 waves are left (96 rows of 2-16 k tokens, 8 KV heads: 2, 4, 8, 12, 16 tiles 35.6, 30.3, 29.0, 30.7, 34.8 us; 4 rows of
// 36-70 k, one head: 5.4, 6.0, 7.5, 8.6, 10.1).  Batches of 4 tiles and workgroups of 8 waves leave a CU fewer waves: 32.7 us.
constexpr int SCORE_BATCH = 2;
constexpr int SCORE_WAVES = 4;
inline int score_heads(int Hkv) { return Hkv > 2 ? 4 : Hkv; }
inline int score_pages(int Hkv, int score_tiles) { return score_tiles * 16 * (SCORE_WAVES / score_heads(Hkv)); }
inline int score_tiles(int64_t tiles) {
    const int64_t t = tiles / 3000 / SCORE_BATCH * SCORE_BATCH;
    return (int)(t < SCORE_BATCH ? SCORE_BATCH : t > 64 ? 64 : t);
}

// ---- launches ----------------------------------------------------------------------------------
// The rows of a launch travel as kernel arguments.  A row with more groups than one launch takes is handed on as a row whose context begins
// further on: a group depends on its tokens' positions alone.

constexpr int SELECT_MAX_REQS = 96;
struct SelectRow {
    int32_t C, L, row_off, req;
    int32_t out0;             // number of the row's first group in the output
    int32_t item0;            // groups of the rows before it in this launch
    int32_t tile0;            // score workgroups of the rows before it in this launch
    uint32_t key0;            // the row's first key in the workspace, in units of 64 keys
};
struct SelectLaunch {
    int n = 0, groups = 0, score_blocks = 0, score_tiles = 0;
    bool codes = false;       // the queries' codes are made by a launch of their own (some row has more than one group, and scores are wanted)
    int64_t keys = 0;         // in the workspace; the codes follow
    int64_t code_offset() const { return (keys + 63) / 64 * 256; }       // bytes
    int64_t max_keys = 0;     // the most pages that a group chooses from
    SelectRow rows[SELECT_MAX_REQS];
};

constexpr int SPARSE_MAX_REQS = 128;
struct SparseRow {
    int32_t C, L, row_off, req;
    int32_t first;            // groups of the rows before it in this launch
};
struct SparseLaunch {
    int n = 0, groups = 0;
    int64_t group0 = 0;       // number of its first group in the batch
    int tiles = 1, waves = 4;  // row tiles of a group; waves of a workgroup
    int splits = 1, chunk = 0; // pieces of a list; keys per piece (a multiple of 32)
    int64_t partial_floats = 0;
    SparseRow rows[SPARSE_MAX_REQS];
};

}  // namespace ampd

#include <type_traits>

namespace ampd {
namespace host {

// A caller's function for the launches of a call; nothing is allocated, so that no exception comes out of an entry point.
template <class L>
class LaunchFn {
    void* ctx_;
    ampd_status (*call_)(void*, const L&);

public:
    template <class F>
    LaunchFn(F&& f) : ctx_((void*)&f), call_([](void* c, const L& l) -> ampd_status { return (*static_cast<std::remove_reference_t<F>*>(c))(l); }) {}
    ampd_status operator()(const L& l) const { return call_(ctx_, l); }
};

ampd_status validate_rope(const ampd_kv_cache* c, const ampd_batch* b, const ampd_rope* rope, const ampd_qkv_rows* rows, const void* q_out);
ampd_status validate_bounds(const ampd_page_bounds* bounds);
ampd_status validate_select(const ampd_kv_cache* c, const ampd_batch* b, const ampd_page_selection* sel);
ampd_status validate_sparse(const ampd_kv_cache* c, const ampd_batch* b, int32_t budget, int32_t group_tokens);
// f for each launch of a call, in order; the first status that is not AMPD_OK ends it
ampd_status select_launches(const ampd_kv_cache* c, const ampd_batch* b, const ampd_page_selection* sel, LaunchFn<SelectLaunch> f);
ampd_status sparse_launches(const ampd_kv_cache* c, const ampd_batch* b, int32_t budget, int32_t group_tokens, LaunchFn<SparseLaunch> f);
// What a call needs of its workspace, and its launch where it has one alone (the usual case: it is then not worked out twice).
struct SelectPlan {
    int64_t bytes = 0;
    int launches = 0;
    SelectLaunch only;
};
void select_plan(const ampd_kv_cache* c, const ampd_batch* b, const ampd_page_selection* sel, SelectPlan* out);
struct SparsePlan {
    int64_t bytes = 0;
    int launches = 0;
    SparseLaunch only;
};
void sparse_plan(const ampd_kv_cache* c, const ampd_batch* b, int32_t budget, int32_t group_tokens, SparsePlan* out);

}  // namespace host

}  // namespace ampd

#if defined(__HIP__)
#include <hip/hip_runtime.h>

#include "kernels.h"

namespace ampd {

struct RopeParams {
    AppendParams a;           // k_new, v_new: the first packed rows; one workgroup column per page that new tokens fall into
    const void* q;
    void* q_out;
    int64_t q_stride, k_stride, v_stride;     // bytes from token to token
    const float* inv_freq;
    const int32_t* positions;
    int8_t* codes;            // bounds, or null
    float* bscale;
    int64_t num_pages;
    int32_t Hq, rd, interleaved;
    float scale;
};

struct BoundsParams {
    AppendParams a;
    int8_t* codes;
    float* bscale;
    int64_t num_pages;
};

struct SelectParams {
    const void* q;
    const int8_t* codes;
    const float* bscale;
    const int32_t* block_table;
    int32_t* selected;
    uint32_t* keys;           // [row][group][KV head][key_stride]
    int8_t* qcodes;           // [group of this launch][KV head][2 limbs][2 d]
    int64_t num_pages;
    int32_t Hq, Hkv, P, logP, max_pages;
    int32_t budget, first, last, g;
    int32_t score_tiles, n;
    SelectRow rows[SELECT_MAX_REQS];
};

struct SparseParams {
    const void* q;
    void* out;
    const void* k_pool;
    const void* v_pool;
    const float* k_scale;
    const float* v_scale;
    const int32_t* block_table;
    const int32_t* selected;  // of this launch's first group
    float* partial;
    int64_t num_pages;
    int32_t Hq, Hkv, P, logP, max_pages;
    int32_t budget, g, tiles, splits, chunk;
    float c_log2;
    int32_t n;
    SparseRow rows[SPARSE_MAX_REQS];
};

hipError_t launch_rope(RopeParams& p, int kvt, int64_t pages, int max_new, hipStream_t st);
hipError_t launch_bounds(BoundsParams& p, int kvt, int64_t pages, hipStream_t st);
hipError_t launch_select(const SelectParams& p, int D, int groups, int score_blocks, bool codes, int64_t max_keys, hipStream_t st);
hipError_t launch_sparse(const SparseParams& p, int D, int kvt, int groups, int waves, hipStream_t st);

}  // namespace ampd
#endif
