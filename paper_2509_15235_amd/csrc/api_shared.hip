// C-ABI entry point of the attention behind a shared prefix: host-side checks, launch planning and enqueues.
#include <stdlib.h>
#include "vs_internal.h"

namespace {

using namespace vs;

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
constexpr int64_t kMaxSharedRows = 1 << 20; // of a KV head: node_of_row_short() is exact up to 2^21, and a partial result of this many rows is 512 MB

// The shared prefix as the cache of one sequence, all sequences' nodes its queries.
vs_attn_desc prefix_as_desc(const vs_attn_desc* d, const vs_prefix_desc* x) {
    vs_attn_desc s = *d;
    s.B = 1;
    s.T = 1; // (set to B * T behind the checks)
    s.max_prefix_len = x->max_len;
    s.paged = x->paged;
    s.block_size = x->block_size;
    s.max_blocks = x->max_blocks;
    s.num_blocks = x->num_blocks;
    s.capacity = x->capacity;
    s.stride_seq = 0;
    s.stride_block = x->stride_block;
    s.stride_head = x->stride_head;
    s.stride_tok = x->stride_tok;
    s.block_table = x->block_table;
    return s;
}

int32_t check_shared(const vs_attn_desc* d, const vs_prefix_desc* x, vs_attn_desc& prefix) {
    if (!d || !x) return VS_ERR_NULL;
    if (d->impl != VS_IMPL_AUTO || d->num_splits != 0 || d->rows_per_wave != 0 || d->waves_per_group != 0 || d->schedule != VS_SCHED_AUTO)
        return VS_ERR_SHAPE;
    if (const int32_t rc = check_attention(d, 1)) return rc;
    if ((int64_t)d->B * d->T * (d->Hq / d->Hkv) > kMaxSharedRows) return VS_ERR_SHAPE;
    prefix = prefix_as_desc(d, x);
    if (const int32_t rc = check_attention(&prefix, 0)) return rc;
    prefix.T = d->B * d->T;
    return VS_OK;
}

// A launch of the shared keys, or of the sequences' own.
struct Cut {
    int32_t rows_per_group, row_groups, num_splits, keys_per_split, total_wgs;
};
struct SharedPlan {
    Cut shared, own;
    int32_t own_waves, own_pipe;
    int32_t both;   // one launch
    int32_t places; // for parts of a row
    int32_t steps, longer, per_line, line_steps; // of a share, of a line of shares
    int32_t waves, shares; // the pipelined kernel on equal shares of all row groups' keys; 0: own tiles, equal splits
    size_t acc_bytes, ml_bytes, word_bytes;
};

SharedPlan plan_shared(const vs_attn_desc* d, const vs_attn_desc& prefix) {
    SharedPlan pl{};
    const int group = d->Hq / d->Hkv;
    const int64_t rows = (int64_t)d->B * d->T * group;
    const bool f32 = d->dtype == VS_F32;
    const int tiles = (prefix.max_prefix_len + kIterKeys - 1) / kIterKeys;
    Cut& s = pl.shared;
    if (!f32 && (int64_t)d->Hkv * ((rows + 255) / 256) * tiles <= 0x7fffffff && rows > (getenv("PIPEROWS") ? atoi(getenv("PIPEROWS")) : 128)) {
        pl.waves = getenv("W4") ? 4 : 8;
        s.rows_per_group = pl.waves * kRowBlock;
        s.row_groups = (int32_t)((rows + s.rows_per_group - 1) / s.rows_per_group);
        const int64_t units = (int64_t)d->Hkv * s.row_groups, steps = units * tiles, places = kNumCUs * (pl.waves == 8 ? 1 : 2);
        // Shares anywhere: all CUs end together, but a share that ends one unit and begins another pays for two beginnings and ends, 8 steps' time or so each.
        // Or every unit in the same number of them.
        int64_t shares = steps / 4 < places ? (steps + 3) / 4 : places, whole = places / units;
        if (whole > tiles / 4) whole = tiles / 4;
        if (whole < 1) whole = 1;
        const int64_t any = (steps + shares - 1) / shares + 9, even = ((tiles + whole - 1) / whole + 4) * ((units * whole + places - 1) / places);
        const bool lines = even <= any;
        const int64_t per = lines ? whole : shares, line = lines ? tiles : steps;
        pl.shares = (int32_t)(lines ? units * whole : shares);
        pl.per_line = (int32_t)per;
        pl.line_steps = (int32_t)line;
        pl.steps = (int32_t)(line / per);
        pl.longer = (int32_t)(line % per);
        // a unit's steps begin in one share and end in another: at most so many
        s.num_splits = lines ? (int32_t)whole : (int32_t)((tiles + pl.steps - 1) / pl.steps) + 1;
        s.keys_per_split = kIterKeys;
        s.total_wgs = pl.shares;
    } else {
        // One launch for both kinds of work where all workgroups run at once (and one row block of the shared keys to a workgroup): us per call,
        // two launches / one
        const int64_t blocks = (rows + kRowBlock - 1) / kRowBlock, own = (int64_t)d->B * d->Hkv;
        pl.both = !f32 && d->T * group <= kRowBlock && (d->paged != 0) == (prefix.paged != 0) && own + blocks * d->Hkv <= kNumCUs && !getenv("NOBOTH");
        s.rows_per_group = f32 ? 8 : d->d == 128 && rows > kRowBlock && !pl.both ? 2 * kRowBlock : kRowBlock;
        s.row_groups = (int32_t)((rows + s.rows_per_group - 1) / s.rows_per_group);
        const int64_t wgs = (int64_t)d->Hkv * s.row_groups;
        int64_t splits = (kNumCUs - (pl.both ? own : 0)) / wgs;
        if (splits > (tiles + 3) / 4) splits = (tiles + 3) / 4;
        if (splits > kMergeMaxSplits) splits = kMergeMaxSplits;
        if (splits < 1) splits = 1;
        const int tps = (int)((tiles + splits - 1) / splits);
        s.keys_per_split = tps * kIterKeys;
        s.num_splits = (tiles + tps - 1) / tps;
        s.total_wgs = (int32_t)(wgs * s.num_splits);
    }
    Cut& o = pl.own;
    const int own_rows = d->T * group;
    o.rows_per_group = f32 ? ((int64_t)d->B * d->Hkv * ((own_rows + 3) / 4) <= kNumCUs ? 4 : 8) : d->d == 128 && own_rows > kRowBlock ? 2 * kRowBlock : kRowBlock;
    if (!f32 && own_rows > 2 * kRowBlock) {
        pl.own_pipe = 1;
        pl.own_waves = getenv("OWN8") ? 8 : 4;
        o.rows_per_group = pl.own_waves * kRowBlock;
    }
    o.row_groups = (own_rows + o.rows_per_group - 1) / o.rows_per_group;
    o.num_splits = 1;
    o.keys_per_split = (int32_t)(((int64_t)d->max_prefix_len + d->T + kIterKeys - 1) / kIterKeys * kIterKeys);
    o.total_wgs = d->B * d->Hkv * o.row_groups;
    if (!pl.own_pipe) pl.own_waves = o.rows_per_group > kRowBlock || o.total_wgs <= kNumCUs ? 8 : d->d == 64 ? 2 : 4;
    pl.places = s.num_splits + (pl.both ? 1 : 0);
    const size_t parts = (size_t)d->Hkv * pl.places;
    const size_t padded = (rows + kRowBlock - 1) / kRowBlock * kRowBlock; // whole row blocks
    pl.acc_bytes = align_up(parts * (f32 ? rows * d->d * sizeof(float) : padded * d->d * sizeof(uint16_t)));
    pl.ml_bytes = align_up(parts * rows * (f32 ? 2 : 4) * sizeof(float));
    if (pl.both) pl.word_bytes = (size_t)d->B * d->Hkv * kArrivalWords * sizeof(uint64_t);
    return pl;
}

SharedParams shared_params(const AttnParams& base, const Cut& c, const SharedPlan& pl, const vs_attn_desc* d, const vs_attn_desc& prefix, const int32_t* shared_len,
                           void* workspace) {
    SharedParams p{};
    (AttnParams&)p = base;
    p.rows_per_group = c.rows_per_group;
    p.row_groups = c.row_groups;
    p.num_splits = c.num_splits;
    p.keys_per_split = c.keys_per_split;
    p.total_wgs = c.total_wgs;
    p.by_splits = fast_div_by(c.num_splits);
    p.by_groups = fast_div_by(c.row_groups);
    p.by_heads = fast_div_by(d->Hkv);
    p.sh_acc = (float*)workspace;
    p.sh_ml = (float*)((char*)workspace + pl.acc_bytes);
    p.sh_words = (uint64_t*)((char*)p.sh_ml + pl.ml_bytes);
    p.shared_len = shared_len;
    p.shared_table = prefix.paged ? prefix.block_table : nullptr;
    p.sh_batch = d->B;
    p.sh_own_rows = d->T * (d->Hq / d->Hkv);
    p.sh_rows = d->B * d->T * (d->Hq / d->Hkv);
    p.sh_blocks = (p.sh_rows + kRowBlock - 1) / kRowBlock;
    p.sh_splits = pl.places;
    p.sh_keys_per_split = pl.shared.keys_per_split;
    p.sh_shares = pl.shares;
    p.sh_steps = pl.steps;
    p.sh_longer = pl.longer;
    p.sh_groups = pl.shared.row_groups;
    p.sh_by_rows = fast_div_by(pl.shared.rows_per_group);
    p.sh_by_steps = fast_div_by((prefix.max_prefix_len + kIterKeys - 1) / kIterKeys);
    if (pl.shares) {
        p.sh_by_line = fast_div_by(pl.per_line);
        p.sh_by_line_steps = fast_div_by(pl.line_steps);
        p.sh_by_share = fast_div_by(pl.steps);
        p.sh_by_longer = fast_div_by(pl.steps + 1);
    }
    p.max_shared = prefix.max_prefix_len;
    while (prefix.paged && (1 << p.sh_block_shift) < prefix.block_size) ++p.sh_block_shift;
    p.sh_num_blocks = prefix.num_blocks;
    p.sh_slots = prefix.paged ? (int64_t)prefix.max_blocks * prefix.block_size : prefix.capacity;
    return p;
}

} // namespace

extern "C" {

size_t vs_shared_prefix_workspace_bytes(const vs_attn_desc* desc, const vs_prefix_desc* prefix) {
    vs_attn_desc x;
    if (check_shared(desc, prefix, x) != VS_OK) return 0;
    const SharedPlan pl = plan_shared(desc, x);
    return pl.acc_bytes + pl.ml_bytes + pl.word_bytes;
}

int32_t vs_shared_prefix_attention(const vs_attn_desc* desc, const vs_prefix_desc* prefix, const void* q, const void* k_shared, const void* v_shared,
                                   const int32_t* shared_len, const void* k_cache, const void* v_cache, const int32_t* prefix_len,
                                   const int32_t* tree_parent, const uint64_t* tree_mask, void* out, int32_t* status, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    if (!desc || !prefix || !q || !k_shared || !v_shared || !shared_len || !k_cache || !v_cache || !prefix_len || !tree_parent || !out) return VS_ERR_NULL;
    vs_attn_desc x;
    if (const int32_t rc = check_shared(desc, prefix, x)) return rc;
    for (const void* at : {q, k_shared, v_shared, k_cache, v_cache, (const void*)out})
        if (!aligned16(at)) return VS_ERR_LAYOUT;
    const SharedPlan pl = plan_shared(desc, x);
    if (!workspace || workspace_bytes < pl.acc_bytes + pl.ml_bytes + pl.word_bytes || ((uintptr_t)workspace & (kAlign - 1))) return VS_ERR_WORKSPACE;
    if (const int32_t dc = check_device()) return dc;
    hipStream_t s = (hipStream_t)stream;
    const bool f32 = desc->dtype == VS_F32;
    const SharedParams first = shared_params(attention_params(&x, 0, q, k_shared, v_shared, shared_len, nullptr, nullptr, nullptr, nullptr), pl.shared, pl, desc, x,
                                             shared_len, workspace);
    const SharedParams second = shared_params(attention_params(desc, 1, q, k_cache, v_cache, prefix_len, tree_parent, tree_mask, out, status), pl.own, pl, desc, x,
                                              shared_len, workspace);
    if (pl.both) return launch_attention_shared_both(first, second, s) == hipSuccess ? VS_OK : VS_ERR_HIP;
    hipError_t e = f32 ? launch_attention_shared_f32(first, kRowsShared, s) : pl.waves ? launch_attention_shared_pipe(first, kRowsShared, pl.waves, s) : launch_attention_shared_rows(first, kRowsShared, 8, s);
    if (e == hipSuccess) e = f32 ? launch_attention_shared_f32(second, kRowsOwn, s) : pl.own_pipe ? launch_attention_shared_pipe(second, kRowsOwn, pl.own_waves, s) : launch_attention_shared_rows(second, kRowsOwn, pl.own_waves, s);
    return e == hipSuccess ? VS_OK : VS_ERR_HIP;
}

} // extern "C"
