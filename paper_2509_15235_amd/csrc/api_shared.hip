// C-ABI entry point of the attention behind a shared prefix: host-side checks, launch planning and enqueues.
#include "vs_internal.h"

namespace {

using namespace vs;

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
constexpr int64_t kMaxSharedRows = 1 << 20; // of a KV head: node_of_row_short() is exact up to 2^21, and a partial result of this many rows is 512 MB
constexpr int32_t kMaxSharedLen = 1 << 30; // keys rounded up to whole tiles stay in 32 bits

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
    if (x->max_len > kMaxSharedLen || d->max_prefix_len > kMaxSharedLen) return VS_ERR_SHAPE;
    prefix = prefix_as_desc(d, x);
    if (const int32_t rc = check_attention(&prefix, 0)) return rc;
    prefix.T = d->B * d->T;
    return VS_OK;
}

// A launch of the shared keys, or of the sequences' own.
struct Cut {
    int32_t rows_per_group, row_groups, num_splits, keys_per_split, total_wgs;
};
// How the shared keys are worked on.
enum Way : int32_t {
    kWayAuto = 0,
    kWayBoth8 = 1, // one launch with the sequences' own keys, workgroups of eight waves with key tiles of their own, one on a CU
    kWayBoth4 = 2, // ... of four waves, two on a CU
    kWayRows = 3,  // a launch of own tiles, equal splits
    kWayLine = 4,  // a launch of the pipelined kernel, all row groups' keys in one line of equal shares
    kWayUnits = 5, // ... every row group's keys in the same number of shares
    kWays = 6
};
thread_local int32_t asked_way = kWayAuto; // vs_internal_set_shared_way
thread_local int32_t asked_own = 0;        // vs_internal_set_shared_own
struct SharedPlan {
    Cut shared, own;
    int32_t way, own_waves, own_pipe;
    int32_t places; // for parts of a row
    int32_t shares, steps, longer, per_line, line_steps; // (kWayLine, kWayUnits) all, steps of one, how many have one more, shares and steps of a line
    float cost;
    size_t acc_bytes, ml_bytes, word_bytes;
};
struct SharedSize {
    int64_t rows, own_rows, own_units; // of a KV head; of a sequence's; (sequence, KV head)s
    int32_t B, Hkv, d, tiles;          // tiles of 64 keys
    bool f32, same_paging;
};

// Equal splits: places / workgroups of them, at most `most`, of `least` tiles or more. Whether the workgroups fit the places.
bool cut_rows(const SharedSize& z, int32_t rows_per_group, int64_t places, int32_t most, Cut& s, int32_t least = 4) {
    s.rows_per_group = rows_per_group;
    s.row_groups = (int32_t)((z.rows + rows_per_group - 1) / rows_per_group);
    const int64_t wgs = (int64_t)z.Hkv * s.row_groups;
    int64_t splits = places / wgs;
    if (splits > (z.tiles + least - 1) / least) splits = (z.tiles + least - 1) / least;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    const int tps = (int)((z.tiles + splits - 1) / splits);
    s.keys_per_split = tps * kIterKeys;
    s.num_splits = (z.tiles + tps - 1) / tps;
    s.total_wgs = (int32_t)(wgs * s.num_splits);
    return wgs <= places;
}
// 32-key tiles that a wave of such a launch takes one after the other
int64_t wave_tiles(const Cut& s, int32_t waves) { return (s.keys_per_split / kTileKeys + waves - 1) / waves; }

// One way's plan with its cost, the call's us as a straight line through what was measured; false: not for this call.
// us per call in a graph, three sets of data in turn, 28 / 4 heads of 128 channels and paged caches unless stated, 64 .. 200 own keys, by way Both8 / Both4 / Rows / Line /
// Units, the way that the lines choose in brackets:
//   4 x 1 token, 1696 keys [9.9] / 10.2 / 13.7 / - / -; 8192 keys [13.7] / 15.7 / 21.0 / - / -; 20 x 1, 600 keys [12.6] / 11.6 / 17.1 / 27.7 / 22.9, 8192 keys [20.3] / 23.2 / 24.5 / 28.0 / 28.0
//   30 x 4, 8192 keys 53.1 / 39.1 / [33.6] / 34.5 / 34.6; 60 x 4, 8 / 1 heads, 8192 keys [23.9] / 24.0 / 25.5 / 33.8 / 33.7
//   64 x 1, 600 keys - / [14.1] / 19.3 / 30.0 / 24.9, 1696 keys - / [16.9] / 20.2 / 30.3 / 25.9, 8192 keys - / 29.3 / [31.5] / 35.9 / 35.8; 80 x 1, 8192 keys - / 43.9 / [31.4] / 43.1 / 39.1
//   64 x 4, 600 keys - / [17.2] / 21.0 / 31.3 / 26.1, 1696 keys - / 26.1 / [25.3] / 34.0 / 28.7, 8192 keys - / 77.3 / 53.8 / 57.6 / [52.4]
//   16 x 60, 1696 keys - / - / 59.8 / 54.7 / [49.3], 6684 keys, up to 700 own ones - / - / 150.6 / [122.8] / 118.2
//   10 x 1, 32 / 32 heads, 4096 keys - / [21.2] / 26.4 / - / -; 14 x 1 - / 30.6 / [28.0] / - / -; 40 x 1, 32 / 8 heads of 64, 8192 keys - / 21.8 / [19.4] / 28.6 / 28.5
// All of them go by the host's bound on the length. Behind 1696 keys with a bound of 1696 / 4096 / 8192 / 32768, by the way chosen then: 4 x 1 9.8 / 10.3 / 11.2 / 17.1;
// 64 x 4 25.4 / 31.0 / 39.8 / 53.7 (Both4 26.0 throughout, Rows 24.9 / 31.4 / 31.4 / 31.3); 16 x 60 49.7 / - / 64.4 / 64.2. fp32, 6 x 5 nodes of 8 / 2 heads behind 601 keys, bounds of
// 601 / 4096 / 32768: 15.7 / 19.7 / 19.7.
bool plan_way(const SharedSize& z, int32_t way, SharedPlan& pl) {
    pl = SharedPlan{};
    pl.way = way;
    Cut& s = pl.shared;
    if (way == kWayBoth8 || way == kWayBoth4) {
        const int32_t waves = way == kWayBoth8 ? 8 : 4;
        // Parts beyond fifteen, with the own one, take the join a third trip to memory: 4 x 1, 8192 keys in 32 / 16 splits 15.5 / 13.5.
        if (z.f32 || z.own_rows > kRowBlock || !z.same_paging) return false;
        const int64_t places = (way == kWayBoth8 ? 1 : 2) * kNumCUs - z.own_units;
        if (places < 1 || !cut_rows(z, kRowBlock, places, 15, s)) return false;
        pl.cost = (waves == 8 ? 8.5f + 1.35f * wave_tiles(s, 8) : 12.f + 1.2f * wave_tiles(s, 4)) + 0.2f * s.num_splits;
        return true;
    }
    if (way == kWayRows) {
        const bool two = z.d == 128 && z.rows > kRowBlock;
        // fp32: four rows to a workgroup, or eight, which share what is read, where four would fill the CUs without key splits; splits of two tiles or more. us per call,
        // eight rows, splits of four / so: 6 x 5 nodes, 8 / 2 heads, 200, 601, 4000 keys 19.5 20.0 26.8 / 13.6 15.6 24.7; 16 x 1, 2000 keys 22.2 / 18.1; 4 x 2, 32 / 32
        // heads, 4000 keys 41.5 / 36.4. (Always four: 16 x 8, 28 / 4 heads, 1100 keys 73.6 / 83.1; 8 x 4, 32 / 8 heads of 64, 2000 keys 19.4 / 21.2.)
        if (z.f32) cut_rows(z, (int64_t)z.Hkv * ((z.rows + 3) / 4) * 128 <= (int64_t)kNumCUs * z.d ? 4 : 8, kNumCUs, kMergeMaxSplits, s, 2);
        else cut_rows(z, two ? 2 * kRowBlock : kRowBlock, kNumCUs, kMergeMaxSplits, s);
        const float rounds = (float)((s.total_wgs + kNumCUs - 1) / kNumCUs);
        pl.cost = 15.5f + (two ? 2.5f : 1.35f) * wave_tiles(s, 8) * rounds + 0.3f * s.num_splits;
        return true;
    }
    if (z.f32 || z.rows <= kRowBlock) return false;
    s.rows_per_group = 8 * kRowBlock;
    s.row_groups = (int32_t)((z.rows + s.rows_per_group - 1) / s.rows_per_group);
    const int64_t units = (int64_t)z.Hkv * s.row_groups, steps = units * z.tiles;
    if (steps > 0x7fffffff) return false;
    int64_t shares, per, line;
    if (way == kWayLine) { // the CUs end together, but a share that ends one row group and begins another pays twice for a beginning and an end
        shares = per = steps / 4 < kNumCUs ? (steps + 3) / 4 : kNumCUs;
        line = steps;
    } else {
        per = kNumCUs / units;
        if (per > z.tiles / 4) per = z.tiles / 4;
        if (per < 1) per = 1;
        shares = units * per;
        line = z.tiles;
    }
    pl.shares = (int32_t)shares;
    pl.per_line = (int32_t)per;
    pl.line_steps = (int32_t)line;
    pl.steps = (int32_t)(line / per);
    pl.longer = (int32_t)(line % per);
    // a row group's steps begin in one share and end in another: at most so many
    s.num_splits = way == kWayUnits ? (int32_t)per : (int32_t)((z.tiles + pl.steps - 1) / pl.steps) + 1;
    s.keys_per_split = kIterKeys;
    s.total_wgs = pl.shares;
    const float rounds = (float)((shares + kNumCUs - 1) / kNumCUs);
    pl.cost = 15.5f + rounds * 2.3f * (float)((line + per - 1) / per) + (way == kWayLine ? 9.f : 0.f) + 0.3f * s.num_splits;
    return true;
}

SharedPlan plan_shared(const vs_attn_desc* d, const vs_attn_desc& prefix) {
    const int group = d->Hq / d->Hkv;
    const bool f32 = d->dtype == VS_F32;
    const SharedSize z{(int64_t)d->B * d->T * group, d->T * group, (int64_t)d->B * d->Hkv, d->B, d->Hkv, d->d, (prefix.max_prefix_len + kIterKeys - 1) / kIterKeys,
                       f32, (d->paged != 0) == (prefix.paged != 0)};
    SharedPlan pl{};
    if (asked_way == kWayAuto || !plan_way(z, asked_way, pl)) {
        plan_way(z, kWayRows, pl);
        for (int32_t way = kWayAuto + 1; way < kWays; ++way) {
            SharedPlan other;
            if (plan_way(z, way, other) && other.cost < pl.cost) pl = other;
        }
    }
    const bool both = pl.way == kWayBoth8 || pl.way == kWayBoth4;
    Cut& o = pl.own;
    const int own_rows = d->T * group;
    // A workgroup for every row block, whose waves share the keys out; four of them together in the pipelined kernel where that would be many rounds of workgroups. us per
    // call behind 600 keys, 28 / 4 heads, 20 / 200 / 700 own keys at most, row blocks / pipelined:
    //   8 x 10 nodes 15.9 17.0 19.3 / 18.2 22.4 32.2; 16 x 30 21.2 23.0 28.6 / 24.8 29.7 39.0; 16 x 60 33.8 35.9 45.2 / 32.5 36.1 46.5; 32 x 60 53.8 56.4 70.7 / 46.3 50.7 66.4
    // (Two row blocks to a workgroup lose to both: 8 x 10 19.8 20.6 24.2.)
    pl.own_pipe = !f32 && own_rows > 2 * kRowBlock && z.own_units * ((own_rows + kRowBlock - 1) / kRowBlock) > 4 * kNumCUs;
    if (asked_own && !f32 && !both) pl.own_pipe = asked_own == 2;
    o.rows_per_group = f32 ? (z.own_units * ((own_rows + 3) / 4) <= kNumCUs ? 4 : 8) : pl.own_pipe ? 4 * kRowBlock : kRowBlock;
    o.row_groups = (own_rows + o.rows_per_group - 1) / o.rows_per_group;
    o.num_splits = 1;
    o.keys_per_split = (int32_t)(((int64_t)d->max_prefix_len + d->T + kIterKeys - 1) / kIterKeys * kIterKeys);
    o.total_wgs = d->B * d->Hkv * o.row_groups;
    // More workgroups than CUs: short ones of fewer waves, several to a CU. us per call, 32 x 1 token of 32 / 32 heads behind 4099 keys, eight waves / four / two
    // 63 / 44.4 / 46.7, 200 .. 1000 own keys - / 79 / 85; 64 x 1 of 16 / 16 heads of 64 - / 21.6 / 19.4.
    pl.own_waves = pl.own_pipe ? 4 : o.total_wgs <= kNumCUs ? 8 : d->d == 64 ? 2 : 4;
    pl.places = pl.shared.num_splits + (both ? 1 : 0);
    const size_t parts = (size_t)d->Hkv * pl.places;
    const size_t padded = (z.rows + kRowBlock - 1) / kRowBlock * kRowBlock; // whole row blocks
    pl.acc_bytes = align_up(parts * (f32 ? z.rows * d->d * sizeof(float) : padded * d->d * sizeof(uint16_t)));
    pl.ml_bytes = align_up(parts * z.rows * (f32 ? 2 : 4) * sizeof(float));
    if (both) pl.word_bytes = (size_t)z.own_units * kArrivalWords * sizeof(uint64_t);
    return pl;
}

// Loads that leave nothing in the caches (nt) where one workgroup alone reads a tile, and there are `least` megabytes of K and V or more, up to the longest
// allowed lengths: faster for who finds nothing there, as layers with caches of their own do. Only contiguous caches, without two rows in one place;
// what several sequences read through their tables, they may find in the caches. us per call, 32 / 32 heads of 128 channels, over other data each
// time (the same data), plain / the shared keys so / the own ones so:
//   16 x 1 behind 8000 keys (131 MB; up to 300 own keys, 79 MB) 41.9 (35.8) / 37.8 (37.6) / 41.5 (37.0); 32 x 1 behind 4099 (67, 158 MB) 44.3 (37.8) / 41.2 (38.8) / 39.9 (39.4);
//   up to 1000 own keys (525 MB) 79.1 (77.6) / 78.2 (73.2) / 71.3 (71.2); 64 x 1 behind 1000 (16, 315 MB) 54.3 (47.8) / 54.4 (47.7) / 50.7 (50.1);
//   32 x 1 behind 500, up to 100 own keys (8, 53 MB) 22.9 (22.7) / 24.1 (24.0) / 23.9 (22.1); 64 x 1 of 16 / 16 heads of 64 behind 4099 (34, 79 MB) 19.7 (19.6) / 19.6 (19.5) / 20.8 (19.8)
bool reads_once(const vs_attn_desc& d, int tree, const Cut& c, double least) {
    const int64_t keys = (int64_t)d.max_prefix_len + (tree ? d.T : 0);
    return !d.paged && c.row_groups == 1 && c.rows_per_group == kRowBlock && d.d == 128 && (double)d.B * d.Hkv * keys * d.d * 4e-6 >= least &&
           rows_apart(d.d, keys, d.stride_tok, d.Hkv, d.stride_head, d.B, d.stride_seq);
}

// Which halves of a call do (a bit each, the shared keys' first).
int32_t once_halves(const vs_attn_desc* d, const vs_attn_desc& prefix, const SharedPlan& pl) {
    if (pl.way != kWayRows || d->dtype == VS_F32) return 0;
    return (reads_once(prefix, 0, pl.shared, 96.) ? 1 : 0) | (!pl.own_pipe && reads_once(*d, 1, pl.own, 128.) ? 2 : 0);
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
    if (p.paged) p.capacity = (base.max_prefix_len + base.tree_keys - 1) >> base.block_shift; // see last_entry()
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

void vs_internal_set_shared_way(int32_t way) { asked_way = way; }
void vs_internal_set_shared_own(int32_t how) { asked_own = how; }
int32_t vs_internal_shared_own(const vs_attn_desc* desc, const vs_prefix_desc* prefix) {
    vs_attn_desc x;
    const int32_t rc = check_shared(desc, prefix, x);
    return rc != VS_OK ? rc : plan_shared(desc, x).own_pipe ? 2 : 1;
}
int32_t vs_internal_shared_way(const vs_attn_desc* desc, const vs_prefix_desc* prefix) {
    vs_attn_desc x;
    const int32_t rc = check_shared(desc, prefix, x);
    return rc != VS_OK ? rc : plan_shared(desc, x).way;
}

int32_t vs_internal_shared_reads_once(const vs_attn_desc* desc, const vs_prefix_desc* prefix) {
    vs_attn_desc x;
    const int32_t rc = check_shared(desc, prefix, x);
    return rc != VS_OK ? rc : once_halves(desc, x, plan_shared(desc, x));
}

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
    SharedParams first = shared_params(attention_params(&x, 0, q, k_shared, v_shared, shared_len, nullptr, nullptr, nullptr, nullptr), pl.shared, pl, desc, x,
                                       shared_len, workspace);
    SharedParams second = shared_params(attention_params(desc, 1, q, k_cache, v_cache, prefix_len, tree_parent, tree_mask, out, status), pl.own, pl, desc, x,
                                        shared_len, workspace);
    const int32_t once = once_halves(desc, x, pl);
    first.once = once & 1;
    second.once = once >> 1;
    hipError_t e;
    if (pl.way == kWayBoth8 || pl.way == kWayBoth4) {
        e = launch_attention_shared_both(first, second, pl.way == kWayBoth8 ? 8 : 4, s);
    } else {
        e = f32 ? launch_attention_shared_f32(first, kRowsShared, s)
            : pl.way == kWayRows ? launch_attention_shared_rows(first, kRowsShared, 8, s)
                                 : launch_attention_shared_pipe(first, kRowsShared, s);
        if (e == hipSuccess)
            e = f32 ? launch_attention_shared_f32(second, kRowsOwn, s)
                : pl.own_pipe ? launch_attention_shared_pipe(second, kRowsOwn, s)
                              : launch_attention_shared_rows(second, kRowsOwn, pl.own_waves, s);
    }
    return e == hipSuccess ? VS_OK : VS_ERR_HIP;
}

} // extern "C"
