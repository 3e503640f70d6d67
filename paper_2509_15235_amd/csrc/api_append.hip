// C-ABI entry points of the rotation and of the cache append: host-side argument checks and launches.
#include "vs_internal.h"

namespace {

using namespace vs;

// How a launch of `rows` rows of H heads of `chunks` items is cut: rows and heads of a workgroup of 256 threads.
struct RowCut {
    int32_t rows, heads;
};
RowCut cut_rows(int64_t rows, int32_t H, int32_t chunks) {
    RowCut c{4, H};
    while (c.rows > 1 && rows < (int64_t)c.rows * kNumCUs) c.rows /= 2;
    // few rows: their heads over more workgroups, as long as every thread has an item
    const int64_t groups = (rows + c.rows - 1) / c.rows;
    while (c.heads > 1 && groups * ((H + c.heads - 1) / c.heads) < kNumCUs && c.rows * ((c.heads + 1) / 2) * chunks >= 256) c.heads = (c.heads + 1) / 2;
    return c;
}

// Whether results go past the L2 caches (nt stores): large ones, which would take the inputs' place there while they are written. us in a graph, three sets of
// data in turn, plain / past. The call alone, 32 heads of 128 channels: 500 rows (4.1 MB written) 3.12 / 3.13, 600 3.68 / 3.44, 1000 4.34 / 3.81, 2000 8.00 / 6.60,
// 6684 25.9 / 17.4 (6.3 TB/s), 16000 52.1 / 49.2; appends of 28 / 4 heads, paged: 16 x 60 nodes (8.8 MB) 6.17 / 5.45, 32 x 60 10.2 / 9.0, 7712 rows 34.2 / 24.5 (5.9 TB/s).
// Who reads the results next pays a part of that back, and from some 30 MB on more, since a plain store would have left him some. The call and a read of all it wrote:
// 600 rows 8.35 / 7.22, 1000 8.79 / 7.88, 2000 12.7 / 11.8, 4000 18.6 / 19.0, 6684 26.6 / 28.6, 16000 64.8 / 73.3, the append of 7712 rows 39.5 / 35.9; appended trees and
// the attention behind them: 10 x 60 42.5 / 42.8, 16 x 60 51.5 / 51.3, 32 x 60 70.8 / 70.4, 64 x 60 115.1 / 116.6.
bool streams_out(int64_t bytes) { return bytes >= (4 << 20); }

int32_t check_rope(const vs_rope_desc* r, int32_t d, int32_t dtype, RopeParams& p) {
    if (!r) return VS_ERR_NULL;
    if (dtype != VS_BF16 && dtype != VS_F32) return VS_ERR_DTYPE;
    const int32_t piece = dtype == VS_BF16 ? 8 : 4; // channels of 16 bytes
    if (d < 1 || d > 2 * kMaxRopePairs || r->rot_dim < 0 || r->rot_dim > d) return VS_ERR_SHAPE;
    if (r->pairing != VS_PAIR_HALVES && r->pairing != VS_PAIR_ADJACENT) return VS_ERR_SHAPE;
    if (r->axis_order != VS_AXES_BLOCKS && r->axis_order != VS_AXES_CYCLIC) return VS_ERR_SHAPE;
    if (r->num_axes < 1 || r->num_axes > 4) return VS_ERR_SHAPE;
    const bool halves = r->pairing == VS_PAIR_HALVES;
    if (r->rot_dim % (halves ? 2 * piece : piece) || d % piece) return VS_ERR_LAYOUT;
    const int32_t pairs = r->rot_dim / 2;
    if (r->num_axes > 1) {
        int64_t sum = 0;
        for (int x = 0; x < r->num_axes; ++x) {
            const int32_t n = r->axis_pairs[x];
            if (n < 0 || n > pairs) return VS_ERR_SHAPE;
            // round robin: the axis's last pair exists
            if (r->axis_order == VS_AXES_CYCLIC && x > 0 && n > 0 && (n - 1) * r->num_axes + x >= pairs) return VS_ERR_SHAPE;
            sum += n;
        }
        if (sum != pairs) return VS_ERR_SHAPE;
        if (r->stride_axis < 0) return VS_ERR_LAYOUT;
    }
    if (pairs > 0 && !r->inv_freq) return VS_ERR_NULL;
    p.inv_freq = r->inv_freq;
    p.stride_axis = r->stride_axis;
    p.pairs = pairs;
    p.num_axes = r->num_axes;
    p.cyclic = r->axis_order == VS_AXES_CYCLIC;
    p.inverse = r->inverse != 0;
    for (int x = 0; x < 4; ++x) p.axis_pairs[x] = x < r->num_axes && r->num_axes > 1 ? r->axis_pairs[x] : 0;
    p.turning = halves ? pairs / piece : r->rot_dim / piece;
    p.chunks = p.turning + (d - r->rot_dim) / piece;
    p.by_chunks = fast_div_by(p.chunks);
    return VS_OK;
}

constexpr int32_t kMaxHeads = 65536; // head numbers share a word with other things, and a row's offsets stay in 32 bits

} // namespace

extern "C" {

int32_t vs_rope_apply(const vs_rope_desc* rope, const void* x, int64_t x_stride_row, int64_t x_stride_head, const int32_t* positions, int64_t rows,
                      int32_t H, int32_t d, int32_t dtype, void* out, int64_t out_stride_row, int64_t out_stride_head, void* stream) {
    if (!rope || !x || !positions || !out) return VS_ERR_NULL;
    RopeApplyParams p{};
    const int32_t rc = check_rope(rope, d, dtype, p.rope);
    if (rc != VS_OK) return rc;
    if (rows < 1 || rows > 0x7fffffff || H < 1 || H > kMaxHeads) return VS_ERR_SHAPE;
    const int64_t eb = dtype == VS_BF16 ? 2 : 4;
    for (const int64_t s : {x_stride_row, x_stride_head, out_stride_row, out_stride_head})
        if (s < 0 || s > ((int64_t)1 << 40) || (s * eb) % 16) return VS_ERR_LAYOUT;
    if (!aligned16(x) || !aligned16(out)) return VS_ERR_LAYOUT;
    // two heads of the result in one place; or the input's place with other strides
    if (!rows_apart(d, rows, out_stride_row, H, out_stride_head, 1, 0)) return VS_ERR_LAYOUT;
    if (x == out && (x_stride_row != out_stride_row || x_stride_head != out_stride_head)) return VS_ERR_LAYOUT;
    if (const int32_t dc = check_device()) return dc;
    p.x = x;
    p.out = out;
    p.positions = positions;
    p.rows = rows;
    p.x_row = x_stride_row * eb;
    p.x_head = x_stride_head * eb;
    p.out_row = out_stride_row * eb;
    p.out_head = out_stride_head * eb;
    p.H = H;
    const RowCut cut = cut_rows(rows, H, p.rope.chunks);
    p.rows_per_wg = cut.rows;
    p.heads_per_wg = cut.heads;
    p.by_heads = fast_div_by(cut.heads);
    p.stream_out = streams_out(rows * H * d * eb);
    return launch_rope(p, dtype, rope->pairing == VS_PAIR_HALVES, (hipStream_t)stream) == hipSuccess ? VS_OK : VS_ERR_HIP;
}

int32_t vs_kv_append(const vs_append_desc* d, const vs_rope_desc* rope, const void* q, const void* k, const void* v, const int32_t* positions,
                     const int32_t* depth, const int32_t* pos_offset, const int32_t* prefix_len, const int32_t* row_start, void* q_out, void* k_cache,
                     void* v_cache, int32_t* status, void* stream) {
    if (!d || !rope || !k || !v || !prefix_len || !k_cache || !v_cache) return VS_ERR_NULL;
    if (d->Hq > 0 && (!q || !q_out)) return VS_ERR_NULL;
    if (d->B < 1 || d->T < 1 || d->Hq < 0 || d->Hkv < 1 || d->Hq > kMaxHeads || d->Hkv > kMaxHeads) return VS_ERR_SHAPE;
    AppendParams p{};
    const int32_t rc = check_rope(rope, d->d, d->dtype, p.rope);
    if (rc != VS_OK) return rc;
    if (rope->inverse) return VS_ERR_SHAPE;
    if (d->rows < 1 || d->rows > 0x7fffffff - kMaxHeads) return VS_ERR_SHAPE;
    if (row_start ? depth != nullptr : d->rows != (int64_t)d->B * d->T) return VS_ERR_SHAPE;
    const int64_t eb = d->dtype == VS_BF16 ? 2 : 4;
    if (d->stride_head < 0 || d->stride_tok < d->d) return VS_ERR_LAYOUT;
    const int64_t q_cols = (int64_t)d->Hq * d->d, kv_cols = (int64_t)d->Hkv * d->d;
    if (d->Hq > 0 && (d->q_stride < q_cols || d->q_out_stride < q_cols)) return VS_ERR_LAYOUT;
    if (d->k_stride < kv_cols || d->v_stride < kv_cols) return VS_ERR_LAYOUT;
    if (d->Hq > 0 && q == q_out && d->q_stride != d->q_out_stride) return VS_ERR_LAYOUT;
    if (d->paged) {
        if (!is_pow2(d->block_size) || d->block_size < 16) return VS_ERR_LAYOUT;
        if (d->max_blocks < 1 || d->num_blocks < 1 || d->stride_block < 0) return VS_ERR_LAYOUT;
        if (!d->block_table) return VS_ERR_NULL;
    } else if (d->stride_seq < 0 || d->capacity < 1) {
        return VS_ERR_LAYOUT;
    }
    if (d->T > (d->paged ? (int64_t)d->max_blocks * d->block_size : d->capacity)) return VS_ERR_LAYOUT;
    for (const int64_t s : {d->Hq > 0 ? d->q_stride : 0, d->Hq > 0 ? d->q_out_stride : 0, d->k_stride, d->v_stride, d->stride_tok, d->stride_head,
                            d->paged ? d->stride_block : d->stride_seq})
        if (s > ((int64_t)1 << 40) || (s * eb) % 16) return VS_ERR_LAYOUT;
    for (const void* at : {q, k, v, (const void*)q_out, (const void*)k_cache, (const void*)v_cache})
        if (!aligned16(at) && !(d->Hq == 0 && (at == q || at == q_out))) return VS_ERR_LAYOUT;
    // two slots in one place, or a key and a value: their writes would race
    if (k_cache == v_cache) return VS_ERR_LAYOUT;
    if (!rows_apart(d->d, d->paged ? d->block_size : d->capacity, d->stride_tok, d->Hkv, d->stride_head, d->paged ? d->num_blocks : d->B,
                    d->paged ? d->stride_block : d->stride_seq))
        return VS_ERR_LAYOUT;
    if (const int32_t dc = check_device()) return dc;
    p.q = q;
    p.k = k;
    p.v = v;
    p.positions = positions;
    p.depth = depth;
    p.pos_offset = pos_offset;
    p.prefix_len = prefix_len;
    p.row_start = row_start;
    p.q_out = q_out;
    p.k_cache = k_cache;
    p.v_cache = v_cache;
    p.status = status;
    p.block_table = d->paged ? d->block_table : nullptr;
    p.rows = d->rows;
    p.q_row = d->q_stride * eb;
    p.k_row = d->k_stride * eb;
    p.v_row = d->v_stride * eb;
    p.q_out_row = d->q_out_stride * eb;
    p.B = d->B;
    p.T = d->T;
    p.Hq = d->Hq;
    p.Hkv = d->Hkv;
    p.row_bytes = (int32_t)(d->d * eb);
    const RowCut cut = cut_rows(d->rows, d->Hq + 2 * d->Hkv, p.rope.chunks);
    p.rows_per_wg = cut.rows;
    p.heads_per_wg = cut.heads;
    p.by_T = fast_div_by(d->T);
    p.by_heads = fast_div_by(cut.heads);
    p.paged = d->paged ? 1 : 0;
    p.block_size = d->paged ? d->block_size : 1;
    while ((1 << p.block_shift) < p.block_size) ++p.block_shift;
    p.max_blocks = d->max_blocks;
    p.num_blocks = d->num_blocks;
    p.capacity = d->capacity;
    p.stride_seq = d->stride_seq * eb;
    p.stride_block = d->stride_block * eb;
    p.stride_head = d->stride_head * eb;
    p.stride_tok = d->stride_tok * eb;
    p.stream_out = streams_out(d->rows * (d->Hq + 2 * (int64_t)d->Hkv) * d->d * eb);
    return launch_kv_append(p, d->dtype, rope->pairing == VS_PAIR_HALVES, (hipStream_t)stream) == hipSuccess ? VS_OK : VS_ERR_HIP;
}

} // extern "C"
