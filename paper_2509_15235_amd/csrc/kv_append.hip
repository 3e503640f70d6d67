// New tokens of one layer into the caches, their positions applied on the way: queries and keys turn like in rope.hip, keys and values
// go to slot prefix_len + i of their sequence's cache.
//
// Bound by memory (every channel is read and written once), and for a few tokens by the trips in a row: which sequence a row belongs to, its
// prefix length, its block id. A workgroup takes up to four consecutive rows, whatever sequences they belong to - so packed sequences
// of very different lengths leave no workgroup idle - and some of their heads; wave w finds row w's sequence (the row_start entries that do not
// lie behind it are counted 64 at a time), works out its slot and its angles, while all threads' first pieces are on their way.
// Measured, 28 / 4 heads of 128 bf16 channels: twelve packed prompts of 7712 rows in all 24.0 us (5.9 TB/s); 16 trees of 60 nodes, paged, 6.0 us; one token 3.5 us.
#include "rope_device.h"

namespace vs {

namespace {

template <bool F32, bool HALVES, bool PAGED, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void kv_append_kernel(const AppendParams p) {
    __shared__ f32x2 cs[kRopeRows][kMaxRopePairs];
    __shared__ int64_t slot_at[kRopeRows]; // bytes from the caches' start to the row's slot of head 0; -1: none
    __shared__ int32_t live[kRopeRows];    // whether the row belongs to a sequence
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row0 = p.first_row + (int)blockIdx.x * p.rows_per_wg;
    const int rows = min(p.rows_per_wg, (int)(p.rows - row0)), h0 = blockIdx.y * p.heads_per_wg;
    const int all_heads = p.Hq + 2 * p.Hkv;
    const int heads = min(p.heads_per_wg, all_heads - h0), items = rows * p.heads_per_wg * p.rope.chunks;
    const int row_bytes = p.row_bytes; // of a head
    u32x4 a[kRopeBatch], b[kRopeBatch];
    int where[kRopeBatch]; // row << 28 | head << 8 | item of the head; -1: no item
    auto load = [&](int first) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kRopeBatch; ++u) {
            uint32_t c, h;
            const uint32_t t = fast_div(fast_div((uint32_t)(first + u * kRopeThreads), p.rope.by_chunks, c), p.by_heads, h);
            where[u] = -1;
            if (first + u * kRopeThreads >= items || (int)h >= heads) continue;
            const int head = h0 + (int)h;
            int piece;
            const bool turns = rope_item<HALVES>(p.rope, (int)c, piece);
            const int64_t row = row0 + (int)t;
            const char* at = head < p.Hq            ? (const char*)p.q + row * p.q_row + head * row_bytes
                             : head < p.Hq + p.Hkv ? (const char*)p.k + row * p.k_row + (head - p.Hq) * row_bytes
                                                   : (const char*)p.v + row * p.v_row + (head - p.Hq - p.Hkv) * row_bytes;
            a[u] = *(const u32x4*)(at + piece * 16);
            if (HALVES && turns) b[u] = *(const u32x4*)(at + piece * 16 + p.rope.turning * 16);
            where[u] = (int)(t << 28 | (uint32_t)head << 8 | c);
        }
    };
    load(tid);

    // ---- wave w: row w's sequence, slot and angles
    const int64_t have = min(PAGED ? (int64_t)p.max_blocks << p.block_shift : p.capacity, (int64_t)INT32_MAX); // (a prefix length has 32 bits)
    if (wave < rows) {
        const int row = row0 + wave;
        int seq, i, n = p.T;
        bool mine = true;
        if (p.row_start) {
            seq = 0;
            for (int first = 0; first < p.B; first += kWave) {
                const int end = first + lane < p.B ? p.row_start[first + lane + 1] : INT32_MAX;
                seq += __popcll(__ballot(end <= row));
            }
            mine = seq < p.B;
            seq = min(seq, p.B - 1);
            const int start = p.row_start[seq], end = p.row_start[seq + 1];
            i = (int)((uint32_t)row - (uint32_t)start);
            n = (int)((uint32_t)end - (uint32_t)start);
            mine = mine && start >= 0 && i >= 0 && row < end && end <= (int)p.rows && n <= p.T; // (the last: 0 <= start <= end)
        } else {
            uint32_t r;
            seq = (int)fast_div((uint32_t)row, p.by_T, r);
            i = (int)r;
        }
        const int32_t S = p.prefix_len[seq];
        const bool fits = mine && S >= 0 && (int64_t)S + n <= have;
        int64_t to = -1;
        if (fits) {
            const int slot = S + i;
            if constexpr (PAGED) {
                const int32_t blk = p.block_table[(int64_t)seq * p.max_blocks + (slot >> p.block_shift)];
                if ((uint32_t)blk < (uint32_t)p.num_blocks) to = blk * p.stride_block + (int64_t)(slot & (p.block_size - 1)) * p.stride_tok;
            } else {
                to = seq * p.stride_seq + (int64_t)slot * p.stride_tok;
            }
        }
        if (lane == 0) {
            slot_at[wave] = to;
            live[wave] = mine;
        }
        int32_t pos = 0;
        if (!p.positions) pos = (int32_t)((uint32_t)S + (uint32_t)(p.pos_offset ? p.pos_offset[seq] : 0) + (uint32_t)(p.depth ? p.depth[row] : i));
        for (int j = lane; j < p.rope.pairs; j += kWave) {
            const int32_t at = p.positions ? p.positions[(int64_t)rope_axis(p.rope, j) * p.rope.stride_axis + row] : pos;
            cs[wave][j] = rope_angle<F32>(p.rope, at, p.rope.inv_freq[j]);
        }
    }
    __syncthreads();
    for (int first = tid;;) {
#pragma unroll
        for (int u = 0; u < kRopeBatch; ++u) {
            if (where[u] < 0) continue;
            const int t = where[u] >> 28, head = (where[u] >> 8) & 0xfffff, c = where[u] & 0xff;
            int piece;
            const bool turns = rope_item<HALVES>(p.rope, c, piece);
            if (turns && head < p.Hq + p.Hkv) rope_turn<F32, HALVES>(a[u], b[u], cs[t], c);
            char* to;
            if (head < p.Hq) {
                if (!live[t]) continue;
                to = (char*)p.q_out + (int64_t)(row0 + t) * p.q_out_row + head * row_bytes;
            } else {
                if (slot_at[t] < 0) continue;
                to = (head < p.Hq + p.Hkv ? (char*)p.k_cache + (head - p.Hq) * p.stride_head : (char*)p.v_cache + (head - p.Hq - p.Hkv) * p.stride_head) + slot_at[t];
            }
            put<STREAM>(to + piece * 16, a[u]);
            if (HALVES && turns) put<STREAM>(to + piece * 16 + p.rope.turning * 16, b[u]);
        }
        first += kRopeBatch * kRopeThreads;
        if (first - tid >= items) break;
        load(first);
    }
    // ---- status: a wave a sequence
    if (!p.status || blockIdx.y != 0) return;
    for (int64_t seq = (int64_t)blockIdx.x * kRopeRows + wave; seq < p.B; seq += (int64_t)gridDim.x * kRopeRows) {
        int n = p.T, code = VS_STATUS_OK;
        if (p.row_start) {
            const int start = p.row_start[seq], end = p.row_start[seq + 1];
            n = (int)((uint32_t)end - (uint32_t)start);
            if (start < 0 || end < start || end > (int)p.rows || n > p.T) code = VS_STATUS_BAD_ROWS;
        }
        const int32_t S = p.prefix_len[seq];
        if (code == VS_STATUS_OK && (S < 0 || (int64_t)S + n > have)) code = VS_STATUS_BAD_PREFIX;
        if (PAGED && code == VS_STATUS_OK && n > 0) {
            bool bad = false;
            for (int j = (S >> p.block_shift) + lane; j <= (S + n - 1) >> p.block_shift; j += kWave)
                bad |= (uint32_t)p.block_table[seq * p.max_blocks + j] >= (uint32_t)p.num_blocks;
            if (__any(bad)) code = VS_STATUS_BAD_BLOCK;
        }
        if (lane == 0) p.status[seq] = code;
    }
}

template <bool F32, bool HALVES, bool STREAM>
void launch(const AppendParams& p, dim3 grid, hipStream_t s) {
    if (p.paged) hipLaunchKernelGGL((kv_append_kernel<F32, HALVES, true, STREAM>), grid, dim3(kRopeThreads), 0, s, p);
    else hipLaunchKernelGGL((kv_append_kernel<F32, HALVES, false, STREAM>), grid, dim3(kRopeThreads), 0, s, p);
}
template <bool F32, bool HALVES>
void launch(const AppendParams& p, dim3 grid, hipStream_t s) { p.stream_out ? launch<F32, HALVES, true>(p, grid, s) : launch<F32, HALVES, false>(p, grid, s); }

} // namespace

hipError_t launch_kv_append(AppendParams p, int dtype, bool halves, hipStream_t s) {
    const int all_heads = p.Hq + 2 * p.Hkv;
    for (int64_t first = 0; first < p.rows; first += kRopeLaunchRows) {
        const int64_t rows = min(p.rows - first, kRopeLaunchRows);
        const dim3 grid((unsigned)((rows + p.rows_per_wg - 1) / p.rows_per_wg), (unsigned)((all_heads + p.heads_per_wg - 1) / p.heads_per_wg));
        p.first_row = (int32_t)first;
        if (dtype == VS_F32) halves ? launch<true, true>(p, grid, s) : launch<true, false>(p, grid, s);
        else halves ? launch<false, true>(p, grid, s) : launch<false, false>(p, grid, s);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        p.status = nullptr; // all sequences' are written
    }
    return hipSuccess;
}

} // namespace vs
