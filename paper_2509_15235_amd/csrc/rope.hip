// Rotary positions on rows of heads: pair i of a row turns by (position on the pair's axis) * inv_freq[i].
//
// Bound by memory: every channel is read and written once, six operations a pair. A workgroup takes up to four rows and some of their
// heads; every wave works out one row's cosines and sines, a pair a lane (fp64 for the turns, see rope_device.h), once for all heads,
// while the rows are on their way; they go through LDS. Measured: 6684 rows of 32 heads of 128 bf16 channels, three axes, 17.2 us (6.4 TB/s of reads and writes,
// more than a plain copy reaches, see streams_out()); 2047 rows of 16 heads of 64 fp32 channels 4.8 us; one row 2.5 us, of which the launch is most.
#include "rope_device.h"

namespace vs {

namespace {

template <bool F32, bool HALVES, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeApplyParams p) {
    __shared__ f32x2 cs[kRopeRows][kMaxRopePairs];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_wg;
    const int rows = (int)min((int64_t)p.rows_per_wg, p.rows - row0), h0 = blockIdx.y * p.heads_per_wg;
    const int heads = min(p.heads_per_wg, p.H - h0), items = rows * p.heads_per_wg * p.rope.chunks;
    u32x4 a[kRopeBatch], b[kRopeBatch];
    int64_t to[kRopeBatch]; // bytes; -1: no item
    int where[kRopeBatch];  // row << 16 | item of the head
    auto load = [&](int first) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kRopeBatch; ++u) {
            uint32_t c, h;
            const uint32_t t = fast_div(fast_div((uint32_t)(first + u * kRopeThreads), p.rope.by_chunks, c), p.by_heads, h);
            to[u] = -1;
            if (first + u * kRopeThreads >= items || (int)h >= heads) continue;
            int piece;
            const bool turns = rope_item<HALVES>(p.rope, (int)c, piece);
            const char* at = (const char*)p.x + (row0 + t) * p.x_row + (h0 + (int)h) * p.x_head + piece * 16;
            a[u] = *(const u32x4*)at;
            if (HALVES && turns) b[u] = *(const u32x4*)(at + p.rope.turning * 16);
            to[u] = (row0 + t) * p.out_row + (h0 + (int)h) * p.out_head + piece * 16;
            where[u] = (int)(t << 16 | c);
        }
    };
    load(tid);
    if (wave < rows)
        for (int i = lane; i < p.rope.pairs; i += kWave)
            cs[wave][i] = rope_angle<F32>(p.rope, p.positions[(int64_t)rope_axis(p.rope, i) * p.rope.stride_axis + row0 + wave], p.rope.inv_freq[i]);
    __syncthreads();
    for (int first = tid;;) {
#pragma unroll
        for (int u = 0; u < kRopeBatch; ++u) {
            if (to[u] < 0) continue;
            const int c = where[u] & 0xffff;
            const bool turns = c < p.rope.turning;
            if (turns) rope_turn<F32, HALVES>(a[u], b[u], cs[where[u] >> 16], c);
            put<STREAM>((char*)p.out + to[u], a[u]);
            if (HALVES && turns) put<STREAM>((char*)p.out + to[u] + p.rope.turning * 16, b[u]);
        }
        first += kRopeBatch * kRopeThreads;
        if (first - tid >= items) break;
        load(first);
    }
}

template <bool F32, bool HALVES>
void launch(const RopeApplyParams& p, dim3 grid, hipStream_t s) {
    if (p.stream_out) hipLaunchKernelGGL((rope_kernel<F32, HALVES, true>), grid, dim3(kRopeThreads), 0, s, p);
    else hipLaunchKernelGGL((rope_kernel<F32, HALVES, false>), grid, dim3(kRopeThreads), 0, s, p);
}

} // namespace

hipError_t launch_rope(RopeApplyParams p, int dtype, bool halves, hipStream_t s) {
    for (int64_t left = p.rows; left > 0; left -= kRopeLaunchRows) {
        p.rows = min(left, kRopeLaunchRows);
        const dim3 grid((unsigned)((p.rows + p.rows_per_wg - 1) / p.rows_per_wg), (unsigned)((p.H + p.heads_per_wg - 1) / p.heads_per_wg));
        if (dtype == VS_F32) halves ? launch<true, true>(p, grid, s) : launch<true, false>(p, grid, s);
        else halves ? launch<false, true>(p, grid, s) : launch<false, false>(p, grid, s);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        p.x = (const char*)p.x + p.rows * p.x_row;
        p.out = (char*)p.out + p.rows * p.out_row;
        p.positions += p.rows;
    }
    return hipSuccess;
}

} // namespace vs
