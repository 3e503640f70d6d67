// Tree-masked attention for launches of few query rows per KV head (one or two row blocks): every wave has key tiles of
// its own.
//
// Math and MFMA layouts are those of attention_mfma.hip (paper Eq. 1 with a softmax scale over the prefix plus the
// ancestor-or-self tree slots, Section 3.1): S^T = K . Q^T with v_mfma_f32_32x32x16_bf16, a lane holds 16 keys of ONE
// query row, the probabilities are the B operand of O^T += V^T . P^T, V is transposed by ds_read_b64_tr_b16 on its way
// out of LDS.
//
// What bounds it: with 32 or 64 rows a 16 KB tile of K and V keeps a SIMD busy for a tenth to a quarter of the time
// in which it comes from memory, so the bytes in flight decide (a CU's share of 6 TB/s times 1.5 us of latency is 35 KB).
// The kernels that share tiles among their waves pay a barrier per tile and leave waves without rows idle. Here the
// waves of a workgroup take the 32-key tiles of a split in turn, each for all rows: a tile goes from memory straight into
// LDS of the wave's own, keys and values by turns (64 to 128 KB in flight per CU), with no barrier anywhere in the
// loop. Through registers the same took 5 % longer at the start of a launch and left no room for a second row
// block. The waves' results are merged through LDS (log-sum-exp), the splits as in merge_splits.
// us per call, before / this kernel (28 / 4 or 32 / 32 heads of 128 channels unless stated):
//   1 x 4 nodes, 484 keys 14.2 / 7.6; 16 x 4 nodes, 1024 .. 8191 keys paged 62.6 / 35.2; 64 x 4 nodes, 8000 keys 304 / 180
//   (5.8 TB/s); 4 x 4 nodes, 32 KV heads, 3100 keys 47.4 / 41.1; 16 x 20 nodes, 16 / 16 heads of 64, up to 3000 keys 46.4 / 31.4;
//   two row blocks: 64 x 9 nodes, 1024 .. 8191 keys 178 / 129; 8 x 60 nodes, 32 / 32 heads, up to 8000 keys 164 / 132.
// (Three and four row blocks, one wave per SIMD with 512 registers, lost: 16 x 13 nodes, up to 8191 keys 57 / 79.)
#include "attn_rows_kernel.h"

namespace vs {

namespace {
template <int D, int NW, int RB>
hipError_t launch_rows(const AttnParams& p, hipStream_t s) {
    const dim3 grid(((p.total_wgs + 7) / 8) * 8);
    if (p.once && p.paged) return hipErrorInvalidValue;
    if constexpr (NW == 8 && RB == 1)
        if (p.crowd) {
            if (p.paged) hipLaunchKernelGGL((attn_mfma_rows_kernel<D, NW, RB, true, false, true>), grid, dim3(NW * kWave), 0, s, p);
            else hipLaunchKernelGGL((attn_mfma_rows_kernel<D, NW, RB, false, false, true>), grid, dim3(NW * kWave), 0, s, p);
            return hipGetLastError();
        }
    if (p.once) hipLaunchKernelGGL((attn_mfma_rows_kernel<D, NW, RB, false, true>), grid, dim3(NW * kWave), 0, s, p);
    else if (p.paged) hipLaunchKernelGGL((attn_mfma_rows_kernel<D, NW, RB, true, false>), grid, dim3(NW * kWave), 0, s, p);
    else hipLaunchKernelGGL((attn_mfma_rows_kernel<D, NW, RB, false, false>), grid, dim3(NW * kWave), 0, s, p);
    return hipGetLastError();
}
} // namespace

// One row block and four or eight waves; with 128 channels also two row blocks and eight waves.
bool attention_rows_supported(int d, int row_blocks, int waves) {
    return (row_blocks == 1 && (waves == 4 || waves == 8)) || (d == 128 && row_blocks == 2 && waves == 8);
}

hipError_t launch_attention_mfma_rows(const AttnParams& p, int waves, hipStream_t s) {
    const int blocks = p.rows_per_group / kRowBlock;
    if (p.row_groups * p.rows_per_group != p.rows_pad || (p.by_length && p.row_groups != 1)) return hipErrorInvalidValue;
    if (p.keys_per_split % kIterKeys || !attention_rows_supported(p.d, blocks, waves)) return hipErrorInvalidValue;
    if (p.d == 128) return blocks == 2 ? launch_rows<128, 8, 2>(p, s) : waves == 8 ? launch_rows<128, 8, 1>(p, s) : launch_rows<128, 4, 1>(p, s);
    if (p.d == 64) return waves == 8 ? launch_rows<64, 8, 1>(p, s) : launch_rows<64, 4, 1>(p, s);
    return hipErrorInvalidValue;
}

} // namespace vs
