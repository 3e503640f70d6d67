// Attention behind a shared prefix by waves with key tiles of their own (attention_mfma_rows.hip): all sequences' rows against the shared keys, a
// sequence's rows against its own, or both in one launch.
//
// What bounds them: keys that no other workgroup reads come from memory once, so a batch of decoded tokens is bound by its bytes (32 x 1 token of 32 / 32 heads behind 4099
// keys, up to 300 own ones: 67 MB of shared keys in 13.7 us, 4.9 TB/s, the own ones' 87 in 27, workgroups that begin and end); a few rows by the
// trips in a row - length, tiles, merge of the waves, arrival, join - 10.3 us for 4 x 1 token of 28 / 4 heads behind 1696 keys, one launch. From some 200 rows of a KV head
// on the matrix instructions bound the call, and the pipelined kernel takes the shared keys (attention_mfma_pipe.hip); which way a call goes is api_shared.hip's.
#include "attn_rows_kernel.h"

namespace vs {

namespace {
template <int D, int NW, int RB, int MODE>
hipError_t launch_shared(const SharedParams& p, hipStream_t s) {
    const dim3 grid(round_up8(p.total_wgs) + (MODE == kRowsOwn && p.status ? (p.B + NW - 1) / NW : 0)), block(NW * kWave);
    if (p.once && p.paged) return hipErrorInvalidValue;
    constexpr bool ONCE = D == 128 && RB == 1 && NW >= 4;
    if (p.once && !ONCE) return hipErrorInvalidValue;
    if (p.once) hipLaunchKernelGGL((attn_shared_rows_kernel<D, NW, RB, false, ONCE, MODE>), grid, block, 0, s, p);
    else if (p.paged) hipLaunchKernelGGL((attn_shared_rows_kernel<D, NW, RB, true, false, MODE>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((attn_shared_rows_kernel<D, NW, RB, false, false, MODE>), grid, block, 0, s, p);
    return hipGetLastError();
}
template <int D>
hipError_t launch_shared_own(const SharedParams& p, int waves, hipStream_t s) { // eight waves, or four (64 channels: two)
    constexpr int FEW = D == 128 ? 4 : 2;
    return waves == 8 ? launch_shared<D, 8, 1, kRowsOwn>(p, s) : waves == FEW ? launch_shared<D, FEW, 1, kRowsOwn>(p, s) : hipErrorInvalidValue;
}

template <int D, int NW>
hipError_t launch_both(const BothParams& p, hipStream_t s) {
    const SharedParams& own = p.work[0];
    const dim3 grid(round_up8(p.work[1].total_wgs) + round_up8(own.total_wgs) + (own.status ? (own.B + NW - 1) / NW : 0)), block(NW * kWave);
    if (own.paged) hipLaunchKernelGGL((attn_shared_rows_kernel<D, NW, 1, true, false, kRowsBoth>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((attn_shared_rows_kernel<D, NW, 1, false, false, kRowsBoth>), grid, block, 0, s, p);
    return hipGetLastError();
}
} // namespace

hipError_t launch_attention_shared_both(const SharedParams& shared, const SharedParams& own, int waves, hipStream_t s) {
    if (shared.rows_per_group != kRowBlock || own.rows > kRowBlock || own.row_groups != 1 || own.num_splits != 1 || shared.paged != own.paged) return hipErrorInvalidValue;
    if ((waves != 4 && waves != 8) || (own.d != 64 && own.d != 128) || shared.sh_splits != shared.num_splits + 1) return hipErrorInvalidValue;
    const BothParams p{{own, shared}};
    if (own.d == 128) return waves == 8 ? launch_both<128, 8>(p, s) : launch_both<128, 4>(p, s);
    return waves == 8 ? launch_both<64, 8>(p, s) : launch_both<64, 4>(p, s);
}

hipError_t launch_attention_shared_rows(const SharedParams& p, RowsMode mode, int waves, hipStream_t s) {
    const int blocks = p.rows_per_group / kRowBlock;
    if (p.row_groups * p.rows_per_group < p.rows || (p.d != 64 && p.d != 128) || blocks < 1 || blocks > (p.d == 128 ? 2 : 1)) return hipErrorInvalidValue;
    if (p.keys_per_split % kIterKeys || (mode == kRowsOwn && p.num_splits != 1)) return hipErrorInvalidValue;
    if (mode == kRowsOwn && blocks != 1) return hipErrorInvalidValue;
    if (mode == kRowsOwn) return p.d == 128 ? launch_shared_own<128>(p, waves, s) : launch_shared_own<64>(p, waves, s);
    if (waves != 8) return hipErrorInvalidValue;
    if (p.d == 64) return launch_shared<64, 8, 1, kRowsShared>(p, s);
    return blocks == 2 ? launch_shared<128, 8, 2, kRowsShared>(p, s) : launch_shared<128, 8, 1, kRowsShared>(p, s);
}

} // namespace vs
