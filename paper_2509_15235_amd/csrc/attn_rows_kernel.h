// The kernel of own key tiles (attention_mfma_rows.hip says what it is for, its mathematics and figures), for whole attention and for its halves with
// keys that all sequences share (attention_shared_rows.hip).
#pragma once
#include <type_traits>

#include "attn_shared.h"

namespace vs {

// NW waves, RB row blocks. (PAGED is part of the kernel for the scalar registers: with a branch 14 of them were spilled, in the loop over the
// tiles too: 4 x 60 nodes, 32 / 32 heads, 3100 keys 39.7 -> 39.2 us, one sequence of 484 keys and four nodes 7.4 -> 7.2.)
// ONCE: tiles as data that is read once (the host's rule says when). Part of the kernel as well: a branch at every load 5 % of two row blocks'
// time, a loop of its own for either kind 3 % of a short call's.
// CROWD: many splits on nearly all CUs, whose workgroups wait for each other at another word (merge_meet).
// MODE (attn_shared.h): kRowsShared, all sequences' rows against the keys that they share (one sequence of B * T nodes, no tree slots), whose results stay
// partial ones; kRowsOwn, a sequence's rows against its own keys, joined with those;
// kRowsBoth, workgroups of either kind in one launch, and those that report.
struct BothParams {
    SharedParams work[2]; // the sequences' own keys, the shared ones
};
template <int MODE>
using RowsArgs = std::conditional_t<MODE == kRowsWhole, AttnParams, std::conditional_t<MODE == kRowsBoth, BothParams, SharedParams>>;
template <int MODE>
__device__ __forceinline__ const auto& rows_params(const RowsArgs<MODE>& args, bool shared_work) {
    // (out of the arguments' own place: an element of a local copy that is chosen at run time would have the copy in scratch memory)
    if constexpr (MODE == kRowsBoth) return *((const SharedParams*)(const void*)__builtin_amdgcn_kernarg_segment_ptr() + (shared_work ? 1 : 0));
    else return args;
}
template <int D, int NW, int RB, bool PAGED, bool ONCE, bool CROWD = false, int MODE = kRowsWhole>
__global__ __launch_bounds__(NW * 64, 2) void attn_mfma_rows_kernel(const RowsArgs<MODE> p) {
    const auto& args = p;
    constexpr bool shared_work = false;
    const uint32_t id = blockIdx.x;
#include "attn_rows_body.h"
}

template <int D, int NW, int RB, bool PAGED, bool ONCE, int MODE>
__global__ __launch_bounds__(NW * 64, 2) void attn_shared_rows_kernel(const RowsArgs<MODE> args) {
    constexpr bool CROWD = false;
    // kRowsBoth: the workgroups of the shared keys come first; what this one works on, and its number there
    bool shared_work = MODE == kRowsShared;
    uint32_t id = blockIdx.x;
    if constexpr (MODE == kRowsBoth) {
        const uint32_t first = round_up8(args.work[1].total_wgs), end = first + round_up8(args.work[0].total_wgs);
        shared_work = id < first;
        if (id >= end) {
            report_shared(args.work[0], end);
            return;
        }
        if (!shared_work) id -= first;
    }
    const auto& p = rows_params<MODE>(args, shared_work);
#include "attn_rows_body.h"
}

} // namespace vs
