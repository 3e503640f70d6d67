// Partial results of rows against the keys that all sequences share, and how a sequence's own part is joined with them.
//
// A row's softmax over shared and own keys is taken in parts: part i has a reference m_i (log2 domain), the sum l_i of its weights 2^(s - m_i) and
// the sum o_i of weights times values; with M the largest reference the row is sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i.
// The parts of the shared keys are written and read in fp32: a row is then rounded once, as if all its keys had been in one place.
#pragma once

#include "attn_mfma_common.h"

namespace vs {

// How many parts there are of the shared keys: none where their number is not one (which is reported), or zero.
__device__ __forceinline__ bool shared_ok(const SharedParams& p, int32_t len) { return len >= 0 && len <= p.max_shared && len <= p.sh_slots; }
__device__ __forceinline__ int shared_parts(const SharedParams& p) {
    const int32_t len = p.shared_len[0];
    return shared_ok(p, len) ? (len + p.sh_keys_per_split - 1) / p.sh_keys_per_split : 0;
}
// first element of (KV head, split, row)'s pair
__device__ __forceinline__ int64_t shared_row(const SharedParams& p, int kvh, int split, int row) {
    return ((int64_t)kvh * p.sh_splits + split) * p.sh_rows + row;
}
// Joins what a lane holds of a row - N groups of four channels, group i at channel at(i) - with the parts of the shared keys: `row` counts the rows of
// all sequences. On return o is to be multiplied by the returned factor.
template <int D, int N, typename At>
__device__ __forceinline__ float join_shared(const SharedParams& p, int kvh, int row, int parts, float m, float l, f32x4 (&o)[N], At at) {
    for (int s = 0; s < parts; ++s) {
        const int64_t r = shared_row(p, kvh, s, row);
        const f32x2 ml = *(const f32x2*)(p.sh_ml + r * 2);
        f32x4 x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = *(const f32x4*)(p.sh_acc + r * D + at(i));
        const float M = fmaxf(m, ml[0]), f = __builtin_amdgcn_exp2f(m - M), g = __builtin_amdgcn_exp2f(ml[0] - M);
        l = l * f + ml[1] * g;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] = o[i][e] * f + x[i][e] * g;
        m = M;
    }
    return 1.f / l;
}
// The workgroup that reports a sequence's status (all of its threads) also looks at what all sequences share. `own`: the code so far, which
// comes first, known to thread 0.
__device__ __forceinline__ void report_shared(const SharedParams& p, int b, int32_t* sflag) {
    if (!p.status) return;
    const int32_t len = p.shared_len[0];
    const bool ok = shared_ok(p, len);
    __syncthreads(); // sflag has been read
    if (threadIdx.x == 0) *sflag = 0;
    __syncthreads();
    if (ok && p.shared_table)
        for (int i = threadIdx.x; i < (len + (1 << p.sh_block_shift) - 1) >> p.sh_block_shift; i += blockDim.x)
            if ((uint32_t)p.shared_table[i] >= (uint32_t)p.sh_num_blocks) atomicOr(sflag, 8);
    __syncthreads();
    if (threadIdx.x == 0 && p.status[b] == VS_STATUS_OK) { // this thread's own store
        if (!ok) p.status[b] = VS_STATUS_BAD_PREFIX;
        else if (*sflag & 8) p.status[b] = VS_STATUS_BAD_BLOCK;
    }
    __syncthreads();
}

} // namespace vs
