// Partial results of rows against the keys that all sequences share, and how a sequence's own part is joined with them.
//
// A row's softmax over shared and own keys is taken in parts: part i has a reference m_i (log2 domain), the sum l_i of its weights 2^(s - m_i) and the
// weighted mean o_i of its values; with M the largest reference the row is sum_i 2^(m_i - M) l_i o_i / sum_i 2^(m_i - M) l_i.
// References and sums are fp32. fp32 storage keeps fp32 means too. For bf16 storage they are what a call writes and reads most of beside K and V (16 x 60
// nodes of 28 / 4 heads, three parts or so of every row: 47 MB in fp32), so they are kept as fp16 with a power of two of its own for every 16 channels
// of a row: 11 bits for every normal number, as long as 2^29 do not lie between them (else eight, see pack_means). That rounding, 2^-11 at most, is an eighth of the
// result's own, 2^-8 at most; a bf16 mean would add as much as either of the two roundings to bf16, the weights' and the result's.
#pragma once

#include "attn_mfma_common.h"

namespace vs {

// The last entry of a block table's row that may be read. Behind a shared prefix rows may begin inside a longer row: max_blocks is their distance only,
// and behind the last entry that a key may lie in there need be none. (Its number stands in place of a contiguous cache's capacity, in a line of the arguments that is
// there by then: out of the lengths' line it took 4 x 1 token 10.45 us, so 10.28; reading to the row's end, behind which a table may end, 10.06.)
__device__ __forceinline__ int32_t last_entry(const AttnParams& p) { return p.max_blocks - 1; }
__device__ __forceinline__ int32_t last_entry(const SharedParams& p) { return (int32_t)p.capacity; }

__device__ __forceinline__ bool shared_ok(const SharedParams& p, int32_t len) { return len >= 0 && len <= p.max_shared && len <= p.sh_slots; }

// ---- Shares: a unit - (KV head, row group) - has as many steps of 64 keys as the longest allowed prefix; all units lie end to end in one line that is
// cut into shares, or each in a line of its own. The first sh_longer shares of a line take sh_steps + 1 steps, the others sh_steps. A unit's
// parts are the pieces of consecutive shares. (By the host's bound, not by the length: the divisions that the length would take, and the trip for
// it, stood in front of every first tile.)
__device__ __forceinline__ uint32_t share_begin(const SharedParams& p, uint32_t w) { // of a line's last share + 1: the next line's begin
    uint32_t i;
    const uint32_t line = fast_div(w, p.sh_by_line, i);
    return line * p.sh_by_line_steps.d + i * (uint32_t)p.sh_steps + min(i, (uint32_t)p.sh_longer);
}
__device__ __forceinline__ int share_of(const SharedParams& p, uint32_t step) {
    const uint32_t longer = (uint32_t)p.sh_longer * (uint32_t)(p.sh_steps + 1);
    uint32_t x, rest;
    const uint32_t line = fast_div(step, p.sh_by_line_steps, x);
    return (int)(line * p.sh_by_line.d + (x < longer ? fast_div(x, p.sh_by_longer, rest) : (uint32_t)p.sh_longer + fast_div(x - longer, p.sh_by_share, rest)));
}

// How many parts there are of a row against the shared keys (none where their number is not one, which is reported, or zero).
__device__ __forceinline__ int shared_parts(const SharedParams& p, int32_t len, int kvh, int row) {
    if (!shared_ok(p, len) || len == 0) return 0;
    if (p.sh_shares == 0) return (len + p.sh_keys_per_split - 1) / p.sh_keys_per_split;
    const uint32_t steps = (uint32_t)(len + kIterKeys - 1) / kIterKeys;
    uint32_t rest;
    const uint32_t first = ((uint32_t)kvh * p.sh_groups + fast_div((uint32_t)row, p.sh_by_rows, rest)) * p.sh_by_steps.d;
    return share_of(p, first + steps - 1) - share_of(p, first) + 1;
}
// Number of (KV head, part, row). fp32 storage: its pair (m, l) and its d sums of weights times values lie there.
__device__ __forceinline__ int64_t shared_row(const SharedParams& p, int kvh, int part, int row) {
    return ((int64_t)kvh * p.sh_splits + part) * p.sh_rows + row;
}
// bf16 storage: sixteen bytes of m, l and the exponents of the row's pieces of 16 channels, and the means as the accumulators hold them, so that whoever
// writes or reads them moves runs of memory: the sixteen bytes of channels 16 pc + 4 half .. + 3 and 8 behind those of row r are number
// ((block of r) * D / 16 + pc) * 64 + 32 half + r % 32 of the part.
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
template <int D>
__device__ __forceinline__ char* shared_means(const SharedParams& p, int kvh, int part, int row, int half) {
    const int64_t block = ((int64_t)kvh * p.sh_splits + part) * p.sh_blocks + (row >> 5);
    return (char*)p.sh_acc + (block * (D / 16) * 64 + half * 32 + (row & 31)) * 16;
}
__device__ __forceinline__ char* shared_head(const SharedParams& p, int kvh, int part, int row) { return (char*)p.sh_ml + shared_row(p, kvh, part, row) * 16; }
// Eight values (both halves' are one piece) as fp16; `exponent`: what gives them back, plus 128, where the largest becomes 2^14 .. 2^15. The largest finite
// one, that is: infinities and NaN of a channel, which stay what they are, cost its neighbours nothing. Nor does a channel that is 2^29 times another
// one, or more: such a piece is kept as bf16, exponent 0, at the price of three bits. The smallest normal number times 2^112 is fp16's smallest: no larger power is
// needed, and a weight divided by it has bits left (2^-14, the least that can matter beside a weight of one there, becomes 2^-126).
__device__ __forceinline__ u32x4 pack_means(const float (&x)[8], uint32_t& exponent) {
    float top = 0.f, low = -INFINITY; // twice the powers of two at or below the largest and (negative) the smallest, zeros aside
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float power = __uint_as_float((__float_as_uint(x[e]) + 0x800000u) & 0x7f800000u); // (the exponent of infinity and NaN wraps to zero)
        top = fmaxf(top, power);
        low = fmaxf(low, __builtin_amdgcn_classf(x[e], 0x267) ? -INFINITY : -power); // (zero, infinity, NaN)
    }
    top = half_max(top);
    low = half_max(low);
    const int k = min(142 - (int)(__float_as_uint(top) >> 23), 112);
    exponent = (uint32_t)(128 - k);
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const f32x2 v = {__builtin_amdgcn_ldexpf(x[2 * e], k), __builtin_amdgcn_ldexpf(x[2 * e + 1], k)};
        w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    }
    if (low * -0x1p28f < top) [[unlikely]] { // (the smallest's eleven bits end at fp16's last one)
        exponent = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f32x2 v = {x[2 * e], x[2 * e + 1]};
            w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
        }
    }
    return w;
}

// A row that sees no key of a part has the reference -inf there, its weights and sums are zero. Where it sees none at all, this is what they are relative to (else
// the differences of references would be NaN), and its result is zeros.
__device__ __forceinline__ float finite_reference(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float one_over_sum(float l) { return l == 0.f ? 0.f : 1.f / l; }

// ---- Joining a row's own part with its parts against the shared keys. Those were written by the launch before, so the first of
// them are asked for when a workgroup begins, and are there when its own keys are done.
struct SharedRow { // a lane's row
    int parts;
    const char* head;   // of its first part
    const char* means;  // its sixteen bytes of piece 0 in the first part
    int64_t head_step, step; // bytes from a part to the next
};
template <int D>
__device__ __forceinline__ SharedRow shared_at(const SharedParams& p, int32_t len, int kvh, int row, int half) {
    return {shared_parts(p, len, kvh, row), shared_head(p, kvh, 0, row), shared_means<D>(p, kvh, 0, row, half), (int64_t)p.sh_rows * 16, (int64_t)p.sh_blocks * (kRowBlock * D * 2)};
}
constexpr int kJoinHeads = 8; // references in flight
__device__ __forceinline__ uint32_t piece_exponent(const u32x4& head, int pc) { return ((pc < 4 ? head[2] : head[3]) >> (8 * (pc & 3))) & 0xff; }
// N parts from s0 on, G pieces from pc on. Past the last part the last one again.
template <int N, int G>
struct JoinParts {
    u32x4 head[N];
    u32x4 x[N][G];
};
template <int N, int G>
__device__ __forceinline__ void load_parts(const SharedRow& r, int s0, int pc, JoinParts<N, G>& j) {
    const int last = max(r.parts - 1, 0); // (no parts: the first place, which is there, is read and not used)
#pragma unroll
    for (int s = 0; s < N; ++s) {
        const int64_t part = min(s0 + s, last);
        j.head[s] = *(const u32x4*)(r.head + part * r.head_step);
#pragma unroll
        for (int i = 0; i < G; ++i) j.x[s][i] = *(const u32x4*)(r.means + part * r.step + (pc + i) * 1024);
    }
}
// The common reference of a row's own part (reference m) and all others.
template <int N, int G>
__device__ __forceinline__ float join_reference(const SharedRow& r, const JoinParts<N, G>& first, float m) {
#pragma unroll
    for (int s = 0; s < N; ++s) m = s < r.parts ? fmaxf(m, __uint_as_float(first.head[s][0])) : m;
    for (int s0 = N; s0 < r.parts; s0 += kJoinHeads) {
        float x[kJoinHeads];
#pragma unroll
        for (int s = 0; s < kJoinHeads; ++s) x[s] = *(const float*)(r.head + (int64_t)min(s0 + s, r.parts - 1) * r.head_step);
#pragma unroll
        for (int s = 0; s < kJoinHeads; ++s) m = fmaxf(m, x[s]);
    }
    return m;
}
// Adds parts to sums that are relative to the reference M, and to the sum of weights l. WIDE: some pieces may be bf16.
template <bool WIDE, int N, int G>
__device__ __forceinline__ void add_parts(const SharedRow& r, int s0, int pc, const JoinParts<N, G>& j, float M, float& l, float (&o)[G][8]) {
#pragma unroll
    for (int s = 0; s < N; ++s) {
        const bool there = s0 + s < r.parts;
        const float w = there ? __builtin_amdgcn_exp2f(__uint_as_float(j.head[s][0]) - M) * __uint_as_float(j.head[s][1]) : 0.f;
        l += w;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const uint32_t exponent = piece_exponent(j.head[s], pc + i);
            const bool wide = WIDE && exponent == 0;
            const float f = wide ? w : __builtin_amdgcn_ldexpf(w, (int)exponent - 128);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t two = j.x[s][i][e]; // (a cast of the vector's element itself takes the first one)
                const f16x2 v = __builtin_bit_cast(f16x2, two);
                const float lo = wide ? __uint_as_float(two << 16) : (float)v[0], hi = wide ? __uint_as_float(two & 0xffff0000u) : (float)v[1];
                o[i][2 * e] = there ? fmaf(lo, f, o[i][2 * e]) : o[i][2 * e];
                o[i][2 * e + 1] = there ? fmaf(hi, f, o[i][2 * e + 1]) : o[i][2 * e + 1];
            }
        }
    }
}
template <int N, int G>
__device__ __forceinline__ void join_parts(const SharedRow& r, int s0, int pc, const JoinParts<N, G>& j, float M, float& l, float (&o)[G][8]) {
    bool wide = false;
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
        for (int i = 0; i < G; ++i) wide |= piece_exponent(j.head[s], pc + i) == 0;
    if (__any(wide)) [[unlikely]] add_parts<true>(r, s0, pc, j, M, l, o);
    else add_parts<false>(r, s0, pc, j, M, l, o);
}
// All of it: j holds the first N parts; on return o, G pieces from pc on, is to be divided by l (one_over_sum).
template <int N, int G>
__device__ __forceinline__ void join_row(const SharedRow& r, int pc, JoinParts<N, G>& j, float m, float& l, float (&o)[G][8]) {
    const float M = finite_reference(join_reference(r, j, m)), f = __builtin_amdgcn_exp2f(m - M);
    l *= f;
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) o[i][e] *= f;
    join_parts(r, 0, pc, j, M, l, o);
    for (int s0 = N; s0 < r.parts; s0 += N) {
        load_parts(r, s0, pc, j);
        join_parts(r, s0, pc, j, M, l, o);
    }
}
// ---- One launch for both kinds of work, where all workgroups run at once: parts then travel between them by stores and loads of device scope, and whoever
// comes last joins. A sequence's own part has the last place of its rows. Nobody waits: every workgroup of a row block of the shared keys arrives at the
// words of all sequences with rows in it, and so does each sequence's own workgroup; the last one at a sequence's word joins its rows.
template <int D>
__device__ __forceinline__ uint32_t means_offset(const SharedParams& p, int kvh, int part, int row, int half) { // bytes; the host keeps them below 2^31
    return (uint32_t)(shared_means<D>(p, kvh, part, row, half) - (char*)p.sh_acc);
}
__device__ __forceinline__ uint32_t head_offset(const SharedParams& p, int kvh, int part, int row) { return (uint32_t)shared_row(p, kvh, part, row) * 16; }
__device__ __forceinline__ uint64_t* own_word(const SharedParams& p, int kvh, int b) { return p.sh_words + (int64_t)kArrivalWords * (b * p.Hkv + kvh); }
// Who arrives at the word of sequence b: `live` parts of every row block that its rows lie in, and its own workgroup.
__device__ __forceinline__ uint32_t own_parties(const SharedParams& p, int b, int live) {
    const int first = b * p.sh_own_rows;
    return (uint32_t)((first + p.sh_own_rows - 1) / kRowBlock - first / kRowBlock + 1) * (uint32_t)live + 1;
}
// G pieces of part `part` of a row from pc on, and m, l and exponents (by wave 0: of the whole row)
template <int D, int G>
__device__ __forceinline__ void store_part(const SharedParams& p, int kvh, int part, int row, int half, int pc, bool heads, float m, float l, const float (&r)[G][8]) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const uint32_t to = means_offset<D>(p, kvh, part, row, half), head = head_offset(p, kvh, part, row);
#pragma unroll
    for (int i = 0; i < G; ++i) {
        float mean[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) mean[e] = r[i][e] * inv;
        uint32_t exponent;
        const u32x4 w = pack_means(mean, exponent);
        __builtin_amdgcn_raw_buffer_store_b128(w, span_of(p.sh_acc), to + (pc + i) * 1024, 0, kDeviceScope);
        if (half == 0) __builtin_amdgcn_raw_buffer_store_b8((uint8_t)exponent, span_of(p.sh_ml), head + 8 + pc + i, 0, kDeviceScope);
    }
    if (heads && half == 0) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(m), __float_as_uint(l)}, span_of(p.sh_ml), head, 0, kDeviceScope);
}
// A row a lane (the same in both halves; rows counted over all sequences) out of all its parts, `parts` of the shared keys and the own one; each wave its
// pieces. p: of the sequences' own keys. Rows that are not `active` are left alone.
template <int D, int NW>
__device__ __forceinline__ void join_rows(const SharedParams& p, int kvh, int parts, int row, bool active) {
    constexpr int NP = D / 16, PPW = NP / NW > 0 ? NP / NW : 1, N = PPW == 1 ? 8 : 4;
    const int half = (threadIdx.x >> 5) & 1, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (wave * PPW >= NP) return;
    row = min(row, p.sh_rows - 1);
    const int pc = wave * PPW, place = p.sh_splits - 1;
    const uint32_t head0 = head_offset(p, kvh, 0, row), from0 = means_offset<D>(p, kvh, 0, row, half);
    const uint32_t head_step = (uint32_t)p.sh_rows * 16, step = (uint32_t)p.sh_blocks * (kRowBlock * D * 2);
    float M = -INFINITY, l = 0.f, o[PPW][8];
#pragma unroll
    for (int i = 0; i < PPW; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) o[i][e] = 0.f;
    SharedRow all{parts + 1, nullptr, nullptr, 0, 0};
    for (int s0 = 0; s0 <= parts; s0 += N) {
        JoinParts<N, PPW> j;
#pragma unroll
        for (int s = 0; s < N; ++s) { // the own part behind the others; past it again
            const uint32_t part = s0 + s < parts ? s0 + s : place;
            j.head[s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(span_of(p.sh_ml), head0 + part * head_step, 0, kDeviceScope));
#pragma unroll
            for (int i = 0; i < PPW; ++i)
                j.x[s][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(span_of(p.sh_acc), from0 + part * step + (pc + i) * 1024, 0, kDeviceScope));
        }
        float top = M;
#pragma unroll
        for (int s = 0; s < N; ++s) top = fmaxf(top, __uint_as_float(j.head[s][0])); // (the own part counts twice at most)
        const float f = __builtin_amdgcn_exp2f(M - top);
        l *= f;
#pragma unroll
        for (int i = 0; i < PPW; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) o[i][e] *= f;
        M = top;
        join_parts(all, s0, pc, j, M, l, o);
    }
    if (active) {
        const int b = row / p.rows, r = row - b * p.rows;
        const float inv = 1.f / l;
        uint16_t* to = (uint16_t*)p.out + row_offset(p, b, kvh, r, row_node(p, r)) + pc * 16 + 4 * half;
#pragma unroll
        for (int i = 0; i < PPW; ++i) {
            *(u32x2*)(to + i * 16) = pack_partial(o[i][0], o[i][1], o[i][2], o[i][3], inv);
            *(u32x2*)(to + i * 16 + 8) = pack_partial(o[i][4], o[i][5], o[i][6], o[i][7], inv);
        }
    }
}

// Statuses, by workgroups of their own behind the last one of the launch over the sequences' own keys, a wave a sequence: the trips of a report in a row, up
// to the block ids, would otherwise be a tail of the workgroups that also compute. `first`: the first such workgroup's number.
__device__ __forceinline__ void report_shared(const SharedParams& p, uint32_t first) {
    const int lane = threadIdx.x & 63, b = (int)(blockIdx.x - first) * ((int)blockDim.x >> 6) + ((int)threadIdx.x >> 6);
    if (!p.status || b >= p.B) return;
    const int32_t parent = p.parent[(int64_t)b * p.T + min(lane, p.T - 1)], S = p.prefix_len[b], len = p.shared_len[0];
    bool bad = false;
    const bool s_ok = prefix_ok(p, S), ok = shared_ok(p, len);
    if (p.paged && s_ok)
        for (int i = lane; i < (S + p.tree_keys + p.block_size - 1) >> p.block_shift; i += kWave)
            bad |= (uint32_t)p.block_table[(int64_t)b * p.max_blocks + i] >= (uint32_t)p.num_blocks;
    if (p.shared_table && ok)
        for (int i = lane; i < (len + (1 << p.sh_block_shift) - 1) >> p.sh_block_shift; i += kWave) bad |= (uint32_t)p.shared_table[i] >= (uint32_t)p.sh_num_blocks;
    int32_t code = VS_STATUS_OK;
    if (!p.tree_mask) {
        if (__any(lane > 0 && lane < p.T && (parent < 0 || parent >= lane))) code = VS_STATUS_BAD_PARENT;
        if (__any(lane == 0 && parent != -1)) code = VS_STATUS_BAD_ROOT;
    }
    if (code == VS_STATUS_OK && !(s_ok && ok)) code = VS_STATUS_BAD_PREFIX;
    if (code == VS_STATUS_OK && __any(bad)) code = VS_STATUS_BAD_BLOCK;
    if (lane == 0) p.status[b] = code;
}

} // namespace vs
