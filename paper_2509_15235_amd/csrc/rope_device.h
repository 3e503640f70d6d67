// Rotary positions on the device: the angle of a pair, and 16-byte pieces of a head on their way through a rotation.
#pragma once

#include "vs_device.h"

namespace vs {

constexpr int kRopeThreads = 256;                 // four waves, each of which takes a row's angles
constexpr int kRopeRows = kRopeThreads / kWave;   // rows of a workgroup, at most
constexpr int64_t kRopeLaunchRows = 1 << 25;       // of a launch: its threads are counted in 32 bits
constexpr int kRopeBatch = 4;                     // pieces a thread has in flight

// cos and sin of a number of turns in [-1/2, 1/2]. fp32 storage keeps 24 bits of the products, bf16 eight: for those the hardware's
// own functions of turns do, whose error (2^-20 or so of a turn's full scale) is far below.
template <bool F32>
__device__ __forceinline__ f32x2 cos_sin_turns(float t) {
    f32x2 r;
    if constexpr (F32) {
        float s, c;
        sincospif(2.f * t, &s, &c);
        r[0] = c;
        r[1] = s;
    } else {
        r[0] = __builtin_amdgcn_cosf(t);
        r[1] = __builtin_amdgcn_sinf(t);
    }
    return r;
}
// In 64 bits up to the fraction of a turn: a far position has many whole turns, and fp32 would have no bits left for the rest.
template <bool F32>
__device__ __forceinline__ f32x2 rope_angle(const RopeParams& p, int32_t position, double inv_freq) {
    const double turns = (double)position * (inv_freq * 0.15915494309189535); // 1 / (2 pi)
    const float t = (float)(turns - __builtin_rint(turns));
    return cos_sin_turns<F32>(p.inverse ? -t : t);
}
// Which axis a pair's positions lie on.
__device__ __forceinline__ int rope_axis(const RopeParams& p, int pair) {
    if (p.num_axes == 1) return 0;
    if (p.cyclic) {
        int a = pair, round = 0; // pair % num_axes, pair / num_axes
        for (; a >= p.num_axes; a -= p.num_axes) ++round;
        const int most = a == 1 ? p.axis_pairs[1] : a == 2 ? p.axis_pairs[2] : p.axis_pairs[3];
        return a > 0 && round < most ? a : 0;
    }
    const int c1 = p.axis_pairs[0], c2 = c1 + p.axis_pairs[1], c3 = c2 + p.axis_pairs[2];
    return (pair >= c1) + (p.num_axes > 2 && pair >= c2) + (p.num_axes > 3 && pair >= c3);
}

// A head is `chunks` items: those that turn (two pieces of 16 bytes half of the rotated channels apart, or one piece of adjacent
// pairs), and behind them the pieces that stay. First piece of item c, in 16-byte units of the head; whether it turns.
template <bool HALVES>
__device__ __forceinline__ bool rope_item(const RopeParams& p, int c, int& piece) {
    const bool turns = c < p.turning;
    piece = HALVES && !turns ? c + p.turning : c;
    return turns;
}
__device__ __forceinline__ f32x2 turn(f32x2 v, f32x2 cs) {
    const f32x2 r = {v[0] * cs[0] - v[1] * cs[1], v[1] * cs[0] + v[0] * cs[1]};
    return r;
}
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
// STREAM: past the L2 caches, see streams_out().
template <bool STREAM>
__device__ __forceinline__ void put(char* to, u32x4 w) {
    if constexpr (STREAM) __builtin_nontemporal_store(w, (u32x4*)to);
    else *(u32x4*)to = w;
}
// Item c's pieces turned; cs: the row's (cos, sin) pairs.
template <bool F32, bool HALVES>
__device__ __forceinline__ void rope_turn(u32x4& a, u32x4& b, const f32x2* cs, int c) {
    constexpr int E = F32 ? 4 : 8; // channels of a piece
    if constexpr (HALVES) {
        const f32x2* w = cs + c * E;
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x2 v = turn(f32x2{__uint_as_float(a[e]), __uint_as_float(b[e])}, w[e]);
                a[e] = __float_as_uint(v[0]);
                b[e] = __float_as_uint(v[1]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x2 lo = turn(f32x2{low_bf16(a[e]), low_bf16(b[e])}, w[2 * e]), hi = turn(f32x2{high_bf16(a[e]), high_bf16(b[e])}, w[2 * e + 1]);
                a[e] = to_bf16x2(lo[0], hi[0]);
                b[e] = to_bf16x2(lo[1], hi[1]);
            }
        }
    } else {
        const f32x2* w = cs + c * (E / 2);
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const f32x2 v = turn(f32x2{__uint_as_float(a[2 * e]), __uint_as_float(a[2 * e + 1])}, w[e]);
                a[2 * e] = __float_as_uint(v[0]);
                a[2 * e + 1] = __float_as_uint(v[1]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x2 v = turn(f32x2{low_bf16(a[e]), high_bf16(a[e])}, w[e]);
                a[e] = to_bf16x2(v[0], v[1]);
            }
        }
    }
}

} // namespace vs
