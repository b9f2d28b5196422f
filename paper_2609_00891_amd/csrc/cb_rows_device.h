// cb_rows_device.h -- what the kernels on rows share (cb_pages.hip,
// cb_pages_blocks.hip): bf16 pairs, pairs of 16-byte chunks and their turn.
#pragma once
#include "cb_serve_internal.h"

namespace cb {
namespace {

typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

__device__ __forceinline__ float bf_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    f32x2_t v = {lo, hi};
    bf16x2_t p = __builtin_convertvector(v, bf16x2_t);
    return __builtin_bit_cast(uint32_t, p);
}

__device__ __forceinline__ uint32_t fast_div(uint32_t n, const FastDiv &f) {
    const uint32_t t = __umulhi(f.m, n);
    return (t + ((n - t) >> f.sh1)) >> f.sh2;
}

struct ChunkPair { uint4 a, b; };
struct Angles { float c[8], s[8]; };

// The angles of the thread's eight pairs: half split: pairs 8c .. 8c+7; interleaved: 4c .. 4c+3 and
// 4(c + NC2) .. +3.  AT_ONCE: all positions are on their way together, then all angles: two trips to memory, where a branch
// at each position makes up to sixteen.  Four caches of up to 2,048 tokens into 8-bit pages, keys turned: 516 -> 494 us; a
// cache of 40 layers turned back into 16 bits, which shares them among more rows and misses the registers, 774 -> 784.
template <bool AT_ONCE>
__device__ __forceinline__ Angles load_angles(const RopeAxes &ro, int64_t tok, int c, int nc2, float sign) {
    Angles an;
    int32_t pos[8];
    float2 w[8];
    auto pair = [&](int q) __attribute__((always_inline)) {
        return ro.style == 0 ? 8 * c + q : (q < 4 ? 4 * c + q : 4 * (c + nc2) + q - 4);
    };
    auto position = [&](int i) __attribute__((always_inline)) {
        return ro.positions[(int)((ro.axis[i >> 4] >> (2 * (i & 15))) & 3) * ro.axis_stride + tok];
    };
    if constexpr (AT_ONCE) {
#pragma unroll
        for (int q = 0; q < 8; ++q) pos[q] = position(pair(q));
        if (ro.n_pos > 0) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                w[q] = ro.table[(int64_t)((uint32_t)pos[q] < (uint32_t)ro.n_pos ? pos[q] : 0) * (8 * nc2) + pair(q)];
        }
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        float2 x = make_float2(__builtin_nanf(""), __builtin_nanf(""));
        if constexpr (AT_ONCE) {
            if ((uint32_t)pos[q] < (uint32_t)ro.n_pos) x = w[q];
        } else {
            const int i = pair(q);
            const int32_t at = position(i);
            if (at >= 0 && at < ro.n_pos) x = ro.table[(int64_t)at * (8 * nc2) + i];
        }
        an.c[q] = x.x;
        an.s[q] = sign * x.y;
    }
    return an;
}

__device__ __forceinline__ void turn(const ChunkPair &x, const Angles &an, int style, float y0[8], float y1[8]) {
    const uint32_t u0[4] = {x.a.x, x.a.y, x.a.z, x.a.w}, u1[4] = {x.b.x, x.b.y, x.b.z, x.b.w};
    if (style == 0) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float p = q & 1 ? bf_hi(u0[q >> 1]) : bf_lo(u0[q >> 1]);
            const float r = q & 1 ? bf_hi(u1[q >> 1]) : bf_lo(u1[q >> 1]);
            y0[q] = __builtin_fmaf(p, an.c[q], -r * an.s[q]);
            y1[q] = __builtin_fmaf(r, an.c[q], p * an.s[q]);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            y0[2 * q] = __builtin_fmaf(bf_lo(u0[q]), an.c[q], -bf_hi(u0[q]) * an.s[q]);
            y0[2 * q + 1] = __builtin_fmaf(bf_hi(u0[q]), an.c[q], bf_lo(u0[q]) * an.s[q]);
            y1[2 * q] = __builtin_fmaf(bf_lo(u1[q]), an.c[4 + q], -bf_hi(u1[q]) * an.s[4 + q]);
            y1[2 * q + 1] = __builtin_fmaf(bf_hi(u1[q]), an.c[4 + q], bf_lo(u1[q]) * an.s[4 + q]);
        }
    }
}

__device__ __forceinline__ uint4 pack8(const float y[8]) {
    return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

__device__ __forceinline__ void unpack8(const uint4 &v, float y[8]) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        y[2 * q] = bf_lo(u[q]);
        y[2 * q + 1] = bf_hi(u[q]);
    }
}

}  // namespace
}  // namespace cb
