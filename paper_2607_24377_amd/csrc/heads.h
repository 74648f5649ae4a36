// heads.h -- the norm of a head and its rotation by position, in registers.
//
// A row of 128 channels lies in 16 consecutive lanes, 8 channels each.  y = x /
// sqrt(mean(x^2) + eps) * w in fp32; then each pair (a, b) of the first `rot`
// channels becomes (a cos - b sin, b cos + a sin) with the angles of the row's
// position.  Pairs are neighbours (2i, 2i + 1) or lie rot / 2 apart (i, i + rot / 2);
// either way a lane holds both of its four pairs (rot is a multiple of 16).
#pragma once

#include "cache.h"
#include "device_common.h"

namespace mxattn {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8), aligned(16)));

// Sum over the 16 lanes of a row, in every lane of it (DPP moves: no LDS traffic).
__device__ __forceinline__ float row_sum16(float x) {
    auto add = [](float a, int b) { return a + __builtin_bit_cast(float, b); };
    x = add(x, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, false));   // lane ^ 1
    x = add(x, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, false));   // lane ^ 2
    x = add(x, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x141, 0xF, 0xF, false));  // 7 - lane of 8
    x = add(x, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x140, 0xF, 0xF, false));  // 15 - lane
    return x;
}

__device__ __forceinline__ f32x8 unpack_bf16(u32x4 v) {
    f32x8 x;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        x[2 * i] = __builtin_bit_cast(float, v[i] << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xFFFF0000u);
    }
    return x;
}

typedef float f32x2v __attribute__((ext_vector_type(2)));
// Round to nearest even (the hardware's packed conversion).
__device__ __forceinline__ u32x4 pack_bf16(f32x8 x) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const f32x2v p = {x[2 * i], x[2 * i + 1]};
        v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
    }
    return v;
}

// The channels of a lane, two groups of four from first and second on: eight in a
// row, or, of rotated halves, four of each (and of the halves of what does not
// rotate, so that the lanes' groups are neighbours there too).
template <bool kHalves>
struct Channels {
    int first, second;
    __device__ __forceinline__ Channels(int rot, int lane) {
        const bool rotates = 8 * lane < rot;
        const int base = rotates ? 0 : rot, width = rotates ? rot : kHeadDim - rot;
        first = kHalves ? base + 4 * (lane - (base >> 3)) : 8 * lane;
        second = kHalves ? first + (width >> 1) : first + 4;
    }
    __device__ __forceinline__ f32x8 weights(const float* w) const {
        const f32x4 x = *reinterpret_cast<const f32x4*>(w + first), y = *reinterpret_cast<const f32x4*>(w + second);
        return f32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    }
    // bf16 channels of the row at p
    __device__ __forceinline__ u32x4 load(const uint16_t* p) const {
        if constexpr (!kHalves) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + first));
        const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p + first));
        const u32x2 y = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p + second));
        return u32x4{x[0], x[1], y[0], y[1]};
    }
};

// The angles of a lane's four pairs.
template <bool kHalves>
struct Rotation {
    f32x4 c, s;
    bool on;  // whether the lane's channels rotate (the others pass as they are, infinities too)

    // Lane `lane` of the row (0..15); rows of angles at cos, sin (null: NaN, of a
    // position that the table does not have).
    __device__ __forceinline__ Rotation(const float* cos, const float* sin, int rot, int lane) {
        on = 8 * lane < rot;
        if (!on) return;
        const float nan = __builtin_nanf("");
        c = s = f32x4{nan, nan, nan, nan};
        if (!cos) return;
        c = *reinterpret_cast<const f32x4*>(cos + 4 * lane);
        s = *reinterpret_cast<const f32x4*>(sin + 4 * lane);
    }
    // Position pos of the table.
    static __device__ __forceinline__ Rotation at(const HeadTransform& t, int64_t pos, int lane) {
        const bool in = (uint64_t)pos < (uint64_t)t.table_rows;
        const int64_t row = pos * (t.rot >> 1);
        return Rotation(in ? t.cos + row : nullptr, t.sin + row, t.rot, lane);
    }

    // The lane's eight channels turned.
    __device__ __forceinline__ f32x8 turned(const f32x8& x) const {
        f32x8 y = x;
        if (on) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int a = kHalves ? i : 2 * i, b = kHalves ? 4 + i : 2 * i + 1;
                y[a] = __builtin_fmaf(x[a], c[i], -(x[b] * s[i]));
                y[b] = __builtin_fmaf(x[b], c[i], x[a] * s[i]);
            }
        }
        return y;
    }
};

// Sum of squares of the row.
__device__ __forceinline__ float sum_of_squares(const f32x8& x) {
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) q = __builtin_fmaf(x[i], x[i], q);
    return row_sum16(q);
}

// x / sqrt(mean(x^2) + eps) * w, from the hardware's reciprocal square root (1 ulp; the
// exact square root and division are 40 instructions).  Squares pass fp32 for
// magnitudes above 2^60 and lose digits below 2^-63: a row whose sum is infinite is
// normed as x 2^-80 and eps 2^-160, one whose mean and eps are below 2^-96 (so |x| below
// 2^-44) as x 2^80 and eps 2^160, which leaves |x| between 2^-53 and 2^48 or without
// effect.
__device__ __forceinline__ f32x8 normed(f32x8 x, const f32x8& w, float eps) {
    float q = sum_of_squares(x), m = __builtin_fmaf(q, 1.0f / kHeadDim, eps);
    const float f = m < 0x1p-96f ? 0x1p80f : q < __builtin_inff() ? 1.f : 0x1p-80f;
    if (__any(f != 1.f)) {
        x *= f;
        m = __builtin_fmaf(sum_of_squares(x), 1.0f / kHeadDim, eps * f * f);
    }
    const float r = __builtin_amdgcn_rsqf(m);
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] *= r * w[i];
    return x;
}

}  // namespace mxattn
