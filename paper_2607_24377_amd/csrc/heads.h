// heads.h -- the norm of a head and its rotation by position, in registers.
//
// A row of 128 channels lies in 16 consecutive lanes, 8 channels each (16
// bytes of bf16).  y = x / sqrt(mean(x^2) + eps) * w in fp32; then each pair
// (a, b) of the first `rot` channels becomes (a cos - b sin, b cos + a sin) with
// the angles of the row's position.  Pairs are neighbours (2i, 2i + 1) or lie
// rot / 2 apart (i, i + rot / 2); rot is a multiple of 16, so that a lane's eight
// channels have their eight partners in one lane.
#pragma once

#include "cache.h"
#include "device_common.h"

namespace mxattn {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
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

// What a lane needs of a head's rotation: its partner lane and its angles.
template <bool kHalves>
struct Rotation {
    f32x8 c, s;   // kHalves: of the lane's 8 channels, s with the sign; else of its 4 pairs in [0..3]
    int partner;  // lane of the wave (kHalves)
    bool on;      // whether the lane's channels rotate (the others pass as they are, infinities too)

    // `lane` of the row (0..15); an angle row outside the table makes NaN.
    __device__ __forceinline__ Rotation(const HeadTransform& t, int64_t pos, int lane) {
        const int self = (int)threadIdx.x & 63;
        partner = self;
        on = 8 * lane < t.rot;
        if (!on) return;
        const int half = t.rot >> 4;  // lanes of half the rotated channels
        const bool second = kHalves && lane >= half;
        if (kHalves) partner = second ? self - half : self + half;
        if ((uint64_t)pos >= (uint64_t)t.table_rows) {
            const float nan = __builtin_nanf("");
            for (int i = 0; i < 8; i++) c[i] = s[i] = nan;
            return;
        }
        const int64_t row = pos * (t.rot >> 1);
        if (kHalves) {
            const int64_t at = row + 8 * (second ? lane - half : lane);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                c[i] = t.cos[at + i];
                s[i] = second ? t.sin[at + i] : -t.sin[at + i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                c[i] = t.cos[row + 4 * lane + i];
                s[i] = t.sin[row + 4 * lane + i];
            }
        }
    }

    // The lane's eight channels turned.
    __device__ __forceinline__ f32x8 turned(f32x8 x) const {
        f32x8 y;
        if constexpr (kHalves) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float p = __shfl(x[i], partner);
                y[i] = on ? __builtin_fmaf(x[i], c[i], p * s[i]) : x[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                y[2 * i] = on ? __builtin_fmaf(x[2 * i], c[i], -(x[2 * i + 1] * s[i])) : x[2 * i];
                y[2 * i + 1] = on ? __builtin_fmaf(x[2 * i + 1], c[i], x[2 * i] * s[i]) : x[2 * i + 1];
            }
        }
        return y;
    }
};

__device__ __forceinline__ f32x8 normed(f32x8 x, const f32x8& w, float eps) {
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) q = __builtin_fmaf(x[i], x[i], q);
    const float r = 1.0f / __builtin_sqrtf(row_sum16(q) * (1.0f / kHeadDim) + eps);
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] *= r * w[i];
    return x;
}

}  // namespace mxattn
