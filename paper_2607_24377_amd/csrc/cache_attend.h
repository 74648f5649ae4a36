// cache_attend.h -- the arithmetic of attention over the 8-bit paged cache, what its
// rows see, and how its work is divided over workgroups (device code of
// cache_attend.hip, cache_attend_tiles.hip and cache_weigh.hip).
// A row is one query token and head.  A wave holds 32 rows of a sequence that
// share a KV head and walks cached blocks of 32 keys:
//
//   S^T = K Q^T   on the FP8 matrix cores (32x32x64), K's codes as they are.  A
//                 bf16 number has 8 significant bits, two E4M3 numbers' worth:
//                 Q = 2^e (hi + lo), hi the nearest E4M3 number to q 2^-e and lo
//                 that of the rest in steps of 2^-13 2^e at least: exact for
//                 magnitudes from 2^-6 2^e on, else off by up to 2^-14 2^e, less than
//                 2^-21 of the row's largest.  Two FP8 products take the time of one
//                 in bf16, and K needs no conversion;
//   softmax       online, in fp32: m' = max(m, s c - 11), p = exp2(s c - m'), which is
//                 at most 2^11;
//   O^T += V^T P^T on the f16 matrix cores: p is rounded to f16, by 2^-11 of it, or below
//                 2^-25 of the largest by 2^-36 of that (bf16 rounds by 2^-8, which
//                 was a third of the result's whole error; 1560 rows x 32760 keys x 40
//                 heads took 1.11 ms with it and 1.14 so, 64 tokens x 8200 keys 119.5 us
//                 and 121).
//                 l sums the unrounded p.  V's codes times 2^-15 to 2^7 are exact in
//                 f16: O~ is held in units of a power of two of the wave's, which
//                 changes where a block's scale is further away (State).
//
// As S^T has keys as rows, a lane holds the scores of one query.  The keys of a
// block are taken in the order in which accumulator i of lane (query, half h) is
// key 16 h + i, which is the operand order of the second product: no exchange
// between lanes.  The cache stores K and V in these operands' orders.
#pragma once

#include "cache.h"
#include "device_common.h"

namespace mxattn {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

// the running maximum before the first key: below every finite score, so that
// masked scores (-inf) give p = 0 and never inf - inf
constexpr float kNoMax = -3.0e38f;
// The largest p is 2^11: f16 holds 2^-35 of that, and 2^15, which p reaches where m, a
// fp32 number below 2^27, is rounded by 4.
constexpr int kTopLog2 = 11;

// row / group, a row below 2^28 (a product and a shift: the division is 25 instructions).
__device__ __forceinline__ int token_of(const CacheAttendArgs& a, int row) {
    return (int)(((uint64_t)(uint32_t)row * a.per_group) >> 36);
}

__device__ __forceinline__ float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ float other_half(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x),
                                                    false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? (uint32_t)r[0] : (uint32_t)r[1]);
}

// Q of one row as two E4M3 numbers per channel: lane (query, h) holds channels
// 64 j + 32 h .. + 31 of product j.  A row that is not there or sees no key is zero:
// whatever it holds, its masked scores (-inf) are -inf, not NaN, and its result 0.
struct QOperand {
    v8i hi[2], lo[2];
    float c;  // scores times c are in units of log2: scale * 2^e; NaN for a row that is not finite
};

__device__ __forceinline__ QOperand load_q(const uint16_t* row, int h, float scale, bool live) {
    uint4 raw[2][4];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int k = 0; k < 4; k++) {
            raw[j][k] = live ? *reinterpret_cast<const uint4*>(row + 64 * j + 32 * h + 8 * k) : make_uint4(0, 0, 0, 0);
            m = max_halves(m, raw[j][k]);
        }
    m = max(m & 0xFFFFu, m >> 16);
    m = max(m, __builtin_bit_cast(uint32_t, other_half(__builtin_bit_cast(float, m))));
    // the smallest e >= -122 with 1.f 2^(E-127) <= 448 2^e (lo's scale, 2^-4 of hi's, is then
    // a number too)
    const int e = max((int)(m >> 7) - 135 + ((m & 0x7Fu) > 0x60u ? 1 : 0), -122);
    const float fh = e8m0_as_f32((uint32_t)(e + 127)), fl = e8m0_as_f32((uint32_t)(e + 123));
    QOperand q;
    q.c = m < 0x7F80u ? __builtin_ldexpf(scale, e) : __builtin_nanf("");
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const uint32_t u[4] = {raw[j][k].x, raw[j][k].y, raw[j][k].z, raw[j][k].w};
#pragma unroll
            for (int g = 0; g < 2; g++) {
                const i16x2 none = {0, 0};
                i16x2 p = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(none, __builtin_bit_cast(bf16x2, u[2 * g]), fh, false);
                p = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(p, __builtin_bit_cast(bf16x2, u[2 * g + 1]), fh, true);
                const uint32_t hi = __builtin_bit_cast(uint32_t, p);
                const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, fh, false);
                const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, fh, true);
                i16x2 r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(
                    none, __builtin_bit_cast(float, u[2 * g] << 16) - a[0],
                    __builtin_bit_cast(float, u[2 * g] & 0xFFFF0000u) - a[1], fl, false);
                r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(
                    r, __builtin_bit_cast(float, u[2 * g + 1] << 16) - b[0],
                    __builtin_bit_cast(float, u[2 * g + 1] & 0xFFFF0000u) - b[1], fl, true);
                q.hi[j][2 * k + g] = (int)hi;
                q.lo[j][2 * k + g] = (int)__builtin_bit_cast(uint32_t, r);
            }
        }
    return q;
}

__device__ __forceinline__ v8i join(uint4 a, uint4 b) {
    return v8i{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// The 32 x 32 scores of a block; `e` is the block's scale byte.
__device__ __forceinline__ v16f scores(const uint4 (&k)[4], int e, const QOperand& q) {
    v16f s;
#pragma unroll
    for (int i = 0; i < 16; i++) s[i] = 0.f;
    constexpr int kOne = 0x7F7F7F7F, kSixteenth = 0x7B7B7B7B;  // 2^0, 2^-4
    const v8i k0 = join(k[0], k[1]), k1 = join(k[2], k[3]);
    s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k0, q.lo[0], s, 0, 0, 0, e, 0, kSixteenth);
    s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k1, q.lo[1], s, 0, 0, 0, e, 0, kSixteenth);
    s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k0, q.hi[0], s, 0, 0, 0, e, 0, kOne);
    s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k1, q.hi[1], s, 0, 0, 0, e, 0, kOne);
    return s;
}

// Q as it is, for attention that weighs the keys: the FP8 matrix cores keep too few digits
// of the products that they add up (their sums are off by up to 2^-15 of sum |q k|,
// measured, so probabilities by 1e-5; beside the rounding of P and O that does not count).
// K's codes are exact in bf16 and bf16 products are added in fp32 (2^-24), in the time of
// the four FP8 products and 32 conversions a block.  The operands' channels in the order
// of the FP8 ones.
struct QExact {
    uint4 r[8];
    float c;  // as QOperand's
};

__device__ __forceinline__ QExact load_q_exact(const uint16_t* row, int h, float scale, bool live) {
    QExact q;
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int k = 0; k < 4; k++) {
            q.r[4 * j + k] = live ? *reinterpret_cast<const uint4*>(row + 64 * j + 32 * h + 8 * k) : make_uint4(0, 0, 0, 0);
            m = max_halves(m, q.r[4 * j + k]);
        }
    m = max(m & 0xFFFFu, m >> 16);
    m = max(m, __builtin_bit_cast(uint32_t, other_half(__builtin_bit_cast(float, m))));
    q.c = m < 0x7F80u ? scale : __builtin_nanf("");
    return q;
}

// Eight codes of a key as bf16, times the scale.
__device__ __forceinline__ bf16x8 to_bf16(uint32_t a, uint32_t b, float scale) {
    const bf16x2 w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
    const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
    const bf16x2 y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
    const bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
    return bf16x8{w[0], w[1], x[0], x[1], y[0], y[1], z[0], z[1]};
}

// A block of K as the operands of eight products (of 16 channels each).
struct KExact {
    bf16x8 k[8];
};
__device__ __forceinline__ KExact exact_keys(const uint4 (&k)[4], int e) {
    KExact x;
    const float scale = e8m0_as_f32((uint32_t)e);
    const uint32_t none = __builtin_amdgcn_readfirstlane(e) == 255 ? 0x7F7F7F7Fu : 0u;  // a scale that is no number: nor is any key
#pragma unroll
    for (int i = 0; i < 4; i++) {
        x.k[2 * i] = to_bf16(k[i].x | none, k[i].y | none, scale);
        x.k[2 * i + 1] = to_bf16(k[i].z | none, k[i].w | none, scale);
    }
    return x;
}

__device__ __forceinline__ v16f scores(const KExact& k, const uint4 (&q)[8]) {
    v16f s;
#pragma unroll
    for (int i = 0; i < 16; i++) s[i] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.k[i], __builtin_bit_cast(bf16x8, q[i]), s, 0, 0, 0);
    return s;
}
__device__ __forceinline__ v16f scores(const uint4 (&k)[4], int e, const QExact& q) { return scores(exact_keys(k, e), q.r); }

// Q as the kernels of a kind take it.
template <AttendKind kKind>
__device__ __forceinline__ auto load_q_of(const uint16_t* row, int h, float scale, bool live) {
    if constexpr (kKind == kWeigh || kKind == kWeighStats)
        return load_q_exact(row, h, scale, live);
    else
        return load_q(row, h, scale, live);
}

// Eight codes (8 keys of a channel) as f16, times the scale.
__device__ __forceinline__ f16x8 to_f16(uint32_t a, uint32_t b, float scale) {
    const f16x2 w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, scale, false);
    const f16x2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, scale, true);
    const f16x2 y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, scale, false);
    const f16x2 z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, scale, true);
    return f16x8{w[0], w[1], x[0], x[1], y[0], y[1], z[0], z[1]};
}

__device__ __forceinline__ f16x8 probabilities(const v16f& p, int s) {
    f16x8 r;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const f32x2 a = {p[8 * s + 2 * i], p[8 * s + 2 * i + 1]};
        const f16x2 b = __builtin_convertvector(a, f16x2);
        r[2 * i] = b[0];
        r[2 * i + 1] = b[1];
    }
    return r;
}

// A block of K and V in a wave's registers, with its scales; `lost`: no such page.
struct Block {
    uint4 k[4], v[4];
    int ke, ve;
    bool lost;
};

// Loads of what no kernel of the library writes while this one runs, at an address
// that the whole wave shares: scalar loads.
__device__ __forceinline__ int uniform_load(const int32_t* p) {
    return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uint64_t>(p));
}

// The page of block `b` of sequence s (the same for the whole wave).
__device__ __forceinline__ int page_of(const CacheArgs& c, int s, int b) {
    return uniform_load(c.page_table + (int64_t)s * c.max_pages + (b >> c.bpp_log2));
}

// The cache block of a page and head; no such page: `lost`, and some block to read.
struct BlockAt {
    int64_t at;
    bool lost;
};
__device__ __forceinline__ BlockAt block_at(const CacheArgs& c, int page, int head, int b) {
    const bool lost = (unsigned)page >= (unsigned)c.pages;
    if (lost) page = 0;
    return {(((int64_t)page * c.heads + head) << c.bpp_log2) + (b & ((1 << c.bpp_log2) - 1)), lost};
}

// The key of a block that is this lane's row of the K operand.
__device__ __forceinline__ int operand_key(int q) { return 16 * ((q >> 2) & 1) + 4 * (q >> 3) + (q & 3); }

__device__ __forceinline__ void load_block(Block& x, const CacheArgs& c, BlockAt p, int q, int h) {
    const uint8_t* kb = c.kc + p.at * kBlockBytes + 2 * h * 512 + operand_key(q) * 16;
    const uint8_t* vb = c.vc + p.at * kBlockBytes + q * 32 + 16 * h;
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int i = 0; i < 2; i++) x.k[2 * j + i] = *reinterpret_cast<const uint4*>(kb + (4 * j + i) * 512);
#pragma unroll
    for (int i = 0; i < 4; i++) x.v[i] = *reinterpret_cast<const uint4*>(vb + i * 1024);
    x.ke = c.ks[p.at];
    x.ve = c.vs[p.at];
    x.lost = p.lost;
}

// The running state of a wave's rows: lane (query, h) holds its half of l and
// channels 32 n + 8 a + 4 h + b of O~ in O[n][4 a + b], in units of 2^(e - 127).
struct State {
    float m, l;
    v16f O[4];
    int e, most;  // (the same for the whole wave) the units' byte, the largest scale byte of V so far
    __device__ __forceinline__ void clear() {
        m = kNoMax;
        l = 0.f;
        e = most = 0;
#pragma unroll
        for (int n = 0; n < 4; n++)
#pragma unroll
            for (int i = 0; i < 16; i++) O[n][i] = 0.f;
    }
    // What V's codes of scale byte `byte` are multiplied by, 2^-15 to 2^7 (as an E8M0 byte
    // 112 to 134), once the units reach it.
    __device__ __forceinline__ float value_scale(int byte) {
        const int b = __builtin_amdgcn_readfirstlane(byte);
        int f = b - e + 127;
        if ((unsigned)(f - 112) > 22u) f = move(b);
        return e8m0_as_f32((uint32_t)f);
    }
    // Moves the units to scale byte b, but to no less than 2^-40 of the largest so far: O~,
    // below 2^51 there, cannot overflow, and blocks whose scale is below 2^-55 of the
    // largest one's lose digits.  Returns what b's codes are multiplied by: NaN for 255,
    // which units of at most 247 do not reach.
    __device__ __forceinline__ int move(int b) {
        if (b == 255) return 255;
        most = max(most, b);
        const int to = min(max(b, most - 40), 247);
#pragma unroll
        for (int n = 0; n < 4; n++)
#pragma unroll
            for (int i = 0; i < 16; i++) O[n][i] = __builtin_ldexpf(O[n][i], e - to);
        e = to;
        return max(b - to + 127, 64);
    }
    // A new running maximum.
    __device__ __forceinline__ void raise(float to) {
        const float alpha = __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= alpha;
#pragma unroll
        for (int n = 0; n < 4; n++) O[n] *= alpha;
    }
    // p of scores s, whose sum goes to l.
    __device__ __forceinline__ v16f exponentials(const v16f& s, float c, float to) {
        v16f p;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i++) {
            p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -to));
            sum += p[i];
        }
        l += sum;
        return p;
    }
};

// Bytes of v that are NaN codes, as 0x80 in each.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t v) { return ((v & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// The lane's 16 keys of a block that its row sees: its first ones, or those of a mask.
struct Below {
    int n;
    __device__ __forceinline__ bool any() const { return n > 0; }
    __device__ __forceinline__ bool operator()(int i) const { return i < n; }
    // x of a key that the row sees, else -inf.
    __device__ __forceinline__ float masked(float x, int i) const { return i < n ? x : -__builtin_inff(); }
};
struct Bits {
    uint32_t b;
    __device__ __forceinline__ bool any() const { return b != 0; }
    __device__ __forceinline__ bool operator()(int i) const { return (b >> i) & 1u; }
    __device__ __forceinline__ float masked(float x, int i) const {  // (a bit field and a bit select)
        const uint32_t m = (uint32_t)((int32_t)(b << (31 - i)) >> 31);
        return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, x) & m) | (0xFF800000u & ~m));
    }
};

// A block that only some rows see and that holds NaN codes of V: a masked key
// has p = 0, and 0 * NaN would reach every row.  The codes are taken out, and
// the rows that see one get NaN: its count, from a product of ones.
template <class Mask>
__device__ __forceinline__ void spread_nan(State& st, uint4 (&v)[4], const Mask& sees) {
    f16x8 seen[2];
#pragma unroll
    for (int i = 0; i < 16; i++) seen[i >> 3][i & 7] = sees(i) ? (_Float16)1.f : (_Float16)0.f;
#pragma unroll
    for (int n = 0; n < 4; n++) {
        uint32_t* x = reinterpret_cast<uint32_t*>(&v[n]);
        uint32_t one[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t bad = nan_bytes(x[i]);
            one[i] = (bad >> 7) * 0x38u;             // the code of 1
            x[i] &= ~((bad >> 7) * 0xFFu);
        }
        v16f z;
#pragma unroll
        for (int i = 0; i < 16; i++) z[i] = 0.f;
        z = __builtin_amdgcn_mfma_f32_32x32x16_f16(to_f16(one[0], one[1], 1.f), seen[0], z, 0, 0, 0);
        z = __builtin_amdgcn_mfma_f32_32x32x16_f16(to_f16(one[2], one[3], 1.f), seen[1], z, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; i++) st.O[n][i] = z[i] > 0.f ? __builtin_nanf("") : st.O[n][i];
    }
}

__device__ __forceinline__ bool has_nan(const uint4 (&v)[4]) {
    uint32_t m = 0;
#pragma unroll
    for (int n = 0; n < 4; n++)
        m |= ((v[n].x & 0x7F7F7F7Fu) + 0x01010101u) | ((v[n].y & 0x7F7F7F7Fu) + 0x01010101u) |
             ((v[n].z & 0x7F7F7F7Fu) + 0x01010101u) | ((v[n].w & 0x7F7F7F7Fu) + 0x01010101u);
    return (m & 0x80808080u) != 0;
}

// V's codes and scale byte of a block whose keys not every row sees, or of no page; the
// sequence holds the first `held` of its keys.
template <class Mask>
__device__ __forceinline__ void clean_values(State& st, uint4 (&v)[4], int& e, const Mask& sees, int held, bool lost, int h) {
    const bool none = !lost && e == 255;  // a scale that is no number: nor is any value
    if (lost || none) e = 127;            // (a zero code times that scale is NaN too)
    if (lost || held < kBlockTokens || __builtin_amdgcn_readfirstlane(none)) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            uint32_t* w = reinterpret_cast<uint32_t*>(&v[i]);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if (none) w[j] = 0x7F7F7F7Fu;
                // what lies behind the last key may be anything: zero
                const int left = lost ? 0 : held - 16 * h - 4 * j;
                w[j] &= left <= 0 ? 0u : left >= 4 ? ~0u : (1u << (8 * left)) - 1;
            }
        }
    }
    if (__any(has_nan(v))) spread_nan(st, v, sees);
}

// Softmax of a block's scores and their product with V of scale byte `e`; `sees`: the
// keys of the block that the lane's row sees, `any`: some row does not see all.
template <class Mask>
__device__ __forceinline__ void consume(State& st, v16f s, uint4 (&v)[4], int e, float c, const Mask& sees, bool any) {
    if (any) {
#pragma unroll
        for (int i = 0; i < 16; i++) s[i] = sees.masked(s[i], i);
    }
    float mx = max2(max2(s[0], s[1]), s[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) mx = max2(max2(mx, s[i]), s[i + 1]);  // (three-input maxima)
    mx = max2(mx, s[15]);
    mx = __builtin_fmaf(mx, c, -kTopLog2);
    const float m = max2(st.m, max2(mx, other_half(mx)));
    if (__any(m > st.m)) st.raise(m);  // else every alpha is 1
    const float vscale = st.value_scale(e);
    const v16f p = st.exponentials(s, c, m);
    const f16x8 p0 = probabilities(p, 0), p1 = probabilities(p, 1);
#pragma unroll
    for (int n = 0; n < 4; n++) {
        st.O[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(to_f16(v[n].x, v[n].y, vscale), p0, st.O[n], 0, 0, 0);
        st.O[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(to_f16(v[n].z, v[n].w, vscale), p1, st.O[n], 0, 0, 0);
    }
}

// What the lane's row sees (end and, by kind, what follows), and the blocks that the rows
// of the wave or workgroup walk: those of the sinks, then those from the first row's
// window or from the start on, to the end of the last row.
template <AttendKind kKind>
struct Sight {
    int end, keys;         // the row's keys end here; the sequence's
    int min_end;           // the end of the first row
    int low, max_low;      // kWindow: where the row's and the last row's window begin
    int sinks;
    const int32_t* mask;   // kTree: the row's
    int words, past;
    int near, skip, count; // kWindow: blocks of the sinks, blocks left out after them; the blocks to walk

    // Row `row` of the n * group rows of a sequence of `keys_` keys; rows row0 .. last are
    // walked together.
    __device__ __forceinline__ Sight(const CacheAttendArgs& a, int first, int n, int keys_, int row, int row0, int last) {
        keys = keys_;
        past = keys - n;
        const bool causal = kKind != kTree && a.causal;
        end = causal ? past + token_of(a, row) + 1 : keys;
        min_end = causal ? past + token_of(a, row0) + 1 : keys;
        const int max_end = max(0, causal ? past + token_of(a, last) + 1 : keys);
        count = (max_end + kBlockTokens - 1) / kBlockTokens;
        if constexpr (kKind == kWindow) {
            sinks = a.sinks;
            low = end - a.window;
            max_low = max_end - a.window;
            near = (min(sinks, max_end) + kBlockTokens - 1) / kBlockTokens;
            const int from = max(near, max(0, min_end - a.window) / kBlockTokens);
            skip = from - near;
            count = near + max(0, count - from);
        }
        if constexpr (kKind == kTree) {
            words = a.tree_words;
            mask = a.tree + (int64_t)(first + token_of(a, row)) * words;
        }
    }
    // Whether the row sees any key.
    __device__ __forceinline__ bool some() const {
        if constexpr (kKind == kTree) {
            if (past > 0 || keys <= 0) return keys > 0;
            uint32_t any = 0;
            for (int b = 0; b < count; b++) any |= bits(b * kBlockTokens);
            return any != 0;
        }
        return end > 0;
    }
    // The block at place v of the walk.
    __device__ __forceinline__ int block(int v) const {
        if constexpr (kKind == kWindow) return v < near ? v : v + skip;
        return v;
    }
    // Whether some row may not see all of the block at `base` (of a wave: the same for all
    // its lanes).
    __device__ __forceinline__ bool partial(int base) const {
        if constexpr (kKind == kTree) return base + kBlockTokens > past;
        if constexpr (kKind == kWindow)
            return base + kBlockTokens > min_end || (base < max_low && base + kBlockTokens > sinks);
        return base + kBlockTokens > min_end;
    }
    // The keys of the block at `base` that the row sees, as bits.
    __device__ __forceinline__ uint32_t bits(int base) const {
        const uint32_t held = ones(min(end, keys) - base);
        if constexpr (kKind == kWindow) return held & (ones(sinks - base) | ~ones(low - base));
        if constexpr (kKind == kTree) {
            const int off = base - past;  // the first key's place among the drafts
            if (off <= -kBlockTokens) return held;
            const int w = off >> 5, r = off & 31;  // (off < 0: word -1 is what was there before)
            const uint32_t lo = w < 0 ? ~0u : w < words ? (uint32_t)mask[w] : 0u;
            const uint32_t hi = w + 1 < words ? (uint32_t)mask[w + 1] : 0u;
            return held & (uint32_t)((((uint64_t)hi << 32) | lo) >> r);
        }
        return held;
    }
    static __device__ __forceinline__ uint32_t ones(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }
    // The mask of lane half h's keys of the block at `base`.
    __device__ __forceinline__ auto mask_of(int base, bool any, int h) const {
        if constexpr (kKind == kWindow || kKind == kTree)
            return Bits{any ? (bits(base) >> (16 * h)) & 0xFFFFu : 0xFFFFu};
        else
            return Below{end - base - 16 * h};
    }
};

// One block for the wave's rows at `base`; `scores_at`: where the row's scores are kept
// (kWeigh; null: nowhere).  `prefetch` loads the next one: first of all, but after stores
// (loads that stores under a condition follow, the compiler has to wait for with those).
template <AttendKind kKind, class Q, class Prefetch>
__device__ __forceinline__ void attend_block(State& st, Block& x, const Q& q, int base, const Sight<kKind>& sight,
                                             float* scores_at, int h, const Prefetch& prefetch) {
    if constexpr (kKind != kWeigh) prefetch();
    const bool any = sight.partial(base);
    const auto sees = sight.mask_of(base, any, h);
    if (any || x.lost) clean_values(st, x.v, x.ve, sees, sight.keys - base, x.lost, h);
    if (x.lost && sees.any()) st.l = __builtin_nanf("");  // no such page: NaN for the rows that would see it
    const v16f s = scores(x.k, x.ke, q);
    if constexpr (kKind == kWeigh) {
        if (scores_at) {
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<float4*>(scores_at + base + 16 * h + i) = make_float4(s[i], s[i + 1], s[i + 2], s[i + 3]);
        }
        prefetch();
    }
    consume(st, s, x.v, x.ve, q.c, sees, any);
}

// ---------------------------------------------------------------------------
// Division of the work.  An item is a tile of kRows rows of one sequence and KV
// head; the items of the whole call lie in a row, sequence by sequence, head by head,
// tile by tile, and are cut into equal shares, whatever the lengths are: only the
// kernel sees them.  A share is a run of items, of which the first and the last may be
// parts; a part's result (m, l, O~ / l) goes to the share's slot in the workspace and
// the parts are joined by cache_attend_join_kernel in a fixed order.

// Keys of sequence s as far as they can be used: -1 where its length is impossible.
__device__ __forceinline__ int keys_of(const CacheArgs& c, int s) {
    const int len = c.kv_len[s];
    return (unsigned)len > (unsigned)((c.max_pages << c.bpp_log2) * kBlockTokens) ? -1 : len;
}
template <AttendKind kKind>
__device__ __forceinline__ int keys_of(const CacheAttendArgs& a, int s) {
    const int len = keys_of(a.c, s);
    if constexpr (kKind == kWeigh || kKind == kWeighStats) return len > a.most_keys ? -1 : len;
    return len;
}

// Blocks that a tile of `rows` rows of a sequence walks at most (Sight::count).
template <AttendKind kKind>
__device__ __forceinline__ int most_blocks(const CacheAttendArgs& a, int keys, int rows) {
    const int all = (max(keys, 1) + kBlockTokens - 1) / kBlockTokens;
    if constexpr (kKind == kWindow) {
        // the tile's tokens but one move the window on
        const int seen = a.window + (a.causal ? (rows + a.group - 2) / a.group : 0);
        return min(all, (a.sinks + kBlockTokens - 1) / kBlockTokens + (seen + kBlockTokens - 2) / kBlockTokens + 1);
    }
    return all;
}

// Where a row's statistics and scores lie: its token and head.
__device__ __forceinline__ int64_t row_number(const CacheAttendArgs& a, int64_t first, int row, int head) {
    const int token = token_of(a, row);
    return ((first + token) * a.c.heads + head) * a.group + (row - token * a.group);
}
// m and 1 / l, 0 for a row without keys.
__device__ __forceinline__ float2 statistics(float m, float l) {
    return l == 0.f ? make_float2(0.f, 0.f) : make_float2(m, 1.0f / l);
}

// Tiles of a sequence are numbered from here on: no two sequences' overlap, whatever
// the number of sequences' tokens before it.
template <int kRows>
__device__ __forceinline__ int tile_number(const CacheAttendArgs& a, int first, int s) {
    return (int)((int64_t)first * a.group / kRows) + s;
}
template <int kRows>
inline int64_t tile_numbers(const CacheAttendArgs& a) {
    return (int64_t)a.c.tokens * a.group / kRows + a.c.seqs;
}

// The shares that an item lies in; what they leave for the join is in slots
// 2 first + 1, 2 (first + 1), 2 (first + 2), ..., 2 last, or nowhere if there is but
// one share, which finishes it.  Item number: that of the items' workgroups
// (tile_number) times the heads, plus the head.
struct PartInfo {
    int first, last;
};

// The workspace of n shares: O~ / l, m and l of their slots' rows, and the items' PartInfo.
template <int kRows>
struct Parts {
    float* o;     // [2 n, kRows, 128]
    float2* ml;   // [2 n, kRows]
    PartInfo* info;
    __device__ __forceinline__ Parts(uint8_t* ws, int n) {
        o = reinterpret_cast<float*>(ws);
        ml = reinterpret_cast<float2*>(ws + (size_t)2 * n * kRows * 512);
        info = reinterpret_cast<PartInfo*>(ws + (size_t)2 * n * kRows * 520);
    }
};

// Where row `row` of a tile's sequence lies in q or out.
__device__ __forceinline__ int64_t row_offset(const CacheAttendArgs& a, int64_t first, int row, int head, int64_t stride) {
    const int token = token_of(a, row);
    return (first + token) * stride + (int64_t)(head * a.group + row - token * a.group) * kHeadDim;
}

// 1 / l, 0 for a row without keys.
__device__ __forceinline__ float inverse(float l, bool bad) {
    return bad ? __builtin_nanf("") : l == 0.f ? 0.f : 1.0f / l;
}

__device__ __forceinline__ uint2 bf16x4(float a, float b, float c, float d) {
    const f32x2 x = {a, b}, y = {c, d};
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2)),
                      __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2)));
}

// Four channels of a joined row as bf16.
__device__ __forceinline__ uint2 finished(const float4& o, bool bad) {
    const float nan = __builtin_nanf("");
    return bad ? bf16x4(nan, nan, nan, nan) : bf16x4(o.x, o.y, o.z, o.w);
}

// What l is divided by: parts without keys weigh nothing.
__device__ __forceinline__ float reciprocal(float l) { return l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l); }

__device__ __forceinline__ void add_scaled(float4& o, const float4& x, float f) {
    o.x = __builtin_fmaf(x.x, f, o.x);
    o.y = __builtin_fmaf(x.y, f, o.y);
    o.z = __builtin_fmaf(x.z, f, o.z);
    o.w = __builtin_fmaf(x.w, f, o.w);
}

// Channels 32 n + 8 g + 4 h on of a lane's half of a row, divided by l.  (Sums of values
// near the largest fp32 do not pass it so, in parts neither.)
__device__ __forceinline__ float4 four(const State& st, int n, int g, float inv) {
    const v16f& o = st.O[n];
    const int e = st.e - 127;
    return make_float4(__builtin_ldexpf(o[4 * g] * inv, e), __builtin_ldexpf(o[4 * g + 1] * inv, e),
                       __builtin_ldexpf(o[4 * g + 2] * inv, e), __builtin_ldexpf(o[4 * g + 3] * inv, e));
}

// A lane's half of a finished row.
__device__ __forceinline__ void store_row(const State& st, float inv, uint16_t* row, int h) {
#pragma unroll
    for (int n = 0; n < 4; n++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const float4 o = four(st, n, g, inv);
            *reinterpret_cast<uint2*>(row + 32 * n + 8 * g + 4 * h) = bf16x4(o.x, o.y, o.z, o.w);
        }
}

// A lane's half of row `row` of the workspace's slots.
template <int kRows>
__device__ __forceinline__ void store_part(const State& st, float l, const Parts<kRows>& parts, int64_t row, int h) {
    const float inv = inverse(l, false);
    if (h == 0) parts.ml[row] = make_float2(st.m, l);
#pragma unroll
    for (int n = 0; n < 4; n++)
#pragma unroll
        for (int g = 0; g < 4; g++)
            *reinterpret_cast<float4*>(parts.o + row * kHeadDim + 32 * n + 8 * g + 4 * h) = four(st, n, g, inv);
}

// Joins the parts of item blockIdx.x in the order of its keys: a row per workgroup
// and turn, whose eight groups of 32 lanes take every eighth part.
template <int kRows, AttendKind kKind>
__global__ __launch_bounds__(256) void cache_attend_join_kernel(CacheAttendArgs a, int shares) {
    __shared__ float4 s_o[8][32];
    __shared__ float s_m[8], s_l[8];
    const int tid = threadIdx.x, number = blockIdx.x / a.c.heads, head = blockIdx.x - number * a.c.heads;
    const Parts<kRows> parts(a.workspace, shares);
    // finished items and (whatever their entry holds) most numbers of no item end here
    const PartInfo info = parts.info[blockIdx.x];
    if (info.first < 0 || info.last <= info.first || info.last >= shares) return;
    const int s = __builtin_amdgcn_readfirstlane(owner_of(a.c, number, a.group, kRows, 1));
    if (s < 0) return;
    const TokenRange range = token_range(a.c, s);
    const int row0 = (number - tile_number<kRows>(a, range.first, s)) * kRows;
    const int rows = min(kRows, (range.last - range.first) * a.group - row0);
    if (rows <= 0) return;
    const int count = info.last - info.first + 1;
    auto slot = [&info](int p) { return p ? 2 * (info.first + p) : 2 * info.first + 1; };
    const bool bad = keys_of<kKind>(a, s) < 0;
    const int g = tid >> 5, ch = 4 * (tid & 31);
    // the parts from p0 on, every `step`th, four in flight
    auto gather = [&](int r, int p0, int step, float& m, float& l, float4& o) {
        m = kNoMax;
        l = 0.f;
        o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p = p0; p < count; p += 4 * step) {
            float2 ml[4];
            float4 x[4];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const int64_t row = (int64_t)slot(min(p + k * step, count - 1)) * kRows + r;
                ml[k] = parts.ml[row];
                x[k] = *reinterpret_cast<const float4*>(parts.o + row * kHeadDim + ch);
            }
#pragma unroll
            for (int k = 0; k < 4; k++) {
                if (p + k * step >= count) break;
                const float top = max2(m, ml[k].x);
                float f = l * __builtin_amdgcn_exp2f(m - top), g = ml[k].y * __builtin_amdgcn_exp2f(ml[k].x - top);
                m = top;
                l = f + g;
                const float r = reciprocal(l);
                f *= r;
                o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
                add_scaled(o, x[k], g * r);
            }
        }
    };
    auto finish = [&](int r, float m, float l, const float4& o) {
        if constexpr (kKind == kWeigh || kKind == kWeighStats)
            if (ch == 0) a.stats[row_number(a, range.first, row0 + r, head)] = statistics(m, l);
        *reinterpret_cast<uint2*>(a.out + row_offset(a, range.first, row0 + r, head, a.out_stride) + ch) = finished(o, bad);
    };
    float m, l;
    float4 o;
    if (count <= 8) {  // a row for each group (128 items of 8 parts and 32 rows 9.8 us, by all groups 12.1)
        for (int r = 8 * blockIdx.y + g; r < rows; r += 8 * gridDim.y) {
            gather(r, 0, 1, m, l, o);
            finish(r, m, l, o);
        }
        return;
    }
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        gather(r, g, 8, m, l, o);
        s_o[g][tid & 31] = o;
        if (ch == 0) {
            s_m[g] = m;
            s_l[g] = l;
        }
        __syncthreads();
        if (g == 0) {
            m = s_m[0];
            for (int k = 1; k < 8; k++) m = max2(m, s_m[k]);
            l = 0.f;
            for (int k = 0; k < 8; k++) l = __builtin_fmaf(s_l[k], __builtin_amdgcn_exp2f(s_m[k] - m), l);
            const float inv = reciprocal(l);
            o = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = 0; k < 8; k++)
                add_scaled(o, s_o[k][tid & 31], s_l[k] * __builtin_amdgcn_exp2f(s_m[k] - m) * inv);
            finish(r, m, l, o);
        }
        __syncthreads();
    }
}

template <int kRows, AttendKind kKind>
inline hipError_t launch_cache_attend_join(const CacheAttendArgs& a, int shares, hipStream_t stream) {
    const int64_t items = tile_numbers<kRows>(a) * a.c.heads;
    // a row each, or eight where that is a workgroup for every one of 2048 slots
    const int64_t rows = items >= 2048 / (kRows / 8) ? kRows / 8 : kRows;
    cache_attend_join_kernel<kRows, kKind><<<dim3((unsigned)items, (unsigned)rows), 256, 0, stream>>>(a, shares);
    return hipGetLastError();
}

template <int kRows>
inline size_t parts_bytes(const CacheAttendArgs& a, int shares) {
    return (size_t)shares * (2 * kRows * 520) + (size_t)(tile_numbers<kRows>(a) * a.c.heads) * sizeof(PartInfo);
}

}  // namespace mxattn
