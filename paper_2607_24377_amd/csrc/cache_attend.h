// cache_attend.h -- the arithmetic of attention over the 8-bit paged cache, and
// how its work is divided over workgroups (device code of cache_attend.hip).
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

// A block that only some rows see and that holds NaN codes of V: a masked key
// has p = 0, and 0 * NaN would reach every row.  The codes are taken out, and
// the rows that see one get NaN: its count, from a product of ones.
__device__ __forceinline__ void spread_nan(State& st, uint4 (&v)[4], int visible, int h) {
    f16x8 seen[2];
#pragma unroll
    for (int i = 0; i < 16; i++) seen[i >> 3][i & 7] = 16 * h + i < visible ? (_Float16)1.f : (_Float16)0.f;
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
    for (int n = 0; n < 4; n++) m |= nan_bytes(v[n].x) | nan_bytes(v[n].y) | nan_bytes(v[n].z) | nan_bytes(v[n].w);
    return m != 0;
}

// V's codes and scale byte of a block whose keys not every row sees, or of no page:
// `base` is its first key's place where the lane's row sees `visible` keys and the
// sequence holds `held`.
__device__ __forceinline__ void clean_values(State& st, uint4 (&v)[4], int& e, int base, int visible, int held, bool lost,
                                             int h) {
    const bool none = !lost && e == 255;  // a scale that is no number: nor is any value
    if (lost || none) e = 127;            // (a zero code times that scale is NaN too)
#pragma unroll
    for (int i = 0; i < 4; i++) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&v[i]);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            if (none) w[j] = 0x7F7F7F7Fu;
            // what lies behind the last key may be anything: zero
            const int left = lost ? 0 : held - base - 16 * h - 4 * j;
            w[j] &= left <= 0 ? 0u : left >= 4 ? ~0u : (1u << (8 * left)) - 1;
        }
    }
    if (__any(has_nan(v))) spread_nan(st, v, visible - base, h);
}

// Softmax of a block's scores and their product with V of scale byte `e`; `visible`:
// keys of the block that the lane's row sees (its first ones), `any`: some row does
// not see all.
__device__ __forceinline__ void consume(State& st, v16f s, uint4 (&v)[4], int e, float c, int visible, bool any, int h) {
    if (any) {
#pragma unroll
        for (int i = 0; i < 16; i++) s[i] = 16 * h + i < visible ? s[i] : -__builtin_inff();
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

// One block for the wave's rows: `end` keys are the lane's row's, `keys` the
// sequence's, `base` the block's first; `any`: some row does not see all of it.
__device__ __forceinline__ void attend_block(State& st, Block& x, const QOperand& q, int base, int end, int keys, bool any,
                                             int h) {
    if (any || x.lost) clean_values(st, x.v, x.ve, 0, end - base, keys - base, x.lost, h);
    if (x.lost && end > base) st.l = __builtin_nanf("");  // no such page: NaN for the rows that would see it
    const v16f s = scores(x.k, x.ke, q);
    consume(st, s, x.v, x.ve, q.c, end - base, any, h);
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
template <int kRows>
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
    const bool bad = keys_of(a.c, s) < 0;
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
    auto finish = [&](int r, const float4& o) {
        *reinterpret_cast<uint2*>(a.out + row_offset(a, range.first, row0 + r, head, a.out_stride) + ch) = finished(o, bad);
    };
    float m, l;
    float4 o;
    if (count <= 8) {  // a row for each group (128 items of 8 parts and 32 rows 9.8 us, by all groups 12.1)
        for (int r = 8 * blockIdx.y + g; r < rows; r += 8 * gridDim.y) {
            gather(r, 0, 1, m, l, o);
            finish(r, o);
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
            finish(r, o);
        }
        __syncthreads();
    }
}

template <int kRows>
inline hipError_t launch_cache_attend_join(const CacheAttendArgs& a, int shares, hipStream_t stream) {
    const int64_t items = tile_numbers<kRows>(a) * a.c.heads;
    // a row each, or eight where that is a workgroup for every one of 2048 slots
    const int64_t rows = items >= 2048 / (kRows / 8) ? kRows / 8 : kRows;
    cache_attend_join_kernel<kRows><<<dim3((unsigned)items, (unsigned)rows), 256, 0, stream>>>(a, shares);
    return hipGetLastError();
}

template <int kRows>
inline size_t parts_bytes(const CacheAttendArgs& a, int shares) {
    return (size_t)shares * (2 * kRows * 520) + (size_t)(tile_numbers<kRows>(a) * a.c.heads) * sizeof(PartInfo);
}

}  // namespace mxattn
