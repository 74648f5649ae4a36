// cache_attend.hip -- attention of new queries over the 8-bit paged cache.
//
// A row is one query token and head; the rows of a sequence that share a KV
// head (its tokens times Hq / Hkv) are cut into tiles of 32, one wave each.  The
// wave walks the cached blocks of 32 keys:
//
//   S^T = K Q^T   on the FP8 matrix cores (32x32x64), K's codes as they are.  A
//                 bf16 number has 8 significant bits, two E4M3 numbers' worth:
//                 Q = 2^e (hi + lo), hi the nearest E4M3 number to q 2^-e and lo
//                 that of the rest, which leaves at most 2^-22 of the row's
//                 largest magnitude.  Two FP8 products take the time of one in
//                 bf16, and K needs no conversion;
//   softmax       online, in fp32: m' = max(m, s c), p = exp2(s c - m');
//   O^T += V^T P^T on the bf16 matrix cores: an E4M3 number times a power of two
//                 is exact in bf16, and p is rounded to bf16 (2^-9 of a value
//                 that is at most 1; l sums the unrounded p).
//
// As S^T has keys as rows, a lane holds the scores of one query.  The keys of a
// block are taken in the order in which accumulator i of lane (query, half h) is
// key 16 h + i, which is the operand order of the second product: no exchange
// between lanes.  The cache stores K and V in these operands' orders.
#include "cache.h"
#include "device_common.h"

namespace mxattn {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kRows = 32;  // query rows of a wave
// the running maximum before the first key: below every finite score, so that
// masked scores (-inf) give p = 0 and never inf - inf
constexpr float kNoMax = -3.0e38f;

__device__ __forceinline__ float max2(float a, float b) { return __builtin_fmaxf(a, b); }

__device__ __forceinline__ float other_half(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x),
                                                    false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? (uint32_t)r[0] : (uint32_t)r[1]);
}

// Q of one row as two E4M3 numbers per channel: lane (query, h) holds channels
// 64 j + 32 h .. + 31 of product j.
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
    // the smallest e >= -127 with 1.f 2^(E-127) <= 448 2^e
    const int e = max((int)(m >> 7) - 135 + ((m & 0x7Fu) > 0x60u ? 1 : 0), -127);
    QOperand q;
    q.c = m < 0x7F80u ? __builtin_ldexpf(scale, e) : __builtin_nanf("");
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const uint32_t u[4] = {raw[j][k].x, raw[j][k].y, raw[j][k].z, raw[j][k].w};
#pragma unroll
            for (int g = 0; g < 2; g++) {
                float x[4];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    x[2 * i] = __builtin_ldexpf(__builtin_bit_cast(float, u[2 * g + i] << 16), -e);
                    x[2 * i + 1] = __builtin_ldexpf(__builtin_bit_cast(float, u[2 * g + i] & 0xFFFF0000u), -e);
                }
                int p = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
                p = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], p, true);
                const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(p, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(p, true);
                int r = __builtin_amdgcn_cvt_pk_fp8_f32((x[0] - a[0]) * 16.f, (x[1] - a[1]) * 16.f, 0, false);
                r = __builtin_amdgcn_cvt_pk_fp8_f32((x[2] - b[0]) * 16.f, (x[3] - b[1]) * 16.f, r, true);
                q.hi[j][2 * k + g] = p;
                q.lo[j][2 * k + g] = r;
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

// Eight codes (8 keys of a channel) as bf16, times the scale.
__device__ __forceinline__ bf16x8 to_bf16(uint32_t a, uint32_t b, float scale) {
    const bf16x2 w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
    const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
    const bf16x2 y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
    const bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
    return bf16x8{w[0], w[1], x[0], x[1], y[0], y[1], z[0], z[1]};
}

__device__ __forceinline__ bf16x8 probabilities(const v16f& p, int s) {
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const f32x2 a = {p[8 * s + 2 * i], p[8 * s + 2 * i + 1]};
        const bf16x2 b = __builtin_convertvector(a, bf16x2);
        r[2 * i] = b[0];
        r[2 * i + 1] = b[1];
    }
    return r;
}

// The running state of a wave's rows: lane (query, h) holds its half of l and
// channels 32 n + 8 a + 4 h + b of O~ in O[n][4 a + b].
struct State {
    float m, l;
    v16f O[4];
    __device__ __forceinline__ void clear() {
        m = kNoMax;
        l = 0.f;
#pragma unroll
        for (int n = 0; n < 4; n++)
#pragma unroll
            for (int i = 0; i < 16; i++) O[n][i] = 0.f;
    }
};

// Bytes of v that are NaN codes, as 0x80 in each.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t v) { return ((v & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// A block that only some rows see and that holds NaN codes of V: a masked key
// has p = 0, and 0 * NaN would reach every row.  The codes are taken out, and
// the rows that see one get NaN: its count, from a product of ones.
__device__ __forceinline__ void spread_nan(State& st, uint4 (&v)[4], int visible, int h) {
    bf16x8 seen[2];
#pragma unroll
    for (int i = 0; i < 16; i++) seen[i >> 3][i & 7] = 16 * h + i < visible ? (__bf16)1.f : (__bf16)0.f;
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
        z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(to_bf16(one[0], one[1], 1.f), seen[0], z, 0, 0, 0);
        z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(to_bf16(one[2], one[3], 1.f), seen[1], z, 0, 0, 0);
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

// Softmax of a block's scores and their product with V; `visible`: keys of the
// block that the lane's row sees (its first ones), `any`: some row does not see all.
__device__ __forceinline__ void consume(State& st, v16f s, uint4 (&v)[4], float vscale, float c, int visible, bool any,
                                        int h) {
    if (any) {
#pragma unroll
        for (int i = 0; i < 16; i++) s[i] = 16 * h + i < visible ? s[i] : -__builtin_inff();
    }
    float mx = max2(s[0], s[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) mx = max2(mx, max2(s[i], s[i + 1]));
    mx *= c;
    const float m = max2(st.m, max2(mx, other_half(mx)));
    const float alpha = __builtin_amdgcn_exp2f(st.m - m);
    st.m = m;
    st.l *= alpha;
#pragma unroll
    for (int n = 0; n < 4; n++) st.O[n] *= alpha;
    v16f p;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -m));
        st.l += p[i];
    }
    const bf16x8 p0 = probabilities(p, 0), p1 = probabilities(p, 1);
#pragma unroll
    for (int n = 0; n < 4; n++) {
        st.O[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(to_bf16(v[n].x, v[n].y, vscale), p0, st.O[n], 0, 0, 0);
        st.O[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(to_bf16(v[n].z, v[n].w, vscale), p1, st.O[n], 0, 0, 0);
    }
}

__global__ __launch_bounds__(64) void cache_attend_kernel(CacheAttendArgs a) {
    const CacheArgs& c = a.c;
    const int lane = threadIdx.x, q = lane & 31, h = lane >> 5;
    const int w = blockIdx.x, head = blockIdx.y;
    int s = -1;
    for (int i = lane; i < c.seqs; i += 64) {
        const TokenRange r = token_range(c, i);
        const int64_t base = (int64_t)r.first * a.group / kRows + i, next = (int64_t)r.last * a.group / kRows + i + 1;
        if (base <= w && w < next) s = i;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s = max(s, __shfl_xor(s, d));
    if (s < 0) return;
    s = __builtin_amdgcn_readfirstlane(s);
    const TokenRange r = token_range(c, s);
    const int n = r.last - r.first;
    const int tile = w - (int)((int64_t)r.first * a.group / kRows + s);
    const int row0 = tile * kRows, rows = n * a.group;
    if (row0 >= rows) return;
    const int row = min(row0 + q, rows - 1);
    const bool live = row0 + q < rows;
    const int token = row / a.group, qhead = head * a.group + row % a.group;
    const int reach = (c.max_pages << c.bpp_log2) * kBlockTokens;
    const int len = c.kv_len[s];
    const bool bad = (unsigned)len > (unsigned)reach;  // no such cache: NaN
    const int keys = bad ? 0 : len;
    // keys that the row sees, and those that the first and the last row see
    const int end = a.causal ? keys - n + token + 1 : keys;
    const int last_row = min(row0 + kRows, rows) - 1;
    const int min_end = a.causal ? keys - n + row0 / a.group + 1 : keys;
    const int max_end = a.causal ? keys - n + last_row / a.group + 1 : keys;

    const int64_t qtoken = r.first + token;
    const QOperand qo = load_q(a.q + qtoken * a.q_stride + (int64_t)qhead * kHeadDim, h, a.scale, live);
    State st;
    st.clear();
    bool nan = bad;
    const int key = 16 * ((q >> 2) & 1) + 4 * (q >> 3) + (q & 3);  // of this lane's row of K
    for (int b = 0; b * kBlockTokens < max_end; b++) {
        int page = c.page_table[(int64_t)s * c.max_pages + (b >> c.bpp_log2)];
        const bool lost = (unsigned)page >= (unsigned)c.pages;
        if (lost) page = 0;
        const int64_t at = (((int64_t)page * c.heads + head) << c.bpp_log2) + (b & ((1 << c.bpp_log2) - 1));
        const uint8_t* kb = c.kc + at * kBlockBytes;
        const uint8_t* vb = c.vc + at * kBlockBytes;
        uint4 k[4], v[4];
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int i = 0; i < 2; i++)
                k[2 * j + i] = *reinterpret_cast<const uint4*>(kb + (4 * j + 2 * h + i) * 512 + key * 16);
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = *reinterpret_cast<const uint4*>(vb + (32 * i + q) * 32 + 16 * h);
        const int visible = end - b * kBlockTokens;
        const bool any = (b + 1) * kBlockTokens > min_end;
        if (any) {
            // what lies behind the last key may be anything: zero
            const int held = keys - b * kBlockTokens - 16 * h;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                uint32_t* x = reinterpret_cast<uint32_t*>(&v[i]);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const int left = held - 4 * j;
                    x[j] &= left <= 0 ? 0u : left >= 4 ? ~0u : (1u << (8 * left)) - 1;
                }
            }
        }
        if (lost) {
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = make_uint4(0, 0, 0, 0);
        }
        if (any && __any(has_nan(v))) spread_nan(st, v, visible, h);
        v16f sc = scores(k, (int)c.ks[at], qo);
        if (lost) {
#pragma unroll
            for (int i = 0; i < 16; i++) sc[i] = __builtin_nanf("");
        }
        consume(st, sc, v, e8m0_as_f32(c.vs[at]), qo.c, visible, any, h);
    }
    const float l = st.l + other_half(st.l);
    const float inv = nan ? __builtin_nanf("") : l == 0.f ? 0.f : 1.0f / l;
    if (!live) return;
    uint16_t* dst = a.out + qtoken * a.out_stride + (int64_t)qhead * kHeadDim + 4 * h;
#pragma unroll
    for (int t = 0; t < 4; t++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const f32x2 lo = {st.O[t][4 * g] * inv, st.O[t][4 * g + 1] * inv};
            const f32x2 hi = {st.O[t][4 * g + 2] * inv, st.O[t][4 * g + 3] * inv};
            *reinterpret_cast<uint2*>(dst + 32 * t + 8 * g) =
                make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
                           __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2)));
        }
}

}  // namespace

hipError_t launch_cache_attend(const CacheAttendArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)a.c.tokens * a.group / kRows + a.c.seqs), (unsigned)a.c.heads);
    cache_attend_kernel<<<grid, 64, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace mxattn
