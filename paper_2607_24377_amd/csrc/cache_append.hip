// cache_append.hip -- new keys and values into the 8-bit paged cache.
//
// A block is 32 consecutive tokens of one sequence and head: 4096 codes (E4M3)
// and one E8M0 scale 2^e, the smallest with max |x| <= 448 2^e over the block.
// A block that gets tokens beside older ones keeps its scale or takes a larger
// one; then the older codes are rounded again, code * 2^(e_old - e), which is
// exact unless it falls below 2^-6 (a power of two leaves the 3 fraction bits
// alone).  Keys are normed and rotated in fp32 and rounded once, to the code.
//
// Block layouts are the operand orders of cache_attend.hip, so that it copies
// them in one piece: K [8 chunks of 16 channels][32 tokens][16], V
// [128 channels][32 tokens].
//
// Bound by HBM: 2 bytes read and 1 written per element.  One wave per block and
// head, the four of a workgroup on four heads of the same tokens, whose angles they
// share in LDS.  Sequence s owns workgroups q_start[s] / 32 +
// 2 s onwards, which are as many as the blocks that its tokens can touch, so that
// the grid follows from the number of tokens and sequences alone.
//
// A lane holds 8 channels of 8 tokens: lane 16 r + c channels of tokens
// 16 i + 4 r + j (i < 2, j < 4).  Four channels of a token are a word of K's block,
// four consecutive tokens of a channel one of V's, which the conversions pack
// directly; the words change places through LDS.  V is done before K is turned, so
// that four waves a SIMD have registers, and the codes are stored past the caches:
// K and V of 32760 tokens x 40 heads, 1.02 GB, 186 us, 5.5 TB/s (two waves and
// ordinary stores 219; three of those 210; a workgroup per block and head 279).
//
// Few tokens: what counts is the chain of loads.  All 16 rows of a lane are in flight
// at once, those that are not new in the place of one that is: 16 prompts of 1000
// tokens, 8 heads, 15.4 us; 64 single tokens 6.9 (with the loads of a block's missing
// tokens branched around, which the compiler makes one after another, 21.2 and 9.0).
#include "heads.h"

namespace mxattn {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

// E8M0 byte of the smallest scale that holds magnitudes up to M (bits of a
// finite fp32 >= 0): M = 1.f 2^(E-127) <= 1.75 2^(8 + e).
__device__ __forceinline__ int scale_byte(uint32_t mbits) {
    const int e = (int)(mbits >> 23) - 8 + ((mbits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return max(e, 0);
}

typedef short i16x2 __attribute__((ext_vector_type(2)));

// Two E4M3 codes of x and y over the scale (an fp32 whose exponent field is the
// E8M0 byte), nearest even, into the low or the high half of `old`.
template <bool kHigh>
__device__ __forceinline__ uint32_t encode2(uint32_t old, float x, float y, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(__builtin_bit_cast(i16x2, old), x, y,
                                                                                 scale, kHigh));
}
template <bool kHigh>
__device__ __forceinline__ uint32_t encode2(uint32_t old, uint32_t bf16_pair, float scale) {
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(__builtin_bit_cast(i16x2, old),
                                                                        __builtin_bit_cast(bf16x2, bf16_pair), scale, kHigh));
}

// Four codes times 2^shift (shift <= 0).
__device__ __forceinline__ uint32_t rescale4(uint32_t c, int shift) {
    const f32x2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
    const f32x2v b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    const int p = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(a[0], shift), __builtin_ldexpf(a[1], shift), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(b[0], shift), __builtin_ldexpf(b[1], shift), p, true);
}

// Largest magnitude of x, at least m; NaN does not count.
__device__ __forceinline__ float magnitude(float m, const f32x8& x) {
#pragma unroll
    for (int i = 0; i < 8; i += 2)
        m = __builtin_fmaxf(__builtin_fmaxf(m, __builtin_fabsf(x[i])), __builtin_fabsf(x[i + 1]));
    return m;
}

// What is not finite becomes NaN (the conversions give inf the largest code); the
// largest magnitude of the rest.
__device__ __forceinline__ uint32_t without_inf(uint32_t m, f32x8& x) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float f = x[i];  // (a bit cast of a vector's element itself reads its first one)
        const uint32_t u = __builtin_bit_cast(uint32_t, f) & 0x7FFFFFFFu;
        m = max(m, u < 0x7F800000u ? u : 0u);
        x[i] = u < 0x7F800000u ? f : __builtin_nanf("");
    }
    return m;
}
__device__ __forceinline__ uint32_t without_inf(uint32_t m, u32x4& x) {  // bf16 pairs
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t lo = x[i] & 0x7FFFu, hi = (x[i] >> 16) & 0x7FFFu;
        m = max(m, lo < 0x7F80u ? lo : 0u);
        m = max(m, hi < 0x7F80u ? hi : 0u);
        x[i] = (lo < 0x7F80u ? x[i] & 0xFFFFu : 0x7FC0u) | (hi < 0x7F80u ? x[i] & 0xFFFF0000u : 0x7FC00000u);
    }
    return m;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
    auto dpp = [](uint32_t a, int ctrl_value) { return max(a, (uint32_t)ctrl_value); };
    m = dpp(m, __builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, false));   // lane ^ 1
    m = dpp(m, __builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, false));   // lane ^ 2
    m = dpp(m, __builtin_amdgcn_mov_dpp((int)m, 0x141, 0xF, 0xF, false));  // 7 - lane of 8
    m = dpp(m, __builtin_amdgcn_mov_dpp((int)m, 0x140, 0xF, 0xF, false));  // 15 - lane of 16
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    return max(m, (uint32_t)__shfl_xor((int)m, 32));
}

// A block in LDS.  K: 512 bytes a chunk of 16 channels and 16 bytes more, V: 32 bytes
// a channel and 16 bytes more every 8 channels, so that the words that 64 lanes write
// at once lie in 64 banks.
constexpr int kTileWords = 128 * 8 + 16 * 4;
__device__ __forceinline__ int k_word(int channel, int token) {
    return (channel >> 4) * 132 + token * 4 + ((channel >> 2) & 3);
}
__device__ __forceinline__ int v_word(int channel) { return channel * 8 + (channel >> 3) * 4; }

// Mask of the first n bytes of a word.
__device__ __forceinline__ uint32_t bytes_below(int n) {
    return n <= 0 ? 0u : n >= 4 ? ~0u : (1u << (8 * n)) - 1;
}

// A wave's block: which of its tokens are new, and where they lie.
struct Place {
    int64_t at;      // the cache block
    int64_t row;     // of slot 0, if it were new, among the call's tokens
    int lead, stop;  // slots lead .. stop - 1 are new, those before it older
    int head;
};

// kWhole: all 32 tokens are new.
template <bool kHalves, bool kWhole>
__device__ __forceinline__ void append_block(const AppendArgs& a, const Place& p, uint32_t* tile, const float* angles) {
    const CacheArgs& c = a.c;
    const int lane = threadIdx.x & 63, ch = lane & 15, r4 = lane >> 4;
    uint8_t* kb = c.kc + p.at * kBlockBytes;
    uint8_t* vb = c.vc + p.at * kBlockBytes;
    // token t of a lane's eight, whether it is new, and whether any lane's is
    auto slot_of = [r4](int t) { return 16 * (t >> 2) + 4 * r4 + (t & 3); };
    auto live = [&](int t) { return kWhole || (slot_of(t) >= p.lead && slot_of(t) < p.stop); };
    auto some = [&](int t) { return kWhole || __any(live(t)); };
    const Channels<kHalves> channels(a.t.rot, ch);
    u32x4 raw_k[8], raw_v[8];  // (of what is not new: the first new token's)
#pragma unroll
    for (int t = 0; t < 8; t++) {
        const int64_t tok = p.row + (live(t) ? slot_of(t) : p.lead);
        raw_v[t] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(a.v + tok * a.v_stride + p.head * kHeadDim + 8 * ch));
    }
#pragma unroll
    for (int t = 0; t < 8; t++) {
        const int64_t tok = p.row + (live(t) ? slot_of(t) : p.lead);
        raw_k[t] = channels.load(a.k + tok * a.k_stride + p.head * kHeadDim);
    }
    // what is there already, if some of it stays
    int was_k = 0, was_v = 0;
    if (!kWhole && p.lead) {
        was_k = c.ks[p.at];
        was_v = c.vs[p.at];
    }

    // V: word i of a channel is tokens 4 i .. 4 i + 3
    uint32_t mv = 0;
#pragma unroll
    for (int t = 0; t < 8; t++)
        if (live(t)) mv = max_halves(mv, make_uint4(raw_v[t][0], raw_v[t][1], raw_v[t][2], raw_v[t][3]));
    mv = wave_max(max(mv & 0xFFFFu, mv >> 16));
    if (__builtin_amdgcn_readfirstlane(mv >= 0x7F80u)) {
        mv = 0;
#pragma unroll
        for (int t = 0; t < 8; t++)
            if (live(t)) mv = without_inf(mv, raw_v[t]);
        mv = wave_max(mv);
    }
    const int bv = max(scale_byte(mv << 16), was_v);
    const float fv = e8m0_as_f32((uint32_t)bv);
#pragma unroll
    for (int i = 0; i < 2; i++) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            // channel e of four tokens: halves of their words
            const uint32_t pick = e & 1 ? 0x07060302u : 0x05040100u;
            const uint32_t x = __builtin_amdgcn_perm(raw_v[4 * i + 1][e >> 1], raw_v[4 * i][e >> 1], pick);
            const uint32_t y = __builtin_amdgcn_perm(raw_v[4 * i + 3][e >> 1], raw_v[4 * i + 2][e >> 1], pick);
            tile[v_word(8 * ch + e) + 4 * i + r4] = encode2<true>(encode2<false>(0, x, fv), y, fv);
        }
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int unit = 64 * i + lane;  // 16 tokens of a channel
        u32x4 q = *reinterpret_cast<const u32x4*>(tile + v_word(unit >> 1) + 4 * (unit & 1));
        if (!kWhole) {
            const int t0 = 16 * (unit & 1);
            const u32x4 had = *reinterpret_cast<const u32x4*>(vb + 16 * unit);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const uint32_t before = bytes_below(p.lead - t0 - 4 * j), fresh = bytes_below(p.stop - t0 - 4 * j) & ~before;
                uint32_t old = had[j];
                if (bv > was_v && before) old = (rescale4(old, was_v - bv) & before) | (old & ~before);
                q[j] = (q[j] & fresh) | (old & ~fresh);
            }
        }
        __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(vb + 16 * unit));
    }

    // K
    f32x8 w;
    if (a.w) w = channels.weights(a.w);
    __syncthreads();  // the angles are in LDS (and V's tile is read)
    f32x8 k[8];
    float largest = 0.f;
#pragma unroll
    for (int t = 0; t < 8; t++) {
        k[t] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (!some(t)) continue;
        k[t] = unpack_bf16(raw_k[t]);
        if (a.w) k[t] = normed(k[t], w, a.t.eps);
        const float* row = angles + slot_of(t) * (kHeadDim / 2);
        k[t] = Rotation<kHalves>(row, row + kBlockTokens * (kHeadDim / 2), a.t.rot, ch).turned(k[t]);
        if (live(t)) largest = magnitude(largest, k[t]);
        __builtin_amdgcn_sched_barrier(0);  // one token after another: their registers are the limit
    }
    uint32_t mk = wave_max(__builtin_bit_cast(uint32_t, largest));
    if (__builtin_amdgcn_readfirstlane(mk >= 0x7F800000u)) {
        mk = 0;
#pragma unroll
        for (int t = 0; t < 8; t++)
            if (live(t)) mk = without_inf(mk, k[t]);
        mk = wave_max(mk);
    }
    const int bk = max(scale_byte(mk), was_k);
    const float fk = e8m0_as_f32((uint32_t)bk);
#pragma unroll
    for (int t = 0; t < 8; t++) {
        if (!some(t)) continue;
        tile[k_word(channels.first, slot_of(t))] =
            encode2<true>(encode2<false>(0, k[t][0], k[t][1], fk), k[t][2], k[t][3], fk);
        tile[k_word(channels.second, slot_of(t))] =
            encode2<true>(encode2<false>(0, k[t][4], k[t][5], fk), k[t][6], k[t][7], fk);
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int unit = 64 * i + lane, slot = unit & 31;  // 16 channels of a token
        u32x4* dst = reinterpret_cast<u32x4*>(kb + 16 * unit);
        if (kWhole || (slot >= p.lead && slot < p.stop)) {
            __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(tile + (unit >> 5) * 132 + slot * 4), dst);
        } else if (bk > was_k && slot < p.lead) {
            u32x4 q = *dst;
#pragma unroll
            for (int j = 0; j < 4; j++) q[j] = rescale4(q[j], was_k - bk);
            *dst = q;
        }
    }
    if (lane == 0) {
        c.ks[p.at] = (uint8_t)bk;
        c.vs[p.at] = (uint8_t)bv;
    }
}

template <bool kHalves>
__global__ __launch_bounds__(kThreads, 4) void cache_append_kernel(AppendArgs a) {
    __shared__ __align__(16) uint32_t s_v[kWaves][kTileWords];
    __shared__ __align__(16) float s_angles[2][kBlockTokens][kHeadDim / 2];  // cos, sin
    const CacheArgs& c = a.c;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int s = __builtin_amdgcn_readfirstlane(owner_of(c, blockIdx.x, 1, kBlockTokens, 2));
    if (s < 0) return;
    const TokenRange r = token_range(c, s);
    const int len = c.kv_len[s];
    if (len < 0 || len > (c.max_pages << c.bpp_log2) * kBlockTokens) return;
    const int first = len - (r.last - r.first);  // the new tokens' positions: first .. len - 1
    const int from = max(first, 0);
    if (from >= len || r.first == r.last) return;
    const int block = from / kBlockTokens + ((int)blockIdx.x - (r.first / kBlockTokens + 2 * s));
    const int p0 = block * kBlockTokens;
    if (p0 >= len) return;
    const int page = c.page_table[(int64_t)s * c.max_pages + (block >> c.bpp_log2)];
    if ((unsigned)page >= (unsigned)c.pages) return;
    Place p;
    p.head = blockIdx.y * kWaves + wave;
    p.at = (((int64_t)page * c.heads + p.head) << c.bpp_log2) + (block & ((1 << c.bpp_log2) - 1));
    p.row = (int64_t)r.first + p0 - first;
    p.lead = max(from - p0, 0);
    p.stop = min(len - p0, kBlockTokens);

    // the angles of the new tokens, eight lanes a row
    if (a.t.rot) {
        const int slot = threadIdx.x >> 3, half = a.t.rot >> 1;
        if (slot >= p.lead && slot < p.stop) {
            const int64_t pos = a.positions ? (int64_t)a.positions[p.row + slot] : (int64_t)(p0 + slot);
            const bool in = (uint64_t)pos < (uint64_t)a.t.table_rows;
            const float nan = __builtin_nanf("");
            for (int i = 4 * (threadIdx.x & 7); i < half; i += 32) {
                *reinterpret_cast<f32x4*>(&s_angles[0][slot][i]) =
                    in ? *reinterpret_cast<const f32x4*>(a.t.cos + pos * half + i) : f32x4{nan, nan, nan, nan};
                *reinterpret_cast<f32x4*>(&s_angles[1][slot][i]) =
                    in ? *reinterpret_cast<const f32x4*>(a.t.sin + pos * half + i) : f32x4{nan, nan, nan, nan};
            }
        }
    }
    if (p.head >= c.heads)
        __syncthreads();  // the others' barrier
    else if (p.lead == 0 && p.stop == kBlockTokens)
        append_block<kHalves, true>(a, p, s_v[wave], &s_angles[0][0][0]);
    else
        append_block<kHalves, false>(a, p, s_v[wave], &s_angles[0][0][0]);
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, bool halves, hipStream_t stream) {
    const dim3 grid((unsigned)(a.c.tokens / kBlockTokens + 2 * a.c.seqs), (unsigned)((a.c.heads + kWaves - 1) / kWaves));
    if (halves)
        cache_append_kernel<true><<<grid, kThreads, 0, stream>>>(a);
    else
        cache_append_kernel<false><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace mxattn
