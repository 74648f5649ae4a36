// cache.h -- argument structures and launchers of the operators around the
// 8-bit paged cache: per-head norm and rotation (rope.hip), appending
// (cache_append.hip) and attention over it (cache_attend.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mxattn {

constexpr int kHeadDim = 128;
constexpr int kBlockTokens = 32;   // tokens of a head that share a scale
constexpr int kBlockBytes = 4096;  // codes of a block of K or V

// Norm and rotation of one tensor's heads; w null: no norm, rot 0: no rotation.
struct HeadTransform {
    const float* cos;  // [table_rows, rot / 2]
    const float* sin;
    int64_t table_rows;
    float eps;
    int rot;
};

// A tensor [B, H, N, 128] of bf16 by the strides of its first three axes (elements).
struct Strided {
    uint16_t* p;
    int64_t b, h, n;
};

struct RopeArgs {
    Strided in[2], out[2];    // Q and K
    const float* w[2];
    HeadTransform t;
    const int32_t* positions; // [B, N] or null: a token's index in its batch
    int64_t tokens;           // B * N
    int N, Hq, Hkv;
    int64_t first;            // set by the launcher: the first token of a launch
};
hipError_t launch_qk_norm_rope(const RopeArgs& a, bool halves, hipStream_t stream);

// The paged cache and what a call does with it.
struct CacheArgs {
    uint8_t *kc, *vc;           // [pages, heads, blocks per page, 4096]
    uint8_t *ks, *vs;           // [pages, heads, blocks per page]
    const int32_t* page_table;  // [seqs, max_pages]
    const int32_t* q_start;     // [seqs + 1]
    const int32_t* kv_len;      // [seqs]
    int seqs, tokens, heads, pages, max_pages;
    int bpp_log2;               // blocks per page
};

struct AppendArgs {
    CacheArgs c;
    const uint16_t *k, *v;  // [tokens, heads, 128] by token strides
    int64_t k_stride, v_stride;
    const float* w;
    HeadTransform t;
    const int32_t* positions;  // [tokens] or null: a token's place in its sequence
};
hipError_t launch_cache_append(const AppendArgs& a, bool halves, hipStream_t stream);

struct CacheAttendArgs {
    CacheArgs c;
    const uint16_t* q;  // [tokens, Hq, 128] by its token stride
    uint16_t* out;
    int64_t q_stride, out_stride;
    int group;          // Hq / heads, at most 256
    uint64_t per_group; // ceil(2^36 / group)
    int causal;
    float scale;        // log2(e) / sqrt(128)
    uint8_t* workspace; // cache_attend_workspace bytes
};
// max_q, max_kv: most new tokens and keys of a sequence, as far as the caller knows
// (wrong ones cost time, and may change where f16 and fp32 round).
size_t cache_attend_workspace(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv);
hipError_t launch_cache_attend(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv, hipStream_t stream);

// Tiles of 128 query rows (cache_attend_tiles.hip).
size_t cache_attend_tiles_workspace(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv);
hipError_t launch_cache_attend_tiles(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv, hipStream_t stream);

// New tokens of sequence s: [first, last) of the call's tokens, whatever
// q_start holds.
struct TokenRange {
    int first, last;
};
__device__ __forceinline__ TokenRange token_range(const CacheArgs& c, int s) {
    const int a = min(max(c.q_start[s], 0), c.tokens);
    const int b = min(max(c.q_start[s + 1], a), c.tokens);
    return {a, b};
}

// Whether sequence s + 1's tokens begin behind the start of sequence s's. Where that
// holds for all, the sequences' tokens add up to at most the call's, and sums over them
// stay within what the launch was sized for.
__device__ __forceinline__ bool starts_ascend(const CacheArgs& c, int s) {
    return min(max(c.q_start[s], 0), c.tokens) <= min(max(c.q_start[s + 1], 0), c.tokens);
}

// The sequence that owns workgroup w where sequence s has workgroups
// (its first token) * group / unit + step * s onwards, up to those of s + 1; -1: none.
// All lanes of a wave call it: 64 places probed at a time.
__device__ __forceinline__ int64_t first_group(const CacheArgs& c, int s, int64_t group, int unit, int step) {
    const int first = min(max(c.q_start[s], 0), c.tokens);
    return (int64_t)first * group / unit + (int64_t)step * s;
}
__device__ __forceinline__ int owner_of(const CacheArgs& c, int64_t w, int64_t group, int unit, int step) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = c.seqs;
    while (true) {
        const int each = (hi - lo + 63) / 64, s = lo + lane * each;
        const uint64_t at = __ballot(s < hi && first_group(c, s, group, unit, step) <= w);
        if (!at) return -1;
        lo += (63 - __builtin_clzll(at)) * each;
        if (each == 1) break;
        hi = min(hi, lo + each);
    }
    return w < first_group(c, lo + 1, group, unit, step) ? lo : -1;
}

}  // namespace mxattn
