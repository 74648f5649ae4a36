// cache.h -- argument structures and launchers of the operators around the
// 8-bit paged cache: per-head norm and rotation (rope.hip), appending
// (cache_append.hip), attention over it (cache_attend.hip), the weights of its keys
// (cache_weigh.hip), and cutting and moving what it holds (cache_evict.hip).
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

// What a call of attention over the cache sees and leaves beside its output.
enum AttendKind {
    kPlain,       // all keys, or causal
    kWindow,      // of those the last `window` and the first `sinks`
    kTree,        // what was there before, and of the new keys those of a row's mask
    kWeigh,       // as kPlain, and every row's scores and softmax statistics are kept
    kWeighStats,  // as kPlain, and the statistics alone
};

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
    AttendKind kind;
    int window, sinks;           // kWindow: at most kMaxKeys each, window >= 1
    const int32_t* tree;         // kTree: [tokens, tree_words]
    int tree_words;
    int most_keys;               // kWeigh, kWeighStats: a longer sequence is none
    float2* stats;               // [tokens * Hq]: m and 1 / l of every row, p = exp2(s c - m) / l
    float* scores;               // kWeigh: [tokens * Hq, score_stride], s (without c) of the keys that a tile of rows sees
    int64_t score_stride;        // a multiple of 32
};
// max_q, max_kv: most new tokens and keys of a sequence, as far as the caller knows
// (wrong ones cost time, and may change where f16 and fp32 round).
size_t cache_attend_workspace(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv);
hipError_t launch_cache_attend(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv, hipStream_t stream);
// Whether such a call's kernel can keep the scores (kWeigh; else kWeighStats).
bool cache_attend_keeps_scores(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv);

// Attention that also adds to every key's weight (cache_weigh.hip); a.kind and what
// follows it are chosen by the call.
struct CacheWeighArgs {
    CacheAttendArgs a;
    const float* before;  // [pages, heads, page_tokens]; null: zeros
    float* after;
    float* partial;          // set by the call, as what follows: [runs, seqs * heads, partial_stride]
    int64_t partial_stride;
    int runs;
};
size_t cache_weigh_workspace(CacheWeighArgs w, int64_t max_q, int64_t max_kv);
hipError_t launch_cache_weigh(CacheWeighArgs w, int64_t max_q, int64_t max_kv, hipStream_t stream);

// Which tokens stay, and moving them together (cache_evict.hip).
struct SelectArgs {
    CacheArgs c;           // pages, table and lengths alone
    const float* weights;  // [pages, heads, page_tokens]
    int budget, sinks, recent;
    int32_t* kept;         // [seqs, heads, budget]
    int32_t* counts;       // [seqs]
    uint8_t* workspace;    // cache_select_workspace bytes, 16-byte aligned
    int chunk_keys, chunks;  // set by the launcher, as what follows
    size_t item_bytes;
};
// items: sequences times heads; reach: the most keys of a sequence that its table holds.
size_t cache_select_workspace(int64_t items, int64_t reach);
hipError_t launch_cache_select(const SelectArgs& a, hipStream_t stream);

struct CompactArgs {
    CacheArgs c;               // (no q_start and kv_len)
    const int32_t* out_table;  // [seqs, out_pages]: where the tokens go
    int out_pages;
    bool in_place;             // out_table is the page table
    const int32_t* kept;       // [seqs, heads or 1, width]
    int64_t kept_head;         // elements from head to head
    int64_t kept_seq;          // from sequence to sequence
    int width;
    const int32_t* counts;     // [seqs]
    const int32_t* base;       // [seqs] or null: 0
    float* weights;            // [pages, heads, page_tokens] or null
};
hipError_t launch_cache_compact(const CompactArgs& a, hipStream_t stream);

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

// Workgroups of a launch over items (a sequence's heads) and chunks of each.  Workgroups go
// to the 8 XCDs in turn and there to its shader engines in turn, so an item's chunks follow
// one another on one XCD, whose L2 holds what they share, and spread over all its engines.
// (In the order of sequences, one of four that was the longest lay on two XCDs, or on an
// engine of each: the sums of 4 prompts' weights took 358 and 272 us, and 169 so.)
struct Placed {
    int s, head, chunk;  // s < 0: none
    __device__ __forceinline__ Placed(const CacheArgs& c, int chunks) {
        const unsigned items = (unsigned)c.seqs * (unsigned)c.heads, n = (unsigned)chunks;
        const unsigned id = blockIdx.x + gridDim.x * blockIdx.y;
        const unsigned t = items < 8 ? id : id >> 3, k = t / n, item = items < 8 ? k : (id & 7) + 8 * k;
        chunk = (int)(t - k * n);
        s = item < items ? (int)(item / (unsigned)c.heads) : -1;
        head = (int)item - s * c.heads;
    }
};
// Its grid, of so many threads each: two dimensions where one would pass a launch's 2^32.
inline dim3 placed_grid(const CacheArgs& c, int64_t chunks, int threads) {
    const int64_t items = (int64_t)c.seqs * c.heads, n = (items < 8 ? items : (items + 7) / 8 * 8) * chunks;
    int64_t rows = 1;  // (n is a multiple of 8 where there are so many)
    while (n / rows * threads >> 32) rows *= 2;
    return dim3((unsigned)(n / rows), (unsigned)rows);
}

}  // namespace mxattn
