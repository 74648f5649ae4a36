// cache_attend.hip -- attention over the 8-bit paged cache where a sequence has
// few query rows per KV head (a token or some drafts): bound by reading the keys.
//
// A wave takes a tile of 32 rows (cache_attend.h) and a run of its keys, straight from
// memory into the operands' registers, the next block in flight while one is worked
// on.  Long sequences: every wave has a share of the whole call's work, whatever the
// lengths are, and no wave waits for another; what a share's ends leave in pieces is
// joined by a second kernel.  Short ones: the four waves of a workgroup take an item's
// blocks in turn and meet in LDS.
//
// 64 sequences' single tokens over 8200 keys, 32 heads on 8: 606 MB, 117 to 120 us and
// 5 for the join, 5.0 TB/s; one over 118801 keys, 24 heads: 730 MB, 134 and 6, 5.4 TB/s
// (reading alone reaches 6.4 TB/s on this card); 16 x 4 tokens over 6000 keys, 40 heads
// on 8: 113 MB, 28 and 7; one over 512 keys, 2 heads: 8.0, a chain of loads (lengths,
// pages, codes).  With a window of 4096 keys and 4 sinks: 64 tokens far behind it 538 MB,
// 100 and 5, 5.4 TB/s; a row of 2 heads over 132 keys 6.6.  With scores kept for weights:
// 64 over 8200 keys 142 and 6, of which the 38 MB of scores are 22 (kept in one place
// instead they cost nothing; as whole 64-byte pieces, past the caches, or by strides of
// other channels the same).
#include "cache_attend.h"

#include <algorithm>

namespace mxattn {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 32;

// The shares of a call: n = 2^log2 of them, of the total number of units; a unit is
// 2^unit blocks of 32 keys of a tile, so that 32 bits hold the total.  An item is a
// tile of 32 rows of one sequence and KV head; the items lie in a row, sequence by
// sequence, head by head, tile by tile.
struct Cut {
    uint32_t total;
    int log2;
    // the first unit of share k; no share is empty before the units are used up
    __device__ __forceinline__ uint32_t first(int k) const {
        if (total >> log2) return (uint32_t)(((uint64_t)total * (uint32_t)k) >> log2);
        return min((uint32_t)k, total);
    }
    // the share that holds unit y (of the total, whatever q_start holds)
    __device__ __forceinline__ int of(uint32_t y) const {
        y = min(y, total - 1);
        if (!(total >> log2)) return (int)y;
        int k = (int)((float)y / (float)total * (float)(1 << log2));
        while (first(k) > y) k--;
        while (first(k + 1) <= y) k++;
        return k;
    }
};

// A sequence as the shares see it.
template <AttendKind kKind>
struct Sequence {
    int first, n;   // its tokens in the call
    int keys;       // -1: an impossible length
    int tiles;
    uint32_t units; // of a tile
    __device__ __forceinline__ Sequence(const CacheAttendArgs& a, int s, int unit) {
        const TokenRange r = token_range(a.c, s);
        first = r.first;
        n = r.last - r.first;
        keys = keys_of<kKind>(a, s);
        tiles = (n * a.group + kRows - 1) / kRows;
        units = (uint32_t)((most_blocks<kKind>(a, keys, kRows) + (1 << unit) - 1) >> unit);
    }
    __device__ __forceinline__ uint32_t all(int heads) const { return (uint32_t)tiles * (uint32_t)heads * units; }
};

// A wave's rows of a tile, and what they see.
template <AttendKind kKind>
struct Rows {
    int count, row;  // this lane's row
    Sight<kKind> sight;
    __device__ __forceinline__ Rows(const CacheAttendArgs& a, int first, int n, int keys, int row0, int q)
        : count(min(kRows, n * a.group - row0)),
          row(row0 + min(q, count - 1)),
          sight(a, first, n, keys, row, row0, row0 + count - 1) {}
};

// Places v0, v0 + step, ... below v1 of the walk of the wave's rows, the next block in
// flight while one is worked on.  (Two in flight through LDS gained nothing, and three
// copies of this loop's body in the instruction cache cost the short calls.)
template <AttendKind kKind, class Q>
__device__ __forceinline__ void attend_run(State& st, const CacheArgs& c, int s, int head, int v0, int v1, int step,
                                           const Q& qo, const Sight<kKind>& sight, float* scores_at, int q, int h) {
    if (v0 >= v1) return;
    const int last = v1 - 1;
    Block x, y;
    load_block(x, c, block_at(c, page_of(c, s, sight.block(v0)), head, sight.block(v0)), q, h);
    int page = page_of(c, s, sight.block(min(v0 + step, last)));
    for (int v = v0;; v += step) {
        // (behind the last block that one again: loads under a condition, the compiler waits
        // for the next block before this one)
        auto prefetch = [&] {
            const int next = sight.block(min(v + step, last));
            load_block(y, c, block_at(c, page, head, next), q, h);
            page = page_of(c, s, sight.block(min(v + 2 * step, last)));
        };
        attend_block<kKind>(st, x, qo, sight.block(v) * kBlockTokens, sight, scores_at, h, prefetch);
        if (v + step >= v1) break;
        x = y;
    }
}

// Where the scores of this lane's row are kept; null: nowhere.
template <AttendKind kKind>
__device__ __forceinline__ float* scores_of(const CacheAttendArgs& a, int64_t first, int row, int head, bool live) {
    if constexpr (kKind == kWeigh)
        return live ? a.scores + row_number(a, first, row, head) * a.score_stride : nullptr;
    else
        return nullptr;
}

// Where a share begins.
struct Start {
    uint32_t at, end;  // units of the whole row
    uint32_t offset;   // of `at` in sequence s
    int s;
};

template <AttendKind kKind>
__global__ __launch_bounds__(kThreads, 2) void cache_attend_shares_kernel(CacheAttendArgs a, int log2, int unit) {
    __shared__ uint32_t s_sum[kWaves];
    __shared__ bool s_ascend[kWaves];
    __shared__ Start s_start[kWaves];
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, q = lane & 31, h = lane >> 5;
    // all sequences' units before each thread's, and the total: none where q_start does not
    // ascend, as the sum would pass 32 bits and a share be found in two places
    const int per = (c.seqs + kThreads - 1) / kThreads;
    const int s0 = min(tid * per, c.seqs), s1 = min(s0 + per, c.seqs);
    uint32_t mine = 0;
    bool ascend = true;
    for (int s = s0; s < s1; s++) {
        mine += Sequence<kKind>(a, s, unit).all(c.heads);
        ascend = ascend && starts_ascend(c, s);
    }
    uint32_t incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t x = (uint32_t)__shfl_up((int)incl, d);
        if (lane >= d) incl += x;
    }
    ascend = __all(ascend);
    if (lane == 63) {
        s_sum[wave] = incl;
        s_ascend[wave] = ascend;
    }
    if (tid < kWaves) s_start[tid] = {0, 0, 0, 0};
    __syncthreads();
    Cut cut{0, log2};
    uint32_t before = incl - mine;
#pragma unroll
    for (int k = 0; k < kWaves; k++) {
        if (k < wave) before += s_sum[k];
        cut.total += s_sum[k];
    }
#pragma unroll
    for (int k = 0; k < kWaves; k++)
        if (!s_ascend[k]) cut.total = 0;
    cut.total = (uint32_t)__builtin_amdgcn_readfirstlane((int)cut.total);
#pragma unroll
    for (int k = 0; k < kWaves; k++) {
        const uint32_t lo = cut.first(blockIdx.x * kWaves + k), hi = cut.first(blockIdx.x * kWaves + k + 1);
        if (lo < hi && before <= lo && lo < before + mine) {
            uint32_t at = before;
            for (int s = s0; s < s1; s++) {
                const uint32_t all = Sequence<kKind>(a, s, unit).all(c.heads);
                if (lo < at + all) {
                    s_start[k] = {lo, hi, lo - at, s};
                    break;
                }
                at += all;
            }
        }
    }
    __syncthreads();
    const int index = blockIdx.x * kWaves + wave;
    uint32_t at = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_start[wave].at);
    const uint32_t end = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_start[wave].end);
    const uint32_t offset = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_start[wave].offset);
    int s = __builtin_amdgcn_readfirstlane(s_start[wave].s);
    const Parts<kRows> parts(a.workspace, 1 << log2);
    if (at < end) {
        Sequence<kKind> seq(a, s, unit);
        const uint32_t per_head = (uint32_t)seq.tiles * seq.units;
        int head = __builtin_amdgcn_readfirstlane((int)(offset / per_head));
        int tile = __builtin_amdgcn_readfirstlane((int)((offset - head * per_head) / seq.units));
        uint32_t x0 = offset - head * per_head - tile * seq.units;
        while (true) {
            const uint32_t x1 = min(seq.units, x0 + (end - at));
            const int keys = max(seq.keys, 0);
            const Rows<kKind> r(a, seq.first, seq.n, keys, tile * kRows, q);
            const int blocks = r.sight.count;
            const auto qo = load_q_of<kKind>(a.q + row_offset(a, seq.first, r.row, head, a.q_stride), h, a.scale,
                                       q < r.count && r.sight.some());
            State st;
            st.clear();
            attend_run<kKind>(st, c, s, head, min((int)(x0 << unit), blocks), min((int)(x1 << unit), blocks), 1, qo, r.sight,
                              scores_of<kKind>(a, seq.first, r.row, head, q < r.count), q, h);
            const float l = st.l + other_half(st.l);
            const bool whole = x0 == 0 && x1 == seq.units;
            if (q < r.count) {
                if (whole) {
                    if constexpr (kKind == kWeigh || kKind == kWeighStats)
                        if (h == 0) a.stats[row_number(a, seq.first, r.row, head)] = statistics(st.m, l);
                    store_row(st, inverse(l, seq.keys < 0), a.out + row_offset(a, seq.first, r.row, head, a.out_stride), h);
                } else {
                    store_part(st, l, parts, (2 * index + (x0 == 0)) * kRows + q, h);
                }
            }
            if (x0 == 0 && lane == 0)
                parts.info[(tile_number<kRows>(a, seq.first, s) + tile) * c.heads + head] = {
                    index, whole ? index : cut.of(at + seq.units - 1)};
            at += x1 - x0;
            if (at >= end) break;
            x0 = 0;
            if (++tile == seq.tiles) {
                tile = 0;
                if (++head == c.heads) {
                    head = 0;
                    do {  // (there is a next one, unless q_start was written meanwhile)
                        if (++s >= c.seqs) return;
                        seq = Sequence<kKind>(a, s, unit);
                    } while (seq.tiles == 0);
                }
            }
        }
    }
}

// One workgroup per item, numbered as the workgroups of the append: sequence s has
// tiles q_start[s] * group / 32 + s onwards.  A wave takes every fourth block.
template <AttendKind kKind>
__global__ __launch_bounds__(kThreads, 2) void cache_attend_items_kernel(CacheAttendArgs a) {
    __shared__ __align__(16) uint8_t s_o[kWaves][kRows * 512];
    __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, q = lane & 31, h = lane >> 5;
    const int s = __builtin_amdgcn_readfirstlane(owner_of(c, blockIdx.x, a.group, kRows, 1)), head = blockIdx.y;
    if (s < 0) return;
    const Sequence<kKind> seq(a, s, 0);
    const int row0 = ((int)blockIdx.x - tile_number<kRows>(a, seq.first, s)) * kRows;
    if (row0 >= seq.n * a.group) return;
    const int keys = max(seq.keys, 0);
    const Rows<kKind> r(a, seq.first, seq.n, keys, row0, q);
    const auto qo = load_q_of<kKind>(a.q + row_offset(a, seq.first, r.row, head, a.q_stride), h, a.scale,
                               q < r.count && r.sight.some());
    State st;
    st.clear();
    attend_run<kKind>(st, c, s, head, wave, r.sight.count, kWaves, qo, r.sight,
                      scores_of<kKind>(a, seq.first, r.row, head, q < r.count), q, h);
    // the 16-byte chunks of a row in an order of its own, so that rows written at once lie
    // in other banks
    auto o_at = [&](int w, int row, int chunk) { return s_o[w] + row * 512 + (chunk ^ row) * 16; };
    const float l = st.l + other_half(st.l);
    if (h == 0) {
        s_m[wave][q] = st.m;
        s_l[wave][q] = l;
    }
    if (q < r.count) {
        const float inv = inverse(l, false);
#pragma unroll
        for (int n = 0; n < 4; n++)
#pragma unroll
            for (int g = 0; g < 4; g++)
                *reinterpret_cast<float4*>(o_at(wave, q, 8 * n + 2 * g + h)) = four(st, n, g, inv);
    }
    __syncthreads();
    for (int e = tid; e < r.count * 32; e += kThreads) {
        const int i = e >> 5, ch = 4 * (e & 31);
        float m = s_m[0][i];
#pragma unroll
        for (int w = 1; w < kWaves; w++) m = max2(m, s_m[w][i]);
        float sum = 0.f, f[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
            f[w] = s_l[w][i] * __builtin_amdgcn_exp2f(s_m[w][i] - m);
            sum += f[w];
        }
        if constexpr (kKind == kWeigh || kKind == kWeighStats)
            if (ch == 0) a.stats[row_number(a, seq.first, row0 + i, head)] = statistics(m, sum);
        const float inv = reciprocal(sum);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWaves; w++) add_scaled(o, *reinterpret_cast<const float4*>(o_at(w, i, e & 31)), f[w] * inv);
        *reinterpret_cast<uint2*>(a.out + row_offset(a, seq.first, row0 + i, head, a.out_stride) + ch) =
            finished(o, seq.keys < 0);
    }
}

// Which kernel, from the caller's bounds on a sequence's query rows per KV head and the
// keys that a row sees (us, kernels with their joins; 8 KV heads):
//   few keys: an item is one workgroup's.  16 sequences x 5 rows x 1000 keys 13.6, in
//   shares 18.2; one sequence's row over 2000 keys 16.7 and 14.3.  Up to 128 rows: 90
//   rows x 290 keys 8.5, in shares 18.8, in tiles of 128 rows 33.  More rows, where 32 x 32
//   scores are not many (plain attention, whose callers know its bits, stays as it was):
//   4 sequences x 290 rows x 294 keys 12, in tiles 41; 35 x 445 rows of one head x 485 keys
//   21 and 37; 4 x 2048 rows x 512 keys (32 K of them) 46 and 63, 15 x 1704 of 3 heads x 569
//   (44 K) 67 and 71, 8 x 2048 x 768 (98 K) 108 and 97.
//   else up to 32 rows: shares; more: tiles of 128 rows, whose four waves read the keys
//   once.  16 sequences x 40 rows x 4000 keys, in shares 57, in tiles 50; 125 rows 83
//   and 61.
constexpr int64_t kFewBlocks = 40960;
int64_t score_blocks(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    return a.c.seqs * ((max_q * a.group + kRows - 1) / kRows) * a.c.heads * ((max_kv + kBlockTokens - 1) / kBlockTokens);
}
enum Way { kItems, kShares, kTiles };
Way way(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    const int64_t rows = max_q * a.group;
    if (max_kv <= 1024 && (rows <= 128 || (a.kind != kPlain && score_blocks(a, max_q, max_kv) <= kFewBlocks))) return kItems;
    return rows <= kRows ? kShares : kTiles;
}

// log2 of the number of shares: four waves per CU, with 16 KiB each in flight, reach the
// memory's rate and leave half as many parts as the eight that fit (one row over 118801
// keys x 24 heads 137 us for 142, 20000 keys x 8 heads 22 for 28; two waves 225 and 23);
// a share has at least two blocks (one of 16: 4 rows over 6000 keys 32 us for 20) and
// an item at most 256 parts (1856 of one row took 44 us to join), as far as the
// caller's bounds say.
int shares_log2(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    const int64_t items = a.c.seqs * ((max_q * a.group + kRows - 1) / kRows) * a.c.heads;
    const int64_t blocks = (max_kv + kBlockTokens - 1) / kBlockTokens;
    int log2 = 2;
    while (log2 < 10 && (items * blocks) >> (log2 + 1) >= 2 && items * 256 >> (log2 + 1) >= 1) log2++;
    return log2;
}

// The keys that a row sees, at most.
int64_t seen_keys(const CacheAttendArgs& a, int64_t max_kv) {
    return a.kind == kWindow ? std::min<int64_t>(max_kv, (int64_t)a.window + a.sinks) : max_kv;
}

template <AttendKind kKind>
hipError_t launch(const CacheAttendArgs& a, Way w, int64_t max_q, int64_t max_kv, hipStream_t stream) {
    const int64_t tiles = tile_numbers<kRows>(a);
    if (w == kItems) {
        cache_attend_items_kernel<kKind><<<dim3((unsigned)tiles, (unsigned)a.c.heads), kThreads, 0, stream>>>(a);
        return hipGetLastError();
    }
    // units that keep the total of all items within 31 bits, however long the sequences are
    int unit = 0;
    while ((tiles * a.c.heads * ((((int64_t)a.c.max_pages << a.c.bpp_log2) >> unit) + 1)) >> 31) unit++;
    const int log2 = shares_log2(a, max_q, max_kv);
    cache_attend_shares_kernel<kKind><<<(1 << log2) / kWaves, kThreads, 0, stream>>>(a, log2, unit);
    if (hipError_t e = hipGetLastError()) return e;
    return launch_cache_attend_join<kRows, kKind>(a, 1 << log2, stream);
}

}  // namespace

size_t cache_attend_workspace(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    max_kv = seen_keys(a, max_kv);
    switch (way(a, max_q, max_kv)) {
        case kItems: return 0;
        case kShares: return parts_bytes<kRows>(a, 1 << shares_log2(a, max_q, max_kv));
        default: return cache_attend_tiles_workspace(a, max_q, max_kv);
    }
}

bool cache_attend_keeps_scores(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    return way(a, max_q, max_kv) != kTiles && max_q * a.group <= 128;
}

hipError_t launch_cache_attend(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv, hipStream_t stream) {
    max_kv = seen_keys(a, max_kv);
    const Way w = way(a, max_q, max_kv);
    if (w == kTiles) return launch_cache_attend_tiles(a, max_q, max_kv, stream);
    switch (a.kind) {
        case kWindow: return launch<kWindow>(a, w, max_q, max_kv, stream);
        case kTree: return launch<kTree>(a, w, max_q, max_kv, stream);
        case kWeigh: return launch<kWeigh>(a, w, max_q, max_kv, stream);
        case kWeighStats: return launch<kWeighStats>(a, w, max_q, max_kv, stream);
        default: return launch<kPlain>(a, w, max_q, max_kv, stream);
    }
}

}  // namespace mxattn
