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
// pages, codes).
#include "cache_attend.h"

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
struct Sequence {
    int first, n;   // its tokens in the call
    int keys;       // -1: an impossible length
    int tiles;
    uint32_t units; // of a tile
    __device__ __forceinline__ Sequence(const CacheAttendArgs& a, int s, int unit) {
        const TokenRange r = token_range(a.c, s);
        first = r.first;
        n = r.last - r.first;
        keys = keys_of(a.c, s);
        tiles = (n * a.group + kRows - 1) / kRows;
        const int blocks = (max(keys, 1) + kBlockTokens - 1) / kBlockTokens;
        units = (uint32_t)((blocks + (1 << unit) - 1) >> unit);
    }
    __device__ __forceinline__ uint32_t all(int heads) const { return (uint32_t)tiles * (uint32_t)heads * units; }
};

// A wave's rows of a tile.
struct Rows {
    int count, row, end, min_end, max_end;  // this lane's row and the keys that it, the first and the last row see
    __device__ __forceinline__ Rows(const CacheAttendArgs& a, int n, int keys, int row0, int q) {
        count = min(kRows, n * a.group - row0);
        row = row0 + min(q, count - 1);
        end = a.causal ? keys - n + token_of(a, row) + 1 : keys;
        min_end = a.causal ? keys - n + token_of(a, row0) + 1 : keys;
        max_end = max(0, a.causal ? keys - n + token_of(a, row0 + count - 1) + 1 : keys);
    }
};

// Blocks b0, b0 + step, ... below b1 for the wave's rows, the next one in flight while
// one is worked on.  (Two in flight through LDS gained nothing, and three copies of
// this loop's body in the instruction cache cost the short calls.)
__device__ __forceinline__ void attend_run(State& st, const CacheArgs& c, int s, int head, int b0, int b1, int step,
                                           const QOperand& qo, const Rows& r, int keys, int q, int h) {
    if (b0 >= b1) return;
    const int last = b1 - 1;
    Block x, y;
    load_block(x, c, block_at(c, page_of(c, s, b0), head, b0), q, h);
    int page = page_of(c, s, min(b0 + step, last));
    for (int b = b0;; b += step) {
        if (b + step < b1) {
            load_block(y, c, block_at(c, page, head, b + step), q, h);
            page = page_of(c, s, min(b + 2 * step, last));
        }
        attend_block(st, x, qo, b * kBlockTokens, r.end, keys, (b + 1) * kBlockTokens > r.min_end, h);
        if (b + step >= b1) break;
        x = y;
    }
}

// Where a share begins.
struct Start {
    uint32_t at, end;  // units of the whole row
    uint32_t offset;   // of `at` in sequence s
    int s;
};

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
        mine += Sequence(a, s, unit).all(c.heads);
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
                const uint32_t all = Sequence(a, s, unit).all(c.heads);
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
        Sequence seq(a, s, unit);
        const uint32_t per_head = (uint32_t)seq.tiles * seq.units;
        int head = __builtin_amdgcn_readfirstlane((int)(offset / per_head));
        int tile = __builtin_amdgcn_readfirstlane((int)((offset - head * per_head) / seq.units));
        uint32_t x0 = offset - head * per_head - tile * seq.units;
        while (true) {
            const uint32_t x1 = min(seq.units, x0 + (end - at));
            const int keys = max(seq.keys, 0);
            const Rows r(a, seq.n, keys, tile * kRows, q);
            const int blocks = (r.max_end + kBlockTokens - 1) / kBlockTokens;
            const QOperand qo = load_q(a.q + row_offset(a, seq.first, r.row, head, a.q_stride), h, a.scale,
                                       q < r.count && r.end > 0);
            State st;
            st.clear();
            attend_run(st, c, s, head, min((int)(x0 << unit), blocks), min((int)(x1 << unit), blocks), 1, qo, r, keys, q, h);
            const float l = st.l + other_half(st.l);
            const bool whole = x0 == 0 && x1 == seq.units;
            if (q < r.count) {
                if (whole) {
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
                        seq = Sequence(a, s, unit);
                    } while (seq.tiles == 0);
                }
            }
        }
    }
}

// One workgroup per item, numbered as the workgroups of the append: sequence s has
// tiles q_start[s] * group / 32 + s onwards.  A wave takes every fourth block.
__global__ __launch_bounds__(kThreads, 2) void cache_attend_items_kernel(CacheAttendArgs a) {
    __shared__ __align__(16) uint8_t s_o[kWaves][kRows * 512];
    __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, q = lane & 31, h = lane >> 5;
    const int s = __builtin_amdgcn_readfirstlane(owner_of(c, blockIdx.x, a.group, kRows, 1)), head = blockIdx.y;
    if (s < 0) return;
    const Sequence seq(a, s, 0);
    const int row0 = ((int)blockIdx.x - tile_number<kRows>(a, seq.first, s)) * kRows;
    if (row0 >= seq.n * a.group) return;
    const int keys = max(seq.keys, 0);
    const Rows r(a, seq.n, keys, row0, q);
    const QOperand qo = load_q(a.q + row_offset(a, seq.first, r.row, head, a.q_stride), h, a.scale,
                               q < r.count && r.end > 0);
    State st;
    st.clear();
    attend_run(st, c, s, head, wave, (r.max_end + kBlockTokens - 1) / kBlockTokens, kWaves, qo, r, keys, q, h);
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
        const float inv = reciprocal(sum);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWaves; w++) add_scaled(o, *reinterpret_cast<const float4*>(o_at(w, i, e & 31)), f[w] * inv);
        *reinterpret_cast<uint2*>(a.out + row_offset(a, seq.first, row0 + i, head, a.out_stride) + ch) =
            finished(o, seq.keys < 0);
    }
}

// Which kernel, from the caller's bounds on a sequence's query rows per KV head and its
// keys (us, kernels with their joins; 8 KV heads):
//   few keys: an item is one workgroup's.  16 sequences x 5 rows x 1000 keys 13.6, in
//   shares 18.2; one sequence's row over 2000 keys 16.7 and 14.3.  Up to 128 rows: 90
//   rows x 290 keys 8.5, in shares 18.8, in tiles of 128 rows 33.
//   else up to 32 rows: shares; more: tiles of 128 rows, whose four waves read the keys
//   once.  16 sequences x 40 rows x 4000 keys, in shares 57, in tiles 50; 125 rows 83
//   and 61.
enum Way { kItems, kShares, kTiles };
Way way(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    const int64_t rows = max_q * a.group;
    if (max_kv <= 1024 && rows <= 128) return kItems;
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

}  // namespace

size_t cache_attend_workspace(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    switch (way(a, max_q, max_kv)) {
        case kItems: return 0;
        case kShares: return parts_bytes<kRows>(a, 1 << shares_log2(a, max_q, max_kv));
        default: return cache_attend_tiles_workspace(a, max_q, max_kv);
    }
}

hipError_t launch_cache_attend(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv, hipStream_t stream) {
    const Way w = way(a, max_q, max_kv);
    if (w == kTiles) return launch_cache_attend_tiles(a, max_q, max_kv, stream);
    const int64_t tiles = tile_numbers<kRows>(a);
    if (w == kItems) {
        cache_attend_items_kernel<<<dim3((unsigned)tiles, (unsigned)a.c.heads), kThreads, 0, stream>>>(a);
        return hipGetLastError();
    }
    // units that keep the total of all items within 31 bits, however long the sequences are
    int unit = 0;
    while ((tiles * a.c.heads * ((((int64_t)a.c.max_pages << a.c.bpp_log2) >> unit) + 1)) >> 31) unit++;
    const int log2 = shares_log2(a, max_q, max_kv);
    cache_attend_shares_kernel<<<(1 << log2) / kWaves, kThreads, 0, stream>>>(a, log2, unit);
    if (hipError_t e = hipGetLastError()) return e;
    return launch_cache_attend_join<kRows>(a, 1 << log2, stream);
}

}  // namespace mxattn
