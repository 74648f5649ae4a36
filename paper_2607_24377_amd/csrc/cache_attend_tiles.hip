// cache_attend_tiles.hip -- attention over the 8-bit paged cache where a sequence
// has many query rows per KV head (prompts, a video's next frame): bound by the
// matrix cores and the softmax's vector work.
//
// A workgroup takes a tile of 128 rows, 32 per wave, and walks its keys 64 at a
// time.  K's and V's codes (16 KiB) are copied straight into LDS, in the lanes'
// operand order, two steps ahead of their use, and each wave reads them as they are:
// FP8 operands for the scores, and codes that become f16 in registers for the
// second product.  Two waves a SIMD (256 registers) run each other's gaps.
//
// 1560 rows x 32760 keys x 40 heads: 1.11 to 1.15 ms, 910 to 940 TFLOP/s; matrix cores
// busy 47 %, vector issue 55 % (141 instructions per 32 x 32 scores, about 830
// cycles), LDS half of its time; 3.4 GB fetched, ten times the keys and values, 3 TB/s
// beside the products.  Other forms, measured with probabilities in bf16 (1.10 to 1.13):
// 256 rows in eight waves 1.10, 64 rows per wave 1.72 (spills), one wave a SIMD 1.21, V as
// 16 bits in LDS, made once for the four waves, 1.25 (more to read there); the next scores
// under this step's softmax, a wait for the step before only, or priorities of the waves
// gained nothing.
//
// With a window the walk leaves blocks out (Sight), and no tile weighs more than window,
// sinks and its own span: 1560 rows, 12480 keys and 1560 sinks of 32760 x 40 heads 0.51 to 0.54
// ms, 830 to 880 TFLOP/s; 4 prompts of up to 2048 tokens, 1000 keys, 32 heads on 8: 142 to 150
// us and 18 for the join, 550 TFLOP/s of the keys that are seen.  4 prompts of 2048 tokens
// with 32 keys take 69 us: what does not grow with the keys is 17 us for each of the four
// tiles of a workgroup, of which three steps are 6.  Trees of 25 drafts of 16 sequences
// over 6000 keys, 40 heads on 8: 48 and 8, of which 20 stay however few the keys are (the
// share's place, first loads, parts of 64 KiB written); trees of 64 over 65536 keys, 2
// sequences: 161 to 166 and 10, 830 to 850 TFLOP/s.  Masked steps are said to be rare, so that the others'
// code runs straight on: those prompts 148 us without, the frame 3 % more.
#include "cache_attend.h"

namespace mxattn {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 32 * kWaves;
constexpr int kKeys = 64;               // keys of a step: two blocks
constexpr int kStageBytes = 4 * kBlockBytes;  // K, K, V, V

typedef __attribute__((address_space(3))) void* lds_ptr_t;

// ---------------------------------------------------------------------------
// Shares.  An item's weight is what it costs, in keys: the same for every tile of a
// sequence, or, causal, growing by a constant from tile to tile.  All items' weights in
// a row are cut into equal shares, one per workgroup.

// The tiles of a sequence: tile t of a head weighs a + b (t + 1), but from tile `full` on
// what tile full - 1 and those behind it would pass: `most`.
template <AttendKind kKind>
struct SeqWork {
    int64_t a, most;
    int tiles, b, full;
    __device__ __forceinline__ int64_t before(int64_t t) const {
        if constexpr (kKind == kWindow)
            if (t > full) return full * a + b * ((int64_t)full * (full + 1) / 2) + (t - full) * most;
        return t * a + b * (t * (t + 1) / 2);
    }
    __device__ __forceinline__ int64_t weight(int t) const {
        if constexpr (kKind == kWindow)
            if (t >= full) return most;
        return a + (int64_t)b * (t + 1);
    }
    __device__ __forceinline__ bool even() const { return kKind != kWindow && b == 0; }
};

template <AttendKind kKind>
__device__ __forceinline__ SeqWork<kKind> seq_work(const CacheAttendArgs& a, int n, int keys) {
    const int64_t rows = (int64_t)n * a.group;
    SeqWork<kKind> w;
    w.tiles = (int)((rows + kRows - 1) / kRows);
    if (kKind != kTree && a.causal) {  // in units of a key times the group: kRows / group keys more per tile
        w.a = (int64_t)max(keys - n, 0) * a.group;
        w.b = kRows;
    } else {
        w.a = max(keys, 1);
        w.b = 0;
    }
    if constexpr (kKind == kWindow) {  // no tile sees more than the window, the sinks and its own rows' span
        w.most = (int64_t)a.window + a.sinks;
        if (w.b) w.most = w.most * a.group + kRows;
        if (!w.b && w.a < w.most) w.most = w.a;
        w.full = w.b ? (int)min(max((w.most - w.a) / kRows, (int64_t)0), (int64_t)w.tiles) : 0;
    }
    return w;
}
template <AttendKind kKind>
__device__ __forceinline__ SeqWork<kKind> seq_work(const CacheAttendArgs& a, int s) {
    const TokenRange r = token_range(a.c, s);
    return seq_work<kKind>(a, r.last - r.first, keys_of<kKind>(a, s));
}

// A workgroup's place in the row of all items, and how far its share goes.
struct Share {
    int64_t at, end;  // of the total weight
    int64_t offset;   // of `at` within sequence s
    int64_t total;
    int s, n;         // n: shares (no more than there is weight, so none is empty)
};

__device__ __forceinline__ int64_t uniform64(int64_t x) {
    const int lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
    return ((int64_t)hi << 32) | (uint32_t)lo;
}

// The share of workgroup i of n, empty for all where q_start does not ascend (the
// sum of the weights could pass 64 bits); all kThreads threads call it.
template <AttendKind kKind>
__device__ __forceinline__ Share find_share(const CacheAttendArgs& a, int i, int n) {
    __shared__ int64_t s_sum[kThreads / 64];
    __shared__ bool s_ascend[kThreads / 64];
    __shared__ Share s_share;
    const int tid = threadIdx.x, seqs = a.c.seqs;
    const int per = (seqs + kThreads - 1) / kThreads;
    const int s0 = min(tid * per, seqs), s1 = min(s0 + per, seqs);
    int64_t mine = 0;
    bool ascend = true;
    for (int s = s0; s < s1; s++) {
        const SeqWork<kKind> w = seq_work<kKind>(a, s);
        mine += w.before(w.tiles) * a.c.heads;
        ascend = ascend && starts_ascend(a.c, s);
    }
    int64_t incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t x = __shfl_up(incl, d);
        if ((tid & 63) >= d) incl += x;
    }
    ascend = __all(ascend);
    if ((tid & 63) == 63) {
        s_sum[tid >> 6] = incl;
        s_ascend[tid >> 6] = ascend;
    }
    if (tid == 0) s_share = {0, 0, 0, 0, -1, 0};
    __syncthreads();
    int64_t total = 0, before = incl - mine;
#pragma unroll
    for (int k = 0; k < kThreads / 64; k++) {
        if (k < (tid >> 6)) before += s_sum[k];
        total += s_sum[k];
    }
#pragma unroll
    for (int k = 0; k < kThreads / 64; k++)
        if (!s_ascend[k]) total = 0;
    n = (int)(total < n ? total : n);
    const int64_t lo = i < n ? total * i / n : total, hi = i < n ? total * (i + 1) / n : total;
    if (i < n && before <= lo && lo < before + mine) {
        int64_t at = before;
        for (int s = s0; s < s1; s++) {
            const SeqWork<kKind> w = seq_work<kKind>(a, s);
            const int64_t all = w.before(w.tiles) * a.c.heads;
            if (lo < at + all) {
                s_share = {lo, hi, lo - at, total, s, n};
                break;
            }
            at += all;
        }
    }
    __syncthreads();
    return {uniform64(s_share.at), uniform64(s_share.end), uniform64(s_share.offset), uniform64(s_share.total),
            __builtin_amdgcn_readfirstlane(s_share.s), __builtin_amdgcn_readfirstlane(s_share.n)};
}

// The place of a share's work: an item, of which the share has the part from x0 on.  Only
// the first one takes divisions and a search; the loads of a sequence's numbers come once.
// (For every item, 2 us of a windowed tile's 10.)
template <AttendKind kKind>
struct Cursor {
    int64_t at, end, total;  // of the whole weight
    int64_t x0;
    int s, n_shares, index;
    int head, tile;
    int first, n, keys;      // the sequence's new tokens and its keys (-1: no such cache)
    SeqWork<kKind> w;
    __device__ __forceinline__ Cursor(const CacheAttendArgs& a, const Share& sh, int index_)
        : at(sh.at), end(sh.end), total(sh.total), s(sh.s), n_shares(sh.n), index(index_) {
        if (!more(a)) return;
        load(a);
        const int64_t per_head = w.before(w.tiles);
        head = __builtin_amdgcn_readfirstlane((int)(sh.offset / per_head));
        const int64_t r = uniform64(sh.offset - head * per_head);
        tile = 0;
        if (w.even()) {
            tile = __builtin_amdgcn_readfirstlane((int)(r / w.a));
        } else {
            int hi = w.tiles - 1;  // the last tile that starts at or before r
            while (tile < hi) {
                const int mid = (tile + hi + 1) >> 1;
                if (w.before(mid) <= r)
                    tile = mid;
                else
                    hi = mid - 1;
            }
        }
        x0 = r - w.before(tile);
    }
    // (s is a sequence, unless q_start was written meanwhile)
    __device__ __forceinline__ bool more(const CacheAttendArgs& a) const { return at < end && s < a.c.seqs; }
    __device__ __forceinline__ void load(const CacheAttendArgs& a) {
        const TokenRange r = token_range(a.c, s);
        first = __builtin_amdgcn_readfirstlane(r.first);
        n = __builtin_amdgcn_readfirstlane(r.last) - first;
        keys = __builtin_amdgcn_readfirstlane(keys_of<kKind>(a, s));
        w = seq_work<kKind>(a, n, keys);
    }
    __device__ __forceinline__ int64_t weight() const { return w.weight(tile); }
    __device__ __forceinline__ int64_t x1() const { return min(x0 + (end - at), weight()); }
    __device__ __forceinline__ bool whole() const { return x0 == 0 && end - at >= weight(); }
    // The item's PartInfo: the share that holds its last unit of weight, y, is the largest k
    // with total k / n <= y.
    __device__ __forceinline__ void describe(const CacheAttendArgs& a, PartInfo* info) const {
        const int64_t y = at + weight() - 1;
        const int last = whole() ? index : (int)(((y + 1) * n_shares - 1) / total);
        info[(tile_number<kRows>(a, first, s) + tile) * a.c.heads + head] = {index, last};
    }
    __device__ __forceinline__ void next(const CacheAttendArgs& a) {
        at += x1() - x0;
        x0 = 0;
        if (++tile < w.tiles) return;
        tile = 0;
        if (++head < a.c.heads) return;
        head = 0;
        if (at >= end) return;
        do {
            if (++s >= a.c.seqs) return;
            load(a);
        } while (w.tiles == 0);
    }
};

// What a step's operands need beside their codes: the blocks' scale bytes.
struct Scales {
    int k[2], v[2];
    bool lost[2];
};

// Copies of a step's blocks into LDS: part p (1 KiB) of a block is the operand
// register group p of all lanes, 16 bytes each.  Wave w copies part w of each.
struct StepLoader {
    int koff, voff;  // of this lane in a block
    int wave;
    __device__ __forceinline__ StepLoader(int wave_, int lane) : wave(wave_) {
        const int q = lane & 31, h = lane >> 5;
        koff = (4 * (wave >> 1) + 2 * h + (wave & 1)) * 512 + operand_key(q) * 16;
        voff = wave * 1024 + q * 32 + 16 * h;
    }
    __device__ __forceinline__ void copy(const uint8_t* block, int off, uint8_t* dst) const {
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)block, 0, kBlockBytes, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)(dst + wave * 1024), 16, off, 0, 0, 0);
    }
    // The blocks at places v and v + 1 of the walk (the second only where there is one: else the last again, for keys
    // that are masked), of these pages.
    template <AttendKind kKind>
    __device__ __forceinline__ void load(Scales& s, uint8_t* stage, const CacheArgs& c, const int (&page)[2], int head,
                                         int v, const Sight<kKind>& sight) const {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const BlockAt p = block_at(c, page[i], head, sight.block(min(v + i, sight.count - 1)));
            copy(c.kc + p.at * kBlockBytes, koff, stage + i * kBlockBytes);
            copy(c.vc + p.at * kBlockBytes, voff, stage + (2 + i) * kBlockBytes);
            s.k[i] = c.ks[p.at];
            s.v[i] = c.vs[p.at];
            s.lost[i] = p.lost;
        }
    }
    template <AttendKind kKind>
    static __device__ __forceinline__ void pages(int (&page)[2], const CacheArgs& c, int seq, int v,
                                                 const Sight<kKind>& sight) {
#pragma unroll
        for (int i = 0; i < 2; i++) page[i] = page_of(c, seq, sight.block(min(v + i, sight.count - 1)));
    }
};

__device__ __forceinline__ uint4 part(const uint8_t* block, int p, int lane) {
    return *reinterpret_cast<const uint4*>(block + p * 1024 + lane * 16);
}

template <class Q>
__device__ __forceinline__ v16f block_scores(const uint8_t* block, int e, const Q& q, int lane) {
    uint4 k[4];
#pragma unroll
    for (int p = 0; p < 4; p++) k[p] = part(block, p, lane);
    return scores(k, e, q);
}

// The softmax of a step's scores and its products with V.  `sees`: the keys of its two
// blocks that the lane's row sees; `held`: keys that the sequence has in them; `any`:
// whether some row does not see all.
template <class Mask>
__device__ __forceinline__ void step(State& st, v16f (&s)[2], const uint8_t* stage, const Scales& x, float c,
                                     const Mask (&sees)[2], const int (&held)[2], bool any, int h, int lane) {
    const bool lost = x.lost[0] || x.lost[1];
    if (__builtin_expect(any || lost, 0)) {
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) s[b][i] = sees[b].masked(x.lost[b] ? __builtin_nanf("") : s[b][i], i);
    }
    float mx = max2(max2(s[0][0], s[0][1]), s[1][0]), my = max2(max2(s[0][2], s[0][3]), s[1][1]);
#pragma unroll
    for (int i = 4; i < 16; i += 4) {  // (a three-input maximum for every two scores)
        mx = max2(max2(mx, s[0][i]), s[0][i + 1]);
        my = max2(max2(my, s[0][i + 2]), s[0][i + 3]);
    }
#pragma unroll
    for (int i = 2; i < 14; i += 4) {
        mx = max2(max2(mx, s[1][i]), s[1][i + 1]);
        my = max2(max2(my, s[1][i + 2]), s[1][i + 3]);
    }
    mx = max2(max2(mx, s[1][14]), max2(my, s[1][15]));
    mx = __builtin_fmaf(mx, c, -kTopLog2);
    const float m = max2(st.m, max2(mx, other_half(mx)));
    if (__any(m > st.m)) st.raise(m);  // else every alpha is 1
#pragma unroll
    for (int b = 0; b < 2; b++) {
        const v16f p = st.exponentials(s[b], c, m);
        const f16x8 p0 = probabilities(p, 0), p1 = probabilities(p, 1);
        uint4 v[4];
#pragma unroll
        for (int n = 0; n < 4; n++) v[n] = part(stage + (2 + b) * kBlockBytes, n, lane);
        int e = x.v[b];
        if (__builtin_expect(any || lost, 0)) clean_values(st, v, e, sees[b], held[b], x.lost[b], h);
        const float vscale = st.value_scale(e);
#pragma unroll
        for (int n = 0; n < 4; n++) {
            st.O[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(to_f16(v[n].x, v[n].y, vscale), p0, st.O[n], 0, 0, 0);
            st.O[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(to_f16(v[n].z, v[n].w, vscale), p1, st.O[n], 0, 0, 0);
        }
    }
}

// Workgroups 8 apart run on one XCD; the shares of one XCD are neighbours, which
// read the same keys.
__device__ __forceinline__ int share_index() { return (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3); }

template <AttendKind kKind>
__global__ __launch_bounds__(kThreads, 2) void cache_attend_tiles_kernel(CacheAttendArgs a) {
    __shared__ __align__(16) uint8_t st0[kStageBytes];
    __shared__ __align__(16) uint8_t st1[kStageBytes];
    __shared__ __align__(16) uint8_t st2[kStageBytes];
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, q = lane & 31, h = lane >> 5;
    const int index = share_index();
    Cursor<kKind> it(a, find_share<kKind>(a, index, gridDim.x), index);
    const Parts<kRows> parts(a.workspace, gridDim.x);
    const StepLoader loader(wave, lane);
    for (; it.more(a); it.next(a)) {
        const int keys = max(it.keys, 0), row0 = it.tile * kRows, rows = min(kRows, it.n * a.group - row0);
        // this wave's rows: the tile's last one for those that are not there
        const int wrow = 32 * wave, wrows = min(32, rows - wrow);
        const bool live = q < wrows;
        const int row = row0 + min(wrow + q, rows - 1);
        const Sight<kKind> all(a, it.first, it.n, keys, row, row0, row0 + rows - 1);
        const Sight<kKind> sight(a, it.first, it.n, keys, row, row0 + min(wrow, rows - 1), row0 + min(wrow + 31, rows - 1));
        const int steps = (all.count + 1) / 2;
        const int64_t x1 = it.x1(), weight = it.weight();
        const int j0 = it.x0 == 0 ? 0 : (int)(it.x0 * steps / weight), j1 = x1 == weight ? steps : (int)(x1 * steps / weight);
        State st;
        Scales x0, x1s, x2;
        int page[2];
        auto load_first = [&] {
            __syncthreads();  // the stages are free
            if (j0 >= j1) return;
            StepLoader::pages(page, c, it.s, 2 * j0, all);
            loader.load(x0, st0, c, page, it.head, 2 * j0, all);
            StepLoader::pages(page, c, it.s, 2 * j0 + 2, all);
            if (j0 + 1 < j1) loader.load(x1s, st1, c, page, it.head, 2 * j0 + 2, all);
            StepLoader::pages(page, c, it.s, 2 * j0 + 4, all);
        };
        if (kKind == kWindow) load_first();
        const auto qo = load_q_of<kKind>(a.q + row_offset(a, it.first, row, it.head, a.q_stride), h, a.scale, live && sight.some());
        st.clear();
        if (kKind != kWindow) load_first();
        if (j0 < j1) {
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            auto one = [&](int j, const uint8_t* cur, uint8_t* far, const Scales& xc, Scales& xf) {
                if (j + 2 < j1) {
                    loader.load(xf, far, c, page, it.head, 2 * j + 4, all);
                    StepLoader::pages(page, c, it.s, 2 * j + 6, all);
                }
                v16f s[2];
                s[0] = block_scores(cur, xc.k[0], qo, lane);
                s[1] = block_scores(cur + kBlockBytes, xc.k[1], qo, lane);
                const int at[2] = {all.block(2 * j) * kBlockTokens, all.block(2 * j + 1) * kBlockTokens};
                const bool any = sight.partial(at[0]) || sight.partial(at[1]);
                const auto m0 = sight.mask_of(at[0], any, h), m1 = sight.mask_of(at[1], any, h);
                const decltype(m0) sees[2] = {m0, m1};
                const int held[2] = {keys - at[0], keys - at[1]};
                step(st, s, cur, xc, qo.c, sees, held, any, h, lane);
                __builtin_amdgcn_s_waitcnt(0);  // the next but one landed
                __syncthreads();
            };
            for (int j = j0; j < j1; j += 3) {
                one(j, st0, st2, x0, x2);
                if (j + 1 < j1) one(j + 1, st1, st0, x1s, x0);
                if (j + 2 < j1) one(j + 2, st2, st1, x2, x1s);
            }
        }
        const float l = st.l + other_half(st.l);
        if (live) {
            if (it.whole()) {
                if constexpr (kKind == kWeighStats)
                    if (h == 0) a.stats[row_number(a, it.first, row, it.head)] = statistics(st.m, l);
                store_row(st, inverse(l, it.keys < 0), a.out + row_offset(a, it.first, row, it.head, a.out_stride), h);
            } else {
                store_part(st, l, parts, (int64_t)(2 * index + (it.x0 == 0)) * kRows + wrow + q, h);
            }
        }
        if (it.x0 == 0 && tid == 0) it.describe(a, parts.info);
    }
}

// Two workgroups per CU are resident (registers); fewer where a share would have less
// than four steps, as far as the caller's bounds say; a multiple of the 8 XCDs.
int workgroups(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    int64_t tiles = a.c.seqs * ((max_q * a.group + kRows - 1) / kRows);
    if (tiles > tile_numbers<kRows>(a)) tiles = tile_numbers<kRows>(a);
    const int64_t n = tiles * a.c.heads * ((max_kv + kKeys - 1) / kKeys) / 4;
    return n >= 512 ? 512 : n < 8 ? 8 : (int)n & ~7;
}

template <AttendKind kKind>
hipError_t launch(const CacheAttendArgs& a, int n, hipStream_t stream) {
    cache_attend_tiles_kernel<kKind><<<n, kThreads, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    return launch_cache_attend_join<kRows, kKind>(a, n, stream);
}

}  // namespace

size_t cache_attend_tiles_workspace(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    return parts_bytes<kRows>(a, workgroups(a, max_q, max_kv));
}

hipError_t launch_cache_attend_tiles(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv, hipStream_t stream) {
    const int n = workgroups(a, max_q, max_kv);
    switch (a.kind) {
        case kWindow: return launch<kWindow>(a, n, stream);
        case kTree: return launch<kTree>(a, n, stream);
        case kWeighStats: return launch<kWeighStats>(a, n, stream);
        case kWeigh: return hipErrorInvalidValue;  // (these kernels keep no scores)
        default: return launch<kPlain>(a, n, stream);
    }
}

}  // namespace mxattn
