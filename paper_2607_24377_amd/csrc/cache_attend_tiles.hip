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

// The tiles of a sequence: tile t of a head weighs a + b (t + 1).
struct SeqWork {
    int64_t a;
    int tiles, b;
    __device__ __forceinline__ int64_t before(int64_t t) const { return t * a + b * (t * (t + 1) / 2); }
    __device__ __forceinline__ int64_t weight(int t) const { return a + (int64_t)b * (t + 1); }
};

__device__ __forceinline__ SeqWork seq_work(const CacheAttendArgs& a, int s) {
    const TokenRange r = token_range(a.c, s);
    const int64_t rows = (int64_t)(r.last - r.first) * a.group;
    const int keys = keys_of(a.c, s);
    SeqWork w;
    w.tiles = (int)((rows + kRows - 1) / kRows);
    if (a.causal) {  // in units of a key times the group: kRows / group keys more per tile
        w.a = (int64_t)max(keys - (r.last - r.first), 0) * a.group;
        w.b = kRows;
    } else {
        w.a = max(keys, 1);
        w.b = 0;
    }
    return w;
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
        const SeqWork w = seq_work(a, s);
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
            const SeqWork w = seq_work(a, s);
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

// One item and the part of it that a workgroup works on.
struct Item {
    int s, head, row0;
    int64_t x0, x1, w;  // from x0 to x1 of its weight w
    int last;           // the share of its last part
    int number;         // PartInfo's
    __device__ __forceinline__ bool whole() const { return x0 == 0 && x1 == w; }
};

// The item at the share's place; the share moves on behind it.
__device__ __forceinline__ Item next_item(const CacheAttendArgs& a, Share& sh) {
    const SeqWork w = seq_work(a, sh.s);
    const int64_t per_head = w.before(w.tiles);
    Item it;
    it.s = sh.s;
    it.head = __builtin_amdgcn_readfirstlane((int)(sh.offset / per_head));
    const int64_t r = uniform64(sh.offset - it.head * per_head);
    int t = 0;
    if (w.b == 0) {
        t = __builtin_amdgcn_readfirstlane((int)(r / w.a));
    } else {
        int hi = w.tiles - 1;  // the last tile that starts at or before r
        while (t < hi) {
            const int mid = (t + hi + 1) >> 1;
            if (w.before(mid) <= r)
                t = mid;
            else
                hi = mid - 1;
        }
    }
    it.row0 = t * kRows;
    it.number = (tile_number<kRows>(a, token_range(a.c, sh.s).first, sh.s) + t) * a.c.heads + it.head;
    it.w = w.weight(t);
    it.x0 = r - w.before(t);
    it.x1 = it.x0 + (sh.end - sh.at) < it.w ? it.x0 + (sh.end - sh.at) : it.w;
    const int64_t step = it.x1 - it.x0;
    // the share that holds the item's last unit of weight, y: the largest k with total k / n <= y
    const int64_t y = sh.at + (it.w - it.x0) - 1;
    it.last = __builtin_amdgcn_readfirstlane((int)(((y + 1) * sh.n - 1) / sh.total));
    sh.at += step;
    sh.offset += step;
    if (sh.at < sh.end && sh.offset >= per_head * a.c.heads) {
        sh.offset = 0;
        do sh.s++;
        while (sh.s < a.c.seqs && seq_work(a, sh.s).tiles == 0);
    }
    return it;
}

// Which rows a tile has and what they see.
struct TileRows {
    int n, keys;           // the sequence's new tokens and keys
    int rows;              // rows of the tile
    int min_end, max_end;  // keys that its first and its last row see
    int64_t first;         // the sequence's first token in the call
    bool bad;              // no such cache
};
__device__ __forceinline__ TileRows tile_rows(const CacheAttendArgs& a, int s, int row0) {
    const TokenRange r = token_range(a.c, s);
    TileRows t;
    t.n = r.last - r.first;
    t.first = r.first;
    const int keys = __builtin_amdgcn_readfirstlane(keys_of(a.c, s));
    t.bad = keys < 0;
    t.keys = max(keys, 0);
    t.rows = min(kRows, t.n * a.group - row0);
    t.min_end = a.causal ? t.keys - t.n + token_of(a, row0) + 1 : t.keys;
    t.max_end = max(0, a.causal ? t.keys - t.n + token_of(a, row0 + t.rows - 1) + 1 : t.keys);
    return t;
}

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
    // Blocks b and b + 1 (the second only below `blocks`: else the first again, for keys that are masked) of
    // these pages.
    __device__ __forceinline__ void load(Scales& s, uint8_t* stage, const CacheArgs& c, const int (&page)[2], int head,
                                         int b, int blocks) const {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const BlockAt p = block_at(c, page[i], head, min(b + i, blocks - 1));
            copy(c.kc + p.at * kBlockBytes, koff, stage + i * kBlockBytes);
            copy(c.vc + p.at * kBlockBytes, voff, stage + (2 + i) * kBlockBytes);
            s.k[i] = c.ks[p.at];
            s.v[i] = c.vs[p.at];
            s.lost[i] = p.lost;
        }
    }
    static __device__ __forceinline__ void pages(int (&page)[2], const CacheArgs& c, int seq, int b, int blocks) {
#pragma unroll
        for (int i = 0; i < 2; i++) page[i] = page_of(c, seq, min(b + i, blocks - 1));
    }
};

__device__ __forceinline__ uint4 part(const uint8_t* block, int p, int lane) {
    return *reinterpret_cast<const uint4*>(block + p * 1024 + lane * 16);
}

__device__ __forceinline__ v16f block_scores(const uint8_t* block, int e, const QOperand& q, int lane) {
    uint4 k[4];
#pragma unroll
    for (int p = 0; p < 4; p++) k[p] = part(block, p, lane);
    return scores(k, e, q);
}

// The softmax of a step's scores and its products with V.  `visible`: keys of the
// step that the lane's row sees; `held`: keys that the sequence has in it; `any`:
// whether some row does not see all.
__device__ __forceinline__ void step(State& st, v16f (&s)[2], const uint8_t* stage, const Scales& x, float c, int visible,
                                     int held, bool any, int h, int lane) {
    const bool lost = x.lost[0] || x.lost[1];
    if (any || lost) {
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const float y = x.lost[b] ? __builtin_nanf("") : s[b][i];
                s[b][i] = 32 * b + 16 * h + i < visible ? y : -__builtin_inff();
            }
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
        if (any || lost) clean_values(st, v, e, 32 * b, visible, held, x.lost[b], h);
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

__global__ __launch_bounds__(kThreads, 2) void cache_attend_tiles_kernel(CacheAttendArgs a) {
    __shared__ __align__(16) uint8_t st0[kStageBytes];
    __shared__ __align__(16) uint8_t st1[kStageBytes];
    __shared__ __align__(16) uint8_t st2[kStageBytes];
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, q = lane & 31, h = lane >> 5;
    const int index = share_index();
    Share sh = find_share(a, index, gridDim.x);
    const Parts<kRows> parts(a.workspace, gridDim.x);
    const StepLoader loader(wave, lane);
    while (sh.at < sh.end && sh.s < c.seqs) {  // (it is, unless q_start was written meanwhile)
        const Item it = next_item(a, sh);
        const TileRows t = tile_rows(a, it.s, it.row0);
        const int blocks = (t.max_end + kBlockTokens - 1) / kBlockTokens;
        const int steps = (blocks + 1) / 2;
        const int j0 = (int)(it.x0 * steps / it.w), j1 = (int)(it.x1 * steps / it.w);
        // this wave's rows
        const int wrow = 32 * wave, wrows = min(32, t.rows - wrow);
        const bool live = q < wrows;
        const int row = it.row0 + min(wrow + q, t.rows - 1);
        const int end = a.causal ? t.keys - t.n + token_of(a, row) + 1 : t.keys;
        const int wmin = a.causal ? t.keys - t.n + token_of(a, it.row0 + min(wrow, t.rows - 1)) + 1 : t.keys;
        const QOperand qo = load_q(a.q + row_offset(a, t.first, row, it.head, a.q_stride), h, a.scale, live && end > 0);
        State st;
        st.clear();
        Scales x0, x1, x2;
        __syncthreads();  // the stages are free
        if (j0 < j1) {
            int page[2];
            StepLoader::pages(page, c, it.s, 2 * j0, blocks);
            loader.load(x0, st0, c, page, it.head, 2 * j0, blocks);
            StepLoader::pages(page, c, it.s, 2 * j0 + 2, blocks);
            if (j0 + 1 < j1) loader.load(x1, st1, c, page, it.head, 2 * j0 + 2, blocks);
            StepLoader::pages(page, c, it.s, 2 * j0 + 4, blocks);
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            auto one = [&](int j, const uint8_t* cur, uint8_t* far, const Scales& xc, Scales& xf) {
                if (j + 2 < j1) {
                    loader.load(xf, far, c, page, it.head, 2 * j + 4, blocks);
                    StepLoader::pages(page, c, it.s, 2 * j + 6, blocks);
                }
                v16f s[2];
                s[0] = block_scores(cur, xc.k[0], qo, lane);
                s[1] = block_scores(cur + kBlockBytes, xc.k[1], qo, lane);
                step(st, s, cur, xc, qo.c, end - j * kKeys, t.keys - j * kKeys, (j + 1) * kKeys > wmin, h, lane);
                __builtin_amdgcn_s_waitcnt(0);  // the next but one landed
                __syncthreads();
            };
            for (int j = j0; j < j1; j += 3) {
                one(j, st0, st2, x0, x2);
                if (j + 1 < j1) one(j + 1, st1, st0, x1, x0);
                if (j + 2 < j1) one(j + 2, st2, st1, x2, x1);
            }
        }
        const float l = st.l + other_half(st.l);
        const bool whole = it.whole();
        if (live) {
            if (whole)
                store_row(st, inverse(l, t.bad), a.out + row_offset(a, t.first, row, it.head, a.out_stride), h);
            else
                store_part(st, l, parts, (int64_t)(2 * index + (it.x0 == 0)) * kRows + wrow + q, h);
        }
        if (it.x0 == 0 && tid == 0) parts.info[it.number] = {index, it.last};
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

}  // namespace

size_t cache_attend_tiles_workspace(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    return parts_bytes<kRows>(a, workgroups(a, max_q, max_kv));
}

hipError_t launch_cache_attend_tiles(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv, hipStream_t stream) {
    const int n = workgroups(a, max_q, max_kv);
    cache_attend_tiles_kernel<<<n, kThreads, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    return launch_cache_attend_join<kRows>(a, n, stream);
}

}  // namespace mxattn
