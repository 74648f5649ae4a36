// cache_weigh.hip -- the weight that attention gives every cached key: the sum of its
// probabilities over a sequence's new tokens and the query heads of its KV head, added
// to what it had.
//
//   w'[j] = (j < past ? w[j] : 0) + sum over rows r of p_rj,  p_rj = 2^(s_rj c - m_r) / l_r
//
// The attention kernels leave m and 1 / l of every row (in fp32, those that divided its
// output).  Few rows: they leave the scores too, 4 bytes per row and key beside the 256
// bytes of a key's codes, and a second pass over them sums.  Many rows: the scores are
// computed once more, keys outside, rows inside, so that every sum stays in a wave's
// registers and no order of additions depends on the schedule.  Either way the scores that
// become weights are fp32 sums of exact products (QExact).
#include "cache_attend.h"

#include <algorithm>

namespace mxattn {
namespace {

constexpr int kThreads = 256;

// A sequence as both kernels see it; no work where `n` is 0.
struct Keys {
    int first, n, keys;
    __device__ __forceinline__ Keys(const CacheAttendArgs& a, int s) {
        const TokenRange r = token_range(a.c, s);
        first = r.first;
        n = r.last - r.first;
        keys = keys_of<kWeigh>(a, s);
        if (keys < 0) n = 0;
    }
};

// Where the weights of key j on lie (up to the end of its page); -1: no such page.
__device__ __forceinline__ int64_t weights_at(const CacheArgs& c, int s, int head, int j) {
    const int log2 = c.bpp_log2 + 5;
    const int page = c.page_table[(int64_t)s * c.max_pages + (j >> log2)];
    if ((unsigned)page >= (unsigned)c.pages) return -1;
    return (((int64_t)page * c.heads + head) << log2) + (j & ((1 << log2) - 1));
}

__device__ __forceinline__ float sum_with(const CacheWeighArgs& w, int64_t at, bool old, float add) {
    return (old && w.before ? w.before[at] : 0.f) + add;
}

// From the scores: four keys a thread, the rows one after another.
__global__ __launch_bounds__(kThreads) void cache_weigh_scores_kernel(CacheWeighArgs w) {
    const CacheAttendArgs& a = w.a;
    const int s = blockIdx.x, head = blockIdx.y;
    const Keys k(a, s);
    if (k.n == 0) return;
    const int past = k.keys - k.n;
    for (int64_t j64 = ((int64_t)blockIdx.z * kThreads + threadIdx.x) * 4; j64 < k.keys;
         j64 += (int64_t)gridDim.z * kThreads * 4) {
        const int j = (int)j64;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int t = a.causal ? max(0, j - past) : 0; t < k.n; t++) {
            const int end = a.causal ? past + t + 1 : k.keys;
            const int64_t row = ((int64_t)(k.first + t) * a.c.heads + head) * a.group;
            for (int g = 0; g < a.group; g++) {
                const float2 ml = a.stats[row + g];
                const float4 x = *reinterpret_cast<const float4*>(a.scores + (row + g) * a.score_stride + j);
                sum.x += __builtin_amdgcn_exp2f(x.x - ml.x) * ml.y;
                if (j + 1 < end) sum.y += __builtin_amdgcn_exp2f(x.y - ml.x) * ml.y;
                if (j + 2 < end) sum.z += __builtin_amdgcn_exp2f(x.z - ml.x) * ml.y;
                if (j + 3 < end) sum.w += __builtin_amdgcn_exp2f(x.w - ml.x) * ml.y;
            }
        }
        const int64_t at = weights_at(a.c, s, head, j);
        if (at < 0) continue;
        const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (j + i < k.keys) w.after[at + i] = sum_with(w, at + i, j + i < past, v[i]);
    }
}

// From K and Q: a wave holds two blocks of keys and walks all rows that see some of them.
constexpr int kWaves = 4;
constexpr int kBlocks = 2;
constexpr int kGroupKeys = kWaves * kBlocks * kBlockTokens;

__global__ __launch_bounds__(64 * kWaves, 2) void cache_weigh_rows_kernel(CacheWeighArgs w) {
    const CacheAttendArgs& a = w.a;
    const CacheArgs& c = a.c;
    const int s = blockIdx.x, head = blockIdx.y;
    const Keys k(a, s);
    if (k.n == 0) return;
    const int past = k.keys - k.n, rows = k.n * a.group;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q = lane & 31, h = lane >> 5;
    for (int64_t j64 = (int64_t)blockIdx.z * kGroupKeys + wave * kBlocks * kBlockTokens; j64 < k.keys;
         j64 += (int64_t)gridDim.z * kGroupKeys) {
        const int base = (int)j64;
        const int last = (k.keys + kBlockTokens - 1) / kBlockTokens - 1;
        KExact keys[kBlocks];
        int scale[kBlocks];
        float sum[kBlocks][16];
#pragma unroll
        for (int b = 0; b < kBlocks; b++) {
            const int i = min(base / kBlockTokens + b, last);
            const BlockAt p = block_at(c, page_of(c, s, i), head, i);
            const uint8_t* kb = c.kc + p.at * kBlockBytes + 2 * h * 512 + operand_key(q) * 16;
            uint4 codes[4];
#pragma unroll
            for (int e = 0; e < 4; e++) codes[e] = *reinterpret_cast<const uint4*>(kb + (4 * (e >> 1) + (e & 1)) * 512);
            scale[b] = c.ks[p.at];
            keys[b] = exact_keys(codes, scale[b]);
#pragma unroll
            for (int e = 0; e < 16; e++) sum[b][e] = 0.f;
        }
        // the first row whose token sees key `base`
        const int from = a.causal ? max(0, base - past) * a.group : 0;
        for (int row0 = from & ~31; row0 < rows; row0 += 32) {
            const int row = min(row0 + q, rows - 1);
            const int end = a.causal ? past + token_of(a, row) + 1 : k.keys;
            const int min_end = a.causal ? past + token_of(a, row0) + 1 : k.keys;
            const bool live = row0 + q < rows && end > 0;
            const QExact qo = load_q_exact(a.q + row_offset(a, k.first, row, head, a.q_stride), h, a.scale, live);
            float2 ml = make_float2(0.f, 0.f);
            if (live) ml = a.stats[row_number(a, k.first, row, head)];
#pragma unroll
            for (int b = 0; b < kBlocks; b++) {
                const int at = base + b * kBlockTokens;
                const v16f x = scores(keys[b], scale[b], qo);
                const bool any = at + kBlockTokens > min_end;
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], qo.c, -ml.x));
                    const float y = __builtin_fmaf(p, ml.y, sum[b][e]);
                    sum[b][e] = any && at + 16 * h + e >= end ? sum[b][e] : y;
                }
            }
        }
        // the sums of the 32 rows' lanes; lane e of each half keeps that of key 16 h + e
#pragma unroll
        for (int b = 0; b < kBlocks; b++) {
            float mine = 0.f;
#pragma unroll
            for (int e = 0; e < 16; e++) {
                float x = sum[b][e];
#pragma unroll
                for (int d = 1; d < 32; d *= 2) x += __shfl_xor(x, d);
                mine = q == e ? x : mine;
            }
            const int j = base + b * kBlockTokens + 16 * h + q;
            if (q >= 16 || j >= k.keys) continue;
            const int64_t at = weights_at(c, s, head, j);
            if (at >= 0) w.after[at] = sum_with(w, at, j < past, mine);
        }
    }
}

// Scores are kept up to this many bytes; beyond, they are computed twice.
constexpr int64_t kMostScores = (int64_t)1 << 30;

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

// Workgroups along z: one for each `keys` keys, but no launch past 2^32 threads.
unsigned chunks(const CacheAttendArgs& a, int64_t max_kv, int keys) {
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 23) / ((int64_t)a.c.seqs * a.c.heads));
    return (unsigned)std::min<int64_t>(std::min<int64_t>(most, 65535), (max_kv + keys - 1) / keys);
}

// Chooses the kind, and where what the kernels leave for the sums lies; returns the bytes.
size_t lay_out(CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    const int64_t rows = (int64_t)a.c.tokens * a.c.heads * a.group;
    a.score_stride = (max_kv + 31) / 32 * 32;
    a.kind = cache_attend_keeps_scores(a, max_q, max_kv) && rows <= kMostScores / 4 / a.score_stride ? kWeigh : kWeighStats;
    const size_t parts = up16(cache_attend_workspace(a, max_q, max_kv));
    const size_t stats = up16((size_t)rows * sizeof(float2));
    a.stats = reinterpret_cast<float2*>(a.workspace + parts);
    a.scores = reinterpret_cast<float*>(a.workspace + parts + stats);
    return parts + stats + (a.kind == kWeigh ? (size_t)rows * (size_t)a.score_stride * 4 : 0);
}

}  // namespace

size_t cache_weigh_workspace(CacheAttendArgs a, int64_t max_q, int64_t max_kv) { return lay_out(a, max_q, max_kv); }

hipError_t launch_cache_weigh(CacheWeighArgs w, int64_t max_q, int64_t max_kv, hipStream_t stream) {
    CacheAttendArgs& a = w.a;
    a.most_keys = (int)max_kv;
    lay_out(a, max_q, max_kv);
    if (hipError_t e = launch_cache_attend(a, max_q, max_kv, stream)) return e;
    if (a.kind == kWeigh) {
        const dim3 grid((unsigned)a.c.seqs, (unsigned)a.c.heads, chunks(a, max_kv, 4 * kThreads));
        cache_weigh_scores_kernel<<<grid, kThreads, 0, stream>>>(w);
    } else {
        const dim3 grid((unsigned)a.c.seqs, (unsigned)a.c.heads, chunks(a, max_kv, kGroupKeys));
        cache_weigh_rows_kernel<<<grid, 64 * kWaves, 0, stream>>>(w);
    }
    return hipGetLastError();
}

}  // namespace mxattn
