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
// registers and no order of additions depends on the schedule.  Either way p's score is
// the very number that l is a sum over: both come from one product of the same operands in
// the same order, an fp32 sum of exact products (QExact), and s c - m is rounded once in
// both.  A row's p then add up to 1 within the roundings of l's additions whatever the
// scores' size, and each is off by its score's error, 2^-20 of sum |q k| / sqrt(d) and less
// (m and l from FP8 products, as attention alone takes them, are off by up to 2^-15 of that:
// 160 rows of scores of some hundreds added up to 159.97).
//
// Bound by what attention leaves and by the exponentials: 64 tokens over 8200 keys, 32 heads
// on 8, 57 MB, 15 us; 4 prompts of up to 2048 tokens 135 to 139 us, beside 261 and 19 for their
// attention, which FP8 products would do in 241 (86 vector instructions for 32 x 32 scores, 16 of them exponentials; vector issue
// busy 44 %, matrix cores 28 %; the longest prompt's 128 steps follow one another); 1560 rows
// x 32760 keys x 40 heads 730.
#include "cache_attend.h"

#include <algorithm>

namespace mxattn {
namespace {

constexpr int kThreads = 64;  // (four waves a workgroup 17.5 us for 15.6)

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
__global__ __launch_bounds__(kThreads) void cache_weigh_scores_kernel(CacheWeighArgs w, int chunks) {
    const CacheAttendArgs& a = w.a;
    const Placed place(a.c, chunks);
    const int s = place.s, head = place.head;
    if (s < 0) return;
    const Keys k(a, s);
    if (k.n == 0) return;
    const int past = k.keys - k.n;
    for (int64_t j64 = ((int64_t)place.chunk * kThreads + threadIdx.x) * 4; j64 < k.keys;
         j64 += (int64_t)chunks * kThreads * 4) {
        const int j = (int)j64;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        // the rows that see key j, four in flight (a token's heads lie in a row)
        const int64_t row0 = ((int64_t)k.first * a.c.heads + head) * a.group, token = (int64_t)a.c.heads * a.group;
        const int rows = k.n * a.group;
        // (s c - m in one rounding, as in l)
        auto weight = [&a](float score, float2 ml) {
            return __builtin_amdgcn_exp2f(__builtin_fmaf(score, a.scale, -ml.x)) * ml.y;
        };
        for (int r = a.causal ? max(0, j - past) * a.group : 0; r < rows; r += 4) {
            float2 ml[4];
            float4 x[4];
            int end[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int ri = min(r + i, rows - 1), t = token_of(a, ri);
                const int64_t row = row0 + t * token + (ri - t * a.group);
                end[i] = r + i >= rows ? 0 : a.causal ? past + t + 1 : k.keys;
                ml[i] = a.stats[row];
                x[i] = *reinterpret_cast<const float4*>(a.scores + row * a.score_stride + j);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (j < end[i]) sum.x += weight(x[i].x, ml[i]);
                if (j + 1 < end[i]) sum.y += weight(x[i].y, ml[i]);
                if (j + 2 < end[i]) sum.z += weight(x[i].z, ml[i]);
                if (j + 3 < end[i]) sum.w += weight(x[i].w, ml[i]);
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

// From K and Q.  A workgroup takes 128 keys, held as operands by its waves, and walks the
// rows that see some of them, 64 a step: waves w and w + 4 have the same block and a half of
// the rows each.  Q comes through LDS, two steps ahead: 16 lanes copy a row,
// its 16-byte chunks in an order of its own, so that lanes that read a chunk of all rows
// read all banks.
constexpr int kWaves = 8;
constexpr int kKeyWaves = 4;
constexpr int kStepRows = 64;
constexpr int kStageBytes = kStepRows * 256;
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef const __attribute__((address_space(1))) void* global_ptr_t;

// s_waitcnt: all but two of the wave's loads have landed (vmcnt 2), and all it read from LDS.
constexpr int kTwoInFlight = 2 | 7 << 4;

// A row of the sequence that moves on by kStepRows, and where what belongs to it lies (the
// division by the group once: 64-bit products for each row of each step took as many
// instructions as the sums).
struct Walk {
    const uint8_t* p;
    int row, g;  // (and its head in the group)
};
// kWhole: a step is whole tokens (the group divides it).
template <bool kWhole>
struct Stride {
    int64_t token, row, step, carry;  // bytes from token to token and head to head, of a step, and where a step passes a token
    int group, g;
    __device__ __forceinline__ Stride(const CacheAttendArgs& a, int64_t token_, int64_t row_) : token(token_), row(row_) {
        const int tokens = token_of(a, kStepRows);
        group = a.group;
        g = kStepRows - tokens * group;
        step = tokens * token + g * row;
        carry = token - group * row;
    }
    // Row r of the sequence whose row 0 is at p.
    __device__ __forceinline__ Walk at(const CacheAttendArgs& a, const void* p, int r) const {
        const int t = token_of(a, r), g = r - t * group;
        return {static_cast<const uint8_t*>(p) + t * token + g * row, r, g};
    }
    __device__ __forceinline__ void advance(Walk& w) const {
        w.row += kStepRows;
        w.p += step;
        if constexpr (kWhole) return;
        w.g += g;
        if (w.g >= group) {
            w.g -= group;
            w.p += carry;
        }
    }
};

template <bool kWhole>
__global__ __launch_bounds__(64 * kWaves, 4) void cache_weigh_rows_kernel(CacheWeighArgs w, int chunks, int runs) {
    __shared__ __align__(16) uint8_t st0[kStageBytes];
    __shared__ __align__(16) uint8_t st1[kStageBytes];
    __shared__ __align__(16) uint8_t st2[kStageBytes];
    __shared__ float s_sum[kKeyWaves * kBlockTokens];
    const CacheAttendArgs& a = w.a;
    const CacheArgs& c = a.c;
    const Placed place(a.c, chunks * runs);
    const int s = place.s, head = place.head;
    if (s < 0) return;
    const Keys k(a, s);
    if (k.n == 0) return;
    const int past = k.keys - k.n, rows = k.n * a.group;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q = lane & 31, h = lane >> 5;
    constexpr int kGroupKeys = kKeyWaves * kBlockTokens;
    const int last = (k.keys + kBlockTokens - 1) / kBlockTokens - 1;
    const int half = wave >> 2, chunk = place.chunk / runs, run = place.chunk - chunk * runs;
    const Stride<kWhole> by_q(a, a.q_stride * 2, kHeadDim * 2), by_stats(a, (int64_t)c.heads * a.group * 8, 8);
    const uint16_t* q0 = a.q + row_offset(a, k.first, 0, head, a.q_stride);
    const float2* stats0 = a.stats + row_number(a, k.first, 0, head);
    const uint8_t* last_q = by_q.at(a, q0, rows - 1).p;
    const uint8_t* last_stats = by_stats.at(a, stats0, rows - 1).p;
    for (int64_t j64 = (int64_t)chunk * kGroupKeys; j64 < k.keys; j64 += (int64_t)chunks * kGroupKeys) {
        const int base = (int)j64 + (wave & 3) * kBlockTokens;
        // the first rows whose tokens see the group's first key
        const int all_from = (a.causal ? max(0, (int)j64 - past) * a.group : 0) & ~(kStepRows - 1);
        const int all_steps = (rows - all_from + kStepRows - 1) / kStepRows, before = all_steps * run / runs;
        const int from = all_from + before * kStepRows, steps = all_steps * (run + 1) / runs - before;
        // (a row's chunks keep their order from step to step, as 16 divides it)
        const int lane_row = 8 * wave + (lane >> 4), ch0 = 16 * ((lane ^ lane_row) & 15), ch1 = 16 * ((lane ^ lane_row ^ 4) & 15);
        Walk r0 = by_q.at(a, q0, from + lane_row), r1 = by_q.at(a, q0, from + lane_row + 4);
        Walk rs = by_stats.at(a, stats0, from + 32 * half + q);
        r0.p += ch0;
        r1.p += ch1;
        // the rows of step `step` into a stage, 16 lanes a row (behind the last row: that one)
        auto copy = [&](int step, uint8_t* stage) {
            const uint8_t *p0 = r0.p, *p1 = r1.p;
            if (from + (step + 1) * kStepRows > rows) {
                if (r0.row >= rows) p0 = last_q + ch0;
                if (r1.row >= rows) p1 = last_q + ch1;
            }
            __builtin_amdgcn_global_load_lds((global_ptr_t)p0, (lds_ptr_t)(stage + 8 * wave * 256), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((global_ptr_t)p1, (lds_ptr_t)(stage + (8 * wave + 4) * 256), 16, 0, 0);
            by_q.advance(r0);
            by_q.advance(r1);
        };
        auto stats = [&](int step) {
            const uint8_t* p = rs.p;
            if (from + (step + 1) * kStepRows > rows && rs.row >= rows) p = last_stats;
            by_stats.advance(rs);
            return *reinterpret_cast<const float2*>(p);
        };
        int off[8];  // of a lane's operands in a stage
#pragma unroll
        for (int i = 0; i < 8; i++) off[i] = (32 * half + q) * 256 + ((8 * (i >> 2) + 4 * h + (i & 3)) ^ (q & 15)) * 16;
        __syncthreads();  // the stages are free
        copy(0, st0);
        if (steps > 1) copy(1, st1);
        float2 next = stats(0);
        KExact keys;
        float sum[16];
        {
            const int i = min(base / kBlockTokens, last);
            const BlockAt p = block_at(c, page_of(c, s, i), head, i);
            const uint8_t* kb = c.kc + p.at * kBlockBytes + 2 * h * 512 + operand_key(q) * 16;
            uint4 codes[4];
#pragma unroll
            for (int e = 0; e < 4; e++) codes[e] = *reinterpret_cast<const uint4*>(kb + (4 * (e >> 1) + (e & 1)) * 512);
            keys = exact_keys(codes, c.ks[p.at]);
        }
#pragma unroll
        for (int e = 0; e < 16; e++) sum[e] = 0.f;
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        auto one = [&](int step, const uint8_t* cur, uint8_t* far) {
            const float2 ml = next;
            if (step + 1 < steps) next = stats(step + 1);
            if (step + 2 < steps) copy(step + 2, far);
            const int row0 = from + step * kStepRows + 32 * half;
            // keys that the first and the last row see
            const int min_end = a.causal ? past + token_of(a, min(row0, rows - 1)) + 1 : k.keys;
            const int max_end = a.causal ? past + token_of(a, min(row0 + 31, rows - 1)) + 1 : k.keys;
            if (row0 < rows && max_end > base) {
                uint4 qr[8];
#pragma unroll
                for (int i = 0; i < 8; i++) qr[i] = *reinterpret_cast<const uint4*>(cur + off[i]);
                v16f x = scores(keys, qr);
                float2 mb = ml;
                if (row0 + 32 > rows || base + kBlockTokens > min_end) {
                    const int end = row0 + q >= rows ? 0 : a.causal ? past + token_of(a, row0 + q) + 1 : k.keys;
                    const int seen = end - base - 16 * h;
#pragma unroll
                    for (int e = 0; e < 16; e++) x[e] = e < seen ? x[e] : -__builtin_inff();
                    if (__any(ml.y != ml.y)) {  // a masked key's p is 0, and 0 * NaN would reach it
                        if (ml.y != ml.y) {
#pragma unroll
                            for (int e = 0; e < 16; e++) sum[e] = e < seen ? __builtin_nanf("") : sum[e];
                            mb = make_float2(0.f, 0.f);
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], a.scale, -mb.x));
                    sum[e] = __builtin_fmaf(p, mb.y, sum[e]);
                }
            }
            // the next step's rows landed: what this step copies may still be on its way
            if (step + 2 < steps)
                __builtin_amdgcn_s_waitcnt(kTwoInFlight);
            else
                __builtin_amdgcn_s_waitcnt(0);
            // (a fence, as __syncthreads has, would wait for those too)
            __asm__ volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            __asm__ volatile("" ::: "memory");
        };
        for (int step = 0; step < steps; step += 3) {
            one(step, st0, st2);
            if (step + 1 < steps) one(step + 1, st1, st0);
            if (step + 2 < steps) one(step + 2, st2, st1);
        }
        // the sums of the 32 rows' lanes: each exchange leaves a lane half of its keys, in the
        // end key 16 h + q / 2
#pragma unroll
        for (int n = 8; n > 0; n /= 2) {
            const bool up = q & (2 * n);
#pragma unroll
            for (int e = 0; e < n; e++) {
                const float away = up ? sum[e] : sum[e + n], mine = up ? sum[e + n] : sum[e];
                sum[e] = mine + __shfl_xor(away, 2 * n);
            }
        }
        float total = sum[0] + __shfl_xor(sum[0], 1);
        const int mine = (wave & 3) * kBlockTokens + 16 * h + (q >> 1), j = base + 16 * h + (q >> 1);
        if (half) s_sum[mine] = total;
        __syncthreads();
        if (half || (q & 1) || j >= k.keys) continue;
        total += s_sum[mine];
        if (runs > 1) {
            w.partial[((int64_t)run * c.seqs * c.heads + (int64_t)s * c.heads + head) * w.partial_stride + j] = total;
            continue;
        }
        const int64_t at = weights_at(c, s, head, j);
        if (at >= 0) w.after[at] = sum_with(w, at, j < past, total);
    }
}

// The runs' sums of a key, one after another.
__global__ __launch_bounds__(kThreads) void cache_weigh_runs_kernel(CacheWeighArgs w, int chunks, int runs) {
    const CacheAttendArgs& a = w.a;
    const Placed place(a.c, chunks);
    if (place.s < 0) return;
    const Keys k(a, place.s);
    const int j = place.chunk * kThreads + threadIdx.x;
    if (k.n == 0 || j >= k.keys) return;
    const int64_t items = (int64_t)a.c.seqs * a.c.heads;
    const float* p = w.partial + ((int64_t)place.s * a.c.heads + place.head) * w.partial_stride + j;
    float sum = 0.f;
#pragma unroll 8
    for (int r = 0; r < runs; r++) sum += p[r * items * w.partial_stride];
    const int64_t at = weights_at(a.c, place.s, place.head, j);
    if (at >= 0) w.after[at] = sum_with(w, at, j < k.keys - k.n, sum);
}

// Scores are kept up to this many bytes; beyond, they are computed twice.
constexpr int64_t kMostScores = (int64_t)1 << 30;

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

// Workgroups of an item: one for each `keys` keys, but no more than 2^22 of all items where
// those are fewer, and one of each otherwise (they are below 2^24).
int chunks_of(const CacheAttendArgs& a, int64_t max_kv, int keys) {
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 22) / ((int64_t)a.c.seqs * a.c.heads));
    return (int)std::min<int64_t>(most, (max_kv + keys - 1) / keys);
}

// Into how many runs the rows are cut, where few keys and heads leave the chip idle: two
// workgroups a CU, as far as the caller's bounds say, each of two steps or more.  (8000 rows x
// 1000 keys of one head: 99 us by 8 workgroups, 14 in runs, 6 of them for their sums.)
int runs_of(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    const int64_t groups = (int64_t)a.c.seqs * a.c.heads * ((max_kv + kKeyWaves * kBlockTokens - 1) / (kKeyWaves * kBlockTokens));
    const int64_t steps = (max_q * a.group + kStepRows - 1) / kStepRows;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / groups, steps / 2), 64));
}

// Chooses the kind, and where what the kernels leave for the sums lies; returns the bytes.
size_t lay_out(CacheWeighArgs& w, int64_t max_q, int64_t max_kv) {
    CacheAttendArgs& a = w.a;
    const int64_t rows = (int64_t)a.c.tokens * a.c.heads * a.group;
    a.score_stride = (max_kv + 31) / 32 * 32;
    a.kind = kWeighStats;
    if (cache_attend_keeps_scores(a, max_q, max_kv) && rows <= kMostScores / 4 / a.score_stride) a.kind = kWeigh;
    const size_t parts = up16(cache_attend_workspace(a, max_q, max_kv));
    const size_t stats = up16((size_t)rows * sizeof(float2));
    a.stats = reinterpret_cast<float2*>(a.workspace + parts);
    a.scores = w.partial = reinterpret_cast<float*>(a.workspace + parts + stats);
    w.partial_stride = a.score_stride;
    w.runs = a.kind == kWeigh ? 1 : runs_of(a, max_q, max_kv);
    const int64_t more = a.kind == kWeigh ? rows : w.runs > 1 ? (int64_t)w.runs * a.c.seqs * a.c.heads : 0;
    return parts + stats + (size_t)more * (size_t)a.score_stride * 4;
}

}  // namespace

size_t cache_weigh_workspace(CacheWeighArgs w, int64_t max_q, int64_t max_kv) { return lay_out(w, max_q, max_kv); }

hipError_t launch_cache_weigh(CacheWeighArgs w, int64_t max_q, int64_t max_kv, hipStream_t stream) {
    CacheAttendArgs& a = w.a;
    a.most_keys = (int)max_kv;
    lay_out(w, max_q, max_kv);
    if (hipError_t e = launch_cache_attend(a, max_q, max_kv, stream)) return e;
    if (a.kind == kWeigh) {
        const int chunks = chunks_of(a, max_kv, 4 * kThreads);
        cache_weigh_scores_kernel<<<placed_grid(a.c, chunks, kThreads), kThreads, 0, stream>>>(w, chunks);
        return hipGetLastError();
    }
    const int chunks = chunks_of(a, max_kv, kKeyWaves * kBlockTokens);
    const dim3 grid = placed_grid(a.c, (int64_t)chunks * w.runs, 64 * kWaves);
    if (kStepRows % a.group == 0)
        cache_weigh_rows_kernel<true><<<grid, 64 * kWaves, 0, stream>>>(w, chunks, w.runs);
    else
        cache_weigh_rows_kernel<false><<<grid, 64 * kWaves, 0, stream>>>(w, chunks, w.runs);
    if (hipError_t e = hipGetLastError()) return e;
    if (w.runs > 1) {
        const int sums = (int)((max_kv + kThreads - 1) / kThreads);
        cache_weigh_runs_kernel<<<placed_grid(a.c, sums, kThreads), kThreads, 0, stream>>>(w, sums, w.runs);
    }
    return hipGetLastError();
}

}  // namespace mxattn
