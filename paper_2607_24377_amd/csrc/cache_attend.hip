// cache_attend.hip -- attention over the 8-bit paged cache where a sequence has
// few query rows per KV head (a token or some drafts): bound by reading the keys.
//
// A workgroup takes one tile of 32 rows (cache_attend.h) and a run of its keys; its
// four waves hold the same rows and take every fourth block of 32 keys, straight
// from memory into the operands' registers, the next block in flight while one is
// worked on.  No barrier until the run's end, where the waves' m, l and O~ meet in
// LDS.
#include "cache_attend.h"

namespace mxattn {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 32;
constexpr int kRowFloats = 132;  // a row of O~ in LDS: 128 channels, padded off the banks of its neighbours

// Four channels of a row, finished: O~ / l as bf16; a row without keys is 0.
__device__ __forceinline__ uint2 finished(float4 o, float l, bool bad) {
    const float inv = bad ? __builtin_nanf("") : l == 0.f ? 0.f : 1.0f / l;
    const f32x2 x = {o.x * inv, o.y * inv}, y = {o.z * inv, o.w * inv};
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2)),
                      __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2)));
}

__device__ __forceinline__ void add_scaled(float4& o, const float4& x, float f) {
    o.x = __builtin_fmaf(x.x, f, o.x);
    o.y = __builtin_fmaf(x.y, f, o.y);
    o.z = __builtin_fmaf(x.z, f, o.z);
    o.w = __builtin_fmaf(x.w, f, o.w);
}

// kDivided: shares of the work by workgroup (cache_attend.h); else one workgroup per
// item, numbered as the workgroups of the append: sequence s has tiles
// q_start[s] * group / 32 + s onwards.
template <bool kDivided>
__global__ __launch_bounds__(kThreads, 2) void cache_attend_kernel(CacheAttendArgs a) {
    __shared__ __align__(16) float s_o[kWaves][kRows][kRowFloats];
    __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, q = lane & 31, h = lane >> 5;
    Share sh{};
    Item it{};
    PartInfo info{};
    if constexpr (kDivided) {
        sh = find_share<kRows, false, kThreads>(a, blockIdx.x, gridDim.x);
        sh = {uniform64(sh.at), uniform64(sh.end), uniform64(sh.offset), __builtin_amdgcn_readfirstlane(sh.s)};
    } else {
        __shared__ int s_seq;
        if (tid == 0) s_seq = -1;
        __syncthreads();
        for (int s = tid; s < c.seqs; s += kThreads) {
            const TokenRange r = token_range(c, s);
            const int64_t base = (int64_t)r.first * a.group / kRows + s, next = (int64_t)r.last * a.group / kRows + s + 1;
            if (base <= blockIdx.x && blockIdx.x < next) s_seq = s;
        }
        __syncthreads();
        const int s = __builtin_amdgcn_readfirstlane(s_seq);
        if (s < 0) return;
        const TokenRange r = token_range(c, s);
        it = {s, (int)blockIdx.y, (int)(blockIdx.x - ((int64_t)r.first * a.group / kRows + s)) * kRows, 0, 1, 1};
        if (it.row0 >= (r.last - r.first) * a.group) return;
        sh.end = 1;
    }
    const Parts<kRows> parts(a.workspace, gridDim.x);
    bool first = true;
    while (sh.at < sh.end) {
        if constexpr (kDivided)
            it = next_item<kRows, false>(a, sh);
        else
            sh.at = sh.end;
        const TileRows t = tile_rows<kRows>(a, it.s, it.row0);
        const int blocks = (t.max_end + kBlockTokens - 1) / kBlockTokens;
        const int b0 = (int)(it.x0 * blocks / it.w), b1 = (int)(it.x1 * blocks / it.w);
        const int row = it.row0 + min(q, t.rows - 1);
        const int end = a.causal ? t.keys - t.n + row / a.group + 1 : t.keys;
        const QOperand qo = load_q(a.q + row_offset(a, t.first, row, it.head, a.q_stride), h, a.scale, q < t.rows);
        State st;
        st.clear();
        int b = b0 + wave;
        if (b < b1) {
            Block x, y;
            load_block(x, c, block_at(c, it.s, it.head, b), q, h);
            while (true) {
                const bool more = b + kWaves < b1;
                if (more) load_block(y, c, block_at(c, it.s, it.head, b + kWaves), q, h);
                attend_block(st, x, qo, b * kBlockTokens, end, t.keys, (b + 1) * kBlockTokens > t.min_end, h);
                if (!more) break;
                x = y;
                b += kWaves;
            }
        }
        const float l = st.l + other_half(st.l);
        if (!first) __syncthreads();  // the rows of the item before are read
        if (h == 0) {
            s_m[wave][q] = st.m;
            s_l[wave][q] = l;
        }
        if (q < t.rows) {
#pragma unroll
            for (int n = 0; n < 4; n++)
#pragma unroll
                for (int g = 0; g < 4; g++)
                    *reinterpret_cast<float4*>(&s_o[wave][q][32 * n + 8 * g + 4 * h]) =
                        make_float4(st.O[n][4 * g], st.O[n][4 * g + 1], st.O[n][4 * g + 2], st.O[n][4 * g + 3]);
        }
        __syncthreads();
        const bool whole = it.whole();
        const int slot = 2 * blockIdx.x + (it.x0 == 0);
        for (int e = tid; e < t.rows * 32; e += kThreads) {
            const int r = e >> 5, ch = 4 * (e & 31);
            float m = s_m[0][r];
#pragma unroll
            for (int w = 1; w < kWaves; w++) m = max2(m, s_m[w][r]);
            float sum = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWaves; w++) {
                const float f = __builtin_amdgcn_exp2f(s_m[w][r] - m);
                sum = __builtin_fmaf(s_l[w][r], f, sum);
                add_scaled(o, *reinterpret_cast<const float4*>(&s_o[w][r][ch]), f);
            }
            if (whole) {
                *reinterpret_cast<uint2*>(a.out + row_offset(a, t.first, it.row0 + r, it.head, a.out_stride) + ch) =
                    finished(o, sum, t.bad);
            } else {
                *reinterpret_cast<float4*>(parts.o + ((int64_t)slot * kRows + r) * kHeadDim + ch) = o;
                if (ch == 0) parts.ml[slot * kRows + r] = make_float2(m, sum);
            }
        }
        if (it.x0 > 0) {
            info.head = 1;
            info.ends = it.x1 == it.w;
        } else if (!whole) {
            info.tail = 1;
            info.s = it.s;
            info.kv_head = it.head;
            info.row0 = it.row0;
        }
        first = false;
    }
    if (kDivided && tid == 0) parts.info[blockIdx.x] = info;
}

// Joins the parts of the item that began in workgroup blockIdx.x and went on
// behind it, in the order of its keys: lane group g of 8 takes every eighth part,
// then the eight meet in LDS.
template <int kRows>
__global__ __launch_bounds__(kThreads) void cache_attend_join_kernel(CacheAttendArgs a) {
    __shared__ float4 s_o[8][32];
    __shared__ float s_m[8], s_l[8];
    __shared__ int s_count;
    __shared__ int s_slot[1024];
    const Parts<kRows> parts(a.workspace, gridDim.x);
    const int i = blockIdx.x, tid = threadIdx.x;
    const PartInfo info = parts.info[i];
    if (!info.tail) return;
    // the parts: this workgroup's tail, then the heads of those behind it up to the one where it ends
    if (tid == 0) {
        int n = 1;
        s_slot[0] = 2 * i + 1;
        for (int k = i + 1; k < (int)gridDim.x; k++) {
            const PartInfo p = parts.info[k];
            if (!p.head) continue;  // no share of its own
            s_slot[n++] = 2 * k;
            if (p.ends) break;
        }
        s_count = n;
    }
    __syncthreads();
    const int count = s_count;
    const TileRows t = tile_rows<kRows>(a, info.s, info.row0);
    const int g = tid >> 5, ch = 4 * (tid & 31);
    for (int r = 0; r < t.rows; r++) {
        float m = kNoMax, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p = g; p < count; p += 8) m = max2(m, parts.ml[s_slot[p] * kRows + r].x);
        for (int p = g; p < count; p += 8) {
            const float2 ml = parts.ml[s_slot[p] * kRows + r];
            const float f = __builtin_amdgcn_exp2f(ml.x - m);
            l = __builtin_fmaf(ml.y, f, l);
            add_scaled(o, *reinterpret_cast<const float4*>(parts.o + ((int64_t)s_slot[p] * kRows + r) * kHeadDim + ch), f);
        }
        s_o[g][tid & 31] = o;
        if (ch == 0) {
            s_m[g] = m;
            s_l[g] = l;
        }
        __syncthreads();
        if (g == 0) {
            m = s_m[0];
            for (int k = 1; k < 8; k++) m = max2(m, s_m[k]);
            l = 0.f;
            o = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = 0; k < 8; k++) {
                const float f = __builtin_amdgcn_exp2f(s_m[k] - m);
                l = __builtin_fmaf(s_l[k], f, l);
                add_scaled(o, s_o[k][tid & 31], f);
            }
            *reinterpret_cast<uint2*>(a.out + row_offset(a, t.first, info.row0 + r, info.kv_head, a.out_stride) + ch) =
                finished(o, l, t.bad);
        }
        __syncthreads();
    }
}

// Two workgroups per CU are resident (registers).
constexpr int kWorkgroups = 512;
// Keys up to which an item is one workgroup's.
constexpr int64_t kUndivided = 1024;

bool divided(int64_t max_kv) { return max_kv > kUndivided; }

}  // namespace

size_t cache_attend_workspace(int64_t max_kv) {
    return divided(max_kv) ? (size_t)kWorkgroups * (2 * kRows * 520 + sizeof(PartInfo)) : 0;
}

hipError_t launch_cache_attend(const CacheAttendArgs& a, int64_t max_kv, hipStream_t stream) {
    if (divided(max_kv)) {
        cache_attend_kernel<true><<<kWorkgroups, kThreads, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
        cache_attend_join_kernel<kRows><<<kWorkgroups, kThreads, 0, stream>>>(a);
    } else {
        const dim3 grid((unsigned)((int64_t)a.c.tokens * a.group / kRows + a.c.seqs), (unsigned)a.c.heads);
        cache_attend_kernel<false><<<grid, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace mxattn
