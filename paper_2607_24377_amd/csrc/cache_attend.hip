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
    } else {
        const int s = __builtin_amdgcn_readfirstlane(owner_of(c, blockIdx.x, a.group, kRows, 1));
        if (s < 0) return;
        const TokenRange r = token_range(c, s);
        it = {s, (int)blockIdx.y, (int)(blockIdx.x - ((int64_t)r.first * a.group / kRows + s)) * kRows, 0, 1, 1, 0};
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
            load_block(x, c, block_at(c, page_of(c, it.s, b), it.head, b), q, h);
            int page = page_of(c, it.s, min(b + kWaves, b1 - 1));
            while (true) {
                const bool more = b + kWaves < b1;
                if (more) {
                    load_block(y, c, block_at(c, page, it.head, b + kWaves), q, h);
                    page = page_of(c, it.s, min(b + 2 * kWaves, b1 - 1));
                }
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
        if (it.x0 == 0 && !whole) info = {it.last, it.s, it.head, it.row0};
        first = false;
    }
    if (kDivided && tid == 0) parts.info[blockIdx.x] = info;
}

// Two workgroups per CU are resident (registers).
constexpr int kWorkgroups = 512;
// Keys up to which an item is one workgroup's.
constexpr int64_t kUndivided = 1024;

bool divided(int64_t max_kv) { return max_kv > kUndivided; }

// Query rows of a sequence and head from which tiles of 128 rows pay.
constexpr int64_t kTileRows = 64;
bool tiled(const CacheAttendArgs& a, int64_t max_q) { return max_q * a.group > kTileRows; }

}  // namespace

size_t cache_attend_workspace(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv) {
    return tiled(a, max_q) ? cache_attend_tiles_workspace() : divided(max_kv) ? parts_bytes<kRows>(kWorkgroups) : 0;
}

hipError_t launch_cache_attend(const CacheAttendArgs& a, int64_t max_q, int64_t max_kv, hipStream_t stream) {
    if (tiled(a, max_q)) return launch_cache_attend_tiles(a, stream);
    if (divided(max_kv)) {
        cache_attend_kernel<true><<<kWorkgroups, kThreads, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
        return launch_cache_attend_join<kRows>(a, kWorkgroups, max_q * a.group < kRows ? max_q * a.group : kRows, stream);
    } else {
        const dim3 grid((unsigned)((int64_t)a.c.tokens * a.group / kRows + a.c.seqs), (unsigned)a.c.heads);
        cache_attend_kernel<false><<<grid, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace mxattn
