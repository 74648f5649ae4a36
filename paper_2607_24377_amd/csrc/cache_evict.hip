// cache_evict.hip -- which tokens of a cache stay, and moving those that stay together.
//
// Selection: of a sequence's L keys of one KV head the first `sinks`, the last `recent`
// and, of those between, the heaviest, `budget` in all.  A workgroup finds the weight of
// the last one that stays digit by digit (11, 11 and 10 bits of the number in an order of
// unsigned integers, a histogram in LDS for each), then writes the kept positions in
// order: each wave starts where the stretches before its own end.  What shares the digits
// found so far is put aside in LDS as soon as it fits, so that the weights are read three
// times (histogram, putting aside, writing).
//
// Compaction: position base + i becomes what was at kept[i].  A block of 32 kept tokens
// takes the largest scale byte of the blocks that they come from, so that no code grows
// and no other channel has to be looked at; code * 2^(e_old - e) is rounded to nearest,
// which is exact unless it falls below 2^-6.  A wave per block of K or V; in place, the
// workgroup that has a head's keys (or values) walks its blocks in order, all loads of a
// turn before its stores: what later blocks need lies behind what was written.
#include "heads.h"

#include <algorithm>

namespace mxattn {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kDigits = 2048;
constexpr int kCopies = 8;      // of the histogram: weights share few of the first digits
constexpr int kAside = 8192;

// Weights in the order of unsigned integers; NaN below every number, -0 with +0.
__device__ __forceinline__ uint32_t ordered(float w) {
    const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.f);
    return w != w ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// The number whose order is u, -0 as +0; NaN for 0.
__device__ __forceinline__ float number_of(uint32_t u) {
    return __builtin_bit_cast(float, u >> 31 ? u & 0x7FFFFFFFu : ~u);
}

// Lanes before this one in a mask.
__device__ __forceinline__ uint32_t lanes_before(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// The weights of a head's stretch j0 .. j1 - 1, j0 a multiple of 256, four a lane, 1024 at a
// time: f gets the lane's first position, its four weights (of no page: NaN), and which of
// them are of the stretch and between m0 and m1 (as bits), or are of it and not between.
// (One at a time: two loads after each other for every 64.)
template <class F>
__device__ __forceinline__ void for_weights(const SelectArgs& a, int s, int head, int j0, int j1, int m0, int m1, const F& f) {
    const CacheArgs& c = a.c;
    const int lane = threadIdx.x & 63, log2 = c.bpp_log2 + 5;
    const int32_t* table = c.page_table + (int64_t)s * c.max_pages;
    constexpr int kTurns = 4;
    for (int j = j0; j < j1; j += 256 * kTurns) {
        int page[kTurns];
        f32x4u w[kTurns];
#pragma unroll
        for (int i = 0; i < kTurns; i++) page[i] = table[min(j + 256 * i + 4 * lane, j1 - 1) >> log2];
#pragma unroll
        for (int i = 0; i < kTurns; i++) {
            const int at = min(j + 256 * i + 4 * lane, (j1 - 1) & ~3);
            const bool there = (unsigned)page[i] < (unsigned)c.pages;
            w[i] = *reinterpret_cast<const f32x4u*>(
                a.weights + (((int64_t)(there ? page[i] : 0) * c.heads + head) << log2) + (at & ((1 << log2) - 1)));
            if (!there) w[i] = f32x4u{0.f, 0.f, 0.f, 0.f} * __builtin_nanf("");
        }
#pragma unroll
        for (int i = 0; i < kTurns; i++) {
            const int at = j + 256 * i, p = at + 4 * lane;
            if (at >= j1) break;
            if (at >= m0 && at + 256 <= min(m1, j1)) {
                f(p, w[i], 15u, 0u);
            } else {
                uint32_t free = 0, forced = 0;
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    if (p + k >= j1) continue;
                    if (p + k >= m0 && p + k < m1)
                        free |= 1u << k;
                    else
                        forced |= 1u << k;
                }
                f(p, w[i], free, forced);
            }
        }
    }
}

__device__ __forceinline__ uint32_t sum64(uint32_t x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += (uint32_t)__shfl_xor((int)x, d);
    return x;
}

__global__ __launch_bounds__(kSelectThreads) void cache_select_kernel(SelectArgs a) {
    __shared__ __align__(16) uint32_t s_hist[kDigits * kCopies];
    __shared__ uint32_t s_aside[kAside];
    __shared__ uint8_t s_whose[kAside];
    __shared__ uint32_t s_wave[kSelectWaves];
    __shared__ uint32_t s_found[3];  // the digit of the last one that stays, how many of it do, how many there are
    __shared__ uint32_t s_above[kSelectWaves], s_equal[kSelectWaves], s_count;
    const CacheArgs& c = a.c;
    // (head by head: the XCDs take workgroups in turn, and the heads of a sequence spread over them)
    const int s = (int)(blockIdx.x / (unsigned)c.heads), head = (int)blockIdx.x - s * c.heads, tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int len = c.kv_len[s], L = (unsigned)len > (unsigned)(c.max_pages << (c.bpp_log2 + 5)) ? 0 : len;
    const int count = min(L, a.budget);
    int32_t* kept = a.kept + ((int64_t)s * c.heads + head) * a.budget;
    if (head == 0 && tid == 0) a.counts[s] = count;
    for (int i = count + tid; i < a.budget; i += kSelectThreads) kept[i] = -1;
    if (L <= a.budget) {
        for (int i = tid; i < L; i += kSelectThreads) kept[i] = i;
        return;
    }
    const int m0 = a.sinks, m1 = L - a.recent;  // what lies between may go
    // a stretch of all positions for each wave
    const int per = (L + 256 * kSelectWaves - 1) / (256 * kSelectWaves) * 256;
    const int j0 = min(wave * per, L), j1 = min(j0 + per, L);
    if (tid < kSelectWaves) s_above[tid] = s_equal[tid] = 0;
    if (tid == 0) s_count = 0;
    // the weight of the last one that stays, `prefix` in the bits of `known`, and how many
    // of exactly that weight do
    uint32_t prefix = 0, known = 0;
    uint32_t need = (uint32_t)(a.budget - a.sinks - a.recent);  // below the number of those between
    const bool any = need > 0;
    bool aside = false;  // what shares the known digits is in s_aside, what is above them counted
    for (int pass = 0; any && pass < 3; pass++) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t mask = pass == 2 ? 1023 : 2047;
        const bool fits = pass > 0 && !aside && s_found[2] <= kAside;
        for (int i = tid; i < kDigits * kCopies / 4; i += kSelectThreads)
            reinterpret_cast<uint4*>(s_hist)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        auto add = [&](uint32_t u) { atomicAdd(&s_hist[((u >> shift) & mask) * kCopies + (lane & (kCopies - 1))], 1u); };
        if (aside) {
            const int n = (int)s_count;
            for (int i = tid; i < n; i += kSelectThreads)
                if ((s_aside[i] & known) == prefix) add(s_aside[i]);
        } else {
            uint32_t above = 0;
            for_weights(a, s, head, j0, j1, m0, m1, [&](int, const f32x4u& w, uint32_t free, uint32_t forced) {
                uint32_t u[4], mine = 0, more = forced;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    u[i] = ordered(w[i]);
                    const uint32_t d = u[i] & known;
                    if (!(free >> i & 1)) continue;
                    if (d == prefix) {
                        add(u[i]);
                        mine |= 1u << i;
                    }
                    if (d > prefix) more |= 1u << i;
                }
                if (!fits) return;
                above += (uint32_t)__popc(more);
                if (__any(mine != 0)) {  // room for the wave's at once
                    uint32_t before = 0, total = 0;
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const uint64_t b = __ballot(mine >> i & 1);
                        before += lanes_before(b);
                        total += (uint32_t)__popcll(b);
                    }
                    uint32_t at = 0;
                    if (lane == 0) at = atomicAdd(&s_count, total);
                    at = __builtin_amdgcn_readfirstlane((int)at) + before;
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        if (!(mine >> i & 1)) continue;
                        s_aside[at] = u[i];
                        s_whose[at++] = (uint8_t)wave;
                    }
                }
            });
            above = sum64(above);
            if (fits && lane == 0) s_above[wave] = above;
        }
        aside = aside || fits;
        __syncthreads();
        // thread t has digits 2 t and 2 t + 1 from the largest down
        uint32_t x = 0, y = 0;
        const uint4* pair = reinterpret_cast<const uint4*>(s_hist + (kDigits - 2 - 2 * tid) * kCopies);
#pragma unroll
        for (int k = 0; k < kCopies / 4; k++) {
            const uint4 v = pair[k], w = pair[kCopies / 4 + k];
            y += v.x + v.y + v.z + v.w;
            x += w.x + w.y + w.z + w.w;
        }
        uint32_t incl = x + y;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t v = (uint32_t)__shfl_up((int)incl, d);
            if (lane >= d) incl += v;
        }
        if (lane == 63) s_wave[wave] = incl;
        __syncthreads();
        uint32_t before = incl - x - y;
        for (int k = 0; k < wave; k++) before += s_wave[k];
        if (before < need && need <= before + x) {
            s_found[0] = (uint32_t)(kDigits - 1 - 2 * tid);
            s_found[1] = need - before;
            s_found[2] = x;
        } else if (before + x < need && need <= before + x + y) {
            s_found[0] = (uint32_t)(kDigits - 2 - 2 * tid);
            s_found[1] = need - before - x;
            s_found[2] = y;
        }
        __syncthreads();
        prefix |= s_found[0] << shift;
        need = s_found[1];
        known |= mask << shift;
    }
    // which of a lane's four stay for their weight or place, and which have the last one's weight
    const float border = number_of(prefix);
    auto look = [&](const f32x4u& w, uint32_t free, uint32_t forced, uint32_t& x, uint32_t& y) {
        x = y = 0;
        if (any) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                // (0 is NaN's place: every number is above it)
                x |= (uint32_t)(prefix ? w[i] > border : w[i] == w[i]) << i;
                y |= (uint32_t)(prefix ? w[i] == border : w[i] != w[i]) << i;
            }
        }
        x = (x & free) | forced;
        y &= free;
    };
    // how many of each wave's stretch do
    if (aside) {
        const int n = (int)s_count;
        for (int i = tid; i < n; i += kSelectThreads) {
            if (s_aside[i] > prefix) atomicAdd(&s_above[s_whose[i]], 1u);
            if (s_aside[i] == prefix) atomicAdd(&s_equal[s_whose[i]], 1u);
        }
    } else {
        uint32_t above = 0, equal = 0;
        for_weights(a, s, head, j0, j1, m0, m1, [&](int, const f32x4u& w, uint32_t free, uint32_t forced) {
            uint32_t x, y;
            look(w, free, forced, x, y);
            above += (uint32_t)__popc(x);
            equal += (uint32_t)__popc(y);
        });
        above = sum64(above);
        equal = sum64(equal);
        if (lane == 0) {
            s_above[wave] = above;
            s_equal[wave] = equal;
        }
    }
    __syncthreads();
    uint32_t at = 0, same = 0;  // those above and those equal before this place
    for (int k = 0; k < wave; k++) {
        at += s_above[k];
        same += s_equal[k];
    }
    for_weights(a, s, head, j0, j1, m0, m1, [&](int j, const f32x4u& w, uint32_t free, uint32_t forced) {
        uint32_t x, y;
        look(w, free, forced, x, y);
        uint32_t ax = at;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint64_t b = __ballot(x >> i & 1);
            ax += lanes_before(b);
            at += (uint32_t)__popcll(b);
        }
        uint32_t ay = same;
        if (__any(y != 0)) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint64_t b = __ballot(y >> i & 1);
                ay += lanes_before(b);
                same += (uint32_t)__popcll(b);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t xi = x >> i & 1, yi = y >> i & 1;
            if (xi | (yi & (uint32_t)(ay < need))) kept[ax + min(ay, need)] = j + i;
            ax += xi;
            ay += yi;
        }
    });
}

// ---------------------------------------------------------------------------

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

// Four codes times 2^shift (shift <= 0).
__device__ __forceinline__ uint32_t rescale4(uint32_t c, int shift) {
    const f32x2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
    const f32x2v b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    const int p = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(a[0], shift), __builtin_ldexpf(a[1], shift), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(b[0], shift), __builtin_ldexpf(b[1], shift), p, true);
}
// One code.
__device__ __forceinline__ uint32_t rescale1(uint32_t c, int shift) {
    const float x = __builtin_ldexpf(__builtin_amdgcn_cvt_f32_fp8((int)c, 0), shift);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xFFu;
}

constexpr uint32_t kNanCodes = 0x7F7F7F7Fu;

// Where a lane's token (slot lane & 31 of the block that is made) comes from.
struct Source {
    int64_t at;    // its cache block
    int slot;      // in it
    int64_t w;     // its weight
    bool live;     // there is such a token
    bool lost;     // but not its page or number
};

__device__ __forceinline__ Source source_of(const CompactArgs& a, int s, int head, int pos, int base, int count,
                                            const int32_t* kept) {
    const CacheArgs& c = a.c;
    const int log2 = c.bpp_log2 + 5;
    Source x{0, 0, 0, pos < base + count, true};
    if (!x.live) return x;
    const int from = pos < base ? pos : kept[pos - base];  // (what was there before stays)
    const int64_t most = (int64_t)(pos < base ? a.out_pages : c.max_pages) << log2;
    if (from < 0 || from >= most) return x;
    const int32_t* table = pos < base ? a.out_table + (int64_t)s * a.out_pages : c.page_table + (int64_t)s * c.max_pages;
    const int page = table[from >> log2];
    if ((unsigned)page >= (unsigned)c.pages) return x;
    const int64_t p = (int64_t)page * c.heads + head;
    x.at = (p << c.bpp_log2) + ((from >> 5) & ((1 << c.bpp_log2) - 1));
    x.slot = from & 31;
    x.w = (p << log2) + (from & ((1 << log2) - 1));
    x.lost = false;
    return x;
}

// Largest of 32 lanes, the same in both halves of the wave.
__device__ __forceinline__ int max32(int x) {
#pragma unroll
    for (int d = 1; d < 32; d *= 2) x = max(x, __shfl_xor(x, d));
    return x;
}

__global__ __launch_bounds__(kThreads) void cache_compact_kernel(CompactArgs a, int runs) {
    // V: a source block in the order of channels, 17 words for every two
    __shared__ uint32_t s_rows[kWaves][64 * 17];
    const CacheArgs& c = a.c;
    const Placed place(c, 2 * runs);  // the runs of V, which take longer, then those of K
    const int s = place.s, head = place.head;
    if (s < 0) return;
    const bool values = place.chunk < runs;
    const int run = values ? place.chunk : place.chunk - runs;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int t = lane & 31, h = lane >> 5;
    const int log2 = c.bpp_log2 + 5;
    const int count = a.counts[s], base = a.base ? a.base[s] : 0;
    if (count <= 0 || count > a.width || base < 0) return;
    const int64_t end = (int64_t)base + count;
    if (end > (int64_t)a.out_pages << log2) return;
    const int d0 = base >> 5, blocks = (int)((end + 31) >> 5) - d0;
    const int turns = (blocks + kWaves - 1) / kWaves;
    const int32_t* kept = a.kept + s * a.kept_seq + head * a.kept_head;
    uint8_t* codes = values ? c.vc : c.kc;
    uint8_t* scales = values ? c.vs : c.ks;
    for (int turn = (int)((int64_t)turns * run / runs); turn < (int)((int64_t)turns * (run + 1) / runs); turn++) {
        const int d = d0 + turn * kWaves + wave;
        const bool here = turn * kWaves + wave < blocks;
        const int page = here ? a.out_table[(int64_t)s * a.out_pages + (d >> c.bpp_log2)] : -1;
        const bool write = (unsigned)page < (unsigned)c.pages;
        const int64_t to_page = (int64_t)(write ? page : 0) * c.heads + head;
        const int64_t to = (to_page << c.bpp_log2) + (d & ((1 << c.bpp_log2) - 1));
        u32x4 out[4];
        int top = 0;
        float weight = 0.f;
        bool live = false;
        if (write) {
            const Source x = source_of(a, s, head, d * 32 + t, base, count, kept);
            live = x.live;
            int e = x.live && !x.lost ? scales[x.at] : 0;
            const bool nan = x.lost || e == 255;
            if (nan) e = 0;
            top = max32(e);
            const int shift = nan ? 0 : e - top;
            const bool some = __any(shift != 0);
            if (!values) {
                if (a.weights && h == 0) weight = x.lost ? 0.f : a.weights[x.w];
#pragma unroll
                for (int p = 0; p < 4; p++) {
                    out[p] = u32x4{0, 0, 0, 0};
                    if (!x.live) continue;
                    const uint32_t n = kNanCodes;
                    out[p] = nan ? u32x4{n, n, n, n}
                                 : *reinterpret_cast<const u32x4*>(codes + x.at * kBlockBytes + (2 * p + h) * 512 + x.slot * 16);
                    if (some) {
#pragma unroll
                        for (int i = 0; i < 4; i++) out[p][i] = rescale4(out[p][i], shift);
                    }
                }
            } else {
                // a lane makes channels 2 lane and 2 lane + 1: 32 bytes each
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; i++) w[i] = 0;
                const uint32_t lost = (uint32_t)__ballot(x.live && nan);
                uint32_t left = (uint32_t)__ballot(x.live && !nan);
                uint32_t* mine = s_rows[wave] + lane * 17;
                while (left) {
                    const int first = __builtin_ctz(left);
                    const int lo = __builtin_amdgcn_readlane((int)x.at, first);
                    const int hi = __builtin_amdgcn_readlane((int)(x.at >> 32), first);
                    const int64_t at = ((int64_t)hi << 32) | (uint32_t)lo;
                    const uint32_t same = (uint32_t)__ballot(x.at == at) & left;
                    left &= ~same;
                    const u32x4* row = reinterpret_cast<const u32x4*>(codes + at * kBlockBytes + lane * 64);
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const u32x4 r = row[i];
#pragma unroll
                        for (int j = 0; j < 4; j++) mine[4 * i + j] = r[j];
                    }
#pragma unroll
                    for (int i = 0; i < 32; i++) {
                        if (!(same >> i & 1)) continue;
                        const int slot = __builtin_amdgcn_readlane(x.slot, i);
                        const int by = __builtin_amdgcn_readlane(shift, i);
#pragma unroll
                        for (int ch = 0; ch < 2; ch++) {
                            uint32_t code = (mine[8 * ch + (slot >> 2)] >> (8 * (slot & 3))) & 0xFFu;
                            if (by) code = rescale1(code, by);
                            w[8 * ch + (i >> 2)] |= code << (8 * (i & 3));
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 32; i++)
                    if (lost >> i & 1) {
                        w[i >> 2] |= 0x7Fu << (8 * (i & 3));
                        w[8 + (i >> 2)] |= 0x7Fu << (8 * (i & 3));
                    }
#pragma unroll
                for (int i = 0; i < 4; i++) out[i] = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
            }
        }
        if (a.in_place) {  // all of a turn is read before any of it is written
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
        }
        if (!write) continue;
        uint8_t* block = codes + to * kBlockBytes;
#pragma unroll
        for (int p = 0; p < 4; p++)
            *reinterpret_cast<u32x4*>(block + (values ? lane * 64 + p * 16 : (2 * p + h) * 512 + t * 16)) = out[p];
        if (lane == 0) scales[to] = (uint8_t)top;
        if (!values && a.weights && h == 0 && live && d * 32 + t >= base)
            a.weights[(to_page << log2) + ((d * 32 + t) & ((1 << log2) - 1))] = weight;
    }
}

}  // namespace

hipError_t launch_cache_select(const SelectArgs& a, hipStream_t stream) {
    cache_select_kernel<<<(unsigned)a.c.seqs * (unsigned)a.c.heads, kSelectThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_cache_compact(const CompactArgs& a, hipStream_t stream) {
    // the turns of a head divided where they need no order
    const int64_t turns = (a.width / kBlockTokens + 2 + kWaves - 1) / kWaves;
    const int64_t most = ((int64_t)1 << 22) / ((int64_t)a.c.seqs * a.c.heads);
    const int64_t runs = a.in_place ? 1 : std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(turns, most), 32767));
    cache_compact_kernel<<<placed_grid(a.c, 2 * runs), kThreads, 0, stream>>>(a, (int)runs);
    return hipGetLastError();
}

}  // namespace mxattn
