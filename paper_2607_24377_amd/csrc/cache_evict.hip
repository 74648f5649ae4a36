// cache_evict.hip -- which tokens of a cache stay, and moving those that stay together.
//
// Selection: of a sequence's L keys of one KV head the first `sinks`, the last `recent`
// and, of those between, the heaviest, `budget` in all.  The weight of the last one that
// stays is found digit by digit (11, 11 and 10 bits of the number in an order of unsigned
// integers, histograms in LDS); then the kept positions are written in order, each wave
// from where the stretches before its own end.  16 sequences of up to 4500 keys, 8 heads:
// 12.4 us, a chain of loads and barriers; one of 118800: 5, 10, 4 and 13 us (by one workgroup
// for a head 88, with one key a lane and load 254); of 1000000 even weights 78 in all.
//
// Compaction: position base + i becomes what was at kept[i].  A block of 32 kept tokens
// takes the largest scale byte of the blocks that they come from, so that no code grows
// and no other channel has to be looked at; code * 2^(e_old - e) is rounded to nearest,
// which is exact unless it falls below 2^-6.  A wave per block of K or V; in place, the
// workgroup that has a head's keys (or values) walks its blocks in order, all loads of a
// turn before its stores: what later blocks need lies behind what was written.
//
// Bound by HBM, and by the layout: V's 32 tokens of a channel are a sector, so that a kept
// token brings its whole block.  118800 keys cut to 14850 at random, 8 heads: 213 MB
// fetched (15 MB kept of each of K and V) and 31 written, 39 us, 6.1 TB/s; 16 sequences of up to
// 4500 cut to 2048: 29 us.  In place a head's turns follow one another, each a chain of loads
// (kept, table, scale, V's source blocks) and a barrier: 4 accepted drafts of 16 sequences 10 us,
// but those 16 sequences 117, and the 118800 keys 1237.
#include "heads.h"

#include <algorithm>

namespace mxattn {
namespace {

constexpr int kDigits = 2048;

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

// A wave's stretch j0 .. j1 - 1 of a head's weights, j0 a multiple of 256; those from m0 to
// m1 - 1 may go.  each(f): f gets the lane's first position of four, their weights (of no
// page: NaN), and which of them are of the stretch and may go (as bits), or may not.
struct Stretch {
    static constexpr int kTurns = 4;  // 1024 positions in flight, and kept if there are no more
    const SelectArgs& a;
    int s, head, j0, j1, m0, m1;
    f32x4u w[kTurns];
    __device__ __forceinline__ Stretch(const SelectArgs& a_, int s_, int head_, int j0_, int j1_, int m0_, int m1_)
        : a(a_), s(s_), head(head_), j0(j0_), j1(j1_), m0(m0_), m1(m1_) {
        if (j0 < j1) load(j0);
    }
    __device__ __forceinline__ void load(int j) {
        const CacheArgs& c = a.c;
        const int lane = threadIdx.x & 63, log2 = c.bpp_log2 + 5;
        const int32_t* table = c.page_table + (int64_t)s * c.max_pages;
        int page[kTurns];
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
    }
    template <class F>
    __device__ __forceinline__ void each(const F& f) {
        for (int j = j0; j < j1; j += 256 * kTurns) {
            if (j1 - j0 > 256 * kTurns) load(j);
#pragma unroll
            for (int i = 0; i < kTurns; i++) {
                const int at = j + 256 * i, p = at + 4 * (threadIdx.x & 63);
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
};

__device__ __forceinline__ uint32_t sum64(uint32_t x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += (uint32_t)__shfl_xor((int)x, d);
    return x;
}

// The search: `prefix` in the bits of `known` is what the weight of the last one that stays
// begins with, and `need` of those that begin so stay.
struct Search {
    uint32_t prefix, known, need;
    // The digits of the three passes.
    static __device__ __forceinline__ int shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
    static __device__ __forceinline__ uint32_t mask(int pass) { return pass == 2 ? 1023 : 2047; }
};

// Histograms of a workgroup of kThreads threads, kCopies of each (weights share few of the first digits).
template <int kThreads, int kCopies>
struct Histogram {
    uint32_t bins[kDigits * kCopies];
    uint32_t wave[kThreads / 64], found[3];
    __device__ __forceinline__ void clear() {
        for (int i = threadIdx.x; i < kDigits * kCopies / 4; i += kThreads)
            reinterpret_cast<uint4*>(bins)[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void add(uint32_t u, int pass) {
        atomicAdd(&bins[((u >> Search::shift(pass)) & Search::mask(pass)) * kCopies + (threadIdx.x & (kCopies - 1))], 1u);
    }
    __device__ __forceinline__ uint32_t total(int digit) const {
        uint32_t n = 0;
#pragma unroll
        for (int k = 0; k < kCopies; k += 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(bins + digit * kCopies + k);
            n += v.x + v.y + v.z + v.w;
        }
        return n;
    }
    // Writes the counts (of no more than 16 bits) to a row of kDigits.
    __device__ __forceinline__ void store(uint16_t* row) const {
        static_assert(kThreads * 8 == kDigits, "eight digits a thread");
        uint32_t n[8];
#pragma unroll
        for (int i = 0; i < 8; i++) n[i] = total(8 * (int)threadIdx.x + i);
        reinterpret_cast<uint4*>(row)[threadIdx.x] =
            make_uint4(n[0] | n[1] << 16, n[2] | n[3] << 16, n[4] | n[5] << 16, n[6] | n[7] << 16);
    }
    // The digit of the last one that stays; n[i]: the number of digit kDigits - 1 - kEach tid - i.
    // Returns how many have it.  Barriers before and after.
    static constexpr int kEach = kDigits / kThreads;
    __device__ __forceinline__ uint32_t find(Search& x, int pass, const uint32_t (&n)[kEach]) {
        const int tid = threadIdx.x, lane = tid & 63;
        uint32_t sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; i++) sum += n[i];
        uint32_t incl = sum;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t v = (uint32_t)__shfl_up((int)incl, d);
            if (lane >= d) incl += v;
        }
        if (lane == 63) wave[tid >> 6] = incl;
        __syncthreads();
        uint32_t before = incl - sum;
        for (int k = 0; k < (tid >> 6); k++) before += wave[k];
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            if (before < x.need && x.need <= before + n[i]) {
                found[0] = (uint32_t)(kDigits - 1 - kEach * tid - i);
                found[1] = x.need - before;
                found[2] = n[i];
            }
            before += n[i];
        }
        __syncthreads();
        x.prefix |= found[0] << Search::shift(pass);
        x.known |= Search::mask(pass) << Search::shift(pass);
        x.need = found[1];
        return found[2];
    }
    __device__ __forceinline__ uint32_t find(Search& x, int pass) {
        uint32_t n[kEach];
#pragma unroll
        for (int i = 0; i < kEach; i++) n[i] = total(kDigits - 1 - kEach * (int)threadIdx.x - i);
        return find(x, pass, n);
    }
};

// What a wave puts aside: the weights (ordered) among a lane's four that begin with the
// prefix, from place `at` of all on; room for the wave's is taken at once.
template <class Store>
__device__ __forceinline__ void put_aside(uint32_t mine, const uint32_t (&u)[4], uint32_t* count, const Store& store) {
    if (!__any(mine != 0)) return;
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint64_t b = __ballot(mine >> i & 1);
        before += lanes_before(b);
        total += (uint32_t)__popcll(b);
    }
    uint32_t at = 0;
    if ((threadIdx.x & 63) == 0) at = atomicAdd(count, total);
    at = __builtin_amdgcn_readfirstlane((int)at) + before;
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (mine >> i & 1) store(at++, u[i]);
}

// Of a lane's four, which begin with x's prefix, and which are above all that do.
__device__ __forceinline__ void sort_out(const Search& x, const f32x4u& w, uint32_t free, uint32_t (&u)[4], uint32_t& mine,
                                         uint32_t& more) {
    mine = more = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        u[i] = ordered(w[i]);
        mine |= (uint32_t)((u[i] & x.known) == x.prefix) << i;
        more |= (uint32_t)((u[i] & x.known) > x.prefix) << i;
    }
    mine &= free;
    more &= free;
}

// Of a lane's four, which stay for their weight or place, and which have the last one's
// weight, when the search has ended (`any`: there was one).
__device__ __forceinline__ void look(const Search& x, bool any, const f32x4u& w, uint32_t free, uint32_t forced, uint32_t& above,
                                     uint32_t& equal) {
    above = equal = 0;
    if (any) {
        const float border = number_of(x.prefix);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            // (0 is NaN's place: every number is above it)
            above |= (uint32_t)(x.prefix ? w[i] > border : w[i] == w[i]) << i;
            equal |= (uint32_t)(x.prefix ? w[i] == border : w[i] != w[i]) << i;
        }
    }
    above = (above & free) | forced;
    equal &= free;
}

// Writes what of a stretch stays; at, same: those above and those equal before it.
__device__ __forceinline__ void write_kept(Stretch& st, const Search& x, bool any, uint32_t at, uint32_t same, int32_t* kept) {
    st.each([&](int j, const f32x4u& w, uint32_t free, uint32_t forced) {
        uint32_t above, equal;
        look(x, any, w, free, forced, above, equal);
        uint32_t ax = at;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint64_t b = __ballot(above >> i & 1);
            ax += lanes_before(b);
            at += (uint32_t)__popcll(b);
        }
        uint32_t ay = same;
        if (__any(equal != 0)) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint64_t b = __ballot(equal >> i & 1);
                ay += lanes_before(b);
                same += (uint32_t)__popcll(b);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t xi = above >> i & 1, yi = equal >> i & 1;
            if (xi | (yi & (uint32_t)(ay < x.need))) kept[ax + min(ay, x.need)] = j + i;
            ax += xi;
            ay += yi;
        }
    });
}

// A sequence's head as the kernels see it.
struct Cutting {
    int s, head, L, count, m0, m1;  // keys, those that stay; those from m0 to m1 - 1 may go
    uint32_t need;                  // of them stay
    int32_t* kept;
    __device__ __forceinline__ Cutting(const SelectArgs& a, int s_, int head_) : s(s_), head(head_) {
        const int len = a.c.kv_len[s];
        L = (unsigned)len > (unsigned)(a.c.max_pages << (a.c.bpp_log2 + 5)) ? 0 : len;
        count = min(L, a.budget);
        m0 = a.sinks;
        m1 = L - a.recent;
        need = (uint32_t)(a.budget - a.sinks - a.recent);
        kept = a.kept + ((int64_t)s * a.c.heads + head) * a.budget;
    }
    __device__ __forceinline__ bool whole() const { return L == count; }
};

// A workgroup for a head, which reads its keys once if its registers hold them (16 a thread),
// else in every pass.
constexpr int kOneMost = 16 * 1024;

template <int kOneThreads>
__global__ __launch_bounds__(kOneThreads) void cache_select_kernel(SelectArgs a) {
    constexpr int kWavesHere = kOneThreads / 64;
    __shared__ __align__(16) Histogram<kOneThreads, 4> hist;
    __shared__ uint32_t s_above[kWavesHere], s_equal[kWavesHere];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const Cutting x(a, (int)(blockIdx.x / (unsigned)a.c.heads), (int)(blockIdx.x % (unsigned)a.c.heads));
    if (x.head == 0 && tid == 0) a.counts[x.s] = x.count;
    for (int i = x.count + tid; i < a.budget; i += kOneThreads) x.kept[i] = -1;
    if (x.whole()) {
        for (int i = tid; i < x.L; i += kOneThreads) x.kept[i] = i;
        return;
    }
    const int per = (x.L + 256 * kWavesHere - 1) / (256 * kWavesHere) * 256;
    const int j0 = min(wave * per, x.L), j1 = min(j0 + per, x.L);
    Stretch st(a, x.s, x.head, j0, j1, x.m0, x.m1);
    Search search{0, 0, x.need};
    const bool any = x.need > 0;
    for (int pass = 0; any && pass < 3; pass++) {
        hist.clear();
        __syncthreads();
        st.each([&](int, const f32x4u& w, uint32_t free, uint32_t) {
            uint32_t u[4], mine, more;
            sort_out(search, w, free, u, mine, more);
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (mine >> i & 1) hist.add(u[i], pass);
        });
        __syncthreads();
        hist.find(search, pass);
    }
    uint32_t above = 0, equal = 0;
    st.each([&](int, const f32x4u& w, uint32_t free, uint32_t forced) {
        uint32_t p, q;
        look(search, any, w, free, forced, p, q);
        above += (uint32_t)__popc(p);
        equal += (uint32_t)__popc(q);
    });
    above = sum64(above);
    equal = sum64(equal);
    if (lane == 0) {
        s_above[wave] = above;
        s_equal[wave] = equal;
    }
    __syncthreads();
    uint32_t at = 0, same = 0;
    for (int k = 0; k < wave; k++) {
        at += s_above[k];
        same += s_equal[k];
    }
    write_kept(st, search, any, at, same, x.kept);
}

// More keys: a workgroup for every chunk of a head's, in four launches.  The first digit
// of all (a histogram of each chunk, added up by everyone who needs it); what begins with
// it put aside, in one list for a head in any order; the rest of the search, by every
// workgroup for itself over that list, which also says what the chunks before keep.
// Where too many begin with it to be listed, the other digits go the first one's way: the
// second in the list's place, the third in the launch that has nothing to do otherwise.
constexpr int kManyThreads = 256;
constexpr int kListMost = 4096;  // (118800 keys, 2000 on the list: 28 us for 32 without; 14000: 38 and 32)

// A head's part of the workspace.
struct Lists {
    uint16_t* digits;  // [chunks, kDigits]: the first, or the third
    uint2* list;       // [kListMost]: weight (ordered), chunk
    uint16_t* second;  // [chunks, kDigits], in the list's place
    uint32_t* above;   // [chunks]: those above all that begin so, or kept for their place
    // entries of the list, the first digit, how many of it stay, how many have it; the first two digits, how many of them stay
    uint32_t* header;
    static constexpr int kHeader = 32;
    static __host__ __device__ size_t list_bytes(int chunks) {
        const size_t second = (size_t)chunks * kDigits * 2;
        return second > kListMost * 8 ? second : kListMost * 8;
    }
    static size_t bytes(int chunks) {
        return ((size_t)chunks * (kDigits * 2 + 4) + list_bytes(chunks) + kHeader + 15) & ~(size_t)15;
    }
    __device__ __forceinline__ Lists(const SelectArgs& a, int64_t item) {
        uint8_t* p = a.workspace + item * a.item_bytes;
        header = reinterpret_cast<uint32_t*>(p);
        list = reinterpret_cast<uint2*>(p + kHeader);
        second = reinterpret_cast<uint16_t*>(p + kHeader);
        digits = reinterpret_cast<uint16_t*>(p + kHeader + list_bytes(a.chunks));
        above = reinterpret_cast<uint32_t*>(p + kHeader + list_bytes(a.chunks) + (size_t)a.chunks * kDigits * 2);
    }
    __device__ __forceinline__ Search first() const { return {header[1], Search::mask(0) << Search::shift(0), header[2]}; }
    __device__ __forceinline__ bool listed() const { return header[3] <= kListMost; }
};

// A thread's eight digits, from the largest of all down, of `chunks` rows together.
__device__ __forceinline__ void add_digits(const uint16_t* rows, int chunks, uint32_t (&n)[8]) {
    const uint4* from = reinterpret_cast<const uint4*>(rows) + (kDigits / 8 - 1 - threadIdx.x);
#pragma unroll 8
    for (int k = 0; k < chunks; k++) {
        const uint4 v = from[(size_t)k * (kDigits / 8)];
        const uint32_t d[4] = {v.w, v.z, v.y, v.x};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            n[2 * i] += d[i] >> 16;
            n[2 * i + 1] += d[i] & 0xFFFFu;
        }
    }
}

// The chunk of a workgroup, and the stretch of one of its four waves.
struct Chunk {
    int j0, j1, all;  // all: chunks that the head's keys fill
    __device__ __forceinline__ Chunk(const SelectArgs& a, const Cutting& x, int chunk) {
        const int wave = threadIdx.x >> 6, each = a.chunk_keys / (kManyThreads / 64);
        j0 = __builtin_amdgcn_readfirstlane(min(chunk * a.chunk_keys + wave * each, x.L));
        j1 = min(j0 + each, x.L);
        all = (x.L + a.chunk_keys - 1) / a.chunk_keys;
    }
};

__global__ __launch_bounds__(kManyThreads) void cache_select_digits_kernel(SelectArgs a) {
    __shared__ __align__(16) Histogram<kManyThreads, 4> hist;
    const Placed place(a.c, a.chunks);
    if (place.s < 0) return;
    const Cutting x(a, place.s, place.head);
    const Chunk chunk(a, x, place.chunk);
    if (x.whole() || x.need == 0 || place.chunk >= chunk.all) return;
    const Lists lists(a, (int64_t)x.s * a.c.heads + x.head);
    if (place.chunk == 0 && threadIdx.x == 0) lists.header[0] = 0;
    hist.clear();
    __syncthreads();
    Stretch st(a, x.s, x.head, chunk.j0, chunk.j1, x.m0, x.m1);
    st.each([&](int, const f32x4u& w, uint32_t free, uint32_t) {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (free >> i & 1) hist.add(ordered(w[i]), 0);
    });
    __syncthreads();
    hist.store(lists.digits + (size_t)place.chunk * kDigits);
}

__global__ __launch_bounds__(kManyThreads) void cache_select_aside_kernel(SelectArgs a) {
    __shared__ __align__(16) Histogram<kManyThreads, 4> hist;
    __shared__ uint32_t s_above, s_count, s_first, s_list[kListMost];
    const Placed place(a.c, a.chunks);
    if (place.s < 0) return;
    const Cutting x(a, place.s, place.head);
    const Chunk chunk(a, x, place.chunk);
    if (x.whole() || place.chunk >= chunk.all) return;
    const Lists lists(a, (int64_t)x.s * a.c.heads + x.head);
    const bool any = x.need > 0;
    Stretch st(a, x.s, x.head, chunk.j0, chunk.j1, x.m0, x.m1);
    Search search{0, 0, x.need};
    if (threadIdx.x == 0) s_above = s_count = 0;
    uint32_t having = 0;
    if (any) {
        uint32_t n[8] = {0, 0, 0, 0, 0, 0, 0, 0};  // of digits from the largest down
        add_digits(lists.digits, chunk.all, n);
        having = hist.find(search, 0, n);
        if (place.chunk == 0 && threadIdx.x == 0) {
            lists.header[1] = search.prefix;
            lists.header[2] = search.need;
            lists.header[3] = having;
        }
    }
    if (having > kListMost) {
        hist.clear();
        __syncthreads();
        st.each([&](int, const f32x4u& w, uint32_t free, uint32_t) {
            uint32_t u[4], mine, more;
            sort_out(search, w, free, u, mine, more);
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (mine >> i & 1) hist.add(u[i], 1);
        });
        __syncthreads();
        hist.store(lists.second + (size_t)place.chunk * kDigits);
        return;
    }
    __syncthreads();
    uint32_t above = 0;
    st.each([&](int, const f32x4u& w, uint32_t free, uint32_t forced) {
        uint32_t u[4], mine = 0, more = 0;
        if (any) {
            sort_out(search, w, free, u, mine, more);
            put_aside(mine, u, &s_count, [&](uint32_t at, uint32_t v) {
                if (at < kListMost) s_list[at] = v;  // (never more, as they are counted)
            });
        }
        above += (uint32_t)__popc(more | forced);
    });
    above = sum64(above);
    if ((threadIdx.x & 63) == 0) atomicAdd(&s_above, above);
    __syncthreads();
    const uint32_t n = min(s_count, (uint32_t)kListMost);
    if (threadIdx.x == 0) {
        lists.above[place.chunk] = s_above;
        s_first = n ? atomicAdd(lists.header, n) : 0;  // (a chunk's room in the head's list at once)
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kManyThreads)
        if (s_first + i < kListMost) lists.list[s_first + i] = make_uint2(s_list[i], (uint32_t)place.chunk);
}

// The third digit, where there is no list.
__global__ __launch_bounds__(kManyThreads) void cache_select_third_kernel(SelectArgs a) {
    __shared__ __align__(16) Histogram<kManyThreads, 4> hist;
    __shared__ uint32_t s_above;
    const Placed place(a.c, a.chunks);
    if (place.s < 0) return;
    const Cutting x(a, place.s, place.head);
    const Chunk chunk(a, x, place.chunk);
    if (x.whole() || x.need == 0 || place.chunk >= chunk.all) return;
    const Lists lists(a, (int64_t)x.s * a.c.heads + x.head);
    if (lists.listed()) return;
    Stretch st(a, x.s, x.head, chunk.j0, chunk.j1, x.m0, x.m1);
    Search search = lists.first();
    uint32_t n[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    add_digits(lists.second, chunk.all, n);
    if (threadIdx.x == 0) s_above = 0;
    hist.clear();
    hist.find(search, 1, n);
    if (place.chunk == 0 && threadIdx.x == 0) {
        lists.header[4] = search.prefix;
        lists.header[5] = search.need;
    }
    uint32_t above = 0;
    st.each([&](int, const f32x4u& w, uint32_t free, uint32_t forced) {
        uint32_t u[4], mine, more;
        sort_out(search, w, free, u, mine, more);
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (mine >> i & 1) hist.add(u[i], 2);
        above += (uint32_t)__popc(more | forced);
    });
    above = sum64(above);
    if ((threadIdx.x & 63) == 0) atomicAdd(&s_above, above);
    __syncthreads();
    hist.store(lists.digits + (size_t)place.chunk * kDigits);
    if (threadIdx.x == 0) lists.above[place.chunk] = s_above;
}

__global__ __launch_bounds__(kManyThreads) void cache_select_write_kernel(SelectArgs a) {
    __shared__ __align__(16) Histogram<kManyThreads, 4> hist;
    __shared__ uint32_t s_before[2], s_above[kManyThreads / 64], s_equal[kManyThreads / 64];
    const Placed place(a.c, a.chunks);
    if (place.s < 0) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Cutting x(a, place.s, place.head);
    const Chunk chunk(a, x, place.chunk);
    if (x.head == 0 && place.chunk == 0 && tid == 0) a.counts[x.s] = x.count;
    const int64_t stride = (int64_t)a.chunks * kManyThreads, here = (int64_t)place.chunk * kManyThreads + tid;
    for (int64_t i = x.count + here; i < a.budget; i += stride) x.kept[i] = -1;
    if (x.whole()) {
        for (int64_t i = here; i < x.L; i += stride) x.kept[i] = (int)i;
        return;
    }
    if (place.chunk >= chunk.all) return;
    const Lists lists(a, (int64_t)x.s * a.c.heads + x.head);
    const bool any = x.need > 0;
    Stretch st(a, x.s, x.head, chunk.j0, chunk.j1, x.m0, x.m1);
    Search search{0, 0, x.need};
    if (tid < 2) s_before[tid] = 0;
    uint32_t at = 0, same = 0;
    if (any && !lists.listed()) {
        search = {lists.header[4], ~Search::mask(2), lists.header[5]};
        uint32_t n[8] = {0, 0, 0, 0, 0, 0, 0, 0}, before[8];
        add_digits(lists.digits, place.chunk, n);
#pragma unroll
        for (int i = 0; i < 8; i++) before[i] = n[i];
        add_digits(lists.digits + (size_t)place.chunk * kDigits, chunk.all - place.chunk, n);
        hist.find(search, 2, n);
        const uint32_t found = search.prefix & Search::mask(2);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t digit = (uint32_t)(kDigits - 1 - 8 * tid - i);
            at += digit > found ? before[i] : 0;
            same += digit == found ? before[i] : 0;
        }
    } else if (any) {
        search = lists.first();
        const uint32_t having = lists.header[3];
        // f of every weight that begins with the prefix and its chunk
        auto each = [&](const auto& f) {
            for (uint32_t i = tid; i < having; i += 8 * kManyThreads) {  // eight in flight
                uint2 e[8];
#pragma unroll
                for (int k = 0; k < 8; k++) e[k] = lists.list[min(i + k * kManyThreads, having - 1)];
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (i + k * kManyThreads < having) f(e[k].x, (int)e[k].y);
            }
        };
        for (int pass = 1; pass < 3; pass++) {
            hist.clear();
            __syncthreads();
            each([&](uint32_t u, int) {
                if ((u & search.known) == search.prefix) hist.add(u, pass);
            });
            __syncthreads();
            hist.find(search, pass);
        }
        each([&](uint32_t u, int k) {
            at += k < place.chunk && u > search.prefix;
            same += k < place.chunk && u == search.prefix;
        });
    }
    for (int k = tid; k < place.chunk; k += kManyThreads) at += lists.above[k];
    uint32_t above = 0, equal = 0;
    st.each([&](int, const f32x4u& w, uint32_t free, uint32_t forced) {
        uint32_t p, q;
        look(search, any, w, free, forced, p, q);
        above += (uint32_t)__popc(p);
        equal += (uint32_t)__popc(q);
    });
    at = sum64(at);
    same = sum64(same);
    above = sum64(above);
    equal = sum64(equal);
    __syncthreads();
    if ((tid & 63) == 0) {
        s_above[wave] = above;
        s_equal[wave] = equal;
        atomicAdd(&s_before[0], at);
        atomicAdd(&s_before[1], same);
    }
    __syncthreads();
    at = s_before[0];
    same = s_before[1];
    for (int k = 0; k < wave; k++) {
        at += s_above[k];
        same += s_equal[k];
    }
    write_kept(st, search, any, at, same, x.kept);
}

// Keys of a chunk: 4096, or more where a head would have more than 64 of them; no more than
// 16 bits count.  0: a workgroup for a head: few keys, or items that pass a launch's 2^32
// threads, or enough of them to fill the chip, where a longest one of 65536 keys takes 58 us
// (256 of 32768 keys 38 us, in chunks 71 to 85; 512 of 65536 120 and 240 to 264; 128 of 32768
// 34 and 40 to 50, of 65536 64 and 72 to 80; but 32 of 65536 58 and 28).
int chunk_keys(int64_t items, int64_t reach) {
    if (reach <= (items >= 128 ? 65536 : kOneMost)) return 0;
    const int64_t n = std::min<int64_t>((reach + 64 * 4096 - 1) / (64 * 4096) * 4096, 61440);
    return (items + 7) * ((reach + n - 1) / n) < (int64_t)1 << 23 ? (int)n : 0;
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

size_t cache_select_workspace(int64_t items, int64_t reach) {
    const int keys = chunk_keys(items, reach);
    return keys ? (size_t)items * Lists::bytes((int)((reach + keys - 1) / keys)) : 0;
}

hipError_t launch_cache_select(const SelectArgs& args, hipStream_t stream) {
    SelectArgs a = args;
    const int64_t reach = ((int64_t)a.c.max_pages << a.c.bpp_log2) * kBlockTokens;
    a.chunk_keys = chunk_keys((int64_t)a.c.seqs * a.c.heads, reach);
    if (!a.chunk_keys) {
        const unsigned items = (unsigned)a.c.seqs * (unsigned)a.c.heads;
        if (reach <= 1024)  // (1080 heads of 102 keys 21 us, by 1024 threads each 27; 512 of 4000 17 and 13)
            cache_select_kernel<256><<<items, 256, 0, stream>>>(a);
        else
            cache_select_kernel<1024><<<items, 1024, 0, stream>>>(a);
        return hipGetLastError();
    }
    a.chunks = (int)((reach + a.chunk_keys - 1) / a.chunk_keys);
    a.item_bytes = Lists::bytes(a.chunks);
    const dim3 grid = placed_grid(a.c, a.chunks, kManyThreads);
    cache_select_digits_kernel<<<grid, kManyThreads, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    cache_select_aside_kernel<<<grid, kManyThreads, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    cache_select_third_kernel<<<grid, kManyThreads, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    cache_select_write_kernel<<<grid, kManyThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_cache_compact(const CompactArgs& a, hipStream_t stream) {
    // the turns of a head divided where they need no order
    const int64_t turns = (a.width / kBlockTokens + 2 + kWaves - 1) / kWaves;
    const int64_t most = ((int64_t)1 << 22) / ((int64_t)a.c.seqs * a.c.heads);
    const int64_t runs = a.in_place ? 1 : std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(turns, most), 32767));
    cache_compact_kernel<<<placed_grid(a.c, 2 * runs, kThreads), kThreads, 0, stream>>>(a, (int)runs);
    return hipGetLastError();
}

}  // namespace mxattn
