// rope.hip -- norm of every head of Q and K and their rotation by position.
//
// Bound by HBM: 2 bytes read and 2 written per element, and per token a row of
// angles (4 * rot bytes) that all its heads share.
//
// A row of 128 channels lies in 16 lanes (heads.h).  A group of 16 lanes takes one
// token and four of its heads, whose rows are in flight at once, so that the angles
// are read once for four rows; a wave holds four consecutive tokens of a head, which
// attention's layout [B, H, N, 128] stores as 1 KiB in one piece.  Q and K of 32760
// tokens x 40 heads, 1.36 GB: 236 us, 5.75 TB/s.  One head per group took 314 us,
// eight in two turns 241, sixteen 247; two rows in flight 244; stores that stay in
// the caches 252.
#include <type_traits>

#include "heads.h"

namespace mxattn {
namespace {

constexpr int kThreads = 256;
constexpr int kTokensPerGroup = kThreads / 16;
constexpr int kHeads = 4;

// Rotated halves, with a lane's eight channels in a row (loads and stores of 16
// bytes; with four of either half, 8 bytes each, rows of which half the channels
// rotate took a quarter longer): a channel's partner is in another lane, which
// hands over its eight.
struct HalvesAcross {
    f32x8 c, s;
    int partner;  // lane of the wave
    bool on;
    __device__ __forceinline__ HalvesAcross(const HeadTransform& t, int64_t pos, int lane) {
        const int self = (int)threadIdx.x & 63, half = t.rot >> 4;
        on = 8 * lane < t.rot;
        const bool second = lane >= half;
        partner = !on ? self : second ? self - half : self + half;
        if (!on) return;
        const float nan = __builtin_nanf("");
        c = s = f32x8{nan, nan, nan, nan, nan, nan, nan, nan};
        if ((uint64_t)pos >= (uint64_t)t.table_rows) return;
        const int64_t at = pos * (t.rot >> 1) + 8 * (second ? lane - half : lane);
        c = *reinterpret_cast<const f32x8*>(t.cos + at);
        s = *reinterpret_cast<const f32x8*>(t.sin + at);
        if (!second) s = -s;
    }
    __device__ __forceinline__ f32x8 turned(f32x8 x) const {
        f32x8 y;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float p = __shfl(x[i], partner);
            y[i] = on ? __builtin_fmaf(x[i], c[i], p * s[i]) : x[i];
        }
        return y;
    }
};

// Neighbours: a lane holds both channels of its four pairs.
struct PairsWithin : Rotation<false> {
    __device__ __forceinline__ PairsWithin(const HeadTransform& t, int64_t pos, int lane)
        : Rotation<false>(Rotation<false>::at(t, pos, lane)) {}
};

template <bool kHalves>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(RopeArgs a) {
    const int lane = threadIdx.x & 15;
    const int64_t token = a.first + (int64_t)blockIdx.x * kTokensPerGroup + (threadIdx.x >> 4);
    const bool live = token < a.tokens;
    const int64_t tok = live ? token : a.tokens - 1;
    const int64_t b = tok / a.N, n = tok - b * a.N;
    const int64_t pos = a.positions ? (int64_t)a.positions[tok] : n;
    const std::conditional_t<kHalves, HalvesAcross, PairsWithin> rotation(a.t, pos, lane);
    f32x8 w[2] = {};
#pragma unroll
    for (int i = 0; i < 2; i++)
        if (a.w[i]) w[i] = *reinterpret_cast<const f32x8*>(a.w[i] + 8 * lane);
    const int h0 = blockIdx.y * kHeads, h1 = min(h0 + kHeads, a.Hq + a.Hkv);
    u32x4 raw[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; i++) {
        const int h = min(h0 + i, h1 - 1), which = h >= a.Hq;
        const Strided& in = a.in[which];
        raw[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
            in.p + b * in.b + (which ? h - a.Hq : h) * in.h + n * in.n + 8 * lane));
    }
#pragma unroll
    for (int i = 0; i < kHeads; i++) {
        const int h = h0 + i, which = h >= a.Hq;
        if (h >= h1) break;
        const Strided& out = a.out[which];
        f32x8 x = unpack_bf16(raw[i]);
        if (a.w[which]) x = normed(x, which ? w[1] : w[0], a.t.eps);
        x = rotation.turned(x);
        u32x4* dst = reinterpret_cast<u32x4*>(out.p + b * out.b + (which ? h - a.Hq : h) * out.h + n * out.n + 8 * lane);
        if (live) __builtin_nontemporal_store(pack_bf16(x), dst);
    }
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs& args, bool halves, hipStream_t stream) {
    RopeArgs a = args;
    const int64_t tiles = (a.tokens + kTokensPerGroup - 1) / kTokensPerGroup;
    const unsigned chunks = (unsigned)((a.Hq + a.Hkv + kHeads - 1) / kHeads);
    constexpr int64_t kMost = 1 << 22;  // workgroups of a launch along the tokens
    for (int64_t t = 0; t < tiles; t += kMost) {
        const dim3 grid((unsigned)(tiles - t < kMost ? tiles - t : kMost), chunks);
        a.first = t * kTokensPerGroup;
        if (halves)
            qk_norm_rope_kernel<true><<<grid, kThreads, 0, stream>>>(a);
        else
            qk_norm_rope_kernel<false><<<grid, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace mxattn
