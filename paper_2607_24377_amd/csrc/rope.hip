// rope.hip -- norm of every head of Q and K and their rotation by position.
//
// Bound by HBM: 2 bytes read and 2 written per element, and per token a row of
// angles (4 * rot bytes) that all its heads share.
//
// A row of 128 channels lies in 16 lanes (heads.h).  A group of 16 lanes keeps
// one token and its angles and walks a chunk of the heads, so that the angles
// are read once per chunk; a wave holds four consecutive tokens of one head,
// which attention's layout [B, H, N, 128] stores as 1 KiB in one piece.
#include "heads.h"

namespace mxattn {
namespace {

constexpr int kThreads = 256;
constexpr int kTokensPerGroup = kThreads / 16;

template <bool kHalves>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(RopeArgs a) {
    const int lane = threadIdx.x & 15;
    const int64_t token = a.first + (int64_t)blockIdx.x * kTokensPerGroup + (threadIdx.x >> 4);
    const bool live = token < a.tokens;
    const int64_t tok = live ? token : a.tokens - 1;
    const int64_t b = tok / a.N, n = tok - b * a.N;
    const int64_t pos = a.positions ? (int64_t)a.positions[tok] : n;
    const Rotation<kHalves> rotation(a.t, pos, lane);
    const int h1 = min((int)(blockIdx.y + 1) * a.heads_per_chunk, a.Hq + a.Hkv);
    for (int h = blockIdx.y * a.heads_per_chunk; h < h1; h++) {
        const int which = h >= a.Hq;
        const int head = which ? h - a.Hq : h;
        const Strided& in = a.in[which];
        const Strided& out = a.out[which];
        f32x8 x = unpack_bf16(*reinterpret_cast<const u32x4*>(in.p + b * in.b + head * in.h + n * in.n + 8 * lane));
        if (const float* wp = a.w[which]) x = normed(x, *reinterpret_cast<const f32x8*>(wp + 8 * lane), a.t.eps);
        x = rotation.turned(x);
        if (live) *reinterpret_cast<u32x4*>(out.p + b * out.b + head * out.h + n * out.n + 8 * lane) = pack_bf16(x);
    }
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs& args, bool halves, hipStream_t stream) {
    RopeArgs a = args;
    const int64_t tiles = (a.tokens + kTokensPerGroup - 1) / kTokensPerGroup;
    const int heads = a.Hq + a.Hkv;
    a.heads_per_chunk = 1;
    const unsigned chunks = (unsigned)((heads + a.heads_per_chunk - 1) / a.heads_per_chunk);
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
