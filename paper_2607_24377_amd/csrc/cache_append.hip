// cache_append.hip -- new keys and values into the 8-bit paged cache.
//
// A block is 32 consecutive tokens of one sequence and head: 4096 codes (E4M3)
// and one E8M0 scale 2^e, the smallest with max |x| <= 448 2^e over the block.
// A block that gets tokens beside older ones keeps its scale or takes a larger
// one; then the older codes are rounded again, code * 2^(e_old - e), which is
// exact unless it falls below 2^-6 (a power of two leaves the 3 fraction bits
// alone).  Keys are normed and rotated in fp32 and rounded once, to the code.
//
// Block layouts are the operand orders of cache_attend.hip, so that it copies
// them in one piece: K [8 chunks of 16 channels][32 tokens][16], V
// [128 channels][32 tokens].
//
// Bound by HBM: 2 bytes read and 1 written per element.  One workgroup per
// block and head; sequence s owns workgroups q_start[s] / 32 + 2 s onwards,
// which are as many as the blocks that its tokens can touch, so that the grid
// follows from the number of tokens and sequences alone.
#include "heads.h"

namespace mxattn {
namespace {

constexpr int kThreads = 256;

// E8M0 byte of the smallest scale that holds magnitudes up to M (bits of a
// finite fp32 >= 0): M = 1.f 2^(E-127) <= 1.75 2^(8 + e).
__device__ __forceinline__ int scale_byte(uint32_t mbits) {
    const int e = (int)(mbits >> 23) - 8 + ((mbits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return max(e, 0);
}

// E4M3 codes of x 2^(127 - byte), nearest even; |x| <= 448 * 2^(byte - 127), or
// not finite: NaN.
__device__ __forceinline__ uint2 encode8(const f32x8& x, int byte) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float v = __builtin_ldexpf(x[i], 127 - byte);
        y[i] = __builtin_fabsf(x[i]) < __builtin_inff() ? v : __builtin_nanf("");
    }
    uint2 r;
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    r.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], p, true);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
    r.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], p, true);
    return r;
}

// Four codes times 2^shift (shift <= 0).
__device__ __forceinline__ uint32_t rescale4(uint32_t c, int shift) {
    const f32x2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
    const f32x2v b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    const int p = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(a[0], shift), __builtin_ldexpf(a[1], shift), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(b[0], shift), __builtin_ldexpf(b[1], shift), p, true);
}

// Largest magnitude bits of the finite values of x.
__device__ __forceinline__ uint32_t magnitude(const f32x8& x) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float f = x[i];  // (a bit cast of a vector's element itself reads its first one)
        const uint32_t u = __builtin_bit_cast(uint32_t, f) & 0x7FFFFFFFu;
        m = max(m, u < 0x7F800000u ? u : 0u);
    }
    return m;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    return m;
}

template <bool kHalves>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(AppendArgs a) {
    __shared__ int s_seq;
    __shared__ uint32_t s_max[2][4];
    __shared__ __align__(16) uint8_t s_v[kBlockBytes];
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, lane = tid & 15;
    const int w = blockIdx.x, head = blockIdx.y;
    if (tid == 0) s_seq = -1;
    __syncthreads();
    for (int s = tid; s < c.seqs; s += kThreads) {
        const TokenRange r = token_range(c, s);
        const int base = r.first / kBlockTokens + 2 * s, next = r.last / kBlockTokens + 2 * (s + 1);
        if (base <= w && w < next) s_seq = s;
    }
    __syncthreads();
    const int s = s_seq;
    if (s < 0) return;
    const TokenRange r = token_range(c, s);
    const int reach = c.max_pages << c.bpp_log2;  // blocks
    const int len = c.kv_len[s];
    if (len < 0 || (int64_t)len > (int64_t)reach * kBlockTokens) return;
    const int first = len - (r.last - r.first);  // the new tokens' positions: first .. len - 1
    const int from = max(first, 0);
    if (from >= len || r.first == r.last) return;
    const int block = from / kBlockTokens + (w - (r.first / kBlockTokens + 2 * s));
    const int p0 = block * kBlockTokens;
    if (p0 >= len) return;
    const int page = c.page_table[(int64_t)s * c.max_pages + (block >> c.bpp_log2)];
    if ((unsigned)page >= (unsigned)c.pages) return;
    const int64_t at = (((int64_t)page * c.heads + head) << c.bpp_log2) + (block & ((1 << c.bpp_log2) - 1));
    uint8_t* kb = a.c.kc + at * kBlockBytes;
    uint8_t* vb = a.c.vc + at * kBlockBytes;
    const int lead = max(from - p0, 0);                 // older tokens in the block
    const int stop = min(len - p0, kBlockTokens);       // tokens lead .. stop - 1 are new

    // two tokens of the block per thread: 8 channels of K and of V
    f32x8 k[2], v[2];
    uint32_t mk = 0, mv = 0;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int slot = (tid >> 4) + 16 * i;
        const bool live = slot >= lead && slot < stop;
        const int64_t tok = r.first + (live ? p0 + slot - first : from - first);
        k[i] = unpack_bf16(*reinterpret_cast<const u32x4*>(a.k + tok * a.k_stride + head * kHeadDim + 8 * lane));
        v[i] = unpack_bf16(*reinterpret_cast<const u32x4*>(a.v + tok * a.v_stride + head * kHeadDim + 8 * lane));
        if (a.w) k[i] = normed(k[i], *reinterpret_cast<const f32x8*>(a.w + 8 * lane), a.t.eps);
        const Rotation<kHalves> rotation(a.t, a.positions ? (int64_t)a.positions[tok] : (int64_t)(p0 + slot), lane);
        k[i] = rotation.turned(k[i]);
        if (live) {
            mk = max(mk, magnitude(k[i]));
            mv = max(mv, magnitude(v[i]));
        }
    }
    mk = wave_max(mk);
    mv = wave_max(mv);
    if ((tid & 63) == 0) {
        s_max[0][tid >> 6] = mk;
        s_max[1][tid >> 6] = mv;
    }
    const int was_k = lead ? c.ks[at] : 0, was_v = lead ? c.vs[at] : 0;
    // a block with older or missing tokens keeps those bytes of V's rows
    if (lead || stop < kBlockTokens)
        *reinterpret_cast<uint4*>(s_v + 16 * tid) = *reinterpret_cast<const uint4*>(vb + 16 * tid);
    __syncthreads();
    mk = max(max(s_max[0][0], s_max[0][1]), max(s_max[0][2], s_max[0][3]));
    mv = max(max(s_max[1][0], s_max[1][1]), max(s_max[1][2], s_max[1][3]));
    const int bk = max(scale_byte(mk), was_k), bv = max(scale_byte(mv), was_v);
    if (lead && bv > was_v) {
        uint32_t* row = reinterpret_cast<uint32_t*>(s_v + 16 * tid);
        const int t0 = 16 * (tid & 1);  // the thread's 16 tokens of a channel
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int n = lead - t0 - 4 * i;  // older ones of these four
            const uint32_t mask = n <= 0 ? 0u : n >= 4 ? ~0u : (1u << (8 * n)) - 1;
            row[i] = (rescale4(row[i], was_v - bv) & mask) | (row[i] & ~mask);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int slot = (tid >> 4) + 16 * i;
        uint2* kd = reinterpret_cast<uint2*>(kb + (lane >> 1) * 512 + slot * 16 + (lane & 1) * 8);
        if (slot >= lead && slot < stop) {
            *kd = encode8(k[i], bk);
            const uint2 q = encode8(v[i], bv);
            uint8_t* vd = s_v + 8 * lane * kBlockTokens + slot;
#pragma unroll
            for (int j = 0; j < 8; j++) vd[j * kBlockTokens] = (uint8_t)((j < 4 ? q.x : q.y) >> (8 * (j & 3)));
        } else if (slot < lead && bk > was_k) {
            const uint2 q = *kd;
            *kd = make_uint2(rescale4(q.x, was_k - bk), rescale4(q.y, was_k - bk));
        }
    }
    __syncthreads();
    *reinterpret_cast<uint4*>(vb + 16 * tid) = *reinterpret_cast<const uint4*>(s_v + 16 * tid);
    if (tid == 0) {
        c.ks[at] = (uint8_t)bk;
        c.vs[at] = (uint8_t)bv;
    }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, bool halves, hipStream_t stream) {
    const dim3 grid((unsigned)(a.c.tokens / kBlockTokens + 2 * a.c.seqs), (unsigned)a.c.heads);
    if (halves)
        cache_append_kernel<true><<<grid, kThreads, 0, stream>>>(a);
    else
        cache_append_kernel<false><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace mxattn
