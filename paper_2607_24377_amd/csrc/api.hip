// api.hip -- the extern "C" entry points of libmxattn (see include/mxattn.h).
//
// Argument validation happens before any HIP call, so every error path is
// free of device work.  The only global state is the workspace memory
// (workspace.h) and the static scratch of the no-allocation entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>
#include <mutex>

#include "../../include/mxattn.h"
#include "cache.h"
#include "launch.h"
#include "workspace.h"

namespace {

using mxattn::g_last_error;
using mxattn::kMaxDevices;
using mxattn::set_error;
using mxattn::Workspace;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Whether the byte ranges [a, a + na) and [b, b + nb) share a byte.
bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

bool valid_mode(int mode) { return mode >= MXATTN_OCP_VANILLA && mode <= MXATTN_UOS_PNQ_ROT; }

// The attention kernel's mode: the rotated mode differs only in how Q and K
// were quantized.
int kernel_mode(int mode) { return mode == MXATTN_UOS_PNQ_ROT ? MXATTN_UOS_PNQ : mode; }

// Shape limits of the kernels: 32-bit token indices, 64-bit byte offsets, and
// at most 2^35 elements per tensor (64 GiB of bf16), which keeps every grid
// below 2^31 workgroups.
int check_shape(int64_t B, int64_t H, int64_t N, int64_t d) {
    if (B < 1 || H < 1 || N < 1 || d < 1) return MXATTN_ERR_SHAPE;
    if (B > (1 << 20) || H > (1 << 20) || N > (1 << 28)) return MXATTN_ERR_SHAPE;
    if (B * H > (int64_t)1 << 24) return MXATTN_ERR_SHAPE;
    if (B * H * N * 128 > (int64_t)1 << 35) return MXATTN_ERR_SHAPE;
    if (d != 128) return MXATTN_ERR_UNSUPPORTED;
    return MXATTN_OK;
}

int rule_of(int mode) { return mode == MXATTN_OCP_VANILLA ? mxattn::kRuleOcp : mxattn::kRuleUos; }

}  // namespace

extern "C" {

int mxattn_version(void) { return 103; }

int mxattn_release_workspace(void) { return mxattn::release_workspace(); }

int mxattn_kv_tile(void) { return mxattn::kKvTile; }

int mxattn_query_tile(void) { return mxattn::kQueryTile; }

const char* mxattn_status_string(int s) {
    switch (s) {
        case MXATTN_OK: return "ok";
        case MXATTN_ERR_NULL: return "null pointer argument";
        case MXATTN_ERR_SHAPE: return "invalid shape (sizes must be >= 1 and within limits, strides not negative, outputs apart from inputs and workspace)";
        case MXATTN_ERR_ALIGN: return "misaligned pointer or stride (tensors need 16-byte alignment, strides multiples of 8 elements)";
        case MXATTN_ERR_MODE: return "invalid mode (0 ocp_vanilla, 1 uos, 2 uos_pnq, 3 uos_pnq_rot)";
        case MXATTN_ERR_AXIS: return "invalid block_axis (2 = tokens, 3 = head dim)";
        case MXATTN_ERR_UNSUPPORTED: return "unsupported head dimension (d must be 128)";
        case MXATTN_ERR_OOM: return "workspace allocation failed";
        case MXATTN_ERR_HIP: return "HIP runtime error";
        case MXATTN_ERR_SCRATCH: return "more scratch needed than there is (the no-allocation entry point: B*H*ceil(Nkv/128) <= 32768; cache attention: a workspace of mxattn_cache_attend_workspace() or mxattn_cache_attend_weights_workspace() bytes, selection: of mxattn_cache_select_workspace(), from the caller, always on a stream under graph capture)";
        case MXATTN_ERR_BOUNDARY: return "invalid scale boundary (need 4 <= q <= 8 and 1 <= nq <= 64) or pre-scale (need 0 < gamma < 3e38)";
        case MXATTN_ERR_VALUE: return "invalid value (rot 0 or a multiple of 16 up to 128, pairs 0 or 1, eps finite and >= 0, page_tokens a power of two from 32 to 4096, Hq a multiple of Hkv, at most 256 of it, window >= 1, sinks and recent >= 0 and together at most a budget of 1 to 2^24)";
        default: return "unknown status";
    }
}

const char* mxattn_last_error(void) { return g_last_error; }

size_t mxattn_codes_bytes(int block_axis, int64_t B, int64_t H, int64_t N, int64_t d) {
    if (check_shape(B, H, N, d) != MXATTN_OK) return 0;
    if (block_axis == MXATTN_AXIS_HEAD_DIM) return (size_t)(B * H * N * (d / 2));
    if (block_axis == MXATTN_AXIS_TOKENS) return (size_t)(B * H * d * ((N + 31) / 32) * 16);
    return 0;
}

size_t mxattn_scales_bytes(int block_axis, int64_t B, int64_t H, int64_t N, int64_t d) {
    if (check_shape(B, H, N, d) != MXATTN_OK) return 0;
    if (block_axis == MXATTN_AXIS_HEAD_DIM) return (size_t)(B * H * N * (d / 32));
    if (block_axis == MXATTN_AXIS_TOKENS) return (size_t)(B * H * d * ((N + 31) / 32));
    return 0;
}

int mxattn_quantize(const void* x, uint8_t* codes, uint8_t* scales, int block_axis, int mode,
                    int64_t B, int64_t H, int64_t N, int64_t d, void* stream) {
    if (!x || !codes || !scales) return MXATTN_ERR_NULL;
    if (block_axis != MXATTN_AXIS_HEAD_DIM && block_axis != MXATTN_AXIS_TOKENS) return MXATTN_ERR_AXIS;
    if (!valid_mode(mode)) return MXATTN_ERR_MODE;
    if (int st = check_shape(B, H, N, d)) return st;
    if (!aligned(x, 16) || !aligned(codes, 16)) return MXATTN_ERR_ALIGN;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipError_t e;
    if (block_axis == MXATTN_AXIS_HEAD_DIM && mode == MXATTN_UOS_PNQ_ROT)
        e = mxattn::launch_quantize_headdim_rotated(x, codes, scales, B * H * N, rule_of(mode), s);
    else if (block_axis == MXATTN_AXIS_HEAD_DIM)
        e = mxattn::launch_quantize_headdim(x, codes, scales, B * H * N, rule_of(mode), s);
    else
        e = mxattn::launch_quantize_tokens(x, codes, scales, B * H, N, rule_of(mode), s);
    if (e != hipSuccess) {
        set_error("quantize launch", e);
        return MXATTN_ERR_HIP;
    }
    return MXATTN_OK;
}

int mxattn_quantize_qmax(const void* x, uint8_t* codes, uint8_t* scales, int block_axis, double qmax,
                         int64_t B, int64_t H, int64_t N, int64_t d, void* stream) {
    if (!x || !codes || !scales) return MXATTN_ERR_NULL;
    if (block_axis != MXATTN_AXIS_HEAD_DIM && block_axis != MXATTN_AXIS_TOKENS) return MXATTN_ERR_AXIS;
    if (!(qmax >= 4.0 && qmax <= 8.0)) return MXATTN_ERR_BOUNDARY;
    if (int st = check_shape(B, H, N, d)) return st;
    if (!aligned(x, 16) || !aligned(codes, 16)) return MXATTN_ERR_ALIGN;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipError_t e = block_axis == MXATTN_AXIS_HEAD_DIM
                       ? mxattn::launch_quantize_headdim(x, codes, scales, B * H * N, mxattn::kRuleQmax, s, qmax)
                       : mxattn::launch_quantize_tokens(x, codes, scales, B * H, N, mxattn::kRuleQmax, s, qmax);
    if (e != hipSuccess) {
        set_error("quantize launch", e);
        return MXATTN_ERR_HIP;
    }
    return MXATTN_OK;
}

int mxattn_qmax_sse(const void* x, int block_axis, const double* qs, int nq, double* sse, int64_t B,
                    int64_t H, int64_t N, int64_t d, void* stream) {
    if (!x || !qs || !sse) return MXATTN_ERR_NULL;
    if (block_axis != MXATTN_AXIS_HEAD_DIM && block_axis != MXATTN_AXIS_TOKENS) return MXATTN_ERR_AXIS;
    if (nq < 1 || nq > MXATTN_MAX_BOUNDARIES) return MXATTN_ERR_BOUNDARY;
    for (int j = 0; j < nq; j++)
        if (!(qs[j] >= 4.0 && qs[j] <= 8.0)) return MXATTN_ERR_BOUNDARY;
    if (int st = check_shape(B, H, N, d)) return st;
    if (!aligned(x, 16) || !aligned(sse, 8)) return MXATTN_ERR_ALIGN;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    Workspace ws;
    if (int st = ws.take((size_t)mxattn::qmax_sse_workspace_bytes(block_axis, B * H, N), s)) return st;
    int st = MXATTN_OK;
    hipError_t e = mxattn::launch_qmax_sse(x, block_axis, qs, nq, sse, ws.get(), B * H, N, s);
    if (e != hipSuccess) {
        set_error("sse sweep launch", e);
        st = MXATTN_ERR_HIP;
    }
    return ws.give_back(st);
}

int mxattn_softmax_rows(const void* q, const void* k, float* p, int64_t B, int64_t H, int64_t Nq,
                        int64_t Nkv, int64_t d, int64_t row0, int64_t rows, int64_t ld, void* stream) {
    if (!q || !k || !p) return MXATTN_ERR_NULL;
    if (int st = check_shape(B, H, Nq, d)) return st;
    if (int st = check_shape(B, H, Nkv, d)) return st;
    if (row0 < 0 || rows < 1 || row0 + rows > Nq || ld < Nkv || ld % 4 != 0 || ld > (1 << 28))
        return MXATTN_ERR_SHAPE;
    const int64_t qtiles = (rows + 127) / 128;
    if (B * H * qtiles > ((int64_t)1 << 31) - 1) return MXATTN_ERR_SHAPE;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(p, 16)) return MXATTN_ERR_ALIGN;
    mxattn::SoftmaxRowsArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.p = p;
    a.Nq = (int)Nq;
    a.Nkv = (int)Nkv;
    a.row0 = (int)row0;
    a.rows = (int)rows;
    a.ld = (int)ld;
    hipError_t e = mxattn::launch_attn_rows(a, B * H, mxattn::kRowsStoreP, reinterpret_cast<hipStream_t>(stream));
    if (e != hipSuccess) {
        set_error("softmax rows launch", e);
        return MXATTN_ERR_HIP;
    }
    return MXATTN_OK;
}

static bool valid_gamma(float gamma) { return gamma > 0.0f && gamma < 3.0e38f; }

int mxattn_rowsum_diag(const float* p, int64_t rows, int64_t N, int64_t ld, int mode, float gamma,
                       double* stats, void* stream) {
    if (!p || !stats) return MXATTN_ERR_NULL;
    if (!valid_mode(mode)) return MXATTN_ERR_MODE;
    if (rows < 1 || rows > ((int64_t)1 << 31) - 1 || N < 1 || N > (1 << 28) || ld < N || ld % 4 != 0)
        return MXATTN_ERR_SHAPE;
    if (!valid_gamma(gamma)) return MXATTN_ERR_BOUNDARY;
    if (!aligned(p, 16) || !aligned(stats, 8)) return MXATTN_ERR_ALIGN;
    mxattn::RowsumDiagArgs a{};
    a.p = p;
    a.N = N;
    a.ld = ld;
    a.gamma = gamma;
    a.g = 1.0 / (double)gamma;
    a.stats = stats;
    a.rows_per_head = rows;
    a.out_rows_per_head = rows;
    a.out_row0 = 0;
    hipError_t e = mxattn::launch_rowsum_diag(a, rows, rule_of(mode), reinterpret_cast<hipStream_t>(stream));
    if (e != hipSuccess) {
        set_error("row-sum diagnostic launch", e);
        return MXATTN_ERR_HIP;
    }
    return MXATTN_OK;
}

int mxattn_attention_rowsum_diag(const void* q, const void* k, int64_t B, int64_t H, int64_t Nq,
                                 int64_t Nkv, int64_t d, int mode, float gamma, double* stats,
                                 void* stream) {
    if (!q || !k || !stats) return MXATTN_ERR_NULL;
    if (!valid_mode(mode)) return MXATTN_ERR_MODE;
    if (int st = check_shape(B, H, Nq, d)) return st;
    if (int st = check_shape(B, H, Nkv, d)) return st;
    if (!valid_gamma(gamma)) return MXATTN_ERR_BOUNDARY;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(stats, 8)) return MXATTN_ERR_ALIGN;
    if (B * H * ((Nq + 127) / 128) > ((int64_t)1 << 31) - 1) return MXATTN_ERR_SHAPE;
    mxattn::SoftmaxRowsArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.Nq = (int)Nq;
    a.Nkv = (int)Nkv;
    a.row0 = 0;
    a.rows = (int)Nq;
    a.gamma = gamma;
    a.g = 1.0 / (double)gamma;
    a.stats = stats;
    const int out = rule_of(mode) == mxattn::kRuleUos ? mxattn::kRowsDiagUos : mxattn::kRowsDiagOcp;
    hipError_t e = mxattn::launch_attn_rows(a, B * H, out, reinterpret_cast<hipStream_t>(stream));
    if (e != hipSuccess) {
        set_error("row-sum diagnostic launch", e);
        return MXATTN_ERR_HIP;
    }
    return MXATTN_OK;
}

// Limits of the fused attention kernel beyond check_shape: the key length
// (32-bit byte offsets within one head's K^/V^) and the workgroup count.
int check_attention_shape(int64_t B, int64_t H, int64_t Nq, int64_t Nkv) {
    if (Nkv > mxattn::kMaxKeys) return MXATTN_ERR_SHAPE;
    if (B * H * ((Nq + mxattn::kQueryTile - 1) / mxattn::kQueryTile) > (int64_t)1 << 30) return MXATTN_ERR_SHAPE;
    return MXATTN_OK;
}

// The fused attention kernel: on Q^ = (qc, qs), or, when qraw is not null, on
// the bf16 Q that the kernel quantizes itself (qc and qs are then unused); sc
// holds the K^/V^ scales in operand order.  v_tiled: V^ codes stored tile by
// tile (launch_prepare_operands) instead of in channel rows.
static int launch_attend(const void* qraw, const uint8_t* qc, const uint8_t* qs, const uint8_t* kc,
                         const uint8_t* vc, bool v_tiled, const uint8_t* sc, uint8_t* split_ws, void* out,
                         int64_t B, int64_t H, int64_t Nq, int64_t Nkv, int mode, hipStream_t s) {
    mxattn::AttnArgs a;
    a.qc = qc;
    a.qs = qs;
    a.qraw = static_cast<const uint16_t*>(qraw);
    a.kc = kc;
    a.vc = vc;
    const int ntiles = (int)((Nkv + mxattn::kKvTile - 1) / mxattn::kKvTile);
    a.vrow = v_tiled ? mxattn::v_tile_row_bytes(Nkv) : (int)((Nkv + 31) / 32) * 16;
    a.vtile = v_tiled ? 128 * a.vrow : 64;
    a.vhead = v_tiled ? ntiles * a.vtile : 128 * a.vrow;
    a.sc = sc;
    a.out = static_cast<uint16_t*>(out);
    a.N = (int)Nkv;
    a.Nq = (int)Nq;
    a.qtiles = (int)((Nq + mxattn::kQueryTile - 1) / mxattn::kQueryTile);
    // one query tile per workgroup; with K^/V^ resident in LDS, chunks of at
    // most 16 query tiles, as many as fill whole rounds of the workgroups
    // resident at once, split evenly by the kernel.  Those are 512, two per CU;
    // of the one-tile kernels on quantized Q (152 VGPRs, 26 KB of LDS) three fit:
    // attend, 40 heads x 32760 queries x 128 keys 108.2 us in rounds of 512, 97.3
    // in rounds of 768; on bf16 Q (164 to 179 VGPRs) the same call 144 and 158
    int64_t nchunks = a.qtiles;
    if (Nkv <= mxattn::kResidentKeys) {
        const int64_t slots = ntiles == 1 && !qraw ? 768 : 512, bh = B * H;
        const int64_t min_chunks = (a.qtiles + 15) / 16;
        const int64_t rounds = (bh * min_chunks + slots - 1) / slots;
        const int64_t k = rounds * slots / bh;
        nchunks = k < min_chunks ? min_chunks : (k > a.qtiles ? a.qtiles : k);
    }
    a.nchunks = (int)nchunks;
    a.nsplit = mxattn::key_splits(B * H, Nq, Nkv);
    const int64_t total = B * H * a.nchunks * a.nsplit;
    if (a.nsplit > 1) {
        // a part has at least four tiles
        const int64_t tiles_per_run = ntiles / a.nsplit;
        a.score_parts = (int)(tiles_per_run / 4 < mxattn::kScoreParts ? tiles_per_run / 4 : mxattn::kScoreParts);
        if (a.score_parts < 1) a.score_parts = 1;
        a.part_o = reinterpret_cast<float4*>(split_ws);
        a.part_ml = reinterpret_cast<float2*>(split_ws + total * (128 * 128 * 4));
        a.run_max = reinterpret_cast<float*>(split_ws + total * (128 * (128 * 4 + 8)));
    }
    a.total_tiles = (int)total;
    a.per_xcd = (int)((total + 7) / 8);
    hipError_t e = mxattn::launch_attention(a, kernel_mode(mode), s);
    if (e != hipSuccess) {
        set_error("attention launch", e);
        return MXATTN_ERR_HIP;
    }
    return MXATTN_OK;
}

// The same on operands in the public layouts: rearranges the K^/V^ scales into
// sc (mxattn::tile_scales_bytes(B*H, Nkv) bytes of workspace) first.
static int launch_attend_public(const uint8_t* qc, const uint8_t* qs, const uint8_t* kc, const uint8_t* ks,
                                const uint8_t* vc, const uint8_t* vs, uint8_t* sc, uint8_t* split_ws, void* out,
                                int64_t B, int64_t H, int64_t Nq, int64_t Nkv, int mode, hipStream_t s) {
    hipError_t e = mxattn::launch_tile_scales(ks, vs, sc, B * H, Nkv, s);
    if (e != hipSuccess) {
        set_error("scale layout launch", e);
        return MXATTN_ERR_HIP;
    }
    return launch_attend(nullptr, qc, qs, kc, vc, false, sc, split_ws, out, B, H, Nq, Nkv, mode, s);
}

// Whether `out` ([B, H, Nq, d] bf16) shares memory with any quantized operand.
static bool attend_out_aliases(const uint8_t* qc, const uint8_t* qs, const uint8_t* kc, const uint8_t* ks,
                               const uint8_t* vc, const uint8_t* vs, const void* out, int64_t B, int64_t H,
                               int64_t Nq, int64_t Nkv, int64_t d) {
    const size_t ob = (size_t)(B * H * Nq * d * 2);
    return overlaps(out, ob, qc, mxattn_codes_bytes(MXATTN_AXIS_HEAD_DIM, B, H, Nq, d)) ||
           overlaps(out, ob, qs, mxattn_scales_bytes(MXATTN_AXIS_HEAD_DIM, B, H, Nq, d)) ||
           overlaps(out, ob, kc, mxattn_codes_bytes(MXATTN_AXIS_HEAD_DIM, B, H, Nkv, d)) ||
           overlaps(out, ob, ks, mxattn_scales_bytes(MXATTN_AXIS_HEAD_DIM, B, H, Nkv, d)) ||
           overlaps(out, ob, vc, mxattn_codes_bytes(MXATTN_AXIS_TOKENS, B, H, Nkv, d)) ||
           overlaps(out, ob, vs, mxattn_scales_bytes(MXATTN_AXIS_TOKENS, B, H, Nkv, d));
}

// Argument checks of the attention calls on quantized operands.
static int check_attend_args(const uint8_t* q_codes, const uint8_t* q_scales, const uint8_t* k_codes,
                             const uint8_t* k_scales, const uint8_t* v_codes, const uint8_t* v_scales,
                             const void* out, int64_t B, int64_t H, int64_t Nq, int64_t Nkv, int64_t d,
                             int mode) {
    if (!q_codes || !q_scales || !k_codes || !k_scales || !v_codes || !v_scales || !out)
        return MXATTN_ERR_NULL;
    if (!valid_mode(mode)) return MXATTN_ERR_MODE;
    if (int st = check_shape(B, H, Nq, d)) return st;
    if (int st = check_shape(B, H, Nkv, d)) return st;
    if (int st = check_attention_shape(B, H, Nq, Nkv)) return st;
    if (!aligned(q_codes, 16) || !aligned(k_codes, 16) || !aligned(v_codes, 16) ||
        !aligned(out, 16) || !aligned(k_scales, 4))
        return MXATTN_ERR_ALIGN;
    if (attend_out_aliases(q_codes, q_scales, k_codes, k_scales, v_codes, v_scales, out, B, H, Nq, Nkv, d))
        return MXATTN_ERR_SHAPE;
    return MXATTN_OK;
}

int mxattn_cross_attend(const uint8_t* q_codes, const uint8_t* q_scales, const uint8_t* k_codes,
                        const uint8_t* k_scales, const uint8_t* v_codes, const uint8_t* v_scales,
                        void* out, int64_t B, int64_t H, int64_t Nq, int64_t Nkv, int64_t d, int mode,
                        void* stream) {
    if (int st = check_attend_args(q_codes, q_scales, k_codes, k_scales, v_codes, v_scales, out, B, H, Nq, Nkv,
                                   d, mode))
        return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const size_t scale_bytes = (size_t)mxattn::tile_scales_bytes(B * H, Nkv);
    Workspace ws;
    if (int st = ws.take(scale_bytes + mxattn::split_bytes(B * H, Nq, mxattn::key_splits(B * H, Nq, Nkv)), s)) return st;
    return ws.give_back(launch_attend_public(q_codes, q_scales, k_codes, k_scales, v_codes, v_scales, ws.get(),
                                             ws.get() + scale_bytes, out, B, H, Nq, Nkv, mode, s));
}

// ---- the entry point that allocates nothing
//
// mxattn_cross_attend_noalloc keeps its one buffer beyond the inputs and the
// output, the K^/V^ scales rearranged into MFMA operand order (1 KiB per
// (batch, head) and 128-key tile), in this static device array instead of
// allocated workspace, with the partial results of divided keys behind it.  A
// device holds its own copy from the first such call on it until the process ends
// (the runtime loads this file's device code, which is nothing else, when its
// address is first asked for).  On the host, `scratch` is only a stand-in symbol,
// never a device address: the device address comes from hipGetSymbolAddress,
// taken once per device with that device current, and only that address is
// passed to kernels.  Every call on a device shares the device's array, so
// calls that overlap in time on one device race.
static __device__ __align__(256) uint8_t scratch[MXATTN_NOALLOC_SCRATCH_BYTES +
                                                  mxattn::kMaxSplitWorkgroups * mxattn::kSplitBytesPerWorkgroup];

struct ScratchSlot {
    std::once_flag once;
    hipError_t err = hipSuccess;
    void* ptr = nullptr;
};
ScratchSlot g_scratch[kMaxDevices];

// The current device's address of `scratch` (looked up on the first call on
// that device).
static int scratch_address(void** out) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) {
        set_error("hipGetDevice", e);
        return MXATTN_ERR_HIP;
    }
    if (dev < 0 || dev >= kMaxDevices) {
        set_error("device index beyond the library's limit", hipErrorInvalidDevice);
        return MXATTN_ERR_HIP;
    }
    ScratchSlot& slot = g_scratch[dev];
    std::call_once(slot.once, [&slot] {
        void* p = nullptr;
        slot.err = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (slot.err == hipSuccess && p)
            slot.ptr = p;
        else
            (void)hipGetLastError();
    });
    if (slot.err != hipSuccess || !slot.ptr) {
        set_error("hipGetSymbolAddress(scratch)", slot.err != hipSuccess ? slot.err : hipErrorInvalidSymbol);
        return MXATTN_ERR_HIP;
    }
    *out = slot.ptr;
    return MXATTN_OK;
}

int mxattn_cross_attend_noalloc(const uint8_t* q_codes, const uint8_t* q_scales, const uint8_t* k_codes,
                                const uint8_t* k_scales, const uint8_t* v_codes, const uint8_t* v_scales,
                                void* out, int64_t B, int64_t H, int64_t Nq, int64_t Nkv, int64_t d,
                                int mode, void* stream) {
    if (int st = check_attend_args(q_codes, q_scales, k_codes, k_scales, v_codes, v_scales, out, B, H, Nq, Nkv,
                                   d, mode))
        return st;
    const int64_t need = mxattn::tile_scales_bytes(B * H, Nkv);
    if (need > (int64_t)MXATTN_NOALLOC_SCRATCH_BYTES) {
        std::snprintf(g_last_error, sizeof g_last_error,
                      "mxattn_cross_attend_noalloc: %lld bytes of scale scratch needed (B*H*ceil(Nkv/128) KiB), "
                      "the static buffer holds %lld",
                      (long long)need, (long long)MXATTN_NOALLOC_SCRATCH_BYTES);
        return MXATTN_ERR_SCRATCH;
    }
    void* sc = nullptr;
    if (int st = scratch_address(&sc)) return st;
    return launch_attend_public(q_codes, q_scales, k_codes, k_scales, v_codes, v_scales, static_cast<uint8_t*>(sc),
                                static_cast<uint8_t*>(sc) + MXATTN_NOALLOC_SCRATCH_BYTES, out, B, H, Nq, Nkv, mode,
                                reinterpret_cast<hipStream_t>(stream));
}

int mxattn_attend(const uint8_t* q_codes, const uint8_t* q_scales, const uint8_t* k_codes,
                  const uint8_t* k_scales, const uint8_t* v_codes, const uint8_t* v_scales,
                  void* out, int64_t B, int64_t H, int64_t N, int64_t d, int mode, void* stream) {
    return mxattn_cross_attend(q_codes, q_scales, k_codes, k_scales, v_codes, v_scales, out, B, H, N,
                               N, d, mode, stream);
}

int mxattn_cross_forward(const void* q, const void* k, const void* v, void* out, int64_t B,
                         int64_t H, int64_t Nq, int64_t Nkv, int64_t d, int mode, void* stream) {
    if (!q || !k || !v || !out) return MXATTN_ERR_NULL;
    if (!valid_mode(mode)) return MXATTN_ERR_MODE;
    if (int st = check_shape(B, H, Nq, d)) return st;
    if (int st = check_shape(B, H, Nkv, d)) return st;
    if (int st = check_attention_shape(B, H, Nq, Nkv)) return st;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16))
        return MXATTN_ERR_ALIGN;
    {
        const size_t ob = (size_t)(B * H * Nq * d * 2), kb = (size_t)(B * H * Nkv * d * 2);
        if (overlaps(out, ob, q, ob) || overlaps(out, ob, k, kb) || overlaps(out, ob, v, kb))
            return MXATTN_ERR_SHAPE;
    }
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);

    // Q is quantized in the attention kernel's prologue (bit-identical to the
    // head-dim quantizer), except for the rotated mode, whose Q is rotated
    // across all 128 channels first by its own quantizer
    const bool q_fused = mode != MXATTN_UOS_PNQ_ROT;
    const size_t q_codes = q_fused ? 0 : mxattn_codes_bytes(MXATTN_AXIS_HEAD_DIM, B, H, Nq, d);
    const size_t q_scales = q_fused ? 0 : mxattn_scales_bytes(MXATTN_AXIS_HEAD_DIM, B, H, Nq, d);
    const size_t k_codes = mxattn_codes_bytes(MXATTN_AXIS_HEAD_DIM, B, H, Nkv, d);
    const int64_t ntiles = (Nkv + mxattn::kKvTile - 1) / mxattn::kKvTile;
    const size_t v_codes = (size_t)(B * H * ntiles * 128 * mxattn::v_tile_row_bytes(Nkv));
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    const size_t tiled = (size_t)mxattn::tile_scales_bytes(B * H, Nkv);
    const size_t split = mxattn::split_bytes(B * H, Nq, mxattn::key_splits(B * H, Nq, Nkv));
    const size_t total = up(q_codes) + up(k_codes) + up(v_codes) + up(q_scales) + up(tiled) + split;

    Workspace ws;
    if (int st = ws.take(total, s)) return st;
    uint8_t* p = ws.get();
    uint8_t* qc = p;
    p += up(q_codes);
    uint8_t* kc = p;
    p += up(k_codes);
    uint8_t* vc = p;
    p += up(v_codes);
    uint8_t* qs = p;
    p += up(q_scales);
    uint8_t* sc = p;

    mxattn::PrepareArgs a{};
    a.q = q_fused ? nullptr : static_cast<const uint4*>(q);
    a.k = static_cast<const uint4*>(k);
    a.v = static_cast<const uint4*>(v);
    a.qc = qc;
    a.qs = qs;
    a.kc = kc;
    a.vc = vc;
    a.sc = sc;
    a.BH = B * H;
    a.N = (int)Nkv;
    a.Nq = (int)Nq;
    a.ntiles = (int)ntiles;
    a.vrow = mxattn::v_tile_row_bytes(Nkv);
    int st = MXATTN_OK;
    if (hipError_t e = mxattn::launch_prepare_operands(a, rule_of(mode), !q_fused, s)) {
        set_error("quantize launch", e);
        st = MXATTN_ERR_HIP;
    } else {
        st = launch_attend(q_fused ? q : nullptr, qc, qs, kc, vc, true, sc, sc + up(tiled), out, B, H, Nq, Nkv, mode, s);
    }
    return ws.give_back(st);
}

int mxattn_forward(const void* q, const void* k, const void* v, void* out, int64_t B, int64_t H,
                   int64_t N, int64_t d, int mode, void* stream) {
    return mxattn_cross_forward(q, k, v, out, B, H, N, N, d, mode, stream);
}

// ---- norm and rotation, and the paged cache

// The last byte + 1 of rows [B, H, N, 128] of bf16 by strides, from their start.
static size_t span_bytes(int64_t B, int64_t H, int64_t N, const int64_t* s) {
    return (size_t)(((B - 1) * s[0] + (H - 1) * s[1] + (N - 1) * s[2] + 128) * 2);
}

static int check_strides(const int64_t* s) {
    for (int i = 0; i < 3; i++) {
        if (s[i] < 0 || s[i] > (int64_t)1 << 36) return MXATTN_ERR_SHAPE;
        if (s[i] % 8 != 0) return MXATTN_ERR_ALIGN;
    }
    return MXATTN_OK;
}

// Whether rows of 128 elements by these strides lie apart from one another: each
// axis steps over all that the axes of smaller stride span.
static bool rows_apart(int64_t B, int64_t H, int64_t N, const int64_t* s) {
    int64_t extent[3] = {B, H, N}, stride[3] = {s[0], s[1], s[2]};
    int64_t span = 128;
    for (int i = 0; i < 3; i++) {
        int least = -1;
        for (int j = 0; j < 3; j++)
            if (extent[j] > 1 && (least < 0 || stride[j] < stride[least])) least = j;
        if (least < 0) return true;
        if (stride[least] < span) return false;
        span += (extent[least] - 1) * stride[least];
        extent[least] = 1;
    }
    return true;
}

static int check_transform(const float* w0, const float* w1, float eps, const float* cos, const float* sin,
                           const int32_t* positions, int64_t table_rows, int64_t rot, int pairs) {
    if (rot < 0 || rot > 128 || rot % 16 != 0) return MXATTN_ERR_VALUE;
    if (pairs != MXATTN_PAIRS_INTERLEAVED && pairs != MXATTN_PAIRS_HALVES) return MXATTN_ERR_VALUE;
    if ((w0 || w1) && !(eps >= 0.0f && eps <= 3.0e38f)) return MXATTN_ERR_VALUE;
    if (rot > 0) {
        if (!cos || !sin) return MXATTN_ERR_NULL;
        if (table_rows < 1 || table_rows > (int64_t)1 << 31) return MXATTN_ERR_SHAPE;
        if (!aligned(cos, 16) || !aligned(sin, 16)) return MXATTN_ERR_ALIGN;
    }
    if (!aligned(w0, 16) || !aligned(w1, 16) || !aligned(positions, 4)) return MXATTN_ERR_ALIGN;
    return MXATTN_OK;
}

int mxattn_qk_norm_rope(const void* q, const void* k, void* q_out, void* k_out, int64_t B, int64_t Hq, int64_t Hkv,
                        int64_t N, int64_t d, const int64_t* q_strides, const int64_t* k_strides,
                        const int64_t* q_out_strides, const int64_t* k_out_strides, const float* q_weight,
                        const float* k_weight, float eps, const float* cos, const float* sin,
                        const int32_t* positions, int64_t table_rows, int64_t rot, int pairs, void* stream) {
    if (!q || !q_out || (k == nullptr) != (k_out == nullptr)) return MXATTN_ERR_NULL;
    if (int st = check_shape(B, Hq, N, d)) return st;
    if (k)
        if (int st = check_shape(B, Hkv, N, d)) return st;
    if (Hq > 65535 || (k && Hkv > 65535)) return MXATTN_ERR_SHAPE;
    if (int st = check_transform(q_weight, k ? k_weight : nullptr, eps, cos, sin, positions, table_rows, rot, pairs))
        return st;
    const int64_t heads[2] = {Hq, k ? Hkv : 0};
    const void* in[2] = {q, k};
    void* out[2] = {q_out, k_out};
    const int64_t* given[4] = {q_strides, k_strides, q_out_strides, k_out_strides};
    int64_t strides[4][3];
    mxattn::RopeArgs a{};
    for (int i = 0; i < 4; i++) {
        const int64_t H = heads[i & 1];
        if (!H) continue;
        const int64_t whole[3] = {H * N * 128, N * 128, 128};
        for (int j = 0; j < 3; j++) strides[i][j] = given[i] ? given[i][j] : whole[j];
        if (int st = check_strides(strides[i])) return st;
    }
    for (int i = 0; i < 2 && heads[i]; i++) {
        if (!aligned(in[i], 16) || !aligned(out[i], 16)) return MXATTN_ERR_ALIGN;
        if (!rows_apart(B, heads[i], N, strides[2 + i])) return MXATTN_ERR_SHAPE;
        const size_t bytes = span_bytes(B, heads[i], N, strides[2 + i]);
        for (int j = 0; j < 2 && heads[j]; j++) {
            if (overlaps(out[i], bytes, in[j], span_bytes(B, heads[j], N, strides[j]))) return MXATTN_ERR_SHAPE;
            if (j > i && overlaps(out[i], bytes, out[j], span_bytes(B, heads[j], N, strides[2 + j])))
                return MXATTN_ERR_SHAPE;
        }
        a.in[i] = {static_cast<uint16_t*>(const_cast<void*>(in[i])), strides[i][0], strides[i][1], strides[i][2]};
        a.out[i] = {static_cast<uint16_t*>(out[i]), strides[2 + i][0], strides[2 + i][1], strides[2 + i][2]};
    }
    a.w[0] = q_weight;
    a.w[1] = k_weight;
    a.t = {cos, sin, table_rows, eps, (int)rot};
    a.positions = positions;
    a.tokens = B * N;
    a.N = (int)N;
    a.Hq = (int)Hq;
    a.Hkv = (int)heads[1];
    hipError_t e = mxattn::launch_qk_norm_rope(a, pairs == MXATTN_PAIRS_HALVES, reinterpret_cast<hipStream_t>(stream));
    if (e != hipSuccess) {
        set_error("norm and rotation launch", e);
        return MXATTN_ERR_HIP;
    }
    return MXATTN_OK;
}

// The sizes of a batch over the paged cache.
static int check_batch(int64_t seqs, int64_t max_pages, int64_t page_tokens, int64_t tokens, int64_t Hkv) {
    if (int st = check_shape(1, Hkv, tokens, mxattn::kHeadDim)) return st;
    if (Hkv > 65535 || seqs < 1 || seqs > 1 << 20) return MXATTN_ERR_SHAPE;
    return max_pages < 1 || max_pages > mxattn::kMaxKeys / page_tokens ? MXATTN_ERR_SHAPE : MXATTN_OK;
}

// Query heads that read the cache's; a launch has a workgroup of 256 threads for every
// number of a tile of at least 32 rows and KV head, and holds 2^32 threads.
static int check_query_heads(int64_t seqs, int64_t tokens, int64_t Hq, int64_t Hkv) {
    if (int st = check_shape(1, Hq, tokens, mxattn::kHeadDim)) return st;
    if (Hq % Hkv != 0 || Hq / Hkv > 256) return MXATTN_ERR_VALUE;
    return (tokens * (Hq / Hkv) / 32 + seqs) * Hkv >> 24 ? MXATTN_ERR_SHAPE : MXATTN_OK;
}

// The sizes of a cache's pages and of a batch over it; fills c.
static int check_pages(mxattn::CacheArgs& c, int64_t pages, int64_t page_tokens, const int32_t* page_table, int64_t seqs,
                       int64_t max_pages, int64_t tokens, int64_t Hkv) {
    if (page_tokens < 32 || page_tokens > 4096 || (page_tokens & (page_tokens - 1)) != 0) return MXATTN_ERR_VALUE;
    const int64_t bpp = page_tokens / 32;
    if (int st = check_batch(seqs, max_pages, page_tokens, tokens, Hkv)) return st;
    if (pages < 1 || pages > (int64_t)1 << 30 || pages * bpp > ((int64_t)1 << 40) / Hkv) return MXATTN_ERR_SHAPE;
    if (!aligned(page_table, 4)) return MXATTN_ERR_ALIGN;
    c.page_table = page_table;
    c.seqs = (int)seqs;
    c.tokens = (int)tokens;
    c.heads = (int)Hkv;
    c.pages = (int)pages;
    c.max_pages = (int)max_pages;
    c.bpp_log2 = __builtin_ctzll((unsigned long long)bpp);
    return MXATTN_OK;
}

static int check_codes(mxattn::CacheArgs& c, const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* v_codes,
                       const uint8_t* v_scales) {
    if (!aligned(k_codes, 16) || !aligned(v_codes, 16)) return MXATTN_ERR_ALIGN;
    c.kc = const_cast<uint8_t*>(k_codes);
    c.vc = const_cast<uint8_t*>(v_codes);
    c.ks = const_cast<uint8_t*>(k_scales);
    c.vs = const_cast<uint8_t*>(v_scales);
    return MXATTN_OK;
}

// The checks that the calls on the paged cache share; fills c.
static int check_cache(mxattn::CacheArgs& c, const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* v_codes,
                       const uint8_t* v_scales, int64_t pages, int64_t page_tokens, const int32_t* page_table,
                       const int32_t* q_start, const int32_t* kv_len, int64_t seqs, int64_t max_pages, int64_t tokens,
                       int64_t Hkv, int64_t d) {
    if (!k_codes || !k_scales || !v_codes || !v_scales || !page_table || !q_start || !kv_len) return MXATTN_ERR_NULL;
    if (int st = check_shape(1, 1, 1, d)) return st;
    if (int st = check_pages(c, pages, page_tokens, page_table, seqs, max_pages, tokens, Hkv)) return st;
    if (int st = check_codes(c, k_codes, k_scales, v_codes, v_scales)) return st;
    if (!aligned(q_start, 4) || !aligned(kv_len, 4)) return MXATTN_ERR_ALIGN;
    c.q_start = q_start;
    c.kv_len = kv_len;
    return MXATTN_OK;
}

// Whether `bytes` at p share a byte with the cache.
static bool in_cache(const void* p, size_t bytes, const mxattn::CacheArgs& c) {
    const size_t blocks = ((size_t)c.pages * (size_t)c.heads) << c.bpp_log2;
    return overlaps(p, bytes, c.kc, blocks * mxattn::kBlockBytes) || overlaps(p, bytes, c.vc, blocks * mxattn::kBlockBytes) ||
           overlaps(p, bytes, c.ks, blocks) || overlaps(p, bytes, c.vs, blocks);
}

// The bytes of `tokens` rows of `heads` heads, and the checks of their stride.
static int check_rows(const void* p, int64_t stride, int64_t tokens, int64_t heads, bool apart, size_t& bytes) {
    if (stride < (apart && tokens > 1 ? heads * 128 : 0) || stride > (int64_t)1 << 32) return MXATTN_ERR_SHAPE;
    if (!aligned(p, 16) || stride % 8 != 0) return MXATTN_ERR_ALIGN;
    bytes = (size_t)(((tokens - 1) * stride + heads * 128) * 2);
    return MXATTN_OK;
}

int mxattn_cache_append(const void* k, const void* v, int64_t k_stride, int64_t v_stride, uint8_t* k_codes,
                        uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, int64_t pages, int64_t page_tokens,
                        const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len, int64_t seqs,
                        int64_t max_pages, int64_t tokens, int64_t Hkv, int64_t d, const float* k_weight, float eps,
                        const float* cos, const float* sin, const int32_t* positions, int64_t table_rows, int64_t rot,
                        int pairs, void* stream) {
    if (!k || !v) return MXATTN_ERR_NULL;
    mxattn::AppendArgs a{};
    if (int st = check_cache(a.c, k_codes, k_scales, v_codes, v_scales, pages, page_tokens, page_table, q_start, kv_len,
                             seqs, max_pages, tokens, Hkv, d))
        return st;
    if (int st = check_transform(k_weight, nullptr, eps, cos, sin, positions, table_rows, rot, pairs)) return st;
    size_t kb = 0, vb = 0;
    if (int st = check_rows(k, k_stride, tokens, Hkv, false, kb)) return st;
    if (int st = check_rows(v, v_stride, tokens, Hkv, false, vb)) return st;
    if (in_cache(k, kb, a.c) || in_cache(v, vb, a.c)) return MXATTN_ERR_SHAPE;
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.w = k_weight;
    a.t = {cos, sin, table_rows, eps, (int)rot};
    a.positions = positions;
    hipError_t e = mxattn::launch_cache_append(a, pairs == MXATTN_PAIRS_HALVES, reinterpret_cast<hipStream_t>(stream));
    if (e != hipSuccess) {
        set_error("cache append launch", e);
        return MXATTN_ERR_HIP;
    }
    return MXATTN_OK;
}

// The caller's bounds on a sequence's new tokens and keys, as far as it gives any.
static void attend_bounds(int64_t& max_q, int64_t& max_kv, int64_t tokens, int64_t reach) {
    if (max_kv == 0 || max_kv > reach) max_kv = reach;
    if (max_q == 0 || max_q > tokens) max_q = tokens;
}

// The sizes of a call of attention over the cache, without its memory; false where it is refused.
static bool sized_attend(mxattn::CacheAttendArgs& a, int64_t page_tokens, int64_t seqs, int64_t max_pages, int64_t tokens,
                         int64_t Hq, int64_t Hkv, int64_t& max_q, int64_t& max_kv) {
    if (page_tokens < 32 || page_tokens > 4096 || (page_tokens & (page_tokens - 1)) != 0 || max_q < 0 || max_kv < 0 ||
        check_batch(seqs, max_pages, page_tokens, tokens, Hkv) || check_query_heads(seqs, tokens, Hq, Hkv))
        return false;
    a.c.seqs = (int)seqs;
    a.c.tokens = (int)tokens;
    a.c.heads = (int)Hkv;
    a.group = (int)(Hq / Hkv);
    attend_bounds(max_q, max_kv, tokens, max_pages * page_tokens);
    return true;
}

size_t mxattn_cache_attend_workspace(int64_t page_tokens, int64_t seqs, int64_t max_pages, int64_t tokens, int64_t Hq,
                                     int64_t Hkv, int64_t max_q, int64_t max_kv) {
    mxattn::CacheAttendArgs a{};
    if (!sized_attend(a, page_tokens, seqs, max_pages, tokens, Hq, Hkv, max_q, max_kv)) return 0;
    return mxattn::cache_attend_workspace(a, max_q, max_kv);
}

size_t mxattn_cache_attend_weights_workspace(int64_t page_tokens, int64_t seqs, int64_t max_pages, int64_t tokens,
                                             int64_t Hq, int64_t Hkv, int64_t max_q, int64_t max_kv) {
    mxattn::CacheWeighArgs w{};
    if (!sized_attend(w.a, page_tokens, seqs, max_pages, tokens, Hq, Hkv, max_q, max_kv)) return 0;
    return mxattn::cache_weigh_workspace(w, max_q, max_kv);
}

// The arguments that the calls of attention over the cache share.
struct AttendCall {
    const char* name;
    const void* q;
    int64_t q_stride;
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    int64_t pages, page_tokens;
    const int32_t *page_table, *q_start, *kv_len;
    int64_t seqs, max_pages, tokens, Hq, Hkv, d;
    int causal;
    int64_t max_q, max_kv;
    void* out;
    int64_t out_stride;
    void* workspace;
    size_t workspace_bytes;
    hipStream_t stream;
    size_t q_bytes, out_bytes;  // set by check_attend
};

// The checks that they share; fills a.
static int check_attend(AttendCall& x, mxattn::CacheAttendArgs& a) {
    if (!x.q || !x.out) return MXATTN_ERR_NULL;
    if (int st = check_cache(a.c, x.k_codes, x.k_scales, x.v_codes, x.v_scales, x.pages, x.page_tokens, x.page_table,
                             x.q_start, x.kv_len, x.seqs, x.max_pages, x.tokens, x.Hkv, x.d))
        return st;
    if (int st = check_query_heads(x.seqs, x.tokens, x.Hq, x.Hkv)) return st;
    if (x.max_q < 0 || x.max_kv < 0) return MXATTN_ERR_SHAPE;
    if (int st = check_rows(x.q, x.q_stride, x.tokens, x.Hq, false, x.q_bytes)) return st;
    if (int st = check_rows(x.out, x.out_stride, x.tokens, x.Hq, true, x.out_bytes)) return st;
    if (overlaps(x.out, x.out_bytes, x.q, x.q_bytes) || in_cache(x.out, x.out_bytes, a.c)) return MXATTN_ERR_SHAPE;
    a.q = static_cast<const uint16_t*>(x.q);
    a.out = static_cast<uint16_t*>(x.out);
    a.q_stride = x.q_stride;
    a.out_stride = x.out_stride;
    a.group = (int)(x.Hq / x.Hkv);
    a.per_group = (((uint64_t)1 << 36) + a.group - 1) / a.group;
    a.causal = x.causal != 0;
    a.scale = 0.12751743082459868f;  // fp32(log2(e) / sqrt(128))
    attend_bounds(x.max_q, x.max_kv, x.tokens, x.max_pages * x.page_tokens);
    return MXATTN_OK;
}

extern "C++" {  // (templates)
// Runs `launch(workspace)` of the call `name` with `bytes` of workspace: the caller's, which must be as large and clash
// with nothing (`clash(from, bytes)`), or the library's where it gives none.
template <class Clash, class Launch>
static int run_with(const char* name, void* workspace, size_t workspace_bytes, size_t bytes, hipStream_t stream,
                    const char* what, Clash clash, Launch launch) {
    uint8_t* memory = nullptr;
    Workspace ws;
    if (bytes && workspace) {
        if (workspace_bytes < bytes) {
            std::snprintf(g_last_error, sizeof g_last_error, "%s: %zu bytes of workspace needed, the caller's has %zu", name,
                          bytes, workspace_bytes);
            return MXATTN_ERR_SCRATCH;
        }
        if (!aligned(workspace, 16)) return MXATTN_ERR_ALIGN;
        if (clash(workspace, bytes)) return MXATTN_ERR_SHAPE;
        memory = static_cast<uint8_t*>(workspace);
        bytes = 0;
    } else if (bytes) {
        // an allocation of the pool is not recorded into a graph: its replays need memory that lasts
        hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
        if (stream) {
            if (hipError_t e = hipStreamIsCapturing(stream, &capture)) {
                set_error("hipStreamIsCapturing", e);
                return MXATTN_ERR_HIP;
            }
        }
        if (capture != hipStreamCaptureStatusNone) {
            std::snprintf(g_last_error, sizeof g_last_error,
                          "%s: %zu bytes of workspace needed from the caller, as the stream is being captured", name, bytes);
            return MXATTN_ERR_SCRATCH;
        }
        if (int st = ws.take(bytes, stream)) return st;
        memory = ws.get();
    }
    int st = MXATTN_OK;
    hipError_t e = launch(memory);
    if (e != hipSuccess) {
        set_error(what, e);
        st = MXATTN_ERR_HIP;
    }
    return bytes ? ws.give_back(st) : st;
}

template <class Launch>
static int run_attend(const AttendCall& x, const mxattn::CacheArgs& c, size_t bytes, Launch launch) {
    return run_with(
        x.name, x.workspace, x.workspace_bytes, bytes, x.stream, "cache attention launch",
        [&](const void* p, size_t n) {
            return overlaps(p, n, x.q, x.q_bytes) || overlaps(p, n, x.out, x.out_bytes) || in_cache(p, n, c);
        },
        launch);
}
}  // extern "C++"

static int run_plain_attend(AttendCall& x, mxattn::CacheAttendArgs& a) {
    return run_attend(x, a.c, mxattn::cache_attend_workspace(a, x.max_q, x.max_kv), [&](uint8_t* memory) {
        a.workspace = memory;
        return mxattn::launch_cache_attend(a, x.max_q, x.max_kv, x.stream);
    });
}

int mxattn_cache_attend(const void* q, int64_t q_stride, const uint8_t* k_codes, const uint8_t* k_scales,
                        const uint8_t* v_codes, const uint8_t* v_scales, int64_t pages, int64_t page_tokens,
                        const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len, int64_t seqs,
                        int64_t max_pages, int64_t tokens, int64_t Hq, int64_t Hkv, int64_t d, int causal,
                        int64_t max_q, int64_t max_kv, void* out, int64_t out_stride, void* workspace,
                        size_t workspace_bytes, void* stream) {
    AttendCall x{"mxattn_cache_attend", q, q_stride, k_codes, k_scales, v_codes, v_scales, pages, page_tokens, page_table,
                 q_start, kv_len, seqs, max_pages, tokens, Hq, Hkv, d, causal, max_q, max_kv, out, out_stride, workspace,
                 workspace_bytes, reinterpret_cast<hipStream_t>(stream), 0, 0};
    mxattn::CacheAttendArgs a{};
    if (int st = check_attend(x, a)) return st;
    return run_plain_attend(x, a);
}

int mxattn_cache_attend_window(const void* q, int64_t q_stride, const uint8_t* k_codes, const uint8_t* k_scales,
                               const uint8_t* v_codes, const uint8_t* v_scales, int64_t pages, int64_t page_tokens,
                               const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len, int64_t seqs,
                               int64_t max_pages, int64_t tokens, int64_t Hq, int64_t Hkv, int64_t d, int64_t window,
                               int64_t sinks, int causal, int64_t max_q, int64_t max_kv, void* out, int64_t out_stride,
                               void* workspace, size_t workspace_bytes, void* stream) {
    AttendCall x{"mxattn_cache_attend_window", q, q_stride, k_codes, k_scales, v_codes, v_scales, pages, page_tokens,
                 page_table, q_start, kv_len, seqs, max_pages, tokens, Hq, Hkv, d, causal, max_q, max_kv, out, out_stride,
                 workspace, workspace_bytes, reinterpret_cast<hipStream_t>(stream), 0, 0};
    mxattn::CacheAttendArgs a{};
    if (int st = check_attend(x, a)) return st;
    if (window < 1 || sinks < 0) return MXATTN_ERR_VALUE;
    a.kind = mxattn::kWindow;
    a.window = (int)std::min(window, mxattn::kMaxKeys);  // (no sequence is longer)
    a.sinks = (int)std::min(sinks, mxattn::kMaxKeys);
    return run_plain_attend(x, a);
}

int mxattn_cache_attend_tree(const void* q, int64_t q_stride, const uint8_t* k_codes, const uint8_t* k_scales,
                             const uint8_t* v_codes, const uint8_t* v_scales, int64_t pages, int64_t page_tokens,
                             const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len, int64_t seqs,
                             int64_t max_pages, int64_t tokens, int64_t Hq, int64_t Hkv, int64_t d, const int32_t* tree,
                             int64_t tree_words, int64_t max_q, int64_t max_kv, void* out, int64_t out_stride,
                             void* workspace, size_t workspace_bytes, void* stream) {
    AttendCall x{"mxattn_cache_attend_tree", q, q_stride, k_codes, k_scales, v_codes, v_scales, pages, page_tokens,
                 page_table, q_start, kv_len, seqs, max_pages, tokens, Hq, Hkv, d, 0, max_q, max_kv, out, out_stride,
                 workspace, workspace_bytes, reinterpret_cast<hipStream_t>(stream), 0, 0};
    if (!tree) return MXATTN_ERR_NULL;
    mxattn::CacheAttendArgs a{};
    if (int st = check_attend(x, a)) return st;
    if (tree_words < 1 || tree_words > mxattn::kMaxKeys / 32) return MXATTN_ERR_SHAPE;
    if (!aligned(tree, 4)) return MXATTN_ERR_ALIGN;
    const size_t tb = (size_t)tokens * (size_t)tree_words * 4;
    if (overlaps(out, x.out_bytes, tree, tb)) return MXATTN_ERR_SHAPE;
    a.kind = mxattn::kTree;
    a.tree = tree;
    a.tree_words = (int)tree_words;
    const size_t bytes = mxattn::cache_attend_workspace(a, x.max_q, x.max_kv);
    if (workspace && bytes && overlaps(workspace, bytes, tree, tb)) return MXATTN_ERR_SHAPE;
    return run_plain_attend(x, a);
}

// Bytes of weights beside a cache.
static size_t weights_bytes(const mxattn::CacheArgs& c) {
    return (((size_t)c.pages * (size_t)c.heads) << c.bpp_log2) * mxattn::kBlockTokens * sizeof(float);
}

int mxattn_cache_attend_weights(const void* q, int64_t q_stride, const uint8_t* k_codes, const uint8_t* k_scales,
                                const uint8_t* v_codes, const uint8_t* v_scales, int64_t pages, int64_t page_tokens,
                                const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len, int64_t seqs,
                                int64_t max_pages, int64_t tokens, int64_t Hq, int64_t Hkv, int64_t d, const float* weights,
                                float* weights_out, int causal, int64_t max_q, int64_t max_kv, void* out,
                                int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream) {
    AttendCall x{"mxattn_cache_attend_weights", q, q_stride, k_codes, k_scales, v_codes, v_scales, pages, page_tokens,
                 page_table, q_start, kv_len, seqs, max_pages, tokens, Hq, Hkv, d, causal, max_q, max_kv, out, out_stride,
                 workspace, workspace_bytes, reinterpret_cast<hipStream_t>(stream), 0, 0};
    if (!weights_out) return MXATTN_ERR_NULL;
    mxattn::CacheWeighArgs w{};
    if (int st = check_attend(x, w.a)) return st;
    if (!aligned(weights, 4) || !aligned(weights_out, 4)) return MXATTN_ERR_ALIGN;
    const size_t wb = weights_bytes(w.a.c);
    if (overlaps(weights_out, wb, q, x.q_bytes) || overlaps(weights_out, wb, out, x.out_bytes) ||
        in_cache(weights_out, wb, w.a.c) || (weights && overlaps(weights, wb, out, x.out_bytes)) ||
        (weights && weights != weights_out && overlaps(weights_out, wb, weights, wb)))
        return MXATTN_ERR_SHAPE;
    const size_t bytes = mxattn::cache_weigh_workspace(w, x.max_q, x.max_kv);
    if (workspace && (overlaps(workspace, bytes, weights_out, wb) || (weights && overlaps(workspace, bytes, weights, wb))))
        return MXATTN_ERR_SHAPE;
    w.before = weights;
    w.after = weights_out;
    return run_attend(x, w.a.c, bytes, [&](uint8_t* memory) {
        w.a.workspace = memory;
        return mxattn::launch_cache_weigh(w, x.max_q, x.max_kv, x.stream);
    });
}

// A launch has up to 1024 threads for every sequence and KV head, and holds 2^32.
static int check_items(int64_t seqs, int64_t Hkv) { return seqs * Hkv >> 22 ? MXATTN_ERR_SHAPE : MXATTN_OK; }

int mxattn_cache_select(const float* weights, int64_t pages, int64_t page_tokens, const int32_t* page_table,
                        const int32_t* kv_len, int64_t seqs, int64_t max_pages, int64_t Hkv, int64_t budget, int64_t sinks,
                        int64_t recent, int32_t* kept, int32_t* counts, void* workspace, size_t workspace_bytes,
                        void* stream) {
    if (!weights || !page_table || !kv_len || !kept || !counts) return MXATTN_ERR_NULL;
    mxattn::SelectArgs a{};
    if (int st = check_pages(a.c, pages, page_tokens, page_table, seqs, max_pages, 1, Hkv)) return st;
    if (int st = check_items(seqs, Hkv)) return st;
    if (budget < 1 || budget > mxattn::kMaxKeys || sinks < 0 || recent < 0 || sinks > budget || recent > budget - sinks)
        return MXATTN_ERR_VALUE;
    if (!aligned(weights, 4) || !aligned(kv_len, 4) || !aligned(kept, 4) || !aligned(counts, 4)) return MXATTN_ERR_ALIGN;
    const size_t kb = (size_t)seqs * (size_t)Hkv * (size_t)budget * 4, cb = (size_t)seqs * 4, wb = weights_bytes(a.c);
    const size_t tb = (size_t)seqs * (size_t)max_pages * 4;
    if (overlaps(kept, kb, weights, wb) || overlaps(kept, kb, counts, cb) || overlaps(kept, kb, kv_len, cb) ||
        overlaps(kept, kb, page_table, tb) || overlaps(counts, cb, weights, wb) || overlaps(counts, cb, kv_len, cb) ||
        overlaps(counts, cb, page_table, tb))
        return MXATTN_ERR_SHAPE;
    a.c.kv_len = kv_len;
    a.weights = weights;
    a.budget = (int)budget;
    a.sinks = (int)sinks;
    a.recent = (int)recent;
    a.kept = kept;
    a.counts = counts;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return run_with(
        "mxattn_cache_select", workspace, workspace_bytes, mxattn::cache_select_workspace(seqs * Hkv, max_pages * page_tokens),
        st, "cache selection launch",
        [&](const void* p, size_t n) {
            return overlaps(p, n, weights, wb) || overlaps(p, n, kept, kb) || overlaps(p, n, counts, cb) ||
                   overlaps(p, n, kv_len, cb) || overlaps(p, n, page_table, tb);
        },
        [&](uint8_t* memory) {
            a.workspace = memory;
            return mxattn::launch_cache_select(a, st);
        });
}

size_t mxattn_cache_select_workspace(int64_t page_tokens, int64_t seqs, int64_t max_pages, int64_t Hkv) {
    if (page_tokens < 32 || page_tokens > 4096 || (page_tokens & (page_tokens - 1)) != 0 ||
        check_batch(seqs, max_pages, page_tokens, 1, Hkv) || check_items(seqs, Hkv))
        return 0;
    return mxattn::cache_select_workspace(seqs * Hkv, max_pages * page_tokens);
}

int mxattn_cache_compact(uint8_t* k_codes, uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, int64_t pages,
                         int64_t page_tokens, const int32_t* page_table, int64_t seqs, int64_t max_pages,
                         const int32_t* out_table, int64_t out_pages, int64_t Hkv, int64_t d, const int32_t* kept,
                         int64_t kept_heads, int64_t width, const int32_t* counts, const int32_t* base, float* weights,
                         void* stream) {
    if (!k_codes || !k_scales || !v_codes || !v_scales || !page_table || !kept || !counts) return MXATTN_ERR_NULL;
    mxattn::CompactArgs a{};
    if (int st = check_shape(1, 1, 1, d)) return st;
    if (int st = check_pages(a.c, pages, page_tokens, page_table, seqs, max_pages, 1, Hkv)) return st;
    if (int st = check_items(seqs, Hkv)) return st;
    if (out_table && (out_pages < 1 || out_pages > mxattn::kMaxKeys / page_tokens)) return MXATTN_ERR_SHAPE;
    if (out_table == page_table && out_pages != max_pages) return MXATTN_ERR_SHAPE;
    if ((kept_heads != 1 && kept_heads != Hkv) || width < 1 || width > mxattn::kMaxKeys) return MXATTN_ERR_SHAPE;
    if (int st = check_codes(a.c, k_codes, k_scales, v_codes, v_scales)) return st;
    if (!aligned(out_table, 4) || !aligned(kept, 4) || !aligned(counts, 4) || !aligned(base, 4) || !aligned(weights, 4))
        return MXATTN_ERR_ALIGN;
    const size_t wb = weights_bytes(a.c);
    if (weights && in_cache(weights, wb, a.c)) return MXATTN_ERR_SHAPE;
    a.in_place = !out_table || out_table == page_table;
    a.out_table = out_table ? out_table : page_table;
    a.out_pages = (int)(out_table ? out_pages : max_pages);
    a.kept = kept;
    a.kept_head = kept_heads == 1 ? 0 : width;
    a.kept_seq = kept_heads * width;
    a.width = (int)width;
    a.counts = counts;
    a.base = base;
    a.weights = weights;
    hipError_t e = mxattn::launch_cache_compact(a, reinterpret_cast<hipStream_t>(stream));
    if (e != hipSuccess) {
        set_error("cache compaction launch", e);
        return MXATTN_ERR_HIP;
    }
    return MXATTN_OK;
}

}  // extern "C"
