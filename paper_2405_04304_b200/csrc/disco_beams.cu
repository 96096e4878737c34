// Host side of the 8-bit LM head and of beam search: argument checks and launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <memory>
#include <new>

#include "disco.h"
#include "context.cuh"
#include "int8_head.cuh"
#include "beam.cuh"

using namespace disco;

namespace disco {

int set_beam_wait_budget(long long clocks) {
    return cudaMemcpyToSymbol(g_wait_budget_clocks, &clocks, sizeof(clocks)) == cudaSuccess ? DISCO_OK : DISCO_ERR_CUDA;
}

}  // namespace disco

namespace {

int type_size(int type) {
    switch (type) {
        case DISCO_F32: return 4;
        case DISCO_BF16: case DISCO_F16: return 2;
        default: return 0;
    }
}

bool aligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(to - 1)) == 0; }

// The calls launch on the current device, with scratch on the context's.
bool on_its_device(const disco_ctx* c) {
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == c->device;
}

// int8 [rows, d], rows `pitch` bytes apart, boxes of box_rows x 128, 128-byte swizzle, zero fill out of bounds
bool encode_int8_2d(const disco_ctx* c, CUtensorMap* map, const void* base, int rows, int d, long long pitch, int box_rows) {
    if (!c->encode_tiled) return false;
    const cuuint64_t gdim[2] = {(cuuint64_t)d, (cuuint64_t)rows};
    const cuuint64_t gstride[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {(cuuint32_t)kI8BK, (cuuint32_t)box_rows};
    const cuuint32_t estride[2] = {1, 1};
    return reinterpret_cast<EncodeTiledFn>(c->encode_tiled)(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), gdim, gstride,
                                                            box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T>
int launch_quantize(disco_ctx* c, QuantParams p, cudaStream_t st) {
    void (*kern)(QuantParams);
    int threads = kQuantThreads, ctas = p.rows;
    if (p.rows >= 2048) {
        // A head: a warp to a narrow row, four to a wide one (32000 x 768 / 40011 x 1000 / 32000 x 5120: 20 / 30 / 105 us; four warps to a narrow
        // row 34 / 45, sixteen to a wide one 171).
        if (p.d <= 2048) ctas = (p.rows + 3) / 4;
        kern = p.d <= 1024   ? quantize_rows_kernel<T, 4, 1>
               : p.d <= 2048 ? quantize_rows_kernel<T, 8, 1>
               : p.d <= 6144 ? quantize_rows_kernel<T, 6, 4>
                             : quantize_rows_kernel<T, 16, 4>;
    } else {
        // Hidden rows, which a product waits for: two chunks to a thread at most while the warps of a CTA go round (us a pass of 64 / 128 / 256
        // rows of a 32000 x 5120 head, four warps -> sixteen: 32.4 / 36.4 / 48.1 -> 31.6 / 34.8 / 45.0).
        threads = p.d <= 2048 ? 128 : p.d <= 4096 ? 256 : 512;
        kern = p.d <= 1024   ? quantize_rows_kernel<T, 1, 4>
               : p.d <= 2048 ? quantize_rows_kernel<T, 2, 4>
               : p.d <= 4096 ? quantize_rows_kernel<T, 2, 8>
               : p.d <= 8192 ? quantize_rows_kernel<T, 2, 16>
                             : quantize_rows_kernel<T, 4, 16>;
        // Many of them would be read behind the head's first tiles, which the product's CTAs request as soon as they may start (us a pass of 256 /
        // 320 / 384 / 448 / 512 / 600 / 704 rows of 32000 x 5120, early -> late: 44.8 / 57.8 / 67.3 / 73.4 / 80.7 / 97.5 / 111.1 -> 44.9 / 57.6 / 65.5 /
        // 68.5 / 80.6 / 98.4 / 109.9).
        p.late = p.rows >= 512;
    }
    const cudaError_t e = launch_after(c, kern, dim3((unsigned)ctas), dim3((unsigned)threads), 0, st, p);
    c->launches += 1;
    return cuda_ok(e, "quantize_rows_kernel launch") ? DISCO_OK : DISCO_ERR_CUDA;
}

int quantize(disco_ctx* c, const void* x, int x_type, long long ldx, int rows, int d, int8_t* q, long long ldq, float* scale, cudaStream_t st) {
    const QuantParams p{x, ldx, rows, d, q, ldq, scale, 0};
    switch (x_type) {
        case DISCO_F32: return launch_quantize<float>(c, p, st);
        case DISCO_BF16: return launch_quantize<__nv_bfloat16>(c, p, st);
        default: return launch_quantize<__half>(c, p, st);
    }
}

// Rows that quantize_rows_kernel reads 16 bytes at a time.
int check_rows(const void* x, int x_type, long long ldx, int rows, int d) {
    if (!x || type_size(x_type) == 0 || rows < 1 || d < 8 || d % 8 || ldx < d) return DISCO_ERR_INVALID_ARG;
    if (!aligned16(x) || (ldx * type_size(x_type)) % 16) return DISCO_ERR_INVALID_ARG;
    return DISCO_OK;
}

int check_head(const disco_ctx* c, const int8_t* W_q, long long ldw, const float* w_scale, int d) {
    if (!W_q || !w_scale || !aligned16(W_q) || !aligned(w_scale, 4)) return DISCO_ERR_INVALID_ARG;
    if (ldw < d || ldw % 16) return DISCO_ERR_INVALID_ARG;
    return d > std::max(c->d_draft, c->d_target) ? DISCO_ERR_WORKSPACE : DISCO_OK;
}

// The product of hidden rows that are in 8 bits already (In = void), or of a few rows of type In.
template <typename Out, typename In, bool STATS, bool PAIR>
int launch_int8_head(disco_ctx* c, const Int8Tiling& t, const int8_t* W_q, long long ldw, const float* w_scale, const void* x, long long ldx,
                     int d, int R, void* y, long long ldy, cudaStream_t st) {
    constexpr bool FEW = !std::is_void<In>::value;
    Int8Params p{};
    p.V = c->V;
    p.d = d;
    p.R = R;
    p.t = t;
    p.w_scale = w_scale;
    p.x_scale = c->int8_scale;
    p.x = x;
    p.ldx = ldx;
    p.y = y;
    p.ldy = ldy;
    p.stats = STATS ? c->beam_stats : nullptr;
    p.chunks = BeamLayout(c->V).i8_chunks;
    p.withhold = c->test_stamp_skew != 0;
    p.status = c->status;
    auto kern = int8_head_kernel<Out, In, STATS, PAIR>;
    static KernelSetup setup;
    size_t limit = 0;
    if (!raise_smem_limit(c, setup, kern, 0, &limit)) return DISCO_ERR_CUDA;
    constexpr int kTurn = STATS ? kI8TurnBytes : 0;
    p.ring = Int8Ring::make(p.t, d, (long long)limit - kTurn, FEW);
    if (p.ring.stages == 0) return DISCO_ERR_UNSUPPORTED_SHAPE;
    CUtensorMap tmap_W, tmap_X{};
    if (!encode_int8_2d(c, &tmap_W, W_q, c->V, d, ldw, p.t.w_box)) return DISCO_ERR_CUDA;
    if (!FEW && !encode_int8_2d(c, &tmap_X, c->int8_rows, R, d, c->int8_pitch, p.t.x_box)) return DISCO_ERR_CUDA;
    const int items = p.t.MT * p.t.NV;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(PAIR ? 2 * std::min(items, c->sm_count / 2) : std::min(items, c->sm_count)));
    cfg.blockDim = dim3(kI8Threads);
    cfg.dynamicSmemBytes = (size_t)(kI8FixedSmem + p.ring.bytes + p.ring.resident + kTurn);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    cfg.numAttrs = launch_attributes(c, PAIR ? 2 : 1, attr);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, tmap_W, tmap_X, p);
    c->launches += 1;
    return cuda_ok(e, "int8_head_kernel launch") ? DISCO_OK : DISCO_ERR_CUDA;
}

// Logits of R hidden rows (and, STATS, their soft-max statistics by chunks).
template <typename Out, bool STATS>
int project(disco_ctx* c, const int8_t* W_q, long long ldw, const float* w_scale, const void* H, int h_type, long long ldh, int d, int R, void* y,
            long long ldy, cudaStream_t st) {
    const Int8Tiling t = Int8Tiling::choose(R, c->V, d, c->sm_count);
    if (Int8Ring::few(R, c->V, d)) {
        switch (h_type) {
            case DISCO_F32: return launch_int8_head<Out, float, STATS, false>(c, t, W_q, ldw, w_scale, H, ldh, d, R, y, ldy, st);
            case DISCO_BF16: return launch_int8_head<Out, __nv_bfloat16, STATS, false>(c, t, W_q, ldw, w_scale, H, ldh, d, R, y, ldy, st);
            default: return launch_int8_head<Out, __half, STATS, false>(c, t, W_q, ldw, w_scale, H, ldh, d, R, y, ldy, st);
        }
    }
    const int rc = quantize(c, H, h_type, ldh, R, d, c->int8_rows, c->int8_pitch, c->int8_scale, st);
    if (rc) return rc;
    return t.kind == kI8Pair ? launch_int8_head<Out, void, STATS, true>(c, t, W_q, ldw, w_scale, nullptr, 0, d, R, y, ldy, st)
                             : launch_int8_head<Out, void, STATS, false>(c, t, W_q, ldw, w_scale, nullptr, 0, d, R, y, ldy, st);
}

int check_beams(const disco_ctx* c, int B, int K, int n, const float* score, const uint8_t* finished, int eos, const float* score_out,
                const int32_t* parent, const int32_t* token, const uint8_t* finished_out) {
    if (!score || !score_out || !parent || !token || B < 1 || K < 1 || n < 1) return DISCO_ERR_INVALID_ARG;
    if (K > DISCO_MAX_BEAMS || n > DISCO_MAX_KEPT || c->V > kBeamMaxVocab) return DISCO_ERR_UNSUPPORTED_SHAPE;
    if (finished ? eos < 0 : eos < -1) return DISCO_ERR_INVALID_ARG;
    if (eos >= c->V) return DISCO_ERR_INVALID_ARG;
    if (!aligned(score, 4) || !aligned(score_out, 4) || !aligned(parent, 4) || !aligned(token, 4)) return DISCO_ERR_INVALID_ARG;
    // the outputs may take the inputs' place where they are of one shape
    if (n != K && ((const void*)score == (const void*)score_out || (finished && finished == finished_out))) return DISCO_ERR_INVALID_ARG;
    if ((long long)B * K > c->part_rows) return DISCO_ERR_WORKSPACE;
    return DISCO_OK;
}

BeamParams beam_params(const disco_ctx* c, const void* z, long long ld, int chunk, int B, int K, int n, const float* score,
                       const uint8_t* finished, int eos, float* score_out, int32_t* parent, int32_t* token, uint8_t* finished_out) {
    BeamParams p{};
    p.z = z;
    p.ld = ld;
    p.V = c->V;
    p.B = B;
    p.K = K;
    p.n = n;
    p.eos = eos;
    p.score = score;
    p.finished = finished;
    const BeamLayout layout(c->V);
    p.chunks = chunk == kBeamChunk ? layout.chunks : layout.i8_chunks;
    p.segs = layout.segs;
    p.pairs = c->beam_stats;
    p.sums = c->beam_stats;
    p.tops = reinterpret_cast<float*>(c->beam_stats) + layout.tops_at((size_t)B * K);
    p.score_out = score_out;
    p.parent = parent;
    p.token = token;
    p.finished_out = finished_out;
    return p;
}

template <typename T, int CHUNK, bool JOINED>
int launch_beam_select(disco_ctx* c, BeamParams p, cudaStream_t st) {
    int warps = BeamDeal::warps(p.K, p.chunks, p.n);
    if (JOINED && warps == 8 && p.K * p.segs > 8 * kBeamCluster) warps = 16;      // (a warp to each segment)
    p.deal = BeamDeal::make(p.K, p.chunks, warps);
    const int lanes = 32 * p.deal.share;
    p.ln_err = beam_ln_err(CHUNK == kBeamChunk ? (p.segs + lanes - 1) / lanes : p.deal.merged);
    // Sixteen warps to a sequence: no register goes to memory where a CTA has an SM to itself (us a pass, two by two -> one: 64 x 8 of 49152 27.6 ->
    // 27.1, 20 x 5 of 40011 bf16 12.8 -> 12.0); two by two where there are more CTAs than SMs (160 x 4 on a head of 32000 x 768, one -> two 48.7 ->
    // 45.4) or, in clusters, half as many, since a GPC's SMs are no multiple of a cluster's CTAs (16 / 32 x 4 of 32000 11.1 / 14.8 -> 9.8 / 11.9).
    const bool few = p.B * (JOINED ? 2 * kBeamCluster : 1) <= c->sm_count;
    auto kern = warps == 8    ? beam_select_kernel<T, CHUNK, 256, false, JOINED>
                : warps == 16 ? (few ? beam_select_kernel<T, CHUNK, 512, false, JOINED> : beam_select_kernel<T, CHUNK, 512, false, JOINED, 2>)
                : p.deal.two  ? beam_select_kernel<T, CHUNK, 1024, true, JOINED>
                              : beam_select_kernel<T, CHUNK, 1024, false, JOINED>;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)p.B * (JOINED ? kBeamCluster : 1));
    cfg.blockDim = dim3((unsigned)(32 * warps));
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    cfg.numAttrs = launch_attributes(c, JOINED ? kBeamCluster : 1, attr);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p);
    c->launches += 1;
    return cuda_ok(e, "beam_select_kernel launch") ? DISCO_OK : DISCO_ERR_CUDA;
}

template <typename T>
int select_beams(disco_ctx* c, const BeamParams& p, cudaStream_t st) {
    if (beam_joined(p.B, p.K, p.segs)) return launch_beam_select<T, kBeamChunk, true>(c, p, st);
    const long long warps = (long long)p.B * p.K * p.segs;
    const long long ctas = (warps + kBeamStatWarps - 1) / kBeamStatWarps;
    if (ctas > 0x7fffffffll) return DISCO_ERR_UNSUPPORTED_SHAPE;
    const cudaError_t e = launch_after(c, beam_stats_kernel<T>, dim3((unsigned)ctas), dim3(kBeamStatWarps * 32), 0, st, p);
    c->launches += 1;
    if (!cuda_ok(e, "beam_stats_kernel launch")) return DISCO_ERR_CUDA;
    return launch_beam_select<T, kBeamChunk, false>(c, p, st);
}

template <typename Word, int N>
int launch_reorder(disco_ctx* c, ReorderParams& p, int tensors, cudaStream_t st) {
    const long long tiles = (p.T * p.unit + kReorderThreads - 1) / kReorderThreads;
    if (tiles * p.B * p.mid > 0x7fffffffll) return DISCO_ERR_UNSUPPORTED_SHAPE;
    p.tiles = (int)tiles;
    const cudaError_t e = launch_after(c, beam_reorder_kernel<Word, N>, dim3((unsigned)(tiles * p.B * p.mid), (unsigned)tensors),
                                       dim3(kReorderThreads), 0, st, p);
    c->launches += 1;
    return cuda_ok(e, "beam_reorder_kernel launch") ? DISCO_OK : DISCO_ERR_CUDA;
}

// What is written lies apart from all else that is written, and (unless in place) read: a state that is there twice would be reordered
// twice at once.
int check_apart(const void* const* src, size_t src_bytes, void* const* dst, size_t dst_bytes, int tensors, bool in_place) {
    auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    if (tensors == 1) {
        const uintptr_t s = at(src[0]), d = at(dst[0]);
        return !in_place && s < d + dst_bytes && d < s + src_bytes ? DISCO_ERR_INVALID_ARG : DISCO_OK;
    }
    const std::unique_ptr<uintptr_t[]> held(new (std::nothrow) uintptr_t[tensors]);
    uintptr_t *first = held.get(), *last = first + tensors;
    if (!first) return DISCO_ERR_WORKSPACE;
    std::transform(dst, dst + tensors, first, at);
    std::sort(first, last);
    for (const uintptr_t* d = first; d + 1 < last; ++d)
        if (d[1] - d[0] < dst_bytes) return DISCO_ERR_INVALID_ARG;
    for (int i = 0; !in_place && i < tensors; ++i) {
        const uintptr_t s = at(src[i]);
        const uintptr_t* d = std::upper_bound(first, last, s);       // the first one behind, and the one before it
        if (d < last && *d - s < src_bytes) return DISCO_ERR_INVALID_ARG;
        if (d > first && s - d[-1] < dst_bytes) return DISCO_ERR_INVALID_ARG;
    }
    return DISCO_OK;
}

// Words of `size` bytes; in place a thread holds its words of all rows at once.
int launch_reorder_words(disco_ctx* c, ReorderParams& p, int size, int tensors, cudaStream_t st) {
    const bool many = p.in_place && p.n > 16;
    switch (size) {
        case 16: return p.n <= 4   ? launch_reorder<uint4, 4>(c, p, tensors, st)
                        : p.n <= 8 ? launch_reorder<uint4, 8>(c, p, tensors, st)
                                   : launch_reorder<uint4, 16>(c, p, tensors, st);
        case 8: return many ? launch_reorder<uint2, 32>(c, p, tensors, st) : launch_reorder<uint2, 16>(c, p, tensors, st);
        case 4: return many ? launch_reorder<uint32_t, 64>(c, p, tensors, st) : launch_reorder<uint32_t, 16>(c, p, tensors, st);
        case 2: return many ? launch_reorder<uint16_t, 64>(c, p, tensors, st) : launch_reorder<uint16_t, 16>(c, p, tensors, st);
        default: return many ? launch_reorder<uint8_t, 64>(c, p, tensors, st) : launch_reorder<uint8_t, 16>(c, p, tensors, st);
    }
}

}  // namespace

extern "C" {

int disco_quantize_rows(disco_ctx* c, const void* x, int x_type, long long ldx, int rows, int d, int8_t* q, long long ldq, float* scale,
                        void* stream) {
    if (!c) return DISCO_ERR_INVALID_ARG;
    const int rc = check_rows(x, x_type, ldx, rows, d);
    if (rc) return rc;
    if (!q || !scale || !aligned16(q) || !aligned(scale, 4) || ldq < d || ldq % 16) return DISCO_ERR_INVALID_ARG;
    if (d > kMaxHidden) return DISCO_ERR_UNSUPPORTED_SHAPE;
    if (!on_its_device(c)) return DISCO_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    c->last_stream = st;
    return quantize(c, x, x_type, ldx, rows, d, q, ldq, scale, st);
}

int disco_project_int8(disco_ctx* c, const int8_t* W_q, long long ldw, const float* w_scale, const void* H, int h_type, long long ldh, int d,
                       int R, void* y, int y_type, long long ldy, void* stream) {
    if (!c) return DISCO_ERR_INVALID_ARG;
    int rc = check_rows(H, h_type, ldh, R, d);
    if (rc) return rc;
    rc = check_head(c, W_q, ldw, w_scale, d);
    if (rc) return rc;
    if (!y || type_size(y_type) == 0 || !aligned(y, type_size(y_type)) || ldy < c->V) return DISCO_ERR_INVALID_ARG;
    if (R > c->part_rows) return DISCO_ERR_WORKSPACE;
    if (!on_its_device(c)) return DISCO_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    c->last_stream = st;
    switch (y_type) {
        case DISCO_F32: return project<float, false>(c, W_q, ldw, w_scale, H, h_type, ldh, d, R, y, ldy, st);
        case DISCO_BF16: return project<__nv_bfloat16, false>(c, W_q, ldw, w_scale, H, h_type, ldh, d, R, y, ldy, st);
        default: return project<__half, false>(c, W_q, ldw, w_scale, H, h_type, ldh, d, R, y, ldy, st);
    }
}

int disco_beam_select(disco_ctx* c, const void* logits, int z_type, long long ldz, int B, int K, const float* score, const uint8_t* finished,
                      int eos, int n, float* score_out, int32_t* parent, int32_t* token, uint8_t* finished_out, void* stream) {
    if (!c || !logits || type_size(z_type) == 0 || !aligned(logits, type_size(z_type)) || ldz < c->V) return DISCO_ERR_INVALID_ARG;
    const int rc = check_beams(c, B, K, n, score, finished, eos, score_out, parent, token, finished_out);
    if (rc) return rc;
    if (!on_its_device(c)) return DISCO_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    c->last_stream = st;
    const BeamParams p = beam_params(c, logits, ldz, kBeamChunk, B, K, n, score, finished, eos, score_out, parent, token, finished_out);
    switch (z_type) {
        case DISCO_F32: return select_beams<float>(c, p, st);
        case DISCO_BF16: return select_beams<__nv_bfloat16>(c, p, st);
        default: return select_beams<__half>(c, p, st);
    }
}

int disco_beam_step_int8(disco_ctx* c, const int8_t* W_q, long long ldw, const float* w_scale, const void* H, int h_type, long long ldh,
                         int d, int B, int K, const float* score, const uint8_t* finished, int eos, int n, float* score_out,
                         int32_t* parent, int32_t* token, uint8_t* finished_out, float* work, void* stream) {
    if (!c || !work || !aligned16(work)) return DISCO_ERR_INVALID_ARG;
    int rc = check_beams(c, B, K, n, score, finished, eos, score_out, parent, token, finished_out);
    if (rc) return rc;
    const int R = B * K;
    rc = check_rows(H, h_type, ldh, R, d);
    if (rc) return rc;
    rc = check_head(c, W_q, ldw, w_scale, d);
    if (rc) return rc;
    if (!on_its_device(c)) return DISCO_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    c->last_stream = st;
    rc = project<float, true>(c, W_q, ldw, w_scale, H, h_type, ldh, d, R, work, c->V, st);
    if (rc) return rc;
    const BeamParams p = beam_params(c, work, c->V, kI8Chunk, B, K, n, score, finished, eos, score_out, parent, token, finished_out);
    return launch_beam_select<float, kI8Chunk, false>(c, p, st);
}

int disco_beam_reorder(disco_ctx* c, const void* const* src, void* const* dst, int tensors, int B, int K, int n, const int32_t* parent,
                       const int32_t* lens, long long mid, long long T, long long unit_bytes, void* stream) {
    if (!c || !src || !dst || !parent || tensors < 1 || B < 1 || K < 1 || n < 1 || mid < 1 || T < 1 || unit_bytes < 1) return DISCO_ERR_INVALID_ARG;
    if (K > DISCO_MAX_BEAMS || n > DISCO_MAX_KEPT) return DISCO_ERR_UNSUPPORTED_SHAPE;
    if (!aligned(parent, 4) || !aligned(lens, 4)) return DISCO_ERR_INVALID_ARG;
    // (no state is larger than this, and what follows multiplies sizes)
    constexpr long long kMost = 1ll << 46;
    if (mid > kMost / T || unit_bytes > kMost / (mid * T) || (long long)B * std::max(K, n) > kMost / (mid * T * unit_bytes)) return DISCO_ERR_INVALID_ARG;
    const size_t row = (size_t)mid * T * unit_bytes, src_bytes = row * B * K, dst_bytes = row * B * n;
    if (!lens) {   // whole rows
        T *= mid;
        mid = 1;
    }
    const bool in_place = src[0] == dst[0];
    if (in_place && n != K) return DISCO_ERR_INVALID_ARG;
    uintptr_t low = (uintptr_t)(lens ? unit_bytes : T * unit_bytes);
    for (int i = 0; i < tensors; ++i) {
        if (!src[i] || !dst[i] || (src[i] == dst[i]) != in_place) return DISCO_ERR_INVALID_ARG;
        low |= reinterpret_cast<uintptr_t>(src[i]) | reinterpret_cast<uintptr_t>(dst[i]);
    }
    const int rc = check_apart(src, src_bytes, dst, dst_bytes, tensors, in_place);
    if (rc) return rc;
    if (!on_its_device(c)) return DISCO_ERR_INVALID_ARG;
    // the widest word that divides everything; in place fewer bytes where a thread has to hold many rows' words
    int size = low & 1 ? 1 : low & 2 ? 2 : low & 4 ? 4 : low & 8 ? 8 : 16;
    if (in_place && n > 16) size = std::min(size, n > 32 ? 4 : 8);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    c->last_stream = st;
    for (int i0 = 0; i0 < tensors; i0 += kReorderTensors) {
        const int count = std::min(kReorderTensors, tensors - i0);
        ReorderParams p{};
        for (int i = 0; i < count; ++i) p.src[i] = src[i0 + i], p.dst[i] = dst[i0 + i];
        p.B = B;
        p.K = K;
        p.n = n;
        p.parent = parent;
        p.lens = lens;
        p.mid = mid;
        p.T = T;
        p.unit = unit_bytes / size;
        if (!lens) p.T = 1, p.unit = T * unit_bytes / size;
        p.in_place = in_place;
        p.status = c->status;
        const int rc = launch_reorder_words(c, p, size, count, st);
        if (rc) return rc;
    }
    return DISCO_OK;
}

}  // extern "C"
