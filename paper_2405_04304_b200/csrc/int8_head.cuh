// An LM head in 8-bit integers, with a scale for each hidden row and each vocabulary row:
//
//   s_x[r] = max_k |x[r, k]| / 127,   q_x[r, k] = rint(127 x[r, k] / max_k |x[r, k]|)
//   y[r, v] = (sum_k q_x[r, k] q_w[v, k]) * s_x[r] * s_w[v]
//
// The sums are exact in 32-bit integers (at most 127 * 127 * 16384 = 2.6e8); a logit sees three roundings to fp32, in this order:
// the sum, times s_x, times s_w.
#pragma once

#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "umma_ptx.cuh"

namespace disco {

// ---------------------------------------------------------------------------------------------
// rows to 8 bits
// ---------------------------------------------------------------------------------------------
constexpr int kQuantThreads = 128;

// 127 x / top to the nearest integer, ties to even, with 0 < top < inf, |x| <= top.  The product with the reciprocal is off by less
// than 127 * 2^-22; only where it comes nearer to the middle between two integers than that is the quotient itself needed.
//   * bf16 and fp16: 127/128 x is exact (7 + 11 bits).  The quotient by `top` is correctly rounded, hence never on the other side
//     of a tie (2k + 1) / 256, and it is on the tie only if the exact one is: 254 x and (2k + 1) top are multiples of the last place
//     of x, at most 254 * 2^11 of them, so they differ by 2^-19 of their size or not at all.
//   * fp32: the same in 64 bits (127 x is exact there, and 254 * 2^24 is well below 2^53).
template <typename T>
__device__ __noinline__ int quantize_exactly(float x, float top) {
    if constexpr (sizeof(T) == 2) return __float2int_rn(__fdiv_rn(x * 0.9921875f, top) * 128.f);
    else return __double2int_rn(__ddiv_rn(127.0 * static_cast<double>(x), static_cast<double>(top)));
}

// The largest |x| of a row by its bits (whose order is that of the numbers; what is not finite comes above all else), and what follows from it.
struct RowScale {
    float top, inv, shift, scale;     // inv = 0: a row of zeros, or one that holds a number that is not finite
    __device__ __forceinline__ explicit RowScale(uint32_t top_bits) {
        const bool finite = top_bits < 0x7f800000u;
        top = __uint_as_float(top_bits);
        scale = finite ? __fdiv_rn(top, 127.f) : __uint_as_float(0x7fc00000u);
        // numbers near the smallest ones are shifted up, which is exact
        shift = top < 0x1p-60f ? 0x1p100f : 1.f;
        top *= shift;
        inv = finite && top > 0.f ? 127.f / top : 0.f;
    }
    // Eight numbers in 8 bits each: the sum with 1.5 * 2^23 leaves the nearest integer in its low bits.  (The rare quotient is a call: in line,
    // 64 times over, it made the kernels' code several times as long, and code that runs once per launch comes from L2.)
    template <typename T>
    __device__ __forceinline__ uint2 round(float (&f)[8]) const {
        constexpr float kWhole = 12582912.f;
        if (!(inv > 0.f)) return make_uint2(0u, 0u);
        if (shift != 1.f) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] *= shift;
        }
        float t[8];
        bool close = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            t[j] = fmaf(f[j], inv, kWhole);
            close = close || fabsf(fmaf(f[j], inv, kWhole - t[j])) >= 0.4995f;
        }
        if (close) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (fabsf(fmaf(f[j], inv, kWhole - t[j])) >= 0.4995f)
                    t[j] = __uint_as_float(__float_as_uint(kWhole) + static_cast<uint32_t>(quantize_exactly<T>(f[j], top)));
        }
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t a = __byte_perm(__float_as_uint(t[4 * h]), __float_as_uint(t[4 * h + 1]), 0x0040);
            const uint32_t b = __byte_perm(__float_as_uint(t[4 * h + 2]), __float_as_uint(t[4 * h + 3]), 0x0040);
            w[h] = __byte_perm(a, b, 0x5410);
        }
        return make_uint2(w[0], w[1]);
    }
};

// Eight consecutive numbers of a row.  (Not by the read-only path: the compiler may move such loads ahead of the wait for the kernel
// that wrote them.)
template <typename T>
struct QuantChunk;
template <>
struct QuantChunk<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldcg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void get(float (&f)[8]) const { unpack_bf16x8(v, f); }
};
template <>
struct QuantChunk<__half> {
    uint4 v;
    __device__ __forceinline__ void load(const __half* p) { v = __ldcg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = t.x;
            f[2 * i + 1] = t.y;
        }
    }
};
template <>
struct QuantChunk<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = __ldcg(reinterpret_cast<const float4*>(p));
        b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w;
        f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    }
};

struct QuantParams {
    const void* x;
    long long ldx;    // elements
    int rows, d;      // d: a multiple of 8
    int8_t* q;
    long long ldq;    // a multiple of 16; columns d .. round_up(d, 16) - 1 are written as zeros
    float* scale;
    int late;         // what comes next may start once the rows have been read, not before
};

// WPR warps to a row (all of a CTA, or one of four for many narrow rows); a thread keeps its share of the row (chunks of eight numbers, up to CH of
// them) in registers between the search for the largest number and the rounding, so that the row is read once.  A row that holds a number
// that is not finite gets the scale NaN.
template <typename T, int CH, int WPR>
__global__ void __launch_bounds__(WPR == 1 ? kQuantThreads : 32 * WPR) quantize_rows_kernel(const QuantParams p) {
    constexpr int kThreads = WPR == 1 ? kQuantThreads : 32 * WPR, kRows = kThreads / 32 / WPR;      // rows of a CTA
    __shared__ uint32_t s_top[kThreads / 32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // (not before the wait: what comes next may read the head ahead of its own, and the head may be what ran before this)
    if (!p.late) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const long long row = (long long)blockIdx.x * kRows + (threadIdx.x >> 5) / WPR;
    const bool mine = row < p.rows;
    const int thread = threadIdx.x % (32 * WPR);
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const int chunks = mine ? p.d >> 3 : 0;
    QuantChunk<T> c[CH];
    uint32_t top_bits = 0u;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int at = i * 32 * WPR + thread;
        if (at < chunks) c[i].load(x + 8 * at);
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (i * 32 * WPR + thread >= chunks) continue;
        float f[8];
        c[i].get(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) top_bits = max(top_bits, __float_as_uint(f[j]) & 0x7fffffffu);
    }
    top_bits = __reduce_max_sync(kFullMask, top_bits);
    if (p.late) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if constexpr (WPR > 1) {
        if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top_bits;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) top_bits = max(top_bits, s_top[i]);
    }
    if (!mine) return;
    const RowScale rs(top_bits);
    if (thread == 0) p.scale[row] = rs.scale;
    int8_t* q = p.q + row * p.ldq;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int at = i * 32 * WPR + thread;
        if (at < chunks) {
            float f[8];
            c[i].get(f);
            *reinterpret_cast<uint2*>(q + 8 * at) = rs.template round<T>(f);
        }
    }
    if ((p.d & 15) && thread == 0) *reinterpret_cast<uint2*>(q + p.d) = make_uint2(0u, 0u);
}

// ---------------------------------------------------------------------------------------------
// the product
// ---------------------------------------------------------------------------------------------
constexpr int kI8BK = 128;                // k elements per stage (one 128-byte swizzle span)
constexpr int kI8MaxStages = 24;
constexpr int kI8EpiWarps = 16;
constexpr int kI8Threads = (2 + kI8EpiWarps) * 32;
constexpr int kI8FewChunks = 4;           // of eight numbers, that a lane holds of a row which the kernel rounds itself
constexpr int kI8FixedSmem = 1024 /*align*/ + 512 /*barriers*/ + 2 * 256 * 4 /*scales of two tiles' hidden rows*/;

__host__ __device__ inline int round_up(int x, int to) { return (x + to - 1) / to * to; }

// How V vocabulary rows and R hidden rows are cut: MT tiles of N hidden rows (the columns of an accumulator) times NV tiles of TR
// vocabulary rows.  Item i is hidden tile i % MT of vocabulary tile i / MT; the workers take items in turn, so those that share a
// vocabulary tile run side by side and the head crosses HBM once.  TR is a multiple of 32: whole lines of y, whole chunks.
//   one    a CTA is a worker, TR <= 128: one block of TMEM lanes, two accumulators, the epilogue under the next item's products
//   two    TR <= 256, two blocks: fewer reads of the hidden rows; beyond 128 hidden rows one accumulator only
//   pair   two CTAs are a worker (cta_group::2), TR <= 256: half of the vocabulary rows lie in each, and half of the hidden rows that both
//          multiply by; two accumulators
enum Int8Kind { kI8One, kI8Two, kI8Pair };
struct Int8Tiling {
    int MT, N, NV, TR, blocks, cols, bufs;
    int w_box, x_box;      // rows of the boxes that a CTA loads
    Int8Kind kind;
    int rounds;            // items to a worker at most
    __host__ __device__ static Int8Tiling make(int R, int V, int grid, Int8Kind kind) {
        Int8Tiling t;
        const int ctas = kind == kI8Pair ? 2 : 1, most_rows = kind == kI8One ? 128 : 256;
        t.kind = kind;
        t.MT = (R + 255) / 256;
        t.N = round_up((R + t.MT - 1) / t.MT, 16 * ctas);
        t.MT = (R + t.N - 1) / t.N;
        // as few rounds of items as the largest tiles need, all items alike
        const int workers = grid / ctas;
        const long long items = (long long)t.MT * ((V + most_rows - 1) / most_rows);
        const long long rounds = (items + workers - 1) / workers;
        const long long most = rounds * workers / t.MT;
        const int nv = (int)(most < V ? (most > 1 ? most : 1) : V);
        t.TR = round_up((V + nv - 1) / nv, kI8Chunk * ctas);
        // (a tile of many hidden rows is worth reading for whole blocks only: 200 rows of 8000 x 2048 / 12000 x 5120, 55 / 82 -> 128
        // vocabulary rows to a CTA, 13.4 / 26.1 -> 12.7 / 23.9 us)
        if (R > 96 && rounds == 1 && t.TR < 128 * ctas) t.TR = 128 * ctas;
        if (t.TR > most_rows) t.TR = most_rows;
        t.NV = (V + t.TR - 1) / t.TR;
        t.rounds = (int)(((long long)t.MT * t.NV + workers - 1) / workers);
        t.blocks = t.TR > 128 && kind == kI8Two ? 2 : 1;
        t.cols = round_up(t.N, 32);
        t.bufs = 2 * t.blocks * t.cols <= 512 ? 2 : 1;
        t.w_box = t.TR / ctas;
        t.x_box = ctas == 2 ? t.N / 2 : (round_up(R, 8) < t.N ? round_up(R, 8) : t.N);
        return t;
    }
    // The kind, from passes of 11 to 320 rows of heads of 8000 x 2048 to 49152 x 2048 and 32000 x 5120 (us, one / two / pair):
    //   * up to 32 hidden rows the epilogue is short and HBM is the bound: two (32000 x 5120, 11 rows 30.6 / 30.3 / 32.8)
    //   * beyond, it pays to have it under the next item's products: one (32000 x 768, 64 / 200 / 300 rows 9.0 / 13.8 / 16.7, 9.0 / 15.3 / 17.8,
    //     10.9 / 15.5 / 21.1)
    //   * long contractions of many rows are bound by the operands' way from L2: pair (32000 x 5120, 128 / 200 / 256 / 320 rows 35.8 / 41.2 /
    //     51.8 / 63.3, 35.2 / 41.2 / 49.8 / 59.0, 35.2 / 42.3 / 47.4 / 55.1)
    // unless it leaves a CTA more vocabulary rows, rounds counted, by over 15 % (200 rows of 20000 x 3000: 2 x 96 for one and pair, 160 for
    // two: 27.2 / 24.1 / 24.6).
    __host__ __device__ int share() const { return rounds * w_box; }
    __host__ __device__ static Int8Tiling choose(int R, int V, int d, int grid) {
        const Int8Tiling two = make(R, V, grid, kI8Two);
        if (R <= 32) return two;
        const Int8Tiling one = make(R, V, grid, kI8One);
        const bool spread = 100 * one.share() > 115 * two.share();
        const Int8Tiling single = spread ? two : one;
        if (R <= 96 || d < 2048 || grid < 2) return single;
        const Int8Tiling pair = make(R, V, grid, kI8Pair);
        return 100 * pair.share() > 115 * single.share() ? single : pair;
    }
};

// Shared memory of the operand stages: `stages` boxes of vocabulary rows, then as many of hidden rows.  An MMA reads all 128 rows of
// a block and as many hidden rows as its item has columns: what lies behind the boxes (always inside the ring) only feeds accumulators
// that nobody reads.
struct Int8Ring {
    int stages, w_bytes, x_bytes, bytes;
    int resident;       // bytes behind the stages: all of the hidden rows (then x_bytes is 0)
    __host__ __device__ static int size(const Int8Ring& r, const Int8Tiling& t, int stages) {
        const int all = stages * (r.w_bytes + r.x_bytes), last = (stages - 1) * r.w_bytes + t.blocks * 128 * kI8BK;
        return round_up(all > last ? all : last, 1024);
    }
    // As many stages as fit `limit` bytes beside the fixed part; none if that is less than two.
    __host__ __device__ static Int8Ring make(const Int8Tiling& t, int d, long long limit, bool few) {
        Int8Ring r{};
        r.w_bytes = round_up(t.w_box * kI8BK, 1024);
        r.x_bytes = few ? 0 : round_up(t.x_box, 16) * kI8BK;      // (all that an MMA reads: N rows, or half of them in each CTA)
        r.resident = few ? (d + kI8BK - 1) / kI8BK * t.N * kI8BK : 0;
        int stages = kI8MaxStages;
        while (stages >= 2 && kI8FixedSmem + size(r, t, stages) + r.resident > limit) --stages;
        if (stages >= 2) r.stages = stages, r.bytes = size(r, t, stages);
        return r;
    }
    // Hidden rows that the kernel rounds itself, in every CTA (its epilogue's warps have nothing else to do meanwhile), rather than a kernel
    // before it: where a lane can hold its part of them, and there are few enough that their loads do not wait behind the head's.  (us a pass,
    // a kernel before -> in the kernel: 1 / 4 / 16 rows of 32000 x 768 9.2 / 9.2 / 9.2 -> 7.6 / 6.9 / 9.0; 1 / 4 / 8 of 32000 x 2048 15.6 / 15.7 /
    // 15.9 -> 14.3 / 14.9 / 16.9; 1 / 8 of 49152 x 1024 12.2 / 12.4 -> 11.7 / 12.4.)
    __host__ __device__ static bool few(int R, int V, int d) {
        if (R > kI8EpiWarps || d > 2048 || d > kI8EpiWarps / R * 256 * kI8FewChunks) return false;
        return R * d <= ((long long)V * d <= 32ll << 20 ? 16384 : 8192);
    }
};

struct Int8Params {
    int V, d, R;
    Int8Tiling t;
    Int8Ring ring;
    const float* w_scale;      // [V]
    const float* x_scale;      // [R]
    const void* x;             // FEW: the hidden rows themselves, ldx elements apart
    long long ldx;
    void* y;
    long long ldy;
    float2* stats;             // [R][chunks] (largest logit of the chunk, sum of exp(z - largest)), or null
    int chunks;
    int withhold;              // disco_test_hooks: no tile is loaded
    int* status;
};

__device__ __forceinline__ void tc_mma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tc_mma_i8_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Instruction descriptor: signed 8-bit x signed 8-bit -> signed 32-bit, both operands K-major, M = m, N = n.
__device__ __forceinline__ uint32_t umma_idesc_i8(int n, uint32_t m = 128) {
    return (2u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | ((m >> 4) << 24);
}
// The largest of a warp's numbers, NaN if one of them is.
__device__ __forceinline__ float warp_max_nan_f32(float x) {
    float m;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(x));
    return m;
}

__device__ __forceinline__ void store_logit(float* p, float z) { *p = z; }
__device__ __forceinline__ void store_logit(__nv_bfloat16* p, float z) { *p = __float2bfloat16_rn(z); }
__device__ __forceinline__ void store_logit(__half* p, float z) { *p = __float2half_rn(z); }

// exp(x - m) for many x and one m: 2^(c x - M) with c = log2 e and M = c m rounded, a single rounding; what M lost to its own rounding is
// made good once, in the sum.  (Two operations instead of three where they are what bounds the kernel.)  |m| < 2^24: M is then off by 1 at
// most, and the terms by a factor of 2.  (The loss grows with m: at 2^31 the terms would pass what fp32 holds.)
struct ExpFrom {
    static constexpr float c = 1.4426950408889634f;
    float M;
    __device__ __forceinline__ explicit ExpFrom(float m) : M(c * m) {}
    __device__ __forceinline__ float operator()(float x) const {
        float e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(x, c, -M)));
        return e;
    }
    __device__ __forceinline__ float sum(float s, float m) const { return s * exp2f(fmaf(-m, c, M)); }      // (M - c m, exactly)
    static __device__ __forceinline__ bool serves(float m) { return fabsf(m) < 0x1p24f; }
};

// Soft-max statistics of 32 vocabulary rows' logits, one per lane, of 16 hidden rows: the largest of each hidden row's (NaN if there is
// one that is not a number) and the sum of exp(z - largest).  By way of a corner turn in shared memory: two lanes to a hidden row, 16
// logits each.
// turn: 16 x kI8TurnStride floats of the warp.  Lane i and lane i + 16 return those of hidden row i.
constexpr int kI8TurnStride = 33;
constexpr int kI8TurnBytes = kI8EpiWarps * 16 * kI8TurnStride * 4;
__device__ __forceinline__ float max_nan(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ float2 warp_chunk_stats(const float* z, bool in, int lane, float* turn) {
#pragma unroll
    for (int i = 0; i < 16; ++i) turn[i * kI8TurnStride + lane] = in ? z[i] : DISCO_NEG_INF;
    __syncwarp();
    const float* mine = turn + (lane & 15) * kI8TurnStride + (lane & 16);
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = mine[j];
    __syncwarp();
    float m = x[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) m = max_nan(m, x[j]);
    m = max_nan(m, __shfl_xor_sync(kFullMask, m, 16));
    float e[4] = {0.f, 0.f, 0.f, 0.f};
    if (ExpFrom::serves(m)) {       // (by the hidden row's own logits alone: equal rows give equal sums whatever their neighbours are)
        const ExpFrom from(m);
#pragma unroll
        for (int j = 0; j < 16; ++j) e[j & 3] += from(x[j]);
        e[0] = from.sum((e[0] + e[1]) + (e[2] + e[3]), m);
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) e[j & 3] += __expf(x[j] - m);
        e[0] = (e[0] + e[1]) + (e[2] + e[3]);
    }
    return make_float2(m, e[0] + __shfl_xor_sync(kFullMask, e[0], 16));      // (NaN where the largest is not finite: nothing is done with it there)
}

// 32 lanes x 16 consecutive 32-bit columns -> 16 registers per thread
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, int (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}

// Vocabulary rows on the TMEM lanes, hidden rows on the columns: a warp's 32 results of a column are neighbours in y, so they go
// from registers to memory in whole lines, and the head, which is what HBM has to deliver, is cut as finely as there are SMs.
//   * warp 0    producer: a box of TR vocabulary rows x 128 k and one of the tile's hidden rows per stage
//   * warp 1    MMA issuer: M = 128 (twice for more than 128 vocabulary rows), N = hidden rows of the tile, K = 32
//   * warps 2+  epilogue: a thread owns a vocabulary row and walks over the hidden rows
// Where a wait runs out, producer and issuer stop, and leave once their loads and products in flight are done; the epilogue's warps go
// through their items all the same (their barriers need all of them), with results that mean nothing.
template <typename Out, typename In, bool STATS, bool PAIR>
__global__ void __launch_bounds__(kI8Threads, 1)
int8_head_kernel(const __grid_constant__ CUtensorMap tmap_W, const __grid_constant__ CUtensorMap tmap_X, const Int8Params p) {
    constexpr bool FEW = !std::is_void<In>::value;
    static_assert(!(FEW && PAIR), "");
    extern __shared__ uint8_t smem_dyn[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
    uint8_t* w_tiles = smem;
    uint8_t* x_tiles = FEW ? smem + p.ring.bytes : smem + p.ring.stages * p.ring.w_bytes;
    uint8_t* fixed = smem + p.ring.bytes + (FEW ? p.ring.resident : 0);
    uint64_t* full = reinterpret_cast<uint64_t*>(fixed);
    uint64_t* empty = full + kI8MaxStages;
    uint64_t* tmem_full = empty + kI8MaxStages;
    uint64_t* tmem_empty = tmem_full + 2;
    uint64_t* rows_full = tmem_empty + 2;
    uint64_t* done = rows_full + 1;        // all products
    uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(done + 1);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const Int8Tiling& t = p.t;
    const int KB = (p.d + kI8BK - 1) / kI8BK;
    const int items = t.MT * t.NV;
    const int rank = PAIR ? (int)cluster_rank() : 0;
    const bool leader = rank == 0;
    const int worker = PAIR ? (int)blockIdx.x >> 1 : (int)blockIdx.x, workers = PAIR ? (int)gridDim.x >> 1 : (int)gridDim.x;
    // columns of an item: the last tile of hidden rows has no more than its rows need (32000 x 5120, 704 rows in tiles of 256, 256 and 192:
    // 110.2 -> 107.5 us; 49152 x 3000, 600 rows in tiles of 224, 224 and 160: 97.0 -> 91.0)
    auto columns = [&](int item) { return min(t.N, round_up(p.R - item % t.MT * t.N, PAIR ? 32 : 16)); };

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.ring.stages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&tmem_full[b], 1);
            mbar_init(&tmem_empty[b], PAIR ? 2 * kI8EpiWarps : kI8EpiWarps);
        }
        mbar_init(rows_full, kI8EpiWarps);
        mbar_init(done, 1);
        fence_mbar_init();
        prefetch_tensormap(&tmap_W);
        if (!FEW) prefetch_tensormap(&tmap_X);
    }
    if (warp == 1) {
        if constexpr (PAIR) {
            tmem_alloc_pair(tmem_base_s, 512);
        } else {
            tmem_alloc(tmem_base_s, 512);
            tmem_relinquish();
        }
    }
    tc_fence_before();
    if constexpr (PAIR) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_base_s;

    if (warp == 0) {
        // ------------------------------ producer ------------------------------
        if (elect_one()) {
            const uint32_t full0 = smem_addr(full), empty0 = smem_addr(empty), w0 = smem_addr(w_tiles), x0 = smem_addr(x_tiles);
            // (a pair's loads are counted on the leader's barriers)
            const uint32_t count0 = PAIR ? leader_addr(full0) : full0, expected = (PAIR ? 2 : 1) * (uint32_t)(t.w_box + (FEW ? 0 : t.x_box)) * 128u;
            const int k_end = KB * kI8BK, v_own = rank * t.w_box;
            // (the second CTA of a pair holds the second half of the item's columns, whatever the height of its box)
            auto first_row = [&](int item) { return item % t.MT * t.N + rank * (columns(item) / 2); };
            auto load = [&](uint32_t dst, const CUtensorMap* map, int c0, int c1, int slot) {
                if constexpr (PAIR) tma_load_2d_pair(dst, map, c0, c1, count0 + slot * 8);
                else tma_load_2d(dst, map, c0, c1, count0 + slot * 8);
            };
            int item = worker;
            // The head is complete before the kernel that rounds the hidden rows lets this one start: its first tiles are
            // requested at once, the hidden rows of the same stages behind the wait for that kernel.
            // (FEW: what ran before this may have written the head.)
            if (FEW) asm volatile("griddepcontrol.wait;" ::: "memory");
            const int end = p.withhold ? 0 : items;
            const int pre = item < end ? min(p.ring.stages, KB) : 0;
            for (int n = 0; n < pre; ++n) {
                if (leader) mbar_arrive_expect_tx(full0 + n * 8, expected);
                load(w0 + n * p.ring.w_bytes, &tmap_W, n * kI8BK, item / t.MT * t.TR + v_own, n);
            }
            if (!FEW) asm volatile("griddepcontrol.wait;" ::: "memory");
            asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
            for (int n = 0; !FEW && n < pre; ++n) load(x0 + n * p.ring.x_bytes, &tmap_X, n * kI8BK, first_row(item), n);
            int stage = pre == p.ring.stages ? 0 : pre, phase = pre == p.ring.stages ? 1 : 0;
            int k = pre * kI8BK;
            bool ok = true;
            for (; ok && item < end; item += workers, k = 0) {
                const int v0 = item / t.MT * t.TR + v_own, r0 = first_row(item);
                for (; k < k_end; k += kI8BK) {
                    ok = mbar_wait(empty0 + stage * 8, phase ^ 1, p.status);
                    if (!ok) break;
                    if (leader) mbar_arrive_expect_tx(full0 + stage * 8, expected);
                    load(w0 + stage * p.ring.w_bytes, &tmap_W, k, v0, stage);
                    if (!FEW) load(x0 + stage * p.ring.x_bytes, &tmap_X, k, r0, stage);
                    if (++stage == p.ring.stages) stage = 0, phase ^= 1;
                }
            }
            if constexpr (PAIR) {   // the leader's arrivals at this CTA's barriers are all in before it leaves
                int s = stage, ph = phase;
                for (int n = 0; n < p.ring.stages; ++n) {
                    ok = mbar_wait(empty0 + s * 8, ph ^ 1, p.status) && ok;
                    if (++s == p.ring.stages) s = 0, ph ^= 1;
                }
            }
            // The last load of each slot is in.  (A slot without one passes: its barrier is in its first phase, and the phase before that is
            // what is asked for.  Those of a pair's second CTA are counted at the leader, which waits for both; where the two have not got
            // equally far, nothing counts them, and only then there is a pause of a millisecond instead.)
            const long long t0 = clock64();
            for (int s = 0; leader && s < p.ring.stages; ++s) mbar_drain(full0 + s * 8, s < stage ? phase : phase ^ 1, t0, p.status);
            if constexpr (PAIR) {
                while (!ok && clock64() - t0 < 2000000) {}
                if (!leader) mbar_drain(smem_addr(done), 0, t0, p.status);
            }
        }
    } else if (warp == 1) {
        // ------------------------------ MMA issuer ------------------------------
        if (leader && elect_one()) {
            uint32_t idesc = 0u;     // (the item's)
            auto mma = [&](uint32_t d, uint64_t w, uint64_t x, uint32_t accumulate) {
                if constexpr (PAIR) tc_mma_i8_pair(d, w, x, idesc, accumulate);
                else tc_mma_i8(d, w, x, idesc, accumulate);
            };
            auto commit = [&](uint32_t bar) {
                if constexpr (PAIR) tc_commit_pair(bar);
                else tc_commit(bar);
            };
            const uint32_t full0 = smem_addr(full), empty0 = smem_addr(empty);
            const uint64_t w_desc0 = umma_smem_desc(w_tiles), x_desc0 = umma_smem_desc(x_tiles);
            const uint32_t w_step = (uint32_t)p.ring.w_bytes >> 4, x_step = (FEW ? (uint32_t)t.N * kI8BK : (uint32_t)p.ring.x_bytes) >> 4;   // descriptor units
            uint64_t w_desc = w_desc0, x_desc = x_desc0;
            int stage = 0, phase = 0, it = 0;
            bool ok = true;
            if (FEW) {
                ok = mbar_wait(rows_full, 0, p.status);
                tc_fence_after();
            }
            for (int item = worker; ok && item < items; item += workers, ++it) {
                if (FEW) x_desc = x_desc0;
                const int b = t.bufs == 2 ? it & 1 : 0;
                const uint32_t parity = ((t.bufs == 2 ? it >> 1 : it) & 1) ^ 1;
                if constexpr (PAIR) ok = mbar_wait_cluster(smem_addr(&tmem_empty[b]), parity, p.status);
                else ok = mbar_wait(&tmem_empty[b], parity, p.status);
                if (!ok) break;
                tc_fence_after();
                idesc = umma_idesc_i8(columns(item), PAIR ? 256 : 128);
                const uint32_t d_tmem = tmem_base + b * t.blocks * t.cols;
                for (int kb = 0; kb < KB; ++kb) {
                    ok = mbar_wait(full0 + stage * 8, phase, p.status);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 4; ++k)       // 32 k elements = 32 bytes = 2 descriptor units
                        mma(d_tmem, w_desc + 2 * k, x_desc + 2 * k, (kb | k) != 0);
                    if (!PAIR && t.blocks == 2) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)   // 128 vocabulary rows further on
                            mma(d_tmem + t.cols, w_desc + (128 * 128 >> 4) + 2 * k, x_desc + 2 * k, (kb | k) != 0);
                    }
                    commit(empty0 + stage * 8);
                    w_desc += w_step;
                    x_desc += x_step;
                    if (++stage == p.ring.stages) {
                        stage = 0, phase ^= 1, w_desc = w_desc0;
                        if (!FEW) x_desc = x_desc0;
                    }
                }
                if (ok) commit(smem_addr(&tmem_full[b]));
            }
            commit(smem_addr(done));
            mbar_drain(smem_addr(done), 0, clock64(), p.status);
        }
    } else {
        // ------------------------------ epilogue ------------------------------
        asm volatile("griddepcontrol.wait;" ::: "memory");
        const int quad = warp & 3;             // TMEM lane quadrant this warp may read
        // the four warps of a quadrant share the columns, 16 at a time, by twos where there are two blocks of 128 vocabulary rows
        const int team = (warp - 2) >> 2, block = t.blocks == 2 ? team & 1 : 0;
        const int c_first = 16 * (t.blocks == 2 ? team >> 1 : team), c_step = t.blocks == 2 ? 32 : 64;
        const int tile_row = rank * t.w_box + block * 128 + quad * 32;
        const int own_end = (rank + 1) * t.w_box;
        float* scales = reinterpret_cast<float*>(fixed + 512);
        float* turn = scales + 2 * 256 + (warp - 2) * 16 * kI8TurnStride;      // (STATS)
        if constexpr (FEW) {
            // this warp's part of its row, in 8 bits, to where the MMAs read it (tiles of N rows x 128 k, 128-byte swizzle)
            const int team_warps = kI8EpiWarps / p.R, ew = warp - 2, row = ew / team_warps;
            const bool mine = row < p.R;
            const int first = ((ew - row * team_warps) * 32 + lane) * 8, stride = team_warps * 256;
            const In* x = static_cast<const In*>(p.x) + row * p.ldx;
            uint32_t* s_top = reinterpret_cast<uint32_t*>(scales + 256);
            QuantChunk<In> c[kI8FewChunks];
            uint32_t top_bits = 0u;
#pragma unroll
            for (int i = 0; i < kI8FewChunks; ++i)
                if (mine && first + i * stride < p.d) c[i].load(x + first + i * stride);
#pragma unroll
            for (int i = 0; i < kI8FewChunks; ++i) {
                if (!mine || first + i * stride >= p.d) continue;
                float f[8];
                c[i].get(f);
#pragma unroll
                for (int j = 0; j < 8; ++j) top_bits = max(top_bits, __float_as_uint(f[j]) & 0x7fffffffu);
            }
            top_bits = __reduce_max_sync(kFullMask, top_bits);
            if (lane == 0) s_top[ew] = top_bits;
            named_barrier_sync(2, kI8EpiWarps * 32);
            if (mine) {
                for (int i = 0; i < team_warps; ++i) top_bits = max(top_bits, s_top[row * team_warps + i]);
                const RowScale rs(top_bits);
                if (first == 0) scales[row] = rs.scale;
#pragma unroll
                for (int i = 0; i < kI8FewChunks; ++i) {
                    const int k = first + i * stride;
                    if (k >= p.d) continue;
                    float f[8];
                    c[i].get(f);
                    uint8_t* to = x_tiles + ((k >> 7) * t.N + row) * kI8BK + ((((k >> 4) & 7) ^ (row & 7)) << 4) + (k & 8);
                    *reinterpret_cast<uint2*>(to) = rs.template round<In>(f);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(rows_full);
            named_barrier_sync(2, kI8EpiWarps * 32);
        }
        int it = 0;
        for (int item = worker; item < items; item += workers, ++it) {
            const int b = t.bufs == 2 ? it & 1 : 0;
            const int vt = item / t.MT, v0 = vt * t.TR, r0 = item % t.MT * t.N;
            const int vocab = min(PAIR ? own_end : t.TR, p.V - v0), rows = min(t.N, p.R - r0);
            const int v = v0 + tile_row + lane;
            const bool in = tile_row + lane < vocab;
            const float ws = in ? __ldcg(p.w_scale + v) : 0.f;
            // (from memory once for each item, while its products are made: in the loop below every other load would miss L1)
            float* x_scale = FEW ? scales : scales + (it & 1) * 256;
            if constexpr (!FEW) {
                const int i = (int)threadIdx.x - 64;
                if (i < rows) x_scale[i] = __ldcg(p.x_scale + r0 + i);
                named_barrier_sync(2, kI8EpiWarps * 32);
            }
            mbar_wait(&tmem_full[b], (t.bufs == 2 ? it >> 1 : it) & 1, p.status);
            tc_fence_after();
            if (tile_row < vocab) {
                const uint32_t tmem = tmem_base + (b * t.blocks + block) * t.cols + (static_cast<uint32_t>(quad * 32) << 16);
                Out* y_tile = static_cast<Out*>(p.y) + (long long)r0 * p.ldy + v;
                float2* stats = STATS ? p.stats + (long long)r0 * p.chunks + vt * (t.TR / kI8Chunk) + tile_row / kI8Chunk : nullptr;
#pragma unroll 1
                for (int c = c_first; c < rows; c += c_step) {
                    float z[16];
                    {
                        float xs[16];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 q = *reinterpret_cast<const float4*>(x_scale + c + 4 * i);
                            xs[4 * i] = q.x, xs[4 * i + 1] = q.y, xs[4 * i + 2] = q.z, xs[4 * i + 3] = q.w;
                        }
                        int acc[16];
                        tmem_ld16(tmem + c, acc);
#pragma unroll
                        for (int i = 0; i < 16; ++i) z[i] = __fmul_rn(__fmul_rn(static_cast<float>(acc[i]), xs[i]), ws);
                    }
                    if (in) {
                        Out* y = y_tile + c * p.ldy;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (c + i < rows) store_logit(y, z[i]);
                            y += p.ldy;
                        }
                    }
                    if constexpr (STATS) {
                        const float2 x = warp_chunk_stats(z, in, lane, turn);
                        if (lane < 16 && c + lane < rows) stats[(long long)(c + lane) * p.chunks] = x;
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR) mbar_arrive_cluster(leader_addr(smem_addr(&tmem_empty[b])));
                else mbar_arrive(&tmem_empty[b]);
            }
        }
    }

    tc_fence_before();
    if constexpr (PAIR) cluster_sync();    // (neither CTA of a pair leaves before the other)
    else __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        if constexpr (PAIR) tmem_dealloc_pair(tmem_base, 512);
        else tmem_dealloc(tmem_base, 512);
    }
}

}  // namespace disco
