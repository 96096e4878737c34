// Beam search: the selection over beams and vocabulary, and the reordering of the beams' states.
//
// Selection.  Of a sequence with K beams of score c_k and logits z_k[v], the n best continuations by
//     l[k, v] = c_k + z_k[v] - ln sum_w exp z_k[w],      ties to the lowest (k, v).
// Every logit is read once, by a pass that leaves the largest of each chunk of neighbouring logits, and sums of exponentials.  (The 8-bit LM
// head's epilogue leaves the same.)  What follows looks at few logits: the n best lie in the n chunks
// that come first by (best score, place), since each of those holds a candidate that beats whatever lies in
// another chunk.  Scores are formed and compared in 64 bits: which of two candidates is the better is a whole number.  The sums of
// exponentials are those of fp32 (beam_ln_err says how far a logarithm may be off) until candidates of different beams come nearer to each
// other than that; then the beams' sums are taken again, in 64 bits and in any order the same: equal beams stay equal.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "int8_head.cuh"   // max_nan, warp_max_nan_f32

namespace disco {

constexpr int kBeamStatWarps = 8;
constexpr int kBeamThreads = 1024;       // of the selection, at most
constexpr int kBeamCluster = 8;          // CTAs that make the pass over a sequence's logits and select, in one launch
constexpr int kBeamItems = 8;            // pieces of rows that a thread of it holds
constexpr int kBeamMaxBeams = DISCO_MAX_BEAMS;
constexpr int kBeamList = 1024;          // candidates that are ranked by counting
constexpr int kBeamPieceList = 512;      // pieces that are looked into
constexpr int kBeamAhead = 4;            // their logits that a thread has on their way at once

// How the chunks of a sequence's K rows are dealt to the warps of its CTA: a lane holds the largest logits of kBeamItems pieces, each of
// `merged` neighbouring chunks of one row.  Up to as many beams as warps: `share` warps to a row; up to twice as many (of 32 warps): two
// rows to a warp, half the pieces each.
struct BeamDeal {
    int two, share, merged, pieces, used;   // pieces of a row; how many of a lane's items there are, of a row
    __host__ __device__ static BeamDeal make(int K, int chunks, int warps) {
        BeamDeal d;
        d.two = K > warps;
        d.share = d.two ? 1 : warps / K;
        const int room = d.share * 32 * (d.two ? kBeamItems / 2 : kBeamItems);
        d.merged = (chunks + room - 1) / room;
        d.pieces = (chunks + d.merged - 1) / d.merged;
        d.used = (d.pieces + d.share * 32 - 1) / (d.share * 32);
        return d;
    }
    // Warps: as few of 8, 16 and 32 as hold every chunk as a piece of its own, otherwise 32; more where many are kept, since step 3 reads
    // about as many pieces.  (us a pass of 64 x 4 of 32000, 4 / 10 / 16 / 24 / 32 kept, 8 warps 14.0 / 15.8 / 17.9 / 21.1 / 24.8, 16 warps 14.1 /
    // 14.8 / 15.9 / 17.4 / 18.9, 32 warps 15.2 / 15.6 / 16.0 / 17.0 / 17.7; of 500 x 2 of 8000, 2 / 10 kept, 17.6 / 23.8, 19.2 / 23.2, 31.0 / 34.0.)
    __host__ __device__ static int warps(int K, int chunks, int n) {
        for (int w = n <= 10 ? 8 : n <= 24 ? 16 : 32; w < 32; w *= 2)
            if (K <= w && make(K, chunks, w).merged == 1) return w;
        return 32;
    }
};

// The pass over the logits and the selection in one launch: where a cluster has a warp for each segment of a sequence's logits, and the
// clusters fit side by side.  (us a pass, two launches -> one: 1 / 4 / 16 / 32 / 64 x 4 beams of 32000 fp32 logits 13.5 / 9.7 / 9.8 / 10.7 / 14.1 ->
// 8.4 / 8.8 / 10.0 / 12.2 / 17.7; with two segments to a warp and more, 20 x 5 of 40011 bf16 12.5 -> 14.7, 1 x 16 of 49152 fp32 11.2 -> 16.3.)
__host__ __device__ inline bool beam_joined(int B, int K, int segs) { return B <= 32 && K * segs <= 16 * kBeamCluster; }

// How far the logarithm of a row's sum of exponentials in fp32 may be off: relatively, the sum.  In units of 2^-24, for N terms a record, S
// records a row: exponentials 4 (2 ulp of ex2), their arguments 1.04 log2 N (a t rounded to fp32, of a rounded log2 e, weighs t 2^-t; weighted
// so, t is log2 N at most), sums 10, what makes good the rounded product 5; records meet with weights exp(top - top') of 6 each, at three
// levels at most, whose arguments take 2.4 ln S.  Given logits: N = 1024, S <= 1024: 64.  The 8-bit head's, N = 32, S <= 8192, and eight additions to
// a lane: 60.  A lane that takes its records in several rounds adds a weight and up to eight terms each time: 16.
__host__ __device__ inline float beam_ln_err(int rounds) { return 0x1p-18f + 0x1p-20f * (rounds - 1); }

struct BeamParams {
    const void* z;               // [B * K, V] logits, rows ld elements apart
    long long ld;
    int V, B, K, n;
    int eos;                     // the continuation of a finished beam (-1: none)
    const float* score;          // [B, K]
    const uint8_t* finished;     // [B, K] or null
    int chunks, segs;
    float* tops;                 // [B * K][chunks] largest logits of chunks of kBeamChunk
    float2* sums;                // [B * K][segs] of kBeamWarpChunks chunks each: their largest logit, the sum of exp(z - largest)
    const float2* pairs;         // [B * K][chunks] both for each chunk of kI8Chunk (instead of tops and sums)
    BeamDeal deal;
    float ln_err;                // beam_ln_err of the deal
    float* score_out;            // [B, n]
    int32_t* parent;
    int32_t* token;
    uint8_t* finished_out;       // or null
};

__device__ __forceinline__ float load_logit(const float* p) { return __ldcg(p); }
__device__ __forceinline__ float load_logit(const __nv_bfloat16* p) {
    return __uint_as_float(static_cast<uint32_t>(__ldcg(reinterpret_cast<const unsigned short*>(p))) << 16);
}
__device__ __forceinline__ float load_logit(const __half* p) {
    return __half2float(__ushort_as_half(__ldcg(reinterpret_cast<const unsigned short*>(p))));
}
__device__ __forceinline__ void load_logits2(const __nv_bfloat16* p, float& a, float& b) {
    const uint32_t q = __ldcg(reinterpret_cast<const uint32_t*>(p));
    a = __uint_as_float(q << 16), b = __uint_as_float(q & 0xffff0000u);
}
__device__ __forceinline__ void load_logits2(const __half* p, float& a, float& b) {
    const uint32_t q = __ldcg(reinterpret_cast<const uint32_t*>(p));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&q));
    a = f.x, b = f.y;
}

// Does the row's beam take part, and by its logits?
__device__ __forceinline__ bool beam_lives(float c) { return c > DISCO_NEG_INF && c < -DISCO_NEG_INF; }
__device__ __forceinline__ bool beam_expands(const BeamParams& p, int row) {
    return beam_lives(p.score[row]) && !(p.finished && p.finished[row]);
}

// The pass over the logits.  A warp takes eight chunks of a row; which lane holds which logit goes by its index alone, so that equal
// rows give equal sums wherever they lie.  (The eight chunks' largest logits meet in nine exchanges, each lane keeping half of what it has
// at each of the first three; with two reductions over the warp for each chunk the pass over bf16 logits took as long as over twice as many
// bytes of fp32.)
template <typename T>
__device__ __forceinline__ void beam_stats(const BeamParams& p, long long row, int seg, int lane) {
    static_assert(kBeamWarpChunks == 8, "three halvings");
    const int first = seg * kBeamWarpChunks;
    // a lane's logits of a chunk: two by two neighbours of 16 bits, so that they can be loaded together, every 32nd of 32 bits
    constexpr int kNext = sizeof(T) == 2 ? 2 : 1;
    const int v0 = first * kBeamChunk + lane * kNext;
    const T* z = static_cast<const T*>(p.z) + row * p.ld + v0;
    float f[kBeamWarpChunks][4];
    const bool whole = (first + kBeamWarpChunks) * kBeamChunk <= p.V;
    if (whole && (kNext == 1 || (reinterpret_cast<uintptr_t>(z) & 3) == 0)) {
#pragma unroll
        for (int c = 0; c < kBeamWarpChunks; ++c) {
            if constexpr (kNext == 2) {
#pragma unroll
                for (int i = 0; i < 2; ++i) load_logits2(z + c * kBeamChunk + i * 64, f[c][2 * i], f[c][2 * i + 1]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) f[c][i] = load_logit(z + c * kBeamChunk + i * 32);
            }
        }
    } else {
#pragma unroll
        for (int c = 0; c < kBeamWarpChunks; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = c * kBeamChunk + (kNext == 2 ? (i >> 1) * 64 + (i & 1) : i * 32);
                f[c][i] = v0 + at < p.V ? load_logit(z + at) : DISCO_NEG_INF;
            }
    }
    float t[kBeamWarpChunks];
#pragma unroll
    for (int c = 0; c < kBeamWarpChunks; ++c) t[c] = max_nan(max_nan(f[c][0], f[c][1]), max_nan(f[c][2], f[c][3]));
#pragma unroll
    for (int half = 4; half >= 1; half >>= 1) {      // lanes apart by 4 * half
        const bool up = lane & (4 * half);
#pragma unroll
        for (int c = 0; c < half; ++c) {
            const float keep = up ? t[c + half] : t[c], send = up ? t[c] : t[c + half];
            t[c] = max_nan(keep, __shfl_xor_sync(kFullMask, send, 4 * half));
        }
    }
    t[0] = max_nan(t[0], __shfl_xor_sync(kFullMask, t[0], 2));
    t[0] = max_nan(t[0], __shfl_xor_sync(kFullMask, t[0], 1));      // chunk lane / 4
    const float m = warp_max_nan_f32(t[0]);
    float s[kBeamWarpChunks];
    const bool serves = ExpFrom::serves(m);
    const ExpFrom from(m);
    if (serves) {
#pragma unroll
        for (int c = 0; c < kBeamWarpChunks; ++c) s[c] = (from(f[c][0]) + from(f[c][1])) + (from(f[c][2]) + from(f[c][3]));
    } else {
#pragma unroll
        for (int c = 0; c < kBeamWarpChunks; ++c) s[c] = (__expf(f[c][0] - m) + __expf(f[c][1] - m)) + (__expf(f[c][2] - m) + __expf(f[c][3] - m));
    }
#pragma unroll
    for (int half = 4; half >= 1; half >>= 1)
#pragma unroll
        for (int c = 0; c < half; ++c) s[c] += s[c + half];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s[0] += __shfl_xor_sync(kFullMask, s[0], off);
    if ((lane & 3) == 0 && first + (lane >> 2) < p.chunks) p.tops[row * p.chunks + first + (lane >> 2)] = t[0];
    if (lane == 0) p.sums[row * p.segs + seg] = make_float2(m, serves ? from.sum(s[0], m) : s[0]);      // (no number where the largest is not finite: nothing is done with it)
}

template <typename T>
__global__ void __launch_bounds__(kBeamStatWarps * 32) beam_stats_kernel(const BeamParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const long long w = (long long)blockIdx.x * kBeamStatWarps + (threadIdx.x >> 5);
    const long long row = w / p.segs;
    if (row >= (long long)p.B * p.K || !beam_expands(p, (int)row)) return;
    beam_stats<T>(p, row, (int)(w % p.segs), threadIdx.x & 31);
}

// ---------------------------------------------------------------------------------------------
// the selection
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned long long ordered_bits64(double x) {
    const unsigned long long u = static_cast<unsigned long long>(__double_as_longlong(__dadd_rn(x, 0.0)));   // (-0 is 0)
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ double from_ordered_bits64(unsigned long long k) {
    return __longlong_as_double(static_cast<long long>((k >> 63) ? (k & 0x7fffffffffffffffull) : ~k));
}

// Sum over the block; s is two sets of words, used in turn (one barrier).
template <int WARPS>
__device__ __forceinline__ int block_sum(int x, int (*s)[32], int& turn) {
    x = __reduce_add_sync(kFullMask, x);
    if ((threadIdx.x & 31) == 0) s[turn][threadIdx.x >> 5] = x;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    x = __reduce_add_sync(kFullMask, lane < WARPS ? s[turn][lane] : 0);
    turn ^= 1;
    return x;
}

// A cut (t, limit) through candidates that are ordered by key, largest first, and then by place: at least `want` and at most `cap` (>= want)
// of them have key > t, or key == t and place <= limit.  reach(t, limit) counts those, over the block.  Starts from lo, which at least
// `want` reach (or all, where there are fewer), and hi, which none does; two bisections, the second one where many are equal.
template <typename Reach>
__device__ __forceinline__ void block_cut(Reach reach, unsigned long long lo, unsigned long long hi, long long last_place, int want, int cap,
                                          unsigned long long& t, long long& limit) {
    t = lo;
    limit = last_place;
    if (reach(t, limit) <= cap) return;
#pragma unroll 1
    while (hi - lo > 1ull) {
        t = lo + (hi - lo) / 2;
        const int c = reach(t, limit);
        if (c < want) hi = t;
        else if (c <= cap) return;
        else lo = t;
    }
    t = lo;    // reached by too many, and what is above it by too few
    long long below = -1;
#pragma unroll 1
    while (limit - below > 1) {
        const long long mid = below + (limit - below) / 2;
        if (reach(t, mid) >= want) limit = mid;
        else below = mid;
    }
}

// 1 + exp(x - top) by its bits, x <= top: less those of 1, the term as a whole number of 2^-52.  2^t = 2^n 2^f with t = (x - top) log2 e, n the
// nearest integer, and 2^f = exp(f ln 2) by its Taylor polynomial of degree 11, off by 0.347^12 / 12! = 2^-47 at most.
constexpr unsigned long long kOneBits = 0x3ff0000000000000ull;
__device__ __forceinline__ unsigned long long one_and_exponential(float x, double top) {
    const double t = (static_cast<double>(x) - top) * 1.4426950408889634074;
    constexpr double kWhole = 0x1.8p52;      // (the sum with it leaves the nearest integer in the low bits)
    const double r = t + kWhole, f = t - (r - kWhole);
    constexpr double kLn2 = 0.69314718055994530942;
    constexpr double c1 = kLn2, c2 = c1 * kLn2 / 2, c3 = c2 * kLn2 / 3, c4 = c3 * kLn2 / 4, c5 = c4 * kLn2 / 5, c6 = c5 * kLn2 / 6, c7 = c6 * kLn2 / 7,
                     c8 = c7 * kLn2 / 8, c9 = c8 * kLn2 / 9, c10 = c9 * kLn2 / 10, c11 = c10 * kLn2 / 11;
    double p = c11;
    p = fma(p, f, c10), p = fma(p, f, c9), p = fma(p, f, c8), p = fma(p, f, c7), p = fma(p, f, c6), p = fma(p, f, c5);
    p = fma(p, f, c4), p = fma(p, f, c3), p = fma(p, f, c2), p = fma(p, f, c1), p = fma(p, f, 1.0);
    p = __hiloint2double(__double2hiint(p) + (__double2loint(r) << 20), __double2loint(p));
    return t > -64.0 ? static_cast<unsigned long long>(__double_as_longlong(1.0 + p)) : kOneBits;      // (-inf: nothing)
}

// The sum of the terms exp(z - top) of a row, by all threads of a block, as whole numbers of 2^-52: the same in any order, and off by no more than
// sums in 64 bits are.  total: three words of it in shared memory, 32 bits apart (2^28 terms at most: no word passes 64 bits).
// kAtOnce logits of a thread on their way while as many are at work, as far as there are registers.
template <int kAtOnce, int THREADS, typename T>
__device__ __forceinline__ void add_exponentials(const T* z, int V, float top, unsigned long long* total) {
    unsigned __int128 sum = 0;
    float next[kAtOnce];
    auto load = [&](int v) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) next[i] = v + i * THREADS < V ? load_logit(z + v + i * THREADS) : DISCO_NEG_INF;
    };
    load(threadIdx.x);
#pragma unroll 1
    for (int v = threadIdx.x; v < V;) {
        unsigned long long some = 0ull;      // 2048 terms of 2^52 at most, modulo 2^64
        int n = 0;
#pragma unroll 1
        for (; v < V && n < 2048; v += kAtOnce * THREADS, n += kAtOnce) {
            float x[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) x[i] = next[i];
            load(v + kAtOnce * THREADS);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) some += one_and_exponential(x[i], static_cast<double>(top));
        }
        sum += some - n * kOneBits;
    }
    unsigned long long w[3] = {static_cast<uint32_t>(sum), static_cast<uint32_t>(sum >> 32), static_cast<unsigned long long>(sum >> 64)};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) w[i] += __shfl_xor_sync(kFullMask, w[i], off);
        if ((threadIdx.x & 31) == 0) atomicAdd(total + i, w[i]);
    }
}

// More candidates or pieces than this are worth another search for a floor.  (n + 8 / 2 n + 8 / 4 n + 8, us a pass: 16 x 8, 32 kept, 16.4 / 14.0 /
// 13.9, 16 x 16, 40 kept, 21.5 / 21.2 / 23.5.)
__device__ __forceinline__ int beam_few(int n) { return 2 * n + 8; }

// What a CTA of the selection holds in shared memory.
struct BeamShared {
    ulonglong2 cand[kBeamList];      // (score, place); in step 3 the logit's bits for the score
    int2 piece[kBeamPieceList];      // its row, its first token
    float piece_top[kBeamPieceList];
    double lse[kBeamMaxBeams];       // the sum of exponentials, then what is taken off a logit
    float score[kBeamMaxBeams], top[kBeamMaxBeams], offset[kBeamMaxBeams], err[kBeamMaxBeams];
    int state[kBeamMaxBeams];        // 0: no continuation, 1: expands, 2: finished
    int sum64[kBeamMaxBeams];        // the row's sum of exponentials is 0: one of fp32, 1: to be one of 64 bits, 2: that, or none
    unsigned long long total[3];
    int sum[2][32];
    uint32_t unsure;                 // how far a score may be off for its sum of exponentials, by the bits
    int pieces, count;
};

// Steps of the selection that its quick way and its thorough one share.
template <typename T, int CHUNK, int THREADS>
struct BeamCta {
    const BeamParams& p;
    BeamShared& s;
    int b;
    float floor;      // no less than this do the n best score

    __device__ __forceinline__ int width() const { return p.deal.merged * CHUNK; }
    // May a logit's score reach the floor?
    __device__ __forceinline__ bool within(int k, float z) const {
        return z > DISCO_NEG_INF && !((z + s.offset[k]) + (s.err[k] + 0x1p-21f * fabsf(z)) < floor);
    }
    __device__ __forceinline__ unsigned long long score_of(int k, float z) const {
        return ordered_bits64(static_cast<double>(s.score[k]) + (static_cast<double>(z) - s.lse[k]));
    }
    __device__ __forceinline__ void finish_lse() const {
        for (int k = threadIdx.x; k < p.K; k += THREADS) s.lse[k] = static_cast<double>(s.top[k]) + log(s.lse[k]);
    }
    __device__ __forceinline__ const T* row(int k) const { return static_cast<const T*>(p.z) + (long long)(b * p.K + k) * p.ld; }
    __device__ __forceinline__ void note_piece(int k, int v, float z) const {
        const int at = atomicAdd(&s.pieces, 1);
        if (at < kBeamPieceList) s.piece[at] = make_int2(k, v), s.piece_top[at] = z;
    }
    // Value i of the pieces.
    __device__ __forceinline__ bool locate(int i, int& k, int& v) const {
        const int l = p.deal.merged == 1 ? i / CHUNK : i / width();
        const int2 piece = s.piece[l];
        k = piece.x;
        v = piece.y + (i - l * width());
        return v < p.V;
    }
    // Values i0, i0 + THREADS, ... of the pieces; -inf where there is none.
    __device__ __forceinline__ void load(int i0, int values, float (&z)[kBeamAhead], int (&k)[kBeamAhead], int (&v)[kBeamAhead]) const {
#pragma unroll
        for (int a = 0; a < kBeamAhead; ++a) {
            const int i = i0 + a * THREADS;
            z[a] = i < values && locate(i, k[a], v[a]) ? load_logit(row(k[a]) + v[a]) : DISCO_NEG_INF;
        }
    }
    static __device__ __forceinline__ unsigned long long place_of(int k, int v) { return (unsigned long long)k << 32 | (unsigned int)v; }
    static __device__ __forceinline__ int beam_of(const ulonglong2& c) { return static_cast<int>(c.y >> 32); }
    __device__ __forceinline__ void take(unsigned long long x, unsigned long long place) const {
        const int at = atomicAdd(&s.count, 1);
        if (at < kBeamList) s.cand[at] = make_ulonglong2(x, place);
    }
    // How near scores of different beams may come before their order is in doubt.
    __device__ __forceinline__ double reach() const { return 2.0 * static_cast<double>(__uint_as_float(s.unsure)); }
    // The key of the least score that may be better than c's if the sums of exponentials are off.
    static __device__ __forceinline__ unsigned long long low_of(const ulonglong2& c, double reach) {
        return ordered_bits64(from_ordered_bits64(c.x) - reach);
    }
    static __device__ __forceinline__ int close_to(const ulonglong2& c, unsigned long long low, const ulonglong2& o) {
        return static_cast<int>(o.x >= low) & static_cast<int>(o.x <= c.x) & static_cast<int>(beam_of(o) != beam_of(c));
    }
    // Ranks of the N candidates, by counting, and what is returned.  Is one of this thread's in doubt?
    __device__ __forceinline__ bool rank(int N) const {
        const long long out = (long long)b * p.n;
        const double r = reach();
        bool unsure = false;
        for (int i = threadIdx.x; i < N; i += THREADS) {
            const ulonglong2 c = s.cand[i];
            const unsigned long long low = low_of(c, r);
            int rank = 0, close = 0;
#pragma unroll 4
            for (int j = 0; j < N; ++j) {       // (no branches: with them a candidate costs 140 cycles)
                const ulonglong2 o = s.cand[j];
                rank += static_cast<int>(o.x > c.x) | (static_cast<int>(o.x == c.x) & static_cast<int>(o.y < c.y));
                close |= close_to(c, low, o);
            }
            if (rank < p.n) {       // (what is read of the beams has been read: the outputs may take the inputs' place)
                const int parent = beam_of(c), token = static_cast<int>(c.y & 0xffffffffull);
                p.score_out[out + rank] = static_cast<float>(from_ordered_bits64(c.x));
                p.parent[out + rank] = parent;
                p.token[out + rank] = token;
                if (p.finished_out) p.finished_out[out + rank] = token == p.eos || s.state[parent] == 2;
                unsure = unsure || close != 0;
            }
        }
        return unsure;
    }
    // Places that no continuation is left for.
    __device__ __forceinline__ void no_more(int N) const {
        const long long out = (long long)b * p.n;
        for (int i = N + threadIdx.x; i < p.n; i += THREADS) {
            p.score_out[out + i] = DISCO_NEG_INF;
            p.parent[out + i] = -1;
            p.token[out + i] = -1;
            if (p.finished_out) p.finished_out[out + i] = 0;
        }
    }
};

// The selection from where its quick way does not lead on, for all threads of a CTA behind a barrier: with more pieces than the list holds (and
// sums of exponentials that are not logarithms yet), more candidates, or candidates of different beams whose order is in doubt.  A function
// of its own, called last of all: among the rest its code and its registers cost every call 2 - 4 us where the kernel's code is not in a cache.
enum BeamDoubt { kBeamPieces, kBeamValues, kBeamOrder };
template <typename T, int CHUNK, int THREADS, int SIDE>
__device__ __noinline__ void beam_settle(const BeamParams& p, BeamShared& s, int b, float floor, BeamDoubt doubt) {
    constexpr int kWarps = THREADS / 32;
    BeamCta<T, CHUNK, THREADS> cta{p, s, b, floor};
    const int tid = threadIdx.x;
    const BeamDeal& deal = p.deal;
    const double reach = cta.reach();
    int turn = 0;
    // The sums of exponentials that are to be of 64 bits (all threads, behind a barrier).
    auto sum_again = [&] {
#pragma unroll 1
        for (int k = 0; k < p.K; ++k) {
            if (s.sum64[k] != 1) continue;
            if (tid == 0) s.total[0] = s.total[1] = s.total[2] = 0ull;
            __syncthreads();
            add_exponentials<THREADS == 512 && SIDE == 1 ? 4 : 2, THREADS>(cta.row(k), p.V, s.top[k], s.total);
            __syncthreads();
            if (tid == 0) {
                const double sum = (static_cast<double>(s.total[2]) * 0x1p64 + static_cast<double>(s.total[1]) * 0x1p32) + static_cast<double>(s.total[0]);
                s.lse[k] = static_cast<double>(s.top[k]) + log(sum * 0x1p-52);
                s.sum64[k] = 2;
            }
        }
        __syncthreads();
    };
    // block_cut, at scores of which those of different beams may be off: with all that may belong before the cut, if these are no more than
    // `most`; otherwise once more, with the sums of all rows that the floor leaves in 64 bits.
    auto sure_cut = [&](auto reaches, auto again, long long last_place, int cap, int most, unsigned long long& t, long long& limit) {
#pragma unroll 1
        for (bool sure = false;; sure = true) {
            block_cut(reaches, 1ull, ~0ull, last_place, p.n, cap, t, limit);
            const bool left = tid < p.K && (s.state[tid] == 2 || (s.state[tid] == 1 && cta.within(tid, s.top[tid])));
            if (__syncthreads_count(left) < 2 || sure) return;
            const unsigned long long low = ordered_bits64(from_ordered_bits64(t) - reach);
            if (reaches(low, last_place) <= most) {
                t = low;
                limit = last_place;
                return;
            }
            if (left && s.sum64[tid] == 0) s.sum64[tid] = 1;
            __syncthreads();
            sum_again();
            again();
        }
    };
    int L = min(s.pieces, kBeamPieceList);
    auto each = [&](auto f) {      // the candidates: (score, place)
        const int values = L * cta.width();
#pragma unroll 1
        for (int i0 = tid; i0 < values; i0 += kBeamAhead * THREADS) {
            float z[kBeamAhead];
            int k[kBeamAhead], v[kBeamAhead];
            cta.load(i0, values, z, k, v);
#pragma unroll
            for (int a = 0; a < kBeamAhead; ++a)
                if (z[a] > DISCO_NEG_INF && cta.within(k[a], z[a])) f(cta.score_of(k[a], z[a]), static_cast<long long>(cta.place_of(k[a], v[a])));
        }
        if (tid < p.K && s.state[tid] == 2) f(ordered_bits64(s.score[tid]), static_cast<long long>(cta.place_of(tid, p.eos)));
    };
    if (doubt == kBeamPieces) {
        cta.finish_lse();
        __syncthreads();
        // (as many pieces as threads hold items of)
        float best[kBeamItems];
        unsigned long long key[kBeamItems];
        const int all = p.K * deal.pieces;
#pragma unroll
        for (int j = 0; j < kBeamItems; ++j) {
            best[j] = DISCO_NEG_INF;
            const int i = j * THREADS + tid, k = i / deal.pieces, first = (i - k * deal.pieces) * deal.merged;
            if (i >= all || s.state[k] != 1) continue;
            const long long at = (long long)(b * p.K + k) * p.chunks;
            for (int c = first; c < min(first + deal.merged, p.chunks); ++c) {
                if constexpr (CHUNK == kBeamChunk) best[j] = fmaxf(best[j], __ldcg(p.tops + at + c));
                else best[j] = fmaxf(best[j], __ldcg(p.pairs + at + c).x);
            }
        }
        auto score_pieces = [&] {
#pragma unroll
            for (int j = 0; j < kBeamItems; ++j) key[j] = best[j] > DISCO_NEG_INF ? cta.score_of((j * THREADS + tid) / deal.pieces, best[j]) : 0ull;
        };
        score_pieces();
        auto pieces_reach = [&](unsigned long long u, long long limit) {
            int c = 0;
#pragma unroll
            for (int j = 0; j < kBeamItems; ++j) c += key[j] > u || (key[j] == u && j * THREADS + tid <= limit);
            return block_sum<kWarps>(c, s.sum, turn);
        };
        unsigned long long t;
        long long limit;
        sure_cut(pieces_reach, score_pieces, all, 2 * p.n, kBeamPieceList, t, limit);
        if (tid == 0) s.pieces = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kBeamItems; ++j) {
            const int i = j * THREADS + tid, k = i / deal.pieces;
            if (key[j] > t || (key[j] == t && i <= limit)) cta.note_piece(k, (i - k * deal.pieces) * cta.width(), best[j]);
        }
        // (more pieces than the list holds, so n at least have been found)
        cta.floor = __double2float_rd(from_ordered_bits64(t));
        __syncthreads();
        L = min(s.pieces, kBeamPieceList);      // (a matter of course, unless the statistics are those of a product whose wait ran out)
        each([&](unsigned long long x, long long place) { cta.take(x, place); });
        __syncthreads();
        if (s.count > kBeamList) doubt = kBeamValues;
    }
    if (doubt == kBeamValues) {      // many equal logits
        auto values_reach = [&](unsigned long long u, long long limit) {
            int c = 0;
            each([&](unsigned long long x, long long place) { c += x > u || (x == u && place <= limit); });
            return block_sum<kWarps>(c, s.sum, turn);
        };
        unsigned long long t;
        long long limit;
        sure_cut(values_reach, [] {}, (long long)kBeamMaxBeams << 32, kBeamList / 2, kBeamList, t, limit);
        __syncthreads();
        if (tid == 0) s.count = 0;
        __syncthreads();
        each([&](unsigned long long x, long long place) {
            if (x > t || (x == t && place <= limit)) cta.take(x, place);
        });
        __syncthreads();
    }
    int N = min(s.count, kBeamList);
    auto score_again = [&] {
        for (int i = tid; i < N; i += THREADS) {
            const int k = cta.beam_of(s.cand[i]);
            if (s.state[k] == 1) s.cand[i].x = cta.score_of(k, load_logit(cta.row(k) + static_cast<int>(s.cand[i].y & 0xffffffffull)));
        }
        __syncthreads();
    };
    if (doubt != kBeamOrder && N > beam_few(p.n)) {      // ranking takes as many steps as there are candidates
        auto list_reach = [&](unsigned long long u, long long limit) {
            int c = 0;
            for (int i = tid; i < N; i += THREADS) c += s.cand[i].x > u || (s.cand[i].x == u && static_cast<long long>(s.cand[i].y) <= limit);
            return block_sum<kWarps>(c, s.sum, turn);
        };
        unsigned long long t;
        long long limit;
        sure_cut(list_reach, score_again, (long long)kBeamMaxBeams << 32, beam_few(p.n), kBeamList, t, limit);
        constexpr int kEach = (kBeamList + THREADS - 1) / THREADS;
        ulonglong2 c[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) c[i] = i * THREADS + tid < N ? s.cand[i * THREADS + tid] : make_ulonglong2(0ull, ~0ull);
        __syncthreads();
        if (tid == 0) s.count = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (c[i].x > t || (c[i].x == t && static_cast<long long>(c[i].y) <= limit)) cta.take(c[i].x, c[i].y);
        __syncthreads();
        N = min(s.count, kBeamList);
    }
#pragma unroll 1
    while (__syncthreads_or(cta.rank(N)) && p.K > 1) {
        // Once more with sums of 64 bits of the beams that matter, if they are not of 64 bits already (so as many rounds as beams, at most).
        bool more = false;
        for (int i = tid; i < N; i += THREADS) {
            const ulonglong2 c = s.cand[i];
            const unsigned long long low = cta.low_of(c, reach);
            const int k = cta.beam_of(c);
#pragma unroll 4
            for (int j = 0; j < N; ++j) {
                const ulonglong2 o = s.cand[j];
                const int l = cta.beam_of(o);
                if (!cta.close_to(c, low, o) || (s.sum64[k] == 2 && s.sum64[l] == 2)) continue;
                if (s.sum64[k] == 0) s.sum64[k] = 1;
                if (s.sum64[l] == 0) s.sum64[l] = 1;
                more = true;
            }
        }
        if (!__syncthreads_or(more)) break;
        sum_again();
        score_again();
    }
    cta.no_more(N);
}

// A CTA to a sequence.  JOINED: a cluster of CTAs, which first of all make the pass over the sequence's logits; one of them goes on.
//   1  each row's soft-max statistics from its chunks'
//   2  the pieces that may hold the n best: every piece is known by its best score.  The n-th largest of what the threads have at best is
//      reached by n pieces at least, and by few more
//   3  the logits of these pieces, of which those count that reach the same score
//   4  what is left is scored in 64 bits and ranked by counting; again, where the order of different beams is within what their sums of
//      exponentials may be off, with the sums of these beams in 64 bits.  (Seldom, 2^-17 apart: of 64 kept of 16 beams 1.5 %
//      of the sequences, of 8 of 8 below 0.1 %.  A beam's sum takes 9 - 19 us, of 32000 logits by 512 threads - of 49152 by 256.)
// Up to 4 everything is in fp32 with a bound on its error, from which a piece or a logit is dropped only if it cannot be among the n best:
// the 64-bit units are too few for a score for every piece (of 32000 logits and 4 beams, 8400 and 4400 cycles for steps 1 and 2 in 64 bits).
// Where too many are equal for the lists (a call that is full of ties), the cuts are made in 64 bits, by bisection (beam_settle, like the
// sums of 64 bits).
// SIDE: CTAs that are to fit an SM side by side.
template <typename T, int CHUNK, int THREADS, bool TWO, bool JOINED, int SIDE = 1>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 3 : SIDE) beam_select_kernel(const __grid_constant__ BeamParams p) {
    static_assert(THREADS <= kBeamThreads && kBeamMaxBeams <= THREADS && DISCO_MAX_KEPT <= THREADS, "a thread to a beam, and to a place");
    constexpr int kWarps = THREADS / 32;
    __shared__ BeamShared s;
    __shared__ float s_max[2][32];
    __shared__ double s_exp[2][32];
    __shared__ uint32_t s_best[3];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int b = JOINED ? blockIdx.x / kBeamCluster : blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if constexpr (JOINED) {
        for (int i = (blockIdx.x % kBeamCluster) * kWarps + warp; i < p.K * p.segs; i += kBeamCluster * kWarps) {
            const int row = b * p.K + i / p.segs;
            if (beam_expands(p, row)) beam_stats<T>(p, row, i % p.segs, lane);
        }
        cluster_sync();
        if (blockIdx.x % kBeamCluster) return;
    }
    const BeamDeal deal = p.deal;
    const int warp_row = TWO ? warp : warp / deal.share, warp_share = TWO ? 0 : warp - warp_row * deal.share;
    constexpr int kHalf = kBeamItems / 2, kRows = TWO ? 2 : 1;      // (rows of a warp)
    auto item_row = [&](int j) { return TWO && j >= kHalf ? warp_row + 32 : warp_row; };
    auto item_piece = [&](int j) { return ((TWO ? j & (kHalf - 1) : j) * deal.share + warp_share) * 32 + lane; };
    auto item_used = [&](int j) { return (TWO ? j & (kHalf - 1) : j) < deal.used; };

    // ---- 1 ----
    float best[kBeamItems], top[kRows];      // the largest logits of this lane's pieces, and of those of a row
    {
        float m[kRows], e[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) m[r] = top[r] = DISCO_NEG_INF, e[r] = 0.f;
        // a row's sums join those of this lane: relative to the larger of the largest logits
        auto join = [&](int r, float top, float sum) {
            if (!(top > DISCO_NEG_INF)) return;       // (NaN: the row's largest logit says so)
            const float now = fmaxf(m[r], top);
            e[r] = e[r] * __expf(m[r] - now) + sum * __expf(top - now);
            m[r] = now;
        };
        if constexpr (CHUNK == kBeamChunk) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int k = warp_row + 32 * r;
                if (k >= p.K) continue;
                for (int i = warp_share * 32 + lane; i < p.segs; i += deal.share * 32) {
                    const float2 x = __ldcg(p.sums + (long long)(b * p.K + k) * p.segs + i);
                    join(r, x.x, x.y);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kBeamItems; ++j) best[j] = DISCO_NEG_INF;
#pragma unroll 1
        for (int g = 0; g < deal.merged; ++g) {
            float2 x[kBeamItems];
#pragma unroll
            for (int j = 0; j < kBeamItems; ++j) {
                x[j] = make_float2(DISCO_NEG_INF, 0.f);
                if (item_used(j)) {
                    const int k = item_row(j), piece = item_piece(j), chunk = piece * deal.merged + g;
                    if (k < p.K && chunk < p.chunks && piece < deal.pieces) {
                        const long long at = (long long)(b * p.K + k) * p.chunks + chunk;
                        if constexpr (CHUNK == kBeamChunk) x[j].x = __ldcg(p.tops + at);
                        else x[j] = __ldcg(p.pairs + at);
                    }
                }
            }
            if (g == 0) {
                if (tid < p.K) {
                    const float c = p.score[b * p.K + tid];
                    const bool over = p.finished && p.finished[b * p.K + tid];
                    s.score[tid] = c;
                    s.state[tid] = !beam_lives(c) ? 0 : over ? 2 : 1;
                }
                if (tid < 3) s_best[tid] = 0u;
                if (tid == 0) s.count = 0, s.pieces = 0, s.unsure = 0u;
            }
#pragma unroll
            for (int j = 0; j < kBeamItems; ++j) {
                if (!item_used(j)) continue;
                const int r = TWO && j >= kHalf;
                best[j] = max_nan(best[j], x[j].x);
                top[r] = max_nan(top[r], x[j].x);
            }
            if constexpr (CHUNK != kBeamChunk) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const float now = warp_max_nan_f32(top[r]);
                    if (now > m[r]) e[r] *= __expf(m[r] - now);
                    m[r] = now;
#pragma unroll
                    for (int j = 0; j < kBeamItems; ++j)
                        if (item_used(j) && (TWO && j >= kHalf) == (r == 1) && x[j].x > DISCO_NEG_INF)
                            e[r] = fmaf(x[j].y, __expf(x[j].x - now), e[r]);
                }
            }
        }
        if constexpr (CHUNK == kBeamChunk) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const float now = warp_max_nan_f32(max_nan(m[r], top[r]));
                e[r] = m[r] > DISCO_NEG_INF ? e[r] * __expf(m[r] - now) : 0.f;
                m[r] = now;
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            double sum = e[r];
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(kFullMask, sum, off);
            if (lane == 0) s_max[r][warp] = m[r], s_exp[r][warp] = sum;
        }
    }
    __syncthreads();
    for (int k = warp; k < p.K; k += kWarps) {       // a warp to a row, a lane to a share
        const int r = k >> 5, w = TWO ? k & 31 : k * deal.share + lane;
        const float x = lane < deal.share ? s_max[r][w] : DISCO_NEG_INF;
        const float top = warp_max_nan_f32(x);
        const bool is = top > DISCO_NEG_INF && top < -DISCO_NEG_INF;     // (otherwise the row is no distribution)
        double sum = is && lane < deal.share && x > DISCO_NEG_INF ? s_exp[r][w] * static_cast<double>(__expf(x - top)) : 0.0;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(kFullMask, sum, off);
        if (lane == 0) {
            if (!is && s.state[k] == 1) s.state[k] = 0;
            s.lse[k] = sum;
            s.top[k] = top;
            // score = logit + offset, and what fp32 makes of that: a few roundings of numbers of these sizes and of the logarithm, and
            // the error of the sum, which the logarithm passes on whatever its size (the sum's own rounding to fp32, 2^-24, among it)
            const float ln = logf(static_cast<float>(sum));
            s.offset[k] = s.score[k] - (top + ln);
            s.err[k] = (0x1p-21f * fabsf(s.score[k]) + 0x1p-21f * fabsf(top)) + (0x1p-21f * ln + p.ln_err);
            // (an offset beyond what fp32 holds says nothing of the scores: no bound, so nothing of the row is dropped)
            if (!(fabsf(s.offset[k]) < -DISCO_NEG_INF)) s.err[k] = -DISCO_NEG_INF;
        }
    }
    __syncthreads();

    // ---- 2 ----
    if (tid < p.K) s.sum64[tid] = s.state[tid] == 1 ? 0 : 2;
    // (a warp's rows, the second one where it has two)
    float offset[kRows], err[kRows];
    float low = DISCO_NEG_INF;      // the least that the best of this thread's pieces may score
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int k = warp_row + 32 * r;
        const bool expands = k < p.K && s.state[k] == 1;
        offset[r] = expands ? s.offset[k] : 0.f;
        err[r] = expands ? s.err[k] : 0.f;
        if (!expands) top[r] = DISCO_NEG_INF;       // (nothing of this row counts)
        const float f = top[r] + offset[r];
        if (top[r] > DISCO_NEG_INF && f < -DISCO_NEG_INF) low = fmaxf(low, f - (err[r] + 0x1p-21f * fabsf(top[r])));       // (beyond what fp32 holds: no bound)
    }
    auto high = [&](int r, float z) { return (z + offset[r]) + (err[r] + 0x1p-21f * fabsf(z)); };      // the most that a logit may score
    // The n-th largest of the threads' bounds, or a little less.  Each step costs a barrier that counts, so the search goes out from the
    // largest one, in strides that grow until n reach it, and only then halves what is left, until 1.5 n at most do (n / 1.5 n / 2 n, us a pass: 20
    // x 5, 10 kept, 13.8 / 12.4 / 12.9, 16 x 8, 32 kept, 14.6 / 14.0 / 16.3, 16 x 16, 40 kept, 19.7 / 21.2 / 21.8).
    auto find_floor = [&](float low, int use) {
        const uint32_t key = ordered_bits(low), top = __reduce_max_sync(kFullMask, key);
        if (lane == 0) atomicMax(&s_best[use], top);
        __syncthreads();
        const uint32_t best = s_best[use];
        uint32_t lo = 0u, hi = best + 1u, stride = 1u << 18;       // reached by n, and by fewer
        bool out = true;
#pragma unroll 1
        while (hi - lo > 1u) {
            const uint32_t at = out ? (best > stride ? best - stride : 0u) : lo + (hi - lo) / 2;
            const int c = __syncthreads_count(key >= at);
            if (c < p.n) {
                hi = at;
                stride <<= 2;
                out = out && stride != 0u && at > 0u;
            } else {
                lo = at;
                out = false;
                if (c <= p.n + (p.n + 1) / 2) break;
            }
        }
        return lo > 0x007fffffu ? from_ordered_bits(lo) : DISCO_NEG_INF;
    };
    BeamCta<T, CHUNK, THREADS> cta{p, s, b, find_floor(low, 0)};
    auto bound = [&](int k, float z) {
        const float f = z + s.offset[k];
        return f < -DISCO_NEG_INF ? f - (s.err[k] + 0x1p-21f * fabsf(z)) : DISCO_NEG_INF;
    };
    if (tid < p.K && s.state[tid] == 1 && cta.within(tid, s.top[tid]))       // (and what 64 bits make of numbers of these sizes)
        atomicMax(&s.unsure, __float_as_uint(p.ln_err + 0x1p-50f * (fabsf(s.score[tid]) + fabsf(s.top[tid]))));
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (!(top[r] > DISCO_NEG_INF) || high(r, top[r]) < cta.floor) continue;      // (so it is with most threads)
#pragma unroll
        for (int j = 0; j < kBeamItems; ++j)
            if (item_used(j) && (TWO && j >= kHalf) == (r == 1) && best[j] > DISCO_NEG_INF && !(high(r, best[j]) < cta.floor))
                cta.note_piece(item_row(j), item_piece(j) * cta.width(), best[j]);
    }
    __syncthreads();
    const int few = beam_few(p.n);
    int L = s.pieces;
    if (L > few && L <= kBeamPieceList) {
        constexpr int kEach = (kBeamPieceList + THREADS - 1) / THREADS;
        int2 piece[kEach];
        float z[kEach], low = DISCO_NEG_INF;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            z[i] = DISCO_NEG_INF;
            if (i * THREADS + tid >= L) continue;
            piece[i] = s.piece[i * THREADS + tid];
            z[i] = s.piece_top[i * THREADS + tid];
            low = fmaxf(low, bound(piece[i].x, z[i]));
        }
        const float next = find_floor(low, 1);
        __syncthreads();
        if (tid == 0) s.pieces = 0;
        cta.floor = fmaxf(cta.floor, next);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (z[i] > DISCO_NEG_INF && cta.within(piece[i].x, z[i])) cta.note_piece(piece[i].x, piece[i].y, z[i]);
        __syncthreads();
        L = s.pieces;
    }
    if (L > kBeamPieceList) return beam_settle<T, CHUNK, THREADS, SIDE>(p, s, b, cta.floor, kBeamPieces);

    // ---- 3 ----
    const int values = L * cta.width();
    bool first = true;
    for (int i0 = tid; i0 - tid < values; i0 += kBeamAhead * THREADS) {
        float z[kBeamAhead];
        int k[kBeamAhead], v[kBeamAhead];
        cta.load(i0, values, z, k, v);
        if (first) cta.finish_lse();       // (while the loads are on their way)
        first = false;
#pragma unroll
        for (int a = 0; a < kBeamAhead; ++a)       // (a logit stands in for its score, which step 4 needs)
            if (z[a] > DISCO_NEG_INF && cta.within(k[a], z[a])) cta.take(__float_as_uint(z[a]), cta.place_of(k[a], v[a]));
    }
    if (first) cta.finish_lse();
    if (tid < p.K && s.state[tid] == 2) cta.take(0ull, cta.place_of(tid, p.eos));
    __syncthreads();
    int N = s.count;
    if (N > kBeamList) return beam_settle<T, CHUNK, THREADS, SIDE>(p, s, b, cta.floor, kBeamValues);
    {
        constexpr int kEach = (kBeamList + THREADS - 1) / THREADS;
        ulonglong2 cand[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) cand[i] = i * THREADS + tid < N ? s.cand[i * THREADS + tid] : make_ulonglong2(0ull, ~0ull);
        auto logit_of = [](const ulonglong2& c) { return __uint_as_float(static_cast<uint32_t>(c.x)); };
        if (N > few) {
            float low = DISCO_NEG_INF;
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (cand[i].y != ~0ull && s.state[cta.beam_of(cand[i])] == 1) low = fmaxf(low, bound(cta.beam_of(cand[i]), logit_of(cand[i])));
            cta.floor = fmaxf(cta.floor, find_floor(low, 2));
        }
        const bool again = N > few;
        if (again) {
            __syncthreads();
            if (tid == 0) s.count = 0;
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (cand[i].y == ~0ull) continue;
            const int k = cta.beam_of(cand[i]);
            const bool ended = s.state[k] == 2;
            if (again && !ended && !cta.within(k, logit_of(cand[i]))) continue;
            const unsigned long long x = ended ? ordered_bits64(s.score[k]) : cta.score_of(k, logit_of(cand[i]));
            if (again) cta.take(x, cand[i].y);
            else s.cand[i * THREADS + tid].x = x;
        }
    }
    __syncthreads();

    // ---- 4 ----
    N = s.count;
    const bool unsure = cta.rank(N);
    cta.no_more(N);
    if (p.K > 1 && __syncthreads_or(unsure)) beam_settle<T, CHUNK, THREADS, SIDE>(p, s, b, cta.floor, kBeamOrder);
}

// ---------------------------------------------------------------------------------------------
// the states
// ---------------------------------------------------------------------------------------------
constexpr int kReorderTensors = 64;     // to a launch
constexpr int kReorderThreads = 256;

struct ReorderParams {
    const void* src[kReorderTensors];   // [B * K][mid][T * unit] words
    void* dst[kReorderTensors];         // [B * n][mid][T * unit]
    int B, K, n;
    const int32_t* parent;              // [B, n]
    const int32_t* lens;                // [B] positions in use, or null: all T
    long long mid, T, unit;             // unit: words to a position
    int tiles;                          // CTAs to a row
    int in_place;
    int* status;
};

// dst[b * n + j] = src[b * K + parent[b, j]], the positions in use of each.  A thread owns one word's place in all rows of a sequence:
// it loads the word of up to N parents, then stores their children's, so a state may be reordered in place, and the loads of a parent
// with several children meet in L1.
template <typename Word, int N>
__global__ void __launch_bounds__(kReorderThreads) beam_reorder_kernel(const __grid_constant__ ReorderParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tile = blockIdx.x % p.tiles;
    const long long bm = blockIdx.x / p.tiles;
    const int b = (int)(bm / p.mid);
    const long long m = bm % p.mid;
    const int32_t* parent = p.parent + (long long)b * p.n;
    if (tile == 0 && m == 0 && blockIdx.y == 0)
        for (int j = threadIdx.x; j < p.n; j += kReorderThreads)
            if (parent[j] < -1 || parent[j] >= p.K) record_status(p.status, DISCO_ERR_INVALID_ARG);
    const long long words = p.T * p.unit;
    const long long used = p.lens ? min(max((long long)p.lens[b], 0ll), p.T) * p.unit : words;
    const long long at = (long long)tile * kReorderThreads + threadIdx.x;
    if (at >= used) return;
    const Word* src = static_cast<const Word*>(p.src[blockIdx.y]) + ((long long)b * p.K * p.mid + m) * words + at;
    Word* dst = static_cast<Word*>(p.dst[blockIdx.y]) + ((long long)b * p.n * p.mid + m) * words + at;
    const long long row = p.mid * words;
    for (int j0 = 0; j0 < p.n; j0 += N) {
        Word w[N];
        uint64_t moved = 0u;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (j0 + j >= p.n) break;
            const int k = parent[j0 + j];
            if (k < 0 || k >= p.K || (p.in_place && k == j0 + j)) continue;
            w[j] = src[k * row];
            moved |= 1ull << j;
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (moved >> j & 1u) dst[(j0 + j) * row] = w[j];
    }
}

}  // namespace disco
