// Beam search: the selection over beams and vocabulary, and the reordering of the beams' states.
//
// Selection.  Of a sequence with K beams of score c_k and logits z_k[v], the n best continuations by
//     l[k, v] = c_k + z_k[v] - ln sum_w exp z_k[w],      ties to the lowest (k, v).
// Every logit is read once, by a pass that leaves two numbers for each chunk of neighbouring logits: the largest, and the sum of
// exp(z - largest).  (The 8-bit LM head's epilogue leaves the same.)  What follows looks at few logits: the n best of a row lie in the
// n chunks that come first by (largest logit, lowest index), since each of those holds a candidate that beats whatever lies in
// another chunk.  A row's n best then meet those of the sequence's other beams.  Scores are formed and compared in 64 bits: which of two
// candidates is the better is a whole number, and the scores of different beams may come as near to each other as they like.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "int8_head.cuh"   // warp_chunk_stats

namespace disco {

constexpr int kBeamChunk = 128;          // logits to a chunk of the pass over given logits
constexpr int kBeamWarpChunks = 8;       // chunks that a warp takes, so that 32 loads are on their way at once
constexpr int kBeamStatWarps = 8;
constexpr int kBeamThreads = 256;        // of the selection
constexpr int kBeamMaxKept = DISCO_MAX_KEPT;
constexpr int kBeamMaxBeams = DISCO_MAX_BEAMS;
constexpr int kBeamList = 512;           // candidates that are ranked by counting
constexpr int kBeamChunkList = 2 * kBeamMaxKept + 8;
constexpr int kBeamSmemKeys = 8192;      // chunks of a row whose keys are held in shared memory

struct BeamParams {
    const void* z;               // [B * K, V] logits, rows ld elements apart
    long long ld;
    int V, B, K, n;
    int eos;                     // the continuation of a finished beam (-1: none)
    const float* score;          // [B, K]
    const uint8_t* finished;     // [B, K] or null
    float2* stats;               // [B * K][chunks]
    int chunks;
    double* cand_score;          // [B * K][n] the best of each row, best first, and how many
    int32_t* cand_token;
    int32_t* cand_count;         // [B * K]
    unsigned int* tickets;       // [B], zero between calls
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
__device__ __forceinline__ float max_nan(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}

// Does the row's beam take part, and by its logits?
__device__ __forceinline__ bool beam_lives(float c) { return c > DISCO_NEG_INF && c < -DISCO_NEG_INF; }
__device__ __forceinline__ bool beam_expands(const BeamParams& p, int row) {
    return beam_lives(p.score[row]) && !(p.finished && p.finished[row]);
}

// The pass over the logits.  A warp takes eight chunks of a row; which lane holds which logit goes by its index alone, so that equal
// rows give equal sums wherever they lie.
template <typename T>
__global__ void __launch_bounds__(kBeamStatWarps * 32) beam_stats_kernel(const BeamParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * kBeamStatWarps + (threadIdx.x >> 5);
    const int per_row = (p.chunks + kBeamWarpChunks - 1) / kBeamWarpChunks;
    const long long row = w / per_row;
    if (row >= (long long)p.B * p.K) return;
    if (!beam_expands(p, (int)row)) return;
    const int first = (int)(w % per_row) * kBeamWarpChunks;
    const int v0 = first * kBeamChunk + lane;
    const T* z = static_cast<const T*>(p.z) + row * p.ld;
    float f[kBeamWarpChunks][4];
#pragma unroll
    for (int c = 0; c < kBeamWarpChunks; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int v = v0 + c * kBeamChunk + i * 32;
            f[c][i] = v < p.V ? load_logit(z + v) : DISCO_NEG_INF;
        }
    float2 mine = make_float2(0.f, 0.f);
#pragma unroll
    for (int c = 0; c < kBeamWarpChunks; ++c) {
        const float m = warp_max_nan_f32(max_nan(max_nan(f[c][0], f[c][1]), max_nan(f[c][2], f[c][3])));
        uint32_t e = 0u;
        if (m > DISCO_NEG_INF && m < -DISCO_NEG_INF) {
            const float s = (__expf(f[c][0] - m) + __expf(f[c][1] - m)) + (__expf(f[c][2] - m) + __expf(f[c][3] - m));
            e = __float2uint_rn(s * 0x1p24f);   // (128 terms of at most 1)
        }
        const float s = static_cast<float>(__reduce_add_sync(kFullMask, e)) * 0x1p-24f;
        if (lane == c) mine = make_float2(m, s);
    }
    if (lane < kBeamWarpChunks && first + lane < p.chunks) p.stats[row * p.chunks + first + lane] = mine;
}

// ---------------------------------------------------------------------------------------------
// the selection
// ---------------------------------------------------------------------------------------------
// Sum over the block; s is two sets of words, used in turn (one barrier).
__device__ __forceinline__ int block_sum(int x, int (*s)[kBeamThreads / 32], int& turn) {
    x = __reduce_add_sync(kFullMask, x);
    if ((threadIdx.x & 31) == 0) s[turn][threadIdx.x >> 5] = x;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kBeamThreads / 32; ++i) sum += s[turn][i];
    turn ^= 1;
    return sum;
}

// A threshold that between `want` and `cap` (>= want >= 1) of the N keys reach, or all of them where there are no more than cap: key(i)
// is 0 for what does not take part, and no two others are equal.  Bisection between lo, which more than cap reach, and hi, which fewer than
// want do, so that it ends when hi = lo + 1 at the latest.  *count: how many reach it.
template <typename Key>
__device__ __forceinline__ unsigned long long block_threshold(Key key, int N, int want, int cap, unsigned long long largest,
                                                              int (*s)[kBeamThreads / 32], int& turn, int* count) {
    auto reach = [&](unsigned long long t) {
        int c = 0;
        for (int i = threadIdx.x; i < N; i += kBeamThreads) c += key(i) >= t;
        return block_sum(c, s, turn);
    };
    unsigned long long lo = 1ull, hi = largest + 1ull;
    int c = reach(lo);
    unsigned long long t = lo;
    while (c > cap && hi - lo > 1ull) {
        t = lo + (hi - lo) / 2;
        c = reach(t);
        if (c < want) {
            hi = t;
            c = cap + 1;
        } else if (c > cap) {
            lo = t;
        }
    }
    *count = c;
    return t;
}

__device__ __forceinline__ unsigned long long ordered_bits64(double x) {
    const unsigned long long u = static_cast<unsigned long long>(__double_as_longlong(x));
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

// A CTA to a row; the last one of a sequence to be done goes on to its beams' candidates.
template <typename T, int CHUNK>
__global__ void __launch_bounds__(kBeamThreads) beam_select_kernel(const BeamParams p) {
    extern __shared__ uint32_t s_keys[];      // [min(chunks, kBeamSmemKeys)]
    __shared__ unsigned long long s_list[kBeamList];
    __shared__ int32_t s_pos[kBeamList];      // chunks of the row; then places of the candidates
    __shared__ int s_sum[2][kBeamThreads / 32];
    __shared__ double s_dsum[kBeamThreads / 32];
    __shared__ float s_max[kBeamThreads / 32];
    __shared__ int s_count, s_last;
    __shared__ int s_counts[kBeamMaxBeams];
    static_assert(kBeamChunkList <= kBeamList, "");

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int row = blockIdx.x, b = row / p.K;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int turn = 0;
    const float c = p.score[row];
    const bool over = p.finished && p.finished[row];
    double* cand_score = p.cand_score + (long long)row * p.n;
    int32_t* cand_token = p.cand_token + (long long)row * p.n;
    int found = 0;

    if (beam_lives(c) && over) {
        if (tid == 0) cand_score[0] = c, cand_token[0] = p.eos;
        found = 1;
    } else if (beam_lives(c)) {
        // soft-max statistics of the row
        const float2* stats = p.stats + (long long)row * p.chunks;
        const bool held = p.chunks <= kBeamSmemKeys;
        float m = DISCO_NEG_INF;
        for (int i = tid; i < p.chunks; i += kBeamThreads) {
            const float x = __ldcg(&stats[i].x);
            m = max_nan(m, x);
            if (held) s_keys[i] = x > DISCO_NEG_INF ? ordered_bits(__fadd_rn(x, 0.f)) : 0u;
        }
        m = warp_max_nan_f32(m);
        if (lane == 0) s_max[warp] = m;
        if (tid == 0) s_count = 0;
        __syncthreads();
        m = s_max[0];
#pragma unroll
        for (int i = 1; i < kBeamThreads / 32; ++i) m = max_nan(m, s_max[i]);
        if (m > DISCO_NEG_INF && m < -DISCO_NEG_INF) {   // (otherwise the row is no distribution)
            double sum = 0.0;
            for (int i = tid; i < p.chunks; i += kBeamThreads) {
                const float2 x = __ldcg(&stats[i]);
                if (x.x > DISCO_NEG_INF) sum += static_cast<double>(x.y) * static_cast<double>(expf(x.x - m));
            }
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(kFullMask, sum, off);
            if (lane == 0) s_dsum[warp] = sum;
            // the chunks that hold the n best
            auto chunk_key = [&](int i) -> unsigned long long {
                uint32_t k;
                if (held) {
                    k = s_keys[i];
                } else {
                    const float x = __ldcg(&stats[i].x);
                    k = x > DISCO_NEG_INF ? ordered_bits(__fadd_rn(x, 0.f)) : 0u;
                }
                return k ? (static_cast<unsigned long long>(k) << 32) | (0xffffffffu - static_cast<uint32_t>(i)) : 0ull;
            };
            const unsigned long long largest = (static_cast<unsigned long long>(ordered_bits(__fadd_rn(m, 0.f))) << 32) | 0xffffffffull;
            int L = 0;
            const unsigned long long t = block_threshold(chunk_key, p.chunks, p.n, 2 * p.n + 6, largest, s_sum, turn, &L);
            for (int i = tid; i < p.chunks; i += kBeamThreads)
                if (chunk_key(i) >= t) s_pos[atomicAdd(&s_count, 1)] = i;
            // their logits; where there are n chunks, none below the least of their largest counts
            const uint32_t floor_key = L >= p.n ? static_cast<uint32_t>(t >> 32) : 1u;
            const T* z = static_cast<const T*>(p.z) + (long long)row * p.ld;
            __syncthreads();
            auto value_key = [&](int i) -> unsigned long long {
                const int v = s_pos[i / CHUNK] * CHUNK + i % CHUNK;
                if (v >= p.V) return 0ull;
                const float x = load_logit(z + v);
                const uint32_t k = x > DISCO_NEG_INF ? ordered_bits(__fadd_rn(x, 0.f)) : 0u;
                return k >= floor_key ? (static_cast<unsigned long long>(k) << 32) | (0xffffffffu - static_cast<uint32_t>(v)) : 0ull;
            };
            if (tid == 0) s_count = 0;
            __syncthreads();
            for (int i = tid; i < L * CHUNK; i += kBeamThreads) {
                const unsigned long long k = value_key(i);
                if (k) {
                    const int at = atomicAdd(&s_count, 1);
                    if (at < kBeamList) s_list[at] = k;
                }
            }
            __syncthreads();
            int N = s_count;
            if (N > kBeamList) {   // many equal logits
                const unsigned long long u = block_threshold(value_key, L * CHUNK, p.n, kBeamList, largest, s_sum, turn, &N);
                if (tid == 0) s_count = 0;
                __syncthreads();
                for (int i = tid; i < L * CHUNK; i += kBeamThreads) {
                    const unsigned long long k = value_key(i);
                    if (k >= u) s_list[atomicAdd(&s_count, 1)] = k;
                }
                __syncthreads();
            }
            sum = s_dsum[0];
#pragma unroll
            for (int i = 1; i < kBeamThreads / 32; ++i) sum += s_dsum[i];
            for (int i = tid; i < N; i += kBeamThreads) {
                const unsigned long long k = s_list[i];
                int rank = 0;
                for (int j = 0; j < N; ++j) rank += s_list[j] > k;
                if (rank < p.n) {
                    const double x = from_ordered_bits(static_cast<uint32_t>(k >> 32));
                    cand_score[rank] = static_cast<double>(c) + (x - (static_cast<double>(m) + log(sum)));
                    cand_token[rank] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(k));
                }
            }
            found = min(N, p.n);
        }
    }
    if (tid == 0) p.cand_count[row] = found;
    __threadfence();
    __syncthreads();
    if (tid == 0) s_last = atomicAdd(p.tickets + b, 1u) == static_cast<unsigned int>(p.K) - 1u;
    __syncthreads();
    if (!s_last) return;
    __threadfence();

    // ---- the sequence: candidates of its beams, by score and then by place (beam by beam, each beam's best first) ----
    if (tid < p.K) s_counts[tid] = __ldcg(p.cand_count + b * p.K + tid);
    if (tid == 0) s_count = 0, p.tickets[b] = 0u;
    __syncthreads();
    const double* scores = p.cand_score + (long long)b * p.K * p.n;
    const int M = p.K * p.n;
    auto score_key = [&](int i) -> unsigned long long {
        return i % p.n < s_counts[i / p.n] ? ordered_bits64(__dadd_rn(__ldcg(scores + i), 0.0)) : 0ull;
    };
    unsigned long long t = 1ull;
    int last = M;            // of those that are equal to t: places up to this one
    if (M > kBeamList) {
        int reached = 0;
        t = block_threshold(score_key, M, p.n, kBeamList, 0xfffffffffffffffeull, s_sum, turn, &reached);
        if (reached > kBeamList) {
            // (equal scores: the bisection ended with two neighbours, of which the lower one is reached by too many; it is the one
            // that a step above is reached by fewer than n)
            auto above = [&](unsigned long long u) {
                int x = 0;
                for (int i = tid; i < M; i += kBeamThreads) x += score_key(i) >= u;
                return block_sum(x, s_sum, turn);
            };
            if (above(t) < p.n) t -= 1ull;
            const int need = p.n - above(t + 1ull);
            int lo = -1, hi = M - 1;     // up to place hi there are enough
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                int x = 0;
                for (int i = tid; i <= mid; i += kBeamThreads) x += score_key(i) == t;
                if (block_sum(x, s_sum, turn) >= need) hi = mid;
                else lo = mid;
            }
            last = hi;
        }
    }
    for (int i = tid; i < M; i += kBeamThreads) {
        const unsigned long long k = score_key(i);
        if (k > t || (k == t && i <= last)) {
            const int at = atomicAdd(&s_count, 1);
            s_list[at] = k;
            s_pos[at] = i;
        }
    }
    __syncthreads();
    const int N = s_count;
    const long long out = (long long)b * p.n;
    // (what is read of the beams is read before anything is written: the outputs may take the inputs' place)
    constexpr int kEach = kBeamList / kBeamThreads;
    int rank[kEach], parent[kEach], token[kEach];
    float score[kEach];
    bool ends[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int i = e * kBeamThreads + tid;
        rank[e] = p.n;
        if (i >= N) continue;
        const unsigned long long key = s_list[i];
        const int pos = s_pos[i];
        int r = 0;
        for (int j = 0; j < N; ++j) r += s_list[j] > key || (s_list[j] == key && s_pos[j] < pos);
        if (r >= p.n) continue;
        rank[e] = r;
        parent[e] = pos / p.n;
        token[e] = __ldcg(p.cand_token + (long long)b * M + pos);
        score[e] = static_cast<float>(__ldcg(scores + pos));
        ends[e] = token[e] == p.eos || (p.finished && p.finished[b * p.K + parent[e]]);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (rank[e] >= p.n) continue;
        p.score_out[out + rank[e]] = score[e];
        p.parent[out + rank[e]] = parent[e];
        p.token[out + rank[e]] = token[e];
        if (p.finished_out) p.finished_out[out + rank[e]] = ends[e];
    }
    for (int i = N + tid; i < p.n; i += kBeamThreads) {
        p.score_out[out + i] = DISCO_NEG_INF;
        p.parent[out + i] = -1;
        p.token[out + i] = -1;
        if (p.finished_out) p.finished_out[out + i] = 0;
    }
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
