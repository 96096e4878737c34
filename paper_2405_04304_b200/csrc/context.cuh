// The context behind the C ABI and the host-side helpers that its source files share.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <mutex>

#include "common.cuh"

struct disco_ctx {
    int device;
    int V, d_draft, d_target, max_batch, max_rows, clf_hidden;
    int sm_count;
    size_t smem_optin;
    int path;
    int pdl;  // launch the streaming kernel with programmatic stream serialization (DISCO_PDL=0 turns it off)
    long long launches;
    cudaStream_t last_stream;  // stream of the most recent enqueue (disco_last_device_status waits for it only)
    unsigned int test_stamp_skew;  // disco_test_hooks
    void* device_mem;  // every device buffer below
    void* host_mem;    // the pinned staging below
    // scratch for cross-block reductions
    int part_rows;  // rows the partial buffers can hold
    int max_grid;
    unsigned long long* keys;
    unsigned int* ticket;
    int* status;
    float* final_stats;            // [part_rows][2] (m, Z) of the rows of a pass
    float* final_stats2;           // the same for the second pass of a feature extraction
    uint8_t* chain_alive;          // [max_batch] draft phase on the device: which sequences still draft
    double* sample_seg_tot;        // verification with sampling: [max_batch][kSampleMaxSegments][2] sums of weights
    int32_t* sample_seg_last;      //   the same shape: last index with positive weight
    unsigned int* sample_tickets;  //   [max_batch]
    void* pack_rows;               // fixed-shape verification with many rows: the rows that count, packed
    int32_t* pack_off;             // [max(max_batch, max_rows) + 1] their offsets; the last entry is the row count
    void* loop_rec;                // persistent draft-phase kernel: stamped 80-byte records, [4][CTA]; written by nothing else
    void* part_rec;                // draft step: 64-byte partial records, [sequence][CTA]
    void* stamped_rec;             // batched draft step: stamped 80-byte records, [sequence][CTA]; written by nothing else
    unsigned int* row_bound;       // batched draft step: two sets of [part_rows][kDbBoundStride] words, see DraftBatchParams
    int8_t* int8_rows;             // hidden rows in 8 bits: [part_rows][int8_pitch]
    float* int8_scale;             //   and their scales
    int int8_pitch;
    float2* beam_stats;            // soft-max statistics of part_rows rows of logits: BeamLayout
    int part_slots;                // partials per row the buffers can hold
    void* encode_tiled;            // cuTensorMapEncodeTiled, resolved through the runtime
    void* pointer_attributes;      // cuPointerGetAttributes, the same way
    // device staging for the *_host entry points
    void* stage_hidden;
    void* stage_hidden_draft;      // disco_iteration_host: the draft hidden states of all steps
    int32_t* stage_dev;            // disco_iteration_host: pos0 | sl_forced (max_batch each) | draft_ids (max_rows)
    cudaStream_t copy_stream;      // disco_iteration_host: the target hidden states travel beside the draft phase
    cudaEvent_t copy_done;
    // Small inputs and outputs of the *_host entry points live in pinned host memory that the GPU maps:
    // the kernels read and write it in place, so a host call costs one copy (the hidden states), one
    // launch and one synchronisation.  *_h: host address, *_d: the same memory as the device sees it.
    int32_t *stage_int_h, *stage_int_d;    // pos | n_drafted | token | draft_ids | row_off | n_accept | bonus | target_ids
    float *stage_float_h, *stage_float_d;  // conf | feats
    uint8_t *stage_byte_h, *stage_byte_d;  // active | halt
};

namespace disco {

constexpr int kMaxHidden = 16384;    // widest hidden dimension the kernels accept
constexpr int kMaxDevices = 64;

// One-time, per-device configuration of one kernel (its dynamic shared-memory limit).  Every template
// instance of a launcher owns one of these; the lock makes first calls from several host threads, and
// contexts on several devices, safe.
struct KernelSetup {
    std::mutex mu;
    bool done[kMaxDevices] = {};
    size_t dyn_limit[kMaxDevices] = {};
};

// With DISCO_DEBUG set in the environment, failed CUDA runtime calls are reported on stderr.
inline bool cuda_ok(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return true;
    static const bool verbose = std::getenv("DISCO_DEBUG") != nullptr;
    if (verbose) std::fprintf(stderr, "[disco] %s: %s\n", what, cudaGetErrorString(e));
    return false;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Raise a kernel's dynamic shared-memory limit once per device: to `bytes`, or (bytes == 0) to all that the
// device allows beside the kernel's static shared memory.  *limit receives the value in force.
template <typename Kern>
inline bool raise_smem_limit(const disco_ctx* c, KernelSetup& ks, Kern kern, size_t bytes, size_t* limit) {
    if (c->device < 0 || c->device >= kMaxDevices) return false;
    std::lock_guard<std::mutex> lock(ks.mu);
    if (!ks.done[c->device]) {
        size_t want = bytes;
        if (want == 0) {
            cudaFuncAttributes fa;
            if (!cuda_ok(cudaFuncGetAttributes(&fa, kern), "cudaFuncGetAttributes")) return false;
            want = c->smem_optin - fa.sharedSizeBytes;
        }
        if (!cuda_ok(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)want),
                     "cudaFuncSetAttribute"))
            return false;
        ks.dyn_limit[c->device] = want;
        ks.done[c->device] = true;
    }
    if (limit) *limit = ks.dyn_limit[c->device];
    return true;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Clusters of CTAs (1: none), and programmatic stream serialization where that is on.
inline int launch_attributes(const disco_ctx* c, int cluster, cudaLaunchAttribute (&attr)[2]) {
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (c->pdl) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    return n;
}

// Launch a small follow-up kernel with programmatic stream serialization (it waits with griddepcontrol.wait
// before it reads anything), so that its launch latency hides behind the kernel before it.
template <typename... KArgs, typename... Args>
cudaError_t launch_after(const disco_ctx* c, void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st,
                         Args... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = c->pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

// The bounded waits of disco_beams.cu's kernels (common.cuh: one copy of the budget per source file).
int set_beam_wait_budget(long long clocks);

}  // namespace disco
