"""Host-only checks of the 8-bit LM head's tiling (compiled from the kernels' own header, run on the CPU), and of what the beam-search entry
points refuse before they touch a GPU."""
import ctypes
import os
import subprocess

from paper_2405_04304_b200 import binding, build

_TILING = r"""
#include "int8_head.cuh"
#include <cstdio>
using namespace disco;
int main() {
    const int grids[] = {1, 3, 147, 148}, vs[] = {1, 31, 128, 129, 300, 4000, 32000, 40011, 49152, 151936};
    for (int grid : grids)
        for (int V : vs)
            for (int R = 1; R < 5000; R += R < 300 ? 1 : 61)
                for (int kind = 0; kind < 3; ++kind) {
                    const bool pairs = kind == kI8Pair;
                    if (pairs && grid < 2) continue;
                    const int ctas = pairs ? 2 : 1;
                    const Int8Tiling t = Int8Tiling::make(R, V, grid, (Int8Kind)kind);
                    bool ok = t.N % (16 * ctas) == 0 && t.N >= 16 && t.N <= 256 && (long long)t.MT * t.N >= R && (long long)(t.MT - 1) * t.N < R;
                    ok = ok && t.TR >= 1 && t.TR <= 256 && t.w_box <= 128 * t.blocks && t.w_box * ctas == t.TR && (long long)t.NV * t.TR >= V && (long long)(t.NV - 1) * t.TR < V;
                    ok = ok && t.w_box % kI8Chunk == 0 && (long long)t.rounds * (grid / ctas) >= (long long)t.MT * t.NV;
                    // accumulators of all buffers, as columns of tensor memory; reads of 32 columns end inside theirs
                    ok = ok && t.bufs * t.blocks * t.cols <= 512 && t.cols >= t.N && t.cols % 32 == 0;
                  for (int d : {8, 136, 768, 5120, 6144, 16384}) {
                    const bool few = !pairs && Int8Ring::few(R, V, d);
                    const Int8Ring r = Int8Ring::make(t, d, 227 * 1024 - kI8TurnBytes, few);
                    ok = ok && r.stages >= 2 && r.stages <= kI8MaxStages && kI8FixedSmem + kI8TurnBytes + r.bytes + r.resident <= 227 * 1024;
                    ok = ok && r.w_bytes % 1024 == 0 && r.x_bytes % 1024 == 0 && r.w_bytes >= t.w_box * kI8BK;
                    // the hidden-row boxes of a tile are what its MMA takes, or all there are
                    ok = ok && (pairs ? 2 * t.x_box == t.N : t.x_box == t.N || (t.x_box >= R && t.x_box % 8 == 0));
                    if (few) { ok = ok && R <= kI8EpiWarps && t.MT == 1 && t.N == 16 && d <= kI8EpiWarps / R * 256 * kI8FewChunks && r.resident >= (d + 127) / 128 * 128 * t.N && r.resident % 1024 == 0; }
                    else ok = ok && r.x_bytes * ctas >= t.N * kI8BK;
                    // what the last stage's MMAs read
                    ok = ok && (r.stages - 1) * r.w_bytes + t.blocks * 128 * kI8BK <= r.bytes && r.stages * (r.w_bytes + r.x_bytes) <= r.bytes;
                  }
                    // no more rounds of items than the largest tiles need
                    const int most = kind == kI8One ? 128 : 256, workers = grid / ctas;
                    const long long whole = (long long)t.MT * ((V + most - 1) / most);
                    ok = ok && t.rounds <= (whole + workers - 1) / workers;
                    if (!ok) return std::printf("R %d V %d grid %d kind %d\n", R, V, grid, kind), 1;
                }
    // which kind is taken, at sizes where all three were measured
    struct { int R, V, d, kind; } taken[] = {{11, 32000, 5120, kI8Two}, {24, 49152, 2048, kI8Two}, {64, 32000, 768, kI8One}, {200, 32000, 768, kI8One},
        {300, 32000, 768, kI8One}, {200, 32000, 5120, kI8Pair}, {256, 32000, 5120, kI8Pair}, {320, 32000, 5120, kI8Pair}, {704, 32000, 5120, kI8Pair},
        {256, 49152, 2048, kI8Pair}, {200, 20000, 3000, kI8Two}, {200, 12000, 5120, kI8Pair}, {100, 40011, 1000, kI8One}};
    for (auto& m : taken) {
        const Int8Tiling t = Int8Tiling::choose(m.R, m.V, m.d, 148);
        if (t.kind != m.kind) return std::printf("kind: %d rows, %d x %d: %d\n", m.R, m.V, m.d, t.kind), 1;
    }
    return 0;
}
"""


_DEAL = r"""
#include "beam.cuh"
#include <cstdio>
#include <cstring>
using namespace disco;
static unsigned char seen[64 * 20000];
int main() {
    for (int K = 1; K <= DISCO_MAX_BEAMS; ++K)
        for (int chunks : {1, 2, 7, 31, 32, 33, 250, 256, 313, 384, 512, 1000, 1251, 1536, 2048, 8594, 19000})
            for (int n : {1, 10, 11, 24, 25, 128}) {
                const int warps = BeamDeal::warps(K, chunks, n);
                const BeamDeal d = BeamDeal::make(K, chunks, warps);
                bool ok = (warps == 8 || warps == 16 || warps == 32) && (d.two ? K <= 2 * warps : K * d.share <= warps) && d.merged >= 1;
                ok = ok && (long long)d.pieces * d.merged >= chunks && (long long)(d.pieces - 1) * d.merged < chunks && d.used <= (d.two ? kBeamItems / 2 : kBeamItems);
                // every piece of every row belongs to one lane's items, by the same arithmetic as the kernel's
                std::memset(seen, 0, sizeof(seen));
                for (int w = 0; w < warps; ++w)
                    for (int lane = 0; lane < 32; ++lane)
                        for (int j = 0; j < kBeamItems; ++j) {
                            const int half = kBeamItems / 2, row0 = d.two ? w : w / d.share, share = d.two ? 0 : w - row0 * d.share;
                            if ((d.two ? j & (half - 1) : j) >= d.used) continue;
                            const int k = d.two && j >= half ? row0 + 32 : row0, piece = ((d.two ? j & (half - 1) : j) * d.share + share) * 32 + lane;
                            if (k < K && piece < d.pieces) ++seen[k * 20000 + piece];
                        }
                for (int k = 0; k < K; ++k)
                    for (int i = 0; i < d.pieces; ++i) ok = ok && seen[k * 20000 + i] == 1;
                if (!ok) return std::printf("K %d chunks %d n %d\n", K, chunks, n), 1;
            }
    return beam_joined(1, 4, 32) && !beam_joined(20, 5, 40) && !beam_joined(64, 4, 32) ? 0 : 2;
}
"""


def _run(tmp_path, source):
    src, exe = tmp_path / "rules.cu", tmp_path / "rules"
    src.write_text(source)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", build.CSRC, "-I", include, "-o", str(exe),
                    str(src)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0, (run.returncode, run.stdout)


def test_int8_tiling_covers_everything_and_stays_in_its_memory(tmp_path):
    _run(tmp_path, _TILING)


def test_every_piece_of_every_row_is_dealt_to_one_lane(tmp_path):
    _run(tmp_path, _DEAL)


def test_null_contexts_are_refused():
    build.build()
    lib = binding.load()
    z = ctypes.c_void_p(None)
    assert lib.disco_quantize_rows(None, z, 0, 8, 1, 8, z, 16, z, z) == binding.ERR_INVALID_ARG
    assert lib.disco_project_int8(None, z, 16, z, z, 1, 8, 8, 1, z, 0, 1, z) == binding.ERR_INVALID_ARG
    assert lib.disco_beam_select(None, z, 0, 1, 1, 1, z, z, -1, 1, z, z, z, z, z) == binding.ERR_INVALID_ARG
    assert lib.disco_beam_step_int8(None, z, 16, z, z, 1, 8, 8, 1, 1, z, z, -1, 1, z, z, z, z, z, z) == binding.ERR_INVALID_ARG
    assert lib.disco_beam_reorder(None, z, z, 1, 1, 1, 1, z, z, 1, 1, 1, z) == binding.ERR_INVALID_ARG


def test_int8_pitch():
    assert [binding.int8_pitch(d) for d in (8, 16, 24, 768, 1000)] == [16, 16, 32, 768, 1008]
