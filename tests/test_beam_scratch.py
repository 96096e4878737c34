"""Host-only checks of where the soft-max statistics of rows of logits lie, and of counts of logits (compiled from the kernels' own header,
run on the CPU)."""
from test_beam_rules import _run

_LAYOUT = r"""
#include "beam.cuh"
#include <cstdio>
using namespace disco;
int main() {
    for (int V = 1; V < 1 << 28; V += V < 6000 ? 1 : V / 7)
        for (int room : {1, 2, 3, 6, 31, 32, 64, 256, 4352}) {
            const BeamLayout l(V);
            const size_t bytes = l.bytes(room);      // what a context of this many rows has
            bool ok = (long long)l.i8_chunks * kI8Chunk >= V && (long long)l.chunks * kBeamChunk >= V && l.segs * kBeamWarpChunks >= l.chunks;
            for (int rows : {1, room / 2, room - 1, room}) {
                if (rows < 1) continue;
                // as the kernels index them: [row][segment] pairs, [row][chunk] floats; or [row][chunk of the 8-bit head] pairs
                const size_t sums_end = ((size_t)(rows - 1) * l.segs + l.segs) * sizeof(float2);
                const size_t tops = l.tops_at(rows) * sizeof(float), tops_end = tops + ((size_t)(rows - 1) * l.chunks + l.chunks) * sizeof(float);
                ok = ok && sums_end <= tops && tops_end <= bytes && (size_t)rows * l.i8_chunks * sizeof(float2) <= bytes;
            }
            if (!ok) return std::printf("V %d, %d rows\n", V, room), 1;
        }
    // the logits of as many pieces as are looked into, by the deals of all numbers of beams
    for (int K = 1; K <= DISCO_MAX_BEAMS; ++K)
        for (int chunk : {kI8Chunk, kBeamChunk}) {
            const BeamLayout l(kBeamMaxVocab);
            const int chunks = chunk == kI8Chunk ? l.i8_chunks : l.chunks, warps = BeamDeal::warps(K, chunks, 1);
            const BeamDeal d = BeamDeal::make(K, chunks, warps);
            const long long width = (long long)d.merged * chunk, values = kBeamPieceList * width + 8 * kBeamThreads;
            if (values > 0x7fffffffll || d.pieces * width + 8 * kBeamThreads > 0x7fffffffll) return std::printf("K %d chunk %d\n", K, chunk), 2;
        }
    return 0;
}
"""


def test_statistics_lie_within_the_contexts_scratch_and_counts_within_32_bits(tmp_path):
    _run(tmp_path, _LAYOUT)
