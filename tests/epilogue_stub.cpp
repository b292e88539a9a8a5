// Which warp of a matrix product's epilogue has which chunk of a tile (linear.cuh), for test_epilogue_chunks_cpu.py.
#include <cuda.h>
#include <cuda_runtime.h>

#include "../paper_2608_23429_gb300/csrc/linear.cuh"

using namespace cbk;

extern "C" {
int stub_warps(int results, int mx) { return epi_warps((Results)results, mx != 0); }
// The warp's place among those of its quarter that has chunk `chunk` of the kernel's tile number `tile`, or -1 (nobody, or more than one).
int stub_owner(int results, int mx, int passes, int tile, int chunk, int chunks) {
    const Results r = (Results)results;
    int owner = -1;
    for (int share = 0; share < epi_warps(r, mx != 0) / 4; ++share) {
        int begin = epi_first_chunk(r, share);
        for (int t = 0; t < tile; ++t) begin = epi_next_first_chunk(r, passes != 0, begin);
        for (int c = begin; c < chunks; c = epi_chunk_behind(r, mx != 0, c)) {
            if (c != chunk) continue;
            if (owner >= 0) return -1;
            owner = share;
        }
    }
    return owner;
}
}
