// project.cuh -- what the kernels of ecasq_project and ecasq_gated share.
#pragma once

#include "epilogue.cuh"

namespace ecasq {

struct ProjectArgs {
    const void *x, *levels, *scales;
    const uint8_t *codes;
    void *y;
    int32_t *status;
    int64_t x_row, code_row, scale_row, y_row, n, k, b;  // n: outputs a row of x; a gated matrix has 2n rows
    int32_t m, group, type, scale_type;
    bool gated;
    uint32_t lost;  // test hook: 1 where blocks begin as if a wait had run out
    Epilogue epi;
};

// How a call with more than eight rows of x is shared out; width 0: it goes to the matrix-vector kernels.
struct ProjectPlan {
    int32_t width, split, held;       // rows of x of a tile; blocks of a cluster that share its columns; clusters, or for tiles of 256 rows pairs of blocks, that the card holds
    int64_t x_tiles, w_tiles, panel;  // tiles of rows of x, and of the matrix; tiles of rows of x that all tiles of the matrix go by before the next ones
};
ProjectPlan plan_project_tc(int64_t b, int64_t n, int64_t k, int32_t type, int32_t group, bool gated);

void project_tc_rings(int width, bool f32, bool gated, int32_t *rings);

// The matrix-vector kernels, which read the matrix again for each eight rows of x.
int launch_project_few(const ProjectArgs &p, cudaStream_t st);
// Tensor cores, or those where they are faster; the workspace it may need.
int launch_project_tc(const ProjectArgs &p, void *ws, size_t ws_bytes, cudaStream_t st);
size_t project_tc_room(int64_t b, int64_t k, int32_t type);

}  // namespace ecasq
