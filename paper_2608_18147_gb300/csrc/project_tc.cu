// project_tc.cu -- ecasq_project and ecasq_gated on the tensor cores: the host's part, and the kernels of ecasq_project.
#include <iterator>

#include "project_tc.cuh"

namespace ecasq {

// ---------------------------------------------------------------- x in rows that tile_load can read
// 16-bit rows copied to rows of `to_row` elements, a multiple of 8; fp32 rows as three bf16 terms, of 8 bits each, in three planes of b rows.  A value that is not finite is its last term
// alone, which is multiplied by the levels' first terms and by no other: theirs are zero only where the level is (an infinity times a lower term that is zero would be NaN).
template <bool F32> __global__ void __launch_bounds__(256) k_lay_out(const void *x, int64_t x_row, int64_t b, int64_t k, uint16_t *to, int64_t to_row) {
    wait_before();
    for (int64_t i = blockIdx.y; i < b; i += gridDim.y) {
        const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
        if (c >= k) continue;
        if (F32) {
            float v = static_cast<const float *>(x)[i * x_row + c];
            const bool finite = fabsf(v) <= 3.402823466e38f;
#pragma unroll
            for (int p = 0; p < 3; p++) {
                const uint32_t bits = __float_as_uint(v) >> 16;
                to[(p * b + i) * to_row + c] = finite ? (uint16_t)bits : p < 2 ? 0 : v == v ? (uint16_t)bits : 0x7FFF;
                if (finite) v -= __uint_as_float(bits << 16);
            }
        } else {
            to[i * to_row + c] = static_cast<const uint16_t *>(x)[i * x_row + c];
        }
    }
}

int make_tile_map(CUtensorMap *map, CUtensorMapDataType type, const void *at, int64_t cols, int64_t rows, int64_t row_bytes, int box_cols, int box_rows,
                  CUtensorMapSwizzle swizzle) {
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<void *> found;
    void *fn = found.load(std::memory_order_acquire);
    if (!fn) {
        cudaDriverEntryPointQueryResult got;
        ECASQ_CUDA_TRY(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &got));
        if (got != cudaDriverEntryPointSuccess || !fn) return ECASQ_ECUDA;
        found.store(fn, std::memory_order_release);
    }
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)row_bytes};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, one[2] = {1, 1};
    const CUresult rc = reinterpret_cast<Encode>(fn)(map, type, 2, const_cast<void *>(at), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                                                     CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? ECASQ_OK : ECASQ_ECUDA;
}

// The rows of x that lie in the workspace, and how far apart.
static int64_t laid_row(int64_t k) { return (k + 7) / 8 * 8; }
size_t project_tc_room(int64_t b, int64_t k, int32_t type) { return align256((size_t)(b * laid_row(k)) * 2 * (type == ECASQ_F32 ? 3 : 1)); }

constexpr int64_t kPanelBytes = 24 << 20;

// Blocks whose sums are taken out together, for groups of whole blocks: kSpanMost where groups hold that many evenly, or there is one group.
static int32_t span_blocks(int64_t group, int64_t blocks) { return group / 128 >= blocks || group / 128 % kSpanMost == 0 ? (int32_t)std::min<int64_t>(kSpanMost, blocks) : 1; }

ProjectPlan plan_project_tc(int64_t b, int64_t n, int64_t k, int32_t type, int32_t group, bool gated) {
    const bool f32 = type == ECASQ_F32;
    const int64_t blocks = cdiv(k, 128), rows = gated ? 2 * n : n;
    ProjectPlan plan{};
    // The width of a tile and the blocks of a cluster that share its columns that take the least time: rounds of tiles over the card, each of its blocks of
    // columns one after another, whose time goes by the width and by the scale groups in one (measured: 0.27 + 0.35 us a group for 128 rows of x), and of
    // the tile's start and results.  Only tiles of 256 rows take pairs of blocks; clusters of more than two leave some SMs out (kHeld: what the card holds
    // of each size).
    struct Choice {
        int width, block, group, tile;  // rows of x; hundredths of a microsecond
    };
    static constexpr Choice kChoices[] = {{32, 24, 21, 110}, {64, 23, 28, 190}, {128, 27, 35, 350}, {256, 38, 40, 690}};
    static constexpr int kHeld[] = {152, 76, 46, 36, 28, 23};
    static_assert(sizeof kHeld / sizeof *kHeld == kSplitMost, "");
    const int terms = f32 ? 6 : 1, share = f32 ? std::min(group, 128) : group % 128 ? std::min(group, 1 << 20) : 128 * span_blocks(group, blocks);
    int64_t best = INT64_MAX;
    for (const Choice &c : kChoices) {
        const bool pair = c.width == 256;
        const int64_t tiles = cdiv(n, (gated ? 64 : 128) * (pair ? 2 : 1)) * cdiv(b, c.width);
        for (int s = 1; s <= (pair ? 1 : kSplitMost) && s <= blocks; s++) {
            const int held = pair ? 76 : kHeld[s - 1];
            const int64_t cost = cdiv(tiles, held) * (cdiv(blocks, s) * terms * (c.block + c.group * 128 / share) + c.tile + (s > 1 ? 20 + 30 * s : 0));
            if (cost >= best) continue;
            best = cost;
            plan.width = c.width;
            plan.split = s;
            plan.held = held;
        }
        if (c.width >= b) break;
    }
    // The matrix-vector kernels, a pass for each eight rows, are the faster ones for small matrices (300 x 8192 by 16 rows: 6.3 us, and 11.8 here; 1024 x 1024
    // 6.8 and 8.3; 4096 x 4096 13.3 and 11.5).  Their blocks take 3.2 us each and their codes at 16 bytes a nanosecond (fp32 6.2 us, 2.4 bytes), a round
    // of 152 after another; these stand at 5 us for a launch, 2 for rows of x that are laid out first, and what is counted above.
    const int64_t few_blocks = std::min<int64_t>(cdiv(n, 8), 152), few = cdiv(few_blocks * cdiv(b, 8), 152) * ((f32 ? 620 : 320) + rows * k / 2 / few_blocks / (f32 ? 24 : 158));
    if (few < best + (f32 ? 700 : 500)) return ProjectPlan{};
    plan.x_tiles = cdiv(b, plan.width);
    plan.w_tiles = cdiv(n, (gated ? 64 : 128) * (plan.width == 256 ? 2 : 1));
    plan.panel = std::max<int64_t>(1, std::min<int64_t>(plan.x_tiles, kPanelBytes / (plan.width * k * 2 * (f32 ? 3 : 1))));
    plan.panel = cdiv(plan.x_tiles, cdiv(plan.x_tiles, plan.panel));  // (panels alike)
    return plan;
}

template <int ND, int NH, bool GATED, bool F32> static void rings_of(int32_t *to) {
    using Shape = TcShape<ND, NH, GATED, F32>;
    const int32_t rings[] = {Shape::kTeams, Shape::kCodeStages, Shape::kCodeBars, Shape::kXStages, Shape::kAStages / 2, NH, Shape::kDBufs};
    std::copy(std::begin(rings), std::end(rings), to);
}
template <bool GATED, bool F32> static void rings_of_width(int width, int32_t *to) {
    if (width == 32) rings_of<32, 1, GATED, F32>(to);
    else if (width == 64) rings_of<64, 1, GATED, F32>(to);
    else if (width == 128) rings_of<128, 1, GATED, F32>(to);
    else rings_of<128, 2, GATED, F32>(to);
}
void project_tc_rings(int width, bool f32, bool gated, int32_t *rings) {
    if (gated) f32 ? rings_of_width<true, true>(width, rings) : rings_of_width<true, false>(width, rings);
    else f32 ? rings_of_width<false, true>(width, rings) : rings_of_width<false, false>(width, rings);
}

int launch_project_tc(const ProjectArgs &p, void *ws, size_t ws_bytes, cudaStream_t st) {
    const ProjectPlan plan = plan_project_tc(p.b, p.n, p.k, p.type, p.group, p.gated);
    if (!plan.width) return launch_project_few(p, st);
    const bool f32 = p.type == ECASQ_F32, pair = plan.width == 256;
    const int64_t rows = p.gated ? 2 * p.n : p.n, tiles = plan.w_tiles * plan.x_tiles;
    if (tiles > INT32_MAX - 1024) return ECASQ_EINVAL;  // (a block's last step goes beyond them by at most a card's clusters)
    TcArgs a{};
    a.levels = p.levels;
    a.scales = p.scales;
    a.y = p.y;
    a.status = p.status;
    a.scale_row = p.scale_row;
    a.y_row = p.y_row;
    a.n = p.n;
    a.b = p.b;
    a.k = p.k;
    a.second = p.n;
    a.m = p.m;
    a.group = p.group;
    a.type = p.type;
    a.scale_type = p.scale_type;
    a.blocks = (int32_t)cdiv(p.k, 128);
    a.span_blocks = span_blocks(p.group, a.blocks);
    a.split = plan.split;
    a.x_tiles = (int32_t)plan.x_tiles;
    a.w_tiles = (int32_t)plan.w_tiles;
    a.tiles = (int32_t)tiles;
    a.panel = (int32_t)plan.panel;
    a.lost = p.lost;
    a.epi = p.epi;
    const int64_t piece = 4 * type_size(p.type);
    const auto in_pieces = [&](const void *at, int64_t row) { return reinterpret_cast<uintptr_t>(at) % piece == 0 && (p.b == 1 || row % 4 == 0); };
    a.wide = in_pieces(p.y, p.y_row) && in_pieces(p.epi.residual, p.epi.residual_row);
    const void *x = p.x;
    int64_t x_row = p.x_row;
    if (f32 || !aligned16(p.x) || (p.b > 1 && p.x_row % 8)) {
        if (!ws || ws_bytes < project_tc_room(p.b, p.k, p.type) || !aligned16(ws)) return ECASQ_EWORKSPACE;
        const dim3 grid((unsigned)cdiv(p.k, 256), (unsigned)std::min<int64_t>(p.b, 4096));
        const int rc = f32 ? launch_early(k_lay_out<true>, grid, 256, 0, st, p.x, p.x_row, p.b, p.k, static_cast<uint16_t *>(ws), laid_row(p.k))
                           : launch_early(k_lay_out<false>, grid, 256, 0, st, p.x, p.x_row, p.b, p.k, static_cast<uint16_t *>(ws), laid_row(p.k));
        if (rc) return rc;
        x = ws;
        x_row = laid_row(p.k);
    }
    CUtensorMap xm, cm;
    const int x_rows = std::min(plan.width, 128) / (pair ? 2 : 1);
    int rc = make_tile_map(&xm, p.type == ECASQ_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, x, p.k, f32 ? 3 * p.b : p.b,
                           (p.b > 1 || f32 ? x_row : laid_row(p.k)) * 2, 64, x_rows, CU_TENSOR_MAP_SWIZZLE_128B);
    if (!rc) rc = make_tile_map(&cm, CU_TENSOR_MAP_DATA_TYPE_UINT8, p.codes, 64 * cdiv(p.k, 128), rows, p.code_row, 64, 64, CU_TENSOR_MAP_SWIZZLE_64B);
    if (rc) return rc;
    return p.gated ? launch_tc_gated(plan.width, xm, cm, a, st) : launch_tc_width<false>(plan.width, xm, cm, a, st);
}

}  // namespace ecasq
