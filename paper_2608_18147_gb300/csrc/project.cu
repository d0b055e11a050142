// project.cu -- ecasq_project and ecasq_gated: the entry points, and the choice of the kernel.
#include "matvec.cuh"
#include "project.cuh"

namespace ecasq {

// Rows of x up to which the matrix-vector kernels take every call, one pass of theirs; plan_project_tc sends them calls with more rows where it counts them the faster ones.  28672 x 8192 by eight rows takes them 36 us, by sixteen, in two passes, twice that,
// and the tensor cores 53 (8192 x 8192: 16, twice that and 21).
constexpr int64_t kFewRows = 8;

int launch_project_few(const ProjectArgs &p, cudaStream_t st) {
    MatvecArgs a{};
    a.x = p.x;
    a.levels = p.levels;
    a.scales = p.scales;
    a.codes = p.codes;
    a.y = p.y;
    a.status = p.status;
    a.x_row = p.x_row;
    a.code_row = p.code_row;
    a.scale_row = p.scale_row;
    a.y_row = p.y_row;
    a.n = p.n;
    a.k = p.k;
    a.b = (int32_t)p.b;
    a.m = p.m;
    a.groups = (int32_t)cdiv(p.k, p.group);
    a.lost = p.lost;
    a.second = p.n;
    a.epi = p.epi;
    const FastDiv div(p.group / 32);
    a.div_mul = div.mul;
    a.div_shift = div.shift;
    if (p.type == ECASQ_F32) return launch_matvec_f32(a, p.gated ? kGated : kProject, p.group, st);
    return p.gated ? launch_matvec_gated(a, p.type, p.scale_type == ECASQ_F32, p.group, st) : launch_matvec_project(a, p.type, p.scale_type == ECASQ_F32, p.group, st);
}

// Both calls: n outputs a row of x, of a matrix with n rows or, gated, 2n.
static int project(const void *x, int64_t x_row, int32_t type, int64_t b, const uint8_t *codes, int64_t code_row, const void *levels, int32_t m,
                   const void *scales, int64_t scale_row, int32_t scale_type, int64_t n, int64_t k, int32_t group, const Epilogue &epi, void *y,
                   int64_t y_row, void *ws, size_t ws_bytes, int32_t *status, bool gated, cudaStream_t st) {
    const bool lost_wait = (type & ECASQ_TEST_LOST_WAIT) != 0;
    type &= ~ECASQ_TEST_LOST_WAIT;
    if (n < 1 || k < 1 || b < 0 || n >= (int64_t)1 << (gated ? 30 : 31) || k >= (int64_t)1 << 31 || b > 8 * 65535 || m < 1 || m > 16 || !type_ok(type) ||
        (scale_type != type && scale_type != ECASQ_F32) || group < 32 || group % 32 || epi.act < ECASQ_ACT_NONE || epi.act > ECASQ_ACT_GELU_TANH)
        return ECASQ_EINVAL;
    if (b == 0) return ECASQ_OK;
    if (!x || !codes || !levels || !scales || !y || y == x || !aligned16(codes) || code_row % 16 || code_row < 64 * cdiv(k, 128) || scale_row < cdiv(k, group) ||
        (b > 1 && (x_row < k || y_row < n || (epi.residual && epi.residual_row < n))))
        return ECASQ_EINVAL;
    const ProjectArgs a{x, levels, scales, codes, y, status, x_row, code_row, scale_row, y_row, n, k, b, m, group, type, scale_type, gated, lost_wait, epi};
    return b > kFewRows ? launch_project_tc(a, ws, ws_bytes, st) : launch_project_few(a, st);
}

}  // namespace ecasq

using namespace ecasq;

extern "C" {

size_t ecasq_workspace_size_project(int64_t b, int64_t n, int64_t k, int32_t type) {
    if (b <= kFewRows || b > 8 * 65535 || n < 1 || k < 1 || k >= (int64_t)1 << 31 || !type_ok(type)) return 0;
    return project_tc_room(b, k, type);
}

int ecasq_project_plan(int64_t b, int64_t n, int64_t k, int32_t type, int32_t group, int32_t gated, int64_t *plan) {
    if (b < 0 || b > 8 * 65535 || n < 1 || n >= (int64_t)1 << (gated ? 30 : 31) || k < 1 || k >= (int64_t)1 << 31 || !type_ok(type) || group < 32 || group % 32 || !plan) return ECASQ_EINVAL;
    const ProjectPlan p = b > kFewRows ? plan_project_tc(b, n, k, type, group, gated != 0) : ProjectPlan{};
    plan[0] = p.width;
    plan[1] = p.split;
    plan[2] = p.held;
    plan[3] = p.x_tiles;
    plan[4] = p.w_tiles;
    plan[5] = p.panel;
    return ECASQ_OK;
}

int ecasq_project_rings(int32_t width, int32_t type, int32_t gated, int32_t *rings) {
    if ((width != 32 && width != 64 && width != 128 && width != 256) || !type_ok(type) || !rings) return ECASQ_EINVAL;
    project_tc_rings(width, type == ECASQ_F32, gated != 0, rings);
    return ECASQ_OK;
}

int ecasq_project(const void *x, int64_t x_row, int32_t type, int64_t b, const uint8_t *codes, int64_t code_row, const void *levels,
                  int32_t m, const void *scales, int64_t scale_row, int32_t scale_type, int64_t n, int64_t k, int32_t group,
                  const void *bias, int32_t activation, const void *residual, int64_t residual_row, void *y, int64_t y_row, void *ws,
                  size_t ws_bytes, int32_t *status, ecasq_stream_t stream) {
    return project(x, x_row, type, b, codes, code_row, levels, m, scales, scale_row, scale_type, n, k, group, Epilogue{bias, residual, residual_row, activation}, y,
                   y_row, ws, ws_bytes, status, false, reinterpret_cast<cudaStream_t>(stream));
}

int ecasq_gated(const void *x, int64_t x_row, int32_t type, int64_t b, const uint8_t *codes, int64_t code_row, const void *levels,
                int32_t m, const void *scales, int64_t scale_row, int32_t scale_type, int64_t n, int64_t k, int32_t group,
                int32_t activation, void *y, int64_t y_row, void *ws, size_t ws_bytes, int32_t *status, ecasq_stream_t stream) {
    return project(x, x_row, type, b, codes, code_row, levels, m, scales, scale_row, scale_type, n, k, group, Epilogue{nullptr, nullptr, 0, activation}, y, y_row, ws,
                   ws_bytes, status, true, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
