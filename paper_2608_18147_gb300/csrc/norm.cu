// norm.cu -- root-mean-square norm with the residual's addition, rounded to the input's type or coded to 8 bits (ecasq_norm).
//
// A row is read once: its sums s stay in registers while their squares are added up, and what is written follows from them.  NT threads take a
// row, P pieces of 16 bytes each.  A row may begin anywhere: its pieces are those of memory, the first and the last with columns that are
// not the row's, as long as all of its tensors begin at the same place of a piece (rows of any length one behind another do); the
// weights are shifted to them.  Rows that lie differently or are too long for 1024 threads are read twice, value by value.
#include <cuda_fp8.h>

#include <algorithm>

#include "codes.cuh"

namespace ecasq {

struct NormArgs {
    const void *x, *residual, *weight;
    void *y, *sum;
    float *scales;
    int64_t x_row, residual_row, y_row, sum_row, scale_row, b, k, group, groups;
    float eps;
    int32_t lanes;  // threads that share a group's columns where pieces and groups begin together, a power of two up to 32; 0: the row is one group; -1: neither
};

constexpr int kNormThreads = 256;

// The larger of two values that are not negative; NaN is above all.
__device__ __forceinline__ float above(float v, float w) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(w));
    return v;
}
template <bool MAX> __device__ __forceinline__ float both(float v, float w) { return MAX ? above(v, w) : v + w; }

// The sum (MAX: the maximum) over a row's NT threads, for each of them.  part: NT / 32 words that nobody reads any more.
template <bool MAX, int NT> __device__ __forceinline__ float over_row(float v, float *part) {
    const unsigned lanes = NT < 32 ? ((1u << NT % 32) - 1) << (threadIdx.x & 31 & ~(NT - 1)) : 0xffffffffu;  // (the warp's other rows may have ended)
#pragma unroll
    for (int o = NT < 32 ? NT / 2 : 16; o; o >>= 1) v = both<MAX>(v, __shfl_xor_sync(lanes, v, o));
    if (NT <= 32) return v;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < NT / 32; i++) v = both<MAX>(v, part[i]);
    return v;
}

// A group's scale from its largest value: the quotient by 448, e4m3's largest, rounded once: a product with the reciprocal, and its remainder's (Markstein 1990).
__device__ __forceinline__ float scale_of(float most) {
    const float q = __fmul_rn(most, 1.f / 448.f), scale = __fmaf_rn(__fmaf_rn(-448.f, q, most), 1.f / 448.f, q);
    return scale == 0.f ? 1.f : scale;
}
// What a value is multiplied by to be divided by its scale: two roundings from the quotient.  Scales so small that their reciprocals
// overflow are left to the division.
__device__ __forceinline__ float inverse_of(float scale) { return __fdividef(1.f, scale); }
__device__ __forceinline__ bool invertible(float scale) { return scale >= 0x1p-125f; }
__device__ __forceinline__ uint32_t two_codes(float v, float w) { return __nv_cvt_float2_to_fp8x2(make_float2(v, w), __NV_SATFINITE, __NV_E4M3); }

// A piece: 16 bytes, as they lie in memory and in fp32.
template <typename T> struct Piece;
template <> struct Piece<float> {
    static constexpr int kValues = 4;
    __device__ static __forceinline__ void widen(const uint4 &p, float (&v)[4]) {
        v[0] = __uint_as_float(p.x), v[1] = __uint_as_float(p.y), v[2] = __uint_as_float(p.z), v[3] = __uint_as_float(p.w);
    }
    __device__ static __forceinline__ uint4 narrow(const float (&v)[4]) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <> struct Piece<__half> {
    static constexpr int kValues = 8;
    __device__ static __forceinline__ void widen(const uint4 &p, float (&v)[8]) {
        const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 f = __half22float2(reinterpret_cast<const __half2 &>(w[i]));
            v[2 * i] = f.x, v[2 * i + 1] = f.y;
        }
    }
    __device__ static __forceinline__ uint4 narrow(const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Piece<__nv_bfloat16> {
    static constexpr int kValues = 8;
    __device__ static __forceinline__ void widen(const uint4 &p, float (&v)[8]) {
        const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
        for (int i = 0; i < 4; i++) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    __device__ static __forceinline__ uint4 narrow(const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// The weights of N columns from byte `from` of their copy in shared memory on: the 16-byte pieces that hold them, shifted.
template <typename W, int N, bool ALIGNED> __device__ __forceinline__ void weights_of(const char *copy, int from, float (&v)[N]) {
    constexpr int kWords = N * sizeof(W) / 4;
    const int skip = ALIGNED ? 0 : from & 15;
    const uint4 *p = reinterpret_cast<const uint4 *>(copy + (from - skip));
    uint32_t w[kWords + 4];
#pragma unroll
    for (int i = 0; i < kWords / 4 + (ALIGNED ? 0 : 1); i++) {
        const uint4 q = p[i];
        w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
    }
    if (!ALIGNED) {
#pragma unroll
        for (int j = 0; j < kWords + 2; j++) w[j] = skip & 8 ? w[j + 2] : w[j];
#pragma unroll
        for (int j = 0; j < kWords + 1; j++) w[j] = skip & 4 ? w[j + 1] : w[j];
        if (sizeof(W) == 2) {
#pragma unroll
            for (int j = 0; j < kWords; j++) w[j] = skip & 2 ? __funnelshift_r(w[j], w[j + 1], 16) : w[j];
        }
    }
#pragma unroll
    for (int i = 0; i < kWords / 4; i++) {
        float f[Piece<W>::kValues];
        Piece<W>::widen(make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]), f);
#pragma unroll
        for (int j = 0; j < Piece<W>::kValues; j++) v[i * Piece<W>::kValues + j] = f[j];
    }
}

// ALIGNED: every row begins and ends with a piece.  Else the first and the last piece hold columns that are not the row's: they are made zero, which
// changes neither the mean nor a maximum, and what is stored of such a piece goes value by value.
// Groups whose columns threads that lie together share: one maximum by shuffles; the whole row: one more reduction; others: words of shared memory,
// of the bits of values that are not negative, raised by atomics (whose order does not matter).
// What bounds it: memory where rows are aligned (8192 x 8192 of bf16 with a residual 91 us, 5.9 TB/s; to 8 bits by groups of 128 95 us, 4.9 TB/s, where the
// normed values are found, their maxima exchanged and the codes made between a row's loads and its stores, with issue slots half used: latency); the shifting of weights where they are not (3001 x 5003 of fp32 27 us, 4.5 TB/s); one
// row of 4096 takes 2.3 us, two memory latencies and a launch.  With weights in registers instead of shared memory, and pieces that every
// thread looked at value by value, the aligned cases took 141 and 185 us: two blocks an SM instead of three, and code that did not fit its cache.
// Chosen at run time, the forms (none, one scale a row, groups by shuffles, groups by atomics) share their registers: 38 of this file's 135 kernels spill, that of the 8192 x 8192 of bf16 to
// 8 bits 24 bytes, fp16 ones read up to 664 back.
template <typename T, typename W, int P, int NT, bool ALIGNED>
__global__ void __launch_bounds__(NT < 256 ? 256 : NT, NT <= 256 ? 3 : NT == 512 && P <= 3 ? 2 : 1) k_norm(const __grid_constant__ NormArgs a) {
    constexpr int kThreads = NT < 256 ? 256 : NT, kAtOnce = kThreads / NT, N = Piece<T>::kValues;  // rows of a block; values of a piece
    static_assert(kAtOnce == 1 || NT <= 32, "rows that share a block have a warp each at most");
    __shared__ float part[2][NT <= 32 ? 1 : NT / 32];
    extern __shared__ __align__(16) char smem[];  // the weights, with room for a piece on either side; then the groups' words
    wait_before();
    const int at = threadIdx.x % NT, k = (int)a.k, weight_room = (int)((k + 4 * N) * sizeof(W) + 15) / 16 * 16;
    char *copy = smem + N * (int)sizeof(W);
    const unsigned lanes = NT < 32 ? ((1u << NT % 32) - 1) << (threadIdx.x & 31 & ~(NT - 1)) : 0xffffffffu;
    const int64_t stride = (int64_t)gridDim.x * kAtOnce;
    int64_t row = (int64_t)blockIdx.x * kAtOnce + threadIdx.x / NT;
    // Columns count from where the first piece begins: `skip` of them are in front of the row.
    int skip, pieces;
    uint4 s[P], r[P];
    auto fetch = [&] {
        const T *x = static_cast<const T *>(a.x) + row * a.x_row;
        skip = ALIGNED ? 0 : (int)(reinterpret_cast<uintptr_t>(x) & 15) / (int)sizeof(T);
        pieces = (skip + k + N - 1) / N;
        const uint4 *from = reinterpret_cast<const uint4 *>(x - skip) + at;
        const uint4 *add = reinterpret_cast<const uint4 *>(static_cast<const T *>(a.residual) + (a.residual ? row * a.residual_row - skip : 0)) + at;
#pragma unroll
        for (int i = 0; i < P; i++) s[i] = i * NT + at < pieces ? from[i * NT] : make_uint4(0, 0, 0, 0);
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < P; i++) r[i] = i * NT + at < pieces ? add[i * NT] : make_uint4(0, 0, 0, 0);
        }
    };
    if (row < a.b) fetch();
    for (int c = (int)threadIdx.x - N; c < k + 3 * N; c += kThreads)
        reinterpret_cast<W *>(copy)[c] = c >= 0 && c < k ? static_cast<const W *>(a.weight)[c] : from_f32<W>(0.f);
    if (NT <= 32) __syncthreads();  // (else the mean's barrier is between these and their use)
    for (; row < a.b; row += stride) {
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < P; i++) {
                float v[N], u[N];
                Piece<T>::widen(s[i], v);
                Piece<T>::widen(r[i], u);
#pragma unroll
                for (int j = 0; j < N; j++) v[j] += u[j];
                s[i] = Piece<T>::narrow(v);
            }
        }
        // Whether a piece is all of the row's; its entry j.
        auto whole = [&](int i) { return ALIGNED || ((i * NT + at) * N >= skip && (i * NT + at + 1) * N - skip <= k); };
        auto inside = [&](int i, int j) { return (unsigned)((i * NT + at) * N + j - skip) < (unsigned)k; };
        if (!ALIGNED) {
#pragma unroll
            for (int i = 0; i < P; i++) {
                if (whole(i)) continue;
                float v[N];
                Piece<T>::widen(s[i], v);
#pragma unroll
                for (int j = 0; j < N; j++) v[j] = inside(i, j) ? v[j] : 0.f;
                s[i] = Piece<T>::narrow(v);
            }
        }
        float squares = 0.f;
#pragma unroll
        for (int i = 0; i < P; i++) {
            float v[N];
            Piece<T>::widen(s[i], v);
#pragma unroll
            for (int j = 0; j < N; j++) squares = fmaf(v[j], v[j], squares);
        }
        const float root = 1.f / sqrtf(over_row<false, NT>(squares, part[0]) / (float)k + a.eps);
        // Piece i of a row of T.
        auto store = [&](void *to, int64_t to_row, int i, const uint4 &p) {
            T *begin = static_cast<T *>(to) + row * to_row - skip;
            if (whole(i)) {
                reinterpret_cast<uint4 *>(begin)[i * NT + at] = p;
            } else {
                const T *v = reinterpret_cast<const T *>(&p);
#pragma unroll
                for (int j = 0; j < N; j++)
                    if (inside(i, j)) begin[(i * NT + at) * N + j] = v[j];
            }
        };
        if (a.sum) {
#pragma unroll
            for (int i = 0; i < P; i++)
                if (i * NT + at < pieces) store(a.sum, a.sum_row, i, s[i]);
        }
        auto normed = [&](int i, float (&v)[N]) {
            float w[N];
            Piece<T>::widen(s[i], v);
            weights_of<W, N, ALIGNED>(copy, (min(i * NT + at, pieces - 1) * N - skip) * (int)sizeof(W), w);
#pragma unroll
            for (int j = 0; j < N; j++) v[j] = v[j] * root * w[j];
        };
        auto largest = [&](const float (&v)[N], int j0, int j1) {  // of the entries [j0, j1)
            float most = 0.f;
#pragma unroll
            for (int j = 0; j < N; j++)
                if (j >= j0 && j < j1) most = above(most, fabsf(v[j]));
            return most;
        };
        // Piece i as codes: its entries below `border` by the scale lo, the others by hi.
        auto code = [&](int i, float (&v)[N], float lo, float hi, int border) {
            if (i * NT + at >= pieces) return;
            const float by_lo = inverse_of(lo), by_hi = inverse_of(hi);
            if (invertible(lo) && invertible(hi)) {
#pragma unroll
                for (int j = 0; j < N; j++) v[j] *= j < border ? by_lo : by_hi;
            } else {
#pragma unroll 1
                for (int j = 0; j < N; j++) {  // (a loop that keeps v in registers: each turn divides the first and moves the others down)
                    const float q = v[0] / (j < border ? lo : hi);
#pragma unroll
                    for (int l = 0; l + 1 < N; l++) v[l] = v[l + 1];
                    v[N - 1] = q;
                }
            }
            uint32_t q[N / 4];
#pragma unroll
            for (int j = 0; j < N; j += 4) q[j / 4] = two_codes(v[j], v[j + 1]) | two_codes(v[j + 2], v[j + 3]) << 16;
            uint8_t *to = static_cast<uint8_t *>(a.y) + row * a.y_row + (i * NT + at) * N - skip;
            if (whole(i)) {
                if (N == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(q[0], q[N / 4 - 1]);
                else *reinterpret_cast<uint32_t *>(to) = q[0];
            } else {
#pragma unroll
                for (int j = 0; j < N; j++)
                    if (inside(i, j)) to[j] = (uint8_t)(q[j / 4] >> 8 * (j & 3));
            }
        };
        float *scales = a.scales + row * a.scale_row;
        if (!a.group) {
#pragma unroll
            for (int i = 0; i < P; i++) {
                if (i * NT + at >= pieces) continue;
                float v[N];
                normed(i, v);
                store(a.y, a.y_row, i, Piece<T>::narrow(v));
            }
        } else if (a.lanes == 0) {
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < P; i++) {
                float v[N];
                normed(i, v);
                most = above(most, largest(v, 0, N));
            }
            const float scale = scale_of(over_row<true, NT>(most, part[1]));
            if (at == 0) scales[0] = scale;
#pragma unroll
            for (int i = 0; i < P; i++) {
                float v[N];
                normed(i, v);
                code(i, v, scale, scale, N);
            }
        } else if (a.lanes > 0 && skip == 0) {
#pragma unroll
            for (int i = 0; i < P; i++) {
                float v[N];
                normed(i, v);
                float most = largest(v, 0, N);
#pragma unroll
                for (int o = 16; o; o >>= 1)
                    if (o < NT && o < a.lanes) most = above(most, __shfl_xor_sync(lanes, most, o));
                const float scale = scale_of(most);
                if ((at & (a.lanes - 1)) == 0 && i * NT + at < pieces) scales[(i * NT + at) / a.lanes] = scale;
                code(i, v, scale, scale, N);
            }
        } else {
            const int group = (int)a.group, groups = (int)a.groups;
            uint32_t *most = reinterpret_cast<uint32_t *>(smem + weight_room) + (threadIdx.x / NT) * groups;  // (a warp's own where rows share a block)
            auto all = [&] {
                if (NT > 32) __syncthreads();
                else __syncwarp(lanes);
            };
            for (int g = at; g < groups; g += NT) most[g] = 0;
            all();
            // Of a piece the entries below `border` lie in group g, the others in the next.
            auto group_of_piece = [&](int i, int &border) {
                const int c = (i * NT + at) * N - skip, g = max(c, 0) / group;
                border = (g + 1) * group - c;
                return g;
            };
#pragma unroll
            for (int i = 0; i < P; i++) {
                if (i * NT + at >= pieces) continue;
                float v[N];
                normed(i, v);
                int border;
                const int g = group_of_piece(i, border);
                atomicMax(most + g, __float_as_uint(largest(v, 0, border)));
                if (border < N && g + 1 < groups) atomicMax(most + g + 1, __float_as_uint(largest(v, border, N)));
            }
            all();
            for (int g = at; g < groups; g += NT) scales[g] = scale_of(__uint_as_float(most[g]));
#pragma unroll
            for (int i = 0; i < P; i++) {
                if (i * NT + at >= pieces) continue;
                float v[N];
                normed(i, v);
                int border;
                const int g = group_of_piece(i, border);
                const float lo = scale_of(__uint_as_float(most[g])), hi = border < N && g + 1 < groups ? scale_of(__uint_as_float(most[g + 1])) : lo;
                code(i, v, lo, hi, border);
            }
            all();
        }
        if (a.b - row > stride) {  // the next row is on its way before the barrier
            row += stride;
            fetch();
            row -= stride;
        }
        if (NT > 32) __syncthreads();  // the reductions' words have been read
    }
}

// Rows that do not fit, or whose tensors lie differently: a block a row, which it reads for the mean, and again for what it writes, a warp a group.
template <typename T, typename W> __global__ void __launch_bounds__(kNormThreads) k_norm_long(const __grid_constant__ NormArgs a) {
    __shared__ float part[kNormThreads / 32];
    wait_before();
    const int lane = threadIdx.x & 31;
    for (int64_t row = blockIdx.x; row < a.b; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_row, *residual = static_cast<const T *>(a.residual) + (a.residual ? row * a.residual_row : 0);
        T *sum = static_cast<T *>(a.sum) + (a.sum ? row * a.sum_row : 0);
        const W *weight = static_cast<const W *>(a.weight);
        auto total = [&](int64_t c) { return a.residual ? from_f32<T>(to_f32(x[c]) + to_f32(residual[c])) : x[c]; };
        float squares = 0.f;
#pragma unroll 4
        for (int64_t c = threadIdx.x; c < a.k; c += kNormThreads) {
            const T s = total(c);
            squares = fmaf(to_f32(s), to_f32(s), squares);
            if (a.sum) sum[c] = s;
        }
        const float root = 1.f / sqrtf(over_row<false, kNormThreads>(squares, part) / (float)a.k + a.eps);  // (behind its barrier all of `sum` is there)
        auto normed = [&](int64_t c) { return to_f32(a.sum ? sum[c] : total(c)) * root * to_f32(weight[c]); };
        if (!a.group) {
            // (A thread reads what it overwrites, or nobody does.)
            T *y = static_cast<T *>(a.y) + row * a.y_row;
#pragma unroll 4
            for (int64_t c = threadIdx.x; c < a.k; c += kNormThreads) y[c] = from_f32<T>(normed(c));
        } else {
            uint8_t *y = static_cast<uint8_t *>(a.y) + row * a.y_row;
            auto group = [&](int64_t start, int64_t end, int first, int step, auto most_of_all) {
                float most = 0.f;
                for (int64_t c = start + first; c < end; c += step) most = above(most, fabsf(normed(c)));
                const float scale = scale_of(most_of_all(most));
                for (int64_t c = start + first; c < end; c += step) {
                    const float v = normed(c);
                    y[c] = (uint8_t)two_codes(invertible(scale) ? v * inverse_of(scale) : v / scale, 0.f);
                }
                return scale;
            };
            if (a.groups == 1) {
                __syncthreads();  // (the words of the reduction before have been read)
                const float scale = group(0, a.k, threadIdx.x, kNormThreads, [&](float v) { return over_row<true, kNormThreads>(v, part); });
                if (threadIdx.x == 0) a.scales[row * a.scale_row] = scale;
            } else {
                for (int64_t g = threadIdx.x / 32; g < a.groups; g += kNormThreads / 32) {
                    const float scale = group(g * a.group, min(a.k, (g + 1) * a.group), lane, 32, [&](float v) { return over_row<true, 32>(v, nullptr); });
                    if (lane == 0) a.scales[row * a.scale_row + g] = scale;
                }
            }
        }
        __syncthreads();
    }
}

template <typename T, typename W, int P, int NT, bool ALIGNED> static int launch_norm_as(NormArgs &a, cudaStream_t st) {
    constexpr int kAtOnce = NT < 256 ? 256 / NT : 1, kThreads = NT < 256 ? 256 : NT, N = Piece<T>::kValues;
    const int64_t lanes = a.group / N;
    if (a.group >= a.k) a.lanes = 0;
    else a.lanes = lanes <= std::min(32, NT) && (lanes & (lanes - 1)) == 0 ? (int32_t)lanes : -1;
    const int words = a.group && (a.lanes < 0 || (!ALIGNED && a.lanes)) ? (int)(4 * a.groups * kAtOnce) : 0;
    const int smem = (int)((a.k + 4 * N) * sizeof(W) + 15) / 16 * 16 + words;
    auto *kernel = k_norm<T, W, P, NT, ALIGNED>;
    if (smem > 47 * 1024) {  // (with the reductions' words, 256 bytes at most, over the 48 KB that a launch has unasked)
        static std::atomic<int> allowed[kDevices];
        const int rc = allow_smem(kernel, 220 * 1024, allowed);
        if (rc) return rc;
    }
    const unsigned blocks = (unsigned)std::min<int64_t>(cdiv(a.b, kAtOnce), 152 * (2048 / kThreads));
    return launch_early(kernel, dim3(blocks), kThreads, smem, st, a);
}
// The threads a row and pieces a thread: as many threads as have a piece where rows are few and each waits for its own loads; else 256, whose
// pieces are on their way together, and whose barriers other blocks of an SM hide from one another.
template <typename T, typename W, bool ALIGNED> static int launch_norm_pieces(NormArgs &a, int64_t pieces, cudaStream_t st) {
    if (a.b <= 304) {
        if (pieces <= 256) return launch_norm_as<T, W, 1, 256, ALIGNED>(a, st);
        if (pieces <= 512) return launch_norm_as<T, W, 1, 512, ALIGNED>(a, st);
        if (pieces <= 1024) return launch_norm_as<T, W, 1, 1024, ALIGNED>(a, st);
        if (pieces <= 2048) return launch_norm_as<T, W, 2, 1024, ALIGNED>(a, st);
        return launch_norm_as<T, W, 4, 1024, ALIGNED>(a, st);
    }
    if (pieces <= 16) return launch_norm_as<T, W, 1, 16, ALIGNED>(a, st);
    if (pieces <= 32) return launch_norm_as<T, W, 1, 32, ALIGNED>(a, st);
    if (pieces <= 64) return launch_norm_as<T, W, 2, 32, ALIGNED>(a, st);
    if (pieces <= 128) return launch_norm_as<T, W, 4, 32, ALIGNED>(a, st);
    if (pieces <= 256) return launch_norm_as<T, W, 1, 256, ALIGNED>(a, st);
    if (pieces <= 512) return launch_norm_as<T, W, 2, 256, ALIGNED>(a, st);
    if (pieces <= 1024) return launch_norm_as<T, W, 4, 256, ALIGNED>(a, st);
    if (pieces <= 1536) return launch_norm_as<T, W, 3, 512, ALIGNED>(a, st);
    if (pieces <= 2048) return launch_norm_as<T, W, 4, 512, ALIGNED>(a, st);
    return launch_norm_as<T, W, 4, 1024, ALIGNED>(a, st);
}
template <typename T, typename W> static int launch_norm(NormArgs &a, bool alike, cudaStream_t st) {
    constexpr int N = Piece<T>::kValues;
    const bool aligned = alike && a.k % N == 0 && reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && (a.b == 1 || a.x_row % N == 0);
    const int64_t pieces = aligned ? a.k / N : cdiv(a.k + N - 1, N);  // wherever a row begins
    if (!alike || pieces > 4096) return launch_early(k_norm_long<T, W>, dim3((unsigned)std::min<int64_t>(a.b, 152 * 8)), kNormThreads, 0, st, a);
    return aligned ? launch_norm_pieces<T, W, true>(a, pieces, st) : launch_norm_pieces<T, W, false>(a, pieces, st);
}

}  // namespace ecasq

using namespace ecasq;

extern "C" int ecasq_norm(const void *x, int64_t x_row, int32_t type, int64_t b, int64_t k, const void *residual, int64_t residual_row,
                          const void *weight, int32_t weight_type, float eps, int64_t group, void *y, int64_t y_row, void *sum,
                          int64_t sum_row, float *scales, int64_t scale_row, ecasq_stream_t stream) {
    if (b < 0 || k < 1 || b >= (int64_t)1 << 31 || !type_ok(type) || (weight_type != type && weight_type != ECASQ_F32) || !(eps >= 0.f) || group < 0 ||
        k >= (int64_t)1 << 31 || (group < k && group % 16))
        return ECASQ_EINVAL;
    if (b == 0) return ECASQ_OK;
    const int64_t groups = !group ? 0 : group >= k ? 1 : cdiv(k, group);  // (any group from k on is one: cdiv would go beyond 64 bits for the largest)
    if (!x || !weight || !y || (sum && (!residual || (!group && sum == y))) || (group && (!scales || (b > 1 && scale_row < groups))) ||
        (b > 1 && (x_row < k || y_row < k || (residual && residual_row < k) || (sum && sum_row < k))))
        return ECASQ_EINVAL;
    NormArgs a{x, residual, weight, y, sum, scales, x_row, residual_row, y_row, sum_row, scale_row, b, k, group, groups, eps, 0};
    // Whether all of a row's tensors begin at the same place of a piece of 16 bytes (codes: of as many bytes as it has values).
    const int64_t size = type_size(type), values = 16 / size, place = reinterpret_cast<uintptr_t>(x) % 16 / size;
    const auto alike = [&](const void *p, int64_t row, int64_t of) {
        return reinterpret_cast<uintptr_t>(p) % (values * of) == (uintptr_t)(place * of) && (b == 1 || (row - x_row) % values == 0);
    };
    const bool all_alike = alike(x, x_row, size) && (!residual || alike(residual, residual_row, size)) && (!sum || alike(sum, sum_row, size)) && alike(y, y_row, group ? 1 : size);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool weight32 = weight_type == ECASQ_F32;
    if (type == ECASQ_F32) return launch_norm<float, float>(a, all_alike, st);
    if (type == ECASQ_F16) return weight32 ? launch_norm<__half, float>(a, all_alike, st) : launch_norm<__half, __half>(a, all_alike, st);
    return weight32 ? launch_norm<__nv_bfloat16, float>(a, all_alike, st) : launch_norm<__nv_bfloat16, __nv_bfloat16>(a, all_alike, st);
}
