// attend.cuh -- attention of one new token a sequence over a paged cache (ecasq_attend).
//
// For query head h and the keys t of its sequence: s_t = scale q . K_t, out = sum softmax(s)_t V_t.
// One pass over the cache with a running maximum m and sum l: a tile of 16 keys with scores s
// moves m to m' = max(m, max s), O and l shrink by 2^(m - m') and gain sum 2^(s - m') V and
// sum 2^(s - m') (s scaled to base 2).  A key row is read once for up to eight query heads.
//
// What bounds it: the cache's bytes.  So each warp works alone on tiles of 16 or 32 keys through a ring of its own in
// shared memory that cp.async fills a few tiles ahead, without a barrier in the loop.  The sequence is cut into
// splits (one block each, so that few sequences still fill the card); a block's warps join in shared memory,
// and the splits in that of a cluster of blocks or, by k_attend_join, in memory.  Measured, both kernels: 32 sequences of up to 8192 bf16 keys of 128, eight heads a key
// head, 94 us or 5.7 TB/s, 84 % of a copy's rate.  Over coded rows the integer pipe, whose byte permutes look the levels up, is the
// fullest unit, but 56 to 60 % busy: twelve warps an SM are too few to fill it (shared memory holds three blocks of four; with sixteen
// levels and rows of 256 registers hold no more either).  16 sequences of 32768 keys of 128 with eight levels 150 us (4.5 TB/s, 66 %), one of
// 70001 keys of 256 with sixteen 53 us (1.7 TB/s).  Short sequences are bound by latency: lengths, page numbers, rows and
// the join follow one another; one sequence of 1000 keys takes 6.1 us.
//
// 16-bit rows: S^T = K Q^T and O^T = V^T P^T on mma.m16n8k16 with the query heads as n, fp32 sums.  (One
// token a sequence is a matrix-vector product for each key head; with eight columns there is nothing for the
// larger tensor tiles to reuse.)  Both products may take their reduction index in any order, so that a lane reads
// 16 consecutive bytes of a row where the fragments want scattered pairs:
//   lane (g, t) = (lane / 4, lane mod 4) holds rows g and g + 8 of K, 16-byte chunks t, t + 4, ...,
//   and of V the chunks g, g + 8, ... of the keys 2t, 2t + 1, 2t + 8, 2t + 9.
// The reduction of the second product runs over keys, but a register of V holds two neighbouring entries of one key.
// With up to four heads (HT = 4) a pair of reduction indices is such a pair of entries instead, and a head has two
// columns, which hold its weights on the even and on the odd index: sum_t V_t[e] P_t and sum_t V_t[e + 1] P_t come
// out side by side, in as many products as before.  With up to eight (HT = 8) the columns are taken, and two keys'
// registers are first permuted into pairs of keys.  (Four heads a key head, 16 sequences of 8192 keys: with HT = 4 and 8 50.1
// and 55.6 us for eight-level rows, 52.3 and 53.6 for sixteen levels and rows of 64, 94.0 and 95.1 for 32 of 4096 bf16 keys.)
// Weights enter the second product as a high and a low 16-bit part: one part alone would add an error as large as the rounding of
// the result.  In bf16 the two keep 16 bits of a weight of any size.  Binary16 has no step below 2^-24, so there the parts are those of
// 2^15 times the weight, which is at most 1: 16 bits of weights down to 2^-24 of the largest, and steps of 2^-40 of it below
// (parts of the weight itself lose bits from 2^-9 on, and all of a weight below 2^-25, which is wrong where the heaviest key holds
// small values).
// Coded rows: a lane holds its row's codebook as planes of low and of high bytes; a byte permute with four
// codes as its selector looks one byte of four entries up in eight levels at once, and two more pair the bytes of the four, so that
// a pair of entries costs two permutes and no shared-memory access.  With sixteen levels the lookups of four entries are nine operations:
// both halves of the levels, and a choice by the codes' fourth bits.
// fp32 rows: fp32 products on the FMA pipe in the same frame.
#pragma once

#include <algorithm>
#include <type_traits>

#include "codes.cuh"

namespace ecasq {

constexpr int kTile = 16;        // keys of a matrix product; tiles are one or two of them
constexpr int kHeads = 8;        // query heads of a block at most
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttendArgs {
    const void *q;
    void *out;
    const int32_t *table, *lengths, *starts;
    float *lse, *part;           // part: splits' results, see PartAt
    void *ws;
    size_t ws_bytes;
    int32_t *status;
    const char *k, *v, *kt, *vt; // rows and codebooks
    uint64_t k_page, k_slot, k_head, v_page, v_slot, v_head;         // strides in bytes (modulo 2^64)
    uint64_t kt_page, kt_slot, kt_head, vt_page, vt_slot, vt_head;
    int64_t q_row, q_head, out_row, out_head, table_row, pages;
    float scale2;                // scale log2(e)
    int32_t heads, group, htiles, d, page_size, max_len, splits, tile, step, least;  // group: query heads a key head; least: keys of a split
    bool cluster;                // the splits are a cluster, which joins them
    uint32_t div_mul, div_shift; // t div page_size = umulhi(t, div_mul) >> div_shift, or t >> div_shift if div_mul is 0
};

// A split's result for one query head: d sums, then its maximum (base 2) and its sum of weights.
struct PartAt {
    int64_t stride;
    __host__ __device__ explicit PartAt(int d) : stride(d + 4) {}
    __device__ float *at(float *part, int64_t seq, int heads, int head, int splits, int split) const {
        return part + ((seq * heads + head) * splits + split) * stride;
    }
};

// What the weights of the values' product are multiplied by (see above); a power of two, taken off again from the sums.
template <typename T> constexpr float kLift = std::is_same<T, __half>::value ? 0x1p15f : 1.f;

// Sets a.splits, a.least and, where there are several, a.part from the workspace; `resident`: blocks that an SM holds; splits are multiples of a.step keys.
int split_attend(AttendArgs &a, int64_t b, int resident);

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes to shared memory, or 16 zero bytes (src is not read then).
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool read) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(read ? 16 : 0));
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N)); }
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t s) {
    uint32_t d;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(s));
    return d;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
template <typename T> __device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two values as a pair of T, the first in the low half.
template <typename T> __device__ __forceinline__ uint32_t pack2(float x, float y);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float x, float y) {
    uint32_t v;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(y), "f"(x));
    return v;
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float x, float y) {
    uint32_t v;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(y), "f"(x));
    return v;
}
template <> __device__ __forceinline__ uint32_t pack2<float>(float, float) { return 0; }  // (unused)
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t v) {
    const uint16_t lo = (uint16_t)v, hi = (uint16_t)(v >> 16);
    return make_float2(to_f32(reinterpret_cast<const T &>(lo)), to_f32(reinterpret_cast<const T &>(hi)));
}

// A row's codebook as byte planes: the levels' low bytes, then their high bytes.
template <int LV> struct Book {
    uint32_t lo[LV / 4], hi[LV / 4];
    // Where they lie as levels, puts them as planes.
    __device__ static __forceinline__ void split(char *p) {
        uint4 *q = reinterpret_cast<uint4 *>(p);
        const uint4 a = q[0];
        const uint32_t l0 = prmt(a.x, a.y, 0x6420), l1 = prmt(a.z, a.w, 0x6420), h0 = prmt(a.x, a.y, 0x7531), h1 = prmt(a.z, a.w, 0x7531);
        if (LV == 8) {
            q[0] = make_uint4(l0, l1, h0, h1);
        } else {
            const uint4 b = q[1];
            q[0] = make_uint4(l0, l1, prmt(b.x, b.y, 0x6420), prmt(b.z, b.w, 0x6420));
            q[1] = make_uint4(h0, h1, prmt(b.x, b.y, 0x7531), prmt(b.z, b.w, 0x7531));
        }
    }
    __device__ __forceinline__ void load(const char *p) {
        const uint4 *q = reinterpret_cast<const uint4 *>(p);
        const uint4 a = q[0];
        if (LV == 8) {
            lo[0] = a.x;
            lo[1] = a.y;
            hi[0] = a.z;
            hi[1] = a.w;
        } else {
            const uint4 b = q[LV / 8 - 1];
            lo[0] = a.x;
            lo[1] = a.y;
            lo[2 % (LV / 4)] = a.z;
            lo[3 % (LV / 4)] = a.w;
            hi[0] = b.x;
            hi[1] = b.y;
            hi[2 % (LV / 4)] = b.z;
            hi[3 % (LV / 4)] = b.w;
        }
    }
    // Entries 4H .. 4H+3 of the word w of eight codes: their low and their high bytes.
    template <int H> __device__ __forceinline__ void look(uint32_t w, uint32_t &l, uint32_t &h) const {
        if (LV == 8) {
            const uint32_t s = H ? w >> 16 : w;
            l = prmt(lo[0], lo[1], s);
            h = prmt(hi[0], hi[1], s);
        } else {
            // The lower and the upper eight levels by the codes' low three bits, then a choice by the fourth: a byte
            // permute spreads the sign bits of w << 4 and of w, which are the codes' fourth bits.
            const uint32_t low3 = w & 0x77777777u, s = H ? low3 >> 16 : low3, m = prmt(w << 4, w, H ? 0xFBEA : 0xD9C8);
            const uint32_t l0 = prmt(lo[0], lo[1], s), l1 = prmt(lo[2 % (LV / 4)], lo[3 % (LV / 4)], s);
            const uint32_t h0 = prmt(hi[0], hi[1], s), h1 = prmt(hi[2 % (LV / 4)], hi[3 % (LV / 4)], s);
            l = (l0 & ~m) | (l1 & m);
            h = (h0 & ~m) | (h1 & m);
        }
    }
};

// A tile in shared memory: rows of K, as many of V, then their codebooks.  Sixteen keys, of coded rows 32, whose
// other costs (maxima, codebooks, addresses) are shared by more keys.  Coded rows of more than 128 entries have many
// registers' worth of sums and of q, so q lies in shared memory and tiles have sixteen keys, with which twelve warps fit an SM instead of
// eight (four sequences of 20000 keys of 256 entries, four heads a key head: 33.1 against 34.6 us with eight levels, 50.6
// against 55.8 with sixteen).  T and LV: the rows' type and levels (0: plain); NV: the row length is at most 64 NV.
template <typename T, int LV, int NV> struct Shape {
    static constexpr bool kF32 = sizeof(T) == 4;
    static constexpr int kRow = LV ? 32 * NV : 64 * NV * (int)sizeof(T);   // bytes of a row's room
    static constexpr int kChunks = kRow / 16;
    static constexpr int kBook = 2 * LV;                                   // bytes of a codebook
    static constexpr int kKeys = LV && NV < 4 ? 32 : kTile, kHalves = kKeys / kTile;
    static constexpr uint32_t kAll = kKeys == 32 ? 0xffffffffu : 0xffffu;
    static constexpr int kBytes = 2 * kKeys * (kRow + kBook);
    static constexpr int kWarps = kBytes > 16384 ? 3 : kBytes > 8192 ? 2 : 4;
    static constexpr int kStages = kBytes > 5120 ? 2 : 3;
    static constexpr int kRing = kStages * kBytes;                         // of a warp
    static constexpr int kJoin = kHeads * 64 * NV * 4;                     // a warp's sums at the end, in its ring
    static constexpr int kExtra = (kF32 ? kHeads * 64 * NV * 4 + kWarps * kTile * kHeads * 4 : 0) + (kWarps + 1) * (2 * kHeads * 4) + kWarps * kStages * 4;
    static constexpr bool kQShared = LV && NV == 4;                        // q's operands lie in shared memory
    static constexpr int kSmem = kWarps * kRing + (kExtra + 15) / 16 * 16 + (kQShared ? 512 * 2 * NV : 0);
    static_assert(kJoin <= kRing, "");
    static_assert(kSmem <= 227 * 1024, "");
    static constexpr int kPieces = kTile * kChunks / 32;                   // 16-byte pieces of K (and of V) for a lane and half
    // Where chunk c of key position r lies: swizzled so that the reads described above do not meet in a bank.
    __device__ static __forceinline__ int k_at(int r, int c) {
        if (LV && NV < 4) return r * kRow + 16 * c;
        return r * kRow + 16 * (c ^ ((r & 1) << 2));
    }
    // Row 2t + e + 8f of V is stored as row t + 4 (e + 2f).
    __device__ static __forceinline__ int v_row(int r) { return ((r >> 1) & 3) + 4 * ((r & 1) + 2 * (r >> 3)); }
    __device__ static __forceinline__ int v_at(int stored, int c) {
        if (kF32) return stored * kRow + 16 * c;
        if (LV) {
            if (NV == 1) return stored * kRow + 16 * c;
            if (NV == 2) return stored * kRow + 16 * (c ^ (stored & 2));
        }
        return stored * kRow + 16 * (c ^ ((stored & 3) << 1));
    }
};

__device__ __forceinline__ int page_of(const AttendArgs &a, int t) {
    return a.div_mul ? (int)(__umulhi((uint32_t)t, a.div_mul) >> a.div_shift) : t >> a.div_shift;
}

// The keys [first, end) that a block sees of its sequence.
struct Span {
    int first, end;
    bool too_long;
};
__device__ __forceinline__ Span seq_span(const AttendArgs &a, int64_t seq) {
    Span s;
    s.end = a.lengths[seq];
    s.first = a.starts ? min(max(a.starts[seq], 0), a.max_len) : 0;  // (at max_len no key is left, and sums of key numbers fit)
    s.too_long = s.end > a.max_len;
    if (s.too_long) s.end = a.max_len;
    return s;
}
// A sequence's splits are counted from the tile of its first key (a.tile keys).  They share its keys evenly, in multiples of a.step,
// but none but the last has fewer than a.least.
struct Cut {
    int lead, chunk, count;
};
__device__ __forceinline__ Cut cut_of(const AttendArgs &a, const Span &s) {
    Cut c{s.first & -a.tile, a.least, 0};
    if (s.end <= s.first) return c;
    const int keys = s.end - c.lead, even = (keys + a.splits - 1) / a.splits;
    c.chunk = max(a.least, (even + a.step - 1) / a.step * a.step);
    c.count = (keys + c.chunk - 1) / c.chunk;
    return c;
}

__device__ __forceinline__ float log_sum(float top, float sum) { return sum == 0.f ? -CUDART_INF_F : top * kLn2 + logf(sum); }
// Four entries of a head's result: sums over keys by the sum of the weights (none: 0).
template <typename T>
__device__ __forceinline__ void store_out(const AttendArgs &a, int64_t seq, int head, int e, float4 v, float sum) {
    T *out = static_cast<T *>(a.out) + seq * a.out_row + head * a.out_head + e;
    const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; i++) out[i] = from_f32<T>(sum == 0.f ? 0.f : x[i] / sum);
}

__device__ __forceinline__ float shared_of_rank(const float *p, uint32_t rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(of_rank(smem_addr(p), rank)) : "memory");
    return v;
}

// HT: query heads of a block, 4 or 8.  CLUSTER: the splits are a cluster of blocks, which joins them (apart from the others, whose loop
// over the tiles comes out slower with this in one kernel: 159 against 149 us for 16 sequences of 32768 eight-level keys).
template <typename T, int LV, int NV, int HT, bool CLUSTER>
__global__ void __launch_bounds__(32 * Shape<T, LV, NV>::kWarps, Shape<T, LV, NV>::kQShared ? 3 : 0)
k_attend(const __grid_constant__ AttendArgs a) {
    using S = Shape<T, LV, NV>;
    constexpr int HL = HT / 4;  // heads of a lane's scores: HT = 8: 2t, 2t + 1; HT = 4: t
    extern __shared__ __align__(16) char smem[];
    wait_before();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int64_t seq = blockIdx.z;
    const int split = blockIdx.y, kh = blockIdx.x / a.htiles, h0 = kh * a.group + (blockIdx.x % a.htiles) * HT;
    const int nh = min(HT, a.group - (int)(blockIdx.x % a.htiles) * HT);
    // 16-bit: q as the second operand of S^T, in the order of the lane's chunks of K
    const T *qp = static_cast<const T *>(a.q) + seq * a.q_row + h0 * a.q_head;
    constexpr int kSteps = S::kF32 ? 2 : 4 * NV;
    uint32_t qf[2 * kSteps];
    if (!S::kF32) {
        constexpr int kRun = LV ? (NV == 1 ? 16 : 32) : 8;  // consecutive entries of a lane's chunk
        const int h = g * HT / 8;
        const bool vec = (reinterpret_cast<uintptr_t>(a.q) & 15) == 0 && a.q_row % 8 == 0 && a.q_head % 8 == 0;
#pragma unroll
        for (int i = 0; i < 2 * kSteps; i += 4) {  // eight entries (d is a multiple of eight)
            const int run = 2 * i / kRun, e = kRun * (t + 4 * run) + 2 * i % kRun;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (h < nh && e < a.d) {
                const T *from = qp + h * a.q_head + e;
                if (vec) {
                    v = *reinterpret_cast<const uint4 *>(from);
                } else {
                    v.x = pack2<T>(to_f32(from[0]), to_f32(from[1]));
                    v.y = pack2<T>(to_f32(from[2]), to_f32(from[3]));
                    v.z = pack2<T>(to_f32(from[4]), to_f32(from[5]));
                    v.w = pack2<T>(to_f32(from[6]), to_f32(from[7]));
                }
            }
            qf[i] = v.x;
            qf[i + 1] = v.y;
            qf[i + 2] = v.z;
            qf[i + 3] = v.w;
        }
    }
    uint4 *q_shared = reinterpret_cast<uint4 *>(smem + S::kWarps * S::kRing + (S::kExtra + 15) / 16 * 16) + lane;
    if (S::kQShared && wid == 0) {
#pragma unroll
        for (int i = 0; i < 2 * kSteps; i += 4) q_shared[8 * i] = make_uint4(qf[i], qf[i + 1], qf[i + 2], qf[i + 3]);
    }
    const Span span = seq_span(a, seq);
    if (span.too_long && threadIdx.x == 0 && split == 0 && a.status) atomicOr(a.status, ECASQ_BAD_LENGTH);
    const Cut cut = cut_of(a, span);
    const int active = cut.count;
    if (split >= max(active, 1)) {
        if (CLUSTER && active > 1) {
            cluster_barrier();
            cluster_barrier();
        }
        return;
    }
    const int begin = cut.lead + split * cut.chunk, end = min(span.end, begin + cut.chunk);  // keys of this split (from `first` on)

    char *ring = smem + wid * S::kRing;
    float *qs = reinterpret_cast<float *>(smem + S::kWarps * S::kRing);  // fp32: q, then each warp's weights
    float *ps = qs + kHeads * 64 * NV + wid * kTile * kHeads;
    float *wmax = qs + (S::kF32 ? kHeads * 64 * NV + S::kWarps * kTile * kHeads : 0), *wsum = wmax + S::kWarps * kHeads;
    float *bmax = wsum + S::kWarps * kHeads, *bsum = bmax + kHeads;                      // of the block, for its cluster
    uint32_t *seen = reinterpret_cast<uint32_t *>(bsum + kHeads) + wid * S::kStages;  // keys of a stage that count

    // ---- copies.  The lane's key of a tile is number lane mod kKeys; find() looks its page up, a tile ahead of fetch().
    const char *kb = a.k + kh * a.k_head, *vb = a.v + kh * a.v_head;
    const char *ktb = LV ? a.kt + kh * a.kt_head : nullptr, *vtb = LV ? a.vt + kh * a.vt_head : nullptr;
    const int32_t *table = a.table + seq * a.table_row;
    const bool tiles_whole = a.page_size % S::kKeys == 0;  // a tile's keys are neighbouring slots of one page
    const int row_chunks = LV ? a.d / 32 : a.d * (int)sizeof(T) / 16;
    bool bad_page = false;
    struct Found {
        int page, slot;  // slot -1: beyond the split, no error (a table may hold any number)
        __device__ uint64_t offset(uint64_t by_page, uint64_t by_slot) const { return (uint32_t)page * by_page + (uint32_t)slot * by_slot; }
    };
    auto find = [&](int t0) {
        const int key = t0 + (lane & (S::kKeys - 1));
        Found f{-1, -1};
        if (key >= span.first && key < end) {
            const int p = page_of(a, key);
            f.slot = key - p * a.page_size;
            f.page = table[p];
        }
        return f;
    };
    auto fetch = [&](Found f, int stage) {
        char *dst = ring + stage * S::kBytes;
        const bool ok = f.page >= 0 && f.page < a.pages;
        bad_page |= f.slot >= 0 && !ok;
        const uint32_t mask = __ballot_sync(0xffffffffu, ok) & S::kAll;
        if (lane == 0) seen[stage] = mask;
        // Rows of one page have one address and a step; others each their own, shuffled from the lane that looked it up (32
        // sequences of 4096 bf16 keys: 94 and 96 us; 16 of 8192 eight-level keys: 50 and 53).
        // Sixteen neighbouring slots, the first at kp and vp (chunk c of row r0 of them), to rows 16 half .. of the tile.
        const int r0 = lane / S::kChunks, c0 = lane % (S::kChunks < 32 ? S::kChunks : 32);
        auto copy_half = [&](int half, const char *kp, const char *vp) {
            char *dk = dst + half * kTile * S::kRow, *dv = dk + S::kKeys * S::kRow;
#pragma unroll
            for (int i = 0; i < S::kPieces; i++) {
                // piece lane + 32 i: chunks come round in a row first
                constexpr int kSame = S::kChunks > 32 ? S::kChunks / 32 : 1, kRows = S::kChunks > 32 ? 1 : 32 / S::kChunks;
                const int r = r0 + i / kSame * kRows, c = c0 + i % kSame * 32;
                if (c < row_chunks) {
                    copy16(smem_addr(dk + S::k_at(r, c)), kp + i % kSame * 512, true);
                    copy16(smem_addr(dv + S::v_at(S::v_row(r), c)), vp + i % kSame * 512, true);
                }
                if (i % kSame == kSame - 1) {
                    kp += kRows * a.k_slot;
                    vp += kRows * a.v_slot;
                }
            }
        };
        if (tiles_whole && mask == S::kAll) {
            const Found first{f.page, f.slot - (lane & (S::kKeys - 1)) + r0};
            const uint64_t ko = first.offset(a.k_page, a.k_slot), vo = first.offset(a.v_page, a.v_slot);
#pragma unroll
            for (int half = 0; half < S::kHalves; half++) copy_half(half, kb + ko + 16 * c0 + half * kTile * a.k_slot, vb + vo + 16 * c0 + half * kTile * a.v_slot);
        } else {
#pragma unroll
            for (int half = 0; half < S::kHalves; half++) {
                const int slot0 = __shfl_sync(0xffffffffu, f.slot, kTile * half), slot15 = __shfl_sync(0xffffffffu, f.slot, kTile * half + kTile - 1);
                if (slot15 - slot0 == kTile - 1 && (mask >> 16 * half & 0xffffu) == 0xffffu) {  // sixteen of them are
                    const Found first{__shfl_sync(0xffffffffu, f.page, kTile * half), slot0 + r0};
                    copy_half(half, kb + first.offset(a.k_page, a.k_slot) + 16 * c0, vb + first.offset(a.v_page, a.v_slot) + 16 * c0);
                    continue;
                }
                const uint64_t krow = ok ? f.offset(a.k_page, a.k_slot) : 0, vrow = ok ? f.offset(a.v_page, a.v_slot) : 0;
                char *dk = dst + half * kTile * S::kRow, *dv = dk + S::kKeys * S::kRow;
#pragma unroll
                for (int i = 0; i < S::kPieces; i++) {
                    const int r = (lane + 32 * i) / S::kChunks, c = (lane + 32 * i) % S::kChunks;
                    const uint64_t ko = __shfl_sync(0xffffffffu, krow, kTile * half + r), vo = __shfl_sync(0xffffffffu, vrow, kTile * half + r);
                    if (c < row_chunks) {
                        const bool read = mask >> (kTile * half + r) & 1;
                        copy16(smem_addr(dk + S::k_at(r, c)), read ? kb + ko + 16 * c : kb, read);
                        copy16(smem_addr(dv + S::v_at(S::v_row(r), c)), read ? vb + vo + 16 * c : vb, read);
                    }
                }
            }
        }
        if (LV) {  // a lane its key's codebooks
            const uint64_t ko = ok ? f.offset(a.kt_page, a.kt_slot) : 0, vo = ok ? f.offset(a.vt_page, a.vt_slot) : 0;
            const char *ks = ktb + ko, *vs = vtb + vo;
            char *to = dst + 2 * S::kKeys * S::kRow;
#pragma unroll
            for (int i = 0; i < LV / 8; i++) {
                if (S::kKeys == 32 || lane < 16) copy16(smem_addr(to + lane * S::kBook + 16 * i), ks + 16 * i, ok);
                if (S::kKeys == 32 || lane >= 16)
                    copy16(smem_addr(to + (S::kKeys + (lane & (S::kKeys - 16)) + S::v_row(lane & 15)) * S::kBook + 16 * i), vs + 16 * i, ok);
            }
        }
    };

    // The first tiles are on their way before anything else: all their pages at once, then the rows.
    const int step = S::kKeys * S::kWarps;
    const int mine = begin + S::kKeys * wid;
    // Chunks beyond the row's end are read but never filled.
    if (row_chunks < S::kChunks) {
        for (int i = lane; i < S::kRing / 16; i += 32) reinterpret_cast<uint4 *>(ring)[i] = make_uint4(0, 0, 0, 0);
        __syncwarp();
    }
    Found found[S::kStages];
#pragma unroll
    for (int i = 0; i < S::kStages; i++) found[i] = find(mine + i * step);
#pragma unroll
    for (int i = 0; i < S::kStages - 1; i++) {
        if (mine + i * step < end) fetch(found[i], i);
        copies_commit();
    }
    Found next_found = found[S::kStages - 1];
    int next = mine + (S::kStages - 1) * step, fill = S::kStages - 1;

    if (S::kQShared) __syncthreads();
    if (S::kF32) {
        for (int i = threadIdx.x; i < kHeads * 64 * NV; i += 32 * S::kWarps) {
            const int h = i / (64 * NV), e = i % (64 * NV);
            qs[i] = h < nh && e < a.d ? to_f32(qp[h * a.q_head + e]) : 0.f;
        }
        __syncthreads();
    }
    // ---- state: maximum and sum of the lane's heads (the sums of this lane's keys alone), and O
    float m[HL], l[HL];
#pragma unroll
    for (int h = 0; h < HL; h++) {
        m[h] = -CUDART_INF_F;
        l[h] = 0.f;
    }
    constexpr int kOut = S::kF32 ? (NV == 4 ? 2 : 1) * kHeads * 4 : 2 * HT * NV;
    float o[kOut];
#pragma unroll
    for (int i = 0; i < kOut; i++) o[i] = 0.f;
    // HT = 4: selectors that put one of a register's two weights on the even or on the odd index
    const uint32_t sel0 = g & 1 ? 0x1044 : 0x4410, sel1 = g & 1 ? 0x3244 : 0x4432;

    int use = 0;
    for (int t0 = mine; t0 < end; t0 += step) {
        if (next < end) {
            fetch(next_found, fill);
            next_found = find(next + step);
        }
        copies_commit();
        next += step;
        fill = fill + 1 == S::kStages ? 0 : fill + 1;
        copies_wait<S::kStages - 1>();
        __syncwarp();
        char *kt = ring + use * S::kBytes, *vt = kt + S::kKeys * S::kRow, *bk = vt + S::kKeys * S::kRow, *bv = bk + S::kKeys * S::kBook;
        const uint32_t mask = seen[use];
        if (LV) {
            Book<LV ? LV : 8>::split(bk + lane * S::kBook);
            if (S::kKeys == 32) Book<LV ? LV : 8>::split(bv + lane * S::kBook);  // (else the lanes 16 .. had those of the values)
            __syncwarp();
        }

        // ---- scores of each half: c[.][0] of key g, c[.][1] of key g + 8
        float c[S::kHalves][2][HL];
        if constexpr (S::kF32) {
            float v[2][kHeads];
#pragma unroll
            for (int h = 0; h < kHeads; h++) v[0][h] = v[1][h] = 0.f;
#pragma unroll
            for (int i = 0; i < 4 * NV; i++) {
                if (16 * i >= a.d) break;
                const float4 x = *reinterpret_cast<const float4 *>(kt + S::k_at(g, t + 4 * i));
                const float4 y = *reinterpret_cast<const float4 *>(kt + S::k_at(g + 8, t + 4 * i));
#pragma unroll
                for (int h = 0; h < kHeads; h++) {
                    if (h >= nh) break;
                    const float4 q4 = *reinterpret_cast<const float4 *>(qs + h * 64 * NV + 4 * (t + 4 * i));
                    v[0][h] = fmaf(x.w, q4.w, fmaf(x.z, q4.z, fmaf(x.y, q4.y, fmaf(x.x, q4.x, v[0][h]))));
                    v[1][h] = fmaf(y.w, q4.w, fmaf(y.z, q4.z, fmaf(y.y, q4.y, fmaf(y.x, q4.x, v[1][h]))));
                }
            }
            // sums over t; lane t keeps the heads 2t, 2t + 1
#pragma unroll
            for (int u = 0; u < 2; u++) {
                float w[4];
#pragma unroll
                for (int h = 0; h < 4; h++) {
                    const float keep = t & 2 ? v[u][h + 4] : v[u][h], give = t & 2 ? v[u][h] : v[u][h + 4];
                    w[h] = keep + __shfl_xor_sync(0xffffffffu, give, 2);
                }
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const float keep = t & 1 ? w[h + 2] : w[h], give = t & 1 ? w[h] : w[h + 2];
                    c[0][u][h % HL] = keep + __shfl_xor_sync(0xffffffffu, give, 1);
                }
            }
        } else {
#pragma unroll
            for (int half = 0; half < S::kHalves; half++) {
                const char *kh16 = kt + half * kTile * S::kRow, *bh16 = bk + half * kTile * S::kBook;
                float c1[4] = {0.f, 0.f, 0.f, 0.f}, c2[4] = {0.f, 0.f, 0.f, 0.f};
                if constexpr (LV == 0) {
#pragma unroll
                    for (int i = 0; i < 2 * NV; i++) {
                        if (32 * i >= a.d) break;
                        const uint4 x = *reinterpret_cast<const uint4 *>(kh16 + S::k_at(g, t + 4 * i));
                        const uint4 y = *reinterpret_cast<const uint4 *>(kh16 + S::k_at(g + 8, t + 4 * i));
                        mma16<T>(c1, x.x, y.x, x.y, y.y, qf[4 * i], qf[4 * i + 1]);
                        mma16<T>(c2, x.z, y.z, x.w, y.w, qf[4 * i + 2], qf[4 * i + 3]);
                    }
                } else {
                    Book<LV> b0, b1;
                    b0.load(bh16 + g * S::kBook);
                    b1.load(bh16 + (g + 8) * S::kBook);
#pragma unroll
                    for (int i = 0; i < (NV == 4 ? 2 : 1); i++) {
                        constexpr int kWords = NV == 1 ? 2 : 4;
                        alignas(16) uint32_t x[kWords], y[kWords];
                        if constexpr (NV == 1) {
                            *reinterpret_cast<uint2 *>(x) = *reinterpret_cast<const uint2 *>(kh16 + g * S::kRow + 8 * t);
                            *reinterpret_cast<uint2 *>(y) = *reinterpret_cast<const uint2 *>(kh16 + (g + 8) * S::kRow + 8 * t);
                        } else {
                            *reinterpret_cast<uint4 *>(x) = *reinterpret_cast<const uint4 *>(kh16 + S::k_at(g, t + 4 * i));
                            *reinterpret_cast<uint4 *>(y) = *reinterpret_cast<const uint4 *>(kh16 + S::k_at(g + 8, t + 4 * i));
                        }
#pragma unroll
                        for (int w = 0; w < kWords; w++) {
                            alignas(16) uint32_t q4[4];
                            if (S::kQShared) *reinterpret_cast<uint4 *>(q4) = q_shared[32 * (kWords * i + w)];
                            else
#pragma unroll
                                for (int j = 0; j < 4; j++) q4[j] = qf[4 * (kWords * i + w) + j];
                            uint32_t xl, xh, yl, yh;
                            b0.template look<0>(x[w], xl, xh);
                            b1.template look<0>(y[w], yl, yh);
                            mma16<T>(c1, prmt(xl, xh, 0x5140), prmt(yl, yh, 0x5140), prmt(xl, xh, 0x7362), prmt(yl, yh, 0x7362), q4[0], q4[1]);
                            b0.template look<1>(x[w], xl, xh);
                            b1.template look<1>(y[w], yl, yh);
                            mma16<T>(c2, prmt(xl, xh, 0x5140), prmt(yl, yh, 0x5140), prmt(xl, xh, 0x7362), prmt(yl, yh, 0x7362), q4[2], q4[3]);
                        }
                    }
                }
#pragma unroll
                for (int h = 0; h < HL; h++) {
                    c[half][0][h] = c1[h] + c2[h];
                    c[half][1][h] = c1[2 + h] + c2[2 + h];
                }
            }
        }

        // ---- running maximum, weights, sums
        if (mask != S::kAll) {  // rows that are not seen hold zeros; their scores do not count
#pragma unroll
            for (int u = 0; u < 2 * S::kHalves; u++)
#pragma unroll
                for (int h = 0; h < HL; h++)
                    c[u >> 1][u & 1][h] = mask >> (8 * u + g) & 1 ? c[u >> 1][u & 1][h] * a.scale2 : -CUDART_INF_F;
        } else {
#pragma unroll
            for (int u = 0; u < 2 * S::kHalves; u++)
#pragma unroll
                for (int h = 0; h < HL; h++) c[u >> 1][u & 1][h] *= a.scale2;
        }
        float top[HL], base[HL];
        bool moved = false;
#pragma unroll
        for (int h = 0; h < HL; h++) {
            top[h] = fmaxf(c[0][0][h], c[0][1][h]);
            if (S::kHalves > 1) top[h] = fmaxf(top[h], fmaxf(c[S::kHalves - 1][0][h], c[S::kHalves - 1][1][h]));
#pragma unroll
            for (int x = 4; x < 32; x *= 2) top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], x));
            top[h] = fmaxf(top[h], m[h]);
            base[h] = top[h] == -CUDART_INF_F ? 0.f : top[h];  // with no weight yet the exponents are taken from 0
            moved |= top[h] != m[h];
        }
        if (__any_sync(0xffffffffu, moved)) {
            float s[HL];
#pragma unroll
            for (int h = 0; h < HL; h++) {
                s[h] = exp2_fast(m[h] - base[h]);
                l[h] *= s[h];
                m[h] = top[h];
            }
            if constexpr (S::kF32) {
#pragma unroll
                for (int h = 0; h < kHeads; h++) {  // this lane holds some entries of all heads
                    const float sh = __shfl_sync(0xffffffffu, s[h % HL], h / HL);
#pragma unroll
                    for (int i = 0; i < kOut / kHeads; i++) o[h * (kOut / kHeads) + i] *= sh;
                }
            } else {
#pragma unroll
                for (int i = 0; i < kOut; i++) o[i] *= s[i % HL];
            }
        }
#pragma unroll
        for (int h = 0; h < HL; h++)
#pragma unroll
            for (int half = 0; half < S::kHalves; half++) {
                c[half][0][h] = exp2_fast(c[half][0][h] - base[h]);
                c[half][1][h] = exp2_fast(c[half][1][h] - base[h]);
                l[h] += c[half][0][h] + c[half][1][h];
            }

        // ---- values
        if constexpr (S::kF32) {
            *reinterpret_cast<float2 *>(ps + g * kHeads + 2 * t) = make_float2(c[0][0][0], c[0][0][HL - 1]);
            *reinterpret_cast<float2 *>(ps + (g + 8) * kHeads + 2 * t) = make_float2(c[0][1][0], c[0][1][HL - 1]);
            __syncwarp();
            constexpr int kLanes = NV == 1 ? 16 : 32, kRows = 32 / kLanes, kCols = NV == 4 ? 2 : 1;
#pragma unroll 4
            for (int r = lane / kLanes; r < kTile; r += kRows) {
                const float4 p0 = *reinterpret_cast<const float4 *>(ps + r * kHeads), p1 = *reinterpret_cast<const float4 *>(ps + r * kHeads + 4);
                const float p[kHeads] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
#pragma unroll
                for (int i = 0; i < kCols; i++) {
                    const float4 x = *reinterpret_cast<const float4 *>(vt + S::v_at(S::v_row(r), lane % kLanes + 32 * i));
#pragma unroll
                    for (int h = 0; h < kHeads; h++) {
                        if (h >= nh) break;
                        float *oh = o + (h * kCols + i) * 4;
                        oh[0] = fmaf(p[h], x.x, oh[0]);
                        oh[1] = fmaf(p[h], x.y, oh[1]);
                        oh[2] = fmaf(p[h], x.z, oh[2]);
                        oh[3] = fmaf(p[h], x.w, oh[3]);
                    }
                }
            }
        } else {
#pragma unroll
          for (int part = 0; part < S::kHalves; part++) {
            const char *v16 = vt + part * kTile * S::kRow, *b16 = bv + part * kTile * S::kBook;
            // The weights as second operand, high parts and low parts.  After the transposition the lane holds those
            // of the keys 2t, 2t + 1 and of 2t + 8, 2t + 9, of head g or (HT = 4) g / 2.
            uint32_t hi[HT == 4 ? 4 : 2], lo[HT == 4 ? 4 : 2];
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const float w0 = c[part][u][0] * kLift<T>, w1 = c[part][u][HL - 1] * kLift<T>;
                const uint32_t h = pack2<T>(w0, w1);
                const float2 f = unpack2<T>(h);
                const uint32_t th = transpose8x8(h), tl = transpose8x8(pack2<T>(w0 - f.x, w1 - f.y));
                if constexpr (HT == 4) {
                    hi[2 * u] = prmt(th, 0, sel0);
                    hi[2 * u + 1] = prmt(th, 0, sel1);
                    lo[2 * u] = prmt(tl, 0, sel0);
                    lo[2 * u + 1] = prmt(tl, 0, sel1);
                } else {
                    hi[u] = th;
                    lo[u] = tl;
                }
            }
            // x[r]: four neighbouring entries (two registers) of the lane's key r; they go to o[HT j ..].
            auto put = [&](int j, const uint32_t (&x)[4][2]) {
                if constexpr (HT == 4) {
                    float(&acc)[4] = *reinterpret_cast<float(*)[4]>(o + 4 * j);
                    mma16<T>(acc, x[0][0], x[0][1], x[1][0], x[1][1], hi[0], hi[1]);
                    mma16<T>(acc, x[2][0], x[2][1], x[3][0], x[3][1], hi[2], hi[3]);
                    mma16<T>(acc, x[0][0], x[0][1], x[1][0], x[1][1], lo[0], lo[1]);
                    mma16<T>(acc, x[2][0], x[2][1], x[3][0], x[3][1], lo[2], lo[3]);
                } else {
#pragma unroll
                    for (int u = 0; u < 2; u++) {
                        float(&acc)[4] = *reinterpret_cast<float(*)[4]>(o + 8 * j + 4 * u);
                        const uint32_t a0 = prmt(x[0][u], x[1][u], 0x5410), a1 = prmt(x[0][u], x[1][u], 0x7632);
                        const uint32_t a2 = prmt(x[2][u], x[3][u], 0x5410), a3 = prmt(x[2][u], x[3][u], 0x7632);
                        mma16<T>(acc, a0, a1, a2, a3, hi[0], hi[1]);
                        mma16<T>(acc, a0, a1, a2, a3, lo[0], lo[1]);
                    }
                }
            };
            if constexpr (LV == 0) {
#pragma unroll
                for (int i = 0; i < NV; i++) {
                    if (64 * i >= a.d) break;
                    uint4 x[4];
#pragma unroll
                    for (int r = 0; r < 4; r++) x[r] = *reinterpret_cast<const uint4 *>(v16 + S::v_at(t + 4 * r, g + 8 * i));
                    put(2 * i, {{x[0].x, x[0].y}, {x[1].x, x[1].y}, {x[2].x, x[2].y}, {x[3].x, x[3].y}});
                    put(2 * i + 1, {{x[0].z, x[0].w}, {x[1].z, x[1].w}, {x[2].z, x[2].w}, {x[3].z, x[3].w}});
                }
            } else {
                Book<LV> bb[4];
                alignas(16) uint32_t x[4][NV];
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    bb[r].load(b16 + (t + 4 * r) * S::kBook);
                    if constexpr (NV == 1) x[r][0] = *reinterpret_cast<const uint32_t *>(v16 + S::v_at(t + 4 * r, 0) + 4 * g);
                    else if constexpr (NV == 2)
                        *reinterpret_cast<uint2 *>(x[r]) = *reinterpret_cast<const uint2 *>(v16 + S::v_at(t + 4 * r, g >> 1) + 8 * (g & 1));
                    else *reinterpret_cast<uint4 *>(x[r]) = *reinterpret_cast<const uint4 *>(v16 + S::v_at(t + 4 * r, g));
                }
                auto half = [&](int w, auto hh) {
                    constexpr int H = decltype(hh)::value;
                    uint32_t p[4][2];
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        uint32_t bl, bh;
                        bb[r].template look<H>(x[r][w], bl, bh);
                        p[r][0] = prmt(bl, bh, 0x5140);
                        p[r][1] = prmt(bl, bh, 0x7362);
                    }
                    put(2 * w + H, p);
                };
#pragma unroll
                for (int w = 0; w < NV; w++) {
                    half(w, std::integral_constant<int, 0>());
                    half(w, std::integral_constant<int, 1>());
                }
            }
          }
        }
        use = use + 1 == S::kStages ? 0 : use + 1;
        __syncwarp();
    }
    copies_wait<0>();
    if (bad_page && a.status) atomicOr(a.status, ECASQ_BAD_PAGE);

    // ---- the block's warps: maxima and sums, then each warp's O shrunk to the common maximum
#pragma unroll
    for (int h = 0; h < HL; h++) {
#pragma unroll
        for (int x = 4; x < 32; x *= 2) l[h] += __shfl_xor_sync(0xffffffffu, l[h], x);
        if (g == 0) {
            wmax[wid * kHeads + HL * t + h] = m[h];
            wsum[wid * kHeads + HL * t + h] = l[h];
        }
    }
    __syncthreads();
    auto top_of = [&](int h) {
        float x = wmax[h];
        for (int w = 1; w < S::kWarps; w++) x = fmaxf(x, wmax[w * kHeads + h]);
        return x;
    };
    auto shrink = [&](int w, int h, float x) { return x == -CUDART_INF_F ? 0.f : exp2_fast(wmax[w * kHeads + h] - x); };
    constexpr int kWide = 64 * NV;
    float *own = reinterpret_cast<float *>(ring);
    if constexpr (S::kF32) {
        constexpr int kLanes = NV == 1 ? 16 : 32, kCols = NV == 4 ? 2 : 1;
#pragma unroll
        for (int h = 0; h < kHeads; h++) {
            const float sh = shrink(wid, h, top_of(h));
#pragma unroll
            for (int i = 0; i < kCols; i++) {
                float *oh = o + (h * kCols + i) * 4;
                float4 x = make_float4(oh[0] * sh, oh[1] * sh, oh[2] * sh, oh[3] * sh);
                if (kLanes == 16) {
                    x.x += __shfl_xor_sync(0xffffffffu, x.x, 16);
                    x.y += __shfl_xor_sync(0xffffffffu, x.y, 16);
                    x.z += __shfl_xor_sync(0xffffffffu, x.z, 16);
                    x.w += __shfl_xor_sync(0xffffffffu, x.w, 16);
                }
                if (lane < kLanes) *reinterpret_cast<float4 *>(own + h * kWide + 4 * (lane + 32 * i)) = x;
            }
        }
    } else {
        float s[HL];
#pragma unroll
        for (int h = 0; h < HL; h++) s[h] = shrink(wid, HL * t + h, top_of(HL * t + h)) * (1.f / kLift<T>);
#pragma unroll
        for (int j = 0; j < 2 * NV; j++) {
            // four entries of the lane's heads: plain 8 (g + 8 i) + 4 (j mod 2), i = j div 2; coded 8 NV g + 4 j
            const int e = LV ? 8 * NV * g + 4 * j : 8 * (g + 8 * (j >> 1)) + 4 * (j & 1);
            const float *x = o + HT * j;
            if constexpr (HT == 4) {
                *reinterpret_cast<float4 *>(own + t * kWide + e) = make_float4(x[0] * s[0], x[1] * s[0], x[2] * s[0], x[3] * s[0]);
            } else {
#pragma unroll
                for (int h = 0; h < 2; h++)
                    *reinterpret_cast<float4 *>(own + (2 * t + h) * kWide + e) =
                        make_float4(x[h] * s[h % HL], x[2 + h] * s[h % HL], x[4 + h] * s[h % HL], x[6 + h] * s[h % HL]);
            }
        }
    }
    __syncthreads();
    const PartAt at(a.d);
    const int quads = a.d / 4;  // four entries a thread
    for (int i = threadIdx.x; i < nh * quads; i += 32 * S::kWarps) {
        const int h = i / quads, e = 4 * (i % quads);
        const float x = top_of(h);
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < S::kWarps; w++) {
            sum += wsum[w * kHeads + h] * shrink(w, h, x);
            const float4 y = *reinterpret_cast<const float4 *>(smem + w * S::kRing + 4 * (h * kWide + e));
            v.x += y.x;
            v.y += y.y;
            v.z += y.z;
            v.w += y.w;
        }
        if (CLUSTER && active > 1) {  // in the place of the first warp's, which only this thread reads
            *reinterpret_cast<float4 *>(smem + 4 * (h * kWide + e)) = v;
            if (e == 0) {
                bmax[h] = x;
                bsum[h] = sum;
            }
        } else if (active > 1) {
            float *part = at.at(a.part, seq, a.heads, h0 + h, a.splits, split);
            *reinterpret_cast<float4 *>(part + e) = v;
            if (e == 0) *reinterpret_cast<float2 *>(part + a.d) = make_float2(x, sum);
        } else {
            store_out<T>(a, seq, h0 + h, e, v, sum);
            if (e == 0 && a.lse) a.lse[seq * a.heads + h0 + h] = log_sum(x, sum);
        }
    }
    if constexpr (CLUSTER) {  // its blocks join each a share of the entries
        if (active <= 1) return;
        cluster_barrier();
        for (int i = threadIdx.x + 32 * S::kWarps * split; i < nh * quads; i += 32 * S::kWarps * active) {
            const int h = i / quads, e = 4 * (i % quads);
            float x = -CUDART_INF_F, sum = 0.f;
            for (int s = 0; s < active; s++) x = fmaxf(x, shared_of_rank(bmax + h, s));
            const float from = x == -CUDART_INF_F ? 0.f : x;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int s = 0; s < active; s++) {
                const float share = exp2_fast(shared_of_rank(bmax + h, s) - from);
                sum = fmaf(shared_of_rank(bsum + h, s), share, sum);
                float4 y;
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(y.x), "=f"(y.y), "=f"(y.z), "=f"(y.w) : "r"(of_rank(smem_addr(smem + 4 * (h * kWide + e)), s)) : "memory");
                v.x = fmaf(y.x, share, v.x);
                v.y = fmaf(y.y, share, v.y);
                v.z = fmaf(y.z, share, v.z);
                v.w = fmaf(y.w, share, v.w);
            }
            store_out<T>(a, seq, h0 + h, e, v, sum);
            if (e == 0 && a.lse) a.lse[seq * a.heads + h0 + h] = log_sum(x, sum);
        }
        cluster_barrier();  // a block's shared memory stays until all have read it
    }
}

// Blocks of a kernel that an SM holds; 0 if the query fails.
template <typename T, int LV, int NV, int HT, bool CLUSTER>
static int prepare_attend() {
    using S = Shape<T, LV, NV>;
    int n = 0;
    if (cudaFuncSetAttribute(k_attend<T, LV, NV, HT, CLUSTER>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem) != cudaSuccess) return 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k_attend<T, LV, NV, HT, CLUSTER>, 32 * S::kWarps, S::kSmem) != cudaSuccess) return 0;
    return n;
}
// Splits the sequences (split_attend) and launches.
template <typename T, int LV, int NV, int HT>
static int launch_attend(AttendArgs &a, int64_t b, cudaStream_t st) {
    using S = Shape<T, LV, NV>;
    static std::atomic<int> known[kDevices];  // by device, once each
    int device = 0;
    ECASQ_CUDA_TRY(cudaGetDevice(&device));
    int resident = device < kDevices ? known[device].load(std::memory_order_acquire) : 0;
    if (resident < 1) {
        resident = std::min(prepare_attend<T, LV, NV, HT, false>(), prepare_attend<T, LV, NV, HT, true>());
        if (resident < 1) return ECASQ_ECUDA;
        if (device < kDevices) known[device].store(resident, std::memory_order_release);
    }
    a.tile = S::kKeys;
    a.step = S::kKeys * 4;
    const int rc = split_attend(a, b, resident);
    if (rc) return rc;
    const dim3 grid((unsigned)(a.heads / a.group * a.htiles), (unsigned)a.splits, (unsigned)b);
    if (a.cluster) return launch_clusters(k_attend<T, LV, NV, HT, true>, grid, dim3(1, (unsigned)a.splits), 32 * S::kWarps, S::kSmem, st, a);
    return launch_early(k_attend<T, LV, NV, HT, false>, grid, 32 * S::kWarps, S::kSmem, st, a);
}
template <typename T, int LV, int HT>
static int launch_attend_rows(AttendArgs &a, int64_t b, cudaStream_t st) {
    if (a.d <= 64) return launch_attend<T, LV, 1, HT>(a, b, st);
    if (a.d <= 128) return launch_attend<T, LV, 2, HT>(a, b, st);
    return launch_attend<T, LV, 4, HT>(a, b, st);
}
template <typename T, int LV>
static int launch_attend_heads(AttendArgs &a, int64_t b, cudaStream_t st) {
    return a.group <= 4 ? launch_attend_rows<T, LV, 4>(a, b, st) : launch_attend_rows<T, LV, 8>(a, b, st);
}

// One translation unit each.
int launch_attend_f32(AttendArgs &a, int64_t b, cudaStream_t st);
int launch_attend_16(AttendArgs &a, bool bf16, int64_t b, cudaStream_t st);
int launch_attend_coded8(AttendArgs &a, bool bf16, int64_t b, cudaStream_t st);
int launch_attend_coded16(AttendArgs &a, bool bf16, int64_t b, cudaStream_t st);

}  // namespace ecasq
