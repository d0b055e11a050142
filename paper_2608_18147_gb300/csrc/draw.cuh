// draw.cuh -- the encodes' random bits: SplitMix64 (Steele, Lea and Flood 2014) of a counter, in 32-bit limbs.
#pragma once

#include <stdint.h>

namespace ecasq {

constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;
constexpr uint32_t kC1lo = 0x1CE4E5B9u, kC1hi = 0xBF58476Du;  // SplitMix64 multipliers (Steele, Lea, Flood 2014)
constexpr uint32_t kC2lo = 0x133111EBu, kC2hi = 0x94D049BBu;

// Bits 32..63 of the SplitMix64 output for state z = (zh:zl).
__device__ __forceinline__ uint32_t splitmix64_hi(uint32_t zl, uint32_t zh) {
    const uint32_t xl = zl ^ __funnelshift_r(zl, zh, 30), xh = zh ^ (zh >> 30);  // z ^ (z >> 30)
    const uint64_t w = (uint64_t)xl * kC1lo;                                       // (xh:xl) * C1 mod 2^64
    const uint32_t al = (uint32_t)w;
    const uint32_t ah = (uint32_t)(w >> 32) + xl * kC1hi + xh * kC1lo;
    const uint32_t yl = al ^ __funnelshift_r(al, ah, 27), yh = ah ^ (ah >> 27);   // a ^ (a >> 27)
    return __umulhi(yl, kC2lo) + yl * kC2hi + yh * kC2lo;                         // top word of y * C2
}

// 64-bit counter state (zh:zl) advanced by gamma.
__device__ __forceinline__ void add_gamma(uint32_t &zl, uint32_t &zh) {
    const uint64_t z = (((uint64_t)zh << 32) | zl) + kGamma;
    zl = (uint32_t)z;
    zh = (uint32_t)(z >> 32);
}

}  // namespace ecasq
