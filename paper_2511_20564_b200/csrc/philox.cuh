// The counter-based generator of the sampler's draws and of dropout.
#pragma once

#include <stdint.h>

namespace e2egrec {

// ---------------------------------------------------------------------------------------
// Philox4x32-10 (Salmon et al., SC'11): ten rounds of two 32x32->64 multiplies with a
// Weyl key schedule.
// ---------------------------------------------------------------------------------------
constexpr uint32_t kPhiloxM0 = 0xD2511F53u, kPhiloxM1 = 0xCD9E8D57u, kPhiloxW0 = 0x9E3779B9u, kPhiloxW1 = 0xBB67AE85u;

// rounds `from` to 9, with the key of round 0
__device__ __forceinline__ uint4 philox_rounds(uint4 c, uint2 k, int from)
{
#pragma unroll
    for (int r = from; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)kPhiloxM0 * c.x, p1 = (uint64_t)kPhiloxM1 * c.z;
        c = make_uint4((uint32_t)(p1 >> 32) ^ c.y ^ (k.x + r * kPhiloxW0), (uint32_t)p1, (uint32_t)(p0 >> 32) ^ c.w ^ (k.y + r * kPhiloxW1), (uint32_t)p0);
    }
    return c;
}
__device__ __forceinline__ uint4 philox4x32_10(uint4 c, uint2 k) { return philox_rounds(c, k, 0); }

// Ten rounds of counters (unit, row, c2, c3) whose units or rows are the same for many: what of the first three rounds depends on one of them alone
// (four of their six products) is formed once.  With a round as (x, y, z, w) -> (hi(M1 z) ^ y ^ k0, lo(M1 z), hi(M0 x) ^ w ^ k1, lo(M0 x)): round 1
// makes x of the row and z, w of the unit, round 2 x, y of the unit and w of the row, round 3 multiplies the unit's x.
struct PhiloxUnit {
    uint32_t w1, y2, z3, w3;                             // w1, y2, z3 with the key of the round that they go into
};
struct PhiloxRow {
    uint32_t hi, lo;
};
__device__ __forceinline__ PhiloxUnit philox_unit(uint32_t unit, uint32_t c2, uint32_t c3, uint2 k)
{
    const uint64_t a = (uint64_t)kPhiloxM0 * unit, b = (uint64_t)kPhiloxM1 * c2;
    const uint64_t p1 = (uint64_t)kPhiloxM1 * ((uint32_t)(a >> 32) ^ c3 ^ k.y);
    const uint64_t p0 = (uint64_t)kPhiloxM0 * ((uint32_t)(p1 >> 32) ^ (uint32_t)b ^ (k.x + kPhiloxW0));
    return PhiloxUnit{(uint32_t)a ^ (k.y + kPhiloxW1), (uint32_t)p1 ^ (k.x + 2 * kPhiloxW0), (uint32_t)(p0 >> 32) ^ (k.y + 2 * kPhiloxW1), (uint32_t)p0};
}
__device__ __forceinline__ PhiloxRow philox_row(uint32_t row, uint32_t c2, uint2 k)
{
    const uint64_t b = (uint64_t)kPhiloxM1 * c2, p0 = (uint64_t)kPhiloxM0 * ((uint32_t)(b >> 32) ^ row ^ k.x);
    return PhiloxRow{(uint32_t)(p0 >> 32), (uint32_t)p0};
}
__device__ __forceinline__ uint4 philox_join(const PhiloxUnit &u, const PhiloxRow &r, uint2 k)
{
    const uint64_t p1 = (uint64_t)kPhiloxM1 * (r.hi ^ u.w1);
    return philox_rounds(make_uint4((uint32_t)(p1 >> 32) ^ u.y2, (uint32_t)p1, u.z3 ^ r.lo, u.w3), k, 3);
}

}  // namespace e2egrec
