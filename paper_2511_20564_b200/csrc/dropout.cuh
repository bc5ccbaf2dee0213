// Dropout from a counter-based generator: which elements stay is formed from (seed, place, step, row, column) wherever it is needed, in
// the backward pass as in the forward pass, and stored nowhere.
//
// Element (row, col) has 16 bits: half col % 8 of the four words of Philox4x32-10 with key seed and counter (col / 8, row, 2^31 + place, step).
// It is dropped where they lie below t = round(p 2^16), else multiplied by 2^16 / (2^16 - t), so that the expectation is the element.  One
// call of the generator serves the 8 elements of 16 bytes of bf16.  (The sampler's counters have 2^8 + hop in their third word.)
#pragma once

#include "common.cuh"
#include "philox.cuh"

namespace e2egrec {

// t is kept shifted up by 16, as the halves are compared
struct DropArgs {
    uint32_t cut;                         // t << 16; 0: nothing is dropped
    float factor;
    uint32_t seed_lo, seed_hi, place, step;
    const uint32_t *step_dev;             // added to step; may be null
};

// The arguments of a call -> the kernels'; a null plan drops nothing
inline int32_t drop_args(const e2egrec_dropout *d, DropArgs &a)
{
    a = DropArgs{};
    a.factor = 1.f;
    if (!d) return E2EGREC_OK;
    if (!(d->p >= 0.) || !(d->p < 1.) || d->place >> 31) return E2EGREC_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(d->step_dev) % sizeof(uint32_t)) return E2EGREC_ERR_ALIGN;
    uint32_t t = (uint32_t)(d->p * 65536. + 0.5);
    if (t > 65535u) t = 65535u;
    a.cut = t << 16;
    a.factor = 65536.f / (float)(65536u - t);
    a.seed_lo = (uint32_t)d->seed;
    a.seed_hi = (uint32_t)(d->seed >> 32);
    a.place = 0x80000000u | d->place;
    a.step = d->step;
    a.step_dev = d->step_dev;
    return E2EGREC_OK;
}

__device__ __forceinline__ uint32_t drop_step(const DropArgs &d) { return d.step + (d.step_dev ? __ldcg(d.step_dev) : 0u); }

__device__ __forceinline__ uint4 drop_words(const DropArgs &d, uint32_t step, uint32_t row, uint32_t unit)
{
    return philox4x32_10(make_uint4(unit, row, d.place, step), make_uint2(d.seed_lo, d.seed_hi));
}

// Which elements of a chunk stay, a bit each: the 8 of a unit (bf16), or its first or second 4 (fp32)
template <int E> __device__ __forceinline__ uint32_t drop_bits(const DropArgs &d, const uint4 &w, int chunk)
{
    const bool second = E == 4 && (chunk & 1);
    const uint32_t words[4] = {second ? w.z : w.x, second ? w.w : w.y, w.z, w.w};
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < E; e += 2) bits |= ((words[e / 2] << 16) >= d.cut ? 1u << e : 0u) | (words[e / 2] >= d.cut ? 2u << e : 0u);
    return bits;
}
template <int E> __device__ __forceinline__ void drop_apply(const DropArgs &d, uint32_t bits, float (&v)[E])
{
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = bits >> e & 1u ? v[e] * d.factor : 0.f;
}
template <typename T> __device__ __forceinline__ uint32_t drop_unit(int chunk) { return (uint32_t)chunk / (8u / Chunk<T>::kElems); }

}  // namespace e2egrec
