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

__device__ __forceinline__ uint2 drop_key(const DropArgs &d) { return make_uint2(d.seed_lo, d.seed_hi); }
__device__ __forceinline__ PhiloxUnit drop_of_unit(const DropArgs &d, uint32_t step, uint32_t unit) { return philox_unit(unit, d.place, step, drop_key(d)); }
__device__ __forceinline__ PhiloxRow drop_of_row(const DropArgs &d, uint32_t row) { return philox_row(row, d.place, drop_key(d)); }
__device__ __forceinline__ uint4 drop_words(const DropArgs &d, const PhiloxUnit &u, const PhiloxRow &r) { return philox_join(u, r, drop_key(d)); }

// The words of a chunk: all four of its unit (bf16, 8 elements), or the first or second two (fp32)
template <int E> __device__ __forceinline__ void drop_halves(const uint4 &w, int chunk, uint32_t (&h)[E / 2])
{
    const bool second = E == 4 && (chunk & 1);
    h[0] = second ? w.z : w.x;
    h[1] = second ? w.w : w.y;
    if constexpr (E == 8) {
        h[2] = w.z;
        h[3] = w.w;
    }
}
// A chunk's elements, two by two
template <int N> __device__ __forceinline__ void drop_apply(const DropArgs &d, const uint32_t (&h)[N], float2 (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float2 x = __fmul2_rn(v[i], make_float2(d.factor, d.factor));
        v[i] = make_float2((h[i] << 16) < d.cut ? 0.f : x.x, h[i] < d.cut ? 0.f : x.y);
    }
}

// 16 bytes of a row as pairs of fp32, and back
__device__ __forceinline__ void unpack_pairs(const uint4 &r, float2 (&v)[4])
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ void unpack_pairs(const uint4 &r, float2 (&v)[2])
{
    v[0] = make_float2(__uint_as_float(r.x), __uint_as_float(r.y));
    v[1] = make_float2(__uint_as_float(r.z), __uint_as_float(r.w));
}
template <typename T, int N> __device__ __forceinline__ void store_pairs(T *p, const float2 (&v)[N])
{
    float x[2 * N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[2 * i] = v[i].x;
        x[2 * i + 1] = v[i].y;
    }
    Chunk<T>::store(p, x);
}

// The unit of a row's chunk
template <typename T> __device__ __forceinline__ uint32_t drop_unit(int chunk) { return (uint32_t)chunk / (8u / Chunk<T>::kElems); }

}  // namespace e2egrec
