// What the attention kernels share: their arguments, the ranges of a sequence, and the launchers of the translation units.
#pragma once

#include <algorithm>

#include "common.cuh"

namespace e2egrec {

constexpr int kMaxAttnDim = 256;
constexpr int kMaxSplits = 256;              // stretches of the keys, at most
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Rows (query i, head g of its group) of one key head count as the rows of one matrix: row i * group + g.
struct AttnArgs {
    const void *q, *k, *v, *o, *dout;     // o, dout: backward only
    void *out, *dq, *dk, *dv;
    int64_t ldq, ldk, ldv, ldo, ldg;      // ld of q, k, v, out (both passes), dout
    int64_t ldq2, ldk2, ldv2;             // ld of dq, dk, dv
    float *lse;                           // [q_rows x heads], forward: may be null
    const int64_t *q_ptr, *k_ptr;
    const uint8_t *mask;
    int32_t *status;
    int64_t n_seq, q_rows, k_rows;
    int32_t kv_heads, group, head_dim;
    float scale;
};

struct SeqRange {
    int64_t q0, q1, k0, k1;
};

// Rows of sequence s, brought into the matrices' bounds; offsets that were not in order are reported.
__device__ inline SeqRange seq_range(const AttnArgs &a, int64_t s, bool report)
{
    SeqRange r{__ldg(a.q_ptr + s), __ldg(a.q_ptr + s + 1), __ldg(a.k_ptr + s), __ldg(a.k_ptr + s + 1)};
    const bool bad = r.q0 < 0 || r.q1 < r.q0 || r.q1 > a.q_rows || r.k0 < 0 || r.k1 < r.k0 || r.k1 > a.k_rows;
    if (bad) {
        r.q0 = min(max(r.q0, (int64_t)0), a.q_rows);
        r.q1 = min(max(r.q1, r.q0), a.q_rows);
        r.k0 = min(max(r.k0, (int64_t)0), a.k_rows);
        r.k1 = min(max(r.k1, r.k0), a.k_rows);
        if (report && a.status) atomicOr(reinterpret_cast<unsigned *>(a.status), E2EGREC_DEV_RANGE);
    }
    return r;
}

// The sequence that owns row `row` of a list of offsets (the last s with ptr[s] <= row), or -1
__device__ inline int64_t owner(const int64_t *ptr, int64_t n_seq, int64_t row)
{
    if (n_seq < 1 || row < ptr[0]) return -1;
    int64_t lo = 0, hi = n_seq;                      // ptr[lo] <= row < ptr[hi], if the list does not decrease
    while (hi - lo > 1) {
        const int64_t m = (lo + hi) >> 1;
        if (ptr[m] <= row) lo = m;
        else hi = m;
    }
    return row < ptr[lo + 1] ? lo : -1;
}

// Lengths that a call is planned by: the longest that a sequence can have (the caller's hint, else all rows), the mean, and the one that
// the kernels are chosen for: the hint, without one the mean.
struct Lengths {
    int64_t longest, mean, typical;
};

// Blocks per unit (a key head of a sequence) for pieces of `per` rows, which walk sequences of more pieces in rounds: as many as a sequence of
// twice the mean takes, or kSpread in all if that is more.  Sized by the longest alone, the units of many sequences are nearly all empty
// ones (4096 of one token and 62 states, longest unknown: 32 million of them, 104 ms, 0.4 so).
constexpr int64_t kSpread = 148 * 64;
inline int64_t blocks_per_unit(const Lengths &l, int64_t factor, int64_t per, int64_t units)
{
    const int64_t want = std::max(ceil_div(2 * l.mean * factor, per), ceil_div(kSpread, units));
    return std::max<int64_t>(1, std::min({ceil_div(l.longest * factor, per), want, (((int64_t)1 << 31) - 1) / units}));
}

// attention_tc.cu: bf16, head_dim <= 128.  tiles: blocks of 256 rows (128 with one_tile) per sequence and key head, longer sequences go
// round again; splits: stretches of the keys, whose results (out in fp32 and (maximum in powers of two, sum)) go to
// part_o [splits x q_rows x heads x head_dim] and part_ml [splits x q_rows x heads] where splits > 1.
bool tc_attention_forward(const AttnArgs &a, int64_t tiles, int splits, bool one_tile, float *part_o, float2 *part_ml, cudaStream_t st);
// q_tiles, k_tiles: tiles of 128 rows and of 128 keys per sequence and key head; dots: [q_rows x heads] scratch
bool tc_attention_backward(const AttnArgs &a, int64_t q_tiles, int64_t k_tiles, float *dots, cudaStream_t st);

// attention_few.cu: streaming kernels, fp32 and bf16, head_dim <= 256
struct FewPlan {
    int rows;                             // rows per unit
    int steps;                            // steps of keys in flight per warp
    bool both;                            // backward: one kernel for dQ, dK and dV
    bool fit;                             // backward, bf16, more keys than one turn: dQ without what D of the stored outputs lacks
    int64_t batches;                      // units of rows per sequence and key head
    int warps, splits;                    // warps per unit, stretches of the keys
    int64_t key_batches;                  // units of keys of the dK, dV kernel
};
FewPlan few_plan(const AttnArgs &a, const Lengths &q, const Lengths &k, int es, bool backward);
bool few_attention_forward(const AttnArgs &a, const FewPlan &p, int32_t dtype, float *part_o, float2 *part_ml, cudaStream_t st);
// part_dq: [splits x q_rows x heads x head_dim] where splits > 1, twice that and [splits x q_rows x heads] with fit; dots: [q_rows x heads] where !both
bool few_attention_backward(const AttnArgs &a, const FewPlan &p, int32_t dtype, float *part_dq, float *dots, cudaStream_t st);

// dQ of stretches of the keys -> dQ, in order; with fit what D lacks is added to dots (where there are any)
void join_dq(const AttnArgs &a, int splits, int32_t dtype, bool fit, const float *part_dq, float *dots, cudaStream_t st);

// attention_simt.cu: fp32, head_dim <= 128, tiles of 64 rows x 64 keys
struct SimtPlan {
    int rows;                             // of a tile: 16, 32 or 64
    int64_t q_tiles, k_tiles;             // blocks of rows / of keys per sequence and key head
    int splits;                           // stretches of the keys (forward, dQ)
};
SimtPlan simt_plan(const AttnArgs &a, const Lengths &q, const Lengths &k);
bool simt_attention_forward(const AttnArgs &a, const SimtPlan &p, float *part_o, float2 *part_ml, cudaStream_t st);
bool simt_attention_backward(const AttnArgs &a, const SimtPlan &p, float *part_dq, float *dots, cudaStream_t st);

}  // namespace e2egrec
