// What the attention kernels share: their arguments, the ranges of a sequence, and the launchers of the translation units.
#pragma once

#include "common.cuh"

namespace e2egrec {

constexpr int kMaxAttnDim = 256;
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

}  // namespace e2egrec
