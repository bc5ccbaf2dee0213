// Attention of ragged sequences of tokens to ragged sequences of states: argument checks and the choice of kernels, and the
// kernels by rows of fp32 FMA that every shape can take.
#include <algorithm>

#include "attention.cuh"

namespace e2egrec {
namespace {

constexpr int kRowThreads = 256;

__device__ inline float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// One warp per (query row, head).
template <typename T, int N>
__global__ void __launch_bounds__(kRowThreads) attn_row_kernel(const __grid_constant__ AttnArgs a)
{
    const int lane = threadIdx.x & 31, heads = a.kv_heads * a.group;
    const int64_t unit = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) >> 5;
    const int64_t row = unit / heads;
    const int h = (int)(unit % heads);
    if (row >= a.q_rows) return;
    const int64_t s = owner(a.q_ptr, a.n_seq, row);
    if (s < 0) return;
    const SeqRange r = seq_range(a, s, lane == 0);
    const int64_t off = (int64_t)(h / a.group) * a.head_dim;
    float q[N], o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + 32 * i;
        q[i] = e < a.head_dim ? to_float<T>(static_cast<const T *>(a.q)[row * a.ldq + (int64_t)h * a.head_dim + e]) : 0.f;
        o[i] = 0.f;
    }
    float m = -INFINITY, l = 0.f;
    for (int64_t j = r.k0; j < r.k1; ++j) {
        if (a.mask && !a.mask[j]) continue;
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = lane + 32 * i;
            if (e < a.head_dim) t += q[i] * to_float<T>(static_cast<const T *>(a.k)[j * a.ldk + off + e]);
        }
        t = warp_sum(t) * a.scale;
        const float m2 = fmaxf(m, t), base = m2 == -INFINITY ? 0.f : m2;
        const float c = expf(m - base), p = expf(t - base);
        m = m2;
        l = l * c + p;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = lane + 32 * i;
            if (e < a.head_dim) o[i] = o[i] * c + p * to_float<T>(static_cast<const T *>(a.v)[j * a.ldv + off + e]);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + 32 * i;
        if (e < a.head_dim) static_cast<T *>(a.out)[row * a.ldo + (int64_t)h * a.head_dim + e] = from_float<T>(l == 0.f ? 0.f : o[i] / l);
    }
    if (a.lse && lane == 0) a.lse[row * heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

// dQ: one warp per (query row, head)
template <typename T, int N>
__global__ void __launch_bounds__(kRowThreads) attn_row_dq_kernel(const __grid_constant__ AttnArgs a)
{
    const int lane = threadIdx.x & 31, heads = a.kv_heads * a.group;
    const int64_t unit = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) >> 5;
    const int64_t row = unit / heads;
    const int h = (int)(unit % heads);
    if (row >= a.q_rows) return;
    const int64_t s = owner(a.q_ptr, a.n_seq, row);
    if (s < 0) return;
    const SeqRange r = seq_range(a, s, lane == 0);
    const int64_t off = (int64_t)(h / a.group) * a.head_dim, hoff = (int64_t)h * a.head_dim;
    float q[N], g[N], dq[N];
    float d = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + 32 * i;
        const bool on = e < a.head_dim;
        q[i] = on ? to_float<T>(static_cast<const T *>(a.q)[row * a.ldq + hoff + e]) : 0.f;
        g[i] = on ? to_float<T>(static_cast<const T *>(a.dout)[row * a.ldg + hoff + e]) : 0.f;
        if (on) d += g[i] * to_float<T>(static_cast<const T *>(a.o)[row * a.ldo + hoff + e]);
        dq[i] = 0.f;
    }
    d = warp_sum(d);
    const float lse = a.lse[row * heads + h];
    if (lse != -INFINITY)
        for (int64_t j = r.k0; j < r.k1; ++j) {
            if (a.mask && !a.mask[j]) continue;
            float t = 0.f, u = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int e = lane + 32 * i;
                if (e < a.head_dim) {
                    t += q[i] * to_float<T>(static_cast<const T *>(a.k)[j * a.ldk + off + e]);
                    u += g[i] * to_float<T>(static_cast<const T *>(a.v)[j * a.ldv + off + e]);
                }
            }
            const float p = expf(warp_sum(t) * a.scale - lse), ds = p * (warp_sum(u) - d) * a.scale;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int e = lane + 32 * i;
                if (e < a.head_dim) dq[i] += ds * to_float<T>(static_cast<const T *>(a.k)[j * a.ldk + off + e]);
            }
        }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + 32 * i;
        if (e < a.head_dim) static_cast<T *>(a.dq)[row * a.ldq2 + hoff + e] = from_float<T>(dq[i]);
    }
}

// dK, dV: one warp per (key row, key head)
template <typename T, int N>
__global__ void __launch_bounds__(kRowThreads) attn_row_dkv_kernel(const __grid_constant__ AttnArgs a)
{
    const int lane = threadIdx.x & 31, heads = a.kv_heads * a.group;
    const int64_t unit = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) >> 5;
    const int64_t row = unit / a.kv_heads;
    const int h = (int)(unit % a.kv_heads);
    if (row >= a.k_rows) return;
    const int64_t s = owner(a.k_ptr, a.n_seq, row);
    if (s < 0) return;
    const SeqRange r = seq_range(a, s, lane == 0);
    const int64_t off = (int64_t)h * a.head_dim;
    const bool seen = !a.mask || a.mask[row];
    float k[N], v[N], dk[N], dv[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + 32 * i;
        k[i] = e < a.head_dim ? to_float<T>(static_cast<const T *>(a.k)[row * a.ldk + off + e]) : 0.f;
        v[i] = e < a.head_dim ? to_float<T>(static_cast<const T *>(a.v)[row * a.ldv + off + e]) : 0.f;
        dk[i] = dv[i] = 0.f;
    }
    if (seen)
        for (int64_t i0 = r.q0; i0 < r.q1; ++i0)
            for (int g = 0; g < a.group; ++g) {
                const int64_t hoff = (int64_t)(h * a.group + g) * a.head_dim;
                const float lse = a.lse[i0 * heads + h * a.group + g];
                if (lse == -INFINITY) continue;
                float q[N], go[N], t = 0.f, u = 0.f, d = 0.f;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int e = lane + 32 * i;
                    const bool on = e < a.head_dim;
                    q[i] = on ? to_float<T>(static_cast<const T *>(a.q)[i0 * a.ldq + hoff + e]) : 0.f;
                    go[i] = on ? to_float<T>(static_cast<const T *>(a.dout)[i0 * a.ldg + hoff + e]) : 0.f;
                    t += q[i] * k[i];
                    u += go[i] * v[i];
                    if (on) d += go[i] * to_float<T>(static_cast<const T *>(a.o)[i0 * a.ldo + hoff + e]);
                }
                const float p = expf(warp_sum(t) * a.scale - lse), ds = p * (warp_sum(u) - warp_sum(d)) * a.scale;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dk[i] += ds * q[i];
                    dv[i] += p * go[i];
                }
            }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + 32 * i;
        if (e < a.head_dim) {
            static_cast<T *>(a.dk)[row * a.ldk2 + off + e] = from_float<T>(dk[i]);
            static_cast<T *>(a.dv)[row * a.ldv2 + off + e] = from_float<T>(dv[i]);
        }
    }
}

unsigned row_grid(int64_t rows, int heads) { return (unsigned)ceil_div(rows * heads, kRowThreads / 32); }

// Results of stretches of the keys -> out, lse: one warp per (row, head), stretches in order
template <typename T>
__global__ void __launch_bounds__(kRowThreads)
attn_join_kernel(const __grid_constant__ AttnArgs a, int splits, const float *__restrict__ part_o, const float2 *__restrict__ part_ml)
{
    const int lane = threadIdx.x & 31, heads = a.kv_heads * a.group;
    const int64_t unit = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) >> 5, stride = a.q_rows * heads;
    const int64_t row = unit / heads;
    const int h = (int)(unit % heads);
    if (row >= a.q_rows || owner(a.q_ptr, a.n_seq, row) < 0) return;
    float m = -INFINITY, l = 0.f;
    for (int z = 0; z < splits; ++z) m = fmaxf(m, part_ml[z * stride + unit].x);
    const float base = m == -INFINITY ? 0.f : m;
    for (int z = 0; z < splits; ++z) {
        const float2 p = part_ml[z * stride + unit];
        l += p.y == 0.f ? 0.f : p.y * exp2f(p.x - base);
    }
    for (int e = lane; e < a.head_dim; e += 32) {
        float o = 0.f;
        for (int z = 0; z < splits; ++z) {
            const float2 p = part_ml[z * stride + unit];
            if (p.y != 0.f) o += p.y * exp2f(p.x - base) * part_o[(z * stride + unit) * a.head_dim + e];
        }
        static_cast<T *>(a.out)[row * a.ldo + (int64_t)h * a.head_dim + e] = from_float<T>(l == 0.f ? 0.f : o / l);
    }
    if (a.lse && lane == 0) a.lse[unit] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <typename T> void row_forward(const AttnArgs &a, cudaStream_t st)
{
    note_launch();
    const unsigned g = row_grid(a.q_rows, a.kv_heads * a.group);
    if (a.head_dim <= 128) attn_row_kernel<T, 4><<<g, kRowThreads, 0, st>>>(a);
    else attn_row_kernel<T, 8><<<g, kRowThreads, 0, st>>>(a);
}

template <typename T> void row_backward(const AttnArgs &a, cudaStream_t st)
{
    note_launch();
    note_launch();
    const unsigned g = row_grid(a.q_rows, a.kv_heads * a.group), gk = row_grid(a.k_rows, a.kv_heads);
    if (a.head_dim <= 128) {
        if (a.q_rows) attn_row_dq_kernel<T, 4><<<g, kRowThreads, 0, st>>>(a);
        if (a.k_rows) attn_row_dkv_kernel<T, 4><<<gk, kRowThreads, 0, st>>>(a);
    } else {
        if (a.q_rows) attn_row_dq_kernel<T, 8><<<g, kRowThreads, 0, st>>>(a);
        if (a.k_rows) attn_row_dkv_kernel<T, 8><<<gk, kRowThreads, 0, st>>>(a);
    }
}

// Shapes, types and alignment of one matrix of heads
int32_t check_heads(const e2egrec_mat *m, int32_t heads, int32_t head_dim, int32_t dtype, int64_t rows)
{
    if (!m || (!m->data && m->rows > 0)) return E2EGREC_ERR_NULL;
    if (m->dtype != E2EGREC_F32 && m->dtype != E2EGREC_BF16) return E2EGREC_ERR_DTYPE;
    if (m->dtype != dtype) return E2EGREC_ERR_DTYPE;
    if (m->rows != rows || (int64_t)heads * head_dim != m->dim || m->ld < m->dim) return E2EGREC_ERR_ARG;
    const int64_t es = (int64_t)dtype_size(dtype);
    if (head_dim * es % 16 || m->ld * es % 16 || reinterpret_cast<uintptr_t>(m->data) % 16) return E2EGREC_ERR_ALIGN;
    return E2EGREC_OK;
}

constexpr int64_t kMaxRows = (int64_t)1 << 31;

// How a forward call is carried out
struct FwdPlan {
    bool tc;
    int64_t tiles;                        // blocks of rows per sequence and key head
    int splits;                           // stretches of the keys
    size_t o_bytes, ml_bytes;             // their results
};

FwdPlan plan_forward(const AttnArgs &a, const e2egrec_sequences &s, int32_t dtype)
{
    FwdPlan p{};
    p.splits = 1;
    p.tc = dtype == E2EGREC_BF16 && a.head_dim <= 128;
    const int64_t max_q = s.max_q ? std::min(s.max_q, a.q_rows) : a.q_rows, max_k = s.max_k ? std::min(s.max_k, a.k_rows) : a.k_rows;
    if (p.tc) {
        const int64_t units = std::max<int64_t>(a.n_seq * a.kv_heads, 1);
        p.tiles = std::max<int64_t>(1, std::min(ceil_div(max_q * a.group, tc_fwd_rows()), (kMaxRows - 1) / units));
        const int64_t blocks = units * p.tiles;
        if (blocks < 148) p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({148 / blocks, max_k / 512, 64}));
    }
    if (p.splits > 1) {
        p.ml_bytes = align_up((size_t)p.splits * a.q_rows * a.kv_heads * a.group * sizeof(float2), 256);
        p.o_bytes = align_up((size_t)p.splits * a.q_rows * a.kv_heads * a.group * a.head_dim * sizeof(float), 256);
    }
    return p;
}

struct BwdPlan {
    bool tc;
    int64_t q_tiles, k_tiles;
    size_t dot_bytes;
};

BwdPlan plan_backward(const AttnArgs &a, const e2egrec_sequences &s, int32_t dtype)
{
    BwdPlan p{};
    p.tc = dtype == E2EGREC_BF16 && a.head_dim <= 128;
    const int64_t max_q = s.max_q ? std::min(s.max_q, a.q_rows) : a.q_rows, max_k = s.max_k ? std::min(s.max_k, a.k_rows) : a.k_rows;
    if (p.tc) {
        const int64_t most = (kMaxRows - 1) / std::max<int64_t>(a.n_seq * a.kv_heads, 1);
        p.q_tiles = std::max<int64_t>(1, std::min(ceil_div(max_q * a.group, 128), most));
        p.k_tiles = std::max<int64_t>(1, std::min(ceil_div(max_k, 128), most));
        p.dot_bytes = align_up((size_t)a.q_rows * a.kv_heads * a.group * sizeof(float), 256);
    }
    return p;
}

// Arguments that a size query has too; fills the sizes of `a`.
int32_t check_shape(const e2egrec_mat *Q, const e2egrec_mat *K, const e2egrec_sequences *seqs, int32_t n_heads, int32_t n_kv_heads,
                    float scale, AttnArgs &a)
{
    if (!Q || !K || !seqs) return E2EGREC_ERR_NULL;
    if (Q->dtype != E2EGREC_F32 && Q->dtype != E2EGREC_BF16) return E2EGREC_ERR_DTYPE;
    if (n_kv_heads < 1 || n_heads < n_kv_heads || n_heads % n_kv_heads || Q->dim < 1 || Q->dim % n_heads) return E2EGREC_ERR_ARG;
    if (Q->rows < 0 || K->rows < 0 || Q->rows >= kMaxRows || K->rows >= kMaxRows) return E2EGREC_ERR_ARG;
    if (seqs->n_seq < 0 || seqs->n_seq > (kMaxRows - 1) / n_kv_heads || seqs->max_q < 0 || seqs->max_k < 0) return E2EGREC_ERR_ARG;
    if (!(scale > 0.f) || !(scale <= 3.0e38f)) return E2EGREC_ERR_ARG;
    if (Q->dim / n_heads > kMaxAttnDim) return E2EGREC_ERR_UNSUPPORTED;
    a.n_seq = seqs->n_seq;
    a.q_ptr = seqs->q_ptr;
    a.k_ptr = seqs->k_ptr;
    a.mask = seqs->k_mask;
    a.q_rows = Q->rows;
    a.k_rows = K->rows;
    a.kv_heads = n_kv_heads;
    a.group = n_heads / n_kv_heads;
    a.head_dim = Q->dim / n_heads;
    a.scale = scale;
    return E2EGREC_OK;
}

}  // namespace
}  // namespace e2egrec

using namespace e2egrec;

extern "C" int32_t e2egrec_cross_attention_forward(const e2egrec_mat *Q, const e2egrec_mat *K, const e2egrec_mat *V,
                                                   const e2egrec_sequences *seqs, int32_t n_heads, int32_t n_kv_heads, float scale,
                                                   const e2egrec_mat *out, float *lse, int32_t *status, void *ws, size_t *ws_bytes,
                                                   void *stream)
{
    if (!ws_bytes) return E2EGREC_ERR_NULL;
    AttnArgs a{};
    int32_t rc = check_shape(Q, K, seqs, n_heads, n_kv_heads, scale, a);
    if (rc != E2EGREC_OK) return rc;
    const FwdPlan plan = plan_forward(a, *seqs, Q->dtype);
    const size_t need = 256 + plan.o_bytes + plan.ml_bytes;
    if (!ws) { *ws_bytes = need; return E2EGREC_OK; }
    if (*ws_bytes < need) { *ws_bytes = need; return E2EGREC_ERR_WORKSPACE; }
    if (reinterpret_cast<uintptr_t>(ws) % 256) return E2EGREC_ERR_ALIGN;
    rc = check_heads(Q, n_heads, a.head_dim, Q->dtype, a.q_rows);
    if (rc == E2EGREC_OK) rc = check_heads(K, n_kv_heads, a.head_dim, Q->dtype, a.k_rows);
    if (rc == E2EGREC_OK) rc = check_heads(V, n_kv_heads, a.head_dim, Q->dtype, a.k_rows);
    if (rc == E2EGREC_OK) rc = check_heads(out, n_heads, a.head_dim, Q->dtype, a.q_rows);
    if (rc != E2EGREC_OK) return rc;
    if (a.n_seq && (!a.q_ptr || !a.k_ptr)) return E2EGREC_ERR_NULL;
    if (a.n_seq == 0 || a.q_rows == 0) return E2EGREC_OK;
    a.q = Q->data; a.ldq = Q->ld;
    a.k = K->data; a.ldk = K->ld;
    a.v = V->data; a.ldv = V->ld;
    a.out = out->data; a.ldo = out->ld;
    a.lse = lse;
    a.status = status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    float2 *part_ml = static_cast<float2 *>(ws);
    float *part_o = reinterpret_cast<float *>(static_cast<char *>(ws) + plan.ml_bytes);
    if (plan.tc) {
        if (!tc_attention_forward(a, plan.tiles, plan.splits, part_o, part_ml, st)) return check_launch("cross_attention_forward");
        if (plan.splits > 1) {
            note_launch();
            attn_join_kernel<__nv_bfloat16><<<row_grid(a.q_rows, n_heads), kRowThreads, 0, st>>>(a, plan.splits, part_o, part_ml);
        }
    } else if (Q->dtype == E2EGREC_F32) row_forward<float>(a, st);
    else row_forward<__nv_bfloat16>(a, st);
    return check_launch("cross_attention_forward");
}

extern "C" int32_t e2egrec_cross_attention_backward(const e2egrec_mat *dOut, const e2egrec_mat *Q, const e2egrec_mat *K,
                                                    const e2egrec_mat *V, const e2egrec_mat *out, const float *lse,
                                                    const e2egrec_sequences *seqs, int32_t n_heads, int32_t n_kv_heads, float scale,
                                                    const e2egrec_mat *dQ, const e2egrec_mat *dK, const e2egrec_mat *dV,
                                                    int32_t *status, void *ws, size_t *ws_bytes, void *stream)
{
    if (!ws_bytes) return E2EGREC_ERR_NULL;
    AttnArgs a{};
    int32_t rc = check_shape(Q, K, seqs, n_heads, n_kv_heads, scale, a);
    if (rc != E2EGREC_OK) return rc;
    const BwdPlan plan = plan_backward(a, *seqs, Q->dtype);
    const size_t need = 256 + plan.dot_bytes;
    if (!ws) { *ws_bytes = need; return E2EGREC_OK; }
    if (*ws_bytes < need) { *ws_bytes = need; return E2EGREC_ERR_WORKSPACE; }
    if (reinterpret_cast<uintptr_t>(ws) % 256) return E2EGREC_ERR_ALIGN;
    for (const e2egrec_mat *m : {Q, dOut, out, dQ}) {
        rc = check_heads(m, n_heads, a.head_dim, Q->dtype, a.q_rows);
        if (rc != E2EGREC_OK) return rc;
    }
    for (const e2egrec_mat *m : {K, V, dK, dV}) {
        rc = check_heads(m, n_kv_heads, a.head_dim, Q->dtype, a.k_rows);
        if (rc != E2EGREC_OK) return rc;
    }
    if (a.n_seq && (!a.q_ptr || !a.k_ptr)) return E2EGREC_ERR_NULL;
    if (a.q_rows && !lse) return E2EGREC_ERR_NULL;
    if (a.n_seq == 0 || (a.q_rows == 0 && a.k_rows == 0)) return E2EGREC_OK;
    a.q = Q->data; a.ldq = Q->ld;
    a.k = K->data; a.ldk = K->ld;
    a.v = V->data; a.ldv = V->ld;
    a.o = out->data; a.ldo = out->ld;
    a.dout = dOut->data; a.ldg = dOut->ld;
    a.dq = dQ->data; a.ldq2 = dQ->ld;
    a.dk = dK->data; a.ldk2 = dK->ld;
    a.dv = dV->data; a.ldv2 = dV->ld;
    a.lse = const_cast<float *>(lse);
    a.status = status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (plan.tc) {
        if (!tc_attention_backward(a, plan.q_tiles, plan.k_tiles, static_cast<float *>(ws), st)) return check_launch("cross_attention_backward");
    } else if (Q->dtype == E2EGREC_F32) row_backward<float>(a, st);
    else row_backward<__nv_bfloat16>(a, st);
    return check_launch("cross_attention_backward");
}
