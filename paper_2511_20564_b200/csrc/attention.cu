// Attention of ragged sequences of tokens to ragged sequences of states: argument checks, the choice of kernels, and the join of
// results that were formed over stretches of the keys.
#include <algorithm>
#include <cmath>

#include "attention.cuh"
#include "gemm_simt.cuh"

namespace e2egrec {
namespace {

constexpr int kRowThreads = 256;

// Results of stretches of the keys -> out, lse.  `warps` warps per (row, head) take every warps-th stretch, four elements per lane;
// their sums are added in order.  Every stretch's weight is formed by one lane, so the loads of a warp do not wait for one another
// (one warp per row and a loop over the stretches took 115 us for 55 stretches of 32 rows, this 5).
template <typename T>
__global__ void __launch_bounds__(kRowThreads)
attn_join_kernel(const __grid_constant__ AttnArgs a, int splits, int warps, const float *__restrict__ part_o, const float2 *__restrict__ part_ml)
{
    __shared__ float weight[kRowThreads / 32][kMaxSplits];
    __shared__ float4 sums[kRowThreads / 32][kMaxAttnDim / 4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, heads = a.kv_heads * a.group, wu = warp & (warps - 1);
    const int64_t unit = (int64_t)blockIdx.x * (kRowThreads / 32 / warps) + warp / warps, stride = a.q_rows * heads;
    const int64_t row = unit / heads;
    const int h = (int)(unit - row * heads);
    const bool on = row < a.q_rows && owner(a.q_ptr, a.n_seq, row) >= 0;
    float2 ml[kMaxSplits / 32];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxSplits / 32; ++i) {
        const int z = lane + 32 * i;
        ml[i] = on && z < splits ? part_ml[z * stride + unit] : make_float2(-INFINITY, 0.f);
        m = fmaxf(m, ml[i].x);
    }
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < kMaxSplits / 32; ++i) {
        const float w = ml[i].y == 0.f ? 0.f : ml[i].y * exp2f(ml[i].x - base);
        weight[warp][lane + 32 * i] = w;
        l += w;
    }
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
    __syncwarp();
    float4 t[kMaxAttnDim / 128];
#pragma unroll
    for (int c = 0; c < kMaxAttnDim / 128; ++c) t[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (on) {
#pragma unroll 4
        for (int z = wu; z < splits; z += warps) {
            const float w = weight[warp][z];
            const float4 *p = reinterpret_cast<const float4 *>(part_o + (z * stride + unit) * a.head_dim);
#pragma unroll
            for (int c = 0; c < kMaxAttnDim / 128; ++c)
                if (c * 128 + lane * 4 < a.head_dim) {
                    const float4 v = p[c * 32 + lane];
                    t[c].x += w * v.x; t[c].y += w * v.y; t[c].z += w * v.z; t[c].w += w * v.w;
                }
        }
    }
    if (warps > 1) {
#pragma unroll
        for (int c = 0; c < kMaxAttnDim / 128; ++c) sums[warp][c * 32 + lane] = t[c];
        __syncthreads();
        for (int w = 1; wu == 0 && w < warps; ++w)
#pragma unroll
            for (int c = 0; c < kMaxAttnDim / 128; ++c) {
                const float4 v = sums[warp + w][c * 32 + lane];
                t[c].x += v.x; t[c].y += v.y; t[c].z += v.z; t[c].w += v.w;
            }
    }
    if (!on || wu) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T *out = static_cast<T *>(a.out) + row * a.ldo + (int64_t)h * a.head_dim;
#pragma unroll
    for (int c = 0; c < kMaxAttnDim / 128; ++c) {
        const int e = c * 128 + lane * 4;
        if (e < a.head_dim) {
            out[e] = from_float<T>(t[c].x * inv);
            out[e + 1] = from_float<T>(t[c].y * inv);
            out[e + 2] = from_float<T>(t[c].z * inv);
            out[e + 3] = from_float<T>(t[c].w * inv);
        }
    }
    if (a.lse && lane == 0) a.lse[unit] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// dQ of stretches of the keys -> dQ: a block per (query, head), a thread per four elements and part of the stretches (a power of two of
// threads side by side over the elements), the parts added up in order.  fit: the sums of p k of every stretch and of dS follow
// (attention_few.cu).  One row of 4 x 24 000 keys, two heads of 128: 125 us with a thread going over all stretches, 60 us so.
template <typename T>
__global__ void __launch_bounds__(kRowThreads)
attn_join_dq_kernel(const __grid_constant__ AttnArgs a, int splits, int wide, bool fit, const float *__restrict__ part, float *__restrict__ dots)
{
    __shared__ float4 sums[2][kRowThreads];
    __shared__ float rests[kRowThreads];
    const int heads = a.kv_heads * a.group, units = a.head_dim / 4, at = threadIdx.x & (wide - 1), first = threadIdx.x / wide, parts = kRowThreads / wide;
    const int64_t cell = blockIdx.x, cells = a.q_rows * heads, row = cell / heads;
    if (owner(a.q_ptr, a.n_seq, row) < 0) return;
    const float4 *p = reinterpret_cast<const float4 *>(part) + cell * units + at;
    const float *rest = part + 2 * splits * cells * a.head_dim + cell;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f), m = t;
    float r = 0.f;
    if (at < units) {
#pragma unroll 4
        for (int z = first; z < splits; z += parts) {
            const float4 v = p[z * cells * units];
            t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
            if (fit) {
                const float4 w = p[(splits + z) * cells * units];
                m.x += w.x; m.y += w.y; m.z += w.z; m.w += w.w;
                r += rest[z * cells];
            }
        }
    }
    sums[0][threadIdx.x] = t;
    sums[1][threadIdx.x] = m;
    rests[threadIdx.x] = r;
    __syncthreads();
    if (first || at >= units) return;
    for (int i = 1; i < parts; ++i) {
        const float4 v = sums[0][i * wide + at], w = sums[1][i * wide + at];
        t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
        m.x += w.x; m.y += w.y; m.z += w.z; m.w += w.w;
        r += rests[i * wide + at];
    }
    if (fit && dots && at == 0) dots[cell] += r;
    T *out = static_cast<T *>(a.dq) + row * a.ldq2 + (cell - row * heads) * a.head_dim + at * 4;
    out[0] = from_float<T>(t.x - r * m.x);
    out[1] = from_float<T>(t.y - r * m.y);
    out[2] = from_float<T>(t.z - r * m.z);
    out[3] = from_float<T>(t.w - r * m.w);
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

constexpr int64_t kMaxTable = 1 << 16;         // entries of a table of biases
constexpr int64_t kMaxUnits = ((int64_t)1 << 31) - 1;
constexpr int64_t kMaxRows = ((int64_t)1 << 31) - (1 << 16);      // the kernels step some hundred rows beyond a sequence's end in 32 bits

// The kernels of a call.  A sequence's keys and rows stream (attention_few.cu) where a key head has up to two rows (fp32 three: 300 of
// 3 x 200, 88 us against 113; four in the backward pass), or where a sequence is so small that the set-up of a tile costs more than its
// products; bf16 heads of up to 128 go to the tensor cores otherwise (gradients with a bias to matrix products of a warp), fp32 ones to tiles of
// fp32 FMA, wider heads always stream.
enum class Path { few, tc, simt, mma };

struct Plan {
    Path path;
    FewPlan few;
    SimtPlan simt;
    MmaPlan mma;
    TablePlan table;
    bool one_tile;                        // tensor cores: a key head's rows fit one tile
    int64_t q_tiles, k_tiles;             // blocks of rows / tiles of keys per sequence and key head
    int splits;                           // stretches of the keys
    size_t part_bytes, ml_bytes, dot_bytes;
    bool table_fused;                     // the kernel of dQ forms them
    int64_t table_rows;                   // backward with a bias: rows of partial gradients of the table
    size_t table_bytes;
};

Plan make_plan(const AttnArgs &a, const e2egrec_sequences &s, int32_t dtype, bool backward)
{
    Plan p{};
    p.splits = 1;
    auto lengths = [&](int64_t hint, int64_t all) {
        Lengths l{hint ? std::min(hint, all) : all, ceil_div(all, std::max<int64_t>(a.n_seq, 1)), 0};
        l.mean = std::min(l.mean, l.longest);
        l.typical = hint ? l.longest : l.mean;
        return l;
    };
    const Lengths q = lengths(s.max_q, a.q_rows), k = lengths(s.max_k, a.k_rows);
    const int64_t rows = q.typical * a.group, units = std::max<int64_t>(a.n_seq * a.kv_heads, 1);
    const size_t cells = (size_t)a.q_rows * a.kv_heads * a.group;
    const int n_heads = a.kv_heads * a.group;
    const bool small = rows <= (backward ? 4 : dtype == E2EGREC_F32 ? 3 : 2) || rows * k.typical <= (dtype == E2EGREC_F32 ? 256 : backward ? 700 : 800);
    // (without rows on one side there is nothing to form a product of)
    p.path = small || a.head_dim > 128 || !a.q_rows || !a.k_rows ? Path::few : dtype == E2EGREC_F32 ? Path::simt : backward && a.bias.buckets ? Path::mma : Path::tc;
    // a table of biases that does not fit beside the tiles
    if (p.path == Path::mma) p.mma = mma_plan(a, q, k);
    if ((p.path == Path::simt && a.bias.buckets * a.group > kSimtTable) || (p.path == Path::tc && a.bias.buckets * n_heads > kTcTable) ||
        (p.path == Path::mma && !p.mma.fits))
        p.path = Path::few;
    if (p.path == Path::tc) {
        p.one_tile = rows <= 128;
        p.q_tiles = blocks_per_unit(q, a.group, backward || p.one_tile ? 128 : 256, units);
        p.k_tiles = blocks_per_unit(k, 1, 128, units);
        const int64_t blocks = p.one_tile ? 296 : 148;
        if (!backward && units * p.q_tiles < blocks)
            p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({blocks / (units * p.q_tiles), k.longest / 512, kMaxSplits}));
    } else if (p.path == Path::simt) {
        p.simt = simt_plan(a, q, k);
        p.splits = p.simt.splits;
    } else if (p.path == Path::few) {
        p.few = few_plan(a, q, k, (int)dtype_size(dtype), backward);
        p.splits = p.few.splits;
    }
    if (backward && !(p.path == Path::few && p.few.both)) p.dot_bytes = align_up(cells * sizeof(float), 256) * (p.path == Path::mma ? 2 : 1);
    if (p.splits > 1) {
        const bool fit = backward && p.path == Path::few && p.few.fit;
        p.part_bytes = align_up(p.splits * cells * (fit ? 2 * a.head_dim + 1 : a.head_dim) * sizeof(float), 256);
        if (!backward) p.ml_bytes = align_up(p.splits * cells * sizeof(float2), 256);
    }
    if (backward && a.bias.buckets) {
        p.table = few_table_plan(a, k, dtype);
        const int64_t slices = p.table.seq_slices * p.table.row_slices * p.table.key_slices;
        p.table_fused = p.path == Path::mma ? p.mma.table : p.path == Path::simt ? simt_forms_table(a, p.simt) : p.few.both;
        p.table_rows = !p.table_fused ? slices
                                      : p.path == Path::few ? p.few.blocks : a.n_seq * (p.path == Path::mma ? p.mma.q_tiles : p.simt.q_tiles * p.simt.splits);
        p.table_bytes = align_up((size_t)p.table_rows * a.bias.buckets * a.kv_heads * a.group * sizeof(float), 256);
    }
    return p;
}

// A kernel could not be given its shared memory, or the device is not one of the first 64
int32_t launch_refused(const char *what)
{
    const int32_t rc = check_launch(what);
    if (rc == E2EGREC_OK) set_last_error(what);
    return E2EGREC_ERR_CUDA;
}

// Arguments that a size query has too; fills the sizes of `a`.
int32_t check_shape(const e2egrec_mat *Q, const e2egrec_mat *K, const e2egrec_sequences *seqs, int32_t n_heads, int32_t n_kv_heads,
                    float scale, AttnArgs &a)
{
    if (!Q || !K || !seqs) return E2EGREC_ERR_NULL;
    if (Q->dtype != E2EGREC_F32 && Q->dtype != E2EGREC_BF16) return E2EGREC_ERR_DTYPE;
    if (n_kv_heads < 1 || n_heads < n_kv_heads || n_heads % n_kv_heads || Q->dim < 1 || Q->dim % n_heads) return E2EGREC_ERR_ARG;
    if (Q->rows < 0 || K->rows < 0 || Q->rows > kMaxRows || K->rows > kMaxRows) return E2EGREC_ERR_ARG;
    if (seqs->n_seq < 0 || seqs->n_seq > kMaxUnits / n_kv_heads || seqs->max_q < 0 || seqs->max_k < 0) return E2EGREC_ERR_ARG;
    if (!(scale > 0.f) || !(scale <= 1.0e38f)) return E2EGREC_ERR_ARG;
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

// A bias, or none
int32_t check_bias(const e2egrec_relative_bias *b, AttnArgs &a)
{
    if (!b) return E2EGREC_OK;
    if (b->n_buckets < 1) return E2EGREC_ERR_ARG;
    if (b->n_buckets > kMaxBuckets || (int64_t)b->n_buckets * a.kv_heads * a.group > kMaxTable) return E2EGREC_ERR_UNSUPPORTED;
    for (const void *p : {(const void *)b->table, (const void *)b->edges, (const void *)b->pos_q, (const void *)b->pos_k})
        if (reinterpret_cast<uintptr_t>(p) % 4) return E2EGREC_ERR_ALIGN;
    a.bias.table = b->table;
    a.bias.edges = b->edges;
    a.bias.pos_q = b->pos_q;
    a.bias.pos_k = b->pos_k;
    a.bias.buckets = b->n_buckets;
    a.bias.top = 0;
    for (int s = 1; s < b->n_buckets; s *= 2) a.bias.top = s;
    return E2EGREC_OK;
}
// The same where work is enqueued: its pointers are there
bool bias_missing(const e2egrec_relative_bias *b) { return b && (!b->table || (b->n_buckets > 1 && !b->edges)); }

__global__ void zero_table_kernel(float *t, int n)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) t[i] = 0.f;
}

}  // namespace

void join_dq(const AttnArgs &a, int splits, int32_t dtype, bool fit, const float *part_dq, float *dots, cudaStream_t st)
{
    note_launch();
    const unsigned grid = (unsigned)(a.q_rows * a.kv_heads * a.group);
    int wide = 1;
    while (wide * 4 < a.head_dim) wide *= 2;
    if (dtype == E2EGREC_F32) attn_join_dq_kernel<float><<<grid, kRowThreads, 0, st>>>(a, splits, wide, fit, part_dq, dots);
    else attn_join_dq_kernel<__nv_bfloat16><<<grid, kRowThreads, 0, st>>>(a, splits, wide, fit, part_dq, dots);
}

}  // namespace e2egrec

using namespace e2egrec;

static int32_t attention_forward(const e2egrec_mat *Q, const e2egrec_mat *K, const e2egrec_mat *V, const e2egrec_sequences *seqs,
                                 const e2egrec_relative_bias *bias, int32_t n_heads, int32_t n_kv_heads, float scale, const e2egrec_mat *out,
                                 float *lse, int32_t *status, void *ws, size_t *ws_bytes, void *stream)
{
    const char *what = bias ? "biased_attention_forward" : "cross_attention_forward";
    if (!ws_bytes) return E2EGREC_ERR_NULL;
    AttnArgs a{};
    int32_t rc = check_shape(Q, K, seqs, n_heads, n_kv_heads, scale, a);
    if (rc == E2EGREC_OK) rc = check_bias(bias, a);
    if (rc != E2EGREC_OK) return rc;
    const Plan plan = make_plan(a, *seqs, Q->dtype, false);
    const size_t need = 256 + plan.part_bytes + plan.ml_bytes;
    if (!ws) { *ws_bytes = need; return E2EGREC_OK; }
    if (*ws_bytes < need) { *ws_bytes = need; return E2EGREC_ERR_WORKSPACE; }
    if (reinterpret_cast<uintptr_t>(ws) % 256) return E2EGREC_ERR_ALIGN;
    rc = check_heads(Q, n_heads, a.head_dim, Q->dtype, a.q_rows);
    if (rc == E2EGREC_OK) rc = check_heads(K, n_kv_heads, a.head_dim, Q->dtype, a.k_rows);
    if (rc == E2EGREC_OK) rc = check_heads(V, n_kv_heads, a.head_dim, Q->dtype, a.k_rows);
    if (rc == E2EGREC_OK) rc = check_heads(out, n_heads, a.head_dim, Q->dtype, a.q_rows);
    if (rc != E2EGREC_OK) return rc;
    if ((a.n_seq && (!a.q_ptr || !a.k_ptr)) || bias_missing(bias)) return E2EGREC_ERR_NULL;
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
    bool ok = true;
    if (plan.path == Path::tc) ok = tc_attention_forward(a, plan.q_tiles, plan.splits, plan.one_tile, part_o, part_ml, st);
    else if (plan.path == Path::simt) ok = simt_attention_forward(a, plan.simt, part_o, part_ml, st);
    else ok = few_attention_forward(a, plan.few, Q->dtype, part_o, part_ml, st);
    if (!ok) return launch_refused(what);
    if (plan.splits > 1) {
        note_launch();
        const int warps = plan.splits > 8 ? kRowThreads / 32 : 1;
        const unsigned grid = (unsigned)ceil_div(a.q_rows * n_heads, kRowThreads / 32 / warps);
        if (Q->dtype == E2EGREC_F32) attn_join_kernel<float><<<grid, kRowThreads, 0, st>>>(a, plan.splits, warps, part_o, part_ml);
        else attn_join_kernel<__nv_bfloat16><<<grid, kRowThreads, 0, st>>>(a, plan.splits, warps, part_o, part_ml);
    }
    return check_launch(what);
}

static int32_t attention_backward(const e2egrec_mat *dOut, const e2egrec_mat *Q, const e2egrec_mat *K, const e2egrec_mat *V,
                                  const e2egrec_mat *out, const float *lse, const e2egrec_sequences *seqs, const e2egrec_relative_bias *bias,
                                  int32_t n_heads, int32_t n_kv_heads, float scale, const e2egrec_mat *dQ, const e2egrec_mat *dK,
                                  const e2egrec_mat *dV, float *dtable, int32_t *status, void *ws, size_t *ws_bytes, void *stream)
{
    const char *what = bias ? "biased_attention_backward" : "cross_attention_backward";
    if (!ws_bytes) return E2EGREC_ERR_NULL;
    AttnArgs a{};
    int32_t rc = check_shape(Q, K, seqs, n_heads, n_kv_heads, scale, a);
    if (rc == E2EGREC_OK) rc = check_bias(bias, a);
    if (rc != E2EGREC_OK) return rc;
    const Plan plan = make_plan(a, *seqs, Q->dtype, true);
    // (a size query does not say whether the table's gradient is wanted)
    const size_t need = 256 + plan.part_bytes + plan.dot_bytes + (!ws || dtable ? plan.table_bytes : 0);
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
    if ((a.n_seq && (!a.q_ptr || !a.k_ptr)) || bias_missing(bias)) return E2EGREC_ERR_NULL;
    if (a.q_rows && !lse) return E2EGREC_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(dtable) % 4) return E2EGREC_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int table_size = a.bias.buckets * n_heads;
    if (dtable && (a.n_seq == 0 || a.q_rows == 0)) {
        note_launch();
        zero_table_kernel<<<(unsigned)ceil_div(table_size, 256), 256, 0, st>>>(dtable, table_size);
        rc = check_launch(what);
        if (rc != E2EGREC_OK) return rc;
        dtable = nullptr;
    }
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
    float *table_part = reinterpret_cast<float *>(static_cast<char *>(ws) + plan.dot_bytes + plan.part_bytes);
    float *dots = static_cast<float *>(ws), *part_dq = reinterpret_cast<float *>(static_cast<char *>(ws) + plan.dot_bytes);
    bool ok = true;
    if (plan.path == Path::tc) {
        ok = tc_attention_backward(a, plan.q_tiles, plan.k_tiles, dots, st);
    } else if (plan.path == Path::mma) {
        ok = mma_attention_backward(a, plan.mma, dots, dots + plan.dot_bytes / 2 / sizeof(float), plan.table_fused && dtable ? table_part : nullptr, st);
    } else if (plan.path == Path::simt) {
        ok = simt_attention_backward(a, plan.simt, part_dq, dots, plan.table_fused && dtable ? table_part : nullptr, st);
        if (ok && plan.splits > 1 && a.q_rows) join_dq(a, plan.splits, Q->dtype, false, part_dq, nullptr, st);
    } else {
        ok = few_attention_backward(a, plan.few, Q->dtype, part_dq, dots, dtable ? table_part : nullptr, st);
    }
    if (ok && dtable) {
        if (!plan.table_fused) ok = few_attention_table(a, plan.table, Q->dtype, dots, table_part, st);
        if (ok) launch_colsum<float>(table_part, table_size, nullptr, nullptr, plan.table_rows, table_size, 0, dtable, st);
    }
    if (!ok) return launch_refused(what);
    return check_launch(what);
}

extern "C" int32_t e2egrec_cross_attention_forward(const e2egrec_mat *Q, const e2egrec_mat *K, const e2egrec_mat *V,
                                                   const e2egrec_sequences *seqs, int32_t n_heads, int32_t n_kv_heads, float scale,
                                                   const e2egrec_mat *out, float *lse, int32_t *status, void *ws, size_t *ws_bytes,
                                                   void *stream)
{
    return attention_forward(Q, K, V, seqs, nullptr, n_heads, n_kv_heads, scale, out, lse, status, ws, ws_bytes, stream);
}

extern "C" int32_t e2egrec_cross_attention_backward(const e2egrec_mat *dOut, const e2egrec_mat *Q, const e2egrec_mat *K,
                                                    const e2egrec_mat *V, const e2egrec_mat *out, const float *lse,
                                                    const e2egrec_sequences *seqs, int32_t n_heads, int32_t n_kv_heads, float scale,
                                                    const e2egrec_mat *dQ, const e2egrec_mat *dK, const e2egrec_mat *dV,
                                                    int32_t *status, void *ws, size_t *ws_bytes, void *stream)
{
    return attention_backward(dOut, Q, K, V, out, lse, seqs, nullptr, n_heads, n_kv_heads, scale, dQ, dK, dV, nullptr, status, ws, ws_bytes,
                              stream);
}

extern "C" int32_t e2egrec_biased_attention_forward(const e2egrec_mat *Q, const e2egrec_mat *K, const e2egrec_mat *V,
                                                    const e2egrec_sequences *seqs, const e2egrec_relative_bias *bias, int32_t n_heads,
                                                    int32_t n_kv_heads, float scale, const e2egrec_mat *out, float *lse, int32_t *status,
                                                    void *ws, size_t *ws_bytes, void *stream)
{
    if (!bias) return E2EGREC_ERR_NULL;
    return attention_forward(Q, K, V, seqs, bias, n_heads, n_kv_heads, scale, out, lse, status, ws, ws_bytes, stream);
}

extern "C" int32_t e2egrec_biased_attention_backward(const e2egrec_mat *dOut, const e2egrec_mat *Q, const e2egrec_mat *K,
                                                     const e2egrec_mat *V, const e2egrec_mat *out, const float *lse,
                                                     const e2egrec_sequences *seqs, const e2egrec_relative_bias *bias, int32_t n_heads,
                                                     int32_t n_kv_heads, float scale, const e2egrec_mat *dQ, const e2egrec_mat *dK,
                                                     const e2egrec_mat *dV, float *dtable, int32_t *status, void *ws, size_t *ws_bytes,
                                                     void *stream)
{
    if (!bias) return E2EGREC_ERR_NULL;
    return attention_backward(dOut, Q, K, V, out, lse, seqs, bias, n_heads, n_kv_heads, scale, dQ, dK, dV, dtable, status, ws, ws_bytes, stream);
}

// Smallest distances of the buckets 1 .. n - 1 of one side: their numbers up to n / 2, from there on half (far / half)^((i - half) / (n - half)),
// rounded up, at least one apart.
extern "C" int32_t e2egrec_relative_edges(int32_t buckets, int64_t far, int32_t both, int32_t *edges)
{
    if (buckets < 1 || far < 1 || far > (1 << 30)) return E2EGREC_ERR_ARG;
    if (buckets > (both ? (kMaxBuckets + 1) / 2 : kMaxBuckets)) return E2EGREC_ERR_UNSUPPORTED;
    if (!edges) return buckets == 1 ? E2EGREC_OK : E2EGREC_ERR_NULL;
    const int half = std::max(buckets / 2, 1);
    int64_t last = 0;
    for (int i = 1; i < buckets; ++i) {
        int64_t t = i;
        if (i >= half) {
            const double x = half * std::pow((double)std::max<int64_t>(far, half + 1) / half, (double)(i - half) / std::max(buckets - half, 1));
            const double whole = std::nearbyint(x);
            t = (int64_t)(std::fabs(x - whole) < 1e-9 * x ? whole : std::ceil(x));       // a whole number that pow missed by a rounding
        }
        last = std::max(t, last + 1);
        edges[buckets - 1 - i] = (int32_t)(1 - last);
        if (both) edges[buckets - 2 + i] = (int32_t)last;
    }
    return E2EGREC_OK;
}
