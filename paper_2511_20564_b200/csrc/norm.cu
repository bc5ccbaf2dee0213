// Dropout, and layer norm of x or of residual + dropout(x), with their gradients.
//
//   z = residual + dropout(x),  m = mean(z),  s = 1 / sqrt(mean((z - m)^2) + eps),  n = (z - m) s,  y = gain n + shift
//   gradient, with g = dy gain:  dz = s (g - mean(g) - n mean(g n)) + dz_in,  dresidual = dz,  dx = dropout(dz),
//                                dgain = sum dy n,  dshift = sum dy  over the rows
// The backward pass forms z and the mask of the dropout anew from x and residual: nothing but m and s is kept, and z is as exact as in the
// forward pass where a stored one would have been rounded.
//
// What bounds these kernels is memory: every matrix is read or written once.  A row stays in the registers of its threads (a part of a warp,
// a warp, or up to eight), the variance is the mean of (z - m)^2 over them, not a difference of sums.  Gains' gradients are added up in the
// registers of a block that goes over many rows, then block by block by a second kernel, in a fixed order.
#include <algorithm>

#include "dropout.cuh"

namespace e2egrec {
namespace {

constexpr int kNormThreads = 256, kNormWarps = kNormThreads / 32;
constexpr int kMaxNormDim = 8192;
constexpr int kGradBlocks = 148 * 4;                 // blocks that sum up the gains' gradients, at most
constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1;

struct NormArgs {
    const void *x, *r, *dy, *dz;                     // r, dz may be null
    void *y, *z, *dx, *dr;                           // z, dr may be null
    int64_t ldx, ldr, lddy, lddz, ldy, ldz, lddx, lddr;
    const float *gain, *shift;                       // null: 1, 0
    float2 *stats;                                   // (m, s) of every row; forward: may be null
    float *part;                                     // backward: [blocks x 2 x dim], null where no gains are wanted
    int64_t rows;
    int32_t dim, chunks, threads;                    // threads of a row: a power of two, 1 .. 256
    float eps, inv_dim;
    DropArgs drop;
};

// Sum over the threads of a row, N values at once.  Rows of more than a warp meet in shared memory: `buf` is used alternately, so that one
// barrier a sum is enough.
template <int N> __device__ inline void row_sums(float (&v)[N], int threads, float (*buf)[kNormWarps])
{
    for (int o = min(threads, 32) >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
    if (threads > 32) {
        const int warp = threadIdx.x >> 5, warps = threads >> 5, first = warp & ~(warps - 1);
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) buf[i][warp] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
            for (int w = 0; w < warps; ++w) v[i] += buf[i][first + w];
        }
    }
}

template <int E> __device__ inline void load_gains(const float *p, int chunk, float none, float (&v)[E])
{
#pragma unroll
    for (int e = 0; e < E; e += 4) {
        const float4 q = p ? __ldg(reinterpret_cast<const float4 *>(p + chunk * E + e)) : make_float4(none, none, none, none);
        v[e] = q.x; v[e + 1] = q.y; v[e + 2] = q.z; v[e + 3] = q.w;
    }
}

// U chunks of 16 bytes per thread, R rows at a time
template <typename T, int U, int R, bool kDrop>
__global__ void __launch_bounds__(kNormThreads)
norm_fwd_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int E = Chunk<T>::kElems;
    __shared__ float buf[2][R][kNormWarps];
    const int at = threadIdx.x & (a.threads - 1), group = threadIdx.x / a.threads, groups = kNormThreads / a.threads;
    const int64_t row0 = (int64_t)blockIdx.x * groups * R + group;
    uint4 raw[R][U], res[R][U];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row0 + i * groups;
            const int c = at + u * a.threads;
            const bool on = row < a.rows && c < a.chunks;
            raw[i][u] = on ? Chunk<T>::load_raw(static_cast<const T *>(a.x) + row * a.ldx + c * E) : make_uint4(0, 0, 0, 0);
            res[i][u] = on && a.r ? Chunk<T>::load_raw(static_cast<const T *>(a.r) + row * a.ldr + c * E) : make_uint4(0, 0, 0, 0);
        }
    const uint32_t step = kDrop ? drop_step(a.drop) : 0u;
    float z[R][U][E], sum[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t row = row0 + i * groups;
        sum[i] = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = at + u * a.threads;
            float v[E];
            Chunk<T>::unpack(raw[i][u], z[i][u]);
            if constexpr (kDrop) drop_apply<E>(a.drop, drop_bits<E>(a.drop, drop_words(a.drop, step, (uint32_t)row, drop_unit<T>(c)), c), z[i][u]);
            Chunk<T>::unpack(res[i][u], v);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                z[i][u][e] += v[e];
                sum[i] += z[i][u][e];
            }
        }
    }
    row_sums<R>(sum, a.threads, buf[0]);
    float sq[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        sum[i] *= a.inv_dim;
        sq[i] = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (at + u * a.threads < a.chunks)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float d = z[i][u][e] - sum[i];
                    sq[i] = fmaf(d, d, sq[i]);
                }
    }
    row_sums<R>(sq, a.threads, buf[1]);
#pragma unroll
    for (int i = 0; i < R; ++i) sq[i] = rsqrtf(fmaf(sq[i], a.inv_dim, a.eps));
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = at + u * a.threads;
        if (c >= a.chunks) continue;
        float gain[E], shift[E];
        load_gains<E>(a.gain, c, 1.f, gain);
        load_gains<E>(a.shift, c, 0.f, shift);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = row0 + i * groups;
            if (row >= a.rows) continue;
            if (a.z) Chunk<T>::store(static_cast<T *>(a.z) + row * a.ldz + c * E, z[i][u]);
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf((z[i][u][e] - sum[i]) * sq[i], gain[e], shift[e]);
            Chunk<T>::store(static_cast<T *>(a.y) + row * a.ldy + c * E, y);
        }
    }
    if (a.stats && at == 0)
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (row0 + i * groups < a.rows) a.stats[row0 + i * groups] = make_float2(sum[i], sq[i]);
}

template <typename T, int U, int R, bool kDrop>
__global__ void __launch_bounds__(kNormThreads)
norm_bwd_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int E = Chunk<T>::kElems;
    extern __shared__ float join[];                  // [U * E][kNormThreads], gains only
    __shared__ float buf[2][2 * R][kNormWarps];
    const int at = threadIdx.x & (a.threads - 1), group = threadIdx.x / a.threads, groups = kNormThreads / a.threads;
    const uint32_t step = kDrop ? drop_step(a.drop) : 0u;
    float dgain[U][E], dshift[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) dgain[u][e] = dshift[u][e] = 0.f;
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * groups * R; first < a.rows; first += (int64_t)gridDim.x * groups * R, turn ^= 1) {
        uint4 raw[R][U], res[R][U], up[R][U];
        float2 st[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = first + group + i * groups;
            st[i] = row < a.rows ? __ldg(a.stats + row) : make_float2(0.f, 0.f);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = at + u * a.threads;
                const bool on = row < a.rows && c < a.chunks;
                raw[i][u] = on ? Chunk<T>::load_raw(static_cast<const T *>(a.x) + row * a.ldx + c * E) : make_uint4(0, 0, 0, 0);
                res[i][u] = on && a.r ? Chunk<T>::load_raw(static_cast<const T *>(a.r) + row * a.ldr + c * E) : make_uint4(0, 0, 0, 0);
                up[i][u] = on ? Chunk<T>::load_raw(static_cast<const T *>(a.dy) + row * a.lddy + c * E) : make_uint4(0, 0, 0, 0);
            }
        }
        float n[R][U][E], g[R][U][E], sums[2 * R];
        uint32_t kept[R][U];                         // a bit per element
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = first + group + i * groups;
            sums[2 * i] = sums[2 * i + 1] = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = at + u * a.threads;
                float v[E], gain[E];
                Chunk<T>::unpack(raw[i][u], n[i][u]);
                kept[i][u] = 0;
                if constexpr (kDrop) {
                    kept[i][u] = drop_bits<E>(a.drop, drop_words(a.drop, step, (uint32_t)row, drop_unit<T>(c)), c);
                    drop_apply<E>(a.drop, kept[i][u], n[i][u]);
                }
                Chunk<T>::unpack(res[i][u], v);
                Chunk<T>::unpack(up[i][u], g[i][u]);
                if (c < a.chunks) load_gains<E>(a.gain, c, 1.f, gain);
                else
#pragma unroll
                    for (int e = 0; e < E; ++e) gain[e] = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    n[i][u][e] = (n[i][u][e] + v[e] - st[i].x) * st[i].y;
                    dgain[u][e] = fmaf(g[i][u][e], n[i][u][e], dgain[u][e]);
                    dshift[u][e] += g[i][u][e];
                    g[i][u][e] *= gain[e];
                    sums[2 * i] += g[i][u][e];
                    sums[2 * i + 1] = fmaf(g[i][u][e], n[i][u][e], sums[2 * i + 1]);
                }
            }
        }
        row_sums<2 * R>(sums, a.threads, buf[turn]);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = first + group + i * groups;
            if (row >= a.rows) continue;
            const float c1 = sums[2 * i] * a.inv_dim, c2 = sums[2 * i + 1] * a.inv_dim;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = at + u * a.threads;
                if (c >= a.chunks) continue;
                float d[E];
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = st[i].y * (g[i][u][e] - c1 - n[i][u][e] * c2);
                if (a.dz) {
                    float v[E];
                    Chunk<T>::load(static_cast<const T *>(a.dz) + row * a.lddz + c * E, v);
#pragma unroll
                    for (int e = 0; e < E; ++e) d[e] += v[e];
                }
                if (a.dr) Chunk<T>::store(static_cast<T *>(a.dr) + row * a.lddr + c * E, d);
                if constexpr (kDrop) drop_apply<E>(a.drop, kept[i][u], d);
                Chunk<T>::store(static_cast<T *>(a.dx) + row * a.lddx + c * E, d);
            }
        }
    }
    if (!a.part) return;
    // the groups of the block, in order: first the gains, then the shifts
    float *part = a.part + (int64_t)blockIdx.x * 2 * a.dim;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) join[(u * E + e) * kNormThreads + threadIdx.x] = side ? dshift[u][e] : dgain[u][e];
        __syncthreads();
        for (int k = threadIdx.x; k < U * E * a.threads; k += kNormThreads) {
            const int v = k / a.threads, t = k & (a.threads - 1), c = t + v / E * a.threads;
            if (c >= a.chunks) continue;
            float s = 0.f;
            for (int q = 0; q < groups; ++q) s += join[v * kNormThreads + q * a.threads + t];
            part[side * a.dim + c * E + v % E] = s;
        }
    }
}

// Sums of the blocks' rows of partial gains: 32 columns per block, 32 lanes over the blocks' rows each
__global__ void __launch_bounds__(1024)
norm_gains_kernel(const float *__restrict__ part, int blocks, int dim, float *__restrict__ dgain, float *__restrict__ dshift)
{
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (col < 2 * dim)
#pragma unroll 4
        for (int b = y; b < blocks; b += 32) s += part[(int64_t)b * 2 * dim + col];
    sums[y][lane] = s;
    __syncthreads();
    if (y) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][lane];
    if (col < dim) {
        if (dgain) dgain[col] = s;
    } else if (col < 2 * dim && dshift) {
        dshift[col - dim] = s;
    }
}

struct DropoutArgs {
    const void *x, *r;
    void *y;
    int64_t ldx, ldr, ldy, total;                    // total: units of 8 elements
    int32_t dim;
    uint32_t units;                                  // of a row
    DropArgs drop;
};

template <typename T>
__global__ void __launch_bounds__(kNormThreads)
dropout_kernel(const __grid_constant__ DropoutArgs a)
{
    constexpr int E = Chunk<T>::kElems, kChunks = 8 / E;
    const uint32_t step = drop_step(a.drop);
    for (int64_t i = (int64_t)blockIdx.x * kNormThreads + threadIdx.x; i < a.total; i += (int64_t)gridDim.x * kNormThreads) {
        const int64_t row = i >> 32 ? i / a.units : (int64_t)((uint32_t)i / a.units);
        const uint32_t unit = (uint32_t)(i - row * a.units);
        const uint4 w = drop_words(a.drop, step, (uint32_t)row, unit);
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            const int64_t c = (int64_t)unit * 8 + k * E;
            if (c >= a.dim) continue;
            float v[E];
            Chunk<T>::load(static_cast<const T *>(a.x) + row * a.ldx + c, v);
            if (a.drop.cut) drop_apply<E>(a.drop, drop_bits<E>(a.drop, w, k), v);
            if (a.r) {
                float q[E];
                Chunk<T>::load(static_cast<const T *>(a.r) + row * a.ldr + c, q);
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] += q[e];
            }
            Chunk<T>::store(static_cast<T *>(a.y) + row * a.ldy + c, v);
        }
    }
}

__global__ void zero_gains_kernel(float *dgain, float *dshift, int dim)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= dim) return;
    if (dgain) dgain[i] = 0.f;
    if (dshift) dshift[i] = 0.f;
}

// Shape, type and alignment of a matrix beside X
int32_t check_beside(const e2egrec_mat *m, const e2egrec_mat *X)
{
    if (!m || (!m->data && X->rows > 0)) return E2EGREC_ERR_NULL;
    if (m->dtype != E2EGREC_F32 && m->dtype != E2EGREC_BF16) return E2EGREC_ERR_DTYPE;
    if (m->dtype != X->dtype) return E2EGREC_ERR_DTYPE;
    if (m->rows != X->rows || m->dim != X->dim || m->ld < m->dim) return E2EGREC_ERR_ARG;
    const int64_t es = (int64_t)dtype_size(m->dtype);
    if (m->dim * es % 16 || m->ld * es % 16 || reinterpret_cast<uintptr_t>(m->data) % 16) return E2EGREC_ERR_ALIGN;
    return E2EGREC_OK;
}
// The sizes of X alone (a size query has no more)
int32_t check_sizes(const e2egrec_mat *X)
{
    if (!X) return E2EGREC_ERR_NULL;
    if (X->dtype != E2EGREC_F32 && X->dtype != E2EGREC_BF16) return E2EGREC_ERR_DTYPE;
    if (X->rows < 0 || X->rows > kMaxRows || X->dim < 1) return E2EGREC_ERR_ARG;
    return E2EGREC_OK;
}
bool misaligned(const float *p) { return reinterpret_cast<uintptr_t>(p) % 16; }

// Threads of a row, chunks per thread (a template argument) and rows at a time
struct NormShape {
    int threads, per;
};
NormShape norm_shape(const e2egrec_mat *X)
{
    const int es = (int)dtype_size(X->dtype), chunks = X->dim * es / 16, most = 32 / (16 / es);      // 32 values per thread at most
    NormShape s{1, 1};
    while (s.threads < 32 && s.threads < chunks) s.threads *= 2;
    while (s.threads * s.per < chunks && s.per < most) s.per *= 2;
    while (s.threads * s.per < chunks) s.threads *= 2;
    return s;
}

template <typename T, int U, int R, bool kDrop, bool kBack> void norm_launch(const NormArgs &a, cudaStream_t st, int blocks)
{
    note_launch();
    const int64_t per = (int64_t)kNormThreads / a.threads * R;
    if constexpr (kBack) {
        const size_t smem = a.part ? (size_t)U * Chunk<T>::kElems * kNormThreads * sizeof(float) : 0;
        norm_bwd_kernel<T, U, R, kDrop><<<blocks, kNormThreads, smem, st>>>(a);
    } else {
        norm_fwd_kernel<T, U, R, kDrop><<<(unsigned)ceil_div(a.rows, per), kNormThreads, 0, st>>>(a);
    }
}

template <typename T, bool kDrop, bool kBack> void norm_of(const NormArgs &a, int per, cudaStream_t st, int blocks)
{
    if (per == 1) norm_launch<T, 1, 2, kDrop, kBack>(a, st, blocks);
    else if (per == 2) norm_launch<T, 2, 2, kDrop, kBack>(a, st, blocks);
    else if (per == 4) norm_launch<T, 4, 1, kDrop, kBack>(a, st, blocks);
    else if constexpr (sizeof(T) == 4) norm_launch<T, 8, 1, kDrop, kBack>(a, st, blocks);
}
constexpr int rows_at_once(int per) { return per <= 2 ? 2 : 1; }

template <bool kBack> void norm_any(const NormArgs &a, int32_t dtype, int per, cudaStream_t st, int blocks = 0)
{
    if (dtype == E2EGREC_F32) a.drop.cut ? norm_of<float, true, kBack>(a, per, st, blocks) : norm_of<float, false, kBack>(a, per, st, blocks);
    else a.drop.cut ? norm_of<__nv_bfloat16, true, kBack>(a, per, st, blocks) : norm_of<__nv_bfloat16, false, kBack>(a, per, st, blocks);
}

// What both norm calls take; leaves the sizes in `a`
int32_t norm_args(const e2egrec_mat *X, const e2egrec_mat *residual, const e2egrec_dropout *drop, const float *gain, NormArgs &a)
{
    int32_t rc = check_beside(X, X);
    if (rc == E2EGREC_OK && residual) rc = check_beside(residual, X);
    if (rc == E2EGREC_OK) rc = drop_args(drop, a.drop);
    if (rc == E2EGREC_OK && misaligned(gain)) rc = E2EGREC_ERR_ALIGN;
    if (rc != E2EGREC_OK) return rc;
    a.x = X->data;
    a.ldx = X->ld;
    a.r = residual ? residual->data : nullptr;
    a.ldr = residual ? residual->ld : 0;
    a.gain = gain;
    a.rows = X->rows;
    a.dim = X->dim;
    a.chunks = X->dim * (int)dtype_size(X->dtype) / 16;
    a.inv_dim = 1.f / (float)X->dim;
    return E2EGREC_OK;
}

}  // namespace
}  // namespace e2egrec

using namespace e2egrec;

extern "C" int32_t e2egrec_dropout_apply(const e2egrec_mat *X, const e2egrec_mat *residual, const e2egrec_dropout *drop, const e2egrec_mat *Y,
                                         void *stream)
{
    int32_t rc = check_sizes(X);
    if (rc == E2EGREC_OK) rc = check_beside(X, X);
    if (rc == E2EGREC_OK && residual) rc = check_beside(residual, X);
    if (rc == E2EGREC_OK) rc = check_beside(Y, X);
    DropoutArgs a{};
    if (rc == E2EGREC_OK) rc = drop_args(drop, a.drop);
    if (rc != E2EGREC_OK || X->rows == 0) return rc;
    a.x = X->data;
    a.ldx = X->ld;
    a.r = residual ? residual->data : nullptr;
    a.ldr = residual ? residual->ld : 0;
    a.y = Y->data;
    a.ldy = Y->ld;
    a.dim = X->dim;
    a.units = (uint32_t)ceil_div(X->dim, 8);
    a.total = X->rows * a.units;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(a.total, kNormThreads), 148 * 8 * 16);
    note_launch();
    if (X->dtype == E2EGREC_F32) dropout_kernel<float><<<grid, kNormThreads, 0, st>>>(a);
    else dropout_kernel<__nv_bfloat16><<<grid, kNormThreads, 0, st>>>(a);
    return check_launch("dropout_apply");
}

extern "C" int32_t e2egrec_layer_norm_forward(const e2egrec_mat *X, const e2egrec_mat *residual, const e2egrec_dropout *drop, const float *gain,
                                              const float *shift, float eps, const e2egrec_mat *Y, const e2egrec_mat *Z, float *stats,
                                              void *stream)
{
    int32_t rc = check_sizes(X);
    if (rc != E2EGREC_OK) return rc;
    if (!(eps > 0.f)) return E2EGREC_ERR_ARG;
    if (X->dim > kMaxNormDim) return E2EGREC_ERR_UNSUPPORTED;
    NormArgs a{};
    rc = norm_args(X, residual, drop, gain, a);
    if (rc == E2EGREC_OK) rc = check_beside(Y, X);
    if (rc == E2EGREC_OK && Z) rc = check_beside(Z, X);
    if (rc == E2EGREC_OK && (misaligned(shift) || reinterpret_cast<uintptr_t>(stats) % 8)) rc = E2EGREC_ERR_ALIGN;
    if (rc != E2EGREC_OK || X->rows == 0) return rc;
    a.y = Y->data;
    a.ldy = Y->ld;
    a.z = Z ? Z->data : nullptr;
    a.ldz = Z ? Z->ld : 0;
    a.shift = shift;
    a.eps = eps;
    a.stats = reinterpret_cast<float2 *>(stats);
    const NormShape s = norm_shape(X);
    a.threads = s.threads;
    norm_any<false>(a, X->dtype, s.per, static_cast<cudaStream_t>(stream));
    return check_launch("layer_norm_forward");
}

extern "C" int32_t e2egrec_layer_norm_backward(const e2egrec_mat *dY, const e2egrec_mat *dZ, const e2egrec_mat *X, const e2egrec_mat *residual,
                                               const e2egrec_dropout *drop, const float *gain, const float *stats, const e2egrec_mat *dX,
                                               const e2egrec_mat *dR, float *dgain, float *dshift, void *ws, size_t *ws_bytes, void *stream)
{
    if (!ws_bytes) return E2EGREC_ERR_NULL;
    int32_t rc = check_sizes(X);
    if (rc != E2EGREC_OK) return rc;
    if (X->dim > kMaxNormDim) return E2EGREC_ERR_UNSUPPORTED;
    const NormShape s = norm_shape(X);
    const int64_t tile = (int64_t)(kNormThreads / s.threads) * rows_at_once(s.per);
    const int blocks = (int)std::min<int64_t>(ceil_div(X->rows, tile), kGradBlocks);
    const size_t need = 256 + align_up((size_t)blocks * 2 * X->dim * sizeof(float), 256);
    if (!ws) { *ws_bytes = need; return E2EGREC_OK; }
    if (*ws_bytes < need) { *ws_bytes = need; return E2EGREC_ERR_WORKSPACE; }
    if (reinterpret_cast<uintptr_t>(ws) % 256) return E2EGREC_ERR_ALIGN;
    NormArgs a{};
    rc = norm_args(X, residual, drop, gain, a);
    if (rc == E2EGREC_OK) rc = check_beside(dY, X);
    if (rc == E2EGREC_OK && dZ) rc = check_beside(dZ, X);
    if (rc == E2EGREC_OK) rc = check_beside(dX, X);
    if (rc == E2EGREC_OK && dR) rc = check_beside(dR, X);
    if (rc == E2EGREC_OK && X->rows && !stats) rc = E2EGREC_ERR_NULL;
    if (rc == E2EGREC_OK && reinterpret_cast<uintptr_t>(stats) % 8) rc = E2EGREC_ERR_ALIGN;
    if (rc != E2EGREC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (X->rows == 0) {
        if (!dgain && !dshift) return E2EGREC_OK;
        note_launch();
        zero_gains_kernel<<<(unsigned)ceil_div(X->dim, 256), 256, 0, st>>>(dgain, dshift, X->dim);
        return check_launch("layer_norm_backward");
    }
    a.dy = dY->data;
    a.lddy = dY->ld;
    a.dz = dZ ? dZ->data : nullptr;
    a.lddz = dZ ? dZ->ld : 0;
    a.dx = dX->data;
    a.lddx = dX->ld;
    a.dr = dR ? dR->data : nullptr;
    a.lddr = dR ? dR->ld : 0;
    a.stats = reinterpret_cast<float2 *>(const_cast<float *>(stats));
    a.part = dgain || dshift ? static_cast<float *>(ws) : nullptr;
    a.threads = s.threads;
    norm_any<true>(a, X->dtype, s.per, st, blocks);
    if (a.part) {
        note_launch();
        norm_gains_kernel<<<(unsigned)ceil_div(2 * X->dim, 32), 1024, 0, st>>>(a.part, blocks, X->dim, dgain, dshift);
    }
    return check_launch("layer_norm_backward");
}
