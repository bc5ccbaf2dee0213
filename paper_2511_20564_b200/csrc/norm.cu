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
constexpr int kGradBlocks = 148 * 2;                 // blocks that sum up the gains' gradients, at most
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

template <int N> __device__ inline void load_gains(const float *p, int chunk, float none, float2 (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float4 q = p ? __ldg(reinterpret_cast<const float4 *>(p + (chunk * N + i) * 2)) : make_float4(none, none, none, none);
        v[i] = make_float2(q.x, q.y);
        v[i + 1] = make_float2(q.z, q.w);
    }
}
__device__ inline float2 both(float x) { return make_float2(x, x); }

// U chunks of 16 bytes per thread; arithmetic on two elements at a time.  The kernel's own time, 131 072 x 256 bf16 with residual and dropout: 46 us,
// 4.4 TB/s; without dropout 39.5 us, 5.1 TB/s (the generator and the conversions are the difference); 32 768 x 1024, the sum stored as well: 50 us with
// dropout, 46 without, 5.4 and 5.8 TB/s.
template <typename T, int U, bool kDrop>
__global__ void __launch_bounds__(kNormThreads, U * Chunk<T>::kElems > 24 ? 3 : 4)
norm_fwd_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int E = Chunk<T>::kElems, P = E / 2;
    __shared__ float buf[2][1][kNormWarps];
    const int at = threadIdx.x & (a.threads - 1), group = threadIdx.x / a.threads, groups = kNormThreads / a.threads;
    const int64_t row = (int64_t)blockIdx.x * groups + group;
    const bool live = row < a.rows;
    uint4 raw[U], res[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = at + u * a.threads;
        const bool on = live && c < a.chunks;
        raw[u] = on ? Chunk<T>::load_raw(static_cast<const T *>(a.x) + row * a.ldx + c * E) : make_uint4(0, 0, 0, 0);
        res[u] = on && a.r ? Chunk<T>::load_raw(static_cast<const T *>(a.r) + row * a.ldr + c * E) : make_uint4(0, 0, 0, 0);
    }
    const uint32_t step = kDrop ? drop_step(a.drop) : 0u;
    PhiloxRow of_row;
    if constexpr (kDrop) of_row = drop_of_row(a.drop, (uint32_t)row);
    float2 z[U][P], s2 = both(0.f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = at + u * a.threads;
        float2 v[P];
        unpack_pairs(raw[u], z[u]);
        if constexpr (kDrop) {
            uint32_t h[P];
            drop_halves<E>(drop_words(a.drop, drop_of_unit(a.drop, step, drop_unit<T>(c)), of_row), c, h);
            drop_apply(a.drop, h, z[u]);
        }
        unpack_pairs(res[u], v);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            z[u][i] = __fadd2_rn(z[u][i], v[i]);
            s2 = __fadd2_rn(s2, z[u][i]);
        }
        if (a.z && live && c < a.chunks) store_pairs(static_cast<T *>(a.z) + row * a.ldz + c * E, z[u]);
    }
    float sum[1] = {s2.x + s2.y};
    row_sums<1>(sum, a.threads, buf[0]);
    const float mean = sum[0] * a.inv_dim;
    s2 = both(0.f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool on = at + u * a.threads < a.chunks;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            z[u][i] = __fadd2_rn(z[u][i], both(-mean));
            const float2 d = on ? z[u][i] : both(0.f);
            s2 = __ffma2_rn(d, d, s2);
        }
    }
    sum[0] = s2.x + s2.y;
    row_sums<1>(sum, a.threads, buf[1]);
    const float rstd = rsqrtf(fmaf(sum[0], a.inv_dim, a.eps));
    if (!live) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = at + u * a.threads;
        if (c >= a.chunks) continue;
        float2 gain[P], shift[P];
        load_gains(a.gain, c, 1.f, gain);
        load_gains(a.shift, c, 0.f, shift);
#pragma unroll
        for (int i = 0; i < P; ++i) z[u][i] = __ffma2_rn(__fmul2_rn(z[u][i], both(rstd)), gain[i], shift[i]);
        store_pairs(static_cast<T *>(a.y) + row * a.ldy + c * E, z[u]);
    }
    if (a.stats && at == 0) a.stats[row] = make_float2(mean, rstd);
}

// The gradient, rows in turn, 16 values per thread as the gains' sums take twice that.  The kernel's own time, 131 072 x 256 bf16 with residual and
// dropout: 68 us, 4.9 TB/s (53 without dropout); 32 768 x 1024 with the gradient of the sum 84 us, 4.8 TB/s (twice that with 250 registers and a block
// per SM, 32 values per thread).  Two blocks per SM at most go over the rows: four and more have more partial sums to write than they hide latency (call
// by call 77 -> 79 us, 20 011 x 320 fp32 30 -> 34 us).
constexpr int kBackValues = 16, kForwardValues = 32;
template <typename T, int U, bool kDrop>
__global__ void __launch_bounds__(kNormThreads, U * Chunk<T>::kElems > kBackValues ? 1 : 2)
norm_bwd_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int E = Chunk<T>::kElems, P = E / 2;
    extern __shared__ float join[];                  // [U * E][kNormThreads], gains only
    __shared__ float buf[2][2][kNormWarps];
    const int at = threadIdx.x & (a.threads - 1), group = threadIdx.x / a.threads, groups = kNormThreads / a.threads;
    const uint32_t step = kDrop ? drop_step(a.drop) : 0u;
    float2 dgain[U][P], dshift[U][P];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < P; ++i) dgain[u][i] = dshift[u][i] = both(0.f);
    PhiloxUnit of_unit[kDrop ? U : 1];
    if constexpr (kDrop)
#pragma unroll
        for (int u = 0; u < U; ++u) of_unit[u] = drop_of_unit(a.drop, step, drop_unit<T>(at + u * a.threads));
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * groups; first < a.rows; first += (int64_t)gridDim.x * groups, turn ^= 1) {
        const int64_t row = first + group;
        const bool live = row < a.rows;
        uint4 raw[U], res[U], up[U], in[U];
        const float2 st = live ? __ldg(a.stats + row) : both(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = at + u * a.threads;
            const bool on = live && c < a.chunks;
            raw[u] = on ? Chunk<T>::load_raw(static_cast<const T *>(a.x) + row * a.ldx + c * E) : make_uint4(0, 0, 0, 0);
            up[u] = on ? Chunk<T>::load_raw(static_cast<const T *>(a.dy) + row * a.lddy + c * E) : make_uint4(0, 0, 0, 0);
            res[u] = on && a.r ? Chunk<T>::load_raw(static_cast<const T *>(a.r) + row * a.ldr + c * E) : make_uint4(0, 0, 0, 0);
            in[u] = on && a.dz ? Chunk<T>::load_raw(static_cast<const T *>(a.dz) + row * a.lddz + c * E) : make_uint4(0, 0, 0, 0);
        }
        float2 n[U][P], g[U][P], s1 = both(0.f), s2 = both(0.f);
        uint32_t h[kDrop ? U : 1][P];
        PhiloxRow of_row;
        if constexpr (kDrop) of_row = drop_of_row(a.drop, (uint32_t)row);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = at + u * a.threads;
            float2 v[P], gain[P];
            unpack_pairs(raw[u], n[u]);
            if constexpr (kDrop) {
                drop_halves<E>(drop_words(a.drop, of_unit[u], of_row), c, h[u]);
                drop_apply(a.drop, h[u], n[u]);
            }
            unpack_pairs(res[u], v);
            unpack_pairs(up[u], g[u]);
            load_gains(c < a.chunks ? a.gain : nullptr, c, 1.f, gain);
#pragma unroll
            for (int i = 0; i < P; ++i) {            // places behind the row's end: g = 0
                n[u][i] = __fmul2_rn(__fadd2_rn(__fadd2_rn(n[u][i], v[i]), both(-st.x)), both(st.y));
                dgain[u][i] = __ffma2_rn(g[u][i], n[u][i], dgain[u][i]);
                dshift[u][i] = __fadd2_rn(dshift[u][i], g[u][i]);
                g[u][i] = __fmul2_rn(g[u][i], gain[i]);
                s1 = __fadd2_rn(s1, g[u][i]);
                s2 = __ffma2_rn(g[u][i], n[u][i], s2);
            }
        }
        float sums[2] = {s1.x + s1.y, s2.x + s2.y};
        row_sums<2>(sums, a.threads, buf[turn]);
        if (!live) continue;
        const float2 c1 = both(-sums[0] * a.inv_dim), c2 = both(-sums[1] * a.inv_dim);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = at + u * a.threads;
            if (c >= a.chunks) continue;
            float2 v[P];
            unpack_pairs(in[u], v);
#pragma unroll
            for (int i = 0; i < P; ++i) g[u][i] = __ffma2_rn(__ffma2_rn(n[u][i], c2, __fadd2_rn(g[u][i], c1)), both(st.y), v[i]);
            if (a.dr) store_pairs(static_cast<T *>(a.dr) + row * a.lddr + c * E, g[u]);
            if constexpr (kDrop) drop_apply(a.drop, h[u], g[u]);
            store_pairs(static_cast<T *>(a.dx) + row * a.lddx + c * E, g[u]);
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
            for (int e = 0; e < E; ++e) {
                const float2 v = side ? dshift[u][e / 2] : dgain[u][e / 2];
                join[(u * E + e) * kNormThreads + threadIdx.x] = e & 1 ? v.y : v.x;
            }
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
    int64_t ldx, ldr, ldy, rows, total;              // total: threads that have something to do
    int32_t dim;
    uint32_t units, magic, shift;                    // units (8 elements) of a row; i / units = (umulhi(i, magic) + i) >> shift for i < 2^31 where shift > 0
    DropArgs drop;
};

// A thread takes one unit of kRows neighbouring rows, whose loads go out together and whose random words share the unit's part.  What bounds it with
// 16-bit elements is the generator and the conversions, 58 % of the integer pipe: 262 144 x 256 takes 46 us, 5.8 TB/s (call by call
// 76 us with a unit after the other per thread, 57 with four under way and comparisons in place of a mask).
constexpr int kDropRows = 4;
template <typename T, bool kRes, int kRows>
__global__ void __launch_bounds__(kNormThreads)
dropout_kernel(const __grid_constant__ DropoutArgs a)
{
    constexpr int E = Chunk<T>::kElems, kChunks = 8 / E;
    const int64_t i = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
    if (i >= a.total) return;
    const uint32_t step = drop_step(a.drop);
    const int64_t tuple = a.shift ? (int64_t)(((uint64_t)__umulhi((uint32_t)i, a.magic) + (uint32_t)i) >> a.shift) : i / a.units, row0 = tuple * kRows;
    const uint32_t unit = (uint32_t)(i - tuple * a.units);
    uint4 x[kRows][kChunks], r[kRes ? kRows : 1][kChunks];
#pragma unroll
    for (int q = 0; q < kRows; ++q)
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            const int c = (int)unit * 8 + k * E;
            const bool on = row0 + q < a.rows && c < a.dim;
            x[q][k] = on ? Chunk<T>::load_raw(static_cast<const T *>(a.x) + (row0 + q) * a.ldx + c) : make_uint4(0, 0, 0, 0);
            if constexpr (kRes) r[q][k] = on ? Chunk<T>::load_raw(static_cast<const T *>(a.r) + (row0 + q) * a.ldr + c) : make_uint4(0, 0, 0, 0);
        }
    const PhiloxUnit of_unit = drop_of_unit(a.drop, step, unit);
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
        if (row0 + q >= a.rows) break;
        const uint4 w = drop_words(a.drop, of_unit, drop_of_row(a.drop, (uint32_t)(row0 + q)));
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            const int c = (int)unit * 8 + k * E;
            if (c >= a.dim) continue;
            float2 v[E / 2];
            uint32_t h[E / 2];
            unpack_pairs(x[q][k], v);
            drop_halves<E>(w, k, h);
            drop_apply(a.drop, h, v);
            if constexpr (kRes) {
                float2 p[E / 2];
                unpack_pairs(r[q][k], p);
#pragma unroll
                for (int j = 0; j < E / 2; ++j) v[j] = __fadd2_rn(v[j], p[j]);
            }
            store_pairs(static_cast<T *>(a.y) + (row0 + q) * a.ldy + c, v);
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
// Two results in one place
bool same_place(const e2egrec_mat *a, const e2egrec_mat *b) { return a && b && a->rows > 0 && a->data == b->data; }

// Threads of a row and chunks per thread (a template argument).  Threads hold as many values as their registers allow, and with that as few as
// possible share a row: what is done once per row, exchanges and addresses, is done for more rows by a warp then.  Of the numbers of chunks the
// one that leaves the fewest places empty (100 000 x 152, call by call: 43 us with one chunk each of 32 threads, 29 so).  Rows so few that every chunk has a
// thread of its own get that: the time is one chunk's then (64 x 256, call by call: 10 -> 6 us, of which the kernel is 4).
struct NormShape {
    int threads, per;
};
NormShape norm_shape(const e2egrec_mat *X, bool back)
{
    const int es = (int)dtype_size(X->dtype), chunks = X->dim * es / 16, values = 16 / es;
    const bool few = X->rows * chunks <= (int64_t)148 * 1024;
    NormShape best{kNormThreads, kForwardValues / values};
    int places = kNormThreads * best.per;
    for (int per = 1; per <= (back ? kBackValues : kForwardValues) / values; ++per) {
        if (per == 7) continue;
        int threads = 1;
        while (threads < kNormThreads && threads * per < chunks) threads *= 2;
        if (threads * per >= chunks && threads * per <= places) {
            best = NormShape{threads, per};
            places = threads * per;
            if (few) break;
        }
    }
    return best;
}

template <typename T, int U, bool kDrop, bool kBack> void norm_launch(const NormArgs &a, cudaStream_t st, int blocks)
{
    note_launch();
    const int64_t per = (int64_t)kNormThreads / a.threads;
    if constexpr (kBack) {
        const size_t smem = a.part ? (size_t)U * Chunk<T>::kElems * kNormThreads * sizeof(float) : 0;
        norm_bwd_kernel<T, U, kDrop><<<blocks, kNormThreads, smem, st>>>(a);
    } else {
        norm_fwd_kernel<T, U, kDrop><<<(unsigned)ceil_div(a.rows, per), kNormThreads, 0, st>>>(a);
    }
}

// (the numbers of chunks that norm_shape gives, of either direction)
template <typename T, bool kDrop, bool kBack> void norm_of(const NormArgs &a, int per, cudaStream_t st, int blocks)
{
    constexpr bool kWide = sizeof(T) == 4;
    if (per == 1) return norm_launch<T, 1, kDrop, kBack>(a, st, blocks);
    if (per == 2) return norm_launch<T, 2, kDrop, kBack>(a, st, blocks);
    if constexpr (kWide || !kBack)
        if (per == 3) return norm_launch<T, 3, kDrop, kBack>(a, st, blocks);
    if (per == 4) return norm_launch<T, 4, kDrop, kBack>(a, st, blocks);
    if constexpr (kWide && !kBack) {
        if (per == 5) return norm_launch<T, 5, kDrop, kBack>(a, st, blocks);
        if (per == 6) return norm_launch<T, 6, kDrop, kBack>(a, st, blocks);
    }
    if constexpr (kWide) norm_launch<T, 8, kDrop, kBack>(a, st, blocks);
}
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

// One row per thread while that leaves no SM more than eight blocks: the time is that of one unit then.
template <typename T, bool kRes> void dropout_launch(DropoutArgs &a, cudaStream_t st)
{
    const int rows = a.rows * a.units <= (int64_t)148 * 8 * kNormThreads ? 1 : kDropRows;
    a.total = ceil_div(a.rows, rows) * a.units;
    if (a.total + kNormThreads < (int64_t)1 << 31) {                     // division by the units of a row as a product
        while (((uint64_t)1 << a.shift) < a.units) ++a.shift;
        a.magic = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << a.shift) - a.units)) / a.units + 1);
    }
    const unsigned grid = (unsigned)ceil_div(a.total, kNormThreads);
    note_launch();
    if (rows == 1) dropout_kernel<T, kRes, 1><<<grid, kNormThreads, 0, st>>>(a);
    else dropout_kernel<T, kRes, kDropRows><<<grid, kNormThreads, 0, st>>>(a);
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
    a.rows = X->rows;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (X->dtype == E2EGREC_F32) a.r ? dropout_launch<float, true>(a, st) : dropout_launch<float, false>(a, st);
    else a.r ? dropout_launch<__nv_bfloat16, true>(a, st) : dropout_launch<__nv_bfloat16, false>(a, st);
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
    if (rc == E2EGREC_OK && same_place(Y, Z)) rc = E2EGREC_ERR_ARG;
    if (rc == E2EGREC_OK && (misaligned(shift) || reinterpret_cast<uintptr_t>(stats) % 8)) rc = E2EGREC_ERR_ALIGN;
    if (rc != E2EGREC_OK || X->rows == 0) return rc;
    a.y = Y->data;
    a.ldy = Y->ld;
    a.z = Z ? Z->data : nullptr;
    a.ldz = Z ? Z->ld : 0;
    a.shift = shift;
    a.eps = eps;
    a.stats = reinterpret_cast<float2 *>(stats);
    const NormShape s = norm_shape(X, false);
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
    const NormShape s = norm_shape(X, true);
    const int64_t tile = kNormThreads / s.threads;
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
    if (rc == E2EGREC_OK && same_place(dX, dR)) rc = E2EGREC_ERR_ARG;
    if (rc == E2EGREC_OK && (reinterpret_cast<uintptr_t>(stats) % 8 || reinterpret_cast<uintptr_t>(dgain) % 4 || reinterpret_cast<uintptr_t>(dshift) % 4))
        rc = E2EGREC_ERR_ALIGN;
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
