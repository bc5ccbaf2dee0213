// Attention of fp32 sequences by tiles of 64 rows x 64 keys on fp32 FMA (head_dim <= 128): scores to fp32 accuracy, which neither TF32
// nor bf16 products give.
//
// 256 threads: thread (ty, tx) of 16 x 16 forms the 4 x 4 scores of rows 4 ty + i and keys tx + 16 j as dot products of row-major
// tiles, four elements of each at a time (eight 16-byte reads of shared memory for 64 FMA).  Tiles have rows of an odd number
// of 16-byte units, so that eight neighbouring rows lie in different banks.  p and dS go through shared memory; the products with V, K, dO
// and Q are outer products over the same row-major tiles, columns 4 tx + 64 c.  FMA throughput bounds it.
#include <algorithm>

#include "attention.cuh"
#include "tcgen05.cuh"

namespace e2egrec {
namespace {

constexpr int kTile = 64, kThreads = 256, kLdP = kTile + 4;

struct SimtShape {
    int ld;                               // floats from row to row of a tile in shared memory
    int tiles, splits;                    // blocks of rows (or keys) per sequence and key head; stretches of the keys
};

__device__ inline float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// sums and maxima over the 16 threads that share rows
__device__ inline float row_sum(float v)
{
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ inline float row_max(float v)
{
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

// One tile -> shared memory: thread t takes row t / 4 and every fourth 16-byte unit of it; src: that row, null for zeros
__device__ inline void load_tile(float *tile, const SimtShape &f, const float *src, const void *any, int head_dim)
{
    const uint32_t dst = smem_u32(tile + (threadIdx.x >> 2) * f.ld);
    for (int u = threadIdx.x & 3; u * 4 < head_dim; u += 4) cp_async16(dst + u * 16, src ? static_cast<const void *>(src + u * 4) : any, src != nullptr);
}

// s[i][j] = a[4 ty + i] . b[tx + 16 j]
__device__ inline void scores(const float *a, const float *b, int ld, int head_dim, int ty, int tx, float (&s)[4][4])
{
    const float *pa = a + 4 * ty * ld, *pb = b + tx * ld;
    float2 t[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) t[i][j] = make_float2(0.f, 0.f);
#pragma unroll 2
    for (int d = 0; d < head_dim; d += 4) {
        float4 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = *reinterpret_cast<const float4 *>(pa + i * ld + d);
            y[i] = *reinterpret_cast<const float4 *>(pb + 16 * i * ld + d);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                t[i][j] = __ffma2_rn(make_float2(x[i].x, x[i].y), make_float2(y[j].x, y[j].y), t[i][j]);
                t[i][j] = __ffma2_rn(make_float2(x[i].z, x[i].w), make_float2(y[j].z, y[j].w), t[i][j]);
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = t[i][j].x + t[i][j].y;
}

__device__ inline void fma4(float (&o)[4], float w, const float4 &v)
{
    const float2 w2 = make_float2(w, w);
    const float2 a = __ffma2_rn(w2, make_float2(v.x, v.y), make_float2(o[0], o[1])), b = __ffma2_rn(w2, make_float2(v.z, v.w), make_float2(o[2], o[3]));
    o[0] = a.x;
    o[1] = a.y;
    o[2] = b.x;
    o[3] = b.y;
}

// o[i][c] += sum_k w[4 ty + i][k] b[k][4 tx + 64 c]     (w row by row)
template <int C> __device__ inline void add_rows(float (&o)[4][C][4], const float *w, const float *b, int ld, int head_dim, int ty, int tx)
{
#pragma unroll 2
    for (int k = 0; k < kTile; k += 4) {
        float4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4 *>(w + (4 * ty + i) * kLdP + k);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (4 * tx + 64 * c >= head_dim) continue;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float4 v = *reinterpret_cast<const float4 *>(b + (k + n) * ld + 4 * tx + 64 * c);
#pragma unroll
                for (int i = 0; i < 4; ++i) fma4(o[i][c], n == 0 ? x[i].x : n == 1 ? x[i].y : n == 2 ? x[i].z : x[i].w, v);
            }
        }
    }
}
// o[i][c] += sum_r w[r][4 ty + i] b[r][4 tx + 64 c]     (w column by column)
template <int C> __device__ inline void add_columns(float (&o)[4][C][4], const float *w, const float *b, int ld, int head_dim, int ty, int tx)
{
#pragma unroll 4
    for (int r = 0; r < kTile; ++r) {
        const float4 x = *reinterpret_cast<const float4 *>(w + r * kLdP + 4 * ty);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (4 * tx + 64 * c >= head_dim) continue;
            const float4 v = *reinterpret_cast<const float4 *>(b + r * ld + 4 * tx + 64 * c);
            fma4(o[0][c], x.x, v);
            fma4(o[1][c], x.y, v);
            fma4(o[2][c], x.z, v);
            fma4(o[3][c], x.w, v);
        }
    }
}

template <int C> __device__ inline void clear(float (&o)[4][C][4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][c][e] = 0.f;
}

// columns 4 tx + 64 c of a row, times f; zeros (whatever the sums hold) where !keep
template <int C> __device__ inline void store_columns(float *row, const float (&o)[C][4], float f, int head_dim, int tx, bool keep = true)
{
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (4 * tx + 64 * c < head_dim)
            *reinterpret_cast<float4 *>(row + 4 * tx + 64 * c) =
                keep ? make_float4(o[c][0] * f, o[c][1] * f, o[c][2] * f, o[c][3] * f) : make_float4(0.f, 0.f, 0.f, 0.f);
}

struct SimtUnit {
    SeqRange rg;
    int64_t kb, ke, rows;
    int z, t0, h;
};
__device__ inline SimtUnit simt_unit(const AttnArgs &a, const SimtShape &f)
{
    SimtUnit x;
    uint32_t u = blockIdx.x;
    x.z = (int)(u % (uint32_t)f.splits);
    u /= (uint32_t)f.splits;
    x.t0 = (int)(u % (uint32_t)f.tiles);
    u /= (uint32_t)f.tiles;
    const uint32_t s = u / (uint32_t)a.kv_heads;
    x.h = (int)(u - s * (uint32_t)a.kv_heads);
    x.rg = seq_range(a, s, threadIdx.x == 0 && x.z == 0 && x.t0 == 0 && x.h == 0);
    x.rows = (x.rg.q1 - x.rg.q0) * a.group;
    const int64_t per = ceil_div(x.rg.k1 - x.rg.k0, f.splits);
    x.kb = min(x.rg.k0 + x.z * per, x.rg.k1);
    x.ke = min(x.kb + per, x.rg.k1);
    return x;
}

// query row and head of row r of the key head's matrix
__device__ inline void row_of(const AttnArgs &a, const SimtUnit &x, int64_t r, int64_t &row, int &head)
{
    const int64_t i = a.group == 1 ? r : (r >> 32 ? r / a.group : (int64_t)((uint32_t)r / (uint32_t)a.group));
    row = x.rg.q0 + i;
    head = x.h * a.group + (int)(r - i * a.group);
}

template <int C>
__global__ void __launch_bounds__(kThreads)
attn_simt_fwd_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ SimtShape f, float *__restrict__ part_o, float2 *__restrict__ part_ml)
{
    extern __shared__ __align__(16) float sm[];
    float *q_s = sm, *k_s = q_s + kTile * f.ld, *v_s = k_s + kTile * f.ld, *p_s = v_s + kTile * f.ld;
    __shared__ uint8_t seen_s[kTile];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, heads = a.kv_heads * a.group, lr = threadIdx.x >> 2;
    const SimtUnit x = simt_unit(a, f);
    const float c1 = a.scale * kLog2e;
    const float *qp = static_cast<const float *>(a.q), *kp = static_cast<const float *>(a.k), *vp = static_cast<const float *>(a.v);
    for (int64_t t = x.t0; t * kTile < x.rows; t += f.tiles) {
        const int64_t r0 = t * kTile;
        __syncthreads();
        {
            int64_t row;
            int head;
            row_of(a, x, min(r0 + lr, x.rows - 1), row, head);
            load_tile(q_s, f, r0 + lr < x.rows ? qp + row * a.ldq + (int64_t)head * a.head_dim : nullptr, qp, a.head_dim);
        }
        float o[4][C][4], m[4], l[4];
        clear<C>(o);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.f;
        }
        for (int64_t j0 = x.kb; j0 < x.ke; j0 += kTile) {
            if (j0 > x.kb) __syncthreads();
            const int64_t key = j0 + lr;
            const bool seen = key < x.ke && (!a.mask || a.mask[key]);
            load_tile(k_s, f, seen ? kp + key * a.ldk + (int64_t)x.h * a.head_dim : nullptr, qp, a.head_dim);
            load_tile(v_s, f, seen ? vp + key * a.ldv + (int64_t)x.h * a.head_dim : nullptr, qp, a.head_dim);
            if ((threadIdx.x & 3) == 0) seen_s[lr] = seen;
            cp_async_wait_all();
            __syncthreads();
            float s[4][4];
            scores(q_s, k_s, f.ld, a.head_dim, ty, tx, s);
            bool on[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) on[j] = seen_s[tx + 16 * j];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[i][j] = on[j] ? s[i][j] * c1 : -INFINITY;
                    top = fmaxf(top, s[i][j]);
                }
                top = fmaxf(m[i], row_max(top));
                const float base = top == -INFINITY ? 0.f : top, c = exp2_fast(m[i] - base);
                m[i] = top;
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p = exp2_fast(s[i][j] - base);
                    sum += p;
                    p_s[(4 * ty + i) * kLdP + tx + 16 * j] = p;
                }
                l[i] = l[i] * c + sum;
#pragma unroll
                for (int n = 0; n < C; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][n][e] *= c;
            }
            __syncwarp();                                // rows of p belong to one half-warp
            add_rows<C>(o, p_s, v_s, f.ld, a.head_dim, ty, tx);
            __syncwarp();
        }
        cp_async_wait_all();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            l[i] = row_sum(l[i]);
            const int64_t r = r0 + 4 * ty + i;
            if (r >= x.rows) continue;
            int64_t row;
            int head;
            row_of(a, x, r, row, head);
            const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
            if (f.splits == 1) {
                store_columns<C>(static_cast<float *>(a.out) + row * a.ldo + (int64_t)head * a.head_dim, o[i], inv, a.head_dim, tx);
                if (a.lse && tx == 0) a.lse[row * heads + head] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * kLn2;
            } else {
                const int64_t p = ((int64_t)x.z * a.q_rows + row) * heads + head;
                store_columns<C>(part_o + p * a.head_dim, o[i], inv, a.head_dim, tx);
                if (tx == 0) part_ml[p] = make_float2(l[i] == 0.f ? -INFINITY : m[i], l[i]);
            }
        }
    }
}

template <int C>
__global__ void __launch_bounds__(kThreads)
attn_simt_dq_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ SimtShape f, float *__restrict__ part_dq, float *__restrict__ dots)
{
    extern __shared__ __align__(16) float sm[];
    float *q_s = sm, *g_s = q_s + kTile * f.ld, *k_s = g_s + kTile * f.ld, *v_s = k_s + kTile * f.ld, *ds_s = v_s + kTile * f.ld;
    __shared__ uint8_t seen_s[kTile];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, heads = a.kv_heads * a.group, lr = threadIdx.x >> 2;
    const SimtUnit x = simt_unit(a, f);
    const float c1 = a.scale * kLog2e;
    const float *qp = static_cast<const float *>(a.q), *kp = static_cast<const float *>(a.k), *vp = static_cast<const float *>(a.v);
    const float *gp = static_cast<const float *>(a.dout), *op = static_cast<const float *>(a.o);
    for (int64_t t = x.t0; t * kTile < x.rows; t += f.tiles) {
        const int64_t r0 = t * kTile;
        __syncthreads();
        {
            int64_t row;
            int head;
            row_of(a, x, min(r0 + lr, x.rows - 1), row, head);
            const bool on = r0 + lr < x.rows;
            load_tile(q_s, f, on ? qp + row * a.ldq + (int64_t)head * a.head_dim : nullptr, qp, a.head_dim);
            load_tile(g_s, f, on ? gp + row * a.ldg + (int64_t)head * a.head_dim : nullptr, qp, a.head_dim);
        }
        float dq[4][C][4], lse[4], d[4];
        int64_t row[4];
        int head[4];
        clear<C>(dq);
        cp_async_wait_all();
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + 4 * ty + i;
            row_of(a, x, min(r, x.rows - 1), row[i], head[i]);
            lse[i] = INFINITY;
            d[i] = 0.f;
            if (r < x.rows) {
                const float v = a.lse[row[i] * heads + head[i]];
                if (v != -INFINITY) {
                    lse[i] = v * kLog2e;
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        if (4 * tx + 64 * c < a.head_dim) {
                            const float4 y = *reinterpret_cast<const float4 *>(op + row[i] * a.ldo + (int64_t)head[i] * a.head_dim + 4 * tx + 64 * c);
                            const float4 g = *reinterpret_cast<const float4 *>(g_s + (4 * ty + i) * f.ld + 4 * tx + 64 * c);
                            d[i] += y.x * g.x + y.y * g.y + y.z * g.z + y.w * g.w;
                        }
                }
            }
            d[i] = row_sum(d[i]);
            if (r < x.rows && x.z == 0 && tx == 0) dots[row[i] * heads + head[i]] = d[i];
        }
        for (int64_t j0 = x.kb; j0 < x.ke; j0 += kTile) {
            __syncthreads();
            const int64_t key = j0 + lr;
            const bool seen = key < x.ke && (!a.mask || a.mask[key]);
            load_tile(k_s, f, seen ? kp + key * a.ldk + (int64_t)x.h * a.head_dim : nullptr, qp, a.head_dim);
            load_tile(v_s, f, seen ? vp + key * a.ldv + (int64_t)x.h * a.head_dim : nullptr, qp, a.head_dim);
            if ((threadIdx.x & 3) == 0) seen_s[lr] = seen;
            cp_async_wait_all();
            __syncthreads();
            float s[4][4], u[4][4];
            scores(q_s, k_s, f.ld, a.head_dim, ty, tx, s);
            scores(g_s, v_s, f.ld, a.head_dim, ty, tx, u);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool on = seen_s[tx + 16 * j];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    ds_s[(4 * ty + i) * kLdP + tx + 16 * j] = on ? exp2_fast(fmaf(s[i][j], c1, -lse[i])) * (u[i][j] - d[i]) : 0.f;
            }
            __syncwarp();
            add_rows<C>(dq, ds_s, k_s, f.ld, a.head_dim, ty, tx);
            __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (r0 + 4 * ty + i >= x.rows) continue;
            const bool keep = lse[i] != INFINITY;        // a row that saw no key passes on nothing
            if (f.splits == 1) store_columns<C>(static_cast<float *>(a.dq) + row[i] * a.ldq2 + (int64_t)head[i] * a.head_dim, dq[i], a.scale, a.head_dim, tx, keep);
            else store_columns<C>(part_dq + (((int64_t)x.z * a.q_rows + row[i]) * heads + head[i]) * a.head_dim, dq[i], a.scale, a.head_dim, tx, keep);
        }
    }
}

template <int C>
__global__ void __launch_bounds__(kThreads)
attn_simt_dkv_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ SimtShape f, const float *__restrict__ dots)
{
    extern __shared__ __align__(16) float sm[];
    float *k_s = sm, *v_s = k_s + kTile * f.ld, *q_s = v_s + kTile * f.ld, *g_s = q_s + kTile * f.ld, *p_s = g_s + kTile * f.ld, *ds_s = p_s + kTile * kLdP;
    __shared__ float lse_s[kTile], dot_s[kTile];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, heads = a.kv_heads * a.group, lr = threadIdx.x >> 2;
    const SimtUnit x = simt_unit(a, f);
    const float c1 = a.scale * kLog2e;
    const float *qp = static_cast<const float *>(a.q), *kp = static_cast<const float *>(a.k), *vp = static_cast<const float *>(a.v);
    const float *gp = static_cast<const float *>(a.dout);
    for (int64_t j0 = x.rg.k0 + (int64_t)x.t0 * kTile; j0 < x.rg.k1; j0 += (int64_t)f.tiles * kTile) {
        __syncthreads();
        {
            const int64_t key = j0 + lr;
            const bool seen = key < x.rg.k1 && (!a.mask || a.mask[key]);
            load_tile(k_s, f, seen ? kp + key * a.ldk + (int64_t)x.h * a.head_dim : nullptr, kp, a.head_dim);
            load_tile(v_s, f, seen ? vp + key * a.ldv + (int64_t)x.h * a.head_dim : nullptr, kp, a.head_dim);
        }
        float dk[4][C][4], dv[4][C][4];
        clear<C>(dk);
        clear<C>(dv);
        for (int64_t r0 = 0; r0 < x.rows; r0 += kTile) {
            if (r0) __syncthreads();
            int64_t row;
            int head;
            row_of(a, x, min(r0 + lr, x.rows - 1), row, head);
            float l = INFINITY;
            if (r0 + lr < x.rows) {
                const float v = a.lse[row * heads + head];
                if (v != -INFINITY) l = v * kLog2e;
            }
            if ((threadIdx.x & 3) == 0) {
                lse_s[lr] = l;
                dot_s[lr] = l != INFINITY ? dots[row * heads + head] : 0.f;
            }
            load_tile(q_s, f, l != INFINITY ? qp + row * a.ldq + (int64_t)head * a.head_dim : nullptr, kp, a.head_dim);
            load_tile(g_s, f, l != INFINITY ? gp + row * a.ldg + (int64_t)head * a.head_dim : nullptr, kp, a.head_dim);
            cp_async_wait_all();
            __syncthreads();
            float s[4][4], u[4][4];
            scores(q_s, k_s, f.ld, a.head_dim, ty, tx, s);
            scores(g_s, v_s, f.ld, a.head_dim, ty, tx, u);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lse = lse_s[4 * ty + i], d = dot_s[4 * ty + i];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p = exp2_fast(fmaf(s[i][j], c1, -lse));
                    p_s[(4 * ty + i) * kLdP + tx + 16 * j] = p;
                    ds_s[(4 * ty + i) * kLdP + tx + 16 * j] = p * (u[i][j] - d);
                }
            }
            __syncthreads();
            add_columns<C>(dv, p_s, g_s, f.ld, a.head_dim, ty, tx);
            add_columns<C>(dk, ds_s, q_s, f.ld, a.head_dim, ty, tx);
        }
        cp_async_wait_all();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t key = j0 + 4 * ty + i;
            if (key >= x.rg.k1) continue;
            const bool keep = !a.mask || a.mask[key];
            store_columns<C>(static_cast<float *>(a.dk) + key * a.ldk2 + (int64_t)x.h * a.head_dim, dk[i], a.scale, a.head_dim, tx, keep);
            store_columns<C>(static_cast<float *>(a.dv) + key * a.ldv2 + (int64_t)x.h * a.head_dim, dv[i], 1.f, a.head_dim, tx, keep);
        }
    }
}

constexpr int kMaxDevices = 64;
template <typename Kernel> bool allow_smem(Kernel kernel, bool (&done)[kMaxDevices])
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return false;
    if (done[dev]) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024) != cudaSuccess) return false;
    done[dev] = true;
    return true;
}

SimtShape shape_of(const AttnArgs &a, int64_t tiles, int splits)
{
    SimtShape f{};
    f.ld = (a.head_dim / 4 | 1) * 4;                 // an odd number of 16-byte units
    f.tiles = (int)tiles;
    f.splits = splits;
    return f;
}

size_t smem_of(const SimtShape &f, int tiles, int scores) { return ((size_t)tiles * kTile * f.ld + (size_t)scores * kTile * kLdP) * sizeof(float); }

template <int C> bool forward_of(const AttnArgs &a, const SimtPlan &p, float *part_o, float2 *part_ml, cudaStream_t st)
{
    static bool done[kMaxDevices] = {};
    if (!allow_smem(attn_simt_fwd_kernel<C>, done)) return false;
    const SimtShape f = shape_of(a, p.q_tiles, p.splits);
    note_launch();
    attn_simt_fwd_kernel<C><<<(unsigned)(a.n_seq * a.kv_heads * p.q_tiles * p.splits), kThreads, smem_of(f, 3, 1), st>>>(a, f, part_o, part_ml);
    return true;
}

template <int C> bool backward_of(const AttnArgs &a, const SimtPlan &p, float *part_dq, float *dots, cudaStream_t st)
{
    static bool done[2][kMaxDevices] = {};
    if (!allow_smem(attn_simt_dq_kernel<C>, done[0]) || !allow_smem(attn_simt_dkv_kernel<C>, done[1])) return false;
    if (a.q_rows) {
        const SimtShape f = shape_of(a, p.q_tiles, p.splits);
        note_launch();
        attn_simt_dq_kernel<C><<<(unsigned)(a.n_seq * a.kv_heads * p.q_tiles * p.splits), kThreads, smem_of(f, 4, 1), st>>>(a, f, part_dq, dots);
    }
    if (a.k_rows) {
        const SimtShape f = shape_of(a, p.k_tiles, 1);
        note_launch();
        attn_simt_dkv_kernel<C><<<(unsigned)(a.n_seq * a.kv_heads * p.k_tiles), kThreads, smem_of(f, 4, 2), st>>>(a, f, dots);
    }
    return true;
}

}  // namespace

SimtPlan simt_plan(const AttnArgs &a, int64_t max_q, int64_t max_k)
{
    SimtPlan p{};
    const int64_t units = std::max<int64_t>(a.n_seq * a.kv_heads, 1), most = (((int64_t)1 << 31) - 1) / units;
    p.q_tiles = std::max<int64_t>(1, std::min(ceil_div(max_q * a.group, kTile), most));
    p.k_tiles = std::max<int64_t>(1, std::min(ceil_div(max_k, kTile), most));
    p.splits = 1;
    if (units * p.q_tiles < 296) p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({296 / (units * p.q_tiles), max_k / (2 * kTile), kMaxSplits}));
    return p;
}

bool simt_attention_forward(const AttnArgs &a, const SimtPlan &p, float *part_o, float2 *part_ml, cudaStream_t st)
{
    return a.head_dim <= 64 ? forward_of<1>(a, p, part_o, part_ml, st) : forward_of<2>(a, p, part_o, part_ml, st);
}

bool simt_attention_backward(const AttnArgs &a, const SimtPlan &p, float *part_dq, float *dots, cudaStream_t st)
{
    return a.head_dim <= 64 ? backward_of<1>(a, p, part_dq, dots, st) : backward_of<2>(a, p, part_dq, dots, st);
}

}  // namespace e2egrec
