// Attention of fp32 sequences on fp32 FMA (head_dim <= 128): scores to fp32 accuracy, which neither TF32 nor bf16 products give.
//
// Tiles of 16 I rows x 64 keys, I = 1, 2 or 4 by the rows that a key head has.  16 x TX threads: thread (ty, tx) forms the scores of
// rows ty + 16 i and keys tx + TX j as dot products of row-major tiles, four elements of each at a time.  TX = 8 where there are up to 32
// rows (more scores per thread, whose reads of shared memory are whole lines) and in the forward pass of heads of up to 32 columns,
// TX = 16 else, which leaves the schedulers twice the warps.  Tiles have rows of an odd number of 16-byte units, so that eight neighbouring
// rows lie in different banks.  p and dS go through shared memory; the products with V, K, dO and Q are outer products over the same
// row-major tiles, columns 4 cx + 4 TX c; of narrow heads the threads of a row take a part of the summed index each, which are added up
// once at the end.  The next tiles are on their way beside a tile's products where shared memory holds both.
// Reads of shared memory and their latency bound it (8 x 512 x 2048, heads of 64: their pipe 65 %, FMA 48 %; tiles by bulk copies instead
// of cp.async change nothing).  Forward and backward, us with TX = 16 everywhere and with this rule: 107 of 372 x 61, heads of 16: 440,
// 417; 300 of 8 x 200, heads of 64: 467, 435; 1000 of 8 x 40, heads of 64: 424, 374.  77 of up to 61 x 307, heads of 36: 166.
#include <algorithm>
#include <atomic>

#include "attention.cuh"
#include "tcgen05.cuh"

namespace e2egrec {
namespace {

constexpr int kTile = 64, kLdP = kTile + 4;

// Blocks per SM, by the registers that the sums take; C columns per thread, in fours
constexpr int blocks_of(int TX, int C, int I) { return TX == 8 ? 3 : (C == 2 && I == 4 ? 1 : 2); }

struct SimtShape {
    int ld;                               // floats from row to row of a tile in shared memory
    int tiles, splits;                    // blocks of rows (or keys) per sequence and key head; stretches of the keys
    int stages;                           // tiles of the side that a block goes over: 2: one lands beside the products of the other
    int cols;                             // threads side by side over a head's columns (a power of two), TX / cols parts of the sums
    int tile_floats;                      // of all tiles; what a bias takes follows
};

__device__ inline float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// sums and maxima over the TX threads that share rows
template <int TX> __device__ inline float row_sum(float v)
{
#pragma unroll
    for (int o = TX / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
template <int TX> __device__ inline float row_max(float v)
{
#pragma unroll
    for (int o = TX / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

// One tile -> shared memory: kPer threads take a row's 16-byte units in turn; src: that row, null for zeros
template <int kPer> __device__ inline void load_tile(float *tile, const SimtShape &f, const float *src, const void *any, int head_dim)
{
    const uint32_t dst = smem_u32(tile + threadIdx.x / kPer * f.ld);
#pragma unroll 4
    for (int u = threadIdx.x % kPer; u * 4 < head_dim; u += kPer) cp_async16(dst + u * 16, src ? static_cast<const void *>(src + u * 4) : any, src != nullptr);
}

// s[i][j] = a[ty + 16 i] . b[tx + TX j]
template <int TX, int I> __device__ inline void scores(const float *a, const float *b, int ld, int head_dim, int ty, int tx, float (&s)[I][kTile / TX])
{
    constexpr int J = kTile / TX;
    const float *pa = a + ty * ld, *pb = b + tx * ld;
    float2 t[I][J];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) t[i][j] = make_float2(0.f, 0.f);
#pragma unroll 2
    for (int d = 0; d < head_dim; d += 4) {
        float4 x[I], y[J];
#pragma unroll
        for (int i = 0; i < I; ++i) x[i] = *reinterpret_cast<const float4 *>(pa + 16 * i * ld + d);
#pragma unroll
        for (int j = 0; j < J; ++j) y[j] = *reinterpret_cast<const float4 *>(pb + TX * j * ld + d);
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) t[i][j] = __ffma2_rn(make_float2(x[i].x, x[i].y), make_float2(y[j].x, y[j].y), t[i][j]);
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) t[i][j] = __ffma2_rn(make_float2(x[i].z, x[i].w), make_float2(y[j].z, y[j].w), t[i][j]);
    }
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) s[i][j] = t[i][j].x + t[i][j].y;
}

// a . b, added up in the order of one of the scores above: D of a row whose softmax is one key's alone is that key's dP to the last bit
__device__ inline float dot_as_scores(const float *a, const float *b, int head_dim)
{
    float2 t = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int d = 0; d < head_dim; d += 4) {
        const float4 x = *reinterpret_cast<const float4 *>(a + d), y = *reinterpret_cast<const float4 *>(b + d);
        t = __ffma2_rn(make_float2(x.x, x.y), make_float2(y.x, y.y), t);
        t = __ffma2_rn(make_float2(x.z, x.w), make_float2(y.z, y.w), t);
    }
    return t.x + t.y;
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

// Columns 4 cx + 4 TX c of a head, part `part` of the sums
template <int TX> struct Columns {
    int cx, part, parts;
    __device__ inline Columns(const SimtShape &f, int tx) : cx(tx & (f.cols - 1)), part(tx / f.cols), parts(TX / f.cols) {}
};

// o[i][c] += sum_k w[ty + 16 i][k] b[k][4 cx + 4 TX c]     (w row by row)
template <int C, int I, int TX>
__device__ inline void add_rows(float (&o)[I][C][4], const float *w, const float *b, int ld, int head_dim, int ty, const Columns<TX> &at)
{
#pragma unroll 2
    for (int k = at.part * 4; k < kTile; k += at.parts * 4) {
        float4 x[I];
#pragma unroll
        for (int i = 0; i < I; ++i) x[i] = *reinterpret_cast<const float4 *>(w + (ty + 16 * i) * kLdP + k);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (4 * at.cx + 4 * TX * c >= head_dim) continue;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float4 v = *reinterpret_cast<const float4 *>(b + (k + n) * ld + 4 * at.cx + 4 * TX * c);
#pragma unroll
                for (int i = 0; i < I; ++i) fma4(o[i][c], n == 0 ? x[i].x : n == 1 ? x[i].y : n == 2 ? x[i].z : x[i].w, v);
            }
        }
    }
}
// o[i][c] += sum_r w[r][4 ty + i] b[r][4 cx + 4 TX c]     (w column by column, 16 I rows)
template <int C, int I, int TX>
__device__ inline void add_columns(float (&o)[4][C][4], const float *w, const float *b, int ld, int head_dim, int ty, const Columns<TX> &at)
{
#pragma unroll 4
    for (int r = at.part; r < 16 * I; r += at.parts) {
        const float4 x = *reinterpret_cast<const float4 *>(w + r * kLdP + 4 * ty);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (4 * at.cx + 4 * TX * c >= head_dim) continue;
            const float4 v = *reinterpret_cast<const float4 *>(b + r * ld + 4 * at.cx + 4 * TX * c);
            fma4(o[0][c], x.x, v);
            fma4(o[1][c], x.y, v);
            fma4(o[2][c], x.z, v);
            fma4(o[3][c], x.w, v);
        }
    }
}
// the parts of the sums together, in every thread (all of a warp)
template <int TX, int C, int N> __device__ inline void add_parts(float (&o)[N][C][4], const SimtShape &f)
{
    if constexpr (C == 1)
        for (int off = f.cols; off < TX; off <<= 1)
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][0][e] += __shfl_xor_sync(0xFFFFFFFFu, o[i][0][e], off);
}

template <int C, int N> __device__ inline void clear(float (&o)[N][C][4])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][c][e] = 0.f;
}

// columns 4 cx + 4 TX c of a row, times f, by the first part's threads; zeros (whatever the sums hold) where !keep
template <int C, int TX> __device__ inline void store_columns(float *row, const float (&o)[C][4], float f, int head_dim, const Columns<TX> &at, bool keep = true)
{
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (at.part == 0 && 4 * at.cx + 4 * TX * c < head_dim)
            *reinterpret_cast<float4 *>(row + 4 * at.cx + 4 * TX * c) =
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
    const int64_t per = ceil_div(ceil_div(x.rg.k1 - x.rg.k0, f.splits), (int64_t)kTile) * kTile;
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

// ---- Bias by distance: positions of a tile's keys (and rows) lie beside it, every score looks its bucket up by bisection, the J of a row side by
// side.  The gradient of the table is formed beside dQ: every thread has bins of its own in shared memory, [buckets x threads], added up at
// the unit's end in a fixed order.  That wants a thread's rows to be of one head: groups that divide 16.  77 x 61 x 307, 4 on 2 heads of 36:
// forward 57 us (47 without a bias), backward 176 (135; 164 without the table's gradient).
struct SimtBias {
    int32_t *edges;                                      // kMaxBuckets, beyond the last the highest number
    float *table;                                        // [heads of the group x buckets], in powers of two
    float *bins;
};
// where they lie: behind `floats` floats of shared memory
__device__ inline SimtBias bias_of(float *sm, size_t floats, const AttnArgs &a)
{
    SimtBias s;
    s.edges = reinterpret_cast<int32_t *>(sm + floats);
    s.table = sm + floats + kMaxBuckets;
    s.bins = s.table + a.bias.buckets * a.group;
    return s;
}
__device__ inline void stage_bias(const AttnArgs &a, const SimtBias &s, int h)
{
    const int nb = a.bias.buckets, heads = a.kv_heads * a.group;
    for (int i = threadIdx.x; i < kMaxBuckets; i += blockDim.x) s.edges[i] = i < nb - 1 ? __ldg(a.bias.edges + i) : INT32_MAX;
    for (int i = threadIdx.x; i < nb * a.group; i += blockDim.x) s.table[i] = bias_at(a.bias, heads, i % nb, h * a.group + i / nb);
}

// Tiles of keys and values (or of rows) that a block goes over: stage b of two pairs of tiles, a turn's loads beside the turn before where
// there are two.  load(j, b) starts the copies of turn j into stage b; use(j, b) works on it.
template <typename Load, typename Use> __device__ inline void turns(const SimtShape &f, int64_t n, Load load, Use use)
{
    if (f.stages == 2 && n > 0) load(0, 0);
    for (int64_t j = 0; j < n; ++j) {
        const int b = f.stages == 2 ? (int)(j & 1) : 0;
        if (f.stages == 1) {
            __syncthreads();
            load(j, 0);
        }
        cp_async_wait_all();
        __syncthreads();
        if (f.stages == 2 && j + 1 < n) load(j + 1, b ^ 1);
        use(b);
    }
}

// position of row r, and where its head's biases begin
__device__ inline void place_row(const AttnArgs &a, const SimtUnit &x, int64_t r, int &pos, int &own)
{
    int64_t row;
    int head;
    row_of(a, x, min(r, x.rows - 1), row, head);
    pos = pos_of(a.bias.pos_q, row, x.rg.q0);
    own = (head - x.h * a.group) * a.bias.buckets;
}
// buckets of a row at pos_q and the thread's keys tx + TX j
template <int TX> __device__ inline void buckets_of(const AttnArgs &a, const SimtBias &s, const int32_t *pos, int tx, int pos_q, int (&bucket)[kTile / TX])
{
    int d[kTile / TX];
#pragma unroll
    for (int j = 0; j < kTile / TX; ++j) d[j] = apart(pos[tx + TX * j], pos_q);
    look_up<kTile / TX>(a.bias, s.edges, d, bucket);
}

// Keys and values from x.kb + 64 j on -> a stage, zeros over hidden ones
template <int TX, bool kBias>
__device__ inline void load_keys(const AttnArgs &a, const SimtUnit &x, const SimtShape &f, float *stage, uint8_t *seen_s, int32_t *pos_s, int64_t j, const float *kp,
                                 const float *vp)
{
    const int64_t key = x.kb + j * kTile + threadIdx.x / (TX / 4);
    const bool seen = key < x.ke && (!a.mask || a.mask[key]);
    load_tile<TX / 4>(stage, f, seen ? kp + key * a.ldk + (int64_t)x.h * a.head_dim : nullptr, kp, a.head_dim);
    load_tile<TX / 4>(stage + kTile * f.ld, f, seen ? vp + key * a.ldv + (int64_t)x.h * a.head_dim : nullptr, kp, a.head_dim);
    if (threadIdx.x % (TX / 4) == 0) seen_s[threadIdx.x / (TX / 4)] = seen;
    if constexpr (kBias)
        if (threadIdx.x % (TX / 4) == 0) pos_s[threadIdx.x / (TX / 4)] = seen ? pos_of(a.bias.pos_k, key, x.rg.k0) : 0;
}

template <int TX, int C, int I, bool kBias>
__global__ void __launch_bounds__(16 * TX, blocks_of(TX, C, I))
attn_simt_fwd_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ SimtShape f, float *__restrict__ part_o, float2 *__restrict__ part_ml)
{
    constexpr int kRows = 16 * I, kPerRow = TX / I, J = kTile / TX;
    extern __shared__ __align__(16) float sm[];
    float *q_s = sm, *p_s = q_s + kRows * f.ld, *kv_s = p_s + kRows * kLdP;          // stage b: K and V at tiles 2 b, 2 b + 1
    __shared__ uint8_t seen_s[2][kTile];
    __shared__ int32_t pos_s[kBias ? 2 : 1][kTile];
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX, heads = a.kv_heads * a.group, lr = threadIdx.x / kPerRow;
    const Columns<TX> at(f, tx);
    const SimtUnit x = simt_unit(a, f);
    const float c1 = a.scale * kLog2e;
    const float *qp = static_cast<const float *>(a.q), *kp = static_cast<const float *>(a.k), *vp = static_cast<const float *>(a.v);
    const SimtBias bias = bias_of(sm, f.tile_floats, a);
    if constexpr (kBias) stage_bias(a, bias, x.h);
    for (int64_t t = x.t0; t * kRows < x.rows; t += f.tiles) {
        const int64_t r0 = t * kRows;
        __syncthreads();
        {
            int64_t row;
            int head;
            row_of(a, x, min(r0 + lr, x.rows - 1), row, head);
            load_tile<kPerRow>(q_s, f, r0 + lr < x.rows ? qp + row * a.ldq + (int64_t)head * a.head_dim : nullptr, qp, a.head_dim);
        }
        float o[I][C][4], m[I], l[I];
        int pos_q[I], own[I];                            // own: the row's table
        clear(o);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.f;
            if constexpr (kBias) place_row(a, x, r0 + ty + 16 * i, pos_q[i], own[i]);
        }
        turns(f, ceil_div(x.ke - x.kb, (int64_t)kTile), [&](int64_t j, int b) { load_keys<TX, kBias>(a, x, f, kv_s + 2 * b * kTile * f.ld, seen_s[b], pos_s[kBias ? b : 0], j, kp, vp); }, [&](int b) {
            const float *k_s = kv_s + 2 * b * kTile * f.ld, *v_s = k_s + kTile * f.ld;
            float s[I][J];
            scores<TX, I>(q_s, k_s, f.ld, a.head_dim, ty, tx, s);
            bool on[J];
#pragma unroll
            for (int j = 0; j < J; ++j) on[j] = seen_s[b][tx + TX * j];
#pragma unroll
            for (int i = 0; i < I; ++i) {
                float top = -INFINITY;
                int bucket[J];
                if constexpr (kBias) buckets_of<TX>(a, bias, pos_s[b], tx, pos_q[i], bucket);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    if constexpr (kBias) s[i][j] = on[j] ? fmaf(s[i][j], c1, bias.table[own[i] + bucket[j]]) : -INFINITY;
                    else s[i][j] = on[j] ? s[i][j] * c1 : -INFINITY;
                    top = fmaxf(top, s[i][j]);
                }
                top = fmaxf(m[i], row_max<TX>(top));
                const float base = top == -INFINITY ? 0.f : top, c = exp2_fast(m[i] - base);
                m[i] = top;
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const float p = exp2_fast(s[i][j] - base);
                    sum += p;
                    p_s[(ty + 16 * i) * kLdP + tx + TX * j] = p;
                }
                l[i] = l[i] * c + sum;
#pragma unroll
                for (int n = 0; n < C; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][n][e] *= c;
            }
            __syncwarp();                                // rows of p belong to one half-warp
            add_rows<C, I, TX>(o, p_s, v_s, f.ld, a.head_dim, ty, at);
            __syncwarp();
        });
        cp_async_wait_all();
        add_parts<TX, C>(o, f);
#pragma unroll
        for (int i = 0; i < I; ++i) l[i] = row_sum<TX>(l[i]);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int64_t r = r0 + ty + 16 * i;
            if (r >= x.rows) continue;
            int64_t row;
            int head;
            row_of(a, x, r, row, head);
            const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
            if (f.splits == 1) {
                store_columns<C, TX>(static_cast<float *>(a.out) + row * a.ldo + (int64_t)head * a.head_dim, o[i], inv, a.head_dim, at);
                if (a.lse && tx == 0) a.lse[row * heads + head] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * kLn2;
            } else {
                const int64_t p = ((int64_t)x.z * a.q_rows + row) * heads + head;
                store_columns<C, TX>(part_o + p * a.head_dim, o[i], inv, a.head_dim, at);
                if (tx == 0) part_ml[p] = make_float2(l[i] == 0.f ? -INFINITY : m[i], l[i]);
            }
        }
    }
}

template <int TX, int C, int I, bool kBias>
__global__ void __launch_bounds__(16 * TX, blocks_of(TX, C, I))
attn_simt_dq_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ SimtShape f, float *__restrict__ part_dq, float *__restrict__ dots,
                    float *__restrict__ table_part)
{
    constexpr int kRows = 16 * I, kPerRow = TX / I, J = kTile / TX;
    extern __shared__ __align__(16) float sm[];
    float *q_s = sm, *g_s = q_s + kRows * f.ld, *ds_s = g_s + kRows * f.ld, *kv_s = ds_s + kRows * kLdP;
    __shared__ uint8_t seen_s[2][kTile];
    __shared__ int32_t pos_s[kBias ? 2 : 1][kTile];
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX, heads = a.kv_heads * a.group, lr = threadIdx.x / kPerRow;
    const Columns<TX> at(f, tx);
    const SimtUnit x = simt_unit(a, f);
    const float c1 = a.scale * kLog2e;
    const float *qp = static_cast<const float *>(a.q), *kp = static_cast<const float *>(a.k), *vp = static_cast<const float *>(a.v);
    const float *gp = static_cast<const float *>(a.dout), *op = static_cast<const float *>(a.o);
    const SimtBias bias = bias_of(sm, f.tile_floats, a);
    float *mine_s = bias.bins + threadIdx.x;             // the thread's bins, 16 TX apart
    if constexpr (kBias) {
        stage_bias(a, bias, x.h);
        if (table_part)
            for (int i = 0; i < a.bias.buckets; ++i) mine_s[i * 16 * TX] = 0.f;
    }
    for (int64_t t = x.t0; t * kRows < x.rows; t += f.tiles) {
        const int64_t r0 = t * kRows;
        __syncthreads();
        {
            int64_t row;
            int head;
            row_of(a, x, min(r0 + lr, x.rows - 1), row, head);
            const bool on = r0 + lr < x.rows;
            load_tile<kPerRow>(q_s, f, on ? qp + row * a.ldq + (int64_t)head * a.head_dim : nullptr, qp, a.head_dim);
            load_tile<kPerRow>(g_s, f, on ? gp + row * a.ldg + (int64_t)head * a.head_dim : nullptr, qp, a.head_dim);
        }
        float dq[I][C][4], lse[I], d[I], mine = 0.f;
        int pos_q[I], own[I];
        if constexpr (kBias)
#pragma unroll
            for (int i = 0; i < I; ++i) place_row(a, x, r0 + ty + 16 * i, pos_q[i], own[i]);
        clear(dq);
        cp_async_wait_all();
        __syncthreads();
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int64_t r = r0 + ty + 16 * i;
            int64_t row;
            int head;
            row_of(a, x, min(r, x.rows - 1), row, head);
            lse[i] = INFINITY;
            if (r < x.rows) {
                const float v = a.lse[row * heads + head];
                if (v != -INFINITY) lse[i] = v * kLog2e;
            }
            if (tx == i && lse[i] != INFINITY) mine = dot_as_scores(g_s + (ty + 16 * i) * f.ld, op + row * a.ldo + (int64_t)head * a.head_dim, a.head_dim);
            if (tx == i && r < x.rows && x.z == 0) dots[row * heads + head] = mine;
        }
#pragma unroll
        for (int i = 0; i < I; ++i) d[i] = __shfl_sync(0xFFFFFFFFu, mine, i, TX);
        turns(f, ceil_div(x.ke - x.kb, (int64_t)kTile), [&](int64_t j, int b) { load_keys<TX, kBias>(a, x, f, kv_s + 2 * b * kTile * f.ld, seen_s[b], pos_s[kBias ? b : 0], j, kp, vp); }, [&](int b) {
            const float *k_s = kv_s + 2 * b * kTile * f.ld, *v_s = k_s + kTile * f.ld;
            float s[I][J], u[I][J];
            scores<TX, I>(q_s, k_s, f.ld, a.head_dim, ty, tx, s);
            scores<TX, I>(g_s, v_s, f.ld, a.head_dim, ty, tx, u);
            if constexpr (kBias) {
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    int bucket[J];
                    buckets_of<TX>(a, bias, pos_s[b], tx, pos_q[i], bucket);
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const float v = exp2_fast(fmaf(s[i][j], c1, bias.table[own[i] + bucket[j]] - lse[i])) * (u[i][j] - d[i]);
                        const float ds = seen_s[b][tx + TX * j] && lse[i] != INFINITY ? v : 0.f;
                        ds_s[(ty + 16 * i) * kLdP + tx + TX * j] = ds;
                        if (table_part) mine_s[bucket[j] * 16 * TX] += ds;
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const bool on = seen_s[b][tx + TX * j];
#pragma unroll
                    for (int i = 0; i < I; ++i)
                        ds_s[(ty + 16 * i) * kLdP + tx + TX * j] = on ? exp2_fast(fmaf(s[i][j], c1, -lse[i])) * (u[i][j] - d[i]) : 0.f;
                }
            }
            __syncwarp();
            add_rows<C, I, TX>(dq, ds_s, k_s, f.ld, a.head_dim, ty, at);
            __syncwarp();
        });
        add_parts<TX, C>(dq, f);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int64_t r = r0 + ty + 16 * i;
            if (r >= x.rows) continue;
            int64_t row;
            int head;
            row_of(a, x, r, row, head);
            const bool keep = lse[i] != INFINITY;        // a row that saw no key passes on nothing
            if (f.splits == 1) store_columns<C, TX>(static_cast<float *>(a.dq) + row * a.ldq2 + (int64_t)head * a.head_dim, dq[i], a.scale, a.head_dim, at, keep);
            else store_columns<C, TX>(part_dq + (((int64_t)x.z * a.q_rows + row) * heads + head) * a.head_dim, dq[i], a.scale, a.head_dim, at, keep);
        }
    }
    if constexpr (kBias)
        if (table_part) {                                // thread ty, tx has the head ty % group: lanes of one head by exchange, then the warps
            __syncthreads();
            constexpr int kWarps = 16 * TX / 32;
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nb = a.bias.buckets;
            const uint32_t u = blockIdx.x;
            const int64_t seq = u / (uint32_t)f.splits / (uint32_t)f.tiles / (uint32_t)a.kv_heads;
            float *part = table_part + ((seq * f.tiles + x.t0) * f.splits + x.z) * nb * heads + x.h * a.group;
            for (int k = warp; k < nb; k += kWarps) {
                for (int g0 = 0; g0 < a.group; g0 += 32 / TX) {
                    // a warp's lanes have the rows 32 / TX w + lane / TX of a step, of heads that follow one another
                    float v = 0.f;
                    for (int w = 0; w < kWarps; ++w) {
                        const int first = w * (32 / TX) % a.group;
                        if (a.group <= 32 / TX || first == g0) v += bias.bins[k * 16 * TX + w * 32 + lane];
                    }
                    const int stop = a.group <= 32 / TX ? TX * a.group : 32;
                    for (int o = 16; o >= stop; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
                    for (int o = TX / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
                    const int g = g0 + lane / TX;
                    if (lane % TX == 0 && lane < stop && g < a.group) part[k * heads + g] = v;
                }
            }
        }
}

template <int TX, int C, int I, bool kBias>
__global__ void __launch_bounds__(16 * TX, blocks_of(TX, C, I))
attn_simt_dkv_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ SimtShape f, const float *__restrict__ dots)
{
    constexpr int kRows = 16 * I, kPerRow = TX / I, J = kTile / TX;
    extern __shared__ __align__(16) float sm[];
    float *k_s = sm, *v_s = k_s + kTile * f.ld, *p_s = v_s + kTile * f.ld, *ds_s = p_s + kRows * kLdP, *qg_s = ds_s + kRows * kLdP;
    __shared__ float lse_s[2][kRows], dot_s[2][kRows];
    __shared__ int32_t pos_s[kBias ? 2 : 1][kRows], own_s[kBias ? 2 : 1][kRows], key_s[kTile];
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX, heads = a.kv_heads * a.group, lr = threadIdx.x / kPerRow;
    const Columns<TX> at(f, tx);
    const SimtUnit x = simt_unit(a, f);
    const float c1 = a.scale * kLog2e;
    const float *qp = static_cast<const float *>(a.q), *kp = static_cast<const float *>(a.k), *vp = static_cast<const float *>(a.v);
    const float *gp = static_cast<const float *>(a.dout);
    const SimtBias bias = bias_of(sm, f.tile_floats, a);
    if constexpr (kBias) stage_bias(a, bias, x.h);
    for (int64_t j0 = x.rg.k0 + (int64_t)x.t0 * kTile; j0 < x.rg.k1; j0 += (int64_t)f.tiles * kTile) {
        __syncthreads();
        {
            const int64_t key = j0 + threadIdx.x / (TX / 4);
            const bool seen = key < x.rg.k1 && (!a.mask || a.mask[key]);
            load_tile<TX / 4>(k_s, f, seen ? kp + key * a.ldk + (int64_t)x.h * a.head_dim : nullptr, kp, a.head_dim);
            load_tile<TX / 4>(v_s, f, seen ? vp + key * a.ldv + (int64_t)x.h * a.head_dim : nullptr, kp, a.head_dim);
            if constexpr (kBias)
                if (threadIdx.x % (TX / 4) == 0) key_s[threadIdx.x / (TX / 4)] = seen ? pos_of(a.bias.pos_k, key, x.rg.k0) : 0;
        }
        float dk[4][C][4], dv[4][C][4];
        clear(dk);
        clear(dv);
        turns(f, ceil_div(x.rows, (int64_t)kRows), [&](int64_t j, int b) {
            const int64_t r = j * kRows + lr;
            float *q_s = qg_s + 2 * b * kRows * f.ld, *g_s = q_s + kRows * f.ld;
            int64_t row;
            int head;
            row_of(a, x, min(r, x.rows - 1), row, head);
            float l = INFINITY;
            if (r < x.rows) {
                const float v = a.lse[row * heads + head];
                if (v != -INFINITY) l = v * kLog2e;
            }
            if (threadIdx.x % kPerRow == 0) {
                lse_s[b][lr] = l;
                dot_s[b][lr] = l != INFINITY ? dots[row * heads + head] : 0.f;
                if constexpr (kBias) place_row(a, x, r, pos_s[b][lr], own_s[b][lr]);
            }
            load_tile<kPerRow>(q_s, f, l != INFINITY ? qp + row * a.ldq + (int64_t)head * a.head_dim : nullptr, kp, a.head_dim);
            load_tile<kPerRow>(g_s, f, l != INFINITY ? gp + row * a.ldg + (int64_t)head * a.head_dim : nullptr, kp, a.head_dim);
        }, [&](int b) {
            const float *q_s = qg_s + 2 * b * kRows * f.ld, *g_s = q_s + kRows * f.ld;
            float s[I][J], u[I][J];
            scores<TX, I>(q_s, k_s, f.ld, a.head_dim, ty, tx, s);
            scores<TX, I>(g_s, v_s, f.ld, a.head_dim, ty, tx, u);
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const float lse = lse_s[b][ty + 16 * i], d = dot_s[b][ty + 16 * i];
                int bucket[J], own = 0;
                if constexpr (kBias) {
                    buckets_of<TX>(a, bias, key_s, tx, pos_s[b][ty + 16 * i], bucket);
                    own = own_s[b][ty + 16 * i];
                }
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    float add = -lse;
                    if constexpr (kBias) add += bias.table[own + bucket[j]];
                    const float p = exp2_fast(fmaf(s[i][j], c1, add));
                    p_s[(ty + 16 * i) * kLdP + tx + TX * j] = p;
                    ds_s[(ty + 16 * i) * kLdP + tx + TX * j] = p * (u[i][j] - d);
                }
            }
            __syncthreads();
            add_columns<C, I, TX>(dv, p_s, g_s, f.ld, a.head_dim, ty, at);
            add_columns<C, I, TX>(dk, ds_s, q_s, f.ld, a.head_dim, ty, at);
        });
        cp_async_wait_all();
        add_parts<TX, C>(dk, f);
        add_parts<TX, C>(dv, f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t key = j0 + 4 * ty + i;
            if (key >= x.rg.k1) continue;
            const bool keep = !a.mask || a.mask[key];
            store_columns<C, TX>(static_cast<float *>(a.dk) + key * a.ldk2 + (int64_t)x.h * a.head_dim, dk[i], a.scale, a.head_dim, at, keep);
            store_columns<C, TX>(static_cast<float *>(a.dv) + key * a.ldv2 + (int64_t)x.h * a.head_dim, dv[i], 1.f, a.head_dim, at, keep);
        }
    }
}

constexpr int kMaxDevices = 64, kMostSmem = 224 * 1024, kSmSmem = 228 * 1024;
template <typename Kernel> bool allow_smem(Kernel kernel, std::atomic<bool> (&done)[kMaxDevices])
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return false;
    if (done[dev]) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem) != cudaSuccess) return false;
    done[dev] = true;
    return true;
}

// kept: floats of shared memory that stay; pair: those of one stage.  Two stages where they leave room for `blocks` blocks per SM.
// bins: threads that have bins of their own.
SimtShape shape_of(const AttnArgs &a, int64_t tiles, int splits, int kept_rows, int pair_rows, int p_rows, int TX, int blocks, int bins, size_t &smem)
{
    SimtShape f{};
    f.ld = (a.head_dim / 4 | 1) * 4;                 // an odd number of 16-byte units
    f.tiles = (int)tiles;
    f.splits = splits;
    f.cols = TX;
    while (f.cols > 1 && f.cols * 2 >= a.head_dim) f.cols /= 2;
    const size_t fixed = ((size_t)kept_rows * f.ld + (size_t)p_rows * kLdP) * sizeof(float), pair = (size_t)pair_rows * f.ld * sizeof(float);
    const size_t beside = a.bias.buckets ? ((size_t)kMaxBuckets + (size_t)a.bias.buckets * (a.group + bins)) * sizeof(float) : 0;
    const size_t two = fixed + 2 * pair + beside;
    f.stages = (two + 2048) * blocks <= (size_t)kSmSmem && two <= (size_t)kMostSmem ? 2 : 1;
    f.tile_floats = (int)((fixed + f.stages * pair) / sizeof(float));
    smem = fixed + f.stages * pair + beside;
    return f;
}

template <int TX, int C, int I, bool kBias> bool launch_fwd(const AttnArgs &a, const SimtPlan &p, float *part_o, float2 *part_ml, cudaStream_t st)
{
    static std::atomic<bool> done[kMaxDevices] = {};
    if (!allow_smem(attn_simt_fwd_kernel<TX, C, I, kBias>, done)) return false;
    size_t smem;
    const SimtShape f = shape_of(a, p.q_tiles, p.splits, 16 * I, 2 * kTile, 16 * I, TX, blocks_of(TX, C, I), 0, smem);
    note_launch();
    attn_simt_fwd_kernel<TX, C, I, kBias><<<(unsigned)(a.n_seq * a.kv_heads * p.q_tiles * p.splits), 16 * TX, smem, st>>>(a, f, part_o, part_ml);
    return true;
}

template <int TX, int C, int I, bool kBias>
bool launch_bwd(const AttnArgs &a, const SimtPlan &p, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    static std::atomic<bool> done[2][kMaxDevices] = {};
    if (!allow_smem(attn_simt_dq_kernel<TX, C, I, kBias>, done[0]) || !allow_smem(attn_simt_dkv_kernel<TX, C, I, kBias>, done[1])) return false;
    size_t smem;
    if (a.q_rows) {
        const SimtShape f = shape_of(a, p.q_tiles, p.splits, 2 * 16 * I, 2 * kTile, 16 * I, TX, blocks_of(TX, C, I), table_part ? 16 * TX : 0, smem);
        note_launch();
        attn_simt_dq_kernel<TX, C, I, kBias><<<(unsigned)(a.n_seq * a.kv_heads * p.q_tiles * p.splits), 16 * TX, smem, st>>>(a, f, part_dq, dots, table_part);
    }
    if (a.k_rows) {
        const SimtShape f = shape_of(a, p.k_tiles, 1, 2 * kTile, 2 * 16 * I, 2 * 16 * I, TX, blocks_of(TX, C, I), 0, smem);
        note_launch();
        attn_simt_dkv_kernel<TX, C, I, kBias><<<(unsigned)(a.n_seq * a.kv_heads * p.k_tiles), 16 * TX, smem, st>>>(a, f, dots);
    }
    return true;
}

template <int TX, int C, int I> bool forward_of(const AttnArgs &a, const SimtPlan &p, float *part_o, float2 *part_ml, cudaStream_t st)
{
    return a.bias.table ? launch_fwd<TX, C, I, true>(a, p, part_o, part_ml, st) : launch_fwd<TX, C, I, false>(a, p, part_o, part_ml, st);
}
template <int TX, int C, int I>
bool backward_of(const AttnArgs &a, const SimtPlan &p, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    return a.bias.table ? launch_bwd<TX, C, I, true>(a, p, part_dq, dots, table_part, st) : launch_bwd<TX, C, I, false>(a, p, part_dq, dots, nullptr, st);
}

}  // namespace

SimtPlan simt_plan(const AttnArgs &a, const Lengths &q, const Lengths &k)
{
    SimtPlan p{};
    const int64_t units = std::max<int64_t>(a.n_seq * a.kv_heads, 1), most = (((int64_t)1 << 31) - 1) / units, rows = q.typical * a.group;
    p.rows = rows <= 16 ? 16 : (rows <= 32 ? 32 : 64);
    p.q_tiles = blocks_per_unit(q, a.group, p.rows, units);
    p.k_tiles = blocks_per_unit(k, 1, kTile, units);
    p.splits = 1;
    if (units * p.q_tiles < 296)
        p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({296 / (units * p.q_tiles), k.longest / (2 * kTile), kMaxSplits, most / p.q_tiles}));
    return p;
}

// heads of up to 32, 64, 128 columns, with 8 or 16 threads side by side
template <int I, int TX> static bool forward_wide(const AttnArgs &a, const SimtPlan &p, float *part_o, float2 *part_ml, cudaStream_t st)
{
    if (a.head_dim > 64) return forward_of<16, 2, I>(a, p, part_o, part_ml, st);
    if (a.head_dim > 32) return forward_of<TX, 64 / (4 * TX), I>(a, p, part_o, part_ml, st);
    return forward_of<8, 1, I>(a, p, part_o, part_ml, st);
}

template <int I, int TX> static bool backward_wide(const AttnArgs &a, const SimtPlan &p, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    if (a.head_dim > 64) return backward_of<16, 2, I>(a, p, part_dq, dots, table_part, st);
    if constexpr (TX == 8)
        if (a.head_dim <= 32) return backward_of<8, 1, I>(a, p, part_dq, dots, table_part, st);
    return backward_of<TX, 64 / (4 * TX), I>(a, p, part_dq, dots, table_part, st);
}

// The bins of all threads fit beside one stage of tiles
bool simt_forms_table(const AttnArgs &a, const SimtPlan &p)
{
    const int TX = a.head_dim > 64 || p.rows == 64 ? 16 : 8;
    size_t smem;
    shape_of(a, 1, 1, 2 * p.rows, 2 * kTile, p.rows, TX, 1 << 20, 16 * TX, smem);       // (one stage where two leave no room for that many blocks)
    return 16 % a.group == 0 && smem <= (size_t)kMostSmem;
}

bool simt_attention_forward(const AttnArgs &a, const SimtPlan &p, float *part_o, float2 *part_ml, cudaStream_t st)
{
    if (p.rows == 16) return forward_wide<1, 8>(a, p, part_o, part_ml, st);
    return p.rows == 32 ? forward_wide<2, 8>(a, p, part_o, part_ml, st) : forward_wide<4, 16>(a, p, part_o, part_ml, st);
}

bool simt_attention_backward(const AttnArgs &a, const SimtPlan &p, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    if (p.rows == 16) return backward_wide<1, 8>(a, p, part_dq, dots, table_part, st);
    return p.rows == 32 ? backward_wide<2, 8>(a, p, part_dq, dots, table_part, st) : backward_wide<4, 16>(a, p, part_dq, dots, table_part, st);
}

}  // namespace e2egrec
