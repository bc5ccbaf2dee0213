// Gradients of attention with a bias by distance where there are many rows, bf16 heads up to 128, by matrix products of a warp
// (mma.sync, 16 x 8 x 16).
//
// A warp holds 16 rows of a product, so a row's scores, p and dS are in the registers of four threads: a score's bucket, its bias and the table's
// gradient are ordinary arithmetic on registers.  Two kernels, no atomics: dQ, D and the table's gradient go over the keys of a block of rows, dK
// and dV over the rows of a block of keys; both form the scores anew.  Tiles of 64 keys (rows) come by cp.async, the next one beside the products
// of this one; rows in shared memory are an odd number of 16-byte units apart, so that ldmatrix meets no bank twice.
//
// D = sum p dP / sum p over the keys, from a pass over them before the one that forms dS (one tile: from the products at hand), about the stored
// out's value as origin: the table's gradient is what is left of dS that cancels, and D of the stored out alone is off by out's rounding.  A row
// whose p is all one key's gets dS = 0 exactly.  dS of dQ goes into its product as two bf16 operands, its rounding and the rest.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "attention.cuh"
#include "tcgen05.cuh"

namespace e2egrec {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kStep = 64;                            // keys (rows) of a tile that a block goes over
constexpr int kMostWarps = 8;
constexpr int kNear = 2048;                          // buckets of the distances -kNear .. kNear - 1 lie in a table
constexpr int kMeta = 4;                             // tiles whose positions are kept: this one's, the next, which is copied, and the one after

// Where things lie in shared memory (bytes); a row of a tile takes 32 KS + 16
struct MmaShape {
    int warps, tiles;                                // 16 rows (keys) per warp; blocks per sequence and key head
    int slots;                                       // bins of a thread: its two rows' heads are one (1) or two (2)
    uint32_t stages, near, table, sums, bins, rows;
    uint32_t total;
};

__device__ inline float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ inline uint32_t pack(float lo, float hi)
{
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&h);
}
__device__ inline void ldsm(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ inline void ldsm_t(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ inline void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Addresses of a lane in a tile of pitch P: of 16 x 16 as the left operand (also, transposed, as the right one whose rows are the sum's index), and
// as the right operand whose columns are rows of the tile
template <int KS> struct Lane {
    static constexpr uint32_t kPitch = KS * 32 + 16;
    uint32_t left, right;
    __device__ inline explicit Lane(int lane)
        : left((lane & 15) * kPitch + (lane >> 4) * 16), right(((lane & 7) + ((lane >> 4) << 3)) * kPitch + ((lane >> 3) & 1) * 16)
    {
    }
};

// acc (16 x 8 N) = rows at `a` (16) times the rows at `b` (8 N), over the head
template <int KS, int N> __device__ inline void products(float (&acc)[N][4], uint32_t a, uint32_t b)
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        uint32_t x[4];
        ldsm(a + k * 32, x);
#pragma unroll
        for (int n = 0; n < N; n += 2) {
            uint32_t y[4];
            ldsm(b + n * 8 * Lane<KS>::kPitch + k * 32, y);
            mma(acc[n], x, y[0], y[1]);
            mma(acc[n + 1], x, y[2], y[3]);
        }
    }
}
// 16 x 16 of an accumulator (two of its 8 columns) as a left operand
__device__ inline void as_left(const float (&c0)[4], const float (&c1)[4], uint32_t (&x)[4])
{
    x[0] = pack(c0[0], c0[1]);
    x[1] = pack(c0[2], c0[3]);
    x[2] = pack(c1[0], c1[1]);
    x[3] = pack(c1[2], c1[3]);
}
// what the rounding of c to bf16 leaves out
__device__ inline void less(float (&c)[4], uint32_t lo, uint32_t hi)
{
    c[0] -= __uint_as_float(lo << 16);
    c[1] -= __uint_as_float(lo & 0xFFFF0000u);
    c[2] -= __uint_as_float(hi << 16);
    c[3] -= __uint_as_float(hi & 0xFFFF0000u);
}

// Rows of a tile -> shared memory; src(r): row r, or null for zeros
template <int KS, typename Src> __device__ inline void load_tile(uint32_t dst, int rows, int head_dim, const void *any, Src src)
{
    constexpr int kUnits = 2 * KS;
    for (int i = threadIdx.x; i < rows * kUnits; i += blockDim.x) {
        const int r = i / kUnits, u = i - r * kUnits;
        const bf16 *p = u * 8 < head_dim ? src(r) : nullptr;
        cp_async16(dst + r * Lane<KS>::kPitch + u * 16, p ? static_cast<const void *>(p + u * 8) : any, p != nullptr);
    }
}
// The same of rows `ld` apart from `first` on; on(r): not zeros.  Where a block holds whole rows of units a thread keeps to one of them.
template <int KS, typename On> __device__ inline void load_rows(uint32_t dst, int rows, int head_dim, const bf16 *first, int64_t ld, On on)
{
    constexpr int kUnits = 2 * KS;
    if constexpr ((kUnits & (kUnits - 1)) == 0) {
        const int u = threadIdx.x % kUnits, r0 = threadIdx.x / kUnits, per = blockDim.x / kUnits;
        const bf16 *p = first + r0 * ld + u * 8;
        const bool in = u * 8 < head_dim;
        dst += r0 * Lane<KS>::kPitch + u * 16;
        for (int r = r0; r < rows; r += per, p += per * ld, dst += per * Lane<KS>::kPitch) {
            const bool take = in && on(r);
            cp_async16(dst, take ? p : first, take);
        }
    } else {
        load_tile<KS>(dst, rows, head_dim, first, [&](int r) { return on(r) ? first + r * ld : nullptr; });
    }
}
__device__ inline void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ inline void landed() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---- bias
struct MmaBias {
    uint8_t near[2 * kNear];
    int32_t edges[kMaxBuckets];                      // beyond the last: the highest number
};
// table: [heads of the group x buckets], in powers of two
__device__ inline void stage_bias(const AttnArgs &a, MmaBias &s, float *table, int h)
{
    const int nb = a.bias.buckets, heads = a.kv_heads * a.group;
    for (int i = threadIdx.x; i < kMaxBuckets; i += blockDim.x) s.edges[i] = i < nb - 1 ? __ldg(a.bias.edges + i) : INT32_MAX;
    for (int i = threadIdx.x; i < nb * a.group; i += blockDim.x) table[i] = bias_at(a.bias, heads, i % nb, h * a.group + i / nb);
    __syncthreads();
    // neighbouring distances by a thread: the bucket of the first, then the edges that follow (2000 x 32 x 100, a bisection each: 1833 us, 1625 so)
    const int per = 2 * kNear / blockDim.x;
    int d = (int)threadIdx.x * per - kNear, at = bucket_of(a.bias, s.edges, d);
    for (int i = 0; i < per; i += 4) {
        uint32_t four = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k, ++d) {
            while (at < nb - 1 && s.edges[at] <= d) ++at;
            four |= (uint32_t)at << (8 * k);
        }
        reinterpret_cast<uint32_t *>(s.near)[((int)threadIdx.x * per + i) / 4] = four;
    }
    __syncthreads();
}
__device__ inline int bucket_fast(const BiasArgs &b, const MmaBias &s, int d)
{
    const uint32_t u = (uint32_t)d + kNear;
    return u < 2u * kNear ? s.near[u] : bucket_of(b, s.edges, d);
}

// How a warp finds the buckets of a tile's scores: from the lowest and the highest distance that a thread's two rows (of the product: queries, or
// keys) meet there.  One bucket for each; one edge, or up to three, as positions that the columns' are compared with; a table of near distances;
// bisection.  kKey: the rows are keys, the columns' positions are the queries'.
enum : int { kOne, kTwo, kFew, kTable, kAny };
__device__ inline int add_sat(int x, int y)
{
    int s;
    asm("add.sat.s32 %0, %1, %2;" : "=r"(s) : "r"(x), "r"(y));
    return s;
}
template <bool kKey> struct Ways {
    int lo[2], hi[2], limit[2][3], way;                  // limit: where a bucket begins (kKey: ends)
    __device__ static inline int distance(int row, int column) { return kKey ? apart(row, column) : apart(column, row); }
    // low, high: positions of the columns that count; low > high: there are none
    __device__ inline void find(const BiasArgs &b, const MmaBias &s, int low, int high, const int (&pos)[2])
    {
        int span = 0;
        bool close = true;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            lo[r] = hi[r] = 0;
            if (low <= high) {
                const int first = distance(pos[r], kKey ? high : low), last = distance(pos[r], kKey ? low : high);
                lo[r] = bucket_fast(b, s, first);
                hi[r] = max(bucket_fast(b, s, last), lo[r]);           // (edges out of order)
                close = close && first >= -kNear && last < kNear;
            }
            span = max(span, hi[r] - lo[r]);
        }
        span = __reduce_max_sync(0xFFFFFFFFu, span);
        way = span == 0 ? kOne : span == 1 ? kTwo : span <= 3 ? kFew : __all_sync(0xFFFFFFFFu, close) ? kTable : kAny;
        if (way == kTwo || way == kFew)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int k = 0; k < 3; ++k) {            // (an edge that some column has reached lies where it can be compared with)
                    const int e = s.edges[min(lo[r] + k, kMaxBuckets - 1)];
                    limit[r][k] = lo[r] + k >= hi[r] ? (kKey ? INT32_MIN : INT32_MAX) : kKey ? apart(pos[r], e) : add_sat(pos[r], e);
                }
    }
    __device__ static inline bool beyond(int limit, int p) { return kKey ? p <= limit : p >= limit; }
    // bucket of a column at p of row r at pos
    template <int WAY> __device__ inline int of(const BiasArgs &b, const MmaBias &s, int r, int pos, int p) const
    {
        if constexpr (WAY == kTwo) return beyond(limit[r][0], p) ? hi[r] : lo[r];
        if constexpr (WAY == kFew) return min(lo[r] + beyond(limit[r][0], p) + beyond(limit[r][1], p) + beyond(limit[r][2], p), hi[r]);
        if constexpr (WAY == kTable) return s.near[min((kKey ? (uint32_t)pos - (uint32_t)p : (uint32_t)p - (uint32_t)pos) + kNear, 2u * kNear - 1)];
        if constexpr (WAY == kAny) return bucket_of(b, s.edges, distance(pos, p));
        return lo[r];
    }
};
template <int W> using Way = std::integral_constant<int, W>;
template <typename F> __device__ inline void by_way(int way, F f)
{
    if (way == kOne) f(Way<kOne>());
    else if (way == kTwo) f(Way<kTwo>());
    else if (way == kFew) f(Way<kFew>());
    else if (way == kTable) f(Way<kTable>());
    else f(Way<kAny>());
}
__device__ inline float2 pair(float x, float y) { return make_float2(x, y); }

struct MmaUnit {
    SeqRange rg;
    int64_t rows, seq;
    int h, t0;
};
__device__ inline MmaUnit mma_unit(const AttnArgs &a, const MmaShape &f, bool report)
{
    MmaUnit x;
    uint32_t u = blockIdx.x;
    x.t0 = (int)(u % (uint32_t)f.tiles);
    u /= (uint32_t)f.tiles;
    x.seq = u / (uint32_t)a.kv_heads;
    x.h = (int)(u % (uint32_t)a.kv_heads);
    x.rg = seq_range(a, x.seq, report && threadIdx.x == 0 && x.t0 == 0 && x.h == 0);
    x.rows = (x.rg.q1 - x.rg.q0) * a.group;
    return x;
}
// query (of the sequence) and head (of the group) of row r
__device__ inline void row_of(const AttnArgs &a, int64_t r, int64_t &i, int &g)
{
    i = a.group == 1 ? r : (r >> 32 ? r / a.group : (int64_t)((uint32_t)r / (uint32_t)a.group));
    g = (int)(r - i * a.group);
}

// 8 columns each of two accumulator rows -> out, rounded
__device__ inline void store_pair(bf16 *row, int col, int head_dim, float x, float y, float scale, bool keep)
{
    if (col >= head_dim) return;
    *reinterpret_cast<uint32_t *>(row + col) = keep ? pack(x * scale, y * scale) : 0u;
}

// ---- dQ, D (dots) and whether a row's p is not one key's alone (some), and the gradient of the table.  A thread has bins of its own in shared memory,
// [slots x buckets x lanes] per warp; dS of a bucket that the thread stays in is added up in a register.  At the end of a block of rows lanes of one
// row, then rows of one head are added up, in order.  The training case (8 x up to 2048 x 2048, 8 heads of 128): 1.52 ms, the kernel below 1.04 ms; what
// bounds both is the latency of their instructions with two warps per scheduler (tensor pipe 20 and 29 %, reads of shared memory 33 and 56 %).
// Two blocks of 8 warps per SM where heads take up to 64 columns: 1000 x 20 x 60, 8 heads of 32, backward 941 -> 670 us, of 64 2000 x 32 x 100
// 1625 -> 1518.  Lanes of one head joined by exchange instead of row by row: 670 -> 433, 1518 -> 1129.
template <int KS>
__global__ void __launch_bounds__(32 * kMostWarps, KS <= 4 ? 2 : 1)
attn_mma_dq_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ MmaShape f, float *__restrict__ dots, float *__restrict__ some,
                   float *__restrict__ table_part)
{
    constexpr uint32_t kPitch = Lane<KS>::kPitch, kTileBytes = kStep * kPitch;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ __align__(16) int32_t pos_s[kMeta][kStep];
    __shared__ uint32_t seen_s[kMeta][2];
    __shared__ int2 range_s[kMeta][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane >> 2, t4 = lane & 3, heads = a.kv_heads * a.group, nb = a.bias.buckets;
    const uint32_t base = smem_u32(smem), rows_bytes = 16 * f.warps * kPitch;
    MmaBias &bias = *reinterpret_cast<MmaBias *>(smem + f.near);
    const float *table = reinterpret_cast<const float *>(smem + f.table);
    float *sums = reinterpret_cast<float *>(smem + f.sums), *bins = reinterpret_cast<float *>(smem + f.bins) + warp * f.slots * nb * 32 + lane;
    float *rows_s = reinterpret_cast<float *>(smem + f.rows) + warp * 16 * f.warps;
    const MmaUnit x = mma_unit(a, f, true);
    const Lane<KS> at(lane);
    const float c1 = a.scale * kLog2e;
    const bf16 *kp = static_cast<const bf16 *>(a.k) + (int64_t)x.h * a.head_dim, *vp = static_cast<const bf16 *>(a.v) + (int64_t)x.h * a.head_dim;
    const int64_t keys = x.rg.k1 - x.rg.k0;
    const int n = (int)ceil_div(keys, (int64_t)kStep), steps = n > 1 ? 2 * n : n;
    if (x.t0 * 16ll * f.warps < x.rows) stage_bias(a, bias, reinterpret_cast<float *>(smem + f.table), x.h);
    if (table_part) {
        for (int i = threadIdx.x; i < nb * a.group; i += blockDim.x) sums[i] = 0.f;
        for (int i = 0; i < f.slots * nb; ++i) bins[i * 32] = 0.f;
    }
    // positions of a tile of keys, 32 by a warp: fetched, and written
    int pos_n[2];
    uint32_t seen_n[2];
    auto fetch = [&](int tile) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if ((b & (f.warps - 1)) != warp) continue;
            const int64_t key = x.rg.k0 + (int64_t)tile * kStep + b * 32 + lane;
            seen_n[b] = key < x.rg.k1 ? (a.mask ? a.mask[key] : 1u) : 0u;
            pos_n[b] = key < x.rg.k1 ? pos_of(a.bias.pos_k, key, x.rg.k0) : 0;
        }
    };
    auto put = [&](int slot) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if ((b & (f.warps - 1)) != warp) continue;
            const bool on = seen_n[b] != 0;
            const uint32_t word = __ballot_sync(0xFFFFFFFFu, on);
            const int first = __reduce_min_sync(0xFFFFFFFFu, on ? pos_n[b] : INT32_MAX), last = __reduce_max_sync(0xFFFFFFFFu, on ? pos_n[b] : INT32_MIN);
            pos_s[slot][b * 32 + lane] = pos_n[b];
            if (lane == 0) {
                seen_s[slot][b] = word;
                range_s[slot][b] = make_int2(first, last);
            }
        }
    };
    auto copy = [&](int tile, int step) {
        const uint32_t dst = base + f.stages + (step & 1) * 2 * kTileBytes;
        const uint32_t w0 = seen_s[step % kMeta][0], w1 = seen_s[step % kMeta][1];
        const int64_t key0 = x.rg.k0 + (int64_t)tile * kStep;
        auto on = [&](int r) { return (r < 32 ? w0 >> r : w1 >> (r - 32)) & 1u; };
        load_rows<KS>(dst, kStep, a.head_dim, kp + key0 * a.ldk, a.ldk, on);
        load_rows<KS>(dst + kTileBytes, kStep, a.head_dim, vp + key0 * a.ldv, a.ldv, on);
        commit();
    };
    for (int64_t t = x.t0; t * 16 * f.warps < x.rows; t += f.tiles) {
        const int64_t r0 = t * 16 * f.warps;
        __syncthreads();
        auto row_at = [&](const void *p, int64_t ld, int r) -> const bf16 * {
            if (r0 + r >= x.rows) return nullptr;
            int64_t i;
            int g;
            row_of(a, r0 + r, i, g);
            const int64_t row = x.rg.q0 + i;
            const int head = x.h * a.group + g;
            return a.lse[row * heads + head] == -INFINITY ? nullptr : static_cast<const bf16 *>(p) + row * ld + (int64_t)head * a.head_dim;
        };
        load_tile<KS>(base, 16 * f.warps, a.head_dim, a.q, [&](int r) { return row_at(a.q, a.ldq, r); });
        load_tile<KS>(base + rows_bytes, 16 * f.warps, a.head_dim, a.q, [&](int r) { return row_at(a.dout, a.ldg, r); });
        commit();
        if (n > 0) {
            fetch(0);
            put(0);
            if (steps > 1) {
                fetch(1 % n);
                put(1);
            }
            __syncthreads();
            copy(0, 0);
        }
        // the thread's two rows
        float lse[2], ref[2], d[2], total[2], lack[2], run[2];
        int pos[2], own[2], cur[2], count[2];                // count: keys whose p is not 0
        bool alone[2], special = true;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int64_t rr = r0 + warp * 16 + quad + 8 * r;
            int64_t i;
            int g;
            row_of(a, min(rr, x.rows - 1), i, g);
            const int64_t row = x.rg.q0 + i;
            const int head = x.h * a.group + g;
            const float l = rr < x.rows ? a.lse[row * heads + head] : -INFINITY;
            lse[r] = l == -INFINITY ? INFINITY : l * kLog2e;
            pos[r] = pos_of(a.bias.pos_q, row, x.rg.q0);
            own[r] = g * nb;
            float s = 0.f;
            if (l != -INFINITY) {
                const bf16 *o = static_cast<const bf16 *>(a.o) + row * a.ldo + (int64_t)head * a.head_dim;
                const bf16 *dout = static_cast<const bf16 *>(a.dout) + row * a.ldg + (int64_t)head * a.head_dim;
                for (int e = t4 * 8; e < a.head_dim; e += 32) {
                    float p[8], q[8];
                    Chunk<bf16>::load(o + e, p);
                    Chunk<bf16>::load(dout + e, q);
#pragma unroll
                    for (int k = 0; k < 8; ++k) s = fmaf(p[k], q[k], s);
                }
            }
            s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
            s += __shfl_xor_sync(0xFFFFFFFFu, s, 2);
            ref[r] = s;
            d[r] = total[r] = lack[r] = run[r] = 0.f;
            cur[r] = count[r] = 0;
            alone[r] = true;
        }
        float dq[2 * KS][4];
#pragma unroll
        for (int c = 0; c < 2 * KS; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) dq[c][i] = 0.f;
        for (int step = 0, tile = 0; step < steps; ++step, tile = tile + 1 < n ? tile + 1 : 0) {
            const int next = tile + 1 < n ? tile + 1 : 0, slot = step % kMeta;
            if (step + 1 < steps) {
                copy(next, step + 1);
                landed<1>();
            } else {
                landed<0>();
            }
            const bool more = step + 2 < steps;
            if (more) fetch(next + 1 < n ? next + 1 : 0);
            __syncthreads();
            const uint32_t k_at = base + f.stages + (step & 1) * 2 * kTileBytes, v_at = k_at + kTileBytes;
            const uint64_t word = (uint64_t)seen_s[slot][1] << 32 | seen_s[slot][0];
            const bool last_pass = step + n >= steps;
            Ways<false> ways;
            {
                const int2 p0 = range_s[slot][0], p1 = range_s[slot][1];
                ways.find(a.bias, bias, min(p0.x, p1.x), max(p0.y, p1.y), pos);
            }
            float p[8][4], ds[8][4];
            const int *columns = &pos_s[slot][t4 * 2];
            products<KS, 8>(p, base + warp * 16 * kPitch + at.left, k_at + at.right);
            by_way(ways.way, [&](auto way) {
                constexpr int WAY = decltype(way)::value;
                // biases of the buckets lo .. lo + 3 (or hi), less lse
                constexpr int kValues = WAY == kOne ? 1 : WAY == kTwo ? 2 : WAY == kFew ? 4 : 0;
                float value[2][kValues + 1];
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int k = 0; k < kValues; ++k) value[r][k] = table[own[r] + min(ways.lo[r] + k, ways.hi[r])] - lse[r];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    int2 at2 = make_int2(0, 0);
                    if constexpr (WAY != kOne) at2 = *reinterpret_cast<const int2 *>(columns + c * 8);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float add[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int at1 = e ? at2.y : at2.x;
                            if constexpr (WAY == kOne) add[e] = value[r][0];
                            else if constexpr (WAY == kTwo) add[e] = at1 >= ways.limit[r][0] ? value[r][1] : value[r][0];
                            else if constexpr (WAY == kFew)
                                add[e] = at1 >= ways.limit[r][2] ? value[r][3] : at1 >= ways.limit[r][1] ? value[r][2] : at1 >= ways.limit[r][0] ? value[r][1] : value[r][0];
                            else add[e] = table[own[r] + ways.template of<WAY>(a.bias, bias, r, pos[r], at1)] - lse[r];
                        }
                        const float2 y = __ffma2_rn(pair(p[c][2 * r], p[c][2 * r + 1]), pair(c1, c1), pair(add[0], add[1]));
                        p[c][2 * r] = exp2_fast(y.x);
                        p[c][2 * r + 1] = exp2_fast(y.y);
                    }
                }
            });
            const uint64_t mine = word >> (t4 * 2);      // the thread's columns: bits 8 c and 8 c + 1
            auto hide = [&](float (&v)[8][4]) {
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint32_t w = (uint32_t)(c < 4 ? mine : mine >> 32) >> (c % 4 * 8);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(w & (1u << (i & 1)))) v[c][i] = 0.f;
                }
            };
            if (word != ~0ull) hide(p);
            products<KS, 8>(ds, base + rows_bytes + warp * 16 * kPitch + at.left, v_at + at.right);
            if (!last_pass || n == 1) {                  // D
                float2 sum[2] = {}, less2[2] = {};
#pragma unroll
                for (int c = 0; c < 8; ++c)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float2 w = pair(p[c][2 * r], p[c][2 * r + 1]);
                        sum[r] = __fadd2_rn(sum[r], w);
                        less2[r] = __ffma2_rn(w, __fadd2_rn(pair(ds[c][2 * r], ds[c][2 * r + 1]), pair(-ref[r], -ref[r])), less2[r]);
                        count[r] += (w.x != 0.f) + (w.y != 0.f);
                    }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    total[r] += sum[r].x + sum[r].y;
                    lack[r] += less2[r].x + less2[r].y;
                }
                if (step + 1 == n) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
#pragma unroll
                        for (int o = 1; o < 4; o <<= 1) {
                            total[r] += __shfl_xor_sync(0xFFFFFFFFu, total[r], o);
                            lack[r] += __shfl_xor_sync(0xFFFFFFFFu, lack[r], o);
                            count[r] += __shfl_xor_sync(0xFFFFFFFFu, count[r], o);
                        }
                        d[r] = total[r] == 0.f ? 0.f : ref[r] + lack[r] / total[r];
                        alone[r] = count[r] <= 1;
                    }
                    // rows without dS, or with a D that is no number: looked at score by score
                    special = __any_sync(0xFFFFFFFFu, alone[0] || alone[1] || !(fabsf(d[0]) < INFINITY) || !(fabsf(d[1]) < INFINITY));
                }
            }
            if (last_pass) {
#pragma unroll
                for (int c = 0; c < 8; ++c)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float2 y = __fmul2_rn(pair(p[c][2 * r], p[c][2 * r + 1]), __fadd2_rn(pair(ds[c][2 * r], ds[c][2 * r + 1]), pair(-d[r], -d[r])));
                        ds[c][2 * r] = y.x;
                        ds[c][2 * r + 1] = y.y;
                    }
                if (special) {
#pragma unroll
                    for (int c = 0; c < 8; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (alone[i >> 1]) ds[c][i] = 0.f;
                    hide(ds);
                }
                if (table_part) {
                    auto flush = [&](int r, int b) {
                        bins[((f.slots == 2 ? r : 0) * nb + cur[r]) * 32] += run[r];
                        run[r] = 0.f;
                        cur[r] = b;
                    };
                    auto add = [&](int r, int b, float v) {
                        if (b != cur[r]) flush(r, b);
                        run[r] += v;
                    };
                    by_way(ways.way, [&](auto way) {
                        constexpr int WAY = decltype(way)::value;
                        if constexpr (WAY == kOne) {
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                float2 v = make_float2(0.f, 0.f);
#pragma unroll
                                for (int c = 0; c < 8; ++c) v = __fadd2_rn(v, pair(ds[c][2 * r], ds[c][2 * r + 1]));
                                add(r, ways.lo[r], v.x + v.y);
                            }
                        } else if constexpr (WAY == kTwo) {
                            float v[2][2] = {};
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const int2 at2 = *reinterpret_cast<const int2 *>(columns + c * 8);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const bool second = (i & 1 ? at2.y : at2.x) >= ways.limit[i >> 1][0];
                                    v[i >> 1][0] += second ? 0.f : ds[c][i];
                                    v[i >> 1][1] += second ? ds[c][i] : 0.f;
                                }
                            }
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                add(r, ways.lo[r], v[r][0]);
                                add(r, ways.hi[r], v[r][1]);
                            }
                        } else {
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const int2 at2 = *reinterpret_cast<const int2 *>(columns + c * 8);
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    add(i >> 1, ways.template of<WAY>(a.bias, bias, i >> 1, pos[i >> 1], i & 1 ? at2.y : at2.x), ds[c][i]);
                            }
                        }
                    });
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t u[4], v[4];
                    as_left(ds[2 * k], ds[2 * k + 1], u);
                    less(ds[2 * k], u[0], u[1]);
                    less(ds[2 * k + 1], u[2], u[3]);
                    as_left(ds[2 * k], ds[2 * k + 1], v);
#pragma unroll
                    for (int c = 0; c < KS; ++c) {
                        uint32_t y[4];
                        ldsm_t(k_at + at.left + k * 16 * kPitch + c * 32, y);
                        mma(dq[2 * c], u, y[0], y[1]);
                        mma(dq[2 * c + 1], u, y[2], y[3]);
                        mma(dq[2 * c], v, y[0], y[1]);
                        mma(dq[2 * c + 1], v, y[2], y[3]);
                    }
                }
            }
            if (more) put((step + 2) % kMeta);
            __syncthreads();
        }
        landed<0>();                                     // (without keys: the rows')
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int64_t rr = r0 + warp * 16 + quad + 8 * r;
            if (table_part) bins[((f.slots == 2 ? r : 0) * nb + cur[r]) * 32] += run[r];
            if (rr >= x.rows) continue;
            int64_t i;
            int g;
            row_of(a, rr, i, g);
            const int64_t row = x.rg.q0 + i;
            const int head = x.h * a.group + g;
            if (t4 == 0) {
                dots[row * heads + head] = d[r];
                some[row * heads + head] = alone[r] ? 0.f : 1.f;
            }
            bf16 *out = static_cast<bf16 *>(a.dq) + row * a.ldq2 + (int64_t)head * a.head_dim;
#pragma unroll
            for (int c = 0; c < 2 * KS; ++c) store_pair(out, c * 8 + t4 * 2, a.head_dim, dq[c][2 * r], dq[c][2 * r + 1], a.scale, lse[r] != INFINITY);
        }
        if (table_part) {
            __syncthreads();
            const int g0 = (int)(r0 % a.group), first = a.group;
            const float *all = reinterpret_cast<const float *>(smem + f.bins) + lane;
            for (int b = warp; b < nb; b += f.warps) {
                if (16 % a.group == 0) {                 // rows of a lane have one head in every warp: heads of neighbouring rows by exchange
                    for (int s = 0; s < f.slots; ++s) {
                        float v = 0.f;
                        for (int w = 0; w < f.warps; ++w) v += all[((w * f.slots + s) * nb + b) * 32];
                        v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
                        v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
                        for (int o = 4 * a.group; o < 32; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
                        if (t4 == 0 && quad < a.group) sums[(s * 8 + quad) * nb + b] += v;
                    }
                    continue;
                }
                for (int w = 0; w < f.warps; ++w)
                    for (int s = 0; s < f.slots; ++s) {
                        float v = all[((w * f.slots + s) * nb + b) * 32];
                        v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
                        v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
                        if (t4 == 0) rows_s[w * 16 + s * 8 + quad] = v;
                    }
                __syncwarp();
                for (int g = lane; g < a.group; g += 32) {
                    float v = 0.f;
                    for (int rr = (g - g0 + first) % a.group; rr < 16 * f.warps; rr += a.group)
                        if (f.slots == 2 || (rr & 15) < 8) v += rows_s[rr];
                    sums[g * nb + b] += v;
                }
                __syncwarp();
            }
            __syncthreads();
            if ((t + f.tiles) * 16 * f.warps < x.rows)
                for (int i = 0; i < f.slots * nb; ++i) bins[i * 32] = 0.f;
        }
    }
    if (table_part) {
        __syncthreads();
        float *part = table_part + (x.seq * f.tiles + x.t0) * (int64_t)nb * heads + x.h * a.group;
        for (int i = threadIdx.x; i < nb * a.group; i += blockDim.x) part[i / a.group * heads + i % a.group] = sums[i % a.group * nb + i / a.group];
    }
}

// ---- dK and dV of 16 keys per warp: S^T = K Q^T and dP^T = V dO^T over the rows of the sequence, 32 at a time
template <int KS>
__global__ void __launch_bounds__(32 * kMostWarps, KS <= 4 ? 2 : 1)
attn_mma_dkv_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ MmaShape f, const float *__restrict__ dots, const float *__restrict__ some)
{
    constexpr uint32_t kPitch = Lane<KS>::kPitch, kTileBytes = kStep * kPitch;
    extern __shared__ __align__(16) uint8_t smem[];
    // of the rows of a tile: -lse in powers of two, D, whether they count in dS, position, where their head's biases begin, query and head
    __shared__ __align__(16) float lse_s[kMeta][kStep], dot_s[kMeta][kStep], some_s[kMeta][kStep];
    __shared__ __align__(16) int32_t pos_s[kMeta][kStep], own_s[kMeta][kStep], query_s[kMeta][kStep], head_s[kMeta][kStep];
    __shared__ uint32_t live_s[kMeta][2];
    __shared__ int2 range_s[kMeta][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane >> 2, t4 = lane & 3, heads = a.kv_heads * a.group, nb = a.bias.buckets;
    const uint32_t base = smem_u32(smem), keys_bytes = 16 * f.warps * kPitch;
    MmaBias &bias = *reinterpret_cast<MmaBias *>(smem + f.near);
    const float *table = reinterpret_cast<const float *>(smem + f.table);
    const MmaUnit x = mma_unit(a, f, false);
    const Lane<KS> at(lane);
    const float c1 = a.scale * kLog2e;
    const int64_t keys = x.rg.k1 - x.rg.k0;
    const int n = (int)ceil_div(x.rows, (int64_t)kStep);
    const bf16 *kp = static_cast<const bf16 *>(a.k) + (int64_t)x.h * a.head_dim, *vp = static_cast<const bf16 *>(a.v) + (int64_t)x.h * a.head_dim;
    if (x.t0 * 16ll * f.warps < keys && n > 0) stage_bias(a, bias, reinterpret_cast<float *>(smem + f.table), x.h);
    float lse_n[2], dot_n[2], some_n[2];
    int pos_n[2], head_n[2], query_n[2];
    auto fetch = [&](int tile) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if ((b & (f.warps - 1)) != warp) continue;
            const int64_t r = (int64_t)tile * kStep + b * 32 + lane;
            int64_t i;
            int g;
            row_of(a, min(r, x.rows - 1), i, g);
            const int64_t row = x.rg.q0 + i, cell = row * heads + x.h * a.group + g;
            lse_n[b] = r < x.rows ? a.lse[cell] : -INFINITY;
            dot_n[b] = r < x.rows ? dots[cell] : 0.f;
            some_n[b] = r < x.rows ? some[cell] : 0.f;
            pos_n[b] = pos_of(a.bias.pos_q, row, x.rg.q0);
            head_n[b] = g;
            query_n[b] = (int)i;
        }
    };
    auto put = [&](int slot) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if ((b & (f.warps - 1)) != warp) continue;
            const bool on = lse_n[b] != -INFINITY;
            const uint32_t word = __ballot_sync(0xFFFFFFFFu, on);
            const int first = __reduce_min_sync(0xFFFFFFFFu, on ? pos_n[b] : INT32_MAX), last = __reduce_max_sync(0xFFFFFFFFu, on ? pos_n[b] : INT32_MIN);
            const int at = b * 32 + lane;
            lse_s[slot][at] = on ? -lse_n[b] * kLog2e : -INFINITY;
            dot_s[slot][at] = on ? dot_n[b] : 0.f;
            some_s[slot][at] = on ? some_n[b] : 0.f;
            pos_s[slot][at] = pos_n[b];
            own_s[slot][at] = head_n[b] * nb;
            head_s[slot][at] = x.h * a.group + head_n[b];
            query_s[slot][at] = query_n[b];
            if (lane == 0) {
                live_s[slot][b] = word;
                range_s[slot][b] = make_int2(first, last);
            }
        }
    };
    auto copy = [&](int step) {
        const uint32_t dst = base + f.stages + (step & 1) * 2 * kTileBytes;
        const int slot = step % kMeta;
        const uint32_t w0 = live_s[slot][0], w1 = live_s[slot][1];
        auto from = [&](const void *p, int64_t ld, int r) -> const bf16 * {
            if (!((r < 32 ? w0 >> r : w1 >> (r - 32)) & 1u)) return nullptr;
            return static_cast<const bf16 *>(p) + (x.rg.q0 + query_s[slot][r]) * ld + (int64_t)head_s[slot][r] * a.head_dim;
        };
        if (a.group == 1) {                              // rows follow one another
            const int64_t row = x.rg.q0 + (int64_t)step * kStep, col = (int64_t)x.h * a.head_dim;
            auto on = [&](int r) { return (r < 32 ? w0 >> r : w1 >> (r - 32)) & 1u; };
            load_rows<KS>(dst, kStep, a.head_dim, static_cast<const bf16 *>(a.q) + row * a.ldq + col, a.ldq, on);
            load_rows<KS>(dst + kTileBytes, kStep, a.head_dim, static_cast<const bf16 *>(a.dout) + row * a.ldg + col, a.ldg, on);
        } else {
            load_tile<KS>(dst, kStep, a.head_dim, a.q, [&](int r) { return from(a.q, a.ldq, r); });
            load_tile<KS>(dst + kTileBytes, kStep, a.head_dim, a.q, [&](int r) { return from(a.dout, a.ldg, r); });
        }
        commit();
    };
    for (int64_t t = x.t0; t * 16 * f.warps < keys; t += f.tiles) {
        const int64_t key0 = x.rg.k0 + t * 16 * f.warps;
        __syncthreads();
        auto key_at = [&](const bf16 *p, int64_t ld, int r) -> const bf16 * {
            const int64_t key = key0 + r;
            return key < x.rg.k1 && (!a.mask || a.mask[key]) ? p + key * ld : nullptr;
        };
        load_tile<KS>(base, 16 * f.warps, a.head_dim, kp, [&](int r) { return key_at(kp, a.ldk, r); });
        load_tile<KS>(base + keys_bytes, 16 * f.warps, a.head_dim, kp, [&](int r) { return key_at(vp, a.ldv, r); });
        commit();
        if (n > 0) {
            fetch(0);
            put(0);
            if (n > 1) {
                fetch(1);
                put(1);
            }
            __syncthreads();
            copy(0);
        }
        int pos[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) pos[r] = pos_of(a.bias.pos_k, min(key0 + warp * 16 + quad + 8 * r, x.rg.k1 - 1), x.rg.k0);
        float dk[2 * KS][4], dv[2 * KS][4];
#pragma unroll
        for (int c = 0; c < 2 * KS; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) dk[c][i] = dv[c][i] = 0.f;
        for (int step = 0; step < n; ++step) {
            const int slot = step % kMeta;
            if (step + 1 < n) {
                copy(step + 1);
                landed<1>();
            } else {
                landed<0>();
            }
            const bool more = step + 2 < n;
            if (more) fetch(step + 2);
            __syncthreads();
            const uint32_t q_at = base + f.stages + (step & 1) * 2 * kTileBytes, g_at = q_at + kTileBytes;
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                if (live_s[slot][half] == 0) continue;
                const int c0 = half * 32 + t4 * 2;
                const uint32_t off = half * 32 * kPitch;
                Ways<true> ways;
                ways.find(a.bias, bias, range_s[slot][half].x, range_s[slot][half].y, pos);
                float p[4][4], ds[4][4];
                products<KS, 4>(p, base + warp * 16 * kPitch + at.left, q_at + off + at.right);
                by_way(ways.way, [&](auto way) {
                    constexpr int WAY = decltype(way)::value;
                    const bool one_head = a.group == 1 && WAY <= kTwo;
                    float value[2][2];
                    if (one_head)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            value[r][0] = table[ways.lo[r]];
                            value[r][1] = table[ways.hi[r]];
                        }
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float2 l = *reinterpret_cast<const float2 *>(&lse_s[slot][c0 + c * 8]);
                        const int2 own = *reinterpret_cast<const int2 *>(&own_s[slot][c0 + c * 8]);
                        int2 at2 = make_int2(0, 0);
                        if constexpr (WAY != kOne) at2 = *reinterpret_cast<const int2 *>(&pos_s[slot][c0 + c * 8]);
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            float2 add;
                            if (one_head) {
                                add = WAY == kOne ? pair(value[r][0], value[r][0])
                                                  : pair(at2.x <= ways.limit[r][0] ? value[r][1] : value[r][0], at2.y <= ways.limit[r][0] ? value[r][1] : value[r][0]);
                            } else {
                                add = pair(table[own.x + ways.template of<WAY>(a.bias, bias, r, pos[r], at2.x)],
                                           table[own.y + ways.template of<WAY>(a.bias, bias, r, pos[r], at2.y)]);
                            }
                            const float2 y = __ffma2_rn(pair(p[c][2 * r], p[c][2 * r + 1]), pair(c1, c1), __fadd2_rn(add, l));
                            p[c][2 * r] = exp2_fast(y.x);
                            p[c][2 * r + 1] = exp2_fast(y.y);
                        }
                    }
                });
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    uint32_t u[4];
                    as_left(p[2 * k], p[2 * k + 1], u);
#pragma unroll
                    for (int c = 0; c < KS; ++c) {
                        uint32_t y[4];
                        ldsm_t(g_at + off + at.left + k * 16 * kPitch + c * 32, y);
                        mma(dv[2 * c], u, y[0], y[1]);
                        mma(dv[2 * c + 1], u, y[2], y[3]);
                    }
                }
                products<KS, 4>(ds, base + keys_bytes + warp * 16 * kPitch + at.left, g_at + off + at.right);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float2 d = *reinterpret_cast<const float2 *>(&dot_s[slot][c0 + c * 8]);
                    const float2 m = *reinterpret_cast<const float2 *>(&some_s[slot][c0 + c * 8]);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float2 y = __fmul2_rn(__fmul2_rn(pair(p[c][2 * r], p[c][2 * r + 1]), m),
                                                    __fadd2_rn(pair(ds[c][2 * r], ds[c][2 * r + 1]), pair(-d.x, -d.y)));
                        ds[c][2 * r] = y.x;
                        ds[c][2 * r + 1] = y.y;
                    }
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    uint32_t u[4];
                    as_left(ds[2 * k], ds[2 * k + 1], u);
#pragma unroll
                    for (int c = 0; c < KS; ++c) {
                        uint32_t y[4];
                        ldsm_t(q_at + off + at.left + k * 16 * kPitch + c * 32, y);
                        mma(dk[2 * c], u, y[0], y[1]);
                        mma(dk[2 * c + 1], u, y[2], y[3]);
                    }
                }
            }
            if (more) put((step + 2) % kMeta);
            __syncthreads();
        }
        landed<0>();
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int64_t key = key0 + warp * 16 + quad + 8 * r;
            if (key >= x.rg.k1) continue;
            const bool keep = !a.mask || a.mask[key];
            bf16 *k_out = static_cast<bf16 *>(a.dk) + key * a.ldk2 + (int64_t)x.h * a.head_dim, *v_out = static_cast<bf16 *>(a.dv) + key * a.ldv2 + (int64_t)x.h * a.head_dim;
#pragma unroll
            for (int c = 0; c < 2 * KS; ++c) {
                store_pair(k_out, c * 8 + t4 * 2, a.head_dim, dk[c][2 * r], dk[c][2 * r + 1], a.scale, keep);
                store_pair(v_out, c * 8 + t4 * 2, a.head_dim, dv[c][2 * r], dv[c][2 * r + 1], 1.f, keep);
            }
        }
    }
}

// ---- host side
constexpr int kMaxDevices = 64;
constexpr uint32_t kMostSmem = 216 * 1024;           // dynamic; the kernels declare up to 9 KB beside it
int steps_of(int head_dim) { return head_dim <= 32 ? 2 : head_dim <= 48 ? 3 : head_dim <= 64 ? 4 : head_dim <= 80 ? 5 : head_dim <= 96 ? 6 : 8; }
// warps of a block for so many rows (or keys)
int warps_of(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 ? 4 : kMostWarps; }

MmaShape shape_of(const AttnArgs &a, int64_t tiles, int warps, bool table)
{
    const uint32_t pitch = steps_of(a.head_dim) * 32 + 16;
    MmaShape f{};
    f.warps = warps;
    f.tiles = (int)tiles;
    f.slots = 8 % a.group == 0 ? 1 : 2;
    f.stages = 2 * 16 * warps * pitch;
    f.near = f.stages + 4 * kStep * pitch;
    f.table = f.near + (uint32_t)sizeof(MmaBias);
    f.sums = f.table + (uint32_t)a.bias.buckets * a.group * 4;
    f.rows = f.sums + (table ? (uint32_t)a.bias.buckets * a.group * 4 : 0);
    f.bins = f.rows + (table ? warps * 16 * warps * 4 : 0);
    f.total = f.bins + (table ? (uint32_t)warps * f.slots * a.bias.buckets * 128 : 0);
    return f;
}

template <typename Kernel> bool allow_smem(Kernel kernel, std::atomic<bool> (&done)[kMaxDevices])
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return false;
    if (done[dev]) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem) != cudaSuccess) return false;
    done[dev] = true;
    return true;
}

template <int KS> bool launch(const AttnArgs &a, const MmaPlan &p, float *dots, float *some, float *table_part, cudaStream_t st)
{
    static std::atomic<bool> done[2][kMaxDevices] = {};
    if (!allow_smem(attn_mma_dq_kernel<KS>, done[0]) || !allow_smem(attn_mma_dkv_kernel<KS>, done[1])) return false;
    const MmaShape fq = shape_of(a, p.q_tiles, p.q_warps, table_part != nullptr), fk = shape_of(a, p.k_tiles, p.k_warps, false);
    note_launch();
    attn_mma_dq_kernel<KS><<<(unsigned)(a.n_seq * a.kv_heads * p.q_tiles), 32 * p.q_warps, fq.total, st>>>(a, fq, dots, some, table_part);
    note_launch();
    attn_mma_dkv_kernel<KS><<<(unsigned)(a.n_seq * a.kv_heads * p.k_tiles), 32 * p.k_warps, fk.total, st>>>(a, fk, dots, some);
    return true;
}

}  // namespace

// Blocks as large as their rows (keys) fill and shared memory holds.  The table's bins: as many warps as have room for theirs, or no table here.
MmaPlan mma_plan(const AttnArgs &a, const Lengths &q, const Lengths &k)
{
    MmaPlan p{};
    const int64_t units = std::max<int64_t>(a.n_seq * a.kv_heads, 1);
    p.table = true;
    p.q_warps = warps_of(q.typical * a.group);
    while (p.q_warps > 1 && shape_of(a, 1, p.q_warps, true).total > kMostSmem) p.q_warps /= 2;
    if (shape_of(a, 1, p.q_warps, true).total > kMostSmem) {
        p.table = false;
        p.q_warps = warps_of(q.typical * a.group);
        while (p.q_warps > 1 && shape_of(a, 1, p.q_warps, false).total > kMostSmem) p.q_warps /= 2;
    }
    p.k_warps = warps_of(k.typical);
    while (p.k_warps > 1 && shape_of(a, 1, p.k_warps, false).total > kMostSmem) p.k_warps /= 2;
    p.q_tiles = blocks_per_unit(q, a.group, 16 * p.q_warps, units);
    p.k_tiles = blocks_per_unit(k, 1, 16 * p.k_warps, units);
    p.fits = shape_of(a, 1, p.q_warps, p.table).total <= kMostSmem && shape_of(a, 1, p.k_warps, false).total <= kMostSmem;
    return p;
}

bool mma_attention_backward(const AttnArgs &a, const MmaPlan &p, float *dots, float *some, float *table_part, cudaStream_t st)
{
    switch (steps_of(a.head_dim)) {
    case 2: return launch<2>(a, p, dots, some, table_part, st);
    case 3: return launch<3>(a, p, dots, some, table_part, st);
    case 4: return launch<4>(a, p, dots, some, table_part, st);
    case 5: return launch<5>(a, p, dots, some, table_part, st);
    case 6: return launch<6>(a, p, dots, some, table_part, st);
    default: return launch<8>(a, p, dots, some, table_part, st);
    }
}

}  // namespace e2egrec
