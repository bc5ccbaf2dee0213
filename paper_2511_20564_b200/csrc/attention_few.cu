// Attention where a sequence has few rows (query, head of the group) per key head: single tokens, a candidate, a stack of a few
// tokens.  Every key and value is used a handful of times, so these kernels stream them: fp32 FMA, 16 bytes per lane and load.
//
// `lanes` neighbouring lanes share a head's part of a key (16 bytes each), `heads` key heads lie side by side in a warp as they do in
// memory, and the rest of the warp is further keys of the step; a turn is up to kUnroll steps.  Keys and values come through a ring of
// kStages turns per warp in shared memory, filled by bulk copies (one per turn where the rows follow one another, else one per row):
// what is under way costs no registers, and a turn's latency passes beside the turns before it (with loads into registers, four
// steps of them, two rows to 4096 x 100 keys of 4 heads of 64 took 186 us, this way 74: 5.6 TB/s).  Each lane group keeps its own running
// maximum, sum and outputs over the keys it meets; groups, then the warps of a unit, then the stretches of a long list of keys are joined
// at the end, in a fixed order.  A unit is up to R rows of one sequence and of each of its key heads.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "attention.cuh"
#include "ring_turns.h"
#include "tcgen05.cuh"

namespace e2egrec {
namespace {

constexpr int kFewThreads = 128, kFewWarps = kFewThreads / 32;
constexpr int kUnroll = 4;                           // steps of a turn (fewer where they hold all keys of a sequence, for many keys a
                                                     // step, and 2 for more than two rows, whose registers four would take)
constexpr int kStages = kRingStages;

template <typename T, int CPL> struct Piece {        // a lane's part of a head's row
    static constexpr int E = Chunk<T>::kElems * CPL;
    uint4 raw[CPL];
    __device__ inline void zero()
    {
#pragma unroll
        for (int c = 0; c < CPL; ++c) raw[c] = make_uint4(0, 0, 0, 0);
    }
    // chunk `at`, and (CPL = 2) the chunk `lanes` behind it
    __device__ inline void load(const T *row, int at, int lanes, int chunks)
    {
#pragma unroll
        for (int c = 0; c < CPL; ++c)
            if (at + c * lanes < chunks) raw[c] = __ldg(reinterpret_cast<const uint4 *>(row) + at + c * lanes);
            else raw[c] = make_uint4(0, 0, 0, 0);
    }
    // the same from shared memory
    __device__ inline void load_shared(uint32_t row, int at, int lanes, int chunks)
    {
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            raw[c] = make_uint4(0, 0, 0, 0);
            if (at + c * lanes < chunks)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(raw[c].x), "=r"(raw[c].y), "=r"(raw[c].z), "=r"(raw[c].w) : "r"(row + (at + c * lanes) * 16));
        }
    }
    __device__ inline void widen(float (&v)[E]) const
    {
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            float x[Chunk<T>::kElems];
            Chunk<T>::unpack(raw[c], x);
#pragma unroll
            for (int i = 0; i < Chunk<T>::kElems; ++i) v[c * Chunk<T>::kElems + i] = x[i];
        }
    }
};

template <typename T, int CPL> __device__ inline void store_piece(T *row, int at, int lanes, int chunks, const float (&v)[Piece<T, CPL>::E], float f)
{
#pragma unroll
    for (int c = 0; c < CPL; ++c)
        if (at + c * lanes < chunks) {
            float x[Chunk<T>::kElems];
#pragma unroll
            for (int i = 0; i < Chunk<T>::kElems; ++i) x[i] = v[c * Chunk<T>::kElems + i] * f;
            Chunk<T>::store(row + (int64_t)(at + c * lanes) * Chunk<T>::kElems, x);
        }
}

template <int E> __device__ inline float dot(const float (&a)[E], const float (&b)[E])
{
    float2 t = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < E; i += 2) t = __ffma2_rn(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]), t);
    return t.x + t.y;
}
template <int E> __device__ inline void axpy(float (&y)[E], float s, const float (&x)[E])
{
#pragma unroll
    for (int i = 0; i < E; i += 2) {
        const float2 t = __ffma2_rn(make_float2(s, s), make_float2(x[i], x[i + 1]), make_float2(y[i], y[i + 1]));
        y[i] = t.x;
        y[i + 1] = t.y;
    }
}

struct FewShape {
    int lanes, chunks;                               // lanes per head of a key (a power of two), 16-byte chunks of a head
    int heads, head_groups;                          // key heads side by side in a warp (a power of two), groups of them
    int warps;                                       // warps per unit: a power of two, at most kFewWarps
    int batches;                                     // batches of R rows per sequence and key head
    int splits;                                      // stretches of the keys
    uint32_t units;
    int slice, packed;                               // bytes of a row's heads of a warp; whether those of consecutive rows are one stretch
    int ring_bytes;                                  // of all rings; bins follow, and what is kept of a warp's keys
    int kept, kept_at;                               // most keys that a warp keeps p and dS of; where they lie
};

// A warp's ring: turns of `keys` rows of K and of V (its heads' slice of them), visible rows as bits beside them.  Turn t of the warp is
// the rows (t * warps + its number) * keys and on; a hidden row may come along or not, its bit keeps it out.
struct Ring {
    const char *k, *v;                               // row kb, slice of the heads
    const uint8_t *mask;                             // of row kb
    int64_t ldk, ldv;                                // bytes
    uint32_t base, half;                             // shared memory; bytes of a turn's keys
    uint64_t *bar;
    uint32_t *seen;
    int keys, stride, first, n, turns, slice, own, packed, lane;      // stride, first: rows; own: bytes of a row that are copied
    uint32_t used;                                   // turns that went through the ring so far: stage and phase
    uint32_t next_mask;
    bool ok;
    __device__ inline uint32_t mask_of(int t) const
    {
        const int j = first + t * stride + lane;
        uint32_t m = 1;
        if (mask && lane < keys && j < n) asm volatile("ld.global.u8 %0, [%1];" : "=r"(m) : "l"(mask + j) : "memory");
        return m;
    }
    // turn t into the stage of use `use`
    __device__ inline void fill(int t, uint32_t use)
    {
        const int j0 = first + t * stride, count = min(keys, n - j0);
        const uint32_t word = __ballot_sync(0xFFFFFFFFu, lane < count && next_mask != 0);
        if (t + 1 < turns) next_mask = mask_of(t + 1);
        const uint32_t s = use % kStages, dst = base + s * 2 * half, b = smem_u32(bar + s);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the stage was read through the generic proxy
        if (lane == 0) {
            seen[s] = word;
            mbar_expect_tx(bar + s, packed ? 2u * count * slice : 2u * __popc(word) * own);
            if (packed) {
                copy(dst, k + j0 * ldk, (uint32_t)(count * slice), b);
                copy(dst + half, v + j0 * ldv, (uint32_t)(count * slice), b);
            }
        }
        __syncwarp();
        if (!packed && (word >> lane & 1u)) {
            copy(dst + lane * slice, k + (j0 + lane) * ldk, own, b);
            copy(dst + half + lane * slice, v + (j0 + lane) * ldv, own, b);
        }
    }
    static __device__ inline void copy(uint32_t dst, const char *src, uint32_t bytes, uint32_t b)
    {
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(b) : "memory");
    }
    __device__ inline void start()
    {
        next_mask = turns > 0 ? mask_of(0) : 0;
        for (int t = 0; t < ring_first(turns, ok); ++t) fill(t, used + t);
    }
    // waits for turn t; its stage's address, and which of its rows are seen
    __device__ inline uint32_t wait(uint32_t &word, int t, volatile int *abort_flag)
    {
        const uint32_t use = used + t;
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar + use % kStages, use / kStages & 1u, abort_flag));
        word = ok ? seen[use % kStages] : 0u;
        return base + use % kStages * 2 * half;
    }
    // the wait for turn t is given up: copies on their way land before the shared memory is released, and start() starts no others
    __device__ inline void land(int t)
    {
        int never = 0;
        for (int i = t; i < ring_pending(t, turns); ++i) mbar_wait(bar + (used + i) % kStages, (used + i) / kStages & 1u, &never);
    }
    // turn t has been read by the whole warp
    __device__ inline void done(int t)
    {
        __syncwarp();
        const int next = ring_next(t, turns, ok);
        if (next >= 0) fill(next, used + next);
    }
};

template <int U> __device__ inline Ring ring_of(const AttnArgs &a, const FewShape &f, int es, uint8_t *smem, uint64_t *bars, uint32_t *seen, int warp, int lane)
{
    Ring r;
    r.keys = U * (32 / (f.lanes * f.heads));
    r.slice = f.slice;
    r.half = (uint32_t)(r.keys * f.slice);
    r.base = smem_u32(smem) + (uint32_t)warp * kStages * 2 * r.half;
    r.bar = bars + warp * kStages;
    r.seen = seen + warp * kStages;
    r.ldk = a.ldk * es;
    r.ldv = a.ldv * es;
    r.packed = f.packed;
    r.lane = lane;
    r.used = 0;
    r.ok = true;
    if (lane == 0) {
        for (int s = 0; s < kStages; ++s) mbar_init(r.bar + s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
    return r;
}
// the keys kb .. ke of a unit, head group hg; wu: the warp's number in the unit
__device__ inline void ring_keys(Ring &r, const AttnArgs &a, const FewShape &f, int es, int64_t kb, int64_t ke, int hg, int wu)
{
    const int64_t col = (int64_t)hg * f.slice;
    r.k = static_cast<const char *>(a.k) + kb * r.ldk + col;
    r.v = static_cast<const char *>(a.v) + kb * r.ldv + col;
    r.mask = a.mask ? a.mask + kb : nullptr;
    r.n = (int)(ke - kb);
    r.stride = f.warps * r.keys;
    r.first = wu * r.keys;
    r.turns = r.n > r.first ? (r.n - r.first + r.stride - 1) / r.stride : 0;
    r.own = min(f.heads, a.kv_heads - hg * f.heads) * a.head_dim * es;
}

// sums over the lanes of a key, N values at once
template <int N> __device__ inline void key_sums(float (&v)[N], int lanes)
{
    for (int o = lanes >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
}


__device__ inline float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct Unit {
    SeqRange rg;
    int64_t kb, ke, rows;
    int z, h, hg, first;                             // h: the lane's key head, hg: the warp's group of them
    bool any, on;                                    // there is such a unit; there is such a head
};
__device__ inline Unit few_unit(const AttnArgs &a, const FewShape &f, uint32_t u)            // fewer than 2^31 units: few_plan
{
    Unit x;
    x.z = x.first = 0;
    x.any = u < f.units;
    if (f.splits > 1) {
        x.z = (int)(u % (uint32_t)f.splits);
        u /= (uint32_t)f.splits;
    }
    if (f.batches > 1) {
        x.first = (int)(u % (uint32_t)f.batches);
        u /= (uint32_t)f.batches;
    }
    const uint32_t s = u / (uint32_t)f.head_groups, hg = u - s * (uint32_t)f.head_groups;
    x.hg = (int)hg;
    x.h = (int)(hg * f.heads + (threadIdx.x & 31) / f.lanes % f.heads);
    x.on = x.any && x.h < a.kv_heads;
    if (!x.any) {
        x.rows = x.kb = x.ke = 0;
        x.rg = SeqRange{0, 0, 0, 0};
        return x;
    }
    x.rg = seq_range(a, s, (threadIdx.x & 31) == 0 && hg == 0 && x.first == 0 && x.z == 0);
    x.rows = (x.rg.q1 - x.rg.q0) * a.group;
    x.kb = x.rg.k0;
    x.ke = x.rg.k1;
    if (f.splits > 1) {
        const int64_t per = (x.rg.k1 - x.rg.k0 + f.splits - 1) / f.splits;
        x.kb = min(x.rg.k0 + x.z * per, x.rg.k1);
        x.ke = min(x.kb + per, x.rg.k1);
    }
    return x;
}

// Biases of the scores of a turn: lane i finds the buckets of the turn's key i, which the lanes of that key then ask it for.  It is found from the
// bucket of the turn before, mostly the same or the next one, and everything before the turn's keys are waited for; positions of the keys are
// fetched a turn ahead.  Forward pass of 4096 x 1 x 100 keys: 43 us, 39 without a bias.
template <int R, int U> struct TurnBias {
    int pos[R], col[R];                              // the rows' positions and heads
    Bucket state[R];
    int next;
    int bucket[R * U];                               // of the lane's scores
    float value[R * U];
    // there: there is such a row.  Its position is every lane's, those of heads that are not there too: they find buckets for the others' keys.
    __device__ inline void row(const AttnArgs &a, const Unit &x, bool there, int r, int64_t row, int head)
    {
        pos[r] = there ? pos_of(a.bias.pos_q, row, x.rg.q0) : 0;
        col[r] = there && x.on ? head : 0;
    }
    // before the first turn of a walk
    __device__ inline void begin(const AttnArgs &a, const Unit &x, const Ring &ring)
    {
#pragma unroll
        for (int r = 0; r < R; ++r) state[r].unknown();
        fetch(a, x, ring, 0);
    }
    __device__ inline void fetch(const AttnArgs &a, const Unit &x, const Ring &ring, int t)
    {
        const int j = min(ring.first + t * ring.stride + ring.lane, ring.n - 1);      // (lanes without a key: near the others)
        next = j >= 0 && ring.lane < ring.keys ? pos_of(a.bias.pos_k, x.kb + j, x.rg.k0) : 0;
    }
    __device__ inline void turn(const AttnArgs &a, const Unit &x, const Ring &ring, int t, int kpw, int grp)
    {
        const int mine = next;
        if (t + 1 < ring.turns) fetch(a, x, ring, t + 1);
        if (ring.lane < ring.keys)
#pragma unroll
            for (int r = 0; r < R; ++r) state[r].to(a.bias, a.bias.edges, apart(mine, pos[r]));
        __syncwarp();
#pragma unroll
        for (int i = 0; i < R * U; ++i) {
            bucket[i] = __shfl_sync(0xFFFFFFFFu, state[i / U].at, i % U * kpw + grp);
            value[i] = bias_at(a.bias, a.kv_heads * a.group, bucket[i], col[i / U]);
        }
    }
};

// Sums of dS by bucket that a warp keeps in shared memory.  Every key of a step and head has bins of its own, [rows x buckets x slots], so no two
// lanes meet; the rows' bins go to the warp's sums, [buckets x heads of the warp], at the end of its rows.
struct WarpBins {
    float *bins, *sums;
    int slots, nb, rows, columns;                        // slots: 32 / lanes; columns: heads of the warp
    __device__ inline void clear(const AttnArgs &a, const FewShape &f, float *smem, int rows, int warp, int lane)
    {
        slots = 32 / f.lanes;
        nb = a.bias.buckets;
        this->rows = rows;
        columns = f.heads * a.group;
        bins = smem + (size_t)warp * nb * (rows * slots + columns);
        sums = bins + nb * rows * slots;
        for (int i = lane; i < nb * (rows * slots + columns); i += 32) bins[i] = 0.f;
        __syncwarp();
    }
    __device__ inline void add(int r, int bucket, int slot, float v) { bins[(r * nb + bucket) * slots + slot] += v; }
    // the bins of rows g, g + 1, ... of the group -> sums
    __device__ inline void flush(const AttnArgs &a, const FewShape &f, int g, int lane)
    {
        __syncwarp();
        for (int r = 0; r < rows; ++r) {
            for (int i = lane; i < nb * f.heads; i += 32) {
                float v = 0.f;
                for (int k = i % f.heads; k < slots; k += f.heads) {
                    float &bin = bins[(r * nb + i / f.heads) * slots + k];
                    v += bin;
                    bin = 0.f;
                }
                sums[i / f.heads * columns + i % f.heads * a.group + g] += v;
            }
            __syncwarp();
            g = g + 1 == a.group ? 0 : g + 1;
        }
    }
};
inline size_t bins_bytes(const AttnArgs &a, const FewShape &f, int rows)
{
    return (size_t)kFewWarps * a.bias.buckets * (rows * (32 / f.lanes) + f.heads * a.group) * sizeof(float);
}

// p and dS of a warp's keys, with a key's buckets behind them
__host__ __device__ inline int kept_bytes_of_warp(const FewShape &f, int rows, int keys) { return keys * rows * (f.heads * 8 + 1); }
inline int kept_bytes(const FewShape &f, int rows, int keys) { return kFewWarps * kept_bytes_of_warp(f, rows, keys); }

// Rows of a unit one after the other: query row and head of (query, head of the group) pair r0, r0 + 1, ...
struct RowWalk {
    int64_t row;
    int g;
    __device__ inline RowWalk(const AttnArgs &a, const Unit &x, int64_t r0)
    {
        const int64_t i = a.group == 1 ? r0 : (r0 >> 32 ? r0 / a.group : (int64_t)((uint32_t)r0 / (uint32_t)a.group));
        row = x.rg.q0 + i;
        g = (int)(r0 - i * a.group);
    }
    __device__ inline int head(const AttnArgs &a, const Unit &x) const { return x.h * a.group + g; }
    __device__ inline void next(const AttnArgs &a)
    {
        if (++g == a.group) {
            g = 0;
            ++row;
        }
    }
};

// kb .. ke in turns of warps * kUnroll * (32 / lanes) keys
template <typename T, int R, int U, int CPL, bool kBias>
__global__ void __launch_bounds__(kFewThreads, CPL == 2 ? 2 : (R > 2 ? 3 : 4))
attn_few_fwd_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ FewShape f, float *__restrict__ part_o, float2 *__restrict__ part_ml)
{
    constexpr int E = Piece<T, CPL>::E;
    extern __shared__ __align__(16) uint8_t ring_smem[];
    __shared__ uint64_t bars[kFewWarps * kStages];
    __shared__ uint32_t seen_words[kFewWarps * kStages];
    __shared__ int abort_flag;
    __shared__ float2 join_ml[kFewWarps][R][32];
    __shared__ float join_o[kFewWarps][E * 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int wu = warp & (f.warps - 1);                                            // the warp's number in its unit
    const Unit x = few_unit(a, f, blockIdx.x * (uint32_t)(kFewWarps / f.warps) + warp / f.warps);
    const int wide = f.lanes * f.heads, grp = lane / wide, at = lane & (f.lanes - 1), kpw = 32 / wide;
    const int heads = a.kv_heads * a.group;
    const float c1 = a.scale * kLog2e;
    if (threadIdx.x == 0) abort_flag = 0;
    Ring ring = ring_of<U>(a, f, sizeof(T), ring_smem, bars, seen_words, warp, lane);
    ring_keys(ring, a, f, sizeof(T), x.kb, x.ke, x.hg, wu);
    const uint32_t mine = (uint32_t)(lane / f.lanes % f.heads * a.head_dim * (int)sizeof(T));       // the lane's head in a slice
    __syncthreads();
    for (int64_t n = 0;; ++n) {
        const int64_t r0 = (x.first + n * f.batches) * R;
        const bool live = x.any && r0 < x.rows;
        if (f.warps == 1 ? !live : !__syncthreads_or((int)live)) break;      // barriers inside: all warps of the block go on, or none
        if (live) ring.start();
        float q[R][E], o[R][E], m[R], l[R];
        TurnBias<R, U> bias;
        if constexpr (kBias)
            if (live) bias.begin(a, x, ring);
        RowWalk in(a, x, r0);
#pragma unroll
        for (int r = 0; r < R; ++r, in.next(a)) {
            Piece<T, CPL> p;
            p.zero();
            if constexpr (kBias) bias.row(a, x, live && r0 + r < x.rows, r, in.row, in.head(a, x));
            if (live && x.on && r0 + r < x.rows) p.load(static_cast<const T *>(a.q) + in.row * a.ldq + in.head(a, x) * (int64_t)a.head_dim, at, f.lanes, f.chunks);
            p.widen(q[r]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                q[r][e] *= c1;
                o[r][e] = 0.f;
            }
            m[r] = -INFINITY;
            l[r] = 0.f;
        }
        for (int t = 0; live && t < ring.turns && ring.ok; ++t) {
            uint32_t word;
            if constexpr (kBias) bias.turn(a, x, ring, t, kpw, grp);
            const uint32_t at_k = ring.wait(word, t, &abort_flag) + grp * f.slice + mine, at_v = at_k + ring.half;
            if (!ring.ok) {
                ring.land(t);
                break;
            }
            bool seen[U];
#pragma unroll
            for (int u = 0; u < U; ++u) seen[u] = x.on && (word >> (u * kpw + grp) & 1u);
            float s[R * U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                Piece<T, CPL> k;
                float w[E];
                k.zero();
                if (seen[u]) k.load_shared(at_k + u * kpw * f.slice, at, f.lanes, f.chunks);
                k.widen(w);
#pragma unroll
                for (int r = 0; r < R; ++r) s[r * U + u] = dot<E>(q[r], w);
            }
            key_sums<R * U>(s, f.lanes);
            if constexpr (kBias)
#pragma unroll
                for (int i = 0; i < R * U; ++i) s[i] += bias.value[i];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float top = m[r];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (!seen[u]) s[r * U + u] = -INFINITY;
                    top = fmaxf(top, s[r * U + u]);
                }
                const float base = top == -INFINITY ? 0.f : top, c = exp2_fast(m[r] - base);
                m[r] = top;
                l[r] *= c;
#pragma unroll
                for (int e = 0; e < E; ++e) o[r][e] *= c;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    s[r * U + u] = exp2_fast(s[r * U + u] - base);
                    l[r] += s[r * U + u];
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                Piece<T, CPL> v;
                float w[E];
                v.zero();
                if (seen[u]) v.load_shared(at_v + u * kpw * f.slice, at, f.lanes, f.chunks);
                v.widen(w);
#pragma unroll
                for (int r = 0; r < R; ++r) axpy<E>(o[r], s[r * U + u], w);
            }
            ring.done(t);
        }
        if (live) ring.used += ring.turns;
        // lane groups of the warp
        for (int d = wide; d < 32; d <<= 1)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float m2 = __shfl_xor_sync(0xFFFFFFFFu, m[r], d), l2 = __shfl_xor_sync(0xFFFFFFFFu, l[r], d), top = fmaxf(m[r], m2);
                const float base = top == -INFINITY ? 0.f : top, c = exp2_fast(m[r] - base), c2 = exp2_fast(m2 - base);
                l[r] = l[r] * c + l2 * c2;
                m[r] = top;
#pragma unroll
                for (int e = 0; e < E; ++e) o[r][e] = o[r][e] * c + __shfl_xor_sync(0xFFFFFFFFu, o[r][e], d) * c2;
            }
        if (f.warps > 1) {
            if (grp == 0 && at == 0)
#pragma unroll
                for (int r = 0; r < R; ++r) join_ml[warp][r][lane] = make_float2(m[r], l[r]);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                __syncthreads();
                if (grp == 0)
#pragma unroll
                    for (int e = 0; e < E; ++e) join_o[warp][e * 32 + lane] = o[r][e];
                __syncthreads();
                if (wu == 0 && grp == 0) {
                    float top = -INFINITY;
                    for (int w = 0; w < f.warps; ++w) top = fmaxf(top, join_ml[warp + w][r][lane - at].x);
                    const float base = top == -INFINITY ? 0.f : top;
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) o[r][e] = 0.f;
                    for (int w = 0; w < f.warps; ++w) {
                        const float2 ml = join_ml[warp + w][r][lane - at];
                        const float c = exp2_fast(ml.x - base);
                        sum += ml.y * c;
#pragma unroll
                        for (int e = 0; e < E; ++e) o[r][e] += c * join_o[warp + w][e * 32 + lane];
                    }
                    m[r] = top;
                    l[r] = sum;
                }
            }
        }
        RowWalk out(a, x, r0);
        if (wu == 0 && grp == 0 && live && x.on)
#pragma unroll
            for (int r = 0; r < R; ++r, out.next(a))
                if (r0 + r < x.rows) {
                    const int64_t row = out.row;
                    const int head = out.head(a, x);
                    const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
                    if (f.splits == 1) {
                        store_piece<T, CPL>(static_cast<T *>(a.out) + row * a.ldo + (int64_t)head * a.head_dim, at, f.lanes, f.chunks, o[r], inv);
                        if (a.lse && at == 0) a.lse[row * heads + head] = l[r] == 0.f ? -INFINITY : (m[r] + log2f(l[r])) * kLn2;
                    } else {
                        const int64_t p = ((int64_t)x.z * a.q_rows + row) * heads + head;
#pragma unroll
                        for (int c = 0; c < CPL; ++c)
                            if (at + c * f.lanes < f.chunks)
#pragma unroll
                                for (int e = 0; e < Chunk<T>::kElems; ++e)
                                    part_o[p * a.head_dim + (at + c * f.lanes) * Chunk<T>::kElems + e] = o[r][c * Chunk<T>::kElems + e] * inv;
                        if (at == 0) part_ml[p] = make_float2(l[r] == 0.f ? -INFINITY : m[r], l[r]);
                    }
                }
        if (f.warps > 1) __syncthreads();
    }
    if (!ring.ok && lane == 0 && a.status) atomicOr(reinterpret_cast<unsigned *>(a.status), E2EGREC_DEV_TIMEOUT);
}

// dK and dV of kKeys keys per lane group (j0 and on), over all rows of the sequence.  dots: D of every row, or null where it is to be
// formed from the stored outputs.
constexpr int kKeys = 2;
template <typename T, int CPL, bool kBias>
__device__ inline void keys_gradients(const AttnArgs &a, const SeqRange &rg, int h, bool on, int64_t j0, int64_t end, int grp, int at, const FewShape &f,
                                      const float *dots)
{
    constexpr int E = Piece<T, CPL>::E;
    const int kpw = 32 / (f.lanes * f.heads), heads = a.kv_heads * a.group;
    const int64_t koff = h * (int64_t)a.head_dim;
    const float c1 = a.scale * kLog2e;
    float k[kKeys][E], v[kKeys][E], dk[kKeys][E], dv[kKeys][E];
    bool seen[kKeys];
    int pos[kKeys];
#pragma unroll
    for (int n = 0; n < kKeys; ++n) {
        const int64_t j = j0 + n * kpw + grp;
        seen[n] = on && j < end && (!a.mask || a.mask[j]);
        if constexpr (kBias) pos[n] = seen[n] ? pos_of(a.bias.pos_k, j, rg.k0) : 0;
        Piece<T, CPL> p, t;
        p.zero();
        t.zero();
        if (seen[n]) {
            p.load(static_cast<const T *>(a.k) + j * a.ldk + koff, at, f.lanes, f.chunks);
            t.load(static_cast<const T *>(a.v) + j * a.ldv + koff, at, f.lanes, f.chunks);
        }
        p.widen(k[n]);
        t.widen(v[n]);
#pragma unroll
        for (int e = 0; e < E; ++e) dk[n][e] = dv[n][e] = 0.f;
    }
    for (int64_t row = rg.q0; row < rg.q1; ++row)
        for (int g = 0; g < a.group; ++g) {
            const int head = (on ? h : 0) * a.group + g;
            const float l = __ldg(a.lse + row * heads + head);
            if (__all_sync(0xFFFFFFFFu, l == -INFINITY)) continue;
            const bool live = l != -INFINITY;
            const int64_t col = (int64_t)head * a.head_dim;
            Piece<T, CPL> p, t;
            p.zero();
            t.zero();
            if (live) {
                p.load(static_cast<const T *>(a.q) + row * a.ldq + col, at, f.lanes, f.chunks);
                t.load(static_cast<const T *>(a.dout) + row * a.ldg + col, at, f.lanes, f.chunks);
            }
            float q[E], go[E], s[2 * kKeys], d[1];
            p.widen(q);
            t.widen(go);
            if (dots) {
                d[0] = __ldg(dots + row * heads + head);
            } else {
                Piece<T, CPL> o;
                o.zero();
                if (live) o.load(static_cast<const T *>(a.o) + row * a.ldo + col, at, f.lanes, f.chunks);
                float y[E];
                o.widen(y);
                d[0] = dot<E>(go, y);
                key_sums<1>(d, f.lanes);
            }
#pragma unroll
            for (int n = 0; n < kKeys; ++n) {
                s[n] = dot<E>(q, k[n]);
                s[kKeys + n] = dot<E>(go, v[n]);
            }
            key_sums<2 * kKeys>(s, f.lanes);
            int pos_q = 0;
            if constexpr (kBias) pos_q = pos_of(a.bias.pos_q, row, rg.q0);
#pragma unroll
            for (int n = 0; n < kKeys; ++n) {
                float base = -l * kLog2e;
                if constexpr (kBias) base += bias_at(a.bias, heads, bucket_of(a.bias, a.bias.edges, apart(pos[n], pos_q)), head);
                const float pr = seen[n] && live ? exp2_fast(fmaf(s[n], c1, base)) : 0.f;
                axpy<E>(dv[n], pr, go);
                axpy<E>(dk[n], seen[n] && live ? pr * (s[kKeys + n] - d[0]) : 0.f, q);
            }
        }
#pragma unroll
    for (int n = 0; n < kKeys; ++n) {
        const int64_t j = j0 + n * kpw + grp;
        if (on && j < end) {
            if (!seen[n])                                // 0 times what a row holds need not be 0
#pragma unroll
                for (int e = 0; e < E; ++e) dk[n][e] = dv[n][e] = 0.f;
            store_piece<T, CPL>(static_cast<T *>(a.dk) + j * a.ldk2 + koff, at, f.lanes, f.chunks, dk[n], a.scale);
            store_piece<T, CPL>(static_cast<T *>(a.dv) + j * a.ldv2 + koff, at, f.lanes, f.chunks, dv[n], 1.f);
        }
    }
}

// What D of the stored outputs lacks, the sum of p (dP - D) over the keys, for R rows of unit u from r0 on.  For sequences of more keys than the
// caller named; apart from the kernel below, whose registers it would take (inlined: 72 -> 80 us for 8192 requests of three tokens).
template <int R> struct RowSums {
    float of[R];
};
template <typename T, int R, int CPL, bool kBias> __device__ __noinline__ RowSums<R> lacking(const AttnArgs &a, const FewShape &f, uint32_t unit, int64_t r0)
{
    constexpr int E = Piece<T, CPL>::E;
    const int lane = threadIdx.x & 31, wide = f.lanes * f.heads, grp = lane / wide, at = lane & (f.lanes - 1), kpw = 32 / wide, heads = a.kv_heads * a.group;
    const Unit x = few_unit(a, f, unit);
    const int64_t koff = x.h * (int64_t)a.head_dim;
    const float c1 = a.scale * kLog2e;
    float q[R][E], g[R][E], lse[R], d[R];
    int pos[R], col[R];
    RowSums<R> sums;
    RowWalk in(a, x, r0);
#pragma unroll
    for (int r = 0; r < R; ++r, in.next(a)) {
        Piece<T, CPL> p, t, o;
        p.zero();
        t.zero();
        o.zero();
        lse[r] = INFINITY;
        pos[r] = col[r] = 0;
        if (x.on && r0 + r < x.rows) {
            const int head = in.head(a, x);
            const int64_t off = (int64_t)head * a.head_dim;
            const float v = a.lse[in.row * heads + head];
            if constexpr (kBias) {
                pos[r] = pos_of(a.bias.pos_q, in.row, x.rg.q0);
                col[r] = head;
            }
            if (v != -INFINITY) {
                lse[r] = v * kLog2e;
                p.load(static_cast<const T *>(a.q) + in.row * a.ldq + off, at, f.lanes, f.chunks);
                t.load(static_cast<const T *>(a.dout) + in.row * a.ldg + off, at, f.lanes, f.chunks);
                o.load(static_cast<const T *>(a.o) + in.row * a.ldo + off, at, f.lanes, f.chunks);
            }
        }
        float y[E];
        p.widen(q[r]);
        t.widen(g[r]);
        o.widen(y);
        d[r] = dot<E>(g[r], y);
        sums.of[r] = 0.f;
    }
    key_sums<R>(d, f.lanes);
    for (int64_t j0 = x.kb; j0 < x.ke; j0 += kpw) {
        const int64_t j = j0 + grp;
        const bool on = x.on && j < x.ke && (!a.mask || a.mask[j]);
        Piece<T, CPL> k, v;
        float w[E], y[E], s[2 * R];
        k.zero();
        v.zero();
        if (on) {
            k.load(static_cast<const T *>(a.k) + j * a.ldk + koff, at, f.lanes, f.chunks);
            v.load(static_cast<const T *>(a.v) + j * a.ldv + koff, at, f.lanes, f.chunks);
        }
        k.widen(w);
        v.widen(y);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            s[r] = dot<E>(q[r], w);
            s[R + r] = dot<E>(g[r], y);
        }
        key_sums<2 * R>(s, f.lanes);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float base = -lse[r];
            if constexpr (kBias)
                if (on) base += bias_at(a.bias, heads, bucket_of(a.bias, a.bias.edges, apart(pos_of(a.bias.pos_k, j, x.rg.k0), pos[r])), col[r]);
            sums.of[r] += on ? exp2_fast(fmaf(s[r], c1, base)) * (s[R + r] - d[r]) : 0.f;
        }
    }
    for (int o = wide; o < 32; o <<= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) sums.of[r] += __shfl_xor_sync(0xFFFFFFFFu, sums.of[r], o);
    return sums;
}

// Zeros into dK and dV of a unit's hidden keys where its rows hold infinities or NaN, whose products with p = 0 are not 0; each by the lanes
// that wrote there.  Apart from the kernel below for its registers: looked for in its loop, this took 98 -> 101 us for 4096 pairs.
template <typename T, int U, int CPL> __device__ __noinline__ void clear_hidden(const AttnArgs &a, const FewShape &f, uint32_t unit)
{
    constexpr int E = Piece<T, CPL>::E;
    const int lane = threadIdx.x & 31, wide = f.lanes * f.heads, grp = lane / wide, at = lane & (f.lanes - 1), kpw = 32 / wide;
    const int wu = (threadIdx.x >> 5) & (f.warps - 1);
    const Unit x = few_unit(a, f, unit);
    const int64_t koff = x.h * (int64_t)a.head_dim, turn = U * kpw;
    float zero = 0.f;
    RowWalk in(a, x, 0);
    for (int r = 0; x.on && r < x.rows; ++r, in.next(a)) {
        const int64_t col = in.head(a, x) * (int64_t)a.head_dim;
        Piece<T, CPL> p, t;
        float q[E], g[E];
        p.load(static_cast<const T *>(a.q) + in.row * a.ldq + col, at, f.lanes, f.chunks);
        t.load(static_cast<const T *>(a.dout) + in.row * a.ldg + col, at, f.lanes, f.chunks);
        p.widen(q);
        t.widen(g);
#pragma unroll
        for (int e = 0; e < E; ++e) zero = fmaf(q[e], 0.f, fmaf(g[e], 0.f, zero));
    }
    if (!__any_sync(0xFFFFFFFFu, zero != 0.f)) return;
    const float none[E] = {};
    for (int64_t j0 = x.kb + wu * turn; j0 < x.ke; j0 += f.warps * turn)
        for (int u = 0; u < U; ++u) {
            const int64_t j = j0 + u * kpw + grp;
            if (!x.on || j >= x.ke || a.mask[j]) continue;
            store_piece<T, CPL>(static_cast<T *>(a.dk) + j * a.ldk2 + koff, at, f.lanes, f.chunks, none, 1.f);
            store_piece<T, CPL>(static_cast<T *>(a.dv) + j * a.ldv2 + koff, at, f.lanes, f.chunks, none, 1.f);
        }
}

// Backward pass of up to R rows over a stretch of the keys.  kBoth: the unit holds every row of its sequence and key head, so dK and
// dV of a key are complete as soon as its own step is done and everything is read once; else only dQ (and D, in dots).  A sequence
// that is longer than the launch was sized for has its rows done batch by batch and its keys' gradients apart.
// Where all keys are in one turn of the warp, D = sum_j p_j dP_j is formed from what the registers hold instead of the stored
// outputs: with a handful of keys dP - D cancels, and the rounding of 16-bit outputs showed (dQ of three keys 3.1e-3 off, 2.0e-3 so).
// p is divided by its sum there, which lse, rounded on its own, leaves a few 2^-23 off 1; a p that is the whole sum becomes 1 exactly, and
// dS of a lone key 0.
// Over more keys (kFit) D comes from the stored outputs, and what 16-bit ones lack, sum_j dS_j (0 with the exact D), is taken out at the end:
// dQ = sum_j dS_j k_j - (sum_j dS_j) (sum_j p_j k_j).  dQ of rows that see 12 000 keys was 3.4e-3 off without it, 1.8e-3 so (a rounding:
// 1.7e-3), and the sum goes to D for the kernel of dK and dV where that is another (dK of sharp softmaxes 5e-3 off, 2e-3 so).  Without kFit
// (a turn holds all keys, the caller said) longer sequences go over their keys twice (lacking).
// With a bias and 16-bit outputs (kTwice) D has to be exact before a dS is used: the table's gradient is what is left of dS that cancels, and D of the
// stored out made dK visibly worse than its rounding.  p and dS with D of the stored out are kept for every key in shared memory (8 bytes
// per key, head and row) where that leaves two blocks per SM; what D lacked is known behind the last key, and dK, dV and the table's sums are formed
// from what was kept: keys and values are read once.  Others go over their keys twice.  4096 x 1 x 100, 4 heads of 32: 120 us (71 without a
// bias; with two walks over the keys 169): the instructions and the latency of three blocks per SM, 3.5 TB/s.
template <typename T, int R, int U, int CPL, bool kBoth, bool kFit, bool kBias>
__global__ void __launch_bounds__(kFewThreads, CPL == 2 || R > 2 ? 2 : (R == 1 ? 4 : 3))
attn_few_bwd_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ FewShape f, float *__restrict__ part_dq, float *__restrict__ dots,
                    float *__restrict__ table_part)
{
    constexpr int E = Piece<T, CPL>::E;
    constexpr bool kTwice = kBias && kBoth && sizeof(T) == 2;
    extern __shared__ __align__(16) uint8_t ring_smem[];
    __shared__ uint64_t bars[kFewWarps * kStages];
    __shared__ uint32_t seen_words[kFewWarps * kStages];
    __shared__ int abort_flag;
    __shared__ float join[kFewWarps][E * 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int wu = warp & (f.warps - 1);
    const uint32_t unit = blockIdx.x * (uint32_t)(kFewWarps / f.warps) + warp / f.warps;
    const Unit x = few_unit(a, f, unit);
    const int wide = f.lanes * f.heads, grp = lane / wide, at = lane & (f.lanes - 1), kpw = 32 / wide;
    const int heads = a.kv_heads * a.group;
    const int64_t koff = x.h * (int64_t)a.head_dim;
    const float c1 = a.scale * kLog2e;
    const bool whole = kBoth && x.rows <= R;
    if (threadIdx.x == 0) abort_flag = 0;
    Ring ring = ring_of<U>(a, f, sizeof(T), ring_smem, bars, seen_words, warp, lane);
    ring_keys(ring, a, f, sizeof(T), x.kb, x.ke, x.hg, wu);
    const uint32_t mine = (uint32_t)(lane / f.lanes % f.heads * a.head_dim * (int)sizeof(T));       // the lane's head in a slice
    const bool binned = kBias && kBoth && table_part != nullptr;
    WarpBins bins;
    if (binned) bins.clear(a, f, reinterpret_cast<float *>(ring_smem + f.ring_bytes), R, warp, lane);
    __syncthreads();
    for (int64_t n = 0;; ++n) {
        const int64_t r0 = (x.first + n * f.batches) * R;
        // with kBoth the keys' gradients are written even where there is no row at all
        const bool live = x.any && (r0 < x.rows || (kBoth && n == 0));
        if (f.warps == 1 ? !live : !__syncthreads_or((int)live)) break;
        if (live) ring.start();
        float q[R][E], g[R][E], dq[R][E], lse[R], d[R];
        float mean[kFit ? R : 1][E], rest[R];             // sum_j p_j k_j; what D lacked
        const bool one_turn = f.warps == 1 && f.splits == 1 && x.ke - x.kb <= U * kpw;
        TurnBias<R, U> bias;
        if constexpr (kBias)
            if (live) bias.begin(a, x, ring);
        RowSums<R> lack = {};
        if constexpr (sizeof(T) == 2 && !kFit && !kTwice)
            if (live && !one_turn) lack = lacking<T, R, CPL, kBias>(a, f, unit, r0);       // one warp per unit and one stretch: few_plan
        RowWalk in(a, x, r0);
#pragma unroll
        for (int r = 0; r < R; ++r, in.next(a)) {
            Piece<T, CPL> p, t;
            p.zero();
            t.zero();
            lse[r] = INFINITY;
            d[r] = 0.f;
            if constexpr (kBias) bias.row(a, x, live && r0 + r < x.rows, r, in.row, in.head(a, x));
            if (live && x.on && r0 + r < x.rows) {
                const int64_t row = in.row;
                const int head = in.head(a, x);
                const int64_t col = (int64_t)head * a.head_dim;
                const float v = a.lse[row * heads + head];
                if (v != -INFINITY) {
                    lse[r] = v * kLog2e;
                    p.load(static_cast<const T *>(a.q) + row * a.ldq + col, at, f.lanes, f.chunks);
                    t.load(static_cast<const T *>(a.dout) + row * a.ldg + col, at, f.lanes, f.chunks);
                    if (!one_turn) {
                        Piece<T, CPL> s;
                        s.load(static_cast<const T *>(a.o) + row * a.ldo + col, at, f.lanes, f.chunks);
                        float y[E];
                        s.widen(y);
                        t.widen(g[r]);
                        d[r] = dot<E>(g[r], y);
                    }
                }
            }
            p.widen(q[r]);
            t.widen(g[r]);
#pragma unroll
            for (int e = 0; e < E; ++e) dq[r][e] = 0.f;
            rest[r] = 0.f;
            if constexpr (kFit)
#pragma unroll
                for (int e = 0; e < E; ++e) mean[r][e] = 0.f;
        }
        key_sums<R>(d, f.lanes);
        if constexpr (sizeof(T) == 2 && !kFit && !kTwice)
#pragma unroll
            for (int r = 0; r < R; ++r) d[r] += lack.of[r];
        bool again = true;                                   // over the keys
        if constexpr (kTwice)
            if (!one_turn) {                                 // (the unit's warps go this way together)
                const bool keeps = (x.ke - x.kb + ring.stride - 1) / ring.stride * ring.keys <= f.kept;
                uint8_t *mine_kept = ring_smem + f.kept_at + warp * kept_bytes_of_warp(f, R, f.kept), *kept_bucket = mine_kept + f.kept * f.heads * 8 * R;
                float2 *kept = reinterpret_cast<float2 *>(mine_kept) + lane / f.lanes % f.heads * R;
                float total[R], lacks[R], mean[R][E];        // sums of p, of dS with D of the stored out, of p k
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    total[r] = lacks[r] = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) mean[r][e] = 0.f;
                }
                for (int t = 0; live && t < ring.turns && ring.ok; ++t) {
                    uint32_t word;
                    bias.turn(a, x, ring, t, kpw, grp);
                    const uint32_t at_k = ring.wait(word, t, &abort_flag) + grp * f.slice + mine, at_v = at_k + ring.half;
                    if (!ring.ok) {
                        ring.land(t);
                        break;
                    }
                    float s[2 * R * U];
                    bool seen[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        seen[u] = x.on && (word >> (u * kpw + grp) & 1u);
                        Piece<T, CPL> k, v;
                        float w[E], y[E];
                        k.zero();
                        v.zero();
                        if (seen[u]) {
                            k.load_shared(at_k + u * kpw * f.slice, at, f.lanes, f.chunks);
                            v.load_shared(at_v + u * kpw * f.slice, at, f.lanes, f.chunks);
                        }
                        k.widen(w);
                        v.widen(y);
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            s[r * U + u] = dot<E>(q[r], w);
                            s[(R + r) * U + u] = dot<E>(g[r], y);
                        }
                    }
                    key_sums<2 * R * U>(s, f.lanes);
#pragma unroll
                    for (int i = 0; i < R * U; ++i) {
                        const float add = bias.value[i] - lse[i / U];
                        const float p = seen[i % U] ? exp2_fast(fmaf(s[i], c1, add)) : 0.f;
                        s[i] = p;
                        s[R * U + i] = p == 0.f ? 0.f : p * (s[R * U + i] - d[i / U]);
                        total[i / U] += p;
                        lacks[i / U] += s[R * U + i];
                    }
                    if (keeps) {
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            Piece<T, CPL> k;
                            float w[E];
                            k.zero();
                            if (seen[u]) k.load_shared(at_k + u * kpw * f.slice, at, f.lanes, f.chunks);
                            k.widen(w);
                            const int i = t * ring.keys + u * kpw + grp;
#pragma unroll
                            for (int r = 0; r < R; ++r) {
                                axpy<E>(dq[r], s[(R + r) * U + u], w);
                                axpy<E>(mean[r], s[r * U + u], w);
                                if (at == 0) kept[i * f.heads * R + r] = make_float2(s[r * U + u], s[(R + r) * U + u]);
                                if (lane % wide == 0) kept_bucket[i * R + r] = (uint8_t)bias.bucket[r * U + u];
                            }
                        }
                    }
                    ring.done(t);
                }
                if (live) ring.used += ring.turns;
                for (int o = wide; o < 32; o <<= 1)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        total[r] += __shfl_xor_sync(0xFFFFFFFFu, total[r], o);
                        lacks[r] += __shfl_xor_sync(0xFFFFFFFFu, lacks[r], o);
                    }
                if (f.warps > 1) {
                    __syncthreads();
                    if (grp == 0)
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            join[warp][2 * r * 32 + lane] = total[r];
                            join[warp][(2 * r + 1) * 32 + lane] = lacks[r];
                        }
                    __syncthreads();
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        total[r] = lacks[r] = 0.f;
                        for (int w = 0; w < f.warps; ++w) {
                            total[r] += join[warp - wu + w][2 * r * 32 + lane % wide];
                            lacks[r] += join[warp - wu + w][(2 * r + 1) * 32 + lane % wide];
                        }
                    }
                    __syncthreads();
                }
                bool finite = true;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    lacks[r] = total[r] == 0.f ? 0.f : lacks[r] / total[r];
                    d[r] += lacks[r];
                    finite = finite && fabsf(lacks[r]) < INFINITY;
                }
                // what is kept goes by p alone: beside keys or values that hold infinities or NaN the second walk leaves hidden keys out
                again = !keeps || !__all_sync(0xFFFFFFFFu, finite);
                if (again && live) {
                    if (keeps)
#pragma unroll
                        for (int r = 0; r < R; ++r)
#pragma unroll
                            for (int e = 0; e < E; ++e) dq[r][e] = 0.f;
                    bias.begin(a, x, ring);
                    ring.start();
                } else if (live && ring.ok) {
                    __syncwarp();
#pragma unroll
                    for (int r = 0; r < R; ++r) axpy<E>(dq[r], -lacks[r], mean[r]);
                    float run[R];                            // dS of the bucket that the lane is in
                    int cur[R];
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        run[r] = 0.f;
                        cur[r] = 0;
                    }
                    for (int t = 0; t < ring.turns; ++t)
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            const int i = t * ring.keys + u * kpw + grp;
                            const int64_t j = x.kb + ring.first + t * ring.stride + u * kpw + grp;
                            float dk[E], dv[E];
#pragma unroll
                            for (int e = 0; e < E; ++e) dk[e] = dv[e] = 0.f;
#pragma unroll
                            for (int r = 0; r < R; ++r) {
                                const float2 w = kept[i * f.heads * R + r];
                                const float ds = fmaf(-lacks[r], w.x, w.y);
                                axpy<E>(dk, ds, q[r]);
                                axpy<E>(dv, w.x, g[r]);
                                if (binned) {
                                    const int bucket = kept_bucket[i * R + r];
                                    if (bucket != cur[r]) {
                                        if (at == 0) bins.add(r, cur[r], lane / f.lanes, run[r]);
                                        run[r] = 0.f;
                                        cur[r] = bucket;
                                    }
                                    run[r] += ds;
                                }
                            }
                            if (whole && x.on && j < x.ke) {
                                store_piece<T, CPL>(static_cast<T *>(a.dk) + j * a.ldk2 + koff, at, f.lanes, f.chunks, dk, a.scale);
                                store_piece<T, CPL>(static_cast<T *>(a.dv) + j * a.ldv2 + koff, at, f.lanes, f.chunks, dv, 1.f);
                            }
                        }
                    if (binned && at == 0)
#pragma unroll
                        for (int r = 0; r < R; ++r) bins.add(r, cur[r], lane / f.lanes, run[r]);
                }
            }
        for (int t = 0; live && again && t < ring.turns && ring.ok; ++t) {
            uint32_t word;
            if constexpr (kBias) bias.turn(a, x, ring, t, kpw, grp);
            const uint32_t at_k = ring.wait(word, t, &abort_flag) + grp * f.slice + mine, at_v = at_k + ring.half;
            if (!ring.ok) {
                ring.land(t);
                break;
            }
            bool seen[U];
#pragma unroll
            for (int u = 0; u < U; ++u) seen[u] = x.on && (word >> (u * kpw + grp) & 1u);
            float s[2 * R * U];                                                     // scores, then p; dP, then dS
#pragma unroll
            for (int u = 0; u < U; ++u) {
                Piece<T, CPL> k, v;
                float w[E], y[E];
                k.zero();
                v.zero();
                if (seen[u]) {
                    k.load_shared(at_k + u * kpw * f.slice, at, f.lanes, f.chunks);
                    v.load_shared(at_v + u * kpw * f.slice, at, f.lanes, f.chunks);
                }
                k.widen(w);
                v.widen(y);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    s[r * U + u] = dot<E>(q[r], w);
                    s[(R + r) * U + u] = dot<E>(g[r], y);
                }
            }
            key_sums<2 * R * U>(s, f.lanes);
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float base = -lse[r];
                    if constexpr (kBias) base += bias.value[r * U + u];
                    s[r * U + u] = seen[u] ? exp2_fast(fmaf(s[r * U + u], c1, base)) : 0.f;
                }
                if (one_turn) {
                    float sum = 0.f, t = 0.f;
#pragma unroll
                    for (int u = 0; u < U; ++u) sum += s[r * U + u];
                    for (int o = wide; o < 32; o <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
                    const float lone = lse[r] == INFINITY ? 0.f : 1.f, inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;      // NaN: hidden keys stay at 0
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        s[r * U + u] = s[r * U + u] == sum ? lone : s[r * U + u] * inv;
                        t += seen[u] ? s[r * U + u] * s[(R + r) * U + u] : 0.f;
                    }
                    for (int o = wide; o < 32; o <<= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
                    d[r] = t;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    s[(R + r) * U + u] = seen[u] ? s[r * U + u] * (s[(R + r) * U + u] - d[r]) : 0.f;
                    rest[r] += s[(R + r) * U + u];
                    if constexpr (kBias && kBoth)
                        if (binned && at == 0 && seen[u]) bins.add(r, bias.bucket[r * U + u], lane / f.lanes, s[(R + r) * U + u]);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                Piece<T, CPL> k;
                float w[E];
                k.zero();
                if (seen[u]) k.load_shared(at_k + u * kpw * f.slice, at, f.lanes, f.chunks);
                k.widen(w);
#pragma unroll
                for (int r = 0; r < R; ++r) axpy<E>(dq[r], s[(R + r) * U + u], w);
                if constexpr (kFit)
                    if (!one_turn)
#pragma unroll
                        for (int r = 0; r < R; ++r) axpy<E>(mean[r], s[r * U + u], w);
                const int64_t j = x.kb + ring.first + t * ring.stride + u * kpw + grp;
                if (kBoth && whole && x.on && j < x.ke) {
                    float dk[E], dv[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) dk[e] = dv[e] = 0.f;
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        axpy<E>(dk, s[(R + r) * U + u], q[r]);
                        axpy<E>(dv, s[r * U + u], g[r]);
                    }
                    store_piece<T, CPL>(static_cast<T *>(a.dk) + j * a.ldk2 + koff, at, f.lanes, f.chunks, dk, a.scale);
                    store_piece<T, CPL>(static_cast<T *>(a.dv) + j * a.ldv2 + koff, at, f.lanes, f.chunks, dv, 1.f);
                }
            }
            ring.done(t);
        }
        if (live && again) ring.used += ring.turns;
        if (binned && live) bins.flush(a, f, (int)(r0 % a.group), lane);
        for (int o = wide; o < 32; o <<= 1)
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int e = 0; e < E; ++e) dq[r][e] += __shfl_xor_sync(0xFFFFFFFFu, dq[r][e], o);
            }
        if constexpr (kFit)
            if (!one_turn)
                for (int o = wide; o < 32; o <<= 1)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        rest[r] += __shfl_xor_sync(0xFFFFFFFFu, rest[r], o);
#pragma unroll
                        for (int e = 0; e < E; ++e) mean[r][e] += __shfl_xor_sync(0xFFFFFFFFu, mean[r][e], o);
                    }
        // the warps' sums of N values per lane together, in the first warp
        auto join_warps = [&](auto &v, int n) {
            __syncthreads();
            if (grp == 0)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e < n) join[warp][e * 32 + lane] = v[e];
            __syncthreads();
            if (wu == 0 && grp == 0)
                for (int w = 1; w < f.warps; ++w)
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (e < n) v[e] += join[warp + w][e * 32 + lane];
        };
        RowWalk out(a, x, r0);
#pragma unroll
        for (int r = 0; r < R; ++r, out.next(a)) {
            if (f.warps > 1) {
                join_warps(dq[r], E);
                if constexpr (kFit) {
                    join_warps(mean[r], E);
                    float one[E];
                    one[0] = rest[r];
                    join_warps(one, 1);
                    rest[r] = one[0];
                }
            }
            if (wu == 0 && grp == 0 && live && x.on && r0 + r < x.rows) {
                const int64_t row = out.row;
                const int head = out.head(a, x);
                // (with stretches of the keys the join adds what D lacks)
                if (!kBoth && x.z == 0 && at == 0) dots[row * heads + head] = kFit && !one_turn && f.splits == 1 ? d[r] + rest[r] : d[r];
                if (f.splits == 1) {
                    if constexpr (kFit)
                        if (!one_turn) axpy<E>(dq[r], -rest[r], mean[r]);
                    store_piece<T, CPL>(static_cast<T *>(a.dq) + row * a.ldq2 + (int64_t)head * a.head_dim, at, f.lanes, f.chunks, dq[r], a.scale);
                } else {
                    const int64_t cells = a.q_rows * heads, cell = (x.z * a.q_rows + row) * heads + head, means = f.splits * cells * a.head_dim;
#pragma unroll
                    for (int c = 0; c < CPL; ++c)
                        if (at + c * f.lanes < f.chunks)
#pragma unroll
                            for (int e = 0; e < Chunk<T>::kElems; ++e) {
                                const int64_t p = cell * a.head_dim + (at + c * f.lanes) * Chunk<T>::kElems + e;
                                part_dq[p] = dq[r][c * Chunk<T>::kElems + e] * a.scale;
                                if constexpr (kFit) part_dq[means + p] = mean[r][c * Chunk<T>::kElems + e] * a.scale;
                            }
                    if (kFit && at == 0) part_dq[2 * means + cell] = rest[r];
                }
            }
        }
        if (f.warps > 1) __syncthreads();
    }
    if (!ring.ok && lane == 0 && a.status) atomicOr(reinterpret_cast<unsigned *>(a.status), E2EGREC_DEV_TIMEOUT);
    if (kBoth && x.any && whole && a.mask) clear_hidden<T, U, CPL>(a, f, unit);
    if (kBoth && x.any && !whole)
        for (int64_t j0 = x.kb + (int64_t)wu * kKeys * kpw; j0 < x.ke; j0 += (int64_t)f.warps * kKeys * kpw)
            keys_gradients<T, CPL, kBias>(a, x.rg, x.h, x.on, j0, x.ke, grp, at, f, nullptr);
    if (binned) {                                            // the block's warps, in order, each with its group of key heads
        __syncthreads();
        const int nb = a.bias.buckets, per = f.heads * a.group;
        const float *sums = reinterpret_cast<float *>(ring_smem + f.ring_bytes) + nb * R * bins.slots;
        for (int i = threadIdx.x; i < nb * heads; i += kFewThreads) {
            const int b = i / heads, head = i % heads;
            float v = 0.f;
            for (int w = 0; w < kFewWarps; ++w) {
                const uint32_t u = blockIdx.x * (uint32_t)(kFewWarps / f.warps) + w / f.warps;
                const int hg = (int)(u / (uint32_t)(f.batches * f.splits) % (uint32_t)f.head_groups), at = head - hg * per;
                if (u < f.units && at >= 0 && at < per) v += sums[w * nb * (R * bins.slots + per) + b * per + at];
            }
            table_part[(int64_t)blockIdx.x * nb * heads + i] = v;
        }
    }
}

// dK and dV where the rows of a sequence do not fit one unit
template <typename T, int CPL, bool kBias>
__global__ void __launch_bounds__(kFewThreads)
attn_few_dkv_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ FewShape f, const float *__restrict__ dots)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t u = blockIdx.x * (uint32_t)kFewWarps + warp;
    if (u >= f.units) return;
    const int first = (int)(u % (uint32_t)f.batches);
    u /= (uint32_t)f.batches;
    const uint32_t s = u / (uint32_t)f.head_groups, hg = u - s * (uint32_t)f.head_groups;
    const int wide = f.lanes * f.heads, h = (int)(hg * f.heads + lane / f.lanes % f.heads);
    const SeqRange rg = seq_range(a, s, lane == 0 && hg == 0 && first == 0);
    const int64_t step = (int64_t)kKeys * (32 / wide);
    for (int64_t j0 = rg.k0 + first * step; j0 < rg.k1; j0 += f.batches * step)
        keys_gradients<T, CPL, kBias>(a, rg, h, h < a.kv_heads, j0, rg.k1, lane / wide, lane & (f.lanes - 1), f, dots);
}

// Gradient of the table of biases: dtable_bh = sum of dS over the pairs whose distance is in bucket b.  A warp takes every row_slices-th row of
// a slice of the sequences, a stretch of the keys, its head group's key heads and one query head g of theirs.  Lane groups (a key each) have bins
// of their own and keep the bucket that they are in in registers, so no two lanes meet.  Rows that share their keys read them again (from
// L2); 4 x 1 x 32 768, 8 on 2 heads of 128: 106 us, 5.1 TB/s of L2 (300 with the next keys not fetched beside these, and a bisection per key).
template <typename T, int CPL>
__global__ void __launch_bounds__(kFewThreads)
attn_few_table_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ FewShape f, const __grid_constant__ TablePlan slices,
                      const float *__restrict__ dots, float *__restrict__ part)
{
    constexpr int E = Piece<T, CPL>::E, U = 4;
    extern __shared__ float bins_smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wide = f.lanes * f.heads, grp = lane / wide, at = lane & (f.lanes - 1), kpw = 32 / wide;
    const int heads = a.kv_heads * a.group, nb = a.bias.buckets, slots = 32 / f.lanes;
    uint32_t u = blockIdx.x * (uint32_t)kFewWarps + warp;
    if (u >= f.units) return;
    const int g = (int)(u % (uint32_t)a.group);
    u /= (uint32_t)a.group;
    const int hg = (int)(u % (uint32_t)f.head_groups);
    u /= (uint32_t)f.head_groups;
    const int64_t slice = u, z = slice % slices.key_slices, r0 = slice / slices.key_slices % slices.row_slices, s0 = slice / slices.key_slices / slices.row_slices;
    const int h = hg * f.heads + lane / f.lanes % f.heads, head = h * a.group + g;
    const bool on = h < a.kv_heads;
    const int64_t koff = h * (int64_t)a.head_dim, qoff = head * (int64_t)a.head_dim;
    const float c1 = a.scale * kLog2e;
    float *bins = bins_smem + (size_t)warp * nb * slots, *mine = bins + lane / f.lanes;      // [buckets x slots]
    for (int i = lane; i < nb * slots; i += 32) bins[i] = 0.f;
    __syncwarp();
    float run = 0.f;
    int cur = 0;
    for (int64_t s = s0; s < a.n_seq; s += slices.seq_slices) {
        const SeqRange rg = seq_range(a, s, false);
        const int64_t per = ceil_div(rg.k1 - rg.k0, slices.key_slices), kb = min(rg.k0 + z * per, rg.k1), ke = min(kb + per, rg.k1);
        if (kb >= ke) continue;
        for (int64_t row = rg.q0 + r0; row < rg.q1; row += slices.row_slices) {
            const float l = on ? a.lse[row * heads + head] : -INFINITY;
            if (__all_sync(0xFFFFFFFFu, l == -INFINITY)) continue;
            Piece<T, CPL> p, t;
            p.zero();
            t.zero();
            float d = 0.f;
            if (l != -INFINITY) {
                p.load(static_cast<const T *>(a.q) + row * a.ldq + qoff, at, f.lanes, f.chunks);
                t.load(static_cast<const T *>(a.dout) + row * a.ldg + qoff, at, f.lanes, f.chunks);
                d = __ldg(dots + row * heads + head);
            }
            float q[E], go[E];
            p.widen(q);
            t.widen(go);
            const int pos_q = pos_of(a.bias.pos_q, row, rg.q0);
            const float lse = l * kLog2e;
            // the next keys are on their way beside the sums of these; hidden ones are read too, and left out
            Piece<T, CPL> k[U], v[U];
            bool seen[U];
            int place[U];
            auto fetch = [&](int64_t j0) {
#pragma unroll
                for (int n = 0; n < U; ++n) {
                    const int64_t j = j0 + n * kpw + grp;
                    k[n].zero();
                    v[n].zero();
                    seen[n] = l != -INFINITY && j < ke;
                    place[n] = 0;
                    if (seen[n]) {
                        k[n].load(static_cast<const T *>(a.k) + j * a.ldk + koff, at, f.lanes, f.chunks);
                        v[n].load(static_cast<const T *>(a.v) + j * a.ldv + koff, at, f.lanes, f.chunks);
                        place[n] = pos_of(a.bias.pos_k, j, rg.k0);
                        seen[n] = !a.mask || a.mask[j];
                    }
                }
            };
            Bucket bucket;
            bucket.unknown();
            fetch(kb);
            for (int64_t j0 = kb; j0 < ke; j0 += U * kpw) {
                float sc[2 * U];
                bool on_now[U];
                int away[U];
#pragma unroll
                for (int n = 0; n < U; ++n) {
                    float w[E], x[E];
                    k[n].widen(w);
                    v[n].widen(x);
                    sc[n] = dot<E>(q, w);
                    sc[U + n] = dot<E>(go, x);
                    on_now[n] = seen[n];
                    away[n] = apart(place[n], pos_q);
                }
                if (j0 + U * kpw < ke) fetch(j0 + U * kpw);
                key_sums<2 * U>(sc, f.lanes);
#pragma unroll
                for (int n = 0; n < U; ++n) {
                    if (!on_now[n]) continue;
                    bucket.to(a.bias, a.bias.edges, away[n]);
                    const float pr = exp2_fast(fmaf(sc[n], c1, bias_at(a.bias, heads, bucket.at, head) - lse));
                    if (bucket.at != cur) {
                        if (at == 0) mine[cur * slots] += run;
                        run = 0.f;
                        cur = bucket.at;
                    }
                    run += pr * (sc[U + n] - d);
                }
            }
        }
    }
    if (at == 0) mine[cur * slots] += run;
    __syncwarp();
    for (int i = lane; i < nb * f.heads; i += 32) {
        const int b = i / f.heads, to = hg * f.heads + i % f.heads;
        float v = 0.f;
        for (int k = i % f.heads; k < slots; k += f.heads) v += bins[b * slots + k];
        if (to < a.kv_heads) part[(slice * nb + b) * heads + to * a.group + g] = v;
    }
}

FewShape few_shape(const AttnArgs &a, int es)
{
    FewShape f{};
    f.chunks = a.head_dim * es / 16;
    f.lanes = 1;
    while (f.lanes < f.chunks && f.lanes < 32) f.lanes <<= 1;
    f.heads = 1;
    while (f.heads * 2 <= a.kv_heads && f.heads * 2 * f.lanes <= 32) f.heads *= 2;
    f.head_groups = (a.kv_heads + f.heads - 1) / f.heads;
    f.slice = f.heads * a.head_dim * es;
    f.packed = f.head_groups == 1 && f.heads == a.kv_heads && a.ldk * es == f.slice && a.ldv * es == f.slice;
    f.warps = f.batches = f.splits = 1;
    return f;
}

unsigned few_grid(const AttnArgs &a, FewShape &f)
{
    f.units = (uint32_t)(a.n_seq * f.head_groups * f.batches * f.splits);
    return (unsigned)ceil_div(f.units, kFewWarps / f.warps);
}

template <int U> size_t few_smem(const FewShape &f) { return (size_t)kFewWarps * kStages * 2 * U * (32 / (f.lanes * f.heads)) * f.slice; }

constexpr int kMaxDevices = 64, kMostSmem = 160 * 1024;
template <typename Kernel> bool allow_smem(Kernel kernel, std::atomic<bool> (&done)[kMaxDevices])
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return false;
    if (done[dev]) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem) != cudaSuccess) return false;
    done[dev] = true;
    return true;
}

template <typename T, int R, int U, int CPL, bool kBias>
bool launch_fwd_of(const AttnArgs &a, const FewShape &f, unsigned grid, float *part_o, float2 *part_ml, cudaStream_t st)
{
    static std::atomic<bool> done[kMaxDevices] = {};
    if (!allow_smem(attn_few_fwd_kernel<T, R, U, CPL, kBias>, done)) return false;
    note_launch();
    attn_few_fwd_kernel<T, R, U, CPL, kBias><<<grid, kFewThreads, few_smem<U>(f), st>>>(a, f, part_o, part_ml);
    return true;
}

template <typename T, int R, int U>
bool launch_fwd(const AttnArgs &a, FewShape f, float *part_o, float2 *part_ml, cudaStream_t st)
{
    const unsigned grid = few_grid(a, f);
    if (f.chunks <= 32)
        return a.bias.table ? launch_fwd_of<T, R, U, 1, true>(a, f, grid, part_o, part_ml, st) : launch_fwd_of<T, R, U, 1, false>(a, f, grid, part_o, part_ml, st);
    if constexpr (sizeof(T) == 4)
        return a.bias.table ? launch_fwd_of<T, R, U, 2, true>(a, f, grid, part_o, part_ml, st) : launch_fwd_of<T, R, U, 2, false>(a, f, grid, part_o, part_ml, st);
    return true;
}

template <typename T, int R, int U, int CPL, bool kBoth, bool kFit, bool kBias>
bool launch_bwd_of(const AttnArgs &a, FewShape f, unsigned grid, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    static std::atomic<bool> done[kMaxDevices] = {};
    if (!allow_smem(attn_few_bwd_kernel<T, R, U, CPL, kBoth, kFit, kBias>, done)) return false;
    f.ring_bytes = (int)few_smem<U>(f);
    f.kept_at = f.ring_bytes + (int)(kBias && kBoth && table_part ? bins_bytes(a, f, R) : 0);
    note_launch();
    attn_few_bwd_kernel<T, R, U, CPL, kBoth, kFit, kBias><<<grid, kFewThreads, f.kept_at + kept_bytes(f, R, f.kept), st>>>(a, f, part_dq, dots, table_part);
    return true;
}

template <typename T, int R, int U, bool kBoth, bool kFit>
bool launch_bwd(const AttnArgs &a, FewShape f, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    const unsigned grid = few_grid(a, f);
    auto launch = [&](auto wide) {
        constexpr int CPL = decltype(wide)::value;
        if constexpr (!(kBoth && kFit))                      // what all gradients in one kernel lack with a bias is found before, not fitted
            if (a.bias.table) return launch_bwd_of<T, R, U, CPL, kBoth, kFit, true>(a, f, grid, part_dq, dots, table_part, st);
        return launch_bwd_of<T, R, U, CPL, kBoth, kFit, false>(a, f, grid, part_dq, dots, nullptr, st);
    };
    if (f.chunks <= 32) return launch(std::integral_constant<int, 1>());
    if constexpr (sizeof(T) == 4) return launch(std::integral_constant<int, 2>());
    return true;
}

template <typename T, int R> bool forward_rows(const AttnArgs &a, const FewPlan &p, const FewShape &f, float *part_o, float2 *part_ml, cudaStream_t st)
{
    if (p.steps == 1) return launch_fwd<T, R, 1>(a, f, part_o, part_ml, st);
    if (p.steps == 2) return launch_fwd<T, R, 2>(a, f, part_o, part_ml, st);
    return launch_fwd<T, R, kUnroll>(a, f, part_o, part_ml, st);
}

template <typename T> bool forward_of(const AttnArgs &a, const FewPlan &p, const FewShape &f, float *part_o, float2 *part_ml, cudaStream_t st)
{
    if (p.rows == 1) return forward_rows<T, 1>(a, p, f, part_o, part_ml, st);
    if (p.rows == 2) return forward_rows<T, 2>(a, p, f, part_o, part_ml, st);
    return forward_rows<T, 4>(a, p, f, part_o, part_ml, st);
}

template <typename T, int R, bool kBoth, bool kFit>
bool backward_steps(const AttnArgs &a, const FewPlan &p, const FewShape &f, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    if (p.steps == 1) return launch_bwd<T, R, 1, kBoth, kFit>(a, f, part_dq, dots, table_part, st);
    if (p.steps == 2) return launch_bwd<T, R, 2, kBoth, kFit>(a, f, part_dq, dots, table_part, st);
    return launch_bwd<T, R, kUnroll, kBoth, kFit>(a, f, part_dq, dots, table_part, st);
}

template <typename T, int R, bool kBoth> bool backward_rows(const AttnArgs &a, const FewPlan &p, const FewShape &f, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    if constexpr (sizeof(T) == 2)
        if (p.fit) return backward_steps<T, R, kBoth, true>(a, p, f, part_dq, dots, table_part, st);
    return backward_steps<T, R, kBoth, false>(a, p, f, part_dq, dots, table_part, st);
}

template <typename T> bool backward_of(const AttnArgs &a, const FewPlan &p, FewShape f, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    bool ok;
    if (!p.both) ok = backward_rows<T, 4, false>(a, p, f, part_dq, dots, table_part, st);
    else if (p.rows == 1) ok = backward_rows<T, 1, true>(a, p, f, part_dq, dots, table_part, st);
    else if (p.rows == 2) ok = backward_rows<T, 2, true>(a, p, f, part_dq, dots, table_part, st);
    else ok = backward_rows<T, 4, true>(a, p, f, part_dq, dots, table_part, st);
    if (!ok) return false;
    if (f.splits > 1 && a.q_rows) join_dq(a, f.splits, sizeof(T) == 4 ? E2EGREC_F32 : E2EGREC_BF16, p.fit, part_dq, p.both ? nullptr : dots, st);
    if (!p.both && a.k_rows) {
        note_launch();
        f.batches = (int)p.key_batches;
        f.splits = 1;
        f.warps = 1;
        const unsigned grid = few_grid(a, f);
        auto *kernel = a.bias.table ? attn_few_dkv_kernel<T, 1, true> : attn_few_dkv_kernel<T, 1, false>;
        if constexpr (sizeof(T) == 4)
            if (f.chunks > 32) kernel = a.bias.table ? attn_few_dkv_kernel<T, 2, true> : attn_few_dkv_kernel<T, 2, false>;
        kernel<<<grid, kFewThreads, 0, st>>>(a, f, dots);
    }
    return true;
}

}  // namespace

// Rows per unit, warps per unit and stretches of the keys.  The aim is 24 warps per SM; a warp gets a turn of keys at least.
FewPlan few_plan(const AttnArgs &a, const Lengths &q, const Lengths &k, int es, bool backward)
{
    FewPlan p{};
    const FewShape f = few_shape(a, es);
    // (backward: rows that fit one unit have their keys' gradients in the same pass, which has to hold for every sequence)
    const int64_t rows = (backward ? q.longest : q.typical) * a.group, max_k = k.longest, units0 = std::max<int64_t>(a.n_seq * f.head_groups, 1), most = (((int64_t)1 << 31) - 1) / units0;
    const int64_t step = 32 / (f.lanes * f.heads);
    p.rows = rows <= 1 ? 1 : (rows <= 2 ? 2 : 4);
    p.both = backward && rows <= p.rows;
    p.steps = max_k <= step ? 1 : (max_k <= 2 * step || (p.rows > 2 && max_k > kUnroll * step) ? 2 : kUnroll);
    while (p.steps * step > 32) p.steps /= 2;        // a turn's rows are the bits of a word
    // With a bias the kernel of all gradients goes over the keys twice, first for D, and keeps the table's bins: not where the keys go in stretches,
    // nor where the bins take more shared memory than the rings of 64 KB beside them.
    if (p.both && a.bias.buckets) {
        const int64_t want = std::min(ceil_div(148 * 24, units0), ceil_div(max_k, step * p.steps));
        if (std::min(want / kFewWarps, max_k / (step * p.steps * kFewWarps * 4)) > 1 || bins_bytes(a, f, p.rows) > 64 * 1024) {
            p.both = false;
            p.rows = 4;
            p.steps = max_k <= step ? 1 : 2;
            while (p.steps * step > 32) p.steps /= 2;
        }
    }
    const int64_t turn = step * p.steps;
    p.fit = backward && es == 2 && max_k > turn && !(p.both && a.bias.buckets);
    p.batches = blocks_per_unit(q, a.group, p.rows, units0);
    const int64_t want = std::max<int64_t>(1, std::min(ceil_div(148 * 24, units0 * p.batches), ceil_div(max_k, turn)));
    p.warps = 1;
    while (p.warps < kFewWarps && p.warps < want) p.warps *= 2;
    // a stretch is worth its join where every warp has four turns of it
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({want / p.warps, max_k / (turn * p.warps * 4), kMaxSplits, most / p.batches}));
    if (p.both && a.bias.buckets) {
        p.splits = 1;
        // what is known of a key is kept where that leaves two blocks per SM
        const int64_t keys = align_up((size_t)(ceil_div(max_k, turn * p.warps) * turn), 8);
        const size_t ring = (size_t)kFewWarps * kStages * 2 * turn * f.slice;
        if (es == 2 && keys <= 4096 && ring + bins_bytes(a, f, p.rows) + kept_bytes(f, p.rows, (int)keys) <= 110 * 1024) p.kept = (int)keys;
    }
    p.blocks = ceil_div(units0 * p.batches, kFewWarps / p.warps);
    p.key_batches = blocks_per_unit(k, 1, step * kKeys, units0);
    return p;
}

// Warps enough for 16 per SM, each with a slice of the sequences; of their rows and their keys where there are fewer sequences than that.  (Its bins
// fit: 32 slots of 128 buckets are 16 KB per warp.)
TablePlan few_table_plan(const AttnArgs &a, const Lengths &k, int32_t dtype)
{
    const FewShape f = few_shape(a, (int)dtype_size(dtype));
    const int64_t want = std::max<int64_t>(1, 148 * 16 / ((int64_t)f.head_groups * a.group)), n = std::max<int64_t>(a.n_seq, 1);
    TablePlan p{std::min(n, want), 1, 1};
    p.row_slices = std::max<int64_t>(1, std::min(want / p.seq_slices, ceil_div(a.q_rows, n)));
    p.key_slices = std::max<int64_t>(1, std::min(want / (p.seq_slices * p.row_slices), k.typical / 64));
    return p;
}

bool few_attention_table(const AttnArgs &a, const TablePlan &p, int32_t dtype, const float *dots, float *part, cudaStream_t st)
{
    static std::atomic<bool> done[3][kMaxDevices] = {};
    FewShape f = few_shape(a, (int)dtype_size(dtype));
    f.units = (uint32_t)(p.seq_slices * p.row_slices * p.key_slices * f.head_groups * a.group);
    const unsigned grid = (unsigned)ceil_div(f.units, kFewWarps);
    const size_t smem = (size_t)kFewWarps * a.bias.buckets * (32 / f.lanes) * sizeof(float);
    auto launch = [&](auto *kernel, int i) {
        if (!allow_smem(kernel, done[i])) return false;
        note_launch();
        kernel<<<grid, kFewThreads, smem, st>>>(a, f, p, dots, part);
        return true;
    };
    if (dtype == E2EGREC_BF16) return launch(attn_few_table_kernel<__nv_bfloat16, 1>, 0);
    return f.chunks <= 32 ? launch(attn_few_table_kernel<float, 1>, 1) : launch(attn_few_table_kernel<float, 2>, 2);
}

static FewShape planned(const AttnArgs &a, const FewPlan &p, int32_t dtype)
{
    FewShape f = few_shape(a, (int)dtype_size(dtype));
    f.kept = p.kept;
    f.warps = p.warps;
    f.batches = (int)p.batches;
    f.splits = p.splits;
    return f;
}

bool few_attention_forward(const AttnArgs &a, const FewPlan &p, int32_t dtype, float *part_o, float2 *part_ml, cudaStream_t st)
{
    return dtype == E2EGREC_F32 ? forward_of<float>(a, p, planned(a, p, dtype), part_o, part_ml, st)
                                : forward_of<__nv_bfloat16>(a, p, planned(a, p, dtype), part_o, part_ml, st);
}

bool few_attention_backward(const AttnArgs &a, const FewPlan &p, int32_t dtype, float *part_dq, float *dots, float *table_part, cudaStream_t st)
{
    return dtype == E2EGREC_F32 ? backward_of<float>(a, p, planned(a, p, dtype), part_dq, dots, table_part, st)
                                : backward_of<__nv_bfloat16>(a, p, planned(a, p, dtype), part_dq, dots, table_part, st);
}

}  // namespace e2egrec
