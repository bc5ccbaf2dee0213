// Attention of ragged sequences on the 5th-generation tensor cores (tcgen05): bf16, head_dim <= 128.
//
// The rows of a product are the (query, head of the group) pairs of one key head of one sequence; tiles are 128 x 128.  Every
// operand tile lies in shared memory as blocks of 64 columns, 128 lines of 128 bytes each, 128-byte swizzled: the same bytes serve
// as an operand whose K index is contiguous (Q, K, V, dO against head_dim) and as one whose N index is (V, K, Q, dO against rows).
// Tiles are TMA boxes of three-dimensional maps (columns of a head, heads, rows): columns behind a head's end read as zeros, a box of
// G heads of 128 / G rows is the rows of G query heads.  Rows behind a sequence's end and hidden keys arrive as whatever they hold;
// where such a row would meet p = 0 or dS = 0 in a product (0 x NaN), one warp overwrites it with zeros first.  Scores and gradients of
// scores go back to the tensor cores through tensor memory (A operand), never through shared memory.
// With cp.async for the tiles, zero-filled on the way, the two copying warps were the bound: 47 cycles per 512 bytes and warp.
// Every wait is bounded; when one runs out the block reports E2EGREC_DEV_TIMEOUT, lets its copies land, frees its tensor memory
// and returns.
#include <algorithm>
#include <atomic>

#include "attention.cuh"
#include "tcgen05.cuh"
#include "tensor_map.cuh"
#include "tile_ring.h"

namespace e2egrec {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kTile = 128;
constexpr int kBlockBytes = kTile * 128;             // 64 columns of 128 rows
constexpr int kSms = 148;

__device__ inline float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ inline float2 exp2_pair(float2 x) { return make_float2(exp2_approx(x.x), exp2_approx(x.y)); }
__device__ inline float2 pair_of(uint32_t x, uint32_t y) { return make_float2(__uint_as_float(x), __uint_as_float(y)); }

__device__ inline uint32_t pack_bf16(float lo, float hi)
{
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&h);
}

// 32 columns of the warp's lanes without waiting for them (tmem_load_wait)
__device__ inline void tmem_load32_async(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}

__device__ inline void tmem_load16_async(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}

// Registers are dealt out anew once the block runs, kCopies to the threads of copies and products, kScores to those of the scores.  One
// block per SM: 384 threads x 168 at launch = 128 x 72 + 256 x 216 (forward) = 128 x 104 + 256 x 200 (backward, whose copies hold statistics
// of rows a tile ahead; spilled, they were waited for).  Two blocks per SM: 256 threads x 128 = 128 x 72 + 128 x 184.
template <int kRegisters> __device__ inline void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegisters)); }
template <int kRegisters> __device__ inline void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegisters)); }

// What a block works on: unit u of `units`, a stretch of the keys of a block of rows of one key head.  A block takes the units
// blockIdx.x, blockIdx.x + gridDim.x, ...
struct TcShape {
    uint32_t units;
    int tiles, splits;                               // blocks of rows (or keys) per sequence and key head; stretches of the keys
    int boxes;                                       // rows of the group's heads come as boxes (the group divides 128)
};
struct Work {
    SeqRange rg;
    int64_t rows, kb, ke;
    int z, t0, h, n;                                 // n: tiles of keys
};
__device__ inline Work work_of(const AttnArgs &a, const TcShape &f, uint32_t u, bool report)
{
    Work x;
    x.z = 0;
    if (f.splits > 1) {
        x.z = (int)(u % (uint32_t)f.splits);
        u /= (uint32_t)f.splits;
    }
    x.t0 = 0;
    if (f.tiles > 1) {
        x.t0 = (int)(u % (uint32_t)f.tiles);
        u /= (uint32_t)f.tiles;
    }
    const uint32_t s = u / (uint32_t)a.kv_heads;
    x.h = (int)(u - s * (uint32_t)a.kv_heads);
    x.rg = seq_range(a, s, report && x.z == 0 && x.t0 == 0 && x.h == 0);
    x.rows = (x.rg.q1 - x.rg.q0) * a.group;
    x.kb = x.rg.k0;
    x.ke = x.rg.k1;
    if (f.splits > 1) {
        const int64_t per = ((x.rg.k1 - x.rg.k0 + f.splits - 1) / f.splits + kTile - 1) / kTile * kTile;
        x.kb = min(x.rg.k0 + x.z * per, x.rg.k1);
        x.ke = min(x.kb + per, x.rg.k1);
    }
    x.n = (int)((x.ke - x.kb + kTile - 1) / kTile);
    return x;
}
// (query row, head) of row r of the key head's matrix
__device__ inline void row_of(const AttnArgs &a, const Work &x, int64_t r, int64_t &row, int &head)
{
    const int64_t i = a.group == 1 ? r : (r >> 32 ? r / a.group : (int64_t)((uint32_t)r / (uint32_t)a.group));
    row = x.rg.q0 + i;
    head = x.h * a.group + (int)(r - i * a.group);
}

// One box of 64 columns x 128 rows: column x of head y, row z and on
__device__ inline void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
                 : "memory");
}
template <int NB> __device__ inline void load_tile(uint32_t dst, const CUtensorMap *map, int head, int64_t row, uint64_t *bar)
{
#pragma unroll
    for (int b = 0; b < NB; ++b) tma_load_3d(dst + b * kBlockBytes, map, b * 64, head, (int)row, bar);
}

// The same tile by cp.async, for groups of heads that do not divide 128 (no box has their rows): 32 rows (a quarter) by one warp.  A
// lane keeps to one 16-byte chunk of the rows, 8 NB lanes side by side take a row; mine: the lane's own row (its first element of the
// head), null for zeros; any: an address that may be named where nothing is read.
template <int NB>
__device__ inline void copy_each(uint32_t tile, int part, const bf16 *mine, const void *any, int head_dim, int lane)
{
    constexpr int kPer = 4 / NB;                          // rows per step
    const int ch = lane & (8 * NB - 1), row = lane / (8 * NB);
    const uint32_t dst = tile + (uint32_t)(ch >> 3) * kBlockBytes + (uint32_t)(part * 32 + row) * 128u + (uint32_t)(((ch & 7) ^ row) << 4);
#pragma unroll
    for (int i = 0; i < 8 * NB; ++i) {
        const uint64_t p = __shfl_sync(0xFFFFFFFFu, reinterpret_cast<uint64_t>(mine), row + i * kPer);
        const bool on = p != 0 && ch * 8 < head_dim;
        // row * 128, and the swizzle's exclusive or of the row's low bits with the chunk
        cp_async16((dst ^ (uint32_t)(((i * kPer) & 7) << 4)) + (uint32_t)(i * kPer) * 128u,
                   on ? static_cast<const void *>(reinterpret_cast<const bf16 *>(p) + ch * 8) : any, on);
    }
}
// Arrivals at the barrier of a tile of rows: its box, or every lane of the copying warp once its copies have landed and the warp itself
constexpr uint32_t kCopyArrivals = 33;
__device__ inline void announce_copies(uint64_t *bar, int lane)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}

// Zeros over the rows of a tile whose bit is off, by one warp, visible to the tensor cores
template <int NB> __device__ inline void clear_rows(uint32_t tile, const uint32_t (&word)[4], int lane)
{
    const int ch = lane & (8 * NB - 1), row = lane / (8 * NB);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        if (word[b] == 0xFFFFFFFFu) continue;
        for (int i = 0; i < 8 * NB; ++i) {
            const int r = i * (4 / NB) + row;
            if (!((word[b] >> r) & 1u))
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + (uint32_t)(ch >> 3) * kBlockBytes + (uint32_t)(b * 32 + r) * 128u +
                                                                             (uint32_t)((ch & 7) << 4)),
                             "r"(0)
                             : "memory");
        }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ inline bool all_seen(const uint32_t (&word)[4]) { return (word[0] & word[1] & word[2] & word[3]) == 0xFFFFFFFFu; }

// Loads that stay where they are written, a tile ahead of their use (the compiler moves plain ones down to it, where their latency
// held up the copies: 2800 cycles a tile of the dK, dV kernel)
__device__ inline float load_now(const float *p)
{
    float v;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
    return v;
}
__device__ inline uint32_t load_now(const uint8_t *p)
{
    uint32_t v;
    asm volatile("ld.global.u8 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// Whether the 128 keys from j * 128 on are seen, one bit each; loads for the next tile go out a tile ahead (ahead, then now)
struct Visible {
    uint32_t next[4];
    __device__ inline void ahead(const AttnArgs &a, const Work &x, int j, int lane)
    {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int64_t key = x.kb + (int64_t)j * kTile + b * 32 + lane;
            next[b] = key < x.ke ? (a.mask ? load_now(a.mask + key) : 1u) : 0u;
        }
    }
    __device__ inline void now(uint32_t (&word)[4]) const
    {
#pragma unroll
        for (int b = 0; b < 4; ++b) word[b] = __ballot_sync(0xFFFFFFFFu, next[b] != 0);
    }
};

// the lane that issues the products: a tile has landed, whoever wrote it
__device__ inline bool tile_ready(uint64_t *bar, uint32_t parity, volatile int *abort_flag)
{
    const bool ok = mbar_wait(bar, parity, abort_flag);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc_fence_after();
    return ok;
}
// all lanes of a warp
__device__ inline bool warp_wait(uint64_t *bar, uint32_t parity, volatile int *abort_flag)
{
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag));
}
// Giving up: the copies that were started into slots of a ring land before the shared memory is released
__device__ inline void let_land(uint64_t *bars, uint32_t stages, uint32_t issued)
{
    int never = 0;
    for (uint32_t j = issued > stages ? issued - stages : 0; j < issued; ++j) mbar_wait(&bars[j % stages], (j / stages) & 1u, &never);
}
// the same for the copies of a ring of two sides, 0 .. g - 1
template <typename R> __device__ inline void let_land_both(uint64_t *bars, uint32_t g)
{
    int never = 0;
    for (uint32_t j = g > R::kSlots ? g - R::kSlots : 0; j < g; ++j) mbar_wait(&bars[R::full(j & 1u, j >> 1)], R::parity(j >> 1), &never);
}

// Products of one tile, K step by K step, with descriptors that move on by constants: the instruction stream of the one issuing lane
// is what feeds the tensor cores (with descriptors built anew for every step an instruction took 122 cycles, its execution 64).
// head_steps: d = A B^T over the head (both operands' K index contiguous); row_steps: d (+)= A B over 128 rows, A in tensor memory
// with its steps 4 to 7 `second` columns behind where they would follow, B's N index contiguous.
template <int NB> __device__ inline void head_steps(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, int ksteps)
{
#pragma unroll
    for (int k = 0; k < 4 * NB; ++k)
        if (k < ksteps) umma(d, desc_at(a, (k >> 2) * kBlockBytes + (k & 3) * 32), desc_at(b, (k >> 2) * kBlockBytes + (k & 3) * 32), idesc, k > 0);
}
__device__ inline void row_steps(uint32_t d, uint32_t a, uint32_t second, uint64_t b, uint32_t idesc, bool add, int from = 0, int to = kTile / 16)
{
#pragma unroll
    for (int k = 0; k < kTile / 16; ++k)
        if (k >= from && k < to) umma_ts(d, a + k * 8 + (k >= 4 ? second : 0), desc_at(b, k * 2048), idesc, k > 0 ? 1u : (uint32_t)add);
}

// ------------------------------------------------------------------------------------------------- forward
// NT tiles of 128 rows per block, a softmax warpgroup each.  Two where a key head has more than 128 rows: they share the copies of
// keys and values, and the products of one run beside the softmax of the other.  One, in half of the shared and tensor memory, where
// the second would idle: two such blocks per SM overlap instead.
template <int NB, int NT> struct Fwd {
    using Ring = TileRing<NT == 2 ? (NB == 2 ? 5 : 8) : (NB == 2 ? 2 : 5)>;      // keys and values
    static constexpr int kSoft = NT * 4, kThreads = (kSoft + 4) * 32, kBlocks = 3 - NT;      // copies, zeros, products; one idle
    static constexpr int kRows = NT * kTile, kTileBytes = NB * kBlockBytes, kColumns = NT * 256;
    // p goes to the product in halves where heads take up to 64 columns, the second formed beside the product of the first: 37 x 256 x 8192
    // with 4 heads of 64 158 -> 141 us, one-tile blocks 55 -> 48 us; with heads of 128 158 -> 167 us, so whole there
    static constexpr int kParts = NB == 1 ? 2 : 1;
    static constexpr size_t kSmem = 1024 + (size_t)(NT + Ring::kSlots) * kTileBytes;
};

template <int NB, int NT>
__global__ void __launch_bounds__(Fwd<NB, NT>::kThreads, Fwd<NB, NT>::kBlocks)
attn_tc_fwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ AttnArgs a, const __grid_constant__ TcShape f, float *__restrict__ part_o, float2 *__restrict__ part_ml)
{
    using F = Fwd<NB, NT>;
    using R = typename F::Ring;
    constexpr int kTileBytes = F::kTileBytes, kRows = F::kRows, kSoft = F::kSoft;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t kv_full[R::kBarriers], kv_empty[R::kSlots], v_clean[kWordRing], q_full, q_empty, s_full[NT], p_full[NT][F::kParts], o_full[NT], o_empty[NT];
    __shared__ __align__(16) uint32_t words[kWordRing][4];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *tiles_smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t q_smem = smem_u32(tiles_smem), kv_smem = q_smem + NT * kTileBytes;
    const int ksteps = (a.head_dim + 15) / 16;

    if (threadIdx.x == 0) {
        for (int s = 0; s < R::kBarriers; ++s) mbar_init(&kv_full[s], 1);
        for (int s = 0; s < R::kSlots; ++s) mbar_init(&kv_empty[s], 1);
        for (int s = 0; s < kWordRing; ++s) mbar_init(&v_clean[s], 1);
        mbar_init(&q_full, f.boxes ? 1 : kCopyArrivals);
        mbar_init(&q_empty, 1);
        for (int t = 0; t < NT; ++t) {
            mbar_init(&s_full[t], 1);
            for (int part = 0; part < F::kParts; ++part) mbar_init(&p_full[t][part], 4);
            mbar_init(&o_full[t], 1);
            mbar_init(&o_empty[t], 4);
        }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kSoft + 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "n"(F::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmem_o = tmem + NT * kTile;      // scores (and p) of tile t: columns 128 t; outputs: 64 NB each behind them

    if (warp >= kSoft) {
        fewer_registers<72>();
        if (warp == kSoft) {
            // ---- copies: queries of a block of rows, then keys and values in turn
            uint32_t g = 0, jj = 0, item = 0, q_issued = 0;
            bool ok = true;
            for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
                const Work x = work_of(a, f, u, lane == 0);
                for (int64_t t = x.t0; t * kRows < x.rows && x.n > 0 && ok; t += f.tiles, ++item) {
                    Visible seen;
                    seen.ahead(a, x, 0, lane);
                    if (item > 0) ok = warp_wait(&q_empty, (item - 1) & 1u, &abort_flag);
                    if (!ok) break;
                    const int nt = NT == 2 && x.rows - t * kRows > kTile ? 2 : 1;
                    if (f.boxes) {
                        if (lane == 0) {
                            mbar_expect_tx(&q_full, nt * kTileBytes);
                            for (int q = 0; q < nt; ++q)
                                load_tile<NB>(q_smem + q * kTileBytes, &map_q, x.h * a.group, x.rg.q0 + (t * kRows + q * kTile) / a.group, &q_full);
                        }
                        ++q_issued;
                    } else {
                        for (int b = 0; b < nt * 4; ++b) {
                            const int64_t r = t * kRows + b * 32 + lane;
                            int64_t row;
                            int head;
                            row_of(a, x, r, row, head);
                            copy_each<NB>(q_smem + (b >> 2) * kTileBytes, b & 3,
                                          r < x.rows ? static_cast<const bf16 *>(a.q) + row * a.ldq + (int64_t)head * a.head_dim : nullptr, a.q, a.head_dim, lane);
                        }
                        announce_copies(&q_full, lane);
                    }
                    for (int j = 0; j < x.n && ok; ++j, ++jj) {
                        uint32_t word[4];
                        seen.now(word);
                        if (j + 1 < x.n) seen.ahead(a, x, j + 1, lane);
                        for (int v = 0; v < 2; ++v, ++g) {
                            const uint32_t s = R::slot(g);
                            if (g >= R::kSlots) ok = warp_wait(&kv_empty[s], (R::use(g) - 1) & 1u, &abort_flag);
                            if (!ok) break;
                            if (lane == 0) {
                                if (v == 0) *reinterpret_cast<uint4 *>(words[jj % kWordRing]) = make_uint4(word[0], word[1], word[2], word[3]);
                                mbar_expect_tx(&kv_full[R::full(v, jj)], kTileBytes);
                                load_tile<NB>(kv_smem + s * kTileBytes, v ? &map_v : &map_k, x.h, x.kb + (int64_t)j * kTile, &kv_full[R::full(v, jj)]);
                            }
                        }
                    }
                }
            }
            if (!ok && lane == 0) {
                let_land_both<R>(kv_full, g);
                if (q_issued) let_land(&q_full, 1, q_issued);
            }
            cp_async_wait_all();
        } else if (warp == kSoft + 1) {
            // ---- zeros over hidden rows of the values
            uint32_t g = 1, jj = 0;
            bool ok = true;
            for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
                const Work x = work_of(a, f, u, false);
                for (int64_t t = x.t0; t * kRows < x.rows && x.n > 0 && ok; t += f.tiles)
                    for (int j = 0; j < x.n && ok; ++j, ++jj, g += 2) {
                        ok = warp_wait(&kv_full[R::full(1, jj)], R::parity(jj), &abort_flag);
                        if (!ok) break;
                        const uint4 w4 = *reinterpret_cast<const uint4 *>(words[jj % kWordRing]);
                        const uint32_t word[4] = {w4.x, w4.y, w4.z, w4.w};
                        if (!all_seen(word)) clear_rows<NB>(kv_smem + R::slot(g) * kTileBytes, word, lane);
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&v_clean[jj % kWordRing]);
                    }
            }
        } else if (warp == kSoft + 2) {
            // ---- products
            if (elect_one()) {
                const uint32_t id_s = make_idesc(kTile, kTile), id_o = make_idesc(kTile, ksteps * 16, false, true);
                uint32_t g = 0, jj = 0, item = 0, pc[NT] = {}, used[NT] = {};
                bool ok = true;
                auto scores = [&](uint32_t gk, int q) {
                    head_steps<NB>(tmem + q * kTile, make_smem_desc(q_smem + q * kTileBytes), make_smem_desc(kv_smem + R::slot(gk) * kTileBytes), id_s,
                                   ksteps);
                    umma_commit(&s_full[q]);
                };
                for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
                    const Work x = work_of(a, f, u, false);
                    for (int64_t t = x.t0; t * kRows < x.rows && x.n > 0 && ok; t += f.tiles, ++item) {
                        const int nt = NT == 2 && x.rows - t * kRows > kTile ? 2 : 1;
                        ok = tile_ready(&q_full, item & 1u, &abort_flag);
                        if (ok) ok = tile_ready(&kv_full[R::full(0, jj)], R::parity(jj), &abort_flag);
#pragma unroll
                        for (int q = 0; q < NT; ++q)
                            if (q < nt && ok) {
                                // the outputs that the tile held last have been read
                                if (used[q] > 0) ok = mbar_wait(&o_empty[q], (used[q] - 1) & 1u, &abort_flag);
                                tc_fence_after();
                                if (ok) scores(g, q);
                                ++used[q];
                            }
                        if (ok) umma_commit(&kv_empty[R::slot(g)]);
                        for (int j = 0; j < x.n && ok; ++j, ++jj, g += 2) {
                            const uint32_t gv = g + 1, gk = g + 2;
                            const uint64_t v_desc = make_smem_desc_mn(kv_smem + R::slot(gv) * kTileBytes, kBlockBytes);
                            ok = tile_ready(&kv_full[R::full(1, jj)], R::parity(jj), &abort_flag);
                            if (ok) ok = tile_ready(&v_clean[jj % kWordRing], (jj / kWordRing) & 1u, &abort_flag);
#pragma unroll
                            for (int q = 0; q < NT; ++q) {
                                if (q >= nt || !ok) continue;
#pragma unroll
                                for (int part = 0; part < F::kParts; ++part) {
                                    if (!ok) continue;
                                    ok = mbar_wait(&p_full[q][part], pc[q] & 1u, &abort_flag);
                                    if (!ok) continue;
                                    tc_fence_after();
                                    row_steps(tmem_o + q * 64 * NB, tmem + q * kTile, 0, v_desc, id_o, j > 0, part * (8 / F::kParts), (part + 1) * (8 / F::kParts));
                                }
                                ++pc[q];
                                if (!ok) continue;
                                if (j + 1 < x.n) {
                                    if (q == nt - 1) umma_commit(&kv_empty[R::slot(gv)]);
                                    if (q == 0) ok = tile_ready(&kv_full[R::full(0, jj + 1)], R::parity(jj + 1), &abort_flag);
                                    if (!ok) continue;
                                    scores(gk, q);
                                    if (q == nt - 1) umma_commit(&kv_empty[R::slot(gk)]);
                                } else {
                                    umma_commit(&o_full[q]);
                                    if (q == nt - 1) {
                                        umma_commit(&kv_empty[R::slot(gv)]);
                                        umma_commit(&q_empty);
                                    }
                                }
                            }
                        }
                    }
                }
            }
        }
    } else {
        more_registers<F::kBlocks == 1 ? 216 : 184>();
        // ---- softmax of tile `q`, one row per thread
        const int q = warp >> 2, w = warp & 3;
        const uint32_t lanes = (uint32_t)(w * 32) << 16;
        const uint32_t s_addr = tmem + lanes + q * kTile, o_addr = tmem_o + lanes + q * 64 * NB;
        const float c1 = a.scale * kLog2e;
        const int heads = a.kv_heads * a.group;
        uint32_t jj = 0, sc = 0, oc = 0;
        bool ok = true;
        for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
            const Work x = work_of(a, f, u, false);
            for (int64_t t = x.t0; t * kRows < x.rows && ok; t += f.tiles) {
                const int64_t r = t * kRows + q * kTile + w * 32 + lane;
                if (x.rows - t * kRows <= q * kTile) {       // no rows for this warpgroup
                    jj += x.n;
                    continue;
                }
                float m = -INFINITY, l = 0.f;
                for (int j = 0; j < x.n; ++j, ++jj) {
                    ok = warp_wait(&s_full[q], sc++ & 1u, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t word[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) word[c] = words[jj % kWordRing][c];
                    // the row's 128 scores stay in registers; four chains for the maximum
                    uint32_t v[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_load32_async(s_addr + c * 32, v[c]);
                    tmem_load_wait();
                    float tops[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (word[c] != 0xFFFFFFFFu) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (!((word[c] >> i) & 1u)) v[c][i] = 0xFF800000u;
                        }
                        tops[c] = __uint_as_float(v[c][0]);
#pragma unroll
                        for (int i = 1; i < 32; ++i) tops[c] = fmaxf(tops[c], __uint_as_float(v[c][i]));
                    }
                    const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                    // The maximum that p and l refer to moves only where a score exceeds it by 8 in the exponent: p <= 2^8 loses
                    // nothing in floating point, and the sums so far are rescaled seldom.
                    const bool moves = top * c1 > m * c1 + 8.f || m == -INFINITY;
                    if (j > 0 && __any_sync(0xFFFFFFFFu, moves && top != -INFINITY)) {
                        const float f = moves && top != -INFINITY ? exp2_approx((m - top) * c1) : 1.f;
                        l *= f;
                        __syncwarp();
                        for (int c = 0; c < NB * 4; ++c) {
                            uint32_t x[16];
                            tmem_load16_async(o_addr + c * 16, x);
                            tmem_load_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * f);
                            tmem_store16(o_addr + c * 16, x);
                        }
                    }
                    if (moves) m = top;
                    const float base = m == -INFINITY ? 0.f : m * c1;
                    const float2 scale2 = make_float2(c1, c1), base2 = make_float2(-base, -base);
                    float2 sums[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t p[16];
                        sums[c] = make_float2(0.f, 0.f);
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            float2 x = __ffma2_rn(make_float2(__uint_as_float(v[c][i]), __uint_as_float(v[c][i + 1])), scale2, base2);
                            x.x = exp2_approx(x.x);
                            x.y = exp2_approx(x.y);
                            sums[c] = __fadd2_rn(sums[c], x);
                            p[i / 2] = pack_bf16(x.x, x.y);
                        }
                        tmem_store16(s_addr + c * 16, p);
                        if ((c + 1) % (4 / F::kParts) == 0) {
                            tmem_store_wait();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&p_full[q][(c + 1) / (4 / F::kParts) - 1]);
                            __syncwarp();                    // the stores to tensor memory are for a converged warp
                        }
                    }
                    const float sum = (sums[0].x + sums[0].y) + (sums[1].x + sums[1].y) + ((sums[2].x + sums[2].y) + (sums[3].x + sums[3].y));
                    l += sum;
                }
                if (!ok) break;
                if (x.n > 0) {
                    ok = warp_wait(&o_full[q], oc++ & 1u, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                }
                int64_t row;
                int head;
                row_of(a, x, r, row, head);
                const bool live = r < x.rows;
                const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
                for (int c = 0; c < NB * 2; ++c) {
                    uint32_t v[32];
                    __syncwarp();                            // the loads of tensor memory are for a converged warp; the stores are not
                    if (x.n > 0) {
                        tmem_load32_async(o_addr + c * 32, v);
                        tmem_load_wait();
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = x.n > 0 && l != 0.f ? __float_as_uint(__uint_as_float(v[e]) * inv) : 0u;
                    if (live && f.splits == 1) {
                        bf16 *out = static_cast<bf16 *>(a.out) + row * a.ldo + (int64_t)head * a.head_dim + c * 32;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (c * 32 + e * 8 < a.head_dim) {
                                uint32_t p[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) p[k] = pack_bf16(__uint_as_float(v[e * 8 + 2 * k]), __uint_as_float(v[e * 8 + 2 * k + 1]));
                                *reinterpret_cast<uint4 *>(out + e * 8) = make_uint4(p[0], p[1], p[2], p[3]);
                            }
                    } else if (live) {
                        float *out = part_o + (((int64_t)x.z * a.q_rows + row) * heads + head) * a.head_dim + c * 32;
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (c * 32 + e * 4 < a.head_dim) *reinterpret_cast<uint4 *>(out + e * 4) = make_uint4(v[e * 4], v[e * 4 + 1], v[e * 4 + 2], v[e * 4 + 3]);
                    }
                }
                if (x.n > 0) {                               // the accumulator has been read: the next block of rows may use it
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&o_empty[q]);
                }
                if (live) {
                    if (f.splits > 1) part_ml[((int64_t)x.z * a.q_rows + row) * heads + head] = make_float2(l == 0.f ? -INFINITY : m * c1, l);
                    else if (a.lse) a.lse[row * heads + head] = l == 0.f ? -INFINITY : (m * c1 + log2f(l)) * kLn2;
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && abort_flag && a.status) atomicOr(reinterpret_cast<unsigned *>(a.status), E2EGREC_DEV_TIMEOUT);
    if (warp == kSoft + 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(F::kColumns) : "memory");
}

// ------------------------------------------------------------------------------------------------- backward
// Two kernels, so that no gradient is added up by atomics: dQ goes over the keys of a tile of rows, dK and dV over the rows of a
// tile of keys; the scores are formed in both.  Two warpgroups share a tile of 128 x 128: 64 columns each, one row per thread.
template <int NB> struct Bwd {
    static constexpr int kThreads = 12 * 32, kTileBytes = NB * kBlockBytes;      // copies, zeros, products; one idle
    using KvRing = TileRing<NB == 2 ? 5 : 8>;
    static constexpr int kQgStages = NB == 2 ? 4 : 8;
    static constexpr size_t kDqSmem = 1024 + (size_t)(2 + KvRing::kSlots) * kTileBytes, kDkvSmem = 1024 + (size_t)(2 + kQgStages) * kTileBytes;
};

// 64 columns of p or dS of a thread's row as an operand in tensor memory: 32 packed columns (the second warpgroup's lie 64 behind the
// first's: each half stays within the columns that its warpgroup has read)
__device__ inline void store_operand(uint32_t taddr, const float (&v)[64])
{
    uint32_t r[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    tmem_store32(taddr, r);
}

// The same, and what the rounding to bf16 leaves out as a second operand
__device__ inline void store_operand_and_rest(uint32_t taddr, uint32_t rest, float (&v)[64])
{
    uint32_t r[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        r[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        v[2 * i] -= __uint_as_float(r[i] << 16);
        v[2 * i + 1] -= __uint_as_float(r[i] & 0xFFFF0000u);
    }
    tmem_store32(taddr, r);
    store_operand(rest, v);
}

// One row (up to 64 NB columns) of an accumulator -> out, times f; zeros where !keep
template <int NB>
__device__ inline void store_row(uint32_t taddr, bf16 *out, int head_dim, float f, bool have, bool keep, bool write)
{
    for (int c = 0; c < NB * 2; ++c) {
        uint32_t v[32];
        __syncwarp();                                    // the loads of tensor memory are for a converged warp; the stores are not
        if (have) {
            tmem_load32_async(taddr + c * 32, v);
            tmem_load_wait();
        }
        if (!write) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c * 32 + e * 8 < head_dim) {
                uint32_t p[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    p[k] = have && keep ? pack_bf16(__uint_as_float(v[e * 8 + 2 * k]) * f, __uint_as_float(v[e * 8 + 2 * k + 1]) * f) : 0u;
                *reinterpret_cast<uint4 *>(out + c * 32 + e * 8) = make_uint4(p[0], p[1], p[2], p[3]);
            }
    }
}

// Passes over the keys
__device__ inline int passes_of(const Work &x, int head_dim) { return (int64_t)x.n * kTile > 32 * head_dim ? 2 : 1; }

// dQ, and D = dO . out of every row for the other kernel.  What the stored out's D lacks is the sum of p (dP - D) over the keys; it meets
// sum p k in dQ, which does not get smaller with the number of keys, as dQ does.  Where one tile holds all keys it is added to D before dS is
// formed: dS of a lone key is 0 then (2000 of 32 x 100, four heads of 64, backward: 610 -> 641 us).  Over more than 32 head_dim keys it comes
// from a pass over them that forms p and dP alone (dQ of 26 000 keys and heads of 16: 9.6e-3 off without, 1.7e-3 so; 20 000 and 64:
// 5.3e-3, 1.6e-3; 8 x 512 x 16 384, four heads of 64, backward: 505 -> 668 us).  In between it is left out, about a rounding of the result
// for values whose mean is a quarter of their spread.
// dS goes into its product as two bf16 operands, its rounding and the rest: with dS rounded once dQ was 2.5 to 2.7e-3 off in the mean (a
// rounding of the result: 1.8e-3), at most 2.4e-3 so; the training case's backward pass takes 550 us with one operand, 585 us so.
template <int NB>
__global__ void __launch_bounds__(Bwd<NB>::kThreads, 1)
attn_tc_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_g, const __grid_constant__ CUtensorMap map_k,
                  const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttnArgs a, const __grid_constant__ TcShape f, float *__restrict__ dots)
{
    using R = typename Bwd<NB>::KvRing;
    constexpr int kTileBytes = Bwd<NB>::kTileBytes;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t kv_full[R::kBarriers], kv_empty[R::kSlots], k_clean[kWordRing], q_full, q_empty, s_full[2], dp_full, ds_full, o_full, o_empty, rest_full;
    __shared__ float rests[2][kTile];                 // sums of p (dP - D) over each warpgroup's columns
    __shared__ __align__(16) uint32_t words[kWordRing][4];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *tiles_smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t q_smem = smem_u32(tiles_smem), g_smem = q_smem + kTileBytes, kv_smem = q_smem + 2 * kTileBytes;
    const int ksteps = (a.head_dim + 15) / 16;
    if (threadIdx.x == 0) {
        for (int s = 0; s < R::kBarriers; ++s) mbar_init(&kv_full[s], 1);
        for (int s = 0; s < R::kSlots; ++s) mbar_init(&kv_empty[s], 1);
        for (int s = 0; s < kWordRing; ++s) mbar_init(&k_clean[s], 1);
        mbar_init(&q_full, f.boxes ? 1 : kCopyArrivals);
        mbar_init(&q_empty, 1);
        mbar_init(&s_full[0], 1);
        mbar_init(&s_full[1], 1);
        mbar_init(&dp_full, 1);
        mbar_init(&ds_full, 8);
        mbar_init(&o_full, 1);
        mbar_init(&o_empty, 8);
        mbar_init(&rest_full, 8);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 10) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;                  // scores: columns 0 and 128 in turn; dP and dS: 256; dQ: 384

    if (warp >= 8) {
        fewer_registers<104>();
        if (warp == 8) {
            // ---- copies: Q and dO of a tile of rows, then keys and values in turn
            uint32_t g = 0, jj = 0, item = 0, q_issued = 0;
            bool ok = true;
            for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
                const Work x = work_of(a, f, u, lane == 0);
                const int steps = x.n * passes_of(x, a.head_dim);
                for (int64_t t = x.t0; t * kTile < x.rows && x.n > 0 && ok; t += f.tiles, ++item) {
                    Visible seen;
                    seen.ahead(a, x, 0, lane);
                    if (item > 0) ok = warp_wait(&q_empty, (item - 1) & 1u, &abort_flag);
                    if (!ok) break;
                    if (f.boxes) {
                        if (lane == 0) {
                            mbar_expect_tx(&q_full, 2 * kTileBytes);
                            load_tile<NB>(q_smem, &map_q, x.h * a.group, x.rg.q0 + t * kTile / a.group, &q_full);
                            load_tile<NB>(g_smem, &map_g, x.h * a.group, x.rg.q0 + t * kTile / a.group, &q_full);
                        }
                        ++q_issued;
                    } else {
                        for (int b = 0; b < 4; ++b) {
                            const int64_t r = t * kTile + b * 32 + lane;
                            int64_t row;
                            int head;
                            row_of(a, x, r, row, head);
                            const int64_t col = (int64_t)head * a.head_dim;
                            copy_each<NB>(q_smem, b, r < x.rows ? static_cast<const bf16 *>(a.q) + row * a.ldq + col : nullptr, a.q, a.head_dim, lane);
                            copy_each<NB>(g_smem, b, r < x.rows ? static_cast<const bf16 *>(a.dout) + row * a.ldg + col : nullptr, a.q, a.head_dim, lane);
                        }
                        announce_copies(&q_full, lane);
                    }
                    for (int j = 0, tile = 0; j < steps && ok; ++j, ++jj) {
                        const int next = tile + 1 < x.n ? tile + 1 : 0;
                        uint32_t word[4];
                        seen.now(word);
                        if (j + 1 < steps) seen.ahead(a, x, next, lane);
                        for (int v = 0; v < 2; ++v, ++g) {
                            const uint32_t s = R::slot(g);
                            if (g >= R::kSlots) ok = warp_wait(&kv_empty[s], (R::use(g) - 1) & 1u, &abort_flag);
                            if (!ok) break;
                            if (lane == 0) {
                                if (v == 0) *reinterpret_cast<uint4 *>(words[jj % kWordRing]) = make_uint4(word[0], word[1], word[2], word[3]);
                                mbar_expect_tx(&kv_full[R::full(v, jj)], kTileBytes);
                                load_tile<NB>(kv_smem + s * kTileBytes, v ? &map_v : &map_k, x.h, x.kb + (int64_t)tile * kTile, &kv_full[R::full(v, jj)]);
                            }
                        }
                        tile = next;
                    }
                }
            }
            if (!ok && lane == 0) {
                let_land_both<R>(kv_full, g);
                if (q_issued) let_land(&q_full, 1, q_issued);
            }
            cp_async_wait_all();
        } else if (warp == 9) {
            // ---- zeros over hidden rows of the keys (the products with K as columns leave what they hold to the mask)
            uint32_t g = 0, jj = 0;
            bool ok = true;
            for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
                const Work x = work_of(a, f, u, false);
                const int steps = x.n * passes_of(x, a.head_dim);
                for (int64_t t = x.t0; t * kTile < x.rows && x.n > 0 && ok; t += f.tiles)
                    for (int j = 0; j < steps && ok; ++j, ++jj, g += 2) {
                        ok = warp_wait(&kv_full[R::full(0, jj)], R::parity(jj), &abort_flag);
                        if (!ok) break;
                        const uint4 w4 = *reinterpret_cast<const uint4 *>(words[jj % kWordRing]);
                        const uint32_t word[4] = {w4.x, w4.y, w4.z, w4.w};
                        if (!all_seen(word)) clear_rows<NB>(kv_smem + R::slot(g) * kTileBytes, word, lane);
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&k_clean[jj % kWordRing]);
                    }
            }
        } else if (warp == 10) {
            // ---- products.  S of the next tile goes out before dQ waits for dS, dP of the next tile behind dQ (whose operand it
            // overwrites): the warpgroups form p of the next tile beside dQ and dP.
            if (elect_one()) {
                const uint32_t id_s = make_idesc(kTile, kTile), id_o = make_idesc(kTile, ksteps * 16, false, true);
                const uint64_t q_desc = make_smem_desc(q_smem), g_desc = make_smem_desc(g_smem);
                uint32_t g = 0, item = 0, jj = 0;
                bool ok = true;
                auto product = [&](uint32_t d, uint64_t a_desc, uint32_t slot) {
                    head_steps<NB>(d, a_desc, make_smem_desc(kv_smem + R::slot(slot) * kTileBytes), id_s, ksteps);
                };
                auto full = [&](uint32_t side, uint32_t tile) {
                    ok = ok && tile_ready(&kv_full[R::full(side, tile)], R::parity(tile), &abort_flag);
                    return ok;
                };
                for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
                    const Work x = work_of(a, f, u, false);
                    const int steps = x.n * passes_of(x, a.head_dim), first = steps - x.n;      // of the last pass
                    for (int64_t t = x.t0; t * kTile < x.rows && x.n > 0 && ok; t += f.tiles, ++item) {
                        ok = tile_ready(&q_full, item & 1u, &abort_flag);
                        if (item > 0 && ok) ok = mbar_wait(&o_empty, (item - 1) & 1u, &abort_flag);
                        if (!full(0, jj)) break;
                        product(tmem + (jj & 1u) * kTile, q_desc, g);
                        umma_commit(&s_full[jj & 1u]);
                        if (!full(1, jj)) break;
                        product(tmem + 256, g_desc, g + 1);
                        umma_commit(&dp_full);
                        umma_commit(&kv_empty[R::slot(g + 1)]);
                        for (int j = 0; j < steps; ++j, g += 2, ++jj) {
                            if (j + 1 < steps) {
                                if (!full(0, jj + 1)) break;
                                product(tmem + ((jj + 1) & 1u) * kTile, q_desc, g + 2);
                                umma_commit(&s_full[(jj + 1) & 1u]);
                            }
                            ok = tile_ready(&k_clean[jj % kWordRing], (jj / kWordRing) & 1u, &abort_flag) && mbar_wait(&ds_full, jj & 1u, &abort_flag);
                            if (!ok) break;
                            tc_fence_after();
                            const uint64_t k_desc = make_smem_desc_mn(kv_smem + R::slot(g) * kTileBytes, kBlockBytes);
                            if (j >= first) row_steps(tmem + 384, tmem + 256, 32, k_desc, id_o, j > first);
                            if (j + 1 < steps) {
                                if (!full(1, jj + 1)) break;
                                product(tmem + 256, g_desc, g + 3);
                                umma_commit(&dp_full);
                                umma_commit(&kv_empty[R::slot(g + 3)]);
                            }
                            // the rest of dS, where the scores were: behind dP, which the warpgroups wait for
                            if (j >= first) row_steps(tmem + 384, tmem + (jj & 1u) * kTile, 32, k_desc, id_o, true);
                            umma_commit(&kv_empty[R::slot(g)]);
                            if (j + 1 == steps) {
                                umma_commit(&o_full);
                                umma_commit(&q_empty);
                            }
                        }
                    }
                }
            }
        }
    } else {
        more_registers<200>();
        // ---- p and dS: 64 columns of one row per thread
        const int q = warp >> 2, w = warp & 3;
        const uint32_t lanes = (uint32_t)(w * 32) << 16;
        const float c1 = a.scale * kLog2e;
        const int heads = a.kv_heads * a.group;
        uint32_t jj = 0, item = 0, corrected = 0;
        bool ok = true;
        for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
            const Work x = work_of(a, f, u, false);
            const int steps = x.n * passes_of(x, a.head_dim), first = steps - x.n;
            for (int64_t t = x.t0; t * kTile < x.rows && ok; t += f.tiles) {
                const int64_t r = t * kTile + w * 32 + lane;
                int64_t row;
                int head;
                row_of(a, x, r, row, head);
                const int64_t col = (int64_t)head * a.head_dim;
                const bool live = r < x.rows;
                float base = INFINITY, dot = 0.f;          // rows that saw no key: p = 0
                if (live) {
                    const float l = a.lse[row * heads + head];
                    if (l != -INFINITY) base = l * kLog2e;
                    const bf16 *o = static_cast<const bf16 *>(a.o) + row * a.ldo + col, *gr = static_cast<const bf16 *>(a.dout) + row * a.ldg + col;
#pragma unroll 4
                    for (int e = 0; e < a.head_dim; e += 8) {
                        float xo[8], xg[8];
                        Chunk<bf16>::load(o + e, xo);
                        Chunk<bf16>::load(gr + e, xg);
#pragma unroll
                        for (int k = 0; k < 8; ++k) dot += xo[k] * xg[k];
                    }
                    if (l == -INFINITY) dot = 0.f;
                }
                float rest = 0.f;
                for (int j = 0; j < steps; ++j, ++jj) {
                    ok = warp_wait(&s_full[jj & 1u], (jj >> 1) & 1u, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    float p[64];
                    {
                        uint32_t v[2][32];
                        tmem_load32_async(tmem + lanes + (jj & 1u) * kTile + q * 64, v[0]);
                        tmem_load32_async(tmem + lanes + (jj & 1u) * kTile + q * 64 + 32, v[1]);
                        tmem_load_wait();
#pragma unroll
                        for (int e = 0; e < 64; e += 2) {
                            const float2 y = exp2_pair(__ffma2_rn(pair_of(v[e >> 5][e & 31], v[e >> 5][(e & 31) + 1]), make_float2(c1, c1), make_float2(-base, -base)));
                            p[e] = y.x;
                            p[e + 1] = y.y;
                        }
                    }
                    ok = warp_wait(&dp_full, jj & 1u, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    if (j < first || x.n == 1) {
                        uint32_t v[2][32];
                        tmem_load32_async(tmem + lanes + 256 + q * 64, v[0]);
                        tmem_load32_async(tmem + lanes + 256 + q * 64 + 32, v[1]);
                        tmem_load_wait();
                        float2 sums[2] = {};
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const uint32_t word = words[jj % kWordRing][q * 2 + c];
                            if (word != 0xFFFFFFFFu) {       // whatever hidden keys hold
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (!((word >> e) & 1u)) {
                                        p[c * 32 + e] = 0.f;
                                        v[c][e] = 0u;
                                    }
                            }
#pragma unroll
                            for (int e = 0; e < 32; e += 2)
                                sums[e / 2 & 1] = __ffma2_rn(make_float2(p[c * 32 + e], p[c * 32 + e + 1]),
                                                             __fadd2_rn(pair_of(v[c][e], v[c][e + 1]), make_float2(-dot, -dot)), sums[e / 2 & 1]);
                        }
                        rest += (sums[0].x + sums[0].y) + (sums[1].x + sums[1].y);
                        if (j + 1 == x.n) {                  // all keys: the other warpgroup's columns as well
                            rests[q][w * 32 + lane] = rest;
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&rest_full);
                            ok = warp_wait(&rest_full, corrected++ & 1u, &abort_flag);
                            if (!ok) break;
                            if (base != INFINITY) dot += rests[0][w * 32 + lane] + rests[1][w * 32 + lane];
                            __syncwarp();                    // the loads of tensor memory are for a converged warp
                        }
                        if (j < first) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&ds_full);
                            continue;
                        }
                    }
                    {
                        uint32_t v[2][32];
                        tmem_load32_async(tmem + lanes + 256 + q * 64, v[0]);
                        tmem_load32_async(tmem + lanes + 256 + q * 64 + 32, v[1]);
                        tmem_load_wait();
#pragma unroll
                        for (int e = 0; e < 64; e += 2) {
                            const float2 y = __fmul2_rn(__fadd2_rn(pair_of(v[e >> 5][e & 31], v[e >> 5][(e & 31) + 1]), make_float2(-dot, -dot)),
                                                        make_float2(p[e], p[e + 1]));
                            p[e] = y.x;
                            p[e + 1] = y.y;
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const uint32_t word = words[jj % kWordRing][q * 2 + c];
                        if (word != 0xFFFFFFFFu) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((word >> e) & 1u)) p[c * 32 + e] = 0.f;
                        }
                    }
                    store_operand_and_rest(tmem + lanes + 256 + q * 64, tmem + lanes + (jj & 1u) * kTile + q * 64, p);
                    tmem_store_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ds_full);
                }
                if (!ok) break;
                if (live && q == 0) dots[row * heads + head] = dot;
                if (x.n > 0) {
                    ok = warp_wait(&o_full, item++ & 1u, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                }
                if (q == 0) store_row<NB>(tmem + lanes + 384, static_cast<bf16 *>(a.dq) + row * a.ldq2 + col, a.head_dim, a.scale, x.n > 0, base != INFINITY, live);
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && x.n > 0) mbar_arrive(&o_empty);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && abort_flag && a.status) atomicOr(reinterpret_cast<unsigned *>(a.status), E2EGREC_DEV_TIMEOUT);
    if (warp == 10) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// dK and dV of a tile of keys: S^T = K Q^T and dP^T = V dO^T over the rows of the sequence
template <int NB>
__global__ void __launch_bounds__(Bwd<NB>::kThreads, 1)
attn_tc_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_g, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttnArgs a, const __grid_constant__ TcShape f,
                   const float *__restrict__ dots)
{
    constexpr int kStages = Bwd<NB>::kQgStages, kTileBytes = Bwd<NB>::kTileBytes;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t qg_full[kStages], qg_clean[kStages], qg_empty[kStages], kv_full, kv_empty, s_full, p_full, dp_full, ds_full, o_full, o_empty;
    __shared__ __align__(16) float stat_lse[kWordRing][kTile], stat_dot[kWordRing][kTile];
    __shared__ __align__(16) uint32_t words[kWordRing][4];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *tiles_smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t k_smem = smem_u32(tiles_smem), v_smem = k_smem + kTileBytes, qg_smem = k_smem + 2 * kTileBytes;
    const int ksteps = (a.head_dim + 15) / 16;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&qg_full[s], f.boxes ? 1 : kCopyArrivals);
            mbar_init(&qg_clean[s], 1);
            mbar_init(&qg_empty[s], 1);
        }
        mbar_init(&kv_full, 1);
        mbar_init(&kv_empty, 1);
        mbar_init(&s_full, 1);
        mbar_init(&p_full, 8);
        mbar_init(&dp_full, 1);
        mbar_init(&ds_full, 8);
        mbar_init(&o_full, 1);
        mbar_init(&o_empty, 8);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 10) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;                  // S^T and P^T: columns 0; dP^T and dS^T: 128; dV: 256; dK: 384

    if (warp >= 8) {
        fewer_registers<104>();
        if (warp == 8) {
            // ---- copies: keys and values of a tile, then Q and dO of the rows in turn, with the rows' lse and D (fetched a tile ahead)
            const int heads = a.kv_heads * a.group;
            uint32_t g = 0, jj = 0, item = 0;
            bool ok = true;
            for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
                const Work x = work_of(a, f, u, lane == 0);
                const int64_t keys = x.ke - x.kb;
                const int n = (int)((x.rows + kTile - 1) / kTile);
                float lse[4], dot[4];
                auto ahead = [&](int j) {
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const int64_t r = (int64_t)j * kTile + b * 32 + lane;
                        int64_t row;
                        int head;
                        row_of(a, x, r, row, head);
                        lse[b] = r < x.rows ? load_now(a.lse + row * heads + head) : -INFINITY;
                        dot[b] = r < x.rows ? load_now(dots + row * heads + head) : 0.f;
                    }
                };
                for (int64_t t = x.t0; t * kTile < keys && n > 0 && ok; t += f.tiles, ++item) {
                    ahead(0);
                    if (item > 0) ok = warp_wait(&kv_empty, (item - 1) & 1u, &abort_flag);
                    if (!ok) break;
                    if (lane == 0) {
                        mbar_expect_tx(&kv_full, 2 * kTileBytes);
                        load_tile<NB>(k_smem, &map_k, x.h, x.kb + t * kTile, &kv_full);
                        load_tile<NB>(v_smem, &map_v, x.h, x.kb + t * kTile, &kv_full);
                    }
                    for (int j = 0; j < n && ok; ++j, ++jj) {
                        float l[4], d[4];
                        uint32_t word[4];
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            const bool on = lse[b] != -INFINITY;
                            l[b] = on ? lse[b] * kLog2e : INFINITY;
                            d[b] = on ? dot[b] : 0.f;
                            word[b] = __ballot_sync(0xFFFFFFFFu, on);
                        }
                        if (j + 1 < n) ahead(j + 1);
                        for (int v = 0; v < 2; ++v, ++g) {
                            const uint32_t s = g % kStages;
                            if (g >= kStages) ok = warp_wait(&qg_empty[s], (g / kStages - 1) & 1u, &abort_flag);
                            if (!ok) break;
                            if (v == 0) {
#pragma unroll
                                for (int b = 0; b < 4; ++b) {
                                    stat_lse[jj % kWordRing][b * 32 + lane] = -l[b];
                                    stat_dot[jj % kWordRing][b * 32 + lane] = -d[b];
                                }
                                if (lane == 0) *reinterpret_cast<uint4 *>(words[jj % kWordRing]) = make_uint4(word[0], word[1], word[2], word[3]);
                                __syncwarp();
                            }
                            if (f.boxes) {
                                if (lane == 0) {
                                    mbar_expect_tx(&qg_full[s], kTileBytes);
                                    load_tile<NB>(qg_smem + s * kTileBytes, v ? &map_g : &map_q, x.h * a.group, x.rg.q0 + (int64_t)j * kTile / a.group,
                                                  &qg_full[s]);
                                }
                            } else {
                                for (int b = 0; b < 4; ++b) {
                                    const int64_t r = (int64_t)j * kTile + b * 32 + lane;
                                    int64_t row;
                                    int head;
                                    row_of(a, x, r, row, head);
                                    const int64_t col = (int64_t)head * a.head_dim;
                                    const bf16 *src = v ? static_cast<const bf16 *>(a.dout) + row * a.ldg + col : static_cast<const bf16 *>(a.q) + row * a.ldq + col;
                                    copy_each<NB>(qg_smem + s * kTileBytes, b, (word[b] >> lane) & 1u ? src : nullptr, a.q, a.head_dim, lane);
                                }
                                announce_copies(&qg_full[s], lane);
                            }
                        }
                    }
                }
            }
            if (!ok && lane == 0) {
                if (f.boxes) let_land(qg_full, kStages, g);
                if (item) let_land(&kv_full, 1, item);
            }
            cp_async_wait_all();
        } else if (warp == 9) {
            // ---- zeros over rows behind the sequence's end and rows that saw no key
            uint32_t g = 0, jj = 0;
            bool ok = true;
            for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
                const Work x = work_of(a, f, u, false);
                const int64_t keys = x.ke - x.kb;
                const int n = (int)((x.rows + kTile - 1) / kTile);
                for (int64_t t = x.t0; t * kTile < keys && n > 0 && ok; t += f.tiles)
                    for (int j = 0; j < n && ok; ++j, ++jj)
                        for (int v = 0; v < 2 && ok; ++v, ++g) {
                            ok = warp_wait(&qg_full[g % kStages], (g / kStages) & 1u, &abort_flag);
                            if (!ok) break;
                            const uint4 w4 = *reinterpret_cast<const uint4 *>(words[jj % kWordRing]);
                            const uint32_t word[4] = {w4.x, w4.y, w4.z, w4.w};
                            if (!all_seen(word)) clear_rows<NB>(qg_smem + (g % kStages) * kTileBytes, word, lane);
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&qg_clean[g % kStages]);
                        }
            }
        } else if (warp == 10) {
            // ---- products.  S^T of the next tile follows dV, whose operand it overwrites, dP^T follows dK: the warpgroups form dS
            // beside dV and the next S^T, and the next p beside dK and the next dP^T.
            if (elect_one()) {
                const uint32_t id_s = make_idesc(kTile, kTile), id_o = make_idesc(kTile, ksteps * 16, false, true);
                const uint64_t k_desc = make_smem_desc(k_smem), v_desc = make_smem_desc(v_smem);
                uint32_t g = 0, item = 0, jj = 0;
                bool ok = true;
                auto product = [&](uint32_t d, uint64_t a_desc, uint32_t slot) {
                    head_steps<NB>(d, a_desc, make_smem_desc(qg_smem + (slot % kStages) * kTileBytes), id_s, ksteps);
                };
                auto gradient = [&](uint32_t d, uint32_t operand, uint32_t slot, bool add) {
                    row_steps(d, operand, 32, make_smem_desc_mn(qg_smem + (slot % kStages) * kTileBytes, kBlockBytes), id_o, add);
                };
                auto full = [&](uint32_t slot) {
                    ok = ok && tile_ready(&qg_full[slot % kStages], (slot / kStages) & 1u, &abort_flag) &&
                         tile_ready(&qg_clean[slot % kStages], (slot / kStages) & 1u, &abort_flag);
                    return ok;
                };
                for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
                    const Work x = work_of(a, f, u, false);
                    const int64_t keys = x.ke - x.kb;
                    const int n = (int)((x.rows + kTile - 1) / kTile);
                    for (int64_t t = x.t0; t * kTile < keys && n > 0 && ok; t += f.tiles, ++item) {
                        ok = tile_ready(&kv_full, item & 1u, &abort_flag);
                        if (item > 0 && ok) ok = mbar_wait(&o_empty, (item - 1) & 1u, &abort_flag);
                        if (!full(g)) break;
                        product(tmem, k_desc, g);
                        umma_commit(&s_full);
                        if (!full(g + 1)) break;
                        product(tmem + 128, v_desc, g + 1);
                        umma_commit(&dp_full);
                        for (int j = 0; j < n; ++j, g += 2, ++jj) {
                            ok = mbar_wait(&p_full, jj & 1u, &abort_flag);
                            if (!ok) break;
                            tc_fence_after();
                            gradient(tmem + 256, tmem, g + 1, j > 0);
                            umma_commit(&qg_empty[(g + 1) % kStages]);
                            if (j + 1 < n) {
                                if (!full(g + 2)) break;
                                product(tmem, k_desc, g + 2);
                                umma_commit(&s_full);
                            }
                            ok = mbar_wait(&ds_full, jj & 1u, &abort_flag);
                            if (!ok) break;
                            tc_fence_after();
                            gradient(tmem + 384, tmem + 128, g, j > 0);
                            umma_commit(&qg_empty[g % kStages]);
                            if (j + 1 < n) {
                                if (!full(g + 3)) break;
                                product(tmem + 128, v_desc, g + 3);
                                umma_commit(&dp_full);
                            } else {
                                umma_commit(&o_full);
                                umma_commit(&kv_empty);
                            }
                        }
                    }
                }
            }
        }
    } else {
        more_registers<200>();
        // ---- p and dS: 64 columns (rows of Q) of one key per thread
        const int q = warp >> 2, w = warp & 3;
        const uint32_t lanes = (uint32_t)(w * 32) << 16;
        const float c1 = a.scale * kLog2e;
        uint32_t jj = 0, item = 0;
        bool ok = true;
        for (uint32_t u = blockIdx.x; u < f.units && ok; u += gridDim.x) {
            const Work x = work_of(a, f, u, false);
            const int64_t keys = x.ke - x.kb;
            const int n = (int)((x.rows + kTile - 1) / kTile);
            for (int64_t t = x.t0; t * kTile < keys && ok; t += f.tiles) {
                const int64_t key = x.kb + t * kTile + w * 32 + lane;
                const bool live = key < x.ke, seen = live && (!a.mask || a.mask[key]);
                for (int j = 0; j < n; ++j, ++jj) {
                    ok = warp_wait(&s_full, jj & 1u, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const float4 *lse4 = reinterpret_cast<const float4 *>(stat_lse[jj % kWordRing] + q * 64);
                    const float4 *dot4 = reinterpret_cast<const float4 *>(stat_dot[jj % kWordRing] + q * 64);
                    float p[64];
                    {
                        uint32_t v[2][32];
                        tmem_load32_async(tmem + lanes + q * 64, v[0]);
                        tmem_load32_async(tmem + lanes + q * 64 + 32, v[1]);
                        tmem_load_wait();
#pragma unroll
                        for (int e = 0; e < 64; e += 4) {
                            const float4 l = lse4[e / 4];            // negated, as the sums of products below
                            const float2 y0 = exp2_pair(__ffma2_rn(pair_of(v[e >> 5][e & 31], v[e >> 5][(e & 31) + 1]), make_float2(c1, c1), make_float2(l.x, l.y)));
                            const float2 y1 = exp2_pair(__ffma2_rn(pair_of(v[e >> 5][(e & 31) + 2], v[e >> 5][(e & 31) + 3]), make_float2(c1, c1), make_float2(l.z, l.w)));
                            p[e] = y0.x;
                            p[e + 1] = y0.y;
                            p[e + 2] = y1.x;
                            p[e + 3] = y1.y;
                        }
                    }
                    store_operand(tmem + lanes + q * 64, p);
                    tmem_store_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full);
                    ok = warp_wait(&dp_full, jj & 1u, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    {
                        uint32_t v[2][32];
                        tmem_load32_async(tmem + lanes + 128 + q * 64, v[0]);
                        tmem_load32_async(tmem + lanes + 128 + q * 64 + 32, v[1]);
                        tmem_load_wait();
#pragma unroll
                        for (int e = 0; e < 64; e += 4) {
                            const float4 d = dot4[e / 4];
                            const float2 y0 = __fmul2_rn(__fadd2_rn(pair_of(v[e >> 5][e & 31], v[e >> 5][(e & 31) + 1]), make_float2(d.x, d.y)), make_float2(p[e], p[e + 1]));
                            const float2 y1 = __fmul2_rn(__fadd2_rn(pair_of(v[e >> 5][(e & 31) + 2], v[e >> 5][(e & 31) + 3]), make_float2(d.z, d.w)), make_float2(p[e + 2], p[e + 3]));
                            p[e] = y0.x;
                            p[e + 1] = y0.y;
                            p[e + 2] = y1.x;
                            p[e + 3] = y1.y;
                        }
                    }
                    store_operand(tmem + lanes + 128 + q * 64, p);
                    tmem_store_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ds_full);
                }
                if (!ok) break;
                if (n > 0) {
                    ok = warp_wait(&o_full, item++ & 1u, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                }
                const int64_t col = x.h * (int64_t)a.head_dim;
                if (q == 0) store_row<NB>(tmem + lanes + 256, static_cast<bf16 *>(a.dv) + key * a.ldv2 + col, a.head_dim, 1.f, n > 0, seen, live);
                else store_row<NB>(tmem + lanes + 384, static_cast<bf16 *>(a.dk) + key * a.ldk2 + col, a.head_dim, a.scale, n > 0, seen, live);
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && n > 0) mbar_arrive(&o_empty);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && abort_flag && a.status) atomicOr(reinterpret_cast<unsigned *>(a.status), E2EGREC_DEV_TIMEOUT);
    if (warp == 10) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// ------------------------------------------------------------------------------------------------- host side
constexpr int kMaxDevices = 64;
template <typename Kernel> bool allow_smem(Kernel kernel, size_t bytes, std::atomic<bool> (&done)[kMaxDevices])
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return false;
    if (done[dev]) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return false;
    done[dev] = true;
    return true;
}

// A matrix of heads as (column of a head, head, row); box: 64 columns of `box_heads` heads of 128 / box_heads rows, 128-byte swizzle
bool make_map(CUtensorMap *map, const void *base, int64_t rows, int heads, int head_dim, int64_t ld, int box_heads)
{
    TensorMapEncodeFn fn = tensor_map_encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)rows};
    const cuuint64_t strides[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)ld * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)(kTile / box_heads)};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Maps of Q, K, V and (backward) dO; false where one cannot be made
struct Maps {
    CUtensorMap q, k, v, g;
    int boxes;
};
bool make_maps(const AttnArgs &a, Maps &m)
{
    m.boxes = kTile % a.group == 0;
    const int box = m.boxes ? a.group : 1, heads = a.kv_heads * a.group;
    if (!make_map(&m.q, a.q, a.q_rows, heads, a.head_dim, a.ldq, box) || !make_map(&m.k, a.k, a.k_rows, a.kv_heads, a.head_dim, a.ldk, 1) ||
        !make_map(&m.v, a.v, a.k_rows, a.kv_heads, a.head_dim, a.ldv, 1))
        return false;
    m.g = m.q;
    return !a.dout || make_map(&m.g, a.dout, a.q_rows, heads, a.head_dim, a.ldg, box);
}

// Small units in numbers go to as many blocks as the machine holds, which prefetch from unit to unit; fewer units get a block each,
// so that the hardware hands them out as blocks end.
uint32_t tc_grid(uint32_t units, int blocks) { return units >= 8u * kSms * blocks ? kSms * blocks : units; }

template <int NB, int NT> bool launch_fwd(const AttnArgs &a, const Maps &m, const TcShape &f, float *part_o, float2 *part_ml, cudaStream_t st)
{
    static std::atomic<bool> done[kMaxDevices] = {};
    using F = Fwd<NB, NT>;
    if (!allow_smem(attn_tc_fwd_kernel<NB, NT>, F::kSmem, done)) return false;
    note_launch();
    attn_tc_fwd_kernel<NB, NT><<<tc_grid(f.units, F::kBlocks), F::kThreads, F::kSmem, st>>>(m.q, m.k, m.v, a, f, part_o, part_ml);
    return true;
}

template <int NB> bool launch_bwd(const AttnArgs &a, const Maps &m, int64_t q_tiles, int64_t k_tiles, float *dots, cudaStream_t st)
{
    static std::atomic<bool> done[2][kMaxDevices] = {};
    using B = Bwd<NB>;
    if (!allow_smem(attn_tc_dq_kernel<NB>, B::kDqSmem, done[0]) || !allow_smem(attn_tc_dkv_kernel<NB>, B::kDkvSmem, done[1])) return false;
    const int64_t units = a.n_seq * a.kv_heads;
    const TcShape fq{(uint32_t)(units * q_tiles), (int)q_tiles, 1, m.boxes}, fk{(uint32_t)(units * k_tiles), (int)k_tiles, 1, m.boxes};
    note_launch();
    attn_tc_dq_kernel<NB><<<tc_grid(fq.units, 1), B::kThreads, B::kDqSmem, st>>>(m.q, m.g, m.k, m.v, a, fq, dots);
    note_launch();
    attn_tc_dkv_kernel<NB><<<tc_grid(fk.units, 1), B::kThreads, B::kDkvSmem, st>>>(m.q, m.g, m.k, m.v, a, fk, dots);
    return true;
}

}  // namespace

bool tc_attention_forward(const AttnArgs &a, int64_t tiles, int splits, bool one_tile, float *part_o, float2 *part_ml, cudaStream_t st)
{
    Maps m;
    if (!make_maps(a, m)) return false;
    const TcShape f{(uint32_t)(a.n_seq * a.kv_heads * tiles * splits), (int)tiles, splits, m.boxes};
    if (a.head_dim <= 64) return one_tile ? launch_fwd<1, 1>(a, m, f, part_o, part_ml, st) : launch_fwd<1, 2>(a, m, f, part_o, part_ml, st);
    return one_tile ? launch_fwd<2, 1>(a, m, f, part_o, part_ml, st) : launch_fwd<2, 2>(a, m, f, part_o, part_ml, st);
}

bool tc_attention_backward(const AttnArgs &a, int64_t q_tiles, int64_t k_tiles, float *dots, cudaStream_t st)
{
    Maps m;
    if (!make_maps(a, m)) return false;
    return a.head_dim <= 64 ? launch_bwd<1>(a, m, q_tiles, k_tiles, dots, st) : launch_bwd<2>(a, m, q_tiles, k_tiles, dots, st);
}

}  // namespace e2egrec
