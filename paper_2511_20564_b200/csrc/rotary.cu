// Rotary positions of the heads of a matrix, and the root-mean-square norm of every head with the rotation in the same pass.
//
//   n = x / sqrt(mean(x^2) + eps),  g_i = w_i n_i,  (y_a, y_b) = scale (g_a cos t - g_b sin t, g_b cos t + g_a sin t),  t = pos f_i
//   over the pairs (a, b) = (i, i + rot / 2) or (2 i, 2 i + 1), i < rot / 2; elements behind rot are passed through as g.
// Gradient, with u = the inverse rotation of dy:  dw = sum u n,  dx = (u w - n mean(u w n)) / sqrt(mean(x^2) + eps).
//
// What bounds these kernels is memory: a row is read once and written once (the gradient reads x and dy).  A thread takes one unit of
// 16 bytes and its partner 16 bytes (the other elements of the pairs) of one row and goes over the heads of the row, so that the
// angles of its pairs are formed once per row; the lanes of one head are neighbours, and a head's sum of squares is a handful of
// shuffles.  (One thread per unit and head, whose accesses are whole lines, forms every angle once per head: 21 us instead of 15
// for 65 536 rows of 4 heads of 64 bf16 values.)
// Angles: a frequency becomes a 64-bit fraction of a turn, once per block and pair (1 / 2 pi and the product in two doubles: what one
// product loses a far position multiplies, 2^-25 of a turn for 1 radian per position and 2^-15 for a thousand); its product with a 32-bit
// position modulo one turn is two integer products, exact to 2^-32 of a turn wherever the position lies, where a product in 32-bit
// floating point has no digit left beyond position 2^23.
#include <algorithm>

#include "common.cuh"

namespace e2egrec {
namespace {

constexpr int kRotThreads = 256;
constexpr int kHeadUnroll = 2;            // heads of a row whose loads are in flight together
constexpr int kMaxHeadDim = 256;
constexpr int kGradUnroll = 1;            // the same in the gradient's kernel
constexpr int kGradBlocks = 148 * 4;      // blocks that sum up the gains' gradients, at most

// V values of a row as they lie in memory (16, 8, 4 or 2 bytes)
template <int BYTES> struct RawOf;
template <> struct RawOf<16> { using type = uint4; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<2> { using type = uint16_t; };
template <typename T, int V> using Raw = typename RawOf<V * (int)sizeof(T)>::type;

template <typename T, int V> __device__ inline void widen(const Raw<T, V> &r, float *v)
{
    if constexpr (sizeof(T) == 2 && V > 1) {         // two bf16 values of a word: a shift and a mask
        uint32_t w[V / 2];
        memcpy(w, &r, sizeof(r));
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
        T e[V];
        memcpy(e, &r, sizeof(r));
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = to_float<T>(e[i]);
    }
}
template <typename T, int V> __device__ inline Raw<T, V> narrow(const float *v)
{
    Raw<T, V> r;
    if constexpr (sizeof(T) == 2 && V > 1) {
        uint32_t w[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            memcpy(&w[i], &h, 4);
        }
        memcpy(&r, w, sizeof(r));
    } else {
        T e[V];
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = from_float<T>(v[i]);
        memcpy(&r, e, sizeof(r));
    }
    return r;
}

// One operand: rows x heads x head_dim, its gradient's input and the result.
struct Operand {
    const void *x, *dy;
    void *y;
    int64_t ldx, ldd, ldy, rows;
    int32_t heads;
    const float *w;
    const int32_t *pos;
    float *dw;                            // partial sums of the gain's gradient, [blocks x head_dim], or null
};

struct RotArgs {
    Operand op[2];
    int32_t blocks0;                      // blocks of the first operand
    int32_t head_dim, half, lanes;        // half = rot / 2; lanes per head: a power of two
    int32_t heads_per;                    // heads per block of the grid's second dimension
    const double *freqs;
    float scale, sign, eps;
};

// Places of a thread's units.  V values per unit, E / V units per thread, `lanes` apart; a unit is two stretches of V values.
template <int V, bool kInter> struct Places {
    int a, b;                             // first elements of the two stretches, -1 where there is none
    int f;                                // the first of its V pairs
    __device__ inline Places(int su, int half, int head_dim)
    {
        if (kInter) {
            a = 2 * su * V;
            b = a + V;
            f = su * V;
        } else if (su * V < half) {
            a = su * V;
            b = a + half;
            f = su * V;
        } else {                          // behind the rotated part: neighbours, passed through
            a = 2 * half + 2 * (su * V - half);
            b = a + V;
            f = half;
        }
        if (a >= head_dim) a = -1;
        if (b >= head_dim) b = -1;
    }
};

// The block's table of turns per position, 2^64 to a turn: high and low words
__device__ inline void make_turns(const RotArgs &r, uint2 *turns)
{
    for (int f = threadIdx.x; f < r.half; f += kRotThreads) {
        const double freq = __ldg(r.freqs + f), hi = 0.15915494309189535, lo = -9.839338337591243e-18;      // 1 / 2 pi = hi + lo
        const double t = freq * hi, rest = fma(freq, lo, fma(freq, hi, -t));
        const unsigned long long n = __double2ull_rz((t - floor(t)) * 18446744073709551616.0) + (unsigned long long)__double2ll_rn(rest * 18446744073709551616.0);
        turns[f] = make_uint2((uint32_t)(n >> 32), (uint32_t)n);
    }
    __syncthreads();
}

// scale * (cos, sin) of pair f at position p; (1, 0) for pairs that are not rotated.  With 16-bit results the hardware's sine and
// cosine of the angle to 2^-24 of a turn are off by less than 2^-19.8, a 2^10th of the result's own rounding.  For 32-bit results the angle is
// taken to the nearest quarter turn, |x| <= pi / 4, and the Taylor series of sine and cosine broken off behind x^9 and x^8 (the next terms
// are below 2^-28 and 2^-25); the quarter turns swap the two and set signs.
template <typename T> __device__ inline void angle(const RotArgs &r, const uint2 *turns, int f, int p, float &c, float &s)
{
    c = 1.f;
    s = 0.f;
    if (f >= r.half) return;
    const uint2 t = turns[f];
    const uint32_t frac = t.x * (uint32_t)p + __umulhi(t.y, (uint32_t)p) - (p < 0 ? t.y : 0u);      // of 2^32, modulo a turn
    if (sizeof(T) == 2) {
        // 1.5 + the signed fraction of a turn, from the bits, rounded to 23 of them (half a turn up may come out as half a turn down)
        const float a = (__uint_as_float(0x3F800000u | ((frac + 0x80000100u) >> 9)) - 1.5f) * 6.28318530718f;
        c = __cosf(a);
        s = __sinf(a);
    } else {
        const uint32_t quarter = (frac + 0x20000000u) >> 30;
        const float x = (float)(int32_t)(frac - (quarter << 30)) * 1.46291807926715968105e-9f, x2 = x * x;      // 2 pi / 2^32
        const float sx = fmaf(fmaf(fmaf(fmaf(1.f / 362880.f, x2, -1.f / 5040.f), x2, 1.f / 120.f), x2, -1.f / 6.f) * x2, x, x);
        const float cx = fmaf(fmaf(fmaf(fmaf(1.f / 40320.f, x2, -1.f / 720.f), x2, 1.f / 24.f), x2, -0.5f), x2, 1.f);
        s = __uint_as_float(__float_as_uint(quarter & 1u ? cx : sx) ^ ((quarter & 2u) << 30));
        c = __uint_as_float(__float_as_uint(quarter & 1u ? sx : cx) ^ (((quarter + 1u) & 2u) << 30));
    }
    c *= r.scale;
    s *= r.scale * r.sign;
}

// The stretches of V values from pa and pb on; what lies behind the rotated part stays as it is (a product with sin 0 = 0 would pass on
// infinities and NaN of a neighbour).
template <bool kInter, int V> __device__ inline void turn_unit(float *a, float *b, const float *c, const float *s, int pa, int pb, int half)
{
    if (kInter) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float u = a[i] * c[i / 2] - a[i + 1] * s[i / 2], v = a[i + 1] * c[i / 2] + a[i] * s[i / 2];
            const float w = b[i] * c[V / 2 + i / 2] - b[i + 1] * s[V / 2 + i / 2], x = b[i + 1] * c[V / 2 + i / 2] + b[i] * s[V / 2 + i / 2];
            const bool first = pa + i < 2 * half, second = pb + i < 2 * half;
            a[i] = first ? u : a[i];
            a[i + 1] = first ? v : a[i + 1];
            b[i] = second ? w : b[i];
            b[i + 1] = second ? x : b[i + 1];
        }
    } else if (pa < half) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float u = a[i] * c[i] - b[i] * s[i], v = b[i] * c[i] + a[i] * s[i];
            a[i] = u;
            b[i] = v;
        }
    }
}

__device__ inline float lanes_sum(float v, int lanes)
{
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Forward: rotation, with kNorm the norm before it.
template <typename T, int V, bool kInter, bool kNorm>
__global__ void __launch_bounds__(kRotThreads, 3)
rotary_kernel(const __grid_constant__ RotArgs r)
{
    constexpr int E = Chunk<T>::kElems, NU = E / V;
    const bool second = (int)blockIdx.x >= r.blocks0;
    const Operand &op = r.op[second];
    const int h0 = blockIdx.y * r.heads_per, h1 = min(h0 + r.heads_per, op.heads);
    if (h0 >= h1) return;
    const int lane = threadIdx.x & (r.lanes - 1);
    const int64_t row = (int64_t)(blockIdx.x - (second ? r.blocks0 : 0)) * (kRotThreads / r.lanes) + threadIdx.x / r.lanes;
    const bool live = row < op.rows;
    const int p = !live ? 0 : (op.pos ? __ldg(op.pos + row) : (int)row);
    __shared__ uint2 turns[kMaxHeadDim / 2];
    make_turns(r, turns);

    int pa[NU], pb[NU];
    float c[E], s[E], wa[E], wb[E];
#pragma unroll
    for (int j = 0; j < NU; ++j) {
        const Places<V, kInter> at(lane + j * r.lanes, r.half, r.head_dim);
        pa[j] = live ? at.a : -1;
        pb[j] = live ? at.b : -1;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            angle<T>(r, turns, at.f + i, p, c[j * V + i], s[j * V + i]);
            if (kNorm) {
                wa[j * V + i] = op.w && at.a >= 0 ? __ldg(op.w + at.a + i) : 1.f;
                wb[j * V + i] = op.w && at.b >= 0 ? __ldg(op.w + at.b + i) : 1.f;
            }
        }
    }
    const T *x = static_cast<const T *>(op.x) + row * op.ldx;
    T *y = static_cast<T *>(op.y) + row * op.ldy;
    for (int h = h0; h < h1; h += kHeadUnroll) {
        Raw<T, V> ra[kHeadUnroll][NU], rb[kHeadUnroll][NU];
#pragma unroll
        for (int u = 0; u < kHeadUnroll; ++u)
#pragma unroll
            for (int j = 0; j < NU; ++j) {
                ra[u][j] = Raw<T, V>{};
                rb[u][j] = Raw<T, V>{};
                if (h + u < h1 && pa[j] >= 0) ra[u][j] = *reinterpret_cast<const Raw<T, V> *>(x + (int64_t)(h + u) * r.head_dim + pa[j]);
                if (h + u < h1 && pb[j] >= 0) rb[u][j] = *reinterpret_cast<const Raw<T, V> *>(x + (int64_t)(h + u) * r.head_dim + pb[j]);
            }
#pragma unroll
        for (int u = 0; u < kHeadUnroll; ++u) {
            if (h + u >= h1) break;
            float a[E], b[E];
            float q = 0.f;
#pragma unroll
            for (int j = 0; j < NU; ++j) {
                widen<T, V>(ra[u][j], a + j * V);
                widen<T, V>(rb[u][j], b + j * V);
            }
            if (kNorm) {
#pragma unroll
                for (int i = 0; i < E; ++i) q += a[i] * a[i] + b[i] * b[i];
                const float rs = rsqrtf(lanes_sum(q, r.lanes) / (float)r.head_dim + r.eps);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    a[i] *= rs * wa[i];
                    b[i] *= rs * wb[i];
                }
            }
#pragma unroll
            for (int j = 0; j < NU; ++j) {
                turn_unit<kInter, V>(a + j * V, b + j * V, c + j * V, s + j * V, pa[j], pb[j], r.half);
                if (pa[j] >= 0) *reinterpret_cast<Raw<T, V> *>(y + (int64_t)(h + u) * r.head_dim + pa[j]) = narrow<T, V>(a + j * V);
                if (pb[j] >= 0) *reinterpret_cast<Raw<T, V> *>(y + (int64_t)(h + u) * r.head_dim + pb[j]) = narrow<T, V>(b + j * V);
            }
        }
    }
}

// Gradient of the normed form.  The blocks of an operand go over its rows in rounds; a thread's share of the gains'
// gradient stays in registers, the block adds its threads' up in a fixed order and leaves one row of partial sums.
template <typename T, int V, bool kInter>
__global__ void __launch_bounds__(kRotThreads, 2)
qk_norm_grad_kernel(const __grid_constant__ RotArgs r)
{
    constexpr int E = Chunk<T>::kElems, NU = E / V;
    __shared__ float part[kRotThreads / 32][kMaxHeadDim];
    __shared__ uint2 turns[kMaxHeadDim / 2];
    make_turns(r, turns);
    const bool second = (int)blockIdx.x >= r.blocks0;
    const Operand &op = r.op[second];
    const int block = (int)blockIdx.x - (second ? r.blocks0 : 0), blocks = second ? (int)gridDim.x - r.blocks0 : r.blocks0;
    const int lane = threadIdx.x & (r.lanes - 1), per_block = kRotThreads / r.lanes;
    int pa[NU], pb[NU], pf[NU];
    float wa[E], wb[E], ga[E], gb[E];
#pragma unroll
    for (int j = 0; j < NU; ++j) {
        const Places<V, kInter> at(lane + j * r.lanes, r.half, r.head_dim);
        pa[j] = at.a;
        pb[j] = at.b;
        pf[j] = at.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            wa[j * V + i] = op.w && at.a >= 0 ? __ldg(op.w + at.a + i) : 1.f;
            wb[j * V + i] = op.w && at.b >= 0 ? __ldg(op.w + at.b + i) : 1.f;
            ga[j * V + i] = gb[j * V + i] = 0.f;
        }
    }
    const int64_t rounds = ceil_div(ceil_div(op.rows, per_block), blocks);
    for (int64_t n = 0; n < rounds; ++n) {
        const int64_t row = (n * blocks + block) * per_block + threadIdx.x / r.lanes;
        const bool live = row < op.rows;
        const int p = !live ? 0 : (op.pos ? __ldg(op.pos + row) : (int)row);
        const T *x = static_cast<const T *>(op.x) + row * op.ldx, *dy = static_cast<const T *>(op.dy) + row * op.ldd;
        T *dx = static_cast<T *>(op.y) + row * op.ldy;
        float c[E], s[E];
        for (int h = 0; h < op.heads; h += kGradUnroll) {
            Raw<T, V> r0[kGradUnroll][NU], r1[kGradUnroll][NU], r2[kGradUnroll][NU], r3[kGradUnroll][NU];
#pragma unroll
            for (int u = 0; u < kGradUnroll; ++u) {
                const bool on = live && h + u < op.heads;
                const int64_t off = (int64_t)(h + u) * r.head_dim;
#pragma unroll
                for (int j = 0; j < NU; ++j) {
                    r0[u][j] = r1[u][j] = r2[u][j] = r3[u][j] = Raw<T, V>{};
                    if (on && pa[j] >= 0) {
                        r0[u][j] = *reinterpret_cast<const Raw<T, V> *>(x + off + pa[j]);
                        r2[u][j] = *reinterpret_cast<const Raw<T, V> *>(dy + off + pa[j]);
                    }
                    if (on && pb[j] >= 0) {
                        r1[u][j] = *reinterpret_cast<const Raw<T, V> *>(x + off + pb[j]);
                        r3[u][j] = *reinterpret_cast<const Raw<T, V> *>(dy + off + pb[j]);
                    }
                }
            }
            if (h == 0) {
#pragma unroll
                for (int j = 0; j < NU; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) angle<T>(r, turns, pf[j] + i, p, c[j * V + i], s[j * V + i]);
            }
#pragma unroll
            for (int u = 0; u < kGradUnroll; ++u) {
                if (h + u >= op.heads) break;
                const int64_t off = (int64_t)(h + u) * r.head_dim;
                float a[E], b[E], da[E], db[E];
#pragma unroll
                for (int j = 0; j < NU; ++j) {
                    widen<T, V>(r0[u][j], a + j * V);
                    widen<T, V>(r1[u][j], b + j * V);
                    widen<T, V>(r2[u][j], da + j * V);
                    widen<T, V>(r3[u][j], db + j * V);
                    turn_unit<kInter, V>(da + j * V, db + j * V, c + j * V, s + j * V, pa[j], pb[j], r.half);
                }
                float q = 0.f, d = 0.f;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    q += a[i] * a[i] + b[i] * b[i];
                    d += da[i] * wa[i] * a[i] + db[i] * wb[i] * b[i];
                }
                q = lanes_sum(q, r.lanes);
                d = lanes_sum(d, r.lanes);
                const float rs = live ? rsqrtf(q / (float)r.head_dim + r.eps) : 0.f;      // (with eps = 0 no inverse of the zeros of no row)
                const float m = d * rs * rs * rs / (float)r.head_dim;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    ga[i] += da[i] * a[i] * rs;
                    gb[i] += db[i] * b[i] * rs;
                    a[i] = da[i] * wa[i] * rs - a[i] * m;
                    b[i] = db[i] * wb[i] * rs - b[i] * m;
                }
#pragma unroll
                for (int j = 0; j < NU; ++j) {
                    if (live && pa[j] >= 0) *reinterpret_cast<Raw<T, V> *>(dx + off + pa[j]) = narrow<T, V>(a + j * V);
                    if (live && pb[j] >= 0) *reinterpret_cast<Raw<T, V> *>(dx + off + pb[j]) = narrow<T, V>(b + j * V);
                }
            }
        }
    }
    if (!op.dw) return;
    // rows of one warp by shuffles, the warps through shared memory
#pragma unroll
    for (int i = 0; i < E; ++i)
        for (int o = r.lanes; o < 32; o <<= 1) {
            ga[i] += __shfl_xor_sync(0xFFFFFFFFu, ga[i], o);
            gb[i] += __shfl_xor_sync(0xFFFFFFFFu, gb[i], o);
        }
    if ((int)(threadIdx.x & 31) < r.lanes) {
#pragma unroll
        for (int j = 0; j < NU; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (pa[j] >= 0) part[threadIdx.x >> 5][pa[j] + i] = ga[j * V + i];
                if (pb[j] >= 0) part[threadIdx.x >> 5][pb[j] + i] = gb[j * V + i];
            }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < r.head_dim; i += kRotThreads) {
        float t = 0.f;
        for (int w = 0; w < kRotThreads / 32; ++w) t += part[w][i];
        op.dw[(int64_t)block * r.head_dim + i] = t;
    }
}

// Partial sums of the blocks -> dw, in a fixed order: 32 stretches of blocks per element (with eight, 592 blocks took 10 us, 4 now)
constexpr int kGainThreads = 1024;
__global__ void __launch_bounds__(kGainThreads)
gain_grad_kernel(const float *__restrict__ part0, const float *__restrict__ part1, int blocks0, int blocks1, int head_dim, float *__restrict__ dw0,
                 float *__restrict__ dw1)
{
    __shared__ float red[32][33];
    const float *part = blockIdx.y ? part1 : part0;
    float *dw = blockIdx.y ? dw1 : dw0;
    const int blocks = blockIdx.y ? blocks1 : blocks0;
    const int e = blockIdx.x * 32 + (threadIdx.x & 31), g = threadIdx.x >> 5;
    if (!dw) return;
    float t = 0.f;
    if (e < head_dim) {
#pragma unroll 8
        for (int b = g; b < blocks; b += 32) t += part[(int64_t)b * head_dim + e];
    }
    red[threadIdx.x & 31][g] = t;
    __syncthreads();
    t = red[g][threadIdx.x & 31];                    // element g of this block, stretch = lane
    t = lanes_sum(t, 32);
    if ((threadIdx.x & 31) == 0 && (int)blockIdx.x * 32 + g < head_dim) dw[blockIdx.x * 32 + g] = t;
}

// frequencies of the pairs, in radians per position
__global__ void rotary_frequencies_kernel(int half, double base, double factor, double trained, double low, double high, double *freqs)
{
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < half; i += gridDim.x * blockDim.x) {
        const double f = pow(base, -(double)i / half);
        double keep = (trained * f * 0.15915494309189533577 - low) / (high - low);
        keep = factor == 1. ? 1. : (keep < 0. ? 0. : (keep > 1. ? 1. : keep));
        freqs[i] = f * (keep + (1. - keep) / factor);
    }
}

__global__ void __launch_bounds__(kRotThreads) zero_kernel(float *a, float *b, int n)
{
    for (int i = threadIdx.x; i < n; i += kRotThreads) {
        if (a) a[i] = 0.f;
        if (b) b[i] = 0.f;
    }
}

int32_t check_heads(const e2egrec_mat *m, int32_t heads, int32_t head_dim, int32_t dtype, int64_t rows)
{
    if (!m || (!m->data && m->rows > 0)) return E2EGREC_ERR_NULL;
    if (m->dtype != E2EGREC_F32 && m->dtype != E2EGREC_BF16) return E2EGREC_ERR_DTYPE;
    if (m->dtype != dtype) return E2EGREC_ERR_DTYPE;
    if (m->rows < rows || (int64_t)heads * head_dim != m->dim || m->ld < m->dim) return E2EGREC_ERR_ARG;
    const int64_t es = (int64_t)dtype_size(dtype);
    if (head_dim * es % 16 || m->ld * es % 16 || reinterpret_cast<uintptr_t>(m->data) % 16) return E2EGREC_ERR_ALIGN;
    return E2EGREC_OK;
}

int32_t check_rotation(int32_t heads, int32_t head_dim, const double *freqs, int32_t rot_dim, float scale, uint32_t flags, uint32_t known)
{
    if (heads < 1 || head_dim < 1 || rot_dim < 0 || rot_dim > head_dim || rot_dim % 2 || (flags & ~known)) return E2EGREC_ERR_ARG;
    if (!(scale > 0.f) || !(scale <= 3.0e38f)) return E2EGREC_ERR_ARG;
    if (head_dim > kMaxHeadDim) return E2EGREC_ERR_UNSUPPORTED;
    if (rot_dim && !freqs) return E2EGREC_ERR_NULL;
    return E2EGREC_OK;
}

// Widest stretch that a thread can take: pairs half a rotation apart need half to be a multiple of it.
int stretch(int es, int half, bool inter)
{
    int v = 16 / es;
    if (!inter)
        while (half % v) v >>= 1;
    return v;
}

void set_lanes(RotArgs &r, int es)
{
    const int need = (int)ceil_div(r.head_dim, 2 * (16 / es));       // threads of 32 bytes each
    r.lanes = 1;
    while (r.lanes < need) r.lanes <<= 1;
}

template <typename T, bool kNorm>
void launch_forward(const RotArgs &r, int v, bool inter, dim3 grid, cudaStream_t st)
{
    note_launch();
    constexpr int E = Chunk<T>::kElems;
    if (inter) rotary_kernel<T, E, true, kNorm><<<grid, kRotThreads, 0, st>>>(r);
    else if (v == E) rotary_kernel<T, E, false, kNorm><<<grid, kRotThreads, 0, st>>>(r);
    else if (v == E / 2) rotary_kernel<T, E / 2, false, kNorm><<<grid, kRotThreads, 0, st>>>(r);
    else if (v == E / 4) rotary_kernel<T, E / 4, false, kNorm><<<grid, kRotThreads, 0, st>>>(r);
    else rotary_kernel<T, 1, false, kNorm><<<grid, kRotThreads, 0, st>>>(r);
}

template <typename T>
void launch_grad(const RotArgs &r, int v, bool inter, dim3 grid, cudaStream_t st)
{
    note_launch();
    constexpr int E = Chunk<T>::kElems;
    if (inter) qk_norm_grad_kernel<T, E, true><<<grid, kRotThreads, 0, st>>>(r);
    else if (v == E) qk_norm_grad_kernel<T, E, false><<<grid, kRotThreads, 0, st>>>(r);
    else if (v == E / 2) qk_norm_grad_kernel<T, E / 2, false><<<grid, kRotThreads, 0, st>>>(r);
    else if (v == E / 4) qk_norm_grad_kernel<T, E / 4, false><<<grid, kRotThreads, 0, st>>>(r);
    else qk_norm_grad_kernel<T, 1, false><<<grid, kRotThreads, 0, st>>>(r);
}

// Blocks of the forward kernel; heads are spread over the grid's second dimension while rows alone leave SMs without work.
dim3 forward_grid(RotArgs &r)
{
    const int per_block = kRotThreads / r.lanes;
    const int64_t b0 = ceil_div(r.op[0].rows, per_block), b1 = ceil_div(r.op[1].rows, per_block);
    const int heads = std::max(r.op[0].heads, r.op[1].heads);
    int split = 1;
    while (split < heads && (b0 + b1) * split < 148 * 4) split *= 2;
    r.blocks0 = (int32_t)b0;
    r.heads_per = (int32_t)ceil_div(heads, split);
    return dim3((unsigned)(b0 + b1), (unsigned)ceil_div(heads, r.heads_per));
}

Operand operand(const e2egrec_mat *x, const e2egrec_mat *dy, const e2egrec_mat *y, int32_t heads, const float *w, const int32_t *pos)
{
    Operand o{};
    o.x = x->data;
    o.ldx = x->ld;
    o.dy = dy ? dy->data : nullptr;
    o.ldd = dy ? dy->ld : 0;
    o.y = y->data;
    o.ldy = y->ld;
    o.rows = x->rows;
    o.heads = heads;
    o.w = w;
    o.pos = pos;
    return o;
}

constexpr int64_t kMaxRows = (int64_t)1 << 31;

}  // namespace
}  // namespace e2egrec

using namespace e2egrec;

extern "C" int32_t e2egrec_rotary_frequencies(int32_t rot_dim, double base, double factor, double trained_len, double low,
                                              double high, double *freqs, void *stream)
{
    if (rot_dim < 2 || rot_dim % 2 || !(base > 0.) || !(factor >= 1.) || !(high > low) || !(trained_len >= 0.)) return E2EGREC_ERR_ARG;
    if (rot_dim > kMaxHeadDim) return E2EGREC_ERR_UNSUPPORTED;
    if (!freqs) return E2EGREC_ERR_NULL;
    note_launch();
    rotary_frequencies_kernel<<<1, 128, 0, static_cast<cudaStream_t>(stream)>>>(rot_dim / 2, base, factor, trained_len, low, high, freqs);
    return check_launch("rotary_frequencies");
}

extern "C" int32_t e2egrec_rotary(const e2egrec_mat *X, int32_t n_heads, const double *freqs, int32_t rot_dim, const int32_t *pos,
                                  float scale, uint32_t flags, const e2egrec_mat *Y, void *stream)
{
    if (!X || !Y) return E2EGREC_ERR_NULL;
    if (n_heads < 1 || X->dim < 1 || X->dim % n_heads || X->rows < 0 || X->rows >= kMaxRows) return E2EGREC_ERR_ARG;
    const int32_t head_dim = X->dim / n_heads;
    int32_t rc = check_rotation(n_heads, head_dim, freqs, rot_dim, scale, flags, E2EGREC_ROTARY_INTERLEAVED | E2EGREC_ROTARY_INVERSE);
    if (rc == E2EGREC_OK) rc = check_heads(X, n_heads, head_dim, X->dtype, 0);
    if (rc == E2EGREC_OK) rc = check_heads(Y, n_heads, head_dim, X->dtype, X->rows);
    if (rc != E2EGREC_OK || X->rows == 0) return rc;
    RotArgs r{};
    r.op[0] = operand(X, nullptr, Y, n_heads, nullptr, pos);
    r.head_dim = head_dim;
    r.half = rot_dim / 2;
    r.freqs = freqs;
    r.scale = scale;
    r.sign = (flags & E2EGREC_ROTARY_INVERSE) ? -1.f : 1.f;
    const bool inter = flags & E2EGREC_ROTARY_INTERLEAVED, f32 = X->dtype == E2EGREC_F32;
    set_lanes(r, f32 ? 4 : 2);
    const int v = stretch(f32 ? 4 : 2, r.half, inter);
    const dim3 grid = forward_grid(r);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (f32) launch_forward<float, false>(r, v, inter, grid, st);
    else launch_forward<__nv_bfloat16, false>(r, v, inter, grid, st);
    return check_launch("rotary");
}

// What the two calls of the normed form check alike; head_dim is left in *hd.
static int32_t check_qk(const e2egrec_mat *Q, const e2egrec_mat *K, int32_t n_heads, int32_t n_kv_heads, float eps, const double *freqs,
                        int32_t rot_dim, float scale, uint32_t flags, int32_t *hd)
{
    if (!Q) return E2EGREC_ERR_NULL;
    if (n_heads < 1 || Q->dim < 1 || Q->dim % n_heads || Q->rows < 0 || Q->rows >= kMaxRows || !(eps >= 0.f)) return E2EGREC_ERR_ARG;
    *hd = Q->dim / n_heads;
    int32_t rc = check_rotation(n_heads, *hd, freqs, rot_dim, scale, flags, E2EGREC_ROTARY_INTERLEAVED);
    if (rc == E2EGREC_OK) rc = check_heads(Q, n_heads, *hd, Q->dtype, 0);
    if (rc == E2EGREC_OK && K) {
        if (n_kv_heads < 1 || K->rows < 0 || K->rows >= kMaxRows) return E2EGREC_ERR_ARG;
        rc = check_heads(K, n_kv_heads, *hd, Q->dtype, 0);
    }
    return rc;
}

extern "C" int32_t e2egrec_qk_norm_rotary_forward(const e2egrec_mat *Q, const e2egrec_mat *K, int32_t n_heads, int32_t n_kv_heads,
                                                  const float *wq, const float *wk, float eps, const double *freqs, int32_t rot_dim,
                                                  const int32_t *pos_q, const int32_t *pos_k, float scale, uint32_t flags,
                                                  const e2egrec_mat *Qn, const e2egrec_mat *Kn, void *stream)
{
    int32_t hd = 0;
    int32_t rc = check_qk(Q, K, n_heads, n_kv_heads, eps, freqs, rot_dim, scale, flags, &hd);
    if (rc == E2EGREC_OK) rc = check_heads(Qn, n_heads, hd, Q->dtype, Q->rows);
    if (rc == E2EGREC_OK && K) rc = check_heads(Kn, n_kv_heads, hd, Q->dtype, K->rows);
    if (rc != E2EGREC_OK || (Q->rows == 0 && (!K || K->rows == 0))) return rc;
    RotArgs r{};
    r.op[0] = operand(Q, nullptr, Qn, n_heads, wq, pos_q);
    if (K) r.op[1] = operand(K, nullptr, Kn, n_kv_heads, wk, pos_k);
    r.head_dim = hd;
    r.half = rot_dim / 2;
    r.freqs = freqs;
    r.scale = scale;
    r.sign = 1.f;
    r.eps = eps;
    const bool inter = flags & E2EGREC_ROTARY_INTERLEAVED, f32 = Q->dtype == E2EGREC_F32;
    set_lanes(r, f32 ? 4 : 2);
    const int v = stretch(f32 ? 4 : 2, r.half, inter);
    const dim3 grid = forward_grid(r);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (f32) launch_forward<float, true>(r, v, inter, grid, st);
    else launch_forward<__nv_bfloat16, true>(r, v, inter, grid, st);
    return check_launch("qk_norm_rotary_forward");
}

extern "C" int32_t e2egrec_qk_norm_rotary_backward(const e2egrec_mat *dQn, const e2egrec_mat *dKn, const e2egrec_mat *Q,
                                                   const e2egrec_mat *K, int32_t n_heads, int32_t n_kv_heads, const float *wq,
                                                   const float *wk, float eps, const double *freqs, int32_t rot_dim,
                                                   const int32_t *pos_q, const int32_t *pos_k, float scale, uint32_t flags,
                                                   const e2egrec_mat *dQ, const e2egrec_mat *dK, float *dwq, float *dwk, void *ws,
                                                   size_t *ws_bytes, void *stream)
{
    if (!ws_bytes) return E2EGREC_ERR_NULL;
    int32_t hd = 0;
    int32_t rc = check_qk(Q, K, n_heads, n_kv_heads, eps, freqs, rot_dim, scale, flags, &hd);
    if (rc != E2EGREC_OK && (ws || rc != E2EGREC_ERR_NULL)) return rc;
    const size_t one = align_up((size_t)(kGradBlocks + 1) * kMaxHeadDim * sizeof(float), 256), need = 2 * one;
    if (!ws) { *ws_bytes = need; return E2EGREC_OK; }
    if (*ws_bytes < need) { *ws_bytes = need; return E2EGREC_ERR_WORKSPACE; }
    if (reinterpret_cast<uintptr_t>(ws) % 256) return E2EGREC_ERR_ALIGN;
    rc = check_heads(dQn, n_heads, hd, Q->dtype, Q->rows);
    if (rc == E2EGREC_OK) rc = check_heads(dQ, n_heads, hd, Q->dtype, Q->rows);
    if (rc == E2EGREC_OK && K) rc = check_heads(dKn, n_kv_heads, hd, Q->dtype, K->rows);
    if (rc == E2EGREC_OK && K) rc = check_heads(dK, n_kv_heads, hd, Q->dtype, K->rows);
    if (rc != E2EGREC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    float *part0 = static_cast<float *>(ws), *part1 = reinterpret_cast<float *>(static_cast<char *>(ws) + one);
    if (!K) dwk = nullptr;
    const int64_t rows = std::max(Q->rows, K ? K->rows : 0);
    if (rows == 0) {
        if (!dwq && !dwk) return E2EGREC_OK;
        note_launch();
        zero_kernel<<<1, kRotThreads, 0, st>>>(dwq, dwk, hd);
        return check_launch("qk_norm_rotary_backward");
    }
    RotArgs r{};
    r.op[0] = operand(Q, dQn, dQ, n_heads, wq, pos_q);
    r.op[0].dw = dwq ? part0 : nullptr;
    if (K) {
        r.op[1] = operand(K, dKn, dK, n_kv_heads, wk, pos_k);
        r.op[1].dw = dwk ? part1 : nullptr;
    }
    r.head_dim = hd;
    r.half = rot_dim / 2;
    r.freqs = freqs;
    r.scale = scale;
    r.sign = -1.f;
    r.eps = eps;
    const bool inter = flags & E2EGREC_ROTARY_INTERLEAVED, f32 = Q->dtype == E2EGREC_F32;
    set_lanes(r, f32 ? 4 : 2);
    const int v = stretch(f32 ? 4 : 2, r.half, inter);
    // the blocks are shared by the operands as their heads are, so that all of them end together
    const int64_t per = kRotThreads / r.lanes, need0 = ceil_div(Q->rows, per), need1 = K ? ceil_div(K->rows, per) : 0;
    const int64_t heads0 = Q->rows * n_heads, heads1 = K ? K->rows * n_kv_heads : 0, all = std::min<int64_t>(kGradBlocks, need0 + need1);
    const int64_t b0 = need0 ? std::min(need0, std::max<int64_t>(1, all * heads0 / (heads0 + heads1))) : 0;
    const int64_t b1 = need1 ? std::min(need1, std::max<int64_t>(1, all - b0)) : 0;
    r.blocks0 = (int32_t)b0;
    const dim3 grid((unsigned)(b0 + b1));
    if (f32) launch_grad<float>(r, v, inter, grid, st);
    else launch_grad<__nv_bfloat16>(r, v, inter, grid, st);
    if (dwq || dwk) {
        note_launch();
        gain_grad_kernel<<<dim3((unsigned)ceil_div(hd, 32), K ? 2 : 1), kGainThreads, 0, st>>>(part0, part1, (int)b0, (int)b1, hd, dwq, dwk);
    }
    return check_launch("qk_norm_rotary_backward");
}
