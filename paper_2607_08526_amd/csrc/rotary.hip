// Rotary positions: of each head's first `rot` channels, the pairs (a, b) =
// (x[j], x[j + rot / 2]) (half layout) or (x[2 j], x[2 j + 1]) (interleaved),
// j < rot / 2, are turned by the angle t = position * freq[j]:
//
//   a' = m (a cos t - b sin t),   b' = m (b cos t + a sin t)
//
// and the other channels kept.  The adjoint (the backward pass: the gradient of
// x from that of the output) turns by -t.
//
// Angles: positions of long contexts leave an fp32 angle no fractional digits
// (2^20 radians: 2^-4), so the angle is formed in fp64, in turns, and reduced
// to [-1/2, 1/2] there.  Plain fp64 products are off by up to 2^-24 of a turn near position
// 2^31, more than what follows, so frequencies in turns have two terms and whole turns
// are taken off the unrounded product: positions to 2^31 are as exact as 0.  The reduced
// angle is rounded to fp32 (2^-26 of a turn at most) for its sine and cosine in fp32,
// whose own steps are as large.
//
// Bound: HBM (every channel read and written once).  A workgroup takes a few rows
// at a time and computes their angles once, in LDS, for all heads; a thread turns
// pairs of 16-byte vectors (half layout) or the pairs inside one (interleaved) at
// places that stay the same from one group of rows to the next, whose vectors are
// loaded and whose angles are formed before the present ones are stored.  8192 rows
// of 64 heads of 64, 32 channels turned, bf16: 134 MB in 25.9 us
// (5.2 TB/s, a large copy's rate) where the caches are warm, 33.0 us as a cold call.
// Four items a thread take 150 registers and 29 us.  Sizes and
// alignments that leave no whole vectors go pair by pair, each with an angle of its
// own.
#include <algorithm>

#include "internal.h"
#include "mx.h"

namespace qlk {
namespace {

constexpr int THREADS = 256;
constexpr int TABLE = 512;  // (cos, sin) pairs of a group of rows
constexpr int NI = 2;       // items of a group per thread

template <bool BF16>
struct Elem {
    using T = typename std::conditional<BF16, uint16_t, float>::type;
    static constexpr int V = BF16 ? 8 : 4;  // elements of a 16-byte vector
    static __device__ inline float get(T v)
    {
        if constexpr (BF16)
            return __uint_as_float((uint32_t)v << 16);
        else
            return v;
    }
    static __device__ inline T put(float v)
    {
        if constexpr (BF16)
            return (T)mx_pack_bf16(v, v);
        else
            return v;
    }
};

__device__ inline int64_t position(const RotaryArgs &a, int64_t row)
{
    return a.positions ? a.positions[row] : a.start + row % a.period;
}

// a frequency in turns per position, as a sum
struct Turns {
    double hi, lo;
};
__device__ inline Turns in_turns(double freq)
{
    constexpr double HI = 0x1.45f306dc9c883p-3, LO = -0x1.6b01ec5417056p-57;  // 1 / (2 pi)
    const double h = freq * HI;
    return Turns{h, __builtin_fma(freq, HI, -h) + freq * LO};
}

// mscale times cosine and sine of the angle at a position
__device__ inline mx_f32x2 angle(const RotaryArgs &a, int64_t pos, Turns freq)
{
    const double p = (double)pos, whole = __builtin_rint(p * freq.hi);
    const float f = (float)(__builtin_fma(p, freq.hi, -whole) + p * freq.lo);
    float s, c;
    sincospif(2.0f * f, &s, &c);
    return mx_f32x2{c * a.mscale, (a.adjoint ? -s : s) * a.mscale};
}

template <bool BF16, bool INTER>
__global__ __launch_bounds__(THREADS) void rotary_kernel(const RotaryArgs a)
{
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int V = E::V;
    typedef T vec __attribute__((ext_vector_type(V)));
    __shared__ mx_f32x2 table[2][TABLE];
    const int half = a.rot / 2;
    // items of a head: pairs of vectors (half layout) or vectors, then those kept
    const int turns = INTER ? a.rot / V : half / V;
    const int per_head = turns + (a.copy ? (a.dh - a.rot) / V : 0);
    const int head0 = blockIdx.y * a.heads_per_wg;
    const int per_row = per_head * min(a.heads_per_wg, a.heads - head0), R = a.rows_per_wg;
    const int64_t stride = (int64_t)gridDim.x * R;
    int64_t row0 = (int64_t)blockIdx.x * R;

    // this thread's items: row of the group, and the channels of both vectors in it
    // (cb < 0: one vector), and the first angle (j0 < 0: kept)
    int ir[NI], ca[NI], cb[NI], j0[NI];
#pragma unroll
    for (int k = 0; k < NI; ++k) {
        const int i = threadIdx.x + k * THREADS;
        const int r = i / per_row, q = i - r * per_row;
        const int h0 = q / per_head, u = q - h0 * per_head, h = head0 + h0;
        ir[k] = r;  // (>= R: none)
        if (u >= turns) {
            ca[k] = h * a.dh + a.rot + (u - turns) * V;
            cb[k] = j0[k] = -1;
        } else {
            ca[k] = h * a.dh + u * V;
            cb[k] = INTER ? -1 : h * a.dh + half + u * V;
            j0[k] = INTER ? u * V / 2 : u * V;
        }
    }
    // and its angles: of row am of the group, pair aj
    const int ai = threadIdx.x;
    const bool mine2 = ai + THREADS < R * half;
    int am[2], aj[2];
    Turns fr[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = ai + k * THREADS;
        am[k] = i / half;
        aj[k] = i - am[k] * half;
        fr[k] = in_turns(i < R * half ? a.freqs[aj[k]] : 0.0);
    }
    const T *const x = static_cast<const T *>(a.x);
    T *const o = static_cast<T *>(a.o);
    vec va[2][NI], vb[2][NI];
    // (positions first: the vectors need not be there for the angles)
    auto load = [&](int64_t first, int buf) {
        int64_t pos[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (ai + k * THREADS < R * half && first + am[k] < a.rows)
                pos[k] = position(a, first + am[k]);
#pragma unroll
        for (int k = 0; k < NI; ++k)
            if (ir[k] < R && first + ir[k] < a.rows) {
                const T *const p = x + (first + ir[k]) * a.ldx;
                va[buf][k] = *reinterpret_cast<const vec *>(p + ca[k]);
                if (cb[k] >= 0)
                    vb[buf][k] = *reinterpret_cast<const vec *>(p + cb[k]);
            }
        if (ai < R * half)
            table[buf][ai] = angle(a, pos[0], fr[0]);
        if (mine2)
            table[buf][ai + THREADS] = angle(a, pos[1], fr[1]);
    };
    auto turn = [&](int64_t first, int buf) {
#pragma unroll
        for (int k = 0; k < NI; ++k) {
            if (ir[k] >= R || first + ir[k] >= a.rows)
                continue;
            T *const p = o + (first + ir[k]) * a.ldo;
            const vec v = va[buf][k];
            if (j0[k] < 0) {
                *reinterpret_cast<vec *>(p + ca[k]) = v;
                continue;
            }
            const mx_f32x2 *const cs = &table[buf][ir[k] * half + j0[k]];
            vec w, z;
            if constexpr (INTER) {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const mx_f32x2 t = cs[e / 2];
                    const float f = E::get(v[e]), s = E::get(v[e + 1]);
                    w[e] = E::put(f * t[0] - s * t[1]);
                    w[e + 1] = E::put(s * t[0] + f * t[1]);
                }
            } else {
                const vec y = vb[buf][k];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const mx_f32x2 t = cs[e];
                    const float f = E::get(v[e]), s = E::get(y[e]);
                    w[e] = E::put(f * t[0] - s * t[1]);
                    z[e] = E::put(s * t[0] + f * t[1]);
                }
                *reinterpret_cast<vec *>(p + cb[k]) = z;
            }
            *reinterpret_cast<vec *>(p + ca[k]) = w;
        }
    };
    // (two groups at a time: the buffers are known at compile time)
    load(row0, 0);
    __syncthreads();
    for (; row0 < a.rows; row0 += 2 * stride) {
        if (row0 + stride < a.rows)
            load(row0 + stride, 1);
        turn(row0, 0);
        __syncthreads();
        if (row0 + 2 * stride < a.rows)
            load(row0 + 2 * stride, 0);
        if (row0 + stride < a.rows)
            turn(row0 + stride, 1);
        __syncthreads();
    }
}

// One pair of channels, or one kept channel, per thread and step.
template <bool BF16>
__global__ __launch_bounds__(THREADS) void rotary_pairs_kernel(const RotaryArgs a)
{
    using E = Elem<BF16>;
    using T = typename E::T;
    const int half = a.rot / 2, per_head = half + (a.copy ? a.dh - a.rot : 0);
    const int64_t per_row = (int64_t)per_head * a.heads, items = a.rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < items;
         i += (int64_t)gridDim.x * THREADS) {
        const int64_t row = i / per_row;
        const int q = (int)(i - row * per_row), h = q / per_head, u = q - h * per_head;
        const T *const x = static_cast<const T *>(a.x) + row * a.ldx + (int64_t)h * a.dh;
        T *const o = static_cast<T *>(a.o) + row * a.ldo + (int64_t)h * a.dh;
        if (u >= half) {
            o[a.rot + u - half] = x[a.rot + u - half];
            continue;
        }
        const mx_f32x2 t = angle(a, position(a, row), in_turns(a.freqs[u]));
        const int ca = a.interleaved ? 2 * u : u, cb = a.interleaved ? 2 * u + 1 : u + half;
        const float f = E::get(x[ca]), s = E::get(x[cb]);
        o[ca] = E::put(f * t[0] - s * t[1]);
        o[cb] = E::put(s * t[0] + f * t[1]);
    }
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int cus, hipStream_t stream)
{
    const int V = a.bf16 ? 8 : 4, half = a.rot / 2;
    const uintptr_t size = a.bf16 ? 2 : 4;
    const int per_head =
        (a.interleaved ? a.rot : half) / V + (a.copy ? (a.dh - a.rot) / V : 0);
    const bool vec = (a.interleaved ? a.rot : half) % V == 0 && a.dh % V == 0 && a.rot % V == 0 &&
                     ((uintptr_t)a.x & 15) == 0 && ((uintptr_t)a.o & 15) == 0 &&
                     a.ldx * size % 16 == 0 && a.ldo * size % 16 == 0 && half <= TABLE &&
                     per_head <= NI * THREADS &&
                     (a.heads - 1) / (NI * THREADS / per_head) < 65535;
    const dim3 block(THREADS);
    if (!vec) {
        const int64_t items =
            a.rows * a.heads * (int64_t)(half + (a.copy ? a.dh - a.rot : 0));
        const dim3 grid((unsigned)std::min<int64_t>((items + THREADS - 1) / THREADS, 1 << 16));
        if (a.bf16)
            hipLaunchKernelGGL(rotary_pairs_kernel<true>, grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL(rotary_pairs_kernel<false>, grid, block, 0, stream, a);
        return hipGetLastError();
    }
    // heads at a time: all, or equal parts that the threads' items hold
    const int fit = NI * THREADS / per_head, parts = (a.heads + fit - 1) / fit;
    a.heads_per_wg = (a.heads + parts - 1) / parts;
    const int per_row = a.heads_per_wg * per_head;
    // rows at a time: as many as the threads' items and the table hold, while every
    // CU has work; eight workgroups a CU
    int64_t rpw = std::min<int64_t>(NI * THREADS / per_row, TABLE / half);
    rpw = std::max<int64_t>(1, std::min<int64_t>(rpw, a.rows * parts / cus));
    a.rows_per_wg = (int)rpw;
    const dim3 grid((unsigned)std::min<int64_t>((a.rows + rpw - 1) / rpw,
                                                std::max(1, 8 * cus / parts)),
                    (unsigned)((a.heads + a.heads_per_wg - 1) / a.heads_per_wg));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    if (a.bf16)
        a.interleaved ? go(rotary_kernel<true, true>) : go(rotary_kernel<true, false>);
    else
        a.interleaved ? go(rotary_kernel<false, true>) : go(rotary_kernel<false, false>);
    return hipGetLastError();
}

}  // namespace qlk
