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
// to [-1/2, 1/2) there; sine and cosine of the reduced angle are fp32.  A
// workgroup computes those of its rows once, in LDS, for all heads.
//
// Bound: HBM (every channel read and written once).  A thread turns a pair of
// 16-byte vectors (half layout) or the pairs inside one (interleaved); sizes
// and alignments that leave no whole vectors go pair by pair.
#include <algorithm>

#include "internal.h"
#include "mx.h"

namespace qlk {
namespace {

constexpr int THREADS = 256;
constexpr int TABLE = 1024;  // (cos, sin) pairs in LDS

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

template <bool BF16, bool INTER, bool VEC>
__global__ __launch_bounds__(THREADS) void rotary_kernel(const RotaryArgs a)
{
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int V = VEC ? E::V : 1;
    typedef T vec __attribute__((ext_vector_type(V)));
    __shared__ mx_f32x2 table[TABLE];
    const int half = a.rot / 2;
    const int64_t row0 = (int64_t)blockIdx.x * a.rows_per_wg;
    const int rows = (int)min((int64_t)a.rows_per_wg, a.rows - row0);
    // items of a head: pairs of vectors (half layout; one by one, pairs of
    // channels in either layout) or vectors, then the kept vectors
    const int turns = INTER && VEC ? a.rot / V : half / V;
    const int per_head = turns + (a.copy ? (a.dh - a.rot) / V : 0);
    const int per_row = per_head * a.heads;
    const bool one_pass = half <= TABLE;  // (else the table holds a run of pairs at a time)
    for (int p0 = 0; p0 < half; p0 += TABLE) {
        const int np = one_pass ? half : min(TABLE, half - p0);
        if (p0)
            __syncthreads();
        for (int i = threadIdx.x; i < rows * np; i += THREADS) {
            const int r = i / np, j = p0 + i - r * np;
            const int64_t row = row0 + r;
            const int64_t pos = a.positions ? a.positions[row] : a.start + row % a.period;
            const double t = (double)pos * (a.freqs[j] * 0.15915494309189533577);  // turns
            const float f = (float)(t - __builtin_rint(t));
            float s, c;
            sincospif(2.0f * f, &s, &c);
            table[i] = mx_f32x2{c * a.mscale, (a.adjoint ? -s : s) * a.mscale};
        }
        __syncthreads();
        for (int i = threadIdx.x; i < rows * per_row; i += THREADS) {
            const int r = i / per_row, q = i - r * per_row;
            const int h = q / per_head, u = q - h * per_head;
            const T *const x = static_cast<const T *>(a.x) + (row0 + r) * a.ldx + (int64_t)h * a.dh;
            T *const o = static_cast<T *>(a.o) + (row0 + r) * a.ldo + (int64_t)h * a.dh;
            if (u >= turns) {
                if (p0 == 0) {
                    const int ch = a.rot + (u - turns) * V;
                    *reinterpret_cast<vec *>(o + ch) = *reinterpret_cast<const vec *>(x + ch);
                }
                continue;
            }
            const mx_f32x2 *const cs = table + r * np - p0;
            if constexpr (INTER && VEC) {
                const int j0 = u * V / 2;
                if (j0 < p0 || j0 >= p0 + np)
                    continue;
                const vec v = *reinterpret_cast<const vec *>(x + u * V);
                vec w;
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const mx_f32x2 t = cs[j0 + e / 2];
                    const float p = E::get(v[e]), s = E::get(v[e + 1]);
                    w[e] = E::put(p * t[0] - s * t[1]);
                    w[e + 1] = E::put(s * t[0] + p * t[1]);
                }
                *reinterpret_cast<vec *>(o + u * V) = w;
            } else {
                const int j0 = u * V;
                if (j0 < p0 || j0 >= p0 + np)
                    continue;
                const int ca = INTER ? 2 * j0 : j0, cb = INTER ? 2 * j0 + 1 : j0 + half;
                const vec v = *reinterpret_cast<const vec *>(x + ca);
                const vec y = *reinterpret_cast<const vec *>(x + cb);
                vec w, z;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const mx_f32x2 t = cs[j0 + e];
                    const float p = E::get(v[e]), s = E::get(y[e]);
                    w[e] = E::put(p * t[0] - s * t[1]);
                    z[e] = E::put(s * t[0] + p * t[1]);
                }
                *reinterpret_cast<vec *>(o + ca) = w;
                *reinterpret_cast<vec *>(o + cb) = z;
            }
        }
    }
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, hipStream_t stream)
{
    const int V = a.bf16 ? 8 : 4;
    const int half = a.rot / 2;
    const uintptr_t size = a.bf16 ? 2 : 4;
    const bool vec = (a.interleaved ? a.rot : half) % V == 0 && a.dh % V == 0 &&
                     a.rot % V == 0 && ((uintptr_t)a.x & 15) == 0 && ((uintptr_t)a.o & 15) == 0 &&
                     a.ldx * size % 16 == 0 && a.ldo * size % 16 == 0;
    // rows of a workgroup: up to four items a thread, and their angles in the table
    const int v = vec ? V : 1;
    const int64_t items = (int64_t)a.heads * ((a.interleaved && vec ? a.rot / v : half / v) +
                                              (a.copy ? (a.dh - a.rot) / v : 0));
    int64_t rpw = std::max<int64_t>(1, 4 * THREADS / std::max<int64_t>(1, items));
    rpw = std::min<int64_t>(rpw, std::max(1, TABLE / half));
    // (a GPU's worth of workgroups before any takes a second row)
    rpw = std::min<int64_t>(rpw, std::max<int64_t>(1, a.rows / 1024));
    a.rows_per_wg = (int)rpw;
    const dim3 grid((unsigned)((a.rows + rpw - 1) / rpw)), block(THREADS);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    auto layout = [&](auto bf) {
        constexpr bool B = decltype(bf)::value;
        if (a.interleaved)
            vec ? go(rotary_kernel<B, true, true>) : go(rotary_kernel<B, true, false>);
        else
            vec ? go(rotary_kernel<B, false, true>) : go(rotary_kernel<B, false, false>);
    };
    if (a.bf16)
        layout(std::true_type{});
    else
        layout(std::false_type{});
    return hipGetLastError();
}

}  // namespace qlk
