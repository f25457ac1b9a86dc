// Root-mean-square normalisation with the residual's addition, and its backward pass.
//
//   v = x + r (one fp32 rounding),  rstd = 1 / sqrt(mean v^2 + eps),  y = v rstd w
//   dv = dres + rstd (g - u mean(g u)),  dw = sum over rows of dy u,
//        with g = dy w and u = v rstd
//
// The squares are summed and the scalars of a row formed in fp64: a square of an
// fp32 value is exact there and neither overflows nor underflows, so rows of any
// size are right.  y is the product in fp64 rounded once to fp32 and then, for bf16
// outputs, to bf16; the int8 outputs are act_quant's of that fp32 y (codes.h), so
// they do not depend on an order of roundings.  fp64 costs nothing here: seven such
// instructions per value against 10 to 14 bytes of HBM.
//
// Bound: HBM; at few rows the latency of one load and of the row's reduction.  A
// row's values stay in registers between the sum and the output (W wavefronts of
// R groups of 8 columns per lane), so each is read once.  Measured, us:
//   forward, fp32 x, r and h, bf16 y, every call on other rows than the last ones: 8192 rows
//   of 2048 (235 MB) 45, 5.2 TB/s (a copy of 4 GiB: 4.4 to 5.1); 2048 rows 15.2, 3.9 TB/s, and
//   12.2 where three sets of them in turn are partly in the last-level cache; 1290 rows of
//   1536, bf16 x, int8 y (22 MB): 9.6, a row's two reductions and its latency; one row:
//   2.5, a launch
//   backward, 8192 rows of 2048, bf16 dy, fp32 h, dres and dx (235 MB): 41 to 44 and 4.7 for
//   the sum of dw, 5.1 TB/s; 107 rows of 1024: 4.3 and 3.4, two launches
#include "codes.h"
#include "internal.h"

namespace qlk {
namespace {

// groups of 8 values at any element address (the hardware takes unaligned vectors)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef f32x4 f32x4_at4 __attribute__((aligned(4)));

__device__ inline uint32_t bf16_bits(float f)
{
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}

// Values 8 g .. 8 g + 7 of a row as they are in memory (n of them; those past the row's end
// are 0), and as numbers: apart, so that a load may be in flight while others are used.
template <bool BF16>
struct Eight {
    u32x4 w[BF16 ? 1 : 2];

    __device__ inline void load(const void *p, int64_t e, int n)
    {
        if constexpr (BF16) {
            const uint16_t *q = static_cast<const uint16_t *>(p) + e;
            if (n >= 8) {
                w[0] = *reinterpret_cast<const u32x4_at2 *>(q);
                return;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[0][j] = (2 * j < n ? q[2 * j] : 0u) | (2 * j + 1 < n ? q[2 * j + 1] : 0u) << 16;
        } else {
            const uint32_t *q = static_cast<const uint32_t *>(p) + e;
            if (n >= 8) {
                w[0] = *reinterpret_cast<const u32x4_at4 *>(q);
                w[1] = *reinterpret_cast<const u32x4_at4 *>(q + 4);
                return;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                w[j / 4][j % 4] = j < n ? q[j] : 0u;
        }
    }
    __device__ inline float operator[](int j) const
    {
        if constexpr (BF16)
            return __uint_as_float(j % 2 ? w[0][j / 2] & 0xFFFF0000u : w[0][j / 2] << 16);
        else
            return __uint_as_float(w[j / 4][j % 4]);
    }
};

__device__ inline void store8(void *p, bool bf16, int64_t e, int n, const float (&v)[8])
{
    if (bf16) {
        uint16_t *q = static_cast<uint16_t *>(p) + e;
        if (n >= 8) {
            u32x4 a;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                a[j] = bf16_bits(v[2 * j]) | bf16_bits(v[2 * j + 1]) << 16;
            *reinterpret_cast<u32x4_at2 *>(q) = a;
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n)
                q[j] = (uint16_t)bf16_bits(v[j]);
    } else {
        float *q = static_cast<float *>(p) + e;
        if (n >= 8) {
            *reinterpret_cast<f32x4_at4 *>(q) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_at4 *>(q + 4) = f32x4{v[4], v[5], v[6], v[7]};
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n)
                q[j] = v[j];
    }
}

__device__ inline double wave_sum(double s)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
        s += __shfl_xor(s, o);
    return s;
}

// 1 / sqrt(x) for x >= 0: the hardware's estimate (2^-26 or better) and two Newton steps;
// infinities and NaN as the estimate has them.  0 for 0, a row of zeros and eps = 0: it has no
// direction u, and 0 as such (not 0 * infinity) keeps it out of the others' dw.
__device__ inline double inverse_sqrt(double x)
{
    if (x == 0.0)
        return 0.0;
    double r = __builtin_amdgcn_rsq(x);
    if (x > 0.0 && x < __builtin_inf()) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            r = __builtin_fma(0.5 * r, __builtin_fma(-x * r, r, 1.0), r);
    }
    return r;
}

// rows per workgroup and threads of it, for W wavefronts a row
template <int W>
constexpr int ROWS = W >= 4 ? 1 : 4 / W;
template <int W>
constexpr int THREADS = 64 * W * ROWS<W>;

template <bool XB, bool HB, int W, int R>
__global__ __launch_bounds__(THREADS<W>) void norm_kernel(const NormArgs a)
{
    constexpr int T = 64 * W;
    __shared__ double ssum[ROWS<W>][W];
    __shared__ uint32_t smax[ROWS<W>][W];
    const int t = (int)threadIdx.x % T, wave = t >> 6, slot = (int)threadIdx.x / T;
    const int64_t m = (int64_t)blockIdx.x * ROWS<W> + slot;
    const bool live = m < a.M;
    if (W == 1 && !live)
        return;  // (a wavefront of its own: no barrier below)
    const int N = live ? a.N : 0;  // (a row past the last: nothing of it)
    float v[R][8];
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int c = 8 * (t + i * T), n = N - c;
        Eight<XB> x;
        x.load(a.x, m * a.ldx + c, n);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[i][j] = x[j];
        if (a.res) {
            Eight<HB> r;
            r.load(a.res, m * a.ldr + c, n);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[i][j] += r[j];
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int c = 8 * (t + i * T);
        if (a.h)
            store8(a.h, HB, m * a.ldh + c, N - c, v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            s = __builtin_fma((double)v[i][j], (double)v[i][j], s);
    }
    s = wave_sum(s);
    if constexpr (W > 1) {
        if ((t & 63) == 0)
            ssum[slot][wave] = s;
        __syncthreads();
        s = 0.0;
#pragma unroll
        for (int w = 0; w < W; ++w)
            s += ssum[slot][w];
    }
    const double rstd = inverse_sqrt(__builtin_fma(s, a.inv_n, a.eps));
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int c = 8 * (t + i * T), n = N - c;
        Eight<false> w;
        if (a.weight)
            w.load(a.weight, c, n);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double u = (double)v[i][j] * rstd;
            v[i][j] = (float)(a.weight ? u * (double)w[j] : u);
        }
        if (a.y)
            store8(a.y, a.ybf16, m * a.ldy + c, n, v[i]);
    }
    if (!a.qx)
        return;

    // act_quant's scale and codes of the row (|y| bit patterns compare like the
    // values; columns past the row's end are 0, or NaN where rstd is: out)
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = __float_as_uint(v[i][j]) & 0x7FFFFFFFu;
            if (8 * (t + i * T) < N)
                amax = b > amax ? b : amax;
        }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t b = (uint32_t)__shfl_xor((int)amax, o);
        amax = b > amax ? b : amax;
    }
    if constexpr (W > 1) {
        if ((t & 63) == 0)
            smax[slot][wave] = amax;
        __syncthreads();
        amax = smax[slot][0];
#pragma unroll
        for (int w = 1; w < W; ++w)
            amax = smax[slot][w] > amax ? smax[slot][w] : amax;
    }
    uint32_t sbits = 0x7C00;
    if (amax < 0x7F800000u)
        sbits = scale_bits<127>(__uint_as_float(amax));
    const bool zero = sbits == 0x7C00 || sbits == 0;
    if (t == 0 && live)
        a.sx[m] = (uint16_t)(sbits == 0x7C00 ? 0x7E00 : sbits);
    const float sc = zero ? 1.0f : f16_value(sbits);
    const float inv = inverse(sc), half_s = 0.5f * sc;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int c = 8 * (t + i * T);
        if (c >= N)  // N % 32 == 0
            continue;
        uint32_t q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            q[j] = zero ? 0u : (uint32_t)nearest_code(v[i][j], sc, inv, half_s, 127) & 0xFFu;
        *reinterpret_cast<uint2 *>(a.qx + m * a.N + c) =
            make_uint2(q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24,
                       q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24);
    }
}

// Each workgroup takes every gridDim.x-th row (ROWS of them at a time) and adds up
// its rows' dy u by columns; those sums go to part[workgroup][N], added in that order
// by norm_dw_kernel, so that dw has one order of additions.
template <bool YB, bool HB, bool DB, int W, int R>
__global__ __launch_bounds__(THREADS<W>) void norm_grad_kernel(const NormGradArgs a)
{
    constexpr int T = 64 * W;
    constexpr bool HOLD = R <= 2;  // registers for a row ahead and the weights
    __shared__ double sums[2][ROWS<W>][W][2];
    __shared__ float shared_dw[W < 4 ? THREADS<W> : 1][8];
    const int t = (int)threadIdx.x % T, wave = t >> 6, slot = (int)threadIdx.x / T;
    const int N = a.N;
    float dw[R][8];
    Eight<false> w[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            dw[i][j] = 0.0f;
        if (HOLD && a.weight)
            w[i].load(a.weight, 8 * (t + i * T), N - 8 * (t + i * T));
    }
    // the next row is loaded before this one's sums are waited for
    Eight<HB> hs[2][R];
    Eight<YB> ys[2][R];
    Eight<DB> rs[2][R];
    // (a row past the last, beside one that is there: nothing of it)
    auto columns = [&](int64_t m) { return ROWS<W> > 1 && m >= a.M ? 0 : N; };
    auto load = [&](int64_t m, int k) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int c = 8 * (t + i * T), n = columns(m) - c;
            hs[k][i].load(a.h, m * a.ldh + c, n);
            ys[k][i].load(a.dy, m * a.lddy + c, n);
            if (HOLD && a.dres)
                rs[k][i].load(a.dres, m * a.ldres + c, n);
        }
    };
    const int64_t step = (int64_t)gridDim.x * ROWS<W>;
    auto row = [&](int64_t m, int k) {
        if (HOLD && m - slot + step < a.M)
            load(m + step, k ^ 1);
        if (!HOLD)
            load(m, k);
        const Eight<HB>(&v)[R] = hs[k];
        const Eight<YB>(&dy)[R] = ys[k];
        const Eight<DB>(&d)[R] = rs[k];
        double s = 0.0, p = 0.0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (!HOLD && a.weight)
                w[i].load(a.weight, 8 * (t + i * T), N - 8 * (t + i * T));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double x = v[i][j], g = a.weight ? (double)dy[i][j] * (double)w[i][j]
                                                       : (double)dy[i][j];
                s = __builtin_fma(x, x, s);
                p = __builtin_fma(x, g, p);
            }
        }
        s = wave_sum(s);
        p = wave_sum(p);
        if constexpr (W > 1) {
            // (two turns' places: a wavefront that is a row ahead writes the other)
            if ((t & 63) == 0) {
                sums[k][slot][wave][0] = s;
                sums[k][slot][wave][1] = p;
            }
            __syncthreads();
            s = p = 0.0;
#pragma unroll
            for (int q = 0; q < W; ++q) {
                s += sums[k][slot][q][0];
                p += sums[k][slot][q][1];
            }
        }
        const double rstd = inverse_sqrt(__builtin_fma(s, a.inv_n, a.eps));
        const double mean = p * rstd * a.inv_n;  // of g u
        // rstd = r 2^e, so that u = v rstd is of size 1 where rstd itself leaves fp32 (rows of
        // subnormals, of the largest numbers): scaling by 2^e is exact, the other roundings
        // are those of products with an fp32 rstd
        const int e = __builtin_amdgcn_frexp_exp(rstd);
        const double r64 = __builtin_amdgcn_frexp_mant(rstd);
        const float r32 = (float)r64, k32 = (float)(mean * r64);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int c = 8 * (t + i * T);
            float out[8];
            if (!HOLD && a.dres)
                rs[k][i].load(a.dres, m * a.ldres + c, N - c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float u = __builtin_ldexpf(v[i][j], e) * r32;
                const float g = a.weight ? dy[i][j] * w[i][j] : dy[i][j];
                const float o = __builtin_ldexpf(__builtin_fmaf(g, r32, -u * k32), e);
                out[j] = a.dres ? d[i][j] + o : o;
                dw[i][j] = __builtin_fmaf(dy[i][j], u, dw[i][j]);
            }
            store8(a.dx, DB, m * a.lddx + c, columns(m) - c, out);
        }
    };
    // (by the workgroup's first row: its wavefronts meet at the sums of several)
    int64_t m0 = (int64_t)blockIdx.x * ROWS<W>;
    if (HOLD && m0 < a.M)
        load(m0 + slot, 0);
    for (; m0 < a.M; m0 += 2 * step) {
        row(m0 + slot, 0);
        if (m0 + step < a.M)
            row(m0 + step + slot, 1);
    }
    if (!a.part)
        return;
    if constexpr (W < 4) {  // the rows that ran beside each other
        static_assert(R == 1, "");
#pragma unroll
        for (int j = 0; j < 8; ++j)
            shared_dw[threadIdx.x][j] = dw[0][j];
        __syncthreads();
        if (threadIdx.x >= T)
            return;
        for (int k = 1; k < ROWS<W>; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                dw[0][j] += shared_dw[k * T + t][j];
    }
    float *const part = a.part + (int64_t)blockIdx.x * N;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int c = 8 * (t + i * T);
        store8(part, false, c, N - c, dw[i]);
    }
}

// dw[c] = the sum of part[0 .. parts)[c], in fp64 and one order (so that results repeat): 64
// columns a workgroup, every 16th part a wavefront.  (fp64 within the parts too would take
// the registers of a row ahead: 8192 rows of 2048 46.5 us for 41.)  768 parts of 2048
// columns: 4.7 us, most of it the launch and the latency of 48 loads, eight in flight.
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float *part, int parts, int N,
                                                       float *dw)
{
    __shared__ double sums[16][64];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int c = (int)blockIdx.x * 64 + lane;
    double s = 0.0;
    if (c < N) {
#pragma unroll 8
        for (int p = wave; p < parts; p += 16)
            s += part[(int64_t)p * N + c];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || c >= N)
        return;
#pragma unroll
    for (int w = 1; w < 16; ++w)
        s += sums[w][lane];
    dw[c] = (float)s;
}

// Wavefronts and groups of 8 columns a lane by the columns (us from HBM, forward of fp32 rows
// with bf16 y / backward of bf16 dy with dw):
//   2048 rows of 4096: 4 and 2 28.2 / 33.5, 8 and 1 26.3 / 34.9
//   2048 rows of 8192: 8 and 2 48.3 / 60.5, 16 and 1 47.7 / 92.5, 4 and 4 51.4 / 70.7
//   1024 rows of 16384: 16 and 2 52.3 / 202, 8 and 4 53.2 / 85.8
// (Backward, 16 wavefronts leave 128 registers a lane, and values are spilled.)  The backward
// pass of more than 8192 columns holds no row ahead and loads weights and dres in every
// row: 2.7 TB/s; up to 8192 columns 3.5 to 4.7.
template <bool XB, bool HB>
void forward(const NormArgs &a, hipStream_t s)
{
#define QL_GO(W, R)                                                                          \
    hipLaunchKernelGGL((norm_kernel<XB, HB, W, R>),                                          \
                       dim3((unsigned)((a.M + ROWS<W> - 1) / ROWS<W>)), dim3(THREADS<W>), 0, s, a)
    if (a.N <= 512)
        QL_GO(1, 1);
    else if (a.N <= 1024)
        QL_GO(2, 1);
    else if (a.N <= 2048)
        QL_GO(4, 1);
    else if (a.N <= 4096)
        QL_GO(4, 2);
    else if (a.N <= 8192)
        QL_GO(8, 2);
    else
        QL_GO(16, 2);
#undef QL_GO
}

template <bool YB, bool HB, bool DB>
void backward(const NormGradArgs &a, int parts, hipStream_t s)
{
#define QL_GO(W, R)                                                                         \
    hipLaunchKernelGGL((norm_grad_kernel<YB, HB, DB, W, R>), dim3((unsigned)parts),         \
                       dim3(THREADS<W>), 0, s, a)
    if (a.N <= 512)
        QL_GO(1, 1);
    else if (a.N <= 1024)
        QL_GO(2, 1);
    else if (a.N <= 2048)
        QL_GO(4, 1);
    else if (a.N <= 4096)
        QL_GO(4, 2);
    else if (a.N <= 8192)
        QL_GO(8, 2);
    else
        QL_GO(8, 4);
#undef QL_GO
}

}  // namespace

hipError_t launch_norm(const NormArgs &a, hipStream_t stream)
{
    if (a.xbf16)
        a.hbf16 ? forward<true, true>(a, stream) : forward<true, false>(a, stream);
    else
        a.hbf16 ? forward<false, true>(a, stream) : forward<false, false>(a, stream);
    return hipGetLastError();
}

// Workgroups of the backward pass, and partial sums of dw: up to three per CU (two and four
// of 8192 x 2048 in fp32 take 42.4 and 45.2 us for 41.1).
int norm_grad_parts(int64_t M, int N, int cus)
{
    const int64_t rows = N <= 512 ? 4 : N <= 1024 ? 2 : 1, groups = (M + rows - 1) / rows;
    const int64_t most = 3 * (int64_t)cus;
    return (int)(groups < most ? groups : most);
}

hipError_t launch_norm_grad(const NormGradArgs &a, int parts, hipStream_t stream)
{
    const int form = (a.ybf16 ? 4 : 0) | (a.hbf16 ? 2 : 0) | (a.dbf16 ? 1 : 0);
    switch (parts ? form : -1) {
    case -1: break;  // no rows: dw is 0
    case 0: backward<false, false, false>(a, parts, stream); break;
    case 1: backward<false, false, true>(a, parts, stream); break;
    case 2: backward<false, true, false>(a, parts, stream); break;
    case 3: backward<false, true, true>(a, parts, stream); break;
    case 4: backward<true, false, false>(a, parts, stream); break;
    case 5: backward<true, false, true>(a, parts, stream); break;
    case 6: backward<true, true, false>(a, parts, stream); break;
    default: backward<true, true, true>(a, parts, stream); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.dw)
        return e;
    hipLaunchKernelGGL(norm_dw_kernel, dim3((unsigned)((a.N + 63) / 64)), dim3(1024), 0, stream,
                       a.part, parts, a.N, a.dw);
    return hipGetLastError();
}

}  // namespace qlk
