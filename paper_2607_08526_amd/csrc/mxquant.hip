// MXFP4 quantization of weights and activations, and the compressed formats
// read back.
//
//   e = clamp(floor(log2 max|x|) - 2, -127, 127)   (-127 for a block of zeros)
//   scale byte = e + 127,  code = nearest magnitude to |x| 2^-e, sign bit of x
//
// over blocks of 32 along a row: the largest magnitude of a block lands in
// [4, 8), ties go to the even code and what is beyond 6 becomes 6 (the OCP
// microscaling rule).  e is the fp32 exponent field of the maximum, x 2^-e is
// exact in fp32 wherever its code is not 0, and one instruction rounds two
// values to codes (v_cvt_scalef32_pk_fp4_f32).
//
// Bound: HBM (2 or 4 bytes read and 17 / 32 written per value; reading back
// the other way).  Four lanes per block with 8 values each, as in the int8 / q4
// quantizer: 16- or 32-byte loads, 4-byte code stores, two butterfly steps for
// the block's maximum.  8192 x 2048 fp32 (76 MB) 14.2 us, 5.4 TB/s; read back as fp32
// 15.9 us, 4.8 TB/s (a large copy: 5.1).
#include <algorithm>

#include "internal.h"
#include "mx.h"

namespace qlk {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int64_t MAX_GRID = 1 << 20;  // workgroups of a launch; more work loops

// STATUS: a block with a NaN or Inf reports QL_ERR_RANGE (weights); otherwise
// it gets the NaN scale 255 and zero codes, so that whatever is computed from
// it is NaN (activations).
template <bool BF16, bool STATUS>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const void *__restrict__ X,
                                                          int64_t n_blocks,
                                                          uint8_t *__restrict__ codes,
                                                          uint8_t *__restrict__ scales,
                                                          int *__restrict__ status)
{
    // (a GPU-filling grid; the base is uniform, so a block's lanes stay together)
    for (int64_t base = (int64_t)blockIdx.x * 64; base < n_blocks; base += (int64_t)gridDim.x * 64) {
        const int64_t blk = base + (threadIdx.x >> 2);
        const int part = (int)(threadIdx.x & 3);
        const bool valid = blk < n_blocks;
        uint32_t v[8];
        if (!valid) {
    #pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = 0;
        } else if constexpr (BF16) {
            const uint4 a = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(X) +
                                                             blk * 32 + part * 8);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
    #pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] = w[j] << 16;
                v[2 * j + 1] = w[j] & 0xFFFF0000u;
            }
        } else {
            const uint4 *p =
                reinterpret_cast<const uint4 *>(static_cast<const float *>(X) + blk * 32 + part * 8);
            const uint4 a = p[0], b = p[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
        uint32_t amax = 0;  // |x| bit patterns compare like the values; NaN/Inf >= 0x7F800000
    #pragma unroll
        for (int j = 0; j < 8; ++j)
            amax = max(amax, v[j] & 0x7FFFFFFFu);
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
        if (!valid)
            continue;
        const bool bad = amax >= 0x7F800000u;
        if (STATUS && bad) {
            *status = QL_ERR_RANGE;
            continue;
        }
        const uint32_t field = amax >> 23;
        const uint32_t s = field > 2 ? field - 2 : 0;  // at most 252 for a finite maximum
        const float inv = __uint_as_float((254u - (bad ? 0u : s)) << 23);  // 2^(127 - s), normal
        uint32_t word = 0;
        if (!bad) {
            auto val = [&](int j) { return __uint_as_float(v[j]) * inv; };
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, val(0), val(1), 1.0f, 0);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, val(2), val(3), 1.0f, 1);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, val(4), val(5), 1.0f, 2);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, val(6), val(7), 1.0f, 3);
        }
        *reinterpret_cast<uint32_t *>(codes + blk * 16 + part * 4) = word;
        if (part == 0)
            scales[blk] = (uint8_t)(bad ? 255u : s);
    }
}

// 8 values of one block per thread: code * scale, exact in fp32 (a bf16 output
// of q4 / int8 is rounded once; with lo, W and lo receive the two bf16 of a product)
struct DequantArgs {
    DequantJob j[2];
};
template <int FMT, bool BF16>
__global__ __launch_bounds__(256) void dequantize_kernel(const DequantArgs a, int64_t groups)
{
    const uint8_t *const codes = static_cast<const uint8_t *>(a.j[blockIdx.y].codes);
    const void *const scales = a.j[blockIdx.y].scales;
    void *const W = a.j[blockIdx.y].W, *const lo = a.j[blockIdx.y].lo;
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups;
         g += (int64_t)gridDim.x * 256) {
        float v[8];
        if constexpr (FMT == QL_FMT_MXFP4) {
            const uint32_t w = reinterpret_cast<const uint32_t *>(codes)[g];
            const float s = mx_scale(static_cast<const uint8_t *>(scales)[g >> 2]);
            mx_f32x2 p[4];
            p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
            p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
            p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
            p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    #pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = p[e >> 1][e & 1] * s;
        } else {
            float s = (float)static_cast<const _Float16 *>(scales)[g >> 2];
            if (lo)
                s = plane_scale(s);
            if constexpr (FMT == QL_FMT_Q4) {
                q4_f32x8(reinterpret_cast<const uint32_t *>(codes)[g], s, v);
            } else {
                const uint2 w = reinterpret_cast<const uint2 *>(codes)[g];
                int8_f32x8(w.x, w.y, s, v);
            }
        }
        if constexpr (BF16) {
            mx_u32x4 h, l;
            if (FMT != QL_FMT_MXFP4 && lo) {
                split2(v, h, l);
                static_cast<mx_u32x4 *>(lo)[g] = l;
            } else {
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    h[w] = mx_pack_bf16(v[2 * w], v[2 * w + 1]);
            }
            static_cast<mx_u32x4 *>(W)[g] = h;
        } else {
            f32x4_t *const o = static_cast<f32x4_t *>(W) + 2 * g;
            o[0] = f32x4_t{v[0], v[1], v[2], v[3]};
            o[1] = f32x4_t{v[4], v[5], v[6], v[7]};
        }
    }
}

}  // namespace

hipError_t launch_mx_quantize(const void *X, bool bf16, int64_t rows, int64_t K, uint8_t *codes,
                              uint8_t *scales, int *status, hipStream_t stream)
{
    const int64_t blocks = rows * (K / 32);
    const dim3 grid((unsigned)std::min<int64_t>((blocks + 63) / 64, MAX_GRID)), block(256);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, stream, X, blocks, codes, scales, status);
    };
    if (status)
        go(mx_quantize_kernel<false, true>);
    else if (bf16)
        go(mx_quantize_kernel<true, false>);
    else
        go(mx_quantize_kernel<false, false>);
    return hipGetLastError();
}

hipError_t launch_dequantize(int fmt, const DequantJob *jobs, int n, int64_t N, int64_t K,
                             bool bf16, hipStream_t stream)
{
    const int64_t groups = N * (K / 8);
    DequantArgs a{};
    for (int i = 0; i < n; ++i)
        a.j[i] = jobs[i];
    const dim3 grid((unsigned)std::min<int64_t>((groups + 255) / 256, MAX_GRID), (unsigned)n);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, groups);
    };
    if (fmt == QL_FMT_MXFP4)
        bf16 ? go(dequantize_kernel<QL_FMT_MXFP4, true>) : go(dequantize_kernel<QL_FMT_MXFP4, false>);
    else if (fmt == QL_FMT_Q4)
        bf16 ? go(dequantize_kernel<QL_FMT_Q4, true>) : go(dequantize_kernel<QL_FMT_Q4, false>);
    else
        bf16 ? go(dequantize_kernel<QL_FMT_INT8, true>) : go(dequantize_kernel<QL_FMT_INT8, false>);
    return hipGetLastError();
}

}  // namespace qlk
