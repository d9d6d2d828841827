// Matrix product of e4m3 operands with a scale for each block of 128 along the depth:
//
//   y[i, j] = sum_b xs[i, b] ws[j / 128, b] sum_{k in b} x[i, k] w[j, k]
//
// Codes become fp16 values in registers (exact) and meet in fp16 matrix instructions, whose sums are fp32; a block's sum is scaled into
// the output's.  The e4m3 matrix instruction would be twice as fast, but it cuts the products of eight neighbours along the
// depth 13 bits below the largest of them: sums of 128 normal values are off by 1.6e-5 of themselves, and by 5e-5 where the
// values' sizes spread, against 1e-8 here.
#include <algorithm>

#include "quamba_internal.h"

namespace quamba {
namespace {

typedef int int8v __attribute__((ext_vector_type(8)));      // 32 e4m3 codes
typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;

// 16 codes at p, of which the first `left` belong to the row; the others count as zeros.
__device__ __forceinline__ int4v load16(const uint8_t *p, int left)
{
    int4v w;
    if (left >= 16) {
        __builtin_memcpy(&w, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * i + j < left) v |= (uint32_t)p[4 * i + j] << 8 * j;
            w[i] = (int)v;
        }
    }
    return w;
}

// 32 codes of a row (a lane's part of a block) as fp16 values.
struct Part {
    half8 h[4];
    __device__ __forceinline__ Part() {}
    __device__ __forceinline__ Part(const int4v &lo, const int4v &hi)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int4v v;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int c = i < 2 ? lo[2 * i + j] : hi[2 * i + j - 4];
                v[2 * j] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, false));
                v[2 * j + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, true));
            }
            h[i] = __builtin_bit_cast(half8, v);
        }
    }
};

// Lane l's part is row l % 16, codes 32 (l / 16) on; of the 16 x 16 sums it gets a's rows 4 (l / 16) + e against b's row l % 16.
__device__ __forceinline__ float4v multiply(const Part &a, const Part &b)
{
    float4v p{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h[i], b.h[i], p, 0, 0, 0);
    return p;
}

__device__ __forceinline__ void store(void *y, int type, int64_t at, float v)
{
    if (type == QUAMBA_F32)
        static_cast<float *>(y)[at] = v;
    else if (type == QUAMBA_F16)
        static_cast<uint16_t *>(y)[at] = f32_to_f16_bits(v);
    else
        static_cast<__bf16 *>(y)[at] = (__bf16)v;
}

// A wave for 16 x 16 outputs, operands from memory to registers.
__global__ __launch_bounds__(64) void fp8_matmul_any_kernel(MatmulArgs a)
{
    const int lane = threadIdx.x, r = lane & 15, part = lane >> 4;
    const int64_t i = (int64_t)blockIdx.y * 16 + r, j = (int64_t)blockIdx.x * 16 + r;  // this lane's rows of x and of w
    const uint8_t *xp = a.x + min(i, (int64_t)a.m - 1) * a.x_stride, *wp = a.w + min(j, (int64_t)a.n - 1) * a.w_stride;
    const float *xs = a.x_scales + min(i, (int64_t)a.m - 1) * a.blocks;
    const float *ws = a.w_scales + (int64_t)(blockIdx.x * 16 / kBlock) * a.blocks;
    float4v sum{0, 0, 0, 0};
    for (int b = 0; b < a.blocks; ++b) {
        const int k = b * kBlock + part * 32;
        const Part x(load16(xp + k, a.k - k), load16(xp + k + 16, a.k - k - 16));
        const Part w(load16(wp + k, a.k - k), load16(wp + k + 16, a.k - k - 16));
        const float4v p = multiply(w, x);
        const float s = xs[b] * ws[b];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(p[e], s, sum[e]);
    }
    const int64_t jo = (int64_t)blockIdx.x * 16 + part * 4;
    if (i < a.m)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (jo + e < a.n) store(a.y, a.y_type, i * a.y_stride + jo + e, sum[e]);
}

}  // namespace

size_t fp8_matmul_workspace_bytes(int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_fp8_matmul(const MatmulArgs &a, void *, hipStream_t stream)
{
    constexpr int kRows = kMaxGridY * 16;  // of a launch
    for (int64_t first = 0; first < a.m; first += kRows) {
        MatmulArgs p = a;
        p.m = (int32_t)std::min<int64_t>(kRows, a.m - first);
        p.x = a.x + first * a.x_stride;
        p.x_scales = a.x_scales + first * a.blocks;
        p.y = static_cast<char *>(a.y) + first * a.y_stride * (a.y_type == QUAMBA_F32 ? 4 : 2);
        fp8_matmul_any_kernel<<<dim3((a.n + 15) / 16, (p.m + 15) / 16), 64, 0, stream>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace quamba
