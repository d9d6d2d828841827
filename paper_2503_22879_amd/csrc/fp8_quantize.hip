// Quantizer of the 8-bit floating-point products: e4m3 codes and one fp32 scale for each block of 1 x 128 or 128 x 128 values.
//
//   scale = max|x| / 448,  code = e4m3(x (1 / scale))
//
// Every value is read once and stays in registers between the maximum and the codes.  Bound: HBM, small matrices by their launch.
// 16384 x 8192 fp16 in blocks of 1 x 128: 68.6 us, 5.93 TB/s of 407 MB (a copy of that size runs at 5.1 - 5.5); 1 x 4096: 3.3 us.
#include <algorithm>

#include "quamba_internal.h"

namespace quamba {
namespace {

constexpr int kBlock = 128;        // values under one scale along a row
constexpr int kLanes = 16;         // lanes that hold a block's part of a row, 8 values each
constexpr int kValues = kBlock / kLanes;
constexpr int kSquareThreads = 512;  // to a block of 128 x 128

template <int TYPE>
struct Values {  // 8 values of a row as they lie in memory
    static constexpr int kBytes = TYPE == QUAMBA_F32 ? 4 : 2;
    uint32_t w[kValues * kBytes / 4];

    // from `left` values on (fewer than 8 at a row's end, none behind it); the missing ones are zeros
    __device__ __forceinline__ void load(const char *p, int left)
    {
        if (left >= kValues) {
            __builtin_memcpy(w, p, sizeof(w));
        } else {
#pragma unroll
            for (int i = 0; i < (int)(sizeof(w) / 4); ++i) w[i] = 0;
#pragma unroll
            for (int i = 0; i < kValues; ++i)
                if (i < left) {
                    if (kBytes == 4) {
                        __builtin_memcpy(&w[i], p + 4 * i, 4);
                    } else {
                        uint16_t h;
                        __builtin_memcpy(&h, p + 2 * i, 2);
                        w[i / 2] |= (uint32_t)h << (i & 1) * 16;
                    }
                }
        }
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if (TYPE == QUAMBA_F32) return from_bits(w[i]);
        const uint32_t h = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
        return TYPE == QUAMBA_BF16 ? from_bits(h << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)h);
    }
    // Largest |x| as bits: ordered like the numbers, infinity above them and NaN above infinity.
    __device__ __forceinline__ uint32_t top() const
    {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < kValues; ++i) t = max(t, __builtin_bit_cast(uint32_t, (*this)[i]) & 0x7fffffffu);
        return t;
    }
    // e4m3 codes of x * inv to a row's `left` values at p
    __device__ __forceinline__ void store(uint8_t *p, int left, float inv, bool finite) const
    {
        uint32_t c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int v = __builtin_amdgcn_cvt_pk_fp8_f32((*this)[4 * i] * inv, (*this)[4 * i + 1] * inv, 0, false);
            v = __builtin_amdgcn_cvt_pk_fp8_f32((*this)[4 * i + 2] * inv, (*this)[4 * i + 3] * inv, v, true);
            c[i] = finite ? (uint32_t)v : 0x7f7f7f7fu;
        }
        if (left >= kValues) {
            __builtin_memcpy(p, c, sizeof(c));
        } else {
#pragma unroll
            for (int i = 0; i < kValues; ++i)
                if (i < left) p[i] = (uint8_t)(c[i / 4] >> (i & 3) * 8);
        }
    }
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v)
{
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true));
}

// Largest over a row of 16 lanes; every lane gets it.
__device__ __forceinline__ uint32_t row_max(uint32_t v)
{
    v = dpp_max<0xB1>(v);
    v = dpp_max<0x4E>(v);
    v = dpp_max<0x141>(v);
    return dpp_max<0x140>(v);
}

// The scale of a block and its reciprocal from the largest |x|'s bits.
struct Scale {
    float s, inv;
    bool finite;
    __device__ __forceinline__ explicit Scale(uint32_t top)
    {
        finite = top < 0x7f800000u;
        s = from_bits(top) / 448.0f;
        s = s >= from_bits(0x00800000u) ? s : 1.0f;
        inv = 1.0f / s;
        if (!finite) s = from_bits(0x7fc00000u);
    }
};

// Blocks of 1 x 128: 16 lanes to a block, blocks counted row by row.
template <int TYPE>
__global__ __launch_bounds__(256) void fp8_quantize_rows_kernel(QuantizeArgs a)
{
    const int g = blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;  // the block
    if (g >= a.blocks) return;
    const int row = quotient(g, a.by_row_blocks), kb = g - row * a.row_blocks;
    const int64_t col = (int64_t)kb * kBlock + threadIdx.x % kLanes * kValues;
    const int left = (int)min((int64_t)kValues, max((int64_t)0, a.cols - col));
    Values<TYPE> v;
    v.load(static_cast<const char *>(a.x) + (row * a.x_stride + col) * Values<TYPE>::kBytes, left);
    const Scale s(row_max(v.top()));
    v.store(a.q + row * a.q_stride + col, left, s.inv, s.finite);
    if (threadIdx.x % kLanes == 0) a.scales[g] = s.s;
}

// Blocks of 128 x 128: a workgroup each, 16 lanes to a row and 4 rows to 16 lanes, all of them loaded before the first is looked at.
// 3352 x 768 fp32: 4.25 us, and 5.25 us with 256 threads (162 blocks leave units idle, and the others have little to wait with);
// 18560 x 4096 fp32 67 us with both (5.7 TB/s), bf16 37 against 38 us; 1024 threads gain on the former (64) and lose on the latter (39).
template <int TYPE>
__global__ __launch_bounds__(kSquareThreads) void fp8_quantize_squares_kernel(QuantizeArgs a)
{
    constexpr int kWaves = kSquareThreads / 64;
    __shared__ uint32_t wave_top[kWaves];
    const int br = quotient((int)blockIdx.x, a.by_row_blocks), kb = blockIdx.x - br * a.row_blocks;
    const int64_t col = (int64_t)kb * kBlock + threadIdx.x % kLanes * kValues;
    const int64_t row0 = (int64_t)br * kBlock + threadIdx.x / kLanes;
    constexpr int kRows = kBlock * kLanes / kSquareThreads, kStep = kSquareThreads / kLanes;
    const int left = (int)min((int64_t)kValues, max((int64_t)0, a.cols - col));
    Values<TYPE> v[kRows];
    uint32_t top = 0;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int64_t row = row0 + r * kStep;
        v[r].load(static_cast<const char *>(a.x) + (row * a.x_stride + col) * Values<TYPE>::kBytes, row < a.rows ? left : 0);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) top = max(top, v[r].top());
    top = row_max(top);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
    if (threadIdx.x % 64 == 0) wave_top[threadIdx.x / 64] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = max(top, wave_top[w]);
    const Scale s(top);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int64_t row = row0 + r * kStep;
        v[r].store(a.q + row * a.q_stride + col, row < a.rows ? left : 0, s.inv, s.finite);
    }
    if (threadIdx.x == 0) a.scales[blockIdx.x] = s.s;
}

template <int TYPE>
void launch(const QuantizeArgs &a, bool squares, hipStream_t stream)
{
    if (squares)
        fp8_quantize_squares_kernel<TYPE><<<a.blocks, kSquareThreads, 0, stream>>>(a);
    else
        fp8_quantize_rows_kernel<TYPE><<<(a.blocks + 15) / 16, 256, 0, stream>>>(a);
}

}  // namespace

// Launches of whole rows of blocks, or of a part of one: at most 2^31 threads and 2^23 blocks, so that threads and indices fit 32 bits.
QuantizeCut fp8_quantize_cut(int64_t row_blocks, int32_t block_rows)
{
    const int64_t most = block_rows > 1 ? ((int64_t)1 << 31) / kSquareThreads : (int64_t)1 << 23;
    return {std::max<int64_t>(1, most / row_blocks), std::min(row_blocks, most)};
}

int64_t fp8_quantize_threads(int64_t blocks, int32_t block_rows)
{
    return block_rows > 1 ? blocks * kSquareThreads : (blocks + 15) / 16 * 256;
}

hipError_t launch_fp8_quantize(QuantizeArgs a, int32_t block_rows, int32_t x_type, hipStream_t stream)
{
    const int64_t row_blocks = (a.cols + kBlock - 1) / kBlock, all = (a.rows + block_rows - 1) / block_rows;
    const QuantizeCut cut = fp8_quantize_cut(row_blocks, block_rows);
    for (int64_t row = 0; row < all; row += cut.rows)
        for (int64_t column = 0; column < row_blocks; column += cut.columns) {
            const int64_t rows = std::min(cut.rows, all - row), columns = std::min(cut.columns, row_blocks - column);
            QuantizeArgs p = a;
            p.x = static_cast<const char *>(a.x) + (row * block_rows * a.x_stride + column * kBlock) * (x_type == QUAMBA_F32 ? 4 : 2);
            p.q = a.q + row * block_rows * a.q_stride + column * kBlock;
            p.scales = a.scales + row * row_blocks + column;  // a part of a row of blocks: there is no other row in the launch
            p.rows = std::min(a.rows - row * block_rows, rows * block_rows);
            p.cols = std::min(a.cols - column * kBlock, columns * kBlock);
            p.row_blocks = (int32_t)columns;
            p.by_row_blocks = divisor((uint32_t)columns);
            p.blocks = (int32_t)(rows * columns);
            switch (x_type) {
                case QUAMBA_F32: launch<QUAMBA_F32>(p, block_rows > 1, stream); break;
                case QUAMBA_F16: launch<QUAMBA_F16>(p, block_rows > 1, stream); break;
                default: launch<QUAMBA_BF16>(p, block_rows > 1, stream); break;
            }
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

}  // namespace quamba
