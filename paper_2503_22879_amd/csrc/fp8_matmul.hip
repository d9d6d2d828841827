// Matrix product of e4m3 operands with a scale for each block of 128 along the depth:
//
//   y[i, j] = sum_b xs[i, b] ws[j / 128, b] sum_{k in b} x[i, k] w[j, k]
//
// Codes become fp16 values in registers (exact) and meet in fp16 matrix instructions, whose sums are fp32; a block's sum is scaled into
// the output's.  The e4m3 matrix instruction would be twice as fast, but it cuts the products of eight neighbours along the
// depth 13 bits below the largest of them: sums of 128 normal values are off by 1.6e-5 of themselves, and by 5e-5 where the
// values' sizes spread, against 1e-8 here.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "quamba_internal.h"

namespace quamba {
namespace {

typedef int int8v __attribute__((ext_vector_type(8)));      // 32 e4m3 codes
typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;

// 16 codes `at` of a row, of which the first `left` belong to it; the others count as zeros.  A row's end is read with the codes in front
// of it, in one access (322 x 12227 x 90: 10.1 us, and 14.1 us byte by byte).
__device__ __forceinline__ int4v load16(const uint8_t *row, int at, int left)
{
    int4v w{0, 0, 0, 0};
    if (left >= 16 || (left > 0 && at >= 16)) {
        const int before = max(0, 16 - left);
        __builtin_memcpy(&w, row + at - before, 16);
        if (before) {
            uint64_t v[2];
            __builtin_memcpy(v, &w, 16);
            const int bits = before % 8 * 8;
            v[0] = before < 8 ? v[0] >> bits | v[1] << 1 << (63 - bits) : v[1] >> bits;
            v[1] = before < 8 ? v[1] >> bits : 0;
            __builtin_memcpy(&w, v, 16);
        }
    } else if (left > 0) {  // a row of fewer than 16
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * i + j < left) v |= (uint32_t)row[4 * i + j] << 8 * j;
            w[i] = (int)v;
        }
    }
    return w;
}

// 32 codes of a row (a lane's part of a block) as fp16 values.
struct Part {
    half8 h[4];
    __device__ __forceinline__ Part() {}
    __device__ __forceinline__ Part(const int4v &lo, const int4v &hi, int n = 4)  // the first n of h
    {
#pragma unroll
        for (int i = 0; i < n; ++i) {
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
__device__ __forceinline__ float4v multiply(const Part &a, const Part &b, int n = 4)
{
    float4v p{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < n; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h[i], b.h[i], p, 0, 0, 0);
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

template <int TYPE>
__device__ __forceinline__ uint16_t half_bits(float v)
{
    return TYPE == QUAMBA_F16 ? f32_to_f16_bits(v) : __builtin_bit_cast(uint16_t, (__bf16)v);
}

// N adjacent values of a row at `at`, of which the first `left` belong to it.
template <int TYPE, int N>
__device__ __forceinline__ void store_row(void *y, int64_t at, const float (&v)[N], int left)
{
    if (TYPE == QUAMBA_F32) {
        float *p = static_cast<float *>(y) + at;
        if (left >= N) {
#pragma unroll
            for (int i = 0; i < N; i += 4) __builtin_memcpy(p + i, &v[i], 16);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < left) p[i] = v[i];
        }
    } else {
        uint16_t *p = static_cast<uint16_t *>(y) + at;
        uint16_t h[N];
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] = half_bits<TYPE>(v[i]);
        if (left >= N) {
#pragma unroll
            for (int i = 0; i < N; i += 8) __builtin_memcpy(p + i, &h[i], N < 8 ? 2 * N : 16);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < left) p[i] = h[i];
        }
    }
}

// 16 (or 4) bytes for each lane from `base` + its offset into LDS at `to` + 16 (4) times the lane, without a register between.  Their
// arrival counts as a vector load's: wait_for_tiles() and wait_for_loads() wait for it.
__device__ __forceinline__ void load_to_lds16(const void *base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_to_lds4(const void *base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory", "m0");
}
// Until all but the wave's last N loads have arrived, and all its reads from LDS; then for the other waves.
template <int N>
__device__ __forceinline__ void wait_for_tiles() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}

// ---- up to 64 rows of x: the weight streams past ----

template <int N>
__device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

constexpr int rows_ahead(int mf, int waves) { return mf * waves > 8 && waves > 4 ? 2 : 3; }  // blocks of a ring
constexpr int rows_stage(int mf) { return (2 + 2 * mf) * 1024 + 256; }                      // bytes of one

// 16 columns of y (rows of w) at a time to a workgroup, over the whole depth, every wave one block in kWaves.  A wave has its own ring of
// kAhead blocks in LDS, of 16 rows of w and 16 MF of x and the scales of x's rows, and waits for nobody until the waves' sums
// meet at the end of a column part; the loads go on into the next part meanwhile.  Rows pass through LDS because 8 lanes that
// take a row's 128 codes together are one access to a cache, and 16 lanes on 16 rows, as the products want them, are 16 (one row of x,
// 18560 x 4096: 15.0 us, 16 rows 24.6 us, straight to registers).  The order of a row's pieces in LDS is the tiles'
// below.  The first block depends on the workgroup: rows 4096 bytes apart lie in one channel of the memory, and
// workgroups that go through the depth together would all be at that one.
template <int MF, int kWaves, bool DIRECT>
__global__ __launch_bounds__(64 * kWaves) void fp8_matmul_rows_kernel(MatmulArgs a, int parts)
{
    constexpr int kAhead = rows_ahead(MF, kWaves), kTurns = 2 + 2 * MF, kStage = rows_stage(MF), kLoads = kTurns + 1;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, r = lane & 15, part = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char *ring = lds + wave * kAhead * kStage;
    auto red = reinterpret_cast<float(*)[kWaves][MF * 4][64]>(lds + kWaves * kAhead * kStage);
    const uint32_t ring_at = lds_address(ring);
    const int whole = a.k / kBlock, each = (a.blocks - wave + kWaves - 1) / kWaves;  // blocks of this wave in a part
    const int mine = (parts - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;  // parts of this workgroup
    auto columns = [&](int q) { return ((int)blockIdx.x + q * (int)gridDim.x) * 16; };
    const int turned = (int)(blockIdx.x >> 3) % a.blocks;
    auto block = [&](int i) {
        const int b = wave + i * kWaves + turned;
        return b >= a.blocks ? b - a.blocks : b;
    };
    // 8 rows in turn, 8 lanes to a row: w's 16, then x's
    auto piece_of = [&](int turn) { return (lane & 7) ^ ((turn & 1) << 2 | lane >> 4); };
    const int last_piece = (a.k - whole * kBlock) / 16 - 1;  // of a last block in part
    uint32_t x_offset[DIRECT ? 2 * MF : 1], scale_offset = 0;
    if (DIRECT) {
#pragma unroll
        for (int t = 0; t < 2 * MF; ++t) x_offset[t] = (uint32_t)min(t * 8 + (lane >> 3), a.m - 1) * (uint32_t)a.x_stride;
        scale_offset = (uint32_t)min(lane, a.m - 1) * (uint32_t)a.blocks * 4;
    }
    auto start = [&](int slot, int n0, int b) {  // DIRECT: any block; the pieces behind the depth repeat the last one
        const int most = b < whole ? 7 : last_piece;
        const uint32_t to = ring_at + slot * kStage;
        const uint8_t *x = a.x + (int64_t)b * kBlock, *w = a.w + (int64_t)n0 * a.w_stride + (int64_t)b * kBlock;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what was read from the slot has arrived
#pragma unroll
        for (int t = 0; t < 2; ++t)
            load_to_lds16(w, (uint32_t)min(t * 8 + (lane >> 3), a.n - 1 - n0) * (uint32_t)a.w_stride + min(piece_of(t), most) * 16, to + t * 1024);
#pragma unroll
        for (int t = 0; t < 2 * MF; ++t) load_to_lds16(x, x_offset[t] + min(piece_of(t), most) * 16, to + 2048 + t * 1024);
        load_to_lds4(a.x_scales + b, scale_offset, to + kTurns * 1024);
    };
    int4v held[kTurns];
    float held_scale;
    auto fetch = [&](int n0, int b) {  // any block, to registers
        auto row = [&](int t) {
            return t < 2 ? a.w + (int64_t)min(n0 + t * 8 + (lane >> 3), a.n - 1) * a.w_stride
                         : a.x + (int64_t)min((t - 2) * 8 + (lane >> 3), a.m - 1) * a.x_stride;
        };
        if (b < whole) {
#pragma unroll
            for (int t = 0; t < kTurns; ++t) __builtin_memcpy(&held[t], row(t) + (int64_t)b * kBlock + piece_of(t) * 16, 16);
        } else {
#pragma unroll
            for (int t = 0; t < kTurns; ++t) held[t] = load16(row(t), b * kBlock + piece_of(t) * 16, a.k - b * kBlock - piece_of(t) * 16);
        }
        held_scale = a.x_scales[(int64_t)min(lane, a.m - 1) * a.blocks + b];
    };
    auto put = [&](int slot) {
        char *to = ring + slot * kStage;
#pragma unroll
        for (int t = 0; t < kTurns; ++t) *reinterpret_cast<int4v *>(to + t * 1024 + lane * 16) = held[t];
        reinterpret_cast<float *>(to + kTurns * 1024)[lane] = held_scale;
    };
    float4v sum[MF];
    const int at = r * kBlock + (part ^ r >> 1) * 16;
    struct Raw {  // a block of the ring in registers
        int4v w[2], x[MF][2];
        float xs[MF], ws;
    };
    auto read = [&](Raw &v, int slot, int n0, int b) {
        const char *from = ring + slot * kStage;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v.w[h] = *reinterpret_cast<const int4v *>(from + (at ^ 64 * h));
#pragma unroll
            for (int f = 0; f < MF; ++f) v.x[f][h] = *reinterpret_cast<const int4v *>(from + 2048 * (1 + f) + (at ^ 64 * h));
        }
#pragma unroll
        for (int f = 0; f < MF; ++f) v.xs[f] = reinterpret_cast<const float *>(from + kTurns * 1024)[f * 16 + r];
        v.ws = ((const __attribute__((address_space(4))) float *)a.w_scales)[(int64_t)(n0 / kBlock) * a.blocks + b];
    };
    auto step = [&](Raw &v, int b) {
        if (DIRECT && b >= whole) {  // what stands behind the depth counts as zeros
            const int4v none{0, 0, 0, 0};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool in = part + 4 * h <= last_piece;
                v.w[h] = in ? v.w[h] : none;
#pragma unroll
                for (int f = 0; f < MF; ++f) v.x[f][h] = in ? v.x[f][h] : none;
            }
        }
        const Part wf(v.w[0], v.w[1]);
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            const float4v p = multiply(wf, Part(v.x[f][0], v.x[f][1]));
            const float scale = v.xs[f] * v.ws;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[f][e] = fmaf(p[e], scale, sum[f][e]);
        }
    };
    auto clear = [&] {
#pragma unroll
        for (int f = 0; f < MF; ++f) sum[f] = float4v{0, 0, 0, 0};
    };
    auto finish = [&](int q) {  // the waves' sums of a part meet
        const int n0 = columns(q);
        auto &sums = red[q & 1];
#pragma unroll
        for (int f = 0; f < MF; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[wave][4 * f + e][lane] = sum[f][e];
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // not for the loads
        for (int t = threadIdx.x; t < MF * 256; t += 64 * kWaves) {
            const int i = t >> 4, j = t & 15;
            const int e = 4 * (i >> 4) + (j & 3), from = (j >> 2) * 16 + (i & 15);
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v += sums[w][e][from];
            if (i < a.m && n0 + j < a.n) store(a.y, a.y_type, i * a.y_stride + n0 + j, v);
        }
        clear();
    };
    clear();
    if (each == 0) {  // fewer blocks than waves
        for (int q = 0; q < mine; ++q) finish(q);
        return;
    }
    if (!DIRECT) {
        Raw v;
        for (int q = 0; q < mine; ++q) {
            fetch(columns(q), block(0));
            for (int i = 0; i < each; ++i) {
                put(0);
                if (i + 1 < each) fetch(columns(q), block(i + 1));
                read(v, 0, columns(q), block(i));
                step(v, block(i));
            }
            finish(q);
        }
        return;
    }
    // The loads run kAhead blocks ahead of the products, through the blocks of this workgroup's parts, and the reads from LDS one
    // block: a wave has its SIMD for itself or nearly so, and would wait for each of them.
    int next_q = 0, next_i = 0, slot = 0, q = 0, i = 0;
    auto ahead = [&](int to) {
        if (next_q < mine) {
            start(to, columns(next_q), block(next_i));
            if (++next_i == each) {
                next_i = 0;
                ++next_q;
            }
        }
    };
    for (int u = 0; u < kAhead; ++u) ahead(u);
    Raw even, odd;
    auto wait = [&] {  // for the block behind the kAhead - 1 last ones
        if (next_q < mine)
            wait_for_loads<kLoads *(kAhead - 1)>();
        else
            wait_for_loads<0>();
    };
    wait();
    read(even, 0, columns(0), block(0));
    auto turn = [&](Raw &now, Raw &then) {  // false behind the last block
        const int b = block(i), this_q = q;
        const bool ends = ++i == each;
        if (ends) {
            i = 0;
            ++q;
        }
        ahead(slot);  // `now` has left it
        slot = slot + 1 == kAhead ? 0 : slot + 1;
        if (q < mine) {
            wait();
            read(then, slot, columns(q), block(i));
        }
        step(now, b);
        if (ends) finish(this_q);
        return q < mine;
    };
    while (turn(even, odd) && turn(odd, even)) {
    }
}

// ---- more rows: tiles of x and w in LDS ----

// The order of the tiles: the device hands workgroups to its 8 dies in turn, so every eighth one belongs to a die; each die gets
// consecutive tiles, and these go up and down bands of 8 tiles along m, so that the die's cache holds what they share.
__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int &tm, int &tn)
{
    constexpr int kDies = 8, kBand = 8;
    const int all = tiles_m * tiles_n, each = all / kDies, more = all % kDies, die = id % kDies;
    id = die * each + min(die, more) + id / kDies;
    const int band = id / (kBand * tiles_n), first = band * kBand, rows = min(kBand, tiles_m - first);
    const int in_band = id - first * tiles_n;
    tn = in_band / rows;
    tm = first + in_band - tn * rows;
}

// The row of w's scales that wave `wn` of the tile at column n0 takes.  A wave's columns lie in one block of 128; one that has
// none in y takes the last row that there is.
template <int BN, int WN>
__host__ __device__ __forceinline__ int32_t scale_row(int32_t n0, int wn, int32_t n)
{
    const int32_t column = n0 + wn * (BN / WN);
    return (column < n ? column : n - 1) / kBlock;
}

// BM x BN outputs to a workgroup of WM x WN waves.  LDS holds STAGES blocks (128 codes deep) of BM + BN rows and the scales of x's rows;
// blocks arrive while earlier ones are multiplied.  A lane takes pieces l / 16 and l / 16 + 4 of the 8 of 16 bytes that a row has (any
// order along the depth will do that is the same for x and w), and piece c of row r lies at c ^ (r / 2 % 8), so that the lanes that
// read together hit different banks.  Which row of w stands where in a 16-row part is free as well: row 4 p + e of part j is the
// wave's row 4 TN p + 4 j + e, so that a lane ends up with 4 TN adjacent columns of y.  DIRECT: rows at multiples of 16 bytes less
// than 2^24 bytes apart, and a depth of whole pieces, go from memory to LDS by themselves; else through registers.
// GROUPS of WM x WN waves take the blocks in turn, each from stages of its own, and their sums meet in LDS at the end: more waves to
// wait for memory and LDS where tiles are small.  `splits`: workgroups to a tile, each with a part of the depth, whose sums go to
// `partial` [splits, m, columns].
template <int BM, int BN, int WM, int WN, int GROUPS, int STAGES, bool DIRECT>
__global__ __launch_bounds__(64 * WM * WN * GROUPS, 2) void fp8_matmul_tile_kernel(MatmulArgs a, int tiles_m, int tiles_n, int splits, float *partial,
                                                                          int64_t columns)
{
    constexpr int kWaves = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int kRows = BM + BN, kScales = kRows * kBlock, kStage = kScales + BM * 4, kTurns = kRows / 8 / kWaves;
    static_assert(kTurns * 8 * kWaves == kRows && kTurns % 2 == 0 && BM / 8 % kWaves == 0 && BM % 64 == 0 && BM / 64 <= kWaves && kBlock % (BN / WN) == 0, "");
    static_assert((GROUPS - 1) * BM * BN * 4 + kWaves * 16 * (64 * TN + 16) <= GROUPS * STAGES * kStage, "");
    extern __shared__ __align__(16) char all_lds[];
    const int lane = threadIdx.x & 63, r = lane & 15, part = lane >> 4, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = any_wave / kWaves, wave = any_wave % kWaves, thread = wave * 64 + lane;
    const int wm = wave % WM, wn = wave / WM;
    char *lds = all_lds + group * STAGES * kStage;
    int tm, tn;
    const int split = blockIdx.y;
    tile_of(blockIdx.x, tiles_m, tiles_n, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;
    const uint8_t *xb = a.x + (int64_t)m0 * a.x_stride, *wb = a.w + (int64_t)n0 * a.w_stride;
    const float *xsb = a.x_scales + (int64_t)m0 * a.blocks;
    const auto *ws = (const __attribute__((address_space(4))) float *)(a.w_scales + (int64_t)scale_row<BN, WN>(n0, wn, a.n) * a.blocks);
    const int last_x = a.m - 1 - m0, last_w = a.n - 1 - n0;
    const int whole = a.k / kBlock, last_piece = (a.k - whole * kBlock) / 16 - 1;  // of a last block in part
    const int first = (int)((int64_t)a.blocks * split / splits), end = (int)((int64_t)a.blocks * (split + 1) / splits);
    const int turns = (end - first + GROUPS - 1) / GROUPS, mine = (end - first - group + GROUPS - 1) / GROUPS;  // blocks
    auto block = [&](int i) { return first + group + i * GROUPS; };

    // 8 rows of a tile in turn: this lane's piece of them
    auto row_of = [&](int turn) { return (turn * kWaves + wave) * 8 + (lane >> 3); };
    auto is_x = [&](int turn) { return (turn * kWaves + wave) * 8 < BM; };
    auto order = [&](int turn) {  // among the 16 rows that are read together
        const int row = row_of(turn);
        return is_x(turn) ? row >> 1 & 7 : (row >> 1 & 1) | (row / (4 * TN) & 3) << 1;
    };
    auto piece_of = [&](int turn) { return (lane & 7) ^ order(turn); };
    // A lane's place in the first rows of x or w that its wave takes in turn: the others are as many rows on.
    auto first_offset = [&](int turn, int64_t stride) { return (uint32_t)(wave * 8 + (lane >> 3)) * (uint32_t)stride + piece_of(turn) * 16; };
    const uint32_t scale_offset = (uint32_t)min(wave % (BM / 64) * 64 + lane, last_x) * (uint32_t)a.blocks * 4;
    const bool inside = last_x >= BM - 1 && last_w >= BN - 1;  // the tile lies in y
    const uint32_t base = lds_address(lds);
    // DIRECT: a half of block b (2: all of it) on its way into a stage.  Every wave issues as many loads as the others (the scales more
    // than once).
    auto start = [&](int b, int stage, int half) {
        const uint32_t to = base + stage * kStage;
        const uint8_t *x = xb + (int64_t)b * kBlock, *w = wb + (int64_t)b * kBlock;
        if (b < whole && inside) {
#pragma unroll
            for (int t = 0; t < kTurns; ++t)
                if (half == 2 || half == t / (kTurns / 2)) {
                    const int on = (is_x(t) ? t : t - BM / 8 / kWaves) * kWaves * 8;
                    load_to_lds16(is_x(t) ? x + on * a.x_stride : w + on * a.w_stride, first_offset(t, is_x(t) ? a.x_stride : a.w_stride),
                                  to + (t * kWaves + wave) * 1024);
                }
        } else {  // rows over the edge repeat the last one, pieces behind the depth too
            const int most = b < whole ? 7 : last_piece;
#pragma unroll
            for (int t = 0; t < kTurns; ++t)
                if (half == 2 || half == t / (kTurns / 2))
                    load_to_lds16(is_x(t) ? x : w,
                                  (is_x(t) ? (uint32_t)min(row_of(t), last_x) * (uint32_t)a.x_stride
                                           : (uint32_t)min(row_of(t) - BM, last_w) * (uint32_t)a.w_stride) + min(piece_of(t), most) * 16,
                                  to + (t * kWaves + wave) * 1024);
        }
        if (half != 1) load_to_lds4(xsb + b, scale_offset, to + kScales + wave % (BM / 64) * 256);
    };
    int4v held[DIRECT ? 1 : kTurns];
    float held_scale = 0.0f;
    auto fetch = [&](int b) {  // any block, to registers
        constexpr int kHeld = DIRECT ? 1 : kTurns;
        auto row = [&](int t) { return is_x(t) ? xb + (int64_t)min(row_of(t), last_x) * a.x_stride : wb + (int64_t)min(row_of(t) - BM, last_w) * a.w_stride; };
        if (b < whole) {
#pragma unroll
            for (int t = 0; t < kHeld; ++t) __builtin_memcpy(&held[t], row(t) + (int64_t)b * kBlock + piece_of(t) * 16, 16);
        } else {
#pragma unroll
            for (int t = 0; t < kHeld; ++t) held[t] = load16(row(t), b * kBlock + piece_of(t) * 16, a.k - b * kBlock - piece_of(t) * 16);
        }
        if (thread < BM) held_scale = xsb[(int64_t)min(thread, last_x) * a.blocks + b];
    };
    auto put = [&](int stage) {
        char *to = lds + stage * kStage;
#pragma unroll
        for (int t = 0; t < (DIRECT ? 1 : kTurns); ++t) *reinterpret_cast<int4v *>(to + (t * kWaves + wave) * 1024 + lane * 16) = held[t];
        if (thread < BM) reinterpret_cast<float *>(to + kScales)[thread] = held_scale;
    };

    float4v sum[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) sum[i][j] = float4v{0, 0, 0, 0};
    const int at = r * kBlock + (part ^ r >> 1) * 16, at_w = ((r >> 2) * 4 * TN + (r & 3)) * kBlock + (part ^ r >> 1) * 16;
    // Multiplies block b; between its first parts block `next` (below 0: none) is started, in two halves: a wave waits where it
    // issues more loads than fit a queue, and after the first part's reads it has products to make meanwhile (16384 x 18560 x 4096: 2.15 -> 2.11 ms).
    // codes_of_it: how many there may be in the block; parts that hold none are not multiplied.
    auto compute = [&](int b, int stage, int next, int next_stage, auto codes_of_it) {
        constexpr int kCodes = decltype(codes_of_it)::value, kHalves = kCodes == 64 ? 2 : 4;
        const char *x = lds + stage * kStage + wm * (BM / WM) * kBlock, *w = lds + stage * kStage + (BM + wn * (BN / WN)) * kBlock;
        const float *xs = reinterpret_cast<const float *>(lds + stage * kStage + kScales) + wm * (BM / WM) + r;
        const float wsc = ws[b];
        auto codes = [&](const char *p, int to) {
            int4v c0 = *reinterpret_cast<const int4v *>(p + to), c1 = c0;
            if (kCodes > 64) c1 = *reinterpret_cast<const int4v *>(p + (to ^ 64));
            if (kCodes < kBlock) {  // what stands behind the depth counts as zeros
                c0 = part <= last_piece ? c0 : int4v{0, 0, 0, 0};
                c1 = part + 4 <= last_piece ? c1 : int4v{0, 0, 0, 0};
            }
            return Part(c0, c1, kHalves);
        };
        Part wf[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) wf[j] = codes(w + j * 4 * kBlock, at_w);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const Part xf = codes(x + i * 16 * kBlock, at);
            if (DIRECT && i < 2 && next >= 0) start(next, next_stage, i);
            const float s = xs[i * 16] * wsc;
            float4v p[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) p[j] = multiply(wf[j], xf, kHalves);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[i][j][e] = fmaf(p[j][e], s, sum[i][j][e]);
        }
    };
    const std::integral_constant<int, kBlock> all_of_it;
    const std::integral_constant<int, kBlock - 16> most_of_it;  // at most
    const std::integral_constant<int, 64> half_of_it;

    if (DIRECT) {
        for (int u = 0; u < STAGES - 1; ++u)
            if (u < mine) start(block(u), u, 2);
        int stage = 0, i = 0;
        for (; i < mine && block(i) < whole; ++i) {
            // block i is there for all waves, and block i - 1 has been read by all
            if (STAGES > 2 && i + STAGES - 2 < mine)
                wait_for_tiles<(kTurns + 1) * (STAGES - 2)>();
            else
                wait_for_tiles<0>();
            const int next = i + STAGES - 1;
            compute(block(i), stage, next < mine ? block(next) : -1, stage ? stage - 1 : STAGES - 1, all_of_it);
            stage = stage + 1 == STAGES ? 0 : stage + 1;
        }
        for (; i < turns; ++i) {  // at most one, for the group's partial block or for the others
            wait_for_tiles<0>();
            if (TM * TN < 32 && i < mine && last_piece < 4)  // (no registers for it where the sums take half of them)
                compute(block(i), stage, -1, 0, half_of_it);
            else if (i < mine)
                compute(block(i), stage, -1, 0, most_of_it);
        }
    } else {
        if (mine) fetch(block(0));
        for (int i = 0; i < turns; ++i) {
            if (i < mine) put(i & 1);
            __syncthreads();
            if (i + 1 < mine) fetch(block(i + 1));
            if (i < mine) compute(block(i), i & 1, -1, 0, all_of_it);
        }
    }
    if (GROUPS > 1) {
        float *sums = reinterpret_cast<float *>(all_lds) + wave * TM * TN * 256 + lane;
        __syncthreads();
        if (group)
#pragma unroll
            for (int i = 0; i < TM * TN * 4; ++i) sums[(group - 1) * BM * BN + i * 64] = sum[i / 4 / TN][i / 4 % TN][i % 4];
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int g = 1; g < GROUPS; ++g)
#pragma unroll
            for (int i = 0; i < TM * TN * 4; ++i) sum[i / 4 / TN][i / 4 % TN][i % 4] += sums[(g - 1) * BM * BN + i * 64];
    }
    // A lane has 4 TN adjacent columns of a row and its neighbours have other rows, so 16 rows at a time pass through LDS, from where
    // lanes take 16 bytes side by side (rows padded by 16 bytes: writes and reads spread over the banks).
    if (GROUPS == 1) __syncthreads();
    char *turn = all_lds + (GROUPS - 1) * BM * BN * 4 + wave * 16 * (64 * TN + 16);
    auto write = [&](auto type, void *y, int64_t stride) {
        constexpr int kType = decltype(type)::value, kBytes = kType == QUAMBA_F32 ? 4 : 2, kVec = 16 / kBytes;
        constexpr int kRow = 16 * TN * kBytes + 16, kLanes = 16 * TN * kBytes / 16;  // bytes of a row in LDS, lanes to it
        const int col = n0 + wn * (BN / WN) + lane % kLanes * kVec;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            uint32_t v[TN * kBytes];
#pragma unroll
            for (int j = 0; j < TN * kBytes; ++j) {
                const int at = kBytes == 4 ? j : 2 * j;  // of the lane's columns
                const float lo = sum[i][at / 4][at % 4], hi = kBytes == 4 ? 0.0f : sum[i][at / 4][(at + 1) % 4];
                v[j] = kBytes == 4 ? __builtin_bit_cast(uint32_t, lo) : (uint32_t)half_bits<kType>(lo) | (uint32_t)half_bits<kType>(hi) << 16;
            }
#pragma unroll
            for (int j = 0; j < TN * kBytes / 4; ++j)
                *reinterpret_cast<int4v *>(turn + r * kRow + part * 4 * TN * kBytes + j * 16) = int4v{(int)v[4 * j], (int)v[4 * j + 1], (int)v[4 * j + 2], (int)v[4 * j + 3]};
#pragma unroll
            for (int q = 0; q < kLanes / 4; ++q) {
                const int in = q * (64 / kLanes) + lane / kLanes, row = m0 + wm * (BM / WM) + i * 16 + in;
                const int4v w = *reinterpret_cast<const int4v *>(turn + in * kRow + lane % kLanes * 16);
                char *to = static_cast<char *>(y) + (row * stride + col) * kBytes;
                if (row < a.m && col + kVec <= a.n) {
                    __builtin_memcpy(to, &w, 16);
                } else if (row < a.m) {
#pragma unroll
                    for (int e = 0; e < kVec; ++e)
                        if (col + e < a.n) {
                            if (kBytes == 4)
                                reinterpret_cast<int *>(to)[e] = w[e];
                            else
                                reinterpret_cast<uint16_t *>(to)[e] = (uint16_t)((uint32_t)w[e / 2] >> e % 2 * 16);
                        }
                }
            }
        }
    };
    if (splits > 1)
        write(std::integral_constant<int, QUAMBA_F32>(), partial + (int64_t)split * a.m * columns, columns);
    else if (a.y_type == QUAMBA_F32)
        write(std::integral_constant<int, QUAMBA_F32>(), a.y, a.y_stride);
    else if (a.y_type == QUAMBA_F16)
        write(std::integral_constant<int, QUAMBA_F16>(), a.y, a.y_stride);
    else
        write(std::integral_constant<int, QUAMBA_BF16>(), a.y, a.y_stride);
}

// y of the splits' sums, in their order; 4 columns to a thread, every gridDim.y-th row to a workgroup.
__global__ __launch_bounds__(256) void fp8_matmul_join_kernel(MatmulArgs a, int splits, const float *partial, int64_t columns)
{
    const int col = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4;
    if (col >= a.n) return;
    for (int64_t row = blockIdx.y; row < a.m; row += gridDim.y) {
        const float *p = partial + row * columns + col;
        float4v v = *reinterpret_cast<const float4v *>(p);
        for (int s = 1; s < splits; ++s) v += *reinterpret_cast<const float4v *>(p + (int64_t)s * a.m * columns);
        const float out[4] = {v[0], v[1], v[2], v[3]};
        const int64_t to = row * a.y_stride + col;
        if (a.y_type == QUAMBA_F32)
            store_row<QUAMBA_F32>(a.y, to, out, a.n - col);
        else if (a.y_type == QUAMBA_F16)
            store_row<QUAMBA_F16>(a.y, to, out, a.n - col);
        else
            store_row<QUAMBA_BF16>(a.y, to, out, a.n - col);
    }
}

template <int BM, int BN, int WM, int WN, int GROUPS, int STAGES, bool DIRECT>
hipError_t launch_tiles(const MatmulArgs &a, int splits, float *partial, hipStream_t stream)
{
    constexpr auto kernel = &fp8_matmul_tile_kernel<BM, BN, WM, WN, GROUPS, STAGES, DIRECT>;
    hipError_t e = allow_full_lds<kernel>();
    if (e != hipSuccess) return e;
    const int tiles_m = (a.m + BM - 1) / BM, tiles_n = (a.n + BN - 1) / BN;
    const int64_t columns = ((int64_t)a.n + 3) / 4 * 4;
    constexpr int kLds = GROUPS * STAGES * ((BM + BN) * kBlock + BM * 4);
    static_assert(kLds <= (int)kLdsPerCu, "");
    kernel<<<dim3(tiles_m * tiles_n, splits), 64 * WM * WN * GROUPS, kLds, stream>>>(a, tiles_m, tiles_n, splits, partial, columns);
    e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    fp8_matmul_join_kernel<<<dim3((a.n + 1023) / 1024, fp8_matmul_join_rows(a.m)), 256, 0, stream>>>(a, splits, partial, columns);
    return hipGetLastError();
}

template <int MF, int kWaves, bool DIRECT>
hipError_t launch_rows_as(const MatmulArgs &a, hipStream_t stream)
{
    constexpr auto kernel = &fp8_matmul_rows_kernel<MF, kWaves, DIRECT>;
    constexpr size_t kRing = (size_t)rows_ahead(MF, kWaves) * rows_stage(MF) * kWaves, kSums = 2 * kWaves * MF * 1024;
    static_assert(kRing + kSums <= kLdsPerCu, "");
    const hipError_t e = allow_full_lds<kernel>();
    if (e != hipSuccess) return e;
    const int parts = (a.n + 15) / 16, resident = (int)(kLdsPerCu / (kRing + kSums)) * compute_units();
    kernel<<<std::min(parts, resident), 64 * kWaves, kRing + kSums, stream>>>(a, parts);
    return hipGetLastError();
}

// Waves of a workgroup for up to 64 rows: the depth in more parts where a unit has no more than one workgroup.
int rows_waves(int32_t m, int32_t n, int32_t blocks) { return m <= 32 && (n + 15) / 16 <= compute_units() && blocks >= 16 ? 8 : 4; }

template <int MF, bool DIRECT>
hipError_t launch_rows(const MatmulArgs &a, hipStream_t stream)
{
    if (MF < 4 && rows_waves(a.m, a.n, a.blocks) == 8) return launch_rows_as<MF, MF < 4 ? 8 : 4, DIRECT>(a, stream);
    return launch_rows_as<MF, 4, DIRECT>(a, stream);
}

constexpr int kMostSplits = 16;  // parts of the depth

// Tiles of 256 x 256, see below.
double tiles256_us(int32_t m, int32_t n, int32_t blocks)
{
    const int64_t tiles = ((int64_t)m + 255) / 256 * (((int64_t)n + 255) / 256), units = compute_units();
    return 1.0 + (double)((tiles + units - 1) / units) * (9.0 + 3.35 * blocks);
}

}  // namespace

// The form that is estimated to be done first, from what a round of workgroups takes in us on 256 units: a fixed time and one for each
// turn (a block of 128 of the depth, or two where two groups of waves share them).
//
//   form                                 fixed  turn   measured                            next best
//   rows, 17 to 32 rows of x             3.5    0.7    32 x 18560 x 4096           28      64 x 128            23 (taken)
//   rows, 33 to 64                       3.5    0.95   64 x 2560 x 5120            11.2    64 x 64 in 4 parts  12.3
//   64 x 64, two groups                  3      0.76   128 x 4096 x 8192, 2 parts  19.9    in one part         27
//   64 x 128, two groups                 3.8    1.17   500 x 4096 x 4096           24      64 x 64             33
//   128 x 128, two groups, one workgroup
//     to a unit                          4.2    1.85   1000 x 4096 x 8192          75      two to a unit       88
//   128 x 128, one group, two to a unit  3.5    2.0    8192 x 3352 x 768           55      256 x 256           59
//                                                      16331 x 4559 x 320          78      256 x 256           90
//   256 x 256                            9      3.35   16384 x 18560 x 4096        2050    128 x 128           2200
//                                                      256 x 50021 x 2560          74      128 x 128           79
//
// Up to 16 rows rings of rows are bound by memory and always taken.
Fp8Plan fp8_matmul_plan(int32_t m, int32_t n, int32_t blocks, bool workspace)
{
    if (m <= 16) return {Fp8Form::rows, 1, 0.0};
    const int units = compute_units();
    auto tiles = [&](int rows, int columns) { return ((int64_t)m + rows - 1) / rows * (((int64_t)n + columns - 1) / columns); };
    auto rounds = [&](int64_t workgroups) { return (double)((workgroups + units - 1) / units); };
    auto pairs = [&](int splits) { return (blocks + 2 * splits - 1) / (2 * splits); };
    Fp8Plan best{Fp8Form::tiles256, 1, tiles256_us(m, n, blocks)};
    auto offer = [&](Fp8Form form, int splits, double time) {
        if (time < best.us) best = {form, splits, time};
    };
    const int64_t t128 = tiles(128, 128);
    // a unit's second workgroup fills the gaps of the first, and a last round that is half empty is half as long
    offer(Fp8Form::tiles128_two, 1,
          t128 <= units ? 5.0 + 1.05 * blocks : 3.0 + (rounds(t128) + (double)t128 / units) / 4 * (3.5 + 2.0 * blocks));
    offer(Fp8Form::tiles128_one, 1, 1.0 + rounds(t128) * (4.2 + 1.85 * pairs(1)));
    offer(Fp8Form::tiles64x128, 1, 1.0 + rounds(tiles(64, 128)) * (3.8 + 1.17 * pairs(1)));
    for (int s = 1; s == 1 || (workspace && s <= kMostSplits && blocks / s >= 4); s *= 2)
        offer(Fp8Form::tiles64, s, 2.0 + rounds(tiles(64, 64) * s) * (3.0 + 0.76 * pairs(s)) + (s > 1 ? 2.5 + 1e-6 * s * m * n : 0.0));
    if (m <= 64) {
        const int64_t parts = ((int64_t)n + 15) / 16;
        offer(Fp8Form::rows, 1, 3.5 + (m <= 32 ? 0.7 : 0.95) * rounds(parts) * ((blocks - 1) / rows_waves(m, n, blocks) + 1));
    }
    return best;
}

// A last round of 256 x 256 with few tiles takes as long as a full one: the rows that make whole rounds so, where these and a form of
// their own for the others are estimated to take less than `us` (16384 x 18560 x 4096: 18.25 rounds; 16148 x 4224 x 7488: 4.25); else 0.
int32_t fp8_matmul_whole_rounds(int32_t m, int32_t n, int32_t blocks, double us)
{
    const int64_t tiles_m = ((int64_t)m + 255) / 256, tiles_n = ((int64_t)n + 255) / 256, units = compute_units();
    const int64_t rows = tiles_m * tiles_n / units * units / tiles_n * 256;
    if (rows == 0 || rows >= m) return 0;
    const double both = tiles256_us((int32_t)rows, n, blocks) + fp8_matmul_plan(m - (int32_t)rows, n, blocks, false).us;
    return both < us ? (int32_t)rows : 0;
}

// The plan where rows do not lie at multiples of 16 bytes or the depth ends inside a piece, so that operands go through registers and
// more workgroups to a unit hide their way better than more stages do.  A turn of a unit with w workgroups of 64 x 64 takes 0.25 + 0.55 w
// us, with one of 128 x 128 1.95 and with w of them 1.65 w: 90 x 11640 x 7641 takes 65 us in 64 x 64 (118 in
// 128 x 128), 1967 x 3304 x 3967 86 us in 128 x 128 (128 in 64 x 64), 50 x 4096 x 8191 18 us in 4 parts (34 with rings of rows).
Fp8Plan fp8_matmul_plan_unaligned(int32_t m, int32_t n, int32_t blocks, int most_splits)
{
    if (m <= 16) return {Fp8Form::rows, 1, 0.0};
    auto to_a_unit = [&](int size) { return (double)(((int64_t)m + size - 1) / size * (((int64_t)n + size - 1) / size)) / compute_units(); };
    const double w128 = to_a_unit(128);
    Fp8Plan best{Fp8Form::tiles128_two, 1, 3.0 + blocks * (w128 <= 1 ? 1.95 : 0.825 * (std::ceil(w128) + w128))};
    for (int s = 1; s == 1 || (s <= most_splits && blocks / s >= 4); s *= 2) {
        const double time = 3.0 + (blocks + s - 1) / s * (0.25 + 0.55 * std::max(1.0, to_a_unit(64) * s)) + (s > 1 ? 2.5 + 1e-6 * s * m * n : 0.0);
        if (time < best.us) best = {Fp8Form::tiles64, s, time};
    }
    return best;
}

namespace {

template <int BN, int WN>
int32_t last_scale_row(int32_t n)
{
    int32_t last = 0;
    for (int64_t n0 = 0; n0 < n; n0 += BN)
        for (int wn = 0; wn < WN; ++wn) last = std::max(last, scale_row<BN, WN>((int32_t)n0, wn, n));
    return last;
}

}  // namespace

int32_t fp8_matmul_last_scale_row(Fp8Form form, int32_t n)
{
    switch (form) {
        case Fp8Form::rows: return (n - 1) / kBlock;
        case Fp8Form::tiles64: return last_scale_row<64, 2>(n);
        case Fp8Form::tiles256: return last_scale_row<256, 4>(n);
        default: return last_scale_row<128, 2>(n);
    }
}

int32_t fp8_matmul_join_rows(int32_t m) { return std::min(m, kMaxGridY); }

namespace {

hipError_t launch_part(const MatmulArgs &a, void *workspace, hipStream_t stream)
{
    auto aligned = [](const uint8_t *p, int64_t stride) { return (reinterpret_cast<uintptr_t>(p) | (uint64_t)stride) % 16 == 0 && stride < 1 << 24; };
    const bool direct = aligned(a.x, a.x_stride) && aligned(a.w, a.w_stride) && a.k % 16 == 0;
    const Fp8Plan plan = fp8_matmul_plan(a.m, a.n, a.blocks, workspace);
    float *partial = static_cast<float *>(workspace);
    if (!direct) {  // the workspace has room for the splits of the depth's own plan
        const Fp8Plan other = fp8_matmul_plan_unaligned(a.m, a.n, a.blocks, !workspace ? 1 : a.k % 16 ? kMostSplits : plan.splits);
        if (other.form == Fp8Form::rows) return launch_rows<1, false>(a, stream);
        if (other.form == Fp8Form::tiles64) return launch_tiles<64, 64, 2, 2, 1, 2, false>(a, other.splits, partial, stream);
        return launch_tiles<128, 128, 2, 2, 1, 2, false>(a, 1, nullptr, stream);
    }
    if (const int32_t rows = fp8_matmul_whole_rounds(a.m, a.n, a.blocks, plan.us)) {
        MatmulArgs top = a, rest = a;
        top.m = rows;
        rest.m = a.m - rows;
        rest.x = a.x + rows * a.x_stride;
        rest.x_scales = a.x_scales + (int64_t)rows * a.blocks;
        rest.y = static_cast<char *>(a.y) + rows * a.y_stride * (a.y_type == QUAMBA_F32 ? 4 : 2);
        const hipError_t e = launch_tiles<256, 256, 2, 4, 1, 2, true>(top, 1, nullptr, stream);
        return e == hipSuccess ? launch_part(rest, nullptr, stream) : e;
    }
    switch (plan.form) {
        case Fp8Form::rows:
            return a.m <= 16 ? launch_rows<1, true>(a, stream) : a.m <= 32 ? launch_rows<2, true>(a, stream) : launch_rows<4, true>(a, stream);
        case Fp8Form::tiles64: return launch_tiles<64, 64, 2, 2, 2, 4, true>(a, plan.splits, partial, stream);
        case Fp8Form::tiles64x128: return launch_tiles<64, 128, 2, 2, 2, 3, true>(a, 1, nullptr, stream);
        case Fp8Form::tiles128_one: return launch_tiles<128, 128, 2, 2, 2, 2, true>(a, 1, nullptr, stream);
        case Fp8Form::tiles128_two: return launch_tiles<128, 128, 2, 2, 1, 2, true>(a, 1, nullptr, stream);
        default: return launch_tiles<256, 256, 2, 4, 1, 2, true>(a, 1, nullptr, stream);
    }
}

}  // namespace

size_t fp8_matmul_workspace_bytes(int32_t m, int32_t n, int32_t k)
{
    const int32_t blocks = (k + kBlock - 1) / kBlock;
    const int splits = k % 16 ? fp8_matmul_plan_unaligned(m, n, blocks, kMostSplits).splits : fp8_matmul_plan(m, n, blocks, true).splits;
    return splits > 1 ? (size_t)splits * m * (((size_t)n + 3) / 4 * 4) * sizeof(float) : 0;
}

hipError_t launch_fp8_matmul(const MatmulArgs &a, void *workspace, hipStream_t stream)
{
    // launches of fewer than 2^22 tiles of 128 x 128 (n has at most 2^19, m any number; 4 times as many of 64 x 64): threads and tiles fit 32 bits
    const int64_t tiles_n = ((int64_t)a.n + 127) / 128;
    const int64_t rows = std::max<int64_t>(1, ((int64_t)1 << 22) / tiles_n) * 128;
    for (int64_t first = 0; first < a.m; first += rows) {
        MatmulArgs p = a;
        p.m = (int32_t)std::min<int64_t>(rows, a.m - first);
        p.x = a.x + first * a.x_stride;
        p.x_scales = a.x_scales + first * a.blocks;
        p.y = static_cast<char *>(a.y) + first * a.y_stride * (a.y_type == QUAMBA_F32 ? 4 : 2);
        const hipError_t e = launch_part(p, first || p.m < a.m ? nullptr : workspace, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace quamba
