// Beam search: the best continuations of every sequence over its beams and the vocabulary, and the move of the cached states
// behind them.
//
//   value(k, v) = score_k + ((x_kv - max_k) - log sum_u exp(x_ku - max_k))
//
// A first launch reads the logits once: a workgroup takes a piece of one beam's row into registers and leaves its largest
// logit, its sum of exponentials against that and its best `count` logits.  A second one, a workgroup to a sequence, joins
// the pieces' sums, turns the pieces' best logits into values and takes the best of them.  Bound: HBM for large batches, two launches for
// small ones.
#include <algorithm>

#include "quamba_internal.h"

namespace quamba {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kGathered = 1024;  // candidates that are ranked against each other

// Floats as whole numbers of the same order; 0 is below all (the place of what is no candidate).
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_ordered(uint32_t o)
{
    return from_bits(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
    return v;
}

struct Chooser {
    uint64_t gathered[kGathered];
    uint32_t tops[kThreads];
    uint64_t wave_best[2][kWaves];
    int n;
};

// The `count` largest of the workgroup's keys, key(e) for e < E in every thread, 0 for none and otherwise all different: out[0 ..
// count - 1], largest first, 0 where there are no more.  `out` is written by some threads; the caller waits before it is read
// elsewhere.
//
// `count` threads have a key at least as large as the count-th largest of the threads' own largest ones, so nothing below that
// is among the best: what is left is mostly little more than `count` keys, which are ranked by counting.  The bound is
// sought bit by bit in the upper half of the keys, by every wave for itself.
template <int E, int BITS, typename Key, typename Out>
__device__ __forceinline__ void choose(Chooser &c, int count, const Key &key, const Out &out)
{
    const int t = threadIdx.x, lane = t & 63;
    uint64_t top = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) top = max(top, key(e));
    const uint32_t top_hi = (uint32_t)(top >> 32);
    c.tops[t] = top_hi;
    if (t == 0) c.n = 0;
    __syncthreads();
    uint32_t mine[kWaves], bound = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mine[w] = c.tops[w * 64 + lane];
    for (int bit = 31; bit >= 32 - BITS; --bit) {
        const uint32_t higher = bound | 1u << bit;
        int n = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[w] >= higher));
        if (n >= count) bound = higher;
    }
    bound = max(bound, 1u);
    if (top_hi >= bound)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint64_t k = key(e);
            if ((uint32_t)(k >> 32) >= bound) {
                const int at = atomicAdd(&c.n, 1);
                if (at < kGathered) c.gathered[at] = k;
            }
        }
    __syncthreads();
    const int n = c.n;
    if (n <= kGathered) {
        for (int i = t; i < n; i += kThreads) {
            const uint64_t k = c.gathered[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += c.gathered[j] > k;
            if (rank < count) out(rank, k);
        }
        for (int i = n + t; i < count; i += kThreads) out(i, (uint64_t)0);
    } else {  // many equal ones: one after the other
        uint64_t last = ~(uint64_t)0;
        for (int i = 0; i < count; ++i) {
            uint64_t best = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint64_t k = key(e);
                if (k < last && k > best) best = k;
            }
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                const uint64_t o = (uint64_t)__shfl_xor((long long)best, d, 64);
                best = max(best, o);
            }
            if (lane == 0) c.wave_best[i & 1][t / 64] = best;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) best = max(best, c.wave_best[i & 1][w]);
            last = best;
            if (t == 0) out(i, best);
        }
    }
}

// What a piece of a row leaves: its best logits (ordered logit above, complement of the token below), and its sum.
struct Piece {
    float max, sum;  // sum of exp(x - max); NaN for a row that has no distribution
};

__device__ __forceinline__ bool offers(const SelectArgs &a, int row)
{
    const float s = a.scores[row];
    return __builtin_fabsf(s) < __builtin_inff();
}

template <int TYPE>
__device__ __forceinline__ float logit_of(const char *p)
{
    if (TYPE == QUAMBA_F32) {
        float v;
        __builtin_memcpy(&v, p, 4);
        return v;
    }
    uint16_t h;
    __builtin_memcpy(&h, p, 2);
    return TYPE == QUAMBA_BF16 ? from_bits((uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
}

// A piece of 256 E logits to a workgroup.
template <int TYPE, int E>
__global__ __launch_bounds__(kThreads) void beam_pieces_kernel(SelectArgs a, int pieces, Divisor by_pieces, uint64_t *best,
                                                               Piece *piece)
{
    __shared__ Chooser chooser;
    __shared__ float wave_f[2][kWaves];
    const int row = quotient((int)blockIdx.x, by_pieces), part = blockIdx.x - row * pieces;
    if (!offers(a, row) || (a.finished && a.finished[row])) return;  // the second launch does not read it
    constexpr int kBytes = TYPE == QUAMBA_F32 ? 4 : 2, kVec = 16 / kBytes;
    const char *p = static_cast<const char *>(a.logits) + (int64_t)row * a.stride * kBytes;
    const int t = threadIdx.x;
    float x[E];
    const int first = part * (kThreads * E);
    auto token = [&](int e) { return first + (e / kVec * kThreads + t) * kVec + e % kVec; };
#pragma unroll
    for (int v = 0; v < E / kVec; ++v) {
        const int at = token(v * kVec);
        if (at + kVec <= a.vocab) {
            char raw[16];
            __builtin_memcpy(raw, p + (int64_t)at * kBytes, 16);
#pragma unroll
            for (int i = 0; i < kVec; ++i) x[v * kVec + i] = logit_of<TYPE>(raw + i * kBytes);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                x[v * kVec + i] = at + i < a.vocab ? logit_of<TYPE>(p + (int64_t)(at + i) * kBytes) : -__builtin_inff();
        }
    }
    float top = -__builtin_inff();
    bool bad = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        top = fmaxf(top, x[e]);
        bad |= !(x[e] < __builtin_inff());
    }
    top = bad ? __builtin_inff() : top;
    top = wave_max(top);
    if (t % 64 == 0) wave_f[0][t / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wave_f[0][0], wave_f[0][1]), fmaxf(wave_f[0][2], wave_f[0][3]));
    float sum = 0.0f;
    if (top > -__builtin_inff()) {
#pragma unroll
        for (int e = 0; e < E; ++e) sum += __expf(x[e] - top);
    }
    sum = group_sum<64>(sum);
    if (t % 64 == 0) wave_f[1][t / 64] = sum;
    uint64_t *to = best + (int64_t)blockIdx.x * a.count;
    choose<E, TYPE == QUAMBA_F32 ? 32 : 20>(
        chooser, a.count,
        [&](int e) {
            const uint32_t o = x[e] > -__builtin_inff() ? ordered(x[e] + 0.0f) : 0u;  // -0 is 0
            return o ? (uint64_t)o << 32 | (uint32_t)~token(e) : (uint64_t)0;
        },
        [&](int i, uint64_t k) { to[i] = k; });
    if (t == 0) {
        const float all = (wave_f[1][0] + wave_f[1][1]) + (wave_f[1][2] + wave_f[1][3]);
        piece[blockIdx.x] = {top, top < __builtin_inff() ? all : __builtin_nanf("")};
    }
}

// A workgroup to a sequence.
__global__ __launch_bounds__(kThreads) void beam_join_kernel(SelectArgs a, int pieces, const uint64_t *best, const Piece *piece)
{
    constexpr int E = 8;
    __shared__ Chooser chooser;
    __shared__ float score[kMaxBeams], row_max[kMaxBeams], row_log[kMaxBeams];
    __shared__ uint8_t kind[kMaxBeams];  // 0: offers nothing, 1: its pieces' tokens, 2: finished
    __shared__ uint64_t list[kMaxChoices];
    const int t = threadIdx.x, lane = t & 63, b = blockIdx.x;
    for (int k = t / 64; k < a.beams; k += kWaves) {
        const int row = b * a.beams + k;
        const bool valid = offers(a, row), done = a.finished && a.finished[row];
        float m = -__builtin_inff(), s = 0.0f;
        if (valid && !done) {
            const Piece *p = piece + (int64_t)row * pieces;
            for (int i = lane; i < pieces; i += 64) m = fmaxf(m, p[i].max);
            m = wave_max(m);
            if (m > -__builtin_inff())
                for (int i = lane; i < pieces; i += 64) s += p[i].sum * __expf(p[i].max - m);
            s = group_sum<64>(s);
        }
        if (lane == 0) {
            score[k] = a.scores[row];
            row_max[k] = m;
            row_log[k] = logf(s);
            kind[k] = !valid ? 0 : done ? 2 : s > 0.0f && m < __builtin_inff() ? 1 : 0;
        }
    }
    for (int i = t; i < kMaxChoices; i += kThreads) list[i] = 0;
    __syncthreads();
    const int per_beam = pieces * a.count;
    const int64_t all = (int64_t)a.beams * per_beam;
    for (int64_t first = 0; first < all; first += kThreads * E) {
        uint64_t key[E + 1];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            key[e] = 0;
            const int64_t i = first + e * kThreads + t;
            if (i < all) {
                const int k = (int)(i / per_beam), j = (int)(i - (int64_t)k * per_beam);
                uint32_t token = 0;
                float v = -__builtin_inff();
                if (kind[k] == 1) {
                    const uint64_t c = best[(int64_t)(b * a.beams + k) * per_beam + j];
                    token = ~(uint32_t)c;
                    if (c) v = score[k] + ((of_ordered((uint32_t)(c >> 32)) - row_max[k]) - row_log[k]);
                } else if (kind[k] == 2 && j == 0) {
                    token = (uint32_t)a.pad;
                    v = score[k];
                }
                if (v > -__builtin_inff())
                    key[e] = (uint64_t)ordered(v + 0.0f) << 32 | ~((uint32_t)k * (uint32_t)a.vocab + token);
            }
        }
        key[E] = t < kMaxChoices ? list[t] : 0;
        __syncthreads();
        choose<E + 1, 32>(chooser, a.count, [&](int e) { return key[e]; }, [&](int i, uint64_t k) { list[i] = k; });
        __syncthreads();
    }
    for (int i = t; i < a.count; i += kThreads) {
        const uint64_t c = list[i];
        const uint32_t at = ~(uint32_t)c;
        const uint32_t k = at / (uint32_t)a.vocab;
        const int64_t o = (int64_t)b * a.count + i;
        a.out_scores[o] = c ? of_ordered((uint32_t)(c >> 32)) : -__builtin_inff();
        a.out_parents[o] = c ? (int32_t)k : i % a.beams;
        a.out_tokens[o] = c ? (int32_t)(at - k * (uint32_t)a.vocab) : a.pad;
    }
}

// Logits of a piece for each of its 256 threads: as many as still give the device enough workgroups.
int piece_values(int64_t rows, int32_t vocab)
{
    int e = 64;
    while (e > 8 && rows * ((vocab + kThreads * e - 1) / (kThreads * e)) < 4 * compute_units()) e /= 2;
    return e;
}

int64_t piece_count(int32_t vocab, int e) { return ((int64_t)vocab + kThreads * e - 1) / (kThreads * e); }

template <int TYPE>
void launch_pieces(const SelectArgs &a, int e, int pieces, uint64_t *best, Piece *piece, hipStream_t stream)
{
    const int grid = a.batch * a.beams * pieces;
    const Divisor d = divisor((uint32_t)pieces);
    switch (e) {
        case 8: beam_pieces_kernel<TYPE, 8><<<grid, kThreads, 0, stream>>>(a, pieces, d, best, piece); break;
        case 16: beam_pieces_kernel<TYPE, 16><<<grid, kThreads, 0, stream>>>(a, pieces, d, best, piece); break;
        case 32: beam_pieces_kernel<TYPE, 32><<<grid, kThreads, 0, stream>>>(a, pieces, d, best, piece); break;
        default: beam_pieces_kernel<TYPE, 64><<<grid, kThreads, 0, stream>>>(a, pieces, d, best, piece); break;
    }
}

// ---- the caches ----

constexpr int kCaches = 32;  // of a launch
struct ReorderArgs {
    const int32_t *parents;
    int32_t batch, beams, n;
    int32_t first[kCaches];  // workgroup of a sequence with which a cache begins
    quamba_beam_cache_t cache[kCaches];
};

// A workgroup moves one slice of 4 KiB of every beam of a sequence: all loads stand before the stores, and no other thread
// touches the bytes, so the move is in place whatever the order of the beams.
template <int BEAMS>
__global__ __launch_bounds__(kThreads) void beam_reorder_kernel(ReorderArgs a)
{
    typedef uint32_t Vec __attribute__((ext_vector_type(4), aligned(1)));  // caches may lie at any address
    const int b = blockIdx.y;
    int c = 0;
    for (int i = 1; i < a.n; ++i) c += (int)blockIdx.x >= a.first[i];
    const int64_t bytes = a.cache[c].bytes, at = ((int64_t)((int)blockIdx.x - a.first[c]) * kThreads + threadIdx.x) * 16;
    if (at >= bytes) return;
    char *base = static_cast<char *>(a.cache[c].data) + (int64_t)b * a.beams * bytes + at;
    const int32_t *parents = a.parents + (int64_t)b * a.beams;
    int from[BEAMS];
#pragma unroll
    for (int k = 0; k < BEAMS; ++k) {
        const int p = k < a.beams ? parents[k] : k;
        from[k] = (uint32_t)p < (uint32_t)a.beams ? p : k;
    }
    if (at + 16 <= bytes) {
        Vec v[BEAMS];
#pragma unroll
        for (int k = 0; k < BEAMS; ++k)
            if (from[k] != k) v[k] = *reinterpret_cast<const Vec *>(base + from[k] * bytes);
#pragma unroll
        for (int k = 0; k < BEAMS; ++k)
            if (from[k] != k) *reinterpret_cast<Vec *>(base + k * bytes) = v[k];
    } else {  // the last bytes one by one, of all beams alike
#pragma unroll 1
        for (int i = 0; at + i < bytes; ++i) {
            char v[BEAMS];
#pragma unroll
            for (int k = 0; k < BEAMS; ++k)
                if (k < a.beams) v[k] = base[from[k] * bytes + i];
#pragma unroll
            for (int k = 0; k < BEAMS; ++k)
                if (k < a.beams) base[k * bytes + i] = v[k];
        }
    }
}

void launch_slices(const ReorderArgs &a, int slices, int sequences, hipStream_t stream)
{
    const dim3 grid(slices, sequences);
    if (a.beams <= 2)
        beam_reorder_kernel<2><<<grid, kThreads, 0, stream>>>(a);
    else if (a.beams <= 4)
        beam_reorder_kernel<4><<<grid, kThreads, 0, stream>>>(a);
    else if (a.beams <= 8)
        beam_reorder_kernel<8><<<grid, kThreads, 0, stream>>>(a);
    else if (a.beams <= 16)
        beam_reorder_kernel<16><<<grid, kThreads, 0, stream>>>(a);
    else if (a.beams <= 32)
        beam_reorder_kernel<32><<<grid, kThreads, 0, stream>>>(a);
    else
        beam_reorder_kernel<64><<<grid, kThreads, 0, stream>>>(a);
}

}  // namespace

bool beam_select_supports(int32_t batch, int32_t beams, int32_t vocab)
{
    const int64_t rows = (int64_t)batch * beams;
    return vocab <= 1 << 30 && rows * piece_count(vocab, piece_values(rows, vocab)) < (int64_t)1 << 24 && (int64_t)beams * vocab <= 0xffffffffLL;
}

size_t beam_select_workspace_bytes(int32_t batch, int32_t beams, int32_t vocab, int32_t count)
{
    const int64_t rows = (int64_t)batch * beams, pieces = rows * piece_count(vocab, piece_values(rows, vocab));
    return (size_t)pieces * (sizeof(uint64_t) * count + sizeof(Piece));
}

hipError_t launch_beam_select(const SelectArgs &a, void *workspace, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.batch * a.beams;
    const int e = piece_values(rows, a.vocab), pieces = (int)piece_count(a.vocab, e);
    uint64_t *best = static_cast<uint64_t *>(workspace);
    Piece *piece = reinterpret_cast<Piece *>(best + rows * pieces * a.count);
    switch (a.type) {
        case QUAMBA_F32: launch_pieces<QUAMBA_F32>(a, e, pieces, best, piece, stream); break;
        case QUAMBA_F16: launch_pieces<QUAMBA_F16>(a, e, pieces, best, piece, stream); break;
        default: launch_pieces<QUAMBA_BF16>(a, e, pieces, best, piece, stream); break;
    }
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    beam_join_kernel<<<a.batch, kThreads, 0, stream>>>(a, pieces, best, piece);
    return hipGetLastError();
}

hipError_t launch_beam_reorder(int32_t batch, int32_t beams, const int32_t *parents, int32_t n, const quamba_beam_cache_t *caches,
                               hipStream_t stream)
{
    // launches of up to kCaches caches, 2^22 slices (16 GiB of a beam, the longest cache) and 65535 sequences
    constexpr int64_t kSlice = kThreads * 16, kSlices = kMaxCacheBytes / kSlice;
    if (beams == 1) return hipSuccess;
    for (int32_t s0 = 0; s0 < batch; s0 += kMaxGridY) {
        const int sequences = std::min(batch - s0, kMaxGridY);
        ReorderArgs a;
        a.parents = parents + (int64_t)s0 * beams;
        a.batch = sequences;
        a.beams = beams;
        a.n = 0;
        int64_t slices = 0;
        auto flush = [&] {
            if (a.n) launch_slices(a, (int)slices, sequences, stream);
            a.n = 0;
            slices = 0;
            return hipGetLastError();
        };
        for (int32_t i = 0; i < n; ++i) {
            const int64_t need = (caches[i].bytes + kSlice - 1) / kSlice;
            if (!need) continue;
            if (a.n == kCaches || slices + need > kSlices) {
                const hipError_t e = flush();
                if (e != hipSuccess) return e;
            }
            a.first[a.n] = (int32_t)slices;
            a.cache[a.n].data = static_cast<char *>(caches[i].data) + (int64_t)s0 * beams * caches[i].bytes;
            a.cache[a.n].bytes = caches[i].bytes;
            ++a.n;
            slices += need;
        }
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace quamba
