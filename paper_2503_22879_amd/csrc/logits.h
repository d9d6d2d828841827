// What the kernels over rows of logits share: floats as whole numbers of the same order, 16 bytes of logits at a time, a row's running sum of
// exponentials, and a wave's best tokens.
#pragma once
#include "quamba_internal.h"

namespace quamba {
namespace {

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

// Sixteen bytes of logits.
template <int TYPE>
struct Logits {
    static constexpr int kBytes = TYPE == QUAMBA_F32 ? 4 : 2, kCount = 16 / kBytes;
    uint32_t w[4];
    __device__ __forceinline__ float operator[](int i) const
    {
        if (TYPE == QUAMBA_F32) return from_bits(w[i]);
        const uint32_t h = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
        return TYPE == QUAMBA_BF16 ? from_bits(h << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)h);
    }
    __device__ __forceinline__ void load(const char *p) { __builtin_memcpy(w, p, 16); }
    __device__ __forceinline__ void load(const char *p, int left)  // the first `left`, -infinity behind them
    {
        if (left >= kCount) {
            load(p);
            return;
        }
        load(p, 0, left);
    }
    __device__ __forceinline__ void load(const char *p, int from, int to)  // those from `from` to `to`, -infinity around them
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = TYPE == QUAMBA_F32 ? 0xff800000u : TYPE == QUAMBA_BF16 ? 0xff80ff80u : 0xfc00fc00u;
#pragma unroll
        for (int i = 0; i < kCount; ++i)
            if (i >= from && i < to) {
                if (kBytes == 4) {
                    __builtin_memcpy(&w[i], p + 4 * i, 4);
                } else {
                    uint16_t h;
                    __builtin_memcpy(&h, p + 2 * i, 2);
                    w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | (uint32_t)h << 16 : (w[i / 2] & 0xffff0000u) | h;
                }
            }
    }
};

// A row of logits as vectors of 16 bytes that lie at multiples of 16 bytes, whatever the row's address: vector j holds the logits from
// j * kCount - skip on; what the first and the last hold around the row reads as -infinity.
template <int TYPE>
struct Row {
    static constexpr int kCount = Logits<TYPE>::kCount, kBytes = Logits<TYPE>::kBytes;
    const char *base;  // of vector 0
    int skip, vocab, vectors;
    __device__ __forceinline__ Row(const void *logits, int64_t at, int vocab_) : vocab(vocab_)
    {
        const char *p = static_cast<const char *>(logits) + at * kBytes;
        skip = (int)(reinterpret_cast<uintptr_t>(p) & 15) / kBytes;
        base = p - skip * kBytes;
        vectors = (vocab + skip + kCount - 1) / kCount;
    }
    __device__ __forceinline__ int token(int j) const { return j * kCount - skip; }  // of vector j's first logit
    // vectors first .. last - 1 lie inside the row
    __device__ __forceinline__ bool whole(int first, int last) const { return (first > 0 || skip == 0) && last * kCount - skip <= vocab; }
    __device__ __forceinline__ void load(Logits<TYPE> &v, int j) const { v.load(base + (int64_t)j * 16); }
    __device__ __forceinline__ void load(Logits<TYPE> &v, int j, int last) const  // vector j of those before `last`
    {
        const int from = j == 0 ? skip : 0, to = j < last ? min(kCount, vocab - token(j)) : 0;
        if (from == 0 && to == kCount)
            load(v, j);
        else
            v.load(base + (int64_t)j * 16, from, to);
    }
    __device__ __forceinline__ float logit(int t) const
    {
        const char *p = base + ((int64_t)t + skip) * kBytes;
        if (TYPE == QUAMBA_F32) return *reinterpret_cast<const float *>(p);
        const uint16_t h = *reinterpret_cast<const uint16_t *>(p);
        return TYPE == QUAMBA_BF16 ? from_bits((uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
    }
};

// Vectors first .. last - 1 of a row by a workgroup of THREADS: each(v, j) for vector j, in every thread as often, with -infinity where
// there is none.  U vectors of a thread are on their way while the U before them are worked on.
template <int TYPE, int THREADS, int U, typename Each>
__device__ __forceinline__ void walk(const Row<TYPE> &row, int first, int last, const Each &each)
{
    constexpr int kStep = THREADS * U;
    const int t = threadIdx.x;
    auto fetch = [&](Logits<TYPE>(&v)[U], int from) {
        if (from + kStep <= last && row.whole(from, from + kStep)) {
#pragma unroll
            for (int u = 0; u < U; ++u) row.load(v[u], from + u * THREADS + t);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) row.load(v[u], from + u * THREADS + t, last);
        }
    };
    Logits<TYPE> v[U], next[U];
    if (first < last) fetch(v, first);
    for (int from = first; from < last; from += kStep) {
        if (from + kStep < last) fetch(next, from + kStep);
#pragma unroll
        for (int u = 0; u < U; ++u) each(v[u], from + u * THREADS + t);
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = next[u];
    }
}

// A sum of exponentials, of e = (x - reference) c and to the base 2, for c = log2(e) / temperature.  The reference is a logit that was among
// the largest when it was met: it is replaced only by one whose exponential would be above 2^8, so the sum is hardly ever rescaled, e
// stays as small as its rounding asks for, and what is lost beside the sum is below 2^-126.  (A difference first and then the factor: x c alone may leave fp32's range,
// and its rounding grows with x.)
struct ExpSum {
    float reference = -__FLT_MAX__;
    float sum = 0.0f;     // NaN where the logits hold a NaN or +infinity
    float second = 0.0f;  // of the same terms: times e (for an entropy), or without some of them
};
constexpr float kFarBelow = -200.0f;  // 2^-200 is 0, and 0 times this as well

__device__ __forceinline__ float exp2_of(float e) { return __builtin_amdgcn_exp2f(e); }

// The sum against another, larger reference.
template <bool ENTROPY>
__device__ __forceinline__ void rebase(ExpSum &s, float reference, float c)
{
    const float e = (s.reference - reference) * c, f = exp2_of(e);
    s.second = f * (ENTROPY ? fmaf(fmaxf(e, kFarBelow), s.sum, s.second) : s.second);
    s.sum *= f;
    s.reference = reference;
}

template <int TYPE>
__device__ __forceinline__ float largest(const Logits<TYPE> &v)
{
    float m = v[0];
#pragma unroll
    for (int i = 1; i < Logits<TYPE>::kCount; ++i) m = fmaxf(m, v[i]);
    return m;
}

// Takes a vector of logits whose largest is `top` into the sum.  SECOND: 0 none, 1 times e, 2 without the logits whose bit in
// `without` is set.
template <int SECOND, int TYPE>
__device__ __forceinline__ void add(ExpSum &s, const Logits<TYPE> &v, float top, float c, uint32_t without = 0)
{
    constexpr int N = Logits<TYPE>::kCount;
    if ((top - s.reference) * c > 8.0f) rebase<SECOND == 1>(s, top, c);
    float part = 0.0f, kept = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float e = (v[i] - s.reference) * c, p = exp2_of(e);
        part += p;
        if (SECOND == 1) s.second = fmaf(p, fmaxf(e, kFarBelow), s.second);
    }
    if (SECOND == 2) {
        kept = part;
        if (without) {
            kept = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) kept += without >> i & 1 ? 0.0f : exp2_of((v[i] - s.reference) * c);
        }
        s.second += kept;
    }
    s.sum += part;
}

// The sums of a workgroup's threads as one, in every thread.
template <bool ENTROPY, int THREADS>
__device__ __forceinline__ ExpSum join(ExpSum s, float c)
{
    constexpr int kWaves = THREADS / 64;
    __shared__ float wave[3][kWaves];
    const int w = threadIdx.x / 64;
    rebase<ENTROPY>(s, wave_max(s.reference), c);
    s.sum = group_sum<64>(s.sum);
    s.second = group_sum<64>(s.second);
    if (kWaves == 1) return s;
    __syncthreads();  // an earlier call's
    if (threadIdx.x % 64 == 0) {
        wave[0][w] = s.reference;
        wave[1][w] = s.sum;
        wave[2][w] = s.second;
    }
    __syncthreads();
    float top = wave[0][0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) top = fmaxf(top, wave[0][i]);
    ExpSum all;
    all.reference = top;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        ExpSum part;
        part.reference = wave[0][i];
        part.sum = wave[1][i];
        part.second = wave[2][i];
        rebase<ENTROPY>(part, top, c);
        all.sum += part.sum;
        all.second += part.second;
    }
    return all;
}

// ... of the segments of a row, which are in memory.
template <bool ENTROPY, int THREADS>
__device__ __forceinline__ ExpSum join(const LogitsPart *parts, int segments, float c)
{
    ExpSum s;
    for (int i = threadIdx.x; i < segments; i += THREADS) {
        ExpSum part;
        part.reference = parts[i].reference;
        part.sum = parts[i].sum;
        part.second = parts[i].second;
        const float top = fmaxf(s.reference, part.reference);
        rebase<ENTROPY>(s, top, c);
        rebase<ENTROPY>(part, top, c);
        s.sum += part.sum;
        s.second += part.second;
    }
    return join<ENTROPY, THREADS>(s, c);
}

// The best tokens that a wave has met, as keys: the ordered logit above, the complement of the token below, so that of equal logits the
// lower token is the larger key; -0 counts as 0.  Keys are gathered in LDS, and when little room is left the `count` largest are kept; from
// then on only logits above the least of them are looked at, so that few of a long row are.
constexpr int kListed = 256;
struct TopList {
    uint64_t *keys;  // of kListed, the wave's own
    int count, n;
    float bound;     // candidates are above
    __device__ __forceinline__ TopList(uint64_t *keys_, int count_) : keys(keys_), count(count_), n(0), bound(-__builtin_inff()) {}

    // Keeps the `count` largest of more.
    __device__ __forceinline__ void shrink()
    {
        const int lane = threadIdx.x & 63;
        uint64_t mine[kListed / 64];
#pragma unroll
        for (int i = 0; i < kListed / 64; ++i) mine[i] = i * 64 + lane < n ? keys[i * 64 + lane] : 0;
        auto reach = [&](uint64_t least) {
            int r = 0;
#pragma unroll
            for (int i = 0; i < kListed / 64; ++i) r += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[i] >= least));
            return r;
        };
        uint64_t least = 0;  // the largest number that `count` keys reach, or one that exactly so many do
        for (int bit = 63; bit >= 0; --bit) {
            const uint64_t higher = least | (uint64_t)1 << bit;
            const int r = reach(higher);
            if (r >= count) least = higher;
            if (r == count) break;
        }
        uint32_t low = 0xffffffffu;
        int at = 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < kListed / 64; ++i) {
            const bool kept = mine[i] >= least;
            const uint64_t those = __builtin_amdgcn_ballot_w64(kept);
            if (kept) {
                keys[at + __builtin_popcountll(those & (((uint64_t)1 << lane) - 1))] = mine[i];
                low = min(low, (uint32_t)(mine[i] >> 32));
            }
            at += __builtin_popcountll(those);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int d = 32; d; d >>= 1) low = min(low, (uint32_t)__shfl_xor((int)low, d, 64));
        n = at;
        bound = of_ordered(low);
    }

    // Candidates value(e) with their keys key(e), e < E, of which `top` is the lane's largest; called by the whole wave.  RISING: every later call's
    // tokens are above all of this one's, so equals of the least that is kept are no candidates there.
    template <int E, bool RISING, typename Value, typename Key>
    __device__ __forceinline__ void offer(float top, const Value &value, const Key &key)
    {
        if (!__builtin_amdgcn_ballot_w64(top > bound)) return;
        const int lane = threadIdx.x & 63;
        float above = bound;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float v = value(e);
            uint64_t those = __builtin_amdgcn_ballot_w64(v > above);
            if (!those) continue;
            if (n > kListed - 64) {
                shrink();
                above = of_ordered(ordered(bound) - (bound == 0.0f ? 2 : 1));  // the next below, which is not -0
                those = __builtin_amdgcn_ballot_w64(v > above);
            }
            if (v > above) keys[n + __builtin_popcountll(those & (((uint64_t)1 << lane) - 1))] = key(e);
            n += __builtin_popcountll(those);
        }
        if (!RISING && bound > -__builtin_inff()) bound = above;
    }
};
__device__ __forceinline__ uint64_t key_of(float logit, int token) { return (uint64_t)ordered(logit + 0.0f) << 32 | (uint32_t)~token; }

// ---- gradients ----

template <int TYPE>
__device__ __forceinline__ uint32_t bits_of(float v)
{
    return TYPE == QUAMBA_F32 ? __builtin_bit_cast(uint32_t, v) : TYPE == QUAMBA_F16 ? f32_to_f16_bits(v) : __builtin_bit_cast(uint16_t, (__bf16)v);
}

// A row of the gradient, cut into the vectors of its row of logits: it may lie elsewhere in 16 bytes.
template <int TYPE>
struct GradientRow {
    static constexpr int kCount = Logits<TYPE>::kCount, kBytes = Logits<TYPE>::kBytes;
    char *base;
    int skip, vocab;
    __device__ __forceinline__ GradientRow(void *gradient, int64_t at, const Row<TYPE> &x) : skip(x.skip), vocab(x.vocab)
    {
        base = static_cast<char *>(gradient) + (at - skip) * kBytes;
    }
    __device__ __forceinline__ void store(const float (&v)[kCount], int j) const
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = kBytes == 4 ? bits_of<TYPE>(v[i]) : bits_of<TYPE>(v[2 * i % kCount]) | bits_of<TYPE>(v[(2 * i + 1) % kCount]) << 16;
        __builtin_memcpy(base + (int64_t)j * 16, w, 16);
    }
    __device__ __forceinline__ void store_one(float v, int token) const
    {
        char *p = base + ((int64_t)token + skip) * kBytes;
        const uint32_t b = bits_of<TYPE>(v);
        if (kBytes == 4)
            *reinterpret_cast<uint32_t *>(p) = b;
        else
            *reinterpret_cast<uint16_t *>(p) = (uint16_t)b;
    }
    __device__ __forceinline__ void store(const float (&v)[kCount], int j, int last) const  // what of vector j, one of those before `last`, is the row's
    {
        const int token = j * kCount - skip;
        if (j >= last) return;
        if (token >= 0 && token + kCount <= vocab) {
            store(v, j);
            return;
        }
#pragma unroll
        for (int i = 0; i < kCount; ++i)
            if (token + i >= 0 && token + i < vocab) store_one(v[i], token + i);
    }
};

// gradient = p (flat + tilted log2 p) with p = 2^e, e = (x - reference) c - log, over vectors first .. last - 1 of a row.  The gradient may
// take the logits' place: a vector's values are read before they are written, by the same thread, and by no other.
template <int TYPE, int THREADS, int U, bool TILTED>
__device__ __forceinline__ void write_gradient(const Row<TYPE> &x, const GradientRow<TYPE> &to, int first, int last, float reference, float c,
                                               float log, float flat, float tilted)
{
    constexpr int N = Logits<TYPE>::kCount;
    walk<TYPE, THREADS, U>(x, first, last, [&](const Logits<TYPE> &v, int j) {
        float g[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float e = fmaf(v[i] - reference, c, -log), p = exp2_of(e);
            g[i] = p * (TILTED ? fmaf(tilted, fmaxf(e, kFarBelow), flat) : flat);
        }
        to.store(g, j, last);
    });
}

// The log sum of a row as the caller has it, in fp32, turned into a reference logit and what is left of it: (x - reference) c - log is
// log2 p up to the rounding of the difference.
struct Saved {
    float reference, log;
    __device__ __forceinline__ Saved(float log_sum, float temperature, float c)
    {
        reference = log_sum * temperature;
        log = fmaf(log_sum, temperature, -reference) * c;
    }
};

template <int TYPE, int THREADS>
__device__ __forceinline__ void write_zeros(const GradientRow<TYPE> &to, int first, int last)
{
    const float zero[Logits<TYPE>::kCount] = {};
    for (int j = first + threadIdx.x; j < last; j += THREADS) to.store(zero, j, last);
}

}  // namespace
}  // namespace quamba
