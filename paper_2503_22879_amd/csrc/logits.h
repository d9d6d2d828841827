// What the kernels over rows of logits share: floats as whole numbers of the same order, 16 bytes of logits at a time, a row's running sum of
// exponentials, and a wave's best tokens.
#pragma once
#include <type_traits>

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

// The largest of 16 lanes, and of a wave, mostly by moves between lanes that are part of an operation.
__device__ __forceinline__ float row_max(float v)
{
    v = fmaxf(v, dpp_move<0xB1>(v));  // the steps of group_sum
    v = fmaxf(v, dpp_move<0x4E>(v));
    v = fmaxf(v, dpp_move<0x141>(v));
    return fmaxf(v, dpp_move<0x140>(v));
}
__device__ __forceinline__ float group_max(float v)
{
    v = row_max(v);
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401F)));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

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
    __device__ __forceinline__ float at(int i) const  // of an i that is known at run time only: by selections, not from memory
    {
        const int word = i * kBytes / 4;
        uint32_t a = w[0], b = w[1], c = w[2], d = w[3];
        asm("" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));  // a choice between them, and not between their addresses
        Logits one;
        one.w[0] = word < 2 ? (word < 1 ? a : b) : (word < 3 ? c : d);
        return kBytes == 2 && i & 1 ? one[1] : one[0];
    }
    __device__ __forceinline__ void load(const char *p) { __builtin_memcpy(w, p, 16); }
    __device__ __forceinline__ void fill()  // with -infinity
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = TYPE == QUAMBA_F32 ? 0xff800000u : TYPE == QUAMBA_BF16 ? 0xff80ff80u : 0xfc00fc00u;
    }
    __device__ __forceinline__ void fill(uint32_t which)  // those whose bit is set
    {
        Logits none;
        none.fill();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const auto all = [&](int k) { return 0u - (which >> k & 1u); };
            const uint32_t mask = kBytes == 4 ? all(i) : (all(2 * i) & 0xffffu) | all(2 * i + 1) << 16;
            w[i] = (none.w[i] & mask) | (w[i] & ~mask);
        }
    }
    __device__ __forceinline__ void load(const char *p, int left)  // the first `left`, -infinity behind them
    {
        if (left >= kCount) {
            load(p);
            return;
        }
        fill();
#pragma unroll
        for (int i = 0; i < kCount; ++i)
            if (i < left) {
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

// A logit as it lies in memory.  Held wider, a 16-bit one would be waited for where it is widened.
template <int TYPE>
using LogitBits = std::conditional_t<TYPE == QUAMBA_F32, uint32_t, uint16_t>;

// A row of logits as vectors of 16 bytes that lie at multiples of 16 bytes, whatever the row's address: vector j holds the logits from
// j * kCount - skip on; what the first and the last hold around the row reads as -infinity.  PAST: the row is not to stay in the
// caches.
template <int TYPE, bool PAST = false>
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
    __device__ __forceinline__ void load(Logits<TYPE> &v, int j) const  // inside the row
    {
        const u32x4 *p = reinterpret_cast<const u32x4 *>(base + (uint32_t)j * 16u);
        const u32x4 w = PAST ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.w[i] = w[i];
    }
    // The bits of logit k of vector j.
    __device__ __forceinline__ uint32_t bits(int j, int k) const
    {
        const char *p = base + (uint32_t)j * 16u;
        return kBytes == 4 ? reinterpret_cast<const uint32_t *>(p)[k] : reinterpret_cast<const uint16_t *>(p)[k];
    }
    static __device__ __forceinline__ float value(uint32_t bits)
    {
        return TYPE == QUAMBA_F32 ? from_bits(bits) : TYPE == QUAMBA_BF16 ? from_bits(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    }
    __device__ __forceinline__ float logit(int t) const { return value(bits(0, t + skip)); }
};

// What of vectors first .. last - 1 lies inside the row, and whether its first or last vector, across the row's ends, are among them.
struct Span {
    int begin, end;  // inside
    int whole;       // the row's last vector, or the one behind it
    bool head, tail;
    Span() = default;
    template <typename Row>
    __device__ __forceinline__ Span(const Row &row, int first, int last)
    {
        head = first == 0 && row.skip > 0;
        whole = (row.vocab + row.skip) / Row::kCount;
        begin = head ? 1 : first;
        end = min(last, whole);
        tail = first < last && last > whole && (whole > 0 || !head);
    }
    __device__ __forceinline__ bool has_ends() const { return head || tail; }
};

// What of a span lies in vectors across the row's ends, in a wave: the head's logits in the first kCount lanes, the tail's in the next, one to a lane, so that
// all are one load.
template <int TYPE>
struct Ends {
    LogitBits<TYPE> bits;
    int token;  // -1: the lane has none
    template <bool PAST>
    __device__ __forceinline__ void load(const Row<TYPE, PAST> &row, const Span &span)
    {
        token = token_of(row, span);
        bits = row.bits(0, row.skip + max(token, 0));
    }
    template <typename Row>
    static __device__ __forceinline__ int token_of(const Row &row, const Span &span)
    {
        constexpr int N = Logits<TYPE>::kCount;
        const int t = threadIdx.x, token = (t < N ? t : span.whole * N + t - N) - row.skip;
        return (t < N ? span.head : t < 2 * N && span.tail) && token >= 0 && token < row.vocab ? token : -1;
    }
    // The lane's logit, and -infinity behind it.
    __device__ __forceinline__ Logits<TYPE> vector() const
    {
        Logits<TYPE> v;
        v.fill();
        if (token >= 0) v.w[0] = Logits<TYPE>::kBytes == 4 ? bits : (v.w[0] & 0xffff0000u) | bits;
        return v;
    }
};

// Vectors first .. last - 1 of a row by a workgroup of THREADS: each(v, j, u) for those that lie inside the row, the vectors of a thread in
// rising order, u = 0 .. U - 1 in turn; in every thread of a wave as often, with -infinity where there is none.  At last end(v, token) for the first and last logits that
// no such vector has, in the first wave, if there are some (Ends; token -1 in lanes that have none); asked for first, they bring single rows nothing and cost
// many (2048 of 50021 bf16 logits 34.4 and 35.2 us).
//
// U loads of a thread are on their way together, and what follows them waits for one after the other; there is no branch between a load
// and its use, since behind one the compiler waits for all loads.  The next U are not asked for ahead: with 8 waves to a SIMD the other
// waves' work is as long as the memory takes.
template <int THREADS, int U, int TYPE, bool PAST, typename Each, typename End>
__device__ __forceinline__ void walk(const Row<TYPE, PAST> &row, int first, int last, const Each &each, const End &end)
{
    constexpr int kStep = THREADS * U;
    const int t = threadIdx.x;
    const Span span(row, first, last);
    int from = span.begin;
    for (; from + kStep <= span.end; from += kStep) {
        Logits<TYPE> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) row.load(v[u], from + u * THREADS + t);
#pragma unroll
        for (int u = 0; u < U; ++u) each(v[u], from + u * THREADS + t, u);
    }
    if (from < span.end) {
        Logits<TYPE> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) row.load(v[u], min(from + u * THREADS + t, span.end - 1));
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (from + u * THREADS < span.end) {
                if (from + u * THREADS + t >= span.end) v[u].fill();
                each(v[u], from + u * THREADS + t, u);
            }
    }
    if (t < 64 && span.has_ends()) {
        Ends<TYPE> ends;
        ends.load(row, span);
        end(ends.vector(), ends.token);
    }
}

// A sum of exponentials 2^e, e = (x - reference) c with c = log2(e) / temperature.  The reference is a logit that was among the largest when
// it was met: it is replaced only where an exponential would be above some 2^8, so the sum is hardly ever rescaled, e stays as small
// as its rounding asks for, and what is lost beside the sum is below 2^-126.
struct ExpSum {
    float reference = -__FLT_MAX__;
    float sum = 0.0f;     // NaN where the logits hold a NaN or +infinity
    float second = 0.0f;  // of the same terms: times e (for an entropy), or without some of them
};
constexpr float kFarBelow = -200.0f;  // 2^-200 is 0, and 0 times this as well

// Products x c below this round to within half a unit, so that 2^ of what the rounding leaves is a factor of at most 2^0.5.  From 2^31 on (a finite mask
// of -10^10, a temperature of 10^-8) it passes 2^127, and a sum of 0 times that is no number.
constexpr float kLargestOffset = 0x1p24f;

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

// A thread's sum while it grows.  SECOND: 0 none, 1 times e, 2 without the logits that are marked.  Mostly e is made by one operation, x c -
// offset with offset = reference c: the product is not rounded, and what the offset's rounding leaves is the same for all terms, so it
// is taken out at the end.  A vector for which the reference is too low (its sum shows it, so no largest logit is sought) and all where
// reference c is no longer a small step of fp32 from its product are made from the difference.
template <int SECOND>
struct Adder {
    ExpSum s;
    float c, offset = -__builtin_inff();  // -infinity: there is none
    __device__ __forceinline__ explicit Adder(float c_) : c(c_) {}

    __device__ __forceinline__ float residue() const { return offset > -__builtin_inff() ? fmaf(s.reference, c, -offset) : 0.0f; }
    // e without the offset's residue, or with it
    __device__ __forceinline__ void shift(float by)
    {
        const float f = exp2_of(by);
        s.second = f * (SECOND == 1 ? fmaf(by, s.sum, s.second) : s.second);
        s.sum *= f;
    }
    __device__ __forceinline__ ExpSum result()
    {
        shift(-residue());
        offset = -__builtin_inff();
        return s;
    }
    template <int TYPE>
    __device__ __forceinline__ void add(const Logits<TYPE> &v, uint32_t marked = 0)
    {
        constexpr int N = Logits<TYPE>::kCount;
        float p[N], part = 0.0f, weighted = s.second;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float e = fmaf(v[i], c, -offset);
            p[i] = exp2_of(e);
            part += p[i];
            if (SECOND == 1) weighted = fmaf(p[i], fmaxf(e, kFarBelow), weighted);
        }
        if (!(part <= 256.0f * N)) {
            const float top = largest(v);
            if ((top - s.reference) * c > 8.0f) {
                result();
                rebase<SECOND == 1>(s, top, c);
                if (__builtin_fabsf(top * c) < kLargestOffset) offset = top * c;
                shift(residue());
            }
            const float r = residue();
            part = 0.0f;
            weighted = s.second;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float e = fmaf(v[i] - s.reference, c, r);
                p[i] = exp2_of(e);
                part += p[i];
                if (SECOND == 1) weighted = fmaf(p[i], fmaxf(e, kFarBelow), weighted);
            }
        }
        s.sum += part;
        if (SECOND == 1) s.second = weighted;
        if (SECOND == 2) {
            if (marked) {
                part = 0.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) part += marked >> i & 1 ? 0.0f : p[i];
            }
            s.second += part;
        }
    }
};

__device__ __forceinline__ float first_lane(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// The sums of a wave's lanes as one, in every lane; LANES: of each 16 lanes, which all hold the same, or of 64.  Lane 0's: a product of rebase and
// the sum behind it may be one operation, and then the lanes' sums differ in their last bit, so that what a thread makes of them would hang
// on which thread makes it.
template <bool ENTROPY, int LANES>
__device__ __forceinline__ ExpSum join_lanes(ExpSum s, float c)
{
    rebase<ENTROPY>(s, LANES == 64 ? group_max(s.reference) : row_max(s.reference), c);
    s.reference = first_lane(s.reference);
    s.sum = first_lane(group_sum<LANES>(s.sum));
    s.second = first_lane(group_sum<LANES>(s.second));
    return s;
}

// The sums of a workgroup's threads as one, in every thread: of the waves', a wave's in a lane of 16.
template <bool ENTROPY, int THREADS>
__device__ __forceinline__ ExpSum join(ExpSum s, float c)
{
    constexpr int kWaves = THREADS / 64;
    static_assert(kWaves <= 16, "a wave to a lane");
    __shared__ float wave[3][16];
    s = join_lanes<ENTROPY, 64>(s, c);
    if (kWaves == 1) return s;
    __syncthreads();  // an earlier call's
    if (threadIdx.x % 64 == 0) {
        wave[0][threadIdx.x / 64] = s.reference;
        wave[1][threadIdx.x / 64] = s.sum;
        wave[2][threadIdx.x / 64] = s.second;
    }
    __syncthreads();
    const int lane = threadIdx.x & 15;
    ExpSum of_wave;
    if (lane < kWaves) {
        of_wave.reference = wave[0][lane];
        of_wave.sum = wave[1][lane];
        of_wave.second = wave[2][lane];
    }
    return join_lanes<ENTROPY, 16>(of_wave, c);
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

// The best tokens that a workgroup has met, as keys: the ordered logit above, the complement of the token below, so that of equal logits the
// lower token is the larger key; -0 counts as 0.  Every wave gathers keys in LDS, and when little room is left it keeps its `count` largest.
// Only logits above a bound are looked at, which at least `count` logits reach: first as many lanes' largest of one vector, then the least
// that is kept; the waves know the highest of their bounds.  So few of a long row are gathered.
constexpr int kListed = 256;  // keys of a wave
constexpr int kTurns = 4;     // of a walk that the best tokens are sought after
template <int WAVES>
struct TopKeys {  // in LDS
    uint64_t keys[WAVES][kListed];
    uint64_t all[WAVES * kMaxChoices];
    uint32_t bound;  // ordered; some keys of a wave that has set it are above, `count` of them
    int n, groups;
    uint32_t tops[WAVES > 1 ? 256 : 1];
    uint16_t group[WAVES * 64 * kTurns];
};
__device__ __forceinline__ float next_below(float v) { return of_ordered(ordered(v + 0.0f) - (v == 0.0f ? 2 : 1)); }  // below 0 is not -0

template <int WAVES>
struct TopList {
    TopKeys<WAVES> &shared;
    uint64_t *keys;  // the wave's own
    int count, n = 0;
    float bound = -__builtin_inff();  // candidates are above

    // The workgroup waits before it offers.
    __device__ __forceinline__ TopList(TopKeys<WAVES> &shared_, int count_) : shared(shared_), keys(shared_.keys[threadIdx.x / 64]), count(count_)
    {
        if (threadIdx.x == 0) {
            shared.bound = 0;
            shared.n = 0;
        }
    }

    // Keeps the `count` largest of more.
    __device__ __forceinline__ void shrink()
    {
        const int lane = threadIdx.x & 63;
        uint64_t mine[kListed / 64];
#pragma unroll
        for (int i = 0; i < kListed / 64; ++i) mine[i] = i * 64 + lane < n ? keys[i * 64 + lane] : 0;
        uint64_t least = 0;  // a number that `count` keys reach: the largest, or one that exactly so many do
        uint32_t high = 0;   // first among the upper halves
        bool exact = false;
        for (int bit = 31; bit >= 0 && !exact; --bit) {
            const uint32_t higher = high | 1u << bit;
            int r = 0;
#pragma unroll
            for (int i = 0; i < kListed / 64; ++i) r += __builtin_popcountll(__builtin_amdgcn_ballot_w64((uint32_t)(mine[i] >> 32) >= higher));
            if (r >= count) high = higher;
            exact = r == count;
        }
        least = (uint64_t)high << 32;
        for (int bit = 31; bit >= 0 && !exact; --bit) {
            const uint64_t higher = least | (uint64_t)1 << bit;
            int r = 0;
#pragma unroll
            for (int i = 0; i < kListed / 64; ++i) r += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[i] >= higher));
            if (r >= count) least = higher;
            exact = r == count;
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
        tell(next_below(bound));
    }

    // `count` keys of this wave are above this.
    __device__ __forceinline__ void tell(float b)
    {
        if (WAVES > 1 && (threadIdx.x & 63) == 0) atomicMax(&shared.bound, ordered(b));
    }

    // Candidates value(e) with their keys key(e), e < E, of which `top` is the lane's largest; called by the whole wave.  RISING: the tokens are above
    // all that were offered before, so equals of the least that is kept are no candidates.
    template <int E, bool RISING, typename Value, typename Key>
    __device__ __forceinline__ void offer(float top, const Value &value, const Key &key)
    {
        if (!RISING && bound > -__builtin_inff()) bound = next_below(bound);
        if (__builtin_expect(!__builtin_amdgcn_ballot_w64(top > bound), 1)) return;
        const int lane = threadIdx.x & 63;
        if (WAVES > 1) {
            const uint32_t b = __builtin_amdgcn_readfirstlane(*(volatile uint32_t *)&shared.bound);
            if (b) bound = fmaxf(bound, of_ordered(b));
        }
        if (n < count && count <= 64) {
            const uint32_t mine = top > -__builtin_inff() ? ordered(top + 0.0f) : 0u;
            uint32_t reached = 0;  // by `count` lanes
#pragma unroll
            for (int bit = 31; bit >= 16; --bit) {
                const uint32_t higher = reached | 1u << bit;
                if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(mine >= higher)) >= count) reached = higher;
            }
            if (reached > ordered(-__FLT_MAX__)) {
                const float b = next_below(of_ordered(reached));
                if (b > bound) {
                    bound = b;
                    tell(b);
                }
            }
        }
        float above = bound;
#pragma unroll 1
        for (int e = 0; e < E; ++e) {
            const float v = value(e);
            uint64_t those = __builtin_amdgcn_ballot_w64(v > above);
            if (!those) continue;
            if (n > kListed - 64) {
                shrink();
                above = next_below(bound);
                those = __builtin_amdgcn_ballot_w64(v > above);
            }
            if (v > above) keys[n + __builtin_popcountll(those & (((uint64_t)1 << lane) - 1))] = key(e);
            n += __builtin_popcountll(those);
        }
    }

    // The workgroup's best: out(i, key) for the i-th largest, i < count, 0 where there are no more.
    template <typename Out>
    __device__ __forceinline__ void ranked(const Out &out)
    {
        const int lane = threadIdx.x & 63;
        if (n > (count < 64 ? 64 : count)) shrink();
        __syncthreads();
        const uint32_t least = shared.bound;
        for (int i = 0; i < n; i += 64) {  // what may be among the best of all waves, one behind the other
            const uint64_t key = i + lane < n ? keys[i + lane] : 0;
            const bool is = (uint32_t)(key >> 32) > least;
            const uint64_t those = __builtin_amdgcn_ballot_w64(is);
            int at = 0;
            if (lane == 0 && those) at = atomicAdd(&shared.n, __builtin_popcountll(those));
            at = __builtin_amdgcn_readfirstlane(at);
            if (is) shared.all[at + __builtin_popcountll(those & (((uint64_t)1 << lane) - 1))] = key;
        }
        __syncthreads();
        const int all = shared.n;
        for (int i = threadIdx.x; i < all; i += WAVES * 64) {
            const uint64_t key = shared.all[i];
            int rank = 0;
#pragma unroll 4
            for (int k = 0; k < all; ++k) rank += shared.all[k] > key;
            if (rank < count) out(rank, key);
        }
        for (int i = all + threadIdx.x; i < count; i += WAVES * 64) out(i, (uint64_t)0);
    }
};
__device__ __forceinline__ uint64_t key_of(float logit, int token) { return (uint64_t)ordered(logit + 0.0f) << 32 | (uint32_t)~token; }

// The best tokens of vectors first .. last - 1 of a row that have been walked through: out(i, key) for the i-th largest, i < count, 0 where there
// are no more.  tops[u] is the thread's largest logit among the vectors of its turns u.
//
// `count` of 256 threads, fours of threads or turns of a lane have a logit at least as large as the count-th largest of their own largest ones, so nothing
// below that is among the best, and little more than `count` logits are above: the turns that hold one are read again, from the caches,
// and what reaches the bound is ranked by counting.  A list that is kept up to date while the row goes by was slower: of some 250 vectors of a
// wave a tenth to a half brought a better token, for ten times the work of one that did not.  Where so many logits are equal that those at
// the bound do not fit, such lists are made after all.
template <int THREADS, int U, int TYPE, bool PAST, typename Out>
__device__ __forceinline__ void best_tokens(TopKeys<THREADS / 64> &shared, const Row<TYPE, PAST> &row, int first, int last, const float (&tops)[U],
                                            int count, const Out &out)
{
    constexpr int WAVES = THREADS / 64, N = Logits<TYPE>::kCount, kStep = THREADS * U, kRoom = WAVES * kListed, kShare = THREADS > 256 ? THREADS / 256 : 1;
    const int t = threadIdx.x, lane = t & 63;
    const Span span(row, first, last);
    Ends<TYPE> ends;
    if (t < 64 && span.has_ends()) ends.load(row, span);
    float top = tops[0];
#pragma unroll
    for (int u = 1; u < U; ++u) top = fmaxf(top, tops[u]);
    static_assert(THREADS == 64 || THREADS == 256 || THREADS == 1024, "256 largest logits: of a lane's turns, of a thread, of a quad");
    static_assert(U == 4, "turns of a lane");
    uint32_t mine[4], bound = 0;
    if (t == 0) shared.n = shared.groups = 0;
    if (THREADS == 64) {
#pragma unroll
        for (int u = 0; u < U; ++u) mine[u] = tops[u] > -__builtin_inff() ? ordered(tops[u] + 0.0f) : 0u;
        __syncthreads();
    } else {
        if (kShare == 4) {
            top = fmaxf(top, dpp_move<0xB1>(top));
            top = fmaxf(top, dpp_move<0x4E>(top));
        }
        if (t % kShare == 0) shared.tops[t / kShare] = top > -__builtin_inff() ? ordered(top + 0.0f) : 0u;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) mine[w] = shared.tops[w * 64 + lane];
    }
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t higher = bound | 1u << bit;
        int n = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[w] >= higher));
        bound = n >= count ? higher : bound;
    }
    const float least = fmaxf(of_ordered(max(bound, 1u)), -__FLT_MAX__);
    auto take = [&](const Logits<TYPE> &v, int token) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (v[e] >= least) {
                const int at = atomicAdd(&shared.n, 1);
                if (at < kRoom) shared.keys[at / kListed][at % kListed] = key_of(v[e], token + e);
            }
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (tops[u] >= least) shared.group[atomicAdd(&shared.groups, 1)] = (uint16_t)(u * THREADS + t);
    __syncthreads();
    const int steps = (span.end - span.begin + kStep - 1) / kStep, items = shared.groups * steps;
    for (int i = t; i < items; i += THREADS) {
        const int g = i / steps, j = span.begin + (i - g * steps) * kStep + shared.group[g];
        if (j < span.end) {
            Logits<TYPE> v;
            row.load(v, j);
            take(v, row.token(j));
        }
    }
    if (t < 64 && span.has_ends()) take(ends.vector(), ends.token);
    __syncthreads();
    const int n = shared.n;
    __syncthreads();  // all know it
    if (n > kRoom) {
        TopList<WAVES> list(shared, count);
        __syncthreads();
        walk<THREADS, 1>(
            row, first, last,
            [&](const Logits<TYPE> &v, int j, int) {
                list.template offer<N, true>(largest(v), [&](int e) { return v.at(e); }, [&](int e) { return key_of(v.at(e), row.token(j) + e); });
            },
            [&](const Logits<TYPE> &v, int token) {
                list.template offer<1, false>(v[0], [&](int) { return v[0]; }, [&](int) { return key_of(v[0], token); });
            });
        list.ranked(out);
        return;
    }
    for (int i = t; i < n; i += THREADS) {
        const uint64_t key = shared.keys[i / kListed][i % kListed];
        int rank = 0;
#pragma unroll 4
        for (int k = 0; k < n; ++k) rank += shared.keys[k / kListed][k % kListed] > key;
        if (rank < count) out(rank, key);
    }
    for (int i = n + t; i < count; i += THREADS) out(i, (uint64_t)0);
}

// ---- gradients ----

template <int TYPE>
__device__ __forceinline__ uint32_t bits_of(float v)
{
    return TYPE == QUAMBA_F32 ? __builtin_bit_cast(uint32_t, v) : TYPE == QUAMBA_F16 ? f32_to_f16_bits(v) : __builtin_bit_cast(uint16_t, (__bf16)v);
}

template <int TYPE>
__device__ __forceinline__ uint32_t pair_of(float low, float high)
{
    typedef float Floats __attribute__((ext_vector_type(2)));
    typedef __bf16 Brain __attribute__((ext_vector_type(2)));
    typedef _Float16 Half __attribute__((ext_vector_type(2)));
    const Floats v = {low, high};
    return TYPE == QUAMBA_BF16 ? __builtin_bit_cast(uint32_t, __builtin_convertvector(v, Brain)) : __builtin_bit_cast(uint32_t, __builtin_convertvector(v, Half));
}

// A row of the gradient, cut into the vectors of its row of logits: it may lie elsewhere in 16 bytes.
template <int TYPE, bool PAST = false>
struct GradientRow {
    static constexpr int kCount = Logits<TYPE>::kCount, kBytes = Logits<TYPE>::kBytes;
    char *base;
    int skip, vocab;
    __device__ __forceinline__ GradientRow(void *gradient, int64_t at, const Row<TYPE, PAST> &x) : skip(x.skip), vocab(x.vocab)
    {
        base = static_cast<char *>(gradient) + (at - skip) * kBytes;
    }
    __device__ __forceinline__ void store(const float (&v)[kCount], int j) const
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = kBytes == 4 ? bits_of<TYPE>(v[i]) : pair_of<TYPE>(v[2 * i % kCount], v[(2 * i + 1) % kCount]);
        typedef uint32_t Vec __attribute__((ext_vector_type(4), aligned(2)));  // at the type's alignment
        const Vec q = {w[0], w[1], w[2], w[3]};
        Vec *p = reinterpret_cast<Vec *>(base + (uint32_t)j * 16u);
        if (PAST)
            __builtin_nontemporal_store(q, p);
        else
            *p = q;
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
};

// Up to THREADS * VECTORS vectors of a row in a workgroup's registers.  All are asked for together and without a branch between them (behind one
// the compiler waits for all): where there are fewer, the last again; there is one.
template <int THREADS, int VECTORS, int TYPE>
struct Held {
    Logits<TYPE> v[VECTORS];
    template <bool PAST>
    __device__ __forceinline__ void load(const Row<TYPE, PAST> &x, const Span &span)
    {
#pragma unroll
        for (int u = 0; u < VECTORS; ++u) x.load(v[u], min(span.begin + u * THREADS + (int)threadIdx.x, span.end - 1));
    }
    // each(v, j, u) in turn; j may be span.end and above in some lanes
    template <typename Each>
    __device__ __forceinline__ void go_through(const Span &span, const Each &each)
    {
#pragma unroll
        for (int u = 0; u < VECTORS; ++u)
            if (span.begin + u * THREADS < span.end) each(v[u], span.begin + u * THREADS + (int)threadIdx.x, u);
    }
};

// A segment of a row's gradient: make(v, token, g) is that of the logits v from `token` on.  It may take the logits' place: a vector's values are read before they are
// written, by the same thread, and by no other.
template <int THREADS, int VECTORS, int TYPE, bool PAST>
struct GradientSegment {
    const Row<TYPE, PAST> &x;
    const GradientRow<TYPE, PAST> &to;
    const Span span;
    Held<THREADS, VECTORS, TYPE> held;
    Ends<TYPE> ends;
    __device__ __forceinline__ GradientSegment(const Row<TYPE, PAST> &x_, const GradientRow<TYPE, PAST> &to_, int first, int last)
        : x(x_), to(to_), span(x_, first, last)
    {
    }
    __device__ __forceinline__ void load()
    {
        if (threadIdx.x < 64 && span.has_ends()) ends.load(x, span);
        if (span.begin < span.end) held.load(x, span);
    }
    template <typename Make>
    __device__ __forceinline__ void write(const Make &make)
    {
        held.go_through(span, [&](const Logits<TYPE> &v, int j, int) {
            float g[Logits<TYPE>::kCount];
            make(v, x.token(j), g);
            if (j < span.end) to.store(g, j);
        });
        if (threadIdx.x < 64 && span.has_ends()) {
            float g[Logits<TYPE>::kCount];
            make(ends.vector(), ends.token, g);
            if (ends.token >= 0) to.store_one(g[0], ends.token);
        }
    }
};

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

template <int THREADS, int TYPE, bool PAST>
__device__ __forceinline__ void write_zeros(const Row<TYPE, PAST> &x, const GradientRow<TYPE, PAST> &to, int first, int last)
{
    const float zero[Logits<TYPE>::kCount] = {};
    const Span span(x, first, last);
    for (int j = span.begin + threadIdx.x; j < span.end; j += THREADS) to.store(zero, j);
    const int token = Ends<TYPE>::token_of(x, span);
    if (token >= 0) to.store_one(0.0f, token);
}

}  // namespace
}  // namespace quamba
