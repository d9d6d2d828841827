// The distance of rows of logits x, at a temperature T, from a teacher that is known by its most likely tokens, and its gradient.
//
//   loss = sum_k q_k (ln q_k - ln p[token_k])  + q_R (ln q_R - ln p_R),      p = softmax(x / T),  p_R = sum of p over the other tokens
//   dx_v = w / T (p_v Q - sum of the q_k with token_k = v),  Q = sum_k q_k + q_R;    of other tokens w / T (p_v / p_R) (Q p_R - q_R)
//
// One pass over a row makes its sum of exponentials and the other tokens' (whose own sum is exact where it is a small part of the row's: a
// difference would not be); the gradient is written as if no token were the teacher's, but for those, which come from their logits and
// places.  Bound: HBM (bf16: 2048 rows of 128000 logits, 64 places and a rest, 80 us, 6.1 TB/s; with the gradient, 4096 rows, 403 us, 5.1 TB/s of what has to
// be read and written once; the gradient alone of 1000 of 50021, 20 places, 36 us, 5.4 TB/s).
#include <algorithm>

#include "logits.h"

namespace quamba {
namespace {

constexpr int kThreads = 256;  // but where a row is held in registers
constexpr int64_t kRowsOfALaunch = (int64_t)1 << 22;
constexpr int kGradientVectors = 3;  // of a thread, of the gradient alone
constexpr float kLog2e = 1.44269504088896341f;

// The teacher's places of a row, two to a lane; every wave reads them for itself, so none waits for another.
struct Places {
    float q[2], log_q[2];
    int token[2];  // -1: an empty place
    float sum;     // of q
    bool any;      // whether there is a place that is not empty

    Places() = default;
    __device__ __forceinline__ Places(const DistillArgs &a, int64_t row) : Places(a, Raw(a, row)) {}

    // As they lie in memory.  Loads return in order: what a wave asks for before its logits does not wait for them.
    struct Raw {
        float value[2];
        int token[2];
        __device__ __forceinline__ Raw(const DistillArgs &a, int64_t row)
        {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = (threadIdx.x & 63) + 64 * h;
                value[h] = -__builtin_inff();
                token[h] = -1;
                if (k < a.places) {
                    value[h] = a.teacher[row * a.places + k];
                    token[h] = a.tokens[row * a.places + k];
                }
            }
        }
    };
    __device__ __forceinline__ Places(const DistillArgs &a, const Raw &raw)
    {
        float value[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            value[h] = raw.value[h];
            token[h] = raw.token[h];
            if ((uint32_t)token[h] >= (uint32_t)a.vocab || value[h] == -__builtin_inff()) {
                token[h] = -1;
                value[h] = -__builtin_inff();
            }
        }
        any = __builtin_amdgcn_ballot_w64(token[0] >= 0 || token[1] >= 0) != 0;
        const float top = a.rest ? 0.0f : group_max(fmaxf(value[0], value[1])), scale = a.rest ? 1.0f : a.per_temperature;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            log_q[h] = (value[h] - top) * scale;
            q[h] = token[h] >= 0 ? expf(log_q[h]) : 0.0f;
        }
        sum = group_sum<64>(q[0] + q[1]);
        if (!a.rest) {  // to sum to 1
            const float log = logf(sum);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                log_q[h] -= log;
                q[h] /= sum;
            }
            sum = group_sum<64>(q[0] + q[1]);
        }
    }
    // Whether place h of the lane has a token in these vectors.
    template <int TYPE>
    __device__ __forceinline__ bool is_in(int h, int skip, int first, int last) const
    {
        const int at = token[h] + skip;
        return token[h] >= 0 && at >= first * Logits<TYPE>::kCount && at < last * Logits<TYPE>::kCount;
    }
    // The sum of q over all places with the token of place h of the lane, which may have several, and whether that place is its first.  By the
    // whole wave.  Places are compared with one another only where two tokens have the same low bits: for each place that is some 10 operations of a
    // wave, which took longer than all else in short rows (4096 rows of 2000, 64 places: 15.4 us, 12.4 without).
    struct Seen {
        static constexpr int kBits = 1 << 15;
        uint32_t words[kBits / 32];
    };
    __device__ __forceinline__ void of_tokens(Seen &seen, int places, float (&all)[2], bool (&first)[2]) const
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < Seen::kBits / 32; i += 64) seen.words[i + lane] = 0;
        bool twice = false;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (token[h] >= 0) {
                const uint32_t at = (uint32_t)token[h] % Seen::kBits;
                twice = twice || (atomicOr(&seen.words[at / 32], 1u << at % 32) >> at % 32 & 1);
            }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            all[h] = q[h];
            first[h] = true;
        }
        if (__builtin_amdgcn_ballot_w64(twice) == 0) return;
        all[0] = all[1] = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            for (int i = 0; i < 64 && 64 * h + i < places; i += 8) {  // eight at a time: a lane's value is a while on its way to all
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int t = __builtin_amdgcn_readlane(token[h], i + j);
                    const float p = from_bits(__builtin_amdgcn_readlane(__builtin_bit_cast(int, q[h]), i + j));
                    all[0] += token[0] == t ? p : 0.0f;
                    all[1] += token[1] == t ? p : 0.0f;
                    first[0] = first[0] && (token[0] != t || 64 * h + i + j >= lane);
                    first[1] = first[1] && (token[1] != t || 64 * h + i + j >= lane + 64);
                }
            }
    }
};

// What the gradient of a row is made from: that of other tokens is flat 2^((x - reference) c - log), that of the teacher's comes from p and q.
struct Slope {
    float reference, log, flat;
    float offset, times;  // 16-bit logits: the same as times 2^(x c - offset), whose rounding is far below the result's; offset +infinity: times may leave fp32's range
    float own_reference, own_log, whole, scale;
    template <int TYPE>
    __device__ __forceinline__ void of_others(const Logits<TYPE> &x, float c, float (&g)[Logits<TYPE>::kCount]) const
    {
        if (TYPE != QUAMBA_F32 && offset != __builtin_inff()) {
#pragma unroll
            for (int i = 0; i < Logits<TYPE>::kCount; ++i) g[i] = exp2_of(fmaf(x[i], c, -offset)) * times;
        } else {
#pragma unroll
            for (int i = 0; i < Logits<TYPE>::kCount; ++i) g[i] = exp2_of(fmaf(x[i] - reference, c, -log)) * flat;
        }
    }
    __device__ __forceinline__ float of_token(float x, float q, float c) const
    {
        return (exp2_of(fmaf(x - own_reference, c, -own_log)) * whole - q) * scale;
    }
};

__device__ __forceinline__ Slope slope_of(const DistillArgs &a, float weight, float reference, float log_sum, float rest_reference, float log_rest,
                                          float share, bool rest, float sum_q)
{
    Slope s;
    const float left = rest ? fmaxf(1.0f - sum_q, 0.0f) : 0.0f;
    s.own_reference = reference;
    s.own_log = log_sum;
    s.whole = sum_q + left;
    s.scale = weight * a.per_temperature;
    s.reference = rest ? rest_reference : reference;
    s.log = rest ? log_rest : log_sum;
    s.flat = (rest ? fmaf(s.whole, share, -left) : s.whole) * s.scale;
    const float offset = fmaf(s.reference, a.c, s.log);
    s.times = s.flat * exp2_of(-(fmaf(s.reference, a.c, -offset) + s.log));
    s.offset = __builtin_fabsf(offset) < kLargestOffset || offset != offset ? offset : __builtin_inff();
    return s;
}

// A row's sums of exponentials, over all tokens and over those without a place, each against a reference logit of its own.
struct RowSums {
    float reference, sum;  // NaN for a row that has no distribution
    float rest_reference, rest;
    RowSums() = default;
    __device__ __forceinline__ RowSums(float reference_, float sum_, float rest_reference_, float rest_)
        : reference(reference_), sum(sum_ > 0.0f ? sum_ : __builtin_nanf("")), rest_reference(rest_reference_), rest(rest_)
    {
    }
    __device__ __forceinline__ explicit RowSums(const ExpSum &s) : RowSums(s.reference, s.sum, s.reference, s.second) {}
    // Whether the rest counts: there is a token outside the teacher's that may come (or no number).
    __device__ __forceinline__ bool has_rest(const DistillArgs &a) const { return a.rest && rest != 0.0f; }
};

// From a row's sums, ...
__device__ __forceinline__ Slope slope_of(const DistillArgs &a, float weight, const RowSums &s, float sum_q)
{
    return slope_of(a, weight, s.reference, log2f(s.sum), s.rest_reference, log2f(s.rest), s.rest * exp2_of((s.rest_reference - s.reference) * a.c) / s.sum,
                    s.has_rest(a), sum_q);
}
// ... and from the log sums that a call before has left.
__device__ __forceinline__ Slope slope_of(const DistillArgs &a, float weight, int64_t row, float sum_q)
{
    const float sum = a.saved_sums[row], rest = a.rest ? a.saved_rests[row] : 0.0f;
    const bool other = a.rest && rest != -__builtin_inff();
    const Saved whole(sum, a.temperature, a.c), part(other ? rest : 0.0f, a.temperature, a.c);
    return slope_of(a, weight, whole.reference, whole.log, part.reference, part.log, exp2_of((rest - sum) * kLog2e), other, sum_q);
}

__device__ __forceinline__ float weight_of(const DistillArgs &a, int64_t row) { return a.weights ? a.weights[row] : 1.0f; }

// The logits at the teacher's tokens: asked for early, values late.
template <int TYPE>
struct TokenLogits {
    LogitBits<TYPE> bits[2];
    template <bool PAST>
    __device__ __forceinline__ void load(const Places &p, const Row<TYPE, PAST> &x)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) bits[h] = x.bits(0, max(p.token[h], 0) + x.skip);
    }
    // ... in vectors first .. last - 1; where a token is elsewhere, the first logit there.
    template <bool PAST>
    __device__ __forceinline__ void load(const Places &p, const Row<TYPE, PAST> &x, int first, int last)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) bits[h] = x.bits(0, p.template is_in<TYPE>(h, x.skip, first, last) ? p.token[h] + x.skip : max(first * Logits<TYPE>::kCount, x.skip));
    }
    __device__ __forceinline__ float operator[](int h) const { return Row<TYPE>::value(bits[h]); }
    // ... that are here, behind this.
    __device__ __forceinline__ void wait() { asm volatile("" : "+v"(bits[0]), "+v"(bits[1])); }
};

// The loss of a row and its log sums, by one wave.
template <int TYPE>
__device__ __forceinline__ void write_loss(const DistillArgs &a, int64_t row, const Places &p, const TokenLogits<TYPE> &logit, const RowSums &s)
{
    const float log_sum = logf(s.sum), log_rest = logf(s.rest);
    float loss = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (p.token[h] >= 0 && p.q[h] != 0.0f) loss += p.q[h] * (p.log_q[h] - ((logit[h] - s.reference) * a.per_temperature - log_sum));
    loss = group_sum<64>(loss);
    if ((threadIdx.x & 63) != 0) return;
    const float left = fmaxf(1.0f - p.sum, 0.0f);
    if (s.has_rest(a) && left > 0.0f) loss += left * (logf(left) - ((s.rest_reference - s.reference) * a.per_temperature + (log_rest - log_sum)));
    a.losses[row] = log_sum == log_sum ? loss : log_sum;  // a row without a distribution may have no place that shows it
    if (a.log_sums) a.log_sums[row] = fmaf(s.reference, a.per_temperature, log_sum);
    // A rest may have a sum where the row has none: what spoils the row may be a token of the teacher's.
    if (a.log_rests) a.log_rests[row] = !a.rest ? 0.0f : log_sum == log_sum ? fmaf(s.rest_reference, a.per_temperature, log_rest) : log_sum;
}
__device__ __forceinline__ void write_no_loss(const DistillArgs &a, int64_t row)
{
    if (threadIdx.x != 0) return;
    a.losses[row] = 0.0f;
    if (a.log_sums) a.log_sums[row] = 0.0f;
    if (a.log_rests) a.log_rests[row] = 0.0f;
}

// The gradients of the teacher's tokens in vectors first .. last - 1, by one wave, in the place of what the workgroup has written there.
template <int TYPE, bool PAST>
__device__ __forceinline__ void put_tokens(const DistillArgs &a, const Places &p, const float (&q)[2], const TokenLogits<TYPE> &logit,
                                           const Slope &slope, const GradientRow<TYPE, PAST> &to, int first, int last)
{
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (p.is_in<TYPE>(h, to.skip, first, last)) to.store_one(slope.of_token(logit[h], q[h], a.c), p.token[h]);
}

// A bit for each logit of some vectors: whether it is the teacher's.
template <int N>
struct Marks {
    uint32_t *bits;  // in LDS
    int first;       // vector
    __device__ __forceinline__ void clear(int vectors, int threads) const
    {
        for (int i = threadIdx.x; i < (vectors * N + 31) / 32; i += threads) bits[i] = 0;
    }
    __device__ __forceinline__ void set(const Places &p, int skip, int vectors) const  // by one wave
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = p.token[h] + skip - first * N;
            if (p.token[h] >= 0 && at >= 0 && at < vectors * N) atomicOr(&bits[at / 32], 1u << at % 32);
        }
    }
    __device__ __forceinline__ uint32_t of(int j) const
    {
        const uint32_t at = (uint32_t)(j - first) * N;
        return bits[at / 32] >> at % 32 & ((1u << N) - 1);
    }
    __device__ __forceinline__ uint32_t is(int place) const  // from vector 0 on
    {
        const uint32_t at = place - first * N;
        return bits[at / 32] >> at % 32 & 1u;
    }
};

// A segment of a row to a workgroup; where a row has one only, that is all.  GRADIENT: with the gradient in a second pass, where there is no
// workspace for what a launch behind this one would need.
template <int TYPE, int THREADS, bool REST, bool PAST, bool GRADIENT>
__global__ __launch_bounds__(THREADS) void distill_kernel(DistillArgs a)
{
    constexpr int N = Logits<TYPE>::kCount, kRange = (1 << 17) / N;  // vectors that are marked at once
    __shared__ uint32_t bits[REST ? (1 << 17) / 32 : 1];
    __shared__ Places::Seen seen;
    const int t = threadIdx.x;
    const int local = quotient((int)blockIdx.x, a.by_segments), segment = (int)blockIdx.x - local * a.segments;
    const int64_t row = a.first_row + local;
    const Row<TYPE, PAST> x(a.logits, row * a.stride, a.vocab);
    const GradientRow<TYPE, PAST> to(a.gradient, GRADIENT ? row * a.gradient_stride : 0, x);
    const bool alone = a.segments == 1;
    const float weight = weight_of(a, row);
    if (weight == 0.0f) {
        if (alone) write_no_loss(a, row);
        if (GRADIENT) write_zeros<THREADS>(x, to, 0, x.vectors);
        return;
    }
    const Places places(a, row);
    if (!places.any) {
        if (alone) write_no_loss(a, row);
        if (GRADIENT) write_zeros<THREADS>(x, to, 0, x.vectors);
        return;
    }
    TokenLogits<TYPE> logit = {};
    if (alone && t < 64) logit.load(places, x);
    Adder<REST ? 2 : 0> adder(a.c);
    const int first = segment * a.segment_vectors, last = alone ? x.vectors : min(first + a.segment_vectors, x.vectors);
    if (REST) {
        for (int from = first; from < last; from += kRange) {
            const int to = min(from + kRange, last);
            const Marks<N> marks{bits, from};
            marks.clear(to - from, THREADS);
            __syncthreads();
            if (t < 64) marks.set(places, x.skip, to - from);
            __syncthreads();
            walk<THREADS, 4>(
                x, from, to, [&](const Logits<TYPE> &v, int j, int) { adder.add(v, marks.of(min(j, to - 1))); },
                [&](const Logits<TYPE> &v, int token) { adder.add(v, token >= 0 ? marks.is(token + x.skip) : 0u); });
            __syncthreads();
        }
    } else {
        walk<THREADS, 4>(
            x, first, last, [&](const Logits<TYPE> &v, int, int) { adder.add(v); }, [&](const Logits<TYPE> &v, int) { adder.add(v); });
    }
    logit.wait();  // before the barriers in join: the gradient may take the logits' place
    const ExpSum s = join<false, THREADS>(adder.result(), a.c);
    if (alone && t < 64) write_loss(a, row, places, logit, RowSums(s));
    if (a.parts && t == 0) a.parts[blockIdx.x] = {s.reference, s.sum, s.second, 0.0f};
    if (GRADIENT) {
        const Slope slope = slope_of(a, weight, RowSums(s), places.sum);
        const Span span(x, 0, x.vectors);
        walk<THREADS, 4>(
            x, 0, x.vectors,
            [&](const Logits<TYPE> &v, int j, int) {
                float g[N];
                slope.of_others(v, a.c, g);
                if (j < span.end) to.store(g, j);
            },
            [&](const Logits<TYPE> &v, int token) {
                float g[N];
                slope.of_others(v, a.c, g);
                if (token >= 0) to.store_one(g[0], token);
            });
        __syncthreads();
        if (t < 64) {
            float q[2];
            bool is_first[2];
            places.of_tokens(seen, a.places, q, is_first);
            put_tokens(a, places, q, logit, slope, to, 0, x.vectors);
        }
    }
}

// A row to a wave: its segments' sums as one, which take the first one's place for the gradient.
template <int TYPE>
__global__ __launch_bounds__(64) void distill_join_kernel(DistillArgs a)
{
    const int64_t row = a.first_row + blockIdx.x;
    const float weight = weight_of(a, row);
    if (weight == 0.0f) {
        write_no_loss(a, row);
        return;
    }
    LogitsPart *parts = a.parts + (int64_t)blockIdx.x * a.segments;
    const ExpSum s = join<false, 64>(parts, a.segments, a.c);
    const Places places(a, row);
    if (!places.any) {
        write_no_loss(a, row);
        return;
    }
    TokenLogits<TYPE> logit;
    logit.load(places, Row<TYPE>(a.logits, row * a.stride, a.vocab));
    write_loss(a, row, places, logit, RowSums(s));
    if (threadIdx.x == 0) parts[0] = {s.reference, s.sum, s.second, 0.0f};
}

// A segment of a row's gradient to a workgroup: from the sums that the launches in front left, or from those of an earlier call.  One wave makes
// what the others need, while their logits are on the way.  Joining: each workgroup joins the sums of the row's parts for itself and the first one of a
// row writes its loss, which saves a launch (1 row of 144086 bf16 logits, 95 places, 10.6 -> 8.5 us, 21 of 90480 11.8 -> 9.3); it reads the teacher's logits while others write, so not
// where the gradient takes their place.
template <int TYPE, bool PAST>
__global__ __launch_bounds__(kThreads) void distill_gradient_kernel(DistillArgs a)
{
    constexpr int N = Logits<TYPE>::kCount;
    __shared__ int shared_tokens;  // whether the segment holds some of the teacher's; -1: the teacher has none
    __shared__ Slope shared_slope;
    __shared__ Places::Seen seen;
    const int t = threadIdx.x;
    const int local = quotient((int)blockIdx.x, a.by_segments), segment = (int)blockIdx.x - local * a.segments;
    const int64_t row = a.first_row + local;
    const Row<TYPE, PAST> x(a.logits, row * a.stride, a.vocab);
    const GradientRow<TYPE, PAST> to(a.gradient, row * a.gradient_stride, x);
    const int first = segment * a.segment_vectors, last = min(first + a.segment_vectors, x.vectors);
    const float weight = weight_of(a, row);
    const bool loss = a.joining && segment == 0;
    if (weight == 0.0f) {
        if (loss) write_no_loss(a, row);
        write_zeros<kThreads>(x, to, first, last);
        return;
    }
    GradientSegment<kThreads, kGradientVectors, TYPE, PAST> segment_of(x, to, first, last);
    Places places;
    TokenLogits<TYPE> logit;
    if (t < 64) {
        places = Places(a, row);
        RowSums sums;
        TokenLogits<TYPE> of_row;
        if (!a.saved_sums) sums = RowSums(join<false, 64>(a.parts + (int64_t)local * a.row_parts, a.joining ? a.row_parts : 1, a.c));
        if (loss) of_row.load(places, x);
        segment_of.load();
        const Slope slope = a.saved_sums ? slope_of(a, weight, row, places.sum) : slope_of(a, weight, sums, places.sum);
        const bool here = places.template is_in<TYPE>(0, x.skip, first, last) || places.template is_in<TYPE>(1, x.skip, first, last);
        const bool tokens = __builtin_amdgcn_ballot_w64(here) != 0;
        if (tokens) {
            logit.load(places, x, first, last);
            logit.wait();
        }
        if (t == 0) {
            shared_tokens = places.any ? (tokens ? 1 : 0) : -1;
            shared_slope = slope;
        }
        if (loss && places.any)
            write_loss(a, row, places, of_row, sums);
        else if (loss)
            write_no_loss(a, row);
    } else {
        segment_of.load();
    }
    __syncthreads();
    const int tokens = shared_tokens;
    if (tokens < 0) {
        write_zeros<kThreads>(x, to, first, last);
        return;
    }
    const Slope slope = shared_slope;
    segment_of.write([&](const Logits<TYPE> &v, int, float(&g)[N]) { slope.of_others(v, a.c, g); });
    if (!tokens) return;
    float q[2];
    bool is_first[2];
    if (t < 64) places.of_tokens(seen, a.places, q, is_first);
    __syncthreads();
    if (t < 64) put_tokens(a, places, q, logit, slope, to, first, last);
}

// A bit for each logit of a row that is held in registers: whether it is the teacher's; the vectors of a thread in neighbouring bytes, the row's ends last.
template <int N, int THREADS, int VECTORS>
struct HeldMarks {
    static constexpr int kOfThread = VECTORS / 4;
    static_assert(VECTORS % 4 == 0, "whole words");
    struct alignas(4 * kOfThread) Word {
        uint32_t w[kOfThread];
        __device__ __forceinline__ uint32_t of(int u) const { return w[u / 4] >> 8 * (u % 4) & 0xffu; }
    };
    Word words[THREADS];
    uint32_t ends;  // as in Ends, a bit for a lane

    // By one wave.  Vectors held_end .. span.end - 1 are not held.
    __device__ __forceinline__ void set(const Places &p, int skip, const Span &span, int held_end)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < THREADS; i += 64) words[i + lane] = {};
        if (lane == 0) ends = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (p.token[h] >= 0) {
                const int at = p.token[h] + skip, j = at / N, i = j - span.begin, u = i / THREADS;
                if (i >= 0 && j < held_end)
                    atomicOr(&words[i % THREADS].w[u / 4], 1u << (8 * (u % 4) + at % N));
                else if (i < 0 || j >= span.end)
                    atomicOr(&ends, 1u << (i < 0 ? 0 : N) + at % N);
            }
    }
};

// A row to a workgroup that holds it in its registers, so that it is read once for the loss and the gradient.  The row has a vector that lies inside
// it.  For a rest the teacher's tokens are taken out of the registers, so that the row's sum is the rest's, to which theirs is added.  MORE: a row of up to
// twice what the registers hold, of which the rest is read again (before the registers are filled and after they are written, when they are free).
template <int TYPE, int THREADS, int VECTORS, bool REST, bool MORE>
__global__ __launch_bounds__(THREADS, VECTORS <= 4 ? 8 : 4) void distill_resident_kernel(DistillArgs a)
{
    using TheirMarks = HeldMarks<Logits<TYPE>::kCount, THREADS, VECTORS>;
    constexpr int kHeld = THREADS * VECTORS;
    __shared__ std::conditional_t<REST, TheirMarks, int> marks;
    __shared__ uint32_t bits[REST && MORE ? kHeld * Logits<TYPE>::kCount / 32 : 1];
    __shared__ Places::Seen seen;
    __shared__ float of_teacher[2];
    constexpr int N = Logits<TYPE>::kCount;
    const int t = threadIdx.x;
    const int64_t row = a.first_row + blockIdx.x;
    const Row<TYPE, true> x(a.logits, row * a.stride, a.vocab);
    const GradientRow<TYPE, true> to(a.gradient, row * a.gradient_stride, x);
    const Span span(x, 0, x.vectors);
    const float weight = weight_of(a, row);
    if (weight == 0.0f) {
        write_no_loss(a, row);
        write_zeros<THREADS>(x, to, 0, x.vectors);
        return;
    }
    const Places::Raw raw(a, row);
    Held<THREADS, VECTORS, TYPE> held;
    if (!MORE) held.load(x, span);
    Ends<TYPE> ends = {};
    if (t < 64 && span.has_ends()) ends.load(x, span);
    const Places places(a, raw);
    if (!places.any) {
        write_no_loss(a, row);
        write_zeros<THREADS>(x, to, 0, x.vectors);
        return;
    }
    TokenLogits<TYPE> logit = {};
    float q[2] = {};
    bool first[2] = {};
    const int held_end = MORE ? min(span.begin + kHeld, span.end) : span.end;
    const Row<TYPE, false> again(a.logits, row * a.stride, a.vocab);  // stays in the caches
    const Marks<N> of_more{bits, held_end};
    if (REST && MORE) {
        of_more.clear(span.end - held_end, THREADS);
        __syncthreads();
    }
    if (t < 64) {
        logit.load(places, x);
        if constexpr (REST) marks.set(places, x.skip, span, held_end);
        if (REST && MORE) of_more.set(places, x.skip, span.end - held_end);
    }
    typename TheirMarks::Word mine = {};
    if constexpr (REST) {
        __syncthreads();
        mine = marks.words[t];
    }
    Adder<0> adder(a.c);
    if (MORE) {
        walk<THREADS, 4>(
            again, held_end, span.end,
            [&](Logits<TYPE> &v, int j, int) {
                const uint32_t which = REST && j < span.end ? of_more.of(j) : 0;
                if (which) v.fill(which);
                adder.add(v);
            },
            [](const Logits<TYPE> &, int) {});
        held.load(x, span);
    }
    if (t < 64) places.of_tokens(seen, a.places, q, first);  // while the logits are on the way
    held.go_through(span, [&](Logits<TYPE> &v, int j, int u) {
        if (j >= span.end) v.fill();
        if (REST && mine.of(u)) v.fill(mine.of(u));
        adder.add(v);
    });
    if (t < 64 && span.has_ends()) {
        Logits<TYPE> v = ends.vector();
        if constexpr (REST) v.fill(t < 32 ? marks.ends >> t & 1u : 0u);
        adder.add(v);
    }
    logit.wait();  // before the barriers in join: the gradient may take the logits' place
    ExpSum s = adder.result(), teachers;
    if (REST && t < 64) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (places.token[h] >= 0 && first[h]) {
                rebase<false>(teachers, fmaxf(teachers.reference, logit[h]), a.c);
                teachers.sum += exp2_of((logit[h] - teachers.reference) * a.c);
            }
        teachers = join_lanes<false, 64>(teachers, a.c);
        if (t == 0) {
            of_teacher[0] = teachers.reference;
            of_teacher[1] = teachers.sum;
        }
    }
    s = join<false, THREADS>(s, a.c);
    RowSums sums(s.reference, s.sum, 0.0f, 0.0f);
    if (REST) {
        if (THREADS > 64) {
            teachers.reference = of_teacher[0];
            teachers.sum = of_teacher[1];
        }
        const ExpSum rest = s;
        const float top = fmaxf(s.reference, teachers.reference);
        rebase<false>(s, top, a.c);
        rebase<false>(teachers, top, a.c);
        sums = RowSums(top, s.sum + teachers.sum, rest.reference, rest.sum);
    }
    if (t < 64) write_loss(a, row, places, logit, sums);
    const Slope slope = slope_of(a, weight, sums, places.sum);
    held.go_through(span, [&](const Logits<TYPE> &v, int j, int) {
        float g[N];
        slope.of_others(v, a.c, g);
        if (j < span.end) to.store(g, j);
    });
    if (MORE)
        walk<THREADS, 4>(
            again, held_end, span.end,
            [&](const Logits<TYPE> &v, int j, int) {
                float g[N];
                slope.of_others(v, a.c, g);
                if (j < span.end) to.store(g, j);
            },
            [](const Logits<TYPE> &, int) {});
    if (t < 64 && span.has_ends()) {
        float g[N];
        slope.of_others(ends.vector(), a.c, g);
        if (ends.token >= 0) to.store_one(g[0], ends.token);
    }
    __syncthreads();
    if (t < 64) put_tokens(a, places, q, logit, slope, to, 0, x.vectors);
}

template <int TYPE, bool REST>
void launch_resident(const DistillArgs &a, const LogitsPlan &form, int64_t rows, hipStream_t stream)
{
    auto kernel = form.threads == 64    ? distill_resident_kernel<TYPE, 64, 4, REST, false>
                  : form.threads == 256 ? distill_resident_kernel<TYPE, 256, 4, REST, false>
                  : form.vectors == 4   ? distill_resident_kernel<TYPE, 512, 4, REST, false>
                  : form.vectors == 8   ? distill_resident_kernel<TYPE, 512, 8, REST, false>
                  : form.threads == 512 ? distill_resident_kernel<TYPE, 512, 16, REST, false>
                  : form.vectors == 16  ? distill_resident_kernel<TYPE, 1024, 16, REST, false>
                                        : distill_resident_kernel<TYPE, 1024, 16, REST, true>;
    if constexpr (REST && TYPE != QUAMBA_F32)
        if (form.threads == 512 && form.vectors == 32) kernel = distill_resident_kernel<TYPE, 512, 16, true, true>;
    kernel<<<(int)rows, form.threads, 0, stream>>>(a);
}

template <int TYPE, int THREADS, bool PAST, bool GRADIENT>
void launch_first(const DistillArgs &a, int grid, hipStream_t stream)
{
    (a.rest ? distill_kernel<TYPE, THREADS, true, PAST, GRADIENT> : distill_kernel<TYPE, THREADS, false, PAST, GRADIENT>)<<<grid, THREADS, 0, stream>>>(a);
}

template <int TYPE, bool PAST>
void launch_sums(const DistillArgs &a, int threads, int64_t rows, hipStream_t stream)
{
    const int grid = (int)(rows * a.segments);
    if (a.gradient && !a.parts)
        launch_first<TYPE, 256, PAST, true>(a, grid, stream);
    else if (threads == 1024)
        launch_first<TYPE, 1024, false, false>(a, grid, stream);
    else if (threads == 64)
        launch_first<TYPE, 64, false, false>(a, grid, stream);
    else
        launch_first<TYPE, 256, PAST, false>(a, grid, stream);
    if (a.segments > 1 && !a.joining) distill_join_kernel<TYPE><<<(int)rows, 64, 0, stream>>>(a);
}

void cut_into(DistillArgs &a, const LogitsPlan &plan)
{
    a.segments = plan.segments;
    a.segment_vectors = plan.vectors;
    a.by_segments = divisor((uint32_t)plan.segments);
}

// The gradient's launch joins segments where it does not take the logits' place.
LogitsWork work_of(bool in_place) { return in_place ? LogitsWork::distance : LogitsWork::step; }

}  // namespace

// Few vectors to a thread while the row's work is mostly waiting (bf16, 32 places and a rest: 256 rows of 8000 by 512 threads with 4 vectors 7.7 us, by 256
// with 8 10.1; of 16000 8.5 and 10.2), more where several workgroups have to share a compute unit so that one's loads go while another computes (4096 rows of
// 20000 by 1024 threads with 4 vectors 88 us, by 512 with 8 65; of 64000 by 1024 with 8 235 and by 512 with 16 186).  So the most work, that of a rest in 16-bit
// logits, is left to two workgroups of 512 threads even where each has to read some of its row again, from the caches (4096 rows of 70000 by 1024 with 16
// vectors 278, by 512 that hold 16 of 32 222; of 128000 414 and 404; without a rest 241 and 218, 375 and 401; 2048 of 50000 in fp32 160 and 165; and where each has
// a unit for itself both take about as long: 96 rows of 128000 21.4 and 21.8, 250 30.1 and 29.5, 257 46.8 and 39.0, 96 of 70000 15.8 and 14.9).
// Rows of up to twice what 1024 threads hold are cheaper in part than in two launches (2048 of 140000 bf16 logits 210 and 271 us, of 260000 439 and 524; 100 of
// 200000 24.6 and 27.8).  Few long rows are cut into segments instead.
LogitsPlan distill_form(int64_t rows, int32_t vocab, int32_t type, bool rest, bool in_place, bool workspace)
{
    const int vectors = logit_vectors(vocab, type);
    if (vocab < (type == QUAMBA_F32 ? 8 : 16)) return {};  // it may have no vector of its own
    if (logits_plan(rows, vocab, type, work_of(in_place), 0, false, workspace).segments > 1) return {};
    if (vectors <= wave_vectors(rows, 4 * 64)) return {64, 1, 4};
    if (vectors <= 4 * 256) return {256, 1, 4};
    for (const int each : {4, 8, 16})
        if (vectors <= each * 512) return {512, 1, each};
    if (vectors <= 16 * 1024) return rest && type != QUAMBA_F32 ? LogitsPlan{512, 1, 32} : LogitsPlan{1024, 1, 16};
    if (vectors <= 32 * 1024) return {1024, 1, 32};
    return {};
}

namespace {

template <int TYPE, bool PAST>
hipError_t launch(DistillArgs a, void *workspace, hipStream_t stream)
{
    const bool sums = !a.saved_sums;
    const bool in_place = a.gradient == a.logits, step = sums && a.gradient;
    const LogitsPlan form = step ? distill_form(a.rows, a.vocab, TYPE, a.rest, in_place, workspace != nullptr) : LogitsPlan{};
    const bool resident = form.threads != 0;
    const LogitsPlan plan = logits_plan(a.rows, a.vocab, TYPE, step ? work_of(in_place) : LogitsWork::distance, 0, false, workspace != nullptr);
    const LogitsPlan gradient = gradient_plan(a.vocab, TYPE, kThreads * kGradientVectors);
    a.parts = static_cast<LogitsPart *>(workspace);
    a.row_parts = plan.segments;
    a.joining = plan.segments > 1 && step && !in_place;
    const int64_t most = a.gradient && !resident ? kRowsOfALaunch / gradient.segments : kRowsOfALaunch;
    for (a.first_row = 0; a.first_row < a.rows; a.first_row += most) {
        const int64_t rows = std::min(a.rows - a.first_row, most);
        if (resident) {
            a.rest ? launch_resident<TYPE, true>(a, form, rows, stream) : launch_resident<TYPE, false>(a, form, rows, stream);
        } else {
            cut_into(a, plan);
            if (sums) launch_sums<TYPE, PAST>(a, plan.threads, rows, stream);
            cut_into(a, gradient);
            if (a.gradient && (a.parts || !sums)) distill_gradient_kernel<TYPE, PAST><<<(int)(rows * a.segments), kThreads, 0, stream>>>(a);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int TYPE>
hipError_t launch(const DistillArgs &a, void *workspace, hipStream_t stream)
{
    return logits_past_caches(a.rows, a.vocab, TYPE) ? launch<TYPE, true>(a, workspace, stream) : launch<TYPE, false>(a, workspace, stream);
}

}  // namespace

size_t distill_workspace_bytes(int64_t rows, int32_t vocab)
{
    size_t most = 0;  // over the types, with the gradient and without
    for (const int type : {QUAMBA_F32, QUAMBA_BF16})
        for (const LogitsWork work : {LogitsWork::distance, LogitsWork::step})
            most = std::max(most, (size_t)rows * logits_plan(rows, vocab, type, work, 0, false, true).segments * sizeof(LogitsPart));
    return most;
}

hipError_t launch_distill(const DistillArgs &a, void *workspace, hipStream_t stream)
{
    switch (a.type) {
        case QUAMBA_F32: return launch<QUAMBA_F32>(a, workspace, stream);
        case QUAMBA_F16: return launch<QUAMBA_F16>(a, workspace, stream);
        default: return launch<QUAMBA_BF16>(a, workspace, stream);
    }
}

}  // namespace quamba
