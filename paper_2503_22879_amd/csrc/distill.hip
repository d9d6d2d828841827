// The distance of rows of logits x, at a temperature T, from a teacher that is known by its most likely tokens, and its gradient.
//
//   loss = sum_k q_k (ln q_k - ln p[token_k])  + q_R (ln q_R - ln p_R),      p = softmax(x / T),  p_R = sum of p over the other tokens
//   dx_v = w / T (p_v Q - sum of the q_k with token_k = v),  Q = sum_k q_k + q_R;    of other tokens w / T (p_v / p_R) (Q p_R - q_R)
//
// One pass over a row makes its sum of exponentials and the other tokens' (whose own sum is exact where it is a small part of the row's: a
// difference would not be); a second one writes the gradient as if no token were the teacher's, and then the teacher's tokens are
// put right one by one from their logits, which were read before.  Bound: HBM.
#include <algorithm>

#include "logits.h"

namespace quamba {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kRowsOfALaunch = (int64_t)1 << 22;
constexpr float kLog2e = 1.44269504088896341f;

// The teacher's places of a row, in LDS.
struct Places {
    float q[kMaxPlaces], log_q[kMaxPlaces], logit[kMaxPlaces];
    int32_t token[kMaxPlaces];  // -1: an empty place
    float wave[4][2];
};

// Fills them in; every thread gets the sum of q.  any: whether there is a place that is not empty.
template <int TYPE>
__device__ __forceinline__ float read_places(Places &s, const DistillArgs &a, int64_t row, const Row<TYPE> &x, bool &any)
{
    const int t = threadIdx.x, w = t / 64;
    float value = -__builtin_inff(), logit = 0.0f, q = 0.0f;
    int token = -1;
    if (t < a.places) {
        value = a.teacher[row * a.places + t];
        token = a.tokens[row * a.places + t];
        if ((uint32_t)token >= (uint32_t)a.vocab || value == -__builtin_inff()) {
            token = -1;
            value = -__builtin_inff();
        } else {
            logit = x.logit(token);
        }
    }
    any = __syncthreads_or(token >= 0);
    float log_q = value;
    if (!a.rest) {  // to sum to 1
        const float top = wave_max(value);
        if (t % 64 == 0 && w < 2) s.wave[w][0] = top;
        __syncthreads();
        log_q = (value - fmaxf(s.wave[0][0], s.wave[1][0])) * a.per_temperature;
    }
    if (token >= 0) q = expf(log_q);
    float sum = group_sum<64>(q);
    if (t % 64 == 0 && w < 2) s.wave[w][1] = sum;
    __syncthreads();
    sum = s.wave[0][1] + s.wave[1][1];
    if (!a.rest) {
        log_q -= logf(sum);
        q /= sum;
        sum = group_sum<64>(q);
        if (t % 64 == 0 && w < 2) s.wave[w + 2][1] = sum;
        __syncthreads();
        sum = s.wave[2][1] + s.wave[3][1];
    }
    if (t < a.places) {
        s.q[t] = q;
        s.log_q[t] = log_q;
        s.logit[t] = logit;
        s.token[t] = token;
    }
    __syncthreads();
    return sum;
}

// What the gradient of a row is made from: that of other tokens is flat 2^((x - reference) c - log), that of the teacher's comes from p and q.
struct Slope {
    float reference, log, flat;
    float own_reference, own_log, whole, scale;
    __device__ __forceinline__ float of_place(const Places &s, int places, int k, float c) const
    {
        float q = 0.0f;  // a token may have several places
        for (int i = 0; i < places; ++i) q += s.token[i] == s.token[k] ? s.q[i] : 0.0f;
        return (exp2_of(fmaf(s.logit[k] - own_reference, c, -own_log)) * whole - q) * scale;
    }
};

__device__ __forceinline__ Slope slope_of(float reference, float log_sum, float rest_reference, float log_rest, float share, bool rest, float sum_q,
                                          float scale)
{
    Slope s;
    const float left = rest ? fmaxf(1.0f - sum_q, 0.0f) : 0.0f;
    s.own_reference = reference;
    s.own_log = log_sum;
    s.whole = sum_q + left;
    s.scale = scale;
    s.reference = rest ? rest_reference : reference;
    s.log = rest ? log_rest : log_sum;
    s.flat = (rest ? fmaf(s.whole, share, -left) : s.whole) * scale;
    return s;
}

// Whether the rest counts: there is a token outside the teacher's that may come (or no number).
__device__ __forceinline__ bool has_rest(const DistillArgs &a, const ExpSum &s) { return a.rest && s.second != 0.0f; }

__device__ __forceinline__ Slope slope_of(const DistillArgs &a, int64_t row, const ExpSum &s, float sum_q)
{
    const float sum = s.sum > 0.0f ? s.sum : __builtin_nanf("");
    return slope_of(s.reference, log2f(sum), s.reference, log2f(s.second), s.second / sum, has_rest(a, s), sum_q,
                    (a.weights ? a.weights[row] : 1.0f) * a.per_temperature);
}

// The losses of a row and its log sums.
__device__ __forceinline__ void write_loss(const DistillArgs &a, int64_t row, Places &p, const ExpSum &s, float sum_q)
{
    const int t = threadIdx.x, w = t / 64;
    const float log_sum = s.sum > 0.0f ? logf(s.sum) : __builtin_nanf("");
    float term = 0.0f;
    if (t < a.places && p.token[t] >= 0 && p.q[t] != 0.0f)
        term = p.q[t] * (p.log_q[t] - ((p.logit[t] - s.reference) * a.per_temperature - log_sum));
    term = group_sum<64>(term);
    if (t % 64 == 0 && w < 2) p.wave[w][0] = term;
    __syncthreads();
    if (t != 0) return;
    float loss = p.wave[0][0] + p.wave[1][0];
    const float left = fmaxf(1.0f - sum_q, 0.0f), log_rest = logf(s.second);
    if (has_rest(a, s) && left > 0.0f) loss += left * (logf(left) - (log_rest - log_sum));
    // a sum of no number may have met no place that shows it
    a.losses[row] = log_sum == log_sum ? loss : log_sum;
    if (a.log_sums) a.log_sums[row] = fmaf(s.reference, a.per_temperature, log_sum);
    if (a.log_rests) a.log_rests[row] = a.rest ? fmaf(s.reference, a.per_temperature, log_rest) : 0.0f;
}
__device__ __forceinline__ void write_no_loss(const DistillArgs &a, int64_t row)
{
    if (threadIdx.x != 0) return;
    a.losses[row] = 0.0f;
    if (a.log_sums) a.log_sums[row] = 0.0f;
    if (a.log_rests) a.log_rests[row] = 0.0f;
}

// The gradient of vectors first .. last - 1 of a row.
template <int TYPE>
__device__ __forceinline__ void write_slope(const DistillArgs &a, const Row<TYPE> &x, const GradientRow<TYPE> &to, const Places &p, const Slope &s,
                                            int first, int last)
{
    write_gradient<TYPE, kThreads, 4, false>(x, to, first, last, s.reference, a.c, s.log, s.flat, 0.0f);
    __syncthreads();
    const int t = threadIdx.x;
    if (t < a.places && p.token[t] >= 0) {
        const int at = p.token[t] + x.skip;
        if (at >= first * Logits<TYPE>::kCount && at < last * Logits<TYPE>::kCount) to.store_one(s.of_place(p, a.places, t, a.c), p.token[t]);
    }
}

// A segment of a row to a workgroup; where a row has one only, that is all, with the gradient.
template <int TYPE, bool REST>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a)
{
    constexpr int N = Logits<TYPE>::kCount, kRange = (1 << 17) / N;  // vectors that are marked at once
    __shared__ Places places;
    __shared__ uint32_t marks[REST ? (1 << 17) / 32 : 1];           // a bit for a logit: whether it is the teacher's
    const int t = threadIdx.x;
    const int local = quotient((int)blockIdx.x, a.by_segments), segment = (int)blockIdx.x - local * a.segments;
    const int64_t row = a.first_row + local;
    const Row<TYPE> x(a.logits, row * a.stride, a.vocab);
    const bool alone = a.segments == 1;
    bool live = !a.weights || a.weights[row] != 0.0f;
    float sum_q = 0.0f;
    if (live) sum_q = read_places(places, a, row, x, live);
    if (!live) {
        if (alone) {
            write_no_loss(a, row);
            if (a.gradient) write_zeros<TYPE, kThreads>(GradientRow<TYPE>(a.gradient, row * a.gradient_stride, x), 0, x.vectors);
        }
        return;
    }
    ExpSum s;
    const int first = segment * a.segment_vectors, last = alone ? x.vectors : min(first + a.segment_vectors, x.vectors);
    if (REST) {
        for (int from = first; from < last; from += kRange) {
            const int to = min(from + kRange, last);
            for (int i = t; i < ((to - from) * N + 31) / 32; i += kThreads) marks[i] = 0;
            __syncthreads();
            if (t < a.places && places.token[t] >= 0) {
                const int at = places.token[t] + x.skip - from * N;
                if (at >= 0 && at < (to - from) * N) atomicOr(&marks[at / 32], 1u << at % 32);
            }
            __syncthreads();
            walk<TYPE, kThreads, 4>(x, from, to, [&](const Logits<TYPE> &v, int j) {
                const int at = (min(j, to - 1) - from) * N;
                add<2>(s, v, largest(v), a.c, marks[at / 32] >> at % 32 & ((1u << N) - 1));
            });
            __syncthreads();
        }
    } else {
        walk<TYPE, kThreads, 4>(x, first, last, [&](const Logits<TYPE> &v, int) { add<0>(s, v, largest(v), a.c); });
    }
    s = join<false, kThreads>(s, a.c);
    if (!alone) {
        if (t == 0) a.parts[blockIdx.x] = {s.reference, s.sum, s.second, 0.0f};
        return;
    }
    write_loss(a, row, places, s, sum_q);
    if (a.gradient) write_slope(a, x, GradientRow<TYPE>(a.gradient, row * a.gradient_stride, x), places, slope_of(a, row, s, sum_q), 0, x.vectors);
}

// A row to a workgroup: its segments' sums as one, which take the first one's place for the gradient.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void distill_join_kernel(DistillArgs a)
{
    __shared__ Places places;
    const int64_t row = a.first_row + blockIdx.x;
    const Row<TYPE> x(a.logits, row * a.stride, a.vocab);
    bool live = !a.weights || a.weights[row] != 0.0f;
    float sum_q = 0.0f;
    if (live) sum_q = read_places(places, a, row, x, live);
    if (!live) {
        write_no_loss(a, row);
        return;
    }
    LogitsPart *parts = a.parts + (int64_t)blockIdx.x * a.segments;
    const ExpSum s = join<false, kThreads>(parts, a.segments, a.c);
    write_loss(a, row, places, s, sum_q);
    if (threadIdx.x == 0) parts[0] = {s.reference, s.sum, s.second, 0.0f};
}

// A segment of a row's gradient to a workgroup: from the sums that the launches in front left, or from those of an earlier call.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void distill_gradient_kernel(DistillArgs a)
{
    __shared__ Places places;
    const int local = quotient((int)blockIdx.x, a.by_segments), segment = (int)blockIdx.x - local * a.segments;
    const int64_t row = a.first_row + local;
    const Row<TYPE> x(a.logits, row * a.stride, a.vocab);
    const GradientRow<TYPE> to(a.gradient, row * a.gradient_stride, x);
    const int first = segment * a.segment_vectors, last = min(first + a.segment_vectors, x.vectors);
    bool live = !a.weights || a.weights[row] != 0.0f;
    float sum_q = 0.0f;
    if (live) sum_q = read_places(places, a, row, x, live);
    if (!live) {
        write_zeros<TYPE, kThreads>(to, first, last);
        return;
    }
    Slope slope;
    if (a.saved_sums) {
        const float sum = a.saved_sums[row], rest = a.rest ? a.saved_rests[row] : 0.0f;
        const bool other = a.rest && rest != -__builtin_inff();
        const Saved whole(sum, a.temperature, a.c), part(other ? rest : 0.0f, a.temperature, a.c);
        slope = slope_of(whole.reference, whole.log, part.reference, part.log, exp2_of((rest - sum) * kLog2e), other, sum_q,
                         (a.weights ? a.weights[row] : 1.0f) * a.per_temperature);
    } else {
        const LogitsPart part = a.parts[(int64_t)local * a.segments];
        ExpSum s;
        s.reference = part.reference;
        s.sum = part.sum;
        s.second = part.second;
        slope = slope_of(a, row, s, sum_q);
    }
    write_slope(a, x, to, places, slope, first, last);
}

template <int TYPE>
void launch_rows(const DistillArgs &a, int64_t rows, hipStream_t stream)
{
    const int grid = (int)(rows * a.segments);
    if (a.rest)
        distill_kernel<TYPE, true><<<grid, kThreads, 0, stream>>>(a);
    else
        distill_kernel<TYPE, false><<<grid, kThreads, 0, stream>>>(a);
    if (a.segments == 1) return;
    distill_join_kernel<TYPE><<<(int)rows, kThreads, 0, stream>>>(a);
    if (a.gradient) distill_gradient_kernel<TYPE><<<grid, kThreads, 0, stream>>>(a);
}

template <int TYPE>
void launch_gradient(const DistillArgs &a, int64_t rows, hipStream_t stream)
{
    distill_gradient_kernel<TYPE><<<(int)(rows * a.segments), kThreads, 0, stream>>>(a);
}

template <typename F>
hipError_t by_launches(DistillArgs &a, const LogitsCut &cut, const F &launch)
{
    a.segments = cut.segments;
    a.segment_vectors = cut.vectors;
    a.by_segments = divisor((uint32_t)cut.segments);
    for (a.first_row = 0; a.first_row < a.rows; a.first_row += kRowsOfALaunch) {
        launch(std::min(a.rows - a.first_row, kRowsOfALaunch));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t distill_workspace_bytes(int64_t rows, int32_t vocab)
{
    size_t most = 0;  // over the types
    for (const int type : {QUAMBA_F32, QUAMBA_BF16}) {
        const int segments = logits_cut(rows, vocab, type).segments;
        if (segments > 1) most = std::max(most, (size_t)rows * segments * sizeof(LogitsPart));
    }
    return most;
}

hipError_t launch_distill(DistillArgs a, void *workspace, hipStream_t stream)
{
    a.parts = static_cast<LogitsPart *>(workspace);
    return by_launches(a, workspace ? logits_cut(a.rows, a.vocab, a.type) : LogitsCut{1, 0}, [&](int64_t rows) {
        switch (a.type) {
            case QUAMBA_F32: launch_rows<QUAMBA_F32>(a, rows, stream); break;
            case QUAMBA_F16: launch_rows<QUAMBA_F16>(a, rows, stream); break;
            default: launch_rows<QUAMBA_BF16>(a, rows, stream); break;
        }
    });
}

hipError_t launch_distill_backward(DistillArgs a, hipStream_t stream)
{
    return by_launches(a, logits_cut(a.rows, a.vocab, a.type), [&](int64_t rows) {
        switch (a.type) {
            case QUAMBA_F32: launch_gradient<QUAMBA_F32>(a, rows, stream); break;
            case QUAMBA_F16: launch_gradient<QUAMBA_F16>(a, rows, stream); break;
            default: launch_gradient<QUAMBA_BF16>(a, rows, stream); break;
        }
    });
}

}  // namespace quamba
