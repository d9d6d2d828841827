// Log probabilities of given tokens under rows of logits x at a temperature T, with the entropy and the most likely alternatives, and the
// gradient of the first two.
//
//   logprob = (x_t - m) / T - ln S,   S = sum_v exp((x_v - m) / T)       entropy = ln S - sum_v exp(e_v) e_v / S,   e_v = (x_v - m) / T
//   dx_v = (g ([v = t] - p_v) - h p_v (ln p_v + entropy)) / T
//
// One pass over a row makes the sum, the entropy's sum and the list of the best tokens (logits.h).  Bound: HBM, the logits read once, and read
// and written once for the gradient.
#include <algorithm>

#include "logits.h"

namespace quamba {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int64_t kRowsOfALaunch = (int64_t)1 << 22;

// The lists of a workgroup's waves as one: out(i, key) for the i-th largest, i < count, 0 where there are no more.
template <int WAVES, typename Out>
__device__ __forceinline__ void ranked(const uint64_t (&keys)[WAVES][kListed], TopList &list, int count, const Out &out)
{
    __shared__ int lengths[WAVES];
    if (list.n > count) list.shrink();
    if (threadIdx.x % 64 == 0) lengths[threadIdx.x / 64] = list.n;
    __syncthreads();
    int n[WAVES], all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all += n[w] = lengths[w];
    for (int i = threadIdx.x; i < WAVES * kMaxChoices; i += WAVES * 64) {
        const int w = i / kMaxChoices, j = i % kMaxChoices;
        if (j >= lengths[w]) continue;
        const uint64_t key = keys[w][j];
        int rank = 0;
#pragma unroll
        for (int o = 0; o < WAVES; ++o)
            for (int k = 0; k < n[o]; ++k) rank += keys[o][k] > key;
        if (rank < count) out(rank, key);
    }
    for (int i = all + threadIdx.x; i < count; i += WAVES * 64) out(i, (uint64_t)0);
}

// A row's results from its sums; every thread has them.
struct Finish {
    const LogprobArgs &a;
    int64_t row;
    float reference, log_sum;  // log_sum: NaN for a row that has no distribution
    __device__ __forceinline__ Finish(const LogprobArgs &a_, int64_t row_, const ExpSum &s) : a(a_), row(row_), reference(s.reference)
    {
        log_sum = s.sum > 0.0f ? logf(s.sum) : __builtin_nanf("");
    }
    __device__ __forceinline__ float value(float logit) const { return (logit - reference) * a.per_temperature - log_sum; }
    __device__ __forceinline__ void write(const ExpSum &s, float chosen) const  // one thread
    {
        if (a.logprobs) a.logprobs[row] = value(chosen);
        if (a.log_sums) a.log_sums[row] = fmaf(reference, a.per_temperature, log_sum);
        if (a.entropies) a.entropies[row] = log_sum - s.second / s.sum * 0.693147180559945309f;
    }
    __device__ __forceinline__ void alternative(int i, uint64_t key) const
    {
        const bool is = key != 0 && log_sum == log_sum;
        a.top_logprobs[row * a.count + i] = is ? value(of_ordered((uint32_t)(key >> 32))) : -__builtin_inff();
        a.top_tokens[row * a.count + i] = is ? (int32_t)~(uint32_t)key : -1;
    }
};

__device__ __forceinline__ bool is_padding(const LogprobArgs &a, int64_t row)
{
    return a.targets && (uint32_t)a.targets[row] >= (uint32_t)a.vocab;
}
template <int THREADS>
__device__ __forceinline__ void write_padding(const LogprobArgs &a, int64_t row)
{
    if (threadIdx.x == 0) {
        if (a.logprobs) a.logprobs[row] = 0.0f;
        if (a.log_sums) a.log_sums[row] = 0.0f;
        if (a.entropies) a.entropies[row] = 0.0f;
    }
    for (int i = threadIdx.x; i < a.count; i += THREADS) {
        a.top_logprobs[row * a.count + i] = -__builtin_inff();
        a.top_tokens[row * a.count + i] = -1;
    }
}

// A segment of a row to a workgroup; where a row has one only, that is all.
template <int TYPE, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(kThreads) void token_logprobs_kernel(LogprobArgs a)
{
    __shared__ uint64_t keys[TOP ? kWaves : 1][kListed];
    const int t = threadIdx.x;
    const int local = quotient((int)blockIdx.x, a.by_segments), segment = (int)blockIdx.x - local * a.segments;
    const int64_t row = a.first_row + local;
    if (is_padding(a, row)) {
        if (a.segments == 1) write_padding<kThreads>(a, row);
        return;
    }
    const Row<TYPE> x(a.logits, row * a.stride, a.vocab);
    const bool alone = a.segments == 1;
    float chosen = 0.0f;
    if (alone && t == 0 && a.targets) chosen = x.logit(a.targets[row]);
    ExpSum s;
    TopList list(keys[TOP ? t / 64 : 0], a.count);
    const int first = segment * a.segment_vectors;
    walk<TYPE, kThreads, 4>(x, first, alone ? x.vectors : min(first + a.segment_vectors, x.vectors), [&](const Logits<TYPE> &v, int j) {
        const float top = largest(v);
        add<ENTROPY ? 1 : 0>(s, v, top, a.c);
        if (TOP)
            list.offer<Logits<TYPE>::kCount, true>(top, [&](int e) { return v[e]; }, [&](int e) { return key_of(v[e], x.token(j) + e); });
    });
    s = join<ENTROPY, kThreads>(s, a.c);
    if (alone) {
        const Finish finish(a, row, s);
        if (t == 0) finish.write(s, chosen);
        if (TOP) ranked(keys, list, a.count, [&](int i, uint64_t key) { finish.alternative(i, key); });
    } else {
        if (t == 0) a.parts[blockIdx.x] = {s.reference, s.sum, s.second, 0.0f};
        if (TOP) ranked(keys, list, a.count, [&](int i, uint64_t key) { a.best[(int64_t)blockIdx.x * a.count + i] = key; });
    }
}

// A row to a workgroup: its segments' sums and best tokens as one.
template <int TYPE, bool TOP>
__global__ __launch_bounds__(kThreads) void token_logprobs_join_kernel(LogprobArgs a)
{
    __shared__ uint64_t keys[TOP ? kWaves : 1][kListed];
    const int t = threadIdx.x;
    const int64_t row = a.first_row + blockIdx.x;
    if (is_padding(a, row)) {
        write_padding<kThreads>(a, row);
        return;
    }
    float chosen = 0.0f;
    if (t == 0 && a.targets) chosen = Row<TYPE>(a.logits, row * a.stride, a.vocab).logit(a.targets[row]);
    const LogitsPart *parts = a.parts + (int64_t)blockIdx.x * a.segments;
    const ExpSum s = join<true, kThreads>(parts, a.segments, a.c);
    const Finish finish(a, row, s);
    if (t == 0) finish.write(s, chosen);
    if (TOP) {
        TopList list(keys[t / 64], a.count);
        const uint64_t *best = a.best + (int64_t)blockIdx.x * a.segments * a.count;
        const int all = a.segments * a.count;
        for (int i = 0; i < all; i += kThreads) {  // place by place, the best of all segments first
            const int k = i + t, place = k / a.segments;
            const uint64_t key = k < all ? best[(int64_t)(k - place * a.segments) * a.count + place] : 0;
            const float v = key ? of_ordered((uint32_t)(key >> 32)) : -__builtin_inff();
            list.offer<1, false>(v, [&](int) { return v; }, [&](int) { return key; });
        }
        ranked(keys, list, a.count, [&](int i, uint64_t key) { finish.alternative(i, key); });
    }
}

// A segment of a row's gradient to a workgroup.
template <int TYPE, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void token_logprobs_backward_kernel(LogprobGradientArgs a)
{
    const int t = threadIdx.x;
    const int local = quotient((int)blockIdx.x, a.by_segments), segment = (int)blockIdx.x - local * a.segments;
    const int64_t row = a.first_row + local;
    const Row<TYPE> x(a.logits, row * a.stride, a.vocab);
    const GradientRow<TYPE> to(a.gradient, row * a.gradient_stride, x);
    const int first = segment * a.segment_vectors, last = min(first + a.segment_vectors, x.vectors);
    const int target = a.targets ? a.targets[row] : -1;
    const float g = a.targets ? a.grad_logprobs[row] : 0.0f, h = ENTROPY ? a.grad_entropies[row] : 0.0f;
    if ((a.targets && (uint32_t)target >= (uint32_t)a.vocab) || (g == 0.0f && h == 0.0f)) {
        write_zeros<TYPE, kThreads>(to, first, last);
        return;
    }
    const float log_sum = a.log_sums[row], entropy = ENTROPY ? a.entropies[row] : 0.0f;
    const Saved saved(log_sum, a.temperature, a.c);
    // -g p - h p (ln p + entropy), over T
    const float flat = -(ENTROPY ? fmaf(h, entropy, g) : g) * a.per_temperature, tilted = -h * 0.693147180559945309f * a.per_temperature;
    const int at = target + x.skip;
    const bool here = t == 0 && target >= 0 && at >= first * Logits<TYPE>::kCount && at < last * Logits<TYPE>::kCount;
    float of_target = 0.0f;
    if (here) {
        const float e = fmaf(x.logit(target) - saved.reference, a.c, -saved.log), p = exp2_of(e);
        of_target = fmaf(g, a.per_temperature, p * (ENTROPY ? fmaf(tilted, fmaxf(e, kFarBelow), flat) : flat));
    }
    __shared__ float kept;  // the target's logit is read before its place is written: the value passes through here
    if (t == 0) kept = of_target;
    __syncthreads();
    write_gradient<TYPE, kThreads, 4, ENTROPY>(x, to, first, last, saved.reference, a.c, saved.log, flat, tilted);
    __syncthreads();
    if (here) to.store_one(kept, target);
}

}  // namespace

// Segments of a row: none where the rows alone fill the device, else enough to give every compute unit 4 workgroups, of at least 512 vectors.
LogitsCut logits_cut(int64_t rows, int32_t vocab, int32_t type)
{
    const int per_vector = type == QUAMBA_F32 ? 4 : 8;
    const int vectors = (vocab + 2 * per_vector - 2) / per_vector;  // the most that a row's address may make of it
    const int64_t want = (4 * compute_units() + rows - 1) / std::max<int64_t>(rows, 1);
    const int segments = (int)std::max<int64_t>(1, std::min<int64_t>({want, (vectors + 511) / 512, 256}));
    const int each = (vectors + segments - 1) / segments;
    return {(vectors + each - 1) / each, each};
}

namespace {

template <int TYPE>
void launch_rows(const LogprobArgs &a, int64_t rows, hipStream_t stream)
{
    const int grid = (int)(rows * a.segments);
    const auto kernel = a.count ? (a.entropies ? token_logprobs_kernel<TYPE, true, true> : token_logprobs_kernel<TYPE, false, true>)
                                : (a.entropies ? token_logprobs_kernel<TYPE, true, false> : token_logprobs_kernel<TYPE, false, false>);
    kernel<<<grid, kThreads, 0, stream>>>(a);
    if (a.segments == 1) return;
    const auto join_kernel = a.count ? token_logprobs_join_kernel<TYPE, true> : token_logprobs_join_kernel<TYPE, false>;
    join_kernel<<<(int)rows, kThreads, 0, stream>>>(a);
}

template <int TYPE>
void launch_gradient(const LogprobGradientArgs &a, int64_t rows, hipStream_t stream)
{
    const int grid = (int)(rows * a.segments);
    const auto kernel = a.grad_entropies ? token_logprobs_backward_kernel<TYPE, true> : token_logprobs_backward_kernel<TYPE, false>;
    kernel<<<grid, kThreads, 0, stream>>>(a);
}

}  // namespace

size_t token_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t count)
{
    size_t most = 0;  // over the types
    for (const int type : {QUAMBA_F32, QUAMBA_BF16}) {
        const int segments = logits_cut(rows, vocab, type).segments;
        if (segments > 1) most = std::max(most, (size_t)rows * segments * (sizeof(LogitsPart) + sizeof(uint64_t) * count));
    }
    return most;
}

hipError_t launch_token_logprobs(LogprobArgs a, void *workspace, hipStream_t stream)
{
    const LogitsCut cut = workspace ? logits_cut(a.rows, a.vocab, a.type) : LogitsCut{1, 0};
    a.segments = cut.segments;
    a.segment_vectors = cut.vectors;
    a.by_segments = divisor((uint32_t)cut.segments);
    a.parts = static_cast<LogitsPart *>(workspace);
    a.best = reinterpret_cast<uint64_t *>(a.parts + (cut.segments > 1 ? a.rows * cut.segments : 0));
    for (a.first_row = 0; a.first_row < a.rows; a.first_row += kRowsOfALaunch) {
        const int64_t rows = std::min(a.rows - a.first_row, kRowsOfALaunch);
        switch (a.type) {
            case QUAMBA_F32: launch_rows<QUAMBA_F32>(a, rows, stream); break;
            case QUAMBA_F16: launch_rows<QUAMBA_F16>(a, rows, stream); break;
            default: launch_rows<QUAMBA_BF16>(a, rows, stream); break;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_token_logprobs_backward(LogprobGradientArgs a, hipStream_t stream)
{
    const LogitsCut cut = logits_cut(a.rows, a.vocab, a.type);
    a.segments = cut.segments;
    a.segment_vectors = cut.vectors;
    a.by_segments = divisor((uint32_t)cut.segments);
    for (a.first_row = 0; a.first_row < a.rows; a.first_row += kRowsOfALaunch) {
        const int64_t rows = std::min(a.rows - a.first_row, kRowsOfALaunch);
        switch (a.type) {
            case QUAMBA_F32: launch_gradient<QUAMBA_F32>(a, rows, stream); break;
            case QUAMBA_F16: launch_gradient<QUAMBA_F16>(a, rows, stream); break;
            default: launch_gradient<QUAMBA_BF16>(a, rows, stream); break;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace quamba
