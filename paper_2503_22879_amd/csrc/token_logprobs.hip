// Log probabilities of given tokens under rows of logits x at a temperature T, with the entropy and the most likely alternatives, and the
// gradient of the first two.
//
//   logprob = (x_t - m) / T - ln S,   S = sum_v exp((x_v - m) / T)       entropy = ln S - sum_v exp(e_v) e_v / S,   e_v = (x_v - m) / T
//   dx_v = (g ([v = t] - p_v) - h p_v (ln p_v + entropy)) / T
//
// One pass over a row makes the sum, the entropy's sum and what bounds the best tokens (logits.h).  Bound: HBM, the logits read once, and read
// and written once for the gradient (8192 rows of 128000 bf16 logits with 5 alternatives and the entropy 318 us, 6.2 TB/s; 2048 of 50021 alone 34 us, 5.6 TB/s;
// the gradient of 4096 of 128000 311 us, 6.5 TB/s); single rows are two to three times a launch (1 of 50021 with 8 alternatives 9.3 us, without 5.3).
#include <algorithm>

#include "logits.h"

namespace quamba {
namespace {

constexpr int64_t kRowsOfALaunch = (int64_t)1 << 22;
constexpr int kThreads = 256;
constexpr int kGradientVectors = 1;  // of a thread

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
template <int TYPE, int THREADS, bool ENTROPY, bool TOP, bool PAST>
__global__ __launch_bounds__(THREADS) void token_logprobs_kernel(LogprobArgs a)
{
    __shared__ TopKeys<TOP ? THREADS / 64 : 1> keys;
    const int t = threadIdx.x;
    const int local = quotient((int)blockIdx.x, a.by_segments), segment = (int)blockIdx.x - local * a.segments;
    const int64_t row = a.first_row + local;
    const bool alone = a.segments == 1;
    if (is_padding(a, row)) {
        if (alone) write_padding<THREADS>(a, row);
        return;
    }
    const Row<TYPE, PAST> x(a.logits, row * a.stride, a.vocab);
    float chosen = 0.0f;
    if (alone && t == 0 && a.targets) chosen = x.logit(a.targets[row]);
    Adder<ENTROPY ? 1 : 0> adder(a.c);
    const int first = segment * a.segment_vectors, last = alone ? x.vectors : min(first + a.segment_vectors, x.vectors);
    ExpSum s;
    const auto at_end = [&](const Logits<TYPE> &v, int) { adder.add(v); };
    if constexpr (TOP) {
        float tops[kTurns];
#pragma unroll
        for (int u = 0; u < kTurns; ++u) tops[u] = -__builtin_inff();
        walk<THREADS, kTurns>(
            x, first, last,
            [&](const Logits<TYPE> &v, int, int u) {
                adder.add(v);
                tops[u] = fmaxf(tops[u], largest(v));
            },
            at_end);
        s = join<ENTROPY, THREADS>(adder.result(), a.c);
        const Finish finish(a, row, s);
        best_tokens<THREADS>(keys, x, first, last, tops, a.count, [&](int i, uint64_t key) {
            if (alone)
                finish.alternative(i, key);
            else
                a.best[(int64_t)blockIdx.x * a.count + i] = key;
        });
    } else {
        walk<THREADS, kTurns>(x, first, last, [&](const Logits<TYPE> &v, int, int) { adder.add(v); }, at_end);
        s = join<ENTROPY, THREADS>(adder.result(), a.c);
    }
    if (t != 0) return;
    if (alone)
        Finish(a, row, s).write(s, chosen);
    else
        a.parts[blockIdx.x] = {s.reference, s.sum, s.second, 0.0f};
}

// A row to a workgroup: its segments' sums and best tokens as one.
template <int TYPE, bool TOP>
__global__ __launch_bounds__(kThreads) void token_logprobs_join_kernel(LogprobArgs a)
{
    __shared__ TopKeys<TOP ? kThreads / 64 : 1> keys;
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
    if constexpr (TOP) {
        TopList<kThreads / 64> list(keys, a.count);
        __syncthreads();
        const uint64_t *best = a.best + (int64_t)blockIdx.x * a.segments * a.count;
        const int all = a.segments * a.count;
        for (int i = 0; i < all; i += kThreads) {  // place by place, the best of all segments first
            const int k = i + t, place = quotient(k, a.by_segments);
            const uint64_t key = k < all ? best[(int64_t)(k - place * a.segments) * a.count + place] : 0;
            const float v = key ? of_ordered((uint32_t)(key >> 32)) : -__builtin_inff();
            list.template offer<1, false>(v, [&](int) { return v; }, [&](int) { return key; });
        }
        list.ranked([&](int i, uint64_t key) { finish.alternative(i, key); });
    }
}

// A segment of a row's gradient to a workgroup.
template <int TYPE, bool ENTROPY, bool PAST>
__global__ __launch_bounds__(kThreads) void token_logprobs_backward_kernel(LogprobGradientArgs a)
{
    constexpr int N = Logits<TYPE>::kCount;
    const int local = quotient((int)blockIdx.x, a.by_segments), segment = (int)blockIdx.x - local * a.segments;
    const int64_t row = a.first_row + local;
    const Row<TYPE, PAST> x(a.logits, row * a.stride, a.vocab);
    const GradientRow<TYPE, PAST> to(a.gradient, row * a.gradient_stride, x);
    const int first = segment * a.segment_vectors, last = min(first + a.segment_vectors, x.vectors);
    GradientSegment<kThreads, kGradientVectors, TYPE, PAST> segment_of(x, to, first, last);
    const int target = a.targets ? a.targets[row] : -(1 << 30);
    const float g = a.targets ? a.grad_logprobs[row] : 0.0f, h = ENTROPY ? a.grad_entropies[row] : 0.0f;
    if ((a.targets && (uint32_t)target >= (uint32_t)a.vocab) || (g == 0.0f && h == 0.0f)) {
        write_zeros<kThreads>(x, to, first, last);
        return;
    }
    segment_of.load();
    const float entropy = ENTROPY ? a.entropies[row] : 0.0f;
    const Saved saved(a.log_sums[row], a.temperature, a.c);
    // -g p - h p (ln p + entropy), over T: p (flat + tilted log2 p)
    const float flat = -(ENTROPY ? fmaf(h, entropy, g) : g) * a.per_temperature, tilted = -h * 0.693147180559945309f * a.per_temperature;
    segment_of.write([&](const Logits<TYPE> &v, int token, float(&d)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float e = fmaf(v[i] - saved.reference, a.c, -saved.log), p = exp2_of(e);
            d[i] = p * (ENTROPY ? fmaf(tilted, fmaxf(e, kFarBelow), flat) : flat);
        }
        const int at = target - token;
        if (at >= 0 && at < N) {
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = i == at ? fmaf(g, a.per_temperature, d[i]) : d[i];
        }
    });
}

}  // namespace

// How many vectors of 16 bytes a row is at most, whatever its address.
int logit_vectors(int32_t vocab, int32_t type)
{
    const int per_vector = type == QUAMBA_F32 ? 4 : 8;
    return (vocab + 2 * per_vector - 2) / per_vector;
}

// Rows of few vectors take a wave each: there is nothing to wait for in it, and four times the rows are on a compute unit (10000 rows of bf16: 256
// logits 11.8 -> 5.5 us, 2000 14.3 -> 10.4, 4000 18.4 -> 15.3, with 8 alternatives 29 -> 12.4, 31 -> 16.7, 36 -> 21.5; 100 rows of 2000 4.3 -> 4.3 and 5.6
// -> 6.0).
int wave_vectors(int64_t rows, int most) { return (int)std::min<int64_t>(most, std::max<int64_t>(128, rows / 4)); }

// A workgroup of 256 threads takes a row, but where rows are few and long.  1024 threads then take one on a compute unit of its own (256 rows of
// 200000 fp32 logits 44 -> 35 us, 128 of 128000 bf16 ones with 8 alternatives 17.8 -> 14.2; up to the borders below both take about as long).
// Where a row still takes longer than a second launch that joins segments, it is cut into these, by its logits and not its bytes (by 1024 threads and in
// segments: 1 row of 70000 bf16 logits 5.8 and 7.3 us, of 70564 fp32 ones 5.9 and 7.3; 13 rows of 100000 both 7.4, with 5 alternatives 11.6 and 10.8; of
// 166139 10.0 and 7.4, 15.2 and 11.8; 64 rows of 128000 with 20 alternatives 14.4 and 15.2).  Entropies and distances take half as much time again for a
// logit.  Without alternatives they are cut from 60000 logits on (1 row of 70000 bf16 ones with the entropy 7.0 and 5.5, the distance with 32 places and a rest 7.9
// and 6.2), with alternatives up to 64 rows instead of 32 (128000 logits, 20 alternatives, the entropy, in fp32 and bf16: 64 rows 17.3 and 16.5, 16.9 and
// 15.0; 65 rows 17.3 and 17.1, 16.9 and 16.2; 96 in fp32 17.6 and 19.4; 128 18.1 and 21.0, 17.3 and 18.6: more segments are more to join) and not earlier (35 rows of 48400
// bf16 logits with 5 and the entropy 10.1 and 10.9, 13 of 45848 9.9 and 10.3; but 6 of 70564 in fp32 with 1 11.1 and 9.4).  Segments are as many as fill the card, but with alternatives half of that and no shorter than 40 vectors for each of them, for the
// launch that joins them goes through all (4 rows of 150000 with 64 alternatives 21.6 and 16.5 us, 64 of 128000 in bf16 with 20 and the entropy 15.8 and 14.8).
// In front of a gradient's launch that joins them they cost no launch (held in registers and in segments, 32 places, a rest: 32 rows of 42000 bf16 logits 9.6 and 9.4,
// of 64000 12.0 and 10.2; 16 of 50000 fp32 ones 12.1, by 1024 threads, and 8.8; 64 rows of 64000 12.3 and 12.6, of 90000 16.2 and 14.1; fp32 ones of 61578 in 32 rows 14.0 and 11.7, in 33 14.1 and
// 11.7, in 64 14.5 and 15.0, in 128 17.9 and 20.9).
LogitsPlan logits_plan(int64_t rows, int32_t vocab, int32_t type, LogitsWork work, int32_t count, bool entropy, bool workspace)
{
    const int units = compute_units(), vectors = logit_vectors(vocab, type);
    const bool best = count > 0, more = entropy || work == LogitsWork::distance;
    const auto few_long = [&](int least_units, int least_vocab) { return rows * least_units <= units && vocab > least_vocab; };
    if (vectors <= wave_vectors(rows, 512)) return {64, 1, 0};
    if (workspace && (work == LogitsWork::step ? few_long(8, 40000) || few_long(4, 80000)
                                               : few_long(best && more ? 4 : 8, more && !best ? 60000 : 100000))) {
        const int least = std::max(512, 40 * count);
        const int segments = (int)std::min<int64_t>({((best ? 2 : 4) * units + rows - 1) / rows, (vectors + least - 1) / least, 256});
        const int each = (vectors + segments - 1) / segments;
        return {256, (vectors + each - 1) / each, each};
    }
    return {rows <= units && vectors > (best ? 8000 : 4000) ? 1024 : 256, 1, 0};
}

LogitsPlan gradient_plan(int32_t vocab, int32_t type, int vectors)
{
    const int all = logit_vectors(vocab, type);
    const int segments = (all + vectors - 1) / vectors, each = std::min(vectors, ((all + segments - 1) / segments + 63) / 64 * 64);
    return {kThreads, (all + each - 1) / each, each};
}

bool logits_past_caches(int64_t rows, int32_t vocab, int32_t type)
{
    return (double)rows * vocab * (type == QUAMBA_F32 ? 4 : 2) > 64 * 1048576.0;
}

namespace {

template <int TYPE, int THREADS, bool PAST>
void launch_first(const LogprobArgs &a, int grid, hipStream_t stream)
{
    const auto kernel = a.count ? (a.entropies ? token_logprobs_kernel<TYPE, THREADS, true, true, PAST> : token_logprobs_kernel<TYPE, THREADS, false, true, PAST>)
                                : (a.entropies ? token_logprobs_kernel<TYPE, THREADS, true, false, PAST> : token_logprobs_kernel<TYPE, THREADS, false, false, PAST>);
    kernel<<<grid, THREADS, 0, stream>>>(a);
}

template <int TYPE>
void launch_rows(const LogprobArgs &a, int threads, int64_t rows, bool past, hipStream_t stream)
{
    const int grid = (int)(rows * a.segments);
    if (threads == 1024)
        launch_first<TYPE, 1024, false>(a, grid, stream);
    else if (threads == 64)
        launch_first<TYPE, 64, false>(a, grid, stream);
    else if (past)
        launch_first<TYPE, 256, true>(a, grid, stream);
    else
        launch_first<TYPE, 256, false>(a, grid, stream);
    if (a.segments == 1) return;
    const auto join_kernel = a.count ? token_logprobs_join_kernel<TYPE, true> : token_logprobs_join_kernel<TYPE, false>;
    join_kernel<<<(int)rows, kThreads, 0, stream>>>(a);
}

template <int TYPE>
hipError_t launch(LogprobArgs a, void *workspace, hipStream_t stream)
{
    const LogitsPlan plan = logits_plan(a.rows, a.vocab, TYPE, LogitsWork::answers, a.count, a.entropies != nullptr, workspace != nullptr);
    a.segments = plan.segments;
    a.segment_vectors = plan.vectors;
    a.by_segments = divisor((uint32_t)plan.segments);
    a.parts = static_cast<LogitsPart *>(workspace);
    a.best = reinterpret_cast<uint64_t *>(a.parts + (plan.segments > 1 ? a.rows * plan.segments : 0));
    const bool past = logits_past_caches(a.rows, a.vocab, TYPE);
    for (a.first_row = 0; a.first_row < a.rows; a.first_row += kRowsOfALaunch) {
        launch_rows<TYPE>(a, plan.threads, std::min(a.rows - a.first_row, kRowsOfALaunch), past, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int TYPE, bool PAST>
hipError_t launch_gradient(LogprobGradientArgs a, hipStream_t stream)
{
    const LogitsPlan plan = gradient_plan(a.vocab, TYPE, kThreads * kGradientVectors);
    a.segments = plan.segments;
    a.segment_vectors = plan.vectors;
    a.by_segments = divisor((uint32_t)plan.segments);
    const auto kernel = a.grad_entropies ? token_logprobs_backward_kernel<TYPE, true, PAST> : token_logprobs_backward_kernel<TYPE, false, PAST>;
    const int64_t most = kRowsOfALaunch / plan.segments;
    for (a.first_row = 0; a.first_row < a.rows; a.first_row += most) {
        kernel<<<(int)(std::min(a.rows - a.first_row, most) * plan.segments), kThreads, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int TYPE>
hipError_t launch_gradient(const LogprobGradientArgs &a, hipStream_t stream)
{
    return logits_past_caches(a.rows, a.vocab, TYPE) ? launch_gradient<TYPE, true>(a, stream) : launch_gradient<TYPE, false>(a, stream);
}

}  // namespace

size_t token_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t count)
{
    size_t most = 0;  // over the types, with entropies and without
    for (const int type : {QUAMBA_F32, QUAMBA_BF16})
        for (const bool entropy : {false, true}) {
            const int segments = logits_plan(rows, vocab, type, LogitsWork::answers, count, entropy, true).segments;
            if (segments > 1) most = std::max(most, (size_t)rows * segments * (sizeof(LogitsPart) + sizeof(uint64_t) * count));
        }
    return most;
}

hipError_t launch_token_logprobs(const LogprobArgs &a, void *workspace, hipStream_t stream)
{
    switch (a.type) {
        case QUAMBA_F32: return launch<QUAMBA_F32>(a, workspace, stream);
        case QUAMBA_F16: return launch<QUAMBA_F16>(a, workspace, stream);
        default: return launch<QUAMBA_BF16>(a, workspace, stream);
    }
}

hipError_t launch_token_logprobs_backward(const LogprobGradientArgs &a, hipStream_t stream)
{
    switch (a.type) {
        case QUAMBA_F32: return launch_gradient<QUAMBA_F32>(a, stream);
        case QUAMBA_F16: return launch_gradient<QUAMBA_F16>(a, stream);
        default: return launch_gradient<QUAMBA_BF16>(a, stream);
    }
}

}  // namespace quamba
