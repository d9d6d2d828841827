// Beam search: the best continuations of every sequence over its beams and the vocabulary, and the move of the cached states
// behind them.
//
//   value(k, v) = score_k + ((x_kv - max_k) - log sum_u exp(x_ku - max_k))
//
// Equal values go by rising beam, and in a beam, whose logits may differ where their values round to one number, by falling logit and
// rising token: the order in which a piece keeps its best, so that the pieces' borders decide nothing.
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
constexpr int kJoined = 1024;    // candidates of a round of the second launch

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

// A key's uppermost 32 bits, an ordered float, decide first; 0 is no candidate.
typedef unsigned __int128 uint128_t;
__device__ __forceinline__ uint32_t upper(uint64_t key) { return (uint32_t)(key >> 32); }
__device__ __forceinline__ uint32_t upper(uint128_t key) { return (uint32_t)(key >> 96); }
__device__ __forceinline__ uint64_t from_lane(uint64_t key, int d) { return (uint64_t)__shfl_xor((long long)key, d, 64); }
__device__ __forceinline__ uint128_t from_lane(uint128_t key, int d)
{
    return (uint128_t)from_lane((uint64_t)(key >> 64), d) << 64 | from_lane((uint64_t)key, d);
}

template <typename K>
struct Chooser {
    K gathered[kGathered];
    K wave_best[2][kWaves];
    uint32_t tops[kThreads];
    int n;
};

// A bound that at least `count` of the threads' tops reach, where so many are above 0, and few more: the largest of those whose lower
// 32 - BITS bits are 0.  Bit by bit, by every wave for itself.
template <int BITS, typename K>
__device__ __forceinline__ uint32_t bound_of(Chooser<K> &c, int count, uint32_t top)
{
    c.tops[threadIdx.x] = top;
    if (threadIdx.x == 0) c.n = 0;
    __syncthreads();
    uint32_t mine[kWaves], bound = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mine[w] = c.tops[w * 64 + (threadIdx.x & 63)];
#pragma unroll
    for (int bit = 31; bit >= 32 - BITS; --bit) {
        const uint32_t higher = bound | 1u << bit;
        int n = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[w] >= higher));
        bound = n >= count ? higher : bound;
    }
    return max(bound, 1u);
}

// The `count` largest of the workgroup's keys, key(e) for e < E in every thread, 0 for none and otherwise all different: out[0 ..
// count - 1], largest first, 0 where there are no more.  `top` is the upper() of the thread's largest key, and from(bound) gives
// the test, for e, whether key(e)'s upper() is at least `bound`.  `out` is written by some threads; the caller waits before
// it is read elsewhere, and before it calls again.
//
// `count` threads have a key at least as large as the count-th largest of the threads' own largest ones, so nothing below that
// is among the best: what is left is mostly little more than `count` keys, which are ranked by counting.  The bound is sought in
// the uppermost BITS of a key: 16 for logits (the sign, the exponent and 7 bits more: the last bits would spare few keys), 20 for values, which
// share their first bits where a score is low (32 x 8 beams of 128000, 16 choices, scores of -1000: 56 us with 16, 35 with 20).  Where
// the best keys lie in a few threads (the frequent tokens of a vocabulary side by side) more are left; as long as they are more than
// threads, they are dealt out to all of them and bounded again.
template <int E, int BITS, typename K, typename From, typename Key, typename Out>
__device__ __forceinline__ void choose(Chooser<K> &c, int count, uint32_t top, const From &from, const Key &key, const Out &out)
{
    const int t = threadIdx.x, lane = t & 63;
    const uint32_t bound = bound_of<BITS>(c, count, top);
    if (top >= bound) {
        const auto candidate = from(bound);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (candidate(e)) {
                const int at = atomicAdd(&c.n, 1);
                if (at < kGathered) c.gathered[at] = key(e);
            }
    }
    __syncthreads();
    int n = c.n;
    if (n <= kGathered) {
        for (int before = kGathered + 1; n > kThreads && n < before;) {
            K mine[kGathered / kThreads];
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < kGathered / kThreads; ++i) {
                mine[i] = i * kThreads + t < n ? c.gathered[i * kThreads + t] : K(0);
                most = max(most, upper(mine[i]));
            }
            __syncthreads();  // all know n
            const uint32_t least = bound_of<32>(c, count, most);
#pragma unroll
            for (int i = 0; i < kGathered / kThreads; ++i)
                if (upper(mine[i]) >= least) c.gathered[atomicAdd(&c.n, 1)] = mine[i];
            __syncthreads();
            before = n;
            n = c.n;
        }
        for (int i = t; i < n; i += kThreads) {
            const K k = c.gathered[i];
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < n; ++j) rank += c.gathered[j] > k;
            if (rank < count) out(rank, k);
        }
        for (int i = n + t; i < count; i += kThreads) out(i, K(0));
    } else {  // many equal ones: one after the other
        K last = ~K(0);
        for (int i = 0; i < count; ++i) {
            K best = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const K k = key(e);
                if (k < last && k > best) best = k;
            }
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                const K o = from_lane(best, d);
                best = o > best ? o : best;
            }
            if (lane == 0) c.wave_best[i & 1][t / 64] = best;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) best = c.wave_best[i & 1][w] > best ? c.wave_best[i & 1][w] : best;
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
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = TYPE == QUAMBA_F32 ? 0xff800000u : TYPE == QUAMBA_BF16 ? 0xff80ff80u : 0xfc00fc00u;
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

// A piece of 256 E logits of a row to a workgroup.
template <int TYPE, int E>
__global__ __launch_bounds__(kThreads) void beam_pieces_kernel(SelectArgs a, int pieces, Divisor by_pieces, uint64_t *best, Piece *piece)
{
    constexpr int kVec = Logits<TYPE>::kCount, VECTORS = E / kVec, kPiece = kThreads * E;
    __shared__ Chooser<uint64_t> chooser;
    __shared__ float wave_f[2][kWaves];
    const int t = threadIdx.x, row = quotient((int)blockIdx.x, by_pieces), first = ((int)blockIdx.x - row * pieces) * kPiece;
    if (!offers(a, row) || (a.finished && a.finished[row])) return;  // the second launch does not read it
    const char *p = static_cast<const char *>(a.logits) + ((int64_t)row * a.stride + first) * Logits<TYPE>::kBytes + t * 16;
    Logits<TYPE> x[VECTORS];
    if (first + kPiece <= a.vocab) {
#pragma unroll
        for (int v = 0; v < VECTORS; ++v) x[v].load(p + v * kThreads * 16);
    } else {
#pragma unroll
        for (int v = 0; v < VECTORS; ++v) x[v].load(p + v * kThreads * 16, a.vocab - first - (v * kThreads + t) * kVec);
    }
    auto logit = [&](int e) { return x[e / kVec][e % kVec]; };
    auto token = [&](int e) { return first + (e / kVec * kThreads + t) * kVec + e % kVec; };
    float mine = -__builtin_inff();  // past a NaN, which the sum shows
#pragma unroll
    for (int e = 0; e < E; ++e) mine = fmaxf(mine, logit(e));
    float top = wave_max(mine);
    if (t % 64 == 0) wave_f[0][t / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wave_f[0][0], wave_f[0][1]), fmaxf(wave_f[0][2], wave_f[0][3]));
    const float against = top > -__builtin_inff() ? top : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) sum += __expf(logit(e) - against);
    sum = group_sum<64>(sum);
    if (t % 64 == 0) wave_f[1][t / 64] = sum;
    uint64_t *to = best + (int64_t)blockIdx.x * a.count;
    choose<E, 16>(
        chooser, a.count, mine > -__builtin_inff() ? ordered(mine + 0.0f) : 0u,  // -0 is 0
        [&](uint32_t bound) {
            const float least = fmaxf(of_ordered(bound), -__FLT_MAX__);
            return [logit, least](int e) { return logit(e) >= least; };
        },
        [&](int e) {
            const float v = logit(e);
            return v > -__builtin_inff() ? (uint64_t)ordered(v + 0.0f) << 32 | (uint32_t)~token(e) : (uint64_t)0;
        },
        [&](int i, uint64_t k) { to[i] = k; });
    if (t == 0) {
        const float total = (wave_f[1][0] + wave_f[1][1]) + (wave_f[1][2] + wave_f[1][3]);
        piece[blockIdx.x] = {top, top < __builtin_inff() ? total : __builtin_nanf("")};
    }
}

template <int CTRL>
__device__ __forceinline__ float row_step_max(float v) { return fmaxf(v, dpp_move<CTRL>(v)); }
__device__ __forceinline__ float row_max(float v)  // of 16 lanes
{
    return row_step_max<0x140>(row_step_max<0x141>(row_step_max<0x4E>(row_step_max<0xB1>(v))));
}

// A workgroup to a sequence: 16 lanes join a beam's pieces, then all take the best of the pieces' best.  These are gone through place by
// place, the first ones of all pieces, then the second ones: each piece's fall, so there are no better ones left once a place of every
// piece brought none, mostly after the first round (1 sequence of 16 beams, 200000 logits each, 32 choices: 112 us in the order of the
// pieces with pieces of 2048 logits, 17 so with 8192).  Where one round holds them all, they are taken as they lie.
__global__ __launch_bounds__(kThreads) void beam_join_kernel(SelectArgs a, int pieces, int places, int lists, int per_beam, Divisor by_place,
                                                             Divisor by_beam, const uint64_t *best, const Piece *piece)
{
    constexpr int E = kJoined / kThreads;
    __shared__ Chooser<uint128_t> chooser;
    __shared__ float score[kMaxBeams], row_top[kMaxBeams], row_log[kMaxBeams];
    __shared__ uint8_t kind[kMaxBeams];  // 0: offers nothing, 1: its pieces' tokens, 2: finished
    __shared__ uint128_t list[kMaxChoices];
    const int t = threadIdx.x, b = blockIdx.x;
    const int all = lists * places;
    const uint64_t *candidates = best + (int64_t)b * all;
    auto candidate = [&](int i) {
        const int place = quotient(i, by_place);
        return candidates[(i - place * lists) * places + place];
    };
    uint64_t c[E];
    if (places == 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) c[e] = candidates[min(e * kThreads + t, all - 1)];
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) c[e] = candidate(min(e * kThreads + t, all - 1));
    }
    for (int k = t / 16; k < a.beams; k += kThreads / 16) {
        const int row = b * a.beams + k;
        const Piece *p = piece + (int64_t)row * pieces;
        const bool valid = offers(a, row), done = a.finished && a.finished[row];
        float m = -__builtin_inff(), s = 0.0f;
        for (int i = t % 16; i < pieces; i += 16) m = fmaxf(m, p[i].max);
        m = row_max(m);
        const float against = m > -__builtin_inff() ? m : 0.0f;
        for (int i = t % 16; i < pieces; i += 16) s += p[i].sum * __expf(p[i].max - against);
        s = group_sum<16>(s);
        if (t % 16 == 0) {
            score[k] = a.scores[row];
            row_top[k] = m;
            row_log[k] = logf(s);
            kind[k] = !valid ? 0 : done ? 2 : s > 0.0f && m < __builtin_inff() ? 1 : 0;
        }
    }
    for (int i = t; i < kMaxChoices; i += kThreads) list[i] = 0;
    __syncthreads();
    int quiet = 0;  // candidates since the last one that was among the best
    for (int first = 0; first < all && quiet < lists; first += kThreads * E) {
        uint128_t key[E + 1];  // value, complement of the beam, logit, complement of the token
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            key[e] = 0;
            const int i = first + e * kThreads + t;
            if (i < all) {
                const int from = places == 1 ? i : i - quotient(i, by_place) * lists, k = quotient(from, by_beam);
                uint64_t in_beam = c[e];
                float v = -__builtin_inff();
                if (kind[k] == 1) {
                    if (c[e]) v = score[k] + ((of_ordered((uint32_t)(c[e] >> 32)) - row_top[k]) - row_log[k]);
                } else if (kind[k] == 2 && i == k * per_beam) {
                    in_beam = (uint32_t)~a.pad;
                    v = score[k];
                }
                if (v > -__builtin_inff())
                    key[e] = (uint128_t)((uint64_t)ordered(v + 0.0f) << 32 | (uint32_t)~k) << 64 | in_beam;
                const int64_t next = (int64_t)i + kThreads * E;
                if (next < all) c[e] = candidate((int)next);
            }
            top = max(top, upper(key[e]));
        }
        if (first && !__syncthreads_or(top >= max(upper(list[a.count - 1]), 1u))) {
            quiet += kThreads * E;
            continue;
        }
        quiet = 0;
        key[E] = t < kMaxChoices ? list[t] : uint128_t(0);
        top = max(top, upper(key[E]));
        __syncthreads();
        choose<E + 1, 20>(
            chooser, a.count, top, [&](uint32_t bound) { return [&key, bound](int e) { return upper(key[e]) >= bound; }; },
            [&](int e) { return key[e]; }, [&](int i, uint128_t k) { list[i] = k; });
        __syncthreads();
    }
    for (int i = t; i < a.count; i += kThreads) {
        const uint128_t chosen = list[i];
        const int64_t o = (int64_t)b * a.count + i;
        a.out_scores[o] = chosen ? of_ordered(upper(chosen)) : -__builtin_inff();
        a.out_parents[o] = chosen ? (int32_t)~(uint32_t)(chosen >> 64) : i % a.beams;
        a.out_tokens[o] = chosen ? (int32_t)~(uint32_t)chosen : a.pad;
    }
}

// Logits of a piece for each of its 256 threads: 16 where 32 leave most of the device without a piece (1 x 4 beams of 50021: 9.8 us with 16,
// 10.8 with 32; 8 x 8 of 50021: 13.7 and 13.2; 1 x 16 of 200000, 32 choices: 19.2 and 16.5; 32 x 8 of 128000: 33.7 and 35.3; pieces of 8 gain nothing
// on small ones).
int piece_values(int64_t rows, int32_t vocab)
{
    return rows * ((vocab + kThreads * 32 - 1) / (kThreads * 32)) < compute_units() / 2 ? 16 : 32;
}

int64_t piece_count(int32_t vocab, int e) { return ((int64_t)vocab + kThreads * e - 1) / (kThreads * e); }

template <int TYPE>
void launch_pieces(const SelectArgs &a, int e, int pieces, uint64_t *best, Piece *piece, hipStream_t stream)
{
    const int grid = a.batch * a.beams * pieces;
    const Divisor d = divisor((uint32_t)pieces);
    if (e == 16)
        beam_pieces_kernel<TYPE, 16><<<grid, kThreads, 0, stream>>>(a, pieces, d, best, piece);
    else
        beam_pieces_kernel<TYPE, 32><<<grid, kThreads, 0, stream>>>(a, pieces, d, best, piece);
}

// ---- the caches ----

constexpr int kCaches = 64;  // of a launch, a lane's each
struct ReorderArgs {
    const int32_t *parents;
    int32_t batch, beams, n;
    int32_t first[kCaches];  // workgroup of a sequence with which a cache begins
    quamba_beam_cache_t cache[kCaches];
};

// Bytes that a thread moves of every beam: 16, fewer for many beams, so that they fit 64 registers.  With twice as many for more than 16 beams:
// 32 beams of 80 MiB in all 18.96 -> 19.28 us, 640 MiB 206 -> 204; 64 beams of 160 MiB 41.0 -> 40.1, 1280 MiB 459 -> 421.
constexpr int move_bytes(int beams) { return beams <= 16 ? 16 : 256 / beams; }

// The parents of a sequence's beams, a byte each in scalar registers.
template <int BEAMS>
struct Parents {
    uint32_t four[(BEAMS + 3) / 4];
    __device__ __forceinline__ int operator[](int k) const { return (int)(four[k / 4] >> k % 4 * 8 & 0xffu); }
};

// Beams K and above: every load stands before every store.
template <int K, int BEAMS, typename Vec, bool PAST>
__device__ __forceinline__ void move_beams(char *base, int64_t bytes, const Parents<BEAMS> &parents, uint64_t &moved)
{
    Vec v;
    if (moved >> K & 1) {
        const Vec *from = reinterpret_cast<const Vec *>(base + parents[K] * bytes);
        v = PAST ? __builtin_nontemporal_load(from) : *from;
    }
    if constexpr (K + 1 < BEAMS)
        move_beams<K + 1, BEAMS, Vec, PAST>(base, bytes, parents, moved);
    else  // the same conditions again, but not to the compiler, which would make a path of its own for each set of beams
        asm volatile("" : "+s"(moved));
    if (moved >> K & 1) {
        Vec *to = reinterpret_cast<Vec *>(base + K * bytes);
        if (PAST)
            __builtin_nontemporal_store(v, to);
        else
            *to = v;
    }
}

// A workgroup moves one slice of every beam of a sequence: all loads stand before the stores, and no other thread touches the
// bytes, so the move is in place whatever the order of the beams.  BEAMS: at least as many as there are.  PAST: the bytes are not to stay in
// a cache.  A wave to a workgroup: 4 layers of 32 x 8 beams of 8-bit states, past the caches, take 281 us so (5.85 TB/s), and 299 us in
// workgroups of 256; through the caches 310 and 332.
constexpr int kMovers = 64;
template <int BEAMS, bool PAST>
__global__ __launch_bounds__(kMovers) void beam_reorder_kernel(ReorderArgs a)
{
    constexpr int kBytes = move_bytes(BEAMS);
    typedef uint32_t Vec __attribute__((ext_vector_type(kBytes / 4), aligned(1)));  // caches may lie at any address
    const int b = blockIdx.y;
    // lane k knows beam k's parent
    const int lane = threadIdx.x, parent = a.parents[(int64_t)b * a.beams + min(lane, a.beams - 1)];
    const bool moves = lane < a.beams && (uint32_t)parent < (uint32_t)a.beams && parent != lane;
    uint64_t moved = __builtin_amdgcn_ballot_w64(moves);
    // read here, where every lane is active: a lane's registers are not its own any more behind a branch that it does not take
    Parents<BEAMS> parents;
#pragma unroll
    for (int k = 0; k < BEAMS; ++k) {
        const uint32_t p = (uint32_t)__builtin_amdgcn_readlane(parent, k) & 0xffu;
        parents.four[k / 4] = k % 4 ? parents.four[k / 4] | p << k % 4 * 8 : p;
    }
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < a.n && (int)blockIdx.x >= a.first[lane])) - 1;
    const int64_t bytes = a.cache[c].bytes, at = ((int64_t)((int)blockIdx.x - a.first[c]) * kMovers + threadIdx.x) * kBytes;
    if (at >= bytes) return;
    char *base = static_cast<char *>(a.cache[c].data) + (int64_t)b * a.beams * bytes + at;
    if (at + kBytes <= bytes) {
        move_beams<0, BEAMS, Vec, PAST>(base, bytes, parents, moved);
    } else {
#pragma unroll 1
        for (int i = 0; at + i < bytes; ++i) {  // the last bytes one by one
            uint64_t m = moved;
            move_beams<0, BEAMS, uint8_t, false>(base + i, bytes, parents, m);
        }
    }
}

template <int BEAMS>
void launch_slices(const ReorderArgs &a, int slices, bool past, hipStream_t stream)
{
    if (past)
        beam_reorder_kernel<BEAMS, true><<<dim3(slices, a.batch), kMovers, 0, stream>>>(a);
    else
        beam_reorder_kernel<BEAMS, false><<<dim3(slices, a.batch), kMovers, 0, stream>>>(a);
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
    const bool one_round = a.beams * pieces * a.count <= kJoined;
    const int places = one_round ? 1 : a.count, per_beam = one_round ? pieces * a.count : pieces, lists = a.beams * per_beam;
    beam_join_kernel<<<a.batch, kThreads, 0, stream>>>(a, pieces, places, lists, per_beam, divisor((uint32_t)lists), divisor((uint32_t)per_beam), best, piece);
    return hipGetLastError();
}

hipError_t launch_beam_reorder(int32_t batch, int32_t beams, const int32_t *parents, int32_t n, const quamba_beam_cache_t *caches,
                               hipStream_t stream)
{
    // launches of up to kCaches caches, as many slices as the longest cache has (2^25 at most), and 65535 sequences
    if (beams == 1) return hipSuccess;
    const auto launch = beams <= 2 ? launch_slices<2> : beams <= 4 ? launch_slices<4> : beams <= 8 ? launch_slices<8>
                      : beams <= 16 ? launch_slices<16> : beams <= 32 ? launch_slices<32> : launch_slices<64>;
    const int64_t slice = kMovers * (beams <= 16 ? move_bytes(16) : beams <= 32 ? move_bytes(32) : move_bytes(64));
    const int64_t most = kMaxCacheBytes / slice;
    // What fits the last cache (256 MiB) is left there for the step that reads the states next.  Layers of 4 beams in fp32, through the caches
    // and past them: 72 MiB 16.5 and 19.5 us, 216 MiB 36 and 52, 288 MiB 64 and 68, 432 MiB 120 and 113, 1152 MiB 319 and 299; 8 beams in 8
    // bits: 256 MiB 50 and 75, 384 MiB 104 both, 1024 MiB 310 and 293.
    double bytes = 0.0;
    for (int32_t i = 0; i < n; ++i) bytes += (double)caches[i].bytes * beams * batch;
    const bool past = bytes > 256.0 * 1024 * 1024;
    for (int32_t s0 = 0; s0 < batch; s0 += kMaxGridY) {
        const int sequences = std::min(batch - s0, kMaxGridY);
        ReorderArgs a;
        a.parents = parents + (int64_t)s0 * beams;
        a.batch = sequences;
        a.beams = beams;
        a.n = 0;
        int64_t slices = 0;
        auto flush = [&] {
            if (a.n) launch(a, (int)slices, past, stream);
            a.n = 0;
            slices = 0;
            return hipGetLastError();
        };
        for (int32_t i = 0; i < n; ++i) {
            const int64_t need = (caches[i].bytes + slice - 1) / slice;
            if (!need) continue;
            if (a.n == kCaches || slices + need > most) {
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
