// Beam search: selection of the best candidates of all beams and categories of a group, and the reordering of what
// the surviving beams take along.
//   score(beam, c) = running[beam] + z_c [- log sum exp(z)],  z = scores[beam]
// Order: score, then lower beam, then higher z, then lower category.  Within a beam that is the order of z itself, so a row
// is first cut to its own best by (z, category), and only those are compared across beams, in 64 bits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "pc_internal.h"
#include "pc_rows.h"

namespace pc {

constexpr int kBeamThreads = 256;
constexpr double kNegInf64 = -__builtin_huge_val();

struct BeamDev {
    int32_t groups, beams, n_cats, n_out;
    const void *scores;
    int64_t ld;
    bool normalise;
    const float *running;
    const uint8_t *done;
    int32_t done_token;
};

// A float as an unsigned key of the same order; +0 and -0 are one value, a NaN counts as -inf.
__device__ inline uint32_t order_key(float v)
{
    v = v != v ? PC_NEG_INF_F : v + 0.0f;
    const uint32_t u = __float_as_uint(v);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ inline uint64_t candidate(float v, int c) { return (uint64_t)order_key(v) << 32 | (uint32_t)~c; }

// Running score of a beam: no number below +inf counts as -inf.
__device__ inline float running_score(const BeamDev &a, int64_t row)
{
    const float v = a.running ? a.running[row] : 0.0f;
    return v < __builtin_inff() ? v : PC_NEG_INF_F;
}

// ---- sorting across the lanes of a wave, best first ----
// Candidates of different beams: score, then lower beam, then the key of its row.
struct Cand {
    double score;
    uint64_t key;
    int32_t beam;
};
template <int J> __device__ inline uint64_t lane_xor(uint64_t v) { return (uint64_t)lane_xor32<J>((uint32_t)(v >> 32)) << 32 | lane_xor32<J>((uint32_t)v); }
__device__ inline bool better(float a, float b) { return a > b; }
__device__ inline bool better(uint64_t a, uint64_t b) { return a > b; }
__device__ inline bool better(const Cand &a, const Cand &b) { return a.score > b.score || (a.score == b.score && (a.beam < b.beam || (a.beam == b.beam && a.key > b.key))); }
// threadIdx.x in a register of its own: conditions on it are made where they are used, not kept for a whole kernel
__device__ inline uint32_t fresh_lane()
{
    uint32_t t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}
// Exchanges over J, J / 2 .. 1 lanes: of a lane and its partner the one whose bit J is clear keeps the better where `up`, the worse elsewhere.
// Keys are distinct, or equal in all that counts.
template <int J, typename V>
__device__ __forceinline__ V exchanges(const V &v, bool up)
{
    const V o = lane_xor<J>(v);
    const V r = better(o, v) == (((fresh_lane() & J) == 0) == up) ? o : v;
    if constexpr (J > 1) return exchanges<J / 2>(r, up);
    else return r;
}
template <int K = 2, typename V>
__device__ __forceinline__ V sort_lanes(const V &v)
{
    const V r = exchanges<K / 2>(v, K == 64 || (fresh_lane() & K) == 0);
    if constexpr (K < 64) return sort_lanes<K * 2>(r);
    else return r;
}
// The 64 best of two sorted lists; `other` holds the second one in reverse (lane i: its entry 63 - i).
template <typename V>
__device__ __forceinline__ V merge_lanes(const V &v, const V &other)
{
    const V r = better(other, v) ? other : v;
    return exchanges<32>(r, true);
}
// The same for candidates, in loops: a group's join runs each step once or twice, and code that long would mostly wait for itself to be fetched.
__device__ inline Cand lane_of(const Cand &v, int lane)
{
    return Cand{__shfl(v.score, lane), (uint64_t)__shfl((unsigned long long)v.key, lane), __shfl(v.beam, lane)};
}
__device__ inline Cand exchange_step(const Cand &v, int j, bool up)
{
    const int lane = threadIdx.x & 63;
    const Cand o = lane_of(v, lane ^ j);
    return better(o, v) == (((lane & j) == 0) == up) ? o : v;
}
__device__ inline Cand sort_candidates(Cand v)
{
#pragma unroll 1
    for (int kj = 0; kj < 21; ++kj) {                  // (k, j) = (2, 1), (4, 2), (4, 1), (8, 4) .. (64, 1)
        const int stage = kj < 1 ? 0 : kj < 3 ? 1 : kj < 6 ? 2 : kj < 10 ? 3 : kj < 15 ? 4 : 5, at = kj - stage * (stage + 1) / 2;
        const int k = 2 << stage;
        v = exchange_step(v, k >> (at + 1), k == 64 || (threadIdx.x & k) == 0);
    }
    return v;
}
__device__ inline Cand merge_candidates(const Cand &v, const Cand &other)
{
    Cand r = better(other, v) ? other : v;
#pragma unroll 1
    for (int j = 32; j > 0; j >>= 1) r = exchange_step(r, j, true);
    return r;
}
// n-th largest (n <= 64) of one value per lane of a wave, or per thread of the workgroup.  No NaN.
__device__ __forceinline__ float wave_nth(float v, int n) { return __shfl(sort_lanes(v), n - 1); }
__device__ __forceinline__ float block_nth(float v, int n, float (&lds)[kBeamThreads])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = sort_lanes(v);
    __syncthreads();
    lds[threadIdx.x] = v;
    __syncthreads();
#pragma unroll
    for (int w = 1; w < kBeamThreads / 64; ++w) v = merge_lanes(v, lds[(wave + w) % (kBeamThreads / 64) * 64 + 63 - lane]);
    return __shfl(v, n - 1);
}
// the next float up; above +inf: NaN, which nothing reaches
__device__ inline float next_above(float t) { return key_value(order_key(t) + 1); }

// ---- stage 1: the n best of a segment of a row, and its part of the log-normaliser ----
// A segment passes through registers once, four 16-byte packs a lane at a time, the next ones on their way.  The n-th largest of the first
// chunk's 256 thread maxima is a bound that at least n categories reach; later chunks count from just above it, for a category further
// back loses a tie.  Packs whose maximum reaches the bound (some n of a chunk) queue up in LDS by their place, and once they fill a wave
// their elements are read again, one a lane, and those that reach it go to the wave's list: looking at every element of such a chunk
// with a ballot each took 140 us where this takes 115 (256 x 16 x 50257 bf16).  A full list (rows in ascending order, ties) is cut to the n
// best, whose last is the new bound; many lanes with such packs raise it by the chunk's own maxima.  Waves do not wait for each other between the first
// bound and the end.  Bound by instructions in 16 bits (unpacking, maximum, exponential: 3.7 TB/s), by reading in 32 (the same rows 157 us, 5.2 TB/s;
// not past the caches 165).
// Five waves a SIMD: 115 us; four 120, six (spilling) 129.
constexpr int kBeamPacks = 4, kWaveList = 256, kQueue = 64 * (kBeamPacks + 1), kBeamWaves = kBeamThreads / 64;
template <typename T> constexpr int chunk_elements() { return kBeamThreads * kBeamPacks * Pack<T>::N; }
struct RowPart { float m; float pad; double sum; };    // reference and sum of exp(z - m) of a segment
// The log-normaliser: exponentials in fp32, added in fp32 within a lane's part of a chunk (16 or 32 of them) and in 64 bits from there on.  A wave's
// reference follows its maximum only where that is more than this above it: a factor in fp32 for each new maximum would be an error for each chunk of a
// row that rises slowly, this way an entry meets one for each 8 that the maximum comes to lie above it.
constexpr float kBeamSlack = 8.0f;

// A wave's list and its length.
struct WaveList {
    uint64_t *list;
    int count;
    // the 64 best in order, a lane each; the list becomes the first n of them
    __device__ __forceinline__ uint64_t cut(int n)
    {
        const int lane = threadIdx.x & 63;
        uint64_t v = sort_lanes(lane < count ? list[lane] : 0), nth = __shfl((unsigned long long)v, n - 1);
        for (int i = 64; i < count; i += 64) {
            uint64_t w = i + lane < count ? list[i + lane] : 0;
            if (!__any(w > nth)) continue;
            w = sort_lanes(w);
            v = merge_lanes(v, (uint64_t)__shfl((unsigned long long)w, 63 - lane));
            nth = __shfl((unsigned long long)v, n - 1);
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        count = min(count, n);
        if (lane < count) list[lane] = v;
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        return v;
    }
    __device__ inline void add(uint64_t key, bool on)   // room for 64
    {
        const uint64_t those = __ballot(on);
        if (on) list[count + __popcll(those & ((1ull << (threadIdx.x & 63)) - 1))] = key;
        count += __popcll(those);
    }
};

template <typename T>
__global__ __launch_bounds__(kBeamThreads, 5) void k_beam_rows(const BeamDev a, int32_t n_seg, int32_t seg_len, uint64_t *__restrict__ best,
                                                            RowPart *__restrict__ parts)
{
    constexpr int N = Pack<T>::N, ELEMS = kBeamPacks * N, CHUNK = chunk_elements<T>();
    __shared__ uint64_t lists[kBeamWaves][kWaveList];
    __shared__ int32_t queues[kBeamWaves][kQueue];
    __shared__ float nth_lds[kBeamThreads], wave_m[kBeamWaves];
    __shared__ double wave_sum[kBeamWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.n_out;
    const int64_t tasks = (int64_t)a.groups * a.beams * n_seg;
    for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
        const int64_t r = task / n_seg;
        if ((a.done && a.done[r]) || running_score(a, r) == PC_NEG_INF_F) continue;       // the join knows these beams' candidates
        // category c is element c + off of a grid of 16-byte packs; none before off is read
        const T *z = (const T *)a.scores + r * a.ld;
        const int off = elements_off(z);
        const T *grid = z - off;
        const uint32_t first = (uint32_t)(task % n_seg) * (uint32_t)seg_len, hi = min((uint32_t)off + (uint32_t)a.n_cats, first + (uint32_t)seg_len), lo = max((uint32_t)off, first);
        float m = PC_NEG_INF_F, t = PC_NEG_INF_F;      // m: reference of the wave's exponentials
        double sum = 0.0;
        bool fresh = false;                            // t is reached by n categories of this chunk or before, not above all of them
        WaveList mine{lists[wave], 0};
        int queued = 0;                                // packs of the wave's queue
        auto raise = [&]() __attribute__((always_inline)) {                           // the bound above the list's n-th
            const uint64_t nth = __shfl((unsigned long long)mine.cut(n), n - 1);
            const float bound = nth ? next_above(key_value((uint32_t)(nth >> 32))) : t;
            if (bound > t || bound != bound) { t = bound; fresh = false; }
        };
        Pack<T> ahead[kBeamPacks];
        auto index = [&](uint32_t base, int k) { return base + (uint32_t)(k * kBeamThreads + threadIdx.x) * N; };
        auto fetch = [&](uint32_t base) {               // whole packs
#pragma unroll
            for (int k = 0; k < kBeamPacks; ++k)
                if (index(base, k) >= lo && index(base, k) + N <= hi) ahead[k] = stream_pack((const T *)__builtin_assume_aligned(grid + index(base, k), 16));
        };
        fetch(first);
        for (uint32_t base = first; base < hi; base += CHUNK) {
            const bool inner = base >= lo && base + CHUNK <= hi;
            float v[ELEMS], tops[kBeamPacks], top = PC_NEG_INF_F;      // v: -inf outside [lo, hi); tops: no NaN
#pragma unroll
            for (int k = 0; k < kBeamPacks; ++k) {
                tops[k] = PC_NEG_INF_F;
                const uint32_t i = index(base, k);
                float x[N];
                unpack_f32(ahead[k], x);
                if (!inner && !(i >= lo && i + N <= hi)) {
#pragma unroll
                    for (int e = 0; e < N; ++e) x[e] = PC_NEG_INF_F;
                    if (i < hi && i + N > lo) {        // all its loads at once
                        T cut[N];
#pragma unroll
                        for (int e = 0; e < N; ++e) cut[e] = grid[min(max(i + e, lo), hi - 1)];
#pragma unroll
                        for (int e = 0; e < N; ++e) x[e] = i + e >= lo && i + e < hi ? to_f32(cut[e]) : PC_NEG_INF_F;
                    }
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    v[k * N + e] = x[e];
                    tops[k] = fmaxf(tops[k], x[e]);
                }
                top = fmaxf(top, tops[k]);
            }
            if (base + CHUNK < hi) fetch(base + CHUNK);
            if (a.normalise) {
                if (__any(top > m + kBeamSlack)) {
                    const float higher = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(wave_all(top, [](float x, float y) { return fmaxf(x, y); }))));
                    sum *= __builtin_amdgcn_exp2f((m - higher) * PC_LOG2E_F);
                    m = higher;
                }
                const float at = m == PC_NEG_INF_F ? 0.0f : m;
                float part = 0.0f;
#pragma unroll
                for (int k = 0; k < kBeamPacks; ++k)
#pragma unroll
                        for (int e = 0; e < N; ++e) part += __builtin_amdgcn_exp2f((v[k * N + e] - at) * PC_LOG2E_F);
                sum += part;
            }
            if (base == first) {
                t = block_nth(top, n, nth_lds);
                fresh = true;
            } else if (t == PC_NEG_INF_F || __popcll(__ballot(top >= t)) > 32) {
                const float bound = wave_nth(top, n);
                if (!(bound <= t)) { t = bound; fresh = true; }
            }
            const bool last = base + CHUNK >= hi;
            if (__any(top >= t) || last) {
#pragma unroll
                for (int k = 0; k < kBeamPacks; ++k) {
                    const uint64_t those = __ballot(tops[k] >= t);
                    if (!those) continue;
                    if (tops[k] >= t) queues[wave][queued + __popcll(those & ((1ull << lane) - 1))] = (int32_t)(index(base, k) / N);
                    queued += __popcll(those);
                }
                __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
                // the queue's elements, a lane each, to the list: as many as fill a wave, or all where the bound is about to leave them behind
                const bool all = fresh || last || t == PC_NEG_INF_F;
                int head = 0;
                for (; queued - head >= (all ? 1 : 64 / N); head += 64 / N) {
                    const int at = head + lane / N;
                    const uint32_t i = at < queued ? (uint32_t)queues[wave][at] * N + lane % N : hi;
                    const bool is = i >= lo && i < hi;
                    const float x = is ? to_f32(grid[i]) : 0.0f;
                    if (mine.count > kWaveList - 64) raise();
                    mine.add(candidate(x, (int)(i - off)), is && (x >= t || t == PC_NEG_INF_F));
                }
                queued = max(queued - head, 0);
                const int32_t rest = lane < queued ? queues[wave][head + lane] : 0;
                __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
                if (lane < queued) queues[wave][lane] = rest;
                if (fresh && t != PC_NEG_INF_F) t = next_above(t);
                else if (t == PC_NEG_INF_F && mine.count >= n) raise();
                fresh = false;
            }
        }
        uint64_t v = mine.cut(n);
        if (wave > 0) lists[wave][lane] = v;
        if (lane == 0) wave_m[wave] = m;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 1; w < kBeamWaves; ++w) v = merge_lanes(v, lists[w][63 - lane]);
            if (lane < n) best[task * n + lane] = v;
        }
        if (a.normalise) {
            float all = m;
            for (int w = 0; w < kBeamWaves; ++w) all = fmaxf(all, wave_m[w]);
            double total = sum * (m == PC_NEG_INF_F ? 1.0 : (double)exp2f((m - all) * PC_LOG2E_F));
            for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
            if (lane == 0) wave_sum[wave] = total;
            __syncthreads();
            if (threadIdx.x == 0) {
                total = 0.0;
                for (int w = 0; w < kBeamWaves; ++w) total += wave_sum[w];
                parts[task] = RowPart{all, 0.0f, total};
            }
        }
        __syncthreads();                               // LDS is read
    }
}

// ---- stage 2: a group's survivors from its rows' lists ----
// One workgroup a group.  The log-normalisers of its beams first, in 64 bits; then all entries of all lists, the first of every list before the
// second of any.  Bound by its chain of loads and comparisons (it moves a few KB): sorting the entries 64 at a time took 10 to 16 us.
constexpr int kJoinWaves = 16, kRanked = 256;
__global__ __launch_bounds__(64 * kJoinWaves) void k_beam_join(const BeamDev a, int32_t n_seg, const uint64_t *__restrict__ best,
                                                               const RowPart *__restrict__ parts, float *out_scores,
                                                               int32_t *__restrict__ parents, int32_t *__restrict__ tokens)
{
    __shared__ Cand lists[kJoinWaves][64];             // or the candidates that are ranked
    __shared__ double norms[PC_MAX_BEAMS], runs[PC_MAX_BEAMS];          // a running score of -inf: nothing but candidates of -inf
    __shared__ int32_t ended[PC_MAX_BEAMS], rank_of[kRanked], few;
    __shared__ float least, heads[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, n = a.n_out;
    const Cand none{kNegInf64, 0, PC_MAX_BEAMS};       // behind every candidate
    for (int64_t g = blockIdx.x; g < a.groups; g += gridDim.x) {
        const int64_t row0 = g * a.beams;
        const int n_lists = a.beams * n_seg, n_entries = n_lists * n;
        // entry e: rank e / n_lists of list e % n_lists (row and segment); read while the normalisers are made
        const int e0 = threadIdx.x;
        const uint64_t first = e0 < n_entries ? best[(row0 * n_seg + e0 % n_lists) * n + e0 / n_lists] : 0;
        for (int b = wave; b < a.beams; b += waves) {
            // everything is requested at once; the part of a beam that is dead or has ended was never written, and is not used
            const RowPart *p = parts + (row0 + b) * n_seg;
            const RowPart part = p[min(lane, n_seg - 1)];
            double run = (double)running_score(a, row0 + b), norm = 0.0;
            const bool done = a.done && a.done[row0 + b];
            if (a.normalise && !done && run != kNegInf64) {
                float m = lane < n_seg ? part.m : PC_NEG_INF_F;
                for (int i = lane + 64; i < n_seg; i += 64) m = fmaxf(m, p[i].m);
                for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
                auto term = [&](const RowPart &q) { return q.m == PC_NEG_INF_F ? q.sum : q.sum * exp((double)q.m - (double)m); };
                double sum = lane < n_seg ? term(part) : 0.0;
                for (int i = lane + 64; i < n_seg; i += 64) sum += term(p[i]);
                for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
                norm = (double)m + log(sum);
                if (!(fabs(norm) < 1e300)) run = kNegInf64;             // no finite number: m is a float
            }
            if (lane == 0) {
                norms[b] = norm;
                runs[b] = run;
                ended[b] = done && run != kNegInf64;
            }
        }
        __syncthreads();
        auto entry = [&](int e) {
            Cand c = none;
            if (e >= n_entries) return c;
            const int list = e % n_lists, rank = e / n_lists, b = list / n_seg, seg = list % n_seg;
            const double run = runs[b];
            if (run == kNegInf64 || ended[b]) {        // candidates of -inf in order, after the one of a finished beam: from the first segment
                const int token = !ended[b] ? rank : rank == 0 ? a.done_token : rank <= a.done_token ? rank - 1 : rank;
                const bool one = ended[b] && rank == 0;
                if (seg == 0 && rank < a.n_cats) c = Cand{one ? run : kNegInf64, candidate(one ? 0.0f : PC_NEG_INF_F, token), b};
            } else {
                const uint64_t key = e == e0 ? first : best[(row0 * n_seg + list) * n + rank];
                if (key) c = Cand{run + ((double)key_value((uint32_t)(key >> 32)) - norms[b]), key, b};
            }
            return c;
        };
        // The n-th best of the first 256 entries bounds the n-th of all from below (of more where that leaves it at -inf: most beams at rest);
        // what reaches it is mostly few enough to be ranked at once, each against all.
        Cand mine = entry(e0);
        float bound = sort_lanes(__double2float_rd(mine.score));
        heads[wave][lane] = bound;
        if (threadIdx.x == 0) few = 0;
        for (int i = threadIdx.x; i < kRanked; i += blockDim.x) rank_of[i] = 0;
        __syncthreads();
        if (wave == 0) {
#pragma unroll 1
            for (int w = 1; w < waves; ++w) {
                bound = merge_lanes(bound, heads[w][63 - lane]);
                if (w >= 3 && __shfl(bound, n - 1) > PC_NEG_INF_F) break;
            }
            if (lane == n - 1) least = bound;
        }
        __syncthreads();
        Cand *const some = lists[0];
        for (int e = e0; e < n_entries; e += 64 * waves) {
            if (e != e0) mine = entry(e);
            if (mine.beam < PC_MAX_BEAMS && mine.score >= (double)least) {
                const int at = atomicAdd(&few, 1);
                if (at < kRanked) some[at] = mine;
            }
        }
        __syncthreads();
        const int n_some = few;
        if (n_some <= kRanked) {
            // candidate i against every parts-th other
            const int parts = max(1, (int)blockDim.x / n_some), part = threadIdx.x / n_some;
            for (int i = part < parts ? threadIdx.x % n_some : n_some; i < n_some; i += parts > 1 ? n_some : blockDim.x) {
                const Cand c = some[i];
                int rank = 0;
                for (int j = parts > 1 ? part : 0; j < n_some; j += parts) rank += better(some[j], c);
                if (rank) atomicAdd(&rank_of[i], rank);
            }
            __syncthreads();
            for (int i = threadIdx.x; i < n_some; i += blockDim.x)
                if (rank_of[i] < n) {
                    const Cand c = some[i];
                    const int64_t at = g * n + rank_of[i];
                    out_scores[at] = (float)c.score;
                    parents[at] = c.beam;
                    tokens[at] = (int32_t)~(uint32_t)c.key;
                }
            __syncthreads();                           // LDS is read
            continue;
        }
        // Many ties, or beams at rest: 64 entries at a time to a wave, which sorts and merges what is better than the n-th best it has; last the
        // waves' lists, half of them at a time.
        __syncthreads();
        mine = none;
        Cand nth = none;
        for (int at = 0; at < n_entries; at += 64 * waves) {
            Cand c = entry(at + e0);
            if (!__any(better(c, nth))) continue;
            c = sort_candidates(c);
            mine = at == 0 ? c : merge_candidates(mine, lane_of(c, 63 - lane));
            nth = lane_of(mine, n - 1);
        }
        for (int half = waves; half > 1;) {
            const int keep = (half + 1) / 2;
            __syncthreads();
            if (wave >= keep && wave < half) lists[wave][lane] = mine;
            __syncthreads();
            if (wave + keep < half) mine = merge_candidates(mine, lists[wave + keep][63 - lane]);
            half = keep;
        }
        if (wave == 0 && lane < n) {
            out_scores[g * n + lane] = (float)mine.score;
            parents[g * n + lane] = mine.beam;
            tokens[g * n + lane] = (int32_t)~(uint32_t)mine.key;
        }
        __syncthreads();                               // LDS is read
    }
}

// A state's rows in units of the widest size that suits its addresses, strides and length; its tasks are workgroups: several rows, or
// part of one.
constexpr int kCopyUnits = 4;                          // a thread's units, all read before the first is written
struct CopyTask {
    const char *src;
    char *dst;
    int64_t src_stride, dst_stride, units;             // units of a row
    int32_t unit, rows, parts;                         // bytes of a unit; rows of a task (1 where a row has several parts); parts of a row
    int64_t tasks;
};
struct CopyTasks { CopyTask t[PC_MAX_STATES]; };

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename U>
__device__ inline void copy_units(const CopyTask &s, int64_t task, const int32_t *__restrict__ parents, int64_t rows, int32_t beams, int32_t n_out)
{
    // unit u of row r: with several rows a task, threads go along a row's units and then to the next row
    const int units = (int)min(s.units, (int64_t)256 * kCopyUnits);
    U held[kCopyUnits];
    int64_t to[kCopyUnits];
#pragma unroll
    for (int k = 0; k < kCopyUnits; ++k) {
        const int t = threadIdx.x + 256 * k;
        const int64_t r = s.parts > 1 ? task / s.parts : task * s.rows + t / units;
        const int64_t u = s.parts > 1 ? task % s.parts * (256 * kCopyUnits) + t : t % units;
        const bool on = r < rows && u < s.units && (s.parts > 1 || t < s.rows * units);
        const int32_t p = parents[on ? r : 0];
        const bool copied = on && p >= 0 && p < beams;
        to[k] = copied ? r * s.dst_stride + u * (int64_t)sizeof(U) : -1;
        held[k] = *reinterpret_cast<const U *>(s.src + (copied ? (r / n_out * beams + p) * s.src_stride + u * (int64_t)sizeof(U) : 0));
    }
#pragma unroll
    for (int k = 0; k < kCopyUnits; ++k)
        if (to[k] >= 0) *reinterpret_cast<U *>(s.dst + to[k]) = held[k];
}
__global__ __launch_bounds__(256) void k_beam_reorder(const CopyTasks states, const int32_t *__restrict__ parents, int64_t rows, int32_t beams, int32_t n_out)
{
    const CopyTask &s = states.t[blockIdx.y];
    for (int64_t task = blockIdx.x; task < s.tasks; task += gridDim.x) {
        if (s.unit == 16) copy_units<u32x4>(s, task, parents, rows, beams, n_out);
        else if (s.unit == 4) copy_units<uint32_t>(s, task, parents, rows, beams, n_out);
        else copy_units<uint8_t>(s, task, parents, rows, beams, n_out);
    }
}

static pc_status check_beam(const pc_beam *a)
{
    if (!a) return fail(PC_ERR_ARG, "NULL argument");
    if (a->groups < 0) return fail(PC_ERR_ARG, "groups must not be negative");
    if (a->beams < 1 || a->beams > PC_MAX_BEAMS) return fail(PC_ERR_ARG, "beams must be in 1 .. PC_MAX_BEAMS");
    if (a->n_cats < 1) return fail(PC_ERR_ARG, "n_cats must be positive");
    if (a->n_out < 1 || a->n_out > PC_MAX_BEAM_OUT) return fail(PC_ERR_ARG, "n_out must be in 1 .. PC_MAX_BEAM_OUT");
    if (a->n_out > (int64_t)a->beams * a->n_cats) return fail(PC_ERR_ARG, "n_out is larger than beams * n_cats");
    if ((int64_t)a->groups * a->beams > INT32_MAX) return fail(PC_ERR_TOO_LARGE, "more than 2^31 - 1 rows");
    if (!type_known(a->scores_type)) return fail(PC_ERR_ARG, "unknown element type");
    if (a->scores_ld < a->n_cats) return fail(PC_ERR_ARG, "scores_ld is smaller than n_cats");
    if (a->groups == 0) return PC_OK;
    if (!a->scores) return fail(PC_ERR_ARG, "NULL argument");
    if (a->done && (a->done_token < 0 || a->done_token >= a->n_cats)) return fail(PC_ERR_ARG, "done_token out of range");
    if (!aligned_to(a->scores, type_bytes(a->scores_type)) || !aligned_to(a->running, 4)) return fail(PC_ERR_ARG, "arrays must be aligned to their elements");
    return PC_OK;
}
// Segments of a row: enough workgroups for four a CU, but none shorter than a chunk.  (The offset of a row from its 16-byte boundary
// makes it up to seven elements longer.)
struct Segments { int32_t n, len; };
static Segments segments_of(const pc_beam *a)
{
    const int64_t chunk = a->scores_type == PC_F32 ? chunk_elements<float>() : chunk_elements<bf16_t>();
    const int64_t rows = (int64_t)a->groups * a->beams, len = (int64_t)a->n_cats + 7, chunks = (len + chunk - 1) / chunk;
    const int64_t most = (1 << 30) / chunk;            // chunks of a segment whose length is an int32
    const int64_t wanted = std::min(chunks, std::max(1024 / std::max<int64_t>(rows, 1), (chunks + most - 1) / most));
    const int64_t each = (chunks + wanted - 1) / std::max<int64_t>(wanted, 1);
    return Segments{(int32_t)((chunks + each - 1) / each), (int32_t)(each * chunk)};
}
static size_t best_bytes(const pc_beam *a) { return ((size_t)a->groups * a->beams * segments_of(a).n * a->n_out * 8 + 15) / 16 * 16; }

}  // namespace pc

using namespace pc;

extern "C" {

pc_status pc_beam_workspace_bytes(const pc_beam *a, size_t *bytes)
{
    const pc_status st = check_beam(a);
    if (st != PC_OK) return st;
    if (!bytes) return fail(PC_ERR_ARG, "NULL argument");
    *bytes = best_bytes(a) + (size_t)a->groups * a->beams * segments_of(a).n * sizeof(RowPart);
    return PC_OK;
}

pc_status pc_beam_select(const pc_beam *a, void *workspace, size_t workspace_bytes, float *out_scores, int32_t *parents, int32_t *tokens, void *stream)
{
    const pc_status st = check_beam(a);
    if (st != PC_OK || a->groups == 0) return st;
    if (!workspace || !out_scores || !parents || !tokens) return fail(PC_ERR_ARG, "NULL argument");
    if (!aligned_to(workspace, 16)) return fail(PC_ERR_ARG, "the workspace must be 16-byte aligned");
    if (!aligned_to(out_scores, 4) || !aligned_to(parents, 4) || !aligned_to(tokens, 4)) return fail(PC_ERR_ARG, "outputs must be 4-byte aligned");
    size_t need = 0;
    pc_beam_workspace_bytes(a, &need);
    if (workspace_bytes < need) return fail(PC_ERR_WORKSPACE, "workspace smaller than pc_beam_workspace_bytes");
    // groups write while others read; a group reads its own running scores before it writes
    const int64_t rows = (int64_t)a->groups * a->beams, out_bytes = (int64_t)a->groups * a->n_out * 4;
    const void *const outs[] = {out_scores, parents, tokens};
    for (int i = 0; i < 3; ++i) {
        const bool in_place = i == 0 && out_scores == a->running && a->n_out == a->beams;
        if (overlap(outs[i], out_bytes, a->scores, span_bytes(rows, a->scores_ld, a->n_cats, type_bytes(a->scores_type))) || (a->done && overlap(outs[i], out_bytes, a->done, rows)) ||
            (a->running && !in_place && overlap(outs[i], out_bytes, a->running, rows * 4)) || overlap(outs[i], out_bytes, outs[(i + 1) % 3], out_bytes))
            return fail(PC_ERR_ARG, "outputs overlap scores, running, done or each other");
    }
    const BeamDev dev{a->groups, a->beams, a->n_cats, a->n_out, a->scores, a->scores_ld, a->normalise != 0, a->running, a->done, a->done_token};
    const Segments seg = segments_of(a);
    uint64_t *best = (uint64_t *)workspace;
    RowPart *parts = (RowPart *)((char *)workspace + best_bytes(a));
    const hipStream_t s = (hipStream_t)stream;
    const unsigned tasks = (unsigned)std::min<int64_t>((int64_t)a->groups * a->beams * seg.n, 1 << 20);
    with_type(a->scores_type, [&](auto t) { hipLaunchKernelGGL((k_beam_rows<decltype(t)>), dim3(tasks), dim3(kBeamThreads), 0, s, dev, seg.n, seg.len, best, parts); });
    // a wave for each 64 entries of the lists and for each beam, up to sixteen
    const int64_t join_waves = std::min<int64_t>(std::max<int64_t>(((int64_t)a->beams * seg.n * a->n_out + 63) / 64, a->beams), kJoinWaves);
    hipLaunchKernelGGL(k_beam_join, dim3((unsigned)std::min(a->groups, 1 << 20)), dim3((unsigned)(64 * join_waves)), 0, s, dev, seg.n, best, parts, out_scores,
                       parents, tokens);
    return launched();
}

pc_status pc_beam_reorder(const pc_state *states, int32_t n_states, const int32_t *parents, int32_t groups, int32_t beams, int32_t n_out, void *stream)
{
    if (!states || n_states < 1 || n_states > PC_MAX_STATES) return fail(PC_ERR_ARG, "1 .. PC_MAX_STATES states");
    if (groups < 0 || beams < 1 || beams > PC_MAX_BEAMS || n_out < 1 || n_out > PC_MAX_BEAM_OUT) return fail(PC_ERR_ARG, "groups, beams or n_out out of range");
    const int64_t rows = (int64_t)groups * n_out, src_rows = (int64_t)groups * beams;
    if (rows > INT32_MAX || src_rows > INT32_MAX) return fail(PC_ERR_TOO_LARGE, "more than 2^31 - 1 rows");
    CopyTasks dev{};
    int64_t most = 1;
    struct Span { uintptr_t at, end; };
    Span span[2 * PC_MAX_STATES];
    for (int32_t i = 0; i < n_states; ++i) {
        const pc_state &s = states[i];
        if (s.row_bytes < 1 || s.src_stride < s.row_bytes || s.dst_stride < s.row_bytes) return fail(PC_ERR_ARG, "row_bytes must be positive, strides at least row_bytes");
        if (groups == 0) continue;
        if (!s.src || !s.dst) return fail(PC_ERR_ARG, "NULL argument");
        span[2 * i] = {(uintptr_t)s.src, (uintptr_t)s.src + (uintptr_t)((src_rows - 1) * s.src_stride + s.row_bytes)};
        span[2 * i + 1] = {(uintptr_t)s.dst, (uintptr_t)s.dst + (uintptr_t)((rows - 1) * s.dst_stride + s.row_bytes)};
        const uint64_t at = (uintptr_t)s.src | (uintptr_t)s.dst | (uint64_t)s.row_bytes | (uint64_t)s.src_stride | (uint64_t)s.dst_stride;
        const int32_t unit = at % 16 == 0 ? 16 : at % 4 == 0 ? 4 : 1;
        const int64_t units = s.row_bytes / unit, per = 256 * kCopyUnits, parts = (units + per - 1) / per, fit = parts > 1 ? 1 : per / units;
        if (parts > INT32_MAX) return fail(PC_ERR_TOO_LARGE, "a row of more than 2^31 - 1 parts");
        dev.t[i] = CopyTask{(const char *)s.src, (char *)s.dst, s.src_stride, s.dst_stride, units, unit, (int32_t)fit, (int32_t)parts,
                            parts > 1 ? rows * parts : (rows + fit - 1) / fit};
        most = std::max(most, dev.t[i].tasks);
    }
    if (groups == 0) return PC_OK;
    if (!parents) return fail(PC_ERR_ARG, "NULL argument");
    if (!aligned_to(parents, 4)) return fail(PC_ERR_ARG, "parents must be 4-byte aligned");
    for (int32_t i = 0; i < n_states; ++i)                                        // a dst against every src and the dst before it
        for (int32_t j = 0; j < 2 * n_states; ++j) {
            const Span &d = span[2 * i + 1], &o = span[j];
            if (j != 2 * i + 1 && d.at < o.end && o.at < d.end) return fail(PC_ERR_ARG, "dst overlaps a src or another dst");
        }
    hipLaunchKernelGGL(k_beam_reorder, dim3((unsigned)std::min<int64_t>(most, 1 << 20), (unsigned)n_states), dim3(256), 0, (hipStream_t)stream, dev, parents, rows,
                       beams, n_out);
    return launched();
}

}  // extern "C"
