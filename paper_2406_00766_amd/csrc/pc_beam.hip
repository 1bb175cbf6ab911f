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
// Candidates of different beams: score, then lower `place` (beam, then rank within the beam).
struct Cand {
    double score;
    uint32_t place;
    int32_t token;
};
constexpr uint32_t kNoPlace = ~0u;
__device__ inline float lane_xor(float v, int j) { return __shfl_xor(v, j); }
__device__ inline uint64_t lane_xor(uint64_t v, int j) { return __shfl_xor((unsigned long long)v, j); }
__device__ inline Cand lane_xor(const Cand &v, int j) { return Cand{__shfl_xor(v.score, j), (uint32_t)__shfl_xor((int)v.place, j), __shfl_xor(v.token, j)}; }
__device__ inline bool better(float a, float b) { return a > b; }
__device__ inline bool better(uint64_t a, uint64_t b) { return a > b; }
__device__ inline bool better(const Cand &a, const Cand &b) { return a.score > b.score || (a.score == b.score && a.place < b.place); }
// One step: of a lane and its partner j away the better stays in the one chosen by `first`.
template <typename V>
__device__ inline V exchange(const V &v, int j, bool first)
{
    const V o = lane_xor(v, j);
    return better(o, v) == first ? o : v;              // keys are distinct, or equal in all that counts
}
template <typename V>
__device__ inline V sort_lanes(V v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) v = exchange(v, j, ((lane & j) == 0) == ((lane & k) == 0));
    return v;
}
// The 64 best of two sorted lists; `other` holds the second one in reverse (lane i: its entry 63 - i).
template <typename V>
__device__ inline V merge_lanes(const V &v, const V &other)
{
    const int lane = threadIdx.x & 63;
    V r = better(other, v) ? other : v;
#pragma unroll
    for (int j = 32; j > 0; j >>= 1) r = exchange(r, j, (lane & j) == 0);
    return r;
}
// n-th largest (n <= 64) of one value per thread.  No NaN.
__device__ inline float block_nth(float v, int n, float (&lds)[kBeamThreads])
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

// ---- stage 1: the n best of a segment of a row, and its part of the log-normaliser ----
// A segment passes through registers once, kChunk categories at a time.  The n-th largest of the first chunk's 256 thread maxima is a
// bound that at least n categories reach; what reaches it (some 1.1 n of a chunk) goes to a list in LDS, and later chunks add
// what lies above it, for a category further back loses a tie.  Should the list overflow (rows in ascending order, ties), the bound is
// raised by the chunk's own maxima, then by the list cut to its n best, and as a last resort the chunk goes through the list 256 at a time.
constexpr int kElems = 16, kChunk = kBeamThreads * kElems, kList = 1024;
struct RowPart { float m; float pad; double sum; };    // maximum and sum of exp(z - m) of a segment

template <typename T> struct Vec { static constexpr int N = 16 / sizeof(T); };

// The categories of a chunk: virtual index i (category + off, where off is the row's distance from a 16-byte boundary) of element e.
template <typename T>
__device__ inline int64_t elem_index(int64_t base, int e)
{
    constexpr int N = Vec<T>::N;
    return base + (e / N) * (kBeamThreads * N) + threadIdx.x * N + e % N;
}
// -inf outside [lo, hi)
template <typename T>
__device__ inline void load_chunk(const T *row, int64_t base, int64_t lo, int64_t hi, float (&v)[kElems])
{
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int j = 0; j < kElems / N; ++j) {
        const int64_t i = elem_index<T>(base, j * N);
        if (i >= lo && i + N <= hi) {
            const uint4 q = *reinterpret_cast<const uint4 *>(row + i);
            const T *t = reinterpret_cast<const T *>(&q);
#pragma unroll
            for (int k = 0; k < N; ++k) v[j * N + k] = to_f32(t[k]);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[j * N + k] = i + k >= lo && i + k < hi ? to_f32(row[i + k]) : PC_NEG_INF_F;
        }
    }
}

struct BeamLds {
    uint64_t list[kList], kept[64];
    float nth[kBeamThreads];
    int count;
};

// Cut the list to its n best, in order; returns the n-th (0: fewer).  All threads; the list is complete and synchronised.
__device__ inline uint64_t cut_list(BeamLds &s, int n)
{
    int count = s.count;
    if (count > 128) {                                 // a bound from thread maxima leaves few for the ranking
        float mine = PC_NEG_INF_F;
        for (int i = threadIdx.x; i < count; i += kBeamThreads) mine = fmaxf(mine, key_value((uint32_t)(s.list[i] >> 32)));
        const uint32_t bound = order_key(block_nth(mine, n, s.nth));
        uint64_t held[kList / kBeamThreads];
#pragma unroll
        for (int i = 0; i < kList / kBeamThreads; ++i) held[i] = threadIdx.x + i * kBeamThreads < count ? s.list[threadIdx.x + i * kBeamThreads] : 0;
        __syncthreads();
        if (threadIdx.x == 0) s.count = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kList / kBeamThreads; ++i)
            if (held[i] && (uint32_t)(held[i] >> 32) >= bound) s.list[atomicAdd(&s.count, 1)] = held[i];
        __syncthreads();
        count = s.count;
    }
    if (threadIdx.x < 64) s.kept[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += kBeamThreads) {
        const uint64_t k = s.list[i];
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += s.list[j] > k;
        if (rank < n) s.kept[rank] = k;
    }
    __syncthreads();
    if (threadIdx.x < n) s.list[threadIdx.x] = s.kept[threadIdx.x];
    if (threadIdx.x == 0) s.count = min(count, n);
    __syncthreads();
    return s.kept[n - 1];
}

// the next float up; above +inf: NaN, which nothing reaches
__device__ inline float next_above(float t) { return key_value(order_key(t) + 1); }

template <typename T>
__global__ __launch_bounds__(kBeamThreads) void k_beam_rows(const BeamDev a, int32_t n_seg, int32_t seg_len, uint64_t *__restrict__ best,
                                                            RowPart *__restrict__ parts)
{
    __shared__ BeamLds s;
    __shared__ float wave_m[kBeamThreads / 64];
    __shared__ double wave_sum[kBeamThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.n_out;
    const int64_t tasks = (int64_t)a.groups * a.beams * n_seg;
    for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
        const int64_t r = task / n_seg;
        if ((a.done && a.done[r]) || running_score(a, r) == PC_NEG_INF_F) continue;       // the join knows these beams' candidates
        const T *z = (const T *)a.scores + r * a.ld;
        const int64_t off = ((uintptr_t)z & 15) / sizeof(T);
        const T *row = z - off;                        // category c is element c + off; none before off is read
        const int64_t first = (task % n_seg) * (int64_t)seg_len, hi = min(off + a.n_cats, first + seg_len), lo = max(off, first);
        float m = PC_NEG_INF_F, sum = 0.0f, t = PC_NEG_INF_F;
        __syncthreads();
        if (threadIdx.x == 0) s.count = 0;
        __syncthreads();
        float v[kElems], ahead[kElems];
        load_chunk(row, first, lo, hi, ahead);
        for (int64_t base = first; base < hi; base += kChunk) {
#pragma unroll
            for (int e = 0; e < kElems; ++e) v[e] = ahead[e];
            if (base + kChunk < hi) load_chunk(row, base + kChunk, lo, hi, ahead);
            float top = v[0];
#pragma unroll
            for (int e = 1; e < kElems; ++e) top = fmaxf(top, v[e]);
            top = fmaxf(top, PC_NEG_INF_F);            // NaN alone
            if (a.normalise) {
                if (top > m) { sum *= exp2f((m - top) * PC_LOG2E_F); m = top; }
                const float at = m == PC_NEG_INF_F ? 0.0f : m;
                float part = 0.0f;
#pragma unroll
                for (int e = 0; e < kElems; ++e) part += __builtin_amdgcn_exp2f((v[e] - at) * PC_LOG2E_F);
                sum += part;
            }
            bool fresh = false, slow = false;          // fresh: t is reached by n categories of this chunk or before
            if (t == PC_NEG_INF_F) {
                t = block_nth(top, n, s.nth);
                fresh = t > PC_NEG_INF_F;
                slow = !fresh;
            }
            // count what reaches t; room for all of it, or a higher t
            int mine = 0, at = 0;
            for (int attempt = 0; !slow; ++attempt) {
                mine = 0;
#pragma unroll
                for (int e = 0; e < kElems; ++e) mine += __popcll(__ballot(v[e] >= t));
                __syncthreads();
                if (lane == 0 && mine) at = atomicAdd(&s.count, mine);
                __syncthreads();
                const int total = s.count;
                if (total <= kList) break;
                __syncthreads();
                if (lane == 0 && mine) atomicSub(&s.count, mine);
                __syncthreads();
                if (attempt == 0) {
                    const float bound = block_nth(top, n, s.nth);
                    if (!(bound < t)) { t = bound; fresh = true; }
                } else if (attempt == 1) {
                    const uint64_t nth = cut_list(s, n);
                    const float bound = nth ? next_above(key_value((uint32_t)(nth >> 32))) : t;
                    if (bound > t || bound != bound) { t = bound; fresh = false; }
                } else {
                    slow = true;
                }
            }
            if (!slow) {
                at = __shfl(at, 0);
                if (mine)
#pragma unroll
                    for (int e = 0; e < kElems; ++e) {
                        const uint64_t on = __ballot(v[e] >= t);
                        if (on == 0) continue;
                        if (v[e] >= t) s.list[at + __popcll(on & ((1ull << lane) - 1))] = candidate(v[e], (int)(elem_index<T>(base, e) - off));
                        at += __popcll(on);
                    }
                if (fresh) t = next_above(t);
            } else {
                uint64_t above = 0;                    // only keys above this one count
                for (int e = 0; e < kElems; ++e) {
                    __syncthreads();
                    const bool full = s.count > kList - kBeamThreads;
                    __syncthreads();                   // all have read it before any adds
                    if (full) above = cut_list(s, n);
                    float x = v[0];
#pragma unroll
                    for (int f = 1; f < kElems; ++f) x = f == e ? v[f] : x;
                    const int64_t i = elem_index<T>(base, e);
                    const uint64_t k = i >= lo && i < hi ? candidate(x, (int)(i - off)) : 0;
                    if (k > above) s.list[atomicAdd(&s.count, 1)] = k;
                }
                __syncthreads();
                const uint64_t nth = cut_list(s, n);
                t = nth ? next_above(key_value((uint32_t)(nth >> 32))) : PC_NEG_INF_F;
            }
        }
        __syncthreads();
        cut_list(s, n);
        if (threadIdx.x < n) best[task * n + threadIdx.x] = s.kept[threadIdx.x];
        if (a.normalise) {
            float all = m;
            for (int d = 32; d > 0; d >>= 1) all = fmaxf(all, __shfl_xor(all, d));
            if (lane == 0) wave_m[wave] = all;
            __syncthreads();
            for (int w = 0; w < kBeamThreads / 64; ++w) all = fmaxf(all, wave_m[w]);
            double total = (double)sum * (m == PC_NEG_INF_F ? 1.0 : (double)exp2f((m - all) * PC_LOG2E_F));
            for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
            if (lane == 0) wave_sum[wave] = total;
            __syncthreads();
            if (threadIdx.x == 0) {
                total = 0.0;
                for (int w = 0; w < kBeamThreads / 64; ++w) total += wave_sum[w];
                parts[task] = RowPart{all, 0.0f, total};
            }
        }
    }
}

// ---- stage 2: a group's survivors from its rows' lists ----
// A wave a beam (up to 16 waves, each taking several beams in turn): the segments' parts of the log-normaliser in 64 bits, the segments'
// lists merged by key, then by score with the wave's beams before; last the waves' lists, half of them at a time.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(64 * kJoinWaves) void k_beam_join(const BeamDev a, int32_t n_seg, const uint64_t *__restrict__ best,
                                                               const RowPart *__restrict__ parts, float *__restrict__ out_scores,
                                                               int32_t *__restrict__ parents, int32_t *__restrict__ tokens)
{
    __shared__ Cand lists[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, n = a.n_out;
    const Cand none{kNegInf64, kNoPlace, 0};
    for (int64_t g = blockIdx.x; g < a.groups; g += gridDim.x) {
        Cand mine = none;
        for (int b = wave; b < a.beams; b += waves) {
            const int64_t r = g * a.beams + b;
            const double run = (double)running_score(a, r);
            const bool done = a.done && a.done[r];
            bool dead = run == kNegInf64;
            Cand c = none;
            if (!dead && !done) {
                double norm = 0.0;
                if (a.normalise) {
                    float m = PC_NEG_INF_F;
                    double sum = 0.0;
                    for (int i = lane; i < n_seg; i += 64) m = fmaxf(m, parts[r * n_seg + i].m);
                    for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
                    for (int i = lane; i < n_seg; i += 64) {
                        const RowPart p = parts[r * n_seg + i];
                        sum += p.m == PC_NEG_INF_F ? p.sum : p.sum * exp((double)p.m - (double)m);
                    }
                    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
                    norm = (double)m + log(sum);
                }
                dead = !(fabs(norm) < 1e300);          // no finite number: m is a float
                uint64_t key = 0;
                for (int s0 = 0; s0 < n_seg; s0 += 8) {
                    uint64_t next[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        next[i] = s0 + i < n_seg && (s0 + i == 0 ? lane : 63 - lane) < n ? best[(r * n_seg + s0 + i) * n + (s0 + i == 0 ? lane : 63 - lane)] : 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (s0 + i == 0) key = next[i];
                        else if (s0 + i < n_seg) key = merge_lanes(key, next[i]);
                }
                if (key && lane < n) c = Cand{run + ((double)key_value((uint32_t)(key >> 32)) - norm), (uint32_t)(b << 8 | lane), (int32_t)~(uint32_t)key};
            }
            if (dead || done) {                        // candidates of -inf in order, after the one of a finished beam
                const bool ended = done && !dead;
                const int token = !ended ? lane : lane == 0 ? a.done_token : lane <= a.done_token ? lane - 1 : lane;
                c = lane < min(n, a.n_cats) ? Cand{ended && lane == 0 ? run : kNegInf64, (uint32_t)(b << 8 | lane), token} : none;
            }
            if (b == wave) mine = c;
            else mine = merge_lanes(mine, Cand{__shfl(c.score, 63 - lane), (uint32_t)__shfl((int)c.place, 63 - lane), __shfl(c.token, 63 - lane)});
        }
        for (int half = waves; half > 1;) {
            const int keep = (half + 1) / 2;
            __syncthreads();
            if (wave >= keep && wave < half) lists[wave][lane] = mine;
            __syncthreads();
            if (wave + keep < half) mine = merge_lanes(mine, lists[wave + keep][63 - lane]);
            half = keep;
        }
        if (wave == 0 && lane < n) {
            out_scores[g * n + lane] = (float)mine.score;
            parents[g * n + lane] = (int32_t)(mine.place >> 8);
            tokens[g * n + lane] = mine.token;
        }
    }
}

struct StatesDev {
    int32_t n;
    pc_state s[PC_MAX_STATES];
};

// One workgroup a surviving row and state; bytes.
__global__ __launch_bounds__(256) void k_beam_reorder(const StatesDev st, const int32_t *__restrict__ parents, int64_t rows, int32_t beams, int32_t n_out)
{
    const pc_state s = st.s[blockIdx.y];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int32_t p = parents[r];
        if (p < 0 || p >= beams) continue;
        const char *src = (const char *)s.src + (r / n_out * beams + p) * s.src_stride;
        char *dst = (char *)s.dst + r * s.dst_stride;
        for (int64_t i = threadIdx.x; i < s.row_bytes; i += 256) dst[i] = src[i];
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
    const int64_t rows = (int64_t)a->groups * a->beams, len = (int64_t)a->n_cats + 7, chunks = (len + kChunk - 1) / kChunk;
    const int64_t most = (1 << 30) / kChunk;           // chunks of a segment whose length is an int32
    const int64_t wanted = std::min(chunks, std::max(1024 / std::max<int64_t>(rows, 1), (chunks + most - 1) / most));
    const int64_t each = (chunks + wanted - 1) / wanted;
    return Segments{(int32_t)((chunks + each - 1) / each), (int32_t)(each * kChunk)};
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
    const BeamDev dev{a->groups, a->beams, a->n_cats, a->n_out, a->scores, a->scores_ld, a->normalise != 0, a->running, a->done, a->done_token};
    const Segments seg = segments_of(a);
    uint64_t *best = (uint64_t *)workspace;
    RowPart *parts = (RowPart *)((char *)workspace + best_bytes(a));
    const hipStream_t s = (hipStream_t)stream;
    const unsigned tasks = (unsigned)std::min<int64_t>((int64_t)a->groups * a->beams * seg.n, 1 << 20);
    with_type(a->scores_type, [&](auto t) { hipLaunchKernelGGL((k_beam_rows<decltype(t)>), dim3(tasks), dim3(kBeamThreads), 0, s, dev, seg.n, seg.len, best, parts); });
    hipLaunchKernelGGL(k_beam_join, dim3((unsigned)std::min(a->groups, 1 << 20)), dim3((unsigned)(64 * std::min(a->beams, kJoinWaves))), 0, s, dev, seg.n, best,
                       parts, out_scores, parents, tokens);
    return launched();
}

pc_status pc_beam_reorder(const pc_state *states, int32_t n_states, const int32_t *parents, int32_t groups, int32_t beams, int32_t n_out, void *stream)
{
    if (!states || n_states < 1 || n_states > PC_MAX_STATES) return fail(PC_ERR_ARG, "1 .. PC_MAX_STATES states");
    if (groups < 0 || beams < 1 || beams > PC_MAX_BEAMS || n_out < 1 || n_out > PC_MAX_BEAM_OUT) return fail(PC_ERR_ARG, "groups, beams or n_out out of range");
    const int64_t rows = (int64_t)groups * n_out, src_rows = (int64_t)groups * beams;
    if (rows > INT32_MAX || src_rows > INT32_MAX) return fail(PC_ERR_TOO_LARGE, "more than 2^31 - 1 rows");
    StatesDev dev{n_states, {}};
    struct Span { uintptr_t at, end; };
    Span span[2 * PC_MAX_STATES];
    for (int32_t i = 0; i < n_states; ++i) {
        const pc_state &s = states[i];
        if (s.row_bytes < 1 || s.src_stride < s.row_bytes || s.dst_stride < s.row_bytes) return fail(PC_ERR_ARG, "row_bytes must be positive, strides at least row_bytes");
        if (groups == 0) continue;
        if (!s.src || !s.dst) return fail(PC_ERR_ARG, "NULL argument");
        span[2 * i] = {(uintptr_t)s.src, (uintptr_t)s.src + (uintptr_t)((src_rows - 1) * s.src_stride + s.row_bytes)};
        span[2 * i + 1] = {(uintptr_t)s.dst, (uintptr_t)s.dst + (uintptr_t)((rows - 1) * s.dst_stride + s.row_bytes)};
        dev.s[i] = s;
    }
    if (groups == 0) return PC_OK;
    if (!parents) return fail(PC_ERR_ARG, "NULL argument");
    if (!aligned_to(parents, 4)) return fail(PC_ERR_ARG, "parents must be 4-byte aligned");
    for (int32_t i = 0; i < n_states; ++i)                                        // a dst against every src and the dst before it
        for (int32_t j = 0; j < 2 * n_states; ++j) {
            const Span &d = span[2 * i + 1], &o = span[j];
            if (j != 2 * i + 1 && d.at < o.end && o.at < d.end) return fail(PC_ERR_ARG, "dst overlaps a src or another dst");
        }
    hipLaunchKernelGGL(k_beam_reorder, dim3((unsigned)std::min<int64_t>(rows, 1 << 20), (unsigned)n_states), dim3(256), 0, (hipStream_t)stream, dev, parents,
                       rows, beams, n_out);
    return launched();
}

}  // extern "C"
