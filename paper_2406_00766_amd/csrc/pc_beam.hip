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

// The n best of each row as keys (best first; 0: none), and its log-normaliser.  One workgroup a row, one pass per survivor.
template <typename T>
__global__ __launch_bounds__(kBeamThreads) void k_beam_rows(const BeamDev a, uint64_t *__restrict__ best, double *__restrict__ lse)
{
    __shared__ uint64_t top[kBeamThreads / 64];
    __shared__ double part[kBeamThreads / 64];
    const int64_t rows = (int64_t)a.groups * a.beams;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *z = (const T *)a.scores + r * a.ld;
        const bool done = a.done && a.done[r], dead = running_score(a, r) == PC_NEG_INF_F;
        double norm = 0.0;
        uint64_t last = ~0ull;
        for (int n = 0; n < a.n_out; ++n) {
            uint64_t mine = 0;
            if (!done && !dead)
                for (int c = threadIdx.x; c < a.n_cats; c += kBeamThreads) {
                    const uint64_t k = candidate(to_f32(z[c]), c);
                    if (k < last && k > mine) mine = k;
                }
            for (int d = 32; d > 0; d >>= 1) mine = max(mine, (uint64_t)__shfl_xor((unsigned long long)mine, d));
            __syncthreads();
            if (threadIdx.x % 64 == 0) top[threadIdx.x / 64] = mine;
            __syncthreads();
            for (int w = 0; w < kBeamThreads / 64; ++w) mine = max(mine, top[w]);
            if (n == 0 && a.normalise && !done && !dead) {
                const float m = key_value((uint32_t)(mine >> 32));
                double s = 0.0;
                for (int c = threadIdx.x; c < a.n_cats; c += kBeamThreads) s += (double)expf(to_f32(z[c]) - m);
                for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
                if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
                __syncthreads();
                s = 0.0;
                for (int w = 0; w < kBeamThreads / 64; ++w) s += part[w];
                norm = (double)m + log(s);
            }
            if (threadIdx.x == 0) best[r * a.n_out + n] = mine;
            last = mine;
        }
        if (threadIdx.x == 0) lse[r] = norm;
    }
}

// The n best of a group's beams * n_out row survivors, one workgroup a group, one pass per survivor.
__global__ __launch_bounds__(kBeamThreads) void k_beam_join(const BeamDev a, const uint64_t *__restrict__ best, const double *__restrict__ lse,
                                                            float *__restrict__ out_scores, int32_t *__restrict__ parents, int32_t *__restrict__ tokens)
{
    __shared__ double top_s[kBeamThreads / 64];
    __shared__ int32_t top_i[kBeamThreads / 64];
    const int n_cand = a.beams * a.n_out;
    // candidate i of group g: its score (NaN: no such candidate) and its category
    auto look = [&](int64_t g, int i, double &score, int32_t &token) {
        const int64_t r = g * a.beams + i / a.n_out;
        const int at = i % a.n_out;
        const double run = (double)running_score(a, r), norm = lse[r];
        const bool done = a.done && a.done[r], dead = run == kNegInf64 || !(fabs(norm) < 1e300);
        if (at >= a.n_cats) { score = __builtin_nan(""); token = 0; return; }
        if (dead) { score = kNegInf64; token = at; return; }
        if (done) {
            token = at == 0 ? a.done_token : at <= a.done_token ? at - 1 : at;
            score = at == 0 ? run : kNegInf64;
            return;
        }
        const uint64_t k = best[r * a.n_out + at];
        score = run + ((double)key_value((uint32_t)(k >> 32)) - norm);
        token = (int32_t)~(uint32_t)k;
    };
    for (int64_t g = blockIdx.x; g < a.groups; g += gridDim.x) {
        double last_s = 0.0;
        int last_i = -1;
        for (int n = 0; n < a.n_out; ++n) {
            double mine = 0.0;
            int at = -1;
            for (int i = threadIdx.x; i < n_cand; i += kBeamThreads) {
                double s;
                int32_t token;
                look(g, i, s, token);
                if (s != s) continue;
                const bool left = last_i < 0 || s < last_s || (s == last_s && i > last_i);
                if (left && (at < 0 || s > mine)) { mine = s; at = i; }
            }
            for (int d = 32; d > 0; d >>= 1) {
                const double s = __shfl_xor(mine, d);
                const int i = __shfl_xor(at, d);
                if (i >= 0 && (at < 0 || s > mine || (s == mine && i < at))) { mine = s; at = i; }
            }
            __syncthreads();
            if (threadIdx.x % 64 == 0) { top_s[threadIdx.x / 64] = mine; top_i[threadIdx.x / 64] = at; }
            __syncthreads();
            at = -1;
            for (int w = 0; w < kBeamThreads / 64; ++w)
                if (top_i[w] >= 0 && (at < 0 || top_s[w] > mine || (top_s[w] == mine && top_i[w] < at))) { mine = top_s[w]; at = top_i[w]; }
            if (threadIdx.x == 0) {
                double s;
                int32_t token;
                look(g, at, s, token);
                out_scores[g * a.n_out + n] = (float)s;
                parents[g * a.n_out + n] = at / a.n_out;
                tokens[g * a.n_out + n] = token;
            }
            last_s = mine;
            last_i = at;
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
static size_t best_bytes(const pc_beam *a) { return ((size_t)a->groups * a->beams * a->n_out * 8 + 15) / 16 * 16; }

}  // namespace pc

using namespace pc;

extern "C" {

pc_status pc_beam_workspace_bytes(const pc_beam *a, size_t *bytes)
{
    const pc_status st = check_beam(a);
    if (st != PC_OK) return st;
    if (!bytes) return fail(PC_ERR_ARG, "NULL argument");
    *bytes = best_bytes(a) + (size_t)a->groups * a->beams * 8;
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
    uint64_t *best = (uint64_t *)workspace;
    double *lse = (double *)((char *)workspace + best_bytes(a));
    const hipStream_t s = (hipStream_t)stream;
    const unsigned rows = (unsigned)std::min<int64_t>((int64_t)a->groups * a->beams, 1 << 20);
    with_type(a->scores_type, [&](auto t) { hipLaunchKernelGGL((k_beam_rows<decltype(t)>), dim3(rows), dim3(kBeamThreads), 0, s, dev, best, lse); });
    hipLaunchKernelGGL(k_beam_join, dim3((unsigned)std::min(a->groups, 1 << 20)), dim3(kBeamThreads), 0, s, dev, best, lse, out_scores, parents, tokens);
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
