// Distillation from a teacher's top logits: loss per row and gradient of the student's rows.
//   q_j = softmax over the list of teacher_j / T (or exp(teacher_j / T - lse));  logp = log-softmax of student / T
//   loss = sum_j q_j (log q_j - logp[id_j]);   gradient_c = (p_c sum_j q_j - sum_{id_j = c} q_j) / T
// A row's maximum is subtracted before the division by T, so that logits as low as their type goes do not overflow at T < 1.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "pc_internal.h"
#include "pc_rows.h"

namespace pc {

constexpr int kRowThreads = 256;

// Sum / maximum over a workgroup of kRowThreads; every thread gets the result.
template <typename F>
__device__ inline float block_all(float v, float *lds, F op)
{
    for (int d = 32; d > 0; d >>= 1) v = op(v, __shfl_xor(v, d));
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < kRowThreads / 64; ++w) v = op(v, lds[w]);
    return v;
}
__device__ inline float add2(float a, float b) { return a + b; }
__device__ inline float max2(float a, float b) { return fmaxf(a, b); }
// exp(a - m) of a running maximum m; nothing seen yet (-inf) counts as 0
__device__ inline float exp_below(float a, float m, float inv_T) { return m == PC_NEG_INF_F ? 0.0f : expf((a - m) * inv_T); }

struct DistillDev {                                   // pc_distill without its types
    int64_t rows, student_ld, ids_ld, teacher_ld;
    int32_t n_cats, top;
    const void *student, *teacher;
    const int32_t *ids;
    const float *teacher_lse;
    float inv_T;
    bool normalised;
};

// The list of a row: q and log q per entry, in registers of thread j mod kRowThreads; out of range or -inf: q = 0.
constexpr int kListRegs = PC_MAX_TOP / kRowThreads;
template <typename TT>
__device__ inline void row_targets(const DistillDev &d, int64_t r, float *lds, int32_t (&id)[kListRegs], float (&q)[kListRegs], float (&logq)[kListRegs])
{
    const TT *teacher = (const TT *)d.teacher + r * d.teacher_ld;
    const int32_t *ids = d.ids + r * d.ids_ld;
    float m = PC_NEG_INF_F;
    for (int i = 0; i < kListRegs; ++i) {
        const int j = threadIdx.x + i * kRowThreads;
        id[i] = -1;
        logq[i] = PC_NEG_INF_F;
        if (j < d.top) {
            const int32_t c = ids[j];
            if (c >= 0 && c < d.n_cats) { id[i] = c; logq[i] = to_f32(teacher[j]); }
        }
        m = max2(m, logq[i]);
    }
    float shift = 0.0f, base = 0.0f;
    if (d.teacher_lse) {
        base = d.teacher_lse[r];
    } else {
        shift = block_all(m, lds, max2);
        if (shift == PC_NEG_INF_F) shift = 0.0f;      // nothing listed: every q is 0
        float s = 0.0f;
        for (int i = 0; i < kListRegs; ++i) s += expf((logq[i] - shift) * d.inv_T);
        base = logf(block_all(s, lds, add2));
    }
    for (int i = 0; i < kListRegs; ++i) {
        logq[i] = logq[i] == PC_NEG_INF_F ? PC_NEG_INF_F : (logq[i] - shift) * d.inv_T - base;
        q[i] = expf(logq[i]);
    }
}

template <typename TS, typename TT>
__global__ __launch_bounds__(kRowThreads) void k_distill_rows(const DistillDev d, float *__restrict__ loss, float *__restrict__ stats)
{
    __shared__ float lds[kRowThreads / 64];
    for (int64_t r = blockIdx.x; r < d.rows; r += gridDim.x) {
        const TS *z = (const TS *)d.student + r * d.student_ld;
        float m = PC_NEG_INF_F, s = 0.0f, log_s = 0.0f;
        if (!d.normalised) {
            for (int c = threadIdx.x; c < d.n_cats; c += kRowThreads) {
                const float v = to_f32(z[c]), above = max2(m, v);
                s = s * exp_below(m, above, d.inv_T) + exp_below(v, above, d.inv_T);
                if (v != v) s = v;
                m = above;
            }
            const float all = block_all(m, lds, max2);
            s = block_all(s * exp_below(m, all, d.inv_T), lds, add2);
            m = s != s && all < __builtin_inff() ? s : all;   // a row with a NaN has no maximum, not even where all else is -inf
            log_s = logf(s);
        } else {
            m = 0.0f;
        }
        int32_t id[kListRegs];
        float q[kListRegs], logq[kListRegs], part = 0.0f;
        row_targets<TT>(d, r, lds, id, q, logq);
        for (int i = 0; i < kListRegs; ++i)
            if (id[i] >= 0 && !(q[i] == 0.0f)) {
                const float v = to_f32(z[id[i]]);
                const float logp = d.normalised ? v : m == PC_NEG_INF_F ? m : (v - m) * d.inv_T - log_s;
                part += q[i] * (logq[i] - logp);
            }
        part = block_all(part, lds, add2);
        if (threadIdx.x == 0) {
            loss[r] = part;
            stats[2 * r] = m;
            stats[2 * r + 1] = log_s;
        }
    }
}

// The listed entries are written after a barrier over what the row's dense part put there.
template <typename TS, typename TT>
__global__ __launch_bounds__(kRowThreads) void k_distill_grad(const DistillDev d, const float *__restrict__ stats, const float *__restrict__ dloss,
                                                              float scale, void *dstudent, int64_t out_ld)
{
    __shared__ float lds[kRowThreads / 64];
    __shared__ int32_t ids[PC_MAX_TOP];
    __shared__ float qs[PC_MAX_TOP];
    for (int64_t r = blockIdx.x; r < d.rows; r += gridDim.x) {
        const TS *z = (const TS *)d.student + r * d.student_ld;
        TS *out = (TS *)dstudent + r * out_ld;
        const float g = (dloss ? scale * dloss[r] : scale) * d.inv_T;
        int32_t id[kListRegs];
        float q[kListRegs], logq[kListRegs], at[kListRegs], Q = 0.0f;
        row_targets<TT>(d, r, lds, id, q, logq);
        __syncthreads();
        for (int i = 0; i < kListRegs; ++i) {
            const int j = threadIdx.x + i * kRowThreads;
            Q += q[i];
            at[i] = id[i] >= 0 && !d.normalised ? to_f32(z[id[i]]) : 0.0f;
            if (j < d.top) { ids[j] = id[i]; qs[j] = q[i]; }
        }
        Q = block_all(Q, lds, add2);
        const bool none = g == 0.0f || Q == 0.0f;
        const float m = stats[2 * r], log_s = stats[2 * r + 1];
        auto dense = [&](float v) {
            return none || d.normalised || m == PC_NEG_INF_F ? 0.0f : expf((v - m) * d.inv_T - log_s) * Q;
        };
        __syncthreads();
        if (none || d.normalised)
            for (int c = threadIdx.x; c < d.n_cats; c += kRowThreads) out[c] = from_f32<TS>(0.0f);
        else
            for (int c = threadIdx.x; c < d.n_cats; c += kRowThreads) out[c] = from_f32<TS>(g * dense(to_f32(z[c])));
        __syncthreads();
        if (none) continue;
        for (int i = 0; i < kListRegs; ++i) {
            const int j = threadIdx.x + i * kRowThreads;
            if (id[i] < 0) continue;
            bool first = true;
            float sum = 0.0f;                         // a category listed more than once: its first entry writes for all
            for (int k = 0; k < d.top; ++k)
                if (ids[k] == id[i]) { first = first && k >= j; sum += qs[k]; }
            if (first) out[id[i]] = from_f32<TS>(g * (dense(at[i]) - sum));
        }
    }
}

static pc_status check_distill(const pc_distill *d)
{
    if (!d) return fail(PC_ERR_ARG, "NULL argument");
    if (d->rows < 0) return fail(PC_ERR_ARG, "rows must not be negative");
    if (d->n_cats < 1) return fail(PC_ERR_ARG, "n_cats must be positive");
    if (d->top < 1 || d->top > PC_MAX_TOP) return fail(PC_ERR_ARG, "top must be in 1 .. PC_MAX_TOP");
    if (!type_known(d->student_type) || !type_known(d->teacher_type)) return fail(PC_ERR_ARG, "unknown element type");
    if (!(d->temperature > 0.0f) || std::isinf(d->temperature) || std::isinf(1.0f / d->temperature))
        return fail(PC_ERR_ARG, "temperature and its reciprocal must be positive and finite");
    if (d->normalised && d->temperature != 1.0f) return fail(PC_ERR_ARG, "normalised rows have temperature 1");
    if (d->student_ld < d->n_cats) return fail(PC_ERR_ARG, "student_ld is smaller than n_cats");
    if (d->ids_ld < d->top || d->teacher_ld < d->top) return fail(PC_ERR_ARG, "ids_ld or teacher_ld is smaller than top");
    if (d->rows == 0) return PC_OK;
    if (!d->student || !d->ids || !d->teacher) return fail(PC_ERR_ARG, "NULL argument");
    if (!aligned_to(d->student, type_bytes(d->student_type)) || !aligned_to(d->teacher, type_bytes(d->teacher_type)) || !aligned_to(d->ids, 4) ||
        !aligned_to(d->teacher_lse, 4))
        return fail(PC_ERR_ARG, "arrays must be aligned to their elements");
    return PC_OK;
}
static DistillDev distill_dev(const pc_distill *d)
{
    return DistillDev{d->rows, d->student_ld, d->ids_ld, d->teacher_ld, d->n_cats, d->top, d->student, d->teacher, d->ids, d->teacher_lse,
                      1.0f / d->temperature, d->normalised != 0};
}
static unsigned row_grid(int64_t rows) { return (unsigned)std::min<int64_t>(rows, 1 << 20); }

// first and last byte of `rows` rows
static bool overlap(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes)
{
    return (uintptr_t)a < (uintptr_t)b + (uintptr_t)b_bytes && (uintptr_t)b < (uintptr_t)a + (uintptr_t)a_bytes;
}

}  // namespace pc

using namespace pc;

extern "C" {

pc_status pc_distill_workspace_bytes(const pc_distill *d, size_t *bytes)
{
    const pc_status st = check_distill(d);
    if (st != PC_OK) return st;
    if (!bytes) return fail(PC_ERR_ARG, "NULL argument");
    *bytes = 0;
    return PC_OK;
}

pc_status pc_distill_forward(const pc_distill *d, void *workspace, size_t workspace_bytes, float *loss, float *stats, void *stream)
{
    const pc_status st = check_distill(d);
    if (st != PC_OK || d->rows == 0) return st;
    if (!loss || !stats) return fail(PC_ERR_ARG, "NULL argument");
    if (!aligned_to(loss, 4) || !aligned_to(stats, 4)) return fail(PC_ERR_ARG, "loss and stats must be 4-byte aligned");
    size_t need = 0;
    pc_distill_workspace_bytes(d, &need);
    if (need && !workspace) return fail(PC_ERR_ARG, "NULL argument");
    if (workspace_bytes < need) return fail(PC_ERR_WORKSPACE, "workspace smaller than pc_distill_workspace_bytes");
    if (need && !aligned_to(workspace, 16)) return fail(PC_ERR_ARG, "the workspace must be 16-byte aligned");
    const DistillDev dev = distill_dev(d);
    with_type(d->student_type, [&](auto s) {
        with_type(d->teacher_type, [&](auto t) {
            hipLaunchKernelGGL((k_distill_rows<decltype(s), decltype(t)>), dim3(row_grid(d->rows)), dim3(kRowThreads), 0, (hipStream_t)stream, dev, loss,
                               stats);
        });
    });
    return launched();
}

pc_status pc_distill_backward(const pc_distill *d, const float *stats, const float *dloss, float scale, void *dstudent, int64_t dstudent_ld, void *stream)
{
    const pc_status st = check_distill(d);
    if (st != PC_OK || d->rows == 0) return st;
    if (!stats || !dstudent) return fail(PC_ERR_ARG, "NULL argument");
    if (dstudent_ld < d->n_cats) return fail(PC_ERR_ARG, "dstudent_ld is smaller than n_cats");
    const int64_t e = type_bytes(d->student_type);
    if (!aligned_to(stats, 4) || !aligned_to(dloss, 4) || !aligned_to(dstudent, e)) return fail(PC_ERR_ARG, "arrays must be aligned to their elements");
    const int64_t in = ((d->rows - 1) * d->student_ld + d->n_cats) * e, out = ((d->rows - 1) * dstudent_ld + d->n_cats) * e;
    if (overlap(d->student, in, dstudent, out) && !(d->student == dstudent && d->student_ld == dstudent_ld))
        return fail(PC_ERR_ARG, "dstudent overlaps the student's rows without being them");
    const DistillDev dev = distill_dev(d);
    with_type(d->student_type, [&](auto s) {
        with_type(d->teacher_type, [&](auto t) {
            hipLaunchKernelGGL((k_distill_grad<decltype(s), decltype(t)>), dim3(row_grid(d->rows)), dim3(kRowThreads), 0, (hipStream_t)stream, dev, stats,
                               dloss, scale, dstudent, dstudent_ld);
        });
    });
    return launched();
}

}  // extern "C"
