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

struct DistillDev {                                   // pc_distill without its types
    int64_t rows, student_ld, ids_ld, teacher_ld;
    int32_t n_cats, top;
    const void *student, *teacher;
    const int32_t *ids;
    const float *teacher_lse;
    float inv_T;
    bool normalised;
};

__device__ inline float add2(float a, float b) { return a + b; }
__device__ inline float max2(float a, float b) { return fmaxf(a, b); }
// A row is worked on by WAVES waves of a workgroup; STREAM: rows that no cache holds until they are read again.  Its list lies with the first of them where it has at most 64 entries (LONG = false: no
// barriers), else with all of them, LIST entries a lane.
constexpr int kShortList = 64;
template <int WAVES, bool LONG, bool STREAM = false>
struct Group {
    static constexpr bool STREAMS = STREAM;
    static constexpr int THREADS = 64 * WAVES, LIST = LONG ? PC_MAX_TOP / THREADS : 1;
    static constexpr int ROWS = WAVES >= 4 ? 1 : 4 / WAVES;              // rows of a workgroup
    static constexpr int BLOCK = THREADS * ROWS;
    // over the lanes that have the list
    template <typename F>
    __device__ static inline float list_all(float v, float *lds, F op)
    {
        v = wave_all(v, op);
        if (!LONG) return v;
        __syncthreads();
        if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
        __syncthreads();
        v = lds[0];
        for (int w = 1; w < WAVES; ++w) v = op(v, lds[w]);
        return v;
    }
};

// The list of a row: category, q and log q of entry t + i * THREADS; out of range or -inf: q = 0.  Fetched first, made into
// probabilities once the rest of the row is on its way.
template <typename G, typename TT>
struct List {
    int32_t id[G::LIST];
    float q[G::LIST], logq[G::LIST], norm;
    __device__ inline void fetch(const DistillDev &d, int64_t r, int t)
    {
        const TT *teacher = (const TT *)d.teacher + r * d.teacher_ld;
        const int32_t *ids = d.ids + r * d.ids_ld;
        norm = d.teacher_lse ? d.teacher_lse[r] : 0.0f;
#pragma unroll
        for (int i = 0; i < G::LIST; ++i) {
            const int j = t + i * G::THREADS;
            id[i] = j < d.top ? ids[j] : -1;
            logq[i] = j < d.top ? to_f32(teacher[j]) : PC_NEG_INF_F;
        }
    }
    __device__ inline void probabilities(const DistillDev &d, float *lds)
    {
        float m = PC_NEG_INF_F, shift = 0.0f;
#pragma unroll
        for (int i = 0; i < G::LIST; ++i) {
            if (id[i] < 0 || id[i] >= d.n_cats) { id[i] = -1; logq[i] = PC_NEG_INF_F; }
            m = max2(m, logq[i]);
        }
        if (!d.teacher_lse) {
            shift = G::list_all(m, lds, max2);
            if (shift == PC_NEG_INF_F) shift = 0.0f;  // nothing listed: every q is 0
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < G::LIST; ++i) s += expf((logq[i] - shift) * d.inv_T);
            norm = logf(G::list_all(s, lds, add2));
        }
#pragma unroll
        for (int i = 0; i < G::LIST; ++i) {
            logq[i] = logq[i] == PC_NEG_INF_F ? PC_NEG_INF_F : (logq[i] - shift) * d.inv_T - norm;
            q[i] = expf(logq[i]);
        }
    }
};

// Loss and statistics.  A row passes through registers once, kPacks x 16 bytes a lane at a time, the next ones on their way, with a running
// maximum and sum per lane: bound by reading it (8192 x 50257: fp32 247 us, 6.7 TB/s; 16 bits 137, 6.0 TB/s).  The list is made into
// probabilities, and its student's logits are fetched, while the first packs are on their way.
constexpr int kPacks = 4;
// The element (of the grid that begins `off` elements before the row and has `end` up to the row's last) that lane t of a row takes of those
// in no whole pack; -1: none.
template <int N>
__device__ inline int64_t edge_of(int t, int off, int64_t end)
{
    const int64_t tail = max(end / N * N, (int64_t)(off > 0 ? N : 0));   // the first element behind the whole packs
    if (t < N) return off > 0 && t >= off && t < end ? t : -1;
    return t < 2 * N && tail + t - N < end ? tail + t - N : -1;
}
template <typename TS, typename TT, int WAVES, bool LONG, bool STREAM>
__global__ __launch_bounds__((Group<WAVES, LONG>::BLOCK)) void k_distill_rows(const DistillDev d, float *__restrict__ loss, float *__restrict__ stats)
{
    using G = Group<WAVES, LONG>;
    constexpr int N = Pack<TS>::N, TH = G::THREADS;
    __shared__ float lds[WAVES], wave_m[WAVES], wave_s[WAVES];
    const int t = threadIdx.x % TH, sub = threadIdx.x / TH;
    for (int64_t r = (int64_t)blockIdx.x * G::ROWS + sub; r < d.rows; r += (int64_t)gridDim.x * G::ROWS) {
        const TS *z = (const TS *)d.student + r * d.student_ld;
        const bool listing = LONG || t < 64;
        List<G, TT> list;
        float listed[G::LIST], m = PC_NEG_INF_F, s = 0.0f, log_s = 0.0f;
        if (listing) list.fetch(d, r, t);
        auto look_up = [&]() {                         // while the row is on its way
            if (!listing) return;
            list.probabilities(d, lds);
#pragma unroll
            for (int i = 0; i < G::LIST; ++i) listed[i] = to_f32(z[max(list.id[i], 0)]);
        };
        if (!d.normalised) {
            // whole packs of the 16-byte grid, and the elements before the first and behind the last, at most one a lane
            const int off = elements_off(z);
            const TS *grid = z - off;
            const int64_t end = off + (int64_t)d.n_cats, p_first = off > 0, p_last = end / N;
            const int64_t edge = edge_of<N>(t, off, end);
            float v[kPacks * N];
            Pack<TS> ahead[kPacks];
            auto fetch = [&](int64_t p0) {
#pragma unroll
                for (int k = 0; k < kPacks; ++k) {
                    const int64_t p = min(p0 + t + k * TH, p_last - 1);
                    const TS *from = (const TS *)__builtin_assume_aligned(grid + p * N, 16);
                    ahead[k] = STREAM ? stream_pack(from) : load_pack(from);
                }
            };
            if (p_first < p_last) fetch(p_first);
            if (edge >= 0) { m = to_f32(grid[edge]); s = m == PC_NEG_INF_F ? 0.0f : m == m ? 1.0f : m; }
            look_up();
            for (int64_t p0 = p_first; p0 < p_last; p0 += kPacks * TH) {
                const bool whole = p0 + kPacks * TH <= p_last;
#pragma unroll
                for (int k = 0; k < kPacks; ++k) {
                    float x[N];
                    unpack_f32(ahead[k], x);
#pragma unroll
                    for (int e = 0; e < N; ++e) v[k * N + e] = whole || p0 + t + k * TH < p_last ? x[e] : PC_NEG_INF_F;
                }
                if (p0 + kPacks * TH < p_last) fetch(p0 + kPacks * TH);
                float top = v[0];
#pragma unroll
                for (int e = 1; e < kPacks * N; ++e) top = max2(top, v[e]);
                if (top > m) { s *= exp2f((m - top) * (d.inv_T * PC_LOG2E_F)); m = top; }
                const float at = m == PC_NEG_INF_F ? 0.0f : m, c = d.inv_T * PC_LOG2E_F;
                float part = 0.0f;
#pragma unroll
                for (int e = 0; e < kPacks * N; ++e) part += __builtin_amdgcn_exp2f((v[e] - at) * c);
                s += part;
            }
            auto below = [&](float a, float b) { return a == PC_NEG_INF_F ? 1.0f : exp2f((a - b) * (d.inv_T * PC_LOG2E_F)); };   // (s is 0, or NaN)
            float all = wave_all(m, max2);
            s = wave_all(s * below(m, all), add2);
            if (WAVES > 1) {
                __syncthreads();                       // the row before is read
                if (t % 64 == 0) { wave_m[t / 64] = all; wave_s[t / 64] = s; }
                __syncthreads();
                for (int w = 0; w < WAVES; ++w) all = max2(all, wave_m[w]);
                s = 0.0f;
                for (int w = 0; w < WAVES; ++w) s += wave_s[w] * below(wave_m[w], all);
            }
            m = s != s && all < __builtin_inff() ? s : all;   // a row with a NaN has no maximum, not even where all else is -inf
            log_s = logf(s);
        } else {
            m = 0.0f;
            look_up();
        }
        if (!listing) continue;
        float part = 0.0f;
#pragma unroll
        for (int i = 0; i < G::LIST; ++i)
            if (list.id[i] >= 0 && !(list.q[i] == 0.0f)) {
                const float v = listed[i];
                const float logp = d.normalised ? (v == __builtin_inff() ? __builtin_nanf("") : v) : m == PC_NEG_INF_F ? m : (v - m) * d.inv_T - log_s;
                part += list.q[i] * (list.logq[i] - logp);
            }
        part = G::list_all(part, lds, add2);
        if (t == 0) {
            loss[r] = part;
            stats[2 * r] = m;
            stats[2 * r + 1] = log_s;
        }
    }
}

// Gradient.  The listed categories' values are made first (from the row itself where the gradient replaces it), then the dense part is
// written in packs of the output's 16-byte grid, then, behind a barrier, the listed ones over it.  Bound by reading and writing (8192 x
// 50257: fp32 628 us, 16 bits 322, 5.1 to 5.2 TB/s).  Fetching the first packs before the list is made gained nothing.
template <typename TS, typename TT, int WAVES, bool LONG, bool STREAM>
__global__ __launch_bounds__((Group<WAVES, LONG>::BLOCK)) void k_distill_grad(const DistillDev d, const float *__restrict__ stats,
                                                                               const float *__restrict__ dloss, float scale, void *dstudent, int64_t out_ld)
{
    using G = Group<WAVES, LONG>;
    constexpr int N = Pack<TS>::N, TH = G::THREADS;
    __shared__ float lds[WAVES], shared_Q[G::ROWS];
    __shared__ int32_t ids[LONG ? PC_MAX_TOP : 1];
    __shared__ float qs[LONG ? PC_MAX_TOP : 1];
    const int t = threadIdx.x % TH, sub = threadIdx.x / TH;
    const bool listing = LONG || t < 64;
    for (int64_t r = (int64_t)blockIdx.x * G::ROWS + sub; r < d.rows; r += (int64_t)gridDim.x * G::ROWS) {
        const TS *z = (const TS *)d.student + r * d.student_ld;
        TS *out = (TS *)dstudent + r * out_ld;
        const float g = (dloss ? scale * dloss[r] : scale) * d.inv_T;
        const float m = stats[2 * r], log_s = stats[2 * r + 1], c = d.inv_T * PC_LOG2E_F;
        List<G, TT> list;
        float at[G::LIST], Q = 0.0f;
        if (listing) {
            list.fetch(d, r, t);
            list.probabilities(d, lds);
#pragma unroll
            for (int i = 0; i < G::LIST; ++i) {
                Q += list.q[i];
                at[i] = list.id[i] >= 0 && !d.normalised ? to_f32(z[list.id[i]]) : 0.0f;
            }
            Q = G::list_all(Q, lds, add2);
            if (LONG)
#pragma unroll
                for (int i = 0; i < G::LIST; ++i)
                    if (t + i * TH < d.top) { ids[t + i * TH] = list.id[i]; qs[t + i * TH] = list.q[i]; }
        }
        if (WAVES > 1) {
            if (t == 0) shared_Q[sub] = Q;
            __syncthreads();                           // also: the listed values are read before anything is written
            Q = shared_Q[sub];
        }
        const bool none = g == 0.0f || Q == 0.0f, zeros = none || d.normalised || m == PC_NEG_INF_F;
        const float f = g * (Q * expf(-log_s));
        auto dense = [&](float v) { return __builtin_amdgcn_exp2f((v - m) * c) * f; };
        if (listing && !none) {                        // a category listed more than once: its first entry writes for all
            bool again = LONG;                         // a short list is looked through for such categories first (lists of 64, 8192 x 50257 bf16
                                                       // 333 us against 373, 20000 x 1000 31 against 49; with doubled ones 55)
            if (!LONG) {
                const int32_t own = list.id[0] >= 0 ? list.id[0] : -1 - t;       // no two of those that are none are alike
                uint64_t others = 0;
#pragma unroll
                for (int k = 0; k < 64; ++k) {
                    if (k % 8 == 0 && k >= d.top) break;
                    others |= __ballot(own == __builtin_amdgcn_readlane(own, k)) & ~(1ull << k);
                }
                again = others != 0;
            }
#pragma unroll
            for (int i = 0; i < G::LIST; ++i) {
                const int j = t + i * TH;
                bool first = list.id[i] >= 0;
                float sum = list.q[i];
                if (again) {
                    sum = 0.0f;
#pragma unroll 4
                    for (int k = 0; k < d.top; ++k) {
                        const int32_t o = LONG ? ids[k] : __builtin_amdgcn_readlane(list.id[0], k);
                        const float oq = LONG ? qs[k] : __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(list.q[0]), k));
                        if (o == list.id[i]) { first = first && k >= j; sum += oq; }
                    }
                }
                at[i] = (zeros ? 0.0f : dense(at[i])) - g * sum;
                if (!first) list.id[i] = -1;
            }
        }
        const int off = elements_off(out);
        const TS *zg = z - off;                        // element i of the grid is category i - off
        TS *grid = out - off;
        const int64_t end = off + (int64_t)d.n_cats, p_first = off > 0, p_last = end / N;
        // past the caches where sixteen waves hasten through a row: lines that wait there are written back after the last one (100 x 50257 fp32
        // 12 us against 19, 8192 x 50257 bf16 325 against 331; with four waves 365 against 358)
        auto put = [&](int64_t p, const Pack<TS> &v) {
            pc_u32x4 *to = reinterpret_cast<pc_u32x4 *>(grid + p * N);
            if (WAVES == 16) __builtin_nontemporal_store(__builtin_bit_cast(pc_u32x4, v), to);
            else *to = __builtin_bit_cast(pc_u32x4, v);
        };
        const int64_t edge = edge_of<N>(t, off, end);
        if (zeros) {
            if (edge >= 0) grid[edge] = from_f32<TS>(0.0f);
            const float x[N] = {};
            for (int64_t p = p_first + t; p < p_last; p += TH) put(p, pack_f32<TS>(x));
        } else {
            if (edge >= 0) grid[edge] = from_f32<TS>(dense(to_f32(zg[edge])));
            auto step = [&](int64_t p0, auto some) {   // kPacks of which not all may be there
                Pack<TS> in[kPacks];
#pragma unroll
                for (int k = 0; k < kPacks; ++k) {
                    const int64_t p = p0 + t + k * TH;
                    const TS *from = zg + (some ? min(p, p_last - 1) : p) * N;
                    in[k] = STREAM ? stream_pack(from) : load_pack(from);
                }
#pragma unroll
                for (int k = 0; k < kPacks; ++k) {
                    const int64_t p = p0 + t + k * TH;
                    float x[N];
                    unpack_f32(in[k], x);
#pragma unroll
                    for (int e = 0; e < N; ++e) x[e] = dense(x[e]);
                    if (!some || p < p_last) put(p, pack_f32<TS>(x));
                }
            };
            int64_t p0 = p_first;
            for (; p0 + kPacks * TH <= p_last; p0 += kPacks * TH) step(p0, std::false_type{});
            if (p0 < p_last) step(p0, std::true_type{});
        }
        if (WAVES > 1) __syncthreads();
        else __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        if (listing && !none)
#pragma unroll
            for (int i = 0; i < G::LIST; ++i)
                if (list.id[i] >= 0) out[list.id[i]] = from_f32<TS>(at[i]);
        if (WAVES > 1) __syncthreads();                // LDS is read
    }
}

static pc_status check_distill(const pc_distill *d)
{
    if (!d) return fail(PC_ERR_ARG, "NULL argument");
    if (d->rows < 0) return fail(PC_ERR_ARG, "rows must not be negative");
    if (d->n_cats < 1) return fail(PC_ERR_ARG, "n_cats must be positive");
    if (d->top < 1 || d->top > PC_MAX_TOP) return fail(PC_ERR_ARG, "top must be in 1 .. PC_MAX_TOP");
    if (!type_known(d->student_type) || !type_known(d->teacher_type)) return fail(PC_ERR_ARG, "unknown element type");
    if (!(d->temperature > 0.0f) || std::isinf(d->temperature) || std::isinf(1.0f / d->temperature * PC_LOG2E_F))   // a factor of exponents
        return fail(PC_ERR_ARG, "temperature and log2(e) / temperature must be positive and finite");
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
// f(waves of a row, whether its list is long), as types: one wave where a row is at most 16 KB, four steps of a wave (one and four waves, us: loss of
// 20000 x 1000 bf16 25 and 78, of 8192 x 4096 fp32 28 and 33, gradient 65 and 59; of 8192 x 8192 fp32 50 and 48); sixteen where rows are
// fewer than `few` or of `large` bytes, else four (sixteen and four: loss of 100 x 50257 fp32 11.4 and 11.5, of 400 24 and 19, gradient of 100
// 12 and 23, of 400 39 and 43, of 800 x 32000 bf16 33 and 29; long rows are written faster when few of them are at work at a time: gradient of
// 8192 x 50257 bf16 325 and 358, of 8192 x 32000 fp32 363 and 427, bf16 224 and 218).
// Rows of 256 MB and more together, which no cache holds until they are read again, are read past the caches by the widest waves that such
// numbers come to: loss of 8192 x 50257 fp32 247 us against 272, 16 bits 137 and 148, gradient 628 and 637, 322 and 332; of 333 x 32003 fp16 18 and 15.
struct RowRule { int64_t few, large; bool stream_four, stream_sixteen; };
struct LossRule { static constexpr RowRule value = {128, INT64_MAX, true, false}; };
struct GradRule { static constexpr RowRule value = {512, 96 << 10, false, true}; };
template <typename Rule, typename F>
static void with_group(const pc_distill *d, Rule, F f)
{
    constexpr RowRule rule = Rule::value;
    const int64_t bytes = d->n_cats * type_bytes(d->student_type);
    const bool streams = d->rows * bytes >= 256 << 20;
    if (d->top > kShortList) f(Group<4, true>{});
    else if (bytes <= 16384) f(Group<1, false>{});
    else if (d->rows < rule.few || bytes >= rule.large) {
        if (rule.stream_sixteen && streams) f(Group<16, false, rule.stream_sixteen>{});
        else f(Group<16, false>{});
    } else {
        if (rule.stream_four && streams) f(Group<4, false, rule.stream_four>{});
        else f(Group<4, false>{});
    }
}
template <typename G>
static dim3 row_grid(int64_t rows) { return dim3((unsigned)std::min<int64_t>((rows + G::ROWS - 1) / G::ROWS, 1 << 20)); }

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

pc_status pc_distill_forward(const pc_distill *d, void *, size_t, float *loss, float *stats, void *stream)
{
    const pc_status st = check_distill(d);
    if (st != PC_OK || d->rows == 0) return st;
    if (!loss || !stats) return fail(PC_ERR_ARG, "NULL argument");
    if (!aligned_to(loss, 4) || !aligned_to(stats, 4)) return fail(PC_ERR_ARG, "loss and stats must be 4-byte aligned");
    const DistillDev dev = distill_dev(d);
    with_type(d->student_type, [&](auto s) {
        with_type(d->teacher_type, [&](auto t) {
            with_group(d, LossRule{}, [&](auto g) {
                using G = decltype(g);
                hipLaunchKernelGGL((k_distill_rows<decltype(s), decltype(t), G::THREADS / 64, (G::LIST > 1), G::STREAMS>), row_grid<G>(d->rows), dim3(G::BLOCK), 0,
                                   (hipStream_t)stream, dev, loss, stats);
            });
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
    if (overlap(d->student, span_bytes(d->rows, d->student_ld, d->n_cats, e), dstudent, span_bytes(d->rows, dstudent_ld, d->n_cats, e)) &&
        !(d->student == dstudent && d->student_ld == dstudent_ld))
        return fail(PC_ERR_ARG, "dstudent overlaps the student's rows without being them");
    const DistillDev dev = distill_dev(d);
    with_type(d->student_type, [&](auto s) {
        with_type(d->teacher_type, [&](auto t) {
            with_group(d, GradRule{}, [&](auto g) {
                using G = decltype(g);
                hipLaunchKernelGGL((k_distill_grad<decltype(s), decltype(t), G::THREADS / 64, (G::LIST > 1), G::STREAMS>), row_grid<G>(d->rows), dim3(G::BLOCK), 0,
                                   (hipStream_t)stream, dev, stats, dloss, scale, dstudent, dstudent_ld);
            });
        });
    });
    return launched();
}

}  // extern "C"
