// Predictive distribution of one variable from the weights of its input nodes, and the flows of its tables.
//   p[b][c] = sum over blocks j, nodes k of  W[rows[j] + k][b] * T[table[j]][c][k]          (a product of H = n_blocks * K states)
//   flow[t][c][k] = T[t][c][k] * sum over b (and the blocks j of table t) of  W[rows[j] + k][b] * g[b][c] / p[b][c]
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "pc_internal.h"
#include "pc_rows.h"

namespace pc {

// Block j of a mixture: its first row of weights and its table; -1 where either lies outside.
struct MixBlock { int64_t row; int32_t table; };
__device__ inline MixBlock mix_block(const pc_mixture &m, int j)
{
    const int64_t row = m.rows ? m.rows[j] : (int64_t)j * m.K;
    const int32_t table = m.table ? m.table[j] : j;
    const bool ok = row >= 0 && row + m.K <= m.n_rows && table >= 0 && table < m.n_tables;
    return ok ? MixBlock{row, table} : MixBlock{-1, -1};
}

constexpr float kLogFltMin = -87.33654475f;           // log FLT_MIN

// 64 categories x 64 samples a workgroup, 4 x 4 sums a thread, the states in steps of 16 through LDS.  Any K.
__global__ __launch_bounds__(256) void k_predict_any(const pc_mixture m, const float *__restrict__ tables, int32_t B,
                                                     float *__restrict__ logp, int64_t ld)
{
    __shared__ float ts[16][68], ws[16][68];
    const int c0 = blockIdx.x * 64, b0 = blockIdx.y * 64, tc = threadIdx.x % 16 * 4, tb = threadIdx.x / 16 * 4;
    const int H = m.n_blocks * m.K;
    float acc[4][4] = {};
    for (int n0 = 0; n0 < H; n0 += 16) {
        {
            const int n = n0 + threadIdx.x % 16;
            const MixBlock blk = n < H ? mix_block(m, n / m.K) : MixBlock{-1, -1};
            const float *src = tables + (int64_t)blk.table * m.n_cats * m.K + n % m.K;
            for (int i = 0; i < 4; ++i) {
                const int c = threadIdx.x / 16 + 16 * i;
                ts[threadIdx.x % 16][c] = blk.row >= 0 && c0 + c < m.n_cats ? src[(int64_t)(c0 + c) * m.K] : 0.0f;
            }
        }
        for (int i = 0; i < 4; ++i) {
            const int n = n0 + threadIdx.x / 64 + 4 * i, b = threadIdx.x % 64;
            const MixBlock blk = n < H ? mix_block(m, n / m.K) : MixBlock{-1, -1};
            ws[threadIdx.x / 64 + 4 * i][b] = blk.row >= 0 && b0 + b < B ? m.weights[(blk.row + n % m.K) * m.stride + b0 + b] : 0.0f;
        }
        __syncthreads();
        for (int n = 0; n < 16; ++n)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] += ws[n][tb + i] * ts[n][tc + j];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
            if (b0 + tb + i < B && c0 + tc + j < m.n_cats) {
                const float p = acc[i][j];
                logp[(int64_t)(b0 + tb + i) * ld + c0 + tc + j] = p < __FLT_MIN__ ? PC_NEG_INF_F : logf(p);
            }
}

// ---- matrix-core kernels: K a multiple of 4 ----
// Operands are fp32; the matrix cores multiply bf16 and add in fp32.  An operand x is taken as a sum of bf16 planes, each the rounding of
// what the planes before it leave: hi + lo keeps 2^-16 of x, hi + mid + lo 2^-24.  Weights (and tables) are scaled by 2^24 on the way, so that the
// lower planes of numbers down to FLT_MIN are normal numbers; the scale is taken out of the fp32 sum, exactly.
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
constexpr float kUp = 16777216.0f, kDown = 1.0f / kUp;

__device__ inline uint32_t round2(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){a, b}, bf16x2)); }
__device__ inline float low_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float high_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// PLANES planes of eight numbers, 16 bytes each
template <int PLANES>
__device__ inline void split8(const float (&x)[8], uint4 (&plane)[PLANES])
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i];
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = round2(v[2 * i], v[2 * i + 1]);
            if (p + 1 < PLANES) { v[2 * i] -= low_of(w[i]); v[2 * i + 1] -= high_of(w[i]); }
        }
        plane[p] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ inline floatx16 mfma(const uint4 &a, const uint4 &b, const floatx16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Predictive distribution.  A wave owns 32 categories x 32 NT samples; a workgroup WAVES * 32 categories of the same samples.  States come
// in chunks of KC: each lane fetches its category's table row (8 contiguous states a step of 16, split in registers, read once from
// memory), the workgroup stages the weights [states][samples] into LDS as planes in operand order, both one chunk ahead, one barrier a chunk.
// Products hi*hi + hi*lo + lo*hi.  The samples are the instruction's rows, so that a store covers 32 neighbouring categories.
// Where a group of four states begins in the tables and in the weights is looked up in LDS, a window of states at a time: blocks need not be
// as long as a chunk.
constexpr int kWindow = 2048;
template <int NT, int WAVES, int KC>
__global__ __launch_bounds__(64 * WAVES, NT == 8 ? 2 : 3) void k_predict(const pc_mixture m, const float *__restrict__ tables, int32_t B,
                                                                        float *__restrict__ logp, int64_t ld)
{
    constexpr int TH = 64 * WAVES, NB = 32 * NT, STEPS = KC / 16, TASKS = NB * KC / 8, FT = (TASKS + TH - 1) / TH;
    __shared__ uint4 planes[2][2][KC / 8][NB];        // [buffer][hi, lo][8 states][sample]
    __shared__ int64_t t_at[kWindow / 4], w_at[kWindow / 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int H = m.n_blocks * m.K, c0 = (blockIdx.x * WAVES + wave) * 32, b0 = blockIdx.y * NB;
    const int64_t mine = (int64_t)min(c0 + col, m.n_cats - 1) * m.K;     // a category behind the last reads that one's row again
    floatx16 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] = 0.0f;

    auto fill_window = [&](int n0) {
        for (int i = threadIdx.x; i < kWindow / 4; i += TH) {
            const int n = n0 + 4 * i;
            int64_t t = -1, w = -1;
            if (n < H) {
                const MixBlock blk = mix_block(m, n / m.K);
                if (blk.row >= 0) { t = (int64_t)blk.table * m.n_cats * m.K + n % m.K; w = (blk.row + n % m.K) * m.stride; }
            }
            t_at[i] = t;
            w_at[i] = w;
        }
    };
    float4 t_raw[STEPS][2];
    float w_raw[FT][8];
    auto fetch = [&](int n0) {                         // n0: first state of the chunk
        const int g0 = n0 % kWindow / 4;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int64_t at = t_at[g0 + 4 * s + 2 * half + q];
                const float4 v = *reinterpret_cast<const float4 *>(tables + (at >= 0 ? at + mine : 0));
                t_raw[s][q] = at >= 0 ? v : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
        for (int f = 0; f < FT; ++f) {
            const int task = threadIdx.x + f * TH, b = task % NB, g = task / NB;
            const bool on = (TASKS % TH == 0 || task < TASKS) && b0 + b < B;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int64_t at = on ? w_at[g0 + 2 * g + q] : -1;
#pragma unroll
                for (int i = 0; i < 4; ++i) w_raw[f][4 * q + i] = at >= 0 ? m.weights[at + i * m.stride + b0 + b] : 0.0f;
            }
        }
    };

    fill_window(0);
    __syncthreads();
    fetch(0);
    for (int n0 = 0, buf = 0; n0 < H; n0 += KC, buf ^= 1) {
#pragma unroll
        for (int f = 0; f < FT; ++f) {
            const int task = threadIdx.x + f * TH;
            if (TASKS % TH != 0 && task >= TASKS) break;
            float x[8];
            uint4 pl[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = w_raw[f][i] * kUp;
            split8(x, pl);
            planes[buf][0][task / NB][task % NB] = pl[0];
            planes[buf][1][task / NB][task % NB] = pl[1];
        }
        uint4 th[STEPS], tl[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const float4 u = t_raw[s][0], v = t_raw[s][1];
            const float x[8] = {u.x * kUp, u.y * kUp, u.z * kUp, u.w * kUp, v.x * kUp, v.y * kUp, v.z * kUp, v.w * kUp};
            uint4 pl[2];
            split8(x, pl);
            th[s] = pl[0];
            tl[s] = pl[1];
        }
        __syncthreads();                               // the chunk's planes are there, and everyone has read the window for it
        const int next = n0 + KC;
        if (next < H) {
            if (next % kWindow == 0) { fill_window(next); __syncthreads(); }
            fetch(next);
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint4 wh = planes[buf][0][2 * s + half][32 * t + col], wl = planes[buf][1][2 * s + half][32 * t + col];
                acc[t] = mfma(wl, th[s], acc[t]);
                acc[t] = mfma(wh, tl[s], acc[t]);
                acc[t] = mfma(wh, th[s], acc[t]);
            }
    }
    if (c0 + col >= m.n_cats) return;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int b = b0 + 32 * t + 8 * (e / 4) + 4 * half + e % 4;
            const float p = acc[t][e] * (kDown * kDown);
            if (b < B) logp[(int64_t)b * ld + c0 + col] = p < __FLT_MIN__ ? PC_NEG_INF_F : logf(p);
        }
}

// g / p of one sample and category; p = 0 adds nothing
__device__ inline float flow_ratio(float logp, float g) { return logp < kLogFltMin - 1e-3f ? 0.0f : g * expf(-logp); }

// 64 categories x 64 nodes of a table a workgroup, the samples of all blocks of that table in steps of 16.  The table's first
// block does the work, so that each entry has one writer.  Any K.
__global__ __launch_bounds__(256) void k_predict_flow_any(const pc_mixture m, const float *__restrict__ tables, int32_t B,
                                                          const float *__restrict__ logp, int64_t lp_ld, const float *__restrict__ dlogp,
                                                          int64_t dl_ld, float scale, int32_t accumulate, float *__restrict__ flow)
{
    __shared__ float rs[16][68], ws[16][68];
    const int k_tiles = (m.K + 63) / 64;
    const int c0 = blockIdx.x * 64, j0 = blockIdx.y / k_tiles, k0 = blockIdx.y % k_tiles * 64;
    const int tk = threadIdx.x % 16 * 4, tc = threadIdx.x / 16 * 4;
    const MixBlock mine = mix_block(m, j0);
    if (mine.row < 0) return;
    for (int j = 0; j < j0; ++j)
        if (mix_block(m, j).table == mine.table) return;
    float acc[4][4] = {};
    for (int j = j0; j < m.n_blocks; ++j) {
        const MixBlock blk = mix_block(m, j);
        if (blk.table != mine.table) continue;
        for (int b0 = 0; b0 < B; b0 += 16) {
            for (int i = 0; i < 4; ++i) {
                const int b = threadIdx.x / 64 + 4 * i, c = threadIdx.x % 64;
                const bool on = b0 + b < B && c0 + c < m.n_cats;
                rs[b][c] = on ? flow_ratio(logp[(int64_t)(b0 + b) * lp_ld + c0 + c], dlogp[(int64_t)(b0 + b) * dl_ld + c0 + c]) : 0.0f;
            }
            for (int i = 0; i < 4; ++i) {
                const int b = threadIdx.x % 16, k = threadIdx.x / 16 + 16 * i;
                ws[b][k] = b0 + b < B && k0 + k < m.K ? m.weights[(blk.row + k0 + k) * m.stride + b0 + b] : 0.0f;
            }
            __syncthreads();
            for (int b = 0; b < 16; ++b)
                for (int i = 0; i < 4; ++i)
                    for (int k = 0; k < 4; ++k) acc[i][k] += rs[b][tc + i] * ws[b][tk + k];
            __syncthreads();
        }
    }
    for (int i = 0; i < 4; ++i)
        for (int k = 0; k < 4; ++k)
            if (c0 + tc + i < m.n_cats && k0 + tk + k < m.K) {
                const int64_t at = ((int64_t)mine.table * m.n_cats + c0 + tc + i) * m.K + k0 + tk + k;
                const float v = scale * (tables[at] * acc[i][k]);
                flow[at] = accumulate ? flow[at] + v : v;
            }
}

// Samples a wave: as many of 256 as there are, so that the tables are read once; fewer where that leaves a SIMD without a wave (the
// tables of few categories stay in the caches).
static void launch_predict(const pc_mixture &m, const float *tables, int32_t B, float *logp, int64_t ld, hipStream_t s)
{
    const int64_t rows = (m.n_cats + 31ll) / 32;
    int nt = B > 128 ? 8 : B > 64 ? 4 : B > 32 ? 2 : 1;
    while (nt > 1 && rows * ((B + 32 * nt - 1) / (32 * nt)) < 1024) nt /= 2;
#define PC_PREDICT(NT, WAVES, KC)                                                                                              \
    if (nt == NT)                                                                                                              \
        hipLaunchKernelGGL((k_predict<NT, WAVES, KC>), dim3((unsigned)((rows + WAVES - 1) / WAVES), (unsigned)((B + 32 * NT - 1) / (32 * NT))), \
                           dim3(64 * WAVES), 0, s, m, tables, B, logp, ld)
    PC_PREDICT(8, 8, 32);
    PC_PREDICT(4, 4, 32);
    PC_PREDICT(2, 4, 64);
    PC_PREDICT(1, 4, 64);
#undef PC_PREDICT
}

static pc_status check_mixture(const pc_mixture *m, const float *tables, int32_t B)
{
    if (!m || !tables || !m->weights) return fail(PC_ERR_ARG, "NULL argument");
    if (m->K < 1 || m->K > 128) return fail(PC_ERR_ARG, "K must be in 1 .. 128");
    if (m->n_blocks < 1 || m->n_cats < 1 || m->n_tables < 1 || m->n_rows < 1)
        return fail(PC_ERR_ARG, "n_blocks, n_cats, n_tables and n_rows must be positive");
    if (B < 1) return fail(PC_ERR_ARG, "B must be positive");
    if (B > PC_MAX_BATCH) return fail(PC_ERR_TOO_LARGE, "more than PC_MAX_BATCH samples in one call");
    if (m->stride < B) return fail(PC_ERR_ARG, "stride is smaller than B");
    if ((int64_t)m->n_blocks * m->K > 1 << 30) return fail(PC_ERR_TOO_LARGE, "more than 2^30 states");
    if (m->n_cats > 1 << 29) return fail(PC_ERR_TOO_LARGE, "more than 2^29 categories");        // a grid has fewer than 2^32 threads along x
    if (!m->rows && (int64_t)m->n_blocks * m->K > m->n_rows) return fail(PC_ERR_ARG, "weights have fewer than n_blocks * K rows");
    if (!m->table && m->n_blocks > m->n_tables) return fail(PC_ERR_ARG, "fewer tables than blocks");
    if (!aligned_to(tables, 16)) return fail(PC_ERR_ARG, "tables must be 16-byte aligned");
    if (!aligned_to(m->weights, 4) || !aligned_to(m->rows, 4) || !aligned_to(m->table, 4))
        return fail(PC_ERR_ARG, "weights, rows and table must be 4-byte aligned");
    return PC_OK;
}

}  // namespace pc

using namespace pc;

extern "C" {

pc_status pc_predict(const pc_mixture *m, const float *tables, int32_t B, float *logp, int64_t ld, void *stream)
{
    const pc_status st = check_mixture(m, tables, B);
    if (st != PC_OK) return st;
    if (!logp) return fail(PC_ERR_ARG, "NULL argument");
    if (ld < m->n_cats) return fail(PC_ERR_ARG, "ld is smaller than n_cats");
    if (!aligned_to(logp, 4)) return fail(PC_ERR_ARG, "logp must be 4-byte aligned");
    if (m->K % 4 == 0) {
        launch_predict(*m, tables, B, logp, ld, (hipStream_t)stream);
        return launched();
    }
    const dim3 grid((unsigned)((m->n_cats + 63ll) / 64), (unsigned)((B + 63) / 64));
    hipLaunchKernelGGL(k_predict_any, grid, dim3(256), 0, (hipStream_t)stream, *m, tables, B, logp, ld);
    return launched();
}

pc_status pc_predict_backward(const pc_mixture *m, const float *tables, int32_t B, const float *logp, int64_t logp_ld,
                              const float *dlogp, int64_t dlogp_ld, float scale, int32_t accumulate, float *table_flow, void *stream)
{
    const pc_status st = check_mixture(m, tables, B);
    if (st != PC_OK) return st;
    if (!logp || !dlogp || !table_flow) return fail(PC_ERR_ARG, "NULL argument");
    if (logp_ld < m->n_cats || dlogp_ld < m->n_cats) return fail(PC_ERR_ARG, "ld is smaller than n_cats");
    if (!aligned_to(logp, 4) || !aligned_to(dlogp, 4)) return fail(PC_ERR_ARG, "logp and dlogp must be 4-byte aligned");
    if (!aligned_to(table_flow, 16)) return fail(PC_ERR_ARG, "table_flow must be 16-byte aligned");
    const int64_t rows = (int64_t)m->n_blocks * ((m->K + 63) / 64);
    if (rows > 65535) return fail(PC_ERR_TOO_LARGE, "more than 65535 blocks in a mixture");
    const dim3 grid((unsigned)((m->n_cats + 63ll) / 64), (unsigned)rows);
    hipLaunchKernelGGL(k_predict_flow_any, grid, dim3(256), 0, (hipStream_t)stream, *m, tables, B, logp, logp_ld, dlogp, dlogp_ld, scale,
                       accumulate, table_flow);
    return launched();
}

}  // extern "C"
