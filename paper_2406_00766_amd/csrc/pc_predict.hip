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

static pc_status check_mixture(const pc_mixture *m, const float *tables, int32_t B)
{
    if (!m || !tables || !m->weights) return fail(PC_ERR_ARG, "NULL argument");
    if (m->K < 1 || m->K > 128) return fail(PC_ERR_ARG, "K must be in 1 .. 128");
    if (m->n_blocks < 1 || m->n_cats < 1 || m->n_tables < 1 || m->n_rows < 1)
        return fail(PC_ERR_ARG, "n_blocks, n_cats, n_tables and n_rows must be positive");
    if (B < 1) return fail(PC_ERR_ARG, "B must be positive");
    if (B > PC_MAX_BATCH) return fail(PC_ERR_TOO_LARGE, "more than PC_MAX_BATCH samples in one call");
    if (m->stride < B) return fail(PC_ERR_ARG, "stride is smaller than B");
    if ((int64_t)m->n_blocks * m->K > INT32_MAX) return fail(PC_ERR_TOO_LARGE, "more than 2^31 - 1 states");
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
