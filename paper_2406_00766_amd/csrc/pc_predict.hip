// Predictive distribution of one variable from the weights of its input nodes, and the flows of its tables.
//   p[b][c] = sum over blocks j, nodes k of  W[rows[j] + k][b] * T[table[j]][c][k]          (a product of H = n_blocks * K states)
//   flow[t][c][k] = T[t][c][k] * sum over b (and the blocks j of table t) of  W[rows[j] + k][b] * g[b][c] / p[b][c]
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

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
__device__ inline float log_p(float p) { return p < __FLT_MIN__ ? PC_NEG_INF_F : logf(p); }

// K below 4.  64 categories x 64 samples a workgroup, 4 x 4 sums a thread, the states in steps of 16 through LDS.
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
            if (b0 + tb + i < B && c0 + tc + j < m.n_cats) logp[(int64_t)(b0 + tb + i) * ld + c0 + tc + j] = log_p(acc[i][j]);
}

// ---- matrix-core kernels: K of at least 4 ----
// States come in groups of four that begin where 16 bytes of a block can be read: a block's last group is its last four states, and where K is
// no multiple of 4 the `skip` weights that the group before has counted are taken as zero.
__device__ inline int group_states(int K) { return (K + 3) & ~3; }      // of a block, with those repeated
__device__ inline int group_start(int K, int k) { return min(k, K - 4); }

// Operands are fp32; the matrix cores multiply bf16 and add in fp32.  An operand x is taken as a sum of three bf16 planes, each the rounding of
// what the planes before it leave: together they keep 2^-24 of x.  Of the products of planes the six down to 2^-16 are added up, those left out are
// 2^-24 of the whole.  (Two planes and three products take half the time of the matrix cores and lose up to 3 * 2^-16 of a product.  Over many states that
// averages out; where one state carries a sample, as the likely categories of a trained model have it, a logarithm near 0 would keep five digits.)
// Weights (and tables) are scaled by 2^24 on the way, so that the lower planes of numbers down to FLT_MIN are normal numbers; the scale is taken
// out of the fp32 sum, exactly.
constexpr int kPlanes = 3;
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
constexpr float kUp = 16777216.0f, kDown = 1.0f / kUp;

__device__ inline uint32_t round2(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){a, b}, bf16x2)); }
__device__ inline float low_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float high_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// the planes of eight numbers, 16 bytes each
__device__ inline void split8(const float (&x)[8], uint4 (&plane)[kPlanes])
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i];
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = round2(v[2 * i], v[2 * i + 1]);
            if (p + 1 < kPlanes) { v[2 * i] -= low_of(w[i]); v[2 * i + 1] -= high_of(w[i]); }
        }
        plane[p] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ inline floatx16 mfma(const uint4 &a, const uint4 &b, const floatx16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Predictive distribution.  A wave owns 32 categories x 32 NT samples and, of each chunk of KC * SPLIT states, its KC: with SPLIT > 1 (few
// samples: waves with little to add up, bound by loads in flight) SPLIT waves of a workgroup share categories and add their sums at the end.
// Each lane fetches its category's table row (8 contiguous states a step of 16, split in registers, read once from memory); the workgroup
// stages the weights [states][samples] into LDS as planes in operand order.  While a chunk is multiplied the next one is split and staged
// and the one after it is on its way; one barrier a chunk.
// The samples are the instruction's rows, so that a store covers 32 neighbouring categories.  Bound by reading the tables and splitting them up to some
// 64 samples (4096 states x 50257: B = 16 215 us, 3.8 TB/s; B = 64 238), then by the matrix cores (B = 128 331 us; B = 256 545: 1160 TFLOP/s of
// bf16 products, six to a product; a large bf16 product reaches 1450.  Both once the clock has settled: of a row of calls the first 30 take up to 770).
// Waves of 128 samples and more (READY) find the weights' planes ready: every workgroup splitting them anew took 364 us at B = 128, 569 at B = 256.
// A workgroup adds up `len` states from blockIdx.z * len on; several parts: the sums go to `sums` and k_predict_join takes the logarithm.
// Where a group of four states begins in the tables and in the weights is looked up in LDS, a window of states at a time, so that
// blocks need not be as long as a chunk; WHOLE: they are multiples of KC, one look-up serves a wave's part.
constexpr int kWindow = 2048;
template <int NT, int WAVES, int SPLIT, int KC, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES, 2) void k_predict(const pc_mixture m, const float *__restrict__ tables, int32_t B,
                                                                        float *__restrict__ logp, int64_t ld, int32_t len, float *__restrict__ sums, const pc_u32x4 *__restrict__ ready)
{
    constexpr bool READY = NT >= 4;
    constexpr int TH = 64 * WAVES, NB = 32 * NT, STEPS = KC / 16, KW = KC * SPLIT, TASKS = NB * KW / 8, FT = (TASKS + TH - 1) / TH;
    __shared__ uint4 planes[2][kPlanes][KW / 8][NB];   // [buffer][plane][8 states][sample]
    __shared__ int64_t t_at[kWindow / 4], w_at[kWindow / 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5, part = wave % SPLIT;
    const int Kg = group_states(m.K), first = blockIdx.z * len, H = min(m.n_blocks * Kg - first, len), c0 = (blockIdx.x * (WAVES / SPLIT) + wave / SPLIT) * 32, b0 = blockIdx.y * NB;
    const int64_t mine = (int64_t)min(c0 + col, m.n_cats - 1) * m.K;     // a category behind the last reads that one's row again
    const int here = min(NB, B - b0);                  // samples of this workgroup
    floatx16 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] = 0.0f;
    // A thread's eight weights of a chunk: sample, group of eight states.  Of 32 columns only those with a sample are staged, -1: none.
    int task_b[FT], task_g[FT];
    bool wave_stages[FT];                              // the same for all lanes: some lane has weights to stage
#pragma unroll
    for (int f = 0; f < FT; ++f) {
        const int task = threadIdx.x + f * TH, width = NT == 1 ? here : NB;
        task_b[f] = task % width;
        task_g[f] = NT > 1 || task / width < KW / 8 ? task / width : -1;
        wave_stages[f] = NT > 1 || __builtin_amdgcn_readfirstlane(__ballot(task_g[f] >= 0) != 0);
    }
    static_assert(NT == 1 || TASKS % TH == 0, "every thread has FT tasks");

    auto fill_window = [&](int n0) {
        for (int i = threadIdx.x; i < kWindow / 4; i += TH) {
            const int n = first + n0 + 4 * i;
            const MixBlock blk = n0 + 4 * i < H ? mix_block(m, n / Kg) : MixBlock{-1, -1};
            const int k = group_start(m.K, n % Kg);
            t_at[i] = blk.row >= 0 ? (int64_t)blk.table * m.n_cats * m.K + k : -1;
            w_at[i] = blk.row >= 0 ? (blk.row + k) * m.stride * 4 + (n % Kg - k) : -1;      // and how many to skip
        }
    };
    // What lies outside (blocks left out, states behind the last, samples behind B) is read from a place that exists and masked when it is
    // split.  A chunk behind the last state is fetched and staged like any other, and not used.
    Pack<float> t_raw[STEPS][2];
    float w_raw[READY ? 1 : FT][8];
    pc_u32x4 w_ready[READY ? FT : 1][kPlanes];
    const int columns = gridDim.y * NB, groups = (m.n_blocks * Kg + 7) / 8;
    uint32_t t_mask[WHOLE ? 1 : STEPS][2];
    int w_skip[FT][2];                                 // 4: all
    auto fetch_weights = [&](int n0, int f) {
        if (READY) {
            const int g = min((first + n0) / 8 + task_g[f], groups - 1);
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) w_ready[f][p] = (ready + ((int64_t)p * groups + g) * columns)[b0 + task_b[f]];
            return;
        }          // of the chunk that begins with state `first` + n0
        const int g0 = n0 % kWindow / 4;
        if (!wave_stages[f]) return;
        const int b = min(task_b[f], here - 1);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int64_t at = task_g[f] >= 0 && task_b[f] < here ? w_at[g0 + 2 * task_g[f] + q] : -1;
            const float *src = m.weights + (at >= 0 ? at >> 2 : 0) + b0 + b;
            w_skip[f][q] = at >= 0 ? (int)at & 3 : 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) w_raw[f][4 * q + i] = src[i * m.stride];
        }
    };
    auto fetch_tables = [&](int n0) {
        const int g0 = n0 % kWindow / 4;
        if (WHOLE) {
            const int64_t v = t_at[g0 + part * (KC / 4)];
            const int64_t at = (int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
            const float *src = tables + (at >= 0 ? at : 0) + (mine + 8 * half);
            t_mask[0][0] = at >= 0 ? ~0u : 0u;
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int q = 0; q < 2; ++q) t_raw[s][q] = load_pack(src + 16 * s + 4 * q);
        } else {
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int64_t at = t_at[g0 + part * (KC / 4) + 4 * s + 2 * half + q];
                    t_mask[s][q] = at >= 0 ? ~0u : 0u;
                    t_raw[s][q] = load_pack(tables + (at >= 0 ? at : 0) + mine);
                }
        }
    };
    auto masked = [](float v, uint32_t mask) { return __uint_as_float(__float_as_uint(v) & mask) * kUp; };
    auto stage_weights = [&](int buf, int f) {
        if (READY) {
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) planes[buf][p][task_g[f]][task_b[f]] = __builtin_bit_cast(uint4, w_ready[f][p]);
            return;
        }
        if (!wave_stages[f]) return;
        float x[8];
        uint4 pl[kPlanes];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i % 4 >= w_skip[f][i / 4] ? w_raw[f][i] * kUp : 0.0f;
        split8(x, pl);
        if (NT > 1 || task_g[f] >= 0)
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) planes[buf][p][task_g[f]][task_b[f]] = pl[p];
    };
    uint4 tp[STEPS][kPlanes];
    auto split_tables = [&](int s) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = masked(t_raw[s][i / 4].v[i % 4], t_mask[WHOLE ? 0 : s][WHOLE ? 0 : i / 4]);
        split8(x, tp[s]);
    };

    if (NT == 1 && here < NB)                          // columns without a sample stay zero
        for (int i = threadIdx.x; i < (int)(sizeof(planes) / 16); i += TH) (&planes[0][0][0][0])[i] = make_uint4(0, 0, 0, 0);
    fill_window(0);
    __syncthreads();
#pragma unroll
    for (int f = 0; f < FT; ++f) fetch_weights(0, f);
    fetch_tables(0);
#pragma unroll
    for (int f = 0; f < FT; ++f) { stage_weights(0, f); if (NT > 1 || KW < H) fetch_weights(KW, f); }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) split_tables(s);
    if (NT > 1 || KW < H) fetch_tables(KW);
    __syncthreads();
    // An iteration is STEPS * NT / G slices of 3 G products, among which the work for the next chunk is dealt out: the two waves of a SIMD
    // then find something for the vector ALU while the other one's products run.
    constexpr int G = NT > 1 ? 2 : 1, SLICES = STEPS * NT / G;
    for (int n0 = 0, buf = 0; n0 < H; n0 += KW, buf ^= 1) {
        const int next = n0 + 2 * KW;
        if (next % kWindow == 0) { fill_window(next); __syncthreads(); }                   // the barrier before: all have read the last one
        uint4 cp[STEPS][kPlanes], wp[2][G][kPlanes];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) cp[s][p] = tp[s][p];
        auto operands = [&](int slice) {
            const int s = slice / (NT / G), t = slice % (NT / G) * G;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int p = 0; p < kPlanes; ++p) wp[slice & 1][g][p] = planes[buf][p][part * (KC / 8) + 2 * s + half][32 * (t + g) + col];
        };
        auto tables_on = [&]() {
#pragma unroll
            for (int q = 0; q < STEPS; ++q) split_tables(q);
            fetch_tables(next);
        };
        if (NT == 1 && n0 + KW < H) {                  // bound by the loads: they leave first
#pragma unroll
            for (int f = 0; f < FT; ++f) { stage_weights(buf ^ 1, f); fetch_weights(next, f); }
            tables_on();
        }
        operands(0);
#pragma unroll
        for (int slice = 0; slice < SLICES; ++slice) {
            const int s = slice / (NT / G), t = slice % (NT / G) * G, o = slice & 1;
            if (slice + 1 < SLICES) operands(slice + 1);
#pragma unroll
            for (int sum = kPlanes - 1; sum >= 0; --sum)  // the small products first
#pragma unroll
                for (int p = sum; p >= 0; --p)
#pragma unroll
                    for (int g = 0; g < G; ++g) acc[t + g] = mfma(wp[o][g][p], cp[s][sum - p], acc[t + g]);
            if (NT > 1) {
#pragma unroll
                for (int f = 0; f < FT; ++f)
                    if (f * SLICES / FT == slice) { stage_weights(buf ^ 1, f); fetch_weights(next, f); }
                if (slice == SLICES - 1) tables_on();
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();
    }
    static_assert(kWindow % KW == 0 && kWindow >= 4 * KW, "a chunk lies in one window, the first two in the first");
    if (SPLIT > 1) {                                   // sums of the other parts, half of them at a time, through the planes' memory
        float *sums = reinterpret_cast<float *>(&planes[0][0][0][0]);
        static_assert(SPLIT == 1 || (NT == 1 && sizeof(planes) >= WAVES / 2 * 16 * 64 * 4), "half the waves' sums fit");
#pragma unroll
        for (int h = SPLIT / 2; h > 0; h /= 2) {
            float *slot = sums + (wave / SPLIT * h + part % h) * 16 * 64 + lane;
            if (part >= h && part < 2 * h)
#pragma unroll
                for (int e = 0; e < 16; ++e) slot[e * 64] = acc[0][e];
            __syncthreads();
            if (part < h)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[0][e] += slot[e * 64];
            __syncthreads();
        }
        if (part != 0) return;
    }
    if (c0 + col >= m.n_cats) return;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int b = b0 + 32 * t + 8 * (e / 4) + 4 * half + e % 4;
            const float p = acc[t][e] * (kDown * kDown);
            if (b < B) {
                if (sums) sums[(blockIdx.z * (int64_t)B + b) * m.n_cats + c0 + col] = p;
                else logp[(int64_t)b * ld + c0 + col] = log_p(p);
            }
        }
}

// The weights as planes in operand order, ready[plane][8 states][sample]: what k_predict with wide waves stages as it is.
__global__ __launch_bounds__(256) void k_predict_ready(const pc_mixture m, int32_t B, int32_t columns, uint4 *__restrict__ ready)
{
    const int Kg = group_states(m.K), groups = (m.n_blocks * Kg + 7) / 8, b = blockIdx.y * 64 + threadIdx.x % 64, g = blockIdx.x * 4 + threadIdx.x / 64;
    if (g >= groups || b >= columns) return;
    float x[8];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int n = 8 * g + 4 * q;
        const MixBlock blk = b < B && n < m.n_blocks * Kg ? mix_block(m, n / Kg) : MixBlock{-1, -1};
        const int k = group_start(m.K, n % Kg), skip = blk.row >= 0 ? n % Kg - k : 4;
        const float *src = m.weights + (blk.row >= 0 ? (blk.row + k) * m.stride + b : 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v = src[blk.row >= 0 ? i * m.stride : 0];
            x[4 * q + i] = i >= skip ? v * kUp : 0.0f;
        }
    }
    uint4 pl[kPlanes];
    split8(x, pl);
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) ready[((int64_t)p * groups + g) * columns + b] = pl[p];
}

// Log-probabilities from the sums over `parts` parts of the states.
__global__ __launch_bounds__(256) void k_predict_join(const float *__restrict__ sums, int32_t parts, int32_t n_cats, int32_t B, float *__restrict__ logp, int64_t ld)
{
    const int64_t i = blockIdx.x * 256ll + threadIdx.x, n = (int64_t)B * n_cats;
    if (i >= n) return;
    float p = 0.0f;
#pragma unroll 4
    for (int s = 0; s < parts; ++s) p += sums[s * n + i];
    logp[i / n_cats * ld + i % n_cats] = log_p(p);
}

// One sample: bound by reading the tables once.  The lanes of a wave cover whole table rows (K / 4 lanes each with four states) of the
// same block, so that loads are contiguous, kOneRows of two blocks in flight; a lane keeps its states' weights of the block in registers
// and a sum per row, and only at the end of all blocks the lanes of a row add theirs.  Products in fp32.  STREAM: tables of 256 MB and more,
// which no cache holds until the next call, are read past the caches (4096 states x 50257 149 us against 162; 512 states, held, 23 against 22).
constexpr int kOneFloats = 4096, kOneRows = 8;         // weights in LDS at a time; loads of a lane in flight, of two blocks each
template <bool STREAM>
__global__ __launch_bounds__(256) void k_predict_one(const pc_mixture m, const float *__restrict__ tables, float *__restrict__ logp)
{
    __shared__ float4 w[kOneFloats / 4];              // [block of the window][piece]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int P = group_states(m.K) / 4, R = 64 / P, piece = lane % P, r = lane / P;      // pieces of a row, rows of an instruction
    const bool idle = r >= R;
    const int per_window = min(m.n_blocks, kOneFloats / (4 * P));
    const int64_t c0 = ((int64_t)blockIdx.x * 4 + wave) * R * kOneRows + (idle ? 0 : r);
    float acc[kOneRows] = {};
    bool on[2];
    int64_t row[kOneRows];                                 // a category behind the last reads that one's row again
#pragma unroll
    for (int u = 0; u < kOneRows; ++u) row[u] = min(c0 + u * R, (int64_t)m.n_cats - 1) * m.K + group_start(m.K, 4 * piece);
    for (int j0 = 0; j0 < m.n_blocks; j0 += per_window) {
        const int here = min(per_window, m.n_blocks - j0);
        __syncthreads();
        for (int i = threadIdx.x; i < here * P; i += 256) {
            const int q = i % P;
            const MixBlock blk = mix_block(m, j0 + i / P);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (blk.row >= 0) {
                const int k = group_start(m.K, 4 * q), skip = 4 * q - k;
                const float *src = m.weights + (blk.row + k) * m.stride;
                v = make_float4(skip > 0 ? 0.f : src[0], skip > 1 ? 0.f : src[m.stride], skip > 2 ? 0.f : src[2 * m.stride], src[3 * m.stride]);
            }
            w[i] = v;
        }
        __syncthreads();
        Pack<float> t[2][kOneRows];                             // a block's rows, while those of the one before are added up
        auto fetch = [&](int j, int set) {             // a block left out reads the first table's rows and is not added
            const MixBlock blk = mix_block(m, j0 + j);
            on[set] = blk.row >= 0;
            const float *src = tables + (int64_t)max(blk.table, 0) * m.n_cats * m.K;
#pragma unroll
            for (int u = 0; u < kOneRows; ++u) t[set][u] = STREAM ? stream_pack(src + row[u]) : load_pack(src + row[u]);
        };
        auto add = [&](int j, int set) {
            if (!on[set]) return;
            const float4 v = w[j * P + piece];
#pragma unroll
            for (int u = 0; u < kOneRows; ++u) acc[u] += t[set][u].v[0] * v.x + t[set][u].v[1] * v.y + t[set][u].v[2] * v.z + t[set][u].v[3] * v.w;
        };
        fetch(0, 0);
        for (int j = 0; j < here; j += 2) {
            fetch(min(j + 1, here - 1), 1);
            add(j, 0);
            if (j + 1 < here) {
                fetch(min(j + 2, here - 1), 0);
                add(j + 1, 1);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kOneRows; ++u) {
        const int64_t c = c0 + u * R;
        float v = acc[u];
        for (int d = 1; d < P; d <<= 1) {              // lane `piece` adds d lanes more each time, none of another row
            const float o = __shfl_down(v, d);
            if (piece + d < P && piece % (2 * d) == 0) v += o;
        }
        if (piece == 0 && !idle && c < m.n_cats) logp[c] = log_p(v);
    }
}

// 2^-24 g / p of one sample and category (the weights are scaled by 2^24: a weight times g / p, which may be as large as g over the smallest
// table entry, stays what it is); p = 0 adds nothing.  exp(-logp) as 2^t times what t = -logp log2(e), rounded, leaves out: good to 2^-23 over the
// whole range, for half the instructions of expf.
__device__ inline float flow_ratio(float logp, float g)
{
    constexpr float kLog2e = 1.44269504f, kRest = 1.92596299e-8f, kLn2 = 0.693147181f;    // log2(e) = kLog2e + kRest
    const float t = -logp * kLog2e, rest = fmaf(-logp, kRest, fmaf(-logp, kLog2e, -t));
    const float e = __builtin_amdgcn_exp2f(t);
    return logp < kLogFltMin - 1e-3f ? 0.0f : g * (fmaf(e, rest * kLn2, e) * kDown);
}

// Column n of the flows: its first weight (-1: none, or another block's column does its table's work), its place in the flows for category 0,
// and whether its table has further blocks.
__device__ inline void flow_column(const pc_mixture &m, int n, int64_t &w_at, int64_t &o_at, int32_t &more)
{
    const int j = n / m.K;
    const MixBlock blk = j < m.n_blocks ? mix_block(m, j) : MixBlock{-1, -1};
    bool mine = blk.row >= 0, again = false;
    if (m.table && mine)
        for (int o = 0; o < m.n_blocks; ++o)
            if (o != j && m.table[o] == blk.table && mix_block(m, o).row >= 0) {
                if (o < j) mine = false;
                else again = true;
            }
    w_at = mine ? (blk.row + n % m.K) * m.stride : -1;
    o_at = blk.row >= 0 ? (int64_t)blk.table * m.n_cats * m.K + n % m.K : 0;      // a place that exists
    more = again;
}

// What k_predict_flow<MARKED> reads, in its workspace.  Samples are dealt out in parts of `part` (several where tiles are few), looked at kSegment at a time.
constexpr int kSegment = 512;
struct FlowPrep {
    float *wt;                                         // weights by sample, [B][H], a table's further blocks added to its first one's column
    uint32_t *marks;                                   // bit b % 32 of [c / 64][b / 32]: sample b has a gradient that is not zero among 64 categories
    pc_u32x4 *wp, *rp;                                 // planes of the weights [8 samples][plane][H] and of g / p [8 samples][plane][n_cats]; zeros behind B
    float *sums;                                       // [part][n_cats][H], or NULL: one part
    int32_t part;
};
__device__ inline bool mostly(int count, int of) { return count * 4 > of * 3; }
// The first `turns` workgroups: weights, 64 columns x 64 samples each.  The others: a segment of 64 I categories each, its marks, and g / p where
// most of its samples count.
constexpr int kPrepareWaves = 8;
template <int I>
__global__ __launch_bounds__(64 * kPrepareWaves) void k_flow_prepare(const pc_mixture m, int32_t B, const float *__restrict__ logp, int64_t lp_ld, const float *__restrict__ dlogp,
                                                      int64_t ld, int32_t turns, const FlowPrep f)
{
    __shared__ float x[64][65];
    __shared__ int64_t w_at[64], o_at[64];
    __shared__ int32_t more[64];
    __shared__ uint32_t bits[I][kSegment / 32];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), H = m.n_blocks * m.K;
    if ((int)blockIdx.x < turns) {
        const int n0 = blockIdx.x % ((H + 63) / 64) * 64, b0 = blockIdx.x / ((H + 63) / 64) * 64, b = min(b0 + lane, B - 1);
        if (wave == 0) flow_column(m, n0 + lane, w_at[lane], o_at[lane], more[lane]);
        __syncthreads();
#pragma unroll
        for (int c = wave; c < 64; c += kPrepareWaves) x[c][lane] = m.weights[max(w_at[c], (int64_t)0) + b];
        for (int c = wave; c < 64; c += kPrepareWaves) {
            if (m.table && w_at[c] >= 0 && more[c])
                for (int o = (n0 + c) / m.K + 1, t = m.table[o - 1]; o < m.n_blocks; ++o) {
                    const MixBlock blk = mix_block(m, o);
                    if (blk.row >= 0 && blk.table == t) x[c][lane] += m.weights[(blk.row + (n0 + c) % m.K) * m.stride + b];
                }
        }
        __syncthreads();
        if (n0 + lane >= H) return;
        for (int s = wave; s < 64; s += kPrepareWaves) {
            if (b0 + s < B) f.wt[(int64_t)(b0 + s) * H + n0 + lane] = x[lane][s];
        }
        for (int g = wave; g < 8 && b0 + 8 * g < (B + 15) / 16 * 16; g += kPrepareWaves) {
            float v[8];
            uint4 pl[3];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = b0 + 8 * g + e < B ? x[lane][8 * g + e] * kUp : 0.0f;
            split8(v, pl);
#pragma unroll
            for (int p = 0; p < 3; ++p) f.wp[((int64_t)(b0 / 8 + g) * 3 + p) * H + n0 + lane] = __builtin_bit_cast(pc_u32x4, pl[p]);
        }
        return;
    }
    const int64_t rows = (m.n_cats + 63ll) / 64, words = (B + 31ll) / 32, tiles = (rows + I - 1) / I, job = blockIdx.x - turns, row0 = job % tiles * I;
    const int64_t segments = (f.part + kSegment - 1) / kSegment, at = job / tiles, s0 = at / segments * f.part + at % segments * kSegment;
    const int here = (int)min(min((int64_t)B, (at / segments + 1) * f.part) - s0, (int64_t)kSegment);
    if (here <= 0) return;
    for (int j = wave; j < (here + 31) / 32 * I; j += kPrepareWaves) {
        const int64_t row = row0 + j % I, b0 = s0 + j / I * 32, c = min(row * 64 + lane, (int64_t)m.n_cats - 1);
        uint32_t w = 0;
        if (row < rows) {
            float g[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) g[e] = dlogp[min(b0 + e, (int64_t)B - 1) * ld + c];
#pragma unroll
            for (int e = 0; e < 32; ++e) w |= (__ballot(g[e] != 0.0f) != 0 && b0 + e < B ? 1u : 0u) << e;
            if (lane == 0) f.marks[row * words + b0 / 32] = w;
        }
        if (lane == 0) bits[j % I][j / I] = w;
    }
    __syncthreads();
    int count = 0;
    for (int j = 0; j < (here + 31) / 32; ++j) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < I; ++i) w |= bits[i][j];
        count += __popc(w);
    }
    if (!mostly(count, here)) return;
    for (int j = wave; j < (here + 15) / 16 * 2 * I; j += kPrepareWaves) {
        const int64_t c = (row0 + j % I) * 64 + lane, b0 = s0 + j / I * 8;
        if (c >= m.n_cats) continue;
        float l[8], d[8], v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t b = min(b0 + e, (int64_t)B - 1);
            l[e] = logp[b * lp_ld + c];
            d[e] = dlogp[b * ld + c];
        }
        uint4 pl[3];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = b0 + e < B ? flow_ratio(l[e], d[e]) : 0.0f;
        split8(v, pl);
#pragma unroll
        for (int p = 0; p < 3; ++p) f.rp[((b0 / 8) * 3 + p) * m.n_cats + c] = __builtin_bit_cast(pc_u32x4, pl[p]);
    }
}

// Table flows.  A workgroup of 2 x 2 waves owns a tile of 64 I categories x 64 I columns, a column being a node of a block.  The samples are
// added up 16 at a time from planes in LDS: g / p of the tile's categories and the weights of its columns, three planes each, six
// products (the terms of a flow have either sign and are few, so that nothing averages out; the fp32 matrix instructions took longer:
// 4096 states x 50257, B = 256, gradients without zeros 1372 us against 795).  While a step is multiplied the next one's operands are staged and the one
// after is on its way.  Bound by the matrix cores' sustained rate from some 100 samples on (B = 256: 742 us in a long row of calls, six products at
// the rate of a large one 436; making the planes in every tile took a quarter more), before by reading the tables and writing their flows (B = 32: 346 us, 4.9 TB/s), which the products of a
// CU's other workgroups cover.
// MARKED: operands as k_flow_prepare has left them.  Of a segment whose samples mostly have no gradient among the tile's categories (targets of
// a few categories a sample: an EM step) only those that do are added up, their g / p made here and their weights taken by sample,
// so that the columns of any sample are neighbours (64 categories a sample, B = 256: 420 us; gathered from the rows of m.weights 737,
// all samples 967).
// LISTS: a table named by several blocks is the first one's: its column adds up all their weights, the others' columns do nothing, so every entry has
// one writer.  The workgroups of a category tile follow one another on one XCD, whose cache keeps its g / p.
template <int I, bool MARKED, bool LISTS>
__global__ __launch_bounds__(256, I == 2 ? 3 : 4) void k_predict_flow(const pc_mixture m, const float *__restrict__ tables, int32_t B, const float *__restrict__ logp,
                                                         int64_t lp_ld, const float *__restrict__ dlogp, int64_t dl_ld, float scale, int32_t accumulate,
                                                         float *__restrict__ flow, const FlowPrep f)
{
    constexpr int TH = 256, TC = 64 * I, TN = 64 * I, NP = TN + 4;   // four more: the two groups of a column lie in other banks
    __shared__ uint4 rs[2][3][2][TC], ws[2][3][2][NP];                            // [buffer][plane][8 samples][category or column]
    __shared__ int64_t w_at[TN], o_at[TN];            // first weight of a column, -1: none; its place in the flows for category 0
    __shared__ int32_t more[TN];                      // the column's table has further blocks
    __shared__ uint16_t list[MARKED ? kSegment : 1];    // samples of the segment that count
    const int H = m.n_blocks * m.K, n_tiles = (H + TN - 1) / TN, q = blockIdx.x / 8;
    const int64_t c0 = ((int64_t)(q / n_tiles) * 8 + blockIdx.x % 8) * TC;
    const int n0 = q % n_tiles * TN;
    if (c0 >= m.n_cats) return;
    const int64_t mark_rows = (m.n_cats + 63ll) / 64, mark_ld = (B + 31ll) / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int cw = wave / 2 * 32 * I, nw = wave % 2 * 32 * I;
    const int first = MARKED ? blockIdx.y * f.part : 0, last = MARKED ? min(B, first + f.part) : B;
    auto marks_of = [&](int s0, int here) {
        uint32_t w = 0;
        if (32 * lane < here)
#pragma unroll
            for (int i = 0; i < I; ++i)
                if (c0 / 64 + i < mark_rows) w |= f.marks[(c0 / 64 + i) * mark_ld + s0 / 32 + lane];
        return w;
    };
    const uint32_t first_word = MARKED ? marks_of(first, min(kSegment, last - first)) : 0;
    for (int i = threadIdx.x; i < TN; i += TH) flow_column(m, n0 + i, w_at[i], o_at[i], more[i]);
    __syncthreads();
    // What a thread stages a step: eight samples of a category (the group of samples is the wave's), and of a column (two lanes read 16 samples
    // of a row).  Categories behind the last and columns without weights repeat others: their sums are not stored.
    static_assert(I == 1 || I == 2, "the dealing below");
    const bool of_ratios = I == 2 || wave < 2, of_weights = I == 2 || wave >= 2;
    const int r_group = I == 2 ? wave / 2 : wave % 2, r_cat = I == 2 ? threadIdx.x % TC : lane;
    const int w_col = MARKED ? (I == 2 ? threadIdx.x % TN : lane) : threadIdx.x % (I == 2 ? TH : TH / 2) / 2;
    const int w_group = MARKED ? r_group : lane % 2;
    const float *w_row = MARKED ? f.wt : m.weights + max(w_at[w_col], (int64_t)0);
    const bool w_more = LISTS && w_at[w_col] >= 0 && more[w_col];
    floatx16 acc[I][I];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int k = 0; k < I; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][k][e] = 0.0f;
    bool none = true;                                  // no sample counts for this tile
    // READY: the segments whose operands are as k_flow_prepare has left them; else the others.  Each way has its own loop: its registers are its own.
    auto pass = [&](auto as_ready) {
        constexpr bool READY = decltype(as_ready)::value;
        for (int s0 = first; s0 < last; s0 += MARKED ? kSegment : B) {
            const int here = MARKED ? min(kSegment, last - s0) : B;
            int n_samples = here;
            if (MARKED) {
                // lane i has the marks of samples 32 i to 32 i + 31; the list is made of them in order
                const uint32_t word = s0 == first ? first_word : marks_of(s0, here);
                int n = 0;
#pragma unroll
                for (int j = 0; j < kSegment / 32; ++j) n += __popc(__builtin_amdgcn_readlane(word, j));
                if (mostly(n, here) != READY || n == 0) continue;
                if (!READY) {
                    n_samples = n;
                    __syncthreads();                       // the list before is read
                    if (wave == 0)
                        for (int j = 0, at = 0; j < (here + 31) / 32; ++j) {
                            const uint32_t those = __builtin_amdgcn_readlane(word, j);
                            if (lane < 32 && those >> lane & 1) list[at + __popc(those & ((1u << lane) - 1))] = (uint16_t)(32 * j + lane);
                            at += __popc(those);
                        }
                    __syncthreads();
                }
            }
            none = false;
            int cat = (int)min(c0 + r_cat, (int64_t)m.n_cats - 1), w_n = min(n0 + w_col, H - 1);
            if (MARKED) asm volatile("" : "+v"(cat), "+v"(w_n));     // addresses are made here, not kept for both ways
            auto sample = [&](int i) { return s0 + (!MARKED ? i : list[i]); };
            float l[READY ? 1 : 8], d[READY ? 1 : 8], w[READY ? 1 : 8];
            pc_u32x4 r_ready[3], w_ready[3];
            auto group = [&](int i, int which) { return (int64_t)min((s0 + i) / 8 + which, (B + 15) / 16 * 2 - 1) * 3; };
            auto fetch_ratios = [&](int i0) {
                if constexpr (READY) {
#pragma unroll
                    for (int p = 0; p < 3; ++p) r_ready[p] = f.rp[(group(i0, r_group) + p) * m.n_cats + cat];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int64_t at = __builtin_amdgcn_readfirstlane(sample(min(i0 + 8 * r_group + e, n_samples - 1)));
                        l[e] = (logp + at * lp_ld)[cat];
                        d[e] = (dlogp + at * dl_ld)[cat];
                    }
                }
            };
            auto stage_ratios = [&](int i0, int buf) {
                if constexpr (READY) {
#pragma unroll
                    for (int p = 0; p < 3; ++p) rs[buf][p][r_group][r_cat] = __builtin_bit_cast(uint4, r_ready[p]);
                } else {
                    float x[8];
                    uint4 pl[3];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = flow_ratio(l[e], d[e]);
                    if (i0 + 16 > n_samples)
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = i0 + 8 * r_group + e < n_samples ? x[e] : 0.0f;
                    split8(x, pl);
#pragma unroll
                    for (int p = 0; p < 3; ++p) rs[buf][p][r_group][r_cat] = pl[p];
                }
            };
            auto eight = [&](const float *row, int i, float (&x)[8]) {
                if (i + 8 <= n_samples) {
                    const Pack<float> u = load_pack(row + i), v = load_pack(row + i + 4);      // a row may begin at any float
#pragma unroll
                    for (int e = 0; e < 4; ++e) { x[e] = u.v[e]; x[4 + e] = v.v[e]; }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = row[min(i + e, n_samples - 1)];
                }
            };
            auto fetch_weights = [&](int i0) {
                if constexpr (READY) {
#pragma unroll
                    for (int p = 0; p < 3; ++p) w_ready[p] = f.wp[(group(i0, w_group) + p) * H + w_n];
                } else if constexpr (MARKED) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        w[e] = (w_row + (int64_t)__builtin_amdgcn_readfirstlane(sample(min(i0 + 8 * w_group + e, n_samples - 1))) * H)[w_n];
                } else {
                    eight(w_row, i0 + 8 * w_group, w);
                    if (w_more)
                        for (int o = (n0 + w_col) / m.K + 1, t = m.table[o - 1]; o < m.n_blocks; ++o) {
                            const MixBlock blk = mix_block(m, o);
                            if (blk.row < 0 || blk.table != t) continue;
                            float y[8];
                            eight(m.weights + (blk.row + (n0 + w_col) % m.K) * m.stride, i0 + 8 * w_group, y);
#pragma unroll
                            for (int e = 0; e < 8; ++e) w[e] += y[e];
                        }
                }
            };
            auto stage_weights = [&](int i0, int buf) {
                if constexpr (READY) {
#pragma unroll
                    for (int p = 0; p < 3; ++p) ws[buf][p][w_group][w_col] = __builtin_bit_cast(uint4, w_ready[p]);
                } else {
                    float x[8];
                    uint4 pl[3];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = w[e] * kUp;
                    if (i0 + 16 > n_samples)
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = i0 + 8 * w_group + e < n_samples ? x[e] : 0.0f;
                    split8(x, pl);
#pragma unroll
                    for (int p = 0; p < 3; ++p) ws[buf][p][w_group][w_col] = pl[p];
                }
            };
            __syncthreads();                               // the segment before is read
            if (of_ratios) fetch_ratios(0);
            if (of_weights) fetch_weights(0);
            if (of_ratios) { stage_ratios(0, 0); fetch_ratios(16); }
            if (of_weights) { stage_weights(0, 0); fetch_weights(16); }
            __syncthreads();
            for (int i0 = 0, buf = 0; i0 < n_samples; i0 += 16, buf ^= 1) {
                const bool next = i0 + 16 < n_samples;
                uint4 rp[I][3];
#pragma unroll
                for (int i = 0; i < I; ++i)
#pragma unroll
                    for (int p = 0; p < 3; ++p) rp[i][p] = rs[buf][p][half][cw + 32 * i + col];
#pragma unroll
                for (int k = 0; k < I; ++k) {
                    uint4 wp[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) wp[p] = ws[buf][p][half][nw + 32 * k + col];
#pragma unroll
                    for (int sum = 2; sum >= 0; --sum)     // the small products first
#pragma unroll
                        for (int p = sum; p >= 0; --p)
#pragma unroll
                            for (int i = 0; i < I; ++i) acc[i][k] = mfma(rp[i][p], wp[sum - p], acc[i][k]);
                    if (next && k == 0 && of_weights) { stage_weights(i0 + 16, buf ^ 1); fetch_weights(i0 + 32); }
                    if (next && k == I - 1 && of_ratios) { stage_ratios(i0 + 16, buf ^ 1); fetch_ratios(i0 + 32); }
                    __builtin_amdgcn_sched_barrier(0);
                }
                __syncthreads();
            }
        }
    };
    if constexpr (MARKED) pass(std::true_type{});
    pass(std::false_type{});
    if (MARKED && I == 1 && f.sums) {                    // a part of the samples
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int64_t c = c0 + cw + 4 * half + 8 * (e / 4) + e % 4;
            if (c < m.n_cats && n0 + nw + col < H) f.sums[(blockIdx.y * (int64_t)m.n_cats + c) * H + n0 + nw + col] = acc[0][0][e];
        }
        return;
    }
    if (MARKED && none && accumulate) return;
    // A whole tile of tables below 4 GiB: 32-bit offsets from addresses that all lanes share, a square's entries on their way while the one
    // before is stored.  Else entry by entry.
    auto finish = [&](auto add) {
        constexpr bool ADD = decltype(add)::value;
        // (tables and flows past the caches, which keep the operands: B = 32 358 us against 383, 64 categories a sample, B = 256 420 against 446)
        float t[2][16];
        auto offset = [&](int sq) { return (uint32_t)((o_at[nw + 32 * (sq / I) + col] + (c0 + cw + 32 * (sq % I) + 4 * half) * m.K) * 4); };
        auto entry = [&](int e) { return (int64_t)(8 * (e / 4) + e % 4) * m.K * 4; };
        auto fetch = [&](int sq) {
            const uint32_t at = offset(sq);
            if (MARKED && none) return;                  // the sums are zero
#pragma unroll
            for (int e = 0; e < 16; ++e) t[sq & 1][e] = __builtin_nontemporal_load(reinterpret_cast<const float *>(reinterpret_cast<const char *>(tables) + entry(e) + at));
        };
        fetch(0);
#pragma unroll
        for (int sq = 0; sq < I * I; ++sq) {
            if (sq + 1 < I * I) fetch(sq + 1);
            const uint32_t at = offset(sq);
            if (w_at[nw + 32 * (sq / I) + col] >= 0) {
                float old[16];
                if (ADD)
#pragma unroll
                    for (int e = 0; e < 16; ++e) old[e] = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(flow) + entry(e) + at);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float v = MARKED && none ? 0.0f : scale * (t[sq & 1][e] * acc[sq % I][sq / I][e]);
                    __builtin_nontemporal_store(ADD ? old[e] + v : v, reinterpret_cast<float *>(reinterpret_cast<char *>(flow) + entry(e) + at));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (c0 + TC <= m.n_cats && (int64_t)m.n_tables * m.n_cats * m.K < 1ll << 30) {
        if (accumulate) finish(std::true_type{});
        else finish(std::false_type{});
        return;
    }
#pragma unroll
    for (int sq = 0; sq < I * I; ++sq) {
        const int n = nw + 32 * (sq / I) + col;
        if (w_at[n] < 0) continue;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int64_t c = c0 + cw + 32 * (sq % I) + 4 * half + 8 * (e / 4) + e % 4, at = o_at[n] + c * m.K;
            if (c < m.n_cats) {
                const float v = scale * (tables[at] * acc[sq % I][sq / I][e]);
                flow[at] = accumulate ? flow[at] + v : v;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// The flows from the sums of `parts` parts of the samples: 64 columns x 16 categories a workgroup.
__global__ __launch_bounds__(256) void k_flow_join(const pc_mixture m, const float *__restrict__ tables, const float *__restrict__ sums, int32_t parts, float scale,
                                                   int32_t accumulate, float *__restrict__ flow)
{
    __shared__ int64_t w_at[64], o_at[64];
    __shared__ int32_t more[64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, H = m.n_blocks * m.K, n = blockIdx.x * 64 + lane;
    if (wave == 0) flow_column(m, n, w_at[lane], o_at[lane], more[lane]);
    __syncthreads();
    if (w_at[lane] < 0) return;
    for (int i = 0; i < 4; ++i) {
        const int64_t c = blockIdx.y * 16ll + wave + 4 * i, at = o_at[lane] + c * m.K;
        if (c >= m.n_cats) return;
        float sum = 0.0f;
#pragma unroll 8
        for (int p = 0; p < parts; ++p) sum += sums[(p * (int64_t)m.n_cats + c) * H + n];
        const float v = scale * (tables[at] * sum);
        flow[at] = accumulate ? flow[at] + v : v;
    }
}

static int64_t one_rows(const pc_mixture &m) { return 64 / ((m.K + 3) / 4) * kOneRows; }      // categories of a wave of k_predict_one

// How a prediction is launched.
// One sample of many categories: no matrix cores (100 states x 20 blocks x 50257 72 us against 116, 32 states x 8 12 against 25; 4096 states 139 and
// 229, 8192 states x 20000 120 and 220), where that makes waves enough for two to a CU.
// Samples a wave: as many of 256 as there are, so that the tables are read once; 128 below 4096 categories (256 and 128: 4096 states x 4000, B = 256
// 68 us and 64, x 9000 116 and 127, x 50257 545 and 645); 64 from 17 samples on (64 and 32: 4096 states x 50257, B = 24 229 us and 268, B = 16 231 and
// 215); fewer where that leaves a SIMD without a wave (the tables of few categories stay in the caches).
// Where there is less than a workgroup to a CU and the states are many (1024: an exchange and a second launch take some 4 us) they are dealt out
// in parts of at least 256, as many as fill the GPU once, whose sums k_predict_join adds up (4096 states x 256, B = 256 17 us against 57;
// x 5000 80 against 470; x 16000, 2048 states, B = 500 181 against 251; with more workgroups, 1024 states x 50257, B = 64 74 against 58).
struct PredictPlan { bool one; int32_t nt, len, parts, columns; size_t sums, bytes; };
static PredictPlan predict_plan(const pc_mixture &m, int32_t B)
{
    PredictPlan p{};
    if (m.K < 4) return p;
    p.one = B == 1 && m.n_cats >= 512 * one_rows(m);
    if (p.one) return p;
    const int64_t rows = (m.n_cats + 31ll) / 32, H = (int64_t)m.n_blocks * ((m.K + 3) / 4 * 4), most = H < 1024 ? 1 : H / 256;
    p.nt = B > 128 && m.n_cats >= 4096 ? 8 : B > 64 ? 4 : B > 16 ? 2 : 1;
    const auto columns = [&] { return (B + 32ll * p.nt - 1) / (32 * p.nt); };
    while (p.nt > 1 && rows * columns() * most < 1024) p.nt /= 2;
    const int64_t groups = (p.nt == 8 ? (rows + 7) / 8 : p.nt > 1 ? (rows + 3) / 4 : rows) * columns();
    const int64_t slots = 256 * (p.nt == 8 ? 1 : p.nt == 2 ? 3 : 2);
    const int64_t want = groups < 256 ? std::min(slots / groups, most) : 1;
    p.len = (int32_t)((H + want * 128 - 1) / (want * 128) * 128);
    p.parts = (int32_t)((H + p.len - 1) / p.len);
    p.columns = (int32_t)(columns() * 32 * p.nt);
    p.sums = p.nt >= 4 ? (size_t)kPlanes * ((H + 7) / 8) * p.columns * 16 : 0;
    p.bytes = p.sums + (p.parts > 1 ? (size_t)p.parts * B * m.n_cats * 4 : 0);
    return p;
}

// Samples of a first launch with the widest waves, the others in a second one: where half of such a wave would do for those (4096 states
// x 50257, B = 257 665 us against 1004, B = 384 876 against 1042).
static int32_t predict_first(const pc_mixture &m, int32_t B)
{
    if (B <= 256 || B % 256 == 0 || B % 256 > 128) return B;
    const PredictPlan p = predict_plan(m, B);
    return p.nt == 8 && p.parts == 1 ? B / 256 * 256 : B;
}

static void launch_predict(const pc_mixture &m, const PredictPlan &p, const float *tables, int32_t B, float *logp, int64_t ld, void *workspace, hipStream_t s)
{
    if (p.one) {
        const dim3 grid((unsigned)((m.n_cats + 4 * one_rows(m) - 1) / (4 * one_rows(m))));
        if ((int64_t)m.n_blocks * m.n_cats * m.K >= 64 << 20) hipLaunchKernelGGL(k_predict_one<true>, grid, dim3(256), 0, s, m, tables, logp);
        else hipLaunchKernelGGL(k_predict_one<false>, grid, dim3(256), 0, s, m, tables, logp);
        return;
    }
    const int64_t rows = (m.n_cats + 31ll) / 32;
    uint4 *ready = (uint4 *)workspace;
    float *sums = p.parts > 1 ? (float *)((char *)workspace + p.sums) : nullptr;
    if (p.nt >= 4) {
        const int64_t groups = ((int64_t)m.n_blocks * ((m.K + 3) / 4 * 4) + 7) / 8;
        const dim3 grid((unsigned)((groups + 3) / 4), (unsigned)((p.columns + 63) / 64));
        hipLaunchKernelGGL(k_predict_ready, grid, dim3(256), 0, s, m, B, p.columns, ready);
    }
#define PC_PREDICT(NT, WAVES, SPLIT, KC)                                                                                       \
    if (p.nt == NT) {                                                                                                          \
        const dim3 grid((unsigned)((rows + WAVES / SPLIT - 1) / (WAVES / SPLIT)), (unsigned)((B + 32 * NT - 1) / (32 * NT)), p.parts);  \
        if (m.K % KC == 0) hipLaunchKernelGGL((k_predict<NT, WAVES, SPLIT, KC, true>), grid, dim3(64 * WAVES), 0, s, m, tables, B, logp, ld, p.len, sums, (const pc_u32x4 *)ready); \
        else hipLaunchKernelGGL((k_predict<NT, WAVES, SPLIT, KC, false>), grid, dim3(64 * WAVES), 0, s, m, tables, B, logp, ld, p.len, sums, (const pc_u32x4 *)ready); \
    }
    PC_PREDICT(8, 8, 1, 32)
    PC_PREDICT(4, 4, 1, 32)
    PC_PREDICT(2, 4, 1, 32)
    PC_PREDICT(1, 4, 4, 32)
#undef PC_PREDICT
    if (sums) {
        const int64_t n = (int64_t)B * m.n_cats;
        hipLaunchKernelGGL(k_predict_join, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, sums, p.parts, m.n_cats, B, logp, ld);
    }
}

// Tiles of 64 ic categories x 64 ic columns, over all of the tables; category tiles in eights, one to an XCD.
static int64_t flow_tiles(const pc_mixture &m, int64_t ic)
{
    return ((m.n_cats + 64 * ic - 1) / (64 * ic) + 7) / 8 * 8 * (((int64_t)m.n_blocks * m.K + 64 * ic - 1) / (64 * ic));
}
// Tiles of 128 x 128 where there are very many (128 and 64 wide, us: 3456 tiles, 3440 states x 15645, B = 94 180 and 210, B = 256 318 and 424,
// with 16 categories a sample 141 and 137); else, where they would cover the GPU in one to three rounds of workgroups, 64 x 64 (1600 tiles,
// 512 states x 50257: B = 16 87 and 59, B = 94 124 and 106, B = 256 198 and 206, with 16 categories a sample 106 and 77).
static bool flow_wide(const pc_mixture &m) { return flow_tiles(m, 2) >= 3000; }

// Scratch of the flows: what k_flow_prepare makes, where it begins, then the sums of parts.  Preparing pays from some 32 samples on (4096 states
// x 50257, B = 40: 64 categories a sample 372 us against 417, gradients without zeros 398 against 419; 512 states x 50257, B = 77: 72 against 96
// and 91 against 98), where there is little to do from 128 (128 states x 256, B = 100: 25 against 18).
// Where 64 x 64 tiles are few the samples are dealt out to several workgroups a tile, `part` each (a multiple of 64), whose sums k_flow_join
// adds up, always in the same order (128 states x 256, B = 512 28 us against 53; 512 states x 4000, B = 256 in 1000 workgroups 39 against 30).
constexpr int64_t kFlowGroups = 512, kFlowParts = 64;
struct FlowSpace { size_t marks, wp, rp, sums, bytes; int32_t part, parts; };
static FlowSpace flow_space(const pc_mixture &m, int32_t B)
{
    if (B < (flow_tiles(m, 1) >= 2048 ? 32 : 128)) return {0, 0, 0, 0, 0, B, 1};
    const int64_t H = (int64_t)m.n_blocks * m.K, tiles = (m.n_cats + 63ll) / 64 * ((H + 63) / 64);
    const int64_t want = std::max<int64_t>(1, std::min(kFlowGroups / tiles, kFlowParts));
    const int32_t part = (int32_t)(((B + want - 1) / want + 63) / 64 * 64), parts = (B + part - 1) / part;
    const size_t groups = (B + 15ull) / 16 * 2;
    FlowSpace f{0, 0, 0, 0, 0, part, parts};
    f.marks = ((size_t)B * H * 4 + 15) / 16 * 16;
    f.wp = f.marks + ((size_t)((m.n_cats + 63ll) / 64 * ((B + 31ll) / 32)) * 4 + 15) / 16 * 16;
    f.rp = f.wp + groups * 3 * H * 16;
    f.sums = f.rp + groups * 3 * m.n_cats * 16;
    f.bytes = f.sums + (parts > 1 ? (size_t)parts * m.n_cats * H * 4 : 0);
    return f;
}

static pc_status check_mixture(const pc_mixture *m, int32_t B)
{
    if (!m || !m->weights) return fail(PC_ERR_ARG, "NULL argument");
    if (m->K < 1 || m->K > 128) return fail(PC_ERR_ARG, "K must be in 1 .. 128");
    if (m->n_blocks < 1 || m->n_cats < 1 || m->n_tables < 1 || m->n_rows < 1)
        return fail(PC_ERR_ARG, "n_blocks, n_cats, n_tables and n_rows must be positive");
    if (B < 1) return fail(PC_ERR_ARG, "B must be positive");
    if (B > PC_MAX_BATCH) return fail(PC_ERR_TOO_LARGE, "more than PC_MAX_BATCH samples in one call");
    if (m->n_rows < m->K) return fail(PC_ERR_ARG, "weights have fewer rows than a block");
    if (m->stride < B) return fail(PC_ERR_ARG, "stride is smaller than B");
    if ((int64_t)m->n_blocks * m->K > 1 << 30) return fail(PC_ERR_TOO_LARGE, "more than 2^30 states");
    if (m->n_cats > (1 << 29) - 32) return fail(PC_ERR_TOO_LARGE, "more than 2^29 - 32 categories");   // a grid has fewer than 2^32 threads along x, 256 for 32 categories
    if (!m->rows && (int64_t)m->n_blocks * m->K > m->n_rows) return fail(PC_ERR_ARG, "weights have fewer than n_blocks * K rows");
    if (!m->table && m->n_blocks > m->n_tables) return fail(PC_ERR_ARG, "fewer tables than blocks");
    if (!aligned_to(m->weights, 4) || !aligned_to(m->rows, 4) || !aligned_to(m->table, 4))
        return fail(PC_ERR_ARG, "weights, rows and table must be 4-byte aligned");
    return PC_OK;
}
// What a call writes may not be what it reads: workgroups read the weights and tables as long as others write.
static bool over_operands(const pc_mixture &m, const float *tables, int32_t B, const float *out, int64_t bytes)
{
    return overlap(out, bytes, tables, (int64_t)m.n_tables * m.n_cats * m.K * 4) || overlap(out, bytes, m.weights, span_bytes(m.n_rows, m.stride, B, 4));
}

}  // namespace pc

using namespace pc;

extern "C" {

pc_status pc_predict_workspace_bytes(const pc_mixture *m, int32_t B, size_t *bytes)
{
    const pc_status st = check_mixture(m, B);
    if (st != PC_OK) return st;
    if (!bytes) return fail(PC_ERR_ARG, "NULL argument");
    const int32_t first = predict_first(*m, B);
    *bytes = std::max(predict_plan(*m, first).bytes, first < B ? predict_plan(*m, B - first).bytes : 0);
    return PC_OK;
}

pc_status pc_predict(const pc_mixture *m, const float *tables, int32_t B, float *logp, int64_t ld, void *workspace, size_t workspace_bytes, void *stream)
{
    const pc_status st = check_mixture(m, B);
    if (st != PC_OK) return st;
    if (!tables || !logp) return fail(PC_ERR_ARG, "NULL argument");
    if (!aligned_to(tables, 16)) return fail(PC_ERR_ARG, "tables must be 16-byte aligned");
    if (ld < m->n_cats) return fail(PC_ERR_ARG, "ld is smaller than n_cats");
    if (!aligned_to(logp, 4)) return fail(PC_ERR_ARG, "logp must be 4-byte aligned");
    size_t need = 0;
    pc_predict_workspace_bytes(m, B, &need);
    if (workspace_bytes < need) return fail(PC_ERR_WORKSPACE, "workspace smaller than pc_predict_workspace_bytes");
    if (need && (!workspace || !aligned_to(workspace, 16))) return fail(PC_ERR_ARG, "workspace must be 16-byte aligned");
    if (over_operands(*m, tables, B, logp, span_bytes(B, ld, m->n_cats, 4))) return fail(PC_ERR_ARG, "logp overlaps the tables or the weights");
    if (m->K < 4) {
        const dim3 grid((unsigned)((m->n_cats + 63ll) / 64), (unsigned)((B + 63) / 64));
        hipLaunchKernelGGL(k_predict_any, grid, dim3(256), 0, (hipStream_t)stream, *m, tables, B, logp, ld);
        return launched();
    }
    const int32_t first = predict_first(*m, B);
    launch_predict(*m, predict_plan(*m, first), tables, first, logp, ld, workspace, (hipStream_t)stream);
    if (first < B) {
        pc_mixture rest = *m;
        rest.weights += first;
        launch_predict(rest, predict_plan(rest, B - first), tables, B - first, logp + first * ld, ld, workspace, (hipStream_t)stream);
    }
    return launched();
}

pc_status pc_predict_backward_workspace_bytes(const pc_mixture *m, int32_t B, size_t *bytes)
{
    const pc_status st = check_mixture(m, B);
    if (st != PC_OK) return st;
    if (!bytes) return fail(PC_ERR_ARG, "NULL argument");
    *bytes = flow_space(*m, B).bytes;
    return PC_OK;
}

pc_status pc_predict_backward(const pc_mixture *m, const float *tables, int32_t B, const float *logp, int64_t logp_ld,
                              const float *dlogp, int64_t dlogp_ld, float scale, int32_t accumulate, float *table_flow, void *workspace,
                              size_t workspace_bytes, void *stream)
{
    const pc_status st = check_mixture(m, B);
    if (st != PC_OK) return st;
    if (!tables || !logp || !dlogp || !table_flow) return fail(PC_ERR_ARG, "NULL argument");
    if (!aligned_to(tables, 16)) return fail(PC_ERR_ARG, "tables must be 16-byte aligned");
    if (logp_ld < m->n_cats || dlogp_ld < m->n_cats) return fail(PC_ERR_ARG, "ld is smaller than n_cats");
    if (!aligned_to(logp, 4) || !aligned_to(dlogp, 4)) return fail(PC_ERR_ARG, "logp and dlogp must be 4-byte aligned");
    if (!aligned_to(table_flow, 16)) return fail(PC_ERR_ARG, "table_flow must be 16-byte aligned");
    const int64_t H = (int64_t)m->n_blocks * m->K;
    const hipStream_t s = (hipStream_t)stream;
    if (flow_tiles(*m, 1) > 1 << 23) return fail(PC_ERR_TOO_LARGE, "more than 2^23 tiles of flows");
    const FlowSpace f = flow_space(*m, B);
    if (workspace_bytes < f.bytes) return fail(PC_ERR_WORKSPACE, "workspace smaller than pc_predict_backward_workspace_bytes");
    if (f.bytes && (!workspace || !aligned_to(workspace, 16))) return fail(PC_ERR_ARG, "workspace must be 16-byte aligned");
    const int64_t flow_bytes = (int64_t)m->n_tables * m->n_cats * m->K * 4;
    if (over_operands(*m, tables, B, table_flow, flow_bytes) || overlap(table_flow, flow_bytes, logp, span_bytes(B, logp_ld, m->n_cats, 4)) ||
        overlap(table_flow, flow_bytes, dlogp, span_bytes(B, dlogp_ld, m->n_cats, 4)))
        return fail(PC_ERR_ARG, "table_flow overlaps the tables, the weights, logp or dlogp");
    char *base = (char *)workspace;
    const FlowPrep prep{(float *)base, (uint32_t *)(base + f.marks), (pc_u32x4 *)(base + f.wp), (pc_u32x4 *)(base + f.rp), f.parts > 1 ? (float *)(base + f.sums) : nullptr, f.part};
    const bool wide = flow_wide(*m);
    if (f.bytes) {
        const int64_t I = wide ? 2 : 1, turns = (H + 63) / 64 * ((B + 63ll) / 64), segments = (f.part + kSegment - 1) / kSegment;
        const int64_t jobs = (m->n_cats + 64 * I - 1) / (64 * I) * f.parts * segments;
        if (turns + jobs >= 1 << 23) return fail(PC_ERR_TOO_LARGE, "more than 2^23 tiles of weights and gradients");
        hipLaunchKernelGGL((wide ? k_flow_prepare<2> : k_flow_prepare<1>), dim3((unsigned)(turns + jobs)), dim3(64 * kPrepareWaves), 0, s, *m, B, logp, logp_ld, dlogp, dlogp_ld, (int32_t)turns, prep);
    }
#define PC_FLOW(I, MARKED, LISTS)                                                                                                       \
    hipLaunchKernelGGL((k_predict_flow<I, MARKED, LISTS>), dim3((unsigned)flow_tiles(*m, I), f.parts), dim3(256), 0, s, *m, tables, B, logp, logp_ld, \
                       dlogp, dlogp_ld, scale, accumulate, table_flow, prep)
    if (f.bytes && wide) PC_FLOW(2, true, false);
    else if (f.bytes) PC_FLOW(1, true, false);
    else if (m->table && wide) PC_FLOW(2, false, true);
    else if (m->table) PC_FLOW(1, false, true);
    else if (wide) PC_FLOW(2, false, false);
    else PC_FLOW(1, false, false);
#undef PC_FLOW
    if (prep.sums)
        hipLaunchKernelGGL(k_flow_join, dim3((unsigned)((H + 63) / 64), (unsigned)((m->n_cats + 15ll) / 16)), dim3(256), 0, s, *m, tables, prep.sums, f.parts, scale, accumulate, table_flow);
    return launched();
}

}  // extern "C"
