// Rows of logits in several element types, and the launch checks that the calls on them share (internal).
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>
#include <type_traits>

#include "pc_internal.h"

namespace pc {

#define PC_LOG2E_F 1.4426950408889634f
#define PC_NEG_INF_F (-__builtin_inff())

struct bf16_t { uint16_t bits; };                     // bfloat16 as it lies in memory
typedef __half f16_t;

__device__ inline float to_f32(float v) { return v; }
__device__ inline float to_f32(bf16_t v) { return __uint_as_float((uint32_t)v.bits << 16); }
__device__ inline float to_f32(f16_t v) { return __half2float(v); }
// to nearest, ties to even; a NaN stays one
template <typename T> __device__ T from_f32(float v);
template <> __device__ inline float from_f32<float>(float v) { return v; }
template <> __device__ inline f16_t from_f32<f16_t>(float v) { return __float2half_rn(v); }
template <> __device__ inline bf16_t from_f32<bf16_t>(float v)
{
    const uint32_t u = __float_as_uint(v);
    return bf16_t{(uint16_t)(v != v ? (u >> 16) | 0x40 : (u + 0x7fff + ((u >> 16) & 1)) >> 16)};
}

// Eight 16-bit or four 32-bit elements, 16 bytes, at any address that suits an element.
template <typename T> struct Pack { static constexpr int N = 16 / sizeof(T); T v[N]; };
typedef uint32_t pc_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t pc_u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t pc_u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
__device__ inline Pack<T> load_pack(const T *p)       // as one vector: element by element it would be as many loads
{
    typedef typename std::conditional<sizeof(T) == 2, pc_u32x4_at2, pc_u32x4_at4>::type loose;
    return __builtin_bit_cast(Pack<T>, (pc_u32x4)*reinterpret_cast<const loose *>(p));
}
template <typename T>
__device__ inline Pack<T> stream_pack(const T *p)     // what is not read again soon: the caches keep other things first
{
    typedef typename std::conditional<sizeof(T) == 2, pc_u32x4_at2, pc_u32x4_at4>::type loose;
    return __builtin_bit_cast(Pack<T>, (pc_u32x4)__builtin_nontemporal_load(reinterpret_cast<const loose *>(p)));
}
template <typename T>
__device__ inline void unpack_f32(const Pack<T> &r, float (&x)[Pack<T>::N])
{
    const pc_u32x4 w = __builtin_bit_cast(pc_u32x4, r);
#pragma unroll
    for (int i = 0; i < Pack<T>::N; ++i)
        if constexpr (std::is_same<T, float>::value) x[i] = __uint_as_float(w[i]);
        else if constexpr (std::is_same<T, f16_t>::value) x[i] = to_f32(r.v[i]);
        else x[i] = __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
}
typedef float pc_float2 __attribute__((ext_vector_type(2)));
typedef __bf16 pc_bf16x2 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ inline Pack<T> pack_f32(const float (&x)[Pack<T>::N])
{
    Pack<T> r;
    if constexpr (sizeof(T) == 2 && !std::is_same<T, f16_t>::value) {
#pragma unroll
        for (int i = 0; i < Pack<T>::N; i += 2) {
            const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector((pc_float2){x[i], x[i + 1]}, pc_bf16x2));
            r.v[i] = bf16_t{(uint16_t)w};
            r.v[i + 1] = bf16_t{(uint16_t)(w >> 16)};
        }
    } else {
#pragma unroll
        for (int i = 0; i < Pack<T>::N; ++i) r.v[i] = from_f32<T>(x[i]);
    }
    return r;
}
// elements before the first 16-byte boundary at or after p's own 16 bytes begin: p is element `off` of an aligned row
template <typename T>
__device__ inline int elements_off(const T *p) { return (int)(((uintptr_t)p & 15) / sizeof(T)); }

// the value of lane ^ J: within 16 lanes by data-parallel moves, across them by swaps of rows and halves
template <int J>
__device__ inline uint32_t lane_xor32(uint32_t v)
{
    const int x = (int)v;
    if constexpr (J == 1) return (uint32_t)__builtin_amdgcn_update_dpp(x, x, 0xb1, 0xf, 0xf, false);            // quad_perm 1 0 3 2
    else if constexpr (J == 2) return (uint32_t)__builtin_amdgcn_update_dpp(x, x, 0x4e, 0xf, 0xf, false);       // quad_perm 2 3 0 1
    else if constexpr (J == 4) {                       // four lanes up for the even fours of a row, four down for the odd ones
        const int up = __builtin_amdgcn_update_dpp(x, x, 0x104, 0xf, 0x5, false);
        return (uint32_t)__builtin_amdgcn_update_dpp(up, x, 0x114, 0xf, 0xa, false);
    } else if constexpr (J == 8) return (uint32_t)__builtin_amdgcn_update_dpp(x, x, 0x128, 0xf, 0xf, false);    // row_ror 8
    else if constexpr (J == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}
template <int J> __device__ inline float lane_xor(float v) { return __uint_as_float(lane_xor32<J>(__float_as_uint(v))); }
// op over all lanes of a wave, the same in all of them
template <int J = 32, typename F>
__device__ inline float wave_all(float v, F op)
{
    v = op(v, lane_xor<J>(v));
    if constexpr (J > 1) return wave_all<J / 2>(v, op);
    else return v;
}

inline int64_t type_bytes(int32_t type) { return type == PC_F32 ? 4 : 2; }
inline bool type_known(int32_t type) { return type == PC_F32 || type == PC_BF16 || type == PC_F16; }
inline bool aligned_to(const void *p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// from the first byte of `rows` rows of n elements, ld apart, to their last
inline int64_t span_bytes(int64_t rows, int64_t ld, int64_t n, int64_t element) { return ((rows - 1) * ld + n) * element; }
inline bool overlap(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes)
{
    return (uintptr_t)a < (uintptr_t)b + (uintptr_t)b_bytes && (uintptr_t)b < (uintptr_t)a + (uintptr_t)a_bytes;
}

// f(element) for the C++ type of `type`
template <typename F>
inline void with_type(int32_t type, F f)
{
    if (type == PC_F32) f(float{});
    else if (type == PC_BF16) f(bf16_t{});
    else f(f16_t{});
}

inline pc_status launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PC_OK : fail(PC_ERR_HIP, std::string("launch: ") + hipGetErrorString(e));
}

}  // namespace pc
