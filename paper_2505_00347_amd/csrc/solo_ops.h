// What the operators around the step have in common: loads and stores of eight consecutive elements, reductions over a
// wavefront and a workgroup, host-side checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/solo.h"

namespace solo {

constexpr int kLanes = 64;
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

// 16 bytes at any even address: gradients in a packed bucket and rows of odd length begin anywhere, and global memory is
// read there by the same instruction.  (An aligned access costs the same whether it is asked for this way or not.)
typedef uint32_t Quad __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 Pair __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two floats to bfloat16, nearest, ties to even.
__device__ __forceinline__ uint32_t to_bf16(float low, float high)
{
    Pair p;
    p[0] = (__bf16)low;
    p[1] = (__bf16)high;
    return __builtin_bit_cast(uint32_t, p);
}

template <bool BF16>
struct Elements {
    static constexpr int kBytes = BF16 ? 2 : 4;

    __device__ __forceinline__ static float load1(const void *base, uint64_t i)
    {
        if (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(base)[i] << 16);
        return static_cast<const float *>(base)[i];
    }
    __device__ __forceinline__ static void store1(void *base, uint64_t i, float x)
    {
        if (BF16) static_cast<uint16_t *>(base)[i] = (uint16_t)to_bf16(x, x);
        else static_cast<float *>(base)[i] = x;
    }
    // Elements i .. i + 7.
    struct Raw { Quad q[BF16 ? 1 : 2]; };
    __device__ __forceinline__ static Raw load8(const void *base, uint64_t i)
    {
        Raw r;
        const char *at = static_cast<const char *>(base) + i * kBytes;
#pragma unroll
        for (int k = 0; k < (BF16 ? 1 : 2); ++k) r.q[k] = *reinterpret_cast<const Quad *>(at + 16 * k);
        return r;
    }
    __device__ __forceinline__ static void unpack(const Raw &r, float x[8])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (BF16) {
                x[2 * k] = bf16_low(r.q[0][k]);
                x[2 * k + 1] = bf16_high(r.q[0][k]);
            } else {
                x[k] = __uint_as_float(r.q[0][k]);
                x[4 + k] = __uint_as_float(r.q[BF16 ? 0 : 1][k]);
            }
        }
    }
    __device__ __forceinline__ static void store8(void *base, uint64_t i, const float x[8])
    {
        char *at = static_cast<char *>(base) + i * kBytes;
        Quad a, b;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            a[k] = BF16 ? to_bf16(x[2 * k], x[2 * k + 1]) : __float_as_uint(x[k]);
            b[k] = __float_as_uint(x[4 + k]);
        }
        *reinterpret_cast<Quad *>(at) = a;
        if (!BF16) *reinterpret_cast<Quad *>(at + 16) = b;
    }
};

template <typename T>
__device__ __forceinline__ T wave_sum(T x)
{
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) x += __shfl_xor(x, d);
    return x;
}

// Sum over a workgroup of `waves` wavefronts, for every thread of it, in an order that is always the same.
template <typename T>
__device__ __forceinline__ T group_sum(T x, T *lds, int waves)
{
    x = wave_sum(x);
    __syncthreads();                                       // (lds may still be read from the sum before)
    if (threadIdx.x % kLanes == 0) lds[threadIdx.x / kLanes] = x;
    __syncthreads();
    T sum = lds[0];
    for (int w = 1; w < waves; ++w) sum += lds[w];
    return sum;
}

inline bool at_multiple(const void *p, uintptr_t a) { return p && reinterpret_cast<uintptr_t>(p) % a == 0; }
inline uintptr_t element_bytes(uint32_t dtype) { return dtype == SOLO_BF16 ? 2 : 4; }
inline bool dtype_ok(uint32_t dtype) { return dtype == SOLO_FP32 || dtype == SOLO_BF16; }
inline int launched() { return hipGetLastError() == hipSuccess ? SOLO_OK : SOLO_E_HIP; }

}  // namespace solo
