// What the operators around the step have in common: loads and stores of consecutive elements, reductions over a wavefront and a
// workgroup, host-side checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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
};

// N elements from element i on, 4 or 8 of them, to floats.
template <bool BF16, int N>
__device__ __forceinline__ void load_floats(const void *base, uint64_t i, float x[N])
{
    typedef uint32_t Half __attribute__((ext_vector_type(2), aligned(2)));
    const char *at = static_cast<const char *>(base) + i * (BF16 ? 2 : 4);
#pragma unroll
    for (int k = 0; k < N; k += 4) {
        if (BF16) {
            const Half h = *reinterpret_cast<const Half *>(at + 2 * k);        // (two halves of eight elements become one access)
            x[k] = bf16_low(h[0]); x[k + 1] = bf16_high(h[0]);
            x[k + 2] = bf16_low(h[1]); x[k + 3] = bf16_high(h[1]);
        } else {
            const Quad q = *reinterpret_cast<const Quad *>(at + 4 * k);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[k + e] = __uint_as_float(q[e]);
        }
    }
}

// The same to memory.
template <bool BF16, int N>
__device__ __forceinline__ void store_floats(void *base, uint64_t i, const float x[N])
{
    typedef uint32_t Half __attribute__((ext_vector_type(2), aligned(2)));
    char *at = static_cast<char *>(base) + i * (BF16 ? 2 : 4);
#pragma unroll
    for (int k = 0; k < N; k += 4) {
        if (BF16) {
            *reinterpret_cast<Half *>(at + 2 * k) = Half{to_bf16(x[k], x[k + 1]), to_bf16(x[k + 2], x[k + 3])};
        } else {
            *reinterpret_cast<Quad *>(at + 4 * k) =
                Quad{__float_as_uint(x[k]), __float_as_uint(x[k + 1]), __float_as_uint(x[k + 2]), __float_as_uint(x[k + 3])};
        }
    }
}

// 16 bytes a lane: eight bf16 or four fp32 elements, so that an instruction of a wavefront reads or writes 1 KB without gaps.
// (Eight fp32 elements a lane, as two halves, leave gaps of 16 bytes: a gradient of 201 MB, stored past the caches, then took 109 us instead of 91.)
// `i` is an element; `near`: less than 4 GiB behind a base that is the same for the wavefront, which saves registers of address.
template <bool BF16>
struct Lane16 {
    static constexpr int kBytes = BF16 ? 2 : 4, kPer = 16 / kBytes;

    template <bool PAST>
    __device__ __forceinline__ static Quad load(const void *base, uint64_t i)
    {
        const Quad *at = reinterpret_cast<const Quad *>(static_cast<const char *>(base) + i * kBytes);
        if (PAST) return __builtin_nontemporal_load(at);
        return *at;
    }
    template <bool PAST>
    __device__ __forceinline__ static Quad load_near(const void *base, uint32_t i) { return load<PAST>(static_cast<const char *>(base) + i * kBytes, 0); }
    __device__ __forceinline__ static void unpack(const Quad &q, float x[kPer])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (BF16) {
                x[2 * k] = bf16_low(q[k]);
                x[(2 * k + 1) % kPer] = bf16_high(q[k]);
            } else {
                x[k] = __uint_as_float(q[k]);
            }
        }
    }
    template <bool PAST>
    __device__ __forceinline__ static void store(void *base, uint64_t i, const float x[kPer])
    {
        Quad *at = reinterpret_cast<Quad *>(static_cast<char *>(base) + i * kBytes);
        Quad q;
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = BF16 ? to_bf16(x[2 * k % kPer], x[(2 * k + 1) % kPer]) : __float_as_uint(x[k]);
        if (PAST) __builtin_nontemporal_store(q, at);
        else *at = q;
    }
    template <bool PAST>
    __device__ __forceinline__ static void store_near(void *base, uint32_t i, const float x[kPer]) { store<PAST>(static_cast<char *>(base) + i * kBytes, 0, x); }
};

// From here on the compiler does not know what `q` holds.
__device__ __forceinline__ void forget(Quad &q) { asm volatile("" : "+v"(q)); }

// One step of a reduction: the values of the lanes of groups of D, which are all alike in a group, and of the neighbouring
// groups of D.  By the data paths of the vector unit: through LDS a step takes several times as long.
template <int D>
__device__ __forceinline__ void neighbours(uint32_t x, uint32_t &a, uint32_t &b)
{
    if constexpr (D >= 16) {
        const auto both = D == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false);
        a = both[0];
        b = both[1];
    } else {                                               // quad_perm 1,0,3,2; quad_perm 2,3,0,1; half of a row mirrored; row rotated by 8
        constexpr int kControl = D == 1 ? 0xB1 : D == 2 ? 0x4E : D == 4 ? 0x141 : 0x128;
        a = x;
        b = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kControl, 0xF, 0xF, true);
    }
}

template <int D, typename T>
__device__ __forceinline__ void neighbours(T x, T &a, T &b)
{
    if constexpr (sizeof(T) == 4) {
        uint32_t p, q;
        neighbours<D>(__builtin_bit_cast(uint32_t, x), p, q);
        a = __builtin_bit_cast(T, p);
        b = __builtin_bit_cast(T, q);
    } else {
        const uint64_t bits = __builtin_bit_cast(uint64_t, x);
        uint32_t p, q, r, s;
        neighbours<D>((uint32_t)bits, p, q);
        neighbours<D>((uint32_t)(bits >> 32), r, s);
        a = __builtin_bit_cast(T, (uint64_t)r << 32 | p);
        b = __builtin_bit_cast(T, (uint64_t)s << 32 | q);
    }
}

// op, which does not mind the order of its two, over the lanes of a wavefront, or of each group of LANES of them, for every lane.
template <int LANES = kLanes, int D = 1, typename T, typename Op>
__device__ __forceinline__ T wave_reduce(T x, Op op)
{
    if constexpr (D >= LANES) {
        return x;
    } else {
        T a, b;
        neighbours<D>(x, a, b);
        return wave_reduce<LANES, 2 * D>(op(a, b), op);
    }
}
template <int LANES = kLanes, typename T>
__device__ __forceinline__ T wave_sum(T x) { return wave_reduce<LANES>(x, [](T a, T b) { return a + b; }); }
template <int LANES = kLanes, typename T>
__device__ __forceinline__ T wave_max(T x) { return wave_reduce<LANES>(x, [](T a, T b) { return a > b ? a : b; }); }
template <int LANES = kLanes>
__device__ __forceinline__ float wave_max(float x) { return wave_reduce<LANES>(x, [](float a, float b) { return fmaxf(a, b); }); }

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

// A launch by its own result: the runtime's last error may be another call's.
template <typename Args>
inline int launch(void (*kernel)(Args), dim3 grid, uint32_t threads, hipStream_t stream, const Args &args, uint32_t lds = 0)
{
    void *at[] = {const_cast<Args *>(&args)};
    if (hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(threads), at, lds, stream) == hipSuccess) return SOLO_OK;
    (void)hipGetLastError();                               // (reported here, not by the caller's next call)
    return SOLO_E_HIP;
}

}  // namespace solo
