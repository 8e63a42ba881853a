// What the operators around a decode step and those that check drafted tokens share: element types, reductions over a few lanes, argument checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "addrms_internal.h"

namespace serving {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

enum : int { DT_BF16 = ADDRMS_BF16, DT_FP16 = ADDRMS_FP16, DT_FP32 = ADDRMS_FP32 };
template <int DT> struct elem;
template <> struct elem<DT_BF16> { typedef __bf16 type; };
template <> struct elem<DT_FP16> { typedef _Float16 type; };
template <> struct elem<DT_FP32> { typedef float type; };

// Tensors reach a kernel as the numbers of their addresses (a pointer argument is looked up at each launch).
typedef uint64_t addr_t;
template <typename T = void>
__device__ __forceinline__ T* at_global(addr_t a)
{
    return (T*)(__attribute__((address_space(1))) T*)a;
}
inline addr_t addr(const void* p) { return reinterpret_cast<addr_t>(p); }

// A lane's value and that of the lane 16, or 32, away, in an order that is the same for both lanes.
struct pair { float a, b; };
__device__ __forceinline__ pair with_row(float x)
{
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    const auto s = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    const uint32_t a = s[0], b = s[1];       // as values of their own: a bit cast of a vector's element takes the first
    return pair{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ pair with_half(float x)
{
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    const auto s = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const uint32_t a = s[0], b = s[1];
    return pair{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}

// Maximum over 2, 4, ... 32 neighbouring lanes, in all of them (NaN is passed over).
template <int CTRL>
__device__ __forceinline__ float dpp(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float max_of_lanes(float x, uint32_t lanes)
{
    if (lanes > 1) x = fmaxf(x, dpp<0xB1>(x));       // quad_perm 1,0,3,2
    if (lanes > 2) x = fmaxf(x, dpp<0x4E>(x));       // quad_perm 2,3,0,1
    if (lanes > 4) x = fmaxf(x, dpp<0x141>(x));      // row_half_mirror: both quads of eight lanes hold one value each by now
    if (lanes > 8) x = fmaxf(x, dpp<0x140>(x));      // row_mirror
    if (lanes > 16) {
        const pair p = with_row(x);
        x = fmaxf(p.a, p.b);
    }
    return x;
}

inline bool aligned_to(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline bool power_of_two(int64_t n) { return n > 0 && (n & (n - 1)) == 0; }
inline int log2_of(int64_t n)
{
    int s = 0;
    while ((1ll << s) < n) ++s;
    return s;
}

// A launch numbers its threads along an axis in 32 bits.
inline bool launchable(int64_t groups, int64_t threads) { return groups * threads < (1ll << 32); }

// A launch whose status is its own: an error that other code of the process left behind is not taken for it.
template <typename Args>
hipError_t launch_kernel(void (*kernel)(Args), dim3 grid, dim3 block, hipStream_t stream, const Args& args)
{
    void* p[] = {const_cast<Args*>(&args)};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, p, 0, stream);
}

#define SERVING_HIP_TRY(expr)                                                                                     \
    do {                                                                                                          \
        const hipError_t e_ = (expr);                                                                             \
        if (e_ != hipSuccess) return addrms_host::fail(ADDRMS_ERR_HIP, "%s failed: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

}  // namespace serving
