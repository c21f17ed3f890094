// Numbers of a training step: 32-bit, bfloat16 and half precision in memory, 32 bits in registers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "host_util.h"
#include "wave.h"

namespace stalloc {

using bf16 = __bf16;
using f16 = _Float16;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T> struct Vec;
template <> struct Vec<float> { typedef float x2 __attribute__((ext_vector_type(2))); typedef float x4 __attribute__((ext_vector_type(4))); typedef float x8 __attribute__((ext_vector_type(8))); };
template <> struct Vec<bf16> { typedef bf16 x2 __attribute__((ext_vector_type(2))); typedef bf16 x4 __attribute__((ext_vector_type(4))); typedef bf16 x8 __attribute__((ext_vector_type(8))); };
template <> struct Vec<f16> { typedef f16 x2 __attribute__((ext_vector_type(2))); typedef f16 x4 __attribute__((ext_vector_type(4))); typedef f16 x8 __attribute__((ext_vector_type(8))); };
typedef float f32x8 __attribute__((ext_vector_type(8)));

// Eight numbers from any address that suits one of them (gfx950 loads and stores 16 bytes from any).
template <typename T> __device__ __forceinline__ f32x8 load8(const T* p)
{
    typename Vec<T>::x8 v;
    __builtin_memcpy(&v, p, sizeof(v));
    return __builtin_convertvector(v, f32x8);
}
// (each number is rounded to the nearest one of the type, ties to even)
template <typename T> __device__ __forceinline__ void store8(T* p, f32x8 x)
{
    const typename Vec<T>::x8 v = __builtin_convertvector(x, typename Vec<T>::x8);
    __builtin_memcpy(p, &v, sizeof(v));
}
// The same past the caches: for numbers that nobody reads again before they would be gone from them.
template <typename T> using Loose = typename Vec<T>::x8 __attribute__((aligned(sizeof(T))));
template <typename T> __device__ __forceinline__ f32x8 load8_once(const T* p) { return __builtin_convertvector(__builtin_nontemporal_load((const Loose<T>*)p), f32x8); }
template <typename T> __device__ __forceinline__ void store8_once(T* p, f32x8 x)
{
    __builtin_nontemporal_store((Loose<T>)__builtin_convertvector(x, typename Vec<T>::x8), (Loose<T>*)p);
}
// The first `n` of eight numbers (n may be 0 or less); `fill` in place of the others.
template <typename T> __device__ __forceinline__ f32x8 load_some(const T* p, int n, float fill)
{
    if (n >= 8) return load8(p);
    f32x8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? (float)p[i] : fill;
    return x;
}
// The same, left in the type it has in memory; zeros in place of the others.
template <typename T> __device__ __forceinline__ typename Vec<T>::x8 packed_some(const T* p, int n)
{
    typename Vec<T>::x8 v = {};
    if (n >= 8) __builtin_memcpy(&v, p, sizeof(v));
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) v[i] = p[i];
    return v;
}
// Both for numbers that nobody reads again soon (kOnce: past the caches).
template <bool kOnce, typename T> __device__ __forceinline__ f32x8 load_some_once(const T* p, int n, float fill) { return kOnce && n >= 8 ? load8_once(p) : load_some(p, n, fill); }
template <bool kOnce, typename T> __device__ __forceinline__ typename Vec<T>::x8 packed_some_once(const T* p, int n)
{
    if (kOnce && n >= 8) return __builtin_nontemporal_load((const Loose<T>*)p);
    return packed_some(p, n);
}
template <typename T> __device__ __forceinline__ void store_some(T* p, int n, f32x8 x)
{
    if (n >= 8) { store8(p, x); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = (T)x[i];
}

__device__ __forceinline__ float as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ uint32_t as_bits(float v) { return __builtin_bit_cast(uint32_t, v); }

template <int kCtrl, int kRowMask = 0xf> __device__ __forceinline__ float dpp(float fill, float v)
{
    return as_float(__builtin_amdgcn_update_dpp(as_bits(fill), as_bits(v), kCtrl, kRowMask, 0xf, false));
}

// Sum over the 64 lanes, in all of them; the same order of additions every time.
__device__ __forceinline__ float wave_sum(float v)
{
    v += dpp<kDppRowShr1>(0.f, v);
    v += dpp<kDppRowShr2>(0.f, v);
    v += dpp<kDppRowShr4>(0.f, v);
    v += dpp<kDppRowShr8>(0.f, v);
    v += dpp<kDppRowBcast15, 0xa>(0.f, v);
    v += dpp<kDppRowBcast31, 0xc>(0.f, v);
    return as_float(__builtin_amdgcn_readlane(as_bits(v), kWave - 1));
}
__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int step = 1; step < kWave; step <<= 1) v += __shfl_xor(v, step, kWave);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int step = 1; step < kWave; step <<= 1) v = fmaxf(v, __shfl_xor(v, step, kWave));
    return v;
}

__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

__device__ __forceinline__ float dot(f32x8 a, f32x8 b)
{
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v = __builtin_fmaf(a[i], b[i], v);
    return v;
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

inline size_t bytes_of(uint32_t dtype) { return dtype == STALLOC_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Calls f(T()) with the C++ type of a stalloc_dtype; the entry points have checked it.
template <typename F> inline void with_type(uint32_t dtype, F f)
{
    if (dtype == STALLOC_F32) f(float());
    else if (dtype == STALLOC_BF16) f(bf16());
    else f(f16());
}

inline uint32_t umin_host(uint32_t a, uint32_t b) { return a < b ? a : b; }

constexpr uint64_t kMostThreads = 0xffffffffu;              // of a launch

// What a thread's HIP calls so far have left behind they have told by their own return values: it is put aside before the first launch of a call, so that `launched` tells of
// the call's own launches.
inline void begin_launches() { (void)hipGetLastError(); }
inline int launched() { return hipGetLastError() == hipSuccess ? STALLOC_OK : STALLOC_ERR_DEVICE; }

}  // namespace stalloc
