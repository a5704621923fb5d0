// formats.cuh -- the element formats of the training operators (fp32, IEEE binary16, bfloat16): vectors of VEC
// elements as they lie in memory, their conversion to and from fp32, and the checks of bases and row strides that
// decide how wide a vector may be.  All arithmetic is fp32; a value is rounded once, to nearest even, when stored.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/ssgd.h"

namespace ssgd {

template <int BYTES> struct RawOf;
template <> struct RawOf<16> { using type = uint4; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<2> { using type = uint16_t; };

// VEC elements of T, the unit of one load or store.
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Vec {
    T e[VEC];
};

template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> load_vec(const T* p) {
    using Raw = typename RawOf<sizeof(T) * VEC>::type;
    union { Raw r; Vec<T, VEC> v; } u;
    u.r = *reinterpret_cast<const Raw*>(p);
    return u.v;
}
// read-only data that is used once: not kept in L1
template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> load_vec_stream(const T* p) {
    using Raw = typename RawOf<sizeof(T) * VEC>::type;
    union { Raw r; Vec<T, VEC> v; } u;
    u.r = __ldcs(reinterpret_cast<const Raw*>(p));
    return u.v;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, VEC>& v) {
    using Raw = typename RawOf<sizeof(T) * VEC>::type;
    union { Raw r; Vec<T, VEC> v; } u;
    u.v = v;
    *reinterpret_cast<Raw*>(p) = u.r;
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <typename T, int VEC>
__device__ __forceinline__ void unpack(const Vec<T, VEC>& v, float (&f)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = to_f32(v.e[i]);
}
template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> pack(const float (&f)[VEC]) {
    Vec<T, VEC> v;
#pragma unroll
    for (int i = 0; i < VEC; ++i) v.e[i] = from_f32<T>(f[i]);
    return v;
}

// Host side -----------------------------------------------------------------------------------------

inline int fmt_bytes(int32_t fmt) {
    return fmt == SSGD_FMT_F32 ? 4 : fmt == SSGD_FMT_F16 || fmt == SSGD_FMT_BF16 ? 2 : 0;
}
inline uint64_t addr(const void* p) { return (uint64_t)reinterpret_cast<uintptr_t>(p); }
inline bool aligned_to(const void* p, int bytes) { return addr(p) % (uint64_t)bytes == 0; }

// Multiprocessors of the current device (looked up once per device).
inline int sm_count_of_current_device(int* out) {
    static int known[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SSGD_ECUDA;
    if (!known[dev]) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return SSGD_ECUDA;
        known[dev] = n;      // the same value whichever thread stores it
    }
    *out = known[dev];
    return SSGD_OK;
}

inline int launched() { return cudaGetLastError() == cudaSuccess ? SSGD_OK : SSGD_ECUDA; }

}  // namespace ssgd
