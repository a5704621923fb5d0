// formats.cuh -- the element formats of the training operators (fp32, IEEE binary16, bfloat16): vectors of VEC
// elements as they lie in memory, their conversion to and from fp32, and the checks of bases and row strides that
// decide how wide a vector may be.  All arithmetic is fp32; a value is rounded once, to nearest even, when stored.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <type_traits>

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

// Pairs of fp32 numbers: one instruction works on both (rounding each like the scalar operation).
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// VEC elements as pairs in fp32; a single element has 0 beside it.
template <int VEC> constexpr int PAIRS = (VEC + 1) / 2;
template <typename T, int VEC>
__device__ __forceinline__ void unpack_pairs(const Vec<T, VEC>& v, float2 (&f)[PAIRS<VEC>]) {
    if constexpr (VEC == 1) {
        f[0] = make_float2(to_f32(v.e[0]), 0.f);
    } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    } else if constexpr (std::is_same<T, __half>::value) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) f[i] = __half22float2(h[i]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) f[i] = make_float2(v.e[2 * i], v.e[2 * i + 1]);
    }
}
template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> pack_pairs(const float2 (&f)[PAIRS<VEC>]) {
    Vec<T, VEC> v;
    if constexpr (VEC == 1) {
        v.e[0] = from_f32<T>(f[0].x);
    } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) h[i] = __floats2bfloat162_rn(f[i].x, f[i].y);
    } else if constexpr (std::is_same<T, __half>::value) {
        __half2* h = reinterpret_cast<__half2*>(&v);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) h[i] = __floats2half2_rn(f[i].x, f[i].y);
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) { v.e[2 * i] = f[i].x; v.e[2 * i + 1] = f[i].y; }
    }
    return v;
}

// Largest over the warp, NaN if any lane has one
__device__ __forceinline__ float warp_max_nan(float x) {
    float y;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// BYTES (4, 8 or 16, both sides aligned to it) on their way from global to shared memory while the thread goes on.  A
// thread that reads only what it has copied itself needs no barrier: the wait below is enough.
template <int BYTES>
__device__ __forceinline__ void copy_async(void* shared, const void* global) {
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(shared);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(global) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(global), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until at most N of this thread's committed groups are still on their way
template <int N>
__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Programmatic dependent launch: a kernel launched with launch_after may start while its predecessor in the stream drains; it
// sees what that wrote once successor_wait has returned.
__device__ __forceinline__ void successor_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void successor_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Host side -----------------------------------------------------------------------------------------

inline int fmt_bytes(int32_t fmt) {
    return fmt == SSGD_FMT_F32 ? 4 : fmt == SSGD_FMT_F16 || fmt == SSGD_FMT_BF16 ? 2 : 0;
}
inline uint64_t addr(const void* p) { return (uint64_t)reinterpret_cast<uintptr_t>(p); }
inline bool aligned_to(const void* p, int bytes) { return addr(p) % (uint64_t)bytes == 0; }

// A fact about each device, 0 until it has been asked for
constexpr int MAX_DEVICES = 64;
struct PerDevice { std::atomic<int> value[MAX_DEVICES] = {}; };

// Multiprocessors of the current device (looked up once per device).
inline int sm_count_of_current_device(int* out) {
    static PerDevice known;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return SSGD_ECUDA;
    int n = known.value[dev];
    if (!n) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return SSGD_ECUDA;
        known.value[dev] = n;      // the same value whichever thread stores it
    }
    *out = n;
    return SSGD_OK;
}

// CTAs of a kernel that fit an SM at once (asked once per kernel and device: the answer does not change, and asking costs as
// much as a launch).  `known` belongs to the kernel; smem above 40 KB is opted into on the way.
template <typename K>
inline int residency(K kernel, int block, size_t smem, PerDevice& known, int* out) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return SSGD_ECUDA;
    int n = known.value[dev];
    if (!n) {
        if (smem > 40 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
            return SSGD_ECUDA;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, block, smem) != cudaSuccess || n < 1) return SSGD_ECUDA;
        known.value[dev] = n;      // the same value whichever thread stores it
    }
    *out = n;
    return SSGD_OK;
}

template <typename... P, typename... A>
int launch_after(cudaStream_t st, void (*kernel)(P...), dim3 grid, int block, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)block);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess ? SSGD_OK : SSGD_ECUDA;
}

inline int launched() { return cudaGetLastError() == cudaSuccess ? SSGD_OK : SSGD_ECUDA; }

}  // namespace ssgd
