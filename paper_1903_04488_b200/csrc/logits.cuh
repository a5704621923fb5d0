// logits.cuh -- what the kernels over rows of logits share: the running maximum of a row with the sums of e^(z - m) and of
// e^(z - m) (z - m) relative to it, in one pass over 16-byte granules, for logits of any size, infinities and NaN.
#pragma once
#include "formats.cuh"

namespace ssgd {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NEG_INF = -INFINITY;

// 2^x within 2 units of the last place; below 2^-126 it is 0.  One instruction of nine in the loop; the sums' own roundings are of the
// same size: against 64 bits the results are off by 4.6e-8 of their size, those of 32-bit exp and sums by 3.4e-8 (4096 x 32000).
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

__device__ __forceinline__ float min_nan(float a, float b) {
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// Largest magnitude of a format for which the fast path below is taken, with room for the floor.
template <typename T> __device__ __forceinline__ float fast_limit() { return 1e30f; }
template <> __device__ __forceinline__ float fast_limit<__half>() { return 6e4f; }

// The running sums of one thread, relative to its maximum logit m, in powers of two: with c = scale * log2 e, s = sum 2^d and
// w = sum 2^d d.  Two forms of d:
//   near    d = z c - shift, one fma, shift = m c rounded.  As every d is taken from the same shift, the rounding only moves the
//           reference: d at the maximum is not 0 but up to half a unit of shift's last place, 2 while |shift| < NEAR = 2^26
//   far     d = (z - m) c, exact at the maximum however large that is.  Beside a far maximum the logits that matter lie
//           within a factor 2 of it, and z - m is exact, in the logits' own format too.
// The far form is for rows or pieces of rows that hold nothing but a mask's large negative numbers, and for logits far from zero.
struct Sums {
    float m, shift, s, w;
};
constexpr float NEAR = 0x1p26f;
constexpr float HUGE_LOGIT = 1e30f;         // beyond, z c might overflow: logits are taken one by one

__device__ __forceinline__ Sums no_sums() { return Sums{NEG_INF, NEG_INF, 0.f, 0.f}; }
__device__ __forceinline__ bool near(float shift) { return fabsf(shift) < NEAR; }

// To the maximum m.  What the sums lose is 2^(old reference - new reference); a far form's reference is m c itself, unrounded.
__device__ __forceinline__ void rebase(Sums& a, float m, float c) {
    const float shift = __fmul_rn(m, c);
    if (a.m > NEG_INF || a.m != a.m) {
        const bool from_near = near(a.shift), to_near = near(shift);
        const float delta = from_near ? (to_near ? a.shift - shift : -fmaf(m, c, -a.shift)) : (to_near ? fmaf(a.m, c, -shift) : (a.m - m) * c);
        const float f = ex2(delta);
        a.w = f * fmaf(delta, a.s, a.w);
        if (f == 0.f && a.s == a.s && a.w != a.w) a.w = 0.f;   // 0 * -inf: the old part has vanished
        a.s *= f;
    }
    a.m = m;
    a.shift = shift;
}

// Any values: infinities, NaN, magnitudes near the end of the format.
__device__ __forceinline__ void add_careful(Sums& a, float z, float c) {
    const float m = max_nan(a.m, z);
    if (!(m == a.m)) rebase(a, m, c);
    if (z == NEG_INF && a.m == a.m) return;                // contributes nothing, whatever the maximum
    const float d = near(a.shift) ? fmaf(z, c, -a.shift) : (z - a.m) * c, e = ex2(d);
    a.s += e;
    if (e > 0.f || e != e) a.w = fmaf(e, d, a.w);
}

// The sums of all lanes, relative to their common maximum, in every lane
__device__ __forceinline__ void join_warp(Sums& a, float c) {
    const float m = warp_max_nan(a.m);
    if (!(m == a.m)) rebase(a, m, c);
    a.s = warp_sum(a.s);
    a.w = warp_sum(a.w);
}

__device__ __forceinline__ int64_t id_of(const void* ids, bool ids64, int64_t row) {
    return ids64 ? static_cast<const int64_t*>(ids)[row] : (int64_t)static_cast<const int32_t*>(ids)[row];
}

// The granules of a row: granule i covers elements [i VEC - phase, (i + 1) VEC - phase) within [0, n).
template <typename T> struct Granules {
    static constexpr int VEC = 16 / sizeof(T);
    const T* row; int32_t n, phase, count;
    __device__ __forceinline__ Granules(const T* p, int32_t n_) : row(p), n(n_) {
        phase = (int32_t)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
        count = (n + phase + VEC - 1) / VEC;
    }
    __device__ __forceinline__ int32_t first(int32_t i) const { return i * VEC - phase; }
    __device__ __forceinline__ bool whole(int32_t i) const { return first(i) >= 0 && first(i) + VEC <= n; }
};

// Running maximum of the elements of granules, two at a time (NaN if one is)
template <typename T> struct PairMax;
template <> struct PairMax<float> {
    float2 m;
    __device__ __forceinline__ explicit PairMax(float x) : m(both(x)) {}
    __device__ __forceinline__ void add(const Vec<float, 4>& v) {
        m.x = max_nan(m.x, max_nan(v.e[0], v.e[1]));
        m.y = max_nan(m.y, max_nan(v.e[2], v.e[3]));
    }
    __device__ __forceinline__ float value() const { return max_nan(m.x, m.y); }
};
template <> struct PairMax<__nv_bfloat16> {
    __nv_bfloat162 m;
    __device__ __forceinline__ explicit PairMax(float x) : m(__float2bfloat162_rn(x)) {}
    __device__ __forceinline__ void add(const Vec<__nv_bfloat16, 8>& v) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        m = __hmax2_nan(m, __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
    }
    __device__ __forceinline__ float value() const { return max_nan(__low2float(m), __high2float(m)); }
};
template <> struct PairMax<__half> {
    __half2 m;
    __device__ __forceinline__ explicit PairMax(float x) : m(__float2half2_rn(x)) {}
    __device__ __forceinline__ void add(const Vec<__half, 8>& v) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
        m = __hmax2_nan(m, __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
    }
    __device__ __forceinline__ float value() const { return max_nan(__low2float(m), __high2float(m)); }
};

// A granule with everything below `low` raised to it (low is a number of the format)
__device__ __forceinline__ Vec<float, 4> raised(Vec<float, 4> v, float low) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v.e[e] = fmaxf(v.e[e], low);
    return v;
}
__device__ __forceinline__ Vec<__nv_bfloat16, 8> raised(Vec<__nv_bfloat16, 8> v, float low) {
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
    const __nv_bfloat162 l = __float2bfloat162_rn(low);
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __hmax2(h[e], l);
    return v;
}
__device__ __forceinline__ Vec<__half, 8> raised(Vec<__half, 8> v, float low) {
    __half2* h = reinterpret_cast<__half2*>(&v);
    const __half2 l = __float2half2_rn(low);
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __hmax2(h[e], l);
    return v;
}

// A granule less m (a number of the format)
__device__ __forceinline__ Vec<float, 4> less(Vec<float, 4> v, float m) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v.e[e] -= m;
    return v;
}
__device__ __forceinline__ Vec<__nv_bfloat16, 8> less(Vec<__nv_bfloat16, 8> v, float m) {
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
    const __nv_bfloat162 l = __float2bfloat162_rn(m);
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __hsub2(h[e], l);
    return v;
}
__device__ __forceinline__ Vec<__half, 8> less(Vec<__half, 8> v, float m) {
    __half2* h = reinterpret_cast<__half2*>(&v);
    const __half2 l = __float2half2_rn(m);
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __hsub2(h[e], l);
    return v;
}

// A value no larger than m - reach, reach = 160 / c rounded up, and below every element that could matter: elements under it
// are raised to it, so that -inf does not make 0 * -inf.  2^-160 is zero in fp32.
template <typename T> __device__ __forceinline__ float floor_for(float m, float reach) { return __fsub_rd(m, reach); }
template <> __device__ __forceinline__ float floor_for<__nv_bfloat16>(float m, float reach) {
    return __bfloat162float(__float2bfloat16_rd(__fsub_rd(m, reach)));
}
template <> __device__ __forceinline__ float floor_for<__half>(float m, float reach) {
    return __half2float(__float2half_rd(__fsub_rd(m, reach)));
}

// What a thread carries along a row
struct Running {
    Sums a;
    float low;           // elements below it are raised to it; -inf: they are taken one by one
    float c, reach;
};

template <typename T>
__device__ __noinline__ Sums add_granule_carefully(Sums a, Vec<T, 16 / sizeof(T)> v, float c) {
    for (int e = 0; e < 16 / (int)sizeof(T); ++e) add_careful(a, to_f32(v.e[e]), c);
    return a;
}

// Granules v[0] .. v[have - 1] (`have` is the same for the whole CTA); returns their maximum.  Elements that are not there are -inf: they change neither
// the maximum nor the sums.
template <typename T, int U>
__device__ __forceinline__ float add_granules(Running& r, Vec<T, 16 / sizeof(T)> (&v)[U], int have) {
    constexpr int VEC = 16 / sizeof(T);
    PairMax<T> top(NEG_INF);
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < have) top.add(v[u]);
    const float here = top.value(), m = max_nan(r.a.m, here);
    if (!(m == r.a.m)) {
        rebase(r.a, m, r.c);
        r.low = fabsf(m) < fast_limit<T>() && fabsf(r.a.shift) < HUGE_LOGIT ? floor_for<T>(m, r.reach) : NEG_INF;
    }
    if (r.low > NEG_INF) {
        float low = r.low, shift = r.a.shift;
        if (!near(shift)) {                                // (z - m) c + 0
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u < have) v[u] = less(raised(v[u], low), m);
            low = -fast_limit<T>();
            shift = 0.f;
        }
        const float2 minus_shift = both(-shift), c2 = both(r.c);
        float2 s = both(0.f), w = both(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u < have) {
                float2 f[VEC / 2];
                unpack_pairs(raised(v[u], low), f);
#pragma unroll
                for (int e = 0; e < VEC / 2; ++e) {
                    const float2 d = fma2(f[e], c2, minus_shift), x = make_float2(ex2(d.x), ex2(d.y));
                    s = add2(s, x);
                    w = fma2(x, d, w);
                }
            }
        }
        r.a.s += s.x + s.y;
        r.a.w += w.x + w.y;
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < have) r.a = add_granule_carefully<T>(r.a, v[u], r.c);
    }
    return here;
}

}  // namespace ssgd
