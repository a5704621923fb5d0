// adamw.cu -- one AdamW step over many tensors at once (ssgd_adamw_step).
//
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2
//   p <- p (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by HBM: with everything in fp32 an element costs 28 bytes (p, g, m, v read, p, m, v written) and some twenty
// operations.  All tensors go in one launch (or one per MAX_TENSORS of them): the table of tensors travels in the
// kernel's arguments, so there is nothing to upload or to keep, and a block finds its tensor by bisection.
//
// 8-bit states.  256 consecutive elements share a scale (fp32, the largest magnitude / 448); m / scale and
// sqrt(v) / scale are held as e4m3 numbers (4 exponent bits, 3 fraction bits).  sqrt(v) and not v: the format spans
// 2^18, which is 2^36 in v.  Rounding is stochastic when a seed is given: with 3 fraction bits the change of one step,
// (1 - b2) g^2, is far below half a unit, and rounding to nearest would never move v.  The dither of an element is a
// hash of (seed, tensor, index), so a step is reproducible and independent of the schedule.  sqrt(v) > 0 never rounds
// to 0: the element would be divided by eps alone.  A value that is not finite becomes the format's NaN and does not
// touch its neighbours' scale.  What decides a code or a scale is rounded operation by operation as ssgd.h states it: a code
// that comes out one higher in one step can be its block's largest in the next, and then the whole block differs by per cents.
// Only the parameter's own update takes approximate roots and reciprocals (2^-23 each, beside 2^-4 from the state's codes).
#include <cuda_fp8.h>

#include <cmath>

#include "formats.cuh"

using namespace ssgd;

namespace {

constexpr int THREADS = 256;
constexpr int MAX_TENSORS = 384;           // 30 KB of kernel arguments
constexpr int FEW_TENSORS = 40;            // 3 KB: small arguments cost less to launch
constexpr int QBLOCK = SSGD_ADAMW_BLOCK;   // elements per scale
constexpr int UNROLL32 = 2;                // vectors of 4 per thread and chunk (fp32 states)
constexpr int CHUNK32 = THREADS * 4 * UNROLL32;
constexpr int MAX_BLOCKS8 = 8;             // blocks of 256 per warp and chunk (8-bit states): up to this many

struct Entry {
    void* p; const void* g; void* m; void* v; float* ms; float* vs; void* copy;
    int64_t n;
    uint32_t key;        // dither key of the tensor
    int32_t head;        // elements before the first aligned vector; -1: no common alignment
};
struct Hyper {
    float b1, omb1, b2, omb2, keep, step_size, inv_bc2, eps, one;
    const float* grad_scale;
    int32_t copy_f16;    // the copy is binary16, else bfloat16
    int32_t blocks8;     // blocks per warp and chunk (8-bit states)
};
template <int CAP>
struct Table {
    Hyper h;
    int32_t count;
    uint32_t first[CAP + 1];   // first chunk of each tensor
    Entry t[CAP];
};

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

// The tensor of a chunk: the last one whose first chunk is not behind it.
template <int CAP>
__device__ __forceinline__ int tensor_of(const Table<CAP>& T, uint32_t chunk) {
    int lo = 0, hi = T.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (T.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// ---- states in fp32 ----------------------------------------------------------------------------------

__device__ __forceinline__ void update(const Hyper& h, float gs, float& p, float g, float& m, float& v) {
    g *= gs;
    m = fmaf(m, h.b1, g * h.omb1);
    v = fmaf(v, h.b2, g * g * h.omb2);
    p = fmaf(p, h.keep, -h.step_size * (m / fmaf(sqrtf(v), h.inv_bc2, h.eps)));
}

// bfloat16 parameters without an fp32 original: with a seed they round stochastically too (16 bits of dither), since
// an update is mostly below half a unit of the parameter's last bit.
__device__ __forceinline__ uint32_t bf16_dithered(float x, uint32_t word) {
    if (!(fabsf(x) < INFINITY)) return __bfloat16_as_ushort(__float2bfloat16_rn(x));
    return (__float_as_uint(x) + ((word * 0x9E3779B9u) >> 16)) >> 16;
}

template <typename P>
__device__ __forceinline__ P round_param(float x, bool stochastic, uint32_t word) {
    if constexpr (sizeof(P) == 2) {
        if (stochastic) return __ushort_as_bfloat16((unsigned short)bf16_dithered(x, word));
        return __float2bfloat16_rn(x);
    } else {
        return x;
    }
}
__device__ __forceinline__ unsigned short round_copy(float x, bool f16) {
    return f16 ? __half_as_ushort(__float2half_rn(x)) : __bfloat16_as_ushort(__float2bfloat16_rn(x));
}
__device__ __forceinline__ uint32_t dither_word(uint32_t key, int64_t i) {
    return mix(key ^ (uint32_t)i ^ ((uint32_t)((uint64_t)i >> 32) * 0x9E3779B9u));
}

// A chunk of 2048 elements per block: two vectors of four per thread from each of p, g, m, v on their way at once, what has no
// common alignment element by element.  Measured in fp32: 11,173,962 elements in 62 tensors at any offset 51.3 us, 6.1 TB/s (0.93
// of a copy), with a bfloat16 copy 55.4; 29,060,773 in 198 tensors 123 us, 6.6 TB/s, with a copy 134.  bfloat16 parameters and
// gradients, 11,173,962 in 62 tensors 42.2 us, 5.8 TB/s; without a common alignment 90.
template <typename P, typename G, int CAP, bool STOCHASTIC>
__global__ void __launch_bounds__(THREADS) k_adamw_f32(const __grid_constant__ Table<CAP> T) {
    const Hyper& h = T.h;
    const int k = tensor_of(T, blockIdx.x);
    const Entry& E = T.t[k];
    P* p = static_cast<P*>(E.p);
    const G* g = static_cast<const G*>(E.g);
    float* m = static_cast<float*>(E.m);
    float* v = static_cast<float*>(E.v);
    unsigned short* copy = static_cast<unsigned short*>(E.copy);
    const int64_t n = E.n;
    const float gs = h.grad_scale ? *h.grad_scale : 1.f;
    auto one = [&](int64_t i) {
        float pi = to_f32(p[i]), mi = m[i], vi = v[i];
        update(h, gs, pi, to_f32(g[i]), mi, vi);
        p[i] = round_param<P>(pi, STOCHASTIC, STOCHASTIC ? dither_word(E.key, i) : 0u);
        m[i] = mi;
        v[i] = vi;
        if (copy) copy[i] = round_copy(pi, h.copy_f16);
    };
    const int64_t base = (int64_t)(blockIdx.x - T.first[k]) * CHUNK32;
    if (E.head < 0) {
        const int64_t end = base + CHUNK32 < n ? base + CHUNK32 : n;
        for (int64_t i = base + threadIdx.x; i < end; i += THREADS) one(i);
        return;
    }
    if (base == 0 && (int)threadIdx.x < E.head && (int64_t)threadIdx.x < n) one(threadIdx.x);
    Vec<P, 4> vp[UNROLL32];
    Vec<G, 4> vg[UNROLL32];
    Vec<float, 4> vm[UNROLL32], vv[UNROLL32];
    const int64_t i0 = base + E.head + threadIdx.x * 4;
#pragma unroll
    for (int u = 0; u < UNROLL32; ++u) {
        const int64_t i = i0 + u * THREADS * 4;
        if (i + 4 <= n) {
            vp[u] = load_vec<P, 4>(p + i);
            vg[u] = load_vec_stream<G, 4>(g + i);
            vm[u] = load_vec<float, 4>(m + i);
            vv[u] = load_vec<float, 4>(v + i);
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL32; ++u) {
        const int64_t i = i0 + u * THREADS * 4;
        if (i + 4 <= n) {
            float fp[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                fp[e] = to_f32(vp[u].e[e]);
                update(h, gs, fp[e], to_f32(vg[u].e[e]), vm[u].e[e], vv[u].e[e]);
                vp[u].e[e] = round_param<P>(fp[e], STOCHASTIC, STOCHASTIC ? dither_word(E.key, i + e) : 0u);
            }
            store_vec<P, 4>(p + i, vp[u]);
            store_vec<float, 4>(m + i, vm[u]);
            store_vec<float, 4>(v + i, vv[u]);
            if (copy) {
                Vec<unsigned short, 4> c;
#pragma unroll
                for (int e = 0; e < 4; ++e) c.e[e] = round_copy(fp[e], h.copy_f16);
                store_vec<unsigned short, 4>(copy + i, c);
            }
        } else {
            for (int64_t j = i; j < n; ++j) one(j);
        }
    }
}

// ---- states in 8 bits --------------------------------------------------------------------------------

// Two e4m3 codes (lower byte first) as numbers
__device__ __forceinline__ float2 e4m3_pair(uint32_t codes) {
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, __NV_E4M3);
    return __half22float2(__half2(r));
}

// Rounding to e4m3 in the bits of fp32.  The code of a magnitude x in a block whose largest is a: y = x (448 (1 / a)), every
// operation rounded by itself, and floor(y / unit + u), where the unit is 2^-9 below y = 2^-5 and 2^(e - 9) in [2^(e - 6),
// 2^(e - 5)), and u in (0, 1) the dither, a multiple of 2^-17.  y times 2^-120 is an fp32 number (a subnormal where y / unit is
// one in e4m3) whose exponent and first three fraction bits ARE the code, at bit 20: adding u 2^20 to the bits and dropping the
// lower 20 does it, carries into the exponent included.  Two things make that inexact: a subnormal is rounded to 2^-20 units of
// the code once more, and the root is sqrt.approx (within 2^-23; with the roundings around it 5 units of y's last place).  Neither
// decides anything unless the sum ends up within ERROR of a multiple of 2^20; then code_of does what the formula says.
constexpr uint32_t ERROR = 8;
constexpr float LARGEST_SCALED = 0x1p14f;                  // of more, 2^-120 448 / a would be a subnormal
__device__ __forceinline__ uint32_t from_border(uint32_t sum) { return (sum << 12) + (ERROR << 12); }
__device__ __forceinline__ bool near_border(uint32_t least) { return least < (2 * ERROR) << 12; }
__device__ __forceinline__ uint32_t code_of(float x, float per_scale, uint32_t u20) {
    const float y = __fmul_rn(x, per_scale);
    if (y >= 0x1p-6f) return __float_as_uint(y) + u20 - (120u << 23);
    return (uint32_t)__fadd_rn(y * 512.f, (float)u20 * 0x1p-20f) << 20;
}
// The codes of four such sums x (sign in front), in one word.  Two at a time: their upper halves side by side and shifted left by
// 4, each half's upper byte is a code once the sign is put in front of it again.
template <bool SIGNED>
__device__ __forceinline__ uint32_t e4m3_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const uint32_t ab = __byte_perm(a, b, 0x7632), cd = __byte_perm(c, d, 0x7632);
    uint32_t lo = ab << 4, hi = cd << 4;
    if (SIGNED) {
        lo = (lo & 0x7fff7fffu) | (ab & 0x80008000u);
        hi = (hi & 0x7fff7fffu) | (cd & 0x80008000u);
    }
    return __byte_perm(lo, hi, 0x7531);
}
__device__ __forceinline__ float sqrt_fast(float x) {
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Smallest of a, b, c; a NaN does not count
__device__ __forceinline__ float min3(float a, float b, float c) {
    float y;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float y;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ float warp_max(float x) {         // of magnitudes, which order like their bits; NaN above all
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x)));
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// What a lane reads of a block
template <typename P, typename G>
struct Block {
    Vec<P, 16 / sizeof(P)> p[sizeof(P) / 2];
    Vec<G, 16 / sizeof(G)> g[sizeof(G) / 2];
    uint2 m, v;
};
// Where a chunk begins (the same in all threads), and its number of elements
template <typename P, typename G>
struct Chunk {
    P* p; const G* g; uint8_t* m; uint8_t* v; unsigned short* copy;
    int32_t n;
};
template <typename T>
__device__ __forceinline__ void eight(const Vec<T, 16 / sizeof(T)> (&v)[sizeof(T) / 2], float2 (&f)[4]) {
    if constexpr (sizeof(T) == 2) {
        unpack_pairs(v[0], f);
    } else {
        f[0] = make_float2(v[0].e[0], v[0].e[1]); f[1] = make_float2(v[0].e[2], v[0].e[3]);
        f[2] = make_float2(v[1].e[0], v[1].e[1]); f[3] = make_float2(v[1].e[2], v[1].e[3]);
    }
}
// A block on its way through shared memory; each lane copies what it will read itself
template <typename P, typename G>
struct alignas(16) Staged {
    Vec<P, 16 / sizeof(P)> p[sizeof(P) / 2][32];
    Vec<G, 16 / sizeof(G)> g[sizeof(G) / 2][32];
    uint2 m[32], v[32];
};
// `at`: the lane's first element within the chunk
template <typename P, typename G>
__device__ __forceinline__ void send(Staged<P, G>& s, const Chunk<P, G>& C, uint32_t at) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < (int)sizeof(P) / 2; ++k) copy_async<16>(&s.p[k][lane], C.p + at + k * 4);
#pragma unroll
    for (int k = 0; k < (int)sizeof(G) / 2; ++k) copy_async<16>(&s.g[k][lane], C.g + at + k * 4);
    copy_async<8>(&s.m[lane], C.m + at);
    copy_async<8>(&s.v[lane], C.v + at);
}
template <typename P, typename G>
__device__ __forceinline__ Block<P, G> taken(const Staged<P, G>& s) {
    const int lane = threadIdx.x & 31;
    Block<P, G> b;
#pragma unroll
    for (int k = 0; k < (int)sizeof(P) / 2; ++k) b.p[k] = s.p[k][lane];
#pragma unroll
    for (int k = 0; k < (int)sizeof(G) / 2; ++k) b.g[k] = s.g[k][lane];
    b.m = s.m[lane];
    b.v = s.v[lane];
    return b;
}

// The step's constants in the form the 8-bit kernel uses them
struct Hyper8 {
    float gs, b1, omb1, b2, omb2, keep, minus_step, inv_bc2, eps;
    float one;      // 1, which the compiler does not know: x * one + y is a sum whose operands it cannot leave unrounded (it
                    // contracts mul.rn.f32x2 and add.rn.f32x2 to one fma, unlike their scalar forms)
};

__device__ __forceinline__ float part(const float2 (&f)[4], int j) { return j & 1 ? f[j / 2].y : f[j / 2].x; }

// One block of 256 elements by a warp: lane l has the elements 8 l .. 8 l + 7 when everything is aligned for it (VECTOR: read
// into `in`), otherwise the elements l, l + 32, ..., as far as the chunk goes.  The codes and scales are the same either way.
// `first` is the block's first element within the chunk, `index` the low half of its index in the tensor, mixed with the
// tensor's key; ms and vs are the block's scales, replaced by the new ones.
template <typename P, typename G, bool STOCHASTIC, bool VECTOR>
__device__ __forceinline__ void block8(const Hyper8& h, uint32_t index, const Chunk<P, G>& C, uint32_t first, const Block<P, G>& in,
                                       int32_t copy_f16, float& ms_io, float& vs_io) {
    const int lane = threadIdx.x & 31;
    const uint32_t lane8 = first + lane * 8;
    auto at = [&](int j) { return first + lane + 32 * j; };
    float2 fp[4], fg[4], fm[4], fr[4];
    if (VECTOR) {
        eight<P>(in.p, fp);
        eight<G>(in.g, fg);
        fm[0] = e4m3_pair(in.m.x & 0xffffu); fm[1] = e4m3_pair(in.m.x >> 16); fm[2] = e4m3_pair(in.m.y & 0xffffu); fm[3] = e4m3_pair(in.m.y >> 16);
        fr[0] = e4m3_pair(in.v.x & 0xffffu); fr[1] = e4m3_pair(in.v.x >> 16); fr[2] = e4m3_pair(in.v.y & 0xffffu); fr[3] = e4m3_pair(in.v.y >> 16);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t i0 = at(2 * j), i1 = at(2 * j + 1);
            const bool in0 = i0 < (uint32_t)C.n, in1 = i1 < (uint32_t)C.n;
            fp[j] = make_float2(in0 ? to_f32(C.p[i0]) : 0.f, in1 ? to_f32(C.p[i1]) : 0.f);
            fg[j] = make_float2(in0 ? to_f32(C.g[i0]) : 0.f, in1 ? to_f32(C.g[i1]) : 0.f);
            fm[j] = e4m3_pair((in0 ? C.m[i0] : 0u) | (in1 ? C.m[i1] : 0u) << 8);
            fr[j] = e4m3_pair((in0 ? C.v[i0] : 0u) | (in1 ? C.v[i1] : 0u) << 8);
        }
    }
    const float2 ms = both(ms_io), vs = both(vs_io);
    float am = 0.f, av = 0.f, ap = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 g = mul2(fg[j], both(h.gs));
        const float2 m = fma2(mul2(mul2(fm[j], ms), both(h.b1)), both(h.one), mul2(g, both(h.omb1)));
        const float2 r0 = mul2(fr[j], vs);
        const float2 v = fma2(mul2(mul2(r0, r0), both(h.b2)), both(h.one), mul2(mul2(g, g), both(h.omb2)));
        const float2 denom = fma2(make_float2(sqrt_fast(v.x), sqrt_fast(v.y)), both(h.inv_bc2), both(h.eps));
        const float2 q = mul2(m, make_float2(rcp_fast(denom.x), rcp_fast(denom.y)));
        fp[j] = fma2(q, both(h.minus_step), mul2(fp[j], both(h.keep)));
        fm[j] = m;
        fr[j] = v;
        am = max3_nan(am, fabsf(m.x), fabsf(m.y));
        av = max3_nan(av, v.x, v.y);
        if (sizeof(P) == 2) ap = max3_nan(ap, fabsf(fp[j].x), fabsf(fp[j].y));
    }
    // Rare: a value that is not finite.  It must not count for the scale, and its code is NaN
    const bool odd = __any_sync(0xffffffffu, !(max3_nan(am, av, ap) < INFINITY));
    if (odd) {
        am = av = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (finite(part(fm, j))) am = fmaxf(am, fabsf(part(fm, j)));
            if (finite(part(fr, j))) av = fmaxf(av, part(fr, j));
        }
    }
    am = warp_max(am);
    const float ar = __fsqrt_rn(warp_max(av));             // roots rounded to nearest are in order
    // Below 2^-100 the block is held as zeros
    const float least = 0x1p-100f, scale_m = am * (1.f / 448.f), scale_r = ar * (1.f / 448.f);
    const float per_m = am < least ? 0.f : __fmul_rn(__frcp_rn(am), 448.f), per_r = ar < least ? 0.f : __fmul_rn(__frcp_rn(ar), 448.f);
    const float im = per_m * 0x1p-120f, ir = per_r * 0x1p-120f;
    if (lane == 0) {
        ms_io = am < least ? 0.f : scale_m;
        vs_io = ar < least ? 0.f : scale_r;
    }
    // The dither of element i is the hash of key ^ i (see dither_word).  What belongs to the chunk, to the lane and to j has no
    // bits in common, and j none above the 16th, so the first step of the mixing is the same for all j.  16 bits each (m: the
    // lower half of the word, v: the upper) at bit 4, in the middle of their interval; without a seed 1/2: to nearest.
    uint32_t seed = index ^ (VECTOR ? lane8 : at(0));
    seed ^= seed >> 16;
    auto mixed = [&](uint32_t seed, int j) {
        uint32_t r = seed ^ (uint32_t)(VECTOR ? j : 32 * j);
        r *= 0x6A09E667u;
        r ^= r >> 15;
        return r * 0xBB67AE85u;                              // the word is r ^ (r >> 16)
    };
    auto dither_m = [&](uint32_t r) { return STOCHASTIC ? ((r >> 12) ^ (r << 4)) & 0xffff0u : 0x80000u - 8u; };
    auto dither_v = [&](uint32_t r) { return STOCHASTIC ? (r >> 12) & 0xffff0u : 0x80000u - 8u; };
    uint32_t out_m[2], out_v[2], out_p[4];
    uint32_t border = ~0u, least_v = ~0u;                    // least_v: bits of v less 1, so that zeros do not count
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t code_m[4], code_v[4], np[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int j = half * 4 + q;
            const float2 v = fr[j / 2], ym = mul2(fm[j / 2], both(im)), yr = mul2(make_float2(sqrt_fast(v.x), sqrt_fast(v.y)), both(ir));
            const uint32_t r = STOCHASTIC ? mixed(seed, j) : 0u;
            code_m[q] = __float_as_uint(j & 1 ? ym.y : ym.x) + dither_m(r) + 8u;
            code_v[q] = __float_as_uint(j & 1 ? yr.y : yr.x) + dither_v(r) + 8u;
            if (sizeof(P) == 2) np[q] = STOCHASTIC ? __float_as_uint(part(fp, j)) + (((r ^ (r >> 16)) * 0x9E3779B9u) >> 16)
                                                   : (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(part(fp, j))) << 16;
            if (q & 1) {
                least_v = __vimin3_u32(least_v, __float_as_uint(v.x) - 1u, __float_as_uint(v.y) - 1u);
                border = __vimin3_u32(border, from_border(code_m[q - 1]), from_border(code_m[q]));
                border = __vimin3_u32(border, from_border(code_v[q - 1]), from_border(code_v[q]));
            }
        }
        out_m[half] = e4m3_codes<true>(code_m[0], code_m[1], code_m[2], code_m[3]);
        out_v[half] = e4m3_codes<false>(code_v[0], code_v[1], code_v[2], code_v[3]);
        if constexpr (sizeof(P) == 2) {                      // bfloat16 parameters: the new value in the upper half of a word
            out_p[half * 2] = __byte_perm(np[0], np[1], 0x7632);
            out_p[half * 2 + 1] = __byte_perm(np[2], np[3], 0x7632);
        }
    }
    // Seldom: everything again, with care.  From the hash on, so that nothing has to be kept for it.
    const float smallest = least_v == ~0u ? INFINITY : sqrt_fast(__uint_as_float(least_v)) * per_r;    // of the positive ones
    if (odd || !(fmaxf(am, ar) <= LARGEST_SCALED) || !(smallest >= 0x1p-8f) || near_border(border)) {
        float again_m = per_m, again_r = per_r;
        asm volatile("" : "+r"(seed), "+f"(again_m), "+f"(again_r));
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t code_m[4], code_v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int j = half * 4 + q;
                const float m = part(fm, j), v = part(fr, j);
                const uint32_t r = STOCHASTIC ? mixed(seed, j) : 0u, dm = dither_m(r) + 8u, dv = dither_v(r) + 8u;
                code_m[q] = __float_as_uint(__fmul_rn(m, again_m) * 0x1p-120f) + dm;
                if (near_border(from_border(code_m[q]))) code_m[q] = code_of(fabsf(m), again_m, dm) | (__float_as_uint(m) & 0x80000000u);
                code_v[q] = __float_as_uint(__fmul_rn(sqrt_fast(v), again_r) * 0x1p-120f) + dv;
                // a positive value keeps at least the smallest code (and here comes what sqrt.approx has flushed to zero)
                if (v > 0.f && (code_v[q] < 1u << 20 || near_border(from_border(code_v[q])))) code_v[q] = max(code_of(__fsqrt_rn(v), again_r, dv), 1u << 20);
                if (!finite(m)) code_m[q] = 0x7fu << 20;     // the format's NaN
                if (!finite(v)) code_v[q] = 0x7fu << 20;
                if constexpr (sizeof(P) == 2) {              // no dither may touch what is not finite
                    const float x = part(fp, j);
                    const uint32_t np = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x));
                    if (STOCHASTIC && !finite(x)) out_p[j / 2] = j & 1 ? (out_p[j / 2] & 0xffffu) | np << 16 : (out_p[j / 2] & 0xffff0000u) | np;
                }
            }
            out_m[half] = e4m3_codes<true>(code_m[0], code_m[1], code_m[2], code_m[3]);
            out_v[half] = e4m3_codes<false>(code_v[0], code_v[1], code_v[2], code_v[3]);
        }
    }
    if (VECTOR) {
        *reinterpret_cast<uint2*>(C.m + lane8) = make_uint2(out_m[0], out_m[1]);
        *reinterpret_cast<uint2*>(C.v + lane8) = make_uint2(out_v[0], out_v[1]);
        if constexpr (sizeof(P) == 2) {
            *reinterpret_cast<uint4*>(C.p + lane8) = make_uint4(out_p[0], out_p[1], out_p[2], out_p[3]);
        } else {
            float4* o = reinterpret_cast<float4*>(C.p + lane8);
            o[0] = make_float4(fp[0].x, fp[0].y, fp[1].x, fp[1].y);
            o[1] = make_float4(fp[2].x, fp[2].y, fp[3].x, fp[3].y);
        }
        if (C.copy) {
            Vec<unsigned short, 8> c;
#pragma unroll
            for (int j = 0; j < 8; ++j) c.e[j] = round_copy(part(fp, j), copy_f16);
            store_vec<unsigned short, 8>(C.copy + lane8, c);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t i = at(j);
            if (i < (uint32_t)C.n) {
                C.m[i] = (uint8_t)(out_m[j / 4] >> (8 * (j % 4)));
                C.v[i] = (uint8_t)(out_v[j / 4] >> (8 * (j % 4)));
                if constexpr (sizeof(P) == 2) C.p[i] = __ushort_as_bfloat16((unsigned short)(out_p[j / 2] >> (16 * (j % 2))));
                else C.p[i] = part(fp, j);
                if (C.copy) C.copy[i] = round_copy(part(fp, j), copy_f16);
            }
        }
    }
}


// A warp takes h.blocks8 blocks, 8 apart (its neighbours have those between); the next one is on its way while one is computed.
// The chunk's scales are read and written as a whole: a store of 4 bytes per block made the kernel's memory traffic alone
// 206 instead of 144 us at 90M elements.  Measured at 90M bfloat16 parameters and gradients: 206 us, 4.4 TB/s, at 1965 MHz; after
// some 2,000 passes on end 222, when the power limit has brought the clock to 1815 MHz.  What bounds it is issue: 66 instructions per
// element, 8 of 10 slots, the integer pipe at 0.74.  The codes' exactness is 30 us of it: 175 with b1 and b2 folded into the
// scales and approximate roots alone.  At 30M, 74 us: with sqrt.rn for every element 78, with the careful branch at every four
// elements 77; where the positive roots of a block span more than 2^16 its lanes take that branch, 115.  Of the form with folded
// constants at 90M: three stages instead of two 175, the next block in registers instead of shared memory 237.
constexpr int STAGES8 = 2;
template <typename P, typename G, int CAP, bool STOCHASTIC>
__global__ void __launch_bounds__(THREADS, 4) k_adamw_8bit(const __grid_constant__ Table<CAP> T) {
    constexpr int WARPS = THREADS / 32, STEP = WARPS * QBLOCK;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float scales[2][WARPS * MAX_BLOCKS8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Staged<P, G>* ring = reinterpret_cast<Staged<P, G>*>(smem) + warp * STAGES8;
    const int k = tensor_of(T, blockIdx.x);
    const Entry& E = T.t[k];
    const int nb = T.h.blocks8, nscales = WARPS * nb, size = STEP * nb;
    const int64_t chunk = blockIdx.x - T.first[k], begin = chunk * size;
    const Chunk<P, G> C{static_cast<P*>(E.p) + begin, static_cast<const G*>(E.g) + begin, static_cast<uint8_t*>(E.m) + begin,
                        static_cast<uint8_t*>(E.v) + begin, E.copy ? static_cast<unsigned short*>(E.copy) + begin : nullptr,
                        E.n - begin < size ? (int32_t)(E.n - begin) : size};
    const uint32_t index = E.key ^ (uint32_t)begin ^ ((uint32_t)((uint64_t)begin >> 32) * 0x9E3779B9u);
    const int32_t vectors = E.head == 0 ? C.n / QBLOCK * QBLOCK : 0;    // blocks up to here are whole and aligned
    int32_t first = warp * QBLOCK;
#pragma unroll
    for (int s = 0; s < STAGES8 - 1; ++s) {
        if (s < nb && first + s * STEP < vectors) send(ring[s], C, first + s * STEP + lane * 8);
        copy_async_commit();
    }
    const int which = threadIdx.x >= THREADS / 2, mine = threadIdx.x % (THREADS / 2);     // one scale to a thread
    float* const scale = (which ? E.vs : E.ms) + chunk * nscales + mine;
    const bool has_scale = mine < nscales && mine * QBLOCK < C.n;
    if (has_scale) scales[which][mine] = *scale;
    const float gs = T.h.grad_scale ? *T.h.grad_scale : 1.f;
    const Hyper8 h{gs, T.h.b1, T.h.omb1, T.h.b2, T.h.omb2, T.h.keep, -T.h.step_size, T.h.inv_bc2, T.h.eps, T.h.one};
    __syncthreads();
    int stage = 0;
#pragma unroll 1
    for (int i = 0; i < nb && first < C.n; ++i, first += STEP) {
        float& ms = scales[0][i * WARPS + warp];
        float& vs = scales[1][i * WARPS + warp];
        const int32_t later = first + (STAGES8 - 1) * STEP;
        if (i + STAGES8 - 1 < nb && later < vectors) send(ring[stage == 0 ? STAGES8 - 1 : stage - 1], C, later + lane * 8);
        copy_async_commit();
        copy_async_wait<STAGES8 - 1>();
        if (first < vectors) block8<P, G, STOCHASTIC, true>(h, index, C, first, taken(ring[stage]), T.h.copy_f16, ms, vs);
        else block8<P, G, STOCHASTIC, false>(h, index, C, first, Block<P, G>{}, T.h.copy_f16, ms, vs);
        stage = stage == STAGES8 - 1 ? 0 : stage + 1;
    }
    copy_async_wait<0>();
    __syncthreads();
    if (has_scale) *scale = scales[which][mine];
}

// ---- host side ---------------------------------------------------------------------------------------

// Elements to skip until p, g, m, v (and the copy) all lie on the boundary of a vector of `vec` elements; -1: never.
int head_of(const ssgd_adamw_tensor& t, int pb, int gb, int sb, int vec, bool scalable) {
    for (int h = 0; h < (scalable ? vec : 1); ++h) {
        auto ok = [&](const void* q, int bytes) {
            const int unit = vec * bytes > 16 ? 16 : vec * bytes;
            return !q || (addr(q) + (uint64_t)h * bytes) % (uint64_t)unit == 0;
        };
        if (ok(t.p, pb) && ok(t.g, gb) && ok(t.m, sb) && ok(t.v, sb) && ok(t.copy, 2)) return h;
    }
    return -1;
}

template <typename P, typename G, int CAP>
int launch_group(const ssgd_adamw_tensor* t, int32_t first, int32_t count, bool small, const Hyper& h, uint32_t key, bool stochastic,
                 cudaStream_t st) {
    Table<CAP> T;
    T.h = h;
    uint64_t chunks = 0;
    int32_t k = 0;
    for (int32_t i = first; i < first + count; ++i) {
        if (t[i].n == 0) continue;
        Entry& e = T.t[k];
        e.p = t[i].p; e.g = t[i].g; e.m = t[i].m; e.v = t[i].v; e.ms = t[i].m_scale; e.vs = t[i].v_scale; e.copy = t[i].copy;
        e.n = t[i].n;
        e.key = mix(key + (uint32_t)i);
        e.head = head_of(t[i], sizeof(P), sizeof(G), small ? 1 : 4, small ? 8 : 4, !small);
        T.first[k++] = (uint32_t)chunks;
        const int64_t chunk = small ? (int64_t)(THREADS / 32) * QBLOCK * h.blocks8 : CHUNK32;
        // the last chunk of a tensor takes what the head has pushed out of the others
        const int64_t body = e.head > 0 ? (e.n > e.head ? e.n - e.head : 1) : e.n;
        chunks += (uint64_t)((body + chunk - 1) / chunk);
    }
    if (k == 0) return SSGD_OK;
    if (chunks > 0x7fffffffull) return SSGD_EINVAL;
    T.first[k] = (uint32_t)chunks;
    T.count = k;
    if (small) {
        auto kernel = stochastic ? k_adamw_8bit<P, G, CAP, true> : k_adamw_8bit<P, G, CAP, false>;
        constexpr int smem = (int)sizeof(Staged<P, G>) * (THREADS / 32) * STAGES8;
        static_assert(smem <= 40 * 1024, "a launch needs no permission for so much shared memory beside the scales");
        kernel<<<(unsigned)chunks, THREADS, smem, st>>>(T);
    } else {
        auto kernel = k_adamw_f32<P, G, CAP, false>;
        if constexpr (sizeof(P) == 2) if (stochastic) kernel = k_adamw_f32<P, G, CAP, true>;
        kernel<<<(unsigned)chunks, THREADS, 0, st>>>(T);
    }
    return launched();
}

template <typename P, typename G>
int launch_all(const ssgd_adamw_tensor* t, int32_t count, bool small, const Hyper& h, uint32_t key, bool stochastic, cudaStream_t st) {
    if (count <= FEW_TENSORS) return launch_group<P, G, FEW_TENSORS>(t, 0, count, small, h, key, stochastic, st);
    for (int32_t i = 0; i < count; i += MAX_TENSORS) {
        const int32_t c = count - i < MAX_TENSORS ? count - i : MAX_TENSORS;
        const int e = launch_group<P, G, MAX_TENSORS>(t, i, c, small, h, key, stochastic, st);
        if (e) return e;
    }
    return SSGD_OK;
}

static_assert(sizeof(Table<FEW_TENSORS>) <= 4096, "kernel arguments");
static_assert(sizeof(Table<MAX_TENSORS>) <= 32764, "kernel arguments");

}  // namespace

extern "C" int ssgd_adamw_step(const ssgd_adamw_tensor* tensors, int32_t count, int32_t fmt_p, int32_t fmt_g, int32_t fmt_state,
                               int32_t fmt_copy, double lr, double beta1, double beta2, double eps, double weight_decay,
                               int64_t step, const float* grad_scale, int32_t stochastic, uint64_t seed, void* stream) {
    if (count < 0 || (count && !tensors) || step < 1) return SSGD_EINVAL;
    if (!(lr >= 0 && std::isfinite(lr)) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) ||
        !(eps >= 0 && std::isfinite(eps)) || !(weight_decay >= 0 && std::isfinite(weight_decay)))
        return SSGD_EINVAL;
    if (fmt_p != SSGD_FMT_F32 && fmt_p != SSGD_FMT_BF16) return SSGD_EINVAL;
    if (!fmt_bytes(fmt_g) || (fmt_state != SSGD_FMT_F32 && fmt_state != SSGD_FMT_E4M3)) return SSGD_EINVAL;
    if (fmt_copy != SSGD_FMT_BF16 && fmt_copy != SSGD_FMT_F16) return SSGD_EINVAL;
    if (!aligned_to(grad_scale, 4)) return SSGD_EALIGN;
    const int pb = fmt_bytes(fmt_p), gb = fmt_bytes(fmt_g);
    const bool small = fmt_state == SSGD_FMT_E4M3;
    for (int32_t i = 0; i < count; ++i) {
        const ssgd_adamw_tensor& t = tensors[i];
        if (t.n < 0) return SSGD_EINVAL;
        if (t.n == 0) continue;
        if (!t.p || !t.g || !t.m || !t.v || (small && (!t.m_scale || !t.v_scale))) return SSGD_EINVAL;
        if (t.copy && fmt_p != SSGD_FMT_F32) return SSGD_EINVAL;
        if (!aligned_to(t.p, pb) || !aligned_to(t.g, gb) || (!small && (!aligned_to(t.m, 4) || !aligned_to(t.v, 4))) ||
            (small && (!aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4))) || !aligned_to(t.copy, 2))
            return SSGD_EALIGN;
    }
    Hyper h;
    h.b1 = (float)beta1;
    h.omb1 = (float)(1.0 - beta1);
    h.b2 = (float)beta2;
    h.omb2 = (float)(1.0 - beta2);
    h.keep = (float)(1.0 - lr * weight_decay);
    h.step_size = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    h.inv_bc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    h.eps = (float)eps;
    h.one = 1.f;
    h.grad_scale = grad_scale;
    h.copy_f16 = fmt_copy == SSGD_FMT_F16;
    h.blocks8 = 1;
    int64_t blocks = 0;
    for (int32_t i = 0; i < count; ++i) blocks += (tensors[i].n + QBLOCK - 1) / QBLOCK;
    if (blocks == 0) return SSGD_OK;
    if (small) {
        // As many blocks to a warp as leave 4 CTAs to an SM: one after the other they take a microsecond each, but share a CTA's
        // start and end.  8 blocks / 1 block: 79,247 elements in 22 tensors 12.4 / 5.1 us; 8 / 4 blocks: 90M 175 / 182.
        int sms = 0;
        const int e = sm_count_of_current_device(&sms);
        if (e) return e;
        while (h.blocks8 < MAX_BLOCKS8 && blocks >= (int64_t)h.blocks8 * 2 * (THREADS / 32) * 4 * sms) h.blocks8 *= 2;
    }
    const uint32_t key = mix(mix((uint32_t)seed) ^ (uint32_t)(seed >> 32));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool sr = stochastic != 0;
    if (fmt_p == SSGD_FMT_F32) {
        if (fmt_g == SSGD_FMT_F32) return launch_all<float, float>(tensors, count, small, h, key, sr, st);
        if (fmt_g == SSGD_FMT_F16) return launch_all<float, __half>(tensors, count, small, h, key, sr, st);
        return launch_all<float, __nv_bfloat16>(tensors, count, small, h, key, sr, st);
    }
    if (fmt_g == SSGD_FMT_F32) return launch_all<__nv_bfloat16, float>(tensors, count, small, h, key, sr, st);
    if (fmt_g == SSGD_FMT_F16) return launch_all<__nv_bfloat16, __half>(tensors, count, small, h, key, sr, st);
    return launch_all<__nv_bfloat16, __nv_bfloat16>(tensors, count, small, h, key, sr, st);
}
