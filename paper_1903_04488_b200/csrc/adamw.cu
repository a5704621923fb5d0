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
// touch its neighbours' scale.
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
constexpr int CHUNK8 = (THREADS / 32) * QBLOCK;   // a warp takes one block of 256

struct Entry {
    void* p; const void* g; void* m; void* v; float* ms; float* vs; void* copy;
    int64_t n;
    uint32_t key;        // dither key of the tensor
    int32_t head;        // elements before the first aligned vector; -1: no common alignment
};
struct Hyper {
    float b1, omb1, b2, omb2, keep, step_size, inv_bc2, eps;
    const float* grad_scale;
    int32_t copy_f16;    // the copy is binary16, else bfloat16
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

__device__ __forceinline__ float e4m3_value(uint32_t code) {
    __half_raw r = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3);
    return __half2float(__half(r));
}

// y = magnitude / scale in [0, 448], rounded down after u in [0, 1) units of its last place is added.  With
// e = max(exponent, -6) a unit is 2^(e - 3); n = floor(y / unit + u) in 0..16 and 8 (e + 6) + n is the code, whose carry
// into the exponent comes out by itself.  (A y above 448 by a rounding error stays at the largest code.)
__device__ __forceinline__ uint32_t e4m3_code(float y, float u) {
    const uint32_t e = max(__float_as_uint(y) & 0x7f800000u, 121u << 23);
    const float per_unit = __uint_as_float((257u << 23) - e);          // 1 / unit
    const uint32_t n = __float_as_uint(__fadd_rd(fmaf(y, per_unit, u), 8388608.f)) & 31u;
    return min((e >> 20) - 968u + n, 126u);
}

__device__ __forceinline__ float finite_magnitude(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }

// A warp owns one block of 256 elements: lane l the elements 8 l .. 8 l + 7 when everything is aligned for it (VEC),
// otherwise the elements l, l + 32, ...  The codes and scales are the same either way.
template <typename P, typename G, int CAP, bool VECTOR>
__device__ __forceinline__ void block8(const Table<CAP>& T, const Entry& E, int64_t block, bool stochastic) {
    const Hyper& h = T.h;
    const int lane = threadIdx.x & 31;
    const int64_t base = block * QBLOCK, n = E.n;
    P* p = static_cast<P*>(E.p) + base;
    const G* g = static_cast<const G*>(E.g) + base;
    uint8_t* mc = static_cast<uint8_t*>(E.m) + base;
    uint8_t* vc = static_cast<uint8_t*>(E.v) + base;
    const int left = n - base < QBLOCK ? (int)(n - base) : QBLOCK;
    auto at = [&](int j) { return VECTOR ? lane * 8 + j : lane + 32 * j; };
    float fp[8], fg[8], fm[8], fr[8];
    const float gs = h.grad_scale ? *h.grad_scale : 1.f, ms = E.ms[block], vs = E.vs[block];
    if (VECTOR && left == QBLOCK) {
        union { uint2 r; uint8_t c[8]; } cm, cv;
        cm.r = *reinterpret_cast<const uint2*>(mc + lane * 8);
        cv.r = *reinterpret_cast<const uint2*>(vc + lane * 8);
        if constexpr (sizeof(P) == 2) {
            unpack(load_vec<P, 8>(p + lane * 8), fp);
        } else {
            const Vec<P, 4> a = load_vec<P, 4>(p + lane * 8), b = load_vec<P, 4>(p + lane * 8 + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { fp[j] = a.e[j]; fp[4 + j] = b.e[j]; }
        }
        if constexpr (sizeof(G) == 2) {
            unpack(load_vec_stream<G, 8>(g + lane * 8), fg);
        } else {
            const Vec<G, 4> a = load_vec_stream<G, 4>(g + lane * 8), b = load_vec_stream<G, 4>(g + lane * 8 + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { fg[j] = a.e[j]; fg[4 + j] = b.e[j]; }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) { fm[j] = e4m3_value(cm.c[j]); fr[j] = e4m3_value(cv.c[j]); }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = at(j);
            const bool in = i < left;
            fp[j] = in ? to_f32(p[i]) : 0.f;
            fg[j] = in ? to_f32(g[i]) : 0.f;
            fm[j] = in ? e4m3_value(mc[i]) : 0.f;
            fr[j] = in ? e4m3_value(vc[i]) : 0.f;
        }
    }
    float am = 0.f, ar = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float gj = fg[j] * gs, r0 = fr[j] * vs;
        const float m = fmaf(fm[j] * ms, h.b1, gj * h.omb1);
        const float v = fmaf(r0 * r0, h.b2, gj * gj * h.omb2);
        const float r = sqrtf(v);
        fp[j] = fmaf(fp[j], h.keep, -h.step_size * (m / fmaf(r, h.inv_bc2, h.eps)));
        fm[j] = m;
        fr[j] = r;
        am = fmaxf(am, finite_magnitude(m));
        ar = fmaxf(ar, finite_magnitude(r));
    }
    // magnitudes order like their bit patterns
    am = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(am)));
    ar = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(ar)));
    const float least = 0x1p-100f;                         // below it 448 / x overflows: the block is held as zeros
    const float im = am < least ? 0.f : 448.f / am, ir = ar < least ? 0.f : 448.f / ar;
    if (lane == 0) {
        E.ms[block] = am < least ? 0.f : am / 448.f;
        E.vs[block] = ar < least ? 0.f : ar / 448.f;
    }
    uint32_t code_m[8], code_v[8], word[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        word[j] = stochastic ? dither_word(E.key, base + at(j)) : 0u;
        // 16 bits of dither each, in the middle of their interval; without a seed 1/2: to nearest
        const float um = stochastic ? __uint_as_float(((word[j] << 7) & 0x007fff80u) | 0x3f800040u) - 1.f : 0.5f;
        const float uv = stochastic ? __uint_as_float(((word[j] >> 9) & 0x007fff80u) | 0x3f800040u) - 1.f : 0.5f;
        const uint32_t sign = (__float_as_uint(fm[j]) >> 24) & 0x80u;
        code_m[j] = e4m3_code(fabsf(fm[j]) * im, um);
        if (fm[j] < 0.f) code_m[j] |= sign;
        code_v[j] = e4m3_code(fr[j] * ir, uv);
        if (fr[j] > 0.f) code_v[j] = max(code_v[j], 1u);
        if (!(fabsf(fm[j]) < INFINITY)) code_m[j] = 0x7fu;
        if (!(fabsf(fr[j]) < INFINITY)) code_v[j] = 0x7fu;
    }
    if (VECTOR && left == QBLOCK) {
        union { uint2 r; uint8_t c[8]; } cm, cv;
#pragma unroll
        for (int j = 0; j < 8; ++j) { cm.c[j] = (uint8_t)code_m[j]; cv.c[j] = (uint8_t)code_v[j]; }
        *reinterpret_cast<uint2*>(mc + lane * 8) = cm.r;
        *reinterpret_cast<uint2*>(vc + lane * 8) = cv.r;
        if constexpr (sizeof(P) == 2) {
            Vec<P, 8> o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o.e[j] = round_param<P>(fp[j], stochastic, word[j]);
            store_vec<P, 8>(p + lane * 8, o);
        } else {
            Vec<P, 4> a, b;
#pragma unroll
            for (int j = 0; j < 4; ++j) { a.e[j] = fp[j]; b.e[j] = fp[4 + j]; }
            store_vec<P, 4>(p + lane * 8, a);
            store_vec<P, 4>(p + lane * 8 + 4, b);
        }
        if (E.copy) {
            Vec<unsigned short, 8> c;
#pragma unroll
            for (int j = 0; j < 8; ++j) c.e[j] = round_copy(fp[j], h.copy_f16);
            store_vec<unsigned short, 8>(static_cast<unsigned short*>(E.copy) + base + lane * 8, c);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = at(j);
            if (i < left) {
                mc[i] = (uint8_t)code_m[j];
                vc[i] = (uint8_t)code_v[j];
                p[i] = round_param<P>(fp[j], stochastic, word[j]);
                if (E.copy) static_cast<unsigned short*>(E.copy)[base + i] = round_copy(fp[j], h.copy_f16);
            }
        }
    }
}

template <typename P, typename G, int CAP, bool STOCHASTIC>
__global__ void __launch_bounds__(THREADS) k_adamw_8bit(const __grid_constant__ Table<CAP> T) {
    const int k = tensor_of(T, blockIdx.x);
    const Entry& E = T.t[k];
    const int64_t block = (int64_t)(blockIdx.x - T.first[k]) * (THREADS / 32) + (threadIdx.x >> 5);
    if (block * QBLOCK >= E.n) return;
    if (E.head == 0) block8<P, G, CAP, true>(T, E, block, STOCHASTIC);
    else block8<P, G, CAP, false>(T, E, block, STOCHASTIC);
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
        const int64_t chunk = small ? CHUNK8 : CHUNK32;
        // the last chunk of a tensor takes what the head has pushed out of the others
        const int64_t body = e.head > 0 ? (e.n > e.head ? e.n - e.head : 1) : e.n;
        chunks += (uint64_t)((body + chunk - 1) / chunk);
    }
    if (k == 0) return SSGD_OK;
    if (chunks > 0x7fffffffull) return SSGD_EINVAL;
    T.first[k] = (uint32_t)chunks;
    T.count = k;
    if (small) {
        if (stochastic) k_adamw_8bit<P, G, CAP, true><<<(unsigned)chunks, THREADS, 0, st>>>(T);
        else k_adamw_8bit<P, G, CAP, false><<<(unsigned)chunks, THREADS, 0, st>>>(T);
    } else {
        if (stochastic && sizeof(P) == 2) k_adamw_f32<P, G, CAP, true><<<(unsigned)chunks, THREADS, 0, st>>>(T);
        else k_adamw_f32<P, G, CAP, false><<<(unsigned)chunks, THREADS, 0, st>>>(T);
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
    h.grad_scale = grad_scale;
    h.copy_f16 = fmt_copy == SSGD_FMT_F16;
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
