// token_logprobs.cu -- log probabilities of given tokens with entropy and the best alternatives, and their gradient
// (ssgd_token_logprobs, ssgd_token_logprobs_backward).
//
// A row of V logits, z = scale * logits:
//   m = max z,  s = sum e^(z - m),  lse = m + log s,  logp = z[id] - lse,  H = log s - (sum e^(z - m) (z - m)) / s
// One pass: every thread keeps a running maximum and the two sums relative to it, and rescales them when the maximum
// rises.  A row is cut into granules of 16 aligned bytes (its first and last may be partial, so any base and stride will
// do); granule i of a segment belongs to thread i mod THREADS.
//
// Alternatives: the k-th largest of the threads' maxima bounds the k-th largest logit from below, so only threads whose
// maximum reaches it can hold one of the k.  Their granules -- k threads' worth when logits are distinct -- are read
// again (from L2) and fed into a sorted list per warp.  Order: larger logit first, then smaller index; a NaN counts as
// the largest; -0 and +0 are equal.
//
// Few rows: a cluster of CTAs shares a row and joins through distributed shared memory, so there is still one launch
// and no scratch.
//
// Gradient, p_j = e^(z_j - lse), A = d_logp + sum of d_top:
//   dlogits_j = scale * (d_logp [j = id] + sum_m d_top_m [j = top_m] - p_j (A + d_entropy (z_j - lse + H)))
// One read and one write per logit; the few columns with an extra term are written a second time by the CTA that owns
// them, after a barrier.
#include <cooperative_groups.h>

#include "formats.cuh"

using namespace ssgd;
namespace cg = cooperative_groups;

namespace {

constexpr int THREADS = 256;
constexpr int WARPS = THREADS / 32;
constexpr int MAX_TOP = SSGD_MAX_TOP;       // one entry per lane of a warp
static_assert(MAX_TOP == 32, "a warp's list has an entry per lane");
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NEG_INF = -INFINITY;

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

// Largest magnitude of a format for which the fast path below is taken, with room for the floor.
template <typename T> __device__ __forceinline__ float fast_limit() { return 1e37f; }
template <> __device__ __forceinline__ float fast_limit<__half>() { return 6e4f; }

// The running sums of one thread, relative to its maximum logit m, in powers of two: with d = (z - m) c, c = scale * log2 e,
// s = sum 2^d and w = sum 2^d d.  The difference comes first: z c alone overflows at the lowest values that masks use.
struct Sums {
    float m, s, w;
};

__device__ __forceinline__ void rebase(Sums& a, float m, float c) {
    if (a.m > NEG_INF || a.m != a.m) {
        const float delta = (a.m - m) * c, f = ex2(delta);
        a.w = f * fmaf(delta, a.s, a.w);
        if (f == 0.f && a.s == a.s && a.w != a.w) a.w = 0.f;   // 0 * -inf: the old part has vanished
        a.s *= f;
    }
    a.m = m;
}

// Any values: infinities, NaN, magnitudes near the end of the format.
__device__ __forceinline__ void add_careful(Sums& a, float z, float c) {
    const float m = max_nan(a.m, z);
    if (!(m == a.m)) rebase(a, m, c);
    if (z == NEG_INF && a.m == a.m) return;                // contributes nothing, whatever the maximum
    const float d = (z - a.m) * c, e = ex2(d);
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

// Sort keys: larger key = earlier.  Upper half the logit's order, lower half the index inverted; 0 = no entry.
__device__ __forceinline__ uint32_t order_of(float z) {
    if (z != z) return 0xffffffffu;
    const uint32_t b = __float_as_uint(z + 0.0f);          // -0 becomes +0
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;       // never 0: that would be a NaN's pattern
}
__device__ __forceinline__ float logit_of(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    if (o == 0xffffffffu) return NAN;
    return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

struct LogprobArgs {
    const void* logits; int64_t ld;
    const void* ids; bool ids64;
    int64_t rows; int32_t vocab;
    float scale;
    int32_t top;
    float* stats;          // [3][rows]: logp, entropy, lse
    int32_t* top_idx; float* top_logp;   // [rows][top]
};

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

// A value no larger than m - 160 / c and below every element that could matter: elements under it are raised to it, so
// that -inf does not make 0 * -inf.  2^-160 is zero in fp32.
template <typename T> __device__ __forceinline__ float floor_for(float m, float c) { return __fsub_rd(m, __fdiv_ru(160.f, c)); }
template <> __device__ __forceinline__ float floor_for<__nv_bfloat16>(float m, float c) {
    return __bfloat162float(__float2bfloat16_rd(__fsub_rd(m, __fdiv_ru(160.f, c))));
}
template <> __device__ __forceinline__ float floor_for<__half>(float m, float c) {
    return __half2float(__float2half_rd(__fsub_rd(m, __fdiv_ru(160.f, c))));
}

// Elements that are not there are -inf: they change neither the maximum nor the sums.  `have` <= U is the same for the
// whole CTA.
template <typename T, int U>
__device__ __forceinline__ void add_granules(Sums& a, float& low, const Vec<T, 16 / sizeof(T)> (&v)[U], int have, float c) {
    constexpr int VEC = 16 / sizeof(T);
    PairMax<T> top(a.m);
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < have) top.add(v[u]);
    const float m = top.value();
    if (!(m == a.m)) {
        rebase(a, m, c);
        low = fabsf(m) < fast_limit<T>() ? floor_for<T>(m, c) : NEG_INF;
    }
    if (low > NEG_INF) {
        const float2 minus_m = both(-a.m), c2 = both(c);
        float2 s = both(0.f), w = both(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u < have) {
                float2 f[VEC / 2];
                unpack_pairs(raised(v[u], low), f);
#pragma unroll
                for (int e = 0; e < VEC / 2; ++e) {
                    const float2 d = mul2(add2(f[e], minus_m), c2), x = make_float2(ex2(d.x), ex2(d.y));
                    s = add2(s, x);
                    w = fma2(x, d, w);
                }
            }
        }
        a.s += s.x + s.y;
        a.w += w.x + w.y;
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < have)
#pragma unroll
                for (int e = 0; e < VEC; ++e) add_careful(a, to_f32(v[u].e[e]), c);
    }
}

// Inserts `key` into the warp's list, lane l holding the l-th largest.
__device__ __forceinline__ void insert(uint64_t& mine, uint64_t key) {
    const uint32_t above = __ballot_sync(0xffffffffu, mine > key);
    const int at = __popc(above), lane = threadIdx.x & 31;
    const uint64_t up = __shfl_up_sync(0xffffffffu, mine, 1);
    if (lane == at) mine = key;
    else if (lane > at) mine = up;
}

// The 32 largest of two lists (lane l of each holding its l-th largest), in order: the larger of a's l-th and b's
// (31 - l)-th are the 32 largest as a bitonic sequence, which five exchanges sort.
__device__ __forceinline__ uint64_t merge(uint64_t a, uint64_t b) {
    const int lane = threadIdx.x & 31;
    const uint64_t r = __shfl_xor_sync(0xffffffffu, b, 31);
    a = a > r ? a : r;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const uint64_t other = __shfl_xor_sync(0xffffffffu, a, o);
        a = ((lane & o) == 0) == (a > other) ? a : other;
    }
    return a;
}
// Lane l gets the l-th largest of the warp's values.
__device__ __forceinline__ uint32_t sort32(uint32_t x) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1) {
#pragma unroll
        for (int o = k >> 1; o > 0; o >>= 1) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, x, o);
            const bool keep_larger = ((lane & o) == 0) == ((lane & k) == 0);
            x = keep_larger ? max(x, other) : min(x, other);
        }
    }
    return x;
}

struct Shared {
    Sums part[WARPS];                 // part[0] is the CTA's in the end
    uint64_t list[WARPS][MAX_TOP];    // list[0] is the CTA's in the end
    uint32_t bound[WARPS];
    int32_t picked[THREADS];
    int32_t npicked;
};

// The CTA's best of its segment [g0, g1) into sh.list[0], in order, at least k of them (0 where there are fewer).
template <typename T>
__device__ void best_of_segment(Shared& sh, const Granules<T>& G, int32_t g0, int32_t g1, float thread_max, bool has, int k) {
    constexpr int VEC = 16 / sizeof(T);
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const uint32_t mine = has ? order_of(thread_max) : 0u;
    // Each warp has ceil(k / WARPS) threads whose maximum reaches its bound, so k logits reach the least of the bounds.
    const uint32_t sorted = sort32(mine);
    if (lane == (k + WARPS - 1) / WARPS - 1) sh.bound[warp] = sorted;
    if (t == 0) sh.npicked = 0;
    __syncthreads();
    uint32_t bound = sh.bound[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i) bound = min(bound, sh.bound[i]);
    if (has && mine >= bound) sh.picked[atomicAdd(&sh.npicked, 1)] = t;
    __syncthreads();
    uint64_t list = 0, last = 0;                           // lane's entry of the warp's list; the k-th entry
    const int np = sh.npicked;
    for (int q = warp; q < np; q += WARPS) {
        const int owner = sh.picked[q];
        for (int32_t base = g0 + owner; base < g1; base += 32 * THREADS) {
            const int32_t i = base + lane * THREADS;
            const int32_t at = G.first(i);
            uint32_t order[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) order[e] = 0;
            if (i < g1) {
                if (G.whole(i)) {
                    const Vec<T, VEC> v = load_vec<T, VEC>(G.row + at);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) order[e] = order_of(to_f32(v.e[e]));
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (at + e >= 0 && at + e < G.n) order[e] = order_of(to_f32(G.row[at + e]));
                }
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                uint32_t todo = __ballot_sync(0xffffffffu, order[e] >= bound && order[e] >= (uint32_t)(last >> 32) && order[e] != 0);
                while (todo) {
                    const int src = __ffs(todo) - 1;
                    todo &= todo - 1;
                    const uint64_t key = ((uint64_t)__shfl_sync(0xffffffffu, order[e], src) << 32) |
                                         (0xffffffffu - (uint32_t)__shfl_sync(0xffffffffu, at + e, src));
                    if (key > last) {
                        insert(list, key);
                        last = __shfl_sync(0xffffffffu, list, k - 1);
                    }
                }
            }
        }
    }
    sh.list[warp][lane] = list;
#pragma unroll
    for (int half = WARPS / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (warp < half) {
            list = merge(list, sh.list[warp + half][lane]);
            sh.list[warp][lane] = list;
        }
    }
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(THREADS) k_token_logprobs(const LogprobArgs A, int split) {
    constexpr int VEC = 16 / sizeof(T), U = 4;
    __shared__ Shared sh;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    // split is a power of two
    const int shift = __ffs(split) - 1, part = blockIdx.x & (split - 1);
    const int64_t row = blockIdx.x >> shift;
    const T* z = static_cast<const T*>(A.logits) + row * A.ld;
    const Granules<T> G(z, A.vocab);
    const int32_t per = (G.count + split - 1) >> shift;
    const int32_t g0 = min(part * per, G.count), g1 = min(g0 + per, G.count);
    const float c = A.scale * LOG2E;
    int64_t id = -1;
    if (part == 0 && t == 0) id = id_of(A.ids, A.ids64, row);
    Sums a{NEG_INF, 0.f, 0.f};
    float low = NEG_INF;
    const int32_t whole0 = G.phase ? 1 : 0, whole1 = G.whole(G.count - 1) ? G.count : G.count - 1;
    for (int32_t b0 = g0; b0 < g1; b0 += THREADS * U) {
        Vec<T, VEC> v[U];
        if (b0 >= whole0 && b0 + THREADS * U <= min(whole1, g1)) {
            const T* p = z + G.first(b0 + t);
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load_vec_stream<T, VEC>(p + u * (THREADS * VEC));
            add_granules<T, U>(a, low, v, U, c);
            continue;
        }
        const int have = (g1 - b0 + THREADS - 1) / THREADS;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t i = b0 + u * THREADS + t, at = G.first(i);
            if (i >= whole0 && i < min(whole1, g1)) {
                v[u] = load_vec_stream<T, VEC>(z + at);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[u].e[e] = from_f32<T>(NEG_INF);
                    if (i < g1 && at + e >= 0 && at + e < A.vocab) v[u].e[e] = z[at + e];
                }
            }
        }
        add_granules<T, U>(a, low, v, have, c);
    }
    const bool has = g0 + t < g1;
    const float thread_max = a.m;
    const bool counted = id >= 0 && id < A.vocab;          // an id outside the vocabulary is ignored
    float z_id = 0.f;
    if (counted) z_id = to_f32(z[id]);
    // join: warp, CTA, cluster
    join_warp(a, c);
    if (lane == 0) sh.part[warp] = a;
    if (TOP) best_of_segment<T>(sh, G, g0, g1, thread_max, has, A.top);
    __syncthreads();
    if (warp == 0) {
        a = lane < WARPS ? sh.part[lane] : Sums{NEG_INF, 0.f, 0.f};
        join_warp(a, c);
        __syncwarp();
        if (lane == 0) sh.part[0] = a;
    }
    cg::cluster_group cluster = cg::this_cluster();
    if (split > 1) cluster.sync();
    if (part == 0 && warp == 0) {
        if (split > 1) {
            a = lane < split ? *cluster.map_shared_rank(&sh.part[0], lane < split ? lane : 0) : Sums{NEG_INF, 0.f, 0.f};
            join_warp(a, c);
        }
        const float log2s = log2f(a.s);
        const bool none = a.s == 0.f;                      // every logit is -inf
        auto logp_of = [&](float x) {
            return none || (x == NEG_INF && a.s == a.s) ? NEG_INF : fmaf(x - a.m, A.scale, -log2s * LN2);
        };
        if (lane == 0) {
            A.stats[row] = counted ? logp_of(z_id) : 0.f;
            A.stats[A.rows + row] = none ? 0.f : (log2s - a.w / a.s) * LN2;
            A.stats[2 * A.rows + row] = none ? NEG_INF : fmaf(a.m, A.scale, log2s * LN2);
        }
        if (TOP) {
            uint64_t list = sh.list[0][lane];
            for (int i = 1; i < split; ++i) list = merge(list, cluster.map_shared_rank(&sh.list[0][0], i)[lane]);
            if (lane < A.top) {
                A.top_idx[row * A.top + lane] = (int32_t)(0xffffffffu - (uint32_t)list);
                A.top_logp[row * A.top + lane] = logp_of(logit_of(list));
            }
        }
    }
    if (split > 1) cluster.sync();                         // nobody leaves while its shared memory is read
}

// ---- backward ----------------------------------------------------------------------------------------

struct LogprobBackArgs {
    const void* logits; int64_t ld;
    const void* ids; bool ids64;
    int64_t rows; int32_t vocab;
    int32_t per;           // granules per CTA, a multiple of THREADS
    float scale;
    const float* lse; const float* entropy;
    const float* d_logp; const float* d_entropy;      // either may be NULL
    int32_t top; const int32_t* top_idx; const float* d_top;
    void* out; int64_t ld_out;
    bool same_phase;       // rows of logits and of the result lie alike within 16 bytes
};

constexpr int BACK_U = 4;

// CTA (row, part) writes `per` granules of a row.
template <typename T, bool ENTROPY>
__global__ void __launch_bounds__(THREADS) k_token_logprobs_back(const LogprobBackArgs A) {
    constexpr int VEC = 16 / sizeof(T);
    __shared__ int32_t special[MAX_TOP + 1];
    __shared__ float extra[MAX_TOP + 1];
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(A.logits) + row * A.ld;
    T* out = static_cast<T*>(A.out) + row * A.ld_out;
    const Granules<T> G(z, A.vocab);
    const int32_t g0 = (int32_t)blockIdx.y * A.per, g1 = min(g0 + A.per, G.count);
    if (g0 >= g1) return;                                 // the last part, where the phase needs no further granule
    // the row's constants
    const int64_t id = A.ids ? id_of(A.ids, A.ids64, row) : -1;
    const bool counted = id >= 0 && id < A.vocab;
    const float g_logp = counted && A.d_logp ? A.d_logp[row] : 0.f;
    float sum = g_logp;
    for (int i = 0; i < A.top; ++i) sum += A.d_top[row * A.top + i];
    const float g_h = ENTROPY ? A.d_entropy[row] : 0.f;
    const float lse = A.lse[row];
    const float minus_lse = lse == NEG_INF ? NEG_INF : -lse;   // of an empty row: p = 0 everywhere
    const float h = ENTROPY ? A.entropy[row] : 0.f;
    const float scale = A.scale;
    const float base = -scale * fmaf(g_h, h, sum), slope = -scale * g_h;
    // gradient of two logits without the columns' own terms: p (base + slope log p)
    auto grad = [&](float2 x) {
        float2 logp = fma2(x, both(scale), both(minus_lse));
        const float2 t = mul2(logp, both(LOG2E)), p = make_float2(ex2(t.x), ex2(t.y));
        if (!ENTROPY) return mul2(p, both(base));
        logp = make_float2(fmaxf(logp.x, -200.f), fmaxf(logp.y, -200.f));
        return mul2(p, fma2(logp, both(slope), both(base)));
    };
    auto one = [&](float x) { return from_f32<T>(grad(both(x)).x); };
    // the columns with a term of their own that this CTA writes
    const int nspecial = A.top + (counted ? 1 : 0);
    int32_t col = -1;
    if (t < nspecial) {
        col = t < A.top ? A.top_idx[row * A.top + t] : (int32_t)id;
        special[t] = col;
        extra[t] = t < A.top ? A.d_top[row * A.top + t] : g_logp;
    }
    const int32_t lo = max(G.first(g0), 0), hi = min(G.first(g1), A.vocab);
    const bool fix = t < nspecial && col >= lo && col < hi;
    float z_fix = 0.f;
    if (fix) z_fix = to_f32(z[col]);                      // before the result, which may lie in the same place, is written
    __syncthreads();
    if (A.same_phase) {
        const int32_t whole0 = G.phase ? 1 : 0, whole1 = min(G.whole(G.count - 1) ? G.count : G.count - 1, g1);
        for (int32_t b0 = g0; b0 < g1; b0 += THREADS * BACK_U) {
            const int32_t at = G.first(b0 + t);
            Vec<T, VEC> v[BACK_U];
            float2 f[VEC / 2];
            if (b0 >= whole0 && b0 + THREADS * BACK_U <= whole1) {
#pragma unroll
                for (int u = 0; u < BACK_U; ++u) v[u] = load_vec_stream<T, VEC>(z + at + u * (THREADS * VEC));
#pragma unroll
                for (int u = 0; u < BACK_U; ++u) {
                    unpack_pairs(v[u], f);
#pragma unroll
                    for (int e = 0; e < VEC / 2; ++e) f[e] = grad(f[e]);
                    store_vec<T, VEC>(out + at + u * (THREADS * VEC), pack_pairs<T, VEC>(f));
                }
                continue;
            }
#pragma unroll
            for (int u = 0; u < BACK_U; ++u) {
                const int32_t i = b0 + u * THREADS + t;
                if (i >= whole0 && i < whole1) v[u] = load_vec_stream<T, VEC>(z + G.first(i));
            }
#pragma unroll
            for (int u = 0; u < BACK_U; ++u) {
                const int32_t i = b0 + u * THREADS + t;
                if (i >= whole0 && i < whole1) {
                    unpack_pairs(v[u], f);
#pragma unroll
                    for (int e = 0; e < VEC / 2; ++e) f[e] = grad(f[e]);
                    store_vec<T, VEC>(out + G.first(i), pack_pairs<T, VEC>(f));
                } else if (i < g1) {
                    for (int32_t j = max(G.first(i), 0); j < min(G.first(i) + VEC, A.vocab); ++j) out[j] = one(to_f32(z[j]));
                }
            }
        }
    } else {
        for (int32_t j = lo + t; j < hi; j += THREADS) out[j] = one(to_f32(z[j]));
    }
    if (nspecial == 0) return;                            // the same for the whole CTA
    __syncthreads();
    if (fix) {
        float own = 0.f;
        for (int i = 0; i < nspecial; ++i)
            if (special[i] == col) own += extra[i];
        out[col] = from_f32<T>(fmaf(scale, own, grad(both(z_fix)).x));
    }
}

// ---- host side ---------------------------------------------------------------------------------------

// CTAs that share a row: enough of them for all SMs, while each still has two granules per thread.
int split_for(int64_t rows, int64_t vocab, int es, int sms) {
    const int64_t granules = vocab * es / 16;
    int split = 1;
    while (split < 8 && rows * split < 2 * sms && granules / (split * 2) >= 2 * THREADS) split *= 2;
    return split;
}

template <typename T>
int launch_logprobs(const LogprobArgs& A, int split, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(A.rows * split));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = split > 1 ? 1 : 0;
    const cudaError_t e = A.top ? cudaLaunchKernelEx(&cfg, k_token_logprobs<T, true>, A, split)
                                : cudaLaunchKernelEx(&cfg, k_token_logprobs<T, false>, A, split);
    return e == cudaSuccess ? SSGD_OK : SSGD_ECUDA;
}

template <typename T>
int launch_logprobs_back(LogprobBackArgs A, int sms, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T);
    const int64_t granules = (A.vocab + 2 * VEC - 2) / VEC;             // whatever the phase
    // Whole batches per CTA, 4 of them where that still makes 8 CTAs per SM: the row's constants cost a CTA as much as
    // a batch.
    int64_t batches = 4;
    while (batches > 1 && A.rows * ((granules + batches * THREADS * BACK_U - 1) / (batches * THREADS * BACK_U)) < 8 * sms) batches /= 2;
    A.per = (int32_t)(batches * THREADS * BACK_U);
    const int64_t parts = (granules + A.per - 1) / A.per;
    if (parts > 65535) return SSGD_EINVAL;
    const dim3 grid((unsigned)A.rows, (unsigned)parts);
    if (A.d_entropy) k_token_logprobs_back<T, true><<<grid, THREADS, 0, st>>>(A);
    else k_token_logprobs_back<T, false><<<grid, THREADS, 0, st>>>(A);
    return launched();
}

constexpr int64_t MAX_VOCAB = (int64_t)1 << 27;

int check_logits(const void* logits, int64_t ld, int32_t fmt, int64_t rows, int64_t vocab, float scale, int32_t top) {
    if (rows < 0 || rows > 0x0fffffff || vocab < 1 || vocab > MAX_VOCAB || ld < vocab) return SSGD_EINVAL;
    if (!fmt_bytes(fmt) || top < 0 || top > vocab) return SSGD_EINVAL;
    if (top > MAX_TOP) return SSGD_ETOOBIG;
    if (!(scale > 0.f) || !(scale < INFINITY)) return SSGD_EINVAL;
    if (rows && !logits) return SSGD_EINVAL;
    return aligned_to(logits, fmt_bytes(fmt)) ? SSGD_OK : SSGD_EALIGN;
}

}  // namespace

extern "C" {

int ssgd_token_logprobs(const void* logits, int64_t ld, int32_t fmt, const void* ids, int32_t ids_bytes, int64_t rows,
                        int64_t vocab, float scale, int32_t top, float* stats, int32_t* top_idx, float* top_logp,
                        void* stream) {
    int e = check_logits(logits, ld, fmt, rows, vocab, scale, top);
    if (e) return e;
    if (ids_bytes != 4 && ids_bytes != 8) return SSGD_EINVAL;
    if (rows == 0) return SSGD_OK;
    if (!ids || !stats || (top && (!top_idx || !top_logp))) return SSGD_EINVAL;
    if (!aligned_to(ids, ids_bytes) || !aligned_to(stats, 4) || !aligned_to(top_idx, 4) || !aligned_to(top_logp, 4))
        return SSGD_EALIGN;
    int sms = 0;
    if ((e = sm_count_of_current_device(&sms))) return e;
    const LogprobArgs A{logits, ld, ids, ids_bytes == 8, rows, (int32_t)vocab, scale, top, stats, top_idx, top_logp};
    const int split = split_for(rows, vocab, fmt_bytes(fmt), sms);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return fmt == SSGD_FMT_F32 ? launch_logprobs<float>(A, split, st)
         : fmt == SSGD_FMT_F16 ? launch_logprobs<__half>(A, split, st) : launch_logprobs<__nv_bfloat16>(A, split, st);
}

int ssgd_token_logprobs_backward(const void* logits, int64_t ld, int32_t fmt, const void* ids, int32_t ids_bytes,
                                 int64_t rows, int64_t vocab, float scale, const float* lse, const float* entropy,
                                 const float* d_logp, const float* d_entropy, int32_t top, const int32_t* top_idx,
                                 const float* d_top, void* dlogits, int64_t ld_d, void* stream) {
    int e = check_logits(logits, ld, fmt, rows, vocab, scale, top);
    if (e) return e;
    if ((ids_bytes != 4 && ids_bytes != 8) || ld_d < vocab) return SSGD_EINVAL;
    if (rows == 0) return SSGD_OK;
    if (!lse || !dlogits || (d_logp && !ids) || (d_entropy && !entropy) || (top && (!top_idx || !d_top))) return SSGD_EINVAL;
    const int es = fmt_bytes(fmt);
    if (!aligned_to(ids, ids_bytes) || !aligned_to(dlogits, es) || !aligned_to(lse, 4) || !aligned_to(entropy, 4) ||
        !aligned_to(d_logp, 4) || !aligned_to(d_entropy, 4) || !aligned_to(top_idx, 4) || !aligned_to(d_top, 4))
        return SSGD_EALIGN;
    int sms = 0;
    if ((e = sm_count_of_current_device(&sms))) return e;
    LogprobBackArgs A{logits, ld, ids, ids_bytes == 8, rows, (int32_t)vocab, 0, scale, lse, entropy, d_logp, d_entropy,
                      top, top_idx, d_top, dlogits, ld_d, false};
    A.same_phase = addr(logits) % 16 == addr(dlogits) % 16 && (rows == 1 || (ld - ld_d) * es % 16 == 0);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return fmt == SSGD_FMT_F32 ? launch_logprobs_back<float>(A, sms, st)
         : fmt == SSGD_FMT_F16 ? launch_logprobs_back<__half>(A, sms, st) : launch_logprobs_back<__nv_bfloat16>(A, sms, st);
}

}  // extern "C"
