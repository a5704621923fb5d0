// token_logprobs.cu -- log probabilities of given tokens with entropy and the best alternatives, and their gradient
// (ssgd_token_logprobs, ssgd_token_logprobs_backward).
//
// A row of V logits, z = scale * logits:
//   m = max z,  s = sum e^(z - m),  lse = m + log s,  logp = z[id] - lse,  H = log s - (sum e^(z - m) (z - m)) / s
// One pass: every thread keeps a running maximum and the two sums relative to it, and rescales them when the maximum
// rises.  A row is cut into granules of 16 aligned bytes (its first and last may be partial, so any base and stride will
// do); granule i of a segment belongs to thread i mod THREADS.
//
// Alternatives: the threads' maxima bound the k-th largest logit from below.  Every thread has left the maximum of each of its
// batches of granules in shared memory; the batches that reach the bound, some 20 to 60, are read again, and the logits that
// reach it are sorted, 32 to a warp, and merged.  Order: larger logit first, then smaller index; a NaN
// counts as the largest; -0 and +0 are equal.
//
// Few rows: a cluster of CTAs shares a row and joins through distributed shared memory, so there is still one launch
// and no scratch.
//
// Gradient, p_j = e^(z_j - lse), A = d_logp + sum of d_top:
//   dlogits_j = scale * (d_logp [j = id] + sum_m d_top_m [j = top_m] - p_j (A + d_entropy (z_j - lse + H)))
// One read and one write per logit; the few columns with an extra term are written a second time by the CTA that owns
// them, after a barrier.
#include <cooperative_groups.h>

#include "logits.cuh"

using namespace ssgd;
namespace cg = cooperative_groups;

namespace {

constexpr int MAX_TOP = SSGD_MAX_TOP;       // one entry per lane of a warp
static_assert(MAX_TOP == 32, "a warp's list has an entry per lane");

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
__device__ __forceinline__ uint64_t sort32(uint64_t x) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1) {
#pragma unroll
        for (int o = k >> 1; o > 0; o >>= 1) {
            const uint64_t other = __shfl_xor_sync(0xffffffffu, x, o);
            const bool keep_larger = ((lane & o) == 0) == ((lane & k) == 0);
            x = keep_larger == (x > other) ? x : other;
        }
    }
    return x;
}

constexpr int CANDIDATES = 256, ITEMS = 256;
constexpr int BATCH = 4;                  // granules that a thread reads at once
constexpr int SLOTS = 16;                 // maxima that a thread leaves behind

template <int NT, bool TOP>
struct Shared {
    Sums part[8];                     // part[0] is the CTA's in the end
    uint64_t list[8][MAX_TOP];        // list[0] is the CTA's in the end
    uint64_t candidate[CANDIDATES];
    uint32_t bound[8];
    float slot[TOP ? SLOTS : 1][TOP ? NT : 1];     // the maximum of each of the thread's batches (or runs of batches)
    int32_t item[ITEMS];
    int32_t nitems, ncandidates;
};

// The order of the elements of a granule (0 where there is none)
template <typename T>
__device__ __forceinline__ void orders_of(const Granules<T>& G, int32_t i, bool there, uint32_t (&order)[16 / sizeof(T)]) {
    constexpr int VEC = 16 / sizeof(T);
    const int32_t at = G.first(i);
#pragma unroll
    for (int e = 0; e < VEC; ++e) order[e] = 0;
    if (!there) return;
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

// Granules [g0, g1) of a row are a CTA's; the whole ones among them are [whole0, whole1), and thread t has whole0 + t + i NT.
struct Segment { int32_t g0, g1, whole0, whole1; };

// Rare: more than CANDIDATES logits reach the bound (many equal ones, or a few batches with nearly all the large ones).  Each
// warp goes through its share of the segment and inserts one by one into its list.
template <typename T, int NT>
__device__ __noinline__ uint64_t best_one_by_one(const Granules<T>& G, const Segment& S, uint32_t bound, int k) {
    constexpr int VEC = 16 / sizeof(T);
    uint64_t list = 0, last = 0;                           // lane's entry of the warp's list; the k-th entry
    for (int32_t base = S.g0 + ((int)threadIdx.x & ~31); base < S.g1; base += NT) {
        const int32_t i = base + ((int)threadIdx.x & 31), at = G.first(i);
        uint32_t order[VEC];
        orders_of<T>(G, i, i < S.g1, order);
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
    return list;
}

// The CTA's best of its segment into sh.list[0], in order, at least k of them (0 where there are fewer).  2^log_run batches
// share a slot of the threads' maxima.
template <typename T, int NT>
__device__ __forceinline__ void best_of_segment(Shared<NT, true>& sh, const Granules<T>& G, const Segment& S, float thread_max, int log_run, int k) {
    constexpr int VEC = 16 / sizeof(T), WARPS = NT / 32;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const bool has = S.whole0 + t < S.whole1;
    const uint32_t mine = has ? order_of(thread_max) : 0u;
    // The q-th largest maximum of each warp whose 32 threads all have granules, q = ceil(k / number of those warps): k logits
    // reach the least of these.  (No such warp: every logit is a candidate, fewer than 32 whole granules.)
    const int full = min((S.whole1 - S.whole0) / 32, WARPS);
    if (warp < full) {
        uint32_t left = mine, best = 0;
        for (int q = 0; q < k; q += full) {
            best = __reduce_max_sync(0xffffffffu, left);
            const uint32_t who = __ballot_sync(0xffffffffu, left == best);
            if (lane == __ffs(who) - 1) left = 0;
        }
        if (lane == 0) sh.bound[warp] = best;
    }
    if (t == 0) sh.nitems = sh.ncandidates = 0;
    __syncthreads();
    uint32_t bound = full > 0 ? 0xffffffffu : 0u;
    for (int i = 0; i < full; ++i) bound = min(bound, sh.bound[i]);
    auto candidate = [&](uint32_t order, int32_t index) {
        if (order >= bound && order != 0) {
            const int at = atomicAdd(&sh.ncandidates, 1);
            if (at < CANDIDATES) sh.candidate[at] = ((uint64_t)order << 32) | (0xffffffffu - (uint32_t)index);
        }
    };
    auto partial = [&](int32_t i) {
        for (int32_t at = max(G.first(i), 0); at < min(G.first(i) + VEC, G.n); ++at) candidate(order_of(to_f32(G.row[at])), at);
    };
    if (t == 0 && S.whole0 > S.g0) partial(S.g0);
    if (t == 32 % NT && S.whole1 < S.g1 && S.g1 - 1 >= S.whole0) partial(S.g1 - 1);
    if (has && mine >= bound) {
        const int slots = (((S.whole1 - S.whole0 + NT * BATCH - 1) / (NT * BATCH) - 1) >> log_run) + 1;
        for (int i = 0; i < slots; ++i) {
            if (order_of(sh.slot[i][t]) >= bound) {
                const int at = atomicAdd(&sh.nitems, 1);
                if (at < ITEMS) sh.item[at] = t | i << 16;
            }
        }
    }
    __syncthreads();
    // all threads share the granules of these batches
    const int log_each = log_run + 2, total = min(sh.nitems, ITEMS) << log_each;
    for (int p = t; p < total; p += NT) {
        const int32_t item = sh.item[p >> log_each];
        const int32_t i = S.whole0 + (item & 0xffff) + (((item >> 16) << log_each) + (p & ((1 << log_each) - 1))) * NT;
        if (i < S.whole1) {
            const Vec<T, VEC> v = load_vec<T, VEC>(G.row + G.first(i));
#pragma unroll
            for (int e = 0; e < VEC; ++e) candidate(order_of(to_f32(v.e[e])), G.first(i) + e);
        }
    }
    __syncthreads();
    const int n = sh.ncandidates;
    int lists = WARPS;
    uint64_t list = 0;
    if (n <= CANDIDATES && sh.nitems <= ITEMS) {
        lists = min((n + 31) / 32, WARPS);
        if (warp < lists) list = sort32(t < n ? sh.candidate[t] : 0);
        for (int at = t + NT; at - lane < n; at += NT) list = merge(list, sort32(at < n ? sh.candidate[at] : 0));
    } else {
        list = best_one_by_one<T, NT>(G, S, bound, k);
    }
    sh.list[warp][lane] = list;
    for (int half = WARPS / 2; half > 0; half >>= 1) {
        if (half >= lists) continue;                       // the same for the whole CTA
        __syncthreads();
        if (warp < half) {
            list = merge(list, sh.list[warp + half][lane]);
            sh.list[warp][lane] = list;
        }
    }
}

// At 4096 x 32000 in bfloat16 50 us, 5.2 TB/s (55 in sustained work).  Per logit 8.8 instructions, 31 us of issue slots at
// 1965 MHz, one of them a 2^x, of which an SM has 16 a cycle: 28 us.  Neither they nor the memory (40 us) are full; loads and
// arithmetic take turns.  The latency of the loads is covered by other CTAs, 6 of 256 threads per SM (with 4: 56 us, 5: 51; the
// next batch in registers while one is summed, 3 CTAs: 69).
template <typename T, bool TOP, int NT>
__global__ void __launch_bounds__(NT, 6 * 256 / NT) k_token_logprobs(const LogprobArgs A, int split) {
    constexpr int VEC = 16 / sizeof(T), WARPS = NT / 32, U = BATCH;
    __shared__ Shared<NT, TOP> sh;
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
    Running r{no_sums(), NEG_INF, c, __fdiv_ru(160.f, c)};
    // the row's first and last granule may be parts of one
    Segment S{g0, g1, g0 == 0 && G.phase ? 1 : g0, g1 == G.count && !G.whole(G.count - 1) ? g1 - 1 : g1};
    S.whole1 = max(S.whole1, min(S.whole0, g1));
    int log_run = 0;
    if (TOP) {
        const int batches = (S.whole1 - S.whole0 + NT * U - 1) / (NT * U);
        while ((batches - 1) >> log_run >= SLOTS) ++log_run;
    }
    {
        int32_t i = S.whole0 + t, b0 = S.whole0;
        const T* p = z + G.first(i);
        int batch = 0;
        float run_max = NEG_INF;
        auto leave = [&](float m) {
            if constexpr (TOP) {
                run_max = (batch & ((1 << log_run) - 1)) ? max_nan(run_max, m) : m;
                sh.slot[batch >> log_run][t] = run_max;
                ++batch;
            }
        };
        for (; b0 + NT * U <= S.whole1; b0 += NT * U, i += NT * U, p += NT * U * VEC) {
            Vec<T, VEC> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = TOP ? load_vec<T, VEC>(p + u * (NT * VEC)) : load_vec_stream<T, VEC>(p + u * (NT * VEC));
            leave(add_granules<T, U>(r, v, U));
        }
        if (b0 < S.whole1) {
            Vec<T, VEC> v[U];
            const int have = (S.whole1 - b0 + NT - 1) / NT;
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[u].e[e] = from_f32<T>(NEG_INF);
                if (i + u * NT < S.whole1)
                    v[u] = TOP ? load_vec<T, VEC>(p + u * (NT * VEC)) : load_vec_stream<T, VEC>(p + u * (NT * VEC));
            }
            leave(add_granules<T, U>(r, v, have));
        }
    }
    const float thread_max = r.a.m;
    auto partial = [&](int32_t i) {
        for (int32_t at = max(G.first(i), 0); at < min(G.first(i) + VEC, A.vocab); ++at) add_careful(r.a, to_f32(z[at]), c);
    };
    if (t == 0 && S.whole0 > g0) partial(g0);
    if (t == 32 % NT && S.whole1 < g1 && g1 - 1 >= S.whole0) partial(g1 - 1);
    Sums& a = r.a;
    const bool counted = id >= 0 && id < A.vocab;          // an id outside the vocabulary is ignored
    float z_id = 0.f;
    if (counted) z_id = to_f32(z[id]);
    // join: warp, CTA, cluster
    join_warp(a, c);
    if (lane == 0) sh.part[warp] = a;
    if constexpr (TOP) best_of_segment<T, NT>(sh, G, S, thread_max, log_run, A.top);
    __syncthreads();
    if (warp == 0) {
        a = lane < WARPS ? sh.part[lane] : no_sums();
        join_warp(a, c);
        if (lane == 0) sh.part[0] = a;
    }
    cg::cluster_group cluster = cg::this_cluster();
    if (split > 1) {
        cluster.sync();
        if (TOP && part == 0) {
            // the CTAs' lists, two by two
            for (int q = warp; q < split / 2; q += WARPS) {
                const uint64_t one = cluster.map_shared_rank(&sh.list[0][0], 2 * q)[lane];
                const uint64_t two = cluster.map_shared_rank(&sh.list[0][0], 2 * q + 1)[lane];
                sh.candidate[q * 32 + lane] = merge(one, two);
            }
            for (int half = split / 4; half > 0; half >>= 1) {
                __syncthreads();
                for (int q = warp; q < half; q += WARPS)
                    sh.candidate[q * 32 + lane] = merge(sh.candidate[q * 32 + lane], sh.candidate[(q + half) * 32 + lane]);
            }
        }
    }
    if (part == 0 && warp == 0) {
        if (split > 1) {
            a = lane < split ? *cluster.map_shared_rank(&sh.part[0], lane < split ? lane : 0) : no_sums();
            join_warp(a, c);
        }
        const float log2s = log2f(a.s);
        const bool none = a.s == 0.f;                      // every logit is -inf
        // relative to the reference that the sums have: log p = (x c - shift) - log2 s in powers of two; in powers of e from the
        // start where that would overflow
        const bool plain = near(a.shift);
        auto logp_of = [&](float x) {
            if (none || (x == NEG_INF && a.s == a.s)) return NEG_INF;
            return plain && fabsf(x) < HUGE_LOGIT ? (fmaf(x, c, -a.shift) - log2s) * LN2 : fmaf(x - a.m, A.scale, -log2s * LN2);
        };
        if (lane == 0) {
            A.stats[row] = counted ? logp_of(z_id) : 0.f;
            A.stats[A.rows + row] = none ? 0.f : (log2s - a.w / a.s) * LN2;
            A.stats[2 * A.rows + row] = none ? NEG_INF : plain ? (a.shift + log2s) * LN2 : fmaf(a.m, A.scale, log2s * LN2);
        }
        if (TOP && lane < A.top) {
            const uint64_t key = split > 1 ? sh.candidate[lane] : sh.list[0][lane];
            A.top_idx[row * A.top + lane] = (int32_t)(0xffffffffu - (uint32_t)key);
            A.top_logp[row * A.top + lane] = logp_of(logit_of(key));
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

// CTA (row, part) writes `per` granules of a row, in batches of BACK_U reads per thread.  At 8192 x 32000 in bfloat16 168 us, 6.2 TB/s
// (0.95 of a copy; 174 in sustained work), 7.5 instructions per logit.
template <typename T, bool ENTROPY, int NT>
__global__ void __launch_bounds__(NT) k_token_logprobs_back(const LogprobBackArgs A) {
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
    // gradient of two logits without the columns' own terms: p (base + slope log p).  p <= 1: far from zero the 32 bits of lse can lie
    // below a logit by hundreds, and 2^x would be inf.  (log p itself keeps the last place that lse has lost: entropy has it too.)
    auto grad = [&](float2 x) {
        const float2 logp = fma2(x, both(scale), both(minus_lse));
        const float2 t = mul2(make_float2(min_nan(logp.x, 0.f), min_nan(logp.y, 0.f)), both(LOG2E)), p = make_float2(ex2(t.x), ex2(t.y));
        if (!ENTROPY) return mul2(p, both(base));
        const float2 bounded = make_float2(fminf(fmaxf(logp.x, -200.f), 1.f), fminf(fmaxf(logp.y, -200.f), 1.f));
        return mul2(p, fma2(bounded, both(slope), both(base)));
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
        for (int32_t b0 = g0; b0 < g1; b0 += NT * BACK_U) {
            const int32_t at = G.first(b0 + t);
            Vec<T, VEC> v[BACK_U];
            float2 f[VEC / 2];
            if (b0 >= whole0 && b0 + NT * BACK_U <= whole1) {
#pragma unroll
                for (int u = 0; u < BACK_U; ++u) v[u] = load_vec_stream<T, VEC>(z + at + u * (NT * VEC));
#pragma unroll
                for (int u = 0; u < BACK_U; ++u) {
                    unpack_pairs(v[u], f);
#pragma unroll
                    for (int e = 0; e < VEC / 2; ++e) f[e] = grad(f[e]);
                    store_vec<T, VEC>(out + at + u * (NT * VEC), pack_pairs<T, VEC>(f));
                }
                continue;
            }
#pragma unroll
            for (int u = 0; u < BACK_U; ++u) {
                const int32_t i = b0 + u * NT + t;
                if (i >= whole0 && i < whole1) v[u] = load_vec_stream<T, VEC>(z + G.first(i));
            }
#pragma unroll
            for (int u = 0; u < BACK_U; ++u) {
                const int32_t i = b0 + u * NT + t;
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
        for (int32_t j = lo + t; j < hi; j += NT) out[j] = one(to_f32(z[j]));
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

// CTAs that share a row: enough of them for 4 per SM, while each still has two granules per thread.  Measured at 300 x 50001
// fp32 (us, without / with 5 alternatives): up to 2 per SM 18.7 / 27.4, 4 16.7 / 22.9, 8 19.9 / 28.2.
int split_for(int64_t rows, int64_t granules, int sms) {
    int split = 1;
    while (split < 8 && rows * split < 4 * sms && granules / (split * 2) >= 2 * 256) split *= 2;
    return split;
}

// Rows of up to this many granules are left to CTAs of 64 threads where there are enough rows: what a CTA spends on a row's joins
// does not depend on its length.  Measured (us, 64 / 256 threads): 3641 x 6156 binary16 (770 granules) 17.3 / 20.7, with 5
// alternatives 28.7 / 36.9; 1637 x 5325 fp32 (1332) with 20 26.9 / 24.6; 4096 x 32000 bfloat16 (4000) 57.4 / 50.0.
constexpr int64_t SHORT_ROW = 1024;
template <typename T, int NT>
int launch_logprobs_nt(const LogprobArgs& A, int split, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(A.rows * split));
    cfg.blockDim = dim3(NT);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = split > 1 ? 1 : 0;
    const cudaError_t e = A.top ? cudaLaunchKernelEx(&cfg, k_token_logprobs<T, true, NT>, A, split)
                                : cudaLaunchKernelEx(&cfg, k_token_logprobs<T, false, NT>, A, split);
    return e == cudaSuccess ? SSGD_OK : SSGD_ECUDA;
}

template <typename T>
int launch_logprobs(const LogprobArgs& A, int sms, cudaStream_t st) {
    const int64_t granules = ((int64_t)A.vocab * sizeof(T) + 15) / 16;
    const int split = split_for(A.rows, granules, sms);
    if (granules <= SHORT_ROW && A.rows >= 4 * sms) return launch_logprobs_nt<T, 64>(A, 1, st);
    return launch_logprobs_nt<T, 256>(A, split, st);
}

template <typename T, int NT>
int launch_logprobs_back_nt(LogprobBackArgs A, int sms, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T), BATCH = NT * BACK_U;
    const int64_t granules = (A.vocab + 2 * VEC - 2) / VEC;             // whatever the phase
    // Whole batches per CTA, 4 of them where that still makes 8 CTAs per SM: the row's constants cost a CTA as much as
    // a batch.
    int64_t batches = 4;
    while (batches > 1 && A.rows * ((granules + batches * BATCH - 1) / (batches * BATCH)) < 8 * sms) batches /= 2;
    A.per = (int32_t)(batches * BATCH);
    const int64_t parts = (granules + A.per - 1) / A.per;
    if (parts > 65535) return SSGD_EINVAL;
    const dim3 grid((unsigned)A.rows, (unsigned)parts);
    if (A.d_entropy) k_token_logprobs_back<T, true, NT><<<grid, NT, 0, st>>>(A);
    else k_token_logprobs_back<T, false, NT><<<grid, NT, 0, st>>>(A);
    return launched();
}
template <typename T>
int launch_logprobs_back(const LogprobBackArgs& A, int sms, cudaStream_t st) {
    // A short row leaves most of 256 threads with the row's constants alone: 64 / 256 threads at 1846 x 3904 binary16 8.3 / 14.4 us,
    // 4000 x 500 bfloat16 8.2 / 16.5.
    if ((int64_t)A.vocab * (int)sizeof(T) / 16 <= 768) return launch_logprobs_back_nt<T, 64>(A, sms, st);
    return launch_logprobs_back_nt<T, 256>(A, sms, st);
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
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return fmt == SSGD_FMT_F32 ? launch_logprobs<float>(A, sms, st)
         : fmt == SSGD_FMT_F16 ? launch_logprobs<__half>(A, sms, st) : launch_logprobs<__nv_bfloat16>(A, sms, st);
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
