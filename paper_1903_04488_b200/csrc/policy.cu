// policy.cu -- the clipped policy loss of sampled tokens with a penalty for leaving a reference and an entropy bonus, and its
// gradient with respect to the logits, in one pass (ssgd_policy_loss).
//
// A row of V logits, z = scale * logits, p = e^(z - lse), logp = z[id] - lse, H = -sum p log p:
//   r = e^(logp - old),  kept = A >= 0 ? min(r, 1 + high) : max(r, 1 - low),  q = ref - logp,  K = e^q - 1 - q
//   loss = w (-kept A + kl K - entropy H)
//   c = -A r [kept = r] - kl (e^q - 1)                                  (the slope along logp)
//   dlogits_j = w scale (c ([j = id] - p_j) + entropy p_j (log p_j + H))
// A loss apart from its gradient would read the logits twice: nothing of the gradient is known before the row's sum is.  Here the row
// stays in shared memory in between (a cluster of CTAs shares one that is too long, or where rows are few), so that every
// logit is read once and every gradient written once, and the memory is what bounds it.  A token of weight 0 is not even read.
//
// At 8192 x 32000 bfloat16 205 us over the same logits again and again, 212 to 216 over new ones: 4.9 to 5.1 TB/s (0.74 to 0.78 of a
// copy).  15 instructions per logit are 109 us of issue slots, two 2^x 58 us of the special-function unit each; three CTAs of 64 KB share
// an SM, and their loads, sums and stores overlap only so far.
//
// Granule i of a CTA's segment belongs to thread i mod threads, which copies it to shared memory (cp.async, up to four batches ahead),
// adds it to its running sums (logits.cuh), and makes its gradient: no barrier but those of the row's sums.
#include <cooperative_groups.h>

#include "logits.cuh"

using namespace ssgd;
namespace cg = cooperative_groups;

namespace {

struct Args {
    const void* logits; int64_t ld;
    const void* ids; bool ids64;
    const float* old_logp; const float* advantages; const float* ref_logp; const float* weights;
    int64_t rows; int32_t vocab;
    float scale, low, high, kl, entropy;
    float* stats;                                   // [5][rows]: loss, logp, entropy, kl, ratio
    void* out; int64_t ld_out;                      // NULL: no gradient
    bool same_phase;                                // rows of logits and of the gradient lie alike within 16 bytes
};

constexpr int BATCH = 4;                            // granules that a thread takes at once
constexpr int AHEAD = 4;                            // batches on their way

template <int OFFSET>
__device__ __forceinline__ void copy_async_at(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0 + %2], [%1 + %2], 16;" ::"r"(to), "l"(from), "n"(OFFSET) : "memory");
}

struct Row {                                        // what the gradient needs of a row
    float m, shift, log2s;                          // log2 p = (z c - shift) - log2 s, or (z - m) c - log2 s
    float base, slope;                              // gradient = p (base + slope log2 p)
    float own;                                      // and this at the id
    bool none;                                      // nothing but -inf
};
template <int NT> struct Shared {
    Sums part[NT / 32];
    Row row;
};

// log2 p of two logits: (z c - shift) - log2 s, or for far rows (z - m) c - log2 s
__device__ __forceinline__ float2 log2_p(const Row& r, float c, bool plain, float2 x) {
    const float2 l = plain ? fma2(x, both(c), both(-r.shift)) : make_float2((x.x - r.m) * c, (x.y - r.m) * c);
    return add2(l, both(-r.log2s));
}
// Two logits' gradients from there, without the id's own term
template <bool ENTROPY>
__device__ __forceinline__ float2 grad(const Row& r, float2 l) {
    const float2 p = make_float2(ex2(l.x), ex2(l.y));
    if (!ENTROPY) return mul2(p, both(r.base));
    // p is zero below; log2 p may be -inf there
    const float2 bounded = make_float2(l.x < -200.f ? -200.f : l.x, l.y < -200.f ? -200.f : l.y);
    return mul2(p, fma2(bounded, both(r.slope), both(r.base)));
}
// Where 16 bits are stored, shift + log2 s may be one number: up to FOLD its rounding is 2^-18, 2.6e-6 of p.
constexpr float FOLD = 64.f;

// KEEP: the CTA's segment stays in shared memory; otherwise it is read again, or there is no gradient to be written.
template <typename T, bool ENTROPY, bool KEEP, int NT>
__global__ void __launch_bounds__(NT) k_policy(const Args A, int split) {
    constexpr int VEC = 16 / sizeof(T), WARPS = NT / 32, U = BATCH, STEP = NT * U;
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ Shared<NT> sh;
    Vec<T, VEC>* seg = reinterpret_cast<Vec<T, VEC>*>(raw);
    cg::cluster_group cluster = cg::this_cluster();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int shift = __ffs(split) - 1, part = blockIdx.x & (split - 1);
    const int64_t row = blockIdx.x >> shift;
    const T* z = static_cast<const T*>(A.logits) + row * A.ld;
    T* out = static_cast<T*>(A.out) + row * A.ld_out;
    const Granules<T> G(z, A.vocab);
    const int32_t per = (G.count + split - 1) >> shift;
    const int32_t g0 = min(part * per, G.count), g1 = min(g0 + per, G.count);
    const int32_t lo = max(G.first(g0), 0), hi = min(G.first(g1), A.vocab);     // columns of the CTA
    const int64_t id = id_of(A.ids, A.ids64, row);
    const float w = A.weights ? A.weights[row] : 1.f;
    if (w == 0.f || id < 0 || id >= A.vocab) {      // the same for the whole cluster
        if (part == 0 && t < 5) A.stats[t * A.rows + row] = 0.f;
        if (A.out) {
            // whole granules of the result, which may lie otherwise than the logits'
            const Granules<T> O(out, A.vocab);
            const int32_t o0 = min(g0, O.count), o1 = part == split - 1 ? O.count : min(g1, O.count);
            Vec<T, VEC> zero;
#pragma unroll
            for (int e = 0; e < VEC; ++e) zero.e[e] = from_f32<T>(0.f);
            for (int32_t i = o0 + t; i < o1; i += NT) {
                if (O.whole(i)) store_vec<T, VEC>(out + O.first(i), zero);
                else for (int32_t j = max(O.first(i), 0); j < min(O.first(i) + VEC, A.vocab); ++j) out[j] = zero.e[0];
            }
        }
        return;
    }
    const float c = A.scale * LOG2E;
    const float z_id = to_f32(z[id]);               // before the gradient, which may lie in the same place, is written
    float adv = 0.f, old_logp = 0.f, ref_logp = 0.f;
    if (t == 0) {                                   // long before they are needed
        adv = A.advantages[row];
        old_logp = A.old_logp[row];
        if (A.ref_logp) ref_logp = A.ref_logp[row];
    }
    Running r{no_sums(), NEG_INF, c, __fdiv_ru(160.f, c)};
    // the row's first and last granule may be parts of one
    const int32_t whole0 = g0 == 0 && G.phase ? 1 : g0;
    const int32_t whole1 = max(g1 == G.count && !G.whole(G.count - 1) ? g1 - 1 : g1, min(whole0, g1));
    const int32_t n = whole1 - whole0;
    // the thread's granules: t, t + NT, ..
    const T* mine = z + G.first(whole0) + (int64_t)t * VEC;
    Vec<T, VEC>* kept = seg + t;
    {
        const T* from = mine;
        uint32_t to = (uint32_t)__cvta_generic_to_shared(kept);
        int32_t left = n - t;                       // the thread has one more granule for every NT of them
        auto copy = [&] {
            if constexpr (KEEP) {
                if (left > (U - 1) * NT) {
                    copy_async_at<0>(to, from);
                    copy_async_at<NT * 16>(to, from);
                    copy_async_at<2 * NT * 16>(to, from);
                    copy_async_at<3 * NT * 16>(to, from);
                } else {
                    if (left > 0) copy_async_at<0>(to, from);
                    if (left > NT) copy_async_at<NT * 16>(to, from);
                    if (left > 2 * NT) copy_async_at<2 * NT * 16>(to, from);
                }
                to += STEP * 16;
                from += STEP * VEC;
                left -= STEP;
                copy_async_commit();
            }
        };
        for (int k = 0; k < AHEAD; ++k) copy();
        const Vec<T, VEC>* at = KEEP ? kept : reinterpret_cast<const Vec<T, VEC>*>(mine);
        int32_t rest = n;
        for (; rest >= STEP; rest -= STEP, at += STEP) {
            Vec<T, VEC> v[U];
            if (KEEP) copy_async_wait<AHEAD - 1>();
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = KEEP ? at[u * NT] : load_vec<T, VEC>(reinterpret_cast<const T*>(at + u * NT));
            copy();
            add_granules<T, U>(r, v, U);
        }
        if (rest > 0) {
            Vec<T, VEC> v[U];
            if (KEEP) copy_async_wait<0>();
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[u].e[e] = from_f32<T>(NEG_INF);
                if (u * NT + t < rest) v[u] = KEEP ? at[u * NT] : load_vec<T, VEC>(reinterpret_cast<const T*>(at + u * NT));
            }
            add_granules<T, U>(r, v, (rest + NT - 1) / NT);
        }
    }
    auto partial = [&](int32_t i) {
        for (int32_t at = max(G.first(i), 0); at < min(G.first(i) + VEC, A.vocab); ++at) add_careful(r.a, to_f32(z[at]), c);
    };
    const bool head = whole0 > g0, tail = whole1 < g1 && g1 - 1 >= whole0;
    if (t == 0 && head) partial(g0);
    if (t == 32 % NT && tail) partial(g1 - 1);
    // join: warp, CTA, cluster
    Sums& a = r.a;
    join_warp(a, c);
    if (lane == 0) sh.part[warp] = a;
    __syncthreads();
    if (warp == 0) {
        a = lane < WARPS ? sh.part[lane] : no_sums();
        join_warp(a, c);
        if (lane == 0) sh.part[0] = a;
    }
    if (split > 1) cluster.sync();
    if (warp == 0) {
        if (split > 1) {
            a = lane < split ? *cluster.map_shared_rank(&sh.part[0], lane < split ? lane : 0) : no_sums();
            join_warp(a, c);
        }
        if (lane == 0) {
            const float log2s = log2f(a.s);
            const bool none = a.s == 0.f, plain = near(a.shift);               // none: every logit is -inf
            float logp = plain && fabsf(z_id) < HUGE_LOGIT ? (fmaf(z_id, c, -a.shift) - log2s) * LN2 : fmaf(z_id - a.m, A.scale, -log2s * LN2);
            if (none || (z_id == NEG_INF && a.s == a.s)) logp = NEG_INF;
            const float h = none ? 0.f : (log2s - a.w / a.s) * LN2;
            const float ratio = expf(logp - old_logp);
            const float kept = adv >= 0.f ? (ratio > 1.f + A.high ? 1.f + A.high : ratio) : (ratio < 1.f - A.low ? 1.f - A.low : ratio);
            float along = kept == ratio ? -adv * ratio : 0.f, kl = 0.f, loss = -kept * adv;
            if (ratio != ratio || adv != adv) along = loss;
            if (A.entropy != 0.f) loss -= A.entropy * h;
            if (A.ref_logp) {
                const float q = ref_logp - logp, e = expm1f(q);
                kl = e - q;
                if (A.kl != 0.f) {
                    loss = fmaf(A.kl, kl, loss);
                    along = fmaf(-A.kl, e, along);
                }
            }
            const float ws = w * A.scale;
            sh.row = Row{a.m, a.shift, log2s, ws * (A.entropy * h - along), ws * A.entropy * LN2, ws * along, none};
            if (part == 0) {
                A.stats[row] = w * loss;
                A.stats[A.rows + row] = logp;
                A.stats[2 * A.rows + row] = h;
                A.stats[3 * A.rows + row] = kl;
                A.stats[4 * A.rows + row] = ratio;
            }
        }
    }
    if (A.out) {
        __syncthreads();
        const Row R = sh.row;
        const bool plain = near(R.shift);
        // the single elements: of partial granules, and of all where the result lies otherwise than the logits
        auto one = [&](int32_t j, float x) {
            float v = R.none || (x == NEG_INF && R.log2s == R.log2s) ? 0.f : grad<ENTROPY>(R, log2_p(R, c, plain && fabsf(x) < HUGE_LOGIT, both(x))).x;
            if (j == (int32_t)id) v += R.own;
            out[j] = from_f32<T>(v);
        };
        if (A.same_phase && !R.none && plain) {
            // the id's element among the others first, then once more by the thread that has its granule
            const int32_t own = ((int32_t)id - G.first(whole0)) / VEC;
            const bool has_id = (int32_t)id >= G.first(whole0) && own < n && own % NT == t;
            const float x_id = has_id ? to_f32(z[id]) : 0.f;
            auto all = [&](auto log2_of) {
                const Vec<T, VEC>* at = KEEP ? kept : reinterpret_cast<const Vec<T, VEC>*>(mine);
                T* to = out + G.first(whole0) + (int64_t)t * VEC;
                auto write = [&](int u) {
                    const Vec<T, VEC> v = KEEP ? at[u * NT] : load_vec<T, VEC>(reinterpret_cast<const T*>(at + u * NT));
                    float2 f[VEC / 2];
                    unpack_pairs(v, f);
#pragma unroll
                    for (int e = 0; e < VEC / 2; ++e) f[e] = grad<ENTROPY>(R, log2_of(f[e]));
                    store_vec<T, VEC>(to + u * (NT * VEC), pack_pairs<T, VEC>(f));
                };
                int32_t left = n - t;
                for (; left > (U - 1) * NT; left -= STEP, at += STEP, to += STEP * VEC) {
#pragma unroll
                    for (int u = 0; u < U; ++u) write(u);
                }
                for (; left > 0; left -= NT, at += NT, to += NT * VEC) write(0);
            };
            const float fold = R.shift + R.log2s;
            if (sizeof(T) == 2 && fabsf(fold) < FOLD) all([&](float2 x) { return fma2(x, both(c), both(-fold)); });
            else all([&](float2 x) { return log2_p(R, c, true, x); });
            if (has_id) one((int32_t)id, x_id);
        } else {
            for (int32_t i = t; i < n; i += NT) {
                const Vec<T, VEC> v = KEEP ? seg[i] : load_vec<T, VEC>(mine + (int64_t)(i - t) * VEC);
                for (int e = 0; e < VEC; ++e) one(G.first(whole0 + i) + e, to_f32(v.e[e]));
            }
        }
        if (t == 0 && head)
            for (int32_t j = lo; j < min(G.first(g0) + VEC, A.vocab); ++j) one(j, to_f32(z[j]));
        if (t == 32 % NT && tail)
            for (int32_t j = max(G.first(g1 - 1), 0); j < hi; ++j) one(j, to_f32(z[j]));
    }
    if (split > 1) cluster.sync();                  // nobody leaves while its shared memory is read
}

// ---- host side ---------------------------------------------------------------------------------------

constexpr int SEGMENT = 72 * 1024;                  // bytes of a row that a CTA keeps at most while rows can be shared: three CTAs to an SM
constexpr int MOST = 208 * 1024;                    // and where a cluster of 8 needs more

template <typename T, bool ENTROPY, bool KEEP, int NT>
int launch_nt(const Args& A, int split, int smem, cudaStream_t st) {
    static PerDevice opted;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return SSGD_ECUDA;
    if (KEEP && !opted.value[dev]) {
        if (cudaFuncSetAttribute(k_policy<T, ENTROPY, KEEP, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST) != cudaSuccess) return SSGD_ECUDA;
        opted.value[dev] = 1;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(A.rows * split));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = split > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k_policy<T, ENTROPY, KEEP, NT>, A, split) == cudaSuccess ? SSGD_OK : SSGD_ECUDA;
}

template <typename T>
int launch_policy(const Args& A, int sms, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T);
    const int64_t granules = (A.vocab + 2 * VEC - 2) / VEC;                     // whatever the phase
    int split = 1;
    while (split < 8 && (granules * 16 > (int64_t)split * SEGMENT || (A.rows * split < 4 * sms && granules / (split * 2) >= 2 * 256))) split *= 2;
    const int64_t smem = (granules + split - 1) / split * 16;
    const bool keep = A.out && smem <= MOST;
    // as for the log probabilities: short rows go to small CTAs
    const bool small = granules <= 1024 && A.rows >= 4 * sms;
    auto go = [&](auto entropy) {
        constexpr bool E = decltype(entropy)::value;
        if (small) return keep ? launch_nt<T, E, true, 64>(A, 1, (int)smem, st) : launch_nt<T, E, false, 64>(A, 1, 0, st);
        return keep ? launch_nt<T, E, true, 256>(A, split, (int)smem, st) : launch_nt<T, E, false, 256>(A, split, 0, st);
    };
    return A.entropy != 0.f && A.out ? go(std::true_type{}) : go(std::false_type{});
}

}  // namespace

extern "C" int ssgd_policy_loss(const void* logits, int64_t ld, int32_t fmt, const void* ids, int32_t ids_bytes, int64_t rows, int64_t vocab,
                                float scale, const float* old_logp, const float* advantages, const float* ref_logp, const float* weights,
                                float clip_low, float clip_high, float kl, float entropy, float* stats, void* dlogits, int64_t ld_d,
                                void* stream) {
    if (rows < 0 || rows > 0x0fffffff || vocab < 1 || vocab > (int64_t)1 << 27 || ld < vocab || !fmt_bytes(fmt)) return SSGD_EINVAL;
    if (!(scale > 0.f) || !(scale < INFINITY) || !(clip_low >= 0.f) || !(clip_low <= 1.f) || !(clip_high >= 0.f)) return SSGD_EINVAL;
    if (!(kl >= 0.f) || !(kl < INFINITY) || !(entropy > -INFINITY) || !(entropy < INFINITY) || (kl != 0.f && !ref_logp && rows)) return SSGD_EINVAL;
    if (ids_bytes != 4 && ids_bytes != 8) return SSGD_EINVAL;
    if (dlogits && ld_d < vocab) return SSGD_EINVAL;
    if (rows == 0) return SSGD_OK;
    if (!logits || !ids || !old_logp || !advantages || !stats) return SSGD_EINVAL;
    const int es = fmt_bytes(fmt);
    if (!aligned_to(logits, es) || !aligned_to(dlogits, es) || !aligned_to(ids, ids_bytes) || !aligned_to(old_logp, 4) ||
        !aligned_to(advantages, 4) || !aligned_to(ref_logp, 4) || !aligned_to(weights, 4) || !aligned_to(stats, 4))
        return SSGD_EALIGN;
    int sms = 0;
    if (int e = sm_count_of_current_device(&sms)) return e;
    Args A{logits, ld, ids, ids_bytes == 8, old_logp, advantages, ref_logp, weights, rows, (int32_t)vocab, scale, clip_low, clip_high, kl, entropy,
           stats, dlogits, ld_d, false};
    A.same_phase = addr(logits) % 16 == addr(dlogits) % 16 && (rows == 1 || (ld - ld_d) * es % 16 == 0);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return fmt == SSGD_FMT_F32 ? launch_policy<float>(A, sms, st)
         : fmt == SSGD_FMT_F16 ? launch_policy<__half>(A, sms, st) : launch_policy<__nv_bfloat16>(A, sms, st);
}
