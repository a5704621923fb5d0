// preference.cu -- the preference loss of pairs of token sequences, and its gradient (ssgd_preference_loss).
//
// Sequence s is tokens [starts[s], starts[s + 1]); pair p is sequences 2 p (preferred) and 2 p + 1.
//   D_s = sum of (logp - ref)  (over its length, with `average`),  x = beta (D_2p - D_2p+1)
//   loss = w l(x),  d_logp of a token of sequence s = +-w beta l'(x)  (over the length, with `average`)
// What bounds it is memory: 8 bytes read and 4 written per token, and every token of a sequence has the same gradient, so nothing is
// read twice.  Lengths are known on the device alone and may be anything, so the work is cut by tokens, 4096 to a CTA, and not by
// pairs: the first launch leaves the sum of every piece of a sequence (a CTA's tokens that belong to it), the second joins the pieces
// of its pairs, each CTA for itself and all in the same order, and writes.  The piece of sequence s in CTA k has place k + s: between
// two pieces that follow one another either grows by one, so no two share a place, and there are CTAs + sequences places.
// A call of one CTA does both in one launch.
#include "formats.cuh"

using namespace ssgd;

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int EACH = 16;                            // consecutive tokens of a thread
constexpr int CHUNK = THREADS * EACH;

struct Args {
    const float* logp; const float* ref;            // ref: NULL for zeros
    const void* starts; bool starts64;
    const float* weights;                           // [pairs] or NULL
    int64_t tokens, pairs;
    float beta, smoothing;
    int32_t kind;
    bool average;
    float* loss; float* rewards;                    // [pairs], [2][pairs]
    float* d_logp;                                  // [tokens] or NULL
    double* pieces;                                 // [chunks + 2 pairs]
    int64_t* ranges;                                // [chunks][2], see Range
    bool vector;                                    // logp and ref are 16-byte aligned
};

// starts[s], kept within the tokens
__device__ __forceinline__ int64_t start_of(const Args& A, int64_t s) {
    const int64_t v = A.starts64 ? static_cast<const int64_t*>(A.starts)[s] : (int64_t)static_cast<const int32_t*>(A.starts)[s];
    return v < 0 ? 0 : v > A.tokens ? A.tokens : v;
}

constexpr int FEW = 64;                             // sequences of a CTA that are gone through one by one
constexpr int SHORT = 32;                           // where there are more, pieces below it are summed by one thread, others by a warp
constexpr int LONG = 256;                           // pieces of a pair that the whole CTA joins
constexpr int32_t NO_MARK = 0x7fa12345;             // the bits of a NaN that no operation makes
struct Shared {
    float diff[CHUNK];                              // then the gradients
    int32_t bound[FEW + 1];                         // where the sequences begin within the CTA's tokens
    float value[FEW];                               // their gradients
    union {
        double part[WARPS][FEW];
        int32_t list[CHUNK / SHORT + 1];
    };
    int32_t listed;
    int32_t last[WARPS];
    double joined[WARPS];
};

// Tokens of the CTA, and the sequences that may have some of them: from the last one that starts before the first token to the last one
// that starts before the end.  The last CTA has those too that start at the end.
struct Range {
    int64_t c0, c1, s0, s1;
    __device__ __forceinline__ int within(int64_t token) const { return (int)((token < c0 ? c0 : token > c1 ? c1 : token) - c0); }
};

// The whole CTA searches, 256 places at a time, for the first starts that are at least c0 and at least c1.
__device__ __forceinline__ Range range_of(const Args& A, int64_t chunk, bool last) {
    Range R;
    R.c0 = chunk * CHUNK;
    R.c1 = min(R.c0 + CHUNK, A.tokens);
    const int64_t n = 2 * A.pairs + 1;
    int64_t lo[2] = {0, 0}, hi[2] = {chunk == 0 ? 0 : n, last ? 0 : n};
    while (lo[0] < hi[0] || lo[1] < hi[1]) {
        bool below[2];
        int64_t step[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            step[q] = (hi[q] - lo[q] + THREADS - 1) / THREADS;
            const int64_t at = lo[q] + (int64_t)threadIdx.x * step[q];
            below[q] = at < hi[q] && start_of(A, at) < (q ? R.c1 : R.c0);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int k = __syncthreads_count(below[q]);   // places lo, lo + step, .. that are before the answer
            if (lo[q] >= hi[q]) continue;
            const int64_t from = k ? lo[q] + (int64_t)(k - 1) * step[q] + 1 : lo[q];
            hi[q] = k ? min(hi[q], lo[q] + (int64_t)k * step[q]) : lo[q];
            lo[q] = from;
        }
    }
    R.s0 = max(lo[0] - 1, (int64_t)0);
    R.s1 = last ? 2 * A.pairs : min(lo[1], 2 * A.pairs);
    if (R.s1 < R.s0) R.s1 = R.s0;                   // starts that do not ascend
    return R;
}

// The CTA's tokens into shared memory
__device__ __forceinline__ void load_tokens(const Args& A, Shared& S, int64_t c0) {
    const int64_t left = A.tokens - c0;
    if (A.vector && left >= CHUNK) {
#pragma unroll
        for (int i = 0; i < EACH / 4; ++i) {
            const int at = (i * THREADS + (int)threadIdx.x) * 4;
            const Vec<float, 4> x = load_vec_stream<float, 4>(A.logp + c0 + at);
            Vec<float, 4> y{};
            if (A.ref) y = load_vec_stream<float, 4>(A.ref + c0 + at);
            store_vec<float, 4>(S.diff + at, Vec<float, 4>{{x.e[0] - y.e[0], x.e[1] - y.e[1], x.e[2] - y.e[2], x.e[3] - y.e[3]}});
        }
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int at = i * THREADS + (int)threadIdx.x;
            if (at < left) S.diff[at] = A.logp[c0 + at] - (A.ref ? A.ref[c0 + at] : 0.f);
        }
    }
    if (threadIdx.x == 0) S.listed = 0;
    __syncthreads();
}

// Sums of the pieces of the CTA's tokens, in 64 bits.  Each is added up by itself, so that what one sequence holds (infinities,
// the lowest number of a mask) stays there.
__device__ __forceinline__ void sum_pieces(const Args& A, Shared& S, int64_t chunk, const Range& R) {
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    auto join = [&](double v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    };
    if (R.s1 - R.s0 <= FEW) {                       // every warp takes an eighth of the tokens
        const int n = (int)(R.s1 - R.s0);
        if (t <= n) S.bound[t] = R.within(start_of(A, R.s0 + t));
        __syncthreads();
        constexpr int SPAN = CHUNK / WARPS;
        for (int q = 0; q < n; ++q) {
            const int a = max(S.bound[q], warp * SPAN), b = min(S.bound[q + 1], (warp + 1) * SPAN);
            double sum[2] = {0.0, 0.0};
            if (a < b) {
                int i = a + lane;
                for (; i + 32 < b; i += 64) {
                    sum[0] += (double)S.diff[i];
                    sum[1] += (double)S.diff[i + 32];
                }
                if (i < b) sum[0] += (double)S.diff[i];
                sum[0] = join(sum[0] + sum[1]);
            }
            if (lane == 0) S.part[warp][q] = sum[0];
        }
        __syncthreads();
        if (t < n && S.bound[t] < S.bound[t + 1]) {
            double sum = 0.0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) sum += S.part[w][t];
            A.pieces[chunk + R.s0 + t] = sum;
        }
        return;
    }
    for (int64_t s = R.s0 + t; s < R.s1; s += THREADS) {
        const int a = R.within(start_of(A, s)), b = R.within(start_of(A, s + 1));
        if (b - a >= SHORT) {
            const int at = atomicAdd(&S.listed, 1);
            if (at <= CHUNK / SHORT) S.list[at] = (int32_t)(s - R.s0);         // more only where starts do not ascend
        } else if (b > a) {
            double sum = 0.0;
            for (int i = a; i < b; ++i) sum += (double)S.diff[i];
            A.pieces[chunk + s] = sum;
        }
    }
    __syncthreads();
    for (int q = warp; q < min(S.listed, CHUNK / SHORT + 1); q += WARPS) {
        const int64_t s = R.s0 + S.list[q];
        const int a = R.within(start_of(A, s)), b = R.within(start_of(A, s + 1));
        double sum = 0.0;
        for (int i = a + lane; i < b; i += 32) sum += (double)S.diff[i];
        sum = join(sum);
        if (lane == 0) A.pieces[chunk + s] = sum;
    }
}

// l(x) and l'(x)
__device__ __forceinline__ float2 loss_of(const Args& A, float x) {
    if (A.kind == SSGD_PREFERENCE_IPO) {            // (x - 1/2)^2 / beta^2 = (h - 1 / (2 beta))^2 with x = beta h
        const float d = (x - 0.5f) / A.beta;
        return make_float2(d * d, 2.f * d / A.beta);
    }
    if (A.kind == SSGD_PREFERENCE_HINGE) return x < 1.f ? make_float2(1.f - x, -1.f) : x >= 1.f ? make_float2(0.f, 0.f) : make_float2(x, x);
    const float e = expf(-fabsf(x)), soft = log1pf(e);
    const float lose = x >= 0.f ? e / (1.f + e) : 1.f / (1.f + e);              // sigmoid(-x)
    float loss = (1.f - A.smoothing) * (fmaxf(-x, 0.f) + soft);
    if (A.smoothing > 0.f) loss += A.smoothing * (fmaxf(x, 0.f) + soft);
    return make_float2(x != x ? x : loss, A.smoothing - lose);
}

// Number of pieces of tokens [a, b), and the first one's CTA
__device__ __forceinline__ int64_t pieces_of(int64_t a, int64_t b, int64_t* first) {
    *first = a / CHUNK;
    return b > a ? (b - 1) / CHUNK - *first + 1 : 0;
}

// Of one pair: sums -> loss, rewards, gradients
struct Outcome { float d0, d1; };
__device__ __forceinline__ Outcome pair_outcome(const Args& A, int64_t p, double D0, double D1, int64_t n0, int64_t n1, bool write) {
    double f0 = 1.0, f1 = 1.0;
    if (A.average) { f0 = n0 > 0 ? 1.0 / (double)n0 : 0.0; f1 = n1 > 0 ? 1.0 / (double)n1 : 0.0; }
    const double r0 = (double)A.beta * (D0 * f0), r1 = (double)A.beta * (D1 * f1);
    const float2 l = loss_of(A, (float)(r0 - r1));
    const float w = A.weights ? A.weights[p] : 1.f;
    if (write) {
        A.loss[p] = w == 0.f ? 0.f : w * l.x;
        A.rewards[p] = (float)r0;
        A.rewards[A.pairs + p] = (float)r1;
    }
    const float slope = w == 0.f ? 0.f : w * A.beta * l.y;
    return Outcome{A.average ? (float)((double)slope * f0) : slope, A.average ? (float)(-(double)slope * f1) : -slope};
}

__device__ __forceinline__ void finish(const Args& A, Shared& S, const Range& R, bool last) {
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const bool few = R.s1 - R.s0 <= FEW;
    const int n = few ? (int)(R.s1 - R.s0) : 0;
    if (few) {
        if (t <= n) S.bound[t] = R.within(start_of(A, R.s0 + t));
    } else {
        // a sequence's gradient stands where it begins in this CTA
        for (int i = t; i < CHUNK; i += THREADS) S.diff[i] = __int_as_float(NO_MARK);
        __syncthreads();
    }
    // of sequence s, which is tokens [a, b)
    auto put = [&](int64_t s, int64_t a, int64_t b, float v) {
        if (few) {
            if (s >= R.s0 && s < R.s1) S.value[s - R.s0] = v;
        } else {
            const int i = R.within(a), j = R.within(b);
            if (i < j) S.diff[i] = v;
        }
    };
    auto pair_of = [&](int64_t p, int64_t (&at)[3]) {
#pragma unroll
        for (int q = 0; q < 3; ++q) at[q] = start_of(A, 2 * p + q);
    };
    auto settle = [&](int64_t p, const int64_t (&at)[3], double D0, double D1) {
        // by the CTA in which the pair begins
        const bool write = (at[0] >= R.c0 && at[0] < R.c1) || (last && at[0] >= R.c1);
        const Outcome g = pair_outcome(A, p, D0, D1, at[1] - at[0], at[2] - at[1], write);
        put(2 * p, at[0], at[1], g.d0);
        put(2 * p + 1, at[1], at[2], g.d1);
    };
    const int64_t p0 = R.s0 / 2, p1 = (R.s1 + 1) / 2;
    // Pairs of more pieces than one to a sequence have tokens in other CTAs too: they are the first or the last of this one.  A warp joins
    // one, or all warps where the pieces are many.
    for (int side = 0; side < 2; ++side) {
        const int64_t p = side ? p1 - 1 : p0;
        if (p >= p1 || (side && p == p0)) break;    // the same for the whole CTA
        int64_t at[3], k[2];
        pair_of(p, at);
        const int64_t n0 = pieces_of(at[0], at[1], &k[0]), n1 = pieces_of(at[1], at[2], &k[1]);
        const bool many = n0 + n1 > LONG;           // the same in every CTA: the order of the sum is
        if (!many && warp != side) continue;
        const int stride = many ? THREADS : 32, first = many ? t : lane;
        double D[2] = {0.0, 0.0};
        for (int64_t i = first; i < n0; i += stride) D[0] += A.pieces[k[0] + i + 2 * p];
        for (int64_t i = first; i < n1; i += stride) D[1] += A.pieces[k[1] + i + 2 * p + 1];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) D[q] += __shfl_xor_sync(0xffffffffu, D[q], o);
        }
        if (many) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                __syncthreads();
                if (lane == 0) S.joined[warp] = D[q];
                __syncthreads();
                D[q] = 0.0;
                for (int w = 0; w < WARPS; ++w) D[q] += S.joined[w];
            }
        }
        if (many ? t == 0 : lane == 0) settle(p, at, D[0], D[1]);
    }
    // the others lie within the CTA: one piece per sequence
    for (int64_t p = p0 + 1 + (t ^ 64); p < p1 - 1; p += THREADS) {            // beginning with warps that join nothing
        int64_t at[3];
        pair_of(p, at);
        settle(p, at, at[1] > at[0] ? A.pieces[at[0] / CHUNK + 2 * p] : 0.0, at[2] > at[1] ? A.pieces[at[1] / CHUNK + 2 * p + 1] : 0.0);
    }
    if (!A.d_logp) return;
    const int tokens = (int)(R.c1 - R.c0);
    float* out = A.d_logp + R.c0;
    if (few) {
        __syncthreads();
        const int begin = n ? S.bound[0] : tokens, end = n ? S.bound[n] : tokens;
        for (int i = t; i < begin; i += THREADS) out[i] = 0.f;                 // tokens of no sequence
        for (int q = 0; q < n; ++q) {
            const float v = S.value[q];
            for (int i = S.bound[q] + t; i < S.bound[q + 1]; i += THREADS) out[i] = v;
        }
        for (int i = end + t; i < tokens; i += THREADS) out[i] = 0.f;
        return;
    }
    if (t == 0) {
        const int end = R.within(start_of(A, 2 * A.pairs));
        if (end < tokens) S.diff[end] = 0.f;
    }
    __syncthreads();
    // every token takes the last mark at or before it
    float v[EACH];
    float mine = __int_as_float(NO_MARK);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        v[i] = S.diff[t * EACH + i];
        if (__float_as_int(v[i]) != NO_MARK) mine = v[i];
    }
    // the last mark of the threads before this one
    const uint32_t votes = __ballot_sync(0xffffffffu, __float_as_int(mine) != NO_MARK);
    const float of_warp = __shfl_sync(0xffffffffu, mine, votes ? 31 - __clz((int)votes) : 0);
    if (lane == 0) S.last[warp] = __float_as_int(of_warp);
    __syncthreads();
    float carry = 0.f;
    for (int w = 0; w < warp; ++w)
        if (S.last[w] != NO_MARK) carry = __int_as_float(S.last[w]);
    const uint32_t below = votes & ((1u << lane) - 1u);
    const float of_lane = __shfl_sync(0xffffffffu, mine, below ? 31 - __clz((int)below) : 0);
    if (below) carry = of_lane;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (__float_as_int(v[i]) != NO_MARK) carry = v[i];
        S.diff[t * EACH + i] = carry;
    }
    __syncthreads();
    for (int i = t; i < tokens; i += THREADS) out[i] = S.diff[i];
}

enum Part { SUMS, FINISH, ALL };

template <Part PART>
__global__ void __launch_bounds__(THREADS) k_preference(const Args A) {
    __shared__ Shared S;
    const int64_t chunk = blockIdx.x;
    const bool last = blockIdx.x + 1 == gridDim.x;
    successor_may_start();
    if (PART != FINISH) load_tokens(A, S, chunk * CHUNK);
    Range R;
    if (PART == FINISH) {
        successor_wait();
        R = Range{chunk * CHUNK, min((chunk + 1) * CHUNK, A.tokens), A.ranges[2 * chunk], A.ranges[2 * chunk + 1]};
    } else {
        R = range_of(A, chunk, last);
        if (PART == SUMS && threadIdx.x == 0) {
            A.ranges[2 * chunk] = R.s0;
            A.ranges[2 * chunk + 1] = R.s1;
        }
        sum_pieces(A, S, chunk, R);
    }
    if (PART == ALL) __syncthreads();
    if (PART != SUMS) finish(A, S, R, last);
}

constexpr int64_t MAX_TOKENS = (int64_t)1 << 40, MAX_PAIRS = (int64_t)1 << 30;
int64_t chunks_of(int64_t tokens) { return tokens ? (tokens + CHUNK - 1) / CHUNK : 1; }

}  // namespace

extern "C" {

int ssgd_preference_loss_workspace(int64_t tokens, int64_t pairs, size_t* out_bytes) {
    if (!out_bytes || tokens < 0 || tokens > MAX_TOKENS || pairs < 0 || pairs > MAX_PAIRS) return SSGD_EINVAL;
    *out_bytes = (size_t)(3 * chunks_of(tokens) + 2 * pairs) * 8;
    return SSGD_OK;
}

int ssgd_preference_loss(const float* logp, const float* ref_logp, int64_t tokens, const void* starts, int32_t starts_bytes, int64_t pairs,
                         const float* weights, int32_t kind, float beta, float label_smoothing, int32_t average, float* loss,
                         float* rewards, float* d_logp, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    if (int e = ssgd_preference_loss_workspace(tokens, pairs, &need)) return e;
    if (starts_bytes != 4 && starts_bytes != 8) return SSGD_EINVAL;
    if (kind != SSGD_PREFERENCE_SIGMOID && kind != SSGD_PREFERENCE_IPO && kind != SSGD_PREFERENCE_HINGE) return SSGD_EINVAL;
    if (!(beta > 0.f) || !(beta < INFINITY) || !(label_smoothing >= 0.f) || !(label_smoothing <= 0.5f)) return SSGD_EINVAL;
    if (label_smoothing != 0.f && kind != SSGD_PREFERENCE_SIGMOID) return SSGD_EINVAL;
    if (tokens == 0 && pairs == 0) return SSGD_OK;
    if (!starts || (tokens && !logp) || (pairs && (!loss || !rewards))) return SSGD_EINVAL;
    if (!aligned_to(logp, 4) || !aligned_to(ref_logp, 4) || !aligned_to(starts, starts_bytes) || !aligned_to(weights, 4) ||
        !aligned_to(loss, 4) || !aligned_to(rewards, 4) || !aligned_to(d_logp, 4))
        return SSGD_EALIGN;
    if (!workspace || workspace_bytes < need) return SSGD_EWORKSPACE;
    if (!aligned_to(workspace, 8)) return SSGD_EALIGN;
    double* pieces = static_cast<double*>(workspace);
    int64_t* ranges = reinterpret_cast<int64_t*>(pieces + chunks_of(tokens) + 2 * pairs);
    const Args A{logp, ref_logp, starts, starts_bytes == 8, weights, tokens, pairs, beta, label_smoothing, kind, average != 0, loss, rewards,
                 d_logp, pieces, ranges, aligned_to(logp, 16) && aligned_to(ref_logp, 16)};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t chunks = chunks_of(tokens);
    if (chunks > 0x7fffffff) return SSGD_ETOOBIG;
    if (chunks == 1) {
        k_preference<ALL><<<1, THREADS, 0, st>>>(A);
        return launched();
    }
    k_preference<SUMS><<<(unsigned)chunks, THREADS, 0, st>>>(A);
    if (int e = launched()) return e;
    return launch_after(st, k_preference<FINISH>, dim3((unsigned)chunks), THREADS, A);
}

}  // extern "C"
