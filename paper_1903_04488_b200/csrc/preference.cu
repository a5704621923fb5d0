// preference.cu -- the preference loss of pairs of token sequences, and its gradient (ssgd_preference_loss).
//
// Sequence s is tokens [starts[s], starts[s + 1]); pair p is sequences 2 p (preferred) and 2 p + 1.
//   D_s = sum of (logp - ref)  (over its length, with `average`),  x = beta (D_2p - D_2p+1)
//   loss = w l(x),  d_logp of a token of sequence s = +-w beta l'(x)  (over the length, with `average`)
// What bounds it is memory: 8 bytes read and 4 written per token, and every token of a sequence has the same gradient, so nothing is
// read twice.  Lengths are known on the device alone and may be anything, so the work is cut by tokens, 8192 to a CTA, and not by
// pairs: the first launch leaves the sum of every piece of a sequence (a CTA's tokens that belong to it), the second joins the pieces
// of its pairs, each CTA for itself and all in the same order, and writes.  The piece of sequence s in CTA k has place k + s: between
// two pieces that follow one another either grows by one, so no two share a place, and there are CTAs + sequences places.
// A call of one CTA does both in one launch.  Measured: 12,000,000 tokens in 4099 pairs 42 us (3.4 TB/s;
// 27 for the sums, where an SM has three CTAs that load and add by turns, 16 for the rest), 262144 tokens 12 us, 2000 tokens 8 us.  What the
// differences logp - ref lose is 2 of the 27: with differences rounded to 24 bits both launches took 40.
#include <cstddef>

#include "formats.cuh"

using namespace ssgd;

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int EACH = 32;                            // tokens of a thread
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
    bool vector;                                    // logp and ref are 16-byte aligned
    double per_token;                               // starts to a token
};

constexpr int FEW = 64;                             // sequences of a CTA that are gone through one by one
constexpr int SHORT = 32;                           // where there are more, pieces below it are summed by one thread, others by a warp
constexpr int LONG = 256;                           // pieces of a pair that the whole CTA joins
constexpr int32_t NO_MARK = 0x7fa12345;             // the bits of a NaN that no operation makes
struct Shared {
    alignas(16) float logp[CHUNK];                  // then the gradients
    int64_t start[FEW + 1];                         // where the sequences begin
    int32_t bound[FEW + 1];                         // the same within the CTA's tokens
    float value[FEW];                               // their gradients
    union {
        double part[WARPS][FEW];
        int32_t list[CHUNK / SHORT + 1];
    };
    int2 before[WARPS];
    int32_t listed;
    int32_t last[WARPS];
    double joined[WARPS];
    alignas(16) float ref[CHUNK];                   // (not there in the second launch)
};
// Where token i's mark stands while each thread goes through EACH tokens that follow one another: the threads of a warp meet no bank twice
// (12M tokens in 200,000 pairs took 86 us with it and 103 without).
__device__ __forceinline__ int place_of(int i) {
    static_assert(EACH == 32, "a row of all banks to a thread");
    return i ^ (i >> 5 & 31);
}
constexpr int LOOK = 4, WINDOW = LOOK * THREADS;

// I: what counts tokens and sequences, 32 bits where they suffice.  Half of the instructions are such counting.
template <typename I> struct Work {
    // starts[s], kept within the tokens
    static __device__ __forceinline__ I start_of(const Args& A, I s) {
        if (A.starts64) {
            const long long v = static_cast<const long long*>(A.starts)[s];
            return (I)(v < 0 ? 0 : v > A.tokens ? A.tokens : v);
        }
        return min(max((I)static_cast<const int32_t*>(A.starts)[s], (I)0), (I)A.tokens);
    }

    // Tokens of the CTA, and the sequences that may have some of them, in whole pairs: from the last one that starts before the first token to
    // the last one that starts before the end.  The last CTA has those too that start at the end.
    struct Range {
        I c0, c1, s0, s1;
        __device__ __forceinline__ bool few() const { return s1 - s0 <= FEW; }
        __device__ __forceinline__ int within(I token) const { return (int)((token < c0 ? c0 : token > c1 ? c1 : token) - c0); }
    };

    // The CTA's range, and the starts of its sequences in shared memory where they are few.  What is looked for are the first starts that
    // are at least c0 and at least c1.  Lengths that are not too unlike put them near chunk / chunks of the way, so the whole CTA looks at
    // 1024 starts there; where they are not among them, it searches, 256 places at a time.
    struct Window {
        I w0, v[LOOK];                            // the thread's starts w0 + t + i THREADS
        __device__ __forceinline__ void load(const Args& A, I chunk) {
            const I n = 2 * (I)A.pairs + 1;
            w0 = max(min((I)((double)(chunk * CHUNK + CHUNK / 2) * A.per_token) - WINDOW / 2, n - WINDOW), (I)0);
#pragma unroll
            for (int i = 0; i < LOOK; ++i) {
                const I at = w0 + threadIdx.x + i * THREADS;
                v[i] = at < n ? start_of(A, at) : (I)(sizeof(I) == 4 ? (long long)INT32_MAX : (long long)INT64_MAX);
            }
        }
        __device__ __forceinline__ Range range(const Args& A, Shared& S, I chunk, I chunks) const {
            const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
            const bool last = chunk + 1 == chunks;
            Range R;
            R.c0 = chunk * CHUNK;
            R.c1 = min(R.c0 + CHUNK, (I)A.tokens);
            const I n = 2 * (I)A.pairs + 1;
            int k0 = 0, k1 = 0;
#pragma unroll
            for (int i = 0; i < LOOK; ++i) {
                k0 += __popc(__ballot_sync(0xffffffffu, v[i] < R.c0));
                k1 += __popc(__ballot_sync(0xffffffffu, v[i] < R.c1));
            }
            if (lane == 0) S.before[warp] = make_int2(k0, k1);
            __syncthreads();
            k0 = k1 = 0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                k0 += S.before[w].x;
                k1 += S.before[w].y;
            }
            I lo[2] = {w0 + k0, w0 + k1};
            const bool found = (k0 >= 2 || w0 == 0) && (k1 <= WINDOW - 2 || w0 + WINDOW >= n);     // with the starts of whole pairs around them
            if (!found) {
                lo[0] = lo[1] = 0;
                I hi[2] = {n, n};
                while (lo[0] < hi[0] || lo[1] < hi[1]) {
                    bool below[2];
                    I step[2];
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        step[q] = (hi[q] - lo[q] + THREADS - 1) / THREADS;
                        const I probe = lo[q] + (I)t * step[q];
                        below[q] = probe < hi[q] && start_of(A, probe) < (q ? R.c1 : R.c0);
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int k = __syncthreads_count(below[q]);               // places lo, lo + step, .. that are before the answer
                        if (lo[q] >= hi[q]) continue;
                        const I from = k ? lo[q] + (I)(k - 1) * step[q] + 1 : lo[q];
                        hi[q] = k ? min(hi[q], lo[q] + (I)k * step[q]) : lo[q];
                        lo[q] = from;
                    }
                }
            }
            R.s0 = min(max(lo[0] - 1, (I)0) & ~(I)1, 2 * (I)A.pairs);
            R.s1 = last ? 2 * (I)A.pairs : min((lo[1] + 1) & ~(I)1, 2 * (I)A.pairs);
            if (R.s1 < R.s0) R.s1 = R.s0;               // starts that do not ascend
            if (R.few()) {
                const int count = (int)(R.s1 - R.s0);
                auto keep = [&](int i, I start) {
                    S.start[i] = start;
                    S.bound[i] = R.within(start);
                };
                if (found && R.s0 >= w0 && R.s1 < w0 + WINDOW) {
#pragma unroll
                    for (int i = 0; i < LOOK; ++i) {
                        const I at = w0 + t + i * THREADS - R.s0;
                        if (at >= 0 && at <= count) keep((int)at, v[i]);
                    }
                } else if (t <= count) {
                    keep(t, start_of(A, R.s0 + t));
                }
            }
            return R;
        }
    };

    // A sum with what its roundings lost beside it: 48 bits or more, in fp32 arithmetic (an SM converts to 64 bits at 16 numbers a cycle).  The
    // range is that of fp32: two masks of the lowest number leave it, and what they lost is NaN then.  Such a piece, and one that holds
    // infinities or NaN, is not `sound` and is added up once more in 64 bits.
    struct Sum {
        float sum = 0.f, lost = 0.f;
        __device__ __forceinline__ void add(float x) {
            const float next = sum + x, back = next - sum;
            lost += (sum - (next - back)) + (x - back);
            sum = next;
        }
        // a - b, with what the difference loses
        __device__ __forceinline__ void add_difference(float a, float b) {
            const float d = a - b, back = d - a;
            lost += (a - (d - back)) - (b + back);
            add(d);
        }
        __device__ __forceinline__ void join_warp() {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const float x = __shfl_xor_sync(0xffffffffu, sum, o), l = __shfl_xor_sync(0xffffffffu, lost, o);
                add(x);
                lost += l;
            }
        }
        __device__ __forceinline__ bool sound() const { return fabsf(sum) < INFINITY && fabsf(lost) < INFINITY; }
        __device__ __forceinline__ double value() const { return (double)sum + (double)lost; }
    };

    // A piece's sum from those of the warps
    static __device__ __forceinline__ double sum_of_warps(const Shared& S, int q) {
        double sum = 0.0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) sum += S.part[w][q];
        return sum;
    }

    // Every warp has an eighth of the CTA's tokens: calls f(q, a, b) for each of the n sequences that has some of them, [a, b)
    template <typename F>
    static __device__ __forceinline__ void for_pieces(const Shared& S, int n, int tokens, F f) {
        const int lane = threadIdx.x & 31, span = (tokens + WARPS - 1) / WARPS, begin = ((int)threadIdx.x >> 5) * span, end = begin + span;
        for (int base = 0; base < n; base += 32) {
            const int q = base + lane;
            int a = 0, b = 0;
            if (q < n) {
                a = max(S.bound[q], begin);
                b = min(S.bound[q + 1], end);
            }
            for (uint32_t todo = __ballot_sync(0xffffffffu, a < b); todo; todo &= todo - 1) {
                const int src = __ffs(todo) - 1;
                f(base + src, __shfl_sync(0xffffffffu, a, src), __shfl_sync(0xffffffffu, b, src));
            }
        }
    }

    // The CTA's tokens on their way to shared memory while it looks for its sequences, 16 bytes at once where they may be
    static __device__ __forceinline__ void start_tokens(const Args& A, Shared& S, I c0) {
        const int left = (int)min((I)A.tokens - c0, (I)CHUNK);
        auto some = [&](int at, auto bytes) {
            copy_async<decltype(bytes)::value>(S.logp + at, A.logp + c0 + at);
            if (A.ref) copy_async<decltype(bytes)::value>(S.ref + at, A.ref + c0 + at);
        };
        const int whole = A.vector ? left & ~3 : 0;
        for (int at = (int)threadIdx.x * 4; at < whole; at += THREADS * 4) some(at, std::integral_constant<int, 16>{});
        for (int at = whole + (int)threadIdx.x; at < left; at += THREADS) some(at, std::integral_constant<int, 4>{});
        copy_async_commit();
    }
    static __device__ __forceinline__ void add_token(const Args& A, const Shared& S, int i, Sum& sum) {
        if (A.ref) sum.add_difference(S.logp[i], S.ref[i]);
        else sum.add(S.logp[i]);
    }
    // Tokens [a, b), every `stride`-th from `first` on, in 64 bits
    static __device__ __forceinline__ double wide_sum(const Args& A, const Shared& S, int a, int b, int first, int stride) {
        double sum = 0.0;
        for (int i = a + first; i < b; i += stride) sum += A.ref ? (double)S.logp[i] - (double)S.ref[i] : (double)S.logp[i];
        return sum;
    }
    // The sum of [a, b), of which every lane of the warp has some: the same answer in all lanes
    static __device__ __forceinline__ double joined(const Args& A, const Shared& S, int a, int b, Sum sum) {
        sum.join_warp();
        if (__all_sync(0xffffffffu, sum.sound())) return sum.value();
        double wide = wide_sum(A, S, a, b, threadIdx.x & 31, 32);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) wide += __shfl_xor_sync(0xffffffffu, wide, o);
        return wide;
    }

    // Sums of the pieces of the CTA's tokens, of 48 bits or more.  Each is added up by itself, so that what one sequence holds (infinities,
    // the lowest number of a mask) stays there.  WRITE: for other CTAs; otherwise those of few sequences are left in S.part alone.
    template <bool WRITE>
    static __device__ __forceinline__ void sum_pieces(const Args& A, Shared& S, I chunk, const Range& R) {
        const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
        if (R.few()) {                                  // every warp takes an eighth of the tokens
            const int n = (int)(R.s1 - R.s0);
            for (int i = lane; i < n; i += 32) S.part[warp][i] = 0.0;
            __syncwarp();
            for_pieces(S, n, (int)(R.c1 - R.c0), [&](int q, int a, int b) {
                // pairs of tokens, and what is left of them at the ends
                const int a2 = (a + 1) & ~1, b2 = b & ~1;
                float2 two = both(0.f), off = both(0.f);
#pragma unroll 4
                for (int i = a2 + 2 * lane; i < b2; i += 64) {
                    float2 x = *reinterpret_cast<const float2*>(S.logp + i);
                    if (A.ref) {
                        const float2 r = *reinterpret_cast<const float2*>(S.ref + i), d = fma2(r, both(-1.f), x), back = fma2(x, both(-1.f), d);
                        off = add2(off, fma2(add2(r, back), both(-1.f), fma2(fma2(back, both(-1.f), d), both(-1.f), x)));
                        x = d;
                    }
                    const float2 next = add2(two, x), back = fma2(two, both(-1.f), next);
                    off = add2(off, add2(fma2(fma2(back, both(-1.f), next), both(-1.f), two), fma2(back, both(-1.f), x)));
                    two = next;
                }
                Sum sum;
                sum.add(two.x);
                sum.add(two.y);
                sum.lost += off.x + off.y;
                if (lane == 0 && a < a2) add_token(A, S, a, sum);
                if (lane == 1 && b2 < b && b2 >= a) add_token(A, S, b2, sum);
                const double all = joined(A, S, a, b, sum);
                if (lane == 0) S.part[warp][q] = all;
            });
            __syncthreads();
            if (WRITE && t < n && S.bound[t] < S.bound[t + 1]) A.pieces[chunk + R.s0 + t] = sum_of_warps(S, t);
            return;
        }
        for (I s = R.s0 + t; s < R.s1; s += THREADS) {
            const int a = R.within(start_of(A, s)), b = R.within(start_of(A, s + 1));
            if (b - a >= SHORT) {
                const int at = atomicAdd(&S.listed, 1);
                if (at <= CHUNK / SHORT) S.list[at] = (int32_t)(s - R.s0);         // more only where starts do not ascend
            } else if (b > a) {
                Sum sum;
                for (int i = a; i < b; ++i) add_token(A, S, i, sum);
                A.pieces[chunk + s] = sum.sound() ? sum.value() : wide_sum(A, S, a, b, 0, 1);
            }
        }
        __syncthreads();
        for (int q = warp; q < min(S.listed, CHUNK / SHORT + 1); q += WARPS) {
            const I s = R.s0 + S.list[q];
            const int a = R.within(start_of(A, s)), b = R.within(start_of(A, s + 1));
            Sum sum;
            for (int i = a + lane; i < b; i += 32) add_token(A, S, i, sum);
            const double all = joined(A, S, a, b, sum);
            if (lane == 0) A.pieces[chunk + s] = all;
        }
    }

    // l(x) and l'(x)
    static __device__ __forceinline__ float2 loss_of(const Args& A, float x) {
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
    static __device__ __forceinline__ I pieces_of(I a, I b, I* first) {
        *first = a / CHUNK;
        return b > a ? (b - 1) / CHUNK - *first + 1 : 0;
    }

    // Of one pair: sums -> loss, rewards, gradients
    struct Outcome { float d0, d1; };
    static __device__ __forceinline__ Outcome pair_outcome(const Args& A, I p, float w, double D0, double D1, I n0, I n1, bool write) {
        double f0 = 1.0, f1 = 1.0;
        if (A.average) { f0 = n0 > 0 ? 1.0 / (double)n0 : 0.0; f1 = n1 > 0 ? 1.0 / (double)n1 : 0.0; }
        const double r0 = (double)A.beta * (D0 * f0), r1 = (double)A.beta * (D1 * f1);
        const float2 l = loss_of(A, (float)(r0 - r1));
        if (write) {
            A.loss[p] = w == 0.f ? 0.f : w * l.x;
            A.rewards[p] = (float)r0;
            A.rewards[A.pairs + p] = (float)r1;
        }
        const float slope = w == 0.f ? 0.f : w * A.beta * l.y;
        return Outcome{A.average ? (float)((double)slope * f0) : slope, A.average ? (float)(-(double)slope * f1) : -slope};
    }

    // ALONE: there is no other CTA
    template <bool ALONE>
    static __device__ __forceinline__ void finish(const Args& A, Shared& S, const Range& R, bool last) {
        const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
        const bool few = R.few();
        const int n = few ? (int)(R.s1 - R.s0) : 0;
        if (!few) {
            // a sequence's gradient stands where it begins in this CTA
            for (int i = t; i < CHUNK; i += THREADS) S.logp[i] = __int_as_float(NO_MARK);
            __syncthreads();
        }
        // of sequence s, which is tokens [a, b)
        auto put = [&](I s, I a, I b, float v) {
            if (few) {
                S.value[s - R.s0] = v;
            } else {
                const int i = R.within(a), j = R.within(b);
                if (i < j) S.logp[place_of(i)] = v;
            }
        };
        auto pair_of = [&](I p, I (&at)[3]) {
#pragma unroll
            for (int q = 0; q < 3; ++q) at[q] = few ? S.start[2 * p + q - R.s0] : start_of(A, 2 * p + q);
        };
        auto settle = [&](I p, const I (&at)[3], float w, double D0, double D1) {
            // by the CTA in which the pair begins
            const bool write = (at[0] >= R.c0 && at[0] < R.c1) || (last && at[0] >= R.c1);
            const Outcome g = pair_outcome(A, p, w, D0, D1, at[1] - at[0], at[2] - at[1], write);
            put(2 * p, at[0], at[1], g.d0);
            put(2 * p + 1, at[1], at[2], g.d1);
        };
        auto weight_of = [&](I p) { return A.weights ? A.weights[p] : 1.f; };
        const I p0 = R.s0 / 2, p1 = R.s1 / 2;
        if (ALONE && few) {
            if (p0 + t < p1) {
                I at[3];
                pair_of(p0 + t, at);
                settle(p0 + t, at, weight_of(p0 + t), sum_of_warps(S, 2 * t), sum_of_warps(S, 2 * t + 1));
            }
        } else {
            // Pairs of more pieces than one to a sequence have tokens in other CTAs too: they are the first or the last of this one.  A warp
            // joins one, or all warps where the pieces are many.
            for (int side = 0; side < 2; ++side) {
                const I p = side ? p1 - 1 : p0;
                if (p >= p1 || (side && p == p0)) break;    // the same for the whole CTA
                I at[3], k[2];
                pair_of(p, at);
                const I n0 = pieces_of(at[0], at[1], &k[0]), n1 = pieces_of(at[1], at[2], &k[1]);
                const bool many = n0 + n1 > LONG;           // the same in every CTA: the order of the sum is
                if (!many && warp != side) continue;
                const int stride = many ? THREADS : 32, first = many ? t : lane;
                const float w = weight_of(p);
                double D[2] = {0.0, 0.0};
                if (n0 <= 4 && n1 <= 4) {                   // the usual case: one lane adds them up
                    if (lane != 0) continue;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (i < n0) D[0] += A.pieces[k[0] + i + 2 * p];
                        if (i < n1) D[1] += A.pieces[k[1] + i + 2 * p + 1];
                    }
                    settle(p, at, w, D[0], D[1]);
                    continue;
                }
                for (I i = first; i < n0; i += stride) D[0] += A.pieces[k[0] + i + 2 * p];
                for (I i = first; i < n1; i += stride) D[1] += A.pieces[k[1] + i + 2 * p + 1];
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
                        for (int i = 0; i < WARPS; ++i) D[q] += S.joined[i];
                    }
                }
                if (many ? t == 0 : lane == 0) settle(p, at, w, D[0], D[1]);
            }
            // the others lie within the CTA: one piece per sequence
            for (I p = p0 + 1 + (t ^ 64); p < p1 - 1; p += THREADS) {        // beginning with warps that join nothing
                I at[3];
                pair_of(p, at);
                settle(p, at, weight_of(p), at[1] > at[0] ? A.pieces[at[0] / CHUNK + 2 * p] : 0.0, at[2] > at[1] ? A.pieces[at[1] / CHUNK + 2 * p + 1] : 0.0);
            }
        }
        if (!A.d_logp) return;
        const int tokens = (int)(R.c1 - R.c0);
        float* out = A.d_logp + R.c0;
        if (few) {
            __syncthreads();
            const int begin = n ? S.bound[0] : tokens, end = n ? S.bound[n] : tokens;
            for (int i = t; i < begin; i += THREADS) out[i] = 0.f;                 // tokens of no sequence
            for_pieces(S, n, (int)(R.c1 - R.c0), [&](int q, int a, int b) {
                const float v = S.value[q];
                for (int i = a + lane; i < b; i += 32) out[i] = v;
            });
            for (int i = end + t; i < tokens; i += THREADS) out[i] = 0.f;
            return;
        }
        if (t == 0) {
            const int end = R.within(start_of(A, 2 * (I)A.pairs));
            if (end < tokens) S.logp[place_of(end)] = 0.f;
        }
        __syncthreads();
        // every token takes the last mark at or before it
        float mine = __int_as_float(NO_MARK);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float v = S.logp[place_of(t * EACH + i)];
            if (__float_as_int(v) != NO_MARK) mine = v;
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
            float& v = S.logp[place_of(t * EACH + i)];
            if (__float_as_int(v) != NO_MARK) carry = v;
            v = carry;
        }
        __syncthreads();
        for (int i = t; i < tokens; i += THREADS) out[i] = S.logp[place_of(i)];
    }
};

enum Part { SUMS, FINISH, ALL };

template <Part PART, typename I>
// The second launch waits for starts, pieces and weights one after the other and has the shared memory for 5 CTAs to an SM: 12M
// tokens in 4099 pairs 1.3 us less than with 4, in 4M pairs 12 less.  A sixth gains nothing.
__global__ void __launch_bounds__(THREADS, PART == FINISH ? 5 : 4) k_preference(const Args A) {
    extern __shared__ __align__(16) uint8_t raw[];
    Shared& S = *reinterpret_cast<Shared*>(raw);
    using W = Work<I>;
    const I chunk = blockIdx.x;
    const bool last = blockIdx.x + 1 == gridDim.x;
    typename W::Window window;
    if constexpr (PART == FINISH) {
        window.load(A, chunk);
        const typename W::Range R = window.range(A, S, chunk, gridDim.x);     // what the caller gave need not wait for the sums
        successor_wait();
        __syncthreads();
        W::template finish<false>(A, S, R, last);
    } else {
        successor_may_start();
        window.load(A, chunk);
        W::start_tokens(A, S, chunk * CHUNK);
        const typename W::Range R = window.range(A, S, chunk, gridDim.x);
        if (threadIdx.x == 0) S.listed = 0;
        copy_async_wait<0>();
        __syncthreads();
        W::template sum_pieces<PART == SUMS>(A, S, chunk, R);
        if constexpr (PART == ALL) {
            __syncthreads();
            W::template finish<true>(A, S, R, last);
        }
    }
}

template <Part PART, typename I>
int launch_part(const Args& A, int64_t chunks, cudaStream_t st) {
    constexpr int smem = PART == FINISH ? (int)offsetof(Shared, ref) : (int)sizeof(Shared);
    static PerDevice known;
    int fits = 0;
    if (int e = residency(k_preference<PART, I>, THREADS, smem, known, &fits)) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)chunks);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = PART == FINISH ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k_preference<PART, I>, A) == cudaSuccess ? SSGD_OK : SSGD_ECUDA;
}
template <typename I>
int launch_all(const Args& A, int64_t chunks, cudaStream_t st) {
    if (chunks == 1) return launch_part<ALL, I>(A, chunks, st);
    if (int e = launch_part<SUMS, I>(A, chunks, st)) return e;
    return launch_part<FINISH, I>(A, chunks, st);
}

constexpr int64_t MAX_TOKENS = (int64_t)1 << 40, MAX_PAIRS = (int64_t)1 << 30;
int64_t chunks_of(int64_t tokens) { return tokens ? (tokens + CHUNK - 1) / CHUNK : 1; }

}  // namespace

extern "C" {

int ssgd_preference_loss_workspace(int64_t tokens, int64_t pairs, size_t* out_bytes) {
    if (!out_bytes || tokens < 0 || tokens > MAX_TOKENS || pairs < 0 || pairs > MAX_PAIRS) return SSGD_EINVAL;
    *out_bytes = (size_t)(chunks_of(tokens) + 2 * pairs) * sizeof(double);
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
    const int64_t chunks = chunks_of(tokens);
    const Args A{logp, ref_logp, starts, starts_bytes == 8, weights, tokens, pairs, beta, label_smoothing, kind, average != 0, loss, rewards,
                 d_logp, static_cast<double*>(workspace), aligned_to(logp, 16) && aligned_to(ref_logp, 16),
                 tokens ? (double)(2 * pairs + 1) / (double)tokens : 0.0};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (chunks > 0x7fffffff) return SSGD_ETOOBIG;
    return tokens < (int64_t)1 << 30 && pairs < (int64_t)1 << 28 ? launch_all<int32_t>(A, chunks, st) : launch_all<int64_t>(A, chunks, st);
}

}  // extern "C"
