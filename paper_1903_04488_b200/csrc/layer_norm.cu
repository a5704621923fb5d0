// layer_norm.cu -- layer norm over the last dimension, forward and backward (ssgd_layer_norm, ssgd_layer_norm_backward).
//
//   forward    mean = 1/n sum x,  rstd = (1/n sum (x - mean)^2 + eps)^-1/2,  y = (x - mean) rstd w + b
//   backward   h = (x - mean) rstd,  a = dy w
//              dx = rstd (a - 1/n sum a - h 1/n sum a h),   dw = sum over rows of dy h,   db = sum over rows of dy
//
// Both are bound by HBM: two streams of rows x n elements forward, three backward, a dozen operations per element.
// So a row is read once and stays on the SM, in its own format, from the first sum to the result: the variance is the mean of
// squared deviations from the mean already known, not a difference of large sums.  What keeps the kernels from the
// memory's rate is the latency of a row's sums on their way through warps and block, and the instructions around them.
#include <algorithm>

#include <cooperative_groups.h>

#include "formats.cuh"

using namespace ssgd;
namespace cg = cooperative_groups;

namespace {

// A group of G threads owns a row; thread t of it holds the vectors t, t + G, ... of VEC elements, E elements in all.
// G = 32: 8 rows per block, sums by shuffles alone.  G > 32: one row per block.
template <int G> struct GroupShape {
    static constexpr int BLOCK = G < 256 && G == 32 ? 256 : G;
    static constexpr int ROWS = BLOCK / G;
    static constexpr int WARPS = G / 32;
};

// Sums of V values (a power of two up to 8) over the warp at once: in each of the first steps a lane hands half of its values
// to its partner and goes on with the other half.  Value i ends up in the lanes l with l / (32 / V) = i.
template <int V>
__device__ __forceinline__ float warp_sums(float (&v)[V]) {
    const int lane = threadIdx.x & 31;
    int o = 16;
#pragma unroll
    for (int half = V / 2; half > 0; half >>= 1, o >>= 1) {
        const bool upper = lane & o;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float keep = upper ? v[i + half] : v[i], give = upper ? v[i] : v[i + half];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    float x = v[0];
#pragma unroll
    for (; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Sum over the group, known to every thread of it.  `slot` [WARPS] is not used again before the next barrier but one.
template <int G>
__device__ __forceinline__ float group_sum(float x, float* slot) {
    x = warp_sum(x);
    if (G == 32) return x;
    constexpr int NW = GroupShape<G>::WARPS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) slot[warp] = x;
    __syncthreads();
    if constexpr (NW <= 8) {
        float s = slot[0];
#pragma unroll
        for (int i = 1; i < NW; ++i) s += slot[i];
        return s;
    } else {
        return warp_sum(lane < NW ? slot[lane] : 0.f);
    }
}

// sum / n by the product with 1 / n and what that leaves over: a mean that is a number of fp32 comes out as it is.  (The product alone
// can be a unit off, and of a row of one value x that unit, divided by the deviation it makes up, would be the result.)
__device__ __forceinline__ float mean_of(float sum, float n, float inv_n) {
    const float m = sum * inv_n, left = fmaf(-m, n, sum);
    return left == left ? fmaf(left, inv_n, m) : m;        // NaN: the sum is not finite
}

// w or b at column `col`, VEC of them, in fp32 or in the row's format
template <typename T, int VEC>
__device__ __forceinline__ void load_param(const void* w, bool w_f32, int col, float2 (&f)[PAIRS<VEC>]) {
    if (w_f32) {
        const float* p = static_cast<const float*>(w) + col;
        if constexpr (VEC == 8) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
            f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w);
            f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w);
        } else {
            unpack_pairs(load_vec<float, VEC>(p), f);
        }
    } else {
        unpack_pairs(load_vec<T, VEC>(static_cast<const T*>(w) + col), f);
    }
}

// y = (x - mean) rstd w + b of one vector
template <typename T, int VEC, typename A>
__device__ __forceinline__ Vec<T, VEC> normalised(const Vec<T, VEC>& v, const A& args, int col, float2 minus_mean, float2 rstd) {
    float2 f[PAIRS<VEC>], w[PAIRS<VEC>], b[PAIRS<VEC>];
    unpack_pairs(v, f);
#pragma unroll
    for (int i = 0; i < PAIRS<VEC>; ++i) f[i] = mul2(add2(f[i], minus_mean), rstd);
    if (args.w && args.b) {
        load_param<T, VEC>(args.w, args.w_f32, col, w);
        load_param<T, VEC>(args.b, args.w_f32, col, b);
#pragma unroll
        for (int i = 0; i < PAIRS<VEC>; ++i) f[i] = fma2(f[i], w[i], b[i]);
    } else if (args.w) {
        load_param<T, VEC>(args.w, args.w_f32, col, w);
#pragma unroll
        for (int i = 0; i < PAIRS<VEC>; ++i) f[i] = mul2(f[i], w[i]);
    } else if (args.b) {
        load_param<T, VEC>(args.b, args.w_f32, col, b);
#pragma unroll
        for (int i = 0; i < PAIRS<VEC>; ++i) f[i] = add2(f[i], b[i]);
    }
    return pack_pairs<T, VEC>(f);
}
// sum of a vector's elements, and of their squared deviations, added to s
template <typename T, int VEC>
__device__ __forceinline__ void add_sum(const Vec<T, VEC>& v, float2& s) {
    float2 f[PAIRS<VEC>];
    unpack_pairs(v, f);
#pragma unroll
    for (int i = 0; i < PAIRS<VEC>; ++i) s = add2(s, f[i]);
}
template <typename T, int VEC>
__device__ __forceinline__ void add_squares(const Vec<T, VEC>& v, float2 minus_mean, float2& q) {
    float2 f[PAIRS<VEC>];
    unpack_pairs(v, f);
#pragma unroll
    for (int i = 0; i < PAIRS<VEC>; ++i) {
        float2 d = add2(f[i], minus_mean);
        if (VEC == 1) d.y = 0.f;
        q = fma2(d, d, q);
    }
}

struct NormArgs {
    const void* x; int64_t ld_x;
    const void* w; const void* b; bool w_f32;
    int64_t rows; int32_t n; float eps;
    void* y; int64_t ld_y;
    float* stats;        // [2][rows]: mean, rstd
};

// FULL: every thread has E elements (n = G E), so no column needs a check.
// One row per group and block: for rows too long to keep w and b in registers beside them.
template <typename T, int VEC, int G, int E, bool FULL>
__global__ void __launch_bounds__(GroupShape<G>::BLOCK) k_layer_norm(const NormArgs A) {
    constexpr int NV = E / VEC;
    __shared__ float slot[2][32];
    const int t = threadIdx.x % G;
    const int64_t row = (int64_t)blockIdx.x * GroupShape<G>::ROWS + threadIdx.x / G;
    if (row >= A.rows) return;                         // a whole warp (G = 32) or nobody
    const T* x = static_cast<const T*>(A.x) + row * A.ld_x + t * VEC;
    const int nv = A.n / VEC;
    auto mine_here = [&](int j) { return FULL || t + j * G < nv; };
    Vec<T, VEC> v[NV];
    float2 s = both(0.f), q = both(0.f);
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (mine_here(j)) v[j] = load_vec_stream<T, VEC>(x + j * G * VEC);
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (mine_here(j)) add_sum(v[j], s);
    const float mean = group_sum<G>(s.x + s.y, slot[0]) / (float)A.n;
    const float2 minus_mean = both(-mean);
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (mine_here(j)) add_squares(v[j], minus_mean, q);
    const float rstd = 1.0f / sqrtf(group_sum<G>(q.x + q.y, slot[1]) / (float)A.n + A.eps);
    if (t == 0) { A.stats[row] = mean; A.stats[A.rows + row] = rstd; }
    T* y = static_cast<T*>(A.y) + row * A.ld_y + t * VEC;
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (mine_here(j)) store_vec<T, VEC>(y + j * G * VEC, normalised(v[j], A, (t + j * G) * VEC, minus_mean, both(rstd)));
}

// A row at a time, rows blockIdx, blockIdx + grid, ... to a block: the threads keep their columns of w and b, and the next row is
// on its way into registers while one is worked on.  For few rows (everything is asked for at once: 6.0 us for one row of
// 2048, 8.1 through the ring below) and for fp32 (8192 x 2048 20.9 us, through the ring 24.7).
template <typename T, int VEC, int G, int E, bool FULL>
__global__ void __launch_bounds__(GroupShape<G>::BLOCK) k_layer_norm_rows(const NormArgs A) {
    constexpr int NV = E / VEC, P = PAIRS<VEC>;
    __shared__ float slot[2][32];
    const int t = threadIdx.x % G;
    const int64_t step = (int64_t)gridDim.x * GroupShape<G>::ROWS;
    int64_t row = (int64_t)blockIdx.x * GroupShape<G>::ROWS + threadIdx.x / G;
    const int nv = A.n / VEC;
    auto mine_here = [&](int j) { return FULL || t + j * G < nv; };
    const T* x = static_cast<const T*>(A.x) + row * A.ld_x + t * VEC;
    T* y = static_cast<T*>(A.y) + row * A.ld_y + t * VEC;
    Vec<T, VEC> v[NV];
    auto fetch = [&]() {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (mine_here(j)) v[j] = load_vec_stream<T, VEC>(x + j * G * VEC);
        x += step * A.ld_x;
    };
    if (row < A.rows) fetch();
    float2 w[NV][P], b[NV][P];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < P; ++i) { w[j][i] = both(1.f); b[j][i] = both(0.f); }
        if (A.w && mine_here(j)) load_param<T, VEC>(A.w, A.w_f32, (t + j * G) * VEC, w[j]);
        if (A.b && mine_here(j)) load_param<T, VEC>(A.b, A.w_f32, (t + j * G) * VEC, b[j]);
    }
    const float inv_n = 1.f / (float)A.n;
#pragma unroll 1
    for (; row < A.rows; row += step) {
        Vec<T, VEC> now[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) now[j] = v[j];
        if (row + step < A.rows) fetch();
        float2 s = both(0.f), q = both(0.f);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (mine_here(j)) add_sum(now[j], s);
        const float mean = mean_of(group_sum<G>(s.x + s.y, slot[0]), (float)A.n, inv_n);
        const float2 minus_mean = both(-mean);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (mine_here(j)) add_squares(now[j], minus_mean, q);
        const float rstd = 1.0f / sqrtf(group_sum<G>(q.x + q.y, slot[1]) * inv_n + A.eps);
        if (t == 0) { A.stats[row] = mean; A.stats[A.rows + row] = rstd; }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (mine_here(j)) {
                float2 f[P];
                unpack_pairs(now[j], f);
#pragma unroll
                for (int i = 0; i < P; ++i) f[i] = fma2(mul2(add2(f[i], minus_mean), both(rstd)), w[j][i], b[j][i]);
                store_vec<T, VEC>(y + j * G * VEC, pack_pairs<T, VEC>(f));
            }
        }
        y += step * A.ld_y;
    }
}

// Several rows at once, and more of them to a block: the threads keep their columns of w and b, which L1 would have to serve
// again for every row (twice as many bytes as the row, if they are fp32 and it is not); the latency of the sums' way through
// warps and block is paid once for R rows; and the next R rows are on their way into shared memory meanwhile.  A thread
// copies what it will read itself.  (Vectors of 2 bytes cannot be copied this way.)
//
// Measured at 16384 x 2048 in bfloat16 (us): 23, 5.8 TB/s (with new results beside the last ones, which the L2 then does not
// hold, 26.5); 2 rows at a time 24.7, 1 row 26.2; k_layer_norm_rows 28.8; a warp per
// row and w, b from L1 29.3, with fp32 w, b 36.9.
constexpr int STAGES = 2;
template <typename T, int VEC> constexpr bool STAGED = sizeof(T) * VEC >= 4;

// Sums of R values over the group, in all its threads.  `slot` is not used again before the next barrier but one.
template <int G, int R>
__device__ __forceinline__ void group_sums(float (&v)[R], float (*slot)[R]) {
    constexpr int NW = GroupShape<G>::WARPS, SPREAD = 32 / R;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float mine = warp_sums<R>(v);
    if constexpr (G == 32) {
#pragma unroll
        for (int i = 0; i < R; ++i) v[i] = __shfl_sync(0xffffffffu, mine, i * SPREAD);
    } else {
        if (lane % SPREAD == 0) slot[warp][lane / SPREAD] = mine;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R; ++i) v[i] = slot[0][i];
#pragma unroll
        for (int q = 1; q < NW; ++q)
#pragma unroll
            for (int i = 0; i < R; ++i) v[i] += slot[q][i];
    }
}

template <typename T, int VEC, int G, int E, int R, bool FULL>
__global__ void __launch_bounds__(GroupShape<G>::BLOCK) k_layer_norm_ring(const NormArgs A) {
    constexpr int NV = E / VEC, P = PAIRS<VEC>, BLOCK = GroupShape<G>::BLOCK;
    extern __shared__ __align__(16) float smem[];
    __shared__ __align__(16) float slot[2][GroupShape<G>::WARPS][R];
    const int t = threadIdx.x % G;
    const int64_t step = (int64_t)gridDim.x * GroupShape<G>::ROWS * R;
    int64_t row = ((int64_t)blockIdx.x * GroupShape<G>::ROWS + threadIdx.x / G) * R;
    const int nv = A.n / VEC;
    auto mine_here = [&](int j) { return FULL || t + j * G < nv; };
    const T* x = static_cast<const T*>(A.x) + row * A.ld_x + t * VEC;
    T* y = static_cast<T*>(A.y) + row * A.ld_y + t * VEC;
    Vec<T, VEC>* ring = reinterpret_cast<Vec<T, VEC>*>(smem) + threadIdx.x;      // [stage][row][j], BLOCK apart
    auto place = [&](int stage, int k, int j) { return ring + ((stage * R + k) * NV + j) * BLOCK; };
    auto send = [&](int64_t r, int stage) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (r + k < A.rows) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (mine_here(j)) copy_async<sizeof(T) * VEC>(place(stage, k, j), x + k * A.ld_x + j * G * VEC);
            }
        }
        x += step * A.ld_x;
        copy_async_commit();
    };
    auto read = [&](int stage, int k, int j) { return *place(stage, k, j); };
    send(row, 0);
    float2 w[NV][P], b[NV][P];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < P; ++i) { w[j][i] = both(1.f); b[j][i] = both(0.f); }
        if (A.w && mine_here(j)) load_param<T, VEC>(A.w, A.w_f32, (t + j * G) * VEC, w[j]);
        if (A.b && mine_here(j)) load_param<T, VEC>(A.b, A.w_f32, (t + j * G) * VEC, b[j]);
    }
    const float inv_n = 1.f / (float)A.n;
    int stage = 0;
    auto rows_in_work = [&](auto all, int have) {
        constexpr bool ALL = decltype(all)::value;
        send(row + step, stage ^ 1);
        copy_async_wait<1>();
        float mean[R], rstd[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            float2 s = both(0.f);
            if (ALL || k < have) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (mine_here(j)) add_sum(read(stage, k, j), s);
            }
            mean[k] = s.x + s.y;
        }
        group_sums<G, R>(mean, slot[0]);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            mean[k] = mean_of(mean[k], (float)A.n, inv_n);
            float2 q = both(0.f);
            if (ALL || k < have) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (mine_here(j)) add_squares(read(stage, k, j), both(-mean[k]), q);
            }
            rstd[k] = q.x + q.y;
        }
        group_sums<G, R>(rstd, slot[1]);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (ALL || k < have) {
                rstd[k] = 1.0f / sqrtf(rstd[k] * inv_n + A.eps);
                if (t == 0) { A.stats[row + k] = mean[k]; A.stats[A.rows + row + k] = rstd[k]; }
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if (mine_here(j)) {
                        float2 f[P];
                        unpack_pairs(read(stage, k, j), f);
#pragma unroll
                        for (int i = 0; i < P; ++i) f[i] = fma2(mul2(add2(f[i], both(-mean[k])), both(rstd[k])), w[j][i], b[j][i]);
                        store_vec<T, VEC>(y + k * A.ld_y + j * G * VEC, pack_pairs<T, VEC>(f));
                    }
                }
            }
        }
        y += step * A.ld_y;
        stage ^= 1;
    };
#pragma unroll 1
    for (; row + R <= A.rows; row += step) rows_in_work(std::true_type{}, R);
    if (R > 1 && row < A.rows) rows_in_work(std::false_type{}, (int)(A.rows - row));
    copy_async_wait<0>();
}

// Rows that do not fit a block's registers: the row is read three times (the second and third mostly from L2).
constexpr int WIDE = 1024;
template <typename T, int VEC>
__global__ void __launch_bounds__(WIDE) k_layer_norm_wide(const NormArgs A) {
    __shared__ float slot[2][32];
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(A.x) + row * A.ld_x;
    const int nv = A.n / VEC;
    float2 s = both(0.f), q = both(0.f);
    for (int i = t; i < nv; i += WIDE) add_sum(load_vec<T, VEC>(x + (int64_t)i * VEC), s);
    const float mean = group_sum<WIDE>(s.x + s.y, slot[0]) / (float)A.n;
    const float2 minus_mean = both(-mean);
    for (int i = t; i < nv; i += WIDE) add_squares(load_vec<T, VEC>(x + (int64_t)i * VEC), minus_mean, q);
    const float rstd = 1.0f / sqrtf(group_sum<WIDE>(q.x + q.y, slot[1]) / (float)A.n + A.eps);
    if (t == 0) { A.stats[row] = mean; A.stats[A.rows + row] = rstd; }
    T* y = static_cast<T*>(A.y) + row * A.ld_y;
    for (int i = t; i < nv; i += WIDE)
        store_vec<T, VEC>(y + (int64_t)i * VEC, normalised(load_vec<T, VEC>(x + (int64_t)i * VEC), A, i * VEC, minus_mean, both(rstd)));
}

// ---- backward ----------------------------------------------------------------------------------------
//
// A block walks rows blockIdx, blockIdx + grid, ...; thread t owns the same columns in every row, so the two sums over
// the rows stay in its registers and leave once, as the block's partial sums [2][n].  k_norm_reduce adds the blocks'
// partials in a fixed order: results do not depend on the schedule, and there are no atomics.

struct NormBackArgs {
    const void* dy; int64_t ld_dy;
    const void* x; int64_t ld_x;
    const void* w; bool w_f32;
    const float* stats;
    int64_t rows; int32_t n;
    void* dx; int64_t ld_dx;
    float* partial;      // [grid][2][n]; NULL: neither dw nor db is wanted
    float* row_sums;     // wide rows: [rows][2]
    int32_t slab;        // columns per CTA of a cluster
    // one block alone has the sums over all rows: it writes them where they belong
    float* dw; float* db; bool direct, accumulate;
};

// What a vector adds to the row's two sums (of a and a h) and to the columns' sums over the rows
template <typename T, int VEC>
__device__ __forceinline__ void back_sums(const Vec<T, VEC>& x, const Vec<T, VEC>& dy, const float2 (&w)[PAIRS<VEC>], float2 minus_mean,
                                          float2 rstd, float2& c1, float2& c2, float2* dw, float2* db) {
    float2 h[PAIRS<VEC>], d[PAIRS<VEC>];
    unpack_pairs(x, h);
    unpack_pairs(dy, d);
#pragma unroll
    for (int i = 0; i < PAIRS<VEC>; ++i) {
        h[i] = mul2(add2(h[i], minus_mean), rstd);
        const float2 a = mul2(d[i], w[i]);
        c1 = add2(c1, a);
        c2 = fma2(a, h[i], c2);
        if (dw) {
            dw[i] = fma2(d[i], h[i], dw[i]);
            db[i] = add2(db[i], d[i]);
        }
    }
}
// dx = rstd (dy w - c1 - (x - mean) (rstd c2))
template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> back_result(const Vec<T, VEC>& x, const Vec<T, VEC>& dy, const float2 (&w)[PAIRS<VEC>],
                                                   float2 minus_mean, float2 rstd, float2 minus_c1, float2 minus_c2) {
    float2 f[PAIRS<VEC>], d[PAIRS<VEC>];
    unpack_pairs(x, f);
    unpack_pairs(dy, d);
    const float2 k = mul2(minus_c2, rstd);
#pragma unroll
    for (int i = 0; i < PAIRS<VEC>; ++i)
        f[i] = mul2(fma2(add2(f[i], minus_mean), k, fma2(d[i], w[i], minus_c1)), rstd);
    return pack_pairs<T, VEC>(f);
}

// R rows at a time: the latency of their sums' way through the warps and the block is paid once for all of them.  The next R
// rows are on their way into shared memory meanwhile; a thread copies what it will read itself.  (Vectors of 2 bytes
// cannot be copied this way: they are read when they are needed.)
//
// Measured at 16384 x 4096 in bfloat16 (us, rows at a time x blocks per SM): 1 x 2 85.9, 2 x 2 80.9, 4 x 2 (128 registers: spills)
// 81.2, 4 x 1 73.4 (in sustained work 79); in fp32, 8192 x 2048 2 x 2 37.2, 4 x 1 37.6, 1999 x 1030 10.5 and 13.4.  Without the ring: with the next row in
// registers 88.6, with the rows ahead asked into L2 86.
template <typename T, int VEC, int G> constexpr int ROWS_AT_ONCE = !STAGED<T, VEC> || sizeof(T) == 4 || G >= 512 ? 2 : 4;
template <typename T, int VEC, int G, int E, int R> constexpr size_t RING_BYTES =
    STAGED<T, VEC> ? (size_t)STAGES * R * 2 * E * sizeof(T) * GroupShape<G>::BLOCK : 0;

// FULL: every thread has E elements (n = G E), so no column needs a check.  SHARED: a cluster of CTAs shares the rows, each with a
// slab of A.slab columns; their sums of a row meet in distributed shared memory.
template <typename T, int VEC, int G, int E, int R, bool FULL, bool SHARED>
__global__ void __launch_bounds__(GroupShape<G>::BLOCK, GroupShape<G>::BLOCK < 128 ? 4 : GroupShape<G>::BLOCK < 256 || (sizeof(T) == 4 && GroupShape<G>::BLOCK == 256) ? 2 : 1)
k_layer_norm_back(const NormBackArgs A) {
    constexpr int NV = E / VEC, ROWS = GroupShape<G>::ROWS, P = PAIRS<VEC>, NW = GroupShape<G>::WARPS, BLOCK = GroupShape<G>::BLOCK;
    constexpr bool RING = STAGED<T, VEC>;
    extern __shared__ __align__(16) float smem[];      // the ring; G = 32: [8][2][n] partial sums at the end
    __shared__ __align__(16) float slot[2][NW][2 * R];
    __shared__ __align__(16) float across[2][8][2 * R];    // SHARED: each CTA's sums
    cg::cluster_group cluster = cg::this_cluster();
    const int t = threadIdx.x % G, sub = threadIdx.x / G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int parts = SHARED ? (int)cluster.num_blocks() : 1, part = SHARED ? (int)cluster.block_rank() : 0;
    const int col0 = SHARED ? part * A.slab : 0, here = SHARED ? min(A.slab, A.n - col0) : A.n;
    const int64_t block = SHARED ? blockIdx.x / parts : blockIdx.x, blocks = SHARED ? gridDim.x / parts : gridDim.x;
    const int nv = here / VEC;
    const float inv_n = 1.0f / (float)A.n;
    auto mine_here = [&](int j) { return FULL || t + j * G < nv; };
    float2 dw[NV][P], db[NV][P], w[NV][P];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < P; ++i) { dw[j][i] = db[j][i] = both(0.f); w[j][i] = both(1.f); }
        if (A.w && mine_here(j)) load_param<T, VEC>(A.w, A.w_f32, col0 + (t + j * G) * VEC, w[j]);
    }
    const int64_t step = blocks * ROWS * R;
    int64_t row = (block * ROWS + sub) * R;
    // this thread's part of the rows in work: dx and (RING: of the rows to be sent next, else of those in work) x, dy
    const T* x = static_cast<const T*>(A.x) + col0 + t * VEC + row * A.ld_x;
    const T* dy = static_cast<const T*>(A.dy) + col0 + t * VEC + row * A.ld_dy;
    T* dx = static_cast<T*>(A.dx) + col0 + t * VEC + row * A.ld_dx;
    Vec<T, VEC>* ring = reinterpret_cast<Vec<T, VEC>*>(smem) + threadIdx.x;      // [stage][row][x, dy][j], BLOCK apart
    auto place = [&](int stage, int k, int which, int j) { return ring + (((stage * R + k) * 2 + which) * NV + j) * BLOCK; };
    auto send = [&](int64_t r, int stage) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (r + k < A.rows) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if (mine_here(j)) {
                        copy_async<sizeof(T) * VEC>(place(stage, k, 0, j), x + k * A.ld_x + j * G * VEC);
                        copy_async<sizeof(T) * VEC>(place(stage, k, 1, j), dy + k * A.ld_dy + j * G * VEC);
                    }
                }
            }
        }
        x += step * A.ld_x;
        dy += step * A.ld_dy;
        copy_async_commit();
    };
    auto read_x = [&](int stage, int k, int j) {
        if constexpr (RING) return *place(stage, k, 0, j);
        else return load_vec<T, VEC>(x + k * A.ld_x + j * G * VEC);
    };
    auto read_dy = [&](int stage, int k, int j) {
        if constexpr (RING) return *place(stage, k, 1, j);
        else return load_vec<T, VEC>(dy + k * A.ld_dy + j * G * VEC);
    };
    if constexpr (RING) {
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) send(row + s * step, s);
    }
    float next_mean[R], next_rstd[R];
    auto next_stats = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            next_mean[k] = r + k < A.rows ? A.stats[r + k] : 0.f;
            next_rstd[k] = r + k < A.rows ? A.stats[A.rows + r + k] : 0.f;
        }
    };
    next_stats(row);
    if constexpr (SHARED) cluster.sync();              // all are there before any of them is written to
    int turn = 0, stage = 0;
    // R rows, all of them there (ALL) or not
    auto rows_in_work = [&](auto all, int have) {
        constexpr bool ALL = decltype(all)::value;
        float2 minus_mean[R], rstd[R];
        float sums[2 * R];
#pragma unroll
        for (int k = 0; k < R; ++k) { minus_mean[k] = both(-next_mean[k]); rstd[k] = both(next_rstd[k]); }
        next_stats(row + step);
        if constexpr (RING) {
            send(row + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1);
            copy_async_wait<STAGES - 1>();
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            float2 c1 = both(0.f), c2 = both(0.f);
            if (ALL || k < have) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (mine_here(j))
                        back_sums<T, VEC>(read_x(stage, k, j), read_dy(stage, k, j), w[j], minus_mean[k], rstd[k], c1, c2, dw[j], db[j]);
            }
            sums[2 * k] = c1.x + c1.y;
            sums[2 * k + 1] = c2.x + c2.y;
        }
        const float mine = warp_sums<2 * R>(sums);
        constexpr int SPREAD = 32 / (2 * R);
        if constexpr (G == 32) {
#pragma unroll
            for (int i = 0; i < 2 * R; ++i) sums[i] = __shfl_sync(0xffffffffu, mine, i * SPREAD);
        } else {
            if (lane % SPREAD == 0) slot[turn][warp][lane / SPREAD] = mine;
            __syncthreads();
            float2 total[R];
#pragma unroll
            for (int k = 0; k < R; ++k) total[k] = both(0.f);
#pragma unroll
            for (int q = 0; q < NW; ++q)
#pragma unroll
                for (int k = 0; k < R; ++k) total[k] = add2(total[k], *reinterpret_cast<const float2*>(&slot[turn][q][2 * k]));
#pragma unroll
            for (int k = 0; k < R; ++k) { sums[2 * k] = total[k].x; sums[2 * k + 1] = total[k].y; }
            if constexpr (SHARED) {
                // to every CTA of the cluster; read behind its barrier, and not written again before the next but one
                if ((int)threadIdx.x < parts) {
                    float2* to = reinterpret_cast<float2*>(cluster.map_shared_rank(&across[turn][part][0], threadIdx.x));
#pragma unroll
                    for (int k = 0; k < R; ++k) to[k] = total[k];
                }
                cluster.sync();
#pragma unroll
                for (int i = 0; i < 2 * R; ++i) sums[i] = across[turn][0][i];
                for (int q = 1; q < parts; ++q)
#pragma unroll
                    for (int i = 0; i < 2 * R; ++i) sums[i] += across[turn][q][i];
            }
            turn ^= 1;
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (ALL || k < have) {
                const float2 m1 = both(-sums[2 * k] * inv_n), m2 = both(-sums[2 * k + 1] * inv_n);
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (mine_here(j))
                        store_vec<T, VEC>(dx + k * A.ld_dx + j * G * VEC,
                                          back_result<T, VEC>(read_x(stage, k, j), read_dy(stage, k, j), w[j], minus_mean[k], rstd[k], m1, m2));
            }
        }
        dx += step * A.ld_dx;
        if constexpr (!RING) { x += step * A.ld_x; dy += step * A.ld_dy; }
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    };
    for (; row + R <= A.rows; row += step) rows_in_work(std::true_type{}, R);
    if (R > 1 && row < A.rows) rows_in_work(std::false_type{}, (int)(A.rows - row));
    if constexpr (RING) copy_async_wait<0>();
    if constexpr (SHARED) cluster.sync();              // nobody leaves while others write to its shared memory
    successor_may_start();                             // k_norm_reduce waits for the partial sums by itself
    if (!A.partial) return;
    float* out = A.partial + block * 2 * A.n + col0;
    auto put = [&](int c, float value) {               // c: 0 .. 2 n - 1, dw then db, from this CTA's first column on
        if (!A.direct) { out[c] = value; return; }
        float* to = c < A.n ? A.dw : A.db;
        const int at = (c < A.n ? c : c - A.n) + col0;
        if (to) to[at] = A.accumulate ? to[at] + value : value;
    };
    float* mine = smem + (int64_t)sub * 2 * A.n;       // G = 32: the block's 8 warps add up in shared memory
    if (G == 32) __syncthreads();                      // every warp is done with the ring
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = t + j * G;
        if (i < nv) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float a = e & 1 ? dw[j][e / 2].y : dw[j][e / 2].x, b = e & 1 ? db[j][e / 2].y : db[j][e / 2].x;
                if constexpr (G == 32) {
                    mine[i * VEC + e] = a;
                    mine[A.n + i * VEC + e] = b;
                } else {
                    put(i * VEC + e, a);
                    put(A.n + i * VEC + e, b);
                }
            }
        }
    }
    if constexpr (G == 32) {
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * A.n; c += GroupShape<G>::BLOCK) {
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) s += smem[(int64_t)r * 2 * A.n + c];
            put(c, s);
        }
    }
}

// Wide rows, first pass: the two sums of each row.
template <typename T, int VEC>
__global__ void __launch_bounds__(WIDE) k_norm_back_sums(const NormBackArgs A) {
    __shared__ float slot[2][32];
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(A.x) + row * A.ld_x;
    const T* d = static_cast<const T*>(A.dy) + row * A.ld_dy;
    const float2 minus_mean = both(-A.stats[row]), rstd = both(A.stats[A.rows + row]);
    const int nv = A.n / VEC;
    float2 c1 = both(0.f), c2 = both(0.f);
    for (int i = threadIdx.x; i < nv; i += WIDE) {
        float2 w[PAIRS<VEC>];
#pragma unroll
        for (int k = 0; k < PAIRS<VEC>; ++k) w[k] = both(1.f);
        if (A.w) load_param<T, VEC>(A.w, A.w_f32, i * VEC, w);
        back_sums<T, VEC>(load_vec<T, VEC>(x + (int64_t)i * VEC), load_vec<T, VEC>(d + (int64_t)i * VEC), w, minus_mean, rstd, c1, c2,
                           nullptr, nullptr);
    }
    const float s1 = group_sum<WIDE>(c1.x + c1.y, slot[0]), s2 = group_sum<WIDE>(c2.x + c2.y, slot[1]);
    if (threadIdx.x == 0) {
        A.row_sums[2 * row] = s1 / (float)A.n;
        A.row_sums[2 * row + 1] = s2 / (float)A.n;
    }
}

// Second pass: blockIdx.x is a slab of 256 vectors of columns, blockIdx.y a share of the rows.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) k_norm_back_slab(const NormBackArgs A) {
    constexpr int P = PAIRS<VEC>;
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= A.n / VEC) return;
    const int64_t col = (int64_t)i * VEC;
    float2 dw[P], db[P], w[P];
#pragma unroll
    for (int e = 0; e < P; ++e) { dw[e] = db[e] = both(0.f); w[e] = both(1.f); }
    if (A.w) load_param<T, VEC>(A.w, A.w_f32, (int)col, w);
    for (int64_t row = blockIdx.y; row < A.rows; row += gridDim.y) {
        float2 c1 = both(0.f), c2 = both(0.f);
        const float2 minus_mean = both(-A.stats[row]), rstd = both(A.stats[A.rows + row]);
        const Vec<T, VEC> vx = load_vec_stream<T, VEC>(static_cast<const T*>(A.x) + row * A.ld_x + col);
        const Vec<T, VEC> vd = load_vec_stream<T, VEC>(static_cast<const T*>(A.dy) + row * A.ld_dy + col);
        back_sums<T, VEC>(vx, vd, w, minus_mean, rstd, c1, c2, dw, db);
        store_vec<T, VEC>(static_cast<T*>(A.dx) + row * A.ld_dx + col,
                          back_result<T, VEC>(vx, vd, w, minus_mean, rstd, both(-A.row_sums[2 * row]), both(-A.row_sums[2 * row + 1])));
    }
    if (!A.partial) return;
    float* out = A.partial + (int64_t)blockIdx.y * 2 * A.n;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        out[col + e] = e & 1 ? dw[e / 2].y : dw[e / 2].x;
        out[A.n + col + e] = e & 1 ? db[e / 2].y : db[e / 2].x;
    }
}

// dw[c], db[c] = sum over the blocks' partials, in a fixed order: 32 columns per block, its warps share the partials.
constexpr int REDUCE_WARPS = 32;
__global__ void __launch_bounds__(REDUCE_WARPS * 32) k_norm_reduce(const float* partial, int parts, int n, float* dw, float* db,
                                                                   int accumulate) {
    __shared__ float s[REDUCE_WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;              // 0 .. 2n - 1
    float a = 0.f;
    successor_wait();
    if (c < 2 * n) {
        constexpr int AT_ONCE = 10;                        // reads on their way, without a remainder that goes one by one
        for (int p0 = warp; p0 < parts; p0 += REDUCE_WARPS * AT_ONCE) {
            float v[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int p = p0 + u * REDUCE_WARPS;
                v[u] = p < parts ? partial[(int64_t)p * 2 * n + c] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) a += v[u];
        }
    }
    s[warp][lane] = a;
    __syncthreads();
    if (warp == 0 && c < 2 * n) {
#pragma unroll
        for (int k = 1; k < REDUCE_WARPS; ++k) a += s[k][lane];
        float* out = c < n ? dw : db;
        if (out) {
            const int at = c < n ? c : c - n;
            out[at] = accumulate ? out[at] + a : a;
        }
    }
}

// rows == 0: the sums over no rows
__global__ void k_norm_zero(float* dw, float* db, int n) {
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c < n) {
        if (dw) dw[c] = 0.f;
        if (db) db[c] = 0.f;
    }
}

// ---- host side ---------------------------------------------------------------------------------------

// Widest vector (elements) that every base, row stride and the row length allow.
int vec_of(int es, int64_t n, std::initializer_list<const void*> bases, std::initializer_list<int64_t> lds,
           std::initializer_list<const void*> f32_params, bool params_f32) {
    for (int vec = 16 / es; vec > 1; vec /= 2) {
        const int bytes = vec * es;
        bool ok = n % vec == 0;
        for (const void* p : bases) ok = ok && aligned_to(p, bytes);
        for (int64_t ld : lds) ok = ok && ld % vec == 0;
        const int pbytes = params_f32 ? (vec * 4 > 16 ? 16 : vec * 4) : bytes;
        for (const void* p : f32_params) ok = ok && aligned_to(p, pbytes);
        if (ok) return vec == 4 && es == 2 ? 2 : vec;  // 16-bit formats: 8, 2 or 1 elements
    }
    return 1;
}

// A grid that fills the SMs; `smem` depends on the kernel alone
template <typename K>
int launch_filling(K kernel, const NormArgs& A, int block, int64_t tile, size_t smem, PerDevice& known, int sms, cudaStream_t st) {
    int per_sm = 0;
    const int e = residency(kernel, block, smem, known, &per_sm);
    if (e) return e;
    const int64_t grid = std::min((A.rows + tile - 1) / tile, (int64_t)sms * per_sm);
    kernel<<<(unsigned)grid, block, smem, st>>>(A);
    return launched();
}

template <typename T, int VEC>
int launch_norm(const NormArgs& A, int sms, cudaStream_t st) {
    const int n = A.n;
#define NORM_ROWS(G, E, R)                                                                                          \
    do {                                                                                                            \
        constexpr bool WIDEST = VEC * sizeof(T) == 16;                                                              \
        constexpr int BLOCK = GroupShape<G>::BLOCK, ROWS = GroupShape<G>::ROWS;                                     \
        const bool full = WIDEST && n == G * E;                                                                     \
        if constexpr (sizeof(T) == 2 && VEC > 1 && G <= 512) {                                                      \
            if (A.rows >= 8 * sms) {                                                                                \
                static PerDevice known[2];                                                                            \
                auto kernel = full ? k_layer_norm_ring<T, VEC, G, E, R, WIDEST> : k_layer_norm_ring<T, VEC, G, E, R, false>; \
                return launch_filling(kernel, A, BLOCK, ROWS * R, (size_t)STAGES * R * E * sizeof(T) * BLOCK, known[full], sms, st); \
            }                                                                                                       \
        }                                                                                                           \
        static PerDevice known[2];                                                                                    \
        auto kernel = full ? k_layer_norm_rows<T, VEC, G, E, WIDEST> : k_layer_norm_rows<T, VEC, G, E, false>;      \
        return launch_filling(kernel, A, BLOCK, ROWS, 0, known[full], sms, st);                                     \
    } while (0)
#define NORM(G, E)                                                                                                  \
    do {                                                                                                            \
        const int64_t grid = (A.rows + GroupShape<G>::ROWS - 1) / GroupShape<G>::ROWS;                              \
        if (grid > 0x7fffffff) return SSGD_EINVAL;                                                                  \
        constexpr bool WIDEST = VEC * sizeof(T) == 16;                                                              \
        auto kernel = WIDEST && n == G * E ? k_layer_norm<T, VEC, G, E, WIDEST> : k_layer_norm<T, VEC, G, E, false>; \
        kernel<<<(unsigned)grid, GroupShape<G>::BLOCK, 0, st>>>(A);                                                 \
        return launched();                                                                                          \
    } while (0)
    constexpr int E = VEC == 1 ? 8 : 16;               // a vector of one element wastes half of a pair's registers
    if (n <= 32 * E) NORM_ROWS(32, E, 4);
    if (n <= 64 * E) NORM_ROWS(64, E, 4);
    if (n <= 128 * E) NORM_ROWS(128, E, 4);
    if (n <= 256 * E) NORM_ROWS(256, E, 4);
    if (n <= 512 * E) NORM_ROWS(512, E, 2);
    if constexpr (VEC == 1) if (n <= 1024 * 8) NORM_ROWS(1024, 8, 1);
    if (n <= 512 * 32) NORM(512, 32);
#undef NORM
#undef NORM_ROWS
    if (A.rows > 0x7fffffff) return SSGD_EINVAL;
    k_layer_norm_wide<T, VEC><<<(unsigned)A.rows, WIDE, 0, st>>>(A);
    return launched();
}

constexpr int64_t PART_BLOCKS = 148 * 4;         // at most so many partial sums of dw and db
constexpr int BACK_NARROW = 512 * 8;             // rows up to here never need the sums of k_norm_back_sums

template <typename T, int VEC>
int launch_norm_back(NormBackArgs A, int sms, int* parts, cudaStream_t st) {
    const int n = A.n;
    int64_t grid = 0;
#define NORM_BACK(G, E)                                                                                             \
    do {                                                                                                            \
        constexpr int R = ROWS_AT_ONCE<T, VEC, G>, BLOCK = GroupShape<G>::BLOCK, TILE = GroupShape<G>::ROWS * R;         \
        constexpr bool WIDEST = VEC * sizeof(T) == 16;                                                              \
        static PerDevice known[2];                                                                                    \
        const bool full = WIDEST && n == G * E;                                                                     \
        auto kernel = full ? k_layer_norm_back<T, VEC, G, E, R, WIDEST, false> : k_layer_norm_back<T, VEC, G, E, R, false, false>; \
        size_t smem = RING_BYTES<T, VEC, G, E, R>;                                                                  \
        if (G == 32) smem = std::max(smem, (size_t)GroupShape<G>::ROWS * 2 * G * E * 4);                            \
        int per_sm = 0;                                                                                             \
        const int e = residency(kernel, BLOCK, smem, known[full], &per_sm);                                         \
        if (e) return e;                                                                                            \
        grid = std::min({(A.rows + TILE - 1) / TILE, (int64_t)sms * per_sm, PART_BLOCKS});                          \
        A.direct = grid == 1;                                                                                       \
        kernel<<<(unsigned)grid, BLOCK, smem, st>>>(A);                                                             \
        *parts = A.direct ? 0 : (int)grid;           /* 0: nothing is left to add up */                             \
        return launched();                                                                                          \
    } while (0)
    // 16 elements of 16 bits per thread or 8 of 32 bits: with their sums, 128 registers
    constexpr int E = sizeof(T) == 4 || VEC == 1 ? 8 : 16;
    if (n <= 32 * E) NORM_BACK(32, E);
    if constexpr (sizeof(T) == 2) if (n <= 64 * E) NORM_BACK(64, E);   // 31296 x 960 binary16 41.1, with 128 threads 45.4
    if (n <= 128 * E) NORM_BACK(128, E);
    if (n <= 256 * E) NORM_BACK(256, E);
    if (n <= 512 * E) NORM_BACK(512, E);
    if constexpr (STAGED<T, VEC>) if (n <= 8 * 256 * E) {
        // a cluster of 4 or 8 CTAs to the rows
        constexpr int G = 256, R = ROWS_AT_ONCE<T, VEC, G>;
        static PerDevice known, clusters[2];
        auto kernel = k_layer_norm_back<T, VEC, G, E, R, false, true>;
        const size_t smem = RING_BYTES<T, VEC, G, E, R>;
        int per_sm = 0, dev = 0;
        const int e = residency(kernel, G, smem, known, &per_sm);
        if (e) return e;
        const int cluster = n <= 4 * G * E ? 4 : 8;
        A.slab = ((n + cluster - 1) / cluster + 8 - 1) / 8 * 8;            // whole vectors
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)cluster);
        cfg.blockDim = dim3(G);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)cluster;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        // clusters lie within a group of SMs: fewer of them fit than their CTAs alone would
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return SSGD_ECUDA;
        int fit = clusters[cluster == 8].value[dev];
        if (!fit) {
            if (cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg) != cudaSuccess || fit < 1) return SSGD_ECUDA;
            clusters[cluster == 8].value[dev] = fit;
        }
        grid = std::min({(A.rows + R - 1) / R, (int64_t)fit, PART_BLOCKS});
        cfg.gridDim = dim3((unsigned)(grid * cluster));
        A.direct = grid == 1;
        *parts = A.direct ? 0 : (int)grid;
        return cudaLaunchKernelEx(&cfg, kernel, A) == cudaSuccess ? SSGD_OK : SSGD_ECUDA;
    }
#undef NORM_BACK
    if (A.rows > 0x7fffffff) return SSGD_EINVAL;
    k_norm_back_sums<T, VEC><<<(unsigned)A.rows, WIDE, 0, st>>>(A);
    const int slabs = (n / VEC + 255) / 256;
    int64_t shares = (PART_BLOCKS * 2 + slabs - 1) / slabs;
    if (shares > PART_BLOCKS) shares = PART_BLOCKS;
    if (shares > A.rows) shares = A.rows;
    k_norm_back_slab<T, VEC><<<dim3((unsigned)slabs, (unsigned)shares), 256, 0, st>>>(A);
    *parts = (int)shares;
    return launched();
}

#define BY_FORMAT(fn, fmt, vec, ...)                                                               \
    ((fmt) == SSGD_FMT_F32                                                                         \
         ? ((vec) == 4 ? fn<float, 4>(__VA_ARGS__) : (vec) == 2 ? fn<float, 2>(__VA_ARGS__) : fn<float, 1>(__VA_ARGS__)) \
     : (fmt) == SSGD_FMT_F16                                                                       \
         ? ((vec) == 8 ? fn<__half, 8>(__VA_ARGS__) : (vec) == 2 ? fn<__half, 2>(__VA_ARGS__) : fn<__half, 1>(__VA_ARGS__)) \
         : ((vec) == 8 ? fn<__nv_bfloat16, 8>(__VA_ARGS__)                                         \
            : (vec) == 2 ? fn<__nv_bfloat16, 2>(__VA_ARGS__) : fn<__nv_bfloat16, 1>(__VA_ARGS__)))

constexpr int64_t MAX_N = (int64_t)1 << 24;      // columns are indexed with 32 bits

int check_shape(int64_t rows, int64_t n, int32_t fmt_x, int32_t fmt_w) {
    if (rows < 0 || n < 1 || n > MAX_N) return SSGD_EINVAL;
    if (fmt_x != SSGD_FMT_F32 && fmt_x != SSGD_FMT_F16 && fmt_x != SSGD_FMT_BF16) return SSGD_EINVAL;
    if (fmt_w != SSGD_FMT_F32 && fmt_w != fmt_x) return SSGD_EINVAL;
    return SSGD_OK;
}

}  // namespace

extern "C" {

int ssgd_layer_norm(const void* x, int64_t ld_x, int32_t fmt_x, const void* w, const void* b, int32_t fmt_w,
                    int64_t rows, int64_t n, float eps, void* y, int64_t ld_y, float* stats, void* stream) {
    int e = check_shape(rows, n, fmt_x, fmt_w);
    if (e) return e;
    if (!(eps >= 0.f) || ld_x < n || ld_y < n) return SSGD_EINVAL;
    if (rows == 0) return SSGD_OK;
    if (!x || !y || !stats) return SSGD_EINVAL;
    const int es = fmt_bytes(fmt_x), ws = fmt_bytes(fmt_w);
    if (!aligned_to(x, es) || !aligned_to(y, es) || !aligned_to(w, ws) || !aligned_to(b, ws) || !aligned_to(stats, 4))
        return SSGD_EALIGN;
    const NormArgs A{x, ld_x, w, b, fmt_w == SSGD_FMT_F32, rows, (int32_t)n, eps, y, ld_y, stats};
    const int vec = vec_of(es, n, {x, y}, {ld_x, ld_y}, {w, b}, A.w_f32);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int sms = 0;
    if ((e = sm_count_of_current_device(&sms))) return e;
    return BY_FORMAT(launch_norm, fmt_x, vec, A, sms, st);
}

int ssgd_layer_norm_backward_workspace(int64_t rows, int64_t n, size_t* out_bytes) {
    if (rows < 0 || n < 1 || n > MAX_N || !out_bytes) return SSGD_EINVAL;
    const int64_t parts = rows < PART_BLOCKS ? rows : PART_BLOCKS;
    size_t bytes = (size_t)parts * 2 * (size_t)n * 4;
    if (n > BACK_NARROW) bytes += (size_t)rows * 2 * 4;
    *out_bytes = bytes;
    return SSGD_OK;
}

int ssgd_layer_norm_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, int32_t fmt_x, const void* w,
                             int32_t fmt_w, const float* stats, int64_t rows, int64_t n, void* dx, int64_t ld_dx,
                             float* dw, float* db, int32_t accumulate, void* workspace, size_t workspace_bytes,
                             void* stream) {
    int e = check_shape(rows, n, fmt_x, fmt_w);
    if (e) return e;
    if (ld_dy < n || ld_x < n || ld_dx < n) return SSGD_EINVAL;
    const int es = fmt_bytes(fmt_x), ws = fmt_bytes(fmt_w);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!aligned_to(dw, 4) || !aligned_to(db, 4)) return SSGD_EALIGN;
    if (rows == 0) {
        if (accumulate || (!dw && !db)) return SSGD_OK;
        k_norm_zero<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(dw, db, (int)n);
        return launched();
    }
    if (!dy || !x || !stats || !dx) return SSGD_EINVAL;
    if (!aligned_to(dy, es) || !aligned_to(x, es) || !aligned_to(dx, es) || !aligned_to(w, ws) || !aligned_to(stats, 4) ||
        !aligned_to(workspace, 16))
        return SSGD_EALIGN;
    size_t need = 0;
    ssgd_layer_norm_backward_workspace(rows, n, &need);
    if (!workspace || workspace_bytes < need) return SSGD_EWORKSPACE;
    int sms = 0;
    if ((e = sm_count_of_current_device(&sms))) return e;
    NormBackArgs A{dy, ld_dy, x, ld_x, w, fmt_w == SSGD_FMT_F32, stats, rows, (int32_t)n, dx, ld_dx, nullptr, nullptr, 0, dw, db, false, accumulate != 0};
    float* base = static_cast<float*>(workspace);
    A.row_sums = base;
    if (n > BACK_NARROW) base += 2 * rows;
    A.partial = dw || db ? base : nullptr;
    const int vec = vec_of(es, n, {dy, x, dx}, {ld_dy, ld_x, ld_dx}, {w}, A.w_f32);
    int parts = 0;
    e = BY_FORMAT(launch_norm_back, fmt_x, vec, A, sms, &parts, st);
    if (e || !A.partial || parts == 0) return e;
    return launch_after(st, k_norm_reduce, dim3((unsigned)((2 * n + 31) / 32)), REDUCE_WARPS * 32, A.partial, parts, (int)n, dw, db,
                        accumulate);
}

}  // extern "C"
