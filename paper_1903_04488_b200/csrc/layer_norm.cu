// layer_norm.cu -- layer norm over the last dimension, forward and backward (ssgd_layer_norm, ssgd_layer_norm_backward).
//
//   forward    mean = 1/n sum x,  rstd = (1/n sum (x - mean)^2 + eps)^-1/2,  y = (x - mean) rstd w + b
//   backward   h = (x - mean) rstd,  a = dy w
//              dx = rstd (a - 1/n sum a - h 1/n sum a h),   dw = sum over rows of dy h,   db = sum over rows of dy
//
// Both are bound by HBM: two streams of rows x n elements forward, three backward, a dozen operations per element.
// So a row is read once and stays in registers (in its own format) from the first sum to the result: the variance is
// the mean of squared deviations from the mean already known, not a difference of large sums.
#include "formats.cuh"

using namespace ssgd;

namespace {

// A group of G threads owns a row; thread t of it holds the vectors t, t + G, ... of VEC elements, E elements in all.
// G = 32: 8 rows per block, sums by shuffles alone.  G > 32: one row per block.
template <int G> struct GroupShape {
    static constexpr int BLOCK = G < 256 && G == 32 ? 256 : G;
    static constexpr int ROWS = BLOCK / G;
    static constexpr int WARPS = G / 32;
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
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
    float s = lane < NW ? slot[lane] : 0.f;
#pragma unroll
    for (int o = NW / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return __shfl_sync(0xffffffffu, s, 0);
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
    float2 f[PAIRS<VEC>], w[PAIRS<VEC>];
    unpack_pairs(v, f);
#pragma unroll
    for (int i = 0; i < PAIRS<VEC>; ++i) f[i] = mul2(add2(f[i], minus_mean), rstd);
    if (args.w) {
        load_param<T, VEC>(args.w, args.w_f32, col, w);
#pragma unroll
        for (int i = 0; i < PAIRS<VEC>; ++i) f[i] = mul2(f[i], w[i]);
    }
    if (args.b) {
        load_param<T, VEC>(args.b, args.w_f32, col, w);
#pragma unroll
        for (int i = 0; i < PAIRS<VEC>; ++i) f[i] = add2(f[i], w[i]);
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

template <typename T, int VEC, int G, int E>
__global__ void __launch_bounds__(GroupShape<G>::BLOCK) k_layer_norm(const NormArgs A) {
    constexpr int NV = E / VEC;
    __shared__ float slot[2][32];
    const int t = threadIdx.x % G;
    const int64_t row = (int64_t)blockIdx.x * GroupShape<G>::ROWS + threadIdx.x / G;
    if (row >= A.rows) return;                         // a whole warp (G = 32) or nobody
    const T* x = static_cast<const T*>(A.x) + row * A.ld_x;
    const int nv = A.n / VEC;
    Vec<T, VEC> v[NV];
    float2 s = both(0.f), q = both(0.f);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = t + j * G;
        if (i < nv) v[j] = load_vec_stream<T, VEC>(x + (int64_t)i * VEC);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (t + j * G < nv) add_sum(v[j], s);
    const float mean = group_sum<G>(s.x + s.y, slot[0]) / (float)A.n;
    const float2 minus_mean = both(-mean);
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (t + j * G < nv) add_squares(v[j], minus_mean, q);
    const float rstd = 1.0f / sqrtf(group_sum<G>(q.x + q.y, slot[1]) / (float)A.n + A.eps);
    if (t == 0) { A.stats[row] = mean; A.stats[A.rows + row] = rstd; }
    T* y = static_cast<T*>(A.y) + row * A.ld_y;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = t + j * G;
        if (i < nv) store_vec<T, VEC>(y + (int64_t)i * VEC, normalised(v[j], A, i * VEC, minus_mean, both(rstd)));
    }
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
};

// h = (x - mean) rstd and a = dy w of one vector, and what it adds to the four sums
template <int P>
struct BackTerms { float2 h[P], a[P]; };
template <typename T, int VEC>
__device__ __forceinline__ BackTerms<PAIRS<VEC>> back_terms(const Vec<T, VEC>& x, const Vec<T, VEC>& dy, const float2 (&w)[PAIRS<VEC>],
                                                            float2 minus_mean, float2 rstd, float2& c1, float2& c2,
                                                            float2* dw, float2* db) {
    BackTerms<PAIRS<VEC>> r;
    float2 d[PAIRS<VEC>];
    unpack_pairs(x, r.h);
    unpack_pairs(dy, d);
#pragma unroll
    for (int i = 0; i < PAIRS<VEC>; ++i) {
        r.h[i] = mul2(add2(r.h[i], minus_mean), rstd);
        r.a[i] = mul2(d[i], w[i]);
        c1 = add2(c1, r.a[i]);
        c2 = fma2(r.a[i], r.h[i], c2);
        if (dw) {
            dw[i] = fma2(d[i], r.h[i], dw[i]);
            db[i] = add2(db[i], d[i]);
        }
    }
    return r;
}
// dx = rstd a - rstd c1 - h (rstd c2)
template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> back_result(const BackTerms<PAIRS<VEC>>& r, float2 rstd, float2 minus_c1, float2 minus_c2) {
    float2 f[PAIRS<VEC>];
#pragma unroll
    for (int i = 0; i < PAIRS<VEC>; ++i) f[i] = mul2(fma2(r.h[i], minus_c2, add2(r.a[i], minus_c1)), rstd);
    return pack_pairs<T, VEC>(f);
}

template <typename T, int VEC, int G, int E>
__global__ void __launch_bounds__(GroupShape<G>::BLOCK) k_layer_norm_back(const NormBackArgs A) {
    constexpr int NV = E / VEC, ROWS = GroupShape<G>::ROWS, P = PAIRS<VEC>;
    extern __shared__ float smem[];                    // G = 32: [8][2][n] partial sums at the end
    __shared__ float2 slot[2][32];
    const int t = threadIdx.x % G, sub = threadIdx.x / G;
    const int nv = A.n / VEC;
    const float inv_n = 1.0f / (float)A.n;
    float2 dw[NV][P], db[NV][P], w[NV][P];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < P; ++i) { dw[j][i] = db[j][i] = both(0.f); w[j][i] = both(1.f); }
        if (A.w && t + j * G < nv) load_param<T, VEC>(A.w, A.w_f32, (t + j * G) * VEC, w[j]);
    }
    // the next row's vectors are on their way while this row is summed and written
    Vec<T, VEC> vx[NV], vd[NV];
    float mean = 0.f, rstd = 0.f;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + sub;
    auto fetch = [&](int64_t r) {
        const T* x = static_cast<const T*>(A.x) + r * A.ld_x;
        const T* d = static_cast<const T*>(A.dy) + r * A.ld_dy;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * G;
            if (i < nv) {
                vx[j] = load_vec_stream<T, VEC>(x + (int64_t)i * VEC);
                vd[j] = load_vec_stream<T, VEC>(d + (int64_t)i * VEC);
            }
        }
        mean = A.stats[r];
        rstd = A.stats[A.rows + r];
    };
    if (row < A.rows) fetch(row);
    int turn = 0;
    for (; row < A.rows; row += step) {
        float2 c1 = both(0.f), c2 = both(0.f);
        BackTerms<P> r[NV];
        const float2 scale = both(rstd);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (t + j * G < nv) r[j] = back_terms<T, VEC>(vx[j], vd[j], w[j], both(-mean), scale, c1, c2, dw[j], db[j]);
        if (row + step < A.rows) fetch(row + step);
        float s1 = warp_sum(c1.x + c1.y), s2 = warp_sum(c2.x + c2.y);
        if constexpr (G > 32) {
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
            constexpr int NW = GroupShape<G>::WARPS;
            if (lane == 0) slot[turn][warp] = make_float2(s1, s2);
            __syncthreads();
            float2 p = lane < NW ? slot[turn][lane] : both(0.f);
#pragma unroll
            for (int o = NW / 2; o > 0; o >>= 1)
                p = add2(p, make_float2(__shfl_xor_sync(0xffffffffu, p.x, o), __shfl_xor_sync(0xffffffffu, p.y, o)));
            s1 = __shfl_sync(0xffffffffu, p.x, 0);
            s2 = __shfl_sync(0xffffffffu, p.y, 0);
            turn ^= 1;
        }
        T* dx = static_cast<T*>(A.dx) + row * A.ld_dx;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * G;
            if (i < nv)
                store_vec<T, VEC>(dx + (int64_t)i * VEC, back_result<T, VEC>(r[j], scale, both(-s1 * inv_n), both(-s2 * inv_n)));
        }
    }
    if (!A.partial) return;
    float* out = A.partial + (int64_t)blockIdx.x * 2 * A.n;
    float* mine = G == 32 ? smem + (int64_t)sub * 2 * A.n : out;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = t + j * G;
        if (i < nv) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                mine[i * VEC + e] = e & 1 ? dw[j][e / 2].y : dw[j][e / 2].x;
                mine[A.n + i * VEC + e] = e & 1 ? db[j][e / 2].y : db[j][e / 2].x;
            }
        }
    }
    if constexpr (G == 32) {
        // the block's 8 warps add up in shared memory first
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * A.n; c += GroupShape<G>::BLOCK) {
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) s += smem[(int64_t)r * 2 * A.n + c];
            out[c] = s;
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
        back_terms<T, VEC>(load_vec<T, VEC>(x + (int64_t)i * VEC), load_vec<T, VEC>(d + (int64_t)i * VEC), w, minus_mean, rstd, c1, c2,
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
        const float2 rstd = both(A.stats[A.rows + row]);
        const BackTerms<P> r =
            back_terms<T, VEC>(load_vec_stream<T, VEC>(static_cast<const T*>(A.x) + row * A.ld_x + col),
                               load_vec_stream<T, VEC>(static_cast<const T*>(A.dy) + row * A.ld_dy + col), w,
                               both(-A.stats[row]), rstd, c1, c2, dw, db);
        store_vec<T, VEC>(static_cast<T*>(A.dx) + row * A.ld_dx + col,
                          back_result<T, VEC>(r, rstd, both(-A.row_sums[2 * row]), both(-A.row_sums[2 * row + 1])));
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
constexpr int REDUCE_WARPS = 16;
__global__ void __launch_bounds__(REDUCE_WARPS * 32) k_norm_reduce(const float* partial, int parts, int n, float* dw, float* db,
                                                                   int accumulate) {
    __shared__ float s[REDUCE_WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;              // 0 .. 2n - 1
    float a = 0.f;
    if (c < 2 * n) {
#pragma unroll 8
        for (int p = warp; p < parts; p += REDUCE_WARPS) a += partial[(int64_t)p * 2 * n + c];
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

template <typename T, int VEC>
int launch_norm(const NormArgs& A, cudaStream_t st) {
    const int n = A.n;
#define NORM(G, E)                                                                                                  \
    do {                                                                                                            \
        const int64_t grid = (A.rows + GroupShape<G>::ROWS - 1) / GroupShape<G>::ROWS;                              \
        if (grid > 0x7fffffff) return SSGD_EINVAL;                                                                  \
        k_layer_norm<T, VEC, G, E><<<(unsigned)grid, GroupShape<G>::BLOCK, 0, st>>>(A);                             \
        return launched();                                                                                          \
    } while (0)
    constexpr int LONG = VEC == 1 ? 32 : 64;           // a vector of one element wastes half of a pair's registers
    if (n <= 32 * 16) NORM(32, 16);
    if (n <= 32 * LONG) NORM(32, LONG);
    if (n <= 128 * 32) NORM(128, 32);
    if (n <= 256 * 32) NORM(256, 32);
    if (n <= 512 * 32) NORM(512, 32);
#undef NORM
    if (A.rows > 0x7fffffff) return SSGD_EINVAL;
    k_layer_norm_wide<T, VEC><<<(unsigned)A.rows, WIDE, 0, st>>>(A);
    return launched();
}

constexpr int64_t PART_BLOCKS = 148 * 4;         // at most so many partial sums of dw and db
constexpr int BACK_NARROW = 512 * 8;             // rows up to here stay in a block's registers, whatever the format

template <typename T, int VEC>
int launch_norm_back(const NormBackArgs& A, int sms, int* parts, cudaStream_t st) {
    const int n = A.n;
    int64_t grid = 0;
#define NORM_BACK(G, E)                                                                                             \
    do {                                                                                                            \
        const size_t smem = G == 32 && A.partial ? (size_t)GroupShape<G>::ROWS * 2 * n * 4 : 0;                     \
        int per_sm = 0;                                                                                             \
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k_layer_norm_back<T, VEC, G, E>,                 \
                                                          GroupShape<G>::BLOCK, smem) != cudaSuccess || per_sm < 1) \
            return SSGD_ECUDA;                                                                                      \
        grid = (A.rows + GroupShape<G>::ROWS - 1) / GroupShape<G>::ROWS;                                            \
        if (grid > (int64_t)sms * per_sm) grid = (int64_t)sms * per_sm;                                             \
        if (grid > PART_BLOCKS) grid = PART_BLOCKS;                                                                 \
        k_layer_norm_back<T, VEC, G, E><<<(unsigned)grid, GroupShape<G>::BLOCK, smem, st>>>(A);                     \
        *parts = (int)grid;                                                                                         \
        return launched();                                                                                          \
    } while (0)
    // 16 elements of 16 bits per thread or 8 of 32 bits: with their sums and the next row's on the way, 128 registers
    constexpr int E = sizeof(T) == 4 || VEC == 1 ? 8 : 16;
    if (n <= 32 * E) NORM_BACK(32, E);
    if (n <= 128 * E) NORM_BACK(128, E);
    if (n <= 256 * E) NORM_BACK(256, E);
    if (n <= 512 * E) NORM_BACK(512, E);
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
    return BY_FORMAT(launch_norm, fmt_x, vec, A, st);
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
    NormBackArgs A{dy, ld_dy, x, ld_x, w, fmt_w == SSGD_FMT_F32, stats, rows, (int32_t)n, dx, ld_dx, nullptr, nullptr};
    float* base = static_cast<float*>(workspace);
    A.row_sums = base;
    if (n > BACK_NARROW) base += 2 * rows;
    A.partial = dw || db ? base : nullptr;
    const int vec = vec_of(es, n, {dy, x, dx}, {ld_dy, ld_x, ld_dx}, {w}, A.w_f32);
    int parts = 0;
    e = BY_FORMAT(launch_norm_back, fmt_x, vec, A, sms, &parts, st);
    if (e || !A.partial) return e;
    k_norm_reduce<<<(unsigned)((2 * n + 31) / 32), REDUCE_WARPS * 32, 0, st>>>(A.partial, parts, (int)n, dw, db, accumulate);
    return launched();
}

}  // extern "C"
