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
__device__ __forceinline__ void load_param(const void* w, bool w_f32, int col, float (&f)[VEC]) {
    if (w_f32) {
        const float* p = static_cast<const float*>(w) + col;
        if constexpr (VEC == 8) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        } else {
            unpack(load_vec<float, VEC>(p), f);
        }
    } else {
        unpack(load_vec<T, VEC>(static_cast<const T*>(w) + col), f);
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
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = t + j * G;
        if (i < nv) v[j] = load_vec_stream<T, VEC>(x + (int64_t)i * VEC);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (t + j * G < nv) {
            float f[VEC];
            unpack(v[j], f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s += f[e];
        }
    }
    const float mean = group_sum<G>(s, slot[0]) / (float)A.n;
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (t + j * G < nv) {
            float f[VEC];
            unpack(v[j], f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) { const float d = f[e] - mean; q = fmaf(d, d, q); }
        }
    }
    const float rstd = 1.0f / sqrtf(group_sum<G>(q, slot[1]) / (float)A.n + A.eps);
    if (t == 0) { A.stats[row] = mean; A.stats[A.rows + row] = rstd; }
    T* y = static_cast<T*>(A.y) + row * A.ld_y;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = t + j * G;
        if (i < nv) {
            float f[VEC], w[VEC], b[VEC];
            unpack(v[j], f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = (f[e] - mean) * rstd;
            if (A.w) {
                load_param<T, VEC>(A.w, A.w_f32, i * VEC, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] *= w[e];
            }
            if (A.b) {
                load_param<T, VEC>(A.b, A.w_f32, i * VEC, b);
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] += b[e];
            }
            store_vec<T, VEC>(y + (int64_t)i * VEC, pack<T, VEC>(f));
        }
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
    float s = 0.f, q = 0.f, f[VEC];
    for (int i = t; i < nv; i += WIDE) {
        unpack(load_vec<T, VEC>(x + (int64_t)i * VEC), f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += f[e];
    }
    const float mean = group_sum<WIDE>(s, slot[0]) / (float)A.n;
    for (int i = t; i < nv; i += WIDE) {
        unpack(load_vec<T, VEC>(x + (int64_t)i * VEC), f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) { const float d = f[e] - mean; q = fmaf(d, d, q); }
    }
    const float rstd = 1.0f / sqrtf(group_sum<WIDE>(q, slot[1]) / (float)A.n + A.eps);
    if (t == 0) { A.stats[row] = mean; A.stats[A.rows + row] = rstd; }
    T* y = static_cast<T*>(A.y) + row * A.ld_y;
    for (int i = t; i < nv; i += WIDE) {
        float w[VEC], b[VEC];
        unpack(load_vec<T, VEC>(x + (int64_t)i * VEC), f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = (f[e] - mean) * rstd;
        if (A.w) {
            load_param<T, VEC>(A.w, A.w_f32, i * VEC, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] *= w[e];
        }
        if (A.b) {
            load_param<T, VEC>(A.b, A.w_f32, i * VEC, b);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] += b[e];
        }
        store_vec<T, VEC>(y + (int64_t)i * VEC, pack<T, VEC>(f));
    }
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

template <typename T, int VEC, int G, int E>
__global__ void __launch_bounds__(GroupShape<G>::BLOCK) k_layer_norm_back(const NormBackArgs A) {
    constexpr int NV = E / VEC, ROWS = GroupShape<G>::ROWS;
    extern __shared__ float smem[];                    // G = 32: [8][2][n] partial sums at the end
    __shared__ float2 slot[2][32];
    const int t = threadIdx.x % G, sub = threadIdx.x / G;
    const int nv = A.n / VEC;
    const float inv_n = 1.0f / (float)A.n;
    float dw[E], db[E];
#pragma unroll
    for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.f;
    Vec<T, VEC> vx[NV], vd[NV];
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + sub;
    int turn = 0;
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
    };
    for (; row < A.rows; row += step) {
        fetch(row);
        const float mean = A.stats[row], rstd = A.stats[A.rows + row];
        float c1 = 0.f, c2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * G;
            if (i < nv) {
                float fx[VEC], fd[VEC], w[VEC];
                unpack(vx[j], fx);
                unpack(vd[j], fd);
                if (A.w) load_param<T, VEC>(A.w, A.w_f32, i * VEC, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float h = (fx[e] - mean) * rstd;
                    const float a = A.w ? fd[e] * w[e] : fd[e];
                    c1 += a;
                    c2 = fmaf(a, h, c2);
                    dw[j * VEC + e] = fmaf(fd[e], h, dw[j * VEC + e]);
                    db[j * VEC + e] += fd[e];
                }
            }
        }
        c1 = warp_sum(c1);
        c2 = warp_sum(c2);
        if constexpr (G > 32) {
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
            constexpr int NW = GroupShape<G>::WARPS;
            if (lane == 0) slot[turn][warp] = make_float2(c1, c2);
            __syncthreads();
            const float2 p = lane < NW ? slot[turn][lane] : make_float2(0.f, 0.f);
            c1 = warp_sum(p.x);
            c2 = warp_sum(p.y);
            turn ^= 1;
        }
        c1 *= inv_n;
        c2 *= inv_n;
        T* dx = static_cast<T*>(A.dx) + row * A.ld_dx;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * G;
            if (i < nv) {
                float fx[VEC], fd[VEC], w[VEC];
                unpack(vx[j], fx);
                unpack(vd[j], fd);
                if (A.w) load_param<T, VEC>(A.w, A.w_f32, i * VEC, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float h = (fx[e] - mean) * rstd;
                    const float a = A.w ? fd[e] * w[e] : fd[e];
                    fd[e] = rstd * (a - c1 - h * c2);
                }
                store_vec<T, VEC>(dx + (int64_t)i * VEC, pack<T, VEC>(fd));
            }
        }
    }
    if (!A.partial) return;
    float* out = A.partial + (int64_t)blockIdx.x * 2 * A.n;
    if constexpr (G == 32) {
        // the block's 8 warps add up in shared memory first
        float* mine = smem + (int64_t)sub * 2 * A.n;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * G;
            if (i < nv) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    mine[i * VEC + e] = dw[j * VEC + e];
                    mine[A.n + i * VEC + e] = db[j * VEC + e];
                }
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * A.n; c += GroupShape<G>::BLOCK) {
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) s += smem[(int64_t)r * 2 * A.n + c];
            out[c] = s;
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * G;
            if (i < nv) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    out[i * VEC + e] = dw[j * VEC + e];
                    out[A.n + i * VEC + e] = db[j * VEC + e];
                }
            }
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
    const float mean = A.stats[row], rstd = A.stats[A.rows + row];
    const int nv = A.n / VEC;
    float c1 = 0.f, c2 = 0.f;
    for (int i = threadIdx.x; i < nv; i += WIDE) {
        float fx[VEC], fd[VEC], w[VEC];
        unpack(load_vec<T, VEC>(x + (int64_t)i * VEC), fx);
        unpack(load_vec<T, VEC>(d + (int64_t)i * VEC), fd);
        if (A.w) load_param<T, VEC>(A.w, A.w_f32, i * VEC, w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float a = A.w ? fd[e] * w[e] : fd[e];
            c1 += a;
            c2 = fmaf(a, (fx[e] - mean) * rstd, c2);
        }
    }
    c1 = group_sum<WIDE>(c1, slot[0]);
    c2 = group_sum<WIDE>(c2, slot[1]);
    if (threadIdx.x == 0) {
        A.row_sums[2 * row] = c1 / (float)A.n;
        A.row_sums[2 * row + 1] = c2 / (float)A.n;
    }
}

// Second pass: blockIdx.x is a slab of 256 vectors of columns, blockIdx.y a share of the rows.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) k_norm_back_slab(const NormBackArgs A) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= A.n / VEC) return;
    const int64_t col = (int64_t)i * VEC;
    float dw[VEC], db[VEC], w[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) { dw[e] = db[e] = 0.f; w[e] = 1.f; }
    if (A.w) load_param<T, VEC>(A.w, A.w_f32, (int)col, w);
    for (int64_t row = blockIdx.y; row < A.rows; row += gridDim.y) {
        float fx[VEC], fd[VEC];
        unpack(load_vec_stream<T, VEC>(static_cast<const T*>(A.x) + row * A.ld_x + col), fx);
        unpack(load_vec_stream<T, VEC>(static_cast<const T*>(A.dy) + row * A.ld_dy + col), fd);
        const float mean = A.stats[row], rstd = A.stats[A.rows + row];
        const float c1 = A.row_sums[2 * row], c2 = A.row_sums[2 * row + 1];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float h = (fx[e] - mean) * rstd;
            dw[e] = fmaf(fd[e], h, dw[e]);
            db[e] += fd[e];
            fd[e] = rstd * (fd[e] * w[e] - c1 - h * c2);
        }
        store_vec<T, VEC>(static_cast<T*>(A.dx) + row * A.ld_dx + col, pack<T, VEC>(fd));
    }
    if (!A.partial) return;
    float* out = A.partial + (int64_t)blockIdx.y * 2 * A.n;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        out[col + e] = dw[e];
        out[A.n + col + e] = db[e];
    }
}

// dw[c], db[c] = sum over the blocks' partials, in a fixed order: 32 columns per block, 8 warps share the partials.
__global__ void __launch_bounds__(256) k_norm_reduce(const float* partial, int parts, int n, float* dw, float* db, int accumulate) {
    __shared__ float s[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;              // 0 .. 2n - 1
    float a = 0.f;
    if (c < 2 * n)
        for (int p = warp; p < parts; p += 8) a += partial[(int64_t)p * 2 * n + c];
    s[warp][lane] = a;
    __syncthreads();
    if (warp == 0 && c < 2 * n) {
#pragma unroll
        for (int k = 1; k < 8; ++k) a += s[k][lane];
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
    if (n <= 32 * 16) NORM(32, 16);
    if (n <= 32 * 64) NORM(32, 64);
    if (n <= 128 * 32) NORM(128, 32);
    if (n <= 256 * 32) NORM(256, 32);
    if (n <= 512 * 32) NORM(512, 32);
#undef NORM
    if (A.rows > 0x7fffffff) return SSGD_EINVAL;
    k_layer_norm_wide<T, VEC><<<(unsigned)A.rows, WIDE, 0, st>>>(A);
    return launched();
}

constexpr int64_t PART_BLOCKS = 148 * 4;         // at most so many partial sums of dw and db
constexpr int BACK_MAX_N = 512 * 16;             // rows up to here stay in a block's registers

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
    if (n <= 32 * 16) NORM_BACK(32, 16);
    if (n <= 128 * 16) NORM_BACK(128, 16);
    if (n <= 256 * 16) NORM_BACK(256, 16);
    if (n <= BACK_MAX_N) NORM_BACK(512, 16);
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
    if (n > BACK_MAX_N) bytes += (size_t)rows * 2 * 4;
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
    if (n > BACK_MAX_N) base += 2 * rows;
    A.partial = dw || db ? base : nullptr;
    const int vec = vec_of(es, n, {dy, x, dx}, {ld_dy, ld_x, ld_dx}, {w}, A.w_f32);
    int parts = 0;
    e = BY_FORMAT(launch_norm_back, fmt_x, vec, A, sms, &parts, st);
    if (e || !A.partial) return e;
    k_norm_reduce<<<(unsigned)((2 * n + 31) / 32), 256, 0, st>>>(A.partial, parts, (int)n, dw, db, accumulate);
    return launched();
}

}  // extern "C"
