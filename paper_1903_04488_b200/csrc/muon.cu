// muon.cu -- orthogonalised matrices, by themselves (ssgd_orthogonalize) and as an optimizer's step (ssgd_muon_step).
//
// The mathematics.  With x_0 = u / (|u| + eps), |u| the root of the sum of squares, every step applies the odd polynomial
// q(s) = a s + b s^3 + c s^5 to the singular values:
//   A = x x',  B = b A + c A A,  x <- a x + B x          (rows <= cols; otherwise A = x' x and x <- a x + x B)
// Three products of matrices per step, fp16 operands, fp32 accumulators; A and B are symmetric.
//
// Precision.  fp16 keeps 11 bits, and a plain iteration in 16 bits loses what it rounds: singular values that are far below the
// largest are multiplied by a at every step, and with them the rounding of x (to 1e-1 of the result at a spread of 1e4).  Here
//   - x is kept as the sum of two fp16 numbers (22 bits).  The term a x, which is what small singular values live on, takes both;
//     only the operands of the products are rounded, and their error lies along the large singular values
//   - the diagonals of A and B, which all but carry the matrices when x is nearly orthogonal, are kept in fp32 beside them:
//       A = R + D:  A A = R R + R (d_i + d_j) + D D;    B = Q + E:  a x + B x = (a + e_i) x + Q x
// leaving 1e-4 to 1.5e-3 of the result (less than its rounding to bfloat16, 1.7e-3).  Where the result has more bits than bfloat16,
// or the caller says so, every matrix is a sum of two fp16 numbers and a product takes three (high high, high low, low high): 4e-7
// to 7e-6, where the same iteration in fp32 is off by 4e-7 to 1.5e-5.  The tensor cores' sums truncate, which shows where few long rows are
// multiplied with themselves (4 x 536: 3.7e-6, fp32 1.3e-6).  Roundings that do not average out take matrices of less than 512 numbers
// to 7e-3 with one product.
// The stored numbers are 1024 times the true ones: x is at most 1.2 and an element mostly far below, so that the second number stays
// clear of fp16's subnormals.
//
// Measured: 8 x 1024 x 2816 bf16 0.72 ms, 550 TFLOP/s of what has to be computed; the matrices of two transformer blocks (2048, 5632) bf16
// 2.4 to 2.5 ms, 780 to 810; of eight (768, 2048) fp32 with three products 1.7 ms, 235.  What bounds the large ones is what an SM takes from L2: 48 to 50
// bytes per cycle, 681 cycles for 64 of the contraction of a 256 x 256 tile, of which the products are 512.
//
// Layout.  All matrices of a call go through every launch together: prepare (momentum and sums of squares; division and layout),
// then 3 launches per step, whose tiles are dealt out over the SMs.  Matrices live in the workspace as blocks (umma.cuh), padded with
// zeros to 64; block (r, c) of a matrix of R x C blocks is the (c R + r)-th.
#include <algorithm>
#include <cmath>

#include "formats.cuh"
#include "umma.cuh"

using namespace ssgd;
using namespace ssgd::umma;

namespace {

constexpr float SCALE = 1024.f;
constexpr int MAX_GROUP = 224;                      // matrices of one set of launches: their descriptors are arguments of the first
constexpr int64_t GROUP_ELEMENTS = (int64_t)1 << 27;  // and no more than this many elements, sides rounded up to 64, unless one matrix has them
constexpr int STRIP_BLOCKS = 4;                     // what a CTA of the preparation takes: 64 rows of 256 columns

enum Kind { GRAM, POLYNOMIAL, APPLY, FINISH };      // A, B, x of the next step, the result

struct Matrix {
    void* out; const void* in; float* m;
    int64_t ld_out, ld_in;
    int32_t rows, cols, rb, cb, mb;                 // size; size in blocks; blocks of the shorter side
    uint32_t x0, x1, a, b;                          // first blocks: x at even and at odd steps, A, B.  Second numbers lie behind the first
    uint32_t vec;                                   // d and e, mb * 64 floats each
    int32_t strip0, strips, first[4];               // first strip and first tile of each product among those of all matrices
    float update;                                   // lr * scale
    __host__ __device__ uint32_t x(int which) const { return which ? x1 : x0; }
    __host__ __device__ bool tall() const { return rb > cb || (rb == cb && rows > cols); }
};
struct Group { Matrix m[MAX_GROUP]; };
static_assert(sizeof(Group) <= 30 * 1024, "an argument of a kernel");

// Where things are in the workspace
struct Space {
    Matrix* matrices;
    double* sums;
    float* vec;
    uint8_t* blocks;
};
struct Common {
    Space at;
    int32_t count;
    int32_t fmt_in, fmt_out;
    bool split;                                     // two numbers in A and B too, three products
    bool nesterov, update;                          // update: out is a parameter to be moved, otherwise it gets the result
    float momentum, share, decay, eps;              // share: 1 - momentum, which fp32 would not hold as 1 less a rounded momentum
    float a, b, c;
    const float* grad_scale;
};

__device__ int g_error;                             // set by a wait that ran out

// ---- preparation -------------------------------------------------------------------------------------

// Whether four neighbours from a multiple of four on may be read and written at once
template <typename T>
__device__ __forceinline__ bool may_load_four(const Matrix& M) {
    return M.ld_in % 4 == 0 && (reinterpret_cast<uintptr_t>(M.in) & (4 * sizeof(T) - 1)) == 0 &&
           (!M.m || (M.cols % 4 == 0 && (reinterpret_cast<uintptr_t>(M.m) & 15u) == 0));
}

// The matrix of a strip or tile: the last whose first is not beyond it
template <typename F>
__device__ __forceinline__ int matrix_of(int count, int what, F first) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first(mid) <= what) lo = mid; else hi = mid;
    }
    return lo;
}

constexpr int PREPARE_THREADS = 256;

__device__ __forceinline__ double block_sum(double v, double* shared) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < PREPARE_THREADS / 32; ++w) s += shared[w];
    return s;
}

// A block of the preparation: thread t has columns 4 (t mod 16) .. of rows t / 16 + 16 i.  What is not there is zero.
constexpr int SHARE = 4;
template <typename T> struct Share {
    Vec<T, 4> g[SHARE];
    Vec<float, 4> m[SHARE];
};
template <typename T>
__device__ __forceinline__ void load_block(const Matrix& M, int r0, int c0, bool vector, Share<T>& s) {
    const int c = c0 + (int)threadIdx.x % 16 * 4, r = r0 + (int)threadIdx.x / 16;
    const T* in = static_cast<const T*>(M.in) + (int64_t)r * M.ld_in + c;
    const float* m = M.m + (int64_t)r * M.cols + c;
    if (vector && r0 + BLOCK <= M.rows && c0 + BLOCK <= M.cols) {      // the same for the whole CTA: all loads on their way at once
#pragma unroll
        for (int i = 0; i < SHARE; ++i) s.g[i] = load_vec<T, 4>(in + (int64_t)(16 * i) * M.ld_in);
        if (M.m) {
#pragma unroll
            for (int i = 0; i < SHARE; ++i) s.m[i] = load_vec<float, 4>(m + (int64_t)(16 * i) * M.cols);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < SHARE; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool there = r + 16 * i < M.rows && c + e < M.cols;
            s.g[i].e[e] = there ? in[(int64_t)(16 * i) * M.ld_in + e] : from_f32<T>(0.f);
            s.m[i].e[e] = there && M.m ? m[(int64_t)(16 * i) * M.cols + e] : 0.f;
        }
    }
}

// The thread's i-th four numbers of a block: the new momentum, left in s.m, and what is to be made orthogonal
template <typename T>
__device__ __forceinline__ float4 momentum_of(const Common& C, const Matrix& M, Share<T>& s, int i, float scale) {
    float u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        u[e] = to_f32(s.g[i].e[e]);
        if (M.m) {
            const float in = u[e] * scale;
            s.m[i].e[e] = fmaf(C.momentum, s.m[i].e[e], C.share * in);
            u[e] = C.nesterov ? fmaf(C.momentum, s.m[i].e[e], C.share * in) : s.m[i].e[e];
        }
    }
    return make_float4(u[0], u[1], u[2], u[3]);
}
// The same where the momentum is the new one already
template <typename T>
__device__ __forceinline__ float4 stored_momentum_of(const Common& C, const Matrix& M, const Share<T>& s, int i, float scale) {
    float u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        u[e] = to_f32(s.g[i].e[e]);
        if (M.m) u[e] = C.nesterov ? fmaf(C.momentum, s.m[i].e[e], C.share * (u[e] * scale)) : s.m[i].e[e];
    }
    return make_float4(u[0], u[1], u[2], u[3]);
}
// The first n of the four, squared and added in 64 bits
__device__ __forceinline__ double squares(const float4& u, int n) {
    return (n > 0 ? (double)u.x * u.x : 0.0) + (n > 1 ? (double)u.y * u.y : 0.0) + (n > 2 ? (double)u.z * u.z : 0.0) +
           (n > 3 ? (double)u.w * u.w : 0.0);
}
// n: how many of the four there are
template <typename T>
__device__ __forceinline__ void put_momentum(const Matrix& M, const Share<T>& s, int i, int r, int c, int n, bool vector) {
    float* to = M.m + (int64_t)r * M.cols + c;
    if (vector && n >= 4) store_vec<float, 4>(to, s.m[i]);
    else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) to[e] = s.m[i].e[e];
    }
}
// 1 / (norm + eps), from the sum of squares, as a factor near one and two powers of two: the norm may lie beyond fp32
struct Inverse {
    float power[2], factor;
    __device__ __forceinline__ Inverse(double sum, float eps) {
        const double inv = 1.0 / (sqrt(sum) + (double)eps);
        int exponent = 0;
        factor = (float)(inv > 0.0 && inv < (double)INFINITY ? frexp(inv, &exponent) : inv) * SCALE;
        exponent = min(max(exponent, -252), 254);
        power[0] = ldexpf(1.f, exponent / 2);
        power[1] = ldexpf(1.f, exponent - exponent / 2);
    }
    __device__ __forceinline__ float of(float u) const { return u * power[0] * power[1] * factor; }
};

// m <- momentum m + (1 - momentum) g, and the sum of squares of what is to be made orthogonal, per strip.  Squares are added in 64
// bits: they may leave the range of 32.
template <typename T>
__global__ void __launch_bounds__(PREPARE_THREADS, 4) k_momentum(const __grid_constant__ Group G, const __grid_constant__ Common C) {
    __shared__ double shared[PREPARE_THREADS / 32];
    successor_wait();
    successor_may_start();
    if (blockIdx.x == 0) {
        const uint32_t* from = reinterpret_cast<const uint32_t*>(&G);
        uint32_t* to = reinterpret_cast<uint32_t*>(C.at.matrices);
        for (int i = threadIdx.x; i < C.count * (int)(sizeof(Matrix) / 4); i += PREPARE_THREADS) to[i] = from[i];
    }
    const int strip = blockIdx.x;
    const Matrix& M = G.m[matrix_of(C.count, strip, [&](int i) { return G.m[i].strip0; })];
    const int local = strip - M.strip0, r0 = local % M.rb * BLOCK, cblock0 = local / M.rb * STRIP_BLOCKS;
    const bool vector = may_load_four<T>(M);
    const float scale = C.grad_scale ? *C.grad_scale : 1.f;
    double sum = 0.0;
    for (int cblock = cblock0; cblock < min(cblock0 + STRIP_BLOCKS, M.cb); ++cblock) {
        Share<T> s;
        load_block<T>(M, r0, cblock * BLOCK, vector, s);
        const int c = cblock * BLOCK + (int)threadIdx.x % 16 * 4;
#pragma unroll
        for (int i = 0; i < SHARE; ++i) {
            const int r = r0 + (int)threadIdx.x / 16 + 16 * i, n = r < M.rows ? M.cols - c : 0;
            const float4 u = momentum_of(C, M, s, i, scale);
            if (M.m) put_momentum(M, s, i, r, c, n, vector);
            sum += squares(u, n);
        }
    }
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) C.at.sums[strip] = sum;
}

// Two numbers as fp16, and what that leaves
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
    const __half2 h = __floats2half2_rn(a, b);
    const float2 back = __half22float2(h);
    const __half2 l = __floats2half2_rn(a - back.x, b - back.y);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = *reinterpret_cast<const uint32_t*>(&l);
}
__device__ __forceinline__ float2 halves(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// x = u / (|u| + eps) as blocks
template <typename T>
__global__ void __launch_bounds__(PREPARE_THREADS, 4) k_layout(const __grid_constant__ Common C) {
    __shared__ double shared[PREPARE_THREADS / 32];
    successor_wait();
    successor_may_start();
    const int strip = blockIdx.x;
    const Matrix M = C.at.matrices[matrix_of(C.count, strip, [&](int i) { return C.at.matrices[i].strip0; })];
    const int local = strip - M.strip0, rblock = local % M.rb, cblock0 = local / M.rb * STRIP_BLOCKS, cblock1 = min(cblock0 + STRIP_BLOCKS, M.cb);
    const bool vector = may_load_four<T>(M);
    // what is read need not wait for the sum, nor the next block for this one
    Share<T> s;
    load_block<T>(M, rblock * BLOCK, cblock0 * BLOCK, vector, s);
    double sum = 0.0;
    for (int i = threadIdx.x; i < M.strips; i += PREPARE_THREADS) sum += C.at.sums[M.strip0 + i];
    sum = block_sum(sum, shared);
    const Inverse inv(sum, C.eps);
    const float scale = C.grad_scale ? *C.grad_scale : 1.f;
    const int64_t second = (int64_t)M.rb * M.cb * BLOCK_BYTES;
    for (int cblock = cblock0; cblock < cblock1; ++cblock) {
        uint8_t* block = C.at.blocks + (int64_t)(M.x0 + (uint32_t)cblock * M.rb + rblock) * BLOCK_BYTES;
        float4 u[SHARE];
#pragma unroll
        for (int i = 0; i < SHARE; ++i) u[i] = stored_momentum_of(C, M, s, i, scale);
        if (cblock + 1 < cblock1) load_block<T>(M, rblock * BLOCK, (cblock + 1) * BLOCK, vector, s);
#pragma unroll
        for (int i = 0; i < SHARE; ++i) {
            const int rr = (int)threadIdx.x / 16 + 16 * i, cc = (int)threadIdx.x % 16 * 4;
            const int n = rblock * BLOCK + rr < M.rows ? M.cols - cblock * BLOCK - cc : 0;
            uint2 hi, lo;                           // the padding is 0 whatever the factor is
            split2(n > 0 ? inv.of(u[i].x) : 0.f, n > 1 ? inv.of(u[i].y) : 0.f, hi.x, lo.x);
            split2(n > 2 ? inv.of(u[i].z) : 0.f, n > 3 ? inv.of(u[i].w) : 0.f, hi.y, lo.y);
            uint8_t* to = block + piece_at(rr, cc / 8) + cc % 8 * 2;
            *reinterpret_cast<uint2*>(to) = hi;
            *reinterpret_cast<uint2*>(to + second) = lo;
        }
    }
}

// ---- products ----------------------------------------------------------------------------------------

// A tile is 256 rows and COLS columns, of a pair of CTAs that has half of the rows each.  What a tile loads per block of the contraction
// grows with its sides, what it computes with their product: 256 x 256 needs 32 KB into each SM per 512 cycles at the tensor cores' full rate,
// 18 TB/s from L2 at 1.9 GHz, 128 x 128 by single CTAs twice that.  Where the larger tiles are too few, 256 x 128.
constexpr int TILE_ROWS = 256;
constexpr int RING = 192 * 1024;                    // bytes of operands on their way
constexpr int RESULT_WARPS = 8;
constexpr int THREADS = 32 * (RESULT_WARPS + 4);     // one more warp copies, one issues products, two complete a group of four
constexpr int SCRATCH = 4096;                       // of each result warp: 32 x 32 numbers change hands there
constexpr int CHUNK = 4;                            // blocks of the contraction that are added up by the tensor cores alone (SPLIT)

// Bytes of a stage of the ring: 128 rows of A and half of the columns of B; with SPLIT the first and the second numbers
template <int COLS, bool SPLIT> constexpr int STAGE = (2 + COLS / 128) * BLOCK_BYTES * (SPLIT ? 2 : 1);
template <int COLS, bool SPLIT> constexpr int STAGES = RING / STAGE<COLS, SPLIT>;

constexpr int LAUNCH_REGISTERS = 168;
struct Shared {
    uint64_t full[8], empty[8], done[2], taken[2];
    uint32_t tmem;
    int gave_up;
    int32_t first[MAX_GROUP];
};
constexpr int SHARED_BYTES = 1024 + RING + RESULT_WARPS * SCRATCH + (int)sizeof(Shared);
static_assert(SHARED_BYTES <= 227 * 1024, "shared memory of a CTA");

// One operand of a product: blocks [R][C]
struct Operand {
    uint32_t base, second;                          // first block; blocks from the first numbers to the second
    int32_t R, mn_blocks;
    bool mn_major;
    // the first block of the contraction at rows or columns 64 mn ..; beyond the edge, rows or columns that are not stored
    __device__ __forceinline__ int32_t at(int mn) const {
        mn = min(mn, mn_blocks - 1);
        return (int32_t)(base + (uint32_t)(mn_major ? mn * R : mn));
    }
    __device__ __forceinline__ int32_t step() const { return mn_major ? 1 : R; }
};
struct Product {
    Operand A, B;
    int32_t steps;                                  // blocks of the contraction
};

template <Kind KIND>
__device__ __forceinline__ Product product_of(const Matrix& M, int which) {
    const uint32_t xs = (uint32_t)M.rb * (uint32_t)M.cb, ms = (uint32_t)M.mb * (uint32_t)M.mb;
    const bool tall = M.tall();
    Product P;
    if (KIND == GRAM) {
        P.A = Operand{M.x(which), xs, M.rb, M.mb, tall};
        P.B = P.A;
        P.steps = tall ? M.rb : M.cb;
    } else if (KIND == POLYNOMIAL) {
        P.A = Operand{M.a, ms, M.mb, M.mb, false};
        P.B = P.A;
        P.steps = M.mb;
    } else {
        const Operand q{M.b, ms, M.mb, M.mb, false};
        P.A = tall ? Operand{M.x(which), xs, M.rb, M.rb, false} : q;
        P.B = tall ? q : Operand{M.x(which), xs, M.rb, M.cb, true};
        P.steps = M.mb;
    }
    return P;
}

// Tiles of a symmetric product with n blocks to a side: those that reach the diagonal or lie below it, row by row.  With 256 columns row I has
// I + 1 of them, with 128 2 I + 2 (but no more than there are).
template <int COLS>
__host__ __device__ inline int64_t symmetric_tiles(int64_t n) {
    const int64_t rows = (n + 3) / 4, cols = (n + COLS / BLOCK - 1) / (COLS / BLOCK);
    return COLS == 256 ? rows * (rows + 1) / 2 : rows * (rows + 1) - (2 * rows - cols);
}
template <int COLS>
__host__ __device__ inline int64_t all_tiles(int64_t rb, int64_t cb) {
    return (rb + 3) / 4 * ((cb + COLS / BLOCK - 1) / (COLS / BLOCK));
}
struct Tile { int row, col; };                      // first blocks
template <Kind KIND, int COLS>
__device__ __forceinline__ Tile tile_of(const Matrix& M, int i) {
    if (KIND == GRAM || KIND == POLYNOMIAL) {
        int I;
        if (COLS == 256) {
            I = (int)((sqrtf(8.f * (float)i + 1.f) - 1.f) * 0.5f);
            while (I * (I + 1) / 2 > i) --I;
            while ((I + 1) * (I + 2) / 2 <= i) ++I;
            return Tile{I * 4, (i - I * (I + 1) / 2) * 4};
        }
        I = (int)((sqrtf(4.f * (float)i + 1.f) - 1.f) * 0.5f);
        while (I * (I + 1) > i) --I;
        while ((I + 1) * (I + 2) <= i) ++I;
        return Tile{I * 4, (i - I * (I + 1)) * 2};
    }
    const int rows = (M.rb + 3) / 4;
    return Tile{i % rows * 4, i / rows * (COLS / BLOCK)};
}

// ---- results ------------------------------------------------------------------------------------------
//
// A warp has 32 rows of the tile and takes 32 columns at a time.  Tensor memory gives a row to a lane; through 4 KB of shared
// memory they are dealt out anew, eight neighbours of a row to a lane and four lanes to 64 bytes of a block's row, which is how blocks
// and outputs are read and written.

__device__ __forceinline__ uint32_t word_at(int r, int piece) { return (uint32_t)(r * 128 + ((piece ^ (r & 7)) << 4)); }
// x, of which the compiler knows nothing
__device__ __forceinline__ int opaque(int x) {
    asm volatile("" : "+r"(x));
    return x;
}

// 32 x 32 fp16 numbers; neither eight rows of a column nor rows meet in a bank
__device__ __forceinline__ uint32_t half_at(int r, int piece) { return (uint32_t)(r * 64 + ((piece ^ (((r >> 1) ^ (r >> 3)) & 3)) << 4)); }

// What is the same for all results of a tile
template <Kind KIND> struct Job {
    uint8_t* blocks;                                // of C.at
    uint32_t from, to;                              // first blocks of what is added (A, x) and of the result
    int32_t R;                                      // blocks to a column
    int32_t second;                                 // blocks from the first numbers to the second
    float* vec;                                     // d, and behind it e
    int32_t side;                                   // floats of d
    bool tall;
    __device__ __forceinline__ Job(const Common& C, const Matrix& M, int which) {
        constexpr bool SYMMETRIC = KIND == GRAM || KIND == POLYNOMIAL;
        blocks = C.at.blocks;
        from = KIND == POLYNOMIAL ? M.a : M.x(which);
        to = KIND == GRAM ? M.a : KIND == POLYNOMIAL ? M.b : M.x(which ^ 1);
        R = SYMMETRIC ? M.mb : M.rb;
        second = SYMMETRIC ? M.mb * M.mb : M.rb * M.cb;
        vec = C.at.vec + M.vec;
        side = M.mb * BLOCK;
        tall = M.tall();
    }
    // The lane's piece of the first eight rows of the 32 x 32 numbers at row0, col0 (multiples of 32); eight rows further is 1 KB further
    __device__ __forceinline__ uint8_t* at(uint32_t first, int row0, int col0, int lane) const {
        return blocks + (int64_t)(first + (uint32_t)(col0 / BLOCK * R + row0 / BLOCK)) * BLOCK_BYTES +
               piece_at(row0 % BLOCK + lane / 4, col0 / 32 % 2 * 4 + lane % 4);
    }
};

// What a piece of results needs beside the products
template <Kind KIND, bool SPLIT> struct Source {
    static constexpr bool NEEDED = KIND != GRAM, BOTH = KIND != POLYNOMIAL || SPLIT;
    uint4 hi[NEEDED ? 4 : 1], lo[NEEDED && BOTH ? 4 : 1];
    float row[4], col[8];                           // d or e of the rows and columns, 0 where only the other counts
};

template <Kind KIND, bool SPLIT>
__device__ __forceinline__ void fetch(const Job<KIND>& J, int row0, int col0, int lane, Source<KIND, SPLIT>& s) {
    if constexpr (KIND == GRAM) return;
    const uint8_t* p = J.at(J.from, row0, col0, lane);
    const int64_t second = (int64_t)J.second * BLOCK_BYTES;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s.hi[i] = *reinterpret_cast<const uint4*>(p + i * 1024);
        if constexpr (Source<KIND, SPLIT>::BOTH) s.lo[i] = *reinterpret_cast<const uint4*>(p + i * 1024 + second);
    }
    const float* d = J.vec + (KIND == POLYNOMIAL ? 0 : J.side);
    const bool rows = KIND == POLYNOMIAL || !J.tall, cols = KIND == POLYNOMIAL || J.tall;
#pragma unroll
    for (int i = 0; i < 4; ++i) s.row[i] = rows ? d[row0 + i * 8 + lane / 4] : 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
    if (cols) {
        a = *reinterpret_cast<const float4*>(d + col0 + lane % 4 * 8);
        b = *reinterpret_cast<const float4*>(d + col0 + lane % 4 * 8 + 4);
    }
    s.col[0] = a.x; s.col[1] = a.y; s.col[2] = a.z; s.col[3] = a.w;
    s.col[4] = b.x; s.col[5] = b.y; s.col[6] = b.z; s.col[7] = b.w;
}

// Eight results in a row of the output
template <typename T>
__device__ __forceinline__ void put_output(const Common& C, const Matrix& M, int row, int col, const float (&v)[8]) {
    constexpr int VEC = 16 / sizeof(T);
    const int n = M.cols - col;
    if (row >= M.rows || n <= 0) return;
    T* out = static_cast<T*>(M.out) + (int64_t)row * M.ld_out + col;
    if (n >= 8 && (reinterpret_cast<uintptr_t>(out) & 15u) == 0) {
        Vec<T, VEC> o[8 / VEC];
        if (C.update) {
#pragma unroll
            for (int i = 0; i < 8 / VEC; ++i) o[i] = load_vec<T, VEC>(out + i * VEC);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            T& to = o[i / VEC].e[i % VEC];
            to = from_f32<T>(C.update ? fmaf(to_f32(to), C.decay, -M.update * v[i]) : v[i]);
        }
#pragma unroll
        for (int i = 0; i < 8 / VEC; ++i) store_vec<T, VEC>(out + i * VEC, o[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) out[i] = from_f32<T>(C.update ? fmaf(to_f32(out[i]), C.decay, -M.update * v[i]) : v[i]);
    }
}

// Exchanges rows and columns of 32 x 32 fp16 numbers, eight of a row to a lane as above, and stores them
__device__ __forceinline__ void put_transposed(uint8_t* to, uint8_t* scratch, int lane, const uint4 (&h)[4]) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {h[i].x, h[i].y, h[i].z, h[i].w};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint16_t*>(scratch + half_at(lane % 4 * 8 + e, i) + lane / 4 * 2) = (uint16_t)(e % 2 ? w[e / 2] >> 16 : w[e / 2]);
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(to + i * 1024) = *reinterpret_cast<const uint4*>(scratch + half_at(i * 8 + lane / 4, lane % 4));
}

// What 32 rows and columns of a product become.  acc: the lane's row; T: the output's type (FINISH).
template <Kind KIND, bool SPLIT, typename T>
__device__ __forceinline__ void take(const Common& C, const Matrix& M, const Job<KIND>& J, int row0, int col0, const uint32_t (&acc)[32],
                                     const Source<KIND, SPLIT>& s, uint8_t* scratch, int lane) {
    constexpr bool SYMMETRIC = KIND == GRAM || KIND == POLYNOMIAL;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i)
        *reinterpret_cast<uint4*>(scratch + word_at(lane, i)) = make_uint4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
    __syncwarp();
    float* diagonal = J.vec + (KIND == POLYNOMIAL ? J.side : 0) + row0;
    const bool on_diagonal = SYMMETRIC && row0 == col0;
    uint8_t* to = J.at(J.to, row0, col0, lane);
    const int64_t second = (int64_t)J.second * BLOCK_BYTES;
    // all of it before the first result is stored: the compiler cannot know that these are other places
    float4 sums[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 2; ++j) sums[i][j] = *reinterpret_cast<const float4*>(scratch + word_at(i * 8 + lane / 4, lane % 4 * 2 + j));
    }
    uint4 hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + lane / 4;
        const float4 a = sums[i][0], b = sums[i][1];
        float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        float x[8];
        if constexpr (KIND != GRAM) {
            const uint32_t h[4] = {s.hi[i].x, s.hi[i].y, s.hi[i].z, s.hi[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) { const float2 f = halves(h[e]); x[2 * e] = f.x; x[2 * e + 1] = f.y; }
            if constexpr (Source<KIND, SPLIT>::BOTH) {
                const uint32_t l[4] = {s.lo[i].x, s.lo[i].y, s.lo[i].z, s.lo[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) { const float2 f = halves(l[e]); x[2 * e] += f.x; x[2 * e + 1] += f.y; }
            }
        }
        if (on_diagonal) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (r != lane % 4 * 8 + e) continue;
                if constexpr (KIND == GRAM) diagonal[r] = v[e] * (1.f / (SCALE * SCALE));
                if constexpr (KIND == POLYNOMIAL) {
                    diagonal[r] = fmaf(C.c, fmaf(s.row[i], s.row[i], v[e] * (1.f / (SCALE * SCALE))), C.b * s.row[i]);
                    x[e] = 0.f;
                }
                v[e] = 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (KIND == GRAM) v[e] *= 1.f / SCALE;
            else if constexpr (KIND == POLYNOMIAL) v[e] = fmaf(C.c, fmaf(x[e], s.row[i] + s.col[e], v[e] * (1.f / SCALE)), C.b * x[e]);
            else v[e] = fmaf(C.a + (s.row[i] + s.col[e]), x[e], v[e] * (1.f / SCALE));
        }
        if constexpr (KIND == FINISH) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= 1.f / SCALE;
            put_output<T>(C, M, row0 + r, col0 + lane % 4 * 8, v);
        } else {
            split2(v[0], v[1], hi[i].x, lo[i].x);
            split2(v[2], v[3], hi[i].y, lo[i].y);
            split2(v[4], v[5], hi[i].z, lo[i].z);
            split2(v[6], v[7], hi[i].w, lo[i].w);
            *reinterpret_cast<uint4*>(to + i * 1024) = hi[i];
            if (SPLIT || !SYMMETRIC) *reinterpret_cast<uint4*>(to + i * 1024 + second) = lo[i];
        }
    }
    if constexpr (SYMMETRIC) {
        if (row0 / BLOCK > col0 / BLOCK) {
            uint8_t* mirror = J.at(J.to, col0, row0, lane);
            put_transposed(mirror, scratch, lane, hi);
            if (SPLIT) put_transposed(mirror + second, scratch, lane, lo);
        }
    }
}

template <Kind KIND, int COLS, bool SPLIT, typename T>
__global__ void __launch_bounds__(THREADS, 1) __cluster_dims__(2, 1, 1)
k_product(const __grid_constant__ Common C, const __grid_constant__ CUtensorMap map, int which, int tiles) {
    constexpr int BYTES = STAGE<COLS, SPLIT>, N = STAGES<COLS, SPLIT>, B_BLOCKS = COLS / 128;
    constexpr bool SYMMETRIC = KIND == GRAM || KIND == POLYNOMIAL;
    extern __shared__ uint8_t raw[];
    uint8_t* ring = raw + ((1024u - (shared_addr(raw) & 1023u)) & 1023u);
    uint8_t* scratches = ring + RING;
    Shared& S = *reinterpret_cast<Shared*>(scratches + RESULT_WARPS * SCRATCH);
    volatile int* gave_up = &S.gave_up;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = pair_rank();
    if (threadIdx.x == 0) {
        // the first CTA's barriers count for both: what has been copied, and which results have been taken
        for (int i = 0; i < N; ++i) { bar_init(&S.full[i], 1); bar_init(&S.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { bar_init(&S.done[i], 1); bar_init(&S.taken[i], 2 * RESULT_WARPS); }
        bar_init_fence();
        S.gave_up = 0;
    }
    if (warp == RESULT_WARPS) tmem_alloc<true>(&S.tmem, 2 * COLS);
    // The descriptors are there before the predecessor is done: every launch lets the next one start only after it has seen its own
    // predecessor's end, so that the one before that is over.
    for (int i = threadIdx.x; i < C.count; i += THREADS) S.first[i] = C.at.matrices[i].first[KIND];
    fence_before();
    __syncthreads();
    pair_sync();
    fence_after();
    const uint32_t tmem = S.tmem;
    auto find = [&](int tile) { return matrix_of(C.count, tile, [&](int i) { return S.first[i]; }); };
    const int tile0 = blockIdx.x / 2, stride = gridDim.x / 2;

    // A result warp holds up to 128 sums to a lane (SPLIT), or two pieces' sources: it gets registers from the group that copies
    // (224 + 224 + 56 = 3 x 168, what the launch has given: LAUNCH_REGISTERS).
    if (warp >= RESULT_WARPS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == RESULT_WARPS && lane == 0) {                    // copies
            int s = 0, issued = 0;
            uint32_t parity = 1;
            bool ok = true;
            for (int tile = tile0; tile < tiles && ok; tile += stride) {
                const int m = find(tile);
                const Matrix& M = C.at.matrices[m];
                const Product P = product_of<KIND>(M, which);
                const Tile at_tile = tile_of<KIND, COLS>(M, tile - S.first[m]);
                const int bm = at_tile.row + (int)rank * 2, bn = at_tile.col + (int)rank * B_BLOCKS;
                int32_t from[4] = {P.A.at(bm), P.A.at(bm + 1), P.B.at(bn), B_BLOCKS == 2 ? P.B.at(bn + 1) : 0};
                const int32_t step[2] = {P.A.step(), P.B.step()}, second[2] = {(int32_t)P.A.second, (int32_t)P.B.second};
                if (tile == tile0) {
                    successor_wait();
                    asm volatile("fence.proxy.async.global;" ::: "memory");
                }
                for (int k = 0; k < P.steps; ++k) {
                    if (!(ok = bar_wait(&S.empty[s], parity, gave_up))) break;
                    if (rank == 0) bar_expect(&S.full[s], 2 * BYTES);
                    uint8_t* to = ring + s * BYTES;
#pragma unroll
                    for (int i = 0; i < 2 + B_BLOCKS; ++i) {
                        block_load(to + i * BLOCK_BYTES, &map, from[i], &S.full[s]);
                        if (SPLIT) block_load(to + (2 + B_BLOCKS + i) * BLOCK_BYTES, &map, from[i] + second[i / 2], &S.full[s]);
                        from[i] += step[i / 2];
                    }
                    ++issued;
                    if (++s == N) { s = 0; parity ^= 1; }
                }
            }
            // Nor may a CTA be gone before the last commits have arrived at its barriers: that of the results (done) says nothing of where the
            // others are.  A stage that was not used passes at once.
            for (int i = 0; i < N && ok; ++i) {
                ok = bar_wait(&S.empty[s], parity, gave_up);
                if (++s == N) { s = 0; parity ^= 1; }
            }
            // no copy may land in a CTA that is gone, nor count there: the first CTA waits for both's, and the second leaves with it
            if (!ok && rank == 0)
                for (int i = 0; i < min(issued, N); ++i) {
                    const int last = issued - 1 - i;
                    const uint64_t t0 = now_ns();
                    while (!bar_try(&S.full[last % N], (uint32_t)(last / N) & 1u) && now_ns() - t0 < WAIT_NS) {}
                }
        } else if (warp == RESULT_WARPS + 1 && lane == 0 && rank == 0) {         // products, of both CTAs
            int s = 0, buffer = 0;
            uint32_t parity = 0, parity_taken = 1;
            bool ok = true;
            for (int tile = tile0; tile < tiles && ok; tile += stride) {
                const Matrix& M = C.at.matrices[find(tile)];
                const Product P = product_of<KIND>(M, which);
                const uint32_t instr = instruction(TILE_ROWS, COLS, P.A.mn_major, P.B.mn_major);
                const uint64_t step_a = operand_step(P.A.mn_major), step_b = operand_step(P.B.mn_major);
                for (int k = 0; k < P.steps && ok; ++k) {
                    const bool begin = SPLIT ? k % CHUNK == 0 : k == 0;
                    if (begin) {
                        if (!(ok = bar_wait(&S.taken[buffer], parity_taken, gave_up))) break;
                        fence_after();
                    }
                    if (!(ok = bar_wait(&S.full[s], parity, gave_up))) break;
                    fence_after();
                    const uint32_t at = shared_addr(ring + s * BYTES), d = tmem + buffer * COLS;
                    const uint64_t a = operand(at, P.A.mn_major), b = operand(at + 2 * BLOCK_BYTES, P.B.mn_major);
                    constexpr uint64_t LOW = (2 + B_BLOCKS) * BLOCK_BYTES / 16;
                    if (SPLIT) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) mma<true>(d, a + i * step_a, b + i * step_b + LOW, instr, !begin || i > 0);
#pragma unroll
                        for (int i = 0; i < 4; ++i) mma<true>(d, a + i * step_a + LOW, b + i * step_b, instr, true);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) mma<true>(d, a + i * step_a, b + i * step_b, instr, SPLIT || !begin || i > 0);
                    commit<true>(&S.empty[s]);
                    if (k + 1 == P.steps || (SPLIT && k % CHUNK == CHUNK - 1)) {
                        commit<true>(&S.done[buffer]);
                        if (buffer) parity_taken ^= 1;
                        buffer ^= 1;
                    }
                    if (++s == N) { s = 0; parity ^= 1; }
                }
            }
            // the second CTA's last arrivals, which the meeting at the end does not wait for
            for (int i = 0; i < 2 && ok; ++i) {
                ok = bar_wait(&S.taken[buffer], parity_taken, gave_up);
                if (buffer) parity_taken ^= 1;
                buffer ^= 1;
            }
        }
    } else {                                                    // results
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        constexpr int MINE = COLS / 2 / 32;                     // pieces of 32 columns of a warp
        int buffer = 0;
        uint32_t parity = 0;
        for (int tile = tile0; tile < tiles; tile += stride) {
            const int m = find(tile);
            const Matrix& M = C.at.matrices[m];
            const Tile at_tile = tile_of<KIND, COLS>(M, tile - S.first[m]);
            const int row0 = at_tile.row * BLOCK + (int)rank * 128 + warp % 4 * 32, col0 = at_tile.col * BLOCK + warp / 4 * (COLS / 2);
            const Job<KIND> J(C, M, which);
            const int R = J.R, K = SYMMETRIC ? M.mb : M.cb;
            // of a symmetric product, what lies above the diagonal comes from below it
            auto wanted = [&](int i) {
                const int col = col0 + i * 32;
                return row0 < R * BLOCK && col < K * BLOCK && (!SYMMETRIC || row0 / BLOCK >= col / BLOCK);
            };
            const uint32_t at = tmem + ((uint32_t)(warp % 4) << 21) + warp / 4 * (COLS / 2);
            auto next = [&] {
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_first(&S.taken[buffer]);
                if (buffer) parity ^= 1;
                buffer ^= 1;
            };
            if (tile == tile0) {
                successor_wait();
                successor_may_start();
            }
            const bool some = wanted(0);                        // the first piece lies farthest to the left
            const int steps = product_of<KIND>(M, which).steps;
            auto done = [&] {
                const bool ok = bar_wait_warp(&S.done[buffer], parity, gave_up);
                fence_after();
                return ok;
            };
            const bool summed = SPLIT && steps > CHUNK;
            if (summed) {
                // the chunks' sums, in the end back in tensor memory in the place of the last
                float sum[2 * MINE][16] = {};
                bool ok = true;
                for (int k = 0; k < steps; k += CHUNK) {
                    if (!(ok = done())) break;
                    if (some) {
#pragma unroll
                        for (int i = 0; i < 2 * MINE; ++i) {
                            float acc[16];
                            tmem_load16(at + buffer * COLS + i * 16, acc);
                            tmem_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) sum[i][j] += acc[j];
                        }
                    }
                    if (k + CHUNK < steps) next();
                }
                if (!ok) break;
                if (some) {
#pragma unroll
                    for (int i = 0; i < 2 * MINE; ++i) tmem_store16(at + buffer * COLS + i * 16, sum[i]);
                    tmem_store_wait();
                }
            }
            Source<KIND, SPLIT> source{};
            if (some) fetch(J, row0, col0, opaque(lane), source);
            if (!summed && !done()) break;
            // What a piece needs is fetched before the one before it is worked on.  One copy of the code: a launch of few tiles waits for
            // every line of it.
#pragma unroll 1
            for (int i = 0; i < MINE; ++i) {
                // addresses are made here each time: kept across the tiles they would take the registers of the sums
                const int l = opaque(lane);
                uint32_t acc[32];
                tmem_load32(at + buffer * COLS + i * 32, acc);
                Source<KIND, SPLIT> following{};
                if (i + 1 < MINE && wanted(i + 1)) fetch(J, row0, col0 + (i + 1) * 32, l, following);
                tmem_wait();
                if (i + 1 == MINE) next();
                if (wanted(i)) take<KIND, SPLIT, T>(C, M, J, row0, col0 + i * 32, acc, source, scratches + opaque(warp) * SCRATCH, l);
                source = following;
            }
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && S.gave_up) atomicExch(&g_error, 1);
    pair_meet();                                    // neither leaves while the other's products read its shared memory
    fence_after();
    if (warp == RESULT_WARPS) tmem_free<true>(tmem, 2 * COLS);
}

// ---- small matrices ----------------------------------------------------------------------------------
//
// Where x and A fit the shared memory of one CTA (the shorter side up to 128, the longer up to 256), one CTA does all of it for one matrix:
// momentum, division, every step.  The launches above would each wait for the one before, 6 us for a microsecond's work (four matrices of
// 64 x 128: 98 us; this way 37).  x, A and B are blocks in shared memory as elsewhere; results replace what they are made from,
// number by number: both halves of the symmetric products are computed, so that each thread needs its own numbers alone.

constexpr int SMALL_SHORT = 2, SMALL_LONG = 4;      // blocks of the sides
constexpr int SMALL_THREADS = 256;
struct SmallShared {
    uint64_t done;
    uint32_t tmem;
    int gave_up;
    double sums[PREPARE_THREADS / 32];
    alignas(16) float d[SMALL_SHORT * BLOCK];
    alignas(16) float e[SMALL_SHORT * BLOCK];
};
static_assert(SMALL_THREADS == PREPARE_THREADS, "blocks are loaded as by the preparation");

struct SmallPlan {
    int32_t x_blocks, a_blocks;                     // of the largest matrix
    int32_t columns;                                // of tensor memory
};

template <typename TIN, typename T, bool SPLIT>
__global__ void __launch_bounds__(SMALL_THREADS) k_small(const __grid_constant__ Group G, const __grid_constant__ Common C, const SmallPlan plan, int steps) {
    extern __shared__ uint8_t raw[];
    uint8_t* const x_hi = raw + ((1024u - (shared_addr(raw) & 1023u)) & 1023u);
    uint8_t* const x_lo = x_hi + plan.x_blocks * BLOCK_BYTES;
    uint8_t* const a_hi = x_lo + plan.x_blocks * BLOCK_BYTES;
    uint8_t* const a_lo = a_hi + plan.a_blocks * BLOCK_BYTES;
    __shared__ SmallShared S;
    volatile int* gave_up = &S.gave_up;
    const Matrix& M = G.m[blockIdx.x];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int R = M.rb, K = M.cb, side = M.mb;
    const bool tall = M.tall();
    if (t == 0) {
        bar_init(&S.done, 1);
        bar_init_fence();
        S.gave_up = 0;
    }
    // The next launch may come when every CTA has its tensor memory: beside two of another plan (256 columns each) one of this would have to wait
    // for memory that they keep until this launch is over.
    if (warp == 0) tmem_alloc<false>(&S.tmem, plan.columns);
    successor_wait();
    if (warp == 0) successor_may_start();

    // momentum and the sum of squares, then x
    const bool vector = may_load_four<TIN>(M);
    const float scale = C.grad_scale ? *C.grad_scale : 1.f;
    double sum = 0.0;
    for (int block = 0; block < R * K; ++block) {
        const int r0 = block % R * BLOCK, c0 = block / R * BLOCK;
        Share<TIN> s;
        load_block<TIN>(M, r0, c0, vector, s);
        const int c = c0 + t % 16 * 4;
#pragma unroll
        for (int i = 0; i < SHARE; ++i) {
            const int r = r0 + t / 16 + 16 * i, n = r < M.rows ? M.cols - c : 0;
            const float4 u = momentum_of(C, M, s, i, scale);
            if (M.m) put_momentum(M, s, i, r, c, n, vector);
            sum += squares(u, n);
        }
    }
    sum = block_sum(sum, S.sums);
    const Inverse inv(sum, C.eps);
    for (int block = 0; block < R * K; ++block) {
        const int r0 = block % R * BLOCK, c0 = block / R * BLOCK;
        Share<TIN> s;
        load_block<TIN>(M, r0, c0, vector, s);      // the momentum as this thread has just stored it
#pragma unroll
        for (int i = 0; i < SHARE; ++i) {
            const int rr = t / 16 + 16 * i, cc = t % 16 * 4, n = r0 + rr < M.rows ? M.cols - c0 - cc : 0;
            const float4 u = stored_momentum_of(C, M, s, i, scale);
            uint2 hi, lo;
            split2(n > 0 ? inv.of(u.x) : 0.f, n > 1 ? inv.of(u.y) : 0.f, hi.x, lo.x);
            split2(n > 2 ? inv.of(u.z) : 0.f, n > 3 ? inv.of(u.w) : 0.f, hi.y, lo.y);
            const uint32_t at = block * BLOCK_BYTES + piece_at(rr, cc / 8) + cc % 8 * 2;
            *reinterpret_cast<uint2*>(x_hi + at) = hi;
            *reinterpret_cast<uint2*>(x_lo + at) = lo;
        }
    }

    uint32_t parity = 0;
    bool ok = true;
    // One product: operands as stacks of blocks whose first numbers begin at a and b, to the accumulators at `column`
    struct Side { const uint8_t *hi, *lo; int first, step, leading; bool mn_major; };
    auto issue = [&](const Side& A, const Side& B, int n, int count, uint32_t column) {
        const uint32_t instr = instruction(128, n, A.mn_major, B.mn_major);
        const uint64_t step_a = operand_step(A.mn_major), step_b = operand_step(B.mn_major);
        const uint32_t d = S.tmem + column;
        for (int k = 0; k < count; ++k) {
            auto of = [&](const Side& s, bool low) {
                return operand(shared_addr((low ? s.lo : s.hi) + (s.first + k * s.step) * BLOCK_BYTES), s.mn_major, s.leading);
            };
            const uint64_t a = of(A, false), b = of(B, false);
            if (SPLIT) {
                const uint64_t al = of(A, true), bl = of(B, true);
                for (int i = 0; i < 4; ++i) mma<false>(d, a + i * step_a, bl + i * step_b, instr, k > 0 || i > 0);
                for (int i = 0; i < 4; ++i) mma<false>(d, al + i * step_a, b + i * step_b, instr, true);
            }
            for (int i = 0; i < 4; ++i) mma<false>(d, a + i * step_a, b + i * step_b, instr, SPLIT || k > 0 || i > 0);
        }
    };
    // What was written by threads is read by the products; then their results are there for all
    auto products = [&](auto f) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        fence_before();
        __syncthreads();
        if (t == 0) {
            fence_after();
            f();
            commit<false>(&S.done);
        }
        ok = __syncthreads_and(bar_wait(&S.done, parity, gave_up));            // all go on, or none
        parity ^= 1;
        fence_after();
    };
    // f(row, col, acc) for the warp's pieces of `rows` x `cols` results (32 columns of the lane's row), tiles of 128 rows side by side
    auto results = [&](int rows, int cols, auto f) {
        const int pieces = cols / 32;
        for (int tile = 0; tile * 128 < rows; ++tile) {
            const int row = tile * 128 + warp % 4 * 32;
            if (row >= rows) continue;
            for (int i = warp / 4; i < pieces; i += 2) {
                uint32_t acc[32];
                tmem_load32(S.tmem + ((uint32_t)(warp % 4) << 21) + tile * cols + i * 32, acc);
                tmem_wait();
                f(row + lane, i * 32, acc);
            }
        }
    };
    auto at = [&](int row, int col, int blocks, int piece) {   // of a matrix of `blocks` blocks to a column
        return (uint32_t)((col / BLOCK * blocks + row / BLOCK) * BLOCK_BYTES) + piece_at(row % BLOCK, col % BLOCK / 8 + piece);
    };
    // All loads before the first store: the compiler cannot know that they are of other places, and one warp alone waits for each
    auto load32 = [&](const uint8_t* hi, const uint8_t* lo, int row, int col, int blocks, bool both, float (&x)[32]) {
        uint4 h[4], l[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            h[p] = *reinterpret_cast<const uint4*>(hi + at(row, col, blocks, p));
            if (both) l[p] = *reinterpret_cast<const uint4*>(lo + at(row, col, blocks, p));
        }
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t w[4] = {h[p].x, h[p].y, h[p].z, h[p].w}, u[4] = {l[p].x, l[p].y, l[p].z, l[p].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float2 f = halves(w[e]);
                if (both) f = add2(f, halves(u[e]));
                x[p * 8 + 2 * e] = f.x;
                x[p * 8 + 2 * e + 1] = f.y;
            }
        }
    };
    auto store32 = [&](uint8_t* hi, uint8_t* lo, int row, int col, int blocks, bool both, const float (&v)[32]) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            uint4 h, l;
            split2(v[p * 8], v[p * 8 + 1], h.x, l.x);
            split2(v[p * 8 + 2], v[p * 8 + 3], h.y, l.y);
            split2(v[p * 8 + 4], v[p * 8 + 5], h.z, l.z);
            split2(v[p * 8 + 6], v[p * 8 + 7], h.w, l.w);
            *reinterpret_cast<uint4*>(hi + at(row, col, blocks, p)) = h;
            if (both) *reinterpret_cast<uint4*>(lo + at(row, col, blocks, p)) = l;
        }
    };
    auto load_vector = [&](const float* from, float (&v)[32]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 f = *reinterpret_cast<const float4*>(from + 4 * i);
            v[4 * i] = f.x; v[4 * i + 1] = f.y; v[4 * i + 2] = f.z; v[4 * i + 3] = f.w;
        }
    };

    const Side x_rows{x_hi, x_lo, 0, R, 1, false}, x_down{x_hi, x_lo, 0, 1, R, true}, q{a_hi, a_lo, 0, side, 1, false};
    for (int step = 0; step < steps && ok; ++step) {
        products([&] {
            if (tall) issue(x_down, x_down, side * BLOCK, R, 0);
            else issue(x_rows, x_rows, side * BLOCK, K, 0);
        });
        if (!ok) break;
        results(side * BLOCK, side * BLOCK, [&](int row, int col, const uint32_t (&acc)[32]) {
            float v[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                v[e] = __uint_as_float(acc[e]) * (1.f / SCALE);
                if (row == col + e) {
                    S.d[row] = v[e] * (1.f / SCALE);
                    v[e] = 0.f;
                }
            }
            store32(a_hi, a_lo, row, col, side, SPLIT, v);
        });
        products([&] { issue(q, q, side * BLOCK, side, 0); });
        if (!ok) break;
        results(side * BLOCK, side * BLOCK, [&](int row, int col, const uint32_t (&acc)[32]) {
            const float mine = S.d[row];
            float v[32];
            load32(a_hi, a_lo, row, col, side, SPLIT, v);
            float other[32];
            load_vector(S.d + col, other);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                const float a = __uint_as_float(acc[e]) * (1.f / SCALE);
                const bool diag = row == col + e;
                if (diag) S.e[row] = fmaf(C.c, fmaf(mine, mine, a * (1.f / SCALE)), C.b * mine);
                v[e] = diag ? 0.f : fmaf(C.c, fmaf(v[e], mine + other[e], a), C.b * v[e]);
            }
            store32(a_hi, a_lo, row, col, side, SPLIT, v);
        });
        products([&] {
            if (tall)
                for (int tile = 0; tile * 2 < R; ++tile) issue(Side{x_hi, x_lo, 2 * tile, R, 1, false}, q, side * BLOCK, side, tile * side * BLOCK);
            else issue(q, x_down, K * BLOCK, side, 0);
        });
        if (!ok) break;
        results(R * BLOCK, K * BLOCK, [&](int row, int col, const uint32_t (&acc)[32]) {
            float v[32], f[32];
            load32(x_hi, x_lo, row, col, R, true, v);
            if (tall) load_vector(S.e + col, f);
            else {
                const float mine = S.e[row];
#pragma unroll
                for (int e = 0; e < 32; ++e) f[e] = mine;
            }
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = fmaf(C.a + f[e], v[e], __uint_as_float(acc[e]) * (1.f / SCALE));
            if (step + 1 < steps) {
                store32(x_hi, x_lo, row, col, R, true, v);
            } else {
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    float o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = v[p * 8 + e] * (1.f / SCALE);
                    put_output<T>(C, M, row, col + p * 8, o);
                }
            }
        });
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (t == 0 && S.gave_up) atomicExch(&g_error, 1);
    if (warp == 0) tmem_free<false>(S.tmem, plan.columns);
}

// ---- a wait that runs out ----------------------------------------------------------------------------

// One warp waits at a barrier, half of its lanes for `limit`, the others until a thread of another warp arrives, which it does once the
// first have given up.  told[lane]: what the lane's wait returned.  Every wait is bounded.
__global__ void __launch_bounds__(64) k_run_out(uint64_t limit, int32_t* told) {
    __shared__ uint64_t late;
    __shared__ int gave_up, patient;
    volatile int* seen = &gave_up;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        bar_init(&late, 1);
        bar_init_fence();
        gave_up = patient = 0;
    }
    __syncthreads();
    if (warp == 0) {
        told[lane] = bar_wait_warp(&late, 0, lane < 16 ? &gave_up : &patient, lane < 16 ? limit : WAIT_NS);
    } else if (lane == 0) {
        const uint64_t t0 = now_ns();
        while (!*seen && now_ns() - t0 < WAIT_NS) {}
        bar_arrive(&late);
    }
    __syncthreads();
    if (threadIdx.x == 0 && gave_up) atomicExch(&g_error, 1);
}

// ---- host side ---------------------------------------------------------------------------------------

// Whether one CTA has room for a matrix
bool is_small(const ssgd_matrix& t) {
    const int64_t rb = (t.rows + BLOCK - 1) / BLOCK, cb = (t.cols + BLOCK - 1) / BLOCK;
    return (rb < cb ? rb : cb) <= SMALL_SHORT && (rb < cb ? cb : rb) <= SMALL_LONG;
}

struct Sizes {
    int64_t blocks = 0, floats = 0, strips = 0, elements = 0;
    int count = 0;
    int64_t sums_at() const { return (int64_t)sizeof(Matrix) * MAX_GROUP; }
    int64_t vec_at() const { return (sums_at() + strips * 8 + 127) / 128 * 128; }
    int64_t blocks_at() const { return (vec_at() + floats * 4 + 1023) / 1024 * 1024; }
    int64_t bytes() const { return blocks_at() + blocks * BLOCK_BYTES; }
};

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Adds a matrix to a group; false if there is no room
bool add(Sizes& s, const ssgd_matrix& t, bool split, Matrix* to) {
    // with the padding, which the workspace holds too: it is most of a matrix of few rows
    const int64_t elements = div_up(t.rows, BLOCK) * div_up(t.cols, BLOCK) * BLOCK * BLOCK;
    if (s.count == MAX_GROUP || (s.count && s.elements + elements > GROUP_ELEMENTS)) return false;
    Matrix M{};
    M.rows = (int32_t)t.rows; M.cols = (int32_t)t.cols;
    M.rb = (int32_t)div_up(t.rows, BLOCK); M.cb = (int32_t)div_up(t.cols, BLOCK);
    M.mb = M.rb < M.cb ? M.rb : M.cb;
    const int64_t xs = (int64_t)M.rb * M.cb, ms = (int64_t)M.mb * M.mb;
    M.x0 = (uint32_t)s.blocks; M.x1 = (uint32_t)(s.blocks + 2 * xs);
    M.a = (uint32_t)(s.blocks + 4 * xs); M.b = (uint32_t)(s.blocks + 4 * xs + (split ? 2 : 1) * ms);
    s.blocks += 4 * xs + (split ? 4 : 2) * ms;
    M.vec = (uint32_t)s.floats;
    s.floats += 2 * (int64_t)M.mb * BLOCK;
    M.strips = (int32_t)(M.rb * div_up(M.cb, STRIP_BLOCKS));
    s.strips += M.strips;
    s.elements += elements;
    s.count++;
    if (to) {
        M.out = t.out; M.in = t.in; M.m = t.m;
        M.ld_out = t.ld_out; M.ld_in = t.ld_in;
        *to = M;
    }
    return true;
}

template <typename... P, typename... A>
int launch(cudaStream_t st, void (*kernel)(P...), int grid, int block, int smem, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess ? SSGD_OK : SSGD_ECUDA;
}

template <typename T>
int launch_prepare(cudaStream_t st, int strips, const Group& G, const Common& C) {
    if (int e = launch(st, k_momentum<T>, strips, PREPARE_THREADS, 0, G, C)) return e;
    return launch(st, k_layout<T>, strips, PREPARE_THREADS, 0, C);
}

template <Kind KIND, int COLS, bool SPLIT, typename T>
int launch_tiles(cudaStream_t st, const Common& C, const CUtensorMap& map, int which, int64_t tiles, int sms) {
    static PerDevice known;
    int fits = 0;
    // The exchange of registers in the kernel would wait forever if it had been launched with others.  The build looks at what the assembler
    // reports; this is for libraries that were built otherwise.
    static const bool as_planned = [] {
        cudaFuncAttributes a{};
        return cudaFuncGetAttributes(&a, k_product<KIND, COLS, SPLIT, T>) == cudaSuccess && a.numRegs == LAUNCH_REGISTERS;
    }();
    if (!as_planned) return SSGD_ECUDA;
    if (int e = residency(k_product<KIND, COLS, SPLIT, T>, THREADS, SHARED_BYTES, known, &fits)) return e;
    return launch(st, k_product<KIND, COLS, SPLIT, T>, (int)(2 * (tiles < sms / 2 ? tiles : sms / 2)), THREADS, SHARED_BYTES, C, map, which, (int)tiles);
}
template <Kind KIND, typename T = void>
int launch_product(cudaStream_t st, const Common& C, const CUtensorMap& map, bool wide, int which, int64_t tiles, int sms) {
    if (C.split)
        return wide ? launch_tiles<KIND, 256, true, T>(st, C, map, which, tiles, sms) : launch_tiles<KIND, 128, true, T>(st, C, map, which, tiles, sms);
    return wide ? launch_tiles<KIND, 256, false, T>(st, C, map, which, tiles, sms) : launch_tiles<KIND, 128, false, T>(st, C, map, which, tiles, sms);
}

// Work of a launch with tiles of 128 and of 256 columns, in blocks of the contraction
struct Work {
    int64_t blocks[2] = {0, 0}, longest = 0;
    void add(int64_t narrow, int64_t wide, int64_t steps) {
        blocks[0] += narrow * steps;
        blocks[1] += wide * steps;
        longest = steps > longest ? steps : longest;
    }
    // What bounds either is what a tile loads, 3 against 4 blocks to a CTA.  A launch ends when the last tile does: about one tile later
    // than if all pairs ended together.
    bool prefers_wide(int sms) const {
        const int64_t pairs = sms / 2;
        return 4 * (blocks[1] + longest * pairs) <= 3 * (blocks[0] + longest * pairs);
    }
};

template <typename TIN, typename T, bool SPLIT>
int launch_small(cudaStream_t st, const Group& G, const Common& C, const SmallPlan& plan, int steps) {
    const int smem = 1024 + 2 * (plan.x_blocks + plan.a_blocks) * BLOCK_BYTES;
    static PerDevice opted;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return SSGD_ECUDA;
    if (!opted.value[dev]) {
        constexpr int MOST = 1024 + 2 * (SMALL_SHORT * SMALL_LONG + SMALL_SHORT * SMALL_SHORT) * BLOCK_BYTES;
        if (cudaFuncSetAttribute(k_small<TIN, T, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST) != cudaSuccess) return SSGD_ECUDA;
        opted.value[dev] = 1;
    }
    return launch(st, k_small<TIN, T, SPLIT>, C.count, SMALL_THREADS, smem, G, C, plan, steps);
}
template <typename TIN, typename T>
int launch_small(cudaStream_t st, const Group& G, const Common& C, const SmallPlan& plan, int steps) {
    return C.split ? launch_small<TIN, T, true>(st, G, C, plan, steps) : launch_small<TIN, T, false>(st, G, C, plan, steps);
}
template <typename T>
int launch_small(cudaStream_t st, const Group& G, const Common& C, const SmallPlan& plan, int steps) {
    if (C.fmt_in == SSGD_FMT_F32) return launch_small<float, T>(st, G, C, plan, steps);
    return C.fmt_in == SSGD_FMT_F16 ? launch_small<__half, T>(st, G, C, plan, steps) : launch_small<__nv_bfloat16, T>(st, G, C, plan, steps);
}

constexpr int64_t MAX_SIDE = (int64_t)1 << 20;
constexpr int MAX_STEPS = 32;

// The polynomial f(s) = a s + b s^3 + c s^5 has to keep what starts within [0, 1] well inside the range of the stored numbers: no more than 4 on
// the way and 8 at the end, and b s^2 + c s^4 within 48.  f is continuous and f(0) = 0, so that it makes of an interval around 0 exactly the
// interval between its extremes there: at the ends, or where a + 3 b t + 5 c t^2 = 0 with t = s^2.
bool stays_in_range(int steps, double a, double b, double c) {
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    auto f = [&](double s) { return s * (a + s * s * (b + c * s * s)); };
    double flat[2] = {-1.0, -1.0};                  // t of these places
    const double d = 9.0 * b * b - 20.0 * a * c;
    if (d >= 0.0) {
        const double h = -0.5 * (3.0 * b + std::copysign(std::sqrt(d), b));     // no cancellation
        if (c != 0.0) flat[0] = h / (5.0 * c);
        if (h != 0.0) flat[1] = a / h;
    }
    double lo = 0.0, hi = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double top = std::max(-lo, hi), q = top * top;
        if (!(top <= 4.0)) return false;
        const double end = b * q + c * q * q, middle = c != 0.0 && -b / (2.0 * c) > 0.0 && -b / (2.0 * c) < q ? -b * b / (4.0 * c) : 0.0;
        if (!(std::fabs(end) < 48.0) || !(std::fabs(middle) < 48.0)) return false;
        double places[6] = {lo, hi, 0.0, 0.0, 0.0, 0.0};
        for (int i = 0; i < 2; ++i) {
            const double s = flat[i] > 0.0 ? std::sqrt(flat[i]) : 0.0;
            if (s <= hi) places[2 + i] = s;
            if (-s >= lo) places[4 + i] = -s;
        }
        lo = hi = 0.0;
        for (double s : places) {
            lo = std::min(lo, f(s));
            hi = std::max(hi, f(s));
        }
    }
    return lo > -8.0 && hi < 8.0;
}

// One product or three (0: by the type of the result)
int products_of(int32_t products, int32_t fmt_out) { return products ? products : fmt_out == SSGD_FMT_BF16 ? 1 : 3; }

int check_sizes(const ssgd_matrix* t, int32_t count, int32_t fmt_out, int32_t products) {
    if (count < 0 || (count && !t) || !fmt_bytes(fmt_out) || (products != 0 && products != 1 && products != 3)) return SSGD_EINVAL;
    for (int32_t i = 0; i < count; ++i) {
        if (t[i].rows < 0 || t[i].cols < 0 || t[i].rows > MAX_SIDE || t[i].cols > MAX_SIDE) return SSGD_EINVAL;
        const int64_t lo = t[i].rows < t[i].cols ? t[i].rows : t[i].cols;
        if (t[i].rows * t[i].cols > (int64_t)1 << 32 || lo > 32768) return SSGD_ETOOBIG;
    }
    return SSGD_OK;
}

int check_matrices(const ssgd_matrix* t, int32_t count, int32_t fmt_in, int32_t fmt_out, int32_t products, bool with_m, int32_t steps,
                   double a, double b, double c, double eps) {
    if (!fmt_bytes(fmt_in)) return SSGD_EINVAL;
    if (int e = check_sizes(t, count, fmt_out, products)) return e;
    if (steps < 1 || steps > MAX_STEPS || !(eps >= 0.0) || !(eps < INFINITY) || !stays_in_range(steps, a, b, c)) return SSGD_EINVAL;
    for (int32_t i = 0; i < count; ++i) {
        if (!t[i].rows || !t[i].cols) continue;
        if (t[i].ld_in < t[i].cols || t[i].ld_out < t[i].cols || !t[i].in || !t[i].out || (with_m && !t[i].m)) return SSGD_EINVAL;
        if (!aligned_to(t[i].in, fmt_bytes(fmt_in)) || !aligned_to(t[i].out, fmt_bytes(fmt_out)) || (with_m && !aligned_to(t[i].m, 4)))
            return SSGD_EALIGN;
    }
    return SSGD_OK;
}

int64_t workspace_of(const ssgd_matrix* t, int32_t count, bool split) {
    int64_t most = 0;
    Sizes s;
    for (int32_t i = 0; i < count; ++i) {
        if (!t[i].rows || !t[i].cols || is_small(t[i])) continue;
        if (!add(s, t[i], split, nullptr)) {
            s = Sizes{};
            add(s, t[i], split, nullptr);
        }
        most = s.bytes() > most ? s.bytes() : most;
    }
    return most;
}

int run(const ssgd_matrix* t, int32_t count, Common C, int32_t steps, double lr, void* workspace, size_t bytes, cudaStream_t st) {
    const int64_t need = workspace_of(t, count, C.split);
    if (std::all_of(t, t + count, [](const ssgd_matrix& m) { return !m.rows || !m.cols; })) return SSGD_OK;
    if (need) {
        if (!workspace || (int64_t)bytes < need) return SSGD_EWORKSPACE;
        if (!aligned_to(workspace, 16)) return SSGD_EALIGN;
    }
    int sms = 0, e = sm_count_of_current_device(&sms);
    if (e) return e;
    // the small ones
    for (int32_t i = 0; i < count;) {
        Group G;
        Sizes s;
        SmallPlan plan{0, 0, 32};
        for (; i < count && s.count < MAX_GROUP; ++i) {
            if (!t[i].rows || !t[i].cols || !is_small(t[i])) continue;
            Matrix& M = G.m[s.count];
            add(s, t[i], C.split, &M);
            M.update = (float)(lr * t[i].scale);
            if (!C.update) M.m = nullptr;           // whatever the caller left there
            const int32_t tiles = M.tall() ? (M.rb + 1) / 2 : 1, columns = BLOCK * (M.tall() ? tiles * M.cb : M.cb);
            plan.x_blocks = std::max(plan.x_blocks, M.rb * M.cb);
            // rows beyond a matrix of one block are read, and their results left
            plan.a_blocks = std::max(plan.a_blocks, std::max(2, M.mb * M.mb));
            while (plan.columns < columns) plan.columns *= 2;
        }
        if (!s.count) break;
        C.count = s.count;
        e = C.fmt_out == SSGD_FMT_F32 ? launch_small<float>(st, G, C, plan, steps)
          : C.fmt_out == SSGD_FMT_F16 ? launch_small<__half, __half>(st, G, C, plan, steps)                // never of another type
                                      : launch_small<__nv_bfloat16>(st, G, C, plan, steps);
        if (e) return e;
    }
    int32_t i = 0;
    while (i < count) {
        Group G;
        Sizes s;
        for (; i < count; ++i) {
            if (!t[i].rows || !t[i].cols || is_small(t[i])) continue;
            if (!add(s, t[i], C.split, s.count < MAX_GROUP ? &G.m[s.count] : nullptr)) break;
            G.m[s.count - 1].update = (float)(lr * t[i].scale);
            if (!C.update) G.m[s.count - 1].m = nullptr;
        }
        if (!s.count) break;
        uint8_t* base = static_cast<uint8_t*>(workspace);
        C.at = Space{reinterpret_cast<Matrix*>(base), reinterpret_cast<double*>(base + s.sums_at()),
                     reinterpret_cast<float*>(base + s.vec_at()), base + s.blocks_at()};
        C.count = s.count;
        CUtensorMap map;
        if (!blocks_map(&map, C.at.blocks, s.blocks)) return SSGD_ECUDA;
        // long tiles first: what is left for the end is short
        std::stable_sort(G.m, G.m + s.count, [](const Matrix& a, const Matrix& b) { return (a.rb > a.cb ? a.rb : a.cb) > (b.rb > b.cb ? b.rb : b.cb); });
        Work gram, polynomial, apply;
        for (int k = 0; k < s.count; ++k) {
            const Matrix& M = G.m[k];
            gram.add(symmetric_tiles<128>(M.mb), symmetric_tiles<256>(M.mb), M.rb > M.cb ? M.rb : M.cb);
            polynomial.add(symmetric_tiles<128>(M.mb), symmetric_tiles<256>(M.mb), M.mb);
            apply.add(all_tiles<128>(M.rb, M.cb), all_tiles<256>(M.rb, M.cb), M.mb);
        }
        const bool wide_gram = gram.prefers_wide(sms), wide_polynomial = polynomial.prefers_wide(sms), wide_apply = apply.prefers_wide(sms);
        int32_t strips = 0, first_gram = 0, first_polynomial = 0, first_apply = 0;
        for (int k = 0; k < s.count; ++k) {
            Matrix& M = G.m[k];
            M.strip0 = strips;
            M.first[GRAM] = first_gram;
            M.first[POLYNOMIAL] = first_polynomial;
            M.first[APPLY] = M.first[FINISH] = first_apply;
            strips += M.strips;
            first_gram += (int32_t)(wide_gram ? symmetric_tiles<256>(M.mb) : symmetric_tiles<128>(M.mb));
            first_polynomial += (int32_t)(wide_polynomial ? symmetric_tiles<256>(M.mb) : symmetric_tiles<128>(M.mb));
            first_apply += (int32_t)(wide_apply ? all_tiles<256>(M.rb, M.cb) : all_tiles<128>(M.rb, M.cb));
        }
        if ((e = C.fmt_in == SSGD_FMT_F32 ? launch_prepare<float>(st, (int)s.strips, G, C)
               : C.fmt_in == SSGD_FMT_F16 ? launch_prepare<__half>(st, (int)s.strips, G, C) : launch_prepare<__nv_bfloat16>(st, (int)s.strips, G, C)))
            return e;
        for (int k = 0; k < steps; ++k) {
            if ((e = launch_product<GRAM>(st, C, map, wide_gram, k & 1, first_gram, sms))) return e;
            if ((e = launch_product<POLYNOMIAL>(st, C, map, wide_polynomial, k & 1, first_polynomial, sms))) return e;
            if (k + 1 < steps) e = launch_product<APPLY>(st, C, map, wide_apply, k & 1, first_apply, sms);
            else if (C.fmt_out == SSGD_FMT_F32) e = launch_product<FINISH, float>(st, C, map, wide_apply, k & 1, first_apply, sms);
            else if (C.fmt_out == SSGD_FMT_F16) e = launch_product<FINISH, __half>(st, C, map, wide_apply, k & 1, first_apply, sms);
            else e = launch_product<FINISH, __nv_bfloat16>(st, C, map, wide_apply, k & 1, first_apply, sms);
            if (e) return e;
        }
    }
    return SSGD_OK;
}

}  // namespace

extern "C" {

int ssgd_orthogonalize_workspace(const ssgd_matrix* matrices, int32_t count, int32_t fmt_out, int32_t products, size_t* out_bytes) {
    if (!out_bytes) return SSGD_EINVAL;
    if (int e = check_sizes(matrices, count, fmt_out, products)) return e;
    *out_bytes = (size_t)workspace_of(matrices, count, products_of(products, fmt_out) == 3);
    return SSGD_OK;
}

int ssgd_orthogonalize(const ssgd_matrix* matrices, int32_t count, int32_t fmt, int32_t products, int32_t steps, double a, double b,
                       double c, double eps, void* workspace, size_t workspace_bytes, void* stream) {
    if (int e = check_matrices(matrices, count, fmt, fmt, products, false, steps, a, b, c, eps)) return e;
    Common C{};
    C.fmt_in = C.fmt_out = fmt;
    C.split = products_of(products, fmt) == 3;
    C.eps = (float)eps;
    C.a = (float)a; C.b = (float)b; C.c = (float)c;
    return run(matrices, count, C, steps, 0.0, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

int ssgd_muon_step(const ssgd_matrix* matrices, int32_t count, int32_t fmt_p, int32_t fmt_g, int32_t products, double lr, double momentum,
                   int32_t nesterov, double weight_decay, int32_t steps, double a, double b, double c, double eps, const float* grad_scale,
                   void* workspace, size_t workspace_bytes, void* stream) {
    if (fmt_p != SSGD_FMT_F32 && fmt_p != SSGD_FMT_BF16) return SSGD_EINVAL;
    if (!(lr >= 0.0) || !(lr < INFINITY) || !(momentum >= 0.0) || !(momentum < 1.0) || !(weight_decay >= 0.0) || !(weight_decay < INFINITY))
        return SSGD_EINVAL;
    if (int e = check_matrices(matrices, count, fmt_g, fmt_p, products, true, steps, a, b, c, eps)) return e;
    if (!aligned_to(grad_scale, 4)) return SSGD_EALIGN;
    Common C{};
    C.fmt_in = fmt_g; C.fmt_out = fmt_p;
    C.split = products_of(products, fmt_p) == 3;
    C.nesterov = nesterov != 0;
    C.update = true;
    C.momentum = (float)momentum;
    C.share = (float)(1.0 - momentum);
    C.decay = (float)(1.0 - lr * weight_decay);
    C.eps = (float)eps;
    C.a = (float)a; C.b = (float)b; C.c = (float)c;
    C.grad_scale = grad_scale;
    return run(matrices, count, C, steps, lr, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

int ssgd_test_run_out(int64_t limit_ns, int32_t* told, void* stream) {
    if (limit_ns < 1000 || limit_ns > 1000000000 || !told) return SSGD_EINVAL;
    if (!aligned_to(told, 4)) return SSGD_EALIGN;
    k_run_out<<<1, 64, 0, static_cast<cudaStream_t>(stream)>>>((uint64_t)limit_ns, told);
    return launched();
}

int ssgd_train_ops_status(void* stream) {
    if (cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) != cudaSuccess) return SSGD_ECUDA;
    int seen = 0, none = 0;
    if (cudaMemcpyFromSymbol(&seen, g_error, sizeof seen) != cudaSuccess) return SSGD_ECUDA;
    if (!seen) return SSGD_OK;
    return cudaMemcpyToSymbol(g_error, &none, sizeof none) == cudaSuccess ? SSGD_EDEVICE : SSGD_ECUDA;
}

}  // extern "C"
