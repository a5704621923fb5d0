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
// leaving 5e-4 to 1.4e-3 of the result (less than its rounding to bfloat16, 1.7e-3).  Where the result has more bits than bfloat16,
// or the caller says so, every matrix is a sum of two fp16 numbers and a product takes three (high high, high low, low high): 3e-7
// to 4e-6, less than the same iteration in fp32.
// The stored numbers are 1024 times the true ones: x is at most 1.2 and an element mostly far below, so that the second number stays
// clear of fp16's subnormals.
//
// Layout.  All matrices of a call go through every launch together: prepare (momentum and sums of squares; division and layout),
// then 3 launches per step, whose tiles are dealt out over the SMs.  Matrices live in the workspace as blocks (umma.cuh), padded with
// zeros to 64; block (r, c) of a matrix of R x C blocks is the (c R + r)-th.
#include "formats.cuh"
#include "umma.cuh"

using namespace ssgd;
using namespace ssgd::umma;

namespace {

constexpr float SCALE = 1024.f;
constexpr int MAX_GROUP = 224;                      // matrices of one set of launches: their descriptors are arguments of the first
constexpr int64_t GROUP_ELEMENTS = (int64_t)1 << 27;  // and no more than this many elements, unless one matrix has them
constexpr int STRIP_BLOCKS = 8;                     // what a CTA of the preparation takes: 64 rows of 512 columns

struct Matrix {
    void* out; const void* in; float* m;
    int64_t ld_out, ld_in;
    int32_t rows, cols, rb, cb, mb;                 // size; size in blocks; blocks of the shorter side
    uint32_t x[2], a, b;                            // first blocks: x before and after a step, A, B.  Second numbers lie behind the first
    uint32_t vec;                                   // d and e, mb * 64 floats each
    int32_t strip0, strips, sym0, full0;            // first strip, first tile of A and B, first tile of x among all
    float update;                                   // lr * scale
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
    int32_t count, strips;
    int32_t fmt_in, fmt_out;
    bool split;                                     // two numbers in A and B too, three products
    bool nesterov, update;                          // update: out is a parameter to be moved, otherwise it gets the result
    float momentum, decay, eps;
    float a, b, c;
    const float* grad_scale;
};

__device__ int g_error;                             // set by a wait that ran out

// ---- preparation -------------------------------------------------------------------------------------

__device__ __forceinline__ float load_any(const void* p, int64_t i, int32_t fmt) {
    return fmt == SSGD_FMT_F32 ? static_cast<const float*>(p)[i]
         : fmt == SSGD_FMT_F16 ? __half2float(static_cast<const __half*>(p)[i]) : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
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

// m <- momentum m + (1 - momentum) g, and the sum of squares of what is to be made orthogonal, per strip.  Squares are added in 64
// bits: they may leave the range of 32.
__global__ void __launch_bounds__(PREPARE_THREADS) k_momentum(const __grid_constant__ Group G, const __grid_constant__ Common C) {
    __shared__ double shared[PREPARE_THREADS / 32];
    successor_may_start();
    successor_wait();
    if (blockIdx.x == 0) {
        const uint32_t* from = reinterpret_cast<const uint32_t*>(&G);
        uint32_t* to = reinterpret_cast<uint32_t*>(C.at.matrices);
        for (int i = threadIdx.x; i < C.count * (int)(sizeof(Matrix) / 4); i += PREPARE_THREADS) to[i] = from[i];
    }
    const int strip = blockIdx.x;
    const Matrix& M = G.m[matrix_of(C.count, strip, [&](int i) { return G.m[i].strip0; })];
    const int local = strip - M.strip0, r0 = local % M.rb * BLOCK, c0 = local / M.rb * (STRIP_BLOCKS * BLOCK);
    const int h = min(BLOCK, M.rows - r0), w = min(STRIP_BLOCKS * BLOCK, M.cols - c0);
    const float scale = C.grad_scale ? *C.grad_scale : 1.f, mu = C.momentum;
    double sum = 0.0;
    int r = threadIdx.x / w, c = threadIdx.x % w;
    const int dr = PREPARE_THREADS / w, dc = PREPARE_THREADS % w;
    while (r < h) {
        float g = load_any(M.in, (int64_t)(r0 + r) * M.ld_in + c0 + c, C.fmt_in) * scale;
        if (M.m) {
            float* at = M.m + (int64_t)(r0 + r) * M.cols + c0 + c;
            const float m = fmaf(mu, *at, (1.f - mu) * g);
            *at = m;
            g = C.nesterov ? fmaf(mu, m, (1.f - mu) * g) : m;
        }
        sum += (double)g * (double)g;
        r += dr;
        c += dc;
        if (c >= w) { c -= w; ++r; }
    }
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) C.at.sums[strip] = sum;
}

// The nearest fp16 number and what it leaves
__device__ __forceinline__ void split(float v, __half& hi, __half& lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}
union Piece { uint4 v; __half h[8]; };

// x = u / (|u| + eps) as blocks
__global__ void __launch_bounds__(PREPARE_THREADS) k_layout(const __grid_constant__ Common C) {
    __shared__ double shared[PREPARE_THREADS / 32];
    successor_may_start();
    successor_wait();
    const int strip = blockIdx.x;
    const Matrix M = C.at.matrices[matrix_of(C.count, strip, [&](int i) { return C.at.matrices[i].strip0; })];
    double sum = 0.0;
    for (int i = threadIdx.x; i < M.strips; i += PREPARE_THREADS) sum += C.at.sums[M.strip0 + i];
    sum = block_sum(sum, shared);
    // 1 / (norm + eps) as a power of two and a factor near one: either alone may be out of range
    const double inv = 1.0 / (sqrt(sum) + (double)C.eps);
    int exponent = 0;
    const float factor = (float)(inv > 0.0 && inv < (double)INFINITY ? frexp(inv, &exponent) : inv) * SCALE;
    const float power = ldexpf(1.f, min(max(exponent, -126), 127));
    const int local = strip - M.strip0, rblock = local % M.rb, cblock0 = local / M.rb * STRIP_BLOCKS;
    const float scale = C.grad_scale ? *C.grad_scale : 1.f, mu = C.momentum;
    const uint32_t second = (uint32_t)M.rb * (uint32_t)M.cb;
    for (int cblock = cblock0; cblock < min(cblock0 + STRIP_BLOCKS, M.cb); ++cblock) {
        uint8_t* block = C.at.blocks + (int64_t)(M.x[0] + (uint32_t)cblock * M.rb + rblock) * BLOCK_BYTES;
        for (int i = threadIdx.x; i < BLOCK * 8; i += PREPARE_THREADS) {
            const int rr = i >> 3, piece = i & 7, r = rblock * BLOCK + rr, c = cblock * BLOCK + piece * 8;
            Piece hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float u = 0.f;
                if (r < M.rows && c + e < M.cols) {
                    u = load_any(M.in, (int64_t)r * M.ld_in + c + e, C.fmt_in) * scale;
                    if (M.m) {
                        const float m = M.m[(int64_t)r * M.cols + c + e];
                        u = C.nesterov ? fmaf(mu, m, (1.f - mu) * u) : m;
                    }
                    u = u * power * factor;
                }
                split(u, hi.h[e], lo.h[e]);
            }
            *reinterpret_cast<uint4*>(block + piece_at(rr, piece)) = hi.v;
            *reinterpret_cast<uint4*>(block + (int64_t)second * BLOCK_BYTES + piece_at(rr, piece)) = lo.v;
        }
    }
    asm volatile("fence.proxy.async.global;" ::: "memory");    // bulk copies read them
}

// ---- products ----------------------------------------------------------------------------------------

enum Kind { GRAM, POLYNOMIAL, APPLY, FINISH };

constexpr int TILE = 128;                           // rows and columns of a tile
constexpr int STAGES = 6;
constexpr int STAGE_BYTES = 4 * BLOCK_BYTES;
constexpr int EPILOGUE_WARPS = 4;
constexpr int THREADS = 32 * (EPILOGUE_WARPS + 2);

struct Shared {
    uint64_t full[STAGES], empty[STAGES], done[2], taken[2];
    uint32_t tmem;
    int gave_up;
    int32_t first[MAX_GROUP];
};
constexpr int SHARED_BYTES = 1024 + STAGES * STAGE_BYTES + (int)sizeof(Shared);

// One operand of a product: blocks [R][C] of which 128 rows or columns are needed at a time
struct Operand {
    const uint8_t* hi; const uint8_t* lo;
    int32_t R, mn_blocks;
    bool mn_major;
    __device__ __forceinline__ const uint8_t* block(bool low, int mn, int k) const {
        mn = min(mn, mn_blocks - 1);                // beyond the edge: rows or columns that are not stored
        const int64_t i = mn_major ? (int64_t)mn * R + k : (int64_t)k * R + mn;
        return (low ? lo : hi) + i * BLOCK_BYTES;
    }
};
struct Product {
    Operand A, B;
    int32_t steps, tiles_m;                         // blocks of the contraction; tiles along the rows
};

template <Kind KIND>
__device__ __forceinline__ Product product_of(const Common& C, const Matrix& M, int which) {
    auto at = [&](uint32_t block) { return C.at.blocks + (int64_t)block * BLOCK_BYTES; };
    const uint32_t xs = (uint32_t)M.rb * (uint32_t)M.cb, ms = (uint32_t)M.mb * (uint32_t)M.mb;
    const bool tall = M.tall();
    Product P;
    if (KIND == GRAM) {
        P.A = Operand{at(M.x[which]), at(M.x[which] + xs), M.rb, M.mb, tall};
        P.B = P.A;
        P.steps = tall ? M.rb : M.cb;
        P.tiles_m = (M.mb + 1) / 2;
    } else if (KIND == POLYNOMIAL) {
        P.A = Operand{at(M.a), at(M.a + ms), M.mb, M.mb, false};
        P.B = P.A;
        P.steps = M.mb;
        P.tiles_m = (M.mb + 1) / 2;
    } else {
        const Operand q{at(M.b), at(M.b + ms), M.mb, M.mb, false};
        P.A = tall ? Operand{at(M.x[which]), at(M.x[which] + xs), M.rb, M.rb, false} : q;
        P.B = tall ? q : Operand{at(M.x[which]), at(M.x[which] + xs), M.rb, M.cb, true};
        P.steps = M.mb;
        P.tiles_m = (M.rb + 1) / 2;
    }
    return P;
}

__device__ __forceinline__ void store_pieces(uint8_t* hi, uint8_t* lo, uint32_t at, const float (&v)[8], bool both) {
    Piece h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) split(v[e], h.h[e], l.h[e]);
    *reinterpret_cast<uint4*>(hi + at) = h.v;
    if (both) *reinterpret_cast<uint4*>(lo + at) = l.v;
}
__device__ __forceinline__ void load_pieces(const uint8_t* hi, const uint8_t* lo, uint32_t at, float (&v)[8], bool both) {
    Piece h, l;
    h.v = *reinterpret_cast<const uint4*>(hi + at);
    if (both) l.v = *reinterpret_cast<const uint4*>(lo + at);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __half2float(h.h[e]) + (both ? __half2float(l.h[e]) : 0.f);
}

// Eight results in a row of the output
template <typename T>
__device__ __forceinline__ void finish(const Common& C, const Matrix& M, int row, int col, const float (&v)[8]) {
    T* out = static_cast<T*>(M.out) + (int64_t)row * M.ld_out + col;
    const int n = min(8, M.cols - col);
    constexpr int VEC = 16 / sizeof(T);
    if (n == 8 && (reinterpret_cast<uintptr_t>(out) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 8; i += VEC) {
            Vec<T, VEC> o;
            if (C.update) o = load_vec<T, VEC>(out + i);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                o.e[e] = from_f32<T>(C.update ? fmaf(to_f32(o.e[e]), C.decay, -M.update * v[i + e]) : v[i + e]);
            store_vec<T, VEC>(out + i, o);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) out[e] = from_f32<T>(C.update ? fmaf(to_f32(out[e]), C.decay, -M.update * v[e]) : v[e]);
    }
}

// Eight accumulators of one row: what a product becomes
template <Kind KIND>
__device__ __forceinline__ void eight(const Common& C, const Matrix& M, int which, int row, int col, const float (&acc)[8], float row_factor) {
    const int rblock = row / BLOCK, rr = row % BLOCK, cblock = col / BLOCK, piece = col % BLOCK / 8;
    const uint32_t at = piece_at(rr, piece);
    auto block = [&](uint32_t first, int R) { return C.at.blocks + (int64_t)(first + (uint32_t)cblock * R + rblock) * BLOCK_BYTES; };
    const int64_t xs = (int64_t)M.rb * M.cb * BLOCK_BYTES, ms = (int64_t)M.mb * M.mb * BLOCK_BYTES;
    float* d = C.at.vec + M.vec;
    float* e = d + M.mb * BLOCK;
    float v[8];
    if constexpr (KIND == GRAM) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = acc[i] * (1.f / SCALE);
            if (row == col + i) {
                d[row] = v[i] * (1.f / SCALE);
                v[i] = 0.f;
            }
        }
        uint8_t* to = block(M.a, M.mb);
        store_pieces(to, to + ms, at, v, C.split);
    } else if constexpr (KIND == POLYNOMIAL) {
        const uint8_t* from = block(M.a, M.mb);
        float r[8];
        load_pieces(from, from + ms, at, r, C.split);
        const float4 d0 = *reinterpret_cast<const float4*>(d + col), d1 = *reinterpret_cast<const float4*>(d + col + 4);
        const float dj[8] = {d0.x, d0.y, d0.z, d0.w, d1.x, d1.y, d1.z, d1.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float square = fmaf(r[i], row_factor + dj[i], acc[i] * (1.f / SCALE));
            v[i] = fmaf(C.c, square, C.b * r[i]);
            if (row == col + i) {
                e[row] = fmaf(C.c, fmaf(row_factor, row_factor, acc[i] * (1.f / (SCALE * SCALE))), C.b * row_factor);
                v[i] = 0.f;
            }
        }
        uint8_t* to = block(M.b, M.mb);
        store_pieces(to, to + ms, at, v, C.split);
    } else {
        const uint8_t* from = block(M.x[which], M.rb);
        float x[8], f[8];
        load_pieces(from, from + xs, at, x, true);
        if (M.tall()) {
            const float4 e0 = *reinterpret_cast<const float4*>(e + col), e1 = *reinterpret_cast<const float4*>(e + col + 4);
            f[0] = e0.x + C.a; f[1] = e0.y + C.a; f[2] = e0.z + C.a; f[3] = e0.w + C.a;
            f[4] = e1.x + C.a; f[5] = e1.y + C.a; f[6] = e1.z + C.a; f[7] = e1.w + C.a;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = row_factor + C.a;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(f[i], x[i], acc[i] * (1.f / SCALE));
        if constexpr (KIND == APPLY) {
            uint8_t* to = block(M.x[which ^ 1], M.rb);
            store_pieces(to, to + xs, at, v, true);
        } else if (row < M.rows && col < M.cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= 1.f / SCALE;
            if (C.fmt_out == SSGD_FMT_F32) finish<float>(C, M, row, col, v);
            else if (C.fmt_out == SSGD_FMT_F16) finish<__half>(C, M, row, col, v);
            else finish<__nv_bfloat16>(C, M, row, col, v);
        }
    }
}

template <Kind KIND>
__global__ void __launch_bounds__(THREADS, 1) k_product(const __grid_constant__ Common C, int which, int tiles) {
    extern __shared__ uint8_t raw[];
    uint8_t* stage = raw + ((1024u - (shared_addr(raw) & 1023u)) & 1023u);
    Shared& S = *reinterpret_cast<Shared*>(stage + STAGES * STAGE_BYTES);
    volatile int* gave_up = &S.gave_up;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) { bar_init(&S.full[i], 1); bar_init(&S.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { bar_init(&S.done[i], 1); bar_init(&S.taken[i], EPILOGUE_WARPS); }
        bar_init_fence();
        S.gave_up = 0;
    }
    if (warp == EPILOGUE_WARPS) tmem_alloc(&S.tmem, 2 * TILE);
    successor_may_start();
    successor_wait();
    for (int i = threadIdx.x; i < C.count; i += THREADS)
        S.first[i] = KIND == GRAM || KIND == POLYNOMIAL ? C.at.matrices[i].sym0 : C.at.matrices[i].full0;
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = S.tmem;
    const int passes = C.split ? 3 : 1;
    auto find = [&](int tile) { return matrix_of(C.count, tile, [&](int i) { return S.first[i]; }); };

    if (warp == EPILOGUE_WARPS && lane == 0) {                  // copies
        asm volatile("fence.proxy.async.global;" ::: "memory");
        int s = 0, issued = 0;
        uint32_t parity = 1;
        bool ok = true;
        for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
            const int which_matrix = find(tile), local = tile - S.first[which_matrix];
            const Product P = product_of<KIND>(C, C.at.matrices[which_matrix], which);
            const int bm = local % P.tiles_m * 2, bn = local / P.tiles_m * 2;
            for (int pass = 0; pass < passes && ok; ++pass) {
                for (int k = 0; k < P.steps; ++k) {
                    if (!(ok = bar_wait(&S.empty[s], parity, gave_up))) break;
                    bar_expect(&S.full[s], STAGE_BYTES);
                    uint8_t* to = stage + s * STAGE_BYTES;
                    for (int i = 0; i < 2; ++i) bulk_load(to + i * BLOCK_BYTES, P.A.block(pass == 2, bm + i, k), BLOCK_BYTES, &S.full[s]);
                    for (int i = 0; i < 2; ++i) bulk_load(to + (2 + i) * BLOCK_BYTES, P.B.block(pass == 1, bn + i, k), BLOCK_BYTES, &S.full[s]);
                    ++issued;
                    if (++s == STAGES) { s = 0; parity ^= 1; }
                }
            }
        }
        // no copy may land in a CTA that is gone
        if (!ok)
            for (int i = 0; i < min(issued, STAGES); ++i) {
                const int last = issued - 1 - i;
                const uint64_t t0 = now_ns();
                while (!bar_try(&S.full[last % STAGES], (uint32_t)(last / STAGES) & 1u) && now_ns() - t0 < WAIT_NS) {}
            }
    } else if (warp == EPILOGUE_WARPS + 1 && lane == 0) {       // products
        int s = 0, buffer = 0;
        uint32_t parity = 0, parity_taken = 1;
        bool ok = true;
        for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
            const Product P = product_of<KIND>(C, C.at.matrices[find(tile)], which);
            const uint32_t instr = instruction(TILE, TILE, P.A.mn_major, P.B.mn_major);
            const uint64_t step_a = operand_step(P.A.mn_major), step_b = operand_step(P.B.mn_major);
            const uint32_t d = tmem + buffer * TILE;
            if (!(ok = bar_wait(&S.taken[buffer], parity_taken, gave_up))) break;
            fence_after();
            const int total = passes * P.steps;
            for (int k = 0; k < total; ++k) {
                if (!(ok = bar_wait(&S.full[s], parity, gave_up))) break;
                fence_after();
                const uint32_t at = shared_addr(stage + s * STAGE_BYTES);
                const uint64_t a = operand(at, P.A.mn_major), b = operand(at + 2 * BLOCK_BYTES, P.B.mn_major);
#pragma unroll
                for (int i = 0; i < 4; ++i) mma(d, a + i * step_a, b + i * step_b, instr, k > 0 || i > 0);
                commit(&S.empty[s]);
                if (++s == STAGES) { s = 0; parity ^= 1; }
            }
            commit(&S.done[buffer]);
            if (buffer) parity_taken ^= 1;
            buffer ^= 1;
        }
    } else if (warp < EPILOGUE_WARPS) {                         // results
        int buffer = 0;
        uint32_t parity = 0;
        for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
            const int which_matrix = find(tile), local = tile - S.first[which_matrix];
            const Matrix& M = C.at.matrices[which_matrix];
            const int tiles_m = KIND == GRAM || KIND == POLYNOMIAL ? (M.mb + 1) / 2 : (M.rb + 1) / 2;
            const int row = local % tiles_m * TILE + warp * 32 + lane, col0 = local / tiles_m * TILE;
            const int R = KIND == GRAM || KIND == POLYNOMIAL ? M.mb : M.rb, K = KIND == GRAM || KIND == POLYNOMIAL ? M.mb : M.cb;
            float factor = 0.f;
            const bool stored = row < R * BLOCK;
            if (stored && KIND == POLYNOMIAL) factor = C.at.vec[M.vec + row];
            if (stored && (KIND == APPLY || KIND == FINISH) && !M.tall()) factor = C.at.vec[M.vec + M.mb * BLOCK + row];
            if (!bar_wait(&S.done[buffer], parity, gave_up)) break;
            __syncwarp();
            fence_after();
#pragma unroll 1
            for (int half = 0; half < TILE / 32; ++half) {
                const int col = col0 + half * 32;
                uint32_t acc[32];
                tmem_load32(tmem + buffer * TILE + half * 32 + ((uint32_t)warp << 21), acc);
                tmem_wait();
                if (stored && col < K * BLOCK) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float v[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(acc[i * 8 + j]);
                        eight<KIND>(C, M, which, row, col + i * 8, v, factor);
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(&S.taken[buffer]);
            if (buffer) parity ^= 1;
            buffer ^= 1;
        }
    }
    __syncwarp();
    // the results were written by ordinary stores and are read by bulk copies, of the next launch
    asm volatile("fence.proxy.async.global;" ::: "memory");
    fence_before();
    __syncthreads();
    fence_after();
    if (threadIdx.x == 0 && S.gave_up) atomicExch(&g_error, 1);
    if (warp == EPILOGUE_WARPS) tmem_free(tmem, 2 * TILE);
}

// ---- host side ---------------------------------------------------------------------------------------

struct Sizes {
    int64_t blocks = 0, floats = 0, strips = 0, sym = 0, full = 0, elements = 0;
    int count = 0;
    int64_t sums_at() const { return (int64_t)sizeof(Matrix) * MAX_GROUP; }
    int64_t vec_at() const { return (sums_at() + strips * 8 + 127) / 128 * 128; }
    int64_t blocks_at() const { return (vec_at() + floats * 4 + 1023) / 1024 * 1024; }
    int64_t bytes() const { return blocks_at() + blocks * BLOCK_BYTES; }
};

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Adds a matrix to a group; false if there is no room
bool add(Sizes& s, const ssgd_matrix& t, bool split, Matrix* to) {
    const int64_t elements = (int64_t)t.rows * t.cols;
    if (s.count == MAX_GROUP || (s.count && s.elements + elements > GROUP_ELEMENTS)) return false;
    Matrix M{};
    M.rows = (int32_t)t.rows; M.cols = (int32_t)t.cols;
    M.rb = (int32_t)div_up(t.rows, BLOCK); M.cb = (int32_t)div_up(t.cols, BLOCK);
    M.mb = M.rb < M.cb ? M.rb : M.cb;
    const int64_t xs = (int64_t)M.rb * M.cb, ms = (int64_t)M.mb * M.mb;
    M.x[0] = (uint32_t)s.blocks; M.x[1] = (uint32_t)(s.blocks + 2 * xs);
    M.a = (uint32_t)(s.blocks + 4 * xs); M.b = (uint32_t)(s.blocks + 4 * xs + (split ? 2 : 1) * ms);
    s.blocks += 4 * xs + (split ? 4 : 2) * ms;
    M.vec = (uint32_t)s.floats;
    s.floats += 2 * (int64_t)M.mb * BLOCK;
    M.strip0 = (int32_t)s.strips; M.strips = (int32_t)(M.rb * div_up(M.cb, STRIP_BLOCKS));
    M.sym0 = (int32_t)s.sym; M.full0 = (int32_t)s.full;
    s.strips += M.strips;
    s.sym += div_up(M.mb, 2) * div_up(M.mb, 2);
    s.full += div_up(M.rb, 2) * div_up(M.cb, 2);
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

template <Kind KIND>
int launch_product(cudaStream_t st, const Common& C, int which, int64_t tiles, int sms) {
    static PerDevice known;
    int fits = 0;
    if (int e = residency(k_product<KIND>, THREADS, SHARED_BYTES, known, &fits)) return e;
    return launch(st, k_product<KIND>, (int)(tiles < sms ? tiles : sms), THREADS, SHARED_BYTES, C, which, (int)tiles);
}

constexpr int64_t MAX_SIDE = (int64_t)1 << 20;
constexpr int MAX_STEPS = 32;

// The polynomial has to keep what starts within [0, 1] well inside the range of the stored numbers.
bool stays_in_range(int steps, double a, double b, double c) {
    for (int i = 0; i <= 64; ++i) {
        double s = i / 64.0;
        for (int k = 0; k < steps; ++k) {
            const double q = s * s, p = b * q + c * q * q;
            if (!(q <= 16.0) || !(p > -48.0 && p < 48.0)) return false;
            s *= a + p;
        }
        if (!(s > -8.0 && s < 8.0)) return false;
    }
    return true;
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
        if (!aligned_to(t[i].in, fmt_bytes(fmt_in)) || !aligned_to(t[i].out, fmt_bytes(fmt_out)) || !aligned_to(t[i].m, 4)) return SSGD_EALIGN;
    }
    return SSGD_OK;
}

int64_t workspace_of(const ssgd_matrix* t, int32_t count, bool split) {
    int64_t most = 0;
    Sizes s;
    for (int32_t i = 0; i < count; ++i) {
        if (!t[i].rows || !t[i].cols) continue;
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
    if (need == 0) return SSGD_OK;
    if (!workspace || (int64_t)bytes < need) return SSGD_EWORKSPACE;
    if (!aligned_to(workspace, 16)) return SSGD_EALIGN;
    int sms = 0, e = sm_count_of_current_device(&sms);
    if (e) return e;
    int32_t i = 0;
    while (i < count) {
        Group G;
        Sizes s;
        for (; i < count; ++i) {
            if (!t[i].rows || !t[i].cols) continue;
            if (!add(s, t[i], C.split, s.count < MAX_GROUP ? &G.m[s.count] : nullptr)) break;
            G.m[s.count - 1].update = (float)(lr * t[i].scale);
        }
        if (!s.count) break;
        uint8_t* base = static_cast<uint8_t*>(workspace);
        C.at = Space{reinterpret_cast<Matrix*>(base), reinterpret_cast<double*>(base + s.sums_at()),
                     reinterpret_cast<float*>(base + s.vec_at()), base + s.blocks_at()};
        C.count = s.count;
        C.strips = (int32_t)s.strips;
        if ((e = launch(st, k_momentum, (int)s.strips, PREPARE_THREADS, 0, G, C))) return e;
        if ((e = launch(st, k_layout, (int)s.strips, PREPARE_THREADS, 0, C))) return e;
        for (int k = 0; k < steps; ++k) {
            if ((e = launch_product<GRAM>(st, C, k & 1, s.sym, sms))) return e;
            if ((e = launch_product<POLYNOMIAL>(st, C, k & 1, s.sym, sms))) return e;
            if ((e = k + 1 < steps ? launch_product<APPLY>(st, C, k & 1, s.full, sms) : launch_product<FINISH>(st, C, k & 1, s.full, sms))) return e;
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
    C.decay = (float)(1.0 - lr * weight_decay);
    C.eps = (float)eps;
    C.a = (float)a; C.b = (float)b; C.c = (float)c;
    C.grad_scale = grad_scale;
    return run(matrices, count, C, steps, lr, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

int ssgd_train_ops_status(void* stream) {
    if (cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) != cudaSuccess) return SSGD_ECUDA;
    int seen = 0, none = 0;
    if (cudaMemcpyFromSymbol(&seen, g_error, sizeof seen) != cudaSuccess) return SSGD_ECUDA;
    if (!seen) return SSGD_OK;
    return cudaMemcpyToSymbol(g_error, &none, sizeof none) == cudaSuccess ? SSGD_EDEVICE : SSGD_ECUDA;
}

}  // extern "C"
