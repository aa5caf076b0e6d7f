// Muon step: momentum, an update orthogonalised by Newton-Schulz products, decay (see rfast_muon_step in rfast.h for the formulas).
//
// With X the update over its norm, m x n and m <= n (transposed where it is higher than wide), an iteration is three products,
//     A = X X'            (symmetric)
//     B = b A + c A A     (symmetric)
//     X = a X + B X       (B holds a on its diagonal as well: X = B X)
// and five iterations are nearly all the work: 5 (3 m^2 n + m^3) operations when only half of each symmetric product is formed.  They
// run on the tensor cores in fp16 with fp32 sums.  A factor is one fp16 number, or (terms = 2) the sum of two, 22 bits, of which three
// products are formed: high by high, high by low, low by high.  X lies within [-1.3, 1.3] and is held times 2^14, A and B within 3.5, times
// 2^13, so that neither the range nor, for the low halves, the least normal number of fp16 is met.
//
// Matrices of one shape lie in one array of the workspace, so that one launch per product serves all matrices of up to eight shapes.
// Tiles go to pairs of thread blocks, 256 x 256 per pair (one matrix instruction for both), or, where those are too few for the
// GPU, to single ones, 128 x 64.  In a block one warp brings tiles by TMA through a ring of stages, one issues the matrix
// instructions, eight read the sums of one tile out of tensor memory while the next is being formed.
//
// What bounds it: the tensor pipe for large matrices (4096 x 4096 bf16: active 89 to 95 %, 1.46 PFLOP/s in A and B, 1.59 in X, at the power limit),
// epilogues and few waves of tiles for middle ones (512 x 784 f32: 53 to 82 %), the 5 us of a launch's chain for small ones.  All products
// in one cooperative launch whose blocks meet after each were no faster (257 x 129: 93 us against 86).
//
// Every wait on a barrier is bounded: when it runs out the block leaves a code in the workspace's first word and ends.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdio>

#include "ops.h"
#include "tensor_core.cuh"
#include "values.cuh"

namespace rfast {

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kXUnit = 16384.f, kSUnit = 8192.f;           // X and A, B as they are held
constexpr int kMats = 128, kGroups = 8;                       // matrices and shapes of one run of launches
constexpr int kPart = 16384;                                  // values of a block of the first kernel
constexpr int kBox = 64, kBoxBytes = kBox * kBox * 2;         // a TMA box: 64 rows of 64 values
// The tensor cores' fp32 sums round towards zero, by up to 2^-23 of the sum with every instruction: a long sum of squares comes out
// small.  With two terms a factor's digits are worth more than that, so X X' is summed in registers every four boxes (256 values):
// 1 x 4096 3.7e-5 -> 1.3e-6 off.  The other products' terms have either sign, and their errors cancel.
constexpr int kSegment = 4;
constexpr int kEpiWarps = 8, kThreads = 64 + 32 * kEpiWarps;
constexpr int kPairs = 74, kSms = 148;

enum Product { kGram = 0, kPoly = 1, kApply = 2, kUpdate = 3 };   // A; B; X; the last X, applied to the parameters

struct MuonMat {
    void* param;
    const void* grad;
    float* momentum;
    int rows, cols;
    int group, slot;
    float step;                        // lr * size
    int wide;                          // 32 bytes of a row at a time
};
struct MuonTable {
    MuonMat mat[kMats];
    int part0[kMats + 1], tile0[kMats + 1];       // running counts of the first two kernels' blocks
    int count;
};
struct MuonGroup {
    int m, n, np, mp, count;
    int turned;                        // parameters are n x m: X is their update's transpose
    int mat0;                          // its first matrix in the table
    int tile0;                         // of the launch
    int64_t x, s;                      // byte offsets of its arrays in the workspace
    int64_t x_plane, s_plane;          // values of [count][m][pitch]: high halves; the low ones follow, then the other buffer
};
struct MuonGemm {
    CUtensorMap x[kGroups], s[kGroups];
    MuonGroup g[kGroups];
    int groups, tiles, in;             // `in`: the buffer of X that is read
    int back;                          // tiles from the last to the first
    float keep;                        // 1 - lr weight_decay
    char* work;
    const MuonMat* mats;               // in the workspace
};

struct MuonScalars {
    float mu, omu;                     // momentum, 1 - momentum
    int nesterov, grad_type, terms;
    double eps;
    const float* scale;
};

__device__ __forceinline__ int find(const int* first, int count, int at) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= at) lo = mid; else hi = mid;
    }
    return lo;
}

// ---- momentum and norm --------------------------------------------------------------------------
// m = mu m + (1 - mu) g; the squares of u = m, or (1 - mu) g + mu m, in 64 bits.
template <class GT>
__device__ __forceinline__ double momentum_part(const MuonMat& a, const MuonScalars& c, int64_t lo, int64_t hi) {
    const float scale = c.scale ? *c.scale : 1.f;
    const GT* g = (const GT*)a.grad;
    double sum = 0.0;
    const auto one = [&](float& m, float gv) {
        gv *= scale;
        m = fmaf(c.mu, m, c.omu * gv);
        const float u = c.nesterov ? fmaf(c.mu, m, c.omu * gv) : m;
        sum = fma((double)u, (double)u, sum);
    };
    if ((uintptr_t)g % (8 * sizeof(GT)) == 0 && (uintptr_t)a.momentum % 32 == 0) {
        const int64_t end = lo + (hi - lo) / 8 * 8;
#pragma unroll 2
        for (int64_t i = lo + threadIdx.x * 8; i < end; i += 256 * 8) {
            float gv[8], mv[8];
            unpack8(load8(g + i), gv);
            unpack8(load8(a.momentum + i), mv);
#pragma unroll
            for (int k = 0; k < 8; ++k) one(mv[k], gv[k]);
            store8(a.momentum + i, mv);
        }
        lo = end;
    }
    for (int64_t i = lo + threadIdx.x; i < hi; i += 256) {
        float m = a.momentum[i];
        one(m, value_of(g[i]));
        a.momentum[i] = m;
    }
    return sum;
}

__device__ __forceinline__ double block_sum(double v, double* sh) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += sh[w];
    return s;
}

__global__ void __launch_bounds__(256)
k_muon_momentum(const __grid_constant__ MuonTable t, MuonScalars c, double* parts, MuonMat* mats, int* status) {
    __shared__ double sh[8];
    let_follow();
    if (blockIdx.x == 0) {
        if (threadIdx.x == 0 && status) *status = 0;
        for (int k = threadIdx.x; k < t.count; k += 256) mats[k] = t.mat[k];
    }
    const int k = find(t.part0, t.count, blockIdx.x);
    const MuonMat a = t.mat[k];
    const int64_t all = (int64_t)a.rows * a.cols, lo = (int64_t)(blockIdx.x - t.part0[k]) * kPart, hi = lo + kPart < all ? lo + kPart : all;
    double s;
    if (c.grad_type == RFAST_TYPE_F32) s = momentum_part<float>(a, c, lo, hi);
    else if (c.grad_type == RFAST_TYPE_BF16) s = momentum_part<__nv_bfloat16>(a, c, lo, hi);
    else s = momentum_part<__half>(a, c, lo, hi);
    s = block_sum(s, sh);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// Eight values as one or two fp16 numbers each.
template <int TERMS>
__device__ __forceinline__ void keep8(__half* to, int64_t low_plane, const float (&v)[8]) {
    uint32_t high[4], low[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
        high[k] = *reinterpret_cast<const uint32_t*>(&h);
        if (TERMS == 2) {
            const float2 f = __half22float2(h);
            const __half2 l = __floats2half2_rn(v[2 * k] - f.x, v[2 * k + 1] - f.y);
            low[k] = *reinterpret_cast<const uint32_t*>(&l);
        }
    }
    *reinterpret_cast<uint4*>(to) = make_uint4(high[0], high[1], high[2], high[3]);
    if (TERMS == 2) *reinterpret_cast<uint4*>(to + low_plane) = make_uint4(low[0], low[1], low[2], low[3]);
}

// 64 x 64 values of u, times f1 f2, zeros beyond the matrix.
template <class GT>
__device__ __forceinline__ void begin_tile(const MuonMat& a, const MuonScalars& c, int r0, int c0, float scale, float f1, float f2, float (*tile)[65]) {
    const GT* const g = (const GT*)a.grad;
    const bool wide = a.cols % 8 == 0 && (uintptr_t)g % (8 * sizeof(GT)) == 0 && (uintptr_t)a.momentum % 32 == 0;
    const auto value = [&](float m, float gv) { return (c.nesterov ? fmaf(c.mu, m, c.omu * (gv * scale)) : m) * f1 * f2; };
    if (wide) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = (threadIdx.x >> 3) + 32 * u, col = (threadIdx.x & 7) * 8;
            float m[8] = {}, gv[8] = {};
            if (r0 + r < a.rows && c0 + col < a.cols) {
                const int64_t i = (int64_t)(r0 + r) * a.cols + c0 + col;
                unpack8(load8((const float*)a.momentum + i), m);
                if (c.nesterov) unpack8(load8(g + i), gv);
            }
#pragma unroll
            for (int w = 0; w < 8; ++w) tile[r][col + w] = value(m[w], gv[w]);
        }
    } else {
#pragma unroll 8
        for (int e = threadIdx.x; e < 64 * 64; e += 256) {
            const int r = e >> 6, col = e & 63;
            float m = 0.f, gv = 0.f;
            if (r0 + r < a.rows && c0 + col < a.cols) {
                const int64_t i = (int64_t)(r0 + r) * a.cols + c0 + col;
                m = a.momentum[i];
                if (c.nesterov) gv = value_of(g[i]);
            }
            tile[r][col] = value(m, gv);
        }
    }
}

// X = u / max(norm, eps), m x n, as it is held: 64 x 64 values of the parameter's shape per block.  Every block adds up its matrix's
// squares from the first kernel's sums by itself: 34 MB out of the L2 cache at 4096 x 4096, 8.6 GB (of 79 ms) at 16384 x 16384.
__global__ void __launch_bounds__(256)
k_muon_begin(const __grid_constant__ MuonTable t, MuonScalars c, const double* parts, const __grid_constant__ MuonGemm q) {
    __shared__ double sh[8];
    __shared__ float tile[64][65];
    follow();
    let_follow();
    const int k = find(t.tile0, t.count, blockIdx.x);
    const MuonMat a = t.mat[k];
    double s = 0.0;
    for (int i = t.part0[k] + threadIdx.x; i < t.part0[k + 1]; i += 256) s += parts[i];
    const double norm = sqrt(block_sum(s, sh));
    // a NaN goes through; the factor is split in two, so that neither it nor what it makes of a value leaves fp32 (a norm above 0 is at
    // least 2^-149, and the factor below 2^170)
    const double unit = (double)kXUnit / (norm < c.eps ? c.eps : norm);
    int e = 0;
    const double digits = frexp(unit < 0x1p170 ? unit : norm > 0 || norm != norm ? unit : 0x1p170, &e);
    const float f1 = (float)ldexp(1.0, e / 2), f2 = (float)ldexp(digits, e - e / 2);
    const int tiles_c = (a.cols + 63) / 64, at = blockIdx.x - t.tile0[k];
    const int r0 = at / tiles_c * 64, c0 = at % tiles_c * 64;
    const float scale = c.scale ? *c.scale : 1.f;
    if (c.grad_type == RFAST_TYPE_F32) begin_tile<float>(a, c, r0, c0, scale, f1, f2, tile);
    else if (c.grad_type == RFAST_TYPE_BF16) begin_tile<__nv_bfloat16>(a, c, r0, c0, scale, f1, f2, tile);
    else begin_tile<__half>(a, c, r0, c0, scale, f1, f2, tile);
    __syncthreads();
    const MuonGroup& g = q.g[a.group];
    const bool turned = a.rows > a.cols;
    __half* x = (__half*)(q.work + g.x) + (int64_t)a.slot * g.m * g.np;
    const int i0 = turned ? c0 : r0, j0 = turned ? r0 : c0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {                           // 64 rows of X, eight values a thread
        const int i = (threadIdx.x >> 3) + 32 * u, j = (threadIdx.x & 7) * 8;
        if (i0 + i >= g.m || j0 + j >= g.np) continue;
        float v[8];
#pragma unroll
        for (int w = 0; w < 8; ++w) v[w] = turned ? tile[j + w][i] : tile[i][j + w];
        __half* const to = x + (int64_t)(i0 + i) * g.np + j0 + j;
        if (c.terms == 2) keep8<2>(to, g.x_plane, v); else keep8<1>(to, 0, v);
    }
}

// ---- products -----------------------------------------------------------------------------------
template <int CG, int TERMS>
struct Shape {
    static constexpr int kTM = CG == 2 ? 256 : 128, kTN = CG == 2 ? 256 : 64;
    static constexpr int kBoxesA = 2, kBoxesB = CG == 2 ? 2 : 1;                 // of one thread block
    static constexpr int kHalf = (kBoxesA + kBoxesB) * kBoxBytes;                // the high (or low) halves of a stage
    static constexpr int kStage = TERMS * kHalf;
    static constexpr int kStages = CG == 2 ? (TERMS == 2 ? 3 : 6) : 4;
    static constexpr int kStaged = 32 * 33 * 4;                                  // a warp's 32 x 32 values
    static constexpr int kShared = 1024 + kStages * kStage + kEpiWarps * kStaged;
    static constexpr int kColumns = 2 * kTN;                                     // of tensor memory: two tiles' sums
};

struct Tile {
    int g, mat, i, j;
};
// Tiles of a matrix's product: m x n, up to the diagonal where SYM.
template <int TM, int TN, bool SYM>
__host__ __device__ inline int tiles_of(int m, int n) {
    const int ti = (m + TM - 1) / TM;
    if (!SYM) return ti * ((n + TN - 1) / TN);
    // columns up to the diagonal: TM / TN tiles more in every row, the last one cut at m
    constexpr int q = TM / TN;
    const int last = (m + TN - 1) / TN;
    return q * ti * (ti - 1) / 2 + (last < q * ti ? last : q * ti);
}
// What a product's result has for rows and columns: the update has the parameter's.
template <int OP> __host__ __device__ inline int result_rows(const MuonGroup& g) { return OP == kUpdate && g.turned ? g.n : g.m; }
template <int OP> __host__ __device__ inline int result_cols(const MuonGroup& g) { return OP == kGram || OP == kPoly || (OP == kUpdate && g.turned) ? g.m : g.n; }
template <int TM, int TN, int OP>
__device__ __forceinline__ Tile tile_at(const MuonGemm& p, int t) {
    constexpr bool SYM = OP == kGram || OP == kPoly;
    if (p.back) t = p.tiles - 1 - t;
    Tile r;
    r.g = 0;
    while (r.g + 1 < p.groups && p.g[r.g + 1].tile0 <= t) ++r.g;
    const MuonGroup& g = p.g[r.g];
    const int per = tiles_of<TM, TN, SYM>(result_rows<OP>(g), result_cols<OP>(g));
    t -= g.tile0;
    r.mat = t / per;
    t -= r.mat * per;
    if (SYM) {
        constexpr int q = TM / TN;
        int i = (int)((sqrtf(1.f + 8.f * (float)t / q) - 1.f) * 0.5f);
        while (q * (i + 1) * (i + 2) / 2 <= t) ++i;
        while (q * i * (i + 1) / 2 > t) --i;
        r.i = i;
        r.j = t - q * i * (i + 1) / 2;
    } else {
        const int ti = (result_rows<OP>(g) + TM - 1) / TM;
        r.i = t % ti;
        r.j = t / ti;
    }
    return r;
}

// A warp finishes 32 x 32 sums at a time, straight from the registers that tensor memory is read into: a lane has a row of X, A or B, 32
// neighbours, whole 32-byte sectors.  (Staging them in shared memory for longer runs was four times slower: the operands' reads
// and the loads' writes take all of its bandwidth.)

// 32 values as one or two fp16 numbers each; `values` of them are stored, in sixteens (a row's room is a multiple of that).
template <int TERMS>
__device__ __forceinline__ void keep32(__half* to, int64_t low_plane, const float (&v)[32], int values) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (q * 16 >= values) break;
        uint32_t high[8], low[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float a = v[16 * q + 2 * k], b = v[16 * q + 2 * k + 1];
            const __half2 h = __floats2half2_rn(a, b);
            high[k] = *reinterpret_cast<const uint32_t*>(&h);
            if (TERMS == 2) {
                const float2 f = __half22float2(h);
                const __half2 l = __floats2half2_rn(a - f.x, b - f.y);
                low[k] = *reinterpret_cast<const uint32_t*>(&l);
            }
        }
        store32(to + 16 * q, high);
        if (TERMS == 2) store32(to + 16 * q + low_plane, low);
    }
}

// What a block's finish reads from memory, fetched while the sums are formed: A for B, the parameters for the update.
template <int OP, int TERMS, class T>
struct Ahead {
    __device__ __forceinline__ void load(const MuonGemm&, const MuonGroup&, int, const MuonMat*, int, int) {}
};
template <int TERMS, class T>
struct Ahead<kPoly, TERMS, T> {
    uint32_t q[2 * TERMS][8];
    __device__ __forceinline__ void load(const MuonGemm& p, const MuonGroup& g, int slot, const MuonMat*, int row0, int col0) {
        const int row = row0 + (threadIdx.x & 31);
        const __half* a = (const __half*)(p.work + g.s) + (int64_t)slot * g.m * g.mp + (int64_t)row * g.mp + col0;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (row < g.m && col0 + 16 * k < g.mp)
#pragma unroll
                for (int h = 0; h < TERMS; ++h) load32(a + 16 * k + h * g.s_plane, q[2 * h + k]);
    }
};
// Parameters, two ways: 32 neighbours of a lane's row, 32 bytes at a time (wide), or 32 rows of a lane's column, the sums brought there
// through shared memory (rows whose length or place does not allow for the first way).
template <class T> __device__ __forceinline__ uint32_t raw_of(const T* p) {
    if constexpr (sizeof(T) == 4) return *reinterpret_cast<const uint32_t*>(p);
    else return *reinterpret_cast<const uint16_t*>(p);
}
template <class T> __device__ __forceinline__ float value_of_raw(uint32_t r);
template <> __device__ __forceinline__ float value_of_raw<float>(uint32_t r) { return __uint_as_float(r); }
template <> __device__ __forceinline__ float value_of_raw<__nv_bfloat16>(uint32_t r) { return __uint_as_float(r << 16); }
template <> __device__ __forceinline__ float value_of_raw<__half>(uint32_t r) { return __half2float(__ushort_as_half((unsigned short)r)); }
template <class T> __device__ __forceinline__ float2 two_values(uint32_t r);
template <> __device__ __forceinline__ float2 two_values<__half>(uint32_t r) { return __half22float2(*reinterpret_cast<const __half2*>(&r)); }
template <> __device__ __forceinline__ float2 two_values<__nv_bfloat16>(uint32_t r) { return make_float2(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u)); }

template <int TERMS, class T>
struct Ahead<kUpdate, TERMS, T> {
    uint32_t q[32];
    __device__ __forceinline__ void load(const MuonGemm&, const MuonGroup&, int, const MuonMat* mat, int row0, int col0) {
        const int lane = threadIdx.x & 31;
        const T* const param = (const T*)mat->param;
        if (mat->wide) {
            constexpr int kValues = 32 / (int)sizeof(T);
            const T* w = param + (int64_t)(row0 + lane) * mat->cols + col0;
            const int n = row0 + lane < mat->rows ? mat->cols - col0 : 0;
#pragma unroll
            for (int k = 0; k < 32 / kValues; ++k)
                if (k * kValues < n) load32(w + k * kValues, *reinterpret_cast<uint32_t(*)[8]>(q + 8 * k));
        } else {
            const T* w = param + (int64_t)row0 * mat->cols + col0 + lane;
            const int m = col0 + lane < mat->cols ? mat->rows - row0 : 0;
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (k < m) q[k] = raw_of(w + (int64_t)k * mat->cols);
        }
    }
};

template <int TERMS, class T>
__device__ __forceinline__ void update_block(const MuonMat* mat, int row0, int col0, float (&v)[32], float (*st)[33], const Ahead<kUpdate, TERMS, T>& now, float keep) {
    const int lane = threadIdx.x & 31;
    const float step = mat->step * (1.f / (kSUnit * kXUnit));
    T* const param = (T*)mat->param;
    if (mat->wide) {
        constexpr int kValues = 32 / (int)sizeof(T);
        T* const w = param + (int64_t)(row0 + lane) * mat->cols + col0;
        const int n = row0 + lane < mat->rows ? mat->cols - col0 : 0;
#pragma unroll
        for (int k = 0; k < 32 / kValues; ++k) {
            if (k * kValues >= n) break;
            uint32_t r[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (sizeof(T) == 4) {
                    r[e] = __float_as_uint(fmaf(-step, v[k * 8 + e], __uint_as_float(now.q[k * 8 + e]) * keep));
                } else {
                    const float2 o = two_values<T>(now.q[k * 8 + e]);
                    r[e] = packed(fmaf(-step, v[k * 16 + 2 * e], o.x * keep), fmaf(-step, v[k * 16 + 2 * e + 1], o.y * keep), (const T*)nullptr);
                }
            }
            store32(w + k * kValues, r);
        }
    } else {
#pragma unroll
        for (int c = 0; c < 32; ++c) st[lane][c] = v[c];
        __syncwarp();
        T* const w = param + (int64_t)row0 * mat->cols + col0 + lane;
        const int m = col0 + lane < mat->cols ? mat->rows - row0 : 0;
#pragma unroll
        for (int k = 0; k < 32; ++k)
            if (k < m) w[(int64_t)k * mat->cols] = rounded<T>(fmaf(-step, st[k][lane], value_of_raw<T>(now.q[k]) * keep));
        __syncwarp();
    }
}

template <int OP, int TERMS, class T>
__device__ __forceinline__ void finish_block(const MuonGemm& p, const MuonGroup& g, int slot, const MuonMat* mat, int row0, int col0, float (&v)[32], float (*st)[33], const Ahead<OP, TERMS, T>& now) {
    const int lane = threadIdx.x & 31, row = row0 + lane;
    if constexpr (OP == kGram || OP == kPoly) {
        // B holds a on the diagonal, so that B X is the next X
        __half* const to = (__half*)(p.work + g.s) + (OP == kPoly ? TERMS * g.s_plane : 0) + (int64_t)slot * g.m * g.mp + (int64_t)row * g.mp + col0;
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
            if constexpr (OP == kPoly) {
                float2 a = two_values<__half>(now.q[c / 16][c / 2 % 8]);
                if constexpr (TERMS == 2) {
                    const float2 low = two_values<__half>(now.q[2 + c / 16][c / 2 % 8]);
                    a.x += low.x;
                    a.y += low.y;
                }
                v[c] = fmaf(kB, a.x, v[c] * (kC / kSUnit));
                v[c + 1] = fmaf(kB, a.y, v[c + 1] * (kC / kSUnit));
                if (row0 == col0) {
                    v[c] += lane == c ? kA * kSUnit : 0.f;
                    v[c + 1] += lane == c + 1 ? kA * kSUnit : 0.f;
                }
            } else {
                v[c] *= kSUnit / (kXUnit * kXUnit);
                v[c + 1] *= kSUnit / (kXUnit * kXUnit);
            }
        }
        if (row < g.m) keep32<TERMS>(to, g.s_plane, v, g.mp - col0);
    } else if constexpr (OP == kApply) {
        __half* const to = (__half*)(p.work + g.x) + (p.in ^ 1) * TERMS * g.x_plane + (int64_t)slot * g.m * g.np + (int64_t)row * g.np + col0;
#pragma unroll
        for (int c = 0; c < 32; ++c) v[c] *= 1.f / kSUnit;
        if (row < g.m) keep32<TERMS>(to, g.x_plane, v, g.np - col0);
    } else {
        update_block<TERMS, T>(mat, row0, col0, v, st, now, p.keep);
    }
}

// Whether an operand is read with rows along the other dimension than the sum's: X but for X X', A and B above what is stored of them.
template <int OP>
__device__ __forceinline__ bool across(bool x, bool above) { return x ? OP != kGram : above; }
// A and B are stored up to this column in the row tile of `row`: only tiles up to the diagonal are formed.  All products of a run use tiles
// of one shape, so that an operand's rows lie in one row tile.
template <class S>
__device__ __forceinline__ int stored_up_to(int row) { return (row / S::kTM + 1) * S::kTM; }
// The first box of a tile's sum.  A, and B with a on its diagonal, are nearly diagonal once X is nearly orthogonal: with two terms, whose
// digits show it, the boxes that hold the diagonal come last, so that no term is added to a large sum and rounded towards zero with
// it (4001 x 2999: 9.6e-5 -> 1.9e-5 off).
template <class S, int OP, int TERMS>
__device__ __forceinline__ int first_box(const Tile& at, int turned, int blocks) {
    if (OP == kGram || TERMS == 1) return 0;
    const int b = (OP == kUpdate && turned ? (at.j + 1) * S::kTN : (at.i + 1) * S::kTM) / kBox;
    return b < blocks ? b : 0;
}

template <int CG, int TERMS, int OP, class T>         // T: of the parameters, for kUpdate
__global__ void __launch_bounds__(kThreads, 1)
k_muon_product(const __grid_constant__ MuonGemm p) {
    using S = Shape<CG, TERMS>;
    constexpr bool kSegmented = OP == kGram && TERMS == 2;
    extern __shared__ uint8_t raw[];
    uint8_t* const base = raw + (0u - tc::smem(raw) & 1023u);      // by an offset: the compiler goes on knowing that this is shared memory
    __shared__ uint64_t full[S::kStages], empty[S::kStages], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem;
    __shared__ volatile int bad;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? tc::cluster_rank() : 0;
    int* const status = (int*)p.work;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) { tc::bar_init(&full[s], 1); tc::bar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { tc::bar_init(&acc_full[b], 1); tc::bar_init(&acc_empty[b], CG * kEpiWarps); }
        bad = 0;
        tc::bar_init_fence();
    }
    if (warp == 0 && lane < p.groups) {
        tc::map_ahead(&p.x[lane]);
        tc::map_ahead(&p.s[lane]);
    }
    if (warp == 1) tc::tmem_alloc<CG>(&tmem, S::kColumns);
    tc::fence_before();
    if (CG == 2) tc::cluster_sync(); else __syncthreads();
    tc::fence_after();
    const uint32_t acc = tmem;
    let_follow();                                           // each warp follows (waits) itself, once it knows its first tile
    const int first = blockIdx.x / CG, stride = gridDim.x / CG;

    if (warp == 0) {                                        // ---- loads
        const uint32_t bar0 = CG == 2 ? tc::smem_of(full, 0) : tc::smem(full), to0 = tc::smem(base);
        int s = 0;
        uint32_t turn = 1;                                  // of the ring: the first goes through without a wait
        bool ok = true;
        for (int t = first; t < p.tiles && ok; t += stride) {
            const Tile at = tile_at<S::kTM, S::kTN, OP>(p, t);
            const MuonGroup& g = p.g[at.g];
            const int blocks = ((OP == kGram ? g.n : g.m) + kBox - 1) / kBox;
            const int row0 = at.i * S::kTM + rank * 128, col0 = at.j * S::kTN + rank * (S::kTN / CG);
            // X X' and A A have one factor twice, B X and (B X)' = X' B two
            const bool x_first = OP == kGram || (OP == kUpdate && g.turned), x_second = OP == kGram || (OP >= kApply && !x_first);
            const CUtensorMap* const map_a = x_first ? &p.x[at.g] : &p.s[at.g];
            const CUtensorMap* const map_b = x_second ? &p.x[at.g] : &p.s[at.g];
            // which matrix of an array: [buffer][terms][count]
            const int in_x = at.mat + g.count * TERMS * p.in, in_s = at.mat + g.count * TERMS * (OP == kPoly ? 0 : 1);
            const int in_a = x_first ? in_x : in_s, in_b = x_second ? in_x : in_s;
            const int limit_a = stored_up_to<S>(row0), limit_b = stored_up_to<S>(col0);
            const int start = first_box<S, OP, TERMS>(at, g.turned, blocks);
            if (t == first) {
                follow();
                tc::fence_for_loads();
            }
            for (int box = 0; box < blocks; ++box) {
                if (!(ok = tc::bar_wait_warp(&empty[s], turn))) break;
                const int k0 = (box + start < blocks ? box + start : box + start - blocks) * kBox;
                // A and B above their stored tiles are read as the transposed ones below, rows along the other dimension
                const bool across_a = across<OP>(x_first, k0 >= limit_a), across_b = across<OP>(x_second, k0 >= limit_b);
                if (tc::elect()) {
                    if (rank == 0) tc::bar_expect(&full[s], CG * S::kStage);
                    const uint32_t bar = bar0 + s * 8;
#pragma unroll
                    for (int h = 0; h < TERMS; ++h) {
                        const uint32_t to = to0 + s * S::kStage + h * S::kHalf;
#pragma unroll
                        for (int b = 0; b < S::kBoxesA; ++b)
                            tc::load_3d<CG>(to + b * kBoxBytes, map_a, bar, across_a ? row0 + b * kBox : k0, across_a ? k0 : row0 + b * kBox, in_a + h * g.count);
#pragma unroll
                        for (int b = 0; b < S::kBoxesB; ++b)
                            tc::load_3d<CG>(to + (S::kBoxesA + b) * kBoxBytes, map_b, bar, across_b ? col0 + b * kBox : k0, across_b ? k0 : col0 + b * kBox, in_b + h * g.count);
                    }
                }
                __syncwarp();
                if (++s == S::kStages) { s = 0; turn ^= 1; }
            }
        }
        if (!ok && lane == 0) { atomicExch(status, 1); bad = 1; }
    } else if (warp == 1) {
        if (rank == 0) {                                    // ---- matrix instructions, of both blocks of a pair
            constexpr uint32_t kAlong = 32 >> 4, kAcross = 2048 >> 4;                   // 16 steps of the sum, by the rows' direction
            const uint64_t a_first = tc::operand(tc::smem(base), kBoxBytes), b_first = tc::operand(tc::smem(base) + S::kBoxesA * kBoxBytes, kBoxBytes);
            int s = 0, sums = 0;                            // stage, sums begun
            uint32_t turn = 0;
            bool ok = true;
            for (int t = first; t < p.tiles && ok; t += stride) {
                const Tile at = tile_at<S::kTM, S::kTN, OP>(p, t);
                const int blocks = ((OP == kGram ? p.g[at.g].n : p.g[at.g].m) + kBox - 1) / kBox;
                const bool x_first = OP == kGram || (OP == kUpdate && p.g[at.g].turned), x_second = OP == kGram || (OP >= kApply && !x_first);
                const int limit_a = stored_up_to<S>(at.i * S::kTM), limit_b = stored_up_to<S>(at.j * S::kTN);
                const int start = first_box<S, OP, TERMS>(at, p.g[at.g].turned, blocks);
                uint32_t to = 0, buf = 0;
                for (int box = 0; box < blocks; ++box) {
                    const bool begin = kSegmented ? box % kSegment == 0 : box == 0;
                    const int k0 = (box + start < blocks ? box + start : box + start - blocks) * kBox;
                    if (begin) {
                        buf = sums & 1;
                        if (!(ok = tc::bar_wait_warp(&acc_empty[buf], ~(sums >> 1) & 1))) break;
                        to = acc + buf * S::kTN;
                        ++sums;
                    }
                    if (!(ok = tc::bar_wait_warp(&full[s], turn))) break;
                    tc::fence_after();
                    const bool across_a = across<OP>(x_first, k0 >= limit_a), across_b = across<OP>(x_second, k0 >= limit_b);
                    const uint32_t instruction = tc::instruction_f16(S::kTM, S::kTN) | (across_a ? tc::kAcrossA : 0u) | (across_b ? tc::kAcrossB : 0u);
                    const uint32_t next_a = across_a ? kAcross : kAlong, next_b = across_b ? kAcross : kAlong;
                    if (tc::elect()) {
                        const uint64_t a0 = a_first + s * (S::kStage >> 4), b0 = b_first + s * (S::kStage >> 4);
                        if (TERMS == 2) {                   // the small products first, for the same reason as first_box's
                            const uint64_t a1 = a0 + (S::kHalf >> 4), b1 = b0 + (S::kHalf >> 4);
#pragma unroll
                            for (int k = 0; k < kBox / 16; ++k) {
                                tc::mma_f16<CG>(to, a0 + next_a * k, b1 + next_b * k, instruction, begin && k == 0 ? 0u : 1u);
                                tc::mma_f16<CG>(to, a1 + next_a * k, b0 + next_b * k, instruction, 1u);
                            }
                        }
#pragma unroll
                        for (int k = 0; k < kBox / 16; ++k) tc::mma_f16<CG>(to, a0 + next_a * k, b0 + next_b * k, instruction, TERMS == 1 && begin && k == 0 ? 0u : 1u);
                        tc::commit<CG>(&empty[s]);
                        if (box + 1 == blocks || (kSegmented && (box + 1) % kSegment == 0)) tc::commit<CG>(&acc_full[buf]);
                    }
                    __syncwarp();
                    if (++s == S::kStages) { s = 0; turn ^= 1; }
                }
            }
            if (!ok && lane == 0) { atomicExch(status, 2); bad = 1; }
        }
    } else {                                                // ---- sums out of tensor memory
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        float (*const st)[33] = (float (*)[33])(base + S::kStages * S::kStage + (warp - 2) * S::kStaged);     // update_narrow's
        constexpr int kChunks = S::kTN / 64;                // of 32 columns, of a warp
        int sums = 0;                                       // read so far
        const auto wait = [&] {
            const bool ok = tc::bar_wait_warp(&acc_full[sums & 1], (sums >> 1) & 1);
            if (!ok && lane == 0) { atomicExch(status, 3); bad = 1; }
            tc::fence_after();
            return ok;
        };
        const auto release = [&] {
            tc::fence_before();
            __syncwarp();
            if (lane == 0) tc::bar_arrive_cluster(tc::smem_of(&acc_empty[sums & 1], 0));
            ++sums;
        };
        const auto column = [&](int ch) { return half * (S::kTN / 2) + ch * 32; };
        const auto read = [&](int ch, float (&v)[32]) { tc::tmem_load32(acc + (sums & 1) * S::kTN + column(ch) + ((uint32_t)(quarter * 32) << 16), v); };
        for (int t = first; t < p.tiles; t += stride) {
            const Tile at = tile_at<S::kTM, S::kTN, OP>(p, t);
            const MuonGroup& g = p.g[at.g];
            float total[kSegmented ? kChunks : 1][32];
            if (kSegmented) {
#pragma unroll
                for (int ch = 0; ch < kChunks; ++ch)
#pragma unroll
                    for (int c = 0; c < 32; ++c) total[ch][c] = 0.f;
                const int segments = (g.n + kBox * kSegment - 1) / (kBox * kSegment);
                bool ok = true;
                for (int q = 0; q < segments && (ok = wait()); ++q) {
#pragma unroll
                    for (int ch = 0; ch < kChunks; ++ch) {
                        float v[32];
                        read(ch, v);
#pragma unroll
                        for (int c = 0; c < 32; ++c) total[ch][c] += v[c];
                    }
                    release();
                }
                if (!ok) break;
            }
            const int row0 = at.i * S::kTM + rank * 128 + quarter * 32;
            const auto kept = [&](int ch) {                 // whether anything of a chunk is
                const int col0 = at.j * S::kTN + column(ch);
                return row0 < result_rows<OP>(g) && col0 < result_cols<OP>(g);
            };
            const MuonMat* const mat = OP == kUpdate ? p.mats + g.mat0 + at.mat : nullptr;
            if (!kSegmented && t == first) follow();
            Ahead<OP, TERMS, T> ahead;
            const auto fetch = [&](int ch) {
                if ((OP == kPoly || OP == kUpdate) && kept(ch)) ahead.load(p, g, at.mat, mat, row0, at.j * S::kTN + column(ch));
            };
            fetch(0);
            if (!kSegmented && !wait()) break;
#pragma unroll
            for (int ch = 0; ch < kChunks; ++ch) {
                const int col0 = at.j * S::kTN + column(ch);
                if (kept(ch)) {
                    float v[32];
                    if (kSegmented) {
#pragma unroll
                        for (int c = 0; c < 32; ++c) v[c] = total[kSegmented ? ch : 0][c];
                    } else {
                        read(ch, v);
                    }
                    const Ahead<OP, TERMS, T> now = ahead;
                    if (ch + 1 < kChunks) fetch(ch + 1);
                    finish_block<OP, TERMS, T>(p, g, at.mat, mat, row0, col0, v, st, now);
                } else if (ch + 1 < kChunks) {
                    fetch(ch + 1);
                }
            }
            if (!kSegmented) release();
        }
    }
    __syncwarp();
    if (bad) {                                              // copies that are still on their way land within microseconds
        const int64_t t0 = clock64();
        while (clock64() - t0 < 4000000) {}
    }
    __syncwarp();
    tc::fence_before();
    if (CG == 2) tc::cluster_sync(); else __syncthreads();
    tc::fence_after();
    if (warp == 1) tc::tmem_free<CG>(acc, S::kColumns);
}

// ---- host ---------------------------------------------------------------------------------------
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
    static const EncodeFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult r;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &r) == cudaSuccess && r == cudaDriverEntryPointSuccess ? (EncodeFn)f : nullptr;
    }();
    return fn;
}
// [2 buffers x terms x count][rows][pitch] fp16, rows of `width` values; boxes of 64 x 64.
bool encode(CUtensorMap* map, void* at, int64_t width, int64_t rows, int64_t pitch, int64_t count, int terms) {
    const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)rows, (cuuint64_t)count * terms * 2};
    const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)rows * pitch * 2};
    const cuuint32_t box[3] = {kBox, kBox, 1}, step[3] = {1, 1, 1};
    return encode_fn()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, at, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A run of launches: matrices of up to eight shapes, and where their arrays lie.
struct MuonRun {
    MuonGroup g[kGroups];
    int groups = 0, count = 0;
    int index[kMats];                  // of the caller's list, by group, then by slot
    int64_t parts = 0, bytes = 0;
};
constexpr int64_t kHead = 256 + ((int64_t)kMats * sizeof(MuonMat) + 255) / 256 * 256;    // status word, table

int64_t parts_of(int64_t rows, int64_t cols) { return (rows * cols + kPart - 1) / kPart; }

// Takes matrices from `at` on that are not empty, as many as a run holds; returns where the next run begins.
int take_run(const int32_t* rows, const int32_t* cols, int n, int at, int terms, MuonRun& r) {
    int group_of[kMats], list[kMats];
    r = MuonRun();
    for (; at < n && r.count < kMats; ++at) {
        if (rows[at] == 0 || cols[at] == 0) continue;
        const int m = rows[at] < cols[at] ? rows[at] : cols[at], w = rows[at] < cols[at] ? cols[at] : rows[at];
        int g = 0;
        const int turned = rows[at] > cols[at];
        while (g < r.groups && (r.g[g].m != m || r.g[g].n != w || r.g[g].turned != turned)) ++g;
        if (g == kGroups) break;
        const int64_t parts = parts_of(rows[at], cols[at]);
        if (r.count > 0 && r.parts + parts > (1 << 24)) break;
        if (g == r.groups) {
            r.g[g] = MuonGroup{};
            r.g[g].m = m;
            r.g[g].n = w;
            r.g[g].turned = turned;
            r.g[g].mp = (m + 15) / 16 * 16;
            r.g[g].np = (w + 15) / 16 * 16;
            ++r.groups;
        }
        group_of[r.count] = g;
        list[r.count++] = at;
        ++r.g[g].count;
        r.parts += parts;
    }
    int64_t bytes = kHead + (8 * r.parts + 255) / 256 * 256;
    int q = 0;
    for (int g = 0; g < r.groups; ++g) {
        MuonGroup& a = r.g[g];
        for (int k = 0; k < r.count; ++k)
            if (group_of[k] == g) r.index[q++] = list[k];
        a.x_plane = (int64_t)a.count * a.m * a.np;
        a.s_plane = (int64_t)a.count * a.m * a.mp;
        a.x = bytes;
        bytes += (a.x_plane * 4 * terms + 255) / 256 * 256;
        a.s = bytes;
        bytes += (a.s_plane * 4 * terms + 255) / 256 * 256;
    }
    r.bytes = bytes;
    return at;
}

template <int CG, int TERMS, int OP, class T = float>
cudaError_t product(MuonGemm& p, cudaStream_t st) {
    using S = Shape<CG, TERMS>;
    constexpr bool kSym = OP == kGram || OP == kPoly;
    int tiles = 0;
    for (int g = 0; g < p.groups; ++g) {
        p.g[g].tile0 = tiles;
        tiles += p.g[g].count * tiles_of<S::kTM, S::kTN, kSym>(result_rows<OP>(p.g[g]), result_cols<OP>(p.g[g]));
    }
    p.tiles = tiles;
    p.back ^= 1;                       // what the product before wrote last is read first, while the L2 cache holds it
    const int slots = CG == 2 ? kPairs : kSms;
    cudaError_t e = cudaFuncSetAttribute(k_muon_product<CG, TERMS, OP, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kShared);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((tiles < slots ? tiles : slots) * CG);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kShared;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CG;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_muon_product<CG, TERMS, OP, T>, (const MuonGemm)p);
}

// Time of a product by tiles of TM x TN on `slots` places, in clocks: whole waves of the mean tile.
template <int CG, bool SYM>
double product_time(const MuonGemm& p, int terms, bool gram) {
    using S = Shape<CG, 1>;
    const double combos = terms == 2 ? 3 : 1, per = CG == 2 ? 512 : 200, set_up = CG == 2 ? 4000 : 2000;
    const int slots = CG == 2 ? kPairs : kSms;
    double all = 0, sum = 0;
    for (int g = 0; g < p.groups; ++g) {
        const double t = (double)p.g[g].count * tiles_of<S::kTM, S::kTN, SYM>(p.g[g].m, p.g[g].n);
        all += t;
        sum += t * (((gram ? p.g[g].n : p.g[g].m) + kBox - 1) / kBox * per * combos + set_up);
    }
    return std::ceil(all / slots) * (sum / all);
}
template <int CG, int TERMS, int OP>
cudaError_t product_type(MuonGemm& p, int type, cudaStream_t st) {
    if (OP != kUpdate || type == RFAST_TYPE_F32) return product<CG, TERMS, OP, float>(p, st);
    if constexpr (OP == kUpdate) return type == RFAST_TYPE_BF16 ? product<CG, TERMS, OP, __nv_bfloat16>(p, st) : product<CG, TERMS, OP, __half>(p, st);
    return cudaErrorInvalidValue;
}
template <int CG, int OP>
cudaError_t product_terms(MuonGemm& p, int terms, int type, cudaStream_t st) { return terms == 2 ? product_type<CG, 2, OP>(p, type, st) : product_type<CG, 1, OP>(p, type, st); }
template <int OP>
cudaError_t product_of(MuonGemm& p, int terms, bool pairs, int type, cudaStream_t st) { return pairs ? product_terms<2, OP>(p, terms, type, st) : product_terms<1, OP>(p, terms, type, st); }
template <int CG>
double iteration_time(const MuonGemm& p, int terms) {
    return product_time<CG, true>(p, terms, true) + product_time<CG, true>(p, terms, false) + product_time<CG, false>(p, terms, false);
}

int muon_terms(const rfast_muon* a) { return a->terms ? a->terms : a->param_type == RFAST_TYPE_BF16 ? 1 : 2; }

const char* muon_shape_fault(int n, const int32_t* rows, const int32_t* cols) {
    if (n < 0) return "n_tensors is negative";
    if (n > 0 && (!rows || !cols)) return "null array";
    for (int k = 0; k < n; ++k)
        if (rows[k] < 0 || cols[k] < 0 || rows[k] > RFAST_MUON_MAX_SIDE || cols[k] > RFAST_MUON_MAX_SIDE) return "rows and cols must be in [0, 65536]";
    return nullptr;
}

cudaError_t muon_run(const rfast_muon* a, const MuonRun& r, char* work, bool first_run, cudaStream_t st) {
    MuonTable t;
    MuonGemm q{};
    const int terms = muon_terms(a);
    int part = 0, tile = 0;
    t.count = r.count;
    int at = 0;
    for (int g = 0; g < r.groups; ++g)
        for (int s = 0; s < r.g[g].count; ++s, ++at) {
            const int k = r.index[at];
            MuonMat& m = t.mat[at];
            m.param = a->param[k];
            m.grad = a->grad[k];
            m.momentum = a->momentum[k];
            m.rows = a->rows[k];
            m.cols = a->cols[k];
            m.group = g;
            m.slot = s;
            const double size = a->size_rule == RFAST_MUON_SIZE_RMS ? 0.2 * std::sqrt((double)r.g[g].n)
                                                                    : std::sqrt(m.rows > m.cols ? (double)m.rows / m.cols : 1.0);
            m.step = (float)(a->lr * size);
            m.wide = m.cols * (int64_t)bytes_of(a->param_type) % 32 == 0 && (uintptr_t)m.param % 32 == 0;
            t.part0[at] = part;
            t.tile0[at] = tile;
            part += (int)parts_of(m.rows, m.cols);
            tile += (m.rows + 63) / 64 * ((m.cols + 63) / 64);
        }
    t.part0[at] = part;
    t.tile0[at] = tile;
    int first = 0;
    for (int g = 0; g < r.groups; ++g) {
        q.g[g] = r.g[g];
        q.g[g].mat0 = first;
        if (!encode(&q.x[g], work + r.g[g].x, r.g[g].n, r.g[g].m, r.g[g].np, r.g[g].count, terms)) return cudaErrorInvalidValue;
        if (!encode(&q.s[g], work + r.g[g].s, r.g[g].m, r.g[g].m, r.g[g].mp, r.g[g].count, terms)) return cudaErrorInvalidValue;
        first += r.g[g].count;
    }
    q.groups = r.groups;
    q.keep = (float)(1.0 - a->lr * a->weight_decay);
    q.work = work;
    MuonMat* mats = (MuonMat*)(work + 256);
    q.mats = mats;
    double* parts = (double*)(work + kHead);
    const MuonScalars c{(float)a->momentum_beta, (float)(1.0 - a->momentum_beta), a->nesterov != 0, a->grad_type, terms, a->eps, a->d_grad_scale};
    cudaError_t e = launch(k_muon_momentum, dim3((unsigned)part), 256, 0, st, false, t, c, parts, mats, first_run ? (int*)work : (int*)nullptr);
    if (e == cudaSuccess) e = launch(k_muon_begin, dim3((unsigned)tile), 256, 0, st, true, t, c, (const double*)parts, q);
    const bool pairs = iteration_time<2>(q, terms) <= iteration_time<1>(q, terms);
    for (int it = 0; it < a->iterations && e == cudaSuccess; ++it) {
        q.in = it & 1;
        e = product_of<kGram>(q, terms, pairs, a->param_type, st);
        if (e == cudaSuccess) e = product_of<kPoly>(q, terms, pairs, a->param_type, st);
        if (e == cudaSuccess) e = it + 1 < a->iterations ? product_of<kApply>(q, terms, pairs, a->param_type, st) : product_of<kUpdate>(q, terms, pairs, a->param_type, st);
    }
    return e;
}

}  // namespace

}  // namespace rfast

using namespace rfast;

extern "C" int64_t rfast_muon_workspace(int32_t n_tensors, const int32_t* rows, const int32_t* cols, int32_t terms) {
    if (muon_shape_fault(n_tensors, rows, cols) || (terms != 1 && terms != 2)) return RFAST_EINVAL;
    int64_t most = kHead;
    MuonRun r;
    for (int at = 0; at < n_tensors;) {
        at = take_run(rows, cols, n_tensors, at, terms, r);
        if (r.bytes > most) most = r.bytes;
    }
    return most;
}

extern "C" int rfast_muon_step(const rfast_muon* a, void* workspace, size_t workspace_bytes, void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_muon_step";
    if (!a) return op_fail(err, err_len, RFAST_EINVAL, "%s: null arguments", me);
    if (const char* fault = muon_shape_fault(a->n_tensors, a->rows, a->cols)) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s", me, fault);
    if (!is_type(a->param_type) || !is_type(a->grad_type)) return op_fail(err, err_len, RFAST_EINVAL, "%s: unknown type", me);
    if (a->terms < 0 || a->terms > 2) return op_fail(err, err_len, RFAST_EINVAL, "%s: terms must be 0, 1 or 2", me);
    // negated comparisons refuse a NaN as well
    if (!(a->momentum_beta >= 0 && a->momentum_beta < 1)) return op_fail(err, err_len, RFAST_EINVAL, "%s: momentum must be in [0, 1)", me);
    if (!(a->eps > 0) || !std::isfinite(a->eps)) return op_fail(err, err_len, RFAST_EINVAL, "%s: eps must be positive and finite", me);
    if (!std::isfinite(a->lr) || !std::isfinite(a->weight_decay)) return op_fail(err, err_len, RFAST_EINVAL, "%s: lr and weight_decay must be finite", me);
    if (a->iterations < 1 || a->iterations > 32) return op_fail(err, err_len, RFAST_EINVAL, "%s: iterations must be in [1, 32]", me);
    if (a->size_rule != RFAST_MUON_SIZE_SPECTRAL && a->size_rule != RFAST_MUON_SIZE_RMS) return op_fail(err, err_len, RFAST_EINVAL, "%s: unknown size_rule", me);
    if ((uintptr_t)a->d_grad_scale % 4) return op_fail(err, err_len, RFAST_EINVAL, "%s: d_grad_scale is not aligned to its type", me);
    if (a->n_tensors == 0) return RFAST_OK;
    if (!a->param || !a->grad || !a->momentum) return op_fail(err, err_len, RFAST_EINVAL, "%s: null array", me);
    int some = -1;
    for (int k = 0; k < a->n_tensors; ++k) {
        if (a->rows[k] == 0 || a->cols[k] == 0) continue;
        if (!a->param[k] || !a->grad[k] || !a->momentum[k]) return op_fail(err, err_len, RFAST_EINVAL, "%s: tensor %d has a null address", me, k);
        if ((uintptr_t)a->param[k] % bytes_of(a->param_type) || (uintptr_t)a->grad[k] % bytes_of(a->grad_type) || (uintptr_t)a->momentum[k] % 4)
            return op_fail(err, err_len, RFAST_EINVAL, "%s: an address of tensor %d is not aligned to its type", me, k);
        if (some < 0) some = k;
    }
    if (some < 0) return RFAST_OK;
    const int64_t need = rfast_muon_workspace(a->n_tensors, a->rows, a->cols, muon_terms(a));
    if (!workspace || (uintptr_t)workspace % 256) return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace must be given, aligned to 256 bytes", me);
    if (workspace_bytes < (size_t)need) return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace needs %lld bytes", me, (long long)need);
    const void* first[] = {a->param[some], a->grad[some], a->momentum[some], a->d_grad_scale, workspace};
    const char* names[] = {"rfast_muon_step: param", "rfast_muon_step: grad", "rfast_muon_step: momentum", "rfast_muon_step: d_grad_scale", "rfast_muon_step: workspace"};
    for (int k = 0; k < 5; ++k)
        if (first[k]) {
            const int rc = check_device_pointer(first[k], names[k], err, err_len);
            if (rc != RFAST_OK) return rc;
        }
    if (!encode_fn()) return op_fail(err, err_len, RFAST_ECUDA, "%s: the driver has no cuTensorMapEncodeTiled", me);
    // a thread whose first call this is has no context yet, which the encoding of tensor maps wants
    int dev = 0;
    cudaError_t bound = cudaGetDevice(&dev);
    if (bound == cudaSuccess) bound = cudaSetDevice(dev);
    if (bound != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: %s", me, cudaGetErrorString(bound));
    MuonRun r;
    bool first_run = true;
    for (int at = 0; at < a->n_tensors;) {
        at = take_run(a->rows, a->cols, a->n_tensors, at, muon_terms(a), r);
        if (r.count == 0) continue;
        const cudaError_t e = muon_run(a, r, (char*)workspace, first_run, (cudaStream_t)cuda_stream);
        first_run = false;
        if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: %s", me, cudaGetErrorString(e));
    }
    return RFAST_OK;
}
