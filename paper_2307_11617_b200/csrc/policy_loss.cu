// Clipped policy loss with a KL term, out of logits, and its gradient (see rfast_policy_loss in rfast.h for the formulas).
//
// What bounds it is memory, where a logit has to come in once and its gradient to leave once.  The first pass over a row holds a running
// maximum and sum of each thread's values, which are merged in a fixed order; one warp forms the row's numbers in 64 bits; the
// second pass writes the gradient out of the logits again.  A warp does a row of up to 1024 logits, a block of 128 threads one of up to
// 40 KB (in the L2 cache between the passes), a block of 256 one of up to 128 KB, a block of 512 longer ones; a cluster of up to eight
// blocks where rows are few.  A thread of the latter two keeps the first logits that it reads in shared memory, 48 or 96 KB a block; the rest
// it reads again, the last first.  Without that the rows under way, 296 of 256 KB, are too much for the L2 cache: 4096 x 128256 bf16 read
// 1.72 GB instead of 0.93, 445 us; with it 1.03 GB, 414 us, 4.7 TB/s and half of the issue slots and of the special function unit.
// (Bringing rows through a ring in shared memory by bulk copies, a cluster to a row and the next row's sum before this one's
// gradient, read every logit once and took 510 us: with 20 instructions a logit in the place of then 13 the issue slots were the bound.)
//
// Powers are taken of two: exp((z - m) / T) = 2^(z k - c) with k = log2(e) / T and c near m k (see Run).  k in fp32 would be another T, by up to 2^-24 of
// itself, which moves all token losses of a call one way; the sums take it in two parts, one multiply-add more (2047 x 50257 f16 94.2 -> 94.5 us, 4096 x
// 128256 bf16 without a gradient 197.5 -> 201), the row's numbers in 64 bits.  The gradient's powers have it in fp32: it matters to their distance
// from c only, c's own share is made up for in p.
#include <cuda_runtime.h>

#include <climits>
#include <cmath>
#include <cstdio>

#include "ops.h"
#include "tensor_core.cuh"
#include "values.cuh"

namespace rfast {

namespace {

constexpr int kBlockTeam = 512, kHalfTeam = 256, kMidTeam = 128;
constexpr int kPlaces = 240;                 // blocks of 512 threads that run at once, less what clusters cannot use
constexpr int kAhead = 4;                    // groups of eight logits that a thread has on their way (four more, fetched while it works: no gain)
constexpr int64_t kShortRow = 1024;          // logits of a row up to which a warp does it
constexpr int kKept = 96 * 1024;             // bytes of a row that a long row's block keeps; two blocks share an SM
// Bytes read again above which pairs of blocks do a row (one block, pairs; us): 4096 rows bf16 at 47 MB 418, 456; 53 MB 466, 496; 61 MB 522, 528; 68 MB 564,
// 545; 77 MB 634, 597.  2000 rows f32 at 48 MB 225, 227; 54 MB 247, 245; 60 MB 270, 256; 90 MB 366, 339.
constexpr int64_t kReadAgain = 56ll << 20;
constexpr int64_t kHalfRow = 128 * 1024, kQuarterRow = 40 * 1024;     // bytes of a row up to which it is a block of half, of a quarter of the threads

struct Policy {
    const void* logits;
    const void* tokens;
    const float *old_logp, *ref_logp, *advantage, *weight, *scale;
    float *token_loss, *logp;
    void* dlogits;
    int64_t rows, vocab, in_stride, out_stride;
    int wide_tokens;
    double exact_k;                    // log2(e) / T
    float k, high, low;                // rounded; its first 12 bits (or the number below), so that the rest is above 0 and takes -infinity as it should
    float beyond;                      // exact_k / k - 1
    float inv_t;
    double clip_lo, clip_hi, kl;       // 1 - clip_low, 1 + clip_high
};

__device__ __forceinline__ float two_to(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Sum of 2^(z k - c) over what a thread has seen.  The reference c is the rounded product of k and an earlier maximum (never one exact in a
// multiply-add): it follows the maximum only where that is 2^kSlack ahead, so that sums are seldom rescaled, and terms below
// 2^-126 at the reference are 2^-126 of the largest term and less.  No logit but -infinity and NaN so far: c is -infinity.
// Beyond kNear the rounding of c would be an exponent of its own, up to 2^-24 |c|, without bound (masks of -1e10 or of the type's lowest value, rows
// that share such an offset).  Nothing is subtracted there: far below zero all powers are 0, which is what they are next to any reference that is near,
// and a row that has no such reference is done again by far_row.
struct Run {
    float c, sum;
};
constexpr float kSlack = 40.f;
constexpr float kNear = 1048576.f;           // c's rounding is up to 2^-4
__device__ __forceinline__ bool is_near(float c) { return fabsf(c) < kNear; }
// what is subtracted: 0 where there is no reference yet, or a far one (-infinity less 0 is -infinity)
__device__ __forceinline__ float base_of(float c) { return is_near(c) ? c : 0.f; }
// the factor that takes a sum to the reference `to`; a run without one keeps its sum, 0 or NaN
__device__ __forceinline__ float rescale(float c, float to) { return c == -INFINITY ? 1.f : two_to(c - to); }
// Merged over a warp: the largest reference first, so that each sum is taken to it once.
__device__ __forceinline__ Run merged_warp(Run r) {
    float c = r.c;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) c = fmaxf(c, __shfl_xor_sync(0xffffffffu, c, o));
    float sum = r.sum * rescale(r.c, base_of(c));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return {c, sum};
}
__device__ __forceinline__ void follow_top(Run& r, float top, float k) {
    const float to = __fmul_rn(top, k);
    if (to > r.c + kSlack) {
        r.sum *= rescale(r.c, to);
        r.c = to;
    }
}
template <int N>
__device__ __forceinline__ void take(Run& r, const float (&v)[N], const Policy& a) {
    float top = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, v[i]);
    follow_top(r, top, a.k);
    const float c = base_of(r.c);
#pragma unroll
    for (int i = 0; i < N; ++i) r.sum += two_to(fmaf(v[i], a.low, fmaf(v[i], a.high, -c)));
}

// What the second pass needs of a row: the gradient is p * 2^(z k - base), at the token plus `slope`.
struct RowOut {
    float base, p, slope;
};

// A warp: the row's loss and slope, in 64 bits, from the merged run, the token's logit and what belongs to the row (lane 0's).  Lanes
// 0 and 1 take the two exponentials side by side.
struct RowIn {
    float zt, adv, w, old, ref, scale;
};
template <class T>
__device__ __forceinline__ RowIn row_in(const Policy& a, int64_t row, const T* z, int64_t t) {
    return {value_of(z[t]), a.advantage ? a.advantage[row] : 0.f, a.weight ? a.weight[row] : 1.f, a.old_logp ? a.old_logp[row] : 0.f,
            a.ref_logp ? a.ref_logp[row] : 0.f, a.scale ? *a.scale : 1.f};
}
__device__ __forceinline__ RowOut row_numbers(const Policy& a, int64_t row, float from, float c, float sum, const RowIn& in, bool keep) {
    const int lane = threadIdx.x & 31;
    const float zt = __shfl_sync(0xffffffffu, in.zt, 0), ref = __shfl_sync(0xffffffffu, in.ref, 0), old = __shfl_sync(0xffffffffu, in.old, 0);
    const double up_to = 0.6931471805599453 * (((double)zt - (double)from) * a.exact_k - (double)c - log2((double)sum));
    const double logp = up_to > 0.0 ? 0.0 : up_to;          // a word that has all of the probability, and a sum that is off; NaN stays
    const double d = (double)ref - logp;
    const double e = lane < 2 ? expm1(lane ? d : logp - (double)old) : 0.0;
    const double e1 = __shfl_sync(0xffffffffu, e, 1);
    RowOut o{};
    if (lane == 0) {
        const double ratio = e + 1.0, adv = in.adv, w = in.w;
        const double held = ratio < a.clip_lo ? a.clip_lo : ratio > a.clip_hi ? a.clip_hi : ratio;
        const double one = ratio * adv, two = held * adv;
        const bool pass = !(one > two);                     // a NaN passes
        double loss = pass ? -one : -two, slope = pass ? -one : 0.0;
        if (a.ref_logp) {
            loss += a.kl * (e1 - d);
            slope -= a.kl * e1;
        }
        if (keep && a.token_loss) a.token_loss[row] = (float)(w * loss);
        if (keep && a.logp) a.logp[row] = (float)logp;
        slope *= w * (double)in.scale * (double)a.inv_t;
        o.base = c;
        o.slope = (float)slope;
        o.p = -o.slope / sum * two_to(c * a.beyond);        // in 32 bits: off by 2^-22, as much as a power is
    }
    return o;
}

// A row cut at multiples of eight values' size: `head` values, then groups of eight, then the rest.  ALIGN: logits and gradients
// begin at the same place within a group, so that the groups are whole in both.
template <class T> __device__ __forceinline__ int head_of(const T* p, int64_t n) {
    constexpr uintptr_t kGroup = 8 * sizeof(T);
    const int h = (int)(((kGroup - ((uintptr_t)p & (kGroup - 1))) & (kGroup - 1)) / sizeof(T));
    return h < n ? h : (int)n;
}

__device__ __forceinline__ uint32_t cluster_blocks() {
    uint32_t n;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
    return n;
}

// A row whose logits are all far from zero (or -infinity, or one of which is +infinity): its maximum m, sum and gradient by 2^((z - m) k), where the
// difference of neighbours is exact.  One value at a time: such rows are rare.  It finds out anew where it is, so that nothing is kept for it.
template <class T, int TEAM>
__device__ __noinline__ void far_row(const Policy& a, int64_t row, Run* sh_run, Run* sh_all, RowOut* sh_out) {
    const int tid = threadIdx.x % TEAM, blocks = TEAM == 32 ? 1 : cluster_blocks(), rank = TEAM == 32 ? 0 : tc::cluster_rank();
    if (TEAM > 32) row = blockIdx.x / blocks;
    const T* z = (const T*)a.logits + row * a.in_stride;
    T* dz = a.dlogits ? (T*)a.dlogits + row * a.out_stride : nullptr;
    const int64_t t = a.wide_tokens ? ((const int64_t*)a.tokens)[row] : (int64_t)((const int*)a.tokens)[row];
    const int64_t per = (a.vocab + blocks - 1) / blocks, lo = per * rank < a.vocab ? per * rank : a.vocab, hi = lo + per < a.vocab ? lo + per : a.vocab;     // this block's
    RowIn in{};
    if (tid == 0) in = row_in(a, row, z, t);
    const float k = a.k;
    float m = -INFINITY, sum = 0.f;
    for (int pass = 0; pass < 2; ++pass) {                  // the maximum (in c), then the sum
        const float from = m == -INFINITY ? 0.f : m;
        if (pass) {
            for (int64_t i = lo + tid; i < hi; i += TEAM) sum += two_to((value_of(z[i]) - from) * k);
        } else {
            for (int64_t i = lo + tid; i < hi; i += TEAM) m = fmaxf(m, value_of(z[i]));
        }
        const auto merged = [&](Run r) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                r.c = fmaxf(r.c, __shfl_xor_sync(0xffffffffu, r.c, o));
                r.sum += __shfl_xor_sync(0xffffffffu, r.sum, o);
            }
            return r;
        };
        Run r = merged({m, sum});
        if (TEAM > 32) {
            __syncthreads();                                // what is in shared memory has been read
            if ((tid & 31) == 0) sh_run[tid >> 5] = r;
            __syncthreads();
            r = merged((tid & 31) < TEAM / 32 ? sh_run[tid & 31] : Run{-INFINITY, 0.f});
            if (blocks > 1) {
                tc::cluster_sync();
                if (tid < blocks) {
                    const uint32_t at = tc::smem_of(&sh_all[rank], tid);
                    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(r.c), "f"(r.sum) : "memory");
                }
                __syncwarp();
                tc::cluster_sync();
                r = merged((tid & 31) < blocks ? sh_all[tid & 31] : Run{-INFINITY, 0.f});
            }
        }
        m = r.c;
        sum = r.sum;
    }
    const float from = m == -INFINITY ? 0.f : m;
    RowOut out;
    if (TEAM == 32 || tid < 32) out = row_numbers(a, row, from, 0.f, sum, in, rank == 0);
    if (TEAM == 32) {
        out.p = __shfl_sync(0xffffffffu, out.p, 0);
        out.slope = __shfl_sync(0xffffffffu, out.slope, 0);
    } else {
        if (tid == 0) *sh_out = out;
        __syncthreads();
        out = *sh_out;
    }
    if (!dz) return;
    for (int64_t i = lo + tid; i < hi; i += TEAM) {
        const float p = out.p * two_to((value_of(z[i]) - from) * k);
        dz[i] = rounded<T>(i == t ? out.slope + p : p);
    }
}

// KEEP: iterations of the block's threads over a row whose logits stay in shared memory, a thread's own.  A cluster's blocks share the
// groups out; the first has what lies before and behind them.
// True: a row that far_row has to do.
template <class T, int TEAM, bool ALIGN, int KEEP>
__device__ __forceinline__ bool policy_row(const Policy& a, int64_t row, int tid, int rank, int blocks, Run* sh_run, Run* sh_all, RowOut* sh_out, Raw8<T>* kept) {
    const T* z = (const T*)a.logits + row * a.in_stride;
    T* dz = a.dlogits ? (T*)a.dlogits + row * a.out_stride : nullptr;
    const int64_t t = a.wide_tokens ? ((const int64_t*)a.tokens)[row] : (int64_t)((const int*)a.tokens)[row];
    const int64_t n = a.vocab;
    const bool live = t >= 0 && t < n && !(a.weight && a.weight[row] == 0.f);
    const float k = a.k;
    const int head = head_of(live ? z : dz, n);
    const int all = (int)((n - head) / 8), per = (all + blocks - 1) / blocks;
    const int g0 = per * rank < all ? per * rank : all, groups = (all - g0 < per ? all - g0 : per);      // this block's
    const int64_t rest0 = head + (int64_t)all * 8;
    // one value before or behind the groups, fewer than eight each
    const int64_t edge = rank ? -1 : tid < head ? tid : tid >= 16 && tid < 32 && rest0 + tid - 16 < n ? rest0 + tid - 16 : -1;
    if (!live) {
        if (tid == 0 && rank == 0) {
            if (a.token_loss) a.token_loss[row] = 0.f;
            if (a.logp) a.logp[row] = 0.f;
        }
        if (dz) {
            const float zero[8] = {};
            T* d = dz + head + (int64_t)g0 * 8;
            for (int g = tid; g < groups; g += TEAM) store8(d + (int64_t)g * 8, zero);
            if (edge >= 0) dz[edge] = rounded<T>(0.f);
        }
        return false;
    }
    RowIn in{};
    if (tid == 0) in = row_in(a, row, z, t);
    Run r{-INFINITY, 0.f};
    const T* zg = z + head + (int64_t)g0 * 8;
    const int its = (groups - tid + TEAM - 1) / TEAM;       // groups of this thread: tid + it TEAM
    for (int it = 0; it < its; it += kAhead) {
        Raw8<T> q[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (it + u < its) q[u] = load8(zg + (int64_t)(tid + (it + u) * TEAM) * 8);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (it + u < its) {
                if (KEEP > 0 && it + u < KEEP) kept[(it + u) * TEAM + tid] = q[u];
                float v[8];
                unpack8(q[u], v);
                take(r, v, a);
            }
    }
    if (edge >= 0) { const float v[1] = {value_of(z[edge])}; take(r, v, a); }
    r = merged_warp(r);
    RowOut out;
    if (TEAM == 32) {
        out = row_numbers(a, row, 0.f, r.c, r.sum, in, true);
        out.base = __shfl_sync(0xffffffffu, out.base, 0);
        out.p = __shfl_sync(0xffffffffu, out.p, 0);
        out.slope = __shfl_sync(0xffffffffu, out.slope, 0);
    } else {
        if ((tid & 31) == 0) sh_run[tid >> 5] = r;
        __syncthreads();
        if (tid < 32) r = merged_warp(tid < TEAM / 32 ? sh_run[tid] : Run{-INFINITY, 0.f});
        if (blocks > 1) {                                   // every block sends its sum to all, and merges them in the same order
            if (tid < blocks) {
                const uint32_t at = tc::smem_of(&sh_all[rank], tid);
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(r.c), "f"(r.sum) : "memory");
            }
            __syncwarp();
            tc::cluster_sync();
            if (tid < 32) r = merged_warp(tid < blocks ? sh_all[tid] : Run{-INFINITY, 0.f});
        }
        if (tid < 32) {
            const RowOut o = row_numbers(a, row, 0.f, r.c, r.sum, in, rank == 0);
            if (tid == 0) *sh_out = o;
        }
        __syncthreads();
        out = *sh_out;
    }
    if (!is_near(out.base)) return true;                    // far_row forms the row's numbers again
    if (!dz) return false;
    const auto slope_of = [&](float v, int64_t i) {
        const float p = out.p * two_to(fmaf(v, k, -out.base));
        return i == t ? out.slope + p : p;
    };
    if (ALIGN) {
        T* dg = dz + head + (int64_t)g0 * 8;
        // of the token, counted from this block's first group; beyond any where it is none of its
        const int64_t from = t - head - (int64_t)g0 * 8;
        const int token_at = from >= 0 && from < (int64_t)groups * 8 ? (int)from : INT_MAX;
        const auto put = [&](int g, const Raw8<T>& q) {
            float v[8];
            unpack8(q, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = out.p * two_to(fmaf(v[j], k, -out.base));
            const unsigned at = (unsigned)(token_at - g * 8);
            if (at < 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += at == j ? out.slope : 0.f;
            }
            store8(dg + (int64_t)g * 8, v);
        };
        for (int it = its - 1; it >= KEEP; it -= kAhead) {  // those from KEEP on are read again, the last first
            Raw8<T> q[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (it - u >= KEEP) q[u] = load8(zg + (int64_t)(tid + (it - u) * TEAM) * 8);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (it - u >= KEEP) put(tid + (it - u) * TEAM, q[u]);
        }
        if (KEEP > 0) {
            const int last = its < KEEP ? its : KEEP;
#pragma unroll 4
            for (int it = 0; it < last; ++it) put(tid + it * TEAM, kept[it * TEAM + tid]);
        }
        if (edge >= 0) dz[edge] = rounded<T>(slope_of(value_of(z[edge]), edge));
    } else {
        for (int64_t i = tid; i < n; i += TEAM) dz[i] = rounded<T>(slope_of(value_of(z[i]), i));
    }
    return false;
}

template <class T, bool ALIGN>
__global__ void __launch_bounds__(256)
k_policy_warp(const __grid_constant__ Policy a) {
    let_follow();
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < a.rows; row += (int64_t)gridDim.x * 8)
        if (policy_row<T, 32, ALIGN, 0>(a, row, threadIdx.x & 31, 0, 1, nullptr, nullptr, nullptr, nullptr)) far_row<T, 32>(a, row, nullptr, nullptr, nullptr);
}

// Nine blocks of 128 threads to an SM, for which far_row has to spill registers (8192 x 9000 bf16: 67 us, 70 with eight, 66 without far_row).
template <class T, int TEAM, bool ALIGN, int KEEP>
__global__ void __launch_bounds__(TEAM, TEAM == kMidTeam && sizeof(T) == 2 ? 9 : 1024 / TEAM)
k_policy_block(const __grid_constant__ Policy a) {
    extern __shared__ __align__(32) uint8_t kept[];
    __shared__ Run sh_run[TEAM / 32], sh_all[8];
    __shared__ RowOut sh_out;
    let_follow();
    uint32_t blocks = 1, rank = 0;
    if (KEEP > 0) {
        blocks = cluster_blocks();
        rank = tc::cluster_rank();
        if (blocks > 1) tc::cluster_sync();                 // all have begun: their shared memory is there
    }
    if (policy_row<T, TEAM, ALIGN, KEEP>(a, blockIdx.x / blocks, threadIdx.x, rank, blocks, sh_run, sh_all, &sh_out, (Raw8<T>*)kept))
        far_row<T, TEAM>(a, 0, sh_run, sh_all, &sh_out);
}

// The sum of the tokens' losses, in 64 bits and a fixed order.  They are still being written when this kernel is set up: no __restrict__, which would
// say that nobody writes them while it runs.
__global__ void __launch_bounds__(1024)
k_policy_total(const float* token_loss, int64_t rows, float* loss) {
    __shared__ double sh[32];
    follow();
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) s += (double)token_loss[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int w = 0; w < 32; ++w) all += sh[w];
        *loss = (float)all;
    }
}

template <class T, int TEAM>
cudaError_t keeping_launch(const Policy& a, cudaStream_t st) {
    constexpr int kBytes = kKept / kBlockTeam * TEAM, kKeep = kBytes / (TEAM * 8 * (int)sizeof(T));
    // few rows: blocks share one out while all fit the GPU at once and each has two iterations of its threads left
    int c = 1;
    while (c < 8 && a.rows * c * 2 <= kPlaces * (kBlockTeam / TEAM) && a.vocab / (c * 2) >= 2 * TEAM * 8) c *= 2;
    // long rows: as many blocks to a row as leave what is read again of the rows under way to the L2 cache
    const int64_t row = a.vocab * (int64_t)sizeof(T);
    // (and a grid holds: repeated rows, their stride 0, can be 2^31 - 1)
    while (c < 8 && a.rows * c * 2 <= INT_MAX && 296 / c * (kBlockTeam / TEAM) * (row - (int64_t)c * kBytes) > kReadAgain) c *= 2;
    const auto kernel = k_policy_block<T, TEAM, true, kKeep>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(a.rows * c));
    cfg.blockDim = dim3(TEAM);
    cfg.dynamicSmemBytes = kBytes;
    cfg.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = c;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = c > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, (const Policy)a);
}
template <class T, bool ALIGN>
cudaError_t policy_launch(const Policy& a, cudaStream_t st) {
    if (a.vocab <= kShortRow) {
        const int64_t blocks = (a.rows + 7) / 8;
        return launch(k_policy_warp<T, ALIGN>, dim3((unsigned)(blocks < 0x7fffffff ? blocks : 0x7fffffff)), 256, 0, st, false, a);
    }
    if constexpr (ALIGN) {
        const int64_t row = a.vocab * (int64_t)sizeof(T);
        if (row > kQuarterRow) return row <= kHalfRow ? keeping_launch<T, kHalfTeam>(a, st) : keeping_launch<T, kBlockTeam>(a, st);
    }
    if (a.vocab * (int64_t)sizeof(T) <= kQuarterRow) return launch(k_policy_block<T, kMidTeam, ALIGN, 0>, dim3((unsigned)a.rows), kMidTeam, 0, st, false, a);
    return launch(k_policy_block<T, kBlockTeam, false, 0>, dim3((unsigned)a.rows), kBlockTeam, 0, st, false, a);
}
template <class T>
cudaError_t policy_types(const Policy& a, bool align, cudaStream_t st) {
    return align ? policy_launch<T, true>(a, st) : policy_launch<T, false>(a, st);
}

}  // namespace

}  // namespace rfast

using namespace rfast;

extern "C" int rfast_policy_loss(const rfast_policy* p, void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_policy_loss";
    if (!p) return op_fail(err, err_len, RFAST_EINVAL, "%s: null arguments", me);
    if (p->tokens < 0 || p->tokens > 0x7fffffff) return op_fail(err, err_len, RFAST_EINVAL, "%s: tokens must be in [0, 2^31)", me);
    if (p->vocab < 1 || p->vocab > 0x7fffffff) return op_fail(err, err_len, RFAST_EINVAL, "%s: vocab must be in [1, 2^31)", me);
    if (!is_type(p->type)) return op_fail(err, err_len, RFAST_EINVAL, "%s: unknown type", me);
    if (p->token_bits != 32 && p->token_bits != 64) return op_fail(err, err_len, RFAST_EINVAL, "%s: token_bits must be 32 or 64", me);
    // negated comparisons refuse a NaN as well
    if (!(p->temperature >= 1e-3) || !(p->temperature <= 1e3)) return op_fail(err, err_len, RFAST_EINVAL, "%s: temperature must be in [0.001, 1000]", me);
    if (!(p->clip_low >= 0) || !(p->clip_low <= 1) || !(p->clip_high >= 0)) return op_fail(err, err_len, RFAST_EINVAL, "%s: clip_low must be in [0, 1], clip_high at least 0", me);
    if (p->d_ref_logp && !std::isfinite(p->kl_coef)) return op_fail(err, err_len, RFAST_EINVAL, "%s: kl_coef must be finite", me);
    if (p->d_loss && !p->d_token_loss) return op_fail(err, err_len, RFAST_EINVAL, "%s: d_loss is summed from d_token_loss, which is null", me);
    if (!p->d_token_loss && !p->d_logp && !p->d_dlogits) return op_fail(err, err_len, RFAST_EINVAL, "%s: no result is wanted", me);
    if (p->tokens > 0) {
        const size_t b = bytes_of(p->type);
        if (!p->d_logits || (uintptr_t)p->d_logits % b) return op_fail(err, err_len, RFAST_EINVAL, "%s: logits are null or not aligned to their type", me);
        if ((uintptr_t)p->d_dlogits % b) return op_fail(err, err_len, RFAST_EINVAL, "%s: dlogits are not aligned to their type", me);
        if (!p->d_tokens || (uintptr_t)p->d_tokens % (p->token_bits / 8)) return op_fail(err, err_len, RFAST_EINVAL, "%s: tokens are null or not aligned to their type", me);
        // log probabilities by themselves, from which old_logp and ref_logp come, have no use for either
        if ((p->d_token_loss || p->d_dlogits) && (!p->d_old_logp || !p->d_advantage))
            return op_fail(err, err_len, RFAST_EINVAL, "%s: old_logp or advantage is null", me);
        const int64_t most = ((int64_t)1 << 56) / p->tokens;
        if (p->logits_stride < 0 || p->logits_stride > most) return op_fail(err, err_len, RFAST_EINVAL, "%s: the stride of logits is negative or spans more than 2^56 elements", me);
        if (p->d_dlogits && ((p->tokens > 1 && p->dlogits_stride < p->vocab) || p->dlogits_stride < 0 || p->dlogits_stride > most))
            return op_fail(err, err_len, RFAST_EINVAL, "%s: the stride of dlogits lets rows overlap or spans more than 2^56 elements", me);
        if (p->d_dlogits == p->d_logits && p->dlogits_stride != p->logits_stride && p->tokens > 1)
            return op_fail(err, err_len, RFAST_EINVAL, "%s: gradients in the place of the logits want their stride", me);
    }
    const void* floats[] = {p->d_old_logp, p->d_ref_logp, p->d_advantage, p->d_weight, p->d_loss_scale, p->d_token_loss, p->d_logp, p->d_loss};
    for (const void* f : floats)
        if ((uintptr_t)f % 4) return op_fail(err, err_len, RFAST_EINVAL, "%s: an fp32 operand is not aligned to its type", me);
    if (p->tokens == 0 && !p->d_loss) return RFAST_OK;
    const void* ptrs[] = {p->d_logits, p->d_tokens, p->d_dlogits, p->d_old_logp, p->d_ref_logp, p->d_advantage, p->d_weight, p->d_loss_scale, p->d_token_loss, p->d_logp};
    const char* names[] = {"logits", "tokens", "dlogits", "old_logp", "ref_logp", "advantage", "weight", "loss_scale", "token_loss", "logp"};
    char what[64];
    for (int k = 0; k < 10; ++k)
        if (ptrs[k] && p->tokens > 0) {
            std::snprintf(what, sizeof what, "%s: %s", me, names[k]);
            const int rc = check_device_pointer(ptrs[k], what, err, err_len);
            if (rc != RFAST_OK) return rc;
        }
    if (p->d_loss) {
        const int rc = check_device_pointer(p->d_loss, "rfast_policy_loss: loss", err, err_len);
        if (rc != RFAST_OK) return rc;
    }
    Policy a{};
    a.logits = p->d_logits; a.tokens = p->d_tokens;
    a.old_logp = p->d_old_logp; a.ref_logp = p->d_ref_logp; a.advantage = p->d_advantage; a.weight = p->d_weight; a.scale = p->d_loss_scale;
    a.token_loss = p->d_token_loss; a.logp = p->d_logp; a.dlogits = p->d_dlogits;
    a.rows = p->tokens; a.vocab = p->vocab; a.in_stride = p->logits_stride; a.out_stride = p->dlogits_stride;
    a.wide_tokens = p->token_bits == 64;
    a.exact_k = 1.4426950408889634 / p->temperature;
    a.k = (float)a.exact_k;
    int binary = 0;
    const double digits = std::frexp(a.exact_k, &binary);
    a.high = (float)std::ldexp(std::ceil(digits * 4096) - 1, binary - 12);
    a.low = (float)(a.exact_k - a.high);
    a.beyond = (float)(a.exact_k / a.k - 1.0);
    a.inv_t = (float)(1.0 / p->temperature);
    a.clip_lo = 1.0 - p->clip_low; a.clip_hi = 1.0 + p->clip_high; a.kl = p->kl_coef;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    if (p->tokens > 0) {
        // the offset within eight values is the same in every row of both (one row has no stride)
        const int64_t b = (int64_t)bytes_of(p->type);
        const bool align = !p->d_dlogits || (((uintptr_t)p->d_logits ^ (uintptr_t)p->d_dlogits) % (8 * b) == 0 &&
                                             (p->tokens == 1 || (p->logits_stride - p->dlogits_stride) % 8 == 0));
        switch (p->type) {
            case RFAST_TYPE_F32: e = policy_types<float>(a, align, st); break;
            case RFAST_TYPE_BF16: e = policy_types<__nv_bfloat16>(a, align, st); break;
            default: e = policy_types<__half>(a, align, st);
        }
    }
    if (e == cudaSuccess && p->d_loss) e = launch(k_policy_total, dim3(1), 1024, 0, st, p->tokens > 0, (const float*)p->d_token_loss, p->tokens, p->d_loss);
    if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
    return RFAST_OK;
}
