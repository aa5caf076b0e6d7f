// Group norm with an activation, channels last, forward and backward (see rfast_group_norm in rfast.h
// for the formulas).
//
// Work item: a sample (or several, where a sample has few positions) x a slab of channels, the
// smallest run of whole groups that is at least 128 bytes wide.  A thread keeps its column of V
// neighbouring channels and walks down the positions, so that all that belongs to a channel -- sums,
// scale, shift -- sits in its registers.  An item is taken by a cluster of 1 to 16 thread blocks that split
// the positions and exchange the groups' sums through distributed shared memory.  Every value crosses
// HBM once: what a thread has read for the sums waits in shared memory (asynchronous copies that
// only this thread reads back, so no barrier guards them) or, for items too large for that, is read
// again out of L2, where the cluster has just put it.
//
// Variances do not come from a difference of two large sums: a thread sums deviations from the first value it
// sees in each channel, and its mean and sum of squared deviations are merged with the others' by the parallel
// form of the two-pass formula (Chan, Golub, LeVeque).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdio>

#include "ops.h"

namespace cg = cooperative_groups;

namespace rfast {

namespace {

constexpr int kT = 256;                                    // threads per block

template <int BYTES> struct Word;
template <> struct Word<16> { typedef uint4 type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };

// V neighbouring channels of one position, as they lie in memory
template <class T, int V>
struct Vec {
    typedef typename Word<(int)sizeof(T) * V>::type W;
    W w;
};
template <class T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T* p) {
    Vec<T, V> v;
    v.w = *reinterpret_cast<const typename Vec<T, V>::W*>(p);
    return v;
}
__device__ __forceinline__ void widen2(uint32_t r, const __nv_bfloat16*, float* f) {
    f[0] = __uint_as_float(r << 16);
    f[1] = __uint_as_float(r & 0xffff0000u);
}
__device__ __forceinline__ void widen2(uint32_t r, const __half*, float* f) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&r));
    f[0] = a.x; f[1] = a.y;
}
__device__ __forceinline__ void widen(Vec<float, 4> v, float (&f)[4]) {
    f[0] = __uint_as_float(v.w.x); f[1] = __uint_as_float(v.w.y); f[2] = __uint_as_float(v.w.z); f[3] = __uint_as_float(v.w.w);
}
__device__ __forceinline__ void widen(Vec<float, 1> v, float (&f)[1]) { f[0] = __uint_as_float(v.w); }
template <class T>
__device__ __forceinline__ void widen(Vec<T, 8> v, float (&f)[8]) {
    const T* t = nullptr;
    widen2(v.w.x, t, f); widen2(v.w.y, t, f + 2); widen2(v.w.z, t, f + 4); widen2(v.w.w, t, f + 6);
}
template <class T>
__device__ __forceinline__ void widen(Vec<T, 2> v, float (&f)[2]) { widen2(v.w, (const T*)nullptr, f); }
template <class T>
__device__ __forceinline__ void widen(Vec<T, 1> v, float (&f)[1]) {
    float t[2];
    widen2((uint32_t)v.w, (const T*)nullptr, t);
    f[0] = t[0];
}
__device__ __forceinline__ uint32_t narrow2(const float* f, const __nv_bfloat16*) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]);
    return *reinterpret_cast<const uint32_t*>(&a);
}
__device__ __forceinline__ uint32_t narrow2(const float* f, const __half*) {
    const __half2 a = __floats2half2_rn(f[0], f[1]);
    return *reinterpret_cast<const uint32_t*>(&a);
}
__device__ __forceinline__ void store_vec(float* p, const float (&f)[4]) { __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3])); }
__device__ __forceinline__ void store_vec(float* p, const float (&f)[1]) { __stcs(p, f[0]); }
template <class T>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[8]) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(narrow2(f, p), narrow2(f + 2, p), narrow2(f + 4, p), narrow2(f + 6, p)));
}
template <class T>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[2]) { __stcs(reinterpret_cast<uint32_t*>(p), narrow2(f, p)); }
template <class T>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[1]) {
    const float t[2] = {f[0], 0.f};
    __stcs(reinterpret_cast<unsigned short*>(p), (unsigned short)narrow2(t, p));
}
template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// 1 / (1 + exp(-u)).  2^t and the reciprocal are the hardware's (2 ulp and 1 ulp), t is rounded once: the result is good
// to about 2^-23.  u = -inf gives 0.
__device__ __forceinline__ float sigmoid_of(float u) {
    float e, q;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q) : "f"(1.f + e));
    return q;
}

// Rows 0 .. cnt of a thread, R at a time: all loads of a batch go out before the first row is worked on (a
// store in between would hold later loads back, the operands being allowed to coincide).
template <int R, class Row, class Load, class Use>
__device__ __forceinline__ void walk(int cnt, Load load, Use use) {
    int r = 0;
    for (; r + R <= cnt; r += R) {
        Row q[R];
#pragma unroll
        for (int k = 0; k < R; ++k) q[k] = load(r + k);
#pragma unroll
        for (int k = 0; k < R; ++k) use(q[k], r + k);
    }
#pragma unroll 1
    for (; r < cnt; ++r) use(load(r), r);
}

// ---- geometry, chosen on the host -------------------------------------------------------------------
struct GnShape {
    int64_t N, S;                      // samples, positions
    int C, G, Cg;                      // channels, groups, channels per group
    int64_t per_set;                   // samples that share a scale and shift
    float eps;
    int act;
};
struct GnPlan {
    int V;                             // channels per access
    int W, gs, slabs;                  // channels and groups of a slab
    int tx, cj;                        // threads across the slab, passes over its width
    int tr, ns;                        // threads down the positions of a sample, samples per item
    int cluster;                       // thread blocks per item
    int64_t rows;                      // positions per thread block
    int rpt;                           // positions per thread
    bool buffered;                     // what was read waits in shared memory
    int64_t items;                     // items per set (forward: over all samples)
    int64_t parts;                     // backward: thread blocks (clusters) that share a set's items
    size_t buf, smem;                  // bytes: the buffer, all
};

struct GnArgs {
    GnShape s;
    GnPlan p;
    const void* x;
    const void* dy;
    void* out;                         // y, dx
    int64_t xn, xs, dn, ds, on, os;    // strides of a sample and of a position, in elements
    const float *gamma, *beta;
    bool quads;                        // their addresses and stride allow 16-byte loads
    int64_t affine_stride;
    const int* set_row;                // row of gamma / beta of a set, or null: the set itself
    int set_row_stride;
    float *mean, *rstd;                // [N][G]: out (forward), in (backward)
    float *dgamma, *dbeta;             // backward: where the sums of a set go
    float* part;                       // backward: [sets][parts * cluster][2][C] when a set has several blocks
};

__device__ __forceinline__ const float* affine_row(const GnArgs& a, const float* base, int64_t set) {
    const int64_t row = a.set_row ? (int64_t)a.set_row[set * a.set_row_stride] : set;
    return base + row * a.affine_stride;
}

// What a thread is in its block: column, sample of the item, first position; the same for both directions.
struct Seat {
    int txi, sl, rr;                   // column of threads, sample within the item, row of the sample's threads
    bool on;
};
__device__ __forceinline__ Seat seat_of(const GnPlan& p) {
    Seat s;
    const int tyi = threadIdx.x / p.tx;
    s.txi = threadIdx.x - tyi * p.tx;
    s.sl = tyi / p.tr;
    s.rr = tyi - s.sl * p.tr;
    s.on = s.sl < p.ns;
    return s;
}

// scale or shift of V neighbouring channels
template <int V>
__device__ __forceinline__ void affine_of(const float* p, bool quads, float (&f)[V]) {
    if constexpr (V % 4 == 0) {
        if (quads) {
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                const float4 q = *reinterpret_cast<const float4*>(p + k);
                f[k] = q.x; f[k + 1] = q.y; f[k + 2] = q.z; f[k + 3] = q.w;
            }
            return;
        }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) f[k] = p[k];
}
// groups of V neighbouring channels from channel c on: one (WHOLE) or one per channel
template <int V, bool WHOLE>
__device__ __forceinline__ void groups_of(int c, int cg, int (&g)[WHOLE ? 1 : V]) {
    int q = c / cg;
    g[0] = q;
    if constexpr (!WHOLE) {
        int rest = c - q * cg;
#pragma unroll
        for (int v = 1; v < V; ++v) {
            if (++rest == cg) { rest = 0; ++q; }
            g[v] = q;
        }
    }
}

// Sum over L neighbouring lanes (L a power of two), all lanes of the warp taking part.
__device__ __forceinline__ float team_sum(float v, int L) {
    for (int o = L >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ int team_size(int entries) {
    int L = 1;
    while (L < entries && L < 32) L <<= 1;
    return L;
}

// ---- forward --------------------------------------------------------------------------------------
// grid = (items * cluster, slabs), clusters along x
template <class T, int V, bool WHOLE, bool BUF>
__global__ void __launch_bounds__(kT, BUF && WHOLE ? 4 : 3)
k_gn_forward(const __grid_constant__ GnArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    typedef Vec<T, V> X;
    const GnShape& s = a.s;
    const GnPlan& p = a.p;
    constexpr int kBatch = 4, kGv = WHOLE ? 1 : V, kAcc = WHOLE ? (V < 4 ? V : 4) : V;
    X* buf = reinterpret_cast<X*>(smem);
    // per thread (WHOLE: an access stays inside a group) or per thread and channel: count, mean, sum of squared deviations
    float* e_n = reinterpret_cast<float*>(smem + p.buf);
    constexpr int width = kGv;
    float* e_mean = e_n + kT;
    float* e_m2 = e_mean + kT * width;
    float* bins = e_m2 + kT * width;                        // [ns * gs][3], then [ns * gs][2] final
    const int gs = min(p.gs, s.G - (int)blockIdx.y * p.gs); // the last slab may be narrower
    const int nb = p.ns * gs;
    float* fin = bins + 3 * nb;

    const int rank = p.cluster > 1 ? blockIdx.x % p.cluster : 0;
    const int64_t item = blockIdx.x / p.cluster;
    const Seat me = seat_of(p);
    const int64_t n = item * p.ns + me.sl;
    const bool on = me.on && n < s.N;
    const int64_t r0 = (int64_t)rank * p.rows + me.rr;
    const int64_t r1 = min(s.S, (int64_t)(rank + 1) * p.rows);
    const int cnt = on && r0 < r1 ? (int)((r1 - r0 + p.tr - 1) / p.tr) : 0;
    const int c0 = blockIdx.y * p.W, cols = gs * s.Cg / V;
    const T* x = (const T*)a.x + n * a.xn + r0 * a.xs + c0;
    const int64_t step = (int64_t)p.tr * a.xs;

    if (BUF) {
        for (int j = 0; j < p.cj; ++j) {
            const int cv = me.txi + j * kT;
            if (cv < cols)
                for (int r = 0; r < cnt; ++r) copy_async<sizeof(X)>(buf + (j * p.rpt + r) * kT + threadIdx.x, x + r * step + cv * V);
        }
        copies_landed();
    }
    // count, mean and squared deviations of what this thread holds
    float t_n = 0.f, t_mean = 0.f, t_m2 = 0.f;
    for (int j = 0; j < p.cj; ++j) {
        const int cv = me.txi + j * kT;
        float first[kGv], s1[kAcc], s2[kAcc];
#pragma unroll
        for (int v = 0; v < kAcc; ++v) s1[v] = s2[v] = 0.f;
#pragma unroll
        for (int v = 0; v < kGv; ++v) first[v] = 0.f;
        if (cnt > 0 && cv < cols) {
            const T* at = x + cv * V;
            const X* bt = buf + j * p.rpt * kT + threadIdx.x;
            auto load = [&](int r) { return BUF ? bt[r * kT] : load_vec<T, V>(at + r * step); };
            {
                float f[V];
                widen(load(0), f);
#pragma unroll
                for (int v = 0; v < kGv; ++v) first[v] = f[v];
            }
            walk<kBatch, X>(cnt, load, [&](const X& q, int) {     // a first value counts as a deviation of 0
                float f[V];
                widen(q, f);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float d = f[v] - first[WHOLE ? 0 : v];
                    s1[v % kAcc] += d;
                    s2[v % kAcc] = fmaf(d, d, s2[v % kAcc]);
                }
            });
            if (WHOLE) {
#pragma unroll
                for (int v = 1; v < kAcc; ++v) { s1[0] += s1[v]; s2[0] += s2[v]; }
            }
            const float nn = (float)cnt * (WHOLE ? V : 1), inv = 1.f / nn;
#pragma unroll
            for (int v = 0; v < kGv; ++v) {
                const float d = s1[v] * inv;
                s2[v] = fmaxf(fmaf(-s1[v], d, s2[v]), 0.f) + (s2[v] - s2[v]);    // the second term is a NaN where there was one
                first[v] += d;                              // now the mean
            }
            if (WHOLE && t_n > 0.f) {                       // a further pass over a wide group
                const float d = first[0] - t_mean, tot = t_n + nn;
                t_mean += d * (nn / tot);
                t_m2 += s2[0] + d * d * (t_n * nn / tot);
                t_n = tot;
            } else {
                t_mean = first[0]; t_m2 = s2[0]; t_n = nn;
            }
        }
        if (!WHOLE) {                                       // a slab of several groups is never wider than the block
            if (me.on && cv < cols) {
#pragma unroll
                for (int v = 0; v < kGv; ++v) { e_mean[threadIdx.x * V + v] = first[v]; e_m2[threadIdx.x * V + v] = s2[v]; }
            }
        }
    }
    e_n[threadIdx.x] = t_n;
    if (WHOLE) { e_mean[threadIdx.x] = t_mean; e_m2[threadIdx.x] = t_m2; }
    __syncthreads();
    // the groups' sums over this block, a team of lanes per group
    {
        const int unit = WHOLE ? min(s.Cg / V, p.tx) : s.Cg;   // entries of a group in one row of threads
        const int entries = unit * p.tr, L = team_size(entries), lane = threadIdx.x & (L - 1);
        for (int b0 = 0; b0 < nb; b0 += kT / L) {
            const int b = b0 + threadIdx.x / L;
            const bool in = b < nb;
            const int sl = in ? b / gs : 0, g = in ? b - sl * gs : 0;
            // means are summed as differences from one of them: a flat group has exactly its level
            const float ref = in ? e_mean[sl * p.tr * p.tx * width + g * unit] : 0.f;
            float cn = 0.f, cm = 0.f;
            for (int q = lane; in && q < entries; q += L) {
                const int row = q / unit, t = (sl * p.tr + row) * p.tx, u = g * unit + (q - row * unit);
                const float k = e_n[t + (WHOLE ? u : u / V)];
                cn += k;
                if (k > 0.f) cm = fmaf(k, e_mean[t * width + u] - ref, cm);
            }
            cn = team_sum(cn, L);
            cm = team_sum(cm, L);
            const float mean = cn > 0.f ? ref + cm / cn : 0.f;
            float m2 = 0.f;
            for (int q = lane; in && q < entries; q += L) {
                const int row = q / unit, t = (sl * p.tr + row) * p.tx, u = g * unit + (q - row * unit);
                const float k = e_n[t + (WHOLE ? u : u / V)];
                if (k > 0.f) {
                    const float d = e_mean[t * width + u] - mean;
                    m2 += fmaf(k * d, d, e_m2[t * width + u]);
                }
            }
            m2 = team_sum(m2, L);
            if (in && lane == 0) { bins[3 * b] = cn; bins[3 * b + 1] = mean; bins[3 * b + 2] = m2; }
        }
    }
    if (p.cluster > 1) cg::this_cluster().sync(); else __syncthreads();
    for (int b = threadIdx.x; b < nb; b += kT) {
        float mean = bins[3 * b + 1], m2 = bins[3 * b + 2];
        if (p.cluster > 1) {                                // every block of the cluster adds up the same, in the same order
            cg::cluster_group cl = cg::this_cluster();
            const float ref = cl.map_shared_rank(bins, 0)[3 * b + 1];
            float cn = 0.f, cm = 0.f;
            for (int r = 0; r < p.cluster; ++r) {
                const float* o = cl.map_shared_rank(bins, r) + 3 * b;
                if (o[0] > 0.f) { cn += o[0]; cm = fmaf(o[0], o[1] - ref, cm); }
            }
            mean = ref + cm / cn;
            m2 = 0.f;
            for (int r = 0; r < p.cluster; ++r) {
                const float* o = cl.map_shared_rank(bins, r) + 3 * b;
                if (o[0] > 0.f) { const float d = o[1] - mean; m2 += fmaf(o[0] * d, d, o[2]); }
            }
        }
        const float rstd = rsqrtf(m2 / ((float)s.S * (float)s.Cg) + s.eps);
        fin[2 * b] = mean;
        fin[2 * b + 1] = rstd;
        const int sl = b / gs;
        const int64_t nn = item * p.ns + sl;
        if (rank == 0 && nn < s.N) {
            const int64_t at = nn * s.G + blockIdx.y * p.gs + (b - sl * gs);
            a.mean[at] = mean;
            a.rstd[at] = rstd;
        }
    }
    if (p.cluster > 1) cg::this_cluster().barrier_arrive();    // this block has read what it needs of the others
    __syncthreads();
    if (cnt > 0) {
        const int64_t set = n / s.per_set;
        const float* gam = affine_row(a, a.gamma, set) + c0;
        const float* bet = affine_row(a, a.beta, set) + c0;
        T* y = (T*)a.out + n * a.on + r0 * a.os + c0;
        const int64_t ostep = (int64_t)p.tr * a.os;
        for (int j = 0; j < p.cj; ++j) {
            const int cv = me.txi + j * kT;
            if (cv >= cols) break;
            float mean[kGv], mul[V], add[V];
            int g[kGv];
            groups_of<V, WHOLE>(cv * V, s.Cg, g);
            affine_of<V>(gam + cv * V, a.quads, mul);
            affine_of<V>(bet + cv * V, a.quads, add);
#pragma unroll
            for (int v = 0; v < kGv; ++v) {
                const float* f = fin + 2 * (me.sl * gs + g[v]);
                mean[v] = f[0];
                if (WHOLE) {
#pragma unroll
                    for (int u = 0; u < V; ++u) mul[u] *= f[1];
                } else {
                    mul[v] *= f[1];
                }
            }
            const T* at = x + cv * V;
            const X* bt = buf + j * p.rpt * kT + threadIdx.x;
            auto load = [&](int r) { return BUF ? bt[r * kT] : load_vec<T, V>(at + r * step); };
            walk<kBatch, X>(cnt, load, [&](const X& q, int r) {
                float o[V];
                widen(q, o);
#pragma unroll
                for (int v = 0; v < V; ++v) o[v] = fmaf(o[v] - mean[WHOLE ? 0 : v], mul[v], add[v]);
                if (s.act == RFAST_ACT_SILU) {
#pragma unroll
                    for (int v = 0; v < V; ++v) o[v] *= sigmoid_of(o[v]);
                } else if (s.act == RFAST_ACT_RELU) {
#pragma unroll
                    for (int v = 0; v < V; ++v) o[v] = o[v] < 0.f ? 0.f : o[v];       // a NaN stays one
                }
                store_vec(y + r * ostep + cv * V, o);
            });
        }
    }
    if (p.cluster > 1) cg::this_cluster().barrier_wait();      // nobody reads this block's sums any more
}

// ---- backward -------------------------------------------------------------------------------------
// dy act'(u)
template <int V>
__device__ __forceinline__ void through(int act, const float (&u)[V], float (&dy)[V]) {
    if (act == RFAST_ACT_SILU) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float q = sigmoid_of(u[v]);
            dy[v] *= fmaf(q, fmaf(-q, u[v], u[v]), q);       // q (1 + u (1 - q))
        }
    } else if (act == RFAST_ACT_RELU) {
#pragma unroll
        for (int v = 0; v < V; ++v) dy[v] = u[v] > 0.f ? dy[v] : 0.f;
    }
}
template <class X> struct Pair { X x, d; };

// With du = dy act'(u), h = (x - mean) rstd, and over the M values of a group
//     one = sum gamma du / M, two = sum gamma du h / M:   dx = rstd (gamma du - one - two h);
// per channel dbeta = sum du, dgamma = sum du h over the samples of a set.  A cluster takes every
// `parts`-th item of a set and keeps the channels' sums of its items in shared memory.
// grid = (parts * cluster, slabs, sets)
template <class T, int V, bool WHOLE, bool BUF>
__global__ void __launch_bounds__(kT, BUF && WHOLE ? 3 : 2)
k_gn_backward(const __grid_constant__ GnArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    typedef Vec<T, V> X;
    const GnShape& s = a.s;
    const GnPlan& p = a.p;
    constexpr int kBatch = BUF ? 2 : 4, kGv = WHOLE ? 1 : V;
    X* bufx = reinterpret_cast<X*>(smem);
    X* bufd = reinterpret_cast<X*>(smem + p.buf / 2);
    float* ent = reinterpret_cast<float*>(smem + p.buf);     // [2][kT * V]: du, du h of a thread's channels
    float* col = ent + 2 * kT * V;                           // [2][ns * width of a pass]: the same, summed down the positions
    const int gs = min(p.gs, s.G - (int)blockIdx.y * p.gs); // the last slab may be narrower
    const int W = gs * s.Cg, nb = p.ns * gs;
    const int wide = min(p.W, kT * V);                       // channels of one pass over the width
    float* sums = col + (p.tr > 1 ? 2 * max(kT, p.ns * wide) : 0);    // [nb][2] this block's, then [nb][2] the cluster's
    float* tot = sums + 2 * nb;
    float* acc = tot + 2 * nb;                               // [2][W]: dbeta, dgamma of the block's items

    const int rank = p.cluster > 1 ? blockIdx.x % p.cluster : 0;
    const int64_t set = blockIdx.z;
    const Seat me = seat_of(p);
    const int64_t r0 = (int64_t)rank * p.rows + me.rr;
    const int64_t r1 = min(s.S, (int64_t)(rank + 1) * p.rows);
    const int c0 = blockIdx.y * p.W, cols = W / V;
    const float* gam = affine_row(a, a.gamma, set) + c0;
    const float* bet = affine_row(a, a.beta, set) + c0;
    const int64_t xstep = (int64_t)p.tr * a.xs, dstep = (int64_t)p.tr * a.ds, ostep = (int64_t)p.tr * a.os;
    const float inv_m = 1.f / ((float)s.S * (float)s.Cg);
    for (int c = threadIdx.x; c < 2 * p.W; c += kT) acc[c] = 0.f;

    for (int64_t item = blockIdx.x / p.cluster; item < p.items; item += p.parts) {
        const int64_t in_set = item * p.ns + me.sl, n = set * s.per_set + in_set;
        const bool on = me.on && in_set < s.per_set;
        const int cnt = on && r0 < r1 ? (int)((r1 - r0 + p.tr - 1) / p.tr) : 0;
        const T* x = (const T*)a.x + n * a.xn + r0 * a.xs + c0;
        const T* dy = (const T*)a.dy + n * a.dn + r0 * a.ds + c0;
        if (BUF) {
            for (int j = 0; j < p.cj; ++j) {
                const int cv = me.txi + j * kT;
                if (cv < cols)
                    for (int r = 0; r < cnt; ++r) {
                        copy_async<sizeof(X)>(bufx + (j * p.rpt + r) * kT + threadIdx.x, x + r * xstep + cv * V);
                        copy_async<sizeof(X)>(bufd + (j * p.rpt + r) * kT + threadIdx.x, dy + r * dstep + cv * V);
                    }
            }
            copies_landed();
        }
        for (int b = threadIdx.x; b < 2 * nb; b += kT) sums[b] = 0.f;
        for (int j = 0; j < p.cj; ++j) {
            const int cv = me.txi + j * kT;
            float s_du[V], s_dh[V];
#pragma unroll
            for (int v = 0; v < V; ++v) s_du[v] = s_dh[v] = 0.f;
            if (cnt > 0 && cv < cols) {
                float mean[kGv], rs[kGv], mul[V], add[V];    // u = (x - mean) mul + add
                int g[kGv];
                groups_of<V, WHOLE>(c0 + cv * V, s.Cg, g);
                affine_of<V>(gam + cv * V, a.quads, mul);
                affine_of<V>(bet + cv * V, a.quads, add);
#pragma unroll
                for (int v = 0; v < kGv; ++v) { mean[v] = a.mean[n * s.G + g[v]]; rs[v] = a.rstd[n * s.G + g[v]]; }
#pragma unroll
                for (int v = 0; v < V; ++v) mul[v] *= rs[WHOLE ? 0 : v];
                const X* bx = bufx + j * p.rpt * kT + threadIdx.x;
                const X* bd = bufd + j * p.rpt * kT + threadIdx.x;
                auto load = [&](int r) {
                    Pair<X> q;
                    q.x = BUF ? bx[r * kT] : load_vec<T, V>(x + r * xstep + cv * V);
                    q.d = BUF ? bd[r * kT] : load_vec<T, V>(dy + r * dstep + cv * V);
                    return q;
                };
                walk<kBatch, Pair<X>>(cnt, load, [&](const Pair<X>& q, int) {
                    float d[V], du[V], u[V];
                    widen(q.x, d);
                    widen(q.d, du);
#pragma unroll
                    for (int v = 0; v < V; ++v) { d[v] -= mean[WHOLE ? 0 : v]; u[v] = fmaf(d[v], mul[v], add[v]); }
                    through(s.act, u, du);
#pragma unroll
                    for (int v = 0; v < V; ++v) { s_du[v] += du[v]; s_dh[v] = fmaf(du[v], d[v], s_dh[v]); }
                });
#pragma unroll
                for (int v = 0; v < V; ++v) s_dh[v] *= rs[WHOLE ? 0 : v];     // h = (x - mean) rstd
            }
            // [row of threads][channel of this pass]
            if (me.on) {
#pragma unroll
                for (int v = 0; v < V; v += (V >= 4 ? 4 : 1)) {
                    float *e0 = ent + threadIdx.x * V + v, *e1 = e0 + kT * V;
                    if constexpr (V >= 4) {
                        *reinterpret_cast<float4*>(e0) = make_float4(s_du[v], s_du[v + 1], s_du[v + 2], s_du[v + 3]);
                        *reinterpret_cast<float4*>(e1) = make_float4(s_dh[v], s_dh[v + 1], s_dh[v + 2], s_dh[v + 3]);
                    } else {
                        *e0 = s_du[v];
                        *e1 = s_dh[v];
                    }
                }
            }
            __syncthreads();
            const int pw = min(p.tx * V, W - j * kT * V);  // channels of this pass
            const int pitch = p.tx * V;
            const float *q0 = ent, *q1 = ent + kT * V;
            int qp = pitch;                                  // floats between a sample's rows
            if (p.tr > 1) {
                // down the rows of threads, `ways` threads per channel, then their sums, in fixed order
                const int nc = p.ns * pw, ways = nc >= kT ? 1 : min(kT / nc, p.tr);
                float *c0s = col, *c1s = col + (kT > p.ns * wide ? kT : p.ns * wide);
                for (int i = threadIdx.x; i < nc * ways; i += kT) {
                    const int w = i / nc, k = i - w * nc, sl = k / pw;
                    float u0 = 0.f, u1 = 0.f;
                    for (int at = (sl * p.tr + w) * pitch + (k - sl * pw), r = w; r < p.tr; r += ways, at += ways * pitch) {
                        u0 += q0[at];
                        u1 += q1[at];
                    }
                    c0s[i] = u0;
                    c1s[i] = u1;
                }
                __syncthreads();
                if (ways > 1) {
                    if ((int)threadIdx.x < nc) {             // nc < kT: one channel per thread
                        float u0 = c0s[threadIdx.x], u1 = c1s[threadIdx.x];
                        for (int w = 1; w < ways; ++w) { u0 += c0s[w * nc + threadIdx.x]; u1 += c1s[w * nc + threadIdx.x]; }
                        c0s[threadIdx.x] = u0;
                        c1s[threadIdx.x] = u1;
                    }
                    __syncthreads();
                }
                q0 = c0s; q1 = c1s; qp = pw;
            }
            // dbeta, dgamma of this item's samples
            for (int c = threadIdx.x; c < pw; c += kT) {
                float u0 = 0.f, u1 = 0.f;
                for (int sl = 0; sl < p.ns; ++sl) { u0 += q0[sl * qp + c]; u1 += q1[sl * qp + c]; }
                acc[j * kT * V + c] += u0;
                acc[p.W + j * kT * V + c] += u1;
            }
            // the groups' sums, a team of lanes per group
            const int unit = min(s.Cg, pw), L = team_size(unit), lane = threadIdx.x & (L - 1);
            for (int b0 = 0; b0 < nb; b0 += kT / L) {
                const int b = b0 + threadIdx.x / L;
                float u0 = 0.f, u1 = 0.f;
                if (b < nb) {
                    const int sl = b / gs, g = b - sl * gs;
                    for (int q = lane; q < unit; q += L) {
                        const int c = g * unit + q;
                        const float ga = gam[j * kT * V + c];
                        u0 = fmaf(ga, q0[sl * qp + c], u0);
                        u1 = fmaf(ga, q1[sl * qp + c], u1);
                    }
                }
                u0 = team_sum(u0, L);
                u1 = team_sum(u1, L);
                if (b < nb && lane == 0) { sums[2 * b] += u0; sums[2 * b + 1] += u1; }
            }
            __syncthreads();                                 // before the next pass or item fills `ent`
        }
        if (p.cluster > 1) {
            cg::cluster_group cl = cg::this_cluster();
            cl.sync();
            for (int b = threadIdx.x; b < 2 * nb; b += kT) {
                float u = 0.f;
                for (int r = 0; r < p.cluster; ++r) u += cl.map_shared_rank(sums, r)[b];
                tot[b] = u;
            }
            cl.sync();                                       // `sums` may be filled again, `tot` stands
        }
        const float* sg = p.cluster > 1 ? tot : sums;
        if (cnt > 0) {
            T* dx = (T*)a.out + n * a.on + r0 * a.os + c0;
            for (int j = 0; j < p.cj; ++j) {
                const int cv = me.txi + j * kT;
                if (cv >= cols) break;
                float mean[kGv], k1[kGv], k2[kGv], mul[V], add[V];   // dx = mul du - k1 - (x - mean) k2
                int g[kGv];
                groups_of<V, WHOLE>(cv * V, s.Cg, g);
                affine_of<V>(gam + cv * V, a.quads, mul);
                affine_of<V>(bet + cv * V, a.quads, add);
#pragma unroll
                for (int v = 0; v < kGv; ++v) {
                    const int64_t at = n * s.G + blockIdx.y * p.gs + g[v];
                    const float rs = a.rstd[at], *q = sg + 2 * (me.sl * gs + g[v]);
                    mean[v] = a.mean[at];
                    k1[v] = rs * (q[0] * inv_m);
                    k2[v] = rs * rs * (q[1] * inv_m);
                    if (WHOLE) {
#pragma unroll
                        for (int u = 0; u < V; ++u) mul[u] *= rs;
                    } else {
                        mul[v] *= rs;
                    }
                }
                const X* bx = bufx + j * p.rpt * kT + threadIdx.x;
                const X* bd = bufd + j * p.rpt * kT + threadIdx.x;
                auto load = [&](int r) {
                    Pair<X> q;
                    q.x = BUF ? bx[r * kT] : load_vec<T, V>(x + r * xstep + cv * V);
                    q.d = BUF ? bd[r * kT] : load_vec<T, V>(dy + r * dstep + cv * V);
                    return q;
                };
                walk<kBatch, Pair<X>>(cnt, load, [&](const Pair<X>& q, int r) {
                    float d[V], du[V], u[V];
                    widen(q.x, d);
                    widen(q.d, du);
#pragma unroll
                    for (int v = 0; v < V; ++v) { d[v] -= mean[WHOLE ? 0 : v]; u[v] = fmaf(d[v], mul[v], add[v]); }
                    through(s.act, u, du);
#pragma unroll
                    for (int v = 0; v < V; ++v) du[v] = fmaf(du[v], mul[v], fmaf(-d[v], k2[WHOLE ? 0 : v], -k1[WHOLE ? 0 : v]));
                    store_vec(dx + r * ostep + cv * V, du);
                });
            }
        }
        if (p.cluster == 1) __syncthreads();                 // `sums` may be filled again
    }
    if (p.parts * p.cluster == 1) {
        for (int c = threadIdx.x; c < W; c += kT) {
            a.dbeta[set * s.C + c0 + c] = acc[c];
            a.dgamma[set * s.C + c0 + c] = acc[p.W + c];
        }
    } else {
        float* row = a.part + ((set * p.parts * p.cluster + blockIdx.x) * 2) * s.C + c0;
        for (int c = threadIdx.x; c < W; c += kT) {
            row[c] = acc[c];
            row[s.C + c] = acc[p.W + c];
        }
    }
}

// dgamma, dbeta of a set from its blocks' sums, in the order of the blocks, eight at a time, in 64 bits.
// grid = (channels / 32, sets), 256 threads
__global__ void __launch_bounds__(kT)
k_gn_affine(const float* __restrict__ part, int rows, int C, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ double sh[2][8][32];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    const float* base = part + (int64_t)blockIdx.y * rows * 2 * C + c;
    double b = 0.0, g = 0.0;
    if (c < C)
        for (int r = w; r < rows; r += 8) {
            b += (double)base[(int64_t)r * 2 * C];
            g += (double)base[(int64_t)r * 2 * C + C];
        }
    sh[0][w][threadIdx.x & 31] = b;
    sh[1][w][threadIdx.x & 31] = g;
    __syncthreads();
    if (w < 2 && c < C) {
        double u = 0.0;
        for (int k = 0; k < 8; ++k) u += sh[w][k][threadIdx.x & 31];
        (w ? dgamma : dbeta)[(int64_t)blockIdx.y * C + c] = (float)u;
    }
}

// ---- host side ------------------------------------------------------------------------------------
constexpr int kSms = 148;
constexpr int kMaxGroupChannels = 8192;                     // a block keeps two sums for every channel of a group
constexpr size_t kBufMost = 200 * 1024, kBufGood = 64 * 1024;

// Blocks that may share a set's sums: bounds the workspace, whatever the plan.
int64_t part_rows(const GnShape& s) {
    const int64_t sets = s.N / s.per_set;
    int64_t cap = 1024 / sets;
    cap = cap < 16 ? 16 : cap > 256 ? 256 : cap;
    const int64_t most = s.per_set * (s.S < 64 ? 1 : 16);
    return cap < most ? cap : most;
}

size_t plan_smem(const GnShape& s, const GnPlan& p, bool backward) {
    const size_t nb = (size_t)p.ns * p.gs;
    if (!backward) {
        const size_t width = s.Cg % p.V == 0 ? 1 : p.V;
        return p.buf + sizeof(float) * (kT + 2 * kT * width + 5 * nb);
    }
    const size_t wide = p.W < kT * p.V ? p.W : kT * p.V;
    return p.buf + sizeof(float) * (2 * (size_t)kT * p.V + (p.tr > 1 ? 2 * (p.ns * wide > kT ? p.ns * wide : (size_t)kT) : 0) + 4 * nb + 2 * (size_t)p.W);
}

// vmax: channels per access that addresses and strides allow (a power of two, times the type at most 16 bytes)
GnPlan make_plan(const GnShape& s, int esize, int vmax, bool backward) {
    GnPlan best{};
    int V = vmax;
    // an access may straddle narrow groups, but a slab has to hold whole accesses
    const bool broad = s.Cg * esize >= 128;
    if (broad) { while (s.Cg % V) V /= 2; } else { while (s.C % V) V /= 2; }
    if (V * esize == 8) V /= 2;                             // accesses of 16, 4 or 2 bytes
    const int64_t batch = backward ? s.per_set : s.N, sets = backward ? s.N / s.per_set : 1;
    const int streams = backward ? 2 : 1;
    for (int target = 128; target >= 32; target /= 2) {
        GnPlan p{};
        p.V = V;
        p.gs = broad ? 1 : s.G;
        if (!broad)
            for (int gs = 1; gs < s.G; ++gs)
                if (gs * s.Cg % V == 0 && gs * s.Cg * esize >= target) { p.gs = gs; break; }
        p.W = p.gs * s.Cg;
        p.slabs = (s.G + p.gs - 1) / p.gs;
        const int cols = p.W / V;
        p.tx = cols < kT ? cols : kT;
        p.cj = (cols + kT - 1) / kT;
        const int ty = kT / p.tx;
        // thread blocks per item: enough of them to fill the SMs twice, each with at least a row per thread,
        // and with what it reads in 64 KB of shared memory if that can be had
        p.cluster = 1;
        auto shape_of = [&](int cl) {
            p.cluster = cl;
            p.rows = (s.S + cl - 1) / cl;
            p.tr = (int)(p.rows < ty ? p.rows : ty);
            p.ns = 1;
            if (cl == 1) {
                int64_t ns = ty / p.tr;
                if (ns > batch) ns = batch;
                p.ns = (int)ns;
            }
            const int64_t rpt = (p.rows + p.tr - 1) / p.tr;
            const int64_t bytes = rpt * p.cj * kT * V * esize * streams;
            p.items = (batch + p.ns - 1) / p.ns;
            p.buffered = V * esize >= 4 && bytes <= (int64_t)kBufMost;
            p.rpt = p.buffered ? (int)rpt : 0;
            p.buf = p.buffered ? (size_t)bytes : 0;
            return p.items * sets * p.slabs * cl;
        };
        int64_t blocks = shape_of(1);
        while (p.cluster < 16 && s.S >= 64 && p.rows > 2 * ty &&
               (blocks < 2 * kSms || !p.buffered || p.buf > kBufGood)) blocks = shape_of(p.cluster * 2);
        p.smem = plan_smem(s, p, backward);
        if (p.buffered && p.smem > 220 * 1024) { p.buffered = false; p.buf = 0; p.rpt = 0; p.smem = plan_smem(s, p, backward); }
        p.parts = 1;
        if (backward) {
            int64_t most = part_rows(s) / p.cluster;
            if (most < 1) most = 1;
            p.parts = p.items < most ? p.items : most;
        }
        if (target == 128) best = p;
        else if (p.slabs > best.slabs) best = p;
        if (blocks >= kSms || broad) break;                 // narrower slabs only where thread blocks are few
    }
    return best;
}

template <class K>
cudaError_t launch_plan(K kernel, dim3 grid, const GnArgs& a, cudaStream_t st) {
    cudaError_t e = cudaSuccess;
    if (a.p.smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)a.p.smem);
    if (e == cudaSuccess && a.p.cluster > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid; cfg.blockDim = dim3(kT); cfg.dynamicSmemBytes = a.p.smem; cfg.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = a.p.cluster; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
    cfg.attrs = &at; cfg.numAttrs = a.p.cluster > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <class T, int V, bool WHOLE>
cudaError_t launch_whole(const GnArgs& a, bool backward, dim3 grid, cudaStream_t st) {
    if constexpr (sizeof(T) * V >= 4) {
        if (a.p.buffered) return backward ? launch_plan(k_gn_backward<T, V, WHOLE, true>, grid, a, st) : launch_plan(k_gn_forward<T, V, WHOLE, true>, grid, a, st);
    }
    return backward ? launch_plan(k_gn_backward<T, V, WHOLE, false>, grid, a, st) : launch_plan(k_gn_forward<T, V, WHOLE, false>, grid, a, st);
}
template <class T, int V>
cudaError_t launch_gn(const GnArgs& a, bool backward, cudaStream_t st) {
    const dim3 grid((unsigned)((backward ? a.p.parts : a.p.items) * a.p.cluster), a.p.slabs, backward ? (unsigned)(a.s.N / a.s.per_set) : 1);
    if (a.s.Cg % V == 0) return launch_whole<T, V, true>(a, backward, grid, st);
    if constexpr (V > 1) return launch_whole<T, V, false>(a, backward, grid, st);
    return cudaErrorInvalidValue;
}

cudaError_t launch_typed(GnArgs& a, int type, bool backward, cudaStream_t st) {
    a.quads = !((uintptr_t)a.gamma % 16 || (uintptr_t)a.beta % 16 || a.affine_stride % 4);
    switch (type) {
        case RFAST_TYPE_F32: return a.p.V == 4 ? launch_gn<float, 4>(a, backward, st) : launch_gn<float, 1>(a, backward, st);
        case RFAST_TYPE_BF16:
            return a.p.V == 8 ? launch_gn<__nv_bfloat16, 8>(a, backward, st)
                 : a.p.V == 2 ? launch_gn<__nv_bfloat16, 2>(a, backward, st) : launch_gn<__nv_bfloat16, 1>(a, backward, st);
        default:
            return a.p.V == 8 ? launch_gn<__half, 8>(a, backward, st)
                 : a.p.V == 2 ? launch_gn<__half, 2>(a, backward, st) : launch_gn<__half, 1>(a, backward, st);
    }
}

int type_bytes(int t) { return t == RFAST_TYPE_F32 ? 4 : 2; }

// channels per access that an address and its strides allow
int allowed(const void* p, int64_t sn, int64_t ss, int esize) {
    int v = 16 / esize;
    while (v > 1 && ((uintptr_t)p % (v * esize) || sn % v || ss % v)) v /= 2;
    return v;
}

int check_shape(const rfast_gn_shape* g, const char* me, char* err, size_t err_len) {
    if (!g) return op_fail(err, err_len, RFAST_EINVAL, "%s: null shape", me);
    if (g->type != RFAST_TYPE_F32 && g->type != RFAST_TYPE_BF16 && g->type != RFAST_TYPE_F16) return op_fail(err, err_len, RFAST_EINVAL, "%s: unknown type", me);
    if (g->act != RFAST_ACT_NONE && g->act != RFAST_ACT_RELU && g->act != RFAST_ACT_SILU) return op_fail(err, err_len, RFAST_EINVAL, "%s: unknown activation", me);
    if (g->samples < 0 || g->samples > 0x7fffffff || g->positions < 0 || g->positions > 0x7fffffff)
        return op_fail(err, err_len, RFAST_EINVAL, "%s: samples and positions must be in [0, 2^31)", me);
    if (g->groups < 1 || g->channels < 1 || g->channels % g->groups) return op_fail(err, err_len, RFAST_EINVAL, "%s: channels must be a positive multiple of groups", me);
    if (g->channels / g->groups > kMaxGroupChannels) return op_fail(err, err_len, RFAST_EINVAL, "%s: a group may have %d channels at most", me, kMaxGroupChannels);
    if (g->channels > (1 << 24)) return op_fail(err, err_len, RFAST_EINVAL, "%s: 2^24 channels at most", me);
    if (g->samples_per_set < 1 || (g->samples > 0 && g->samples % g->samples_per_set)) return op_fail(err, err_len, RFAST_EINVAL, "%s: samples must be a multiple of samples_per_set", me);
    return RFAST_OK;
}

GnShape shape_from(const rfast_gn_shape* g, float eps) {
    GnShape s{};
    s.N = g->samples; s.S = g->positions; s.C = g->channels; s.G = g->groups; s.Cg = g->channels / g->groups;
    s.per_set = g->samples_per_set; s.eps = eps; s.act = g->act;
    return s;
}

// strides of an operand: contiguous where none are given
int strides_of(const int64_t* given, const GnShape& s, int64_t* sn, int64_t* ss, const char* me, const char* what, char* err, size_t err_len) {
    *ss = given ? given[1] : s.C;
    *sn = given ? given[0] : (int64_t)s.C * s.S;
    if (*sn < 0 || *ss < 0) return op_fail(err, err_len, RFAST_EINVAL, "%s: a stride of %s is negative", me, what);
    return RFAST_OK;
}

// Whether two of the N x S rows of C values share one (rows that interleave in other ways than one stride
// inside the other count as overlapping).
bool overlaps(const GnShape& s, int64_t sn, int64_t ss) {
    int64_t near = ss, far = sn, inner = s.S, outer = s.N;
    if (outer > 1 && (inner == 1 || sn < ss)) { near = sn; far = ss; inner = s.N; outer = s.S; }
    if (inner > 1 && near < s.C) return true;
    return outer > 1 && far < (inner - 1) * near + s.C;
}

}  // namespace

}  // namespace rfast

using namespace rfast;

#define GN_TRY(expr) do { const int rc_ = (expr); if (rc_ != RFAST_OK) return rc_; } while (0)

extern "C" int64_t rfast_group_norm_workspace(const rfast_gn_shape* g, int backward) {
    const int rc = check_shape(g, "rfast_group_norm_workspace", nullptr, 0);
    if (rc != RFAST_OK) return rc;
    if (!backward || g->samples == 0) return 0;
    const GnShape s = shape_from(g, 1.f);
    return (s.N / s.per_set) * part_rows(s) * 2 * s.C * (int64_t)sizeof(float);
}

extern "C" int rfast_group_norm(const rfast_gn_shape* g, const void* d_x, const int64_t* x_strides, const float* d_gamma, const float* d_beta, float eps,
                                void* d_y, const int64_t* y_strides, float* d_mean, float* d_rstd, void* workspace, size_t workspace_bytes,
                                void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_group_norm";
    (void)workspace; (void)workspace_bytes;                 // none needed so far
    GN_TRY(check_shape(g, me, err, err_len));
    if (!(eps >= 1.17549435e-38f) || !std::isfinite(eps)) return op_fail(err, err_len, RFAST_EINVAL, "%s: eps must be at least 2^-126", me);
    GnArgs a{};
    a.s = shape_from(g, eps);
    GN_TRY(strides_of(x_strides, a.s, &a.xn, &a.xs, me, "x", err, err_len));
    GN_TRY(strides_of(y_strides, a.s, &a.on, &a.os, me, "y", err, err_len));
    if (a.s.N == 0 || a.s.S == 0) return RFAST_OK;
    if (overlaps(a.s, a.on, a.os)) return op_fail(err, err_len, RFAST_EINVAL, "%s: the strides of y make it overlap itself", me);
    const void* ptrs[] = {d_x, d_gamma, d_beta, d_y, d_mean, d_rstd};
    const char* names[] = {"x", "gamma", "beta", "y", "mean", "rstd"};
    const int es = type_bytes(g->type);
    for (int k = 0; k < 6; ++k) {
        if (!ptrs[k]) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s is null", me, names[k]);
        if ((uintptr_t)ptrs[k] % (k == 0 || k == 3 ? es : 4)) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s is not aligned to its type", me, names[k]);
    }
    for (int k = 0; k < 6; ++k) GN_TRY(check_device_pointer(ptrs[k], names[k], err, err_len));
    a.x = d_x; a.out = d_y; a.gamma = d_gamma; a.beta = d_beta; a.affine_stride = a.s.C; a.mean = d_mean; a.rstd = d_rstd;
    const int vx = allowed(d_x, a.xn, a.xs, es), vy = allowed(d_y, a.on, a.os, es);
    a.p = make_plan(a.s, es, vx < vy ? vx : vy, false);
    if (a.p.items * a.p.cluster > 0x7fffffff || a.p.slabs > 65535) return op_fail(err, err_len, RFAST_EINVAL, "%s: too many samples or groups", me);
    const cudaError_t e = launch_typed(a, g->type, false, (cudaStream_t)cuda_stream);
    if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
    return RFAST_OK;
}

extern "C" int rfast_group_norm_backward(const rfast_gn_shape* g, const void* d_dy, const int64_t* dy_strides, const void* d_x, const int64_t* x_strides,
                                         const float* d_gamma, const float* d_beta, const float* d_mean, const float* d_rstd, void* d_dx,
                                         const int64_t* dx_strides, float* d_dgamma, float* d_dbeta, void* workspace, size_t workspace_bytes,
                                         void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_group_norm_backward";
    GN_TRY(check_shape(g, me, err, err_len));
    GnArgs a{};
    a.s = shape_from(g, 1.f);
    GN_TRY(strides_of(x_strides, a.s, &a.xn, &a.xs, me, "x", err, err_len));
    GN_TRY(strides_of(dy_strides, a.s, &a.dn, &a.ds, me, "dy", err, err_len));
    GN_TRY(strides_of(dx_strides, a.s, &a.on, &a.os, me, "dx", err, err_len));
    if (a.s.N == 0) return RFAST_OK;                        // no sets either
    const int64_t sets = a.s.N / a.s.per_set;
    if (a.s.S > 0 && overlaps(a.s, a.on, a.os)) return op_fail(err, err_len, RFAST_EINVAL, "%s: the strides of dx make it overlap itself", me);
    const void* ptrs[] = {d_dgamma, d_dbeta, d_gamma, d_beta, d_mean, d_rstd, d_dy, d_x, d_dx};
    const char* names[] = {"dgamma", "dbeta", "gamma", "beta", "mean", "rstd", "dy", "x", "dx"};
    const int es = type_bytes(g->type);
    const int count = a.s.S > 0 ? 9 : 2;
    for (int k = 0; k < count; ++k) {
        if (!ptrs[k]) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s is null", me, names[k]);
        if ((uintptr_t)ptrs[k] % (k >= 6 ? es : 4)) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s is not aligned to its type", me, names[k]);
    }
    if (a.s.S > 0) {
        const int64_t need = rfast_group_norm_workspace(g, 1);
        if (!workspace || (uintptr_t)workspace % 4 || (int64_t)workspace_bytes < need)
            return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace needs %lld bytes, aligned to 4", me, (long long)need);
        GN_TRY(check_device_pointer(workspace, "workspace", err, err_len));
    }
    for (int k = 0; k < count; ++k) GN_TRY(check_device_pointer(ptrs[k], names[k], err, err_len));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (a.s.S == 0) {                                       // sums over nothing
        e = cudaMemsetAsync(d_dgamma, 0, sets * a.s.C * sizeof(float), st);
        if (e == cudaSuccess) e = cudaMemsetAsync(d_dbeta, 0, sets * a.s.C * sizeof(float), st);
        return e == cudaSuccess ? RFAST_OK : op_fail(err, err_len, RFAST_ECUDA, "%s: %s", me, cudaGetErrorString(e));
    }
    a.x = d_x; a.dy = d_dy; a.out = d_dx; a.gamma = d_gamma; a.beta = d_beta; a.affine_stride = a.s.C;
    a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
    a.dgamma = d_dgamma; a.dbeta = d_dbeta; a.part = (float*)workspace;
    int v = allowed(d_x, a.xn, a.xs, es);
    const int v2 = allowed(d_dy, a.dn, a.ds, es), v3 = allowed(d_dx, a.on, a.os, es);
    v = v < v2 ? v : v2;
    v = v < v3 ? v : v3;
    a.p = make_plan(a.s, es, v, true);
    if (a.p.slabs > 65535 || sets > 65535) return op_fail(err, err_len, RFAST_EINVAL, "%s: too many groups or sets", me);
    e = launch_typed(a, g->type, true, st);
    if (e == cudaSuccess && a.p.parts * a.p.cluster > 1) {
        k_gn_affine<<<dim3((a.s.C + 31) / 32, (unsigned)sets), kT, 0, st>>>(a.part, (int)(a.p.parts * a.p.cluster), a.s.C, d_dgamma, d_dbeta);
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
    return RFAST_OK;
}
