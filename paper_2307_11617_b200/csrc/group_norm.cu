// Group norm with an activation, channels last, forward and backward (see rfast_group_norm in rfast.h
// for the formulas).
//
// A thread keeps its column of V neighbouring channels and walks down the positions, so that all that belongs to a
// channel -- sums, scale, shift -- sits in its registers.  A thread block's columns make up a slab, the smallest run
// of whole groups that is at least 128 bytes wide.  There are two ways through a sample's slab:
//   - one thread block takes it whole (or several samples' where they have few positions).  What a thread has read for the
//     sums waits in shared memory: asynchronous copies that only this thread reads back, so no barrier guards them;
//   - slabs that are too large for that, or too few to fill the GPU, are cut into equal chunks of positions, as many as thread
//     blocks run at a time: one launch for the chunks' sums, one that merges them and goes over the values again, from the
//     last position to the first, so that the L2 cache serves what it still holds (32 x 3136 x 256 bf16 backward, x and dy
//     103 MB: the second launch reads 48 MB from memory, in the order of the first 87 MB).
// Measured and dropped, all for 32 x 3136 x 256 bf16 and against 31 us forward and 48 us backward (before sigmoid2 bounded its argument,
// which costs 0.5 and 0.8 us):
//   - spans of equal length over slabs laid end to end, which give every SM the same work: a block whose span holds the end
//     of a slab and the start of the next sets up and sums up twice, and the launch waits for it (36 and 84 us);
//   - a cluster of thread blocks that keep a slab in their shared memory and merge its sums there: loading, summing and
//     writing then follow one another on the whole GPU (37 and 122 us);
//   - wider slabs: 256 bytes 31 and 52 us, 512 bytes 32 and 52 us (2 x 16384 x 320 f16: 17 us at 128 bytes, 23 and 34 us);
//   - smaller chunks, half as many again: 35 and 57 us.
//
// Variances do not come from a difference of two large sums: a thread sums deviations from the first value it
// sees in each channel, and its mean and sum of squared deviations are merged with the others' by the parallel
// form of the two-pass formula (Chan, Golub, LeVeque).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdio>
#include <type_traits>

#include "ops.h"
#include "pairs.cuh"

namespace rfast {

namespace {

constexpr int kT = 256;                                    // threads per block
constexpr int kRingPairs = 3;                              // pairs of rows that a thread's ring holds

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

// pairs of V channels; a single channel has a zero beside it
template <int V> constexpr int kPairs = (V + 1) / 2;

__device__ __forceinline__ F2 widen2(uint32_t r, const __nv_bfloat16*) { return pair(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u)); }
__device__ __forceinline__ F2 widen2(uint32_t r, const __half*) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&r));
    return pair(a.x, a.y);
}
__device__ __forceinline__ void widen(Vec<float, 4> v, F2 (&f)[2]) {
    f[0] = pair(__uint_as_float(v.w.x), __uint_as_float(v.w.y));
    f[1] = pair(__uint_as_float(v.w.z), __uint_as_float(v.w.w));
}
__device__ __forceinline__ void widen(Vec<float, 1> v, F2 (&f)[1]) { f[0] = pair(__uint_as_float(v.w), 0.f); }
template <class T>
__device__ __forceinline__ void widen(Vec<T, 8> v, F2 (&f)[4]) {
    const T* t = nullptr;
    f[0] = widen2(v.w.x, t); f[1] = widen2(v.w.y, t); f[2] = widen2(v.w.z, t); f[3] = widen2(v.w.w, t);
}
template <class T>
__device__ __forceinline__ void widen(Vec<T, 2> v, F2 (&f)[1]) { f[0] = widen2(v.w, (const T*)nullptr); }
template <class T>
__device__ __forceinline__ void widen(Vec<T, 1> v, F2 (&f)[1]) { f[0] = widen2((uint32_t)v.w, (const T*)nullptr); }
__device__ __forceinline__ uint32_t narrow2(F2 f, const __nv_bfloat16*) {
    float a, b;
    split(f, a, b);
    const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t narrow2(F2 f, const __half*) {
    float a, b;
    split(f, a, b);
    const __half2 r = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
}
// V is the number of channels, the pairs holding that many
template <int V, class T>
__device__ __forceinline__ void store_vec(T* p, const F2 (&f)[kPairs<V>]) {
    if constexpr (sizeof(T) == 4) {
        float q[2 * kPairs<V>];
#pragma unroll
        for (int k = 0; k < kPairs<V>; ++k) split(f[k], q[2 * k], q[2 * k + 1]);
        if constexpr (V == 4) __stcs(reinterpret_cast<float4*>(p), make_float4(q[0], q[1], q[2], q[3]));
        else __stcs(p, q[0]);
    } else if constexpr (V == 8) {
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(narrow2(f[0], p), narrow2(f[1], p), narrow2(f[2], p), narrow2(f[3], p)));
    } else if constexpr (V == 2) {
        __stcs(reinterpret_cast<uint32_t*>(p), narrow2(f[0], p));
    } else {
        __stcs(reinterpret_cast<unsigned short*>(p), (unsigned short)narrow2(f[0], p));
    }
}
template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// until at most `left` of the youngest groups are on their way
__device__ __forceinline__ void copies_wait(int left) {
    switch (left) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    }
}

template <int LEFT> __device__ __forceinline__ void copies_pending() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// 1 / (1 + exp(-u)) of a pair.  2^t and the reciprocal are the hardware's (2 ulp and 1 ulp), t = -u log2(e) carries the roundings of
// the constant and of the product, and the products after it one each: the result is good to 2^-22 + |u| 2^-23.  The special
// function unit, with a result every other cycle where the adders have eight, is what bounds a pass with this in it, so one
// reciprocal, of the product of both denominators, serves two values (3 instead of 4 of its operations per pair).  To keep the
// product in range exp(-u) stops growing at 2^60, below u = -41.6.  u comes back bounded there as well: u / (1 + exp(-u)) and the
// slope are then between -4e-17 and 0 however far u is, and not u 2^-60.  A NaN gives 2^-60: it must not reach its neighbour
// through the product, and the caller multiplies by u, in which it stays.  e: exp(-u)
__device__ __forceinline__ F2 sigmoid2(F2& u, F2& e) {
    float a, b;
    split(u, a, b);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(-41.58883f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(b) : "f"(-41.58883f));
    u = pair(a, b);
    split(u * both(-1.4426950408889634f), a, b);
    asm("min.f32 %0, %0, %1;" : "+f"(a) : "f"(60.f));        // a NaN's
    asm("min.f32 %0, %0, %1;" : "+f"(b) : "f"(60.f));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    e = pair(a, b);
    split(e + both(1.f), a, b);
    float r = a * b;
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r));
    return pair(b, a) * both(r);
}
__device__ __forceinline__ F2 silu2(F2 u) { F2 e; const F2 q = sigmoid2(u, e); return u * q; }

// cnt rows of a thread out of shared memory, R at a time: all loads of a batch go out before the first row is worked on.
template <int R, class Row, class Load, class Use>
__device__ __forceinline__ void walk(int cnt, Load load, Use use) {
    int r = 0;
#pragma unroll 1
    for (; r + R <= cnt; r += R) {
        Row q[R];
#pragma unroll
        for (int k = 0; k < R; ++k) q[k] = load();
#pragma unroll
        for (int k = 0; k < R; ++k) use(q[k]);
    }
#pragma unroll 1
    for (; r < cnt; ++r) { Row q = load(); use(q); }
}
// The same out of memory, through a ring of 2 PAIRS slots in shared memory that only this thread uses: `fetch(slot)` starts the
// asynchronous copies of the next row into a slot, `held(slot)` reads one.  What is on its way costs no registers, so there can be
// enough of it: rows fetched ahead into registers left 40 to 50 KB on their way in an SM, and 4 TB/s.  (Two pairs: backward 50 us in the
// place of 48; four: forward 31.2 in the place of 30.8 us, see the kernels for the shape, and above for what came after.)
template <int PAIRS> struct Ring {
    int in, sent;
    template <class Fetch> __device__ __forceinline__ void send(int cnt, Fetch& fetch) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (sent < cnt) { fetch(in); in = in + 1 == 2 * PAIRS ? 0 : in + 1; ++sent; }
        copies_commit();
    }
    template <class Fetch> __device__ __forceinline__ void begin(int cnt, Fetch& fetch) {
        in = sent = 0;
        for (int k = 0; k < PAIRS - 1; ++k) send(cnt, fetch);
    }
    template <class Row, class Fetch, class Held, class Use> __device__ __forceinline__ void run(int cnt, Fetch& fetch, Held held, Use use) {
        int out = 0, r = 0;
        // while all that a turn of the ring fetches and uses exists, its slots are constants
        constexpr int kTurn = 2 * PAIRS;
#pragma unroll 1
        for (; r + kTurn + 2 * (PAIRS - 1) <= cnt; r += kTurn) {
#pragma unroll
            for (int p = 0; p < PAIRS; ++p) {
                fetch((2 * p + 2 * (PAIRS - 1)) % kTurn);
                fetch((2 * p + 2 * (PAIRS - 1) + 1) % kTurn);
                copies_commit();
                copies_pending<PAIRS - 1>();
                Row q[2];
                q[0] = held(2 * p);
                q[1] = held(2 * p + 1);
                use(q[0]);
                use(q[1]);
            }
            sent += kTurn;
        }
#pragma unroll 1
        for (; r < cnt; r += 2) {
            send(cnt, fetch);
            copies_pending<PAIRS - 1>();
            Row q[2];
            q[0] = held(out);
            q[1] = held(out + 1);                            // past the last row: what lay there, unused
            out = out + 2 == 2 * PAIRS ? 0 : out + 2;
            use(q[0]);
            if (r + 1 < cnt) use(q[1]);
        }
    }
};
// Where accesses are too narrow for copies: a batch's loads go out before the batch ahead of it is worked on (its stores would hold them back,
// the operands being allowed to coincide), the first batch's as early as the caller likes.
template <int R, class Row> struct Ahead {
    Row q[R];
    template <class Load> __device__ __forceinline__ void begin(int cnt, Load& load) {
#pragma unroll
        for (int k = 0; k < R; ++k) if (k < cnt) q[k] = load();
    }
    template <class Load, class Use> __device__ __forceinline__ void run(int cnt, Load& load, Use use) {
        int r = 0;
#pragma unroll 1
        for (; r + 2 * R <= cnt; r += R) {
            Row n[R];
#pragma unroll
            for (int k = 0; k < R; ++k) n[k] = load();
#pragma unroll
            for (int k = 0; k < R; ++k) use(q[k]);
#pragma unroll
            for (int k = 0; k < R; ++k) q[k] = n[k];
        }
        const int left = cnt - r;                            // fewer than 2 R; the first R of them are here
        Row n[R - 1];
#pragma unroll
        for (int k = 0; k < R - 1; ++k) if (R + k < left) n[k] = load();
#pragma unroll
        for (int k = 0; k < R; ++k) if (k < left) use(q[k]);
#pragma unroll
        for (int k = 0; k < R - 1; ++k) if (R + k < left) use(n[k]);
    }
};

// ---- geometry, chosen on the host -------------------------------------------------------------------
// Quotients of numbers below 2^16 by a divisor that the host knows: one multiplication.  m = floor(2^32 / d) + 1 overshoots
// 2^32 / d by at most 1, so the product's high word is exact while n d < 2^32.
struct Divisor {
    uint32_t m;                        // 0: d = 1
    int d;
    __host__ void set(int64_t v) { d = (int)v; m = v == 1 ? 0u : (uint32_t)(((uint64_t)1 << 32) / (uint64_t)v + 1); }
    __device__ __forceinline__ unsigned of(unsigned n) const { return m ? __umulhi(n, m) : n; }
};
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
    int chunks;                        // of a slab's positions; 0: one launch, a thread block taking whole slabs
    int rows;                          // positions of a chunk
    int each, more;                    // one launch: positions per thread, the first `more` rows of threads one more
    Divisor by_tx, by_tr, by_gs, by_cg, by_unit;    // by_unit: entries of a group in one row of threads
    int rpt;                           // positions per thread (buffered)
    bool buffered;                     // what was read waits in shared memory
    int64_t items;                     // one launch: items per set (forward: over all samples)
    int64_t parts;                     // one launch, backward: thread blocks that share a set's items
    size_t buf;                        // bytes of the buffer
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
    float4* gpart;                     // chunks: [N][G][chunks] count, mean and squared deviations, or the two sums of the backward pass
    float* part;                       // backward: rows of [2][C], du and du h summed; a row per thread block of a set or per
                                       // sample and chunk
    int64_t n0;                        // chunks: first sample of this launch
};

// A thread block's task: everything in one launch (what it reads kept in shared memory, or read twice where that is too small
// or accesses are too narrow), the sums over a chunk, or what follows from them.
enum { kWhole = 0, kSums = 1, kApply = 2, kReread = 3 };

__device__ __forceinline__ const float* affine_row(const GnArgs& a, const float* base, int64_t set) {
    const int64_t row = a.set_row ? (int64_t)a.set_row[set * a.set_row_stride] : set;
    return base + row * a.affine_stride;
}

// What a thread is in its block: column, sample of the item, first position; the same for both directions.
struct Seat {
    int txi, sl, rr;                   // column of threads, sample within the item, row of the sample's threads
    int rows;                          // one launch: positions of this thread
    bool on;
};
__device__ __forceinline__ Seat seat_of(const GnPlan& p) {
    Seat s;
    const unsigned tyi = p.by_tx.of(threadIdx.x);
    s.txi = threadIdx.x - tyi * p.tx;
    s.sl = p.by_tr.of(tyi);
    s.rr = tyi - s.sl * p.tr;
    s.on = s.sl < p.ns;
    s.rows = s.on ? p.each + (s.rr < p.more ? 1 : 0) : 0;
    return s;
}

// What a thread block has before it: all positions of a slab, or a chunk of them.
struct Part {
    int64_t n;                         // (first) sample
    int slab;
    int64_t from;                      // chunks: positions [from, from + count)
    int count;
    int piece;                         // which chunk
};
// Chunks come on x, slabs on y, samples on z; BACK: from the end.
template <bool BACK>
__device__ __forceinline__ Part part_of(const GnArgs& a) {
    Part q;
    q.piece = BACK ? a.p.chunks - 1 - (int)blockIdx.x : blockIdx.x;
    q.slab = blockIdx.y;
    q.n = a.n0 + (BACK ? gridDim.z - 1 - blockIdx.z : blockIdx.z);
    q.from = (int64_t)q.piece * a.p.rows;
    const int64_t left = a.s.S - q.from;
    q.count = left < a.p.rows ? (int)left : a.p.rows;
    return q;
}
__device__ __forceinline__ int rows_of(int count, int rr, int tr) { return rr < count ? (int)((unsigned)(count - rr - 1) / (unsigned)tr) + 1 : 0; }

// scale or shift of V neighbouring channels
template <int V>
__device__ __forceinline__ void affine_of(const float* p, bool quads, F2 (&f)[kPairs<V>]) {
    if constexpr (V % 4 == 0) {
        if (quads) {
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                const float4 q = *reinterpret_cast<const float4*>(p + k);
                f[k / 2] = pair(q.x, q.y);
                f[k / 2 + 1] = pair(q.z, q.w);
            }
            return;
        }
    }
#pragma unroll
    for (int k = 0; k < V; k += 2) f[k / 2] = pair(p[k], k + 1 < V ? p[k + 1] : 0.f);
}
// groups of V neighbouring channels from channel c on: one (WHOLE) or one per channel
template <int V, bool WHOLE>
__device__ __forceinline__ void groups_of(int c, const Divisor& by_cg, int (&g)[WHOLE ? 1 : V]) {
    const int cg = by_cg.d;
    int q = by_cg.of(c);
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
// kWhole, kReread: grid = (items, slabs).  kSums, kApply: grid = (chunks, slabs, samples of the launch).
// 32 x 3136 x 256 bf16 with u / (1 + exp(-u)): 31.7 us, 3.2 TB/s of x read and y written once; 26.9 us without an activation.  The
// sums take 11 us of it whether x comes from memory or from the L2 cache, the second launch 20 us: its 51 MB of writes
// alone take 14 us (a plain fill does), the special function unit is busy for 9 us, and what is in the way is that all blocks
// merge and set up at the same time.  Registers for two blocks per SM, four where a group's channels fill accesses (2 x 16384 x
// 320 f16, ten channels a group: 17.0 us with two, 18.6 us with three, now 17.7; 32 x 3136 x 256 bf16: 31.4 us with two, 30.8 us with
// four).  Samples that one block takes whole wait for their one load and several barriers, with nothing on its way meanwhile:
// 8192 x 30 x 48 fp32 62 us (135 backward) where the bytes take 15 (22), 4096 x 4 x 512 fp32 60 us (118) where they take 10 (16).
template <class T, int V, bool WHOLE, int TASK>
__global__ void __launch_bounds__(kT, WHOLE ? 4 : 2)
k_gn_forward(const __grid_constant__ GnArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    typedef Vec<T, V> X;
    const GnShape& s = a.s;
    const GnPlan& p = a.p;
    constexpr bool BUF = TASK == kWhole, kOne = TASK == kWhole || TASK == kReread;
    constexpr int kBatch = 4, kP = kPairs<V>, kGv = WHOLE ? 1 : V, kGp = WHOLE ? 1 : kP, kAcc = WHOLE ? (kP < 2 ? 1 : 2) : kP;
    X* buf = reinterpret_cast<X*>(smem);
    // per thread (WHOLE: an access stays inside a group) or per thread and channel: count, mean, sum of squared deviations
    constexpr int width = kGv, kEnt = TASK == kApply ? 0 : kT;
    constexpr bool RING = !BUF && sizeof(X) >= 4;
    constexpr int kPairsAhead = kRingPairs;
    X* ring = buf + threadIdx.x;
    float* e_n = reinterpret_cast<float*>(smem + p.buf);
    float* e_mean = e_n + kEnt;
    float* e_m2 = e_mean + kEnt * width;
    const int nb = p.ns * p.gs;
    float2* fin = reinterpret_cast<float2*>(e_m2 + kEnt * width);      // [nb] mean, rstd
    const Seat me = seat_of(p);
    const int64_t rows_on = TASK == kApply ? -p.tr : p.tr;   // from row to row of a thread
    const int64_t step = rows_on * a.xs, ostep = rows_on * a.os;
    if (TASK == kSums) asm volatile("griddepcontrol.launch_dependents;");
    {
        Part part;
        if (kOne) { part.n = (int64_t)blockIdx.x * p.ns; part.slab = blockIdx.y; part.from = 0; part.piece = 0; }
        else part = part_of<TASK == kApply>(a);
        const int slab = part.slab, gs = min(p.gs, s.G - slab * p.gs);      // the last slab may be narrower
        const int64_t n = part.n + me.sl;                    // this thread's sample, positions and the first of them
        const int cnt = kOne ? (n < s.N ? me.rows : 0) : me.on ? rows_of(part.count, me.rr, p.tr) : 0;
        const int64_t r0 = part.from + me.rr + (TASK == kApply ? (cnt - 1) * (int64_t)p.tr : 0);
        const int c0 = slab * p.W, cols = gs * s.Cg / V;
        const T* x = (const T*)a.x + n * a.xn + r0 * a.xs + c0;
        const T* px = x + me.txi * V;                        // of the pass over the width that is under way
        auto load = [&]() { const X q = load_vec<T, V>(px); px += step; return q; };
        auto fetch = [&](int slot) { copy_async<sizeof(X)>(ring + slot * kT, px); px += step; };
        auto waiting = [&](int slot) { return ring[slot * kT]; };
        typename std::conditional<RING, Ring<kPairsAhead>, Ahead<kBatch, X>>::type rows;
        auto begin = [&]() { if constexpr (RING) rows.begin(cnt, fetch); else rows.begin(cnt, load); };

        if constexpr (TASK != kApply) {
            // what is read comes in up to four lots of rows; the first is worked on while the others are on their way
            const int lot = BUF ? (cnt + 3) / 4 : cnt;
            if (BUF) {
                for (int j = 0; j < p.cj; ++j) {
                    const int cv = me.txi + j * kT;
                    if (cv < cols) {
                        const T* from = x + cv * V;
                        X* to = buf + j * p.rpt * kT + threadIdx.x;
                        int r = 0;
                        for (int k = 0; k < 4; ++k) {
                            for (const int stop = min(cnt, r + lot); r < stop; ++r, from += step, to += kT) copy_async<sizeof(X)>(to, from);
                            if (p.cj == 1) copies_commit();
                        }
                    }
                }
                if (p.cj > 1) { copies_commit(); copies_wait(0); }
            }
            // count, mean and squared deviations of what this thread holds
            float t_n = 0.f, t_mean = 0.f, t_m2 = 0.f;
            for (int j = 0; j < p.cj; ++j) {
                const int cv = me.txi + j * kT;
                F2 first[kGp], s1[kAcc], s2[kAcc];           // the first value, negated
#pragma unroll
                for (int v = 0; v < kAcc; ++v) s1[v] = s2[v] = both(0.f);
                float mean[2 * kGp], m2[2 * kGp];
#pragma unroll
                for (int v = 0; v < 2 * kGp; ++v) mean[v] = m2[v] = 0.f;
                if (cnt > 0 && cv < cols) {
                    const X* bt = buf + j * p.rpt * kT + threadIdx.x;
                    X x0;
                    if constexpr (BUF) {
                        if (p.cj == 1) copies_wait(3);
                        x0 = *bt;
                    } else {
                        px = x + cv * V;
                        x0 = load_vec<T, V>(px);
                        begin();
                    }
                    {
                        F2 f[kP];
                        widen(x0, f);
#pragma unroll
                        for (int v = 0; v < kGp; ++v) {
                            float lo, hi;
                            split(f[v], lo, hi);
                            mean[2 * v] = lo;
                            mean[2 * v + 1] = WHOLE ? lo : hi;
                            first[v] = pair(-lo, WHOLE ? -lo : -hi);
                        }
                    }
                    auto use = [&](const X& q) {             // a first value counts as a deviation of 0
                        F2 f[kP];
                        widen(q, f);
#pragma unroll
                        for (int v = 0; v < kP; ++v) {
                            const F2 d = f[v] + first[WHOLE ? 0 : v];
                            s1[v % kAcc] = s1[v % kAcc] + d;
                            s2[v % kAcc] = fma2(d, d, s2[v % kAcc]);
                        }
                    };
                    if constexpr (BUF) {
                        auto held = [&]() { const X q = *bt; bt += kT; return q; };
                        if (p.cj == 1) {
                            for (int k = 0, r = 0; k < 4; ++k, r += lot) {
                                if (k) copies_wait(3 - k);
                                walk<kBatch, X>(min(cnt - r, lot), held, use);
                            }
                        } else {
                            walk<kBatch, X>(cnt, held, use);
                        }
                    } else if constexpr (RING) {
                        rows.template run<X>(cnt, fetch, waiting, use);
                    } else {
                        rows.run(cnt, load, use);
                    }
                    if (WHOLE) {
                        if (kAcc == 2) { s1[0] = s1[0] + s1[kAcc - 1]; s2[0] = s2[0] + s2[kAcc - 1]; }
                        float lo, hi;
                        split(s1[0], lo, hi);
                        s1[0] = both(V > 1 ? lo + hi : lo);
                        split(s2[0], lo, hi);
                        s2[0] = both(V > 1 ? lo + hi : lo);
                    }
                    const float nn = (float)cnt * (WHOLE ? V : 1), inv = __frcp_rn(nn);
#pragma unroll
                    for (int v = 0; v < kGp; ++v) {
                        float a1[2], a2[2];
                        split(s1[v], a1[0], a1[1]);
                        split(s2[v], a2[0], a2[1]);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float d = a1[k] * inv;
                            m2[2 * v + k] = fmaxf(fmaf(-a1[k], d, a2[k]), 0.f) + (a2[k] - a2[k]);   // the second term is a NaN where there was one
                            mean[2 * v + k] += d;
                        }
                    }
                    if (WHOLE && t_n > 0.f) {                // a further pass over a wide group
                        const float d = mean[0] - t_mean, tot = t_n + nn;
                        t_mean += d * (nn / tot);
                        t_m2 += m2[0] + d * d * (t_n * nn / tot);
                        t_n = tot;
                    } else {
                        t_mean = mean[0]; t_m2 = m2[0]; t_n = nn;
                    }
                }
                if (!WHOLE) {                                // a slab of several groups is never wider than the block
                    if (me.on && cv < cols) {
#pragma unroll
                        for (int v = 0; v < kGv; ++v) { e_mean[threadIdx.x * V + v] = mean[v]; e_m2[threadIdx.x * V + v] = m2[v]; }
                    }
                }
            }
            e_n[threadIdx.x] = t_n;
            if (WHOLE) { e_mean[threadIdx.x] = t_mean; e_m2[threadIdx.x] = t_m2; }
            __syncthreads();
            // the groups' sums over this block, a team of lanes per group
            const int unit = WHOLE ? min(s.Cg / V, p.tx) : s.Cg;    // entries of a group in one row of threads
            const int entries = unit * p.tr, L = team_size(entries), lane = threadIdx.x & (L - 1);
            for (int b0 = 0; b0 < nb; b0 += kT / L) {
                const int b = b0 + threadIdx.x / L;
                const int sl = p.ns > 1 ? (int)p.by_gs.of(b) : 0, g = b - sl * p.gs;
                const bool in = b < nb && g < gs;
                // means are summed as differences from one of them: a flat group has exactly its level
                const float ref = in ? e_mean[sl * p.tr * p.tx * width + g * unit] : 0.f;
                float cn = 0.f, cm = 0.f;
                for (int q = lane; in && q < entries; q += L) {
                    const int row = p.by_unit.of(q), t = (sl * p.tr + row) * p.tx, u = g * unit + (q - row * unit);
                    const float k = e_n[t + (WHOLE ? u : u / V)];
                    cn += k;
                    if (k > 0.f) cm = fmaf(k, e_mean[t * width + u] - ref, cm);
                }
                cn = team_sum(cn, L);
                cm = team_sum(cm, L);
                const float mean = cn > 0.f ? ref + cm / cn : 0.f;
                float m2 = 0.f;
                for (int q = lane; in && q < entries; q += L) {
                    const int row = p.by_unit.of(q), t = (sl * p.tr + row) * p.tx, u = g * unit + (q - row * unit);
                    const float k = e_n[t + (WHOLE ? u : u / V)];
                    if (k > 0.f) {
                        const float d = e_mean[t * width + u] - mean;
                        m2 += fmaf(k * d, d, e_m2[t * width + u]);
                    }
                }
                m2 = team_sum(m2, L);
                if (in && lane == 0) {
                    const int64_t to = (part.n + sl) * s.G + slab * p.gs + g;
                    if (TASK == kSums) {
                        a.gpart[to * p.chunks + part.piece] = make_float4(cn, mean, m2, 0.f);
                    } else {
                        const float rstd = rsqrtf(m2 / ((float)s.S * (float)s.Cg) + s.eps);
                        fin[b] = make_float2(mean, rstd);
                        if (part.n + sl < s.N) { a.mean[to] = mean; a.rstd[to] = rstd; }
                    }
                }
            }
            if (TASK == kSums) return;
        } else {
            if (cnt > 0 && me.txi < cols) begin();           // on their way while the sums are merged
            asm volatile("griddepcontrol.wait;" ::: "memory");
            // a team of lanes per group
            const int L = team_size(p.chunks), lane = threadIdx.x & (L - 1);
            const float all = (float)s.S * (float)s.Cg;
            for (int b0 = 0; b0 < gs; b0 += kT / L) {
                const int g = b0 + threadIdx.x / L;
                const bool in = g < gs;
                const int64_t to = part.n * s.G + slab * p.gs + g;
                const float4* q = a.gpart + to * p.chunks;
                const float4 mine = in && lane < p.chunks ? q[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
                const float ref = __shfl_sync(0xffffffffu, mine.y, threadIdx.x & 31 & ~(L - 1));
                float cm = mine.x * (mine.x > 0.f ? mine.y - ref : 0.f);
                for (int k = lane + L; in && k < p.chunks; k += L) { const float4 v = q[k]; cm = fmaf(v.x, v.y - ref, cm); }
                const float mean = ref + team_sum(cm, L) / all;
                float d = mine.y - mean, m2 = mine.x > 0.f ? fmaf(mine.x * d, d, mine.z) : 0.f;
                for (int k = lane + L; in && k < p.chunks; k += L) { const float4 v = q[k]; d = v.y - mean; m2 += fmaf(v.x * d, d, v.z); }
                m2 = team_sum(m2, L);
                if (in && lane == 0) {
                    const float rstd = rsqrtf(m2 / all + s.eps);
                    fin[g] = make_float2(mean, rstd);
                    if (part.piece == 0) { a.mean[to] = mean; a.rstd[to] = rstd; }
                }
            }
        }
        __syncthreads();
        if (cnt > 0) {
            const int64_t set = (unsigned)n / (unsigned)s.per_set;      // both below 2^31
            const float* gam = affine_row(a, a.gamma, set) + c0;
            const float* bet = affine_row(a, a.beta, set) + c0;
            T* y = (T*)a.out + n * a.on + r0 * a.os + c0;
            for (int j = 0; j < p.cj; ++j) {
                const int cv = me.txi + j * kT;
                if (cv >= cols) break;
                if constexpr (!BUF) { if (kOne || j > 0) { px = x + cv * V; begin(); } }
                F2 mean[kGp], mul[kP], add[kP];              // the mean, negated
                int g[kGv];
                groups_of<V, WHOLE>(cv * V, p.by_cg, g);
                affine_of<V>(gam + cv * V, a.quads, mul);
                affine_of<V>(bet + cv * V, a.quads, add);
                const float2* f = fin + me.sl * p.gs;
                if (WHOLE) {
                    const float2 q = f[g[0]];
                    mean[0] = both(-q.x);
#pragma unroll
                    for (int v = 0; v < kP; ++v) mul[v] = mul[v] * both(q.y);
                } else {
#pragma unroll
                    for (int v = 0; v < kP; ++v) {
                        const float2 q = f[g[2 * v]], r = f[g[(2 * v + 1) % kGv]];
                        mean[v] = pair(-q.x, -r.x);
                        mul[v] = mul[v] * pair(q.y, r.y);
                    }
                }
                const X* bt = buf + j * p.rpt * kT + threadIdx.x;
                T* to = y + cv * V;
                auto use = [&](const X& q) {
                    F2 o[kP];
                    widen(q, o);
#pragma unroll
                    for (int v = 0; v < kP; ++v) o[v] = fma2(o[v] + mean[WHOLE ? 0 : v], mul[v], add[v]);
                    if (s.act == RFAST_ACT_SILU) {
#pragma unroll
                        for (int v = 0; v < kP; ++v) o[v] = silu2(o[v]);
                    } else if (s.act == RFAST_ACT_RELU) {
#pragma unroll
                        for (int v = 0; v < kP; ++v) {
                            float lo, hi;
                            split(o[v], lo, hi);
                            o[v] = pair(lo < 0.f ? 0.f : lo, hi < 0.f ? 0.f : hi);       // a NaN stays one
                        }
                    }
                    store_vec<V>(to, o);
                    to += ostep;
                };
                if constexpr (BUF) walk<kBatch, X>(cnt, [&]() { const X q = *bt; bt += kT; return q; }, use);
                else if constexpr (RING) rows.template run<X>(cnt, fetch, waiting, use);
                else rows.run(cnt, load, use);
            }
        }
    }
}

// ---- backward -------------------------------------------------------------------------------------
// dy act'(u)
__device__ __forceinline__ F2 through(int act, F2 u, F2 dy) {
    if (act == RFAST_ACT_SILU) {
        F2 e;
        const F2 q = sigmoid2(u, e);
        return dy * fma2(q, q * e * u, q);                   // q (1 + u (1 - q)); q e has the digits that 1 - q loses at large u
    }
    if (act == RFAST_ACT_RELU) {
        float a, b, c, d;
        split(u, a, b);
        split(dy, c, d);
        return pair(a > 0.f ? c : 0.f, b > 0.f ? d : 0.f);
    }
    return dy;
}
template <class X> struct Pair { X x, d; };
// A thread's fp32 values of a row, kept between the passes: 16 bytes (or 8) per thread and plane, so that a warp's
// accesses spread over all banks.
template <int P> struct alignas(P >= 2 ? 16 : 8) Plane { F2 f[P >= 2 ? 2 : 1]; };
template <int P> constexpr int kPlanes = P >= 4 ? P / 2 : 1;
template <int P>
__device__ __forceinline__ void put(Plane<P>* at, const F2 (&f)[P]) {
#pragma unroll
    for (int k = 0; k < kPlanes<P>; ++k) {
        Plane<P> q;
#pragma unroll
        for (int v = 0; v < (P >= 2 ? 2 : 1); ++v) q.f[v] = f[2 * k + v];
        at[k * kT] = q;
    }
}
template <int P>
__device__ __forceinline__ void get(const Plane<P>* at, F2 (&f)[P]) {
#pragma unroll
    for (int k = 0; k < kPlanes<P>; ++k) {
        const Plane<P> q = at[k * kT];
#pragma unroll
        for (int v = 0; v < (P >= 2 ? 2 : 1); ++v) f[2 * k + v] = q.f[v];
    }
}

// dgamma, dbeta of 32 channels of a set from the set's rows of sums, by a thread block, in a fixed order, in 64 bits.
__device__ __forceinline__ void affine_sums(const float* part, int64_t rows, int C, int64_t set, int c32, float* dgamma, float* dbeta) {
    __shared__ double sh[2][kT / 32][32];
    const int lane = threadIdx.x & 31, c = c32 * 32 + lane, w = threadIdx.x >> 5;
    const float* base = part + set * rows * 2 * C + c;
    double b = 0.0, g = 0.0;
    if (c < C) {
#pragma unroll 4
        for (int64_t r = w; r < rows; r += kT / 32) {
            b += (double)base[r * 2 * C];
            g += (double)base[r * 2 * C + C];
        }
    }
    __syncthreads();                                         // a block may have several turns
    sh[0][w][lane] = b;
    sh[1][w][lane] = g;
    __syncthreads();
    if (w < 2 && c < C) {
        double u = 0.0;
        for (int k = 0; k < kT / 32; ++k) u += sh[w][k][lane];
        (w ? dgamma : dbeta)[set * C + c] = (float)u;
    }
}
// grid = (channels / 32, sets)
__global__ void __launch_bounds__(kT)
k_gn_affine(const float* __restrict__ part, int64_t rows, int C, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    affine_sums(part, rows, C, blockIdx.y, blockIdx.x, dgamma, dbeta);
}

// With du = dy act'(u), h = (x - mean) rstd, and over the M values of a group
//     one = sum gamma du / M, two = sum gamma du h / M:   dx = rstd (gamma du - one - two h);
// per channel dbeta = sum du, dgamma = sum du h over the samples of a set.
// kWhole, kReread: grid = (parts, slabs, sets); a block takes every `parts`-th item of a set, keeps the channels' sums of its items in
// shared memory and, buffered, du in fp32 in the place of dy, so that the second pass has no exponentials.
// kSums, kApply: grid = (chunks, slabs, samples of the launch), the last kApply with one slab more, whose blocks form dgamma and dbeta
// meanwhile.
// 32 x 3136 x 256 bf16: 49 us, 3.1 TB/s of x and dy read and dx written once, 42 us without an activation.  Bound by the arithmetic of
// a row (about 100 instructions for 8 channels) and its latency: the sums take as long with half of x and dy in the L2 cache.  So registers for two
// blocks per SM, in which two rows' work interleaves: 48 us against 51 us with three (before the bound of sigmoid2).
template <class T, int V, bool WHOLE, int TASK>
__global__ void __launch_bounds__(kT, 2)
k_gn_backward(const __grid_constant__ GnArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    typedef Vec<T, V> X;
    const GnShape& s = a.s;
    const GnPlan& p = a.p;
    constexpr bool BUF = TASK == kWhole, kOne = TASK == kWhole || TASK == kReread;
    constexpr int kBatch = BUF ? 2 : 3, kP = kPairs<V>, kGv = WHOLE ? 1 : V, kGp = WHOLE ? 1 : kP;
    typedef Plane<kP> K;
    constexpr int kRow = kPlanes<kP> * kT;                   // planes of a row, one after the other
    X* bufx = reinterpret_cast<X*>(smem);
    K* bufd = reinterpret_cast<K*>(smem + (size_t)p.rpt * p.cj * kT * sizeof(X));      // dy in the first plane, then du
    constexpr bool RING = !BUF && sizeof(X) >= 4;
    constexpr int kPairsAhead = kRingPairs;
    X* ring = bufx + threadIdx.x;                            // slots of x and dy
    const int nb = p.ns * p.gs;
    const int wide = min(p.W, kT * V);                       // channels of one pass over the width
    const int across = p.tr > 1 ? max(kT, p.ns * wide) : 0;
    float* ent = reinterpret_cast<float*>(smem + p.buf);     // [2][kT * V]: du, du h of a thread's channels
    float* col = ent + (TASK == kApply ? 0 : 2 * kT * V);    // [2][across]: the same, summed down the positions
    float2* sums = reinterpret_cast<float2*>(col + (TASK == kApply ? 0 : 2 * across));     // [nb] the groups' two sums
    float* acc = reinterpret_cast<float*>(sums + nb);        // [2][W]: dbeta, dgamma of the block's items

    if (TASK == kApply && blockIdx.y == (unsigned)p.slabs) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        const int64_t rows = s.per_set * p.chunks;
        const unsigned tiles = (s.C + 31) / 32, sets = (unsigned)s.N / (unsigned)s.per_set;
        for (unsigned t = blockIdx.x + blockIdx.z * gridDim.x; t < tiles * sets; t += gridDim.x * gridDim.z)
            affine_sums(a.part, rows, s.C, t / tiles, (int)(t % tiles), a.dgamma, a.dbeta);
        return;
    }
    if (TASK == kSums) asm volatile("griddepcontrol.launch_dependents;");
    const Seat me = seat_of(p);
    const int64_t rows_on = TASK == kApply ? -p.tr : p.tr;   // from row to row of a thread
    const int64_t xstep = rows_on * a.xs, dstep = rows_on * a.ds, ostep = rows_on * a.os;
    const float inv_m = 1.f / ((float)s.S * (float)s.Cg);
    if (TASK != kApply)
        for (int c = threadIdx.x; c < 2 * p.W; c += kT) acc[c] = 0.f;

    for (int64_t item = kOne ? blockIdx.x : 0; item < (kOne ? p.items : 1); item += kOne ? p.parts : 1) {
        Part part;
        int64_t in_set = 0;                                  // one launch: this thread's sample within its set
        if (kOne) {
            part.slab = blockIdx.y; part.from = 0; part.piece = 0;
            in_set = item * p.ns + me.sl;
            part.n = (int64_t)blockIdx.z * s.per_set + in_set;
        } else {
            part = part_of<TASK == kApply>(a);
        }
        const int slab = part.slab, gs = min(p.gs, s.G - slab * p.gs), W = gs * s.Cg;      // the last slab may be narrower
        const int64_t n = part.n;                             // this thread's sample
        const int64_t set = kOne ? (int64_t)blockIdx.z : (int64_t)((unsigned)n / (unsigned)s.per_set);
        const int c0 = slab * p.W, cols = W / V;
        const float* gam = affine_row(a, a.gamma, set) + c0;
        const float* bet = affine_row(a, a.beta, set) + c0;
        const int cnt = kOne ? (in_set < s.per_set ? me.rows : 0) : me.on ? rows_of(part.count, me.rr, p.tr) : 0;
        const int64_t r0 = part.from + me.rr + (TASK == kApply ? (cnt - 1) * (int64_t)p.tr : 0);      // its first position
        const T* x = (const T*)a.x + n * a.xn + r0 * a.xs + c0;
        const T* dy = (const T*)a.dy + n * a.dn + r0 * a.ds + c0;
        const T *px = x + me.txi * V, *pd = dy + me.txi * V;  // of the pass over the width that is under way
        auto load = [&]() {
            Pair<X> q;
            q.x = load_vec<T, V>(px);
            q.d = load_vec<T, V>(pd);
            px += xstep; pd += dstep;
            return q;
        };
        auto fetch = [&](int slot) {
            copy_async<sizeof(X)>(ring + 2 * slot * kT, px);
            copy_async<sizeof(X)>(ring + (2 * slot + 1) * kT, pd);
            px += xstep; pd += dstep;
        };
        auto waiting = [&](int slot) { Pair<X> q; q.x = ring[2 * slot * kT]; q.d = ring[(2 * slot + 1) * kT]; return q; };
        typename std::conditional<RING, Ring<kPairsAhead>, Ahead<kBatch, Pair<X>>>::type rows;
        auto begin = [&]() { if constexpr (RING) rows.begin(cnt, fetch); else rows.begin(cnt, load); };
        if constexpr (!BUF) { if (cnt > 0 && me.txi < cols) begin(); }       // on their way before anything else
        if constexpr (TASK != kApply) {
            const int lot = BUF ? (cnt + 3) / 4 : cnt;       // rows of a group of copies
            if (BUF) {
                for (int j = 0; j < p.cj; ++j) {
                    const int cv = me.txi + j * kT;
                    if (cv < cols) {
                        const T *ax = x + cv * V, *ad = dy + cv * V;
                        X* tx = bufx + j * p.rpt * kT + threadIdx.x;
                        K* td = bufd + j * p.rpt * kRow + threadIdx.x;
                        int r = 0;
                        for (int k = 0; k < 4; ++k) {
                            for (const int stop = min(cnt, r + lot); r < stop; ++r, ax += xstep, ad += dstep, tx += kT, td += kRow) {
                                copy_async<sizeof(X)>(tx, ax);
                                copy_async<sizeof(X)>(td, ad);
                            }
                            if (p.cj == 1) copies_commit();
                        }
                    }
                }
                if (p.cj > 1) { copies_commit(); copies_wait(0); }
            }
            for (int b = threadIdx.x; b < nb; b += kT) sums[b] = make_float2(0.f, 0.f);
            for (int j = 0; j < p.cj; ++j) {
                const int cv = me.txi + j * kT;
                F2 s_du[kP], s_dh[kP];
#pragma unroll
                for (int v = 0; v < kP; ++v) s_du[v] = s_dh[v] = both(0.f);
                if (cnt > 0 && cv < cols) {
                    F2 mean[kGp], rs[kGp], mul[kP], add[kP]; // u = (x - mean) mul + add; the mean, negated
                    int g[kGv];
                    groups_of<V, WHOLE>(cv * V, p.by_cg, g);
                    affine_of<V>(gam + cv * V, a.quads, mul);
                    affine_of<V>(bet + cv * V, a.quads, add);
                    const float *pm = a.mean + n * s.G + slab * p.gs, *pr = a.rstd + n * s.G + slab * p.gs;
#pragma unroll
                    for (int v = 0; v < kGp; ++v) {
                        const int g0 = g[WHOLE ? 0 : 2 * v], g1 = g[WHOLE ? 0 : (2 * v + 1) % kGv];
                        mean[v] = pair(-pm[g0], -pm[g1]);
                        rs[v] = pair(pr[g0], pr[g1]);
                    }
#pragma unroll
                    for (int v = 0; v < kP; ++v) mul[v] = mul[v] * rs[WHOLE ? 0 : v];
                    const X* bx = bufx + j * p.rpt * kT + threadIdx.x;
                    K* bd = bufd + j * p.rpt * kRow + threadIdx.x;
                    K* keep = bd;
                    auto held = [&]() {
                        Pair<X> q;
                        q.x = *bx;
                        q.d = *reinterpret_cast<const X*>(bd);
                        bx += kT; bd += kRow;
                        return q;
                    };
                    auto use = [&](const Pair<X>& q) {
                        F2 d[kP], du[kP];
                        widen(q.x, d);
                        widen(q.d, du);
#pragma unroll
                        for (int v = 0; v < kP; ++v) {
                            d[v] = d[v] + mean[WHOLE ? 0 : v];
                            du[v] = through(s.act, fma2(d[v], mul[v], add[v]), du[v]);
                            s_du[v] = s_du[v] + du[v];
                            s_dh[v] = fma2(du[v], d[v], s_dh[v]);
                        }
                        if (BUF) { put<kP>(keep, du); keep += kRow; }
                    };
                    if constexpr (BUF) {
                        if (p.cj == 1) {
                            for (int k = 0, r = 0; k < 4; ++k, r += lot) {
                                copies_wait(3 - k);
                                walk<kBatch, Pair<X>>(min(cnt - r, lot), held, use);
                            }
                        } else {
                            walk<kBatch, Pair<X>>(cnt, held, use);
                        }
                    } else {
                        if (j > 0) { px = x + cv * V; pd = dy + cv * V; begin(); }
                        if constexpr (RING) rows.template run<Pair<X>>(cnt, fetch, waiting, use);
                        else rows.run(cnt, load, use);
                    }
#pragma unroll
                    for (int v = 0; v < kP; ++v) s_dh[v] = s_dh[v] * rs[WHOLE ? 0 : v];     // h = (x - mean) rstd
                }
                // [row of threads][channel of this pass]
                if (me.on) {
                    float *e0 = ent + threadIdx.x * V, *e1 = e0 + kT * V;
                    if constexpr (V == 1) {
                        float z;
                        split(s_du[0], *e0, z);
                        split(s_dh[0], *e1, z);
                    } else {
#pragma unroll
                        for (int v = 0; v < kP; v += (kP >= 2 ? 2 : 1)) {
                            K k0, k1;
#pragma unroll
                            for (int u = 0; u < (kP >= 2 ? 2 : 1); ++u) { k0.f[u] = s_du[v + u]; k1.f[u] = s_dh[v + u]; }
                            *reinterpret_cast<K*>(e0 + 2 * v) = k0;
                            *reinterpret_cast<K*>(e1 + 2 * v) = k1;
                        }
                    }
                }
                __syncthreads();
                const int pw = min(p.tx * V, W - j * kT * V);    // channels of this pass
                const int pitch = p.tx * V;
                const float *q0 = ent, *q1 = ent + kT * V;
                int qp = pitch;                              // floats between a sample's rows
                if (p.tr > 1) {
                    // down the rows of threads, `ways` threads per channel, then their sums, in fixed order
                    const int nc = p.ns * pw, ways = nc >= kT ? 1 : min(kT / nc, p.tr);
                    float *c0s = col, *c1s = col + across;
                    for (int i = threadIdx.x; i < nc * ways; i += kT) {
                        const int w = ways > 1 ? (unsigned)i / (unsigned)nc : 0, k = i - w * nc, sl = p.ns > 1 ? (unsigned)k / (unsigned)pw : 0;
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
                        if ((int)threadIdx.x < nc) {         // nc < kT: one channel per thread
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
                    const int sl = p.ns > 1 ? (int)p.by_gs.of(b) : 0, g = b - sl * p.gs;
                    const bool in = b < nb && g < gs;
                    if (in) {
                        for (int q = lane; q < unit; q += L) {
                            const int c = g * unit + q;
                            const float ga = gam[j * kT * V + c];
                            u0 = fmaf(ga, q0[sl * qp + c], u0);
                            u1 = fmaf(ga, q1[sl * qp + c], u1);
                        }
                    }
                    u0 = team_sum(u0, L);
                    u1 = team_sum(u1, L);
                    if (in && lane == 0) { sums[b].x += u0; sums[b].y += u1; }
                }
                __syncthreads();                             // before the next pass or item fills `ent`
            }
            if (TASK == kSums) {
                for (int g = threadIdx.x; g < gs; g += kT) {
                    const float2 q = sums[g];
                    a.gpart[(n * s.G + slab * p.gs + g) * p.chunks + part.piece] = make_float4(q.x, q.y, 0.f, 0.f);
                }
                float* to = a.part + (n * p.chunks + part.piece) * 2 * s.C + c0;        // the channels' sums
                for (int c = threadIdx.x; c < W; c += kT) {
                    to[c] = acc[c];
                    to[s.C + c] = acc[p.W + c];
                }
                return;
            }
        } else {
            asm volatile("griddepcontrol.wait;" ::: "memory");
            // merge the chunks, a team of lanes per group
            const int L = team_size(p.chunks), lane = threadIdx.x & (L - 1);
            for (int b0 = 0; b0 < gs; b0 += kT / L) {
                const int g = b0 + threadIdx.x / L;
                float u0 = 0.f, u1 = 0.f;
                if (g < gs) {
                    const float4* q = a.gpart + (n * s.G + slab * p.gs + g) * p.chunks;
                    for (int k = lane; k < p.chunks; k += L) { const float4 v = q[k]; u0 += v.x; u1 += v.y; }
                }
                u0 = team_sum(u0, L);
                u1 = team_sum(u1, L);
                if (g < gs && lane == 0) sums[g] = make_float2(u0, u1);
            }
            __syncthreads();
        }
        if (cnt > 0) {
            T* dx = (T*)a.out + n * a.on + r0 * a.os + c0;
            for (int j = 0; j < p.cj; ++j) {
                const int cv = me.txi + j * kT;
                if (cv >= cols) break;
                if constexpr (!BUF) { if (kOne || j > 0) { px = x + cv * V; pd = dy + cv * V; begin(); } }
                F2 mean[kGp], k1[kGp], k2[kGp], mul[kP], add[kP];   // dx = mul du - k1 - (x - mean) k2; all but mul and add negated
                int g[kGv];
                groups_of<V, WHOLE>(cv * V, p.by_cg, g);
                affine_of<V>(gam + cv * V, a.quads, mul);
                if (!BUF) affine_of<V>(bet + cv * V, a.quads, add);
                const float *pm = a.mean + n * s.G + slab * p.gs, *pr = a.rstd + n * s.G + slab * p.gs;
                const float2* q = sums + me.sl * p.gs;
#pragma unroll
                for (int v = 0; v < kGp; ++v) {
                    const int g0 = g[WHOLE ? 0 : 2 * v], g1 = g[WHOLE ? 0 : (2 * v + 1) % kGv];
                    const F2 rs = pair(pr[g0], pr[g1]);
                    mean[v] = pair(-pm[g0], -pm[g1]);
                    k1[v] = rs * pair(-inv_m * q[g0].x, -inv_m * q[g1].x);
                    k2[v] = rs * rs * pair(-inv_m * q[g0].y, -inv_m * q[g1].y);
                    if (!WHOLE) mul[v] = mul[v] * rs;
                    else {
#pragma unroll
                        for (int u = 0; u < kP; ++u) mul[u] = mul[u] * rs;
                    }
                }
                const X* bx = bufx + j * p.rpt * kT + threadIdx.x;
                const K* bd = bufd + j * p.rpt * kRow + threadIdx.x;
                T* to = dx + cv * V;
                auto last = [&](F2 (&d)[kP], F2 (&du)[kP]) {  // d: x - mean
#pragma unroll
                    for (int v = 0; v < kP; ++v) du[v] = fma2(du[v], mul[v], fma2(d[v], k2[WHOLE ? 0 : v], k1[WHOLE ? 0 : v]));
                    store_vec<V>(to, du);
                    to += ostep;
                };
                if constexpr (BUF) {
                    struct Held { X x; F2 d[kP]; };
                    walk<kBatch, Held>(cnt, [&]() { Held h; h.x = *bx; get<kP>(bd, h.d); bx += kT; bd += kRow; return h; }, [&](Held& h) {
                        F2 d[kP];
                        widen(h.x, d);
#pragma unroll
                        for (int v = 0; v < kP; ++v) d[v] = d[v] + mean[WHOLE ? 0 : v];
                        last(d, h.d);
                    });
                } else {
                    auto use = [&](const Pair<X>& h) {
                        F2 d[kP], du[kP];
                        widen(h.x, d);
                        widen(h.d, du);
#pragma unroll
                        for (int v = 0; v < kP; ++v) {
                            d[v] = d[v] + mean[WHOLE ? 0 : v];
                            du[v] = through(s.act, fma2(d[v], mul[v], add[v]), du[v]);
                        }
                        last(d, du);
                    };
                    if constexpr (RING) rows.template run<Pair<X>>(cnt, fetch, waiting, use);
                    else rows.run(cnt, load, use);
                }
            }
        }
        if (!kOne) return;
        __syncthreads();                                     // `sums` may be filled again
    }
    if constexpr (kOne) {
        const int slab = blockIdx.y, c0 = slab * p.W, W = min(p.gs, s.G - slab * p.gs) * s.Cg;
        const int64_t set = blockIdx.z;
        float *to0, *to1;                                    // dbeta, dgamma
        if (p.parts == 1) {
            to0 = a.dbeta + set * s.C + c0;
            to1 = a.dgamma + set * s.C + c0;
        } else {
            to0 = a.part + (set * p.parts + blockIdx.x) * 2 * s.C + c0;
            to1 = to0 + s.C;
        }
        for (int c = threadIdx.x; c < W; c += kT) {
            to0[c] = acc[c];
            to1[c] = acc[p.W + c];
        }
    }
}

// ---- one position per sample ----------------------------------------------------------------------
// The rows of a hidden layer: a team of lanes takes a sample's group, K accesses per lane, and everything that belongs to
// it stays in their registers; no barrier until the channels' sums of the backward pass are added up at the very end.
// A block has teams for `gt` neighbouring groups (128 bytes and more) of `sp` samples and walks down the samples; in the
// forward pass neighbouring ones, so that it reads a set's scale and shift once (every block taking every 592nd row of teams:
// 4096 x 2048 fp32, 64 sets, 44 us in the place of 15).
// A lane holds 8 channels, 4 accesses where a team of 32 lanes with 8 each does not cover the group.  4096 x 512 fp32 in 16
// groups, 64 sets: 7.0 us forward, 7.5 us backward; the general path, whose blocks hold 32 samples and meet at five barriers for
// them, takes 15 and 39 us.  32768 x 512 fp32: 32 and 51 us with one set (4.2 and 3.9 TB/s), 45 and 50 us with 512; what bounds these is
// not settled: a second turn of loads ahead gains nothing forward.  16-bit loads of the backward pass go out two turns ahead and
// registers are for two blocks of an SM (32768 x 512 bf16, one set: 33 us; one turn and three blocks: 44 us).  With 4
// channels per lane 4096 x 512 fp32 takes 7.2 and 7.7 us; with 16 of 16-bit types the registers spill (bf16 backward 13 us
// in the place of 7).  Groups of 264 to 1024 channels of 16-bit types have 32 channels per lane, and these kernels do spill (96 bytes forward, 152
// backward): 4096 x 4096 bf16 in 8 groups 32 and 58 us, where the bytes take 10 and 16.  Groups of 16-bit types that are no multiple
// of 8 channels are not in rows at all: 4096 x 640 bf16 in 32 groups 78 and 62 us, the same layer in fp32 9 and 16.
// 4096 x 2048 fp32 in 4 groups, 64 sets: 18 us, 3.7 TB/s, and 33 us backward, 3.1 TB/s; the general path takes 60 and 146 us.
constexpr int kRowChannels = 8;
template <int V, int K, bool BACKWARD> constexpr int kRowBlocks = BACKWARD ? K * V <= kRowChannels ? 2 : 1 : K == 1 ? 4 : K == 2 ? 3 : 2;
struct RowPlan {
    int L, gt, sp, slabs;              // lanes of a team, groups and samples of a block, blocks across the groups
    int parts;                         // blocks down the samples (backward: of a set)
    int turns;                         // forward: of a block
    Divisor by_gt;
};

template <class T, int V, int K>
struct RowSeat {
    int lane, sp, g;
    bool on;
    int64_t c;                         // first channel of the lane's first access
    int left;                          // accesses of the lane that exist
    __device__ __forceinline__ RowSeat(const GnShape& s, const RowPlan& r) {
        lane = threadIdx.x & (r.L - 1);
        const unsigned team = threadIdx.x / (unsigned)r.L;
        sp = r.by_gt.of(team);
        g = blockIdx.y * r.gt + (team - sp * r.gt);
        on = sp < r.sp && g < s.G;
        c = (int64_t)g * s.Cg + lane * V;
        left = on ? (s.Cg / V - lane + r.L - 1) / r.L : 0;
    }
};

// grid = (parts, slabs); all lanes of a warp go through every turn, the shuffles being the warp's
template <class T, int V, int K>
__global__ void __launch_bounds__(kT, kRowBlocks<V, K, false>)
k_gn_rows_forward(const __grid_constant__ GnArgs a, const __grid_constant__ RowPlan r) {
    const GnShape& s = a.s;
    typedef Vec<T, V> X;
    constexpr int kP = kPairs<V>;
    const RowSeat<T, V, K> me(s, r);
    const float inv = 1.f / (float)s.Cg;
    F2 mul[K][kP], add[K][kP];
    int64_t set = -1;
    X q[K], next[K];
    // neighbouring samples, whose sets are few
    const int64_t jump = r.sp, from = (int64_t)blockIdx.x * r.turns * r.sp, stop = min(s.N, from + (int64_t)r.turns * r.sp);
    auto load = [&](int64_t n, X (&to)[K]) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < me.left && n < stop) to[k] = load_vec<T, V>((const T*)a.x + n * a.xn + me.c + (int64_t)k * r.L * V);
    };
    load(from + me.sp, q);
    for (int64_t base = from; base < stop; base += jump) {
        const int64_t n = base + me.sp;
        load(n + jump, next);
        const int left = n < stop ? me.left : 0;
        if (left && (int64_t)((unsigned)n / (unsigned)s.per_set) != set) {
            set = (unsigned)n / (unsigned)s.per_set;
            const float *gam = affine_row(a, a.gamma, set) + me.c, *bet = affine_row(a, a.beta, set) + me.c;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (k < left) { affine_of<V>(gam + k * r.L * V, a.quads, mul[k]); affine_of<V>(bet + k * r.L * V, a.quads, add[k]); }
        }
        // deviations from the group's first value: a flat group has exactly its level
        F2 d[K][kP];
        float ref, other;
        widen(q[0], d[0]);
        split(d[0][0], ref, other);
        ref = __shfl_sync(0xffffffffu, ref, threadIdx.x & 31 & ~(r.L - 1));
        F2 sum = both(0.f);
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < left) {
                if (k) widen(q[k], d[k]);
#pragma unroll
                for (int v = 0; v < kP; ++v) { d[k][v] = d[k][v] + both(-ref); sum = sum + d[k][v]; }
            }
        float lo, hi;
        split(sum, lo, hi);
        const float off = team_sum(lo + hi, r.L) * inv;      // mean - ref
        sum = both(0.f);
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < left) {
#pragma unroll
                for (int v = 0; v < kP; ++v) { d[k][v] = d[k][v] + both(-off); sum = fma2(d[k][v], d[k][v], sum); }
            }
        split(sum, lo, hi);
        const float rstd = rsqrtf(fmaf(team_sum(lo + hi, r.L), inv, s.eps));
        if (left && me.lane == 0) { a.mean[n * s.G + me.g] = ref + off; a.rstd[n * s.G + me.g] = rstd; }
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < left) {
                F2 o[kP];
#pragma unroll
                for (int v = 0; v < kP; ++v) o[v] = fma2(d[k][v], mul[k][v] * both(rstd), add[k][v]);
                if (s.act == RFAST_ACT_SILU) {
#pragma unroll
                    for (int v = 0; v < kP; ++v) o[v] = silu2(o[v]);
                } else if (s.act == RFAST_ACT_RELU) {
#pragma unroll
                    for (int v = 0; v < kP; ++v) {
                        split(o[v], lo, hi);
                        o[v] = pair(lo < 0.f ? 0.f : lo, hi < 0.f ? 0.f : hi);
                    }
                }
                store_vec<V>((T*)a.out + n * a.on + me.c + (int64_t)k * r.L * V, o);
            }
#pragma unroll
        for (int k = 0; k < K; ++k) q[k] = next[k];
    }
}

// grid = (parts, slabs, sets); dynamic shared memory: [2][kT * K * V] floats
template <class T, int V, int K>
__global__ void __launch_bounds__(kT, kRowBlocks<V, K, true>)
k_gn_rows_backward(const __grid_constant__ GnArgs a, const __grid_constant__ RowPlan r) {
    extern __shared__ __align__(16) uint8_t smem[];
    const GnShape& s = a.s;
    typedef Vec<T, V> X;
    constexpr int kP = kPairs<V>;
    const RowSeat<T, V, K> me(s, r);
    const int64_t set = blockIdx.z;
    const float *gam = affine_row(a, a.gamma, set) + me.c, *bet = affine_row(a, a.beta, set) + me.c;
    const float inv = -1.f / (float)s.Cg;
    F2 ga[K][kP], be[K][kP], s_du[K][kP], s_dh[K][kP];
    constexpr int kAhead = K == 1 ? 2 : 1;                 // turns whose values are on their way while a lane works on one
    Pair<X> q[kAhead + 1][K];                                // this turn's values, then the following ones'
    float means[kAhead + 1], rstds[kAhead + 1];
    const int64_t jump = (int64_t)gridDim.x * r.sp, end = (set + 1) * s.per_set;
    auto load = [&](int64_t n, Pair<X> (&to)[K], float& m, float& t) {
        if (n < end && me.left) {
            m = a.mean[n * s.G + me.g];
            t = a.rstd[n * s.G + me.g];
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (k < me.left) {
                    to[k].x = load_vec<T, V>((const T*)a.x + n * a.xn + me.c + (int64_t)k * r.L * V);
                    to[k].d = load_vec<T, V>((const T*)a.dy + n * a.dn + me.c + (int64_t)k * r.L * V);
                }
        }
    };
    const int64_t first = set * s.per_set + (int64_t)blockIdx.x * r.sp;
#pragma unroll
    for (int t = 0; t <= kAhead; ++t) means[t] = rstds[t] = 0.f;
#pragma unroll
    for (int t = 0; t < kAhead; ++t) load(first + me.sp + t * jump, q[t], means[t], rstds[t]);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (k < me.left) { affine_of<V>(gam + k * r.L * V, a.quads, ga[k]); affine_of<V>(bet + k * r.L * V, a.quads, be[k]); }
#pragma unroll
        for (int v = 0; v < kP; ++v) s_du[k][v] = s_dh[k][v] = both(0.f);
    }
    for (int64_t base = first; base < end; base += jump) {
        const int64_t n = base + me.sp;
        load(n + kAhead * jump, q[kAhead], means[kAhead], rstds[kAhead]);
        const int left = n < end ? me.left : 0;
        const float mean = means[0], rs = rstds[0];
        F2 h[K][kP], du[K][kP], one = both(0.f), two = both(0.f);
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < left) {
                widen(q[0][k].x, h[k]);
                widen(q[0][k].d, du[k]);
#pragma unroll
                for (int v = 0; v < kP; ++v) {
                    h[k][v] = (h[k][v] + both(-mean)) * both(rs);
                    du[k][v] = through(s.act, fma2(h[k][v], ga[k][v], be[k][v]), du[k][v]);
                    s_du[k][v] = s_du[k][v] + du[k][v];
                    s_dh[k][v] = fma2(du[k][v], h[k][v], s_dh[k][v]);
                    du[k][v] = du[k][v] * ga[k][v];
                    one = one + du[k][v];
                    two = fma2(du[k][v], h[k][v], two);
                }
            }
        float lo, hi;
        split(one, lo, hi);
        const float s1 = team_sum(lo + hi, r.L) * inv;       // both negated
        split(two, lo, hi);
        const float s2 = team_sum(lo + hi, r.L) * inv;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < left) {
                F2 o[kP];
#pragma unroll
                for (int v = 0; v < kP; ++v) o[v] = (fma2(h[k][v], both(s2), du[k][v]) + both(s1)) * both(rs);
                store_vec<V>((T*)a.out + n * a.on + me.c + (int64_t)k * r.L * V, o);
            }
#pragma unroll
        for (int t = 0; t < kAhead; ++t) {
#pragma unroll
            for (int k = 0; k < K; ++k) q[t][k] = q[t + 1][k];
            means[t] = means[t + 1];
            rstds[t] = rstds[t + 1];
        }
    }
    // the channels' sums of the block's teams: [sample's row of teams][group of the block][channel]
    float* sh0 = reinterpret_cast<float*>(smem);
    float* sh1 = sh0 + r.sp * r.gt * s.Cg;
    const int width = r.gt * s.Cg, mine = me.sp * width + (me.g - blockIdx.y * r.gt) * s.Cg + me.lane * V;
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k < me.left) {
#pragma unroll
            for (int v = 0; v < kP; ++v) {
                const int at = mine + k * r.L * V + 2 * v;
                split(s_du[k][v], sh0[at], sh0[at + 1]);
                split(s_dh[k][v], sh1[at], sh1[at + 1]);
            }
        }
    __syncthreads();
    const int have = min(r.gt, s.G - (int)blockIdx.y * r.gt) * s.Cg, c0 = blockIdx.y * width;
    float *to0, *to1;
    if (gridDim.x == 1) {
        to0 = a.dbeta + set * s.C + c0;
        to1 = a.dgamma + set * s.C + c0;
    } else {
        to0 = a.part + (set * gridDim.x + blockIdx.x) * 2 * s.C + c0;
        to1 = to0 + s.C;
    }
    for (int c = threadIdx.x; c < have; c += kT) {
        float u0 = 0.f, u1 = 0.f;
        for (int k = 0; k < r.sp; ++k) { u0 += sh0[k * width + c]; u1 += sh1[k * width + c]; }
        to0[c] = u0;
        to1[c] = u1;
    }
}

// ---- host side ------------------------------------------------------------------------------------
constexpr int kSms = 148;
constexpr int kMaxGroupChannels = 8192;                     // a block keeps two sums for every channel of a group
constexpr size_t kMostSmem = 220 * 1024;
// Into how many chunks the positions of slabs of W channels are cut; 0: not at all.  They are where a slab does not fit the buffer
// (backward: x and du in fp32), or where there are fewer than SMs and each takes longer than a microsecond or two to read.  There
// are as many as thread blocks run at a time, of 32 positions and 8 KB at least.
int chunks_of(const GnShape& s, int esize, int W, int slabs, bool whole, bool backward) {
    const int64_t item = s.S * W * esize, items = s.N * slabs;
    if (s.S < 64 || (item <= (backward ? 32 * 1024 : 64 * 1024) && (items >= kSms || item <= 16 * 1024))) return 0;
    const int64_t at_a_time = (backward ? 2 : whole ? 4 : 2) * kSms;
    int64_t chunks = at_a_time / items;
    if (chunks > item / (8 * 1024)) chunks = item / (8 * 1024);
    if (chunks > s.S / 32) chunks = s.S / 32;
    const int64_t least = (s.S + 0x3fffffff) / 0x40000000;   // a chunk's positions are counted in 32 bits
    return (int)(chunks < least ? least : chunks);
}

// One launch: blocks that share a set's sums at most.
int64_t part_rows(const GnShape& s) {
    const int64_t sets = s.N / s.per_set;
    int64_t cap = 2048 / sets;
    cap = cap < 16 ? 16 : cap > 256 ? 256 : cap;
    return cap < s.per_set ? cap : s.per_set;
}

// the rings of a plan that is not buffered (accesses of four bytes and more)
size_t ring_bytes(int V, int esize, bool backward) { return V * esize >= 4 ? (size_t)2 * kRingPairs * kT * V * esize * (backward ? 2 : 1) : 0; }

size_t smem_bytes(const GnShape& s, const GnPlan& p, bool backward, int task) {
    const size_t nb = (size_t)p.ns * p.gs;
    if (!backward) {
        const size_t width = s.Cg % p.V == 0 ? 1 : p.V;
        return p.buf + (task == kApply ? 0 : sizeof(float) * (kT + 2 * kT * width)) + sizeof(float2) * nb;
    }
    const size_t wide = p.W < kT * p.V ? p.W : kT * p.V;
    const size_t across = p.tr > 1 ? (p.ns * wide > kT ? p.ns * wide : (size_t)kT) : 0;
    if (task == kApply) return p.buf + sizeof(float2) * nb;
    return p.buf + sizeof(float) * (2 * (size_t)kT * p.V + 2 * across + 2 * (size_t)p.W) + sizeof(float2) * nb;
}

// vmax: channels per access that addresses and strides allow (a power of two, times the type at most 16 bytes)
GnPlan make_plan(const GnShape& s, int esize, int vmax, bool backward) {
    GnPlan p{};
    int V = vmax;
    // an access may straddle narrow groups, but a slab has to hold whole accesses
    const bool broad = s.Cg * esize >= 128;
    if (broad) { while (s.Cg % V) V /= 2; } else { while (s.C % V) V /= 2; }
    if (V * esize == 8) V /= 2;                             // accesses of 16, 4 or 2 bytes
    p.V = V;
    p.gs = broad ? 1 : s.G;
    if (!broad) {
        int unit = 1;                                       // groups that hold whole accesses
        while (unit < s.G && unit * s.Cg % V) ++unit;
        for (int gs = unit; gs < s.G; gs += unit)
            if (gs * s.Cg * esize >= 128) { p.gs = gs; break; }
        // A narrower last slab leaves its blocks with little to do.  Where samples alone are blocks enough, a width of less than two
        // slabs is one: 128 samples x 1881 x 96 f16 in 32 groups, no activation, 32 us, backward 42 against 58 with two slabs (72 and 24
        // channels); 5 samples 16 against 12.6 us, wide slabs of few samples having many chunks to merge.  At the border 31 samples with
        // two slabs take 17.0 and 19.7 us, 32 with one 16.5 and 17.3.  (Three even slabs in the place of four, 200 channels in 25
        // groups: 128 samples x 1881 backward 111 against 94 us.)
        if (s.N >= 32 && s.S > 1 && s.G % p.gs && s.C * esize < 256) p.gs = s.G;
    }
    p.W = p.gs * s.Cg;
    p.slabs = (s.G + p.gs - 1) / p.gs;
    const int cols = p.W / V;
    p.tx = cols < kT ? cols : kT;
    p.cj = (cols + kT - 1) / kT;
    const int ty = kT / p.tx;
    p.tr = (int)(s.S < ty ? s.S : ty);
    p.ns = 1;
    p.parts = 1;
    const int unit = s.Cg % V == 0 ? s.Cg / V : s.Cg;
    p.by_tx.set(p.tx); p.by_tr.set(p.tr); p.by_gs.set(p.gs); p.by_cg.set(s.Cg); p.by_unit.set(unit < p.tx || s.Cg % V ? unit : p.tx);
    p.buf = ring_bytes(V, esize, backward);
    p.chunks = chunks_of(s, esize, p.W, p.slabs, s.Cg % V == 0, backward);
    if (p.chunks) {
        p.rows = (int)((s.S + p.chunks - 1) / p.chunks);
        p.chunks = (int)((s.S + p.rows - 1) / p.rows);      // none is empty
        return p;
    }
    p.each = (int)(s.S / p.tr); p.more = (int)(s.S % p.tr);
    const int64_t batch = backward ? s.per_set : s.N;
    const int64_t ns = ty / p.tr;
    p.ns = (int)(ns > batch ? batch : ns);
    p.items = (batch + p.ns - 1) / p.ns;
    if (backward) {
        const int64_t most = part_rows(s);
        p.parts = p.items < most ? p.items : most;
    }
    if (V * esize >= 4) {
        const int64_t rpt = (s.S + p.tr - 1) / p.tr;
        GnPlan q = p;
        q.buffered = true;
        q.buf = (size_t)(rpt * p.cj * kT * (V * esize + (backward ? 8 * ((V + 1) / 2) : 0)));   // x, and du in pairs
        q.rpt = (int)rpt;
        if (smem_bytes(s, q, backward, kWhole) <= kMostSmem) return q;
    }
    return p;
}

// Bytes of the workspace for a plan: the groups' partial sums, then the channels' rows.
size_t group_bytes(const GnShape& s, const GnPlan& p) { return p.chunks ? (size_t)s.N * s.G * p.chunks * sizeof(float4) : 0; }
size_t row_bytes(const GnShape& s, const GnPlan& p) { return (size_t)(p.chunks ? s.N * p.chunks : s.N / s.per_set * part_rows(s)) * 2 * s.C * sizeof(float); }
// The most that any plan of the shape takes, whatever addresses and strides allow.
size_t workspace_bytes_of(const GnShape& s, int esize, bool backward) {
    size_t most = 0;
    for (int v = 1; v * esize <= 16; v *= 2) {
        const GnPlan p = make_plan(s, esize, v, backward);
        const size_t b = group_bytes(s, p) + (backward ? row_bytes(s, p) : 0);
        if (b > most) most = b;
    }
    return most;
}

template <class K>
cudaError_t launch_task(K kernel, dim3 grid, const GnArgs& a, size_t smem, bool follows, cudaStream_t st) {
    if (smem > 48 * 1024) {                                 // a limit; the same for every call, so that threads may launch side by side
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid; cfg.blockDim = dim3(kT); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute at{};                               // the launch after the sums is on its way while they are formed
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = follows ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

// One position per sample, groups of whole accesses, 128 of them at most.
bool in_rows(const GnShape& s, int V, int esize) { return s.S == 1 && V * esize == 16 && s.Cg % V == 0 && s.Cg / V <= 128; }

template <class T, int V, int K>
cudaError_t launch_rows(GnArgs& a, bool backward, cudaStream_t st) {
    const GnShape& s = a.s;
    const int64_t sets = s.N / s.per_set, batch = backward ? s.per_set : s.N;
    RowPlan r{};
    r.L = 1;
    while (r.L * K < s.Cg / V) r.L *= 2;
    const int teams = kT / r.L;
    r.gt = 1;
    while (r.gt < teams && r.gt < s.G && r.gt * s.Cg * (int)sizeof(T) < 128) r.gt *= 2;
    // more groups and fewer samples per block while blocks are more than run at a time: a block's set-up then serves more turns
    const int at_a_time = (backward ? kRowBlocks<V, K, true> : kRowBlocks<V, K, false>) * kSms;
    auto slabs = [&](int gt) { return (s.G + gt - 1) / gt; };
    while (r.gt * 2 <= teams && r.gt < s.G && (int64_t)slabs(r.gt) * (backward ? sets : 1) > at_a_time) r.gt *= 2;
    r.slabs = slabs(r.gt);
    r.sp = teams / r.gt;
    if (r.sp > batch) r.sp = (int)batch;
    int64_t parts = at_a_time / ((int64_t)r.slabs * (backward ? sets : 1));
    const int64_t turns = (batch + r.sp - 1) / r.sp;
    if (parts > turns) parts = turns;
    if (backward && parts > part_rows(s)) parts = part_rows(s);
    r.parts = parts < 1 ? 1 : (int)parts;
    if (!backward) {
        r.turns = (int)((turns + r.parts - 1) / r.parts);
        r.parts = (int)((turns + r.turns - 1) / r.turns);
    }
    r.by_gt.set(r.gt);
    if (!backward) {
        k_gn_rows_forward<T, V, K><<<dim3(r.parts, r.slabs), kT, 0, st>>>(a, r);
        return cudaGetLastError();
    }
    const size_t smem = (size_t)2 * r.sp * r.gt * s.Cg * sizeof(float);
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(k_gn_rows_backward<T, V, K>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
        if (e != cudaSuccess) return e;
    }
    k_gn_rows_backward<T, V, K><<<dim3(r.parts, r.slabs, (unsigned)sets), kT, smem, st>>>(a, r);
    cudaError_t e = cudaGetLastError();
    a.p.parts = r.parts;                                    // what is left to add up
    a.p.chunks = 0;
    return e;
}

template <class T, int V, bool WHOLE>
cudaError_t launch_whole(GnArgs& a, bool backward, cudaStream_t st) {
    const GnPlan& p = a.p;
    auto smem = [&](int task) { return smem_bytes(a.s, p, backward, task); };
    if (!p.chunks) {
        const dim3 grid((unsigned)(backward ? p.parts : p.items), p.slabs, backward ? (unsigned)(a.s.N / a.s.per_set) : 1);
        if constexpr (sizeof(T) * V >= 4) {
            if (p.buffered) return backward ? launch_task(k_gn_backward<T, V, WHOLE, kWhole>, grid, a, smem(kWhole), false, st)
                                            : launch_task(k_gn_forward<T, V, WHOLE, kWhole>, grid, a, smem(kWhole), false, st);
        }
        return backward ? launch_task(k_gn_backward<T, V, WHOLE, kReread>, grid, a, smem(kReread), false, st)
                        : launch_task(k_gn_forward<T, V, WHOLE, kReread>, grid, a, smem(kReread), false, st);
    }
    cudaError_t e = cudaSuccess;
    for (a.n0 = 0; a.n0 < a.s.N && e == cudaSuccess; a.n0 += 65535) {
        const int64_t left = a.s.N - a.n0;
        const dim3 grid(p.chunks, p.slabs, (unsigned)(left < 65535 ? left : 65535)), next(grid.x, grid.y + (backward && left <= 65535 ? 1 : 0), grid.z);
        if (backward) {
            e = launch_task(k_gn_backward<T, V, WHOLE, kSums>, grid, a, smem(kSums), false, st);
            if (e == cudaSuccess) e = launch_task(k_gn_backward<T, V, WHOLE, kApply>, next, a, smem(kApply), true, st);
        } else {
            e = launch_task(k_gn_forward<T, V, WHOLE, kSums>, grid, a, smem(kSums), false, st);
            if (e == cudaSuccess) e = launch_task(k_gn_forward<T, V, WHOLE, kApply>, grid, a, smem(kApply), true, st);
        }
    }
    return e;
}
template <class T, int V>
cudaError_t launch_gn(GnArgs& a, bool backward, cudaStream_t st) {
    if constexpr (V * sizeof(T) == 16) {
        if (in_rows(a.s, V, (int)sizeof(T)))
            return a.s.Cg <= 32 * kRowChannels ? launch_rows<T, V, kRowChannels / V>(a, backward, st) : launch_rows<T, V, 4>(a, backward, st);
    }
    if (a.s.Cg % V == 0) return launch_whole<T, V, true>(a, backward, st);
    if constexpr (V > 1) return launch_whole<T, V, false>(a, backward, st);
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
    // addresses have 57 bits at most; sums of offsets then stay far from 64
    const __int128 reach = (__int128)(s.N > 0 ? s.N - 1 : 0) * *sn + (__int128)(s.S > 0 ? s.S - 1 : 0) * *ss + s.C;
    if (reach > ((__int128)1 << 56)) return op_fail(err, err_len, RFAST_EINVAL, "%s: the strides of %s reach beyond any memory", me, what);
    return RFAST_OK;
}

int check_workspace(const rfast_gn_shape* g, int backward, const void* workspace, size_t bytes, const char* me, char* err, size_t err_len) {
    const int64_t need = rfast_group_norm_workspace(g, backward);
    if (need == 0) return RFAST_OK;
    if (!workspace || (uintptr_t)workspace % 16 || (int64_t)bytes < need)
        return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace needs %lld bytes, aligned to 16", me, (long long)need);
    return check_device_pointer(workspace, "workspace", err, err_len);
}

// Whether two of the N x S rows of C values share one (rows that interleave in other ways than one stride
// inside the other count as overlapping).
bool overlaps(const GnShape& s, int64_t sn, int64_t ss) {
    int64_t near = ss, far = sn, inner = s.S, outer = s.N;
    if (outer > 1 && (inner == 1 || sn < ss)) { near = sn; far = ss; inner = s.N; outer = s.S; }
    if (inner > 1 && near < s.C) return true;
    return outer > 1 && far < (inner - 1) * near + s.C;
}

// Whether a result lies where an operand does, but in other strides: values would be overwritten before they are read.
bool torn(const GnShape& s, const void* out, int64_t on, int64_t os, const void* in, int64_t sn, int64_t ss) {
    return out == in && ((s.N > 1 && on != sn) || (s.S > 1 && os != ss));
}

}  // namespace

// Partial sums of the channels: as many rows as a set's samples at most.
size_t norm_rows_workspace(int max_events, int batch, int hidden) { return (size_t)max_events * batch * 2 * hidden * sizeof(float); }

cudaError_t norm_rows_launch(const NormRows& r, bool backward, cudaStream_t st, int64_t* launches) {
    GnArgs a{};
    a.s.N = (int64_t)r.n_events * r.batch; a.s.S = 1; a.s.C = r.hidden; a.s.G = r.groups; a.s.Cg = r.hidden / r.groups;
    a.s.per_set = r.batch; a.s.eps = r.eps; a.s.act = r.act;
    a.x = r.x; a.dy = r.dy; a.out = r.out;
    a.xn = a.xs = a.dn = a.ds = a.on = a.os = r.hidden;
    a.gamma = r.gamma; a.beta = r.beta; a.affine_stride = r.stride;
    a.set_row = &r.ev->node;                                // a device address: it is not read here
    a.set_row_stride = (int)(sizeof(EvDesc) / sizeof(int));
    a.mean = r.mean; a.rstd = r.rstd; a.dgamma = r.dgamma; a.dbeta = r.dbeta;
    a.p = make_plan(a.s, 4, allowed(r.x, a.xn, a.xs, 4), backward);
    a.part = (float*)r.workspace;
    cudaError_t e = launch_typed(a, RFAST_TYPE_F32, backward, st);
    *launches += 1;
    if (e == cudaSuccess && backward && a.p.parts > 1) {
        k_gn_affine<<<dim3((r.hidden + 31) / 32, r.n_events), kT, 0, st>>>(a.part, a.p.parts, r.hidden, r.dgamma, r.dbeta);
        e = cudaGetLastError();
        *launches += 1;
    }
    return e;
}

}  // namespace rfast

using namespace rfast;

#define GN_TRY(expr) do { const int rc_ = (expr); if (rc_ != RFAST_OK) return rc_; } while (0)

extern "C" int64_t rfast_group_norm_workspace(const rfast_gn_shape* g, int backward) {
    const int rc = check_shape(g, "rfast_group_norm_workspace", nullptr, 0);
    if (rc != RFAST_OK) return rc;
    if (g->samples == 0 || g->positions == 0) return 0;
    const GnShape s = shape_from(g, 1.f);
    return (int64_t)workspace_bytes_of(s, type_bytes(g->type), backward != 0);
}

extern "C" int rfast_group_norm(const rfast_gn_shape* g, const void* d_x, const int64_t* x_strides, const float* d_gamma, const float* d_beta, float eps,
                                void* d_y, const int64_t* y_strides, float* d_mean, float* d_rstd, void* workspace, size_t workspace_bytes,
                                void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_group_norm";
    GN_TRY(check_shape(g, me, err, err_len));
    if (!(eps >= 1.17549435e-38f) || !std::isfinite(eps)) return op_fail(err, err_len, RFAST_EINVAL, "%s: eps must be at least 2^-126", me);
    GnArgs a{};
    a.s = shape_from(g, eps);
    GN_TRY(strides_of(x_strides, a.s, &a.xn, &a.xs, me, "x", err, err_len));
    GN_TRY(strides_of(y_strides, a.s, &a.on, &a.os, me, "y", err, err_len));
    if (a.s.N == 0 || a.s.S == 0) return RFAST_OK;
    if (overlaps(a.s, a.on, a.os)) return op_fail(err, err_len, RFAST_EINVAL, "%s: the strides of y make it overlap itself", me);
    if (torn(a.s, d_y, a.on, a.os, d_x, a.xn, a.xs)) return op_fail(err, err_len, RFAST_EINVAL, "%s: y is x, but with other strides", me);
    const void* ptrs[] = {d_x, d_gamma, d_beta, d_y, d_mean, d_rstd};
    const char* names[] = {"x", "gamma", "beta", "y", "mean", "rstd"};
    const int es = type_bytes(g->type);
    for (int k = 0; k < 6; ++k) {
        if (!ptrs[k]) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s is null", me, names[k]);
        if ((uintptr_t)ptrs[k] % (k == 0 || k == 3 ? es : 4)) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s is not aligned to its type", me, names[k]);
    }
    GN_TRY(check_workspace(g, 0, workspace, workspace_bytes, me, err, err_len));
    for (int k = 0; k < 6; ++k) GN_TRY(check_device_pointer(ptrs[k], names[k], err, err_len));
    a.x = d_x; a.out = d_y; a.gamma = d_gamma; a.beta = d_beta; a.affine_stride = a.s.C; a.mean = d_mean; a.rstd = d_rstd;
    const int vx = allowed(d_x, a.xn, a.xs, es), vy = allowed(d_y, a.on, a.os, es);
    a.p = make_plan(a.s, es, vx < vy ? vx : vy, false);
    a.gpart = (float4*)workspace;
    if (a.p.slabs > 65535) return op_fail(err, err_len, RFAST_EINVAL, "%s: too many samples or groups", me);
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
    if (a.s.S > 0 && (torn(a.s, d_dx, a.on, a.os, d_x, a.xn, a.xs) || torn(a.s, d_dx, a.on, a.os, d_dy, a.dn, a.ds)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: dx is x or dy, but with other strides", me);
    const void* ptrs[] = {d_dgamma, d_dbeta, d_gamma, d_beta, d_mean, d_rstd, d_dy, d_x, d_dx};
    const char* names[] = {"dgamma", "dbeta", "gamma", "beta", "mean", "rstd", "dy", "x", "dx"};
    const int es = type_bytes(g->type);
    const int count = a.s.S > 0 ? 9 : 2;
    for (int k = 0; k < count; ++k) {
        if (!ptrs[k]) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s is null", me, names[k]);
        if ((uintptr_t)ptrs[k] % (k >= 6 ? es : 4)) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s is not aligned to its type", me, names[k]);
    }
    if (a.s.S > 0) GN_TRY(check_workspace(g, 1, workspace, workspace_bytes, me, err, err_len));
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
    a.dgamma = d_dgamma; a.dbeta = d_dbeta;
    int v = allowed(d_x, a.xn, a.xs, es);
    const int v2 = allowed(d_dy, a.dn, a.ds, es), v3 = allowed(d_dx, a.on, a.os, es);
    v = v < v2 ? v : v2;
    v = v < v3 ? v : v3;
    a.p = make_plan(a.s, es, v, true);
    a.gpart = (float4*)workspace;
    a.part = (float*)((char*)workspace + group_bytes(a.s, a.p));
    if (a.p.slabs > 65534 || sets > 65535) return op_fail(err, err_len, RFAST_EINVAL, "%s: too many groups or sets", me);
    e = launch_typed(a, g->type, true, st);
    if (e == cudaSuccess && !a.p.chunks && a.p.parts > 1) {
        k_gn_affine<<<dim3((a.s.C + 31) / 32, (unsigned)sets), kT, 0, st>>>(a.part, a.p.parts, a.s.C, d_dgamma, d_dbeta);
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
    return RFAST_OK;
}
