// Gradient norm and AdamW step over many tensors (see rfast_grad_norm and rfast_adamw_step in
// rfast.h for the formulas).
//
// Both walk a list of tensors with one launch for hundreds of them: the table of addresses and
// sizes travels in the kernel's parameters (no copy to the device, nothing that outlives the
// call), tensors are cut into chunks, and a thread block finds its tensor by bisection in the
// table's running chunk counts.
//
// A warp takes a block of 256 values at a time.  Where the tensor's addresses allow it, lane l holds
// quads l and l + 32 of the block, so that a request covers 512, 256 or 128 contiguous bytes for
// 4-, 2- and 1-byte types; in ragged last blocks and misaligned tensors it holds values l + 32 j.
// Either way the block's largest value is one warp reduction away.
#include <cuda_bf16.h>
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <type_traits>
#include <utility>

#include "ops.h"
#include "pairs.cuh"

namespace rfast {

namespace {

constexpr int kThreadsOp = 256;
constexpr int kWarps = kThreadsOp / 32;

// ---- types ------------------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <class T> struct Raw4 { typedef uint2 type; };          // four 16-bit values
template <> struct Raw4<float> { typedef float4 type; };
template <> struct Raw4<uint8_t> { typedef uint32_t type; };     // four codes

__device__ __forceinline__ void unpack2(uint32_t r, const __nv_bfloat16*, float* v) {
    v[0] = __uint_as_float(r << 16);
    v[1] = __uint_as_float(r & 0xffff0000u);
}
__device__ __forceinline__ void unpack2(uint32_t r, const __half*, float* v) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&r));
    v[0] = a.x; v[1] = a.y;
}
__device__ __forceinline__ void unpack4(float4 r, const float*, float* v) { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
template <class T>
__device__ __forceinline__ void unpack4(uint2 r, const T* t, float* v) { unpack2(r.x, t, v); unpack2(r.y, t, v + 2); }

__device__ __forceinline__ void store4(float* t, const float* v) { __stcs(reinterpret_cast<float4*>(t), make_float4(v[0], v[1], v[2], v[3])); }
__device__ __forceinline__ void store4(__nv_bfloat16* t, const float* v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    __stcs(reinterpret_cast<uint2*>(t), make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b)));
}
__device__ __forceinline__ void store4(__half* t, const float* v) {
    const __half2 a = __floats2half2_rn(v[0], v[1]), b = __floats2half2_rn(v[2], v[3]);
    __stcs(reinterpret_cast<uint2*>(t), make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b)));
}

// ---- 8-bit codes: e4m3, four to a word ----------------------------------------------------------
__device__ __forceinline__ void decode4(uint32_t c, float* v) {
    uint32_t lo, hi;
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(c));
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo)), y = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    v[0] = x.x; v[1] = x.y; v[2] = y.x; v[3] = y.y;
}
// nearest, ties to even, beyond the largest value: the largest value
__device__ __forceinline__ uint32_t encode4(const float* v) {
    uint32_t c;
    asm("{\n.reg .b16 a, b;\ncvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\ncvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\nmov.b32 %0, {a, b};\n}"
        : "=r"(c) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]));
    return c;
}

// maxima that a NaN goes through
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max_nan(float v) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
// Scale of a block from its largest value.  The floor keeps 1 / scale finite; blocks that small
// (all below 2^-91) just use fewer codes.
__device__ __forceinline__ float block_scale(float top) {
    return max_nan(__fmul_rn(top, (float)(1.0 / 448.0)), 7.888609052210118e-31f);   // 2^-100
}
constexpr float kLeastNormal = 0x1p-126f, kMostFinite = 0x1.fffffep127f;
// 1 ulp; below the least normal number 0
__device__ __forceinline__ float root_of(float v) {
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// 1 ulp, down to the least number of all: 32-bit second moments are held that far
__device__ __forceinline__ float root_of_any(float v) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// 1 ulp; the denominators are at least eps, a normal number
__device__ __forceinline__ float inverse_of(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

struct TensorView {
    void* p;
    const void* g;
    void *m, *v;
    float *ms, *vs;
    int64_t n;
    bool wide;
};

// Factors of a step that do not change from value to value.
struct StepFactors {
    float scale;         // of the gradients
    float b1, g1;        // 32-bit moments: m = b1 m + g1 g, the scale within g1; 8-bit moments: m = b1 m + g1 (scale g)
    float b2, g2;        // 32-bit moments: v = b2 v + (g2 g)^2, likewise; 8-bit moments: v = (b2 r)^2 + (g2 scale g)^2
    float root, eps, keep, step;
};
template <bool S8>
__device__ __forceinline__ StepFactors factors(const AdamCoef& c, float gscale) {
    if (S8) return {gscale, c.beta1, c.omb1, c.root_beta2, c.root_omb2, c.root, c.eps, c.keep, c.step};
    return {1.f, c.beta1, gscale * c.omb1, c.beta2, gscale * c.root_omb2, c.root, c.eps, c.keep, c.step};
}

// Eight values with 32-bit moments: moments and parameter after the step.
__device__ __forceinline__ void advance(const StepFactors& f, float (&p)[8], const float (&g)[8], float (&m)[8], float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float h = f.g2 * g[k];
        m[k] = fmaf(f.g1, g[k], f.b1 * m[k]);
        v[k] = fmaf(f.b2, v[k], h * h);
        const float r = root_of_any(v[k]);
        p[k] = fmaf(-f.step, m[k] * inverse_of(fmaf(r, f.root, f.eps)), p[k] * f.keep);
    }
}

// 8-bit moments come as codes with their block's scales and leave as the first moment and the root of the second.
//
// First moments.  Value, products and sum are rounded one after the other, as the formula has them: the sum decides between two
// codes, and formed in fewer roundings it falls on the other side of a border in other places than a plain evaluation does
// (26M values: some 30 codes, each off by 2^-4 of itself).  The scaled gradients are left in g.
__device__ __forceinline__ void first_moments8(const StepFactors& f, float sm, float (&g)[8], float (&m)[8]) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const F2 s = pair(g[k], g[k + 1]) * both(f.scale);
        split(s, g[k], g[k + 1]);
        float a[2], b[2];
        split(pair(m[k], m[k + 1]) * both(sm) * both(f.b1), a[0], a[1]);
        split(s * both(f.g1), b[0], b[1]);
        m[k] = __fadd_rn(a[0], b[0]);                       // (a sum of pairs would be merged with the product before it)
        m[k + 1] = __fadd_rn(a[1], b[1]);
    }
}
// Roots and parameters where the second moments may leave the range of fp32: q and h are brought near 1 by a power of two first, and
// so are numerator and denominator of the quotient where the root is large.  Any finite gradient then has a finite root, and any
// gradient but 0 (down to where its product with sqrt(1 - beta2) is 0) a positive one.  g: scaled
__device__ __forceinline__ void finish8_far(const StepFactors& f, float bv, float (&p)[8], const float (&g)[8], const float (&m)[8], float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float q = bv * v[k], h = f.g2 * g[k], top = fmaxf(fabsf(q), fabsf(h));
        const bool high = top > 0x1p60f, low = top < 0x1p-60f;
        const float in = high ? 0x1p-70f : low ? 0x1p100f : 1.f, out = high ? 0x1p70f : low ? 0x1p-100f : 1.f;
        const float a = q * in, b = h * in, r = root_of(fmaf(a, a, b * b)), near = high ? in : 1.f;
        v[k] = r * out;
        p[k] = fmaf(-f.step, m[k] * near * inverse_of(fmaf(high ? r : v[k], f.root, f.eps * near)), p[k] * f.keep);
    }
}
// The roots q of before reach from 2^-109 to 2^128, and a gradient may be any fp32 value, so that q^2 + h^2 can leave fp32's range
// where its root does not.  Lanes with such a value take the way above.  again(q): what came in v
template <class Again>
__device__ __forceinline__ void advance8(const StepFactors& f, float sm, float sv, float (&p)[8], float (&g)[8], float (&m)[8], float (&v)[8], Again again) {
    const float bv = sv * f.b2;
    first_moments8(f, sm, g, m);
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const F2 q = pair(v[k], v[k + 1]) * both(bv), h = pair(g[k], g[k + 1]) * both(f.g2);
        split(fma2(q, q, h * h), v[k], v[k + 1]);
    }
    float least = v[0], most = v[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) { least = fminf(least, v[k]); most = fmaxf(most, v[k]); }
    if (!(least >= kLeastNormal && most <= kMostFinite)) {
        float q[8];
        again(q);                                           // decoded once more rather than kept
        bool far = most > kMostFinite;
#pragma unroll
        for (int k = 0; k < 8; ++k) far = far || (v[k] < kLeastNormal && fabsf(bv * q[k]) + fabsf(f.g2 * g[k]) > 0.f);      // not 0, exactly
        if (far) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = q[k];
            finish8_far(f, bv, p, g, m, v);
            return;
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        v[k] = root_of(v[k]);
        p[k] = fmaf(-f.step, m[k] * inverse_of(fmaf(v[k], f.root, f.eps)), p[k] * f.keep);
    }
}

// Scales and codes of a block's moments, eight values in every lane.  A positive root keeps a positive
// code: a first moment that survives its rounding must not meet a denominator of eps alone.
__device__ __forceinline__ void to_codes(const float (&m)[8], const float (&r)[8], float& sm, float& sv, float (&cm)[8], float (&cv)[8]) {
    float tm = fabsf(m[0]), tv = r[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) { tm = max_nan(tm, fabsf(m[k])); tv = max_nan(tv, r[k]); }
    sm = block_scale(warp_max_nan(tm));
    sv = block_scale(warp_max_nan(tv));
    const float im = __frcp_rn(sm), iv = __frcp_rn(sv);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        cm[k] = m[k] * im;
        const float q = r[k] * iv;
        cv[k] = r[k] > 0.f ? max_nan(q, 0.001953125f) : q;      // 2^-9
    }
}

// A block as it lies in memory, two quads of every stream per lane.
template <class PT, class GT, class MT>
struct RawBlock {
    typename Raw4<PT>::type p[2];
    typename Raw4<GT>::type g[2];
    typename Raw4<MT>::type m[2], v[2];
    float sm, sv;
};
template <class PT, class GT, class MT>
__device__ __forceinline__ void fetch(RawBlock<PT, GT, MT>& r, const TensorView& t, int64_t b, int lane) {
    const int64_t i = b * kAdamBlock + lane * 4;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        r.g[k] = __ldcs(reinterpret_cast<const typename Raw4<GT>::type*>((const GT*)t.g + i + k * 128));
        r.p[k] = __ldcs(reinterpret_cast<const typename Raw4<PT>::type*>((const PT*)t.p + i + k * 128));
        r.m[k] = __ldcs(reinterpret_cast<const typename Raw4<MT>::type*>((const MT*)t.m + i + k * 128));
        r.v[k] = __ldcs(reinterpret_cast<const typename Raw4<MT>::type*>((const MT*)t.v + i + k * 128));
    }
}
template <class PT, class GT, class MT, bool S8>
__device__ __forceinline__ void finish(const RawBlock<PT, GT, MT>& r, const TensorView& t, const StepFactors& f, int64_t b, int lane) {
    const int64_t i = b * kAdamBlock + lane * 4;
    float p[8], g[8], m[8], v[8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        unpack4(r.g[k], (const GT*)nullptr, g + 4 * k);
        unpack4(r.p[k], (const PT*)nullptr, p + 4 * k);
        if constexpr (S8) {
            decode4(r.m[k], m + 4 * k);
            decode4(r.v[k], v + 4 * k);
        } else {
            unpack4(r.m[k], (const float*)nullptr, m + 4 * k);
            unpack4(r.v[k], (const float*)nullptr, v + 4 * k);
        }
    }
    if constexpr (S8) advance8(f, r.sm, r.sv, p, g, m, v, [&](float (&q)[8]) { decode4(r.v[0], q); decode4(r.v[1], q + 4); });
    else advance(f, p, g, m, v);
#pragma unroll
    for (int k = 0; k < 2; ++k) store4((PT*)t.p + i + k * 128, p + 4 * k);
    if constexpr (S8) {
        float sm, sv, cm[8], cv[8];
        to_codes(m, v, sm, sv, cm, cv);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            __stcs(reinterpret_cast<uint32_t*>((uint8_t*)t.m + i + k * 128), encode4(cm + 4 * k));
            __stcs(reinterpret_cast<uint32_t*>((uint8_t*)t.v + i + k * 128), encode4(cv + 4 * k));
        }
        if (lane == 0) { t.ms[b] = sm; t.vs[b] = sv; }
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            store4((float*)t.m + i + k * 128, m + 4 * k);
            store4((float*)t.v + i + k * 128, v + 4 * k);
        }
    }
}

// A block that ends early or whose tensor is misaligned, value by value.  Values beyond the end
// count as zeros: they raise no maximum.
template <class PT, class GT, class MT, bool S8>
__device__ __forceinline__ void block_by_values(const TensorView& t, const StepFactors& f, int64_t b, int lane) {
    const int64_t i = b * kAdamBlock + lane;
    float p[8], g[8], m[8], v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t j = i + 32 * k;
        const bool in = j < t.n;
        p[k] = in ? to_f32(((const PT*)t.p)[j]) : 0.f;
        g[k] = in ? to_f32(((const GT*)t.g)[j]) : 0.f;
        if constexpr (S8) {
            float q[4];
            const uint32_t c = in ? (uint32_t)((const uint8_t*)t.m)[j] | (uint32_t)((const uint8_t*)t.v)[j] << 8 : 0u;
            decode4(c, q);
            m[k] = q[0]; v[k] = q[1];
        } else {
            m[k] = in ? ((const float*)t.m)[j] : 0.f;
            v[k] = in ? ((const float*)t.v)[j] : 0.f;
        }
    }
    if constexpr (S8) {
        first_moments8(f, t.ms[b], g, m);
        finish8_far(f, t.vs[b] * f.b2, p, g, m, v);         // right at any size
    } else {
        advance(f, p, g, m, v);
    }
    float sm, sv, cm[8], cv[8];
    if constexpr (S8) to_codes(m, v, sm, sv, cm, cv);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t j = i + 32 * k;
        if (j >= t.n) break;
        ((PT*)t.p)[j] = from_f32<PT>(p[k]);
        if constexpr (S8) {
            const float q[4] = {cm[k], cv[k], 0.f, 0.f};
            const uint32_t c = encode4(q);
            ((uint8_t*)t.m)[j] = (uint8_t)c;
            ((uint8_t*)t.v)[j] = (uint8_t)(c >> 8);
        } else {
            ((float*)t.m)[j] = m[k];
            ((float*)t.v)[j] = v[k];
        }
    }
    if constexpr (S8) if (lane == 0) { t.ms[b] = sm; t.vs[b] = sv; }
}

constexpr int kMaxRun = 16;                                 // most blocks of 256 values per warp

// Ragged and misaligned blocks of a chunk.
template <class PT, class GT, class MT, bool S8>
__device__ __forceinline__ void rest_of_chunk(const TensorView& t, const StepFactors& f, int64_t full, int64_t c0, int run) {
    const int64_t end = c0 + (int64_t)run * kWarps;
    if (end <= full) return;
#pragma unroll 1
    for (int64_t b = c0 + (threadIdx.x >> 5); b < end && b * kAdamBlock < t.n; b += kWarps)
        if (b >= full) block_by_values<PT, GT, MT, S8>(t, f, b, threadIdx.x & 31);
}

// The chunk of run * 8 blocks from c0 on, by one thread block: warp w takes blocks w, w + 8, ...
// 32-bit moments: a block is fetched into registers while the one before it is worked on (26M fp32 values: 110 us,
// 6.6 TB/s, the memory's rate).
template <class PT, class GT>
__device__ __forceinline__ void adamw_chunk32(const TensorView& t, const StepFactors& f, int64_t c0, int run) {
    const int lane = threadIdx.x & 31;
    const int64_t b0 = c0 + (threadIdx.x >> 5), full = t.wide ? t.n / kAdamBlock : 0;
    const int64_t end = min(full, c0 + (int64_t)run * kWarps);
    RawBlock<PT, GT, float> raw[2];
    if (b0 < end) fetch(raw[0], t, b0, lane);
    for (int64_t b = b0; b < end; b += 2 * kWarps) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t at = b + u * kWarps;
            if (at + kWarps < end) fetch(raw[u ^ 1], t, at + kWarps, lane);
            if (at < end) finish<PT, GT, float, false>(raw[u], t, f, at, lane);
        }
    }
    rest_of_chunk<PT, GT, float, false>(t, f, full, c0, run);
}

// 8-bit moments: twice to four times the arithmetic per byte.  A warp's next blocks wait in its own
// ring in shared memory (asynchronous 16-byte copies), so that the registers hold one block only and
// 32 warps fit an SM.  With the blocks ahead in registers 24 warps did, and the pass over
// 78M bf16 values with bf16 gradients ran at 3.4 TB/s, waiting for loads; in the ring they take 128 us, 6.2 TB/s,
// with 84 % of the issue slots taken, and 26M fp32 values 66 us, 6.4 TB/s.  Misaligned tensors take the way of the
// ragged blocks, without loads ahead: 33.6M values one element off 16 bytes 129 us in the place of 83 (fp32), 140 of 55 (bf16);
// with 32-bit moments 290 of 142 and 166 of 116.
template <class PT, class GT>
struct Ring {
    static constexpr int kP = kAdamBlock * sizeof(PT), kG = kAdamBlock * sizeof(GT);
    static constexpr int kStage = kP + kG + 2 * kAdamBlock;
    static constexpr int kDepth = 6000 / kStage;            // 2 or 3 stages: four rings of 8 warps fit an SM
};
__device__ __forceinline__ void copy16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
template <class PT, class GT>
__device__ __forceinline__ void adamw_chunk8(const TensorView& t, const StepFactors& f, int64_t c0, int run, uint8_t* smem) {
    typedef Ring<PT, GT> R;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint8_t* ring = smem + warp * R::kDepth * R::kStage;
    const int64_t b0 = c0 + warp, full = t.wide ? t.n / kAdamBlock : 0;
    const int64_t left = full - b0;
    const int count = left <= 0 ? 0 : (int)min((int64_t)run, (left + kWarps - 1) / kWarps);
    // the scales of all blocks of the warp: lane u the first moment's of block u, lane 16 + u the second's
    float scales = 0.f;
    if ((lane & 15) < count) scales = (lane < 16 ? t.ms : t.vs)[b0 + (int64_t)(lane & 15) * kWarps];
    auto issue = [&](int u) {
        if (u < count) {
            uint8_t* s = ring + (u % R::kDepth) * R::kStage;
            const int64_t i = (b0 + (int64_t)u * kWarps) * kAdamBlock;
            const char* p = (const char*)((const PT*)t.p + i);
            const char* g = (const char*)((const GT*)t.g + i);
#pragma unroll
            for (int o = 0; o < R::kP; o += 512) copy16(s + o + lane * 16, p + o + lane * 16);
#pragma unroll
            for (int o = 0; o < R::kG; o += 512) copy16(s + R::kP + o + lane * 16, g + o + lane * 16);
            copy16(s + R::kP + R::kG + lane * 16, (const uint8_t*)(lane < 16 ? t.m : t.v) + i + (lane & 15) * 16);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int u = 0; u < R::kDepth - 1; ++u) issue(u);
#pragma unroll 1
    for (int u = 0; u < count; ++u) {
        issue(u + R::kDepth - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(R::kDepth - 1) : "memory");
        __syncwarp();                                       // every lane's copies of this stage have landed
        const uint8_t* s = ring + (u % R::kDepth) * R::kStage;
        RawBlock<PT, GT, uint8_t> raw;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            raw.p[k] = reinterpret_cast<const typename Raw4<PT>::type*>(s)[lane + 32 * k];
            raw.g[k] = reinterpret_cast<const typename Raw4<GT>::type*>(s + R::kP)[lane + 32 * k];
            raw.m[k] = reinterpret_cast<const uint32_t*>(s + R::kP + R::kG)[lane + 32 * k];
            raw.v[k] = reinterpret_cast<const uint32_t*>(s + R::kP + R::kG + kAdamBlock)[lane + 32 * k];
        }
        raw.sm = __shfl_sync(0xffffffffu, scales, u);
        raw.sv = __shfl_sync(0xffffffffu, scales, 16 + u);
        __syncwarp();                                       // the stage may be filled again
        finish<PT, GT, uint8_t, true>(raw, t, f, b0 + (int64_t)u * kWarps, lane);
    }
    rest_of_chunk<PT, GT, uint8_t, true>(t, f, full, c0, run);
}
template <class PT, class GT, bool S8>
__device__ __forceinline__ void adamw_chunk(const TensorView& t, const StepFactors& f, int64_t c0, int run) {
    if constexpr (S8) {
        __shared__ __align__(16) uint8_t smem[kWarps * Ring<PT, GT>::kDepth * Ring<PT, GT>::kStage];
        adamw_chunk8<PT, GT>(t, f, c0, run, smem);
    } else {
        adamw_chunk32<PT, GT>(t, f, c0, run);
    }
}

template <int T>
struct AdamTable {
    void* p[T];
    const void* g[T];
    void* m[T];
    void* v[T];
    float* ms[T];
    float* vs[T];
    int64_t n[T];                                           // negative: -1 - n, no quad accesses
    int first[T + 1];                                       // first thread block of a tensor
    int count;
    int run;                                                // blocks of 256 values per warp
    // step count on the device
    const int64_t* d_step;
    double lr, beta1, beta2;
    const float* d_scale;
    AdamCoef c;
};

// index of the last entry of first[0 .. count) that is at most b
__device__ __forceinline__ int find_tensor(const int* first, int count, int b) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= b) lo = mid; else hi = mid;
    }
    return lo;
}

template <class PT, class GT, bool S8, int T>
__global__ void __launch_bounds__(kThreadsOp, S8 ? 4 : 2)
k_adamw(const __grid_constant__ AdamTable<T> a) {
    AdamCoef c = a.c;
    if (a.d_step) {
        __shared__ float s_step, s_root;
        if (threadIdx.x == 0) {                             // 64 bits: 1 - beta^t cancels at small t
            const double t = (double)*a.d_step;
            s_step = (float)(a.lr / (1.0 - pow(a.beta1, t)));
            s_root = (float)(1.0 / sqrt(1.0 - pow(a.beta2, t)));
        }
        __syncthreads();
        c.step = s_step;
        c.root = s_root;
    }
    const float gscale = a.d_scale ? *a.d_scale : 1.f;
    const int k = find_tensor(a.first, a.count, blockIdx.x);
    TensorView t{a.p[k], a.g[k], a.m[k], a.v[k], nullptr, nullptr, a.n[k], true};
    if (S8) { t.ms = a.ms[k]; t.vs = a.vs[k]; }
    if (t.n < 0) { t.n = -1 - t.n; t.wide = false; }
    adamw_chunk<PT, GT, S8>(t, factors<S8>(c, gscale), (int64_t)(blockIdx.x - a.first[k]) * (a.run * kWarps), a.run);
}

// The engine's rows.  grid = (chunks of a row, events)
template <bool S8>
__global__ void __launch_bounds__(kThreadsOp, S8 ? 4 : 2)
k_adamw_rows(AdamRows r, AdamCoef c, int run) {
    const EvDesc e = r.ev[blockIdx.y];
    const float2 f = r.factor[e.stamp - 1];
    c.step = r.lr * f.x;
    c.root = f.y;
    const int64_t row = (int64_t)e.node * r.stride, srow = (int64_t)e.node * r.scale_stride;
    TensorView t{r.x + row, r.z + row, nullptr, nullptr, nullptr, nullptr, r.p, true};
    if (S8) {
        t.m = (uint8_t*)r.m + row; t.v = (uint8_t*)r.v + row;
        t.ms = r.m_scale + srow; t.vs = r.v_scale + srow;
    } else {
        t.m = (float*)r.m + row; t.v = (float*)r.v + row;
    }
    adamw_chunk<float, float, S8>(t, factors<S8>(c, 1.f), (int64_t)blockIdx.x * (run * kWarps), run);
}

// ---- gradient norm ----------------------------------------------------------------------------------
constexpr int kNormU = 4;                                   // 16-byte loads of a thread in flight
constexpr int kNormBytes = kThreadsOp * 16 * kNormU;        // bytes of a chunk
constexpr int kNormParts = RFAST_GRAD_NORM_WORKSPACE / 8;   // partial sums that the workspace holds
constexpr int kNormGrid = 148 * 6;

template <int T>
struct NormTable {
    const void* g[T];
    int64_t n[T];                                           // negative: -1 - n, no quad accesses
    int64_t first[T + 1];                                   // first chunk of a tensor
    int count;
    double* part;                                           // one partial sum per thread block
};

// Sum of the squares of eight values.  In 32 bits the squares of values beyond 1e19 overflow and
// those below 1e-19 lose digits; such groups (and those of zeros) are summed in 64 bits.
__device__ __forceinline__ double square_sum(const float (&v)[8]) {
    float s = v[0] * v[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) s = fmaf(v[k], v[k], s);
    if (s > 1e-25f && s < 1e37f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int k = 0; k < 8; ++k) d = fma((double)v[k], (double)v[k], d);
    return d;
}
__device__ __forceinline__ void unpack_pair(uint4 a, uint4 b, const float*, float (&x)[8], float (&)[8]) {   // 8 values, the rest unused
    x[0] = __uint_as_float(a.x); x[1] = __uint_as_float(a.y); x[2] = __uint_as_float(a.z); x[3] = __uint_as_float(a.w);
    x[4] = __uint_as_float(b.x); x[5] = __uint_as_float(b.y); x[6] = __uint_as_float(b.z); x[7] = __uint_as_float(b.w);
}
template <class T>
__device__ __forceinline__ void unpack_pair(uint4 a, uint4 b, const T* t, float (&x)[8], float (&y)[8]) {
    unpack2(a.x, t, x); unpack2(a.y, t, x + 2); unpack2(a.z, t, x + 4); unpack2(a.w, t, x + 6);
    unpack2(b.x, t, y); unpack2(b.y, t, y + 2); unpack2(b.z, t, y + 4); unpack2(b.w, t, y + 6);
}

// Sum over a thread block in a fixed tree; the result in thread 0.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* sh) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < THREADS / 32; ++w) s += sh[w];
    return s;
}

// Thread `tid` of 256: its share of the squares of chunk ch.  k: the last tensor to look for it in (chunks of a
// thread come in descending order), left at the chunk's tensor.
template <class GT, int T>
__device__ __forceinline__ double norm_chunk(const NormTable<T>& a, int64_t ch, int& k, int tid) {
    double sum = 0.0;
    int lo = 0, hi = k + 1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= ch) lo = mid; else hi = mid;
    }
    k = lo;
    int64_t n = a.n[k];
    const bool wide = n >= 0;
    if (!wide) n = -1 - n;
    const GT* g = (const GT*)a.g[k];
    constexpr int kPer = kNormBytes / (int)sizeof(GT);      // values of a chunk
    const int64_t i0 = (ch - a.first[k]) * kPer;
    const int64_t end = i0 + kPer < n ? i0 + kPer : n;
    if (wide) {
        constexpr int kV = 16 / (int)sizeof(GT);            // values of a 16-byte load
        const uint4* src = reinterpret_cast<const uint4*>(g + i0) + tid;
        const int loads = (int)((end - i0) / kV);
        uint4 q[kNormU];
#pragma unroll
        for (int u = 0; u < kNormU; ++u) q[u] = tid + u * kThreadsOp < loads ? __ldg(src + u * kThreadsOp) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < kNormU; u += 2) {
            float x[8], y[8];
            unpack_pair(q[u], q[u + 1], (const GT*)nullptr, x, y);
            sum += square_sum(x);
            if (sizeof(GT) == 2) sum += square_sum(y);
        }
        const int64_t i = i0 + (int64_t)loads * kV + tid;   // the tensor's last values, fewer than a load holds
        if (i < end) { const double v = (double)to_f32(g[i]); sum = fma(v, v, sum); }
    } else {
        for (int64_t i = i0 + tid; i < end; i += 8 * kThreadsOp) {
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = i + u * kThreadsOp < end ? to_f32(g[i + u * kThreadsOp]) : 0.f;
            sum += square_sum(x);
        }
    }
    return sum;
}

__device__ __forceinline__ void norm_out(double sum, float max_norm, float* norm_out, float* scale_out) {
    const double norm = sqrt(sum);
    if (norm_out) *norm_out = (float)norm;
    // a NaN goes through; an infinite norm gives 0
    if (scale_out) *scale_out = norm != norm ? (float)norm : norm <= (double)max_norm ? 1.f : (float)((double)max_norm / norm);
}

// Reads at the rate of the memory: 9 x 11.2M bf16 values in 33 us with the closing kernel, 6.1 TB/s.
template <class GT, int T>
__global__ void __launch_bounds__(kThreadsOp)
k_grad_norm(const __grid_constant__ NormTable<T> a) {
    __shared__ double sh[kWarps];
    asm volatile("griddepcontrol.launch_dependents;");
    double sum = 0.0;
    const int64_t chunks = a.first[a.count];
    int k = a.count - 1;
    // back to front: what is read last is what the step after it reads first, while the L2 cache holds it
    for (int64_t ch = chunks - 1 - blockIdx.x; ch >= 0; ch -= gridDim.x) sum += norm_chunk<GT, T>(a, ch, k, threadIdx.x);
    const double s = block_sum<kThreadsOp>(sum, sh);
    if (threadIdx.x == 0) a.part[blockIdx.x] = s;
}

__global__ void __launch_bounds__(kThreadsOp)
k_grad_norm_end(const double* __restrict__ part, int parts, float max_norm, float* norm, float* scale) {
    __shared__ double sh[kWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreadsOp) sum += part[i];
    const double s = block_sum<kThreadsOp>(sum, sh);
    if (threadIdx.x == 0) norm_out(s, max_norm, norm, scale);
}

// Little data: one cluster of eight thread blocks, whose sums meet in the first one's shared memory, does
// it all in one launch.
constexpr int kOneCtas = 8, kOneThreads = 1024, kOneTeams = kOneCtas * kOneThreads / kThreadsOp;
template <class GT, int T>
__global__ void __cluster_dims__(kOneCtas, 1, 1) __launch_bounds__(kOneThreads)
k_grad_norm_one(const __grid_constant__ NormTable<T> a, float max_norm, float* norm, float* scale) {
    __shared__ double sh[kOneThreads / 32], all[kOneCtas];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    auto begun = cluster.barrier_arrive();
    double sum = 0.0;
    const int64_t chunks = a.first[a.count];
    int k = a.count - 1;
    for (int64_t ch = chunks - 1 - blockIdx.x * (kOneThreads / kThreadsOp) - threadIdx.x / kThreadsOp; ch >= 0; ch -= kOneTeams)
        sum += norm_chunk<GT, T>(a, ch, k, threadIdx.x % kThreadsOp);
    const double s = block_sum<kOneThreads>(sum, sh);
    cluster.barrier_wait(std::move(begun));                 // the first block has begun: its shared memory is there
    if (threadIdx.x == 0) cluster.map_shared_rank(all, 0)[blockIdx.x] = s;
    cluster.sync();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        double t = 0.0;
        for (int r = 0; r < kOneCtas; ++r) t += all[r];
        norm_out(t, max_norm, norm, scale);
    }
}

size_t type_bytes(int t) { return t == RFAST_TYPE_F32 ? 4 : 2; }
bool known_type(int t) { return t == RFAST_TYPE_F32 || t == RFAST_TYPE_BF16 || t == RFAST_TYPE_F16; }

template <class PT, class GT, bool S8, int T>
cudaError_t launch_adamw(const AdamTable<T>& a, cudaStream_t st) {
    k_adamw<PT, GT, S8, T><<<a.first[a.count], kThreadsOp, 0, st>>>(a);
    return cudaGetLastError();
}
template <class PT, class GT, int T>
cudaError_t pick_state(const AdamTable<T>& a, int bits, cudaStream_t st) {
    return bits == 8 ? launch_adamw<PT, GT, true, T>(a, st) : launch_adamw<PT, GT, false, T>(a, st);
}
template <class PT, int T>
cudaError_t pick_grad(const AdamTable<T>& a, int gt, int bits, cudaStream_t st) {
    switch (gt) {
        case RFAST_TYPE_F32: return pick_state<PT, float, T>(a, bits, st);
        case RFAST_TYPE_BF16: return pick_state<PT, __nv_bfloat16, T>(a, bits, st);
        default: return pick_state<PT, __half, T>(a, bits, st);
    }
}
template <int T>
cudaError_t pick_param(const AdamTable<T>& a, int pt, int gt, int bits, cudaStream_t st) {
    switch (pt) {
        case RFAST_TYPE_F32: return pick_grad<float, T>(a, gt, bits, st);
        case RFAST_TYPE_BF16: return pick_grad<__nv_bfloat16, T>(a, gt, bits, st);
        default: return pick_grad<__half, T>(a, gt, bits, st);
    }
}

// A table of T entries is copied into every launch; few tensors take the small one.
constexpr int kFew = 64, kMany = 480;

// Blocks of 256 values per warp: as long as every SM gets several rounds of thread blocks, longer runs
// pay the look-up in the table and the first, exposed fetch less often.
int run_length(int64_t blocks) {
    const int64_t run = blocks / ((int64_t)kWarps * 148 * 16);
    return (int)(run < 1 ? 1 : run > kMaxRun ? kMaxRun : run);
}

// Launches the tensors [k0, k1) that are not empty.
template <int T>
cudaError_t adamw_span(const rfast_adamw* a, const AdamCoef& c, int k0, int k1, int run, cudaStream_t st) {
    AdamTable<T> t;
    t.run = run;
    const int64_t per = (int64_t)run * kWarps * kAdamBlock;
    t.c = c;
    t.d_step = a->d_step;
    t.lr = a->lr; t.beta1 = a->beta1; t.beta2 = a->beta2;
    t.d_scale = a->d_grad_scale;
    int q = 0;
    int64_t blocks = 0;
    const bool s8 = a->state_bits == 8;                     // its copies are 16 bytes wide whatever the type
    const size_t pq = s8 ? 16 : 4 * type_bytes(a->param_type), gq = s8 ? 16 : 4 * type_bytes(a->grad_type);
    for (int k = k0; k < k1; ++k) {
        const int64_t n = a->numel[k];
        if (n == 0) continue;
        const bool wide = !((uintptr_t)a->param[k] % pq || (uintptr_t)a->grad[k] % gq || (uintptr_t)a->m[k] % 16 || (uintptr_t)a->v[k] % 16);
        t.p[q] = a->param[k]; t.g[q] = a->grad[k]; t.m[q] = a->m[k]; t.v[q] = a->v[k];
        t.ms[q] = a->state_bits == 8 ? a->m_scale[k] : nullptr;
        t.vs[q] = a->state_bits == 8 ? a->v_scale[k] : nullptr;
        t.n[q] = wide ? n : -1 - n;
        t.first[q] = (int)blocks;
        blocks += (n + per - 1) / per;
        ++q;
    }
    if (q == 0) return cudaSuccess;
    t.count = q;
    t.first[q] = (int)blocks;
    return pick_param<T>(t, a->param_type, a->grad_type, a->state_bits, st);
}

// Up to this many chunks the single cluster does the work: 1 MB, which it reads in 2 to 3 us; a second launch
// costs as much.
constexpr int64_t kOneChunks = 64;

struct NormOut {
    float max_norm;
    float *norm, *scale;
};
// `out`: this launch holds all there is, and may write the results itself (it then leaves *blocks_out = -1).
template <class GT, int T>
cudaError_t norm_span(const int64_t* numel, const void* const* grad, int k0, int k1, int max_blocks, double* part, const NormOut* out, int* blocks_out, cudaStream_t st) {
    NormTable<T> t;
    int q = 0;
    int64_t chunks = 0;
    for (int k = k0; k < k1; ++k) {
        const int64_t n = numel[k];
        if (n == 0) continue;
        t.g[q] = grad[k];
        t.n[q] = (uintptr_t)grad[k] % 16 == 0 ? n : -1 - n;
        t.first[q] = chunks;
        const int64_t per = kNormBytes / (int64_t)sizeof(GT);
        chunks += (n + per - 1) / per;
        ++q;
    }
    t.count = q;
    t.first[q] = chunks;
    t.part = part;
    *blocks_out = 0;
    if (out && chunks <= kOneChunks) {
        k_grad_norm_one<GT, T><<<kOneCtas, kOneThreads, 0, st>>>(t, out->max_norm, out->norm, out->scale);
        *blocks_out = -1;
        return cudaGetLastError();
    }
    if (q == 0) return cudaSuccess;
    const int blocks = (int)(chunks < max_blocks ? chunks : max_blocks);
    k_grad_norm<GT, T><<<blocks, kThreadsOp, 0, st>>>(t);
    *blocks_out = blocks;
    return cudaGetLastError();
}
template <int T>
cudaError_t norm_pick(int type, const int64_t* numel, const void* const* grad, int k0, int k1, int max_blocks, double* part, const NormOut* out, int* blocks_out, cudaStream_t st) {
    switch (type) {
        case RFAST_TYPE_F32: return norm_span<float, T>(numel, grad, k0, k1, max_blocks, part, out, blocks_out, st);
        case RFAST_TYPE_BF16: return norm_span<__nv_bfloat16, T>(numel, grad, k0, k1, max_blocks, part, out, blocks_out, st);
        default: return norm_span<__half, T>(numel, grad, k0, k1, max_blocks, part, out, blocks_out, st);
    }
}
constexpr int kNormFew = 48, kNormMany = 1280;

}  // namespace

int op_fail(char* err, size_t err_len, int code, const char* fmt, ...) {
    if (err && err_len) {
        va_list ap;
        va_start(ap, fmt);
        std::vsnprintf(err, err_len, fmt, ap);
        va_end(ap);
    }
    return code;
}

int check_device_pointer(const void* p, const char* what, char* err, size_t err_len) {
    cudaPointerAttributes at;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaPointerGetAttributes(&at, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return op_fail(err, err_len, RFAST_ECUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    if (at.type == cudaMemoryTypeManaged) return RFAST_OK;
    if (at.type != cudaMemoryTypeDevice) return op_fail(err, err_len, RFAST_EINVAL, "%s: not device memory", what);
    if (at.device != dev) return op_fail(err, err_len, RFAST_EINVAL, "%s: memory of device %d, but device %d is current", what, at.device, dev);
    return RFAST_OK;
}

AdamCoef adamw_coef(double lr, double beta1, double beta2, double eps, double weight_decay, int64_t t) {
    AdamCoef c;
    c.beta1 = (float)beta1; c.omb1 = (float)(1.0 - beta1);
    c.beta2 = (float)beta2; c.root_beta2 = (float)std::sqrt(beta2); c.root_omb2 = (float)std::sqrt(1.0 - beta2);
    c.eps = (float)eps; c.keep = (float)(1.0 - lr * weight_decay);
    c.step = (float)(lr / (1.0 - std::pow(beta1, (double)t)));
    c.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)t)));
    return c;
}

cudaError_t adamw_rows_launch(const AdamRows& r, const AdamCoef& c, int state_bits, int n_events, cudaStream_t st) {
    const int64_t blocks = (r.p + kAdamBlock - 1) / kAdamBlock;
    const int run = run_length(blocks * n_events);
    const dim3 grid((unsigned)((blocks + run * kWarps - 1) / (run * kWarps)), n_events);
    if (state_bits == 8) k_adamw_rows<true><<<grid, kThreadsOp, 0, st>>>(r, c, run);
    else k_adamw_rows<false><<<grid, kThreadsOp, 0, st>>>(r, c, run);
    return cudaGetLastError();
}

}  // namespace rfast

using namespace rfast;

extern "C" int rfast_adamw_step(const rfast_adamw* a, void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_adamw_step";
    if (!a) return op_fail(err, err_len, RFAST_EINVAL, "%s: null arguments", me);
    if (a->n_tensors < 0) return op_fail(err, err_len, RFAST_EINVAL, "%s: n_tensors is negative", me);
    if (!known_type(a->param_type) || !known_type(a->grad_type)) return op_fail(err, err_len, RFAST_EINVAL, "%s: unknown type", me);
    if (a->state_bits != 32 && a->state_bits != 8) return op_fail(err, err_len, RFAST_EINVAL, "%s: state_bits must be 32 or 8", me);
    // negated comparisons refuse a NaN as well
    if (!(a->beta1 >= 0 && a->beta1 < 1) || !(a->beta2 >= 0 && a->beta2 < 1)) return op_fail(err, err_len, RFAST_EINVAL, "%s: beta1 and beta2 must be in [0, 1)", me);
    // down to the least normal number: the reciprocal of the denominator stays finite
    if (!((float)a->eps >= 1.17549435e-38f) || !std::isfinite((float)a->eps)) return op_fail(err, err_len, RFAST_EINVAL, "%s: eps must be at least 2^-126", me);
    if (!std::isfinite(a->lr) || !std::isfinite(a->weight_decay)) return op_fail(err, err_len, RFAST_EINVAL, "%s: lr and weight_decay must be finite", me);
    if (!a->d_step && a->step < 1) return op_fail(err, err_len, RFAST_EINVAL, "%s: step counts from 1", me);
    if ((uintptr_t)a->d_step % 8 || (uintptr_t)a->d_grad_scale % 4) return op_fail(err, err_len, RFAST_EINVAL, "%s: d_step or d_grad_scale is not aligned to its type", me);
    if (a->n_tensors == 0) return RFAST_OK;
    const bool s8 = a->state_bits == 8;
    if (!a->numel || !a->param || !a->grad || !a->m || !a->v || (s8 && (!a->m_scale || !a->v_scale)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: null array", me);
    int some = -1;
    const size_t pb = type_bytes(a->param_type), gb = type_bytes(a->grad_type);
    for (int k = 0; k < a->n_tensors; ++k) {
        const int64_t n = a->numel[k];
        if (n < 0 || n > ((int64_t)1 << 40)) return op_fail(err, err_len, RFAST_EINVAL, "%s: numel of tensor %d is out of range", me, k);
        if (n == 0) continue;
        if (!a->param[k] || !a->grad[k] || !a->m[k] || !a->v[k] || (s8 && (!a->m_scale[k] || !a->v_scale[k])))
            return op_fail(err, err_len, RFAST_EINVAL, "%s: tensor %d has a null address", me, k);
        if ((uintptr_t)a->param[k] % pb || (uintptr_t)a->grad[k] % gb || (!s8 && ((uintptr_t)a->m[k] % 4 || (uintptr_t)a->v[k] % 4)) ||
            (s8 && ((uintptr_t)a->m_scale[k] % 4 || (uintptr_t)a->v_scale[k] % 4)))
            return op_fail(err, err_len, RFAST_EINVAL, "%s: an address of tensor %d is not aligned to its type", me, k);
        if (some < 0) some = k;
    }
    if (some < 0) return RFAST_OK;
    const void* first[] = {a->param[some], a->grad[some], a->m[some], a->v[some], s8 ? a->m_scale[some] : nullptr, s8 ? a->v_scale[some] : nullptr, a->d_step, a->d_grad_scale};
    const char* names[] = {"param", "grad", "m", "v", "m_scale", "v_scale", "d_step", "d_grad_scale"};
    for (int k = 0; k < 8; ++k)
        if (first[k]) {
            char what[64];
            std::snprintf(what, sizeof what, "%s: %s", me, names[k]);
            const int rc = check_device_pointer(first[k], what, err, err_len);
            if (rc != RFAST_OK) return rc;
        }
    const AdamCoef c = adamw_coef(a->lr, a->beta1, a->beta2, a->eps, a->weight_decay, a->d_step ? 1 : a->step);
    for (int k0 = 0; k0 < a->n_tensors;) {
        // as many tensors as a table holds and a launch has thread blocks for, at one block per warp
        int k1 = k0;
        int64_t blocks = 0;                                  // of 256 values
        while (k1 < a->n_tensors && k1 - k0 < kMany) {
            const int64_t more = ((a->numel[k1] + kAdamBlock - 1) / kAdamBlock + kWarps - 1) / kWarps * kWarps;
            if (k1 > k0 && blocks + more > (int64_t)kWarps * 0x7fffffff) break;
            blocks += more;
            ++k1;
        }
        const int run = run_length(blocks);
        const cudaError_t e = k1 - k0 <= kFew ? adamw_span<kFew>(a, c, k0, k1, run, (cudaStream_t)cuda_stream)
                                              : adamw_span<kMany>(a, c, k0, k1, run, (cudaStream_t)cuda_stream);
        if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
        k0 = k1;
    }
    return RFAST_OK;
}

extern "C" int rfast_grad_norm(int32_t n_tensors, int32_t grad_type, const int64_t* numel, const void* const* grad, float max_norm,
                               float* d_norm, float* d_scale, void* workspace, size_t workspace_bytes, void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_grad_norm";
    if (n_tensors < 0) return op_fail(err, err_len, RFAST_EINVAL, "%s: n_tensors is negative", me);
    if (!known_type(grad_type)) return op_fail(err, err_len, RFAST_EINVAL, "%s: unknown type", me);
    if (!d_norm && !d_scale) return op_fail(err, err_len, RFAST_EINVAL, "%s: neither d_norm nor d_scale is given", me);
    if (d_scale && !(max_norm > 0)) return op_fail(err, err_len, RFAST_EINVAL, "%s: max_norm must be positive", me);
    if (!workspace || (uintptr_t)workspace % 8) return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace must be given, aligned to 8 bytes", me);
    if (workspace_bytes < RFAST_GRAD_NORM_WORKSPACE) return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace needs %d bytes", me, RFAST_GRAD_NORM_WORKSPACE);
    if ((uintptr_t)d_norm % 4 || (uintptr_t)d_scale % 4) return op_fail(err, err_len, RFAST_EINVAL, "%s: an output is not aligned to its type", me);
    if (n_tensors > 0 && (!numel || !grad)) return op_fail(err, err_len, RFAST_EINVAL, "%s: null array", me);
    int some = -1;
    for (int k = 0; k < n_tensors; ++k) {
        if (numel[k] < 0 || numel[k] > ((int64_t)1 << 40)) return op_fail(err, err_len, RFAST_EINVAL, "%s: numel of tensor %d is out of range", me, k);
        if (numel[k] == 0) continue;
        if (!grad[k]) return op_fail(err, err_len, RFAST_EINVAL, "%s: tensor %d has a null address", me, k);
        if ((uintptr_t)grad[k] % type_bytes(grad_type)) return op_fail(err, err_len, RFAST_EINVAL, "%s: the address of tensor %d is not aligned to its type", me, k);
        if (some < 0) some = k;
    }
    const int launches = (n_tensors + kNormMany - 1) / kNormMany;
    if (launches > kNormParts) return op_fail(err, err_len, RFAST_EINVAL, "%s: too many tensors", me);
    const void* ptrs[] = {some >= 0 ? grad[some] : nullptr, d_norm, d_scale, workspace};
    const char* names[] = {"rfast_grad_norm: grad", "rfast_grad_norm: d_norm", "rfast_grad_norm: d_scale", "rfast_grad_norm: workspace"};
    for (int k = 0; k < 4; ++k)
        if (ptrs[k]) {
            const int rc = check_device_pointer(ptrs[k], names[k], err, err_len);
            if (rc != RFAST_OK) return rc;
        }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    double* part = (double*)workspace;
    int parts = 0;
    cudaError_t e = cudaSuccess;
    const NormOut out{max_norm, d_norm, d_scale};
    for (int k0 = 0; (k0 < n_tensors || k0 == 0) && e == cudaSuccess; k0 += kNormMany) {
        const int k1 = n_tensors - k0 < kNormMany ? n_tensors : k0 + kNormMany;
        const int room = launches > 1 ? kNormParts / launches : kNormParts;
        const int most = room < kNormGrid ? room : kNormGrid;
        const NormOut* whole = launches <= 1 ? &out : nullptr;
        int blocks = 0;
        e = k1 - k0 <= kNormFew ? norm_pick<kNormFew>(grad_type, numel, grad, k0, k1, most, part + parts, whole, &blocks, st)
                                : norm_pick<kNormMany>(grad_type, numel, grad, k0, k1, most, part + parts, whole, &blocks, st);
        if (blocks < 0 && e == cudaSuccess) return RFAST_OK;
        parts += blocks;
    }
    if (e == cudaSuccess) {
        // the closing kernel is on its way while the sums are formed; it waits for them before it reads
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(1); cfg.blockDim = dim3(kThreadsOp); cfg.stream = st;
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &at; cfg.numAttrs = parts > 0 ? 1 : 0;
        e = cudaLaunchKernelEx(&cfg, k_grad_norm_end, (const double*)part, parts, max_norm, d_norm, d_scale);
    }
    if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
    return RFAST_OK;
}
