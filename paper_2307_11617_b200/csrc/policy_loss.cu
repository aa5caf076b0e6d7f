// Clipped policy loss with a KL term, out of logits, and its gradient (see rfast_policy_loss in rfast.h for the formulas).
//
// A row of logits is a team's work: a warp's for short rows, a thread block's for long ones.  The first pass holds a running
// maximum and sum of each thread's values (one pass, rescaled where the maximum grows), which are merged in a fixed order; one
// thread forms the row's numbers in 64 bits; the second pass writes the gradient, reading the logits again.  That second read
// finds them in the L2 cache, so that memory sees each logit once in and each gradient once out, which is what bounds it.
//
// Powers are taken of two: exp((z - c) / T) = 2^(z k - c') with k = log2(e) / T in fp32 and c' the rounded z_max k.  k is the only
// constant that both passes and the row's numbers share, so rounding it is a change of T by 2^-25 of itself and nothing else.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdio>

#include "ops.h"
#include "values.cuh"

namespace rfast {

namespace {

constexpr int kBlockTeam = 1024;             // threads of a long row's block
constexpr int kAhead = 4;                    // groups of eight logits that a thread has on their way
constexpr int64_t kShortRow = 2048;          // up to so many logits a warp does the row

struct Policy {
    const void* logits;
    const void* tokens;
    const float *old_logp, *ref_logp, *advantage, *weight, *scale;
    float *token_loss, *logp;
    void* dlogits;
    int64_t rows, vocab, in_stride, out_stride;
    int wide_tokens;
    float k;                           // log2(e) / T
    double ln2k;                       // ln 2, of which k makes 1 / T
    float inv_t;
    double clip_lo, clip_hi, kl;       // 1 - clip_low, 1 + clip_high
};

__device__ __forceinline__ float two_to(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Running maximum and sum of 2^(z k - max k) over what a thread has seen.
struct Run {
    float top, sum;
};
// The reference of exponents: the rounded product of the maximum and k (never one exact in a multiply-add), 0 where there is no
// maximum yet.
__device__ __forceinline__ float base_of(float top, float k) { return top == -INFINITY ? 0.f : __fmul_rn(top, k); }
// The factor that takes a sum to the reference c.  A run that saw nothing but -infinity and NaN keeps its sum, 0 or NaN.
__device__ __forceinline__ float rescale(float top, float c, float k) { return top == -INFINITY ? 1.f : two_to(__fmul_rn(top, k) - c); }
__device__ __forceinline__ Run merged(Run a, Run b, float k) {
    Run r;
    r.top = fmaxf(a.top, b.top);
    const float c = base_of(r.top, k);
    r.sum = a.sum * rescale(a.top, c, k) + b.sum * rescale(b.top, c, k);
    return r;
}
template <int N>
__device__ __forceinline__ void take(Run& r, const float (&v)[N], float k) {
    float top = r.top;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, v[i]);
    const float c = base_of(top, k);
    float sum = top > r.top ? r.sum * rescale(r.top, c, k) : r.sum;
#pragma unroll
    for (int i = 0; i < N; ++i) sum += two_to(fmaf(v[i], k, -c));
    r.top = top;
    r.sum = sum;
}

// What the second pass needs of a row: the gradient is p * 2^(z k - base), at the token plus `slope`.
struct RowOut {
    float base, p, slope;
    int live;
};

// One thread: the row's loss and slope, in 64 bits, from the merged run and the token's logit.
__device__ __forceinline__ RowOut row_numbers(const Policy& a, int64_t row, Run r, float zt) {
    const double base = (double)base_of(r.top, a.k);
    const double logp = a.ln2k * ((double)zt * (double)a.k - base - log2((double)r.sum));
    const double adv = a.advantage[row], w = a.weight ? (double)a.weight[row] : 1.0;
    const double ratio = exp(logp - (double)a.old_logp[row]);
    const double held = ratio < a.clip_lo ? a.clip_lo : ratio > a.clip_hi ? a.clip_hi : ratio;
    const double one = ratio * adv, two = held * adv;
    const bool pass = !(one > two);                         // a NaN passes
    double loss = pass ? -one : -two, slope = pass ? -one : 0.0;
    if (a.ref_logp) {
        const double d = (double)a.ref_logp[row] - logp, e = expm1(d);
        loss += a.kl * (e - d);
        slope -= a.kl * e;
    }
    if (a.token_loss) a.token_loss[row] = (float)(w * loss);
    if (a.logp) a.logp[row] = (float)logp;
    slope *= w * (a.scale ? (double)*a.scale : 1.0) * (double)a.inv_t;
    RowOut o;
    o.base = (float)base;
    o.p = (float)(-slope / (double)r.sum);
    o.slope = (float)slope;
    o.live = 1;
    return o;
}

// A row cut at multiples of eight values' size: `head` values, then groups of eight, then the rest.  ALIGN: logits and gradients
// begin at the same place within a group, so that the groups are whole in both.
template <class T> __device__ __forceinline__ int head_of(const T* p, int64_t n) {
    constexpr uintptr_t kGroup = 8 * sizeof(T);
    const int h = (int)(((kGroup - ((uintptr_t)p & (kGroup - 1))) & (kGroup - 1)) / sizeof(T));
    return h < n ? h : (int)n;
}

template <class T, int TEAM, bool ALIGN>
__device__ __forceinline__ void policy_row(const Policy& a, int64_t row, int tid, Run* sh_run, RowOut* sh_out) {
    const T* z = (const T*)a.logits + row * a.in_stride;
    T* dz = a.dlogits ? (T*)a.dlogits + row * a.out_stride : nullptr;
    const int64_t t = a.wide_tokens ? ((const int64_t*)a.tokens)[row] : (int64_t)((const int*)a.tokens)[row];
    const int64_t n = a.vocab;
    const bool live = t >= 0 && t < n && !(a.weight && a.weight[row] == 0.f);
    const float k = a.k;
    if (!live) {
        if (tid == 0) {
            if (a.token_loss) a.token_loss[row] = 0.f;
            if (a.logp) a.logp[row] = 0.f;
        }
        if (!dz) return;
        const int head = head_of(dz, n);
        const int64_t groups = (n - head) / 8;
        const float zero[8] = {};
        if (tid < head) dz[tid] = rounded<T>(0.f);
        for (int64_t g = tid; g < groups; g += TEAM) store8(dz + head + g * 8, zero);
        for (int64_t i = head + groups * 8 + tid; i < n; i += TEAM) dz[i] = rounded<T>(0.f);
        return;
    }
    const int head = head_of(z, n);
    const int64_t groups = (n - head) / 8;
    const float zt = tid == 0 ? value_of(z[t]) : 0.f;
    Run r{-INFINITY, 0.f};
    {
        const T* g0 = z + head;
        for (int64_t g = tid; g < groups; g += kAhead * TEAM) {
            Raw8<T> q[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (g + u * TEAM < groups) q[u] = load8(g0 + (g + u * TEAM) * 8);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (g + u * TEAM < groups) {
                    float v[8];
                    unpack8(q[u], v);
                    take(r, v, k);
                }
        }
        if (tid < head) { const float v[1] = {value_of(z[tid])}; take(r, v, k); }
        for (int64_t i = head + groups * 8 + tid; i < n; i += TEAM) { const float v[1] = {value_of(z[i])}; take(r, v, k); }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Run b;
        b.top = __shfl_xor_sync(0xffffffffu, r.top, o);
        b.sum = __shfl_xor_sync(0xffffffffu, r.sum, o);
        r = merged(r, b, k);
    }
    RowOut out;
    if (TEAM == 32) {
        if (tid == 0) out = row_numbers(a, row, r, zt);
        out.base = __shfl_sync(0xffffffffu, out.base, 0);
        out.p = __shfl_sync(0xffffffffu, out.p, 0);
        out.slope = __shfl_sync(0xffffffffu, out.slope, 0);
    } else {
        if ((tid & 31) == 0) sh_run[tid >> 5] = r;
        __syncthreads();
        if (tid < 32) {
            r = tid < TEAM / 32 ? sh_run[tid] : Run{-INFINITY, 0.f};
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                Run b;
                b.top = __shfl_xor_sync(0xffffffffu, r.top, o);
                b.sum = __shfl_xor_sync(0xffffffffu, r.sum, o);
                r = merged(r, b, k);
            }
            if (tid == 0) *sh_out = row_numbers(a, row, r, zt);
        }
        __syncthreads();
        out = *sh_out;
    }
    if (!dz) return;
    const auto slope_of = [&](float v, int64_t i) {
        const float p = out.p * two_to(fmaf(v, k, -out.base));
        return i == t ? out.slope + p : p;
    };
    if (ALIGN) {
        const T* g0 = z + head;
        T* d0 = dz + head;
        for (int64_t g = tid; g < groups; g += kAhead * TEAM) {
            Raw8<T> q[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (g + u * TEAM < groups) q[u] = load8(g0 + (g + u * TEAM) * 8);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (g + u * TEAM < groups) {
                    float v[8];
                    unpack8(q[u], v);
                    const int64_t i0 = head + (g + u * TEAM) * 8;
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = out.p * two_to(fmaf(v[j], k, -out.base));
                    if ((uint64_t)(t - i0) < 8) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] += i0 + j == t ? out.slope : 0.f;
                    }
                    store8(d0 + (g + u * TEAM) * 8, v);
                }
        }
        if (tid < head) dz[tid] = rounded<T>(slope_of(value_of(z[tid]), tid));
        for (int64_t i = head + groups * 8 + tid; i < n; i += TEAM) dz[i] = rounded<T>(slope_of(value_of(z[i]), i));
    } else {
        for (int64_t i = tid; i < n; i += TEAM) dz[i] = rounded<T>(slope_of(value_of(z[i]), i));
    }
}

template <class T, bool ALIGN>
__global__ void __launch_bounds__(256)
k_policy_warp(const __grid_constant__ Policy a) {
    let_follow();
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < a.rows; row += (int64_t)gridDim.x * 8)
        policy_row<T, 32, ALIGN>(a, row, threadIdx.x & 31, nullptr, nullptr);
}

template <class T, bool ALIGN>
__global__ void __launch_bounds__(kBlockTeam, 2)
k_policy_block(const __grid_constant__ Policy a) {
    __shared__ Run sh_run[kBlockTeam / 32];
    __shared__ RowOut sh_out;
    let_follow();
    policy_row<T, kBlockTeam, ALIGN>(a, blockIdx.x, threadIdx.x, sh_run, &sh_out);
}

// The sum of the tokens' losses, in 64 bits and a fixed order.
__global__ void __launch_bounds__(1024)
k_policy_total(const float* __restrict__ token_loss, int64_t rows, float* __restrict__ loss) {
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

template <class T, bool ALIGN>
cudaError_t policy_launch(const Policy& a, cudaStream_t st) {
    if (a.vocab <= kShortRow) {
        const int64_t blocks = (a.rows + 7) / 8;
        return launch(k_policy_warp<T, ALIGN>, dim3((unsigned)(blocks < 0x7fffffff ? blocks : 0x7fffffff)), 256, 0, st, false, a);
    }
    return launch(k_policy_block<T, ALIGN>, dim3((unsigned)a.rows), kBlockTeam, 0, st, false, a);
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
        if (!p->d_old_logp || !p->d_advantage) return op_fail(err, err_len, RFAST_EINVAL, "%s: old_logp or advantage is null", me);
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
    a.k = (float)(1.4426950408889634 / p->temperature);
    a.ln2k = 0.6931471805599453;
    a.inv_t = (float)(1.0 / p->temperature);
    a.clip_lo = 1.0 - p->clip_low; a.clip_hi = 1.0 + p->clip_high; a.kl = p->kl_coef;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    if (p->tokens > 0) {
        // the offset within eight values is the same in every row of both
        const int64_t b = (int64_t)bytes_of(p->type);
        const bool align = !p->d_dlogits || (((uintptr_t)p->d_logits ^ (uintptr_t)p->d_dlogits) % (8 * b) == 0 &&
                                             (p->logits_stride - p->dlogits_stride) % 8 == 0);
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
