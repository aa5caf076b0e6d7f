// Embedding look-up and its gradient by sorted tokens (see rfast_embedding in rfast.h for the formulas).
//
// The gradient of a table row is the sum of the rows of dout that carry its token.  Tokens are sorted first (a stable radix
// sort of token and position), so that every sum runs over neighbours in the sorted order, in the order of the positions,
// without atomics: the same inputs give the same bits.  What bounds it is memory: dout is read once and the table's gradient
// written once (65536 of 131072 x 2048 bf16: 169 us, sums and zeros at 5.2 and 5.4 TB/s behind 25 us of sorting).
//
// Text uses some tokens thousands of times and most of a table's never, so work is shared out by sorted places, not by rows:
// a warp takes a chunk of 16 places and 256 columns, adds up in fp32 with eight rows on their way, and writes the rows whose
// run lies in its chunk.  Of a run that crosses a chunk's border it leaves the piece's sum, and the sum of sixteen chunks that lie in one
// run.  A last kernel writes zeros where a token does not occur and adds up the pieces of the runs that cross: two, and the
// chunks between them, at most 15 + tokens / 256 + 15.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdio>

#include "ops.h"
#include "values.cuh"

namespace rfast {

namespace {

constexpr int kCols = 256;                   // columns of a warp: eight per lane
constexpr int kShort = 256;                  // columns up to which a look-up's rows are not a warp's each (90000 x 64 f32 to bf16: 31 -> 8 us); a
                                             // quarter of it where values go one at a time
constexpr int kSortThreads = 256, kSortWarps = 8, kSortItems = 4;
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kDigitBits = 10, kDigits = 1 << kDigitBits;
constexpr int kSortBlocks = 64;              // every block reads the counts of all blocks: 64 keep that below 256 KB
constexpr int64_t kSortOne = 2048;           // up to so many tokens one block sorts in shared memory, in one launch
constexpr int kChunk = 16, kChunksPerSum = 16, kSpan = kChunk * kChunksPerSum;
constexpr int kFlight = 8;                   // rows of dout on their way at once
constexpr int64_t kMaxTokens = (int64_t)1 << 30, kMaxVocab = (int64_t)1 << 30;
constexpr int64_t kMaxWidth = (int64_t)1 << 24;

// ---- look-up ------------------------------------------------------------------------------------
// A warp takes one row's 1024 (wide) or 256 columns; four loads of a lane are on their way at once.
template <class I, class TT, class OT, bool WIDE>
__global__ void __launch_bounds__(256)
k_embedding(const I* __restrict__ tokens, const TT* __restrict__ table, int64_t table_stride, OT* __restrict__ out, int64_t out_stride, int64_t n,
            int64_t vocab, int width, int parts, float scale) {
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * 8;
    for (int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); w < n * parts; w += warps) {
        const int64_t i = w / parts;
        const int part = (int)(w - i * parts);
        const int64_t t = (int64_t)tokens[i];
        const bool some = t >= 0 && t < vocab;
        const TT* src = table + (some ? t : 0) * table_stride;
        OT* dst = out + i * out_stride;
        if (WIDE) {
            const int c0 = part * 1024 + lane * 8;
            Raw8<TT> r[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (some && c0 + u * 256 < width) r[u] = load8(src + c0 + u * 256);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c0 + u * 256 < width) {
                    float v[8];
                    if (some) {
                        unpack8(r[u], v);
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] *= scale;
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = 0.f;
                    }
                    store8(dst + c0 + u * 256, v);
                }
        } else {
            const int c0 = part * kCols + lane;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = some && c0 + 32 * k < width ? value_of(src[c0 + 32 * k]) * scale : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c0 + 32 * k < width) dst[c0 + 32 * k] = rounded<OT>(v[k]);
        }
    }
}

// Short rows: lanes go from one to the next, four values (WIDE: groups of eight) of a thread on their way.  L: 32 bits where all are counted
// in them.
template <class I, class TT, class OT, bool WIDE, class L>
__global__ void __launch_bounds__(256)
k_embedding_short(const I* __restrict__ tokens, const TT* __restrict__ table, int64_t table_stride, OT* __restrict__ out, int64_t out_stride, L all, int64_t vocab,
                  unsigned per, float scale) {
    constexpr int kOf = WIDE ? 8 : 1;
    const L step = (L)gridDim.x * 256;
    for (L at = (L)blockIdx.x * 1024 + threadIdx.x; at < all; at += step * 4) {
        const TT* src[4];
        OT* dst[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const L v = at + (L)u * 256;
            src[u] = nullptr;
            dst[u] = nullptr;
            if (v < all) {
                const L row = v / per;
                const int c = (int)(v - row * per) * kOf;
                const int64_t t = (int64_t)tokens[row];
                if (t >= 0 && t < vocab) src[u] = table + t * table_stride + c;
                dst[u] = out + (int64_t)row * out_stride + c;
            }
        }
        if constexpr (WIDE) {
            Raw8<TT> r[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (src[u]) r[u] = load8(src[u]);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (dst[u]) {
                    float v[8] = {};
                    if (src[u]) {
                        unpack8(r[u], v);
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] *= scale;
                    }
                    store8(dst[u], v);
                }
        } else {
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = src[u] ? value_of(*src[u]) * scale : 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (dst[u]) *dst[u] = rounded<OT>(v[u]);
        }
    }
}

// ---- sort ---------------------------------------------------------------------------------------
// Least significant digit first.  A key is the token, or `vocab` where there is none, so that those come last.
struct SortPass {
    const void* tokens;                // the first pass reads these, later ones keys_in and pos_in
    const uint32_t* keys_in;
    const int* pos_in;
    uint32_t* keys_out;
    int* pos_out;
    int* counts;                       // [block][digit]
    int2* range;                       // [vocab] of sorted places, cleared beside the first pass
    int64_t n, per_block, vocab;
    int wide_tokens, shift, bits, blocks;
};
__device__ __forceinline__ uint32_t sort_key(const SortPass& a, int64_t i) {
    if (!a.tokens) return a.keys_in[i];
    const int64_t t = a.wide_tokens ? ((const int64_t*)a.tokens)[i] : (int64_t)((const int*)a.tokens)[i];
    return t >= 0 && t < a.vocab ? (uint32_t)t : (uint32_t)a.vocab;
}

__device__ __forceinline__ void sort_count(const SortPass& a, int64_t lo, int64_t hi, int* sh) {
    const int digits = 1 << a.bits;
    for (int d = threadIdx.x; d < digits; d += kSortThreads) sh[d] = 0;
    __syncthreads();
    for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads) atomicAdd(&sh[(sort_key(a, i) >> a.shift) & (digits - 1)], 1);
    __syncthreads();
}

// Thread blocks from `first` on clear the ranges.
__device__ __forceinline__ void clear_ranges(const SortPass& a, int first) {
    const int64_t step = (int64_t)(gridDim.x - first) * kSortThreads;
    for (int64_t v = (int64_t)(blockIdx.x - first) * kSortThreads + threadIdx.x; v < a.vocab; v += step) a.range[v] = make_int2(0, 0);
}

__global__ void __launch_bounds__(kSortThreads)
k_sort_count(SortPass a) {
    __shared__ int sh[kDigits];
    follow();
    let_follow();
    if ((int)blockIdx.x >= a.blocks) { clear_ranges(a, a.blocks); return; }
    const int64_t lo = blockIdx.x * a.per_block, hi = lo + a.per_block < a.n ? lo + a.per_block : a.n;
    sort_count(a, lo, hi, sh);
    for (int d = threadIdx.x; d < 1 << a.bits; d += kSortThreads) a.counts[(blockIdx.x << a.bits) + d] = sh[d];
}

struct SortShared {
    int at[kDigits];                   // where a digit's next token goes
    int before[kDigits];
    int warp[kSortWarps][kDigits];
    int sums[kSortWarps];
};

// at[] holds the digits' counts over all blocks; `before[j]` those of earlier blocks, of digits 4 tid + j.
__device__ __forceinline__ void sort_starts(SortShared& sh, const int (&before)[4], int digits) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d0 = threadIdx.x * 4;
    int own[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        own[j] = sum;
        if (d0 + j < digits) sum += sh.at[d0 + j];
    }
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += u;
    }
    if (lane == 31) sh.sums[warp] = run;
    __syncthreads();
    int first = run - sum;
    for (int w = 0; w < warp; ++w) first += sh.sums[w];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (d0 + j < digits) sh.at[d0 + j] = first + own[j] + before[j];
    __syncthreads();
}

// Places [lo, hi) in order: lanes of one digit rank themselves by a match, warps by their counts.
__device__ __forceinline__ void sort_place(const SortPass& a, int64_t lo, int64_t hi, SortShared& sh) {
    const int digits = 1 << a.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int64_t t0 = lo; t0 < hi; t0 += kSortTile) {
        for (int q = threadIdx.x; q < kSortWarps * digits; q += kSortThreads) sh.warp[q >> a.bits][q & (digits - 1)] = 0;
        __syncthreads();
        uint32_t key[kSortItems];
        int pos[kSortItems], rank[kSortItems];
#pragma unroll
        for (int s = 0; s < kSortItems; ++s) {
            const int64_t i = t0 + warp * (32 * kSortItems) + s * 32 + lane;
            const bool in = i < hi;
            key[s] = in ? sort_key(a, i) : 0;
            pos[s] = in ? (a.tokens ? (int)i : a.pos_in[i]) : -1;
        }
#pragma unroll
        for (int s = 0; s < kSortItems; ++s) {
            const int d = (int)((key[s] >> a.shift) & (digits - 1));
            const unsigned peers = __match_any_sync(0xffffffffu, pos[s] >= 0 ? d : -1);
            const int ahead = __popc(peers & ((1u << lane) - 1));
            const int old = sh.warp[warp][d];
            rank[s] = old + ahead;
            __syncwarp();
            if (pos[s] >= 0 && ahead == 0) sh.warp[warp][d] = old + __popc(peers);
            __syncwarp();
        }
        __syncthreads();
        for (int d = threadIdx.x; d < digits; d += kSortThreads) {
            int run = sh.at[d];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                const int c = sh.warp[w][d];
                sh.warp[w][d] = run;
                run += c;
            }
            sh.at[d] = run;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kSortItems; ++s)
            if (pos[s] >= 0) {
                const int to = sh.warp[warp][(key[s] >> a.shift) & (digits - 1)] + rank[s];
                a.keys_out[to] = key[s];
                a.pos_out[to] = pos[s];
            }
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kSortThreads)
k_sort_place(SortPass a) {
    __shared__ SortShared sh;
    follow();
    let_follow();
    // the counts of all blocks, and of those before this one: four digits a thread, the blocks shared out among threads
    const int digits = 1 << a.bits, quads = digits / 4;      // two bits at least
    for (int d = threadIdx.x; d < digits; d += kSortThreads) sh.at[d] = sh.before[d] = 0;
    __syncthreads();
    {
        const int q = threadIdx.x % quads, share = threadIdx.x / quads, shares = kSortThreads / quads;
        int all[4] = {0, 0, 0, 0}, ahead[4] = {0, 0, 0, 0};
        for (int b0 = share; b0 < a.blocks; b0 += 16 * shares) {
            int4 c[16];                                     // on their way together
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                const int b = b0 + u * shares;
                c[u] = b < a.blocks ? *reinterpret_cast<const int4*>(a.counts + (b << a.bits) + q * 4) : make_int4(0, 0, 0, 0);
            }
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                all[0] += c[u].x; all[1] += c[u].y; all[2] += c[u].z; all[3] += c[u].w;
                if (b0 + u * shares < (int)blockIdx.x) { ahead[0] += c[u].x; ahead[1] += c[u].y; ahead[2] += c[u].z; ahead[3] += c[u].w; }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (all[j]) atomicAdd(&sh.at[q * 4 + j], all[j]);
            if (ahead[j]) atomicAdd(&sh.before[q * 4 + j], ahead[j]);
        }
    }
    __syncthreads();
    int before[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) before[j] = threadIdx.x * 4 + j < digits ? sh.before[threadIdx.x * 4 + j] : 0;
    __syncthreads();
    sort_starts(sh, before, digits);
    const int64_t lo = blockIdx.x * a.per_block, hi = lo + a.per_block < a.n ? lo + a.per_block : a.n;
    sort_place(a, lo, hi, sh);
}

// All passes in one block, keys and positions in shared memory in between (generic addresses serve both).
struct SortOne {
    SortShared sh;
    uint32_t keys[2][kSortOne];
    int pos[2][kSortOne];
};
__global__ void __launch_bounds__(kSortThreads)
k_sort_one(SortPass a, int passes) {
    extern __shared__ __align__(16) uint8_t raw[];
    SortOne& s = *reinterpret_cast<SortOne*>(raw);
    let_follow();
    if (blockIdx.x > 0) { clear_ranges(a, 1); return; }
    for (int p = 0; p < passes; ++p) {
        SortPass b = a;
        b.shift = p * a.bits;
        if (p) { b.tokens = nullptr; b.keys_in = s.keys[(p - 1) & 1]; b.pos_in = s.pos[(p - 1) & 1]; }
        if (p + 1 < passes) { b.keys_out = s.keys[p & 1]; b.pos_out = s.pos[p & 1]; }
        sort_count(b, 0, b.n, s.sh.at);
        const int before[4] = {0, 0, 0, 0};
        sort_starts(s.sh, before, 1 << b.bits);
        sort_place(b, 0, b.n, s.sh);
    }
}

// ---- sums ---------------------------------------------------------------------------------------
struct EmbSums {
    const uint32_t* keys;              // sorted
    const int* order;                  // their positions
    int2* range;                       // [vocab] sorted places of a token, none: {0, 0}
    float *chunk, *tail, *span;        // [..][pitch] sums of chunks: of the first run, if it began before (all of the chunk, perhaps); of the
                                       // last, if it goes on; of sixteen chunks in one run
    int64_t n, vocab, dout_stride, table_stride;
    int width, pitch, col_tiles, rows_per_warp, accumulate;
    float scale;
};

// Eight columns of a lane, of `take` <= kFlight rows of dout: neighbours where WIDE, 32 apart elsewhere.  The position of row k is in
// lane (first + k) of `mine`.
template <class DT, bool WIDE>
struct Flight {
    Raw8<DT> r[kFlight];
    __device__ __forceinline__ void load(const EmbSums& a, const DT* __restrict__ dout, int mine, int first, int take, int c0) {
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const DT* p = dout + (int64_t)__shfl_sync(0xffffffffu, mine, (first + k) & 31) * a.dout_stride;
            if (k < take && c0 < a.width) r[k] = load8(p + c0);
        }
    }
    __device__ __forceinline__ void add(int k, float (&acc)[8]) const {
        float v[8];
        unpack8(r[k], v);
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[q] += v[q];
    }
};
template <class DT>
struct Flight<DT, false> {
    DT r[kFlight][8];
    __device__ __forceinline__ void load(const EmbSums& a, const DT* __restrict__ dout, int mine, int first, int take, int c0) {
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const DT* p = dout + (int64_t)__shfl_sync(0xffffffffu, mine, (first + k) & 31) * a.dout_stride;
#pragma unroll
            for (int q = 0; q < 8; ++q) r[k][q] = k < take && c0 + 32 * q < a.width ? p[c0 + 32 * q] : rounded<DT>(0.f);
        }
    }
    __device__ __forceinline__ void add(int k, float (&acc)[8]) const {
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[q] += value_of(r[k][q]);
    }
};
// Sums [i, j) of a list of them, one after the other.  MANY: eight are fetched at once, for long runs (90000 tokens of 3, 64 columns: the
// gradient in 28 us, not 39).  Elsewhere the registers would be missed by the warps that write zeros (65536 of 131072 x 2048 bf16: 262 us, not 169).
template <bool WIDE, bool MANY>
__device__ __forceinline__ void add_sums(const EmbSums& a, const float* __restrict__ from, int64_t i, int64_t j, int c0, float (&acc)[8]) {
    if constexpr (MANY) {
        for (; i < j; i += 8) {
            float r[8][8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float* p = from + (i + u) * a.pitch;
                if (WIDE) {
                    if (i + u < j && c0 < a.width) unpack8(load8(p + c0), r[u]);
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q) r[u][q] = i + u < j && c0 + 32 * q < a.width ? p[c0 + 32 * q] : 0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i + u < j && c0 < a.width)
#pragma unroll
                    for (int q = 0; q < 8; ++q) acc[q] += r[u][q];
        }
    } else {
#pragma unroll 4
        for (; i < j; ++i) {
            const float* p = from + i * a.pitch;
            if (WIDE) {
                if (c0 < a.width) {
                    float v[8];
                    unpack8(load8(p + c0), v);
#pragma unroll
                    for (int q = 0; q < 8; ++q) acc[q] += v[q];
                }
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) acc[q] += c0 + 32 * q < a.width ? p[c0 + 32 * q] : 0.f;
            }
        }
    }
}

// One row of the gradient: scale acc, on top of what is there if that is wanted.
template <class TT, bool WIDE>
__device__ __forceinline__ void put_row(const EmbSums& a, TT* __restrict__ to, int c0, const float (&acc)[8]) {
    if (WIDE) {
        if (c0 >= a.width) return;
        float v[8];
        if (a.accumulate) {
            unpack8(load8(to + c0), v);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = fmaf(acc[q], a.scale, v[q]);
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = acc[q] * a.scale;
        }
        store8(to + c0, v);
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int col = c0 + 32 * q;
            if (col < a.width) to[col] = rounded<TT>(a.accumulate ? fmaf(acc[q], a.scale, value_of(to[col])) : acc[q] * a.scale);
        }
    }
}

template <bool WIDE>
__device__ __forceinline__ void put_sum(const EmbSums& a, float* __restrict__ to, int c0, const float (&acc)[8]) {
    if (WIDE) {
        if (c0 >= a.width) return;
        uint32_t r[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) r[q] = __float_as_uint(acc[q]);
        store32(to + c0, r);
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (c0 + 32 * q < a.width) to[c0 + 32 * q] = acc[q];
    }
}

// What lies before and behind the chunk decides what becomes of its first and last run.
template <class DT, class TT, bool WIDE>
__global__ void __launch_bounds__(256, sizeof(DT) == 4 || !WIDE ? 2 : 3)
k_emb_chunks(EmbSums a, const DT* __restrict__ dout, TT* __restrict__ dtable) {
    __shared__ float sh[kChunksPerSum / 2][kCols];
    follow();
    let_follow();
    const int64_t s = blockIdx.x / a.col_tiles;
    const int tile = (int)(blockIdx.x - s * a.col_tiles), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c0 = tile * kCols + (WIDE ? lane * 8 : lane);
    const uint32_t none = (uint32_t)a.vocab;
    float both[8] = {};                                     // of two whole chunks, for the span
    for (int h = 0; h < 2; ++h) {
        const int64_t c = s * kChunksPerSum + warp * 2 + h, i = c * kChunk;
        if (i >= a.n) break;
        const bool in = lane < kChunk && i + lane < a.n;
        const uint32_t key = in ? a.keys[i + lane] : none;
        const int mine = in ? a.order[i + lane] : 0;
        uint32_t before = __shfl_up_sync(0xffffffffu, key, 1), after = __shfl_down_sync(0xffffffffu, key, 1);
        if (lane == 0) before = i > 0 ? a.keys[i - 1] : none;
        if (lane == kChunk - 1) after = i + kChunk < a.n ? a.keys[i + kChunk] : none;
        const int places = __popc(__ballot_sync(0xffffffffu, key < none));               // those without a token come last
        const unsigned ends = __ballot_sync(0xffffffffu, key < none && after != key);     // last places of runs
        const bool goes_on = __shfl_sync(0xffffffffu, before == key, 0);                  // the first run began before the chunk
        if (tile == 0 && key < none) {
            if (before != key) a.range[key].x = (int)(i + lane);
            if (after != key) a.range[key].y = (int)(i + lane) + 1;
        }
        if (places == 0) break;
        float acc[8] = {};
        bool first = goes_on;                               // the run at hand is the rest of an earlier one
#pragma unroll 1
        for (int k = 0; k < places; k += kFlight) {
            const int take = places - k < kFlight ? places - k : kFlight;
            Flight<DT, WIDE> f;
            f.load(a, dout, mine, k, take, c0);
#pragma unroll
            for (int u = 0; u < kFlight; ++u) {
                if (u >= take) break;
                f.add(u, acc);
                if (ends >> (k + u) & 1) {
                    const int64_t row = __shfl_sync(0xffffffffu, key, k + u);
                    if (first) put_sum<WIDE>(a, a.chunk + c * a.pitch, c0, acc);
                    else put_row<TT, WIDE>(a, dtable + row * a.table_stride, c0, acc);
                    first = false;
                    if (ends == 1u << (kChunk - 1)) break;            // a whole chunk: the span wants its sum
#pragma unroll
                    for (int q = 0; q < 8; ++q) acc[q] = 0.f;
                }
            }
        }
        if (!(ends >> (places - 1) & 1)) {                  // the last run goes on: all of the chunk, or its tail
            put_sum<WIDE>(a, (first || !ends ? a.chunk : a.tail) + c * a.pitch, c0, acc);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) both[q] += acc[q];
    }
    const int64_t s0 = s * kSpan;
    if (s0 + kSpan > a.n) return;
    const uint32_t key = a.keys[s0];
    if (key != a.keys[s0 + kSpan - 1] || key >= none) return;                            // the whole block alike
#pragma unroll
    for (int q = 0; q < 8; ++q) sh[warp][WIDE ? lane * 8 + q : lane + 32 * q] = both[q];
    __syncthreads();
    if (tile * kCols + (int)threadIdx.x < a.width) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kChunksPerSum / 2; ++w) sum += sh[w][threadIdx.x];
        a.span[s * a.pitch + tile * kCols + threadIdx.x] = sum;
    }
}

// Zeros for tokens that do not occur, sums of the pieces of runs that cross a chunk's border.
template <class TT, bool WIDE, bool MANY>
__global__ void __launch_bounds__(256)
k_emb_rows(EmbSums a, TT* __restrict__ dtable) {
    follow();
    const int lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t group = w / a.col_tiles;
    const int tile = (int)(w - group * a.col_tiles);
    const int64_t v0 = group * a.rows_per_warp;
    if (v0 >= a.vocab) return;
    const int rows = a.vocab - v0 < a.rows_per_warp ? (int)(a.vocab - v0) : a.rows_per_warp;
    const int2 mine = lane < rows ? a.range[v0 + lane] : make_int2(0, 0);
    const int c0 = tile * kCols + (WIDE ? lane * 8 : lane);
    const unsigned some = __ballot_sync(0xffffffffu, mine.x < mine.y);
    if (!a.accumulate) {
        const float zero[8] = {};
        for (int r = 0; r < rows; ++r)
            if (!(some >> r & 1)) put_row<TT, WIDE>(a, dtable + (v0 + r) * a.table_stride, c0, zero);
    }
    unsigned cross = __ballot_sync(0xffffffffu, mine.x < mine.y && mine.x / kChunk != (mine.y - 1) / kChunk);
    for (; cross; cross &= cross - 1) {
        const int r = __ffs(cross) - 1;
        const int begin = __shfl_sync(0xffffffffu, mine.x, r), end = __shfl_sync(0xffffffffu, mine.y, r);
        float acc[8] = {};
        int64_t c = begin / kChunk;
        if (begin % kChunk) { add_sums<WIDE, MANY>(a, a.tail, c, c + 1, c0, acc); ++c; }
        const int64_t whole = end / kChunk, all = (end + kChunk - 1) / kChunk;           // chunks that the run fills end before `whole`
        const int64_t s = (c + kChunksPerSum - 1) / kChunksPerSum;
        const int64_t s1 = whole / kChunksPerSum;
        if (s < s1) {
            add_sums<WIDE, MANY>(a, a.chunk, c, s * kChunksPerSum, c0, acc);
            add_sums<WIDE, MANY>(a, a.span, s, s1, c0, acc);
            c = s1 * kChunksPerSum;
        }
        add_sums<WIDE, MANY>(a, a.chunk, c, all, c0, acc);
        put_row<TT, WIDE>(a, dtable + (v0 + r) * a.table_stride, c0, acc);
    }
}

// ---- host ---------------------------------------------------------------------------------------
struct EmbRoom {
    int64_t keys[2], pos[2], counts, range, chunk, tail, span, total;      // offsets in bytes
    int pitch;
};
EmbRoom emb_room(const rfast_emb_shape& s) {
    EmbRoom r;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) { const int64_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    r.pitch = (s.width + 7) / 8 * 8;
    for (int k = 0; k < 2; ++k) { r.keys[k] = take(4 * s.tokens); r.pos[k] = take(4 * s.tokens); }
    r.counts = take(4 * (int64_t)kDigits * kSortBlocks);
    r.range = take(8 * s.vocab);
    const int64_t chunks = (s.tokens + kChunk - 1) / kChunk;
    r.chunk = take(4 * chunks * r.pitch);
    r.tail = take(4 * chunks * r.pitch);
    r.span = take(4 * (s.tokens / kSpan) * r.pitch);
    r.total = at;
    return r;
}

const char* emb_shape_fault(const rfast_emb_shape* s) {
    if (!s) return "null shape";
    if (s->tokens < 0 || s->tokens > kMaxTokens) return "tokens must be in [0, 2^30]";
    if (s->vocab < 1 || s->vocab > kMaxVocab) return "vocab must be in [1, 2^30]";
    if (s->width < 1 || s->width > kMaxWidth) return "width must be in [1, 2^24]";
    if (s->token_bits != 32 && s->token_bits != 64) return "token_bits must be 32 or 64";
    if (!is_type(s->table_type) || !is_type(s->out_type)) return "unknown type";
    return nullptr;
}

// Rows of `rows` times `width` values at `p`: null, alignment, stride.  A written operand's rows may not meet.
const char* emb_rows_fault(const void* p, int type, int64_t stride, int64_t rows, int width, bool written) {
    if (!p) return "is null";
    if ((uintptr_t)p % bytes_of(type)) return "is not aligned to its type";
    if (stride < 0 || (written && rows > 1 && stride < width)) return "has rows that overlap (its stride is negative or too small)";
    if (stride > ((int64_t)1 << 56) / (rows > 0 ? rows : 1)) return "spans more than 2^56 elements";
    return nullptr;
}
bool emb_wide(const void* p, int type, int64_t stride, int width) {
    const int64_t b = (int64_t)bytes_of(type);
    return width % 8 == 0 && (uintptr_t)p % (8 * b) == 0 && stride % 8 == 0;
}

struct EmbCall {
    const rfast_emb_shape* s;
    const void* tokens;
    const void* in;                    // table or dout
    int64_t in_stride;
    void* out;                         // out or dtable
    int64_t out_stride;
    float scale;
    bool wide;
    cudaStream_t st;
};

template <class I, class TT, class OT, bool WIDE>
cudaError_t look_up(const EmbCall& c) {
    if (c.s->width <= (WIDE ? kShort : kShort / 4)) {
        const int of = WIDE ? 8 : 1;
        const unsigned in_row = (unsigned)(c.s->width / of);
        const int64_t all = c.s->tokens * in_row, blocks = (all + 1023) / 1024;
        const dim3 grid((unsigned)(blocks < 0x7fffffff ? blocks : 0x7fffffff));
        if (all < (int64_t)1 << 31)
            return launch(k_embedding_short<I, TT, OT, WIDE, uint32_t>, grid, 256, 0, c.st, false, (const I*)c.tokens, (const TT*)c.in, c.in_stride, (OT*)c.out, c.out_stride,
                          (uint32_t)all, c.s->vocab, in_row, c.scale);
        return launch(k_embedding_short<I, TT, OT, WIDE, uint64_t>, grid, 256, 0, c.st, false, (const I*)c.tokens, (const TT*)c.in, c.in_stride, (OT*)c.out, c.out_stride,
                      (uint64_t)all, c.s->vocab, in_row, c.scale);
    }
    const int per = WIDE ? 1024 : kCols;
    const int parts = (c.s->width + per - 1) / per;
    const int64_t blocks = (c.s->tokens * parts + 7) / 8;
    return launch(k_embedding<I, TT, OT, WIDE>, dim3((unsigned)(blocks < 0x7fffffff ? blocks : 0x7fffffff)), 256, 0, c.st, false, (const I*)c.tokens, (const TT*)c.in,
                  c.in_stride, (OT*)c.out, c.out_stride, c.s->tokens, c.s->vocab, c.s->width, parts, c.scale);
}
template <class TT, class OT>
cudaError_t look_up_types(const EmbCall& c) {
    if (c.s->token_bits == 32) return c.wide ? look_up<int, TT, OT, true>(c) : look_up<int, TT, OT, false>(c);
    return c.wide ? look_up<int64_t, TT, OT, true>(c) : look_up<int64_t, TT, OT, false>(c);
}

template <class DT, class TT, bool WIDE>
cudaError_t sums(const EmbSums& a, const void* dout, void* dtable, cudaStream_t st) {
    const int64_t blocks = (a.n + kSpan - 1) / kSpan * a.col_tiles;
    if (blocks > 0) {
        const cudaError_t e = launch(k_emb_chunks<DT, TT, WIDE>, dim3((unsigned)blocks), 256, 0, st, true, a, (const DT*)dout, (TT*)dtable);
        if (e != cudaSuccess) return e;
    }
    const int64_t groups = (a.vocab + a.rows_per_warp - 1) / a.rows_per_warp;
    const dim3 grid((unsigned)((groups * a.col_tiles + 7) / 8));
    // a token has eight places on average: long runs and few zeros
    if (a.n >= 8 * a.vocab) return launch(k_emb_rows<TT, WIDE, true>, grid, 256, 0, st, true, a, (TT*)dtable);
    return launch(k_emb_rows<TT, WIDE, false>, grid, 256, 0, st, true, a, (TT*)dtable);
}
template <class DT, class TT>
cudaError_t sums_types(const EmbSums& a, const void* dout, void* dtable, bool wide, cudaStream_t st) {
    return wide ? sums<DT, TT, true>(a, dout, dtable, st) : sums<DT, TT, false>(a, dout, dtable, st);
}

}  // namespace

}  // namespace rfast

using namespace rfast;

// f<first type, second type>(args), by the two types' numbers
#define RFAST_TWO_TYPES(f, one, two, ...)                                                                                     \
    ((one) == RFAST_TYPE_F32    ? ((two) == RFAST_TYPE_F32    ? f<float, float>(__VA_ARGS__)                                  \
                                   : (two) == RFAST_TYPE_BF16 ? f<float, __nv_bfloat16>(__VA_ARGS__)                          \
                                                              : f<float, __half>(__VA_ARGS__))                                \
     : (one) == RFAST_TYPE_BF16 ? ((two) == RFAST_TYPE_F32    ? f<__nv_bfloat16, float>(__VA_ARGS__)                          \
                                   : (two) == RFAST_TYPE_BF16 ? f<__nv_bfloat16, __nv_bfloat16>(__VA_ARGS__)                  \
                                                              : f<__nv_bfloat16, __half>(__VA_ARGS__))                        \
                                : ((two) == RFAST_TYPE_F32    ? f<__half, float>(__VA_ARGS__)                                 \
                                   : (two) == RFAST_TYPE_BF16 ? f<__half, __nv_bfloat16>(__VA_ARGS__)                         \
                                                              : f<__half, __half>(__VA_ARGS__)))

extern "C" int rfast_embedding(const rfast_emb_shape* shape, const void* d_tokens, const void* d_table, int64_t table_stride, float scale, void* d_out,
                               int64_t out_stride, void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_embedding";
    const char* fault = emb_shape_fault(shape);
    if (fault) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s", me, fault);
    if (!std::isfinite(scale)) return op_fail(err, err_len, RFAST_EINVAL, "%s: scale must be finite", me);
    if (shape->tokens == 0) return RFAST_OK;
    if (!d_tokens || (uintptr_t)d_tokens % (shape->token_bits / 8)) return op_fail(err, err_len, RFAST_EINVAL, "%s: tokens are null or not aligned to their type", me);
    if ((fault = emb_rows_fault(d_table, shape->table_type, table_stride, shape->vocab, shape->width, false)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: table %s", me, fault);
    if ((fault = emb_rows_fault(d_out, shape->out_type, out_stride, shape->tokens, shape->width, true)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: out %s", me, fault);
    const void* ptrs[] = {d_tokens, d_table, d_out};
    const char* names[] = {"rfast_embedding: tokens", "rfast_embedding: table", "rfast_embedding: out"};
    for (int k = 0; k < 3; ++k) {
        const int rc = check_device_pointer(ptrs[k], names[k], err, err_len);
        if (rc != RFAST_OK) return rc;
    }
    const bool wide = emb_wide(d_table, shape->table_type, table_stride, shape->width) && emb_wide(d_out, shape->out_type, out_stride, shape->width);
    const EmbCall c{shape, d_tokens, d_table, table_stride, d_out, out_stride, scale, wide, (cudaStream_t)cuda_stream};
    const cudaError_t e = RFAST_TWO_TYPES(look_up_types, shape->table_type, shape->out_type, c);
    if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
    return RFAST_OK;
}

extern "C" int64_t rfast_embedding_workspace(const rfast_emb_shape* shape) {
    return emb_shape_fault(shape) ? RFAST_EINVAL : emb_room(*shape).total;
}

extern "C" int rfast_embedding_backward(const rfast_emb_shape* shape, const void* d_tokens, const void* d_dout, int64_t dout_stride, float scale, int accumulate,
                                        void* d_dtable, int64_t dtable_stride, void* workspace, size_t workspace_bytes, void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_embedding_backward";
    const char* fault = emb_shape_fault(shape);
    if (fault) return op_fail(err, err_len, RFAST_EINVAL, "%s: %s", me, fault);
    if (!std::isfinite(scale)) return op_fail(err, err_len, RFAST_EINVAL, "%s: scale must be finite", me);
    const int64_t n = shape->tokens;
    if (n > 0 && (!d_tokens || (uintptr_t)d_tokens % (shape->token_bits / 8)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: tokens are null or not aligned to their type", me);
    if (n > 0 && (fault = emb_rows_fault(d_dout, shape->out_type, dout_stride, n, shape->width, false)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: dout %s", me, fault);
    if ((fault = emb_rows_fault(d_dtable, shape->table_type, dtable_stride, shape->vocab, shape->width, true)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: dtable %s", me, fault);
    const EmbRoom room = emb_room(*shape);
    if (!workspace || (uintptr_t)workspace % 32) return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace must be given, aligned to 32 bytes", me);
    if (workspace_bytes < (size_t)room.total)
        return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace needs %lld bytes", me, (long long)room.total);
    if (n == 0 && accumulate) return RFAST_OK;
    const int64_t col_tiles = (shape->width + kCols - 1) / kCols;
    const int rows_per_warp = shape->vocab * col_tiles >= (int64_t)8 * 148 * 32 ? 8 : 1;    // few rows: a warp each
    if ((shape->vocab / rows_per_warp + 1) * col_tiles / 8 >= 0x7fffffff || (n / kSpan + 1) * col_tiles >= 0x7fffffff)
        return op_fail(err, err_len, RFAST_EINVAL, "%s: more thread blocks than a launch takes", me);
    const void* ptrs[] = {n > 0 ? d_tokens : nullptr, n > 0 ? d_dout : nullptr, d_dtable, workspace};
    const char* names[] = {"rfast_embedding_backward: tokens", "rfast_embedding_backward: dout", "rfast_embedding_backward: dtable", "rfast_embedding_backward: workspace"};
    for (int k = 0; k < 4; ++k)
        if (ptrs[k]) {
            const int rc = check_device_pointer(ptrs[k], names[k], err, err_len);
            if (rc != RFAST_OK) return rc;
        }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    char* const base = (char*)workspace;
    uint32_t* const keys[2] = {(uint32_t*)(base + room.keys[0]), (uint32_t*)(base + room.keys[1])};
    int* const pos[2] = {(int*)(base + room.pos[0]), (int*)(base + room.pos[1])};
    // digits of equal length: ceil(bits / 10) passes over the bits of `vocab`, the largest key
    int bits = 1;
    while (shape->vocab >> bits) ++bits;
    const int passes = (bits + kDigitBits - 1) / kDigitBits;
    SortPass p{};
    p.n = n;
    p.vocab = shape->vocab;
    p.wide_tokens = shape->token_bits == 64;
    p.bits = (bits + passes - 1) / passes;
    if (p.bits < 2) p.bits = 2;
    p.counts = (int*)(base + room.counts);
    p.range = (int2*)(base + room.range);
    // blocks that clear the ranges: 2048 of them each, up to two per SM
    const int64_t clear = (shape->vocab + 2047) / 2048, clear_blocks = clear < 296 ? clear : 296;
    cudaError_t e = cudaSuccess;
    if (n <= kSortOne) {                                    // no tokens: the ranges are cleared all the same
        p.tokens = d_tokens;
        p.keys_out = keys[(passes - 1) & 1];
        p.pos_out = pos[(passes - 1) & 1];
        p.per_block = n;
        p.blocks = 1;
        e = cudaFuncSetAttribute(k_sort_one, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortOne));
        if (e == cudaSuccess) e = launch(k_sort_one, dim3(1 + (unsigned)clear_blocks), kSortThreads, sizeof(SortOne), st, false, p, passes);
    } else {
        const int64_t want = (n + kSortTile - 1) / kSortTile;
        const int64_t blocks = want < kSortBlocks ? want : kSortBlocks;
        p.per_block = (n + blocks - 1) / blocks;
        p.blocks = (int)((n + p.per_block - 1) / p.per_block);
        for (int k = 0; k < passes && e == cudaSuccess; ++k) {
            p.shift = k * p.bits;
            p.tokens = k ? nullptr : d_tokens;
            p.keys_in = k ? keys[(k - 1) & 1] : nullptr;
            p.pos_in = k ? pos[(k - 1) & 1] : nullptr;
            p.keys_out = keys[k & 1];
            p.pos_out = pos[k & 1];
            e = launch(k_sort_count, dim3((unsigned)(p.blocks + (k ? 0 : clear_blocks))), kSortThreads, 0, st, k > 0, p);
            if (e == cudaSuccess) e = launch(k_sort_place, dim3((unsigned)p.blocks), kSortThreads, 0, st, true, p);
        }
    }
    if (e == cudaSuccess) {
        EmbSums a{};
        a.keys = keys[(passes - 1) & 1];
        a.order = pos[(passes - 1) & 1];
        a.range = (int2*)(base + room.range);
        a.chunk = (float*)(base + room.chunk);
        a.tail = (float*)(base + room.tail);
        a.span = (float*)(base + room.span);
        a.n = n;
        a.vocab = shape->vocab;
        a.dout_stride = dout_stride;
        a.table_stride = dtable_stride;
        a.width = shape->width;
        a.pitch = room.pitch;
        a.col_tiles = (int)col_tiles;
        a.rows_per_warp = rows_per_warp;
        a.accumulate = accumulate != 0;
        a.scale = scale;
        const bool wide = emb_wide(d_dtable, shape->table_type, dtable_stride, shape->width) && (n == 0 || emb_wide(d_dout, shape->out_type, dout_stride, shape->width));
        e = RFAST_TWO_TYPES(sums_types, shape->out_type, shape->table_type, a, d_dout, d_dtable, wide, st);
    }
    if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
    return RFAST_OK;
}
