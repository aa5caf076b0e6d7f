// Embedding look-up and its gradient by sorted tokens (see rfast_embedding in rfast.h for the formulas).
//
// The gradient of a table row is the sum of the rows of dout that carry its token.  Tokens are sorted first (a stable radix
// sort of token and position), so that every sum runs over neighbours in the sorted order, in the order of the positions,
// without atomics: the same inputs give the same bits.  Then a warp owns some rows of the table and 256 columns, finds its
// rows' runs in `start`, adds up in fp32 and writes each value once, zeros of unused rows among them.  What bounds it is
// memory: dout is read once and the table's gradient written once.
//
// Text uses some tokens thousands of times.  A run longer than a chunk (64 sorted places) is therefore cut at multiples of 64:
// chunks that lie wholly in one run are summed beforehand, by a warp each, and sixteen whole neighbours to one sum again, so
// that the row's owner adds at most 64 + 16 + tokens / 1024 + 16 + 64 rows one after the other.
#include <cuda_runtime.h>

#include <cstdio>

#include "ops.h"
#include "values.cuh"

namespace rfast {

namespace {

constexpr int kCols = 256;                   // columns of a warp: eight per lane
constexpr int kSortThreads = 256, kSortWarps = 8, kSortItems = 4;
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kDigitBits = 10, kDigits = 1 << kDigitBits;
constexpr int kSortBlocks = 64;              // every block reads the counts of all blocks: 64 keep that below 256 KB
constexpr int64_t kSortOne = 2048;           // up to so many tokens one block sorts in one launch
constexpr int kChunk = 64, kChunksPerSum = 16, kSpan = kChunk * kChunksPerSum;
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

// ---- sort ---------------------------------------------------------------------------------------
// Least significant digit first.  A key is the token, or `vocab` where there is none, so that those come last.
struct SortPass {
    const void* tokens;                // the first pass reads these, later ones keys_in and pos_in
    const uint32_t* keys_in;
    const int* pos_in;
    uint32_t* keys_out;
    int* pos_out;
    int* counts;                       // [digit][block]
    int64_t n, per_block, vocab;
    int wide_tokens, shift, bits;
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

__global__ void __launch_bounds__(kSortThreads)
k_sort_count(SortPass a) {
    __shared__ int sh[kDigits];
    follow();
    let_follow();
    const int64_t lo = blockIdx.x * a.per_block, hi = lo + a.per_block < a.n ? lo + a.per_block : a.n;
    sort_count(a, lo, hi, sh);
    for (int d = threadIdx.x; d < 1 << a.bits; d += kSortThreads) a.counts[d * gridDim.x + blockIdx.x] = sh[d];
}

struct SortShared {
    int at[kDigits];                   // where a digit's next token goes
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
    const int digits = 1 << a.bits, blocks = gridDim.x;
    int before[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int d = threadIdx.x * 4 + j;
        if (d >= digits) continue;
        int all = 0;
        for (int b = 0; b < blocks; ++b) {
            const int c = a.counts[d * blocks + b];
            all += c;
            if (b < (int)blockIdx.x) before[j] += c;
        }
        sh.at[d] = all;
    }
    __syncthreads();
    sort_starts(sh, before, digits);
    const int64_t lo = blockIdx.x * a.per_block, hi = lo + a.per_block < a.n ? lo + a.per_block : a.n;
    sort_place(a, lo, hi, sh);
}

// All passes in one block.  keys / pos: two buffers each; the sorted ones end in buffer (passes - 1) & 1.
__global__ void __launch_bounds__(kSortThreads)
k_sort_one(SortPass a, uint32_t* keys1, int* pos1, int passes) {
    __shared__ SortShared sh;
    uint32_t* const keys[2] = {a.keys_out, keys1};
    int* const pos[2] = {a.pos_out, pos1};
    let_follow();
    for (int p = 0; p < passes; ++p) {
        SortPass b = a;
        b.shift = p * a.bits;
        if (p) { b.tokens = nullptr; b.keys_in = keys[(p - 1) & 1]; b.pos_in = pos[(p - 1) & 1]; }
        b.keys_out = keys[p & 1];
        b.pos_out = pos[p & 1];
        sort_count(b, 0, b.n, sh.at);
        const int before[4] = {0, 0, 0, 0};
        sort_starts(sh, before, 1 << b.bits);
        sort_place(b, 0, b.n, sh);
    }
}

// ---- sums ---------------------------------------------------------------------------------------
struct EmbSums {
    const uint32_t* keys;              // sorted
    const int* order;                  // their positions
    int* start;                        // [vocab + 1] first sorted place of a token
    float *chunk, *span;               // sums of whole chunks and of sixteen of them, [..][pitch]
    int64_t n, vocab, dout_stride, table_stride;
    int width, pitch, col_tiles, rows_per_warp, bound_blocks, accumulate;
    float scale;
};

// Eight columns of a lane, of the rows order[i .. j) of dout, added in order: neighbours where WIDE, 32 apart elsewhere.
template <class DT, bool WIDE>
__device__ __forceinline__ void add_rows(const EmbSums& a, const DT* __restrict__ dout, int64_t i, int64_t j, int c0, float (&acc)[8]) {
    const int lane = threadIdx.x & 31;
    for (; i < j; i += 32) {
        const int take = j - i < 32 ? (int)(j - i) : 32;
        const int mine = lane < take ? a.order[i + lane] : 0;
        for (int k = 0; k < take; k += 4) {
            const DT* p[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) p[u] = dout + (int64_t)__shfl_sync(0xffffffffu, mine, (k + u) & 31) * a.dout_stride;
            if (WIDE) {
                Raw8<DT> r[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (k + u < take && c0 < a.width) r[u] = load8(p[u] + c0);
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (k + u < take && c0 < a.width) {
                        float v[8];
                        unpack8(r[u], v);
#pragma unroll
                        for (int q = 0; q < 8; ++q) acc[q] += v[q];
                    }
            } else {
                float v[4][8];
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[u][q] = k + u < take && c0 + 32 * q < a.width ? value_of(p[u][c0 + 32 * q]) : 0.f;
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (k + u < take)
#pragma unroll
                        for (int q = 0; q < 8; ++q) acc[q] += v[u][q];
            }
        }
    }
}
template <bool WIDE>
__device__ __forceinline__ void add_sums(const EmbSums& a, const float* __restrict__ from, int64_t i, int64_t j, int c0, float (&acc)[8]) {
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

// The first blocks find `start`, one token per thread; the others sum whole chunks, a warp each, and whole spans.
template <class DT, bool WIDE>
__global__ void __launch_bounds__(512)
k_emb_chunks(EmbSums a, const DT* __restrict__ dout) {
    __shared__ float sh[kChunksPerSum][kCols];
    follow();
    let_follow();
    if ((int)blockIdx.x < a.bound_blocks) {
        const int64_t v = (int64_t)blockIdx.x * 512 + threadIdx.x;
        if (v > a.vocab) return;
        int64_t lo = 0, hi = a.n;                           // the first place whose key is not below v
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (a.keys[mid] < (uint32_t)v) lo = mid + 1; else hi = mid;
        }
        a.start[v] = (int)lo;
        return;
    }
    const int64_t job = blockIdx.x - a.bound_blocks;
    const int64_t s = job / a.col_tiles;
    const int tile = (int)(job - s * a.col_tiles), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c0 = tile * kCols + (WIDE ? lane * 8 : lane);
    const int64_t c = s * kChunksPerSum + warp, i = c * kChunk;
    float acc[8] = {};
    if (i + kChunk <= a.n) {
        const uint32_t key = a.keys[i];
        if (key == a.keys[i + kChunk - 1] && key < (uint32_t)a.vocab) {
            add_rows<DT, WIDE>(a, dout, i, i + kChunk, c0, acc);
            float* to = a.chunk + c * a.pitch;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int col = WIDE ? c0 + q : c0 + 32 * q;
                if (col < a.width) to[col] = acc[q];
            }
        }
    }
    const int64_t s0 = s * kSpan;
    if (s0 + kSpan > a.n) return;
    const uint32_t key = a.keys[s0];
    if (key != a.keys[s0 + kSpan - 1] || key >= (uint32_t)a.vocab) return;      // the whole block alike
#pragma unroll
    for (int q = 0; q < 8; ++q) sh[warp][WIDE ? lane * 8 + q : lane + 32 * q] = acc[q];
    __syncthreads();
    if (threadIdx.x < kCols && tile * kCols + (int)threadIdx.x < a.width) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kChunksPerSum; ++w) sum += sh[w][threadIdx.x];
        a.span[s * a.pitch + tile * kCols + threadIdx.x] = sum;
    }
}

template <class DT, class TT, bool WIDE>
__global__ void __launch_bounds__(256)
k_emb_rows(EmbSums a, const DT* __restrict__ dout, TT* __restrict__ dtable) {
    follow();
    const int lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t group = w / a.col_tiles;
    const int tile = (int)(w - group * a.col_tiles);
    const int64_t v0 = group * a.rows_per_warp;
    if (v0 >= a.vocab) return;
    const int rows = a.vocab - v0 < a.rows_per_warp ? (int)(a.vocab - v0) : a.rows_per_warp;
    const int mine = lane <= rows ? a.start[v0 + lane] : 0;
    const int c0 = tile * kCols + (WIDE ? lane * 8 : lane);
    for (int r = 0; r < rows; ++r) {
        int64_t i = __shfl_sync(0xffffffffu, mine, r);
        const int64_t j = __shfl_sync(0xffffffffu, mine, r + 1);
        if (a.accumulate && i == j) continue;
        float acc[8] = {};
        if (j - i > kChunk) {
            const int64_t head = (i + kChunk - 1) / kChunk * kChunk;
            add_rows<DT, WIDE>(a, dout, i, head, c0, acc);
            const int64_t c1 = j / kChunk;
            int64_t c = head / kChunk;
            // whole chunks up to a whole span, whole spans, the chunks behind them
            const int64_t s = (c + kChunksPerSum - 1) / kChunksPerSum, s1 = c1 / kChunksPerSum;
            if (s < s1) {
                add_sums<WIDE>(a, a.chunk, c, s * kChunksPerSum, c0, acc);
                add_sums<WIDE>(a, a.span, s, s1, c0, acc);
                c = s1 * kChunksPerSum;
            }
            add_sums<WIDE>(a, a.chunk, c, c1, c0, acc);
            i = c1 > head / kChunk ? c1 * kChunk : head;
        }
        add_rows<DT, WIDE>(a, dout, i, j, c0, acc);
        TT* to = dtable + (v0 + r) * a.table_stride;
        if (WIDE) {
            if (c0 < a.width) {
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
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int col = c0 + 32 * q;
                if (col < a.width) to[col] = rounded<TT>(a.accumulate ? fmaf(acc[q], a.scale, value_of(to[col])) : acc[q] * a.scale);
            }
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------
struct EmbRoom {
    int64_t keys[2], pos[2], counts, start, chunk, span, total;      // offsets in bytes
    int pitch;
};
EmbRoom emb_room(const rfast_emb_shape& s) {
    EmbRoom r;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) { const int64_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    r.pitch = (s.width + 7) / 8 * 8;
    for (int k = 0; k < 2; ++k) { r.keys[k] = take(4 * s.tokens); r.pos[k] = take(4 * s.tokens); }
    r.counts = take(4 * (int64_t)kDigits * kSortBlocks);
    r.start = take(4 * (s.vocab + 1));
    r.chunk = take(4 * (s.tokens / kChunk) * r.pitch);
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
    return width % 8 == 0 && (uintptr_t)p % 16 == 0 && stride * (int64_t)bytes_of(type) % 16 == 0;
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
cudaError_t sums(const EmbSums& a, const void* dout, void* dtable, cudaStream_t st, bool after) {
    const int64_t spans = a.n / kChunk > 0 ? (a.n + kSpan - 1) / kSpan : 0;
    const int64_t blocks = a.bound_blocks + spans * a.col_tiles;
    cudaError_t e = launch(k_emb_chunks<DT, WIDE>, dim3((unsigned)blocks), 512, 0, st, after, a, (const DT*)dout);
    if (e != cudaSuccess) return e;
    const int64_t groups = (a.vocab + a.rows_per_warp - 1) / a.rows_per_warp;
    return launch(k_emb_rows<DT, TT, WIDE>, dim3((unsigned)((groups * a.col_tiles + 7) / 8)), 256, 0, st, true, a, (const DT*)dout, (TT*)dtable);
}
template <class DT, class TT>
cudaError_t sums_types(const EmbSums& a, const void* dout, void* dtable, bool wide, cudaStream_t st, bool after) {
    return wide ? sums<DT, TT, true>(a, dout, dtable, st, after) : sums<DT, TT, false>(a, dout, dtable, st, after);
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
    const int64_t n = shape->tokens;
    if (n > 0 && (!d_tokens || (uintptr_t)d_tokens % (shape->token_bits / 8)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: tokens are null or not aligned to their type", me);
    if (n > 0 && (fault = emb_rows_fault(d_dout, shape->out_type, dout_stride, n, shape->width, false)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: dout %s", me, fault);
    if ((fault = emb_rows_fault(d_dtable, shape->table_type, dtable_stride, shape->vocab, shape->width, true)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: dtable %s", me, fault);
    const EmbRoom room = emb_room(*shape);
    if (!workspace || (uintptr_t)workspace % 16) return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace must be given, aligned to 16 bytes", me);
    if (workspace_bytes < (size_t)room.total)
        return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace needs %lld bytes", me, (long long)room.total);
    if (n == 0 && accumulate) return RFAST_OK;
    const int64_t col_tiles = (shape->width + kCols - 1) / kCols;
    const int rows_per_warp = shape->vocab * col_tiles >= (int64_t)8 * 148 * 32 ? 8 : 1;    // few rows: a warp each
    const int64_t bound_blocks = (shape->vocab + 1 + 511) / 512;
    if ((shape->vocab / rows_per_warp + 1) * col_tiles / 8 >= 0x7fffffff || bound_blocks + (n / kSpan + 1) * col_tiles >= 0x7fffffff)
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
    p.counts = (int*)(base + room.counts);
    cudaError_t e = cudaSuccess;
    if (n > 0 && n <= kSortOne) {
        p.tokens = d_tokens;
        p.keys_out = keys[0];
        p.pos_out = pos[0];
        p.per_block = n;
        e = launch(k_sort_one, dim3(1), kSortThreads, 0, st, false, p, keys[1], pos[1], passes);
    } else if (n > 0) {
        const int64_t want = (n + kSortOne - 1) / kSortOne;
        const int64_t blocks = want < kSortBlocks ? want : kSortBlocks;
        p.per_block = (n + blocks - 1) / blocks;
        const int64_t used = (n + p.per_block - 1) / p.per_block;
        for (int k = 0; k < passes && e == cudaSuccess; ++k) {
            p.shift = k * p.bits;
            p.tokens = k ? nullptr : d_tokens;
            p.keys_in = k ? keys[(k - 1) & 1] : nullptr;
            p.pos_in = k ? pos[(k - 1) & 1] : nullptr;
            p.keys_out = keys[k & 1];
            p.pos_out = pos[k & 1];
            e = launch(k_sort_count, dim3((unsigned)used), kSortThreads, 0, st, k > 0, p);
            if (e == cudaSuccess) e = launch(k_sort_place, dim3((unsigned)used), kSortThreads, 0, st, true, p);
        }
    }
    if (e == cudaSuccess) {
        EmbSums a{};
        a.keys = keys[(passes - 1) & 1];
        a.order = pos[(passes - 1) & 1];
        a.start = (int*)(base + room.start);
        a.chunk = (float*)(base + room.chunk);
        a.span = (float*)(base + room.span);
        a.n = n;
        a.vocab = shape->vocab;
        a.dout_stride = dout_stride;
        a.table_stride = dtable_stride;
        a.width = shape->width;
        a.pitch = room.pitch;
        a.col_tiles = (int)col_tiles;
        a.rows_per_warp = rows_per_warp;
        a.bound_blocks = (int)bound_blocks;
        a.accumulate = accumulate != 0;
        a.scale = scale;
        const bool wide = emb_wide(d_dtable, shape->table_type, dtable_stride, shape->width) && (n == 0 || emb_wide(d_dout, shape->out_type, dout_stride, shape->width));
        e = RFAST_TWO_TYPES(sums_types, shape->out_type, shape->table_type, a, d_dout, d_dtable, wide, st, n > 0);
    }
    if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
    return RFAST_OK;
}
