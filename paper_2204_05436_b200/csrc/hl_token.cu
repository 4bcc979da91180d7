// A token embedding: the scaled rows of tokens, and the gradient of the table, summed over the tokens of a row.
#include <math.h>

#include "hl_rows.cuh"

namespace hl {
namespace {

constexpr int kNT = 256;

__device__ __forceinline__ int64_t live_tokens(const int32_t* n_tokens, int64_t max_tokens) {
    return n_tokens ? min((int64_t)max(__ldg(n_tokens), 0), max_tokens) : max_tokens;
}

// ---- rows of tokens ---------------------------------------------------------------------------------------------------
// out[i] = scale * table[tokens[i]], W values at a time, U of them a thread, dealt out in turn over the rows.  Bound by memory: 16 384 rows
// of 2 048 bf16 17 us (67 MB written), 131 072 of 512 fp32 to bf16 34.6 (134 MB written, 70 read: 5.9 TB/s).
// (item / vectors: by 2^64 / vectors, rounded up; exact for less than 2^40 items and rows of less than 2^24 vectors)
template <typename TT, typename TO, int W, int U>
__global__ void __launch_bounds__(kNT) k_token_embed(const TT* __restrict__ table, int64_t ld_table, unsigned n_rows,
                                                     const int32_t* __restrict__ tokens, int64_t max_tokens, const int32_t* n_tokens,
                                                     float scale, TO* __restrict__ out, int64_t ld_out, int vectors,
                                                     unsigned long long inverse, int32_t* status) {
    const int64_t n = live_tokens(n_tokens, max_tokens), first = (int64_t)blockIdx.x * (kNT * U) + threadIdx.x;
    int64_t at[U];
    int column[U], token[U];
    Pack<TT, W> in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned long long item = first + u * kNT;
        at[u] = vectors == 1 ? item : __umul64hi(item, inverse);
        column[u] = (int)(item - at[u] * vectors) * W;
        token[u] = at[u] < n ? __ldg(&tokens[at[u]]) : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        in[u].zero();
        if ((unsigned)token[u] < n_rows) in[u].load(table + token[u] * ld_table + column[u]);
        else if (token[u] != -1 && status) set_status(status, HL_EBOUNDS);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (at[u] >= n) continue;
        float x[W];
        in[u].get(x);
        const bool there = (unsigned)token[u] < n_rows;
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = there ? x[i] * scale : 0.f;
        Pack<TO, W> v;
        v.set(x);
        v.store(out + at[u] * ld_out + column[u]);
    }
}

// The same for rows that begin anywhere: eight values a thread, from where the written row's 16-byte lines begin, so that all but
// those at its ends are written whole.  28 657 rows of 337 fp16, 339 apart: 11 us, 22 MB; two of three cycles issue an instruction (a value
// a thread: 23).
template <typename TT, typename TO>
__global__ void __launch_bounds__(kNT) k_token_embed_loose(const TT* __restrict__ table, int64_t ld_table, unsigned n_rows,
                                                           const int32_t* __restrict__ tokens, int64_t max_tokens,
                                                           const int32_t* n_tokens, float scale, int dim, TO* __restrict__ out,
                                                           int64_t ld_out, int vectors, unsigned long long inverse, int32_t* status) {
    const int64_t n = live_tokens(n_tokens, max_tokens);
    const unsigned long long item = (int64_t)blockIdx.x * kNT + threadIdx.x;
    const int64_t at = vectors == 1 ? item : __umul64hi(item, inverse);
    if (at >= n) return;
    TO* row = out + at * ld_out;
    const int c = (int)(item - at * vectors) * 8 - (int)(reinterpret_cast<uintptr_t>(row) & 15) / (int)sizeof(TO);
    if (c >= dim) return;
    const int token = __ldg(&tokens[at]);
    const bool there = (unsigned)token < n_rows;
    Loose<TT> in;
    in.zero();
    if (there) in.load(table + token * ld_table, c, dim);
    else if (token != -1 && status) set_status(status, HL_EBOUNDS);
    float x[8];
    in.get(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = there ? x[i] * scale : 0.f;
    Pack<TO, 8> v;
    v.set(x);
    if (c >= 0 && c + 8 <= dim) v.store(row + c);
    else store_some(row, c, dim, v);
}

// ---- the sort -----------------------------------------------------------------------------------------------------------
// Few tokens: a token's place is how many are below it, and equal ones in front of it; each is compared with all.  (Some 5 us of one
// kernel for 2 048, where a cluster's sort takes 12 whatever their number.)
constexpr int kFewTokens = 2048, kFewNT = 128;
__global__ void __launch_bounds__(kFewNT) k_token_rank(const int32_t* __restrict__ tokens, int max_tokens, const int32_t* n_tokens,
                                                       int n_rows, int32_t* __restrict__ sorted, int32_t* __restrict__ order,
                                                       int32_t* status) {
    __shared__ __align__(16) int32_t s_key[kFewTokens + 4];
    const int n = (int)live_tokens(n_tokens, max_tokens), me = blockIdx.x * kFewNT + threadIdx.x;
    if ((int)blockIdx.x * kFewNT >= n) return;
    for (int i = threadIdx.x; i < (n + 3) / 4 * 4; i += kFewNT) {
        const int t = i < n ? __ldg(&tokens[i]) : n_rows;        // (those that fill the last four up are behind all)
        const bool row = (unsigned)t < (unsigned)n_rows;
        if (!row && t != -1 && i == me && i < n && status) set_status(status, HL_EBOUNDS);
        s_key[i] = row ? t : n_rows;
    }
    __syncthreads();
    if (me >= n) return;
    const int key = s_key[me];
    int rank = 0;
    // keys in front of mine count if they are not above it, those behind if they are below it
    const int quads = me / 4;
#pragma unroll 4
    for (int i = 0; i < quads; ++i) {
        const int4 k = reinterpret_cast<const int4*>(s_key)[i];
        rank += (k.x <= key) + (k.y <= key) + (k.z <= key) + (k.w <= key);
    }
    for (int i = quads * 4; i < quads * 4 + 4; ++i) rank += i < me ? s_key[i] <= key : s_key[i] < key;
#pragma unroll 4
    for (int i = quads + 1; i < (n + 3) / 4; ++i) {
        const int4 k = reinterpret_cast<const int4*>(s_key)[i];
        rank += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
    }
    sorted[rank] = key;
    order[rank] = me;
}

// Many: pairs of row and place, for the sort by digits, whose counts are made here too.
__global__ void __launch_bounds__(kNT) k_token_pairs(const int32_t* __restrict__ tokens, int64_t max_tokens, const int32_t* n_tokens,
                                                     int n_rows, int32_t* __restrict__ keys, int32_t* __restrict__ vals,
                                                     int32_t* n_out, int passes, uint32_t* __restrict__ counts, int32_t* status) {
    __shared__ uint32_t s_counts[4 * 256];
    const int64_t n = live_tokens(n_tokens, max_tokens);
    if (blockIdx.x == 0 && threadIdx.x == 0) *n_out = (int32_t)n;
    for (int i = threadIdx.x; i < passes * 256; i += kNT) s_counts[i] = 0;
    __syncthreads();
    for (int64_t i = (int64_t)blockIdx.x * kNT + threadIdx.x; i < n; i += (int64_t)gridDim.x * kNT) {
        const int t = __ldg(&tokens[i]);
        const bool row = (unsigned)t < (unsigned)n_rows;
        if (!row && t != -1) set_status(status, HL_EBOUNDS);
        const int key = row ? t : n_rows;
        keys[i] = key;
        vals[i] = (int32_t)i;
        for (int p = 0; p < passes; ++p) atomicAdd(&s_counts[p * 256 + ((key >> (8 * p)) & 255)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < passes * 256; i += kNT)
        if (s_counts[i]) atomicAdd(&counts[i], s_counts[i]);
}

// ---- the table's gradient -------------------------------------------------------------------------------------------------
// The sorted tokens are cut into windows of `window`.  A group of P threads takes one, its columns W a thread, and adds up the
// gradients of each run of equal tokens.  A run inside the window goes to its row; of one that begins before the window or goes on
// behind it only a piece is known, which goes to memory: piece 2w is that of the run which began before window w, 2w + 1 that of the
// one that begins in it and goes on.  A second kernel adds the pieces of such a run up, in their order.  Rows without tokens are
// zeroed by CTAs of their own.  Bound by memory: 16 384 gradients of 2 048 bf16, summed into 32 000 rows of fp32, 58 us (67 MB in, 262 out:
// 5.7 TB/s) and 12 for the joined ones; 131 072 of 512 into 200 000 rows 95 (544 MB) and 19.  28 657 of 337 fp16, 339 apart: 20, where
// instructions and the latency of order, then row, are what bounds it, and 16.  LOOSE: rows that begin anywhere; a group is a warp at most then, eight columns a lane.
constexpr int kPieceStep = 8;          // a piece's columns are filled up to a multiple of this
__device__ __forceinline__ int64_t piece_pitch(int dim) { return (dim + kPieceStep - 1) / kPieceStep * kPieceStep; }

// first place in sorted[lo, hi) whose token is not below u
__device__ __forceinline__ int64_t not_below(const int32_t* __restrict__ sorted, int64_t lo, int64_t hi, int u) {
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (__ldg(&sorted[mid]) < u) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// row[c ..] = scale * sum (+ row).  LOOSE: by a whole warp, 256 columns from c - 8 * lane on, in the order of the lanes (s: [256]), or,
// without s, each thread by itself.
template <typename TT, int W, bool LOOSE>
__device__ __forceinline__ void put(TT* row, int c, int dim, const float (&sum)[W], float scale, bool accumulate, float* s) {
    if (LOOSE && !s) {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (c + i < dim) row[c + i] = from_float<TT>(scale * sum[i] + (accumulate ? as_float(row[c + i]) : 0.f));
    } else if constexpr (LOOSE) {
        const int lane = threadIdx.x & 31;
        __syncwarp();
        Pack<float, W> mine;
        mine.set(sum);
        mine.store(s + lane * W);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int k = c - lane * W + i * 32 + lane;
            if (k < dim) row[k] = from_float<TT>(scale * s[i * 32 + lane] + (accumulate ? as_float(row[k]) : 0.f));
        }
    } else {
        float x[W];
        Pack<TT, W> v;
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = scale * sum[i];
        if (accumulate) {
            float old[W];
            v.load(row + c);
            v.get(old);
#pragma unroll
            for (int i = 0; i < W; ++i) x[i] += old[i];
        }
        v.set(x);
        v.store(row + c);
    }
}

// The same by a whole warp, 32 places a step.
__device__ __forceinline__ int64_t not_below_by_warp(const int32_t* __restrict__ sorted, int64_t n, int u) {
    const int lane = threadIdx.x & 31;
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step - 1;           // the last of the lane's part
        const unsigned below = __ballot_sync(0xffffffffu, at < hi && __ldg(&sorted[min(at, n - 1)]) < u);
        const int parts = __popc(below);                         // (the first so many are wholly below)
        lo += parts * step;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}

// rows [first, last) that no token names become zeros
template <typename TT>
__device__ void zero_rows(const int32_t* __restrict__ sorted, int64_t n, int64_t first, int64_t last, int dim, TT* __restrict__ table,
                          int64_t ld) {
    __shared__ uint32_t s_there[kNT / 32];
    __shared__ int64_t s_range[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int64_t r0 = first; r0 < last; r0 += kNT) {
        const int64_t r1 = min(r0 + kNT, last);
        if (warp < 2) {
            const int64_t at = not_below_by_warp(sorted, n, (int)(warp ? r1 - 1 : r0));
            if (lane == 0) s_range[warp] = at;
        }
        if (threadIdx.x < kNT / 32) s_there[threadIdx.x] = 0;
        __syncthreads();
        const int64_t lo = s_range[0], hi = s_range[1];          // those of row r1 - 1 begin at hi
        if (hi - lo <= 4 * kNT) {
            for (int64_t i = lo + threadIdx.x; i < hi; i += kNT) {
                const unsigned r = (unsigned)(__ldg(&sorted[i]) - (int)r0);
                if (r < (unsigned)kNT) atomicOr(&s_there[r >> 5], 1u << (r & 31));
            }
        } else if (r0 + threadIdx.x < r1 - 1) {                  // (many tokens of few rows: a row a thread)
            const int64_t at = not_below(sorted, lo, hi, (int)(r0 + threadIdx.x));
            if (at < hi && __ldg(&sorted[at]) == (int)(r0 + threadIdx.x)) atomicOr(&s_there[warp], 1u << lane);
        }
        if (threadIdx.x == 0 && hi < n && __ldg(&sorted[hi]) == (int)(r1 - 1))
            atomicOr(&s_there[(r1 - 1 - r0) >> 5], 1u << ((r1 - 1 - r0) & 31));
        __syncthreads();
        const int rows = (int)(r1 - r0);
        if (dim * (int)sizeof(TT) >= 8192) {                     // (a row that gives the whole CTA something to do)
            for (int k = 0; k < rows; ++k)
                if (!((s_there[k >> 5] >> (k & 31)) & 1u)) zero_row(table + (r0 + k) * ld, dim, threadIdx.x, kNT);
        } else {
            const int L = dim * (int)sizeof(TT) <= 512 ? 8 : 32;                     // (lanes of a short row)
            for (int k = threadIdx.x / L; k < rows; k += kNT / L)
                if (!((s_there[k >> 5] >> (k & 31)) & 1u)) zero_row(table + (r0 + k) * ld, dim, threadIdx.x % L, L);
        }
        __syncthreads();
    }
}

// a thread's W values of a row
template <typename T, int W, bool LOOSE>
struct Values {
    std::conditional_t<LOOSE, Loose<T>, Pack<T, W>> v;
    __device__ __forceinline__ void load(const T* row, int c, int dim) {
        if constexpr (LOOSE) v.load(row, c, dim);
        else v.load(row + c);
    }
    __device__ __forceinline__ void get(float (&x)[W]) const { v.get(x); }
};

template <typename TG, typename TT, int W, int U, bool LOOSE>
__global__ void __launch_bounds__(kNT, LOOSE ? 3 : 2) k_token_sums(const int32_t* __restrict__ sorted, const int32_t* __restrict__ order,
                                                    int64_t max_tokens, const int32_t* n_tokens, int n_rows, int dim,
                                                    const TG* __restrict__ grad, int64_t ld_grad, float scale,
                                                    TT* __restrict__ table, int64_t ld_table, int accumulate, int window, int P,
                                                    int passes, int sum_ctas, int rows_per_cta, float* __restrict__ pieces) {
    static_assert(!LOOSE || W == 8, "eight columns a lane");
    __shared__ __align__(16) float s_put[LOOSE ? kNT * W : 4];
    let_next_start();
    const int64_t n = live_tokens(n_tokens, max_tokens);
    // (CTAs of the two kinds alternate, evenly, so that the ones' stores go along with the others' loads)
    const unsigned zeros = gridDim.x - sum_ctas;
    const unsigned zeros_before = zeros ? (unsigned)((unsigned long long)blockIdx.x * zeros / gridDim.x) : 0;
    if (zeros && (unsigned)((unsigned long long)(blockIdx.x + 1) * zeros / gridDim.x) > zeros_before) {
        const int64_t first = (int64_t)zeros_before * rows_per_cta;
        zero_rows<TT>(sorted, n, first, min(first + rows_per_cta, (int64_t)n_rows), dim, table, ld_table);
        return;
    }
    const int sub = threadIdx.x & (P - 1);
    const unsigned mine = blockIdx.x - zeros_before, group = mine / (unsigned)passes;       // (all columns of some windows, one pass after the other)
    const int64_t w = (int64_t)group * (kNT / P) + threadIdx.x / P, first = w * window;
    if (first >= n) return;
    const int begin = (int)first, end = (int)min(first + window, n);       // (there are less than 2^30 tokens)
    const int c = ((int)(mine - group * passes) * P + sub) * W;
    if (c >= dim && !(LOOSE && P == 32)) return;                 // (a warp that writes together stays together)
    float* s = LOOSE && P == 32 ? s_put + (threadIdx.x & ~31) * W : nullptr;
    float sum[W] = {};
    int run = __ldg(&sorted[begin]);
    bool open = begin > 0 && __ldg(&sorted[begin - 1]) == run;             // began before the window
    const auto flush = [&](bool goes_on) {
        if ((unsigned)run < (unsigned)n_rows) {
            if (open || goes_on) {
                if (c < dim) {
                    Pack<float, W> v;
                    v.set(sum);
                    v.store(pieces + (2 * w + (open ? 0 : 1)) * piece_pitch(dim) + c);
                }
            } else {
                put<TT, W, LOOSE>(table + run * ld_table, c, dim, sum, scale, accumulate, s);
            }
        }
#pragma unroll
        for (int i = 0; i < W; ++i) sum[i] = 0.f;
        open = false;
    };
    for (int i0 = begin; i0 < end; i0 += U) {
        int key[U], at[U];
        Values<TG, W, LOOSE> in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            key[u] = i0 + u < end ? __ldg(&sorted[i0 + u]) : run;
            at[u] = i0 + u < end ? __ldg(&order[i0 + u]) : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            in[u].v.zero();
            if ((unsigned)key[u] < (unsigned)n_rows && (unsigned)at[u] < (unsigned)n && c < dim)
                in[u].load(grad + at[u] * ld_grad, c, dim);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u >= end) break;
            if (key[u] != run) {
                flush(false);
                run = key[u];
            }
            float x[W];
            in[u].get(x);
#pragma unroll
            for (int i = 0; i < W; ++i) sum[i] += x[i];
        }
    }
    flush(end < n && __ldg(&sorted[end]) == run);
}

// Runs over several windows: their pieces.  A warp looks at one window, of which a run may begin there and go on, and adds up the run's
// pieces in order if it is short; what reaches over more than kShort windows is left to the CTA, whose warps take a part of the
// pieces each, in order, and add the parts up in order.  32 W columns a CTA.  (A CTA a window, most of which end at once: 30 us
// instead of 12 for 1 024 windows of 2 048 columns.)  Bound by latency: those 13 us, 1 876 windows of 337 ragged columns 9.5.
constexpr int kShort = 16;
// Pieces p0 .. p1 of the run that begins in window w.  A warp's groups of P lanes, which have all columns, take every so many of them
// and are added up by halves.
template <int W>
__device__ __forceinline__ void add_pieces(const float* __restrict__ pieces, int64_t pitch, int64_t w, int p0, int p1, int c, int dim, int P,
                                           float (&sum)[W]) {
    constexpr int U = 8;
    const int groups = 32 / P;
    const float* column = pieces + (c < dim ? c : 0);
    for (int p = p0 + (threadIdx.x & 31) / P; p < p1; p += U * groups) {
        float in[U][W];                // (asked for without a condition and in this order, so that all are on their way before one is added)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = min(p + u * groups, p1 - 1);
            const float* from = column + (2 * (w + at) + (at == 0 ? 1 : 0)) * pitch;
#pragma unroll
            for (int i = 0; i < W; i += 4)
                asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(in[u][i]), "=f"(in[u][i + 1]), "=f"(in[u][i + 2]), "=f"(in[u][i + 3])
                             : "l"(from + i)
                             : "memory");
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < W; ++i) sum[i] += p + u * groups < p1 ? in[u][i] : 0.f;
    }
    __syncwarp();
    for (int d = P; d < 32; d *= 2)
#pragma unroll
        for (int i = 0; i < W; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], d);
}

template <typename TT, int W, bool LOOSE>
__global__ void __launch_bounds__(kNT, 2) k_token_joins(const int32_t* __restrict__ sorted, int64_t max_tokens, const int32_t* n_tokens,
                                                     int n_rows, int dim, float scale, TT* __restrict__ table, int64_t ld_table,
                                                     int accumulate, int window, int P, const float* __restrict__ pieces) {
    constexpr int kWarps = kNT / 32;
    __shared__ __align__(16) float s_sum[kNT * W];               // of each warp: [32 W]
    __shared__ int s_long[kWarps];                               // the run of a warp's window, if it is long
    wait_for_last();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = live_tokens(n_tokens, max_tokens), first = (int64_t)blockIdx.x * kWarps, pitch = piece_pitch(dim);
    const int c = ((int)blockIdx.y * P + lane % P) * W;          // (P lanes: 32, or as many as have all columns)
    const bool writes = lane < P;
    const int64_t w = first + warp, end = (w + 1) * window;
    int begins = -1;                                             // the run that begins in the window and goes on
    if (end < n) {
        // (lanes: before the window, its last token, the first behind it, and those of the windows behind that)
        const int64_t at = lane == 0 ? w * window - 1 : lane == 1 ? end - 1 : (w + lane - 1) * window;
        const int v = at >= 0 && at < n ? __ldg(&sorted[at]) : -1;
        const int run = __shfl_sync(0xffffffffu, v, 2);
        const unsigned same = __ballot_sync(0xffffffffu, v == run);
        const int more = __ffs(~(same >> 2)) - 1;                // windows behind that begin with it; at most 30
        if ((unsigned)run < (unsigned)n_rows && (same & 3) == 2) {
            begins = run;
            if (more < kShort) {
                float sum[W] = {};
                add_pieces<W>(pieces, pitch, w, 0, more + 1, c, dim, P, sum);
                if (writes && (LOOSE || c < dim))
                    put<TT, W, LOOSE>(table + run * ld_table, c, dim, sum, scale, accumulate, P == 32 ? s_sum + warp * 32 * W : nullptr);
                begins = -1;
            }
        }
    }
    if (lane == 0) s_long[warp] = begins;
    if (!__syncthreads_or(begins >= 0)) return;
    for (int k = 0; k < kWarps; ++k) {
        const int run = s_long[k];
        if (run < 0) continue;
        int all = 1;                                             // its pieces
        for (int64_t v = first + k + 1; v * window < n; v += kNT) {
            const int64_t at = (v + threadIdx.x) * window;
            const int more = __syncthreads_count(at < n && __ldg(&sorted[min(at, n - 1)]) == run);
            all += more;
            if (more < kNT) break;
        }
        const int per = (all + kWarps - 1) / kWarps, p0 = min(warp * per, all), p1 = min(p0 + per, all);
        float sum[W] = {};
        add_pieces<W>(pieces, pitch, first + k, p0, p1, c, dim, P, sum);
#pragma unroll
        for (int i = 0; i < W; ++i) s_sum[(warp * W + i) * 32 + lane] = sum[i];
        __syncthreads();
        if (warp == 0) {
            for (int s = 1; s < kWarps; ++s)
#pragma unroll
                for (int i = 0; i < W; ++i) sum[i] += s_sum[(s * W + i) * 32 + lane];
            if (writes && (LOOSE || c < dim))
                put<TT, W, LOOSE>(table + run * ld_table, c, dim, sum, scale, accumulate, P == 32 ? s_sum : nullptr);
        }
        __syncthreads();
    }
}

// ---- arguments ------------------------------------------------------------------------------------------------------------
constexpr int64_t kMostDim = 1 << 22;  // (of a gradient: columns are a grid's second dimension)
bool tokens_ok(int64_t max_tokens) { return max_tokens >= 0 && max_tokens < (int64_t(1) << 30); }
unsigned long long inverse_of(int64_t vectors) { return vectors == 1 ? 0 : ~0ull / vectors + 1; }

// Tokens of a window: up to 32 tokens are one, so that no run is cut.  Else a power of two from 16 to 128: so many that the windows' threads, of eight columns, fill the chip once, but not
// more than 8 192 windows where 128 tokens each make fewer of them.
constexpr int64_t kChipThreads = 148 * 2048;
int window_of(int64_t max_tokens, int64_t dim) {
    if (max_tokens <= 32) return 32;
    int w = 16;
    while (w < 128 && (max_tokens * div_up(dim, 8) > w * kChipThreads || max_tokens > w * int64_t(8192))) w *= 2;
    return w;
}

// The windows that at most so many tokens can make: fewer tokens may have shorter windows, but of those that fill the chip.
int64_t most_windows(int64_t max_tokens, int64_t dim) {
    const int64_t now = div_up(max_tokens, window_of(max_tokens, dim)), shortest = div_up(max_tokens, 16);
    int64_t filled = kChipThreads / div_up(dim, 8) + 1;
    filled = filled < 8192 ? filled : 8192;
    filled = filled < shortest ? filled : shortest;
    return now > filled ? now : filled;
}

// the workspace: two words, and then what either call needs
struct Workspace {
    int32_t *n, *status, *keys, *vals;
    uint32_t* hist;
    float* pieces;
};
constexpr int64_t kWorkspaceHead = 256;
int64_t padded(int64_t words) { return (words + 63) & ~int64_t(63); }
Workspace layout(void* p, int64_t max_tokens) {
    int32_t* base = static_cast<int32_t*>(p);
    int32_t* body = base + kWorkspaceHead / 4;
    return {base, base + 1, body, body + padded(max_tokens), reinterpret_cast<uint32_t*>(body + 2 * padded(max_tokens)),
            reinterpret_cast<float*>(body)};
}

template <typename TT, typename TO>
int32_t launch_embed(int64_t n_rows, int64_t dim, const void* table, int64_t ld_table, const int32_t* tokens, int64_t max_tokens,
                     const int32_t* n_tokens, float scale, void* out, int64_t ld_out, int32_t* status, bool whole, cudaStream_t stream) {
    constexpr int N = 8, U = 2;        // (the 16 bytes of a 16-bit type)
    const int64_t vectors = whole ? dim / N : (dim + 16 / (int)sizeof(TO) - 1 + N - 1) / N, items = max_tokens * vectors;
    const int64_t ctas = div_up(items, kNT * (whole ? U : 1));
    if (ctas > 0x7fffffff || items >= (int64_t(1) << 40)) return HL_EINVAL;
    const TT* t = static_cast<const TT*>(table);
    TO* o = static_cast<TO*>(out);
    if (whole)
        HL_CUDA_TRY(launch(k_token_embed<TT, TO, N, U>, (unsigned)ctas, kNT, stream, t, ld_table, (unsigned)n_rows, tokens, max_tokens,
                           n_tokens, scale, o, ld_out, (int)vectors, inverse_of(vectors), status));
    else
        HL_CUDA_TRY(launch(k_token_embed_loose<TT, TO>, (unsigned)ctas, kNT, stream, t, ld_table, (unsigned)n_rows, tokens, max_tokens,
                           n_tokens, scale, (int)dim, o, ld_out, (int)vectors, inverse_of(vectors), status));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

template <typename TG, typename TT, int W, int U, bool LOOSE>
int32_t launch_sums(int64_t n_rows, int64_t dim, const int32_t* sorted, const int32_t* order, int64_t max_tokens,
                    const int32_t* n_tokens, const void* grad, int64_t ld_grad, float scale, void* table, int64_t ld_table,
                    int accumulate, float* pieces, cudaStream_t stream) {
    int P = 1;
    while (P < (LOOSE ? 32 : kNT) && P * W < dim) P *= 2;
    const int window = window_of(max_tokens, dim);
    const int64_t windows = div_up(max_tokens, window), passes = div_up(dim, P * W), sums = div_up(windows, kNT / P) * passes;
    // rows without tokens: some 128 KB a CTA, as many for each of its warps
    int64_t per = (128 << 10) / (dim * (int64_t)sizeof(TT)) / (kNT / 32) * (kNT / 32);
    per = per < kNT / 32 ? kNT / 32 : per > kNT ? kNT : per;
    const int64_t zeros = accumulate ? 0 : div_up(n_rows, per);
    if (sums + zeros > 0x7fffffff || div_up(dim, 32 * W) > 65535 || windows > 0x7fffffff) return HL_EINVAL;
    if (sums + zeros == 0) return HL_OK;
    HL_CUDA_TRY(launch(k_token_sums<TG, TT, W, U, LOOSE>, (unsigned)(sums + zeros), kNT, stream, sorted, order, max_tokens, n_tokens,
                       (int)n_rows, (int)dim, static_cast<const TG*>(grad), ld_grad, scale, static_cast<TT*>(table), ld_table, accumulate,
                       window, P, (int)passes, (int)sums, (int)per, pieces));
    note_launches(1);
    if (windows > 1) {
        const int Q = P < 32 ? P : 32;
        HL_CUDA_TRY(launch_after(k_token_joins<TT, W, LOOSE>, dim3((unsigned)div_up(windows - 1, kNT / 32), (unsigned)div_up(dim, Q * W)),
                                 kNT, 0, stream, sorted, max_tokens, n_tokens, (int)n_rows, (int)dim, scale, static_cast<TT*>(table),
                                 ld_table, accumulate, window, Q, (const float*)pieces));
        note_launches(1);
    }
    HL_LAUNCH_CHECK();
    return HL_OK;
}

}  // namespace
}  // namespace hl

using namespace hl;

extern "C" int32_t hl_token_embed(int32_t table_dtype, int64_t n_rows, int64_t dim, const void* d_table, int64_t ld_table,
                                  const int32_t* d_tokens, int64_t max_tokens, const int32_t* d_n_tokens, float scale,
                                  int32_t out_dtype, void* d_out, int64_t ld_out, int32_t* d_status, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (n_rows < 0 || n_rows >= (int64_t(1) << 31) || !tokens_ok(max_tokens) || (!d_tokens && max_tokens > 0) ||
        !row_matrix_ok(table_dtype, n_rows, dim, d_table, ld_table) || !row_matrix_ok(out_dtype, max_tokens, dim, d_out, ld_out) ||
        !lies_at(d_tokens, 4) || !lies_at(d_n_tokens, 4) || !lies_at(d_status, 4))
        return HL_EINVAL;
    if (max_tokens == 0) return HL_OK;
    const bool whole = dim % 8 == 0 && rows_lie_at(table_dtype, d_table, ld_table, 16) && rows_lie_at(out_dtype, d_out, ld_out, 16);
#define HL_EMBED(TT, TO)                                                                                                       \
    launch_embed<TT, TO>(n_rows, dim, d_table, ld_table, d_tokens, max_tokens, d_n_tokens, scale, d_out, ld_out, d_status, whole, \
                         stream)
#define HL_EMBED_TO(TT) (out_dtype == HL_F32 ? HL_EMBED(TT, float) : out_dtype == HL_BF16 ? HL_EMBED(TT, __nv_bfloat16) : HL_EMBED(TT, __half))
    return table_dtype == HL_F32 ? HL_EMBED_TO(float) : table_dtype == HL_BF16 ? HL_EMBED_TO(__nv_bfloat16) : HL_EMBED_TO(__half);
#undef HL_EMBED_TO
#undef HL_EMBED
}

extern "C" size_t hl_token_workspace_bytes(int64_t max_tokens, int64_t dim) {
    if (!tokens_ok(max_tokens) || dim < 1 || dim > kMostDim) return 0;
    const int64_t sort = (2 * padded(max_tokens) + padded(sort_hist_words(max_tokens))) * 4;
    const int64_t sums = 2 * most_windows(max_tokens, dim) * (div_up(dim, kPieceStep) * kPieceStep) * 4;
    return (size_t)(kWorkspaceHead + ((sort > sums ? sort : sums) + 255) / 256 * 256);
}

extern "C" int32_t hl_token_sort(const int32_t* d_tokens, int64_t max_tokens, const int32_t* d_n_tokens, int64_t n_rows,
                                 int32_t* d_sorted, int32_t* d_order, int32_t* d_status, void* d_workspace, size_t ws_bytes,
                                 void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (n_rows < 0 || n_rows >= (int64_t(1) << 31) || !tokens_ok(max_tokens) ||
        (max_tokens > 0 && (!d_tokens || !d_sorted || !d_order)) || !lies_at(d_tokens, 4) || !lies_at(d_n_tokens, 4) ||
        !lies_at(d_sorted, 4) || !lies_at(d_order, 4) || !lies_at(d_status, 4) || !d_workspace || !lies_at(d_workspace, 256))
        return HL_EINVAL;
    if (ws_bytes < hl_token_workspace_bytes(max_tokens, 1)) return HL_ECAPACITY;
    if (max_tokens == 0) return HL_OK;
    const Workspace ws = layout(d_workspace, max_tokens);
    if (max_tokens <= kFewTokens) {
        HL_CUDA_TRY(launch(k_token_rank, (unsigned)div_up(max_tokens, kFewNT), kFewNT, stream, d_tokens, (int)max_tokens, d_n_tokens,
                           (int)n_rows, d_sorted, d_order, d_status));
        note_launches(1);
        HL_LAUNCH_CHECK();
        return HL_OK;
    }
    int bits = 1;
    while ((n_rows >> bits) != 0) ++bits;
    if (sorts_tokens(max_tokens))
        return sort_tokens(d_tokens, d_n_tokens, max_tokens, (int)n_rows, bits, d_sorted, d_order, d_status, stream);
    const int passes = (bits + 7) / 8, out = passes & 1;         // (which of the two buffers the sort ends in)
    int32_t *keys[2], *vals[2], *sorted, *order;
    keys[out] = d_sorted;
    vals[out] = d_order;
    keys[out ^ 1] = ws.keys;
    vals[out ^ 1] = ws.vals;
    int32_t* status = d_status ? d_status : ws.status;
    HL_CUDA_TRY(clear_words(ws.hist, sort_clear_words(max_tokens, bits, WaitCfg()), stream));
    HL_CUDA_TRY(launch(k_token_pairs, grid_for(max_tokens, kNT * 2, 1024), kNT, stream, d_tokens, max_tokens, d_n_tokens, (int)n_rows,
                       keys[0], vals[0], ws.n, passes, ws.hist, status));
    note_launches(1);
    return radix_sort_pairs(keys, vals, ws.n, max_tokens, bits, ws.hist, status, &sorted, &order, stream, WaitCfg(), true);
}

extern "C" int32_t hl_token_embed_bwd(int64_t n_rows, int64_t dim, const int32_t* d_sorted, const int32_t* d_order,
                                      int64_t max_tokens, const int32_t* d_n_tokens, int32_t grad_dtype, const void* d_grad_out,
                                      int64_t ld_grad, float scale, int32_t table_dtype, void* d_grad_table, int64_t ld_table,
                                      int32_t accumulate, void* d_workspace, size_t ws_bytes, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (n_rows < 0 || n_rows >= (int64_t(1) << 31) || dim > kMostDim || !tokens_ok(max_tokens) ||
        (max_tokens > 0 && (!d_sorted || !d_order)) ||
        !row_matrix_ok(grad_dtype, max_tokens, dim, d_grad_out, ld_grad) ||
        !row_matrix_ok(table_dtype, n_rows, dim, d_grad_table, ld_table) || !lies_at(d_sorted, 4) || !lies_at(d_order, 4) ||
        !lies_at(d_n_tokens, 4) || !d_workspace || !lies_at(d_workspace, 256))
        return HL_EINVAL;
    if (ws_bytes < hl_token_workspace_bytes(max_tokens, dim)) return HL_ECAPACITY;
    const int N = 16 / dtype_size(grad_dtype);
    const bool whole = dim % N == 0 && rows_lie_at(grad_dtype, d_grad_out, ld_grad, 16) &&
                       rows_lie_at(table_dtype, d_grad_table, ld_table, 8) &&
                       (N * dtype_size(table_dtype) == 8 || rows_lie_at(table_dtype, d_grad_table, ld_table, 16));
    float* pieces = layout(d_workspace, max_tokens).pieces;
#define HL_SUMS(TG, TT)                                                                                                           \
    (whole ? launch_sums<TG, TT, 16 / sizeof(TG), 8, false>(n_rows, dim, d_sorted, d_order, max_tokens, d_n_tokens, d_grad_out,  \
                                                            ld_grad, scale, d_grad_table, ld_table, accumulate, pieces, stream)  \
           : launch_sums<TG, TT, 8, 4, true>(n_rows, dim, d_sorted, d_order, max_tokens, d_n_tokens, d_grad_out, ld_grad, scale, \
                                             d_grad_table, ld_table, accumulate, pieces, stream))
#define HL_SUMS_TO(TG) \
    (table_dtype == HL_F32 ? HL_SUMS(TG, float) : table_dtype == HL_BF16 ? HL_SUMS(TG, __nv_bfloat16) : HL_SUMS(TG, __half))
    return grad_dtype == HL_F32 ? HL_SUMS_TO(float) : grad_dtype == HL_BF16 ? HL_SUMS_TO(__nv_bfloat16) : HL_SUMS_TO(__half);
#undef HL_SUMS_TO
#undef HL_SUMS
}
