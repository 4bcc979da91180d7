// Matrices in 4 bits: blocks of 32 values of a row share a power of two.  Quantisation, the way back, and the experts' product
// on the tensor cores, which multiply such blocks as they are.
#include "hl_rows.cuh"

namespace hl {
namespace {

// ---- how a matrix lies ------------------------------------------------------------------------------------------------
// In tiles of 128 rows by 256 columns, those of 128 rows side by side, filled up with zeros at both ends; a tile is the 17 408 bytes
// that a product's step takes as they are, in one copy: 16 KB of values, 128 bytes a row in the 16-byte pieces' order in which the
// tensor cores read shared memory without bank conflicts (piece p of row r lies at p ^ (r & 7)), and 1 KB of exponents, for each half
// of the columns 32 pieces of 16 bytes, of which piece r % 32 holds four of each of the rows r % 32, + 32, + 64 and + 96.
constexpr int kTileRows = 128, kTileCols = 256, kBlock = 32;
constexpr int kValueBytes = kTileRows * kTileCols / 2, kTileBytes = kValueBytes + kTileRows * kTileCols / kBlock;
static_assert(kTileBytes == 17408 && kTileBytes % 1024 == 0, "tiles side by side begin where the pieces' order does");

// a lane's eight values among the 256 of a row's part: lanes 4b .. 4b + 3 have block b
__device__ __forceinline__ int value_at(int row, int lane) { return row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + ((lane & 3) << 2); }
// a block's exponent, behind the values
__device__ __forceinline__ int exponent_at(int row, int block) {
    return (row >> 7) * 1024 + (block >> 2) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// The rows that experts get lie in tiles of 240: as many columns as the tensor memory has room for twice, next to the exponents.  The
// exponents of rows 128 to 239 lie behind those of the first 128.
constexpr int kPanelRows = 240, kPanelValueBytes = kPanelRows * kTileCols / 2, kPanelBytes = kPanelValueBytes + 2048;
static_assert(kPanelBytes == 32768 && kPanelValueBytes % 1024 == 0, "as above");

// A row's part from column c on, eight values a lane, as they are; zeros behind its end and where there is no row.  WHOLE: rows begin
// at multiples of 16 bytes and have a multiple of eight values.
template <typename T, bool WHOLE>
struct Part {
    std::conditional_t<WHOLE, Pack<T, 8>, Loose<T>> v;
    int there;                         // values of the eight that there are (!WHOLE)
    __device__ __forceinline__ void load(const T* row, int c, int dim) {
        v.zero();
        there = row ? dim - c : 0;
        if (there <= 0) return;
        if constexpr (WHOLE) v.load(row + c);
        else v.load(row, c, dim);
    }
    __device__ __forceinline__ Pack<T, 8> values() const {
        if constexpr (WHOLE) {
            return v;
        } else {
            Pack<T, 8> p = v.values();
            if (there < 8) {
#pragma unroll
                for (int i = 0; i < Pack<T, 8>::kWords; ++i) {
                    if constexpr (sizeof(T) == 4) p.w[i] = i < there ? p.w[i] : 0u;
                    else p.w[i] &= (2 * i < there ? 0xffffu : 0u) | (2 * i + 1 < there ? 0xffff0000u : 0u);
                }
            }
            return p;
        }
    }
};
// The largest absolute value of the lane's block, among its four lanes, as a 32-bit float's bits (infinities and NaN: 255 << 23 and
// more).  Bits without the sign are in the order of the values, NaN largest; those of 16-bit types two at a time.
template <typename T>
__device__ __forceinline__ uint32_t largest(const Pack<T, 8>& p) {
    constexpr uint32_t kAbs = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    uint32_t top = p.w[0] & kAbs;
#pragma unroll
    for (int i = 1; i < Pack<T, 8>::kWords; ++i) top = sizeof(T) == 4 ? max(top, p.w[i] & kAbs) : __vmaxu2(top, p.w[i] & kAbs);
    if constexpr (sizeof(T) == 2) top = max(top >> 16, top & 0xffffu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    if constexpr (sizeof(T) == 4) return top;
    else if constexpr (std::is_same_v<T, __nv_bfloat16>) return top << 16;
    else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)top)));
}

// Eight values of a row's part in 4 bits, and their block's exponent (in all of its lanes): 2^(E - 127) with E two below the
// largest value's own, so that this one lies in 4 .. 8, of which what is above 6 becomes 6; values are rounded to the nearest of 0, 1/2, 1,
// 3/2, 2, 3, 4, 6, ties to the one of even mantissa.  A block with an infinity or NaN is NaN (exponent 255).
template <typename T, bool WHOLE>
__device__ __forceinline__ uint32_t to_four_bits(const Part<T, WHOLE>& part, uint32_t* exponent) {
    const Pack<T, 8> p = part.values();
    const int e = (int)(largest(p) >> 23);
    const uint32_t E = e == 255 ? 255u : (uint32_t)max(e - 2, 0);
    const float up = __uint_as_float((254u - min(E, 253u)) << 23);         // 2^(127 - E)
    float x[8];
    p.get(x);
    uint32_t packed;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(packed)
        : "f"(x[0] * up), "f"(x[1] * up), "f"(x[2] * up), "f"(x[3] * up), "f"(x[4] * up), "f"(x[5] * up), "f"(x[6] * up),
          "f"(x[7] * up));
    *exponent = E;
    return packed;
}


constexpr int kRowNT = 256;

// n / d by 2^64 / d, rounded up: exact for n * d < 2^64
struct Divisor {
    uint64_t inverse;
    int64_t d;
    __device__ __forceinline__ int64_t operator()(int64_t n) const { return d == 1 ? n : (int64_t)__umul64hi((uint64_t)n, inverse); }
};

// n_matrices of `rows` rows: a warp takes U parts of a row, side by side.  Bound by memory: 134 M bf16 59 us, 339 MB: 5.7 TB/s.  (rows_of: a matrix' rows, here with
// those that fill its last tile up; chunks: of U parts, in a row)
template <typename T, bool WHOLE, int U>
__global__ void __launch_bounds__(kRowNT) k_mx4_quantise(const T* __restrict__ x, int64_t rows, int64_t dim, int64_t ld, int64_t stride,
                                                         uint64_t rows_inverse, int64_t rows_d, uint64_t chunks_inverse,
                                                         int64_t chunks_d, int col_tiles, int64_t items, uint8_t* __restrict__ q) {
    const Divisor rows_of{rows_inverse, rows_d}, chunks{chunks_inverse, chunks_d};
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * (kRowNT / 32) + (threadIdx.x >> 5);
    if (item >= items) return;
    const int64_t row = chunks(item), m = rows_of(row), of = row - m * rows_of.d;
    const int ct = (int)(item - row * chunks.d) * U, r = (int)(of & (kTileRows - 1));
    const T* from = of < rows ? x + m * stride + of * ld : nullptr;
    uint8_t* tile = q + ((row >> 7) * col_tiles + ct) * kTileBytes;
    Part<T, WHOLE> in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) in[u].load(from, (ct + u) * kTileCols + lane * 8, (int)dim);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (ct + u >= col_tiles) break;
        uint32_t e;
        const uint32_t packed = to_four_bits(in[u], &e);
        *reinterpret_cast<uint32_t*>(tile + u * kTileBytes + value_at(r, lane)) = packed;
        if ((lane & 3) == 0) tile[u * kTileBytes + kValueBytes + exponent_at(r, lane >> 2)] = (uint8_t)e;
    }
}

// N values in 4 bits each, the first in the lowest
template <int N>
__device__ __forceinline__ void from_four_bits(uint32_t packed, uint32_t E, float* x) {
    const float unit = E == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(E ? E << 23 : 0x00400000u);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        uint32_t two;                  // fp16
        asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(two) : "r"(packed >> (8 * i)));
        x[2 * i] = __half2float(__ushort_as_half((unsigned short)(two & 0xffffu))) * unit;
        x[2 * i + 1] = __half2float(__ushort_as_half((unsigned short)(two >> 16))) * unit;
    }
}

// The way back: a lane writes 16 bytes of a row's part at a time, so that a warp's stores are whole lines (with 32 bytes of fp32 in a
// row of a lane's own, two halves of a line each: 127 us instead of 92 for 134 M values).  Rows that begin anywhere are written value by
// value: 40 000 of 2 500 values 102 us in fp32 and 275 in 16 bits, where such of 2 496 that begin at 16 bytes take 74 and 45.
template <typename T, bool WHOLE, int U>
__global__ void __launch_bounds__(kRowNT) k_mx4_dequantise(const uint8_t* __restrict__ q, int64_t row_tiles, int64_t dim,
                                                           uint64_t rows_inverse, int64_t rows_d, uint64_t chunks_inverse,
                                                           int64_t chunks_d, int col_tiles, int64_t items, T* __restrict__ out,
                                                           int64_t ld, int64_t stride) {
    const Divisor rows_of{rows_inverse, rows_d}, chunks{chunks_inverse, chunks_d};
    constexpr int N = 16 / sizeof(T), S = 8 / N;                 // values of a store, stores of a part
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * (kRowNT / 32) + (threadIdx.x >> 5);
    if (item >= items) return;
    const int64_t row = chunks(item), m = rows_of(row), of = row - m * rows_of.d;
    const int ct = (int)(item - row * chunks.d) * U, r = (int)(of & (kTileRows - 1));
    const uint8_t* tile = q + ((m * row_tiles + (of >> 7)) * col_tiles + ct) * kTileBytes;
    T* to = out + m * stride + of * ld;
    uint32_t packed[U][S], E[U][S];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int c = i * 32 * N + lane * N;                 // of the part
            const uint8_t* p = tile + u * kTileBytes + r * 128 + (((c >> 5) ^ (r & 7)) << 4) + ((c & 31) >> 1);
            packed[u][i] = E[u][i] = 0;
            if (ct + u >= col_tiles) continue;
            packed[u][i] = N == 8 ? __ldg(reinterpret_cast<const uint32_t*>(p)) : __ldg(reinterpret_cast<const unsigned short*>(p));
            E[u][i] = __ldg(tile + u * kTileBytes + kValueBytes + exponent_at(r, c >> 5));
        }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int64_t c = (int64_t)(ct + u) * kTileCols + i * 32 * N + lane * N;
            if (ct + u >= col_tiles || c >= dim) continue;
            float x[N];
            from_four_bits<N>(packed[u][i], E[u][i], x);
            if constexpr (WHOLE) {
                Pack<T, N> v;
                v.set(x);
                v.store(to + c);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (c + k < dim) to[c + k] = from_float<T>(x[k]);
            }
        }
}

// ---- the experts' rows ------------------------------------------------------------------------------------------------
// Expert e's rows are cut into tiles of 240 of their own, wherever they begin in the expert-ordered buffers: first[e] is its first
// tile's number, first[E] how many there are (never more than the workspace holds).
struct Experts {
    const int32_t *counts, *offsets;
    int E;
    int64_t cap_rows;
    __device__ __forceinline__ int begin(int e) const { return (int)min((int64_t)max(__ldg(&offsets[e]), 0), cap_rows); }
    __device__ __forceinline__ int rows(int e, int from) const { return (int)min((int64_t)max(__ldg(&counts[e]), 0), cap_rows - from); }
};

// Fills s_first [E + 1] (and s_begin [E], if there): by all NT threads of a CTA.
template <int NT>
__device__ void tile_numbers(const Experts& x, int most, int* s_first, int* s_begin) {
    constexpr int kPer = (HL_MAX_EXPERTS + NT - 1) / NT;
    __shared__ int s_warp[NT / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int tiles[kPer], sum = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int e = threadIdx.x * kPer + k;
        tiles[k] = 0;
        if (e >= x.E) continue;
        const int from = x.begin(e);
        if (s_begin) s_begin[e] = from;
        tiles[k] = (x.rows(e, from) + kPanelRows - 1) / kPanelRows;
        sum += tiles[k];
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += v;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int at = incl - sum;
    for (int w = 0; w < warp; ++w) at += s_warp[w];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int e = threadIdx.x * kPer + k;
        if (e >= x.E) break;
        s_first[e] = min(at, most);
        at += tiles[k];
        if (e == x.E - 1) s_first[x.E] = min(at, most);
    }
    __syncthreads();
}
// the last e of [0, n) with list[e] <= v (list[0] <= v)
__device__ __forceinline__ int last_not_above(const int* list, int n, int v) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (list[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Rows in the experts' order (top_k 0), or the tokens', each to all of its experts' rows: read and converted once.  A warp takes `span`
// times U parts of a row; its lanes find where each of the row's choices lies.  16 384 rows of 4 096 bf16 to two experts each: 42 us, 206 MB;
// 60 % of the cycles issue an instruction.
template <int U>
constexpr int kRowCtas = U == 8 ? 3 : U == 4 ? 4 : 6;            // CTAs of a multiprocessor
template <typename T, bool WHOLE, int U>
__global__ void __launch_bounds__(kRowNT, kRowCtas<U>) k_mx4_rows(const T* __restrict__ x, int64_t ld, int dim, int col_tiles, int span,
                                                        uint64_t items_inverse, int64_t items_d, const int32_t* n_tokens, int64_t max_rows, int top_k,
                                                        const int32_t* __restrict__ place, const int32_t* __restrict__ counts,
                                                        const int32_t* __restrict__ offsets, int E, int64_t cap_rows, int max_tiles,
                                                        uint8_t* __restrict__ q, int32_t* status) {
    __shared__ int s_first[HL_MAX_EXPERTS + 1], s_begin[HL_MAX_EXPERTS];
    const Divisor items_of{items_inverse, items_d};
    let_next_start();
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = HL_OK;
    const Experts experts{counts, offsets, E, cap_rows};
    tile_numbers<kRowNT>(experts, max_tiles, s_first, s_begin);
    const int lane = threadIdx.x & 31;
    int64_t n = max_rows;
    if (top_k == 0) n = min(n, (int64_t)max(__ldg(&offsets[E]), 0));
    else if (n_tokens) n = min(n, (int64_t)max(__ldg(n_tokens), 0));
    const int64_t items = n * items_of.d;
    for (int64_t i = (int64_t)blockIdx.x * (kRowNT / 32) + (threadIdx.x >> 5); i < items; i += (int64_t)gridDim.x * (kRowNT / 32)) {
        const int64_t row = items_of(i);
        const int begin = (int)(i - row * items_of.d) * span * U, end = min(begin + span * U, col_tiles);
        const T* from = x + row * ld;
        for (int k0 = 0; k0 < max(top_k, 1); k0 += 32) {
            int64_t to = -1;           // of choice k0 + lane: its tile's number times 256, and its row in it
            int at = -1;
            if (top_k == 0) at = lane == 0 ? (int)row : -1;
            else if (k0 + lane < top_k) at = __ldg(&place[row * top_k + k0 + lane]);
            if (at >= 0 && at < cap_rows) {
                // (experts without rows begin where the next does: the last that begins there is the one)
                const int e = last_not_above(s_begin, E, at), r = at - s_begin[e], tile = s_first[e] + r / kPanelRows;
                if (r >= 0 && r < experts.rows(e, s_begin[e]) && tile < s_first[e + 1])
                    to = (int64_t)tile << 8 | (r - r / kPanelRows * kPanelRows);
            }
            const unsigned there = __ballot_sync(0xffffffffu, to >= 0);
            if (!there) continue;
            for (int ct = begin; ct < end; ct += U) {
                Part<T, WHOLE> in[U];
                uint32_t packed[U], exponent[U];
#pragma unroll
                for (int u = 0; u < U; ++u) in[u].load(from, (ct + u) * kTileCols + lane * 8, dim);
#pragma unroll
                for (int u = 0; u < U; ++u) packed[u] = to_four_bits(in[u], &exponent[u]);
                for (unsigned left = there; left; left &= left - 1) {
                    const int64_t dst = __shfl_sync(0xffffffffu, to, __ffs(left) - 1);
                    const int r = (int)(dst & 255);
                    uint8_t* tile = q + ((dst >> 8) * col_tiles + ct) * kPanelBytes;
                    uint8_t *values = tile + value_at(r, lane), *exponents = tile + kPanelValueBytes + exponent_at(r, lane >> 2);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (ct + u >= end) break;
                        *reinterpret_cast<uint32_t*>(values + u * kPanelBytes) = packed[u];
                        if ((lane & 3) == 0) exponents[u * kPanelBytes] = (uint8_t)exponent[u];
                    }
                }
            }
        }
    }
}

// ---- the product --------------------------------------------------------------------------------------------------------
// Few rows, 16 in all at most (a token or two that are being served): the product's CTAs put them into 4 bits themselves, each those of
// its tile, straight into shared memory -- one kernel instead of two, one behind the other.
constexpr int kFewRows = 16;
// The row of x that expert-ordered row `at` gets (-1: none), asked by a whole warp; place: of x's rows by token, NULL: they are in the
// experts' order.
__device__ __forceinline__ int64_t row_of(int64_t at, const int32_t* __restrict__ place, const int32_t* n_tokens, int64_t max_tokens, int top_k) {
    if (!place) return at;
    const int lane = threadIdx.x & 31;
    int64_t tokens = max_tokens;
    if (n_tokens) tokens = min(tokens, (int64_t)max(__ldg(n_tokens), 0));
    const int choices = (int)tokens * top_k;                     // (kFewRows at most)
    const unsigned here = __ballot_sync(0xffffffffu, lane < choices && __ldg(&place[min(lane, max(choices - 1, 0))]) == at);
    return here ? (__ffs(here) - 1) / top_k : -1;
}

// y[row, f] = sum over d of x[row, d] * w[e, f, d] for the rows of expert e: 128 outputs f (the lanes of the tensor memory) by up to
// 240 rows (its columns) at a time, 256 of d a step.  One warp's thread has the tiles of a step copied, one issues the products,
// eight warps take the sums out, those of one tile while the next one's are made.
// Bound by what the multiprocessors can read of the L2, for many rows: 32 768 rows by 4 096 outputs of 4 096: 211 to 225 us, 5 PFLOP/s, 3.7 GB
// of tiles at 17 TB/s.  (With the copies left out it was 215 us at tiles of 128 rows, with the products left out 290; w' and x' tiles
// go to each multiprocessor anew, and wider ones would need two of them for a tile.)  Few rows: latency of a copy and a launch.
constexpr int kProductNT = 320;
constexpr uint32_t kExponentCols = 2 * kPanelRows;               // tensor-memory columns: two tiles' sums, 8 of w's exponents, 16 of x'
// A stage is a step's tile of w and as many of x' rows as an expert can have: few rows leave room for more steps on their way.
constexpr int kMostStages = 10, kStagesBytes = 4 * (kTileBytes + kPanelBytes);
constexpr int kProductSmem = kStagesBytes + 1024 + (HL_MAX_EXPERTS + 1) * 4 + 256;

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, int n) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_done(uint64_t* b, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_u32(b)), "r"(parity)
        : "memory");
    return done;
}
// Waits for a phase, not for ever: false if it did not come, or somebody else has given up.
constexpr int kMaxPolls = 1 << 22;
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile int* gave_up) {
    for (int i = 0; i < kMaxPolls; ++i) {
        if (bar_done(b, parity)) return true;
        if (*gave_up) return false;
    }
    *gave_up = 1;
    return false;
}
// The same by a whole warp, which goes on together, or gives up together.
__device__ __forceinline__ bool bar_wait_all(uint64_t* b, uint32_t parity, volatile int* gave_up) {
    return __all_sync(0xffffffffu, bar_wait(b, parity, gave_up));
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// Where an operand lies in shared memory, as the tensor cores want it said: the address in 16 bytes (the lower half, which alone
// changes from one to the next), bytes from one group of eight rows to the next, and whether pieces of 16 bytes are in the order of
// the tiles' values (or of their exponents: as they come).
constexpr uint32_t kOrderedHigh = (1024u >> 4) | 1u << 14 | 2u << 29, kPlainHigh = (128u >> 4) | 1u << 14;
__device__ __forceinline__ uint32_t operand_low(uint32_t address) { return (address & 0x3ffffu) >> 4 | 1u << 16; }
__device__ __forceinline__ uint64_t operand(uint32_t low, uint32_t high) { return (uint64_t)high << 32 | low; }

// These are for one thread: `one` says who.  (The warp's threads go through the loop together, so that what is the same in all of them
// stays in the registers that the tensor cores' instructions take; with the loop in one thread alone each of them took some 200
// cycles to put together.)
__device__ __forceinline__ void exponents_to_tmem(bool one, uint32_t tmem, uint32_t low) {
    asm volatile("{\n\t.reg .pred o;\n\tsetp.ne.b32 o, %2, 0;\n\t@o tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(tmem),
                 "l"(operand(low, kPlainHigh)), "r"((uint32_t)one)
                 : "memory");
}
// 64 of d: both operands of e2m1 (code 1 in bits 7 and 10), exponents alone as factors (bit 23), 128 by n, the pair of each row's
// four exponents that counts
__device__ __forceinline__ uint32_t multiplication(uint32_t n, int pair) {
    return (uint32_t)(2 * pair) << 4 | 1u << 7 | 1u << 10 | (n >> 3) << 17 | 1u << 23 | (128u >> 4) << 24 | (uint32_t)(2 * pair) << 29;
}
__device__ __forceinline__ void multiply(bool one, uint32_t acc, uint32_t a, uint32_t b, uint32_t what, uint32_t ea, uint32_t eb, bool add) {
    asm volatile(
        "{\n\t.reg .pred p, o;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 o, %7, 0;\n\t"
        "@o tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(acc),
        "l"(operand(a, kOrderedHigh)), "l"(operand(b, kOrderedHigh)), "r"(what), "r"(ea), "r"(eb), "r"((uint32_t)add), "r"((uint32_t)one)
        : "memory");
}
__device__ __forceinline__ void commit(bool one, uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .pred o;\n\tsetp.ne.b32 o, %1, 0;\n\t"
        "@o tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)), "r"((uint32_t)one)
        : "memory");
}
__device__ __forceinline__ bool elected() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one;
}

// 32 columns of a warp's 32 lanes
__device__ __forceinline__ void tmem_load(uint32_t (&v)[32], uint32_t from) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
          "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
          "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(from)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// What a CTA does next: the tile of rows, the expert's, and the tile of outputs.
struct Item {
    int e, rows, f;                    // rows: of the tile
    int64_t row0, tile, pad;           // its first row's number; pad: rows behind the expert's last that fill it up, if it is the last tile
};
__device__ __forceinline__ Item item_of(int64_t i, int f_tiles, const Experts& x, const int* s_first, int panel_rows) {
    Item it;
    it.tile = i / f_tiles;
    it.f = (int)(i - it.tile * f_tiles);
    it.e = last_not_above(s_first, x.E, (int)it.tile);
    const int begin = x.begin(it.e), rows = x.rows(it.e, begin), at = ((int)it.tile - s_first[it.e]) * kPanelRows;
    it.rows = min(rows - at, panel_rows);
    it.row0 = (int64_t)begin + at;
    const int64_t end = min((int64_t)max(__ldg(&x.offsets[it.e + 1]), 0), x.cap_rows);
    it.pad = it.tile + 1 == s_first[it.e + 1] ? max(end - begin - rows, (int64_t)0) : 0;
    return it;
}

template <typename T, bool DIRECT, bool WHOLE>
__global__ void __launch_bounds__(kProductNT, 1) k_mx4_product(const T* __restrict__ few_x, int64_t few_ld, const int32_t* n_tokens,
                                                               const int32_t* __restrict__ few_place, int64_t max_tokens, int top_k,
                                                               int dim, const uint8_t* __restrict__ xq, const uint8_t* __restrict__ wq,
                                                               const int32_t* __restrict__ counts, const int32_t* __restrict__ offsets,
                                                               int E, int64_t cap_rows, int max_tiles, int col_tiles, int f_tiles,
                                                               int64_t outputs, T* __restrict__ y, int64_t ld, bool lines, int stages,
                                                               int panel_rows, int32_t* status, int32_t* first_error) {
    extern __shared__ uint8_t s_raw[];
    uint8_t* base = s_raw + ((1024 - (smem_u32(s_raw) & 1023)) & 1023);
    int* s_first = reinterpret_cast<int*>(base + kStagesBytes);
    const int panel_bytes = panel_rows * 128, stage_bytes = kTileBytes + panel_bytes + (panel_rows > kTileRows ? 2048 : 1024);
    __shared__ uint64_t s_full[kMostStages], s_empty[kMostStages], s_sums[2], s_taken[2];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_gave_up;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            bar_init(&s_full[s], DIRECT ? 1 + 8 : 1);            // (and the warps that put x' rows into 4 bits)
            bar_init(&s_empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(&s_sums[b], 1);
            bar_init(&s_taken[b], 8);
        }
        s_gave_up = 0;
        if (DIRECT && blockIdx.x == 0) *status = HL_OK;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    const Experts experts{counts, offsets, E, cap_rows};
    tile_numbers<kProductNT>(experts, max_tiles, s_first, nullptr);        // (ends with a barrier)
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    const int64_t items = (int64_t)s_first[E] * f_tiles;

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 1;
            bool ok = true;
            // the weights of the first steps, while the rows are still being put into 4 bits
            const auto ask = [&](const uint8_t* a, uint32_t b_bytes, uint32_t e_bytes) {
                bar_expect(&s_full[stage], kTileBytes + b_bytes + e_bytes);
                bulk_load(smem_u32(base + stage * stage_bytes), a, kTileBytes, &s_full[stage]);
            };
            const auto next = [&]() {
                if (++stage == stages) {
                    stage = 0;
                    phase ^= 1;
                }
            };
            int early = 0;
            if (blockIdx.x < items) {
                const Item it = item_of(blockIdx.x, f_tiles, experts, s_first, panel_rows);
                const uint8_t* a = wq + ((int64_t)it.e * f_tiles + it.f) * col_tiles * kTileBytes;
                for (; early < min(stages, col_tiles); ++early, a += kTileBytes) {
                    ask(a, DIRECT ? 0 : ((it.rows + 15) & ~15) * 128, DIRECT ? 0 : it.rows > kTileRows ? 2048 : 1024);
                    next();
                }
            }
            wait_for_last();
            stage = 0;
            phase = 1;
            for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
                const Item it = item_of(i, f_tiles, experts, s_first, panel_rows);
                const uint8_t* a = wq + ((int64_t)it.e * f_tiles + it.f) * col_tiles * kTileBytes;
                const uint8_t* b = xq + it.tile * col_tiles * kPanelBytes;
                const uint32_t b_bytes = DIRECT ? 0 : ((it.rows + 15) & ~15) * 128, e_bytes = DIRECT ? 0 : it.rows > kTileRows ? 2048 : 1024;
                for (int c = 0; c < col_tiles; ++c, a += kTileBytes, b += kPanelBytes) {
                    if (early > 0) {
                        --early;
                    } else {
                        if (!(ok = bar_wait(&s_empty[stage], phase, &s_gave_up))) break;
                        ask(a, b_bytes, e_bytes);
                    }
                    if (!DIRECT) {
                        const uint32_t at = smem_u32(base + stage * stage_bytes) + kTileBytes;
                        bulk_load(at, b, b_bytes, &s_full[stage]);
                        bulk_load(at + panel_bytes, b + kPanelValueBytes, e_bytes, &s_full[stage]);
                    }
                    next();
                }
            }
            for (int s = 0; ok && s < stages; ++s) {             // (nothing may arrive here after this CTA's end)
                ok = bar_wait(&s_empty[stage], phase, &s_gave_up);
                next();
            }
        }
    } else if (warp == 1) {
        const bool one = elected();
        const uint32_t base_low = operand_low(__shfl_sync(0xffffffffu, smem_u32(base), 0)), d = __shfl_sync(0xffffffffu, tmem, 0);
        int stage = 0, buffer = 0;
        uint32_t phase = 0, taken = 1;
        bool ok = true;
        for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
            const uint32_t n = __shfl_sync(0xffffffffu, (item_of(i, f_tiles, experts, s_first, panel_rows).rows + 15) & ~15, 0);
            const uint32_t acc = d + buffer * kPanelRows, what0 = multiplication(n, 0), what1 = multiplication(n, 1);
            if (!(ok = bar_wait_all(&s_taken[buffer], taken, &s_gave_up))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (int c = 0; c < col_tiles; ++c) {
                if (!(ok = bar_wait_all(&s_full[stage], phase, &s_gave_up))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t a = base_low + stage * (stage_bytes >> 4), b = a + (kTileBytes >> 4), eb_at = b + (panel_bytes >> 4);
                // (copies and products run in the order in which they are issued)
                const uint32_t ea = d + kExponentCols, eb = ea + 8;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    exponents_to_tmem(one, ea + 4 * h, a + ((kValueBytes + 512 * h) >> 4));
                    exponents_to_tmem(one, eb + 8 * h, eb_at + ((512 * h) >> 4));
                    if (n > kTileRows) exponents_to_tmem(one, eb + 8 * h + 4, eb_at + ((1024 + 512 * h) >> 4));
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    multiply(one, acc, a + 2 * k, b + 2 * k, k & 1 ? what1 : what0, ea + 4 * (k >> 1), eb + 8 * (k >> 1), c > 0 || k > 0);
                commit(one, &s_empty[stage]);
                if (++stage == stages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
            commit(one, &s_sums[buffer]);
            buffer ^= 1;
            taken ^= buffer == 0;
        }
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;    // the lanes of the tensor memory that this warp can read; its columns
        int buffer = 0, stage = 0;
        uint32_t phase = 0, empty = 1;
        for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
            const Item it = item_of(i, f_tiles, experts, s_first, panel_rows);
            if constexpr (DIRECT) {
                // x' rows step by step, each row's part by one of the warps in turn.  (As a rule an expert has one row or two here; several
                // parts of a warp on their way at a time: 10.8 us instead of 8.8 a call of one token, 20 instead of 23 for twelve rows
                // of one expert.)
                bool ok = true;
                for (int c = 0, part = 0; ok && c < col_tiles; ++c) {
                    ok = bar_wait_all(&s_empty[stage], empty, &s_gave_up);
                    for (int r = 0; ok && r < it.rows; ++r, ++part) {
                        if ((part & 7) != warp - 2) continue;
                        const int64_t from = row_of(it.row0 + r, few_place, n_tokens, max_tokens, top_k);
                        Part<T, WHOLE> in;
                        in.load(from < 0 ? nullptr : few_x + from * few_ld, c * kTileCols + lane * 8, dim);
                        uint32_t e;
                        const uint32_t packed = to_four_bits(in, &e);
                        uint8_t* panel = base + stage * stage_bytes + kTileBytes;
                        *reinterpret_cast<uint32_t*>(panel + value_at(r, lane)) = packed;
                        if ((lane & 3) == 0) panel[panel_bytes + exponent_at(r, lane >> 2)] = (uint8_t)e;
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    __syncwarp();
                    if (ok && lane == 0) bar_arrive(&s_full[stage]);
                    if (++stage == stages) {
                        stage = 0;
                        empty ^= 1;
                    }
                }
                if (!ok) break;
            }
            if (!bar_wait_all(&s_sums[buffer], phase, &s_gave_up)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int64_t f = (int64_t)it.f * kTileRows + quarter * 32 + lane;
            const int middle = min((it.rows + 31) / 32 * 16, it.rows), end = half ? it.rows : middle;
            for (int c0 = half ? middle : 0; c0 < end; c0 += 32) {
                uint32_t v[32];
                __syncwarp();          // (the whole warp reads tensor memory together; lanes behind the last output skipped the stores)
                tmem_load(v, tmem + buffer * kPanelRows + c0 + ((uint32_t)(quarter * 32) << 16));
                if (f < outputs) {
                    T* out = y + (it.row0 + c0) * ld + f;
                    if (c0 + 32 <= end) {
#pragma unroll
                        for (int k = 0; k < 32; ++k, out += ld) *out = from_float<T>(__uint_as_float(v[k]));
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; ++k, out += ld)
                            if (c0 + k < end) *out = from_float<T>(__uint_as_float(v[k]));
                    }
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(&s_taken[buffer]);
            if (it.pad) {
                const int64_t f0 = (int64_t)it.f * kTileRows;
                const int width = (int)min((int64_t)kTileRows, outputs - f0), tid = threadIdx.x - 64;
                T* pads = y + (it.row0 + it.rows) * ld + f0;
                constexpr int N = 16 / sizeof(T);
                if (lines) {           // (all rows of y, and their tiles of outputs, begin at multiples of 16 bytes, and are whole ones)
                    const int per = width / N;
                    for (int64_t p = tid / (kTileRows / N); p < it.pad; p += 256 / (kTileRows / N))
                        if (tid % (kTileRows / N) < per) reinterpret_cast<uint4*>(pads + p * ld)[tid % (kTileRows / N)] = make_uint4(0, 0, 0, 0);
                } else {
                    for (int64_t p = tid / kTileRows; p < it.pad; p += 256 / kTileRows)
                        if (tid % kTileRows < width) pads[p * ld + tid % kTileRows] = from_float<T>(0.f);
                }
            }
            buffer ^= 1;
            phase ^= buffer == 0;
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (s_gave_up) {
        // (copies and products that are still on their way get some time to end)
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
        if (threadIdx.x == 0) {
            *status = HL_ETIMEOUT;
            if (first_error) set_status(first_error, HL_ETIMEOUT);
        }
        __syncthreads();
    }
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// ---- arguments ------------------------------------------------------------------------------------------------------------
constexpr int kSMs = 148;              // grids are made for a B200's multiprocessors
int64_t tiles_of(int64_t n, int per) { return div_up(n, per); }
bool matrix_dims_ok(int64_t rows, int64_t dim) { return rows >= 0 && rows < (int64_t(1) << 31) && dim >= 1 && dim <= (int64_t(1) << 24); }

uint64_t inverse_of(int64_t d) { return d == 1 ? 0 : ~uint64_t(0) / (uint64_t)d + 1; }

constexpr int64_t kWorkspaceHead = 1024;
int64_t row_tiles_most(int64_t cap_rows, int64_t E) { return cap_rows / kPanelRows + (E < cap_rows ? E : cap_rows); }

// Parts of a row that a warp takes: as many as there are, up to four.
int parts_of(int64_t col_tiles) { return col_tiles >= 3 ? 4 : (int)col_tiles; }
#define HL_PARTS(KERNEL, T)                                                                                             \
    (U == 4 ? (whole ? KERNEL<T, true, 4> : KERNEL<T, false, 4>)                                                        \
            : U == 2 ? (whole ? KERNEL<T, true, 2> : KERNEL<T, false, 2>) : (whole ? KERNEL<T, true, 1> : KERNEL<T, false, 1>))

template <typename T>
int32_t launch_quantise(int64_t n, int64_t rows, int64_t dim, const void* x, int64_t ld, int64_t stride, void* q, bool whole,
                        cudaStream_t stream) {
    const int64_t rt = tiles_of(rows, kTileRows), ct = tiles_of(dim, kTileCols);
    const int U = parts_of(ct);
    const int64_t chunks = div_up(ct, U), items = n * rt * kTileRows * chunks, ctas = div_up(items, kRowNT / 32);
    if (ctas > 0x7fffffff || n * rt * kTileRows >= (int64_t(1) << 32)) return HL_EINVAL;
    HL_CUDA_TRY(launch(HL_PARTS(k_mx4_quantise, T), (unsigned)ctas, kRowNT, stream, static_cast<const T*>(x), rows, dim, ld, stride,
                       inverse_of(rt * kTileRows), rt * kTileRows, inverse_of(chunks), chunks, ct, items, static_cast<uint8_t*>(q)));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}
template <typename T>
int32_t launch_dequantise(int64_t n, int64_t rows, int64_t dim, const void* q, void* out, int64_t ld, int64_t stride, bool whole,
                          cudaStream_t stream) {
    const int64_t rt = tiles_of(rows, kTileRows), ct = tiles_of(dim, kTileCols);
    const int U = parts_of(ct);
    const int64_t chunks = div_up(ct, U), items = n * rows * chunks, ctas = div_up(items, kRowNT / 32);
    if (ctas > 0x7fffffff || n * rows >= (int64_t(1) << 32)) return HL_EINVAL;
    HL_CUDA_TRY(launch(HL_PARTS(k_mx4_dequantise, T), (unsigned)ctas, kRowNT, stream, static_cast<const uint8_t*>(q), rt, dim,
                       inverse_of(rows), rows, inverse_of(chunks), chunks, ct, items, static_cast<T*>(out), ld, stride));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}
template <typename T>
int32_t launch_product(const hl_route* r, int64_t dim, int64_t outputs, const void* x, int64_t ld_x, bool by_token, const void* w,
                       void* y, int64_t ld_y, void* workspace, bool whole, int32_t* first_error, cudaStream_t stream) {
    int32_t* status = static_cast<int32_t*>(workspace);
    uint8_t* q = static_cast<uint8_t*>(workspace) + kWorkspaceHead;
    const int64_t ct = tiles_of(dim, kTileCols), ft = tiles_of(outputs, kTileRows), rt = row_tiles_most(r->cap_rows, r->n_experts);
    // (an expert can have all rows that there are)
    const int64_t choices = r->max_tokens * r->top_k, most_rows = by_token && choices < r->cap_rows ? choices : r->cap_rows;
    const bool direct = most_rows <= kFewRows && (!by_token || choices <= kFewRows);
    if (!direct) {
        // Parts of a row that a warp has on their way at a time: as many as there are, up to four, or eight of 16-bit types where there are
        // enough rows for the chip's warps all the same; twice that one after the other where that leaves them eight rounds.  Eight / four, a whole call
        // of 32 outputs: 16 384 rows of 4 096 bf16 to two experts each 57 / 69 us, that begin anywhere 77 / 83, by expert 82 / 101 and 118 / 132; fp32,
        // whose eight do not fit the registers, 76 / 74, 129 / 107, 118 / 110 and 213 / 174.
        constexpr int kMost = sizeof(T) == 2 ? 8 : 4;
        const int64_t rows = by_token ? r->max_tokens : r->cap_rows;
        const int U = ct <= 2 ? (int)ct : kMost == 8 && ct >= 7 && rows * div_up(ct, 8) >= 8 * kRowCtas<8> * kSMs ? 8 : 4;
        const int ctas = U == 8 ? kRowCtas<8> : U == 4 ? kRowCtas<4> : kRowCtas<1>;
        const int64_t chunks = div_up(ct, U), span = U == 8 && rows * chunks >= 8 * 8 * ctas * kSMs ? 2 : 1, per_row = div_up(chunks, span);
#define HL_ROWS(U) (whole ? k_mx4_rows<T, true, U> : k_mx4_rows<T, false, U>)
        const auto convert = U == kMost ? HL_ROWS(kMost) : U == 4 ? HL_ROWS(4) : U == 2 ? HL_ROWS(2) : HL_ROWS(1);
#undef HL_ROWS
        HL_CUDA_TRY(launch(convert, grid_for(rows * per_row, kRowNT / 32, ctas * kSMs), kRowNT, stream,
                           static_cast<const T*>(x), ld_x, dim, ct, span, inverse_of(per_row), per_row, r->n_tokens, rows,
                           by_token ? r->top_k : 0, r->place, r->counts, r->offsets, r->n_experts, r->cap_rows, rt, q, status));
        note_launches(1);
    }
    const int64_t panel = most_rows < kPanelRows ? div_up(most_rows, 16) * 16 : kPanelRows;      // (at least 16: most_rows > 0)
    const int64_t stage = kTileBytes + panel * 128 + (panel > kTileRows ? 2048 : 1024);
    const int64_t stages = kStagesBytes / stage < kMostStages ? kStagesBytes / stage : kMostStages;
    const auto kernel = !direct ? k_mx4_product<T, false, true> : whole ? k_mx4_product<T, true, true> : k_mx4_product<T, true, false>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem) != cudaSuccess) return HL_ECUDA;
    HL_CUDA_TRY(launch_cluster(kernel, grid_for(rt * ft, 1, kSMs), kProductNT, kProductSmem, direct ? 0 : kAfterLast, stream,
                               static_cast<const T*>(direct ? x : nullptr), ld_x, r->n_tokens, by_token ? r->place : nullptr,
                               r->max_tokens, r->top_k, dim, (const uint8_t*)q, static_cast<const uint8_t*>(w), r->counts, r->offsets, r->n_experts, r->cap_rows, rt, ct,
                               ft, outputs, static_cast<T*>(y), ld_y,
                               outputs * sizeof(T) % 16 == 0 && ld_y * sizeof(T) % 16 == 0 && lies_at(y, 16), stages, panel, status, first_error));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

}  // namespace
}  // namespace hl

using namespace hl;

#define HL_FOR_TYPE(CALL) (dtype == HL_F32 ? CALL(float) : dtype == HL_BF16 ? CALL(__nv_bfloat16) : CALL(__half))

extern "C" size_t hl_mx4_bytes(int64_t rows, int64_t dim) {
    if (!matrix_dims_ok(rows, dim)) return 0;
    return (size_t)(tiles_of(rows, kTileRows) * tiles_of(dim, kTileCols) * kTileBytes);
}

extern "C" int32_t hl_mx4_quantise(int32_t dtype, int64_t n_matrices, int64_t rows, int64_t dim, const void* d_x, int64_t ld,
                                   int64_t stride, void* d_q, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!matrix_dims_ok(rows, dim) || n_matrices < 0 || n_matrices >= (int64_t(1) << 31) || !row_matrix_ok(dtype, rows * n_matrices, dim, d_x, ld) ||
        stride < 0 || (!d_q && rows * n_matrices > 0) || !lies_at(d_q, 16))
        return HL_EINVAL;
    if (rows == 0 || n_matrices == 0) return HL_OK;
    if (n_matrices == 1) stride = 0;
    const bool whole = dim % 8 == 0 && rows_lie_at(dtype, d_x, ld, 16) && rows_lie_at(dtype, d_x, stride, 16);
#define HL_QUANTISE(T) launch_quantise<T>(n_matrices, rows, dim, d_x, ld, stride, d_q, whole, stream)
    return HL_FOR_TYPE(HL_QUANTISE);
#undef HL_QUANTISE
}

extern "C" int32_t hl_mx4_dequantise(int64_t n_matrices, int64_t rows, int64_t dim, const void* d_q, int32_t dtype, void* d_out,
                                     int64_t ld, int64_t stride, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!matrix_dims_ok(rows, dim) || n_matrices < 0 || n_matrices >= (int64_t(1) << 31) ||
        !row_matrix_ok(dtype, rows * n_matrices, dim, d_out, ld) || stride < 0 || (!d_q && rows * n_matrices > 0) || !lies_at(d_q, 16))
        return HL_EINVAL;
    if (rows == 0 || n_matrices == 0) return HL_OK;
    if (n_matrices == 1) stride = 0;
    const bool whole = dim % 8 == 0 && rows_lie_at(dtype, d_out, ld, 16) && rows_lie_at(dtype, d_out, stride, 16);
#define HL_DEQUANTISE(T) launch_dequantise<T>(n_matrices, rows, dim, d_q, d_out, ld, stride, whole, stream)
    return HL_FOR_TYPE(HL_DEQUANTISE);
#undef HL_DEQUANTISE
}

extern "C" size_t hl_expert_mx4_workspace_bytes(int64_t cap_rows, int32_t n_experts, int64_t dim) {
    if (cap_rows < 0 || cap_rows >= (int64_t(1) << 31) - 65536 || n_experts < 1 || n_experts > HL_MAX_EXPERTS || dim < 1 ||
        dim > (int64_t(1) << 24))
        return 0;
    return (size_t)(kWorkspaceHead + row_tiles_most(cap_rows, n_experts) * tiles_of(dim, kTileCols) * kPanelBytes);
}

extern "C" int32_t hl_expert_mx4_checked(const hl_route* route, int32_t dtype, int64_t dim, int64_t outputs, const void* d_x, int64_t ld_x,
                                         int32_t by_token, const void* d_weights, void* d_y, int64_t ld_y, void* d_workspace,
                                         size_t ws_bytes, int32_t* d_status, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const hl_route* r = route;
    if (!r || !lies_at(r->n_tokens, 4) || !lies_at(r->place, 4) || !lies_at(r->counts, 4) || !lies_at(r->offsets, 4) ||
        r->max_tokens < 0 || r->max_tokens >= (int64_t(1) << 30) || r->top_k < 1 || r->top_k > HL_MAX_TOP_K || r->n_experts < 1 ||
        r->n_experts > HL_MAX_EXPERTS || r->max_tokens * r->top_k >= (int64_t(1) << 30) || r->cap_rows < 0 ||
        r->cap_rows >= (int64_t(1) << 31) - 65536 || !r->counts || !r->offsets || (by_token && !r->place && r->max_tokens > 0))
        return HL_EINVAL;
    if (!row_matrix_ok(dtype, by_token ? r->max_tokens : r->cap_rows, dim, d_x, ld_x) || !row_matrix_ok(dtype, r->cap_rows, outputs, d_y, ld_y) ||
        !d_weights || !lies_at(d_weights, 16) || !d_workspace || !lies_at(d_workspace, 256) || !lies_at(d_status, 4))
        return HL_EINVAL;
    if (ws_bytes < hl_expert_mx4_workspace_bytes(r->cap_rows, r->n_experts, dim)) return HL_ECAPACITY;
    if (r->cap_rows == 0 || (by_token && r->max_tokens == 0)) {  // (no more than the status)
        HL_CUDA_TRY(clear_words(static_cast<uint32_t*>(d_workspace), 4, stream));
        return HL_OK;
    }
    const bool whole = dim % 8 == 0 && rows_lie_at(dtype, d_x, ld_x, 16);
#define HL_PRODUCT(T) launch_product<T>(r, dim, outputs, d_x, ld_x, by_token != 0, d_weights, d_y, ld_y, d_workspace, whole, d_status, stream)
    return HL_FOR_TYPE(HL_PRODUCT);
#undef HL_PRODUCT
}

extern "C" int32_t hl_expert_mx4(const hl_route* route, int32_t dtype, int64_t dim, int64_t outputs, const void* d_x, int64_t ld_x,
                                 int32_t by_token, const void* d_weights, void* d_y, int64_t ld_y, void* d_workspace, size_t ws_bytes,
                                 void* stream) {
    return hl_expert_mx4_checked(route, dtype, dim, outputs, d_x, ld_x, by_token, d_weights, d_y, ld_y, d_workspace, ws_bytes, nullptr, stream);
}
