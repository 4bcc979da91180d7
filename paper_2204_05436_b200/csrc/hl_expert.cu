// Tokens sorted by expert and back: the routing plan, the copies to the experts' rows, the weighted sums back, and the
// gradients of both.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "hl_common.cuh"

namespace cg = cooperative_groups;

namespace hl {
namespace {

// ---- the sort ---------------------------------------------------------------------------------------------------
// A stable counting sort of the choices by expert.  The choices are dealt out evenly, a run of them to each CTA and of those one
// to each warp, which takes 32 at a time: the choices of one expert among them rank by lane, behind those the warp has counted
// before.  A choice's row is: rows of the experts before + choices of the expert in CTAs before + in warps before + in the warp.
// (Choices are counted in 32 bits: there are less than 2^30.)
// No call here is near the memory's rate: a few choices cost what a launch does (4.7 us a call back to back, one token), some ten
// thousand the latency of one kernel's steps -- load, rank, counts of the other CTAs, places -- (16 384 x 4 choices of 64 experts
// with 5 899 tokens of them there: 5.5 us of kernel, 8.2 a call), and 2.1 M of 256 experts 25.3 us, 25 MB at 1.0 TB/s: 12.7 the ranks,
// which issue an instruction in 60 % of the cycles, 5.5 the sums over the tiles, 11.3 the places, half of it at barriers and in
// shared memory.  (The sums of several kernels overlap: each starts while the one before it ends.)
constexpr uint32_t kNone = 0xffffu;

// what the sort writes, and the words it goes by
struct SortOut {
    int32_t *place, *source, *counts, *offsets, *status;
    int cap_rows, expert_cap, align;
};

__device__ __forceinline__ int live_choices(const int32_t* n_tokens, int max_tokens, int top_k) {
    int t = max_tokens;
    if (n_tokens) t = min(max(__ldg(n_tokens), 0), max_tokens);
    return t * top_k;
}

// CTAs of NT threads with at most ITEMS rounds of 32 choices per warp.
template <int NT, int ITEMS>
struct Sort {
    static constexpr int kWarps = NT / 32, kChoices = NT * ITEMS, kPer = HL_MAX_EXPERTS / NT;     // experts of a thread
    static_assert(HL_MAX_EXPERTS == 1024 && kChoices <= 32768, "ten bits of expert, ranks of 15");

    uint16_t* warp_hist;               // [kWarps][E]; then choices of the expert in the warps before
    int32_t* hist;                     // [E + 1] of this CTA, [E]: ids that are no expert's; then of the CTAs before
    int32_t* offset;                   // [E + 1]
    int32_t* count;                    // [E + 1]
    int E, pitch;

    static constexpr size_t smem_bytes(int E) { return 4 * ((size_t)kWarps * ((E + 1) / 2) + 3 * (size_t)(E + 1)); }

    __device__ __forceinline__ Sort(uint32_t* base, int E_) : E(E_), pitch(2 * ((E_ + 1) / 2)) {
        warp_hist = reinterpret_cast<uint16_t*>(base);
        hist = reinterpret_cast<int32_t*>(base + kWarps * (pitch / 2));
        offset = hist + E + 1;
        count = offset + E + 1;
    }

    // The lanes with the same value of BITS bits, among those that are valid.  (A match over the warp does it in one
    // instruction, which takes the multiprocessor 60 cycles; a ballot a bit takes three: eight bits 24.)
    template <int BITS>
    static __device__ __forceinline__ unsigned same_value(unsigned v, bool valid) {
        unsigned peers = __ballot_sync(0xffffffffu, valid);
#pragma unroll
        for (int b = 0; b < BITS; ++b) {
            const unsigned bit = (v >> b) & 1u;
            peers &= __ballot_sync(0xffffffffu, bit) ^ (bit - 1u);           // those with the bit, or those without
        }
        return peers;
    }

    // A warp's rounds: e in, packed out (expert in the upper 16 bits, kNone: none; rank in the warp), counted into h.
    template <int BITS>
    __device__ __forceinline__ void rank_rounds(const int (&e)[ITEMS], int rounds, uint16_t* h, uint32_t (&packed)[ITEMS]) const {
        const unsigned lt = lanemask_lt();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            packed[i] = kNone << 16;
            if (i >= rounds) continue;
            const bool ok = e[i] >= 0;
            const unsigned peers = same_value<BITS>((unsigned)e[i], ok), below = peers & lt;
            if (ok) packed[i] = ((uint32_t)e[i] << 16) | (h[e[i]] + __popc(below));
            __syncwarp();
            if (ok && below == 0) h[e[i]] = (uint16_t)(packed[i] + __popc(peers));
            __syncwarp();
        }
    }

    // Ranks the CTA's choices [first, first + rounds * NT) below n, of `most` that can be read, and counts them: warp_hist, hist.
    template <int BITS>
    __device__ __forceinline__ void rank(const int32_t* __restrict__ experts, int first, int rounds, int n, int most,
                                         uint32_t (&packed)[ITEMS]) const {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, seg = first + warp * (rounds * 32) + lane;
        int e[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) e[i] = i < rounds && seg + i * 32 < most ? __ldg(&experts[seg + i * 32]) : -1;
        for (int i = threadIdx.x; i < kWarps * pitch / 2; i += NT) reinterpret_cast<uint32_t*>(warp_hist)[i] = 0;
        if (threadIdx.x == 0) hist[E] = 0;
        __syncthreads();
        bool bad = false;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (seg + i * 32 >= n) e[i] = -1;
            if ((unsigned)e[i] >= (unsigned)E) {
                bad = bad || e[i] != -1;
                e[i] = -1;
            }
        }
        rank_rounds<BITS>(e, rounds, warp_hist + warp * pitch, packed);
        if (__any_sync(0xffffffffu, bad) && lane == 0) atomicAdd(&hist[E], 1);
        __syncthreads();
        for (int x = threadIdx.x; x < E; x += NT) {
            int c[kWarps], sum = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) c[w] = warp_hist[w * pitch + x];
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                warp_hist[w * pitch + x] = (uint16_t)sum;
                sum += c[w];
            }
            hist[x] = sum;
        }
        __syncthreads();
    }

    // Sum of v over the threads before; *all: over all of them.
    static __device__ __forceinline__ int before(int v, int* all) {
        __shared__ int s_warp[kWarps];
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        int incl = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += x;
        }
        __syncthreads();
        if (lane == 31) s_warp[warp] = incl;
        __syncthreads();
        int at = incl - v;
        *all = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            at += w < warp ? s_warp[w] : 0;
            *all += s_warp[w];
        }
        return at;
    }

    // count holds every expert's choices: turns them into the rows it gets and their offsets, both inside cap_rows.  Returns
    // whether some rows did not fit, those that fill experts up among them.  (All together: less than 2^30 + 2^26.)  A thread has
    // kPer experts in a row.
    __device__ __forceinline__ bool place(const SortOut& o) const {
        int rows[kPer], cnt[kPer], sum = 0, all;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int e = kPer * threadIdx.x + k;
            rows[k] = cnt[k] = 0;
            if (e >= E) continue;
            cnt[k] = count[e];
            if (o.expert_cap > 0) cnt[k] = min(cnt[k], o.expert_cap);
            rows[k] = o.align == 1 ? cnt[k] : (int)((uint32_t)(cnt[k] + o.align - 1) / (uint32_t)o.align) * o.align;
            sum += rows[k];
        }
        int at = before(sum, &all);
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int e = kPer * threadIdx.x + k;
            if (e >= E) break;
            offset[e] = min(at, o.cap_rows);
            count[e] = min(cnt[k], max(o.cap_rows - at, 0));
            at += rows[k];
        }
        if (threadIdx.x == 0) offset[E] = min(all, o.cap_rows);
        __syncthreads();
        return all > o.cap_rows;
    }

    // The rows that fill an expert up, and the plan's words, by CTA `cta` of `ctas`.
    __device__ __forceinline__ void write_plan(const SortOut& o, int cta, int ctas, bool over, bool bad) const {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (o.source && o.align > 1)
            for (int e = cta * kWarps + warp; e < E; e += ctas * kWarps)
                for (int r = offset[e] + count[e] + lane; r < offset[e + 1]; r += 32) o.source[r] = -1;
        if (cta != 0) return;
        for (int e = threadIdx.x; e < E; e += NT) {
            o.counts[e] = count[e];
            o.offsets[e] = offset[e];
        }
        if (threadIdx.x == 0) {
            o.offsets[E] = offset[E];
            if (o.status) *o.status = bad ? HL_EBOUNDS : over ? HL_ECAPACITY : HL_OK;
        }
    }
};

// All of it in one cluster, whose CTAs read each other's counts.  (A kernel for every two bits of the experts' numbers: what one
// holds it has to fetch first, and a call alone pays for that -- all four in one: 14.6 us instead of 8.6 where nothing is cached.)
template <int CTAS, int NT, int ITEMS, int BITS>
__global__ void __launch_bounds__(NT) k_expert_sort(const int32_t* __restrict__ experts, const int32_t* n_tokens,
                                                    int max_tokens, int top_k, int E, int expert_cap, int align, int cap_rows,
                                                    int32_t* place, int32_t* source, int32_t* counts, int32_t* offsets,
                                                    int32_t* status) {
    extern __shared__ uint32_t s_base[];
    const Sort<NT, ITEMS> s(s_base, E);
    const SortOut o{place, source, counts, offsets, status, cap_rows, expert_cap, align};
    const int n = live_choices(n_tokens, max_tokens, top_k);
    // (one CTA asks for what there can be at once, rather than wait for how many there are)
    const int most = CTAS == 1 ? max_tokens * top_k : n, rounds = (most + CTAS * NT - 1) / (CTAS * NT);
    const int first = (int)blockIdx.x * rounds * NT;
    uint32_t packed[ITEMS];
    s.template rank<BITS>(experts, first, rounds, n, most, packed);
    if constexpr (CTAS > 1) {
        constexpr int kMine = HL_MAX_EXPERTS / NT + 1;
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        int before[kMine] = {};
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int e = threadIdx.x + k * NT;
            if (e > E) break;
            int v[CTAS], all = 0;
#pragma unroll
            for (int c = 0; c < CTAS; ++c) v[c] = *cluster.map_shared_rank(&s.hist[e], c);
#pragma unroll
            for (int c = 0; c < CTAS; ++c) {
                if (c < (int)blockIdx.x) before[k] += v[c];
                all += v[c];
            }
            s.count[e] = all;
        }
        cluster.sync();                // (nobody reads this CTA's counts any more)
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int e = threadIdx.x + k * NT;
            if (e <= E) s.hist[e] = before[k];
        }
    } else {
        for (int e = threadIdx.x; e <= E; e += NT) {
            s.count[e] = s.hist[e];
            s.hist[e] = 0;
        }
    }
    __syncthreads();
    const bool bad = s.count[E] != 0;
    const bool over = s.place(o);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int a = first + (warp * rounds + i) * 32 + lane;
        if (i >= rounds || a >= n) continue;
        const uint32_t e = packed[i] >> 16;
        int32_t row = -1;
        if (e != kNone) {
            const int r = s.hist[e] + s.warp_hist[warp * s.pitch + e] + (int)(packed[i] & 0xffffu);
            if (r < s.count[e]) row = s.offset[e] + r;
        }
        place[a] = row;
        if (row >= 0 && source) source[row] = a;
    }
    s.write_plan(o, blockIdx.x, CTAS, over, bad);
}

// In three kernels: every tile's choices ranked (their expert and rank in the tile, as packed above, into `ranked`) and
// counted, sums of the counts over the tiles before, places.  tile_counts: [tiles][E + 1].
constexpr int kTileNT = 512, kTileItems = 16;
using Tile = Sort<kTileNT, kTileItems>;
__device__ __forceinline__ int tile_rounds(int n, int tiles) {
    return (int)(((int64_t)n + (int64_t)tiles * kTileNT - 1) / ((int64_t)tiles * kTileNT));
}

template <int BITS>
__global__ void __launch_bounds__(kTileNT) k_expert_rank(const int32_t* __restrict__ experts, const int32_t* n_tokens,
                                                         int max_tokens, int top_k, int E, int32_t* __restrict__ tile_counts,
                                                         uint32_t* __restrict__ ranked) {
    extern __shared__ uint32_t s_base[];
    let_next_start();
    const Tile s(s_base, E);
    const int n = live_choices(n_tokens, max_tokens, top_k), tiles = gridDim.x, rounds = tile_rounds(n, tiles);
    const int first = min((int64_t)blockIdx.x * rounds * kTileNT, (int64_t)n);
    uint32_t packed[kTileItems];
    s.rank<BITS>(experts, first, rounds, n, n, packed);
    for (int e = threadIdx.x; e <= E; e += kTileNT) tile_counts[(int64_t)blockIdx.x * (E + 1) + e] = s.hist[e];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int a = first + (warp * rounds + i) * 32 + lane;
        const uint32_t e = packed[i] >> 16;
        if (i < rounds && a < n) ranked[a] = e == kNone ? packed[i] : packed[i] + s.warp_hist[warp * s.pitch + e];
    }
}

// tile_counts[t][e] := sum over the tiles before t; totals[e].  A CTA takes 32 experts, its warps a run of tiles each.
constexpr int kScanNT = 1024;
__global__ void __launch_bounds__(kScanNT) k_expert_scan(int32_t* __restrict__ tile_counts, int tiles, int E,
                                                         int32_t* __restrict__ totals) {
    constexpr int kWarps = kScanNT / 32, kAhead = 16;
    __shared__ int s_sum[kWarps][33];                // (33: read by rows and by columns)
    let_next_start();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = (int)blockIdx.x * 32 + lane;
    const int per = (tiles + kWarps - 1) / kWarps, t0 = min(warp * per, tiles), t1 = min(t0 + per, tiles);
    int32_t* column = tile_counts + min(e, E);
    wait_for_last();
    int c[kAhead], sum = 0;            // the first of the run's tiles stay in registers
#pragma unroll
    for (int i = 0; i < kAhead; ++i) c[i] = t0 + i < t1 ? column[(int64_t)(t0 + i) * (E + 1)] : 0;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) sum += c[i];
    for (int t = t0 + kAhead; t < t1; ++t) sum += column[(int64_t)t * (E + 1)];
    s_sum[warp][lane] = sum;
    __syncthreads();
    const int v = s_sum[lane][warp];                 // of expert `warp`: the sum of warp `lane`
    int incl = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += x;
    }
    s_sum[lane][warp] = incl - v;
    __syncthreads();
    int before = s_sum[warp][lane];
    if (e > E) return;
    if (warp == kWarps - 1) totals[e] = before + sum;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        if (t0 + i < t1) column[(int64_t)(t0 + i) * (E + 1)] = before;
        before += c[i];
    }
    for (int t = t0 + kAhead; t < t1; ++t) {
        const int x = column[(int64_t)t * (E + 1)];
        column[(int64_t)t * (E + 1)] = before;
        before += x;
    }
}

// A tile's choices are put in order of their rows in shared memory first, so that what `source` gets are runs: written as they
// come, 32 choices of a warp go to 32 lines.
constexpr size_t place_smem_bytes(int E) { return 12 * (size_t)(E + 1) + 4 * (size_t)Tile::kChoices; }
__global__ void __launch_bounds__(kTileNT) k_expert_place(const int32_t* n_tokens, int max_tokens, int top_k, int E,
                                                          int expert_cap, int align, int cap_rows, int32_t* place,
                                                          int32_t* source, int32_t* counts, int32_t* offsets, int32_t* status,
                                                          const int32_t* tile_counts, const int32_t* totals,
                                                          const uint32_t* ranked) {
    extern __shared__ uint32_t s_base[];
    Tile s(s_base, E);
    s.hist = reinterpret_cast<int32_t*>(s_base);
    s.offset = s.hist + E + 1;
    s.count = s.offset + E + 1;
    uint32_t* s_order = reinterpret_cast<uint32_t*>(s.count + E + 1);      // expert (16 bits), choice of the tile
    const SortOut o{place, source, counts, offsets, status, cap_rows, expert_cap, align};
    const int n = live_choices(n_tokens, max_tokens, top_k), tiles = gridDim.x, rounds = tile_rounds(n, tiles);
    const int first = min((int64_t)blockIdx.x * rounds * kTileNT, (int64_t)n), here = min(rounds * kTileNT, n - first);
    wait_for_last();
    uint32_t packed[kTileItems];
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int j = i * kTileNT + threadIdx.x;
        packed[i] = j < here ? ranked[first + j] : kNone << 16;
    }
    int in_tile[Tile::kPer], mine = 0;                         // of the experts that place() gives a thread
    const int e0 = Tile::kPer * threadIdx.x;
#pragma unroll
    for (int k = 0; k < Tile::kPer; ++k) {
        in_tile[k] = 0;
        if (e0 + k >= E) continue;
        const int32_t* row = &tile_counts[(int64_t)blockIdx.x * (E + 1) + e0 + k];
        const int before = row[0], all = totals[e0 + k];
        s.hist[e0 + k] = before;
        s.count[e0 + k] = all;
        in_tile[k] = ((int)blockIdx.x + 1 < tiles ? row[E + 1] : all) - before;
        mine += in_tile[k];
    }
    const bool bad = totals[E] != 0;
    const bool over = s.place(o);
    s.write_plan(o, blockIdx.x, gridDim.x, over, bad);
    // from here on: hist: row of an expert's first choice in the tile, count: end of its rows, offset: its first choice in order
    int in_order, at = Tile::before(mine, &in_order);
#pragma unroll
    for (int k = 0; k < Tile::kPer; ++k) {
        if (e0 + k >= E) continue;
        const int off = s.offset[e0 + k];
        s.hist[e0 + k] += off;
        s.count[e0 + k] += off;
        s.offset[e0 + k] = at;
        at += in_tile[k];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int j = i * kTileNT + threadIdx.x;
        if (j >= here) continue;
        const uint32_t e = packed[i] >> 16, rank = packed[i] & 0xffffu;
        int32_t row = -1;
        if (e != kNone) {
            row = s.hist[e] + (int)rank;
            if (row >= s.count[e]) row = -1;
            s_order[s.offset[e] + rank] = (e << 16) | (uint32_t)j;
        }
        place[first + j] = row;
    }
    if (!source) return;
    __syncthreads();
    for (int j = threadIdx.x; j < in_order; j += kTileNT) {
        const uint32_t x = s_order[j], e = x >> 16;
        const int row = s.hist[e] + j - s.offset[e];
        if (row < s.count[e]) source[row] = first + (int)(x & 0xffffu);
    }
}

// Which of them sorts n choices, up to kOneCluster.  One CTA for as many as its first loads take; then clusters of 8 CTAs, beyond
// 8 192 choices of 16, with as few rounds unrolled as there can be.  us each, back to back, 8 / 16 CTAs: 4 096 choices of 64 experts
// 3.9 / 4.0, of 500 4.8 / 5.7 (every CTA reads all the others' counts); 16 000 of 64 5.2 / 4.4, of 500 6.5 / 6.3; 65 536 of 64 11.0 /
// 7.7, of 500 13.8 / 10.1.  Three kernels take 11.5 (64 experts) to 12.3 us (500) from 17 000 to 131 072 choices, a cluster 11.7 and
// 15.1 at 131 072, 9.8 and 12.3 at 90 000.
constexpr int64_t kFewChoices = 128 * 4, kOneCluster = 16 * 512 * 12;

// ---- rows -----------------------------------------------------------------------------------------------------------
// 16 bytes of a row are moved as one.  Where all rows of a call begin at multiples of 16 bytes and have whole ones, that is a load or
// a store; other rows are "ragged", below.
template <typename T>
struct Vec {
    static constexpr int N = 16 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ Vec() : raw(make_uint4(0, 0, 0, 0)) {}
    __device__ __forceinline__ void load(const T* p) { raw = __ldg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = raw; }
    // (two values of a word at a time: the conversions to fp32 and back have instructions for that)
    __device__ __forceinline__ void get(float (&x)[N]) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                x[i] = __uint_as_float(w[i]);
            } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            } else {
                const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                x[2 * i] = v.x;
                x[2 * i + 1] = v.y;
            }
        }
    }
    __device__ __forceinline__ void set(const float (&x)[N]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                w[i] = __float_as_uint(x[i]);
            } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&v);
            } else {
                const __half2 v = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&v);
            }
        }
        raw = make_uint4(w[0], w[1], w[2], w[3]);
    }
    // value i, for an i known when this is compiled
    __device__ __forceinline__ T value(int i) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        if constexpr (sizeof(T) == 4) {
            return *reinterpret_cast<const T*>(&w[i]);
        } else {
            const uint16_t h = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
            return *reinterpret_cast<const T*>(&h);
        }
    }
};

// rows, ld values from one's begin to the next's
template <typename T>
struct Rows {
    T* p;
    int ld;
    __device__ __forceinline__ T* at(int r) const { return p + (int64_t)r * ld; }
};

constexpr int kRowNT = 256;

template <typename T>
__device__ __forceinline__ int in_line(const T* p) {           // values between the 16-byte line's begin and p
    return (int)(reinterpret_cast<uintptr_t>(p) & 15) / (int)sizeof(T);
}
// values [e, e + N) of a row of dim values, as much of them as there is; row + e is where a line begins
template <typename T>
__device__ __forceinline__ void store_line(T* row, int e, int dim, const Vec<T>& v) {
    constexpr int N = Vec<T>::N;
    if (e >= 0 && e + N <= dim) {
        v.store(row + e);
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if ((unsigned)(e + j) < (unsigned)dim) row[e + j] = v.value(j);
}

// Rows that fill experts up: CTA u of units x E takes every units-th of expert u % E's, several side by side if they are short.
template <typename T>
__device__ __forceinline__ void zero_pads(int u, int units, int E, const int32_t* __restrict__ counts,
                                          const int32_t* __restrict__ offsets, int cap_rows, Rows<T> y, int dim) {
    constexpr int N = Vec<T>::N;
    const int e = u % E, part = u / E, end = min(__ldg(&offsets[e + 1]), cap_rows);
    const int64_t first = __ldg(&offsets[e]), count = __ldg(&counts[e]);
    if (first < 0 || count < 0) return;
    int P = 1;                         // threads of a row
    while (P < kRowNT && P * N < dim) P *= 2;
    const int sub = threadIdx.x & (P - 1), side = threadIdx.x / P, sides = kRowNT / P;
    const Vec<T> zero;
    for (int64_t r = first + count + part * sides + side; r < end; r += units * sides) {
        T* row = y.at((int)r);
        for (int c = sub * N - in_line(row); c < dim; c += P * N) store_line(row, c, dim, zero);
    }
}

// Which token and vector a thread's item is: items are dealt out in turn, kRowNT * U to a CTA.  Divisions would be a good part of
// the kernels' instructions: the host gives 2^64 / vectors, rounded up (exact quotients for less than 2^40 items and rows of less
// than 2^24 vectors); inside a CTA 2^32 / vectors does for less than 32 768 of them, beyond which one token at most follows the first.
template <int U>
struct Items {
    int t0;
    unsigned r0, magic;
    int vectors;
    __device__ __forceinline__ Items(int vectors_, uint64_t inverse) : vectors(vectors_) {
        const uint64_t first = (uint64_t)blockIdx.x * (kRowNT * U);
        t0 = vectors == 1 ? (int)first : (int)__umul64hi(first, inverse);
        r0 = (unsigned)(first - (uint64_t)t0 * vectors);
        magic = (unsigned)((inverse + 0xffffffffu) >> 32);
    }
    __device__ __forceinline__ void get(int u, int* t, int* vector) const {
        const unsigned i = r0 + u * kRowNT + threadIdx.x;
        const unsigned q = vectors == 1 ? i : vectors >= 32768 ? i >= (unsigned)vectors : __umulhi(i, magic);
        *t = t0 + (int)q;
        *vector = (int)(i - q * vectors);
    }
};
uint64_t inverse_of(int vectors) { return vectors == 1 ? 0 : ~uint64_t(0) / vectors + 1; }

// y[place[t, k]] = x[t], V at a time: 16 bytes, or as many as all rows begin at multiples of and have whole ones of.  A thread takes U
// of them of tokens' rows, which it reads once for all of a token's rows.  T: what a value is, as far as copying goes.
// Bound by memory: 16 384 rows of 1 664 fp32 to two rows each, 327 MB in 48 us: 6.8 TB/s.  (Stores that the L2 gives up first: the
// same.)
template <typename V>
constexpr int kDispatchVectors = sizeof(V) == 16 ? 2 : 4;
template <typename T, typename V>
__global__ void __launch_bounds__(kRowNT, 6) k_expert_dispatch(const T* __restrict__ x_, int ld_x, const int32_t* n_tokens,
                                                               int max_tokens, int top_k, int dim,
                                                               const int32_t* __restrict__ place, int cap_rows,
                                                               T* __restrict__ y_, int ld_y, int vectors, uint64_t inverse,
                                                               int row_ctas, int E, int pad_units,
                                                               const int32_t* __restrict__ counts,
                                                               const int32_t* __restrict__ offsets) {
    constexpr int KU = 4, U = kDispatchVectors<V>, W = sizeof(V) / sizeof(T);
    const Rows<const T> x{x_, ld_x};
    const Rows<T> y{y_, ld_y};
    if ((int)blockIdx.x >= row_ctas) {
        zero_pads<T>(blockIdx.x - row_ctas, pad_units, E, counts, offsets, cap_rows, y, dim);
        return;
    }
    const int tokens = live_choices(n_tokens, max_tokens, 1);
    const Items<U> items(vectors, inverse);
    V v[U];
    int t[U], c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        items.get(u, &t[u], &c[u]);
        c[u] *= W;
        if (t[u] < tokens) v[u] = __ldg(reinterpret_cast<const V*>(x.at(t[u]) + c[u]));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (t[u] >= tokens) continue;
        const int32_t* at = place + t[u] * top_k;
        for (int k0 = 0; k0 < top_k; k0 += KU) {
            int row[KU];
#pragma unroll
            for (int q = 0; q < KU; ++q) row[q] = k0 + q < top_k ? __ldg(&at[k0 + q]) : -1;
#pragma unroll
            for (int q = 0; q < KU; ++q)
                if ((unsigned)row[q] < (unsigned)cap_rows) *reinterpret_cast<V*>(y.at(row[q]) + c[u]) = v[u];
        }
    }
}

// out[t] = sum over k of w[t, k] * y[place[t, k]], in fp32, in the order of k, rounded once.  (Without weights: the sum.)  A
// thread takes a vector of out, or U of them one after the other, and KU of the token's rows at a time.  Bound by memory: 8 rows of
// 2 048 bf16 for each of 16 384 tokens, 604 MB in 92.5 us: 6.5 TB/s; two of 1 664 fp32, 327 MB in 53.5: 6.1.
template <typename T, int KU, int U>
__global__ void __launch_bounds__(kRowNT, 6) k_expert_combine(const T* __restrict__ y_, int ld_y, int cap_rows,
                                                              const int32_t* n_tokens, int max_tokens, int top_k,
                                                              const int32_t* __restrict__ place,
                                                              const float* __restrict__ weights, T* __restrict__ out_,
                                                              int ld_out, int vectors, uint64_t inverse) {
    constexpr int W = Vec<T>::N;
    const Rows<const T> y{y_, ld_y};
    const Rows<T> out{out_, ld_out};
    const int tokens = live_choices(n_tokens, max_tokens, 1);
    const Items<U> items(vectors, inverse);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        int t, c;
        items.get(u, &t, &c);
        if (t >= tokens) return;
        c *= W;
        const int32_t* at = place + t * top_k;
        const float* w_at = weights + t * top_k;
        float acc[W] = {};
        for (int k0 = 0; k0 < top_k; k0 += KU) {
            int row[KU];
            float w[KU];
            Vec<T> v[KU];
#pragma unroll
            for (int q = 0; q < KU; ++q) {
                row[q] = k0 + q < top_k ? __ldg(&at[k0 + q]) : -1;
                w[q] = weights && k0 + q < top_k ? __ldg(&w_at[k0 + q]) : 1.f;
            }
#pragma unroll
            for (int q = 0; q < KU; ++q) {
                const bool ok = (unsigned)row[q] < (unsigned)cap_rows;
                if (ok) v[q].load(y.at(row[q]) + c);
                w[q] = ok ? w[q] : 0.f;
            }
#pragma unroll
            for (int q = 0; q < KU; ++q) {
                float x[W];
                v[q].get(x);
#pragma unroll
                for (int j = 0; j < W; ++j) acc[j] = fmaf(w[q], x[j], acc[j]);
            }
        }
        Vec<T> r;
        r.set(acc);
        r.store(out.at(t) + c);
    }
}

// The sums of P threads' dot products, in the first of them.  (All threads of the CTA call it.)
template <int KU>
__device__ __forceinline__ void sum_dots(float (&dot)[KU], int P, float* s_dot) {
    for (int d = min(P, 32) / 2; d > 0; d >>= 1)
#pragma unroll
        for (int q = 0; q < KU; ++q) dot[q] += __shfl_xor_sync(0xffffffffu, dot[q], d);
    if (P <= 32) return;
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int q = 0; q < KU; ++q) s_dot[warp * KU + q] = dot[q];
    __syncthreads();
    if ((threadIdx.x & (P - 1)) == 0)
        for (int o = 1; o < P / 32; ++o)
#pragma unroll
            for (int q = 0; q < KU; ++q) dot[q] += s_dot[(warp + o) * KU + q];
    __syncthreads();
}

// grad_y[place[t, k]] = w[t, k] * grad_out[t]; grad_w[t, k] = <grad_out[t], y[place[t, k]]>.  P threads (a power of two) take a
// token, KU of its rows at a time, so that grad_out is read once for those and the dot products need no atomics.  Bound by memory:
// 16 384 tokens, 8 rows of 2 048 bf16 each, 1 141 MB in 190 us: 6.0 TB/s.
template <typename T>
__global__ void __launch_bounds__(kRowNT, 4) k_expert_combine_bwd(
    const T* __restrict__ go_, int ld_go, const T* __restrict__ y_, int ld_y, int cap_rows, const int32_t* n_tokens,
    int max_tokens, int top_k, int dim, const int32_t* __restrict__ place, const float* __restrict__ weights,
    T* __restrict__ gy_, int ld_gy, float* __restrict__ grad_w, int P, int row_ctas, int E, int pad_units,
    const int32_t* __restrict__ counts, const int32_t* __restrict__ offsets) {
    constexpr int KU = 4, W = Vec<T>::N;
    const Rows<const T> go{go_, ld_go}, y{y_, ld_y};
    const Rows<T> gy{gy_, ld_gy};
    if ((int)blockIdx.x >= row_ctas) {
        zero_pads<T>(blockIdx.x - row_ctas, pad_units, E, counts, offsets, cap_rows, gy, dim);
        return;
    }
    __shared__ float s_dot[kRowNT / 32 * KU];
    const int sub = threadIdx.x & (P - 1);
    const int tokens = live_choices(n_tokens, max_tokens, 1);
    const int t = (int)((int64_t)blockIdx.x * (kRowNT / P)) + (int)threadIdx.x / P;
    for (int k0 = 0; k0 < top_k; k0 += KU) {
        int row[KU];
        float w[KU], dot[KU];
#pragma unroll
        for (int q = 0; q < KU; ++q) {
            row[q] = t < tokens && k0 + q < top_k ? __ldg(&place[t * top_k + k0 + q]) : -1;
            if (row[q] >= cap_rows) row[q] = -1;
            w[q] = row[q] >= 0 && weights ? __ldg(&weights[t * top_k + k0 + q]) : 1.f;
            dot[q] = 0.f;
        }
        for (int c = t < tokens ? sub * W : dim; c < dim; c += P * W) {
            Vec<T> g, v[KU];
            float x[W];
            g.load(go.at(t) + c);
#pragma unroll
            for (int q = 0; q < KU; ++q)
                if (row[q] >= 0 && grad_w) v[q].load(y.at(row[q]) + c);
#pragma unroll
            for (int q = 0; q < KU; ++q) {
                if (row[q] < 0) continue;
                Vec<T> r;
                float y[W], z[W];
                g.get(x);
                v[q].get(y);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    dot[q] = fmaf(x[j], y[j], dot[q]);
                    z[j] = w[q] * x[j];
                }
                r.set(z);
                r.store(gy.at(row[q]) + c);
            }
        }
        sum_dots(dot, P, s_dot);
        if (sub == 0 && t < tokens && grad_w)
#pragma unroll
            for (int q = 0; q < KU; ++q)
                if (k0 + q < top_k) grad_w[t * top_k + k0 + q] = dot[q];
    }
}

// ---- ragged rows ----------------------------------------------------------------------------------------------------
// A row that is written is cut where its own 16-byte lines begin, so that all stores but those at its ends are whole lines; the 16
// bytes that belong there lie anywhere in the row that is read, and are put together from the two lines that they lie in.  Lines that
// are not all inside a buffer are not read.  Neither at the memory's rate nor at that of instructions (66 and 53 % of the cycles issue
// one, a third of them to put lines together): the latency of two loads in a row with half of the warps there, every line that is read
// asked for twice, by neighbours, and in the sums place, weight and address found out again for every line.  Three rows of 337 fp16 for
// each of 28 657 tokens, a tenth of them none: sums 71 MB in 22 us, gradients 123 MB in 34: 3.2 and 3.6 TB/s.  Value by value they took
// 23 to 29 and 64 to 118; a line a thread for both, with the lines in registers, 119 together.
template <typename T>
struct Buffer {
    const T* p;
    int ld, dim;
    int64_t values;                    // of all its rows
    __device__ __forceinline__ Buffer(const T* p_, int ld_, int rows, int dim_)
        : p(p_), ld(ld_), dim(dim_), values((int64_t)(rows - 1) * ld_ + dim_) {}
    // whether the lines that a row's values lie in, and one more on either side, are inside
    __device__ __forceinline__ bool inside(int r) const {
        const int64_t at = (int64_t)r * ld;
        return at >= 2 * Vec<T>::N && at + dim + 2 * Vec<T>::N <= values;
    }
};

// What is read of a row by lines of another that begin at values -shift, N - shift, ... of it.
struct Lines {
    uint4 a, b;
};
template <typename T>
struct Ragged {
    const uint4* line;                 // the line in which value -shift lies
    int s;                             // its byte in there
    __device__ __forceinline__ Ragged() {}
    __device__ __forceinline__ Ragged(const Buffer<T>& b, int r, int shift) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(b.p + ((int64_t)r * b.ld - shift));
        line = reinterpret_cast<const uint4*>(a & ~(uintptr_t)15);
        s = (int)(a & 15);
    }
    __device__ __forceinline__ Lines ask(int l) const { return {__ldg(line + l), __ldg(line + l + 1)}; }
    // what line l of the other begins with; values outside of the row are anything
    __device__ __forceinline__ Vec<T> take(const Lines& x) const {
        const bool far = s & 8, odd = s & 4;
        const uint32_t w0 = far ? x.a.z : x.a.x, w1 = far ? x.a.w : x.a.y, w2 = far ? x.b.x : x.a.z, w3 = far ? x.b.y : x.a.w,
                       w4 = far ? x.b.z : x.b.x, w5 = far ? x.b.w : x.b.y;
        const uint32_t y0 = odd ? w1 : w0, y1 = odd ? w2 : w1, y2 = odd ? w3 : w2, y3 = odd ? w4 : w3, y4 = odd ? w5 : w4;
        const int bits = s * 8;        // (a funnel shift takes it modulo 32)
        Vec<T> r;
        r.raw = sizeof(T) == 4 ? make_uint4(y0, y1, y2, y3)
                               : make_uint4(__funnelshift_r(y0, y1, bits), __funnelshift_r(y1, y2, bits),
                                            __funnelshift_r(y2, y3, bits), __funnelshift_r(y3, y4, bits));
        return r;
    }
};

__device__ __forceinline__ float value_of(const float* p) { return *p; }
__device__ __forceinline__ float value_of(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float value_of(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ void put_value(float* p, float x) { *p = x; }
__device__ __forceinline__ void put_value(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
__device__ __forceinline__ void put_value(__half* p, float x) { *p = __float2half_rn(x); }

// The forward kernel takes a line a thread, as that of whole rows does.  Lines are asked for into shared memory of the thread's own:
// registers for them would leave room for half as many threads.
template <typename T>
__device__ __noinline__ uint4 line_by_value(const T* p, int64_t at, int64_t values) {          // (at a buffer's end)
    alignas(16) T x[Vec<T>::N] = {};
    for (int j = 0; j < Vec<T>::N; ++j)
        if (at + j >= 0 && at + j < values) x[j] = p[at + j];
    return *reinterpret_cast<const uint4*>(x);
}
template <typename T>
struct LineBuffer {
    const T* p;
    int64_t values;
    uint64_t most;                     // places N to most + N have two lines inside the buffer, whatever its alignment
    __device__ __forceinline__ LineBuffer(const T* p_, int ld, int rows, int dim)
        : p(p_), values((int64_t)(rows - 1) * ld + dim), most(values > 3 * Vec<T>::N ? values - 3 * Vec<T>::N : 0) {}
    // slot: two of the thread's, kRowNT apart.  Returns the bytes of the first line that are not wanted, or -1: by value.
    __device__ __forceinline__ int ask(int64_t at, uint4* slot) const {
        if ((uint64_t)(at - Vec<T>::N) >= most) return -1;
        const uintptr_t a = reinterpret_cast<uintptr_t>(p + at), line = a & ~(uintptr_t)15;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot);
        asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(to), "l"(line) : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(to + kRowNT * 16), "l"(line + 16) : "memory");
        return (int)(a & 15);
    }
    __device__ __forceinline__ Vec<T> take(int s, const uint4* slot, int64_t at) const {
        Vec<T> r;
        if (s < 0) {
            r.raw = line_by_value(p, at, values);
            return r;
        }
        Ragged<T> x;
        x.s = s;
        return x.take({slot[0], slot[kRowNT]});
    }
};
__device__ __forceinline__ void wait_lines() { asm volatile("cp.async.wait_all;" ::: "memory"); }

template <typename T>
__global__ void __launch_bounds__(kRowNT, 5) k_expert_combine_ragged(const T* __restrict__ y_, int ld_y, int cap_rows,
                                                                     const int32_t* n_tokens, int max_tokens, int top_k,
                                                                     int dim, const int32_t* __restrict__ place,
                                                                     const float* __restrict__ weights, T* __restrict__ out_,
                                                                     int ld_out, int lines, uint64_t inverse) {
    constexpr int N = Vec<T>::N, KU = 4;
    __shared__ uint4 s_lines[KU][2][kRowNT];
    const LineBuffer<T> y(y_, ld_y, cap_rows, dim);
    int t, line;
    Items<1>(lines, inverse).get(0, &t, &line);
    if (t >= live_choices(n_tokens, max_tokens, 1)) return;
    T* to = Rows<T>{out_, ld_out}.at(t);
    const int e = line * N - in_line(to);
    if (e >= dim) return;
    const int32_t* at = place + t * top_k;
    const float* w_at = weights + t * top_k;
    float acc[N] = {};
    for (int k0 = 0; k0 < top_k; k0 += KU) {
        int row[KU], s[KU];
        float w[KU];
#pragma unroll
        for (int q = 0; q < KU; ++q) {
            row[q] = k0 + q < top_k ? __ldg(&at[k0 + q]) : -1;
            w[q] = weights && k0 + q < top_k ? __ldg(&w_at[k0 + q]) : 1.f;
        }
#pragma unroll
        for (int q = 0; q < KU; ++q)
            if ((unsigned)row[q] < (unsigned)cap_rows) s[q] = y.ask((int64_t)row[q] * ld_y + e, &s_lines[q][0][threadIdx.x]);
        wait_lines();
#pragma unroll
        for (int q = 0; q < KU; ++q) {
            if ((unsigned)row[q] >= (unsigned)cap_rows) continue;
            float x[N];
            y.take(s[q], &s_lines[q][0][threadIdx.x], (int64_t)row[q] * ld_y + e).get(x);
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j] = fmaf(w[q], x[j], acc[j]);
        }
    }
    Vec<T> r;
    r.set(acc);
    store_line(to, e, dim, r);
}

// The gradients: P threads (a power of two) take a choice, so that where its rows lie is found out once for all of their lines: the
// whole lines of grad_y's row, and the values before and behind them, a thread each.  (A token's choices one after the other, which
// need no second load of grad_out's row from the caches, took 40 us where this takes 34: a chain of place, rows, stores for each.  32
// threads a row instead of 8: 42.)  Rows next to a buffer's ends are done value by value.  SAME: y's rows lie in their lines as grad_y's
// do, so that y needs no putting together.
template <typename T, bool SAME>
__global__ void __launch_bounds__(kRowNT, 4) k_expert_combine_bwd_ragged(
    const T* __restrict__ go_, int ld_go, const T* __restrict__ y_, int ld_y, int cap_rows, const int32_t* n_tokens,
    int max_tokens, int top_k, int dim, const int32_t* __restrict__ place, const float* __restrict__ weights,
    T* __restrict__ gy_, int ld_gy, float* __restrict__ grad_w, int P, int row_ctas, int E, int pad_units,
    const int32_t* __restrict__ counts, const int32_t* __restrict__ offsets) {
    constexpr int N = Vec<T>::N, L = 2;              // lines of a thread on their way
    const Rows<T> gy{gy_, ld_gy};
    if ((int)blockIdx.x >= row_ctas) {
        zero_pads<T>(blockIdx.x - row_ctas, pad_units, E, counts, offsets, cap_rows, gy, dim);
        return;
    }
    __shared__ float s_dot[kRowNT / 32];
    const Buffer<T> go(go_, ld_go, max_tokens, dim), y(grad_w ? y_ : gy_, grad_w ? ld_y : ld_gy, cap_rows, dim);
    const int sub = threadIdx.x & (P - 1), a = (int)((int64_t)blockIdx.x * (kRowNT / P)) + (int)threadIdx.x / P, t = a / top_k;
    const bool live = t < live_choices(n_tokens, max_tokens, 1);
    const int row = live ? __ldg(&place[a]) : -1;
    const float w = live && weights ? __ldg(&weights[a]) : 1.f;
    float dot[1] = {};
    if ((unsigned)row < (unsigned)cap_rows) {
        T* to = gy.at(row);
        if (go.inside(t) && y.inside(row)) {
            // whole lines of grad_y's row; then the values before and behind them, a thread each
            const int in = in_line(to), head = min(in ? N - in : 0, dim), lines = (dim - head) / N;
            const int tail = head + lines * N, edges = head + dim - tail;
            const T *x_row = go.p + (int64_t)t * ld_go, *y_row = y.p + (int64_t)row * y.ld;
            const auto edge = [&](int i) { return i < head ? i : tail + i - head; };
            float edge_x = 0.f, edge_y = 0.f;
            if (sub < edges) {
                edge_x = value_of(x_row + edge(sub));
                if (grad_w) edge_y = value_of(y_row + edge(sub));
            }
            const Ragged<T> g(go, t, -head), v(y, row, -head);
            T* first_line = to + head;
            for (int l0 = sub; l0 < lines; l0 += P * L) {
                Lines gl[L], vl[L];
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    if (l0 + i * P >= lines) break;
                    gl[i] = g.ask(l0 + i * P);
                    if (!grad_w) continue;
                    if constexpr (SAME) vl[i].a = __ldg(v.line + l0 + i * P);
                    else vl[i] = v.ask(l0 + i * P);
                }
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    if (l0 + i * P >= lines) break;
                    float x[N], z[N];
                    g.take(gl[i]).get(x);
                    if (grad_w) {
                        Vec<T> b;
                        if constexpr (SAME) b.raw = vl[i].a;
                        else b = v.take(vl[i]);
                        b.get(z);
#pragma unroll
                        for (int j = 0; j < N; ++j) dot[0] = fmaf(x[j], z[j], dot[0]);
                    }
#pragma unroll
                    for (int j = 0; j < N; ++j) z[j] = w * x[j];
                    Vec<T> r;
                    r.set(z);
                    r.store(first_line + (l0 + i * P) * N);
                }
            }
            for (int i = sub; i < edges; i += P) {
                if (i != sub) {
                    edge_x = value_of(x_row + edge(i));
                    if (grad_w) edge_y = value_of(y_row + edge(i));
                }
                dot[0] = fmaf(edge_x, edge_y, dot[0]);
                put_value(to + edge(i), w * edge_x);
            }
        } else {
#pragma unroll 1
            for (int c = sub; c < dim; c += P) {
                const float x = value_of(go.p + (int64_t)t * ld_go + c);
                if (grad_w) dot[0] = fmaf(x, value_of(y.p + (int64_t)row * ld_y + c), dot[0]);
                put_value(to + c, w * x);
            }
        }
    }
    if (!grad_w) return;
    sum_dots(dot, P, s_dot);
    if (sub == 0 && live) grad_w[a] = dot[0];
}

// ---- arguments ------------------------------------------------------------------------------------------------------
bool words(std::initializer_list<const void*> ps) {            // (NULL, too)
    for (const void* p : ps)
        if (reinterpret_cast<uintptr_t>(p) & 3) return false;
    return true;
}
bool route_ok(const hl_route* r) {
    return r && words({r->n_tokens, r->place, r->source, r->counts, r->offsets}) && r->max_tokens >= 0 &&
           r->max_tokens < (int64_t(1) << 30) && r->top_k >= 1 && r->top_k <= HL_MAX_TOP_K && r->n_experts >= 1 &&
           r->n_experts <= HL_MAX_EXPERTS && r->max_tokens * r->top_k < (int64_t(1) << 30) && r->align >= 1 &&
           r->align <= 65536 && r->cap_rows >= 0 && r->cap_rows < (int64_t(1) << 31) - 65536 &&
           (r->place || r->max_tokens == 0);
}
int size_of(int32_t dtype) { return dtype == HL_F32 ? 4 : dtype == HL_BF16 || dtype == HL_F16 ? 2 : 0; }

struct Matrix {
    const void* p;
    int64_t ld, rows;
};
// Whether all of their rows begin at multiples of `bytes` and have whole ones.
bool in_lines(int bytes, int size, int64_t dim, std::initializer_list<Matrix> ms) {
    bool all = dim * size % bytes == 0;
    for (const Matrix& m : ms) all = all && reinterpret_cast<uintptr_t>(m.p) % bytes == 0 && m.ld * size % bytes == 0;
    return all;
}
bool matrices_ok(int32_t dtype, int64_t dim, std::initializer_list<Matrix> ms) {
    const int size = size_of(dtype);
    if (!size || dim < 1 || dim > (int64_t(1) << 24)) return false;
    for (const Matrix& m : ms)
        if ((!m.p && m.rows > 0) || m.ld < dim || m.ld >= (int64_t(1) << 31) || reinterpret_cast<uintptr_t>(m.p) % size)
            return false;
    return true;
}

// Grids are made for a B200's multiprocessors, whatever device is current: the sort's workspace, which holds the tiles' counts, may be
// asked for while another one is.
constexpr int kSMs = 148;

// CTAs per expert for the rows that fill it up: four a multiprocessor in all, or as many as leave each some 128 KB to write where
// half of those rows are there (1 000 CTAs with 300 KB each ran in two rounds: 122 us instead of 98).
int pad_units(const hl_route* r, int64_t row_bytes) {
    if (r->align <= 1 || !r->counts || !r->offsets) return 0;
    const int64_t fill = div_up(4 * kSMs, r->n_experts), work = div_up((r->align - 1) * row_bytes, 256 << 10);
    const int64_t u = fill > work ? fill : work;
    return (int)(u < r->align - 1 ? u : r->align - 1);
}

// Whether the current device can place clusters of 16 CTAs (a non-portable size) of the sort; asked once per device.
template <int ITEMS, int BITS>
bool wide_cluster() {
    auto* kernel = k_expert_sort<16, 512, ITEMS, BITS>;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 16;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(16);
    cfg.blockDim = dim3(512);
    cfg.dynamicSmemBytes = Sort<512, ITEMS>::smem_bytes(HL_MAX_EXPERTS);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
           cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters >= 1;
}
template <int ITEMS>
bool wide_cluster_of() {
    return wide_cluster<ITEMS, 4>() && wide_cluster<ITEMS, 6>() && wide_cluster<ITEMS, 8>() && wide_cluster<ITEMS, 10>();
}
bool wide_clusters() {
    static std::atomic<int> known[64];               // 0: not asked yet, 1: no, 2: yes
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    const int k = known[dev].load(std::memory_order_acquire);
    if (k) return k == 2;
    const bool yes = wide_cluster_of<2>() && wide_cluster_of<4>() && wide_cluster_of<8>() && wide_cluster_of<12>();
    (void)cudaGetLastError();
    known[dev].store(yes ? 2 : 1, std::memory_order_release);
    return yes;
}

// Tiles of at most Tile::kChoices choices: as many CTAs as fill whole rounds of the chip.
int64_t sort_tiles(int64_t n) { return div_up(div_up(n > 0 ? n : 1, Tile::kChoices), kSMs) * kSMs; }

// Threads of a row, a power of two: enough for `each` vectors a thread, few of them without one in the last round, and at most `most`.
// More than a warp's only where there are few rows, or for rows of which each still has seven vectors (gradients of 4 000 choices of
// 16 383 fp32 with 256 threads a row 141 us, with 32 226; of 12 000 of 8 192 bf16 80 and 88; but of 131 072 of 2 050 bf16, two vectors
// each with 128 threads, 418 instead of 272).
int threads_of(int64_t rows, int64_t vectors, int each, int most) {
    int P = 1;
    while (P < most && P * each < vectors) {
        const bool few = rows * P < (int64_t)kSMs * 1024;
        const int64_t round = 2 * P * each, idle = div_up(vectors, round) * round - vectors;
        if (!few && ((P >= 32 && vectors < 14 * P) || 4 * idle > vectors)) break;
        P *= 2;
    }
    return P;
}

template <typename T, typename V>
int32_t launch_dispatch(const hl_route* r, int64_t dim, const void* x, int64_t ld_x, void* y, int64_t ld_y, cudaStream_t stream) {
    const int vectors = (int)(dim * sizeof(T) / sizeof(V)), units = pad_units(r, dim * sizeof(T));
    const int64_t ctas = div_up(r->max_tokens * vectors, kRowNT * kDispatchVectors<V>);
    if (ctas + units == 0) return HL_OK;
    if (ctas + (int64_t)units * r->n_experts > 0x7fffffff) return HL_EINVAL;
    HL_CUDA_TRY(launch(k_expert_dispatch<T, V>, ctas + units * r->n_experts, kRowNT, stream, static_cast<const T*>(x), ld_x,
                       r->n_tokens, r->max_tokens, r->top_k, dim, r->place, r->cap_rows, static_cast<T*>(y), ld_y, vectors,
                       inverse_of(vectors), ctas, r->n_experts, units, r->counts, r->offsets));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

template <typename T>
int32_t launch_combine(const hl_route* r, int64_t dim, const void* y, int64_t ld_y, const float* w, void* out, int64_t ld_out,
                       bool ragged, cudaStream_t stream) {
    const int vectors = (int)div_up(dim + (ragged ? Vec<T>::N - 1 : 0), Vec<T>::N);
    const bool few = !ragged && r->top_k <= 2;
    const int64_t ctas = div_up(r->max_tokens * vectors, kRowNT * (few ? 2 : 1));
    if (ctas > 0x7fffffff) return HL_EINVAL;
    if (ragged) {
        HL_CUDA_TRY(launch(k_expert_combine_ragged<T>, ctas, kRowNT, stream, static_cast<const T*>(y), ld_y, r->cap_rows, r->n_tokens,
                           r->max_tokens, r->top_k, dim, r->place, w, static_cast<T*>(out), ld_out, vectors, inverse_of(vectors)));
    } else {
        HL_CUDA_TRY(launch(few ? k_expert_combine<T, 2, 2> : k_expert_combine<T, 4, 1>, ctas, kRowNT, stream,
                           static_cast<const T*>(y), ld_y, r->cap_rows, r->n_tokens, r->max_tokens, r->top_k, r->place, w,
                           static_cast<T*>(out), ld_out, vectors, inverse_of(vectors)));
    }
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

template <typename T>
int32_t launch_combine_bwd(const hl_route* r, int64_t dim, const void* go, int64_t ld_go, const void* y, int64_t ld_y,
                           const float* w, void* gy, int64_t ld_gy, float* gw, bool ragged, cudaStream_t stream) {
    const int units = pad_units(r, dim * sizeof(T));
    const int64_t vectors = ragged ? dim / Vec<T>::N : div_up(dim, Vec<T>::N);
    const int64_t each = r->max_tokens * (ragged ? r->top_k : 1);        // tokens, or choices
    const int P = threads_of(each, vectors, ragged ? 2 : 1, kRowNT);
    const int64_t ctas = div_up(each, kRowNT / P);
    if (ctas + units == 0) return HL_OK;
    if (ctas + (int64_t)units * r->n_experts > 0x7fffffff) return HL_EINVAL;
    const bool same = ld_y == ld_gy && (reinterpret_cast<uintptr_t>(y) - reinterpret_cast<uintptr_t>(gy)) % 16 == 0;
    const int grid = (int)(ctas + (int64_t)units * r->n_experts);
    const T *go_t = static_cast<const T*>(go), *y_t = static_cast<const T*>(y);
    if (ragged)
        HL_CUDA_TRY(launch(same ? k_expert_combine_bwd_ragged<T, true> : k_expert_combine_bwd_ragged<T, false>, grid, kRowNT, stream,
                           go_t, ld_go, y_t, ld_y, r->cap_rows, r->n_tokens, r->max_tokens, r->top_k, dim, r->place, w,
                           static_cast<T*>(gy), ld_gy, gw, P, ctas, r->n_experts, units, r->counts, r->offsets));
    else
        HL_CUDA_TRY(launch(k_expert_combine_bwd<T>, grid, kRowNT, stream, go_t, ld_go, y_t, ld_y, r->cap_rows, r->n_tokens,
                           r->max_tokens, r->top_k, dim, r->place, w, static_cast<T*>(gy), ld_gy, gw, P, ctas, r->n_experts, units,
                           r->counts, r->offsets));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

}  // namespace
}  // namespace hl

using namespace hl;

extern "C" size_t hl_expert_workspace_bytes(int64_t max_tokens, int32_t top_k, int32_t n_experts) {
    if (max_tokens < 0 || max_tokens >= (int64_t(1) << 30) || top_k < 1 || top_k > HL_MAX_TOP_K || n_experts < 1 ||
        n_experts > HL_MAX_EXPERTS || max_tokens * top_k >= (int64_t(1) << 30))
        return 0;
    const int64_t n = max_tokens * top_k;
    if (n <= 8 * 512 * 2) return 256;
    return (((sort_tiles(n) + 1) * (n_experts + 1) + n) * sizeof(int32_t) + 255) & ~size_t(255);
}

extern "C" int32_t hl_expert_sort(const hl_route* route, const int32_t* d_experts, int64_t expert_cap, int32_t* d_status,
                                  void* d_workspace, size_t ws_bytes, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!route_ok(route) || !route->counts || !route->offsets || (!d_experts && route->max_tokens > 0) || expert_cap < 0 ||
        !words({d_experts, d_status}))
        return HL_EINVAL;
    const int64_t n = route->max_tokens * route->top_k;
    const int E = route->n_experts;
    if (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 255)) return HL_EINVAL;
    if (ws_bytes < hl_expert_workspace_bytes(route->max_tokens, route->top_k, E)) return HL_ECAPACITY;
    const int32_t cap = (int32_t)(expert_cap < (int64_t(1) << 30) ? expert_cap : 0);
    const int bits = E <= 16 ? 0 : E <= 64 ? 1 : E <= 256 ? 2 : 3;
#define HL_BITS(KERNEL, ...)                                                                        \
    (bits == 0 ? KERNEL<__VA_ARGS__ 4> : bits == 1 ? KERNEL<__VA_ARGS__ 6> : bits == 2 ? KERNEL<__VA_ARGS__ 8> \
                                                                                     : KERNEL<__VA_ARGS__ 10>)
    if (n <= 8 * 512 * 2 || (n <= kOneCluster && wide_clusters())) {
#define HL_SORT(CTAS, NT, ITEMS)                                                                                              \
    launch_cluster(HL_BITS(k_expert_sort, CTAS, NT, ITEMS, ), CTAS, NT, (Sort<NT, ITEMS>::smem_bytes(E)), CTAS > 1 ? CTAS : 0, \
                   stream, d_experts, route->n_tokens, route->max_tokens, route->top_k, E, cap, route->align,                  \
                   route->cap_rows, route->place, route->source, route->counts, route->offsets, d_status)
        HL_CUDA_TRY(n <= kFewChoices    ? HL_SORT(1, 128, 4)
                    : n <= 8 * 512 * 2  ? HL_SORT(8, 512, 2)
                    : n <= 16 * 512 * 2 ? HL_SORT(16, 512, 2)
                    : n <= 16 * 512 * 4 ? HL_SORT(16, 512, 4)
                    : n <= 16 * 512 * 8 ? HL_SORT(16, 512, 8)
                                        : HL_SORT(16, 512, 12));
#undef HL_SORT
        note_launches(1);
        HL_LAUNCH_CHECK();
        return HL_OK;
    }
    const int64_t tiles = sort_tiles(n);
    int32_t* totals = static_cast<int32_t*>(d_workspace);
    int32_t* tile_counts = totals + (E + 1);
    uint32_t* ranked = reinterpret_cast<uint32_t*>(tile_counts + tiles * (E + 1));
    HL_CUDA_TRY(launch_cluster(HL_BITS(k_expert_rank, ), tiles, kTileNT, Tile::smem_bytes(E), 0, stream, d_experts, route->n_tokens,
                               route->max_tokens, route->top_k, E, tile_counts, ranked));
    HL_CUDA_TRY(launch_after(k_expert_scan, div_up(E + 1, 32), kScanNT, 0, stream, tile_counts, tiles, E, totals));
    HL_CUDA_TRY(launch_after(k_expert_place, tiles, kTileNT, place_smem_bytes(E), stream, route->n_tokens, route->max_tokens,
                             route->top_k, E, cap, route->align, route->cap_rows, route->place, route->source, route->counts,
                             route->offsets, d_status, (const int32_t*)tile_counts, (const int32_t*)totals,
                             (const uint32_t*)ranked));
    note_launches(3);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

extern "C" int32_t hl_expert_dispatch(const hl_route* route, int32_t dtype, int64_t dim, const void* d_x, int64_t ld_x,
                                      void* d_y, int64_t ld_y, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!route_ok(route)) return HL_EINVAL;
    if (route->align > 1 && (!route->counts || !route->offsets)) return HL_EINVAL;
    const Matrix x{d_x, ld_x, route->max_tokens}, y{d_y, ld_y, route->cap_rows};
    if (!matrices_ok(dtype, dim, {x, y})) return HL_EINVAL;
    if (route->cap_rows == 0) return HL_OK;
    const int size = size_of(dtype);
#define HL_DISPATCH(T, V) launch_dispatch<T, V>(route, dim, d_x, ld_x, d_y, ld_y, stream)
    if (in_lines(16, size, dim, {x, y})) return size == 4 ? HL_DISPATCH(uint32_t, uint4) : HL_DISPATCH(uint16_t, uint4);
    if (in_lines(8, size, dim, {x, y})) return size == 4 ? HL_DISPATCH(uint32_t, uint2) : HL_DISPATCH(uint16_t, uint2);
    if (size == 4) return HL_DISPATCH(uint32_t, uint32_t);
    return in_lines(4, size, dim, {x, y}) ? HL_DISPATCH(uint16_t, uint32_t) : HL_DISPATCH(uint16_t, uint16_t);
#undef HL_DISPATCH
}

#define HL_FOR_TYPE(CALL) \
    return dtype == HL_F32 ? CALL(float) : dtype == HL_BF16 ? CALL(__nv_bfloat16) : CALL(__half)

extern "C" int32_t hl_expert_combine(const hl_route* route, int32_t dtype, int64_t dim, const void* d_y, int64_t ld_y,
                                     const float* d_weights, void* d_out, int64_t ld_out, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!route_ok(route) || !words({d_weights})) return HL_EINVAL;
    const Matrix y{d_y, ld_y, route->cap_rows}, out{d_out, ld_out, route->max_tokens};
    if (!matrices_ok(dtype, dim, {y, out})) return HL_EINVAL;
    if (route->max_tokens == 0) return HL_OK;
    const bool ragged = !in_lines(16, size_of(dtype), dim, {y, out});
#define HL_COMBINE(T) launch_combine<T>(route, dim, d_y, ld_y, d_weights, d_out, ld_out, ragged, stream)
    HL_FOR_TYPE(HL_COMBINE);
#undef HL_COMBINE
}

extern "C" int32_t hl_expert_combine_bwd(const hl_route* route, int32_t dtype, int64_t dim, const void* d_grad_out,
                                         int64_t ld_grad_out, const void* d_y, int64_t ld_y, const float* d_weights,
                                         void* d_grad_y, int64_t ld_grad_y, float* d_grad_weights, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!route_ok(route) || !words({d_weights, d_grad_weights})) return HL_EINVAL;
    if (route->align > 1 && (!route->counts || !route->offsets)) return HL_EINVAL;
    const Matrix go{d_grad_out, ld_grad_out, route->max_tokens}, gy{d_grad_y, ld_grad_y, route->cap_rows};
    const Matrix y{d_grad_weights ? d_y : d_grad_y, d_grad_weights ? ld_y : ld_grad_y, route->cap_rows};   // (else not read)
    if (!matrices_ok(dtype, dim, {go, y, gy})) return HL_EINVAL;
    const bool ragged = !in_lines(16, size_of(dtype), dim, {go, y, gy});
#define HL_COMBINE_BWD(T)                                                                                                      \
    launch_combine_bwd<T>(route, dim, d_grad_out, ld_grad_out, d_y, ld_y, d_weights, d_grad_y, ld_grad_y, d_grad_weights, ragged, \
                          stream)
    HL_FOR_TYPE(HL_COMBINE_BWD);
#undef HL_COMBINE_BWD
}
