// Tokens sorted by expert and back: the routing plan, the copies to the experts' rows, the weighted sums back, and the
// gradients of both.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hl_common.cuh"

namespace cg = cooperative_groups;

namespace hl {
namespace {

// ---- the sort ---------------------------------------------------------------------------------------------------
// A stable counting sort of the choices by expert.  A warp takes kItems * 32 consecutive choices, 32 at a time; the choices
// of one expert among them rank by lane (a match over the warp) behind those the warp has counted before.  Behind that, a
// choice's row is: rows of the experts before + choices of the expert in CTAs before + in warps before + in the warp.
constexpr int kSortNT = 512, kSortWarps = kSortNT / 32, kItems = 16;
constexpr int kSortChoices = kSortNT * kItems;       // of a CTA
constexpr int kExpertsPerThread = HL_MAX_EXPERTS / kSortNT + 1;
static_assert(HL_MAX_EXPERTS <= 2 * kSortNT, "place_experts: two experts a thread");

// what the sort writes, and the words it goes by
struct SortOut {
    int32_t *place, *source, *counts, *offsets, *status;
    int64_t cap_rows;
    int32_t expert_cap, align;
};

__device__ __forceinline__ int live_choices(const int32_t* n_tokens, int max_tokens, int top_k) {
    int t = max_tokens;
    if (n_tokens) t = min(max(*n_tokens, 0), max_tokens);
    return t * top_k;
}

struct SortSmem {
    uint16_t* warp_hist;               // [kSortWarps][E]; then choices of the expert in the warps before
    int32_t* hist;                     // [E + 1] of this CTA, [E]: ids that are no expert's; then of the CTAs before
    int32_t* offset;                   // [E + 1]
    int32_t* count;                    // [E + 1]
};
__host__ __device__ constexpr size_t sort_smem_words(int E) {
    return (size_t)kSortWarps * ((E + 1) / 2) + 3 * (size_t)(E + 1);
}
__device__ __forceinline__ SortSmem sort_smem(uint32_t* base, int E) {
    SortSmem s;
    s.warp_hist = reinterpret_cast<uint16_t*>(base);
    s.hist = reinterpret_cast<int32_t*>(base + kSortWarps * ((E + 1) / 2));
    s.offset = s.hist + E + 1;
    s.count = s.offset + E + 1;
    return s;
}
__device__ __forceinline__ int hist_pitch(int E) { return 2 * ((E + 1) / 2); }

// Ranks the CTA's choices [first, first + kSortChoices) below n.  packed[i]: expert (16 bits; 0xffff: none), rank in the warp.
__device__ __forceinline__ void rank_choices(const SortSmem& s, const int32_t* __restrict__ experts, int64_t first, int64_t n,
                                             int E, uint32_t packed[kItems]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pitch = hist_pitch(E);
    for (int i = threadIdx.x; i < kSortWarps * pitch / 2; i += kSortNT) reinterpret_cast<uint32_t*>(s.warp_hist)[i] = 0;
    if (threadIdx.x == 0) s.hist[E] = 0;
    const int64_t seg = first + warp * (kItems * 32) + lane;
    int e[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) e[i] = seg + i * 32 < n ? __ldg(&experts[seg + i * 32]) : -1;
    __syncthreads();
    uint16_t* h = s.warp_hist + warp * pitch;
    int bad = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const bool ok = e[i] >= 0 && e[i] < E;
        bad += !ok && e[i] != -1;
        packed[i] = 0xffff0000u;
        if (first + warp * (kItems * 32) + i * 32 >= n) continue;            // (the same for the warp)
        const unsigned peers = __match_any_sync(0xffffffffu, ok ? e[i] : -1);
        if (ok) {
            const unsigned mine = __popc(peers & lanemask_lt());
            const unsigned base = h[e[i]];
            packed[i] = ((uint32_t)e[i] << 16) | (base + mine);
        }
        __syncwarp();
        if (ok && (peers & lanemask_lt()) == 0) h[e[i]] = (uint16_t)((packed[i] & 0xffffu) + __popc(peers));
        __syncwarp();
    }
    if (__any_sync(0xffffffffu, bad != 0) && lane == 0) atomicAdd(&s.hist[E], 1);
    __syncthreads();
    for (int x = threadIdx.x; x < E; x += kSortNT) {
        int sum = 0;
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = s.warp_hist[w * pitch + x];
            s.warp_hist[w * pitch + x] = (uint16_t)sum;
            sum += c;
        }
        s.hist[x] = sum;
    }
    __syncthreads();
}

// s.count holds every expert's choices: turns them into the rows it gets and their offsets, both inside cap_rows.
// *over: rows that did not fit.
__device__ __forceinline__ void place_experts(const SortSmem& s, int E, const SortOut& o, bool* over) {
    __shared__ int64_t s_warp[kSortWarps];
    __shared__ int s_over;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) s_over = 0;
    int64_t rows[2], sum = 0;
    int cnt[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {      // two neighbouring experts a thread
        const int e = 2 * threadIdx.x + k;
        cnt[k] = e < E ? s.count[e] : 0;
        if (o.expert_cap > 0) cnt[k] = min(cnt[k], o.expert_cap);
        rows[k] = ((int64_t)cnt[k] + o.align - 1) / o.align * o.align;
        sum += rows[k];
    }
    int64_t incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += v;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int64_t at = incl - sum;
    for (int w = 0; w < warp; ++w) at += s_warp[w];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int e = 2 * threadIdx.x + k;
        if (e < E) {
            if (at + cnt[k] > o.cap_rows) s_over = 1;
            s.offset[e] = (int32_t)min(at, o.cap_rows);
            s.count[e] = (int32_t)min((int64_t)cnt[k], max(o.cap_rows - at, (int64_t)0));
            if (e == E - 1) s.offset[E] = (int32_t)min(at + rows[k], o.cap_rows);
        }
        at += rows[k];
    }
    __syncthreads();
    *over = s_over != 0;
}

__device__ __forceinline__ void write_places(const SortSmem& s, const SortOut& o, int64_t first, int64_t n, int E,
                                             const uint32_t packed[kItems]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pitch = hist_pitch(E);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int64_t a = first + warp * (kItems * 32) + i * 32 + lane;
        if (a >= n) continue;
        const uint32_t e = packed[i] >> 16;
        int32_t row = -1;
        if (e != 0xffffu) {
            const int r = s.hist[e] + s.warp_hist[warp * pitch + e] + (int)(packed[i] & 0xffffu);
            if (r < s.count[e]) row = s.offset[e] + r;
        }
        o.place[a] = row;
        if (row >= 0 && o.source) o.source[row] = (int32_t)a;
    }
}

// The rows that fill an expert up, and the plan's words, by CTA `cta` of `ctas`.
__device__ __forceinline__ void write_plan(const SortSmem& s, const SortOut& o, int E, int cta, int ctas, bool over, bool bad) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (o.source && o.align > 1)
        for (int e = cta * kSortWarps + warp; e < E; e += ctas * kSortWarps)
            for (int r = s.offset[e] + s.count[e] + lane; r < s.offset[e + 1]; r += 32) o.source[r] = -1;
    if (cta != 0) return;
    for (int e = threadIdx.x; e < E; e += kSortNT) {
        o.counts[e] = s.count[e];
        o.offsets[e] = s.offset[e];
    }
    if (threadIdx.x == 0) {
        o.offsets[E] = s.offset[E];
        if (o.status) *o.status = bad ? HL_EBOUNDS : over ? HL_ECAPACITY : HL_OK;
    }
}

// All of it in one cluster, whose CTAs read each other's counts.
template <int CTAS>
__global__ void __launch_bounds__(kSortNT) k_expert_sort(const int32_t* __restrict__ experts, const int32_t* n_tokens,
                                                         int max_tokens, int top_k, int E, int expert_cap, int align,
                                                         int64_t cap_rows, int32_t* place, int32_t* source, int32_t* counts,
                                                         int32_t* offsets, int32_t* status) {
    extern __shared__ uint32_t s_base[];
    const SortSmem s = sort_smem(s_base, E);
    const SortOut o{place, source, counts, offsets, status, cap_rows, expert_cap, align};
    const int64_t n = live_choices(n_tokens, max_tokens, top_k), first = (int64_t)blockIdx.x * kSortChoices;
    uint32_t packed[kItems];
    rank_choices(s, experts, first, n, E, packed);
    int bad = 0;
    if constexpr (CTAS > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        int before[kExpertsPerThread] = {};
#pragma unroll
        for (int k = 0; k < kExpertsPerThread; ++k) {
            const int e = threadIdx.x + k * kSortNT;
            if (e > E) break;
            int all = 0;
#pragma unroll
            for (int c = 0; c < CTAS; ++c) {
                const int v = *cluster.map_shared_rank(&s.hist[e], c);
                if (c < (int)blockIdx.x) before[k] += v;
                all += v;
            }
            s.count[e] = all;
        }
        cluster.sync();                // (nobody reads this CTA's counts any more)
#pragma unroll
        for (int k = 0; k < kExpertsPerThread; ++k) {
            const int e = threadIdx.x + k * kSortNT;
            if (e <= E) s.hist[e] = before[k];
        }
    } else {
        for (int e = threadIdx.x; e <= E; e += kSortNT) {
            s.count[e] = s.hist[e];
            s.hist[e] = 0;
        }
    }
    __syncthreads();
    bad = s.count[E];
    bool over;
    place_experts(s, E, o, &over);
    write_places(s, o, first, n, E, packed);
    write_plan(s, o, E, blockIdx.x, CTAS, over, bad != 0);
}

// In three kernels: every tile's counts, sums of them over the tiles before, places.
__global__ void __launch_bounds__(kSortNT) k_expert_count(const int32_t* __restrict__ experts, const int32_t* n_tokens,
                                                          int max_tokens, int top_k, int E, int32_t* __restrict__ tile_counts) {
    extern __shared__ uint32_t s_base[];
    const SortSmem s = sort_smem(s_base, E);
    const int64_t n = live_choices(n_tokens, max_tokens, top_k), first = (int64_t)blockIdx.x * kSortChoices;
    uint32_t packed[kItems];
    rank_choices(s, experts, first, n, E, packed);
    for (int e = threadIdx.x; e <= E; e += kSortNT) tile_counts[(int64_t)blockIdx.x * (E + 1) + e] = s.hist[e];
}

// tile_counts[t][e] := sum over the tiles before t; totals[e].  A CTA takes 32 experts, its warps a run of tiles each.
__global__ void __launch_bounds__(1024) k_expert_scan(int32_t* __restrict__ tile_counts, int64_t n_tiles, int E,
                                                      int32_t* __restrict__ totals) {
    __shared__ int32_t s_sum[32][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    const int64_t per = (n_tiles + 31) / 32, t0 = warp * per, t1 = min(t0 + per, n_tiles);
    int sum = 0;
    if (e <= E)
        for (int64_t t = t0; t < t1; ++t) sum += tile_counts[t * (E + 1) + e];
    s_sum[warp][lane] = sum;
    __syncthreads();
    if (e > E) return;
    int before = 0;
    for (int w = 0; w < warp; ++w) before += s_sum[w][lane];
    for (int64_t t = t0; t < t1; ++t) {
        const int c = tile_counts[t * (E + 1) + e];
        tile_counts[t * (E + 1) + e] = before;
        before += c;
    }
    if (warp == 31) totals[e] = before;
}

__global__ void __launch_bounds__(kSortNT) k_expert_place(const int32_t* __restrict__ experts, const int32_t* n_tokens,
                                                          int max_tokens, int top_k, int E, int expert_cap, int align,
                                                          int64_t cap_rows, int32_t* place, int32_t* source, int32_t* counts,
                                                          int32_t* offsets, int32_t* status,
                                                          const int32_t* __restrict__ tile_counts,
                                                          const int32_t* __restrict__ totals) {
    extern __shared__ uint32_t s_base[];
    const SortSmem s = sort_smem(s_base, E);
    const SortOut o{place, source, counts, offsets, status, cap_rows, expert_cap, align};
    const int64_t n = live_choices(n_tokens, max_tokens, top_k), first = (int64_t)blockIdx.x * kSortChoices;
    uint32_t packed[kItems];
    rank_choices(s, experts, first, n, E, packed);
    for (int e = threadIdx.x; e <= E; e += kSortNT) {
        s.hist[e] = tile_counts[(int64_t)blockIdx.x * (E + 1) + e];
        s.count[e] = totals[e];
    }
    __syncthreads();
    const bool bad = s.count[E] != 0;
    bool over;
    place_experts(s, E, o, &over);
    write_places(s, o, first, n, E, packed);
    write_plan(s, o, E, blockIdx.x, gridDim.x, over, bad);
}

constexpr int kClusterCtas = 8;
constexpr int64_t kOneCluster = (int64_t)kClusterCtas * kSortChoices;

// ---- rows -----------------------------------------------------------------------------------------------------------
// N values of type T, moved as one.
template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
    T v[N];
};
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

constexpr int kRowNT = 256, kRowWarps = kRowNT / 32;

// Rows that fill experts up: CTA u of n_units x E takes every n_units-th of expert u % E's.
template <typename V>
__device__ __forceinline__ void zero_pads(int u, int units, int E, const int32_t* __restrict__ counts,
                                          const int32_t* __restrict__ offsets, int64_t cap_rows, V* y, int64_t ld, int nv) {
    const int e = u % E, part = u / E;
    const int64_t begin = (int64_t)__ldg(&offsets[e]) + __ldg(&counts[e]), end = min((int64_t)__ldg(&offsets[e + 1]), cap_rows);
    if (__ldg(&offsets[e]) < 0 || __ldg(&counts[e]) < 0) return;
    for (int64_t r = begin + part; r < end; r += units)
        for (int c = threadIdx.x; c < nv; c += kRowNT) y[r * ld + c] = V{};
}

// y[place[t, k]] = x[t].  A warp takes 32 * U vectors of a token's row at a time: it reads them once and writes them to the
// token's rows, so that every row crosses memory once.
template <typename V, int U>
__global__ void __launch_bounds__(kRowNT) k_expert_dispatch(const V* __restrict__ x, int64_t ld_x,
                                                            const int32_t* n_tokens, int max_tokens, int top_k, int nv,
                                                            const int32_t* __restrict__ place, int64_t cap_rows,
                                                            V* __restrict__ y, int64_t ld_y, int row_ctas, int E,
                                                            int pad_units, const int32_t* __restrict__ counts,
                                                            const int32_t* __restrict__ offsets) {
    if ((int)blockIdx.x >= row_ctas) {
        zero_pads(blockIdx.x - row_ctas, pad_units, E, counts, offsets, cap_rows, y, ld_y, nv);
        return;
    }
    const int lane = threadIdx.x & 31;
    const int tokens = live_choices(n_tokens, max_tokens, 1), blocks = (nv + 32 * U - 1) / (32 * U);
    const int64_t items = (int64_t)tokens * blocks;
    for (int64_t i = (int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5); i < items; i += (int64_t)row_ctas * kRowWarps) {
        const int64_t t = i / blocks;
        const int c0 = (int)(i - t * blocks) * 32 * U + lane;
        V v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c0 + u * 32 < nv) v[u] = x[t * ld_x + c0 + u * 32];
        for (int k = 0; k < top_k; ++k) {
            const int64_t row = __ldg(&place[t * top_k + k]);
            if (row < 0 || row >= cap_rows) continue;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c0 + u * 32 < nv) y[row * ld_y + c0 + u * 32] = v[u];
        }
    }
}

// out[t] = sum over k of w[t, k] * y[place[t, k]], in fp32, in the order of k, rounded once.  (Without weights: the sum.)
template <typename T, int N, int U>
__global__ void __launch_bounds__(kRowNT) k_expert_combine(const Vec<T, N>* __restrict__ y, int64_t ld_y, int64_t cap_rows,
                                                           const int32_t* n_tokens, int max_tokens, int top_k, int nv,
                                                           const int32_t* __restrict__ place,
                                                           const float* __restrict__ weights, Vec<T, N>* __restrict__ out,
                                                           int64_t ld_out) {
    const int lane = threadIdx.x & 31;
    const int tokens = live_choices(n_tokens, max_tokens, 1), blocks = (nv + 32 * U - 1) / (32 * U);
    const int64_t items = (int64_t)tokens * blocks;
    for (int64_t i = (int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5); i < items; i += (int64_t)gridDim.x * kRowWarps) {
        const int64_t t = i / blocks;
        const int c0 = (int)(i - t * blocks) * 32 * U + lane;
        float acc[U][N] = {};
        for (int k = 0; k < top_k; ++k) {
            const int64_t row = __ldg(&place[t * top_k + k]);
            if (row < 0 || row >= cap_rows) continue;
            const float w = weights ? __ldg(&weights[t * top_k + k]) : 1.f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (c0 + u * 32 >= nv) continue;
                const Vec<T, N> v = y[row * ld_y + c0 + u * 32];
#pragma unroll
                for (int j = 0; j < N; ++j) acc[u][j] = fmaf(w, to_f32(v.v[j]), acc[u][j]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u * 32 >= nv) continue;
            Vec<T, N> v;
#pragma unroll
            for (int j = 0; j < N; ++j) v.v[j] = from_f32<T>(acc[u][j]);
            out[t * ld_out + c0 + u * 32] = v;
        }
    }
}

// grad_y[place[t, k]] = w[t, k] * grad_out[t]; grad_w[t, k] = <grad_out[t], y[place[t, k]]>.  W warps of a CTA take a token:
// 32 * U vectors each at a time, which stay in registers for all of the token's rows.
template <typename T, int N, int U>
__global__ void __launch_bounds__(kRowNT) k_expert_combine_bwd(
    const Vec<T, N>* __restrict__ grad_out, int64_t ld_go, const Vec<T, N>* __restrict__ y, int64_t ld_y, int64_t cap_rows,
    const int32_t* n_tokens, int max_tokens, int top_k, int nv, const int32_t* __restrict__ place,
    const float* __restrict__ weights, Vec<T, N>* __restrict__ grad_y, int64_t ld_gy, float* __restrict__ grad_w, int W,
    int row_ctas, int E, int pad_units, const int32_t* __restrict__ counts, const int32_t* __restrict__ offsets) {
    if ((int)blockIdx.x >= row_ctas) {
        zero_pads(blockIdx.x - row_ctas, pad_units, E, counts, offsets, cap_rows, grad_y, ld_gy, nv);
        return;
    }
    __shared__ float s_dot[kRowWarps][HL_MAX_TOP_K];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % W, per_cta = kRowWarps / W;
    const int tokens = live_choices(n_tokens, max_tokens, 1);
    for (int64_t t0 = (int64_t)blockIdx.x * per_cta; t0 < tokens; t0 += (int64_t)row_ctas * per_cta) {
        const int64_t t = t0 + warp / W;
        if (t < tokens) {
            if (grad_w)
                for (int k = lane; k < top_k; k += 32) s_dot[warp][k] = 0.f;
            __syncwarp();
            for (int c0 = part * 32 * U + lane; c0 - lane < nv; c0 += W * 32 * U) {
                Vec<T, N> g[U];
#pragma unroll
                for (int u = 0; u < U; ++u) g[u] = c0 + u * 32 < nv ? grad_out[t * ld_go + c0 + u * 32] : Vec<T, N>{};
                for (int k = 0; k < top_k; ++k) {
                    const int64_t row = __ldg(&place[t * top_k + k]);
                    if (row < 0 || row >= cap_rows) continue;
                    const float w = weights ? __ldg(&weights[t * top_k + k]) : 1.f;
                    float dot = 0.f;
                    if (grad_w) {
                        Vec<T, N> v[U];
#pragma unroll
                        for (int u = 0; u < U; ++u) v[u] = c0 + u * 32 < nv ? y[row * ld_y + c0 + u * 32] : Vec<T, N>{};
#pragma unroll
                        for (int u = 0; u < U; ++u)
#pragma unroll
                            for (int j = 0; j < N; ++j) dot = fmaf(to_f32(g[u].v[j]), to_f32(v[u].v[j]), dot);
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (c0 + u * 32 >= nv) continue;
                        Vec<T, N> r;
#pragma unroll
                        for (int j = 0; j < N; ++j) r.v[j] = from_f32<T>(w * to_f32(g[u].v[j]));
                        grad_y[row * ld_gy + c0 + u * 32] = r;
                    }
                    if (grad_w) {
#pragma unroll
                        for (int d = 16; d > 0; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
                        if (lane == 0) s_dot[warp][k] += dot;
                    }
                }
            }
        }
        if (!grad_w) continue;
        __syncthreads();
        for (int i = threadIdx.x; i < per_cta * top_k; i += kRowNT) {
            const int j = i / top_k, k = i - j * top_k;
            if (t0 + j >= tokens) continue;
            float dot = 0.f;
            for (int p = 0; p < W; ++p) dot += s_dot[j * W + p][k];
            grad_w[(t0 + j) * top_k + k] = dot;
        }
        __syncthreads();
    }
}

// ---- arguments ------------------------------------------------------------------------------------------------------
bool route_ok(const hl_route* r) {
    return r && r->max_tokens >= 0 && r->max_tokens < (int64_t(1) << 30) && r->top_k >= 1 && r->top_k <= HL_MAX_TOP_K && r->n_experts >= 1 &&
           r->n_experts <= HL_MAX_EXPERTS && r->max_tokens * r->top_k < (int64_t(1) << 30) && r->align >= 1 &&
           r->align <= 65536 && r->cap_rows >= 0 && r->cap_rows < (int64_t(1) << 31) - 65536 &&
           (r->place || r->max_tokens == 0);
}
int size_of(int32_t dtype) { return dtype == HL_F32 ? 4 : dtype == HL_BF16 || dtype == HL_F16 ? 2 : 0; }

struct Matrix {
    const void* p;
    int64_t ld, rows;
};
// Whether all of them can be read and written `bytes` at a time.
bool aligned_to(int bytes, int size, int64_t dim, std::initializer_list<Matrix> ms) {
    if (dim * size % bytes) return false;
    for (const Matrix& m : ms)
        if (m.p && (reinterpret_cast<uintptr_t>(m.p) % bytes || m.ld * size % bytes)) return false;
    return true;
}
bool matrices_ok(int32_t dtype, int64_t dim, std::initializer_list<Matrix> ms) {
    const int size = size_of(dtype);
    if (!size || dim < 1 || dim > (int64_t(1) << 24)) return false;
    for (const Matrix& m : ms)
        if ((!m.p && m.rows > 0) || m.ld < dim || m.ld > (int64_t(1) << 31) || reinterpret_cast<uintptr_t>(m.p) % size)
            return false;
    return true;
}

int sms() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return kSMsFallback;
    return n;
}
int pad_units(const hl_route* r) {
    if (r->align <= 1 || !r->counts || !r->offsets) return 0;
    const int64_t u = div_up(4 * kSMsFallback, r->n_experts);
    return (int)(u < r->align - 1 ? u : r->align - 1);
}

template <typename V, int U>
int32_t launch_dispatch(const hl_route* r, int64_t dim, const void* x, int64_t ld_x, void* y, int64_t ld_y, int size,
                        cudaStream_t stream) {
    const int per = sizeof(V) / size, nv = (int)(dim / per), units = pad_units(r);
    const int ctas = r->max_tokens ? grid_for(r->max_tokens * div_up(nv, 32 * U), kRowWarps, 1 << 20) : 0;
    if (ctas + units == 0) return HL_OK;
    HL_CUDA_TRY(launch(k_expert_dispatch<V, U>, ctas + units * r->n_experts, kRowNT, stream, static_cast<const V*>(x), ld_x / per,
                       r->n_tokens, r->max_tokens, r->top_k, nv, r->place, r->cap_rows, static_cast<V*>(y), ld_y / per, ctas,
                       r->n_experts, units, r->counts, r->offsets));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

template <typename T, int N, int U>
int32_t launch_combine(const hl_route* r, int64_t dim, const void* y, int64_t ld_y, const float* w, void* out, int64_t ld_out,
                       cudaStream_t stream) {
    using V = Vec<T, N>;
    const int nv = (int)(dim / N);
    HL_CUDA_TRY(launch(k_expert_combine<T, N, U>, grid_for(r->max_tokens * div_up(nv, 32 * U), kRowWarps, 1 << 20), kRowNT,
                       stream, static_cast<const V*>(y), ld_y / N, r->cap_rows, r->n_tokens, r->max_tokens, r->top_k, nv,
                       r->place, w, static_cast<V*>(out), ld_out / N));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

template <typename T, int N, int U>
int32_t launch_combine_bwd(const hl_route* r, int64_t dim, const void* go, int64_t ld_go, const void* y, int64_t ld_y,
                           const float* w, void* gy, int64_t ld_gy, float* gw, cudaStream_t stream) {
    using V = Vec<T, N>;
    const int nv = (int)(dim / N), units = pad_units(r);
    int W = 1;
    while (W < kRowWarps && W * 32 * U < nv) W *= 2;
    const int ctas = r->max_tokens ? grid_for(r->max_tokens, kRowWarps / W, 1 << 20) : 0;
    if (ctas + units == 0) return HL_OK;
    HL_CUDA_TRY(launch(k_expert_combine_bwd<T, N, U>, ctas + units * r->n_experts, kRowNT, stream, static_cast<const V*>(go),
                       ld_go / N, static_cast<const V*>(y), ld_y / N, r->cap_rows, r->n_tokens, r->max_tokens, r->top_k, nv,
                       r->place, w, static_cast<V*>(gy), ld_gy / N, gw, W, ctas, r->n_experts, units, r->counts, r->offsets));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

int64_t sort_tiles(int64_t n) { return div_up(n > 0 ? n : 1, kSortChoices); }

}  // namespace
}  // namespace hl

using namespace hl;

extern "C" size_t hl_expert_workspace_bytes(int64_t max_tokens, int32_t top_k, int32_t n_experts) {
    if (max_tokens < 0 || max_tokens >= (int64_t(1) << 30) || top_k < 1 || top_k > HL_MAX_TOP_K || n_experts < 1 || n_experts > HL_MAX_EXPERTS ||
        max_tokens * top_k >= (int64_t(1) << 30))
        return 0;
    return ((sort_tiles(max_tokens * top_k) + 1) * (n_experts + 1) * sizeof(int32_t) + 255) & ~size_t(255);
}

extern "C" int32_t hl_expert_sort(const hl_route* route, const int32_t* d_experts, int64_t expert_cap, int32_t* d_status,
                                  void* d_workspace, size_t ws_bytes, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!route_ok(route) || !route->counts || !route->offsets || (!d_experts && route->max_tokens > 0) || expert_cap < 0)
        return HL_EINVAL;
    const int64_t n = route->max_tokens * route->top_k;
    const int E = route->n_experts;
    if (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 255)) return HL_EINVAL;
    if (ws_bytes < hl_expert_workspace_bytes(route->max_tokens, route->top_k, E)) return HL_ECAPACITY;
    const int32_t cap = (int32_t)(expert_cap < (int64_t(1) << 30) ? expert_cap : 0);
    const size_t smem = sort_smem_words(E) * 4;
    if (n <= kOneCluster) {
        const bool one = n <= kSortChoices;
        HL_CUDA_TRY(launch_cluster(one ? k_expert_sort<1> : k_expert_sort<kClusterCtas>, one ? 1 : kClusterCtas, kSortNT, smem,
                                   one ? 0 : kClusterCtas, stream, d_experts, route->n_tokens, route->max_tokens, route->top_k,
                                   E, cap, route->align, route->cap_rows, route->place, route->source, route->counts,
                                   route->offsets, d_status));
        note_launches(1);
        HL_LAUNCH_CHECK();
        return HL_OK;
    }
    const int64_t tiles = sort_tiles(n);
    int32_t* totals = static_cast<int32_t*>(d_workspace);
    int32_t* tile_counts = totals + (E + 1);
    HL_CUDA_TRY(launch_cluster(k_expert_count, tiles, kSortNT, smem, 0, stream, d_experts, route->n_tokens, route->max_tokens,
                               route->top_k, E, tile_counts));
    HL_CUDA_TRY(launch(k_expert_scan, div_up(E + 1, 32), 1024, stream, tile_counts, tiles, E, totals));
    HL_CUDA_TRY(launch_cluster(k_expert_place, tiles, kSortNT, smem, 0, stream, d_experts, route->n_tokens, route->max_tokens,
                               route->top_k, E, cap, route->align, route->cap_rows, route->place, route->source, route->counts,
                               route->offsets, d_status, (const int32_t*)tile_counts, (const int32_t*)totals));
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
#define HL_DISPATCH(V, U) launch_dispatch<V, U>(route, dim, d_x, ld_x, d_y, ld_y, size, stream)
    if (aligned_to(16, size, dim, {x, y})) return HL_DISPATCH(uint4, 4);
    if (aligned_to(8, size, dim, {x, y})) return HL_DISPATCH(uint2, 4);
    if (aligned_to(4, size, dim, {x, y})) return HL_DISPATCH(uint32_t, 8);
    return HL_DISPATCH(uint16_t, 8);
#undef HL_DISPATCH
}

#define HL_FOR_TYPE(CALL)                                                                        \
    do {                                                                                         \
        if (dtype == HL_F32) return wide ? CALL(float, 4, 4) : CALL(float, 1, 8);                \
        if (dtype == HL_BF16) return wide ? CALL(__nv_bfloat16, 8, 4) : CALL(__nv_bfloat16, 1, 8); \
        return wide ? CALL(__half, 8, 4) : CALL(__half, 1, 8);                                   \
    } while (0)

extern "C" int32_t hl_expert_combine(const hl_route* route, int32_t dtype, int64_t dim, const void* d_y, int64_t ld_y,
                                     const float* d_weights, void* d_out, int64_t ld_out, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!route_ok(route)) return HL_EINVAL;
    const Matrix y{d_y, ld_y, route->cap_rows}, out{d_out, ld_out, route->max_tokens};
    if (!matrices_ok(dtype, dim, {y, out})) return HL_EINVAL;
    if (route->max_tokens == 0) return HL_OK;
    const bool wide = aligned_to(16, size_of(dtype), dim, {y, out});
#define HL_COMBINE(T, N, U) launch_combine<T, N, U>(route, dim, d_y, ld_y, d_weights, d_out, ld_out, stream)
    HL_FOR_TYPE(HL_COMBINE);
#undef HL_COMBINE
}

extern "C" int32_t hl_expert_combine_bwd(const hl_route* route, int32_t dtype, int64_t dim, const void* d_grad_out,
                                         int64_t ld_grad_out, const void* d_y, int64_t ld_y, const float* d_weights,
                                         void* d_grad_y, int64_t ld_grad_y, float* d_grad_weights, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!route_ok(route)) return HL_EINVAL;
    if (route->align > 1 && (!route->counts || !route->offsets)) return HL_EINVAL;
    const Matrix go{d_grad_out, ld_grad_out, route->max_tokens}, gy{d_grad_y, ld_grad_y, route->cap_rows};
    const Matrix y{d_grad_weights ? d_y : d_grad_y, d_grad_weights ? ld_y : ld_grad_y, route->cap_rows};   // (else not read)
    if (!matrices_ok(dtype, dim, {go, y, gy})) return HL_EINVAL;
    const bool wide = aligned_to(16, size_of(dtype), dim, {go, y, gy});
#define HL_COMBINE_BWD(T, N, U) \
    launch_combine_bwd<T, N, U>(route, dim, d_grad_out, ld_grad_out, d_y, ld_y, d_weights, d_grad_y, ld_grad_y, d_grad_weights, stream)
    HL_FOR_TYPE(HL_COMBINE_BWD);
#undef HL_COMBINE_BWD
}
