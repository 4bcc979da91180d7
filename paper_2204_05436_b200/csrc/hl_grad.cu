// The global norm of gradients and clipping: sums of squares over many tensors, the squared norm of an embedding's row
// gradients, and the tensors scaled.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <string.h>

#include "hl_common.cuh"

namespace hl {
namespace {

constexpr int kNT = 256, kWarps = kNT / 32;

__device__ __forceinline__ double block_sum(double v) {        // the same in every thread
    __shared__ double s[kWarps];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum += s[w];
    return sum;
}

// ---- many tensors ---------------------------------------------------------------------------------------------------
// A call's tensors are cut into tiles of kTile values, which are dealt out to the CTAs in turn.
constexpr int kTile = 8192;
constexpr int kGradCtas = 8;                         // CTAs per multiprocessor
constexpr int kMaxPartials = 2048;                   // sums of squares, one per CTA

// N tensors and where their tiles begin, as a kernel argument.
template <int N>
struct TensorPairArgs {
    const void* src[N];
    void* dst[N];
    int64_t n[N];
    int32_t first_tile[N];
    uint8_t kind[N];                                 // type of src, type of dst
    int32_t n_tensors, n_tiles;
};

template <typename T>
struct Wide {
    static constexpr int N = 16 / sizeof(T);
    union {
        uint4 raw;
        T v[N];
    };
    __device__ Wide() {}
};
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
__device__ __forceinline__ void put(__half* p, float x) { *p = __float2half_rn(x); }

// values before p's next multiple of 16 bytes
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int n) {
    const int h = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T);
    return h < n ? h : n;
}

template <typename T>
__device__ __forceinline__ double tile_squares(const T* __restrict__ p, int n) {
    double sum = 0.0;
    const int head = head_of(p, n), nv = (n - head) / Wide<T>::N, tail = head + nv * Wide<T>::N;
    const uint4* q = reinterpret_cast<const uint4*>(p + head);
    for (int i = threadIdx.x; i < nv; i += kNT) {
        Wide<T> w;
        w.raw = __ldg(&q[i]);
#pragma unroll
        for (int j = 0; j < Wide<T>::N; ++j) {
            const double x = to_f32(w.v[j]);
            sum = fma(x, x, sum);
        }
    }
    for (int i = threadIdx.x; i < head + n - tail; i += kNT) {
        const double x = to_f32(p[i < head ? i : tail + i - head]);
        sum = fma(x, x, sum);
    }
    return sum;
}

template <typename S, typename D>
__device__ __forceinline__ void tile_scale(const S* p, D* d, int n, float f) {
    constexpr int N = Wide<S>::N;
    const int head = head_of(p, n), nv = (n - head) / N, tail = head + nv * N;
    const uint4* q = reinterpret_cast<const uint4*>(p + head);
    const bool wide = (reinterpret_cast<uintptr_t>(d + head) & (N * sizeof(D) < 16 ? N * sizeof(D) - 1 : 15)) == 0;
    for (int i = threadIdx.x; i < nv; i += kNT) {
        Wide<S> w;
        w.raw = q[i];
        alignas(16) D r[N];
#pragma unroll
        for (int j = 0; j < N; ++j) put(&r[j], f * to_f32(w.v[j]));
        D* to = d + head + i * N;
        if (!wide) {
#pragma unroll
            for (int j = 0; j < N; ++j) to[j] = r[j];
        } else if constexpr (N * sizeof(D) == 8) {
            *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(r);
        } else {
#pragma unroll
            for (int j = 0; j < (int)(N * sizeof(D) / 16); ++j)
                reinterpret_cast<uint4*>(to)[j] = reinterpret_cast<const uint4*>(r)[j];
        }
    }
    for (int i = threadIdx.x; i < head + n - tail; i += kNT) {
        const int at = i < head ? i : tail + i - head;
        put(&d[at], f * to_f32(p[at]));
    }
}

// The tensor that a tile belongs to: the last one whose tiles begin at it or before.
template <int N>
__device__ __forceinline__ int tensor_of(const TensorPairArgs<N>& a, int tile) {
    int lo = 0, hi = a.n_tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.first_tile[mid] <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

// partial[b] (+)= the squares of CTA b's tiles
template <int N>
__global__ void __launch_bounds__(kNT) k_grad_squares(const __grid_constant__ TensorPairArgs<N> a, int more,
                                                      double* __restrict__ partial) {
    double sum = 0.0;
    for (int tile = blockIdx.x; tile < a.n_tiles; tile += gridDim.x) {
        const int t = tensor_of(a, tile);
        const int kind = a.kind[t];
        const int64_t at = (int64_t)(tile - a.first_tile[t]) * kTile;
        const int n = (int)min((int64_t)kTile, a.n[t] - at);
        if ((kind & 3) == HL_F32) sum += tile_squares(static_cast<const float*>(a.src[t]) + at, n);
        else if ((kind & 3) == HL_BF16) sum += tile_squares(static_cast<const __nv_bfloat16*>(a.src[t]) + at, n);
        else sum += tile_squares(static_cast<const __half*>(a.src[t]) + at, n);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = more ? partial[blockIdx.x] + sum : sum;
}

__device__ __forceinline__ double total_squares(const double* __restrict__ partial, int n_partials,
                                                const double* __restrict__ further, int n_further) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n_partials; i += kNT) sum += partial[i];
    for (int i = threadIdx.x; i < n_further; i += kNT) sum += further[i];
    return block_sum(sum);
}

__global__ void __launch_bounds__(kNT) k_grad_norm(const double* __restrict__ partial, int n_partials,
                                                   const double* __restrict__ further, int n_further, float* norm) {
    const double sum = total_squares(partial, n_partials, further, n_further);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

template <int N>
__global__ void __launch_bounds__(kNT) k_grad_scale(const __grid_constant__ TensorPairArgs<N> a,
                                                    const double* __restrict__ partial, int n_partials,
                                                    const double* __restrict__ further, int n_further, float max_norm,
                                                    float* norm) {
    const double total = sqrt(total_squares(partial, n_partials, further, n_further));
    if (blockIdx.x == 0 && threadIdx.x == 0 && norm) *norm = (float)total;
    const double c = (double)max_norm / (total + 1e-6);
    const float f = c > 1.0 ? 1.f : (float)c;        // (NaN: NaN)
    for (int tile = blockIdx.x; tile < a.n_tiles; tile += gridDim.x) {
        const int t = tensor_of(a, tile);
        const int64_t at = (int64_t)(tile - a.first_tile[t]) * kTile;
        const int n = (int)min((int64_t)kTile, a.n[t] - at);
        const void* s = a.src[t];
        void* d = a.dst[t];
        const int from = a.kind[t] & 3, to = (a.kind[t] >> 2) & 3;
        if (d == nullptr || (d == s && f == 1.f)) continue;
        using B = __nv_bfloat16;
        using H = __half;
#define HL_SCALE(S, D) tile_scale(static_cast<const S*>(s) + at, static_cast<D*>(d) + at, n, f)
        if (from == HL_F32) {
            if (to == HL_F32) HL_SCALE(float, float);
            else if (to == HL_BF16) HL_SCALE(float, B);
            else HL_SCALE(float, H);
        } else if (from == HL_BF16) {
            if (to == HL_F32) HL_SCALE(B, float);
            else if (to == HL_BF16) HL_SCALE(B, B);
            else HL_SCALE(B, H);
        } else {
            if (to == HL_F32) HL_SCALE(H, float);
            else if (to == HL_BF16) HL_SCALE(H, B);
            else HL_SCALE(H, H);
        }
#undef HL_SCALE
    }
}

int type_size(int32_t dtype) { return dtype == HL_F32 ? 4 : dtype == HL_BF16 || dtype == HL_F16 ? 2 : 0; }

bool tensors_ok(const hl_tensor* ts, int32_t n) {
    if (n < 0 || (n > 0 && !ts)) return false;
    for (int i = 0; i < n; ++i) {
        const hl_tensor& t = ts[i];
        const int s = type_size(t.src_dtype), d = type_size(t.dst_dtype);
        if (t.n < 0 || t.n >= (int64_t(1) << 40) || !s || !d || (t.flags & ~HL_TENSOR_NOT_IN_NORM) || t.reserved)
            return false;
        if (t.n == 0) continue;
        if (!t.src || reinterpret_cast<uintptr_t>(t.src) % s || reinterpret_cast<uintptr_t>(t.dst) % d) return false;
        if (t.dst == t.src && t.src_dtype != t.dst_dtype) return false;
    }
    return true;
}

int grad_grid() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        sms = kSMsFallback;
    return sms * kGradCtas < kMaxPartials ? sms * kGradCtas : kMaxPartials;
}

// f(args) for the tensors that count (of the norm, or those to write) in groups of at most N, each a kernel's argument
template <int N, typename F>
int32_t in_groups(const hl_tensor* ts, int32_t n, bool norm, F f) {
    TensorPairArgs<N> a;
    int i = 0;
    while (i < n) {
        memset(&a, 0, sizeof(a));
        int64_t tiles = 0;
        for (; i < n && a.n_tensors < N; ++i) {
            const hl_tensor& t = ts[i];
            if (t.n == 0 || (norm ? (t.flags & HL_TENSOR_NOT_IN_NORM) != 0 : t.dst == nullptr)) continue;
            const int64_t more = div_up(t.n, kTile);
            if (tiles + more > 0x7fffffff) break;
            const int k = a.n_tensors++;
            a.src[k] = t.src;
            a.dst[k] = t.dst;
            a.n[k] = t.n;
            a.first_tile[k] = (int32_t)tiles;
            a.kind[k] = (uint8_t)(t.src_dtype | (t.dst_dtype << 2));
            tiles += more;
        }
        a.n_tiles = (int32_t)tiles;
        if (a.n_tensors == 0) break;
        const int32_t st = f(a);
        if (st != HL_OK) return st;
    }
    return HL_OK;
}

template <int N>
int32_t clip(const hl_tensor* ts, int32_t n, const double* further, int32_t n_further, bool scale, float max_norm, float* norm,
             double* partial, cudaStream_t stream) {
    const int most = grad_grid();
    int64_t tiles = 0;
    for (int i = 0; i < n; ++i) tiles += ts[i].flags & HL_TENSOR_NOT_IN_NORM ? 0 : div_up(ts[i].n, kTile);
    const int n_partials = tiles ? grid_for(tiles, 1, most) : 0;
    bool more = false;
    int32_t st = in_groups<N>(ts, n, true, [&](const TensorPairArgs<N>& a) -> int32_t {
        HL_CUDA_TRY(launch(k_grad_squares<N>, n_partials, kNT, stream, a, more ? 1 : 0, partial));   // (later groups add)
        more = true;
        note_launches(1);
        return HL_OK;
    });
    if (st != HL_OK) return st;
    bool said = false;
    if (scale) {
        st = in_groups<N>(ts, n, false, [&](const TensorPairArgs<N>& a) -> int32_t {
            HL_CUDA_TRY(launch(k_grad_scale<N>, grid_for(a.n_tiles, 1, most), kNT, stream, a, (const double*)partial, n_partials,
                               further, n_further, max_norm, said ? nullptr : norm));
            said = true;
            note_launches(1);
            return HL_OK;
        });
        if (st != HL_OK) return st;
    }
    if (!said && norm) {
        HL_CUDA_TRY(launch(k_grad_norm, 1, kNT, stream, (const double*)partial, n_partials, further, n_further, norm));
        note_launches(1);
    }
    HL_LAUNCH_CHECK();
    return HL_OK;
}

int32_t clip_call(const hl_tensor* ts, int32_t n, const double* further, int32_t n_further, bool scale, float max_norm,
                  float* norm, void* ws, size_t ws_bytes, cudaStream_t stream) {
    if (!tensors_ok(ts, n) || n_further < 0 || (n_further > 0 && !further) || !(max_norm >= 0.f) || (!scale && !norm) || !ws ||
        (reinterpret_cast<uintptr_t>(further) & 7) || (reinterpret_cast<uintptr_t>(norm) & 3) ||
        (reinterpret_cast<uintptr_t>(ws) & 255))
        return HL_EINVAL;
    if (ws_bytes < hl_grad_workspace_bytes()) return HL_ECAPACITY;
    double* partial = static_cast<double*>(ws);
    if (n <= 32) return clip<32>(ts, n, further, n_further, scale, max_norm, norm, partial, stream);
    return clip<1000>(ts, n, further, n_further, scale, max_norm, norm, partial, stream);
}

// ---- an embedding's row gradients -----------------------------------------------------------------------------------
// Sum over the distinct slots u of |sum over the lookups j of u of grad[bag(j)]|^2, from the (slot, bag) pairs sorted by slot.
// A CTA takes windows of consecutive lookups, each of its groups of G lanes kRun of them and 4 * G columns; blockIdx.y: which
// columns.  A group sums its lookups run by run in fp64; the pieces of a run over several groups meet in shared memory, and
// those of a run over several windows go through `pieces` to k_rows_long.
constexpr int kRun = 16;
template <int G>
struct RowShape {
    static constexpr int kGroups = kNT / G, kWindow = kGroups * kRun;
};

__device__ __forceinline__ double square(const double a[4]) { return a[0] * a[0] + a[1] * a[1] + a[2] * a[2] + a[3] * a[3]; }

template <int G>
__global__ void __launch_bounds__(kNT) k_rows_squares(const int32_t* __restrict__ slots, const int32_t* __restrict__ bags,
                                                      const int32_t* __restrict__ d_n, int64_t max_n, int64_t n_slots,
                                                      int64_t n_bags, const float4* __restrict__ grad, int D4,
                                                      double* __restrict__ pieces, int32_t* __restrict__ starts,
                                                      double* __restrict__ partial) {
    using Shape = RowShape<G>;
    __shared__ double s_head[kNT][4];                // of a run that an earlier group began, by lane
    __shared__ bool s_cont[Shape::kGroups], s_whole[Shape::kGroups];
    const int64_t n = min((int64_t)max(*d_n, 0), max_n);
    const int64_t windows = (n + Shape::kWindow - 1) / Shape::kWindow;
    const int g = threadIdx.x / G, sub = threadIdx.x % G, c = blockIdx.y * G + sub;
    const bool mine = c < D4;
    double total = 0.0;
    for (int64_t w = blockIdx.x; w < windows; w += gridDim.x) {
        const int64_t first = w * Shape::kWindow + g * kRun;
        const int len = (int)max((int64_t)0, min((int64_t)kRun, n - first));
        double acc[4] = {}, tail[4] = {};
        bool cont = false, whole = false, open = false;
        if (len > 0) {
            int32_t slot = slots[first];
            const int32_t before = first > 0 ? slots[first - 1] : -1;
            cont = first > 0 && before == slot;
            bool head = cont;                        // the run at hand began before this group's lookups
#pragma unroll 4
            for (int i = 0; i < len; ++i) {
                const int32_t s = slots[first + i], b = bags[first + i];
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (mine && s >= 0 && s < n_slots && b >= 0 && b < n_bags) v = __ldg(&grad[(int64_t)b * D4 + c]);
                if (s != slot) {                     // a run ends
                    if (head) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) s_head[threadIdx.x][k] = acc[k];
                    } else {
                        total += square(acc);
                    }
                    head = false;
                    slot = s;
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[k] = 0.0;
                }
                acc[0] += v.x;
                acc[1] += v.y;
                acc[2] += v.z;
                acc[3] += v.w;
            }
            const bool goes_on = first + len < n && slots[first + len] == slot;
            if (head) {                              // one run, from before the first to the last of them
                whole = goes_on;
#pragma unroll
                for (int k = 0; k < 4; ++k) s_head[threadIdx.x][k] = acc[k];
            } else if (goes_on) {
                open = true;
#pragma unroll
                for (int k = 0; k < 4; ++k) tail[k] = acc[k];
            } else {
                total += square(acc);
            }
        }
        if (sub == 0) {
            s_cont[g] = cont;
            s_whole[g] = whole;
        }
        __syncthreads();
        // the group that began a run puts it together; the window's first group also what an earlier window's run left here
        if (g == 0 && cont) {
            double a[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) a[k] = s_head[sub][k];
            for (int h = 1; h < Shape::kGroups && s_whole[h - 1] && s_cont[h]; ++h)
#pragma unroll
                for (int k = 0; k < 4; ++k) a[k] += s_head[h * G + sub][k];
            if (mine)
#pragma unroll
                for (int k = 0; k < 4; ++k) pieces[((w * 2 + 0) * D4 + c) * 4 + k] = a[k];
        }
        bool out = false;
        if (open) {
            int h = g + 1;
            bool more = true;
            for (; more && h < Shape::kGroups; ++h) {
#pragma unroll
                for (int k = 0; k < 4; ++k) tail[k] += s_head[h * G + sub][k];
                more = s_whole[h];
            }
            out = more;                              // on into the next window
            if (!out) total += square(tail);
            else if (mine)
#pragma unroll
                for (int k = 0; k < 4; ++k) pieces[((w * 2 + 1) * D4 + c) * 4 + k] = tail[k];
        }
        const int any = __syncthreads_or(out);
        if (threadIdx.x == 0 && blockIdx.y == 0) starts[w] = any;
    }
    total = block_sum(mine ? total : 0.0);
    if (threadIdx.x == 0) partial[blockIdx.y * gridDim.x + blockIdx.x] = total;
}

// The runs over several windows: a CTA looks for the windows in which one starts.
template <int G>
__global__ void __launch_bounds__(kNT) k_rows_long(const int32_t* __restrict__ slots, const int32_t* __restrict__ d_n,
                                                   int64_t max_n, int D4, const double* __restrict__ pieces,
                                                   const int32_t* __restrict__ starts, double* __restrict__ partial) {
    using Shape = RowShape<G>;
    __shared__ double s_sum[kNT][4];
    const int64_t n = min((int64_t)max(*d_n, 0), max_n);
    const int64_t windows = (n + Shape::kWindow - 1) / Shape::kWindow;
    const int g = threadIdx.x / G, sub = threadIdx.x % G, c = blockIdx.y * G + sub;
    const bool mine = c < D4;
    double total = 0.0;
    for (int64_t w = blockIdx.x; w < windows; w += gridDim.x) {
        if (!starts[w]) continue;
        const int32_t slot = slots[(w + 1) * Shape::kWindow - 1];
        int64_t last = w + 1;                        // the window in which the run ends
        for (;;) {
            const int64_t x = last + threadIdx.x, next = (x + 1) * Shape::kWindow;
            const bool ends = next >= n || slots[next] != slot;
            const int any = __syncthreads_or(ends);
            if (any) {
                __shared__ int s_first;
                if (threadIdx.x == 0) s_first = kNT;
                __syncthreads();
                if (ends) atomicMin(&s_first, (int)threadIdx.x);
                __syncthreads();
                last += s_first;
                __syncthreads();
                break;
            }
            last += kNT;
        }
        double a[4] = {};
        if (mine) {
            if (g == 0)
#pragma unroll
                for (int k = 0; k < 4; ++k) a[k] = pieces[((w * 2 + 1) * D4 + c) * 4 + k];
            for (int64_t x = w + 1 + g; x <= last; x += Shape::kGroups)
#pragma unroll
                for (int k = 0; k < 4; ++k) a[k] += pieces[((x * 2 + 0) * D4 + c) * 4 + k];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) s_sum[threadIdx.x][k] = a[k];
        __syncthreads();
        if (g == 0) {
            for (int h = 1; h < Shape::kGroups; ++h)
#pragma unroll
                for (int k = 0; k < 4; ++k) a[k] += s_sum[h * G + sub][k];
            total += square(a);
        }
        __syncthreads();
    }
    total = block_sum(mine ? total : 0.0);
    if (threadIdx.x == 0) partial[blockIdx.y * gridDim.x + blockIdx.x] = total;
}

__global__ void __launch_bounds__(kNT) k_rows_total(const double* __restrict__ partial, int n_partials, double* sumsq) {
    const double sum = total_squares(partial, n_partials, nullptr, 0);
    if (threadIdx.x == 0) *sumsq = sum;
}

// In the backward region: the pieces of runs over several windows where hl_embbag_bwd_apply keeps its own (a call of one window
// has none; of more, a window's two pieces of D doubles take less room than its four or more chunks' two of D floats), the
// CTAs' sums and the windows' flags in scratch of the sort.
template <int G>
int32_t rows_squares(hl_ctx* ctx, const int32_t* slots, const int32_t* bags, const int32_t* d_n, const float* grad,
                     double* sumsq, cudaStream_t stream) {
    using Shape = RowShape<G>;
    static_assert(Shape::kWindow >= 4 * kBwdChunk, "room for the pieces");
    const int D4 = ctx->D / 4, cols = (int)div_up(D4, G);
    const int64_t windows = div_up(ctx->max_nnz > 0 ? ctx->max_nnz : 1, Shape::kWindow);
    const int short_ctas = grid_for(windows, 1, 4 * ctx_sms(ctx)), long_ctas = grid_for(windows, 1, ctx_sms(ctx));
    const int n_partials = (short_ctas + long_ctas) * cols;
    double* pieces = reinterpret_cast<double*>(ctx->r.bwd_part);
    double* partial = reinterpret_cast<double*>(ctx->r.bwd_hist[1]);
    int32_t* starts = reinterpret_cast<int32_t*>(partial + n_partials);
    if ((n_partials * 2 + windows) > sort_hist_words(ctx->max_nnz)) return HL_EINVAL;        // (rows of up to 1 024 fp32: never)
    const auto grid = [&](int ctas) { return dim3((unsigned)ctas, (unsigned)cols); };
    HL_CUDA_TRY(launch(k_rows_squares<G>, grid(short_ctas), kNT, stream, slots, bags, d_n, ctx->max_nnz,
                       ctx->hot_cap + ctx->staging_cap, ctx->max_bags, reinterpret_cast<const float4*>(grad), D4, pieces, starts,
                       partial));
    HL_CUDA_TRY(launch(k_rows_long<G>, grid(long_ctas), kNT, stream, slots, d_n, ctx->max_nnz, D4, (const double*)pieces,
                       (const int32_t*)starts, partial + short_ctas * cols));
    HL_CUDA_TRY(launch(k_rows_total, 1, kNT, stream, (const double*)partial, n_partials, sumsq));
    note_launches(3);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

}  // namespace
}  // namespace hl

using namespace hl;

extern "C" size_t hl_grad_workspace_bytes(void) { return kMaxPartials * sizeof(double); }

extern "C" int32_t hl_grad_norm(const hl_tensor* tensors, int32_t n_tensors, const double* d_further, int32_t n_further,
                                float* d_norm, void* d_workspace, size_t ws_bytes, void* stream) {
    return clip_call(tensors, n_tensors, d_further, n_further, false, 0.f, d_norm, d_workspace, ws_bytes,
                     static_cast<cudaStream_t>(stream));
}

extern "C" int32_t hl_grad_clip(const hl_tensor* tensors, int32_t n_tensors, const double* d_further, int32_t n_further,
                                float max_norm, float* d_norm, void* d_workspace, size_t ws_bytes, void* stream) {
    return clip_call(tensors, n_tensors, d_further, n_further, true, max_norm, d_norm, d_workspace, ws_bytes,
                     static_cast<cudaStream_t>(stream));
}

extern "C" int32_t hl_embbag_grad_sumsq(hl_ctx* ctx, const int32_t* d_sorted_slots, const int32_t* d_sorted_bags,
                                        const int32_t* d_n_lookups, const float* d_grad_out, double* d_sumsq, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!ctx || !d_n_lookups || !d_sumsq || (ctx->max_nnz > 0 && (!d_sorted_slots || !d_sorted_bags || !d_grad_out)))
        return HL_EINVAL;
    const int D4 = ctx->D / 4;
    if (D4 > 256 || (reinterpret_cast<uintptr_t>(d_grad_out) & 15)) return HL_EINVAL;
    return as_graph(kept_launches(ctx), [&] {
#define HL_ROWS(G) rows_squares<G>(ctx, d_sorted_slots, d_sorted_bags, d_n_lookups, d_grad_out, d_sumsq, stream)
        return D4 <= 4 ? HL_ROWS(4) : D4 <= 8 ? HL_ROWS(8) : D4 <= 16 ? HL_ROWS(16) : HL_ROWS(32);
#undef HL_ROWS
    });
}
