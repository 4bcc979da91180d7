// The global norm of gradients and clipping: sums of squares over many tensors, the squared norm of an embedding's row
// gradients, and the tensors scaled.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstring>

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
// A call's tensors are cut into tiles of 2^tile_bits values, and every CTA takes a run of tiles: two kernels, of which the second
// needs the first's sums, so that tensors beyond the L2's size are read twice.  420 tensors, 153 M values, bf16 scaled into fp32:
// squares 306 MB in 58 us (5.3 TB/s), scaling 919 MB in 165 us (5.6 TB/s, some of it from the L2); 14 tensors of 0.2 M fp32 in all:
// 6.9 us a call, two launches.  One cluster of 16 CTAs for both, for few values, took 8.2 to 12.3 instead of 6.8 to 8.4: a CTA's
// tiles one after the other.  Squares are exact in fp64; the sums' order is the same in every call.  Tried: fp64 made from the bits by shifts instead of
// conversions 67 us, eight loads ahead 94 (half as many CTAs fit).
constexpr int kMinTileBits = 10, kMaxTileBits = 13;
constexpr int kGradCtas = 8;                         // CTAs per multiprocessor
constexpr int kMaxPartials = 2048;                   // sums of squares, one per CTA
constexpr int kAhead = 4;                            // loads of a thread on their way

// N tensors and where their tiles begin, as a kernel argument.
template <int N>
struct TensorPairArgs {
    const void* src[N];
    void* dst[N];
    int64_t n[N];
    int32_t first_tile[N];
    uint8_t kind[N];                                 // type of src, type of dst (two bits each)
    int32_t n_tensors, n_tiles, tile_bits, unused;
};

template <typename T>
constexpr int kWide = 16 / sizeof(T);                // values in 16 bytes
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
__device__ __forceinline__ void put(__half* p, float x) { *p = __float2half_rn(x); }
// a word's values, and a word from values
template <typename T>
__device__ __forceinline__ void unpack(uint32_t w, float* x) {
    if constexpr (sizeof(T) == 4) {
        x[0] = __uint_as_float(w);
    } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        x[0] = __uint_as_float(w << 16);
        x[1] = __uint_as_float(w & 0xffff0000u);
    } else {
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
        x[0] = v.x;
        x[1] = v.y;
    }
}
template <typename T>
__device__ __forceinline__ uint32_t pack(const float* x) {
    if constexpr (sizeof(T) == 4) {
        return __float_as_uint(x[0]);
    } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[0], x[1]);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const __half2 v = __floats2half2_rn(x[0], x[1]);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
}
template <typename T>
__device__ __forceinline__ void unpack4(const uint4& r, float (&x)[kWide<T>]) {
    constexpr int n = 4 / sizeof(T);
    unpack<T>(r.x, x);
    unpack<T>(r.y, x + n);
    unpack<T>(r.z, x + 2 * n);
    unpack<T>(r.w, x + 3 * n);
}

// values before p's next multiple of 16 bytes
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int n) {
    const int h = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T);
    return h < n ? h : n;
}

template <typename T>
__device__ __forceinline__ double tile_squares(const T* __restrict__ p, int n) {
    constexpr int W = kWide<T>;
    double sum = 0.0;
    const int head = head_of(p, n), nv = (n - head) / W, tail = head + nv * W;
    const uint4* q = reinterpret_cast<const uint4*>(p + head);
    for (int i = threadIdx.x; i < nv; i += kNT * kAhead) {
        uint4 r[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) r[u] = i + u * kNT < nv ? __ldg(&q[i + u * kNT]) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float x[W];
            unpack4<T>(r[u], x);
#pragma unroll
            for (int j = 0; j < W; ++j) sum = fma((double)x[j], (double)x[j], sum);
        }
    }
    for (int i = threadIdx.x; i < head + n - tail; i += kNT) {
        const double x = to_f32(p[i < head ? i : tail + i - head]);
        sum = fma(x, x, sum);
    }
    return sum;
}

// As many values at a time as are 16 bytes in the wider type, so that a warp's stores are whole lines, which the L2 gives up first:
// what the sums of squares read last stays in it (165 us instead of 177).  (p and d may be the same.)
template <typename S, typename D>
__device__ __forceinline__ void tile_scale(const S* p, D* d, int n, float f) {
    constexpr int W = sizeof(S) > sizeof(D) ? kWide<S> : kWide<D>, kIn = W * sizeof(S) / 4, kOut = W * sizeof(D) / 4;   // words
    const int head = head_of(p, n);
    if (reinterpret_cast<uintptr_t>(d + head) % (kOut * 4)) {  // no common lines
#pragma unroll 4
        for (int i = threadIdx.x; i < n; i += kNT) put(&d[i], f * to_f32(p[i]));
        return;
    }
    const int nv = (n - head) / W, tail = head + nv * W;
    constexpr int kFly = kIn == 4 ? kAhead : 2 * kAhead;
    using In = std::conditional_t<kIn == 4, uint4, uint2>;
    const In* q = reinterpret_cast<const In*>(p + head);
    for (int i = threadIdx.x; i < nv; i += kNT * kFly) {
        In r[kFly];
#pragma unroll
        for (int u = 0; u < kFly; ++u) r[u] = i + u * kNT < nv ? __ldcs(&q[i + u * kNT]) : In{};
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            if (i + u * kNT >= nv) break;
            constexpr int kPerIn = 4 / sizeof(S), kPerOut = 4 / sizeof(D);
            float x[W];
            unpack<S>(r[u].x, x);
            unpack<S>(r[u].y, x + kPerIn);
            if constexpr (kIn == 4) {
                unpack<S>(r[u].z, x + 2 * kPerIn);
                unpack<S>(r[u].w, x + 3 * kPerIn);
            }
#pragma unroll
            for (int j = 0; j < W; ++j) x[j] *= f;
            D* to = d + head + (int64_t)(i + u * kNT) * W;
            if constexpr (kOut == 2)
                __stcs(reinterpret_cast<uint2*>(to), make_uint2(pack<D>(x), pack<D>(x + kPerOut)));
            else
                __stcs(reinterpret_cast<uint4*>(to), make_uint4(pack<D>(x), pack<D>(x + kPerOut), pack<D>(x + 2 * kPerOut), pack<D>(x + 3 * kPerOut)));
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
// CTA b's tiles are [first_of(b), first_of(b + 1)).
template <int N>
__device__ __forceinline__ int first_of(const TensorPairArgs<N>& a, unsigned b) {
    return (int)((int64_t)a.n_tiles * b / gridDim.x);
}

template <int N>
__device__ __forceinline__ double squares_of(const TensorPairArgs<N>& a, int t, int tile) {
    const int64_t at = (int64_t)(tile - a.first_tile[t]) << a.tile_bits;
    const int n = (int)min((int64_t)1 << a.tile_bits, a.n[t] - at), from = a.kind[t] & 3;
    if (from == HL_F32) return tile_squares(static_cast<const float*>(a.src[t]) + at, n);
    if (from == HL_BF16) return tile_squares(static_cast<const __nv_bfloat16*>(a.src[t]) + at, n);
    return tile_squares(static_cast<const __half*>(a.src[t]) + at, n);
}

// What the tensors are scaled by.
__device__ __forceinline__ float factor_of(double norm, double max_norm) {
    const double c = max_norm / (norm + 1e-6);
    return c > 1.0 ? 1.f : (float)c;                 // (NaN: NaN)
}

template <int N>
__device__ __forceinline__ void scale(const TensorPairArgs<N>& a, int t, int tile, float f) {
    const int64_t at = (int64_t)(tile - a.first_tile[t]) << a.tile_bits;
    const int n = (int)min((int64_t)1 << a.tile_bits, a.n[t] - at);
    const void* s = a.src[t];
    void* d = a.dst[t];
    const int from = a.kind[t] & 3, to = (a.kind[t] >> 2) & 3;
    if (d == nullptr || (d == s && f == 1.f)) return;
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

// partial[b] (+)= the squares of CTA b's tiles
template <int N>
__global__ void __launch_bounds__(kNT) k_grad_squares(const __grid_constant__ TensorPairArgs<N> a, int more,
                                                      double* __restrict__ partial) {
    let_next_start();
    double sum = 0.0;
    const int end = first_of(a, blockIdx.x + 1);
    int tile = first_of(a, blockIdx.x), t = tensor_of(a, tile);
    for (; tile < end; ++tile) {
        if (t + 1 < a.n_tensors && a.first_tile[t + 1] <= tile) ++t;
        sum += squares_of(a, t, tile);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = more ? partial[blockIdx.x] + sum : sum;
}

__device__ __forceinline__ double total_squares(const double* partial, int n_partials, const double* further, int n_further) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n_partials; i += kNT) sum += partial[i];
    for (int i = threadIdx.x; i < n_further; i += kNT) sum += further[i];
    return block_sum(sum);
}

__global__ void __launch_bounds__(kNT) k_grad_norm(const double* partial, int n_partials, const double* further, int n_further,
                                                   float* norm) {
    wait_for_last();
    const double sum = total_squares(partial, n_partials, further, n_further);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

// A CTA takes its tiles from the last to the first: what the sums of squares read last is still in the L2.  max_norm: the bits of a
// double.
template <int N>
__global__ void __launch_bounds__(kNT, 4) k_grad_scale(const __grid_constant__ TensorPairArgs<N> a, const double* partial,
                                                    int n_partials, const double* further, int n_further, long long max_norm,
                                                    float* norm) {
    const int begin = first_of(a, blockIdx.x);
    int tile = first_of(a, blockIdx.x + 1) - 1, t = tensor_of(a, tile);
    wait_for_last();
    const double total = sqrt(total_squares(partial, n_partials, further, n_further));
    if (blockIdx.x == 0 && threadIdx.x == 0 && norm) *norm = (float)total;
    const float f = factor_of(total, __longlong_as_double(max_norm));
    for (; tile >= begin; --tile) {
        if (a.first_tile[t] > tile) --t;
        scale(a, t, tile, f);
    }
}

int type_size(int32_t dtype) { return dtype == HL_F32 ? 4 : dtype == HL_BF16 || dtype == HL_F16 ? 2 : 0; }

// The tensors that count: those of the norm, or those to write.
enum Which { kOfNorm, kToWrite };
bool counts(const hl_tensor& t, Which which) {
    return t.n > 0 && (which == kOfNorm ? !(t.flags & HL_TENSOR_NOT_IN_NORM) : t.dst != nullptr);
}
// How many they are, and their values.
struct Count {
    int64_t values = 0;
    int32_t tensors = 0;
};

bool tensors_ok(const hl_tensor* ts, int32_t n, Count (&count)[2]) {
    if (n < 0 || (n > 0 && !ts)) return false;
    for (int i = 0; i < n; ++i) {
        const hl_tensor& t = ts[i];
        const int s = type_size(t.src_dtype), d = type_size(t.dst_dtype);
        if (t.n < 0 || t.n >= (int64_t(1) << 40) || !s || !d || (t.flags & ~HL_TENSOR_NOT_IN_NORM) || t.reserved)
            return false;
        if (t.n == 0) continue;
        if (!t.src || (reinterpret_cast<uintptr_t>(t.src) & (s - 1)) || (reinterpret_cast<uintptr_t>(t.dst) & (d - 1))) return false;
        // (over the whole of itself, with the same type, or over nothing of it; of other tensors nothing is compared here)
        const uintptr_t from = reinterpret_cast<uintptr_t>(t.src), to = reinterpret_cast<uintptr_t>(t.dst);
        if (from == to ? t.src_dtype != t.dst_dtype : to && from < to + t.n * d && to < from + t.n * s) return false;
        for (const Which which : {kOfNorm, kToWrite}) {
            if (!counts(t, which)) continue;
            count[which].values += t.n;
            ++count[which].tensors;
        }
    }
    return true;
}

int grad_grid() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        sms = kSMsFallback;
    return sms * kGradCtas < kMaxPartials ? sms * kGradCtas : kMaxPartials;
}

// f(args) for the tensors that count in groups of at most N, each a kernel's argument
template <int N, typename F>
int32_t in_groups(const hl_tensor* ts, int32_t n, Which which, int tile_bits, F f) {
    TensorPairArgs<N> a;
    int i = 0;
    while (i < n) {
        a.n_tensors = 0;
        int64_t tiles = 0;
        for (; i < n && a.n_tensors < N; ++i) {
            const hl_tensor& t = ts[i];
            if (!counts(t, which)) continue;
            const int64_t more = (t.n + (int64_t(1) << tile_bits) - 1) >> tile_bits;
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
        a.tile_bits = tile_bits;
        if (a.n_tensors == 0) break;
        const int32_t st = f(a);
        if (st != HL_OK) return st;
    }
    return HL_OK;
}

// Their tiles: the smallest that leave a CTA one, as near as their number and all their values tell.
struct Tiling {
    int bits;
    int64_t tiles;
};
Tiling tiling_of(const Count& c, int most) {
    int bits = kMinTileBits;
    while (bits < kMaxTileBits && (c.values >> bits) + c.tensors > most) ++bits;
    return {bits, (c.values >> bits) + c.tensors};
}

template <int N>
int32_t clip(const hl_tensor* ts, int32_t n, const Count (&count)[2], const double* further, int32_t n_further, bool scale,
             double max_norm, float* norm, double* partial, cudaStream_t stream) {
    long long max_norm_bits;
    std::memcpy(&max_norm_bits, &max_norm, sizeof max_norm_bits);
    const int most = grad_grid();
    const Tiling of_norm = tiling_of(count[kOfNorm], most);
    const int n_partials = count[kOfNorm].tensors ? grid_for(of_norm.tiles, 1, most) : 0;
    const int first_after = n_partials ? kAfterLast : 0;       // (of what the caller has on the stream, all has to be over)
    bool more = false, said = false;
    const auto add_squares = [&](const TensorPairArgs<N>& a) -> int32_t {
        HL_CUDA_TRY(launch(k_grad_squares<N>, n_partials, kNT, stream, a, more ? 1 : 0, partial));   // (later groups add)
        more = true;
        note_launches(1);
        return HL_OK;
    };
    const auto write_scaled = [&](const TensorPairArgs<N>& a) -> int32_t {
        HL_CUDA_TRY(launch_cluster(k_grad_scale<N>, grid_for(a.n_tiles, 1, most), kNT, 0, said ? 0 : first_after, stream, a,
                                   (const double*)partial, n_partials, further, n_further, max_norm_bits, said ? nullptr : norm));
        said = true;
        note_launches(1);
        return HL_OK;
    };
    // one list for both, where all tensors are one group and count in both
    const bool same = scale && n <= N && of_norm.tiles <= 0x7fffffff && count[kOfNorm].tensors == n &&
                      count[kToWrite].tensors == n;
    int32_t st = in_groups<N>(ts, n, kOfNorm, of_norm.bits, [&](const TensorPairArgs<N>& a) -> int32_t {
        const int32_t s = add_squares(a);
        return s == HL_OK && same ? write_scaled(a) : s;
    });
    if (st == HL_OK && scale && !same) st = in_groups<N>(ts, n, kToWrite, tiling_of(count[kToWrite], most).bits, write_scaled);
    if (st != HL_OK) return st;
    if (!said && norm) {
        HL_CUDA_TRY(launch_cluster(k_grad_norm, 1, kNT, 0, first_after, stream, (const double*)partial, n_partials, further,
                                   n_further, norm));
        note_launches(1);
    }
    HL_LAUNCH_CHECK();
    return HL_OK;
}

int32_t clip_call(const hl_tensor* ts, int32_t n, const double* further, int32_t n_further, bool scale, double max_norm,
                  float* norm, void* ws, size_t ws_bytes, cudaStream_t stream) {
    Count count[2];
    if (!tensors_ok(ts, n, count) || n_further < 0 || (n_further > 0 && !further) || !(max_norm >= 0.0) || (!scale && !norm) || !ws ||
        (reinterpret_cast<uintptr_t>(further) & 7) || (reinterpret_cast<uintptr_t>(norm) & 3) ||
        (reinterpret_cast<uintptr_t>(ws) & 255))
        return HL_EINVAL;
    if (ws_bytes < hl_grad_workspace_bytes()) return HL_ECAPACITY;
    double* partial = static_cast<double*>(ws);
    // (A kilobyte of arguments costs the host 0.1 us a launch: 453 tensors 10.8 us a call with room for 512 of them, 14 with room for
    // 1 000.)
#define HL_CLIP(N) clip<N>(ts, n, count, further, n_further, scale, max_norm, norm, partial, stream)
    return n <= 32 ? HL_CLIP(32) : n <= 128 ? HL_CLIP(128) : n <= 256 ? HL_CLIP(256) : n <= 512 ? HL_CLIP(512) : HL_CLIP(1000);
#undef HL_CLIP
}

// ---- an embedding's row gradients -----------------------------------------------------------------------------------
// Sum over the distinct slots u of |sum over the lookups j of u of grad[bag(j)]|^2, from the (slot, bag) pairs sorted by slot.
// A CTA takes windows of consecutive lookups, each of its groups of G lanes a few of them and 4 * G columns; blockIdx.y: which
// columns.  A group sums its lookups run by run in fp64; the pieces of a run over several groups meet in shared memory, and
// those of a run over several windows go through `pieces` to k_rows_long.  Bound by the latency of rows read in the slots' order:
// 426 K lookups of 64 fp32, 109 MB in 26.8 us (4.1 TB/s) and 10 for the long runs, a chain of five dependent loads; 129 K of 16
// fp32: 8 and 8.5.  Windows of a CTA by itself took 62 instead of 44, four CTAs a multiprocessor 26.2, five with half the rows on
// their way 27.2.
template <int G>
struct RowShape {
    static constexpr int kGroups = kNT / G, kRun = G < 16 ? 8 : 16, kWindow = kGroups * kRun;
    static constexpr int kAsk = (kWindow + kNT - 1) / kNT;     // lookups of a window that a thread asks for
    static_assert(kGroups <= 64, "a bit per group");
};

__device__ __forceinline__ double square(const double (&a)[4]) { return a[0] * a[0] + a[1] * a[1] + a[2] * a[2] + a[3] * a[3]; }

template <int G>
__global__ void __launch_bounds__(kNT, G < 32 ? 3 : 2) k_rows_squares(const int32_t* __restrict__ slots, const int32_t* __restrict__ bags,
                                                      const int32_t* __restrict__ d_n, int64_t max_n, int64_t n_slots,
                                                      int64_t n_bags, const float4* __restrict__ grad, int D4,
                                                      double* __restrict__ pieces, int32_t* __restrict__ starts,
                                                      int64_t max_windows, double* __restrict__ partial,
                                                      double* __restrict__ sumsq) {
    using Shape = RowShape<G>;
    constexpr int kGroups = Shape::kGroups, kWindow = Shape::kWindow, kRun = Shape::kRun, kRows = kRun < 8 ? kRun : 8;
    __shared__ int32_t s_slot[kWindow + 2], s_bag[kWindow];    // s_slot[0]: the lookup before the window's; s_bag -1: none to add
    __shared__ __align__(16) double s_head[kNT][4];            // of a run that an earlier group began, by lane
    __shared__ int32_t s_start;
    __shared__ uint32_t s_whole[kGroups / 32 + 1];             // groups whose lookups are all of a run that goes on behind them
    let_next_start();
    const int64_t n = min((int64_t)max(__ldg(d_n), 0), max_n), windows = (n + kWindow - 1) / kWindow;
    const int g = threadIdx.x / G, sub = threadIdx.x % G, c = blockIdx.y * G + sub;
    const bool mine = c < D4;
    const int col = mine ? c : 0;
    double total = 0.0;
    if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) starts[max_windows] = 0;      // (k_rows_long's tally)
    // the next window's pairs are on their way while this one's rows are summed; two threads also take the lookups around it
    constexpr int kAsk = Shape::kAsk;
    int32_t slot_ahead[kAsk] = {}, bag_ahead[kAsk] = {}, around_ahead = 0;
    const auto ask = [&](int64_t w) {
        const int64_t around = threadIdx.x == 0 ? w * kWindow - 1 : (w + 1) * kWindow;
#pragma unroll
        for (int i = 0; i < kAsk; ++i) {
            const int l = threadIdx.x + i * kNT;
            const int64_t at = w * kWindow + l;
            if (l < kWindow && at < n) {
                slot_ahead[i] = __ldg(&slots[at]);
                bag_ahead[i] = __ldg(&bags[at]);
            }
        }
        if (threadIdx.x < 2 && around >= 0 && around < n) around_ahead = __ldg(&slots[around]);
    };
    if (blockIdx.x < windows) ask(blockIdx.x);
    for (int64_t w = blockIdx.x; w < windows; w += gridDim.x) {
        const int64_t begin = w * kWindow;
        const int here = (int)min((int64_t)kWindow, n - begin);    // lookups of the window
#pragma unroll
        for (int i = 0; i < kAsk; ++i) {
            const int l = threadIdx.x + i * kNT;
            if (l >= kWindow) break;
            const int32_t slot = slot_ahead[i], bag = bag_ahead[i];
            s_slot[1 + l] = slot;
            s_bag[l] = l < here && bag >= 0 && bag < n_bags && slot >= 0 && slot < n_slots ? bag : -1;
        }
        if (threadIdx.x < 2) s_slot[threadIdx.x ? kWindow + 1 : 0] = around_ahead;
        if (threadIdx.x <= kGroups / 32) s_whole[threadIdx.x] = 0;
        if (threadIdx.x == 0) s_start = 0;
        __syncthreads();
        if (w + gridDim.x < windows) ask(w + gridDim.x);
        const int l0 = g * kRun, len = max(0, min(kRun, here - l0));
        double acc[4] = {};
        bool cont = false, whole = false, open = false;
        int32_t slot = 0;
        if (len > 0) {
            slot = s_slot[1 + l0];
            cont = begin + l0 > 0 && s_slot[l0] == slot;
            bool head = cont;                            // the run at hand began before this group's lookups
#pragma unroll 1
            for (int i0 = 0; i0 < len; i0 += kRows) {
                float4 v[kRows];                     // (all of them asked for, whether they add anything or not: no branches)
                int32_t b[kRows];
#pragma unroll
                for (int j = 0; j < kRows; ++j) b[j] = s_bag[l0 + i0 + j];
#pragma unroll
                for (int j = 0; j < kRows; ++j) v[j] = __ldg(&grad[(int64_t)max(b[j], 0) * D4 + col]);
#pragma unroll
                for (int j = 0; j < kRows; ++j) {
                    if (i0 + j >= len) break;
                    const int32_t s = s_slot[1 + l0 + i0 + j];
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
                    if (b[j] >= 0) {
                        acc[0] += v[j].x;
                        acc[1] += v[j].y;
                        acc[2] += v[j].z;
                        acc[3] += v[j].w;
                    }
                }
            }
            const bool goes_on = begin + l0 + len < n && s_slot[1 + l0 + len] == slot;
            if (head) {                                  // one run, from before the first to the last of them
                whole = goes_on;
#pragma unroll
                for (int k = 0; k < 4; ++k) s_head[threadIdx.x][k] = acc[k];
            } else if (goes_on) {
                open = true;
            } else {
                total += square(acc);
            }
        }
        if (sub == 0 && whole) atomicOr(&s_whole[g >> 5], 1u << (g & 31));
        __syncthreads();
        // The group that began a run puts it together, the window's first group also what an earlier window's run left here.  They
        // add what groups first .. last - 1 left: those that are all the run's, and the one behind them, in which it ends.
        const uint64_t mask = (uint64_t)s_whole[0] | (kGroups > 32 ? (uint64_t)s_whole[kGroups > 32] << 32 : 0);
        const auto add_from = [&](int h, double (&a)[4]) {         // returns whether the run goes on into the next window
            const uint64_t rest = h < 64 ? ~(mask >> h) : ~0ull;
            const int last = h + (rest ? __ffsll((long long)rest) - 1 : 64);       // the group in which it ends
#pragma unroll 4
            for (; h <= last && h < kGroups; ++h) {
                const double2 lo = *reinterpret_cast<const double2*>(&s_head[h * G + sub][0]);
                const double2 hi = *reinterpret_cast<const double2*>(&s_head[h * G + sub][2]);
                a[0] += lo.x;
                a[1] += lo.y;
                a[2] += hi.x;
                a[3] += hi.y;
            }
            return last >= kGroups;
        };
        if (g == 0 && cont) {
            double a[4] = {};
            (void)add_from(0, a);
            if (mine)
#pragma unroll
                for (int k = 0; k < 4; ++k) pieces[((w * 2 + 0) * D4 + c) * 4 + k] = a[k];
        }
        if (open) {
            if (!add_from(g + 1, acc)) {
                total += square(acc);
            } else {                                         // on into the next window (one run at most)
                if (sub == 0) s_start = slot + 1;
                if (mine)
#pragma unroll
                    for (int k = 0; k < 4; ++k) pieces[((w * 2 + 1) * D4 + c) * 4 + k] = acc[k];
            }
        }
        __syncthreads();
        if (threadIdx.x == 0 && blockIdx.y == 0) starts[w] = s_start;        // (0: none; the same thread clears it)
    }
    total = block_sum(mine ? total : 0.0);
    if (threadIdx.x == 0) *(sumsq ? sumsq : &partial[blockIdx.y * gridDim.x + blockIdx.x]) = total;      // sumsq: of the only CTA
}

// The sum of a run's pieces: the one in window w, in which it starts, and those of the windows up to `last`, by P threads of which
// this is number `i`: group i / G of P / G.
template <int G>
__device__ __forceinline__ void add_pieces(const double* pieces, int D4, int c, int64_t w, int64_t last, int i, int P, double (&a)[4]) {
    const auto add = [&](int64_t at) {
        const double2* p = reinterpret_cast<const double2*>(&pieces[(at * D4 + c) * 4]);
        const double2 lo = p[0], hi = p[1];
        a[0] += lo.x;
        a[1] += lo.y;
        a[2] += hi.x;
        a[3] += hi.y;
    };
    if (i / G == 0) add(w * 2 + 1);
#pragma unroll 8
    for (int64_t x = w + 1 + i / G; x <= last; x += P / G) add(x * 2);
}

// The runs over several windows, each where it starts: a warp takes a window, and a run that goes on for more than 32 others is
// the whole CTA's.  The last CTA to be done adds everything up.
template <int G>
__global__ void __launch_bounds__(kNT) k_rows_long(const int32_t* slots, const int32_t* d_n, int64_t max_n, int D4,
                                                   const double* pieces, int32_t* starts, int64_t max_windows, double* partial,
                                                   int n_partials, double* sumsq) {
    using Shape = RowShape<G>;
    constexpr int kGroups = Shape::kGroups, kWindow = Shape::kWindow;
    __shared__ double s_sum[kNT][4];
    __shared__ int64_t s_long[kWarps];
    __shared__ int s_first;
    __shared__ bool s_last;
    wait_for_last();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t first = (int64_t)blockIdx.x * kWarps + warp;
    int start = first < max_windows ? starts[first] : 0;       // (of windows that there are not: not looked at)
    const int64_t n = min((int64_t)max(*d_n, 0), max_n), windows = (n + kWindow - 1) / kWindow;
    const int sub = lane % G, c = blockIdx.y * G + sub;
    const bool mine = c < D4;
    double total = 0.0;
    for (int64_t w0 = (int64_t)blockIdx.x * kWarps; w0 < windows; w0 += (int64_t)gridDim.x * kWarps) {
        const int64_t w = w0 + warp;
        bool too_long = false;
        if (w != first && w < windows) start = starts[w];
        if (w < windows && start) {
            const int32_t slot = start - 1;
            const int64_t next = (w + 2 + lane) * kWindow;
            const unsigned ends = __ballot_sync(0xffffffffu, next >= n || slots[next] != slot);
            too_long = ends == 0;
            if (!too_long) {
                double a[4] = {};
                if (mine) add_pieces<G>(pieces, D4, c, w, w + __ffs(ends), lane, 32, a);
#pragma unroll
                for (int d = 16; d >= G; d >>= 1)
#pragma unroll
                    for (int k = 0; k < 4; ++k) a[k] += __shfl_xor_sync(0xffffffffu, a[k], d);
                if (lane < G && mine) total += square(a);
            }
        }
        if (lane == 0) s_long[warp] = too_long ? w : -1;
        __syncthreads();
        for (int i = 0; i < kWarps; ++i) {
            const int64_t x = s_long[i];
            if (x < 0) continue;                     // (the same for all threads)
            const int32_t slot = slots[(x + 1) * kWindow - 1];
            if (threadIdx.x == 0) s_first = kNT;
            __syncthreads();
            int64_t last = x + 33;                   // the window in which the run ends
            for (;; last += kNT) {
                const int64_t next = (last + threadIdx.x + 1) * kWindow;
                const bool ends = next >= n || slots[next] != slot;
                if (ends) atomicMin(&s_first, (int)threadIdx.x);
                if (__syncthreads_or(ends)) break;
            }
            double a[4] = {};
            if (mine) add_pieces<G>(pieces, D4, c, x, last + s_first, threadIdx.x, kNT, a);
#pragma unroll
            for (int k = 0; k < 4; ++k) s_sum[threadIdx.x][k] = a[k];
            __syncthreads();
            if (threadIdx.x < G && mine) {
#pragma unroll 8
                for (int h = 1; h < kGroups; ++h)
#pragma unroll
                    for (int k = 0; k < 4; ++k) a[k] += s_sum[h * G + sub][k];
                total += square(a);
            }
            __syncthreads();
        }
        __syncthreads();
    }
    total = block_sum(total);
    const int n_ctas = gridDim.x * gridDim.y;
    if (threadIdx.x == 0) {
        partial[n_partials - n_ctas + blockIdx.y * gridDim.x + blockIdx.x] = total;
        __threadfence();
        s_last = atomicAdd(&starts[max_windows], 1) == n_ctas - 1;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    double sum = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n_partials; i += kNT) sum += __ldcg(&partial[i]);
    sum = block_sum(sum);
    if (threadIdx.x == 0) *sumsq = sum;
}

// In the backward region: the pieces of runs over several windows where hl_embbag_bwd_apply keeps its own (a call of one window
// has none; of more, a window's two pieces of D doubles take less room than its four or more chunks' two of D floats), the
// CTAs' sums and the windows' flags in scratch of the sort.
template <int G>
int32_t rows_squares(hl_ctx* ctx, const int32_t* slots, const int32_t* bags, const int32_t* d_n, const float* grad,
                     double* sumsq, cudaStream_t stream) {
    using Shape = RowShape<G>;
    static_assert(Shape::kWindow >= 4 * kBwdChunk && Shape::kGroups <= 64, "room for the pieces");
    const int D4 = ctx->D / 4, cols = (int)div_up(D4, G);
    const int64_t windows = div_up(ctx->max_nnz > 0 ? ctx->max_nnz : 1, Shape::kWindow);
    const int rows_ctas = grid_for(windows, 1, (G < 32 ? 3 : 2) * ctx_sms(ctx)), long_ctas = grid_for(windows, kWarps, 2 * ctx_sms(ctx));
    const int n_partials = (rows_ctas + long_ctas) * cols;
    double* pieces = reinterpret_cast<double*>(ctx->r.bwd_part);
    double* partial = reinterpret_cast<double*>(ctx->r.bwd_hist[1]);
    int32_t* starts = reinterpret_cast<int32_t*>(partial + n_partials);
    if (2 * n_partials + windows + 1 > sort_hist_words(ctx->max_nnz)) return HL_EINVAL;      // (rows of up to 1 024 fp32: never)
    const bool only = windows == 1 && cols == 1;     // no run goes on behind it
    HL_CUDA_TRY(launch(k_rows_squares<G>, dim3((unsigned)rows_ctas, (unsigned)cols), kNT, stream, slots, bags, d_n, ctx->max_nnz,
                       ctx->hot_cap + ctx->staging_cap, ctx->max_bags, reinterpret_cast<const float4*>(grad), D4, pieces, starts,
                       windows, partial, only ? sumsq : nullptr));
    note_launches(1);
    if (only) {
        HL_LAUNCH_CHECK();
        return HL_OK;
    }
    HL_CUDA_TRY(launch_after(k_rows_long<G>, dim3((unsigned)long_ctas, (unsigned)cols), kNT, 0, stream, slots, d_n, ctx->max_nnz,
                             D4, (const double*)pieces, starts, windows, partial, n_partials, sumsq));
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

}  // namespace
}  // namespace hl

using namespace hl;

extern "C" size_t hl_grad_workspace_bytes(void) { return kMaxPartials * sizeof(double); }

extern "C" int32_t hl_grad_norm(const hl_tensor* tensors, int32_t n_tensors, const double* d_further, int32_t n_further,
                                float* d_norm, void* d_workspace, size_t ws_bytes, void* stream) {
    return clip_call(tensors, n_tensors, d_further, n_further, false, 0.0, d_norm, d_workspace, ws_bytes,
                     static_cast<cudaStream_t>(stream));
}

extern "C" int32_t hl_grad_clip(const hl_tensor* tensors, int32_t n_tensors, const double* d_further, int32_t n_further,
                                double max_norm, float* d_norm, void* d_workspace, size_t ws_bytes, void* stream) {
    return clip_call(tensors, n_tensors, d_further, n_further, true, max_norm, d_norm, d_workspace, ws_bytes,
                     static_cast<cudaStream_t>(stream));
}

extern "C" int32_t hl_embbag_grad_sumsq(hl_ctx* ctx, const int32_t* d_sorted_slots, const int32_t* d_sorted_bags,
                                        const int32_t* d_n_lookups, const float* d_grad_out, double* d_sumsq, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!ctx || !d_n_lookups || !d_sumsq || (reinterpret_cast<uintptr_t>(d_sumsq) & 7) ||
        (ctx->max_nnz > 0 && (!d_sorted_slots || !d_sorted_bags || !d_grad_out)))
        return HL_EINVAL;
    const int D4 = ctx->D / 4;
    if (D4 > 256 || (reinterpret_cast<uintptr_t>(d_grad_out) & 15)) return HL_EINVAL;
#define HL_ROWS(G) rows_squares<G>(ctx, d_sorted_slots, d_sorted_bags, d_n_lookups, d_grad_out, d_sumsq, stream)
    return D4 <= 4 ? HL_ROWS(4) : D4 <= 8 ? HL_ROWS(8) : D4 <= 16 ? HL_ROWS(16) : HL_ROWS(32);
#undef HL_ROWS
}
