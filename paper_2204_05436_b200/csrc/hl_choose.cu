// Routing to experts: the router's logits become the chosen experts and their weights, and the weights' gradient the logits'.
#include <math.h>

#include "hl_rows.cuh"

namespace hl {
namespace {

// ---- who is chosen ----------------------------------------------------------------------------------------------------
// A token has P lanes of a warp (1 to 32), each of which holds ITEMS of its experts: lane q those with numbers q, q + P, ...
// The choices are made one after the other: the largest key among a lane's, then over the lanes; a tie goes to the lowest
// number.  Without a bias the key is the logit itself, which orders as the score does.  With one it is score + bias, and the
// definition is in 64 bits; what decides is computed in 32, and a token for which it decides by less than 32 bits can tell
// (kSure) is done again in 64: under one in a hundred of 256 experts whose logits are random.
template <int ITEMS, int P>
struct Shape {
    static constexpr int kNT = 128;
    static constexpr int kTokens = kNT / P;                      // of a CTA
    static constexpr int kExperts = ITEMS * P;                   // at most
    static constexpr int kChosen = kExperts < HL_MAX_TOP_K ? kExperts : HL_MAX_TOP_K;
};

// |score in 32 bits - score| < 2^-18: exp is off by 2 ulp and by its argument's rounding, |x| e^x 2^-24 < 2^-25, a sum of up to
// 32 + 5 of them one after the other by 37 * 2^-24 of it and theirs, the quotient by half an ulp; adding the bias rounds by 2^-24
// of the key.  So keys further apart than 2^-17 (1 + |key|) are in order, and sums of two than twice that.
constexpr float kSure = 0x1p-17f;

// numbers in the order of the floats (which have no NaN among them, and no -0)
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t u = __float_as_uint(v);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }

constexpr int kNobody = 0x7fffffff;

// The largest key over a token's lanes, and the lowest number that has it.
template <int P, typename Key>
__device__ __forceinline__ void largest(Key& key, int& e) {
    if constexpr (P == 32 && sizeof(Key) == 4) {
        const uint32_t u = ordered(key), all = __reduce_max_sync(0xffffffffu, u);
        e = (int)__reduce_min_sync(0xffffffffu, u == all ? (unsigned)e : (unsigned)kNobody);
        key = unordered(all);
    } else {
#pragma unroll
        for (int d = P / 2; d > 0; d >>= 1) {
            const Key k = __shfl_xor_sync(0xffffffffu, key, d);
            const int x = __shfl_xor_sync(0xffffffffu, e, d);
            if (k > key || (k == key && x < e)) {
                key = k;
                e = x;
            }
        }
    }
}
template <int P, typename V>
__device__ __forceinline__ V sum_of(V v) {
#pragma unroll
    for (int d = P / 2; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
template <int P>
__device__ __forceinline__ float max_of(float v) {
#pragma unroll
    for (int d = P / 2; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}

__device__ __forceinline__ float sigmoid(float l) { return 1.f / (1.f + expf(-l)); }
__device__ __forceinline__ double sigmoid(double l) { return 1.0 / (1.0 + exp(-l)); }
// e^(l - m) for l <= m, where both may be infinite
__device__ __forceinline__ float part(float l, float m) { return l == m ? 1.f : expf(l - m); }
__device__ __forceinline__ double part(double l, double m) { return l == m ? 1.0 : exp(l - m); }

// what a call goes by
struct Router {
    int top_k, E, G, per_group, top_groups;
    uint32_t group_magic;              // 2^21 / per_group, rounded up: exact for numbers and sizes of at most 1 024
    bool softmax, pair, renorm;
    __device__ __forceinline__ int group_of(int e) const { return (int)(((uint32_t)e * group_magic) >> 21); }
};
enum { kSoftmax = 1, kPair = 2, kRenorm = 4 };

// Keys of experts outside the groups that are kept become -inf.  `value` is what the groups are compared by, which is -inf for
// experts that cannot be chosen.  Returns whether it was clear which.
template <int ITEMS, int P, typename Key>
__device__ bool keep_groups(const Router& r, const Key (&value)[ITEMS], Key (&key)[ITEMS], int q, Key* s_value, Key* s_group,
                            Key* s_ranked) {
    const Key none = -(Key)INFINITY;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (j * P + q < r.E) s_value[j * P + q] = value[j];
    __syncwarp();
    for (int g = q; g < r.G; g += P) {
        Key best = none, second = none;
        int at = g % r.per_group;                                // (each lane begins elsewhere in its group, for the banks' sake)
        for (int i = 0; i < r.per_group; ++i) {
            const Key v = s_value[g * r.per_group + at];
            second = v > best ? best : v > second ? v : second;
            best = v > best ? v : best;
            if (++at == r.per_group) at = 0;
        }
        if (r.pair && second > none) best += second;
        s_group[g] = best;
    }
    __syncwarp();
    for (int g = q; g < r.G; g += P) {
        const Key v = s_group[g];
        int rank = 0;
        for (int i = 0; i < r.G; ++i) rank += s_group[i] > v || (s_group[i] == v && i < g);
        s_ranked[rank] = v;
        s_value[g] = rank < r.top_groups ? (Key)1 : (Key)0;      // (everybody has read the experts' values)
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (j * P + q < r.E && s_value[r.group_of(j * P + q)] == (Key)0) key[j] = none;
    bool clear = true;
    if (r.top_groups < r.G) {
        const Key in = s_ranked[r.top_groups - 1], out = s_ranked[r.top_groups];
        clear = out == none || in - out > (Key)(2 * kSure) * ((Key)1 + (in < 0 ? -in : in));
    }
    __syncwarp();
    return clear;
}

// The largest keys, in order: their experts go to s_e (-1: none left).  Where `check`, returns whether their order was clear;
// same(a, b): two experts whose keys are equal by definition.
template <int ITEMS, int P, typename Key, typename Same>
__device__ __forceinline__ bool choose(int top_k, Key (&key)[ITEMS], int q, bool check, int32_t* s_e, Same same) {
    const Key none = -(Key)INFINITY;
    bool clear = true;
    Key last = 0;
    int last_e = -1;
    for (int k = 0; k < top_k + (check ? 1 : 0); ++k) {
        Key best = key[0];
        int j_best = 0;
#pragma unroll
        for (int j = 1; j < ITEMS; ++j)
            if (key[j] > best) {
                best = key[j];
                j_best = j;
            }
        int e = j_best * P + q;
        largest<P>(best, e);
        const bool any = best > none;
        if (check && k > 0 && any && last_e >= 0 && !(last - best > (Key)kSure * ((Key)1 + (last < 0 ? -last : last))))
            clear = clear && same(last_e, e);
        last = best;
        last_e = any ? e : -1;
        if (k < top_k && q == 0) s_e[k] = last_e;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (e == j * P + q) key[j] = none;
    }
    return clear;
}

// Bound by its instructions where there are many tokens: a choice takes a lane some 3 ITEMS of them, and the warp two reductions.
template <typename T, int ITEMS, int P>
__global__ void __launch_bounds__(Shape<ITEMS, P>::kNT) k_expert_choose(const T* __restrict__ logits, int64_t ld,
                                                                        const float* __restrict__ bias, const int32_t* n_tokens,
                                                                        int64_t max_tokens, int top_k, int E, int G, int top_groups,
                                                                        int flags, float scale, int32_t* __restrict__ experts,
                                                                        float* __restrict__ weights, int32_t* status) {
    using S = Shape<ITEMS, P>;
    __shared__ int32_t s_chosen[S::kTokens][S::kChosen];
    extern __shared__ double s_base[];                           // with groups, of every token: [E] values, [2][G] groups
    const Router r{top_k, E, G, E / G, top_groups, ((1u << 21) + E / G - 1) / (unsigned)(E / G), (flags & kSoftmax) != 0,
                   (flags & kPair) != 0, (flags & kRenorm) != 0};
    const int q = threadIdx.x % P, mine = threadIdx.x / P;
    int64_t tokens = max_tokens;
    if (n_tokens) tokens = min((int64_t)max(__ldg(n_tokens), 0), max_tokens);
    const int64_t t = (int64_t)blockIdx.x * S::kTokens + mine;
    if (t - (int)(threadIdx.x & 31) / P >= tokens) return;                 // (a warp whose first token is behind the last)
    const bool live = t < tokens;
    const T* row = logits + (live ? t : tokens - 1) * ld;
    int32_t* s_e = s_chosen[mine];
    double* s_value = s_base + mine * (E + 2 * G);
    float* s_value32 = reinterpret_cast<float*>(s_value);
    const float none = -INFINITY;

    float l[ITEMS];
    bool bad = false;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) l[j] = j * P + q < E ? as_float(row[j * P + q]) + 0.f : none;     // (-0 becomes +0)
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (l[j] != l[j]) {
            bad = true;
            l[j] = none;
        }
    // of all scores, where they are needed: the largest logit and the sum of e^(l - largest)
    const bool scores = bias || (G > 1 && r.pair);
    float top = none, z = 1.f;
    if (r.softmax && (scores || !r.renorm)) {
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) top = fmaxf(top, l[j]);
        top = max_of<P>(top);
        z = 0.f;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) z += l[j] > none ? part(l[j], top) : 0.f;
        z = sum_of<P>(z);
    }
    bool clear = true;
    {
        float key[ITEMS];
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) key[j] = l[j];
        if (scores) {
            float value[ITEMS];
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) {
                value[j] = none;
                if (l[j] > none) {
                    value[j] = r.softmax ? part(l[j], top) / z : sigmoid(l[j]);
                    if (bias) {
                        value[j] += __ldg(&bias[j * P + q]) + 0.f;
                        if (value[j] != value[j]) {
                            bad = true;
                            value[j] = none;
                        }
                        key[j] = value[j];
                    }
                }
            }
            if (G > 1)
                clear = keep_groups<ITEMS, P>(r, value, key, q, s_value32, s_value32 + E, s_value32 + E + G);
        } else if (G > 1) {
            keep_groups<ITEMS, P>(r, l, key, q, s_value32, s_value32 + E, s_value32 + E + G);
        }
        clear &= choose<ITEMS, P>(top_k, key, q, bias != nullptr, s_e, [&](int a, int b) {
            return as_float(row[a]) == as_float(row[b]) && __ldg(&bias[a]) == __ldg(&bias[b]);
        });
    }
    if (__any_sync(0xffffffffu, scores && live && !clear)) {     // (all tokens of the warp once more)
        const double none64 = -(double)INFINITY;
        double key[ITEMS], z64 = 0.0;
        if (r.softmax) {
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) z64 += l[j] > none ? part((double)l[j], (double)top) : 0.0;
            z64 = sum_of<P>(z64);
        }
        double value[ITEMS];
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            key[j] = value[j] = none64;
            if (l[j] > none) {
                value[j] = r.softmax ? part((double)l[j], (double)top) / z64 : sigmoid((double)l[j]);
                if (bias) {
                    value[j] += (double)__ldg(&bias[j * P + q]);
                    if (value[j] != value[j]) value[j] = none64;
                }
                key[j] = bias ? value[j] : (double)l[j];
            }
        }
        __syncwarp();
        if (G > 1) keep_groups<ITEMS, P>(r, value, key, q, s_value, s_value + E, s_value + E + G);
        choose<ITEMS, P>(top_k, key, q, false, s_e, [](int, int) { return true; });
    }
    if (status && __any_sync(0xffffffffu, bad && live) && (threadIdx.x & 31) == 0) set_status(status, HL_EINVAL);
    __syncwarp();

    // Weights.  With the sum of the chosen scores below, only their ratios count: all are taken relative to e^m, m the largest of
    // the logits, so that none is lost to underflow (of sigmoids: min(m, 0), as that of a positive logit is 1/2 and more).
    float m = none, sum = 0.f;
    for (int k = q; k < top_k; k += P)
        if (s_e[k] >= 0) m = fmaxf(m, as_float(row[s_e[k]]) + 0.f);
    m = max_of<P>(m);
    if (!r.softmax) m = r.renorm ? fminf(m, 0.f) : 0.f;
    else if (!r.renorm) m = top;
    const auto weight = [&](float x) {
        if (r.softmax) return part(x, m);
        return x > 0.f ? sigmoid(x) : part(x, m) / (1.f + expf(x));
    };
    if (r.renorm) {
        for (int k = q; k < top_k; k += P)
            if (s_e[k] >= 0) sum += weight(as_float(row[s_e[k]]) + 0.f);
        sum = sum_of<P>(sum);
    } else {
        sum = r.softmax ? z : 1.f;
    }
    if (!live) return;
    for (int k = q; k < top_k; k += P) {
        const int e = s_e[k];
        experts[t * top_k + k] = e;
        weights[t * top_k + k] = e < 0 ? 0.f : scale * (weight(as_float(row[e]) + 0.f) / sum);
    }
}

// ---- the logits' gradient -----------------------------------------------------------------------------------------------
// Of the scores' sum over a token only what the chosen experts contribute depends on k: every expert's gradient is
// -c * score of it (softmax without the sum of the chosen below; 0 otherwise), the chosen ones' are written over it.  Bound by
// writing the rows.
template <typename T, int ITEMS, int P>
__global__ void __launch_bounds__(Shape<ITEMS, P>::kNT) k_expert_choose_bwd(const T* __restrict__ logits, int64_t ld,
                                                                            const int32_t* n_tokens, int64_t max_tokens, int top_k,
                                                                            int E, int flags, float scale,
                                                                            const int32_t* __restrict__ experts,
                                                                            const float* __restrict__ grad_w, T* __restrict__ grad,
                                                                            int64_t ld_grad) {
    using S = Shape<ITEMS, P>;
    __shared__ int32_t s_chosen[S::kTokens][S::kChosen];
    __shared__ float s_grad[S::kTokens][S::kChosen];
    const bool softmax = flags & kSoftmax, renorm = flags & kRenorm;
    const int q = threadIdx.x % P, mine = threadIdx.x / P;
    int64_t tokens = max_tokens;
    if (n_tokens) tokens = min((int64_t)max(__ldg(n_tokens), 0), max_tokens);
    const int64_t t = (int64_t)blockIdx.x * S::kTokens + mine;
    if (t - (int)(threadIdx.x & 31) / P >= tokens) return;
    const bool live = t < tokens;
    const int64_t at = live ? t : tokens - 1;
    const T* row = logits + at * ld;
    const float none = -INFINITY;
    const auto logit = [&](int e) {
        const float x = as_float(row[e]) + 0.f;
        return x != x ? none : x;
    };

    float l[ITEMS], top = none, z = 1.f;
    if (softmax && !renorm) {
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) l[j] = j * P + q < E ? logit(j * P + q) : none;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) top = fmaxf(top, l[j]);
        top = max_of<P>(top);
        z = 0.f;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) z += l[j] > none ? part(l[j], top) : 0.f;
        z = sum_of<P>(z);
    }
    // the chosen: their scores (relative, as above), and sums over them
    float m = none;
    for (int k = q; k < top_k; k += P) {
        const int e = __ldg(&experts[at * top_k + k]);
        s_chosen[mine][k] = (unsigned)e < (unsigned)E ? e : -1;
        if ((unsigned)e < (unsigned)E) m = fmaxf(m, logit(e));
    }
    m = max_of<P>(m);
    if (!softmax) m = renorm ? fminf(m, 0.f) : 0.f;
    else if (!renorm) m = top;
    const auto score = [&](float x) {
        if (x == none) return 0.f;
        if (softmax) return part(x, m);
        return x > 0.f ? sigmoid(x) : part(x, m) / (1.f + expf(x));
    };
    float sum = 0.f, dot = 0.f;
    for (int k = q; k < top_k; k += P) {
        const int e = s_chosen[mine][k];
        if (e < 0) continue;
        const float s = score(logit(e));
        sum += s;
        dot += s * __ldg(&grad_w[at * top_k + k]);
    }
    sum = sum_of<P>(sum);
    dot = sum_of<P>(dot);
    if (!renorm) sum = softmax ? z : 1.f;
    const float mean = renorm || softmax ? dot / sum : 0.f;
    // d/dl of the weights: scale * share * (grad - mean), times 1 - score for sigmoids
    for (int k = q; k < top_k; k += P) {
        const int e = s_chosen[mine][k];
        float g = 0.f;
        if (e >= 0) {
            const float x = logit(e), share = sum > 0.f ? score(x) / sum : 0.f;
            g = scale * share * (__ldg(&grad_w[at * top_k + k]) - mean);
            if (!softmax) g *= 1.f / (1.f + expf(x));            // 1 - sigmoid(x)
        }
        s_grad[mine][k] = g;
    }
    if (!live) return;
    T* out = grad + t * ld_grad;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (j * P + q < E) {
            float g = 0.f;
            if (softmax && !renorm && l[j] > none) g = -scale * (part(l[j], top) / z) * mean;
            out[j * P + q] = from_float<T>(g);
        }
    __syncwarp();
    for (int k = q; k < top_k; k += P) {
        const int e = s_chosen[mine][k];
        if (e < 0) continue;
        float g = 0.f;                                           // (an expert that is there twice gets the sum)
        for (int i = 0; i < top_k; ++i) g += s_chosen[mine][i] == e ? s_grad[mine][i] : 0.f;
        out[e] = from_float<T>(g);
    }
}

// ---- arguments ------------------------------------------------------------------------------------------------------------
bool router_ok(const hl_router* r) {
    return r && (r->score == HL_SCORE_SOFTMAX || r->score == HL_SCORE_SIGMOID) && r->n_experts >= 1 && r->n_experts <= HL_MAX_EXPERTS &&
           r->top_k >= 1 && r->top_k <= HL_MAX_TOP_K && r->top_k <= r->n_experts && r->n_groups >= 1 && r->n_groups <= HL_MAX_GROUPS &&
           r->n_experts % r->n_groups == 0 && r->top_groups >= 1 && r->top_groups <= r->n_groups &&
           r->top_k <= r->n_experts / r->n_groups * r->top_groups &&
           (r->group_score == HL_GROUP_MAX || r->group_score == HL_GROUP_TOP2) && (r->renorm == 0 || r->renorm == 1) &&
           isfinite(r->scale);
}
bool tokens_ok(const hl_router* r, int32_t dtype, const void* logits, int64_t ld, int64_t max_tokens, const int32_t* n_tokens) {
    return dtype_size(dtype) && max_tokens >= 0 && max_tokens * r->top_k < (int64_t(1) << 30) && max_tokens < (int64_t(1) << 30) &&
           ld >= r->n_experts && ld < (int64_t(1) << 31) && (logits || max_tokens == 0) && lies_at(logits, dtype_size(dtype)) &&
           lies_at(n_tokens, 4);
}
int flags_of(const hl_router* r) {
    return (r->score == HL_SCORE_SOFTMAX ? kSoftmax : 0) | (r->group_score == HL_GROUP_TOP2 ? kPair : 0) | (r->renorm ? kRenorm : 0);
}

// As few lanes a token as hold its experts, eight a lane; above 256 experts more.
#define HL_SHAPES(E, RUN)                                                                                             \
    ((E) <= 8 ? RUN(8, 1) : (E) <= 16 ? RUN(8, 2) : (E) <= 32 ? RUN(8, 4) : (E) <= 64 ? RUN(8, 8) : (E) <= 128 ? RUN(8, 16) \
     : (E) <= 256 ? RUN(8, 32) : (E) <= 512 ? RUN(16, 32) : RUN(32, 32))

template <typename T>
int32_t launch_choose(const hl_router* r, const void* logits, int64_t ld, const float* bias, int64_t max_tokens,
                      const int32_t* n_tokens, int32_t* experts, float* weights, int32_t* status, cudaStream_t stream) {
#define HL_RUN(ITEMS, P)                                                                                                      \
    launch_cluster(k_expert_choose<T, ITEMS, P>, (unsigned)div_up(max_tokens, Shape<ITEMS, P>::kTokens), Shape<ITEMS, P>::kNT, \
                   r->n_groups > 1 ? Shape<ITEMS, P>::kTokens * (r->n_experts + 2 * r->n_groups) * sizeof(double) : 0, 0,      \
                   stream, static_cast<const T*>(logits), ld, bias, n_tokens, max_tokens, r->top_k, r->n_experts, r->n_groups, \
                   r->top_groups, flags_of(r), r->scale, experts, weights, status)
    HL_CUDA_TRY(HL_SHAPES(r->n_experts, HL_RUN));
#undef HL_RUN
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}
template <typename T>
int32_t launch_choose_bwd(const hl_router* r, const void* logits, int64_t ld, int64_t max_tokens, const int32_t* n_tokens,
                          const int32_t* experts, const float* grad_w, void* grad, int64_t ld_grad, cudaStream_t stream) {
#define HL_RUN(ITEMS, P)                                                                                                          \
    launch(k_expert_choose_bwd<T, ITEMS, P>, (unsigned)div_up(max_tokens, Shape<ITEMS, P>::kTokens), Shape<ITEMS, P>::kNT, stream, \
           static_cast<const T*>(logits), ld, n_tokens, max_tokens, r->top_k, r->n_experts, flags_of(r), r->scale, experts, grad_w, \
           static_cast<T*>(grad), ld_grad)
    HL_CUDA_TRY(HL_SHAPES(r->n_experts, HL_RUN));
#undef HL_RUN
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}

}  // namespace
}  // namespace hl

using namespace hl;

extern "C" int32_t hl_expert_choose(const hl_router* router, int32_t dtype, const void* d_logits, int64_t ld, const float* d_bias,
                                    int64_t max_tokens, const int32_t* d_n_tokens, int32_t* d_experts, float* d_weights,
                                    int32_t* d_status, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!router_ok(router) || !tokens_ok(router, dtype, d_logits, ld, max_tokens, d_n_tokens) || !lies_at(d_bias, 4) ||
        !lies_at(d_experts, 4) || !lies_at(d_weights, 4) || !lies_at(d_status, 4) || (max_tokens > 0 && (!d_experts || !d_weights)))
        return HL_EINVAL;
    if (max_tokens == 0) return HL_OK;
#define HL_CHOOSE(T) launch_choose<T>(router, d_logits, ld, d_bias, max_tokens, d_n_tokens, d_experts, d_weights, d_status, stream)
    return dtype == HL_F32 ? HL_CHOOSE(float) : dtype == HL_BF16 ? HL_CHOOSE(__nv_bfloat16) : HL_CHOOSE(__half);
#undef HL_CHOOSE
}

extern "C" int32_t hl_expert_choose_bwd(const hl_router* router, int32_t dtype, const void* d_logits, int64_t ld, int64_t max_tokens,
                                        const int32_t* d_n_tokens, const int32_t* d_experts, const float* d_grad_weights,
                                        void* d_grad_logits, int64_t ld_grad, void* stream_) {
    const cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!router_ok(router) || !tokens_ok(router, dtype, d_logits, ld, max_tokens, d_n_tokens) || !lies_at(d_experts, 4) ||
        !lies_at(d_grad_weights, 4) || !lies_at(d_grad_logits, dtype_size(dtype)) || ld_grad < router->n_experts ||
        ld_grad >= (int64_t(1) << 31) || (max_tokens > 0 && (!d_experts || !d_grad_weights || !d_grad_logits)))
        return HL_EINVAL;
    if (max_tokens == 0) return HL_OK;
#define HL_CHOOSE_BWD(T) \
    launch_choose_bwd<T>(router, d_logits, ld, max_tokens, d_n_tokens, d_experts, d_grad_weights, d_grad_logits, ld_grad, stream)
    return dtype == HL_F32 ? HL_CHOOSE_BWD(float) : dtype == HL_BF16 ? HL_CHOOSE_BWD(__nv_bfloat16) : HL_CHOOSE_BWD(__half);
#undef HL_CHOOSE_BWD
}
