// Routing to experts: the router's logits become the chosen experts and their weights, and the weights' gradient the logits'.
#include <math.h>

#include "hl_rows.cuh"

namespace hl {
namespace {

// ---- who is chosen ----------------------------------------------------------------------------------------------------
// A token has P lanes of a warp (1 to 32), each of which holds up to ITEMS of its experts side by side: `per_lane`, so that a group is
// that of whole lanes if that can be.  Without a bias an expert's key is
// its logit, which orders as the score does.  With one it is score + bias, and the definition is in 64 bits; what decides is
// computed in 32, and a token for which 32 bits cannot tell is done again in 64: one or two in a thousand of 256 experts whose
// logits are random.
template <int ITEMS, int P>
struct Shape {
    static constexpr int kNT = 128, kCtas = ITEMS == 8 ? 8 : ITEMS == 16 ? 5 : 1;       // threads; CTAs of a multiprocessor
    static constexpr int kTokens = kNT / P;                      // of a CTA
    static constexpr int kExperts = ITEMS * P;                   // at most
    static constexpr int kChosen = kExperts < HL_MAX_TOP_K ? kExperts : HL_MAX_TOP_K;
};

// How far scores of 32 bits may be off, in steps of 2^-24.  A sigmoid s: s (1 - s) times the relative error of the exponential -- 4 of
// the instruction's, and its argument's roundings, 1.5 |x|, where s (1 - s) |x| < 0.23 --, 1 for the sum and 2 for the inverse:
// less than 4.5.  A softmax: s times the exponential's 4 + 2 |x|, where s |x| < 0.37, the same of the sum's terms on average
// (less than 4 + 14), up to 32 + 5 roundings of the sum and 2 of the inverse: less than 61 s + 1, and s is at most 1 / z, z the sum of
// e^(x - largest).  Adding the bias rounds by 1 of the key.  So keys further apart than twice that, times 1 + |key| with room for the
// rounding, are in order, and sums of two than four times.
constexpr float kSureSigmoid = 0x1p-20f;
__device__ __forceinline__ float sure_of_softmax(float z) { return 0x1p-23f * (64.f / z + 2.f); }

// numbers in the order of the floats (which have no NaN among them; -0 is 0)
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t u = __float_as_uint(v + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }

constexpr int kNobody = 0x7fffffff;
constexpr unsigned kAll = 0xffffffffu;

// The largest key over a token's lanes, and the lowest number that has it.
template <int P, typename Key>
__device__ __forceinline__ void largest(Key& key, int& e) {
    if constexpr (P == 32 && sizeof(Key) == 4) {
        const uint32_t u = ordered(key), all = __reduce_max_sync(kAll, u);
        e = (int)__reduce_min_sync(kAll, u == all ? (unsigned)e : (unsigned)kNobody);
        key = unordered(all);
    } else {
#pragma unroll
        for (int d = P / 2; d > 0; d >>= 1) {
            const Key k = __shfl_xor_sync(kAll, key, d);
            const int x = __shfl_xor_sync(kAll, e, d);
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
    for (int d = P / 2; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
    return v;
}
template <int P>
__device__ __forceinline__ float max_of(float v) {
#pragma unroll
    for (int d = P / 2; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, d));
    return v;
}
// a token's lanes among the warp's, as a mask
template <int P>
__device__ __forceinline__ unsigned lanes_of(int lane) { return P == 32 ? kAll : ((1u << (P & 31)) - 1u) << (lane & ~(P - 1) & 31); }

__device__ __forceinline__ double sigmoid(double l) { return 1.0 / (1.0 + exp(-l)); }
// e^(l - m) for l <= m, where both may be infinite
__device__ __forceinline__ float part(float l, float m) { return l == m ? 1.f : expf(l - m); }
__device__ __forceinline__ double part(double l, double m) { return l == m ? 1.0 : exp(l - m); }
// the same, as exact as choosing needs it: 2^x and 1 / x as the hardware has them
__device__ __forceinline__ float near_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float near_inverse(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float near_sigmoid(float l) { return near_inverse(1.f + near_exp2(-kLog2e * l)); }

// what a call goes by
struct Router {
    int top_k, E, G, per_group, top_groups, per_lane;
    int group_lanes;                   // lanes of a group; 0: groups are not of whole lanes
    uint32_t group_magic;              // 2^21 / per_group, rounded up: exact for numbers and sizes of at most 1 024
    float sure;                        // how far keys have to be apart (in 32 bits)
    bool softmax, pair, renorm;
    __device__ __forceinline__ int group_of(int e) const { return (int)(((uint32_t)e * group_magic) >> 21); }
};
enum { kSoftmax = 1, kPair = 2, kRenorm = 4 };

template <typename Key>
__device__ __forceinline__ void two_best(Key v, Key& best, Key& second) {
    if constexpr (sizeof(Key) == 4) {
        second = fmaxf(second, fminf(best, v));
        best = fmaxf(best, v);
    } else {
        second = fmax(second, fmin(best, v));
        best = fmax(best, v);
    }
}

// The sum of a group's two best.  Of numbers it may be below the lowest of 32 bits, and -inf would say that nobody can be chosen there: the
// lowest itself, then, as any other such sum, and who comes first is not clear.  (Above the largest, infinities are not clear either.)
template <typename Key>
__device__ __forceinline__ Key both(Key best, Key second) {
    if constexpr (sizeof(Key) == 4) return fmaxf(best + second, -3.402823466e38f);
    else return best + second;
}

// Keys of experts outside the groups that are kept become -inf.  `value` is what the groups are compared by, which is -inf for
// experts that cannot be chosen.  Returns whether it was clear which.  Groups of whole lanes find their two best between those;
// others go through shared memory (s: [E + 2 G]).
template <int ITEMS, int P, typename Key>
__device__ bool keep_groups(const Router& r, const Key (&value)[ITEMS], Key (&key)[ITEMS], int q, Key* s) {
    const Key none = -(Key)INFINITY;
    Key in = none, out = none;
    if (r.group_lanes) {
        const int lanes = r.group_lanes, lane = threadIdx.x & 31, first = lane & ~(P - 1), mine = q / lanes;
        Key best = none, second = none;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) two_best(value[j], best, second);
        const Key my_best = best, my_second = second;
        const int from = first + min(mine, r.G - 1) * lanes;
        for (int d = 1, at = q - mine * lanes; d < lanes; ++d) {         // (the group's other lanes, one after the other)
            at = at + 1 < lanes ? at + 1 : 0;
            const Key b = __shfl_sync(kAll, my_best, from + at), c = __shfl_sync(kAll, my_second, from + at);
            two_best(b, best, second);
            second = c > second ? c : second;
        }
        if (r.pair && second > none) best = both(best, second);
        int rank = 0;
#pragma unroll 4
        for (int g = 0; g < r.G; ++g) {
            const Key v = __shfl_sync(kAll, best, first + g * lanes);
            rank += g < mine ? v >= best : v > best;
        }
        if (rank >= r.top_groups) {
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) key[j] = none;
        }
        if (r.top_groups < r.G) {
            const unsigned us = lanes_of<P>(lane);
            const unsigned i = __ballot_sync(kAll, rank == r.top_groups - 1) & us, o = __ballot_sync(kAll, rank == r.top_groups) & us;
            in = __shfl_sync(kAll, best, __ffs(i) - 1);
            out = __shfl_sync(kAll, best, __ffs(o) - 1);
        }
    } else {
        Key *s_group = s + r.E, *s_ranked = s_group + r.G;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (j < r.per_lane && q * r.per_lane + j < r.E) s[q * r.per_lane + j] = value[j];
        __syncwarp();
        for (int g = q; g < r.G; g += P) {
            Key best = none, second = none;
            int at = g % r.per_group;                            // (each lane begins elsewhere in its group, for the banks' sake)
            for (int i = 0; i < r.per_group; ++i) {
                two_best(s[g * r.per_group + at], best, second);
                if (++at == r.per_group) at = 0;
            }
            if (r.pair && second > none) best = both(best, second);
            s_group[g] = best;
        }
        __syncwarp();
        for (int g = q; g < r.G; g += P) {
            const Key v = s_group[g];
            int rank = 0;
            for (int i = 0; i < r.G; ++i) rank += s_group[i] > v || (s_group[i] == v && i < g);
            s_ranked[rank] = v;
            s[g] = rank < r.top_groups ? (Key)1 : (Key)0;        // (everybody has read the experts' values)
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (j < r.per_lane && q * r.per_lane + j < r.E && s[r.group_of(q * r.per_lane + j)] == (Key)0) key[j] = none;
        if (r.top_groups < r.G) {
            in = s_ranked[r.top_groups - 1];
            out = s_ranked[r.top_groups];
        }
        __syncwarp();
    }
    return out == none || in - out > (Key)(2 * r.sure) * ((Key)1 + (in < 0 ? -in : in));
}

// Whether keys a >= b are in order for certain; a NaN (of infinite keys) says no.
template <typename Key>
__device__ __forceinline__ bool surely(Key a, Key b, float sure) { return a - b > (Key)sure * ((Key)1 + (a < 0 ? -a : a)); }

// The largest keys, in order: their experts go to s_e (-1: none left), one after the other -- the largest of a lane's, then over the
// lanes; a tie goes to the lowest number.  Where `check`, returns whether their order was clear; same(a, b): two experts whose
// keys are equal by definition.
template <int ITEMS, int P, typename Key, typename Same>
__device__ __forceinline__ bool choose(int top_k, Key (&key)[ITEMS], int e0, int q, bool check, float sure, int32_t* s_e, Same same) {
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
        int e = e0 + j_best;
        largest<P>(best, e);
        const bool any = best > none;
        if (check && k > 0 && any && last_e >= 0 && !surely(last, best, sure)) clear = clear && same(last_e, e);
        last = best;
        last_e = any ? e : -1;
        if (k < top_k && q == 0) s_e[k] = last_e;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (e == e0 + j) key[j] = none;                      // (behind the lane's own: -inf already)
    }
    return clear;
}

// v over a token's lanes, in descending order
template <int P>
__device__ __forceinline__ float in_descending_order(float v, int q) {
#pragma unroll
    for (int size = 2; size <= P; size *= 2)
#pragma unroll
        for (int d = size / 2; d > 0; d /= 2) {
            const float other = __shfl_xor_sync(kAll, v, d);
            const bool upper = ((q & d) != 0) != ((q & size) != 0 && size < P);
            v = upper ? fminf(v, other) : fmaxf(v, other);
        }
    return v;
}

// The same, all at once, for top_k < P: top_k + 1 keys are known that are among the largest of eight side by side, and what is below the
// least of them does not count.  Those few that do, a lane each, are ranked by comparing each with all.  Returns false, with nothing
// done, if there are more than P of them (equal keys, or few lanes with any).
template <int ITEMS, int P, typename Same>
__device__ __forceinline__ bool choose_few(int top_k, const float (&key)[ITEMS], int e0, int q, bool check, float sure, int32_t* s_e, float2* s_few,
                                           bool* clear, Same same) {
    const float none = -INFINITY;
    const int lane = threadIdx.x & 31, first = lane & ~(P - 1);
    float least;
    if constexpr (ITEMS == 16) {
        // of a lane's two largest of eight, the larger ones h and the smaller ones l of all lanes, each in order: i of l's first and
        // top_k + 1 - i of h's first are top_k + 1 keys, whatever i is
        float a = key[0], b = key[8];
#pragma unroll
        for (int j = 1; j < 8; ++j) {
            a = fmaxf(a, key[j]);
            b = fmaxf(b, key[8 + j]);
        }
        const float h = in_descending_order<P>(fmaxf(a, b), q), l = in_descending_order<P>(fminf(a, b), q);
        const float other = __shfl_sync(kAll, h, first + max(top_k - 1 - q, 0));
        least = max_of<P>(q < top_k ? fminf(l, other) : q == top_k ? h : none);
    } else {
        float best = key[0];
#pragma unroll
        for (int j = 1; j < ITEMS; ++j) best = fmaxf(best, key[j]);
        best = in_descending_order<P>(best, q);
        least = __shfl_sync(kAll, best, first + top_k);
    }
    least = fmaxf(least, -3.402823466e38f);                      // (not those that cannot be chosen)
    int mine = 0;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) mine += key[j] >= least;
    int at = mine;
#pragma unroll
    for (int d = 1; d < P; d *= 2) {
        const int v = __shfl_up_sync(kAll, at, d, P);
        if (q >= d) at += v;
    }
    const int few = __shfl_sync(kAll, at, first + P - 1);
    if (__any_sync(kAll, few > P)) return false;
    at -= mine;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (key[j] >= least) s_few[at++] = make_float2(key[j], __int_as_float(e0 + j));
    __syncwarp();
    float2 me = make_float2(none, __int_as_float(-1));
    if (q < few) me = s_few[q];
    int rank = 0;                      // (they lie in the order of their numbers)
    const int most = P == 32 ? few : (int)__reduce_max_sync(kAll, (unsigned)few);
#pragma unroll 4
    for (int i = 0; i < most; ++i) {
        const float v = __shfl_sync(kAll, me.x, first + i);
        rank += i < q ? v >= me.x : v > me.x;
    }
    if (q < few && rank < top_k) s_e[rank] = __float_as_int(me.y);
    if (q >= few && q < top_k) s_e[q] = -1;
    if (check) {
        __syncwarp();
        if (q < few) s_few[rank] = me;
        __syncwarp();
        bool mine_clear = true;
        if (q > 0 && q < few && q <= top_k) {
            const float2 a = s_few[q - 1], b = s_few[q];
            if (!surely(a.x, b.x, sure)) mine_clear = same(__float_as_int(a.y), __float_as_int(b.y));
        }
        *clear = (__ballot_sync(kAll, !mine_clear) & lanes_of<P>(lane)) == 0;
    }
    return true;
}

// Bound by its instructions where there are many tokens: 65 536 tokens, 8 of 256 experts in 8 groups, sigmoids with a bias: 70 us, 34 MB
// that memory gives in 6; an instruction is issued in two of three cycles.  Of that some 15 the rows and what is done once a
// token, 8 scores and bias, 15 the groups, 20 the choice, 8 the weights.  WHOLE: rows are read in pieces of 16 bytes.
template <typename T, int ITEMS, int P, bool WHOLE>
__global__ void __launch_bounds__(Shape<ITEMS, P>::kNT, Shape<ITEMS, P>::kCtas) k_expert_choose(const T* __restrict__ logits, int64_t ld,
                                                                        const float* __restrict__ bias, const int32_t* n_tokens,
                                                                        int64_t max_tokens, int top_k, int E, int G, int per_group,
                                                                        unsigned group_magic, int top_groups, int per_lane,
                                                                        int group_lanes, int flags,
                                                                        float scale, int32_t* __restrict__ experts,
                                                                        float* __restrict__ weights, int32_t* status) {
    using S = Shape<ITEMS, P>;
    __shared__ int32_t s_chosen[S::kTokens][S::kChosen];
    __shared__ float2 s_few[P >= 16 ? S::kNT : 1];
    extern __shared__ double s_base[];                           // with groups that are not whole lanes', of every token: [E + 2 G]
    Router r{top_k, E, G, per_group, top_groups, per_lane, group_lanes, group_magic, kSureSigmoid, (flags & kSoftmax) != 0, (flags & kPair) != 0, (flags & kRenorm) != 0};
    const int q = threadIdx.x % P, mine = threadIdx.x / P;
    int64_t tokens = max_tokens;
    if (n_tokens) tokens = min((int64_t)max(__ldg(n_tokens), 0), max_tokens);
    const int64_t t = (int64_t)blockIdx.x * S::kTokens + mine;
    if (t - (int)(threadIdx.x & 31) / P >= tokens) return;                 // (a warp whose first token is behind the last)
    const bool live = t < tokens;
    const T* row = logits + (live ? t : tokens - 1) * ld;
    int32_t* s_e = s_chosen[mine];
    double* s_value = s_base + (group_lanes ? 0 : mine * (E + 2 * G));
    float* s_value32 = reinterpret_cast<float*>(s_value);
    const float none = -INFINITY;
    const int e0 = q * per_lane, e1 = min(e0 + per_lane, E);     // the lane's experts

    float l[ITEMS], any_nan = 0.f;                               // (0 * an infinity makes a NaN, too)
    bool bad = false;
    if constexpr (WHOLE) {
        constexpr int N = 16 / sizeof(T);
        Pack<T, N> in[ITEMS / N];
#pragma unroll
        for (int i = 0; i < ITEMS / N; ++i) {
            in[i].zero();
            if (e0 + i * N < e1) in[i].load(row + e0 + i * N);
        }
#pragma unroll
        for (int i = 0; i < ITEMS / N; ++i) {
            float x[N];
            in[i].get(x);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                any_nan = fmaf(x[k], 0.f, any_nan);
                l[i * N + k] = e0 + i * N < e1 ? x[k] : none;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            const float x = e0 + j < e1 ? as_float(row[e0 + j]) : 0.f;
            any_nan = fmaf(x, 0.f, any_nan);
            l[j] = e0 + j < e1 ? x : none;
        }
    }
    if (any_nan != 0.f) {
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (l[j] != l[j]) {
                bad = true;
                l[j] = none;
            }
    }
    // Of all scores, where they are needed: the largest logit and the sum of e^(l - largest), as exact as choosing needs it.  The weights
    // of a softmax over all are divided by the same sum: the largest error of 65 536 tokens, 8 of 256, was 4.9 steps of 2^-24, with expf
    // here 4.3 (43 us instead of 40; 44 instead of 42 for 32 000, 8 of 500).
    const bool scores = bias || (G > 1 && r.pair);
    float top = none, z = 1.f, value[ITEMS];
    if (r.softmax && (scores || !r.renorm)) {
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) top = fmaxf(top, l[j]);
        top = max_of<P>(top);
        z = 0.f;
        if (fabsf(top) < INFINITY) {
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) value[j] = near_exp2(kLog2e * (l[j] - top));      // (0 of -inf)
        } else {
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) value[j] = l[j] > none && l[j] == top ? 1.f : 0.f;
        }
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) z += value[j];
        z = sum_of<P>(z);
        r.sure = sure_of_softmax(z);
    }
    bool clear = true;
    {
        float key[ITEMS];
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) key[j] = l[j];
        if (scores) {
            if (r.softmax) {
                const float per = near_inverse(z);
#pragma unroll
                for (int j = 0; j < ITEMS; ++j) value[j] *= per;
            } else {
#pragma unroll
                for (int j = 0; j < ITEMS; ++j) value[j] = near_sigmoid(l[j]);
            }
            if (bias) {
                if constexpr (WHOLE) {
#pragma unroll
                    for (int i = 0; i < ITEMS / 4; ++i) {
                        Pack<float, 4> in;
                        float x[4];
                        in.zero();
                        if (e0 + i * 4 < e1) in.load(bias + e0 + i * 4);
                        in.get(x);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            value[4 * i + k] += x[k];
                            bad = bad || x[k] != x[k];
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < ITEMS; ++j) {
                        const float x = e0 + j < e1 ? __ldg(&bias[e0 + j]) : 0.f;
                        value[j] += x;
                        bad = bad || x != x;
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) {
                const bool there = l[j] > none;
                value[j] = there && value[j] == value[j] ? value[j] : none;
                if (bias) key[j] = value[j];
            }
            if (G > 1) clear = keep_groups<ITEMS, P>(r, value, key, q, s_value32);
        } else if (G > 1) {
            keep_groups<ITEMS, P>(r, l, key, q, s_value32);
        }
        const auto same = [&](int a, int b) { return as_float(row[a]) == as_float(row[b]) && __ldg(&bias[a]) == __ldg(&bias[b]); };
        const bool check = bias != nullptr;
        bool done = false, in_order = true;
        if constexpr (P >= 16)
            if (top_k < P) done = choose_few<ITEMS, P>(top_k, key, e0, q, check, r.sure, s_e, s_few + mine * P, &in_order, same);
        if (!done) in_order = choose<ITEMS, P>(top_k, key, e0, q, check, r.sure, s_e, same);
        clear = clear && in_order;
    }
    if (__any_sync(kAll, scores && live && !clear)) {            // (all tokens of the warp once more)
        const double none64 = -(double)INFINITY;
        double key[ITEMS], value[ITEMS], z64 = 0.0;
        if (r.softmax) {
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) z64 += l[j] > none ? part((double)l[j], (double)top) : 0.0;
            z64 = sum_of<P>(z64);
        }
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            key[j] = value[j] = none64;
            if (l[j] > none) {
                value[j] = r.softmax ? part((double)l[j], (double)top) / z64 : sigmoid((double)l[j]);
                if (bias) {
                    value[j] += (double)__ldg(&bias[e0 + j]);
                    if (value[j] != value[j]) value[j] = none64;
                }
                key[j] = bias ? value[j] : (double)l[j];
            }
        }
        __syncwarp();
        if (G > 1) keep_groups<ITEMS, P>(r, value, key, q, s_value);
        choose<ITEMS, P>(top_k, key, e0, q, false, 0.f, s_e, [](int, int) { return true; });
    }
    if (status && __any_sync(kAll, bad && live) && (threadIdx.x & 31) == 0) set_status(status, HL_EINVAL);
    __syncwarp();

    // Weights.  With the sum of the chosen scores below, only their ratios count: all are taken relative to e^m, m the largest of
    // the logits, so that none is lost to underflow (of sigmoids: min(m, 0), as that of a positive logit is 1/2 and more).
    float m = none, sum = 0.f, mine_x = none, mine_w = 0.f;      // (of the lane's first choice, which is all it has as a rule)
    for (int k = q; k < top_k; k += P) {
        const float x = s_e[k] >= 0 ? as_float(row[s_e[k]]) : none;
        if (k == q) mine_x = x;
        m = fmaxf(m, x);
    }
    m = max_of<P>(m);
    if (!r.softmax) m = r.renorm ? fminf(m, 0.f) : 0.f;
    else if (!r.renorm) m = top;
    const auto weight = [&](float x) {
        if (r.softmax) return part(x, m);
        const float e = expf(x > 0.f ? -x : x);
        return (x > 0.f ? 1.f : m == 0.f ? e : part(x, m)) / (1.f + e);
    };
    if (mine_x > none) mine_w = weight(mine_x);
    if (r.renorm) {
        sum = mine_w;
        for (int k = q + P; k < top_k; k += P)
            if (s_e[k] >= 0) sum += weight(as_float(row[s_e[k]]));
        sum = sum_of<P>(sum);
    } else {
        sum = r.softmax ? z : 1.f;
    }
    if (!live) return;
    for (int k = q; k < top_k; k += P) {
        const int e = s_e[k];
        experts[t * top_k + k] = e;
        weights[t * top_k + k] = e < 0 ? 0.f : scale * ((k == q ? mine_w : weight(as_float(row[e]))) / sum);
    }
}

// ---- the logits' gradient -----------------------------------------------------------------------------------------------
// Only the chosen experts' gradients depend on the weights' one by one.  Every expert's is -mean * score of it in a softmax without the
// sum of the chosen below (DENSE), 0 otherwise; the chosen ones' are written over it.  P lanes of a warp for a token: the chosen ones' loads,
// one behind the other, are what a token takes, and many tokens are on their way so.  65 536 tokens, 8 of 256 bf16: 14 us, 38 MB
// (37 us with a warp a token); DENSE, which goes three times through a row's exponentials, 43.  N values of a row at a time: 16 bytes,
// or one.  Shares, sums and gradients are of 32 bits, relative to the largest share's.
template <typename T, int P, bool WHOLE, bool DENSE>
__global__ void __launch_bounds__(128) k_expert_choose_bwd(const T* __restrict__ logits, int64_t ld, const int32_t* n_tokens,
                                                           int64_t max_tokens, int top_k, int E, int flags, float scale,
                                                           const int32_t* __restrict__ experts, const float* __restrict__ grad_w,
                                                           T* __restrict__ grad, int64_t ld_grad) {
    constexpr int kTokens = 128 / P, N = WHOLE ? 16 / (int)sizeof(T) : 1;
    constexpr int kChosen = P == 2 ? 16 : HL_MAX_TOP_K;          // (two lanes: of up to 16 experts)
    __shared__ int32_t s_chosen[kTokens][kChosen];
    __shared__ float s_grad[kTokens][kChosen];
    constexpr int kWords = P == 2 ? 1 : P;                       // (two lanes: of up to 16 experts, eight: of up to 256)
    __shared__ uint32_t s_there[DENSE ? kTokens : 1][kWords];    // a bit for each that is chosen
    const bool softmax = DENSE || (flags & kSoftmax), renorm = !DENSE && (flags & kRenorm);
    const int q = threadIdx.x % P, mine = threadIdx.x / P;
    int64_t tokens = max_tokens;
    if (n_tokens) tokens = min((int64_t)max(__ldg(n_tokens), 0), max_tokens);
    const int64_t t = (int64_t)blockIdx.x * kTokens + mine;
    if (t - (int)(threadIdx.x & 31) / P >= tokens) return;
    const bool live = t < tokens;
    const int64_t at = live ? t : tokens - 1;
    const T* row = logits + at * ld;
    T* out = grad + at * ld_grad;
    const float none = -INFINITY;
    const auto logit = [&](int e) {
        const float x = as_float(row[e]);
        return x != x ? none : x;
    };
    if (!DENSE && live)
        for (int c = q * N; c < E; c += P * N) {
            Pack<T, N> v;
            v.zero();
            v.store(out + c);
        }

    float top = none;
    if constexpr (DENSE) {
        if (q < kWords) s_there[mine][q] = 0;
        // (the row stays in the L1 for the next two rounds)
        for (int c = q * N; c < E; c += P * N) {
            Pack<T, N> v;
            float x[N];
            v.load(row + c);
            v.get(x);
#pragma unroll
            for (int k = 0; k < N; ++k) top = fmaxf(top, x[k]);  // (which is not NaN where one of the two is)
        }
        top = max_of<P>(top);
        __syncwarp();
    }
    // the chosen: their scores (relative, as above), and sums over them
    float m = none, base = 0.f;
    for (int k = q; k < top_k; k += P) {
        const int e = __ldg(&experts[at * top_k + k]);
        s_chosen[mine][k] = (unsigned)e < (unsigned)E ? e : -1;
        if ((unsigned)e >= (unsigned)E) continue;
        const float x = logit(e), g = renorm || DENSE ? __ldg(&grad_w[at * top_k + k]) : 0.f;
        if (x > m) {
            m = x;
            base = g;
        }
        if constexpr (DENSE) atomicOr(&s_there[mine][e >> 5], 1u << (e & 31));
    }
    const float mine_m = m;
    m = max_of<P>(m);
    // Shares do not change with what all gradients have in common.  Without the gradient of the one with the largest share, what is
    // left of that one is the others' mean, which is small where they have little, and of the others the differences that count: nothing
    // is lost between large numbers (with one share all but 1, that would be all digits), and nothing at all is left where gradients
    // are alike, or there is one alone.  In a softmax over all, those that were not chosen have a gradient of 0: -base is left of it.
    if (renorm || DENSE) {
        base = __shfl_sync(kAll, base, __ffs(__ballot_sync(kAll, mine_m == m) & lanes_of<P>(threadIdx.x & 31)) - 1);
        if (!isfinite(base)) base = 0.f;
    }
    float z = 1.f, rest = 0.f;                                   // rest: of z, what those have that were not chosen
    if constexpr (DENSE) {
        if (m != top) base = 0.f;                                // (the one with the largest share was not chosen)
        __syncwarp();
        z = 0.f;
        for (int c = q * N; c < E; c += P * N) {
            Pack<T, N> v;
            float x[N];
            v.load(row + c);
            v.get(x);
            const uint32_t there = s_there[mine][c >> 5] >> (c & 31);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float s = x[k] > none ? part(x[k], top) : 0.f;
                z += s;
                rest += (there >> k) & 1u ? 0.f : s;
            }
        }
        z = sum_of<P>(z);
        rest = sum_of<P>(rest);
    }
    if (!softmax) m = renorm ? fminf(m, 0.f) : 0.f;
    else if (!renorm) m = top;
    const auto score = [&](float x, float* other) {              // *other: 1 - sigmoid(x)
        *other = 1.f;
        if (x == none) return 0.f;
        if (softmax) return part(x, m);
        const float e = expf(x > 0.f ? -x : x), per = 1.f / (1.f + e);
        *other = (x > 0.f ? e : 1.f) * per;
        return (x > 0.f ? 1.f : m == 0.f ? e : part(x, m)) * per;
    };
    // (in a softmax over all an expert counts once, however often it is there: at its first place)
    const auto gradient = [&](int k, int e, bool* again) {
        *again = false;
        if constexpr (DENSE)
            for (int i = 0; i < k; ++i) *again = *again || s_chosen[mine][i] == e;
        return __ldg(&grad_w[at * top_k + k]) - (*again ? 0.f : base);
    };
    float sum = 0.f, dot = 0.f, first = 0.f, first_other = 1.f, first_g = 0.f;               // (of the lane's first choice)
    bool first_again = false;
    for (int k = q; k < top_k; k += P) {
        const int e = s_chosen[mine][k];
        if (e < 0) continue;
        float other;
        bool again;
        const float s = score(logit(e), &other), g = gradient(k, e, &again);
        if (k == q) {
            first = s;
            first_other = other;
            first_g = g;
            first_again = again;
        }
        sum += s;
        dot += s * g;
    }
    sum = sum_of<P>(sum);
    dot = sum_of<P>(dot);
    if constexpr (DENSE) dot -= base * rest;
    if (!renorm) sum = softmax ? z : 1.f;
    const float per = sum > 0.f ? 1.f / sum : 0.f, mean = renorm || softmax ? dot * per : 0.f;
    // d/dl of the weights: scale * share * (grad - mean), times 1 - score for sigmoids
    for (int k = q; k < top_k; k += P) {
        float s = first, other = first_other, g = first_g;
        bool again = first_again;
        const int e = s_chosen[mine][k];
        if (k != q && e >= 0) {
            s = score(logit(e), &other);
            g = gradient(k, e, &again);
        }
        s_grad[mine][k] = e < 0 ? 0.f : scale * (s * per) * (again ? g : g - mean) * other;
    }
    if (!live) return;
    if constexpr (DENSE)
        for (int c = q * N; c < E; c += P * N) {
            Pack<T, N> v;
            float x[N];
            v.load(row + c);
            v.get(x);
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = x[k] > none ? -scale * (part(x[k], top) * per) * (base + mean) : 0.f;
            v.set(x);
            v.store(out + c);
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

// Lanes of a token and how many experts each holds at most: as few lanes as hold all, eight a lane, above 128 experts sixteen (two
// tokens of 256 experts a warp, for which most steps take the time of one: 69 us instead of 82 for 65 536), above 512 more.  With
// groups, one in which a group is that of whole lanes, of as many experts each as divide it: that one, or a wider one of less than 16 lanes
// (16 lanes for 60 experts in five groups: 54 us instead of 33 through shared memory, 45 282 tokens; 384 in eight: 115 instead of
// 190 for 65 536).
#define HL_SHAPES(S, RUN, WHOLE)                                                                                        \
    ((S) == 0   ? RUN(8, 1, WHOLE)                                                                                      \
     : (S) == 1 ? RUN(8, 2, WHOLE)                                                                                      \
     : (S) == 2 ? RUN(8, 4, WHOLE)                                                                                      \
     : (S) == 3 ? RUN(8, 8, WHOLE)                                                                                      \
     : (S) == 4 ? RUN(8, 16, WHOLE)                                                                                     \
     : (S) == 5 ? RUN(16, 16, WHOLE)                                                                                    \
     : (S) == 6 ? RUN(16, 32, WHOLE)                                                                                    \
                : RUN(32, 32, WHOLE))
constexpr int kShapes = 8, kShapeItems[kShapes] = {8, 8, 8, 8, 8, 16, 16, 32}, kShapeLanes[kShapes] = {1, 2, 4, 8, 16, 16, 32, 32};
struct Layout {
    int shape, per_lane, group_lanes;
};
Layout layout_of(const hl_router* r) {
    const int E = r->n_experts, per = E / r->n_groups;
    int first = 0;
    while (kShapeItems[first] * kShapeLanes[first] < E) ++first;
    if (r->n_groups > 1)
        for (int s = first; s == first || (s < kShapes && kShapeLanes[s] < 16); ++s)
            for (int d = kShapeItems[s]; 2 * d >= kShapeItems[s]; --d)     // (at least half of what a lane can hold)
                if (per % d == 0 && E / d <= kShapeLanes[s]) return {s, d, per / d};
    return {first, kShapeItems[first], 0};
}

template <typename T>
int32_t launch_choose(const hl_router* r, const void* logits, int64_t ld, const float* bias, int64_t max_tokens,
                      const int32_t* n_tokens, int32_t* experts, float* weights, int32_t* status, cudaStream_t stream) {
    const Layout at = layout_of(r);
    const int per = r->n_experts / r->n_groups;
#define HL_RUN(ITEMS, P, WHOLE)                                                                                               \
    launch_cluster(k_expert_choose<T, ITEMS, P, WHOLE>, (unsigned)div_up(max_tokens, Shape<ITEMS, P>::kTokens), Shape<ITEMS, P>::kNT, \
                   r->n_groups > 1 && !at.group_lanes ? Shape<ITEMS, P>::kTokens * (r->n_experts + 2 * r->n_groups) * sizeof(double) : 0, 0,      \
                   stream, static_cast<const T*>(logits), ld, bias, n_tokens, max_tokens, r->top_k, r->n_experts, r->n_groups, \
                   per, ((1u << 21) + per - 1) / (unsigned)per, r->top_groups, at.per_lane, at.group_lanes, flags_of(r), r->scale,    \
                   experts, weights, status)
    constexpr int N = 16 / (int)sizeof(T);
    const bool whole = r->n_experts % N == 0 && at.per_lane % N == 0 && lies_at(logits, 16) && ld * sizeof(T) % 16 == 0 && lies_at(bias, 16);
    if (whole) HL_CUDA_TRY(HL_SHAPES(at.shape, HL_RUN, true));
    else HL_CUDA_TRY(HL_SHAPES(at.shape, HL_RUN, false));
#undef HL_RUN
    note_launches(1);
    HL_LAUNCH_CHECK();
    return HL_OK;
}
template <typename T>
int32_t launch_choose_bwd(const hl_router* r, const void* logits, int64_t ld, int64_t max_tokens, const int32_t* n_tokens,
                          const int32_t* experts, const float* grad_w, void* grad, int64_t ld_grad, cudaStream_t stream) {
    const bool whole = r->n_experts % (16 / (int)sizeof(T)) == 0 && lies_at(logits, 16) && ld * sizeof(T) % 16 == 0 &&
                       lies_at(grad, 16) && ld_grad * sizeof(T) % 16 == 0;
    // (eight lanes a token: 32 experts' rows a line's half each; many experts: a warp)
    const int E = r->n_experts, P = E <= 16 ? 2 : E <= 256 ? 8 : 32;
    const bool dense = r->score == HL_SCORE_SOFTMAX && !r->renorm;                 // (every expert's has a part)
#define HL_RUN(P)                                                                                                               \
    launch(dense ? (whole ? k_expert_choose_bwd<T, P, true, true> : k_expert_choose_bwd<T, P, false, true>)                       \
                 : (whole ? k_expert_choose_bwd<T, P, true, false> : k_expert_choose_bwd<T, P, false, false>),                    \
           (unsigned)div_up(max_tokens, 128 / P), 128, stream, static_cast<const T*>(logits), ld, n_tokens, max_tokens, r->top_k, E, flags_of(r), r->scale, experts, grad_w,   \
           static_cast<T*>(grad), ld_grad)
    HL_CUDA_TRY(P == 2 ? HL_RUN(2) : P == 8 ? HL_RUN(8) : HL_RUN(32));
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
