// Which experts a token has and with what weights, from its logits: what the router and the layer for a few tokens share.
// Which of two experts comes first is defined by their exact scores; router.hip says how that is decided.
#pragma once
#include "common.h"
#include "lanes.h"
#include "wide.h"

namespace moe {

namespace {

struct RouterArgs {
    const void* logits; const float* bias; int* idx; float* w; int* load;
    long long ld, first;             // first: token of the launch
    int T, E, k, sigmoid, groups, group_k, group_top, renorm;
    int group_lanes;                 // lanes that hold a group, if that is a whole number and a power of two, else 0
    int exact_lanes;                 // the same with a token dealt out to 64 lanes, up to 16
    unsigned group_mul;              // e / (experts of a group) = e * group_mul >> 20 for e < 512
    float scale;
};

__device__ __forceinline__ float exp_of(float x) { return __expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }

constexpr int LANES = 16;            // of a token: as many as there may be choices and groups

__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return fmin(a, b); }
__device__ __forceinline__ int smaller(int a, int b) { return a < b ? a : b; }

template <typename V> __device__ __forceinline__ V lanes_max(V v) {
    v = larger(v, from_lane<AWAY_1>(v));
    v = larger(v, from_lane<AWAY_2>(v));
    v = larger(v, from_lane<MIRROR_8>(v));
    return larger(v, from_lane<MIRROR_16>(v));
}
template <typename V> __device__ __forceinline__ V lanes_sum(V v) {
    v += from_lane<AWAY_1>(v);
    v += from_lane<AWAY_2>(v);
    v += from_lane<MIRROR_8>(v);
    return v + from_lane<MIRROR_16>(v);
}
__device__ __forceinline__ int lanes_min(int v) {
    v = smaller(v, from_lane<AWAY_1>(v));
    v = smaller(v, from_lane<AWAY_2>(v));
    v = smaller(v, from_lane<MIRROR_8>(v));
    return smaller(v, from_lane<MIRROR_16>(v));
}

constexpr int K_MOST = 16;

// NaN counts as -inf.
template <typename T> __device__ __forceinline__ float load_logit(const T* p) {
    const float v = Elem<T>::ld(p);
    return v != v ? -__builtin_inff() : v;
}
// A lane's VALUES elements of a row of E; `past` where there are none.
template <typename T, int VALUES> __device__ __forceinline__ void load_values(const T* row, int E, int lane, bool there, float past, float* l) {
    constexpr int WIDE = VALUES < 16 / (int)sizeof(T) ? VALUES : 16 / (int)sizeof(T);       // elements of an access
    if (there && (lane + 1) * VALUES <= E && WIDE * sizeof(T) >= 4) {
#pragma unroll
        for (int v = 0; v < VALUES; v += WIDE) {
            constexpr int BYTES = WIDE * (int)sizeof(T) < 4 ? 4 : WIDE * (int)sizeof(T);
            const auto u = *reinterpret_cast<const Anywhere<BYTES, (int)sizeof(T)>*>(row + lane * VALUES + v);
#pragma unroll
            for (int i = 0; i < WIDE; ++i) {
                if constexpr (sizeof(T) == 4) l[v + i] = __uint_as_float(u.w[i]);
                else l[v + i] = __uint_as_float((i & 1) ? u.w[i / 2] & 0xffff0000u : u.w[i / 2] << 16);
            }
        }
    } else {
#pragma unroll
        for (int v = 0; v < VALUES; ++v) {
            const int e = lane * VALUES + v;
            l[v] = there && e < E ? Elem<T>::ld(row + e) : past;
        }
    }
}
template <typename T, int VALUES> __device__ __forceinline__ void load_logits(const T* row, int E, int lane, bool there, float* l) {
    load_values<T, VALUES>(row, E, lane, there, -__builtin_inff(), l);
#pragma unroll
    for (int v = 0; v < VALUES; ++v) l[v] = l[v] != l[v] ? -__builtin_inff() : l[v];
}

// exp(a - b), b finite or a smaller than it: what the difference's rounding leaves out is put back, as its share of the result grows
// with the difference.  For weights, a value to a lane; the scores of all experts do with __expf, since small parts of a sum
// need not be as exact as large ones.
__device__ __forceinline__ float exp_of_difference(float a, float b) {
    const float d = a - b, back = d - a, rest = (a - (d - back)) - (b + back), e = expf(d);
    return d == -__builtin_inff() ? 0.0f : fmaf(e, rest, e);
}

// Of a softmax: the largest logit and 1 / the sum of exp(l - it).  Infinite logits share it evenly.
template <typename F> struct Softmax { float m; F inv; };
template <typename F> __device__ __forceinline__ F softmax_term(float l, float m) {
    return l == -__builtin_inff() ? F(0) : l == m ? F(1) : exp_of(F(l) - F(m));
}
template <typename F, int VALUES> __device__ __forceinline__ F in_pairs(const F* s) {
    if constexpr (VALUES == 1) return s[0];
    else return in_pairs<F, VALUES / 2>(s) + in_pairs<F, VALUES / 2>(s + VALUES / 2);
}
// A lane's terms are added in pairs: one after the other a largest term would swallow up to 31 small ones.
template <typename F, int VALUES> __device__ __forceinline__ Softmax<F> softmax_of(const float* l, F* s) {
    float m = l[0];
#pragma unroll
    for (int v = 1; v < VALUES; ++v) m = fmaxf(m, l[v]);
    m = lanes_max(m);
#pragma unroll
    for (int v = 0; v < VALUES; ++v) s[v] = softmax_term<F>(l[v], m);
    const F sum = lanes_sum(in_pairs<F, VALUES>(s));
    const F inv = sum > F(0) ? F(1) / sum : F(0);
#pragma unroll
    for (int v = 0; v < VALUES; ++v) s[v] *= inv;
    return {m, inv};
}

// first, second: the two largest of what was in them and of f >= q
template <typename F> __device__ __forceinline__ void join_two(F& first, F& second, F f, F q) {
    const F lo = smaller(first, f);
    first = larger(first, f);
    second = larger(larger(second, lo), q);
}

// The choices of a wavefront's four tokens by float scores: lane j of a token returns its j-th choice in *chosen (-1:
// none).  False in a token's lanes: float scores do not decide.
template <int VALUES>
__device__ __forceinline__ bool choose(const RouterArgs& a, const float* l, const float* bias, Softmax<float>* soft, int* chosen) {
    constexpr float NONE = -__builtin_inff();
    const int lane = threadIdx.x & (LANES - 1), e0 = lane * VALUES;
    const bool by_score = a.bias != nullptr, scored = by_score || a.groups > 1;
    // How far apart two scores have to be.  In units of 2^-24 a sigmoid is less than 3 off (the exponential's rounded argument,
    // itself, the sum, the reciprocal), the sum with the bias one of its size.  A softmax's parts, in such units of the largest part:
    // each its exponential's 3 and a product's 1; and what all share but the bias does not, the sum's error: 9 additions for 512
    // experts, 11 of the terms' exponentials (the most that 511 terms of equal size can make), the reciprocal's 1.  29 for two.
    float rank[VALUES], error = 0x1p-21f;
    if (scored || !a.sigmoid) {                       // a softmax's parts are wanted for the weights in any case
        if (a.sigmoid) {
#pragma unroll
            for (int v = 0; v < VALUES; ++v) rank[v] = __builtin_amdgcn_rcpf(1.0f + __expf(-l[v]));
        } else {
            *soft = softmax_of<float, VALUES>(l, rank);
            error = 0x1p-19f * soft->inv;
        }
    }
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        if (by_score) {
            rank[v] += bias[v];
            if (!(rank[v] > NONE)) rank[v] = NONE;
        }
        if (!scored) rank[v] = l[v];
        if (l[v] == NONE) rank[v] = NONE;
    }
    bool sure = true;
    if (a.groups > 1) {
        float mine = NONE;                            // this lane's group's score; the slow way: that of group number `lane`
        float size = 0.0f;                            // the magnitudes of its two parts, which may nearly cancel
        if (a.group_lanes) {
            // a group is group_lanes (a power of two) whole lanes
            float first = NONE, second = NONE;
#pragma unroll
            for (int v = 0; v < VALUES; ++v) {
                second = larger(second, smaller(first, rank[v]));
                first = larger(first, rank[v]);
            }
            if (a.group_lanes > 1) join_two(first, second, from_lane<AWAY_1>(first), from_lane<AWAY_1>(second));
            if (a.group_lanes > 2) join_two(first, second, from_lane<AWAY_2>(first), from_lane<AWAY_2>(second));
            if (a.group_lanes > 4) join_two(first, second, from_lane<MIRROR_8>(first), from_lane<MIRROR_8>(second));
            const bool two = a.group_top == 2 && second > NONE;
            mine = two ? first + second : first;
            size = fabsf(first) + (two ? fabsf(second) : 0.0f);
        } else {
            for (int g = 0; g < a.groups; ++g) {
                float first = NONE, second = NONE;
#pragma unroll
                for (int v = 0; v < VALUES; ++v) {
                    const float r = ((unsigned)(e0 + v) * a.group_mul >> 20) == (unsigned)g ? rank[v] : NONE;
                    second = larger(second, smaller(first, r));
                    first = larger(first, r);
                }
                join_two(first, second, from_lane<AWAY_1>(first), from_lane<AWAY_1>(second));
                join_two(first, second, from_lane<AWAY_2>(first), from_lane<AWAY_2>(second));
                join_two(first, second, from_lane<MIRROR_8>(first), from_lane<MIRROR_8>(second));
                join_two(first, second, from_lane<MIRROR_16>(first), from_lane<MIRROR_16>(second));
                const bool two = a.group_top == 2 && second > NONE;
                if (lane == g) {
                    mine = two ? first + second : first;
                    size = fabsf(first) + (two ? fabsf(second) : 0.0f);
                }
            }
        }
        // a group stays if fewer than group_k others are ahead of it; each lane meets all others by rotations
        const int lanes = a.group_lanes ? a.group_lanes : 1;
        const int group = a.group_lanes ? lane / a.group_lanes : lane;
        int ahead = 0;
#define ROUTER_MEET(R) do { \
            const float o = from_lane<ROTATE + R>(mine); \
            const int og = from_lane<ROTATE + R>(group); \
            ahead += o > mine || (o == mine && og < group); } while (0)
        ROUTER_MEET(1); ROUTER_MEET(2); ROUTER_MEET(3); ROUTER_MEET(4); ROUTER_MEET(5);
        ROUTER_MEET(6); ROUTER_MEET(7); ROUTER_MEET(8); ROUTER_MEET(9); ROUTER_MEET(10);
        ROUTER_MEET(11); ROUTER_MEET(12); ROUTER_MEET(13); ROUTER_MEET(14); ROUTER_MEET(15);
#undef ROUTER_MEET
        const bool in = ahead < a.group_k * lanes;
        // The last that stays and the first that does not.  Their scores are sums of two, each part with the error of a score,
        // rounded at its own size with its bias and once more with the other: four units of 2^-24 of the larger one's parts.
        const float last = -lanes_max(in && mine > NONE ? -mine : NONE), next = lanes_max(in ? NONE : mine);
        const float parts = lanes_max(mine == (in ? last : next) ? size : 0.0f);
        sure = next == NONE || last - next > 2.0f * error + 0x1p-21f * parts;
        const unsigned stays = (unsigned)(__ballot(in && group < a.groups) >> ((threadIdx.x & 63) & ~(LANES - 1))) & 0xffffu;
#pragma unroll
        for (int v = 0; v < VALUES; ++v) {
            const bool mine_in = a.group_lanes ? in : (stays >> ((unsigned)(e0 + v) * a.group_mul >> 20) & 1) != 0;
            if (!by_score && rank[v] > NONE) rank[v] = l[v];
            if (!mine_in) rank[v] = NONE;
        }
    }
    *chosen = -1;
    const int shift = (threadIdx.x & 63) & ~(LANES - 1);
    if (by_score) {
        // The lowest bits of a score give way to its place in the lane, so that the largest says by itself which it is and
        // taking it out is one comparison.  k + 1 maxima: the last choice too is compared with the next, without the places:
        // both scores are cut towards zero then, and what lies between them is off by less than one place's VALUES units (with
        // the places in it, by twice as much).
        constexpr int PLACE = VALUES - 1;
        float before = NONE;
#pragma unroll
        for (int v = 0; v < VALUES; ++v)
            rank[v] = rank[v] > NONE ? __uint_as_float((__float_as_uint(fminf(rank[v], 0x1.fffffep127f)) & ~(unsigned)PLACE) | v) : NONE;
        for (int j = 0; j <= a.k; ++j) {
            float mine = rank[0];
#pragma unroll
            for (int v = 1; v < VALUES; ++v) mine = larger(mine, rank[v]);
            const float m = lanes_max(mine), cut = __uint_as_float(__float_as_uint(m) & ~(unsigned)PLACE);
            if (j > 0 && m > NONE) sure = sure && before - cut > error + (0x1p-21f + 0x1p-23f * VALUES) * fabsf(before);
            before = cut;
            if (j == a.k) break;
            const unsigned owners = (unsigned)(__ballot(mine == m && m > NONE) >> shift) & 0xffffu;
            const int owner = __builtin_ctz(owners | 0x10000u);
            if (lane == owner) {
#pragma unroll
                for (int v = 0; v < VALUES; ++v) rank[v] = rank[v] == m ? NONE : rank[v];
            }
            if (lane == j && owner < LANES) *chosen = owner * VALUES + (int)(__float_as_uint(m) & PLACE);
        }
    } else {
        for (int j = 0; j < a.k; ++j) {
            float mine = rank[0];
#pragma unroll
            for (int v = 1; v < VALUES; ++v) mine = larger(mine, rank[v]);
            const float m = lanes_max(mine);
            int at = 1 << 30;
#pragma unroll
            for (int v = VALUES - 1; v >= 0; --v) at = rank[v] == m ? e0 + v : at;
            at = m > NONE ? lanes_min(at) : 1 << 30;
            const int won = at - e0;
#pragma unroll
            for (int v = 0; v < VALUES; ++v) rank[v] = won == v ? NONE : rank[v];
            if (lane == j && at < a.E) *chosen = at;
        }
    }
    return sure;
}

// a lane's value, the same for all (its number has to be)
__device__ __forceinline__ int of_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float of_lane(float v, int lane) { return __int_as_float(of_lane(__float_as_int(v), lane)); }
__device__ __forceinline__ double of_lane(double v, int lane) {
    const long long b = __double_as_longlong(v);
    return __longlong_as_double((long long)of_lane((int)(b >> 32), lane) << 32 | (unsigned)of_lane((int)b, lane));
}
template <typename V> __device__ __forceinline__ V wave_max(V v) {
    v = lanes_max(v);
    return larger(larger(of_lane(v, 0), of_lane(v, 16)), larger(of_lane(v, 32), of_lane(v, 48)));
}

// The k largest of what a wavefront's lanes have, VALUES neighbouring experts' each: lane j returns the j-th, -1 where nothing above -inf is left.
template <int VALUES, typename F> __device__ __forceinline__ int choose_largest(const RouterArgs& a, const F* values) {
    constexpr F NONE = -(F)__builtin_inf();
    const int lane = threadIdx.x & 63, e0 = lane * VALUES;
    F s[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) s[v] = values[v];
    int chosen = -1;
    for (int j = 0; j < a.k; ++j) {
        F mine = s[0];
#pragma unroll
        for (int v = 1; v < VALUES; ++v) mine = larger(mine, s[v]);
        const F most = wave_max(mine);
        if (!(most > NONE)) break;
        int at = 0;
#pragma unroll
        for (int v = VALUES - 1; v >= 0; --v) at = s[v] == most ? e0 + v : at;
        at = of_lane(at, __builtin_ctzll(__ballot(mine == most)));       // the lowest lane has the lowest experts
#pragma unroll
        for (int v = 0; v < VALUES; ++v) s[v] = at == e0 + v ? NONE : s[v];
        if (lane == j) chosen = at;
    }
    return chosen;
}

// The choices of one token by 64-bit scores, by a whole wavefront, whose lanes have its logits (NaN counts as -inf), VALUES
// neighbouring ones each: lane j returns the j-th.  *soft: of a softmax.  What counts is the length of the chain.
template <int VALUES>
__device__ __forceinline__ int choose_exactly(const RouterArgs& a, const float* l, Softmax<float>* soft) {
    constexpr double NONE = -__builtin_inf();
    const int lane = threadIdx.x & 63, e0 = lane * VALUES;
    const bool by_score = a.bias != nullptr, scored = by_score || a.groups > 1;
    double s[VALUES];
    float bias[VALUES], m = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < VALUES; ++v) bias[v] = by_score && e0 + v < a.E ? a.bias[e0 + v] : 0.0f;
#pragma unroll
    for (int v = 0; v < VALUES; ++v) m = fmaxf(m, l[v]);
    if (!scored) {
        // the logits decide; a softmax that is not renormalised still needs its sum
        if (!a.sigmoid && !a.renorm) {
            m = wave_max(m);
            float terms[VALUES];
#pragma unroll
            for (int v = 0; v < VALUES; ++v) terms[v] = softmax_term<float>(l[v], m);
            float sum = lanes_sum(in_pairs<float, VALUES>(terms));
            sum = (of_lane(sum, 0) + of_lane(sum, 16)) + (of_lane(sum, 32) + of_lane(sum, 48));
            *soft = {m, sum > 0.0f ? 1.0f / sum : 0.0f};
        }
        return choose_largest<VALUES>(a, l);
    } else if (a.sigmoid) {
#pragma unroll
        for (int v = 0; v < VALUES; ++v) s[v] = 1.0 / (1.0 + exp(-(double)l[v]));
    } else {
        m = wave_max(m);
        double sum = 0.0;
#pragma unroll
        for (int v = 0; v < VALUES; ++v) {
            s[v] = softmax_term<double>(l[v], m);
            sum += s[v];
        }
        sum = lanes_sum(sum);
        sum = (of_lane(sum, 0) + of_lane(sum, 16)) + (of_lane(sum, 32) + of_lane(sum, 48));
        *soft = {m, sum > 0.0 ? (float)(1.0 / sum) : 0.0f};
#pragma unroll
        for (int v = 0; v < VALUES; ++v) s[v] = sum > 0.0 ? s[v] / sum : 0.0;
    }
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        s[v] += (double)bias[v];
        if (!(s[v] > NONE) || l[v] == -__builtin_inff()) s[v] = NONE;
    }
    if (a.groups > 1) {
        double mine = NONE;                               // lane g: the score of group g
        if (a.exact_lanes) {
            // a group is exact_lanes (a power of two up to 16) whole lanes of the 64
            double first = NONE, second = NONE;
#pragma unroll
            for (int v = 0; v < VALUES; ++v) {
                second = larger(second, smaller(first, s[v]));
                first = larger(first, s[v]);
            }
            if (a.exact_lanes > 1) join_two(first, second, from_lane<AWAY_1>(first), from_lane<AWAY_1>(second));
            if (a.exact_lanes > 2) join_two(first, second, from_lane<AWAY_2>(first), from_lane<AWAY_2>(second));
            if (a.exact_lanes > 4) join_two(first, second, from_lane<MIRROR_8>(first), from_lane<MIRROR_8>(second));
            if (a.exact_lanes > 8) join_two(first, second, from_lane<MIRROR_16>(first), from_lane<MIRROR_16>(second));
            const double score = a.group_top == 2 && second > NONE ? first + second : first;
            mine = __shfl(score, lane * a.exact_lanes & 63, 64);
            if (lane >= a.groups) mine = NONE;
        } else for (int g = 0; g < a.groups; ++g) {
            double first = NONE, second = NONE;
#pragma unroll
            for (int v = 0; v < VALUES; ++v) {
                const double r = ((unsigned)(e0 + v) * a.group_mul >> 20) == (unsigned)g ? s[v] : NONE;
                second = larger(second, smaller(first, r));
                first = larger(first, r);
            }
            join_two(first, second, from_lane<AWAY_1>(first), from_lane<AWAY_1>(second));
            join_two(first, second, from_lane<AWAY_2>(first), from_lane<AWAY_2>(second));
            join_two(first, second, from_lane<MIRROR_8>(first), from_lane<MIRROR_8>(second));
            join_two(first, second, from_lane<MIRROR_16>(first), from_lane<MIRROR_16>(second));
            double f = of_lane(first, 0), q = of_lane(second, 0);
            join_two(f, q, of_lane(first, 16), of_lane(second, 16));
            join_two(f, q, of_lane(first, 32), of_lane(second, 32));
            join_two(f, q, of_lane(first, 48), of_lane(second, 48));
            const double score = a.group_top == 2 && q > NONE ? f + q : f;
            if (lane == g) mine = score;
        }
        int ahead = 0;
        for (int g = 0; g < a.groups; ++g) {
            const double o = of_lane(mine, g);
            ahead += o > mine || (o == mine && g < lane);
        }
        const unsigned long long stays = __ballot(lane < a.groups && ahead < a.group_k);       // (64 bits wide: lanes past E shift by up to 63)
#pragma unroll
        for (int v = 0; v < VALUES; ++v)
            if (!(stays >> ((unsigned)(e0 + v) * a.group_mul >> 20) & 1)) s[v] = NONE;
    }
#pragma unroll
    for (int v = 0; v < VALUES; ++v)
        if (!by_score && s[v] > NONE) s[v] = (double)l[v];
    return choose_largest<VALUES>(a, s);
}
template <typename T, int VALUES>
__device__ __forceinline__ int choose_exactly(const RouterArgs& a, const T* row) {
    const int e0 = (threadIdx.x & 63) * VALUES;
    float l[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) l[v] = e0 + v < a.E ? load_logit(row + e0 + v) : -__builtin_inff();
    Softmax<float> soft;
    return choose_exactly<VALUES>(a, l, &soft);
}

// The weight of a lane's choice, whose logit is z, before the scale; the choices of a token are in 16 neighbouring lanes.
__device__ __forceinline__ float choice_weight(const RouterArgs& a, int chosen, float z, const Softmax<float>& soft) {
    float w;
    if (a.renorm) {
        // Scores that are all tiny are scaled up together before they are divided by their sum.
        const float m = lanes_max(z);
        if (a.sigmoid) {
            const float shift = fminf(m, 0.0f);
            w = z >= 0.0f ? 1.0f / (1.0f + expf(-z)) : exp_of_difference(z, shift) / (1.0f + expf(z));
        } else {
            w = z == m ? 1.0f : exp_of_difference(z, m);
        }
        if (chosen < 0) w = 0.0f;
        const float sum = lanes_sum(w);
        w = sum > 0.0f ? w / sum : 0.0f;
    } else {
        w = a.sigmoid ? 1.0f / (1.0f + expf(-z)) : chosen < 0 ? 0.0f : (z == soft.m ? 1.0f : exp_of_difference(z, soft.m)) * soft.inv;
    }
    return w;
}

// values, exact_values: logits to a lane of 16 and of 64
inline RouterArgs router_args(const moe_router_config* cfg, const void* logits, const float* bias, int* idx, float* w, int* load, int values,
                              int exact_values) {
    const int per = cfg->E / cfg->groups;
    // lanes that hold a group, where that is a power of two
    auto whole = [per](int v) { return per % v == 0 && ((per / v) & (per / v - 1)) == 0 ? per / v : 0; };
    const int exact = whole(exact_values);
    return {logits, bias, idx, w, load, cfg->ld ? (long long)cfg->ld : (long long)cfg->E, 0, cfg->T, cfg->E, cfg->k,
            cfg->scores == MOE_SIGMOID, cfg->groups, cfg->group_k, cfg->group_top, cfg->renormalize, whole(values),
            exact <= 16 ? exact : 0, ((1u << 20) + per - 1) / per, cfg->scale};
}

}  // namespace

}  // namespace moe
