// Router: the k experts of a token and their weights, from its logits, and the logits' gradient.
//
//   s = softmax(l) or sigmoid(l);  v = s + bias;  groups of experts rank by the sum of their largest v;  the k largest v (no
//   bias: the largest l) among the groups that stay are chosen;  w = scale s [/ sum of the chosen s]
//
// A token is dealt out to 16 neighbouring lanes of a wavefront, VALUES neighbouring logits to each, and its choice is one
// maximum after another in registers: what a lane hands to the others goes through the vector unit's lane permutations,
// without LDS or barriers.  What bounds it is that selection: for every choice a lane goes through its VALUES twice.  32768 tokens,
// 2 of 64 experts: 6.3 us (1.4 TB/s); 16384 tokens, 8 of 256 experts in 8 groups: 18 us.  Backward has no selection: the first 5 us.
//
// Which of two experts comes first is defined by their exact scores, and float scores are some 2^-22 off.  So the scores
// are compared in float, and where two that follow one another lie within that error (one token in a few hundred) the
// wavefront's tokens are done again with 64-bit scores.
#include "common.h"
#include "lanes.h"
#include "wide.h"
#include <cmath>

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
constexpr int BLOCK = 512;

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

// The choices of one token by 64-bit scores, by a whole wavefront: lane j returns the j-th.  Few tokens come here, but the
// launch waits for the last one, so what counts is the length of the chain.
template <typename T, int VALUES>
__device__ __forceinline__ int choose_exactly(const RouterArgs& a, const T* row) {
    constexpr double NONE = -__builtin_inf();
    const int lane = threadIdx.x & 63, e0 = lane * VALUES;
    const bool by_score = a.bias != nullptr;
    double s[VALUES];
    float l[VALUES], bias[VALUES], m = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        l[v] = e0 + v < a.E ? load_logit(row + e0 + v) : -__builtin_inff();
        bias[v] = by_score && e0 + v < a.E ? a.bias[e0 + v] : 0.0f;
    }
#pragma unroll
    for (int v = 0; v < VALUES; ++v) m = fmaxf(m, l[v]);
    if (a.sigmoid) {
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
    int chosen = -1;
    for (int j = 0; j < a.k; ++j) {
        double mine = s[0];
#pragma unroll
        for (int v = 1; v < VALUES; ++v) mine = larger(mine, s[v]);
        const double most = wave_max(mine);
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

template <typename T, int VALUES>
__global__ __launch_bounds__(BLOCK, VALUES <= 16 ? 4 : 2) void router_kernel(RouterArgs a) {
    constexpr int TOKENS = BLOCK / LANES;
    __shared__ int hist[512];
    const int lane = threadIdx.x & (LANES - 1);
    if (a.load) {
        for (int e = threadIdx.x; e < a.E; e += BLOCK) hist[e] = 0;
        __syncthreads();
    }
    const long long base = a.first + (long long)blockIdx.x * TOKENS, t = base + threadIdx.x / LANES;
    const bool there = t < a.T;
    const T* row = reinterpret_cast<const T*>(a.logits) + (there ? t : 0) * a.ld;
    float l[VALUES], bias[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) bias[v] = 0.0f;
    if (a.bias) load_values<float, VALUES>(a.bias, a.E, lane, true, 0.0f, bias);
    load_logits<T, VALUES>(row, a.E, lane, there, l);
    int chosen;
    Softmax<float> soft = {0.0f, 0.0f};
    const bool sure = choose<VALUES>(a, l, bias, &soft, &chosen);
    unsigned long long unsure = __ballot(!sure && there);
    while (unsure) {
        const int token = __builtin_ctzll(unsure) / LANES;           // of the wavefront
        unsure &= ~(0xffffull << (token * LANES));
        const long long ut = base + (threadIdx.x >> 6) * (64 / LANES) + token;
        const int c = choose_exactly<T, (VALUES + 3) / 4>(a, reinterpret_cast<const T*>(a.logits) + ut * a.ld);
        const int mine = __shfl(c, lane, 64);
        if (((threadIdx.x & 63) / LANES) == token) chosen = mine;
    }
    // the chosen logits: from the lanes that have them, or, where those have many, from memory again
    float z = -__builtin_inff();
    if constexpr (VALUES <= 4) {
#pragma unroll
        for (int v = 0; v < VALUES; ++v) {
            const float o = __shfl(l[v], chosen / VALUES, LANES);
            z = chosen >= 0 && chosen % VALUES == v ? o : z;
        }
    } else if (chosen >= 0) {
        z = load_logit(row + chosen);
    }
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
    if (there && lane < a.k) {
        a.idx[t * a.k + lane] = chosen;
        a.w[t * a.k + lane] = w * a.scale;
        if (a.load && chosen >= 0) atomicAdd(&hist[chosen], 1);       // whole numbers: the order does not matter
    }
    if (a.load) {
        __syncthreads();
        for (int e = threadIdx.x; e < a.E; e += BLOCK)
            if (hist[e]) atomicAdd(&a.load[e], hist[e]);
    }
}

// load[e] += how often e is in idx.  Many of the router's own workgroups adding their counts up would take longer than they
// have taken to choose: what they add meets in a few cache lines, which take a request about every 5 ns (32768 tokens, 64
// experts: 24 us with that, 9.9 us with this launch behind it, 3 of them this kernel's).
__global__ __launch_bounds__(1024) void router_load_kernel(const int* __restrict__ idx, long long n, int E, int* __restrict__ load) {
    __shared__ int hist[512];
    for (int e = threadIdx.x; e < E; e += 1024) hist[e] = 0;
    __syncthreads();
    const long long step = (long long)gridDim.x * 1024;
#pragma unroll 4
    for (long long i = (long long)blockIdx.x * 1024 + threadIdx.x; i < n; i += step) {
        const int e = idx[i];
        if (e >= 0) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += 1024)
        if (hist[e]) atomicAdd(&load[e], hist[e]);
}

struct RouterBwdArgs {
    const void* logits; const int* idx; const float* dw; void* dl;
    long long ld, first;
    int T, E, k, sigmoid, renorm;
    float scale;
};

// Lane j of a token holds its j-th choice: expert, logit and weight gradient.  Only a softmax over all experts needs the
// other logits.
template <typename T, int VALUES>
__global__ __launch_bounds__(256) void router_bwd_kernel(RouterBwdArgs a) {
    constexpr int TOKENS = 256 / LANES;
    const int lane = threadIdx.x & (LANES - 1), e0 = lane * VALUES;
    const long long t = a.first + (long long)blockIdx.x * TOKENS + threadIdx.x / LANES;
    const bool there = t < a.T;
    const T* row = reinterpret_cast<const T*>(a.logits) + (there ? t : 0) * a.ld;
    const bool full = !a.sigmoid && !a.renorm;
    float s[VALUES];
    if (full) load_logits<T, VALUES>(row, a.E, lane, there, s);
    int mine = there && lane < a.k ? a.idx[t * a.k + lane] : -1;
    if ((unsigned)mine >= (unsigned)a.E) mine = -1;
    const float d = mine >= 0 ? a.dw[t * a.k + lane] * a.scale : 0.0f;
    float g = d;                                       // what the lane's choice contributes to its logit's gradient
    if (full) {
        float l[VALUES];
#pragma unroll
        for (int v = 0; v < VALUES; ++v) l[v] = s[v];
        softmax_of<float, VALUES>(l, s);
    } else {
        const float z = mine >= 0 ? load_logit(row + mine) : -__builtin_inff();
        const bool open = z > -__builtin_inff();
        if (!a.renorm) {
            // s (1 - s) = e / (1 + e)^2, e = exp(-|l|)
            const float e = expf(-fabsf(z)), q = 1.0f + e;
            g = open ? d * (e / (q * q)) : 0.0f;
        } else {
            const float m = lanes_max(z);
            float w;
            if (a.sigmoid) {
                const float shift = fminf(m, 0.0f);
                w = z >= 0.0f ? 1.0f / (1.0f + expf(-z)) : exp_of_difference(z, shift) / (1.0f + expf(z));
            } else {
                w = z == m ? 1.0f : exp_of_difference(z, m);
            }
            if (!open) w = 0.0f;
            const float sum = lanes_sum(w);
            w = sum > 0.0f ? w / sum : 0.0f;
            const float inner = lanes_sum(open ? w * d : 0.0f);
            g = open ? w * (d - inner) : 0.0f;
            if (a.sigmoid) g *= 1.0f / (1.0f + expf(z));             // ds/dl = s (1 - s)
            if (!open) g = 0.0f;
        }
    }
    float ds[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) ds[v] = 0.0f;
    for (int j = 0; j < a.k; ++j) {
        const int at = __shfl(mine, j, LANES) - e0;
        const float q = __shfl(g, j, LANES);
#pragma unroll
        for (int v = 0; v < VALUES; ++v)
            if (at == v) ds[v] = q;
    }
    if (full) {
        float sub = 0.0f;
#pragma unroll
        for (int v = 0; v < VALUES; ++v) sub = fmaf(ds[v], s[v], sub);
        sub = lanes_sum(sub);
#pragma unroll
        for (int v = 0; v < VALUES; ++v) ds[v] = s[v] * (ds[v] - sub);
    }
    if (!there) return;
    T* out = reinterpret_cast<T*>(a.dl) + t * a.ld + e0;
#pragma unroll
    for (int v = 0; v < VALUES; v += 4) {
        if constexpr (VALUES >= 4) {
            store_columns(out + v, ds + v, a.E - e0 - v);
        } else {
#pragma unroll
            for (int i = 0; i < VALUES; ++i)
                if (e0 + i < a.E) Elem<T>::st(out + i, ds[i]);
        }
    }
}

}  // namespace

moe_status router_check(const moe_router_config* c) {
    if (!c) return MOE_ERR_NULL;
    if (c->T < 0 || c->E <= 0 || c->k <= 0 || c->groups <= 0 || c->group_k <= 0) return MOE_ERR_SHAPE;
    if (c->ld != 0 && c->ld < c->E) return MOE_ERR_SHAPE;
    if (c->dtype != MOE_F32 && c->dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (c->scores != MOE_SOFTMAX && c->scores != MOE_SIGMOID) return MOE_ERR_UNSUPPORTED;
    if (c->renormalize != 0 && c->renormalize != 1) return MOE_ERR_UNSUPPORTED;
    if (c->group_top != 1 && c->group_top != 2) return MOE_ERR_UNSUPPORTED;
    if (!std::isfinite(c->scale)) return MOE_ERR_SHAPE;
    if (c->E > 512 || c->k > K_MOST || c->groups > 16) return MOE_ERR_UNSUPPORTED;
    if (c->E % c->groups != 0 || c->group_k > c->groups || c->k > c->E / c->groups * c->group_k) return MOE_ERR_SHAPE;
    return MOE_OK;
}

namespace {

// As many values to a lane as the experts need.
int router_values(int E) { return E <= 16 ? 1 : E <= 32 ? 2 : E <= 64 ? 4 : E <= 128 ? 8 : E <= 256 ? 16 : 32; }
#define ROUTER_BY_VALUES(E, LAUNCH) do { switch (router_values(E)) { \
        case 1: LAUNCH(1); break; case 2: LAUNCH(2); break; case 4: LAUNCH(4); break; \
        case 8: LAUNCH(8); break; case 16: LAUNCH(16); break; default: LAUNCH(32); } } while (0)

// Workgroups of the router that may add up their own counts (4096 tokens, 64 experts: 6.9 us so, 7.4 with a launch for it, of 256
// experts 11.1 / 11.8; 8192 tokens, 64 experts 9.6 / 7.5); and the workgroups of the launch that counts instead.
constexpr int OWN_COUNTS = 128, COUNT_BLOCKS = 32;

// Tokens of a launch, and its workgroups from token `first` on.
constexpr long long LAUNCH_TOKENS = LAUNCH_THREADS / LANES;
int router_blocks(int T, long long first, int tokens) {
    const long long here = T - first < LAUNCH_TOKENS ? T - first : LAUNCH_TOKENS;
    return (int)((here + tokens - 1) / tokens);
}

template <typename T> void router_launch(RouterArgs a, hipStream_t s) {
    const int tokens = BLOCK / LANES;
    int* const load = a.load;
    if (a.T > OWN_COUNTS * tokens) a.load = nullptr;
    for (a.first = 0; a.first < a.T; a.first += LAUNCH_TOKENS) {
        const int blocks = router_blocks(a.T, a.first, tokens);
#define ROUTER_LAUNCH(V) router_kernel<T, V><<<blocks, BLOCK, 0, s>>>(a)
        ROUTER_BY_VALUES(a.E, ROUTER_LAUNCH);
#undef ROUTER_LAUNCH
    }
    if (load && !a.load) {
        const long long n = (long long)a.T * a.k, most = (n + 4095) / 4096;
        router_load_kernel<<<most < COUNT_BLOCKS ? (int)most : COUNT_BLOCKS, 1024, 0, s>>>(a.idx, n, a.E, load);
    }
}
template <typename T> void router_bwd_launch(RouterBwdArgs a, hipStream_t s) {
    for (a.first = 0; a.first < a.T; a.first += LAUNCH_TOKENS) {
        const int blocks = router_blocks(a.T, a.first, 256 / LANES);
#define ROUTER_LAUNCH(V) router_bwd_kernel<T, V><<<blocks, 256, 0, s>>>(a)
        ROUTER_BY_VALUES(a.E, ROUTER_LAUNCH);
#undef ROUTER_LAUNCH
    }
}

}  // namespace

moe_status router_run(const moe_router_config* cfg, const void* logits, const float* bias, int32_t* topk_idx, float* topk_w,
                      int32_t* load, hipStream_t s) {
    const int per = cfg->E / cfg->groups, values = router_values(cfg->E);
    // lanes that hold a group, where that is a power of two
    auto whole = [per](int v) { return per % v == 0 && ((per / v) & (per / v - 1)) == 0 ? per / v : 0; };
    const int exact = whole((values + 3) / 4);
    RouterArgs a = {logits, bias, topk_idx, topk_w, load, cfg->ld ? (long long)cfg->ld : (long long)cfg->E, 0, cfg->T, cfg->E, cfg->k,
                    cfg->scores == MOE_SIGMOID, cfg->groups, cfg->group_k, cfg->group_top, cfg->renormalize, whole(values),
                    exact <= 16 ? exact : 0,
                    ((1u << 20) + per - 1) / per, cfg->scale};
    if (cfg->dtype == MOE_F32) router_launch<float>(a, s); else router_launch<bf16_t>(a, s);
    MOE_CHECK_LAUNCH();
    return MOE_OK;
}

}  // namespace moe

extern "C" moe_status moe_router_fwd(const moe_router_config* cfg, const void* logits, const float* bias, int32_t* topk_idx,
                                     float* topk_w, int32_t* load, void* stream) {
    MOE_TRY(moe::router_check(cfg));
    if (cfg->T == 0) return MOE_OK;
    if (!logits || !topk_idx || !topk_w) return MOE_ERR_NULL;
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_ROUTER, s);
        MOE_TRY(moe::router_run(cfg, logits, bias, topk_idx, topk_w, load, s));
    }
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

extern "C" moe_status moe_router_bwd(const moe_router_config* cfg, const void* logits, const int32_t* topk_idx, const float* dw,
                                     void* dlogits, void* stream) {
    MOE_TRY(moe::router_check(cfg));
    if (cfg->T == 0) return MOE_OK;
    if (!logits || !topk_idx || !dw || !dlogits) return MOE_ERR_NULL;
    moe::RouterBwdArgs a = {logits, topk_idx, dw, dlogits, cfg->ld ? (long long)cfg->ld : (long long)cfg->E, 0, cfg->T, cfg->E, cfg->k,
                            cfg->scores == MOE_SIGMOID, cfg->renormalize, cfg->scale};
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_ROUTER_BWD, s);
        if (cfg->dtype == MOE_F32) moe::router_bwd_launch<float>(a, s); else moe::router_bwd_launch<moe::bf16_t>(a, s);
    }
    MOE_CHECK_LAUNCH();
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}
