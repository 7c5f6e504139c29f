// Router: the k experts of a token and their weights, from its logits, and the logits' gradient.
//
//   s = softmax(l) or sigmoid(l);  v = s + bias;  groups of experts rank by the sum of their largest v;  the k largest v (no
//   bias: the largest l) among the groups that stay are chosen;  w = scale s [/ sum of the chosen s]
//
// A token is dealt out to LANES neighbouring lanes of a wavefront, VALUES logits to each, so that a choice is LANES-wide
// maximum after maximum in registers, without LDS or barriers.  What bounds it is that selection: for each choice a lane
// goes through its VALUES twice and the maximum travels through log2(LANES) lanes.  Few lanes with many values each need fewest
// instructions per token; many lanes the shortest chain for a single token.
//
// Which of two experts comes first is defined by their exact scores, and float scores are some 2^-22 off.  So the scores
// are compared in float, and where two that follow one another lie within that error (one token in a few hundred) the
// wavefront's tokens are done again with 64-bit scores.
#include "common.h"
#include <cmath>

namespace moe {

namespace {

struct RouterArgs {
    const void* logits; const float* bias; int* idx; float* w; int* load;
    long long ld;
    int T, E, k, sigmoid, groups, group_k, group_top, renorm;
    unsigned per_group;              // experts of a group
    unsigned group_mul;              // e / per_group = e * group_mul >> 20 for e < 512
    float scale;
};

template <typename F> struct Minus;
template <> struct Minus<float> { static __device__ __forceinline__ float inf() { return -__builtin_inff(); } };
template <> struct Minus<double> { static __device__ __forceinline__ double inf() { return -__builtin_inf(); } };

__device__ __forceinline__ float exp_of(float x) { return __expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }

template <int LANES, typename V> __device__ __forceinline__ V lanes_max(V v) {
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) {
        const V o = __shfl_xor(v, off, LANES);
        v = o > v ? o : v;
    }
    return v;
}
template <int LANES, typename V> __device__ __forceinline__ V lanes_sum(V v) {
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off, LANES);
    return v;
}
template <int LANES> __device__ __forceinline__ int lanes_min(int v) {
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) {
        const int o = __shfl_xor(v, off, LANES);
        v = o < v ? o : v;
    }
    return v;
}

constexpr int K_MOST = 16;

template <typename T> __device__ __forceinline__ float load_logit(const T* p) {
    const float v = Elem<T>::ld(p);
    return v != v ? -__builtin_inff() : v;
}

// The scores of a lane's logits.  -inf has none; infinite logits share a softmax evenly.
template <typename F, int LANES, int VALUES>
__device__ __forceinline__ void scores_of(const float* l, int sigmoid, F* s, F* largest) {
    if (sigmoid) {
#pragma unroll
        for (int v = 0; v < VALUES; ++v) s[v] = F(1) / (F(1) + exp_of(-F(l[v])));
        *largest = F(1);
        return;
    }
    float m = l[0];
#pragma unroll
    for (int v = 1; v < VALUES; ++v) m = fmaxf(m, l[v]);
    m = lanes_max<LANES>(m);
    F sum = F(0);
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        s[v] = l[v] == -__builtin_inff() ? F(0) : l[v] == m ? F(1) : exp_of(F(l[v]) - F(m));
        sum += s[v];
    }
    sum = lanes_sum<LANES>(sum);
    const F inv = sum > F(0) ? F(1) / sum : F(0);
#pragma unroll
    for (int v = 0; v < VALUES; ++v) s[v] *= inv;
    *largest = inv;
}

// The choices of a wavefront's tokens in F.  Lane j of a token returns its j-th choice in *chosen (-1: none).  False in
// any lane: float scores do not decide, nothing has been chosen.
template <typename F, int LANES, int VALUES>
__device__ __forceinline__ bool choose(const RouterArgs& a, const float* l, F* s_chosen, int* chosen) {
    constexpr bool FLOAT = sizeof(F) == 4;
    const int lane = threadIdx.x & (LANES - 1);
    F s[VALUES], rank[VALUES], largest;
    scores_of<F, LANES, VALUES>(l, a.sigmoid, s, &largest);
    const bool by_score = a.bias != nullptr;
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        const int e = v * LANES + lane;
        F r = s[v];
        if (by_score && e < a.E) {
            r += F(a.bias[e]);
            if (!(r > Minus<F>::inf())) r = Minus<F>::inf();
        }
        if (l[v] == -__builtin_inff() || e >= a.E) r = Minus<F>::inf();
        rank[v] = r;
    }
    bool sure = true;
    unsigned long long stays = ~0ull;
    if (a.groups > 1) {
        // Each lane keeps the two largest of its own v of every group; the lanes' pairs join by shuffles.
        F mine = Minus<F>::inf();
        for (int g = 0; g < a.groups; ++g) {
            F first = Minus<F>::inf(), second = Minus<F>::inf();
#pragma unroll
            for (int v = 0; v < VALUES; ++v) {
                const unsigned e = v * LANES + lane;
                const F r = (e * a.group_mul >> 20) == (unsigned)g ? rank[v] : Minus<F>::inf();
                const F lo = r < first ? r : first;
                first = r > first ? r : first;
                second = lo > second ? lo : second;
            }
#pragma unroll
            for (int off = LANES / 2; off >= 1; off >>= 1) {
                const F f = __shfl_xor(first, off, LANES), q = __shfl_xor(second, off, LANES);
                const F lo = f < first ? f : first;
                first = f > first ? f : first;
                second = lo > second ? lo : second;
                second = q > second ? q : second;
            }
            const F score = a.group_top == 2 && second > Minus<F>::inf() ? first + second : first;
            if (lane == g) mine = score;
        }
        // a group stays if fewer than group_k others are ahead of it
        int ahead = 0;
        const F most = lanes_max<LANES>(mine == mine && mine > Minus<F>::inf() && mine < -Minus<F>::inf() ? (mine < 0 ? -mine : mine) : F(0));
        const F near = F(0x1p-19) * (F(2) * largest + most);
        for (int g = 0; g < a.groups; ++g) {
            const F o = __shfl(mine, g, LANES);
            ahead += o > mine || (o == mine && g < lane);
            if (FLOAT && lane < a.groups && g != lane && mine > Minus<F>::inf() && o > Minus<F>::inf()) {
                const F d = o - mine;
                sure = sure && (d > near || d < -near);
            }
        }
        const unsigned long long b = __ballot(lane < a.groups && ahead < a.group_k);
        stays = b >> ((threadIdx.x & 63) & ~(LANES - 1));
    }
    if (!by_score || a.groups > 1) {
#pragma unroll
        for (int v = 0; v < VALUES; ++v) {
            const unsigned e = v * LANES + lane;
            if (!by_score && rank[v] > Minus<F>::inf()) rank[v] = F(l[v]);
            if (a.groups > 1 && !(stays >> (e * a.group_mul >> 20) & 1)) rank[v] = Minus<F>::inf();
        }
    }
    // k + 1 maxima, so that the last choice too is compared with the next
    const int rounds = FLOAT && by_score ? a.k + 1 : a.k;
    F before = Minus<F>::inf();
    *chosen = -1;
    *s_chosen = F(0);
    for (int j = 0; j < rounds; ++j) {
        F m = rank[0];
#pragma unroll
        for (int v = 1; v < VALUES; ++v) m = rank[v] > m ? rank[v] : m;
        m = lanes_max<LANES>(m);
        if (FLOAT && by_score) {
            if (j > 0 && m > Minus<F>::inf()) {
                const F size = before < 0 ? -before : before;
                sure = sure && before - m > F(0x1p-20) * (F(2) * largest + size);   // infinite scores: not sure either
            }
            before = m;
            if (j == a.k) break;
        }
        int at = 1 << 30;
        if (m > Minus<F>::inf()) {
#pragma unroll
            for (int v = VALUES - 1; v >= 0; --v) at = rank[v] == m ? v * LANES + lane : at;
        }
        at = lanes_min<LANES>(at);
        F won = F(0);
#pragma unroll
        for (int v = 0; v < VALUES; ++v)
            if (at == v * LANES + lane) {
                rank[v] = Minus<F>::inf();
                won = s[v];
            }
        won = __shfl(won, at & (LANES - 1), LANES);
        if (lane == j && at < a.E) {
            *chosen = at;
            *s_chosen = won;
        }
    }
    return __all(sure);
}

template <typename T, int LANES, int VALUES>
__global__ __launch_bounds__(256) void router_kernel(RouterArgs a) {
    constexpr int TOKENS = 256 / LANES;
    __shared__ int hist[512];
    const int lane = threadIdx.x & (LANES - 1);
    if (a.load) {
        for (int e = threadIdx.x; e < a.E; e += 256) hist[e] = 0;
        __syncthreads();
    }
    const long long t = (long long)blockIdx.x * TOKENS + threadIdx.x / LANES;
    const bool there = t < a.T;
    const T* row = reinterpret_cast<const T*>(a.logits) + (there ? t : 0) * a.ld;
    float l[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        const int e = v * LANES + lane;
        l[v] = there && e < a.E ? load_logit(row + e) : -__builtin_inff();
    }
    int chosen;
    float s;
    if (!choose<float, LANES, VALUES>(a, l, &s, &chosen)) {
        double s64;
        choose<double, LANES, VALUES>(a, l, &s64, &chosen);
        s = (float)s64;
    }
    float w = s;
    if (a.renorm) {
        // Scores that are all tiny are scaled up together before they are divided by their sum.
        const float mine = chosen >= 0 ? Elem<T>::ld(row + chosen) : -__builtin_inff();
        float m = lanes_max<LANES>(mine);
        if (a.sigmoid) {
            const float shift = fminf(m, 0.0f);
            w = mine >= 0.0f ? 1.0f / (1.0f + __expf(-mine)) : __expf(mine - shift) / (1.0f + __expf(mine));
        } else {
            w = mine == m ? 1.0f : __expf(mine - m);
        }
        if (chosen < 0) w = 0.0f;
        const float sum = lanes_sum<LANES>(w);
        w = sum > 0.0f ? w / sum : 0.0f;
    }
    if (there && lane < a.k) {
        a.idx[t * a.k + lane] = chosen;
        a.w[t * a.k + lane] = w * a.scale;
        if (a.load && chosen >= 0) atomicAdd(&hist[chosen], 1);           // whole numbers: the order does not matter
    }
    if (a.load) {
        __syncthreads();
        for (int e = threadIdx.x; e < a.E; e += 256)
            if (hist[e]) atomicAdd(&a.load[e], hist[e]);
    }
}

struct RouterBwdArgs {
    const void* logits; const int* idx; const float* dw; void* dl;
    long long ld;
    int T, E, k, sigmoid, renorm;
    float scale;
};

// Lane j of a token holds its j-th choice: expert, logit and weight gradient.  Only a softmax over all experts needs the
// other logits.
template <typename T, int LANES, int VALUES>
__global__ __launch_bounds__(256) void router_bwd_kernel(RouterBwdArgs a) {
    constexpr int TOKENS = 256 / LANES;
    const int lane = threadIdx.x & (LANES - 1);
    const long long t = (long long)blockIdx.x * TOKENS + threadIdx.x / LANES;
    const bool there = t < a.T;
    const T* row = reinterpret_cast<const T*>(a.logits) + (there ? t : 0) * a.ld;
    const bool full = !a.sigmoid && !a.renorm;
    float l[VALUES];
    if (full) {
#pragma unroll
        for (int v = 0; v < VALUES; ++v) {
            const int e = v * LANES + lane;
            l[v] = there && e < a.E ? load_logit(row + e) : -__builtin_inff();
        }
    }
    int mine = there && lane < a.k ? a.idx[t * a.k + lane] : -1;
    if ((unsigned)mine >= (unsigned)a.E) mine = -1;
    float d = mine >= 0 ? a.dw[t * a.k + lane] * a.scale : 0.0f;
    float g = 0.0f;                                    // what the lane's choice contributes to its logit's gradient
    float sub = 0.0f;                                  // softmax over all: sum of ds * s
    if (!full) {
        const float z = mine >= 0 ? load_logit(row + mine) : -__builtin_inff();
        const bool open = z > -__builtin_inff();
        if (!a.renorm) {
            // s (1 - s) = e / (1 + e)^2, e = exp(-|l|)
            const float e = __expf(-fabsf(z)), q = 1.0f + e;
            g = open ? d * (e / (q * q)) : 0.0f;
        } else {
            const float m = lanes_max<LANES>(z);
            float w;
            if (a.sigmoid) {
                const float shift = fminf(m, 0.0f);
                w = z >= 0.0f ? 1.0f / (1.0f + __expf(-z)) : __expf(z - shift) / (1.0f + __expf(z));
            } else {
                w = z == m ? 1.0f : __expf(z - m);
            }
            if (!open) w = 0.0f;
            const float sum = lanes_sum<LANES>(w);
            w = sum > 0.0f ? w / sum : 0.0f;
            const float inner = lanes_sum<LANES>(open ? w * d : 0.0f);
            g = open ? w * (d - inner) : 0.0f;
            if (a.sigmoid) g *= 1.0f / (1.0f + __expf(z));             // ds/dl = s (1 - s)
            if (!open) g = 0.0f;
        }
    } else {
        float largest;
        float s[VALUES];
        scores_of<float, LANES, VALUES>(l, 0, s, &largest);
#pragma unroll
        for (int v = 0; v < VALUES; ++v) l[v] = s[v];
        g = d;
    }
    float ds[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) ds[v] = 0.0f;
    for (int j = 0; j < a.k; ++j) {
        const int e = __shfl(mine, j, LANES);
        const float q = __shfl(g, j, LANES);
#pragma unroll
        for (int v = 0; v < VALUES; ++v)
            if (e == v * LANES + lane) ds[v] = q;
    }
    if (full) {
#pragma unroll
        for (int v = 0; v < VALUES; ++v) sub = fmaf(ds[v], l[v], sub);
        sub = lanes_sum<LANES>(sub);
#pragma unroll
        for (int v = 0; v < VALUES; ++v) ds[v] = l[v] * (ds[v] - sub);
    }
    if (!there) return;
    T* out = reinterpret_cast<T*>(a.dl) + t * a.ld;
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        const int e = v * LANES + lane;
        if (e < a.E) Elem<T>::st(out + e, ds[v]);
    }
}

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

// Sixteen lanes to a token (as many as there may be choices and groups), as many values as the experts need.
#define ROUTER_BY_EXPERTS(E, LAUNCH) do { \
        if ((E) <= 16) { LAUNCH(16, 1); } else if ((E) <= 32) { LAUNCH(16, 2); } else if ((E) <= 64) { LAUNCH(16, 4); } \
        else if ((E) <= 128) { LAUNCH(16, 8); } else if ((E) <= 256) { LAUNCH(16, 16); } else { LAUNCH(16, 32); } } while (0)

template <typename T> void router_launch(const RouterArgs& a, hipStream_t s) {
#define ROUTER_LAUNCH(L, V) router_kernel<T, L, V><<<(a.T + 256 / L - 1) / (256 / L), 256, 0, s>>>(a)
    ROUTER_BY_EXPERTS(a.E, ROUTER_LAUNCH);
#undef ROUTER_LAUNCH
}
template <typename T> void router_bwd_launch(const RouterBwdArgs& a, hipStream_t s) {
#define ROUTER_LAUNCH(L, V) router_bwd_kernel<T, L, V><<<(a.T + 256 / L - 1) / (256 / L), 256, 0, s>>>(a)
    ROUTER_BY_EXPERTS(a.E, ROUTER_LAUNCH);
#undef ROUTER_LAUNCH
}

}  // namespace

}  // namespace moe

extern "C" moe_status moe_router_fwd(const moe_router_config* cfg, const void* logits, const float* bias, int32_t* topk_idx,
                                     float* topk_w, int32_t* load, void* stream) {
    MOE_TRY(moe::router_check(cfg));
    if (cfg->T == 0) return MOE_OK;
    if (!logits || !topk_idx || !topk_w) return MOE_ERR_NULL;
    const unsigned per = (unsigned)(cfg->E / cfg->groups);
    moe::RouterArgs a = {logits, bias, topk_idx, topk_w, load, cfg->ld ? (long long)cfg->ld : (long long)cfg->E, cfg->T, cfg->E, cfg->k,
                         cfg->scores == MOE_SIGMOID, cfg->groups, cfg->group_k, cfg->group_top, cfg->renormalize, per,
                         ((1u << 20) + per - 1) / per, cfg->scale};
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_ROUTER, s);
        if (cfg->dtype == MOE_F32) moe::router_launch<float>(a, s); else moe::router_launch<moe::bf16_t>(a, s);
    }
    MOE_CHECK_LAUNCH();
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

extern "C" moe_status moe_router_bwd(const moe_router_config* cfg, const void* logits, const int32_t* topk_idx, const float* dw,
                                     void* dlogits, void* stream) {
    MOE_TRY(moe::router_check(cfg));
    if (cfg->T == 0) return MOE_OK;
    if (!logits || !topk_idx || !dw || !dlogits) return MOE_ERR_NULL;
    moe::RouterBwdArgs a = {logits, topk_idx, dw, dlogits, cfg->ld ? (long long)cfg->ld : (long long)cfg->E, cfg->T, cfg->E, cfg->k,
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
