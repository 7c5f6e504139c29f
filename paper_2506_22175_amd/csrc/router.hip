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
#include "router_choose.h"
#include "wide.h"
#include <cmath>

namespace moe {

namespace {

constexpr int BLOCK = 512;

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
    const float w = choice_weight(a, chosen, z, soft);
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

}  // namespace moe

extern "C" moe_status moe_router_fwd(const moe_router_config* cfg, const void* logits, const float* bias, int32_t* topk_idx,
                                     float* topk_w, int32_t* load, void* stream) {
    MOE_TRY(moe::router_check(cfg));
    if (cfg->T == 0) return MOE_OK;
    if (!logits || !topk_idx || !topk_w) return MOE_ERR_NULL;
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_ROUTER, s);
        const int values = moe::router_values(cfg->E);
        const moe::RouterArgs a = moe::router_args(cfg, logits, bias, topk_idx, topk_w, load, values, (values + 3) / 4);
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
