// The whole expert layer for a few tokens: gate, router, both expert products, weighted sum.  Nothing has a capacity.
//
//   logits = x Wg + gate_bias;  the router's choices and weights (router.hip);
//   a[t,j] = gelu(x[t] W1[e]),  y[t] = sum over j of w[t,j] a[t,j] W2[e],  e = topk_idx[t,j]
//
// What has to move are the chosen experts' weights, 2 M H elements each, once.  Both products go through few_rows.h: a
// workgroup has 64 columns of one expert and all of the rows that chose it.  The logits are sums in 64 bits, rounded to float:
// which expert is chosen hangs on their last bits.  The rows between the products are kept in float, or as two bfloat16 that add up
// to 16 bits of mantissa, which costs the matrix pipe a second instruction where it waits for memory anyway: nothing is rounded to
// the storage type but y.
#include "common.h"
#include "few_rows.h"
#include "wide.h"

namespace moe {

namespace {

constexpr int FEW_TOKENS = 256, FEW_K = 16, FEW_E = 512;
constexpr int FEW_WAVES = 8, FEW_THREADS = 64 * FEW_WAVES;

struct FewArgs {
    const void* x; const void* Wg; const float* gate_bias; const void* W1; const void* W2; void* y;
    float* logits; const int* idx; const float* w;
    void* a;                                 // [T*k, H] float, or twice that in bfloat16, the upper parts first
    float* partial;                          // [slices][T*k][M]
    long long ldx, ldy;
    int T, M, H, E, k, slices, steps;        // of the second product: slices of H, steps of a slice
};

// ---- gate -------------------------------------------------------------------------------------------------
// A workgroup has one or two tokens and 64 experts: a lane eight of them (fewer lanes to a row of Wg where there are fewer experts),
// the lanes and wavefronts share out the rows of Wg.
constexpr int GATE_TOKENS = 2, GATE_WAVES = 16;

template <typename T> __device__ __forceinline__ void load_eight(const T* p, int left, bool wide, float* o) {
    if (wide) {
        Raw8<T> r;
        r.load(p);
        r.to_float(o);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = i < left ? Elem<T>::ld(p + i) : 0.0f;
    }
}

template <typename T, int TOKENS>
__global__ __launch_bounds__(GATE_WAVES * 64) void few_gate_kernel(FewArgs a) {
    __shared__ double s_sum[GATE_WAVES][TOKENS][64];
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const int e_first = blockIdx.x * 64, experts = a.E - e_first < 64 ? a.E - e_first : 64;
    int chunks = 1;                                        // lanes to a row
    while (chunks * 8 < experts) chunks *= 2;
    const int chunk = lane & (chunks - 1), rows = 64 / chunks, e0 = e_first + chunk * 8, left = a.E - e0;
    const bool wide = a.E % 8 == 0 && left >= 8;
    const int t0 = blockIdx.y * TOKENS;
    double sum[TOKENS][8];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[t][i] = 0.0;
    if (left > 0) {
        // so many rows of a lane are requested before the first is multiplied
        constexpr int AT_ONCE = 4;
        const int step = GATE_WAVES * rows;
        for (int m0 = wid * rows + lane / chunks; m0 < a.M; m0 += AT_ONCE * step) {
            float w[AT_ONCE][8], x[AT_ONCE][TOKENS];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int m = m0 + u * step;
                if (m < a.M) {
                    load_eight(reinterpret_cast<const T*>(a.Wg) + (long long)m * a.E + e0, left, wide, w[u]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[u][i] = 0.0f;
                }
#pragma unroll
                for (int t = 0; t < TOKENS; ++t)
                    x[u][t] = m < a.M && t0 + t < a.T ? Elem<T>::ld(reinterpret_cast<const T*>(a.x) + (t0 + t) * a.ldx + m) : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double v = (double)w[u][i];
#pragma unroll
                    for (int t = 0; t < TOKENS; ++t) sum[t][i] = fma((double)x[u][t], v, sum[t][i]);
                }
        }
    }
    for (int off = chunks; off < 64; off *= 2)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[t][i] += __shfl_xor(sum[t][i], off, 64);
    if (lane < chunks) {
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
#pragma unroll
            for (int i = 0; i < 8; ++i) s_sum[wid][t][lane * 8 + i] = sum[t][i];
    }
    __syncthreads();
    const int t = threadIdx.x / 64, e = threadIdx.x & 63;
    if (t < TOKENS && t0 + t < a.T && e < experts) {
        double v = 0.0;
        for (int q = 0; q < GATE_WAVES; ++q) v += s_sum[q][t][e];
        if (a.gate_bias) v += (double)a.gate_bias[e_first + e];
        a.logits[(long long)(t0 + t) * a.E + e_first + e] = (float)v;
    }
}

// ---- which rows ---------------------------------------------------------------------------------------------
struct FewPlan {
    int idx[FEW_TOKENS * FEW_K];
    int rows[FEW_TOKENS];                    // assignments with the workgroup's expert, ascending
    unsigned there[FEW_E / 32];              // experts that are chosen
    int expert, n_rows, n_experts;
};
// Fills `p` for the `slot`-th of the chosen experts (expert -1: there are fewer).  Every thread comes here.
__device__ __forceinline__ void few_plan(const FewArgs& a, int slot, FewPlan& p) {
    const int n = a.T * a.k, tid = threadIdx.x;
    if (tid < FEW_E / 32) p.there[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += blockDim.x) {
        const int e = a.idx[i];
        p.idx[i] = e;
        if (e >= 0) atomicOr(&p.there[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
    if (tid < 64) {
        // lane l has the experts 32 l .. + 31; which lane has the slot-th, and where in it
        const unsigned mine = tid < FEW_E / 32 ? p.there[tid] : 0;
        const int count = __popc(mine);
        int end = count;
#pragma unroll
        for (int off = 1; off < FEW_E / 32; off <<= 1) {
            const int o = __shfl_up(end, off, 64);
            if (tid >= off) end += o;
        }
        const int all = __shfl(end, FEW_E / 32 - 1, 64);
        int expert = -1;
        if (tid < FEW_E / 32 && slot >= end - count && slot < end) {
            unsigned bits = mine;
            for (int q = slot - (end - count); q > 0; --q) bits &= bits - 1;
            expert = tid * 32 + __builtin_ctz(bits);
        }
        const unsigned long long who = __ballot(expert >= 0);
        expert = who ? __shfl(expert, __builtin_ctzll(who), 64) : -1;
        int rows = 0;
        if (expert >= 0) {
            for (int base = 0; base < n; base += 64) {
                const bool is = base + tid < n && p.idx[base + tid] == expert;
                const unsigned long long b = __ballot(is);
                if (is) p.rows[rows + __popcll(b & ((1ull << tid) - 1))] = base + tid;
                rows += __popcll(b);
            }
        }
        if (tid == 0) { p.expert = expert; p.n_rows = rows; p.n_experts = all; }
    }
    __syncthreads();
}

__device__ __forceinline__ float gelu_of(float z) { return 0.5f * z * erfcf(-0.70710678118654752440f * z); }

// ---- first product ----------------------------------------------------------------------------------------------
template <typename T, int GROUPS>
__global__ __launch_bounds__(FEW_THREADS) void few_first_kernel(FewArgs a) {
    __shared__ FewSums<T, FEW_WAVES> sums;
    __shared__ FewPlan plan;
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, n0 = blockIdx.x * FEW_COLS;
    few_plan(a, blockIdx.y, plan);
    if (plan.expert < 0) return;
    constexpr int ROWS = Few<T>::ROWS;
    const T* W = reinterpret_cast<const T*>(a.W1) + (long long)plan.expert * a.M * a.H + n0;
    const long long size = (long long)a.T * a.k * a.H;
    for (int r0 = 0; r0 < plan.n_rows; r0 += GROUPS * ROWS) {
        const T* row[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int r = r0 + g * ROWS + Few<T>::row(lane);
            row[g] = reinterpret_cast<const T*>(a.x) + plan.rows[r < plan.n_rows ? r : r0] / a.k * a.ldx;
        }
        few_acc acc[GROUPS][Few<T>::ACCS];
        few_sums<T, GROUPS, 1, FEW_WAVES>(W, a.H, a.H - n0, row, 0, a.M, wid, (a.M + Few<T>::STEP - 1) / Few<T>::STEP, acc);
        few_finish<T, GROUPS, FEW_WAVES>(sums, acc, plan.n_rows - r0, a.H - n0, [&](int r, int n, float z) {
            const float v = gelu_of(z);
            const long long at = (long long)plan.rows[r0 + r] * a.H + n0 + n;
            if constexpr (sizeof(T) == 4) {
                reinterpret_cast<float*>(a.a)[at] = v;
            } else {
                const bf16_t hi = f32_to_bf16(v);
                const float h = bf16_to_f32(hi);
                reinterpret_cast<bf16_t*>(a.a)[at] = hi;
                // (an infinity has no rest)
                reinterpret_cast<bf16_t*>(a.a)[size + at] = (__float_as_uint(h) & 0x7f800000u) == 0x7f800000u ? 0 : f32_to_bf16(v - h);
            }
        });
    }
}

// ---- second product ----------------------------------------------------------------------------------------------
// A workgroup has 64 columns of an expert and a slice of H.  It leaves its rows' sums, which few_join_kernel adds up: a launch of its
// own, since making sums visible from one workgroup to another of the same launch empties the caches of eight dies (the last
// workgroup of a column block to finish, adding them up: 89 us for what takes 14 without).
template <typename T, int GROUPS>
__global__ __launch_bounds__(FEW_THREADS) void few_second_kernel(FewArgs a) {
    __shared__ FewSums<T, FEW_WAVES> sums;
    __shared__ FewPlan plan;
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, n0 = blockIdx.x * FEW_COLS;
    few_plan(a, blockIdx.y, plan);
    if (plan.expert < 0) return;
    constexpr int ROWS = Few<T>::ROWS, PARTS = sizeof(T) == 2 ? 2 : 1;
    const T* W = reinterpret_cast<const T*>(a.W2) + (long long)plan.expert * a.H * a.M + n0;
    const int all = (a.H + Few<T>::STEP - 1) / Few<T>::STEP, begin = blockIdx.z * a.steps, end = begin + a.steps < all ? begin + a.steps : all;
    const long long size = (long long)a.T * a.k * a.H;
    float* partial = a.partial + (long long)blockIdx.z * a.T * a.k * a.M;
    for (int r0 = 0; r0 < plan.n_rows; r0 += GROUPS * ROWS) {
        const T* row[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int r = r0 + g * ROWS + Few<T>::row(lane);
            row[g] = reinterpret_cast<const T*>(a.a) + (long long)plan.rows[r < plan.n_rows ? r : r0] * a.H;
        }
        few_acc acc[GROUPS][Few<T>::ACCS];
        few_sums<T, GROUPS, PARTS, FEW_WAVES>(W, a.M, a.M - n0, row, size, a.H, begin + wid, end, acc);
        few_finish<T, GROUPS, FEW_WAVES>(sums, acc, plan.n_rows - r0, a.M - n0,
                                         [&](int r, int n, float v) { partial[(long long)plan.rows[r0 + r] * a.M + n0 + n] = v; });
    }
}

// y[t] = sum over the choices of w times the sum of their slices; four columns to a thread, the slices' loads in eights
constexpr int JOIN_THREADS = 64;
template <typename T> __global__ __launch_bounds__(JOIN_THREADS) void few_join_kernel(FewArgs a) {
    const int t = blockIdx.y, n = (blockIdx.x * JOIN_THREADS + threadIdx.x) * 4;
    if (n >= a.M) return;
    const long long step = (long long)a.T * a.k * a.M;
    float4 y = make_float4(0, 0, 0, 0);
    for (int j = 0; j < a.k; ++j) {
        const int at = t * a.k + j;
        if (a.idx[at] < 0) continue;                      // (nothing was written for it)
        const float w = a.w[at];
        const float* p = a.partial + (long long)at * a.M + n;
        float4 v = make_float4(0, 0, 0, 0);
        for (int s0 = 0; s0 < a.slices; s0 += 8) {
            float4 o[8];
#pragma unroll
            for (int s = 0; s < 8; ++s)
                if (s0 + s < a.slices) o[s] = *reinterpret_cast<const float4*>(p + (s0 + s) * step);
#pragma unroll
            for (int s = 0; s < 8; ++s)
                if (s0 + s < a.slices) { v.x += o[s].x; v.y += o[s].y; v.z += o[s].z; v.w += o[s].w; }
        }
        y.x = fmaf(w, v.x, y.x); y.y = fmaf(w, v.y, y.y); y.z = fmaf(w, v.z, y.z); y.w = fmaf(w, v.w, y.w);
    }
    const float o[4] = {y.x, y.y, y.z, y.w};
    store_columns(reinterpret_cast<T*>(a.y) + t * a.ldy + n, o, 4);
}

struct FewDims {
    moe_router_config router;
    int slots, slices, steps;                // experts that may be chosen; of the second product
    size_t a_bytes, partial_bytes;
};
int up(long long a, long long b) { return (int)((a + b - 1) / b); }
size_t align16(size_t b) { return (b + 15) & ~(size_t)15; }

moe_status few_dims(const moe_few_config* c, FewDims* d) {
    if (!c) return MOE_ERR_NULL;
    if (c->T < 0 || c->M <= 0 || c->H <= 0) return MOE_ERR_SHAPE;
    d->router = {c->T, c->E, c->k, c->scores, c->groups, c->group_k, c->group_top, c->renormalize, c->scale, MOE_F32, 0};
    MOE_TRY(router_check(&d->router));
    if ((c->ldx && c->ldx < c->M) || (c->ldy && c->ldy < c->M)) return MOE_ERR_SHAPE;
    if (c->dtype != MOE_F32 && c->dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (c->T > FEW_TOKENS || c->M % 8 || c->H % 8 || c->ldx % 8) return MOE_ERR_UNSUPPORTED;
    if (c->M > (1 << 20) || c->H > (1 << 20)) return MOE_ERR_UNSUPPORTED;
    const bool bf16 = c->dtype == MOE_BF16;
    const long long n = (long long)c->T * c->k;
    d->slots = (int)(n < c->E ? n : c->E);
    if (d->slots < 1) d->slots = 1;
    const int step = bf16 ? 64 : 32, steps = up(c->H, step), blocks = up(c->M, FEW_COLS) * d->slots;
    int slices = blocks < 512 ? up(512, blocks) : 1;
    const int most = up(steps, FEW_WAVES);
    if (slices > most) slices = most;
    d->steps = up(steps, slices);
    d->slices = up(steps, d->steps);
    d->a_bytes = align16((size_t)n * c->H * 4);
    d->partial_bytes = align16((size_t)n * c->M * d->slices * 4);
    return MOE_OK;
}

template <typename T> moe_status few_launch(const FewArgs& a, const FewDims& d, hipStream_t s, const float* bias, int* idx, float* w) {
    if (a.T == 1) few_gate_kernel<T, 1><<<dim3(up(a.E, 64), 1), GATE_WAVES * 64, 0, s>>>(a);
    else few_gate_kernel<T, GATE_TOKENS><<<dim3(up(a.E, 64), up(a.T, GATE_TOKENS)), GATE_WAVES * 64, 0, s>>>(a);
    MOE_CHECK_LAUNCH();
    MOE_TRY(router_run(&d.router, a.logits, bias, idx, w, nullptr, s));
    // Groups of rows that go through together: as many as an expert is expected to have, and some more.
    const int mean = up((long long)a.T * a.k, a.E), groups = up(mean + (mean > 1 ? up(mean, 2) : 0), Few<T>::ROWS);
    const dim3 first(up(a.H, FEW_COLS), d.slots), second(up(a.M, FEW_COLS), d.slots, a.slices);
    if (groups <= 1) {
        few_first_kernel<T, 1><<<first, FEW_THREADS, 0, s>>>(a);
        few_second_kernel<T, 1><<<second, FEW_THREADS, 0, s>>>(a);
    } else if (groups <= 2) {
        few_first_kernel<T, 2><<<first, FEW_THREADS, 0, s>>>(a);
        few_second_kernel<T, 2><<<second, FEW_THREADS, 0, s>>>(a);
    } else {
        few_first_kernel<T, 4><<<first, FEW_THREADS, 0, s>>>(a);
        few_second_kernel<T, 4><<<second, FEW_THREADS, 0, s>>>(a);
    }
    MOE_CHECK_LAUNCH();
    few_join_kernel<T><<<dim3(up(a.M, 4 * JOIN_THREADS), a.T), JOIN_THREADS, 0, s>>>(a);
    MOE_CHECK_LAUNCH();
    return MOE_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

}  // namespace moe

extern "C" moe_status moe_few_scratch_bytes(const moe_few_config* cfg, size_t* bytes) {
    moe::FewDims d;
    MOE_TRY(moe::few_dims(cfg, &d));
    if (!bytes) return MOE_ERR_NULL;
    *bytes = cfg->T == 0 ? 0 : d.a_bytes + d.partial_bytes;
    return MOE_OK;
}

extern "C" moe_status moe_few_forward(const moe_few_config* cfg, const void* x, const void* Wg, const float* gate_bias, const float* bias,
                                      const void* W1, const void* W2, void* y, float* logits, int32_t* topk_idx, float* topk_w,
                                      void* scratch, void* stream) {
    moe::FewDims d;
    MOE_TRY(moe::few_dims(cfg, &d));
    if (cfg->T == 0) return MOE_OK;
    if (!x || !Wg || !W1 || !W2 || !y || !logits || !topk_idx || !topk_w || !scratch) return MOE_ERR_NULL;
    if (!moe::aligned16(x) || !moe::aligned16(Wg) || !moe::aligned16(W1) || !moe::aligned16(W2) || !moe::aligned16(scratch)) return MOE_ERR_UNSUPPORTED;
    char* p = (char*)scratch;
    moe::FewArgs a = {x, Wg, gate_bias, W1, W2, y, logits, topk_idx, topk_w, p, (float*)(p + d.a_bytes),
                      cfg->ldx ? (long long)cfg->ldx : cfg->M, cfg->ldy ? (long long)cfg->ldy : cfg->M,
                      cfg->T, cfg->M, cfg->H, cfg->E, cfg->k, d.slices, d.steps};
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_FEW, s);
        MOE_TRY(cfg->dtype == MOE_BF16 ? moe::few_launch<moe::bf16_t>(a, d, s, bias, topk_idx, topk_w)
                                       : moe::few_launch<float>(a, d, s, bias, topk_idx, topk_w));
    }
    moe::count_launch(moe::LC_GEMM, 2);
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}
