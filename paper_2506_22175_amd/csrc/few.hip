// The whole expert layer for a few tokens: gate, router, both expert products, weighted sum.  Nothing has a capacity.
//
//   logits = x Wg + gate_bias;  the router's choices and weights (router.hip);
//   a[t,j] = gelu(x[t] W1[e]),  y[t] = sum over j of w[t,j] a[t,j] W2[e],  e = topk_idx[t,j]
//
// What has to move are the chosen experts' weights, 2 M H elements each, once.  Both products go through few_rows.h: a
// workgroup has 128 columns (float: 64) of one expert, or half as many, and all of the rows that chose it.  The logits are sums in 64 bits, rounded to float:
// which expert is chosen hangs on their last bits.  The rows between the products are kept in float, or as two bfloat16 that add up
// to 16 bits of mantissa, which costs the matrix pipe a second instruction where it waits for memory anyway: nothing is rounded to
// the storage type but y.
//
// One token, 2 of 16 experts of 2048/8192 in bfloat16 (134 MB, at the 7 TB/s of a read 19 us): 38 us, of which the first product 20
// (3.9 of gate and router in front of its 67 MB), the second 14.8, the join 4.  48 tokens, 4 of 64 experts of 1024/4096 (1.03 GB): 151 us,
// 6.8 TB/s; the products alone 55 to 61 and 71 to 77.  Seven tokens of 520/1000 in float (67 MB): 35 us, two steps to a wavefront and the way to
// the first of them, five times over.
#include "common.h"
#include "few_rows.h"
#include "router_choose.h"
#include "wide.h"

namespace moe {

namespace {

constexpr int FEW_TOKENS = 256, FEW_K = 16, FEW_E = 512;
constexpr int FEW_WAVES = 8;

struct FewArgs {
    const void* x; const void* Wg; const float* gate_bias; const void* W1; const void* W2; void* y;
    float* logits;
    RouterArgs route;                        // where choices and weights go, among others
    double* gate_part;                       // [gate_slices][T][E]
    int gate_slices, gate_rows;              // slices of the rows of Wg, rows of each
    void* a;                                 // [T*k, H] float, or twice that in bfloat16, the upper parts first
    float* partial;                          // [slices][T*k][M]
    long long ldx, ldy;
    int T, M, H, E, k, slices, steps;        // of the second product: slices of H, steps of a slice
};

// ---- gate -------------------------------------------------------------------------------------------------
// TOKENS tokens' sums of x Wg over the rows [m0, m1), of 64 experts from e_first on, for each of WAVES wavefronts into `out`: a lane
// has eight experts (there are fewer lanes to a row of Wg where there are fewer experts), and the lanes and wavefronts share out
// the rows.  Bound by the way to Wg, which the next caches have after the first workgroup: eight rows of a lane are under way at once.  A lane's eight sums are dealt out to the lanes that have the same experts while they are added.
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
template <typename T, int TOKENS, int WAVES>
__device__ __forceinline__ void gate_sums(const FewArgs& a, int t0, int e_first, int m0, int m1, double (&out)[WAVES][TOKENS][64]) {
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const int experts = a.E - e_first < 64 ? a.E - e_first : 64;
    int chunks = 1;                                        // lanes to a row
    while (chunks * 8 < experts) chunks *= 2;
    const int chunk = lane & (chunks - 1), rows = 64 / chunks, e0 = e_first + chunk * 8, left = a.E - e0;
    const bool wide = a.E % 8 == 0;
    double sum[TOKENS][8];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[t][i] = 0.0;
    if (left > 0) {
        // so many rows of a lane are requested before the first is multiplied
        constexpr int AT_ONCE = TOKENS == 1 && sizeof(T) == 2 ? 8 : 4;
        const int step = WAVES * rows;
        for (int mm = m0 + wid * rows + lane / chunks; mm < m1; mm += AT_ONCE * step) {
            float w[AT_ONCE][8], x[AT_ONCE][TOKENS];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int m = mm + u * step;
                if (m < m1) {
                    load_eight(reinterpret_cast<const T*>(a.Wg) + (long long)m * a.E + e0, left, wide, w[u]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[u][i] = 0.0f;
                }
#pragma unroll
                for (int t = 0; t < TOKENS; ++t)
                    x[u][t] = m < m1 && t0 + t < a.T ? Elem<T>::ld(reinterpret_cast<const T*>(a.x) + (t0 + t) * a.ldx + m) : 0.0f;
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
    int mine = 0;                                          // which of the eight the lane ends up with
#pragma unroll
    for (int half = 4; half > 0; half >>= 1) {
        const int off = chunks * (4 / half);
        const bool up = (lane & off) != 0;
        mine += up ? half : 0;
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
#pragma unroll
            for (int i = 0; i < half; ++i) {
                const double keep = up ? sum[t][half + i] : sum[t][i], give = up ? sum[t][i] : sum[t][half + i];
                sum[t][i] = keep + __shfl_xor(give, off, 64);
            }
    }
    for (int off = chunks * 8; off < 64; off *= 2)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) sum[t][0] += __shfl_xor(sum[t][0], off, 64);
    if (lane < chunks * 8) {
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) out[wid][t][chunk * 8 + mine] = sum[t][0];
    }
}

// By many workgroups: each has one or two tokens, 64 experts and a slice of the rows of Wg, whose sums it leaves in gate_part.  (48 tokens,
// 1024 x 64: 4.9 us, and the router's launch 4.7.  Both in one, a workgroup of 16 wavefronts to a token: the whole call 151 us either way, 1 to 3 us
// less for 256 tokens, but 37.9 us instead of 35.5 for 7 x 33 of 520/1000, and 74.6 instead of 65.0 where Wg is 4096 x 64.)
constexpr int GATE_TOKENS = 2, GATE_WAVES = 8;
template <typename T, int TOKENS>
__global__ __launch_bounds__(GATE_WAVES * 64) void few_gate_kernel(FewArgs a) {
    __shared__ double s_sum[GATE_WAVES][TOKENS][64];
    const int e_first = blockIdx.x * 64, t0 = blockIdx.y * TOKENS, m0 = blockIdx.z * a.gate_rows;
    gate_sums<T, TOKENS, GATE_WAVES>(a, t0, e_first, m0, m0 + a.gate_rows < a.M ? m0 + a.gate_rows : a.M, s_sum);
    __syncthreads();
    const int t = threadIdx.x / 64, e = threadIdx.x & 63;
    if (t < TOKENS && t0 + t < a.T && e_first + e < a.E) {
        double v = 0.0;
#pragma unroll
        for (int q = 0; q < GATE_WAVES; ++q) v += s_sum[q][t][e];
        a.gate_part[((long long)blockIdx.z * a.T + t0 + t) * a.E + e_first + e] = v;
    }
}

// ---- router -----------------------------------------------------------------------------------------------
// A token's choices and weights by a wavefront whose lanes have its logits' sums, VALUES neighbouring experts each: lane j returns the
// j-th in *weight and as its result.  `record`: logits, choices and weights are written down.
template <int VALUES> __device__ __forceinline__ int route_token(const FewArgs& a, int t, const double* sum, bool record, float* weight) {
    const int lane = threadIdx.x & 63, e0 = lane * VALUES;
    float l[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        l[v] = -__builtin_inff();
        if (e0 + v < a.E) {
            l[v] = (float)(a.gate_bias ? sum[v] + (double)a.gate_bias[e0 + v] : sum[v]);
            if (record) a.logits[(long long)t * a.E + e0 + v] = l[v];
            if (l[v] != l[v]) l[v] = -__builtin_inff();
        }
    }
    Softmax<float> soft = {0.0f, 0.0f};
    const int chosen = choose_exactly<VALUES>(a.route, l, &soft);
    float z = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        const float o = __shfl(l[v], chosen < 0 ? 0 : chosen / VALUES, 64);
        z = chosen >= 0 && chosen % VALUES == v ? o : z;
    }
    *weight = choice_weight(a.route, chosen, z, soft) * a.route.scale;
    if (record && lane < a.k) {
        a.route.idx[t * a.k + lane] = chosen;
        a.route.w[t * a.k + lane] = *weight;
    }
    return chosen;
}
// The sums of a lane's experts, from the gate's slices.
template <int VALUES> __device__ __forceinline__ void gate_total(const FewArgs& a, int t, double* sum) {
    const int e0 = (threadIdx.x & 63) * VALUES;
#pragma unroll
    for (int v = 0; v < VALUES; ++v) sum[v] = 0.0;
    const double* p = a.gate_part + (long long)t * a.E + e0;
    const long long step = (long long)a.T * a.E;
    for (int s0 = 0; s0 < a.gate_slices; s0 += 4) {
        double o[4][VALUES];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int v = 0; v < VALUES; ++v) o[s][v] = s0 + s < a.gate_slices && e0 + v < a.E ? p[(s0 + s) * step + v] : 0.0;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int v = 0; v < VALUES; ++v) sum[v] += o[s][v];
    }
}
// A wavefront to a token
template <int VALUES> __global__ __launch_bounds__(64) void few_route_kernel(FewArgs a) {
    double sum[VALUES];
    float weight;
    gate_total<VALUES>(a, blockIdx.x, sum);
    route_token<VALUES>(a, blockIdx.x, sum, true, &weight);
}

// ---- which rows ---------------------------------------------------------------------------------------------
struct FewPlan {
    int rows[FEW_TOKENS];                    // assignments with the workgroup's expert, ascending
    unsigned there[FEW_E / 32];              // experts that are chosen
    int expert, n_rows, n_experts;
};
// What a workgroup has in LDS: the choices, which only the plan looks at, then the sums.
template <typename T, bool NARROW = false> struct FewLds {
    FewPlan plan;
    union { int idx[FEW_TOKENS * FEW_K]; FewSums<T, FEW_WAVES, NARROW> sums; };
};
// The workgroup's expert, the slot-th of those that are chosen (-1: there are fewer), how many are, and how many assignments it has,
// which are in FewPlan::rows.
struct FewPick { int expert, n_rows, n_experts; };

// Up to 32 assignments, whose choices the lanes of every wavefront have: each finds out by itself, and writes down the same (0.6 to 0.9 us of
// the call sooner than through LDS).
constexpr int FEW_IN_LANES = 32;
__device__ __forceinline__ FewPick few_pick(int e, int slot, FewPlan& p) {
    const int lane = threadIdx.x & 63;
    FewPick pick = {-1, 0, 0};
    unsigned long long left = __ballot(e >= 0), rows = 0;
    while (left) {
        const int one = __builtin_amdgcn_readlane(e, __builtin_ctzll(left));
        const unsigned long long same = __ballot(e == one);
        if (pick.n_experts == slot) { pick.expert = one; rows = same; }
        ++pick.n_experts;
        left &= ~same;
    }
    pick.n_rows = __popcll(rows);
    if (rows >> lane & 1) p.rows[__popcll(rows & ((1ull << lane) - 1))] = lane;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return pick;
}
// More of them, from the choices in LDS.  Every thread comes here.
__device__ __forceinline__ FewPick few_plan(const FewArgs& a, int slot, const int* idx, FewPlan& p) {
    const int n = a.T * a.k, tid = threadIdx.x;
    if (tid < FEW_E / 32) p.there[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += blockDim.x) {
        const int e = idx[i];
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
                const bool is = base + tid < n && idx[base + tid] == expert;
                const unsigned long long b = __ballot(is);
                if (is) p.rows[rows + __popcll(b & ((1ull << tid) - 1))] = base + tid;
                rows += __popcll(b);
            }
        }
        if (tid == 0) { p.expert = expert; p.n_rows = rows; p.n_experts = all; }
    }
    __syncthreads();
    return {__builtin_amdgcn_readfirstlane(p.expert), __builtin_amdgcn_readfirstlane(p.n_rows), __builtin_amdgcn_readfirstlane(p.n_experts)};
}

// Where the choices come from: they are there; or, in the first product, a workgroup routes for itself, which saves the launches between
// it and the gate: from the gate's sums, or from x and Wg (one or two tokens).
enum { FEW_ROUTED = 0, FEW_SUMMED = 1, FEW_ALONE = 2 };
template <typename T, int MODE, bool NARROW> __device__ __forceinline__ FewPick few_choices(const FewArgs& a, int slot, bool record, FewLds<T, NARROW>& lds) {
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = a.T * a.k;
    if constexpr (MODE == FEW_ROUTED) {
        if (n <= FEW_IN_LANES) return few_pick(lane < n ? a.route.idx[lane] : -1, slot, lds.plan);
        for (int i = threadIdx.x; i < n; i += FEW_WAVES * 64) lds.idx[i] = a.route.idx[i];
    } else {
        __shared__ double s_sum[MODE == FEW_ALONE ? FEW_WAVES : 1][2][64];
        if constexpr (MODE == FEW_ALONE) {
            if (a.T == 1) {
                auto& sums = reinterpret_cast<double (&)[FEW_WAVES][1][64]>(s_sum);
                gate_sums<T, 1, FEW_WAVES>(a, 0, 0, 0, a.M, sums);
                __syncthreads();
                double sum = 0.0;
#pragma unroll
                for (int q = 0; q < FEW_WAVES; ++q) sum += sums[q][0][lane];
                float weight;
                return few_pick(route_token<1>(a, 0, &sum, record && wid == 0, &weight), slot, lds.plan);
            }
            gate_sums<T, 2, FEW_WAVES>(a, 0, 0, 0, a.M, s_sum);
            __syncthreads();
        }
        for (int t = wid; t < a.T; t += FEW_WAVES) {
            float weight;
            double sum = 0.0;
            if constexpr (MODE == FEW_ALONE) {
#pragma unroll
                for (int q = 0; q < FEW_WAVES; ++q) sum += s_sum[q][t][lane];
            } else {
                gate_total<1>(a, t, &sum);
            }
            const int chosen = route_token<1>(a, t, &sum, record, &weight);
            if (lane < a.k) lds.idx[t * a.k + lane] = chosen;
        }
        if (n <= FEW_IN_LANES) {
            __syncthreads();
            const int e = lane < n ? lds.idx[lane] : -1;
            __syncthreads();                               // (the sums will lie there)
            return few_pick(e, slot, lds.plan);
        }
    }
    __syncthreads();
    return few_plan(a, slot, lds.idx, lds.plan);
}

__device__ __forceinline__ float gelu_of(float z) { return 0.5f * z * erfcf(-0.70710678118654752440f * z); }

// ---- first product ----------------------------------------------------------------------------------------------
// Bound by the weights' way from memory.  A workgroup has 128 columns (float: 64) of an expert, or with few workgroups half as many, and all of M, as nothing may be added up
// between here and the activation.
template <typename T, int GROUPS, int MODE, bool NARROW>
__global__ __launch_bounds__(FEW_WAVES * 64, GROUPS > 2 ? 2 : 4) void few_first_kernel(FewArgs a) {
    __shared__ FewLds<T, NARROW> lds;
    const FewPlan& plan = lds.plan;
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, n0 = blockIdx.x * Few<T, NARROW>::COLS;
    const FewPick pick = few_choices<T, MODE, NARROW>(a, blockIdx.y, blockIdx.x == 0 && blockIdx.y == 0, lds);
    if (pick.expert < 0) return;
    constexpr int ROWS = Few<T, NARROW>::ROWS;
    const T* W = reinterpret_cast<const T*>(a.W1) + (long long)pick.expert * a.M * a.H + n0;
    const long long size = (long long)a.T * a.k * a.H;
    for (int r0 = 0; r0 < pick.n_rows; r0 += GROUPS * ROWS) {
        const T* const rows[1] = {reinterpret_cast<const T*>(a.x)};
        unsigned row[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int r = r0 + g * ROWS + Few<T, NARROW>::row(lane);
            row[g] = (unsigned)(plan.rows[r < pick.n_rows ? r : r0] / a.k) * (unsigned)a.ldx * (unsigned)sizeof(T);
        }
        few_acc acc[GROUPS][Few<T>::ACCS];
        few_sums<T, GROUPS, 1, FEW_WAVES, NARROW>(W, a.H, a.H - n0, rows, row, a.M, wid, (a.M + Few<T, NARROW>::STEP - 1) / Few<T, NARROW>::STEP, acc);
        few_finish<T, GROUPS, FEW_WAVES, NARROW>(lds.sums, acc, pick.n_rows - r0, a.H - n0, [&](int r, int n, float z) {
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
// A workgroup has 128 columns (float: 64) of an expert and a slice of H.  It leaves its rows' sums, which few_join_kernel adds up: a launch of
// its own.  (The last workgroup of a column block to finish, adding them up: with fences, which write back and empty the caches of
// eight dies, 89 us for what takes 14 without; with stores and loads that go past the caches 44.5 us for the whole of one token, 2048/8192,
// and 37.5 for seven of 520/1000 in float, against 45.1 and 35.5 with the launch.)
// Two groups of bfloat16 rows in two parts need three registers more than two workgroups to a CU have: they are spilled once for 32 rows, outside
// the loop over the steps.
template <typename T, int GROUPS>
__global__ __launch_bounds__(FEW_WAVES * 64, GROUPS > 2 ? 2 : 4) void few_second_kernel(FewArgs a) {
    __shared__ FewLds<T> lds;
    const FewPlan& plan = lds.plan;
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, n0 = blockIdx.x * Few<T>::COLS;
    const FewPick pick = few_choices<T, FEW_ROUTED, false>(a, blockIdx.y, false, lds);
    if (pick.expert < 0) return;
    constexpr int ROWS = Few<T>::ROWS, PARTS = sizeof(T) == 2 ? 2 : 1;
    const T* W = reinterpret_cast<const T*>(a.W2) + (long long)pick.expert * a.H * a.M + n0;
    const int all = (a.H + Few<T>::STEP - 1) / Few<T>::STEP, begin = blockIdx.z * a.steps, end = begin + a.steps < all ? begin + a.steps : all;
    const T* rows[PARTS];
#pragma unroll
    for (int c = 0; c < PARTS; ++c) rows[c] = reinterpret_cast<const T*>(a.a) + (long long)c * a.T * a.k * a.H;
    float* partial = a.partial + (long long)blockIdx.z * a.T * a.k * a.M;
    for (int r0 = 0; r0 < pick.n_rows; r0 += GROUPS * ROWS) {
        unsigned row[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int r = r0 + g * ROWS + Few<T>::row(lane);
            row[g] = (unsigned)plan.rows[r < pick.n_rows ? r : r0] * (unsigned)a.H * (unsigned)sizeof(T);
        }
        few_acc acc[GROUPS][Few<T>::ACCS];
        few_sums<T, GROUPS, PARTS, FEW_WAVES>(W, a.M, a.M - n0, rows, row, a.H, begin + wid, end, acc);
        few_finish<T, GROUPS, FEW_WAVES>(lds.sums, acc, pick.n_rows - r0, a.M - n0,
                                         [&](int r, int n, float v) { partial[(long long)plan.rows[r0 + r] * a.M + n0 + n] = v; });
    }
}

// y[t] = sum over the choices of w times the sum of their slices.  Four columns to a thread; the wavefronts share out the choices and add
// up in the choices' order.  Loads go out in eights, without a look at whether there is a choice (nothing was written for one that is not).
constexpr int JOIN_WAVES = 4;
template <typename T> __global__ __launch_bounds__(JOIN_WAVES * 64) void few_join_kernel(FewArgs a) {
    __shared__ float4 part[FEW_K][64];
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const int t = blockIdx.y, n = (blockIdx.x * 64 + lane) * 4;
    const long long step = (long long)a.T * a.k * a.M;
    for (int j = wid; j < a.k; j += JOIN_WAVES) {
        const float* p = a.partial + ((long long)t * a.k + j) * a.M + (n < a.M ? n : 0);
        const int chosen = a.route.idx[t * a.k + j];
        const float w = a.route.w[t * a.k + j];
        float4 v = make_float4(0, 0, 0, 0);
        for (int s0 = 0; s0 < a.slices; s0 += 8) {
            float4 o[8];
#pragma unroll
            for (int s = 0; s < 8; ++s) o[s] = *reinterpret_cast<const float4*>(p + (s0 + s < a.slices ? s0 + s : 0) * step);
#pragma unroll
            for (int s = 0; s < 8; ++s)
                if (s0 + s < a.slices) { v.x += o[s].x; v.y += o[s].y; v.z += o[s].z; v.w += o[s].w; }
        }
        part[j][lane] = chosen >= 0 ? make_float4(w * v.x, w * v.y, w * v.z, w * v.w) : make_float4(0, 0, 0, 0);
    }
    __syncthreads();
    if (wid > 0 || n >= a.M) return;
    float y[4] = {0, 0, 0, 0};
    for (int j = 0; j < a.k; ++j) {
        const float4 v = part[j][lane];
        y[0] += v.x; y[1] += v.y; y[2] += v.z; y[3] += v.w;
    }
    store_columns(reinterpret_cast<T*>(a.y) + t * a.ldy + n, y, 4);
}

struct FewDims {
    moe_router_config router;
    int slots, slices, steps;                // experts that may be chosen; of the second product
    int mode, exact_values, few_groups;
    int gate_slices, gate_rows;
    size_t a_bytes, partial_bytes, gate_bytes;
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
    const long long limit = 1 << 30;                       // of offsets in elements
    if ((long long)c->M * c->H >= limit || (long long)c->T * c->k * c->H >= limit || (c->ldx ? c->ldx : c->M) >= limit / FEW_TOKENS) return MOE_ERR_UNSUPPORTED;
    const bool bf16 = c->dtype == MOE_BF16;
    const long long n = (long long)c->T * c->k;
    d->slots = (int)(n < c->E ? n : c->E);
    if (d->slots < 1) d->slots = 1;
    const int cols = bf16 ? Few<bf16_t>::COLS : Few<float>::COLS, steps = up(c->H, Few<float>::STEP), blocks = up(c->M, cols) * d->slots;
    // (two workgroups fit a compute unit: slices of H until the 512 places are taken; 256 of them: 3 x 16 of 2048/8192 92 us instead of 85,
    // 7 x 33 of 520/1000 in float 35.8 and 35.3, but 1 x 8 of 2048/8192 37.9 and 39.2; 1024: 84.5, 33.8 and 41.6)
    int slices = blocks < 512 ? up(512, blocks) : 1;
    const int most = up(steps, FEW_WAVES);
    if (slices > most) slices = most;
    d->steps = up(steps, slices);
    d->slices = up(steps, d->steps);
    // Who routes (tokens x experts of M/H, us).  Little gate in all: every workgroup of the first product by itself, which saves two launches
    // (1 x 16 of 1024/4096 22.2, 24.0 with the gate's launch, 24.5 with both; 2 x 16 25.2, 26.2, 27.0; 2 x 64, which is too much, 31.8, 28.2,
    // 29.1).  Up to four tokens and 64 experts: it does so from the gate's sums (4 x 64 of 1024/1024 28.6, 29.3 with a launch for it).  More: a launch of
    // its own (16 x 16 of 1024/4096 56.4 and 57.8 without; 64 x 64 of 1024/1024 55.4 and 67.6).
    // Groups of rows that go through together: as many as an expert is expected to have, and half as many again (8 experts of 1024/4096,
    // choices 2: 64 tokens, two groups, 51.7, one 63.5; 128 tokens, four, 74.4, two 78.5, one 97.8; 48 x 64 of four, one, 150.7, two 156.2).
    const int mean = up(n, c->E);
    d->few_groups = up(mean + (mean > 1 ? up(mean, 2) : 0), Few<float>::ROWS);
    d->mode = c->T > 4 || c->E > 64 ? FEW_ROUTED : c->T <= 2 && (long long)c->T * c->M * c->E <= 65536 ? FEW_ALONE : FEW_SUMMED;
    d->exact_values = c->E <= 64 ? 1 : c->E <= 128 ? 2 : c->E <= 256 ? 4 : 8;
    // The gate's workgroups: enough for the chip, of 128 rows of Wg at least (64 or 256: the same within 3 %).
    const int tiles = up(c->E, 64) * up(c->T > 0 ? c->T : 1, c->T == 1 ? 1 : GATE_TOKENS);
    d->gate_slices = up(256, tiles);
    if (d->gate_slices > 16) d->gate_slices = 16;
    if (d->gate_slices > up(c->M, 128)) d->gate_slices = up(c->M, 128);
    d->gate_rows = up(c->M, d->gate_slices);
    d->gate_slices = up(c->M, d->gate_rows);
    d->gate_bytes = align16((size_t)d->gate_slices * c->T * c->E * 8);
    d->a_bytes = align16((size_t)n * c->H * 4);
    d->partial_bytes = align16((size_t)n * c->M * d->slices * 4);
    return MOE_OK;
}

template <typename T> moe_status few_launch(const FewArgs& a, const FewDims& d, hipStream_t s) {
    if (d.mode != FEW_ALONE) {
        const dim3 grid(up(a.E, 64), up(a.T, a.T == 1 ? 1 : GATE_TOKENS), a.gate_slices);
        if (a.T == 1) few_gate_kernel<T, 1><<<grid, GATE_WAVES * 64, 0, s>>>(a);
        else few_gate_kernel<T, GATE_TOKENS><<<grid, GATE_WAVES * 64, 0, s>>>(a);
        MOE_CHECK_LAUNCH();
    }
    if (d.mode == FEW_ROUTED) {
        if (d.exact_values == 1) few_route_kernel<1><<<a.T, 64, 0, s>>>(a);
        else if (d.exact_values == 2) few_route_kernel<2><<<a.T, 64, 0, s>>>(a);
        else if (d.exact_values == 4) few_route_kernel<4><<<a.T, 64, 0, s>>>(a);
        else few_route_kernel<8><<<a.T, 64, 0, s>>>(a);
        MOE_CHECK_LAUNCH();
    }
    // The first product in pieces of half the columns: up to eight tokens, and twice the workgroups are no more than the chip has room for at once
    // (tokens x experts of M/H, us so / otherwise: 1 x 16 of 1024/4096 20.3 / 21.9; 1 x 64 of 2048/1024, four choices, 26.3 / 30.1; 1 x 16 of 2048/8192
    // 38.1 / 39.0; too many: 4 x 33 of 520/1000 in float 29.4 / 27.2, 4 x 16 of 1024/4096 34.0 / 32.7).
    const bool narrow = a.T <= Few<T, true>::ROWS && up(a.H, Few<T>::COLS) * d.slots <= 128;
    const dim3 first(up(a.H, narrow ? Few<T, true>::COLS : Few<T>::COLS), d.slots), second(up(a.M, Few<T>::COLS), d.slots, a.slices);
#define FEW_FIRST(G, MODE, NARROW) few_first_kernel<T, G, MODE, NARROW><<<first, FEW_WAVES * 64, 0, s>>>(a)
#define FEW_SECOND(G) few_second_kernel<T, G><<<second, FEW_WAVES * 64, 0, s>>>(a)
    if (d.few_groups <= 1) {
        if (d.mode == FEW_ALONE) { if (narrow) FEW_FIRST(1, FEW_ALONE, true); else FEW_FIRST(1, FEW_ALONE, false); }
        else if (d.mode == FEW_SUMMED) { if (narrow) FEW_FIRST(1, FEW_SUMMED, true); else FEW_FIRST(1, FEW_SUMMED, false); }
        else { if (narrow) FEW_FIRST(1, FEW_ROUTED, true); else FEW_FIRST(1, FEW_ROUTED, false); }
        FEW_SECOND(1);
    } else if (d.few_groups <= 2) {
        FEW_FIRST(2, FEW_ROUTED, false);
        FEW_SECOND(2);
    } else {
        FEW_FIRST(4, FEW_ROUTED, false);
        FEW_SECOND(4);
    }
#undef FEW_FIRST
#undef FEW_SECOND
    MOE_CHECK_LAUNCH();
    few_join_kernel<T><<<dim3(up(a.M, 256), a.T), JOIN_WAVES * 64, 0, s>>>(a);
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
    *bytes = cfg->T == 0 ? 0 : d.a_bytes + d.partial_bytes + d.gate_bytes;
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
    moe::FewArgs a = {x, Wg, gate_bias, W1, W2, y, logits,
                      moe::router_args(&d.router, logits, bias, topk_idx, topk_w, nullptr, d.exact_values, d.exact_values),
                      (double*)(p + d.a_bytes + d.partial_bytes), d.gate_slices, d.gate_rows, p, (float*)(p + d.a_bytes),
                      cfg->ldx ? (long long)cfg->ldx : cfg->M, cfg->ldy ? (long long)cfg->ldy : cfg->M,
                      cfg->T, cfg->M, cfg->H, cfg->E, cfg->k, d.slices, d.steps};
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_FEW, s);
        MOE_TRY(cfg->dtype == MOE_BF16 ? moe::few_launch<moe::bf16_t>(a, d, s) : moe::few_launch<float>(a, d, s));
    }
    moe::count_launch(moe::LC_GEMM, 2);
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}
