// Products of routed rows with their experts' 4-bit weights, and the packing of such weights.
//
//   y[t,j,n] = f(sum over c of x_row[c] W[e][n,c]) w[t,j],  e = topk_idx[t,j];  or y[t,n] = their sum over j
//   W[e][n,c] = e2m1 value of 4 bits * 2^(Ws - 127) of 32 columns
//
// Few rows meet each expert's matrix, so what has to move is the matrix: K N (1/2 + 1/32) bytes for every expert that is
// chosen, read once.  A wavefront multiplies 16 weight rows of 128 columns at a time: lane (r, q) holds 32 consecutive
// columns of weight row r, which is one 16-byte load, one scale, and exactly what the matrix instructions take, so packed
// weights go from memory into registers with no detour.  The weights are the left operand and the routed rows, padded to
// 16, the right one: an output's lanes then hold four neighbouring columns of one row.
//   bfloat16 rows  the weights become bfloat16 (exact: the scale is a power of two) eight to an instruction of 16 x 16 x 32
//   float rows     the same with each float cut into three bfloat16 parts, whose sum it is: every product is exact
//   e4m3 rows      become bfloat16 as well (exact), and 128 columns' sum is multiplied by the rows' scale.  The 16 x 16 x 128
//                  instruction that takes 4-bit and 8-bit operands as they are would save all the conversions, but among each
//                  eight neighbouring products it drops what lies some 2^14 below the largest (measured: sums up to 2^-14 of
//                  their largest term off, where the bfloat16 instruction is exact), and sums are to be those of float.
// The workgroup's wavefronts share out K and add up their sums in their order.
#include "common.h"
#include "wide.h"
#include <climits>

namespace moe {

namespace {

typedef __bf16 bf16x8_hw __attribute__((ext_vector_type(8)));
typedef float f32x4_hw __attribute__((ext_vector_type(4)));

constexpr int W4_WAVES = 4;

struct W4Args {
    const void* x; const float* x_scales; const int* idx; const float* w; const uint8_t* Wq; const uint8_t* Ws;
    void* y;
    long long ldx, ldy;
    int n_rows;                      // T * k assignments
    int k, E, K, N, n_scales, per_choice, gelu;
    int by_choice;                   // blockIdx.y is an assignment (whose expert it serves if it is its first), else an expert
};

// 32 columns of a routed row: the right operand's share of a lane
template <int XT> struct Rows32;
template <> struct Rows32<MOE_BF16> {
    uint4 u[4];
    __device__ __forceinline__ void load(const void* row, int col) {
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const bf16_t*>(row) + col);
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = p[i];
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = make_uint4(0, 0, 0, 0);
    }
    static constexpr int PARTS = 1;
    __device__ __forceinline__ void parts(int i, bf16x8_hw* o) const { o[0] = __builtin_bit_cast(bf16x8_hw, u[i]); }
};
template <> struct Rows32<MOE_F32> {
    float4 u[8];
    __device__ __forceinline__ void load(const void* row, int col) {
        const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(row) + col);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = p[i];
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = make_float4(0, 0, 0, 0);
    }
    static constexpr int PARTS = 3;
    // Cut, not rounded: 8 + 8 + 8 bits of mantissa, exact, and no part is larger than the whole.  Infinities and NaN have
    // one part.
    __device__ __forceinline__ void parts(int i, bf16x8_hw* o) const {
        unsigned hi[4], mid[4], lo[4];
        const float v[8] = {u[2 * i].x, u[2 * i].y, u[2 * i].z, u[2 * i].w, u[2 * i + 1].x, u[2 * i + 1].y, u[2 * i + 1].z, u[2 * i + 1].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            unsigned h[2], m[2], l[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const float f = v[2 * j + b];
                const bool special = (__float_as_uint(f) & 0x7f800000u) == 0x7f800000u;
                h[b] = __float_as_uint(f) & 0xffff0000u;
                if (f != f) h[b] = 0x7fc00000u;
                const float rest = special ? 0.0f : f - __uint_as_float(h[b]);
                m[b] = __float_as_uint(rest) & 0xffff0000u;
                l[b] = __float_as_uint(rest - __uint_as_float(m[b])) & 0xffff0000u;
            }
            hi[j] = h[0] >> 16 | h[1];
            mid[j] = m[0] >> 16 | m[1];
            lo[j] = l[0] >> 16 | l[1];
        }
        o[0] = __builtin_bit_cast(bf16x8_hw, make_uint4(hi[0], hi[1], hi[2], hi[3]));
        o[1] = __builtin_bit_cast(bf16x8_hw, make_uint4(mid[0], mid[1], mid[2], mid[3]));
        o[2] = __builtin_bit_cast(bf16x8_hw, make_uint4(lo[0], lo[1], lo[2], lo[3]));
    }
};
template <> struct Rows32<MOE_E4M3> {
    uint4 u[2];
    __device__ __forceinline__ void load(const void* row, int col) {
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row) + col);
        u[0] = p[0];
        u[1] = p[1];
    }
    __device__ __forceinline__ void zero() { u[0] = u[1] = make_uint4(0, 0, 0, 0); }
    static constexpr int PARTS = 1;
    __device__ __forceinline__ void parts(int i, bf16x8_hw* o) const {
        const uint4& v = u[i / 2];
        const unsigned a = i % 2 ? v.z : v.x, b = i % 2 ? v.w : v.y;
        uint4 d;
        d.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false));
        d.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true));
        d.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false));
        d.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true));
        o[0] = __builtin_bit_cast(bf16x8_hw, d);
    }
};

// Rows of assignments with expert e (e < 0: with none of the experts), number `from` to from + cap - 1 of them, into `list`;
// returns how many there are in all.  Every thread of the workgroup calls it.
__device__ int collect_rows(const int* idx, int n, int e, int E, int from, int cap, int* list, int* s_count) {
    const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int total = 0;
    for (int base = 0; base < n; base += W4_WAVES * 64) {
        const int i = base + threadIdx.x;
        bool mine = false;
        if (i < n) {
            const int v = idx[i];
            mine = e < 0 ? (unsigned)v >= (unsigned)E : v == e;
        }
        const unsigned long long b = __ballot(mine);
        if (lane == 0) s_count[wid] = __popcll(b);
        __syncthreads();
        int rank = total + __popcll(b & ((1ull << lane) - 1));
#pragma unroll
        for (int w = 0; w < W4_WAVES; ++w) {
            if (w < wid) rank += s_count[w];
            total += s_count[w];
        }
        if (mine && rank >= from && rank < from + cap) list[rank - from] = i;
        __syncthreads();
    }
    return total;
}

__device__ __forceinline__ void decode_weights(const uint4& q, float scale, int i, bf16x8_hw* o) {
    const unsigned w = i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w;
    uint4 d;
    d.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    d.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    d.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    d.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    *o = __builtin_bit_cast(bf16x8_hw, d);
}

// NT tiles of 16 weight rows and RT tiles of 16 routed rows to a workgroup
template <int XT, typename OUT, int NT, int RT>
__global__ __launch_bounds__(W4_WAVES * 64) void w4_kernel(W4Args a) {
    constexpr int CAP = 16 * RT;
    __shared__ int s_list[CAP], s_count[W4_WAVES];
    __shared__ float4 s_sum[W4_WAVES][NT * RT][64];
    const int tid = threadIdx.x, wid = tid >> 6, lane = tid & 63, r = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16 * NT;
    int e = 0;
    if (a.idx) {
        e = a.by_choice ? a.idx[blockIdx.y] : (int)blockIdx.y;
        if ((unsigned)e >= (unsigned)a.E) e = -1;
    }
    const uint8_t* Wq = a.Wq + (long long)(e < 0 ? 0 : e) * a.N * (a.K / 2);
    const uint8_t* Ws = a.Ws + (long long)(e < 0 ? 0 : e) * a.N * (a.K / 32);
    const int tiles = (a.K + 127) / 128;
    for (int from = 0;; from += CAP) {
        int total;
        if (a.idx) {
            total = collect_rows(a.idx, a.n_rows, e, a.E, from, CAP, s_list, s_count);
            if (total <= from) return;
            if (from == 0 && a.by_choice && s_list[0] != (int)blockIdx.y) return;     // an earlier assignment has this expert too
        } else {
            total = a.n_rows;
            if (total <= from) return;
            __syncthreads();
            if (tid < CAP) s_list[tid] = from + tid;
            __syncthreads();
        }
        const int here = total - from < CAP ? total - from : CAP;
        f32x4_hw acc[NT][RT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[nt][rt] = f32x4_hw{0, 0, 0, 0};
        if (e >= 0) {
            const void* row[RT];
            const float* row_scale[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int at = rt * 16 + r;
                row[rt] = nullptr;
                row_scale[rt] = nullptr;
                if (at < here) {
                    const long long xr = a.per_choice ? s_list[at] : s_list[at] / a.k;
                    row[rt] = reinterpret_cast<const char*>(a.x) + xr * a.ldx * (XT == MOE_F32 ? 4 : XT == MOE_BF16 ? 2 : 1);
                    if (XT == MOE_E4M3) row_scale[rt] = a.x_scales + xr * a.n_scales;
                }
            }
            for (int tile = wid; tile < tiles; tile += W4_WAVES) {
                const int col = tile * 128 + q * 32;
                const bool inside = col < a.K;
                uint4 wq[NT];
                int ws[NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int n = n0 + nt * 16 + r;
                    wq[nt] = make_uint4(0, 0, 0, 0);
                    ws[nt] = 127;
                    if (inside && n < a.N) {
                        wq[nt] = *reinterpret_cast<const uint4*>(Wq + (long long)n * (a.K / 2) + col / 2);
                        ws[nt] = Ws[(long long)n * (a.K / 32) + col / 32];
                    }
                }
                Rows32<XT> x[RT];
                f32x4_hw part[NT][RT];                          // e4m3: the tile's sums, before their 128 columns' scale
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    x[rt].zero();
                    if (row[rt] && inside) x[rt].load(row[rt], col);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) part[nt][rt] = XT == MOE_E4M3 ? f32x4_hw{0, 0, 0, 0} : acc[nt][rt];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    bf16x8_hw w[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) decode_weights(wq[nt], __uint_as_float((unsigned)ws[nt] << 23), i, &w[nt]);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        bf16x8_hw p[Rows32<XT>::PARTS];
                        x[rt].parts(i, p);
#pragma unroll
                        for (int c = Rows32<XT>::PARTS - 1; c >= 0; --c)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
                                part[nt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[nt], p[c], part[nt][rt], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float xs = XT == MOE_E4M3 && row[rt] ? row_scale[rt][a.n_scales > 1 ? tile : 0] : 0.0f;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            acc[nt][rt][j] = XT == MOE_E4M3 ? fmaf(xs, part[nt][rt][j], acc[nt][rt][j]) : part[nt][rt][j];
                }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                s_sum[wid][nt * RT + rt][lane] = make_float4(acc[nt][rt][0], acc[nt][rt][1], acc[nt][rt][2], acc[nt][rt][3]);
        __syncthreads();
        for (int i = tid; i < NT * RT * 64; i += W4_WAVES * 64) {
            const int tile = i >> 6, l = i & 63, at = (tile % RT) * 16 + (l & 15);
            if (at >= here) continue;
            float v[4] = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < W4_WAVES; ++w) {
                const float4 p = s_sum[w][tile][l];
                v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
            }
            const int n = n0 + (tile / RT) * 16 + (l >> 4) * 4;
            const float weight = a.w ? a.w[s_list[at]] : 1.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (a.gelu) v[j] = v[j] * (0.5f + 0.5f * erff(v[j] * 0.70710678118654752440f));
                v[j] = e < 0 ? 0.0f : v[j] * weight;
            }
            store_columns(reinterpret_cast<OUT*>(a.y) + s_list[at] * a.ldy + n, v, a.N - n);
        }
        __syncthreads();
    }
}

// y[t] = sum over j, ascending, of the rows of assignments with an expert
template <typename OUT>
__global__ __launch_bounds__(256) void w4_join_kernel(const float* __restrict__ rows, const int* __restrict__ idx, OUT* __restrict__ y,
                                                      long long ldy, int k, int E, int N) {
    const int n = (blockIdx.x * 256 + threadIdx.x) * 4;
    const long long t = blockIdx.y;
    if (n >= N) return;
    float v[4] = {0, 0, 0, 0};
    for (int j = 0; j < k; ++j) {
        if (idx && (unsigned)idx[t * k + j] >= (unsigned)E) continue;
        float p[4];
        load_columns(rows + (t * k + j) * N + n, p, N - n);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += p[i];
    }
    store_columns(y + t * ldy + n, v, N - n);
}

// One thread packs 32 columns of one weight row; neighbouring threads have neighbouring weight rows, which lie next to one
// another in W.
template <typename T>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const T* __restrict__ W, uint8_t* __restrict__ Wq, uint8_t* __restrict__ Ws,
                                                          int K, int N) {
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    const long long e = blockIdx.z, b = blockIdx.y;
    const T* p = W + (e * K + b * 32) * N + n;
    float v[32];
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        v[i] = Elem<T>::ld(p + (long long)i * N);
        const unsigned m = __float_as_uint(v[i]) & 0x7fffffffu;
        most = m > most ? m : most;
    }
    unsigned packed[4] = {0, 0, 0, 0}, scale = 255;
    if (most < 0x7f800000u) {
        // the least power of two 2^(scale - 127) with most <= 6 * 2^(scale - 127): 6 = 1.5 * 2^2
        const int up = (int)(most >> 23) - 2 + ((most & 0x7fffffu) > 0x400000u ? 1 : 0);
        scale = up < 1 ? 1u : (unsigned)up;
        const float inv = __uint_as_float((254u - scale) << 23);          // exact; scale is at most 253
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float m = fabsf(v[i]) * inv;                             // exact, or below half the least step
            // nearest of 0 .5 1 1.5 2 3 4 6, ties to the even code
            const unsigned c = (m > 0.25f) + (m >= 0.75f) + (m > 1.25f) + (m >= 1.75f) + (m > 2.5f) + (m >= 3.5f) + (m > 5.0f);
            packed[i / 8] |= (c | (__float_as_uint(v[i]) >> 31 << 3)) << (4 * (i % 8));
        }
    }
    *reinterpret_cast<uint4*>(Wq + ((e * N + n) * K + b * 32) / 2) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
    Ws[(e * N + n) * (K / 32) + b] = (uint8_t)scale;
}

struct W4Plan { long long ldx, ldy; int n_scales, NT, RT; size_t scratch; };

moe_status w4_plan(const moe_w4_config* c, W4Plan* p) {
    if (!c) return MOE_ERR_NULL;
    if (c->T < 0 || c->k <= 0 || c->E <= 0 || c->K <= 0 || c->N <= 0 || c->k > c->E) return MOE_ERR_SHAPE;
    if (c->dtype != MOE_F32 && c->dtype != MOE_BF16 && c->dtype != MOE_E4M3) return MOE_ERR_UNSUPPORTED;
    if (c->out != MOE_F32 && c->out != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (c->group != 0 && (c->group != 128 || c->dtype != MOE_E4M3)) return MOE_ERR_UNSUPPORTED;
    if ((c->per_choice | c->combine | c->gelu) & ~1) return MOE_ERR_UNSUPPORTED;
    if (c->K % 32 != 0 || c->k > 64 || c->E > 4096) return MOE_ERR_UNSUPPORTED;
    if ((c->ldx != 0 && c->ldx < c->K) || (c->ldy != 0 && c->ldy < c->N)) return MOE_ERR_SHAPE;
    p->ldx = c->ldx ? (long long)c->ldx : (long long)c->K;
    p->ldy = c->ldy ? (long long)c->ldy : (long long)c->N;
    if (p->ldx % (c->dtype == MOE_F32 ? 4 : c->dtype == MOE_BF16 ? 8 : 16) != 0) return MOE_ERR_UNSUPPORTED;
    if ((long long)c->T * c->k > (1 << 24) || (c->combine && c->T > 65535)) return MOE_ERR_UNSUPPORTED;
    p->n_scales = c->group ? (c->K + 127) / 128 : 1;
    p->scratch = c->combine && c->k > 1 ? (size_t)c->T * c->k * c->N * sizeof(float) : 0;
    p->NT = 1;
    p->RT = 1;
    return MOE_OK;
}

template <int XT, typename OUT> void w4_launch(const W4Args& a, dim3 grid, hipStream_t s) {
    w4_kernel<XT, OUT, 1, 1><<<grid, W4_WAVES * 64, 0, s>>>(a);
}
template <typename OUT> void w4_launch_x(int dtype, const W4Args& a, dim3 grid, hipStream_t s) {
    if (dtype == MOE_F32) w4_launch<MOE_F32, OUT>(a, grid, s);
    else if (dtype == MOE_BF16) w4_launch<MOE_BF16, OUT>(a, grid, s);
    else w4_launch<MOE_E4M3, OUT>(a, grid, s);
}

}  // namespace

}  // namespace moe

extern "C" moe_status moe_w4_scratch_bytes(const moe_w4_config* cfg, size_t* bytes) {
    moe::W4Plan p;
    MOE_TRY(moe::w4_plan(cfg, &p));
    if (!bytes) return MOE_ERR_NULL;
    *bytes = p.scratch;
    return MOE_OK;
}

extern "C" moe_status moe_w4_product(const moe_w4_config* cfg, const void* x, const float* x_scales, const int32_t* topk_idx,
                                     const float* topk_w, const uint8_t* Wq, const uint8_t* Ws, void* y, void* scratch, void* stream) {
    moe::W4Plan p;
    MOE_TRY(moe::w4_plan(cfg, &p));
    if (cfg->T == 0) return MOE_OK;
    if (!x || !Wq || !Ws || !y || (cfg->dtype == MOE_E4M3 && !x_scales) || (p.scratch && !scratch)) return MOE_ERR_NULL;
    if (((uintptr_t)x | (uintptr_t)Wq | (uintptr_t)scratch) & 15) return MOE_ERR_UNSUPPORTED;
    hipStream_t s = (hipStream_t)stream;
    const int rows = cfg->T * cfg->k;
    const bool join = p.scratch != 0;
    moe::W4Args a = {x, x_scales, topk_idx, topk_w, Wq, Ws, join ? scratch : y, p.ldx, join ? cfg->N : p.ldy, rows,
                     cfg->k, cfg->E, cfg->K, cfg->N, p.n_scales, cfg->per_choice, cfg->gelu, rows <= cfg->E};
    // without an assignment each: the expert's number, and one more for the assignments without an expert, whose rows are zeroed
    const int slots = !topk_idx ? 1 : a.by_choice ? rows : join ? cfg->E : cfg->E + 1;
    const dim3 grid((cfg->N + 16 * p.NT - 1) / (16 * p.NT), slots);
    {
        moe::ProfScope prof(moe::PK_W4, s);
        if (join || cfg->out == MOE_F32) moe::w4_launch_x<float>(cfg->dtype, a, grid, s);
        else moe::w4_launch_x<moe::bf16_t>(cfg->dtype, a, grid, s);
        MOE_CHECK_LAUNCH();
        if (join) {
            const dim3 jgrid((cfg->N + 1023) / 1024, cfg->T);
            if (cfg->out == MOE_F32)
                moe::w4_join_kernel<float><<<jgrid, 256, 0, s>>>((const float*)scratch, topk_idx, (float*)y, p.ldy, cfg->k, cfg->E, cfg->N);
            else
                moe::w4_join_kernel<moe::bf16_t><<<jgrid, 256, 0, s>>>((const float*)scratch, topk_idx, (moe::bf16_t*)y, p.ldy, cfg->k, cfg->E, cfg->N);
            MOE_CHECK_LAUNCH();
        }
    }
    moe::count_launch(moe::LC_GEMM);
    return MOE_OK;
}

extern "C" moe_status moe_w4_quantize(int32_t E, int32_t K, int32_t N, int32_t dtype, const void* W, uint8_t* Wq, uint8_t* Ws,
                                      void* stream) {
    if (E <= 0 || K <= 0 || N <= 0) return MOE_ERR_SHAPE;
    if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (K % 32 != 0 || E > 4096 || K / 32 > 65535) return MOE_ERR_UNSUPPORTED;
    if (!W || !Wq || !Ws) return MOE_ERR_NULL;
    if ((uintptr_t)Wq & 15) return MOE_ERR_UNSUPPORTED;
    const dim3 grid((N + 255) / 256, K / 32, E);
    hipStream_t s = (hipStream_t)stream;
    if (dtype == MOE_F32) moe::w4_quantize_kernel<float><<<grid, 256, 0, s>>>((const float*)W, Wq, Ws, K, N);
    else moe::w4_quantize_kernel<moe::bf16_t><<<grid, 256, 0, s>>>((const moe::bf16_t*)W, Wq, Ws, K, N);
    MOE_CHECK_LAUNCH();
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}
