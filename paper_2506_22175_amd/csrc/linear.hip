// A dense product with its epilogue, for what stands beside the routed experts (a shared expert, projections), and its gradients.
//
//   z = x W + bias;  y = act(z) + residual        W [K,N] as the layer's W1 and W2
//   dz = dy act'(z);  dbias = sum over rows of dz;  dx = dz W^T;  dW = x^T dz
//
// Many rows are the layer's grouped GEMM's (gemm_bf16.hip, gemm_f32.hip) with blocks of rows for experts: one unless 32-bit offsets want more.
// Where the output has too few tiles for the chip, the sum is cut into slices whose partial sums a second launch adds up: rows in the
// weight gradient, columns of x or dz in the others (64 rows, 8192 x 2048: 15 us, 41 without; float 31 and 177).  8192 rows of 2048 x 8192
// take 255 us with GeLU and z kept (1.08 PFLOP/s; a library's product of 8192^3 1.10), back 380 us (1.45).  Up to 32 rows are bound by reading
// W once and go through few_rows.h: one of 8192 x 2048 10 to 11 us, of which the second launch and what lies between are half.
#include "common.h"
#include "activation.h"
#include "few_rows.h"
#include "wide.h"

namespace moe {

namespace {

struct LinearDims {
    int T, K, N, act, overwrite;
    bool bf16;
    long long ldx, ldy, ldr, ldz;
    int block, blocks;                       // rows of a block of the GEMMs over rows, how many there are
    int wblock, wblocks;                     // the same of the weight gradient
    int slices;                              // few rows: workgroups that share a column block's K
};

// Up to so many rows (2048 x 8192: 16 rows 11.7 us, 15.5 through the GEMM; 32 rows 15.6 and 15.6; 48 rows 19.8 and 15.8).
constexpr int FEW_LINEAR_ROWS = 32;
constexpr int FEW_WAVES = 8;
constexpr int ACT_WAVES = 4, ACT_COLS = 512; // of act_bwd_kernel: wavefronts, columns of each

int up(long long a, long long b) { return (int)((a + b - 1) / b); }

// Workgroups that share a column block's K: 256 in all, or as many fewer as it takes for a whole number to a block, down to half of them (one row, 8192 x 2048: 11.7 us, with 128 12.7, with 512 12.4; 2048 x 8192 11.0, 12.4, 10.9),
// or one, which finishes by itself, where K is three steps to a wavefront (one row, 520 x 1000: 4.7 us, 7.3 with a second launch; 1024 x 4096, which is
// too much, 8.5 and 7.6).  Rounded up they would be more than 256, some CUs with two and most with one, and a second launch for wide matrices
// (K = 4096, N = 16640: 26.5 us in one slice, 33.7 in two; 11008 in two 19.5, in three 23.9; 28 rows, 5152 x 2192 14.1 and 16.2).
int few_slices(int K, int N, bool bf16) {
    const int columns = up(N, bf16 ? Few<bf16_t>::COLS : Few<float>::COLS), steps = up(K, Few<float>::STEP);
    if (columns >= 256 || steps <= 3 * FEW_WAVES) return 1;
    const int s = 256 / columns, most = up(steps, FEW_WAVES);
    return s < most ? s : most;
}

moe_status linear_dims(const moe_linear_config* c, LinearDims* d) {
    if (!c) return MOE_ERR_NULL;
    if (c->T < 0 || c->K <= 0 || c->N <= 0) return MOE_ERR_SHAPE;
    if (c->dtype != MOE_F32 && c->dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (c->act != MOE_ACT_NONE && c->act != MOE_ACT_GELU && c->act != MOE_ACT_SILU) return MOE_ERR_UNSUPPORTED;
    if (c->grad_overwrite != 0 && c->grad_overwrite != 1) return MOE_ERR_UNSUPPORTED;
    if ((c->ldx && c->ldx < c->K) || (c->ldy && c->ldy < c->N) || (c->ldr && c->ldr < c->N) || (c->ldz && c->ldz < c->N)) return MOE_ERR_SHAPE;
    if (c->K % 8 || c->N % 8 || c->ldx % 8 || c->ldy % 8 || c->ldr % 8 || c->ldz % 8) return MOE_ERR_UNSUPPORTED;
    d->T = c->T; d->K = c->K; d->N = c->N; d->act = c->act; d->overwrite = c->grad_overwrite;
    d->bf16 = c->dtype == MOE_BF16;
    d->ldx = c->ldx ? c->ldx : c->K;
    d->ldy = c->ldy ? c->ldy : c->N;
    d->ldr = c->ldr ? c->ldr : c->N;
    d->ldz = c->ldz ? c->ldz : c->N;
    long long most = d->ldx;
    for (long long l : {d->ldy, d->ldr, d->ldz, (long long)d->N, (long long)d->K})
        if (l > most) most = l;
    // What the GEMMs' 32-bit offsets allow: 2^30 elements from a matrix's first to its last, some rows more; longer calls go in up to 64
    // blocks of rows, of which a launch of the float GEMM takes no more than 65535 tiles each.
    const long long widest = d->K > d->N ? d->K : d->N;
    if (most > (1 << 18) || (widest + 1024) * most > (1ll << 30) || c->T > (1 << 27) || c->T * most > (1ll << 35)) return MOE_ERR_UNSUPPORTED;
    long long rows = ((1ll << 30) / most - 1024) / 256 * 256;
    if (!d->bf16 && rows > 65535 / 4 * 256) rows = 65535 / 4 * 256;
    const int T = d->T > 0 ? d->T : 1;
    d->block = T <= rows ? T : (int)rows;
    d->blocks = up(T, d->block);
    // The weight gradient's sum is cut up until its 128 x 128 tiles fill the chip twice, but not below 1024 rows (30011 rows, 520 x 1000: 125 us;
    // once or four times 139 and 140; 512 or 2048 rows 123 and 124, but 4096 rows, 1024 x 1024, 36, 44 and 40), or 256 where the partial sums
    // are small (2480 rows, 72 x 1144, with the input gradient: 20.8 us and 23.8; 1688 rows, 152 x 664: 19.8 and 22.1; 8192 rows, 512 x 512,
    // which is too much: 29.4 and 26.4).  Float has smaller tiles and its own reckoning (the first two: 32.5 us and 38, 26 and 36), which is too
    // careful with many rows (8192 rows, 512 x 512: 92.6 us and 89.4).
    const long long tiles = (long long)up(d->K, 128) * up(d->N, 128), fill = tiles < 512 ? 512 / tiles : 1, size = (long long)d->K * d->N;
    long long parts = d->blocks, want = fill < up(T, 1024) ? fill : up(T, 1024);
    const long long more = fill < up(T, 256) ? fill : up(T, 256);
    if (more * size <= 1 << 20) want = more;
    if (!d->bf16) {
        GemmArgs g = {};
        g.Cp = d->K; g.N = d->N; g.K = T;
        const int slices = gemm_f32_slices(g, 128);
        if (want < slices) want = slices;
    }
    if (want > 64) want = 64;
    if (want > parts) parts = want;
    d->wblock = up(up(T, parts), 64) * 64;
    d->wblocks = up(T, d->wblock);
    d->slices = few_slices(d->K, d->N, d->bf16);
    return MOE_OK;
}

// What the choice of a tile goes by, of the GEMMs over the rows and of the weight gradient's.
GemmArgs rows_gemm(const LinearDims& d, int N, int K, int act) {
    GemmArgs g = {};
    g.E = d.blocks; g.Cp = d.block; g.mean_rows = up(d.T, d.blocks);
    g.N = N; g.K = K; g.act = act; g.rows = d.T;
    return g;
}
GemmArgs fwd_gemm(const LinearDims& d) { return rows_gemm(d, d.N, d.K, d.act); }
GemmArgs dx_gemm(const LinearDims& d) { return rows_gemm(d, d.K, d.N, MOE_ACT_NONE); }
GemmArgs dw_gemm(const LinearDims& d) {
    GemmArgs g = {};
    g.E = d.wblocks; g.Cp = d.wblock; g.mean_rows = up(d.T, d.wblocks); g.rows = d.T;
    g.Mo = d.K; g.N = d.N;
    return g;
}
// Slices of the sum in which a GEMM over the rows goes (few tiles, long sums), and one of them.
int gemm_slices(const LinearDims& d, GemmLayout lay, const GemmArgs& g) {
    return d.blocks > 1 ? 1 : d.bf16 ? gemm_bf16_slices(lay, g, 256) : gemm_f32_slices(g, 128);
}
int fwd_slices(const LinearDims& d) { return gemm_slices(d, GEMM_NN, fwd_gemm(d)); }
int dx_slices(const LinearDims& d) { return gemm_slices(d, GEMM_NT, dx_gemm(d)); }
GemmArgs slice_of(GemmArgs g, int slices) {
    g.k_total = g.K;
    g.K = up(up(g.K, slices), 64) * 64;
    g.E = up(g.k_total, g.K);
    return g;
}

size_t align16(size_t b) { return (b + 15) & ~(size_t)15; }
// A dz of more bytes than this, which would not be found in the memory-side cache by the products behind it anyway, is written past the caches
// (268 MB: 153 us so, 164 with ordinary stores).
constexpr long long ACT_PAST = 128ll << 20;
// Wavefronts side by side, and blocks of rows: enough for the chip, of two rows to a wavefront at least.  (1024 workgroups: 16384 x 8192
// 156 us, 4096 x 4096 25; 512 of them 160 and 26, 2048 157 and 26.)
int act_beside(const LinearDims& d) { return d.N > 2 * ACT_COLS ? 4 : d.N > ACT_COLS ? 2 : 1; }
int act_blocks(const LinearDims& d) {
    const int beside = act_beside(d), columns = up(d.N, beside * ACT_COLS);
    const int blocks = up(1024, columns), most = up(d.T > 0 ? d.T : 1, 2 * (ACT_WAVES / beside));
    return blocks < most ? blocks : most;
}

// ---- few rows -------------------------------------------------------------------------------------------
struct FewLinearArgs {
    const void* x; const void* W; const float* bias; const void* R; void* Z; void* y;
    float* partial;                          // [slices][T][N], or NULL: the only slice finishes
    long long ldx, ldy, ldr, ldz;
    int T, K, N, act, steps;                 // steps of a slice
};

template <typename T> __device__ __forceinline__ void linear_finish(const FewLinearArgs& a, int t, int n, float z) {
    if (a.bias) z += a.bias[n];
    if (a.Z) Elem<T>::st(reinterpret_cast<T*>(a.Z) + t * a.ldz + n, z);
    float y = activate<T>(z, a.act);
    if (a.R) y += Elem<T>::ld(reinterpret_cast<const T*>(a.R) + t * a.ldr + n);
    Elem<T>::st(reinterpret_cast<T*>(a.y) + t * a.ldy + n, y);
}

// Bound by W's way from memory: one row, 8192 x 2048 (33.6 MB, 4.8 us at the rate of a read) 5.2 us of this launch back to back, two steps to
// a wavefront.
template <typename T, int GROUPS>
__global__ __launch_bounds__(FEW_WAVES * 64, 4) void few_linear_kernel(FewLinearArgs a) {
    __shared__ FewSums<T, FEW_WAVES> sums;
    const int n0 = blockIdx.x * Few<T>::COLS, lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const int all = (a.K + Few<T>::STEP - 1) / Few<T>::STEP, begin = blockIdx.y * a.steps, end = begin + a.steps < all ? begin + a.steps : all;
    const T* const rows[1] = {reinterpret_cast<const T*>(a.x)};
    unsigned row[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int t = g * Few<T>::ROWS + Few<T>::row(lane);
        row[g] = (unsigned)(t < a.T ? t : 0) * (unsigned)a.ldx * (unsigned)sizeof(T);
    }
    few_acc acc[GROUPS][Few<T>::ACCS];
    few_sums<T, GROUPS, 1, FEW_WAVES>(reinterpret_cast<const T*>(a.W) + n0, a.N, a.N - n0, rows, row, a.K, begin + wid, end, acc);
    float* partial = a.partial ? a.partial + (long long)blockIdx.y * a.T * a.N : nullptr;
    few_finish<T, GROUPS, FEW_WAVES>(sums, acc, a.T, a.N - n0, [&](int t, int n, float v) {
        if (partial) partial[(long long)t * a.N + n0 + n] = v;
        else linear_finish<T>(a, t, n0 + n, v);
    });
}
// The slices' partial sums and the epilogue, four columns to a thread; sixteen slices are requested at a time, so that the launch (3 us) is the
// way to memory once.
template <typename T> __global__ __launch_bounds__(64) void linear_finish_kernel(FewLinearArgs a, int slices) {
    const int t = blockIdx.x, n = (blockIdx.y * 64 + threadIdx.x) * 4;
    if (n >= a.N) return;
    const long long size = (long long)a.T * a.N;
    const float* p = a.partial + (long long)t * a.N + n;
    float z[4] = {0, 0, 0, 0}, y[4];
    for (int s0 = 0; s0 < slices; s0 += 16) {
        float4 o[16];
#pragma unroll
        for (int s = 0; s < 16; ++s)
            if (s0 + s < slices) o[s] = *reinterpret_cast<const float4*>(p + (s0 + s) * size);
#pragma unroll
        for (int s = 0; s < 16; ++s)
            if (s0 + s < slices) { z[0] += o[s].x; z[1] += o[s].y; z[2] += o[s].z; z[3] += o[s].w; }
    }
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] += a.bias[n + i];
    }
    if (a.Z) store_columns(reinterpret_cast<T*>(a.Z) + t * a.ldz + n, z, 4);
    activate_all<T, 4>(z, y, a.act);
    if (a.R) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += Elem<T>::ld(reinterpret_cast<const T*>(a.R) + t * a.ldr + n + i);
    }
    store_columns(reinterpret_cast<T*>(a.y) + t * a.ldy + n, y, 4);
}
template <typename T> moe_status linear_finish_launch(const FewLinearArgs& a, int slices, hipStream_t s) {
    linear_finish_kernel<T><<<dim3(a.T, up(a.N, 256)), 64, 0, s>>>(a, slices);
    MOE_CHECK_LAUNCH();
    return MOE_OK;
}

// Slices that have steps to do.
int few_linear_slices(const LinearDims& d) {
    const int steps = up(d.K, Few<float>::STEP);
    return up(steps, up(steps, d.slices));
}
template <typename T> moe_status few_linear(const LinearDims& d, FewLinearArgs a, hipStream_t s) {
    a.steps = up(up(d.K, Few<T>::STEP), d.slices);
    const int slices = few_linear_slices(d);
    if (slices == 1) a.partial = nullptr;
    const dim3 grid(up(d.N, Few<T>::COLS), slices);
    const int groups = up(d.T, Few<T>::ROWS);
    if (groups <= 1) few_linear_kernel<T, 1><<<grid, FEW_WAVES * 64, 0, s>>>(a);
    else few_linear_kernel<T, 2><<<grid, FEW_WAVES * 64, 0, s>>>(a);
    MOE_CHECK_LAUNCH();
    return slices > 1 ? linear_finish_launch<T>(a, slices, s) : MOE_OK;
}

// ---- gradients --------------------------------------------------------------------------------------------
struct ActBwdArgs {
    const void* dy; const void* z; void* dz; float* part;       // part: [blocks][N], or NULL
    float* dbias; int store;                                    // of few rows
    long long ldy, ldz;
    int T, N, act, rows, beside;                                // rows of a workgroup; wavefronts side by side
    int past;                                                   // dz goes past the caches
};

__device__ __forceinline__ void load_eight_once(Raw8<bf16_t>& r, const bf16_t* p) { r.u = load_once<uint4>(p); }
__device__ __forceinline__ void load_eight_once(Raw8<float>& r, const float* p) { r.a = load_once<float4>(p); r.b = load_once<float4>(p + 4); }

// Eight columns of a row from n on: dz, which is added to sum.
template <typename T, int ACT> __device__ __forceinline__ void act_row(const ActBwdArgs& a, const Raw8<T>& dy, const Raw8<T>& z, long long t, int n, float* sum) {
    constexpr bool by_z = ACT != MOE_ACT_NONE;
    float d[8], v[8];
    dy.to_float(d);
    if (by_z) z.to_float(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (by_z) d[i] *= activation_slope<T>(v[i], ACT);
        sum[i] += d[i];
    }
    if (a.dz) {
        T* o = reinterpret_cast<T*>(a.dz) + t * a.ldz + n;
        if constexpr (sizeof(T) == 2) {
            const uint4 w = make_uint4(pack_bf16x2(d[0], d[1]), pack_bf16x2(d[2], d[3]), pack_bf16x2(d[4], d[5]), pack_bf16x2(d[6], d[7]));
            if (a.past) store_once_anywhere(o, w); else *reinterpret_cast<uint4*>(o) = w;
        } else {
            const float4 lo = make_float4(d[0], d[1], d[2], d[3]), hi = make_float4(d[4], d[5], d[6], d[7]);
            if (a.past) {
                store_once_anywhere(o, lo);
                store_once_anywhere(o + 4, hi);
            } else {
                reinterpret_cast<float4*>(o)[0] = lo;
                reinterpret_cast<float4*>(o)[1] = hi;
            }
        }
    }
}

// A wavefront has 512 columns, eight to a lane, and some of the workgroup's rows; as many of the wavefronts as there are columns for
// stand side by side in a row, the others have other rows.  The columns' sums stay in registers over the rows.  Bound by memory: 16384 x 8192,
// GeLU, bfloat16 148 us, 5.4 TB/s (a copy of as much 155), and 4.6 us of the sums' launch.
template <typename T, int ACT>
__global__ __launch_bounds__(ACT_WAVES * 64) void act_bwd_kernel(ActBwdArgs a) {
    __shared__ float sums[ACT_WAVES][ACT_COLS];
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, beside = wid % a.beside, below = wid / a.beside, rows = ACT_WAVES / a.beside;
    const int n = (blockIdx.x * a.beside + beside) * ACT_COLS + lane * 8;
    const int begin = blockIdx.y * a.rows, end = begin + a.rows < a.T ? begin + a.rows : a.T;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (n < a.N) {
        constexpr bool by_z = ACT != MOE_ACT_NONE;
        // so many rows of a wavefront are requested before the first is worked on
        constexpr int AT_ONCE = 2;
        for (int t0 = begin + below; t0 < end; t0 += AT_ONCE * rows) {
            Raw8<T> dy[AT_ONCE], z[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const long long t = t0 + u * rows;
                if (t >= end) continue;
                load_eight_once(dy[u], reinterpret_cast<const T*>(a.dy) + t * a.ldy + n);
                if (by_z) load_eight_once(z[u], reinterpret_cast<const T*>(a.z) + t * a.ldz + n);
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const long long t = t0 + u * rows;
                if (t >= end) continue;
                act_row<T, ACT>(a, dy[u], z[u], t, n, sum);
            }
        }
    }
    if (!a.part) return;
    *reinterpret_cast<float4*>(&sums[wid][lane * 8]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
    *reinterpret_cast<float4*>(&sums[wid][lane * 8 + 4]) = make_float4(sum[4], sum[5], sum[6], sum[7]);
    __syncthreads();
    for (int c = threadIdx.x; c < a.beside * ACT_COLS; c += ACT_WAVES * 64) {
        const int col = blockIdx.x * a.beside * ACT_COLS + c;
        float v = 0.0f;
        for (int r = 0; r < rows; ++r) v += sums[r * a.beside + c / ACT_COLS][c % ACT_COLS];
        if (col < a.N) a.part[(long long)blockIdx.y * a.N + col] = v;
    }
}

// Few rows: a workgroup has 64 columns of all of them, eight threads to a row, and with them the whole of the bias's gradient, which saves the
// second launch (us so / otherwise, with the bias's gradient: 64 rows of 3648 floats 4.8 / 7.0; 64 x 8192 floats, GeLU 5.2 / 8.5; 256 x 8192, SiLU 6.2 / 8.9;
// but 200 x 512 floats, GeLU, whose float form is a few hundred instructions, 11.6 / 7.3).
constexpr int ACT_FEW_COLS = 64, ACT_FEW_THREADS = 256;
int act_few(const LinearDims& d) { return d.bf16 || d.act == MOE_ACT_NONE ? 256 : 64; }
template <typename T, int ACT>
__global__ __launch_bounds__(ACT_FEW_THREADS) void act_bwd_few_kernel(ActBwdArgs a) {
    __shared__ float sums[ACT_FEW_THREADS / 64][ACT_FEW_COLS];
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, c = (lane & 7) * 8, n = blockIdx.x * ACT_FEW_COLS + c;
    constexpr int ROWS = ACT_FEW_THREADS / 8, AT_ONCE = 2;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (n < a.N) {
        for (int t0 = threadIdx.x / 8; t0 < a.T; t0 += AT_ONCE * ROWS) {
            Raw8<T> dy[AT_ONCE], z[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const long long t = t0 + u * ROWS;
                if (t >= a.T) continue;
                load_eight_once(dy[u], reinterpret_cast<const T*>(a.dy) + t * a.ldy + n);
                if (ACT != MOE_ACT_NONE) load_eight_once(z[u], reinterpret_cast<const T*>(a.z) + t * a.ldz + n);
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const long long t = t0 + u * ROWS;
                if (t < a.T) act_row<T, ACT>(a, dy[u], z[u], t, n, sum);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int off = 8; off < 64; off <<= 1) sum[i] += __shfl_xor(sum[i], off, 64);
    }
    if (lane < 8) {
        *reinterpret_cast<float4*>(&sums[wid][c]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
        *reinterpret_cast<float4*>(&sums[wid][c + 4]) = make_float4(sum[4], sum[5], sum[6], sum[7]);
    }
    __syncthreads();
    const int col = blockIdx.x * ACT_FEW_COLS + threadIdx.x;
    if (threadIdx.x >= ACT_FEW_COLS || col >= a.N) return;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < ACT_FEW_THREADS / 64; ++w) v += sums[w][threadIdx.x];
    a.dbias[col] = a.store ? v : a.dbias[col] + v;
}

template <typename T, int ACT> void act_bwd_launch(const ActBwdArgs& a, dim3 grid, hipStream_t s) {
    if (a.dbias) act_bwd_few_kernel<T, ACT><<<up(a.N, ACT_FEW_COLS), ACT_FEW_THREADS, 0, s>>>(a);
    else act_bwd_kernel<T, ACT><<<grid, ACT_WAVES * 64, 0, s>>>(a);
}
template <typename T> moe_status act_bwd_launch(const ActBwdArgs& a, dim3 grid, hipStream_t s) {
    if (a.act == MOE_ACT_GELU) act_bwd_launch<T, MOE_ACT_GELU>(a, grid, s);
    else if (a.act == MOE_ACT_SILU) act_bwd_launch<T, MOE_ACT_SILU>(a, grid, s);
    else act_bwd_launch<T, MOE_ACT_NONE>(a, grid, s);
    MOE_CHECK_LAUNCH();
    return MOE_OK;
}

// out (+)= sum over p of part[p].  A wavefront adds every 16th of them, in order, and the wavefronts' sums are added in theirs.
__global__ __launch_bounds__(1024) void join_columns_kernel(const float* __restrict__ part, int parts, int size, float* __restrict__ out, int store) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, i = blockIdx.x * 64 + lane;
    float v = 0.0f;
    if (i < size) {
#pragma unroll 8
        for (int p = wid; p < parts; p += 16) v += part[(long long)p * size + i];
    }
    sums[wid][lane] = v;
    __syncthreads();
    if (wid > 0 || i >= size) return;
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) v += sums[w][lane];
    out[i] = store ? v : out[i] + v;
}
// The same for many columns, a thread to each (520 x 1000, twelve parts of a weight gradient: 25 MB, mostly cached, in 5.8 us)
__global__ __launch_bounds__(256) void join_parts_kernel(const float* __restrict__ part, int parts, long long size, float* __restrict__ out, int store) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= size) return;
    float v = 0.0f;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) v += part[p * size + i];
    out[i] = store ? v : out[i] + v;
}
moe_status join_parts(const float* part, int parts, long long size, float* out, int store, hipStream_t s) {
    join_parts_kernel<<<up(size, 256), 256, 0, s>>>(part, parts, size, out, store);
    MOE_CHECK_LAUNCH();
    return MOE_OK;
}

moe_status gemm(const LinearDims& d, GemmLayout lay, int epi, const GemmArgs& a, hipStream_t s) {
    return d.bf16 ? gemm_bf16(lay, epi, a, s) : gemm_f32(lay, epi, a, s);
}

// A product of one block of rows in slices of its sum, whose partial sums the epilogue adds up.  g: A, B, their strides, N, K.
moe_status sliced(const LinearDims& d, GemmLayout lay, int slices, GemmArgs g, const FewLinearArgs& a, hipStream_t s) {
    g = slice_of(g, slices);
    g.a_estride = g.K;
    g.b_estride = lay == GEMM_NN ? (long long)g.K * g.ldb : g.K;
    g.C = a.partial;
    g.c_estride = (long long)d.T * g.N;
    g.ldc = g.N;
    MOE_TRY(gemm(d, lay, EPI_STORE_F32 | EPI_SLICES, g, s));
    return d.bf16 ? linear_finish_launch<bf16_t>(a, g.E, s) : linear_finish_launch<float>(a, g.E, s);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

}  // namespace moe

extern "C" moe_status moe_linear_scratch_bytes(const moe_linear_config* cfg, size_t* bytes) {
    moe::LinearDims d;
    MOE_TRY(moe::linear_dims(cfg, &d));
    if (!bytes) return MOE_ERR_NULL;
    *bytes = 0;
    if (d.T == 0) return MOE_OK;
    size_t most = 16;
    if (d.wblocks > 1) most = (size_t)d.wblocks * d.K * d.N * 4;
    const size_t act = (size_t)moe::act_blocks(d) * d.N * 4;
    if (act > most) most = act;
    if (d.T <= moe::FEW_LINEAR_ROWS && d.slices > 1) {
        const size_t few = (size_t)d.slices * d.T * d.N * 4;
        if (few > most) most = few;
    }
    const size_t fwd = (size_t)moe::fwd_slices(d) * d.T * d.N * 4, dx = (size_t)moe::dx_slices(d) * d.T * d.K * 4;
    if (moe::fwd_slices(d) > 1 && fwd > most) most = fwd;
    if (moe::dx_slices(d) > 1 && dx > most) most = dx;
    *bytes = moe::align16(most);
    return MOE_OK;
}

extern "C" moe_status moe_linear_tile(const moe_linear_config* cfg, int32_t gemm, int32_t* rows, int32_t* cols, int32_t* sums) {
    moe::LinearDims d;
    MOE_TRY(moe::linear_dims(cfg, &d));
    if (!rows || !cols || !sums) return MOE_ERR_NULL;
    if (gemm < MOE_LINEAR_FWD || gemm > MOE_LINEAR_DW) return MOE_ERR_SHAPE;
    *rows = *cols = *sums = 0;
    if (d.T == 0) return MOE_OK;
    if (gemm == MOE_LINEAR_FWD && d.T <= moe::FEW_LINEAR_ROWS) {
        *rows = (d.T > moe::Few<float>::ROWS ? 2 : 1) * moe::Few<float>::ROWS;
        *cols = d.bf16 ? moe::Few<moe::bf16_t>::COLS : moe::Few<float>::COLS;
        *sums = moe::few_linear_slices(d);
        return MOE_OK;
    }
    const moe::GemmLayout lay = gemm == MOE_LINEAR_FWD ? moe::GEMM_NN : gemm == MOE_LINEAR_DX ? moe::GEMM_NT : moe::GEMM_TN;
    moe::GemmArgs g = gemm == MOE_LINEAR_FWD ? moe::fwd_gemm(d) : gemm == MOE_LINEAR_DX ? moe::dx_gemm(d) : moe::dw_gemm(d);
    int epi = gemm == MOE_LINEAR_FWD ? moe::EPI_LINEAR : moe::EPI_STORE;
    if (gemm == MOE_LINEAR_DW) {
        *sums = d.wblocks;
        epi = d.wblocks > 1 || d.overwrite ? moe::EPI_STORE_F32 : moe::EPI_ACCUM_F32;
    } else {
        const int slices = moe::gemm_slices(d, lay, g);
        if (slices > 1) {
            g = moe::slice_of(g, slices);
            epi = moe::EPI_STORE_F32 | moe::EPI_SLICES;
        }
        *sums = slices > 1 ? g.E : 1;
    }
    if (d.bf16) moe::gemm_bf16_tile(lay, epi, g, rows, cols);
    else moe::gemm_f32_tile(rows, cols);
    return MOE_OK;
}

extern "C" moe_status moe_linear_fwd(const moe_linear_config* cfg, const void* x, const void* W, const float* bias, const void* residual,
                                     void* z, void* y, void* scratch, void* stream) {
    moe::LinearDims d;
    MOE_TRY(moe::linear_dims(cfg, &d));
    if (d.T == 0) return MOE_OK;
    if (!x || !W || !y || !scratch) return MOE_ERR_NULL;
    if (!moe::aligned16(x) || !moe::aligned16(W) || !moe::aligned16(residual) || !moe::aligned16(z) || !moe::aligned16(y) || !moe::aligned16(scratch))
        return MOE_ERR_UNSUPPORTED;
    hipStream_t s = (hipStream_t)stream;
    if (d.T <= moe::FEW_LINEAR_ROWS) {
        moe::FewLinearArgs a = {x, W, bias, residual, z, y, (float*)scratch, d.ldx, d.ldy, d.ldr, d.ldz, d.T, d.K, d.N, d.act, 0};
        {
            moe::ProfScope prof(moe::PK_LINEAR, s);
            MOE_TRY(d.bf16 ? moe::few_linear<moe::bf16_t>(d, a, s) : moe::few_linear<float>(d, a, s));
        }
        moe::count_launch(moe::LC_GEMM);
        return MOE_OK;
    }
    moe::GemmArgs g = moe::fwd_gemm(d);
    g.A = x; g.B = W; g.C = y;
    g.a_estride = d.block * d.ldx; g.b_estride = 0; g.c_estride = d.block * d.ldy;
    g.lda = (int)d.ldx; g.ldb = d.N; g.ldc = (int)d.ldy;
    g.Z = z; g.ldz = (int)d.ldz;
    g.bias = bias; g.R = residual; g.ldr = (int)d.ldr;
    const int slices = moe::fwd_slices(d);
    if (slices > 1)
        return moe::sliced(d, moe::GEMM_NN, slices, g,
                           {x, W, bias, residual, z, y, (float*)scratch, d.ldx, d.ldy, d.ldr, d.ldz, d.T, d.K, d.N, d.act, 0}, s);
    return moe::gemm(d, moe::GEMM_NN, moe::EPI_LINEAR, g, s);
}

extern "C" moe_status moe_act_bwd(const moe_linear_config* cfg, const void* dy, const void* z, void* dz, float* dbias, void* scratch, void* stream) {
    moe::LinearDims d;
    MOE_TRY(moe::linear_dims(cfg, &d));
    hipStream_t s = (hipStream_t)stream;
    if (d.T == 0) {
        if (dbias && d.overwrite) MOE_TRY(moe::join_parts(nullptr, 0, d.N, dbias, 1, s));
        return MOE_OK;
    }
    if (!dy || (!dz && !dbias) || (!z && d.act != MOE_ACT_NONE) || (dbias && !scratch)) return MOE_ERR_NULL;
    if (!moe::aligned16(dy) || !moe::aligned16(z) || !moe::aligned16(dz) || !moe::aligned16(scratch)) return MOE_ERR_UNSUPPORTED;
    const int blocks = moe::act_blocks(d);
    const bool few = dbias && d.T <= moe::act_few(d);
    moe::ActBwdArgs a = {dy, z, dz, dbias && !few ? (float*)scratch : nullptr, few ? dbias : nullptr, d.overwrite, d.ldy, d.ldz, d.T, d.N, d.act, moe::up(d.T, blocks), moe::act_beside(d),
                         (long long)d.T * d.N * (d.bf16 ? 2 : 4) > moe::ACT_PAST};
    const int parts = moe::up(d.T, a.rows);
    {
        moe::ProfScope prof(moe::PK_ACT_BWD, s);
        const dim3 grid(moe::up(d.N, a.beside * moe::ACT_COLS), parts);
        MOE_TRY(d.bf16 ? moe::act_bwd_launch<moe::bf16_t>(a, grid, s) : moe::act_bwd_launch<float>(a, grid, s));
        if (a.part) {
            moe::join_columns_kernel<<<moe::up(d.N, 64), 1024, 0, s>>>(a.part, parts, d.N, dbias, d.overwrite);
            MOE_CHECK_LAUNCH();
        }
    }
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

extern "C" moe_status moe_linear_bwd(const moe_linear_config* cfg, const void* dz, const void* x, const void* W, const void* add, void* dx,
                                     float* dW, void* scratch, void* stream) {
    moe::LinearDims d;
    MOE_TRY(moe::linear_dims(cfg, &d));
    hipStream_t s = (hipStream_t)stream;
    if (d.T == 0) {
        if (dW && d.overwrite) MOE_TRY(moe::join_parts(nullptr, 0, (long long)d.K * d.N, dW, 1, s));
        return MOE_OK;
    }
    if (!dz || (!dx && !dW) || (dx && !W) || (dW && !x) || !scratch) return MOE_ERR_NULL;
    if (!moe::aligned16(dz) || !moe::aligned16(x) || !moe::aligned16(W) || !moe::aligned16(add) || !moe::aligned16(dx) || !moe::aligned16(dW) ||
        !moe::aligned16(scratch))
        return MOE_ERR_UNSUPPORTED;
    if (dx) {
        moe::GemmArgs g = moe::dx_gemm(d);
        g.A = dz; g.B = W; g.C = dx;
        g.a_estride = d.block * d.ldz; g.b_estride = 0; g.c_estride = d.block * d.ldx;
        g.lda = (int)d.ldz; g.ldb = d.N; g.ldc = (int)d.ldx;
        g.R = add; g.ldr = (int)d.ldx;
        const int slices = moe::dx_slices(d);
        if (slices > 1) {
            MOE_TRY(moe::sliced(d, moe::GEMM_NT, slices, g,
                                {dz, W, nullptr, add, nullptr, dx, (float*)scratch, d.ldz, d.ldx, d.ldx, 0, d.T, d.N, d.K, MOE_ACT_NONE, 0}, s));
        } else {
            // (with nothing to add, the plain store's epilogue, us back to back against the one that adds: 30011 rows, 520 x 1000 64.7 and 71.8,
            // 4096 rows, 4096 x 1024 31.1 and 37.6, 8192 rows, 2048 x 8192 190 and 191; between the weight gradient's launches the first
            // takes 71)
            MOE_TRY(moe::gemm(d, moe::GEMM_NT, add ? moe::EPI_LINEAR : moe::EPI_STORE | moe::EPI_BLOCKS, g, s));
        }
    }
    if (dW) {
        moe::GemmArgs g = moe::dw_gemm(d);
        const bool split = d.wblocks > 1;
        float* parts = (float*)scratch;
        g.A = x; g.B = dz; g.C = split ? parts : dW;
        g.a_estride = d.wblock * d.ldx; g.b_estride = d.wblock * d.ldz; g.c_estride = (long long)d.K * d.N;
        g.lda = (int)d.ldx; g.ldb = (int)d.ldz; g.ldc = d.N;
        MOE_TRY(moe::gemm(d, moe::GEMM_TN, (split || d.overwrite ? moe::EPI_STORE_F32 : moe::EPI_ACCUM_F32) | moe::EPI_BLOCKS, g, s));
        if (split) MOE_TRY(moe::join_parts(parts, d.wblocks, (long long)d.K * d.N, dW, d.overwrite, s));
    }
    return MOE_OK;
}
