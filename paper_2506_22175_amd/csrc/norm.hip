// Root-mean-square norm behind the residual's addition, and its backward pass.
//
//   forward   h = x + r,  rstd = 1 / sqrt(mean(h^2) + eps),  y = h rstd g
//   backward  n = h rstd,  dx = dh + rstd (g dy - n mean(g dy n)),  dg = sum over rows of dy n
//
// Both move each row once and are bound by memory: a row stays in the registers of the threads that loaded it, from the
// loads through the row's sum to the stores, so nothing is read twice.  A row is dealt out in units of eight columns (16
// bytes of bfloat16), to a thread one (forward) or a few; a wavefront has a row of up to 512 columns to itself, a workgroup a
// longer one.  Rows need the alignment of their elements only: the hardware does wide accesses
// at any address, and a row's last unit, if it is not full, goes element by element.  32768 rows of 2048 in bfloat16 with h: 94 us
// (5.7 TB/s; a copy of 1 GiB 4.7); 7001 rows of 4040 to e4m3 42 us (4.8 TB/s); backward, the first 103 us (5.2 TB/s).
#include "common.h"
#include "lanes.h"
#include "wide.h"
#include <cmath>

namespace moe {

namespace {

template <int ALIGN> using Any16 = Anywhere<16, ALIGN>;
using Any8 = Anywhere<8, 1>;

// eight columns as stored
template <typename T> struct Unit8;
template <> struct Unit8<bf16_t> {
    Any16<2> u;
    __device__ __forceinline__ void load(const bf16_t* p, int left) {
        if (left >= 8) {
            u = *reinterpret_cast<const Any16<2>*>(p);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned lo = 2 * i < left ? p[2 * i] : 0, hi = 2 * i + 1 < left ? p[2 * i + 1] : 0;
                u.w[i] = lo | hi << 16;
            }
        }
    }
    __device__ __forceinline__ void zero() { u.w[0] = u.w[1] = u.w[2] = u.w[3] = 0; }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float((i & 1) ? u.w[i / 2] & 0xffff0000u : u.w[i / 2] << 16); }
    static __device__ __forceinline__ void store(bf16_t* p, const float* v, int left) {
        if (left >= 8) {
            Any16<2> o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o.w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
            *reinterpret_cast<Any16<2>*>(p) = o;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i] = f32_to_bf16(v[i]);
        }
    }
};
template <> struct Unit8<float> {
    Any16<4> u[2];
    __device__ __forceinline__ void load(const float* p, int left) {
        if (left >= 8) {
            u[0] = reinterpret_cast<const Any16<4>*>(p)[0];
            u[1] = reinterpret_cast<const Any16<4>*>(p)[1];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i / 4].w[i % 4] = i < left ? __float_as_uint(p[i]) : 0u;
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i / 4].w[i % 4] = 0;
    }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(u[i / 4].w[i % 4]); }
    static __device__ __forceinline__ void store(float* p, const float* v, int left) {
        if (left >= 8) {
            Any16<4> o[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i / 4].w[i % 4] = __float_as_uint(v[i]);
            reinterpret_cast<Any16<4>*>(p)[0] = o[0];
            reinterpret_cast<Any16<4>*>(p)[1] = o[1];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i] = v[i];
        }
    }
};

__device__ __forceinline__ void load_gain(const float* gain, int col, int left, float* g) {
    if (!gain) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.0f;
        return;
    }
    Unit8<float> u;
    u.load(gain + col, left);
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = u.at(i);
}

// sum / largest over the threads of a row (one wavefront, or the workgroup's waves through `s`)
template <int WAVES> __device__ __forceinline__ float row_sum(float v, float* s) {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += s[i];
        __syncthreads();
    }
    return v;
}
template <int WAVES> __device__ __forceinline__ unsigned row_max(unsigned v, float* s) {
    v = wave_max_bits(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = __uint_as_float(v);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const unsigned o = __float_as_uint(s[i]);
            v = v > o ? v : o;
        }
        __syncthreads();
    }
    return v;
}

struct NormArgs {
    const void* x; const void* r; const float* gain; void* h; void* y; float* scales; float* rstd;
    long long ldx, ldr, ldh, ldy, first;     // first: row of the launch
    int T, M, group, n_scales;
    float eps;
};

constexpr float E4M3_MOST = 448.0f;

// The magnitudes' bits order like the magnitudes, infinities above all numbers and NaN above those, so that a NaN is the
// largest of its group and makes the scale NaN.
__device__ __forceinline__ float scale_of(unsigned bits) {
    const float s = __uint_as_float(bits) / E4M3_MOST;
    return s < 1.17549435e-38f ? 1.17549435e-38f : s;
}

// WAVES wavefronts a row, UNITS units of eight columns a thread; four rows to a workgroup of 256 where WAVES = 1
template <typename T, bool E4M3, int WAVES, int UNITS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void norm_kernel(NormArgs a) {
    constexpr int ROWS = WAVES == 1 ? 4 : 1, THREADS = WAVES * 64;
    __shared__ float s_part[WAVES > 1 ? WAVES : 1];
    const long long row = a.first + (long long)blockIdx.x * ROWS + (WAVES == 1 ? threadIdx.x >> 6 : 0);
    if (row >= a.T) return;                                // whole wavefronts, and only where a row is one
    const int tid = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const T* x = reinterpret_cast<const T*>(a.x) + row * a.ldx;
    const T* r = a.r ? reinterpret_cast<const T*>(a.r) + row * a.ldr : nullptr;
    Unit8<T> ux[UNITS], ur[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int col = (u * THREADS + tid) * 8, left = a.M - col;
        ux[u].zero();
        if (left > 0) ux[u].load(x + col, left);
    }
    if (r) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int col = (u * THREADS + tid) * 8, left = a.M - col;
            ur[u].zero();
            if (left > 0) ur[u].load(r + col, left);
        }
    }
    float h[UNITS][8], sum = 0.0f;
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[u][i] = r ? ux[u].at(i) + ur[u].at(i) : ux[u].at(i);
            sum = fmaf(h[u][i], h[u][i], sum);
        }
    // The gain is requested before the stores of h, behind which it cannot go ahead, where it does not cost wavefronts.
    constexpr bool EARLY = UNITS <= 2;
    Unit8<float> ug[EARLY ? UNITS : 1];
    if (EARLY && a.gain) {
#pragma unroll
        for (int u = 0; u < (EARLY ? UNITS : 0); ++u) {
            const int col = (u * THREADS + tid) * 8, left = a.M - col;
            if (left > 0) ug[u].load(a.gain + col, left);
        }
    }
    if (a.h) {
        T* ho = reinterpret_cast<T*>(a.h) + row * a.ldh;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int col = (u * THREADS + tid) * 8, left = a.M - col;
            if (left > 0) Unit8<T>::store(ho + col, h[u], left);
        }
    }
    sum = row_sum<WAVES>(sum, s_part);
    const float rstd = 1.0f / sqrtf(sum / (float)a.M + a.eps);
    if (a.rstd && tid == 0) a.rstd[row] = rstd;
    unsigned most[UNITS], row_most = 0;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int col = (u * THREADS + tid) * 8, left = a.M - col;
        most[u] = 0;
        if (left <= 0) {
            if constexpr (E4M3) {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[u][i] = 0.0f;   // columns past the row's end: not the NaN of 0 * a row's NaN
            }
            continue;
        }
        if (!EARLY && a.gain) ug[0].load(a.gain + col, left);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[u][i] *= rstd;
            if (a.gain) h[u][i] *= ug[EARLY ? u : 0].at(i);
            if constexpr (E4M3) {
                const unsigned m = __float_as_uint(h[u][i]) & 0x7fffffffu;
                if (i < left && m > most[u]) most[u] = m;
            }
        }
        if constexpr (!E4M3) Unit8<T>::store(reinterpret_cast<T*>(a.y) + row * a.ldy + col, h[u], left);
    }
    if constexpr (E4M3) {
        if (a.group) {
#pragma unroll
            for (int u = 0; u < UNITS; ++u) most[u] = row_max_bits(most[u]);        // 16 lanes' units make 128 columns
        } else {
#pragma unroll
            for (int u = 0; u < UNITS; ++u) row_most = row_most > most[u] ? row_most : most[u];
            row_most = row_max<WAVES>(row_most, s_part);
        }
        unsigned char* y = reinterpret_cast<unsigned char*>(a.y) + row * a.ldy;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int col = (u * THREADS + tid) * 8, left = a.M - col;
            if (left <= 0) continue;
            const float scale = scale_of(a.group ? most[u] : row_most);
            if (a.group ? (tid & 15) == 0 : u == 0 && tid == 0) a.scales[row * a.n_scales + (a.group ? col >> 7 : 0)] = scale;
            Any8 o;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                int w = __builtin_amdgcn_cvt_pk_fp8_f32(h[u][4 * q] / scale, h[u][4 * q + 1] / scale, 0, false);
                w = __builtin_amdgcn_cvt_pk_fp8_f32(h[u][4 * q + 2] / scale, h[u][4 * q + 3] / scale, w, true);
                o.w[q] = (unsigned)w;
            }
            if (left >= 8) {
                *reinterpret_cast<Any8*>(y + col) = o;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < left) y[col + i] = (unsigned char)(o.w[i / 4] >> (8 * (i % 4)));
            }
        }
    }
}

struct NormBwdArgs {
    const void* dy; const void* h; const float* gain; const float* rstd; const void* dh; void* dx;
    float* part;          // [row workgroups, M] sums of the gain's gradient; one workgroup: the gradient itself
    float* dgain;         // of the column workgroups
    long long ldx, ldh, ldy;
    int T, M, add;        // add: what is there is added to (one workgroup, or column workgroups)
    int col_blocks;       // the first workgroups have columns of the gain's gradient, the others rows
};

// The gain's gradient of 32 columns: four threads a row, eight columns each, the others every THREADS / 4-th row.
constexpr int GAIN_UNITS = 4;
template <typename T, int THREADS> __device__ __forceinline__ void gain_columns(const NormBwdArgs& a) {
    __shared__ float s[THREADS / 64][GAIN_UNITS * 8];
    const int unit = threadIdx.x % GAIN_UNITS, col = (blockIdx.x * GAIN_UNITS + unit) * 8, left = a.M - col;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (left > 0) {
        const T* dy = reinterpret_cast<const T*>(a.dy) + col;
        const T* h = reinterpret_cast<const T*>(a.h) + col;
#pragma unroll 4
        for (int row = threadIdx.x / GAIN_UNITS; row < a.T; row += THREADS / GAIN_UNITS) {
            Unit8<T> ud, uh;
            ud.load(dy + row * a.ldy, left);
            uh.load(h + row * a.ldh, left);
            const float rstd = a.rstd[row];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(ud.at(i), uh.at(i) * rstd, v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int away = GAIN_UNITS; away < 64; away *= 2) v[i] += __shfl_xor(v[i], away, 64);
    if ((threadIdx.x & 63) < GAIN_UNITS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[threadIdx.x >> 6][unit * 8 + i] = v[i];
    }
    __syncthreads();
    const int c = blockIdx.x * GAIN_UNITS * 8 + threadIdx.x;
    if (threadIdx.x >= GAIN_UNITS * 8 || c >= a.M) return;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) sum += s[w][threadIdx.x];
    a.dgain[c] = a.add ? a.dgain[c] + sum : sum;
}

// Each wavefront (WAVES = 1) or workgroup takes every gridDim-th row and keeps its sums of the gain's gradient in registers.
template <typename T, int WAVES, int UNITS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void norm_bwd_kernel(NormBwdArgs a) {
    constexpr int ROWS = WAVES == 1 ? 4 : 1, THREADS = WAVES * 64;
    if ((int)blockIdx.x < a.col_blocks) {
        gain_columns<T, WAVES == 1 ? 256 : THREADS>(a);
        return;
    }
    const int block = blockIdx.x - a.col_blocks, blocks = gridDim.x - a.col_blocks;
    __shared__ float s_part[WAVES > 1 ? WAVES : 1];
    __shared__ float s_dg[WAVES == 1 ? 3 * UNITS * THREADS * 8 : 1];
    const int tid = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int sub = WAVES == 1 ? threadIdx.x >> 6 : 0;
    float dg[UNITS][8];
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[u][i] = 0.0f;
    const long long step = (long long)blocks * ROWS;
    Unit8<T> ud[UNITS], uh[UNITS], ub[UNITS];
    float rstd = 0.0f;
    auto request = [&](long long row) {
        const T* dy = reinterpret_cast<const T*>(a.dy) + row * a.ldy;
        const T* hp = reinterpret_cast<const T*>(a.h) + row * a.ldh;
        const T* dh = reinterpret_cast<const T*>(a.dh) + row * a.ldh;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int col = (u * THREADS + tid) * 8, left = a.M - col;
            if (left <= 0) continue;
            ud[u].load(dy + col, left);
            uh[u].load(hp + col, left);
            if (a.dh) ub[u].load(dh + col, left);
        }
        rstd = a.rstd[row];
    };
    // Where the registers allow it the next row is on its way while one is summed up and stored.
    constexpr bool AHEAD = UNITS <= 2;
    long long row = (long long)block * ROWS + sub;
    if (AHEAD && row < a.T) request(row);
    for (; row < a.T; row += step) {
        if (!AHEAD) request(row);
        float n[UNITS][8], d[UNITS][8], sum = 0.0f;
        Unit8<T> plus[UNITS];
        const float r = rstd;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int col = (u * THREADS + tid) * 8, left = a.M - col;
            if (left <= 0) continue;
            plus[u] = ub[u];
            float g[8];
            load_gain(a.gain, col, left, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[u][i] = uh[u].at(i) * r;
                d[u][i] = ud[u].at(i);
                dg[u][i] = fmaf(d[u][i], n[u][i], dg[u][i]);
                d[u][i] *= g[i];
                if (i < left) sum = fmaf(d[u][i], n[u][i], sum);
            }
        }
        if (AHEAD && row + step < a.T) request(row + step);
        const float mean = row_sum<WAVES>(sum, s_part) / (float)a.M;
        T* dx = reinterpret_cast<T*>(a.dx) + row * a.ldx;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int col = (u * THREADS + tid) * 8, left = a.M - col;
            if (left <= 0) continue;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                o[i] = r * fmaf(-n[u][i], mean, d[u][i]);
                if (a.dh) o[i] += plus[u].at(i);
            }
            Unit8<T>::store(dx + col, o, left);
        }
    }
    if (!a.part) return;
    if constexpr (WAVES == 1) {
        // the four wavefronts' sums, in their order
        if (sub > 0) {
            float* s = s_dg + (sub - 1) * UNITS * THREADS * 8;
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[(u * 8 + i) * THREADS + tid] = dg[u][i];
        }
        __syncthreads();
        if (sub > 0) return;
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) dg[u][i] += s_dg[q * UNITS * THREADS * 8 + (u * 8 + i) * THREADS + tid];
    }
    float* part = a.part + (long long)block * a.M;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int col = (u * THREADS + tid) * 8, left = a.M - col;
        if (left <= 0) continue;
        if (a.add) {
            Unit8<float> old;
            old.load(part + col, left);
#pragma unroll
            for (int i = 0; i < 8; ++i) dg[u][i] += old.at(i);
        }
        Unit8<float>::store(part + col, dg[u], left);
    }
}

// dgain (+)= the sums of `parts` workgroups, 16 columns to a workgroup: 64 threads a column, each takes every 64th part
constexpr int DG_COLS = 16, DG_SPLIT = 64;
__global__ __launch_bounds__(DG_COLS * DG_SPLIT) void norm_dgain_kernel(const float* __restrict__ part, int parts, int M, int add,
                                                                        float* __restrict__ dgain) {
    __shared__ float s[DG_SPLIT][DG_COLS + 1];
    const int c = threadIdx.x % DG_COLS, q = threadIdx.x / DG_COLS;
    const int col = blockIdx.x * DG_COLS + c;
    float v = 0.0f;
    if (col < M) {
#pragma unroll 8
        for (int p = q; p < parts; p += DG_SPLIT) v += part[(long long)p * M + col];
    }
    s[q][c] = v;
    __syncthreads();
    if (q == 0 && col < M) {
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < DG_SPLIT; ++i) v += s[i][c];
        dgain[col] = add ? dgain[col] + v : v;
    }
}

struct NormDims { int T, M, es; long long ldx, ldr, ldh, ldy; int n_scales; };

moe_status norm_dims(const moe_norm_config* c, NormDims* d) {
    if (!c) return MOE_ERR_NULL;
    if (c->T < 0 || c->M <= 0 || !(c->eps >= 0.0f) || !std::isfinite(c->eps)) return MOE_ERR_SHAPE;
    if (c->dtype != MOE_F32 && c->dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (c->out != c->dtype && c->out != MOE_E4M3) return MOE_ERR_UNSUPPORTED;
    if (c->group != 0 && (c->group != 128 || c->out != MOE_E4M3)) return MOE_ERR_UNSUPPORTED;
    if (c->grad_overwrite != 0 && c->grad_overwrite != 1) return MOE_ERR_UNSUPPORTED;
    if (c->M > 32768) return MOE_ERR_UNSUPPORTED;
    d->T = c->T; d->M = c->M; d->es = c->dtype == MOE_F32 ? 4 : 2;
    const int64_t given[4] = {c->ldx, c->ldr, c->ldh, c->ldy};
    long long* ld[4] = {&d->ldx, &d->ldr, &d->ldh, &d->ldy};
    for (int i = 0; i < 4; ++i) {
        if (given[i] != 0 && given[i] < c->M) return MOE_ERR_SHAPE;
        *ld[i] = given[i] ? given[i] : c->M;
    }
    d->n_scales = c->group ? (c->M + 127) / 128 : 1;
    return MOE_OK;
}

// How a row is dealt out: wavefronts per row and units per thread.  One unit to a thread as far as that goes, which leaves the
// most requests under way: two or four units to a thread and fewer wavefronts without a barrier take longer for few rows (64
// of 2048, bfloat16: 4.5 us, so 2.9) and for float ones (8192 of 1024: 39 us, so 33; of 4096: 134 and 110), and as long for many
// of bfloat16 (32768 of 2048: 95 and 95 us; of 600, where the second wavefront has little to do: 32 and 34).
struct RowPlan { int waves, units; };
RowPlan norm_plan(int M) {
    const int units = (M + 7) / 8;
    if (units <= 64) return {1, 1};
    if (units <= 128) return {2, 1};
    if (units <= 256) return {4, 1};
    if (units <= 512) return {8, 1};
    if (units <= 1024) return {16, 1};
    if (units <= 2048) return {16, 2};
    return {16, 4};
}

// Backward has several rows after one another: few units to a thread, so that the next row can be on its way.  Two and four
// units to the threads of one wavefront instead of a workgroup's: 4096 rows of 2048 25 us, so 20; 512 of 1024 6.9 and 7.5.
RowPlan norm_bwd_plan(int M) {
    const int units = (M + 7) / 8;
    if (units <= 64) return {1, 1};
    if (units <= 256) return {4, 1};
    if (units <= 512) return {4, 2};
    if (units <= 1024) return {16, 1};
    if (units <= 2048) return {16, 2};
    return {16, 4};
}

template <typename T, bool E4M3> void norm_launch(NormArgs a, RowPlan p, hipStream_t s) {
    const long long most = LAUNCH_THREADS / (p.waves * 64);
    for (a.first = 0; a.first < a.T; a.first += most) {
        const int rows = (int)(a.T - a.first < most ? a.T - a.first : most);
#define NORM_CASE(W, U) if (p.waves == W && p.units == U) \
            norm_kernel<T, E4M3, W, U><<<W == 1 ? (rows + 3) / 4 : rows, W == 1 ? 256 : W * 64, 0, s>>>(a);
        NORM_CASE(1, 1) NORM_CASE(2, 1) NORM_CASE(4, 1) NORM_CASE(8, 1) NORM_CASE(16, 1) NORM_CASE(16, 2) NORM_CASE(16, 4)
#undef NORM_CASE
    }
}

template <typename T> void norm_bwd_launch(const NormBwdArgs& a, RowPlan p, int blocks, hipStream_t s) {
#define NORM_CASE(W, U) if (p.waves == W && p.units == U) { \
        norm_bwd_kernel<T, W, U><<<blocks + a.col_blocks, W == 1 ? 256 : W * 64, 0, s>>>(a); return; }
    NORM_CASE(1, 1) NORM_CASE(4, 1) NORM_CASE(4, 2) NORM_CASE(16, 1) NORM_CASE(16, 2) NORM_CASE(16, 4)
#undef NORM_CASE
}

// Workgroups of the backward kernel.  Each leaves M floats of partial sums, which the second launch reads, so there are only as many
// as fill the chip, and half of that where wide rows are fewer (bfloat16, half / all: 1024 rows of 2048 10.4 / 12.7 us, of 8192
// 20 / 26; 4096 of 8192 56 / 61; 32768 of 2048 108 / 104; 4096 of 768, where 96 of 256 threads have columns: 13.7 / 12.7).
int norm_bwd_blocks(int T, int M, RowPlan p) {
    const int rows = p.waves == 1 ? 4 : 1;
    const int want = T / rows + (T % rows != 0), fill = p.waves == 16 ? 512 : 1024, most = M > 1024 && T < 8192 ? fill / 2 : fill;
    return want < most ? want : most;
}

// Rows up to which the gain's gradient has workgroups of its own in the same launch, which read dy and h once more, from the caches
// (so / with sums by the rows' workgroups and a second launch: 32 rows of 2048 in bfloat16 2.8 / 5.3 us, 256 3.1 / 7.7, 512 6.3 /
// 8.9, 1024 10.0 / 10.3, 2048 17 / 13; float, 512 8.4 / 10, 1024 14.4 / 13.1).
constexpr int GAIN_TOGETHER = 512;

}  // namespace

}  // namespace moe

extern "C" moe_status moe_norm_fwd(const moe_norm_config* cfg, const void* x, const void* residual, const float* gain,
                                   void* h, void* y, float* scales, float* rstd, void* stream) {
    moe::NormDims d;
    MOE_TRY(moe::norm_dims(cfg, &d));
    if (d.T == 0) return MOE_OK;
    if (!x || !y || (cfg->out == MOE_E4M3 && !scales)) return MOE_ERR_NULL;
    moe::NormArgs a = {x, residual, gain, h, y, scales, rstd, d.ldx, d.ldr, d.ldh, d.ldy, 0, d.T, d.M, cfg->group, d.n_scales, cfg->eps};
    const moe::RowPlan p = moe::norm_plan(d.M);
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_NORM, s);
        if (cfg->dtype == MOE_F32) {
            if (cfg->out == MOE_E4M3) moe::norm_launch<float, true>(a, p, s); else moe::norm_launch<float, false>(a, p, s);
        } else {
            if (cfg->out == MOE_E4M3) moe::norm_launch<moe::bf16_t, true>(a, p, s); else moe::norm_launch<moe::bf16_t, false>(a, p, s);
        }
    }
    MOE_CHECK_LAUNCH();
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

extern "C" moe_status moe_norm_scratch_bytes(const moe_norm_config* cfg, size_t* bytes) {
    moe::NormDims d;
    MOE_TRY(moe::norm_dims(cfg, &d));
    if (!bytes) return MOE_ERR_NULL;
    const int blocks = moe::norm_bwd_blocks(d.T, d.M, moe::norm_bwd_plan(d.M));
    *bytes = blocks > 1 ? (size_t)blocks * d.M * sizeof(float) : 0;
    return MOE_OK;
}

extern "C" moe_status moe_norm_bwd(const moe_norm_config* cfg, const void* dy, const void* h, const float* gain, const float* rstd,
                                   const void* dh, void* dx, float* dgain, void* scratch, void* stream) {
    moe::NormDims d;
    MOE_TRY(moe::norm_dims(cfg, &d));
    if (cfg->out == MOE_E4M3) return MOE_ERR_UNSUPPORTED;      // gradients of rounded rows are not defined here
    const moe::RowPlan p = moe::norm_bwd_plan(d.M);
    const int blocks = moe::norm_bwd_blocks(d.T, d.M, p);
    if (d.T > 0 && (!dy || !h || !rstd || !dx)) return MOE_ERR_NULL;
    if (dgain && blocks > 1 && !scratch) return MOE_ERR_NULL;
    hipStream_t s = (hipStream_t)stream;
    const int add = !cfg->grad_overwrite;
    // (rows that are overwritten are not there any more for other workgroups)
    const bool together = dgain && blocks > 1 && d.T <= moe::GAIN_TOGETHER && dx != dy;
    if (d.T == 0 && (!dgain || add)) return MOE_OK;
    {
        moe::ProfScope prof(moe::PK_NORM_BWD, s);
        if (d.T > 0) {
            const bool direct = blocks == 1;
            moe::NormBwdArgs a = {dy, h, gain, rstd, dh, dx, dgain && !together ? (direct ? dgain : (float*)scratch) : nullptr, dgain,
                                  d.ldx, d.ldh, d.ldy, d.T, d.M, (direct || together) && add,
                                  together ? (d.M + 8 * moe::GAIN_UNITS - 1) / (8 * moe::GAIN_UNITS) : 0};
            if (cfg->dtype == MOE_F32) moe::norm_bwd_launch<float>(a, p, blocks, s); else moe::norm_bwd_launch<moe::bf16_t>(a, p, blocks, s);
            MOE_CHECK_LAUNCH();
        }
        if (dgain && blocks != 1 && !together) {
            moe::norm_dgain_kernel<<<(d.M + moe::DG_COLS - 1) / moe::DG_COLS, moe::DG_COLS * moe::DG_SPLIT, 0, s>>>(
                (const float*)scratch, blocks, d.M, add, dgain);
            MOE_CHECK_LAUNCH();
        }
    }
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}
