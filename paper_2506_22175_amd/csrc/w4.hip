// Products of routed rows with their experts' 4-bit weights, and the packing of such weights.
//
//   y[t,j,n] = f(sum over c of x_row[c] W[e][n,c]) w[t,j],  e = topk_idx[t,j];  or y[t,n] = their sum over j
//   W[e][n,c] = e2m1 value of 4 bits * 2^(Ws - 127) of 32 columns
//
// Few rows meet each expert's matrix, so what has to move is the matrix: K N (1/2 + 1/32) bytes for every expert that is
// chosen, read once.  A wavefront multiplies 16 weight rows of 128 columns at a time: lane (r, q) holds 32 consecutive
// columns of weight row r, 16 bytes and one scale, which is what the matrix instructions take (they get
// there through LDS: Block16 says why).  The weights are the left operand and the routed rows, padded to
// 16, the right one: an output's lanes then hold four neighbouring columns of one row.
//   bfloat16 rows  the weights become bfloat16 (exact: the scale is a power of two) eight to an instruction of 16 x 16 x 32
//   float rows     the same with each float cut into three bfloat16 parts, whose sum it is: every product is exact (what of a
//                  value lies below 2^-133, the least bfloat16, is cut off)
//   e4m3 rows      become bfloat16 as well (exact), and 128 columns' sum is multiplied by the rows' scale.  The 16 x 16 x 128
//                  instruction that takes 4-bit and 8-bit operands as they are would save all the conversions, but among each
//                  eight neighbouring products it drops what lies some 2^14 below the largest (measured: sums up to 2^-14 of
//                  their largest term off, where the bfloat16 instruction is exact), and sums are to be those of float.
// The workgroup's wavefronts share out K and add up their sums in their order.
#include "common.h"
#include "wide.h"
#include <climits>
#include <cmath>

namespace moe {

namespace {

typedef __bf16 bf16x8_hw __attribute__((ext_vector_type(8)));
typedef float f32x4_hw __attribute__((ext_vector_type(4)));

struct W4Args {
    const void* x; const float* x_scales; const int* idx; const float* w; const uint8_t* Wq; const uint8_t* Ws;
    void* y;
    const int* list; const int* begins;      // of many assignments: w4_list_kernel's, else NULL
    long long ldx, ldy;
    int n_rows;                      // T * k assignments
    int k, E, K, N, n_scales, per_choice, gelu, out_f32;
};

__host__ __device__ constexpr int row_bytes(int xt, int cols) { return xt == MOE_F32 ? 4 * cols : xt == MOE_BF16 ? 2 * cols : cols; }
__host__ __device__ constexpr int row_parts(int xt) { return xt == MOE_F32 ? 3 : 1; }

// Eight columns of a routed row as the matrix instructions take them: PARTS times eight bfloat16.
template <int XT> struct Rows8;
template <> struct Rows8<MOE_BF16> {
    uint4 u;
    __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const char* p) { u = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void parts(uint4* o) const { o[0] = u; }
};
template <> struct Rows8<MOE_E4M3> {
    uint2 u;
    __device__ __forceinline__ void zero() { u = make_uint2(0, 0); }
    __device__ __forceinline__ void load(const char* p) { u = *reinterpret_cast<const uint2*>(p); }
    __device__ __forceinline__ void parts(uint4* o) const {
        o[0].x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.x, 1.0f, false));
        o[0].y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.x, 1.0f, true));
        o[0].z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.y, 1.0f, false));
        o[0].w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.y, 1.0f, true));
    }
};
template <> struct Rows8<MOE_F32> {
    float4 u[2];
    __device__ __forceinline__ void zero() { u[0] = u[1] = make_float4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const char* p) {
        u[0] = reinterpret_cast<const float4*>(p)[0];
        u[1] = reinterpret_cast<const float4*>(p)[1];
    }
    // Cut, not rounded: 8 + 8 + 8 bits of mantissa, exact, and no part is larger than the whole.  Infinities and NaN have
    // one part.
    __device__ __forceinline__ void parts(uint4* o) const {
        unsigned hi[4], mid[4], lo[4];
        const float v[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w};
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
        o[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        o[1] = make_uint4(mid[0], mid[1], mid[2], mid[3]);
        o[2] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
};

// Eight columns of the 4-bit weights in `w` as bfloat16: exact, the scale is a power of two.
__device__ __forceinline__ bf16x8_hw decode_weights(unsigned w, unsigned scale_byte) {
    const float scale = __uint_as_float(scale_byte << 23);
    uint4 d;
    d.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    d.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    d.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    d.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    return __builtin_bit_cast(bf16x8_hw, d);
}
__device__ __forceinline__ unsigned word_of(const uint4& u, int i) { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; }

// 16 weight rows of TILES tiles of 128 columns on their way to a wavefront's registers.
//
// The matrix instructions want the four lanes of a row 16 lanes apart, but the unit that takes requests apart needs a cycle for
// each 64 bytes of neighbouring lanes: loaded as they are wanted, every lane's 16 bytes were a cycle of their own, and that
// unit the limit (16 experts of 2048 x 8192, a row each: 39 us).  So neighbouring lanes load neighbouring pieces of a row
// and the rows change lanes through LDS that the wavefront has for itself; piece p of row r goes to place p ^ (r TILES / 4) of its
// row, so that the 16 rows' pieces, which are read at a time, are in different banks.
template <int TILES> struct Block16 {
    static constexpr int PIECES = 4 * TILES, ROWS = 64 / PIECES;           // of a row; rows of a request
    static constexpr int SLOTS = 64 * TILES;                               // of 16 bytes in LDS
    uint4 u[TILES];
    unsigned mask;                   // of the columns that are there; what is loaded is not looked at before put()
    static __device__ __forceinline__ int slot(int row, int piece) { return row * PIECES + (piece ^ (row * PIECES / 16)); }
    // Offsets in an expert's weights of the rows that the lane loads from; rows past the last are the last again, their products
    // of no use.
    static __device__ __forceinline__ void offsets(int n0, int N, int K, int lane, unsigned* o) {
#pragma unroll
        for (int j = 0; j < TILES; ++j) {
            const int n = n0 + j * ROWS + lane / PIECES;
            o[j] = (unsigned)(n < N ? n : N - 1) * (unsigned)(K / 2);
        }
    }
    // From the first column of `tile` on.  Columns past the last are zeros: loaded from the row's beginning, so that nothing branches.
    __device__ __forceinline__ void load(const uint8_t* Wq, const unsigned* o, int tile, int lane, int K) {
        const bool there = tile * 128 + lane % PIECES * 32 < K;
        const unsigned at = there ? tile * 64 + lane % PIECES * 16 : 0;
        mask = there ? ~0u : 0u;
#pragma unroll
        for (int j = 0; j < TILES; ++j) u[j] = *reinterpret_cast<const uint4*>(Wq + (o[j] + at));
    }
    __device__ __forceinline__ void put(uint4* lds, int lane) const {
#pragma unroll
        for (int j = 0; j < TILES; ++j)
            lds[slot(j * ROWS + lane / PIECES, lane % PIECES)] = make_uint4(u[j].x & mask, u[j].y & mask, u[j].z & mask, u[j].w & mask);
    }
    // columns 32 q .. + 31 of row r in tile t
    static __device__ __forceinline__ uint4 get(const uint4* lds, int t, int r, int q) { return lds[slot(r, t * 4 + q)]; }
};

// What a wavefront writes to LDS and reads from there stays in this order; nothing is waited for.
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The scales of a tile of a weight row, a byte for each 32 columns; 1 where there are no columns.  Four bytes of the row that has
// them are loaded, those before the row's end where the tile is not full (K < 128: byte by byte).
struct Scales {
    unsigned u;
    int past;                        // bytes of u that belong to the tile before; 4 and more: none is this tile's
    __device__ __forceinline__ void load(const uint8_t* Ws, int tile, int K) {
        const int blocks = K / 32, first = tile * 4, at = first + 4 <= blocks ? first : blocks - 4;
        past = first - at;
        if (blocks >= 4) {
            u = reinterpret_cast<const Anywhere<4, 1>*>(Ws + at)->w[0];
        } else {
            u = 0x7f7f7f7f;
            past = 0;
            if (first < blocks) u = (u & ~0xffu) | Ws[first];
            if (first + 1 < blocks) u = (u & ~0xff00u) | (unsigned)Ws[first + 1] << 8;
            if (first + 2 < blocks) u = (u & ~0xff0000u) | (unsigned)Ws[first + 2] << 16;
        }
    }
    __device__ __forceinline__ unsigned get() const {
        return past == 0 ? u : past >= 4 ? 0x7f7f7f7fu : u >> (8 * past) | 0x7f7f7f7fu << (32 - 8 * past);
    }
};
// The scales of 64 weight rows in 16 tiles, 64 bytes of each, through the wavefront's LDS as well: four bytes of 64 rows at a time
// would cost as many cycles as the 4 KiB of weights that they belong to (16 experts of 2048 x 8192, a row each: 42 us, and 32
// without any scales).
constexpr int SCALE_TILES = 16, SCALE_SLOTS = 256;
__device__ __forceinline__ int scale_slot(int row, int piece) { return row * 4 + (piece ^ (row / 4 & 3)); }
__device__ __forceinline__ void fetch_scales(const uint8_t* Ws, int n0, int N, int K, int tile, int lane, uint4* lds) {
    const int bytes = K / 32, at = tile * 4 + lane % 4 * 16;
    uint4 u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + j * 16 + lane / 4;
        const uint8_t* row = Ws + (long long)(n < N ? n : N - 1) * bytes;
        if (at + 16 <= bytes) {
            const auto v = *reinterpret_cast<const Anywhere<16, 1>*>(row + at);
            u[j] = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
        } else if (at >= bytes) {
            u[j] = make_uint4(0x7f7f7f7f, 0x7f7f7f7f, 0x7f7f7f7f, 0x7f7f7f7f);
        } else {
            // the row's last words, the last one's bytes one by one, 1 behind them
            unsigned w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int first = at + 4 * i;
                w[i] = 0x7f7f7f7f;
                if (first + 4 <= bytes) {
                    w[i] = reinterpret_cast<const Anywhere<4, 1>*>(row + first)->w[0];
                } else if (first < bytes) {
#pragma unroll
                    for (int b = 0; b < 3; ++b)
                        if (first + b < bytes) w[i] = (w[i] & ~(0xffu << (8 * b))) | (unsigned)row[first + b] << (8 * b);
                }
            }
            u[j] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) lds[scale_slot(j * 16 + lane / 4, lane % 4)] = u[j];
}
// of columns 32 q .. + 31 of a row's tile
__device__ __forceinline__ unsigned scale_at(const uint4* lds, int row, int tile, int q) {
    tile %= SCALE_TILES;
    return reinterpret_cast<const uint8_t*>(lds + scale_slot(row, tile / 4))[tile % 4 * 4 + q];
}

__device__ __forceinline__ unsigned from_any_lane(unsigned v, int lane) { return (unsigned)__builtin_amdgcn_ds_bpermute(lane * 4, (int)v); }

__device__ __forceinline__ float w4_finish(float v, int gelu, float weight) {
    if (gelu) v = v * (0.5f + 0.5f * erff(v * 0.70710678118654752440f));
    return v * weight;
}
__device__ __forceinline__ void w4_store(const W4Args& a, long long row, int n, const float* v) {
    if (a.out_f32) store_columns(reinterpret_cast<float*>(a.y) + row * a.ldy + n, v, a.N - n);
    else store_columns(reinterpret_cast<bf16_t*>(a.y) + row * a.ldy + n, v, a.N - n);
}

// ---- tokens by themselves ---------------------------------------------------------------------------------
// A workgroup has 16 weight rows of one choice of a token (SUM: of all its choices, and adds them up), its wavefronts share out
// the choices and K in pieces of 512 columns.  A piece of the routed row is one request of the wavefront and goes through LDS
// that no other wavefront uses, from where all 16 columns of the right operand get the same.  Bound by the way to the first
// weights: 2 experts of 2048 x 8192 6.4 us (17.8 MB, 2.8 TB/s), 8 of them (4 tokens) 14.2 us (5 TB/s).
constexpr int TOKEN_TILES = 4;       // of a piece
constexpr int TOKEN_WAVES = 16;      // at most; four where that is enough, so that LDS has room for more workgroups

template <int XT> struct TokenPiece {
    Block16<TOKEN_TILES> w;
    Scales s;                        // lane l: the scales of weight row l / 4 in tile l % 4
    Rows8<XT> x;
    bool there;                      // x is not past the row's end
    float xs[TOKEN_TILES];
    // row: of the assignment; xs_row: its scales
    __device__ __forceinline__ void load(const uint8_t* Wq, const unsigned* offset, const uint8_t* Ws, const char* row, const float* xs_row,
                                         int n_scales, int tile, int K) {
        const int lane = threadIdx.x & 63, col = tile * 128 + lane * 8;
        w.load(Wq, offset, tile, lane, K);
        s.load(Ws, tile + lane % 4, K);
        x.load(row + row_bytes(XT, col < K ? col : 0));
        there = col < K;
        if constexpr (XT == MOE_E4M3) {
#pragma unroll
            for (int t = 0; t < TOKEN_TILES; ++t) xs[t] = (tile + t) * 128 < K ? xs_row[n_scales > 1 ? tile + t : 0] : 0.0f;
        }
    }
};

template <int XT, bool SUM, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void w4_token_kernel(W4Args a, int slices) {
    constexpr int PARTS = row_parts(XT);
    __shared__ uint4 s_w[WAVES][Block16<TOKEN_TILES>::SLOTS], s_x[WAVES][PARTS][64];
    __shared__ float4 s_sum[WAVES][4];
    const int tid = threadIdx.x, wid = tid >> 6, lane = tid & 63, r = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const long long token = blockIdx.z;
    const int* idx = a.idx ? a.idx + token * a.k : nullptr;
    const float* weights = a.w ? a.w + token * a.k : nullptr;
    unsigned offset[TOKEN_TILES];
    Block16<TOKEN_TILES>::offsets(n0, a.N, a.K, lane, offset);
    const int scale_row = n0 + lane / 4 < a.N ? n0 + lane / 4 : a.N - 1;
    const int pieces = (a.K + 128 * TOKEN_TILES - 1) / (128 * TOKEN_TILES), waves = blockDim.x >> 6;
    // the wavefront's choices: one, or (SUM, more choices than wavefronts) every `waves`-th
    const int first = SUM ? wid / slices : (int)blockIdx.y, slice = SUM ? wid % slices : wid, step = waves / slices;
    float4 sum = make_float4(0, 0, 0, 0);                 // SUM and slices = 1: of the wavefront's choices, weighted
    for (int j = first; j < a.k; j += step) {
        const int e = idx ? idx[j] : 0;
        f32x4_hw acc = {0, 0, 0, 0};
        if ((unsigned)e < (unsigned)a.E) {
            const long long xr = a.per_choice ? token * a.k + j : token;
            const uint8_t* Wq = a.Wq + (long long)e * a.N * (a.K / 2);
            const uint8_t* Ws = a.Ws + ((long long)e * a.N + scale_row) * (a.K / 32);
            const char* row = reinterpret_cast<const char*>(a.x) + xr * row_bytes(XT, 1) * a.ldx;
            const float* xs_row = a.x_scales + xr * a.n_scales;
            TokenPiece<XT> v;
            if (slice < pieces) v.load(Wq, offset, Ws, row, xs_row, a.n_scales, slice * TOKEN_TILES, a.K);
            for (int piece = slice; piece < pieces; piece += slices) {
                uint4 p[PARTS];
                v.x.parts(p);
#pragma unroll
                for (int c = 0; c < PARTS; ++c) s_x[wid][c][lane] = v.there ? p[c] : make_uint4(0, 0, 0, 0);
                v.w.put(s_w[wid], lane);
                wave_order();
                const unsigned scales = v.s.get();
                float xs[TOKEN_TILES];
                if constexpr (XT == MOE_E4M3) {
#pragma unroll
                    for (int t = 0; t < TOKEN_TILES; ++t) xs[t] = v.xs[t];
                }
                if (piece + slices < pieces) v.load(Wq, offset, Ws, row, xs_row, a.n_scales, (piece + slices) * TOKEN_TILES, a.K);
#pragma unroll
                for (int t = 0; t < TOKEN_TILES; ++t) {
                    const uint4 w = Block16<TOKEN_TILES>::get(s_w[wid], t, r, q);
                    const unsigned scale = from_any_lane(scales, r * 4 + t) >> (8 * q) & 0xffu;
                    f32x4_hw part = XT == MOE_E4M3 ? f32x4_hw{0, 0, 0, 0} : acc;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bf16x8_hw d = decode_weights(word_of(w, i), scale);
#pragma unroll
                        for (int c = PARTS - 1; c >= 0; --c)
                            part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                d, __builtin_bit_cast(bf16x8_hw, s_x[wid][c][t * 16 + q * 4 + i]), part, 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i] = XT == MOE_E4M3 ? fmaf(xs[t], part[i], acc[i]) : part[i];
                }
                wave_order();
            }
        }
        if (SUM && slices == 1) {
            const float weight = weights ? weights[j] : 1.0f;
            if ((unsigned)e < (unsigned)a.E) {
                sum.x += w4_finish(acc[0], a.gelu, weight); sum.y += w4_finish(acc[1], a.gelu, weight);
                sum.z += w4_finish(acc[2], a.gelu, weight); sum.w += w4_finish(acc[3], a.gelu, weight);
            }
        } else {
            sum = make_float4(acc[0], acc[1], acc[2], acc[3]);
            break;
        }
    }
    // every column has the row's sums
    if (r == 0) s_sum[wid][q] = sum;
    const int tq = tid & 3;                                // thread q < 4 will have columns n0 + 4 q .. + 3
    const float weight = !SUM && weights ? weights[first] : 1.0f;
    __syncthreads();
    if (tid >= 4) return;
    float v[4] = {0, 0, 0, 0};
    if (!SUM || slices == 1) {
        for (int w = 0; w < waves; ++w) {
            const float4 p = s_sum[w][tq];
            v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
        }
        if (!SUM) {
            // (an expert out of range has sums of zero, and GeLU keeps them)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = w4_finish(v[i], a.gelu, weight);
            const int e = idx ? idx[first] : 0;
            if ((unsigned)e >= (unsigned)a.E) v[0] = v[1] = v[2] = v[3] = 0.0f;      // whatever its weight
        }
    } else {
        for (int j = 0; j < a.k; ++j) {
            const int e = idx ? idx[j] : 0;
            if ((unsigned)e >= (unsigned)a.E) continue;
            const float wj = weights ? weights[j] : 1.0f;
            float c[4] = {0, 0, 0, 0};
            for (int w = 0; w < slices; ++w) {
                const float4 p = s_sum[j * slices + w][tq];
                c[0] += p.x; c[1] += p.y; c[2] += p.z; c[3] += p.w;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += w4_finish(c[i], a.gelu, wj);
        }
    }
    if (n0 + 4 * tq < a.N) w4_store(a, SUM ? token : token * a.k + first, n0 + 4 * tq, v);
}

// ---- several tokens ----------------------------------------------------------------------------
constexpr int W4_WAVES = 8;

// Rows of assignments with expert e (e < 0: with none of the experts), number `from` to from + cap - 1 of them, into `list`;
// returns how many there are in all.  Every thread of the workgroup calls it.  Each wavefront counts its share of the
// assignments, and goes through it again when it knows where its numbers begin.
template <int WAVES> __device__ int collect_rows(const int* idx, int n, int e, int E, int from, int cap, int* list, int* s_count) {
    constexpr int AT_ONCE = 4;                             // requests of a wavefront under way
    const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int share = (n + WAVES * 64 - 1) / (WAVES * 64) * 64, begin = wid * share, end = begin + share < n ? begin + share : n;
    int rank = 0;
    for (int pass = 0; pass < 2; ++pass) {
        for (int base = begin; base < end; base += AT_ONCE * 64) {
            int v[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int i = base + u * 64 + lane;
                v[u] = idx[i < end ? i : end - 1];
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int i = base + u * 64 + lane;
                const bool mine = i < end && (e < 0 ? (unsigned)v[u] >= (unsigned)E : v[u] == e);
                const unsigned long long b = __ballot(mine);
                const int at = rank + __popcll(b & ((1ull << lane) - 1));
                if (pass == 1 && mine && at >= from && at < from + cap) list[at - from] = i;
                rank += __popcll(b);
            }
        }
        if (pass == 0) {
            if (lane == 0) s_count[wid] = rank;
            __syncthreads();
            rank = 0;
            for (int w = 0; w < wid; ++w) rank += s_count[w];
        }
    }
    int total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total += s_count[w];
    __syncthreads();
    return total;
}

// Assignments in the order of their experts: list[begins[e] .. begins[e + 1] - 1] have expert e, ascending; behind the last
// expert's those with none.  A workgroup has an expert, counts its assignments and those of the experts before it, and goes
// through all of them again to write its own down: two readings for each expert, whatever the product's grid.
constexpr int LIST_WAVES = 16;
__global__ __launch_bounds__(LIST_WAVES * 64) void w4_list_kernel(const int* __restrict__ idx, int n, int E, int* __restrict__ begins,
                                                                  int* __restrict__ list) {
    constexpr int AT_ONCE = 8;                             // requests of a wavefront under way
    __shared__ int s_mine[LIST_WAVES], s_before[LIST_WAVES];
    const int e = blockIdx.x, wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int share = (n + LIST_WAVES * 64 - 1) / (LIST_WAVES * 64) * 64, begin = wid * share, end = begin + share < n ? begin + share : n;
    int at = 0, before = 0;
    for (int pass = 0; pass < 2; ++pass) {
        for (int base = begin; base < end; base += AT_ONCE * 64) {
            int v[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int i = base + u * 64 + lane;
                v[u] = idx[i < end ? i : end - 1];
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int i = base + u * 64 + lane;
                const bool mine = i < end && (e < E ? v[u] == e : (unsigned)v[u] >= (unsigned)E);
                const unsigned long long b = __ballot(mine);
                if (pass == 1 && mine) list[at + __popcll(b & ((1ull << lane) - 1))] = i;
                at += __popcll(b);
                if (pass == 0) before += __popcll(__ballot(i < end && (unsigned)v[u] < (unsigned)e));
            }
        }
        if (pass == 0) {
            if (lane == 0) { s_mine[wid] = at; s_before[wid] = before; }
            __syncthreads();
            at = 0;
#pragma unroll
            for (int w = 0; w < LIST_WAVES; ++w) at += s_before[w] + (w < wid ? s_mine[w] : 0);
            if (threadIdx.x == 0) {
                begins[e] = at;
                if (e == E) begins[E + 1] = n;
            }
        }
    }
}

// The rows of a workgroup's expert (e < 0: of none) from number `from` on, up to CAP, into `s_list`; returns how many there are in
// all.  Every thread of the workgroup calls it.
template <int WAVES, int CAP> __device__ __forceinline__ int find_rows(const W4Args& a, int e, int from, int* s_list, int* s_count) {
    static_assert(CAP <= WAVES * 64, "a thread to a row");
    if (a.idx && !a.list) return collect_rows<WAVES>(a.idx, a.n_rows, e, a.E, from, CAP, s_list, s_count);
    int first = 0, total = a.n_rows;
    if (a.list) {
        const int slot = e < 0 ? a.E : e;
        first = a.begins[slot];
        total = a.begins[slot + 1] - first;
    }
    if ((int)threadIdx.x < CAP && from + (int)threadIdx.x < total) {
        const int at = first + from + (int)threadIdx.x;
        s_list[threadIdx.x] = a.list ? a.list[at] : at;
    }
    __syncthreads();
    return total;
}

// Few rows to an expert (up to 16 RT at a time): a wavefront has 64 weight rows and a share of K, which it streams by itself; `shares` of the
// workgroup's wavefronts have the same weight rows and add up their sums at the end.  The routed rows come straight from the L2
// cache, once for 64 weight rows.  There is no barrier on the way, and the next tile's requests are out while one is
// multiplied.  shares is such that there are some eight wavefronts to a compute unit in all: each of them pays the way to its
// first weights (its rows' numbers, their addresses, the first request), and experts with more rows take longer.  Bound by the
// weights' bytes where loads are even: 37 tokens, 4 of 64 experts of 1024 x 4093, e4m3 rows 28 us, 4.7 TB/s; by the experts with most
// rows where they are not: 64 tokens, 2 of 16 experts of 8192 x 2048 with up to 29 rows 38 us, 3.7 TB/s.
constexpr int FEW_WAVES = 4, FEW_MORE = 8;       // of a workgroup; more where K has to be cut finer to fill the chip

// A tile of 16 routed rows: as stored, in pieces of 16 bytes, neighbouring lanes with neighbouring pieces.  Through LDS to the lanes
// that want them as the weights.
template <int XT> struct RowTile {
    static constexpr int PIECES = row_bytes(XT, 128) / 16, ROWS = 64 / PIECES, LOADS = 16 / ROWS;
    static constexpr int SLOTS = 16 * PIECES;
    uint4 u[LOADS];
    unsigned mask;                   // as Block16's
    static __device__ __forceinline__ int slot(int row, int piece) { return row * PIECES + (piece ^ (row % PIECES)); }
    // row[j]: the offset in x of the lane's row of load j; loads of nothing but rows past `here` are left out
    __device__ __forceinline__ void load(const char* x, const unsigned* row, int here, int tile, int lane, int K) {
        const unsigned col = tile * 128 + lane % PIECES * (16 / row_bytes(XT, 1));
        const bool there = col < (unsigned)K;
        const unsigned at = there ? row_bytes(XT, 1) * col : 0;
        mask = there ? ~0u : 0u;
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
            if (j == 0 || j * ROWS < here) u[j] = *reinterpret_cast<const uint4*>(x + (row[j] + at));
    }
    __device__ __forceinline__ void put(uint4* lds, int lane) const {
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
            lds[slot(j * ROWS + lane / PIECES, lane % PIECES)] = make_uint4(u[j].x & mask, u[j].y & mask, u[j].z & mask, u[j].w & mask);
    }
    // columns 32 q + 8 i .. + 7 of row r
    static __device__ __forceinline__ Rows8<XT> get(const uint4* lds, int r, int q, int i) {
        Rows8<XT> x;
        if constexpr (XT == MOE_BF16) {
            x.u = lds[slot(r, q * 4 + i)];
        } else if constexpr (XT == MOE_F32) {
            x.u[0] = __builtin_bit_cast(float4, lds[slot(r, q * 8 + 2 * i)]);
            x.u[1] = __builtin_bit_cast(float4, lds[slot(r, q * 8 + 2 * i + 1)]);
        } else {
            x.u = reinterpret_cast<const uint2*>(&lds[slot(r, q * 2 + i / 2)])[i % 2];
        }
        return x;
    }
};

// A wavefront's share: tiles begin .. end - 1.
struct FewShare { const uint8_t* Wq; const uint8_t* Ws; int n0, begin, end; };

// The sums of 4 x 16 weight rows with the first `here` rows of the list.
template <int XT, int RT>
__device__ __forceinline__ void few_stream(const W4Args& a, const FewShare& f, const int* s_list, int here, uint4* s_w, uint4* s_x, uint4* s_s, f32x4_hw (*acc)[RT]) {
    typedef RowTile<XT> X;
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    unsigned offset[4][1];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        Block16<1>::offsets(f.n0 + t * 16, a.N, a.K, lane, offset[t]);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[t][rt] = f32x4_hw{0, 0, 0, 0};
    }
    // of the lane's row in each load; and the scales of row r
    const char* const x = reinterpret_cast<const char*>(a.x);
    unsigned row[RT][X::LOADS], xs_row[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int j = 0; j < X::LOADS; ++j) {
            const int i = rt * 16 + j * X::ROWS + lane / X::PIECES, at = s_list[i < here ? i : 0];
            row[rt][j] = (unsigned)(a.per_choice ? at : at / a.k) * (unsigned)row_bytes(XT, 1) * (unsigned)a.ldx;
        }
        const int at = s_list[rt * 16 + r < here ? rt * 16 + r : 0];
        xs_row[rt] = (unsigned)(a.per_choice ? at : at / a.k) * (unsigned)a.n_scales;
    }
    struct Next {                                                          // a tile on its way
        Block16<1> w[4];
        X x[RT];
        float xs[RT];
    };
    float xs[RT];
    auto request = [&](Next& v, int tile) {
#pragma unroll
        for (int t = 0; t < 4; ++t) v.w[t].load(f.Wq, offset[t], tile, lane, a.K);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            v.x[rt].load(x, row[rt], here - rt * 16, tile, lane, a.K);
            if (XT == MOE_E4M3) v.xs[rt] = a.x_scales[xs_row[rt] + (a.n_scales > 1 ? tile : 0)];
        }
    };
    auto put = [&](const Next& v) {
#pragma unroll
        for (int t = 0; t < 4; ++t) v.w[t].put(s_w + t * Block16<1>::SLOTS, lane);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            v.x[rt].put(s_x + rt * X::SLOTS, lane);
            if (XT == MOE_E4M3) xs[rt] = v.xs[rt];
        }
        wave_order();
    };
    auto multiply = [&](int tile) {                                        // which is in LDS
        f32x4_hw part[4][RT];
        uint4 w[4];
        unsigned s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) part[t][rt] = XT == MOE_E4M3 ? f32x4_hw{0, 0, 0, 0} : acc[t][rt];
            w[t] = Block16<1>::get(s_w + t * Block16<1>::SLOTS, 0, r, q);
            s[t] = scale_at(s_s, t * 16 + r, tile - f.begin, q);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint4 p[RT][row_parts(XT)];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) X::get(s_x + rt * X::SLOTS, r, q, i).parts(p[rt]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const bf16x8_hw d = decode_weights(word_of(w[t], i), s[t]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int c = row_parts(XT) - 1; c >= 0; --c)
                        part[t][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(d, __builtin_bit_cast(bf16x8_hw, p[rt][c]), part[t][rt], 0, 0, 0);
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[t][rt][j] = XT == MOE_E4M3 ? fmaf(xs[rt], part[t][rt][j], acc[t][rt][j]) : part[t][rt][j];
        wave_order();
    };
    // A tile goes to LDS, the next one's requests go out, and then it is multiplied (the barriers keep the compiler from moving
    // the requests behind that).  Behind the last one it is requested again, and not multiplied.
    if (f.begin >= f.end) return;
    Next v;
    request(v, f.begin);
    for (int tile = f.begin; tile < f.end; ++tile) {
        if ((tile - f.begin) % SCALE_TILES == 0) fetch_scales(f.Ws, f.n0, a.N, a.K, tile, lane, s_s);
        put(v);
        request(v, tile + 1 < f.end ? tile + 1 : tile);
        __builtin_amdgcn_sched_barrier(0);
        multiply(tile);
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int XT, int RT, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void w4_few_kernel(W4Args a, int shares) {
    constexpr int CAP = 16 * RT, W_SLOTS = 4 * Block16<1>::SLOTS, X_SLOTS = RowTile<XT>::SLOTS;
    __shared__ uint4 s_own[WAVES][W_SLOTS + RT * X_SLOTS], s_scales[WAVES][SCALE_SLOTS];    // a wavefront's tile, later its sums
    __shared__ int s_list[CAP], s_count[WAVES];
    static_assert(W_SLOTS + RT * X_SLOTS >= 4 * RT * 64, "4 RT sums of 64 lanes");
    const int tid = threadIdx.x, wid = tid >> 6, lane = tid & 63, r = lane & 15, q = lane >> 4;
    const int group = wid / shares, part_k = wid % shares, groups = WAVES / shares;
    const int n0 = (blockIdx.x * groups + group) * 64;
    int e = a.idx ? (int)blockIdx.y : 0;
    if (e >= a.E) e = -1;                                  // the rows of no expert, which are zeroed
    FewShare f;
    f.n0 = n0;
    const int tiles = (a.K + 127) / 128, share = (tiles + shares - 1) / shares;
    f.begin = part_k * share;
    f.end = f.begin + share < tiles ? f.begin + share : tiles;
    f.Wq = a.Wq + (long long)(e < 0 ? 0 : e) * a.N * (a.K / 2);
    f.Ws = a.Ws + (long long)(e < 0 ? 0 : e) * a.N * (a.K / 32);
    for (int from = blockIdx.z * CAP;; from += gridDim.z * CAP) {
        const int total = find_rows<WAVES, CAP>(a, e, from, s_list, s_count);
        if (total <= from) return;
        const int here = total - from < CAP ? total - from : CAP;
        float weight[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) weight[rt] = a.w ? a.w[s_list[rt * 16 + r < here ? rt * 16 + r : 0]] : 1.0f;
        f32x4_hw acc[4][RT];                               // of 16 weight rows and 16 routed rows each
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[t][rt] = f32x4_hw{0, 0, 0, 0};
        if (e >= 0 && n0 < a.N) {
            if (RT > 1 && here <= 16) {                    // half of the rows' requests and products
                f32x4_hw one[4][1];
                few_stream<XT, 1>(a, f, s_list, here, s_own[wid], s_own[wid] + W_SLOTS, s_scales[wid], one);
#pragma unroll
                for (int t = 0; t < 4; ++t) acc[t][0] = one[t][0];
            } else {
                few_stream<XT, RT>(a, f, s_list, here, s_own[wid], s_own[wid] + W_SLOTS, s_scales[wid], acc);
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                reinterpret_cast<float4*>(s_own[wid])[(t * RT + rt) * 64 + lane] = make_float4(acc[t][rt][0], acc[t][rt][1], acc[t][rt][2], acc[t][rt][3]);
        if (shares > 1) __syncthreads();
        else wave_order();
        // each wavefront finishes its share of its group's sums
        for (int c = part_k; c < 4 * RT; c += shares) {
            const int n = n0 + c / RT * 16 + q * 4, at = c % RT * 16 + r;
            if (at >= here || n >= a.N) continue;
            float v[4] = {0, 0, 0, 0};
            for (int w = group * shares; w < (group + 1) * shares; ++w) {
                const float4 p = reinterpret_cast<const float4*>(s_own[w])[c * 64 + lane];
                v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = e < 0 ? 0.0f : w4_finish(v[j], a.gelu, c % RT ? weight[RT - 1] : weight[0]);
            w4_store(a, s_list[at], n, v);
        }
        if (from + (int)gridDim.z * CAP >= total) return;
        __syncthreads();
    }
}

// How many tiles of 128 columns are staged at a time for each share of K, and shares of K where there are too few workgroups: as
// many as 16 RT rows leave room for.
template <int XT, int RT, int WK> constexpr int staged_tiles() { return row_parts(XT) * RT * WK <= 4 ? 2 : 1; }
template <int XT, int RT> constexpr int most_shares() { return row_parts(XT) * RT <= 6 ? 2 : 1; }

// A workgroup's eight wavefronts have 8 / WK tiles of 16 weight rows and WK shares of K.  The routed rows, RT tiles of 16, pass
// through LDS in the order in which the matrix instructions take them, converted on the way once for all wavefronts, while
// the weights of the next columns are on their way into registers.  512 tokens, 2 of 16 experts of 2048 x 8192: 101 us, 340 TFLOP/s,
// bound by the weights' conversion, which four tiles of rows share.
template <int XT, int RT, int WK>
__global__ __launch_bounds__(W4_WAVES * 64) void w4_rows_kernel(W4Args a) {
    constexpr int CAP = 16 * RT, PARTS = row_parts(XT), TILES = staged_tiles<XT, RT, WK>(), WN = W4_WAVES / WK;
    // 16 bytes of lane (r, q) for instruction i of a tile: slots padded so that neighbouring columns are not all in one bank
    constexpr int Q_SLOTS = 17, I_SLOTS = 4 * Q_SLOTS + 1, TILE_SLOTS = 4 * I_SLOTS;
    constexpr int STAGE = TILES * RT * PARTS * TILE_SLOTS;                    // of one share of K
    constexpr int UNITS = WK * CAP * TILES * 16, PER_THREAD = (UNITS + W4_WAVES * 64 - 1) / (W4_WAVES * 64);
    __shared__ uint4 s_x[2][WK * STAGE], s_w[W4_WAVES][Block16<TILES>::SLOTS];
    __shared__ float s_scale[2][XT == MOE_E4M3 ? WK * TILES * CAP : 1];
    __shared__ int s_list[CAP], s_count[W4_WAVES];
    static_assert(sizeof(s_x) >= (size_t)(WK > 1 ? W4_WAVES * RT * 64 * 16 : 0), "the joined sums need room");
    const int tid = threadIdx.x, wid = tid >> 6, lane = tid & 63, r = lane & 15, q = lane >> 4;
    const int part_k = wid / WN, n0 = (blockIdx.x * WN + wid % WN) * 16;
    int e = a.idx ? (int)blockIdx.y : 0;
    if (e >= a.E) e = -1;                                  // the rows of no expert, which are zeroed
    const uint8_t* Wq = a.Wq + (long long)(e < 0 ? 0 : e) * a.N * (a.K / 2);
    unsigned offset[TILES];
    Block16<TILES>::offsets(n0, a.N, a.K, lane, offset);
    // lane l has the scales of weight row l / TILES in tile l % TILES (of 16 rows: then they begin again)
    const int scale_row = n0 + lane / TILES % 16 < a.N ? n0 + lane / TILES % 16 : a.N - 1;
    const uint8_t* Ws = a.Ws + ((long long)(e < 0 ? 0 : e) * a.N + scale_row) * (a.K / 32);
    const int tiles = (a.K + 127) / 128, per_share = ((tiles + WK - 1) / WK + TILES - 1) / TILES * TILES;
    for (int from = blockIdx.z * CAP;; from += gridDim.z * CAP) {
        const int total = find_rows<W4_WAVES, CAP>(a, e, from, s_list, s_count);
        if (total <= from) return;
        const int here = total - from < CAP ? total - from : CAP;
        if (e < 0) {
            const float zero[4] = {0, 0, 0, 0};
            for (int i = tid; i < here * WN * 4; i += W4_WAVES * 64) {
                const int col = (blockIdx.x * WN * 4 + i % (WN * 4)) * 4;
                if (col < a.N) w4_store(a, s_list[i / (WN * 4)], col, zero);
            }
            __syncthreads();
            continue;
        }
        f32x4_hw acc[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt] = f32x4_hw{0, 0, 0, 0};
        // what this thread stages: unit u is eight columns of a row of a share of K
        const char* src[PER_THREAD];
        int dst[PER_THREAD], col0[PER_THREAD];
#pragma unroll
        for (int u = 0; u < PER_THREAD; ++u) {
            const int unit = u * W4_WAVES * 64 + tid, c8 = unit % (TILES * 16), row = unit / (TILES * 16) % CAP, share = unit / (TILES * 16 * CAP);
            src[u] = nullptr;
            col0[u] = share * per_share * 128 + c8 * 8;
            dst[u] = -1;
            if (UNITS % (W4_WAVES * 64) == 0 || unit < UNITS) {
                const int t = c8 / 16, sq = c8 % 16 / 4, i = c8 % 4;
                dst[u] = share * STAGE + ((t * RT + row / 16) * PARTS) * TILE_SLOTS + i * I_SLOTS + sq * Q_SLOTS + row % 16;
                if (row < here) {
                    const long long xr = a.per_choice ? s_list[row] : s_list[row] / a.k;
                    src[u] = reinterpret_cast<const char*>(a.x) + xr * row_bytes(XT, 1) * a.ldx;
                }
            }
        }
        Rows8<XT> staged[PER_THREAD];
        float scale = 0.0f;
        auto request = [&](int tile) {                     // tile: of a share, the first of those to be staged
#pragma unroll
            for (int u = 0; u < PER_THREAD; ++u) {
                staged[u].zero();
                const int col = col0[u] + tile * 128;
                if (src[u] && col < a.K) staged[u].load(src[u] + row_bytes(XT, col));
            }
            if (XT == MOE_E4M3 && tid < WK * TILES * CAP) {
                const int row = tid % CAP, t = tid / CAP % TILES, share = tid / (CAP * TILES), at = share * per_share + tile + t;
                scale = 0.0f;
                if (row < here && at < tiles) {
                    const long long xr = a.per_choice ? s_list[row] : s_list[row] / a.k;
                    scale = a.x_scales[xr * a.n_scales + (a.n_scales > 1 ? at : 0)];
                }
            }
        };
        auto put = [&](int buf) {
#pragma unroll
            for (int u = 0; u < PER_THREAD; ++u) {
                uint4 p[PARTS];
                staged[u].parts(p);
                if (dst[u] >= 0) {
#pragma unroll
                    for (int c = 0; c < PARTS; ++c) s_x[buf][dst[u] + c * TILE_SLOTS] = p[c];
                }
            }
            if (XT == MOE_E4M3 && tid < WK * TILES * CAP) s_scale[buf][tid] = scale;
        };
        Block16<TILES> w;
        Scales next;
        unsigned now;
        const int w_tile0 = part_k * per_share;
        auto request_weights = [&](int tile) {
            w.load(Wq, offset, tile, lane, a.K);
            next.load(Ws, tile + lane % TILES, a.K);
        };
        request_weights(w_tile0);
        request(0);
        put(0);
        __syncthreads();
        for (int tile = 0, buf = 0; tile < per_share; tile += TILES, buf ^= 1) {
            const bool more = tile + TILES < per_share;
            w.put(s_w[wid], lane);
            now = next.get();
            wave_order();
            if (more) {
                request_weights(w_tile0 + tile + TILES);
                request(tile + TILES);
            }
            __builtin_amdgcn_sched_barrier(0);
            const uint4* x = s_x[buf] + part_k * STAGE;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                f32x4_hw part[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) part[rt] = XT == MOE_E4M3 ? f32x4_hw{0, 0, 0, 0} : acc[rt];
                const uint4 wt = Block16<TILES>::get(s_w[wid], t, r, q);
                const unsigned st = from_any_lane(now, r * TILES + t) >> (8 * q) & 0xffu;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bf16x8_hw d = decode_weights(word_of(wt, i), st);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int c = PARTS - 1; c >= 0; --c)
                            part[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                d, __builtin_bit_cast(bf16x8_hw, x[((t * RT + rt) * PARTS + c) * TILE_SLOTS + i * I_SLOTS + q * Q_SLOTS + r]),
                                part[rt], 0, 0, 0);
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float xs = XT == MOE_E4M3 ? s_scale[buf][(part_k * TILES + t) * CAP + rt * 16 + r] : 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[rt][j] = XT == MOE_E4M3 ? fmaf(xs, part[rt][j], acc[rt][j]) : part[rt][j];
                }
            }
            wave_order();
            if (more) put(buf ^ 1);
            __syncthreads();
        }
        if constexpr (WK > 1) {
            // the shares' sums, in their order
            float4* s_sum = reinterpret_cast<float4*>(&s_x[0][0]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s_sum[(wid * RT + rt) * 64 + lane] = make_float4(acc[rt][0], acc[rt][1], acc[rt][2], acc[rt][3]);
            __syncthreads();
            if (part_k == 0) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int s = 1; s < WK; ++s) {
                        const float4 p = s_sum[((s * WN + wid) * RT + rt) * 64 + lane];
                        acc[rt][0] += p.x; acc[rt][1] += p.y; acc[rt][2] += p.z; acc[rt][3] += p.w;
                    }
            }
        }
        if (part_k == 0 && n0 + q * 4 < a.N) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int at = rt * 16 + r;
                if (at >= here) continue;
                const float weight = a.w ? a.w[s_list[at]] : 1.0f;
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = w4_finish(acc[rt][j], a.gelu, weight);
                w4_store(a, s_list[at], n0 + q * 4, v);
            }
        }
        if (from + (int)gridDim.z * CAP >= total) return;
        __syncthreads();
    }
}

// y[t] = sum over j, ascending, of the rows of assignments with an expert.  All rows of up to eight choices are requested at
// once, before it is known which count.  64 tokens, two choices of 2048 columns: 4.7 us, most of it a launch's start and end.
constexpr int JOIN_THREADS = 64;
template <typename OUT>
__global__ __launch_bounds__(JOIN_THREADS) void w4_join_kernel(const float* __restrict__ rows, const int* __restrict__ idx, OUT* __restrict__ y,
                                                               long long ldy, int k, int E, int N) {
    const int n = (blockIdx.x * JOIN_THREADS + threadIdx.x) * 4;
    const long long t = blockIdx.y;
    if (n >= N) return;
    float v[4] = {0, 0, 0, 0};
    for (int j0 = 0; j0 < k; j0 += 8) {
        float p[8][4];
        int e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            e[j] = -1;
            if (j0 + j >= k) continue;
            e[j] = idx ? idx[t * k + j0 + j] : 0;
            load_columns(rows + (t * k + j0 + j) * N + n, p[j], N - n);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += (unsigned)e[j] < (unsigned)E ? p[j][i] : 0.0f;
    }
    store_columns(y + t * ldy + n, v, N - n);
}

// One thread packs 32 columns of one weight row; neighbouring threads have neighbouring weight rows, which lie next to one
// another in W.  16 experts of 2048 x 8192 from bfloat16: 175 us, 3.9 TB/s.
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

// by_token: each token by itself (w4_token_kernel).  chosen: experts that may be expected to be chosen by T tokens, or the one
// that all have without topk_idx.
// The scratch: rows to be joined (0 bytes where there are none), then the list of many assignments.
struct W4Plan { long long ldx, ldy; int n_scales; size_t rows_bytes, list_bytes; bool by_token; double chosen; };

// Up to so many assignments every workgroup looks for its rows itself.  What that reads grows with their number times the grid, which
// grows with them too: T k = 2^24 would take hours.  Beyond that one launch lists them by expert (by themselves / listed: 1200
// assignments to 4 experts of 128 x 256 7.1 / 10 us, 2048 to 64 of 512 x 64 15.0 / 16.1, of 1024 x 4096 83 / 73, to 16 of 2048 x 8192
// 229 / 198; 4096 of these 470 / 354, to 8 of 512 x 2048 75 / 48; 65536 to 64 of 1024 x 4096 15 / 1.7 ms).
constexpr int LIST_FROM = 2048;

// Tokens by themselves read an expert's weights once for each of its rows, but have neither rows to collect nor shares of K to
// add up between launches.  That is worth 20 MB of weights more than are chosen, whatever the sizes (by tokens / by experts: 2 tokens, 2
// of 16 experts of 2048 x 8192 10 / 16 us, 4 tokens 14 / 21, 8 tokens 23.5 / 24, 12 tokens 33 / 26; 4096 x 1024, joined, 2 of 8
// experts, 4 tokens 6.1 / 11.7, 8 tokens 11.2 / 12.2, 12 tokens 15.2 / 12.5; 1024 x 4096, 8 of 64, 4 tokens 17 / 22, 6 tokens 23.5
// / 22.6; one token, 2 of 16 experts of 2048 x 8192 6.4 / 23).  Beyond 16 tokens, small matrices: 512 x 2048, 2 of 8 experts, 12
// tokens 6.2 / 6.4, 24 tokens 9.6 / 7.3.  Without topk_idx it is the same matrix every time, from the caches, and worth 30 MB: 2048 x
// 8192, 4 tokens 6.4 / 7.6, 6 tokens 8.5 / 7.8; 8192 x 8192, 2 tokens 15.5 / 12.9.
constexpr double TOKEN_MORE = 20e6, TOKEN_MORE_OF_ONE = 30e6;
constexpr int TOKENS_MOST = 16;

moe_status w4_plan(const moe_w4_config* c, bool routed, W4Plan* p) {
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
    if ((long long)c->N * c->K > INT_MAX) return MOE_ERR_UNSUPPORTED;          // offsets within an expert are 32-bit
    if (c->N > (1 << 26) - 16) return MOE_ERR_UNSUPPORTED;       // 16 columns and up to 1024 threads to a workgroup: below 2^32 of these
    if ((long long)c->T * c->k > (1 << 24) || (c->combine && c->T > 65535)) return MOE_ERR_UNSUPPORTED;
    p->n_scales = c->group ? (c->K + 127) / 128 : 1;
    p->chosen = !routed ? 1.0 : c->E * (1.0 - std::pow(1.0 - (double)c->k / c->E, (double)c->T));
    p->by_token = c->T == 1 || (c->T <= TOKENS_MOST && ((double)c->T * c->k - p->chosen) * c->K * c->N * (17.0 / 32.0) <=
                                     (routed ? TOKEN_MORE : TOKEN_MORE_OF_ONE));
    // Rows of several tokens' choices that are still to be added up.  Workgroups that have a token to themselves do that and need
    // none, but the size is to grow with T alone: a scratch for many tokens does for fewer.
    p->rows_bytes = c->combine && c->k > 1 && c->T > 1 ? (size_t)c->T * c->k * c->N * sizeof(float) : 0;
    p->list_bytes = c->T * c->k > LIST_FROM ? ((size_t)c->T * c->k + c->E + 2) * sizeof(int) : 0;
    return MOE_OK;
}

template <int XT> void w4_token_launch(const W4Args& a, int T, bool sum, hipStream_t s) {
    const int blocks = (a.N + 15) / 16, want = (a.K + 128 * TOKEN_TILES - 1) / (128 * TOKEN_TILES);
    if (sum && a.k > 1) {
        // the choices first, then K, among sixteen wavefronts; beyond sixteen choices a wavefront has several
        int slices = a.k <= TOKEN_WAVES ? TOKEN_WAVES / a.k : 1;
        slices = slices < want ? slices : want;
        const int waves = a.k <= TOKEN_WAVES ? slices * a.k : TOKEN_WAVES;
        if (waves <= 4) w4_token_kernel<XT, true, 4><<<dim3(blocks, 1, T), waves * 64, 0, s>>>(a, slices);
        else w4_token_kernel<XT, true, TOKEN_WAVES><<<dim3(blocks, 1, T), waves * 64, 0, s>>>(a, slices);
    } else {
        const int waves = want < TOKEN_WAVES ? want : TOKEN_WAVES;
        if (waves <= 4) w4_token_kernel<XT, false, 4><<<dim3(blocks, a.k, T), waves * 64, 0, s>>>(a, waves);
        else w4_token_kernel<XT, false, TOKEN_WAVES><<<dim3(blocks, a.k, T), waves * 64, 0, s>>>(a, waves);
    }
}

// Workgroups that share out an expert's rows: as many as three times the mean number wants (a gate's loads differ), or all of
// them want where they all have one expert.  Those that find no rows left end at once.
int w4_row_groups(const W4Args& a, int rows, int cap) {
    const int most = !a.idx || a.n_rows < 3 * rows ? a.n_rows : 3 * rows, groups = (most + cap - 1) / cap;
    return groups < 64 ? groups : 64;
}

template <int XT, int RT> void w4_rows_launch(const W4Args& a, int experts, int slots, int rows, hipStream_t s) {
    // All eight wavefronts side by side where that leaves a workgroup for every compute unit, else K in shares.
    constexpr int WK = most_shares<XT, RT>();
    const int wide = (a.N + 127) / 128, narrow = (a.N + 128 / WK - 1) / (128 / WK), groups = w4_row_groups(a, rows, 16 * RT);
    if (WK == 1 || (long long)wide * experts * groups >= compute_units())
        w4_rows_kernel<XT, RT, 1><<<dim3(wide, slots, groups), W4_WAVES * 64, 0, s>>>(a);
    else
        w4_rows_kernel<XT, RT, WK><<<dim3(narrow, slots, groups), W4_WAVES * 64, 0, s>>>(a);
}

template <int XT, int RT> void w4_few_launch(const W4Args& a, double chosen, int slots, int rows, hipStream_t s) {
    // As many shares of K as still let all wavefronts be there at once (eight to a compute unit): with a third more of them than
    // that, a second round for these few takes as long as the first.
    const int columns = (a.N + 63) / 64, tiles = (a.K + 127) / 128, row_groups = w4_row_groups(a, rows, 16 * RT);
    const int waves = 2 * FEW_WAVES * chosen * columns <= 8.0 * compute_units() && 2 * FEW_WAVES <= tiles ? FEW_MORE : FEW_WAVES;
    int shares = 1;
    while (shares < waves && 2 * shares * chosen * columns <= 8.0 * compute_units() && 2 * shares <= tiles) shares *= 2;
    const int groups = waves / shares;
    const dim3 grid((columns + groups - 1) / groups, slots, row_groups);
    if (waves == FEW_WAVES) w4_few_kernel<XT, RT, FEW_WAVES><<<grid, FEW_WAVES * 64, 0, s>>>(a, shares);
    else w4_few_kernel<XT, RT, FEW_MORE><<<grid, FEW_MORE * 64, 0, s>>>(a, shares);
}

template <int XT> void w4_launch(const W4Args& a, const W4Plan& p, int T, bool join, bool sum, hipStream_t s) {
    if (p.by_token) {
        w4_token_launch<XT>(a, T, sum, s);
        return;
    }
    // experts that may have rows, and how many each; and one more slot for rows of no expert
    const int experts = !a.idx ? 1 : a.n_rows < a.E ? a.n_rows : a.E, slots = !a.idx ? 1 : join ? a.E : a.E + 1;
    const int rows = (a.n_rows + experts - 1) / experts;
    // Two tiles of rows at a time and a workgroup for each 32 are as fast as four and one matrix read for 64 at some 40 rows each
    // (16 experts of 1024 x 4096: 16 rows 19 / 23 us, 32 rows 22 / 30, 40 rows 34 / 30).  Offsets in x are 32-bit in the kernel
    // for few rows.
    const long long x_bytes = (a.per_choice ? (long long)a.n_rows : (long long)T) * a.ldx * row_bytes(XT, 1);
    if (rows <= 32 && x_bytes < (1ll << 32)) {
        // 16 rows at a time, or 32 (of float rows 16: more would not fit into LDS).  The mean says little of the experts that have
        // most: 16 experts of 2048 x 8192 as a skewed gate loads them, mean 4: 16 rows 34 us, 32 rows 38; mean 5: 44, 37; mean 8:
        // 45, 41; 8192 x 2048, 64 experts, mean 8: 194, 197.
        if constexpr (XT != MOE_F32) {
            if (rows > 4) {
                w4_few_launch<XT, 2>(a, p.chosen, slots, rows, s);
                return;
            }
        }
        w4_few_launch<XT, 1>(a, p.chosen, slots, rows, s);
        return;
    }
    w4_rows_launch<XT, 4>(a, experts, slots, rows, s);
}

}  // namespace

}  // namespace moe

extern "C" moe_status moe_w4_scratch_bytes(const moe_w4_config* cfg, size_t* bytes) {
    moe::W4Plan p;
    MOE_TRY(moe::w4_plan(cfg, true, &p));                  // (the scratch is the same either way)
    if (!bytes) return MOE_ERR_NULL;
    *bytes = p.rows_bytes + p.list_bytes;
    return MOE_OK;
}

extern "C" moe_status moe_w4_product(const moe_w4_config* cfg, const void* x, const float* x_scales, const int32_t* topk_idx,
                                     const float* topk_w, const uint8_t* Wq, const uint8_t* Ws, void* y, void* scratch, void* stream) {
    moe::W4Plan p;
    MOE_TRY(moe::w4_plan(cfg, topk_idx != nullptr, &p));
    if (cfg->T == 0) return MOE_OK;
    if (!x || !Wq || !Ws || !y || (cfg->dtype == MOE_E4M3 && !x_scales)) return MOE_ERR_NULL;
    const bool listed = p.list_bytes != 0 && topk_idx;
    if ((p.rows_bytes || listed) && !scratch) return MOE_ERR_NULL;
    if (((uintptr_t)x | (uintptr_t)Wq | (uintptr_t)scratch) & 15) return MOE_ERR_UNSUPPORTED;
    hipStream_t s = (hipStream_t)stream;
    const int rows = cfg->T * cfg->k;
    const bool join = p.rows_bytes != 0 && !p.by_token;
    int* const begins = listed ? (int*)((char*)scratch + p.rows_bytes) : nullptr;
    int* const list = listed ? begins + cfg->E + 2 : nullptr;
    moe::W4Args a = {x, x_scales, topk_idx, topk_w, Wq, Ws, join ? scratch : y, list, begins, p.ldx, join ? cfg->N : p.ldy, rows,
                     cfg->k, cfg->E, cfg->K, cfg->N, p.n_scales, cfg->per_choice, cfg->gelu, join || cfg->out == MOE_F32};
    {
        moe::ProfScope prof(moe::PK_W4, s);
        if (listed) {
            moe::w4_list_kernel<<<cfg->E + 1, moe::LIST_WAVES * 64, 0, s>>>(topk_idx, rows, cfg->E, begins, list);
            MOE_CHECK_LAUNCH();
        }
        if (cfg->dtype == MOE_F32) moe::w4_launch<MOE_F32>(a, p, cfg->T, join, cfg->combine, s);
        else if (cfg->dtype == MOE_BF16) moe::w4_launch<MOE_BF16>(a, p, cfg->T, join, cfg->combine, s);
        else moe::w4_launch<MOE_E4M3>(a, p, cfg->T, join, cfg->combine, s);
        MOE_CHECK_LAUNCH();
        if (join) {
            const dim3 jgrid((cfg->N + 4 * moe::JOIN_THREADS - 1) / (4 * moe::JOIN_THREADS), cfg->T);
            if (cfg->out == MOE_F32)
                moe::w4_join_kernel<float><<<jgrid, moe::JOIN_THREADS, 0, s>>>((const float*)scratch, topk_idx, (float*)y, p.ldy, cfg->k, cfg->E, cfg->N);
            else
                moe::w4_join_kernel<moe::bf16_t><<<jgrid, moe::JOIN_THREADS, 0, s>>>((const float*)scratch, topk_idx, (moe::bf16_t*)y, p.ldy, cfg->k, cfg->E, cfg->N);
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
