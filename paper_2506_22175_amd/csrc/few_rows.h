// Products of a few rows with a matrix W [K,N] as the layer lays it out, N contiguous: y[r,n] = sum over k of row[r,k] W[k,n].
//
// Few rows meet the whole matrix, so what has to move is the matrix, once.  It goes from memory straight into the registers
// that the matrix instructions take; nothing of it passes through LDS.
//   bfloat16  A wavefront's step is 32 k x 128 columns: lane l loads columns 8 (l % 16) .. + 7 of the eight k rows 8 (l / 16) .. + 7,
//             256 neighbouring bytes to a row.  An 8 x 8 block to a lane turns around in registers (32 byte permutations), and its
//             column i is what instruction i of 16 x 16 x 32 wants as the lane's eight k of a row of the left operand, whose 16 rows
//             are the columns of W numbered i in their eights.  The right operand has 16 rows of the product.  (The matrix pipe has
//             room: eight instructions of 16 cycles on one of four SIMDs for 8 KiB, which take a CU 700 cycles to come when all read.)
//   float     A step is 32 k x 64 columns: lane l loads columns 4 (l % 16) .. + 3 of the k rows 8 (l / 16) .. + 7; load j and column
//             i of the four are an operand of 16 x 16 x 4, as they are.
// Rows are read in pieces of 256 bytes, past the caches (537 MB in 64 matrices: pieces of 128 bytes 5.9 TB/s, of 256 6.6, 512 7.1, and
// 10 % less with ordinary loads; wider pieces would leave a single matrix too few workgroups).
// The workgroup's wavefronts take the steps in turn and add up their sums through LDS, in their order.
// Up to eight rows may go in pieces of 128 bytes (NARROW), which is twice the workgroups where there are too few for the chip: a step is twice
// the k of half the columns.  Lanes l and l + 8 have the same columns and other k, each with its row number l % 8 of the right operand
// at its own k; of the instruction's result the rows and columns below eight are a sum over the first of these k, those from eight on over the others,
// and the rest means nothing.
#pragma once
#include "common.h"
#include "wide.h"

namespace moe {

typedef float few_acc __attribute__((ext_vector_type(4)));
typedef __bf16 few_bf16x8 __attribute__((ext_vector_type(8)));

template <typename T, bool NARROW = false> struct Few {
    static constexpr int LANES = NARROW ? 8 : 16;    // to a piece
    static constexpr int COLS = LANES * 16 / sizeof(T);      // of a workgroup
    static constexpr int ROWS = LANES;               // of a group
    static constexpr int STEP = 512 / LANES;         // k
    static constexpr int ACCS = 16 / sizeof(T);      // columns of a lane's load
    static __device__ __forceinline__ int col(int lane) { return ACCS * (lane % LANES); }    // first of a lane's columns
    static __device__ __forceinline__ int k(int lane) { return 8 * (lane / LANES); }         // first of its k
    static __device__ __forceinline__ int row(int lane) { return lane % LANES; }             // its row in the right operand
};

// What a step loads: eight k of W's columns, and of GROUPS groups of rows, each in PARTS (bfloat16) that add up to it.
template <typename T, int GROUPS, int PARTS> struct FewStep;
template <int GROUPS, int PARTS> struct FewStep<bf16_t, GROUPS, PARTS> {
    uint4 w[8], r[GROUPS][PARTS];
    __device__ __forceinline__ void load(const bf16_t* W, unsigned ldw, unsigned col, int k, int K) {
        const char* p = reinterpret_cast<const char*>(W);
        unsigned at = ((k < K ? k : 0) * ldw + col) * 2u;
#pragma unroll
        for (int j = 0; j < 8; ++j, at += ldw * 2u) w[j] = load_once<uint4>(p + at);
    }
    __device__ __forceinline__ void load_rows(const bf16_t* const (&rows)[PARTS], const unsigned (&row)[GROUPS], int k, int K) {
        const unsigned at = (k < K ? k : 0) * 2u;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int c = 0; c < PARTS; ++c) r[g][c] = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(rows[c]) + (row[g] + at));
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int c = 0; c < PARTS; ++c) r[g][c] = make_uint4(0, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned word(const uint4& u, int i) { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; }
    __device__ __forceinline__ void multiply(few_acc (&acc)[GROUPS][8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned pick = i & 1 ? 0x07060302u : 0x05040100u;
            uint4 a;
            a.x = __builtin_amdgcn_perm(word(w[1], i / 2), word(w[0], i / 2), pick);
            a.y = __builtin_amdgcn_perm(word(w[3], i / 2), word(w[2], i / 2), pick);
            a.z = __builtin_amdgcn_perm(word(w[5], i / 2), word(w[4], i / 2), pick);
            a.w = __builtin_amdgcn_perm(word(w[7], i / 2), word(w[6], i / 2), pick);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int c = 0; c < PARTS; ++c)
                    acc[g][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(few_bf16x8, a), __builtin_bit_cast(few_bf16x8, r[g][c]), acc[g][i], 0, 0, 0);
        }
    }
};
template <int GROUPS, int PARTS> struct FewStep<float, GROUPS, PARTS> {
    static_assert(PARTS == 1, "a float is one part");
    float4 w[8], r[GROUPS][2];
    __device__ __forceinline__ void load(const float* W, unsigned ldw, unsigned col, int k, int K) {
        const char* p = reinterpret_cast<const char*>(W);
        unsigned at = ((k < K ? k : 0) * ldw + col) * 4u;
#pragma unroll
        for (int j = 0; j < 8; ++j, at += ldw * 4u) w[j] = load_once<float4>(p + at);
    }
    __device__ __forceinline__ void load_rows(const float* const (&rows)[1], const unsigned (&row)[GROUPS], int k, int K) {
        const char* p = reinterpret_cast<const char*>(rows[0]);
        const unsigned at = (k < K ? k : 0) * 4u;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            r[g][0] = *reinterpret_cast<const float4*>(p + (row[g] + at));
            r[g][1] = *reinterpret_cast<const float4*>(p + (row[g] + at + 16u));
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) r[g][0] = r[g][1] = make_float4(0, 0, 0, 0);
    }
    static __device__ __forceinline__ float part(const float4& u, int i) { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; }
    __device__ __forceinline__ void multiply(few_acc (&acc)[GROUPS][4]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
                    acc[g][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(part(w[j], i), part(r[g][j / 4], j & 3), acc[g][i], 0, 0, 0);
    }
};

// Where the wavefronts' sums of eight rows go: rows a bank's width more apart.
constexpr int FEW_PASS = 8;
template <typename T, int WAVES, bool NARROW = false> struct FewSums { float v[NARROW ? 2 * WAVES : WAVES][FEW_PASS][Few<T, NARROW>::COLS + 4]; };

// Sums over the steps first, first + WAVES, ... below `steps` of K (a multiple of 8), each wavefront its own.  W: the workgroup's
// first column; cols: columns there are from it on; rows: the rows' parts, row: where the lane's row of each group begins, in bytes (any
// row will do where there is none).  Offsets are 32 bits wide: a matrix has less than 2^32 bytes.
// A wavefront waits for a step's loads and has no others under way meanwhile: registers for two steps would leave a CU half the wavefronts
// (and the compiler waits for both where it copies one's to the other's), and sixteen of them have 128 KiB under way, twice what the memory's
// latency asks of a CU.
template <typename T, int GROUPS, int PARTS, int WAVES, bool NARROW = false>
__device__ __forceinline__ void few_sums(const T* W, unsigned ldw, int cols, const T* const (&rows)[PARTS], const unsigned (&row)[GROUPS], int K, int first,
                                         int steps, few_acc (&acc)[GROUPS][Few<T>::ACCS]) {
    const int lane = threadIdx.x & 63;
    // columns past the last are the first ones again, and not looked at
    const int c = Few<T, NARROW>::col(lane);
    const unsigned col = c < cols ? c : 0;
    const int k0 = Few<T, NARROW>::k(lane);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int i = 0; i < Few<T>::ACCS; ++i) acc[g][i] = few_acc{0, 0, 0, 0};
#pragma unroll 1
    for (int s = __builtin_amdgcn_readfirstlane(first); s < steps; s += WAVES) {
        FewStep<T, GROUPS, PARTS> x;
        const int k = s * Few<T, NARROW>::STEP + k0;
        x.load(W, ldw, col, k, K);
        x.load_rows(rows, row, k, K);
        if ((s + 1) * Few<T, NARROW>::STEP > K) {                  // (nothing meets what was loaded in the place of what is not there)
            if (k >= K) x.zero();
        }
        x.multiply(acc);
    }
}

// f(row of the groups, column, sum) for the sums of all of them, eight rows at a time; every thread of the workgroup comes here.
template <typename T, int GROUPS, int WAVES, bool NARROW = false, typename F>
__device__ __forceinline__ void few_finish(FewSums<T, WAVES, NARROW>& s, const few_acc (&acc)[GROUPS][Few<T>::ACCS], int rows, int cols, F&& f) {
    constexpr int COLS = Few<T, NARROW>::COLS, ACCS = Few<T>::ACCS, SUMS = NARROW ? 2 * WAVES : WAVES;
    static_assert(!NARROW || GROUPS == 1, "eight rows");
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
#pragma unroll
    for (int p = 0; p < GROUPS * Few<T, NARROW>::ROWS / FEW_PASS; ++p) {
        if (p * FEW_PASS >= rows) break;
        // lane l has row l % 16 of the group, and in register j of accumulator i column i of the eight (four) number 4 (l / 16) + j
        const int g = p * FEW_PASS / Few<T>::ROWS, half = lane >> 5, r0 = NARROW ? 8 * half : p * FEW_PASS % Few<T>::ROWS, r = (lane & 15) - r0;
        if (r >= 0 && r < FEW_PASS) {
            float* o = NARROW ? &s.v[2 * wid + half][r][ACCS * 4 * (lane >> 4 & 1)] : &s.v[wid][r][ACCS * 4 * (lane >> 4)];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < ACCS; i += 4)
                    *reinterpret_cast<float4*>(o + ACCS * j + i) = make_float4(acc[g][i][j], acc[g][i + 1][j], acc[g][i + 2][j], acc[g][i + 3][j]);
        }
        __syncthreads();
        for (int o = threadIdx.x; o < FEW_PASS * COLS; o += WAVES * 64) {
            const int row = o / COLS, n = o % COLS;
            if (p * FEW_PASS + row >= rows || n >= cols) continue;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < SUMS; ++w) v += s.v[w][row][n];
            f(p * FEW_PASS + row, n, v);
        }
        __syncthreads();
    }
}

}  // namespace moe
