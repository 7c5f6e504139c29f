// Products of a few rows with a matrix W [K,N] as the layer lays it out, N contiguous: y[r,n] = sum over k of row[r,k] W[k,n].
//
// Few rows meet the whole matrix, so what has to move is the matrix, once.  It goes from memory straight into the registers
// that the matrix instructions take; nothing of it passes through LDS.
//   bfloat16  A wavefront's step is 64 k x 64 columns: lane l loads columns 8 (l % 8) .. + 7 of the eight k rows 8 (l / 8) .. + 7,
//             whole lines, eight lanes to a row.  An 8 x 8 block to a lane turns around in registers (32 byte permutations), and its
//             column i is what instruction i of 16 x 16 x 32 wants as the lane's eight k of one row of the left operand: its 16 rows
//             are 8 columns of W (those numbered i in their eights) with the even blocks of 8 k in rows 0 to 7 and the same columns
//             with the odd blocks in rows 8 to 15.  The right operand has eight rows of the product, with the even blocks in
//             columns 0 to 7 and the odd ones in 8 to 15; of the 16 x 16 results the two 8 x 8 blocks on the diagonal are halves
//             of the sums, the others are of no use.  (The matrix pipe has room: eight instructions of 16 cycles on one of four
//             SIMDs for 8 KiB, which take a CU 1000 cycles to come when all of them read.)
//   float     A step is 32 k x 64 columns: lane l loads columns 4 (l % 16) .. + 3 of the k rows 8 (l / 16) .. + 7; load j and column
//             i of the four are an operand of 16 x 16 x 4, 16 columns against 16 rows of the product, as they are.
// The workgroup's wavefronts take the steps in turn and add up their sums through LDS, in their order.
#pragma once
#include "common.h"

namespace moe {

constexpr int FEW_COLS = 64;                         // columns of a workgroup
typedef float few_acc __attribute__((ext_vector_type(4)));
typedef __bf16 few_bf16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Few;
template <> struct Few<bf16_t> {
    static constexpr int ROWS = 8;                   // of a group
    static constexpr int STEP = 64;                  // k
    static constexpr int ACCS = 8;
    static constexpr int HALVES = 2;                 // sums of a wavefront that belong together
    static __device__ __forceinline__ int col(int lane) { return 8 * (lane & 7); }       // first of a lane's columns
    static __device__ __forceinline__ int k(int lane) { return 8 * (lane >> 3); }        // first of its k
    static __device__ __forceinline__ int row(int lane) { return lane & 7; }             // its row in the right operand
};
template <> struct Few<float> {
    static constexpr int ROWS = 16, STEP = 32, ACCS = 4, HALVES = 1;
    static __device__ __forceinline__ int col(int lane) { return 4 * (lane & 15); }
    static __device__ __forceinline__ int k(int lane) { return 8 * (lane >> 4); }
    static __device__ __forceinline__ int row(int lane) { return lane & 15; }
};

// What a step loads: eight k of W's columns, and of GROUPS groups of rows, each in PARTS (bfloat16) that add up to it.
template <typename T, int GROUPS, int PARTS> struct FewStep;
template <int GROUPS, int PARTS> struct FewStep<bf16_t, GROUPS, PARTS> {
    uint4 w[8], r[GROUPS][PARTS];
    __device__ __forceinline__ void load(const bf16_t* W, long long ldw, int k, int K) {
        const bf16_t* p = W + (long long)(k < K ? k : 0) * ldw;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const uint4*>(p + j * ldw);
    }
    __device__ __forceinline__ void load_rows(const bf16_t* const (&row)[GROUPS], long long part, int k, int K) {
        const int at = k < K ? k : 0;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int c = 0; c < PARTS; ++c) r[g][c] = *reinterpret_cast<const uint4*>(row[g] + c * part + at);
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
    __device__ __forceinline__ void load(const float* W, long long ldw, int k, int K) {
        const float* p = W + (long long)(k < K ? k : 0) * ldw;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const float4*>(p + j * ldw);
    }
    __device__ __forceinline__ void load_rows(const float* const (&row)[GROUPS], long long, int k, int K) {
        const int at = k < K ? k : 0;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            r[g][0] = *reinterpret_cast<const float4*>(row[g] + at);
            r[g][1] = *reinterpret_cast<const float4*>(row[g] + at + 4);
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

// Where the sums of one group of a wavefront, or of half of one, go: [rows][columns], rows apart by a bank's width more.
constexpr int FEW_PITCH = FEW_COLS + 4;
template <typename T, int WAVES> struct FewSums { float v[WAVES * Few<T>::HALVES][Few<T>::ROWS][FEW_PITCH]; };

// Sums over the steps first, first + WAVES, ... below `steps` of K (a multiple of 8), each wavefront its own.  W: the workgroup's
// first column; cols: columns there are from it on; row: the lane's row of each group (any row will do where there is none).
template <typename T, int GROUPS, int PARTS, int WAVES>
__device__ __forceinline__ void few_sums(const T* W, long long ldw, int cols, const T* const (&row)[GROUPS], long long part, int K, int first,
                                         int steps, few_acc (&acc)[GROUPS][Few<T>::ACCS]) {
    const int lane = threadIdx.x & 63;
    // columns past the last are the first ones again, and not looked at
    const int c = Few<T>::col(lane);
    W += c < cols ? c : 0;
    const int k0 = Few<T>::k(lane);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int i = 0; i < Few<T>::ACCS; ++i) acc[g][i] = few_acc{0, 0, 0, 0};
    // The next step's loads are under way while one is multiplied; of eight fragments of rows (which come from the caches) there are no
    // registers to hold two steps'.
    constexpr bool EARLY = GROUPS * PARTS < 8;
    FewStep<T, GROUPS, PARTS> a, b;
    int s = __builtin_amdgcn_readfirstlane(first);
    if (s < steps) {
        a.load(W, ldw, s * Few<T>::STEP + k0, K);
        if (EARLY) a.load_rows(row, part, s * Few<T>::STEP + k0, K);
    }
    while (s < steps) {
        const int next = s + WAVES;
        if (!EARLY) a.load_rows(row, part, s * Few<T>::STEP + k0, K);
        if (next < steps) {
            b.load(W, ldw, next * Few<T>::STEP + k0, K);
            if (EARLY) b.load_rows(row, part, next * Few<T>::STEP + k0, K);
        }
        if ((s + 1) * Few<T>::STEP > K && s * Few<T>::STEP + k0 >= K) a.zero();        // (nothing meets what was loaded in its place)
        a.multiply(acc);
        s = next;
        a = b;
    }
}

// A group's sums from the wavefronts' registers to LDS.
template <typename T, int GROUPS, int WAVES>
__device__ __forceinline__ void few_put(FewSums<T, WAVES>& s, const few_acc (&acc)[GROUPS][Few<T>::ACCS], int g) {
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    if constexpr (sizeof(T) == 2) {
        const int col = lane & 15, q = lane >> 4;
        if ((q >> 1) != (col >> 3)) return;              // beside the diagonal
        float* p = &s.v[wid * 2 + (q >> 1)][col & 7][8 * (4 * (q & 1))];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            *reinterpret_cast<float4*>(p + 8 * j) = make_float4(acc[g][0][j], acc[g][1][j], acc[g][2][j], acc[g][3][j]);
            *reinterpret_cast<float4*>(p + 8 * j + 4) = make_float4(acc[g][4][j], acc[g][5][j], acc[g][6][j], acc[g][7][j]);
        }
    } else {
        float* p = &s.v[wid][lane & 15][4 * (4 * (lane >> 4))];
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<float4*>(p + 4 * j) = make_float4(acc[g][0][j], acc[g][1][j], acc[g][2][j], acc[g][3][j]);
    }
}
template <typename T, int WAVES> __device__ __forceinline__ float few_sum(const FewSums<T, WAVES>& s, int row, int col) {
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES * Few<T>::HALVES; ++w) v += s.v[w][row][col];
    return v;
}

// f(row of the groups, column, sum) for the sums of all of them; every thread of the workgroup comes here.
template <typename T, int GROUPS, int WAVES, typename F>
__device__ __forceinline__ void few_finish(FewSums<T, WAVES>& s, const few_acc (&acc)[GROUPS][Few<T>::ACCS], int rows, int cols, F&& f) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        if (g * Few<T>::ROWS >= rows) break;
        few_put<T, GROUPS, WAVES>(s, acc, g);
        __syncthreads();
        for (int o = threadIdx.x; o < Few<T>::ROWS * FEW_COLS; o += WAVES * 64) {
            const int r = o / FEW_COLS, n = o % FEW_COLS;
            if (g * Few<T>::ROWS + r < rows && n < cols) f(g * Few<T>::ROWS + r, n, few_sum<T, WAVES>(s, r, n));
        }
        __syncthreads();
    }
}

}  // namespace moe
