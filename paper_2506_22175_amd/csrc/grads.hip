// The norm of all gradients together, and their clipping by it.
//
//   norm = sqrt(sum over all tensors of g^2);  out = g * min(1, most / norm)
//
// Nothing but memory bounds either: the norm reads every element once, clipping reads it again and writes it.  Squares and sums
// are in 64 bits, which the vector unit does in the shadow of the loads and in which nothing overflows or vanishes.
//
// The tensors' places are in a table in device memory, written once for a list of tensors, so that one launch covers any number
// of them.  It cuts them into chunks of 32 KiB, of which a workgroup takes every so many-th; eight 16-byte loads of a thread are
// a chunk.  The workgroups leave a partial sum each, and the last one to finish adds them up, always in the same order.
#include "common.h"
#include "wide.h"
#include <algorithm>
#include <cmath>
#include <new>

namespace moe {

namespace {

constexpr int GRAD_THREADS = 256, GRAD_LOADS = 8;
constexpr int GRAD_CHUNK = GRAD_THREADS * GRAD_LOADS * 16;         // bytes
constexpr int GRAD_BLOCKS = 2048;                                  // workgroups at most
constexpr int GRAD_MOST = 65536;                                   // tensors

struct GradEntry { const void* grad; void* out; long long n; int first, bf16; };      // first: number of its first chunk
struct GradHead { unsigned arrived; };
constexpr size_t GRAD_HEAD_BYTES = 256;

__host__ __device__ long long grad_chunk_elements(int bf16) { return bf16 ? GRAD_CHUNK / 2 : GRAD_CHUNK / 4; }

// which tensor each chunk belongs to, behind the tensors
__host__ __device__ size_t grad_map_offset(int count) { return GRAD_HEAD_BYTES + (size_t)count * sizeof(GradEntry); }

constexpr int GRAD_BATCH = 64;                                     // entries of a launch's arguments
struct GradTableArgs { GradEntry e[GRAD_BATCH]; int from, here; };

__global__ __launch_bounds__(256) void grad_table_kernel(GradTableArgs a, char* table, int count) {
    const GradEntry e = a.e[blockIdx.x];
    const int number = a.from + blockIdx.x;
    if (threadIdx.x == 0) {
        if (number == 0) reinterpret_cast<GradHead*>(table)->arrived = 0;
        if (number < count) reinterpret_cast<GradEntry*>(table + GRAD_HEAD_BYTES)[number] = e;
    }
    int* map = reinterpret_cast<int*>(table + grad_map_offset(count));
    const long long per = grad_chunk_elements(e.bf16), chunks = (e.n + per - 1) / per;
    for (long long i = threadIdx.x; i < chunks; i += 256) map[e.first + i] = number;
}

struct GradArgs { char* table; int count, chunks; double* partial; float* norm; float most; };

struct Chunk { GradEntry e; long long at; int left; };             // first element, elements
__device__ __forceinline__ Chunk chunk_of(const GradArgs& a, int number) {
    const int t = reinterpret_cast<const int*>(a.table + grad_map_offset(a.count))[number];
    Chunk c;
    c.e = reinterpret_cast<const GradEntry*>(a.table + GRAD_HEAD_BYTES)[t];
    const long long per = grad_chunk_elements(c.e.bf16);
    c.at = (number - c.e.first) * per;
    const long long left = c.e.n - c.at;
    c.left = (int)(left < per ? left : per);
    return c;
}

// Elements of 16 bytes.
template <typename T> struct Unit;
template <> struct Unit<float> {
    static constexpr int N = 4;
    Anywhere<16, 4> u;
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(u.w[i]); }
};
template <> struct Unit<bf16_t> {
    static constexpr int N = 8;
    Anywhere<16, 2> u;
    __device__ __forceinline__ float at(int i) const { return __uint_as_float((i & 1) ? u.w[i / 2] & 0xffff0000u : u.w[i / 2] << 16); }
};

template <typename T> __device__ __forceinline__ double chunk_squares(const Chunk& c) {
    constexpr int N = Unit<T>::N;
    const T* p = reinterpret_cast<const T*>(c.e.grad) + c.at;
    double sum = 0.0;
    Unit<T> v[GRAD_LOADS];
    const int whole = c.left / N;
#pragma unroll
    for (int j = 0; j < GRAD_LOADS; ++j) {
        const int i = j * GRAD_THREADS + threadIdx.x;
        if (i < whole) v[j].u = *reinterpret_cast<const decltype(v[j].u)*>(p + i * N);
        else v[j].u.w[0] = v[j].u.w[1] = v[j].u.w[2] = v[j].u.w[3] = 0;
    }
#pragma unroll
    for (int j = 0; j < GRAD_LOADS; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const double d = (double)v[j].at(i);
            sum = fma(d, d, sum);
        }
    const int rest = whole * N + threadIdx.x;
    if (rest < c.left) {
        const double d = (double)Elem<T>::ld(p + rest);
        sum = fma(d, d, sum);
    }
    return sum;
}

// over a workgroup; thread 0 has the sum
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_down(v, off, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) sum += lds[w];
    __syncthreads();
    return sum;
}

__global__ __launch_bounds__(GRAD_THREADS) void grad_norm_kernel(GradArgs a) {
    __shared__ double lds[GRAD_THREADS / 64];
    __shared__ bool last;
    double sum = 0.0;
    for (int number = blockIdx.x; number < a.chunks; number += gridDim.x) {
        const Chunk c = chunk_of(a, number);
        sum += c.e.bf16 ? chunk_squares<bf16_t>(c) : chunk_squares<float>(c);
    }
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) {
        a.partial[blockIdx.x] = sum;
        unsigned* arrived = &reinterpret_cast<GradHead*>(a.table)->arrived;
        last = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
        if (last) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next call
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double total = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += GRAD_THREADS) total += a.partial[i];
    total = block_sum(total, lds);
    if (threadIdx.x == 0) *a.norm = (float)sqrt(total);
}

template <typename T> __device__ __forceinline__ void chunk_scale(const Chunk& c, double factor) {
    constexpr int N = Unit<T>::N;
    const T* p = reinterpret_cast<const T*>(c.e.grad) + c.at;
    T* o = reinterpret_cast<T*>(c.e.out) + c.at;
    Unit<T> v[GRAD_LOADS];
    const int whole = c.left / N;
#pragma unroll
    for (int j = 0; j < GRAD_LOADS; ++j) {
        const int i = j * GRAD_THREADS + threadIdx.x;
        if (i < whole) v[j].u = *reinterpret_cast<const decltype(v[j].u)*>(p + i * N);
    }
    const int rest = whole * N + threadIdx.x;
    float tail = 0.0f;
    if (rest < c.left) tail = Elem<T>::ld(p + rest);
#pragma unroll
    for (int j = 0; j < GRAD_LOADS; ++j) {
        const int i = j * GRAD_THREADS + threadIdx.x;
        if (i < whole) {
            Unit<T> r;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if constexpr (sizeof(T) == 4) r.u.w[q] = __float_as_uint((float)((double)v[j].at(q) * factor));
                else r.u.w[q] = pack_bf16x2((float)((double)v[j].at(2 * q) * factor), (float)((double)v[j].at(2 * q + 1) * factor));
            }
            *reinterpret_cast<decltype(r.u)*>(o + i * N) = r.u;
        }
    }
    if (rest < c.left) Elem<T>::st(o + rest, (float)((double)tail * factor));
}

__global__ __launch_bounds__(GRAD_THREADS) void grad_scale_kernel(GradArgs a) {
    const double norm = (double)*a.norm;
    // (NaN and infinity: nothing is scaled)
    const double factor = norm > (double)a.most && norm < (double)__builtin_inff() ? (double)a.most / norm : 1.0;
    for (int back = blockIdx.x; back < a.chunks; back += gridDim.x) {
        const Chunk c = chunk_of(a, a.chunks - 1 - back);
        if (factor == 1.0 && c.e.grad == c.e.out) continue;
        if (c.e.bf16) chunk_scale<bf16_t>(c, factor); else chunk_scale<float>(c, factor);
    }
}

moe_status grad_check(const moe_grad_tensor* t, int count, long long* chunks) {
    if (count < 0) return MOE_ERR_SHAPE;
    if (count > 0 && !t) return MOE_ERR_NULL;
    if (count > GRAD_MOST) return MOE_ERR_UNSUPPORTED;
    *chunks = 0;
    for (int i = 0; i < count; ++i) {
        if (t[i].n < 0) return MOE_ERR_SHAPE;
        if (t[i].dtype != MOE_F32 && t[i].dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
        const int es = t[i].dtype == MOE_BF16 ? 2 : 4;
        if (t[i].n > (1ll << 46)) return MOE_ERR_UNSUPPORTED;
        if (t[i].n > 0 && !t[i].grad) return MOE_ERR_NULL;
        if ((((uintptr_t)t[i].grad | (uintptr_t)t[i].out) & (es - 1)) != 0) return MOE_ERR_UNSUPPORTED;
        const long long per = grad_chunk_elements(t[i].dtype == MOE_BF16);
        *chunks += (t[i].n + per - 1) / per;
        if (*chunks > (1ll << 30)) return MOE_ERR_UNSUPPORTED;
    }
    return MOE_OK;
}

// Outputs may not overlap each other, nor another tensor's input, nor their own input but by being it.
moe_status grad_overlaps(const moe_grad_tensor* t, int count) {
    struct Span { uintptr_t from, to; int tensor; bool out; };
    Span* spans = new (std::nothrow) Span[(size_t)count * 2 + 1];
    if (!spans) return MOE_ERR_WORKSPACE;
    int n = 0;
    for (int i = 0; i < count; ++i) {
        const uintptr_t bytes = (uintptr_t)t[i].n * (t[i].dtype == MOE_BF16 ? 2 : 4), g = (uintptr_t)t[i].grad, o = (uintptr_t)t[i].out;
        if (bytes == 0) continue;
        if (o != g) spans[n++] = {g, g + bytes, i, false};
        if (o) spans[n++] = {o, o + bytes, i, true};
    }
    std::sort(spans, spans + n, [](const Span& a, const Span& b) { return a.from < b.from; });
    // the furthest end so far of outputs, and of anything
    uintptr_t out_end = 0, any_end = 0;
    moe_status s = MOE_OK;
    for (int i = 0; i < n && s == MOE_OK; ++i) {
        if (spans[i].from < (spans[i].out ? any_end : out_end)) s = MOE_ERR_SHAPE;
        if (spans[i].to > any_end) any_end = spans[i].to;
        if (spans[i].out && spans[i].to > out_end) out_end = spans[i].to;
    }
    delete[] spans;
    return s;
}

moe_status grad_list_check(const moe_grad_list* l) {
    if (!l) return MOE_ERR_NULL;
    if (l->tensors < 0 || l->chunks < 0 || l->chunks > (1ll << 30)) return MOE_ERR_SHAPE;
    if (!l->table) return MOE_ERR_NULL;
    return MOE_OK;
}

int grad_blocks(long long chunks) { return chunks < 1 ? 1 : chunks < GRAD_BLOCKS ? (int)chunks : GRAD_BLOCKS; }

}  // namespace

}  // namespace moe

extern "C" moe_status moe_grad_bytes(const moe_grad_tensor* tensors, int32_t count, size_t* table, size_t* scratch) {
    long long chunks;
    MOE_TRY(moe::grad_check(tensors, count, &chunks));
    if (!table || !scratch) return MOE_ERR_NULL;
    *table = moe::grad_map_offset(count) + (size_t)chunks * 4;
    *scratch = (size_t)moe::grad_blocks(chunks) * 8;
    return MOE_OK;
}

extern "C" moe_status moe_grad_table(const moe_grad_tensor* tensors, int32_t count, void* table, moe_grad_list* list, void* stream) {
    long long chunks;
    MOE_TRY(moe::grad_check(tensors, count, &chunks));
    if (!table || !list) return MOE_ERR_NULL;
    if ((uintptr_t)table & 15) return MOE_ERR_UNSUPPORTED;
    MOE_TRY(moe::grad_overlaps(tensors, count));
    moe_grad_list l = {table, chunks, count, 1};
    hipStream_t s = (hipStream_t)stream;
    int first = 0;
    moe::GradTableArgs a = {};
    for (int i = 0; i < count; ++i) {
        moe::GradEntry& e = a.e[a.here++];
        e = {tensors[i].grad, tensors[i].out, (long long)tensors[i].n, first, tensors[i].dtype == MOE_BF16};
        const long long per = moe::grad_chunk_elements(e.bf16);
        first += (int)((e.n + per - 1) / per);
        if (e.n > 0 && !e.out) l.outs = 0;
        if (a.here == moe::GRAD_BATCH || i == count - 1) {
            moe::grad_table_kernel<<<a.here, 256, 0, s>>>(a, (char*)table, count);
            MOE_CHECK_LAUNCH();
            a.from += a.here;
            a.here = 0;
        }
    }
    if (count == 0) {                                    // its head all the same
        moe::grad_table_kernel<<<1, 256, 0, s>>>(a, (char*)table, count);
        MOE_CHECK_LAUNCH();
    }
    *list = l;
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

extern "C" moe_status moe_grad_norm(const moe_grad_list* list, float* norm, void* scratch, void* stream) {
    MOE_TRY(moe::grad_list_check(list));
    if (!norm || !scratch) return MOE_ERR_NULL;
    if ((uintptr_t)scratch & 7) return MOE_ERR_UNSUPPORTED;
    moe::GradArgs a = {(char*)list->table, list->tensors, (int)list->chunks, (double*)scratch, norm, 0.0f};
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_GRADS, s);
        moe::grad_norm_kernel<<<moe::grad_blocks(list->chunks), moe::GRAD_THREADS, 0, s>>>(a);
    }
    MOE_CHECK_LAUNCH();
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

extern "C" moe_status moe_grad_scale(const moe_grad_list* list, float most, const float* norm, void* stream) {
    MOE_TRY(moe::grad_list_check(list));
    if (!(most >= 0.0f) || !std::isfinite(most)) return MOE_ERR_SHAPE;
    if (!norm || !list->outs) return MOE_ERR_NULL;
    if (list->chunks == 0) return MOE_OK;
    moe::GradArgs a = {(char*)list->table, list->tensors, (int)list->chunks, nullptr, const_cast<float*>(norm), most};
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_GRADS, s);
        moe::grad_scale_kernel<<<moe::grad_blocks(list->chunks), moe::GRAD_THREADS, 0, s>>>(a);
    }
    MOE_CHECK_LAUNCH();
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

extern "C" moe_status moe_grad_clip(const moe_grad_list* list, float most, float* norm, void* scratch, void* stream) {
    MOE_TRY(moe::grad_list_check(list));
    if (!(most >= 0.0f) || !std::isfinite(most)) return MOE_ERR_SHAPE;
    if (!list->outs) return MOE_ERR_NULL;
    MOE_TRY(moe_grad_norm(list, norm, scratch, stream));
    return moe_grad_scale(list, most, norm, stream);
}
