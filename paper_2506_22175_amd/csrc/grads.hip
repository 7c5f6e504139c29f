// The norm of all gradients together, and their clipping by it.
//
//   norm = sqrt(sum over all tensors of g^2);  out = g * min(1, most / norm)
//
// Nothing but memory bounds either: the norm reads every element once, clipping reads it again and writes it (537 MB of a block's gradients:
// 80 us, 6.7 TB/s, and 183 us, 5.9 TB/s, the reads and writes of a copy of as much 207; 300 tensors with 23 MB: 17 us in all).  Squares and sums
// are in 64 bits, which the vector unit does in the shadow of the loads and in which nothing overflows or vanishes.
//
// The tensors' chunks of 32 KiB are in a table in device memory, written once for a list of tensors, so that one launch covers any number
// of them, and a workgroup needs one look at the table for a chunk.  Of the chunks a workgroup takes every so many-th; eight 16-byte loads of a thread are
// a chunk, and there are enough workgroups for some to wait while others add.  The workgroups leave a partial sum each.  Whoever needs
// the norm adds those up: a workgroup of its own, or every workgroup of the scaling while its first chunk is on its way.  (The last
// workgroup to finish cannot do it cheaply: what makes its neighbours' sums visible to it empties the caches of eight dies, and cost
// 888 workgroups 25 us.)
#include "common.h"
#include "wide.h"
#include <algorithm>
#include <cmath>
#include <new>

namespace moe {

namespace {

constexpr int GRAD_THREADS = 256, GRAD_LOADS = 8;
constexpr int GRAD_CHUNK = GRAD_THREADS * GRAD_LOADS * 16;         // bytes
constexpr int GRAD_BLOCKS = 2048;                                  // workgroups at most (1024: the same within 1 %)
constexpr int GRAD_MOST = 65536;                                   // tensors

struct GradEntry { const void* grad; void* out; long long n; int first, bf16; };      // first: number of its first chunk
struct alignas(16) GradChunk { const char* grad; char* out; int whole, rest, bf16, unused; };        // units of 16 bytes, elements behind them

__host__ __device__ long long grad_chunk_elements(int bf16) { return bf16 ? GRAD_CHUNK / 2 : GRAD_CHUNK / 4; }

constexpr int GRAD_BATCH = 64;                                     // entries of a launch's arguments
struct GradTableArgs { GradEntry e[GRAD_BATCH]; };

__global__ __launch_bounds__(256) void grad_table_kernel(GradTableArgs a, GradChunk* table) {
    const GradEntry e = a.e[blockIdx.x];
    const long long per = grad_chunk_elements(e.bf16), chunks = (e.n + per - 1) / per;
    const int es = e.bf16 ? 2 : 4;
    for (long long i = threadIdx.x; i < chunks; i += 256) {
        const long long left = e.n - i * per, here = left < per ? left : per;
        GradChunk c;
        c.grad = reinterpret_cast<const char*>(e.grad) + i * GRAD_CHUNK;
        c.out = e.out ? reinterpret_cast<char*>(e.out) + i * GRAD_CHUNK : nullptr;
        c.whole = (int)(here * es / 16);
        c.rest = (int)(here - (long long)c.whole * 16 / es);
        c.bf16 = e.bf16;
        c.unused = 0;
        table[e.first + i] = c;
    }
}

// kept: the list is small enough to stay in the caches from the norm to the scaling, and is read in a way that leaves it there; larger
// ones are read past them.  (Clipping of 5 MB 9.2 us, 10.4 past the caches; 20 MB 16.3 and 15.2; 46 MB 24.9 and 28.5; 537 MB 308 and 270.)
constexpr long long GRAD_KEPT = 128 * 1024 * 1024 / GRAD_CHUNK;
struct GradArgs { const GradChunk* table; int chunks, kept, partials; double* partial; float* norm; float most; };

// A float that rounds to bfloat16 as d does: 14 bits of its mantissa, the last one set where anything follows it, which float has room for wherever
// a bfloat16 may come of it.  (d's nearest float may lie in the middle of two bfloat16 where d does not.)
__device__ __forceinline__ float for_bf16(double d) {
    const unsigned long long b = __double_as_longlong(d);
    const unsigned hi = (unsigned)(b >> 32), below = (hi & 63u) | (unsigned)b;
    const unsigned odd = (hi & ~63u) | (below < 1u ? below : 1u) << 6;
    return (float)__longlong_as_double((long long)((unsigned long long)odd << 32));
}

// A chunk and what a thread has of it: units of 16 bytes, and an element behind the last whole one.
struct Chunk {
    const char* grad; char* out;
    int whole, rest;                                               // units, elements behind them
    bool bf16;
    Anywhere<16, 2> v[GRAD_LOADS];
    float tail;
    __device__ __forceinline__ bool has_tail() const { return (int)threadIdx.x < rest; }
    __device__ __forceinline__ int unit(int j) const { return j * GRAD_THREADS + (int)threadIdx.x; }
    __device__ __forceinline__ void find(const GradArgs& a, int number) {
        const GradChunk c = a.table[number];
        grad = c.grad;
        out = c.out;
        whole = c.whole;
        rest = c.rest;
        bf16 = c.bf16 != 0;
    }
    __device__ __forceinline__ void place(const Chunk& o) { grad = o.grad; out = o.out; whole = o.whole; rest = o.rest; bf16 = o.bf16; }
    template <bool ONCE> __device__ __forceinline__ void load() {
#pragma unroll
        for (int j = 0; j < GRAD_LOADS; ++j)
            if (unit(j) < whole) v[j] = ONCE ? load_once_anywhere<Anywhere<16, 2>>(grad + unit(j) * 16) : *reinterpret_cast<const Anywhere<16, 2>*>(grad + unit(j) * 16);
            else v[j].w[0] = v[j].w[1] = v[j].w[2] = v[j].w[3] = 0;
        tail = 0.0f;
        if (has_tail()) {
            const char* p = grad + whole * 16;
            tail = bf16 ? Elem<bf16_t>::ld(reinterpret_cast<const bf16_t*>(p) + threadIdx.x) : reinterpret_cast<const float*>(p)[threadIdx.x];
        }
    }
    __device__ __forceinline__ double squares() const {
        double sum = (double)tail * (double)tail, more = 0.0;
        auto add = [](double& s, float f) { const double d = (double)f; s = fma(d, d, s); };
#pragma unroll
        for (int j = 0; j < GRAD_LOADS; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const unsigned w = v[j].w[q];
                if (bf16) {
                    add(sum, __uint_as_float(w << 16));
                    add(more, __uint_as_float(w & 0xffff0000u));
                } else {
                    add(q & 1 ? more : sum, __uint_as_float(w));
                }
            }
        return sum + more;
    }
    template <bool ONCE> __device__ __forceinline__ void store(double factor) const {
        auto times = [factor](float f) { return (float)((double)f * factor); };
        auto times_bf16 = [factor](float f) { return for_bf16((double)f * factor); };
#pragma unroll
        for (int j = 0; j < GRAD_LOADS; ++j) {
            if (unit(j) >= whole) continue;
            Anywhere<16, 2> o;
            if (bf16) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const unsigned w = v[j].w[q];
                    o.w[q] = pack_bf16x2(times_bf16(__uint_as_float(w << 16)), times_bf16(__uint_as_float(w & 0xffff0000u)));
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) o.w[q] = __float_as_uint(times(__uint_as_float(v[j].w[q])));
            }
            if (ONCE) store_once_anywhere(out + unit(j) * 16, o); else *reinterpret_cast<Anywhere<16, 2>*>(out + unit(j) * 16) = o;
        }
        if (has_tail()) {
            char* p = out + whole * 16;
            if (bf16) Elem<bf16_t>::st(reinterpret_cast<bf16_t*>(p) + threadIdx.x, times_bf16(tail));
            else reinterpret_cast<float*>(p)[threadIdx.x] = times(tail);
        }
    }
};

// over a workgroup; every thread has the sum
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < GRAD_THREADS / 64; ++w) sum += lds[w];
    return sum;
}
// The norm of the partial sums, the same bits in every workgroup.
__device__ __forceinline__ float norm_of(const double* partial, int n, double* lds) {
    constexpr int AT_ONCE = GRAD_BLOCKS / GRAD_THREADS;
    double v[AT_ONCE], sum = 0.0;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        const int at = i * GRAD_THREADS + threadIdx.x;
        v[i] = at < n ? partial[at] : 0.0;
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) sum += v[i];
    return (float)sqrt(block_sum(sum, lds));
}

__global__ __launch_bounds__(GRAD_THREADS) void grad_norm_kernel(GradArgs a) {
    __shared__ double lds[GRAD_THREADS / 64];
    double sum = 0.0;
    Chunk c;
    int number = blockIdx.x;
    c.find(a, number);
    while (number < a.chunks) {
        if (a.kept) c.load<false>(); else c.load<true>();
        const int next = number + gridDim.x;
        Chunk n;
        n.find(a, next < a.chunks ? next : number);
        sum += c.squares();
        c.place(n);
        number = next;
    }
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
}
// Few chunks: one workgroup, four of them at a time, and no second launch (three tensors of a chunk 4.5 us, 6.9 in two launches; six 5.4 and
// 6.9; nine 7.0 and 6.9; fourteen 9.5 and 7.0).  (Chunk takes its thread's number from threadIdx.x, which
// counts the threads of a chunk here; y counts the chunks.)
constexpr int GRAD_ALONE = 8, GRAD_AT_ONCE = 4;
__global__ __launch_bounds__(GRAD_THREADS * GRAD_AT_ONCE) void grad_norm_alone_kernel(GradArgs a) {
    __shared__ double lds[GRAD_AT_ONCE][GRAD_THREADS];
    const int tid = threadIdx.x, q = threadIdx.y;
    double sum = 0.0;
    for (int number = q; number < a.chunks; number += GRAD_AT_ONCE) {
        Chunk c;
        c.find(a, number);
        c.load<true>();
        sum += c.squares();
    }
    lds[q][tid] = sum;
    __syncthreads();
    sum = (lds[0][tid] + lds[1][tid]) + (lds[2][tid] + lds[3][tid]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    __shared__ double waves[GRAD_THREADS / 64];
    if (q == 0 && (tid & 63) == 0) waves[tid >> 6] = sum;
    __syncthreads();
    if (q == 0 && tid == 0) *a.norm = (float)sqrt((waves[0] + waves[1]) + (waves[2] + waves[3]));
}
// (1.7 us beside the norm's 3.6 for 14 chunks; between them, 2 us of a launch)
__global__ __launch_bounds__(GRAD_THREADS) void grad_join_kernel(GradArgs a) {
    __shared__ double lds[GRAD_THREADS / 64];
    const float norm = norm_of(a.partial, a.partials, lds);
    if (threadIdx.x == 0) *a.norm = norm;
}

// a.partials: so many partial sums are to be added up and their norm written down; 0: the norm is there.  The chunks are taken from
// the last on, which are the likeliest to be in the caches still.
__global__ __launch_bounds__(GRAD_THREADS) void grad_scale_kernel(GradArgs a) {
    __shared__ double lds[GRAD_THREADS / 64];
    Chunk c;
    int back = blockIdx.x;
    c.find(a, a.chunks - 1 - back);
    if (a.kept) c.load<false>(); else c.load<true>();
    float norm;
    if (a.partials > 0) {
        norm = norm_of(a.partial, a.partials, lds);
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
    } else {
        norm = *a.norm;
    }
    // (NaN and infinity: nothing is scaled)
    const double factor = norm > a.most && norm < __builtin_inff() ? (double)a.most / (double)norm : 1.0;
    while (true) {
        const int next = back + gridDim.x;
        Chunk n;
        n.find(a, a.chunks - 1 - (next < a.chunks ? next : back));
        if (factor != 1.0 || c.grad != c.out) {
            if (a.kept) c.store<false>(factor); else c.store<true>(factor);
        }
        if (next >= a.chunks) break;
        back = next;
        c.place(n);
        if (a.kept) c.load<false>(); else c.load<true>();
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
    *table = ((size_t)chunks + 1) * sizeof(moe::GradChunk);
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
    int first = 0, here = 0;
    moe::GradTableArgs a = {};
    for (int i = 0; i < count; ++i) {
        const long long per = moe::grad_chunk_elements(tensors[i].dtype == MOE_BF16);
        if (tensors[i].n > 0) {
            a.e[here++] = {tensors[i].grad, tensors[i].out, (long long)tensors[i].n, first, tensors[i].dtype == MOE_BF16};
            first += (int)((tensors[i].n + per - 1) / per);
            if (!tensors[i].out) l.outs = 0;
        }
        if (here == moe::GRAD_BATCH || (here > 0 && i == count - 1)) {
            moe::grad_table_kernel<<<here, 256, 0, s>>>(a, (moe::GradChunk*)table);
            MOE_CHECK_LAUNCH();
            here = 0;
        }
    }
    *list = l;
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

namespace moe {
namespace {

// The partial sums, or (few chunks: a launch less) the norm itself, *partials = 0.
moe_status grad_sums(const moe_grad_list* l, int kept, float* norm, void* scratch, hipStream_t s, GradArgs* a) {
    const int blocks = grad_blocks(l->chunks);
    *a = {(const GradChunk*)l->table, (int)l->chunks, kept, 0, (double*)scratch, norm, 0.0f};
    if (l->chunks <= GRAD_ALONE) {
        grad_norm_alone_kernel<<<1, dim3(GRAD_THREADS, GRAD_AT_ONCE), 0, s>>>(*a);
    } else {
        grad_norm_kernel<<<blocks, GRAD_THREADS, 0, s>>>(*a);
        a->partials = blocks;
    }
    MOE_CHECK_LAUNCH();
    return MOE_OK;
}

}  // namespace
}  // namespace moe

extern "C" moe_status moe_grad_norm(const moe_grad_list* list, float* norm, void* scratch, void* stream) {
    MOE_TRY(moe::grad_list_check(list));
    if (!norm || !scratch) return MOE_ERR_NULL;
    if ((uintptr_t)scratch & 7) return MOE_ERR_UNSUPPORTED;
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_GRADS, s);
        moe::GradArgs a;
        MOE_TRY(moe::grad_sums(list, 0, norm, scratch, s, &a));
        if (a.partials) {
            moe::grad_join_kernel<<<1, moe::GRAD_THREADS, 0, s>>>(a);
            MOE_CHECK_LAUNCH();
        }
    }
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

extern "C" moe_status moe_grad_scale(const moe_grad_list* list, float most, const float* norm, void* stream) {
    MOE_TRY(moe::grad_list_check(list));
    if (!(most >= 0.0f) || !std::isfinite(most)) return MOE_ERR_SHAPE;
    if (!norm || !list->outs) return MOE_ERR_NULL;
    if (list->chunks == 0) return MOE_OK;
    moe::GradArgs a = {(const moe::GradChunk*)list->table, (int)list->chunks, 0, 0, nullptr, const_cast<float*>(norm), most};
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_GRADS, s);
        moe::grad_scale_kernel<<<moe::grad_blocks(list->chunks), moe::GRAD_THREADS, 0, s>>>(a);
        MOE_CHECK_LAUNCH();
    }
    moe::count_launch(moe::LC_OTHER);
    return MOE_OK;
}

extern "C" moe_status moe_grad_clip(const moe_grad_list* list, float most, float* norm, void* scratch, void* stream) {
    MOE_TRY(moe::grad_list_check(list));
    if (!(most >= 0.0f) || !std::isfinite(most)) return MOE_ERR_SHAPE;
    if (!norm || !scratch || !list->outs) return MOE_ERR_NULL;
    if ((uintptr_t)scratch & 7) return MOE_ERR_UNSUPPORTED;
    hipStream_t s = (hipStream_t)stream;
    {
        moe::ProfScope prof(moe::PK_GRADS, s);
        moe::GradArgs a;
        MOE_TRY(moe::grad_sums(list, list->chunks <= moe::GRAD_KEPT, norm, scratch, s, &a));
        if (list->chunks > 0) {
            a.most = most;
            moe::grad_scale_kernel<<<moe::grad_blocks(list->chunks), moe::GRAD_THREADS, 0, s>>>(a);
            MOE_CHECK_LAUNCH();
        }
    }
    moe::count_launch(moe::LC_OTHER, 2);
    return MOE_OK;
}
