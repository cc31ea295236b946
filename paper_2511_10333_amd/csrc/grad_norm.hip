// The global norm of a list of gradients and their clipping.
//
//   S = sum over all tensors of g^2,  norm = sqrt S,  c = min(1, max_norm / (norm + 1e-6)),  out = round(c g)
//
// Two launches: k_grad_sumsq reads the list and leaves S, k_clip reads it again and writes.  Both are bounded by memory.  Squares
// and sums are in 64 bits: fp32 squares overflow from 1.8e19 on and vanish below 1e-23, and the conversions and multiply-adds of
// 64 bits hide behind the loads.  The sums are taken in a fixed order (a thread's items, the block's threads, the blocks in the
// last one), so that the same list gives the same bits.  32 matrices of eight hidden-4096 layers, 6.4 GB of fp32: k_grad_sumsq 1.12 ms
// (5.8 TB/s), k_clip 2.50 (5.2 TB/s); the 11 bf16 tensors of a hidden-512 layer: 13 us for both.
#include "edgc_internal.h"

#include <algorithm>
#include <cmath>

namespace edgc {
namespace {

constexpr int kThreads = 256, kUnroll = 8;
constexpr uint32_t kChunk = kThreads * kUnroll;     // items of 16 bytes that a block takes at a time: 32 KB
constexpr int kMaxGrads = 64;                       // tensors per launch: their list travels in the kernel arguments
constexpr double kClipEps = 1e-6;

struct GradItem {
    const void* src;
    void* dst;
    uint64_t ld_src, ld_dst, n;     // elements; a contiguous tensor is one row of all its elements
    uint32_t m, _pad;
};
struct GradList {
    uint64_t first[kMaxGrads];      // first chunk of each tensor, ~0 beyond the last
    GradItem t[kMaxGrads];
    uint64_t chunks;
};
static_assert(sizeof(GradList) <= 3840, "kernel arguments are limited to 4 KiB");

// 16 bytes at any address that is a multiple of the element's size
typedef float f32x4_at __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t bf16x8_at __attribute__((ext_vector_type(4), aligned(2)));

template <typename T> struct Items;
template <> struct Items<float> {
    static constexpr uint32_t N = 4;
    using vec = f32x4_at;
    static __device__ __forceinline__ float get(const vec& v, int i) { return v[i]; }
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float x) { *p = x; }
    static __device__ __forceinline__ vec scaled(const vec& v, float c) { return vec{v[0] * c, v[1] * c, v[2] * c, v[3] * c}; }
};
template <> struct Items<__bf16> {
    static constexpr uint32_t N = 8;
    using vec = bf16x8_at;
    static __device__ __forceinline__ float get(const vec& v, int i) { return __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16); }
    static __device__ __forceinline__ float one(const __bf16* p) { return static_cast<float>(*p); }
    static __device__ __forceinline__ void put(__bf16* p, float x) { *p = static_cast<__bf16>(x); }
    static __device__ __forceinline__ uint32_t pair(float a, float b)
    {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), b2));
    }
    static __device__ __forceinline__ vec scaled(const vec& v, float c)
    {
        vec w;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = pair(get(v, 2 * k) * c, get(v, 2 * k + 1) * c);
        return w;
    }
};

// Tensor of a chunk: lane i of the wave holds the first chunk of tensor i
__device__ __forceinline__ uint32_t tensor_of_chunk(uint64_t chunk, uint64_t lane_first)
{
    return static_cast<uint32_t>(__popcll(__ballot(chunk >= lane_first))) - 1u;
}

// Where the items of a chunk are: item `i` of the chunk begins `col` elements into row `row` and holds `len` of them (0: none).
struct ItemAt {
    uint64_t row, col;
    uint32_t len;
};
template <uint32_t N>
struct ChunkWalk {
    uint64_t n, row0, at0, ipr;     // elements of a row; row and item in the row that the chunk begins at; items of a row
    uint32_t m;
    __device__ __forceinline__ ChunkWalk(const GradItem& t, uint64_t chunk) : n(t.n), row0(0), at0(chunk * kChunk), ipr((t.n + N - 1) / N), m(t.m)
    {
        if (m > 1) {
            row0 = at0 / ipr;
            at0 -= row0 * ipr;
        }
    }
    __device__ __forceinline__ ItemAt at(uint32_t i) const
    {
        uint64_t row = row0, it = at0 + i;
        if (m > 1) {                // rows of fewer than 2^32 elements: the item is below 2^30 + a chunk
            const uint32_t it32 = static_cast<uint32_t>(it), ipr32 = static_cast<uint32_t>(ipr), over = it32 / ipr32;
            row += over;
            it = it32 - over * ipr32;
        }
        const uint64_t col = it * N;
        const uint32_t len = row >= m || col >= n ? 0u : static_cast<uint32_t>(min(static_cast<uint64_t>(N), n - col));
        return {row, col, len};
    }
};

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
// the block's sum, in every thread of the first wave
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double s[kThreads / 64];
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x / 64] = v;
    __syncthreads();
    double t = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) t += s[w];
    return t;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_grad_sumsq(const GradList list, double* part, unsigned int* ticket, double* sumsq, int add)
{
    using I = Items<T>;
    const uint64_t lane_first = list.first[threadIdx.x & 63];
    double acc = 0.0;
    for (uint64_t c = blockIdx.x; c < list.chunks; c += gridDim.x) {
        const uint32_t ti = __builtin_amdgcn_readfirstlane(tensor_of_chunk(c, lane_first));
        const GradItem& t = list.t[ti];
        const ChunkWalk<I::N> walk(t, c - list.first[ti]);
        const T* const src = static_cast<const T*>(t.src);
        typename I::vec v[kUnroll];
        ItemAt a[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            a[u] = walk.at(threadIdx.x + u * kThreads);
            if (a[u].len == I::N) v[u] = *reinterpret_cast<const typename I::vec*>(src + a[u].row * t.ld_src + a[u].col);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (a[u].len == I::N) {
#pragma unroll
                for (uint32_t i = 0; i < I::N; ++i) {
                    const double x = I::get(v[u], i);
                    acc = __builtin_fma(x, x, acc);
                }
            } else {
                for (uint32_t i = 0; i < a[u].len; ++i) {
                    const double x = I::one(src + a[u].row * t.ld_src + a[u].col + i);
                    acc = __builtin_fma(x, x, acc);
                }
            }
        }
    }
    acc = block_sum(acc);
    // the last block to finish adds the blocks up; the partials go where every XCD sees them, so no release is needed
    __shared__ bool s_last;
    if (threadIdx.x == 0) {
        __hip_atomic_store(part + blockIdx.x, acc, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const bool last = atomicAdd(ticket, 1u) == gridDim.x - 1u;
        if (last) *ticket = 0u;
        s_last = last;
    }
    __syncthreads();
    if (!s_last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    double all = 0.0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kThreads)
        all += __hip_atomic_load(part + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    all = block_sum(all);
    if (threadIdx.x == 0) *sumsq = add ? *sumsq + all : all;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_clip(const GradList list, const double* sumsq, double max_norm, float* norm_coef)
{
    using I = Items<T>;
    // a norm that is not finite clips nothing: the caller sees it in norm_coef
    const double norm = sqrt(*sumsq);
    const float coef = isfinite(norm) ? static_cast<float>(fmin(1.0, max_norm / (norm + kClipEps))) : 1.0f;
    if (norm_coef && blockIdx.x == 0 && threadIdx.x == 0) {
        norm_coef[0] = static_cast<float>(isfinite(norm) ? fmin(norm, 3.4028234663852886e38) : norm);
        norm_coef[1] = coef;
    }
    const uint64_t lane_first = list.first[threadIdx.x & 63];
    // from the end: what k_grad_sumsq read last is in the caches
    for (uint64_t k = blockIdx.x; k < list.chunks; k += gridDim.x) {
        const uint64_t c = list.chunks - 1 - k;
        const uint32_t ti = __builtin_amdgcn_readfirstlane(tensor_of_chunk(c, lane_first));
        const GradItem& t = list.t[ti];
        if (coef == 1.0f && t.src == t.dst) continue;
        const ChunkWalk<I::N> walk(t, c - list.first[ti]);
        const T* const src = static_cast<const T*>(t.src);
        T* const dst = static_cast<T*>(t.dst);
        typename I::vec v[kUnroll];
        ItemAt a[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            a[u] = walk.at(threadIdx.x + u * kThreads);
            if (a[u].len == I::N) v[u] = *reinterpret_cast<const typename I::vec*>(src + a[u].row * t.ld_src + a[u].col);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (a[u].len == I::N) {
                *reinterpret_cast<typename I::vec*>(dst + a[u].row * t.ld_dst + a[u].col) = I::scaled(v[u], coef);
            } else {
                for (uint32_t i = 0; i < a[u].len; ++i)
                    I::put(dst + a[u].row * t.ld_dst + a[u].col + i, I::one(src + a[u].row * t.ld_src + a[u].col + i) * coef);
            }
        }
    }
}

// launches `go` over the list, at most kMaxGrads tensors at a time; go(list, blocks, first tensor of the launch, bytes read)
template <typename F>
int over_list(edgc_ctx* ctx, const edgc_tensor* tensors, uint32_t count, edgc_dtype dtype, bool with_out, F&& go)
{
    const uint32_t esz = dtype == EDGC_F32 ? 4 : 2, per = 16 / esz;
    for (uint32_t i0 = 0; i0 < count; i0 += kMaxGrads) {
        GradList list{};
        double bytes = 0.0;
        for (int k = 0; k < kMaxGrads; ++k) {
            if (i0 + k >= count) { list.first[k] = ~0ull; continue; }
            const edgc_tensor& d = tensors[i0 + k];
            GradItem& t = list.t[k];
            const bool whole = d.m == 1 || (d.ld == d.n && (!with_out || d.ld_out == d.n));
            t.src = d.grad; t.dst = with_out ? d.grad_out : nullptr;
            t.ld_src = d.ld; t.ld_dst = d.ld_out;
            t.m = whole ? 1 : d.m;
            t.n = whole ? static_cast<uint64_t>(d.m) * d.n : d.n;
            list.first[k] = list.chunks;
            list.chunks += (t.m * ((t.n + per - 1) / per) + kChunk - 1) / kChunk;
            bytes += static_cast<double>(d.m) * d.n * esz;
        }
        const uint64_t most = std::min<uint64_t>(kMaxReduceBlocks, static_cast<uint64_t>(ctx->num_cu) * 8u);
        const uint32_t blocks = static_cast<uint32_t>(std::min<uint64_t>(list.chunks, most));
        if (int rc = go(list, blocks, i0, bytes)) return rc;
    }
    return EDGC_OK;
}

}  // namespace

int check_gradients(edgc_ctx* ctx, const edgc_tensor* tensors, uint32_t count, edgc_dtype dtype, bool with_out)
{
    if (count && !tensors) return fail(ctx, EDGC_EINVAL, "null tensor list");
    if (dtype != EDGC_F32 && dtype != EDGC_BF16) return fail(ctx, EDGC_EINVAL, "unknown dtype");
    const uint32_t esz = dtype == EDGC_F32 ? 4 : 2;
    for (uint32_t i = 0; i < count; ++i) {
        const edgc_tensor& d = tensors[i];
        if (d.m == 0 || d.n == 0) return fail(ctx, EDGC_EINVAL, "empty tensor in list");
        if (!d.grad || (with_out && !d.grad_out)) return fail(ctx, EDGC_EINVAL, "null gradient pointer in list");
        if (!aligned_to(d.grad, esz) || (with_out && !aligned_to(d.grad_out, esz))) return fail(ctx, EDGC_EINVAL, "gradient misaligned in list");
        if (d.m > 1 && (d.ld < d.n || (with_out && d.ld_out < d.n))) return fail(ctx, EDGC_EINVAL, "leading dimension too small in list");
        if (d.m > 1 && (d.ld > kMaxSpan || (with_out && d.ld_out > kMaxSpan))) return fail(ctx, EDGC_EINVAL, "leading dimension over 2^40");
        if (with_out && d.grad == d.grad_out && d.m > 1 && d.ld != d.ld_out) return fail(ctx, EDGC_EINVAL, "a gradient that is written in place has one leading dimension");
    }
    return EDGC_OK;
}

}  // namespace edgc

using namespace edgc;

extern "C" int edgc_grad_sumsq_batch(edgc_ctx* ctx, const edgc_tensor* tensors, uint32_t count, edgc_dtype dtype, int accumulate,
                                     double* sumsq, void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    if (int rc = check_gradients(ctx, tensors, count, dtype, false)) return rc;
    if (sumsq && !aligned_to(sumsq, 8)) return fail(ctx, EDGC_EINVAL, "sumsq misaligned");
    double* const to = sumsq ? sumsq : ctx->s.sumsq;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    if (count == 0 && accumulate) return EDGC_OK;
    if (count == 0) {                                   // one block that finds no chunk: the sum of nothing
        GradList none{};
        for (uint64_t& f : none.first) f = ~0ull;
        EDGC_LAUNCH(ctx, st, KID_SUMSQ, 0.0, 0.0, k_grad_sumsq<float><<<1, kThreads, 0, st>>>(none, ctx->s.sumsq_part, ctx->s.sumsq_ticket, to, 0));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        return EDGC_OK;
    }
    return over_list(ctx, tensors, count, dtype, false, [&](const GradList& list, uint32_t blocks, uint32_t i0, double bytes) -> int {
        const int add = accumulate || i0 > 0;
        EDGC_LAUNCH(ctx, st, KID_SUMSQ, bytes, 0.0,
                    dtype == EDGC_F32
                        ? k_grad_sumsq<float><<<blocks, kThreads, 0, st>>>(list, ctx->s.sumsq_part, ctx->s.sumsq_ticket, to, add)
                        : k_grad_sumsq<__bf16><<<blocks, kThreads, 0, st>>>(list, ctx->s.sumsq_part, ctx->s.sumsq_ticket, to, add));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        return EDGC_OK;
    });
}

extern "C" int edgc_clip_batch(edgc_ctx* ctx, const edgc_tensor* tensors, uint32_t count, edgc_dtype dtype, double max_norm,
                               const double* sumsq, float* norm_coef, void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    if (int rc = check_gradients(ctx, tensors, count, dtype, true)) return rc;
    if (!(max_norm > 0.0) || !std::isfinite(max_norm)) return fail(ctx, EDGC_EINVAL, "max_norm must be positive and finite");
    if (sumsq && !aligned_to(sumsq, 8)) return fail(ctx, EDGC_EINVAL, "sumsq misaligned");
    if (norm_coef && !aligned_to(norm_coef, 4)) return fail(ctx, EDGC_EINVAL, "norm_coef misaligned");
    const double* const from = sumsq ? sumsq : ctx->s.sumsq;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    if (count == 0 && norm_coef) {
        GradList none{};
        for (uint64_t& f : none.first) f = ~0ull;
        EDGC_LAUNCH(ctx, st, KID_CLIP, 0.0, 0.0, k_clip<float><<<1, kThreads, 0, st>>>(none, from, max_norm, norm_coef));
        EDGC_HIP_TRY(ctx, hipGetLastError());
    }
    return over_list(ctx, tensors, count, dtype, true, [&](const GradList& list, uint32_t blocks, uint32_t i0, double bytes) -> int {
        (void)i0;
        EDGC_LAUNCH(ctx, st, KID_CLIP, 2.0 * bytes, 0.0,
                    dtype == EDGC_F32 ? k_clip<float><<<blocks, kThreads, 0, st>>>(list, from, max_norm, norm_coef)
                                      : k_clip<__bf16><<<blocks, kThreads, 0, st>>>(list, from, max_norm, norm_coef));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        return EDGC_OK;
    });
}
