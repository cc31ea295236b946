// The feed-forward block's forward products for few tokens: bounded by reading the weights once.
//
// A wave has 16 rows of a weight matrix (gated: of both projections) and all tokens, in groups of 16, and a share of k; the
// waves of a block share k and are added up in LDS, in their order.  Where that makes too few waves for the memory, several blocks
// (gridDim.y) share k, and the last of them to finish adds their sums up, in their order too.  The weights go from memory to the matrix
// instructions' registers as they lie there, whatever their alignment: a lane brings 16 bytes of a row, 64 bytes of each row per load.
// bf16: 16 x 16 x 32.  fp32: 16 x 16 x 4 in fp32, four for the four values of a lane; any order of k will do that both operands have.
//
// Weights from memory, both launches: one token, 403 MB of bf16, 78 to 82 us (5.0 TB/s), 16 tokens 103, 32 133; 201 MB of fp32, one
// token 44, 24 tokens 69.  What more tokens cost is x on its way into every compute unit: together with the weights 6 to 6.7 TB/s.
// (Its rows at other strides, its loads behind all of the weights', four steps on their way instead of two: the same.)
#pragma once

#include "ff_gemm.h"

namespace edgc {

// Measured, weights from memory, these kernels / the products of ff_gemm.h, in us: bf16, 32 tokens, 1024 x 4096 18 / 35, 704 x 6026 29 / 45,
// 2048 x 8192 41 / 49, 8192 x 2048 43 / 51, 4096 x 16384 133 / 121 (24 tokens 120 / 121), 5120 x 20480 278 / 171 (16 tokens 202 / 168);
// fp32, 64 tokens, 997 x 2731 43 / 71, 2048 x 8192 113 / 225, 4096 x 16384 401 / 829.  The limit is right for matrices
// of up to 2^24 elements; of larger ones in bf16 the two cross at fewer tokens (x is fetched again for every 16 rows), which it does not know.
template <typename T> constexpr uint32_t kFfFewTokens = sizeof(T) == 4 ? 64 : 32;
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct FfFewArgs {
    const void *x, *w, *w2;     // tokens x K, N x K (gated: and the second)
    uint64_t ldx, ldw, ldw2;
    uint32_t tokens, N, K;
    int32_t act;
    void* out;                  // tokens x N
    uint64_t ldo;
    void *keep, *keep2;         // gated: the projections, or null
    uint64_t ldk;
    float* part;                // [gridDim.y][gridDim.x][MATS * GROUPS][64][4], where several blocks share k
    unsigned int* tickets;      // [gridDim.x], zero between calls
};
constexpr uint32_t kFfFewBlocks = 4096, kFfFewSplits = 4;      // gridDim.x and .y of such a launch are at most these

template <typename T> struct FfFew;
template <> struct FfFew<__bf16> {
    static constexpr uint32_t kStep = 32, kLane = 8;        // k of a step, of a lane
    using reg = bf16x8;
    static __device__ __forceinline__ reg load(const __bf16* p)
    {
        typedef uint32_t any4 __attribute__((ext_vector_type(4), aligned(2)));
        return __builtin_bit_cast(reg, static_cast<u32x4>(*reinterpret_cast<const any4*>(p)));
    }
    static __device__ __forceinline__ f32x4 mma(const reg& a, const reg& b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct FfFew<float> {
    static constexpr uint32_t kStep = 16, kLane = 4;
    using reg = f32x4;
    static __device__ __forceinline__ reg load(const float* p)
    {
        typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
        return static_cast<reg>(*reinterpret_cast<const any4*>(p));
    }
    static __device__ __forceinline__ f32x4 mma(const reg& a, const reg& b, f32x4 c)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// Waves of a block at most: with four groups of tokens a wave takes over 128 registers
template <int GROUPS> constexpr uint32_t kFfFewWaves = GROUPS == 4 ? 8 : 16;

// GROUPS: of 16 tokens
template <typename T, int GROUPS, bool GATED>
__global__ __launch_bounds__(64 * kFfFewWaves<GROUPS>) void k_ff_few(const FfFewArgs a)
{
    using F = FfFew<T>;
    constexpr int MATS = GATED ? 2 : 1, UNROLL = MATS + GROUPS <= 3 ? 4 : 2;
    extern __shared__ __align__(16) float red[];            // [waves][MATS * GROUPS][64 lanes][4]
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, waves = blockDim.x / 64, r = lane % 16, h = lane / 16;
    const uint32_t n0 = blockIdx.x * 16, row = min(n0 + r, a.N - 1);
    const uint32_t whole = a.K / F::kStep, steps = (a.K + F::kStep - 1) / F::kStep;
    const uint32_t part = blockIdx.y * waves + wave, parts = gridDim.y * waves;
    const uint32_t s0 = static_cast<uint32_t>(static_cast<uint64_t>(steps) * part / parts), s1 = static_cast<uint32_t>(static_cast<uint64_t>(steps) * (part + 1) / parts);
    const T* w[MATS];
    w[0] = static_cast<const T*>(a.w) + row * a.ldw + h * F::kLane;
    if constexpr (GATED) w[1] = static_cast<const T*>(a.w2) + row * a.ldw2 + h * F::kLane;
    const T* x[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) x[g] = static_cast<const T*>(a.x) + min(g * 16 + r, a.tokens - 1) * a.ldx + h * F::kLane;

    f32x4 acc[MATS][GROUPS] = {};
    // the loads of UNROLL steps are on their way while those before are multiplied
    typename F::reg rw[2][UNROLL][MATS], rx[2][UNROLL][GROUPS];
    auto ask = [&](auto to, uint32_t step) {
        constexpr int b = decltype(to)::value;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
            for (int m = 0; m < MATS; ++m) rw[b][u][m] = F::load(w[m] + (step + u) * static_cast<uint64_t>(F::kStep));
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) rx[b][u][g] = F::load(x[g] + (step + u) * static_cast<uint64_t>(F::kStep));
        }
    };
    auto multiply = [&](auto from) {
        constexpr int b = decltype(from)::value;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int m = 0; m < MATS; ++m)
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) acc[m][g] = F::mma(rw[b][u][m], rx[b][u][g], acc[m][g]);
    };
    using std::integral_constant;
    constexpr integral_constant<int, 0> even;
    constexpr integral_constant<int, 1> odd;
    uint32_t s = s0;
    const uint32_t whole_end = min(s1, whole);
    if (s + UNROLL <= whole_end) {
        ask(even, s);
        for (; s + 3 * UNROLL <= whole_end; s += 2 * UNROLL) {
            ask(odd, s + UNROLL);
            multiply(even);
            ask(even, s + 2 * UNROLL);
            multiply(odd);
        }
        if (s + 2 * UNROLL <= whole_end) {
            ask(odd, s + UNROLL);
            multiply(even);
            multiply(odd);
            s += 2 * UNROLL;
        } else {
            multiply(even);
            s += UNROLL;
        }
    }
    for (; s < s1; ++s) {
        const uint64_t at = s * static_cast<uint64_t>(F::kStep);
        auto part = [&](const T* p) {                       // what of the step's k there is, zeros beyond
            typename F::reg v = {};
            if (s < whole) return F::load(p + at);
#pragma unroll
            for (uint32_t e = 0; e < F::kLane; ++e)
                if (at + h * F::kLane + e < a.K) v[e] = p[at + e];
            return v;
        };
        typename F::reg rw[MATS];
#pragma unroll
        for (int m = 0; m < MATS; ++m) rw[m] = part(w[m]);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const typename F::reg rx = part(x[g]);
#pragma unroll
            for (int m = 0; m < MATS; ++m) acc[m][g] = F::mma(rw[m], rx, acc[m][g]);
        }
    }
#pragma unroll
    for (int m = 0; m < MATS; ++m)
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) *reinterpret_cast<f32x4*>(red + (((wave * MATS + m) * GROUPS + g) * 64 + lane) * 4) = acc[m][g];
    __syncthreads();
    // a thread: four neighbouring rows of the weights (columns of the output) of one token
    const uint32_t g = threadIdx.x / 64;
    f32x4 sum[MATS] = {};
    if (g < GROUPS)
        for (uint32_t k = 0; k < waves; ++k)
#pragma unroll
            for (int m = 0; m < MATS; ++m) sum[m] += *reinterpret_cast<const f32x4*>(red + (((k * MATS + m) * GROUPS + g) * 64 + lane) * 4);
    if (gridDim.y > 1) {
        // Stores and loads that take effect where every XCD sees them, and neither a release nor an acquire: those write an L2 back
        // and empty caches that the other blocks' x is in (512 blocks, four sharing k: 30.6 us with an acquire, 22.2 without).
        __shared__ bool s_last;
        auto at = [&](uint32_t split, int m) {
            return a.part + (((static_cast<uint64_t>(split) * gridDim.x + blockIdx.x) * MATS + m) * GROUPS + g) * 256 + lane * 4;
        };
        if (g < GROUPS)
#pragma unroll
            for (int m = 0; m < MATS; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) __hip_atomic_store(at(blockIdx.y, m) + e, sum[m][e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
            const bool last = atomicAdd(a.tickets + blockIdx.x, 1u) == gridDim.y - 1u;
            if (last) a.tickets[blockIdx.x] = 0u;
            s_last = last;
        }
        __syncthreads();
        if (!s_last) return;
        asm volatile("" ::: "memory");
        if (g < GROUPS)
#pragma unroll
            for (int m = 0; m < MATS; ++m) {
                f32x4 v[kFfFewSplits], all = {};
#pragma unroll
                for (uint32_t k = 0; k < kFfFewSplits; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[k][e] = k < gridDim.y ? __hip_atomic_load(at(k, m) + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.f;
#pragma unroll
                for (uint32_t k = 0; k < kFfFewSplits; ++k) all += v[k];
                sum[m] = all;
            }
    }
    if (g >= GROUPS) return;
    const uint32_t t = g * 16 + r, n = n0 + h * 4;
    if (t >= a.tokens || n >= a.N) return;
    float v[4] = {sum[0][0], sum[0][1], sum[0][2], sum[0][3]};
    if constexpr (GATED) {
        const float u[4] = {sum[1][0], sum[1][1], sum[1][2], sum[1][3]};
        if (a.keep) {
            ff_store4<T, false>(static_cast<T*>(a.keep) + t * a.ldk, n, a.N, v);
            ff_store4<T, false>(static_cast<T*>(a.keep2) + t * a.ldk, n, a.N, u);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float f, df;
            ff_act(a.act, v[e], f, df);
            v[e] = f * u[e];
        }
    }
    ff_store4<T, false>(static_cast<T*>(a.out) + t * a.ldo, n, a.N, v);
}

}  // namespace edgc
