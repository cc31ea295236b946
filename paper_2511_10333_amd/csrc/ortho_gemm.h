// The matrix products of the orthogonalised update: C[m][n] = sum over k of A[m][k] B[n][k], or (TB) B[k][n], of operands in fp16 planes.
//
// A value x, scaled by a power of two that keeps it below 2^15, is hi + lo, hi = fp16(x), lo = fp16(x - hi): 22 bits of it and the residual's sign, and
// an absolute 2^-25 at least (the matrix instructions take subnormal numbers as they are).  Three products, lo hi, hi lo and hi hi, are summed in fp32;
// the fourth is left out: below 2^-24 of the product, of either sign.  bf16 inputs are one plane, exactly.  (bf16 planes would take three and six.)
//
// The products are segments of one sum, the small ones first.  An MFMA adds its 16 k to the sum in several roundings, so that the errors of these
// roundings, not of the planes, are what an update is off by: with the three products of every 16 k one after the other it was 3.4e-6 off for a
// block of hidden 512 and 3.7e-6 for odd matrices up to 2731, where fp32 products are 2.5e-6 and 2.2e-6.
#pragma once

#include "ff_gemm.h"

namespace edgc {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kOrthoSegs = 3;
struct OrthoProblem {
    const uint16_t *a[kOrthoSegs], *b[kOrthoSegs];      // operands, per segment (ff_sums)
    uint64_t lda, ldb;                  // elements
    uint32_t M, N;                      // of the output
    uint32_t ktiles, nseg;              // times 64 k of a segment; segments
    uint32_t tiles_m, tiles_n, first;   // tiles of the output; the first's number
    uint32_t begin;                     // the first of its steps of k among those that are shared
    uint32_t rows, cols;                // of `out`, with what is padding: zeros
    uint16_t* out;                      // the output's hi plane, its lo `plane` elements behind it; or
    void* to;                           // the caller's matrix
    const uint16_t* e;                  // planes like `out`'s that are added, or null
    const float* f;                     // what the sums are multiplied by, to the power `power`
    uint64_t ldo, plane;                // of out and e, or to
    uint32_t power, transposed;         // transposed: to[n][m]
    float alpha, beta, gamma;           // alpha f^power sum + beta e + gamma I
};
constexpr uint32_t kOrthoProblems = 20;
// Tiles are given out as in FfArgs: those of whole rounds of the compute units a block each, the others' steps of k in even shares to `workers` further
// blocks, which leave the sums of tiles that they have a part of in `part`, for k_ortho_join.  Problems may differ in their steps: the longest come first.
struct OrthoArgs {
    OrthoProblem p[kOrthoProblems];
    uint32_t count, whole, rest, workers;
    uint32_t steps;                     // of the other tiles, all together
    float* part;                        // [workers + rest][BM * BM]
};
static_assert(sizeof(OrthoArgs) <= 4032, "kernel arguments are limited to 4 KiB");

__host__ __device__ inline uint32_t ortho_share(const OrthoArgs& a, uint32_t worker) { return static_cast<uint32_t>(static_cast<uint64_t>(a.steps) * worker / a.workers); }
__device__ __forceinline__ const OrthoProblem& ortho_problem_of(const OrthoArgs& a, uint32_t tile)
{
    uint32_t i = 0;
    while (i + 1 < a.count && tile >= a.p[i + 1].first) ++i;
    return a.p[i];
}
// hi and lo of eight neighbours
__device__ __forceinline__ void ortho_planes(const float (&v)[8], u32x4& hi, u32x4& lo)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f16x2 h = {static_cast<_Float16>(v[2 * i]), static_cast<_Float16>(v[2 * i + 1])};
        const f16x2 l = {static_cast<_Float16>(v[2 * i] - static_cast<float>(h[0])), static_cast<_Float16>(v[2 * i + 1] - static_cast<float>(h[1]))};
        hi[i] = __builtin_bit_cast(uint32_t, h);
        lo[i] = __builtin_bit_cast(uint32_t, l);
    }
}
__device__ __forceinline__ void ortho_put(uint16_t* to, uint64_t plane, const float (&v)[8])
{
    u32x4 hi, lo;
    ortho_planes(v, hi, lo);
    *reinterpret_cast<u32x4*>(to) = hi;
    *reinterpret_cast<u32x4*>(to + plane) = lo;
}

// eight neighbours of a row of n columns, from column c on
__device__ __forceinline__ void ortho_store8(float* row, uint32_t c, uint32_t n, const float (&v)[8])
{
    if (c + 8 <= n) {
        put_any(row + c, Floats4{v[0], v[1], v[2], v[3]});
        put_any(row + c + 4, Floats4{v[4], v[5], v[6], v[7]});
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (c + i < n) row[c + i] = v[i];
    }
}
__device__ __forceinline__ void ortho_store8(__bf16* row, uint32_t c, uint32_t n, const float (&v)[8])
{
    if (c + 8 <= n) {
        const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
        FfType<__bf16>::store4(row + c, a);
        FfType<__bf16>::store4(row + c + 4, b);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (c + i < n) row[c + i] = static_cast<__bf16>(v[i]);
    }
}

// Tile of a symmetric output of `tiles` x `tiles`: those on and below the diagonal, in bands of kFfBand rows, column by column, each XCD's
// neighbours of each other (ff_tile_of)
__device__ __forceinline__ void ortho_tile_of(uint32_t id, uint32_t tiles, uint32_t& tm, uint32_t& tn)
{
    constexpr uint32_t B = kFfBand;
    const uint32_t total = tiles * (tiles + 1) / 2, per = total / 8, left = total % 8, xcd = id % 8, at = id / 8;
    id = xcd * per + min(xcd, left) + at;
    // band b begins after sum over the bands before it of B B b + B (B + 1) / 2
    auto begin = [](uint32_t b) { return B * B * (b * (b - 1) / 2) + B * (B + 1) / 2 * b; };
    uint32_t band = 0;
    while ((band + 1) * B < tiles && begin(band + 1) <= id) ++band;
    const uint32_t rows = min(B, tiles - band * B);
    uint32_t in = id - begin(band);
    if (in < rows * B * band) {             // left of the band's diagonal
        tm = band * B + in % rows;
        tn = in / rows;
        return;
    }
    in -= rows * B * band;
    uint32_t c = 0;
    while (in >= rows - c) in -= rows - c++;
    tm = band * B + c + in;
    tn = band * B + c;
}

// The sums of a square of 32 rows and columns, of which a lane holds row lane % 32 and columns 8 (v / 4) + 4 (lane / 32) + v % 4: through the wave's
// part of LDS, so that eight neighbours of a row are stored together, and of the square's transpose (SYM: where it is another square).
constexpr uint32_t kOrthoRow = 36;      // floats: 32 and a pad that spreads the rows over the banks
__device__ __forceinline__ void ortho_spread(float factor, const f32x16& acc, float* mine, uint32_t lane)
{
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(mine + (lane & 31) * kOrthoRow + 8 * q + 4 * (lane >> 5)) =
            float4{factor * acc[4 * q], factor * acc[4 * q + 1], factor * acc[4 * q + 2], factor * acc[4 * q + 3]};
}
template <bool SYM, typename T>
__device__ __forceinline__ void ortho_square(const OrthoProblem& p, float* mine, uint32_t lane, uint32_t m0, uint32_t n0, bool mirror)
{
    constexpr bool PLANES = std::is_same<T, void>::value;
    ff_wave_sync();
    const uint32_t c = lane % 4 * 8;
    const bool across = PLANES ? SYM && mirror : p.transposed != 0;
    if (PLANES || !across) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t r = half * 16 + lane / 4, m = m0 + r, n = n0 + c;
            if constexpr (PLANES) {
                if (m >= p.rows || n >= p.cols) continue;
            } else {
                if (m >= p.M || n >= p.N) continue;
            }
            const float4 x = *reinterpret_cast<const float4*>(mine + r * kOrthoRow + c), y = *reinterpret_cast<const float4*>(mine + r * kOrthoRow + c + 4);
            float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
            if constexpr (PLANES) {
                const uint64_t at = m * p.ldo + n;
                if (SYM && p.e) {
                    const f16x8 h = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4*>(p.e + at)),
                                l = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4*>(p.e + at + p.plane));
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) {
                        v[i] = fmaf(p.beta, static_cast<float>(h[i]) + static_cast<float>(l[i]), v[i]);
                        if (m == n + i) v[i] += p.gamma;
                    }
                }
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) v[i] = m < p.M && n + i < p.N ? v[i] : 0.f;
                if (SYM && mirror) {
                    *reinterpret_cast<float4*>(mine + r * kOrthoRow + c) = float4{v[0], v[1], v[2], v[3]};
                    *reinterpret_cast<float4*>(mine + r * kOrthoRow + c + 4) = float4{v[4], v[5], v[6], v[7]};
                }
                ortho_put(p.out + at, p.plane, v);
            } else {
                ortho_store8(static_cast<T*>(p.to) + m * p.ldo, n, p.N, v);
            }
        }
    }
    if (across) {
        ff_wave_sync();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t r = half * 16 + lane / 4, n = n0 + r, m = m0 + c;
            if constexpr (PLANES) {
                if (n >= p.rows || m >= p.cols) continue;
            } else {
                if (n >= p.N || m >= p.M) continue;
            }
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = mine[(c + i) * kOrthoRow + r];
            if constexpr (PLANES) ortho_put(p.out + n * p.ldo + m, p.plane, v);
            else ortho_store8(static_cast<T*>(p.to) + n * p.ldo, m, p.M, v);
        }
    }
    ff_wave_sync();
}

template <bool SYM>
__device__ __forceinline__ void ortho_place(const OrthoProblem& p, uint32_t tile, uint32_t& tm, uint32_t& tn)
{
    if constexpr (SYM) ortho_tile_of(tile - p.first, p.tiles_m, tm, tn);
    else ff_tile_of(tile - p.first, p.tiles_m, p.tiles_n, tm, tn);
}
__device__ __forceinline__ float ortho_factor(const OrthoProblem& p)
{
    float factor = p.alpha;
    for (uint32_t i = 0; i < p.power; ++i) factor *= *p.f;
    return factor;
}

// A block of 2 x 2 waves makes a BM x BM tile of the output.  !TB: the output is symmetric, M = N.  T: void, planes, or the caller's type.
template <int BM, bool TB, typename T>
__global__ __launch_bounds__(256) void k_ortho_gemm(const OrthoArgs args)
{
    constexpr bool SYM = !TB;
    constexpr int I = BM / 64;                                  // squares of a wave, either way
    extern __shared__ __align__(16) unsigned char lds[];        // ff_sums' tiles
    static_assert(4 * 32 * kOrthoRow * 4 <= ff_lds_bytes(BM, BM), "the waves' parts of LDS in ortho_square fit where the tiles were");

    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), wm = wave / 2, wn = wave % 2;
    const bool shares = blockIdx.x >= args.whole;
    const uint32_t worker = blockIdx.x - args.whole;
    uint32_t step = shares ? ortho_share(args, worker) : 0;
    const uint32_t steps_end = shares ? ortho_share(args, worker + 1) : 1;
    while (step < steps_end) {
        uint32_t tile = blockIdx.x, pi = 0, kt0 = 0, kt1;
        if (shares) {
            while (pi + 1 < args.count && step >= args.p[pi + 1].begin) ++pi;
        } else {
            while (pi + 1 < args.count && tile >= args.p[pi + 1].first) ++pi;
        }
        const OrthoProblem& p = args.p[pi];
        const uint32_t ksteps = p.ktiles * p.nseg;
        kt1 = ksteps;
        if (shares) {
            const uint32_t in = (step - p.begin) / ksteps;
            tile = max(p.first, args.whole) + in;
            kt0 = step - p.begin - in * ksteps;
            kt1 = min(ksteps, kt0 + (steps_end - step));
        }
        step += kt1 - kt0;
        uint32_t tm, tn;
        ortho_place<SYM>(p, tile, tm, tn);
        const uint32_t m0 = tm * BM, n0 = tn * BM;

        f32x16 acc[I][I];
        ff_sums<BM, BM, false, TB, false, true>(p, lds, lane, wave, m0, n0, kt0, kt1, acc);

        if (kt1 - kt0 == ksteps) {
            const float factor = ortho_factor(p);
            float* const mine = reinterpret_cast<float*>(lds) + wave * (32 * kOrthoRow);
            // a loop, whose code stays in the instruction cache
#pragma unroll 1
            for (int s = 0; s < I * I; ++s) {
                ff_each<I * I>([&](auto q) {
                    constexpr int k = decltype(q)::value;
                    if (s == k) ortho_spread(factor, acc[k / I][k % I], mine, lane);
                });
                ortho_square<SYM, T>(p, mine, lane, m0 + (wm * I + s / I) * 32, n0 + (wn * I + s % I) * 32, SYM && tm != tn);
            }
        } else {
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < I; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *ff_slot<BM, BM, I>(args.part, worker + tile - args.whole, i, j, q, tid) =
                            float4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        }
        if (step < steps_end) __syncthreads();      // the next tile's rows go where this one's sums were
    }
}

// Adds up the sums that several workers have of a tile, in the order of the workers: one square of every wave's part per block
template <int BM, bool TB, typename T>
__global__ __launch_bounds__(256) void k_ortho_join(const OrthoArgs args)
{
    constexpr bool SYM = !TB;
    constexpr uint32_t I = BM / 64;
    __shared__ __align__(16) float stage[4 * 32 * kOrthoRow];
    const uint32_t at = blockIdx.x / (I * I), i = blockIdx.x / I % I, j = blockIdx.x % I, tile = args.whole + at;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    const OrthoProblem& p = ortho_problem_of(args, tile);
    const uint32_t ksteps = p.ktiles * p.nseg, s0 = p.begin + (tile - max(p.first, args.whole)) * ksteps, s1 = s0 + ksteps;
    // the workers that have a step of this tile
    uint32_t first = static_cast<uint32_t>(static_cast<uint64_t>(s0) * args.workers / args.steps), last = static_cast<uint32_t>(static_cast<uint64_t>(s1 - 1) * args.workers / args.steps);
    while (ortho_share(args, first + 1) <= s0) ++first;
    while (last + 1 < args.workers && ortho_share(args, last + 1) < s1) ++last;
    if (first == last) return;                      // one, which has finished it
    f32x16 acc = {};
#pragma unroll 4
    for (uint32_t w = first; w <= last; ++w) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 v = *ff_slot<BM, BM, static_cast<int>(I)>(args.part, w + at, i, j, q, tid);
            acc[4 * q] += v.x; acc[4 * q + 1] += v.y; acc[4 * q + 2] += v.z; acc[4 * q + 3] += v.w;
        }
    }
    uint32_t tm, tn;
    ortho_place<SYM>(p, tile, tm, tn);
    float* const mine = stage + wave * (32 * kOrthoRow);
    ortho_spread(ortho_factor(p), acc, mine, lane);
    ortho_square<SYM, T>(p, mine, lane, tm * BM + (wave / 2 * I + i) * 32, tn * BM + (wave % 2 * I + j) * 32, SYM && tm != tn);
}

}  // namespace edgc
