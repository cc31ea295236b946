// The matrix products of the orthogonalised update: C[m][n] = sum over k of A[m][k] B[n][k], or (TB) B[k][n], of operands in fp16 planes.
//
// A value x, scaled by a power of two that keeps it below 2^15, is hi + lo, hi = fp16(x), lo = fp16(x - hi): 22 bits of it and an
// absolute 2^-25 at least (the matrix instructions take subnormal numbers as they are).  Three products, hi lo, lo hi and hi hi, are summed in fp32; the
// fourth is left out: below 2^-24 of the product, of either sign.  bf16 inputs are one plane, exactly.
//
// The planes lie next to each other: 32 neighbours of a row's hi, then their lo, 128 bytes.  So a tile of 32 k of two planes is a tile of
// 64 columns of memory, and all fragments of a step are read once for its three products (as three sums over k one after the other each plane would be
// brought and read twice: 6 tiles instead of 4).
#pragma once

#include "ff_gemm.h"

namespace edgc {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct OrthoProblem {
    const uint16_t *a, *b;              // operands
    uint16_t* out;                      // planes, or
    void* to;                           // the caller's matrix
    const uint16_t* e;                  // planes like `out`'s that are added, or null
    const float* f;                     // what the sums are multiplied by, to the power `power`
    uint64_t ldto;
    uint32_t lda, ldb, ldo;             // 16-bit elements from row to row (out, e: of planes)
    uint32_t M, N;
    uint32_t rows, cols;                // of `out`, with what is padding: zeros
    uint32_t steps;                     // tiles of k
    uint32_t b_cols;                    // TB: 16-bit elements of a row of b
    uint32_t tiles_m, tiles_n, first;   // tiles of the output; first block
    uint32_t power, transposed;         // transposed: to[n][m]
    float alpha, beta, gamma;           // alpha f^power sum + beta e + gamma I
};
constexpr uint32_t kOrthoProblems = 24;
struct OrthoArgs {
    OrthoProblem p[kOrthoProblems];
    uint32_t count, tiles;
};
static_assert(sizeof(OrthoArgs) <= 4032, "kernel arguments are limited to 4 KiB");

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
// where eight neighbours' hi are in a row of planes; lo: 32 further on
__device__ __forceinline__ uint32_t ortho_at(uint32_t column) { return column / 32 * 64 + column % 32; }

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
        FfType<__bf16>::put4(reinterpret_cast<uint16_t*>(row + c), 0, a);
        FfType<__bf16>::put4(reinterpret_cast<uint16_t*>(row + c + 4), 0, b);
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
template <bool SYM, typename T>
__device__ __forceinline__ void ortho_square(const OrthoProblem& p, float factor, const f32x16& acc, float* mine, uint32_t lane, uint32_t m0, uint32_t n0,
                                             bool mirror)
{
    constexpr bool PLANES = std::is_same<T, void>::value;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(mine + (lane & 31) * kOrthoRow + 8 * q + 4 * (lane >> 5)) = float4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
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
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= factor;
            if constexpr (PLANES) {
                const uint64_t at = static_cast<uint64_t>(m) * p.ldo + ortho_at(n);
                if (SYM && p.e) {
                    const f16x8 h = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4*>(p.e + at)),
                                l = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4*>(p.e + at + 32));
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
                u32x4 hi, lo;
                ortho_planes(v, hi, lo);
                *reinterpret_cast<u32x4*>(p.out + at) = hi;
                *reinterpret_cast<u32x4*>(p.out + at + 32) = lo;
            } else {
                ortho_store8(static_cast<T*>(p.to) + m * p.ldto, n, p.N, v);
            }
        }
    }
    if (across) {
        ff_wave_sync();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t r = half * 16 + lane / 4, n = n0 + r, m = m0 + c;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = mine[(c + i) * kOrthoRow + r];
            if constexpr (PLANES) {
                if (n >= p.rows || m >= p.cols) continue;
                const uint64_t at = static_cast<uint64_t>(n) * p.ldo + ortho_at(m);
                u32x4 hi, lo;
                ortho_planes(v, hi, lo);
                *reinterpret_cast<u32x4*>(p.out + at) = hi;
                *reinterpret_cast<u32x4*>(p.out + at + 32) = lo;
            } else {
                if (n >= p.N) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= factor;
                if (m < p.M) ortho_store8(static_cast<T*>(p.to) + n * p.ldto, m, p.M, v);
            }
        }
    }
    ff_wave_sync();
}

constexpr uint32_t ortho_buffers_a(int bm) { return bm == 256 ? 3 : 2; }
template <int BM, int PA, int PB, bool TB> constexpr uint32_t kOrthoBytesB = TB ? 32u * BM * PB * 2u : BM * 128u;
template <int BM, int PA, int PB, bool TB> constexpr uint32_t kOrthoLds = ortho_buffers_a(BM) * BM * 128u + 2u * kOrthoBytesB<BM, PA, PB, TB>;

// A block of 2 x 2 waves makes a BM x BM tile of the output; PA, PB: planes of the operands.  SYM (of !TB): the output is symmetric, M = N.
template <int BM, int PA, int PB, bool TB, typename T>
__global__ __launch_bounds__(256) void k_ortho_gemm(const OrthoArgs args)
{
    constexpr bool LARGE = BM == 256, SYM = !TB;
    constexpr int I = BM / 64, BK = PA == 1 && PB == 1 ? 64 : 32, KK = BK / 16;     // squares of a wave; k of a tile; steps of 16 k
    constexpr int WIDTH = BM * PB;                                                 // TB: 16-bit elements of a tile's row of k
    constexpr int LA = BM / 32, LB = TB ? WIDTH / 64 : BM / 32;                    // a wave's loads of a tile
    constexpr int FA = I * PA, FB = I * PB, F = FA + FB, MM = I * I * (PA + PB - 1);    // fragments and products of a step
    constexpr uint32_t kBufsA = ortho_buffers_a(BM), kBytesA = BM * 128, kBytesB = kOrthoBytesB<BM, PA, PB, TB>, kAtB = kBufsA * kBytesA;
    static_assert(!TB || PA == 2, "the transposed operand is the gradient, multiplied by two planes");
    static_assert(PA == PB || PB == 1, "");
    extern __shared__ __align__(16) unsigned char lds[];        // [kBufsA][kBytesA], [2][kBytesB]
    static_assert(4 * 32 * kOrthoRow * 4 <= kAtB + 2 * kBytesB, "the waves' parts of LDS in ortho_square fit where the tiles were");

    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), wm = wave / 2, wn = wave % 2;
    const uint32_t tile = blockIdx.x;
    uint32_t pi = 0;
    while (pi + 1 < args.count && tile >= args.p[pi + 1].first) ++pi;
    const OrthoProblem& p = args.p[pi];
    uint32_t tm, tn;
    if constexpr (SYM) ortho_tile_of(tile - p.first, p.tiles_m, tm, tn);
    else ff_tile_of(tile - p.first, p.tiles_m, p.tiles_n, tm, tn);
    const uint32_t m0 = tm * BM, n0 = tn * BM;

    uint32_t oa[LA], ob[LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) oa[i] = ff_place<false, BM>(wave, lane, i, [](uint32_t r) { return r; }, p.M - 1 - m0, p.lda);
#pragma unroll
    for (int i = 0; i < LB; ++i)
        ob[i] = ff_place<TB, WIDTH>(wave, lane, i, [](uint32_t r) { return r; }, TB ? p.b_cols - 1 - n0 * PB : p.N - 1 - n0, p.ldb);
    const uint64_t b_step = TB ? static_cast<uint64_t>(BK) * p.ldb : 64;
    const uint16_t *pa = p.a + static_cast<uint64_t>(m0) * p.lda, *pb = p.b + (TB ? static_cast<uint64_t>(n0) * PB : static_cast<uint64_t>(n0) * p.ldb);
    const uint32_t base = lds_address(lds) + wave * 1024;
    auto bring_a = [&](uint32_t buf, int i) { load_to_lds(pa, oa[i], base + buf * kBytesA + i * 4096); };
    auto bring_b = [&](uint32_t buf, int i) { load_to_lds(pb, ob[i], base + kAtB + buf * kBytesB + i * 4096); };

    f32x16 acc[I][I];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < I; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    // As in k_ff_gemm: while a step of 16 k is multiplied, the fragments of the next are read (in a tile's last step, the first of the next
    // tile); the barrier before the last step ends the reads of the tile, and from there on B of the tile after the next is asked for, into
    // its place.  A, in three buffers (LARGE), is asked for in the first half of the steps.
    const FfFragments<false, BM> frag_a(lane, wm * I * 32);
    const FfFragments<TB, WIDTH> frag_b(lane, wn * I * 32 * (TB ? PB : 1));
    const uint32_t n = p.steps;
    f16x8 fa[2][FA], fb[2][FB];
    // fragment f of the step: first B's, then A's; of a square its planes one after the other
    auto read = [&](uint32_t buf_a, uint32_t buf_b, int kk, int f) {
        const int to = kk & 1;
        if (f < FB) {
            const unsigned char* const at = lds + kAtB + buf_b * kBytesB;
            fb[to][f] = __builtin_bit_cast(f16x8, TB ? frag_b.read(at, kk, f) : frag_b.read(at, f % PB * 2 + kk, f / PB));
        } else {
            fa[to][f - FB] = __builtin_bit_cast(f16x8, frag_a.read(lds + buf_a * kBytesA, (f - FB) % PA * 2 + kk, (f - FB) / PA));
        }
    };
    for (uint32_t t = 0; t < 2 && t < n; ++t) {
#pragma unroll
        for (int i = 0; i < LA; ++i) bring_a(t, i);
        pa += 64;
#pragma unroll
        for (int i = 0; i < LB; ++i) bring_b(t, i);
        pb += b_step;
    }
    if (n > 1) tile_barrier<LA + LB>();
    else tile_barrier<0>();
#pragma unroll
    for (int f = 0; f < F; ++f) read(0, 0, 0, f);
    uint32_t buf_a = 0, ask_a = kBufsA - 1;
    for (uint32_t t = 0; t < n; ++t) {
        const uint32_t buf_b = t & 1, next_buf_a = buf_a + 1 == kBufsA ? 0 : buf_a + 1;
        const bool more_a = LARGE && t + 2 < n, more_b = t + 2 < n;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (kk == KK - 1) {
                if (more_a) tile_barrier<LA>();
                else tile_barrier<0>();
            }
            const int from = kk & 1;
#pragma unroll
            for (int c = 0; c < F; ++c) {
                if (kk < KK - 1) read(buf_a, buf_b, kk + 1, c);
                else read(next_buf_a, buf_b ^ 1, 0, c);
                if (LARGE && kk < KK / 2 && more_a) {
                    constexpr int SLOTS = KK / 2 * F;
                    const int s = kk * F + c;
#pragma unroll
                    for (int i = s * LA / SLOTS; i < (s + 1) * LA / SLOTS; ++i) bring_a(ask_a, i);
                }
                if (kk == KK - 1 && more_b) {
#pragma unroll
                    for (int i = c * LB / F; i < (c + 1) * LB / F; ++i) bring_b(buf_b, i);
                    if (!LARGE)
#pragma unroll
                        for (int i = c * LA / F; i < (c + 1) * LA / F; ++i) bring_a(buf_b, i);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int m = c * MM / F; m < (c + 1) * MM / F; ++m) {
                    // the planes' products: lo hi, hi lo (of the first operand's and the second's), hi hi
                    const int which = m / (I * I), i = m % (I * I) / I, j = m % I;
                    const int qa = PA == 2 && which == 0 ? 1 : 0, qb = PB == 2 && which == 1 ? 1 : 0;
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb[from][j * PB + qb], fa[from][i * PA + qa], acc[i][j], 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (LARGE && kk == KK / 2 - 1 && more_a) pa += 64;
        }
        if (more_b) {
            pb += b_step;
            if (!LARGE) pa += 64;
        }
        buf_a = next_buf_a;
        ask_a = ask_a + 1 == kBufsA ? 0 : ask_a + 1;
    }
    tile_barrier<0>();

    float factor = p.alpha;
    for (uint32_t i = 0; i < p.power; ++i) factor *= *p.f;
    float* const mine = reinterpret_cast<float*>(lds) + wave * (32 * kOrthoRow);
    // a loop, whose code stays in the instruction cache
#pragma unroll 1
    for (int s = 0; s < I * I; ++s) {
        f32x16 v = acc[0][0];
        ff_each<I * I>([&](auto q) {
            constexpr int k = decltype(q)::value;
            if (s == k) v = acc[k / I][k % I];
        });
        const uint32_t m = m0 + (wm * I + s / I) * 32, nn = n0 + (wn * I + s % I) * 32;
        ortho_square<SYM, T>(p, factor, v, mine, lane, m, nn, SYM && tm != tn);
    }
}

}  // namespace edgc
