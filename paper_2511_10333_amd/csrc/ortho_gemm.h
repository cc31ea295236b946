// The matrix products of the orthogonalised update: C[m][n] = sum over k of A[m][k] B[n][k], or (TB) B[k][n], of operands in fp16 planes.
//
// A value x, scaled by a power of two that keeps it below 2^15, is hi + lo, hi = fp16(x), lo = fp16(x - hi): 22 bits of it and the residual's sign, and
// an absolute 2^-25 at least (the matrix instructions take subnormal numbers as they are).  Three products, lo hi, hi lo and hi hi, are summed in fp32;
// the fourth is left out: below 2^-24 of the product, of either sign.  bf16 inputs are one plane: all bits of those above 2^-17,
// beside a matrix's norm of 2^14.  (bf16 planes would take three and six.)
//
// The planes lie next to each other: 32 neighbours of a row's hi, then their lo, 128 bytes.  A tile of 32 k of both is 64 columns of memory, and a
// step's fragments are read from LDS once for its three products.  (As three sums over k, with each plane brought and read twice, a hidden-2048 block took
// 4.64 ms instead of 3.80 at the time.)
//
// The two small products have a sum of their own.  An MFMA adds its 16 k to the sum in several roundings, and the errors of these, not of the planes, are
// what an update is off by: with all three products in one sum and X formed again after two steps, then three, it was 3.4e-6 off for a block of hidden 512 and
// 3.7e-6 for odd matrices up to 2731, where fp32 products are 2.5e-6 and 2.2e-6; with two sums 1.6e-6 and 1.8e-6, and with an X every two steps
// 1.2e-6 and 0.9e-6.  (Sums that begin anew with every tile of k took a hidden-2048 block from 3.45 to 5.25 ms, for errors a quarter to a half smaller.)
#pragma once

#include "ff_gemm.h"
#include "ortho_tiles.h"

namespace edgc {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// X = G / (|G| + eps) is as much smaller than one as eps is larger than the norm, and so are all later ones.  rho = |G| / (|G| + eps) < 2^exponent.  The first
// X is 2^exponent value times the planes.  A later one, which is at most 2^reach times rho beside what its planes are scaled for, is held 2^-min(0,
// exponent + reach) times larger.
struct OrthoFactor {
    float value;
    int32_t exponent;
};
constexpr int32_t kOrthoFirst = INT32_MIN, kOrthoPlain = INT32_MAX;     // in the place of a reach: of the first X; of what is not scaled

struct OrthoProblem {
    const uint16_t *a, *b;              // operands
    uint64_t lda, ldb;                  // 16-bit elements from row to row
    uint32_t M, N;                      // of the output
    uint32_t ktiles;                    // tiles of k
    uint32_t tiles_m, tiles_n;          // tiles of the output
    uint32_t rows, cols;                // of `out`, with what is padding: zeros
    int32_t from;                       // see OrthoFactor
    uint16_t* out;                      // planes, or
    void* to;                           // the caller's matrix
    const uint16_t* e;                  // planes like `out`'s that are added, or null
    const OrthoFactor* f;               // of X, or null
    uint64_t ldo;                       // of out and e (16-bit elements), or to
    uint32_t power, transposed;         // how often X is in the product; transposed: to[n][m]
    float alpha, beta, gamma;           // alpha (X's factor)^power sum + beta e + gamma I; to: beta alpha (X's factor)^power sum
    int32_t into;                       // of an X that is written, or kOrthoPlain
};
constexpr uint32_t kOrthoProblems = 20;
// Tiles are given out as in FfArgs: those of whole rounds of the compute units a block each, the others' steps of k in even shares to `workers` further
// blocks, which leave the sums of tiles that they have a part of in `part`, for k_ortho_join.  Problems may differ in their steps: the longest come first.
struct OrthoArgs {
    uint32_t whole, rest, workers;
    uint32_t steps;                     // of the other tiles, all together
    float* part;                        // [workers + rest][BM * BM]
    // A problem's first tile, and the first of its steps of k that are shared: next to each other, for ortho_problem_of.  Of problems that are not there, the
    // largest number.
    uint32_t first[kOrthoProblems], begin[kOrthoProblems];
    uint32_t count;
    OrthoProblem p[kOrthoProblems];
};
static_assert(sizeof(OrthoArgs) <= 4032, "kernel arguments are limited to 4 KiB");

__host__ __device__ inline uint32_t ortho_share(const OrthoArgs& a, uint32_t worker) { return static_cast<uint32_t>(static_cast<uint64_t>(a.steps) * worker / a.workers); }
// The problem that tile (or step) `at` is of.  (All numbers are loaded at once: one after the other, each with its problem, they were waited for in turn.)
__device__ __forceinline__ uint32_t ortho_problem_of(const uint32_t (&first)[kOrthoProblems], uint32_t at)
{
    uint32_t i = 0;
#pragma unroll
    for (uint32_t k = 1; k < kOrthoProblems; ++k) i += at >= first[k];
    return __builtin_amdgcn_readfirstlane(i);
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
// where eight neighbours' hi are in a row of planes; lo: 32 further on
__device__ __forceinline__ uint32_t ortho_at(uint32_t column) { return column / 32 * 64 + column % 32; }
__device__ __forceinline__ void ortho_put(uint16_t* row, uint32_t column, const float (&v)[8])
{
    u32x4 hi, lo;
    ortho_planes(v, hi, lo);
    uint16_t* const to = row + ortho_at(column);
    *reinterpret_cast<u32x4*>(to) = hi;
    *reinterpret_cast<u32x4*>(to + 32) = lo;
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

// The sums of a square of 32 rows and columns, of which a lane holds row lane % 32 and columns 8 (v / 4) + 4 (lane / 32) + v % 4: through the wave's
// part of LDS, so that eight neighbours of a row are stored together.  SYM: a square below the diagonal is stored as its transpose above it too, and one
// above it not at all.
constexpr uint32_t kOrthoRow = 36;      // floats: 32 and a pad that spreads the rows over the banks
template <typename T>
__device__ __forceinline__ void ortho_spread(float factor, float scale, const f32x16& acc, float* mine, uint32_t lane)
{
    // the caller's scale by itself: the smallest ones would lose bits beside a factor of 2^-27
    auto times = [&](float v) { return std::is_same<T, void>::value ? factor * v : factor * v * scale; };
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(mine + (lane & 31) * kOrthoRow + 8 * q + 4 * (lane >> 5)) =
            float4{times(acc[4 * q]), times(acc[4 * q + 1]), times(acc[4 * q + 2]), times(acc[4 * q + 3])};
}
// alpha times the sums of a square, and what is added to them, still in the order of the registers: a loop of squares whose stores are on their way must
// not load anything, or each waits for the last one's stores
__device__ __forceinline__ void ortho_add(const OrthoProblem& p, float factor, f32x16& acc, uint32_t lane, uint32_t m0, uint32_t n0)
{
    const uint32_t m = m0 + lane % 32;
    const uint16_t* const row = p.e + min(m, p.rows - 1) * p.ldo;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t n = n0 + 8 * q + 4 * (lane / 32);
        const uint16_t* const from = row + ortho_at(min(n, p.cols - 4));
        const f16x4 h = *reinterpret_cast<const f16x4*>(from), l = *reinterpret_cast<const f16x4*>(from + 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v = fmaf(p.beta, static_cast<float>(h[i]) + static_cast<float>(l[i]), factor * acc[4 * q + i]);
            acc[4 * q + i] = m == n + i ? v + p.gamma : v;
        }
    }
}
template <bool SYM, typename T>
__device__ __forceinline__ void ortho_square(const OrthoProblem& p, float* mine, uint32_t lane, uint32_t m0, uint32_t n0)
{
    constexpr bool PLANES = std::is_same<T, void>::value;
    const bool mirror = SYM && m0 != n0;
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
                if (m0 + 32 > p.M || n0 + 32 > p.N) {
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) v[i] = m < p.M && n + i < p.N ? v[i] : 0.f;
                    if (SYM && mirror) {
                        *reinterpret_cast<float4*>(mine + r * kOrthoRow + c) = float4{v[0], v[1], v[2], v[3]};
                        *reinterpret_cast<float4*>(mine + r * kOrthoRow + c + 4) = float4{v[4], v[5], v[6], v[7]};
                    }
                }
                ortho_put(p.out + m * p.ldo, n, v);
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
            if constexpr (PLANES) ortho_put(p.out + n * p.ldo, m, v);
            else ortho_store8(static_cast<T*>(p.to) + n * p.ldo, m, p.M, v);
        }
    }
    ff_wave_sync();
}

template <bool SYM>
__device__ __forceinline__ void ortho_place(const OrthoProblem& p, uint32_t tile, uint32_t& tm, uint32_t& tn)
{
    if constexpr (SYM) ortho_tile_of(tile, p.tiles_m, tm, tn);
    else ff_tile_of(tile, p.tiles_m, p.tiles_n, tm, tn);
}
__device__ __forceinline__ float ortho_factor(const OrthoProblem& p)
{
    if (!p.f) return p.alpha;
    const OrthoFactor f = *p.f;
    const bool first = p.from == kOrthoFirst;
    auto held = [&](int32_t reach) { return reach == kOrthoPlain ? 0 : min(0, f.exponent + reach); };
    float factor = p.alpha;
    if (first)
        for (uint32_t i = 0; i < p.power; ++i) factor *= f.value;
    return ldexpf(factor, static_cast<int>(p.power) * (first ? f.exponent : held(p.from)) - held(p.into));
}

// k of a tile, bytes of either operand's tile in LDS, tiles of A and B that are there, all of LDS.  Blocks of 256 rows have a compute unit for themselves, of the
// others two share it.  A tile of 64 x 64 is multiplied in a fraction of the time that the next takes to come: four are on their way.
template <int PA, int PB> constexpr int kOrthoK = PA == 1 && PB == 1 ? 64 : 32;
template <int BM, int PB, bool TB> constexpr uint32_t kOrthoBytesB = TB ? 32u * BM * PB * 2u : BM * 128u;
template <int BM> constexpr uint32_t kOrthoTilesA = BM == 256 ? 3u : BM == 128 ? 2u : 5u;
template <int BM> constexpr uint32_t kOrthoTilesB = BM == 64 ? 5u : 2u;
template <int BM, int PB, bool TB> constexpr uint32_t kOrthoLds = kOrthoTilesA<BM> * BM * 128u + kOrthoTilesB<BM> * kOrthoBytesB<BM, PB, TB>;

// The sums of a tile over tiles kt0 to kt1 of k, by 2 x 2 waves: of a wave, I x J squares of 32 x 32.  The loop of ff_gemm.h: while a step of 16 k is
// multiplied, the fragments of the next are read (in a tile's last step, the first of the next tile); the barrier before the last step ends the reads of the
// tile, and from there on B of the tile after the next is asked for, into its place.  A, in three buffers (LARGE), is asked for in the first half of
// the steps: the barrier of tile t finds tile t + 1 there, after which A of tile t + 2 alone was asked for.  (Smaller blocks ask for both operands there, as many
// tiles ahead as they have buffers.)
template <int BM, int PA, int PB, bool TB>
__device__ __forceinline__ void ortho_sums(const OrthoProblem& p, unsigned char* lds, uint32_t lane, uint32_t wave, uint32_t m0, uint32_t n0, uint32_t kt0, uint32_t kt1,
                                           f32x16 (&acc)[BM / 64][BM / 64])
{
    constexpr bool LARGE = BM == 256, SMALL = PA + PB > 2;                          // SMALL: there are small products
    constexpr int I = BM / 64, J = BM / 64, BK = kOrthoK<PA, PB>, KK = BK / 16;     // squares of a wave; k of a tile; steps of 16 k
    constexpr int WIDTH = BM * PB;                                                 // TB: elements of a tile's row of k
    constexpr int LA = BM / 32, LB = TB ? WIDTH / 64 : BM / 32;                    // a wave's loads of a tile
    constexpr int FA = I * PA, FB = J * PB, F = FA + FB, MM = I * J * (PA + PB - 1);    // fragments and products of a step
    // lds: [kBufsA][kBytesA], [kBufsB][kBytesB]
    constexpr uint32_t kBufsA = kOrthoTilesA<BM>, kBufsB = kOrthoTilesB<BM>, kBytesA = BM * 128, kBytesB = kOrthoBytesB<BM, PB, TB>, kAtB = kBufsA * kBytesA;
    constexpr uint32_t AHEAD = kBufsB;                  // tiles
    static_assert(!TB || PA == 2, "the transposed operand is the gradient, multiplied by two planes");
    static_assert(PA == PB || (PB == 1 && TB), "");
    const uint32_t wm = wave / 2, wn = wave % 2;

    // Bytes from the tile's first element to the units of 16 that this thread brings (ff_place).
    uint32_t oa[LA], ob[LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) oa[i] = ff_place<false, BM>(wave, lane, i, [](uint32_t r) { return r; }, p.M - 1 - m0, static_cast<uint32_t>(p.lda));
#pragma unroll
    for (int i = 0; i < LB; ++i)
        ob[i] = ff_place<TB, WIDTH>(wave, lane, i, [](uint32_t r) { return r; }, TB ? static_cast<uint32_t>(p.ldb) - 1 - n0 * PB : p.N - 1 - n0, static_cast<uint32_t>(p.ldb));
    const uint64_t a_step = 64, b_step = TB ? BK * p.ldb : a_step;
    const uint16_t *pa = p.a + m0 * p.lda + kt0 * a_step, *pb = p.b + (TB ? static_cast<uint64_t>(n0) * PB : n0 * p.ldb) + kt0 * b_step;
    const uint32_t base = lds_address(lds) + wave * 1024;
    auto bring_a = [&](uint32_t buf, int i) { load_to_lds(pa, oa[i], base + buf * kBytesA + i * 4096); };
    auto bring_b = [&](uint32_t buf, int i) { load_to_lds(pb, ob[i], base + kAtB + buf * kBytesB + i * 4096); };

    f32x16 small[SMALL ? I : 1][SMALL ? J : 1];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                acc[i][j][v] = 0.f;
                if constexpr (SMALL) small[i][j][v] = 0.f;
            }

    const FfFragments<false, BM> frag_a(lane, wm * I * 32);
    const FfFragments<TB, WIDTH> frag_b(lane, wn * J * 32 * (TB ? PB : 1));
    const uint32_t n = kt1 - kt0;
    f16x8 fa[2][FA], fb[2][FB];
    // fragment f of a step: first B's, then A's; of a square its planes one after the other
    auto read = [&](uint32_t buf_a, uint32_t buf_b, int kk, int f) {
        const int to = kk & 1;
        if (f < FB) {
            const unsigned char* const at = lds + kAtB + buf_b * kBytesB;
            fb[to][f] = __builtin_bit_cast(f16x8, TB ? frag_b.read(at, kk, f) : frag_b.read(at, f % PB * 2 + kk, f / PB));
        } else {
            fa[to][f - FB] = __builtin_bit_cast(f16x8, frag_a.read(lds + buf_a * kBytesA, (f - FB) % PA * 2 + kk, (f - FB) / PA));
        }
    };
    for (uint32_t t = 0; t < AHEAD && t < n; ++t) {
#pragma unroll
        for (int i = 0; i < LA; ++i) bring_a(t, i);
        pa += a_step;
#pragma unroll
        for (int i = 0; i < LB; ++i) bring_b(t, i);
        pb += b_step;
    }
    if (n >= AHEAD) tile_barrier<(AHEAD - 1) * (LA + LB)>();
    else tile_barrier<0>();
#pragma unroll
    for (int f = 0; f < F; ++f) read(0, 0, 0, f);
    uint32_t buf_a = 0, buf_b = 0, ask_a = kBufsA - 1;      // buffers of this tile's operands; LARGE: of the A asked for next
    for (uint32_t t = 0; t < n; ++t) {
        const uint32_t next_buf_a = buf_a + 1 == kBufsA ? 0 : buf_a + 1, next_buf_b = buf_b + 1 == kBufsB ? 0 : buf_b + 1;
        const bool more_a = LARGE && t + AHEAD < n, more_b = t + AHEAD < n;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (kk == KK - 1) {                             // tile t + 1 has to be there; what may be on its way still
                if (LARGE && more_a) tile_barrier<LA>();
                else if (!LARGE && AHEAD > 2 && t + AHEAD <= n) tile_barrier<(AHEAD - 2) * (LA + LB)>();
                else tile_barrier<0>();
            }
            const int from = kk & 1;
#pragma unroll
            for (int c = 0; c < F; ++c) {
                if (kk < KK - 1) read(buf_a, buf_b, kk + 1, c);
                else read(next_buf_a, next_buf_b, 0, c);
                if (LARGE && kk < KK / 2 && more_a) {
                    constexpr int SLOTS = KK / 2 * F;
#pragma unroll
                    for (int i = (kk * F + c) * LA / SLOTS; i < (kk * F + c + 1) * LA / SLOTS; ++i) bring_a(ask_a, i);
                }
                if (kk == KK - 1 && more_b) {
#pragma unroll
                    for (int i = c * LB / F; i < (c + 1) * LB / F; ++i) bring_b(buf_b, i);
                    if constexpr (!LARGE) {
#pragma unroll
                        for (int i = c * LA / F; i < (c + 1) * LA / F; ++i) bring_a(buf_a, i);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                // the products of the planes: lo hi, hi lo (of the first operand's and the second's), hi hi
#pragma unroll
                for (int m = c * MM / F; m < (c + 1) * MM / F; ++m) {
                    const int which = m / (I * J), i = m % (I * J) / J, j = m % J;
                    const int qa = PA == 2 && which == 0 ? 1 : 0, qb = PB == 2 && which == 1 ? 1 : 0;
                    f32x16& sum = SMALL && which < PA + PB - 2 ? small[SMALL ? i : 0][SMALL ? j : 0] : acc[i][j];
                    sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb[from][j * PB + qb], fa[from][i * PA + qa], sum, 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (LARGE && kk == KK / 2 - 1 && more_a) pa += a_step;
        }
        if (more_b) {
            pb += b_step;
            if (!LARGE) pa += a_step;
        }
        buf_a = next_buf_a;
        buf_b = next_buf_b;
        ask_a = ask_a + 1 == kBufsA ? 0 : ask_a + 1;
    }
    tile_barrier<0>();
    if constexpr (SMALL) {
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) acc[i][j] += small[i][j];
    }
}

// Where a worker leaves the sums of a tile: in the order of its registers
template <int BM>
__device__ __forceinline__ float4* ortho_slot(float* part, uint32_t slot, uint32_t i, uint32_t j, uint32_t q, uint32_t tid)
{
    return ff_slot<BM, BM, BM / 64>(part, slot, i, j, q, tid);
}

// A block of 2 x 2 waves makes a BM x BM tile of the output; PA, PB: planes of the operands.  !TB: the output is symmetric, M = N.  T: void, planes, or
// the caller's type.
template <int BM, int PA, int PB, bool TB, typename T>
__global__ __launch_bounds__(256, BM == 256 ? 1 : 2) void k_ortho_gemm(const OrthoArgs args)
{
    constexpr bool SYM = !TB;
    constexpr int I = BM / 64, J = BM / 64;
    extern __shared__ __align__(16) unsigned char lds[];        // ortho_sums' tiles
    static_assert(4 * 32 * kOrthoRow * 4 <= kOrthoLds<BM, PB, TB>, "the waves' parts of LDS in ortho_square fit where the tiles were");

    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), wm = wave / 2, wn = wave % 2;
    const bool shares = blockIdx.x >= args.whole;
    const uint32_t worker = blockIdx.x - args.whole;
    uint32_t step = shares ? ortho_share(args, worker) : 0;
    const uint32_t steps_end = shares ? ortho_share(args, worker + 1) : 1;
    while (step < steps_end) {
        const uint32_t pi = shares ? ortho_problem_of(args.begin, step) : ortho_problem_of(args.first, blockIdx.x);
        const OrthoProblem& p = args.p[pi];
        uint32_t tile = blockIdx.x, kt0 = 0, kt1 = p.ktiles;
        if (shares) {
            const uint32_t from = step - args.begin[pi], in = from / p.ktiles;
            tile = max(args.first[pi], args.whole) + in;
            kt0 = from - in * p.ktiles;
            kt1 = min(p.ktiles, kt0 + (steps_end - step));
        }
        step += kt1 - kt0;
        uint32_t tm, tn;
        ortho_place<SYM>(p, tile - args.first[pi], tm, tn);
        const uint32_t m0 = tm * BM, n0 = tn * BM;

        f32x16 acc[I][J];
        ortho_sums<BM, PA, PB, TB>(p, lds, lane, wave, m0, n0, kt0, kt1, acc);

        if (kt1 - kt0 == p.ktiles) {
            // (The lane is hidden from what comes before, and all loads are waited for here: addresses kept over the products would be spilled, and waiting for
            // one of them inside the loop waits for the last square's stores too.  A square took 2 us.)
            uint32_t l = lane;
            asm volatile("" : "+v"(l));
            float factor = ortho_factor(p);
            float* const mine = reinterpret_cast<float*>(lds) + wave * (32 * kOrthoRow);
            auto m_of = [&](int s) { return m0 + (wm * I + s / J) * 32; };
            auto n_of = [&](int s) { return n0 + (wn * J + s % J) * 32; };
            if (SYM && p.e) {
                ff_each<I * J>([&](auto q) {
                    constexpr int k = decltype(q)::value;
                    ortho_add(p, factor, acc[k / J][k % J], l, m_of(k), n_of(k));
                    if constexpr (k % 2 == 1) __builtin_amdgcn_sched_barrier(0);        // (two squares' loads at a time have registers)
                });
                factor = 1.0f;
            }
            __builtin_amdgcn_s_waitcnt(0);
            // a loop, whose code stays in the instruction cache
#pragma unroll 1
            for (int s = 0; s < I * J; ++s) {
                if (SYM && n_of(s) > m_of(s)) continue;
                ff_each<I * J>([&](auto q) {
                    constexpr int k = decltype(q)::value;
                    if (s == k) ortho_spread<T>(factor, p.beta, acc[k / J][k % J], mine, l);
                });
                ortho_square<SYM, T>(p, mine, l, m_of(s), n_of(s));
            }
        } else {
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *ortho_slot<BM>(args.part, worker + tile - args.whole, i, j, q, tid) =
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
    constexpr uint32_t I = BM / 64, J = BM / 64;
    __shared__ __align__(16) float stage[4 * 32 * kOrthoRow];
    const uint32_t at = blockIdx.x / (I * J), i = blockIdx.x / J % I, j = blockIdx.x % J, tile = args.whole + at;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    const uint32_t pi = ortho_problem_of(args.first, tile);
    const OrthoProblem& p = args.p[pi];
    const uint32_t s0 = args.begin[pi] + (tile - max(args.first[pi], args.whole)) * p.ktiles, s1 = s0 + p.ktiles;
    // the workers that have a step of this tile
    uint32_t first = static_cast<uint32_t>(static_cast<uint64_t>(s0) * args.workers / args.steps), last = static_cast<uint32_t>(static_cast<uint64_t>(s1 - 1) * args.workers / args.steps);
    while (ortho_share(args, first + 1) <= s0) ++first;
    while (last + 1 < args.workers && ortho_share(args, last + 1) < s1) ++last;
    if (first == last) return;                      // one, which has finished it
    uint32_t tm, tn;
    ortho_place<SYM>(p, tile - args.first[pi], tm, tn);
    const uint32_t m = tm * BM + (wave / 2 * I + i) * 32, n = tn * BM + (wave % 2 * J + j) * 32;
    if (SYM && n > m) return;
    f32x16 acc = {};
#pragma unroll 4
    for (uint32_t w = first; w <= last; ++w) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 v = *ortho_slot<BM>(args.part, w + at, i, j, q, tid);
            acc[4 * q] += v.x; acc[4 * q + 1] += v.y; acc[4 * q + 2] += v.z; acc[4 * q + 3] += v.w;
        }
    }
    float* const mine = stage + wave * (32 * kOrthoRow);
    float factor = ortho_factor(p);
    if (SYM && p.e) {
        ortho_add(p, factor, acc, lane, m, n);
        factor = 1.0f;
    }
    ortho_spread<T>(factor, p.beta, acc, mine, lane);
    ortho_square<SYM, T>(p, mine, lane, m, n);
}

}  // namespace edgc
