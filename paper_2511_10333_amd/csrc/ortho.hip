// The orthogonalised update of a list of gradients: Newton-Schulz steps of the normalised matrix, on its smaller side.
//
//   X = G / (|G| + eps), s x l, s <= l (a tall matrix is transposed);  steps times:  A = X X^T,  W = a I + b A + c A^2,  X <- W X;  out = scale X
//
// All matrices on the smaller side are polynomials of the same A: they commute and are symmetric.  So a segment of steps needs X twice only,
//
//   A_0 = X X^T,  W_k = a I + b A_k + c A_k^2,  V_k = W_k A_k,  A_k+1 = V_k W_k,  Q_k+1 = W_k Q_k (Q_0 = I),  X <- Q X,
//
// and of the symmetric products half the tiles are made: of s^3 operations 4 a step, instead of 3 l / s + 1 in every step as written above.  A_k+1 by
// products instead of from X carries its rounding errors on, a^2 = 12 times larger relative to the small singular values with each step, so segments are
// bounded (ortho_plan).  Operands are fp16 planes (ortho_gemm.h); every sum is in fp32.
//
// Bounded by the matrix instructions at the clock that the power allows: the four matrices of a block of hidden 4096, bf16, take 21.2 ms, their products
// 1.06 to 1.16 PFLOP/s (the library's of one fp16 product of 8192 a side: 1.08 to 1.12), of hidden 2048, fp32, 4.0 ms.  Small ones by launches that wait for
// each other: a block of hidden 512 has 22 in 226 us.
#include "ortho_gemm.h"

#include <algorithm>
#include <cmath>

namespace edgc {
namespace {

// ---------------------------------------------------------------------------------------------
// the gradient's norm, and the gradient as planes
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kOrthoGroup = 10, kOrthoParts = 1024;    // matrices of a launch; blocks that one is spread over
struct OrthoItem {
    const void* src;
    uint16_t* x;                        // planes
    double* part;                       // per block
    OrthoFactor* f;
    uint64_t ld, ldx;
    uint32_t m, n, tiles_c, tiles, first, blocks, tall, _pad;
};
struct OrthoList {
    OrthoItem t[kOrthoGroup];
    uint32_t count, blocks;
    double eps;
};
__device__ __forceinline__ const OrthoItem& ortho_item_of(const OrthoList& list)
{
    uint32_t k = 0;
    while (k + 1 < list.count && blockIdx.x >= list.t[k + 1].first) ++k;
    return list.t[k];
}
// Four neighbours of a row of a tile of 64 x 64, of which a quarter is loaded at a time.  (With eight, whose loads leave gaps, the planes of a hidden-2048
// block took 145 us instead of 78, 5.2 TB/s.)
template <typename T>
__device__ __forceinline__ void ortho_load4(const OrthoItem& t, uint32_t tile, uint32_t quarter, float (&v)[4])
{
    const uint32_t r = tile / t.tiles_c * 64 + quarter * 16 + threadIdx.x / 16, c = tile % t.tiles_c * 64 + threadIdx.x % 16 * 4;
    if (r >= t.m) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 0.f;
        return;
    }
    ff_load4<T, false>(static_cast<const T*>(t.src) + r * t.ld, c, t.n, v);
}
__device__ __forceinline__ double ortho_block_sum(double v)
{
    __shared__ double s[4];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x / 64] = v;
    __syncthreads();
    return (s[0] + s[1]) + (s[2] + s[3]);
}
// Squares and sums in 64 bits, in a fixed order
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_sumsq(const OrthoList list)
{
    const OrthoItem& t = ortho_item_of(list);
    const uint32_t at = blockIdx.x - t.first;
    double acc = 0.0;
    for (uint32_t tile = at; tile < t.tiles; tile += t.blocks)
#pragma unroll
        for (uint32_t quarter = 0; quarter < 4; ++quarter) {
            float v[4];
            ortho_load4<T>(t, tile, quarter, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc = __builtin_fma(static_cast<double>(v[i]), static_cast<double>(v[i]), acc);
        }
    acc = ortho_block_sum(acc);
    if (threadIdx.x == 0) t.part[at] = acc;
}
// X = f 2^k G: 2^k G, whose norm is in [2^14, 2^15), as planes (P of them), f = 1 / ((norm + eps) 2^k) beside them (OrthoFactor).  Of a gradient that has a
// value that is not finite f is NaN, and so is the whole update.
template <typename T, int P>
__global__ __launch_bounds__(256) void k_ortho_pack(const OrthoList list)
{
    __shared__ float turn[64 * 65];
    const OrthoItem& t = ortho_item_of(list);
    const uint32_t at = blockIdx.x - t.first;
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < t.blocks; i += 256) sum += t.part[i];
    const double norm = sqrt(ortho_block_sum(sum));
    int k = 0;
    if (norm > 0.0 && norm < 1e300) {
        (void)frexp(norm, &k);
        k = 15 - k;
    }
    if (at == 0 && threadIdx.x == 0) {
        OrthoFactor f{norm < 1e300 ? 0.f : __builtin_nanf(""), 0};
        if (norm > 0.0 && norm < 1e300) {
            (void)frexp(norm / (norm + list.eps), &f.exponent);
            f.value = static_cast<float>(ldexp(1.0 / (norm + list.eps), -k - f.exponent));
        }
        *t.f = f;
    }
    auto put = [&](uint32_t row, uint32_t col, const float (&v)[4]) {         // of X
        f16x4 h, l;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = ldexpf(v[i], k);
            h[i] = static_cast<_Float16>(x);
            l[i] = static_cast<_Float16>(x - static_cast<float>(h[i]));
        }
        uint16_t* const to = t.x + row * t.ldx + (P == 2 ? ortho_at(col) : col);
        *reinterpret_cast<f16x4*>(to) = h;
        if constexpr (P == 2) *reinterpret_cast<f16x4*>(to + 32) = l;
    };
    const uint32_t row = threadIdx.x / 16, col = threadIdx.x % 16 * 4;
    for (uint32_t tile = at; tile < t.tiles; tile += t.blocks) {
        const uint32_t r0 = tile / t.tiles_c * 64, c0 = tile % t.tiles_c * 64;
        float v[4][4];
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) ortho_load4<T>(t, tile, q, v[q]);
        if (!t.tall) {
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) put(r0 + q * 16 + row, c0 + col, v[q]);
            continue;
        }
        __syncthreads();                // the last tile's reads are done
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) turn[(q * 16 + row) * 65 + col + i] = v[q][i];
        __syncthreads();
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[q][i] = turn[(col + i) * 65 + q * 16 + row];
            put(c0 + q * 16 + row, r0 + col, v[q]);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kOrthoMaxSide = 1u << 14, kOrthoMaxLong = 1u << 20, kOrthoMaxSteps = 64;
// Steps of a segment at most, and what its errors may grow by.  A_0 is off by some 2^-22 of its largest value (its sums of l products as well as its
// planes), which each further step on the same A makes w^2 larger relative to what comes of the smallest singular values, w the largest value of W: 12, of
// 3.4445.  bf16, three: of a gradient of one direction above noise, 256 x 2048, five steps on one A were 9.9e-3 off in the directions of its rows, three and two
// are 7.4e-4, the output's rounding alone 6e-4.  fp32, two: of 460 lists of all sizes seven are more than 1.5 times and 1e-6 further off than fp32 products
// in X itself, up to 3 times, matrices of a side of 13 or less; with three and two 19 of 60, up to 3.5 times; five single steps: none of 60.  A block of
// hidden 2048 takes 4.0 ms, with three and two 3.45.
constexpr uint32_t ortho_most(edgc_dtype dt) { return dt == EDGC_F32 ? 2 : 3; }
constexpr double ortho_carried(edgc_dtype dt) { return dt == EDGC_F32 ? 12.0 : 145.0; }

// A reservation for up to so many steps is for calls of up to so many, one for more is for any
constexpr uint32_t ortho_few(edgc_dtype dt) { return dt == EDGC_F32 ? 3 : 5; }

uint64_t pad64(uint64_t n) { return (n + 63) / 64 * 64; }

struct OrthoShape {
    uint64_t s, l, S, L;                // the smaller and the larger side, padded
    bool tall;
    OrthoShape() = default;
    OrthoShape(uint64_t m, uint64_t n) : s(std::min(m, n)), l(std::max(m, n)), S(pad64(s)), L(pad64(l)), tall(m > n) {}
    // 16-bit elements: X, the X of a later segment, five matrices of the smaller side
    uint64_t x_elems(uint32_t planes) const { return S * L * planes; }
    uint64_t side_elems() const { return S * S * 2; }
    uint64_t elems() const { return 2 * x_elems(2) + 5 * side_elems(); }
    uint64_t tiles() const { const uint64_t t = (s + 255) / 256; return t * (t + 1) / 2; }
};

// Matrices i, i + 1, .. that are worked on together: as many as give the smaller side's products a few rounds of tiles, and fit
template <typename F>
uint32_t ortho_group(const edgc_ctx* ctx, uint32_t i, uint32_t count, uint64_t held, F&& shape_of, uint64_t* used)
{
    uint64_t elems = 0, tiles = 0;
    uint32_t k = 0;
    for (; i + k < count && k < kOrthoGroup; ++k) {
        const OrthoShape sh = shape_of(i + k);
        const uint64_t e = sh.elems();
        if (k && (e > held - elems || tiles >= 4ull * ctx->num_cu)) break;
        elems += e;
        tiles += sh.tiles();
    }
    if (used) *used = elems;
    return k;
}

// Powers of two that the matrices of a step are scaled by, so that none of their entries passes 2^15: an entry of a symmetric matrix is at
// most its largest eigenvalue, a polynomial's largest value over the singular values that there can be.
struct OrthoScale {
    static int of(double most) { int e; (void)std::frexp(std::max(most * 1.1, 1e-6), &e); return 15 - e; }
    // bits by which values that small ones have `grown` to may pass `most`
    static int reach(double grown, double most)
    {
        const double ratio = grown / std::max(most, 1e-6);
        int e = 0;
        if (ratio > 1.0) (void)std::frexp(std::min(ratio, 1e300), &e);
        return e;
    }
};

struct OrthoCoefs {
    double a, b, c;
    // the largest |p0 + p1 u + p2 u^2| u^power over [0, top], of which the derivative's quadratic is d0 + d1 u + d2 u^2
    double most_of(double top, double power, double d0, double d1, double d2) const
    {
        double best = 0.0;
        auto look = [&](double u) {
            if (u >= 0.0 && u <= top) best = std::max(best, std::fabs(a + u * (b + u * c)) * std::pow(u, power));
        };
        look(0.0);
        look(top);
        if (d2 == 0.0) {
            if (d1 != 0.0) look(-d0 / d1);
        } else if (const double disc = d1 * d1 - 4.0 * d2 * d0; disc >= 0.0) {
            look((-d1 + std::sqrt(disc)) / (2.0 * d2));
            look((-d1 - std::sqrt(disc)) / (2.0 * d2));
        }
        return best;
    }
    // the largest values of W, W A and W s over singular values s up to `top`: of a + b u + c u^2 and its products with u and sqrt u, u = s^2
    void most(double top, double& w_top, double& v_top, double& s_top) const
    {
        const double u = top * top;
        w_top = most_of(u, 0.0, b, 2.0 * c, 0.0);
        v_top = most_of(u, 1.0, a, 2.0 * b, 3.0 * c);
        s_top = most_of(u, 0.5, a, 3.0 * b, 5.0 * c);
    }
};
constexpr double kOrthoMost = 1e9;      // beyond this the steps diverge

// Which steps are made on one A
struct OrthoPlan {
    uint32_t steps, segments;
    // the step that segment `seg` ends before: the longer segments come first
    uint32_t end(uint32_t seg) const { return (steps * (seg + 1) + segments - 1) / segments; }
};

// Cuts `steps` of them into segments; false where they do not keep every matrix representable
bool ortho_plan(const OrthoCoefs& co, edgc_dtype dt, uint32_t steps, OrthoPlan* plan)
{
    double top = 1.0, w[kOrthoMaxSteps];
    for (uint32_t k = 0; k < steps; ++k) {
        double v, s;
        co.most(top, w[k], v, s);
        if (!(w[k] <= kOrthoMost && v <= kOrthoMost && s <= kOrthoMost && s * s <= kOrthoMost)) return false;
        top = s;
    }
    auto fits = [&]() {
        for (uint32_t seg = 0, k = 0; seg < plan->segments; ++seg) {
            double q = 1.0, carried = 1.0;
            for (const uint32_t end = plan->end(seg); k < end; ++k) {
                q *= w[k];
                if (k + 1 < end) carried *= w[k] * w[k];
            }
            if (!(q <= kOrthoMost && carried <= ortho_carried(dt))) return false;
        }
        return true;
    };
    for (uint32_t most = ortho_most(dt); most > 0; --most) {
        *plan = OrthoPlan{steps, (steps + most - 1) / most};
        if (fits()) break;              // (single steps do)
    }
    return true;
}

// The tile shapes: blocks of 256 rows have a compute unit for themselves, of 128 x 128 two share it
uint32_t ortho_places(const edgc_ctx* ctx, int bm) { return static_cast<uint32_t>(ctx->num_cu) * (bm == 256 ? 1 : 2); }
// sums that workers can leave behind: at most two tiles per place
uint64_t ortho_sums_elems(const edgc_ctx* ctx) { return 2ull * 256 * 256 * ctx->num_cu; }
// the least tiles of k that are worth a worker, whose sums go through memory: those of a small tile are soon done (of a hidden-512 block, products whose 16
// tiles of k are shared among workers cost 230 us, 225 if not; a hidden-2048 block's, in tiles of 128 x 128, 3616 and 3841)
constexpr uint32_t ortho_least(int bm) { return bm == 64 ? 64 : 8; }

template <int BM, int PA, int PB, bool TB, typename T>
hipError_t prepare_ortho_tiles()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_ortho_gemm<BM, PA, PB, TB, T>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               kOrthoLds<BM, PB, TB>);
}

struct OrthoPass {
    edgc_ctx* ctx;
    hipStream_t st;
    edgc_dtype dt;
    const edgc_tensor* tensors;
    const float* scales;
    uint32_t count;
    OrthoPlan plan;
    double eps;
    OrthoCoefs co;
    struct Mat {
        OrthoShape sh;
        uint16_t *x[2], *a, *v, *w[3];
        OrthoFactor* f;
    };
    uint32_t first_planes() const { return dt == EDGC_F32 ? 2 : 1; }
    Mat mats[kOrthoGroup] = {};
    uint32_t n = 0;                             // of them

    template <int BM, int PA, int PB, bool TB, typename T>
    int launch(OrthoArgs& args, int kid)
    {
        uint32_t tiles = 0;
        double flops = 0.0, bytes = 0.0;
        std::fill(args.first, args.first + kOrthoProblems, UINT32_MAX);
        std::fill(args.begin, args.begin + kOrthoProblems, UINT32_MAX);
        for (uint32_t i = 0; i < args.count; ++i) {
            OrthoProblem& p = args.p[i];
            p.tiles_m = (p.M + BM - 1) / BM;
            p.tiles_n = (p.N + BM - 1) / BM;
            args.first[i] = tiles;
            tiles += tiles_of<BM, TB>(p);
            const double k = static_cast<double>(p.ktiles) * kOrthoK<PA, PB>;
            flops += (TB ? 2.0 : 1.0) * p.M * p.N * k * (PA + PB - 1);
            bytes += 2.0 * k * (static_cast<double>(p.M) * PA + static_cast<double>(p.N) * PB);
        }
        const uint32_t places = ortho_places(ctx, BM);
        args.whole = tiles / places * places;
        auto count_rest = [&]() {
            args.rest = tiles - args.whole;
            args.steps = 0;
            for (uint32_t i = 0; i < args.count; ++i) {
                OrthoProblem& p = args.p[i];
                const uint32_t end = i + 1 < args.count ? args.first[i + 1] : tiles;
                args.begin[i] = args.steps;
                if (end > args.whole) args.steps += (end - std::max(args.first[i], args.whole)) * p.ktiles;
            }
        };
        count_rest();
        args.workers = std::min(places, args.steps / ortho_least(BM));
        // (a last round that is nearly full is not worth the sums' way through memory)
        if (args.workers <= args.rest || args.rest * 10ull > places * 9ull) {
            args.whole = tiles;
            args.workers = 0;
            count_rest();
        }
        args.part = ctx->ortho.sums;
        EDGC_LAUNCH(ctx, st, kid, bytes, flops, k_ortho_gemm<BM, PA, PB, TB, T><<<args.whole + args.workers, 256, kOrthoLds<BM, PB, TB>, st>>>(args));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        if (args.rest) {
            EDGC_LAUNCH(ctx, st, KID_ORTHO_JOIN, 4.0 * BM * BM * (args.workers + args.rest), 0.0,
                        k_ortho_join<BM, TB, T><<<args.rest * (BM / 64) * (BM / 64), 256, 0, st>>>(args));
            EDGC_HIP_TRY(ctx, hipGetLastError());
        }
        return EDGC_OK;
    }
    template <int BM, bool TB>
    static uint32_t tiles_of(const OrthoProblem& p)
    {
        const uint32_t tm = (p.M + BM - 1) / BM, tn = (p.N + BM - 1) / BM;
        return TB ? tm * tn : ortho_tiles(tm);
    }
    template <int PA, int PB, bool TB, typename T>
    int product(OrthoArgs& args, int kid)
    {
        std::stable_sort(args.p, args.p + args.count, [](const OrthoProblem& x, const OrthoProblem& y) { return x.ktiles > y.ktiles; });
        // The time that a tile shape would take, in us: `step`: for a tile of k of each of a compute unit's blocks at a time, `alone`: where a block has its
        // compute unit for itself; sums that go through memory and are joined cost a launch.  Measured on products of 512 to 4096.  A block of hidden 512 takes
        // 231 us with tiles of 64 x 64, 329 with 128 x 128; odd matrices up to 2731 282 and 531; a block of hidden 2048 4540 and 3616.
        auto time_of = [&](auto bm, double step, double alone) {
            constexpr double share = 8.0;
            double steps = 0.0, tiles = 0.0, longest = 0.0;
            for (uint32_t i = 0; i < args.count; ++i) {
                const double n = tiles_of<bm, TB>(args.p[i]);
                tiles += n;
                steps += n * args.p[i].ktiles;
                longest = std::max(longest, 1.0 * args.p[i].ktiles);
            }
            const double places = ortho_places(ctx, bm), least = ortho_least(bm);
            if (tiles >= places || longest <= least) return std::max(step * steps / places, alone * longest);
            return share + std::max(step * steps / places, alone * std::min(longest, least));
        };
        using Large = std::integral_constant<int, 256>;
        using Middle = std::integral_constant<int, 128>;
        using Small = std::integral_constant<int, 64>;
        constexpr double work = PA == 1 || PB == 2 ? 1.0 : 2.0 / 3.0;     // a tile of k: 64 of one product, or 32 of three or two
        const double middle = time_of(Middle{}, work * 1.58, work * 0.9);
        // (one plane of a transposed operand is too narrow for the small tiles' reads)
        if constexpr (!(TB && PB == 1)) {
            if (time_of(Small{}, work * 0.53, work * 0.33) < middle) return launch<64, PA, PB, TB, T>(args, kid);
        }
        // The first products of bf16 matrices, of one plane: for a block of hidden 4096 they take 880 us, with tiles of 128 x 128 949.  (Of two planes, with
        // two sums, a wave has room for 128 x 64, and tiles of 256 x 128 took 1643 us for the products of a hidden-2048 block's smaller sides, not 1505.)
        if constexpr (PA == 1) {
            if (time_of(Large{}, work * 2.2, work * 2.2) <= middle) return launch<256, PA, PB, TB, T>(args, kid);
        }
        return launch<128, PA, PB, TB, T>(args, kid);
    }
    // a product of two matrices of the smaller side, or the first of a segment
    static OrthoProblem symmetric(const Mat& m, const uint16_t* a, const uint16_t* b, uint16_t* out, double alpha)
    {
        OrthoProblem p{};
        p.a = a; p.b = b; p.out = out;
        p.lda = p.ldb = p.ldo = 2 * m.sh.S;
        p.M = p.N = static_cast<uint32_t>(m.sh.s);
        p.rows = p.cols = static_cast<uint32_t>(m.sh.S);
        p.ktiles = static_cast<uint32_t>(m.sh.S / 32);
        p.alpha = static_cast<float>(alpha);
        p.into = kOrthoPlain;
        return p;
    }

    int group(uint32_t i0, uint32_t many)
    {
        place(i0, many);
        if (int rc = dt == EDGC_F32 ? pack<float>(i0) : pack<__bf16>(i0)) return rc;
        double top = 1.0;
        double grown = 1.0;                     // what singular values may have been multiplied by
        int x_scale = 0, reach = kOrthoFirst;   // of X; the first one's scale is in f
        for (uint32_t seg = 0, done = 0; seg < plan.segments; ++seg) {
            const uint32_t end = plan.end(seg), from = seg % 2;
            const bool first = seg == 0, single = first && first_planes() == 1;
            // A = X X^T
            int a_scale = OrthoScale::of(top * top), q_scale = 0;
            {
                OrthoArgs g{};
                for (const Mat& m : these()) {
                    OrthoProblem p = symmetric(m, m.x[from], m.x[from], m.a, std::ldexp(1.0, a_scale - (first ? 0 : 2 * x_scale)));
                    p.lda = p.ldb = m.sh.L * (single ? 1 : 2);
                    p.ktiles = static_cast<uint32_t>(m.sh.L / (single ? 64 : 32));
                    p.f = m.f; p.power = 2; p.from = reach;
                    g.p[g.count++] = p;
                }
                if (int rc = single ? product<1, 1, false, void>(g, KID_ORTHO_GRAM) : product<2, 2, false, void>(g, KID_ORTHO_GRAM)) return rc;
            }
            double q = 1.0;
            uint32_t at_q = 0;                  // which of w[] holds Q
            for (bool begin = true; done < end; ++done, begin = false) {
                const bool last = done + 1 == end;
                double w_top, v_top, s_top;
                co.most(top, w_top, v_top, s_top);
                q *= w_top;
                grown *= w_top;
                const int w_scale = OrthoScale::of(w_top), v_scale = OrthoScale::of(v_top), next_a = OrthoScale::of(s_top * s_top), next_q = OrthoScale::of(q);
                const uint32_t at_w = begin ? 0 : (at_q + 1) % 3, at_new = (at_q + 2) % 3;
                OrthoArgs g{};
                for (const Mat& m : these()) {     // W
                    OrthoProblem p = symmetric(m, m.a, m.a, m.w[at_w], std::ldexp(co.c, w_scale - 2 * a_scale));
                    p.e = m.a;
                    p.beta = static_cast<float>(std::ldexp(co.b, w_scale - a_scale));
                    p.gamma = static_cast<float>(std::ldexp(co.a, w_scale));
                    g.p[g.count++] = p;
                }
                if (int rc = product<2, 2, false, void>(g, KID_ORTHO_CHAIN)) return rc;
                g = OrthoArgs{};
                for (const Mat& m : these()) {     // V, and the next Q
                    if (!last) g.p[g.count++] = symmetric(m, m.w[at_w], m.a, m.v, std::ldexp(1.0, v_scale - w_scale - a_scale));
                    if (!begin) g.p[g.count++] = symmetric(m, m.w[at_w], m.w[at_q], m.w[at_new], std::ldexp(1.0, next_q - w_scale - q_scale));
                }
                if (g.count)
                    if (int rc = product<2, 2, false, void>(g, KID_ORTHO_CHAIN)) return rc;
                if (!last) {                    // the next A
                    g = OrthoArgs{};
                    for (const Mat& m : these()) g.p[g.count++] = symmetric(m, m.v, m.w[at_w], m.a, std::ldexp(1.0, next_a - v_scale - w_scale));
                    if (int rc = product<2, 2, false, void>(g, KID_ORTHO_CHAIN)) return rc;
                }
                a_scale = next_a;
                q_scale = begin ? w_scale : next_q;
                at_q = begin ? 0 : at_new;
                top = s_top;
            }
            // X <- Q X
            const bool out = seg + 1 == plan.segments;
            const int next_x = OrthoScale::of(top), next_reach = out ? kOrthoPlain : OrthoScale::reach(grown, top);
            OrthoArgs g{};
            for (uint32_t i = 0; i < n; ++i) {
                const Mat& m = mats[i];
                const edgc_tensor& d = tensors[i0 + i];
                OrthoProblem p{};
                p.a = m.w[at_q]; p.b = m.x[from];
                p.lda = 2 * m.sh.S; p.ldb = m.sh.L * (single ? 1 : 2);
                p.M = static_cast<uint32_t>(m.sh.s); p.N = static_cast<uint32_t>(m.sh.l);
                p.ktiles = static_cast<uint32_t>(m.sh.S / 32);
                p.alpha = static_cast<float>(std::ldexp(1.0, (out ? 0 : next_x) - q_scale - (first ? 0 : x_scale)));
                p.beta = scales ? scales[i0 + i] : 1.0f;
                p.f = m.f; p.power = 1; p.from = reach; p.into = next_reach;
                if (out) {
                    p.to = d.grad_out; p.ldo = d.ld_out; p.transposed = m.sh.tall;
                } else {
                    p.out = m.x[1 - from]; p.ldo = 2 * m.sh.L;
                    p.rows = static_cast<uint32_t>(m.sh.S); p.cols = static_cast<uint32_t>(m.sh.L);
                }
                g.p[g.count++] = p;
            }
            if (int rc = apply(g, single, out)) return rc;
            x_scale = next_x;
            reach = next_reach;
        }
        return EDGC_OK;
    }
    int apply(OrthoArgs& g, bool single, bool out)
    {
        if (!out) return single ? product<2, 1, true, void>(g, KID_ORTHO_APPLY) : product<2, 2, true, void>(g, KID_ORTHO_APPLY);
        if (dt == EDGC_F32) return product<2, 2, true, float>(g, KID_ORTHO_APPLY);
        return single ? product<2, 1, true, __bf16>(g, KID_ORTHO_APPLY) : product<2, 2, true, __bf16>(g, KID_ORTHO_APPLY);
    }

    struct Some {
        const Mat *from, *to;
        const Mat* begin() const { return from; }
        const Mat* end() const { return to; }
    };
    Some these() const { return {mats, mats + n}; }

    void place(uint32_t i0, uint32_t many)
    {
        n = many;
        uint16_t* at = static_cast<uint16_t*>(ctx->ortho.ws);
        auto take = [&](uint64_t elems) { uint16_t* const p = at; at += elems; return p; };
        for (uint32_t i = 0; i < n; ++i) {
            Mat m{OrthoShape(tensors[i0 + i].m, tensors[i0 + i].n), {}, nullptr, nullptr, {}, nullptr};
            for (uint16_t*& x : m.x) x = take(m.sh.x_elems(2));
            m.a = take(m.sh.side_elems());
            m.v = take(m.sh.side_elems());
            for (uint16_t*& w : m.w) w = take(m.sh.side_elems());
            m.f = static_cast<OrthoFactor*>(ctx->ortho.f) + i;
            mats[i] = m;
        }
    }
    template <typename T>
    int pack(uint32_t i0)
    {
        OrthoList list{};
        list.eps = eps;
        const uint32_t planes = first_planes();
        double elems = 0.0;
        for (uint32_t i = 0; i < n; ++i) {
            const edgc_tensor& d = tensors[i0 + i];
            OrthoItem& t = list.t[list.count++];
            t.src = d.grad; t.ld = d.ld; t.m = d.m; t.n = d.n;
            t.x = mats[i].x[0]; t.ldx = mats[i].sh.L * planes; t.tall = mats[i].sh.tall;
            t.part = ctx->ortho.part + static_cast<size_t>(i) * kOrthoParts; t.f = mats[i].f;
            t.tiles_c = (d.n + 63) / 64;
            t.tiles = t.tiles_c * ((d.m + 63) / 64);
            t.first = list.blocks;
            t.blocks = std::min(t.tiles, kOrthoParts);
            list.blocks += t.blocks;
            elems += static_cast<double>(d.m) * d.n;
        }
        EDGC_LAUNCH(ctx, st, KID_ORTHO_SUMSQ, elems * sizeof(T), 0.0, k_ortho_sumsq<T><<<list.blocks, 256, 0, st>>>(list));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        if (planes == 2) EDGC_LAUNCH(ctx, st, KID_ORTHO_PACK, elems * (sizeof(T) + 4.0), 0.0, k_ortho_pack<T, 2><<<list.blocks, 256, 0, st>>>(list));
        else EDGC_LAUNCH(ctx, st, KID_ORTHO_PACK, elems * (sizeof(T) + 2.0), 0.0, k_ortho_pack<T, 1><<<list.blocks, 256, 0, st>>>(list));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        return EDGC_OK;
    }
};

int check_shape(edgc_ctx* ctx, uint64_t m, uint64_t n)
{
    if (m == 0 || n == 0) return fail(ctx, EDGC_EINVAL, "empty tensor in list");
    if (std::min(m, n) > kOrthoMaxSide || std::max(m, n) > kOrthoMaxLong)
        return fail(ctx, EDGC_EINVAL, "the smaller side of a matrix is at most 2^14, the larger 2^20");
    return EDGC_OK;
}

}  // namespace

int prepare_ortho_kernels(edgc_ctx* ctx)
{
    for (hipError_t e : {prepare_ortho_tiles<64, 1, 1, false, void>(), prepare_ortho_tiles<64, 2, 2, false, void>(),
                         prepare_ortho_tiles<64, 2, 2, true, void>(), prepare_ortho_tiles<64, 2, 2, true, float>(),
                         prepare_ortho_tiles<64, 2, 2, true, __bf16>(), prepare_ortho_tiles<128, 1, 1, false, void>(),
                         prepare_ortho_tiles<256, 1, 1, false, void>(), prepare_ortho_tiles<128, 2, 2, false, void>(),
                         prepare_ortho_tiles<128, 2, 1, true, void>(), prepare_ortho_tiles<128, 2, 2, true, void>(),
                         prepare_ortho_tiles<128, 2, 2, true, float>(), prepare_ortho_tiles<128, 2, 1, true, __bf16>(),
                         prepare_ortho_tiles<128, 2, 2, true, __bf16>()})
        EDGC_HIP_TRY(ctx, e);
    return EDGC_OK;
}

void free_ortho(edgc_ctx* ctx)
{
    if (ctx->ortho.sums) (void)hipFree(ctx->ortho.sums);
    if (ctx->ortho.ws) (void)hipFree(ctx->ortho.ws);
    if (ctx->ortho.part) (void)hipFree(ctx->ortho.part);
    ctx->ortho = OrthoScratch{};
}

}  // namespace edgc

using namespace edgc;

extern "C" int edgc_reserve_orthogonalize(edgc_ctx* ctx, edgc_dtype dtype, const uint32_t* rows, const uint32_t* cols, uint32_t count, uint32_t steps)
{
    if (!ctx) return EDGC_EINVAL;
    if (dtype != EDGC_F32 && dtype != EDGC_BF16) return fail(ctx, EDGC_EINVAL, "unknown dtype");
    if (count && (!rows || !cols)) return fail(ctx, EDGC_EINVAL, "null list of shapes");
    if (count && (steps == 0 || steps > kOrthoMaxSteps)) return fail(ctx, EDGC_EINVAL, "steps must be 1 to 64");
    for (uint32_t i = 0; i < count; ++i)
        if (int rc = check_shape(ctx, rows[i], cols[i])) return rc;
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    uint64_t need = 0;
    for (uint32_t i = 0; i < count;) {
        uint64_t used = 0;
        i += ortho_group(ctx, i, count, ~0ull, [&](uint32_t k) { return OrthoShape(rows[k], cols[k]); }, &used);
        need = std::max(need, used);
    }
    if (need && need <= ctx->ortho.held) {
        ctx->ortho.elems = need;
        ctx->ortho.steps = steps;
        return EDGC_OK;
    }
    EDGC_HIP_TRY(ctx, hipDeviceSynchronize());          // nothing may still be using the old scratch
    free_ortho(ctx);
    if (need == 0) return EDGC_OK;
    const size_t parts = static_cast<size_t>(kOrthoGroup) * kOrthoParts;
    bool ok = hipMalloc(&ctx->ortho.ws, need * 2) == hipSuccess;
    ok = ok && hipMalloc(reinterpret_cast<void**>(&ctx->ortho.part), parts * sizeof(double) + kOrthoGroup * sizeof(OrthoFactor)) == hipSuccess;
    ok = ok && hipMalloc(reinterpret_cast<void**>(&ctx->ortho.sums), ortho_sums_elems(ctx) * sizeof(float)) == hipSuccess;
    if (!ok) {
        (void)hipGetLastError();
        free_ortho(ctx);
        return fail(ctx, EDGC_ENOMEM, "scratch allocation of the orthogonalised update failed");
    }
    ctx->ortho.f = ctx->ortho.part + parts;
    ctx->ortho.elems = ctx->ortho.held = need;
    ctx->ortho.steps = steps;
    return EDGC_OK;
}

extern "C" int edgc_orthogonalize_batch(edgc_ctx* ctx, const edgc_tensor* tensors, uint32_t count, edgc_dtype dtype, uint32_t steps, double a, double b,
                                        double c, double eps, const float* scales, void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    if (int rc = check_gradients(ctx, tensors, count, dtype, true)) return rc;
    if (steps == 0 || steps > kOrthoMaxSteps) return fail(ctx, EDGC_EINVAL, "steps must be 1 to 64");
    if (!(eps >= 0.0) || !std::isfinite(eps)) return fail(ctx, EDGC_EINVAL, "eps must be finite and not negative");
    const OrthoCoefs co{a, b, c};
    OrthoPlan plan{};
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c) || !ortho_plan(co, dtype, steps, &plan))
        return fail(ctx, EDGC_EINVAL, "coefficients must be finite, and so that the steps keep singular values bounded");
    const uint32_t few = ortho_few(dtype);
    for (uint32_t i = 0; i < count; ++i) {
        if (int rc = check_shape(ctx, tensors[i].m, tensors[i].n)) return rc;
        if (scales && !std::isfinite(scales[i])) return fail(ctx, EDGC_EINVAL, "scales must be finite");
        if (OrthoShape(tensors[i].m, tensors[i].n).elems() > ctx->ortho.elems || (steps > few && ctx->ortho.steps <= few))
            return fail(ctx, EDGC_EINVAL, "larger than what edgc_reserve_orthogonalize was called for");
    }
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    OrthoPass pass{ctx, static_cast<hipStream_t>(hip_stream), dtype, tensors, scales, count, plan, eps, co};
    for (uint32_t i = 0; i < count;) {
        const uint32_t n = ortho_group(ctx, i, count, ctx->ortho.elems, [&](uint32_t k) { return OrthoShape(tensors[k].m, tensors[k].n); }, nullptr);
        if (int rc = pass.group(i, n)) return rc;
        i += n;
    }
    return EDGC_OK;
}
