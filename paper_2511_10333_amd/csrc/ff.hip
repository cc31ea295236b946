// The gated feed-forward block and its backward pass.
//
//   G = x Wg^T, U = x Wu^T, A = act(G) U, y = A Wd^T               (Wg, Wu: ff x hidden, Wd: hidden x ff)
//   dA = dy Wd;  dG = dA U act'(G), dU = dA act(G);  dx = dG Wg + dU Wu;  dWg = dG^T x, dWu = dU^T x, dWd = dy^T A
//
// Forward: one product whose tiles hold both projections and whose epilogue applies the activation and the product, and one for y.
// Backward: dA, whose epilogue makes dG, dU and A from the kept projections (dA itself is never stored), dx over both halves in one
// sum, and the three weight gradients in one launch.  Products: ff_gemm.h, few tokens forward: ff_few.h.  Either takes the operands as
// they lie in memory, transposed or not.  Where that cannot be (ff_gemm.h: rows that are not 16-byte aligned, k not a multiple of 64,
// fp32) they are first copied into the reserved scratch, padded, and in fp32 split into planes.
#include "ff_few.h"

#include <algorithm>
#include <cmath>
#include <utility>

namespace edgc {
namespace {

// ---------------------------------------------------------------------------------------------
// Copies into operand form: rows and columns padded with zeros to multiples of 64, fp32 as three planes.  64 x 64 elements per block, a
// thread eight neighbours at a time; up to kPacks matrices per launch.  Bounded by memory: five fp32 matrices, 235 MB, and their planes
// 101 us (5.8 TB/s)
// ---------------------------------------------------------------------------------------------
constexpr int kPacks = 5;
struct PackItem {
    const void* src;
    uint16_t* dst;
    uint64_t ld, ldd, plane;                // elements: of the source, the copy; between planes of the copy
    uint32_t rows, cols, tiles_c, first;    // of the source; tiles across; first block
};
struct PackList {
    PackItem t[kPacks];
    uint32_t count, blocks;
};
template <typename T>
__global__ __launch_bounds__(256) void k_ff_pack(const PackList list)
{
    constexpr int P = FfType<T>::kPlanes;
    uint32_t k = 0;
#pragma unroll
    for (int i = 1; i < kPacks; ++i) k += (static_cast<uint32_t>(i) < list.count && blockIdx.x >= list.t[i].first) ? 1u : 0u;
    const PackItem& t = list.t[k];
    const uint32_t id = blockIdx.x - t.first, c = id % t.tiles_c * 64 + threadIdx.x % 8 * 8;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const uint32_t r = id / t.tiles_c * 64 + half * 32 + threadIdx.x / 8;
        float v[2][4] = {};
        if (r < t.rows) {
            const T* const row = static_cast<const T*>(t.src) + r * t.ld;
            ff_load4<T, false>(row, c, t.cols, v[0]);
            ff_load4<T, false>(row, c + 4, t.cols, v[1]);
        }
        uint16_t* const to = t.dst + r * t.ldd + c;
        if constexpr (P == 1) {
            bf16x8 w[1];
            const float all[8] = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]};
            pack8<1>(all, w);
            *reinterpret_cast<bf16x8*>(to) = w[0];
        } else {
            uint16_t q[8][3];
#pragma unroll
            for (int e = 0; e < 8; ++e) ff_planes(v[e / 4][e % 4], q[e]);
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = q[2 * e][p] | static_cast<uint32_t>(q[2 * e + 1][p]) << 16;
                *reinterpret_cast<u32x4*>(to + p * t.plane) = w;
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
uint64_t pad64(uint64_t n) { return (n + 63) / 64 * 64; }

struct Operand {
    const uint16_t* p;
    uint64_t ld, plane;
};

// Where a pass keeps its operands, in elements of 16 bits from the start of the scratch; the sizes count every operand as copied.
struct FfPlan {
    uint64_t T, H, F, planes, used = 0;     // tokens, hidden, ff, padded
    FfPlan(uint64_t tokens, uint64_t hidden, uint64_t ff, edgc_dtype dt)
        : T(pad64(tokens)), H(pad64(hidden)), F(pad64(ff)), planes(dt == EDGC_F32 ? 3 : 1) {}
    uint64_t take(uint64_t rows, uint64_t ld)
    {
        const uint64_t at = used;
        used += planes * rows * ld;         // (rows of 128 bytes: everything stays 16-byte aligned)
        return at;
    }
    uint64_t x = 0, wg = 0, wu = 0, wd = 0, h = 0, dy = 0, dg = 0, du = 0;
    uint64_t forward()
    {
        used = 0;
        x = take(T, H); wg = take(F, H); wu = take(F, H); wd = take(H, F); h = take(T, F);
        return used;
    }
    uint64_t backward()
    {
        forward();
        dy = take(T, H); dg = take(T, F); du = take(T, F);
        return used;
    }
};

constexpr uint32_t kFfMaxTokens = 1u << 21, kFfMaxWidth = 1u << 20;

struct Packer {
    edgc_ctx* ctx;
    hipStream_t st;
    PackList list{};
    void add(const void* src, uint64_t ld, uint64_t rows, uint64_t cols, uint16_t* dst)
    {
        PackItem& t = list.t[list.count++];
        t.src = src; t.dst = dst; t.ld = ld;
        t.rows = static_cast<uint32_t>(rows); t.cols = static_cast<uint32_t>(cols);
        t.ldd = pad64(cols); t.plane = pad64(rows) * t.ldd;
        t.tiles_c = static_cast<uint32_t>(pad64(cols) / 64);
        t.first = list.blocks;
        list.blocks += static_cast<uint32_t>(pad64(rows) / 64) * t.tiles_c;
    }
    template <typename T>
    int flush()
    {
        if (list.count == 0) return EDGC_OK;
        double bytes = 0.0;
        for (uint32_t i = 0; i < list.count; ++i)
            bytes += static_cast<double>(list.t[i].rows) * list.t[i].cols * (sizeof(T) + 2.0 * FfType<T>::kPlanes);
        EDGC_LAUNCH(ctx, st, KID_FF_PACK, bytes, 0.0, k_ff_pack<T><<<list.blocks, 256, 0, st>>>(list));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        list = PackList{};
        return EDGC_OK;
    }
};

// LDS of a tile shape: two buffers, of A three where there is room; blocks that share a compute unit's
constexpr uint32_t lds_bytes(int bm, int bn) { return ((bm == 256 ? 3u : 2u) * bm + 2u * bn) * 128u; }
constexpr uint32_t blocks_per_cu(int bm, int bn) { return 160u * 1024u / lds_bytes(bm, bn); }
// The least k that is worth a worker, which then writes a tile's sums and has them read again
constexpr uint64_t kMinK = 512;

template <int BM, int BN, bool TA, bool TB, typename T, int EPI>
int launch_tiles(edgc_ctx* ctx, FfArgs& a, int kid, hipStream_t st)
{
    uint32_t tiles = 0;
    double flops = 0.0, bytes = 0.0;
    constexpr uint32_t COLS = EPI == kFfGate ? BN / 2 : BN;
    a.ksteps = a.p[0].ktiles * a.p[0].nseg;
    for (uint32_t i = 0; i < a.count; ++i) {
        FfProblem& p = a.p[i];
        p.tiles_m = (p.M + BM - 1) / BM;
        p.tiles_n = (p.N + COLS - 1) / COLS;
        p.first = tiles;
        tiles += p.tiles_m * p.tiles_n;
        const double k = static_cast<double>(a.ksteps) * kFfBk, both = EPI == kFfGate ? 2.0 : 1.0;
        flops += 2.0 * p.M * p.N * k * both;
        bytes += 2.0 * (p.M + p.N * both) * k;
    }
    const uint32_t places = static_cast<uint32_t>(ctx->num_cu) * blocks_per_cu(BM, BN);
    a.whole = tiles / places * places;
    a.rest = tiles - a.whole;
    a.workers = static_cast<uint32_t>(std::min<uint64_t>(places, static_cast<uint64_t>(a.rest) * a.ksteps * kFfBk / kMinK));
    // dgate: where there are few tiles the join, whose blocks have a square of four waves each, gets through the long epilogue sooner
    // than the tile's four waves, and two workers a tile will do (841 tokens, 320 x 279, bf16: 14 us, one worker 31)
    if (EPI == kFfDgate && a.ksteps >= 2 && a.rest * 2 <= places) a.workers = std::max(a.workers, a.rest * 2);
    // (A last round that is nearly full is not worth the sums' way through memory.  The rule does not know k: where a tile has few steps the sums
    // cost more than the sharing saves.  1888 tokens, 704 x 6026, bf16, projections: 11 steps, 128 of 384 tiles shared by 176 workers, joins
    // 27 us in a pass whose products take 63 and 28.)
    if (a.workers <= a.rest || a.rest * 10ull > places * 9ull) a.whole = tiles, a.rest = a.workers = 0;
    a.part = ctx->ff.part;
    constexpr uint32_t lds = lds_bytes(BM, BN);
    EDGC_LAUNCH(ctx, st, kid, bytes, flops, k_ff_gemm<BM, BN, TA, TB, T, EPI><<<a.whole + a.workers, 256, lds, st>>>(a));
    EDGC_HIP_TRY(ctx, hipGetLastError());
    if (a.rest) {
        EDGC_LAUNCH(ctx, st, KID_FF_JOIN, 4.0 * BM * BN * (a.workers + a.rest), 0.0,
                    k_ff_join<BM, BN, T, EPI><<<a.rest * (BM / 64) * (BN / (EPI == kFfGate ? 128 : 64)), 256, 0, st>>>(a));
        EDGC_HIP_TRY(ctx, hipGetLastError());
    }
    return EDGC_OK;
}

// Sums that workers can leave behind: at most two per place of the larger tile shape
uint64_t part_elems(const edgc_ctx* ctx) { return 2ull * ctx->num_cu * std::max(256 * 256 * blocks_per_cu(256, 256), 128 * 128 * blocks_per_cu(128, 128)); }

template <bool TA, bool TB, typename T, int EPI>
int launch_product(edgc_ctx* ctx, FfArgs& a, int kid, hipStream_t st)
{
    // The time that either tile shape would take, in steps of 64 k of a 256 x 256 tile on a compute unit.  Measured: a tile of 128 x 128
    // has a quarter of the work and gets it done at 0.65 of the rate.
    auto time_of = [&](uint64_t bm, uint64_t bn, double step) {
        uint64_t tiles = 0;
        for (uint32_t i = 0; i < a.count; ++i) tiles += ((a.p[i].M + bm - 1) / bm) * ((a.p[i].N + bn - 1) / bn);
        const uint64_t steps = static_cast<uint64_t>(a.p[0].ktiles) * a.p[0].nseg, places = static_cast<uint64_t>(ctx->num_cu) * blocks_per_cu(bm, bm);
        const double each = static_cast<double>(tiles * steps) / places;
        return step * std::max(each, static_cast<double>(std::min<uint64_t>(steps, kMinK / kFfBk)));
    };
    constexpr uint64_t half = EPI == kFfGate ? 2 : 1;
    if (time_of(256, 256 / half, 1.0) <= time_of(128, 128 / half, 0.25 * blocks_per_cu(128, 128) / 0.65))
        return launch_tiles<256, 256, TA, TB, T, EPI>(ctx, a, kid, st);
    return launch_tiles<128, 128, TA, TB, T, EPI>(ctx, a, kid, st);
}

template <int BM, int BN, typename T>
hipError_t prepare_tiles()
{
    for (const void* f : {reinterpret_cast<const void*>(&k_ff_gemm<BM, BN, false, false, T, kFfStore>),
                          reinterpret_cast<const void*>(&k_ff_gemm<BM, BN, false, true, T, kFfStore>),
                          reinterpret_cast<const void*>(&k_ff_gemm<BM, BN, true, true, T, kFfStore>),
                          reinterpret_cast<const void*>(&k_ff_gemm<BM, BN, false, false, T, kFfGate>),
                          reinterpret_cast<const void*>(&k_ff_gemm<BM, BN, false, true, T, kFfDgate>)})
        if (hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes(BM, BN))) return e;
    return hipSuccess;
}

// Segments of a sum over k: one for bf16, six products of planes for fp32, the smallest first
void add_segments(FfProblem& p, const Operand& a, const Operand& b, const Operand* b2, uint64_t planes)
{
    static const int order[6][2] = {{0, 2}, {2, 0}, {1, 1}, {0, 1}, {1, 0}, {0, 0}};
    for (int s = planes == 1 ? 5 : 0; s < 6; ++s) {
        const int i = order[s][0], j = order[s][1];
        p.a[p.nseg] = a.p + i * a.plane;
        p.b[p.nseg] = b.p + j * b.plane;
        p.b2[p.nseg] = b2 ? b2->p + j * b2->plane : nullptr;
        ++p.nseg;
    }
    p.lda = a.ld;
    p.ldb = b.ld;
}

template <typename T>
struct FfPass {
    static constexpr int P = FfType<T>::kPlanes;
    edgc_ctx* ctx;
    uint16_t* ws;
    Packer pk;
    FfPass(edgc_ctx* c, hipStream_t s) : ctx(c), ws(static_cast<uint16_t*>(c->ff.ws)), pk{c, s} {}

    // a matrix in the scratch
    Operand own(uint64_t at, uint64_t rows, uint64_t cols) const { return {ws + at, pad64(cols), pad64(rows) * pad64(cols)}; }
    // Whether a caller's matrix can be an operand as it stands, with k along its columns, its rows, or (in two products) either:
    // whole 16-byte units, whole tiles of 64 k
    static bool stands(const void* src, uint64_t ld, uint64_t rows, uint64_t cols, bool k_cols, bool k_rows)
    {
        return P == 1 && aligned_to(src, 16) && ld % 8 == 0 && ld <= kFfMaxLd && cols % (k_cols ? 64 : 8) == 0 && (!k_rows || rows % 64 == 0);
    }
    // it, or a copy of it
    Operand operand(const void* src, uint64_t ld, uint64_t rows, uint64_t cols, bool as_it_stands, uint64_t at)
    {
        if (as_it_stands) return {static_cast<const uint16_t*>(src), ld, 0};
        pk.add(src, ld, rows, cols, ws + at);
        return own(at, rows, cols);
    }
    Operand operand(const void* src, uint64_t ld, uint64_t rows, uint64_t cols, bool k_cols, bool k_rows, uint64_t at)
    {
        return operand(src, ld, rows, cols, stands(src, ld, rows, cols, k_cols, k_rows), at);
    }
    // the weights of the two projections: one leading dimension for both
    std::pair<Operand, Operand> projections(const edgc_ff& w, bool k_cols, const FfPlan& plan)
    {
        const bool both = w.ld_gate == w.ld_up && stands(w.w_gate, w.ld_gate, w.ff, w.hidden, k_cols, !k_cols) &&
                          stands(w.w_up, w.ld_up, w.ff, w.hidden, k_cols, !k_cols);
        return {operand(w.w_gate, w.ld_gate, w.ff, w.hidden, both, plan.wg), operand(w.w_up, w.ld_up, w.ff, w.hidden, both, plan.wu)};
    }
};

// Few tokens.  About 16 waves on a compute unit, each with eight steps of k at least: 4 to 16 waves of a block share k, and where there
// are fewer blocks than compute units eight waves and up to four blocks.  (24 tokens, fp32, 2048 rows of 8192: 128 blocks of 16 waves
// 45 us, 512 of 8 28; one token, bf16, 4096 rows of 16384: 256 of 16 29.4 us, 512 of 8 30.8.)
template <typename T, bool GATED>
int launch_few(edgc_ctx* ctx, FfFewArgs& a, int kid, hipStream_t st)
{
    const uint32_t blocks = (a.N + 15) / 16, steps = (a.K + FfFew<T>::kStep - 1) / FfFew<T>::kStep, cu = static_cast<uint32_t>(ctx->num_cu);
    uint32_t waves = 4, splits = 1;
    while (waves < (blocks < cu || a.tokens > 32 ? 8u : 16u) && blocks * waves < cu * 16 && steps >= waves * 16) waves *= 2;
    while (splits < kFfFewSplits && blocks < cu && blocks * splits < cu * 2 && steps >= waves * splits * 16) splits *= 2;
    a.part = ctx->ff.part;
    a.tickets = ctx->ff.tickets;
    const double mats = GATED ? 2.0 : 1.0;
    auto go = [&](auto groups) {
        constexpr int G = decltype(groups)::value;
        const uint32_t lds = waves * (GATED ? 2 : 1) * G * 64 * 16;
        EDGC_LAUNCH(ctx, st, kid, sizeof(T) * mats * a.N * a.K, 2.0 * mats * a.tokens * a.N * a.K,
                    k_ff_few<T, G, GATED><<<dim3(blocks, splits), waves * 64, lds, st>>>(a));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        return static_cast<int>(EDGC_OK);
    };
    if (a.tokens <= 16) return go(std::integral_constant<int, 1>{});
    if (a.tokens <= 32) return go(std::integral_constant<int, 2>{});
    if constexpr (kFfFewTokens<T> > 32) return go(std::integral_constant<int, 4>{});
    else return static_cast<int>(EDGC_EINVAL);      // (not reached)
}

template <typename T, int GROUPS>
hipError_t prepare_few()
{
    for (const void* f : {reinterpret_cast<const void*>(&k_ff_few<T, GROUPS, false>), reinterpret_cast<const void*>(&k_ff_few<T, GROUPS, true>)})
        if (hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, kFfFewWaves<GROUPS> * 2 * GROUPS * 1024)) return e;
    return hipSuccess;
}

template <typename T>
int ff_forward_few(edgc_ctx* ctx, const edgc_ff& w, const void* x, uint64_t ldx, uint32_t tokens, void* y, uint64_t ldy, void* gate, void* up,
                   uint64_t ldg, hipStream_t st)
{
    FfFewArgs a{};
    a.x = x; a.ldx = ldx; a.w = w.w_gate; a.w2 = w.w_up; a.ldw = w.ld_gate; a.ldw2 = w.ld_up;
    a.tokens = tokens; a.N = w.ff; a.K = w.hidden; a.act = w.act;
    a.out = ctx->ff.ws; a.ldo = w.ff; a.keep = gate; a.keep2 = up; a.ldk = ldg;
    if (int rc = launch_few<T, true>(ctx, a, KID_FF_GATE, st)) return rc;
    FfFewArgs b{};
    b.x = ctx->ff.ws; b.ldx = w.ff; b.w = w.w_down; b.ldw = w.ld_down;
    b.tokens = tokens; b.N = w.hidden; b.K = w.ff; b.out = y; b.ldo = ldy;
    return launch_few<T, false>(ctx, b, KID_FF_DOWN, st);
}

template <typename T>
int ff_forward(edgc_ctx* ctx, const edgc_ff& w, const void* x, uint64_t ldx, uint64_t tokens, void* y, uint64_t ldy, void* gate, void* up,
               uint64_t ldg, hipStream_t st)
{
    if (tokens <= kFfFewTokens<T>) return ff_forward_few<T>(ctx, w, x, ldx, static_cast<uint32_t>(tokens), y, ldy, gate, up, ldg, st);
    constexpr int P = FfType<T>::kPlanes;
    const uint64_t H = w.hidden, F = w.ff;
    FfPlan plan(tokens, H, F, w.dtype);
    plan.forward();
    FfPass<T> pass(ctx, st);
    const Operand ox = pass.operand(x, ldx, tokens, H, true, false, plan.x);
    const auto [og, ou] = pass.projections(w, true, plan);
    const Operand od = pass.operand(w.w_down, w.ld_down, H, F, true, false, plan.wd), oh = pass.own(plan.h, tokens, F);
    if (int rc = pass.pk.template flush<T>()) return rc;
    FfArgs a{};
    a.count = 1;
    FfProblem& p = a.p[0];
    add_segments(p, ox, og, &ou, P);
    p.M = static_cast<uint32_t>(tokens); p.N = w.ff; p.ktiles = static_cast<uint32_t>(plan.H / kFfBk);
    p.out = pass.ws + plan.h; p.ldo = oh.ld; p.plane = oh.plane; p.n_pad = static_cast<uint32_t>(plan.F); p.m_pad = p.M;
    p.e0 = gate; p.e1 = up; p.lde = ldg; p.act = w.act;
    if (int rc = launch_product<false, false, T, kFfGate>(ctx, a, KID_FF_GATE, st)) return rc;
    FfArgs b{};
    b.count = 1;
    FfProblem& q = b.p[0];
    add_segments(q, oh, od, nullptr, P);
    q.M = static_cast<uint32_t>(tokens); q.N = w.hidden; q.ktiles = static_cast<uint32_t>(plan.F / kFfBk);
    q.out = y; q.ldo = ldy;
    return launch_product<false, false, T, kFfStore>(ctx, b, KID_FF_DOWN, st);
}

template <typename T>
int ff_backward(edgc_ctx* ctx, const edgc_ff& w, const void* x, uint64_t ldx, uint64_t tokens, const void* gate, const void* up, uint64_t ldg,
                const void* dy, uint64_t ldy, void* dx, uint64_t lddx, void* dwg, uint64_t lddg, void* dwu, uint64_t lddu, void* dwd,
                uint64_t lddd, int accumulate, hipStream_t st)
{
    constexpr int P = FfType<T>::kPlanes;
    const uint64_t H = w.hidden, F = w.ff;
    FfPlan plan(tokens, H, F, w.dtype);
    plan.backward();
    FfPass<T> pass(ctx, st);
    const Operand ody = pass.operand(dy, ldy, tokens, H, true, true, plan.dy), ox = pass.operand(x, ldx, tokens, H, false, true, plan.x),
                  od = pass.operand(w.w_down, w.ld_down, H, F, false, true, plan.wd), oh = pass.own(plan.h, tokens, F),
                  odg = pass.own(plan.dg, tokens, F), odu = pass.own(plan.du, tokens, F);
    const auto [og, ou] = pass.projections(w, false, plan);
    if (int rc = pass.pk.template flush<T>()) return rc;
    {
        FfArgs a{};
        a.count = 1;
        FfProblem& p = a.p[0];
        add_segments(p, ody, od, nullptr, P);
        p.M = static_cast<uint32_t>(tokens); p.N = w.ff; p.ktiles = static_cast<uint32_t>(plan.H / kFfBk);
        p.out = pass.ws + plan.h; p.o1 = pass.ws + plan.dg; p.o2 = pass.ws + plan.du;
        p.ldo = oh.ld; p.plane = oh.plane; p.n_pad = static_cast<uint32_t>(plan.F); p.m_pad = static_cast<uint32_t>(plan.T);
        p.e0 = const_cast<void*>(gate); p.e1 = const_cast<void*>(up); p.lde = ldg; p.act = w.act;
        if (int rc = launch_product<false, true, T, kFfDgate>(ctx, a, KID_FF_DGATE, st)) return rc;
    }
    {
        FfArgs a{};
        a.count = 1;
        FfProblem& p = a.p[0];
        add_segments(p, odg, og, nullptr, P);
        add_segments(p, odu, ou, nullptr, P);
        p.M = static_cast<uint32_t>(tokens); p.N = w.hidden; p.ktiles = static_cast<uint32_t>(plan.F / kFfBk);
        p.out = dx; p.ldo = lddx;
        if (int rc = launch_product<false, true, T, kFfStore>(ctx, a, KID_FF_DX, st)) return rc;
    }
    FfArgs a{};
    a.count = 3;
    const Operand left[3] = {odg, odu, ody}, right[3] = {ox, ox, oh};
    void* const out[3] = {dwg, dwu, dwd};
    const uint64_t ldo[3] = {lddg, lddu, lddd};
    for (int i = 0; i < 3; ++i) {
        FfProblem& p = a.p[i];
        add_segments(p, left[i], right[i], nullptr, P);
        p.M = i < 2 ? w.ff : w.hidden; p.N = i < 2 ? w.hidden : w.ff;
        p.ktiles = static_cast<uint32_t>(plan.T / kFfBk);
        p.out = out[i]; p.ldo = ldo[i]; p.accumulate = accumulate ? 1 : 0;
    }
    return launch_product<true, true, T, kFfStore>(ctx, a, KID_FF_DW, st);
}

// zeros in a matrix (the weight gradients of no tokens)
__global__ __launch_bounds__(256) void k_ff_zero(uint16_t* p, uint64_t ld, uint32_t rows, uint64_t cols)
{
    for (uint32_t r = blockIdx.y; r < rows; r += gridDim.y)
        for (uint64_t c = blockIdx.x * 256ull + threadIdx.x; c < cols; c += gridDim.x * 256ull) p[r * ld + c] = 0;
}

int check_ff(edgc_ctx* ctx, const edgc_ff* w, uint64_t tokens, bool backward)
{
    if (!w) return fail(ctx, EDGC_EINVAL, "null edgc_ff");
    if (w->dtype != EDGC_F32 && w->dtype != EDGC_BF16) return fail(ctx, EDGC_EINVAL, "unknown dtype");
    if (w->act != EDGC_SILU && w->act != EDGC_GELU && w->act != EDGC_GELU_TANH) return fail(ctx, EDGC_EINVAL, "unknown activation");
    if (w->hidden == 0 || w->ff == 0 || w->hidden > kFfMaxWidth || w->ff > kFfMaxWidth) return fail(ctx, EDGC_EINVAL, "hidden and ff must be 1 to 2^20");
    if (tokens > kFfMaxTokens) return fail(ctx, EDGC_EINVAL, "more than 2^21 tokens");
    const size_t esz = w->dtype == EDGC_F32 ? 4 : 2;
    if (!w->w_gate || !w->w_up || !w->w_down || !aligned_to(w->w_gate, esz) || !aligned_to(w->w_up, esz) || !aligned_to(w->w_down, esz))
        return fail(ctx, EDGC_EINVAL, "null or misaligned weight");
    if (w->ld_gate < w->hidden || w->ld_up < w->hidden || w->ld_down < w->ff || w->ld_gate > kMaxSpan || w->ld_up > kMaxSpan || w->ld_down > kMaxSpan)
        return fail(ctx, EDGC_EINVAL, "leading dimension of a weight too small, or over 2^40");
    if (tokens) {
        FfPlan plan(tokens, w->hidden, w->ff, w->dtype);
        if ((backward ? plan.backward() : plan.forward()) > ctx->ff.elems)
            return fail(ctx, EDGC_EINVAL, "larger than what edgc_reserve_ff was called for");
    }
    return EDGC_OK;
}
int check_rows(edgc_ctx* ctx, const void* p, uint64_t ld, uint64_t cols, size_t esz)
{
    if (!p || !aligned_to(p, esz)) return fail(ctx, EDGC_EINVAL, "null or misaligned pointer");
    if (ld < cols || ld > kMaxSpan) return fail(ctx, EDGC_EINVAL, "leading dimension too small, or over 2^40");
    return EDGC_OK;
}

}  // namespace

int prepare_ff_kernels(edgc_ctx* ctx)
{
    hipError_t e = prepare_tiles<256, 256, __bf16>();
    if (e == hipSuccess) e = prepare_tiles<256, 256, float>();
    if (e == hipSuccess) e = prepare_few<__bf16, 1>();
    if (e == hipSuccess) e = prepare_few<__bf16, 2>();
    if (e == hipSuccess) e = prepare_few<float, 1>();
    if (e == hipSuccess) e = prepare_few<float, 2>();
    if (e == hipSuccess) e = prepare_few<float, 4>();
    EDGC_HIP_TRY(ctx, e);
    return EDGC_OK;
}

}  // namespace edgc

using namespace edgc;

extern "C" int edgc_reserve_ff(edgc_ctx* ctx, edgc_dtype dtype, uint32_t tokens, uint32_t hidden, uint32_t ff, int backward)
{
    if (!ctx) return EDGC_EINVAL;
    if (dtype != EDGC_F32 && dtype != EDGC_BF16) return fail(ctx, EDGC_EINVAL, "unknown dtype");
    if (hidden == 0 || ff == 0 || hidden > kFfMaxWidth || ff > kFfMaxWidth || tokens > kFfMaxTokens)
        return fail(ctx, EDGC_EINVAL, "hidden and ff must be 1 to 2^20, tokens at most 2^21");
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    FfPlan plan(tokens, hidden, ff, dtype);
    uint64_t elems = tokens ? plan.forward() : 0;
    if (tokens && backward) elems = std::max(elems, plan.backward());
    if (elems && elems <= ctx->ff.held) {
        ctx->ff.elems = elems;
        return EDGC_OK;
    }
    EDGC_HIP_TRY(ctx, hipDeviceSynchronize());          // nothing may still be using the old scratch
    if (ctx->ff.ws) (void)hipFree(ctx->ff.ws);
    if (ctx->ff.part) (void)hipFree(ctx->ff.part);
    ctx->ff = FfScratch{};
    if (elems == 0) return EDGC_OK;
    const uint64_t part_bytes = part_elems(ctx) * sizeof(float);
    bool ok = hipMalloc(&ctx->ff.ws, elems * 2) == hipSuccess;
    // the tickets lie behind the sums
    ok = ok && hipMalloc(reinterpret_cast<void**>(&ctx->ff.part), part_bytes + kFfFewBlocks * sizeof(unsigned int)) == hipSuccess;
    ctx->ff.tickets = reinterpret_cast<unsigned int*>(ctx->ff.part + part_elems(ctx));
    ok = ok && hipMemset(ctx->ff.tickets, 0, kFfFewBlocks * sizeof(unsigned int)) == hipSuccess && hipDeviceSynchronize() == hipSuccess;
    if (!ok) {
        (void)hipGetLastError();
        if (ctx->ff.ws) (void)hipFree(ctx->ff.ws);
        if (ctx->ff.part) (void)hipFree(ctx->ff.part);
        ctx->ff = FfScratch{};
        return fail(ctx, EDGC_ENOMEM, "feed-forward scratch allocation failed");
    }
    ctx->ff.elems = ctx->ff.held = elems;
    return EDGC_OK;
}

extern "C" int edgc_ff_forward(edgc_ctx* ctx, const edgc_ff* w, const void* x, uint64_t ldx, uint32_t tokens, void* y, uint64_t ldy,
                               void* gate, void* up, uint64_t ld_kept, void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    if (int rc = check_ff(ctx, w, tokens, false)) return rc;
    if (tokens == 0) return EDGC_OK;
    const size_t esz = w->dtype == EDGC_F32 ? 4 : 2;
    if (int rc = check_rows(ctx, x, ldx, w->hidden, esz)) return rc;
    if (int rc = check_rows(ctx, y, ldy, w->hidden, esz)) return rc;
    if (!gate != !up) return fail(ctx, EDGC_EINVAL, "gate and up are kept together");
    if (gate) {
        if (int rc = check_rows(ctx, gate, ld_kept, w->ff, esz)) return rc;
        if (int rc = check_rows(ctx, up, ld_kept, w->ff, esz)) return rc;
    }
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return w->dtype == EDGC_F32 ? ff_forward<float>(ctx, *w, x, ldx, tokens, y, ldy, gate, up, ld_kept, st)
                                : ff_forward<__bf16>(ctx, *w, x, ldx, tokens, y, ldy, gate, up, ld_kept, st);
}

extern "C" int edgc_ff_backward(edgc_ctx* ctx, const edgc_ff* w, const void* x, uint64_t ldx, uint32_t tokens, const void* gate,
                                const void* up, uint64_t ld_kept, const void* dy, uint64_t ldy, void* dx, uint64_t lddx, void* dw_gate,
                                uint64_t ld_dgate, void* dw_up, uint64_t ld_dup, void* dw_down, uint64_t ld_ddown, int accumulate,
                                void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    if (int rc = check_ff(ctx, w, tokens, true)) return rc;
    const size_t esz = w->dtype == EDGC_F32 ? 4 : 2;
    if (int rc = check_rows(ctx, dw_gate, ld_dgate, w->hidden, esz)) return rc;
    if (int rc = check_rows(ctx, dw_up, ld_dup, w->hidden, esz)) return rc;
    if (int rc = check_rows(ctx, dw_down, ld_ddown, w->ff, esz)) return rc;
    if (tokens) {
        if (int rc = check_rows(ctx, x, ldx, w->hidden, esz)) return rc;
        if (int rc = check_rows(ctx, dy, ldy, w->hidden, esz)) return rc;
        if (int rc = check_rows(ctx, dx, lddx, w->hidden, esz)) return rc;
        if (int rc = check_rows(ctx, gate, ld_kept, w->ff, esz)) return rc;
        if (int rc = check_rows(ctx, up, ld_kept, w->ff, esz)) return rc;
    }
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (tokens == 0) {
        if (accumulate) return EDGC_OK;
        const uint64_t u = esz / 2;
        k_ff_zero<<<dim3(4, std::min(w->ff, 65535u)), 256, 0, st>>>(static_cast<uint16_t*>(dw_gate), ld_dgate * u, w->ff, w->hidden * u);
        k_ff_zero<<<dim3(4, std::min(w->ff, 65535u)), 256, 0, st>>>(static_cast<uint16_t*>(dw_up), ld_dup * u, w->ff, w->hidden * u);
        k_ff_zero<<<dim3(4, std::min(w->hidden, 65535u)), 256, 0, st>>>(static_cast<uint16_t*>(dw_down), ld_ddown * u, w->hidden, w->ff * u);
        EDGC_HIP_TRY(ctx, hipGetLastError());
        return EDGC_OK;
    }
    return w->dtype == EDGC_F32 ? ff_backward<float>(ctx, *w, x, ldx, tokens, gate, up, ld_kept, dy, ldy, dx, lddx, dw_gate, ld_dgate, dw_up,
                                                     ld_dup, dw_down, ld_ddown, accumulate, st)
                                : ff_backward<__bf16>(ctx, *w, x, ldx, tokens, gate, up, ld_kept, dy, ldy, dx, lddx, dw_gate, ld_dgate,
                                                      dw_up, ld_dup, dw_down, ld_ddown, accumulate, st);
}
