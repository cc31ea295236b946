// The gated feed-forward block and its backward pass.
//
//   G = x Wg^T, U = x Wu^T, A = act(G) U, y = A Wd^T               (Wg, Wu: ff x hidden, Wd: hidden x ff)
//   dA = dy Wd;  dG = dA U act'(G), dU = dA act(G);  dx = dG Wg + dU Wu;  dWg = dG^T x, dWu = dU^T x, dWd = dy^T A
//
// Forward: one product whose tiles hold both projections and whose epilogue applies the activation and the product, and one for y.
// Backward: dA, whose epilogue makes dG, dU and A from the kept projections (dA itself is never stored), dx over both halves in one
// sum, and the three weight gradients in one launch.  Products: ff_gemm.h.  Operands that are not laid out for them (k contiguous
// and a multiple of 64, 16-byte aligned, bf16) are first copied into the reserved scratch, transposed or split where needed.
#include "ff_gemm.h"

#include <algorithm>
#include <cmath>

namespace edgc {
namespace {

// ---------------------------------------------------------------------------------------------
// Copies into operand form: 64 x 64 elements per block, up to kPacks matrices per launch
// ---------------------------------------------------------------------------------------------
constexpr int kPacks = 6;
struct PackItem {
    const void* src;
    uint16_t* dst;
    uint64_t ld, ldd, plane, src_plane;     // elements: of the source, the copy; between planes of the copy, of the source
    uint32_t rows, cols, tiles_c, first;    // of the source; tiles across; first block
    uint32_t trans;
};
struct PackList {
    PackItem t[kPacks];
    uint32_t count, blocks;
};

// T: element of the source; PLANES: what one element becomes
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void k_ff_pack(const PackList list)
{
    __shared__ uint16_t s[PLANES][64][66];
    uint32_t k = 0;
#pragma unroll
    for (int i = 1; i < kPacks; ++i) k += (static_cast<uint32_t>(i) < list.count && blockIdx.x >= list.t[i].first) ? 1u : 0u;
    const PackItem& t = list.t[k];
    const uint32_t id = blockIdx.x - t.first, r0 = id / t.tiles_c * 64, c0 = id % t.tiles_c * 64;
    const uint32_t cl = threadIdx.x % 64, rl = threadIdx.x / 64;
    const T* const src = static_cast<const T*>(t.src) + blockIdx.y * t.src_plane;
    uint16_t* const dst = t.dst + blockIdx.y * t.plane;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t r = rl + i * 4;
        uint16_t p[PLANES] = {};
        if (r0 + r < t.rows && c0 + cl < t.cols) {
            const T v = src[(r0 + r) * t.ld + c0 + cl];
            if constexpr (PLANES == 3) ff_planes(v, p);
            else p[0] = __builtin_bit_cast(uint16_t, v);
        }
#pragma unroll
        for (int q = 0; q < PLANES; ++q) s[q][r][cl] = p[q];
    }
    __syncthreads();
    // rows of the copy: source rows (columns of the source where transposed); zeros up to its padded length
    const uint32_t d0 = t.trans ? c0 : r0, e0 = t.trans ? r0 : c0, dn = t.trans ? t.cols : t.rows;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t r = rl + i * 4;
        if (d0 + r >= dn) continue;
#pragma unroll
        for (int q = 0; q < PLANES; ++q) dst[q * t.plane + (d0 + r) * t.ldd + e0 + cl] = t.trans ? s[q][cl][r] : s[q][r][cl];
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
    uint64_t T, H, F, Tp, Hp, Fp, planes, used = 0;
    FfPlan(uint64_t tokens, uint64_t hidden, uint64_t ff, edgc_dtype dt)
        : T(tokens), H(hidden), F(ff), Tp(pad64(tokens)), Hp(pad64(hidden)), Fp(pad64(ff)), planes(dt == EDGC_F32 ? 3 : 1) {}
    uint64_t take(uint64_t rows, uint64_t ld)
    {
        const uint64_t at = used;
        used += planes * rows * ld;         // (rows of 128 bytes: everything stays 16-byte aligned)
        return at;
    }
    // forward
    uint64_t x = 0, wg = 0, wu = 0, wd = 0, h = 0;
    uint64_t forward()
    {
        used = 0;
        x = take(T, Hp); wg = take(F, Hp); wu = take(F, Hp); wd = take(H, Fp); h = take(T, Fp);
        return used;
    }
    // backward
    uint64_t dy = 0, wdt = 0, dg = 0, du = 0, wgt = 0, wut = 0, ht = 0, dgt = 0, dut = 0, xt = 0, dyt = 0;
    uint64_t backward()
    {
        used = 0;
        dy = take(T, Hp); wdt = take(F, Hp); h = take(T, Fp); dg = take(T, Fp); du = take(T, Fp); wgt = take(H, Fp); wut = take(H, Fp);
        ht = take(F, Tp); dgt = take(F, Tp); dut = take(F, Tp); xt = take(H, Tp); dyt = take(H, Tp);
        return used;
    }
};

constexpr uint32_t kFfMaxTokens = 1u << 21, kFfMaxWidth = 1u << 20;

struct Packer {
    edgc_ctx* ctx;
    hipStream_t st;
    PackList list{};
    // copies rows x cols (ld) to `dst`, k padded; planes: of a source that is planes already
    void add(const void* src, uint64_t ld, uint64_t src_plane, uint64_t rows, uint64_t cols, bool trans, uint16_t* dst, uint64_t plane)
    {
        PackItem& t = list.t[list.count++];
        t.src = src; t.dst = dst; t.ld = ld; t.src_plane = src_plane;
        t.rows = static_cast<uint32_t>(rows); t.cols = static_cast<uint32_t>(cols);
        t.trans = trans; t.plane = plane; t.ldd = pad64(trans ? rows : cols);
        t.tiles_c = static_cast<uint32_t>(pad64(cols) / 64);
        t.first = list.blocks;
        list.blocks += static_cast<uint32_t>(pad64(rows) / 64) * t.tiles_c;
    }
    template <typename T, int PLANES>
    int flush(uint32_t z)
    {
        if (list.count == 0) return EDGC_OK;
        double bytes = 0.0;
        for (uint32_t i = 0; i < list.count; ++i)
            bytes += static_cast<double>(list.t[i].rows) * list.t[i].cols * z * (sizeof(T) + 2.0 * PLANES);
        EDGC_LAUNCH(ctx, st, KID_FF_PACK, bytes, 0.0, k_ff_pack<T, PLANES><<<dim3(list.blocks, z), 256, 0, st>>>(list));
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

template <int BM, int BN, typename T, int EPI>
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
    // (a last round that is nearly full is not worth the sums' way through memory)
    if (a.workers <= a.rest || a.rest * 10ull > places * 9ull) a.whole = tiles, a.rest = a.workers = 0;
    a.part = ctx->ff.part;
    constexpr uint32_t lds = lds_bytes(BM, BN);
    EDGC_LAUNCH(ctx, st, kid, bytes, flops, k_ff_gemm<BM, BN, T, EPI><<<a.whole + a.workers, 256, lds, st>>>(a));
    EDGC_HIP_TRY(ctx, hipGetLastError());
    if (a.rest) {
        EDGC_LAUNCH(ctx, st, KID_FF_JOIN, 4.0 * BM * BN * (a.workers + a.rest), 0.0,
                    k_ff_join<BM, BN, T, EPI><<<a.rest * (BM / 64) * (BN / 128), 256, 0, st>>>(a));
        EDGC_HIP_TRY(ctx, hipGetLastError());
    }
    return EDGC_OK;
}

// Sums that workers can leave behind: at most two per place of the larger tile shape
uint64_t part_elems(const edgc_ctx* ctx) { return 2ull * ctx->num_cu * std::max(256 * 256 * blocks_per_cu(256, 256), 128 * 128 * blocks_per_cu(128, 128)); }

template <typename T, int EPI>
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
        return launch_tiles<256, 256, T, EPI>(ctx, a, kid, st);
    return launch_tiles<128, 128, T, EPI>(ctx, a, kid, st);
}

template <int BM, int BN, typename T>
hipError_t prepare_tiles()
{
    const int lds = lds_bytes(BM, BN);
    for (const void* f : {reinterpret_cast<const void*>(&k_ff_gemm<BM, BN, T, kFfStore>), reinterpret_cast<const void*>(&k_ff_gemm<BM, BN, T, kFfGate>),
                          reinterpret_cast<const void*>(&k_ff_gemm<BM, BN, T, kFfDgate>)})
        if (hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, lds)) return e;
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
    hipStream_t st;
    uint16_t* ws;
    Packer pk;
    FfPass(edgc_ctx* c, hipStream_t s) : ctx(c), st(s), ws(static_cast<uint16_t*>(c->ff.ws)), pk{c, s} {}

    // a caller's matrix as an operand: as it stands where its rows allow it
    Operand operand(const void* src, uint64_t ld, uint64_t rows, uint64_t cols, bool trans, uint64_t at)
    {
        if (P == 1 && !trans && aligned_to(src, 16) && ld % 8 == 0 && cols % 64 == 0 && ld <= kFfMaxLd)
            return {static_cast<const uint16_t*>(src), ld, 0};
        const uint64_t ldd = pad64(trans ? rows : cols), plane = (trans ? cols : rows) * ldd;
        pk.add(src, ld, 0, rows, cols, trans, ws + at, plane);
        return {ws + at, ldd, plane};
    }
    // planes in the scratch, transposed
    Operand transposed(uint64_t from, uint64_t rows, uint64_t cols, uint64_t at)
    {
        const uint64_t ld = pad64(cols), ldd = pad64(rows), plane = cols * ldd;
        pk.add(ws + from, ld, rows * ld, rows, cols, true, ws + at, plane);
        return {ws + at, ldd, plane};
    }
};

template <typename T>
int ff_forward(edgc_ctx* ctx, const edgc_ff& w, const void* x, uint64_t ldx, uint64_t T_, void* y, uint64_t ldy, void* gate, void* up,
               uint64_t ldg, hipStream_t st)
{
    constexpr int P = FfType<T>::kPlanes;
    FfPlan plan(T_, w.hidden, w.ff, P == 3 ? EDGC_F32 : EDGC_BF16);
    plan.forward();
    FfPass<T> pass(ctx, st);
    const uint64_t H = w.hidden, F = w.ff;
    const Operand ox = pass.operand(x, ldx, T_, H, false, plan.x), og = pass.operand(w.w_gate, w.ld_gate, F, H, false, plan.wg),
                  ou = pass.operand(w.w_up, w.ld_up, F, H, false, plan.wu), od = pass.operand(w.w_down, w.ld_down, H, F, false, plan.wd);
    Operand og2 = og, ou2 = ou;
    if (og.ld != ou.ld) {       // one stride for both projections: copy what is not
        if (og.ld != plan.Hp) og2 = {pass.ws + plan.wg, plan.Hp, F * plan.Hp}, pass.pk.add(w.w_gate, w.ld_gate, 0, F, H, false, pass.ws + plan.wg, F * plan.Hp);
        if (ou.ld != plan.Hp) ou2 = {pass.ws + plan.wu, plan.Hp, F * plan.Hp}, pass.pk.add(w.w_up, w.ld_up, 0, F, H, false, pass.ws + plan.wu, F * plan.Hp);
    }
    if (int rc = pass.pk.template flush<T, P>(1)) return rc;
    FfArgs a{};
    a.count = 1;
    FfProblem& p = a.p[0];
    add_segments(p, ox, og2, &ou2, P);
    p.M = static_cast<uint32_t>(T_); p.N = w.ff; p.ktiles = static_cast<uint32_t>(plan.Hp / kFfBk);
    p.out = pass.ws + plan.h; p.ldo = plan.Fp; p.plane = T_ * plan.Fp; p.n_pad = static_cast<uint32_t>(plan.Fp);
    p.e0 = gate; p.e1 = up; p.lde = ldg; p.act = w.act;
    if (int rc = launch_product<T, kFfGate>(ctx, a, KID_FF_GATE, st)) return rc;
    FfArgs b{};
    b.count = 1;
    FfProblem& q = b.p[0];
    add_segments(q, {pass.ws + plan.h, plan.Fp, T_ * plan.Fp}, od, nullptr, P);
    q.M = static_cast<uint32_t>(T_); q.N = w.hidden; q.ktiles = static_cast<uint32_t>(plan.Fp / kFfBk);
    q.out = y; q.ldo = ldy;
    return launch_product<T, kFfStore>(ctx, b, KID_FF_DOWN, st);
}

template <typename T>
int ff_backward(edgc_ctx* ctx, const edgc_ff& w, const void* x, uint64_t ldx, uint64_t T_, const void* gate, const void* up, uint64_t ldg,
                const void* dy, uint64_t ldy, void* dx, uint64_t lddx, void* dwg, uint64_t lddg, void* dwu, uint64_t lddu, void* dwd,
                uint64_t lddd, int accumulate, hipStream_t st)
{
    constexpr int P = FfType<T>::kPlanes;
    FfPlan plan(T_, w.hidden, w.ff, P == 3 ? EDGC_F32 : EDGC_BF16);
    plan.backward();
    FfPass<T> pass(ctx, st);
    const uint64_t H = w.hidden, F = w.ff;
    const Operand ody = pass.operand(dy, ldy, T_, H, false, plan.dy), owd = pass.operand(w.w_down, w.ld_down, H, F, true, plan.wdt),
                  owg = pass.operand(w.w_gate, w.ld_gate, F, H, true, plan.wgt), owu = pass.operand(w.w_up, w.ld_up, F, H, true, plan.wut),
                  oxt = pass.operand(x, ldx, T_, H, true, plan.xt), odyt = pass.operand(dy, ldy, T_, H, true, plan.dyt);
    if (int rc = pass.pk.template flush<T, P>(1)) return rc;
    {
        FfArgs a{};
        a.count = 1;
        FfProblem& p = a.p[0];
        add_segments(p, ody, owd, nullptr, P);
        p.M = static_cast<uint32_t>(T_); p.N = w.ff; p.ktiles = static_cast<uint32_t>(plan.Hp / kFfBk);
        p.out = pass.ws + plan.h; p.o1 = pass.ws + plan.dg; p.o2 = pass.ws + plan.du;
        p.ldo = plan.Fp; p.plane = T_ * plan.Fp; p.n_pad = static_cast<uint32_t>(plan.Fp);
        p.e0 = const_cast<void*>(gate); p.e1 = const_cast<void*>(up); p.lde = ldg; p.act = w.act;
        if (int rc = launch_product<T, kFfDgate>(ctx, a, KID_FF_DGATE, st)) return rc;
    }
    const Operand oht = pass.transposed(plan.h, T_, F, plan.ht), odgt = pass.transposed(plan.dg, T_, F, plan.dgt),
                  odut = pass.transposed(plan.du, T_, F, plan.dut);
    if (int rc = pass.pk.template flush<__bf16, 1>(P)) return rc;
    {
        FfArgs a{};
        a.count = 1;
        FfProblem& p = a.p[0];
        add_segments(p, {pass.ws + plan.dg, plan.Fp, T_ * plan.Fp}, owg, nullptr, P);
        add_segments(p, {pass.ws + plan.du, plan.Fp, T_ * plan.Fp}, owu, nullptr, P);
        p.M = static_cast<uint32_t>(T_); p.N = w.hidden; p.ktiles = static_cast<uint32_t>(plan.Fp / kFfBk);
        p.out = dx; p.ldo = lddx;
        if (int rc = launch_product<T, kFfStore>(ctx, a, KID_FF_DX, st)) return rc;
    }
    FfArgs a{};
    a.count = 3;
    const Operand left[3] = {odgt, odut, odyt}, right[3] = {oxt, oxt, oht};
    void* const out[3] = {dwg, dwu, dwd};
    const uint64_t ldo[3] = {lddg, lddu, lddd};
    for (int i = 0; i < 3; ++i) {
        FfProblem& p = a.p[i];
        add_segments(p, left[i], right[i], nullptr, P);
        p.M = i < 2 ? w.ff : w.hidden; p.N = i < 2 ? w.hidden : w.ff;
        p.ktiles = static_cast<uint32_t>(plan.Tp / kFfBk);
        p.out = out[i]; p.ldo = ldo[i]; p.accumulate = accumulate ? 1 : 0;
    }
    return launch_product<T, kFfStore>(ctx, a, KID_FF_DW, st);
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
    EDGC_HIP_TRY(ctx, hipDeviceSynchronize());          // nothing may still be using the old scratch
    if (ctx->ff.ws) (void)hipFree(ctx->ff.ws);
    if (ctx->ff.part) (void)hipFree(ctx->ff.part);
    ctx->ff = FfScratch{};
    if (tokens == 0) return EDGC_OK;
    FfPlan plan(tokens, hidden, ff, dtype);
    uint64_t elems = plan.forward();
    if (backward) elems = std::max(elems, plan.backward());
    if (hipMalloc(&ctx->ff.ws, elems * 2) != hipSuccess || hipMalloc(reinterpret_cast<void**>(&ctx->ff.part), part_elems(ctx) * sizeof(float)) != hipSuccess) {
        (void)hipGetLastError();
        if (ctx->ff.ws) (void)hipFree(ctx->ff.ws);
        ctx->ff = FfScratch{};
        return fail(ctx, EDGC_ENOMEM, "feed-forward scratch allocation failed");
    }
    ctx->ff.elems = elems;
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
