// The matrix products of the gated feed-forward block: C[m][n] = sum over segments and k of A[m][k] B[n][k], both operands bf16 with
// 16-byte aligned rows and k a multiple of 64.  Either lies in memory with k along its rows, or (TA, TB) as its transpose, m or n
// along the rows.
//
// fp32 operands come as three bf16 planes that add up to them exactly (24 significant bits = 3 x 8: a plane is the value's leading
// bits, cut off, not rounded); six products of planes are six segments of one sum.  The other three are left out: always of the
// product's sign, below 2^-21 of it and 2^-24.5 in the mean over normal operands.  Six bf16 MFMAs take less time than one of fp32 (2.5e15 / 6
// against 0.16e15 operations a second).
//
// A block of 2 x 2 waves makes a BM x BN tile; tiles of 64 k of the operands come straight to LDS while earlier ones are multiplied.  A
// row of 128 bytes lies there as eight 16-byte units, unit c at c ^ (row / 2 & 7): a read of 16 bytes per lane takes lanes 0-3, 12-15
// and 20-27 of either half at once, then the other sixteen, and their rows then lie in different banks.  (At c ^ (row & 7) half of
// LDS's cycles were conflicts.)  A transposed operand lies there as it does in memory, 64 rows of k, and is read by the instruction
// that transposes: of 16 lanes, lane s brings four neighbours of row s / 4, and lane d gets element d of the four rows' 16.  Its 32-byte
// pieces c of row k lie at c ^ (2 (k & 3) + (k / 8 & 1)), so that the rows that lanes 0-31, and lanes 0-15 and 32-47, take are in
// different banks.  The MFMA's first operand is B: a lane then holds four neighbouring n of one m, which is what the epilogues load
// and store.
//
// Bounded by the matrix instructions at the clock that the card's power allows (1.6 to 1.9 GHz of 2.4; a loop of them without any
// loads: 1390 TFLOP/s).  Measured: 4096 x 16384 bf16, 4096 tokens: dgate 643 us (855 TFLOP/s: a quarter of it is the epilogue, 640 KB
// a tile, in all tiles at once), dx 840 (1310), dw 1370 (1205); 5120 x 20480, 8192 tokens: gate 2910 (1180), down 1275 (1350).  fp32,
// 2048 tokens of 2048 x 8192, in products of planes: dgate 410 (1005; 1.6 MB a tile), dx 635 (1300), dw 975 (1270).
#pragma once

#include "compress_common.h"

#include <type_traits>

namespace edgc {

constexpr int kFfBk = 64;               // operands' k are padded to a multiple of this
constexpr int kFfSegs = 12;
constexpr uint64_t kFfMaxLd = 1ull << 22;   // rows of a tile are addressed in 32 bits from its first

struct FfProblem {
    const uint16_t* a[kFfSegs];         // per segment
    const uint16_t* b[kFfSegs];
    const uint16_t* b2[kFfSegs];        // the gated form: the second matrix of the same shape as b
    uint64_t lda, ldb;                  // elements
    uint32_t M, N;                      // of the output (gated: N columns of each of the two)
    uint32_t ktiles, nseg;              // times 64 k of a segment; segments
    uint32_t tiles_m, tiles_n, first;   // tiles of the output; first block
    uint32_t accumulate;
    void* out;                          // store: the output; gate, dgate: planes of h
    uint64_t ldo;
    // gate: h -> out, the projections -> e0, e1 where given.  dgate: the projections <- e0, e1; their gradients' planes -> o1, o2
    void *e0, *e1, *o1, *o2;
    uint64_t lde;
    uint64_t plane;                     // elements between planes of out, o1, o2
    uint32_t n_pad, m_pad;              // columns and rows of out, o1, o2: those from N and M on are zeros
    int32_t act;
};
constexpr int kFfProblems = 3;
// The tiles of the output that make whole rounds of the compute units are a block each.  The rest's steps of k are shared evenly by
// `workers` further blocks, so that all of them end together; a worker goes through its steps tile by tile, and leaves the sums of
// tiles that it has a part of in `part` (slot: worker + tile), where k_ff_join adds them up.
struct FfArgs {
    FfProblem p[kFfProblems];
    uint32_t count, whole;              // problems; tiles of a block each
    uint32_t rest, workers, ksteps;     // the other tiles; blocks that share them; steps of k of a tile (the same in all problems)
    float* part;                        // [workers + rest][BM * BN]
};
// steps of worker w: [ff_share(w), ff_share(w + 1)) of rest * ksteps
__host__ __device__ inline uint64_t ff_share(const FfArgs& a, uint32_t w)
{
    return static_cast<uint64_t>(a.rest) * a.ksteps * w / a.workers;
}

enum FfEpi { kFfStore = 0, kFfGate = 1, kFfDgate = 2 };

// Activation and derivative.  gelu_tanh by the identity (1 + tanh t) / 2 = 1 / (1 + exp(-2 t)).  The hardware's powers of two and
// reciprocals, exact to an ulp: an epilogue of library calls took a quarter of the time of the products of a tile of 5120 k.
__device__ __forceinline__ float ff_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z)); }
__device__ __forceinline__ void ff_act(int act, float z, float& a, float& da)
{
    if (act == EDGC_SILU) {
        const float s = ff_sigmoid(z);
        a = z * s;
        da = s * (1.0f + z * (1.0f - s));
    } else if (act == EDGC_GELU) {
        // Phi(-|z|) = exp(-z^2 / 2) t p(t), t = 1 / (1 + |z| / sqrt 8): p by least squares of the relative error, weighted towards its
        // peaks (9.4e-8 of the result up to |z| = 20; 1.8e-7 absolute with fp32's roundings).  The library's function took
        // 3.23 ms instead of 3.09 in the projections of 8192 tokens, 5120 x 20480 (SiLU 2.97).
        constexpr float p[9] = {1.410421729e-01f, 1.412060559e-01f, 1.214175522e-01f,
                                1.018762514e-01f, -1.457415149e-02f, 1.408663541e-01f,
                                -2.452028543e-01f, 1.430617869e-01f, -2.969318256e-02f};
        const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.35355339059327376f, 1.0f)), e = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
        float q = p[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) q = fmaf(q, t, p[i]);
        q *= t * e;
        const float cdf = z < 0.f ? q : 1.0f - q;
        a = z * cdf;
        da = cdf + z * e * 0.39894228040143268f;
    } else {
        const float k = 0.79788456080286536f, c = 0.044715f;
        const float s = ff_sigmoid(2.0f * k * (z + c * z * z * z));
        // (from the middle outwards: t is zero long before z^2 overflows)
        const float t = z * s * (1.0f - s);
        a = z * s;
        da = s + 2.0f * k * (t + 3.0f * c * (t * z) * z);
    }
}

// x = p[0] + p[1] + p[2] in bf16, exactly (unless its last bits lie below bf16's smallest number: |x| under 2^-110).  What is not finite is plane 0 alone.
__device__ __forceinline__ void ff_planes(float x, uint16_t (&p)[3])
{
    const uint32_t u = __float_as_uint(x);
    if ((u & 0x7f800000u) == 0x7f800000u) {
        p[0] = static_cast<uint16_t>((u >> 16) | ((u & 0x7fffffu) ? 0x40u : 0u));
        p[1] = p[2] = 0;
        return;
    }
    const uint32_t h = u & 0xffff0000u;
    const float r = x - __uint_as_float(h);
    const uint32_t m = __float_as_uint(r) & 0xffff0000u;
    p[0] = static_cast<uint16_t>(h >> 16);
    p[1] = static_cast<uint16_t>(m >> 16);
    p[2] = static_cast<uint16_t>(__float_as_uint(r - __uint_as_float(m)) >> 16);
}

// T's planes of four values, to planes `plane` elements apart.  bf16 has one: A, dG and dU are rounded to 8 bits as operands of the next
// product, as the matrix instruction takes them; a second plane would double that product.  With the output's own rounding errors
// in the norm are 0.0023 of it instead of 0.0017 (8192 tokens, 5120 x 20480; the plain form rounds the output alone).
template <typename T> struct FfType;
template <> struct FfType<__bf16> {
    static constexpr int kPlanes = 1;
    static __device__ __forceinline__ void put4(uint16_t* to, uint64_t, const float (&v)[4])
    {
        uint32_t a[1], b[1];
        pack_pair<1>(v[0], v[1], a);
        pack_pair<1>(v[2], v[3], b);
        put_any(to, Bf16Quad{a[0], b[0]});
    }
    static __device__ __forceinline__ Bf16Quad load4(const __bf16* p) { return at_any<Bf16Quad>(p); }
    static __device__ __forceinline__ void widen(const Bf16Quad& q, float (&v)[4])
    {
        v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xffff0000u);
        v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xffff0000u);
    }
    static __device__ __forceinline__ void store4(__bf16* p, const float (&v)[4]) { put4(reinterpret_cast<uint16_t*>(p), 0, v); }
};
template <> struct FfType<float> {
    static constexpr int kPlanes = 3;
    static __device__ __forceinline__ void put4(uint16_t* to, uint64_t plane, const float (&v)[4])
    {
        uint16_t q[4][3];
#pragma unroll
        for (int i = 0; i < 4; ++i) ff_planes(v[i], q[i]);
#pragma unroll
        for (int p = 0; p < 3; ++p)
            put_any(to + p * plane, Bf16Quad{q[0][p] | static_cast<uint32_t>(q[1][p]) << 16, q[2][p] | static_cast<uint32_t>(q[3][p]) << 16});
    }
    static __device__ __forceinline__ Floats4 load4(const float* p) { return at_any<Floats4>(p); }
    static __device__ __forceinline__ void widen(const Floats4& q, float (&v)[4]) { v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w; }
    static __device__ __forceinline__ void store4(float* p, const float (&v)[4]) { put_any(p, Floats4{v[0], v[1], v[2], v[3]}); }
};
// Four neighbours of a row of n columns; FULL: all of them in it.  What lies beyond is zero, and is not written.
template <typename T, bool FULL>
__device__ __forceinline__ void ff_load4(const T* row, uint32_t n0, uint32_t n, float (&v)[4])
{
    if (FULL || n0 + 4 <= n) {
        FfType<T>::widen(FfType<T>::load4(row + n0), v);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = n0 + i < n ? static_cast<float>(row[n0 + i]) : 0.f;
    }
}
template <typename T, bool FULL>
__device__ __forceinline__ void ff_store4(T* row, uint32_t n0, uint32_t n, const float (&v)[4])
{
    if (FULL || n0 + 4 <= n) {
        FfType<T>::store4(row + n0, v);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (n0 + i < n) row[n0 + i] = static_cast<T>(v[i]);
    }
}

// What the epilogue of four neighbouring sums of a row loads: the kept projections, or what is added to
struct FfLoaded {
    float a[4], b[4];
};
template <typename T, int EPI, bool FULL>
__device__ __forceinline__ void ff_load(const FfProblem& p, uint32_t m, uint32_t n0, FfLoaded& x)
{
    if constexpr (EPI == kFfDgate) {
        ff_load4<T, FULL>(static_cast<const T*>(p.e0) + m * p.lde, n0, p.N, x.a);
        ff_load4<T, FULL>(static_cast<const T*>(p.e1) + m * p.lde, n0, p.N, x.b);
    } else if constexpr (EPI == kFfStore) {
        if (p.accumulate) ff_load4<T, FULL>(static_cast<const T*>(p.out) + m * p.ldo, n0, p.N, x.a);
    }
}
// What becomes of the sums
template <typename T, int EPI, bool FULL>
__device__ __forceinline__ void ff_epilogue(const FfProblem& p, uint32_t m, uint32_t n0, float (&v)[4], float (&v2)[4], const FfLoaded& x)
{
    if constexpr (EPI == kFfStore) {
        if (p.accumulate)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += x.a[i];
        ff_store4<T, FULL>(static_cast<T*>(p.out) + m * p.ldo, n0, p.N, v);
    } else if constexpr (EPI == kFfGate) {
        float h[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            float a, da;
            ff_act(p.act, v[i], a, da);
            h[i] = FULL || (n0 + i < p.N && m < p.M) ? a * v2[i] : 0.f;
        }
        FfType<T>::put4(static_cast<uint16_t*>(p.out) + m * p.ldo + n0, p.plane, h);
        if (p.e0 && (FULL || m < p.M)) {
            ff_store4<T, FULL>(static_cast<T*>(p.e0) + m * p.lde, n0, p.N, v);
            ff_store4<T, FULL>(static_cast<T*>(p.e1) + m * p.lde, n0, p.N, v2);
        }
    } else {
        float dg[4], du[4], h[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            float a, da;
            ff_act(p.act, x.a[i], a, da);
            const bool in = FULL || (n0 + i < p.N && m < p.M);
            h[i] = in ? a * x.b[i] : 0.f;
            dg[i] = in ? v[i] * x.b[i] * da : 0.f;
            du[i] = in ? v[i] * a : 0.f;
        }
        const uint64_t at = m * p.ldo + n0;
        FfType<T>::put4(static_cast<uint16_t*>(p.out) + at, p.plane, h);
        FfType<T>::put4(static_cast<uint16_t*>(p.o1) + at, p.plane, dg);
        FfType<T>::put4(static_cast<uint16_t*>(p.o2) + at, p.plane, du);
    }
}

// Tile of a block: the blocks that the dispatcher places on one XCD (equal id modulo 8) take neighbouring tiles, columns of
// kFfBand rows of tiles at a time, so that an XCD's L2 holds the operand rows that they share.
constexpr uint32_t kFfBand = 8;
__device__ __forceinline__ void ff_tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn)
{
    const uint32_t total = tiles_m * tiles_n, per = total / 8, rest = total % 8, xcd = id % 8, at = id / 8;
    id = xcd * per + min(xcd, rest) + at;       // XCDs below `rest` have one more
    const uint32_t band = id / (kFfBand * tiles_n), in = id - band * kFfBand * tiles_n;
    const uint32_t rows = min(kFfBand, tiles_m - band * kFfBand);
    tm = band * kFfBand + in % rows;
    tn = in / rows;
}

// Shared memory's own addresses, for the instructions that take them
typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef const __attribute__((address_space(1))) unsigned char global_byte;
__device__ __forceinline__ uint32_t lds_address(const void* p)
{
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)p));
}
// 16 bytes per lane from `base` + its offset to LDS, one lane's after the other's, from address `to` on.  An instruction of its own,
// since the compiler would otherwise have every later read of LDS wait for it: tile_barrier stands before the reads.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t to)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(to), "v"(offset), "s"(base));
}
// every wave's reads of LDS and all but its last N loads are done
template <int N>
__device__ __forceinline__ void tile_barrier()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ const FfProblem& ff_problem_of(const FfArgs& args, uint32_t tile)
{
    uint32_t pi = 0;
#pragma unroll
    for (int i = 1; i < kFfProblems; ++i) pi += (static_cast<uint32_t>(i) < args.count && tile >= args.p[i].first) ? 1u : 0u;
    return args.p[pi];
}

// f(0), f(1), .. f(N - 1), each with a constant (a loop of this length is not unrolled whatever it is told)
template <int N, int I = 0, typename F>
__device__ __forceinline__ void ff_each(F&& f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        ff_each<N, I + 1>(f);
    }
}

// The sums of 32 rows and 2 x 32 columns (gated: of either projection), of which a lane holds row lane % 32 and of either half the
// columns 8 (v / 4) + 4 (lane / 32) + v % 4: through LDS (the wave's own part of it), so that a row's columns are loaded and stored together.
constexpr uint32_t kFfRow = 68;         // floats: 64 and a pad that spreads the rows over the banks
// SINGLE: of one square of 32 columns alone
template <int EPI, bool SINGLE> constexpr uint32_t kFfLanes = EPI == kFfGate || SINGLE ? 8 : 16;   // per row, four columns each
template <int EPI, bool SINGLE> constexpr int kFfPasses = 32 * kFfLanes<EPI, SINGLE> / 64;         // over the rows

// whether all of it lies inside the output
template <int EPI, bool SINGLE>
__device__ __forceinline__ bool ff_inside(const FfProblem& p, uint32_t m0, uint32_t n0) { return m0 + 32 <= p.M && n0 + kFfLanes<EPI, SINGLE> * 4 <= p.N; }
// what the epilogue of such a square loads, asked for ahead of it
template <typename T, int EPI, bool SINGLE>
__device__ __forceinline__ void ff_ask(const FfProblem& p, FfLoaded (&x)[kFfPasses<EPI, SINGLE>], uint32_t lane, uint32_t m0, uint32_t n0)
{
#pragma unroll
    for (int k = 0; k < kFfPasses<EPI, SINGLE>; ++k)
        ff_load<T, EPI, true>(p, m0 + k * (64 / kFfLanes<EPI, SINGLE>) + lane / kFfLanes<EPI, SINGLE>, n0 + lane % kFfLanes<EPI, SINGLE> * 4, x[k]);
}
// the sums to the wave's part of LDS
template <int EPI, bool SINGLE>
__device__ __forceinline__ void ff_spread(const f32x16& left, const f32x16& right, float* mine, uint32_t lane)
{
#pragma unroll
    for (int j = 0; j < (EPI != kFfGate && SINGLE ? 1 : 2); ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x16& a = j ? right : left;
            const float4 v = {a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
            *reinterpret_cast<float4*>(mine + (lane & 31) * kFfRow + j * 32 + 8 * q + 4 * (lane >> 5)) = v;
        }
}
__device__ __forceinline__ void ff_wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// and from there through the epilogue.  FULL: the square lies inside the output, and `x` holds what its epilogue loads
template <typename T, int EPI, bool SINGLE, bool FULL>
__device__ __forceinline__ void ff_finish(const FfProblem& p, const float* mine, uint32_t lane, uint32_t m0, uint32_t n0,
                                          const FfLoaded (&x)[kFfPasses<EPI, SINGLE>])
{
    constexpr bool GATED = EPI == kFfGate;
    const uint32_t c4 = lane % kFfLanes<EPI, SINGLE> * 4, n = n0 + c4;
    auto row = [&](int k, const FfLoaded& loaded) {
        const uint32_t r = k * (64 / kFfLanes<EPI, SINGLE>) + lane / kFfLanes<EPI, SINGLE>;
        const float4 s = *reinterpret_cast<const float4*>(mine + r * kFfRow + c4);
        const float4 s2 = GATED ? *reinterpret_cast<const float4*>(mine + r * kFfRow + 32 + c4) : s;
        float v[4] = {s.x, s.y, s.z, s.w}, v2[4] = {s2.x, s2.y, s2.z, s2.w};
        ff_epilogue<T, EPI, FULL>(p, m0 + r, n, v, v2, loaded);
    };
    if constexpr (FULL) {
#pragma unroll
        for (int k = 0; k < kFfPasses<EPI, SINGLE>; ++k) row(k, x[k]);
    } else {
        const uint32_t n_end = EPI == kFfStore ? p.N : p.n_pad, m_end = EPI == kFfStore ? p.M : p.m_pad;
        auto m_of = [&](int k) { return m0 + k * (64 / kFfLanes<EPI, SINGLE>) + lane / kFfLanes<EPI, SINGLE>; };
        FfLoaded loaded = {}, next = {};
        if (EPI == kFfDgate && m_of(0) < p.M) ff_load<T, EPI, false>(p, m_of(0), n, loaded);
#pragma unroll 1
        for (int k = 0; k < kFfPasses<EPI, SINGLE>; ++k) {
            if (EPI == kFfDgate && k + 1 < kFfPasses<EPI, SINGLE> && m_of(k + 1) < p.M) ff_load<T, EPI, false>(p, m_of(k + 1), n, next);
            if (m_of(k) >= m_end || n >= n_end) continue;
            if (EPI != kFfDgate && m_of(k) < p.M) ff_load<T, EPI, false>(p, m_of(k), n, loaded);
            row(k, loaded);
            if constexpr (EPI == kFfDgate) loaded = next;
        }
    }
}

// Where a worker leaves the sums of a tile: in the order of its registers, NI squares of 32 x 32 in a row of them
template <int BM, int BN, int NI>
__device__ __forceinline__ float4* ff_slot(float* part, uint32_t slot, uint32_t i, uint32_t j, uint32_t q, uint32_t tid)
{
    constexpr uint32_t threads = 256;
    return reinterpret_cast<float4*>(part + static_cast<uint64_t>(slot) * (BM * BN)) + ((i * NI + j) * 4 + q) * threads + tid;
}

// Bytes from the tile's first element to the unit of 16 bytes that a lane brings in load i of its wave.  `last`: the last row of the
// operand that there is, from the tile's first; transposed: its last column.
template <bool TRANS, int WIDTH, typename F>
__device__ __forceinline__ uint32_t ff_place(uint32_t wave, uint32_t lane, int i, F&& row_of, uint32_t last, uint32_t ld)
{
    if constexpr (!TRANS) {
        const uint32_t row = (i * 4 + wave) * 8 + lane / 8, unit = lane % 8 ^ row / 2 % 8;
        return min(row_of(row), last) * ld * 2 + unit * 16;
    } else {
        constexpr uint32_t UNITS = WIDTH / 8;       // of a row of k
        const uint32_t k = (i * 4 + wave) * (64 / UNITS) + lane / UNITS, unit = lane % UNITS ^ (k % 4 * 2 + k / 8 % 2) * 2;
        return k * ld * 2 + min(unit, last / 8) * 16;
    }
}
// A wave's fragments, of 32 rows (columns, transposed) and 16 k each, from column `first` of the tile on
template <bool TRANS, int WIDTH>
struct FfFragments {
    uint32_t at;
    __device__ __forceinline__ FfFragments(uint32_t lane, uint32_t first)
    {
        if constexpr (!TRANS) {
            const uint32_t row = lane % 32;
            at = (first + row) * 128 + (lane / 32 ^ row / 2 % 8) * 16;              // to be xored with 16 k's 32 bytes
        } else {
            const uint32_t k = lane / 32 * 8 + lane % 16 / 4;
            at = k * (WIDTH * 2) + ((first + lane / 16 % 2 * 16 + lane % 4 * 4) * 2 ^ (k % 4 * 2 + k / 8 % 2) * 32);    // with f's 64 bytes
        }
    }
    __device__ __forceinline__ bf16x8 read(const unsigned char* tile, int kk, int f) const
    {
        if constexpr (!TRANS) {
            return *reinterpret_cast<const bf16x8*>(tile + (at ^ (kk * 32)) + f * 4096);
        } else {
            typedef __attribute__((address_space(3))) bf16x4 lds_x4;
            const unsigned char* const q = tile + (at ^ (f * 64)) + kk * (WIDTH * 32);
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_x4*)q);
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_x4*)(q + WIDTH * 8));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// Rows of B that a wave has of its NI * 32: gated, the first half are the first projection's and the others the second's
template <bool GATED, int NI>
__device__ __forceinline__ uint32_t ff_column(uint32_t row) { return GATED ? row / (NI * 32) * (NI * 16) + row % (NI * 16) : row; }

template <int BM, int BN, bool TA, bool TB, typename T, int EPI>
__global__ __launch_bounds__(256) void k_ff_gemm(const FfArgs args)
{
    constexpr bool GATED = EPI == kFfGate, LARGE = BM == 256;
    static_assert(!GATED || !TB, "the projections' weights have k along their rows");
    constexpr int MI = BM / 64, NI = BN / 64, LA = BM / 32, LB = BN / 32;       // squares of a wave; its loads per tile of 64 k
    constexpr uint32_t COLS = GATED ? BN / 2 : BN;
    constexpr uint32_t kBufsA = LARGE ? 3 : 2, kBytesA = BM * 128, kBytesB = BN * 128, kAtB = kBufsA * kBytesA;
    static_assert(MI == NI, "");
    extern __shared__ __align__(16) unsigned char lds[];        // [kBufsA][kBytesA], [2][kBytesB]
    static_assert(4 * 32 * kFfRow * 4 <= kAtB + 2 * kBytesB, "the waves' parts of LDS in ff_finish fit where the tiles were");

    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), wm = wave / 2, wn = wave % 2;
    const bool shares = blockIdx.x >= args.whole;
    const uint32_t worker = blockIdx.x - args.whole;
    uint64_t step = shares ? ff_share(args, worker) : 0;
    const uint64_t steps_end = shares ? ff_share(args, worker + 1) : args.ksteps;
    while (step < steps_end) {
        const uint32_t at = shares ? static_cast<uint32_t>(step / args.ksteps) : 0;
        const uint32_t tile = shares ? args.whole + at : blockIdx.x;
        const uint32_t kt0 = static_cast<uint32_t>(step - static_cast<uint64_t>(at) * args.ksteps);
        const uint32_t kt1 = static_cast<uint32_t>(min(static_cast<uint64_t>(args.ksteps), kt0 + (steps_end - step)));
        step += kt1 - kt0;
        const FfProblem& p = ff_problem_of(args, tile);
        uint32_t tm, tn;
        ff_tile_of(tile - p.first, p.tiles_m, p.tiles_n, tm, tn);
        const uint32_t m0 = tm * BM, n0 = tn * COLS;

        // Bytes from the tile's first element to the units that this thread brings.  Load i of a wave fills 1 KB of LDS, from
        // 1024 (4 i + wave) on: eight rows of an operand, or two or four rows of k of a transposed one.  What lies beyond the matrix
        // is its last row or unit again.
        uint32_t oa[LA], ob[LB];
#pragma unroll
        for (int i = 0; i < LA; ++i) oa[i] = ff_place<TA, BM>(wave, lane, i, [&](uint32_t r) { return r; }, p.M - 1 - m0, static_cast<uint32_t>(p.lda));
#pragma unroll
        for (int i = 0; i < LB; ++i)
            ob[i] = ff_place<TB, BN>(wave, lane, i, [&](uint32_t r) { return ff_column<GATED, NI>(r); }, p.N - 1 - n0, static_cast<uint32_t>(p.ldb));

        const uint32_t per_seg = p.ktiles;
        // elements from an operand's first to the tile's, and from a tile of k to the next
        const uint64_t a_first = TA ? m0 : m0 * p.lda, b_first = TB ? n0 : n0 * p.ldb;
        const uint64_t a_step = TA ? kFfBk * p.lda : kFfBk, b_step = TB ? kFfBk * p.ldb : kFfBk;
        // where the next tile of either operand is; B is asked for later than A, so each has a place of its own
        struct Place {
            uint32_t seg, left;
        };
        Place na{kt0 / per_seg, 0}, nb;
        const uint32_t in_seg = kt0 - na.seg * per_seg;
        na.left = per_seg - in_seg;
        nb = na;
        const uint16_t *pa = p.a[na.seg] + a_first + in_seg * a_step, *pb = p.b[nb.seg] + b_first + in_seg * b_step;
        const uint16_t* pb2 = GATED ? p.b2[nb.seg] + b_first + in_seg * b_step : pb;
        auto next_a = [&]() {
            pa += a_step;
            if (--na.left == 0 && na.seg + 1 < p.nseg) {
                pa = p.a[++na.seg] + a_first;
                na.left = per_seg;
            }
        };
        auto next_b = [&]() {
            pb += b_step;
            pb2 += b_step;
            if (--nb.left == 0 && nb.seg + 1 < p.nseg) {
                pb = p.b[++nb.seg] + b_first;
                pb2 = GATED ? p.b2[nb.seg] + b_first : pb;
                nb.left = per_seg;
            }
        };
        const uint32_t base = lds_address(lds) + wave * 1024;
        auto bring_a = [&](uint32_t buf, int i) { load_to_lds(pa, oa[i], base + buf * kBytesA + i * 4096); };
        auto bring_b = [&](uint32_t buf, int i) {
            // gated: LB / 2 loads of either matrix for each wave of the tile's columns
            const bool second = GATED && (i * 32) % (NI * 32) >= NI * 16;
            load_to_lds(second ? pb2 : pb, ob[i], base + kAtB + buf * kBytesB + i * 4096);
        };

        f32x16 acc[MI][NI];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

        // A tile's four steps of 16 k: while one is multiplied, the fragments of the next are read (in the last one, the first of the
        // next tile).  The barrier before the last step ends the reads of the tile: from there on B of tile t + 2 is asked for, into
        // the place of tile t's.  A has three buffers where they fit (LARGE), and A of tile t + 2 is asked for in the first two
        // steps of tile t.  Either has four steps at least to come: the barrier of tile t has to find tile t + 1 there, and after that
        // tile was asked for came A of tile t + 2 only.
        const FfFragments<TA, BM> frag_a(lane, wm * MI * 32);
        const FfFragments<TB, BN> frag_b(lane, wn * NI * 32);
        const uint32_t n = kt1 - kt0;
        bf16x8 fa[2][MI], fb[2][NI];
        auto read = [&](uint32_t buf_a, uint32_t buf_b, int kk, int f) {        // fragment f of the step: NI of B, MI of A, as they are used
            const int to = kk & 1;
            if (f < NI) fb[to][f] = frag_b.read(lds + kAtB + buf_b * kBytesB, kk, f);
            else fa[to][f - NI] = frag_a.read(lds + buf_a * kBytesA, kk, f - NI);
        };
        for (uint32_t t = 0; t < 2 && t < n; ++t) {
#pragma unroll
            for (int i = 0; i < LA; ++i) bring_a(t, i);
            next_a();
#pragma unroll
            for (int i = 0; i < LB; ++i) bring_b(t, i);
            next_b();
        }
        if (n > 1) tile_barrier<LA + LB>();
        else tile_barrier<0>();
#pragma unroll
        for (int f = 0; f < MI + NI; ++f) read(0, 0, 0, f);
        uint32_t buf_a = 0, ask_a = kBufsA - 1;     // buffers of this tile's A and of the one asked for next
        for (uint32_t t = 0; t < n; ++t) {
            const uint32_t buf_b = t & 1, next_buf_a = buf_a + 1 == kBufsA ? 0 : buf_a + 1;
            const bool more_a = LARGE && t + 2 < n, more_b = t + 2 < n;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                if (kk == 3) {
                    if (more_a) tile_barrier<LA>();
                    else tile_barrier<0>();
                }
                const int from = kk & 1;
#pragma unroll
                for (int c = 0; c < MI + NI; ++c) {
                    if (kk < 3) read(buf_a, buf_b, kk + 1, c);
                    else read(next_buf_a, buf_b ^ 1, 0, c);
                    if (LARGE && kk < 2 && more_a && c % 2 == 0) bring_a(ask_a, kk * (LA / 2) + c / 2);
                    if (kk == 3 && more_b) {
                        bring_b(buf_b, c);
                        if (!LARGE) bring_a(buf_b, c);
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int m = c * MI * NI / (MI + NI); m < (c + 1) * MI * NI / (MI + NI); ++m)
                        acc[m / NI][m % NI] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[from][m % NI], fa[from][m / NI], acc[m / NI][m % NI], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (LARGE && kk == 1 && more_a) next_a();
            }
            if (more_b) {
                next_b();
                if (!LARGE) next_a();
            }
            buf_a = next_buf_a;
            ask_a = ask_a + 1 == kBufsA ? 0 : ask_a + 1;
        }
        tile_barrier<0>();

        if (kt1 - kt0 == args.ksteps) {
            float* const mine = reinterpret_cast<float*>(lds) + wave * (32 * kFfRow);
            auto m_of = [&](int s) { return m0 + (wm * MI + s / (NI / 2)) * 32; };
            auto n_of = [&](int s) { return n0 + (GATED ? wn * NI * 16 + s % (NI / 2) * 32 : wn * NI * 32 + s % (NI / 2) * 64); };
            constexpr int SQUARES = MI * NI / 2;
            FfLoaded x[kFfPasses<EPI, false>], next[kFfPasses<EPI, false>];
            auto inside = [&](int s) { return ff_inside<EPI, false>(p, m_of(s), n_of(s)); };
            if (inside(0)) ff_ask<T, EPI, false>(p, x, lane, m_of(0), n_of(0));
            auto square = [&](auto s) {
                if (s + 1 < SQUARES && inside(s + 1)) ff_ask<T, EPI, false>(p, next, lane, m_of(s + 1), n_of(s + 1));
                ff_each<SQUARES>([&](auto sq) {
                    constexpr int k = decltype(sq)::value, i = k / (NI / 2), j = k % (NI / 2);
                    if (s == k) ff_spread<EPI, false>(acc[i][(GATED ? 1 : 2) * j], acc[i][GATED ? j + NI / 2 : 2 * j + 1], mine, lane);
                });
                ff_wave_sync();
                if (inside(s)) ff_finish<T, EPI, false, true>(p, mine, lane, m_of(s), n_of(s), x);
                else ff_finish<T, EPI, false, false>(p, mine, lane, m_of(s), n_of(s), x);
                ff_wave_sync();
#pragma unroll
                for (int k = 0; k < kFfPasses<EPI, false>; ++k) x[k] = next[k];
            };
            // Long epilogues as a loop, whose code stays in the instruction cache (256 x 256, dgate / gate / dw of 4096 x 16384, unrolled
            // and not: 674 and 641 us / 2975 and 2920 / 1368 and 1380)
            if constexpr (EPI == kFfStore) {
                ff_each<SQUARES>(square);
            } else {
#pragma unroll 1
                for (int s = 0; s < SQUARES; ++s) square(s);
            }
        } else {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *ff_slot<BM, BN, NI>(args.part, worker + at, i, j, q, tid) =
                            float4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        }
        if (step < steps_end) __syncthreads();      // the next tile's rows go where this one's sums were
    }
}

// Adds up the sums that several workers have of a tile, in the order of the workers: one square (gated: of both projections) of every
// wave's part per block
template <int BM, int BN, typename T, int EPI>
__global__ __launch_bounds__(256) void k_ff_join(const FfArgs args)
{
    constexpr bool GATED = EPI == kFfGate;
    constexpr int MI = BM / 64, NI = BN / 64, BOTH = GATED ? 2 : 1, ACROSS = NI / BOTH;
    __shared__ float stage[4 * 32 * kFfRow];
    const uint32_t per = MI * ACROSS, at = blockIdx.x / per, i = blockIdx.x % per / ACROSS, j = blockIdx.x % ACROSS;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    const uint64_t s0 = static_cast<uint64_t>(at) * args.ksteps, s1 = s0 + args.ksteps, all = static_cast<uint64_t>(args.rest) * args.ksteps;
    // the workers that have a step of this tile
    uint32_t first = static_cast<uint32_t>(s0 * args.workers / all), last = static_cast<uint32_t>((s1 - 1) * args.workers / all);
    while (ff_share(args, first + 1) <= s0) ++first;
    while (last + 1 < args.workers && ff_share(args, last + 1) < s1) ++last;
    if (first == last) return;                      // one, which has finished it
    f32x16 acc[BOTH] = {};
#pragma unroll 4
    for (uint32_t w = first; w <= last; ++w) {
#pragma unroll
        for (int h = 0; h < BOTH; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 v = *ff_slot<BM, BN, NI>(args.part, w + at, i, j + h * (NI / 2), q, tid);
                acc[h][4 * q] += v.x; acc[h][4 * q + 1] += v.y; acc[h][4 * q + 2] += v.z; acc[h][4 * q + 3] += v.w;
            }
    }
    const uint32_t tile = args.whole + at;
    const FfProblem& p = ff_problem_of(args, tile);
    uint32_t tm, tn;
    ff_tile_of(tile - p.first, p.tiles_m, p.tiles_n, tm, tn);
    const uint32_t m0 = tm * BM + (wave / 2 * MI + i) * 32, n0 = tn * (BN / BOTH) + (wave % 2 * ACROSS + j) * 32;
    float* const mine = stage + wave * (32 * kFfRow);
    FfLoaded x[kFfPasses<EPI, true>];
    const bool inside = ff_inside<EPI, true>(p, m0, n0);
    if (inside) ff_ask<T, EPI, true>(p, x, lane, m0, n0);
    ff_spread<EPI, true>(acc[0], acc[BOTH - 1], mine, lane);
    ff_wave_sync();
    if (inside) ff_finish<T, EPI, true, true>(p, mine, lane, m0, n0, x);
    else ff_finish<T, EPI, true, false>(p, mine, lane, m0, n0, x);
}

}  // namespace edgc
