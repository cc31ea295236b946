// The matrix products of the gated feed-forward block: C[m][n] = sum over segments and k of A[m][k] B[n][k], both operands bf16 with
// k contiguous, 16-byte aligned rows and k padded with zeros to whole tiles of 64.
//
// fp32 operands come as three bf16 planes that add up to them exactly (24 significant bits = 3 x 8: a plane is the value's leading
// bits, cut off, not rounded); six products of planes, 2^-24 of the operands left out, are six segments of one sum.  Six bf16 MFMAs
// take less time than one of fp32 (2.5e15 / 6 against 0.16e15 operations a second).
//
// A block of WM x WN waves makes a BM x BN tile; tiles of 64 or 32 k of the operands come to LDS buffers while earlier ones are
// multiplied.  A row of 128 (64) bytes lies in LDS as eight (four) 16-byte units, unit c at c ^ (row / 2 & 7) (at
// c ^ (row / 4 & 3)): a read of 16 bytes per lane takes lanes 0-3, 12-15 and 20-27 of either half at once, then the other sixteen,
// and their rows then lie in different banks.  (At c ^ (row & 7) and c ^ (row / 2 & 3) half of LDS's cycles were conflicts.)  The MFMA's first operand is B: a lane then holds four
// neighbouring n of one m, which is what the epilogues load and store.
#pragma once

#include "compress_common.h"

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
    uint32_t n_pad;                     // columns of out, o1, o2: those from N on are zeros
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

// Activation and derivative.  gelu_tanh by the identity (1 + tanh t) / 2 = 1 / (1 + exp(-2 t)).
__device__ __forceinline__ void ff_act(int act, float z, float& a, float& da)
{
    if (act == EDGC_SILU) {
        const float s = 1.0f / (1.0f + expf(-z));
        a = z * s;
        da = s * (1.0f + z * (1.0f - s));
    } else if (act == EDGC_GELU) {
        const float cdf = 0.5f * erfcf(z * -0.70710678118654752f);
        a = z * cdf;
        da = cdf + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    } else {
        const float k = 0.79788456080286536f, c = 0.044715f;
        const float s = 1.0f / (1.0f + expf(-2.0f * k * (z + c * z * z * z)));
        a = z * s;
        da = s + 2.0f * k * z * s * (1.0f - s) * (1.0f + 3.0f * c * z * z);
    }
}

// x = p[0] + p[1] + p[2] in bf16, exactly (unless its last bits lie below the smallest number).  What is not finite is plane 0 alone.
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

// T's planes of four values, to planes `plane` elements apart
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
// four neighbours of a row of n columns: what lies beyond is zero, and is not written
template <typename T>
__device__ __forceinline__ void ff_load4(const T* row, uint32_t n0, uint32_t n, float (&v)[4])
{
    if (n0 + 4 <= n) {
        FfType<T>::widen(FfType<T>::load4(row + n0), v);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = n0 + i < n ? static_cast<float>(row[n0 + i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void ff_store4(T* row, uint32_t n0, uint32_t n, const float (&v)[4])
{
    if (n0 + 4 <= n) {
        FfType<T>::store4(row + n0, v);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (n0 + i < n) row[n0 + i] = static_cast<T>(v[i]);
    }
}

// What becomes of four neighbouring sums of row m
template <typename T, int EPI>
__device__ __forceinline__ void ff_epilogue(const FfProblem& p, uint32_t m, uint32_t n0, float (&v)[4], float (&v2)[4])
{
    if constexpr (EPI == kFfStore) {
        T* const row = static_cast<T*>(p.out) + m * p.ldo;
        if (p.accumulate) {
            float o[4];
            ff_load4<T>(row, n0, p.N, o);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += o[i];
        }
        ff_store4<T>(row, n0, p.N, v);
    } else if constexpr (EPI == kFfGate) {
        float h[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            float a, da;
            ff_act(p.act, v[i], a, da);
            h[i] = n0 + i < p.N ? a * v2[i] : 0.f;
        }
        FfType<T>::put4(static_cast<uint16_t*>(p.out) + m * p.ldo + n0, p.plane, h);
        if (p.e0) ff_store4<T>(static_cast<T*>(p.e0) + m * p.lde, n0, p.N, v);
        if (p.e1) ff_store4<T>(static_cast<T*>(p.e1) + m * p.lde, n0, p.N, v2);
    } else {
        float g[4], u[4], dg[4], du[4], h[4];
        ff_load4<T>(static_cast<const T*>(p.e0) + m * p.lde, n0, p.N, g);
        ff_load4<T>(static_cast<const T*>(p.e1) + m * p.lde, n0, p.N, u);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            float a, da;
            ff_act(p.act, g[i], a, da);
            const bool in = n0 + i < p.N;
            h[i] = in ? a * u[i] : 0.f;
            dg[i] = in ? v[i] * u[i] * da : 0.f;
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
// 16 bytes from each lane's address to 16 bytes per lane, one after the other, from `to` on
__device__ __forceinline__ void load_to_lds(const unsigned char* from, unsigned char* to)
{
    __builtin_amdgcn_global_load_lds((global_byte*)from, (lds_byte*)to, 16, 0, 0);
}
// The fragments of a tile of 32 k: rows 32 apart lie 2048 bytes apart in LDS, the second 16 k at the address ^ 32
__device__ __forceinline__ void read_fragments(uint32_t at_a, uint32_t at_b, bf16x8 (&fa)[2][4], bf16x8 (&fb)[2][2])
{
    asm volatile("ds_read_b128 %0, %12\n\t"
                 "ds_read_b128 %8, %14\n\t"
                 "ds_read_b128 %9, %14 offset:2048\n\t"
                 "ds_read_b128 %1, %12 offset:2048\n\t"
                 "ds_read_b128 %2, %12 offset:4096\n\t"
                 "ds_read_b128 %3, %12 offset:6144\n\t"
                 "ds_read_b128 %4, %13\n\t"
                 "ds_read_b128 %10, %15\n\t"
                 "ds_read_b128 %11, %15 offset:2048\n\t"
                 "ds_read_b128 %5, %13 offset:2048\n\t"
                 "ds_read_b128 %6, %13 offset:4096\n\t"
                 "ds_read_b128 %7, %13 offset:6144\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0][0]), "=&v"(fa[0][1]), "=&v"(fa[0][2]), "=&v"(fa[0][3]), "=&v"(fa[1][0]), "=&v"(fa[1][1]),
                   "=&v"(fa[1][2]), "=&v"(fa[1][3]), "=&v"(fb[0][0]), "=&v"(fb[0][1]), "=&v"(fb[1][0]), "=&v"(fb[1][1])
                 : "v"(at_a), "v"(at_a ^ 32u), "v"(at_b), "v"(at_b ^ 32u)
                 : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void slot_end()
{
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ const FfProblem& ff_problem_of(const FfArgs& args, uint32_t tile)
{
    uint32_t pi = 0;
#pragma unroll
    for (int i = 1; i < kFfProblems; ++i) pi += (static_cast<uint32_t>(i) < args.count && tile >= args.p[i].first) ? 1u : 0u;
    return args.p[pi];
}

// The sums of 32 rows of a wave, of which a lane holds row lane % 32 and of either half the columns 8 (v / 4) + 4 (lane / 32) + v % 4:
// through LDS (the wave's own part of it), so that a row's columns are loaded and stored together.
constexpr uint32_t kFfRow = 68;         // floats: 64 and a pad that spreads the rows over the banks
template <typename T, int EPI>
__device__ __forceinline__ void ff_finish(const FfProblem& p, const f32x16 (&acc)[2], float* mine, uint32_t lane, uint32_t m0, uint32_t n0)
{
    constexpr bool GATED = EPI == kFfGate;
    constexpr uint32_t kLanes = GATED ? 8 : 16;     // per row, four columns each
    const uint32_t c4 = (lane % kLanes) * 4, n = n0 + c4;
    const uint32_t n_end = (EPI == kFfGate || EPI == kFfDgate) ? p.n_pad : p.N;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 v = {acc[j][4 * q], acc[j][4 * q + 1], acc[j][4 * q + 2], acc[j][4 * q + 3]};
            *reinterpret_cast<float4*>(mine + (lane & 31) * kFfRow + j * 32 + 8 * q + 4 * (lane >> 5)) = v;
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 4
    for (uint32_t r0 = 0; r0 < 32; r0 += 64 / kLanes) {
        const uint32_t r = r0 + lane / kLanes, m = m0 + r;
        const float4 x = *reinterpret_cast<const float4*>(mine + r * kFfRow + c4);
        const float4 x2 = GATED ? *reinterpret_cast<const float4*>(mine + r * kFfRow + 32 + c4) : x;
        if (m >= p.M || n >= n_end) continue;
        float v[4] = {x.x, x.y, x.z, x.w}, v2[4] = {x2.x, x2.y, x2.z, x2.w};
        ff_epilogue<T, EPI>(p, m, n, v, v2);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Where a worker leaves the sums of a tile: in the order of its registers
template <int BM, int BN>
__device__ __forceinline__ float4* ff_slot(float* part, uint32_t slot, uint32_t i, uint32_t j, uint32_t q, uint32_t tid, uint32_t threads)
{
    return reinterpret_cast<float4*>(part + static_cast<uint64_t>(slot) * (BM * BN)) + ((i * 2 + j) * 4 + q) * threads + tid;
}

// Waves of a block that take turns (below): tiles of 32 k in four buffers.  Otherwise tiles of 64 k in two.
constexpr bool ff_turns(int wm, int wn) { return wm * wn == 8; }
constexpr int ff_bk(int wm, int wn) { return ff_turns(wm, wn) ? 32 : 64; }

template <int BM, int BN, int WM, int WN, typename T, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void k_ff_gemm(const FfArgs args)
{
    constexpr bool GATED = EPI == kFfGate, TURNS = ff_turns(WM, WN);
    constexpr int NTH = 64 * WM * WN, MI = BM / WM / 32, NI = 2, BK = ff_bk(WM, WN), UNITS = BK / 8;
    constexpr int ROWS = NTH / UNITS, LA = BM / ROWS, LB = BN / ROWS;       // rows that the block brings at a time
    static_assert(BN / WN == 64, "a wave has 64 columns; gated: 32 of either projection");
    static_assert(ROWS == 128 || ROWS == 32, "rows of the two projections alternate by 32");
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr uint32_t kBuf = (BM + BN) * BK * 2, kBufs = TURNS ? 4 : 2;
    constexpr uint32_t COLS = GATED ? BN / 2 : BN;
    static_assert(WM * WN * 32 * kFfRow * 4 <= kBufs * kBuf, "the waves' parts of LDS in ff_finish fit where the tiles were");

    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), wm = wave / WN, wn = wave % WN;
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

        // Bytes from the tile's first row to the units that this thread brings (rows beyond the matrix: its last): to unit
        // tid % UNITS of the LDS row tid / UNITS and of those ROWS apart from it, whose bits choose which unit of the operand's.
        uint32_t oa[LA], ob[LB];
        const uint32_t unit = ((tid % UNITS) ^ (TURNS ? tid / UNITS / 4 & 3 : tid / UNITS / 2 & 7)) * 16;
#pragma unroll
        for (int i = 0; i < LA; ++i) {
            const uint32_t row = min(tid / UNITS + i * ROWS, p.M - 1 - m0);
            oa[i] = row * static_cast<uint32_t>(p.lda) * 2 + unit;
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            uint32_t row = tid / UNITS + i * ROWS;
            if constexpr (GATED) row = row / 64 * 32 + row % 32;        // rows 64 w .. + 31: the first matrix, + 32 .. 63: the second
            row = min(row, p.N - 1 - n0);
            ob[i] = row * static_cast<uint32_t>(p.ldb) * 2 + unit;
        }
        // which of the two this wave brings, where it is the same for all its rows
        const bool second = GATED && ROWS == 128 && (wave * (64 / UNITS) & 32);

        const uint32_t per_seg = p.ktiles * (64 / BK);
        uint32_t seg = kt0 / per_seg, left = per_seg - (kt0 - seg * per_seg);
        const unsigned char *pa, *pb, *pb2;
        auto to_segment = [&](uint32_t k) {
            const uint64_t a_at = m0 * p.lda + k, b_at = n0 * p.ldb + k;
            pa = reinterpret_cast<const unsigned char*>(p.a[seg] + a_at);
            pb = reinterpret_cast<const unsigned char*>((second ? p.b2[seg] : p.b[seg]) + b_at);
            pb2 = GATED && ROWS == 32 ? reinterpret_cast<const unsigned char*>(p.b2[seg] + b_at) : pb;
        };
        to_segment((kt0 - seg * per_seg) * BK);
        auto bring_a = [&](uint32_t buf, int i) { load_to_lds(pa + oa[i], lds + buf * kBuf + wave * 1024 + i * (ROWS * BK * 2)); };
        auto bring_b = [&](uint32_t buf, int i) {
            load_to_lds((GATED && ROWS == 32 && (i & 1) ? pb2 : pb) + ob[i], lds + buf * kBuf + BM * BK * 2 + wave * 1024 + i * (ROWS * BK * 2));
        };
        auto next = [&]() {
            pa += BK * 2;
            pb += BK * 2;
            pb2 += BK * 2;
            if (--left == 0 && seg + 1 < p.nseg) {
                ++seg;
                left = per_seg;
                to_segment(0);
            }
        };
        auto bring = [&](uint32_t buf) {
#pragma unroll
            for (int i = 0; i < LA; ++i) bring_a(buf, i);
#pragma unroll
            for (int i = 0; i < LB; ++i) bring_b(buf, i);
            next();
        };

        f32x16 acc[MI][NI];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
        const uint32_t fr = lane & 31;          // row of a fragment

        if constexpr (TURNS) {
            // Of the two waves on a SIMD, one reads the fragments of a tile while the other multiplies the ones that it has read (and
            // asks for a later tile in between); a barrier ends either's slot.  Group 0 reads tile t in slot 2 t and multiplies in
            // 2 t + 1, group 1 one slot later.  Tile t + 3 is asked for in the multiplying of tile t, slots 2 t + 1 and 2 t + 2, into
            // the buffer that was read last in slot 2 t - 1, and each group waits for its part of tile t + 1 before the barrier
            // that ends slot 2 t + 1, four loads per tile.
            static_assert(LA == 2 && LB == 2 && MI == 4, "");
            const bool behind = wave >= 4;
            const uint32_t fu = ((lane >> 5) ^ (fr / 4 & 3)) * 16, base = lds_address(lds);
            const uint32_t ra0 = base + (wm * 128 + fr) * 64 + fu, rb0 = base + BM * 64 + (wn * 64 + fr) * 64 + fu;
            // (beyond the last tile the last one is asked for again, and not read: the loop has no cases)
            const uint32_t n = kt1 - kt0;
            uint32_t asked = 0;
            auto next_or_stay = [&]() {
                if (++asked < n) next();
            };
#pragma unroll
            for (uint32_t b = 0; b < 3; ++b) {
#pragma unroll
                for (int i = 0; i < 2; ++i) bring_a(b, i);
#pragma unroll
                for (int i = 0; i < 2; ++i) bring_b(b, i);
                next_or_stay();
            }
            wait_loads<8>();
            slot_end();
            if (behind) slot_end();
            for (uint32_t t = 0; t < n; ++t) {
                const uint32_t buf = (t & 3) * kBuf, to = (t + 3) & 3;
                bf16x8 fa[2][4], fb[2][2];
                read_fragments(ra0 + buf, rb0 + buf, fa, fb);
                if (behind) wait_loads<4>();
                slot_end();
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (i < 2) bring_a(to, i);
                    else bring_b(to, i - 2);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int kk = i / 2, ii = i % 2 * 2 + h;
#pragma unroll
                        for (int j = 0; j < NI; ++j) acc[ii][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[kk][j], fa[kk][ii], acc[ii][j], 0, 0, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
                next_or_stay();
                if (!behind) wait_loads<8>();
                slot_end();
            }
            if (!behind) slot_end();
            wait_loads<0>();
            slot_end();
        } else {
            const uint32_t fu = ((lane >> 5) ^ (fr / 2 & 7)) * 16;      // to be xored with 2 k / 16
            const uint32_t ra0 = (wm * MI * 32 + fr) * 128 + fu, rb0 = BM * 128 + (wn * NI * 32 + fr) * 128 + fu;
            auto multiply = [&](uint32_t buf) {
                const unsigned char* const la = lds + buf * kBuf;
#pragma unroll
                for (int kk = 0; kk < BK / 16; ++kk) {
                    bf16x8 fa[MI], fb[NI];
#pragma unroll
                    for (int i = 0; i < MI; ++i) fa[i] = *reinterpret_cast<const bf16x8*>(la + (ra0 ^ (kk * 32)) + i * 4096);
#pragma unroll
                    for (int j = 0; j < NI; ++j) fb[j] = *reinterpret_cast<const bf16x8*>(la + (rb0 ^ (kk * 32)) + j * 4096);
#pragma unroll
                    for (int i = 0; i < MI; ++i)
#pragma unroll
                        for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
                }
            };
            uint32_t buf = 0;
            bring(0);
            for (uint32_t t = kt0; t < kt1; ++t) {
                wait_loads<0>();
                __syncthreads();            // tile t is there, and every wave is past its reads of tile t - 1
                if (t + 1 < kt1) bring(buf ^ 1);
                multiply(buf);
                buf ^= 1;
            }
            __syncthreads();
        }

        if (kt1 - kt0 == args.ksteps) {
            float* const mine = reinterpret_cast<float*>(lds) + wave * (32 * kFfRow);
#pragma unroll
            for (int i = 0; i < MI; ++i)
                ff_finish<T, EPI>(p, acc[i], mine, lane, m0 + (wm * MI + i) * 32, n0 + wn * (GATED ? 32 : 64));
        } else {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *ff_slot<BM, BN>(args.part, worker + at, i, j, q, tid, NTH) =
                            float4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        }
        if (step < steps_end) __syncthreads();      // the next tile's rows go where this one's sums were
    }
}

// Adds up the sums that several workers have of a tile, in the order of the workers: 32 rows of every wave's part per block
template <int BM, int BN, int WM, int WN, typename T, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void k_ff_join(const FfArgs args)
{
    constexpr int NTH = 64 * WM * WN, MI = BM / WM / 32;
    constexpr bool GATED = EPI == kFfGate;
    __shared__ float stage[WM * WN * 32 * kFfRow];
    const uint32_t at = blockIdx.x / MI, i = blockIdx.x % MI, tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    const uint64_t s0 = static_cast<uint64_t>(at) * args.ksteps, s1 = s0 + args.ksteps, all = static_cast<uint64_t>(args.rest) * args.ksteps;
    uint32_t w = static_cast<uint32_t>(s0 * args.workers / all);
    while (ff_share(args, w + 1) <= s0) ++w;        // the first worker with a step of this tile
    if (ff_share(args, w) <= s0 && ff_share(args, w + 1) >= s1) return;     // which had them all
    f32x16 acc[2] = {};
    for (; w < args.workers && ff_share(args, w) < s1; ++w) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 v = *ff_slot<BM, BN>(args.part, w + at, i, j, q, tid, NTH);
                acc[j][4 * q] += v.x; acc[j][4 * q + 1] += v.y; acc[j][4 * q + 2] += v.z; acc[j][4 * q + 3] += v.w;
            }
    }
    const uint32_t tile = args.whole + at;
    const FfProblem& p = ff_problem_of(args, tile);
    uint32_t tm, tn;
    ff_tile_of(tile - p.first, p.tiles_m, p.tiles_n, tm, tn);
    ff_finish<T, EPI>(p, acc, stage + wave * (32 * kFfRow), lane, tm * BM + (wave / WN * MI + i) * 32,
                      tn * (GATED ? BN / 2 : BN) + wave % WN * (GATED ? 32 : 64));
}

}  // namespace edgc
