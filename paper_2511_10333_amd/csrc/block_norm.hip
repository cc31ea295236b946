// The norms before and after a block, fused with its gate and its residual scale, and their backward pass.
//
//   forward   yh = y r1, r1 = (mean y^2 + eps)^-1/2;   x' = x + s g (yh w_post);   xh = x' r2, r2 = (mean x'^2 + eps)^-1/2;
//             n = xh w_pre
//   backward  u = dn w_pre;   d = dx' + r2 (u - xh mean(u xh));   dx = d;   v = s g w_post d;   dy = r1 (v - yh mean(v yh));
//             dw_pre = sum_t dn xh;   S_k = sum over the tokens of gate row k of d yh;
//             dg_k = s w_post S_k;    dw_post = s sum_k g_k S_k
//
// Either norm can be missing (y null: x' = x; w_pre null: no n).  Bounded by memory: a row is read once into registers, its sums
// are taken across the threads that hold it, and what it gives is written once.  A row is held by a wave (no barrier) or by a block.
// bf16: 16384 rows of 5120 forward, 671 MB, 150 us (4.5 TB/s); 8192 rows of 4096 backward, 403 MB, 94 us (4.3 TB/s) and 4 for the
// column sums; one row 7 us, the launch.
#include "row_pack.h"

#include <algorithm>
#include <cmath>

namespace edgc {
namespace {

// A value's sum over the wave, in every lane: within rows of 16 lanes, then across them
__device__ __forceinline__ float wave_sum(float v)
{
    auto add = [&](auto ctrl, auto rows) {
        v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, true));
    };
    using std::integral_constant;
    add(integral_constant<int, 0xb1>{}, integral_constant<int, 0xf>{});      // lane ^ 1
    add(integral_constant<int, 0x4e>{}, integral_constant<int, 0xf>{});      // lane ^ 2
    add(integral_constant<int, 0x141>{}, integral_constant<int, 0xf>{});     // mirrored in 8
    add(integral_constant<int, 0x140>{}, integral_constant<int, 0xf>{});     // mirrored in 16
    add(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});     // lane 15 of rows 0 and 2 onto the next row
    add(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});     // lane 31 onto rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Its sum over the threads that hold a row, in every one of them.  Sums one after the other use the two halves of `s` in turn, so
// that one barrier per sum is enough.
constexpr int kMaxWaves = 16;
template <bool WAVE>
__device__ __forceinline__ float row_sum(float v, float* s, uint32_t& turn)
{
    v = wave_sum(v);
    if constexpr (!WAVE) {
        const uint32_t waves = blockDim.x / 64, lane = threadIdx.x & 63;
        float* const h = s + (turn & 1u) * kMaxWaves;
        ++turn;
        if (lane == 0) h[threadIdx.x / 64] = v;
        __syncthreads();
        v = wave_sum(lane < waves ? h[lane] : 0.f);
    }
    return v;
}

struct NormArgs {
    const void *x, *y, *w_post, *gate, *w_pre, *dx_out, *dn;
    void *x_out, *n, *dx, *dy;
    float *rstd_post, *rstd_pre;
    void* dgate;
    float* part;                    // backward: [blocks][4][hidden]
    uint64_t tokens;
    uint32_t hidden, rows;          // rows: tokens per group of threads
    uint64_t rows_per_gate;
    float scale, eps, inv_hidden;
};

constexpr int kWaveRows = 4;        // rows per block where a wave holds one
template <typename T, int VPT, bool WAVE>
__global__ __launch_bounds__(WAVE ? 64 * kWaveRows : 64 * kMaxWaves) void k_norm_forward(const NormArgs a)
{
    constexpr int N = Pack<T>::N;
    __shared__ float s[2 * kMaxWaves];
    uint32_t turn = 0;
    const uint32_t NT = WAVE ? 64u : blockDim.x, tid = WAVE ? threadIdx.x & 63u : threadIdx.x, H = a.hidden;
    const uint32_t group = WAVE ? blockIdx.x * kWaveRows + threadIdx.x / 64u : blockIdx.x;
    const uint64_t r0 = static_cast<uint64_t>(group) * a.rows, r1 = min(a.tokens, r0 + a.rows);
    uint32_t col[VPT], len[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        col[j] = (tid + j * NT) * N;
        len[j] = col[j] < H ? min(static_cast<uint32_t>(N), H - col[j]) : 0u;
    }
    Pack<T> wpost[VPT], wpre[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        if (a.y) wpost[j].load(static_cast<const T*>(a.w_post) + col[j], len[j]);
        if (a.w_pre) wpre[j].load(static_cast<const T*>(a.w_pre) + col[j], len[j]);
    }
    for (uint64_t r = r0; r < r1; ++r) {
        const uint64_t at = r * H;
        Pack<T> x[VPT], y[VPT];
        float xo[VPT][N];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            x[j].load(static_cast<const T*>(a.x) + at + col[j], len[j]);
            if (a.y) y[j].load(static_cast<const T*>(a.y) + at + col[j], len[j]);
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) xo[j][i] = x[j].get(i);
        if (a.y) {
            float q = 0.f;
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) q = __builtin_fmaf(y[j].get(i), y[j].get(i), q);
            q = row_sum<WAVE>(q, s, turn);
            const float rs = 1.0f / sqrtf(q * a.inv_hidden + a.eps);
            if (a.rstd_post && tid == 0) a.rstd_post[r] = rs;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                Pack<T> g;
                if (a.gate) g.load(static_cast<const T*>(a.gate) + (r / a.rows_per_gate) * H + col[j], len[j]);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float c = a.gate ? a.scale * g.get(i) : a.scale;
                    xo[j][i] = __builtin_fmaf(c, y[j].get(i) * rs * wpost[j].get(i), xo[j][i]);
                }
            }
        }
        if (a.x_out) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                Pack<T> o;
                o.set(xo[j]);
                o.store(static_cast<T*>(a.x_out) + at + col[j], len[j]);
            }
        }
        if (a.w_pre) {
            float q = 0.f;
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) q = __builtin_fmaf(xo[j][i], xo[j][i], q);
            q = row_sum<WAVE>(q, s, turn);
            const float rs = 1.0f / sqrtf(q * a.inv_hidden + a.eps);
            if (a.rstd_pre && tid == 0) a.rstd_pre[r] = rs;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                float f[N];
#pragma unroll
                for (int i = 0; i < N; ++i) f[i] = xo[j][i] * rs * wpre[j].get(i);
                Pack<T> o;
                o.set(f);
                o.store(static_cast<T*>(a.n) + at + col[j], len[j]);
            }
        }
    }
}

// Column sums of a group of rows (part, four rows of `hidden` per group of threads): 0 dn xh, 1 g_k d yh, 2 and 3 the group's share
// of S of a gate row whose tokens other groups have too: 2 of a row begun before this group, 3 of one that begins here and goes on.
// A gate row that begins and ends here is written at once.
enum { kSumPre = 0, kSumPost = 1, kSumHead = 2, kSumTail = 3, kSums = 4 };

template <typename T, int VPT, bool WAVE>
__global__ __launch_bounds__(WAVE ? 64 * kWaveRows : 64 * kMaxWaves) void k_norm_backward(const NormArgs a)
{
    constexpr int N = Pack<T>::N;
    __shared__ float s[2 * kMaxWaves];
    uint32_t turn = 0;
    const uint32_t NT = WAVE ? 64u : blockDim.x, tid = WAVE ? threadIdx.x & 63u : threadIdx.x, H = a.hidden;
    const uint32_t group = WAVE ? blockIdx.x * kWaveRows + threadIdx.x / 64u : blockIdx.x;
    const uint64_t r0 = static_cast<uint64_t>(group) * a.rows, r1 = min(a.tokens, r0 + a.rows);
    if (r0 >= r1) return;           // (whole waves where a wave holds a row, whole blocks otherwise)
    uint32_t col[VPT], len[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        col[j] = (tid + j * NT) * N;
        len[j] = col[j] < H ? min(static_cast<uint32_t>(N), H - col[j]) : 0u;
    }
    Pack<T> wpost[VPT], wpre[VPT], g[VPT];
    float sum_pre[VPT][N] = {}, sum_post[VPT][N] = {}, sum_gate[VPT][N] = {};
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        if (a.y) wpost[j].load(static_cast<const T*>(a.w_post) + col[j], len[j]);
        if (a.w_pre) wpre[j].load(static_cast<const T*>(a.w_pre) + col[j], len[j]);
    }
    float* const part = a.part + static_cast<uint64_t>(group) * kSums * H;
    auto put_sums = [&](float* to, const float (&v)[VPT][N]) {
#pragma unroll
        for (int j = 0; j < VPT; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (static_cast<uint32_t>(i) < len[j]) to[col[j] + i] = v[j][i];
    };
    uint64_t gate_row = a.gate ? r0 / a.rows_per_gate : 0;
    uint64_t gate_end = a.gate ? (gate_row + 1) * a.rows_per_gate : a.tokens;
    if (a.gate)
#pragma unroll
        for (int j = 0; j < VPT; ++j) g[j].load(static_cast<const T*>(a.gate) + gate_row * H + col[j], len[j]);
    for (uint64_t r = r0; r < r1; ++r) {
        const uint64_t at = r * H;
        const float rs1 = a.y ? a.rstd_post[r] : 0.f, rs2 = a.w_pre ? a.rstd_pre[r] : 0.f;
        Pack<T> xo[VPT], y[VPT], dn[VPT], dxo[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if (a.dx_out) dxo[j].load(static_cast<const T*>(a.dx_out) + at + col[j], len[j]);
            else dxo[j].v = u32x4r{0, 0, 0, 0};
            if (a.w_pre) {
                dn[j].load(static_cast<const T*>(a.dn) + at + col[j], len[j]);
                xo[j].load(static_cast<const T*>(a.x_out) + at + col[j], len[j]);
            }
            if (a.y) y[j].load(static_cast<const T*>(a.y) + at + col[j], len[j]);
        }
        float d[VPT][N];
#pragma unroll
        for (int j = 0; j < VPT; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) d[j][i] = dxo[j].get(i);
        if (a.w_pre) {
            float q = 0.f;
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float xh = xo[j].get(i) * rs2, dni = dn[j].get(i);
                    q = __builtin_fmaf(dni * wpre[j].get(i), xh, q);
                    sum_pre[j][i] = __builtin_fmaf(dni, xh, sum_pre[j][i]);
                }
            q = row_sum<WAVE>(q, s, turn);
            const float c = q * a.inv_hidden;
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float xh = xo[j].get(i) * rs2;
                    d[j][i] = __builtin_fmaf(rs2, dn[j].get(i) * wpre[j].get(i) - xh * c, d[j][i]);
                }
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            Pack<T> o;
            o.set(d[j]);
            o.store(static_cast<T*>(a.dx) + at + col[j], len[j]);
        }
        if (a.y) {
            if (r == gate_end) {
                ++gate_row;
                gate_end += a.rows_per_gate;
#pragma unroll
                for (int j = 0; j < VPT; ++j) g[j].load(static_cast<const T*>(a.gate) + gate_row * H + col[j], len[j]);
            }
            float q = 0.f;
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float yh = y[j].get(i) * rs1, dyh = d[j][i] * yh;
                    sum_gate[j][i] += dyh;
                    const float c = a.gate ? a.scale * g[j].get(i) : a.scale;
                    q = __builtin_fmaf(c * wpost[j].get(i), dyh, q);
                }
            q = row_sum<WAVE>(q, s, turn);
            const float m = q * a.inv_hidden;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                float f[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float c = a.gate ? a.scale * g[j].get(i) : a.scale;
                    f[i] = rs1 * (c * wpost[j].get(i) * d[j][i] - y[j].get(i) * rs1 * m);
                }
                Pack<T> o;
                o.set(f);
                o.store(static_cast<T*>(a.dy) + at + col[j], len[j]);
            }
            if (r + 1 == min(gate_end, r1)) {           // the last of these tokens that have this row of the gate
                if (a.gate) {
                    const uint64_t begun = gate_row * a.rows_per_gate, end = min(gate_end, a.tokens);
                    if (begun >= r0 && end <= r1) {
#pragma unroll
                        for (int j = 0; j < VPT; ++j) {
                            float f[N];
#pragma unroll
                            for (int i = 0; i < N; ++i) f[i] = a.scale * wpost[j].get(i) * sum_gate[j][i];
                            Pack<T> o;
                            o.set(f);
                            o.store(static_cast<T*>(a.dgate) + gate_row * H + col[j], len[j]);
                        }
                    } else {
                        put_sums(part + (begun < r0 ? kSumHead : kSumTail) * static_cast<uint64_t>(H), sum_gate);
                    }
                }
#pragma unroll
                for (int j = 0; j < VPT; ++j)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        sum_post[j][i] = a.gate ? __builtin_fmaf(g[j].get(i), sum_gate[j][i], sum_post[j][i]) : sum_gate[j][i];
                        sum_gate[j][i] = 0.f;
                    }
            }
        }
    }
    if (a.w_pre) put_sums(part + kSumPre * static_cast<uint64_t>(H), sum_pre);
    if (a.y) put_sums(part + kSumPost * static_cast<uint64_t>(H), sum_post);
}

// Adds the groups' column sums up: blockIdx.y 0 dw_pre, 1 dw_post, 2 + k gate row k, or (by_group, where there are more of those than
// groups) the one that begins in group k and goes on in the next; nothing where that row is one group's.  A block takes 32 columns;
// eight threads share a column's groups.  (Looking in every group for a row that goes on, 512 of them for four rows, the launch
// took 27 us of the 120 of 8192 x 4096 bf16 rows.)
constexpr int kSumCols = 32, kSumWays = 8;
struct NormSumArgs {
    const float* part;
    const void* w_post;
    void *dw_pre, *dw_post, *dgate;
    uint64_t tokens, rows_per_gate;
    uint32_t hidden, rows, groups, by_group;
    float scale;
};
template <typename T>
__global__ __launch_bounds__(kSumCols * kSumWays) void k_norm_sum(const NormSumArgs a)
{
    __shared__ float s[kSumWays][kSumCols];
    const uint32_t c = blockIdx.x * kSumCols + threadIdx.x % kSumCols, way = threadIdx.x / kSumCols;
    const uint32_t H = a.hidden;
    const uint64_t step = static_cast<uint64_t>(kSums) * H;
    uint32_t k0 = 0, k1 = a.groups;
    uint64_t gate_row = 0;
    int which = blockIdx.y == 0 ? kSumPre : kSumPost;
    if (blockIdx.y == 0 && !a.dw_pre) return;
    if (blockIdx.y == 1 && !a.dw_post) return;
    if (blockIdx.y >= 2) {
        which = kSumHead;
        gate_row = blockIdx.y - 2;
        if (a.by_group) {
            const uint64_t next = (gate_row + 1) * a.rows;                              // the first row after the group's
            if (next >= a.tokens || (next - 1) / a.rows_per_gate * a.rows_per_gate < next - a.rows) return;     // no next, or begun earlier
            gate_row = (next - 1) / a.rows_per_gate;
        }
        const uint64_t begun = gate_row * a.rows_per_gate, end = min(begun + a.rows_per_gate, a.tokens);
        k0 = static_cast<uint32_t>(begun / a.rows);
        k1 = static_cast<uint32_t>((end - 1) / a.rows) + 1;
        if (k1 == k0 + 1) return;
    }
    float acc = 0.f;
    if (c < H) {
        const float* p = a.part + which * static_cast<uint64_t>(H) + c;
        uint32_t k = k0 + way;
        if (which == kSumHead && way == 0) {
            acc = a.part[k0 * step + kSumTail * static_cast<uint64_t>(H) + c];
            k += kSumWays;
        }
#pragma unroll 8
        for (; k < k1; k += kSumWays) acc += p[k * step];
    }
    s[way][threadIdx.x % kSumCols] = acc;
    __syncthreads();
    if (way || c >= H) return;
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kSumWays; ++w) t += s[w][threadIdx.x];
    if (blockIdx.y == 0) static_cast<T*>(a.dw_pre)[c] = static_cast<T>(t);
    else if (blockIdx.y == 1) static_cast<T*>(a.dw_post)[c] = static_cast<T>(a.scale * t);
    else static_cast<T*>(a.dgate)[gate_row * H + c] = static_cast<T>(a.scale * static_cast<float>(static_cast<const T*>(a.w_post)[c]) * t);
}

// Who holds a row: a wave up to 1024 columns, beyond that a block of as many waves as it takes.  A thread has 8 columns of it, or
// 16 where 8 are too few (a wave above 512 columns, a block above 8192).
constexpr uint32_t kMaxHidden = 16384;
template <typename T, typename F>
int by_width(uint32_t hidden, F&& f)
{
    constexpr int V = 8 / Pack<T>::N;           // items of eight columns
    using std::integral_constant;
    using std::bool_constant;
    if (hidden <= 512) return f(integral_constant<int, V>{}, bool_constant<true>{});
    if (hidden <= 1024) return f(integral_constant<int, 2 * V>{}, bool_constant<true>{});
    if (hidden <= 8192) return f(integral_constant<int, V>{}, bool_constant<false>{});
    return f(integral_constant<int, 2 * V>{}, bool_constant<false>{});
}
template <typename T>
uint32_t threads_of(uint32_t hidden, int vpt, bool wave)
{
    const uint32_t cols = 64u * vpt * Pack<T>::N;
    return wave ? 64u * kWaveRows : (hidden + cols - 1) / cols * 64u;
}

// Groups of threads that a pass is spread over at most (the backward pass leaves four rows of sums for each)
uint32_t most_groups(const edgc_ctx* ctx) { return static_cast<uint32_t>(ctx->num_cu) * 4u; }

int check_norm(edgc_ctx* ctx, edgc_dtype dtype, uint64_t tokens, uint32_t hidden, const void* gate, uint64_t rows_per_gate, float scale)
{
    if (dtype != EDGC_F32 && dtype != EDGC_BF16) return fail(ctx, EDGC_EINVAL, "unknown dtype");
    if (hidden == 0 || hidden > kMaxHidden) return fail(ctx, EDGC_EINVAL, "hidden must be 1 to 16384");
    if (tokens > (1ull << 31)) return fail(ctx, EDGC_EINVAL, "more than 2^31 tokens");
    if (gate && rows_per_gate == 0) return fail(ctx, EDGC_EINVAL, "rows_per_gate must be >= 1 with a gate");
    if (!std::isfinite(scale)) return fail(ctx, EDGC_EINVAL, "scale must be finite");
    return EDGC_OK;
}
bool any_misaligned(std::initializer_list<const void*> ps, size_t a)
{
    for (const void* p : ps)
        if (p && !aligned_to(p, a)) return true;
    return false;
}

}  // namespace
}  // namespace edgc

using namespace edgc;

extern "C" int edgc_reserve_block_norm(edgc_ctx* ctx, uint32_t tokens, uint32_t hidden)
{
    if (!ctx) return EDGC_EINVAL;
    if (hidden == 0 || hidden > kMaxHidden) return fail(ctx, EDGC_EINVAL, "hidden must be 1 to 16384");
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    const size_t need = static_cast<size_t>(std::min(tokens, most_groups(ctx))) * kSums * hidden;
    if (need == 0 || need > ctx->norm.held) {
        EDGC_HIP_TRY(ctx, hipDeviceSynchronize());      // nothing may still be using the old scratch
        if (ctx->norm.part) (void)hipFree(ctx->norm.part);
        ctx->norm = NormScratch{};
        if (need == 0) return EDGC_OK;
        if (hipMalloc(reinterpret_cast<void**>(&ctx->norm.part), need * sizeof(float)) != hipSuccess) {
            (void)hipGetLastError();
            ctx->norm = NormScratch{};
            return fail(ctx, EDGC_ENOMEM, "norm scratch allocation failed");
        }
        ctx->norm.held = need;
    }
    ctx->norm.tokens = tokens;
    ctx->norm.hidden = hidden;
    return EDGC_OK;
}

extern "C" int edgc_block_norm_forward(edgc_ctx* ctx, edgc_dtype dtype, uint64_t tokens, uint32_t hidden, const void* x, const void* y,
                                       const void* w_post, const void* gate, uint64_t rows_per_gate, const void* w_pre, float scale,
                                       float eps, void* x_out, void* n_out, float* rstd_post, float* rstd_pre, void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    if (int rc = check_norm(ctx, dtype, tokens, hidden, gate, rows_per_gate, scale)) return rc;
    if (tokens == 0) return EDGC_OK;
    if (!x || (!y && !w_pre)) return fail(ctx, EDGC_EINVAL, "null x, or neither norm given");
    if (y && (!w_post || !x_out)) return fail(ctx, EDGC_EINVAL, "y needs w_post and x_out");
    if (!y && (w_post || gate)) return fail(ctx, EDGC_EINVAL, "w_post and gate belong to y");
    if (w_pre && !n_out) return fail(ctx, EDGC_EINVAL, "w_pre needs n_out");
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(ctx, EDGC_EINVAL, "eps must be finite and not negative");
    if (any_misaligned({x, y, w_post, gate, w_pre, x_out, n_out}, dtype == EDGC_F32 ? 4 : 2) || any_misaligned({rstd_post, rstd_pre}, 4))
        return fail(ctx, EDGC_EINVAL, "misaligned pointer");
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    NormArgs a{};
    a.x = x; a.y = y; a.w_post = w_post; a.gate = gate; a.w_pre = w_pre;
    a.x_out = x_out; a.n = n_out; a.rstd_post = rstd_post; a.rstd_pre = rstd_pre;
    a.tokens = tokens; a.hidden = hidden; a.rows_per_gate = rows_per_gate;
    a.scale = scale; a.eps = eps; a.inv_hidden = 1.0f / static_cast<float>(hidden);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto go = [&](auto type) {
        using T = decltype(type);
        return by_width<T>(hidden, [&](auto vpt, auto wave) -> int {
            constexpr int VPT = decltype(vpt)::value;
            constexpr bool WAVE = decltype(wave)::value;
            constexpr uint32_t G = WAVE ? kWaveRows : 1;
            const uint32_t threads = threads_of<T>(hidden, VPT, WAVE);
            const uint64_t most = static_cast<uint64_t>(ctx->num_cu) * (2048u / threads) * G;
            const uint64_t groups = std::min(tokens, most);
            a.rows = static_cast<uint32_t>((tokens + groups - 1) / groups);
            const uint32_t blocks = static_cast<uint32_t>(((tokens + a.rows - 1) / a.rows + G - 1) / G);
            const double bytes = static_cast<double>(tokens) * hidden * sizeof(T) * (1 + (y ? 2 : 0) + (w_pre ? 1 : 0));
            EDGC_LAUNCH(ctx, st, KID_NORM_FORWARD, bytes, 0.0, k_norm_forward<T, VPT, WAVE><<<blocks, threads, 0, st>>>(a));
            EDGC_HIP_TRY(ctx, hipGetLastError());
            return EDGC_OK;
        });
    };
    return dtype == EDGC_F32 ? go(float{}) : go(__bf16{});
}

extern "C" int edgc_block_norm_backward(edgc_ctx* ctx, edgc_dtype dtype, uint64_t tokens, uint32_t hidden, const void* dx_out,
                                        const void* dn, const void* x_out, const void* y, const void* w_post, const void* gate,
                                        uint64_t rows_per_gate, const void* w_pre, const float* rstd_post, const float* rstd_pre,
                                        float scale, void* dx, void* dy, void* dw_post, void* dgate, void* dw_pre, void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    if (int rc = check_norm(ctx, dtype, tokens, hidden, gate, rows_per_gate, scale)) return rc;
    if (!w_post && !w_pre) return fail(ctx, EDGC_EINVAL, "neither norm given");
    if (tokens && (!dx || (y && (!rstd_post || !dy || !dx_out)) || (w_pre && (!dn || !x_out || !rstd_pre))))
        return fail(ctx, EDGC_EINVAL, "null dx, or null inputs or gradients of a norm");
    if ((w_post && !dw_post) || (w_pre && !dw_pre)) return fail(ctx, EDGC_EINVAL, "null weight gradient of a norm");
    if ((tokens && !y != !w_post) || (gate && !w_post)) return fail(ctx, EDGC_EINVAL, "y and w_post go together, and gate belongs to them");
    if (gate && !dgate) return fail(ctx, EDGC_EINVAL, "gate needs dgate");
    if (any_misaligned({dx_out, dn, x_out, y, w_post, gate, w_pre, dx, dy, dw_post, dgate, dw_pre}, dtype == EDGC_F32 ? 4 : 2) ||
        any_misaligned({rstd_post, rstd_pre}, 4))
        return fail(ctx, EDGC_EINVAL, "misaligned pointer");
    if (tokens > ctx->norm.tokens || (tokens && hidden > ctx->norm.hidden))
        return fail(ctx, EDGC_EINVAL, "more tokens or hidden units than edgc_reserve_block_norm was called for");
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    NormArgs a{};
    a.dx_out = dx_out; a.dn = dn; a.x_out = const_cast<void*>(x_out); a.y = y; a.w_post = w_post; a.gate = gate; a.w_pre = w_pre;
    a.rstd_post = const_cast<float*>(rstd_post); a.rstd_pre = const_cast<float*>(rstd_pre);
    a.dx = dx; a.dy = dy; a.dgate = dgate; a.part = ctx->norm.part;
    a.tokens = tokens; a.hidden = hidden; a.rows_per_gate = rows_per_gate;
    a.scale = scale; a.inv_hidden = 1.0f / static_cast<float>(hidden);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto go = [&](auto type) {
        using T = decltype(type);
        return by_width<T>(hidden, [&](auto vpt, auto wave) -> int {
            constexpr int VPT = decltype(vpt)::value;
            constexpr bool WAVE = decltype(wave)::value;
            constexpr uint32_t G = WAVE ? kWaveRows : 1;
            const uint32_t threads = threads_of<T>(hidden, VPT, WAVE);
            uint32_t groups = 0;
            if (tokens) {
                const uint64_t most = std::min<uint64_t>({tokens, most_groups(ctx), static_cast<uint64_t>(ctx->num_cu) * std::max(1u, 1024u / threads) * G});
                a.rows = static_cast<uint32_t>((tokens + most - 1) / most);
                groups = static_cast<uint32_t>((tokens + a.rows - 1) / a.rows);
                const uint32_t blocks = (groups + G - 1) / G;
                const double bytes = static_cast<double>(tokens) * hidden * sizeof(T) * (1 + (dx_out ? 1 : 0) + (y ? 2 : 0) + (w_pre ? 2 : 0));
                EDGC_LAUNCH(ctx, st, KID_NORM_BACKWARD, bytes, 0.0, k_norm_backward<T, VPT, WAVE><<<blocks, threads, 0, st>>>(a));
                EDGC_HIP_TRY(ctx, hipGetLastError());
            }
            NormSumArgs b{};
            b.part = ctx->norm.part; b.w_post = w_post; b.dw_pre = w_pre ? dw_pre : nullptr; b.dw_post = w_post ? dw_post : nullptr; b.dgate = dgate;
            b.tokens = tokens; b.rows_per_gate = rows_per_gate; b.hidden = hidden; b.rows = a.rows; b.groups = groups; b.scale = scale;
            // gate rows that go over a group's end can only be where rows of the gate are longer than one token
            const uint64_t gates = gate && groups > 1 && rows_per_gate > 1 ? (tokens - 1) / rows_per_gate + 1 : 0;
            b.by_group = gates && gates >= groups;
            const uint32_t crossing = b.by_group ? groups - 1 : static_cast<uint32_t>(gates);
            const dim3 grid((hidden + kSumCols - 1) / kSumCols, 2 + crossing);
            EDGC_LAUNCH(ctx, st, KID_NORM_SUM, static_cast<double>(groups) * hidden * 4.0 * 2.0, 0.0,
                        k_norm_sum<T><<<grid, kSumCols * kSumWays, 0, st>>>(b));
            EDGC_HIP_TRY(ctx, hipGetLastError());
            return EDGC_OK;
        });
    };
    return dtype == EDGC_F32 ? go(float{}) : go(__bf16{});
}
