// The norms of queries and keys, head by head, with the rotation by position in the same pass, and their backward pass.
//
//   forward   r = (mean x^2 + eps)^-1/2,  y = R(x r w):  pairs (a, b) of the first 2 n dimensions become (a cos - b sin, b cos + a sin), of the angles
//             position * inv_freq[i]
//   backward  d = R^T dy,  u = d w,  xh = x r,  dx = r (u - xh mean(u xh)),  dw = sum over tokens and heads of d xh
//
// Bounded by memory.  Angles are taken in 64 bits (a position of a million leaves 32 bits two digits) once per token, for all heads, into LDS.  A head is held
// by as many lanes as it has units of two packs of 16 bytes, a pack of each half's or two neighbours, so that a lane has both of a pair.
#include "row_pack.h"

#include <algorithm>
#include <cmath>

namespace edgc {
namespace {

constexpr uint32_t kQkMaxDim = 512, kQkMaxHeads = 1u << 16;
constexpr uint32_t kQkTokens = 8;               // whose angles are in LDS at a time

struct QkHeads {
    const void *x, *dy;
    void* out;                                  // y, or dx
    const void* w;
    uint64_t x_token, x_head, dy_token, dy_head, out_token, out_head;       // elements
    uint32_t heads;
};
struct QkArgs {
    QkHeads h[2];                               // queries, keys
    const void* positions;
    const double* inv_freq;
    float* part;                                // backward: [blocks][2][dim]
    uint64_t tokens;
    uint32_t dim, pairs, per;                   // pairs that are rotated; tokens of a block
    uint32_t lanes;                             // of a head: a power of two
    int interleaved, pos_bytes;
    float eps, inv_dim;
};

// N elements of a head: 16 bytes, or one.  STREAM: past the caches
template <typename T, int N, bool STREAM> struct QkPack {
    static_assert(N == Pack<T>::N, "");
    Pack<T> v;
    __device__ __forceinline__ void load(const T* p, uint32_t len) { v.template load<STREAM>(p, len); }
    __device__ __forceinline__ float get(int i) const { return v.get(i); }
    static __device__ __forceinline__ void store(T* p, uint32_t len, const float (&f)[N])
    {
        Pack<T> o;
        o.set(f);
        o.template store<STREAM>(p, len);
    }
};
template <typename T> struct QkPack<T, 1, false> {
    float v;
    __device__ __forceinline__ void load(const T* p, uint32_t len) { v = len ? static_cast<float>(*p) : 0.f; }
    __device__ __forceinline__ float get(int) const { return v; }
    static __device__ __forceinline__ void store(T* p, uint32_t len, const float (&f)[1])
    {
        if (len) *p = static_cast<T>(f[0]);
    }
};

// Where the two packs of unit u are, and the angle of their first pair; the pairs are (first, second) or neighbours in either.  Units behind the rotated ones
// are neighbours without an angle.
template <int N>
struct QkUnit {
    uint32_t first, second, angle;
    bool turns;
    __device__ __forceinline__ QkUnit(const QkArgs& a, uint32_t u)
    {
        const uint32_t turned = a.pairs / N;    // (a multiple, where N > 1)
        turns = u < turned;
        if (turns && !a.interleaved) {
            first = u * N;
            second = a.pairs + u * N;
            angle = u * N;
        } else {
            first = 2 * u * N;
            second = first + N;
            angle = u * N;
        }
    }
};
// (sin, cos) of a position's angle
__device__ __forceinline__ float2 qk_angle(const QkArgs& a, uint64_t token, uint32_t i)
{
    const double p = a.pos_bytes == 8 ? static_cast<double>(static_cast<const int64_t*>(a.positions)[token]) : static_cast<double>(static_cast<const int32_t*>(a.positions)[token]);
    // parts of a circle, 1 / 2 pi and the product with it in two doubles each: of a far position whole circles take the digits of one
    const double angle = p * a.inv_freq[i], turn = angle * 0.15915494309189535, rest = fma(angle, 0.15915494309189535, -turn) + angle * -9.839338337591243e-18;
    const double quarters = 4.0 * ((turn - rint(turn)) + rest), q = rint(quarters);
    float s, c;
    sincospif(0.5f * static_cast<float>(quarters - q), &s, &c);
    const int k = static_cast<int>(q) & 3;
    const float sn = k & 1 ? c : s, cs = k & 1 ? s : c;
    return {k & 2 ? -sn : sn, (k + 1) & 2 ? -cs : cs};
}

// Rotates the N pairs of a unit, by its angles or (BACK) back
template <int N, bool BACK>
__device__ __forceinline__ void qk_turn(const QkArgs& a, const QkUnit<N>& u, const float2* angles, float (&x)[N], float (&y)[N])
{
    if (!u.turns) return;
    auto one = [&](float& p, float& q, const float2& t) {
        const float s = BACK ? -t.x : t.x, r = p * t.y - q * s;
        q = q * t.y + p * s;
        p = r;
    };
    if (!a.interleaved || N == 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) one(x[i], y[i], angles[u.angle + i]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            one(x[2 * i], x[2 * i + 1], angles[u.angle + i]);
            one(y[2 * i], y[2 * i + 1], angles[u.angle + N / 2 + i]);
        }
    }
}
// A value's sum over a head's lanes, in every one of them
__device__ __forceinline__ float qk_head_sum(float v, uint32_t lanes)
{
    auto add = [&](auto ctrl) { v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    using std::integral_constant;
    if (lanes > 1) add(integral_constant<int, 0xb1>{});         // lane ^ 1
    if (lanes > 2) add(integral_constant<int, 0x4e>{});         // lane ^ 2
    if (lanes > 4) add(integral_constant<int, 0x141>{});        // mirrored in 8
    if (lanes > 8) add(integral_constant<int, 0x140>{});        // mirrored in 16
    if (lanes > 16) v += __shfl_xor(v, 16, 64);
    if (lanes > 32) v += __shfl_xor(v, 32, 64);
    return v;
}

// A block has `per` tokens.  Few tokens: blockIdx.z: queries, keys; forward, blockIdx.y: a share of the heads
template <typename T, int N, int U, bool BACK, bool STREAM>
__global__ __launch_bounds__(256, 4) void k_qk_norm(const QkArgs a)
{
    using Item = QkPack<T, N, STREAM>;
    extern __shared__ float2 angles[];          // [kQkTokens][pairs]; BACK: and [groups][dim] sums
    const uint32_t lane = threadIdx.x & 63, in = lane & (a.lanes - 1), group = (threadIdx.x / a.lanes), groups = 256 / a.lanes;
    const uint64_t t0 = static_cast<uint64_t>(blockIdx.x) * a.per, t1 = min(a.tokens, t0 + a.per);
    const uint32_t units = (a.dim + 2 * N - 1) / (2 * N);
    auto len = [&](uint32_t u, uint32_t at) { return u < units && at < a.dim ? min(static_cast<uint32_t>(N), a.dim - at) : 0u; };
    auto turn_by = [&](uint64_t b0, uint32_t n) {       // the angles of n tokens
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < n * a.pairs; i += 256) angles[i] = qk_angle(a, b0 + i / a.pairs, i % a.pairs);
        __syncthreads();
    };
    // queries, then keys: of one of them the sums fit a wave's registers with three others on its SIMD (both: 161, a third of the blocks in a second round)
    const int K0 = gridDim.z > 1 ? blockIdx.z : 0, K1 = gridDim.z > 1 ? K0 + 1 : 2;
    for (int K = K0; K < K1; ++K) {
        const QkHeads& h = a.h[K];
        const uint32_t share = (h.heads + gridDim.y - 1) / gridDim.y, h0 = blockIdx.y * share, h1 = min(h.heads, h0 + share), H = h1 > h0 ? h1 - h0 : 0u;
        float sums[U][2][BACK ? N : 1] = {};
        Item w[U][2];
        if (H) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const QkUnit<N> u(a, in + k * a.lanes);
                w[k][0].load(static_cast<const T*>(h.w) + u.first, len(in + k * a.lanes, u.first));
                w[k][1].load(static_cast<const T*>(h.w) + u.second, len(in + k * a.lanes, u.second));
            }
        }
        for (uint64_t b0 = t0; b0 < t1; b0 += kQkTokens) {
            const uint32_t n = static_cast<uint32_t>(min(static_cast<uint64_t>(kQkTokens), t1 - b0));
            // heads of the tokens one after the other, a group of lanes each; forward, the next one's elements are on their way during a head
            const uint32_t items = n * H, rounds = (items + groups - 1) / groups;      // (all lanes of a wave take part in the sums)
            const uint32_t some = max(H, 1u), tokens_on = groups / some, heads_on = groups - tokens_on * some;
            uint32_t it = group, tok = group / some, hd = group - tok * some;
            Item v[U][2], d[U][2], next[U][2];
            auto ask = [&](Item (&xs)[U][2], Item (&ds)[U][2]) {
                const uint64_t token = b0 + tok, head = h0 + hd;
                const T* const x = static_cast<const T*>(h.x) + token * h.x_token + head * h.x_head;
                const T* const dy = BACK ? static_cast<const T*>(h.dy) + token * h.dy_token + head * h.dy_head : nullptr;
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const uint32_t unit = in + k * a.lanes;
                    const QkUnit<N> u(a, unit);
                    xs[k][0].load(x + u.first, len(unit, u.first));
                    xs[k][1].load(x + u.second, len(unit, u.second));
                    if constexpr (BACK) {
                        ds[k][0].load(dy + u.first, len(unit, u.first));
                        ds[k][1].load(dy + u.second, len(unit, u.second));
                    }
                }
            };
            // (on their way during the angles)
            if (it < items) ask(BACK ? v : next, d);
            if (K == K0 || t1 - t0 > kQkTokens) turn_by(b0, n);
            for (uint32_t round = 0; round < rounds; ++round) {
                const bool there = it < items;
                const uint64_t token = b0 + tok, head = h0 + hd;
                T* const out = static_cast<T*>(h.out) + token * h.out_token + head * h.out_head;
                const float2* const turn = angles + (there ? tok : 0u) * a.pairs;
                if constexpr (BACK) {
                    if (there && round) ask(v, d);
                } else {
#pragma unroll
                    for (int k = 0; k < U; ++k) v[k][0] = next[k][0], v[k][1] = next[k][1];
                }
                it += groups;
                tok += tokens_on;
                hd += heads_on;
                if (hd >= H) hd -= H, ++tok;
                if (!BACK && it < items) ask(next, d);
                float q = 0.f, s = 0.f;
                float g[U][2][N];               // BACK: d, rotated back
#pragma unroll
                for (int k = 0; k < U; ++k) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        q = __builtin_fmaf(v[k][0].get(i), v[k][0].get(i), q);
                        q = __builtin_fmaf(v[k][1].get(i), v[k][1].get(i), q);
                    }
                    if constexpr (BACK) {
                        const QkUnit<N> u(a, in + k * a.lanes);
#pragma unroll
                        for (int i = 0; i < N; ++i) g[k][0][i] = d[k][0].get(i), g[k][1][i] = d[k][1].get(i);
                        qk_turn<N, true>(a, u, turn, g[k][0], g[k][1]);
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int i = 0; i < N; ++i) s = __builtin_fmaf(g[k][e][i] * w[k][e].get(i), v[k][e].get(i), s);
                    }
                }
                q = qk_head_sum(q, a.lanes);
                const float r = 1.0f / sqrtf(q * a.inv_dim + a.eps);
                float m = 0.f;
                if constexpr (BACK) m = qk_head_sum(s, a.lanes) * r * a.inv_dim;       // mean(u xh)
                if (!there) continue;
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const uint32_t unit = in + k * a.lanes;
                    const QkUnit<N> u(a, unit);
                    float y[2][N];
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const float xh = v[k][e].get(i) * r;
                            if constexpr (BACK) {
                                y[e][i] = r * (g[k][e][i] * w[k][e].get(i) - xh * m);
                                sums[k][e][i] = __builtin_fmaf(g[k][e][i], xh, sums[k][e][i]);
                            } else {
                                y[e][i] = xh * w[k][e].get(i);
                            }
                        }
                    if constexpr (!BACK) qk_turn<N, false>(a, u, turn, y[0], y[1]);
                    Item::store(out + u.first, len(unit, u.first), y[0]);
                    Item::store(out + u.second, len(unit, u.second), y[1]);
                }
            }
        }
        if constexpr (BACK) {
            // the block's sums, in the order of the groups
            float* const all = reinterpret_cast<float*>(angles + kQkTokens * a.pairs);
            __syncthreads();        // queries' have been read
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const uint32_t unit = in + k * a.lanes;
                const QkUnit<N> u(a, unit);
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const uint32_t at = e ? u.second : u.first;
                        if (static_cast<uint32_t>(i) < len(unit, at)) all[group * a.dim + at + i] = sums[k][e][i];
                    }
            }
            __syncthreads();
            for (uint32_t c = threadIdx.x; c < a.dim; c += 256) {
                float t = 0.f;
                for (uint32_t g = 0; g < groups; ++g) t += all[g * a.dim + c];
                a.part[(static_cast<uint64_t>(blockIdx.x) * 2 + K) * a.dim + c] = t;
            }
        }
    }
}

// The blocks' sums, 32 columns and kQkWays shares of the blocks per block; blockIdx.y: of queries, keys.  (With eight shares, 1024 blocks' of 128 columns 6.4 us.)
constexpr uint32_t kQkWays = 32;
template <typename T>
__global__ __launch_bounds__(32 * kQkWays) void k_qk_sum(const float* part, uint32_t blocks, uint32_t dim, void* dw_q, void* dw_k)
{
    __shared__ float s[kQkWays][33];
    const uint32_t c = blockIdx.x * 32 + threadIdx.x % 32, way = threadIdx.x / 32;
    float acc = 0.f;
    if (c < dim)
#pragma unroll 16
        for (uint32_t b = way; b < blocks; b += kQkWays) acc += part[(static_cast<uint64_t>(b) * 2 + blockIdx.y) * dim + c];
    s[way][threadIdx.x % 32] = acc;
    __syncthreads();
    T* const to = static_cast<T*>(blockIdx.y ? dw_k : dw_q);
    if (way || c >= dim || !to) return;
    float t = 0.f;
#pragma unroll
    for (uint32_t w = 0; w < kQkWays; ++w) t += s[w][threadIdx.x];
    to[c] = static_cast<T>(t);
}

// blocks of the backward pass at most: each leaves a row of sums for queries and one for keys
uint32_t qk_most_blocks(const edgc_ctx* ctx) { return static_cast<uint32_t>(ctx->num_cu) * 4u; }

struct QkShape {
    edgc_dtype dtype;
    uint64_t tokens;
    uint32_t heads_q, heads_k, dim, rot;
};
int check_heads(edgc_ctx* ctx, const edgc_heads* h, uint32_t heads, const QkShape& s, bool written)
{
    if (!h || !h->p || !aligned_to(h->p, s.dtype == EDGC_F32 ? 4 : 2)) return fail(ctx, EDGC_EINVAL, "null or misaligned heads");
    if (h->token > kMaxSpan || h->head > kMaxSpan) return fail(ctx, EDGC_EINVAL, "stride over 2^40");
    if (!written) return EDGC_OK;
    // no element twice: the nearer of the two dimensions a head or more apart, the other all of it
    const bool heads_near = h->head <= h->token;
    const uint64_t near_n = heads_near ? heads : s.tokens, far_n = heads_near ? s.tokens : heads, near = heads_near ? h->head : h->token, far = heads_near ? h->token : h->head;
    // (far is at most kMaxSpan: what passes that needs no exact span)
    const uint64_t span = near_n > 1 ? (near > kMaxSpan / (near_n - 1) ? 2 * kMaxSpan : (near_n - 1) * near + s.dim) : s.dim;
    if ((near_n > 1 && near < s.dim) || (far_n > 1 && far < span)) return fail(ctx, EDGC_EINVAL, "heads that are written overlap");
    return EDGC_OK;
}
int check_qk(edgc_ctx* ctx, const QkShape& s, const void* w_q, const void* w_k, const void* positions, int pos_bytes, const double* inv_freq, float eps)
{
    if (s.dtype != EDGC_F32 && s.dtype != EDGC_BF16) return fail(ctx, EDGC_EINVAL, "unknown dtype");
    if (s.dim == 0 || s.dim > kQkMaxDim) return fail(ctx, EDGC_EINVAL, "a head has 1 to 512 dimensions");
    if (s.heads_q == 0 || s.heads_q > kQkMaxHeads || s.heads_k > kQkMaxHeads) return fail(ctx, EDGC_EINVAL, "heads must be 1 to 2^16 (of keys, 0 too)");
    if (s.tokens > (1ull << 31)) return fail(ctx, EDGC_EINVAL, "more than 2^31 tokens");
    if (s.rot > s.dim || s.rot % 2) return fail(ctx, EDGC_EINVAL, "the rotated dimensions must be even and no more than a head has");
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(ctx, EDGC_EINVAL, "eps must be finite and not negative");
    const size_t esz = s.dtype == EDGC_F32 ? 4 : 2;
    if (!w_q || !aligned_to(w_q, esz) || (s.heads_k && (!w_k || !aligned_to(w_k, esz)))) return fail(ctx, EDGC_EINVAL, "null or misaligned weight");
    if (s.rot && s.tokens) {
        if (pos_bytes != 4 && pos_bytes != 8) return fail(ctx, EDGC_EINVAL, "positions have 4 or 8 bytes");
        if (!positions || !aligned_to(positions, static_cast<size_t>(pos_bytes)) || !inv_freq || !aligned_to(inv_freq, 8))
            return fail(ctx, EDGC_EINVAL, "null or misaligned positions or frequencies");
    }
    return EDGC_OK;
}

// f(type, elements of a pack, units of a lane): packs of 16 bytes where halves, or pairs, and what is not rotated are whole units of two of them
template <typename F>
int by_head(const QkShape& s, QkArgs& a, F&& f)
{
    using std::integral_constant;
    auto lanes = [&](uint32_t units) {
        a.lanes = 1;
        while (a.lanes < units && a.lanes < 64) a.lanes *= 2;
        return (units + a.lanes - 1) / a.lanes;
    };
    auto go = [&](auto type) -> int {
        using T = decltype(type);
        constexpr uint32_t N = Pack<T>::N;
        if (s.dim % (2 * N) == 0 && s.rot % (2 * N) == 0) {
            (void)lanes(s.dim / (2 * N));
            return f(type, integral_constant<int, N>{}, integral_constant<int, 1>{});
        }
        switch (lanes((s.dim + 1) / 2)) {
            case 1: return f(type, integral_constant<int, 1>{}, integral_constant<int, 1>{});
            case 2: return f(type, integral_constant<int, 1>{}, integral_constant<int, 2>{});
            default: return f(type, integral_constant<int, 1>{}, integral_constant<int, 4>{});
        }
    };
    return s.dtype == EDGC_F32 ? go(float{}) : go(__bf16{});
}

// f(whether heads go past the caches): what moves more than 2^27 bytes is not there any more when it is next looked for.  (16384 tokens of 40 and 8 heads of 128,
// bf16, 403 MB: 84.5 us through the caches, 81.5 past them; backward, 8192 tokens of 32 and 8, 251 MB: 58.5 and 55; 1001 of 7 and 3 of 72, fp32, 9 MB: 6.3 and
// 7.4.)
template <int N, typename F>
int by_size(double bytes, F&& f)
{
    if constexpr (N > 1)
        if (bytes > 134217728.0) return f(std::true_type{});
    return f(std::false_type{});
}

QkHeads qk_heads(const edgc_heads* x, const edgc_heads* dy, const edgc_heads* out, const void* w, uint32_t heads)
{
    QkHeads h{};
    h.heads = heads;
    if (!heads) return h;
    h.x = x->p; h.x_token = x->token; h.x_head = x->head;
    if (dy) h.dy = dy->p, h.dy_token = dy->token, h.dy_head = dy->head;
    h.out = out->p; h.out_token = out->token; h.out_head = out->head;
    h.w = w;
    return h;
}

}  // namespace

void free_qk(edgc_ctx* ctx)
{
    if (ctx->qk.part) (void)hipFree(ctx->qk.part);
    ctx->qk = QkScratch{};
}

}  // namespace edgc

using namespace edgc;

extern "C" int edgc_qk_norm_forward(edgc_ctx* ctx, edgc_dtype dtype, uint64_t tokens, uint32_t heads_q, uint32_t heads_k, uint32_t dim, const edgc_heads* q,
                                    const edgc_heads* k, const void* w_q, const void* w_k, const void* positions, int pos_bytes, const double* inv_freq,
                                    uint32_t rot, int interleaved, float eps, const edgc_heads* q_out, const edgc_heads* k_out, void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    const QkShape s{dtype, tokens, heads_q, heads_k, dim, rot};
    if (int rc = check_qk(ctx, s, w_q, w_k, positions, pos_bytes, inv_freq, eps)) return rc;
    if (tokens == 0) return EDGC_OK;
    if (int rc = check_heads(ctx, q, heads_q, s, false)) return rc;
    if (int rc = check_heads(ctx, q_out, heads_q, s, true)) return rc;
    if (heads_k) {
        if (int rc = check_heads(ctx, k, heads_k, s, false)) return rc;
        if (int rc = check_heads(ctx, k_out, heads_k, s, true)) return rc;
    }
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    QkArgs a{};
    a.h[0] = qk_heads(q, nullptr, q_out, w_q, heads_q);
    a.h[1] = qk_heads(k, nullptr, k_out, w_k, heads_k);
    a.positions = positions; a.inv_freq = inv_freq; a.tokens = tokens; a.dim = dim; a.pairs = rot / 2;
    a.interleaved = interleaved; a.pos_bytes = pos_bytes; a.eps = eps; a.inv_dim = 1.0f / static_cast<float>(dim);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return by_head(s, a, [&](auto type, auto n, auto u) -> int {
        using T = decltype(type);
        const uint64_t most = static_cast<uint64_t>(ctx->num_cu) * 8;
        a.per = static_cast<uint32_t>(std::max<uint64_t>(1, (tokens + most - 1) / most));
        const uint32_t blocks = static_cast<uint32_t>((tokens + a.per - 1) / a.per), groups = 256 / a.lanes;
        // few tokens: a block for as many heads as it takes at a time, of queries or keys (eight tokens of 32 and 8 heads: 2.8 us, with
        // both in turn 5.0)
        const bool few = blocks < static_cast<uint32_t>(ctx->num_cu);
        const uint32_t shares = few ? std::max(1u, std::min((std::max(heads_q, heads_k) + groups - 1) / groups, 64u)) : 1u;
        const double bytes = 2.0 * sizeof(T) * tokens * (heads_q + heads_k) * dim;
        return by_size<n>(bytes, [&](auto stream) -> int {
            EDGC_LAUNCH(ctx, st, KID_QK_FORWARD, bytes, 0.0,
                        k_qk_norm<T, n, u, false, stream>
                        <<<dim3(blocks, shares, few && heads_k ? 2 : 1), 256, kQkTokens * std::max(1u, a.pairs) * sizeof(float2), st>>>(a));
            EDGC_HIP_TRY(ctx, hipGetLastError());
            return EDGC_OK;
        });
    });
}

extern "C" int edgc_reserve_qk_norm(edgc_ctx* ctx, uint32_t tokens, uint32_t heads_q, uint32_t heads_k, uint32_t dim)
{
    if (!ctx) return EDGC_EINVAL;
    if (dim == 0 || dim > kQkMaxDim) return fail(ctx, EDGC_EINVAL, "a head has 1 to 512 dimensions");
    if (heads_q == 0 || heads_q > kQkMaxHeads || heads_k > kQkMaxHeads) return fail(ctx, EDGC_EINVAL, "heads must be 1 to 2^16 (of keys, 0 too)");
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    const size_t need = static_cast<size_t>(std::min(tokens, qk_most_blocks(ctx))) * 2 * dim;
    if (need == 0 || need > ctx->qk.held) {
        EDGC_HIP_TRY(ctx, hipDeviceSynchronize());      // nothing may still be using the old scratch
        free_qk(ctx);
        if (need == 0) return EDGC_OK;
        if (hipMalloc(reinterpret_cast<void**>(&ctx->qk.part), need * sizeof(float)) != hipSuccess) {
            (void)hipGetLastError();
            ctx->qk = QkScratch{};
            return fail(ctx, EDGC_ENOMEM, "scratch allocation of the norms of queries and keys failed");
        }
        ctx->qk.held = need;
    }
    ctx->qk.tokens = tokens;
    ctx->qk.dim = dim;
    ctx->qk.heads_q = heads_q;
    ctx->qk.heads_k = heads_k;
    return EDGC_OK;
}

extern "C" int edgc_qk_norm_backward(edgc_ctx* ctx, edgc_dtype dtype, uint64_t tokens, uint32_t heads_q, uint32_t heads_k, uint32_t dim, const edgc_heads* dq_out,
                                     const edgc_heads* dk_out, const edgc_heads* q, const edgc_heads* k, const void* w_q, const void* w_k,
                                     const void* positions, int pos_bytes, const double* inv_freq, uint32_t rot, int interleaved, float eps,
                                     const edgc_heads* dq, const edgc_heads* dk, void* dw_q, void* dw_k, void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    const QkShape s{dtype, tokens, heads_q, heads_k, dim, rot};
    if (int rc = check_qk(ctx, s, w_q, w_k, positions, pos_bytes, inv_freq, eps)) return rc;
    const size_t esz = dtype == EDGC_F32 ? 4 : 2;
    if (!dw_q || !aligned_to(dw_q, esz) || (heads_k && !dw_k) || (dw_k && !aligned_to(dw_k, esz))) return fail(ctx, EDGC_EINVAL, "null or misaligned weight gradient");
    if (tokens) {
        for (const edgc_heads* h : {q, dq_out})
            if (int rc = check_heads(ctx, h, heads_q, s, false)) return rc;
        if (int rc = check_heads(ctx, dq, heads_q, s, true)) return rc;
        if (heads_k) {
            for (const edgc_heads* h : {k, dk_out})
                if (int rc = check_heads(ctx, h, heads_k, s, false)) return rc;
            if (int rc = check_heads(ctx, dk, heads_k, s, true)) return rc;
        }
        if (tokens > ctx->qk.tokens || dim > ctx->qk.dim || heads_q > ctx->qk.heads_q || heads_k > ctx->qk.heads_k)
            return fail(ctx, EDGC_EINVAL, "more tokens, heads or dimensions than edgc_reserve_qk_norm was called for");
    }
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    QkArgs a{};
    if (tokens) {
        a.h[0] = qk_heads(q, dq_out, dq, w_q, heads_q);
        a.h[1] = qk_heads(k, dk_out, dk, w_k, heads_k);
    }
    a.positions = positions; a.inv_freq = inv_freq; a.tokens = tokens; a.dim = dim; a.pairs = rot / 2; a.part = ctx->qk.part;
    a.interleaved = interleaved; a.pos_bytes = pos_bytes; a.eps = eps; a.inv_dim = 1.0f / static_cast<float>(dim);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return by_head(s, a, [&](auto type, auto n, auto u) -> int {
        using T = decltype(type);
        uint32_t blocks = 0;
        if (tokens) {
            // few tokens: queries and keys in blocks of their own (1001 tokens of 7 and 3 heads of 72: 5.8 us, with both in turn 9.2)
            const bool few = tokens <= qk_most_blocks(ctx) && heads_k;
            const uint64_t most = std::min<uint64_t>(tokens, qk_most_blocks(ctx) / (few ? 2 : 1));
            a.per = static_cast<uint32_t>((tokens + most - 1) / most);
            blocks = static_cast<uint32_t>((tokens + a.per - 1) / a.per);
            const uint32_t groups = 256 / a.lanes, lds = kQkTokens * a.pairs * static_cast<uint32_t>(sizeof(float2)) + groups * dim * 4u;
            const double bytes = 3.0 * sizeof(T) * tokens * (heads_q + heads_k) * dim;
            const int rc = by_size<n>(bytes, [&](auto stream) -> int {
                EDGC_LAUNCH(ctx, st, KID_QK_BACKWARD, bytes, 0.0, k_qk_norm<T, n, u, true, stream><<<dim3(blocks, 1, few ? 2 : 1), 256, lds, st>>>(a));
                EDGC_HIP_TRY(ctx, hipGetLastError());
                return EDGC_OK;
            });
            if (rc) return rc;
        }
        EDGC_LAUNCH(ctx, st, KID_QK_SUM, 8.0 * blocks * dim, 0.0,
                    k_qk_sum<T><<<dim3((dim + 31) / 32, dw_k ? 2 : 1), 32 * kQkWays, 0, st>>>(a.part, blocks, dim, dw_q, dw_k));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        return EDGC_OK;
    });
}
