// The embedding of tokens and its gradient.
//
//   forward   out[t] = scale table[ids[t] - first], zeros where that is no row of the table
//   backward  dtable[v] = scale sum of dy[t] over the tokens t with ids[t] - first = v
//
// Bounded by memory.  The backward pass sorts the tokens by row, so that a row's gradient is the sum of neighbours, in the tokens' order, and is written
// once: the same bits for the same tokens, whatever ran before.  k_embed_sort leaves the order and where each row's tokens begin in it, k_embed_sum adds up
// chunks of the order (a row whose tokens lie in several leaves a part in each) and writes the rows without a token, and k_embed_join adds up the parts.
#include "row_pack.h"

#include <algorithm>
#include <cmath>

namespace edgc {
namespace {

constexpr uint32_t kEmbedMaxVocab = 1u << 20, kEmbedMaxHidden = 1u << 20, kEmbedMaxTokens = 1u << 26;
constexpr int kEmbedUnroll = 4;                         // items of 16 bytes of a row that a lane has at a time
template <typename T> constexpr uint32_t kEmbedCols = 64u * kEmbedUnroll * Pack<T>::N;      // columns of a wave

struct EmbedArgs {
    const void* ids;
    int64_t first;
    uint64_t tokens;
    const void* table;                  // forward
    const void* dy;                     // backward
    void* out;                          // the tokens' rows, or the table's gradient
    uint64_t ld_in, ld_out;
    uint32_t vocab, hidden;
    float scale;
    int accumulate;
};

// A wave's number in a grid of blocks of four; a launch takes fewer than 2^32 threads along x
constexpr uint32_t kGridX = 1u << 20;
dim3 embed_grid(uint64_t waves)
{
    const uint64_t blocks = (waves + 3) / 4;
    return blocks <= kGridX ? dim3(static_cast<uint32_t>(blocks)) : dim3(kGridX, static_cast<uint32_t>((blocks + kGridX - 1) / kGridX));
}
__device__ __forceinline__ uint64_t embed_wave()
{
    return (static_cast<uint64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
}

// Row of a token's id, or one that is not there (2^32 - 1)
template <typename I>
__device__ __forceinline__ uint32_t embed_row(const EmbedArgs& a, uint64_t token)
{
    const uint64_t r = static_cast<uint64_t>(static_cast<int64_t>(static_cast<const I*>(a.ids)[token])) - static_cast<uint64_t>(a.first);
    return r < a.vocab ? static_cast<uint32_t>(r) : ~0u;
}

// A wave takes kEmbedCols columns of a token.  STREAM: what is written goes past the caches
template <typename T, typename I, bool STREAM>
__global__ __launch_bounds__(256) void k_embed_forward(const EmbedArgs a, uint32_t parts)
{
    constexpr int N = Pack<T>::N;
    const uint64_t unit = embed_wave();
    const uint64_t token = unit / parts;
    if (token >= a.tokens) return;
    const uint32_t c0 = static_cast<uint32_t>(unit - token * parts) * kEmbedCols<T> + threadIdx.x % 64 * N, row = embed_row<I>(a, token);
    const T* const src = static_cast<const T*>(a.table) + row * a.ld_in;
    T* const dst = static_cast<T*>(a.out) + token * a.ld_out;
    Pack<T> v[kEmbedUnroll];
    auto len = [&](int u) { const uint32_t c = c0 + u * 64 * N; return c < a.hidden ? min(static_cast<uint32_t>(N), a.hidden - c) : 0u; };
#pragma unroll
    for (int u = 0; u < kEmbedUnroll; ++u) {
        v[u].v = u32x4r{0, 0, 0, 0};
        if (row != ~0u) v[u].load(src + c0 + u * 64 * N, len(u));
    }
#pragma unroll
    for (int u = 0; u < kEmbedUnroll; ++u) {
        float f[N];
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = row != ~0u ? a.scale * v[u].get(i) : 0.f;
        Pack<T> o;
        o.set(f);
        o.template store<STREAM>(dst + c0 + u * 64 * N, len(u));
    }
}

// ---------------------------------------------------------------------------------------------
// The tokens in the order of their rows
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kSortBlocks = 256, kSortWaves = 16, kSortMaxKeys = 512,       // keys: 96 KB of LDS
                   kSortAhead = 16;             // tokens of a lane on their way at a time

// A block has `keys` neighbouring rows of the table and looks at all tokens twice: once to count those of its rows (and those of rows before them, which is
// where its own begin), once to put them in their places.  A wave has a run of the tokens; the places of a row's tokens in it follow those in the waves
// before it.
template <typename I>
__global__ __launch_bounds__(64 * kSortWaves) void k_embed_sort(const EmbedArgs a, uint32_t keys, uint32_t* order, uint32_t* starts)
{
    extern __shared__ uint32_t count[];                 // [kSortWaves][keys], then the first place of each; and as many sets of lanes
    __shared__ uint32_t s_below[kSortWaves], s_scan[kSortWaves];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid / 64, row0 = blockIdx.x * keys;
    const uint64_t per = ((a.tokens + kSortWaves - 1) / kSortWaves + 63) / 64 * 64, t0 = wave * per, t1 = min(a.tokens, t0 + per);
    for (uint32_t i = tid; i < 3 * kSortWaves * keys; i += 64 * kSortWaves) count[i] = 0;
    __syncthreads();
    uint32_t below = 0;
    uint32_t* const mine = count + wave * keys;
    uint32_t rows[kSortAhead];
    // rows of kSortAhead x 64 tokens, from t on
    auto look = [&](uint64_t t) {
#pragma unroll
        for (uint32_t i = 0; i < kSortAhead; ++i) rows[i] = t + i * 64 + lane < t1 ? embed_row<I>(a, t + i * 64 + lane) : ~0u;
    };
    for (uint64_t t = t0; t < t1; t += kSortAhead * 64) {
        look(t);
#pragma unroll
        for (uint32_t i = 0; i < kSortAhead; ++i) {
            below += rows[i] < row0 ? 1u : 0u;
            if (rows[i] != ~0u && rows[i] - row0 < keys) atomicAdd(mine + (rows[i] - row0), 1u);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) below += __shfl_xor(below, o, 64);
    if (lane == 0) s_below[wave] = below;
    __syncthreads();
    uint32_t base = 0;
    for (uint32_t w = 0; w < kSortWaves; ++w) base += s_below[w];
    // first places, a row at a time per thread
    for (uint32_t k0 = 0; k0 < keys; k0 += 64 * kSortWaves) {
        const uint32_t k = k0 + tid;
        uint32_t sum = 0;
        if (k < keys)
            for (uint32_t w = 0; w < kSortWaves; ++w) {
                const uint32_t c = count[w * keys + k];
                count[w * keys + k] = sum;
                sum += c;
            }
        uint32_t in = sum;                              // inclusive over the wave
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t v = __shfl_up(in, o, 64);
            if (lane >= static_cast<uint32_t>(o)) in += v;
        }
        if (lane == 63) s_scan[wave] = in;
        __syncthreads();
        uint32_t before = base, all = 0;
        for (uint32_t w = 0; w < kSortWaves; ++w) {
            if (w < wave) before += s_scan[w];
            all += s_scan[w];
        }
        const uint32_t at = before + in - sum;
        if (k < keys) {
            for (uint32_t w = 0; w < kSortWaves; ++w) count[w * keys + k] += at;
            if (row0 + k <= a.vocab) starts[row0 + k] = at;
        }
        base += all;
        __syncthreads();
    }
    if (tid == 0 && row0 + keys >= a.vocab && row0 < a.vocab) starts[a.vocab] = base;
    // Which lanes of a wave have a token of the same row they find in LDS, where each leaves its bit.  (Comparing the rows' bits one after the other, ballots of
    // the wave, took 18.7 us instead of 13.8 for 16384 tokens of 50000 words, the block with the
    // most frequent ones the longest.)
    auto wave_sync = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    uint32_t* const sets = count + kSortWaves * keys + wave * keys * 2;
    const uint64_t before = (1ull << lane) - 1;
    for (uint64_t t = t0; t < t1; t += kSortAhead * 64) {
        if (t1 - t0 > kSortAhead * 64) look(t);         // (else they are there still)
#pragma unroll
        for (uint32_t i = 0; i < kSortAhead; ++i) {
            const uint32_t k = rows[i] - row0;
            const bool ours = rows[i] != ~0u && k < keys;
            if (__ballot(ours) == 0) continue;
            if (ours) atomicOr(sets + 2 * k + lane / 32, 1u << (lane & 31));
            wave_sync();
            uint64_t same = 0;
            uint32_t at = 0;
            if (ours) {
                same = sets[2 * k] | static_cast<uint64_t>(sets[2 * k + 1]) << 32;
                at = mine[k];
            }
            wave_sync();
            if (ours) {
                order[at + __popcll(same & before)] = static_cast<uint32_t>(t + i * 64 + lane);
                if ((same & before) == 0) {
                    mine[k] = at + static_cast<uint32_t>(__popcll(same));
                    sets[2 * k] = sets[2 * k + 1] = 0;
                }
            }
            wave_sync();
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Their sums, past the caches (4096 columns of bf16 with the list's norm behind them: 2000 rows 29.2 us, through the caches 30.5; 8000 76.8 and 75.5; 32000
// 201 and 254)
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kEmbedChunk = 32, kSumAhead = 8;     // tokens of a wave at most; on their way at a time
constexpr uint32_t kZeroRows = 8;                       // rows that a wave looks for tokens of
enum { kPartHead = 0, kPartTail = 1 };                  // of a row begun in an earlier chunk; of one that goes on in the next

template <typename T>
__device__ __forceinline__ void embed_write(const EmbedArgs& a, uint32_t row, uint32_t c, uint32_t len, const float (&sum)[Pack<T>::N])
{
    constexpr int N = Pack<T>::N;
    T* const to = static_cast<T*>(a.out) + row * a.ld_out + c;
    float f[N];
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = a.scale * sum[i];
    Pack<T> o;
    if (a.accumulate) {
        o.load(to, len);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] += o.get(i);
    }
    o.set(f);
    o.template store<true>(to, len);
}
// A wave's share of a part: rows of `hidden` padded to the columns of whole waves, so that it is stored and loaded whole
__host__ __device__ inline uint64_t embed_part_ld(uint32_t hidden) { return (static_cast<uint64_t>(hidden) + 511) / 512 * 512; }
template <int N>
__device__ __forceinline__ float4* embed_part(float* part, uint32_t hidden, uint32_t chunk, int which, uint32_t c)
{
    return reinterpret_cast<float4*>(part + (static_cast<uint64_t>(chunk) * 2 + which) * embed_part_ld(hidden) + c);
}

struct EmbedWork {
    const uint32_t *order, *starts;     // starts null: no tokens
    float* part;
    uint32_t chunk, chunks, zeros, parts;       // tokens of a wave; those of the order, groups of rows that may be without tokens, both; waves of a row
};

// A wave adds up a chunk of the order, 64 items of 16 bytes of each, or writes zeros to those of a group of rows that have no token.  Chunks and groups take
// turns, so that reading and writing go on at the same time.
template <typename T, typename I>
__global__ __launch_bounds__(256) void k_embed_sum(const EmbedArgs a, const EmbedWork w)
{
    constexpr int N = Pack<T>::N;
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t unit = embed_wave();
    const uint32_t total = w.chunks + w.zeros;
    if (unit >= static_cast<uint64_t>(total) * w.parts) return;
    const uint32_t which = static_cast<uint32_t>(unit / w.parts);
    const uint32_t c = static_cast<uint32_t>(unit - static_cast<uint64_t>(which) * w.parts) * (64 * N) + lane * N;
    const uint32_t len = c < a.hidden ? min(static_cast<uint32_t>(N), a.hidden - c) : 0u;
    const uint32_t every = w.chunks ? total / w.chunks : 0u, turn = every ? which / every : 0u;
    if (!every || which % every || turn >= w.chunks) {
        const uint32_t r0 = (which - (every ? min(w.chunks, turn + 1) : 0u)) * kZeroRows, r = r0 + lane;
        uint64_t empty = __ballot(lane < kZeroRows && r < a.vocab && (!w.starts || w.starts[r] == w.starts[r + 1]));
        const float none[N] = {};
        for (; empty; empty &= empty - 1) embed_write<T>(a, r0 + __builtin_ctzll(empty), c, len, none);
        return;
    }
    // lane l: token l - 1 of the chunk, so that the neighbours on both sides are there
    const uint32_t all = w.starts[a.vocab], p0 = turn * w.chunk;
    if (p0 >= all) return;
    const uint32_t n = min(all - p0, w.chunk);
    static_assert(kEmbedChunk + 2 <= 64, "");
    const bool there = lane <= n + 1 && p0 + lane > 0 && p0 + lane - 1 < all;
    const uint32_t token = there ? w.order[p0 + lane - 1] : 0u, row = there ? embed_row<I>(a, token) : ~0u;
    auto row_of = [&](uint32_t k) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(row, k)); };       // (lanes)
    float sum[N] = {};
    bool open = row_of(0) == row_of(1);                 // begun in an earlier chunk
    for (uint32_t k0 = 1; k0 <= n; k0 += kSumAhead) {
        Pack<T> v[kSumAhead];
#pragma unroll
        for (uint32_t k = 0; k < kSumAhead; ++k)
            if (k0 + k <= n) v[k].load(static_cast<const T*>(a.dy) + static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(token, k0 + k))) * a.ld_in + c, len);
#pragma unroll
        for (uint32_t k = 0; k < kSumAhead; ++k) {
            if (k0 + k > n) break;
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] += v[k].get(i);
            const uint32_t mine = row_of(k0 + k);
            const bool more = row_of(k0 + k + 1) == mine;
            if (more && k0 + k < n) continue;
            if (!open && !more) {
                embed_write<T>(a, mine, c, len, sum);
            } else {
                float4* const to = embed_part<N>(w.part, a.hidden, turn, open ? kPartHead : kPartTail, c);
#pragma unroll
                for (int i = 0; i < N / 4; ++i) to[i] = float4{sum[4 * i], sum[4 * i + 1], sum[4 * i + 2], sum[4 * i + 3]};
            }
            open = false;
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = 0.f;
        }
    }
}

// Adds up the parts of a row that begins in a chunk and goes on in the next: a wave for every chunk and 64 items of 16 bytes
template <typename T, typename I>
__global__ __launch_bounds__(64) void k_embed_join(const EmbedArgs a, const EmbedWork w)
{
    constexpr int N = Pack<T>::N;
    const uint32_t k = blockIdx.x, all = w.starts[a.vocab], p1 = (k + 1) * w.chunk;
    if (p1 >= all) return;                              // the last one, or none
    const uint32_t row = embed_row<I>(a, w.order[p1 - 1]), s0 = w.starts[row], s1 = w.starts[row + 1];
    if (s0 < k * w.chunk || s1 <= p1) return;
    const uint32_t c = blockIdx.y * (64 * N) + threadIdx.x * N, len = c < a.hidden ? min(static_cast<uint32_t>(N), a.hidden - c) : 0u;
    float sum[N] = {};
    auto add = [&](uint32_t at, int which) {
        const float4* const from = embed_part<N>(w.part, a.hidden, at, which, c);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 v = from[i];
            sum[4 * i] += v.x; sum[4 * i + 1] += v.y; sum[4 * i + 2] += v.z; sum[4 * i + 3] += v.w;
        }
    };
    add(k, kPartTail);
    const uint32_t last = (s1 - 1) / w.chunk;
#pragma unroll 8
    for (uint32_t j = k + 1; j <= last; ++j) add(j, kPartHead);
    embed_write<T>(a, row, c, len, sum);
}

// Tokens of a wave: 32, or fewer where that leaves compute units with less than eight waves (2999 tokens of 1001 fp32 columns, 32 / 8: 16.4 / 4.8 us).
constexpr uint64_t kEmbedWaves = 2048;
uint32_t embed_chunk(uint64_t tokens, uint32_t parts)
{
    uint32_t chunk = kEmbedChunk;
    while (chunk > 8 && (tokens + chunk - 1) / chunk * parts < kEmbedWaves) chunk /= 2;
    return chunk;
}
uint64_t pad256(uint64_t bytes) { return (bytes + 255) / 256 * 256; }
struct EmbedPlan {
    uint64_t order, starts, part, bytes;        // where each begins
    EmbedPlan(uint64_t tokens, uint64_t vocab, uint64_t hidden)
    {
        order = 0;
        starts = pad256(tokens * 4);
        part = starts + pad256((vocab + 1) * 4);
        // chunks of 32, or shorter ones: fewer than 2 kEmbedWaves and a row's waves, each of 512 columns at most (fp32: 256, padded)
        const uint64_t ld = embed_part_ld(static_cast<uint32_t>(hidden));
        bytes = part + 8 * std::max((tokens + kEmbedChunk - 1) / kEmbedChunk * ld, (2 * kEmbedWaves + 4096) * 512 + ld);
    }
};

int check_embed(edgc_ctx* ctx, edgc_dtype dtype, const void* ids, int id_bytes, int64_t first, uint64_t tokens, uint32_t vocab, uint32_t hidden, float scale)
{
    if (dtype != EDGC_F32 && dtype != EDGC_BF16) return fail(ctx, EDGC_EINVAL, "unknown dtype");
    if (id_bytes != 4 && id_bytes != 8) return fail(ctx, EDGC_EINVAL, "ids have 4 or 8 bytes");
    if (vocab == 0 || hidden == 0 || vocab > kEmbedMaxVocab || hidden > kEmbedMaxHidden) return fail(ctx, EDGC_EINVAL, "vocab and hidden must be 1 to 2^20");
    if (tokens > kEmbedMaxTokens) return fail(ctx, EDGC_EINVAL, "more than 2^26 tokens");
    if (first > (1ll << 62) || first < -(1ll << 62)) return fail(ctx, EDGC_EINVAL, "first_id beyond 2^62");
    if (!std::isfinite(scale)) return fail(ctx, EDGC_EINVAL, "scale must be finite");
    if (tokens && (!ids || !aligned_to(ids, static_cast<size_t>(id_bytes)))) return fail(ctx, EDGC_EINVAL, "null or misaligned ids");
    return EDGC_OK;
}
int check_embed_rows(edgc_ctx* ctx, edgc_dtype dtype, const void* p, uint64_t ld, uint32_t hidden)
{
    if (!p || !aligned_to(p, dtype == EDGC_F32 ? 4 : 2)) return fail(ctx, EDGC_EINVAL, "null or misaligned pointer");
    if (ld < hidden || ld > kMaxSpan) return fail(ctx, EDGC_EINVAL, "leading dimension too small, or over 2^40");
    return EDGC_OK;
}

}  // namespace

int prepare_embed_kernels(edgc_ctx* ctx)
{
    for (const void* f : {reinterpret_cast<const void*>(&k_embed_sort<int32_t>), reinterpret_cast<const void*>(&k_embed_sort<int64_t>)})
        EDGC_HIP_TRY(ctx, hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, kSortWaves * kSortMaxKeys * 12));
    return EDGC_OK;
}

void free_embed(edgc_ctx* ctx)
{
    if (ctx->embed.ws) (void)hipFree(ctx->embed.ws);
    ctx->embed = EmbedScratch{};
}

}  // namespace edgc

using namespace edgc;

extern "C" int edgc_embed_forward(edgc_ctx* ctx, edgc_dtype dtype, const void* table, uint64_t ld_table, uint32_t vocab, uint32_t hidden, const void* ids,
                                  int id_bytes, int64_t first_id, uint64_t tokens, float scale, void* out, uint64_t ld_out, void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    if (int rc = check_embed(ctx, dtype, ids, id_bytes, first_id, tokens, vocab, hidden, scale)) return rc;
    if (tokens == 0) return EDGC_OK;
    if (int rc = check_embed_rows(ctx, dtype, table, ld_table, hidden)) return rc;
    if (int rc = check_embed_rows(ctx, dtype, out, ld_out, hidden)) return rc;
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    EmbedArgs a{};
    a.ids = ids; a.first = first_id; a.tokens = tokens; a.table = table; a.out = out; a.ld_in = ld_table; a.ld_out = ld_out;
    a.vocab = vocab; a.hidden = hidden; a.scale = scale;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    // What the next operator can still find in the caches stays there: rows of 4096 bf16 and the norm of them take 48 us for 8192 tokens (past the caches 53), for
    // 16384, 2^27 bytes, 103 (110), for 32768 220 (215).
    auto launch = [&](auto type, auto id, auto stream) -> int {
        using T = decltype(type);
        const uint32_t parts = (hidden + kEmbedCols<T> - 1) / kEmbedCols<T>;
        EDGC_LAUNCH(ctx, st, KID_EMBED_FORWARD, 2.0 * sizeof(T) * tokens * hidden, 0.0,
                    k_embed_forward<T, decltype(id), stream><<<embed_grid(tokens * parts), 256, 0, st>>>(a, parts));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        return EDGC_OK;
    };
    auto go = [&](auto type, auto id) -> int {
        return static_cast<double>(sizeof(type)) * tokens * hidden > 134217728.0 ? launch(type, id, std::true_type{}) : launch(type, id, std::false_type{});
    };
    if (dtype == EDGC_F32) return id_bytes == 8 ? go(float{}, int64_t{}) : go(float{}, int32_t{});
    return id_bytes == 8 ? go(__bf16{}, int64_t{}) : go(__bf16{}, int32_t{});
}

extern "C" int edgc_reserve_embed(edgc_ctx* ctx, uint32_t tokens, uint32_t vocab, uint32_t hidden)
{
    if (!ctx) return EDGC_EINVAL;
    if (vocab == 0 || hidden == 0 || vocab > kEmbedMaxVocab || hidden > kEmbedMaxHidden || tokens > kEmbedMaxTokens)
        return fail(ctx, EDGC_EINVAL, "vocab and hidden must be 1 to 2^20, tokens at most 2^26");
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    const uint64_t need = tokens ? EmbedPlan(tokens, vocab, hidden).bytes : 0;
    if (need && need <= ctx->embed.held) {
        ctx->embed.bytes = need;
        return EDGC_OK;
    }
    EDGC_HIP_TRY(ctx, hipDeviceSynchronize());          // nothing may still be using the old scratch
    free_embed(ctx);
    if (need == 0) return EDGC_OK;
    if (hipMalloc(&ctx->embed.ws, need) != hipSuccess) {
        (void)hipGetLastError();
        ctx->embed = EmbedScratch{};
        return fail(ctx, EDGC_ENOMEM, "embedding scratch allocation failed");
    }
    ctx->embed.bytes = ctx->embed.held = need;
    return EDGC_OK;
}

extern "C" int edgc_embed_backward(edgc_ctx* ctx, edgc_dtype dtype, const void* ids, int id_bytes, int64_t first_id, uint64_t tokens, const void* dy,
                                   uint64_t ld_dy, uint32_t vocab, uint32_t hidden, float scale, void* dtable, uint64_t ld_dtable, int accumulate,
                                   void* hip_stream)
{
    if (!ctx) return EDGC_EINVAL;
    if (int rc = check_embed(ctx, dtype, ids, id_bytes, first_id, tokens, vocab, hidden, scale)) return rc;
    if (int rc = check_embed_rows(ctx, dtype, dtable, ld_dtable, hidden)) return rc;
    if (tokens)
        if (int rc = check_embed_rows(ctx, dtype, dy, ld_dy, hidden)) return rc;
    if (tokens == 0 && accumulate) return EDGC_OK;
    const EmbedPlan plan(tokens, vocab, hidden);
    if (tokens && plan.bytes > ctx->embed.bytes) return fail(ctx, EDGC_EINVAL, "larger than what edgc_reserve_embed was called for");
    EDGC_HIP_TRY(ctx, hipSetDevice(ctx->device));
    EmbedArgs a{};
    a.ids = ids; a.first = first_id; a.tokens = tokens; a.dy = dy; a.out = dtable; a.ld_in = ld_dy; a.ld_out = ld_dtable;
    a.vocab = vocab; a.hidden = hidden; a.scale = scale; a.accumulate = accumulate;
    unsigned char* const ws = static_cast<unsigned char*>(ctx->embed.ws);
    uint32_t *const order = reinterpret_cast<uint32_t*>(ws + plan.order), *const starts = reinterpret_cast<uint32_t*>(ws + plan.starts);
    float* const part = reinterpret_cast<float*>(ws + plan.part);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto go = [&](auto type, auto id) -> int {
        using T = decltype(type);
        using I = decltype(id);
        const uint32_t keys = std::min((vocab + kSortBlocks - 1) / kSortBlocks, kSortMaxKeys), sorts = (vocab + keys - 1) / keys;
        if (tokens)
            EDGC_LAUNCH(ctx, st, KID_EMBED_SORT, 2.0 * sizeof(I) * tokens * sorts, 0.0,
                    k_embed_sort<I><<<sorts, 64 * kSortWaves, kSortWaves * keys * 12, st>>>(a, keys, order, starts));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        const uint32_t cols = 64 * Pack<T>::N;
        const uint32_t parts = (hidden + cols - 1) / cols, chunk = embed_chunk(tokens, parts);
        EmbedWork w{order, tokens ? starts : nullptr, part, chunk, static_cast<uint32_t>((tokens + chunk - 1) / chunk),
                    accumulate ? 0u : (vocab + kZeroRows - 1) / kZeroRows, parts};
        EDGC_LAUNCH(ctx, st, KID_EMBED_SUM, static_cast<double>(sizeof(T)) * hidden * (static_cast<double>(tokens) + vocab), 0.0,
                    k_embed_sum<T, I><<<embed_grid((static_cast<uint64_t>(w.chunks) + w.zeros) * w.parts), 256, 0, st>>>(a, w));
        EDGC_HIP_TRY(ctx, hipGetLastError());
        if (w.chunks > 1) {
            EDGC_LAUNCH(ctx, st, KID_EMBED_JOIN, 0.0, 0.0, k_embed_join<T, I><<<dim3(w.chunks - 1, w.parts), 64, 0, st>>>(a, w));
            EDGC_HIP_TRY(ctx, hipGetLastError());
        }
        return EDGC_OK;
    };
    if (dtype == EDGC_F32) return id_bytes == 8 ? go(float{}, int64_t{}) : go(float{}, int32_t{});
    return id_bytes == 8 ? go(__bf16{}, int64_t{}) : go(__bf16{}, int32_t{});
}
