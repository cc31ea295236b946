// 16 bytes of a row in registers: what the operators that are bounded by memory load and store.
#pragma once

#include "edgc_internal.h"

namespace edgc {

typedef float f32x4_at __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_at __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4r __attribute__((ext_vector_type(4)));

// STREAM: what is not read again soon, and need not stay in the caches
template <bool STREAM, typename V>
__device__ __forceinline__ V pack_read(const void* p)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const V*>(p));
    else return *static_cast<const V*>(p);
}
template <bool STREAM, typename V>
__device__ __forceinline__ void pack_write(void* p, V v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<V*>(p));
    else *static_cast<V*>(p) = v;
}

// 16 bytes of a row in registers, as they stand in memory
template <typename T> struct Pack;
template <> struct Pack<float> {
    static constexpr int N = 4;
    u32x4r v;
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(v[i]); }
    __device__ __forceinline__ void set(const float (&f)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __float_as_uint(f[i]);
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void load(const float* p, uint32_t len)
    {
        if (len == N) {
            const f32x4_at x = pack_read<STREAM, f32x4_at>(p);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = __float_as_uint(x[i]);
            return;
        }
        v = u32x4r{0, 0, 0, 0};
        for (int i = 0; i < N; ++i)
            if (static_cast<uint32_t>(i) < len) v[i] = __float_as_uint(p[i]);
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void store(float* p, uint32_t len) const
    {
        if (len == N) {
            f32x4_at x;
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = __uint_as_float(v[i]);
            pack_write<STREAM>(p, x);
            return;
        }
        for (int i = 0; i < N; ++i)
            if (static_cast<uint32_t>(i) < len) p[i] = __uint_as_float(v[i]);
    }
};
template <> struct Pack<__bf16> {
    static constexpr int N = 8;
    u32x4r v;
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16); }
    __device__ __forceinline__ void set(const float (&f)[N])
    {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{f[2 * i], f[2 * i + 1]}), b2));
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void load(const __bf16* p, uint32_t len)
    {
        if (len == N) {
            const u32x4_at x = pack_read<STREAM, u32x4_at>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = x[i];
            return;
        }
        v = u32x4r{0, 0, 0, 0};
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
        for (int i = 0; i < N; ++i)
            if (static_cast<uint32_t>(i) < len) v[i / 2] |= static_cast<uint32_t>(q[i]) << (16 * (i & 1));
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void store(__bf16* p, uint32_t len) const
    {
        if (len == N) {
            u32x4_at x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = v[i];
            pack_write<STREAM>(p, x);
            return;
        }
        uint16_t* q = reinterpret_cast<uint16_t*>(p);
        for (int i = 0; i < N; ++i)
            if (static_cast<uint32_t>(i) < len) q[i] = static_cast<uint16_t>(v[i / 2] >> (16 * (i & 1)));
    }
};

}  // namespace edgc
