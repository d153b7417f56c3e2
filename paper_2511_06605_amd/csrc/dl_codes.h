// Element types and 8-bit codes of the operators over a quantised cache, and what their kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/dmalatte.h"

// 16 (8, 4) bytes at any address: gfx950 loads and stores whole vectors there.
typedef uint32_t dl_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t dl_u32x2 __attribute__((ext_vector_type(2)));
typedef float dl_f32x4 __attribute__((ext_vector_type(4)));
typedef float dl_f32x16 __attribute__((ext_vector_type(16)));
typedef float dl_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 dl_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 dl_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 dl_f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 dl_f16x8 __attribute__((ext_vector_type(8)));

template <class T>
struct __attribute__((packed, aligned(1))) dl_anywhere {
    T v;
};
template <class T>
__device__ __forceinline__ T dl_load_at(const void *p)
{
    return ((const dl_anywhere<T> *)p)->v;
}
template <class T>
__device__ __forceinline__ void dl_store_at(void *p, T v)
{
    ((dl_anywhere<T> *)p)->v = v;
}

template <class To, class From>
__device__ __forceinline__ To dl_bits(From f)
{
    static_assert(sizeof(To) == sizeof(From), "same bits");
    return __builtin_bit_cast(To, f);
}

// Division of whole numbers n < 2^31 by d in 1 .. 2^17: n * m >> sh with sh = 31 + l, 2^l the power of two at or above d, and
// m = 2^sh / d rounded up (< 2^32).  Exact: m d = 2^sh + e with e < d, so n m / 2^sh is n / d and less than n d / (d 2^sh) <= 1 / d more.
struct dl_divider {
    uint32_t d, m, sh;
};
static inline dl_divider dl_make_divider(uint32_t d)
{
    uint32_t l = 0;
    while ((1u << l) < d) ++l;  // d <= 2^17
    const uint64_t two = 1ull << (31 + l);
    return {d, (uint32_t)((two + d - 1) / d), 31 + l};
}
__device__ __forceinline__ uint32_t dl_divide(uint32_t n, const dl_divider &v)
{
    return (uint32_t)((uint64_t)n * v.m >> v.sh);
}

// ------------------------------------------------------------------ element types

struct dl_f32 {
    static constexpr int size = 4;
};
struct dl_bf16 {
    static constexpr int size = 2;
    // Weights relative to a reference, at most 2^8, are held as 2^lift times as much.  Floats of 16 bits lose bits below 2^-14,
    // so there they use the range above as well: what is 2^-21 of the reference still has all of its bits.
    static constexpr float lift = 0.0f;
    // Scales of values from twice this one on are taken apart (dl_value_scale below), and a product with what that leaves over
    // is brought into the type's range.
    static constexpr float scale_most = 0x1p40f;
    static __device__ __forceinline__ float in_range(float w) { return w; }
    static __device__ __forceinline__ float lo(uint32_t w) { return dl_bits<float>(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return dl_bits<float>(w & 0xFFFF0000u); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return dl_bits<uint32_t>(dl_bf16x2{(__bf16)a, (__bf16)b}); }
    static __device__ __forceinline__ float one(uint16_t v) { return dl_bits<float>((uint32_t)v << 16); }
    static __device__ __forceinline__ dl_f32x4 mfma16(dl_u32x4 a, dl_u32x4 b, dl_f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(dl_bits<dl_bf16x8>(a), dl_bits<dl_bf16x8>(b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ dl_f32x16 mfma32(dl_u32x4 a, dl_u32x4 b, dl_f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(dl_bits<dl_bf16x8>(a), dl_bits<dl_bf16x8>(b), c, 0, 0, 0);
    }
};
struct dl_f16 {
    static constexpr int size = 2;
    static constexpr float lift = 7.0f;
    // (Such products may saturate, in rows with values above 448 x 2^50 = 5e17; an output of this type is finite only where such a row's
    // weight is less than 2^-40 of the others'.)
    static constexpr float scale_most = 0x1p50f;
    static __device__ __forceinline__ float in_range(float w) { return fminf(fmaxf(w, -65504.0f), 65504.0f); }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)dl_bits<dl_f16x2>(w)[0]; }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)dl_bits<dl_f16x2>(w)[1]; }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return dl_bits<uint32_t>(dl_f16x2{(_Float16)a, (_Float16)b}); }
    static __device__ __forceinline__ float one(uint16_t v) { return (float)dl_bits<_Float16>(v); }
    static __device__ __forceinline__ dl_f32x4 mfma16(dl_u32x4 a, dl_u32x4 b, dl_f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(dl_bits<dl_f16x8>(a), dl_bits<dl_f16x8>(b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ dl_f32x16 mfma32(dl_u32x4 a, dl_u32x4 b, dl_f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(dl_bits<dl_f16x8>(a), dl_bits<dl_f16x8>(b), c, 0, 0, 0);
    }
};

// ------------------------------------------------------------------ codes

struct dl_fp8 {
    static constexpr float limit = 448.0f;
    // four floats, |x| <= 448 (1 + 2^-22), to codes: rounded to nearest, ties to even
    static __device__ __forceinline__ uint32_t code4(float a, float b, float c, float d)
    {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
        return (uint32_t)w;
    }
    static __device__ __forceinline__ void value4(uint32_t w, float (&x)[4])
    {
        const dl_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
    }
    // four codes to four elements of Q: every code is a value of both types
    template <class Q>
    static __device__ __forceinline__ dl_u32x2 spread(uint32_t w)
    {
        if constexpr (std::is_same<Q, dl_bf16>::value)
            return {dl_bits<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false)),
                    dl_bits<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true))};
        else
            return {dl_bits<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false)),
                    dl_bits<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true))};
    }
};
struct dl_int8 {
    static constexpr float limit = 127.0f;
    static __device__ __forceinline__ uint32_t code4(float a, float b, float c, float d)
    {
        // 1.5 * 2^23 + x is x rounded to a whole number, ties to even, in the low bits (the sums are kept apart from the products
        // that x comes from: one rounding each)
        asm("" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
        const uint32_t p = dl_bits<uint32_t>(a + 12582912.0f), q = dl_bits<uint32_t>(b + 12582912.0f);
        const uint32_t r = dl_bits<uint32_t>(c + 12582912.0f), s = dl_bits<uint32_t>(d + 12582912.0f);
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(s, r, 0x0C0C0400u), __builtin_amdgcn_perm(q, p, 0x0C0C0400u), 0x05040100u);
    }
    static __device__ __forceinline__ void value4(uint32_t w, float (&x)[4])
    {
        x[0] = (float)(int8_t)w, x[1] = (float)(int8_t)(w >> 8), x[2] = (float)(int8_t)(w >> 16), x[3] = (float)((int32_t)w >> 24);
    }
    template <class Q>
    static __device__ __forceinline__ dl_u32x2 spread(uint32_t w)
    {
        if constexpr (std::is_same<Q, dl_bf16>::value) {
            float x[4];
            value4(w, x);
            return {dl_bf16::pack(x[0], x[1]), dl_bf16::pack(x[2], x[3])};
        } else {
            // 1024 + u is 0x6400 | u for u < 1024: two bytes behind 0x64 each, then 1024 + 128 taken off again
            const uint32_t u = w ^ 0x80808080u;
            const uint32_t a = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u), b = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
            const dl_f16x2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
            return {dl_bits<uint32_t>(dl_bits<dl_f16x2>(a) - off), dl_bits<uint32_t>(dl_bits<dl_f16x2>(b) - off)};
        }
    }
};

// ------------------------------------------------------------------ what the kernels share

// x + the lanes before it; lane 63 ends with the sum of all.
__device__ __forceinline__ uint32_t dl_sum_up_to(uint32_t x)
{
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);  // row_shr:1, 2, 4, 8
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);  // row_bcast:15, 31
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);
    return x;
}

// The largest over a wavefront.
__device__ __forceinline__ uint32_t dl_largest(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false));  // row_shr:1, 2, 4, 8
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false));  // row_bcast:15, 31
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// N elements of a row as floats
template <class T, int N>
__device__ __forceinline__ void dl_load_row(const char *p, float (&x)[N])
{
    if constexpr (T::size == 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const dl_f32x4 w = dl_load_at<dl_f32x4>(p + 16 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = w[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const dl_u32x4 w = dl_load_at<dl_u32x4>(p + 16 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[8 * i + 2 * j] = T::lo(w[j]), x[8 * i + 2 * j + 1] = T::hi(w[j]);
        }
    }
}

// STREAM: past the caches
template <bool STREAM, class V>
__device__ __forceinline__ void dl_put(char *p, V v)
{
    typedef V anywhere __attribute__((aligned(1)));
    if constexpr (STREAM)
        __builtin_nontemporal_store(v, (anywhere *)p);
    else
        dl_store_at(p, v);
}

template <class T, bool STREAM, int N>
__device__ __forceinline__ void dl_store_row(char *p, const float (&x)[N])
{
    if constexpr (T::size == 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) dl_put<STREAM>(p + 16 * i, dl_f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]});
    } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            dl_u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = T::pack(x[8 * i + 2 * j], x[8 * i + 2 * j + 1]);
            dl_put<STREAM>(p + 16 * i, w);
        }
    }
}

// A vector of N bytes, N = 4, 8, 16, as words
template <int N>
struct dl_words {
    uint32_t w[N / 4];
};
template <int N>
__device__ __forceinline__ dl_words<N> dl_load_words(const char *p)
{
    return dl_load_at<dl_words<N>>(p);
}
// A value's scale u = c d for the sums, d a power of two.  c: what log2 u and 1 / u are taken of, so that neither they nor a product with
// 2^(log2 u) or 1 / u leave the range of 32 bits, however far apart the scales of the rows are that a query sees.  d: 1, or what that
// leaves out; it goes to the product with the values alone (never to l), and is finite, so that a weight of zero takes it out.
// Scales below 2^-126 (dl_kv_write gives 2^-100 / 448 and more) count as zero, and so do negative ones.  A NaN stays in c.
template <class Q>
struct dl_value_scale {
    float c, d;
    __device__ __forceinline__ explicit dl_value_scale(float u)
    {
        constexpr float LOW = 0x1p-40f, HIGH = Q::scale_most;
        // u's power of two (none for what is no positive number, infinite for infinities), and what it is more than the limit's
        const float power = dl_bits<float>(dl_bits<uint32_t>(fmaxf(u, 0.0f)) & 0x7F800000u);
        const bool low = u < LOW, high = u >= 2.0f * HIGH;
        d = low ? power * (1.0f / LOW) : high ? fminf(power, 0x1p127f) * (1.0f / HIGH) : 1.0f;
        // (the mantissa of u with the limit's power)
        const float c_limit = dl_bits<float>((dl_bits<uint32_t>(u) & 0x007FFFFFu) | dl_bits<uint32_t>(low ? LOW : HIGH));
        c = low || high ? c_limit : u;
    }
    __device__ __forceinline__ float log2_c() const { return __builtin_amdgcn_logf(c); }
    // (finite for a NaN as well: its readers' weights have it from the logarithm)
    __device__ __forceinline__ float over_c() const { return __builtin_amdgcn_rcpf(c == c ? c : 1.0f); }
};

template <class F>
static inline void dl_with_bool(bool b, F f)
{
    if (b)
        f(std::true_type{});
    else
        f(std::false_type{});
}

// Calls f with the types that belong to a dl_kv_format / to a 16-bit dl_type.
template <class F>
static inline void dl_with_format(int32_t format, F f)
{
    if (format == DL_KV_FP8)
        f(dl_fp8{});
    else
        f(dl_int8{});
}
template <class F>
static inline void dl_with_16bit(int32_t type, F f)
{
    if (type == DL_TYPE_BF16)
        f(dl_bf16{});
    else
        f(dl_f16{});
}
template <class F>
static inline void dl_with_type(int32_t type, F f)
{
    if (type == DL_TYPE_F32)
        f(dl_f32{});
    else
        dl_with_16bit(type, f);
}

// The lanes that a row takes, a power of two.
template <int N, class F>
static inline void dl_with_lanes(uint32_t head_dim, F f)
{
    if (head_dim <= 16)
        f(std::integral_constant<int, 16 / N>{});
    else if (head_dim <= 32)
        f(std::integral_constant<int, 32 / N>{});
    else if (head_dim <= 64)
        f(std::integral_constant<int, 64 / N>{});
    else if (head_dim <= 128)
        f(std::integral_constant<int, 128 / N>{});
    else
        f(std::integral_constant<int, 256 / N>{});
}

// The cache as the kernels get it.
struct dl_cache_view {
    char *k, *v;
    float *k_scale, *v_scale;
    int64_t head_stride, scale_head_stride;                                          // bytes, all of them
    uint32_t page_stride, token_stride, scale_page_stride, scale_token_stride;
    uint32_t pages, heads, head_dim;
    dl_divider page;
};
// dl_kv.hip: what is wrong with a cache, or its view (sides: 1 keys, 2 values, those that must be there).
int dl_cache_check(const dl_kv_cache *c, int sides, dl_cache_view *view);

constexpr size_t DL_CONTROL_BYTES = 65536;  // the front of a workspace: counters, zero between calls
