// vp_fp8_device.h -- device helpers of the 8-bit operators' kernels: loads and
// stores of eight elements, the block exponent, 16-lane reductions.
#pragma once

#include <cstdint>
#include <type_traits>

#include <hip/hip_runtime.h>

#include "vp_fp8.h"

namespace vp {

using bf16_t = __bf16;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Memory operations of 16 bytes need no more than their element's alignment
// here, so rows of any width and distance take the same path.
typedef f32x4 __attribute__((aligned(4))) f32x4_any;
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef bf16x8 __attribute__((aligned(2))) bf16x8_any;

// Eight elements as they lie in memory, of which `left` lie inside the row (the
// others read as zero and are not touched).  Widened by widen8 afterwards, so
// that several loads can be under way; load8s puts those of several matrices
// into one branch, whose short side would wait for each of them otherwise.
template <class T>
struct Raw8;
template <>
struct Raw8<float> {
    f32x4 a, b;
};
template <>
struct Raw8<bf16_t> {
    bf16x8 a;
};
// FAR: the launch reads or writes more than the memory-side cache keeps, so its
// lines are not kept for anyone (nontemporal).  bf16 alone: eight floats are two
// pieces of 16 bytes a lane, half a line of every second lane's each, and past
// the cache a half line costs a whole one.
template <bool FAR>
__device__ __forceinline__ void load_whole(const float* p, Raw8<float>& r) {
    static_assert(!FAR);
    r.a = *reinterpret_cast<const f32x4_any*>(p);
    r.b = *reinterpret_cast<const f32x4_any*>(p + 4);
}
template <bool FAR>
__device__ __forceinline__ void load_whole(const bf16_t* p, Raw8<bf16_t>& r) {
    if constexpr (FAR)
        r.a = __builtin_bit_cast(bf16x8, __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p)));
    else
        r.a = *reinterpret_cast<const bf16x8_any*>(p);
}
__device__ __forceinline__ void load_part(const float* p, int64_t left, Raw8<float>& r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.a[i] = i < left ? p[i] : 0.0f;
        r.b[i] = 4 + i < left ? p[4 + i] : 0.0f;
    }
}
__device__ __forceinline__ void load_part(const bf16_t* p, int64_t left, Raw8<bf16_t>& r) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.a[i] = i < left ? p[i] : static_cast<bf16_t>(0.0f);
}
__device__ __forceinline__ void widen8(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = r.a[i];
        v[4 + i] = r.b[i];
    }
}
__device__ __forceinline__ void widen8(const Raw8<bf16_t>& r, float (&v)[8]) {
    const u32x4 a = __builtin_bit_cast(u32x4, r.a);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
}
template <bool FAR, class T, class... R>
__device__ __forceinline__ void load8s(int64_t left, const T* p, Raw8<T>& r, R&&... more) {
    auto whole = [&](auto&& self, const T* q, Raw8<T>& x, auto&&... rest) {
        load_whole<FAR>(q, x);
        if constexpr (sizeof...(rest) > 0) self(self, rest...);
    };
    auto part = [&](auto&& self, const T* q, Raw8<T>& x, auto&&... rest) {
        load_part(q, left, x);
        if constexpr (sizeof...(rest) > 0) self(self, rest...);
    };
    if (left >= 8) whole(whole, p, r, more...);
    else part(part, p, r, more...);
}
template <bool FAR = false, class T>
__device__ __forceinline__ void load8(const T* p, int64_t left, float (&v)[8]) {
    Raw8<T> r;
    load8s<FAR>(left, p, r);
    widen8(r, v);
}

// Stores round to nearest even.
template <bool FAR = false>
__device__ __forceinline__ void store8(float* p, int64_t left, const float (&v)[8]) {
    static_assert(!FAR);
    if (left >= 8) {
        *reinterpret_cast<f32x4_any*>(p) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4_any*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = v[i];
    }
}
template <bool FAR = false>
__device__ __forceinline__ void store8(bf16_t* p, int64_t left, const float (&v)[8]) {
    if (left >= 8) {
        bf16x8 a;
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = static_cast<bf16_t>(v[i]);
        if constexpr (FAR) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, a), reinterpret_cast<u32x4_any*>(p));
        else *reinterpret_cast<bf16x8_any*>(p) = a;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = static_cast<bf16_t>(v[i]);
    }
}

// |v| as an integer: ordered as the magnitudes, with infinities and NaN last.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t max8(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
    return m;
}

// Scale byte of a block whose largest magnitude has these bits, m * 2^p with
// m in [1, 2): the smallest e with m * 2^(p - e) <= 448 = 1.75 * 2^8 is p - 8,
// one more where m > 1.75.  255 where the block holds an infinity or a NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return 255u;
    const int b = static_cast<int>(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return static_cast<uint32_t>(max(b, 1));
}

// 2^-e of a scale byte (a NaN for 255); e <= 120, so the result is normal.
__device__ __forceinline__ float inverse_scale(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7fc00000u : (254u - byte) << 23);
}
// 2^e of a scale byte (a NaN for 255).
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7fc00000u : byte << 23);
}

// Eight values times `inv` as e4m3, to nearest even.
__device__ __forceinline__ u32x2 pack8(const float (&v)[8], float inv) {
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inv, v[4 * i + 1] * inv, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inv, v[4 * i + 3] * inv, w, true);
        r[i] = static_cast<uint32_t>(w);
    }
    return r;
}
__device__ __forceinline__ void unpack8(u32x2 q, float scale, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(q[i]), false);
        const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(q[i]), true);
        v[4 * i] = lo[0] * scale;
        v[4 * i + 1] = lo[1] * scale;
        v[4 * i + 2] = hi[0] * scale;
        v[4 * i + 3] = hi[1] * scale;
    }
}

// Rotations within rows of 16 lanes (data-parallel primitives: no LDS).
template <int N>
__device__ __forceinline__ uint32_t rotate16(uint32_t v) {
    return static_cast<uint32_t>(
        __builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x120 + N, 0xf, 0xf, false));
}
__device__ __forceinline__ uint32_t max16(uint32_t v) {
    v = max(v, rotate16<8>(v));
    v = max(v, rotate16<4>(v));
    v = max(v, rotate16<2>(v));
    return max(v, rotate16<1>(v));
}
// The sum over a wave, the same in every lane.
__device__ __forceinline__ float sum64(float v) {
    v += __uint_as_float(rotate16<8>(__float_as_uint(v)));
    v += __uint_as_float(rotate16<4>(__float_as_uint(v)));
    v += __uint_as_float(rotate16<2>(__float_as_uint(v)));
    v += __uint_as_float(rotate16<1>(__float_as_uint(v)));
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// A launch has less than 2^32 threads: `total` workgroups of `threads` each, in as many launches as that takes.
template <class F>
int in_launches(int64_t total, int threads, F&& launch) {
    const int64_t most = 0xffffffff / threads;
    for (int64_t first = 0; first < total; first += most) {
        launch(first, static_cast<uint32_t>(total - first < most ? total - first : most));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Whether bytes read once, or results that a later launch reads, are found no
// sooner for having been kept: the memory-side cache holds 256 MB.  In us, past the
// cache and through it: norm of 28,160 x 4096 in bf16 with a residual to 8 bits 149
// and 154, its gradients 157 and 173; dequantise to bf16 50 and 63; 28,160 x 1280
// and shorter within 1 either way.
inline bool is_far(int64_t bytes) { return bytes > int64_t(200) << 20; }

// launch(FAR) for elements of T.  In f32 the same norm takes 323 past the cache and
// 277 through it, its gradients 382 and 350, dequantise 189 and 142, quantise 110 and
// 106, both forms 148 and 135.
template <class T, class F>
int past_cache(int64_t bytes, F&& launch) {
    if constexpr (sizeof(T) == 2)
        if (is_far(bytes)) return launch(std::true_type());
    return launch(std::false_type());
}

}  // namespace vp
