// vp_fp8.hip -- matrices into 8 bits, out of them, and transposed.
//
// A block of 128 columns is 16 lanes of 8 values: its largest magnitude is a
// maximum over 8 registers and four lane rotations, its exponent comes from
// that maximum's bits, and the eight products are rounded by the conversion
// instructions.  Nothing is divided and no logarithm is taken.
#include <type_traits>

#include "vp_fp8_device.h"

namespace vp {
namespace {

// ---------------------------------------------------------------------------
// Rows form, a scale for each row: one pass over memory, bound by it.  Each
// group of 16 lanes takes kItems blocks of 128 columns, and asks for all of
// them before it uses the first.  89,600 x 1536 in bf16: 66 us, 6.2 TB/s.
// ---------------------------------------------------------------------------
constexpr int kItems = 4;

template <class T, bool FAR>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* x, int64_t ld, int32_t cols,
                                                            int32_t blocks, int64_t total, int64_t first_wg,
                                                            Fp8View out) {
    const int lane = threadIdx.x & 15;
    const int64_t first = (first_wg + blockIdx.x) * (16 * kItems) + (threadIdx.x >> 4);
    int64_t row = first / blocks;
    int32_t kb = static_cast<int32_t>(first - row * blocks);
    float v[kItems][8];
    int64_t at_row[kItems];
    int32_t at_kb[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        at_row[i] = first + 16 * i < total ? row : -1;
        at_kb[i] = kb;
        const int32_t c = kb * kBlock + lane * 8;
        load8<FAR>(x + row * ld + c, at_row[i] < 0 ? 0 : cols - c, v[i]);
        kb += 16;
        while (kb >= blocks) {
            kb -= blocks;
            ++row;
        }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const uint32_t byte = scale_byte(max16(max8(v[i])));
        if (at_row[i] < 0) continue;
        const u32x2 q = pack8(v[i], inverse_scale(byte));
        *reinterpret_cast<u32x2*>(out.q + at_row[i] * out.ld + at_kb[i] * int64_t(kBlock) + lane * 8) = q;
        uint8_t* s = out.scale + at_row[i] * out.sld + at_kb[i];
        if (lane == 0) *s = static_cast<uint8_t>(byte);
        // the bytes between the last block's and the row's end
        if (at_kb[i] == blocks - 1 && lane > 0 && at_kb[i] + lane < out.sld) s[lane] = 0;
    }
}

// ---------------------------------------------------------------------------
// Any form: a workgroup takes 128 x 128 values, 4 rows x 8 columns a thread,
// in registers.  Row maxima are rotations over 16 lanes; column maxima a
// maximum over the thread's rows, two lane exchanges and a step through LDS;
// the transposed bytes go through LDS so that both forms are stored in whole
// lines.  The tile's row c lies at c with its lowest bit turned over for c >=
// 64, its 16-byte pieces permuted by c / 8: the 64 lanes of a wave, 8 columns
// and 4 rows apart, then write 64 different banks.  Bound by memory where there
// are many tiles (28,160 x 4096 in bf16 to both forms 97 us, 4.8 TB/s, to one with a
// scale for 128 x 128 60 us, 5.8 TB/s), by the chain through its two or three barriers
// where there are few (576 x 1280: 6 us).  Of a matrix in 8 bits, 8190 x 4096 in 20 us,
// 3.4 TB/s: a lane's loads are of 8 bytes and a scale.
// ---------------------------------------------------------------------------
struct Source {
    const void* x;
    int64_t ld;
    Fp8View in;
};

template <bool FAR, class T>
__device__ __forceinline__ void load_source(const Source& s, const T*, int64_t r, int32_t c,
                                            int64_t left, float (&v)[8]) {
    load8<FAR>(static_cast<const T*>(s.x) + r * s.ld + c, left, v);
}
// Values in 8 bits reach 448 * 2^127, past f32's 2^128, so a tile whose rows have
// scales of their own holds them kDown powers of two smaller, which is exact: they
// are multiples of 2^-135, and f32's least is 2^-149.
constexpr int kDown = 8;
__device__ __forceinline__ float held_scale(uint32_t byte) {
    return byte == 255u ? __uint_as_float(0x7fc00000u) : ldexpf(1.0f, static_cast<int>(byte) - 127 - kDown);
}
// scale_byte of a largest magnitude held so: m * 2^e with m in [0.5, 1), below f32's normal numbers too.
__device__ __forceinline__ uint32_t held_scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return 255u;
    const float v = __uint_as_float(top);
    const int b = __builtin_amdgcn_frexp_expf(v) + kDown + 118 + (__builtin_amdgcn_frexp_mantf(v) > 0.875f ? 1 : 0);
    return static_cast<uint32_t>(top == 0 ? 1 : max(b, 1));
}
// The factor from a value held so to its quotient by a byte's power of two, 2^(127 + kDown - byte), as far as f32 holds
// it; the rest of it, for the least bytes.
__device__ __forceinline__ float held_inverse_scale(uint32_t byte) {
    return byte == 255u ? __uint_as_float(0x7fc00000u) : ldexpf(1.0f, min(127 + kDown - static_cast<int>(byte), 127));
}
__device__ __forceinline__ float held_inverse_rest(uint32_t byte) {
    return ldexpf(1.0f, max(kDown - static_cast<int>(byte), 0));
}

template <bool FAR>
__device__ __forceinline__ void load_source(const Source& s, const uint8_t*, int64_t r, int32_t c,
                                            int64_t left, float (&v)[8]) {
    if (left <= 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        return;
    }
    const u32x2 q = *reinterpret_cast<const u32x2*>(s.in.q + r * s.in.ld + c);   // rows are whole 128s
    // a tile with one scale keeps it: its bytes move as they are
    unpack8(q, s.in.block == 1 ? held_scale(s.in.scale[r * s.in.sld + c / kBlock]) : 1.0f, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? v[i] : 0.0f;
}

__device__ __forceinline__ int tile_at(int c, int piece) {
    return (c ^ ((c >> 6) & 1)) * 128 + ((piece ^ (c >> 3)) & 7) * 16;
}

// The byte of block `kb` of a row of scales, and zeros after the last of `blocks`.
__device__ __forceinline__ void put_scale(const Fp8View& f, int64_t row, int64_t kb, int64_t blocks, uint32_t byte) {
    uint8_t* s = f.scale + row * f.sld + kb;
    s[0] = static_cast<uint8_t>(byte);
    if (kb == blocks - 1)
        for (int p = 1; kb + p < f.sld; ++p) s[p] = 0;
}

// T: float, bf16_t, or uint8_t for a matrix that is held in 8 bits.
template <class T, bool FAR>
__global__ __launch_bounds__(512) void quantize_tile_kernel(Source src, int32_t rows, int32_t cols,
                                                            int32_t tiles_r, int32_t tiles_c, uint32_t first_wg,
                                                            int32_t block, Fp8View by_rows, Fp8View by_cols) {
    constexpr bool kHeld = sizeof(T) == 1;
    __shared__ __align__(16) uint8_t tile[128 * 128];
    __shared__ uint32_t top[8][128];
    __shared__ __align__(16) float inverse[128];
    __shared__ float rest[kHeld ? 128 : 1];
    const int t = threadIdx.x, cg = t & 15, rg = t >> 4, wave = t >> 6;
    const uint32_t at = first_wg + blockIdx.x;
    const int64_t rb = at / static_cast<uint32_t>(tiles_c);
    const int32_t cb = static_cast<int32_t>(at - rb * tiles_c);
    const int64_t r0 = rb * 128 + rg * 4;
    const int32_t c0 = cb * 128 + cg * 8;

    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        load_source<FAR>(src, static_cast<const T*>(nullptr), r0 + i, c0, r0 + i < rows ? int64_t(cols) - c0 : 0, v[i]);

    uint32_t tile_byte = 0;
    float tile_inverse = 1.0f;
    if (kHeld && block != 1) tile_byte = src.in.scale[rb * src.in.sld + cb];
    if (!kHeld && block != 1) {   // one scale for the tile
        uint32_t all = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) all = max(all, max8(v[i]));
        all = max16(all);
        all = max(all, static_cast<uint32_t>(__shfl_xor(static_cast<int>(all), 16)));
        all = max(all, static_cast<uint32_t>(__shfl_xor(static_cast<int>(all), 32)));
        if ((t & 63) == 0) top[0][wave] = all;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) all = max(all, top[0][w]);
        tile_byte = scale_byte(all);
        tile_inverse = inverse_scale(tile_byte);
    }
    if (block != 1 && t == 0) {
        if (by_rows.q != nullptr) put_scale(by_rows, rb, cb, tiles_c, tile_byte);
        if (by_cols.q != nullptr) put_scale(by_cols, cb, rb, tiles_r, tile_byte);
    }

    if (by_rows.q != nullptr) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t byte = block == 1 ? scale_byte(max16(max8(v[i]))) : tile_byte;
            if (r0 + i >= rows) continue;
            *reinterpret_cast<u32x2*>(by_rows.q + (r0 + i) * by_rows.ld + c0) =
                pack8(v[i], block == 1 ? inverse_scale(byte) : tile_inverse);
            if (block == 1 && cg == 0) put_scale(by_rows, r0 + i, cb, tiles_c, byte);
        }
    }
    if (by_cols.q == nullptr) return;   // the same for the whole launch

    if (block == 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) m = max(m, magnitude(v[i][j]));
            m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16)));
            m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32)));
            if ((t & 63) < 16) top[wave][cg * 8 + j] = m;
        }
        __syncthreads();
        if (t < 128) {
            uint32_t m = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) m = max(m, top[w][t]);
            const uint32_t byte = kHeld ? held_scale_byte(m) : scale_byte(m);
            inverse[t] = kHeld ? held_inverse_scale(byte) : inverse_scale(byte);
            if constexpr (kHeld) rest[t] = held_inverse_rest(byte);
            if (cb * int64_t(128) + t < cols) put_scale(by_cols, cb * int64_t(128) + t, rb, tiles_r, byte);
        }
        __syncthreads();
    }
    const f32x4 low = *reinterpret_cast<const f32x4*>(inverse + cg * 8);
    const f32x4 high = *reinterpret_cast<const f32x4*>(inverse + cg * 8 + 4);
    if (kHeld && block == 1) {
        float most = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) most = fmaxf(most, fmaxf(low[j], high[j]));
        if (most == 0x1p127f) {   // bytes of kDown and less
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i][j] *= rest[cg * 8 + j];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float inv = block != 1 ? tile_inverse : j < 4 ? low[j] : high[j - 4];
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0][j] * inv, v[1][j] * inv, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2][j] * inv, v[3][j] * inv, w, true);
        *reinterpret_cast<int*>(tile + tile_at(cg * 8 + j, rg >> 2) + (rg & 3) * 4) = w;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {   // 8 lanes write one column's 128 bytes
        const int c = i * 64 + (t >> 3), piece = t & 7;
        if (cb * int64_t(128) + c < cols)
            *reinterpret_cast<u32x4*>(by_cols.q + (cb * int64_t(128) + c) * by_cols.ld + rb * 128 + piece * 16) =
                *reinterpret_cast<const u32x4*>(tile + tile_at(c, piece));
    }
}

// ---------------------------------------------------------------------------
// Out of 8 bits, bound by memory: 16 lanes a block of 128 columns, so that their
// stores are whole lines; each takes kItems blocks, all asked for first.
// 28,160 x 4096 to bf16: 50 us, 6.9 TB/s; to f32, eight floats a lane in two stores, 139
// us, 4.2 TB/s.
// ---------------------------------------------------------------------------
template <class T, bool FAR>
__global__ __launch_bounds__(256) void dequantize_kernel(Fp8View in, T* out, int64_t ld, int32_t blocks,
                                                         int64_t total, int64_t first_wg) {
    const int lane = threadIdx.x & 15;
    const int64_t first = (first_wg + blockIdx.x) * (16 * kItems) + (threadIdx.x >> 4);
    int64_t row = first / blocks;
    int32_t kb = static_cast<int32_t>(first - row * blocks);
    u32x2 q[kItems];
    uint32_t byte[kItems];
    int64_t at_row[kItems];
    int32_t at_kb[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        at_row[i] = first + 16 * i < total ? row : -1;
        at_kb[i] = kb;
        if (at_row[i] >= 0) {
            q[i] = *reinterpret_cast<const u32x2*>(in.q + row * in.ld + kb * int64_t(kBlock) + lane * 8);
            byte[i] = in.scale[(in.block == 1 ? row : row / kBlock) * in.sld + kb];
        }
        kb += 16;
        while (kb >= blocks) {
            kb -= blocks;
            ++row;
        }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        if (at_row[i] < 0) continue;
        const int32_t c = at_kb[i] * kBlock + lane * 8;
        float v[8];
        unpack8(q[i], scale_value(byte[i]), v);
        store8<FAR>(out + at_row[i] * ld + c, int64_t(in.cols) - c, v);
    }
}

template <class T>
int tile_launch(const QuantizeArgs& a, hipStream_t stream) {
    const int64_t tr = (int64_t(a.rows) + 127) / 128, tc = (int64_t(a.cols) + 127) / 128;
    const int32_t block = a.by_rows.q != nullptr ? a.by_rows.block : a.by_cols.block;
    auto launch = [&]<bool FAR>(std::bool_constant<FAR>) {
        return in_launches(tr * tc, 512, [&](int64_t first, uint32_t wgs) {
            quantize_tile_kernel<T, FAR><<<wgs, 512, 0, stream>>>(
                Source{a.x, a.ld, a.in}, a.rows, a.cols, static_cast<int32_t>(tr), static_cast<int32_t>(tc),
                static_cast<uint32_t>(first), block, a.by_rows, a.by_cols);
        });
    };
    return past_cache<T>(int64_t(a.rows) * a.cols * sizeof(T), launch);   // (what is held in 8 bits is read one way)
}

template <class T>
int quantize_launch(const QuantizeArgs& a, hipStream_t stream) {
    if (a.by_cols.q != nullptr || a.by_rows.block != 1) return tile_launch<T>(a, stream);
    const int32_t blocks = static_cast<int32_t>((int64_t(a.cols) + 127) / 128);
    const int64_t total = int64_t(a.rows) * blocks;
    const int64_t wgs = (total + 16 * kItems - 1) / (16 * kItems);
    auto launch = [&]<bool FAR>(std::bool_constant<FAR>) {
        return in_launches(wgs, 256, [&](int64_t first, uint32_t n) {
            quantize_rows_kernel<T, FAR><<<n, 256, 0, stream>>>(static_cast<const T*>(a.x), a.ld, a.cols, blocks, total,
                                                                first, a.by_rows);
        });
    };
    return past_cache<T>(int64_t(a.rows) * a.cols * sizeof(T), launch);
}

template <class T>
int dequantize_launch(const Fp8View& in, T* out, int64_t ld, hipStream_t stream) {
    const int32_t blocks = static_cast<int32_t>((int64_t(in.cols) + 127) / 128);
    const int64_t total = int64_t(in.rows) * blocks;
    const int64_t wgs = (total + 16 * kItems - 1) / (16 * kItems);
    auto launch = [&]<bool FAR>(std::bool_constant<FAR>) {
        return in_launches(wgs, 256, [&](int64_t first, uint32_t n) {
            dequantize_kernel<T, FAR><<<n, 256, 0, stream>>>(in, out, ld, blocks, total, first);
        });
    };
    // (only the stores pass by the cache: what is held in 8 bits may have been written just before)
    return past_cache<T>(int64_t(in.rows) * in.cols * sizeof(T), launch);
}

}  // namespace

int launch_quantize(const QuantizeArgs& a, hipStream_t stream) {
    switch (a.type) {
        case In::fp8: return tile_launch<uint8_t>(a, stream);
        case In::f32: return quantize_launch<float>(a, stream);
        default: return quantize_launch<bf16_t>(a, stream);
    }
}

int launch_dequantize(const Fp8View& in, void* out, bool bf16, int64_t ld, hipStream_t stream) {
    return bf16 ? dequantize_launch(in, static_cast<bf16_t*>(out), ld, stream)
                : dequantize_launch(in, static_cast<float*>(out), ld, stream);
}

}  // namespace vp
