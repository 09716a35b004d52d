// vp_fp8.h -- what the host side (vp_fp8_api.cpp) and the kernels of the 8-bit
// operators (vp_fp8.hip, vp_norm.hip, vp_matmul.hip) share.
//
// A launcher checks nothing: vp_fp8_api.cpp has checked every pointer, size
// and stride before it calls one.  It returns a hipError_t as an int.
#pragma once

#include <cstdint>

#include <hip/hip_runtime_api.h>

namespace vp {

constexpr int kBlock = 128;   // columns that share a scale

constexpr int64_t q_ld(int64_t cols) { return (cols + 127) / 128 * 128; }
constexpr int64_t scale_ld(int64_t cols) { return (cols + 511) / 512 * 4; }

// Records the detail of a failed call for vp_last_error_message (vp_api.cpp).
int32_t set_error(int32_t status, const char* msg) noexcept;

// A matrix in 8 bits as the kernels take it; q == nullptr: not wanted.
struct Fp8View {
    uint8_t* q;
    uint8_t* scale;
    int64_t ld;        // bytes between rows of q, a multiple of 128
    int64_t sld;       // bytes between rows of scale, a multiple of 4
    int32_t rows, cols;
    int32_t block;     // rows that share a scale: 1 or 128
};

enum class In { f32, bf16, fp8 };

struct QuantizeArgs {
    const void* x;     // f32 / bf16 source, or
    Fp8View in;        // the 8-bit one
    In type;
    int64_t ld;
    int32_t rows, cols;
    Fp8View by_rows, by_cols;
};
int launch_quantize(const QuantizeArgs& a, hipStream_t stream);

int launch_dequantize(const Fp8View& in, void* out, bool bf16, int64_t ld, hipStream_t stream);

struct NormArgs {
    const void *x, *residual, *weight;
    void *h, *out;
    Fp8View out8;
    float* rstd;
    int64_t ldx, ldr, ldh, ldo;
    int32_t rows, cols;
    float eps;
};
int launch_norm(const NormArgs& a, bool bf16, hipStream_t stream);

struct NormBackwardArgs {
    const void *dy, *h, *weight, *dh;
    const float* rstd;
    void* dx;
    float* dweight;
    float* partial;    // [groups][cols] partial sums of dweight, or nullptr
    int64_t ldy, ldh, lddh, lddx;
    int32_t rows, cols;
};
// Rows of partial sums that the launch writes for this shape and elements of `size` bytes; bf16 has the most.
int norm_backward_groups(int64_t rows, int64_t cols, int size = 2);
int launch_norm_backward(const NormBackwardArgs& a, bool bf16, hipStream_t stream);

struct MatmulArgs {
    Fp8View a, b;      // [M][K], [N][K]
    void* out;
    int64_t ld;
    bool bf16;
    float* partial;
};
// Bytes; -1 where the result has more tiles than a launch takes.
int64_t matmul_workspace(int64_t m, int64_t n, int64_t k, bool bf16);
// The launches of launch_matmul for these sizes, as vp_fp8_matmul_kernels gives them, and how many (2 at most).
int describe_matmul(int64_t m, int64_t n, int64_t k, int64_t ld, bool bf16, int32_t (*rows)[4]);
int launch_matmul(const MatmulArgs& a, hipStream_t stream);

}  // namespace vp
