// vp_norm.hip -- root-mean-square norm of a residual stream, and its gradients.
//
// Both are bound by memory.  A row stays in registers between its sum of
// squares and its output, so each input is read once: 8 columns in each of V
// vectors a thread, NT threads a row (a wave for short rows, so that no row
// waits at a barrier; 256 threads up to 8192 columns).  Longer rows are read
// a second time, from beyond L2, which does not hold the rows of 1024 workgroups
// (4096 x 12,288 in bf16 with a residual: 401 MB read, 201 needed).  Sums are in
// f32: V * 8 products in a thread, then a tree over lanes and waves.  28,160 x 4096
// in bf16: with a residual, and h, to 8 bits 130 us, 6.2 TB/s; gradients 151 us, 6.1
// TB/s, and the sum of the workgroups' shares, 5 us.  4096 x 12,288: 92 us, 6.0
// TB/s of what is moved; gradients 84 us for dx, which reads dy and h twice, and 60
// for dweight, which reads them once more.
#include "vp_fp8_device.h"

namespace vp {
namespace {

constexpr int kMostGroups = 1024;   // workgroups of a launch: four a CU
constexpr int kLongGroups = 32;     // of rows, for dweight of long rows
// Rows that dweight adds in one sequence, then the parts.  (All of a wave's rows in one, 2^22 rows of 64 equal values came
// out 1.7e-5 off, 2^26 rows 1.2e-4.)
constexpr int kPart = 64;
constexpr int64_t kMostAcross = 0xffff;   // workgroups across a row's columns: a launch has less than 2^32 threads

// Sum over the NT threads of a row, the same in all of them.
template <int NT>
__device__ __forceinline__ float sum_row(float v, float* shared) {
    v = sum64(v);
    if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) v += shared[w];
        __syncthreads();   // before the next row writes it
    }
    return v;
}

template <class T>
__device__ __forceinline__ void round_to(float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(static_cast<T>(v[i]));
    }
}

// y = h * rstd * w of eight columns from c on, to `out` and as 8 bits.
template <class T>
__device__ __forceinline__ void write_norm(const NormArgs& a, int64_t row, int64_t c, float rstd,
                                           const float (&h)[8], const float (&w)[8]) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = h[i] * rstd * w[i];
    if (a.out != nullptr) store8(static_cast<T*>(a.out) + row * a.ldo + c, a.cols - c, y);
    if (a.out8.q != nullptr) {
        const int lane = threadIdx.x & 15;
        const uint32_t byte = scale_byte(max16(max8(y)));
        if (c < a.out8.ld) {
            *reinterpret_cast<u32x2*>(a.out8.q + row * a.out8.ld + c) = pack8(y, inverse_scale(byte));
            const int64_t kb = c / kBlock;
            uint8_t* s = a.out8.scale + row * a.out8.sld + kb;
            if (lane == 0) *s = static_cast<uint8_t>(byte);
            if (kb == a.out8.ld / kBlock - 1 && lane > 0 && kb + lane < a.out8.sld) s[lane] = 0;
        }
    }
}

// h = x + residual of eight columns, rounded to T.
template <class T, bool FAR>
__device__ __forceinline__ void load_sum(const NormArgs& a, int64_t row, int64_t c, float (&h)[8]) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx + c;
    if (a.residual == nullptr) {
        load8<FAR>(x, a.cols - c, h);
        return;
    }
    Raw8<T> rx, rr;
    float r[8];
    load8s<FAR>(a.cols - c, x, rx, static_cast<const T*>(a.residual) + row * a.ldr + c, rr);
    widen8(rx, h);
    widen8(rr, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] += r[i];
    round_to<T>(h);
}

// Rows of up to NT * V * 8 columns.
template <class T, int NT, int V, bool FAR>
__global__ __launch_bounds__(256) void norm_kernel(NormArgs a) {
    __shared__ float shared[4];
    const int t = threadIdx.x % NT;
    const int64_t step = int64_t(gridDim.x) * (256 / NT);
    float w[V][8];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int64_t c = (k * NT + t) * 8;
        load8(static_cast<const T*>(a.weight) + c, a.cols - c, w[k]);
    }
    for (int64_t row = blockIdx.x * int64_t(256 / NT) + threadIdx.x / NT; row < a.rows; row += step) {
        float h[V][8], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) load_sum<T, FAR>(a, row, (k * NT + t) * 8, h[k]);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int64_t c = (k * NT + t) * 8;
            if (a.h != nullptr) store8<FAR>(static_cast<T*>(a.h) + row * a.ldh + c, a.cols - c, h[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += h[k][i] * h[k][i];
        }
        const float rstd = 1.0f / sqrtf(sum_row<NT>(sum, shared) / a.cols + a.eps);
        if (a.rstd != nullptr && t == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int k = 0; k < V; ++k) write_norm<T>(a, row, (k * NT + t) * 8, rstd, h[k], w[k]);
    }
}

// A thread's share of a sum over a long row, of eight columns at a time: those of
// 128 rounds first, so that no term is added to a sum of many more than a thousand
// (2^27 columns in one sequence: 7e-5 off in rstd).
template <class F>
__device__ __forceinline__ float sum_long(int64_t cols, F&& eight) {
    float sum = 0.0f;
    for (int64_t c0 = 0; c0 < cols; c0 += 128 * 2048) {
        const int64_t end = min(cols, c0 + 128 * 2048);
        float part = 0.0f;
#pragma unroll 4
        for (int64_t c = c0 + threadIdx.x * 8; c < end; c += 2048) part += eight(c);
        sum += part;
    }
    return sum;
}

// Rows of any length: 256 threads, read twice.
template <class T>
__global__ __launch_bounds__(256) void norm_long_kernel(NormArgs a) {
    __shared__ float shared[4];
    const int64_t padded = q_ld(a.cols);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float sum = sum_long(a.cols, [&](int64_t c) {
            float h[8], s = 0.0f;
            load_sum<T, false>(a, row, c, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += h[i] * h[i];
            return s;
        });
        const float rstd = 1.0f / sqrtf(sum_row<256>(sum, shared) / a.cols + a.eps);
        if (a.rstd != nullptr && threadIdx.x == 0) a.rstd[row] = rstd;
        // whole blocks of 128 columns, so that 16 lanes stay together
        for (int64_t c = threadIdx.x * 8; c < padded; c += 256 * 8) {
            float h[8], w[8];
            load_sum<T, false>(a, row, c, h);
            if (a.h != nullptr) store8(static_cast<T*>(a.h) + row * a.ldh + c, a.cols - c, h);
            load8(static_cast<const T*>(a.weight) + c, a.cols - c, w);
            write_norm<T>(a, row, c, rstd, h, w);
        }
    }
}

// ---------------------------------------------------------------------------
// Backward.  g = dy w, n = h rstd: dx = rstd (g - n mean(g n)) + dh.  A
// workgroup keeps its rows' share of dweight = sum dy n in registers and
// writes it once, as one row of `partial`, which a second kernel sums in order.
// ---------------------------------------------------------------------------
template <bool FAR, class T>
__device__ __forceinline__ void write_dx(const NormBackwardArgs& a, int64_t row, int64_t c, float rstd,
                                         float mean, const float (&dy)[8], const float (&n)[8],
                                         const float (&w)[8], const Raw8<T>& dh) {
    float dx[8], d[8];
    widen8(dh, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        dx[i] = rstd * (dy[i] * w[i] - n[i] * mean);
        if (a.dh != nullptr) dx[i] += d[i];
    }
    store8<FAR>(static_cast<T*>(a.dx) + row * a.lddx + c, a.cols - c, dx);
}

// Eight columns of a row's inputs.
template <bool FAR, class T>
__device__ __forceinline__ void load_row(const NormBackwardArgs& a, int64_t row, int64_t c, Raw8<T>& dy, Raw8<T>& h,
                                         Raw8<T>& dh) {
    const T* y = static_cast<const T*>(a.dy) + row * a.ldy + c;
    const T* x = static_cast<const T*>(a.h) + row * a.ldh + c;
    if (a.dh != nullptr) load8s<FAR>(a.cols - c, y, dy, x, h, static_cast<const T*>(a.dh) + row * a.lddh + c, dh);
    else load8s<FAR>(a.cols - c, y, dy, x, h);
}

// AHEAD: a row's inputs are asked for while the row before it is summed.  That
// pays where a workgroup's row is no more than 16 bytes a lane, which alone are
// too little under way: 28,160 x 1280 in 58.1 us against 77.6.  Wider rows lose
// waves to the registers that it takes (4096: 162 us against 157), and rows of
// one wave have other waves' loads beside theirs (768: 42.2 against 36.3).
// MANY: a thread has more than kPart rows, and adds their dweight in parts.  (Compiled in, it costs launches of fewer
// rows 2 to 3 %: 28,160 x 384 in 25.6 us against 24.8.)
template <class T, int NT, int V, bool FAR, bool MANY>
__global__ __launch_bounds__(256) void norm_backward_kernel(NormBackwardArgs a) {
    constexpr bool AHEAD = NT == 256 && V == 1;
    __shared__ float shared[4];
    __shared__ float join[NT == 64 ? 4 * 64 * V * 8 : 1];
    const int t = threadIdx.x % NT;
    const int64_t step = int64_t(gridDim.x) * (256 / NT);
    float w[V][8], dw[V][8];
    float parts[NT == 64 ? V : 1][8];   // a wave's finished parts of dweight; a workgroup's are in `partial`
    Raw8<T> y[V], h[V], dh[V];
    float rstd = 0.0f;
    int64_t row = blockIdx.x * int64_t(256 / NT) + threadIdx.x / NT;
    const auto fetch = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < V; ++k) load_row<FAR>(a, r, (k * NT + t) * 8, y[k], h[k], dh[k]);
        rstd = a.rstd[r];
    };
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int64_t c = (k * NT + t) * 8;
        load8(static_cast<const T*>(a.weight) + c, a.cols - c, w[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dw[k][i] = 0.0f;
            if constexpr (NT == 64) parts[k][i] = 0.0f;
        }
    }
    float* to = a.partial + blockIdx.x * int64_t(a.cols);
    bool begun = false;
    const auto end_part = [&]() {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int64_t c = (k * NT + t) * 8;
            if constexpr (NT != 64) {
                if (MANY && begun) {
                    float before[8];
                    load8(to + c, a.cols - c, before);
#pragma unroll
                    for (int i = 0; i < 8; ++i) dw[k][i] += before[i];
                }
                store8(to + c, a.cols - c, dw[k]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (NT == 64) parts[k][i] += dw[k][i];
                dw[k][i] = 0.0f;
            }
        }
        begun = true;
    };
    if (AHEAD && row < a.rows) fetch(row);
    for (int in_part = 0; row < a.rows; row += step) {
        if (MANY) {
            if (in_part == kPart) {
                end_part();
                in_part = 0;
            }
            ++in_part;
        }
        if constexpr (!AHEAD) fetch(row);
        float g[V][8], n[V][8], sum = 0.0f;
        Raw8<T> add[V];
        const float r = rstd;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            widen8(y[k], g[k]);
            widen8(h[k], n[k]);
            add[k] = dh[k];
        }
        if (AHEAD && row + step < a.rows) fetch(row + step);
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[k][i] *= r;
                sum += g[k][i] * w[k][i] * n[k][i];
                dw[k][i] += g[k][i] * n[k][i];
            }
        const float mean = sum_row<NT>(sum, shared) / a.cols;
#pragma unroll
        for (int k = 0; k < V; ++k) write_dx<FAR, T>(a, row, (k * NT + t) * 8, r, mean, g[k], n[k], w[k], add[k]);
    }
    if (a.partial == nullptr) return;
    end_part();
    if constexpr (NT == 64) {   // four waves, each with rows of its own
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) join[(wave * V * 8 + k * 8 + i) * 64 + t] = parts[k][i];
        __syncthreads();
        for (int e = wave; e < V * 8; e += 4) {
            const int64_t c = ((e / 8) * 64 + t) * 8 + e % 8;
            float s = 0.0f;
#pragma unroll
            for (int u = 0; u < 4; ++u) s += join[(u * V * 8 + e) * 64 + t];
            if (c < a.cols) to[c] = s;
        }
    }
}

// Rows of any length: dx, reading dy and h twice.
template <class T>
__global__ __launch_bounds__(256) void norm_backward_long_kernel(NormBackwardArgs a) {
    __shared__ float shared[4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float rstd = a.rstd[row];
        const float sum = sum_long(a.cols, [&](int64_t c) {
            float dy[8], h[8], w[8], s = 0.0f;
            load8(static_cast<const T*>(a.dy) + row * a.ldy + c, a.cols - c, dy);
            load8(static_cast<const T*>(a.h) + row * a.ldh + c, a.cols - c, h);
            load8(static_cast<const T*>(a.weight) + c, a.cols - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += dy[i] * w[i] * (h[i] * rstd);
            return s;
        });
        const float mean = sum_row<256>(sum, shared) / a.cols;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += 256 * 8) {
            float dy[8], h[8], w[8];
            load8(static_cast<const T*>(a.dy) + row * a.ldy + c, a.cols - c, dy);
            load8(static_cast<const T*>(a.h) + row * a.ldh + c, a.cols - c, h);
            load8(static_cast<const T*>(a.weight) + c, a.cols - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] *= rstd;
            Raw8<T> dh;
            if (a.dh != nullptr) load8s<false>(a.cols - c, static_cast<const T*>(a.dh) + row * a.lddh + c, dh);
            write_dx<false, T>(a, row, c, rstd, mean, dy, h, w, dh);
        }
    }
}

// Rows of any length: a share of dweight, 64 columns a wave, 4 waves a
// workgroup with rows of their own.  Runs before the long kernel, which may
// write dx over dy or h.
template <class T>
__global__ __launch_bounds__(256) void norm_dweight_long_kernel(NormBackwardArgs a) {
    __shared__ float join[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t c0 = blockIdx.x * int64_t(64); c0 < a.cols; c0 += gridDim.x * int64_t(64)) {
        const int64_t c = c0 + lane;
        const int64_t step = gridDim.y * int64_t(4);
        float s = 0.0f;
        if (c < a.cols)
            for (int64_t row0 = blockIdx.y * int64_t(4) + wave; row0 < a.rows; row0 += kPart * step) {
                const int64_t end = min(int64_t(a.rows), row0 + kPart * step);
                float part = 0.0f;
                for (int64_t row = row0; row < end; row += step)
                    part += static_cast<float>(static_cast<const T*>(a.dy)[row * a.ldy + c]) *
                            (static_cast<float>(static_cast<const T*>(a.h)[row * a.ldh + c]) * a.rstd[row]);
                s += part;
            }
        join[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && c < a.cols)
            a.partial[blockIdx.y * int64_t(a.cols) + c] =
                (join[0][lane] + join[1][lane]) + (join[2][lane] + join[3][lane]);
        __syncthreads();   // before the next columns' sums
    }
}

// dweight = the sum of the groups' rows: 32 columns a workgroup, four in a
// thread, every 128th row, so that all of them are asked for at once; then a
// tree over the 8 parts of a wave and the 16 waves.
__global__ __launch_bounds__(1024) void sum_partial_kernel(const float* partial, float* dweight,
                                                           int32_t groups, int32_t cols) {
    __shared__ __align__(16) f32x4 join[16][8];
    const int lane = threadIdx.x & 7, part = threadIdx.x >> 3;
    for (int64_t c0 = blockIdx.x * int64_t(32); c0 < cols; c0 += gridDim.x * int64_t(32)) {
        const int64_t c = c0 + lane * 4;
        f32x4 v[kMostGroups / 128], s{0.0f, 0.0f, 0.0f, 0.0f};
        if (c + 4 <= cols) {
#pragma unroll
            for (int k = 0; k < kMostGroups / 128; ++k)   // rows past the end read the last one again
                v[k] = *reinterpret_cast<const f32x4_any*>(partial + min(part + k * 128, groups - 1) * int64_t(cols) + c);
        } else {
#pragma unroll
            for (int k = 0; k < kMostGroups / 128; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[k][i] = c + i < cols ? partial[min(part + k * 128, groups - 1) * int64_t(cols) + c + i] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < kMostGroups / 128; ++k)
            if (part + k * 128 < groups) s += v[k];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[i] += __shfl_xor(s[i], 8);
            s[i] += __shfl_xor(s[i], 16);
            s[i] += __shfl_xor(s[i], 32);
        }
        if ((threadIdx.x & 63) < 8) join[threadIdx.x >> 6][lane] = s;
        __syncthreads();
        if (threadIdx.x < 32 && c0 + threadIdx.x < cols) {
            float all = 0.0f;
#pragma unroll
            for (int w = 0; w < 16; ++w) all += join[w][threadIdx.x / 4][threadIdx.x % 4];
            dweight[c0 + threadIdx.x] = all;
        }
        __syncthreads();   // before the next columns' sums
    }
}

// No rows: no gradient.
__global__ __launch_bounds__(256) void zero_kernel(float* dweight, int32_t cols) {
    const int64_t c = blockIdx.x * int64_t(256) + threadIdx.x;
    if (c < cols) dweight[c] = 0.0f;
}

// A row's threads: a wave up to 2048 columns in bf16, 1024 in f32, where there
// are rows enough to fill the chip with waves, a workgroup otherwise, with one
// vector a lane for each 2048 columns up to 8192 (4000 x 5120 with three: 24.5 us
// against 27.1 with four, its gradients 32.0 against 34.7).  Kernel times in us on
// inputs that repeat, a wave's and a workgroup's: bf16, 28,160 x 1280 45.4 and 51.2, 4096 x 1280 10.7 and
// 11.2, 3000 x 1280 9.2 and 9.1, 1024 x 1280 6.6 and 5.1; f32, 28,160 x 2048 147 and
// 138, 4096 x 1280 15.9 and 15.2, 4096 x 1000 11.7 and 12.4.  (Rows of up to 1024
// columns gain by it sooner: 2048 x 1000 in bf16 5.7 and 7.0, in f32 7.2 and 7.1.)
constexpr int kFewRows = 4096;

bool is_long(int64_t cols) { return cols > 8192; }
bool by_wave(int64_t rows, int64_t cols, int size) {
    return cols <= 512 || (cols <= (size == 2 ? 2048 : 1024) && rows >= kFewRows);
}
// The backward pass holds twice as much a row: up to 1024 columns (28,160 rows in
// bf16, of 1000 in 40.1 us against 46.9 by workgroups, of 600 in 33.6 against 45.8;
// 4096 x 1000 12.5 against 15.4, in f32 17.2 against 17.8).
bool backward_by_wave(int64_t rows, int64_t cols) { return cols <= 1024 && by_wave(rows, cols, 4); }

uint32_t groups_of(int64_t rows, bool wave, int64_t most) {
    const int64_t per = wave ? 4 : 1, g = (rows + per - 1) / per;
    return static_cast<uint32_t>(g < most ? g : most);
}

// A workgroup's share of dweight is a row of floats, written and read again, so
// there are half as many as in the forward pass: 28,160 x 4096 in bf16 in 156 us
// against 171, 1024 x 8192 in 20 against 26.  Shorter rows in bf16, 16 bytes a lane of
// each input, need more of them under way once they are many; with 512 and 1024
// workgroups: 28,160 x 1280 77.7 and 57.2, 10,000 x 1536 28.0 and 25.6, 3000 x 1280
// 14.5 and 14.0, but 2048 x 1280 12.1 and 12.9, 28,160 x 2048 75.9 and 85.8, and in f32
// 28,160 x 1280 112 and 116.
uint32_t backward_groups(int64_t rows, int64_t cols, int size) {
    const bool wave = backward_by_wave(rows, cols);
    const bool more = size == 2 && !wave && cols <= 1792 && rows >= 2560;
    return groups_of(rows, wave, more ? kMostGroups : kMostGroups / 2);
}

template <class T, bool FAR>
int norm_rows(const NormArgs& a, hipStream_t s) {
    const bool wave = by_wave(a.rows, a.cols, sizeof(T));
    const uint32_t g = groups_of(a.rows, wave, kMostGroups);
    if (wave) {
        if (a.cols <= 512) norm_kernel<T, 64, 1, FAR><<<g, 256, 0, s>>>(a);
        else if (a.cols <= 1024) norm_kernel<T, 64, 2, FAR><<<g, 256, 0, s>>>(a);
        else if constexpr (sizeof(T) == 2) norm_kernel<T, 64, 4, FAR><<<g, 256, 0, s>>>(a);
    } else if (a.cols <= 2048) norm_kernel<T, 256, 1, FAR><<<g, 256, 0, s>>>(a);
    else if (a.cols <= 4096) norm_kernel<T, 256, 2, FAR><<<g, 256, 0, s>>>(a);
    else if (a.cols <= 6144) norm_kernel<T, 256, 3, FAR><<<g, 256, 0, s>>>(a);
    else norm_kernel<T, 256, 4, FAR><<<g, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
int norm_launch(const NormArgs& a, hipStream_t s) {
    if (is_long(a.cols)) {
        norm_long_kernel<T><<<groups_of(a.rows, false, kMostGroups), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    const int64_t reads = int64_t(a.rows) * a.cols * sizeof(T) * (a.residual != nullptr ? 2 : 1);
    return past_cache<T>(reads, [&]<bool FAR>(std::bool_constant<FAR>) { return norm_rows<T, FAR>(a, s); });
}

uint32_t across(int64_t cols, int64_t each) {
    const int64_t n = (cols + each - 1) / each;
    return static_cast<uint32_t>(n < kMostAcross ? n : kMostAcross);
}

template <class T, bool FAR, bool MANY>
int norm_backward_rows(const NormBackwardArgs& a, bool wave, uint32_t g, hipStream_t s) {
    if (wave) {
        if (a.cols <= 512) norm_backward_kernel<T, 64, 1, FAR, MANY><<<g, 256, 0, s>>>(a);
        else norm_backward_kernel<T, 64, 2, FAR, MANY><<<g, 256, 0, s>>>(a);
    } else if (a.cols <= 2048) norm_backward_kernel<T, 256, 1, FAR, MANY><<<g, 256, 0, s>>>(a);
    else if (a.cols <= 4096) norm_backward_kernel<T, 256, 2, FAR, MANY><<<g, 256, 0, s>>>(a);
    else if (a.cols <= 6144) norm_backward_kernel<T, 256, 3, FAR, MANY><<<g, 256, 0, s>>>(a);
    else norm_backward_kernel<T, 256, 4, FAR, MANY><<<g, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
int norm_backward_launch(const NormBackwardArgs& a, hipStream_t s) {
    const int groups = norm_backward_groups(a.rows, a.cols, sizeof(T));
    if (a.rows > 0 && is_long(a.cols)) {
        if (a.partial != nullptr)
            norm_dweight_long_kernel<T><<<dim3(across(a.cols, 64), static_cast<uint32_t>(groups)), 256, 0, s>>>(a);
        norm_backward_long_kernel<T><<<groups_of(a.rows, false, kMostGroups), 256, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    } else if (a.rows > 0) {
        const int64_t reads = int64_t(a.rows) * a.cols * sizeof(T) * (a.dh != nullptr ? 3 : 2);
        const bool wave = backward_by_wave(a.rows, a.cols);
        const uint32_t g = backward_groups(a.rows, a.cols, sizeof(T));
        const bool many = a.partial != nullptr && a.rows > int64_t(g) * (wave ? 4 : 1) * kPart;
        const int e = past_cache<T>(reads, [&]<bool FAR>(std::bool_constant<FAR>) {
            return many ? norm_backward_rows<T, FAR, true>(a, wave, g, s) : norm_backward_rows<T, FAR, false>(a, wave, g, s);
        });
        if (e != hipSuccess) return e;
    }
    if (a.dweight != nullptr && groups == 0) {
        zero_kernel<<<static_cast<uint32_t>((int64_t(a.cols) + 255) / 256), 256, 0, s>>>(a.dweight, a.cols);
    } else if (a.dweight != nullptr) {
        sum_partial_kernel<<<across(a.cols, 32), 1024, 0, s>>>(
            a.partial, a.dweight, groups, a.cols);
    }
    return hipGetLastError();
}

}  // namespace

int norm_backward_groups(int64_t rows, int64_t cols, int size) {
    if (rows == 0) return 0;
    if (!is_long(cols)) return static_cast<int>(backward_groups(rows, cols, size));
    const int64_t g = (rows + 3) / 4;
    return static_cast<int>(g < kLongGroups ? g : kLongGroups);
}

int launch_norm(const NormArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? norm_launch<bf16_t>(a, s) : norm_launch<float>(a, s);
}

int launch_norm_backward(const NormBackwardArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? norm_backward_launch<bf16_t>(a, s) : norm_backward_launch<float>(a, s);
}

}  // namespace vp
