// vp_matmul.hip -- out [M][N] = a [M][K] b [N][K]^T of matrices in 8 bits.
//
// Both operands' rows are whole blocks of 128 bytes with zeros past K, so the
// sum runs over whole blocks.  In a 32 x 32 tile of the result, lane l holds
// bytes [32 (l / 32), + 32) of a 64-byte half block of row l % 32; the dot
// product does not depend on the order of the block's columns as long as both
// sides share it.
#include <type_traits>
#include <utility>

#include "vp.h"
#include "vp_fp8_device.h"

namespace vp {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------------------
// Tiles: 4 waves, 2 x 2, each FM x FN squares of 32 x 32 of the result, so a
// workgroup has 64 FM x 64 FN.  Half blocks of 64 columns of both operands go
// from memory to LDS directly, into a ring of SLOTS; a wave's registers run one
// half block ahead of its matrix instructions.  Step H multiplies half block H,
// reads H + 1 from LDS and asks for H + SLOTS where H was, with one barrier at
// its start: H + 1 has arrived, H is in registers everywhere.  A load so has
// the time of SLOTS - 2 steps at least to arrive.
//
// LDS rows are 64 bytes, a quarter of its 64 banks, their four 16-byte pieces
// permuted by the four rows (piece p of row r lies at p ^ (r / 4 % 4)), so the
// 16 lanes that are served together, four groups of four neighbours, read 64
// different banks; the permutation is made by the addresses that the lanes
// fetch from memory.
//
// Small results are bound by what a CU's loads bring, 16 KB a block in 0.25 us
// with tiles of 64 (a ring of 16 half blocks, and half the barriers with the sum
// shared by two sets of waves, were 5 to 40 % slower): 320 x 1280 x 1536 to bf16
// in 6.1 us, 1280 x 1176 x 576 to f32 in 8.1.
// ---------------------------------------------------------------------------

// f(0), f(1), ... f(N - 1) as constants, for loops longer than the compiler unrolls.
template <int N, class F>
__device__ __forceinline__ void each(F&& f) {
    [&]<int... I>(std::integer_sequence<int, I...>) {
        (f(std::integral_constant<int, I>()), ...);
    }(std::make_integer_sequence<int, N>());
}

// A buffer descriptor over `bytes` bytes; loads past them read as zero.
__device__ __forceinline__ i32x4 descriptor(const uint8_t* p, uint32_t bytes) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return i32x4{__builtin_amdgcn_readfirstlane(static_cast<int>(a)),
                 __builtin_amdgcn_readfirstlane(static_cast<int>(a >> 32) & 0xffff),
                 __builtin_amdgcn_readfirstlane(static_cast<int>(bytes)), 0x00027000};
}

// 16 bytes a lane from memory to LDS at `lds` + 16 * lane.  The caller waits
// for it (vmcnt) and meets a barrier before anyone reads them.
__device__ __forceinline__ void load_to_lds(i32x4 from, uint32_t lane_offset, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(lds), "v"(lane_offset), "s"(from), "s"(offset)
                 : "memory", "m0");
}

// The same with 4 bytes a lane.
__device__ __forceinline__ void load_to_lds_word(i32x4 from, uint32_t lane_offset, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
                 :
                 : "s"(lds), "v"(lane_offset), "s"(from), "s"(offset)
                 : "memory", "m0");
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}

// c += x y over 64 columns.  F8: the scaled 8-bit instruction, which takes the
// powers of two as they are.  It cuts the products of 8 neighbouring columns
// toward zero at 2^-13 of the power of two of their largest (256 + 2^-6 is 256
// where both are of one run of 8, and exact where they are not) and adds the runs
// to c in 32 bits.  Results in bf16 are rounded at 2^-9 of themselves afterwards,
// so they take it, at twice the rate of values widened to bf16; results in f32 do
// not.
__device__ __forceinline__ f32x16 multiply8(i32x8 x, i32x8 y, uint32_t sx, uint32_t sy, f32x16 c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 0, 0, 0, static_cast<int>(sx), 0,
                                                           static_cast<int>(sy));
}
// Eight of a lane's values, times 2^e, as bf16: exact for e >= -124 (bf16 has
// no bits below 2^-133) and values below 2^128.
__device__ __forceinline__ bf16x8 widen(int lo, int hi, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

struct TileArgs {
    Fp8View a, b;
    void* out;          // rows of `ld` elements; with splits, [split][M][N] floats
    int64_t ld;
    int32_t tiles_m, tiles_n;
    int32_t blocks;     // of 128 columns, in one split
};

// Place of a workgroup's tile.  Workgroups go round the 8 dies in turn, each
// with an L2 of its own: a die takes a run of consecutive tiles, in columns of
// 8 tiles of M, so that the tiles in flight on it share rows of both operands.
__device__ __forceinline__ uint32_t run_of_die(uint32_t id, uint32_t total) {
    const uint32_t die = id % 8, step = id / 8, per = total / 8, more = total % 8;
    return die * per + (die < more ? die : more) + step;
}
__device__ __forceinline__ void place(uint32_t id, int32_t tiles_m, int32_t tiles_n, int32_t* tm, int32_t* tn) {
    const uint32_t group = 8u * static_cast<uint32_t>(tiles_n);
    const uint32_t g = id / group, first = g * 8;
    const uint32_t high = min(8u, static_cast<uint32_t>(tiles_m) - first), in = id - g * group;
    *tm = static_cast<int32_t>(first + in % high);
    *tn = static_cast<int32_t>(in / high);
}

template <class T>
__device__ __forceinline__ f32x4 multiply16(i32x8 x, i32x8 y, uint32_t sx, uint32_t sy, f32x4 c, T) {
    if constexpr (T::value) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 0, 0, 0, static_cast<int>(sx), 0,
                                                                static_cast<int>(sy));
    } else {
        const float fx = scale_value(sx), fy = scale_value(sy);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(x[2 * i], x[2 * i + 1], fx),
                                                        widen(y[2 * i], y[2 * i + 1], fy), c, 0, 0, 0);
        return c;
    }
}

// A wave's ROWS x COLS of the result, bf16 in LDS, to memory.
template <int ROWS, int COLS>
__device__ __forceinline__ void store_rows(const TileArgs& p, const uint8_t* from, int pitch, int64_t m0, int64_t n0,
                                           int lane) {
    bf16_t* out = static_cast<bf16_t*>(p.out);
    constexpr int kLanes = COLS / 8;                // of 8 values for a row
    if (n0 + COLS <= p.b.rows) {
#pragma unroll
        for (int i = 0; i < ROWS * kLanes / 64; ++i) {
            const int row = i * (64 / kLanes) + lane / kLanes, at = (lane % kLanes) * 8;
            if (m0 + row < p.a.rows)
                *reinterpret_cast<u32x4_any*>(out + (m0 + row) * p.ld + n0 + at) =
                    *reinterpret_cast<const u32x4*>(from + row * pitch + at * 2);
        }
    } else {
        constexpr int kAcross = COLS < 64 ? COLS : 64;
        for (int row = lane / kAcross; row < ROWS; row += 64 / kAcross)
            for (int at = lane % kAcross; at < COLS; at += kAcross)
                if (m0 + row < p.a.rows && n0 + at < p.b.rows)
                    out[(m0 + row) * p.ld + n0 + at] = *reinterpret_cast<const bf16_t*>(from + row * pitch + at * 2);
    }
}

template <bool F8, class Out, int FM, int FN, int SLOTS>
__global__ __launch_bounds__(256, 1) void tile_kernel(TileArgs p) {
    constexpr int kRowsA = 64 * FM, kRowsB = 64 * FN;
    constexpr int kBytesA = kRowsA * 64, kSlot = (kRowsA + kRowsB) * 64;
    constexpr int kScales = (kRowsA + kRowsB) * 4;              // four blocks' scales of every row
    constexpr int kLoop = SLOTS * kSlot + 2 * kScales;
    constexpr int kPitch = 64 * FN + 16;                        // bytes a row of a wave's bf16 result in LDS
    constexpr int kOut = sizeof(Out) == 2 ? 4 * 32 * FM * kPitch : 0;
    constexpr int kFetches = FM + FN;                           // of a wave for a half block
    static_assert(SLOTS == 4 || SLOTS == 8);                    // at most 8: see fetch_scales
    __shared__ __align__(1024) uint8_t lds[kLoop > kOut ? kLoop : kOut];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, r = lane & 31, half = lane >> 5;
    int32_t tm, tn;
    place(run_of_die(blockIdx.x, gridDim.x), p.tiles_m, p.tiles_n, &tm, &tn);
    const int64_t m0 = int64_t(tm) * kRowsA, n0 = int64_t(tn) * kRowsB;
    const int32_t total = static_cast<int32_t>(p.a.ld / kBlock);
    const int32_t first = blockIdx.y * p.blocks, nk = min(p.blocks, total - first);

    f32x16 c[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) c[i][j][e] = 0.0f;

    if (nk > 0) {
        // rows past the end fetch the last one; their results are not stored
        const int32_t left_a = static_cast<int32_t>(min(int64_t(kRowsA), p.a.rows - m0));
        const int32_t left_b = static_cast<int32_t>(min(int64_t(kRowsB), p.b.rows - n0));
        i32x4 from_a = descriptor(p.a.q + m0 * p.a.ld, static_cast<uint32_t>(left_a * p.a.ld));
        i32x4 from_b = descriptor(p.b.q + n0 * p.b.ld, static_cast<uint32_t>(left_b * p.b.ld));
        uint32_t fetch_a[FM], fetch_b[FN];
        const uint32_t piece = ((lane & 3) ^ (lane >> 4)) * 16;
#pragma unroll
        for (int i = 0; i < FM; ++i)
            fetch_a[i] = min((wave * FM + i) * 16 + (lane >> 2), left_a - 1) * static_cast<uint32_t>(p.a.ld) + piece;
#pragma unroll
        for (int i = 0; i < FN; ++i)
            fetch_b[i] = min((wave * FN + i) * 16 + (lane >> 2), left_b - 1) * static_cast<uint32_t>(p.b.ld) + piece;
        const uint32_t base = lds_address(lds);
        auto fetch = [&](int i, int32_t h) {   // piece i of this wave's share of half block h
            const uint32_t to = base + (h & (SLOTS - 1)) * kSlot;
            const uint32_t at = h < 2 * nk ? static_cast<uint32_t>(first) * kBlock + h * 64 : 0;
            if (i < FM) load_to_lds(from_a, fetch_a[i], at, to + (wave * FM + i) * 1024);
            else load_to_lds(from_b, fetch_b[i - FM], at, to + kBytesA + (wave * FN + i - FM) * 1024);
        };
        auto end_at = [&](int32_t h) {
            if (h >= 2 * nk) {   // nothing there: empty buffers, whose loads touch no memory and count all the same
                from_a[2] = 0;
                from_b[2] = 0;
            }
        };

        // Scales: words of four blocks, 64 rows a load, to LDS like the blocks.  Word w goes before the first
        // block that it covers, so it has arrived when that block has; two words are held, and the one that a
        // load replaces was last used at least 4 >= SLOTS / 2 blocks before.
        const uint8_t *sa = p.a.scale + (p.a.block == 1 ? m0 : m0 / kBlock) * p.a.sld;
        const uint8_t *sb = p.b.scale + (p.b.block == 1 ? n0 : n0 / kBlock) * p.b.sld;
        const i32x4 scales_a = descriptor(sa, static_cast<uint32_t>((p.a.block == 1 ? left_a : (left_a - 1) / kBlock + 1) * p.a.sld));
        const i32x4 scales_b = descriptor(sb, static_cast<uint32_t>((p.b.block == 1 ? left_b : (left_b - 1) / kBlock + 1) * p.b.sld));
        uint32_t fetch_s[(FM + FN + 3) / 4];
#pragma unroll
        for (int i = 0; i < (FM + FN + 3) / 4; ++i) {
            const int k = i * 4 + wave;        // 64 rows: k < FM of a, then of b
            const int row = (k < FM ? k : k - FM) * 64 + lane;
            const bool is_a = k < FM;
            const uint32_t at = min(row, (is_a ? left_a : left_b) - 1) / (is_a ? p.a.block : p.b.block);
            fetch_s[i] = at * static_cast<uint32_t>(is_a ? p.a.sld : p.b.sld);
        }
        auto fetch_scales = [&](int32_t word) {
#pragma unroll
            for (int i = 0; i < (FM + FN + 3) / 4; ++i) {
                const int k = i * 4 + wave;
                const uint32_t to = base + SLOTS * kSlot + (word & 1) * kScales + k * 256;
                if (k < FM) load_to_lds_word(scales_a, fetch_s[i], word * 4, to);
                else if (k < FM + FN) load_to_lds_word(scales_b, fetch_s[i], word * 4, to);
            }
        };
        const uint32_t scale_at = SLOTS * kSlot + r * 4;
        uint32_t scale_a[FM], scale_b[FN], word_a[FM], word_b[FN];
        auto read_scales = [&](int32_t kb) {   // the words of block kb
            const uint8_t* from = lds + scale_at + ((kb >> 2) & 1) * kScales;
#pragma unroll
            for (int i = 0; i < FM; ++i) word_a[i] = *reinterpret_cast<const uint32_t*>(from + (wm * FM + i) * 128);
#pragma unroll
            for (int j = 0; j < FN; ++j)
                word_b[j] = *reinterpret_cast<const uint32_t*>(from + kRowsA * 4 + (wn * FN + j) * 128);
        };
        auto use_scales = [&](int32_t kb) {   // its byte lowest
#pragma unroll
            for (int i = 0; i < FM; ++i) scale_a[i] = word_a[i] >> ((kb & 3) * 8);
#pragma unroll
            for (int j = 0; j < FN; ++j) scale_b[j] = word_b[j] >> ((kb & 3) * 8);
        };

        // a lane's two pieces of a half block: 16-byte pieces 2 (lane / 32) and the next, of its row
        const uint32_t at0 = r * 64 + (((half * 2) ^ ((r >> 2) & 3)) * 16);
        i32x8 xa[2][FM], xb[2][FN];
        auto read = [&](int set, int f, int32_t h) {   // operand f of half block h
            const uint8_t* from = lds + (h & (SLOTS - 1)) * kSlot +
                                  (f < FM ? (wm * FM + f) * 2048 : kBytesA + (wn * FN + f - FM) * 2048);
            const i32x4 lo = *reinterpret_cast<const i32x4*>(from + at0);
            const i32x4 hi = *reinterpret_cast<const i32x4*>(from + (at0 ^ 16));
            const i32x8 x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            if (f < FM) xa[set][f] = x;
            else xb[set][f - FM] = x;
        };
        // for every wave: its reads of LDS are done, and its fetches, but for the last `LATER` half blocks', have arrived
        auto meet = [&]<int LATER>(std::integral_constant<int, LATER>) {
            constexpr int n = LATER * kFetches;
            static_assert(n < 64);
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | (7 << 4));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        auto multiply = [&](int set, int q) {
            const int i = q / FN, j = q % FN;
            if constexpr (F8) {
                const uint32_t ea = scale_a[i], eb = scale_b[j];
                // bf16 results: rows of the tile are n, so that a lane holds runs of n
                if constexpr (sizeof(Out) == 2) c[i][j] = multiply8(xb[set][j], xa[set][i], eb, ea, c[i][j]);
                else c[i][j] = multiply8(xa[set][i], xb[set][j], ea, eb, c[i][j]);
            } else {
                const float ea = scale_value(scale_a[i] & 255), eb = scale_value(scale_b[j] & 255);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    c[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        widen(xa[set][i][2 * k], xa[set][i][2 * k + 1], ea),
                        widen(xb[set][j][2 * k], xb[set][j][2 * k + 1], eb), c[i][j], 0, 0, 0);
            }
        };

        fetch_scales(first >> 2);
#pragma unroll
        for (int h = 0; h < SLOTS; ++h) {
            if (h > 0 && h % 2 == 0 && h < 2 * nk && ((first + h / 2) & 3) == 0) fetch_scales((first + h / 2) >> 2);
            end_at(h);
#pragma unroll
            for (int i = 0; i < kFetches; ++i) fetch(i, h);
        }
        meet(std::integral_constant<int, SLOTS - 1>());
        read_scales(first);
        use_scales(first);
#pragma unroll
        for (int f = 0; f < FM + FN; ++f) read(0, f, 0);

        for (int32_t t = 0; t < nk; ++t) {
            const int32_t later = first + t + SLOTS / 2;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int32_t h = 2 * t + s;
                meet(std::integral_constant<int, SLOTS - 2>());
                if (s == 0 && (later & 3) == 0 && t + SLOTS / 2 < nk) fetch_scales(later >> 2);
                end_at(h + SLOTS);
                if (s == 1) read_scales(first + t + 1);
#pragma unroll
                for (int q = 0; q < FM * FN; ++q) {
                    multiply(s, q);
#pragma unroll
                    for (int f = q * (FM + FN) / (FM * FN); f < (q + 1) * (FM + FN) / (FM * FN); ++f) read(1 - s, f, h + 1);
#pragma unroll
                    for (int f = q * kFetches / (FM * FN); f < (q + 1) * kFetches / (FM * FN); ++f) fetch(f, h + SLOTS);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            use_scales(first + t + 1);
        }
        meet(std::integral_constant<int, 0>());
    }

    const int64_t wave_m = m0 + wm * 32 * FM, wave_n = n0 + wn * 32 * FN;
    if constexpr (sizeof(Out) == 2) {
        // a lane has, for row r, n = 8 q + 4 (lane / 32) + 0..3: through LDS, to store whole rows
        uint8_t* mine = lds + wave * 32 * FM * kPitch;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                    bf16x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = static_cast<bf16_t>(c[i][j][q * 4 + e]);
                    *reinterpret_cast<bf16x4*>(mine + (i * 32 + r) * kPitch + (j * 32 + q * 8 + half * 4) * 2) = v;
                }
        store_rows<32 * FM, 32 * FN>(p, mine, kPitch, wave_m, wave_n, lane);
    } else {
        // a lane has column r of 16 rows: 32 lanes store 128 bytes of a row
        float* out = static_cast<float*>(p.out) + (gridDim.y > 1 ? blockIdx.y * int64_t(p.a.rows) * p.ld : 0);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int64_t m = wave_m + i * 32 + (e & 3) + 8 * (e >> 2) + 4 * half;
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const int64_t n = wave_n + j * 32 + r;
                    if (m < p.a.rows && n < p.b.rows) out[m * p.ld + n] = c[i][j][e];
                }
            }
    }
}

// ---------------------------------------------------------------------------
// Large results: 256 x 256 a workgroup, 128 x 128 a wave, four by four squares.
// LDS holds two whole blocks, so that every fetch is of whole 128-byte lines
// (half blocks, 64 bytes a row, take a fifth longer here), and a wave's registers
// run half a block ahead:
//   first half:  multiply half 0 of block u, read half 1 of it from LDS;
//   one barrier: block u + 1 has arrived, block u is in registers everywhere;
//   second half: multiply half 1, read half 0 of block u + 1, and ask for
//                block u + 2 where block u was.
// LDS rows are 128 bytes, half of its 64 banks, piece p of row r at p ^ (r / 2 %
// 8): the 16 lanes that are served together read 64 banks.
//
// A workgroup's fetches go through its tiles without a pause: the blocks of all of
// them are one sequence, so while a tile's results are stored, through LDS, where
// they are turned round to whole lines, the next tile's first blocks are on their
// way, and the writes, 33 MB for each round of tiles, go on beside its arithmetic.
// The matrix cores wait while the results pass through LDS, about 6 us a round.
//
// Bound by the matrix cores: 8192^3 to bf16 in 418 to 450 us, 2.4 to 2.6 PFLOP/s,
// their instructions busy 71 % of the time at the 1.6 to 1.8 GHz that the power
// limit leaves; 4096 x 4096 x 8190 to f32, widened, in 193 us, busy 78 %.
// ---------------------------------------------------------------------------
struct Piece {           // of the work: a tile, and of its sum blocks [first, first + nk)
    uint32_t item;       // of tiles * splits; past the end: none
    int32_t tm, tn, split;
    int32_t first, nk;
};

// Every piece has two blocks at least.
// Without F8 the values are widened to bf16, a quarter of a half block (8 values
// a lane) at a time, one quarter ahead of the instructions: 16 x 32 cycles, in
// which 32 conversions stand, so the registers hold two quarters widened.
// FAR: the result is more than the memory-side cache keeps and does not go
// through it (to bf16, 28,160 x 4096 x 1280 in 142 us, otherwise 151, 89,600 x 1280 x
// 1536 in 174 and 190; to f32 the same alone, with the norm that reads the result 362
// and 377; results of 32 to 128 MiB 1 to 6 % slower for their reader).
template <class Out, bool F8, bool FAR>
__global__ __launch_bounds__(256, 1) void big_kernel(TileArgs p, int32_t splits) {
    constexpr int kBytes = 256 * 128;                           // of an operand's block
    constexpr int kScales = 512 * 4, kScaleAt = 4 * kBytes;     // a word of scales of every row
    constexpr int kSize = sizeof(Out);
    constexpr int kNoneAt = kScaleAt + 2 * kScales;             // for what no one reads
    constexpr int kPitch = 128 + 16, kOutAt = kNoneAt + kScales;   // of a wave's results on their way out
    __shared__ __align__(1024) uint8_t lds[kOutAt + 4 * 32 * kPitch];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, r = lane & 31, half = lane >> 5;
    const uint32_t tiles = static_cast<uint32_t>(p.tiles_m) * static_cast<uint32_t>(p.tiles_n);
    const uint32_t items = tiles * static_cast<uint32_t>(splits);
    const int32_t total = static_cast<int32_t>(p.a.ld / kBlock);

    auto locate = [&](uint32_t item) {
        Piece x{item, 0, 0, 0, 0, 0};
        if (item >= items) return x;
        const uint32_t id = run_of_die(item, items);
        x.split = static_cast<int32_t>(id / tiles);
        place(id - x.split * tiles, p.tiles_m, p.tiles_n, &x.tm, &x.tn);
        x.first = x.split * p.blocks;
        x.nk = min(p.blocks, total - x.first);
        return x;
    };
    // Rows past the end lie past a descriptor's end, whose loads read zeros; so does all of no piece's.
    auto rows_of = [&](const Fp8View& f, int32_t tile, const Piece& x) {
        const int64_t r0 = tile * int64_t(256);
        const int64_t left = min(int64_t(256), f.rows - r0);
        return descriptor(f.q + r0 * f.ld, x.item < items ? static_cast<uint32_t>(left * f.ld) : 0u);
    };
    auto scales_of = [&](const Fp8View& f, int32_t tile, const Piece& x) {
        const int64_t r0 = tile * int64_t(256), left = min(int64_t(256), f.rows - r0);
        const int64_t groups = f.block == 1 ? left : (left - 1) / kBlock + 1;
        return descriptor(f.scale + (f.block == 1 ? r0 : r0 / kBlock) * f.sld,
                          x.item < items ? static_cast<uint32_t>(groups * f.sld) : 0u);
    };

    uint32_t fetch_a[8], fetch_b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = (wave * 8 + i) * 8 + (lane >> 3);
        const uint32_t piece = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
        fetch_a[i] = row * static_cast<uint32_t>(p.a.ld) + piece;
        fetch_b[i] = row * static_cast<uint32_t>(p.b.ld) + piece;
    }
    const uint32_t base = lds_address(lds);
    // Piece i of this wave's share of the u-th block of the sequence, block kb of its rows.
    auto fetch = [&](i32x4 from, int i, uint32_t u, int32_t kb) {
        load_to_lds(from, i < 8 ? fetch_a[i & 7] : fetch_b[i & 7], static_cast<uint32_t>(kb) * kBlock,
                    base + (i < 8 ? 0 : 2 * kBytes) + (u & 1) * kBytes + (wave * 8 + (i & 7)) * 1024);
    };
    // Scales: words of four blocks, 64 rows a load, with the first block that each covers; with the others a load
    // that touches no memory.  The words of a workgroup's sequence take two places in turn: the one that a new word
    // takes was last used by the block before the last one that was fetched.
    const uint32_t scale_a_at = static_cast<uint32_t>((wave * 64 + lane) / p.a.block) * static_cast<uint32_t>(p.a.sld);
    const uint32_t scale_b_at = static_cast<uint32_t>((wave * 64 + lane) / p.b.block) * static_cast<uint32_t>(p.b.sld);
    auto fetch_scales = [&](i32x4 from, bool is_b, bool any, uint32_t word, int32_t kb) {
        from[2] = any ? from[2] : 0;
        load_to_lds_word(from, is_b ? scale_b_at : scale_a_at, any ? static_cast<uint32_t>(kb >> 2) * 4 : 0u,
                         base + (any ? kScaleAt + (word & 1) * kScales : kNoneAt) + (is_b ? 1024 : 0) + wave * 256);
    };
    uint32_t scale_a[4], scale_b[4], word_a[4], word_b[4];
    auto read_scales = [&](uint32_t word) {
        const uint8_t* from = lds + kScaleAt + (word & 1) * kScales + r * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            word_a[i] = *reinterpret_cast<const uint32_t*>(from + (wm * 4 + i) * 128);
            word_b[i] = *reinterpret_cast<const uint32_t*>(from + 1024 + (wn * 4 + i) * 128);
        }
    };
    // a lane's two pieces of half h of a block: 16-byte pieces 4 h + 2 (lane / 32) and the next, of its row
    const uint32_t at0 = r * 128 + ((half * 2) ^ ((r >> 1) & 7)) * 16;
    i32x8 xa[2][4], xb[2][4];
    auto read = [&](int h, int f, uint32_t u) {   // square f of a, or f - 4 of b, half h of the u-th block
        const uint8_t* from = lds + (f < 4 ? wm * 16384 + f * 4096 : 2 * kBytes + wn * 16384 + (f - 4) * 4096) + (u & 1) * kBytes;
        const i32x4 lo = *reinterpret_cast<const i32x4*>(from + (at0 ^ (h * 64)));
        const i32x4 hi = *reinterpret_cast<const i32x4*>(from + (at0 ^ (h * 64 + 16)));
        const i32x8 x{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        if (f < 4) xa[h][f] = x;
        else xb[h][f - 4] = x;
    };
    // for every wave: its reads of LDS are done and its fetches have arrived
    auto meet = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(7 << 4);   // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    // Results: squares' rows are n, so a lane has, for row r of a square, n = 8 q + 4 half + 0..3, q = 0..3.
    f32x16 c[4][4];
    // A wave stores 32 rows of 128 bytes at a time, turned round in LDS so that whole lines go out (straight from
    // the registers, 16 bytes a lane, L2 had eight times the requests).
    uint8_t* mine = lds + kOutAt + wave * 32 * kPitch;
    const uint32_t row_at = ((wm * 128 + (lane >> 3)) * static_cast<uint32_t>(p.ld) + wn * 128) * kSize;
    constexpr int kRun = 16 / kSize, kAcross = 128 / kSize;   // values of a lane's store, of a row at a time
    auto store_tile = [&](const Piece& x) {
        const int64_t m0 = x.tm * int64_t(256), n0 = x.tn * int64_t(256);
        const int64_t left_m = min(int64_t(256), p.a.rows - m0);
        // what a row holds beyond N is the caller's, or, where the sum is in pieces, the workspace's own padding
        const int64_t left = min(int64_t(256), (splits > 1 ? p.ld : p.b.rows) - n0);
        const int32_t left_n = static_cast<int32_t>(left) - wn * 128;
        const auto rows = __builtin_amdgcn_make_buffer_rsrc(
            static_cast<uint8_t*>(p.out) + ((x.split * int64_t(p.a.rows) + m0) * p.ld + n0) * kSize, 0,
            static_cast<uint32_t>(((left_m - 1) * p.ld + left) * kSize), 0x00027000);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < 128; n += kAcross) {
#pragma unroll
                for (int j = n / 32; j < (n + kAcross) / 32; ++j) {
                    asm volatile("" : "+a"(c[i][j]));   // one square's values at a time in registers
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint8_t* to = mine + r * kPitch + (j * 32 - n + q * 8 + half * 4) * kSize;
                        if constexpr (sizeof(Out) == 2) {
                            typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                            bf16x4 v;
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = static_cast<bf16_t>(c[i][j][q * 4 + e]);
                            *reinterpret_cast<bf16x4*>(to) = v;
                        } else {
                            *reinterpret_cast<f32x4*>(to) =
                                f32x4{c[i][j][q * 4], c[i][j][q * 4 + 1], c[i][j][q * 4 + 2], c[i][j][q * 4 + 3]};
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {   // 8 rows each
                    const u32x4 v = *reinterpret_cast<const u32x4*>(mine + (k * 8 + (lane >> 3)) * kPitch + (lane & 7) * 16);
                    // values past the last row or column go past the descriptor's end, where nothing is stored
                    const int at = n + (lane & 7) * kRun;
                    const uint32_t to = row_at + ((i * 32 + k * 8) * static_cast<uint32_t>(p.ld) + at) * kSize;
                    __builtin_amdgcn_raw_buffer_store_b128(v, rows, at + kRun <= left_n ? to : 0x80000000u, 0,
                                                           FAR ? 2 : 0);   // nontemporal
                }
            }
    };

    // The next fetches are of block at, two blocks ahead of the arithmetic; they go over to the next piece in the
    // step before the last of this one.
    Piece now = locate(blockIdx.x);
    i32x4 from_a = rows_of(p.a, now.tm, now), from_b = rows_of(p.b, now.tn, now);
    i32x4 from_sa = scales_of(p.a, now.tm, now), from_sb = scales_of(p.b, now.tn, now);
    int32_t at = now.first + 1, before = at;   // before: the block that was fetched last, of word `held`
    uint32_t word = 0, held = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const bool any = u == 0 || (at & 3) == 0;
        word += u == 1 && any;
        fetch_scales(from_sa, false, any, word, now.first + u);
        fetch_scales(from_sb, true, any, word, now.first + u);
#pragma unroll
        for (int i = 0; i < 16; ++i) fetch(i < 8 ? from_a : from_b, i, u, now.first + u);
    }
    held = word;
    meet();
    read_scales(0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        scale_a[i] = word_a[i] >> ((now.first & 3) * 8);
        scale_b[i] = word_b[i] >> ((now.first & 3) * 8);
    }
#pragma unroll
    for (int f = 0; f < 8; ++f) read(0, f, 0);
    // Widened quarters k and k + 1, and the scales that they take.
    bf16x8 wa[2][4], wb[2][4];
    float widen_a[4], widen_b[4];
    auto widen_scales = [&](uint32_t shift) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            widen_a[i] = scale_value((word_a[i] >> shift) & 255);
            widen_b[i] = scale_value((word_b[i] >> shift) & 255);
        }
    };
    auto widen_square = [&](int f, int h, int k) {
        if (f < 4) wa[k & 1][f] = widen(xa[h][f][2 * k], xa[h][f][2 * k + 1], widen_a[f]);
        else wb[k & 1][f - 4] = widen(xb[h][f - 4][2 * k], xb[h][f - 4][2 * k + 1], widen_b[f - 4]);
    };
    if constexpr (!F8) {
        widen_scales((now.first & 3) * 8);
#pragma unroll
        for (int f = 0; f < 8; ++f) widen_square(f, 0, 0);
    }

    for (uint32_t u = 0;;) {   // pieces
        const Piece next = locate(now.item + gridDim.x);
        const i32x4 next_a = rows_of(p.a, next.tm, next), next_b = rows_of(p.b, next.tn, next);
        const i32x4 next_sa = scales_of(p.a, next.tm, next), next_sb = scales_of(p.b, next.tn, next);
        // Where nothing follows, both of the last two fetches are of block 0 of empty buffers: their size less an
        // offset, which is what a load's address is held against, stays 0.
        const int32_t second = next.item < items ? 1 : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) c[i][j][e] = 0.0f;

        // A step is one block: 32 instructions of 64 cycles (widened: 128 of 32); what else there is to do stands
        // between them, where it costs nothing.  No branch in it: one would let the compiler sink the
        // multiplications past it.
        for (int32_t left = now.nk; left > 0; --left, ++u) {
            const bool over = left == 2;
            bool any = false;
            auto move_on = [&](int part) {   // the next fetches' place
                if (part == 0) {
                    at = over ? next.first : at + (left == 1 ? second : 1);
                    any = over || (at & 3) == 0;
                    word += any;
                }
#pragma unroll
                for (int e = 0; e < 3; ++e) {
                    if (part == 1) from_a[e] = over ? next_a[e] : from_a[e];
                    if (part == 2) from_b[e] = over ? next_b[e] : from_b[e];
                    if (part == 3) from_sa[e] = over ? next_sa[e] : from_sa[e];
                    if (part == 4) from_sb[e] = over ? next_sb[e] : from_sb[e];
                }
            };
            uint32_t shift = 0;
            auto turn = [&]() {   // to the second half
                meet();
                read_scales(held);
                held = word;
                shift = (before & 3) * 8;
                before = at;
            };
            if constexpr (F8) {
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int i = q / 4, j = q % 4;
                    c[i][j] = multiply8(xb[0][j], xa[0][i], scale_b[j], scale_a[i], c[i][j]);
                    if (q < 8) read(1, q, u);
                    if (q >= 8 && q < 13) move_on(q - 8);
                    __builtin_amdgcn_sched_barrier(0);
                }
                turn();
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int i = q / 4, j = q % 4;
                    c[i][j] = multiply8(xb[1][j], xa[1][i], scale_b[j], scale_a[i], c[i][j]);
                    if (q < 8) read(0, q, u + 1);
                    fetch(q < 8 ? from_a : from_b, q, u + 2, at);
                    if (q == 8) fetch_scales(from_sa, false, any, word, at);
                    if (q == 9) fetch_scales(from_sb, true, any, word, at);
                    // each after its last use, and not before its word is there
                    auto byte = [&](uint32_t& word) {
                        asm volatile("" : "+v"(word));
                        return word >> shift;
                    };
                    if (q == 7 || q == 8) scale_a[q - 7] = byte(word_a[q - 7]);
                    if (q == 11 || q == 15) scale_a[i] = byte(word_a[i]);
                    if (q >= 12) scale_b[j] = byte(word_b[j]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                auto half_step = [&]<int H>(std::integral_constant<int, H>) {
                    each<64>([&]<int S>(std::integral_constant<int, S>) {
                        constexpr int k = S / 16, q = S % 16, i = q / 4, j = q % 4;
                        c[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[k & 1][j], wa[k & 1][i], c[i][j], 0, 0, 0);
                        if constexpr (S % 5 == 0 && S < 40) read(1 - H, S / 5, u + H);
                        if constexpr (H == 0 && S >= 40 && S < 45) move_on(S - 40);
                        if constexpr (H == 1 && S % 3 == 0 && S < 48) fetch(S < 24 ? from_a : from_b, S / 3, u + 2, at);
                        if constexpr (H == 1 && S == 49) fetch_scales(from_sa, false, any, word, at);
                        if constexpr (H == 1 && S == 52) fetch_scales(from_sb, true, any, word, at);
                        if constexpr (H == 1 && S == 48) {   // this block's last quarter is widened
#pragma unroll
                            for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(word_a[e]), "+v"(word_b[e]));
                            widen_scales(shift);
                        }
                        if constexpr (q % 2 == 1) widen_square(q / 2, k < 3 ? H : 1 - H, (k + 1) & 3);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                };
                half_step(std::integral_constant<int, 0>());
                turn();
                half_step(std::integral_constant<int, 1>());
            }
        }
        store_tile(now);
        if (next.item >= items) break;
        now = next;
    }
}

// ---------------------------------------------------------------------------
// Few rows, or a small result: W waves take the same 16 FM x 16 FN of it, each
// every W-th block of 128 columns, straight from memory to registers, and join
// their sums through LDS in order.  The chain of dependent steps is K / (128 W)
// long instead of K / 128, and 4 lanes read a row's whole 128-byte line.  Bound
// by the latency of those steps and by what a CU's loads in flight bring: 1 x
// 4096 x 4096 in 5.2 us (3.2 TB/s of weights, launch included), 77 x 1001 x
// 1176 to f32 in 7.0.
// ---------------------------------------------------------------------------
template <bool F8, class Out, int FM, int FN, int W>
__global__ __launch_bounds__(64 * W) void wave_kernel(TileArgs p) {
    constexpr int kM = 16 * FM, kN = 16 * FN, kAhead = FM + FN > 4 ? 2 : 4;
    __shared__ float join[W][kM][kN + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int32_t tn = static_cast<int32_t>(blockIdx.x / static_cast<uint32_t>(p.tiles_m));
    const int32_t tm = static_cast<int32_t>(blockIdx.x - static_cast<uint32_t>(tn) * p.tiles_m);
    const int64_t m0 = int64_t(tm) * kM, n0 = int64_t(tn) * kN;
    const int32_t nk = p.blocks;

    const uint8_t *a[FM], *b[FN], *sa[FM], *sb[FN];
    f32x4 c[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) {   // rows past the end read the last one; their results are not stored
        const int64_t row = min(m0 + i * 16 + r, int64_t(p.a.rows) - 1);
        a[i] = p.a.q + row * p.a.ld + g * 32;
        sa[i] = p.a.scale + (p.a.block == 1 ? row : row / kBlock) * p.a.sld;
#pragma unroll
        for (int j = 0; j < FN; ++j) c[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t row = min(n0 + j * 16 + r, int64_t(p.b.rows) - 1);
        b[j] = p.b.q + row * p.b.ld + g * 32;
        sb[j] = p.b.scale + (p.b.block == 1 ? row : row / kBlock) * p.b.sld;
    }
    for (int32_t k0 = wave; k0 < nk; k0 += W * kAhead) {
        i32x8 xa[kAhead][FM], xb[kAhead][FN];
        uint32_t ea[kAhead][FM], eb[kAhead][FN];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            // past the end: the last block again, not multiplied below
            const int32_t k = min(k0 + u * W, nk - 1);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                xb[u][j] = *reinterpret_cast<const i32x8*>(b[j] + int64_t(k) * kBlock);
                eb[u][j] = sb[j][k];
            }
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                xa[u][i] = *reinterpret_cast<const i32x8*>(a[i] + int64_t(k) * kBlock);
                ea[u][i] = sa[i][k];
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (k0 + u * W < nk) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        c[i][j] = multiply16(xa[u][i], xb[u][j], ea[u][i], eb[u][j], c[i][j], std::bool_constant<F8>());
            }
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) join[wave][i * 16 + g * 4 + e][j * 16 + r] = c[i][j][e];
    __syncthreads();
    for (int at = threadIdx.x; at < kM * kN; at += 64 * W) {
        const int m = at / kN, n = at % kN;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) sum += join[w][m][n];
        if (m0 + m < p.a.rows && n0 + n < p.b.rows)
            static_cast<Out*>(p.out)[(m0 + m) * p.ld + n0 + n] = static_cast<Out>(sum);
    }
}

// Rows of the splits' floats are whole eights apart.
constexpr int64_t partial_ld(int64_t cols) { return (cols + 7) / 8 * 8; }

// out = the sum of the splits' [M][partial_ld] floats, in order, four a thread.
template <class Out>
__global__ __launch_bounds__(256) void join_kernel(const float* partial, Out* out, int64_t ld, int64_t rows,
                                                   int32_t cols, int32_t splits) {
    const int32_t fours = static_cast<int32_t>(partial_ld(cols) / 4);
    const int64_t size = rows * fours;
    for (int64_t at = blockIdx.x * int64_t(256) + threadIdx.x; at < size; at += gridDim.x * int64_t(256)) {
        const f32x4* from = reinterpret_cast<const f32x4*>(partial) + at;
        f32x4 sum = *from;
        for (int s = 1; s < splits; ++s) sum += from[s * size];
        const int64_t m = at / fours;
        const int32_t n = static_cast<int32_t>(at - m * fours) * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < cols) out[m * ld + n + i] = static_cast<Out>(sum[i]);
    }
}

template <class Out>
int join_launch(const MatmulArgs& a, Out* out, int splits, hipStream_t stream) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t size = int64_t(a.a.rows) * partial_ld(a.b.rows), wgs = (size + 1023) / 1024;
    join_kernel<Out><<<static_cast<uint32_t>(wgs < 0xfffff ? wgs : 0xfffff), 256, 0, stream>>>(
        a.partial, out, a.ld, a.a.rows, a.b.rows, splits);
    return hipGetLastError();
}

TileArgs tile_args(const MatmulArgs& a, int rows_m, int rows_n) {
    TileArgs p{};
    p.a = a.a;
    p.b = a.b;
    p.out = a.out;
    p.ld = a.ld;
    p.tiles_m = static_cast<int32_t>((int64_t(a.a.rows) + rows_m - 1) / rows_m);
    p.tiles_n = static_cast<int32_t>((int64_t(a.b.rows) + rows_n - 1) / rows_n);
    p.blocks = static_cast<int32_t>(a.a.ld / kBlock);
    return p;
}

// How a product is cut: tiles of 64 F x 64 F with the sum in `splits` pieces,
// or F = 0: 16 FM x 16 FN by waves that split the sum among them; F < 0: more
// tiles than a launch takes.
struct Cut {
    int f, fm, fn, splits;
};

// The cut whose estimated time is least.
// Tiles: a round of workgroups (one a CU for 256, two for 128 and 64) takes
// the time of a step for each block of its piece, and a start and an end; a
// step takes less where the chip is not full.  Sums in pieces add a launch and
// the time to write and read their floats at 5 TB/s.
// Waves: what a CU has to load, at the 26 GB/s that one workgroup's loads in
// flight reach (to f32, 16 x 4096 x 4096 in 7.1 us, 64 x 4096 x 4096 in 12.4, where
// 64-tiles in four pieces take 10.4 and 12.0; 128 x 4096 x 4096 in 17.9 and 17.6).
// The steps (us) are measured, with 8-bit and, for f32 results, widened
// products.  Over 26 shapes from 1 x 1024 x 1024 to 28,160 x 1280 x 1536, in both
// types, 43 of the 52 take the fastest of the 6 to 26 cuts that they allow, and the
// others one within 10 % of it (the most: 128 x 4096 x 4096 to f32, 17.6 us, 16.1
// by 64-tiles in two pieces).
Cut choose(int64_t m, int64_t n, int64_t k, bool f8) {
    struct Tile {
        int f, slots;
        double alone8, full8, alone32, full32, ends;
    };
    constexpr Tile tiles[] = {{4, 256, 1.25, 1.63, 2.3, 2.8, 6.0},
                              {2, 512, 0.65, 1.08, 1.0, 1.77, 3.0},
                              {1, 512, 0.34, 0.47, 0.5, 0.68, 2.5}};
    const int64_t nk = (k + 127) / 128;
    Cut best{-1, 0, 0, 1};
    double least = 1e300;
    for (const Tile& t : tiles) {
        if ((t.f == 4 && nk < 4) || 64 * t.f * nk * 128 >= (int64_t(1) << 32)) continue;
        const int64_t count = ((m + 64 * t.f - 1) / (64 * t.f)) * ((n + 64 * t.f - 1) / (64 * t.f));
        for (int s = 1; s <= 16 && (s == 1 || s <= nk); s = s < 4 ? s + 1 : s + 2) {
            const int64_t per = (nk + s - 1) / s, wgs = count * s;
            // workgroups of 256 threads in a launch (tiles of 256 may go to tiles of 128, four for each)
            if (wgs > (t.f == 4 ? 0x3fffff : 0xffffff)) continue;
            if (s > 1 && (per < 4 || (s - 1) * per + 2 > nk)) continue;   // two blocks at least in every piece
            const double step = wgs <= (t.f == 4 ? 128 : 256) ? (f8 ? t.alone8 : t.alone32) : (f8 ? t.full8 : t.full32);
            const double rounds = static_cast<double>((wgs + t.slots - 1) / t.slots);
            const double time = rounds * (per * step + t.ends) + (s > 1 ? 4.0 + m * n * (8.0 * s + 4.0) / 5e6 : 0.0);
            if (time < least) {
                least = time;
                best = {t.f, 0, 0, s};
            }
        }
    }
    constexpr int waves[][2] = {{1, 1}, {1, 2}, {2, 2}, {4, 2}};   // FM, FN
    for (const auto& w : waves) {
        const int64_t wgs = ((m + 16 * w[0] - 1) / (16 * w[0])) * ((n + 16 * w[1] - 1) / (16 * w[1]));
        if (wgs > 4096) continue;
        const double time = 2.0 + (wgs + 255) / 256 * ((w[0] + w[1]) * 16.0 * nk * 128 / 26e3);
        if (time < least) {
            least = time;
            best = {0, w[0], w[1], 1};
        }
    }
    return best;
}

// The same for a result whose rows are ld apart: a descriptor of the widest tiles' stores spans a tile's rows of it.
Cut cut_for(int64_t m, int64_t n, int64_t k, int64_t ld, bool f8) {
    Cut c = choose(m, n, k, f8);
    if (c.f == 4 && (ld >= (1 << 21) || n >= (1 << 21))) c.f = 2;
    return c;
}

// The widest tiles store 16 bytes at a time: where the rows of the result are not whole pieces of 16 bytes, the columns
// that they take, up to the last whole tile; tiles of 128 take the rest.  (What the workspace holds is padded.)
int64_t wide_columns(int64_t n, int splits, int size) {
    return splits == 1 && n % (16 / size) != 0 ? n / 256 * 256 : n;
}

// Rows [n, rows) of a matrix; n a multiple of 128.
Fp8View rows_from(Fp8View f, int32_t n) {
    f.q += n * f.ld;
    f.scale += n / f.block * f.sld;
    f.rows -= n;
    return f;
}

template <bool F8, class Out, int F, int SLOTS>
int tile_launch(const MatmulArgs& a, int splits, hipStream_t stream) {
    TileArgs p = tile_args(a, 64 * F, 64 * F);
    const int64_t tiles = int64_t(p.tiles_m) * p.tiles_n;
    if (splits == 1) {
        tile_kernel<F8, Out, F, F, SLOTS><<<static_cast<uint32_t>(tiles), 256, 0, stream>>>(p);
        return hipGetLastError();
    }
    p.out = a.partial;
    p.ld = partial_ld(a.b.rows);
    p.blocks = (p.blocks + splits - 1) / splits;
    tile_kernel<F8, float, F, F, SLOTS>
        <<<dim3(static_cast<uint32_t>(tiles), static_cast<uint32_t>(splits)), 256, 0, stream>>>(p);
    return join_launch(a, static_cast<Out*>(a.out), splits, stream);
}

// Tiles of 256, one workgroup a CU.
template <bool F8, class Out>
int big_launch(const MatmulArgs& a, int splits, hipStream_t stream) {
    MatmulArgs main = a;
    main.b.rows = static_cast<int32_t>(wide_columns(a.b.rows, splits, sizeof(Out)));
    TileArgs p = tile_args(main, 256, 256);
    const int64_t items = int64_t(p.tiles_m) * p.tiles_n * splits;
    const uint32_t wgs = static_cast<uint32_t>(items < 256 ? items : 256);
    if (splits > 1) {
        p.out = a.partial;
        p.ld = partial_ld(a.b.rows);
        p.blocks = (p.blocks + splits - 1) / splits;
        big_kernel<float, F8, false><<<wgs, 256, 0, stream>>>(p, splits);
        return join_launch(a, static_cast<Out*>(a.out), splits, stream);
    }
    if (items > 0) {
        if (is_far(int64_t(a.a.rows) * a.b.rows * sizeof(Out))) big_kernel<Out, F8, true><<<wgs, 256, 0, stream>>>(p, 1);
        else big_kernel<Out, F8, false><<<wgs, 256, 0, stream>>>(p, 1);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || main.b.rows == a.b.rows) return e;
    MatmulArgs rest = a;
    rest.b = rows_from(a.b, main.b.rows);
    rest.out = static_cast<Out*>(a.out) + main.b.rows;
    return tile_launch<F8, Out, 2, 4>(rest, 1, stream);
}

template <bool F8, class Out, int FM, int FN>
int wave_launch(const MatmulArgs& a, hipStream_t stream) {
    const TileArgs p = tile_args(a, 16 * FM, 16 * FN);
    const int64_t tiles = int64_t(p.tiles_m) * p.tiles_n;
    wave_kernel<F8, Out, FM, FN, 8><<<static_cast<uint32_t>(tiles), 512, 0, stream>>>(p);
    return hipGetLastError();
}

template <bool F8, class Out>
int matmul_launch(const MatmulArgs& a, hipStream_t stream) {
    const Cut c = cut_for(a.a.rows, a.b.rows, a.a.cols, a.ld, F8);
    switch (c.f) {
        case 4: return big_launch<F8, Out>(a, c.splits, stream);
        case 2: return tile_launch<F8, Out, 2, 4>(a, c.splits, stream);
        case 1: return tile_launch<F8, Out, 1, 8>(a, c.splits, stream);
        default:
            if (c.fn == 1) return wave_launch<F8, Out, 1, 1>(a, stream);
            if (c.fm == 1) return wave_launch<F8, Out, 1, 2>(a, stream);
            if (c.fm == 2) return wave_launch<F8, Out, 2, 2>(a, stream);
            return wave_launch<F8, Out, 4, 2>(a, stream);
    }
}

}  // namespace

int64_t matmul_workspace(int64_t m, int64_t n, int64_t k, bool bf16) {
    const Cut c = choose(m, n, k, bf16);
    if (c.f < 0) return -1;
    return c.splits > 1 ? c.splits * m * partial_ld(n) * 4 : 0;
}

int describe_matmul(int64_t m, int64_t n, int64_t k, int64_t ld, bool bf16, int32_t (*rows)[4]) {
    if (m == 0 || n == 0) return 0;
    const Cut c = cut_for(m, n, k, ld, bf16);
    int count = 0;
    const auto add = [&](int32_t kind, int32_t tile_m, int32_t tile_n, int32_t pieces) {
        const int32_t row[4] = {kind, tile_m, tile_n, pieces};
        for (int i = 0; i < 4; ++i) rows[count][i] = row[i];
        ++count;
    };
    if (c.f == 0) {
        add(VP_PRODUCT_WAVES, 16 * c.fm, 16 * c.fn, 1);
    } else {
        const int64_t wide = c.f == 4 ? wide_columns(n, c.splits, bf16 ? 2 : 4) : n;
        if (wide > 0) add(VP_PRODUCT_TILES, 64 * c.f, 64 * c.f, c.splits);
        if (wide < n) add(VP_PRODUCT_TILES, 128, 128, 1);
        if (c.splits > 1) add(VP_PRODUCT_JOIN, 0, 0, c.splits);
    }
    return count;
}

int launch_matmul(const MatmulArgs& a, hipStream_t stream) {
    return a.bf16 ? matmul_launch<true, bf16_t>(a, stream) : matmul_launch<false, float>(a, stream);
}

}  // namespace vp
