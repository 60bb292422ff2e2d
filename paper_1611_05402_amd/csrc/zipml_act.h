// Activations stored in 8 bits: the layout and the device code that writes and reads it.
//
// 32 columns of a row share a step 2^e, e the least integer >= -126 with max |v| <= 127 * 2^e; a value is kept as
// floor(v * 2^-e + u), u uniform on the odd multiples of 2^-17 in (0, 1).  With a power of two as the step a
// code times its step has at most 7 significant bits, so it is a bf16 (and fp32) number exactly: what reads the
// codes may feed the bf16 matrix cores without rounding again.  Against a step of max / 127 this costs a step
// up to twice as large, one bit at worst and half a bit on average (over magnitudes spread evenly in the logarithm).
#pragma once
#include "zipml_device.h"
#include "zipml_host.h"

namespace zipml {

constexpr int kActGroup = 32;    // columns that share a step
constexpr int kActStream = 16;   // Philox stream of tag 0 (1 .. 4 are those of the quantisers)
constexpr int kActMaxTag = 239;  // streams have 8 bits

// Codes, int8 [rows][pitch], then the steps' biased exponents, uint8 [rows][pitch / 32]; pitch = cols rounded up to
// 32.  The codes of the columns beyond cols are zeros.
struct ActLayout {
    int64_t rows, cols, pitch, groups;
    int64_t steps;   // where the exponents start
    size_t bytes() const { return (size_t)(steps + rows * groups); }
};
inline ActLayout act_layout(int64_t rows, int64_t cols)
{
    const int64_t pitch = round_up(cols, kActGroup);
    return ActLayout{rows, cols, pitch, pitch / kActGroup, rows * pitch};
}
// Sizes whose byte offsets stay far below 2^63 (fp32 rows with any admissible stride).
inline bool act_sizes_ok(int64_t rows, int64_t cols)
{
    return rows > 0 && cols > 0 && rows <= (1ll << 40) && cols <= (1ll << 31) - 64 && rows <= (1ll << 56) / cols;
}
inline bool valid_dtype(int dtype) { return dtype == ZIPML_F32 || dtype == ZIPML_BF16; }
inline size_t dtype_bytes(int dtype) { return dtype == ZIPML_F32 ? 4 : 2; }

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float as_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u32(float f) { return __builtin_bit_cast(uint32_t, f); }

// ---- eight neighbouring values of a row, as fp32 ----------------------------------------------
// `left` values of the eight exist, the others read as zero.  Rows may start at any element: global memory is read 16
// bytes at a time at any alignment (rows aligned to 16 bytes take fewer cycles, no other code).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef bf16x8 bf16x8_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

template <typename T>
__device__ __forceinline__ void load8(const T *p, int64_t left, float (&v)[8])
{
    if (left >= 8) {
        if constexpr (sizeof(T) == 2) {
            const u32x4 w = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[2 * k] = as_f32(w[k] << 16);
                v[2 * k + 1] = as_f32(w[k] & 0xFFFF0000u);
            }
        } else {
            const f32x4 a = reinterpret_cast<const f32x4_any *>(p)[0], b = reinterpret_cast<const f32x4_any *>(p)[1];
#pragma unroll
            for (int k = 0; k < 4; ++k) { v[k] = a[k]; v[4 + k] = b[k]; }
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < left ? (float)p[k] : 0.0f;
    }
}
// (rounded to T once, to the nearest; THROUGH: past the caches)
template <bool THROUGH = false, typename T>
__device__ __forceinline__ void store8(T *p, int64_t left, const float (&v)[8])
{
    auto put = [](auto *to, auto w) {
        if constexpr (THROUGH) __builtin_nontemporal_store(w, to);
        else *to = w;
    };
    if (left >= 8) {
        if constexpr (sizeof(T) == 2) {
            bf16x8 o;
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = (__bf16)v[k];
            put(reinterpret_cast<bf16x8_any *>(p), (bf16x8_any)o);
        } else {
            put(reinterpret_cast<f32x4_any *>(p), (f32x4_any)f32x4{v[0], v[1], v[2], v[3]});
            put(reinterpret_cast<f32x4_any *>(p) + 1, (f32x4_any)f32x4{v[4], v[5], v[6], v[7]});
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < left) p[k] = (T)v[k];
    }
}

// ---- storing ----------------------------------------------------------------------------------
struct ActStep {
    uint32_t byte;     // biased exponent of the step, 255 for a group that is not finite
    float inverse;     // 1 / step
    bool finite;
};
// From the largest magnitude of a group, as the bits of an fp32 number (as integers: finite < infinity < NaN): the exponent of
// max minus 6, one more where its mantissa is above 127 / 64.
__device__ __forceinline__ ActStep act_step_of(uint32_t top)
{
    int byte = (int)((top + 0x1FFFFu) >> 23) - 6;
    byte = byte < 1 ? 1 : byte;
    const bool finite = top < 0x7F800000u;
    return ActStep{finite ? (uint32_t)byte : 255u, as_f32((uint32_t)(254 - byte) << 23), finite};
}
// floor as an integer, in one operation.
__device__ __forceinline__ int floor_int(float x)
{
    int i;
    __asm__("v_cvt_flr_i32_f32 %0, %1" : "=v"(i) : "v"(x));
    return i;
}
// Four codes from their 16-bit draws (the halves of w0, w1, low first).
//   fp32: floor(v / step + (k + 1/2) / 2^16) as it stands; (k + 1/2) / 2^16 is exact, and so is the product, so the fused form
//   rounds the sum as two operations would.
//   bf16: floor(2^16 v / step + 1/2) + k, the code in bits 16 and up: two operations less.  A bf16 value has 8 bits, so that sum
//   is rounded only where v / step is below 2^-16, and the two forms agree on all values but 255/256 * 2^-17 with
//   k = 2^16 - 1, where the sum above rounds up to 1; with 1/2 + 2^-9 in place of 1/2 they agree there too, and nowhere else does
//   the 2^-9 matter (it would take a fraction within 2^-9 below 1/2, which 8 bits cannot hold at any other value).
//   Steps below 2^-109 would overflow 2^16 / step; then (top says) the fp32 form is taken.
template <typename T>
__device__ __forceinline__ uint32_t act_codes4(const float (&v)[4], const ActStep &s, uint32_t w0, uint32_t w1, uint32_t top)
{
    const uint32_t w[2] = {w0, w1};
    uint32_t c[4];
    if (sizeof(T) == 2 && (top == 0 || s.byte >= 17)) {
        const uint32_t e = 270u - s.byte;
        const float scale = as_f32((e < 254u ? e : 254u) << 23);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            c[k] = (uint32_t)floor_int(__builtin_fmaf(v[k], scale, 0.5f + 1.0f / 512.0f)) + (k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xFFFFu);
        return __builtin_amdgcn_perm(c[1], c[0], 0x0C0C0602u) | __builtin_amdgcn_perm(c[3], c[2], 0x06020C0Cu);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t draw = k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xFFFFu;
        const float u = __builtin_fmaf((float)draw, 1.0f / 65536.0f, 1.0f / 131072.0f);
        c[k] = (uint32_t)floor_int(__builtin_fmaf(v[k], s.inverse, u));
    }
    return __builtin_amdgcn_perm(c[1], c[0], 0x0C0C0400u) | __builtin_amdgcn_perm(c[3], c[2], 0x04000C0Cu);
}

struct ActCodes8 {
    u32x2 codes;
    uint32_t byte;   // of the whole group
};

// Four neighbouring lanes, the first a multiple of four, hold the 32 values of a group, eight each (zeros beyond the
// row's end).  All four have to be active.  One Philox block gives the eight draws, 16 bits each: the chance of the
// upper neighbour is right to 2^-17 of a step, and half the multiplies of 24-bit draws are saved.
template <typename T>
__device__ __forceinline__ ActCodes8 act_encode8(const float (&v)[8], uint64_t seed, uint32_t epoch, int64_t row,
                                                 uint32_t col8, uint32_t stream)
{
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t m = as_u32(v[k]) & 0x7FFFFFFFu;
        top = top > m ? top : m;
    }
    uint32_t o = dpp_move<0xB1>(top);
    top = top > o ? top : o;
    o = dpp_move<0x4E>(top);
    top = top > o ? top : o;
    const ActStep s = act_step_of(top);
    const Philox4 r = philox_block(seed, epoch, (uint64_t)row, col8, stream);
    ActCodes8 out;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const float x[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        out.codes[q] = s.finite ? act_codes4<T>(x, s, r.w[2 * q], r.w[2 * q + 1], top) : 0u;
    }
    out.byte = s.byte;
    return out;
}

// ---- reading ----------------------------------------------------------------------------------
// Step of a group.  Byte 255 gives infinity, and a code of 0 times it NaN.
__device__ __forceinline__ float act_step(uint32_t byte) { return as_f32(byte << 23); }

__device__ __forceinline__ void act_decode8(u32x2 codes, float step, float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)(int8_t)(codes[k >> 2] >> (8 * (k & 3))) * step;
}

// ---- elementwise launches over rows of units of eight columns ---------------------------------
// A thread takes eight columns of kActRows rows; the loads of all of them are issued before the first is used (2 rows measure the
// same, 8 are 3 % slower).
constexpr int kActRows = 4;
// Threads side by side in x take the units of eight columns of a row, those side by side in y rows; a workgroup takes tx * 8
// columns of 256 / tx * kActRows rows at a time.
struct ActGrid {
    int tx_log;       // log2 of the threads along a row
    int64_t col_blocks, row_blocks;
};
inline ActGrid act_grid(int64_t rows, int64_t units)
{
    ActGrid g;
    g.tx_log = 2;
    while (g.tx_log < 8 && (1ll << g.tx_log) < units) ++g.tx_log;
    g.col_blocks = (units + (1 << g.tx_log) - 1) >> g.tx_log;
    const int64_t rows_block = (256 >> g.tx_log) * kActRows;
    g.row_blocks = (rows + rows_block - 1) / rows_block;
    return g;
}
// Workgroups of a grid-stride launch.
inline int act_blocks(const ActGrid &g)
{
    const int64_t all = g.col_blocks * g.row_blocks;
    return (int)(all < (1 << 20) ? all : 1 << 20);
}

}  // namespace zipml
