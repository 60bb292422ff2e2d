// Rows of 8-bit codes with one scale a row: the device code that makes them, and the checks that their entry points share.
//
// s = max(max |v| / 127, 2^-126), code = rint(v * (1 / s)) or floor(v * (1 / s) + u), value = code * s.  The scale is a plain
// fp32 number, not a power of two as in zipml_act.h: what reads these codes multiplies them as integers, and the scale at the
// end, so a row keeps the half bit that a power of two costs.
#pragma once
#include "zipml_act.h"

namespace zipml {

constexpr int64_t kFewRows = 512;                  // fewer rows than these are given more threads each
constexpr int64_t kRowUnits = 4096;                // longest rows (in units of eight values) that wait in registers
constexpr int kRow8Unit = 16;                       // bytes that a row of codes is padded to
constexpr int64_t kRow8MaxPitch = 1ll << 22;        // so that the offsets within a tile of rows stay below 2^31

inline bool row8_pitch_ok(int64_t rows, int64_t cols, int64_t ld)
{
    return ld % kRow8Unit == 0 && ld >= cols && ld <= (1ll << 60) / rows;
}


struct Row8Scale {
    float scale, inverse;
    bool finite;
};
// From the largest magnitude of a row, as the bits of an fp32 number (as integers: finite < infinity < NaN).
__device__ __forceinline__ Row8Scale row8_scale_of(uint32_t top)
{
    const bool finite = top < 0x7F800000u;
    const float s = fmaxf(as_f32(finite ? top : 0u) / 127.0f, 0x1p-126f);
    return Row8Scale{finite ? s : as_f32(0x7FC00000u), 1.0f / s, finite};
}

template <int N>
__device__ __forceinline__ uint32_t top_of(const float (&v)[N], uint32_t top)
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t m = as_u32(v[k]) & 0x7FFFFFFFu;
        top = top > m ? top : m;
    }
    return top;
}

// Eight codes.  To the nearest: 1.5 * 2^23 added in fp32 rounds to an integer, ties to even, and leaves it in the low bits.
__device__ __forceinline__ u32x2 row8_nearest8(const float (&v)[8], const Row8Scale &s)
{
    u32x2 out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = as_u32(v[4 * h + k] * s.inverse + 12582912.0f);
        out[h] = __builtin_amdgcn_perm(c[1], c[0], 0x0C0C0400u) | __builtin_amdgcn_perm(c[3], c[2], 0x04000C0Cu);
    }
    return s.finite ? out : u32x2{0, 0};
}
// By the draws of a Philox block, 16 bits each.  Where |v| / s is 127 the sum may round up to 128 (or its floor be -128).
__device__ __forceinline__ u32x2 row8_stochastic8(const float (&v)[8], const Row8Scale &s, const Philox4 &r)
{
    u32x2 out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t w = r.w[2 * h + (k >> 1)], draw = k & 1 ? w >> 16 : w & 0xFFFFu;
            const float u = __builtin_fmaf((float)draw, 1.0f / 65536.0f, 1.0f / 131072.0f);
            const int i = floor_int(v[4 * h + k] * s.inverse + u);
            c[k] = (uint32_t)(i < -127 ? -127 : i > 127 ? 127 : i);
        }
        out[h] = __builtin_amdgcn_perm(c[1], c[0], 0x0C0C0400u) | __builtin_amdgcn_perm(c[3], c[2], 0x04000C0Cu);
    }
    return s.finite ? out : u32x2{0, 0};
}

// ---- teams of threads that share a row --------------------------------------------------------
// Sixteen lanes, a wave, or a workgroup of TPR threads; scratch: one value for each wave of the workgroup, another one for each reduction
// between two uses of the same scratch a barrier has to pass.
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    return wave_reduce_dpp(v, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
}
template <int TPR>
__device__ __forceinline__ uint32_t team_max(uint32_t v, uint32_t *scratch)
{
    if constexpr (TPR < kWave) {
        static_assert(TPR == 16, "rows of DPP");
        return row_reduce_dpp(v, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    }
    v = wave_max(v);
    if constexpr (TPR > kWave) {
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        lds_barrier();
#pragma unroll
        for (int w = 0; w < TPR / kWave; ++w) v = v > scratch[w] ? v : scratch[w];
    }
    return v;
}
template <int TPR, typename F>
__device__ __forceinline__ F team_sum(F v, F *scratch)
{
    if constexpr (TPR < kWave) return row_sum_dpp(v);
    v = wave_sum_dpp(v);
    if constexpr (TPR > kWave) {
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        lds_barrier();
        v = scratch[0];
#pragma unroll
        for (int w = 1; w < TPR / kWave; ++w) v += scratch[w];
    }
    return v;
}

// ---- rows as buffers --------------------------------------------------------------------------
// A row of at most 2^28 values, read and written eight neighbouring values at a time without a branch: what lies behind its end reads
// as zeros and is not written.  (With a branch each load would wait for the one before.)  The end is exact to a dword: the last of an odd
// number of bf16 values goes by itself.  Rows may start at any element.
template <typename T>
struct Row {
    T *base;
    __amdgpu_buffer_rsrc_t r;
    int cols;
    __device__ __forceinline__ Row(const void *tensor, int64_t at, int64_t cols_) : base((T *)tensor + at), cols((int)cols_)
    {
        r = __builtin_amdgcn_make_buffer_rsrc(base, 0, cols * (int)sizeof(T), 0x00020000);
    }
    __device__ __forceinline__ bool odd() const { return sizeof(T) == 2 && (cols & 1); }
    __device__ __forceinline__ void load8(int u, float (&v)[8]) const
    {
        const u32x4 a = __builtin_amdgcn_raw_buffer_load_b128(r, u * 8 * (int)sizeof(T), 0, 0);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[2 * k] = as_f32(a[k] << 16);
                v[2 * k + 1] = as_f32(a[k] & 0xFFFF0000u);
            }
        } else {
            const u32x4 b = __builtin_amdgcn_raw_buffer_load_b128(r, u * 32 + 16, 0, 0);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t x = a[k], y = b[k];
                v[k] = as_f32(x);
                v[4 + k] = as_f32(y);
            }
        }
        if (odd()) {                       // (cols - 1 is even, so the value is one of v[0], v[2], v[4], v[6])
            const float last = u == (cols >> 3) ? (float)base[cols - 1] : 0.0f;
#pragma unroll
            for (int k = 0; k < 8; k += 2) v[k] = u * 8 + k == cols - 1 ? last : v[k];
        }
    }
    __device__ __forceinline__ void store8(int u, const float (&v)[8]) const
    {
        if constexpr (sizeof(T) == 2) {
            bf16x8 o;
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = (__bf16)v[k];
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), r, u * 16, 0, 0);
        } else {
            __builtin_amdgcn_raw_buffer_store_b128(u32x4{as_u32(v[0]), as_u32(v[1]), as_u32(v[2]), as_u32(v[3])}, r, u * 32, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b128(u32x4{as_u32(v[4]), as_u32(v[5]), as_u32(v[6]), as_u32(v[7])}, r, u * 32 + 16, 0, 0);
        }
        if (odd())
#pragma unroll
            for (int k = 0; k < 8; k += 2)
                if (u * 8 + k == cols - 1) base[cols - 1] = (T)v[k];
    }
};

// How a row of `units` units of eight values is dealt: TPR threads, up to NV units each; NV = 0: as many as there are.
template <int TPR_, int NV_>
struct RowShape {
    static constexpr int TPR = TPR_, NV = NV_, kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR;
    static constexpr bool kBuffer = NV > 0 && TPR >= kWave;       // rows are read and written as buffers, whose base a wave shares
    // the team's number in the workgroup, the same for a whole wave where that is no more than a team
    static __device__ __forceinline__ int team()
    {
        const int t = (int)threadIdx.x / TPR;
        return TPR == kThreads ? 0 : TPR < kWave ? t : __builtin_amdgcn_readfirstlane(t);
    }
    static __device__ __forceinline__ int lane() { return threadIdx.x % TPR; }
};
// Calls f with the shape for `rows` rows of so many units, of which registers are to hold `most` at most.  A wave to a row needs no
// barrier; where there are few rows, more waves to each bring its loads under way at once (one row of 2,048 through the norm: 2.6 us
// with four waves, 4.8 with one; at 1,000 rows of 1,001 four waves are as fast as one, and 15 % slower in encoding).
template <typename F>
inline int with_row_shape(int64_t rows, int64_t units, int64_t most, F f)
{
    if (units > most) return f(RowShape<1024, 0>());
    if (units <= 16) return f(RowShape<16, 1>());
    if (rows >= kFewRows && units <= 32) return f(RowShape<16, 2>());
    if (units <= 64) return f(RowShape<64, 1>());
    if (rows < kFewRows && units <= 256) return f(RowShape<256, 1>());
    if (rows < kFewRows && units <= 1024) return f(RowShape<1024, 1>());
    if (units <= 128) return f(RowShape<64, 2>());
    if (units <= 256) return f(RowShape<64, 4>());
    if (units <= 512) return f(RowShape<256, 2>());
    if (units <= 1024) return f(RowShape<256, 4>());
    if (units <= 2048) return f(RowShape<1024, 2>());
    return f(RowShape<1024, 4>());
}

}  // namespace zipml
