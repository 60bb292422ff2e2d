// Rows of 8-bit codes with one scale a row: the device code that makes them, and the checks that their entry points share.
//
// s = max(max |v| / 127, 2^-126), code = rint(v * (1 / s)) or floor(v * (1 / s) + u), value = code * s.  The scale is a plain
// fp32 number, not a power of two as in zipml_act.h: what reads these codes multiplies them as integers, and the scale at the
// end, so a row keeps the half bit that a power of two costs.
#pragma once
#include "zipml_act.h"

namespace zipml {

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
// A wave, or a workgroup of TPR threads; scratch: one value for each wave of the workgroup, another one for each reduction
// between two uses of the same scratch a barrier has to pass.
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    return wave_reduce_dpp(v, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
}
template <int TPR>
__device__ __forceinline__ uint32_t team_max(uint32_t v, uint32_t *scratch)
{
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

// How a row of `units` units of eight values is dealt: TPR threads, up to NV units each; NV = 0: as many as there are.
template <int TPR_, int NV_>
struct RowShape {
    static constexpr int TPR = TPR_, NV = NV_, kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR;
};
// Calls f with the shape for rows of so many units.
template <typename F>
inline int with_row_shape(int64_t units, F f)
{
    if (units <= 64) return f(RowShape<64, 1>());
    if (units <= 128) return f(RowShape<64, 2>());
    if (units <= 256) return f(RowShape<64, 4>());
    if (units <= 512) return f(RowShape<256, 2>());
    if (units <= 1024) return f(RowShape<256, 4>());
    if (units <= 2048) return f(RowShape<1024, 2>());
    if (units <= 4096) return f(RowShape<1024, 4>());
    return f(RowShape<1024, 0>());
}

}  // namespace zipml
