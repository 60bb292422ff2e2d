// Weight gradient of a linear layer from its stored input: dW[o][i] = sum_t dY[t][o] Q(X)[t][i].
//
// A product whose two operands are both contracted along their slow axis (tokens).  A workgroup owns a tile of dW and
// walks over the tokens: rows of dY and of the codes come in with wide loads, the codes are turned into bf16 on
// their way into LDS (once per workgroup; exact, a step is a power of two), both tiles lie in LDS as they lie in
// memory, [token][column], and are read through the transposing LDS read, which hands every lane four tokens of one
// column.  Which tokens a lane gets does not matter as long as both operands agree.
//
// bf16 dY: the products are exact and the sums fp32.  fp32 dY is split into three bf16 terms of 8 bits each, which
// together are the value exactly, and takes three matrix instructions in place of one.
#include "zipml_act.h"

namespace zipml {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct WgradArgs {
    const void *dy;
    const uint8_t *act;
    float *out;            // dW, or the partial sums of the token ranges one after the other
    int64_t lddy, rows, pitch, groups, steps;
    int64_t ldo, out_split;   // elements between rows of out, and between the partial sums
    int64_t rows_split;       // tokens of a range
    int d_out, d_in, tiles_o, tiles_i, add;
};

// MT x NT is the tile of dW, BK the tokens of one step; WM x WN waves share the tile.
template <typename T, int MT_, int NT_, int BK_, int WM_, int WN_>
struct WgradShape {
    static constexpr int MT = MT_, NT = NT_, BK = BK_, WM = WM_, WN = WN_;
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;        // bf16 terms of a dY value
    // LDS rows of 64 bytes more than a multiple of 256: the four rows that 16 lanes of a transposing read touch, and
    // the 64 bytes that the neighbouring 16 lanes add to each, then fall on all banks once.
    static constexpr int kRowA = MT * 2 + 64, kRowB = NT * 2 + 64;
    static constexpr int kBytesA = BK * kRowA, kBytesB = BK * kRowB;
    static constexpr int kStage = kPlanes * kBytesA + kBytesB;
    static constexpr int kLoadsA = BK * MT / 8 / kThreads;        // eight dY values each
    static constexpr int kLoadsB = BK * NT / 16 / kThreads;       // sixteen codes each
    static constexpr int TM = MT / WM / 32, TN = NT / WN / 32;    // 32 x 32 tiles of a wave
    static_assert(kLoadsA * 8 * kThreads == BK * MT && kLoadsB * 16 * kThreads == BK * NT, "whole loads");
    static_assert(MT % 128 == 0 && NT % 128 == 0, "LDS rows");
    static_assert(2 * kStage <= 160 * 1024, "LDS");
};

// Four tokens of one column of an LDS tile, transposed (see the file's head).
__device__ __forceinline__ bf16x4 read_transposed(const char *p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
        (__attribute__((address_space(3))) bf16x4 *)(__attribute__((address_space(3))) char *)p);
}
__device__ __forceinline__ bf16x8 fragment(const char *tile, int row_bytes)
{
    // tokens 0..7 of the sixteen from the first read, 8..15 from the second
    const bf16x4 a = read_transposed(tile), b = read_transposed(tile + 8 * row_bytes);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Eight dY values as bf16 terms; the first takes the upper 8 bits of the mantissa by truncation, so that it never
// overflows, the second those of the rest, the third what is left (an infinity or a NaN has only the first).
template <typename T>
__device__ __forceinline__ void split8(const float (&v)[8], u32x4 (&plane)[sizeof(T) == 4 ? 3 : 1])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t hi[2], mid[2], lo[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float x = v[2 * k + h];
            const uint32_t bits = as_u32(x);
            if constexpr (sizeof(T) == 2) {
                hi[h] = bits;
            } else {
                const bool finite = (bits & 0x7F800000u) != 0x7F800000u;
                hi[h] = x != x ? 0x7FC00000u : bits & 0xFFFF0000u;
                const float r = finite ? x - as_f32(hi[h]) : 0.0f;
                mid[h] = as_u32(r) & 0xFFFF0000u;
                lo[h] = as_u32(r - as_f32(mid[h]));
            }
        }
        plane[0][k] = __builtin_amdgcn_perm(hi[1], hi[0], 0x07060302u);
        if constexpr (sizeof(T) == 4) {
            plane[1][k] = __builtin_amdgcn_perm(mid[1], mid[0], 0x07060302u);
            plane[2][k] = __builtin_amdgcn_perm(lo[1], lo[0], 0x07060302u);
        }
    }
}

template <typename T, typename S, bool VEC>
__global__ __launch_bounds__(S::kThreads) void k_act_wgrad(WgradArgs a)
{
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tiles = a.tiles_o * a.tiles_i;
    const int split = blockIdx.x / tiles, tile = blockIdx.x - split * tiles;
    const int o0 = tile / a.tiles_i * S::MT, i0 = tile % a.tiles_i * S::NT;
    const int64_t t_begin = split * a.rows_split;
    const int64_t t_end = t_begin + a.rows_split < a.rows ? t_begin + a.rows_split : a.rows;
    const T *dy = (const T *)a.dy;

    float va[S::kLoadsA][8];
    u32x4 vb[S::kLoadsB];
    uint32_t step[S::kLoadsB];

    auto load = [&](int64_t t0) {
#pragma unroll
        for (int q = 0; q < S::kLoadsA; ++q) {
            const int c = tid + q * S::kThreads, r = c / (S::MT / 8), col = o0 + c % (S::MT / 8) * 8;
            const int64_t t = t0 + r;
            load8<T, VEC>(dy + t * a.lddy + col, t < t_end ? a.d_out - col : 0, va[q]);
        }
#pragma unroll
        for (int q = 0; q < S::kLoadsB; ++q) {
            const int c = tid + q * S::kThreads, r = c / (S::NT / 16), col = i0 + c % (S::NT / 16) * 16;
            const int64_t t = t0 + r;
            const bool there = t < t_end && col < a.pitch;      // the pitch is a multiple of 32
            vb[q] = there ? *reinterpret_cast<const u32x4 *>(a.act + t * a.pitch + col) : u32x4{0, 0, 0, 0};
            step[q] = there ? a.act[a.steps + t * a.groups + (col >> 5)] : 0u;
        }
    };
    auto store = [&](char *stage) {
#pragma unroll
        for (int q = 0; q < S::kLoadsA; ++q) {
            const int c = tid + q * S::kThreads, r = c / (S::MT / 8), col = c % (S::MT / 8) * 8;
            u32x4 plane[S::kPlanes];
            split8<T>(va[q], plane);
#pragma unroll
            for (int p = 0; p < S::kPlanes; ++p)
                *reinterpret_cast<u32x4 *>(stage + p * S::kBytesA + r * S::kRowA + col * 2) = plane[p];
        }
#pragma unroll
        for (int q = 0; q < S::kLoadsB; ++q) {
            const int c = tid + q * S::kThreads, r = c / (S::NT / 16), col = c % (S::NT / 16) * 16;
            const float s = act_step(step[q]);
            u32x4 o[2];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t w = vb[q][k >> 1];
                const float x = (float)(int8_t)(w >> (16 * (k & 1))) * s, y = (float)(int8_t)(w >> (16 * (k & 1) + 8)) * s;
                o[k >> 2][k & 3] = __builtin_amdgcn_perm(as_u32(y), as_u32(x), 0x07060302u);
            }
            u32x4 *p = reinterpret_cast<u32x4 *>(stage + S::kPlanes * S::kBytesA + r * S::kRowB + col * 2);
            p[0] = o[0];
            p[1] = o[1];
        }
    };

    const int wm = wave / S::WN, wn = wave % S::WN;
    // where this lane's four columns of the transposing reads start
    const int tr_row = 4 * (lane >> 5) + ((lane & 15) >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const int off_a = tr_row * S::kRowA + (wm * S::TM * 32 + tr_col) * 2;
    const int off_b = tr_row * S::kRowB + (wn * S::TN * 32 + tr_col) * 2 + S::kPlanes * S::kBytesA;
    f32x16 acc[S::TM][S::TN] = {};

    if (t_begin < t_end) {
        load(t_begin);
        store(lds);
        __syncthreads();
        int cur = 0;
        for (int64_t t0 = t_begin; t0 < t_end; t0 += S::BK) {
            const bool more = t0 + S::BK < t_end;
            if (more) load(t0 + S::BK);
            const char *stage = lds + cur * S::kStage;
#pragma unroll
            for (int k = 0; k < S::BK / 16; ++k) {
                bf16x8 fb[S::TN];
#pragma unroll
                for (int n = 0; n < S::TN; ++n) fb[n] = fragment(stage + off_b + k * 16 * S::kRowB + n * 64, S::kRowB);
#pragma unroll
                for (int p = 0; p < S::kPlanes; ++p)
#pragma unroll
                    for (int m = 0; m < S::TM; ++m) {
                        const bf16x8 fa = fragment(stage + off_a + p * S::kBytesA + k * 16 * S::kRowA + m * 64, S::kRowA);
#pragma unroll
                        for (int n = 0; n < S::TN; ++n)
                            acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa, fb[n], acc[m][n], 0, 0, 0);
                    }
            }
            cur ^= 1;
            if (more) store(lds + cur * S::kStage);
            __syncthreads();
        }
    }

    float *out = a.out + split * a.out_split;
#pragma unroll
    for (int m = 0; m < S::TM; ++m)
#pragma unroll
        for (int n = 0; n < S::TN; ++n) {
            const int i = i0 + (wn * S::TN + n) * 32 + (lane & 31);
            if (i >= a.d_in) continue;
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int o = o0 + (wm * S::TM + m) * 32 + 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3);
                if (o >= a.d_out) continue;
                float *p = out + o * a.ldo + i;
                *p = a.add ? *p + acc[m][n][q] : acc[m][n][q];
            }
        }
}

// Sum of the ranges' partial sums, in their order.
__global__ __launch_bounds__(256) void k_wgrad_sum(const float *__restrict__ part, int splits, int64_t out_split, int d_out,
                                                   int d_in, int64_t ld_part, float *__restrict__ dw, int64_t lddw, int add)
{
    const int i = (blockIdx.x % ((d_in + 255) / 256)) * 256 + threadIdx.x, o = blockIdx.x / ((d_in + 255) / 256);
    if (i >= d_in || o >= d_out) return;
    const float *p = part + o * ld_part + i;
    float sum = 0.0f;
    for (int s = 0; s < splits; ++s) sum += p[s * out_split];
    float *w = dw + o * lddw + i;
    *w = add ? *w + sum : sum;
}

struct WgradPlan {
    int tile, splits, tiles_o, tiles_i;
    int64_t rows_split;
    size_t workspace() const { return splits > 1 ? (size_t)splits * tiles_o * tiles_i * tile * tile * 4 : 0; }
};
static WgradPlan wgrad_plan(int64_t rows, int64_t d_out, int64_t d_in)
{
    WgradPlan p;
    auto tiles = [&](int t) { return ((d_out + t - 1) / t) * ((d_in + t - 1) / t); };
    p.tile = tiles(256) >= 128 ? 256 : 128;
    p.tiles_o = (int)((d_out + p.tile - 1) / p.tile);
    p.tiles_i = (int)((d_in + p.tile - 1) / p.tile);
    const int64_t n = tiles(p.tile);
    int64_t s = p.tile == 256 ? 1 : 256 / n;
    const int64_t most = (rows + 127) / 128;
    s = s < 1 ? 1 : s > most ? most : s;
    p.rows_split = round_up((rows + s - 1) / s, 64);
    p.splits = (int)((rows + p.rows_split - 1) / p.rows_split);
    return p;
}

template <typename T, typename S>
static int launch_wgrad(hipStream_t s, const WgradArgs &a, int splits)
{
    const bool vec = a.lddy * (int64_t)sizeof(T) % 16 == 0;
    auto k = vec ? k_act_wgrad<T, S, true> : k_act_wgrad<T, S, false>;
    if (HIP_FAILED(hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * S::kStage)))
        return ZIPML_ELAUNCH;
    hipLaunchKernelGGL(k, dim3(a.tiles_o * a.tiles_i * splits), dim3(S::kThreads), 2 * S::kStage, s, a);
    return hip_check(hipGetLastError());
}

}  // namespace zipml

using namespace zipml;

static bool wgrad_sizes_ok(int64_t rows, int64_t d_out, int64_t d_in)
{
    return act_sizes_ok(rows, d_in) && d_out > 0 && d_out <= (1 << 24) && d_in <= (1 << 24) &&
           ((d_out + 127) / 128) * ((d_in + 127) / 128) <= (1ll << 30);
}

extern "C" size_t zipml_act_wgrad_workspace_bytes(int64_t rows, int64_t d_out, int64_t d_in, int dtype)
{
    if (!wgrad_sizes_ok(rows, d_out, d_in) || !valid_dtype(dtype)) return 0;
    const size_t b = wgrad_plan(rows, d_out, d_in).workspace();
    return b < 256 ? 256 : b;
}

extern "C" int zipml_act_wgrad(void *stream, const void *dy_dev, int dtype, int64_t lddy, const void *act_dev,
                               int64_t rows, int64_t d_out, int64_t d_in, int flags, float *dw_dev, int64_t lddw,
                               void *workspace_dev, size_t workspace_bytes)
{
    if (!dy_dev || !act_dev || !dw_dev || !valid_dtype(dtype) || !wgrad_sizes_ok(rows, d_out, d_in)) return ZIPML_EINVAL;
    if (lddy < d_out || lddy > (1ll << 60) / rows || lddw < d_in || lddw > (1ll << 60) / d_out) return ZIPML_EINVAL;
    if (flags & ~ZIPML_WGRAD_ADD) return ZIPML_EINVAL;
    if (!workspace_dev || workspace_bytes < zipml_act_wgrad_workspace_bytes(rows, d_out, d_in, dtype))
        return ZIPML_EWORKSPACE;
    if (!aligned16(dy_dev) || !aligned16(act_dev) || !aligned16(dw_dev) || !aligned16(workspace_dev)) return ZIPML_EALIGN;
    const ActLayout lay = act_layout(rows, d_in);
    const WgradPlan p = wgrad_plan(rows, d_out, d_in);
    hipStream_t s = entry_stream(stream);
    const int add = flags & ZIPML_WGRAD_ADD ? 1 : 0;
    WgradArgs a{dy_dev, (const uint8_t *)act_dev, dw_dev, lddy, rows, lay.pitch, lay.groups, lay.steps, lddw, 0,
                p.rows_split, (int)d_out, (int)d_in, p.tiles_o, p.tiles_i, add};
    if (p.splits > 1) {
        a.out = (float *)workspace_dev;
        a.ldo = (int64_t)p.tiles_i * p.tile;
        a.out_split = a.ldo * p.tiles_o * p.tile;
        a.add = 0;
    }
    int rc;
    if (dtype == ZIPML_BF16)
        rc = p.tile == 256 ? launch_wgrad<__bf16, WgradShape<__bf16, 256, 256, 64, 2, 2>>(s, a, p.splits)
                           : launch_wgrad<__bf16, WgradShape<__bf16, 128, 128, 64, 2, 2>>(s, a, p.splits);
    else
        rc = p.tile == 256 ? launch_wgrad<float, WgradShape<float, 256, 256, 32, 2, 2>>(s, a, p.splits)
                           : launch_wgrad<float, WgradShape<float, 128, 128, 32, 2, 2>>(s, a, p.splits);
    if (rc || p.splits == 1) return rc;
    const int64_t blocks = (d_in + 255) / 256 * d_out;
    hipLaunchKernelGGL(k_wgrad_sum, dim3((uint32_t)blocks), dim3(256), 0, s, a.out, p.splits, a.out_split, (int)d_out,
                       (int)d_in, a.ldo, dw_dev, lddw, add);
    return hip_check(hipGetLastError());
}
