// Rows of 8-bit codes with one scale a row: zipml_row8_encode and zipml_row8_decode.
#include "zipml_row8.h"

namespace zipml {

struct Row8Args {
    const void *x;
    uint8_t *codes;
    float *scales;
    int64_t ldx, ldc, rows, cols, units;   // units of eight codes, those of the padding included
    uint64_t seed;
    uint32_t epoch, stream;
};

// A row waits in registers between the search for its largest magnitude and the rounding; rows too long for that are read twice.  Bound by
// the bytes: 16,384 x 4,096 bf16, 201 MB in 37 to 46 us (4.4 to 5.4 TB/s), by draws 40 to 42 (floor of both 41, at the rate of a copy).
// 1,000 x 1,001 fp32 by draws: 3.0 to 3.4 us, of which 1.4 are an empty launch.
template <typename T, typename S, bool DRAWS>
__global__ __launch_bounds__(S::kThreads) void k_row8_encode(Row8Args a)
{
    __shared__ uint32_t scratch[2][S::kThreads / kWave];
    const int lane = S::lane(), team = S::team();
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * S::kRows + team; row < a.rows; row += (int64_t)gridDim.x * S::kRows, turn ^= 1) {
        const T *x = (const T *)a.x + row * a.ldx;
        uint8_t *codes = a.codes + row * a.ldc;
        float v[S::NV ? S::NV : 1][8];
        uint32_t top = 0;
        auto encode = [&](const float (&w)[8], int64_t u, const Row8Scale &s) {
            u32x2 c;
            if constexpr (DRAWS) c = row8_stochastic8(w, s, philox_block(a.seed, a.epoch, (uint64_t)row, (uint32_t)u, a.stream));
            else c = row8_nearest8(w, s);
            *reinterpret_cast<u32x2 *>(codes + u * 8) = c;
        };
        if constexpr (S::NV > 0) {
#pragma unroll
            for (int k = 0; k < S::NV; ++k) {
                const int u = lane + k * S::TPR;
                if constexpr (S::kBuffer) Row<T>(a.x, row * a.ldx, a.cols).load8(u, v[k]);
                else load8(x + u * 8, a.cols - u * 8, v[k]);
            }
#pragma unroll
            for (int k = 0; k < S::NV; ++k) top = top_of(v[k], top);
        } else {
            for (int64_t u = lane; u < a.units; u += S::TPR) {
                load8(x + u * 8, a.cols - u * 8, v[0]);
                top = top_of(v[0], top);
            }
        }
        const Row8Scale s = row8_scale_of(team_max<S::TPR>(top, scratch[turn]));
        if constexpr (S::NV > 0) {
#pragma unroll
            for (int k = 0; k < S::NV; ++k)
                if (lane + k * S::TPR < a.units) encode(v[k], lane + k * S::TPR, s);
        } else {
            for (int64_t u = lane; u < a.units; u += S::TPR) {
                load8(x + u * 8, a.cols - u * 8, v[0]);
                encode(v[0], u, s);
            }
        }
        if (lane == 0) a.scales[row] = s.scale;
    }
}

// Four rows of eight columns a thread, as in zipml_act.hip.  16,384 x 4,096 to bf16: 30 to 32 us, the codes out of the cache that the
// encoder left them in, 37 out of memory (201 MB, floor 41); to fp32 73 (336 MB, floor 68).  All results go through the caches.
template <typename T>
__global__ __launch_bounds__(256) void k_row8_decode(const uint8_t *codes, int64_t ldc, const float *scales, int64_t rows,
                                                     int64_t cols, ActGrid g, T *out, int64_t ldo)
{
    const int tx = threadIdx.x & ((1 << g.tx_log) - 1), ty = threadIdx.x >> g.tx_log, ny = 256 >> g.tx_log;
    for (int64_t b = blockIdx.x; b < g.col_blocks * g.row_blocks; b += gridDim.x) {
        const int64_t rb = b / g.col_blocks, unit = ((b - rb * g.col_blocks) << g.tx_log) + tx;
        if (unit * 8 >= cols) continue;
        const int64_t row0 = rb * (ny * kActRows) + ty;
        u32x2 c[kActRows];
        float s[kActRows];
#pragma unroll
        for (int q = 0; q < kActRows; ++q) {
            const int64_t row = row0 + q * ny;
            const bool there = row < rows;
            c[q] = there ? *reinterpret_cast<const u32x2 *>(codes + row * ldc + unit * 8) : u32x2{0, 0};
            s[q] = there ? scales[row] : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < kActRows; ++q) {
            const int64_t row = row0 + q * ny;
            if (row >= rows) break;
            float v[8];
            act_decode8(c[q], s[q], v);
            store8(out + row * ldo + unit * 8, cols - unit * 8, v);
        }
    }
}

template <typename T, typename S>
static int launch_encode(hipStream_t s, const Row8Args &a, bool draws)
{
    const int64_t blocks = (a.rows + S::kRows - 1) / S::kRows;
    const auto k = draws ? k_row8_encode<T, S, true> : k_row8_encode<T, S, false>;
    hipLaunchKernelGGL(k, dim3((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20)), dim3(S::kThreads), 0, s, a);
    return hip_check(hipGetLastError());
}

}  // namespace zipml

using namespace zipml;

extern "C" int zipml_row8_encode(void *stream, const void *x_dev, int dtype, int64_t rows, int64_t cols, int64_t ldx,
                                 int rounding, uint64_t seed, uint32_t epoch, int tag, void *codes_dev, int64_t ldc,
                                 float *scales_dev)
{
    if (!x_dev || !codes_dev || !scales_dev || !act_sizes_ok(rows, cols) || ldx < cols || ldx > (1ll << 60) / rows ||
        !valid_dtype(dtype) || !row8_pitch_ok(rows, cols, ldc))
        return ZIPML_EINVAL;
    if (rounding != ZIPML_NEAREST && rounding != ZIPML_STOCHASTIC) return ZIPML_EINVAL;
    if (epoch >= (1u << 24) || tag < 0 || tag > kActMaxTag) return ZIPML_EINVAL;
    if (!aligned16(x_dev) || !aligned16(codes_dev) || !aligned4(scales_dev)) return ZIPML_EALIGN;
    const Row8Args a{x_dev, (uint8_t *)codes_dev, scales_dev, ldx, ldc, rows, cols, round_up(cols, kRow8Unit) / 8, seed, epoch,
                     (uint32_t)(kActStream + tag)};
    hipStream_t s = entry_stream(stream);
    return with_row_shape(rows, a.units, kRowUnits, [&](auto shape) {
        using S = decltype(shape);
        const bool draws = rounding == ZIPML_STOCHASTIC;
        return dtype == ZIPML_F32 ? launch_encode<float, S>(s, a, draws) : launch_encode<__bf16, S>(s, a, draws);
    });
}

extern "C" int zipml_row8_decode(void *stream, const void *codes_dev, int64_t ldc, const float *scales_dev, int64_t rows,
                                 int64_t cols, void *out_dev, int dtype, int64_t ldo)
{
    if (!codes_dev || !scales_dev || !out_dev || !act_sizes_ok(rows, cols) || ldo < cols || ldo > (1ll << 60) / rows ||
        !valid_dtype(dtype) || !row8_pitch_ok(rows, cols, ldc))
        return ZIPML_EINVAL;
    if (!aligned16(codes_dev) || !aligned4(scales_dev) || !aligned16(out_dev)) return ZIPML_EALIGN;
    const ActGrid g = act_grid(rows, (cols + 7) / 8);
    hipStream_t s = entry_stream(stream);
    const auto *c = (const uint8_t *)codes_dev;
    if (dtype == ZIPML_F32)
        hipLaunchKernelGGL(k_row8_decode<float>, dim3(act_blocks(g)), dim3(256), 0, s, c, ldc, scales_dev, rows, cols, g,
                           (float *)out_dev, ldo);
    else
        hipLaunchKernelGGL(k_row8_decode<__bf16>, dim3(act_blocks(g)), dim3(256), 0, s, c, ldc, scales_dev, rows, cols, g,
                           (__bf16 *)out_dev, ldo);
    return hip_check(hipGetLastError());
}
