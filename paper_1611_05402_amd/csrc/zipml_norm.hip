// Root-mean-square norm with the residual's addition: zipml_norm_forward and zipml_norm_backward.
//
//   r = round(x + add),  rstd = 1 / sqrt(mean r^2 + eps),  n = r rstd,  v = n gain
//   backward, a = dy gain:  dx = dsum + rstd (a - n mean(a n)),  dgain = sum over the rows of dy n
//
// The mean square is summed in 64 bits (such adds cost nothing next to the bytes), rstd is rounded to fp32 once, and every further step is a single
// fp32 operation.  The order of the sum, which is another one where a row has more threads (few rows) and in a plain evaluation, moves the
// mean by some 2^-53 of itself, and rstd's rounding to 24 bits with it in some 2^-28 of all rows: a row's results are all but certain to
// be the same alone, in a batch and in a check bit for bit, not promised to be.
//
// Both passes read and write every byte once and are bound by them.  16,384 x 4,096 bf16: forward 91 to 98 us (two tensors in, the sum
// and codes out 470 MB, the sum and y 537 MB: 5.0 to 5.6 TB/s), backward 107 to 109 (537 MB, and 17 of dgain's sums), joining these 7.
// 1,000 x 1,001 fp32: 5.9, 5.8 and 3.6 us, of which an empty launch is 1.4.
#include "zipml_row8.h"

namespace zipml {

struct NormArgs {
    const void *x, *add;
    const float *gain;
    void *sum, *y;
    uint8_t *codes;
    float *scales, *rstd;
    int64_t ldx, ldadd, ldsum, ldy, ldc, rows, cols, units;
    float eps;
};

// The type's nearest value.
template <typename T>
__device__ __forceinline__ float rounded(float v)
{
    return sizeof(T) == 4 ? v : (float)(__bf16)v;
}

template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void k_norm_forward(NormArgs a)
{
    __shared__ double scratch_sum[2][S::kThreads / kWave];
    __shared__ uint32_t scratch_max[2][S::kThreads / kWave];
    const int lane = S::lane(), team = S::team();
    constexpr int NV = S::NV ? S::NV : 1;
    float gain[NV][8];
    auto load_gain = [&](int64_t u, float (&g)[8]) {
        if (!a.gain) {
#pragma unroll
            for (int k = 0; k < 8; ++k) g[k] = 1.0f;
        } else if constexpr (S::kBuffer) {
            Row<float>(a.gain, 0, a.cols).load8((int)u, g);
        } else {
            load8(a.gain + u * 8, a.cols - u * 8, g);
        }
    };
    if constexpr (S::NV > 0)
#pragma unroll
        for (int k = 0; k < NV; ++k) load_gain(lane + k * S::TPR, gain[k]);
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * S::kRows + team; row < a.rows; row += (int64_t)gridDim.x * S::kRows, turn ^= 1) {
        float v[NV][8];
        double square = 0;
        // eight values of a tensor's row
        auto get = [&](const void *tensor, int64_t ld, int64_t u, float (&w)[8]) {
            if constexpr (S::kBuffer) Row<T>(tensor, row * ld, a.cols).load8((int)u, w);
            else load8((const T *)tensor + row * ld + u * 8, a.cols - u * 8, w);
        };
        auto set = [&](void *tensor, int64_t ld, int64_t u, const float (&w)[8]) {
            if constexpr (S::kBuffer) Row<T>(tensor, row * ld, a.cols).store8((int)u, w);
            else store8((T *)tensor + row * ld + u * 8, a.cols - u * 8, w);
        };
        auto added = [&](float (&w)[8], const float (&o)[8]) {
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = rounded<T>(w[k] + o[k]);
        };
        auto take = [&](int64_t u, float (&w)[8]) {
            get(a.x, a.ldx, u, w);
            if (a.add) {
                float o[8];
                get(a.add, a.ldadd, u, o);
                added(w, o);
            }
        };
        auto squares = [&](int64_t u, const float (&w)[8]) {
            if (a.sum) set(a.sum, a.ldsum, u, w);
#pragma unroll
            for (int k = 0; k < 8; ++k) square = __builtin_fma((double)w[k], (double)w[k], square);
        };
        if constexpr (S::NV > 0) {
            if (a.add) {                   // (all loads before the first is used)
                float o[NV][8];
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    get(a.x, a.ldx, lane + k * S::TPR, v[k]);
                    get(a.add, a.ldadd, lane + k * S::TPR, o[k]);
                }
#pragma unroll
                for (int k = 0; k < NV; ++k) added(v[k], o[k]);
            } else {
#pragma unroll
                for (int k = 0; k < NV; ++k) get(a.x, a.ldx, lane + k * S::TPR, v[k]);
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) squares(lane + k * S::TPR, v[k]);
        } else {
            for (int64_t u = lane; u < a.units; u += S::TPR) {
                take(u, v[0]);
                squares(u, v[0]);
            }
        }
        square = team_sum<S::TPR>(square, scratch_sum[turn]);
        const float rstd = (float)(1.0 / __builtin_sqrt(square / (double)a.cols + (double)a.eps));
        if (a.rstd && lane == 0) a.rstd[row] = rstd;
        // a row too long for the registers is read again: from the sum, which may stand in the place of x
        auto again = [&](int64_t u, float (&w)[8]) {
            if (a.sum) get(a.sum, a.ldsum, u, w);
            else take(u, w);
            load_gain(u, gain[0]);
        };
        auto normed = [&](float (&w)[8], const float (&g)[8]) {
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = w[k] * rstd * g[k];
        };
        uint32_t top = 0;
        if constexpr (S::NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                normed(v[k], gain[k]);
                top = top_of(v[k], top);
            }
        } else if (a.codes) {
            for (int64_t u = lane; u < a.units; u += S::TPR) {
                again(u, v[0]);
                normed(v[0], gain[0]);
                top = top_of(v[0], top);
            }
        }
        Row8Scale s{};
        if (a.codes) {
            s = row8_scale_of(team_max<S::TPR>(top, scratch_max[turn]));
            if (lane == 0) a.scales[row] = s.scale;
        }
        auto put = [&](int64_t u, const float (&w)[8]) {
            if (a.codes && u < a.units) *reinterpret_cast<u32x2 *>(a.codes + row * a.ldc + u * 8) = row8_nearest8(w, s);
            if (a.y) set(a.y, a.ldy, u, w);
        };
        if constexpr (S::NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) put(lane + k * S::TPR, v[k]);
        } else {
            for (int64_t u = lane; u < a.units; u += S::TPR) {
                again(u, v[0]);
                normed(v[0], gain[0]);
                put(u, v[0]);
            }
        }
    }
}

struct NormGradArgs {
    const void *dy, *sum, *dsum;
    const float *gain, *rstd;
    void *dx;
    float *part;       // [workgroups][pitch]: each one's sums of dy n, NULL if dgain is not wanted
    int64_t lddy, ldsum, lddsum, lddx, rows, cols, units, pitch;
};

// A workgroup takes every gridDim.x-th row (or set of rows, one for each team: a wave, or sixteen lanes) and keeps dgain's sums of its rows in registers.  1,024
// workgroups: 512 have too few loads under way (157 us in place of 108 at 16,384 x 4,096).  Rows of more than 16,384 values are read
// twice: the registers of 1,024 threads do not hold four such arrays.
template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void k_norm_backward(NormGradArgs a)
{
    __shared__ float scratch[2][S::kThreads / kWave];
    const int lane = S::lane(), team = S::team();
    constexpr int NV = S::NV ? S::NV : 1;
    float gain[NV][8], dgain[NV][8] = {};
    auto load_gain = [&](int64_t u, float (&g)[8]) {
        if (!a.gain) {
#pragma unroll
            for (int k = 0; k < 8; ++k) g[k] = 1.0f;
        } else if constexpr (S::kBuffer) {
            Row<float>(a.gain, 0, a.cols).load8((int)u, g);
        } else {
            load8(a.gain + u * 8, a.cols - u * 8, g);
        }
    };
    float *part = a.part ? a.part + blockIdx.x * a.pitch : nullptr;
    if constexpr (S::NV > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k) load_gain(lane + k * S::TPR, gain[k]);
    } else if (part) {
        for (int64_t u = lane; u < a.units; u += S::TPR) store8(part + u * 8, 8, dgain[0]);
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * S::kRows + team; row < a.rows; row += (int64_t)gridDim.x * S::kRows, turn ^= 1) {
        const float rstd = a.rstd[row];
        float g[NV][8], n[NV][8], o[NV][8] = {}, along = 0.0f;
        auto get = [&](const void *tensor, int64_t ld, int64_t u, float (&w)[8]) {
            if constexpr (S::kBuffer) Row<T>(tensor, row * ld, a.cols).load8((int)u, w);
            else load8((const T *)tensor + row * ld + u * 8, a.cols - u * 8, w);
        };
        // g = dy, n = r rstd of unit u
        auto scaled = [&](float (&q)[8]) {
#pragma unroll
            for (int k = 0; k < 8; ++k) q[k] *= rstd;
        };
        auto take = [&](int64_t u, float (&p)[8], float (&q)[8]) {
            get(a.dy, a.lddy, u, p);
            get(a.sum, a.ldsum, u, q);
        };
        // dy n into dgain's sums, g = dy gain
        auto weigh = [&](float (&p)[8], const float (&q)[8], const float (&w)[8], float (&sums)[8]) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                sums[k] = __builtin_fmaf(p[k], q[k], sums[k]);
                p[k] *= w[k];
                along = __builtin_fmaf(p[k], q[k], along);
            }
        };
        if constexpr (S::NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) take(lane + k * S::TPR, g[k], n[k]);
            if (a.dsum)
#pragma unroll
                for (int k = 0; k < NV; ++k) get(a.dsum, a.lddsum, lane + k * S::TPR, o[k]);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                scaled(n[k]);
                weigh(g[k], n[k], gain[k], dgain[k]);
            }
        } else {
            for (int64_t u = lane; u < a.units; u += S::TPR) {
                take(u, g[0], n[0]);
                scaled(n[0]);
                load_gain(u, gain[0]);
                if (part) load8(part + u * 8, 8, dgain[0]);
                weigh(g[0], n[0], gain[0], dgain[0]);
                if (part) store8(part + u * 8, 8, dgain[0]);
            }
        }
        along = team_sum<S::TPR>(along, scratch[turn]) / (float)a.cols;
        auto put = [&](int64_t u, const float (&p)[8], const float (&q)[8], float (&d)[8]) {
#pragma unroll
            for (int k = 0; k < 8; ++k) d[k] = __builtin_fmaf(rstd, __builtin_fmaf(-along, q[k], p[k]), d[k]);
            if constexpr (S::kBuffer) Row<T>(a.dx, row * a.lddx, a.cols).store8((int)u, d);
            else store8((T *)a.dx + row * a.lddx + u * 8, a.cols - u * 8, d);
        };
        if constexpr (S::NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) put(lane + k * S::TPR, g[k], n[k], o[k]);
        } else {
            for (int64_t u = lane; u < a.units; u += S::TPR) {
                take(u, g[0], n[0]);
                scaled(n[0]);
                load_gain(u, gain[0]);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    g[0][k] *= gain[0][k];
                    o[0][k] = 0.0f;
                }
                if (a.dsum) get(a.dsum, a.lddsum, u, o[0]);
                put(u, g[0], n[0], o[0]);
            }
        }
    }
    if constexpr (S::NV > 0) {
        if (!part) return;
        if constexpr (S::kRows > 1) {      // the teams' sums: of four waves, or of sixteen times sixteen lanes
            __shared__ float sums[S::kRows - 1][NV][8][S::TPR];
            if (team > 0)
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sums[team - 1][k][j][lane] = dgain[k][j];
            __syncthreads();
            if (team > 0) return;
#pragma unroll
            for (int w = 0; w < S::kRows - 1; ++w)
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) dgain[k][j] += sums[w][k][j][lane];
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t u = lane + k * S::TPR;
            if (u < a.units) store8(part + u * 8, 8, dgain[k]);
        }
    }
}

// dgain from the workgroups' sums, in an order of their number alone: sixteen lanes take sixteen columns, each of a workgroup's 64 such
// sets every 64th row of sums.
__global__ __launch_bounds__(1024) void k_norm_dgain(const float *part, int parts, int64_t pitch, int64_t cols, float *dgain, int add)
{
    __shared__ float sums[64][17];
    const int lane = threadIdx.x & 15, set = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + lane;     // (the rows of sums are padded to sixteen)
    float s = 0.0f;
#pragma unroll 4
    for (int p = set; p < parts; p += 64) s += part[p * pitch + c];
    sums[set][lane] = s;
    __syncthreads();
    if (set >= 4) return;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += sums[set * 16 + w][lane];
    s += __shfl_xor(s, 16, kWave);
    s += __shfl_xor(s, 32, kWave);
    if (set == 0 && c < cols) dgain[c] = add ? dgain[c] + s : s;
}

// Columns of a launch of k_norm_dgain, which takes 64 threads a column and holds fewer than 2^32.
constexpr int64_t kNormColumns = 1ll << 25;

// Workgroups of the backward pass: each one writes a row of sums, 256 MiB of them at most.
constexpr int64_t kNormGroups = 1024;
static int64_t norm_groups(int64_t rows, int64_t cols, int64_t rows_group)
{
    const int64_t g = (rows + rows_group - 1) / rows_group, room = (1ll << 26) / cols, most = room < kNormGroups ? room : kNormGroups;
    return g < most ? g : most > 1 ? most : 1;
}

}  // namespace zipml

using namespace zipml;

static bool norm_rows_ok(const void *p, int64_t ld, int64_t rows, int64_t cols) { return !p || (ld >= cols && ld <= (1ll << 60) / rows); }

// An output may stand in an input's place row by row, not at another pitch.
static bool in_place_ok(const void *out, int64_t ldo, const void *in, int64_t ldi, int64_t rows)
{
    return out != in || !out || ldo == ldi || rows == 1;
}

extern "C" int zipml_norm_forward(void *stream, const void *x_dev, int64_t ldx, const void *add_dev, int64_t ldadd, int dtype,
                                  int64_t rows, int64_t cols, const float *gain_dev, float eps, void *sum_dev, int64_t ldsum,
                                  void *y_dev, int64_t ldy, void *codes_dev, int64_t ldc, float *scales_dev, float *rstd_dev)
{
    if (!x_dev || !act_sizes_ok(rows, cols) || !valid_dtype(dtype) || !(eps >= 0.0f) || !(eps < __builtin_inff())) return ZIPML_EINVAL;
    if (!norm_rows_ok(x_dev, ldx, rows, cols) || !norm_rows_ok(add_dev, ldadd, rows, cols) ||
        !norm_rows_ok(sum_dev, ldsum, rows, cols) || !norm_rows_ok(y_dev, ldy, rows, cols))
        return ZIPML_EINVAL;
    if (!in_place_ok(sum_dev, ldsum, x_dev, ldx, rows) || !in_place_ok(sum_dev, ldsum, add_dev, ldadd, rows) ||
        !in_place_ok(y_dev, ldy, x_dev, ldx, rows) || !in_place_ok(y_dev, ldy, add_dev, ldadd, rows) || (y_dev && y_dev == sum_dev))
        return ZIPML_EINVAL;
    if ((!y_dev && !codes_dev) || !codes_dev != !scales_dev || (codes_dev && !row8_pitch_ok(rows, cols, ldc))) return ZIPML_EINVAL;
    if (!aligned16(x_dev) || !aligned16(add_dev) || !aligned4(gain_dev) || !aligned16(sum_dev) || !aligned16(y_dev) ||
        !aligned16(codes_dev) || !aligned4(scales_dev) || !aligned4(rstd_dev))
        return ZIPML_EALIGN;
    const NormArgs a{x_dev, add_dev, gain_dev, sum_dev, y_dev, (uint8_t *)codes_dev, scales_dev, rstd_dev, ldx, ldadd, ldsum, ldy,
                     ldc, rows, cols, round_up(cols, kRow8Unit) / 8, eps};
    hipStream_t s = entry_stream(stream);
    return with_row_shape(rows, a.units, kRowUnits, [&](auto shape) {
        using S = decltype(shape);
        const int64_t blocks = (rows + S::kRows - 1) / S::kRows;
        const auto k = dtype == ZIPML_F32 ? k_norm_forward<float, S> : k_norm_forward<__bf16, S>;
        hipLaunchKernelGGL(k, dim3((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20)), dim3(S::kThreads), 0, s, a);
        return hip_check(hipGetLastError());
    });
}

extern "C" size_t zipml_norm_backward_workspace_bytes(int64_t rows, int64_t cols)
{
    if (!act_sizes_ok(rows, cols)) return 0;
    // (rows that share a workgroup need fewer)
    return (size_t)norm_groups(rows, cols, 1) * (size_t)round_up(cols, kRow8Unit) * 4;
}

extern "C" int zipml_norm_backward(void *stream, const void *dy_dev, int64_t lddy, const void *sum_dev, int64_t ldsum, int dtype,
                                   int64_t rows, int64_t cols, const float *gain_dev, const float *rstd_dev,
                                   const void *dsum_dev, int64_t lddsum, void *dx_dev, int64_t lddx, float *dgain_dev, int flags,
                                   void *workspace_dev, size_t workspace_bytes)
{
    if (!dy_dev || !sum_dev || !rstd_dev || !dx_dev || !act_sizes_ok(rows, cols) || !valid_dtype(dtype)) return ZIPML_EINVAL;
    if (!norm_rows_ok(dy_dev, lddy, rows, cols) || !norm_rows_ok(sum_dev, ldsum, rows, cols) ||
        !norm_rows_ok(dsum_dev, lddsum, rows, cols) || !norm_rows_ok(dx_dev, lddx, rows, cols))
        return ZIPML_EINVAL;
    if (!in_place_ok(dx_dev, lddx, dy_dev, lddy, rows) || !in_place_ok(dx_dev, lddx, sum_dev, ldsum, rows) ||
        !in_place_ok(dx_dev, lddx, dsum_dev, lddsum, rows))
        return ZIPML_EINVAL;
    if ((flags & ~ZIPML_NORM_ADD) || ((flags & ZIPML_NORM_ADD) && !dgain_dev)) return ZIPML_EINVAL;
    if (dgain_dev && (!workspace_dev || workspace_bytes < zipml_norm_backward_workspace_bytes(rows, cols))) return ZIPML_EWORKSPACE;
    if (!aligned16(dy_dev) || !aligned16(sum_dev) || !aligned4(gain_dev) || !aligned16(dsum_dev) || !aligned16(dx_dev) ||
        !aligned4(dgain_dev) || !aligned4(rstd_dev) || (dgain_dev && !aligned16(workspace_dev)))
        return ZIPML_EALIGN;
    NormGradArgs a{dy_dev, sum_dev, dsum_dev, gain_dev, rstd_dev, dx_dev, dgain_dev ? (float *)workspace_dev : nullptr, lddy, ldsum,
                   lddsum, lddx, rows, cols, round_up(cols, kRow8Unit) / 8, round_up(cols, kRow8Unit)};
    hipStream_t s = entry_stream(stream);
    return with_row_shape(rows, a.units, kRowUnits / 2, [&](auto shape) {
        using S = decltype(shape);
        const int64_t groups = norm_groups(rows, cols, S::kRows);
        const auto k = dtype == ZIPML_F32 ? k_norm_backward<float, S> : k_norm_backward<__bf16, S>;
        hipLaunchKernelGGL(k, dim3((uint32_t)groups), dim3(S::kThreads), 0, s, a);
        if (const int rc = hip_check(hipGetLastError()); rc || !dgain_dev) return rc;
        for (int64_t c = 0; c < cols; c += kNormColumns) {
            const int64_t n = cols - c < kNormColumns ? cols - c : kNormColumns;
            hipLaunchKernelGGL(k_norm_dgain, dim3((uint32_t)((n + 15) / 16)), dim3(1024), 0, s, a.part + c, (int)groups, a.pitch, n,
                               dgain_dev + c, flags & ZIPML_NORM_ADD ? 1 : 0);
            if (const int rc = hip_check(hipGetLastError())) return rc;
        }
        return ZIPML_OK;
    });
}
