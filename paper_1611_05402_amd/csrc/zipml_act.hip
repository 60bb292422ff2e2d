// Activations stored in 8 bits: zipml_act_encode and zipml_act_decode.
#include "zipml_act.h"

namespace zipml {

// Both kernels stream; every byte is moved once.  16,384 x 4,096 bf16: storing 203 MB in 36 to 41 us (4.9 to 5.6 TB/s; its generator, ten
// rounds for eight values, keeps the vector units busy for more than half of that), restoring 203 MB in 30 us (the codes
// come out of the cache that the storing left them in).  fp32: storing 336 MB in 61 us, restoring to fp32 110 (3.1 TB/s).  Small calls are bound by their launch: 2.5 and 1.6 us for 2,048 values.

template <typename T>
__global__ __launch_bounds__(256) void k_act_encode(const T *__restrict__ x, ActLayout lay, int64_t ldx, ActGrid g,
                                                    uint64_t seed, uint32_t epoch, uint32_t stream,
                                                    uint8_t *__restrict__ act)
{
    const int tx = threadIdx.x & ((1 << g.tx_log) - 1), ty = threadIdx.x >> g.tx_log, ny = 256 >> g.tx_log;
    for (int64_t b = blockIdx.x; b < g.col_blocks * g.row_blocks; b += gridDim.x) {
        const int64_t rb = b / g.col_blocks, unit = ((b - rb * g.col_blocks) << g.tx_log) + tx;
        if (unit * 8 >= lay.pitch) continue;               // whole groups of four lanes
        const int64_t row0 = rb * (ny * kActRows) + ty;
        float v[kActRows][8];
        // (where all is there the loads stand in no branch of their own, or each would wait for the one before)
        const bool whole = (rb + 1) * (ny * kActRows) <= lay.rows && (unit - tx + (1 << g.tx_log)) * 8 <= lay.cols;
        if (__builtin_expect(whole, 1)) {
#pragma unroll
            for (int q = 0; q < kActRows; ++q) load8(x + (row0 + q * ny) * ldx + unit * 8, 8, v[q]);
        } else {
#pragma unroll
            for (int q = 0; q < kActRows; ++q) {
                const int64_t row = row0 + q * ny;
                load8(x + row * ldx + unit * 8, row < lay.rows ? lay.cols - unit * 8 : 0, v[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < kActRows; ++q) {
            const int64_t row = row0 + q * ny;
            if (!whole && row >= lay.rows) break;
            const ActCodes8 c = act_encode8<T>(v[q], seed, epoch, row, (uint32_t)unit, stream);
            *reinterpret_cast<u32x2 *>(act + row * lay.pitch + unit * 8) = c.codes;
            if ((unit & 3) == 0) act[lay.steps + row * lay.groups + (unit >> 2)] = (uint8_t)c.byte;
        }
    }
}

// THROUGH: the result is written past the caches.
template <typename T, bool THROUGH>
__global__ __launch_bounds__(256) void k_act_decode(const uint8_t *__restrict__ act, ActLayout lay, ActGrid g,
                                                    T *__restrict__ out, int64_t ldo)
{
    const int tx = threadIdx.x & ((1 << g.tx_log) - 1), ty = threadIdx.x >> g.tx_log, ny = 256 >> g.tx_log;
    for (int64_t b = blockIdx.x; b < g.col_blocks * g.row_blocks; b += gridDim.x) {
        const int64_t rb = b / g.col_blocks, unit = ((b - rb * g.col_blocks) << g.tx_log) + tx;
        if (unit * 8 >= lay.cols) continue;
        const int64_t row0 = rb * (ny * kActRows) + ty;
        u32x2 c[kActRows];
        uint32_t byte[kActRows];
#pragma unroll
        for (int q = 0; q < kActRows; ++q) {
            const int64_t row = row0 + q * ny;
            const bool there = row < lay.rows;
            c[q] = there ? *reinterpret_cast<const u32x2 *>(act + row * lay.pitch + unit * 8) : u32x2{0, 0};
            byte[q] = there ? act[lay.steps + row * lay.groups + (unit >> 2)] : 0;
        }
#pragma unroll
        for (int q = 0; q < kActRows; ++q) {
            const int64_t row = row0 + q * ny;
            if (row >= lay.rows) break;
            float v[8];
            act_decode8(c[q], act_step(byte[q]), v);
            store8<THROUGH>(out + row * ldo + unit * 8, lay.cols - unit * 8, v);
        }
    }
}

template <typename T>
static int launch_encode(hipStream_t s, const T *x, const ActLayout &lay, int64_t ldx, uint64_t seed, uint32_t epoch,
                         uint32_t stream, uint8_t *act)
{
    const ActGrid g = act_grid(lay.rows, lay.pitch / 8);
    hipLaunchKernelGGL(k_act_encode<T>, dim3(act_blocks(g)), dim3(256), 0, s, x, lay, ldx, g, seed, epoch, stream, act);
    return hip_check(hipGetLastError());
}

// Results of which the caches would hold little when they are read: 16,384 x 4,096 to bf16 and an elementwise kernel that reads it
// next 74.6 us against 78.4 (storing and restoring alone 67 against 75).  Smaller ones are faster to restore too (8,192 x 4,096 15.5 us
// against 16.3), but slower to read next (37.9 against 36.2 for both).
constexpr int64_t kThroughLeast = 96ll << 20;

template <typename T>
static int launch_decode(hipStream_t s, const uint8_t *act, const ActLayout &lay, T *out, int64_t ldo)
{
    const ActGrid g = act_grid(lay.rows, lay.pitch / 8);
    const auto k = lay.rows * lay.cols * (int64_t)sizeof(T) > kThroughLeast ? k_act_decode<T, true> : k_act_decode<T, false>;
    hipLaunchKernelGGL(k, dim3(act_blocks(g)), dim3(256), 0, s, act, lay, g, out, ldo);
    return hip_check(hipGetLastError());
}

}  // namespace zipml

using namespace zipml;

extern "C" size_t zipml_act_bytes(int64_t rows, int64_t cols)
{
    return act_sizes_ok(rows, cols) ? act_layout(rows, cols).bytes() : 0;
}

extern "C" int zipml_act_encode(void *stream, const void *x_dev, int dtype, int64_t rows, int64_t cols, int64_t ldx,
                                uint64_t seed, uint32_t epoch, int tag, void *act_dev)
{
    if (!x_dev || !act_dev || !act_sizes_ok(rows, cols) || ldx < cols || ldx > (1ll << 60) / rows || !valid_dtype(dtype))
        return ZIPML_EINVAL;
    if (epoch >= (1u << 24) || tag < 0 || tag > kActMaxTag) return ZIPML_EINVAL;
    if (!aligned16(x_dev) || !aligned16(act_dev)) return ZIPML_EALIGN;
    const ActLayout lay = act_layout(rows, cols);
    hipStream_t s = entry_stream(stream);
    if (dtype == ZIPML_F32)
        return launch_encode(s, (const float *)x_dev, lay, ldx, seed, epoch, kActStream + tag, (uint8_t *)act_dev);
    return launch_encode(s, (const __bf16 *)x_dev, lay, ldx, seed, epoch, kActStream + tag, (uint8_t *)act_dev);
}

extern "C" int zipml_act_decode(void *stream, const void *act_dev, int64_t rows, int64_t cols, void *out_dev, int dtype,
                                int64_t ldo)
{
    if (!act_dev || !out_dev || !act_sizes_ok(rows, cols) || ldo < cols || ldo > (1ll << 60) / rows || !valid_dtype(dtype))
        return ZIPML_EINVAL;
    if (!aligned16(act_dev) || !aligned16(out_dev)) return ZIPML_EALIGN;
    const ActLayout lay = act_layout(rows, cols);
    hipStream_t s = entry_stream(stream);
    if (dtype == ZIPML_F32) return launch_decode(s, (const uint8_t *)act_dev, lay, (float *)out_dev, ldo);
    return launch_decode(s, (const uint8_t *)act_dev, lay, (__bf16 *)out_dev, ldo);
}
