// Linear layer on 8-bit codes: y[t][o] = (sum_i x[t][i] w[o][i]) sx[t] sw[o] + bias[o], x and w codes with a scale a row.
//
// The sums are integers: exact in any order (|code| <= 128 and d_in < 2^17 keep them in 32 bits), so how the contraction is split
// changes no bit of the result.  Both operands are contracted along their rows, 16 codes of a row are 16 bytes, and a lane of
// v_mfma_i32_32x32x32_i8 wants just those of one row: tiles lie in LDS as they lie in memory, and are read 16 bytes at a time.
#include "zipml_row8.h"

namespace zipml {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

struct ProductArgs {
    const uint8_t *x, *w;
    const float *sx, *sw, *bias;
    void *y;
    int64_t ldx, ldw, ldy, rows;
    int d_out, bytes;           // bytes: of a row, padding included
    int tiles_t, tiles_o;
};

constexpr int kStep = 128;      // codes of a row that are in LDS at a time

// Rows of codes as a buffer: rows behind the last one, and what lies behind a row's padding, read as zeros.
struct CodeRows {
    __amdgpu_buffer_rsrc_t r;
    int ld, bytes;
    __device__ __forceinline__ CodeRows(const uint8_t *base, int64_t left, int64_t ld_, int bytes_) : ld((int)ld_), bytes(bytes_)
    {
        const int64_t n = (left - 1) * ld_ + bytes_;
        r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), 0, left < 1 ? 0 : n > 0x7FFFFF00 ? 0x7FFFFF00 : (int)n, 0x00020000);
    }
    __device__ __forceinline__ u32x4 load16(int row, int at) const
    {
        return __builtin_amdgcn_raw_buffer_load_b128(r, at < bytes ? row * ld + at : 0x7FFFFFF0, 0, 0);
    }
};

// MO x MT outputs x tokens of a workgroup, WO x WT waves.
template <int MO_, int MT_, int WO_, int WT_>
struct ProductShape {
    static constexpr int MO = MO_, MT = MT_, WO = WO_, WT = WT_, kThreads = 64 * WO * WT;
    static constexpr int TO = MO / WO / 32, TT = MT / WT / 32;
    static constexpr int kLoadsW = MO * kStep / 16 / kThreads, kLoadsX = MT * kStep / 16 / kThreads;
    static constexpr int kStage = (MO + MT) * kStep, kLds = 2 * kStage;
    static_assert(kLoadsW * 16 * kThreads == MO * kStep && kLoadsX * 16 * kThreads == MT * kStep, "whole loads");
};

// Where the 16 bytes `chunk` of a row lie in an LDS tile: turned by the row's number, so that 16 rows' same chunk, which 16 lanes
// read at once, fall on all banks.
__device__ __forceinline__ int lds_at(int row, int chunk) { return row * kStep + ((chunk ^ (row >> 1 & 7)) << 4); }

template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void k_row8_product(ProductArgs a)
{
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tile_o = blockIdx.x % a.tiles_o, tile_t = blockIdx.x / a.tiles_o;
    const int o0 = tile_o * S::MO;
    const int64_t t0 = (int64_t)tile_t * S::MT;
    const CodeRows w(a.w + o0 * a.ldw, a.d_out - o0, a.ldw, a.bytes), x(a.x + t0 * a.ldx, a.rows - t0, a.ldx, a.bytes);

    u32x4 vw[S::kLoadsW], vx[S::kLoadsX];
    auto load = [&](int k0) {
#pragma unroll
        for (int q = 0; q < S::kLoadsW; ++q) {
            const int c = tid + q * S::kThreads;
            vw[q] = w.load16(c >> 3, k0 + (c & 7) * 16);
        }
#pragma unroll
        for (int q = 0; q < S::kLoadsX; ++q) {
            const int c = tid + q * S::kThreads;
            vx[q] = x.load16(c >> 3, k0 + (c & 7) * 16);
        }
    };
    auto store = [&](char *stage) {
#pragma unroll
        for (int q = 0; q < S::kLoadsW; ++q) {
            const int c = tid + q * S::kThreads;
            *reinterpret_cast<u32x4 *>(stage + lds_at(c >> 3, c & 7)) = vw[q];
        }
#pragma unroll
        for (int q = 0; q < S::kLoadsX; ++q) {
            const int c = tid + q * S::kThreads;
            *reinterpret_cast<u32x4 *>(stage + S::MO * kStep + lds_at(c >> 3, c & 7)) = vx[q];
        }
    };

    const int wo = wave / S::WT, wt = wave % S::WT;
    i32x16 acc[S::TO][S::TT] = {};
    load(0);
    store(lds);
    char *here = lds, *next = lds + S::kStage;
    for (int k0 = 0; k0 < a.bytes; k0 += kStep) {
        load(k0 + kStep);
        lds_barrier();
#pragma unroll
        for (int s = 0; s < kStep / 32; ++s) {
            const int chunk = 2 * s + (lane >> 5);
            i32x4 fw[S::TO], fx[S::TT];
#pragma unroll
            for (int m = 0; m < S::TO; ++m)
                fw[m] = *reinterpret_cast<const i32x4 *>(here + lds_at((wo * S::TO + m) * 32 + (lane & 31), chunk));
#pragma unroll
            for (int n = 0; n < S::TT; ++n)
                fx[n] = *reinterpret_cast<const i32x4 *>(here + S::MO * kStep + lds_at((wt * S::TT + n) * 32 + (lane & 31), chunk));
#pragma unroll
            for (int m = 0; m < S::TO; ++m)
#pragma unroll
                for (int n = 0; n < S::TT; ++n) acc[m][n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[m], fx[n], acc[m][n], 0, 0, 0);
        }
        store(next);
        char *const t = here;
        here = next;
        next = t;
    }

    // a lane holds four neighbouring outputs of one token at a time
    T *const y = (T *)a.y;
#pragma unroll
    for (int n = 0; n < S::TT; ++n) {
        const int64_t t = t0 + (wt * S::TT + n) * 32 + (lane & 31);
        if (t >= a.rows) continue;
        const float sx = a.sx[t];
#pragma unroll
        for (int m = 0; m < S::TO; ++m)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int o = o0 + (wo * S::TO + m) * 32 + 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3);
                if (o >= a.d_out) continue;
                const float v = (float)acc[m][n][q] * sx * a.sw[o];
                y[t * a.ldy + o] = (T)(a.bias ? v + a.bias[o] : v);
            }
    }
}

template <typename T, typename S>
static int launch_product(hipStream_t s, ProductArgs a)
{
    a.tiles_o = (a.d_out + S::MO - 1) / S::MO;
    const int64_t tiles = (a.rows + S::MT - 1) / S::MT;
    if (tiles * a.tiles_o > 0x7FFFFFFF) return ZIPML_EINVAL;
    a.tiles_t = (int)tiles;
    static std::atomic<uint64_t> done;
    const auto k = k_row8_product<T, S>;
    if (allow_lds((const void *)k, S::kLds, done)) return ZIPML_ELAUNCH;
    hipLaunchKernelGGL(k, dim3((uint32_t)(tiles * a.tiles_o)), dim3(S::kThreads), S::kLds, s, a);
    return hip_check(hipGetLastError());
}

}  // namespace zipml

using namespace zipml;

static bool product_sizes_ok(int64_t rows, int64_t d_out, int64_t d_in)
{
    return rows > 0 && d_out > 0 && d_in > 0 && rows <= (1ll << 31) && d_out <= (1 << 24) && d_in <= (1ll << 40) && rows <= (1ll << 40) / d_out;
}
constexpr int64_t kProductMaxIn = 131071;      // 128 * 128 * d_in < 2^31

extern "C" size_t zipml_row8_product_workspace_bytes(int64_t rows, int64_t d_out, int64_t d_in)
{
    return product_sizes_ok(rows, d_out, d_in) && d_in <= kProductMaxIn ? 256 : 0;
}

extern "C" int zipml_row8_product(void *stream, const void *x_dev, int64_t ldx, const float *x_scales_dev, const void *w_dev,
                                  int64_t ldw, const float *w_scales_dev, const float *bias_dev, int64_t rows, int64_t d_out,
                                  int64_t d_in, void *y_dev, int dtype, int64_t ldy, void *workspace_dev, size_t workspace_bytes)
{
    if (!x_dev || !x_scales_dev || !w_dev || !w_scales_dev || !y_dev || !valid_dtype(dtype) || !product_sizes_ok(rows, d_out, d_in))
        return ZIPML_EINVAL;
    if (!row8_pitch_ok(rows, d_in, ldx) || !row8_pitch_ok(d_out, d_in, ldw) || ldx > kRow8MaxPitch || ldw > kRow8MaxPitch ||
        ldy < d_out || ldy > (1ll << 60) / rows)
        return ZIPML_EINVAL;
    if (d_in > kProductMaxIn) return ZIPML_ERANGE;
    if (!workspace_dev || workspace_bytes < zipml_row8_product_workspace_bytes(rows, d_out, d_in)) return ZIPML_EWORKSPACE;
    if (!aligned16(x_dev) || !aligned16(w_dev) || !aligned16(y_dev) || !aligned16(workspace_dev) || !aligned4(x_scales_dev) ||
        !aligned4(w_scales_dev) || !aligned4(bias_dev))
        return ZIPML_EALIGN;
    ProductArgs a{(const uint8_t *)x_dev, (const uint8_t *)w_dev, x_scales_dev, w_scales_dev, bias_dev, y_dev, ldx, ldw, ldy, rows,
                  (int)d_out, (int)round_up(d_in, kRow8Unit), 0, 0};
    hipStream_t s = entry_stream(stream);
    typedef ProductShape<128, 128, 2, 2> S;
    return dtype == ZIPML_F32 ? launch_product<float, S>(s, a) : launch_product<__bf16, S>(s, a);
}
