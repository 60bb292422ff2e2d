// Gated linear recurrence  h_t = f_t h_{t-1} + (1 - f_t) x_t,  f = sigmoid(z): packed sequences, forward and backward.
//
// Both directions are scans of pairs: a run of tokens takes a state h to A h + B, and two runs one after the other
// to (A2 A1) h + (A2 B1 + B2).  A workgroup owns 64 channels and kBlock tokens: eight lanes side by side take eight
// channels each (128 bytes of a bf16 row), 32 such rows of lanes take eight tokens each, which a thread walks through in
// registers.  The rows of lanes are joined by shuffles and LDS, the blocks by the pairs in global memory.
//
// A = 0 marks a run that contains the start of a sequence (or lies outside all): what is before it does not matter, and
// is not multiplied, so that a NaN or an infinity of one sequence never reaches the next.  Every other A is kept at
// 2^-126 or more, so that within a sequence they do pass on; what that adds to a state is below 2^-126 of it.
#include "zipml_act.h"

namespace zipml {

constexpr int kBlock = ZIPML_SCAN_BLOCK;   // tokens of a workgroup
constexpr int kCh = 64;                    // channels of a workgroup
constexpr int kRun = 8;                    // tokens of a thread
constexpr int kSubs = kBlock / kRun;       // rows of lanes
constexpr int kThreads = kSubs * kCh / 8;
constexpr int kWaves = kThreads / kWave;
constexpr float kTiny = 1.17549435e-38f;
constexpr float kZMax = 16.0f;             // gates are stored clamped to +-kZMax: sigmoid(16) is 1 - 2^-23.1

struct ScanArgs {
    const void *x, *z;                     // forward
    void *y;
    int64_t ldx, ldz, ldy;
    const uint8_t *rx, *rz;                // backward: stored inputs
    uint8_t *wx, *wz;                      // forward: where they are stored, or NULL
    ActLayout lay;
    float *states;                         // states before each block, or NULL (forward)
    const void *dy;
    void *dx, *dz;
    int64_t lddy, lddx, lddz;
    const int64_t *seq_start;              // n_seq + 1 offsets, or NULL: one sequence
    const float *h0, *dh_last;
    float *h_last, *dh0;
    float2 *pairs;                         // [blocks][channels]: of each block, then the states that enter it
    uint64_t seed;
    uint32_t epoch, stream;
    int64_t tokens, channels, n_seq, blocks, groups;
};

// sigmoid(z) and sigmoid(-z), neither by subtraction.
__device__ __forceinline__ void gates(float z, float &f, float &g)
{
    const float e = __expf(-__builtin_fabsf(z));
    const float q = __builtin_amdgcn_rcpf(1.0f + e), eq = e * q;
    f = z >= 0.0f ? q : eq;
    g = z >= 0.0f ? eq : q;
}

__device__ __forceinline__ float join(float a, float prev, float b) { return a == 0.0f ? b : __builtin_fmaf(a, prev, b); }
__device__ __forceinline__ float times(float a, float b) { return a == 0.0f || b == 0.0f ? 0.0f : __builtin_fmaxf(a * b, kTiny); }

// Which of the block's tokens are a sequence's first and last.
struct BlockMap {
    int first[kBlock], last[kBlock];       // the sequence, or -1
    int some;                              // any token is either, or outside
};
struct Range { int64_t begin, end; };      // tokens inside sequences

__device__ __forceinline__ Range block_map(const ScanArgs &a, int64_t blk, BlockMap &m)
{
    for (int i = threadIdx.x; i < kBlock; i += kThreads) m.first[i] = m.last[i] = -1;
    if (threadIdx.x == 0) m.some = 0;
    __syncthreads();
    const int64_t t0 = blk * kBlock;
    Range r{0, a.tokens};
    if (a.seq_start) {
        r.begin = a.seq_start[0];
        r.end = a.seq_start[a.n_seq];
        r.end = r.end > a.tokens ? a.tokens : r.end;
    }
    auto mark = [&](int64_t s, int64_t p, int64_t q) {
        if (p >= q) return;
        if (p >= t0 && p < t0 + kBlock) { m.first[p - t0] = (int)s; m.some = 1; }
        if (q > t0 && q <= t0 + kBlock) { m.last[q - 1 - t0] = (int)s; m.some = 1; }
    };
    if (a.seq_start) {
        for (int64_t s = threadIdx.x; s < a.n_seq; s += kThreads) mark(s, a.seq_start[s], a.seq_start[s + 1]);
    } else if (threadIdx.x == 0) {
        mark(0, 0, a.tokens);
    }
    if (threadIdx.x == 0 && (r.begin > t0 || r.end < t0 + kBlock)) m.some = 1;
    __syncthreads();
    return r;
}

// Eight floats of a row of `channels`, zeros beyond it or without the row.
__device__ __forceinline__ void load_row(const float *row, int64_t left, float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = row && k < left ? row[k] : 0.0f;
}
__device__ __forceinline__ void store_row(float *row, int64_t left, const float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < left) row[k] = v[k];
}

// Pair of all runs before this thread's in its block (REVERSE: behind it), from each thread's own pair; total: of
// the whole block.
template <bool REVERSE>
__device__ __forceinline__ void block_scan(float (&A)[8], float (&B)[8], float2 (&lds)[kWaves][kCh], float (&tA)[8],
                                           float (&tB)[8])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cl = lane & 7;
    const int pos = REVERSE ? 7 - (lane >> 3) : lane >> 3;
#pragma unroll
    for (int s = 1; s < 8; s <<= 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int from = REVERSE ? lane + 8 * s : lane - 8 * s;
            const float pa = __shfl(A[k], from & 63, 64), pb = __shfl(B[k], from & 63, 64);
            if (pos >= s) {
                B[k] = join(A[k], pb, B[k]);
                A[k] = times(A[k], pa);
            }
        }
    }
    __syncthreads();                       // (whatever was read from lds before)
    if (pos == 7)
#pragma unroll
        for (int k = 0; k < 8; ++k) lds[wave][cl * 8 + k] = float2{A[k], B[k]};
#pragma unroll
    for (int k = 0; k < 8; ++k) {          // of the runs before this one
        const int from = (REVERSE ? lane + 8 : lane - 8) & 63;
        const float pa = __shfl(A[k], from, 64), pb = __shfl(B[k], from, 64);
        A[k] = pos == 0 ? 1.0f : pa;
        B[k] = pos == 0 ? 0.0f : pb;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        float wa = 1.0f, wb = 0.0f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            const int w = REVERSE ? kWaves - 1 - i : i;
            const float2 p = lds[w][cl * 8 + k];
            if (w == wave) {               // (uniform over a wave)
                B[k] = join(A[k], wb, B[k]);
                A[k] = times(A[k], wa);
            }
            wb = join(p.x, wb, p.y);
            wa = times(p.x, wa);
        }
        tA[k] = wa;
        tB[k] = wb;
    }
}

// What both passes of the forward direction need: the pair (a, b) of each of the thread's tokens.
__device__ __forceinline__ void forward_tokens(const ScanArgs &p, const BlockMap &m, Range r, int64_t t0, int sub, int64_t c,
                                               const float (&x)[kRun][8], float (&a)[kRun][8], float (&b)[kRun][8])
{
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float f, g;
            gates(a[j][k], f, g);
            a[j][k] = f;
            b[j][k] = g * x[j][k];
        }
    }
    if (!m.some) return;
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
        const int64_t t = t0 + sub * kRun + j;
        const int s = m.first[sub * kRun + j];
        if (t < r.begin || t >= r.end) {
#pragma unroll
            for (int k = 0; k < 8; ++k) a[j][k] = b[j][k] = 0.0f;
        } else if (s >= 0) {
            float h[8];
            load_row(p.h0 ? p.h0 + s * p.channels + c : nullptr, p.channels - c, h);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                b[j][k] = p.h0 ? __builtin_fmaf(a[j][k], h[k], b[j][k]) : b[j][k];
                a[j][k] = 0.0f;
            }
        }
    }
}

// APPLY = false: the pair of each block.  APPLY = true: states, from what enters the block.
template <typename T, bool APPLY>
__global__ __launch_bounds__(kThreads, 2) void k_scan_forward(ScanArgs p)
{
    __shared__ BlockMap map;
    __shared__ float2 lds[kWaves][kCh];
    const int64_t blk = blockIdx.x / p.groups, c0 = (blockIdx.x - blk * p.groups) * kCh;
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 3;
    const int64_t c = c0 + (lane & 7) * 8, left = p.channels - c, t0 = blk * kBlock;
    const Range r = block_map(p, blk, map);

    float x[kRun][8], a[kRun][8], b[kRun][8];
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
        const int64_t t = t0 + sub * kRun + j;
        const int64_t n = t < p.tokens ? left : 0;
        load8((const T *)p.x + t * p.ldx + c, n, x[j]);
        load8((const T *)p.z + t * p.ldz + c, n, a[j]);
    }
    if (APPLY && p.wx) {
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int64_t t = t0 + sub * kRun + j;
            float zc[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) zc[k] = a[j][k] > kZMax ? kZMax : a[j][k] < -kZMax ? -kZMax : a[j][k];
            const ActCodes8 cx = act_encode8(x[j], p.seed, p.epoch, t, (uint32_t)(c >> 3), p.stream);
            const ActCodes8 cz = act_encode8(zc, p.seed, p.epoch, t, (uint32_t)(c >> 3), p.stream + 1);
            if (t < p.tokens && c < p.lay.pitch) {
                *reinterpret_cast<u32x2 *>(p.wx + t * p.lay.pitch + c) = cx.codes;
                *reinterpret_cast<u32x2 *>(p.wz + t * p.lay.pitch + c) = cz.codes;
                if ((lane & 3) == 0) {
                    p.wx[p.lay.steps + t * p.lay.groups + (c >> 5)] = (uint8_t)cx.byte;
                    p.wz[p.lay.steps + t * p.lay.groups + (c >> 5)] = (uint8_t)cz.byte;
                }
            }
        }
    }
    forward_tokens(p, map, r, t0, sub, c, x, a, b);

    float A[8], B[8], tA[8], tB[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) { A[k] = 1.0f; B[k] = 0.0f; }
#pragma unroll
    for (int j = 0; j < kRun; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            B[k] = join(a[j][k], B[k], b[j][k]);
            A[k] = times(a[j][k], A[k]);
        }
    block_scan<false>(A, B, lds, tA, tB);

    if constexpr (!APPLY) {
        if (sub == 0)
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) p.pairs[blk * p.channels + c + k] = float2{tA[k], tB[k]};
    } else {
        float h[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float in = k < left && p.blocks > 1 ? p.pairs[blk * p.channels + c + k].y : 0.0f;
            if (sub == 0 && p.states && k < left) p.states[blk * p.channels + c + k] = in;
            h[k] = join(A[k], in, B[k]);
        }
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int64_t t = t0 + sub * kRun + j;
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] = join(a[j][k], h[k], b[j][k]);
            if (t < p.tokens) store8((T *)p.y + t * p.ldy + c, left, h);
            if (p.h_last && map.some && map.last[sub * kRun + j] >= 0)
                store_row(p.h_last + (int64_t)map.last[sub * kRun + j] * p.channels + c, left, h);
        }
        // empty sequences hand their states on
        if (p.h_last && p.seq_start)
            for (int64_t s = blk * kWaves + (threadIdx.x >> 6); s < p.n_seq; s += p.blocks * kWaves)
                if (p.seq_start[s] >= p.seq_start[s + 1] && c0 + lane < p.channels)
                    p.h_last[s * p.channels + c0 + lane] = p.h0 ? p.h0[s * p.channels + c0 + lane] : 0.0f;
    }
}

// From the blocks' pairs to the states that enter them, in y; REVERSE: from the last block to the first.
template <bool REVERSE>
__global__ __launch_bounds__(64) void k_scan_blocks(float2 *pairs, int64_t blocks, int64_t channels)
{
    const int64_t c = blockIdx.x * 64ll + threadIdx.x;
    if (c >= channels) return;
    float h = 0.0f;
    for (int64_t i = 0; i < blocks; ++i) {
        float2 *q = pairs + (REVERSE ? blocks - 1 - i : i) * channels + c;
        const float2 v = *q;
        q->y = h;
        h = join(v.x, h, v.y);
    }
}

template <typename T, bool APPLY>
__global__ __launch_bounds__(kThreads, 2) void k_scan_backward(ScanArgs p)
{
    __shared__ BlockMap map;
    __shared__ float2 lds[kWaves][kCh];
    const int64_t blk = blockIdx.x / p.groups, c0 = (blockIdx.x - blk * p.groups) * kCh;
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 3;
    const int64_t c = c0 + (lane & 7) * 8, left = p.channels - c, t0 = blk * kBlock;
    const Range r = block_map(p, blk, map);

    u32x2 qx[kRun], qz[kRun];
    uint32_t ex[kRun], ez[kRun];
    float d[kRun][8], f[kRun][8], g[kRun][8];
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
        const int64_t t = t0 + sub * kRun + j;
        const bool there = t < p.tokens && c < p.lay.pitch;
        const int64_t at = t * p.lay.pitch + c, step = p.lay.steps + t * p.lay.groups + (c >> 5);
        qz[j] = there ? *reinterpret_cast<const u32x2 *>(p.rz + at) : u32x2{0, 0};
        ez[j] = there ? p.rz[step] : 0u;
        if (APPLY) {
            qx[j] = there ? *reinterpret_cast<const u32x2 *>(p.rx + at) : u32x2{0, 0};
            ex[j] = there ? p.rx[step] : 0u;
        }
        load8((const T *)p.dy + t * p.lddy + c, t < p.tokens ? left : 0, d[j]);
    }
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
        float z[8];
        act_decode8(qz[j], act_step(ez[j]), z);
#pragma unroll
        for (int k = 0; k < 8; ++k) gates(z[k], f[j][k], g[j][k]);
    }
    // whether a token is outside all sequences, its sequence's last, its first
    auto outside = [&](int j) { const int64_t t = t0 + sub * kRun + j; return map.some && (t < r.begin || t >= r.end); };
    auto last = [&](int j) { return map.some && map.last[sub * kRun + j] >= 0; };
    auto first = [&](int j) { return map.some && map.first[sub * kRun + j] >= 0; };

    // p_t = f_t (d_t + p_{t+1}) from right to left
    float A[8], B[8], tA[8], tB[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) { A[k] = 1.0f; B[k] = 0.0f; }
#pragma unroll
    for (int j = kRun - 1; j >= 0; --j) {
        if (outside(j)) {
#pragma unroll
            for (int k = 0; k < 8; ++k) A[k] = B[k] = 0.0f;
            continue;
        }
        if (last(j)) {
            float h[8];
            load_row(p.dh_last ? p.dh_last + (int64_t)map.last[sub * kRun + j] * p.channels + c : nullptr, left, h);
#pragma unroll
            for (int k = 0; k < 8; ++k) { d[j][k] += h[k]; A[k] = B[k] = 0.0f; }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            B[k] = f[j][k] * (d[j][k] + B[k]);
            A[k] = A[k] == 0.0f ? 0.0f : __builtin_fmaxf(f[j][k] * A[k], kTiny);
        }
    }
    block_scan<true>(A, B, lds, tA, tB);
    if constexpr (!APPLY) {
        if (sub == 0)
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) p.pairs[blk * p.channels + c + k] = float2{tA[k], tB[k]};
        return;
    } else {
        float q[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float in = k < left && p.blocks > 1 ? p.pairs[blk * p.channels + c + k].y : 0.0f;
            q[k] = join(A[k], in, B[k]);
        }
        // d becomes the gradient of each state
#pragma unroll
        for (int j = kRun - 1; j >= 0; --j) {
            if (outside(j)) {
#pragma unroll
                for (int k = 0; k < 8; ++k) d[j][k] = q[k] = 0.0f;
                continue;
            }
            const bool end = last(j);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                d[j][k] = end ? d[j][k] : d[j][k] + q[k];
                q[k] = f[j][k] * d[j][k];
            }
            if (p.dh0 && first(j)) store_row(p.dh0 + (int64_t)map.first[sub * kRun + j] * p.channels + c, left, q);
        }

        // the states again, from the one that the forward pass kept
#pragma unroll
        for (int k = 0; k < 8; ++k) { A[k] = 1.0f; B[k] = 0.0f; }
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            float x[8];
            act_decode8(qx[j], act_step(ex[j]), x);
            if (first(j) || outside(j)) {
                float h[8];
                load_row(p.h0 && first(j) ? p.h0 + (int64_t)map.first[sub * kRun + j] * p.channels + c : nullptr, left, h);
                const bool out = outside(j);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    A[k] = 0.0f;
                    B[k] = out ? 0.0f : __builtin_fmaf(f[j][k], h[k], g[j][k] * x[k]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    B[k] = __builtin_fmaf(f[j][k], B[k], g[j][k] * x[k]);
                    A[k] = A[k] == 0.0f ? 0.0f : __builtin_fmaxf(f[j][k] * A[k], kTiny);
                }
            }
        }
        block_scan<false>(A, B, lds, tA, tB);
        float h[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) h[k] = join(A[k], k < left ? p.states[blk * p.channels + c + k] : 0.0f, B[k]);
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int64_t t = t0 + sub * kRun + j;
            float x[8], dx[8], dz[8];
            act_decode8(qx[j], act_step(ex[j]), x);
            const bool out = outside(j);
            if (first(j)) load_row(p.h0 ? p.h0 + (int64_t)map.first[sub * kRun + j] * p.channels + c : nullptr, left, h);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                dx[k] = out ? 0.0f : g[j][k] * d[j][k];
                dz[k] = out ? 0.0f : f[j][k] * dx[k] * (h[k] - x[k]);
                h[k] = out ? 0.0f : __builtin_fmaf(f[j][k], h[k], g[j][k] * x[k]);
            }
            if (t < p.tokens) {
                store8((T *)p.dx + t * p.lddx + c, left, dx);
                store8((T *)p.dz + t * p.lddz + c, left, dz);
            }
        }
        // empty sequences hand their gradients on
        if (p.dh0 && p.seq_start)
            for (int64_t s = blk * kWaves + (threadIdx.x >> 6); s < p.n_seq; s += p.blocks * kWaves)
                if (p.seq_start[s] >= p.seq_start[s + 1] && c0 + lane < p.channels)
                    p.dh0[s * p.channels + c0 + lane] = p.dh_last ? p.dh_last[s * p.channels + c0 + lane] : 0.0f;
    }
}

// One token of each of `rows` requests: the state in slot slots[row] (or row) of the pool is taken one step on.
template <typename T>
__global__ __launch_bounds__(256) void k_scan_step(const T *__restrict__ x, int64_t ldx, const T *__restrict__ z, int64_t ldz,
                                                   int64_t rows, int64_t channels, float *h, int64_t n_slots,
                                                   const int32_t *__restrict__ slots, T *__restrict__ y, int64_t ldy)
{
    const int64_t units = (channels + 7) / 8, i = blockIdx.x * 256ll + threadIdx.x;
    if (i >= rows * units) return;
    const int64_t row = i / units, c = (i - row * units) * 8, left = channels - c;
    const int64_t slot = slots ? slots[row] : row;
    float v[8] = {};
    if (slot >= 0 && slot < n_slots) {
        float xv[8], zv[8];
        load8(x + row * ldx + c, left, xv);
        load8(z + row * ldz + c, left, zv);
        float *s = h + slot * channels + c;
        load_row(s, left, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float f, g;
            gates(zv[k], f, g);
            v[k] = __builtin_fmaf(f, v[k], g * xv[k]);
        }
        store_row(s, left, v);
    }
    store8(y + row * ldy + c, left, v);
}

static int64_t scan_blocks(int64_t tokens) { return (tokens + kBlock - 1) / kBlock; }
static bool scan_sizes_ok(int64_t tokens, int64_t channels)
{
    return act_sizes_ok(tokens, channels) && scan_blocks(tokens) * ((channels + kCh - 1) / kCh) <= (1ll << 31) - 1;
}
static bool stride_ok(int64_t ld, int64_t rows, int64_t cols) { return ld >= cols && ld <= (1ll << 60) / rows; }

template <typename T>
static int launch_forward(hipStream_t s, const ScanArgs &p)
{
    const dim3 grid((uint32_t)(p.blocks * p.groups));
    if (p.blocks > 1) {
        hipLaunchKernelGGL((k_scan_forward<T, false>), grid, dim3(kThreads), 0, s, p);
        hipLaunchKernelGGL(k_scan_blocks<false>, dim3((uint32_t)((p.channels + 63) / 64)), dim3(64), 0, s, p.pairs, p.blocks,
                           p.channels);
    }
    hipLaunchKernelGGL((k_scan_forward<T, true>), grid, dim3(kThreads), 0, s, p);
    return hip_check(hipGetLastError());
}
template <typename T>
static int launch_backward(hipStream_t s, const ScanArgs &p)
{
    const dim3 grid((uint32_t)(p.blocks * p.groups));
    if (p.blocks > 1) {
        hipLaunchKernelGGL((k_scan_backward<T, false>), grid, dim3(kThreads), 0, s, p);
        hipLaunchKernelGGL(k_scan_blocks<true>, dim3((uint32_t)((p.channels + 63) / 64)), dim3(64), 0, s, p.pairs, p.blocks,
                           p.channels);
    }
    hipLaunchKernelGGL((k_scan_backward<T, true>), grid, dim3(kThreads), 0, s, p);
    return hip_check(hipGetLastError());
}

}  // namespace zipml

using namespace zipml;

extern "C" size_t zipml_scan_workspace_bytes(int64_t tokens, int64_t channels)
{
    if (!scan_sizes_ok(tokens, channels)) return 0;
    const int64_t blocks = scan_blocks(tokens);
    return blocks > 1 ? (size_t)blocks * (size_t)channels * sizeof(float2) : 256;
}

extern "C" int zipml_scan_forward(void *stream, const void *x_dev, int64_t ldx, const void *z_dev, int64_t ldz, int dtype,
                                  int64_t tokens, int64_t channels, const int64_t *seq_start_dev, int64_t n_seq,
                                  const float *h0_dev, void *y_dev, int64_t ldy, float *h_last_dev, void *act_x_dev,
                                  void *act_z_dev, float *states_dev, uint64_t seed, uint32_t epoch, int tag,
                                  void *workspace_dev, size_t workspace_bytes)
{
    if (!x_dev || !z_dev || !y_dev || !valid_dtype(dtype) || !scan_sizes_ok(tokens, channels)) return ZIPML_EINVAL;
    if (!stride_ok(ldx, tokens, channels) || !stride_ok(ldz, tokens, channels) || !stride_ok(ldy, tokens, channels))
        return ZIPML_EINVAL;
    if (n_seq < 1 || n_seq > (1ll << 31) - 1 || (!seq_start_dev && n_seq != 1)) return ZIPML_EINVAL;
    const bool train = act_x_dev || act_z_dev || states_dev;
    if (train && !(act_x_dev && act_z_dev && states_dev)) return ZIPML_EINVAL;
    if (epoch >= (1u << 24) || tag < 0 || tag >= kActMaxTag) return ZIPML_EINVAL;
    if (!workspace_dev || workspace_bytes < zipml_scan_workspace_bytes(tokens, channels)) return ZIPML_EWORKSPACE;
    if (!aligned16(x_dev) || !aligned16(z_dev) || !aligned16(y_dev) || !aligned16(seq_start_dev) || !aligned16(h0_dev) ||
        !aligned16(h_last_dev) || !aligned16(act_x_dev) || !aligned16(act_z_dev) || !aligned16(states_dev) ||
        !aligned16(workspace_dev))
        return ZIPML_EALIGN;
    ScanArgs p{};
    p.x = x_dev; p.z = z_dev; p.y = y_dev;
    p.ldx = ldx; p.ldz = ldz; p.ldy = ldy;
    p.wx = (uint8_t *)act_x_dev; p.wz = (uint8_t *)act_z_dev; p.states = states_dev;
    p.lay = act_layout(tokens, channels);
    p.seq_start = seq_start_dev; p.h0 = h0_dev; p.h_last = h_last_dev;
    p.pairs = (float2 *)workspace_dev;
    p.seed = seed; p.epoch = epoch; p.stream = kActStream + tag;
    p.tokens = tokens; p.channels = channels; p.n_seq = n_seq;
    p.blocks = scan_blocks(tokens); p.groups = (channels + kCh - 1) / kCh;
    hipStream_t s = entry_stream(stream);
    return dtype == ZIPML_F32 ? launch_forward<float>(s, p) : launch_forward<__bf16>(s, p);
}

extern "C" int zipml_scan_backward(void *stream, const void *act_x_dev, const void *act_z_dev, const float *states_dev,
                                   const void *dy_dev, int64_t lddy, int dtype, int64_t tokens, int64_t channels,
                                   const int64_t *seq_start_dev, int64_t n_seq, const float *h0_dev,
                                   const float *dh_last_dev, void *dx_dev, int64_t lddx, void *dz_dev, int64_t lddz,
                                   float *dh0_dev, void *workspace_dev, size_t workspace_bytes)
{
    if (!act_x_dev || !act_z_dev || !states_dev || !dy_dev || !dx_dev || !dz_dev || !valid_dtype(dtype) ||
        !scan_sizes_ok(tokens, channels))
        return ZIPML_EINVAL;
    if (!stride_ok(lddy, tokens, channels) || !stride_ok(lddx, tokens, channels) || !stride_ok(lddz, tokens, channels))
        return ZIPML_EINVAL;
    if (n_seq < 1 || n_seq > (1ll << 31) - 1 || (!seq_start_dev && n_seq != 1)) return ZIPML_EINVAL;
    if (!workspace_dev || workspace_bytes < zipml_scan_workspace_bytes(tokens, channels)) return ZIPML_EWORKSPACE;
    if (!aligned16(act_x_dev) || !aligned16(act_z_dev) || !aligned16(states_dev) || !aligned16(dy_dev) ||
        !aligned16(seq_start_dev) || !aligned16(h0_dev) || !aligned16(dh_last_dev) || !aligned16(dx_dev) ||
        !aligned16(dz_dev) || !aligned16(dh0_dev) || !aligned16(workspace_dev))
        return ZIPML_EALIGN;
    ScanArgs p{};
    p.rx = (const uint8_t *)act_x_dev; p.rz = (const uint8_t *)act_z_dev;
    p.states = const_cast<float *>(states_dev);
    p.lay = act_layout(tokens, channels);
    p.dy = dy_dev; p.dx = dx_dev; p.dz = dz_dev;
    p.lddy = lddy; p.lddx = lddx; p.lddz = lddz;
    p.seq_start = seq_start_dev; p.h0 = h0_dev; p.dh_last = dh_last_dev; p.dh0 = dh0_dev;
    p.pairs = (float2 *)workspace_dev;
    p.tokens = tokens; p.channels = channels; p.n_seq = n_seq;
    p.blocks = scan_blocks(tokens); p.groups = (channels + kCh - 1) / kCh;
    hipStream_t s = entry_stream(stream);
    return dtype == ZIPML_F32 ? launch_backward<float>(s, p) : launch_backward<__bf16>(s, p);
}

template <typename T>
static int launch_step(hipStream_t s, const void *x, int64_t ldx, const void *z, int64_t ldz, int64_t rows, int64_t channels,
                       float *h, int64_t n_slots, const int32_t *slots, void *y, int64_t ldy)
{
    const int64_t blocks = (rows * ((channels + 7) / 8) + 255) / 256;
    hipLaunchKernelGGL(k_scan_step<T>, dim3((uint32_t)blocks), dim3(256), 0, s, (const T *)x, ldx, (const T *)z, ldz, rows, channels, h,
                       n_slots, slots, (T *)y, ldy);
    return hip_check(hipGetLastError());
}

extern "C" int zipml_scan_step(void *stream, const void *x_dev, int64_t ldx, const void *z_dev, int64_t ldz, int dtype,
                               int64_t rows, int64_t channels, float *h_dev, int64_t n_slots, const int32_t *slots_dev,
                               void *y_dev, int64_t ldy)
{
    if (!x_dev || !z_dev || !h_dev || !y_dev || !valid_dtype(dtype) || !act_sizes_ok(rows, channels)) return ZIPML_EINVAL;
    if (rows > (1ll << 38) / channels) return ZIPML_EINVAL;
    if (!stride_ok(ldx, rows, channels) || !stride_ok(ldz, rows, channels) || !stride_ok(ldy, rows, channels))
        return ZIPML_EINVAL;
    if (n_slots < 1 || n_slots > (1ll << 60) / channels || (!slots_dev && n_slots < rows)) return ZIPML_EINVAL;
    if (!aligned16(x_dev) || !aligned16(z_dev) || !aligned16(h_dev) || !aligned16(slots_dev) || !aligned16(y_dev))
        return ZIPML_EALIGN;
    hipStream_t s = entry_stream(stream);
    if (dtype == ZIPML_F32)
        return launch_step<float>(s, x_dev, ldx, z_dev, ldz, rows, channels, h_dev, n_slots, slots_dev, y_dev, ldy);
    return launch_step<__bf16>(s, x_dev, ldx, z_dev, ldz, rows, channels, h_dev, n_slots, slots_dev, y_dev, ldy);
}
