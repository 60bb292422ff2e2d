// Gated linear recurrence  h_t = f_t h_{t-1} + (1 - f_t) x_t,  f = sigmoid(z): packed sequences, forward and backward.
//
// Both directions are scans of pairs: a run of tokens takes a state h to A h + B, and two runs one after the other
// to (A2 A1) h + (A2 B1 + B2).  A workgroup owns 64 channels and a block of 256 tokens: sixteen lanes side by side take four
// channels each (128 bytes of a bf16 row), 32 such rows of lanes eight tokens each, which a thread walks through in
// registers.  Everything is read and written once: the rows of lanes are joined by shuffles and LDS, the blocks by a chain in
// global memory while their tokens stay in registers.
//
// The chain.  A block publishes its pair, takes the pairs of the blocks before it up to the last multiple of kSuper and the
// state there, which the block before that multiple has published, and so has the state that enters it.  What is
// joined in which order depends on the block's number alone, so the results do not depend on timing.  A word is a pair of
// floats stored and polled as 64 bits, all ones before it is there (A is never a NaN).  Blocks are handed out by a
// counter for each 64 channels, in the chain's order: a block waits only for blocks that were handed out before it, to
// workgroups that run, and those wait for nothing that is behind them, so every wait ends.
//
// A = 0 marks a run that contains the start of a sequence (or lies outside all): what is before it does not matter, and
// is not multiplied, so that a NaN or an infinity of one sequence never reaches the next.  Every other A that leaves a
// thread's block is kept at 2^-126 or more, so that within a sequence they do pass on; what that adds to a state is below
// 2^-126 of it.
#include "zipml_act.h"

namespace zipml {

constexpr int kBlock = ZIPML_SCAN_BLOCK;   // tokens of a workgroup
constexpr int kCh = 64;                    // channels of a workgroup
constexpr int kRun = 8;                    // tokens of a thread
constexpr int kOwn = 4;                    // channels of a thread
constexpr int kLanes = kCh / kOwn;         // lanes side by side
constexpr int kRows = kWave / kLanes;      // runs of a wave
constexpr int kSuper = 32;                 // blocks between two published states
// A workgroup of W waves takes a block of W * kRows * kRun tokens.
constexpr int kForwardWaves = 8, kBackwardWaves = 8;
constexpr int kWaveTokens = kRows * kRun;
constexpr float kTiny = 1.17549435e-38f;
constexpr float kZMax = 16.0f;             // gates are stored clamped to +-kZMax: sigmoid(16) is 1 - 2^-23.1
static_assert(kSuper % kBackwardWaves == 0 && kSuper % kForwardWaves == 0, "the waves share the pairs of kSuper blocks");
static_assert(kBackwardWaves * kWaveTokens == kBlock && kBlock % (kForwardWaves * kWaveTokens) == 0, "states by the block");

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
    uint64_t *pairs;                       // [blocks][channels], then
    uint64_t *supers;                      // [blocks / kSuper][channels], then
    uint32_t *counters;                    // [groups]
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

// Joins of runs.  SOME = false: no sequence starts or ends within, plain arithmetic.
template <bool SOME>
__device__ __forceinline__ float join(float a, float prev, float b)
{
    return SOME && a == 0.0f ? b : __builtin_fmaf(a, prev, b);
}
template <bool SOME>
__device__ __forceinline__ float times(float a, float b)
{
    return !SOME ? a * b : a == 0.0f || b == 0.0f ? 0.0f : __builtin_fmaxf(a * b, kTiny);
}

// ---- four neighbouring values of a row, as fp32 -----------------------------------------------
typedef u32x2 u32x2_any __attribute__((aligned(2)));

// The loads of a block are all issued before the first is used, so none of them stands in a branch: a thread whose columns or
// rows are not all there reads the last ones that are, and `settle` moves columns to their places.
struct Columns {
    int64_t c, at;     // the thread's first column, and where it reads
    bool few;          // fewer than four columns in all: read one by one
    bool tail;         // (for the workgroup) columns beyond the last
    __device__ __forceinline__ Columns(int64_t c0, int64_t c_, int64_t channels)
    {
        c = c_;
        few = channels < kOwn;
        tail = c0 + kCh > channels;
        at = c <= channels - kOwn ? c : channels - kOwn;
    }
};
template <typename T>
__device__ __forceinline__ void load_few(const T *row, const Columns &q, int64_t channels, float (&v)[kOwn])
{
#pragma unroll
    for (int k = 0; k < kOwn; ++k) v[k] = q.c + k < channels ? (float)row[q.c + k] : 0.0f;
}
template <typename T>
__device__ __forceinline__ void load4(const T *row, const Columns &q, float (&v)[kOwn])
{
    if constexpr (sizeof(T) == 2) {
        const u32x2 w = *reinterpret_cast<const u32x2_any *>(row + q.at);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            v[2 * k] = as_f32(w[k] << 16);
            v[2 * k + 1] = as_f32(w[k] & 0xFFFF0000u);
        }
    } else {
        const f32x4 w = *reinterpret_cast<const f32x4_any *>(row + q.at);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = w[k];
    }
}
__device__ __forceinline__ void settle(const Columns &q, float (&v)[kOwn])
{
    if (!q.tail || q.few) return;
    const int64_t s = q.c - q.at;
    if (s & 1) { v[0] = v[1]; v[1] = v[2]; v[2] = v[3]; v[3] = 0.0f; }
    if (s & 2) { v[0] = v[2]; v[1] = v[3]; v[2] = v[3] = 0.0f; }
    if (s >= kOwn) v[0] = v[1] = v[2] = v[3] = 0.0f;
}
template <typename T>
__device__ __forceinline__ void store4(T *p, int64_t left, const float (&v)[kOwn])
{
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    typedef bf16x4 bf16x4_any __attribute__((aligned(2)));
    if (left >= kOwn) {
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<bf16x4_any *>(p) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        else
            *reinterpret_cast<f32x4_any *>(p) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int k = 0; k < kOwn; ++k)
            if (k < left) p[k] = (T)v[k];
    }
}
// Row s of an [n_seq][channels] array that may be missing (zeros then).
__device__ __forceinline__ void load_state(const float *a, int64_t s, int64_t channels, int64_t c, float (&v)[kOwn])
{
#pragma unroll
    for (int k = 0; k < kOwn; ++k) v[k] = a && c + k < channels ? a[s * channels + c + k] : 0.0f;
}

// ---- sequences ---------------------------------------------------------------------------------
template <int W>
struct BlockMap {
    int first[W * kWaveTokens], last[W * kWaveTokens];   // the sequence of which a token is the first or last, or -1
    int some;                              // some token is either, or outside
};
struct Range { int64_t begin, end; };      // tokens inside sequences

template <int W>
__device__ __forceinline__ Range block_map(const ScanArgs &a, int64_t t0, BlockMap<W> &m)
{
    constexpr int kBlock = W * kWaveTokens, kThreads = W * kWave;
    for (int i = threadIdx.x; i < kBlock; i += kThreads) m.first[i] = m.last[i] = -1;
    if (threadIdx.x == 0) m.some = 0;
    __syncthreads();
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

// Empty sequences hand on what they are given.
template <int W>
__device__ __forceinline__ void pass_on(const ScanArgs &p, int64_t blk, int64_t c0, const float *from, float *to)
{
    if (!to || !p.seq_start) return;
    const int64_t c = c0 + (threadIdx.x & 63);
    for (int64_t s = blk * W + (threadIdx.x >> 6); s < p.n_seq; s += p.blocks * W)
        if (p.seq_start[s] >= p.seq_start[s + 1] && c < p.channels)
            to[s * p.channels + c] = from ? from[s * p.channels + c] : 0.0f;
}

// ---- joining runs ------------------------------------------------------------------------------
template <int W>
struct ScanShared {
    BlockMap<W> map;
    float2 waves[W][kCh];             // pairs of the waves, later of the blocks before
    float2 total[kCh];
    float carry[kCh];
    uint32_t ticket;
};

// A, B: in, the pair of each thread's run; out, that of all runs before it in the block (REVERSE: behind it).  sh.total gets
// the whole block's.
template <bool REVERSE, bool SOME, int W>
__device__ __forceinline__ void block_scan(float (&A)[kOwn], float (&B)[kOwn], ScanShared<W> &sh)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cl = lane & (kLanes - 1);
    const int pos = REVERSE ? kRows - 1 - lane / kLanes : lane / kLanes;
    auto before = [&](float v, int s) { return __shfl(v, (REVERSE ? lane + kLanes * s : lane - kLanes * s) & 63, 64); };
#pragma unroll
    for (int s = 1; s < kRows; s <<= 1)
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const float pa = before(A[k], s), pb = before(B[k], s);
            B[k] = pos >= s ? join<SOME>(A[k], pb, B[k]) : B[k];
            A[k] = pos >= s ? times<SOME>(A[k], pa) : A[k];
        }
    __syncthreads();                       // (whatever was read from sh before)
    if (pos == kRows - 1)
#pragma unroll
        for (int k = 0; k < kOwn; ++k) sh.waves[wave][cl * kOwn + k] = float2{A[k], B[k]};
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {       // of the runs before this one
        const float pa = before(A[k], 1), pb = before(B[k], 1);
        A[k] = pos == 0 ? 1.0f : pa;
        B[k] = pos == 0 ? 0.0f : pb;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        float wa = 1.0f, wb = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int w = REVERSE ? W - 1 - i : i;
            const float2 p = sh.waves[w][cl * kOwn + k];
            if (w == wave) {               // (uniform over a wave)
                B[k] = join<SOME>(A[k], wb, B[k]);
                A[k] = times<SOME>(A[k], wa);
            }
            wb = join<SOME>(p.x, wb, p.y);
            wa = times<SOME>(p.x, wa);
        }
        if (threadIdx.x < kLanes) sh.total[cl * kOwn + k] = float2{SOME ? wa : __builtin_fmaxf(wa, kTiny), wb};
    }
}

constexpr uint64_t kAbsent = ~0ull;
__device__ __forceinline__ uint64_t word(float a, float b) { return (uint64_t)as_u32(a) << 32 | as_u32(b); }
// The word once it is there.  (The limit is never reached; a NaN would tell.)
__device__ __forceinline__ uint64_t await(const uint64_t *p)
{
    uint64_t w = load_dev(p);
    for (int n = 0; w == kAbsent && n < (1 << 22); ++n) {
        __builtin_amdgcn_s_sleep(1);
        w = load_dev(p);
    }
    return w == kAbsent ? word(0.0f, __builtin_nanf("")) : w;
}

// The state that enters block `k` of the chain (k counts in the direction of the scan; at(k) is the block), in sh.carry, from
// sh.total; the block's own pair, and the state behind it where one is due, are published.
template <bool REVERSE, int W>
__device__ __forceinline__ void chain(const ScanArgs &p, int64_t k, int64_t c0, ScanShared<W> &sh)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = c0 + lane;
    const bool live = c < p.channels;
    __syncthreads();                       // sh.total is there, sh.waves free
    auto at = [&](int64_t i) { return (REVERSE ? p.blocks - 1 - i : i) * p.channels + c; };
    const float2 own = sh.total[lane];
    if (wave == 0 && live && p.blocks > 1) store_dev(p.pairs + at(k), word(own.x, own.y));

    // the pairs from the last multiple of kSuper on, a few of them to each wave
    constexpr int kEach = kSuper / W;
    const int64_t base = k - k % kSuper, from = base + wave * kEach;
    uint64_t w[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) w[i] = from + i < k && live ? load_dev(p.pairs + at(from + i)) : word(1.0f, 0.0f);
    float a = 1.0f, b = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (w[i] == kAbsent) w[i] = await(p.pairs + at(from + i));
        const float wa = as_f32((uint32_t)(w[i] >> 32)), wb = as_f32((uint32_t)w[i]);
        b = join<true>(wa, b, wb);
        a = times<true>(wa, a);
    }
    sh.waves[wave][lane] = float2{a, b};
    __syncthreads();
    if (wave == 0) {
        float h = base > 0 && live ? as_f32((uint32_t)await(p.supers + (base / kSuper - 1) * p.channels + c)) : 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) h = join<true>(sh.waves[i][lane].x, h, sh.waves[i][lane].y);
        sh.carry[lane] = h;
        if (live && k % kSuper == kSuper - 1)
            store_dev(p.supers + k / kSuper * p.channels + c, word(0.0f, join<true>(own.x, h, own.y)));
    }
    __syncthreads();
}

// Which channels and which block a workgroup takes.  Workgroups go to the eight XCDs in turn; where there are enough channels,
// two neighbouring groups of 64 stay on one XCD, since each writes half of a cache line of codes.
struct Place { int64_t k, c0; };
template <int W>
__device__ __forceinline__ Place take(const ScanArgs &p, ScanShared<W> &sh)
{
    const uint32_t n = (uint32_t)p.groups, b = blockIdx.x;
    uint32_t g = b % n;
    if (n % 16 == 0) g = (g & ~15u) | (g & 7) << 1 | (g >> 3 & 1);
    if (p.blocks == 1) return Place{0, g * (int64_t)kCh};
    if (threadIdx.x == 0) sh.ticket = __hip_atomic_fetch_add(p.counters + g, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    return Place{sh.ticket, g * (int64_t)kCh};
}

// The words and counters of a chain before it starts.
__global__ __launch_bounds__(256) void k_scan_clear(uint64_t *words, int64_t n, uint32_t *counters, int64_t groups)
{
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += step) words[i] = kAbsent;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < groups; i += step) counters[i] = 0;
}

// ---- storing and reading the inputs ---------------------------------------------------------------
// Two tokens (rows row, row + 1) of four columns; eight lanes hold a group's 32 columns.  A Philox block serves eight columns:
// the two lanes that share them make that of one token each and exchange halves.
__device__ __forceinline__ void encode_two(const float (&v)[2][kOwn], uint64_t seed, uint32_t epoch, int64_t row, uint32_t col8,
                                           uint32_t stream, uint32_t (&codes)[2], uint32_t (&byte)[2])
{
    const bool odd = threadIdx.x & 1;
    const Philox4 r = philox_block(seed, epoch, (uint64_t)(row + (odd ? 1 : 0)), col8, stream);
    const uint32_t x0 = dpp_move<0xB1>(odd ? r.w[0] : r.w[2]), x1 = dpp_move<0xB1>(odd ? r.w[1] : r.w[3]);
    const uint32_t w[2][2] = {{odd ? x0 : r.w[0], odd ? x1 : r.w[1]}, {odd ? r.w[2] : x0, odd ? r.w[3] : x1}};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const uint32_t m = as_u32(v[t][k]) & 0x7FFFFFFFu;
            top = top > m ? top : m;
        }
        uint32_t o = dpp_move<0xB1>(top);
        top = top > o ? top : o;
        o = dpp_move<0x4E>(top);
        top = top > o ? top : o;
        o = dpp_move<0x141>(top);
        top = top > o ? top : o;
        const ActStep s = act_step_of(top);
        uint32_t c[kOwn];
#pragma unroll
        for (int k = 0; k < kOwn; ++k) c[k] = act_code(v[t][k], s.inverse, k & 1 ? w[t][k >> 1] >> 16 : w[t][k >> 1] & 0xFFFFu);
        codes[t] = s.finite ? act_pack4(c) : 0u;
        byte[t] = s.byte;
    }
}
__device__ __forceinline__ void decode4(uint32_t codes, float step, float (&v)[kOwn])
{
#pragma unroll
    for (int k = 0; k < kOwn; ++k) v[k] = (float)(int8_t)(codes >> (8 * k)) * step;
}

// ---- forward -----------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kForwardWaves * kWave, 4) void k_scan_forward(ScanArgs p)
{
    constexpr int W = kForwardWaves;
    __shared__ ScanShared<W> sh;
    const Place at = take(p, sh);
    const int64_t blk = at.k, t0 = blk * (W * kWaveTokens);
    const int run = threadIdx.x / kLanes * kRun;                    // the first token of the thread's run, in the block
    const int64_t c = at.c0 + (threadIdx.x & (kLanes - 1)) * kOwn, left = p.channels - c;
    const Columns cols(at.c0, c, p.channels);

    float a[kRun][kOwn], b[kRun][kOwn];                             // z and x, later f and (1 - f) x
    auto row = [&](int j) { return t0 + run + j < p.tokens ? t0 + run + j : p.tokens - 1; };
    if (!cols.few) {
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            load4((const T *)p.x + row(j) * p.ldx, cols, b[j]);
            load4((const T *)p.z + row(j) * p.ldz, cols, a[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            load_few((const T *)p.x + row(j) * p.ldx, cols, p.channels, b[j]);
            load_few((const T *)p.z + row(j) * p.ldz, cols, p.channels, a[j]);
        }
    }
    const Range r = block_map(p, t0, sh.map);

#pragma unroll
    for (int j = 0; j < kRun; ++j) {
        settle(cols, b[j]);
        settle(cols, a[j]);
    }
    if (p.wx) {
#pragma unroll
        for (int j = 0; j < kRun; j += 2) {
            float v[2][kOwn], z[2][kOwn];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int k = 0; k < kOwn; ++k) {
                    const float q = a[j + i][k];
                    v[i][k] = b[j + i][k];
                    z[i][k] = q > kZMax ? kZMax : q < -kZMax ? -kZMax : q;
                }
            const int64_t t = t0 + run + j;
            uint32_t cx[2], cz[2], ex[2], ez[2];
            encode_two(v, p.seed, p.epoch, t, (uint32_t)(c >> 3), p.stream, cx, ex);
            encode_two(z, p.seed, p.epoch, t, (uint32_t)(c >> 3), p.stream + 1, cz, ez);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (t + i < p.tokens && c < p.lay.pitch) {
                    const int64_t o = (t + i) * p.lay.pitch + c;
                    *reinterpret_cast<uint32_t *>(p.wx + o) = cx[i];
                    *reinterpret_cast<uint32_t *>(p.wz + o) = cz[i];
                    if ((threadIdx.x & 7) == 0) {
                        const int64_t e = p.lay.steps + (t + i) * p.lay.groups + (c >> 5);
                        p.wx[e] = (uint8_t)ex[i];
                        p.wz[e] = (uint8_t)ez[i];
                    }
                }
        }
    }
#pragma unroll
    for (int j = 0; j < kRun; ++j)
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            float f, g;
            gates(a[j][k], f, g);
            a[j][k] = f;
            b[j][k] *= g;
        }

    float A[kOwn], B[kOwn];
    uint32_t reset = 0;                                             // tokens that do not look back
    if (!sh.map.some) {
#pragma unroll
        for (int k = 0; k < kOwn; ++k) { A[k] = a[0][k]; B[k] = b[0][k]; }
#pragma unroll
        for (int j = 1; j < kRun; ++j)
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                B[k] = __builtin_fmaf(a[j][k], B[k], b[j][k]);
                A[k] *= a[j][k];
            }
        block_scan<false, false>(A, B, sh);
    } else {
#pragma unroll
        for (int k = 0; k < kOwn; ++k) { A[k] = 1.0f; B[k] = 0.0f; }
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int64_t t = t0 + run + j;
            const int s = sh.map.first[run + j];
            if (t < r.begin || t >= r.end) {
#pragma unroll
                for (int k = 0; k < kOwn; ++k) b[j][k] = 0.0f;
                reset |= 1u << j;
            } else if (s >= 0) {
                if (p.h0) {
                    float h[kOwn];
                    load_state(p.h0, s, p.channels, c, h);
#pragma unroll
                    for (int k = 0; k < kOwn; ++k) b[j][k] = __builtin_fmaf(a[j][k], h[k], b[j][k]);
                }
                reset |= 1u << j;
            }
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                B[k] = reset >> j & 1 ? b[j][k] : __builtin_fmaf(a[j][k], B[k], b[j][k]);
                A[k] *= a[j][k];
            }
        }
#pragma unroll
        for (int k = 0; k < kOwn; ++k) A[k] = reset ? 0.0f : __builtin_fmaxf(A[k], kTiny);
        block_scan<false, true>(A, B, sh);
    }
    chain<false>(p, at.k, at.c0, sh);

    float h[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        const float in = sh.carry[c - at.c0 + k];
        h[k] = sh.map.some ? join<true>(A[k], in, B[k]) : join<false>(A[k], in, B[k]);
    }
    if (p.states && t0 % kBlock == 0 && threadIdx.x < kCh && at.c0 + threadIdx.x < p.channels)
        p.states[t0 / kBlock * p.channels + at.c0 + threadIdx.x] = sh.carry[threadIdx.x];
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
        const int64_t t = t0 + run + j;
#pragma unroll
        for (int k = 0; k < kOwn; ++k) h[k] = reset >> j & 1 ? b[j][k] : __builtin_fmaf(a[j][k], h[k], b[j][k]);
        if (t < p.tokens) store4<T>((T *)p.y + t * p.ldy + c, left, h);
        if (p.h_last && sh.map.some && sh.map.last[run + j] >= 0)
            store4<float>(p.h_last + (int64_t)sh.map.last[run + j] * p.channels + c, left, h);
    }
    pass_on<W>(p, blk, at.c0, p.h0, p.h_last);
}

// ---- backward ----------------------------------------------------------------------------------
// p_t = f_t d_t, d_t = dy_t + p_{t+1}, is a scan from right to left with the same factors as that of the states from left to
// right; a run's pairs of both come from one walk: B of the right-to-left one is the sum of d_t times the product of the f
// up to t.
template <typename T>
__global__ __launch_bounds__(kBackwardWaves * kWave, 2) void k_scan_backward(ScanArgs p)
{
    constexpr int W = kBackwardWaves;
    __shared__ ScanShared<W> sh;
    const Place at = take(p, sh);
    const int64_t blk = p.blocks - 1 - at.k, t0 = blk * kBlock;
    const int run = threadIdx.x / kLanes * kRun;
    const int64_t c = at.c0 + (threadIdx.x & (kLanes - 1)) * kOwn, left = p.channels - c;
    const Columns cols(at.c0, c, p.channels);

    uint32_t qx[kRun], ex[kRun];
    float d[kRun][kOwn], f[kRun][kOwn], g[kRun][kOwn];
    {
        uint32_t qz[kRun], ez[kRun];
        auto row = [&](int j) { return t0 + run + j < p.tokens ? t0 + run + j : p.tokens - 1; };
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int64_t t = row(j), cc = c < p.lay.pitch ? c : p.lay.pitch - kOwn;
            const int64_t o = t * p.lay.pitch + cc, e = p.lay.steps + t * p.lay.groups + (cc >> 5);
            qz[j] = *reinterpret_cast<const uint32_t *>(p.rz + o);
            ez[j] = p.rz[e];
            qx[j] = *reinterpret_cast<const uint32_t *>(p.rx + o);
            ex[j] = p.rx[e];
        }
        if (!cols.few) {
#pragma unroll
            for (int j = 0; j < kRun; ++j) load4((const T *)p.dy + row(j) * p.lddy, cols, d[j]);
        } else {
#pragma unroll
            for (int j = 0; j < kRun; ++j) load_few((const T *)p.dy + row(j) * p.lddy, cols, p.channels, d[j]);
        }
#pragma unroll
        for (int j = 0; j < kRun; ++j) settle(cols, d[j]);
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            float z[kOwn];
            decode4(qz[j], act_step(ez[j]), z);
#pragma unroll
            for (int k = 0; k < kOwn; ++k) gates(z[k], f[j][k], g[j][k]);
        }
    }
    const Range r = block_map(p, t0, sh.map);
    const bool some = sh.map.some;

    float A[kOwn], H[kOwn], AR[kOwn], P[kOwn];                      // pairs (A, H) from the left, (AR, P) from the right
    uint32_t outside = 0, first = 0, last = 0;                      // tokens, by bit
#pragma unroll
    for (int k = 0; k < kOwn; ++k) { A[k] = 1.0f; H[k] = P[k] = 0.0f; }
    if (!some) {
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            float x[kOwn];
            decode4(qx[j], act_step(ex[j]), x);
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                A[k] *= f[j][k];
                H[k] = __builtin_fmaf(f[j][k], H[k], g[j][k] * x[k]);
                P[k] = __builtin_fmaf(A[k], d[j][k], P[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kOwn; ++k) AR[k] = A[k];
        block_scan<true, false>(AR, P, sh);
    } else {
        bool cut = false;                                           // a sequence has ended in this run
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int64_t t = t0 + run + j;
            float x[kOwn];
            decode4(qx[j], act_step(ex[j]), x);
            if (t < r.begin || t >= r.end) {
                outside |= 1u << j;
                cut = true;
#pragma unroll
                for (int k = 0; k < kOwn; ++k) H[k] = 0.0f;
                continue;
            }
            if (sh.map.last[run + j] >= 0) {
                last |= 1u << j;
                float h[kOwn];
                load_state(p.dh_last, sh.map.last[run + j], p.channels, c, h);
#pragma unroll
                for (int k = 0; k < kOwn; ++k) d[j][k] += h[k];
            }
            if (sh.map.first[run + j] >= 0) {
                first |= 1u << j;
                load_state(p.h0, sh.map.first[run + j], p.channels, c, H);
            }
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                A[k] *= f[j][k];
                H[k] = __builtin_fmaf(f[j][k], H[k], g[j][k] * x[k]);
                P[k] = cut ? P[k] : __builtin_fmaf(A[k], d[j][k], P[k]);
            }
            cut |= last >> j & 1;
        }
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const float m = __builtin_fmaxf(A[k], kTiny);
            A[k] = first | outside ? 0.0f : m;
            AR[k] = cut ? 0.0f : m;
        }
        block_scan<true, true>(AR, P, sh);
    }
    chain<true>(p, at.k, at.c0, sh);
    float q[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        const float in = sh.carry[c - at.c0 + k];
        q[k] = some ? join<true>(AR[k], in, P[k]) : join<false>(AR[k], in, P[k]);
    }

    // d becomes the gradient of each state
#pragma unroll
    for (int j = kRun - 1; j >= 0; --j) {
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            d[j][k] = outside >> j & 1 ? 0.0f : last >> j & 1 ? d[j][k] : d[j][k] + q[k];
            q[k] = outside >> j & 1 ? 0.0f : f[j][k] * d[j][k];
        }
        if (p.dh0 && first >> j & 1) store4<float>(p.dh0 + (int64_t)sh.map.first[run + j] * p.channels + c, left, q);
    }

    // the states again, from the one that the forward pass kept
    if (!some) block_scan<false, false>(A, H, sh);
    else block_scan<false, true>(A, H, sh);
    float h[kOwn];
    load_state(p.states, blk, p.channels, c, h);
#pragma unroll
    for (int k = 0; k < kOwn; ++k) h[k] = some ? join<true>(A[k], h[k], H[k]) : join<false>(A[k], h[k], H[k]);
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
        const int64_t t = t0 + run + j;
        float x[kOwn], dx[kOwn], dz[kOwn];
        decode4(qx[j], act_step(ex[j]), x);
        if (first >> j & 1) load_state(p.h0, sh.map.first[run + j], p.channels, c, h);
        const bool out = outside >> j & 1;
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            dx[k] = out ? 0.0f : g[j][k] * d[j][k];
            dz[k] = out ? 0.0f : f[j][k] * dx[k] * (h[k] - x[k]);
            h[k] = out ? 0.0f : __builtin_fmaf(f[j][k], h[k], g[j][k] * x[k]);
        }
        if (t < p.tokens) {
            store4<T>((T *)p.dx + t * p.lddx + c, left, dx);
            store4<T>((T *)p.dz + t * p.lddz + c, left, dz);
        }
    }
    pass_on<W>(p, blk, at.c0, p.dh_last, p.dh0);
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
        load8<float>(s, left, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float f, g;
            gates(zv[k], f, g);
            v[k] = __builtin_fmaf(f, v[k], g * xv[k]);
        }
        store8<float>(s, left, v);
    }
    store8(y + row * ldy + c, left, v);
}

static int64_t scan_blocks(int64_t tokens, int waves) { return (tokens + waves * kWaveTokens - 1) / (waves * kWaveTokens); }
static bool scan_sizes_ok(int64_t tokens, int64_t channels)
{
    return act_sizes_ok(tokens, channels) && scan_blocks(tokens, kForwardWaves) * ((channels + kCh - 1) / kCh) <= (1ll << 31) - 1;
}
static bool stride_ok(int64_t ld, int64_t rows, int64_t cols) { return ld >= cols && ld <= (1ll << 60) / rows; }

// The chain's words behind one another in the workspace.
struct ScanSpace { int64_t pairs, supers, groups; size_t bytes() const { return (size_t)(pairs + supers) * 8 + (size_t)groups * 4; } };
static ScanSpace scan_space(int64_t tokens, int64_t channels, int waves)
{
    const int64_t blocks = scan_blocks(tokens, waves);
    if (blocks == 1) return ScanSpace{0, 0, 0};
    return ScanSpace{blocks * channels, blocks / kSuper * channels, (channels + kCh - 1) / kCh};
}
static int scan_launch(hipStream_t s, ScanArgs &p, void *workspace, int waves, void (*kernel)(ScanArgs))
{
    const ScanSpace w = scan_space(p.tokens, p.channels, waves);
    p.blocks = scan_blocks(p.tokens, waves);
    p.pairs = (uint64_t *)workspace;
    p.supers = p.pairs + w.pairs;
    p.counters = (uint32_t *)(p.supers + w.supers);
    if (p.blocks > 1) {
        const int64_t n = w.pairs + w.supers, blocks = (n + 1023) / 1024;
        hipLaunchKernelGGL(k_scan_clear, dim3((uint32_t)(blocks < 1024 ? blocks : 1024)), dim3(256), 0, s, p.pairs, n, p.counters,
                           w.groups);
    }
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(p.blocks * p.groups)), dim3(waves * kWave), 0, s, p);
    return hip_check(hipGetLastError());
}

}  // namespace zipml

using namespace zipml;

extern "C" size_t zipml_scan_workspace_bytes(int64_t tokens, int64_t channels)
{
    if (!scan_sizes_ok(tokens, channels)) return 0;
    // (the forward pass has the more blocks)
    const size_t b = scan_space(tokens, channels, kForwardWaves).bytes();
    return b < 256 ? 256 : b;
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
    p.seed = seed; p.epoch = epoch; p.stream = kActStream + tag;
    p.tokens = tokens; p.channels = channels; p.n_seq = n_seq;
    p.groups = (channels + kCh - 1) / kCh;
    hipStream_t s = entry_stream(stream);
    return scan_launch(s, p, workspace_dev, kForwardWaves, dtype == ZIPML_F32 ? k_scan_forward<float> : k_scan_forward<__bf16>);
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
    p.tokens = tokens; p.channels = channels; p.n_seq = n_seq;
    p.groups = (channels + kCh - 1) / kCh;
    hipStream_t s = entry_stream(stream);
    return scan_launch(s, p, workspace_dev, kBackwardWaves, dtype == ZIPML_F32 ? k_scan_backward<float> : k_scan_backward<__bf16>);
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
