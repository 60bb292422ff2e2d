// Gated linear recurrence  h_t = f_t h_{t-1} + (1 - f_t) x_t,  f = sigmoid(z): packed sequences, forward and backward.
//
// Both directions are scans of pairs: a run of tokens takes a state h to A h + B, and two runs one after the other
// to (A2 A1) h + (A2 B1 + B2).  A workgroup owns 64 channels and a block of 256 tokens: sixteen lanes side by side take four
// channels each (128 bytes of a bf16 row), 32 such rows of lanes eight tokens each, which a thread walks through in
// registers (with few blocks 32 channels: eight lanes side by side, four tokens each).  Everything is read and written once,
// but for dy in the backward pass: the rows of lanes are joined by shuffles and LDS, the blocks by a chain in global memory
// while their tokens stay in registers.
//
// The chain.  A block publishes its pair, takes the pairs of the blocks before it up to the last multiple of kSuper and the
// state there, which the block before that multiple has published, and so has the state that enters it.  What is
// joined in which order depends on the block's number alone, so the results do not depend on timing.  A word is a pair of
// floats stored and polled as 64 bits, all ones before it is there (A is never a NaN).  Blocks are handed out by a
// counter for each group of channels, in the chain's order: a block waits only for blocks that were handed out before it, to
// workgroups that run, and those wait for nothing that is behind them, so every wait ends.
//
// A = 0 marks a run that contains the start of a sequence (or lies outside all): what is before it does not matter, and
// is not multiplied, so that a NaN or an infinity of one sequence never reaches the next.  Every other A that leaves a
// thread's block is kept at 2^-126 or more, so that within a sequence they do pass on; what that adds to a state is below
// 2^-126 of it.
//
// Open gates.  f is near 1 then and fp32 holds 1 - f to 2^-25 at best, with the same error at every token: with f multiplied up a
// state at z = 12 is off by 0.3 to 0.6 % after 100,000 tokens, and at z = 17 nothing is ever forgotten.  So what a run forgets,
// D = 1 - A, is summed beside A, each token's 1 - f times the A before it, from the tokens up to the block: all terms are positive, so D
// keeps its relative accuracy, and A = 1 - D is rounded once where D is the smaller one.  A state is then off by 2^-25 of itself a
// block, as from its own rounding.  This costs 0 to 6 % (131,072 x 256 forward 60 us against 57.6, 32,768 x 2,048 forward and
// backward bf16 316 against 309, fp32 419 either way).
#include "zipml_act.h"

namespace zipml {

constexpr int kBlock = ZIPML_SCAN_BLOCK;   // tokens of a workgroup
constexpr int kOwn = 4;                    // channels of a thread
constexpr int kSuper = 32;                 // blocks between two published states
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kMostCh = 64;
constexpr float kTiny = 1.17549435e-38f;
constexpr float kZMax = 16.0f;             // gates are stored clamped to +-kZMax: sigmoid(16) is 1 - 2^-23.1 (a group with one there has step 1/4)
static_assert(kSuper % kWaves == 0, "the waves share the pairs of kSuper blocks");
static_assert(kThreads == 2 * kBlock, "a thread for each token of x and z");

// How a block is cut up: channels of a workgroup and tokens of a thread.
template <int CH, int RUN> struct Cut {
    static constexpr int kCh = CH, kRun = RUN;
    static constexpr bool kThrough = CH == 64;     // results do not stay in the L2
    static constexpr int kLanes = kCh / kOwn;      // lanes side by side
    static constexpr int kRows = kWave / kLanes;   // runs of a wave
    static_assert(kWaves * kRows * kRun == kBlock && kRun % 4 == 0 && kCh % kActGroup == 0 && kCh <= kMostCh, "whole blocks");
    static __device__ __forceinline__ int lane() { return threadIdx.x & (kLanes - 1); }
    static __device__ __forceinline__ int run() { return threadIdx.x / kLanes * kRun; }   // the thread's first token, in the block
};
typedef Cut<64, 8> Wide;
typedef Cut<32, 4> Narrow;

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
    int *status;                           // ZIPML_OK, or ZIPML_ETIMEOUT where a wait gave up
    uint32_t spin_limit;                   // polls before one does
    uint64_t *pairs;                       // [blocks][channels], then
    uint64_t *supers;                      // [blocks / kSuper][channels], then
    uint32_t *counters;                    // [groups], `apart` words apart
    uint32_t apart;
    uint64_t seed;
    uint32_t epoch, stream;
    int64_t tokens, channels, n_seq, blocks, groups;
};

// A and D = 1 - A of a run in one number, the smaller one: -D where D is below 1/2 (by its sign; -0 for none), else A.
__device__ __forceinline__ float packed(float a, float d) { return d < 0.5f ? -d : a; }
__device__ __forceinline__ float kept_of(float m) { return as_u32(m) >> 31 ? 1.0f + m : m; }
__device__ __forceinline__ float forgotten_of(float m) { return as_u32(m) >> 31 ? -m : 1.0f - m; }

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

// ---- four neighbouring values of a row -----------------------------------------------------------
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef u32x4 u32x4_four __attribute__((aligned(4)));

// As they lie in memory; of() is value k in fp32.
template <typename T> struct Raw4;
template <> struct Raw4<__bf16> {
    u32x2 w;
    __device__ __forceinline__ float of(int k) const { return as_f32(k & 1 ? w[k >> 1] & 0xFFFF0000u : w[k >> 1] << 16); }
    __device__ __forceinline__ void load(const __bf16 *p) { w = *reinterpret_cast<const u32x2_any *>(p); }
    __device__ __forceinline__ void move(int s)            // value k becomes value k + s
    {
        const uint64_t v = s >= kOwn ? 0 : __builtin_bit_cast(uint64_t, w) >> (16 * (s & 3));
        w = __builtin_bit_cast(u32x2, v);
    }
};
template <> struct Raw4<float> {
    u32x4 w;
    __device__ __forceinline__ float of(int k) const { return as_f32(w[k]); }
    __device__ __forceinline__ void load(const float *p) { w = *reinterpret_cast<const u32x4_four *>(p); }
    __device__ __forceinline__ void move(int s)
    {
        if (s & 1) w = u32x4{w[1], w[2], w[3], 0u};
        if (s & 2) w = u32x4{w[2], w[3], 0u, 0u};
        if (s >= kOwn) w = u32x4{0u, 0u, 0u, 0u};
    }
};

// A thread's part of a block's rows.  The loads of a block are all issued before the first is used, so none of them stands in a
// branch of its own: a thread whose rows or columns are not all there reads the last ones that are, and `settle` moves columns
// to their places.  Fewer than four columns in all are read one by one.
template <typename S>
struct Part {
    static constexpr int kRun = S::kRun;
    int64_t tokens, channels;
    int64_t t;             // first token
    int c, at;             // first column, and the column at which it reads
    bool whole;            // (for the workgroup) all rows are there
    __device__ __forceinline__ Part(const ScanArgs &p, int64_t t0, int64_t c0)
    {
        tokens = p.tokens;
        channels = p.channels;
        t = t0 + S::run();
        c = (int)c0 + S::lane() * kOwn;
        at = c <= channels - kOwn ? c : (int)channels - kOwn;
        whole = t0 + kBlock <= tokens;
    }
    __device__ __forceinline__ int64_t left() const { return channels - c; }
    // what(j, element offset of row j at column `col`)
    template <typename What>
    __device__ __forceinline__ void rows(int64_t ld, int64_t col, What what) const
    {
        if (__builtin_expect(whole, 1)) {
            int64_t o = t * ld + col;
#pragma unroll
            for (int j = 0; j < kRun; ++j, o += ld) what(j, o);
        } else {
#pragma unroll
            for (int j = 0; j < kRun; ++j) what(j, (t + j < tokens ? t + j : tokens - 1) * ld + col);
        }
    }
    template <typename T>
    __device__ __forceinline__ void load(const T *p, int64_t ld, Raw4<T> (&v)[kRun]) const
    {
        if (__builtin_expect(channels >= kOwn, 1)) {
            rows(ld, at, [&](int j, int64_t o) { v[j].load(p + o); });
        } else {
            rows(ld, 0, [&](int j, int64_t o) {
                T w[16 / sizeof(T)] = {};
#pragma unroll
                for (int k = 0; k < kOwn; ++k)
                    if (c + k < channels) w[k] = p[o + c + k];
                __builtin_memcpy(&v[j], w, sizeof v[j]);
            });
        }
    }
    template <typename T>
    __device__ __forceinline__ void settle(Raw4<T> (&v)[kRun], int64_t c0) const
    {
        if (c0 + S::kCh <= channels || channels < kOwn) return;
        const int s = c - at < kOwn ? c - at : kOwn;
#pragma unroll
        for (int j = 0; j < kRun; ++j) v[j].move(s);
    }
};
// THROUGH: past the caches, which leaves them more of what is read a second time: of dy in the backward pass half to three quarters,
// by the bytes that leave the L2 (when this was measured, 32,768 tokens x 2,048 channels, forward and backward: bf16 310 us against
// 322, fp32 417 against 454; 131,072 x 256 forward 57 against 58.7).  An elementwise kernel that reads the result next loses some of it:
// together with the forward pass 0.99 to 1.04 of the time, with the backward pass 0.98 to 1.01.
template <bool THROUGH, typename T>
__device__ __forceinline__ void store4(T *p, int64_t left, const float (&v)[kOwn])
{
    auto put = [](auto *to, auto w) {
        if constexpr (THROUGH) __builtin_nontemporal_store(w, to);
        else *to = w;
    };
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    typedef bf16x4 bf16x4_any __attribute__((aligned(2)));
    if (__builtin_expect(left >= kOwn, 1)) {
        if constexpr (sizeof(T) == 2)
            put(reinterpret_cast<bf16x4_any *>(p), (bf16x4_any)bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]});
        else
            put(reinterpret_cast<f32x4_any *>(p), (f32x4_any)f32x4{v[0], v[1], v[2], v[3]});
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
struct BlockMap {
    int first[kBlock], last[kBlock];       // the sequence of which a token is the first or last, or -1
    int some;                              // some token is either, or outside
};
struct Range { int64_t begin, end; };      // tokens inside sequences

// With many sequences the one that holds the block's first token is searched for, kThreads probes at a time; the offsets
// from it on are looked at up to the block's end.
constexpr int64_t kManySeqs = 4 * kThreads;
__device__ __forceinline__ int64_t first_seq(const ScanArgs &a, int64_t t0)
{
    int64_t lo = 0, hi = a.n_seq;          // the last s in [lo, hi) with seq_start[s] <= t0, or 0
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kThreads - 1) / kThreads, at = lo + threadIdx.x * step;
        const int n = __syncthreads_count(at < hi && a.seq_start[at] <= t0);
        lo += n > 0 ? (n - 1) * step : 0;
        hi = n > 0 && lo + step < hi ? lo + step : n > 0 ? hi : lo + 1;
    }
    return lo;
}
__device__ __forceinline__ Range block_map(const ScanArgs &a, int64_t t0, BlockMap &m)
{
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
        const int64_t from = __builtin_expect(a.n_seq > kManySeqs, 0) ? first_seq(a, t0) : 0;
        for (int64_t s = from + threadIdx.x; s < a.n_seq; s += kThreads) {
            const int64_t p = a.seq_start[s], q = a.seq_start[s + 1];
            mark(s, p, q);
            if (p >= t0 + kBlock) break;
        }
    } else if (threadIdx.x == 0) {
        mark(0, 0, a.tokens);
    }
    if (threadIdx.x == 0 && (r.begin > t0 || r.end < t0 + kBlock)) m.some = 1;
    __syncthreads();
    return r;
}

// Empty sequences hand on what they are given.
template <typename S>
__device__ __forceinline__ void pass_on(const ScanArgs &p, int64_t blk, int64_t c0, const float *from, float *to)
{
    if (!to || !p.seq_start) return;
    const int64_t c = c0 + (threadIdx.x & 63);
    for (int64_t s = blk * kWaves + (threadIdx.x >> 6); s < p.n_seq; s += p.blocks * kWaves)
        if (p.seq_start[s] >= p.seq_start[s + 1] && (threadIdx.x & 63) < S::kCh && c < p.channels)
            to[s * p.channels + c] = from ? from[s * p.channels + c] : 0.0f;
}

// ---- joining runs ------------------------------------------------------------------------------
typedef float2 WavePairs[kWaves][kMostCh];
struct ScanShared {
    BlockMap map;
    WavePairs left, right;                 // pairs of the waves in either direction, then of those before
    WavePairs blocks;                      // pairs of the blocks before, a few to each wave
    float carry[kMostCh];
    float kept[kMostCh];                       // backward: the state that the forward pass kept
    uint32_t ticket;
    __align__(8) uint8_t steps[2][kMostCh / kActGroup][kBlock];   // of x and z: the stored inputs' exponents
};
// The exponents of a block, between global memory (a token's side by side) and LDS (a group's side by side, so that a thread has
// those of its run in one piece).  Each thread takes one token of x or z.
template <typename S>
__device__ __forceinline__ void steps_in(const ScanArgs &p, int64_t t0, int64_t c0, ScanShared &sh)
{
    const int which = threadIdx.x / kBlock, i = threadIdx.x % kBlock;
    const int64_t t = t0 + i < p.tokens ? t0 + i : p.tokens - 1, g = c0 / kActGroup;
    const uint8_t *a = (which ? p.rz : p.rx) + p.lay.steps + t * p.lay.groups + g;
    uint8_t e[S::kCh / kActGroup];
#pragma unroll
    for (int k = 0; k < S::kCh / kActGroup; ++k) e[k] = a[g + k < p.lay.groups ? k : 0];
#pragma unroll
    for (int k = 0; k < S::kCh / kActGroup; ++k) sh.steps[which][k][i] = e[k];
}
template <typename S>
__device__ __forceinline__ void steps_out(const ScanArgs &p, int64_t t0, int64_t c0, const ScanShared &sh)
{
    const int which = threadIdx.x / kBlock, i = threadIdx.x % kBlock;
    const int64_t g = c0 / kActGroup;
    if (t0 + i >= p.tokens) return;
    uint8_t *a = (which ? p.wz : p.wx) + p.lay.steps + (t0 + i) * p.lay.groups + g;
#pragma unroll
    for (int k = 0; k < S::kCh / kActGroup; ++k)
        if (g + k < p.lay.groups) a[k] = sh.steps[which][k][i];
}
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// Sum over the runs of a wave (lanes a multiple of 16 apart, or of 8).
template <int ROWS>
__device__ __forceinline__ float sum_rows(float v)
{
    static_assert(ROWS == 4 || ROWS == 8, "lanes of a run");
    if (ROWS == 8) v += as_f32(dpp_move<0x128>(as_u32(v)));         // the other half of sixteen lanes
    const auto a = __builtin_amdgcn_permlane16_swap(as_u32(v), as_u32(v), false, false);
    v = as_f32(a[0]) + as_f32(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(as_u32(v), as_u32(v), false, false);
    return as_f32(b[0]) + as_f32(b[1]);
}
// m, B: the pair of each thread's run, A packed; A, B: out, that of the runs of its wave before it (REVERSE: behind it).  The wave's
// pair goes to `waves`, for the direction of the chain with A packed.
template <typename S, bool REVERSE, bool SOME, bool CHAIN>
__device__ __forceinline__ void wave_scan(const float (&m)[kOwn], float (&A)[kOwn], float (&B)[kOwn], WavePairs &waves)
{
    constexpr int kLanes = S::kLanes, kRows = S::kRows;
    const int lane = threadIdx.x & 63, cl = S::lane();
    const int pos = REVERSE ? kRows - 1 - lane / kLanes : lane / kLanes;
    auto before = [&](float v, int s) { return __shfl(v, (REVERSE ? lane + kLanes * s : lane - kLanes * s) & 63, 64); };
#pragma unroll
    for (int k = 0; k < kOwn; ++k) A[k] = kept_of(m[k]);
#pragma unroll
    for (int s = 1; s < kRows; s <<= 1)
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const float pa = before(A[k], s), pb = before(B[k], s);
            B[k] = pos >= s ? join<SOME>(A[k], pb, B[k]) : B[k];
            A[k] = pos >= s ? times<SOME>(A[k], pa) : A[k];
        }
    if (pos == kRows - 1)
#pragma unroll
        for (int k = 0; k < kOwn; ++k) waves[wave_id()][cl * kOwn + k] = float2{A[k], B[k]};
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        const float pa = before(A[k], 1), pb = before(B[k], 1);
        A[k] = pos == 0 ? 1.0f : pa;
        B[k] = pos == 0 ? 0.0f : pb;
    }
    if (CHAIN)
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const float d = sum_rows<kRows>(forgotten_of(m[k]) * A[k]);
            if (pos == kRows - 1 && d < 0.5f) waves[wave_id()][cl * kOwn + k].x = -d;
        }
}
// By one wave, a channel to each lane: the waves' pairs become those of all waves before; returns the whole block's.
template <bool REVERSE, bool SOME, bool CHAIN>
__device__ __forceinline__ float2 block_prefix(WavePairs &waves)
{
    const int lane = threadIdx.x & 63;
    float a = 1.0f, b = 0.0f, d = 0.0f;
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // (all eight pairs at once do not fit the registers beside the run's own values)
        float2 p[kWaves / 2];
#pragma unroll
        for (int i = 0; i < kWaves / 2; ++i) p[i] = waves[REVERSE ? kWaves - 1 - half * (kWaves / 2) - i : half * (kWaves / 2) + i][lane];
#pragma unroll
        for (int i = 0; i < kWaves / 2; ++i) {
            const int w = REVERSE ? kWaves - 1 - half * (kWaves / 2) - i : half * (kWaves / 2) + i;
            const float wa = CHAIN ? kept_of(p[i].x) : p[i].x;
            waves[w][lane] = float2{a, b};
            if (CHAIN) d = __builtin_fmaf(a, forgotten_of(p[i].x), d);
            b = join<SOME>(wa, b, p[i].y);
            a = times<SOME>(wa, a);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if (CHAIN && d < 0.5f) a = 1.0f - d;
    return float2{SOME ? a : __builtin_fmaxf(a, kTiny), b};
}
// The state that enters the thread's run, in A's place, from the one that enters the block.
template <typename S, bool SOME>
__device__ __forceinline__ void enter(const float (&A)[kOwn], const float (&B)[kOwn], const WavePairs &waves,
                                      const float (&block)[kOwn], float (&h)[kOwn])
{
    const int cl = S::lane(), wave = wave_id();
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        const float2 w = waves[wave][cl * kOwn + k];
        h[k] = join<SOME>(A[k], join<SOME>(w.x, block[k], w.y), B[k]);
    }
}

constexpr uint64_t kAbsent = ~0ull;
__device__ __forceinline__ uint64_t word(float a, float b) { return (uint64_t)as_u32(a) << 32 | as_u32(b); }
// The word once it is there.  Blocks are handed out in the chain's order, so it comes; still no wait is without a limit (kSpinLimit polls,
// some seconds): at it, the states that depend on the word are NaN, and the status word says so.
constexpr uint32_t kSpinLimit = 1u << 22;
__device__ __forceinline__ uint64_t await(const ScanArgs &p, const uint64_t *from)
{
    uint64_t w = load_dev(from);
    for (uint32_t n = 0; w == kAbsent && n < p.spin_limit; ++n) {
        __builtin_amdgcn_s_sleep(1);
        w = load_dev(from);
    }
    if (__builtin_expect(w == kAbsent, 0)) store_dev(p.status, (int)ZIPML_ETIMEOUT);
    return w;                              // (all ones is a pair of NaNs)
}

// From the waves' pairs to the state that enters block `k` of the chain (k counts in the direction of the scan), in sh.carry; the
// block's own pair, and the state behind it where one is due, are published.  `other` is what a second wave does meanwhile.
template <typename S, bool REVERSE, typename Other>
__device__ __forceinline__ void chain(const ScanArgs &p, int64_t k, int64_t c0, ScanShared &sh, WavePairs &waves, Other other)
{
    const int lane = threadIdx.x & 63, wave = wave_id();
    const int64_t c = c0 + lane;
    const bool live = lane < S::kCh && c < p.channels;
    auto at = [&](int64_t i) { return (REVERSE ? p.blocks - 1 - i : i) * p.channels + c; };
    // the pairs from the last multiple of kSuper on are asked for first, a few by each wave
    constexpr int kEach = kSuper / kWaves;
    const int64_t base = k - k % kSuper, from = base + wave * kEach;
    uint64_t w[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) w[i] = from + i < k && live ? load_dev(p.pairs + at(from + i)) : word(1.0f, 0.0f);
    __syncthreads();                       // the waves' pairs are there
    float2 own{};
    if (wave == 0) {
        own = sh.map.some ? block_prefix<REVERSE, true, true>(waves) : block_prefix<REVERSE, false, true>(waves);
        if (live && p.blocks > 1) store_dev(p.pairs + at(k), word(own.x, own.y));
    } else if (wave == 1) {
        other();
    }
    float a = 1.0f, b = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (w[i] == kAbsent) w[i] = await(p, p.pairs + at(from + i));
        const float wa = as_f32((uint32_t)(w[i] >> 32)), wb = as_f32((uint32_t)w[i]);
        b = join<true>(wa, b, wb);
        a = times<true>(wa, a);
    }
    sh.blocks[wave][lane] = float2{a, b};
    __syncthreads();
    if (wave == 0) {
        float2 q[kWaves];
#pragma unroll
        for (int i = 0; i < kWaves; ++i) q[i] = sh.blocks[i][lane];
        float h = base > 0 && live ? as_f32((uint32_t)await(p, p.supers + (base / kSuper - 1) * p.channels + c)) : 0.0f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) h = join<true>(q[i].x, h, q[i].y);
        sh.carry[lane] = h;
        if (live && k % kSuper == kSuper - 1)
            store_dev(p.supers + k / kSuper * p.channels + c, word(0.0f, join<true>(own.x, h, own.y)));
    }
    __syncthreads();
}

// Which channels and which block a workgroup takes.  Workgroups go to the eight XCDs in turn.  Each XCD gets every group of 64
// channels in turn, not some of them always: rows lie a power of two apart more often than not, so that a group's 128 bytes of
// all rows fall on one or two of an L2's sixteen channels.
struct Place { int64_t k, c0; };
template <typename S>
__device__ __forceinline__ Place take(const ScanArgs &p, ScanShared &sh)
{
    const uint32_t n = (uint32_t)p.groups, b = blockIdx.x, even = (uint32_t)p.blocks / 8 * 8 * n;
    const uint32_t g = (b < even ? b >> 3 : b - even) % n;
    if (p.blocks == 1) {
        if (b == 0 && threadIdx.x == 0) *p.status = ZIPML_OK;
        return Place{0, g * (int64_t)S::kCh};
    }
    if (threadIdx.x == 0) sh.ticket = __hip_atomic_fetch_add(p.counters + g * p.apart, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    return Place{sh.ticket, g * (int64_t)S::kCh};
}

// The words (an even number of them), counters and status of a chain before it starts: a launch, 2 to 5 us.
__global__ __launch_bounds__(256) void k_scan_clear(uint64_t *words, int64_t n, uint32_t *counters, int64_t groups, int *status)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = ZIPML_OK;
    const int64_t step = (int64_t)gridDim.x * 256, i0 = blockIdx.x * 256ll + threadIdx.x;
    u32x4 *w = reinterpret_cast<u32x4 *>(words);
    for (int64_t i = i0; i < n / 2; i += step) w[i] = u32x4{~0u, ~0u, ~0u, ~0u};
    for (int64_t i = i0; i < groups; i += step) counters[i] = 0;
}

// ---- storing and reading the inputs ---------------------------------------------------------------
// The draws of two tokens (rows row, row + 1) of four columns, four halves each.  A Philox block serves eight columns: the two
// lanes that share them make that of one token each and exchange words.
__device__ __forceinline__ void draw_two(uint64_t seed, uint32_t epoch, int64_t row, uint32_t col8, uint32_t stream,
                                         uint32_t (&w)[2][2])
{
    const bool odd = threadIdx.x & 1;
    const Philox4 r = philox_block(seed, epoch, (uint64_t)(row + (odd ? 1 : 0)), col8, stream);
    const uint32_t x0 = dpp_move<0xB1>(odd ? r.w[0] : r.w[2]), x1 = dpp_move<0xB1>(odd ? r.w[1] : r.w[3]);
    w[0][0] = odd ? x0 : r.w[0];
    w[0][1] = odd ? x1 : r.w[1];
    w[1][0] = odd ? r.w[2] : x0;
    w[1][1] = odd ? r.w[3] : x1;
}
// Largest magnitudes of two tokens over a group's 32 columns (eight lanes), as fp32 bits.
__device__ __forceinline__ void top_two(const Raw4<float> &v0, const Raw4<float> &v1, uint32_t (&top)[2])
{
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const u32x4 v = (t ? v1.w : v0.w) & 0x7FFFFFFFu;
        uint32_t m = v[0] > v[1] ? v[0] : v[1];
        const uint32_t n = v[2] > v[3] ? v[2] : v[3];
        m = m > n ? m : n;
        auto most = [&](uint32_t o) { m = m > o ? m : o; };
        most(dpp_move<0xB1>(m));
        most(dpp_move<0x4E>(m));
        most(dpp_move<0x141>(m));
        top[t] = m;
    }
}
__device__ __forceinline__ void top_two(const Raw4<__bf16> &v0, const Raw4<__bf16> &v1, uint32_t (&top)[2])
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    auto most = [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    };
    const u32x2 a = v0.w & 0x7FFF7FFFu, b = v1.w & 0x7FFF7FFFu;
    const uint32_t m = most(a[0], a[1]), n = most(b[0], b[1]);
    // both tokens side by side: 0 in the low half, 1 in the high one
    uint32_t r = most(__builtin_amdgcn_perm(n, m, 0x05040100u), __builtin_amdgcn_perm(n, m, 0x07060302u));
    r = most(r, dpp_move<0xB1>(r));
    r = most(r, dpp_move<0x4E>(r));
    r = most(r, dpp_move<0x141>(r));
    top[0] = r << 16;
    top[1] = r & 0xFFFF0000u;
}
// Codes and step of four columns of a token.  CLAMP: the values are taken as clamped to +-kZMax (a NaN stays one).
template <bool CLAMP, typename T>
__device__ __forceinline__ void encode4(const Raw4<T> &v, uint32_t top, const uint32_t (&w)[2], uint32_t &codes, uint32_t &byte)
{
    bool finite = top < 0x7F800000u;
    if (CLAMP) {
        finite = top <= 0x7F800000u;
        const uint32_t most = as_u32(kZMax);
        top = top < most ? top : most;
    }
    const ActStep s = act_step_of(top);
    float x[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) x[k] = CLAMP ? __builtin_amdgcn_fmed3f(v.of(k), -kZMax, kZMax) : v.of(k);
    codes = finite ? act_codes4<T>(x, s, w[0], w[1], top) : 0u;
    byte = finite ? s.byte : 255u;
}
__device__ __forceinline__ void decode4(uint32_t codes, float step, float (&v)[kOwn])
{
#pragma unroll
    for (int k = 0; k < kOwn; ++k) v[k] = (float)(int8_t)(codes >> (8 * k)) * step;
}

// ---- forward -----------------------------------------------------------------------------------
// What bounds it: storing the inputs, vector instructions (62 a value, 36 of them for the two codes; two thirds of the cycles at
// 32,768 tokens x 2,048 channels, 163 us, 3.3 TB/s); without storing, what a block has to do one after the other -- ticket, loads,
// pairs, state, stores: 8 us, two blocks to a compute unit -- (131,072 x 256: 58 us, 3.5 TB/s; a copy reaches 4.9).  128 tokens to
// a workgroup in place of 256: 241 and 98 us against 229 and 85 (an earlier form), the chain being twice as long.
template <typename T, typename S>
__global__ __launch_bounds__(kThreads, 4) void k_scan_forward(ScanArgs p)
{
    constexpr int kRun = S::kRun, kCh = S::kCh;
    __shared__ ScanShared sh;
    const Place at = take<S>(p, sh);
    const int64_t blk = at.k, t0 = blk * kBlock;
    const int run = S::run();
    const Part<S> part(p, t0, at.c0);
    const int c = part.c;

    Raw4<T> x[kRun], z[kRun];
    part.load((const T *)p.x, p.ldx, x);
    part.load((const T *)p.z, p.ldz, z);
    const Range r = block_map(p, t0, sh.map);
    part.settle(x, at.c0);
    part.settle(z, at.c0);

    if (p.wx && c < p.lay.pitch) {
        const int64_t o = part.t * p.lay.pitch + c;
        uint32_t e[2][kRun / 4] = {};                               // steps of x and z, a byte a token
        auto put = [&](uint8_t *a, int which, int j, uint32_t codes, uint32_t byte) {
            e[which][j >> 2] |= byte << (8 * (j & 3));
            if (part.whole || part.t + j < p.tokens) *reinterpret_cast<uint32_t *>(a + o + j * p.lay.pitch) = codes;
        };
#pragma unroll
        for (int j = 0; j < kRun; j += 2) {
            uint32_t w[2][2], top[2], codes, byte;
            draw_two(p.seed, p.epoch, part.t + j, (uint32_t)(c >> 3), p.stream, w);
            top_two(x[j], x[j + 1], top);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                encode4<false>(x[j + i], top[i], w[i], codes, byte);
                put(p.wx, 0, j + i, codes, byte);
            }
            draw_two(p.seed, p.epoch, part.t + j, (uint32_t)(c >> 3), p.stream + 1, w);
            top_two(z[j], z[j + 1], top);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                encode4<true>(z[j + i], top[i], w[i], codes, byte);
                put(p.wz, 1, j + i, codes, byte);
            }
        }
        if (c % kActGroup == 0)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                __builtin_memcpy(__builtin_assume_aligned(&sh.steps[i][(c - (int)at.c0) / kActGroup][run], kRun), e[i], kRun);
    }
    float a[kRun][kOwn], b[kRun][kOwn], m[kOwn];                    // f and (1 - f) x; the run's A, packed
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        float A = 1.0f, D = 0.0f;
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            float f, g;
            gates(z[j].of(k), f, g);
            a[j][k] = f;
            b[j][k] = g * x[j].of(k);
            D = __builtin_fmaf(g, A, D);
            A *= f;
        }
        m[k] = packed(__builtin_fmaxf(A, kTiny), D);
    }

    const bool some = sh.map.some;
    float A[kOwn], B[kOwn];
    uint32_t reset = 0;                                             // tokens that do not look back
    if (__builtin_expect(!some, 1)) {
#pragma unroll
        for (int k = 0; k < kOwn; ++k) B[k] = b[0][k];
#pragma unroll
        for (int j = 1; j < kRun; ++j)
#pragma unroll
            for (int k = 0; k < kOwn; ++k) B[k] = __builtin_fmaf(a[j][k], B[k], b[j][k]);
        wave_scan<S, false, false, true>(m, A, B, sh.left);
    } else {
#pragma unroll
        for (int k = 0; k < kOwn; ++k) B[k] = 0.0f;
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int64_t t = part.t + j;
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
            for (int k = 0; k < kOwn; ++k) B[k] = reset >> j & 1 ? b[j][k] : __builtin_fmaf(a[j][k], B[k], b[j][k]);
        }
#pragma unroll
        for (int k = 0; k < kOwn; ++k) m[k] = reset ? 0.0f : m[k];
        wave_scan<S, false, true, true>(m, A, B, sh.left);
    }
    chain<S, false>(p, at.k, at.c0, sh, sh.left, [] {});

    float in[kOwn], h[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) in[k] = sh.carry[c - at.c0 + k];
    if (p.wx) steps_out<S>(p, t0, at.c0, sh);
    if (p.states && threadIdx.x < kCh && at.c0 + threadIdx.x < p.channels)
        p.states[blk * p.channels + at.c0 + threadIdx.x] = sh.carry[threadIdx.x];
    auto walk = [&](auto flag) {
        constexpr bool SOME = decltype(flag)::value;                // (a block with all its rows has it false)
        enter<S, SOME>(A, B, sh.left, in, h);
        T *y = (T *)p.y + part.t * p.ldy + c;
#pragma unroll
        for (int j = 0; j < kRun; ++j, y += p.ldy) {
#pragma unroll
            for (int k = 0; k < kOwn; ++k) h[k] = SOME && reset >> j & 1 ? b[j][k] : __builtin_fmaf(a[j][k], h[k], b[j][k]);
            if (!SOME || part.t + j < p.tokens) store4<S::kThrough>(y, part.left(), h);
            __builtin_amdgcn_sched_barrier(0);
            if (SOME && p.h_last && sh.map.last[run + j] >= 0)
                store4<false>(p.h_last + (int64_t)sh.map.last[run + j] * p.channels + c, part.left(), h);
        }
    };
    if (__builtin_expect(some, 0)) walk(std::true_type());
    else walk(std::false_type());
    pass_on<S>(p, blk, at.c0, p.h0, p.h_last);
}

// ---- backward ----------------------------------------------------------------------------------
// p_t = f_t d_t, d_t = dy_t + p_{t+1}, is a scan from right to left with the same factors as that of the states from left to
// right; a run's pairs of both come from one walk: B of the right-to-left one is the sum of d_t times the product of the f
// up to t.  What waits for the chain has to fit 128 registers, so that two workgroups fit a compute unit: f does; g = 1 - f waits in
// LDS, each thread's own in its place; x is decoded and dy read a second time behind the chain (kept in registers, dy costs 2 %
// at 32,768 tokens x 2,048 channels of bf16 and, with 69 registers spilled, 18 % of fp32).
// What bounds it: as in the forward direction, what a block does one after the other, at two blocks to a compute unit (128
// registers a thread; 32,768 tokens x 2,048 channels: 152 us, 3.6 TB/s).  With one block of 232 registers to a compute unit it took
// 321 us against 230 in the same form.  A block in which sequences begin or end takes a path of its own from the pairs on: it is the
// rarer one, and the registers of both together would not fit (stores and loads are counted together, so a register fetched back
// after a store waits for that store).  The common path has no register in memory; the boundary path (fp32: 12 bytes a lane, 8 in the forward pass) and that of fewer
// than four channels (bf16: 52 bytes) have.  Blocks with boundaries take longer, not only for that: 400 sequences in 32,768 x 1,024
// 202 us forward and backward, 8 sequences 177 (fp32 262 and 239).
template <typename S>
struct BackwardShared {
    ScanShared s;
    f32x4 g[S::kRun][kThreads];
};
template <typename T, typename S>
__global__ __launch_bounds__(kThreads, 4) void k_scan_backward(ScanArgs p)
{
    constexpr int kRun = S::kRun, kCh = S::kCh;
    extern __shared__ __align__(16) char lds[];
    BackwardShared<S> &all = *reinterpret_cast<BackwardShared<S> *>(lds);
    ScanShared &sh = all.s;
    const Place at = take<S>(p, sh);
    const int64_t blk = p.blocks - 1 - at.k, t0 = blk * kBlock;
    const int run = S::run();
    const Part<S> part(p, t0, at.c0);
    const int c = part.c;

    uint32_t qx[kRun];
    uint32_t ex[kRun / 4];                                          // the steps of x, a byte a token
    Range r;
    auto step_x = [&](int j) { return act_step(ex[j >> 2] >> (8 * (j & 3)) & 255u); };
    float f[kRun][kOwn];
    Raw4<T> dy[kRun];
    {
        uint32_t qz[kRun];
        const int cc = c < p.lay.pitch ? c : (int)p.lay.pitch - kOwn;
        part.rows(p.lay.pitch, cc, [&](int j, int64_t o) {
            qz[j] = *reinterpret_cast<const uint32_t *>(p.rz + o);
            qx[j] = *reinterpret_cast<const uint32_t *>(p.rx + o);
        });
        part.load((const T *)p.dy, p.lddy, dy);
        const bool keeper = threadIdx.x < kCh && at.c0 + threadIdx.x < p.channels;
        const float kept = keeper ? p.states[blk * p.channels + at.c0 + threadIdx.x] : 0.0f;
        steps_in<S>(p, t0, at.c0, sh);
        if (threadIdx.x < kCh) sh.kept[threadIdx.x] = kept;
        r = block_map(p, t0, sh.map);
        const int group = (c - (int)at.c0) / kActGroup;
        uint32_t ez[kRun / 4];
        __builtin_memcpy(ez, __builtin_assume_aligned(&sh.steps[1][group][run], kRun), kRun);
        __builtin_memcpy(ex, __builtin_assume_aligned(&sh.steps[0][group][run], kRun), kRun);
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            float z[kOwn];
            f32x4 g;
            decode4(qz[j], act_step(ez[j >> 2] >> (8 * (j & 3)) & 255u), z);
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                const float e = __expf(-z[k]);                      // |z| <= kZMax
                f[j][k] = __builtin_amdgcn_rcpf(1.0f + e);
                g[k] = e * f[j][k];
            }
            all.g[j][threadIdx.x] = g;
        }
    }
    const bool some = sh.map.some;
    part.settle(dy, at.c0);

    float A[kOwn], H[kOwn], AR[kOwn], P[kOwn];                      // pairs (A, H) from the left, (AR, P) from the right
    float D[kOwn];                                                  // 1 - A
    uint32_t outside = 0, first = 0, last = 0;                      // tokens, by bit
#pragma unroll
    for (int k = 0; k < kOwn; ++k) { A[k] = 1.0f; H[k] = P[k] = D[k] = 0.0f; }
    if (__builtin_expect(!some, 1)) {
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            float x[kOwn];
            const f32x4 g = all.g[j][threadIdx.x];
            decode4(qx[j], step_x(j), x);
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                D[k] = __builtin_fmaf(g[k], A[k], D[k]);
                A[k] *= f[j][k];
                H[k] = __builtin_fmaf(f[j][k], H[k], g[k] * x[k]);
                P[k] = __builtin_fmaf(A[k], dy[j].of(k), P[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kOwn; ++k) D[k] = packed(A[k], D[k]);
        wave_scan<S, true, false, true>(D, AR, P, sh.right);
        wave_scan<S, false, false, false>(D, A, H, sh.left);
    } else {
        bool cut = false;                                           // a sequence has ended in this run
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int64_t t = part.t + j;
            float x[kOwn], d[kOwn];
            const f32x4 g = all.g[j][threadIdx.x];
            decode4(qx[j], step_x(j), x);
            if (t < r.begin || t >= r.end) {
                outside |= 1u << j;
                cut = true;
#pragma unroll
                for (int k = 0; k < kOwn; ++k) H[k] = 0.0f;
                continue;
            }
#pragma unroll
            for (int k = 0; k < kOwn; ++k) d[k] = dy[j].of(k);
            if (sh.map.last[run + j] >= 0) {
                last |= 1u << j;
                float h[kOwn];
                load_state(p.dh_last, sh.map.last[run + j], p.channels, c, h);
#pragma unroll
                for (int k = 0; k < kOwn; ++k) d[k] += h[k];
            }
            if (sh.map.first[run + j] >= 0) {
                first |= 1u << j;
                load_state(p.h0, sh.map.first[run + j], p.channels, c, H);
            }
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                D[k] = __builtin_fmaf(g[k], A[k], D[k]);
                A[k] *= f[j][k];
                H[k] = __builtin_fmaf(f[j][k], H[k], g[k] * x[k]);
                P[k] = cut ? P[k] : __builtin_fmaf(A[k], d[k], P[k]);
            }
            cut |= last >> j & 1;
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const float m = packed(__builtin_fmaxf(A[k], kTiny), D[k]);
            A[k] = first | outside ? 0.0f : m;
            D[k] = cut ? 0.0f : m;
        }
        wave_scan<S, true, true, true>(D, AR, P, sh.right);
        wave_scan<S, false, true, false>(A, A, H, sh.left);
    }
    chain<S, true>(p, at.k, at.c0, sh, sh.right, [&] {
        if (some) (void)block_prefix<false, true, false>(sh.left);
        else (void)block_prefix<false, false, false>(sh.left);
    });

    auto walk = [&](auto flag) {
        constexpr bool SOME = decltype(flag)::value;                // (a block with all its rows has it false)
        float in[kOwn], q[kOwn];
        part.load((const T *)p.dy, p.lddy, dy);                     // again, out of the caches
        part.settle(dy, at.c0);
#pragma unroll
        for (int k = 0; k < kOwn; ++k) in[k] = sh.carry[c - at.c0 + k];
        enter<S, SOME>(AR, P, sh.right, in, q);
        // the gradient of each state
        float d[kRun][kOwn];
#pragma unroll
        for (int j = kRun - 1; j >= 0; --j) {
            float h[kOwn] = {};
            if (SOME && last >> j & 1) load_state(p.dh_last, sh.map.last[run + j], p.channels, c, h);
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                d[j][k] = dy[j].of(k) + (SOME && last >> j & 1 ? h[k] : q[k]);
                if (SOME && outside >> j & 1) d[j][k] = 0.0f;
                q[k] = SOME && outside >> j & 1 ? 0.0f : f[j][k] * d[j][k];
            }
            if (SOME) __builtin_amdgcn_sched_barrier(0);
            if (SOME && p.dh0 && first >> j & 1)
                store4<false>(p.dh0 + (int64_t)sh.map.first[run + j] * p.channels + c, part.left(), q);
        }
        // the states again, from the one that the forward pass kept
        float h[kOwn];
#pragma unroll
        for (int k = 0; k < kOwn; ++k) in[k] = sh.kept[c - at.c0 + k];
        enter<S, SOME>(A, H, sh.left, in, h);
        T *px = (T *)p.dx + part.t * p.lddx + c, *pz = (T *)p.dz + part.t * p.lddz + c;
#pragma unroll
        for (int j = 0; j < kRun; ++j, px += p.lddx, pz += p.lddz) {
            float x[kOwn], dx[kOwn], dz[kOwn];
            const f32x4 g = all.g[j][threadIdx.x];
            decode4(qx[j], step_x(j), x);
            if (SOME && first >> j & 1) load_state(p.h0, sh.map.first[run + j], p.channels, c, h);
            const bool out = SOME && outside >> j & 1;
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                dx[k] = out ? 0.0f : g[k] * d[j][k];
                dz[k] = out ? 0.0f : f[j][k] * dx[k] * (h[k] - x[k]);
                h[k] = out ? 0.0f : __builtin_fmaf(f[j][k], h[k], g[k] * x[k]);
            }
            if (!SOME || part.t + j < p.tokens) {
                store4<S::kThrough>(px, part.left(), dx);
                store4<S::kThrough>(pz, part.left(), dz);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll
    for (int j = 0; j < kRun; ++j) __asm__ volatile("" : "+v"(qx[j]));   // codes wait for the chain, not the values decoded above
    if (__builtin_expect(some, 0)) walk(std::true_type());
    else walk(std::false_type());
    pass_on<S>(p, blk, at.c0, p.dh_last, p.dh0);
}

// (64 requests x 2,048 channels: 3.3 us, a launch.)
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
            // an open gate by what it forgets, not by what it keeps: h + (b - g h)  (an infinity stays one: h + b)
            const float h = v[k], b = g * xv[k], open = __builtin_fmaf(-g, h, b);
            v[k] = !(g < 0.5f) ? __builtin_fmaf(f, h, b) : __builtin_fabsf(h) == __builtin_inff() ? h + b : h + open;
        }
        store8(s, left, v);
    }
    store8(y + row * ldy + c, left, v);
}

static int64_t scan_blocks(int64_t tokens) { return (tokens + kBlock - 1) / kBlock; }
static bool scan_sizes_ok(int64_t tokens, int64_t channels)
{
    return act_sizes_ok(tokens, channels) && scan_blocks(tokens) * ((channels + Wide::kCh - 1) / Wide::kCh) < (1ll << 32) / kThreads;
}
static bool stride_ok(int64_t ld, int64_t rows, int64_t cols) { return ld >= cols && ld <= (1ll << 60) / rows; }

// Narrow blocks as long as no compute unit gets two of them: a thread has half as much to do one after the other.  Forward and
// backward, bf16: 64 tokens x 2,048 channels 20 us against 27, 1,000 x 512 28 against 35, 2,000 x 1,024 (128 wide blocks) 34
// against 41; above that wide ones read whole lines of codes: 4,000 x 2,048 (512) 71 us narrow, 64 wide.  Without storing the kernel alone
// gains 0 to 10 % and loses as much above.
constexpr int64_t kNarrowMost = 128;

// A line of memory to each counter for up to 512 blocks, which all start at once, or up to 1,024 of few groups; side by side else.
// Measured at 68 sizes, 2 to 128 groups, 160 to 2,560 blocks (bf16, of the time with counters side by side): up to 512 blocks forward 0.76 to
// 1.01 and with the backward pass 0.87 to 1.03, least with 8 to 24 groups; 513 to 1,024 blocks of fewer than 32 groups 0.90 to 1.02 and 0.96 to
// 1.01, of 32 groups 1.01 to 1.09 and 1.00 to 1.04, of 64 and 128 0.93 to 0.99 and 0.98 to 1.00; more blocks 0.98 to 1.09 and 0.99 to 1.07.
// Why the larger calls lose was not found out.
constexpr uint32_t kApart = 16;
static bool start_together(int64_t blocks, int64_t groups) { return blocks * groups <= (groups < 32 ? 1024 : 512); }

// The status word and the chain's words behind one another in the workspace.
struct ScanSpace {
    static constexpr size_t kStatusBytes = 256;
    int64_t pairs, supers, groups;
    int64_t words() const { return (pairs + supers + 1) / 2 * 2; }
    size_t bytes() const { return kStatusBytes + (size_t)words() * 8 + (size_t)groups * 4; }
};
static ScanSpace scan_space(int64_t tokens, int64_t channels)
{
    const int64_t blocks = scan_blocks(tokens);
    if (blocks == 1) return ScanSpace{0, 0, 0};
    return ScanSpace{blocks * channels, blocks / kSuper * channels, (channels + Narrow::kCh - 1) / Narrow::kCh * kApart};
}
static bool scan_narrow(int64_t tokens, int64_t channels)
{
    return scan_blocks(tokens) * ((channels + Wide::kCh - 1) / Wide::kCh) <= kNarrowMost;
}
template <typename S>
static int scan_launch(hipStream_t s, ScanArgs &p, void *workspace, size_t lds, void (*kernel)(ScanArgs))
{
    const ScanSpace w = scan_space(p.tokens, p.channels);
    p.blocks = scan_blocks(p.tokens);
    p.groups = (p.channels + S::kCh - 1) / S::kCh;
    p.status = (int *)workspace;
    p.spin_limit = kSpinLimit;
    if (const long long v = knob(ZIPML_KNOB_SPIN_LIMIT); v >= 0 && v <= (long long)kSpinLimit) p.spin_limit = (uint32_t)v;
    p.pairs = (uint64_t *)((char *)workspace + ScanSpace::kStatusBytes);
    p.supers = p.pairs + w.pairs;
    p.counters = (uint32_t *)(p.pairs + w.words());
    p.apart = start_together(p.blocks, p.groups) ? kApart : 1;
    if (p.blocks > 1) {
        const int64_t n = w.words(), blocks = (n + 511) / 512;
        hipLaunchKernelGGL(k_scan_clear, dim3((uint32_t)(blocks < 1024 ? blocks : 1024)), dim3(256), 0, s, p.pairs, n, p.counters,
                           w.groups, p.status);
    }
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(p.blocks * p.groups)), dim3(kThreads), lds, s, p);
    return hip_check(hipGetLastError());
}
template <typename S>
static int forward_launch(hipStream_t s, ScanArgs &p, void *workspace, int dtype)
{
    return scan_launch<S>(s, p, workspace, 0, dtype == ZIPML_F32 ? k_scan_forward<float, S> : k_scan_forward<__bf16, S>);
}
template <typename S>
static int backward_launch(hipStream_t s, ScanArgs &p, void *workspace, int dtype)
{
    const auto k = dtype == ZIPML_F32 ? k_scan_backward<float, S> : k_scan_backward<__bf16, S>;
    static std::atomic<uint64_t> done[2];
    if (allow_lds((const void *)k, sizeof(BackwardShared<S>), done[dtype == ZIPML_F32])) return ZIPML_ELAUNCH;
    return scan_launch<S>(s, p, workspace, sizeof(BackwardShared<S>), k);
}

}  // namespace zipml

using namespace zipml;

extern "C" size_t zipml_scan_workspace_bytes(int64_t tokens, int64_t channels)
{
    if (!scan_sizes_ok(tokens, channels)) return 0;
    return scan_space(tokens, channels).bytes();
}

extern "C" int zipml_scan_status(void *stream, const void *workspace_dev, size_t workspace_bytes)
{
    if (!workspace_dev || workspace_bytes < ScanSpace::kStatusBytes) return ZIPML_EWORKSPACE;
    if (!aligned16(workspace_dev)) return ZIPML_EALIGN;
    int st = 0;
    hipStream_t s = entry_stream(stream);
    if (HIP_FAILED(hipMemcpyAsync(&st, workspace_dev, sizeof(int), hipMemcpyDeviceToHost, s))) return ZIPML_ELAUNCH;
    if (HIP_FAILED(hipStreamSynchronize(s))) return ZIPML_ELAUNCH;
    return st;
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
    hipStream_t s = entry_stream(stream);
    return scan_narrow(tokens, channels) ? forward_launch<Narrow>(s, p, workspace_dev, dtype)
                                         : forward_launch<Wide>(s, p, workspace_dev, dtype);
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
    hipStream_t s = entry_stream(stream);
    return scan_narrow(tokens, channels) ? backward_launch<Narrow>(s, p, workspace_dev, dtype)
                                         : backward_launch<Wide>(s, p, workspace_dev, dtype);
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
    if (rows > ((1ll << 32) - 256) / ((channels + 7) / 8)) return ZIPML_EINVAL;   // threads of a launch
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
