// Linear layer on 8-bit codes: y[t][o] = (sum_i x[t][i] w[o][i]) sx[t] sw[o] + bias[o], x and w codes with a scale a row.
//
// The sums are integers: exact in any order (|code| <= 128 and d_in < 2^17 keep them in 32 bits), so how the contraction is split
// changes no bit of the result.  Both operands are contracted along their rows, 16 codes of a row are 16 bytes, and a lane of
// the matrix instructions wants just those of one row: tiles lie in LDS as they lie in memory, and are read 16 bytes at a time.
//
// Two kinds of kernels, chosen by a model of their times (product_plan): few tokens or outputs are bound by the bytes of W and by latency
// (one token, 4,096 x 4,096: 5.4 us, 3.4 at the rate of a copy, 1.4 an empty launch; 64 tokens, 8,192 -> 1,024: 6.0; 1,000 tokens,
// 520 -> 1,001, fp32: 6.1), many of both by the power that the matrix cores draw, and a third of their cycles in which they wait (16,384
// tokens, 4,096 x 4,096: 207 to 220 us from box to box, 2,500 to 2,650 TOP/s, to fp32 221 on the first of them; a library product of the same
// codes without scales 232 to 285; 4,096 tokens, 16,384 -> 4,096: 195 to 208 us, 2,640 to 2,820 TOP/s, the library 211 to 223).  With the
// first, 134 MB of results go out.
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
    int range, ranges;          // bytes of a row that a workgroup takes, a multiple of kStep; how many such ranges there are
    int through;                // results go past the caches
    int64_t part;               // sums of a range, [rows][ldy], behind those of the one before
};

// Results of which the caches would hold little until they are read, in rows that begin at a line of 128 bytes, are written past them:
// 16,384 x 4,096 bf16 and 520 inputs 60 us against 70 (with an elementwise kernel that reads them next 106 against 110), 4,096 inputs 223
// against 233, 8,192 x 4,096 and 520 inputs 32 against 34 (54 against 56); 4,096 x 4,096 is slower to read next (30 against 28.7 for both).
// Rows that share lines need the caches to put these together: 10,022 x 8,825, 112 inputs, 142 us past them and 74 through them.
constexpr int64_t kThroughLeast = 48ll << 20;
constexpr int kComputeUnits = 256;
constexpr int kStep = 128;      // codes of a row that are in LDS at a time (2^7)

// Rows of codes as a buffer: rows behind the last one, and what lies behind a row's padding, read as zeros.
struct CodeRows {
    __amdgpu_buffer_rsrc_t r;
    int ld, bytes;
    CodeRows() = default;
    __device__ __forceinline__ CodeRows(const uint8_t *base, int64_t left, int64_t ld_, int bytes_) : ld((int)ld_), bytes(bytes_)
    {
        const int64_t n = (left - 1) * ld_ + bytes_;
        r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), 0, left < 1 ? 0 : n > 0x7FFE0000 ? 0x7FFE0000 : (int)n, 0x00020000);
    }
    // 16 codes at an offset, `rows` rows further down; zeros where there are none
    __device__ __forceinline__ u32x4 load16(bool there, int at, int rows) const
    {
        return __builtin_amdgcn_raw_buffer_load_b128(r, there ? at + rows * ld : 0x7FFFFFF0, 0, 0);
    }
};

// Where the 16 bytes `chunk` of a row lie in an LDS tile: turned by the row's number, so that 16 rows' same chunk, which 16 lanes
// read at once, fall on all banks.
__device__ __forceinline__ int lds_at(int row, int chunk) { return row * kStep + ((chunk ^ (row >> 1 & 7)) << 4); }

// Orders a wave's own LDS accesses, of all its lanes.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Scales (and bias) of four neighbouring outputs and of a token, and four results from them.
struct Out4 {
    f32x4 sw, bias;
    float sx;
    int n;                      // how many of the outputs there are
    __device__ __forceinline__ Out4() {}
    __device__ __forceinline__ Out4(const ProductArgs &a, int64_t t, int o) : n(a.d_out - o)
    {
        const auto scales = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(a.sw), 0, a.d_out * 4, 0x00020000);
        const auto biases = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(a.bias), 0, a.bias ? a.d_out * 4 : 0, 0x00020000);
        sw = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(scales, o * 4, 0, 0));
        bias = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(biases, o * 4, 0, 0));
        sx = a.sx[t < a.rows ? t : a.rows - 1];
    }
    template <typename T>
    __device__ __forceinline__ void put(const ProductArgs &a, T *y, i32x4 sum) const
    {
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = (float)sum[k] * sx * sw[k];
            if (a.bias) v[k] += bias[k];
        }
        if (n >= 4) {
            typedef T T4 __attribute__((ext_vector_type(4)));
            typedef T4 T4_any __attribute__((aligned(sizeof(T))));
            *reinterpret_cast<T4_any *>(y) = T4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < n) y[k] = (T)v[k];
        }
    }
};

// Workgroups go to the eight XCDs in turn; each XCD gets a run of neighbouring tiles, in bands eight outputs deep, so that its L2
// serves rows of both operands to several of them (16,384 tokens, 4,096 x 4,096: 237 us, with four or sixteen 240).
__device__ __forceinline__ void tile_of(const ProductArgs &a, uint32_t n, uint32_t at, int &o, int &t)
{
    const uint32_t xcd = at & 7, per = n >> 3, more = n & 7;
    const uint32_t id = xcd * per + (xcd < more ? xcd : more) + (at >> 3), band = id / (8 * a.tiles_t), in = id - band * 8 * a.tiles_t;
    const uint32_t deep = a.tiles_o - band * 8 < 8 ? a.tiles_o - band * 8 : 8;
    o = band * 8 + in % deep;
    t = in / deep;
}

// ---- many tokens: tiles whose waves share the rows ----------------------------------------------
// MO x MT outputs x tokens of a workgroup, WO x WT waves.  16 x 16 x 64 instructions: what bounds large products is the power that the
// matrix cores draw, and on random codes these do 3,985 TOP/s by themselves where 32 x 32 x 32 ones do 3,310 (on zeros 4,710 and 4,785).
template <typename T, int MO_, int MT_, int WO_, int WT_>
struct ProductShape {
    static constexpr int MO = MO_, MT = MT_, WO = WO_, WT = WT_, kThreads = 64 * WO * WT;
    static constexpr int TO = MO / WO / 16, TT = MT / WT / 16;      // 16 x 16 tiles of a wave
    static constexpr int kLoadsW = MO * kStep / 16 / kThreads, kLoadsX = MT * kStep / 16 / kThreads, kLoads = kLoadsW + kLoadsX;
    static constexpr int kStage = (MO + MT) * kStep;
    static constexpr int kBeats = kStep / 64 * TO;                  // of a round: 64 codes of 16 outputs, times all tokens
    static constexpr bool kParts = std::is_same<T, int>::value;     // sums of a range of the contraction, not results
    static constexpr int HO = 8 / (int)sizeof(T);                   // tiles side by side in a line of 128 bytes of results
    static constexpr int kOut = 32 * 128;                           // LDS of a wave's results on their way out: 32 tokens
    static constexpr bool kStay = MO * MT == 256 * 256;
    static constexpr int kLds = kStay ? 2 * kStage + kOut * WO * WT : 2 * kStage > kOut * WO * WT ? 2 * kStage : kOut * WO * WT;
    static_assert(kLoadsW * 16 * kThreads == MO * kStep && kLoadsX * 16 * kThreads == MT * kStep, "whole loads");
    static_assert(TO % HO == 0 && TT % 2 == 0 && kBeats % 4 == 0 && kLoads <= kBeats - 2, "beats");
    static_assert(kLds <= 160 * 1024, "LDS");
};

// What a wave has summed, on its way out.  A lane holds four neighbouring outputs of one token at a time.  Through LDS of its own (`out`), a
// wave turns 32 tokens' lines of 128 bytes around and writes them 16 bytes a lane.
template <typename T, typename S, bool THROUGH>
__device__ __forceinline__ void write_out(const ProductArgs &a, const i32x4 (&acc)[S::TO][S::TT], char *out, int o_wave, int64_t t_wave,
                                          uint32_t split)
{
    const int lane = threadIdx.x & 63;
    const auto scales = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(a.sw), 0, a.d_out * 4, 0x00020000);
    const auto biases = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(a.bias), 0, a.bias ? a.d_out * 4 : 0, 0x00020000);
    float sx[S::TT];
#pragma unroll
    for (int n = 0; n < S::TT && !S::kParts; ++n) {
        const int64_t t = t_wave + n * 16 + (lane & 15);
        sx[n] = a.sx[t < a.rows ? t : a.rows - 1];
    }
    // (all at once: a load at each use waited for the one before, 15 us a tile of 256 x 256)
    f32x4 sw[S::TO];
    const int at = (o_wave + 4 * (lane >> 4)) * 4;
#pragma unroll
    for (int m = 0; m < S::TO && !S::kParts; ++m)
        sw[m] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(scales, at + m * 64, 0, 0));
    // (a token's lines one after the other: rows that do not begin at a line's start share lines, which the L2 has to put together)
#pragma unroll
    for (int n0 = 0; n0 < S::TT; n0 += 2) {
#pragma unroll
        for (int m0 = 0; m0 < S::TO; m0 += S::HO) {
            constexpr int V = 16 / (int)sizeof(T);                  // results in 16 bytes
            const int o = o_wave + m0 * 16 + (lane & 7) * V, left = a.d_out - o;
            f32x4 bias[S::HO];                                      // (-0 leaves every value as it is)
#pragma unroll
            for (int m = 0; m < S::HO; ++m) bias[m] = f32x4{-0.0f, -0.0f, -0.0f, -0.0f};
            if (a.bias && !S::kParts)
#pragma unroll
                for (int m = 0; m < S::HO; ++m)
                    bias[m] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(biases, at + (m0 + m) * 64, 0, 0));
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int m = 0; m < S::HO; ++m) {
                    typedef T T4 __attribute__((ext_vector_type(4)));
                    T4 r;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int sum = acc[m0 + m][n0 + n][k];
                        if constexpr (S::kParts) r[k] = sum;
                        else r[k] = (T)((float)sum * sx[n0 + n] * sw[m0 + m][k] + bias[m][k]);
                    }
                    const int row = n * 16 + (lane & 15), byte = (m * 16 + 4 * (lane >> 4)) * (int)sizeof(T);
                    *reinterpret_cast<T4 *>(out + lds_at(row, byte >> 4) + (byte & 15)) = r;
                }
            wave_fence();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 8 * i + (lane >> 3);
                const u32x4 line = *reinterpret_cast<const u32x4 *>(out + lds_at(r, lane & 7));
                const int64_t t = t_wave + n0 * 16 + r;
                if (t >= a.rows) continue;
                T *const y = (T *)a.y + split * a.part + t * a.ldy + o;
                if (left >= V) {
                    if constexpr (THROUGH) __builtin_nontemporal_store((u32x4_any)line, reinterpret_cast<u32x4_any *>(y));
                    else *reinterpret_cast<u32x4_any *>(y) = line;
                } else {
#pragma unroll
                    for (int k = 0; k < V; ++k)
                        if (k < left) {
                            const uint32_t word = line[k * (int)sizeof(T) / 4];   // (a cast of the vector's element itself takes its first)
                            if constexpr (sizeof(T) == 4) y[k] = __builtin_bit_cast(T, word);
                            else y[k] = __builtin_bit_cast(__bf16, (uint16_t)(word >> (16 * (k & 1))));
                        }
                }
            }
            wave_fence();
        }
    }
}

// THROUGH: results are written past the caches (a kernel of its own: of a branch the compiler makes one store, which is not).
// Where one workgroup fills a compute unit (S::kStay) it stays and takes every gridDim.x-th piece of work: the first two rounds of the next
// are under way during the last two of the one before and while its results are written (16,384 tokens, 520 -> 4,096: 61 -> 56 us).
// (Two waves a SIMD at least: with all 512 registers to itself a wave of 128 x 64 keeps its sums in the upper half and moves them in each
// round, 1,024 tokens, 4,096 -> 2,048: 19.7 us in place of 15.6.)
template <typename T, typename S, bool THROUGH>
__global__ __launch_bounds__(S::kThreads, 2) void k_row8_product(ProductArgs a)
{
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wo = wave / S::WT, wt = wave % S::WT;
    const uint32_t tiles = (uint32_t)a.tiles_o * a.tiles_t, work = tiles * a.ranges;
    // where a piece of work (a tile, a range of its contraction) lies
    struct Place {
        int o0, k_begin, k_end;
        int64_t t0;
        uint32_t split;
    };
    auto place = [&](uint32_t at) {
        Place p;
        int tile_o, tile_t;
        p.split = at / tiles;
        tile_of(a, tiles, at - p.split * tiles, tile_o, tile_t);
        p.o0 = tile_o * S::MO;
        p.t0 = (int64_t)tile_t * S::MT;
        p.k_begin = (int)p.split * a.range;
        p.k_end = p.k_begin + a.range < a.bytes ? p.k_begin + a.range : a.bytes;
        return p;
    };

    // What is loaded next: 128 codes from k_load on of these rows.
    constexpr int kRowsLoad = S::kThreads / 8;                      // rows that one load of all threads takes
    const int at_w = (tid >> 3) * (int)a.ldw + (tid & 7) * 16, at_x = (tid >> 3) * (int)a.ldx + (tid & 7) * 16;
    CodeRows w, x;
    uint32_t load_at = blockIdx.x;
    int k_load = 0, k_stop = 0;
    auto take = [&]() {
        const bool there = load_at < work;
        const Place p = place(there ? load_at : 0);
        w = CodeRows(a.w + p.o0 * a.ldw, there ? a.d_out - p.o0 : 0, a.ldw, a.bytes);
        x = CodeRows(a.x + p.t0 * a.ldx, there ? a.rows - p.t0 : 0, a.ldx, a.bytes);
        k_load = p.k_begin;
        k_stop = p.k_end;
    };
    auto loaded = [&]() {
        k_load += kStep;
        if (S::kStay && k_load >= k_stop) {
            load_at += gridDim.x;
            take();
        }
    };
    auto load = [&](int q) {
        const bool there = k_load + (tid & 7) * 16 < a.bytes;
        return q < S::kLoadsW ? w.load16(there, at_w + k_load, q * kRowsLoad) : x.load16(there, at_x + k_load, (q - S::kLoadsW) * kRowsLoad);
    };
    auto store = [&](u32x4 v, char *stage, int q) {
        const int c = tid + (q < S::kLoadsW ? q : q - S::kLoadsW) * S::kThreads;
        *reinterpret_cast<u32x4 *>(stage + (q < S::kLoadsW ? 0 : S::MO * kStep) + lds_at(c >> 3, c & 7)) = v;
    };

    // While a round is multiplied, the next one goes from registers to LDS, and each register is loaded anew for the one after it.  A
    // beat's rows of W are read two beats ahead, all of its tokens' codes in the two beats before their first; so the barrier stands
    // two beats before the round's end.  What a beat reads, stores and loads stands between its products, in this order (216 us in place of
    // 220 for 16,384 tokens, 4,096 x 4,096, with all of it before them); the compiler otherwise moves all loads to a round's end.  A load
    // has one round until its register is stored, which is short in 128-wide tiles: by the constants below 0.47 and 0.55 us, their products
    // alone 0.21 and 0.43.
    i32x4 fw[4], fx[2][S::TT];
    auto read_w = [&](const char *stage, int beat) {
        const int m = beat % S::TO, s = beat / S::TO;
        fw[beat & 3] = *reinterpret_cast<const i32x4 *>(stage + lds_at((wo * S::TO + m) * 16 + (lane & 15), 4 * s + (lane >> 4)));
    };
    auto read_x = [&](const char *stage, int s, int half) {
#pragma unroll
        for (int n = half * S::TT / 2; n < (half + 1) * S::TT / 2; ++n)
            fx[s][n] = *reinterpret_cast<const i32x4 *>(stage + S::MO * kStep + lds_at((wt * S::TT + n) * 16 + (lane & 15), 4 * s + (lane >> 4)));
    };
    char *here = lds, *next = lds + S::kStage;
    u32x4 v[S::kLoads];
    take();
    {                                      // both first rounds asked for at once: the memory's latency once, not twice
        u32x4 first[S::kLoads];
#pragma unroll
        for (int q = 0; q < S::kLoads; ++q) first[q] = load(q);
        loaded();
#pragma unroll
        for (int q = 0; q < S::kLoads; ++q) v[q] = load(q);
        loaded();
#pragma unroll
        for (int q = 0; q < S::kLoads; ++q) store(first[q], here, q);
    }
    lds_barrier();
    for (uint32_t at = blockIdx.x; at < work; at += gridDim.x) {
        const Place p = place(at);
        i32x4 acc[S::TO][S::TT] = {};
        read_x(here, 0, 0);
        read_w(here, 0);
        read_x(here, 0, 1);
        read_w(here, 1);
        for (int k0 = p.k_begin; k0 < p.k_end; k0 += kStep) {
#pragma unroll
            for (int beat = 0; beat < S::kBeats; ++beat) {
                const int ahead = beat + 2;
#pragma unroll
                for (int n = 0; n < S::TT; ++n) {
                    acc[beat % S::TO][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[beat & 3], fx[beat / S::TO][n], acc[beat % S::TO][n], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if (n == 0) {
                        if (ahead == S::kBeats) lds_barrier();
                        read_w(ahead < S::kBeats ? here : next, ahead % S::kBeats);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    if (n == S::TT / 4 && ahead % S::TO < 2) {
                        read_x(ahead < S::kBeats ? here : next, ahead / S::TO & 1, ahead % S::TO);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int q = 0; q < S::kLoads; ++q)
                        if (q * (S::kBeats - 2) / S::kLoads == beat) {
                            if (n == S::TT / 2) store(v[q], next, q);
                            if (n == S::TT * 3 / 4) v[q] = load(q);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                }
            }
            loaded();
            char *const t = here;
            here = next;
            next = t;
        }
        if (!S::kStay) lds_barrier();          // (the results lie where another wave may still read)
        write_out<T, S, THROUGH>(a, acc, lds + (S::kStay ? 2 * S::kStage : 0) + wave * S::kOut, p.o0 + wo * S::TO * 16, p.t0 + wt * S::TT * 16, p.split);
        if (!S::kStay) return;
    }
}

// ---- few tokens, few outputs: the waves of a workgroup share the contraction -------------------
// Where a tile has few products for its bytes, nothing is gained by sharing rows between waves; what counts is that all of a
// compute unit's waves have loads under way.  So the waves of a workgroup take steps of 128 codes of the same MO x MT tile by turns,
// each through LDS of its own and without a barrier, and add up their sums at the end.
template <int MO_, int MT_, int WAVES_>
struct SplitShape {
    static constexpr int MO = MO_, MT = MT_, WAVES = WAVES_, kThreads = 64 * WAVES;
    static constexpr bool kSmall = MO == 16;                      // 16 x 16 x 64 instructions, otherwise 32 x 32 x 32
    static constexpr int kLoadsW = MO / 8, kLoadsX = MT / 8;
    static constexpr int TO = kSmall ? 1 : MO / 32, TT = kSmall ? 1 : MT / 32;
    static constexpr int kStage = (MO + MT) * kStep;
    static constexpr int kRow = MO + 4;                           // a token's sums in LDS, with room against bank conflicts
    static constexpr int kSums = MT * kRow * 4;
    static constexpr int kWave = kStage > kSums ? kStage : kSums; // LDS of a wave
    static constexpr int kLds = kWave * WAVES;
    static constexpr bool kStay = false;
    static_assert(kSmall ? MT == 16 : MO % 32 == 0 && MT % 32 == 0, "tile");
    static_assert(kLds <= 160 * 1024, "LDS");
};

template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void k_row8_product_split(ProductArgs a)
{
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tile_o = blockIdx.x % a.tiles_o, tile_t = blockIdx.x / a.tiles_o;
    const int o0 = tile_o * S::MO;
    const int64_t t0 = (int64_t)tile_t * S::MT;
    const CodeRows w(a.w + o0 * a.ldw, a.d_out - o0, a.ldw, a.bytes), x(a.x + t0 * a.ldx, a.rows - t0, a.ldx, a.bytes);
    char *const mine = lds + wave * S::kWave;

    u32x4 vw[S::kLoadsW], vx[S::kLoadsX];
    const int at_w = (lane >> 3) * (int)a.ldw + (lane & 7) * 16, at_x = (lane >> 3) * (int)a.ldx + (lane & 7) * 16;
    auto load = [&](int k0) {
        const bool there = k0 + (lane & 7) * 16 < a.bytes;
#pragma unroll
        for (int q = 0; q < S::kLoadsW; ++q) vw[q] = w.load16(there, at_w + k0, q * 8);
#pragma unroll
        for (int q = 0; q < S::kLoadsX; ++q) vx[q] = x.load16(there, at_x + k0, q * 8);
    };
    load(wave * kStep);
    // what the results need, long before they are there (5.7 -> 5.4 us at one token, 4,096 x 4,096)
    constexpr int kUnits = S::MT * S::MO / 4, kMine = (kUnits + S::kThreads - 1) / S::kThreads;
    Out4 out[kMine];
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        const int i = threadIdx.x + k * S::kThreads;
        if (kUnits % S::kThreads == 0 || i < kUnits) out[k] = Out4(a, t0 + i / (S::MO / 4), o0 + i % (S::MO / 4) * 4);
    }
    i32x16 acc[S::TO][S::TT] = {};
    i32x4 small = {};
    for (int k0 = wave * kStep; k0 < a.bytes; k0 += S::WAVES * kStep) {
#pragma unroll
        for (int q = 0; q < S::kLoadsW; ++q)
            *reinterpret_cast<u32x4 *>(mine + lds_at(q * 8 + (lane >> 3), lane & 7)) = vw[q];
#pragma unroll
        for (int q = 0; q < S::kLoadsX; ++q)
            *reinterpret_cast<u32x4 *>(mine + S::MO * kStep + lds_at(q * 8 + (lane >> 3), lane & 7)) = vx[q];
        wave_fence();
        load(k0 + S::WAVES * kStep);
        const char *const pw = mine, *const px = mine + S::MO * kStep;
        if constexpr (S::kSmall) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int at = lds_at(lane & 15, 4 * s + (lane >> 4));
                small = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(pw + at),
                                                              *reinterpret_cast<const i32x4 *>(px + at), small, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                i32x4 fw[S::TO], fx[S::TT];
#pragma unroll
                for (int m = 0; m < S::TO; ++m)
                    fw[m] = *reinterpret_cast<const i32x4 *>(pw + lds_at(m * 32 + (lane & 31), 2 * s + (lane >> 5)));
#pragma unroll
                for (int n = 0; n < S::TT; ++n)
                    fx[n] = *reinterpret_cast<const i32x4 *>(px + lds_at(n * 32 + (lane & 31), 2 * s + (lane >> 5)));
#pragma unroll
                for (int m = 0; m < S::TO; ++m)
#pragma unroll
                    for (int n = 0; n < S::TT; ++n) acc[m][n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[m], fx[n], acc[m][n], 0, 0, 0);
            }
        }
        wave_fence();
    }

    // [token][output] of each wave, then the waves' sums
    int *const sums = reinterpret_cast<int *>(mine);
    if constexpr (S::kSmall) {
        *reinterpret_cast<i32x4 *>(sums + (lane & 15) * S::kRow + 4 * (lane >> 4)) = small;
    } else {
#pragma unroll
        for (int m = 0; m < S::TO; ++m)
#pragma unroll
            for (int n = 0; n < S::TT; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<i32x4 *>(sums + (n * 32 + (lane & 31)) * S::kRow + m * 32 + 8 * q + 4 * (lane >> 5)) =
                        i32x4{acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
    }
    lds_barrier();
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        const int i = threadIdx.x + k * S::kThreads, t = i / (S::MO / 4), o = i % (S::MO / 4) * 4;
        if (i >= kUnits || t0 + t >= a.rows || o0 + o >= a.d_out) continue;
        i32x4 sum = {};
#pragma unroll
        for (int v = 0; v < S::WAVES; ++v) sum += *reinterpret_cast<const i32x4 *>(lds + v * S::kWave + (t * S::kRow + o) * 4);
        out[k].put(a, (T *)a.y + (t0 + t) * a.ldy + o0 + o, sum);
    }
}

// Results from the sums of the ranges: four neighbouring outputs of a token a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_row8_product_join(ProductArgs a, const int *part, int64_t ld_part, int ranges)
{
    const uint32_t units = (uint32_t)(ld_part / 4);
    const int64_t i = blockIdx.x * 256ll + threadIdx.x, t = i / units;
    const int o = (int)(i - t * units) * 4;
    if (t >= a.rows) return;
    const Out4 out(a, t, o);
    const int *p = part + t * ld_part + o;
    i32x4 sum = *reinterpret_cast<const i32x4 *>(p);
#pragma unroll 4
    for (int r = 1; r < ranges; ++r) sum += *reinterpret_cast<const i32x4 *>(p + r * a.part);
    out.put(a, (T *)a.y + t * a.ldy + o, sum);
}

// The shapes: tiles whose waves share the contraction (outputs, tokens, waves), tiles whose waves share the rows (outputs, tokens, waves
// along each).
#define ZIPML_PRODUCT_SPLIT(F)                                                                                                  \
    F(0, 16, 16, 4) F(1, 16, 16, 8) F(2, 16, 16, 16) F(3, 32, 32, 4) F(4, 32, 32, 8) F(5, 32, 32, 16) F(6, 64, 32, 8) F(7, 64, 64, 8)
#define ZIPML_PRODUCT_TILE(F) F(8, 128, 64, 2, 2) F(9, 128, 128, 2, 4) F(10, 256, 256, 2, 4)

// Which shape, and (of the second kind) in how many ranges the contraction is taken, whose sums a second launch joins: the least of
//   start + further turns of a compute unit * turn + rounds of 128 codes of a wave * (one workgroup on a compute unit: lone, k of
//   them: k * shared, k the most for the second kind, for the first, which wait for memory that all share, the mean) + (ranges > 1: a
//   launch, sums written and read).
// The constants (us) are those that come nearest to 4,700 times measured over 253 sizes, 1 to 60,000 tokens, 20 to 16,000 outputs, 100 to
// 32,000 inputs, both types, all shapes and numbers of ranges below; the choice is 3 % slower than the fastest on average, 14 % in one of
// twenty, a third at most (16 ranges, or k the most for both: 18 % in one of twenty).  They order the shapes; a time by itself may be a fifth
// off (1,000 tokens, 4,096 x 4,096: 21.7 us by the model, 21.6 to 26 measured).
struct ProductPlan {
    int shape, ranges, range;              // range: bytes of a row
    size_t workspace;
};
// room: bytes that the sums of ranges may take.  What is wanted falls and rises with the rows (10,240 -> 2,560: 12 MB at 300 tokens, none at
// 1,024, 63 MB at 2,048); with less the contraction is taken in fewer ranges, which changes no bit (512 tokens 26 us, with no room at all 38;
// 195 tokens, 18,880 -> 7,035, 47 and 101).
static ProductPlan product_plan(int64_t rows, int64_t d_out, int64_t d_in, size_t room)
{
    // outputs, tokens and waves of a tile as powers of two: the choice is made in every call, and divisions are what it would cost
    struct Cost { int outs, tokens, waves; double start, turn, lone, shared; };
    static const Cost costs[] = {
        {4, 4, 2, 2.18, 0.00, 0.29, 0.25}, {4, 4, 3, 2.15, 0.00, 0.47, 0.50},
        {4, 4, 4, 1.87, 0.00, 0.91, 1.12}, {5, 5, 2, 2.25, 0.03, 0.56, 0.51},
        {5, 5, 3, 2.15, 0.04, 0.95, 1.05}, {5, 5, 4, 1.22, 0.00, 2.09, 2.44},
        {6, 5, 3, 2.19, 2.25, 1.50, 1.37}, {6, 6, 3, 3.03, 3.28, 1.95, 1.89},
        {7, 6, 0, 3.69, 1.30, 0.47, 0.41}, {7, 7, 0, 4.05, 2.55, 0.55, 0.58},
        {8, 8, 0, 9.44, 11.96, 1.25, 1.40},
    };
    const auto parts = [](int64_t n, int log) { return (n + (1ll << log) - 1) >> log; };
    const int64_t bytes = round_up(d_in, kRow8Unit), sums = rows * round_up(d_out, 4) * 4;
    ProductPlan best{-1, 1, 0, 0};
    double least = 0;
    for (int shape = 0; shape < (int)(sizeof(costs) / sizeof(costs[0])); ++shape) {
        const Cost &c = costs[shape];
        const int64_t tiles = parts(d_out, c.outs) * parts(rows, c.tokens);
        // (a launch has fewer than 2^32 threads; the second kind's tiles are shared by eight waves at most, of the last shape 256 workgroups stay)
        const bool stays = c.outs == 8;
        if ((!stays && tiles >= (1ll << 32) >> (6 + (c.waves > 0 ? c.waves : 3))) || (best.shape >= 0 && c.start + (double)(parts(tiles, 8) - 1) * c.turn >= least)) continue;
        for (const int wanted : {1, 2, 3, 4, 8}) {
            // (ranges of two rounds at least, whose sums stay in the caches)
            if (wanted > 1 && (c.waves > 0 || bytes < 2 * wanted * kStep || wanted * sums > (1ll << 28) || wanted * tiles > (1 << 16))) break;
            const int64_t range = wanted == 1 ? parts(bytes, 7) << 7 : round_up((bytes + wanted - 1) / wanted, kStep);
            const int64_t ranges = wanted == 1 ? 1 : (bytes + range - 1) / range;
            if (ranges > 1 && (size_t)(ranges * sums) > room) break;
            const double k = (double)parts(tiles * ranges, 8), rounds = (double)parts(range < bytes ? range : bytes, 7 + c.waves);
            const double busy = c.waves > 0 ? (double)tiles * (1.0 / 256) : k;
            const double us = c.start + (k - 1) * c.turn + rounds * (k > 1 && busy * c.shared > c.lone ? busy * c.shared : c.lone) +
                              (ranges > 1 ? 3.0 + (double)(ranges * sums) * 2 / 6.4e6 : 0.0);
            if (best.shape < 0 || us < least) {
                least = us;
                best = ProductPlan{shape, (int)ranges, (int)range, ranges > 1 ? (size_t)(ranges * sums) : 0};
            }
        }
    }
    return best;
}

// Workgroups that a shape is launched with.
template <typename S>
static int64_t product_groups(int64_t rows, int64_t d_out, int ranges)
{
    const int64_t all = (rows + S::MT - 1) / S::MT * ((d_out + S::MO - 1) / S::MO) * ranges;
    return S::kStay && all > kComputeUnits ? kComputeUnits : all;
}

// (T tells kernels of one shape apart: each is asked for its LDS once)
template <typename T, typename S, typename K>
static int launch_tiles(hipStream_t s, ProductArgs a, K k)
{
    a.tiles_o = (a.d_out + S::MO - 1) / S::MO;
    a.tiles_t = (int)((a.rows + S::MT - 1) / S::MT);
    static std::atomic<uint64_t> done[2];
    if (allow_lds((const void *)k, S::kLds, done[a.through])) return ZIPML_ELAUNCH;
    hipLaunchKernelGGL(k, dim3((uint32_t)product_groups<S>(a.rows, a.d_out, a.ranges)), dim3(S::kThreads), S::kLds, s, a);
    return hip_check(hipGetLastError());
}

template <typename T>
static int launch_product(hipStream_t s, ProductArgs a, const ProductPlan &p, void *workspace)
{
    a.range = p.range;
    a.ranges = p.ranges;
    a.part = 0;
    if (p.ranges > 1) {
        ProductArgs parts = a;
        parts.through = 0;
        parts.y = workspace;
        parts.ldy = round_up(a.d_out, 4);
        a.part = parts.part = a.rows * parts.ldy;
        int rc = ZIPML_EINVAL;
        switch (p.shape) {
#define TILE(n, ...) case n: { typedef ProductShape<int, __VA_ARGS__> S; rc = launch_tiles<int, S>(s, parts, k_row8_product<int, S, false>); break; }
            ZIPML_PRODUCT_TILE(TILE)
#undef TILE
        }
        if (rc) return rc;
        const int64_t blocks = (a.rows * (parts.ldy / 4) + 255) / 256;
        hipLaunchKernelGGL(k_row8_product_join<T>, dim3((uint32_t)blocks), dim3(256), 0, s, a, (const int *)workspace, parts.ldy, p.ranges);
        return hip_check(hipGetLastError());
    }
    switch (p.shape) {
#define SPLIT(n, o, t, waves) case n: { typedef SplitShape<o, t, waves> S; return launch_tiles<T, S>(s, a, k_row8_product_split<T, S>); }
#define TILE(n, ...) case n: { typedef ProductShape<T, __VA_ARGS__> S; return launch_tiles<T, S>(s, a, a.through ? k_row8_product<T, S, true> : k_row8_product<T, S, false>); }
        ZIPML_PRODUCT_SPLIT(SPLIT)
        ZIPML_PRODUCT_TILE(TILE)
#undef SPLIT
#undef TILE
    }
    return ZIPML_EINVAL;
}

}  // namespace zipml

using namespace zipml;

static bool product_sizes_ok(int64_t rows, int64_t d_out, int64_t d_in)
{
    return rows > 0 && d_out > 0 && d_in > 0 && rows <= (1ll << 31) && d_out <= (1 << 24) && d_in <= (1ll << 40) && rows <= (1ll << 40) / d_out;
}
constexpr int64_t kProductMaxIn = 131071;      // 128 * 128 * d_in < 2^31

// (y's rows begin at lines of 128 bytes where its first one does)
static bool past_caches(int64_t rows, int64_t d_out, int dtype, int64_t ldy)
{
    const int64_t size = (int64_t)dtype_bytes(dtype);
    return rows * d_out * size > kThroughLeast && ldy * size % 128 == 0;
}

constexpr size_t kProductRoom = 256;           // the least workspace
static size_t product_workspace(const ProductPlan &p) { return p.workspace < kProductRoom ? kProductRoom : p.workspace; }

extern "C" size_t zipml_row8_product_workspace_bytes(int64_t rows, int64_t d_out, int64_t d_in)
{
    if (!product_sizes_ok(rows, d_out, d_in) || d_in > kProductMaxIn) return 0;
    return product_workspace(product_plan(rows, d_out, d_in, SIZE_MAX));
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
    if (!workspace_dev || workspace_bytes < kProductRoom) return ZIPML_EWORKSPACE;
    const ProductPlan p = product_plan(rows, d_out, d_in, workspace_bytes);
    if (!aligned16(x_dev) || !aligned16(w_dev) || !aligned16(y_dev) || !aligned16(workspace_dev) || !aligned4(x_scales_dev) ||
        !aligned4(w_scales_dev) || !aligned4(bias_dev))
        return ZIPML_EALIGN;
    const int through = past_caches(rows, d_out, dtype, ldy) && reinterpret_cast<uintptr_t>(y_dev) % 128 == 0;
    ProductArgs a{(const uint8_t *)x_dev, (const uint8_t *)w_dev, x_scales_dev, w_scales_dev, bias_dev, y_dev, ldx, ldw, ldy, rows,
                  (int)d_out, (int)round_up(d_in, kRow8Unit), 0, 0, 0, 0,
                  through, 0};
    hipStream_t s = entry_stream(stream);
    return dtype == ZIPML_F32 ? launch_product<float>(s, a, p, workspace_dev) : launch_product<__bf16>(s, a, p, workspace_dev);
}

extern "C" int zipml_debug_product_plan(int64_t rows, int64_t d_out, int64_t d_in, int dtype, int64_t ldy, size_t workspace_bytes,
                                        zipml_product_plan *plan_host)
{
    if (!plan_host || !valid_dtype(dtype) || !product_sizes_ok(rows, d_out, d_in) || ldy < d_out || ldy > (1ll << 60) / rows) return ZIPML_EINVAL;
    if (d_in > kProductMaxIn) return ZIPML_ERANGE;
    if (workspace_bytes < kProductRoom) return ZIPML_EWORKSPACE;
    const ProductPlan p = product_plan(rows, d_out, d_in, workspace_bytes);
    switch (p.shape) {
#define SPLIT(n, o, t, w) case n: { typedef SplitShape<o, t, w> S; *plan_host = zipml_product_plan{o, t, w, 1, 0, product_groups<S>(rows, d_out, 1)}; break; }
#define TILE(n, o, t, wo, wt)                                                                                                   \
    case n: {                                                                                                                   \
        typedef ProductShape<float, o, t, wo, wt> S;                                                                            \
        *plan_host = zipml_product_plan{o, t, wo * wt, p.ranges, p.ranges == 1 && past_caches(rows, d_out, dtype, ldy),         \
                                        product_groups<S>(rows, d_out, p.ranges)};                                              \
        break;                                                                                                                  \
    }
        ZIPML_PRODUCT_SPLIT(SPLIT)
        ZIPML_PRODUCT_TILE(TILE)
#undef SPLIT
#undef TILE
    }
    return ZIPML_OK;
}
