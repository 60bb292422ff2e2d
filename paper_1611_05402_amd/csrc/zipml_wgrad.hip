// Weight gradient of a linear layer from its stored input: dW[o][i] = sum_t dY[t][o] Q(X)[t][i].
//
// A product whose two operands are both contracted along their slow axis (tokens).  A workgroup owns a tile of dW and
// walks over the tokens: rows of dY and of the codes come in with wide loads, the codes are turned into bf16 on
// their way into LDS (once per workgroup; exact, a step is a power of two), both tiles lie in LDS as they lie in
// memory, [token][column], and are read through the transposing LDS read, which hands every lane four tokens of one
// column.  Which tokens a lane gets does not matter as long as both operands agree.
//
// What bounds it: at 16,384 tokens, 4,096 x 4,096, the power that the matrix cores draw at this rate (458 us, 1,200 TFLOP/s in a long
// run, 457 to 476; 465 to 550 in runs of a few calls, with the clock; the matrix instructions fill 63 % of the cycles; a library product of the same form, both operands
// transposed, 1,083 TFLOP/s).  Small dW: LDS reads and the steps between barriers (65,536 tokens, 512 x 256: 30 us and 5 for
// the joining of 32 ranges; the bytes alone would be 17).  fp32 dY at the first of these sizes: 1.29 to 1.34 ms, the same rate of matrix
// instructions.  Adding to dW: 514 us at the first size, 13.9 in place of 10.2 at 1,000 tokens, 1,001 x 520 (the values of dW are read
// one by one behind the last product), nothing where ranges are joined.
//
// bf16 dY: the products are exact and the sums fp32.  fp32 dY is split into three bf16 terms of 8 bits each and takes three matrix
// instructions in place of one.  Together the terms are the value exactly from 2^-110 on; below that its bits under 2^-133, where bf16
// ends, are left out.
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

// MT x NT is the tile of dW, BK the tokens of one round; WM x WN waves share the tile.  TEAMS such sets of waves take the
// rounds by turns, each with its own LDS, and add up their sums at the end.
template <typename T, int MT_, int NT_, int BK_, int WM_, int WN_, int TEAMS_ = 1>
struct WgradShape {
    static constexpr int MT = MT_, NT = NT_, BK = BK_, WM = WM_, WN = WN_, TEAMS = TEAMS_;
    static constexpr int kThreads = 64 * WM * WN;                 // of a team
    static constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;        // bf16 terms of a dY value
    // LDS rows of 64 or 192 bytes more than a multiple of 256: the four rows that 16 lanes of a transposing read touch, and
    // the 64 bytes that the neighbouring 16 lanes add to each, then fall on all banks once.
    static constexpr int kRowA = MT * 2 + 64, kRowB = NT * 2 + 64;
    static constexpr int kBytesA = BK * kRowA, kBytesB = BK * kRowB;
    static constexpr int kStage = kPlanes * kBytesA + kBytesB;
    static constexpr int kLoadsA = BK * MT / 8 / kThreads;        // eight dY values each
    static constexpr int kLoadsB = BK * NT / 8 / kThreads;        // eight codes each
    static constexpr int kSteps = BK / 16 * kPlanes;              // steps of a product: sixteen tokens, one term
    // Whether a step's reads, stores and products stay in this order; otherwise the compiler mixes them.  Measured: in order 4 to 10 %
    // faster with fp32 dY and on tiles of 64, 4 to 8 % slower on the others.
    static constexpr bool kInOrder = kPlanes == 3 || MT == 64;
    static constexpr int TM = MT / WM / 32, TN = NT / WN / 32;    // 32 x 32 tiles of a wave
    static_assert(kLoadsA * 8 * kThreads == BK * MT && kLoadsB * 8 * kThreads == BK * NT, "whole loads");
    static_assert(MT % 64 == 0 && NT % 64 == 0, "LDS rows");
    static constexpr int kLds = 2 * kStage * TEAMS;
    static_assert(kLds <= 160 * 1024 && (TEAMS - 1) * MT * NT * 4 <= kLds, "LDS");
    static_assert(kSteps % 2 == 0 && BK / 16 % 2 == 0, "operands of the steps by turns");
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

// Rows of a tile as a buffer: what lies behind its last value reads as zeros, so that neither the last tokens of a range
// nor tiles beyond the layer's edge need a branch.  (A column beyond the edge reads the next row's values where there
// is one: they reach only sums that are not kept.)  The end is exact to a dword: of bf16 rows of an odd number of values
// the very last value reads as zero, and its product is added to the sums at the end.
struct Rows {
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ Rows(const void *base, int64_t bytes)
    {
        const int n = bytes < 0 ? 0 : bytes > 0x7FFFFFFF ? 0x7FFFFFFF : (int)bytes;
        r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, n, 0x00020000);
    }
    __device__ __forceinline__ u32x4 load16(int at) const { return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0); }
    __device__ __forceinline__ u32x2 load8(int at) const { return __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0); }
    __device__ __forceinline__ uint32_t load1(int at) const { return __builtin_amdgcn_raw_buffer_load_b8(r, at, 0, 0); }
};

// Eight dY values as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<__bf16> { u32x4 w; };
template <> struct Raw8<float> { u32x4 w, w2; };

// Four fp32 values as three bf16 terms each; the first takes the upper 8 bits of the mantissa by truncation, so that it
// never overflows, the second those of the rest, the third what is left down to 2^-133 (an infinity or a NaN has only the
// first).
__device__ __forceinline__ void split4(u32x4 v, uint32_t (&plane)[3][2])
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        uint32_t hi[2], mid[2], lo[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float x = as_f32(v[2 * k + h]);
            const uint32_t bits = v[2 * k + h];
            const bool finite = (bits & 0x7F800000u) != 0x7F800000u;
            hi[h] = x != x ? 0x7FC00000u : bits & 0xFFFF0000u;
            const float r = finite ? x - as_f32(hi[h]) : 0.0f;
            mid[h] = as_u32(r) & 0xFFFF0000u;
            lo[h] = as_u32(r - as_f32(mid[h]));
        }
        plane[0][k] = __builtin_amdgcn_perm(hi[1], hi[0], 0x07060302u);
        plane[1][k] = __builtin_amdgcn_perm(mid[1], mid[0], 0x07060302u);
        plane[2][k] = __builtin_amdgcn_perm(lo[1], lo[0], 0x07060302u);
    }
}

// Workgroups go to the eight XCDs in turn; each XCD gets a run of neighbouring ones: all tiles of a range of tokens
// before those of the next, tiles in bands four deep, so that its L2 serves rows of dY and codes to several of them.
__device__ __forceinline__ void place_of(const WgradArgs &a, int &split, int &o, int &i)
{
    const uint32_t n = gridDim.x, xcd = blockIdx.x & 7, per = n >> 3, more = n & 7;
    const uint32_t id = xcd * per + (xcd < more ? xcd : more) + (blockIdx.x >> 3), tiles = a.tiles_o * a.tiles_i;
    split = id / tiles;
    const uint32_t tile = id - split * tiles, band = tile / (4 * a.tiles_i), in = tile - band * 4 * a.tiles_i;
    const uint32_t deep = a.tiles_o - band * 4 < 4 ? a.tiles_o - band * 4 : 4;
    o = band * 4 + in % deep;
    i = in / deep;
}

// WIDE: rows of dY are read 16 bytes at a time; otherwise value by value.  LAST: the last value of dY is not among what the
// loads bring (see Rows); a kernel of its own, since the others lose 2 to 10 % with these lines in them.
template <typename T, typename S, bool WIDE, bool LAST>
__global__ __launch_bounds__(S::kThreads * S::TEAMS) void k_act_wgrad(WgradArgs a)
{
    extern __shared__ __align__(16) char lds[];
    const int team = S::TEAMS == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / S::kThreads);
    const int tid = threadIdx.x - team * S::kThreads, lane = tid & 63, wave = tid >> 6;
    int split, o0, i0;
    place_of(a, split, o0, i0);
    o0 *= S::MT;
    i0 *= S::NT;
    const int64_t t_begin = split * a.rows_split;
    const int64_t t_end = t_begin + a.rows_split < a.rows ? t_begin + a.rows_split : a.rows;
    const T *dy = (const T *)a.dy;

    struct Tile {                          // a thread's part of one round
        Raw8<T> va[S::kLoadsA];
        u32x2 vb[S::kLoadsB];
        uint32_t step[S::kLoadsB];
    };

    // The loads and the stores of a tile are dealt over the steps of a round but the last.
    constexpr int kDeals = S::kSteps - 1;
    auto load = [&](Tile &tile, int64_t t0, int k) {
        const int64_t left = t_end - t0;
        // (of an odd width, the dword of a row's last value is there to its end while rows follow)
        const int64_t values = (left - 1) * a.lddy + a.d_out - o0 + (LAST && t_end < a.rows ? 1 : 0);
        const Rows ra(dy + t0 * a.lddy + o0, WIDE ? values * (int64_t)sizeof(T) : 0);
        const Rows rb(a.act + t0 * a.pitch + i0, left * a.pitch - i0);
        const Rows rs(a.act + a.steps + t0 * a.groups + (i0 >> 5), left * a.groups - (i0 >> 5));
#pragma unroll
        for (int q = 0; q < S::kLoadsA; ++q) {
            if (q * kDeals / S::kLoadsA != k) continue;
            const int c = tid + q * S::kThreads, r = c / (S::MT / 8), col = c % (S::MT / 8) * 8;
            if constexpr (WIDE) {
                const int at = (r * (int)a.lddy + col) * (int)sizeof(T);
                tile.va[q].w = ra.load16(at);
                if constexpr (sizeof(T) == 4) tile.va[q].w2 = ra.load16(at + 16);
            } else {
                const T *p = dy + (t0 + r) * a.lddy + o0 + col;
                const int n = r < left ? a.d_out - o0 - col : 0;
                T v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : (T)0.0f;
                tile.va[q] = __builtin_bit_cast(Raw8<T>, v);
            }
        }
#pragma unroll
        for (int q = 0; q < S::kLoadsB; ++q) {
            if (q * kDeals / S::kLoadsB != k) continue;
            const int c = tid + q * S::kThreads, r = c / (S::NT / 8), col = c % (S::NT / 8) * 8;
            tile.vb[q] = rb.load8(r * (int)a.pitch + col);
            tile.step[q] = rs.load1(r * (int)a.groups + (col >> 5));
        }
    };
    auto store = [&](const Tile &tile, char *stage, int k) {
#pragma unroll
        for (int q = 0; q < S::kLoadsA; ++q) {
            if (q * kDeals / S::kLoadsA != k) continue;
            const int c = tid + q * S::kThreads, r = c / (S::MT / 8), col = c % (S::MT / 8) * 8;
            char *p = stage + r * S::kRowA + col * 2;
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<u32x4 *>(p) = tile.va[q].w;
            } else {
                uint32_t x[3][2], y[3][2];
                split4(tile.va[q].w, x);
                split4(tile.va[q].w2, y);
#pragma unroll
                for (int t = 0; t < 3; ++t)
                    *reinterpret_cast<u32x4 *>(p + t * S::kBytesA) = u32x4{x[t][0], x[t][1], y[t][0], y[t][1]};
            }
        }
#pragma unroll
        for (int q = 0; q < S::kLoadsB; ++q) {
            if (q * kDeals / S::kLoadsB != k) continue;
            const int c = tid + q * S::kThreads, r = c / (S::NT / 8), col = c % (S::NT / 8) * 8;
            const float s = act_step(tile.step[q]);
            u32x4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w = tile.vb[q][j >> 1];
                const float x = (float)(int8_t)(w >> (16 * (j & 1))) * s, y = (float)(int8_t)(w >> (16 * (j & 1) + 8)) * s;
                o[j] = __builtin_amdgcn_perm(as_u32(y), as_u32(x), 0x07060302u);
            }
            *reinterpret_cast<u32x4 *>(stage + S::kPlanes * S::kBytesA + r * S::kRowB + col * 2) = o;
        }
    };

    const int wm = wave / S::WN, wn = wave % S::WN;
    // where this lane's four columns of the transposing reads start
    const int tr_row = 4 * (lane >> 5) + ((lane & 15) >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const int off_a = tr_row * S::kRowA + (wm * S::TM * 32 + tr_col) * 2;
    const int off_b = tr_row * S::kRowB + (wn * S::TN * 32 + tr_col) * 2 + S::kPlanes * S::kBytesA;
    f32x16 acc[S::TM][S::TN] = {};

    bf16x8 fa[2][S::TM], fb[2][S::TN];
    auto read = [&](const char *stage, int s) {
        const int k = s / S::kPlanes, p = s % S::kPlanes;
#pragma unroll
        for (int m = 0; m < S::TM; ++m)
            fa[s & 1][m] = fragment(stage + off_a + p * S::kBytesA + k * 16 * S::kRowA + m * 64, S::kRowA);
        if (p == 0)
#pragma unroll
            for (int n = 0; n < S::TN; ++n) fb[k & 1][n] = fragment(stage + off_b + k * 16 * S::kRowB + n * 64, S::kRowB);
    };

    // While the tile of these tokens is multiplied, the next one goes from registers to LDS, and each register is loaded
    // anew for the one after it as soon as it is free.  The operands of a step are read during the step before; the
    // barrier stands before a round's last step, whose own are in registers by then.  The steps are kept apart, since the
    // compiler otherwise moves all loads to a round's end, where their latency shows (555 us in place of 460 for 16,384
    // tokens, 4,096 x 4,096, in the same arrangement).
    char *here = lds + team * 2 * S::kStage, *next = here + S::kStage;
    const int64_t t_first = t_begin + team * S::BK;
    constexpr int kTurn = S::TEAMS * S::BK;
    Tile tile;
    if constexpr (S::MT < 256) {           // both rounds asked for at once: the memory's latency once, not twice
        Tile first;
#pragma unroll
        for (int k = 0; k < kDeals; ++k) load(first, t_first, k);
#pragma unroll
        for (int k = 0; k < kDeals; ++k) load(tile, t_first + kTurn, k);
#pragma unroll
        for (int k = 0; k < kDeals; ++k) store(first, here, k);
    } else {                               // (no registers for two; 1 % on the whole kernel)
#pragma unroll
        for (int k = 0; k < kDeals; ++k) load(tile, t_first, k);
#pragma unroll
        for (int k = 0; k < kDeals; ++k) {
            store(tile, here, k);
            load(tile, t_first + kTurn, k);
        }
    }
    lds_barrier();
    read(here, 0);
    for (int64_t t0 = t_begin; t0 < t_end; t0 += kTurn) {
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) {
            if (s < kDeals) {
                read(here, s + 1);
                if (S::kInOrder) __builtin_amdgcn_sched_barrier(0);
                store(tile, next, s);
                load(tile, t0 + team * S::BK + 2 * kTurn, s);
            } else {
                lds_barrier();
                read(next, 0);
            }
            if (S::kInOrder) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int m = 0; m < S::TM; ++m)
#pragma unroll
                for (int n = 0; n < S::TN; ++n)
                    acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[s & 1][m], fb[s / S::kPlanes & 1][n], acc[m][n], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        char *const t = here;
        here = next;
        next = t;
    }

    if constexpr (S::TEAMS > 1) {
        lds_barrier();
        f32x16 *const sums = reinterpret_cast<f32x16 *>(lds);
        const auto slot = [&](int other, int m, int n) { return (((other - 1) * S::TM + m) * S::TN + n) * S::kThreads + tid; };
        if (team > 0)
#pragma unroll
            for (int m = 0; m < S::TM; ++m)
#pragma unroll
                for (int n = 0; n < S::TN; ++n) sums[slot(team, m, n)] = acc[m][n];
        lds_barrier();
        if (team > 0) return;
#pragma unroll
        for (int other = 1; other < S::TEAMS; ++other)
#pragma unroll
            for (int m = 0; m < S::TM; ++m)
#pragma unroll
                for (int n = 0; n < S::TN; ++n) acc[m][n] += sums[slot(other, m, n)];
    }
    const bool last = LAST && t_end == a.rows && o0 + S::MT >= a.d_out;
    const float last_dy = last ? (float)dy[(a.rows - 1) * a.lddy + a.d_out - 1] : 0.0f;
    float *out = a.out + split * a.out_split;
#pragma unroll
    for (int m = 0; m < S::TM; ++m)
#pragma unroll
        for (int n = 0; n < S::TN; ++n) {
            const int i = i0 + (wn * S::TN + n) * 32 + (lane & 31);
            if (i >= a.d_in) continue;
            float last_x = 0.0f;
            if (last) {
                const int64_t t = a.rows - 1;
                last_x = (float)(int8_t)a.act[t * a.pitch + i] * act_step(a.act[a.steps + t * a.groups + (i >> 5)]);
            }
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int o = o0 + (wm * S::TM + m) * 32 + 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3);
                if (o >= a.d_out) continue;
                if (last && o == a.d_out - 1) acc[m][n][q] = __builtin_fmaf(last_dy, last_x, acc[m][n][q]);
                float *p = out + o * a.ldo + i;
                *p = a.add ? *p + acc[m][n][q] : acc[m][n][q];
            }
        }
}

// Sum of the ranges' partial sums, in an order of their number alone: each of a workgroup's four waves takes a quarter of the
// ranges, a lane four neighbouring elements, the partial sums' rows being multiples of 64.
__global__ __launch_bounds__(256) void k_wgrad_sum(const float *__restrict__ part, int splits, int64_t out_split, int d_out,
                                                   int d_in, int64_t ld_part, float *__restrict__ dw, int64_t lddw, int add)
{
    __shared__ f32x4 quarter[3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t units = (d_in + 3) / 4, u = blockIdx.x * 64u + lane, o = u / units, i = (u - o * units) * 4;
    const bool there = o < (uint32_t)d_out;
    const float *p = part + (there ? o * ld_part + i : 0);
    f32x4 sum = {};
    const int end = splits * (wave + 1) / 4;
#pragma unroll 8
    for (int s = splits * wave / 4; s < end; ++s) sum += *reinterpret_cast<const f32x4 *>(p + s * out_split);
    if (wave > 0) quarter[wave - 1][lane] = sum;
    __syncthreads();
    if (wave > 0 || !there) return;
#pragma unroll
    for (int q = 0; q < 3; ++q) sum += quarter[q][lane];
    float *w = dw + o * lddw + i;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if ((int)i + k < d_in) w[k] = add ? w[k] + sum[k] : sum[k];
}

// The shapes.  256 x 256: per value of an operand the most products, one workgroup a compute unit; the smaller ones fill
// the machine where dW is small, two or more workgroups to a compute unit; two teams on a tile where there are not that many.
template <typename T> struct Shapes {
    static constexpr int BK = sizeof(T) == 4 ? 32 : 64;
    // 2 x 4 waves or 4 x 2: the three terms of fp32 dY make its side the dearer one to read from LDS (1 to 2 % either way)
    static constexpr int WM = sizeof(T) == 4 ? 4 : 2, WN = 8 / WM;
    typedef WgradShape<T, 256, 256, BK, WM, WN> Large;
    typedef WgradShape<T, 128, 128, BK, WM, WN> Middle;
    typedef WgradShape<T, 64, 64, BK, 2, 2> Small;
    typedef WgradShape<T, 64, 64, BK, 2, 2, 2> Teams;
};

// Which shape, and in how many ranges the tokens are taken (whose partial sums a second launch joins): the least of
//   start + turns of a range * (one workgroup on a compute unit: lone, k of them: k * shared)
//         + (ranges > 1: a launch, partial sums written and read),
// a turn being 64 tokens of bf16 or 32 of fp32 dY, twice that with two teams.  The constants (us) are those that come nearest to 1,978
// times measured over 55 sizes, both types, all shapes and numbers of ranges that are powers of two, the only ones tried here; of these
// the choice is 1.4 % (bf16) and 0.3 % (fp32) slower than the fastest on average, 15 % at most.  The operands of those runs held one
// value throughout, at which the matrix cores draw less power and clock higher: on random data large products take a third longer
// than the sum says (16,384 tokens, 4,096 x 4,096: 458 us, 352 by the sum).  Without teams it was 4.4 and 3.8 %, 34 % at most: 1,000 tokens, 1,001 x 520 12.8 in
// place of 9.6 us with bf16 and 19.9 in place of 16.7 with fp32; 4,096 tokens, 1,024 x 1,024 28 in place of 22.  A team alone
// is faster up to some hundred tokens (128 tokens, 512 x 512: 4.8 us against 5.2).
struct WgradPlan {
    int tile, teams, splits, tiles_o, tiles_i;
    int64_t rows_split;
    size_t workspace() const { return splits > 1 ? (size_t)splits * tiles_o * tiles_i * tile * tile * 4 : 0; }
};
static WgradPlan wgrad_plan(int64_t rows, int64_t d_out, int64_t d_in, int dtype)
{
    struct { int tile, teams; double start, lone, shared; } const shapes[2][4] = {
        {{256, 1, 6.2, 1.35, 1.35}, {128, 1, 4.5, 0.69, 0.54}, {64, 1, 4.1, 0.44, 0.30}, {64, 2, 4.7, 0.61, 0.61}},
        {{256, 1, 5.2, 2.5, 2.5}, {128, 1, 3.5, 1.03, 0.84}, {64, 1, 3.9, 0.57, 0.37}, {64, 2, 4.8, 0.74, 0.74}}};
    const int64_t round = dtype == ZIPML_F32 ? 32 : 64;
    WgradPlan best{};
    double least = 0;
    for (const auto &c : shapes[dtype == ZIPML_F32]) {
        const int64_t to = (d_out + c.tile - 1) / c.tile, ti = (d_in + c.tile - 1) / c.tile, turn = round * c.teams;
        // (ranges only where dW is at most 2^16 tiles, so that the partial sums can be counted in 32 bits)
        for (int64_t s = 1; s <= 256 && (s == 1 || ((s - 1) * 128 < rows && to * ti <= 1 << 16)); s *= 2) {
            const int64_t rows_split = round_up((rows + s - 1) / s, 64), splits = (rows + rows_split - 1) / rows_split;
            const double k = (double)((to * ti * splits + 255) / 256), turns = (double)((rows_split + turn - 1) / turn);
            const double us = c.start + turns * (k > 1 ? k * c.shared : c.lone) +
                              (splits > 1 ? 3.0 + (double)splits * to * ti * c.tile * c.tile * 8.0 / 6e6 : 0.0);
            if (best.tile == 0 || us < least) {
                least = us;
                best = WgradPlan{c.tile, c.teams, (int)splits, (int)to, (int)ti, rows_split};
            }
        }
    }
    return best;
}

template <typename T, typename S>
static int launch_wgrad(hipStream_t s, WgradArgs a, int splits)
{
    // 16 bytes at a time, at any alignment, where the offsets of a round fit 31 bits
    const bool wide = a.lddy * (int64_t)sizeof(T) < (1 << 24);
    const bool last = wide && sizeof(T) == 2 && a.d_out % 2 == 1;
    auto k = !wide ? k_act_wgrad<T, S, false, false> : !last ? k_act_wgrad<T, S, true, false> : k_act_wgrad<T, S, true, sizeof(T) == 2>;
    static std::atomic<uint64_t> done[3];
    if (allow_lds((const void *)k, S::kLds, done[wide + last])) return ZIPML_ELAUNCH;
    hipLaunchKernelGGL(k, dim3(a.tiles_o * a.tiles_i * splits), dim3(S::kThreads * S::TEAMS), S::kLds, s, a);
    return hip_check(hipGetLastError());
}

template <typename T>
static int launch_tile(hipStream_t s, const WgradArgs &a, const WgradPlan &p)
{
    if (p.tile == 256) return launch_wgrad<T, typename Shapes<T>::Large>(s, a, p.splits);
    if (p.tile == 128) return launch_wgrad<T, typename Shapes<T>::Middle>(s, a, p.splits);
    if (p.teams == 2) return launch_wgrad<T, typename Shapes<T>::Teams>(s, a, p.splits);
    return launch_wgrad<T, typename Shapes<T>::Small>(s, a, p.splits);
}

}  // namespace zipml

using namespace zipml;

static bool wgrad_sizes_ok(int64_t rows, int64_t d_out, int64_t d_in)
{
    return act_sizes_ok(rows, d_in) && d_out > 0 && d_out <= (1 << 24) && d_in <= (1 << 24) &&
           d_out <= (1ll << 37) / d_in;
}

extern "C" size_t zipml_act_wgrad_workspace_bytes(int64_t rows, int64_t d_out, int64_t d_in, int dtype)
{
    if (!wgrad_sizes_ok(rows, d_out, d_in) || !valid_dtype(dtype)) return 0;
    const size_t b = wgrad_plan(rows, d_out, d_in, dtype).workspace();
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
    const WgradPlan p = wgrad_plan(rows, d_out, d_in, dtype);
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
    const int rc = dtype == ZIPML_F32 ? launch_tile<float>(s, a, p) : launch_tile<__bf16>(s, a, p);
    if (rc || p.splits == 1) return rc;
    const int64_t blocks = ((d_in + 3) / 4 * d_out + 63) / 64;
    hipLaunchKernelGGL(k_wgrad_sum, dim3((uint32_t)blocks), dim3(256), 0, s, a.out, p.splits, a.out_split, (int)d_out,
                       (int)d_in, a.ldo, dw_dev, lddw, add);
    return hip_check(hipGetLastError());
}
