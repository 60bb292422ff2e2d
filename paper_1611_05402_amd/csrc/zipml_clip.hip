// Global norm of many gradients, and the gradients scaled down to it: zipml_clip.
//
//   norm = sqrt(sum g^2) over all tensors, factor = norm <= max_norm ? 1 : max_norm / norm, out = round(factor g)
//
// Two passes over the gradients, each one launch for kClipTensors of them: the first leaves one sum a workgroup, the second adds
// these up (every workgroup for itself, in the same order, unless they are many) and scales.  Squares are summed in 64 bits, so that no gradient that
// fp32 holds overflows and the order, one of the sizes alone, hardly shows in the fp32 norm.  The second pass goes from the last chunk to the first: what the
// first pass has read last is still in the caches, and results are written past them.  302 million fp32 values into a bf16 bucket: 193 us
// for 1.2 GB, then 327 for 1.8 GB (6.2 and 5.5 TB/s, part of it out of the caches); in one pass over the gradients, which no cache holds,
// it cannot be done.  Few values: 1.6 million in 3.6 and 5.4 us, of the second launch 4.2 until each workgroup has added up the first's 765 sums.
#include "zipml_row8.h"

namespace zipml {

constexpr int kClipTensors = 160;         // of a launch: what its arguments hold
constexpr int kClipGroups = 1024;         // workgroups of a launch
// Units of eight values that a thread has under way: four, or one where chunks of four would leave compute units idle (1.6 million
// values: 8.6 us in both launches, 9.6 with four and with the tensors searched for in the arguments).
constexpr int kClipMany = 4, kClipFew = 1;
// More sums than these are joined once, by a launch of its own, not by each workgroup (tensors of 20,000 values: 320 of them, 2,048 sums, 24 us
// and 26 with such a launch, 480 37 and 33, 4,000 592 and 298).
constexpr int kClipParts = 2048;
constexpr int64_t clip_chunk(int units) { return 256 * 8 * units; }

constexpr int64_t kClipMost = 1ll << 33;  // values of a tensor: 160 of them are fewer than 2^28 chunks

struct ClipTensor {
    const void *grad;
    void *out;
    uint32_t count;                       // its low 32 bits
    uint32_t more;                        // chunks of the tensors before it, 28 bits; bf16 gradient; bf16 output; two more bits of the count
    __host__ __device__ uint32_t first() const { return more & 0x0FFFFFFFu; }
    __host__ __device__ bool grad_bf16() const { return more >> 28 & 1; }
    __host__ __device__ bool out_bf16() const { return more >> 29 & 1; }
    __host__ __device__ int64_t values() const { return (int64_t)(more >> 30) << 32 | count; }
};
struct ClipArgs {
    ClipTensor t[kClipTensors];
    int n;
    uint32_t chunks;
};
static_assert(sizeof(ClipArgs) + 64 <= 4096, "kernel arguments");

// The launch's tensors, in the registers of each wave: a lane keeps every 64th.  Read all at once: kernel
// arguments lie far away, and a search among them would wait for each step.
struct ClipTable {
    static constexpr int kSets = (kClipTensors + 63) / 64;
    ClipTensor own[kSets];
    int n;
    __device__ __forceinline__ explicit ClipTable(const ClipArgs &a) : n(a.n)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int k = 0; k < kSets; ++k) own[k] = a.t[lane + 64 * k < n ? lane + 64 * k : 0];
    }
    static __device__ __forceinline__ uint64_t lane_of(uint64_t v, int l)
    {
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, l), hi = __builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), l);
        return (uint64_t)hi << 32 | lo;
    }
    // The tensor that a chunk belongs to: the last of those that begin at it or before.
    __device__ __forceinline__ ClipTensor at(uint32_t chunk) const
    {
        const int lane = threadIdx.x & 63;
        int at = -1;
#pragma unroll
        for (int k = 0; k < kSets; ++k) at += __builtin_popcountll(__ballot(lane + 64 * k < n && own[k].first() <= chunk));
        // (each set's value is read from its lane before one is chosen: a choice among the registers would put them in memory)
        const int l = at & 63;
        ClipTensor r{};
#pragma unroll
        for (int k = 0; k < kSets; ++k) {
            const uint64_t grad = lane_of((uint64_t)own[k].grad, l), out = lane_of((uint64_t)own[k].out, l);
            const uint32_t count = (uint32_t)__builtin_amdgcn_readlane((int)own[k].count, l);
            const uint32_t more = (uint32_t)__builtin_amdgcn_readlane((int)own[k].more, l);
            if (at >> 6 == k) {
                r.grad = (const void *)grad;
                r.out = (void *)out;
                r.count = count;
                r.more = more;
            }
        }
        return r;
    }
};

template <typename T, int U>
__device__ __forceinline__ void clip_load(const void *p, int64_t at, int64_t count, float (&v)[U][8])
{
    const T *x = (const T *)p + at;
    if (at - threadIdx.x * 8 + clip_chunk(U) <= count) {
#pragma unroll
        for (int q = 0; q < U; ++q) load8(x + q * 2048, 8, v[q]);
    } else {
#pragma unroll
        for (int q = 0; q < U; ++q) load8(x + q * 2048, count - at - q * 2048, v[q]);
    }
}
template <int U>
__device__ __forceinline__ void clip_values(const ClipTensor &t, int64_t at, float (&v)[U][8])
{
    if (t.grad_bf16()) clip_load<__bf16>(t.grad, at, t.values(), v);
    else clip_load<float>(t.grad, at, t.values(), v);
}

template <int U>
__global__ __launch_bounds__(256) void k_clip_norm(ClipArgs a, double *part)
{
    __shared__ double scratch[4];
    const ClipTable table(a);
    double sum = 0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipTensor t = table.at(c);
        float v[U][8];
        clip_values(t, (int64_t)(c - t.first()) * clip_chunk(U) + threadIdx.x * 8, v);
#pragma unroll
        for (int q = 0; q < U; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum = __builtin_fma((double)v[q][k], (double)v[q][k], sum);
    }
    sum = team_sum<256>(sum, scratch);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

template <int U>
__global__ __launch_bounds__(256) void k_clip_scale(ClipArgs a, const double *part, int parts, float max_norm, float *norm_out)
{
    __shared__ double scratch[4];
    double sum = 0;
    for (int p = threadIdx.x; p < parts; p += 256) sum += part[p];
    // (the first chunk is on its way while the norm is formed)
    const ClipTable table(a);
    float v[U][8];
    uint32_t i = blockIdx.x;
    ClipTensor t{};
    auto fetch = [&]() {
        t = table.at(a.chunks - 1 - i);
        if (t.out) clip_values(t, (int64_t)(a.chunks - 1 - i - t.first()) * clip_chunk(U) + threadIdx.x * 8, v);
    };
    if (i < a.chunks) fetch();
    const double norm = __builtin_sqrt(team_sum<256>(sum, scratch));
    const float factor = norm <= (double)max_norm ? 1.0f : (float)((double)max_norm / norm);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) {
        norm_out[0] = (float)norm;
        norm_out[1] = factor;
    }
    while (i < a.chunks) {
        const int64_t at = (int64_t)(a.chunks - 1 - i - t.first()) * clip_chunk(U) + threadIdx.x * 8;
        // (a tensor in place stays as it is where nothing is scaled)
        if (t.out && (t.out != t.grad || factor != 1.0f))
#pragma unroll
            for (int q = 0; q < U; ++q) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[q][j] *= factor;
                const int64_t to = at + q * 2048, left = t.values() - to;
                if (t.out_bf16()) store8<true>((__bf16 *)t.out + to, left, v[q]);
                else store8<true>((float *)t.out + to, left, v[q]);
            }
        i += gridDim.x;
        if (i < a.chunks) fetch();
    }
}

// All sums into the first of them, by one workgroup.
__global__ __launch_bounds__(1024) void k_clip_join(double *part, int parts)
{
    __shared__ double scratch[16];
    double sum = 0;
#pragma unroll 8
    for (int p = threadIdx.x; p < parts; p += 1024) sum += part[p];
    sum = team_sum<1024>(sum, scratch);    // (its barrier stands between the last read and the write)
    if (threadIdx.x == 0) part[0] = sum;
}

}  // namespace zipml

using namespace zipml;

extern "C" size_t zipml_clip_workspace_bytes(int64_t n_tensors)
{
    if (n_tensors < 1 || n_tensors > (1 << 20)) return 0;
    return (size_t)((n_tensors + kClipTensors - 1) / kClipTensors) * kClipGroups * sizeof(double);
}

static bool clip_tensor_ok(const zipml_clip_tensor &t)
{
    return valid_dtype(t.grad_dtype) && valid_dtype(t.out_dtype) && t.count >= 0 && t.count <= kClipMost &&
           (!t.count || (t.grad_dev && (t.out_dev != t.grad_dev || t.out_dtype == t.grad_dtype)));
}
static bool aligned_as(const void *p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype_bytes(dtype) - 1)) == 0; }

extern "C" int zipml_clip(void *stream, const zipml_clip_tensor *tensors_host, int64_t n_tensors, float max_norm, float *norm_dev,
                          void *workspace_dev, size_t workspace_bytes)
{
    if (!tensors_host || !norm_dev || n_tensors < 1 || n_tensors > (1 << 20) || !(max_norm >= 0.0f)) return ZIPML_EINVAL;
    for (int64_t i = 0; i < n_tensors; ++i)
        if (!clip_tensor_ok(tensors_host[i])) return ZIPML_EINVAL;
    if (!workspace_dev || workspace_bytes < zipml_clip_workspace_bytes(n_tensors)) return ZIPML_EWORKSPACE;
    if (!aligned16(workspace_dev) || !aligned4(norm_dev)) return ZIPML_EALIGN;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const zipml_clip_tensor &t = tensors_host[i];
        if (!aligned_as(t.grad_dev, t.grad_dtype) || !aligned_as(t.out_dev, t.out_dtype)) return ZIPML_EALIGN;
    }
    int64_t most = 0;                      // chunks of four units of the launch with most of them
    for (int64_t i0 = 0, n = 0; i0 < n_tensors; ++i0) {
        n = (i0 % kClipTensors ? n : 0) + (tensors_host[i0].count + clip_chunk(kClipMany) - 1) / clip_chunk(kClipMany);
        most = n > most ? n : most;
    }
    const bool few = most < kClipGroups;
    const int64_t chunk = clip_chunk(few ? kClipFew : kClipMany);
    hipStream_t s = entry_stream(stream);
    double *part = (double *)workspace_dev;
    int parts = 0;
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 1 && parts > kClipParts) {
            hipLaunchKernelGGL(k_clip_join, dim3(1), dim3(1024), 0, s, part, parts);
            if (const int rc = hip_check(hipGetLastError())) return rc;
            parts = 1;
        }
        for (int64_t i0 = 0; i0 < n_tensors; i0 += kClipTensors) {
            ClipArgs a;
            a.n = (int)(n_tensors - i0 < kClipTensors ? n_tensors - i0 : kClipTensors);
            a.chunks = 0;
            bool writes = i0 == 0;         // (the first launch of the second pass hands the norm on)
            for (int k = 0; k < a.n; ++k) {
                const zipml_clip_tensor &t = tensors_host[i0 + k];
                a.t[k] = ClipTensor{t.grad_dev, t.out_dev, (uint32_t)t.count,
                                    a.chunks | (t.grad_dtype == ZIPML_BF16 ? 1u << 28 : 0u) | (t.out_dtype == ZIPML_BF16 ? 1u << 29 : 0u) |
                                        (uint32_t)(t.count >> 32) << 30};
                a.chunks += (uint32_t)((t.count + chunk - 1) / chunk);
                writes |= t.out_dev != nullptr;
            }
            const int groups = a.chunks < 1 ? 1 : a.chunks < (uint32_t)kClipGroups ? (int)a.chunks : kClipGroups;
            if (pass == 0) {
                hipLaunchKernelGGL(few ? k_clip_norm<kClipFew> : k_clip_norm<kClipMany>, dim3(groups), dim3(256), 0, s, a, part + parts);
                parts += groups;
            } else if (writes) {
                hipLaunchKernelGGL(few ? k_clip_scale<kClipFew> : k_clip_scale<kClipMany>, dim3(groups), dim3(256), 0, s, a, part, parts, max_norm, i0 == 0 ? norm_dev : nullptr);
            }
            if (const int rc = hip_check(hipGetLastError())) return rc;
        }
    }
    return ZIPML_OK;
}
