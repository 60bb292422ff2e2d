// Global norm of many gradients, and the gradients scaled down to it: zipml_clip.
//
//   norm = sqrt(sum g^2) over all tensors, factor = norm <= max_norm ? 1 : max_norm / norm, out = round(factor g)
//
// Two passes over the gradients, each one launch for kClipTensors of them: the first leaves one sum a workgroup, the second adds
// these up (every workgroup for itself, in the same order) and scales.  Squares are summed in 64 bits, so that no gradient that
// fp32 holds overflows and the norm does not depend on the order.  The second pass goes from the last chunk to the first: what the
// first pass has read last is still in the caches.
#include "zipml_act.h"

namespace zipml {

constexpr int kClipTensors = 96;          // of a launch: what its arguments hold
constexpr int kClipGroups = 1024;         // workgroups of a launch
constexpr int kClipUnits = 4;             // units of eight values that a thread has under way
constexpr int64_t kClipChunk = 256 * 8 * kClipUnits;

struct ClipTensor {
    const void *grad;
    void *out;
    int64_t count;
    uint32_t first;                       // chunks of the tensors before it
    uint8_t grad_bf16, out_bf16;
};
struct ClipArgs {
    ClipTensor t[kClipTensors];
    int n;
    uint32_t chunks;
};
static_assert(sizeof(ClipArgs) + 64 <= 4096, "kernel arguments");

// The tensor that a chunk belongs to.
__device__ __forceinline__ int clip_tensor(const ClipArgs &a, uint32_t chunk)
{
    int lo = 0, hi = a.n;                 // t[lo].first <= chunk < t[hi].first
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.t[mid].first <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename T>
__device__ __forceinline__ void clip_load(const void *p, int64_t at, int64_t count, float (&v)[kClipUnits][8])
{
    const T *x = (const T *)p + at;
    if (at - threadIdx.x * 8 + kClipChunk <= count) {
#pragma unroll
        for (int q = 0; q < kClipUnits; ++q) load8(x + q * 2048, 8, v[q]);
    } else {
#pragma unroll
        for (int q = 0; q < kClipUnits; ++q) load8(x + q * 2048, count - at - q * 2048, v[q]);
    }
}
__device__ __forceinline__ void clip_values(const ClipTensor &t, int64_t at, float (&v)[kClipUnits][8])
{
    if (t.grad_bf16) clip_load<__bf16>(t.grad, at, t.count, v);
    else clip_load<float>(t.grad, at, t.count, v);
}

__global__ __launch_bounds__(256) void k_clip_norm(ClipArgs a, double *part)
{
    __shared__ double scratch[8];
    double sum = 0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipTensor &t = a.t[clip_tensor(a, c)];
        float v[kClipUnits][8];
        clip_values(t, (int64_t)(c - t.first) * kClipChunk + threadIdx.x * 8, v);
#pragma unroll
        for (int q = 0; q < kClipUnits; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum = __builtin_fma((double)v[q][k], (double)v[q][k], sum);
    }
    sum = block_sum(sum, scratch);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void k_clip_scale(ClipArgs a, const double *part, int parts, float max_norm, float *norm_out)
{
    __shared__ double scratch[8];
    double sum = 0;
    for (int p = threadIdx.x; p < parts; p += 256) sum += part[p];
    const double norm = __builtin_sqrt(block_sum(sum, scratch));
    const float factor = norm <= (double)max_norm ? 1.0f : (float)((double)max_norm / norm);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) {
        norm_out[0] = (float)norm;
        norm_out[1] = factor;
    }
    for (uint32_t i = blockIdx.x; i < a.chunks; i += gridDim.x) {
        const uint32_t c = a.chunks - 1 - i;
        const ClipTensor &t = a.t[clip_tensor(a, c)];
        // (a tensor in place needs no second pass where nothing is scaled)
        if (!t.out || (t.out == t.grad && factor == 1.0f)) continue;
        const int64_t at = (int64_t)(c - t.first) * kClipChunk + threadIdx.x * 8;
        float v[kClipUnits][8];
        clip_values(t, at, v);
#pragma unroll
        for (int q = 0; q < kClipUnits; ++q) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[q][k] *= factor;
            const int64_t to = at + q * 2048, left = t.count - to;
            if (t.out_bf16) store8((__bf16 *)t.out + to, left, v[q]);
            else store8((float *)t.out + to, left, v[q]);
        }
    }
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
    return valid_dtype(t.grad_dtype) && valid_dtype(t.out_dtype) && t.count >= 0 && t.count <= (1ll << 34) &&
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
    hipStream_t s = entry_stream(stream);
    double *part = (double *)workspace_dev;
    int parts = 0;
    for (int pass = 0; pass < 2; ++pass) {
        for (int64_t i0 = 0; i0 < n_tensors; i0 += kClipTensors) {
            ClipArgs a;
            a.n = (int)(n_tensors - i0 < kClipTensors ? n_tensors - i0 : kClipTensors);
            a.chunks = 0;
            bool writes = i0 == 0;         // (the first launch of the second pass hands the norm on)
            for (int k = 0; k < a.n; ++k) {
                const zipml_clip_tensor &t = tensors_host[i0 + k];
                a.t[k] = ClipTensor{t.grad_dev, t.out_dev, t.count, a.chunks, t.grad_dtype == ZIPML_BF16, t.out_dtype == ZIPML_BF16};
                a.chunks += (uint32_t)((t.count + kClipChunk - 1) / kClipChunk);
                writes |= t.out_dev != nullptr;
            }
            const int groups = a.chunks < 1 ? 1 : a.chunks < (uint32_t)kClipGroups ? (int)a.chunks : kClipGroups;
            if (pass == 0) {
                hipLaunchKernelGGL(k_clip_norm, dim3(groups), dim3(256), 0, s, a, part + parts);
                parts += groups;
            } else if (writes) {
                hipLaunchKernelGGL(k_clip_scale, dim3(groups), dim3(256), 0, s, a, part, parts, max_norm, i0 == 0 ? norm_dev : nullptr);
            }
            if (const int rc = hip_check(hipGetLastError())) return rc;
        }
    }
    return ZIPML_OK;
}
