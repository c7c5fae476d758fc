// Global 2-norm of a list of gradient tensors, and clipping by it:
//   norm = sqrt(sum over all tensors of g^2);   dst = g * (norm > max_norm and finite ? max_norm / norm : 1)
// The squares are added in 64 bits: a square of an fp32 number fits the range of a double, so neither large nor tiny
// gradients leave it, and the order of the sums is fixed.
#include <algorithm>

#include "common.cuh"

namespace sgcn {
namespace {

constexpr int kClipThreads = 256;
constexpr int kClipBlocks = 148 * 4;
constexpr int64_t kClipChunk = 4096;   // elements per work item

struct ClipEntry {
    const void* src;
    void* dst;
    int64_t elems;
    int64_t first;   // index of the tensor's first chunk
    int bf16;
};
struct ClipTable {
    int count;
    int64_t chunks;
    ClipEntry e[SLICEGCN_MAX_TENSORS];
};

// the tensor a chunk belongs to
__device__ __forceinline__ int find_entry(const ClipTable& t, int64_t chunk) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.e[mid].first <= chunk)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

__global__ void __launch_bounds__(kClipThreads) clip_norm_kernel(const __grid_constant__ ClipTable t, double* partial) {
    __shared__ double sm[kClipThreads];
    double s = 0.0;
    for (int64_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int k = find_entry(t, c);
        const int64_t i0 = (c - t.e[k].first) * kClipChunk, i1 = min(t.e[k].elems, i0 + kClipChunk);
        for (int64_t i = i0 + threadIdx.x; i < i1; i += kClipThreads) {
            const double v = t.e[k].bf16 ? (double)__bfloat162float(static_cast<const __nv_bfloat16*>(t.e[k].src)[i])
                                         : (double)static_cast<const float*>(t.e[k].src)[i];
            s += v * v;
        }
    }
    sm[threadIdx.x] = s;
    __syncthreads();
    for (int o = kClipThreads / 2; o > 0; o >>= 1) {
        if (threadIdx.x < o) sm[threadIdx.x] += sm[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) partial[blockIdx.x] = sm[0];
}

__global__ void __launch_bounds__(kClipThreads) clip_scale_kernel(const __grid_constant__ ClipTable t, const double* partial, int n_partial,
                                                                  double max_norm, float* norm_out) {
    __shared__ double sm[kClipThreads];
    double s = 0.0;
    for (int i = threadIdx.x; i < n_partial; i += kClipThreads) s += partial[i];
    sm[threadIdx.x] = s;
    __syncthreads();
    for (int o = kClipThreads / 2; o > 0; o >>= 1) {
        if (threadIdx.x < o) sm[threadIdx.x] += sm[threadIdx.x + o];
        __syncthreads();
    }
    const double norm = sqrt(sm[0]);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const float f = (norm > max_norm && isfinite(norm)) ? (float)(max_norm / norm) : 1.f;
    for (int64_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int k = find_entry(t, c);
        if (!t.e[k].dst) continue;
        const int64_t i0 = (c - t.e[k].first) * kClipChunk, i1 = min(t.e[k].elems, i0 + kClipChunk);
        for (int64_t i = i0 + threadIdx.x; i < i1; i += kClipThreads) {
            if (t.e[k].bf16)
                static_cast<__nv_bfloat16*>(t.e[k].dst)[i] =
                    __float2bfloat16_rn(__bfloat162float(static_cast<const __nv_bfloat16*>(t.e[k].src)[i]) * f);
            else
                static_cast<float*>(t.e[k].dst)[i] = static_cast<const float*>(t.e[k].src)[i] * f;
        }
    }
}

}  // namespace
}  // namespace sgcn

using namespace sgcn;

extern "C" {

slicegcn_status_t slicegcn_clip_workspace_bytes(int64_t* bytes) {
    if (!bytes) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_workspace_bytes: NULL argument");
    *bytes = kClipBlocks * (int64_t)sizeof(double);
    return SLICEGCN_OK;
}

slicegcn_status_t slicegcn_clip_grads(const slicegcn_tensor_list* list, double max_norm, float* norm_out, void* workspace,
                                      int64_t workspace_bytes, void* stream) {
    if (!list || list->count < 0) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: bad tensor list");
    if (list->count > SLICEGCN_MAX_TENSORS)
        SGCN_FAIL(SLICEGCN_ERR_UNSUPPORTED, "clip_grads: %d tensors, at most %d", list->count, SLICEGCN_MAX_TENSORS);
    if (list->count > 0 && (!list->src || !list->elems)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: bad tensor list");
    if (!(max_norm > 0)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: max_norm must be positive");
    if (!list->dst && !norm_out) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: neither clipped gradients nor the norm are asked for");
    ClipTable t;
    t.count = 0;
    t.chunks = 0;
    for (int i = 0; i < list->count; ++i) {
        ClipEntry& e = t.e[t.count];
        const int dt = list->dtypes ? list->dtypes[i] : SLICEGCN_F32;
        if (dt != SLICEGCN_F32 && dt != SLICEGCN_BF16) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: bad dtype of tensor %d", i);
        const int esz = dt == SLICEGCN_BF16 ? 2 : 4;
        e.src = list->src[i];
        e.dst = list->dst ? list->dst[i] : nullptr;
        e.elems = list->elems[i];
        if (e.elems < 0) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: tensor %d has a negative size", i);
        if (e.elems == 0) continue;
        if (!e.src || (list->dst && !e.dst)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: tensor %d is NULL", i);
        if ((uintptr_t)e.src % esz || (uintptr_t)e.dst % esz)
            SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: tensor %d is not aligned to its element type", i);
        e.bf16 = dt == SLICEGCN_BF16;
        e.first = t.chunks;
        t.chunks += (e.elems + kClipChunk - 1) / kClipChunk;
        ++t.count;
    }
    if ((uintptr_t)norm_out % 4 || (uintptr_t)workspace % 16)
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: norm_out or the workspace (16 bytes) is not aligned");
    if (!workspace || workspace_bytes < kClipBlocks * (int64_t)sizeof(double))
        SGCN_FAIL(SLICEGCN_ERR_ALLOC, "clip_grads: workspace too small (%lld < %lld bytes)", (long long)workspace_bytes,
                  (long long)(kClipBlocks * sizeof(double)));
    cudaStream_t st = (cudaStream_t)stream;
    double* partial = static_cast<double*>(workspace);
    const int blocks = (int)std::min<int64_t>(std::max<int64_t>(t.chunks, 1), kClipBlocks);
    clip_norm_kernel<<<blocks, kClipThreads, 0, st>>>(t, partial);
    SGCN_LAUNCH_CHECK();
    clip_scale_kernel<<<blocks, kClipThreads, 0, st>>>(t, partial, blocks, max_norm, norm_out);
    SGCN_LAUNCH_CHECK();
    count_launch(2);
    return SLICEGCN_OK;
}

}  // extern "C"
