// Global 2-norm of a list of gradient tensors, and clipping by it:
//   norm = sqrt(sum over all tensors of g^2);   dst = g * (norm > max_norm and finite ? max_norm / norm : 1)
// The order of the sums is fixed.
#include <cooperative_groups.h>

#include <algorithm>

#include "common.cuh"

namespace sgcn {
namespace {

constexpr int kClipChunk = 4096;     // elements per work item: 4 per thread of a large CTA, 16 per thread of a small one
constexpr int kSMs = 148;

struct ClipEntry {
    const void* src;
    void* dst;
    int64_t elems;
    int64_t first;   // index of the tensor's first chunk
    int bf16, vec;   // vec: four elements at a time are aligned in src and dst
};
// N: room for tensors.  A short list travels as a short kernel argument, which costs less to launch (512 tensors: 20 KB).
template <int N>
struct ClipTable {
    int count;
    int64_t chunks;
    ClipEntry e[N];
};
constexpr int kShortList = 32;

struct Four {
    float v[4];
};

// four elements from i (fewer where the tensor ends; the rest zeros)
__device__ __forceinline__ Four load4(const ClipEntry& e, int64_t i) {
    Four f{{0.f, 0.f, 0.f, 0.f}};
    if (i >= e.elems) return f;
    if (e.vec && i + 4 <= e.elems) {
        if (e.bf16) {
            const uint2 t = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(e.src) + i);
            f.v[0] = __uint_as_float(t.x << 16), f.v[1] = __uint_as_float(t.x & 0xffff0000u);
            f.v[2] = __uint_as_float(t.y << 16), f.v[3] = __uint_as_float(t.y & 0xffff0000u);
        } else {
            const float4 t = *reinterpret_cast<const float4*>(static_cast<const float*>(e.src) + i);
            f.v[0] = t.x, f.v[1] = t.y, f.v[2] = t.z, f.v[3] = t.w;
        }
        return f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < e.elems)
            f.v[j] = e.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(e.src)[i + j]) : static_cast<const float*>(e.src)[i + j];
    return f;
}

__device__ __forceinline__ void store4(const ClipEntry& e, int64_t i, const Four& f, float factor) {
    if (i >= e.elems) return;
    const float a = f.v[0] * factor, b = f.v[1] * factor, c = f.v[2] * factor, d = f.v[3] * factor;
    if (e.vec && i + 4 <= e.elems) {
        if (e.bf16) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(a, b), hi = __floats2bfloat162_rn(c, d);
            uint2 t;
            t.x = *reinterpret_cast<const uint32_t*>(&lo), t.y = *reinterpret_cast<const uint32_t*>(&hi);
            __stcs(reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(e.dst) + i), t);
        } else {
            __stcs(reinterpret_cast<float4*>(static_cast<float*>(e.dst) + i), make_float4(a, b, c, d));
        }
        return;
    }
    const float o[4] = {a, b, c, d};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < e.elems) {
            if (e.bf16)
                static_cast<__nv_bfloat16*>(e.dst)[i + j] = __float2bfloat16_rn(o[j]);
            else
                static_cast<float*>(e.dst)[i + j] = o[j];
        }
}

// The squares are taken and added in 64 bits: the square of any fp32 number fits a double, so neither large nor tiny
// gradients leave its range, and this GPU's 64-bit rate is far above what HBM delivers to it.
__device__ __forceinline__ double squares(const Four& f) {
    const double a = f.v[0], b = f.v[1], c = f.v[2], d = f.v[3];
    return fma(a, a, b * b) + fma(c, c, d * d);
}

// sum over the CTA, the same order every time; every thread gets it
template <int THREADS>
__device__ __forceinline__ double cta_sum(double s, double* smem) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = s;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) t += smem[k];
    return t;
}

__device__ __forceinline__ float clip_factor(double norm, double max_norm) {
    return norm > max_norm && isfinite(norm) ? (float)(max_norm / norm) : 1.f;
}

// Small lists (up to kClusterChunks chunks): one launch of one cluster that keeps every gradient in registers between the
// sum and the scaling, so each is read once.  The eight sums meet in distributed shared memory.
constexpr int kClusterCtas = 8, kClusterThreads = 1024, kHeld = 8;
constexpr int kClusterChunks = kClusterCtas * kHeld;
__global__ void __cluster_dims__(kClusterCtas, 1, 1) __launch_bounds__(kClusterThreads)
    clip_cluster_kernel(const __grid_constant__ ClipTable<kShortList> t, double max_norm, float* norm_out) {
    namespace cg = cooperative_groups;
    __shared__ double smem[kClusterThreads / 32];
    __shared__ double sums[kClusterCtas];
    const cg::cluster_group cluster = cg::this_cluster();
    const int rank = blockIdx.x;
    Four held[kHeld];
    double s = 0.0;
    int k = 0;
#pragma unroll
    for (int q = 0; q < kHeld; ++q) {
        const int64_t c = rank + q * kClusterCtas;
        if (c < t.chunks) {
            while (k + 1 < t.count && t.e[k + 1].first <= c) ++k;
            held[q] = load4(t.e[k], (c - t.e[k].first) * kClipChunk + threadIdx.x * 4);
        }
    }
#pragma unroll
    for (int q = 0; q < kHeld; ++q)
        if (rank + q * kClusterCtas < t.chunks) s += squares(held[q]);
    s = cta_sum<kClusterThreads>(s, smem);
    if (threadIdx.x < kClusterCtas) *cluster.map_shared_rank(&sums[rank], threadIdx.x) = s;
    cluster.sync();   // hardware barrier; no CTA reads another's memory after it
    double total = 0.0;
#pragma unroll
    for (int r = 0; r < kClusterCtas; ++r) total += sums[r];
    const double norm = sqrt(total);
    if (norm_out && rank == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const float f = clip_factor(norm, max_norm);
    k = 0;
#pragma unroll
    for (int q = 0; q < kHeld; ++q) {
        const int64_t c = rank + q * kClusterCtas;
        if (c < t.chunks) {
            while (k + 1 < t.count && t.e[k + 1].first <= c) ++k;
            if (t.e[k].dst) store4(t.e[k], (c - t.e[k].first) * kClipChunk + threadIdx.x * 4, held[q], f);
        }
    }
}

// Larger lists: two launches bound by HBM.  The second one walks the chunks backwards, since what the first one read last is
// still in L2, and its launch overlaps the end of the first (it waits for the sums on the device).
constexpr int kThreads = 256, kPer = kClipChunk / kThreads / 4, kMaxCtas = 8 * kSMs;
template <int N>
__global__ void __launch_bounds__(kThreads) clip_norm_kernel(const __grid_constant__ ClipTable<N> t, double* partial) {
    __shared__ double smem[kThreads / 32];
    cudaTriggerProgrammaticLaunchCompletion();
    double s = 0.0;
    int k = 0;
    for (int64_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        while (k + 1 < t.count && t.e[k + 1].first <= c) ++k;
        const int64_t i = (c - t.e[k].first) * kClipChunk + threadIdx.x * 4;
        Four f[kPer];
#pragma unroll
        for (int q = 0; q < kPer; ++q) f[q] = load4(t.e[k], i + q * kThreads * 4);
#pragma unroll
        for (int q = 0; q < kPer; ++q) s += squares(f[q]);
    }
    s = cta_sum<kThreads>(s, smem);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

template <int N>
__global__ void __launch_bounds__(kThreads) clip_scale_kernel(const __grid_constant__ ClipTable<N> t, const double* partial, int n_partial,
                                                              double max_norm, float* norm_out) {
    __shared__ double smem[kThreads / 32];
    cudaGridDependencySynchronize();
    double s = 0.0;
    for (int i = threadIdx.x; i < n_partial; i += kThreads) s += partial[i];
    const double norm = sqrt(cta_sum<kThreads>(s, smem));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const float factor = clip_factor(norm, max_norm);
    int k = t.count - 1;
    for (int64_t c = t.chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
        while (t.e[k].first > c) --k;
        if (!t.e[k].dst || (factor == 1.f && t.e[k].dst == t.e[k].src)) continue;
        const int64_t i = (c - t.e[k].first) * kClipChunk + threadIdx.x * 4;
        Four f[kPer];
#pragma unroll
        for (int q = 0; q < kPer; ++q) f[q] = load4(t.e[k], i + q * kThreads * 4);
#pragma unroll
        for (int q = 0; q < kPer; ++q) store4(t.e[k], i + q * kThreads * 4, f[q], factor);
    }
}

constexpr int64_t kClipWorkspace = kMaxCtas * (int64_t)sizeof(double);

template <int N>
slicegcn_status_t fill_table(const slicegcn_tensor_list* list, ClipTable<N>& t) {
    t.count = 0;
    t.chunks = 0;
    for (int i = 0; i < list->count; ++i) {
        const int dt = list->dtypes ? list->dtypes[i] : SLICEGCN_F32;
        if (dt != SLICEGCN_F32 && dt != SLICEGCN_BF16) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: bad dtype of tensor %d", i);
        const int esz = dt == SLICEGCN_BF16 ? 2 : 4;
        const int64_t elems = list->elems[i];
        if (elems < 0) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: tensor %d has a negative size", i);
        if (elems == 0) continue;
        const void* src = list->src[i];
        void* dst = list->dst ? list->dst[i] : nullptr;
        if (!src || (list->dst && !dst)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: tensor %d is NULL", i);
        if ((uintptr_t)src % esz || (uintptr_t)dst % esz)
            SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: tensor %d is not aligned to its element type", i);
        ClipEntry& e = t.e[t.count++];
        e.src = src;
        e.dst = dst;
        e.elems = elems;
        e.first = t.chunks;
        e.bf16 = dt == SLICEGCN_BF16;
        e.vec = (uintptr_t)src % (4 * esz) == 0 && (uintptr_t)dst % (4 * esz) == 0;
        t.chunks += (elems + kClipChunk - 1) / kClipChunk;
    }
    return SLICEGCN_OK;
}

template <int N>
slicegcn_status_t run_two(const ClipTable<N>& t, double max_norm, float* norm_out, double* partial, cudaStream_t st) {
    const int ctas = (int)std::min<int64_t>(std::max<int64_t>(t.chunks, 1), kMaxCtas);
    clip_norm_kernel<N><<<ctas, kThreads, 0, st>>>(t, partial);
    SGCN_LAUNCH_CHECK();
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    SGCN_CUDA(cudaLaunchKernelEx(&cfg, clip_scale_kernel<N>, t, (const double*)partial, ctas, max_norm, norm_out));
    count_launch(2);
    return SLICEGCN_OK;
}

}  // namespace
}  // namespace sgcn

using namespace sgcn;

extern "C" {

slicegcn_status_t slicegcn_clip_workspace_bytes(int64_t* bytes) {
    if (!bytes) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_workspace_bytes: NULL argument");
    *bytes = kClipWorkspace;
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
    if ((uintptr_t)norm_out % 4 || (uintptr_t)workspace % 16)
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "clip_grads: norm_out or the workspace (16 bytes) is not aligned");
    const bool room = workspace && workspace_bytes >= kClipWorkspace;
    cudaStream_t st = (cudaStream_t)stream;
    double* partial = static_cast<double*>(workspace);
    if (list->count <= kShortList) {
        ClipTable<kShortList> t;
        SGCN_TRY(fill_table(list, t));
        if (!room)
            SGCN_FAIL(SLICEGCN_ERR_ALLOC, "clip_grads: workspace too small (%lld < %lld bytes)", (long long)workspace_bytes, (long long)kClipWorkspace);
        if (t.chunks > kClusterChunks) return run_two(t, max_norm, norm_out, partial, st);
        clip_cluster_kernel<<<kClusterCtas, kClusterThreads, 0, st>>>(t, max_norm, norm_out);
        SGCN_LAUNCH_CHECK();
        count_launch();
        return SLICEGCN_OK;
    }
    ClipTable<SLICEGCN_MAX_TENSORS> t;
    SGCN_TRY(fill_table(list, t));
    if (!room)
        SGCN_FAIL(SLICEGCN_ERR_ALLOC, "clip_grads: workspace too small (%lld < %lld bytes)", (long long)workspace_bytes, (long long)kClipWorkspace);
    return run_two(t, max_norm, norm_out, partial, st);
}

}  // extern "C"
