// Global 2-norm of a list of gradient tensors, and clipping by it:
//   norm = sqrt(sum over all tensors of g^2);   dst = g * (norm > max_norm and finite ? max_norm / norm : 1)
// The order of the sums is fixed.
#include <cooperative_groups.h>

#include <algorithm>

#include "common.cuh"

namespace sgcn {
namespace {

constexpr int kPieceBytes = 16384;   // of one tensor: the work item of a CTA, 16 bytes per thread and step
constexpr int kSMs = 148;

// A stretch of one tensor of at most kPieceBytes.
struct Piece {
    const char* src;
    char* dst;
    int bytes;
    int bf16, vec;   // vec: 16 bytes at a time are aligned in src and dst
};

// The 16 bytes at `off` of a piece.  The load has no condition on it (past the end it reads the piece's start, and the last
// 16 bytes may reach past the end, never past an aligned 16-byte unit that the tensor shares): with one, the compiler waits
// for each value where the cases meet, and a thread has one load on its way instead of several.
struct Raw {
    uint32_t w[4];
};
__device__ __forceinline__ Raw load16(const Piece& p, int off) {
    Raw r;
    if (p.vec) {
        const uint4 t = *reinterpret_cast<const uint4*>(p.src + (off < p.bytes ? off : 0));
        r.w[0] = t.x, r.w[1] = t.y, r.w[2] = t.z, r.w[3] = t.w;
    } else if (p.bf16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint16_t* at = reinterpret_cast<const uint16_t*>(p.src + off) + 2 * k;
            r.w[k] = off + 4 * k < p.bytes ? at[0] : 0u;
            if (off + 4 * k + 2 < p.bytes) r.w[k] |= (uint32_t)at[1] << 16;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) r.w[k] = off + 4 * k < p.bytes ? reinterpret_cast<const uint32_t*>(p.src + off)[k] : 0u;
    }
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The squares are taken and added in 64 bits: the square of any fp32 number fits a double, so neither large nor tiny
// gradients leave its range.  The 64-bit units about keep up with HBM: 245 M numbers take 474 us in fp32 (both launches together
// move 6.2 TB/s) and 259 us in bf16 (5.7 TB/s), where there are twice as many conversions per byte.
__device__ __forceinline__ double squares(const Piece& p, int off, const Raw& r) {
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int left = p.bytes - off - 4 * k;   // bytes from this word on
        if (p.bf16) {
            const double a = left > 0 ? bf16_lo(r.w[k]) : 0.f, b = left > 2 ? bf16_hi(r.w[k]) : 0.f;
            s = fma(a, a, fma(b, b, s));
        } else {
            const double a = left > 0 ? __uint_as_float(r.w[k]) : 0.f;
            s = fma(a, a, s);
        }
    }
    return s;
}

// max_norm / norm, or 1.
__device__ __forceinline__ double clip_factor(double norm, double max_norm) {
    return norm > max_norm && isfinite(norm) ? max_norm / norm : 1.0;
}
// Below the normal fp32 numbers (a norm of 3e38 against a limit of 1e-3) a factor loses its digits in 32 bits, and the products
// are taken in 64.  The whole launch takes one way or the other: a choice per product costs 1.5 % of the large lists' time.
constexpr double kLeastNormal = 1.17549435e-38;
__device__ __forceinline__ float times(float g, float f) { return g * f; }
__device__ __forceinline__ float times(float g, double f) { return (float)(g * f); }

template <typename F>
__device__ __forceinline__ void store16(const Piece& p, int off, const Raw& r, F f) {
    if (off >= p.bytes) return;
    if (p.bf16) {
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 t = __floats2bfloat162_rn(times(bf16_lo(r.w[k]), f), times(bf16_hi(r.w[k]), f));
            o[k] = *reinterpret_cast<const uint32_t*>(&t);
        }
        if (p.vec && off + 16 <= p.bytes) {
            __stcs(reinterpret_cast<uint4*>(p.dst + off), make_uint4(o[0], o[1], o[2], o[3]));
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (off + 2 * k < p.bytes) reinterpret_cast<uint16_t*>(p.dst + off)[k] = (uint16_t)(k & 1 ? o[k / 2] >> 16 : o[k / 2]);
        }
        return;
    }
    const float v[4] = {times(__uint_as_float(r.w[0]), f), times(__uint_as_float(r.w[1]), f), times(__uint_as_float(r.w[2]), f), times(__uint_as_float(r.w[3]), f)};
    if (p.vec && off + 16 <= p.bytes) {
        __stcs(reinterpret_cast<float4*>(p.dst + off), make_float4(v[0], v[1], v[2], v[3]));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (off + 4 * k < p.bytes) reinterpret_cast<float*>(p.dst + off)[k] = v[k];
    }
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

// Small lists (up to kClusterPieces pieces, laid out by the host): one launch of one cluster that keeps every gradient in
// registers between the sum and the scaling, so each is read once.  The CTAs' sums meet in distributed shared memory.  Sixteen
// CTAs, the most a cluster may have: the SMs' rate of conversions and stores bounds it (13 tensors of 117,800 numbers in all:
// 3.9 us, 5.6 with eight CTAs).
constexpr int kClusterCtas = 16, kClusterThreads = 1024, kHeld = 4;
constexpr int kClusterPieces = kClusterCtas * kHeld;
struct PieceTable {
    int count;
    Piece p[kClusterPieces];
};
__global__ void __cluster_dims__(kClusterCtas, 1, 1) __launch_bounds__(kClusterThreads)
    clip_cluster_kernel(const __grid_constant__ PieceTable t, double max_norm, float* norm_out) {
    namespace cg = cooperative_groups;
    __shared__ double smem[kClusterThreads / 32];
    __shared__ double sums[kClusterCtas];
    const cg::cluster_group cluster = cg::this_cluster();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int rank = blockIdx.x, off = threadIdx.x * 16;
    Raw held[kHeld];
#pragma unroll
    for (int q = 0; q < kHeld; ++q)
        if (rank + q * kClusterCtas < t.count) held[q] = load16(t.p[rank + q * kClusterCtas], off);
    double s = 0.0;
#pragma unroll
    for (int q = 0; q < kHeld; ++q)
        if (rank + q * kClusterCtas < t.count) s += squares(t.p[rank + q * kClusterCtas], off, held[q]);
    // Only the first warp takes the CTA's sum, the root and the quotient: 64-bit steps by all 32 warps queue up (6.5 us
    // instead of 5.9 for 117,800 numbers in 13 tensors).
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        s = smem[threadIdx.x];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    }
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");   // another CTA's shared memory exists once that CTA runs; a CTA without a piece is here at once
    if (threadIdx.x < kClusterCtas) *cluster.map_shared_rank(&sums[rank], threadIdx.x) = s;
    cluster.sync();   // hardware barrier; no CTA reads another's memory after it
    if (threadIdx.x == 0) {
        double total = 0.0;
#pragma unroll
        for (int r = 0; r < kClusterCtas; ++r) total += sums[r];
        const double norm = sqrt(total);
        if (norm_out && rank == 0) *norm_out = (float)norm;
        smem[0] = clip_factor(norm, max_norm);
    }
    __syncthreads();
    const double factor = smem[0];
    auto store = [&](auto f) {
#pragma unroll
        for (int q = 0; q < kHeld; ++q)
            if (rank + q * kClusterCtas < t.count && t.p[rank + q * kClusterCtas].dst) store16(t.p[rank + q * kClusterCtas], off, held[q], f);
    };
    if (factor < kLeastNormal)
        store(factor);
    else
        store((float)factor);
}

// Larger lists: two launches bound by HBM.  The second one walks the pieces backwards, since what the first one read last is
// still in L2, and its launch overlaps the end of the first (it waits for the sums on the device).
struct ClipEntry {
    const char* src;
    char* dst;
    int64_t bytes;
    int64_t first;   // index of the tensor's first piece
    int bf16, vec;
};
// N: room for tensors.  A short list travels as a short kernel argument, which costs less to launch (512 tensors: 20 KB).
template <int N>
struct ClipTable {
    int count;
    int64_t pieces;
    ClipEntry e[N];
};
constexpr int kShortList = 32;
__device__ __forceinline__ Piece piece_of(const ClipEntry& e, int64_t piece) {
    const int64_t at = (piece - e.first) * kPieceBytes;
    return Piece{e.src + at, e.dst ? e.dst + at : nullptr, (int)min(e.bytes - at, (int64_t)kPieceBytes), e.bf16, e.vec};
}
constexpr int kThreads = 256, kPer = kPieceBytes / kThreads / 16, kMaxCtas = 8 * kSMs;
template <int N>
__global__ void __launch_bounds__(kThreads) clip_norm_kernel(const __grid_constant__ ClipTable<N> t, double* partial) {
    __shared__ double smem[kThreads / 32];
    cudaTriggerProgrammaticLaunchCompletion();
    double s = 0.0;
    int k = 0;
    for (int64_t c = blockIdx.x; c < t.pieces; c += gridDim.x) {
        while (k + 1 < t.count && t.e[k + 1].first <= c) ++k;
        const Piece p = piece_of(t.e[k], c);
        Raw r[kPer];
#pragma unroll
        for (int q = 0; q < kPer; ++q) r[q] = load16(p, (q * kThreads + threadIdx.x) * 16);
#pragma unroll
        for (int q = 0; q < kPer; ++q) s += squares(p, (q * kThreads + threadIdx.x) * 16, r[q]);
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
    const double factor = clip_factor(norm, max_norm);
    auto scale = [&](auto f) {
        int k = t.count - 1;
        for (int64_t c = t.pieces - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
            while (t.e[k].first > c) --k;
            const Piece p = piece_of(t.e[k], c);
            if (!p.dst || (f == 1 && p.dst == p.src)) continue;
            Raw r[kPer];
#pragma unroll
            for (int q = 0; q < kPer; ++q) r[q] = load16(p, (q * kThreads + threadIdx.x) * 16);
#pragma unroll
            for (int q = 0; q < kPer; ++q) store16(p, (q * kThreads + threadIdx.x) * 16, r[q], f);
        }
    };
    if (factor < kLeastNormal)
        scale(factor);
    else
        scale((float)factor);
}

constexpr int64_t kClipWorkspace = kMaxCtas * (int64_t)sizeof(double);

template <int N>
slicegcn_status_t fill_table(const slicegcn_tensor_list* list, ClipTable<N>& t) {
    t.count = 0;
    t.pieces = 0;
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
        e.src = static_cast<const char*>(src);
        e.dst = static_cast<char*>(dst);
        e.bytes = elems * esz;
        e.first = t.pieces;
        e.bf16 = dt == SLICEGCN_BF16;
        e.vec = (uintptr_t)src % 16 == 0 && (uintptr_t)dst % 16 == 0;
        t.pieces += (e.bytes + kPieceBytes - 1) / kPieceBytes;
    }
    return SLICEGCN_OK;
}

template <int N>
slicegcn_status_t run_two(const ClipTable<N>& t, double max_norm, float* norm_out, double* partial, cudaStream_t st) {
    const int ctas = (int)std::min<int64_t>(std::max<int64_t>(t.pieces, 1), kMaxCtas);
    clip_norm_kernel<N><<<ctas, kThreads, 0, st>>>(t, partial);
    SGCN_LAUNCH_CHECK();
    count_launch();
    SGCN_TRY(launch_after(clip_scale_kernel<N>, dim3(ctas), kThreads, 0, st, t, (const double*)partial, ctas, max_norm, norm_out));
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
        if (t.pieces > kClusterPieces) return run_two(t, max_norm, norm_out, partial, st);
        PieceTable small;
        small.count = (int)t.pieces;
        for (int k = 0, c = 0; k < t.count; ++k)
            for (int64_t at = 0; at < t.e[k].bytes; at += kPieceBytes, ++c)
                small.p[c] = Piece{t.e[k].src + at, t.e[k].dst ? t.e[k].dst + at : nullptr,
                                   (int)std::min<int64_t>(t.e[k].bytes - at, kPieceBytes), t.e[k].bf16, t.e[k].vec};
        SGCN_CUDA(cudaFuncSetAttribute(clip_cluster_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));   // more than eight
        clip_cluster_kernel<<<kClusterCtas, kClusterThreads, 0, st>>>(small, max_norm, norm_out);
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
