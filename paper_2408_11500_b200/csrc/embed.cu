// Embedding lookup with scaling, and its gradient by sorted ids.
//   forward   out[i, :] = scale * table[ids[i], :]            (ids[i] = -1: a row of zeros)
//   gradient  dtable[v, :] = sum over {i : ids[i] = v} of scale * dout[i, :]
// The gradient sorts the ids (stable least-significant-digit radix sort), so the positions of one id lie next to each
// other in their own order and every row of dtable is one sum in a fixed order: no floating-point atomics.
#include <algorithm>

#include "common.cuh"

namespace sgcn {
namespace {

constexpr int kSortThreads = 256;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortTile = 4096;   // positions per CTA and digit pass

__device__ __forceinline__ float ld_elem(const float* p) { return __ldg(p); }
__device__ __forceinline__ float ld_elem(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void st_elem(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// An id the kernels may index with, or -1: the padding id and ids outside the table (reported in *status).
__device__ __forceinline__ int32_t checked_id(int32_t id, int64_t vocab, int32_t* status) {
    if (id >= 0 && id < vocab) return id;
    if (id != -1 && status) atomicExch(status, SLICEGCN_DEVSTATUS_BAD_ID);
    return -1;
}

template <typename TT, typename TO>
__global__ void embed_forward_kernel(int64_t n, int64_t vocab, int width, const int32_t* ids, const TT* table, int64_t table_ld,
                                     TO* out, int64_t out_ld, float scale, int32_t* status) {
    const int64_t total = n * width;
    for (int64_t e = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; e < total; e += (int64_t)gridDim.x * blockDim.x) {
        const int64_t r = e / width;
        const int c = (int)(e - r * width);
        const int32_t id = checked_id(ids[r], vocab, status);
        st_elem(out + r * out_ld + c, id < 0 ? 0.f : scale * ld_elem(table + (int64_t)id * table_ld + c));
    }
}

// Sort keys: the id, or `vocab` (sorted last) for positions that take no part.
__device__ __forceinline__ uint32_t sort_key(int32_t id, int64_t vocab, int32_t* status) {
    const int32_t v = checked_id(id, vocab, status);
    return v < 0 ? (uint32_t)vocab : (uint32_t)v;
}

__global__ void sort_init_kernel(int64_t n, int64_t vocab, const int32_t* ids, uint2* pairs, int32_t* status) {
    for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x)
        pairs[i] = make_uint2(sort_key(ids[i], vocab, status), (uint32_t)i);
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(int64_t n, const uint2* pairs, int shift, int tiles, uint32_t* counts) {
    __shared__ uint32_t hist[256];
    hist[threadIdx.x] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * kSortTile, i1 = min(n, i0 + kSortTile);
    for (int64_t i = i0 + threadIdx.x; i < i1; i += kSortThreads) atomicAdd(&hist[(pairs[i].x >> shift) & 255u], 1u);
    __syncthreads();
    counts[(int64_t)threadIdx.x * tiles + blockIdx.x] = hist[threadIdx.x];
}

__global__ void __launch_bounds__(1024) sort_scan_kernel(int64_t m, uint32_t* counts) {   // exclusive scan by one CTA
    __shared__ uint32_t warp_sum[32];
    __shared__ uint32_t carry;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    for (int64_t base = 0; base < m; base += 1024) {
        const int64_t i = base + threadIdx.x;
        const uint32_t v = i < m ? counts[i] : 0;
        uint32_t s = v;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t t = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += t;
        }
        if (lane == 31) warp_sum[w] = s;
        __syncthreads();
        uint32_t before = carry;
        for (int k = 0; k < w; ++k) before += warp_sum[k];
        if (i < m) counts[i] = before + s - v;
        __syncthreads();
        if (threadIdx.x == 1023) carry = before + s;
        __syncthreads();
    }
}

// Stable scatter: each warp owns a contiguous run of the tile and walks it 32 positions at a time.
__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(int64_t n, const uint2* in, int shift, int tiles, const uint32_t* offsets,
                                                                    uint2* out) {
    __shared__ uint32_t next[kSortWarps][256];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    for (int k = threadIdx.x; k < kSortWarps * 256; k += kSortThreads) (&next[0][0])[k] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * kSortTile + (int64_t)w * (kSortTile / kSortWarps);
    const int64_t i1 = min(n, i0 + kSortTile / kSortWarps);
    for (int64_t i = i0 + lane; i < i1; i += 32) atomicAdd(&next[w][(in[i].x >> shift) & 255u], 1u);
    __syncthreads();
    {
        uint32_t at = offsets[(int64_t)threadIdx.x * tiles + blockIdx.x];
        for (int k = 0; k < kSortWarps; ++k) {
            const uint32_t c = next[k][threadIdx.x];
            next[k][threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();
    for (int64_t b = i0; b < i1; b += 32) {
        const int64_t i = b + lane;
        const bool live = i < i1;
        const uint2 p = live ? in[i] : make_uint2(0, 0);
        const uint32_t d = live ? (p.x >> shift) & 255u : 256u + lane;   // idle lanes match nobody
        const uint32_t peers = __match_any_sync(0xffffffffu, d);
        const uint32_t rank = __popc(peers & ((1u << lane) - 1u));
        uint32_t at = 0;
        if (live) at = next[w][d] + rank;
        __syncwarp();
        if (live && rank == 0) next[w][d] += __popc(peers);
        __syncwarp();
        if (live) out[at] = p;
    }
}

__device__ int64_t lower_bound_key(const uint2* pairs, int64_t n, uint32_t key) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (pairs[mid].x < key)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

// One warp per row of dtable: the positions of its id, summed in order.
__global__ void embed_reduce_kernel(int64_t n, int64_t vocab, int width, const uint2* pairs, const float* dout, int64_t dout_ld,
                                    float* dtable, int64_t dtable_ld, float scale, int accumulate) {
    const int lane = threadIdx.x & 31;
    const int64_t v = (blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5;
    if (v >= vocab) return;
    const int64_t a = lower_bound_key(pairs, n, (uint32_t)v), b = lower_bound_key(pairs, n, (uint32_t)v + 1);
    for (int c = lane; c < width; c += 32) {
        float s = 0.f;
        for (int64_t i = a; i < b; ++i) s += scale * __ldg(dout + (int64_t)pairs[i].y * dout_ld + c);
        float* t = dtable + v * dtable_ld + c;
        if (!accumulate)
            *t = s;
        else if (b > a)
            *t += s;
    }
}

slicegcn_status_t check_desc(const slicegcn_embed_desc* d, const char* who) {
    if (!d) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: NULL description", who);
    if (d->n < 0 || d->vocab < 1 || d->width < 1) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: bad sizes", who);
    if (d->n >= ((int64_t)1 << 31) || d->vocab >= ((int64_t)1 << 31) - 1)
        SGCN_FAIL(SLICEGCN_ERR_OVERFLOW, "%s: n or vocab does not fit int32", who);
    return SLICEGCN_OK;
}

int64_t align256(int64_t b) { return (b + 255) / 256 * 256; }

struct SortLayout {
    int64_t tiles, pairs_bytes, counts_bytes, total;
};
SortLayout sort_layout(const slicegcn_embed_desc* d) {
    SortLayout L;
    L.tiles = std::max<int64_t>(1, (d->n + kSortTile - 1) / kSortTile);
    L.pairs_bytes = align256(d->n * (int64_t)sizeof(uint2));
    L.counts_bytes = align256(L.tiles * 256 * (int64_t)sizeof(uint32_t));
    L.total = 2 * L.pairs_bytes + L.counts_bytes;
    return L;
}

template <typename TT, typename TO>
slicegcn_status_t forward_typed(const slicegcn_embed_desc* d, const int32_t* ids, const void* table, void* out, int32_t* status,
                                cudaStream_t st) {
    const unsigned blocks = (unsigned)std::min<int64_t>((d->n * d->width + 255) / 256, 148 * 32);
    embed_forward_kernel<TT, TO><<<blocks, 256, 0, st>>>(d->n, d->vocab, d->width, ids, static_cast<const TT*>(table), d->table_ld,
                                                         static_cast<TO*>(out), d->out_ld, (float)d->scale, status);
    SGCN_LAUNCH_CHECK();
    count_launch();
    return SLICEGCN_OK;
}

}  // namespace
}  // namespace sgcn

using namespace sgcn;

extern "C" {

slicegcn_status_t slicegcn_embed_forward(const slicegcn_embed_desc* d, const int32_t* ids, const void* table, void* out,
                                         int32_t* status, void* stream) {
    SGCN_TRY(check_desc(d, "embed_forward"));
    const bool tbf = d->table_dtype == SLICEGCN_BF16, obf = d->out_dtype == SLICEGCN_BF16;
    if ((!tbf && d->table_dtype != SLICEGCN_F32) || (!obf && d->out_dtype != SLICEGCN_F32))
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_forward: bad dtype");
    if (d->table_ld < d->width || d->out_ld < d->width) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_forward: leading dimension too small");
    if (d->n == 0) return SLICEGCN_OK;
    if (!ids || !table || !out) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_forward: NULL argument");
    if ((uintptr_t)ids % 4 || (uintptr_t)status % 4 || (uintptr_t)table % (tbf ? 2 : 4) || (uintptr_t)out % (obf ? 2 : 4))
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_forward: a pointer is not aligned to its element type");
    cudaStream_t st = (cudaStream_t)stream;
    if (tbf) return obf ? forward_typed<__nv_bfloat16, __nv_bfloat16>(d, ids, table, out, status, st)
                        : forward_typed<__nv_bfloat16, float>(d, ids, table, out, status, st);
    return obf ? forward_typed<float, __nv_bfloat16>(d, ids, table, out, status, st) : forward_typed<float, float>(d, ids, table, out, status, st);
}

slicegcn_status_t slicegcn_embed_workspace_bytes(const slicegcn_embed_desc* d, int64_t* bytes) {
    SGCN_TRY(check_desc(d, "embed_workspace_bytes"));
    if (!bytes) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_workspace_bytes: NULL argument");
    *bytes = sort_layout(d).total;
    return SLICEGCN_OK;
}

slicegcn_status_t slicegcn_embed_backward(const slicegcn_embed_desc* d, const int32_t* ids, const float* dout, float* dtable,
                                          int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
    SGCN_TRY(check_desc(d, "embed_backward"));
    if (d->dout_ld < d->width || d->dtable_ld < d->width) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_backward: leading dimension too small");
    if (!dtable || (d->n > 0 && (!ids || !dout))) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_backward: NULL argument");
    if ((uintptr_t)ids % 4 || (uintptr_t)status % 4 || (uintptr_t)dout % 4 || (uintptr_t)dtable % 4 || (uintptr_t)workspace % 16)
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_backward: a pointer is not aligned to its element type (workspace: 16 bytes)");
    const SortLayout L = sort_layout(d);
    if (!workspace || workspace_bytes < L.total)
        SGCN_FAIL(SLICEGCN_ERR_ALLOC, "embed_backward: workspace too small (%lld < %lld bytes)", (long long)workspace_bytes, (long long)L.total);
    cudaStream_t st = (cudaStream_t)stream;
    char* ws = static_cast<char*>(workspace);
    uint2* a = reinterpret_cast<uint2*>(ws);
    uint2* b = reinterpret_cast<uint2*>(ws + L.pairs_bytes);
    uint32_t* counts = reinterpret_cast<uint32_t*>(ws + 2 * L.pairs_bytes);
    if (d->n > 0) {
        sort_init_kernel<<<(unsigned)std::min<int64_t>((d->n + 255) / 256, 148 * 16), 256, 0, st>>>(d->n, d->vocab, ids, a, status);
        SGCN_LAUNCH_CHECK();
        count_launch();
        for (int shift = 0; (d->vocab >> shift) > 0; shift += 8) {   // keys run up to vocab itself
            sort_count_kernel<<<(unsigned)L.tiles, kSortThreads, 0, st>>>(d->n, a, shift, (int)L.tiles, counts);
            SGCN_LAUNCH_CHECK();
            sort_scan_kernel<<<1, 1024, 0, st>>>(L.tiles * 256, counts);
            SGCN_LAUNCH_CHECK();
            sort_scatter_kernel<<<(unsigned)L.tiles, kSortThreads, 0, st>>>(d->n, a, shift, (int)L.tiles, counts, b);
            SGCN_LAUNCH_CHECK();
            count_launch(3);
            std::swap(a, b);
        }
    }
    embed_reduce_kernel<<<(unsigned)((d->vocab + 7) / 8), 256, 0, st>>>(d->n, d->vocab, d->width, a, dout, d->dout_ld, dtable, d->dtable_ld,
                                                                        (float)d->scale, d->accumulate);
    SGCN_LAUNCH_CHECK();
    count_launch();
    return SLICEGCN_OK;
}

}  // extern "C"
