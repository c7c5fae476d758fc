// Residual step around a sliced layer: norms before and after the block, the gate and the residual scale, with statistics
// per slice (every block of h_s columns is normalised by itself, so the slices stay independent of each other).
//   h = x + s * sigmoid(gate) * (N(y) * w_post + b_post)          u = N(h) * w_pre + b_pre
//   N(t) = t / sqrt(mean(t^2) + eps)   or   (t - mean(t)) / sqrt(var(t) + eps)
// Gradient, with g' = J_N(t)^T g = r * (g - mean(g) - that * mean(g * that)) (r = 1 / the root, that = N(t), the plain mean
// only for the layer norm):
//   D = dh + J_N(h)^T (w_pre * du),  dx = D,  v = N(y) * w_post + b_post,  dt = D * s * sigmoid(gate)
//   dgate = D * s * v * sigmoid'(gate),  dy = J_N(y)^T (w_post * dt)
//   dw_post = sum(dt * N(y)), db_post = sum(dt), dw_pre = sum(du * N(h)), db_pre = sum(du)   over the rows
#include <algorithm>

#include "common.cuh"

namespace sgcn {
namespace {

__device__ __forceinline__ float ld_elem(const float* p) { return *p; }
__device__ __forceinline__ float ld_elem(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void st_elem(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ float sigmoid(float g) { return 1.f / (1.f + expf(-g)); }

struct Stats {
    float mean, r;   // N(t) = (t - mean) * r
};

// f(c) is element c of the slice row; the mean first, then the squares about it: nothing cancels
template <typename F>
__device__ __forceinline__ Stats slice_stats(F f, int w, int lane, bool layer, float eps) {
    Stats st{0.f, 0.f};
    if (layer) {
        float s = 0.f;
        for (int c = lane; c < w; c += 32) s += f(c);
        st.mean = warp_sum(s) / (float)w;
    }
    float q = 0.f;
    for (int c = lane; c < w; c += 32) {
        const float t = f(c) - st.mean;
        q = fmaf(t, t, q);
    }
    st.r = rsqrtf(warp_sum(q) / (float)w + eps);
    return st;
}

struct NormArgs {
    int64_t n;
    int p, w, layer;
    float eps, s;
    int64_t x_ld, y_ld, gate_ld, h_ld, u_ld, dh_ld, du_ld, dx_ld, dy_ld, dgate_ld;
    const float *w_post, *b_post, *w_pre, *b_pre;
};

template <typename T>
__global__ void norm_forward_kernel(const NormArgs a, const T* x, const T* y, const T* gate, T* h, T* u) {
    const int lane = threadIdx.x & 31;
    const int64_t item = (blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5;
    if (item >= a.n * a.p) return;
    const int64_t row = item / a.p;
    const int c0 = (int)(item - row * a.p) * a.w;
    Stats sy{0.f, 0.f}, sh{0.f, 0.f};
    if (y) sy = slice_stats([&](int c) { return ld_elem(y + row * a.y_ld + c0 + c); }, a.w, lane, a.layer, a.eps);
    auto hv = [&](int c) {   // unrounded h
        const int k = c0 + c;
        float v = x ? ld_elem(x + row * a.x_ld + k) : 0.f;
        if (y) {
            float t = (ld_elem(y + row * a.y_ld + k) - sy.mean) * sy.r;
            if (a.w_post) t *= a.w_post[k];
            if (a.b_post) t += a.b_post[k];
            if (gate) t *= sigmoid(ld_elem(gate + row * a.gate_ld + k));
            v = fmaf(a.s, t, v);
        }
        return v;
    };
    if (u) sh = slice_stats(hv, a.w, lane, a.layer, a.eps);
    for (int c = lane; c < a.w; c += 32) {
        const int k = c0 + c;
        const float v = hv(c);
        if (h) st_elem(h + row * a.h_ld + k, v);
        if (u) {
            float t = (v - sh.mean) * sh.r;
            if (a.w_pre) t *= a.w_pre[k];
            if (a.b_pre) t += a.b_pre[k];
            st_elem(u + row * a.u_ld + k, t);
        }
    }
}

// stats [n * p][4]: mean and r of y, then of h, for the column sums
template <typename T>
__global__ void norm_backward_kernel(const NormArgs a, const T* y, const T* gate, const T* h, const float* dh, const float* du,
                                     float* dx, float* dy, float* dgate, float4* stats) {
    const int lane = threadIdx.x & 31;
    const int64_t item = (blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5;
    if (item >= a.n * a.p) return;
    const int64_t row = item / a.p;
    const int c0 = (int)(item - row * a.p) * a.w;
    const float inv_w = 1.f / (float)a.w;
    Stats sy{0.f, 0.f}, sh{0.f, 0.f};
    float mg = 0.f, mgh = 0.f;
    if (du) {
        sh = slice_stats([&](int c) { return ld_elem(h + row * a.h_ld + c0 + c); }, a.w, lane, a.layer, a.eps);
        float s1 = 0.f, s2 = 0.f;
        for (int c = lane; c < a.w; c += 32) {
            const int k = c0 + c;
            const float g = du[row * a.du_ld + k] * (a.w_pre ? a.w_pre[k] : 1.f);
            s1 += g;
            s2 = fmaf(g, (ld_elem(h + row * a.h_ld + k) - sh.mean) * sh.r, s2);
        }
        mg = a.layer ? warp_sum(s1) * inv_w : 0.f;
        mgh = warp_sum(s2) * inv_w;
    }
    auto D = [&](int k) {
        float v = dh ? dh[row * a.dh_ld + k] : 0.f;
        if (du) {
            const float g = du[row * a.du_ld + k] * (a.w_pre ? a.w_pre[k] : 1.f);
            const float that = (ld_elem(h + row * a.h_ld + k) - sh.mean) * sh.r;
            v = fmaf(sh.r, g - mg - that * mgh, v);
        }
        return v;
    };
    float mt = 0.f, mty = 0.f;
    auto dt = [&](int k) { return D(k) * a.s * (gate ? sigmoid(ld_elem(gate + row * a.gate_ld + k)) : 1.f); };
    if (y) {
        sy = slice_stats([&](int c) { return ld_elem(y + row * a.y_ld + c0 + c); }, a.w, lane, a.layer, a.eps);
        float s1 = 0.f, s2 = 0.f;
        for (int c = lane; c < a.w; c += 32) {
            const int k = c0 + c;
            const float g = dt(k) * (a.w_post ? a.w_post[k] : 1.f);
            s1 += g;
            s2 = fmaf(g, (ld_elem(y + row * a.y_ld + k) - sy.mean) * sy.r, s2);
        }
        mt = a.layer ? warp_sum(s1) * inv_w : 0.f;
        mty = warp_sum(s2) * inv_w;
    }
    for (int c = lane; c < a.w; c += 32) {
        const int k = c0 + c;
        const float d = D(k);
        if (y) {
            const float yhat = (ld_elem(y + row * a.y_ld + k) - sy.mean) * sy.r;
            const float w = a.w_post ? a.w_post[k] : 1.f;
            const float g = gate ? ld_elem(gate + row * a.gate_ld + k) : 0.f;
            const float t = d * a.s * (gate ? sigmoid(g) : 1.f);
            if (dy) dy[row * a.dy_ld + k] = sy.r * (t * w - mt - yhat * mty);
            if (dgate) {
                const float e = expf(-fabsf(g));
                dgate[row * a.dgate_ld + k] = d * a.s * (yhat * w + (a.b_post ? a.b_post[k] : 0.f)) * (e / ((1.f + e) * (1.f + e)));
            }
        }
        if (dx) dx[row * a.dx_ld + k] = d;
    }
    if (stats && lane == 0) stats[item] = make_float4(sy.mean, sy.r, sh.mean, sh.r);
}

constexpr int kNormChunk = 256;   // rows per partial sum

template <typename T>
__global__ void norm_colsum_kernel(const NormArgs a, const T* y, const T* gate, const T* h, const float* du, const float* dx,
                                   const float4* stats, float* partial) {
    const int cols = a.p * a.w;
    const int k = blockIdx.x * blockDim.x + threadIdx.x;
    if (k >= cols) return;
    const int64_t r0 = (int64_t)blockIdx.y * kNormChunk, r1 = min(a.n, r0 + kNormChunk);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t r = r0; r < r1; ++r) {
        const float4 st = stats[r * a.p + k / a.w];
        if (y) {
            const float t = dx[r * a.dx_ld + k] * a.s * (gate ? sigmoid(ld_elem(gate + r * a.gate_ld + k)) : 1.f);
            s[0] = fmaf(t, (ld_elem(y + r * a.y_ld + k) - st.x) * st.y, s[0]);
            s[1] += t;
        }
        if (du) {
            const float g = du[r * a.du_ld + k];
            s[2] = fmaf(g, (ld_elem(h + r * a.h_ld + k) - st.z) * st.w, s[2]);
            s[3] += g;
        }
    }
    for (int i = 0; i < 4; ++i) partial[((int64_t)blockIdx.y * 4 + i) * cols + k] = s[i];
}

__global__ void norm_colsum_join_kernel(int64_t chunks, int cols, const float* partial, float* dw_post, float* db_post, float* dw_pre,
                                        float* db_pre) {
    const int k = blockIdx.x * blockDim.x + threadIdx.x, i = blockIdx.y;
    float* out = i == 0 ? dw_post : i == 1 ? db_post : i == 2 ? dw_pre : db_pre;
    if (k >= cols || !out) return;
    float s = 0.f;
    for (int64_t c = 0; c < chunks; ++c) s += partial[(c * 4 + i) * cols + k];
    out[k] = s;
}

slicegcn_status_t check_desc(const slicegcn_residual_norm_desc* d, const char* who) {
    if (!d) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: NULL description", who);
    if (d->n < 0 || d->num_slices < 1 || d->h_s < 1) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: bad sizes", who);
    if ((int64_t)d->num_slices * d->h_s >= ((int64_t)1 << 31)) SGCN_FAIL(SLICEGCN_ERR_OVERFLOW, "%s: the columns do not fit int32", who);
    if (d->num_slices > SLICEGCN_MAX_SLICES || d->h_s > SLICEGCN_MAX_NORM_WIDTH)
        SGCN_FAIL(SLICEGCN_ERR_UNSUPPORTED, "%s: at most %d slices of %d columns", who, SLICEGCN_MAX_SLICES, SLICEGCN_MAX_NORM_WIDTH);
    if (d->kind != SLICEGCN_ROWNORM_RMS && d->kind != SLICEGCN_ROWNORM_LAYER) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: bad kind", who);
    if (d->dtype != SLICEGCN_F32 && d->dtype != SLICEGCN_BF16) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: bad dtype", who);
    if (!(d->eps > 0)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: eps must be positive", who);
    const float* vec[] = {d->w_post, d->b_post, d->w_pre, d->b_pre};
    for (const float* v : vec)
        if ((uintptr_t)v % 4) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: a pointer is not aligned to its element type", who);
    return SLICEGCN_OK;
}

slicegcn_status_t check_matrix(const slicegcn_residual_norm_desc* d, const void* ptr, int64_t ld, int esz, const char* who, const char* what) {
    if (!ptr) return SLICEGCN_OK;
    if (ld < (int64_t)d->num_slices * d->h_s) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: leading dimension of %s too small", who, what);
    if ((uintptr_t)ptr % esz) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: %s is not aligned to its element type", who, what);
    return SLICEGCN_OK;
}

NormArgs make_args(const slicegcn_residual_norm_desc* d) {
    NormArgs a;
    a.n = d->n;
    a.p = d->num_slices;
    a.w = d->h_s;
    a.layer = d->kind == SLICEGCN_ROWNORM_LAYER;
    a.eps = (float)d->eps;
    a.s = (float)d->residual_scale;
    a.x_ld = d->x_ld, a.y_ld = d->y_ld, a.gate_ld = d->gate_ld, a.h_ld = d->h_ld, a.u_ld = d->u_ld;
    a.dh_ld = d->dh_ld, a.du_ld = d->du_ld, a.dx_ld = d->dx_ld, a.dy_ld = d->dy_ld, a.dgate_ld = d->dgate_ld;
    a.w_post = d->w_post, a.b_post = d->b_post, a.w_pre = d->w_pre, a.b_pre = d->b_pre;
    return a;
}

struct NormScratch {
    int64_t chunks, stats_bytes, dx_bytes, total;
};
NormScratch norm_scratch(const slicegcn_residual_norm_desc* d) {
    NormScratch s;
    const int64_t cols = (int64_t)d->num_slices * d->h_s;
    s.chunks = std::max<int64_t>(1, (d->n + kNormChunk - 1) / kNormChunk);
    s.stats_bytes = d->n * d->num_slices * 16;
    s.dx_bytes = d->n * cols * 4;
    s.total = s.stats_bytes + s.dx_bytes + s.chunks * 4 * cols * 4;
    return s;
}

}  // namespace
}  // namespace sgcn

using namespace sgcn;

extern "C" {

slicegcn_status_t slicegcn_residual_norm_forward(const slicegcn_residual_norm_desc* d, const void* x, const void* y, const void* gate,
                                                 void* h, void* u, void* stream) {
    const char* who = "residual_norm_forward";
    SGCN_TRY(check_desc(d, who));
    const int esz = d->dtype == SLICEGCN_BF16 ? 2 : 4;
    SGCN_TRY(check_matrix(d, x, d->x_ld, esz, who, "x"));
    SGCN_TRY(check_matrix(d, y, d->y_ld, esz, who, "y"));
    SGCN_TRY(check_matrix(d, gate, d->gate_ld, esz, who, "gate"));
    SGCN_TRY(check_matrix(d, h, d->h_ld, esz, who, "h"));
    SGCN_TRY(check_matrix(d, u, d->u_ld, esz, who, "u"));
    if (d->n == 0) return SLICEGCN_OK;
    if (!x && !y) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: neither x nor y is given", who);
    if (gate && !y) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: a gate without y", who);
    if (!h && !u) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: neither h nor u is asked for", who);
    const NormArgs a = make_args(d);
    cudaStream_t st = (cudaStream_t)stream;
    const unsigned blocks = (unsigned)((a.n * a.p + 7) / 8);
    if (d->dtype == SLICEGCN_BF16) {
        using T = __nv_bfloat16;
        norm_forward_kernel<T><<<blocks, 256, 0, st>>>(a, (const T*)x, (const T*)y, (const T*)gate, (T*)h, (T*)u);
    } else {
        norm_forward_kernel<float><<<blocks, 256, 0, st>>>(a, (const float*)x, (const float*)y, (const float*)gate, (float*)h, (float*)u);
    }
    SGCN_LAUNCH_CHECK();
    count_launch();
    return SLICEGCN_OK;
}

slicegcn_status_t slicegcn_residual_norm_workspace_bytes(const slicegcn_residual_norm_desc* d, int64_t* bytes) {
    SGCN_TRY(check_desc(d, "residual_norm_workspace_bytes"));
    if (!bytes) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "residual_norm_workspace_bytes: NULL argument");
    *bytes = norm_scratch(d).total;
    return SLICEGCN_OK;
}

slicegcn_status_t slicegcn_residual_norm_backward(const slicegcn_residual_norm_desc* d, const void* y, const void* gate, const void* h,
                                                  const float* dh, const float* du, float* dx, float* dy, float* dgate, float* dw_post,
                                                  float* db_post, float* dw_pre, float* db_pre, void* workspace,
                                                  int64_t workspace_bytes, void* stream) {
    const char* who = "residual_norm_backward";
    SGCN_TRY(check_desc(d, who));
    const int esz = d->dtype == SLICEGCN_BF16 ? 2 : 4;
    SGCN_TRY(check_matrix(d, y, d->y_ld, esz, who, "y"));
    SGCN_TRY(check_matrix(d, gate, d->gate_ld, esz, who, "gate"));
    SGCN_TRY(check_matrix(d, h, d->h_ld, esz, who, "h"));
    SGCN_TRY(check_matrix(d, dh, d->dh_ld, 4, who, "dh"));
    SGCN_TRY(check_matrix(d, du, d->du_ld, 4, who, "du"));
    SGCN_TRY(check_matrix(d, dx, d->dx_ld, 4, who, "dx"));
    SGCN_TRY(check_matrix(d, dy, d->dy_ld, 4, who, "dy"));
    SGCN_TRY(check_matrix(d, dgate, d->dgate_ld, 4, who, "dgate"));
    const float* vec[] = {dw_post, db_post, dw_pre, db_pre};
    for (const float* v : vec)
        if ((uintptr_t)v % 4) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: a pointer is not aligned to its element type", who);
    if (d->n > 0) {
        if (!dh && !du) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: neither dh nor du is given", who);
        if (du && !h) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: du without h", who);
        if (gate && !y) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: a gate without y", who);
        if (!y && dy) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: dy without y", who);
        if (!gate && dgate) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: dgate without gate", who);
    }
    if (!y && (dw_post || db_post) && d->n > 0) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: dw_post / db_post without y", who);
    if (!du && (dw_pre || db_pre) && d->n > 0) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: dw_pre / db_pre without du", who);
    const bool sums = dw_post || db_post || dw_pre || db_pre;
    const NormScratch sc = norm_scratch(d);
    if ((sums || !dx) && (!workspace || workspace_bytes < sc.total))
        SGCN_FAIL(SLICEGCN_ERR_ALLOC, "%s: workspace too small (%lld < %lld bytes)", who, (long long)workspace_bytes, (long long)sc.total);
    if ((uintptr_t)workspace % 16) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: the workspace is not aligned to 16 bytes", who);
    NormArgs a = make_args(d);
    cudaStream_t st = (cudaStream_t)stream;
    const int cols = a.p * a.w;
    char* ws = static_cast<char*>(workspace);
    float4* stats = sums ? reinterpret_cast<float4*>(ws) : nullptr;
    float* partial = sums ? reinterpret_cast<float*>(ws + sc.stats_bytes + sc.dx_bytes) : nullptr;
    if (!dx && sums) {
        dx = reinterpret_cast<float*>(ws + sc.stats_bytes);
        a.dx_ld = cols;
    }
    if (a.n > 0) {
        const unsigned blocks = (unsigned)((a.n * a.p + 7) / 8);
        if (d->dtype == SLICEGCN_BF16) {
            using T = __nv_bfloat16;
            norm_backward_kernel<T><<<blocks, 256, 0, st>>>(a, (const T*)y, (const T*)gate, (const T*)h, dh, du, dx, dy, dgate, stats);
        } else {
            using T = float;
            norm_backward_kernel<T><<<blocks, 256, 0, st>>>(a, (const T*)y, (const T*)gate, (const T*)h, dh, du, dx, dy, dgate, stats);
        }
        SGCN_LAUNCH_CHECK();
        count_launch();
    }
    if (sums) {
        const dim3 grid((cols + 127) / 128, (unsigned)sc.chunks);
        if (d->dtype == SLICEGCN_BF16) {
            using T = __nv_bfloat16;
            norm_colsum_kernel<T><<<grid, 128, 0, st>>>(a, (const T*)y, (const T*)gate, (const T*)h, du, dx, stats, partial);
        } else {
            using T = float;
            norm_colsum_kernel<T><<<grid, 128, 0, st>>>(a, (const T*)y, (const T*)gate, (const T*)h, du, dx, stats, partial);
        }
        SGCN_LAUNCH_CHECK();
        norm_colsum_join_kernel<<<dim3((cols + 127) / 128, 4), 128, 0, st>>>(sc.chunks, cols, partial, dw_post, db_post, dw_pre, db_pre);
        SGCN_LAUNCH_CHECK();
        count_launch(2);
    }
    return SLICEGCN_OK;
}

}  // extern "C"
