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

struct NormArgs {
    int64_t n;
    int p, w, layer;
    float eps, s;
    int64_t x_ld, y_ld, gate_ld, h_ld, u_ld, dh_ld, du_ld, dx_ld, dy_ld, dgate_ld;
    const float *w_post, *b_post, *w_pre, *b_pre;
    int64_t lanes_rows;   // rows that are worked on at a time: groups / p
    float* partial;       // gradient: [partial rows][4][p * w] column sums, or NULL when none is asked for
    int whole_rows;       // a CTA's groups cover whole rows: it leaves one partial row, not one per group
};

// ---- four columns of a slice row, as one access (VEC) or as four columns L apart ---------------
// VEC needs rows whose slices start on boundaries of four elements; the last four columns may then reach past the slice
// (one slice of 602 columns): what is read there is ignored, and such a quad is stored element by element.
template <typename T>
struct Quad;
template <>
struct Quad<float> {
    float4 v;
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w; }
    __device__ __forceinline__ void load(const float* p) { v = __ldcs(reinterpret_cast<const float4*>(p)); }
    static __device__ __forceinline__ void store(float* p, const float (&f)[4]) {
        __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    }
    __device__ __forceinline__ void set(int j, float x) { (&v.x)[j] = x; }
};
template <>
struct Quad<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void get(float (&f)[4]) const {
        f[0] = __uint_as_float(v.x << 16), f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16), f[3] = __uint_as_float(v.y & 0xffff0000u);
    }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldcs(reinterpret_cast<const uint2*>(p)); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&f)[4]) {
        uint2 o;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o.x) : "f"(f[1]), "f"(f[0]));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o.y) : "f"(f[3]), "f"(f[2]));
        __stcs(reinterpret_cast<uint2*>(p), o);
    }
    __device__ __forceinline__ void set(int j, float x) {   // x is a bf16 value
        uint32_t& t = j < 2 ? v.x : v.y;
        t = j & 1 ? (t & 0xffffu) | (__float_as_uint(x) & 0xffff0000u) : (t & 0xffff0000u) | (__float_as_uint(x) >> 16);
    }
};
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// `left` columns of the slice are at or after the first of the four
template <typename T, bool VEC>
__device__ __forceinline__ Quad<T> quad_load(const T* p, int step, int left) {
    Quad<T> q;
    q.v = {};
    if (VEC) {
        if (left > 0) q.load(p);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j * step < left) q.set(j, to_float(p[j * step]));
    }
    return q;
}
template <typename T, bool VEC>
__device__ __forceinline__ void quad_store(T* p, int step, int left, const float (&f)[4]) {
    if (VEC && left >= 4) {
        Quad<T>::store(p, f);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j * (VEC ? 1 : step) < left) put(p + j * (VEC ? 1 : step), f[j]);
    }
}
template <bool VEC>
__device__ __forceinline__ void vector_load(const float* p, int step, int left, float otherwise, float (&f)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = p && j * (VEC ? 1 : step) < left ? __ldg(p + j * (VEC ? 1 : step)) : otherwise;
}

// ---- sums over the lanes of one slice row -------------------------------------------------------
// L = 1 .. 32: L neighbouring lanes of a warp (every lane of the warp takes part in the shuffles).  L = 0: the whole CTA;
// two buffers in turn, so that one barrier per sum is enough.
constexpr int kMaxNormWarps = 32;
template <int L, int K>
__device__ __forceinline__ void group_sum(float (&v)[K], float (*smem)[kMaxNormWarps][4], int& turn) {
#pragma unroll
    for (int o = (L ? L : 32) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if (L == 0) {
        const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        if (warps == 1) return;
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) smem[turn][threadIdx.x >> 5][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = lane < warps ? smem[turn][lane][k] : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
        turn ^= 1;
    }
}

// sigmoid(g) = 1 / (1 + e^-g).  The hardware's exponential and division are good to a few units in the last place of fp32;
// e^-g overflows to infinity for very negative g, which gives the right 0.
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }

// Where a thread works: its group's slice, first row, and the columns of its quads.
template <int L>
struct Place {
    int lane, slice;
    int64_t row;        // first row; then every lanes_rows-th
    bool idle;
    int64_t partial_row;
    __device__ __forceinline__ Place(const NormArgs& a) {
        const int per_cta = L ? (int)blockDim.x / (L ? L : 1) : 1;
        lane = L ? (int)threadIdx.x & (L - 1) : (int)threadIdx.x;
        const int64_t g = (int64_t)blockIdx.x * per_cta + (L ? (int)threadIdx.x / (L ? L : 1) : 0);
        row = g / a.p;
        slice = (int)(g - row * a.p);
        idle = row >= a.lanes_rows;
        partial_row = row;
    }
};

// Bound by HBM: x, y and gate are read once, h and u written once.  A slice row lives in the registers of its lanes from
// the first load to the last store, so both norms cost shuffles and no second pass; the next row is requested before this
// one is worked on.  NV = 1: four columns per lane, whose weights stay in registers over all rows.
template <typename T, bool VEC, int L, int NV>
__global__ void __launch_bounds__(L ? 256 : 1024) norm_forward_kernel(const NormArgs a, const T* x, const T* y, const T* gate, T* h, T* u) {
    __shared__ float smem[2][kMaxNormWarps][4];
    int turn = 0;
    const Place<L> at(a);
    const int lanes = L ? L : blockDim.x;
    const int c0 = at.slice * a.w, c = VEC ? 4 * at.lane : at.lane, step = lanes, hop = 4 * lanes;   // quad i: columns c + i hop ...
    const float inv_w = 1.f / (float)a.w;
    const int left = at.idle ? 0 : a.w - c;
    float wp[4], bp[4], wq[4], bq[4];
    auto weights_post = [&](int i) {
        vector_load<VEC>(a.w_post ? a.w_post + c0 + c + i * hop : nullptr, step, left - i * hop, 1.f, wp);
        vector_load<VEC>(a.b_post ? a.b_post + c0 + c + i * hop : nullptr, step, left - i * hop, 0.f, bp);
    };
    auto weights_pre = [&](int i) {
        vector_load<VEC>(a.w_pre ? a.w_pre + c0 + c + i * hop : nullptr, step, left - i * hop, 1.f, wq);
        vector_load<VEC>(a.b_pre ? a.b_pre + c0 + c + i * hop : nullptr, step, left - i * hop, 0.f, bq);
    };
    if (NV == 1) weights_post(0), weights_pre(0);
    Quad<T> qx[NV], qy[NV], qg[NV];
    auto request = [&](int64_t row) {
        const bool live = row < a.n;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int rest = live ? left - i * hop : 0;
            const int64_t k = c0 + c + i * hop;
            if (y) qy[i] = quad_load<T, VEC>(y + row * a.y_ld + k, step, rest);
            if (gate) qg[i] = quad_load<T, VEC>(gate + row * a.gate_ld + k, step, rest);
            if (x) qx[i] = quad_load<T, VEC>(x + row * a.x_ld + k, step, rest);
        }
    };
    request(at.row);
    const int64_t rounds = (a.n + a.lanes_rows - 1) / a.lanes_rows;   // the same for all lanes
    for (int64_t r = 0; r < rounds; ++r) {
        const int64_t row = at.row + r * a.lanes_rows;
        const bool live = row < a.n;
        float v[NV][4], t[NV][4], gt[NV][4];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (x)
                qx[i].get(v[i]);
            else
                v[i][0] = v[i][1] = v[i][2] = v[i][3] = 0.f;
            if (y) qy[i].get(t[i]);
            if (gate) qg[i].get(gt[i]);
        }
        if (r + 1 < rounds) request(row + a.lanes_rows);
        if (y) {
            float sum[1] = {0.f}, mean = 0.f;
            if (a.layer) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j * (VEC ? 1 : step) < left - i * hop) sum[0] += t[i][j];
                group_sum<L>(sum, smem, turn);
                mean = sum[0] * inv_w;
                sum[0] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    t[i][j] -= mean;
                    if (j * (VEC ? 1 : step) < left - i * hop) sum[0] = fmaf(t[i][j], t[i][j], sum[0]);
                }
            group_sum<L>(sum, smem, turn);
            const float ry = rsqrtf(fmaf(sum[0], inv_w, a.eps));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (NV > 1) weights_post(i);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float b = fmaf(t[i][j] * ry, wp[j], bp[j]);
                    if (gate) b *= sigmoid(gt[i][j]);
                    v[i][j] = fmaf(a.s, b, v[i][j]);
                }
            }
        }
        if (h && live)
#pragma unroll
            for (int i = 0; i < NV; ++i) quad_store<T, VEC>(h + row * a.h_ld + c0 + c + i * hop, step, left - i * hop, v[i]);
        if (!u) continue;
        float sum[1] = {0.f}, mean = 0.f;
        if (a.layer) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j * (VEC ? 1 : step) < left - i * hop) sum[0] += v[i][j];
            group_sum<L>(sum, smem, turn);
            mean = sum[0] * inv_w;
            sum[0] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[i][j] -= mean;
                if (j * (VEC ? 1 : step) < left - i * hop) sum[0] = fmaf(v[i][j], v[i][j], sum[0]);
            }
        group_sum<L>(sum, smem, turn);
        const float rh = rsqrtf(fmaf(sum[0], inv_w, a.eps));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (NV > 1) weights_pre(i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = fmaf(v[i][j] * rh, wq[j], bq[j]);
            if (live) quad_store<T, VEC>(u + row * a.u_ld + c0 + c + i * hop, step, left - i * hop, v[i]);
        }
    }
}

// Bound by HBM as well: y, gate, h, dh and du are read once, dx, dy and dgate written once.  The sums over a slice are
// taken together as far as they can be: (means), then squares of h and y with the products of du w_pre, then the
// products of dt w_post.  The columns' sums over the rows stay in registers until the end.
template <typename T, bool VEC, int L, int NV>
__global__ void __launch_bounds__(L ? 256 : NV == 1 ? 1024 : 1024) norm_backward_kernel(const NormArgs a, const T* y, const T* gate, const T* h,
                                                                                     const float* dh, const float* du, float* dx,
                                                                                     float* dy, float* dgate) {
    __shared__ float smem[2][kMaxNormWarps][4];
    int turn = 0;
    const Place<L> at(a);
    const int lanes = L ? L : blockDim.x;
    const int c0 = at.slice * a.w, c = VEC ? 4 * at.lane : at.lane, step = lanes, hop = 4 * lanes;
    const float inv_w = 1.f / (float)a.w;
    const int left = at.idle ? 0 : a.w - c;
    float wp[4], bp[4], wq[4];
    auto weights = [&](int i) {
        vector_load<VEC>(a.w_post ? a.w_post + c0 + c + i * hop : nullptr, step, left - i * hop, 1.f, wp);
        vector_load<VEC>(a.b_post ? a.b_post + c0 + c + i * hop : nullptr, step, left - i * hop, 0.f, bp);
        vector_load<VEC>(a.w_pre ? a.w_pre + c0 + c + i * hop : nullptr, step, left - i * hop, 1.f, wq);
    };
    if (NV == 1) weights(0);
    float acc[4][NV][4];   // dw_post, db_post, dw_pre, db_pre
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[k][i][j] = 0.f;
    Quad<T> qy[NV], qg[NV], qh[NV];
    Quad<float> qd[NV], qu[NV];
    auto request = [&](int64_t row) {
        const bool live = row < a.n;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int rest = live ? left - i * hop : 0;
            const int64_t k = c0 + c + i * hop;
            if (du) qh[i] = quad_load<T, VEC>(h + row * a.h_ld + k, step, rest);
            if (du) qu[i] = quad_load<float, VEC>(du + row * a.du_ld + k, step, rest);
            if (y) qy[i] = quad_load<T, VEC>(y + row * a.y_ld + k, step, rest);
            if (dh) qd[i] = quad_load<float, VEC>(dh + row * a.dh_ld + k, step, rest);
            if (gate) qg[i] = quad_load<T, VEC>(gate + row * a.gate_ld + k, step, rest);
        }
    };
    auto inside = [&](int i, int j) { return j * (VEC ? 1 : step) < left - i * hop; };
    request(at.row);
    const int64_t rounds = (a.n + a.lanes_rows - 1) / a.lanes_rows;
    for (int64_t r = 0; r < rounds; ++r) {
        const int64_t row = at.row + r * a.lanes_rows;
        const bool live = row < a.n && !at.idle;
        float hv[NV][4], uv[NV][4], yv[NV][4], d[NV][4], gv[NV][4];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) hv[i][j] = uv[i][j] = yv[i][j] = d[i][j] = gv[i][j] = 0.f;
            if (du) qh[i].get(hv[i]), qu[i].get(uv[i]);
            if (y) qy[i].get(yv[i]);
            if (dh) qd[i].get(d[i]);
            if (gate) qg[i].get(gv[i]);
        }
        if (r + 1 < rounds) request(row + a.lanes_rows);
        if (a.layer) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (inside(i, j)) m[0] += hv[i][j], m[1] += yv[i][j];
            group_sum<L>(m, smem, turn);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) hv[i][j] -= m[0] * inv_w, yv[i][j] -= m[1] * inv_w;
        }
        float q[4] = {0.f, 0.f, 0.f, 0.f};   // squares of h and y, sum of du w_pre, of its product with h
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (NV > 1) weights(i);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (inside(i, j)) {
                    const float g = uv[i][j] * wq[j];
                    q[0] = fmaf(hv[i][j], hv[i][j], q[0]);
                    q[1] = fmaf(yv[i][j], yv[i][j], q[1]);
                    q[2] += g;
                    q[3] = fmaf(g, hv[i][j], q[3]);
                }
        }
        group_sum<L>(q, smem, turn);
        const float rh = rsqrtf(fmaf(q[0], inv_w, a.eps)), ry = rsqrtf(fmaf(q[1], inv_w, a.eps));
        const float mg = a.layer ? q[2] * inv_w : 0.f, mgh = q[3] * inv_w * rh;
        float z[2] = {0.f, 0.f};             // sum of dt w_post, of its product with y
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (NV > 1) weights(i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (du) {
                    const float hhat = hv[i][j] * rh;
                    d[i][j] = fmaf(rh, uv[i][j] * wq[j] - mg - hhat * mgh, d[i][j]);
                    if (live && inside(i, j)) {
                        acc[2][i][j] = fmaf(uv[i][j], hhat, acc[2][i][j]);
                        acc[3][i][j] += uv[i][j];
                    }
                }
                if (y) {
                    // sigmoid and its slope e / (1 + e)^2 from e = e^-|g|: neither cancels
                    float open = 1.f, slope = 0.f;
                    if (gate) {
                        const float e = __expf(-fabsf(gv[i][j])), f = __fdividef(1.f, 1.f + e);
                        open = gv[i][j] >= 0.f ? f : e * f;
                        slope = e * f * f;
                        if (gv[i][j] != gv[i][j]) open = slope = gv[i][j];
                    }
                    const float ds = d[i][j] * a.s, yhat = yv[i][j] * ry, dt = ds * open;
                    gv[i][j] = ds * slope * fmaf(yhat, wp[j], bp[j]);
                    uv[i][j] = dt * wp[j];
                    if (inside(i, j)) {
                        z[0] += uv[i][j];
                        z[1] = fmaf(uv[i][j], yv[i][j], z[1]);
                        if (live) {
                            acc[0][i][j] = fmaf(dt, yhat, acc[0][i][j]);
                            acc[1][i][j] += dt;
                        }
                    }
                }
            }
            const int64_t k = c0 + c + i * hop;
            if (dx && live) quad_store<float, VEC>(dx + row * a.dx_ld + k, step, left - i * hop, d[i]);
            if (dgate && live) quad_store<float, VEC>(dgate + row * a.dgate_ld + k, step, left - i * hop, gv[i]);
        }
        if (!dy) continue;
        group_sum<L>(z, smem, turn);
        const float mt = a.layer ? z[0] * inv_w : 0.f, mty = z[1] * inv_w * ry;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) yv[i][j] = ry * (uv[i][j] - mt - yv[i][j] * ry * mty);
            if (live) quad_store<float, VEC>(dy + row * a.dy_ld + c0 + c + i * hop, step, left - i * hop, yv[i]);
        }
    }
    if (!a.partial) return;
    const int cols = a.p * a.w;
    if (L && a.whole_rows) {
        // the CTA's groups of one slice lie p apart: their sums are added in order, and one partial row is left
        __shared__ float sums[256][4];
        const int per_slice = a.p * (L ? L : 1);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[threadIdx.x][j] = acc[k][0][j];
            __syncthreads();
            if ((int)threadIdx.x < per_slice) {
                float t[4] = {0.f, 0.f, 0.f, 0.f};
                for (int o = threadIdx.x; o < 256; o += per_slice)
#pragma unroll
                    for (int j = 0; j < 4; ++j) t[j] += sums[o][j];
                float* out = a.partial + ((int64_t)blockIdx.x * 4 + k) * cols + c0 + c;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (inside(0, j)) out[j * (VEC ? 1 : step)] = t[j];
            }
        }
        return;
    }
    if (at.idle) return;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (inside(i, j)) a.partial[(at.partial_row * 4 + k) * cols + c0 + c + i * hop + j * (VEC ? 1 : step)] = acc[k][i][j];
}

// partial rows -> column sums: 32 columns per CTA, 32 warps that take every 32nd row, then the warps in order
__global__ void __launch_bounds__(1024) norm_join_kernel(int64_t rows, int cols, const float* partial, float* dw_post, float* db_post,
                                                         float* dw_pre, float* db_pre) {
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, k = blockIdx.y;
    float* out = k == 0 ? dw_post : k == 1 ? db_post : k == 2 ? dw_pre : db_pre;
    if (!out) return;
    const int c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < cols)
#pragma unroll 8
        for (int64_t r = g; r < rows; r += 32) s += partial[(r * 4 + k) * cols + c];
    part[g][lane] = s;
    __syncthreads();
    // warp g adds up column g, so that 32 sums run at once
    float t = part[lane][g];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (lane == 0 && blockIdx.x * 32 + g < cols) out[blockIdx.x * 32 + g] = t;
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

// How a call is cut: lanes per slice row (0: a CTA per slice row), quads per lane, threads and CTAs.
constexpr int kSMs = 148;
struct NormPlan {
    int lanes, quads, threads;
    int64_t ctas, lanes_rows;
    int whole_rows;
    int64_t partial_rows;
};
NormPlan norm_plan(const slicegcn_residual_norm_desc* d, bool backward) {
    NormPlan p;
    const int need = (d->h_s + 3) / 4;   // quads per slice row
    p.quads = 1;
    p.lanes = 1;
    while (p.lanes < 32 && p.lanes < need) p.lanes *= 2;
    p.threads = 256;
    if (need > 32) {
        if (!backward && need <= 256) {
            // a warp per slice row, up to eight quads per lane: no barriers
            while (p.quads * 32 < need) p.quads *= 2;
        } else {
            p.lanes = 0;
            // the gradient keeps four column sums per column in registers: few columns per thread
            const int per = backward ? 1024 : 256;
            while (p.quads < 4 && need > per * p.quads) p.quads *= 2;
            p.threads = ((need + p.quads - 1) / p.quads + 31) / 32 * 32;
        }
    }
    const int groups = p.lanes ? p.threads / p.lanes : 1;   // per CTA
    const int64_t items = d->n * d->num_slices;
    const int64_t resident = (backward ? 2 : 8) * kSMs * std::max(1, 256 / p.threads);
    int64_t ctas = std::min((items + groups - 1) / groups, resident);
    p.ctas = std::max<int64_t>(ctas, (d->num_slices + groups - 1) / groups);   // at least one row at a time
    p.lanes_rows = p.ctas * groups / d->num_slices;
    p.whole_rows = p.lanes && p.quads == 1 && groups % d->num_slices == 0;
    p.partial_rows = p.whole_rows ? p.ctas : p.lanes_rows;
    return p;
}

template <typename T>
struct ForwardCall {
    const NormPlan& pl;
    const NormArgs& a;
    const T *x, *y, *gate;
    T *h, *u;
    cudaStream_t st;
    template <bool VEC, int L, int NV>
    void go() const { norm_forward_kernel<T, VEC, L, NV><<<(unsigned)pl.ctas, pl.threads, 0, st>>>(a, x, y, gate, h, u); }
    template <bool VEC>
    void pick() const {
        switch (pl.lanes) {
            case 0: pl.quads == 1 ? go<VEC, 0, 1>() : pl.quads == 2 ? go<VEC, 0, 2>() : go<VEC, 0, 4>(); break;
            case 1: go<VEC, 1, 1>(); break;
            case 2: go<VEC, 2, 1>(); break;
            case 4: go<VEC, 4, 1>(); break;
            case 8: go<VEC, 8, 1>(); break;
            case 16: go<VEC, 16, 1>(); break;
            default: pl.quads == 1 ? go<VEC, 32, 1>() : pl.quads == 2 ? go<VEC, 32, 2>() : pl.quads == 4 ? go<VEC, 32, 4>() : go<VEC, 32, 8>(); break;
        }
    }
};

template <typename T>
struct BackwardCall {
    const NormPlan& pl;
    const NormArgs& a;
    const T *y, *gate, *h;
    const float *dh, *du;
    float *dx, *dy, *dgate;
    cudaStream_t st;
    template <bool VEC, int L, int NV>
    void go() const { norm_backward_kernel<T, VEC, L, NV><<<(unsigned)pl.ctas, pl.threads, 0, st>>>(a, y, gate, h, dh, du, dx, dy, dgate); }
    template <bool VEC>
    void pick() const {
        switch (pl.lanes) {
            case 0: pl.quads == 1 ? go<VEC, 0, 1>() : pl.quads == 2 ? go<VEC, 0, 2>() : go<VEC, 0, 4>(); break;
            case 1: go<VEC, 1, 1>(); break;
            case 2: go<VEC, 2, 1>(); break;
            case 4: go<VEC, 4, 1>(); break;
            case 8: go<VEC, 8, 1>(); break;
            case 16: go<VEC, 16, 1>(); break;
            default: go<VEC, 32, 1>(); break;
        }
    }
};

// four elements at a time: every matrix that is given allows it
struct VecCheck {
    bool ok;
    explicit VecCheck(const slicegcn_residual_norm_desc* d) : ok(d->num_slices == 1 || d->h_s % 4 == 0) {}
    VecCheck& with(const void* p, int64_t ld, int esz) {
        if (p) ok = ok && ld % 4 == 0 && (uintptr_t)p % (4 * esz) == 0;
        return *this;
    }
};

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
    NormArgs a = make_args(d);
    const NormPlan pl = norm_plan(d, false);
    a.lanes_rows = pl.lanes_rows;
    cudaStream_t st = (cudaStream_t)stream;
    const bool vec = VecCheck(d).with(x, d->x_ld, esz).with(y, d->y_ld, esz).with(gate, d->gate_ld, esz).with(h, d->h_ld, esz).with(u, d->u_ld, esz).ok;
    if (d->dtype == SLICEGCN_BF16) {
        using T = __nv_bfloat16;
        const ForwardCall<T> call{pl, a, (const T*)x, (const T*)y, (const T*)gate, (T*)h, (T*)u, st};
        vec ? call.template pick<true>() : call.template pick<false>();
    } else {
        using T = float;
        const ForwardCall<T> call{pl, a, (const T*)x, (const T*)y, (const T*)gate, (T*)h, (T*)u, st};
        vec ? call.template pick<true>() : call.template pick<false>();
    }
    SGCN_LAUNCH_CHECK();
    count_launch();
    return SLICEGCN_OK;
}

slicegcn_status_t slicegcn_residual_norm_workspace_bytes(const slicegcn_residual_norm_desc* d, int64_t* bytes) {
    SGCN_TRY(check_desc(d, "residual_norm_workspace_bytes"));
    if (!bytes) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "residual_norm_workspace_bytes: NULL argument");
    *bytes = norm_plan(d, true).partial_rows * 4 * d->num_slices * d->h_s * (int64_t)sizeof(float);
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
    const NormPlan pl = norm_plan(d, true);
    const int cols = d->num_slices * d->h_s;
    const int64_t need = pl.partial_rows * 4 * cols * (int64_t)sizeof(float);
    if (sums && (!workspace || workspace_bytes < need))
        SGCN_FAIL(SLICEGCN_ERR_ALLOC, "%s: workspace too small (%lld < %lld bytes)", who, (long long)workspace_bytes, (long long)need);
    if ((uintptr_t)workspace % 16) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: the workspace is not aligned to 16 bytes", who);
    NormArgs a = make_args(d);
    a.lanes_rows = pl.lanes_rows;
    a.whole_rows = pl.whole_rows;
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    cudaStream_t st = (cudaStream_t)stream;
    if (a.n > 0) {
        const bool vec = VecCheck(d).with(y, d->y_ld, esz).with(gate, d->gate_ld, esz).with(h, d->h_ld, esz).with(dh, d->dh_ld, 4)
                             .with(du, d->du_ld, 4).with(dx, d->dx_ld, 4).with(dy, d->dy_ld, 4).with(dgate, d->dgate_ld, 4).ok;
        if (d->dtype == SLICEGCN_BF16) {
            using T = __nv_bfloat16;
            const BackwardCall<T> call{pl, a, (const T*)y, (const T*)gate, (const T*)h, dh, du, dx, dy, dgate, st};
            vec ? call.template pick<true>() : call.template pick<false>();
        } else {
            using T = float;
            const BackwardCall<T> call{pl, a, (const T*)y, (const T*)gate, (const T*)h, dh, du, dx, dy, dgate, st};
            vec ? call.template pick<true>() : call.template pick<false>();
        }
        SGCN_LAUNCH_CHECK();
        count_launch();
    }
    if (sums) {
        norm_join_kernel<<<dim3((cols + 31) / 32, 4), 1024, 0, st>>>(a.n > 0 ? pl.partial_rows : 0, cols, a.partial, dw_post, db_post, dw_pre, db_pre);
        SGCN_LAUNCH_CHECK();
        count_launch();
    }
    return SLICEGCN_OK;
}

}  // extern "C"
