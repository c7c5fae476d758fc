// AdamW over a list of tensors: one pass over parameters, gradients and states, one launch.
//   g = grad * c,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   param = param (1 - rate wd) - rate / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
// States in 32 bits, or in 8: int8 codes of m and uint8 codes of sqrt(v), a scale each per block of 256 elements.  sqrt(v) instead
// of v, since the update needs no more of v and a linear code of the root reaches 255^2 down in v.
//
// Bound by HBM: 28 bytes an element with 32-bit states (245 M elements in 1,095 us, 6.3 TB/s), 16 with 8-bit ones (fp32 gradients; 2
// more for a bf16 copy), where instructions come before it (95 an element: 245 M with bf16 gradients and copies in 840 us, 4.7
// TB/s).  A warp takes a block of 256 elements, eight per lane, all its loads on their way together: the block's largest
// magnitudes are then one reduction of the warp away, and no shared memory or barrier is needed.
#include <algorithm>
#include <cmath>

#include "common.cuh"

namespace sgcn {
namespace {

constexpr int kBlock = SLICEGCN_ADAMW_BLOCK, kPerLane = kBlock / 32;
constexpr int kSMs = 148;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr float kLeastNormal = 1.17549435e-38f;

struct Entry {
    float* p;
    const void* g;
    void *m, *v;
    float *m_scale, *v_scale;
    __nv_bfloat16* copy;
    int64_t elems;
    int64_t first;   // index of the tensor's first block among the launch's
    int g_bf16, vec, decayed;   // vec: four elements at a time are aligned in every array
};
// A short list travels as a short kernel argument; a long one in several launches.
constexpr int kShortList = 32, kLongList = 256;
template <int N>
struct Table {
    int count;
    int64_t blocks;
    Entry e[N];
};
struct Hyper {
    float beta1, one_minus_beta1, beta2, one_minus_beta2, eps;
    double lr, log_beta1, log_beta2, weight_decay, max_norm;
    const float *grad_norm, *lr_scale;
    int64_t* step;
    int last;        // this launch is the call's last: it advances the step
};

// Element k (of eight) of a lane within its block: two quads where four elements at a time are aligned, else every 32nd.
template <bool VEC>
__device__ __forceinline__ int place(int lane, int k) {
    return VEC ? (k >> 2) * 128 + lane * 4 + (k & 3) : k * 32 + lane;
}

template <bool VEC>
__device__ __forceinline__ void load_f32(const float* t, int lane, int left, float (&x)[kPerLane]) {
    if (VEC) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float4 f = *reinterpret_cast<const float4*>(t + q * 128 + lane * 4);
            x[4 * q] = f.x, x[4 * q + 1] = f.y, x[4 * q + 2] = f.z, x[4 * q + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) x[k] = place<false>(lane, k) < left ? t[place<false>(lane, k)] : 0.f;
    }
}
template <bool VEC>
__device__ __forceinline__ void store_f32(float* t, int lane, int left, const float (&x)[kPerLane]) {
    if (VEC) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
            *reinterpret_cast<float4*>(t + q * 128 + lane * 4) = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
    } else {
#pragma unroll
        for (int k = 0; k < kPerLane; ++k)
            if (place<false>(lane, k) < left) t[place<false>(lane, k)] = x[k];
    }
}
template <bool VEC>
__device__ __forceinline__ void load_bf16(const __nv_bfloat16* t, int lane, int left, float (&x)[kPerLane]) {
    if (VEC) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint2 w = *reinterpret_cast<const uint2*>(t + q * 128 + lane * 4);
            x[4 * q] = __uint_as_float(w.x << 16), x[4 * q + 1] = __uint_as_float(w.x & 0xffff0000u);
            x[4 * q + 2] = __uint_as_float(w.y << 16), x[4 * q + 3] = __uint_as_float(w.y & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) x[k] = place<false>(lane, k) < left ? __bfloat162float(t[place<false>(lane, k)]) : 0.f;
    }
}
template <bool VEC>
__device__ __forceinline__ void store_bf16(__nv_bfloat16* t, int lane, int left, const float (&x)[kPerLane]) {
    if (VEC) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const __nv_bfloat162 a = __floats2bfloat162_rn(x[4 * q], x[4 * q + 1]), b = __floats2bfloat162_rn(x[4 * q + 2], x[4 * q + 3]);
            *reinterpret_cast<uint2*>(t + q * 128 + lane * 4) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
        }
    } else {
#pragma unroll
        for (int k = 0; k < kPerLane; ++k)
            if (place<false>(lane, k) < left) t[place<false>(lane, k)] = __float2bfloat16_rn(x[k]);
    }
}
// Conversions between codes and floats go through the significand of a number whose last bit counts one (or 2^-16): the conversion
// instructions share a unit of an eighth of the rate with roots and quotients.
constexpr float kTwo23 = 8388608.f;
// Codes as they lie in memory, one byte each, in the lowest byte of 2^23's pattern.
template <bool VEC>
__device__ __forceinline__ void load_codes(const uint8_t* t, int lane, int left, uint32_t (&x)[kPerLane]) {
    if (VEC) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(t + q * 128 + lane * 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[4 * q + k] = __byte_perm(w, 0x4B000000u, 0x7650 + k);
        }
    } else {
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) x[k] = 0x4B000000u | (place<false>(lane, k) < left ? t[place<false>(lane, k)] : 0u);
    }
}
template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t* t, int lane, int left, const uint32_t (&x)[kPerLane]) {
    if (VEC) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t lo = __byte_perm(x[4 * q], x[4 * q + 1], 0x0040), hi = __byte_perm(x[4 * q + 2], x[4 * q + 3], 0x0040);
            *reinterpret_cast<uint32_t*>(t + q * 128 + lane * 4) = __byte_perm(lo, hi, 0x5410);
        }
    } else {
#pragma unroll
        for (int k = 0; k < kPerLane; ++k)
            if (place<false>(lane, k) < left) t[place<false>(lane, k)] = (uint8_t)x[k];
    }
}

// Two thresholds of 16 bits each from an element's index and the step.
__device__ __forceinline__ uint32_t thresholds(uint32_t index, uint32_t t_mixed) {
    uint32_t h = index * 0x9E3779B1u + t_mixed;
    h = (h ^ (h >> 15)) * 0x2C1B3C6Du;
    h = (h ^ (h >> 13)) * 0x297A2D39u;
    return h ^ (h >> 16);
}
// Largest magnitude of a block: magnitudes as whole numbers, so that NaN counts as the largest.
__device__ __forceinline__ float block_max(const float (&x)[kPerLane]) {
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) top = max(top, __float_as_uint(x[k]) & 0x7fffffffu);
    return __uint_as_float(__reduce_max_sync(0xffffffffu, top));
}

struct Step {
    float factor;         // of the gradients
    double factor64;      // the same where it lies below the normal numbers, else 0
    float rate, inv_root_corr, decay;
    uint32_t t_mixed;
};

// One block of 256 elements (`left` of them, where it is a tensor's last).  m and v are rounded operation by operation: their
// codes then are a function of the inputs that a plain program reproduces bit for bit.
template <bool Q8, bool VEC>
__device__ __forceinline__ void update_block(const Entry& e, int64_t block, int lane, const Hyper& h, const Step& s) {
    const int64_t at = block * kBlock;
    const int left = (int)min(e.elems - at, (int64_t)kBlock);
    float p[kPerLane], g[kPerLane], m[kPerLane], v[kPerLane];
    uint32_t mc[kPerLane], vc[kPerLane];
    float ms0 = 0.f, vs0 = 0.f;
    load_f32<VEC>(e.p + at, lane, left, p);
    if (Q8) {
        load_codes<VEC>(static_cast<const uint8_t*>(e.m) + at, lane, left, mc);
        load_codes<VEC>(static_cast<const uint8_t*>(e.v) + at, lane, left, vc);
        ms0 = e.m_scale[block], vs0 = e.v_scale[block];
    } else {
        load_f32<VEC>(static_cast<const float*>(e.m) + at, lane, left, m);
        load_f32<VEC>(static_cast<const float*>(e.v) + at, lane, left, v);
    }
    // last, since the two cases' loads are waited for where they meet
    if (e.g_bf16)
        load_bf16<VEC>(static_cast<const __nv_bfloat16*>(e.g) + at, lane, left, g);
    else
        load_f32<VEC>(static_cast<const float*>(e.g) + at, lane, left, g);
    if (Q8) {
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) {
            m[k] = __fmul_rn(__uint_as_float(mc[k] ^ 0x80u) - (kTwo23 + 128.f), ms0);   // a signed code plus 128 is unsigned
            const float root = __fmul_rn(__uint_as_float(vc[k]) - kTwo23, vs0);
            v[k] = __fmul_rn(root, root);
        }
    }
    const float shrink = e.decayed ? s.decay : 1.f;
    if (s.factor64 != 0.0) {
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) g[k] = (float)((double)g[k] * s.factor64);
    } else {
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) g[k] = __fmul_rn(g[k], s.factor);
    }
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
        const float gk = g[k];
        m[k] = __fadd_rn(__fmul_rn(m[k], h.beta1), __fmul_rn(gk, h.one_minus_beta1));
        v[k] = __fadd_rn(__fmul_rn(v[k], h.beta2), __fmul_rn(__fmul_rn(gk, h.one_minus_beta2), gk));
        const float root = __fsqrt_rn(v[k]);
        // the quotient is off by 2 units of the last place, of an update that is small beside the parameter
        p[k] = p[k] * shrink - s.rate * __fdividef(m[k], root * s.inv_root_corr + h.eps);
        if (Q8) v[k] = root;
    }
    store_f32<VEC>(e.p + at, lane, left, p);
    if (e.copy) store_bf16<VEC>(e.copy + at, lane, left, p);
    if (!Q8) {
        store_f32<VEC>(static_cast<float*>(e.m) + at, lane, left, m);
        store_f32<VEC>(static_cast<float*>(e.v) + at, lane, left, v);
        return;
    }
    // elements past the tensor's end were loaded as zeros and stay zeros
    float ms = __fmul_rn(block_max(m), 1.f / 127.f), vs = __fmul_rn(block_max(v), 1.f / 255.f);
    if (ms < kLeastNormal) ms = 0.f;
    if (vs < kLeastNormal) vs = 0.f;
    const float mi = ms > 0.f ? __fdiv_rn(1.f, ms) : 0.f, vi = vs > 0.f ? __fdiv_rn(1.f, vs) : 0.f;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
        const uint32_t u = thresholds((uint32_t)(at + place<VEC>(lane, k)), s.t_mixed);
        // sixteen bits as a fraction: behind the point of a number between 1 and 2
        const float um = __uint_as_float(0x3f800000u | (u & 0xffffu) << 7) - 1.f, uv = __uint_as_float(0x3f800000u | u >> 16 << 7) - 1.f;
        // rounded down by the addition of 2^23 (for either sign: and 2^22); the codes are the sums' lowest bytes
        const float mx = fminf(fmaxf(__fadd_rn(__fmul_rn(m[k], mi), um), -127.f), 127.5f);
        const float vx = fminf(fmaxf(__fadd_rn(__fmul_rn(v[k], vi), uv), 1.f), 255.5f);
        mc[k] = __float_as_uint(__fadd_rd(mx, 1.5f * kTwo23));
        vc[k] = v[k] > 0.f ? __float_as_uint(__fadd_rd(vx, kTwo23)) : 0u;
    }
    store_codes<VEC>(static_cast<uint8_t*>(e.m) + at, lane, left, mc);
    store_codes<VEC>(static_cast<uint8_t*>(e.v) + at, lane, left, vc);
    if (lane == 0) e.m_scale[block] = ms, e.v_scale[block] = vs;
}

template <bool Q8, int N>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table<N> t, const __grid_constant__ Hyper h) {
    __shared__ Step shared;
    __shared__ double corr[2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t step = h.step[0] + 1;
    if (threadIdx.x < 2) corr[threadIdx.x] = -expm1((double)step * (threadIdx.x ? h.log_beta2 : h.log_beta1));   // 1 - beta^t, two lanes side by side
    __syncwarp();
    if (threadIdx.x == 0) {
        const double rate = h.lr * (h.lr_scale ? (double)*h.lr_scale : 1.0);
        double factor = 1.0;
        if (h.grad_norm) {
            const double norm = *h.grad_norm;
            if (norm > h.max_norm && isfinite(norm)) factor = h.max_norm / norm;
        }
        shared.factor = (float)factor;
        shared.factor64 = factor < (double)kLeastNormal ? factor : 0.0;
        shared.rate = (float)(rate / corr[0]);
        shared.inv_root_corr = (float)(1.0 / sqrt(corr[1]));
        shared.decay = (float)(1.0 - rate * h.weight_decay);
        shared.t_mixed = (uint32_t)step * 0x85EBCA6Bu;
    }
    __syncthreads();
    const Step s = shared;
    int k = 0;
    for (int64_t b = (int64_t)blockIdx.x * kWarps + warp; b < t.blocks; b += (int64_t)gridDim.x * kWarps) {
        while (k + 1 < t.count && t.e[k + 1].first <= b) ++k;
        const Entry& e = t.e[k];
        const int64_t at = b - e.first;
        if (e.vec && e.elems - at * kBlock >= kBlock)
            update_block<Q8, true>(e, at, lane, h, s);
        else
            update_block<Q8, false>(e, at, lane, h, s);
    }
    // Every CTA has read the step when its turn at the counter comes; the last one advances it.
    if (h.last) {
        __syncthreads();
        if (threadIdx.x == 0) {
            __threadfence();
            unsigned long long* turns = reinterpret_cast<unsigned long long*>(h.step + 1);
            if (atomicAdd(turns, 1ull) == gridDim.x - 1) {
                h.step[0] = step;
                *turns = 0;
            }
        }
    }
}

template <int N>
slicegcn_status_t run(const slicegcn_adamw_desc* d, int from, int to, Hyper h, cudaStream_t st) {
    Table<N> t;
    t.count = 0;
    t.blocks = 0;
    for (int i = from; i < to; ++i) {
        const int64_t elems = d->elems[i];
        if (elems == 0) continue;
        Entry& e = t.e[t.count++];
        e.p = d->params[i], e.g = d->grads[i], e.m = d->m[i], e.v = d->v[i];
        e.m_scale = d->state_dtype == SLICEGCN_Q8 ? d->m_scale[i] : nullptr;
        e.v_scale = d->state_dtype == SLICEGCN_Q8 ? d->v_scale[i] : nullptr;
        e.copy = d->copies ? static_cast<__nv_bfloat16*>(d->copies[i]) : nullptr;
        e.elems = elems;
        e.first = t.blocks;
        e.g_bf16 = d->grad_dtypes && d->grad_dtypes[i] == SLICEGCN_BF16;
        e.decayed = !d->decayed || d->decayed[i];
        const uintptr_t state = d->state_dtype == SLICEGCN_Q8 ? 4 : 16;
        e.vec = (uintptr_t)e.p % 16 == 0 && (uintptr_t)e.g % (e.g_bf16 ? 8 : 16) == 0 && (uintptr_t)e.m % state == 0 &&
                (uintptr_t)e.v % state == 0 && (uintptr_t)e.copy % 8 == 0;
        t.blocks += (elems + kBlock - 1) / kBlock;
    }
    // an empty launch still advances the step
    const int ctas = (int)std::max<int64_t>(1, std::min<int64_t>((t.blocks + kWarps - 1) / kWarps, 8 * kSMs));
    if (d->state_dtype == SLICEGCN_Q8)
        adamw_kernel<true, N><<<ctas, kThreads, 0, st>>>(t, h);
    else
        adamw_kernel<false, N><<<ctas, kThreads, 0, st>>>(t, h);
    SGCN_LAUNCH_CHECK();
    count_launch();
    return SLICEGCN_OK;
}

slicegcn_status_t check(const slicegcn_adamw_desc* d) {
    if (!d || d->count < 0) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: bad description");
    if (d->count > SLICEGCN_MAX_TENSORS)
        SGCN_FAIL(SLICEGCN_ERR_UNSUPPORTED, "adamw_step: %d tensors, at most %d", d->count, SLICEGCN_MAX_TENSORS);
    if (d->state_dtype != SLICEGCN_F32 && d->state_dtype != SLICEGCN_Q8) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: bad state_dtype");
    const bool q8 = d->state_dtype == SLICEGCN_Q8;
    if (d->count > 0 && (!d->params || !d->grads || !d->m || !d->v || !d->elems || (q8 && (!d->m_scale || !d->v_scale))))
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: a list is NULL");
    if (!(d->lr >= 0) || !std::isfinite(d->lr) || !(d->beta1 >= 0 && d->beta1 < 1) || !(d->beta2 >= 0 && d->beta2 < 1) || !(d->eps > 0) ||
        !std::isfinite(d->eps) || !(d->weight_decay >= 0) || !std::isfinite(d->weight_decay) || !(d->max_norm > 0))
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: bad lr, beta, eps, weight_decay or max_norm");
    if ((uintptr_t)d->lr_scale % 4) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: lr_scale is not aligned");
    for (int i = 0; i < d->count; ++i) {
        if (d->elems[i] < 0) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: tensor %d has a negative size", i);
        const int dt = d->grad_dtypes ? d->grad_dtypes[i] : SLICEGCN_F32;
        if (dt != SLICEGCN_F32 && dt != SLICEGCN_BF16) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: bad gradient dtype of tensor %d", i);
        if (d->elems[i] == 0) continue;
        if (!d->params[i] || !d->grads[i] || !d->m[i] || !d->v[i] || (q8 && (!d->m_scale[i] || !d->v_scale[i])))
            SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: tensor %d is NULL", i);
        uintptr_t bits = (uintptr_t)d->params[i];
        if (!q8) bits |= (uintptr_t)d->m[i] | (uintptr_t)d->v[i];
        if (q8) bits |= (uintptr_t)d->m_scale[i] | (uintptr_t)d->v_scale[i];
        if (bits % 4 || (uintptr_t)d->grads[i] % (dt == SLICEGCN_BF16 ? 2 : 4) || (d->copies && (uintptr_t)d->copies[i] % 2))
            SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: tensor %d is not aligned to its element type", i);
    }
    return SLICEGCN_OK;
}

}  // namespace
}  // namespace sgcn

using namespace sgcn;

extern "C" {

slicegcn_status_t slicegcn_adamw_step(const slicegcn_adamw_desc* d, int64_t* step, const float* grad_norm, void* stream) {
    SGCN_TRY(check(d));
    if (!step || (uintptr_t)step % 8 || (uintptr_t)grad_norm % 4)
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "adamw_step: step is NULL, or step or grad_norm is not aligned");
    Hyper h;
    h.beta1 = (float)d->beta1, h.one_minus_beta1 = (float)(1.0 - d->beta1);
    h.beta2 = (float)d->beta2, h.one_minus_beta2 = (float)(1.0 - d->beta2);
    h.eps = std::max((float)d->eps, kLeastNormal);   // 0 / 0 otherwise, where gradients have been zero
    h.lr = d->lr, h.log_beta1 = std::log(d->beta1), h.log_beta2 = std::log(d->beta2), h.weight_decay = d->weight_decay, h.max_norm = d->max_norm;
    h.grad_norm = grad_norm, h.lr_scale = d->lr_scale;
    h.step = step;
    h.last = 1;
    cudaStream_t st = (cudaStream_t)stream;
    if (d->count <= kShortList) return run<kShortList>(d, 0, d->count, h, st);
    for (int from = 0; from < d->count; from += kLongList) {
        const int to = std::min(from + kLongList, d->count);
        h.last = to == d->count;
        SGCN_TRY(run<kLongList>(d, from, to, h, st));
    }
    return SLICEGCN_OK;
}

}  // extern "C"
