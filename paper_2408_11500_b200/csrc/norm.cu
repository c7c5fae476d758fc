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
#include <type_traits>

#include "common.cuh"

namespace sgcn {
namespace {

struct NormArgs {
    int64_t n;
    int p, w, layer;
    float eps, s;
    int64_t x_ld, y_ld, gate_ld, h_ld, u_ld, dh_ld, du_ld, dx_ld, dy_ld, dgate_ld;
    const float *w_post, *b_post, *w_pre, *b_pre;
    int64_t lanes_rows;   // rows that are worked on at a time
    float* partial;       // gradient: [partial rows][4][p * w] column sums, or NULL when none is asked for
    int whole_rows;       // a CTA's groups cover whole rows: it leaves one partial row, not one per group
};

// ---- E columns of a slice row, neighbouring ones (VEC) or ones that lie L apart -----------------
// VEC needs rows whose slices start on boundaries of E elements and takes 16 bytes of fp32 (E = 4), 8 or 16 of bf16 (E = 4,
// 8) per access.  The last columns may reach past the slice (one slice of 602 columns): what is read there counts as zero,
// and such a chunk is stored element by element.
template <typename T, int E>
struct Chunk;
template <>
struct Chunk<float, 4> {
    float4 v;
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w; }
    __device__ __forceinline__ void load(const float* p) { v = __ldcs(reinterpret_cast<const float4*>(p)); }
    static __device__ __forceinline__ void store(float* p, const float (&f)[4]) {
        __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    }
    __device__ __forceinline__ void set(int j, float x) {
        if (j == 0) v.x = x;
        if (j == 1) v.y = x;
        if (j == 2) v.z = x;
        if (j == 3) v.w = x;
    }
};
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t o;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(hi), "f"(lo));
    return o;
}
template <int E>
struct Chunk<__nv_bfloat16, E> {
    uint32_t word[E / 2];
    __device__ __forceinline__ void get(float (&f)[E]) const {
#pragma unroll
        for (int k = 0; k < E / 2; ++k) f[2 * k] = __uint_as_float(word[k] << 16), f[2 * k + 1] = __uint_as_float(word[k] & 0xffff0000u);
    }
    __device__ __forceinline__ void take(const uint2& v) { word[0] = v.x, word[1] = v.y; }
    __device__ __forceinline__ void take(const uint4& v) { word[0] = v.x, word[1] = v.y, word[E / 2 - 2] = v.z, word[E / 2 - 1] = v.w; }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        take(__ldcs(reinterpret_cast<const uint2*>(p)));   // four columns; eight go through shared memory
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&f)[E]) {
        if constexpr (E == 8)
            __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])));
        else
            __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])));
    }
    __device__ __forceinline__ void set(int j, __nv_bfloat16 x) {
        const uint32_t b = __bfloat16_as_ushort(x);
        word[j >> 1] = j & 1 ? word[j >> 1] | b << 16 : b;   // even ones come first
    }
};
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Columns of a thread: chunk i holds columns at(i), at(i) + step, ...; `left` columns of the slice follow the first one.
template <bool VEC, int E>
struct Columns {
    int first, hop, step, left;   // of chunk 0; chunks lie `hop` apart
    __device__ __forceinline__ Columns(int lane, int lanes, int w, bool idle)
        : first(VEC ? E * lane : lane), hop(E * lanes), step(VEC ? 1 : lanes), left(idle ? 0 : w - first) {}
    __device__ __forceinline__ int at(int i) const { return first + i * hop; }
    __device__ __forceinline__ bool inside(int i, int j) const { return j * step < left - i * hop; }
    // Loads are unconditional: a condition on each would make the compiler wait for the value where its two cases meet, and
    // nothing would be on its way ahead.  What lies past the slice is read at its start instead, and made zero by keep().
    template <typename T>
    __device__ __forceinline__ void load(Chunk<T, E>& q, const T* row, int i) const {
        if (VEC) {
            q.load(row + (inside(i, 0) ? at(i) : 0));
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) q.set(j, row[inside(i, j) ? at(i) + j * step : 0]);
        }
    }
    __device__ __forceinline__ void keep(float (&f)[E], int i, bool full) const {
        if (full) return;
#pragma unroll
        for (int j = 0; j < E; ++j) f[j] = inside(i, j) ? f[j] : 0.f;
    }
    template <typename T>
    __device__ __forceinline__ void store(T* row, int i, const float (&f)[E], bool ragged) const {
        if (VEC && (!ragged || inside(i, E - 1))) {
            if (inside(i, 0)) Chunk<T, E>::store(row + at(i), f);
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (inside(i, j)) put(row + at(i) + j * step, f[j]);
        }
    }
    // a vector of the columns (weight, bias), `otherwise` where there is none; zero past the slice
    __device__ __forceinline__ void vector(const float* v, int i, float otherwise, float (&f)[E]) const {
#pragma unroll
        for (int j = 0; j < E; ++j) f[j] = !inside(i, j) ? 0.f : v ? __ldg(v + at(i) + j * step) : otherwise;
    }
};
// sums over the L neighbouring lanes of one slice row (every lane of the warp takes part in the shuffles)
template <int L, int K>
__device__ __forceinline__ void group_sum(float (&v)[K]) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
}

// 2^x and 1 / x by the hardware's approximations (a few units in the last place of fp32, denormals as zero): the exact forms
// would make the forward step issue-bound.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float recip_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// These keep a NaN.
__device__ __forceinline__ float at_most(float x, float y) {
    float z;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
__device__ __forceinline__ float at_least(float x, float y) {
    float z;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
// e^-t for -88 <= t <= 128 (zero beyond 87.3).  2^h at h = -t log2 e would be off by the rounding of h, which grows with t
// (5e-7 at 8, 3.5e-6 at 60); what h is short of, -t - h ln 2, is left exactly by one fma and put back by another: e^d = 1 + d.
__device__ __forceinline__ float exp_minus(float t) {
    const float h = -1.44269504f * t, e = exp2_fast(h);
    return fmaf(e, fmaf(h, -0.693147181f, -t), e);
}
// 1 / (1 + e^-g).  In fp32 e^88 is still finite, and what g < -88 makes is zero.  For a result that is rounded to bf16 the plain
// 2^h does: its 4e-6 at most are a thousandth of that rounding, and the four instructions more are 14 % of the time of the gated
// bf16 step (1,047 and 1,197 us for 2,449,029 x 256), which issues instructions at most of the time.
template <typename RESULT>
__device__ __forceinline__ float sigmoid(float g) {
    if (sizeof(RESULT) == 2) return recip_fast(1.f + exp2_fast(-1.44269504f * g));
    return recip_fast(1.f + exp_minus(at_most(at_least(g, -88.f), 128.f)));
}

// An asynchronous copy of one chunk to shared memory, and its values from there.  The thread that copies a chunk is the one
// that reads it, so its own count of finished copies is all the waiting there is.
__device__ __forceinline__ void copy_async16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async8(uint32_t to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
template <int E, typename T>
__device__ __forceinline__ void copy_chunk(uint32_t to, const T* from) {
    if constexpr (E * sizeof(T) == 16)
        copy_async16(to, from);
    else
        copy_async8(to, from);
}
template <typename T, int E>
__device__ __forceinline__ void staged_get(const unsigned char* at, float (&f)[E]) {
    if constexpr (sizeof(T) == 4) {
        const float4 v = *reinterpret_cast<const float4*>(at);
        f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
    } else {
        Chunk<T, E> q;
        if constexpr (E == 8)
            q.take(*reinterpret_cast<const uint4*>(at));
        else
            q.take(*reinterpret_cast<const uint2*>(at));
        q.get(f);
    }
}

// Columns that allow no wide accesses go to shared memory as the aligned 4-byte words that hold them; a bf16 row may start in
// the middle of a word (odd_of: then its element c is element c + 1 there).  Other lanes' words are read as well, so the
// group's lanes meet (__syncwarp) before they read and before the words are replaced.
__device__ __forceinline__ void copy_async4(uint32_t to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
template <typename T>
__device__ __forceinline__ int odd_of(const T* row) {
    return sizeof(T) == 4 ? 0 : (int)((uintptr_t)row >> 1 & 1);
}
// the words of `count` elements, every `lanes`-th by one lane; at most MOST per lane
template <int MOST, typename T>
__device__ __forceinline__ void copy_words(uint32_t to, const T* row, int count, int lane, int lanes) {
    constexpr int PER = 4 / (int)sizeof(T);
    const char* from = reinterpret_cast<const char*>((uintptr_t)row & ~(uintptr_t)3);
    const int words = (count + odd_of(row) + PER - 1) / PER;
#pragma unroll
    for (int q = 0; q < MOST; ++q) {
        const int k = lane + q * lanes;
        if (k < words) copy_async4(to + 4 * k, from + 4 * k);
    }
}
template <typename T, int E>
__device__ __forceinline__ void words_get(const unsigned char* at, int odd, const Columns<false, E>& cols, int i, float (&f)[E]) {
#pragma unroll
    for (int j = 0; j < E; ++j) f[j] = to_float(reinterpret_cast<const T*>(at)[odd + (cols.inside(i, j) ? cols.at(i) + j * cols.step : 0)]);
}

// Where a thread works: its group's slice and first row (then every lanes_rows-th).
template <int L>
struct Place {
    int lane, slice;
    int64_t row;
    bool idle;
    __device__ __forceinline__ Place(const NormArgs& a) {
        lane = (int)threadIdx.x & (L - 1);
        const int64_t g = (int64_t)blockIdx.x * (blockDim.x / L) + threadIdx.x / L;
        row = g / a.p;
        slice = (int)(g - row * a.p);
        idle = row >= a.lanes_rows;
    }
};

// Columns past the slice hold zeros in every array below, so that sums need no tests; a mean is taken off with a factor
// that is zero there.  t becomes t - mean (layer norm); the result is 1 / the root.
template <int E, int L, int NV>
__device__ __forceinline__ float centre_and_scale(float (&t)[NV][E], const float (&in)[NV][E], const NormArgs& a, float inv_w) {
    float sum[1] = {0.f};
    if (a.layer) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < E; ++j) sum[0] += t[i][j];
        group_sum<L>(sum);
        const float mean = sum[0] * inv_w;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < E; ++j) t[i][j] = fmaf(-mean, in[i][j], t[i][j]);
        sum[0] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) sum[0] = fmaf(t[i][j], t[i][j], sum[0]);
    group_sum<L>(sum);
    return rsqrtf(fmaf(sum[0], inv_w, a.eps));
}

// Bound by HBM: x, y and gate are read once, h and u written once.  A slice row lives in the registers of its lanes from
// the first use to the last store, so both norms cost shuffles and no second pass.  What decides is how much is on its way:
// kForwardAhead rows are copied to shared memory ahead.  One chunk per lane (up to 256 columns of bf16, 128 of fp32), whose
// weights stay in registers over all rows.
constexpr int kForwardAhead = 4;
template <typename T, bool VEC, int E>
constexpr int kForwardSlot = VEC ? E * (int)sizeof(T) : 16;   // bytes of shared memory per thread, tensor and row
template <typename T, bool VEC, int E, int L>
__global__ void __launch_bounds__(256, 2) norm_forward_kernel(const NormArgs a, const T* x, const T* y, const T* gate, T* h, T* u) {
    constexpr int S = kForwardAhead, kSlot = kForwardSlot<T, VEC, E>, kTensor = 256 * kSlot;
    extern __shared__ __align__(16) unsigned char ring[];   // [S][x, y, gate][thread] slots
    const Place<L> place(a);
    const Columns<VEC, E> cols(place.lane, L, a.w, place.idle);
    const int c0 = place.slice * a.w;
    const float inv_w = 1.f / (float)a.w;
    const bool ragged = a.w % E != 0, full = a.w == E * L;
    float wp[E], bp[E], wq[E], bq[E], in[1][E];
    const int64_t rounds = (a.n + a.lanes_rows - 1) / a.lanes_rows;   // the same for all lanes
    const int slot = (VEC ? threadIdx.x : threadIdx.x & ~(L - 1)) * kSlot;   // the thread's, or its group's
    const uint32_t ring_u = (uint32_t)__cvta_generic_to_shared(ring) + slot;
    int next_in = 0, next_out = 0;   // ring stages
    auto row_of = [&](int64_t r) { return min(place.row + r * a.lanes_rows, a.n - 1); };   // a row past the end is worked on, and not stored
    auto request = [&](int64_t r) {
        const int64_t at = row_of(r);
        const uint32_t to = ring_u + next_in * 3 * kTensor;
        next_in = next_in + 1 == S ? 0 : next_in + 1;
        if (r < rounds) {
            if constexpr (VEC) {
                const int c = c0 + (cols.inside(0, 0) ? cols.at(0) : 0);
                if (x) copy_chunk<E>(to, x + at * a.x_ld + c);
                if (y) copy_chunk<E>(to + kTensor, y + at * a.y_ld + c);
                if (gate) copy_chunk<E>(to + 2 * kTensor, gate + at * a.gate_ld + c);
            } else {
                if (x) copy_words<4>(to, x + at * a.x_ld + c0, a.w, place.lane, L);
                if (y) copy_words<4>(to + kTensor, y + at * a.y_ld + c0, a.w, place.lane, L);
                if (gate) copy_words<4>(to + 2 * kTensor, gate + at * a.gate_ld + c0, a.w, place.lane, L);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int r = 0; r < S - 1; ++r) request(r);
    cols.vector(a.w_post ? a.w_post + c0 : nullptr, 0, 1.f, wp);
    cols.vector(a.b_post ? a.b_post + c0 : nullptr, 0, 0.f, bp);
    cols.vector(a.w_pre ? a.w_pre + c0 : nullptr, 0, 1.f, wq);
    cols.vector(a.b_pre ? a.b_pre + c0 : nullptr, 0, 0.f, bq);
#pragma unroll
    for (int j = 0; j < E; ++j) in[0][j] = cols.inside(0, j) ? 1.f : 0.f;
    for (int64_t r = 0; r < rounds; ++r) {
        const int64_t row = place.row + r * a.lanes_rows;
        const bool live = row < a.n;
        float v[1][E], t[1][E], gt[E];
#pragma unroll
        for (int j = 0; j < E; ++j) v[0][j] = 0.f;
        if (!VEC) __syncwarp();
        request(r + S - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
        const unsigned char* from = ring + slot + next_out * 3 * kTensor;
        next_out = next_out + 1 == S ? 0 : next_out + 1;
        if constexpr (VEC) {
            if (x) staged_get<T>(from, v[0]);
            if (y) staged_get<T>(from + kTensor, t[0]);
            if (gate) staged_get<T>(from + 2 * kTensor, gt);
        } else {
            __syncwarp();
            const int64_t at = row_of(r);
            if (x) words_get<T>(from, odd_of(x + at * a.x_ld + c0), cols, 0, v[0]);
            if (y) words_get<T>(from + kTensor, odd_of(y + at * a.y_ld + c0), cols, 0, t[0]);
            if (gate) words_get<T>(from + 2 * kTensor, odd_of(gate + at * a.gate_ld + c0), cols, 0, gt);
        }
        cols.keep(v[0], 0, full);
        if (y) {
            cols.keep(t[0], 0, full);
            if (gate) cols.keep(gt, 0, full);
            const float ry = centre_and_scale<E, L, 1>(t, in, a, inv_w);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                float b = fmaf(t[0][j] * ry, wp[j], bp[j]);
                if (gate) b *= sigmoid<T>(gt[j]);
                v[0][j] = fmaf(a.s, b, v[0][j]);
            }
        }
        if (h && live) cols.store(h + row * a.h_ld + c0, 0, v[0], ragged);
        if (!u) continue;
        const float rh = centre_and_scale<E, L, 1>(v, in, a, inv_w);
#pragma unroll
        for (int j = 0; j < E; ++j) v[0][j] = fmaf(v[0][j] * rh, wq[j], bq[j]);
        if (live) cols.store(u + row * a.u_ld + c0, 0, v[0], ragged);
    }
}

// Slices of up to 1024 columns: a warp per slice row, one row ahead in shared memory, as the gradient below does it (see
// there).  The weights lie in shared memory; a CTA works on one slice.
template <typename T, int NV>
struct StagedForward {
    static constexpr int kT = NV * 32 * 4 * (int)sizeof(T) + 16, kRow = 3 * kT, kF = NV * 32 * 16, kVectors = 4 * kF;
    static constexpr int smem(int warps) { return kVectors + warps * 2 * kRow; }
};
constexpr int kForwardWarps = 12;
template <typename T, bool VEC, int NV>
__global__ void __launch_bounds__(kForwardWarps * 32) norm_forward_staged_kernel(const NormArgs a, const T* x, const T* y, const T* gate, T* h, T* u) {
    using S = StagedForward<T, NV>;
    constexpr int E = 4, HF = 512, HT = 32 * E * (int)sizeof(T);
    extern __shared__ __align__(16) unsigned char ring[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int slice = blockIdx.x % a.p;
    const int64_t first = (int64_t)(blockIdx.x / a.p) * warps + warp;             // then every lanes_rows-th row
    const int c0 = slice * a.w;
    const Columns<VEC, E> cols(lane, 32, a.w, false);
    const bool ragged = a.w % E != 0;
    const float inv_w = 1.f / (float)a.w;
    unsigned char* mine = ring + S::kVectors + warp * 2 * S::kRow;
    const uint32_t mine_u = (uint32_t)__cvta_generic_to_shared(ring) + S::kVectors + warp * 2 * S::kRow;
    const unsigned char* vectors = ring + lane * 16;
    if (warp == 0)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const float* from[4] = {a.w_post, a.b_post, a.w_pre, a.b_pre};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float f[E];
                cols.vector(from[k] ? from[k] + c0 : nullptr, i, k & 1 ? 0.f : 1.f, f);
                *reinterpret_cast<float4*>(ring + lane * 16 + i * HF + k * S::kF) = make_float4(f[0], f[1], f[2], f[3]);
            }
        }
    __syncthreads();
    auto copy = [&](uint32_t to, const T* row) {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (cols.inside(i, 0)) copy_chunk<E>(to + (i * 32 + lane) * E * (int)sizeof(T), row + cols.at(i));
        } else {
            copy_words<NV * (int)sizeof(T) + 1>(to, row, a.w, lane, 32);
        }
    };
    auto request = [&](int64_t row, int buf) {
        if (row < a.n) {
            const uint32_t to = mine_u + buf * S::kRow;
            if (x) copy(to, x + row * a.x_ld + c0);
            if (y) copy(to + S::kT, y + row * a.y_ld + c0);
            if (gate) copy(to + 2 * S::kT, gate + row * a.gate_ld + c0);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // chunk i of a staged row; what lies past the slice becomes zero
    auto get = [&](const unsigned char* at, int odd, int i, float(&f)[E]) {
        if constexpr (VEC)
            staged_get<T>(at + i * HT + lane * E * (int)sizeof(T), f);
        else
            words_get<T>(at, odd, cols, i, f);
        if (a.w < 128 * (i + 1)) cols.keep(f, i, false);
    };
    float in[NV][E];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) in[i][j] = cols.inside(i, j) ? 1.f : 0.f;
    request(first, 0);
    int buf = 0;
    for (int64_t row = first; row < a.n; row += a.lanes_rows, buf ^= 1) {
        if (!VEC) __syncwarp();
        request(row + a.lanes_rows, buf ^ 1);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        if (!VEC) __syncwarp();
        const unsigned char* at = mine + buf * S::kRow;
        float v[NV][E];
        if (y) {
            const int odd = odd_of(y + row * a.y_ld + c0);
            float t[NV][E];
#pragma unroll
            for (int i = 0; i < NV; ++i) get(at + S::kT, odd, i, t[i]);
            const float ry = centre_and_scale<E, 32, NV>(t, in, a, inv_w);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float wp[E], bp[E], gt[E];
                staged_get<float>(vectors + i * HF, wp), staged_get<float>(vectors + S::kF + i * HF, bp);
#pragma unroll
                for (int j = 0; j < E; ++j) v[i][j] = fmaf(t[i][j] * ry, wp[j], bp[j]) * a.s;
                if (gate) {
                    get(at + 2 * S::kT, odd_of(gate + row * a.gate_ld + c0), i, gt);
#pragma unroll
                    for (int j = 0; j < E; ++j) v[i][j] *= sigmoid<T>(gt[j]);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < E; ++j) v[i][j] = 0.f;
        }
        if (x) {
            const int odd = odd_of(x + row * a.x_ld + c0);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float f[E];
                get(at, odd, i, f);
#pragma unroll
                for (int j = 0; j < E; ++j) v[i][j] += f[j];
            }
        }
        if (h)
#pragma unroll
            for (int i = 0; i < NV; ++i) cols.store(h + row * a.h_ld + c0, i, v[i], ragged);
        if (!u) continue;
        const float rh = centre_and_scale<E, 32, NV>(v, in, a, inv_w);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float wq[E], bq[E];
            staged_get<float>(vectors + 2 * S::kF + i * HF, wq), staged_get<float>(vectors + 3 * S::kF + i * HF, bq);
#pragma unroll
            for (int j = 0; j < E; ++j) v[i][j] = fmaf(v[i][j] * rh, wq[j], bq[j]);
            cols.store(u + row * a.u_ld + c0, i, v[i], ragged);
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// sums over a CTA of kWideThreads, the same order every time; two buffers in turn, so that one barrier per sum is enough
constexpr int kWideThreads = 256;
template <int K>
__device__ __forceinline__ void cta_sum(float (&v)[K], float (*buf)[kWideThreads / 32][K]) {
    group_sum<32>(v);
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) (*buf)[threadIdx.x >> 5][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k] = 0.f;
#pragma unroll
        for (int o = 0; o < kWideThreads / 32; ++o) v[k] += (*buf)[o][k];
    }
}

// Slices of more than 1024 columns: a CTA per slice row, which it keeps in shared memory in fp32 between the passes (every
// thread reads back its own columns), so that x, y and gate are read once here too.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kWideThreads) norm_forward_wide_kernel(const NormArgs a, const T* x, const T* y, const T* gate, T* h, T* u) {
    constexpr int E = 4;
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ float sums[4][kWideThreads / 32][1];   // one for each sum
    float* const kept = reinterpret_cast<float*>(ring);
    const int64_t item = blockIdx.x, row = item / a.p;
    const int c0 = (int)(item - row * a.p) * a.w;
    const Columns<VEC, E> cols(threadIdx.x, kWideThreads, a.w, false);
    const bool ragged = a.w % E != 0;
    const float inv_w = 1.f / (float)a.w;
    const int chunks = (a.w + E * kWideThreads - 1) / (E * kWideThreads);
    auto get = [&](const T* from, int i, float(&f)[E]) {
        Chunk<T, E> q;
        cols.load(q, from, i);
        q.get(f);
        cols.keep(f, i, false);
    };
    // slots [chunk][j][thread] of shared memory
    auto keep = [&](int i, const float(&f)[E]) {
#pragma unroll
        for (int j = 0; j < E; ++j) kept[(i * E + j) * kWideThreads + threadIdx.x] = f[j];
    };
    auto kept_at = [&](int i, float(&f)[E]) {
#pragma unroll
        for (int j = 0; j < E; ++j) f[j] = kept[(i * E + j) * kWideThreads + threadIdx.x];
    };
    // sum of the squares about the mean (of the kept row) -> 1 / the root; the mean comes back in `mean`
    auto scale_of = [&](float total, float& mean, float(*means)[kWideThreads / 32][1], float(*squares)[kWideThreads / 32][1]) {
        float sum[1] = {total};
        mean = 0.f;
        if (a.layer) {
            cta_sum(sum, means);
            mean = sum[0] * inv_w;
        }
        sum[0] = 0.f;
        for (int i = 0; i < chunks; ++i) {
            float f[E];
            kept_at(i, f);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float t = cols.inside(i, j) ? f[j] - mean : 0.f;
                sum[0] = fmaf(t, t, sum[0]);
            }
        }
        cta_sum(sum, squares);
        return rsqrtf(fmaf(sum[0], inv_w, a.eps));
    };
    float my = 0.f, ry = 0.f;
    if (y) {
        float total = 0.f;
#pragma unroll 4
        for (int i = 0; i < chunks; ++i) {
            float f[E];
            get(y + row * a.y_ld + c0, i, f);
            keep(i, f);
#pragma unroll
            for (int j = 0; j < E; ++j) total += f[j];
        }
        ry = scale_of(total, my, sums + 0, sums + 1);
    }
    float total = 0.f;
#pragma unroll 2
    for (int i = 0; i < chunks; ++i) {   // h may be x: an element is read before it is written, and by the same thread
        float v[E] = {0.f, 0.f, 0.f, 0.f};
        if (x) get(x + row * a.x_ld + c0, i, v);
        if (y) {
            float t[E], g[E], wp[E], bp[E];
            kept_at(i, t);
            if (gate) get(gate + row * a.gate_ld + c0, i, g);
            cols.vector(a.w_post ? a.w_post + c0 : nullptr, i, 1.f, wp);
            cols.vector(a.b_post ? a.b_post + c0 : nullptr, i, 0.f, bp);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                float b = fmaf((t[j] - my) * ry, wp[j], bp[j]);
                if (gate) b *= sigmoid<T>(g[j]);
                v[j] = fmaf(a.s, b, v[j]);
            }
            cols.keep(v, i, false);
        }
        keep(i, v);
#pragma unroll
        for (int j = 0; j < E; ++j) total += v[j];
        if (h) cols.store(h + row * a.h_ld + c0, i, v, ragged);
    }
    if (!u) return;
    float mh;
    const float rh = scale_of(total, mh, sums + 2, sums + 3);
#pragma unroll 2
    for (int i = 0; i < chunks; ++i) {
        float v[E], wq[E], bq[E];
        kept_at(i, v);
        cols.vector(a.w_pre ? a.w_pre + c0 : nullptr, i, 1.f, wq);
        cols.vector(a.b_pre ? a.b_pre + c0 : nullptr, i, 0.f, bq);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = fmaf((v[j] - mh) * rh, wq[j], bq[j]);
        cols.store(u + row * a.u_ld + c0, i, v, ragged);
    }
}

// sigmoid(g) and its slope e / (1 + e)^2 from e = e^-|g|: neither cancels
__device__ __forceinline__ void gate_and_slope(float g, float& open, float& slope) {
    const float e = exp_minus(at_most(fabsf(g), 128.f)), f = recip_fast(1.f + e);
    open = g < 0.f ? e * f : f;
    slope = e * f * f;
}

// Bound by HBM as well: y, gate, h, dh and du are read once, dx, dy and dgate written once.  The sums over a slice are
// taken together as far as they can be: (means), then squares of h and y with the products of du w_pre, then the
// products of dt w_post.  Slices of up to 128 columns: four per lane, whose sums over the rows stay in registers until the
// end, as do the weights; kBackwardAhead rows are copied to shared memory ahead.
constexpr int kBackwardAhead = 3;
// bytes of a CTA's chunks of one row each: dh, du, then h, y, gate
template <typename T, bool VEC>
struct BackwardRing {
    static constexpr int kSlot = VEC ? 4 * (int)sizeof(T) : 16, kF = 256 * 16, kT = 256 * kSlot, kStage = 2 * kF + 3 * kT;
};
template <typename T, bool VEC, int L>
__global__ void __launch_bounds__(256, 2) norm_backward_kernel(const NormArgs a, const T* y, const T* gate, const T* h, const float* dh,
                                                               const float* du, float* dx, float* dy, float* dgate) {
    cudaTriggerProgrammaticLaunchCompletion();
    using R = BackwardRing<T, VEC>;
    constexpr int E = 4, S = kBackwardAhead;
    extern __shared__ __align__(16) unsigned char ring[];
    const Place<L> place(a);
    const Columns<VEC, E> cols(place.lane, L, a.w, place.idle);
    const int c0 = place.slice * a.w;
    const float inv_w = 1.f / (float)a.w;
    const bool ragged = a.w % E != 0, full = a.w == E * L;
    const int all = a.p * a.w;
    const int64_t rounds = (a.n + a.lanes_rows - 1) / a.lanes_rows;
    const uint32_t ring_u = (uint32_t)__cvta_generic_to_shared(ring);
    const int owner = VEC ? threadIdx.x : threadIdx.x & ~(L - 1);   // whose slots: the thread's, or its group's
    const int at_f = owner * 16, at_t = 2 * R::kF + owner * R::kSlot;
    int next_in = 0, next_out = 0;   // ring stages
    auto row_of = [&](int64_t r) { return min(place.row + r * a.lanes_rows, a.n - 1); };   // a row past the end is worked on, and not kept
    auto request = [&](int64_t r) {
        const int64_t at = row_of(r);
        const uint32_t to = ring_u + next_in * R::kStage;
        next_in = next_in + 1 == S ? 0 : next_in + 1;
        if (r < rounds) {
            auto copy = [&](uint32_t slot, const auto* row) {
                if constexpr (VEC)
                    copy_chunk<E>(slot, row + (cols.inside(0, 0) ? cols.at(0) : 0));
                else
                    copy_words<4>(slot, row, a.w, place.lane, L);
            };
            if (du) copy(to + at_t, h + at * a.h_ld + c0);
            if (du) copy(to + R::kF + at_f, du + at * a.du_ld + c0);
            if (y) copy(to + at_t + R::kT, y + at * a.y_ld + c0);
            if (dh) copy(to + at_f, dh + at * a.dh_ld + c0);
            if (gate) copy(to + at_t + 2 * R::kT, gate + at * a.gate_ld + c0);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int r = 0; r < S - 1; ++r) request(r);
    float wp[E], bp[E], wq[E], in[E];
    cols.vector(a.w_post ? a.w_post + c0 : nullptr, 0, 1.f, wp);
    cols.vector(a.b_post ? a.b_post + c0 : nullptr, 0, 0.f, bp);
    cols.vector(a.w_pre ? a.w_pre + c0 : nullptr, 0, 1.f, wq);
    float acc[4][E];   // dw_post, db_post, dw_pre, db_pre
#pragma unroll
    for (int j = 0; j < E; ++j) {
        in[j] = cols.inside(0, j) ? 1.f : 0.f;
        acc[0][j] = acc[1][j] = acc[2][j] = acc[3][j] = 0.f;
    }
    for (int64_t r = 0; r < rounds; ++r) {
        const int64_t row = place.row + r * a.lanes_rows;
        const bool live = row < a.n && !place.idle;
        float hv[E], uv[E], yv[E], d[E], gv[E];
#pragma unroll
        for (int j = 0; j < E; ++j) hv[j] = uv[j] = yv[j] = d[j] = gv[j] = 0.f;
        if (!VEC) __syncwarp();
        request(r + S - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
        const unsigned char* from = ring + next_out * R::kStage;
        next_out = next_out + 1 == S ? 0 : next_out + 1;
        if constexpr (VEC) {
            if (du) staged_get<T>(from + at_t, hv), staged_get<float>(from + R::kF + at_f, uv);
            if (y) staged_get<T>(from + at_t + R::kT, yv);
            if (dh) staged_get<float>(from + at_f, d);
            if (gate) staged_get<T>(from + at_t + 2 * R::kT, gv);
        } else {
            __syncwarp();
            const int64_t at = row_of(r);
            if (du) words_get<T>(from + at_t, odd_of(h + at * a.h_ld + c0), cols, 0, hv), words_get<float>(from + R::kF + at_f, 0, cols, 0, uv);
            if (y) words_get<T>(from + at_t + R::kT, odd_of(y + at * a.y_ld + c0), cols, 0, yv);
            if (dh) words_get<float>(from + at_f, 0, cols, 0, d);
            if (gate) words_get<T>(from + at_t + 2 * R::kT, odd_of(gate + at * a.gate_ld + c0), cols, 0, gv);
        }
        cols.keep(hv, 0, full), cols.keep(uv, 0, full), cols.keep(yv, 0, full), cols.keep(d, 0, full), cols.keep(gv, 0, full);
        if (a.layer) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int j = 0; j < E; ++j) m[0] += hv[j], m[1] += yv[j];
            group_sum<L>(m);
            m[0] *= inv_w, m[1] *= inv_w;
#pragma unroll
            for (int j = 0; j < E; ++j) hv[j] = fmaf(-m[0], in[j], hv[j]), yv[j] = fmaf(-m[1], in[j], yv[j]);
        }
        float q[4] = {0.f, 0.f, 0.f, 0.f};   // squares of h and y, sum of du w_pre, of its product with h
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float g = uv[j] * wq[j];
            q[0] = fmaf(hv[j], hv[j], q[0]);
            q[1] = fmaf(yv[j], yv[j], q[1]);
            q[2] += g;
            q[3] = fmaf(g, hv[j], q[3]);
        }
        group_sum<L>(q);
        const float rh = rsqrtf(fmaf(q[0], inv_w, a.eps)), ry = rsqrtf(fmaf(q[1], inv_w, a.eps));
        const float mg = a.layer ? q[2] * inv_w : 0.f, mgh = q[3] * inv_w * rh;
        float z[2] = {0.f, 0.f};             // sum of dt w_post, of its product with y
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (du) {
                const float hhat = hv[j] * rh;
                d[j] = fmaf(rh, fmaf(-mg, in[j], uv[j] * wq[j]) - hhat * mgh, d[j]);
                if (live) {
                    acc[2][j] = fmaf(uv[j], hhat, acc[2][j]);
                    acc[3][j] += uv[j];
                }
            }
            if (y) {
                float open = 1.f, slope = 0.f;
                if (gate) gate_and_slope(gv[j], open, slope);
                const float ds = d[j] * a.s, yhat = yv[j] * ry, dt = ds * open;
                gv[j] = ds * slope * fmaf(yhat, wp[j], bp[j]);
                uv[j] = dt * wp[j];
                z[0] += uv[j];
                z[1] = fmaf(uv[j], yv[j], z[1]);
                if (live) {
                    acc[0][j] = fmaf(dt, yhat, acc[0][j]);
                    acc[1][j] += dt;
                }
            }
        }
        if (dx && live) cols.store(dx + row * a.dx_ld + c0, 0, d, ragged);
        if (dgate && live) cols.store(dgate + row * a.dgate_ld + c0, 0, gv, ragged);
        if (!dy) continue;
        group_sum<L>(z);
        const float mt = a.layer ? z[0] * inv_w : 0.f, mty = z[1] * inv_w * ry;
#pragma unroll
        for (int j = 0; j < E; ++j) yv[j] = ry * (uv[j] - mt - yv[j] * ry * mty);
        if (live) cols.store(dy + row * a.dy_ld + c0, 0, yv, ragged);
    }
    if (!a.partial) return;
    if (a.whole_rows) {
        // the CTA's groups of one slice lie p apart: their sums are added in order, and one partial row is left
        __shared__ float sums[256][E];
        const int per_slice = a.p * L;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < E; ++j) sums[threadIdx.x][j] = acc[k][j];
            __syncthreads();
            if ((int)threadIdx.x < per_slice) {
                float t[E] = {0.f, 0.f, 0.f, 0.f};
                for (int o = threadIdx.x; o < 256; o += per_slice)
#pragma unroll
                    for (int j = 0; j < E; ++j) t[j] += sums[o][j];
                float* out = a.partial + ((int64_t)blockIdx.x * 4 + k) * all + c0;
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (cols.inside(0, j)) out[cols.at(0) + j * cols.step] = t[j];
            }
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float* out = a.partial + (place.row * 4 + k) * all + c0;
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (cols.inside(0, j)) out[cols.at(0) + j * cols.step] = acc[k][j];
    }
}

// Slices of 129 to 1024 columns: a warp per slice row, whose five inputs are copied to shared memory one row ahead.  With
// accesses of four elements every lane copies, and reads back, its own columns only (4 lane + 128 i).  No barrier of the
// CTA stands in the loop.  The row is read from shared memory in each of the passes over it, which leaves the registers to the
// columns' sums (BIAS: those of the biases too).  A CTA works on one slice: its warps' sums are added in order at the end.
// What is not given is left in shared memory as values that change nothing (zeros; an infinite gate is an open one).
// Shared memory (two rows per warp) and registers (the sums) bound the warps per SM, so what counts here is instructions per element
// and latency: 232,965 x 602 bf16, gated, plain norm without biases, moves 5.0-5.4 TB/s (680-730 us where the bytes take 557).
// With biases the sums take twice the registers and part of them spills (up to 500 bytes a thread with accesses of four
// elements, 850 without): 1.5 times the time at 602 columns, 1.9 at 1,024.
template <int NV>
constexpr int staged_warps() { return NV <= 5 ? 12 : 8; }
// bytes of one row of a warp: dh, du in fp32 and y, gate, h in T, 32 lanes x NV chunks each
template <typename T, int NV>
struct Staged {
    static constexpr int kF = NV * 32 * 16, kT = NV * 32 * 4 * (int)sizeof(T) + 16;   // (a bf16 row may start in a word)
    static constexpr int kDh = 0, kDu = kF, kY = 2 * kF, kGate = kY + kT, kH = kGate + kT, kRow = kH + kT;
    static constexpr int kVectors = 3 * NV * 32 * 16;                             // w_post, b_post, w_pre
    static constexpr int smem(int warps) { return kVectors + warps * 2 * kRow; }
};
template <typename T, bool VEC, int NV, bool BIAS, bool LAYER>
__global__ void __launch_bounds__(staged_warps<NV>() * 32) norm_backward_staged_kernel(const NormArgs a, const T* y, const T* gate, const T* h,
                                                                                       const float* dh, const float* du, float* dx,
                                                                                       float* dy, float* dgate) {
    cudaTriggerProgrammaticLaunchCompletion();
    using S = Staged<T, NV>;
    constexpr int E = 4;
    constexpr int HF = 512, HT = 32 * E * (int)sizeof(T);   // bytes from one chunk of a lane to its next
    extern __shared__ __align__(16) unsigned char stage[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int slice = blockIdx.x % a.p;
    const int64_t first = (int64_t)(blockIdx.x / a.p) * warps + warp;             // then every lanes_rows-th row
    const int c0 = slice * a.w;
    const Columns<VEC, E> cols(lane, 32, a.w, false);
    const bool ragged = a.w % E != 0;
    const float inv_w = 1.f / (float)a.w;
    unsigned char* mine = stage + S::kVectors + warp * 2 * S::kRow;
    const uint32_t mine_u = (uint32_t)__cvta_generic_to_shared(mine);
    const unsigned char* vectors = stage + lane * 16;
    if (warp == 0)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float f[E];
            float4* to = reinterpret_cast<float4*>(stage + lane * 16 + i * HF);
            cols.vector(a.w_post ? a.w_post + c0 : nullptr, i, 1.f, f);
            to[0] = make_float4(f[0], f[1], f[2], f[3]);
            cols.vector(a.b_post ? a.b_post + c0 : nullptr, i, 0.f, f);
            to[NV * 32] = make_float4(f[0], f[1], f[2], f[3]);
            cols.vector(a.w_pre ? a.w_pre + c0 : nullptr, i, 1.f, f);
            to[2 * NV * 32] = make_float4(f[0], f[1], f[2], f[3]);
        }
    {   // columns past the slice are never copied: they stay as they are here
        const uint32_t inf = sizeof(T) == 4 ? 0x7f800000u : 0x7f807f80u;
        for (int k = lane * 16; k < 2 * S::kRow; k += 512) {
            const int in = k < S::kRow ? k : k - S::kRow;
            const uint32_t fill = !gate && in >= S::kGate && in < S::kH ? inf : 0u;
            *reinterpret_cast<uint4*>(mine + k) = make_uint4(fill, fill, fill, fill);
        }
    }
    __syncthreads();
    auto request = [&](int64_t row, int buf) {
        if (row < a.n) {
            const uint32_t to = mine_u + buf * S::kRow;
            auto copy = [&](uint32_t at, const auto* from) {
                using F = typename std::remove_cv<typename std::remove_reference<decltype(*from)>::type>::type;
                if constexpr (VEC) {
#pragma unroll
                    for (int i = 0; i < NV; ++i)
                        if (cols.inside(i, 0)) copy_chunk<E>(at + (i * 32 + lane) * E * (int)sizeof(F), from + cols.at(i));
                } else {
                    copy_words<NV * (int)sizeof(F) + 1>(at, from, a.w, lane, 32);
                }
            };
            if (du) copy(to + S::kH, h + row * a.h_ld + c0);
            if (du) copy(to + S::kDu, du + row * a.du_ld + c0);
            if (y) copy(to + S::kY, y + row * a.y_ld + c0);
            if (dh) copy(to + S::kDh, dh + row * a.dh_ld + c0);
            if (gate) copy(to + S::kGate, gate + row * a.gate_ld + c0);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // zero what a chunk holds past the slice, and what subtracting a mean leaves there; every chunk but the last ones is whole
    auto whole = [&](int i) { return a.w >= 128 * (i + 1); };
    auto store = [&](float* to, int i, const float(&f)[E]) {
        if (VEC && whole(i))
            Chunk<float, E>::store(to + cols.at(i), f);
        else
            cols.store(to, i, f, ragged);
    };
    float acc[BIAS ? 4 : 2][NV][E];   // dw_post, dw_pre, db_post, db_pre
#pragma unroll
    for (int k = 0; k < (BIAS ? 4 : 2); ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < E; ++j) acc[k][i][j] = 0.f;
    request(first, 0);
    int buf = 0;
    for (int64_t row = first; row < a.n; row += a.lanes_rows, buf ^= 1) {
        if (!VEC) __syncwarp();
        request(row + a.lanes_rows, buf ^ 1);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        if (!VEC) __syncwarp();
        const unsigned char* at = mine + buf * S::kRow;
        const int odd_h = du ? odd_of(h + row * a.h_ld + c0) : 0, odd_y = y ? odd_of(y + row * a.y_ld + c0) : 0;
        const int odd_gate = gate ? odd_of(gate + row * a.gate_ld + c0) : 0;
        auto get_t = [&](int tensor, int odd, int i, float(&f)[E]) {
            if constexpr (VEC)
                staged_get<T>(at + tensor + i * HT + lane * E * (int)sizeof(T), f);
            else
                words_get<T>(at + tensor, odd, cols, i, f);
        };
        auto get_f = [&](int tensor, int i, float(&f)[E]) {
            if constexpr (VEC)
                staged_get<float>(at + tensor + i * HF + lane * 16, f);
            else
                words_get<float>(at + tensor, 0, cols, i, f);
        };
        float mh = 0.f, my = 0.f;
        if (LAYER) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float hv[E], yv[E];
                get_t(S::kH, odd_h, i, hv), get_t(S::kY, odd_y, i, yv);
                if (!whole(i)) cols.keep(hv, i, false), cols.keep(yv, i, false);
#pragma unroll
                for (int j = 0; j < E; ++j) m[0] += hv[j], m[1] += yv[j];
            }
            group_sum<32>(m);
            mh = m[0] * inv_w, my = m[1] * inv_w;
        }
        float q[4] = {0.f, 0.f, 0.f, 0.f};   // squares of h and y, sum of du w_pre, of its product with h
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float hv[E], uv[E], yv[E], wq[E];
            get_t(S::kH, odd_h, i, hv);
            get_f(S::kDu, i, uv);
            get_t(S::kY, odd_y, i, yv);
            staged_get<float>(vectors + 2 * S::kF + i * HF, wq);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (LAYER) hv[j] -= mh, yv[j] -= my;
            if (!whole(i)) cols.keep(hv, i, false), cols.keep(yv, i, false), cols.keep(uv, i, false);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float g = uv[j] * wq[j];
                q[0] = fmaf(hv[j], hv[j], q[0]);
                q[1] = fmaf(yv[j], yv[j], q[1]);
                if (LAYER) q[2] += g;
                q[3] = fmaf(g, hv[j], q[3]);
            }
        }
        group_sum<32>(q);
        const float rh = rsqrtf(fmaf(q[0], inv_w, a.eps)), ry = rsqrtf(fmaf(q[1], inv_w, a.eps));
        const float mg = LAYER ? q[2] * inv_w : 0.f, mgh = q[3] * inv_w * rh;
        float t[NV][E], z[2] = {0.f, 0.f};   // dt w_post; its sum, and that of its product with y
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float hv[E], uv[E], yv[E], d[E], gv[E], wp[E], bp[E], wq[E];
            get_t(S::kH, odd_h, i, hv);
            get_f(S::kDu, i, uv);
            get_t(S::kY, odd_y, i, yv);
            get_f(S::kDh, i, d);
            get_t(S::kGate, odd_gate, i, gv);
            staged_get<float>(vectors + i * HF, wp);
            staged_get<float>(vectors + S::kF + i * HF, bp);
            staged_get<float>(vectors + 2 * S::kF + i * HF, wq);
            if (!whole(i)) {
                cols.keep(uv, i, false), cols.keep(d, i, false), cols.keep(yv, i, false);
                cols.keep(gv, i, false), cols.keep(hv, i, false);
            }
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float hhat = (LAYER ? hv[j] - mh : hv[j]) * rh;
                d[j] = fmaf(rh, (LAYER ? fmaf(uv[j], wq[j], -mg) : uv[j] * wq[j]) - hhat * mgh, d[j]);
                acc[1][i][j] = fmaf(uv[j], hhat, acc[1][i][j]);
                if (BIAS) acc[BIAS ? 3 : 1][i][j] += uv[j];
                float open, slope;
                gate_and_slope(gv[j], open, slope);
                const float ds = d[j] * a.s, yc = LAYER ? yv[j] - my : yv[j], yhat = yc * ry, dt = ds * open;
                gv[j] = ds * slope * fmaf(yhat, wp[j], bp[j]);
                t[i][j] = dt * wp[j];              // w_post is zero past the slice
                if (LAYER) z[0] += t[i][j];
                z[1] = fmaf(t[i][j], yc, z[1]);
                acc[0][i][j] = fmaf(dt, yhat, acc[0][i][j]);
                if (BIAS) acc[BIAS ? 2 : 0][i][j] += dt;
            }
            if (dx) store(dx + row * a.dx_ld + c0, i, d);
            if (dgate) store(dgate + row * a.dgate_ld + c0, i, gv);
        }
        if (!dy) continue;
        group_sum<32>(z);
        const float mt = LAYER ? z[0] * inv_w : 0.f, mty = z[1] * inv_w * ry;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float yv[E];
            get_t(S::kY, odd_y, i, yv);
#pragma unroll
            for (int j = 0; j < E; ++j) yv[j] = LAYER ? ry * (t[i][j] - mt - (yv[j] - my) * ry * mty) : ry * (t[i][j] - yv[j] * ry * mty);
            store(dy + row * a.dy_ld + c0, i, yv);
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!a.partial) return;
    const int all = a.p * a.w;
    unsigned char* sums = stage + S::kVectors;   // [warp][columns]
#pragma unroll
    for (int k = 0; k < (BIAS ? 4 : 2); ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < E; ++j) reinterpret_cast<float*>(sums + warp * S::kF)[cols.at(i) + j * cols.step] = acc[k][i][j];
        __syncthreads();
        const int which = BIAS ? (k == 0 ? 0 : k == 1 ? 2 : k == 2 ? 1 : 3) : 2 * k;   // order of the partial rows
        float* out = a.partial + ((int64_t)(blockIdx.x / a.p) * 4 + which) * all + c0;
        for (int c = threadIdx.x; c < a.w; c += blockDim.x) {
            float v = 0.f;
            for (int o = 0; o < warps; ++o) v += *reinterpret_cast<const float*>(sums + o * S::kF + c * 4);
            out[c] = v;
        }
    }
}

// Wider slices.  First a CTA per slice row takes the sums over the row, reading it twice, or three times for the layer norm (from L2
// but for the first time); then every thread applies them to columns of its own for many rows, whose sums it keeps in
// registers.  The second kernel reads everything from HBM again: 20,000 x 4,096 fp32 takes 1.07 ms where the bytes take 400 us.
struct RowStats {
    float mh, rh, mg, mgh, my, ry, mt, mty;
};
template <typename T, bool VEC>
__global__ void __launch_bounds__(kWideThreads) norm_stats_kernel(const NormArgs a, const T* y, const T* gate, const T* h, const float* dh,
                                                         const float* du, RowStats* stats) {
    constexpr int E = 4;
    __shared__ float means[1][kWideThreads / 32][2], squares[1][kWideThreads / 32][4], products[1][kWideThreads / 32][2];
    const int64_t item = blockIdx.x, row = item / a.p;
    const int c0 = (int)(item - row * a.p) * a.w;
    const Columns<VEC, E> cols(threadIdx.x, kWideThreads, a.w, false);
    const float inv_w = 1.f / (float)a.w;
    const int chunks = (a.w + 4 * kWideThreads - 1) / (4 * kWideThreads);
    auto get = [&](auto* from, int i, float(&f)[E]) {
        Chunk<typename std::remove_cv<typename std::remove_pointer<decltype(from)>::type>::type, E> q;
        cols.load(q, from, i);
        q.get(f);
        cols.keep(f, i, false);
    };
    RowStats s{};
    if (a.layer) {
        float m[2] = {0.f, 0.f};
        for (int i = 0; i < chunks; ++i) {
            float f[E];
            if (du) {
                get(h + row * a.h_ld + c0, i, f);
                for (int j = 0; j < E; ++j) m[0] += f[j];
            }
            if (y) {
                get(y + row * a.y_ld + c0, i, f);
                for (int j = 0; j < E; ++j) m[1] += f[j];
            }
        }
        cta_sum(m, means);
        s.mh = m[0] * inv_w, s.my = m[1] * inv_w;
    }
    float q[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
    for (int i = 0; i < chunks; ++i) {
        float hv[E] = {0.f, 0.f, 0.f, 0.f}, uv[E] = {0.f, 0.f, 0.f, 0.f}, yv[E] = {0.f, 0.f, 0.f, 0.f}, wq[E];
        if (du) get(h + row * a.h_ld + c0, i, hv), get(du + row * a.du_ld + c0, i, uv);
        if (y) get(y + row * a.y_ld + c0, i, yv);
        cols.vector(a.w_pre ? a.w_pre + c0 : nullptr, i, 1.f, wq);
        for (int j = 0; j < E; ++j) {
            if (!cols.inside(i, j)) continue;
            const float g = uv[j] * wq[j], hc = hv[j] - s.mh, yc = yv[j] - s.my;
            q[0] = fmaf(hc, hc, q[0]);
            q[1] = fmaf(yc, yc, q[1]);
            q[2] += g;
            q[3] = fmaf(g, hc, q[3]);
        }
    }
    cta_sum(q, squares);
    s.rh = rsqrtf(fmaf(q[0], inv_w, a.eps)), s.ry = rsqrtf(fmaf(q[1], inv_w, a.eps));
    s.mg = a.layer ? q[2] * inv_w : 0.f, s.mgh = q[3] * inv_w * s.rh;
    if (y) {
        float z[2] = {0.f, 0.f};
#pragma unroll 2
        for (int i = 0; i < chunks; ++i) {
            float hv[E] = {0.f, 0.f, 0.f, 0.f}, uv[E] = {0.f, 0.f, 0.f, 0.f}, d[E] = {0.f, 0.f, 0.f, 0.f}, yv[E], gv[E], wq[E], wp[E];
            if (du) get(h + row * a.h_ld + c0, i, hv), get(du + row * a.du_ld + c0, i, uv);
            if (dh) get(dh + row * a.dh_ld + c0, i, d);
            get(y + row * a.y_ld + c0, i, yv);
            if (gate) get(gate + row * a.gate_ld + c0, i, gv);
            cols.vector(a.w_pre ? a.w_pre + c0 : nullptr, i, 1.f, wq);
            cols.vector(a.w_post ? a.w_post + c0 : nullptr, i, 1.f, wp);
            for (int j = 0; j < E; ++j) {
                if (!cols.inside(i, j)) continue;
                if (du) d[j] = fmaf(s.rh, fmaf(uv[j], wq[j], -s.mg) - (hv[j] - s.mh) * s.rh * s.mgh, d[j]);
                const float t = d[j] * a.s * (gate ? sigmoid<float>(gv[j]) : 1.f) * wp[j];
                z[0] += t;
                z[1] = fmaf(t, yv[j] - s.my, z[1]);
            }
        }
        cta_sum(z, products);
        s.mt = a.layer ? z[0] * inv_w : 0.f, s.mty = z[1] * inv_w * s.ry;
    }
    if (threadIdx.x == 0) stats[item] = s;
}

// blockIdx.x: 128 columns of one slice per warp; blockIdx.y: every gridDim.y-th row
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) norm_apply_kernel(const NormArgs a, const T* y, const T* gate, const T* h, const float* dh,
                                                         const float* du, float* dx, float* dy, float* dgate, const RowStats* stats) {
    cudaTriggerProgrammaticLaunchCompletion();
    constexpr int E = 4;
    const int per_slice = (a.w + 127) / 128;
    const int tile = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (tile >= per_slice * a.p) return;
    const int slice = tile / per_slice, i = tile - slice * per_slice, c0 = slice * a.w;
    const Columns<VEC, E> cols(threadIdx.x & 31, 32, a.w, false);
    const bool ragged = a.w % E != 0;
    float wp[E], bp[E], wq[E], acc[4][E];
    cols.vector(a.w_post ? a.w_post + c0 : nullptr, i, 1.f, wp);
    cols.vector(a.b_post ? a.b_post + c0 : nullptr, i, 0.f, bp);
    cols.vector(a.w_pre ? a.w_pre + c0 : nullptr, i, 1.f, wq);
#pragma unroll
    for (int j = 0; j < E; ++j) acc[0][j] = acc[1][j] = acc[2][j] = acc[3][j] = 0.f;
#pragma unroll 2
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        Chunk<T, E> qy, qg, qh;
        Chunk<float, E> qd, qu;
        const RowStats s = stats[row * a.p + slice];
        if (du) cols.load(qh, h + row * a.h_ld + c0, i), cols.load(qu, du + row * a.du_ld + c0, i);
        if (y) cols.load(qy, y + row * a.y_ld + c0, i);
        if (dh) cols.load(qd, dh + row * a.dh_ld + c0, i);
        if (gate) cols.load(qg, gate + row * a.gate_ld + c0, i);
        float hv[E], uv[E], yv[E], d[E] = {0.f, 0.f, 0.f, 0.f}, gv[E] = {0.f, 0.f, 0.f, 0.f};
        if (dh) qd.get(d);
        if (gate) qg.get(gv);
        if (du) {
            qh.get(hv), qu.get(uv);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float hhat = (hv[j] - s.mh) * s.rh;
                d[j] = fmaf(s.rh, fmaf(uv[j], wq[j], -s.mg) - hhat * s.mgh, d[j]);
                acc[2][j] = fmaf(uv[j], hhat, acc[2][j]);
                acc[3][j] += uv[j];
            }
        }
        if (dx) cols.store(dx + row * a.dx_ld + c0, i, d, ragged);
        if (!y) continue;
        qy.get(yv);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            float open = 1.f, slope = 0.f;
            if (gate) gate_and_slope(gv[j], open, slope);
            const float ds = d[j] * a.s, yhat = (yv[j] - s.my) * s.ry, dt = ds * open;
            gv[j] = ds * slope * fmaf(yhat, wp[j], bp[j]);
            yv[j] = s.ry * (dt * wp[j] - s.mt - yhat * s.mty);
            acc[0][j] = fmaf(dt, yhat, acc[0][j]);
            acc[1][j] += dt;
        }
        if (dgate) cols.store(dgate + row * a.dgate_ld + c0, i, gv, ragged);
        if (dy) cols.store(dy + row * a.dy_ld + c0, i, yv, ragged);
    }
    if (!a.partial) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float* out = a.partial + ((int64_t)blockIdx.y * 4 + k) * (a.p * a.w) + c0;
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (cols.inside(i, j)) out[cols.at(i) + j * cols.step] = acc[k][j];
    }
}

// partial rows -> column sums: 32 columns per CTA, 32 warps that take every 32nd row, then the warps in order
__global__ void __launch_bounds__(1024) norm_join_kernel(int64_t rows, int cols, const float* partial, float* dw_post, float* db_post,
                                                         float* dw_pre, float* db_pre) {
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, k = blockIdx.y;
    float* out = k == 0 ? dw_post : k == 1 ? db_post : k == 2 ? dw_pre : db_pre;
    cudaGridDependencySynchronize();
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
    a.eps = std::max((float)d->eps, 1.17549435e-38f);   // the least normal number: a row of zeros is divided by its root
    a.s = (float)d->residual_scale;
    a.x_ld = d->x_ld, a.y_ld = d->y_ld, a.gate_ld = d->gate_ld, a.h_ld = d->h_ld, a.u_ld = d->u_ld;
    a.dh_ld = d->dh_ld, a.du_ld = d->du_ld, a.dx_ld = d->dx_ld, a.dy_ld = d->dy_ld, a.dgate_ld = d->dgate_ld;
    a.w_post = d->w_post, a.b_post = d->b_post, a.w_pre = d->w_pre, a.b_pre = d->b_pre;
    return a;
}

constexpr int kSMs = 148;
constexpr int kMaxWarpWidth = 1024;   // columns of a slice that one warp takes

// Forward, up to 1024 columns.  By lanes (one chunk of E columns each), or staged with a warp per slice row.
struct ForwardPlan {
    int lanes;                 // 0: staged
    int chunks, warps, smem;   // staged: chunks per lane, warps per CTA
    int64_t ctas, lanes_rows;
};
// Shared memory of a CTA's staged rows at most.  Kernels whose size follows the call are allowed all of it, always: the limit
// belongs to the kernel, and one that followed the call could be lowered by another host thread between here and the launch.
constexpr int kStagedSmem = 226 * 1024, kWideSmem = SLICEGCN_MAX_NORM_WIDTH * (int)sizeof(float);
int64_t rows_at_a_time(int64_t ctas, int groups, int p) { return ctas * groups / p; }
int lanes_for(int need) {
    int lanes = 1;
    while (lanes < 32 && lanes < need) lanes *= 2;
    return lanes;
}
int staged_chunks(int w) { return w <= 256 ? 2 : w <= 512 ? 4 : w <= 640 ? 5 : 8; }
template <template <typename, int> class S>
int smem_for(int dtype, int chunks, int warps) {
    const bool bf = dtype == SLICEGCN_BF16;
    switch (chunks) {
        case 2: return bf ? S<__nv_bfloat16, 2>::smem(warps) : S<float, 2>::smem(warps);
        case 4: return bf ? S<__nv_bfloat16, 4>::smem(warps) : S<float, 4>::smem(warps);
        case 5: return bf ? S<__nv_bfloat16, 5>::smem(warps) : S<float, 5>::smem(warps);
        default: return bf ? S<__nv_bfloat16, 8>::smem(warps) : S<float, 8>::smem(warps);
    }
}
// Warps per CTA: as many as fit, but no more than leave every SM a CTA when there are few rows.  Row CTAs per slice.
template <template <typename, int> class S>
void staged_shape(const slicegcn_residual_norm_desc* d, int chunks, int most, int per_sm, int* warps, int* smem, int64_t* row_ctas) {
    *warps = most;
    while (smem_for<S>(d->dtype, chunks, *warps) > kStagedSmem / per_sm) --*warps;
    const int64_t share = (d->n * d->num_slices + kSMs * per_sm - 1) / (kSMs * per_sm);
    *warps = (int)std::max<int64_t>(1, std::min<int64_t>(*warps, share));
    *smem = smem_for<S>(d->dtype, chunks, *warps);
    *row_ctas = std::max<int64_t>(1, std::min<int64_t>((d->n + *warps - 1) / *warps, kSMs * per_sm / d->num_slices));
}
ForwardPlan forward_plan(const slicegcn_residual_norm_desc* d, int E) {
    ForwardPlan p{};
    const int need = (d->h_s + E - 1) / E;
    const int64_t items = d->n * d->num_slices;
    if (need <= 32) {
        p.lanes = lanes_for(need);
        const int groups = 256 / p.lanes;
        p.ctas = std::max<int64_t>(std::min<int64_t>((items + groups - 1) / groups, 8 * kSMs), (d->num_slices + groups - 1) / groups);
        p.lanes_rows = rows_at_a_time(p.ctas, groups, d->num_slices);
    } else {
        p.chunks = staged_chunks(d->h_s);
        int64_t row_ctas;
        staged_shape<StagedForward>(d, p.chunks, kForwardWarps, 1, &p.warps, &p.smem, &row_ctas);
        p.ctas = row_ctas * d->num_slices;
        p.lanes_rows = row_ctas * p.warps;
    }
    return p;
}

// Gradient.  The workspace holds the partial rows of the columns' sums and, for the third form, the rows' statistics.
enum { kByLanes, kStaged, kTwoPasses };
struct BackwardPlan {
    int form;
    int lanes;                         // kByLanes: lanes per slice row
    int chunks, warps, smem;           // kStaged: chunks per lane, warps per CTA
    int64_t ctas, lanes_rows;
    int whole_rows;
    int64_t partial_rows, stats_bytes;
};
constexpr int kApplyRows = 4 * kSMs;   // kTwoPasses: partial rows at most
BackwardPlan backward_plan(const slicegcn_residual_norm_desc* d) {
    BackwardPlan p{};
    const int64_t items = d->n * d->num_slices;
    if (d->h_s <= 128) {
        p.form = kByLanes;
        p.lanes = lanes_for((d->h_s + 3) / 4);
        const int groups = 256 / p.lanes;
        p.ctas = std::max<int64_t>(std::min<int64_t>((items + groups - 1) / groups, 2 * kSMs), (d->num_slices + groups - 1) / groups);
        p.lanes_rows = rows_at_a_time(p.ctas, groups, d->num_slices);
        p.whole_rows = groups % d->num_slices == 0;
        p.partial_rows = p.whole_rows ? p.ctas : p.lanes_rows;
    } else if (d->h_s <= kMaxWarpWidth) {
        p.form = kStaged;
        p.chunks = staged_chunks(d->h_s);
        const int most = p.chunks <= 5 ? staged_warps<5>() : staged_warps<8>();
        staged_shape<Staged>(d, p.chunks, most, 1, &p.warps, &p.smem, &p.partial_rows);
        p.ctas = p.partial_rows * d->num_slices;
        p.lanes_rows = p.partial_rows * p.warps;
    } else {
        p.form = kTwoPasses;
        p.partial_rows = std::max<int64_t>(1, std::min<int64_t>(d->n, kApplyRows));
        p.stats_bytes = items * (int64_t)sizeof(RowStats);
    }
    return p;
}
int64_t backward_bytes(const slicegcn_residual_norm_desc* d, const BackwardPlan& p) {
    return p.stats_bytes + p.partial_rows * 4 * d->num_slices * d->h_s * (int64_t)sizeof(float);
}

template <typename T>
struct ForwardCall {
    const ForwardPlan& pl;
    const NormArgs& a;
    const T *x, *y, *gate;
    T *h, *u;
    cudaStream_t st;
    template <bool VEC, int E, int L>
    slicegcn_status_t go() const {
        constexpr int smem = kForwardAhead * 3 * 256 * kForwardSlot<T, VEC, E>;   // 48 KB at most
        norm_forward_kernel<T, VEC, E, L><<<(unsigned)pl.ctas, 256, smem, st>>>(a, x, y, gate, h, u);
        return SLICEGCN_OK;
    }
    template <bool VEC, int NV>
    slicegcn_status_t staged() const {
        SGCN_CUDA(cudaFuncSetAttribute(norm_forward_staged_kernel<T, VEC, NV>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStagedSmem));
        norm_forward_staged_kernel<T, VEC, NV><<<(unsigned)pl.ctas, pl.warps * 32, pl.smem, st>>>(a, x, y, gate, h, u);
        return SLICEGCN_OK;
    }
    template <bool VEC, int E>
    slicegcn_status_t pick() const {
        switch (pl.lanes) {
            case 0: return pl.chunks == 2 ? staged<VEC, 2>() : pl.chunks == 4 ? staged<VEC, 4>() : pl.chunks == 5 ? staged<VEC, 5>() : staged<VEC, 8>();
            case 1: return go<VEC, E, 1>();
            case 2: return go<VEC, E, 2>();
            case 4: return go<VEC, E, 4>();
            case 8: return go<VEC, E, 8>();
            case 16: return go<VEC, E, 16>();
            default: return go<VEC, E, 32>();
        }
    }
    template <bool VEC>
    slicegcn_status_t wide() const {
        const int smem = (a.w + 4 * kWideThreads - 1) / (4 * kWideThreads) * 4 * kWideThreads * (int)sizeof(float);   // 64 KB at most
        SGCN_CUDA(cudaFuncSetAttribute(norm_forward_wide_kernel<T, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWideSmem));
        norm_forward_wide_kernel<T, VEC><<<(unsigned)(a.n * a.p), kWideThreads, smem, st>>>(a, x, y, gate, h, u);
        return SLICEGCN_OK;
    }
};

template <typename T>
struct BackwardCall {
    const BackwardPlan& pl;
    const NormArgs& a;
    const T *y, *gate, *h;
    const float *dh, *du;
    float *dx, *dy, *dgate;
    RowStats* stats;
    cudaStream_t st;
    template <bool VEC, int L>
    slicegcn_status_t go() const {
        constexpr int smem = kBackwardAhead * BackwardRing<T, VEC>::kStage;
        if (smem > 48 * 1024) SGCN_CUDA(cudaFuncSetAttribute(norm_backward_kernel<T, VEC, L>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        norm_backward_kernel<T, VEC, L><<<(unsigned)pl.ctas, 256, smem, st>>>(a, y, gate, h, dh, du, dx, dy, dgate);
        return SLICEGCN_OK;
    }
    template <bool VEC, int NV, bool BIAS, bool LAYER>
    slicegcn_status_t staged() const {
        SGCN_CUDA(cudaFuncSetAttribute(norm_backward_staged_kernel<T, VEC, NV, BIAS, LAYER>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStagedSmem));
        norm_backward_staged_kernel<T, VEC, NV, BIAS, LAYER><<<(unsigned)pl.ctas, pl.warps * 32, pl.smem, st>>>(a, y, gate, h, dh, du, dx, dy, dgate);
        return SLICEGCN_OK;
    }
    template <bool VEC, bool BIAS, bool LAYER>
    slicegcn_status_t staged_for() const {
        return pl.chunks == 2   ? staged<VEC, 2, BIAS, LAYER>()
               : pl.chunks == 4 ? staged<VEC, 4, BIAS, LAYER>()
               : pl.chunks == 5 ? staged<VEC, 5, BIAS, LAYER>()
                                : staged<VEC, 8, BIAS, LAYER>();
    }
    template <bool VEC>
    slicegcn_status_t run(bool bias) const {
        if (pl.form == kByLanes) {
            switch (pl.lanes) {
                case 1: SGCN_TRY((go<VEC, 1>())); break;
                case 2: SGCN_TRY((go<VEC, 2>())); break;
                case 4: SGCN_TRY((go<VEC, 4>())); break;
                case 8: SGCN_TRY((go<VEC, 8>())); break;
                case 16: SGCN_TRY((go<VEC, 16>())); break;
                default: SGCN_TRY((go<VEC, 32>())); break;
            }
        } else if (pl.form == kStaged) {
            if (a.layer)
                SGCN_TRY((bias ? staged_for<VEC, true, true>() : staged_for<VEC, false, true>()));
            else
                SGCN_TRY((bias ? staged_for<VEC, true, false>() : staged_for<VEC, false, false>()));
        } else {
            norm_stats_kernel<T, VEC><<<(unsigned)(a.n * a.p), kWideThreads, 0, st>>>(a, y, gate, h, dh, du, stats);
            SGCN_LAUNCH_CHECK();
            count_launch();
            const int tiles = (a.w + 127) / 128 * a.p;
            const dim3 grid((tiles + 7) / 8, (unsigned)pl.partial_rows);
            norm_apply_kernel<T, VEC><<<grid, 256, 0, st>>>(a, y, gate, h, dh, du, dx, dy, dgate, stats);
        }
        SGCN_LAUNCH_CHECK();
        count_launch();
        return SLICEGCN_OK;
    }
};

// Whether every matrix that is given allows accesses of E elements at once.
struct VecCheck {
    int E;
    bool ok;
    VecCheck(const slicegcn_residual_norm_desc* d, int e) : E(e), ok(d->num_slices == 1 || d->h_s % e == 0) {}
    VecCheck& with(const void* p, int64_t ld, int esz) {
        if (p) ok = ok && ld % E == 0 && (uintptr_t)p % std::min(E * esz, 16) == 0;
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
    cudaStream_t st = (cudaStream_t)stream;
    auto check = [&](int E) {
        return VecCheck(d, E).with(x, d->x_ld, esz).with(y, d->y_ld, esz).with(gate, d->gate_ld, esz).with(h, d->h_ld, esz).with(u, d->u_ld, esz).ok;
    };
    const bool vec4 = check(4), vec8 = esz == 2 && check(8), wide = d->h_s > kMaxWarpWidth;
    const ForwardPlan pl = forward_plan(d, vec8 ? 8 : 4);
    a.lanes_rows = pl.lanes_rows;
    if (d->dtype == SLICEGCN_BF16) {
        using T = __nv_bfloat16;
        const ForwardCall<T> call{pl, a, (const T*)x, (const T*)y, (const T*)gate, (T*)h, (T*)u, st};
        if (wide)
            SGCN_TRY(vec4 ? call.template wide<true>() : call.template wide<false>());
        else
            SGCN_TRY((vec8 ? call.template pick<true, 8>() : vec4 ? call.template pick<true, 4>() : call.template pick<false, 4>()));
    } else {
        using T = float;
        const ForwardCall<T> call{pl, a, (const T*)x, (const T*)y, (const T*)gate, (T*)h, (T*)u, st};
        if (wide)
            SGCN_TRY(vec4 ? call.template wide<true>() : call.template wide<false>());
        else
            SGCN_TRY((vec4 ? call.template pick<true, 4>() : call.template pick<false, 4>()));
    }
    SGCN_LAUNCH_CHECK();
    count_launch();
    return SLICEGCN_OK;
}

slicegcn_status_t slicegcn_residual_norm_workspace_bytes(const slicegcn_residual_norm_desc* d, int64_t* bytes) {
    SGCN_TRY(check_desc(d, "residual_norm_workspace_bytes"));
    if (!bytes) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "residual_norm_workspace_bytes: NULL argument");
    *bytes = backward_bytes(d, backward_plan(d));
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
    const bool fours = VecCheck(d, 4).with(y, d->y_ld, esz).with(gate, d->gate_ld, esz).with(h, d->h_ld, esz).with(dh, d->dh_ld, 4)
                         .with(du, d->du_ld, 4).with(dx, d->dx_ld, 4).with(dy, d->dy_ld, 4).with(dgate, d->dgate_ld, 4).ok;
    const BackwardPlan pl = backward_plan(d);
    const int cols = d->num_slices * d->h_s;
    const int64_t need = backward_bytes(d, pl);
    if ((sums || pl.form == kTwoPasses) && (!workspace || workspace_bytes < need))
        SGCN_FAIL(SLICEGCN_ERR_ALLOC, "%s: workspace too small (%lld < %lld bytes)", who, (long long)workspace_bytes, (long long)need);
    if ((uintptr_t)workspace % 16) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: the workspace is not aligned to 16 bytes", who);
    NormArgs a = make_args(d);
    // the kernels take what is not there as zeros; weights beside it, which the caller may have left as they were, are left out too
    if (!du) a.w_pre = a.b_pre = nullptr;
    if (!y) a.w_post = a.b_post = nullptr;
    a.lanes_rows = pl.lanes_rows;
    a.whole_rows = pl.whole_rows;
    RowStats* stats = static_cast<RowStats*>(workspace);
    a.partial = sums ? reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.stats_bytes) : nullptr;
    cudaStream_t st = (cudaStream_t)stream;
    if (a.n > 0) {
        const bool bias = db_post || db_pre;
        if (d->dtype == SLICEGCN_BF16) {
            using T = __nv_bfloat16;
            const BackwardCall<T> call{pl, a, (const T*)y, (const T*)gate, (const T*)h, dh, du, dx, dy, dgate, stats, st};
            SGCN_TRY(fours ? call.template run<true>(bias) : call.template run<false>(bias));
        } else {
            using T = float;
            const BackwardCall<T> call{pl, a, (const T*)y, (const T*)gate, (const T*)h, dh, du, dx, dy, dgate, stats, st};
            SGCN_TRY(fours ? call.template run<true>(bias) : call.template run<false>(bias));
        }
    }
    if (sums) {
        SGCN_TRY(launch_after(norm_join_kernel, dim3((cols + 31) / 32, 4), 1024, 0, st, a.n > 0 ? pl.partial_rows : (int64_t)0, cols,
                              (const float*)a.partial, dw_post, db_post, dw_pre, db_pre));
    }
    return SLICEGCN_OK;
}

}  // extern "C"
