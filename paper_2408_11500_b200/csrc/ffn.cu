// Feed-forward projections per slice and their gradients:
//   a = x W + b,  c = x W2 + b2,   out = r + scale * act(a) [* c]
//   g = scale * dout,  da = g act'(a) [* c],  dc = g act(a)
//   dx = da W^T + dc W2^T,  dW = x^T da,  dW2 = x^T dc,  db = sum of da over rows,  db2 of dc
// One kernel does every matrix product: D = sum over k of A[m, k] B[n, k], operands bf16, fp32 accumulators in tensor memory.
//
//   * A pair of SMs (a cluster of two CTAs) makes a tile of 256 rows x 2*nt columns: each CTA brings its own 128 rows of A and
//     its own nt columns of B, and the pair's MMA reads both halves.  Per 64-wide step of k a CTA copies 32 KB for 512 cycles of MMA;
//     single CTAs with the same tile would copy 48 KB, and shared memory would pace the MMA.
//   * Both operands come by tensor copy from where they lie, whichever of their axes is contiguous (x and dW's operands along
//     rows, W along columns): nothing is transposed.  Odd strides, and fp32, are laid out in the workspace first.
//   * fp32 values are three bf16 numbers (8 bits of the significand each), and a product of two of them is the six products
//     of parts that reach fp32's last digit, the small ones first.  One code path, at a sixth of the bf16 rate.
//   * Tensor memory's accumulation cuts digits off; over k in the hundreds of 16-wide steps that would show in fp32.  There the
//     accumulator is emptied into registers every few hundred k ("chunk"), and the registers are added to with rounding.
//   * Two accumulators: the sixteen epilogue warps work on one while the MMA fills the other.
//   * The gate needs no second pass: the two halves of B are columns of W and of W2, so a and c of the same columns
//     meet in the same thread.
//   * dW = x^T da runs over rows; they are split over the SMs, and the pieces' sums are added in a fixed order.
#include <cuda.h>

#include <algorithm>
#include <cmath>

#include "common.cuh"

namespace sgcn {
namespace {

constexpr int kPairs = 74;                       // pairs of SMs
constexpr int kStages = 5, kStageBytes = 32768;  // A: 128 x 64 bf16, B: up to 128 x 64
constexpr int kEpiWarps = 16, kThreads = (kEpiWarps + 2) * 32;
constexpr int kSlabBytes = 2048;                 // of an epilogue warp: 32 rows x 64 bytes
constexpr int kBiasBytes = 256;                  // and 32 columns of both biases
constexpr int kSmem = kStages * kStageBytes + kEpiWarps * (kSlabBytes + kBiasBytes) + 1024 + 256;
constexpr long long kWaitClocks = 2000000000LL;  // about a second

enum Mode { kFwd, kFwdGated, kDz, kDzGated, kDx, kDw };

// n / d for 0 <= n < 2^31 by a multiplication
struct Divide {
    uint32_t mul, shift;
    int d;
    __device__ __forceinline__ int operator()(int n) const { return (int)((__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift); }
};
Divide divide_by(int d) {
    Divide r;
    r.d = d;
    for (r.shift = 0; (1ll << r.shift) < d; ++r.shift) {}
    r.mul = (uint32_t)(((1ull << 32) * ((1ull << r.shift) - (uint64_t)d)) / (uint64_t)d + 1);
    return r;
}

struct Params {
    CUtensorMap a, b0, b1;
    int n;                         // rows of x
    int p, slices;                 // slices; slices times parts of the output (kDw), else the same
    int tiles_m, tiles_n, group;   // per slice; m tiles that follow one another before the next n tile
    Divide by_first, by_n, by_m, by_last;   // what item_of divides by
    int items;
    int nt;                        // columns of B per CTA: 64 or 128
    int kb_total, kb_part, k_part; // 64-wide steps of an item, of one part of k, and that part's extent
    int chunk;                     // steps between emptyings of the accumulator
    int pairs;                     // products of operand parts
    int8_t ia[6], ib[6];
    int splits;                    // kDw: pieces of the rows, kb_total steps each
    int splits_rows;               // kDw
    // epilogue
    int act, cols;                 // columns of D per slice
    float scale;
    const float *b, *b2;           // [slices][cols]
    const void* in;                // r or dout
    int64_t in_ld;
    int in_bf16, in_vec;
    void* out;
    int64_t out_ld;
    int out_bf16, out_vec;
    // kDz: planes of da (and dc after it) in the workspace, and sums over 32 rows each
    __nv_bfloat16* dz;
    int64_t dz_plane, dz_row;      // elements between planes and between rows
    int dz_planes, dz_pad;         // columns of one (part, slice)
    float* sums;                   // [ceil(n/32)][parts * p][cols], or NULL
    // kDw
    float* partial;                // [splits][slices][k][cols of A]
    void *dw, *dw2;                // splits == 1
    int32_t* status;
};

// ------------------------------------------------------------------------------------------ instructions

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void mbar_init(uint64_t* bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count));
}
__device__ __forceinline__ bool mbar_try(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// Gives up after about a second.
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity) {
    if (mbar_try(bar, parity)) return true;
    const long long t0 = clock64();
    for (int i = 0; i < (1 << 22); ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 63) == 63 && clock64() - t0 > kWaitClocks) break;
    }
    return false;
}
__device__ __forceinline__ void mbar_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// Arrives at the same barrier of the pair's first CTA.  Relaxed: what it hands over are accumulators that have been read (the wait for
// those reads is behind this thread); a release would first wait for all results the warp has stored (17 % of all warp stalls).
__device__ __forceinline__ void mbar_arrive_first(uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, 0;\n\t"
        "mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [a];\n\t}" ::"r"(smem_u32(bar))
        : "memory");
}
// One box of a tensor map into this CTA's memory; the bytes are counted at the barrier of the pair's first CTA.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar) & 0xFEFFFFFFu)
        : "memory");
}
__device__ __forceinline__ void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// Arrives at the barrier of both CTAs when all MMAs issued so far are done.
__device__ __forceinline__ void umma_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 lanes x 16 columns: a lane gets its row
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}
// The wait takes part in the registers' dataflow, so that no use of them moves in front of it.
#define SGCN_R16(r)                                                                                                                              \
    "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), \
        "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
__device__ __forceinline__ void tmem_wait(uint32_t* r) { asm volatile("tcgen05.wait::ld.sync.aligned;" : SGCN_R16(r)::"memory"); }
__device__ __forceinline__ void after_wait(uint32_t* r) { asm volatile("" : SGCN_R16(r)::"memory"); }
#undef SGCN_R16

// Operand tiles, 128-byte swizzle.  k contiguous: rows of 64 k, 8-row groups 1 KB apart.  Rows (or columns) contiguous: blocks of
// 64 of them x 64 k, 8-k groups 1 KB apart, blocks 8 KB apart.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, bool k_contiguous) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)(k_contiguous ? 1 : 8192 >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}

// ------------------------------------------------------------------------------------------ pieces of the epilogue

// A warp's 32 rows x UB bytes pass through its slab, so that lanes that hold a row each meet global memory in whole lines.
template <int UB>
__device__ __forceinline__ uint32_t slab_at(int row, int chunk) {   // bank-conflict free both by rows and by lines
    constexpr int per = UB / 16;
    const int swz = per == 8 ? row & 7 : per == 4 ? (row >> 1) & 3 : (row >> 2) & 1;
    return (uint32_t)(row * UB + ((chunk ^ swz) << 4));
}
__device__ __forceinline__ void sts16(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}

// U columns x 32 rows of a matrix as the lines a warp reads them; `rows` and `cols` are what exists of them.
template <int U, bool BF16>
struct Lines {
    static constexpr int UB = U * (BF16 ? 2 : 4), per = UB / 16;
    uint4 raw[per];
    __device__ __forceinline__ void load(const char* at, int64_t ld_bytes, int rows, int cols, bool vec, uint32_t slab, int lane) {
        constexpr int E = BF16 ? 2 : 4;
        if (vec) {
#pragma unroll
            for (int i = 0; i < per; ++i) {
                const int row = i * (32 / per) + lane / per, c = lane % per;
                const int left = cols * E - c * 16;
                const char* src = at + (int64_t)(row < rows ? row : 0) * ld_bytes + c * 16;
                raw[i] = make_uint4(0, 0, 0, 0);
                if (row < rows && left > 0) {
                    if (left >= 16)
                        raw[i] = *reinterpret_cast<const uint4*>(src);
                    else {
                        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                        for (int k = 0; k < 16 / E; ++k)
                            if (k * E < left) {
                                if (BF16)
                                    w[k / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(src)[k] << (16 * (k & 1));
                                else
                                    w[k & 3] = reinterpret_cast<const uint32_t*>(src)[k];
                            }
                        raw[i] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
        } else {   // element by element, a row (U = 16: two rows) at a time; they go to the slab at once
            __syncwarp();
#pragma unroll 8
            for (int i = 0; i < U; ++i) {
                const int row = i * (32 / U) + lane / U, c = lane % U;
                const bool there = row < rows && c < cols;
                const uint32_t to = slab + slab_at<UB>(row, c * E / 16) + (uint32_t)(c * E % 16);
                if (BF16) {
                    const uint16_t v = there ? *reinterpret_cast<const uint16_t*>(at + (int64_t)row * ld_bytes + c * 2) : (uint16_t)0;
                    asm volatile("st.shared.u16 [%0], %1;" ::"r"(to), "h"(v) : "memory");
                } else {
                    const uint32_t v = there ? *reinterpret_cast<const uint32_t*>(at + (int64_t)row * ld_bytes + c * 4) : 0u;
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(to), "r"(v) : "memory");
                }
            }
        }
    }
    // The lane's own row.
    __device__ __forceinline__ void row(float* v, bool vec, uint32_t slab, int lane) {
        if (vec) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < per; ++i) sts16(slab + slab_at<UB>(i * (32 / per) + lane / per, lane % per), raw[i]);
        }
        __syncwarp();
#pragma unroll
        for (int c = 0; c < per; ++c) {
            const uint4 t = lds16(slab + slab_at<UB>(lane, c));
            const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (BF16) {
                    v[c * 8 + 2 * k] = __uint_as_float(w[k] << 16);
                    v[c * 8 + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
                } else {
                    v[c * 4 + k] = __uint_as_float(w[k]);
                }
            }
        }
    }
};

// The lanes' rows of U words or halves to memory.
template <int U, bool BF16>
__device__ __forceinline__ void store_lines(const uint32_t* w, char* at, int64_t ld_bytes, int rows, int cols, bool vec, uint32_t slab, int lane) {
    constexpr int E = BF16 ? 2 : 4, UB = U * E, per = UB / 16;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < per; ++c) sts16(slab + slab_at<UB>(lane, c), make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]));
    __syncwarp();
    if (vec) {
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const int row = i * (32 / per) + lane / per, c = lane % per;
            const int left = cols * E - c * 16;
            if (row >= rows || left <= 0) continue;
            const uint4 t = lds16(slab + slab_at<UB>(row, c));
            char* dst = at + (int64_t)row * ld_bytes + c * 16;
            if (left >= 16)
                *reinterpret_cast<uint4*>(dst) = t;
            else {
                const uint32_t v[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                for (int k = 0; k < 16 / E; ++k)
                    if (k * E < left) {
                        if (BF16)
                            reinterpret_cast<uint16_t*>(dst)[k] = (uint16_t)(v[k / 2] >> (16 * (k & 1)));
                        else
                            reinterpret_cast<uint32_t*>(dst)[k] = v[k & 3];
                    }
            }
        }
    } else {
#pragma unroll 8
        for (int i = 0; i < U; ++i) {
            const int row = i * (32 / U) + lane / U, c = lane % U;
            const uint32_t from = slab + slab_at<UB>(row, c * E / 16) + (uint32_t)(c * E % 16);
            if (row < rows && c < cols) {
                if (BF16) {
                    uint16_t v;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(from) : "memory");
                    *reinterpret_cast<uint16_t*>(at + (int64_t)row * ld_bytes + c * 2) = v;
                } else {
                    uint32_t v;
                    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(from) : "memory");
                    *reinterpret_cast<uint32_t*>(at + (int64_t)row * ld_bytes + c * 4) = v;
                }
            }
        }
    }
}

// 1 / (1 + exp(-w)).  Where results are rounded to bf16 the hardware's exponential and reciprocal (2^-22 each, and 2^-24 |w| of the
// argument) are exact enough; `t` is -w log2(e).
__device__ __forceinline__ float sigmoid_of(float t) {
    float e, q;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q) : "f"(1.f + e));
    return q;
}
constexpr float kLog2e = 1.4426950408889634f, kGeluA = 0.7978845608028654f, kGeluB = 0.044715f;
template <bool ACCURATE>
__device__ __forceinline__ float sigmoid(float w) {
    return ACCURATE ? 1.f / (1.f + expf(-w)) : sigmoid_of(-kLog2e * w);
}
template <bool ACCURATE>
__device__ __forceinline__ float gelu_gate(float a) {   // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u))
    const float s = a * a;
    return ACCURATE ? sigmoid<true>(2.f * kGeluA * a * fmaf(kGeluB, s, 1.f)) : sigmoid_of(a * fmaf(-2.f * kLog2e * kGeluA * kGeluB, s, -2.f * kLog2e * kGeluA));
}
// act(a)
template <bool ACCURATE>
__device__ __forceinline__ float act_of(int act, float a) {
    if (act == SLICEGCN_ACT_SILU) return a * sigmoid<ACCURATE>(a);
    if (act == SLICEGCN_ACT_GELU) return a * gelu_gate<ACCURATE>(a);
    if (act == SLICEGCN_ACT_RELU) return a > 0.f || isnan(a) ? a : 0.f;
    return a;
}
// act(a) and act'(a)
template <bool ACCURATE>
__device__ __forceinline__ void act_both(int act, float a, float& y, float& dy) {
    if (act == SLICEGCN_ACT_SILU) {
        const float q = sigmoid<ACCURATE>(a);
        y = a * q;
        dy = fmaf(y, 1.f - q, q);
    } else if (act == SLICEGCN_ACT_GELU) {
        const float q = gelu_gate<ACCURATE>(a);
        y = a * q;
        dy = fmaf(y * (1.f - q), 2.f * kGeluA * fmaf(3.f * kGeluB, a * a, 1.f), q);
    } else if (act == SLICEGCN_ACT_RELU) {
        y = a > 0.f || isnan(a) ? a : 0.f;
        dy = a > 0.f ? 1.f : 0.f;
    } else {
        y = a;
        dy = 1.f;
    }
}

// Sums of 16 columns over the warp's rows: lane l gets column l / 2.
__device__ __forceinline__ float column_sums16(float (&v)[16], int lane) {
#pragma unroll
    for (int half = 8, mask = 16; half >= 1; half >>= 1, mask >>= 1) {
        const bool up = lane & mask;
#pragma unroll
        for (int j = 0; j < half; ++j) {
            const float keep = up ? v[j + half] : v[j], give = up ? v[j] : v[j + half];
            v[j] = keep + __shfl_xor_sync(0xffffffffu, give, mask);
        }
    }
    return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
}

// Parts of an fp32 number whose sum it is: 8 bits each.  Cut, not rounded: no part leaves the range, and each is exact.
__device__ __forceinline__ void split3(float x, float (&part)[3]) {
    if (isnan(x)) x = __int_as_float(0x7fc00000);   // one whose upper half alone is a NaN too
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        part[k] = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
        x = isfinite(x) ? x - part[k] : 0.f;
    }
}

struct Where {
    int slice, row, col;   // of the warp's rows in D and of its first column there
    int rows;              // how many of its 32 rows exist
};

template <int U>
__device__ __forceinline__ void add_bias(float (&v)[U], const float* b, int slice, int cols, int col) {
    if (!b) return;
    const float* at = b + (int64_t)slice * cols;
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const float t = __ldg(at + min(col + j, cols - 1));   // the same address in every lane
        v[j] += col + j < cols ? t : 0.f;
    }
}

// U columns of a forward product (or of dx): bias, activation, gate, scale, residual.
template <int U, bool GATED, bool ACCURATE, bool IN_BF16, bool OUT_BF16>
__device__ __forceinline__ void finish_forward_as(const Params& P, const Where& w, int col, float (&a)[U], float (&c)[U], Lines<U, IN_BF16>& lines, uint32_t slab, int lane) {
    add_bias<U>(a, P.b, w.slice, P.cols, col);
    if (GATED) add_bias<U>(c, P.b2, w.slice, P.cols, col);
#define SGCN_ACT(A)                                                       \
    _Pragma("unroll") for (int j = 0; j < U; ++j) {                       \
        float y = act_of<ACCURATE>(A, a[j]);                              \
        if (GATED) y *= c[j];                                             \
        a[j] = y * P.scale;                                               \
    }
    if (P.act == SLICEGCN_ACT_SILU) {
        SGCN_ACT(SLICEGCN_ACT_SILU)
    } else if (P.act == SLICEGCN_ACT_GELU) {
        SGCN_ACT(SLICEGCN_ACT_GELU)
    } else if (P.act == SLICEGCN_ACT_RELU) {
        SGCN_ACT(SLICEGCN_ACT_RELU)
    } else {
        SGCN_ACT(SLICEGCN_ACT_NONE)
    }
#undef SGCN_ACT
    if (P.in) {
        float r[U];
        lines.row(r, P.in_vec, slab, lane);
#pragma unroll
        for (int j = 0; j < U; ++j) a[j] += r[j];
    }
    constexpr int E = OUT_BF16 ? 2 : 4, W = U * E / 4;
    uint32_t words[W];
#pragma unroll
    for (int j = 0; j < W; ++j) words[j] = OUT_BF16 ? pack2(a[(2 * j) % U], a[(2 * j + 1) % U]) : __float_as_uint(a[j % U]);
    char* at = static_cast<char*>(P.out) + ((int64_t)w.row * P.out_ld + (int64_t)w.slice * P.cols + col) * E;
    store_lines<U, OUT_BF16>(words, at, P.out_ld * E, w.rows, P.cols - col, P.out_vec, slab, lane);
}

template <int U, bool GATED, bool ACCURATE>
__device__ __forceinline__ void finish_forward(const Params& P, const Where& w, int col, float (&a)[U], float (&c)[U], uint32_t slab, int lane) {
    // residual and output have one type
    if (P.out_bf16) {
        Lines<U, true> lines;
        if (P.in)
            lines.load(static_cast<const char*>(P.in) + ((int64_t)w.row * P.in_ld + (int64_t)w.slice * P.cols + col) * 2, P.in_ld * 2, w.rows, P.cols - col,
                       P.in_vec, slab, lane);
        finish_forward_as<U, GATED, ACCURATE, true, true>(P, w, col, a, c, lines, slab, lane);
    } else {
        Lines<U, false> lines;
        if (P.in)
            lines.load(static_cast<const char*>(P.in) + ((int64_t)w.row * P.in_ld + (int64_t)w.slice * P.cols + col) * 4, P.in_ld * 4, w.rows, P.cols - col,
                       P.in_vec, slab, lane);
        finish_forward_as<U, GATED, ACCURATE, false, false>(P, w, col, a, c, lines, slab, lane);
    }
}

// Sixteen columns of one of da and dc: planes to the workspace, and the sums over the warp's rows.
__device__ __forceinline__ void put_dz(const Params& P, const Where& w, int part, int col, float (&v)[16], uint32_t slab, int lane) {
    const int ps = part * P.p + w.slice;
    __nv_bfloat16* at = P.dz + (int64_t)w.row * P.dz_row + (int64_t)ps * P.dz_pad + col;
    uint32_t words[8];
    if (P.dz_planes == 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) words[j] = pack2(v[2 * j], v[2 * j + 1]);
        store_lines<16, true>(words, reinterpret_cast<char*>(at), P.dz_row * 2, w.rows, P.dz_pad - col, true, slab, lane);
    } else {
        float rest[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) rest[j] = v[j];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t lo = __float_as_uint(rest[2 * j]) & 0xffff0000u, hi = __float_as_uint(rest[2 * j + 1]) & 0xffff0000u;
                words[j] = lo >> 16 | hi;
                rest[2 * j] = isfinite(rest[2 * j]) ? rest[2 * j] - __uint_as_float(lo) : 0.f;
                rest[2 * j + 1] = isfinite(rest[2 * j + 1]) ? rest[2 * j + 1] - __uint_as_float(hi) : 0.f;
            }
            store_lines<16, true>(words, reinterpret_cast<char*>(at + k * P.dz_plane), P.dz_row * 2, w.rows, P.dz_pad - col, true, slab, lane);
        }
    }
    if (P.sums) {
        const float s = column_sums16(v, lane);
        const int c = col + (lane >> 1);
        if (!(lane & 1) && c < P.cols && w.rows > 0) P.sums[((int64_t)(w.row >> 5) * (P.slices) + ps) * P.cols + c] = s;
    }
}

// Sixteen columns of da (and dc).
template <bool GATED, bool ACCURATE>
__device__ __forceinline__ void finish_dz(const Params& P, const Where& w, int col, float (&a)[16], float (&c)[16], uint32_t slab, int lane) {
    float g[16];
    if (P.in_bf16) {
        Lines<16, true> lines;
        lines.load(static_cast<const char*>(P.in) + ((int64_t)w.row * P.in_ld + (int64_t)w.slice * P.cols + col) * 2, P.in_ld * 2, w.rows, P.cols - col, P.in_vec,
                   slab, lane);
        lines.row(g, P.in_vec, slab, lane);
    } else {
        Lines<16, false> lines;
        lines.load(static_cast<const char*>(P.in) + ((int64_t)w.row * P.in_ld + (int64_t)w.slice * P.cols + col) * 4, P.in_ld * 4, w.rows, P.cols - col, P.in_vec,
                   slab, lane);
        lines.row(g, P.in_vec, slab, lane);
    }
    add_bias<16>(a, P.b, w.slice, P.cols, col);
    if (GATED) add_bias<16>(c, P.b2, w.slice, P.cols, col);
#define SGCN_ACT(A)                                                       \
    _Pragma("unroll") for (int j = 0; j < 16; ++j) {                      \
        float y, dy;                                                      \
        act_both<ACCURATE>(A, a[j], y, dy);                               \
        const float gj = g[j] * P.scale;                                  \
        a[j] = GATED ? gj * c[j] * dy : gj * dy;                          \
        if (GATED) c[j] = gj * y;                                         \
    }
    if (P.act == SLICEGCN_ACT_SILU) {
        SGCN_ACT(SLICEGCN_ACT_SILU)
    } else if (P.act == SLICEGCN_ACT_GELU) {
        SGCN_ACT(SLICEGCN_ACT_GELU)
    } else if (P.act == SLICEGCN_ACT_RELU) {
        SGCN_ACT(SLICEGCN_ACT_RELU)
    } else {
        SGCN_ACT(SLICEGCN_ACT_NONE)
    }
#undef SGCN_ACT
    put_dz(P, w, 0, col, a, slab, lane);
    if (GATED) put_dz(P, w, 1, col, c, slab, lane);
}

// ---- bf16: 32 columns at a time

__device__ __forceinline__ void sts4(uint32_t a, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory"); }
// Sixteen numbers that every lane reads alike, added.
__device__ __forceinline__ void add16(float (&v)[16], uint32_t at) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint4 t = lds16(at + k * 16);
        v[4 * k] += __uint_as_float(t.x), v[4 * k + 1] += __uint_as_float(t.y);
        v[4 * k + 2] += __uint_as_float(t.z), v[4 * k + 3] += __uint_as_float(t.w);
    }
}
// Where a lane finds its row's chunk c of eight columns, and its line i of eight (row i * 8 + lane / 4, chunk lane % 4).
__device__ __forceinline__ uint32_t own_chunk(uint32_t slab, int lane, int c) { return (slab + lane * 64 + (((lane >> 1) & 3) << 4)) ^ (c << 4); }
__device__ __forceinline__ uint32_t own_line(uint32_t slab, int lane, int i) {
    return slab + i * 512 + (lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 3) & 3)) << 4);
}
__device__ __forceinline__ void put_rows(const uint32_t* w, uint32_t slab, int lane) {
#pragma unroll
    for (int c = 0; c < 4; ++c) sts16(own_chunk(slab, lane, c), make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]));
}
// The slab's 32 rows x 32 columns to memory, `rows` and `cols` of them.
__device__ __forceinline__ void slab_out(char* at, int64_t ld_bytes, int rows, int cols, bool vec, uint32_t slab, int lane) {
    if (vec && cols >= 8) {
        const int left = cols - (lane & 3) * 8;
        char* to = at + (int64_t)(lane >> 2) * ld_bytes + (lane & 3) * 16;
        if (rows == 32 && cols >= 32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(to + i * 8 * ld_bytes) = lds16(own_line(slab, lane, i));
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i * 8 + (lane >> 2) < rows && left >= 8) *reinterpret_cast<uint4*>(to + i * 8 * ld_bytes) = lds16(own_line(slab, lane, i));
        if (cols >= 32 || cols % 8 == 0) return;
    }
    // element by element: all columns, or those behind the last eight
    const int c = lane, from = vec ? min(cols, 32) & ~7 : 0;
    if (c >= from && c < cols)
#pragma unroll 4
        for (int i = 0; i < rows; ++i) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(slab + slab_at<64>(i, c >> 3) + (c & 7) * 2) : "memory");
            *reinterpret_cast<uint16_t*>(at + (int64_t)i * ld_bytes + c * 2) = v;
        }
}
// 32 rows x 32 columns of r or dout: asked for here (whole chunks where they are aligned) ...
__device__ __forceinline__ void load_in(const Params& P, const Where& w, int col, uint4 (&raw)[4], int lane) {
    const int left = P.cols - col - (lane & 3) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = make_uint4(0, 0, 0, 0);
    if (!P.in_vec || w.rows <= 0 || left < 8) return;
    const char* at = static_cast<const char*>(P.in) + ((int64_t)w.row * P.in_ld + (int64_t)w.slice * P.cols + col + (lane & 3) * 8) * 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 8 + (lane >> 2);
        const uint4 t = *reinterpret_cast<const uint4*>(at + (int64_t)min(row, w.rows - 1) * P.in_ld * 2);
        if (row < w.rows) raw[i] = t;
    }
}
// ... and laid into the slab here, with what no whole chunk holds.
__device__ __forceinline__ void put_in(const Params& P, const Where& w, int col, const uint4 (&raw)[4], uint32_t slab, int lane) {
    const int cols = min(32, P.cols - col), from = P.in_vec ? max(cols, 0) & ~7 : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sts16(own_line(slab, lane, i), raw[i]);
    if (from >= cols || w.rows <= 0) return;
    __syncwarp();
    const int c = lane;
    const char* at = static_cast<const char*>(P.in) + ((int64_t)w.row * P.in_ld + (int64_t)w.slice * P.cols + col + c) * 2;
    if (c >= from && c < cols)
#pragma unroll 8
        for (int i = 0; i < w.rows; ++i) {
            const uint16_t v = *reinterpret_cast<const uint16_t*>(at + (int64_t)i * P.in_ld * 2);
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(slab + slab_at<64>(i, c >> 3) + (c & 7) * 2), "h"(v) : "memory");
        }
}
// Sixteen columns of the lane's row in the slab.
__device__ __forceinline__ void own_row16(float (&v)[16], uint32_t slab, int lane, int h) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const uint4 t = lds16(own_chunk(slab, lane, 2 * h + q));
        const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[q * 8 + 2 * k] = __uint_as_float(w[k] << 16);
            v[q * 8 + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    }
}

// Half of 32 columns of a forward product (of dx: PLAIN), packed.
template <bool GATED, bool PLAIN>
__device__ __forceinline__ void forward_half(const Params& P, int h, float (&a)[16], const float (&c)[16], uint32_t* words, uint32_t slab, int lane) {
    if (!PLAIN) {
#define SGCN_ACT(A) _Pragma("unroll") for (int j = 0; j < 16; ++j) a[j] = act_of<false>(A, a[j])
        if (P.act == SLICEGCN_ACT_SILU)
            SGCN_ACT(SLICEGCN_ACT_SILU);
        else if (P.act == SLICEGCN_ACT_GELU)
            SGCN_ACT(SLICEGCN_ACT_GELU);
        else if (P.act == SLICEGCN_ACT_RELU)
            SGCN_ACT(SLICEGCN_ACT_RELU);
#undef SGCN_ACT
        if (GATED) {
#pragma unroll
            for (int j = 0; j < 16; ++j) a[j] *= c[j];
        }
    }
    if (P.scale != 1.f) {
#pragma unroll
        for (int j = 0; j < 16; ++j) a[j] *= P.scale;
    }
    if (!PLAIN && P.in) {
        float r[16];
        own_row16(r, slab, lane, h);
#pragma unroll
        for (int j = 0; j < 16; ++j) a[j] += r[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) words[j] = pack2(a[2 * j], a[2 * j + 1]);
}
// Half of 32 columns of da, which takes dout's place in the slab, and of dc, packed; their sums over the warp's rows.
template <bool GATED>
__device__ __forceinline__ void dz_half(const Params& P, const Where& w, int col, int h, float (&a)[16], float (&c)[16], uint32_t* words, uint32_t slab, int lane) {
    float g[16];
    own_row16(g, slab, lane, h);
#define SGCN_ACT(A)                                                       \
    _Pragma("unroll") for (int j = 0; j < 16; ++j) {                      \
        float y, dy;                                                      \
        act_both<false>(A, a[j], y, dy);                                  \
        const float gj = g[j] * P.scale;                                  \
        a[j] = GATED ? gj * c[j] * dy : gj * dy;                          \
        if (GATED) c[j] = gj * y;                                         \
    }
    if (P.act == SLICEGCN_ACT_SILU) {
        SGCN_ACT(SLICEGCN_ACT_SILU)
    } else if (P.act == SLICEGCN_ACT_GELU) {
        SGCN_ACT(SLICEGCN_ACT_GELU)
    } else if (P.act == SLICEGCN_ACT_RELU) {
        SGCN_ACT(SLICEGCN_ACT_RELU)
    } else {
        SGCN_ACT(SLICEGCN_ACT_NONE)
    }
#undef SGCN_ACT
#pragma unroll
    for (int q = 0; q < 2; ++q)
        sts16(own_chunk(slab, lane, 2 * h + q), make_uint4(pack2(a[8 * q], a[8 * q + 1]), pack2(a[8 * q + 2], a[8 * q + 3]), pack2(a[8 * q + 4], a[8 * q + 5]),
                                                           pack2(a[8 * q + 6], a[8 * q + 7])));
    if (GATED) {
#pragma unroll
        for (int j = 0; j < 8; ++j) words[j] = pack2(c[2 * j], c[2 * j + 1]);
    }
    if (P.sums) {
        const int at = col + (lane >> 1);
        const bool mine = !(lane & 1) && at < P.cols && w.rows > 0;
        float* to = P.sums + ((int64_t)(w.row >> 5) * P.slices + w.slice) * P.cols + at;
        const float s = column_sums16(a, lane);
        if (mine) *to = s;
        if (GATED) {
            const float s2 = column_sums16(c, lane);
            if (mine) to[(int64_t)P.p * P.cols] = s2;
        }
    }
}

// ------------------------------------------------------------------------------------------ the product

struct Item {
    int slice, m, n, split;   // slice (times part), first row and column of the tile, piece of k
};
template <int MODE>
__device__ __forceinline__ Item item_of(const Params& P, int i) {
    Item t;
    const int cols = 2 * P.nt;
    const int per_tile = MODE == kFwdGated || MODE == kDzGated ? P.nt : cols;   // columns of D that a tile makes
    if (MODE == kDw) {
        t.split = P.by_first(i);
        i -= t.split * P.by_first.d;
        const int above = P.by_n(i);
        t.n = (i - above * P.tiles_n) * per_tile;
        t.slice = P.by_m(above);
        t.m = (above - t.slice * P.tiles_m) * 256;
    } else {   // `group` row tiles side by side, then the next column tile: operands come from L2 in between
        const int g = P.by_first(i), rest = i - g * P.by_first.d, size = min(P.group, P.tiles_m - g * P.group);
        const int c = size == P.group ? P.by_m(rest) : P.by_last(rest);
        t.m = (g * P.group + rest - c * size) * 256;
        t.slice = P.by_n(c);
        t.n = (c - t.slice * P.tiles_n) * per_tile;
        t.split = 0;
    }
    return t;
}

// PROMO: the accumulator is emptied into registers every P.chunk steps (fp32 digits, or long sums).
template <int MODE, bool PROMO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) ffn_kernel(const __grid_constant__ Params P) {
    constexpr bool kGated = MODE == kFwdGated || MODE == kDzGated;
    constexpr bool kIsDz = MODE == kDz || MODE == kDzGated;
    constexpr bool kAK = MODE != kDw;    // A's k is contiguous
    constexpr bool kBK = MODE == kDx;    // B's
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* tail = smem_raw + (base - smem_u32(smem_raw)) + kStages * kStageBytes + kEpiWarps * (kSlabBytes + kBiasBytes);
    uint64_t* full = reinterpret_cast<uint64_t*>(tail);
    uint64_t* empty = full + kStages;
    uint64_t* tfull = empty + kStages;    // [2]
    uint64_t* tempty = tfull + 2;         // [2]
    uint32_t* tmem_at = reinterpret_cast<uint32_t*>(tempty + 2);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int first = blockIdx.x >> 1, stride = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) mbar_init(full + s, 1), mbar_init(empty + s, 1);
        for (int s = 0; s < 2; ++s) mbar_init(tfull + s, 1), mbar_init(tempty + s, 2 * kEpiWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        fence_before();
    }
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = *tmem_at;
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();

    const int chunks = (P.kb_total + P.chunk - 1) / P.chunk;
    // The two issuing warps walk their loops as whole warps, and one lane issues: what copies and MMAs are given then stays in
    // uniform registers.  (One lane in a loop of its own: 880 cycles per 64-wide step where the MMAs take 512.)
    if (warp == kEpiWarps) {
        const bool one = elect_one();
        bool ok = true;
        int fill = 0, st = 0;
        uint32_t phase = 1;
        const uint32_t bytes = 2u * (16384u + (uint32_t)P.nt * 128u);
        const CUtensorMap* other = kGated && rank ? &P.b1 : &P.b0;
        for (int i = first; ok && i < P.items; i += stride) {
            const Item t = item_of<MODE>(P, i);
            const int row0 = t.m + (int)rank * 128;
            const int slice = MODE == kDw && t.slice >= P.p ? t.slice - P.p : t.slice;
            const int bcol = kGated ? t.n : t.n + (int)rank * P.nt;
            const int k0 = MODE == kDw ? t.split * P.kb_total * 64 : 0;
            for (int c = 0; ok && c < chunks; ++c) {
                const int kb0 = c * P.chunk, kb1 = min(kb0 + P.chunk, P.kb_total);
                for (int q = 0; ok && q < P.pairs; ++q)
                    for (int kb = kb0; kb < kb1; ++kb, ++fill) {
                        ok = __all_sync(0xffffffffu, mbar_wait(empty + st, phase));
                        if (!ok) break;
                        const uint32_t a = base + st * kStageBytes, b = a + 16384u;
                        const bool second = MODE == kDx && kb >= P.kb_part;
                        const int k = k0 + (second ? kb - P.kb_part : kb) * 64;
                        if (one) {
                            if (rank == 0) mbar_expect(full + st, bytes);
                            if (kAK) {
                                tma_load(a, &P.a, k, row0, second ? P.p + slice : slice, P.ia[q], full + st);
                            } else {
                                tma_load(a, &P.a, row0, k, t.slice, P.ia[q], full + st);
                                tma_load(a + 8192, &P.a, row0 + 64, k, t.slice, P.ia[q], full + st);
                            }
                            if (kBK) {
                                tma_load(b, second ? &P.b1 : &P.b0, k, bcol, slice, P.ib[q], full + st);
                            } else {
                                tma_load(b, other, bcol, k, slice, P.ib[q], full + st);
                                if (P.nt > 64) tma_load(b + 8192, other, bcol + 64, k, slice, P.ib[q], full + st);
                            }
                        }
                        __syncwarp();
                        if (++st == kStages) st = 0, phase ^= 1;
                    }
            }
        }
        // the pair's last arrivals at this CTA's barriers, before its memory is given up
        for (int s = max(0, fill - kStages); ok && s < fill; ++s) ok = mbar_wait(empty + s % kStages, (s / kStages) & 1);
        if (!ok && P.status) atomicExch(P.status, SLICEGCN_DEVSTATUS_WAIT);
    } else if (warp == kEpiWarps + 1) {
        if (rank == 0) {
            const bool one = elect_one();
            bool ok = true;
            int use = 0, st = 0;
            uint32_t phase = 0;
            const uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | (kAK ? 0u : 1u << 15) | (kBK ? 0u : 1u << 16) | (uint32_t)(2 * P.nt >> 3) << 17 | 16u << 24;
            for (int i = first; ok && i < P.items; i += stride) {
                for (int c = 0; ok && c < chunks; ++c, ++use) {
                    const int kb0 = c * P.chunk, kb1 = min(kb0 + P.chunk, P.kb_total);
                    const uint32_t d = tmem + (use & 1) * 256;
                    ok = __all_sync(0xffffffffu, mbar_wait(tempty + (use & 1), ((use >> 1) & 1) ^ 1));
                    if (!ok) break;
                    fence_after();
                    bool more = false;
                    for (int q = 0; ok && q < P.pairs; ++q)
                        for (int kb = kb0; kb < kb1; ++kb) {
                            ok = __all_sync(0xffffffffu, mbar_wait(full + st, phase));
                            if (!ok) break;
                            fence_after();
                            const uint32_t at = base + st * kStageBytes;
                            const uint64_t ad = tile_desc(at, kAK), bd = tile_desc(at + 16384u, kBK);
                            const int left = MODE == kDw ? 64 : P.k_part - (kb >= P.kb_part ? kb - P.kb_part : kb) * 64;   // past the end there are only zeros
                            if (one) {
#pragma unroll
                                for (int s = 0; s < 4; ++s)
                                    if (s * 16 < left) umma(d, ad + (uint64_t)(s * (kAK ? 2 : 128)), bd + (uint64_t)(s * (kBK ? 2 : 128)), idesc, s > 0 || more);
                                umma_commit(empty + st);
                            }
                            __syncwarp();
                            more = true;
                            if (++st == kStages) st = 0, phase ^= 1;
                        }
                    if (one) umma_commit(tfull + (use & 1));
                    __syncwarp();
                }
            }
            if (!ok) {   // the copies on their way, before this memory is given up
                for (int s = 0; s < kStages; ++s) {
                    mbar_wait(full + st, phase);
                    if (++st == kStages) st = 0, phase ^= 1;
                }
                if (P.status) atomicExch(P.status, SLICEGCN_DEVSTATUS_WAIT);
            }
        }
    } else {
        const uint32_t slab = base + kStages * kStageBytes + warp * kSlabBytes;
        const uint32_t biases = base + kStages * kStageBytes + kEpiWarps * kSlabBytes + warp * kBiasBytes;
        const int quarter = warp & 3, part = warp >> 2;   // 32 rows of the tile, and a share of its columns
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        // columns of D per warp, and where they start in the accumulator; gated: c's lie nt further on
        const int share = kGated ? (PROMO ? P.nt / 4 : 32) : P.nt / 2;
        const bool busy = part * share < (kGated ? P.nt : 2 * P.nt);
        int use = 0;
        bool ok = true;
        for (int i = first; ok && i < P.items; i += stride) {
            const Item t = item_of<MODE>(P, i);
            Where w;
            w.slice = t.slice;
            w.row = t.m + (int)rank * 128 + quarter * 32;
            w.rows = min(32, max(0, P.n - w.row));
            w.col = t.n + part * share;
            if (PROMO) {
                float acc[64];
#pragma unroll
                for (int j = 0; j < 64; ++j) acc[j] = 0.f;
                for (int c = 0; ok && c < chunks; ++c, ++use) {
                    if (!mbar_wait(tfull + (use & 1), (use >> 1) & 1)) {
                        ok = false;
                        break;
                    }
                    fence_after();
                    const uint32_t d = tmem + (use & 1) * 256 + lanes + part * share;
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        // gated: 16 or 32 columns of a in the first half of the registers, c's in the second
                        const int off = kGated ? (u & 1) * 16 : u * 16;
                        if (off >= share) continue;
                        uint32_t r[16];
                        tmem_ld16(d + off + (kGated && u >= 2 ? P.nt : 0), r);
                        tmem_wait(r);
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[u * 16 + j] += __uint_as_float(r[j]);
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_first(tempty + (use & 1));
                }
                if (!ok) break;
                if (MODE == kDw) {
                    const int f = w.row + lane, fs = P.cols;   // this lane's column of dW; its rows are this tile's columns
                    const int ks = P.k_part;
                    if (f < fs) {
                        if (P.splits > 1) {
                            float* to = P.partial + (((int64_t)t.split * P.slices + t.slice) * ks + w.col) * fs + f;
#pragma unroll
                            for (int j = 0; j < 64; ++j)
                                if (j < share && w.col + j < ks) to[(int64_t)j * fs] = acc[j];
                        } else {
                            const int64_t at = ((int64_t)(t.slice % P.p) * ks + w.col) * fs + f;
                            void* dw = t.slice < P.p ? P.dw : P.dw2;
                            if (dw) {
#pragma unroll
                                for (int j = 0; j < 64; ++j)
                                    if (j < share && w.col + j < ks) {
                                        const float v = acc[j] * P.scale;
                                        if (P.out_bf16)
                                            static_cast<__nv_bfloat16*>(dw)[at + (int64_t)j * fs] = __float2bfloat16_rn(v);
                                        else
                                            static_cast<float*>(dw)[at + (int64_t)j * fs] = v;
                                    }
                            }
                        }
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < (kGated ? 2 : 4); ++u) {
                        if (u * 16 >= share) continue;
                        const int col = w.col + u * 16;
                        if (col >= P.cols || w.rows <= 0) continue;
                        float a[16], cc[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) a[j] = acc[u * 16 + j], cc[j] = kGated ? acc[(32 + u * 16 + j) & 63] : 0.f;
                        if (MODE == kDz || MODE == kDzGated)
                            finish_dz<kGated, true>(P, w, col, a, cc, slab, lane);
                        else
                            finish_forward<16, kGated, true>(P, w, col, a, cc, slab, lane);
                    }
                }
            } else {
                // what the columns need besides the product is on its way while the product is waited for
                const int units = busy ? share / 32 : 0;
                float bias[2] = {0.f, 0.f}, bias2 = 0.f;
                uint4 raw[4];
                const bool with_in = kIsDz || (MODE != kDx && P.in);
                if (units > 0) {
                    const int64_t bat = (int64_t)t.slice * P.cols;
                    if (MODE != kDx) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int c = w.col + u * 32 + lane;
                            if (u < units && P.b && c < P.cols) bias[u] = __ldg(P.b + bat + c);
                        }
                        if (kGated && P.b2 && w.col + lane < P.cols) bias2 = __ldg(P.b2 + bat + w.col + lane);
                    }
                    if (with_in) load_in(P, w, w.col, raw, lane);
                }
                if (!mbar_wait(tfull + (use & 1), (use >> 1) & 1)) {
                    ok = false;
                    break;
                }
                fence_after();
                const uint32_t d = tmem + (use & 1) * 256 + lanes + part * share;
                for (int u = 0; u < units; ++u) {
                    const int col = w.col + u * 32;
                    const bool last = u == units - 1, there = col < P.cols && w.rows > 0;
                    uint32_t ra[16], rc[16];
                    tmem_ld16(d + u * 32, ra);
                    if (kGated) tmem_ld16(d + u * 32 + P.nt, rc);
                    if (MODE != kDx) {
                        __syncwarp();
                        sts4(biases + lane * 4, u ? bias[1] : bias[0]);
                        if (kGated) sts4(biases + 128 + lane * 4, bias2);
                    }
                    if (with_in) put_in(P, w, col, raw, slab, lane);
                    __syncwarp();
                    tmem_wait(ra);
                    if (kGated) after_wait(rc);
                    uint32_t words[16], words2[16];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t na[16], nc[16];
                        if (h == 0) {   // the second half's numbers come while the first half's are worked on
                            tmem_ld16(d + u * 32 + 16, na);
                            if (kGated) tmem_ld16(d + u * 32 + 16 + P.nt, nc);
                        }
                        float a[16], c[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) a[j] = __uint_as_float(ra[j]), c[j] = kGated ? __uint_as_float(rc[j]) : 0.f;
                        if (MODE != kDx) {
                            add16(a, biases + h * 64);
                            if (kGated) add16(c, biases + 128 + h * 64);
                        }
                        if constexpr (kIsDz)
                            dz_half<kGated>(P, w, col + 16 * h, h, a, c, words2 + 8 * h, slab, lane);
                        else
                            forward_half<kGated, MODE == kDx>(P, h, a, c, words + 8 * h, slab, lane);
                        if (h == 0) {
                            tmem_wait(na);
                            if (kGated) after_wait(nc);
                            if (last) {
                                fence_before();
                                __syncwarp();
                                if (lane == 0) mbar_arrive_first(tempty + (use & 1));
                            }
#pragma unroll
                            for (int j = 0; j < 16; ++j) ra[j] = na[j], rc[j] = kGated ? nc[j] : 0u;
                        }
                    }
                    if (with_in && !last) load_in(P, w, col + 32, raw, lane);
                    if constexpr (kIsDz) {
                        if (there) {
                            __nv_bfloat16* at = P.dz + (int64_t)w.row * P.dz_row + (int64_t)w.slice * P.dz_pad + col;
                            __syncwarp();
                            slab_out(reinterpret_cast<char*>(at), P.dz_row * 2, w.rows, P.dz_pad - col, true, slab, lane);
                            if (kGated) {
                                __syncwarp();
                                put_rows(words2, slab, lane);
                                __syncwarp();
                                slab_out(reinterpret_cast<char*>(at + (int64_t)P.p * P.dz_pad), P.dz_row * 2, w.rows, P.dz_pad - col, true, slab, lane);
                            }
                        }
                    } else if (there) {
                        __syncwarp();
                        put_rows(words, slab, lane);
                        __syncwarp();
                        slab_out(static_cast<char*>(P.out) + ((int64_t)w.row * P.out_ld + (int64_t)w.slice * P.cols + col) * 2, P.out_ld * 2, w.rows, P.cols - col,
                                 P.out_vec, slab, lane);
                    }
                }
                if (units == 0 && lane == 0) mbar_arrive_first(tempty + (use & 1));
                ++use;
            }
        }
        if (!ok && lane == 0 && P.status) atomicExch(P.status, SLICEGCN_DEVSTATUS_WAIT);
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    cluster_sync();
    if (warp == 0) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// ------------------------------------------------------------------------------------------ small kernels

// A matrix of rows x groups x width (row stride ld) as bf16 planes [plane][row][group][pad], pad the next multiple of 8 (filled with
// zeros): fp32 as three planes, bf16 as one.  A thread makes 16 bytes of each plane.
struct PackArgs {
    const void* src;
    int64_t ld, rows, plane;
    int groups, width, pad, bf16;
    __nv_bfloat16* dst;
};
__global__ void __launch_bounds__(256) ffn_pack_kernel(const __grid_constant__ PackArgs A) {
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    const int per_group = A.pad / 8, per_row = per_group * A.groups;
    const int64_t total = A.rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row;
        const int in_row = (int)(i - row * per_row), g = in_row / per_group, c = (in_row - g * per_group) * 8;
        const int64_t at = row * A.ld + (int64_t)g * A.width + c;
        const int left = A.width - c;
        uint4 out[3];
        if (A.bf16) {
            const uint16_t* s = static_cast<const uint16_t*>(A.src) + at;
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = (2 * k < left ? (uint32_t)s[2 * k] : 0u) | (2 * k + 1 < left ? (uint32_t)s[2 * k + 1] << 16 : 0u);
            out[0] = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            const float* s = static_cast<const float*>(A.src) + at;
            uint32_t w[3][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float lo[3], hi[3];
                split3(2 * k < left ? s[2 * k] : 0.f, lo);
                split3(2 * k + 1 < left ? s[2 * k + 1] : 0.f, hi);
#pragma unroll
                for (int q = 0; q < 3; ++q) w[q][k] = __float_as_uint(lo[q]) >> 16 | (__float_as_uint(hi[q]) & 0xffff0000u);
            }
#pragma unroll
            for (int q = 0; q < 3; ++q) out[q] = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
        }
        __nv_bfloat16* d = A.dst + i * 8;
        *reinterpret_cast<uint4*>(d) = out[0];
        if (!A.bf16) {
            *reinterpret_cast<uint4*>(d + A.plane) = out[1];
            *reinterpret_cast<uint4*>(d + 2 * A.plane) = out[2];
        }
    }
}

// Sums of columns, in a fixed order: chunks of rows by the first kernel, the chunks by the second.
constexpr int kSumChunks = 128;
struct SumArgs {
    const void* src;
    int64_t rows, ld, per;    // rows of a chunk
    int cols, bf16;
    float* partial;           // [chunks][cols]
};
__global__ void __launch_bounds__(256) ffn_colsum_kernel(const __grid_constant__ SumArgs A) {
    __shared__ float sh[8][33];
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    const int64_t r0 = blockIdx.y * A.per, r1 = min(r0 + A.per, A.rows);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < A.cols) {
        int64_t r = r0 + y;
        for (; r + 24 < r1; r += 32) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t at = (r + 8 * k) * A.ld + c;
                s[k] += A.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(A.src)[at]) : static_cast<const float*>(A.src)[at];
            }
        }
        for (; r < r1; r += 8) {
            const int64_t at = r * A.ld + c;
            s[0] += A.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(A.src)[at]) : static_cast<const float*>(A.src)[at];
        }
    }
    sh[y][x] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (y == 0 && c < A.cols) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) t += sh[k][x];
        A.partial[(int64_t)blockIdx.y * A.cols + c] = t;
    }
}
// out[0][i] (i < each) and out[1][i - each] = scale * the sum over `count` pieces of `total` numbers each
struct JoinArgs {
    const float* partial;
    int count, bf16;
    int64_t total, each;
    float scale;
    void* out[2];
};
__global__ void __launch_bounds__(256) ffn_join_kernel(const __grid_constant__ JoinArgs A) {
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < A.total; i += (int64_t)gridDim.x * 256) {
        const int second = i >= A.each;
        if (!A.out[second]) continue;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        int k = 0;
        for (; k + 4 <= A.count; k += 4)
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] += A.partial[(k + q) * A.total + i];
        for (; k < A.count; ++k) s[0] += A.partial[k * A.total + i];
        const float v = ((s[0] + s[1]) + (s[2] + s[3])) * A.scale;
        const int64_t at = second ? i - A.each : i;
        if (A.bf16)
            static_cast<__nv_bfloat16*>(A.out[second])[at] = __float2bfloat16_rn(v);
        else
            static_cast<float*>(A.out[second])[at] = v;
    }
}

// ------------------------------------------------------------------------------------------ host

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// An operand: bf16, [plane][row][group][width] by strides in elements (multiples of 8 where there is more than one).
struct Operand {
    const void* base = nullptr;
    int64_t rows = 0, ld = 0, group_stride = 0, plane_stride = 0;
    int width = 0, groups = 1, planes = 1;
};
slicegcn_status_t make_map(CUtensorMap* map, const Operand& o, int box_rows) {
    static EncodeFn encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
            fn = nullptr;
        return reinterpret_cast<EncodeFn>(fn);
    }();
    if (!encode) SGCN_FAIL(SLICEGCN_ERR_CUDA, "ffn: the driver has no tensor map encoder");
    const cuuint64_t dims[4] = {(cuuint64_t)o.width, (cuuint64_t)o.rows, (cuuint64_t)o.groups, (cuuint64_t)o.planes};
    const cuuint64_t strides[3] = {(cuuint64_t)(o.rows > 1 ? o.ld : 8) * 2, (cuuint64_t)(o.groups > 1 ? o.group_stride : 8) * 2,
                                   (cuuint64_t)(o.planes > 1 ? o.plane_stride : 8) * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 1, 1}, ones[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(o.base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) SGCN_FAIL(SLICEGCN_ERR_CUDA, "ffn: tensor map refused (%d)", (int)r);
    return SLICEGCN_OK;
}

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// What a call needs in the workspace, and where.
struct Plan {
    bool pack_x = false, pack_w = false, pack_g = false, dz = false;
    int x_planes = 1, w_planes = 1, z_planes = 1;
    int in_pad = 0, out_pad = 0, parts = 1, splits = 1, dw_nt = 128;
    int64_t x_at = 0, w_at = 0, w2_at = 0, z_at = 0, sums_at = 0, chunks_at = 0, partial_at = 0, bytes = 0;
};

bool unaligned(const void* p, int64_t ld, int groups, int width) {
    return (uintptr_t)p % 16 || ld % 8 || (groups > 1 && width % 8);
}

// Pieces of the rows for dW: as many as fill the pairs of SMs evenly, if each still is 1,024 rows or more and their sums stay a
// fraction of what is read.
int splits_of(int64_t tiles, int64_t n) {
    int best = 1;
    double cost = 1e300;
    for (int s = 1; s <= 148; ++s) {
        if (s > 1 && n / s < 1024) break;
        const double c = (double)((tiles * s + kPairs - 1) / kPairs) / s * (1.0 + 0.004 * s);
        if (c < cost) cost = c, best = s;
    }
    return best;
}

void plan(const slicegcn_ffn_desc* d, const void* x, const void* dout, Plan& q) {
    const int64_t n = d->n;
    const int p = d->num_slices;
    const bool f32 = d->dtype == SLICEGCN_F32, back = dout != nullptr;
    q.parts = d->W2 ? 2 : 1;
    q.in_pad = (int)up(d->in_s, 8);
    q.out_pad = (int)up(d->out_s, 8);
    q.x_planes = q.w_planes = f32 ? 3 : 1;
    q.z_planes = d->grad_dtype == SLICEGCN_F32 ? 3 : 1;
    q.pack_x = f32 || unaligned(x, d->x_ld, p, d->in_s);
    q.pack_w = f32 || unaligned(d->W, d->out_s, 1, 8) || unaligned(d->W2, d->out_s, 1, 8);
    q.dz = back && (d->act != SLICEGCN_ACT_NONE || d->W2);
    q.pack_g = back && !q.dz && (q.z_planes == 3 || unaligned(dout, d->dout_ld, p, d->out_s));
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    if (q.pack_x) q.x_at = take(2 * q.x_planes * n * p * q.in_pad);
    if (q.pack_w) {
        q.w_at = take(2LL * q.w_planes * p * d->in_s * q.out_pad);
        if (d->W2) q.w2_at = take(2LL * q.w_planes * p * d->in_s * q.out_pad);
    }
    if (back) {
        const int64_t cols = (int64_t)q.parts * p * d->out_s;
        if (q.dz || q.pack_g) q.z_at = take(2 * q.z_planes * n * q.parts * p * q.out_pad);
        if (q.dz) q.sums_at = take(4 * ((n + 31) / 32) * cols);
        q.chunks_at = take(4 * kSumChunks * cols);
        q.dw_nt = d->in_s <= 128 ? 64 : 128;
        q.splits = splits_of((int64_t)q.parts * p * ceil_div(d->out_s, 256) * ceil_div(d->in_s, 2 * q.dw_nt), n);
        if (q.splits > 1) q.partial_at = take(4LL * q.splits * d->in_s * cols);
    }
    q.bytes = at;
}

slicegcn_status_t check(const slicegcn_ffn_desc* d) {
    if (!d || d->n < 0 || d->num_slices < 1 || d->in_s < 1 || d->out_s < 1) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: bad description");
    if (d->num_slices > SLICEGCN_MAX_SLICES || d->in_s > SLICEGCN_MAX_FFN_WIDTH || d->out_s > SLICEGCN_MAX_FFN_WIDTH)
        SGCN_FAIL(SLICEGCN_ERR_UNSUPPORTED, "ffn: %d slices of %d and %d columns, at most %d of %d", d->num_slices, d->in_s, d->out_s, SLICEGCN_MAX_SLICES,
                  SLICEGCN_MAX_FFN_WIDTH);
    if (d->n > INT32_MAX - 16384) SGCN_FAIL(SLICEGCN_ERR_OVERFLOW, "ffn: too many rows");
    if (d->act < SLICEGCN_ACT_NONE || d->act > SLICEGCN_ACT_GELU) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: bad act");
    if ((d->dtype != SLICEGCN_F32 && d->dtype != SLICEGCN_BF16) || (d->grad_dtype != SLICEGCN_F32 && d->grad_dtype != SLICEGCN_BF16))
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: bad dtype");
    if (d->dtype == SLICEGCN_F32 && d->grad_dtype != SLICEGCN_F32) SGCN_FAIL(SLICEGCN_ERR_UNSUPPORTED, "ffn: fp32 with bf16 gradients");
    if (!std::isfinite(d->scale)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: scale is not finite");
    const uintptr_t e = d->dtype == SLICEGCN_F32 ? 4 : 2;
    if (!d->W || (uintptr_t)d->W % e || (uintptr_t)d->W2 % e || (uintptr_t)d->b % 4 || (uintptr_t)d->b2 % 4)
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: W is NULL, or a weight or bias is not aligned to its type");
    if (d->b2 && !d->W2) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: b2 without W2");
    return SLICEGCN_OK;
}
slicegcn_status_t check_matrix(const char* name, const void* p, int64_t ld, int64_t cols, int dtype, bool needed) {
    if (!p && needed) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: %s is NULL", name);
    if (!p) return SLICEGCN_OK;
    if (ld < cols) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: leading dimension of %s too small", name);
    if (ld > ((int64_t)1 << 38)) SGCN_FAIL(SLICEGCN_ERR_OVERFLOW, "ffn: leading dimension of %s too large", name);
    if ((uintptr_t)p % (dtype == SLICEGCN_F32 ? 4 : 2)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: %s is not aligned to its type", name);
    return SLICEGCN_OK;
}
slicegcn_status_t check_workspace(const void* ws, int64_t have, int64_t need, const int32_t* status) {
    if ((uintptr_t)ws % 128 || (uintptr_t)status % 4) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: the workspace (128 bytes) or status is not aligned");
    if (need > 0 && (!ws || have < need)) SGCN_FAIL(SLICEGCN_ERR_ALLOC, "ffn: workspace too small (%lld < %lld bytes)", (long long)have, (long long)need);
    return SLICEGCN_OK;
}

slicegcn_status_t pack(const void* src, int64_t ld, int64_t rows, int groups, int width, bool bf16, void* dst, Operand& o, cudaStream_t st) {
    PackArgs A;
    A.src = src, A.ld = ld, A.rows = rows, A.groups = groups, A.width = width, A.pad = (int)up(width, 8), A.bf16 = bf16;
    A.plane = rows * groups * A.pad;
    A.dst = static_cast<__nv_bfloat16*>(dst);
    o.base = dst, o.rows = rows, o.ld = (int64_t)groups * A.pad, o.group_stride = A.pad, o.plane_stride = A.plane;
    o.width = width, o.groups = groups, o.planes = bf16 ? 1 : 3;
    const int64_t chunks = A.plane / 8;
    const int ctas = (int)std::min<int64_t>((chunks + 255) / 256, 148 * 16);
    return launch_after(ffn_pack_kernel, dim3(ctas), 256, 0, st, A);
}

// Products of operand parts, the smallest first.
void set_pairs(Params& P, int pa, int pb) {
    P.pairs = 0;
    for (int order = 2; order >= 0; --order)
        for (int i = std::min(order, pa - 1); i >= 0; --i)
            if (order - i < pb) P.ia[P.pairs] = (int8_t)i, P.ib[P.pairs] = (int8_t)(order - i), ++P.pairs;
}

template <int MODE, bool PROMO>
slicegcn_status_t launch(const Params& P, cudaStream_t st) {
    SGCN_CUDA(cudaFuncSetAttribute(ffn_kernel<MODE, PROMO>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem));
    return launch_after(ffn_kernel<MODE, PROMO>, dim3(2 * std::min(P.items, kPairs)), kThreads, kSmem, st, P);
}

// Steps between emptyings: fp32's digits allow 256 k (16 additions in tensor memory); bf16 results only need it for long sums.
constexpr int kChunkF32 = 4, kChunkLong = 64;

// Tiles of a product over the rows of x; columns of B per CTA by what wastes least: half-width tiles where they cover the columns,
// or where whole ones would leave pairs of SMs idle.
void set_tiles(Params& P, int64_t n, int p, int cols, bool gated) {
    const int one = gated ? 64 : 128;
    P.n = (int)n, P.p = P.slices = p, P.cols = cols;
    P.tiles_m = ceil_div(n, 256);
    P.nt = cols <= one || (int64_t)P.tiles_m * p * ceil_div(cols, 2 * one) * 2 <= kPairs ? 64 : 128;
    P.tiles_n = ceil_div(cols, gated ? P.nt : 2 * P.nt);
    P.group = std::min(P.tiles_m, 8);
    P.splits = 1;
}

slicegcn_status_t item_count(Params& P) {
    const int64_t items = (int64_t)P.slices * P.tiles_m * P.tiles_n * P.splits;
    if (items > (1 << 30)) SGCN_FAIL(SLICEGCN_ERR_OVERFLOW, "ffn: too many tiles");
    P.items = (int)items;
    P.by_n = divide_by(P.tiles_n);
    if (P.splits_rows) {
        P.by_first = divide_by(P.slices * P.tiles_m * P.tiles_n);
        P.by_m = P.by_last = divide_by(P.tiles_m);
    } else {
        P.by_first = divide_by(P.group * P.slices * P.tiles_n);
        P.by_m = divide_by(P.group);
        P.by_last = divide_by(std::max(1, P.tiles_m % P.group));
    }
    return SLICEGCN_OK;
}

// x, W and W2 as operands, laid out anew where they have to be.
slicegcn_status_t operands(const slicegcn_ffn_desc* d, const Plan& q, const void* x, char* ws, Operand& ox, Operand& ow, Operand& ow2, cudaStream_t st) {
    const bool bf16 = d->dtype == SLICEGCN_BF16;
    const int p = d->num_slices;
    if (q.pack_x) {
        SGCN_TRY(pack(x, d->x_ld, d->n, p, d->in_s, bf16, ws + q.x_at, ox, st));
    } else {
        ox.base = x, ox.rows = d->n, ox.ld = d->x_ld, ox.group_stride = d->in_s, ox.width = d->in_s, ox.groups = p;
    }
    for (int k = 0; k < q.parts; ++k) {
        Operand& o = k ? ow2 : ow;
        const void* w = k ? d->W2 : d->W;
        if (q.pack_w) {
            SGCN_TRY(pack(w, d->out_s, (int64_t)p * d->in_s, 1, d->out_s, bf16, ws + (k ? q.w2_at : q.w_at), o, st));
            o.groups = p, o.rows = d->in_s, o.group_stride = (int64_t)d->in_s * q.out_pad;
        } else {
            o.base = w, o.rows = d->in_s, o.ld = d->out_s, o.group_stride = (int64_t)d->in_s * d->out_s, o.width = d->out_s, o.groups = p;
        }
    }
    return SLICEGCN_OK;
}

// The product a = x W (and c = x W2) and its epilogue.
slicegcn_status_t forward_product(Params& P, const slicegcn_ffn_desc* d, const Plan& q, const Operand& ox, const Operand& ow, const Operand& ow2, bool back,
                                  cudaStream_t st) {
    const bool gated = d->W2 != nullptr, promo = d->dtype == SLICEGCN_F32 || (back && d->grad_dtype == SLICEGCN_F32);
    set_tiles(P, d->n, d->num_slices, d->out_s, gated);
    SGCN_TRY(item_count(P));
    SGCN_TRY(make_map(&P.a, ox, 128));
    SGCN_TRY(make_map(&P.b0, ow, 64));
    SGCN_TRY(make_map(&P.b1, gated ? ow2 : ow, 64));
    P.kb_total = P.kb_part = ceil_div(d->in_s, 64);
    P.k_part = d->in_s;
    set_pairs(P, q.x_planes, q.w_planes);
    P.chunk = P.pairs > 1 ? kChunkF32 : P.kb_total;
    P.act = d->act, P.scale = (float)d->scale, P.b = d->b, P.b2 = d->b2;
    if (back) {
        P.slices = q.parts * d->num_slices;   // of the sums
        if (gated) return promo ? launch<kDzGated, true>(P, st) : launch<kDzGated, false>(P, st);
        return promo ? launch<kDz, true>(P, st) : launch<kDz, false>(P, st);
    }
    if (gated) return promo ? launch<kFwdGated, true>(P, st) : launch<kFwdGated, false>(P, st);
    return promo ? launch<kFwd, true>(P, st) : launch<kFwd, false>(P, st);
}

bool wide_access(const void* p, int64_t ld, int elem, int groups, int width) {
    return (uintptr_t)p % 16 == 0 && ld * elem % 16 == 0 && (groups == 1 || width * elem % 16 == 0);
}

}  // namespace
}  // namespace sgcn

using namespace sgcn;

extern "C" {

slicegcn_status_t slicegcn_ffn_workspace_bytes(const slicegcn_ffn_desc* d, const void* x, const void* dout, int64_t* bytes) {
    SGCN_TRY(check(d));
    if (!bytes || (!x && d->n > 0)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn_workspace_bytes: NULL argument");
    if (d->x_ld < (int64_t)d->num_slices * d->in_s || (dout && d->dout_ld < (int64_t)d->num_slices * d->out_s))
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn_workspace_bytes: leading dimension too small");
    *bytes = 0;
    if (d->n == 0) return SLICEGCN_OK;
    Plan q;
    plan(d, x, dout, q);
    *bytes = q.bytes;
    return SLICEGCN_OK;
}

slicegcn_status_t slicegcn_ffn_forward(const slicegcn_ffn_desc* d, const void* x, const void* r, void* out, int32_t* status, void* workspace,
                                       int64_t workspace_bytes, void* stream) {
    SGCN_TRY(check(d));
    const int p = d->num_slices, e = d->dtype == SLICEGCN_F32 ? 4 : 2;
    const int64_t ins = (int64_t)p * d->in_s, outs = (int64_t)p * d->out_s;
    const bool some = d->n > 0;
    SGCN_TRY(check_matrix("x", x, d->x_ld, ins, d->dtype, some));
    SGCN_TRY(check_matrix("r", r, d->r_ld, outs, d->dtype, false));
    SGCN_TRY(check_matrix("out", out, d->out_ld, outs, d->dtype, some));
    Plan q;
    if (some) plan(d, x, nullptr, q);
    SGCN_TRY(check_workspace(workspace, workspace_bytes, q.bytes, status));
    if (!some) return SLICEGCN_OK;
    cudaStream_t st = (cudaStream_t)stream;
    Operand ox, ow, ow2;
    SGCN_TRY(operands(d, q, x, static_cast<char*>(workspace), ox, ow, ow2, st));
    Params P = {};
    P.status = status;
    P.in = r, P.in_ld = d->r_ld, P.in_bf16 = e == 2, P.in_vec = r && wide_access(r, d->r_ld, e, p, d->out_s);
    P.out = out, P.out_ld = d->out_ld, P.out_bf16 = e == 2, P.out_vec = wide_access(out, d->out_ld, e, p, d->out_s);
    return forward_product(P, d, q, ox, ow, ow2, false, st);
}

slicegcn_status_t slicegcn_ffn_backward(const slicegcn_ffn_desc* d, const void* x, const void* dout, void* dx, void* dW, void* dW2, float* db,
                                        float* db2, int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
    SGCN_TRY(check(d));
    const int p = d->num_slices, ge = d->grad_dtype == SLICEGCN_F32 ? 4 : 2;
    const int64_t n = d->n, ins = (int64_t)p * d->in_s, outs = (int64_t)p * d->out_s;
    const bool some = n > 0;
    SGCN_TRY(check_matrix("x", x, d->x_ld, ins, d->dtype, some));
    SGCN_TRY(check_matrix("dout", dout, d->dout_ld, outs, d->grad_dtype, some));
    SGCN_TRY(check_matrix("dx", dx, d->dx_ld, ins, d->grad_dtype, false));
    if ((uintptr_t)dW % ge || (uintptr_t)dW2 % ge || (uintptr_t)db % 4 || (uintptr_t)db2 % 4)
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: a gradient is not aligned to its type");
    if ((dW2 || db2) && !d->W2) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: gradients of W2 or b2 without W2");
    Plan q;
    if (some) plan(d, x, dout, q);
    SGCN_TRY(check_workspace(workspace, workspace_bytes, q.bytes, status));
    cudaStream_t st = (cudaStream_t)stream;
    if (!some) {
        if (dW) SGCN_CUDA(cudaMemsetAsync(dW, 0, (size_t)(d->in_s * outs * ge), st));
        if (dW2) SGCN_CUDA(cudaMemsetAsync(dW2, 0, (size_t)(d->in_s * outs * ge), st));
        if (db) SGCN_CUDA(cudaMemsetAsync(db, 0, (size_t)(outs * 4), st));
        if (db2) SGCN_CUDA(cudaMemsetAsync(db2, 0, (size_t)(outs * 4), st));
        return SLICEGCN_OK;
    }
    char* ws = static_cast<char*>(workspace);
    Operand ox, ow, ow2, oz;
    SGCN_TRY(operands(d, q, x, ws, ox, ow, ow2, st));
    const bool sums = db || db2;
    const float scale = q.dz ? 1.f : (float)d->scale;   // what the products still have to be multiplied by
    if (q.dz) {
        Params P = {};
        P.status = status;
        P.in = dout, P.in_ld = d->dout_ld, P.in_bf16 = ge == 2, P.in_vec = wide_access(dout, d->dout_ld, ge, p, d->out_s);
        P.dz = reinterpret_cast<__nv_bfloat16*>(ws + q.z_at);
        P.dz_row = (int64_t)q.parts * p * q.out_pad, P.dz_plane = n * P.dz_row, P.dz_planes = q.z_planes, P.dz_pad = q.out_pad;
        P.sums = sums ? reinterpret_cast<float*>(ws + q.sums_at) : nullptr;
        SGCN_TRY(forward_product(P, d, q, ox, ow, ow2, true, st));
        oz.base = P.dz, oz.rows = n, oz.ld = P.dz_row, oz.group_stride = q.out_pad, oz.plane_stride = P.dz_plane;
        oz.width = d->out_s, oz.groups = q.parts * p, oz.planes = q.z_planes;
    } else if (q.pack_g) {
        SGCN_TRY(pack(dout, d->dout_ld, n, p, d->out_s, ge == 2, ws + q.z_at, oz, st));
    } else {
        oz.base = dout, oz.rows = n, oz.ld = d->dout_ld, oz.group_stride = d->out_s, oz.width = d->out_s, oz.groups = p;
    }
    if (dx) {
        Params P = {};
        P.status = status;
        set_tiles(P, n, p, d->in_s, false);
        SGCN_TRY(item_count(P));
        SGCN_TRY(make_map(&P.a, oz, 128));
        SGCN_TRY(make_map(&P.b0, ow, P.nt));
        SGCN_TRY(make_map(&P.b1, q.parts == 2 ? ow2 : ow, P.nt));
        P.kb_part = ceil_div(d->out_s, 64), P.kb_total = P.kb_part * q.parts, P.k_part = d->out_s;
        set_pairs(P, q.z_planes, q.w_planes);
        const bool promo = P.pairs > 1;
        P.chunk = promo ? kChunkF32 : P.kb_total;
        P.act = SLICEGCN_ACT_NONE, P.scale = scale;
        P.out = dx, P.out_ld = d->dx_ld, P.out_bf16 = ge == 2, P.out_vec = wide_access(dx, d->dx_ld, ge, p, d->in_s);
        SGCN_TRY((promo ? launch<kDx, true>(P, st) : launch<kDx, false>(P, st)));
    }
    if (dW || dW2) {
        Params P = {};
        P.status = status;
        P.n = d->out_s, P.p = p, P.slices = q.parts * p, P.cols = d->out_s, P.k_part = d->in_s;
        P.nt = q.dw_nt, P.tiles_m = ceil_div(d->out_s, 256), P.tiles_n = ceil_div(d->in_s, 2 * P.nt), P.group = 1;
        P.kb_total = P.kb_part = ceil_div(ceil_div(n, 64), q.splits);
        P.splits = q.splits, P.splits_rows = 1;
        SGCN_TRY(item_count(P));
        SGCN_TRY(make_map(&P.a, oz, 64));
        SGCN_TRY(make_map(&P.b0, ox, 64));
        P.b1 = P.b0;
        set_pairs(P, q.z_planes, q.x_planes);
        P.chunk = P.pairs > 1 ? kChunkF32 : kChunkLong;
        P.scale = scale, P.out_bf16 = ge == 2;
        P.partial = reinterpret_cast<float*>(ws + q.partial_at);
        P.dw = dW, P.dw2 = dW2;
        SGCN_TRY((launch<kDw, true>(P, st)));
        if (q.splits > 1) {
            JoinArgs J = {P.partial, q.splits, ge == 2, (int64_t)q.parts * d->in_s * outs, d->in_s * outs, scale, {dW, dW2}};
            SGCN_TRY(launch_after(ffn_join_kernel, dim3((unsigned)std::min<int64_t>((J.total + 255) / 256, 148 * 8)), 256, 0, st, J));
        }
    }
    if (sums) {
        SumArgs A;
        A.src = q.dz ? (const void*)(ws + q.sums_at) : dout;
        A.rows = q.dz ? (n + 31) / 32 : n;
        A.cols = (int)(q.parts * outs);
        A.ld = q.dz ? A.cols : d->dout_ld;
        A.bf16 = !q.dz && ge == 2;
        const int chunks = (int)std::min<int64_t>(kSumChunks, std::max<int64_t>(1, A.rows / 32));
        A.per = (A.rows + chunks - 1) / chunks;
        A.partial = reinterpret_cast<float*>(ws + q.chunks_at);
        SGCN_TRY(launch_after(ffn_colsum_kernel, dim3(ceil_div(A.cols, 32), chunks), 256, 0, st, A));
        JoinArgs J = {A.partial, chunks, 0, A.cols, outs, scale, {db, db2}};
        SGCN_TRY(launch_after(ffn_join_kernel, dim3(ceil_div(J.total, 256)), 256, 0, st, J));
    }
    return SLICEGCN_OK;
}

}  // extern "C"
