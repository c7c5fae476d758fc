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
//   * fp32 values are three bf16 numbers (8 bits of the significand each, all 24 from 2^-110 up), and a product of two of them is the six products
//     of parts that reach fp32's last digit, the small ones first, each tile of parts copied once.  A sixth of the bf16 rate.
//   * Tensor memory's accumulation cuts digits off; over k in the hundreds of 16-wide steps that would show in fp32.  There the
//     accumulator is emptied into registers every few steps ("chunk"), and the registers are added to with rounding.
//   * Two accumulators: the sixteen epilogue warps work on one while the MMA fills the other.
//   * The gate needs no second pass: the two halves of B are columns of W and of W2, so a and c of the same columns
//     meet in the same thread.
//   * dW = x^T da runs over rows; they are split over the SMs, and the pieces' sums are added in a fixed order.
//   * Narrow slices are computed together, their weights as one block-diagonal matrix.  Up to eight rows, and little work in
//     layouts that the tensor cores cannot read, go by plain multiply-adds (further down).
#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "common.cuh"

namespace sgcn {
namespace {

constexpr int kPairs = 74;                       // pairs of SMs
constexpr int kStages = 5, kStageBytes = 32768;  // A: 128 x 64 bf16, B: up to 128 x 64
constexpr int kEpiWarps = 16, kThreads = (kEpiWarps + 2) * 32;
constexpr int kSlabBytes = 4096;                 // of an epilogue warp: twice 32 rows x 64 bytes
constexpr int kSmem = kStages * kStageBytes + kEpiWarps * kSlabBytes + 1024 + 256;
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
    CUtensorMap a, b0, b1, o;      // o: bf16 results, da and dc
    int n;                         // rows of x
    int p, slices;                 // slices; slices times parts of the output (kDw), else the same
    int tiles_m, tiles_n, group;   // per slice; m tiles that follow one another before the next n tile
    Divide by_split, by_group, by_n, by_m, by_last;   // what item_of divides by
    int items, clusters;
    int nt;                        // columns of B per CTA: 64 or 128
    int kb_total, kb_part, k_part; // 64-wide steps of an item, of one part of k, and that part's extent
    int chunk;                     // steps between emptyings of the accumulator
    int a_planes, b_planes;        // 3: parts of fp32
    int splits;                    // pieces of k (kDw: of the rows), kb_total steps each
    int swapped, pair;             // kDw: a tile's rows are dW's; and its column halves are dW's and dW2's
    // epilogue
    int cols;                      // columns of D per slice
    float scale;
    const float *b, *b2;           // [slices][cols]
    int bias_vec;                  // two of them at a time are aligned
    const void* in;                // r or dout
    int in_ld;
    int in_bf16, in_vec, in_pairs; // vec: 16 bytes at a time are aligned; pairs: 8
    void* out;
    int out_ld;
    int out_bf16, out_vec, out_pairs;   // vec: tensor copies reach it; pairs: 8 bytes at a time are aligned
    int out_edge;                  // columns from here on are stored one by one: a tensor copy writes whole 16 bytes
    int planes;                    // kDz, emptied into registers: of da and dc
    int fixed;                     // every pair of SMs stays with one column tile
    // kDz: sums over 32 rows each, or (fixed) over all rows that an epilogue warp has seen
    float* sums;                   // [ceil(n/32) or epilogue warps per column tile][parts * p][cols], or NULL
    float* partial;                // pieces' products, where they are joined by another kernel; kDw: [splits][slices][in_s][out_s], else [splits][slices][n][cols]
    int matrices;                  // kDw: slices times parts
    void *dw, *dw2;                // kDw, splits == 1
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
// Arrives at the same barrier of the pair's first CTA.  Relaxed: what it hands over are accumulators that have been read into registers (the
// wait for those reads is behind this thread, and so is its tcgen05 fence, whose other half follows the issuing warp's wait); no data in
// memory goes with it.  A release would first wait for all results the warp has stored (17 % of all warp stalls; 157 and 219 us for the gated
// forward of 169,343 x 256 -> 2 x 1,024).
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
// One box of shared memory to a tensor map; what lies outside the tensor is left out, but a row's end only from the next 16 bytes on.  Groups of them are waited for by the lane that
// issued them; a turn without a box commits its (empty) group too, since the waits count groups.
__device__ __forceinline__ void tma_store(const CUtensorMap* map, uint32_t src, int x, int y, int z, int w) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(map), "r"(src),
                 "r"(x), "r"(y), "r"(z), "r"(w)
                 : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
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
__device__ __forceinline__ void tmem_rows(uint32_t addr, float (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
          "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
        : "r"(addr)
        : "memory");
}
// 16 lanes x 32 columns as fragments of 8x8 matrices
__device__ __forceinline__ void tmem_fragments(uint32_t addr, float (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
          "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
        : "r"(addr)
        : "memory");
}
// The wait takes part in the registers' dataflow, so that no use of them moves in front of it.
#define SGCN_R16(r)                                                                                                                              \
    "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), \
        "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15])
__device__ __forceinline__ void tmem_wait(float (&r)[16]) { asm volatile("tcgen05.wait::ld.sync.aligned;" : SGCN_R16(r)::"memory"); }
__device__ __forceinline__ void after_wait(float (&r)[16]) { asm volatile("" : SGCN_R16(r)::"memory"); }
#undef SGCN_R16

// Operand tiles, 128-byte swizzle.  k contiguous: rows of 64 k, 8-row groups 1 KB apart.  Rows (or columns) contiguous: blocks of
// 64 of them x 64 k, 8-k groups 1 KB apart, blocks 8 KB apart.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, bool k_contiguous) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)(k_contiguous ? 1 : 8192 >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}

// ------------------------------------------------------------------------------------------ pieces of the epilogue
//
// A warp works on units of 32 rows x 32 columns, in halves of 16 rows.  Its registers hold them as tensor memory's 16x256b form, the
// form of 8x8 matrix fragments, gives them: v[4 j + 2 q + e] is row 8 q + lane / 4, column 8 j + 2 (lane % 4) + e.  A lane then
// needs the biases of eight columns only and adds up columns mostly within itself (a row per lane took 64 broadcast reads of biases
// and 136 instructions per 32 columns' sums; the gated forward's epilogue fell from 552 instructions a unit to 419), and 8x8
// matrix loads and stores bring bf16 fragments to shared memory, from where they leave in whole lines.

// Two fp32 operations in one instruction, each rounded as the single one is: half the issue slots of the epilogue's sums and products.
__device__ __forceinline__ void add2(float& x, float& y, float a, float b) {
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tadd.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ void mul2(float& x, float& y, float a, float b) {
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tmul.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
// x, y = x a + c, y b + d
__device__ __forceinline__ void fma2(float& x, float& y, float a, float b, float c, float d) {
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tmov.b64 r, {%4, %5};\n\tfma.rn.f32x2 p, p, q, r;\n\tmov.b64 {%0, %1}, p;\n\t}"
        : "+f"(x), "+f"(y)
        : "f"(a), "f"(b), "f"(c), "f"(d));
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}
// A slab: 32 rows of 64 bytes, 16-byte chunks exchanged as tensor copies with the 64-byte swizzle do; neither matrices nor lines meet
// bank conflicts.
__device__ __forceinline__ uint32_t slab_at(int row, int chunk) { return (uint32_t)(row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4)); }
__device__ __forceinline__ void sts16(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Line i of eight rows: row 8 i + lane / 4, chunk lane % 4.
__device__ __forceinline__ uint32_t line_at(uint32_t slab, int lane, int i) { return slab + i * 512 + (lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 3) & 3)) << 4); }
// Where this lane points for the four 8x8 matrices of half h and columns 16 q .. 16 q + 15.
__device__ __forceinline__ uint32_t matrix_at(uint32_t slab, int lane, int h, int q) {
    return slab + h * 1024 + ((lane >> 3) & 1) * 512 + (lane & 7) * 64 + (((2 * q + (lane >> 4)) ^ ((lane >> 1) & 3)) << 4);
}
__device__ __forceinline__ void half_to_slab(const uint32_t (&w)[8], uint32_t slab, int lane, int h) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
        asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(matrix_at(slab, lane, h, q)), "r"(w[4 * q]), "r"(w[4 * q + 1]),
                     "r"(w[4 * q + 2]), "r"(w[4 * q + 3])
                     : "memory");
}
__device__ __forceinline__ void half_from_slab(float (&v)[16], uint32_t slab, int lane, int h) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        uint32_t w[4];
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                     : "r"(matrix_at(slab, lane, h, q))
                     : "memory");
#pragma unroll
        for (int k = 0; k < 4; ++k) v[8 * q + 2 * k] = __uint_as_float(w[k] << 16), v[8 * q + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
}
__device__ __forceinline__ void pack_half(const float (&v)[16], uint32_t (&w)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = pack2(v[2 * k], v[2 * k + 1]);
}

struct Where {
    int slice, row;        // first of the warp's 32 rows in D
    int rows;              // how many of them exist
};

// The slab to memory whose rows no tensor copy can reach, element by element.
__device__ __forceinline__ void slab_out(__nv_bfloat16* at, int ld, int rows, int cols, uint32_t slab, int lane) {
    if (lane < cols)
#pragma unroll 4
        for (int i = 0; i < rows; ++i) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(slab + slab_at(i, lane >> 3) + (lane & 7) * 2) : "memory");
            reinterpret_cast<uint16_t*>(at)[(int64_t)i * ld + lane] = v;
        }
    __syncwarp();
}
// 32 rows x 32 columns of r or dout in bf16: asked for here (whole chunks, where they are aligned) ...
__device__ __forceinline__ void load_in(const Params& P, const Where& w, int col, uint4 (&raw)[4], int lane) {
    const int left = P.cols - col - (lane & 3) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = make_uint4(0, 0, 0, 0);
    if (!P.in_vec || w.rows <= 0 || left < 8) return;
    const __nv_bfloat16* at = static_cast<const __nv_bfloat16*>(P.in) + ((int64_t)w.row * P.in_ld + (w.slice * P.cols + col + (lane & 3) * 8));
    if (w.rows == 32) {
        at += (int64_t)(lane >> 2) * P.in_ld;
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = *reinterpret_cast<const uint4*>(at + (int64_t)i * 8 * P.in_ld);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 8 + (lane >> 2);
        if (row < w.rows) raw[i] = *reinterpret_cast<const uint4*>(at + (int64_t)row * P.in_ld);
    }
}
// ... and laid into the slab here, with what no whole chunk holds.
__device__ __forceinline__ void put_in(const Params& P, const Where& w, int col, const uint4 (&raw)[4], uint32_t slab, int lane) {
    const int cols = min(32, P.cols - col), from = P.in_vec ? max(cols, 0) & ~7 : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sts16(line_at(slab, lane, i), raw[i]);
    if (from >= cols || w.rows <= 0) return;
    __syncwarp();
    if (lane >= from && lane < cols) {
        const uint16_t* at = static_cast<const uint16_t*>(P.in) + (int64_t)w.row * P.in_ld + (w.slice * P.cols + col + lane);
#pragma unroll 8
        for (int i = 0; i < w.rows; ++i) {
            const uint16_t v = at[(int64_t)i * P.in_ld];
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(slab + slab_at(i, lane >> 3) + (lane & 7) * 2), "h"(v) : "memory");
        }
    }
}
// Where the accumulator is emptied into registers, r or dout come into the slab by asynchronous copies that are asked for before the
// product is there (loads of fragments from memory took 4,800 cycles a half where the MMAs run 12,000 ahead): halves of 16 rows, 2 KB apart, rows of
// 64 bytes of bf16 or 128 of fp32, chunks exchanged as tensor copies with that swizzle do.  Zeros where nothing is there.
__device__ __forceinline__ void fetch_in(const Params& P, const Where& w, int col, uint32_t slab, int lane) {
    const int elem = P.in_bf16 ? 2 : 4, chunks_log = P.in_bf16 ? 2 : 3;
    const char* at = static_cast<const char*>(P.in) + ((int64_t)w.row * P.in_ld + (w.slice * P.cols + col)) * elem;
    const int64_t step = (int64_t)P.in_ld * elem;
    const int have = min(32, P.cols - col) * elem;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= 4 && P.in_bf16) break;
        const int id = i * 32 + lane, row = id >> chunks_log, c = id & ((1 << chunks_log) - 1), left = row < w.rows ? max(0, min(16, have - c * 16)) : 0;
        const uint32_t dst = slab + (row >> 4) * 2048 + ((row & 15) << (chunks_log + 4)) + ((c ^ (P.in_bf16 ? (row >> 1) & 3 : row & 7)) << 4);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(left ? at + row * step + c * 16 : static_cast<const char*>(P.in)), "r"(left) : "memory");
    }
}
__device__ __forceinline__ void fetched() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Element pair k of a lane's half of fp32.
__device__ __forceinline__ uint32_t pair_at(uint32_t slab, int lane, int h, int k) {
    return slab + h * 2048 + (8 * (k & 1) + (lane >> 2)) * 128 + (((2 * (k >> 1) + ((lane >> 1) & 1)) ^ (lane >> 2)) << 4) + (lane & 1) * 8;
}
__device__ __forceinline__ void half_of_in(const Params& P, uint32_t slab, int lane, int h, float (&v)[16]) {
    if (P.in_bf16) return half_from_slab(v, slab + h * 1024, lane, h);
#pragma unroll
    for (int k = 0; k < 8; ++k)
        asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v[2 * k]), "=f"(v[2 * k + 1]) : "r"(pair_at(slab, lane, h, k)) : "memory");
}
// The same from and to memory whose rows no such copy can reach; fp32 in pairs, where they are aligned.
__device__ __forceinline__ void load_half(const Params& P, const Where& w, int col, int h, float (&v)[16], int lane) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int c = col + 8 * (k >> 1) + 2 * (lane & 3), row = 16 * h + 8 * (k & 1) + (lane >> 2);
        const int64_t at = (int64_t)(w.row + row) * P.in_ld + (w.slice * P.cols + c);
        v[2 * k] = v[2 * k + 1] = 0.f;
        if (row >= w.rows) continue;
        if (P.in_bf16) {
            if (c < P.cols) v[2 * k] = __bfloat162float(static_cast<const __nv_bfloat16*>(P.in)[at]);
            if (c + 1 < P.cols) v[2 * k + 1] = __bfloat162float(static_cast<const __nv_bfloat16*>(P.in)[at + 1]);
        } else if (P.in_pairs && c + 1 < P.cols) {
            const float2 t = *reinterpret_cast<const float2*>(static_cast<const float*>(P.in) + at);
            v[2 * k] = t.x, v[2 * k + 1] = t.y;
        } else {
            if (c < P.cols) v[2 * k] = static_cast<const float*>(P.in)[at];
            if (c + 1 < P.cols) v[2 * k + 1] = static_cast<const float*>(P.in)[at + 1];
        }
    }
}
__device__ __forceinline__ void store_half(const Params& P, const Where& w, int col, int h, const float (&v)[16], int lane) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int c = col + 8 * (k >> 1) + 2 * (lane & 3), row = 16 * h + 8 * (k & 1) + (lane >> 2);
        float* p = static_cast<float*>(P.out) + (int64_t)(w.row + row) * P.out_ld + (w.slice * P.cols + c);
        if (row >= w.rows) continue;
        if (P.out_pairs && c + 1 < P.cols) {
            *reinterpret_cast<float2*>(p) = make_float2(v[2 * k], v[2 * k + 1]);
        } else {
            if (c < P.cols) p[0] = v[2 * k];
            if (c + 1 < P.cols) p[1] = v[2 * k + 1];
        }
    }
}
// The biases of this lane's eight columns of a unit.
__device__ __forceinline__ void load_bias(const Params& P, const float* b, int slice, int col, float (&v)[8], int lane) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    if (!b) return;
    const int c0 = col + 2 * (lane & 3);
    const float* at = b + (slice * P.cols + c0);
    if (P.bias_vec && col + 32 <= P.cols) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 t = __ldg(reinterpret_cast<const float2*>(at) + 4 * j);
            v[2 * j] = t.x, v[2 * j + 1] = t.y;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c0 + 8 * (j >> 1) + (j & 1) < P.cols) v[j] = __ldg(at + 8 * (j >> 1) + (j & 1));
}
__device__ __forceinline__ void add_bias(float (&v)[16], const float (&b)[8]) {
#pragma unroll
    for (int k = 0; k < 16; k += 2) add2(v[k], v[k + 1], b[(k >> 2) * 2], b[(k >> 2) * 2 + 1]);
}
// Column sums of a unit: each lane's over its rows, then over the eight lanes that hold the same columns, each of which ends with one.
__device__ __forceinline__ void sum_half(const float (&v)[16], float (&s)[8]) {
#pragma unroll
    for (int k = 0; k < 16; k += 2) add2(s[(k >> 2) * 2], s[(k >> 2) * 2 + 1], v[k], v[k + 1]);
}
__device__ __forceinline__ float sum_lanes(float (&s)[8], int lane) {   // of column 8 (k >> 1) + 2 (lane % 4) + (k & 1), k = sum_column(lane)
#pragma unroll
    for (int half = 4, mask = 16; half >= 1; half >>= 1, mask >>= 1) {
        const bool upper = lane & mask;
#pragma unroll
        for (int j = 0; j < half; ++j) {
            const float keep = upper ? s[j + half] : s[j], give = upper ? s[j] : s[j + half];
            s[j] = keep + __shfl_xor_sync(0xffffffffu, give, mask);
        }
    }
    return s[0];
}
__device__ __forceinline__ int sum_column(int lane) {
    const int k = lane >> 2;
    return 8 * (k >> 1) + 2 * (lane & 3) + (k & 1);
}

// SILU and GELU multiply a by a gate 1 / (1 + exp(-w)): w = a, or 2 u with (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)).
constexpr float kLog2e = 1.4426950408889634f, kGeluA = 0.7978845608028654f, kGeluB = 0.044715f;
template <int ACT>
__device__ __forceinline__ float gate_of(float a) {   // by the exponential of -|w|, which passes no range's end: 1 / (1 + t) or t / (1 + t)
    const float w = ACT == SLICEGCN_ACT_SILU ? a : 2.f * kGeluA * a * fmaf(kGeluB, a * a, 1.f);
    const float t = expf(-fabsf(w)), r = __fdividef(1.f, 1.f + t);   // 2 units of the last place each
    return w < 0.f ? t * r : r;
}
// Where results are rounded to bf16 the hardware's exponential and reciprocal (2^-22 each, and 2^-24 |w| of the argument) are exact
// enough (one reciprocal for two numbers, 1/x = y/(xy), gained nothing); a gate below 2^-126 is 0.  These two operations keep the
// special-function unit busy for 63 % of the gated forward kernels' time.  Two numbers at a time; s = a^2.
template <int ACT>
__device__ __forceinline__ void gates_of(float a0, float a1, float s0, float s1, float& q0, float& q1) {
    if (ACT == SLICEGCN_ACT_SILU) {
        q0 = a0, q1 = a1;
        mul2(q0, q1, -kLog2e, -kLog2e);
    } else {
        constexpr float c0 = -2.f * kLog2e * kGeluA, c1 = c0 * kGeluB;
        q0 = s0, q1 = s1;
        fma2(q0, q1, c1, c1, c0, c0);
        mul2(q0, q1, a0, a1);
    }
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(q0));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(q1));
    add2(q0, q1, 1.f, 1.f);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(q0));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(q1));
}
__device__ __forceinline__ float relu(float a) { return a > 0.f || isnan(a) ? a : 0.f; }
__device__ __forceinline__ float relu_slope(float a) { return a > 0.f ? 1.f : isnan(a) ? a : 0.f; }   // a NaN stays one
// a -> act(a) [* c]
template <int ACT, bool GATED, bool ACCURATE, int N>
__device__ __forceinline__ void forward_as(float (&a)[N], const float (&c)[N]) {
    constexpr bool kSmooth = ACT == SLICEGCN_ACT_SILU || ACT == SLICEGCN_ACT_GELU;
    if constexpr (ACCURATE) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (kSmooth) a[k] *= gate_of<ACT>(a[k]);
            if (ACT == SLICEGCN_ACT_RELU) a[k] = relu(a[k]);
            if (GATED) a[k] *= c[k];
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            if (kSmooth) {
                float s0 = a[k], s1 = a[k + 1], q0, q1;
                if (ACT == SLICEGCN_ACT_GELU) mul2(s0, s1, a[k], a[k + 1]);
                gates_of<ACT>(a[k], a[k + 1], s0, s1, q0, q1);
                mul2(a[k], a[k + 1], q0, q1);
            }
            if (ACT == SLICEGCN_ACT_RELU) a[k] = relu(a[k]), a[k + 1] = relu(a[k + 1]);
            if (GATED) mul2(a[k], a[k + 1], c[k], c[k + 1]);
        }
    }
}
// a, c -> da, dc:  SILU' = q + y (1 - q),  GELU' = q + y (1 - q) 2 A (1 + 3 B a^2)  with the gate q and y = a q.  Far from zero
// y (1 - q) is 0, and a^2 is kept from infinity, since 0 times that is none.
constexpr float kGeluFar = 1e30f;
template <int ACT, bool GATED, bool ACCURATE, int N>
__device__ __forceinline__ void backward_as(float scale, const float (&g)[N], float (&a)[N], float (&c)[N]) {
    constexpr bool kSmooth = ACT == SLICEGCN_ACT_SILU || ACT == SLICEGCN_ACT_GELU;
    if constexpr (ACCURATE) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float y = a[k], dy = 1.f;
            if (kSmooth) {
                const float q = gate_of<ACT>(a[k]);
                y *= q;
                dy = fmaf(y * (1.f - q), ACT == SLICEGCN_ACT_GELU ? 2.f * kGeluA * fmaf(3.f * kGeluB, fminf(a[k] * a[k], kGeluFar), 1.f) : 1.f, q);
            }
            if (ACT == SLICEGCN_ACT_RELU) y = relu(a[k]), dy = relu_slope(a[k]);
            const float gk = g[k] * scale;
            a[k] = GATED ? gk * c[k] * dy : gk * dy;
            if (GATED) c[k] = gk * y;
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            float y0 = a[k], y1 = a[k + 1], d0 = 1.f, d1 = 1.f, g0 = g[k], g1 = g[k + 1];
            mul2(g0, g1, scale, scale);
            if (kSmooth) {
                float s0 = a[k], s1 = a[k + 1], q0, q1;
                if (ACT == SLICEGCN_ACT_GELU) mul2(s0, s1, a[k], a[k + 1]);
                gates_of<ACT>(a[k], a[k + 1], s0, s1, q0, q1);
                mul2(y0, y1, q0, q1);
                d0 = q0, d1 = q1;
                fma2(d0, d1, -1.f, -1.f, 1.f, 1.f);
                if (ACT == SLICEGCN_ACT_GELU) {
                    s0 = fminf(s0, kGeluFar), s1 = fminf(s1, kGeluFar);
                    fma2(s0, s1, 6.f * kGeluA * kGeluB, 6.f * kGeluA * kGeluB, 2.f * kGeluA, 2.f * kGeluA);
                    mul2(d0, d1, s0, s1);
                }
                fma2(d0, d1, y0, y1, q0, q1);
            }
            if (ACT == SLICEGCN_ACT_RELU) {
                y0 = relu(a[k]), y1 = relu(a[k + 1]);
                d0 = relu_slope(a[k]), d1 = relu_slope(a[k + 1]);
            }
            a[k] = g0, a[k + 1] = g1;
            if (GATED) mul2(a[k], a[k + 1], c[k], c[k + 1]);
            if (ACT != SLICEGCN_ACT_NONE) mul2(a[k], a[k + 1], d0, d1);
            if (GATED) {
                c[k] = y0, c[k + 1] = y1;
                mul2(c[k], c[k + 1], g0, g1);
            }
        }
    }
}

// Parts of an fp32 number: 8 bits each, cut, not rounded, so that none leaves the range at its upper end.  From 2^-110 up their sum is
// the number; below that the third part's last bits fall under bf16's least number, 2^-133, and are left out.  (A power of two in front
// of tiny operands would need their largest magnitude first, a pass over them.)  Takes the next part off x (off an infinity or a NaN:
// NaN is left).
__device__ __forceinline__ uint32_t next_part(float& x) {
    const uint32_t part = __float_as_uint(x) & 0xffff0000u;
    x -= __uint_as_float(part);
    return part;
}
// Half h of da or dc as three planes, or rounded as one, by way of two slots in turn in the half's place.
__device__ __forceinline__ void planes_out(const Params& P, const Where& w, int part, int col, int h, float (&v)[16], uint32_t slab, int& slots, int lane) {
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        if (q >= P.planes) break;
        uint32_t words[8];
        if (P.planes == 1) {
            pack_half(v, words);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t lo = __float_as_uint(v[2 * k]), hi = __float_as_uint(v[2 * k + 1]);
                words[k] = __byte_perm(lo, hi, 0x7632);
                if (q < 2) add2(v[2 * k], v[2 * k + 1], __uint_as_float((lo & 0xffff0000u) ^ 0x80000000u), __uint_as_float((hi & 0xffff0000u) ^ 0x80000000u));
            }
        }
        if (lane == 0) stores_read<1>();
        __syncwarp();
        const uint32_t at = slab + h * 2048 + (slots & 1) * 1024;
        ++slots;
        half_to_slab(words, at, lane, 0);
        proxy_fence();
        __syncwarp();
        if (lane == 0) {
            if (w.rows > 16 * h) tma_store(&P.o, at, col, w.row + 16 * h, part * P.p + w.slice, q);
            stores_commit();
        }
    }
}
__device__ __forceinline__ void sums_out(const Params& P, int row, int matrix, int col, float (&s)[8], int lane) {
    const float t = sum_lanes(s, lane);
    const int c = col + sum_column(lane);
    if (c < P.cols) P.sums[((int64_t)row * P.slices + matrix) * P.cols + c] = t;
}

// ------------------------------------------------------------------------------------------ the product

struct Item {
    int slice, m, n, split;   // slice (times part), first row and column of the tile, piece of k
};
template <int MODE>
__device__ __forceinline__ Item item_of(const Params& P, int i) {
    Item t;
    const int cols = 2 * P.nt;
    const int per_tile = MODE == kFwdGated || MODE == kDzGated || (MODE == kDw && P.pair) ? P.nt : cols;   // columns of D that a tile makes
    t.split = P.splits > 1 ? P.by_split(i) : 0;
    i -= t.split * P.by_split.d;
    if (MODE == kDw) {
        const int above = P.by_n(i);
        t.n = (i - above * P.tiles_n) * per_tile;
        t.slice = P.by_m(above);
        t.m = (above - t.slice * P.tiles_m) * 256;
    } else {   // `group` row tiles side by side, then the next column tile: operands come from L2 in between
        const int g = P.by_group(i), rest = i - g * P.by_group.d, size = min(P.group, P.tiles_m - g * P.group);
        const int c = size == P.group ? P.by_m(rest) : P.by_last(rest);
        t.m = (g * P.group + rest - c * size) * 256;
        t.slice = P.by_n(c);
        t.n = (c - t.slice * P.tiles_n) * per_tile;
    }
    return t;
}

// PROMO: the accumulator is emptied into registers every P.chunk steps (fp32 digits, or long sums).
template <int MODE, bool PROMO, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) ffn_kernel(const __grid_constant__ Params P) {
    constexpr bool kGated = MODE == kFwdGated || MODE == kDzGated;
    constexpr bool kIsDz = MODE == kDz || MODE == kDzGated;
    constexpr bool kAK = MODE != kDw;    // A's k is contiguous
    constexpr bool kBK = MODE == kDx;    // B's
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* tail = smem_raw + (base - smem_u32(smem_raw)) + kStages * kStageBytes + kEpiWarps * kSlabBytes;
    uint64_t* full = reinterpret_cast<uint64_t*>(tail);
    uint64_t* empty = full + kStages;
    uint64_t* tfull = empty + kStages;    // [2 groups]
    uint64_t* tempty = tfull + 4;         // [2 groups]
    uint32_t* tmem_at = reinterpret_cast<uint32_t*>(tempty + 4);
    // Tiles of half width: two groups of eight epilogue warps take turns at the tiles, each with two accumulators of its own (a
    // group waits for its own ones in order, whatever the other does).  Else all sixteen warps work on each tile.
    const int groups_log = P.nt == 64, groups = 1 << groups_log;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int first = blockIdx.x >> 1, stride = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) mbar_init(full + s, 1), mbar_init(empty + s, 1);
        for (int s = 0; s < 2 * groups; ++s) mbar_init(tfull + s, 1), mbar_init(tempty + s, 2 * kEpiWarps >> groups_log);   // of both CTAs
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
    // Two operands in parts of fp32 come in three stages for 64 k -- parts 2 of both, then 0, then 1 -- and each is multiplied with all
    // of the others that it is needed with: six products from six tiles, where a pair of tiles for each is twice the traffic
    // from L2 (gradients of 232,965 x 600 -> 2 x 128: 1,620 -> 1,510 us).  Small products come first, since every addition cuts digits
    // off the sum: the product of parts 0, which makes it large, is put off until the next 64 k's parts 2 are done; by then its
    // stage's place in the ring is not needed yet.  One operand in parts: three products one after another over a chunk of k (in
    // this way of three stages 480 instead of 340 us for dx of 169,343 x 256 -> 2 x 1,024, since two of three stages then are half empty).
    const bool six = P.a_planes == 3 && P.b_planes == 3;
    const int products = six ? 1 : max(P.a_planes, P.b_planes);
    // The two issuing warps walk their loops as whole warps, and one lane issues: what copies and MMAs are given then stays in
    // uniform registers.  (One lane in a loop of its own: 880 cycles per 64-wide step where the MMAs take 512.)
    if (warp == kEpiWarps) {
        const bool one = elect_one();
        bool ok = true;
        int fill = 0, st = 0;
        uint32_t phase = 1;
        const uint32_t bytes = 2u * (16384u + (uint32_t)P.nt * 128u);
        for (int i = first; ok && i < P.items; i += stride) {
            const Item t = item_of<MODE>(P, i);
            const int row0 = t.m + (int)rank * 128;
            const bool upper = !kGated && t.slice >= P.p;            // the second projection's
            const int slice = upper ? t.slice - P.p : t.slice;
            const int aslice = MODE == kDw && !P.swapped ? t.slice : slice;
            const int bslice = MODE == kDw && P.swapped ? t.slice + (P.pair ? (int)rank * P.p : 0) : slice;
            const CUtensorMap* bmap = (kGated && rank) || (MODE == kFwd && upper) ? &P.b1 : &P.b0;
            const int bcol = kGated || (MODE == kDw && P.pair) ? t.n : t.n + (int)rank * P.nt;
            const int first_kb = t.split * P.kb_total;
            const auto fetch = [&](int kb, int plane) {   // of the operands that have it, else plane 0
                ok = __all_sync(0xffffffffu, mbar_wait(empty + st, phase));
                if (!ok) return;
                const uint32_t a = base + st * kStageBytes, b = a + 16384u;
                const bool second = MODE == kDx && first_kb + kb >= P.kb_part;
                const int k = (first_kb + kb - (second ? P.kb_part : 0)) * 64;   // past the end there are only zeros
                const int a_plane = min(plane, P.a_planes - 1), b_plane = min(plane, P.b_planes - 1);
                if (one) {
                    if (rank == 0) mbar_expect(full + st, bytes);
                    if (kAK) {
                        tma_load(a, &P.a, k, row0, second ? P.p + slice : slice, a_plane, full + st);
                    } else {
                        tma_load(a, &P.a, row0, k, aslice, a_plane, full + st);
                        tma_load(a + 8192, &P.a, row0 + 64, k, aslice, a_plane, full + st);
                    }
                    if (kBK) {
                        tma_load(b, second ? &P.b1 : &P.b0, k, bcol, slice, b_plane, full + st);
                    } else {
                        tma_load(b, bmap, bcol, k, bslice, b_plane, full + st);
                        if (P.nt > 64) tma_load(b + 8192, bmap, bcol + 64, k, bslice, b_plane, full + st);
                    }
                }
                __syncwarp();
                ++fill;
                if (++st == kStages) st = 0, phase ^= 1;
            };
            for (int c = 0; ok && c < chunks; ++c) {
                const int kb0 = c * P.chunk, kb1 = min(kb0 + P.chunk, P.kb_total);
                for (int q = products - 1; ok && q >= 0; --q)
                    for (int kb = kb0; ok && kb < kb1; ++kb) {
                        if (six) {
                            fetch(kb, 2);
                            if (ok) fetch(kb, 0);
                            if (ok) fetch(kb, 1);
                        } else {
                            fetch(kb, q);
                        }
                    }
            }
        }
        // the pair's last arrivals at this CTA's barriers, before its memory is given up
        for (int s = max(0, fill - kStages); ok && s < fill; ++s) ok = mbar_wait(empty + s % kStages, (s / kStages) & 1);
        if (!ok && P.status) atomicOr(P.status, SLICEGCN_DEVSTATUS_WAIT);
    } else if (warp == kEpiWarps + 1) {
        if (rank == 0) {
            const bool one = elect_one();
            bool ok = true;
            int turn = 0, st = 0;
            uint32_t phase = 0;
            const uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | (kAK ? 0u : 1u << 15) | (kBK ? 0u : 1u << 16) | (uint32_t)(2 * P.nt >> 3) << 17 | 16u << 24;
            for (int i = first; ok && i < P.items; i += stride, ++turn) {
                int use = (turn >> groups_log) * chunks;
                const int first_kb = P.splits > 1 ? P.by_split(i) * P.kb_total : 0;
                for (int c = 0; ok && c < chunks; ++c, ++use) {
                    const int kb0 = c * P.chunk, kb1 = min(kb0 + P.chunk, P.kb_total);
                    const int acc = (turn & (groups - 1)) * 2 + (use & 1);
                    const uint32_t d = tmem + acc * (2 * P.nt);
                    ok = __all_sync(0xffffffffu, mbar_wait(tempty + acc, ((use >> 1) & 1) ^ 1));
                    if (!ok) break;
                    fence_after();
                    bool more = false;
                    const auto arrived = [&](int& s) {   // the next stage of the ring
                        s = st;
                        ok = ok && __all_sync(0xffffffffu, mbar_wait(full + st, phase));
                        fence_after();
                        if (++st == kStages) st = 0, phase ^= 1;
                        return ok;
                    };
                    const auto multiply = [&](int kb, int sa, int sb) {
                        const uint64_t ad = tile_desc(base + sa * kStageBytes, kAK), bd = tile_desc(base + sb * kStageBytes + 16384u, kBK);
                        const int at_kb = first_kb + kb;
                        const int left = MODE == kDw ? 64 : P.k_part - (at_kb >= P.kb_part ? at_kb - P.kb_part : at_kb) * 64;   // past the end there are only zeros
                        if (one) {
#pragma unroll
                            for (int s = 0; s < 4; ++s)
                                if (s == 0 || s * 16 < left) umma(d, ad + (uint64_t)(s * (kAK ? 2 : 128)), bd + (uint64_t)(s * (kBK ? 2 : 128)), idesc, s > 0 || more);
                        }
                        more = true;
                    };
                    const auto done_with = [&](int s) {
                        if (one) umma_commit(empty + s);
                        __syncwarp();
                    };
                    int x, y, z, held = -1;
                    for (int q = 0; ok && q < products; ++q)
                        for (int kb = kb0; kb < kb1; ++kb) {
                            if (!six) {
                                if (!arrived(z)) break;
                                multiply(kb, z, z);
                                done_with(z);
                                continue;
                            }
                            if (!arrived(x) || !arrived(z)) break;
                            multiply(kb, x, z);
                            multiply(kb, z, x);
                            done_with(x);
                            if (held >= 0) {
                                multiply(kb - 1, held, held);
                                done_with(held);
                            }
                            if (!arrived(y)) break;
                            multiply(kb, y, y);
                            multiply(kb, y, z);
                            multiply(kb, z, y);
                            done_with(y);
                            held = z;
                        }
                    if (ok && held >= 0) {
                        multiply(kb1 - 1, held, held);
                        done_with(held);
                    }
                    if (one) umma_commit(tfull + acc);
                    __syncwarp();
                }
            }
            if (!ok) {   // the copies on their way, before this memory is given up
                for (int s = 0; s < kStages; ++s) {
                    mbar_wait(full + st, phase);
                    if (++st == kStages) st = 0, phase ^= 1;
                }
                if (P.status) atomicOr(P.status, SLICEGCN_DEVSTATUS_WAIT);
            }
        }
    } else {
        const uint32_t slab = base + kStages * kStageBytes + warp * kSlabBytes, slab2 = slab + 2048;
        // a warp has 32 rows and 64 columns of the accumulator, gated: 32 of a and the same 32 of c
        const int group = (warp >> 2) & (groups - 1), part = (warp >> 2) >> groups_log;
        const int quarter = warp & 3, share = kGated ? 32 : 64;
        const uint32_t mine = tmem + ((uint32_t)(quarter * 32) << 16) + part * share;
        const int second = kGated ? P.nt : 32;   // columns from the first 32 to the other 32
        bool ok = true;
        int turn = 0, halves = 0;
        float bias[8], bias2[8], s[8], s2[8];   // s, s2: column sums of da and dc; not gated: of da's two units
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = s2[j] = 0.f;
        Item ahead;   // of turn / 32 * 32 + lane: 32 tiles are worked out at once, each lane one, and passed around when their turn comes
        for (int i = first; ok && i < P.items; i += stride, ++turn) {
            if ((turn & 31) == 0) ahead = item_of<MODE>(P, min(i + lane * stride, P.items - 1));
            if ((turn & (groups - 1)) != group) continue;
            Item t;
            t.m = __shfl_sync(0xffffffffu, ahead.m, turn & 31);
            t.n = __shfl_sync(0xffffffffu, ahead.n, turn & 31);
            t.slice = __shfl_sync(0xffffffffu, ahead.slice, turn & 31);
            t.split = PROMO ? __shfl_sync(0xffffffffu, ahead.split, turn & 31) : 0;
            Where w;
            w.slice = t.slice;
            w.row = t.m + (int)rank * 128 + quarter * 32;
            w.rows = min(32, max(0, P.n - w.row));
            const int col0 = t.n + part * share;
            int use = (turn >> groups_log) * chunks;
            if constexpr (MODE == kDw) {
                float acc[64];
#pragma unroll
                for (int j = 0; j < 64; ++j) acc[j] = 0.f;
                for (int c = 0; c < chunks; ++c, ++use) {
                    ok = __all_sync(0xffffffffu, mbar_wait(tfull + group * 2 + (use & 1), (use >> 1) & 1));
                    if (!ok) break;
                    fence_after();
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        float r[16];
                        tmem_rows(mine + (group * 2 + (use & 1)) * (2 * P.nt) + u * 16, r);
                        tmem_wait(r);
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[u * 16 + j] += r[j];
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_first(tempty + group * 2 + (use & 1));
                }
                if (!ok) break;
                // this lane's row of the tile, dW's column (swapped: its row); the tile's columns are dW's rows (columns)
                const int m = w.row + lane, fs = P.cols, ks = P.k_part;
                const int m_end = P.swapped ? ks : fs, n_end = P.swapped ? fs : ks;
                const int64_t m_step = P.swapped ? fs : 1, n_step = P.swapped ? 1 : fs, matrix = (int64_t)ks * fs;
                const bool upper = P.pair ? part * share >= P.nt : t.slice >= P.p;   // dW2's
                const int slice = P.pair || !upper ? t.slice : t.slice - P.p, n0 = P.pair && upper ? col0 - P.nt : col0;
                if (m < m_end) {
                    const int64_t from = m * m_step + n0 * n_step;
                    if (P.partial) {
                        float* to = P.partial + ((int64_t)t.split * P.matrices + (upper ? P.p : 0) + slice) * matrix + from;
#pragma unroll
                        for (int j = 0; j < 64; ++j)
                            if (n0 + j < n_end) to[j * n_step] = acc[j];
                    } else if (void* dw = upper ? P.dw2 : P.dw) {
                        const int64_t at = slice * matrix + from;
#pragma unroll
                        for (int j = 0; j < 64; ++j)
                            if (n0 + j < n_end) {
                                if (P.out_bf16)
                                    static_cast<__nv_bfloat16*>(dw)[at + j * n_step] = __float2bfloat16_rn(acc[j] * P.scale);
                                else
                                    static_cast<float*>(dw)[at + j * n_step] = acc[j] * P.scale;
                            }
                    }
                }
            } else if constexpr (PROMO) {
                float acc[64];   // half h of the first 32 columns at 16 h, of the other 32 at 32 + 16 h
#pragma unroll
                for (int j = 0; j < 64; ++j) acc[j] = 0.f;
                const bool with_in = P.splits == 1 && (kIsDz || (MODE != kDx && P.in)), staged = with_in && P.in_vec;
                if (staged) {
                    if (lane == 0) stores_read<0>();
                    __syncwarp();
                    fetch_in(P, w, col0, slab, lane);
                }
                // a column's bias each, passed around later: loads in the epilogue took 4,000 cycles
                float lower_bias = 0.f, upper_bias = 0.f;
                if (MODE != kDx) {
                    if (P.b && col0 + lane < P.cols) lower_bias = __ldg(P.b + (w.slice * P.cols + col0 + lane));
                    const float* b = kGated ? P.b2 : P.b;
                    const int c = kGated ? col0 + lane : col0 + 32 + lane;
                    if (b && c < P.cols) upper_bias = __ldg(b + (w.slice * P.cols + c));
                }
                for (int c = 0; c < chunks; ++c, ++use) {
                    ok = __all_sync(0xffffffffu, mbar_wait(tfull + group * 2 + (use & 1), (use >> 1) & 1));
                    if (!ok) break;
                    fence_after();
                    const uint32_t d = mine + (group * 2 + (use & 1)) * (2 * P.nt);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        float r[16];
                        tmem_fragments(d + (u & 2 ? second : 0) + ((uint32_t)((u & 1) * 16) << 16), r);
                        tmem_wait(r);
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[u * 16 + j] += r[j];
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_first(tempty + group * 2 + (use & 1));
                }
                if (staged) fetched();
                __syncwarp();
                if (!ok) break;
#pragma unroll
                for (int u = 0; u < (kGated ? 1 : 2); ++u) {
                    const int col = col0 + u * 32;
                    if (col >= P.cols || w.rows <= 0) continue;
                    if ((MODE == kFwd || MODE == kDx) && P.splits > 1) {   // a piece's product, as it is
                        float* at = P.partial + ((int64_t)t.split * P.slices + w.slice) * P.n * P.cols;
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            const int row = w.row + 8 * ((k >> 1) & 1) + 16 * (k >> 4) + (lane >> 2), c = col + 8 * ((k >> 2) & 3) + 2 * (lane & 3) + (k & 1);
                            if (row < P.n && c < P.cols) at[(int64_t)row * P.cols + c] = acc[u * 32 + k];
                        }
                        continue;
                    }
                    if (u && staged) {
                        if (lane == 0) stores_read<0>();
                        __syncwarp();
                        fetch_in(P, w, col, slab, lane);
                        fetched();
                        __syncwarp();
                    }
                    float bias[8], bias2[8], s[8], s2[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int from = 8 * (j >> 1) + 2 * (lane & 3) + (j & 1);
                        if (MODE != kDx) bias[j] = __shfl_sync(0xffffffffu, u ? upper_bias : lower_bias, from);
                        if (kGated) bias2[j] = __shfl_sync(0xffffffffu, upper_bias, from);
                        s[j] = s2[j] = 0.f;
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float a[16], c[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) a[j] = acc[u * 32 + h * 16 + j], c[j] = kGated ? acc[(32 + h * 16 + j) & 63] : 0.f;
                        if (MODE != kDx) add_bias(a, bias);
                        if (kGated) add_bias(c, bias2);
                        float in[16];
                        if (staged) {
                            half_of_in(P, slab, lane, h, in);
                            __syncwarp();   // its place is used from here on
                        } else if (with_in) {
                            load_half(P, w, col, h, in, lane);
                        }
                        if constexpr (kIsDz) {
                            if (P.planes == 1)
                                backward_as<ACT, kGated, false>(P.scale, in, a, c);
                            else
                                backward_as<ACT, kGated, true>(P.scale, in, a, c);
                            sum_half(a, s);
                            if (kGated) sum_half(c, s2);
                            planes_out(P, w, 0, col, h, a, slab, halves, lane);
                            if (kGated) planes_out(P, w, 1, col, h, c, slab, halves, lane);
                        } else {
                            if (MODE != kDx) forward_as<ACT, kGated, true>(a, c);
#pragma unroll
                            for (int j = 0; j < 16; ++j) a[j] = with_in ? fmaf(a[j], P.scale, in[j]) : a[j] * P.scale;
                            if (P.out_vec && col < P.out_edge) {
                                if (lane == 0) stores_read<1>();   // of the same half before
                                __syncwarp();
#pragma unroll
                                for (int k = 0; k < 8; ++k)
                                    asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(pair_at(slab, lane, h, k)), "f"(a[2 * k]), "f"(a[2 * k + 1]) : "memory");
                                proxy_fence();
                                __syncwarp();
                                if (lane == 0) {
                                    if (w.rows > 16 * h) tma_store(&P.o, slab + h * 2048, col, w.row + 16 * h, w.slice, 0);
                                    stores_commit();
                                }
                            } else {
                                store_half(P, w, col, h, a, lane);
                            }
                        }
                    }
                    if (kIsDz && P.sums) {
                        sums_out(P, w.row >> 5, w.slice, col, s, lane);
                        if (kGated) sums_out(P, w.row >> 5, P.p + w.slice, col, s2, lane);
                    }
                }
            } else {
                // what a unit needs besides the product is on its way while the product is waited for
                const bool with_in = kIsDz || (MODE != kDx && P.in);
                uint4 raw[4];
                if (!kGated || !P.fixed || turn == group) {
                    load_bias(P, MODE == kDx ? nullptr : P.b, w.slice, col0, bias, lane);
                    if (kGated) load_bias(P, P.b2, w.slice, col0, bias2, lane);
                }
                if (with_in) load_in(P, w, col0, raw, lane);
                ok = __all_sync(0xffffffffu, mbar_wait(tfull + group * 2 + (use & 1), (use >> 1) & 1));
                if (!ok) break;
                fence_after();
                const uint32_t d = mine + (group * 2 + (use & 1)) * (2 * P.nt);
                if (kIsDz && !P.fixed) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[j] = s2[j] = 0.f;
                }
#pragma unroll(kIsDz ? 2 : 1)
                for (int u = 0; u < (kGated ? 1 : 2); ++u) {
                    const int col = col0 + u * 32;
                    const bool last = kGated || u == 1;
                    float a[16], c[16];
                    // da and dc need both slabs, else the two take turns, so that one leaves while the other is filled
                    const uint32_t to = kIsDz && kGated ? slab : slab + (halves++ & 1) * 2048;
                    tmem_fragments(d + u * 32, a);
                    if (kGated) tmem_fragments(d + second, c);
                    if (lane == 0) stores_read<kIsDz && kGated ? 0 : 1>();
                    __syncwarp();
                    if (with_in) {
                        put_in(P, w, col, raw, to, lane);
                        __syncwarp();
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (h) {
                            tmem_fragments(d + u * 32 + (16u << 16), a);
                            if (kGated) tmem_fragments(d + second + (16u << 16), c);
                        }
                        tmem_wait(a);
                        if (kGated) after_wait(c);
                        if (h && last) {
                            fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive_first(tempty + group * 2 + (use & 1));
                        }
                        if (MODE != kDx) add_bias(a, bias);
                        if (kGated) add_bias(c, bias2);
                        float in[16];
                        if (with_in) half_from_slab(in, to, lane, h);
                        uint32_t words[8];
                        if constexpr (kIsDz) {
                            backward_as<ACT, kGated, false>(P.scale, in, a, c);
                            if (P.sums) {
                                if (u == 0)
                                    sum_half(a, s);
                                else
                                    sum_half(a, s2);
                                if (kGated) sum_half(c, s2);
                            }
                            if (kGated) {
                                pack_half(c, words);
                                half_to_slab(words, slab2, lane, h);
                            }
                        } else {
                            if (MODE != kDx) forward_as<ACT, kGated, false>(a, c);
                            if (with_in) {
#pragma unroll
                                for (int j = 0; j < 16; j += 2) fma2(a[j], a[j + 1], P.scale, P.scale, in[j], in[j + 1]);
                            } else if (P.scale != 1.f) {
#pragma unroll
                                for (int j = 0; j < 16; j += 2) mul2(a[j], a[j + 1], P.scale, P.scale);
                            }
                        }
                        pack_half(a, words);
                        half_to_slab(words, to, lane, h);   // in the place of what came in
                    }
                    proxy_fence();
                    __syncwarp();
                    const bool there = col < P.cols && w.rows > 0;
                    if (kIsDz || (P.out_vec && col < P.out_edge)) {
                        if (lane == 0) {
                            if (there) {
                                tma_store(&P.o, to, col, w.row, w.slice, 0);
                                if (kIsDz && kGated) tma_store(&P.o, slab2, col, w.row, P.p + w.slice, 0);
                            }
                            stores_commit();
                        }
                    } else {
                        if (lane == 0) stores_commit();
                        if (there) slab_out(static_cast<__nv_bfloat16*>(P.out) + (int64_t)w.row * P.out_ld + (w.slice * P.cols + col), P.out_ld, w.rows, P.cols - col, to, lane);
                    }
                    if (kIsDz && P.sums && !P.fixed && there) {
                        sums_out(P, w.row >> 5, w.slice, col, u == 0 ? s : s2, lane);
                        if (kGated) sums_out(P, w.row >> 5, P.p + w.slice, col, s2, lane);
                    }
                    if (!last) {
                        load_bias(P, MODE == kDx ? nullptr : P.b, w.slice, col + 32, bias, lane);
                        if (with_in) load_in(P, w, col + 32, raw, lane);
                    }
                }
            }
        }
        if constexpr (kIsDz && !PROMO) {
            if (ok && P.sums && P.fixed) {   // the first item's columns are all items' columns; a warp without an item adds zeros
                const Item t = item_of<MODE>(P, first);
                const int per = P.slices / (kGated ? 2 : 1) * P.tiles_n;   // column tiles; pairs of SMs `per` apart share one
                const int row = ((first / per * 2 + (int)rank) * 4 + quarter) * groups + group, col = t.n + part * share;
                sums_out(P, row, t.slice, col, s, lane);
                sums_out(P, row, kGated ? P.p + t.slice : t.slice, kGated ? col : col + 32, s2, lane);
            }
        }
        if (lane == 0) stores_done();
        if (!ok && lane == 0 && P.status) atomicOr(P.status, SLICEGCN_DEVSTATUS_WAIT);
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
// zeros): fp32 as three planes, bf16 as one.  A thread makes 16 bytes of each plane.  Up to four matrices in a launch.
struct PackJob {
    const void* src;
    int64_t ld, rows, plane;
    int groups, width, pad, bf16, vec;
    int merge, block_rows, block_cols;   // weights of `merge` slices as one block-diagonal matrix: a slice's block, else merge = 1
    int ctas;
    __nv_bfloat16* dst;
};
struct PackArgs {
    int count;
    PackJob job[4];
};
__global__ void __launch_bounds__(256) ffn_pack_kernel(const __grid_constant__ PackArgs args) {
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    int cta = blockIdx.x, k = 0;
    while (cta >= args.job[k].ctas) cta -= args.job[k++].ctas;
    const PackJob& A = args.job[k];
    const int per_group = A.pad / 8, per_row = per_group * A.groups;
    const int64_t total = A.rows * per_row;
    for (int64_t i = (int64_t)cta * 256 + threadIdx.x; i < total; i += (int64_t)A.ctas * 256) {
        const int64_t row = total < (1ll << 32) ? (int64_t)((uint32_t)i / (uint32_t)per_row) : i / per_row;
        const int in_row = (int)(i - row * per_row), g = in_row / per_group, c = (in_row - g * per_group) * 8;
        // columns [first, left) of the eight have a source
        const int shift = A.merge > 1 ? (int)(row / A.block_rows % A.merge) * A.block_cols : 0;
        const int64_t at = row * A.ld + (int64_t)g * A.width + c - shift;
        const int first = shift - c, left = A.merge > 1 ? first + A.block_cols : A.width - c;
        uint4 out[3];
        if (A.bf16) {
            const uint16_t* s = static_cast<const uint16_t*>(A.src) + at;
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[q] = (2 * q >= first && 2 * q < left ? (uint32_t)s[2 * q] : 0u) |
                       (2 * q + 1 >= first && 2 * q + 1 < left ? (uint32_t)s[2 * q + 1] << 16 : 0u);
            out[0] = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            const float* s = static_cast<const float*>(A.src) + at;
            float v[8];
            if (A.vec && first <= 0 && left >= 8) {
                const float4 a = *reinterpret_cast<const float4*>(s), b = *reinterpret_cast<const float4*>(s + 4);
                v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = q >= first && q < left ? s[q] : 0.f;
            }
            uint32_t w[3][4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int part = 0; part < 3; ++part) {
                    const uint32_t lo = next_part(v[2 * q]);
                    w[part][q] = lo >> 16 | next_part(v[2 * q + 1]);
                }
#pragma unroll
            for (int part = 0; part < 3; ++part) out[part] = make_uint4(w[part][0], w[part][1], w[part][2], w[part][3]);
        }
        __nv_bfloat16* d = A.dst + i * 8;
        *reinterpret_cast<uint4*>(d) = out[0];
        if (!A.bf16) {
            *reinterpret_cast<uint4*>(d + A.plane) = out[1];
            *reinterpret_cast<uint4*>(d + 2 * A.plane) = out[2];
        }
    }
}

// Sums of columns, in a fixed order: chunks of rows by the first kernel, the chunks by the second.  A warp reads whole lines, 16 bytes
// a lane where they are aligned, and eight rows are on their way together.
constexpr int kSumChunks = 512;
// Rows of sums that the joining kernel adds by itself, without this kernel in front: eight at a time, one after another (gradients of
// 300 x 256 -> 2 x 256 bf16, ten rows: 26.5 -> 24 us; of 4,000 rows, 125 of sums: 54 -> 56.5).
constexpr int kJoinRows = 16;
struct SumArgs {
    const void* src;
    int64_t rows, ld, per;    // rows of a chunk
    int cols, bf16, vec;
    float* partial;           // [chunks][cols]
};
template <bool BF16, bool VEC>
__global__ void __launch_bounds__(256) ffn_colsum_kernel(const __grid_constant__ SumArgs A) {
    constexpr int W = VEC ? (BF16 ? 8 : 4) : 1;
    __shared__ float sh[8][32 * W + 1];
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = (blockIdx.x * 32 + x) * W;
    const int64_t r0 = blockIdx.y * A.per, r1 = min(r0 + A.per, A.rows);
    float s[W];
#pragma unroll
    for (int k = 0; k < W; ++k) s[k] = 0.f;
    if (c < A.cols) {
        auto add = [&](const uint4& t) {
            const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int k = 0; k < (VEC ? 4 : 0); ++k) {
                if (BF16)
                    s[(2 * k) % W] += __uint_as_float(w[k] << 16), s[(2 * k + 1) % W] += __uint_as_float(w[k] & 0xffff0000u);
                else
                    s[k % W] += __uint_as_float(w[k]);
            }
        };
        auto get = [&](int64_t r) {
            const int64_t at = r * A.ld + c;
            if (VEC) return BF16 ? *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(A.src) + at)
                                 : *reinterpret_cast<const uint4*>(static_cast<const float*>(A.src) + at);
            const float v = BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(A.src)[at]) : static_cast<const float*>(A.src)[at];
            return make_uint4(__float_as_uint(v), 0, 0, 0);
        };
        auto put = [&](const uint4& t) {
            if (VEC)
                add(t);
            else
                s[0] += __uint_as_float(t.x);
        };
        int64_t r = r0 + y;
        for (; r + 56 < r1; r += 64) {
            uint4 t[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = get(r + 8 * k);
#pragma unroll
            for (int k = 0; k < 8; ++k) put(t[k]);
        }
        for (; r < r1; r += 8) put(get(r));
    }
#pragma unroll
    for (int k = 0; k < W; ++k) sh[y][x * W + k] = s[k];
    __syncthreads();
    for (int k = threadIdx.x; k < 32 * W; k += 256) {
        const int col = blockIdx.x * 32 * W + k;
        if (col >= A.cols) break;
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) t += sh[q][k];
        A.partial[(int64_t)blockIdx.y * A.cols + col] = t;
    }
}
// out[0][i] (i < each) and out[1][i - each] = scale * the sum over `count` pieces of `total` numbers each.  Up to two such jobs in a launch.
struct JoinJob {
    const float* partial;
    int count, bf16;
    int64_t total, each, piece;   // piece: numbers of a piece, more than `total` where slices were merged
    float scale;
    void* out[2];
    int merge, rows, cols;        // merge > 1: of a slice's block, which lies on the diagonal of a piece's matrix of `merge` slices
    int ctas;
};
struct JoinArgs {
    JoinJob job[2];
};
__global__ void __launch_bounds__(256) ffn_join_kernel(const __grid_constant__ JoinArgs args) {
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    const int second_job = blockIdx.x >= args.job[0].ctas, cta = blockIdx.x - (second_job ? args.job[0].ctas : 0);
    const JoinJob& A = args.job[second_job];
    for (int64_t i = (int64_t)cta * 256 + threadIdx.x; i < A.total; i += (int64_t)A.ctas * 256) {
        const int second = i >= A.each;
        if (!A.out[second]) continue;
        const float* from = A.partial + i;
        if (A.merge > 1) {
            const int64_t row = i / A.cols, slice = row / A.rows;
            const int b = (int)(slice % A.merge);
            from = A.partial + row * A.cols * A.merge + b * A.cols + (i - row * A.cols);
        }
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        int k = 0;
        for (; k + 8 <= A.count; k += 8) {
            float t[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) t[q] = from[(k + q) * A.piece];
#pragma unroll
            for (int q = 0; q < 8; ++q) s[q & 3] += t[q];
        }
        for (; k < A.count; ++k) s[0] += from[k * A.piece];
        const float v = ((s[0] + s[1]) + (s[2] + s[3])) * A.scale;
        const int64_t at = second ? i - A.each : i;
        if (A.bf16)
            static_cast<__nv_bfloat16*>(A.out[second])[at] = __float2bfloat16_rn(v);
        else
            static_cast<float*>(A.out[second])[at] = v;
    }
}

// Where few tiles have a long k, pieces of k are different items, and this kernel adds their products up and does what the
// product's epilogue does otherwise.  A CTA has 32 rows x 32 columns, a thread four rows of a column.
struct FinishArgs {
    const float* partial;     // [splits][parts * p][n][cols]
    int splits, n, p, cols, gated, act, back;
    float scale;
    const float *b, *b2;
    const void* in;           // r or dout
    int64_t in_ld;
    void* out;                // out or dx
    int64_t out_ld;
    int in_bf16, out_bf16;
    __nv_bfloat16* dz;        // back: planes of da and dc
    int64_t dz_plane;
    int dz_row, dz_pad, dz_planes;
    float* sums;
};
template <int ACT>
__device__ __forceinline__ void finish_as(const FinishArgs& A, const float (&in)[4], float (&a)[4], float (&c)[4]) {
    if (A.back) {
        if (A.gated)
            backward_as<ACT, true, true>(A.scale, in, a, c);
        else
            backward_as<ACT, false, true>(A.scale, in, a, c);
    } else {
        if (A.gated)
            forward_as<ACT, true, true>(a, c);
        else
            forward_as<ACT, false, true>(a, c);
    }
}
__global__ void __launch_bounds__(256) ffn_finish_kernel(const __grid_constant__ FinishArgs A) {
    __shared__ float sh[2][8][33];
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int blocks = (A.cols + 31) / 32, slice = blockIdx.x / blocks, col = (blockIdx.x - slice * blocks) * 32 + x;
    const int row0 = blockIdx.y * 32 + y;
    const bool there = col < A.cols;
    const int64_t slot = (int64_t)A.n * A.cols, piece = slot * A.p * (1 + A.gated);
    float a[4], c[4], in[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int row = row0 + 8 * k;
        a[k] = c[k] = in[k] = 0.f;
        if (!there || row >= A.n) continue;
        const float* at = A.partial + slice * slot + (int64_t)row * A.cols + col;
        for (int s = 0; s < A.splits; ++s) {
            a[k] += at[s * piece];
            if (A.gated) c[k] += at[s * piece + A.p * slot];
        }
        if (A.b) a[k] += A.b[slice * A.cols + col];
        if (A.b2) c[k] += A.b2[slice * A.cols + col];
        if (A.in) {
            const int64_t i = (int64_t)row * A.in_ld + slice * A.cols + col;
            in[k] = A.in_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(A.in)[i]) : static_cast<const float*>(A.in)[i];
        }
    }
    if (A.act == SLICEGCN_ACT_SILU)
        finish_as<SLICEGCN_ACT_SILU>(A, in, a, c);
    else if (A.act == SLICEGCN_ACT_GELU)
        finish_as<SLICEGCN_ACT_GELU>(A, in, a, c);
    else if (A.act == SLICEGCN_ACT_RELU)
        finish_as<SLICEGCN_ACT_RELU>(A, in, a, c);
    else
        finish_as<SLICEGCN_ACT_NONE>(A, in, a, c);
    if (!A.back) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = row0 + 8 * k;
            if (!there || row >= A.n) continue;
            const int64_t i = (int64_t)row * A.out_ld + slice * A.cols + col;
            const float v = fmaf(a[k], A.scale, in[k]);
            if (A.out_bf16)
                static_cast<__nv_bfloat16*>(A.out)[i] = __float2bfloat16_rn(v);
            else
                static_cast<float*>(A.out)[i] = v;
        }
        return;
    }
    if (A.sums) {
        sh[0][y][x] = (a[0] + a[1]) + (a[2] + a[3]);   // rows past the end have no dout and add nothing
        sh[1][y][x] = (c[0] + c[1]) + (c[2] + c[3]);
    }
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        if (part && !A.gated) break;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = row0 + 8 * k;
            if (!there || row >= A.n) continue;
            __nv_bfloat16* to = A.dz + (int64_t)row * A.dz_row + (part * A.p + slice) * A.dz_pad + col;
            float v = part ? c[k] : a[k];
            if (A.dz_planes == 1) {
                *to = __float2bfloat16_rn(v);
            } else {
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<uint16_t*>(to + q * A.dz_plane) = (uint16_t)(next_part(v) >> 16);
            }
        }
    }
    if (A.sums) {
        __syncthreads();
        if (y < 1 + A.gated && there) {
            float t = 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) t += sh[y][q][x];
            A.sums[((int64_t)blockIdx.y * (A.p * (1 + A.gated)) + y * A.p + slice) * A.cols + col] = t;
        }
    }
}

// ------------------------------------------------------------------------------------------ a few rows
//
// Up to eight rows (serving): bound by reading the weights once, which tiles of 256 rows would do with few SMs and, in fp32, three
// times over.  A cluster has 128 columns; its CTAs and their warps split k.  Plain fp32 multiply-adds; the warps' sums meet in shared memory, the
// CTAs' in distributed shared memory.  One launch, no workspace.
constexpr int kRowsThreads = 256, kRowsCols = 128;
struct RowsArgs {
    const void* x;
    int64_t x_ld;
    const void *W, *W2;
    const float *b, *b2;
    const void* r;
    int64_t r_ld;
    void* out;
    int64_t out_ld;
    int n, in_s, out_s, act, per;   // per: k of a CTA, a multiple of 8
    float scale;
};
template <bool BF16>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
    return BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}
// Four of a lane's columns of one row of weights, as they lie in memory: neighbours (VEC), else every 32nd.
template <bool BF16, bool VEC>
struct Quad {
    float v[4];
    __device__ __forceinline__ void load(const void* W, int64_t at, int col, int out_s, int lane) {
        if (VEC) {
            const int64_t i = at + min(col + lane * 4, out_s - 4);
            if (BF16) {
                const uint2 t = __ldg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(W) + i));
                v[0] = __uint_as_float(t.x), v[1] = __uint_as_float(t.y);
            } else {
                const float4 t = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(W) + i));
                v[0] = t.x, v[1] = t.y, v[2] = t.z, v[3] = t.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = load_one<BF16>(W, at + min(col + lane + 32 * j, out_s - 1));
        }
    }
    __device__ __forceinline__ float get(int j) const {
        if (VEC && BF16) {
            const uint32_t t = __float_as_uint(v[j >> 1]);
            return __uint_as_float(j & 1 ? t & 0xffff0000u : t << 16);
        }
        return v[j];
    }
};
template <int R, bool GATED, bool BF16, bool VEC>
__global__ void __launch_bounds__(kRowsThreads) ffn_rows_kernel(const __grid_constant__ RowsArgs A) {
    constexpr int V = R * (1 + GATED);
    extern __shared__ __align__(16) float rows_smem[];
    float* xs = rows_smem;                        // [R][per]
    float* red = rows_smem + R * A.per;           // [8][V][128], then [V][128] in its first part
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t parts;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(parts));
    const uint32_t rank = cluster_rank();
    const int slice = blockIdx.y, col0 = (int)(blockIdx.x / parts) * kRowsCols, k0 = (int)rank * A.per;
    const int kc = max(0, min(A.per, A.in_s - k0));
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    for (int i = threadIdx.x; i < R * A.per; i += kRowsThreads) {
        const int r = i / A.per, k = i - r * A.per;
        xs[i] = r < A.n && k < kc ? load_one<BF16>(A.x, r * A.x_ld + (int64_t)slice * A.in_s + k0 + k) : 0.f;
    }
    __syncthreads();
    float acc[V][4];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[v][j] = 0.f;
    const int64_t base = ((int64_t)slice * A.in_s + k0) * A.out_s;
    constexpr int D = R == 1 && !GATED ? 16 : 8;  // rows of weights on their way together
    for (int k = warp * D; k < kc; k += 8 * D) {
        Quad<BF16, VEC> w[D], w2[D];
#pragma unroll
        for (int q = 0; q < D; ++q) {             // rows past the end repeat the last one; x is zero there
            const int64_t at = base + (int64_t)min(k + q, kc - 1) * A.out_s;
            w[q].load(A.W, at, col0, A.out_s, lane);
            if (GATED) w2[q].load(A.W2, at, col0, A.out_s, lane);
        }
#pragma unroll
        for (int q0 = 0; q0 < D; q0 += 4) {
            if (q0 >= 8 && k + q0 >= A.per) break;   // per is a multiple of 8, D may be 16
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 x4 = *reinterpret_cast<const float4*>(xs + r * A.per + k + q0);
                const float xv[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        acc[r][j] = fmaf(xv[q], w[q0 + q].get(j), acc[r][j]);
                        if (GATED) acc[(R + r) % V][j] = fmaf(xv[q], w2[q0 + q].get(j), acc[(R + r) % V][j]);
                    }
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float* to = red + (warp * V + v) * kRowsCols;
#pragma unroll
        for (int j = 0; j < 4; ++j) to[VEC ? lane * 4 + j : lane + 32 * j] = acc[v][j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < V * kRowsCols; i += kRowsThreads) {
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) t += red[q * V * kRowsCols + i];
        red[i] = t;                               // read by this thread alone so far
    }
    if (parts > 1)
        cluster_sync();
    else
        __syncthreads();
    const int share = kRowsCols / (int)parts;     // columns that this CTA finishes
    for (int i = threadIdx.x; i < R * share; i += kRowsThreads) {
        const int r = i / share, c = (int)rank * share + (i - r * share), col = col0 + c;
        float a[1] = {0.f}, g[1] = {0.f};
        for (uint32_t q = 0; q < parts; ++q) {
            uint32_t at = smem_u32(red + r * kRowsCols + c);
            asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(at) : "r"(q));
            float t;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(t) : "r"(at) : "memory");
            a[0] += t;
            if (GATED) {
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(t) : "r"(at + R * kRowsCols * 4) : "memory");
                g[0] += t;
            }
        }
        if (r >= A.n || col >= A.out_s) continue;
        const int at = slice * A.out_s + col;
        if (A.b) a[0] += A.b[at];
        if (GATED && A.b2) g[0] += A.b2[at];
        if (A.act == SLICEGCN_ACT_SILU)
            forward_as<SLICEGCN_ACT_SILU, GATED, true>(a, g);
        else if (A.act == SLICEGCN_ACT_GELU)
            forward_as<SLICEGCN_ACT_GELU, GATED, true>(a, g);
        else if (A.act == SLICEGCN_ACT_RELU)
            forward_as<SLICEGCN_ACT_RELU, GATED, true>(a, g);
        else
            forward_as<SLICEGCN_ACT_NONE, GATED, true>(a, g);
        const float v = A.r ? fmaf(a[0], A.scale, load_one<BF16>(A.r, r * A.r_ld + at)) : a[0] * A.scale;
        if (BF16)
            static_cast<__nv_bfloat16*>(A.out)[r * A.out_ld + at] = __float2bfloat16_rn(v);
        else
            static_cast<float*>(A.out)[r * A.out_ld + at] = v;
    }
    if (parts > 1) cluster_sync();                // no CTA's memory goes while another reads it
}

// ------------------------------------------------------------------------------------------ little work in awkward layouts
//
// Forward products of fp32, or of bf16 rows off 16 bytes, would be laid out anew before the tensor cores can read them; where there is
// little arithmetic, or few columns for much of x, that costs more than plain fp32 multiply-adds (19,697 x 25 -> 14 fp32: 7 us, by
// way of the tensor cores 16; 200,000 x 600 -> 8: 179 and 543).  Tiles of 64 x 64, sixteen k at a time through shared memory, 4 x 4
// results a thread (gated: of both products); one launch, no workspace.
constexpr int kLittleK = 16, kLittleTile = 64;
struct LittleArgs {
    const void* x;
    int64_t x_ld;
    const void *W, *W2;
    const float *b, *b2;
    const void* r;
    int64_t r_ld;
    void* out;
    int64_t out_ld;
    int n, in_s, out_s, act, tiles_n;
    float scale;
    int x_vec, w_vec;   // fp32: 16 bytes at a time are aligned
};
// Bias, activation, gate, scale, residual and store of a thread's R rows x 4 columns.
template <bool GATED, bool BF16, int R>
__device__ __forceinline__ void little_finish(const LittleArgs& A, int slice, int row0, int col0, float (&a)[R * 4], float (&c)[R * 4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int col = col0 + j;
        const float b = A.b && col < A.out_s ? A.b[slice * A.out_s + col] : 0.f, b2 = GATED && A.b2 && col < A.out_s ? A.b2[slice * A.out_s + col] : 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i) a[i * 4 + j] += b, c[i * 4 + j] += b2;
    }
    if (A.act == SLICEGCN_ACT_SILU)
        forward_as<SLICEGCN_ACT_SILU, GATED, true>(a, c);
    else if (A.act == SLICEGCN_ACT_GELU)
        forward_as<SLICEGCN_ACT_GELU, GATED, true>(a, c);
    else if (A.act == SLICEGCN_ACT_RELU)
        forward_as<SLICEGCN_ACT_RELU, GATED, true>(a, c);
    else
        forward_as<SLICEGCN_ACT_NONE, GATED, true>(a, c);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int row = row0 + i;
        if (row >= A.n) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = col0 + j;
            if (col >= A.out_s) break;
            const int64_t o = (int64_t)slice * A.out_s + col;
            const float v = A.r ? fmaf(a[i * 4 + j], A.scale, load_one<BF16>(A.r, row * A.r_ld + o)) : a[i * 4 + j] * A.scale;
            if (BF16)
                static_cast<__nv_bfloat16*>(A.out)[row * A.out_ld + o] = __float2bfloat16_rn(v);
            else
                static_cast<float*>(A.out)[row * A.out_ld + o] = v;
        }
    }
}
template <bool GATED, bool BF16>
__global__ void __launch_bounds__(256) ffn_little_kernel(const __grid_constant__ LittleArgs A) {
    __shared__ __align__(16) float xs[2][kLittleK][kLittleTile + 4];
    __shared__ __align__(16) float ws[2][1 + GATED][kLittleK][kLittleTile];
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    const int tile_n = blockIdx.x % A.tiles_n, slice = blockIdx.x / A.tiles_n, row0 = blockIdx.y * kLittleTile, col0 = tile_n * kLittleTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t wat = (int64_t)slice * A.in_s * A.out_s;
    float fx[4], fw[1 + GATED][4];
    // of x: row threadIdx / 16 + 16 q, k threadIdx % 16; of W: k threadIdx / 64 + 4 q, column threadIdx % 64
    auto fetch = [&](int k0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int row = row0 + (threadIdx.x >> 4) + 16 * q, k = k0 + (threadIdx.x & 15);
            fx[q] = row < A.n && k < A.in_s ? load_one<BF16>(A.x, row * A.x_ld + (int64_t)slice * A.in_s + k) : 0.f;
            const int wk = k0 + (threadIdx.x >> 6) + 4 * q, col = col0 + (threadIdx.x & 63);
            const bool there = wk < A.in_s && col < A.out_s;
            fw[0][q] = there ? load_one<BF16>(A.W, wat + (int64_t)wk * A.out_s + col) : 0.f;
            if (GATED) fw[GATED][q] = there ? load_one<BF16>(A.W2, wat + (int64_t)wk * A.out_s + col) : 0.f;
        }
    };
    auto put = [&](int to) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            xs[to][threadIdx.x & 15][(threadIdx.x >> 4) + 16 * q] = fx[q];
#pragma unroll
            for (int g = 0; g < 1 + GATED; ++g) ws[to][g][(threadIdx.x >> 6) + 4 * q][threadIdx.x & 63] = fw[g][q];
        }
    };
    float a[16], c[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) a[j] = c[j] = 0.f;
    fetch(0);
    put(0);
    __syncthreads();
    int at = 0;
    for (int k0 = 0; k0 < A.in_s; k0 += kLittleK, at ^= 1) {
        const bool more = k0 + kLittleK < A.in_s;
        if (more) fetch(k0 + kLittleK);   // on its way while this step is worked on
#pragma unroll
        for (int k = 0; k < kLittleK; ++k) {
            const float4 xv = *reinterpret_cast<const float4*>(&xs[at][k][ty * 4]);
            const float xr[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
            for (int g = 0; g < 1 + GATED; ++g) {
                const float4 wv = *reinterpret_cast<const float4*>(&ws[at][g][k][tx * 4]);
                const float wr[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float& to = g ? c[i * 4 + j] : a[i * 4 + j];
                        to = fmaf(xr[i], wr[j], to);
                    }
            }
        }
        if (more) put(at ^ 1);
        __syncthreads();
    }
    little_finish<GATED, BF16, 4>(A, slice, row0 + ty * 4, col0 + tx * 4, a, c);
}

// The same for fp32, by asynchronous copies of 16 bytes or (other alignments) 4, two steps ahead.  TN: columns of a tile; with 16 it
// has 128 rows, since few columns make x the main traffic.
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool there, int bytes) {   // zeros where nothing is there
    const int have = there ? bytes : 0;
    if (bytes == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(have) : "memory");
}
template <bool GATED, int TN>
__global__ void __launch_bounds__(256) ffn_little_f32_kernel(const __grid_constant__ LittleArgs A) {
    constexpr int TM = TN == 16 ? 128 : 64, R = TM * TN / 1024, XS = kLittleK + 4, kDeep = 3, kTx = TN / 4;
    __shared__ __align__(16) float xs[kDeep][TM][XS];
    __shared__ __align__(16) float ws[kDeep][1 + GATED][kLittleK][TN];
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    const int tile_n = blockIdx.x % A.tiles_n, slice = blockIdx.x / A.tiles_n, row0 = blockIdx.y * TM, col0 = tile_n * TN;
    const int tx = threadIdx.x % kTx, ty = threadIdx.x / kTx, tid = threadIdx.x;
    const float* x = static_cast<const float*>(A.x) + (int64_t)slice * A.in_s;
    const float* W[2] = {static_cast<const float*>(A.W) + (int64_t)slice * A.in_s * A.out_s,
                         GATED ? static_cast<const float*>(A.W2) + (int64_t)slice * A.in_s * A.out_s : nullptr};
    const int steps = (A.in_s + kLittleK - 1) / kLittleK;
    auto fetch = [&](int step) {
        const int k0 = step * kLittleK, to = step % kDeep;
        if (step < steps) {
            if (A.x_vec) {
#pragma unroll
                for (int q = 0; q < TM / 64; ++q) {
                    const int r = q * 64 + (tid >> 2), k = (tid & 3) * 4;
                    const bool there = row0 + r < A.n && k0 + k < A.in_s;   // in_s is a multiple of 4
                    copy_async(smem_u32(&xs[to][r][k]), there ? x + (row0 + r) * A.x_ld + k0 + k : x, there, 16);
                }
            } else {
#pragma unroll
                for (int q = 0; q < TM / 16; ++q) {
                    const int r = q * 16 + (tid >> 4), k = tid & 15;
                    const bool there = row0 + r < A.n && k0 + k < A.in_s;
                    copy_async(smem_u32(&xs[to][r][k]), there ? x + (row0 + r) * A.x_ld + k0 + k : x, there, 4);
                }
            }
#pragma unroll
            for (int g = 0; g < 1 + GATED; ++g) {
                if (A.w_vec) {
                    if (tid < kLittleK * kTx) {
                        const int k = tid / kTx, c = tid % kTx * 4;
                        const bool there = k0 + k < A.in_s && col0 + c < A.out_s;   // out_s is a multiple of 4
                        copy_async(smem_u32(&ws[to][g][k][c]), there ? W[g] + (int64_t)(k0 + k) * A.out_s + col0 + c : W[g], there, 16);
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < TN / 16; ++q) {
                        const int e = q * 256 + tid, k = e / TN, c = e % TN;
                        const bool there = k0 + k < A.in_s && col0 + c < A.out_s;
                        copy_async(smem_u32(&ws[to][g][k][c]), there ? W[g] + (int64_t)(k0 + k) * A.out_s + col0 + c : W[g], there, 4);
                    }
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    float a[R * 4], c[R * 4];
#pragma unroll
    for (int j = 0; j < R * 4; ++j) a[j] = c[j] = 0.f;
    fetch(0);
    fetch(1);
    for (int step = 0; step < steps; ++step) {
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncthreads();   // this step has come, and the one before is no longer read
        fetch(step + 2);
        const int at = step % kDeep;
#pragma unroll
        for (int k0 = 0; k0 < kLittleK; k0 += 4) {
            float xr[R][4];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float4 t = *reinterpret_cast<const float4*>(&xs[at][ty * R + i][k0]);
                xr[i][0] = t.x, xr[i][1] = t.y, xr[i][2] = t.z, xr[i][3] = t.w;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int g = 0; g < 1 + GATED; ++g) {
                    const float4 t = *reinterpret_cast<const float4*>(&ws[at][g][k0 + k][tx * 4]);
                    const float wr[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                    for (int i = 0; i < R; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float& to = g ? c[i * 4 + j] : a[i * 4 + j];
                            to = fmaf(xr[i][k], wr[j], to);
                        }
                }
        }
    }
    little_finish<GATED, false, R>(A, slice, row0 + ty * R, col0 + tx * 4, a, c);
}

// ------------------------------------------------------------------------------------------ host

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// An operand (bf16) or a result: [plane][row][group][width] by strides in elements (multiples of 16 bytes where there is more than one).
struct Operand {
    const void* base = nullptr;
    int64_t rows = 0, ld = 0, group_stride = 0, plane_stride = 0;
    int width = 0, groups = 1, planes = 1;
    bool f32 = false;      // a result of fp32
};
slicegcn_status_t make_map(CUtensorMap* map, const Operand& o, int box_rows, bool result = false) {
    static EncodeFn encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
            fn = nullptr;
        return reinterpret_cast<EncodeFn>(fn);
    }();
    if (!encode) SGCN_FAIL(SLICEGCN_ERR_CUDA, "ffn: the driver has no tensor map encoder");
    const cuuint64_t dims[4] = {(cuuint64_t)o.width, (cuuint64_t)o.rows, (cuuint64_t)o.groups, (cuuint64_t)o.planes};
    const int elem = o.f32 ? 4 : 2;
    const cuuint64_t strides[3] = {(cuuint64_t)(o.rows > 1 ? o.ld : 8) * elem, (cuuint64_t)(o.groups > 1 ? o.group_stride : 8) * elem,
                                   (cuuint64_t)(o.planes > 1 ? o.plane_stride : 8) * elem};
    const cuuint32_t box[4] = {result ? 32u : 64u, (cuuint32_t)box_rows, 1, 1}, ones[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, o.f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(o.base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              result && !o.f32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) SGCN_FAIL(SLICEGCN_ERR_CUDA, "ffn: tensor map refused (%d)", (int)r);
    return SLICEGCN_OK;
}

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Steps between emptyings.  fp32's digits allow some twenty additions in tensor memory at the sum's full size: of six products two
// steps' (those of parts 0 and four between them), else the last product of four steps.  For biases' gradients beside results of bf16: 512 k.
// Weights' gradients of bf16, which are sums over all rows: 512 rows, a shift of 2^-20 on average (4,096 rows: 2^-16.7 measured, for the
// same time: 219 and 220 us for 169,343 x 1,024 -> 256, 575 and 579 us for 169,343 x 256 -> 2 x 1,024).
constexpr int kChunkRows = 8;
int chunk_of(int pairs) { return pairs == 6 ? 2 : 4; }
constexpr int kChunkBiases = 8;
// Biases' gradients are fp32 sums over da, whatever its type, and the accumulator's cuts go in one direction, so that sums over rows do
// not average them out: 2^-28 of the whole sum a column at worst, half of that where the sum grows evenly.  Up to this many steps
// (768 columns: 2^-18.4 and 2^-19.4; measured 2^-20.2 over rows of random numbers) they are left in; longer sums are emptied as for fp32,
// every 512 columns (1,024 and 4,096 columns: 2^-20.7).
constexpr int kLongSteps = 12;

// How a product is cut up.
struct Cut {
    int nt = 128, tiles_m = 1, tiles_n = 1, splits = 1, kb = 1, chunk = 1;   // kb: steps of a piece of k, the same for each
    bool swapped = false, pair = false;
    int fixed = 0;   // pairs of SMs that work, where each stays with one column tile
    double cost = 1e300;
};
// SM cycles of `items` tiles: a 64-wide step takes its MMAs' time, or with half-width tiles rather what its copies take; a tile's start
// and end about 4,500.  Splitting k adds 16,000 (a launch, a kernel that keeps the sums in registers) and each piece's way to memory and back (3,400 bytes a cycle over all SMs).
double cost_of(int64_t tiles, int splits, int64_t kb, int pairs, int nt, double piece_bytes) {
    const double step = nt == 128 ? 512 : 430;
    return (double)ceil_div(tiles * splits, kPairs) * ((double)kb * pairs * step + 4500.0) +
           (splits > 1 ? 16000.0 + 2.0 * splits * piece_bytes / 3400.0 : 0.0);
}
int pairs_of(int pa, int pb) {
    int n = 0;
    for (int i = 0; i < pa; ++i)
        for (int j = 0; j < pb; ++j) n += i + j < 3;
    return n;
}
// Tiles of a product over the rows of x (gated: of two at once); half-width ones where they cover the columns, or where whole ones
// would leave pairs of SMs idle; pieces of k where there are few tiles (as two separate products then, if gated).  emptied: steps between
// emptyings, 0: none but those of pieces.
Cut cut_rows(int64_t n, int p, int cols, bool gated, int64_t kb, int pairs, int emptied) {
    Cut best;
    const int chunk = pairs > 1 ? chunk_of(pairs) : 1;
    auto consider = [&](int s) {
        Cut c;
        const int per = s > 1 ? (int)up(ceil_div(kb, s), chunk) : (int)kb;
        s = (int)ceil_div(kb, per);
        const bool two = gated && s == 1;
        const int one = two ? 64 : 128, slices = p * (gated && !two ? 2 : 1);
        c.tiles_m = (int)ceil_div(n, 256);
        c.nt = cols <= one || (int64_t)c.tiles_m * slices * ceil_div(cols, 2 * one) * s * 2 <= kPairs ? 64 : 128;
        c.tiles_n = (int)ceil_div(cols, two ? c.nt : 2 * c.nt);
        c.splits = s, c.kb = per, c.chunk = emptied ? emptied : s > 1 ? chunk_of(pairs) : per;
        const int64_t tiles = (int64_t)slices * c.tiles_m * c.tiles_n;
        c.cost = cost_of(tiles, s, per, pairs, c.nt, 4.0 * n * slices * cols);
        if (c.cost < best.cost) best = c;
        return tiles;
    };
    const int64_t tiles = consider(1);
    if (tiles < kPairs)   // else the SMs have work anyway
        for (int r = 1; r <= 2; ++r)
            for (int wide = 1; wide <= 4; wide *= 2) {   // the pieces' tiles are other ones, to be met once or twice by each pair of SMs
                const int64_t s = std::min<int64_t>(32, kPairs * r / std::max<int64_t>(1, tiles * wide / 2));
                if (s > 1) consider((int)s);
            }
    return best;
}
// Pairs of SMs that stay with a column tile each, item after item: their biases and column sums stay in registers (gradients of
// 169,343 x 256 -> 2 x 1,024: 610 -> 580 us).  Where that leaves no more than two idle, else 0.
int fixed_pairs(const Cut& c, int p) {
    const int64_t per = (int64_t)p * c.tiles_n;
    if (c.splits > 1 || per > kPairs) return 0;
    const int64_t used = std::min<int64_t>(kPairs / per, c.tiles_m) * per;
    return used >= 72 ? (int)used : 0;
}
// Pieces of the rows for dW; which of the two operands gives the tile's 256 rows.
Cut cut_dw(int64_t n, int p, int parts, int in_s, int out_s, int pairs) {
    Cut best;
    for (int swapped = 0; swapped < 2; ++swapped) {
        const int m = swapped ? in_s : out_s, k = swapped ? out_s : in_s;
        const int64_t all = ceil_div(n, 64);
        const bool pair = swapped && parts == 2;
        const int one = pair ? 64 : 128, slices = pair ? p : parts * p, nt = k <= one ? 64 : 128;
        const int64_t tiles_m = ceil_div(m, 256), tiles_n = ceil_div(k, pair ? nt : 2 * nt), tiles = slices * tiles_m * tiles_n;
        for (int r : {0, 1, 2, 4, 8, 12, 16}) {   // pieces that fill a quarter, a half of the pairs of SMs, all once, twice ...
            Cut c;
            c.swapped = swapped, c.pair = pair, c.nt = nt, c.tiles_m = (int)tiles_m, c.tiles_n = (int)tiles_n;
            c.kb = (int)ceil_div(all, std::max<int64_t>(1, std::min<int64_t>(2 * kPairs, kPairs * r / (4 * tiles))));
            c.splits = (int)ceil_div(all, c.kb);
            c.chunk = pairs > 1 ? chunk_of(pairs) : kChunkRows;
            c.cost = cost_of(tiles, c.splits, c.kb, pairs, c.nt, 4.0 * parts * p * in_s * out_s);
            if (c.cost < best.cost) best = c;
        }
    }
    return best;
}

// What a call needs in the workspace, and where.
//
// Slices are taken together, their weights as one block-diagonal matrix, where that costs less: tiles and 64-wide steps of k have room for
// columns of several narrow slices (8 slices of 14 -> 23 columns: a third of the time).
struct Plan {
    int p = 1, in_s = 1, out_s = 1, merge = 1;   // slices and their columns as the products see them
    bool digits = false;    // of the product that gives da and dc: those of fp32
    bool rows = false, little = false, pack_x = false, pack_w = false, pack_g = false, dz = false;
    int x_planes = 1, w_planes = 1, z_planes = 1;
    int in_pad = 0, out_pad = 0, parts = 1, sum_chunks = 1;
    Cut product, dx, dw;
    int64_t sum_rows = 0;   // of what the column sums are taken of
    int64_t x_at = 0, w_at = 0, w2_at = 0, z_at = 0, sums_at = 0, chunks_at = 0, partial_at = 0, bytes = 0;
};

bool unaligned(const void* p, int64_t ld, int groups, int width) {
    return (uintptr_t)p % 16 || ld % 8 || (groups > 1 && width % 8);
}
// CTAs of a cluster that split k for a few rows, and k of each.
int rows_parts(const slicegcn_ffn_desc* d, int* per) {
    const int64_t blocks = ceil_div(d->out_s, kRowsCols) * d->num_slices;
    int parts = 1;
    while (parts < 8 && blocks * parts < 2 * 148 && d->in_s / (2 * parts) >= 64) parts *= 2;
    while (parts < 8 && ceil_div(d->in_s, parts) > 2048) parts *= 2;
    *per = (int)up(ceil_div(d->in_s, parts), 8);
    return parts;
}

void plan(const slicegcn_ffn_desc* d, const void* x, const void* dout, Plan& q) {
    const int64_t n = d->n;
    const bool f32 = d->dtype == SLICEGCN_F32, back = dout != nullptr;
    q.parts = d->W2 ? 2 : 1;
    q.x_planes = q.w_planes = f32 ? 3 : 1;
    q.z_planes = d->grad_dtype == SLICEGCN_F32 ? 3 : 1;
    if (!back && n <= 8 && d->in_s <= 16384) {
        q.rows = true;
        return;
    }
    const bool dz = back && (d->act != SLICEGCN_ACT_NONE || d->W2), gated = d->W2 != nullptr;
    const int pairs = pairs_of(q.x_planes, q.w_planes);
    double least = 1e300;
    const int dx_pairs = pairs_of(q.z_planes, q.w_planes), dw_pairs = pairs_of(q.z_planes, q.x_planes);
    for (int m = 1; m <= d->num_slices; ++m) {
        const int64_t ins = (int64_t)m * d->in_s, outs = (int64_t)m * d->out_s;
        if (d->num_slices % m || (m > 1 && (ins > 2048 || outs > 8192))) continue;
        const int p = d->num_slices / m;
        const bool digits = f32 || (back && (q.z_planes == 3 || ceil_div(ins, 64) > kLongSteps));
        Cut c[3];
        if (!back || dz) c[0] = cut_rows(n, p, (int)outs, gated, ceil_div(ins, 64), pairs, !digits ? 0 : f32 || q.z_planes == 3 ? chunk_of(pairs) : kChunkBiases);
        if (back) c[1] = cut_rows(n, p, (int)ins, false, q.parts * ceil_div(outs, 64), dx_pairs, dx_pairs > 1 ? chunk_of(dx_pairs) : 0), c[2] = cut_dw(n, p, q.parts, (int)ins, (int)outs, dw_pairs);
        double cost = (!back || dz ? c[0].cost : 0.0) + (back ? c[1].cost + c[2].cost : 0.0);
        if (m > 1) cost += 0.1 * cost + 4000 + (double)q.parts * p * ins * outs * (f32 ? 10 : 4) / 3400;            // weights are laid out anew; the model's margin
        if (!f32 && unaligned(x, d->x_ld, p, (int)ins)) cost += 4000 + (double)n * p * ins * 6 / 3400;              // x is, or needs not to be
        if (cost < least) least = cost, q.merge = m, q.p = p, q.in_s = (int)ins, q.out_s = (int)outs, q.digits = digits, q.product = c[0], q.dx = c[1], q.dw = c[2];
    }
    q.in_pad = (int)up(q.in_s, 8);
    q.out_pad = (int)up(q.out_s, 8);
    const int p = q.p;
    q.pack_x = f32 || unaligned(x, d->x_ld, p, q.in_s);
    q.pack_w = f32 || q.merge > 1 || unaligned(d->W, d->out_s, 1, 8) || unaligned(d->W2, d->out_s, 1, 8);
    q.dz = dz;
    q.pack_g = back && !q.dz && (q.z_planes == 3 || unaligned(dout, d->dout_ld, p, q.out_s));
    int64_t at = 0, partial = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    if (q.pack_x) q.x_at = take(2 * q.x_planes * n * p * q.in_pad);
    if (q.pack_w) {
        q.w_at = take(2LL * q.w_planes * p * q.in_s * q.out_pad);
        if (d->W2) q.w2_at = take(2LL * q.w_planes * p * q.in_s * q.out_pad);
    }
    const int64_t cols = (int64_t)q.parts * p * q.out_s;
    if (!back && (q.pack_x || q.pack_w)) {
        // SM cycles, as measured: a step of a tile where there are tiles enough for all SMs, and where there is one; against the tensor
        // cores' tiles, the matrices' way through the workspace and the packing launch
        const bool narrow = f32 && d->out_s <= 16;
        const int64_t tiles = ceil_div(n, narrow ? 128 : kLittleTile) * ceil_div(d->out_s, narrow ? 16 : kLittleTile) * d->num_slices;
        const double steps = (double)ceil_div(d->in_s, kLittleK), wave = (double)tiles / 148;
        const double step = narrow ? (gated ? 1070 : 825) : f32 ? (gated ? 2280 : 1180) : (gated ? 3200 : 1600);
        const double least_step = narrow ? 1270 : f32 ? (gated ? 2050 : 1400) : (gated ? 2600 : 1800);
        const double little = 1.2 * steps * std::max(least_step, step * wave) + 1200 * wave + 6000;
        const double packed = (double)n * p * q.in_s * (f32 ? 16 : 6) + (double)q.parts * p * q.in_s * q.out_s * (f32 ? 16 : 6);
        if (ceil_div(n, narrow ? 128 : kLittleTile) <= 65535 && little < q.product.cost + packed / 3400 + 10000) {
            q.little = true;
            q.bytes = 0;
            return;
        }
    }
    if (!back || q.dz) {
        if (q.product.splits > 1) partial = 4LL * q.product.splits * n * cols;
        // a long k leaves little to gain, and idle pairs of SMs to lose
        if (!back && d->W2 && !f32 && q.in_s <= 512) q.product.fixed = fixed_pairs(q.product, p);
    }
    if (back) {
        if (q.dz || q.pack_g) q.z_at = take(2 * q.z_planes * n * q.parts * p * q.out_pad);
        if (q.dz && !q.digits) q.product.fixed = fixed_pairs(q.product, p);
        q.sum_rows = !q.dz ? n : !q.product.fixed ? ceil_div(n, 32) : q.product.fixed / (p * q.product.tiles_n) * (q.product.nt == 64 ? 16 : 8);
        if (q.dz) q.sums_at = take(4 * q.sum_rows * cols);
        const int64_t rows = q.sum_rows;
        q.sum_chunks = (int)std::max<int64_t>(1, std::min<int64_t>({kSumChunks, ceil_div(148 * 6, ceil_div(cols, 128)), rows / 64}));
        q.chunks_at = take(4 * q.sum_chunks * cols);
        if (q.dx.splits > 1) partial = std::max<int64_t>(partial, 4LL * q.dx.splits * n * p * q.in_s);
        if (q.dw.splits > 1 || q.merge > 1) partial = std::max<int64_t>(partial, 4LL * q.dw.splits * q.in_s * cols);
    }
    if (partial) q.partial_at = take(partial);
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
    if (!std::isfinite((float)d->scale)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: scale is not finite, or past the range of fp32");
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
    if (ld > INT32_MAX) SGCN_FAIL(SLICEGCN_ERR_OVERFLOW, "ffn: leading dimension of %s too large", name);
    if ((uintptr_t)p % (dtype == SLICEGCN_F32 ? 4 : 2)) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: %s is not aligned to its type", name);
    return SLICEGCN_OK;
}
slicegcn_status_t check_workspace(const void* ws, int64_t have, int64_t need, const int32_t* status) {
    if ((uintptr_t)ws % 128 || (uintptr_t)status % 4) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "ffn: the workspace (128 bytes) or status is not aligned");
    if (need > 0 && (!ws || have < need)) SGCN_FAIL(SLICEGCN_ERR_ALLOC, "ffn: workspace too small (%lld < %lld bytes)", (long long)have, (long long)need);
    return SLICEGCN_OK;
}

void add_pack(PackArgs& args, const void* src, int64_t ld, int64_t rows, int groups, int width, bool bf16, void* dst, Operand& o) {
    PackJob& A = args.job[args.count++];
    A.src = src, A.ld = ld, A.rows = rows, A.groups = groups, A.width = width, A.pad = (int)up(width, 8), A.bf16 = bf16;
    A.vec = !bf16 && (uintptr_t)src % 16 == 0 && ld % 4 == 0 && (groups == 1 || width % 4 == 0);
    A.merge = 1, A.block_rows = 1, A.block_cols = width;
    A.plane = rows * groups * A.pad;
    A.dst = static_cast<__nv_bfloat16*>(dst);
    A.ctas = (int)std::min<int64_t>(ceil_div(A.plane / 8, 256), 148 * 16);
    o.base = dst, o.rows = rows, o.ld = (int64_t)groups * A.pad, o.group_stride = A.pad, o.plane_stride = A.plane;
    o.width = width, o.groups = groups, o.planes = bf16 ? 1 : 3;
}
slicegcn_status_t run_packs(const PackArgs& args, cudaStream_t st) {
    int ctas = 0;
    for (int k = 0; k < args.count; ++k) ctas += args.job[k].ctas;
    return ctas ? launch_after(ffn_pack_kernel, dim3(ctas), 256, 0, st, args) : SLICEGCN_OK;
}

// A kernel's limit of dynamic shared memory, a constant of the kernel, set at its first launch on each device (a call costs a
// microsecond).  Threads that come at the same time all set it.
struct SmemLimit {
    std::atomic<uint64_t> devices{0};
    slicegcn_status_t set(const void* kernel, int bytes) {
        int dev = 0;
        SGCN_CUDA(cudaGetDevice(&dev));
        const uint64_t bit = 1ull << (dev & 63);
        if (dev < 64 && (devices.load(std::memory_order_relaxed) & bit)) return SLICEGCN_OK;
        SGCN_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
        devices.fetch_or(bit, std::memory_order_relaxed);
        return SLICEGCN_OK;
    }
};
template <int MODE, bool PROMO, int ACT>
slicegcn_status_t launch_as(const Params& P, cudaStream_t st) {
    static SmemLimit limit;
    SGCN_TRY(limit.set((const void*)ffn_kernel<MODE, PROMO, ACT>, kSmem));
    return launch_after(ffn_kernel<MODE, PROMO, ACT>, dim3(2 * P.clusters), kThreads, kSmem, st, P);
}
template <int MODE, bool PROMO>
slicegcn_status_t launch(const Params& P, int act, cudaStream_t st) {
    switch (act) {
        case SLICEGCN_ACT_RELU: return launch_as<MODE, PROMO, SLICEGCN_ACT_RELU>(P, st);
        case SLICEGCN_ACT_SILU: return launch_as<MODE, PROMO, SLICEGCN_ACT_SILU>(P, st);
        case SLICEGCN_ACT_GELU: return launch_as<MODE, PROMO, SLICEGCN_ACT_GELU>(P, st);
        default: return launch_as<MODE, PROMO, SLICEGCN_ACT_NONE>(P, st);
    }
}

slicegcn_status_t set_cut(Params& P, const Cut& c, bool dw) {
    P.nt = c.nt, P.tiles_m = c.tiles_m, P.tiles_n = c.tiles_n, P.splits = c.splits, P.kb_total = c.kb, P.chunk = c.chunk;
    P.clusters = c.fixed ? c.fixed : (int)std::min<int64_t>((int64_t)P.slices * P.tiles_m * P.tiles_n * P.splits, kPairs);
    P.fixed = c.fixed > 0;
    P.group = dw || P.fixed ? 1 : std::min(c.tiles_m, 8);
    const int64_t tiles = (int64_t)P.slices * P.tiles_m * P.tiles_n;
    if (tiles * P.splits > (1 << 30)) SGCN_FAIL(SLICEGCN_ERR_OVERFLOW, "ffn: too many tiles");
    P.items = (int)tiles * P.splits;
    P.by_split = divide_by((int)tiles);
    P.by_n = divide_by(P.tiles_n);
    P.by_group = divide_by(P.group * P.slices * P.tiles_n);
    P.by_m = divide_by(dw ? P.tiles_m : P.group);
    P.by_last = divide_by(std::max(1, P.tiles_m % P.group));
    return SLICEGCN_OK;
}

// x, W and W2 as operands; what has to be laid out anew is added to the packs.
void operands(const slicegcn_ffn_desc* d, const Plan& q, const void* x, char* ws, Operand& ox, Operand (&ow)[2], PackArgs& packs) {
    const bool bf16 = d->dtype == SLICEGCN_BF16;
    const int p = q.p;
    if (q.pack_x)
        add_pack(packs, x, d->x_ld, d->n, p, q.in_s, bf16, ws + q.x_at, ox);
    else
        ox.base = x, ox.rows = d->n, ox.ld = d->x_ld, ox.group_stride = q.in_s, ox.width = q.in_s, ox.groups = p;
    for (int k = 0; k < q.parts; ++k) {
        const void* w = k ? d->W2 : d->W;
        if (q.pack_w) {
            add_pack(packs, w, d->out_s, (int64_t)p * q.in_s, 1, q.out_s, bf16, ws + (k ? q.w2_at : q.w_at), ow[k]);
            PackJob& job = packs.job[packs.count - 1];
            job.merge = q.merge, job.block_rows = d->in_s, job.block_cols = d->out_s;
            job.vec = job.vec && q.merge == 1;
            ow[k].groups = p, ow[k].rows = q.in_s, ow[k].group_stride = (int64_t)q.in_s * q.out_pad;
        } else {
            ow[k].base = w, ow[k].rows = q.in_s, ow[k].ld = q.out_s, ow[k].group_stride = (int64_t)q.in_s * q.out_s, ow[k].width = q.out_s, ow[k].groups = p;
        }
    }
    if (q.parts == 1) ow[1] = ow[0];
}

// The product a = x W (and c = x W2) and its epilogue, which `F` repeats for a product in pieces.
slicegcn_status_t forward_product(Params& P, FinishArgs& F, const slicegcn_ffn_desc* d, const Plan& q, const Operand& ox, const Operand (&ow)[2], char* ws, bool back,
                                  cudaStream_t st) {
    const bool gated = d->W2 != nullptr, split = q.product.splits > 1;
    const bool promo = q.digits || split;
    P.n = (int)d->n, P.p = q.p, P.slices = split ? q.parts * q.p : q.p, P.cols = q.out_s;
    SGCN_TRY(set_cut(P, q.product, false));
    SGCN_TRY(make_map(&P.a, ox, 128));
    SGCN_TRY(make_map(&P.b0, ow[0], 64));
    SGCN_TRY(make_map(&P.b1, ow[1], 64));
    P.kb_part = (int)ceil_div(q.in_s, 64), P.k_part = q.in_s;
    P.a_planes = q.x_planes, P.b_planes = q.w_planes;
    P.scale = (float)d->scale;
    // a product in pieces has the second projection's columns as slices of their own, which no array of biases has: they are the finishing kernel's
    if (!split) P.b = d->b, P.b2 = d->b2;
    P.bias_vec = q.out_s % 2 == 0 && (uintptr_t)d->b % 8 == 0 && (uintptr_t)d->b2 % 8 == 0;
    if (split) {
        P.partial = reinterpret_cast<float*>(ws + q.partial_at);
        SGCN_TRY((launch_as<kFwd, true, SLICEGCN_ACT_NONE>(P, st)));
        F.partial = P.partial, F.splits = q.product.splits, F.n = P.n, F.p = P.p, F.cols = P.cols, F.gated = gated, F.act = d->act, F.back = back;
        F.scale = P.scale, F.b = d->b, F.b2 = d->b2;
        return launch_after(ffn_finish_kernel, dim3((unsigned)(ceil_div(P.cols, 32) * P.p), (unsigned)ceil_div(P.n, 32)), 256, 0, st, F);
    }
    if (back) {
        P.slices = q.parts * q.p;   // of the sums
        if (gated) return promo ? launch<kDzGated, true>(P, d->act, st) : launch<kDzGated, false>(P, d->act, st);
        return promo ? launch<kDz, true>(P, d->act, st) : launch<kDz, false>(P, d->act, st);
    }
    if (gated) return promo ? launch<kFwdGated, true>(P, d->act, st) : launch<kFwdGated, false>(P, d->act, st);
    return promo ? launch<kFwd, true>(P, d->act, st) : launch<kFwd, false>(P, d->act, st);
}

// `unit` bytes at a time are aligned, in every row and slice.
bool wide_access(const void* p, int64_t ld, int elem, int groups, int width, int unit = 16) {
    return (uintptr_t)p % unit == 0 && ld * elem % unit == 0 && (groups == 1 || width * elem % unit == 0);
}
// Where a product's result goes: by tensor copies, where they can reach it.
slicegcn_status_t set_result(Params& P, FinishArgs& F, void* out, int64_t ld, int elem, int groups, int width, int64_t rows) {
    P.out = F.out = out, P.out_ld = (int)ld, F.out_ld = ld, P.out_bf16 = F.out_bf16 = elem == 2, P.out_vec = wide_access(out, ld, elem, groups, width);
    P.out_pairs = wide_access(out, ld, elem, groups, width, 8);
    P.out_edge = width * elem % 16 ? width / 32 * 32 : width;
    if (!P.out_vec) return SLICEGCN_OK;
    Operand o;
    o.base = out, o.rows = rows, o.ld = ld, o.group_stride = width, o.width = width, o.groups = groups, o.f32 = elem == 4;
    return make_map(&P.o, o, elem == 4 ? 16 : 32, true);
}
void set_input(Params& P, FinishArgs& F, const void* in, int64_t ld, int elem, int groups, int width) {
    P.in = F.in = in, P.in_ld = (int)ld, F.in_ld = ld, P.in_bf16 = F.in_bf16 = elem == 2, P.in_vec = in && wide_access(in, ld, elem, groups, width);
    P.in_pairs = in && wide_access(in, ld, elem, groups, width, 8);
}

template <int R, bool GATED, bool BF16, bool VEC>
slicegcn_status_t launch_rows(const RowsArgs& A, int parts, int slices, cudaStream_t st) {
    const size_t smem = sizeof(float) * ((size_t)R * A.per + 8 * R * (1 + GATED) * kRowsCols);
    static SmemLimit limit;
    SGCN_TRY(limit.set((const void*)ffn_rows_kernel<R, GATED, BF16, VEC>, 4 * (R * 16384 / 8 + 8 * R * (1 + GATED) * kRowsCols)));
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)parts, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(ceil_div(A.out_s, kRowsCols) * parts), (unsigned)slices);
    cfg.blockDim = dim3(kRowsThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    SGCN_CUDA(cudaLaunchKernelEx(&cfg, ffn_rows_kernel<R, GATED, BF16, VEC>, A));
    count_launch();
    return SLICEGCN_OK;
}
template <int R, bool GATED, bool BF16>
slicegcn_status_t launch_rows(const RowsArgs& A, bool vec, int parts, int slices, cudaStream_t st) {
    return vec ? launch_rows<R, GATED, BF16, true>(A, parts, slices, st) : launch_rows<R, GATED, BF16, false>(A, parts, slices, st);
}
template <int R>
slicegcn_status_t launch_rows(const RowsArgs& A, bool bf16, bool vec, int parts, int slices, cudaStream_t st) {
    if (A.W2) return bf16 ? launch_rows<R, true, true>(A, vec, parts, slices, st) : launch_rows<R, true, false>(A, vec, parts, slices, st);
    return bf16 ? launch_rows<R, false, true>(A, vec, parts, slices, st) : launch_rows<R, false, false>(A, vec, parts, slices, st);
}
slicegcn_status_t rows_forward(const slicegcn_ffn_desc* d, const void* x, const void* r, void* out, cudaStream_t st) {
    RowsArgs A = {x, d->x_ld, d->W, d->W2, d->b, d->b2, r, d->r_ld, out, d->out_ld, (int)d->n, d->in_s, d->out_s, d->act, 0, (float)d->scale};
    const int parts = rows_parts(d, &A.per);
    const bool bf16 = d->dtype == SLICEGCN_BF16;
    const bool vec = d->out_s % 4 == 0 && (uintptr_t)d->W % (bf16 ? 8 : 16) == 0 && (uintptr_t)d->W2 % (bf16 ? 8 : 16) == 0;
    if (d->n == 1) return launch_rows<1>(A, bf16, vec, parts, d->num_slices, st);
    if (d->n <= 4) return launch_rows<4>(A, bf16, vec, parts, d->num_slices, st);
    return launch_rows<8>(A, bf16, vec, parts, d->num_slices, st);
}

slicegcn_status_t little_forward(const slicegcn_ffn_desc* d, const void* x, const void* r, void* out, cudaStream_t st) {
    LittleArgs A = {x, d->x_ld, d->W, d->W2, d->b, d->b2, r, d->r_ld, out, d->out_ld, (int)d->n, d->in_s, d->out_s, d->act, 0, (float)d->scale, 0, 0};
    const bool narrow = d->dtype == SLICEGCN_F32 && d->out_s <= 16;
    A.tiles_n = (int)ceil_div(d->out_s, narrow ? 16 : kLittleTile);
    const dim3 grid((unsigned)(A.tiles_n * d->num_slices), (unsigned)ceil_div(d->n, narrow ? 128 : kLittleTile));
    if (d->dtype == SLICEGCN_BF16)
        return d->W2 ? launch_after(ffn_little_kernel<true, true>, grid, 256, 0, st, A) : launch_after(ffn_little_kernel<false, true>, grid, 256, 0, st, A);
    A.x_vec = (uintptr_t)x % 16 == 0 && d->x_ld % 4 == 0 && d->in_s % 4 == 0;
    A.w_vec = (uintptr_t)d->W % 16 == 0 && (uintptr_t)d->W2 % 16 == 0 && d->out_s % 4 == 0;
    if (narrow)
        return d->W2 ? launch_after(ffn_little_f32_kernel<true, 16>, grid, 256, 0, st, A) : launch_after(ffn_little_f32_kernel<false, 16>, grid, 256, 0, st, A);
    return d->W2 ? launch_after(ffn_little_f32_kernel<true, 64>, grid, 256, 0, st, A) : launch_after(ffn_little_f32_kernel<false, 64>, grid, 256, 0, st, A);
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
    if (q.rows) return rows_forward(d, x, r, out, st);
    if (q.little) return little_forward(d, x, r, out, st);
    char* ws = static_cast<char*>(workspace);
    Operand ox, ow[2];
    PackArgs packs = {};
    operands(d, q, x, ws, ox, ow, packs);
    SGCN_TRY(run_packs(packs, st));
    Params P = {};
    FinishArgs F = {};
    P.status = status;
    set_input(P, F, r, d->r_ld, e, q.p, q.out_s);
    SGCN_TRY(set_result(P, F, out, d->out_ld, e, q.p, q.out_s, d->n));
    return forward_product(P, F, d, q, ox, ow, ws, false, st);
}

slicegcn_status_t slicegcn_ffn_backward(const slicegcn_ffn_desc* d, const void* x, const void* dout, void* dx, void* dW, void* dW2, float* db,
                                        float* db2, int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
    SGCN_TRY(check(d));
    const int ge = d->grad_dtype == SLICEGCN_F32 ? 4 : 2;
    const int64_t n = d->n, ins = (int64_t)d->num_slices * d->in_s, outs = (int64_t)d->num_slices * d->out_s;
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
    const int p = q.p;
    char* ws = static_cast<char*>(workspace);
    Operand ox, ow[2], oz;
    PackArgs packs = {};
    operands(d, q, x, ws, ox, ow, packs);
    if (q.pack_g)
        add_pack(packs, dout, d->dout_ld, n, p, q.out_s, ge == 2, ws + q.z_at, oz);
    else if (!q.dz)
        oz.base = dout, oz.rows = n, oz.ld = d->dout_ld, oz.group_stride = q.out_s, oz.width = q.out_s, oz.groups = p;
    SGCN_TRY(run_packs(packs, st));
    const bool sums = db || db2;
    const float scale = q.dz ? 1.f : (float)d->scale;   // what the products still have to be multiplied by
    if (q.dz) {
        Params P = {};
        FinishArgs F = {};
        P.status = status;
        set_input(P, F, dout, d->dout_ld, ge, p, q.out_s);
        P.sums = F.sums = sums ? reinterpret_cast<float*>(ws + q.sums_at) : nullptr;
        oz.base = ws + q.z_at, oz.rows = n, oz.ld = (int64_t)q.parts * p * q.out_pad, oz.group_stride = q.out_pad, oz.plane_stride = n * oz.ld;
        oz.width = q.out_s, oz.groups = q.parts * p, oz.planes = q.z_planes;
        F.dz = reinterpret_cast<__nv_bfloat16*>(ws + q.z_at);
        F.dz_plane = oz.plane_stride, F.dz_row = (int)oz.ld, F.dz_pad = q.out_pad, F.dz_planes = q.z_planes;
        P.planes = q.z_planes;
        SGCN_TRY(make_map(&P.o, oz, q.digits ? 16 : 32, true));
        SGCN_TRY(forward_product(P, F, d, q, ox, ow, ws, true, st));
    }
    if (dx) {
        Params P = {};
        FinishArgs F = {};
        P.status = status;
        P.n = (int)n, P.p = P.slices = p, P.cols = q.in_s;
        SGCN_TRY(set_cut(P, q.dx, false));
        SGCN_TRY(make_map(&P.a, oz, 128));
        SGCN_TRY(make_map(&P.b0, ow[0], P.nt));
        SGCN_TRY(make_map(&P.b1, ow[1], P.nt));
        P.kb_part = (int)ceil_div(q.out_s, 64), P.k_part = q.out_s;
        P.a_planes = q.z_planes, P.b_planes = q.w_planes;
        P.scale = scale;
        SGCN_TRY(set_result(P, F, dx, d->dx_ld, ge, p, q.in_s, n));
        const bool split = P.splits > 1;
        if (split) P.partial = reinterpret_cast<float*>(ws + q.partial_at);
        SGCN_TRY((P.a_planes > 1 || split ? launch_as<kDx, true, SLICEGCN_ACT_NONE>(P, st) : launch_as<kDx, false, SLICEGCN_ACT_NONE>(P, st)));
        if (split) {
            F.partial = P.partial, F.splits = P.splits, F.n = P.n, F.p = p, F.cols = P.cols, F.act = SLICEGCN_ACT_NONE, F.scale = scale;
            SGCN_TRY(launch_after(ffn_finish_kernel, dim3((unsigned)(ceil_div(P.cols, 32) * p), (unsigned)ceil_div(n, 32)), 256, 0, st, F));
        }
    }
    JoinArgs J = {};
    if (dW || dW2) {
        Params P = {};
        P.status = status;
        P.swapped = q.dw.swapped, P.pair = q.dw.pair, P.matrices = q.parts * p;
        P.n = P.swapped ? q.in_s : q.out_s, P.p = p, P.slices = P.pair ? p : q.parts * p, P.cols = q.out_s, P.k_part = q.in_s;
        SGCN_TRY(set_cut(P, q.dw, true));
        P.kb_part = P.kb_total;
        SGCN_TRY(make_map(&P.a, P.swapped ? ox : oz, 64));
        SGCN_TRY(make_map(&P.b0, P.swapped ? oz : ox, 64));
        P.b1 = P.b0;
        P.a_planes = P.swapped ? q.x_planes : q.z_planes, P.b_planes = P.swapped ? q.z_planes : q.x_planes;
        P.scale = scale, P.out_bf16 = ge == 2;
        const bool join = P.splits > 1 || q.merge > 1;
        if (join) P.partial = reinterpret_cast<float*>(ws + q.partial_at);
        P.dw = dW, P.dw2 = dW2;
        SGCN_TRY((launch_as<kDw, true, SLICEGCN_ACT_NONE>(P, st)));
        if (join) {
            const int64_t each = d->in_s * outs, total = q.parts * each;
            J.job[0] = {P.partial, P.splits, ge == 2, total, each, total * q.merge, scale, {dW, dW2}, q.merge, d->in_s, d->out_s,
                        (int)std::min<int64_t>(ceil_div(total, 256), 148 * 8)};
        }
    }
    if (sums && q.dz && q.sum_rows <= kJoinRows) {
        const int64_t cols = q.parts * outs;
        J.job[1] = {reinterpret_cast<const float*>(ws + q.sums_at), (int)q.sum_rows, 0, cols, outs, cols, scale, {db, db2}, 1, 1, 1, (int)ceil_div(cols, 256)};
    } else if (sums) {
        SumArgs A;
        A.src = q.dz ? (const void*)(ws + q.sums_at) : dout;
        A.rows = q.sum_rows;
        A.cols = (int)(q.parts * outs);
        A.ld = q.dz ? A.cols : d->dout_ld;
        A.bf16 = !q.dz && ge == 2;
        const int width = A.bf16 ? 8 : 4;
        A.vec = (uintptr_t)A.src % 16 == 0 && A.ld % width == 0 && A.cols % width == 0;
        A.per = ceil_div(A.rows, q.sum_chunks);
        A.partial = reinterpret_cast<float*>(ws + q.chunks_at);
        const dim3 grid((unsigned)ceil_div(A.cols, 32 * (A.vec ? width : 1)), (unsigned)q.sum_chunks);
        if (A.bf16)
            SGCN_TRY((A.vec ? launch_after(ffn_colsum_kernel<true, true>, grid, 256, 0, st, A) : launch_after(ffn_colsum_kernel<true, false>, grid, 256, 0, st, A)));
        else
            SGCN_TRY((A.vec ? launch_after(ffn_colsum_kernel<false, true>, grid, 256, 0, st, A) : launch_after(ffn_colsum_kernel<false, false>, grid, 256, 0, st, A)));
        J.job[1] = {A.partial, q.sum_chunks, 0, A.cols, outs, A.cols, scale, {db, db2}, 1, 1, 1, (int)ceil_div(A.cols, 256)};
    }
    if (J.job[0].ctas + J.job[1].ctas > 0) SGCN_TRY(launch_after(ffn_join_kernel, dim3(J.job[0].ctas + J.job[1].ctas), 256, 0, st, J));
    return SLICEGCN_OK;
}

}  // extern "C"
