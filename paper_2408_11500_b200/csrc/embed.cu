// Embedding lookup with scaling, and its gradient by sorted ids.
//   forward   out[i, :] = scale * table[ids[i], :]            (ids[i] = -1: a row of zeros)
//   gradient  dtable[v, :] = sum over {i : ids[i] = v} of scale * dout[i, :]
// The gradient sorts the ids (stable least-significant-digit radix sort), so the positions of one id lie next to each
// other in their own order and every row of dtable is one sum in a fixed order: no floating-point atomics.
#include <algorithm>
#include <type_traits>

#include "common.cuh"

namespace sgcn {
namespace {

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 8;       // positions a lane loads ahead
constexpr int kMaxDigitBits = 9;    // 512 digits: one pass less for 17 and 18 key bits, 64 KB of counters per CTA
constexpr int kSMs = 148;

// ---- lookup -----------------------------------------------------------------------------------
// Four columns of a row: neighbouring ones (VEC) or ones `step` apart.  Loads are unconditional (a column past the end reads
// the row's first one), so that a thread can have several rows on their way.
template <typename T, bool VEC>
struct RowPart;
template <>
struct RowPart<float, true> {
    float4 v;
    __device__ __forceinline__ void load(const float* row, int col, int, int) { v = __ldg(reinterpret_cast<const float4*>(row + col)); }
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w; }
};
template <>
struct RowPart<__nv_bfloat16, true> {
    uint2 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* row, int col, int, int) { v = __ldg(reinterpret_cast<const uint2*>(row + col)); }
    __device__ __forceinline__ void get(float (&f)[4]) const {
        f[0] = __uint_as_float(v.x << 16), f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16), f[3] = __uint_as_float(v.y & 0xffff0000u);
    }
};
template <typename T>
struct RowPart<T, false> {
    T v[4];
    __device__ __forceinline__ void load(const T* row, int col, int step, int width) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = row[col + j * step < width ? col + j * step : 0];
    }
    __device__ __forceinline__ void get(float (&f)[4]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = (float)v[j];
    }
};
template <bool VEC>
__device__ __forceinline__ void put4(float* row, int col, int step, int width, const float (&f)[4]) {
    if (VEC) {
        __stcs(reinterpret_cast<float4*>(row + col), make_float4(f[0], f[1], f[2], f[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j * step < width) row[col + j * step] = f[j];
    }
}
template <bool VEC>
__device__ __forceinline__ void put4(__nv_bfloat16* row, int col, int step, int width, const float (&f)[4]) {
    if (VEC) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(f[0], f[1]), hi = __floats2bfloat162_rn(f[2], f[3]);
        __stcs(reinterpret_cast<uint2*>(row + col), make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi)));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j * step < width) row[col + j * step] = __float2bfloat16_rn(f[j]);
    }
}

// L lanes per row and 128 columns (blockIdx.y); a warp takes ROWS rows per lane group, all of them on their way before the
// first is stored.  A table that the L2 holds answers soon, and more warps with fewer rows each do better; rows that come
// from HBM in random order want more on their way than the registers of many warps allow.  Measured, 4 / 8 / 16 rows:
// 20.5 / 22.3 / 22.5 us for 169,343 rows of a 20 MB table, 329 / 340 / 290 us for 2,449,029 rows of a 980 MB table.
// Bound by HBM: a 400-byte row in random order costs 7 of its 64-byte granules wherever it starts, 12 % more than its bytes.
// Rows that allow no accesses of four columns go element by element: 2 to 4 times their bytes' time (681,284 x 174 fp32: 365 us
// of 145, 2,449,029 x 9: 87 of 28).
constexpr int kRowsFromL2 = 4, kRowsFromHbm = 16;
constexpr int64_t kTableInL2 = 64ll << 20;   // bytes; half of the L2, the rest is for what is written
template <typename TT, typename TO, int L, bool VEC, int ROWS>
__global__ void __launch_bounds__(256) embed_forward_kernel(int64_t n, int64_t vocab, int width, const int32_t* ids, const TT* table,
                                                            int64_t table_ld, TO* out, int64_t out_ld, float scale, int32_t* status) {
    constexpr int G = 32 / L;   // lane groups
    const int lane = threadIdx.x & 31, l = lane & (L - 1), g = lane / L;
    const int64_t first = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * (G * ROWS);
    if (first >= n) return;
    const int col = blockIdx.y * 4 * L + (VEC ? 4 * l : l);
    const bool live_col = col < width;
    int32_t id[ROWS];
    RowPart<TT, VEC> part[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int64_t i = first + k * G + g;
        id[k] = i < n ? ids[i] : -1;
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const bool known = (uint32_t)id[k] < (uint32_t)vocab;
        if (!known && id[k] != -1 && status) atomicOr(status, SLICEGCN_DEVSTATUS_BAD_ID);
        part[k].load(table + (int64_t)(known ? id[k] : 0) * table_ld, live_col ? col : 0, L, width);
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int64_t i = first + k * G + g;
        float f[4];
        part[k].get(f);
        const bool known = (uint32_t)id[k] < (uint32_t)vocab;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = known ? f[j] * scale : 0.f;
        if (i < n && live_col) put4<VEC>(out + i * out_ld, col, L, width, f);
    }
}

// ---- rows of ids that do not occur ------------------------------------------------------------
// They are cleared 32 at a time by a warp.  Rows that follow one another without a gap go in aligned 16-byte pieces, whatever their
// width (8 ids of 1,900,000 x 131: 426 us element by element, 156 us so); rows that lie apart one by one.
struct RowClear {
    float* table;
    int64_t ld;
    int width, lane;
    bool pieces;                      // rows of four columns and more, without gaps: a piece lies in two of them at most
    int lead;                         // elements before a block's first piece: the same for all blocks, which lie 128 width bytes apart
    int row, col, row_step, col_step; // where the lane's first piece starts in a block, and how far its next one is
    // blocks start `row0` and multiples of 32 rows from there on
    __device__ __forceinline__ RowClear(float* t, int64_t ld_, int width_, int64_t row0)
        : table(t), ld(ld_), width(width_), lane(threadIdx.x & 31), pieces(ld_ == width_ && width_ >= 4) {
        lead = (int)(-(int64_t)((uintptr_t)(t + row0 * ld_) >> 2) & 3);
        const int e = lead + 4 * lane;
        row = e / width, col = e - row * width;
        row_step = 128 / width, col_step = 128 - row_step * width;
    }
    // rows v .. v + rows - 1 (32 at most), those whose bit is set
    __device__ __forceinline__ void block(int64_t v, int rows, uint32_t absent) const {
        if (!absent) return;
        float* const from = table + v * ld;
        if (pieces) {
            const int count = rows * width, whole = (count - lead) / 4, loose = count - 4 * whole;   // lead <= 3 < width
            if (lane < loose) {
                const int e = lane < lead ? lane : 4 * whole + lane;
                if (absent >> (e < width ? 0 : rows - 1) & 1u) from[e] = 0.f;   // of the first row or the last
            }
            const bool all = absent == 0xffffffffu >> (32 - rows);
            int r = row, c = col;
            for (int k = lane; k < whole; k += 32) {
                float* const to = from + lead + 4 * k;
                const bool here = all || absent >> r & 1u, next = c + 4 > width ? all || absent >> (r + 1) & 1u : here;
                if (here && next) {
                    *reinterpret_cast<float4*>(to) = make_float4(0.f, 0.f, 0.f, 0.f);
                } else if (here || next) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (c + j < width ? here : next) to[j] = 0.f;
                }
                r += row_step, c += col_step;
                if (c >= width) c -= width, ++r;
            }
            return;
        }
        const bool fours = width % 4 == 0 && ld % 4 == 0 && (uintptr_t)table % 16 == 0;
        const int per = fours ? 4 : 1;
        int group = 1;
        while (group < 32 && group * per < width) group *= 2;
        for (int r = lane / group; r < rows; r += 32 / group) {
            if (!(absent >> r & 1u)) continue;
            for (int c = (lane & (group - 1)) * per; c < width; c += group * per) {
                if (fours)
                    *reinterpret_cast<float4*>(from + r * ld + c) = make_float4(0.f, 0.f, 0.f, 0.f);
                else
                    from[r * ld + c] = 0.f;
            }
        }
    }
};
// The whole table, by CTAs that stand beside those of the sort's launches (below): a share of the rows per launch.
struct ClearShare {
    float* table;
    int64_t ld;
    int width;
    int64_t rows, row0, rows_per_cta;   // of the table; first of this launch; of a CTA (a multiple of 32)
};
__device__ __forceinline__ void clear_share(const ClearShare& c, int cta) {
    const int64_t r0 = c.row0 + cta * c.rows_per_cta, r1 = min(c.rows, r0 + c.rows_per_cta);
    if (r0 >= r1) return;
    if (c.ld == c.width) {   // a span
        float* const from = c.table + r0 * c.width;
        const int64_t count = (r1 - r0) * c.width, lead = min(count, -(int64_t)((uintptr_t)from >> 2) & 3), whole = (count - lead) / 4;
        for (int64_t k = threadIdx.x; k < whole; k += blockDim.x)
            *reinterpret_cast<float4*>(from + lead + 4 * k) = make_float4(0.f, 0.f, 0.f, 0.f);
        if (threadIdx.x < lead) from[threadIdx.x] = 0.f;
        if (lead + 4 * whole + threadIdx.x < count) from[lead + 4 * whole + threadIdx.x] = 0.f;
        return;
    }
    const RowClear rows(c.table, c.ld, c.width, r0);
    for (int64_t v = r0 + threadIdx.x / 32 * 32; v < r1; v += blockDim.x) {
        const int n = (int)min((int64_t)32, r1 - v);
        rows.block(v, n, 0xffffffffu >> (32 - n));
    }
}

// ---- stable sort of the ids -------------------------------------------------------------------
// Keys run from 0 to `vocab`: the id, or `vocab` (sorted last) for positions that take no part.  Per digit two launches:
// sort_count_kernel counts every tile's digits, sort_scatter_kernel turns the counts into offsets (each CTA reads the whole
// table of tiles x digits, a few hundred KB that stay in L2, so no scan launch stands between the two) and moves the pairs.
// lanes that are live and hold the same digit of at most BITS bits
template <int BITS>
__device__ __forceinline__ uint32_t same_digit(uint32_t d, bool live) {
    uint32_t peers = __ballot_sync(0xffffffffu, live);
#pragma unroll
    for (int k = 0; k < BITS; ++k) {
        const bool set = (d >> k) & 1u;
        const uint32_t with = __ballot_sync(0xffffffffu, set);
        peers &= set ? with : ~with;
    }
    return peers;
}

struct SortArgs {
    int32_t n;
    int64_t vocab;
    const int32_t* ids;      // read by the first digit's pass
    const uint2* in;         // (key, position), read by the others
    uint2* out;
    uint32_t* counts;        // [tiles][bins]
    uint8_t* present;        // [vocab] cleared by the first count, see SumArgs; NULL: not wanted
    ClearShare clear;        // for the CTAs past the tiles
    int32_t* status;
    int shift, bits, tiles;
    int32_t tile;            // positions per tile, a multiple of kSortWarps * 32
};

template <bool FIRST>
__device__ __forceinline__ uint2 sort_load(const SortArgs& a, int32_t i) {
    if (FIRST) return make_uint2(min((uint32_t)a.ids[i], (uint32_t)a.vocab), (uint32_t)i);   // a negative id is a large number
    return a.in[i];
}

template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortArgs a) {
    __shared__ uint32_t hist[1 << kMaxDigitBits];
    if ((int)blockIdx.x >= a.tiles) {
        cudaTriggerProgrammaticLaunchCompletion();
        if (!FIRST) cudaGridDependencySynchronize();
        clear_share(a.clear, blockIdx.x - a.tiles);
        return;
    }
    if (FIRST && a.present)
        for (int64_t i = (blockIdx.x * (int64_t)kSortThreads + threadIdx.x) * 16; i < a.vocab; i += (int64_t)a.tiles * kSortThreads * 16)
            *reinterpret_cast<uint4*>(a.present + i) = make_uint4(0, 0, 0, 0);   // (rounded up to 16 bytes)
    if (threadIdx.x < 1 << kMaxDigitBits) hist[threadIdx.x] = 0;
    __syncthreads();
    cudaTriggerProgrammaticLaunchCompletion();
    if (!FIRST) cudaGridDependencySynchronize();
    const uint32_t mask = (1u << a.bits) - 1u;
    const int64_t i0 = (int64_t)blockIdx.x * a.tile, i1 = min((int64_t)a.n, i0 + a.tile);
#pragma unroll 8
    for (int64_t i = i0 + threadIdx.x; i < i1; i += kSortThreads) {
        const uint32_t key = sort_load<FIRST>(a, (int32_t)i).x;
        if (FIRST && key == (uint32_t)a.vocab && a.status && a.ids[i] != -1) atomicOr(a.status, SLICEGCN_DEVSTATUS_BAD_ID);
        atomicAdd(&hist[(key >> a.shift) & mask], 1u);
    }
    __syncthreads();
    if (threadIdx.x <= mask) a.counts[((int64_t)blockIdx.x << a.bits) + threadIdx.x] = hist[threadIdx.x];
}

// Each warp owns a contiguous run of the tile and walks it 32 positions at a time; lanes with the same digit are ranked by
// ballots, so the order of equal digits is kept.
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(const SortArgs a) {
    extern __shared__ uint32_t next[];   // [kSortWarps][bins] counts of each warp's run, then where its next pair goes
    __shared__ uint4 part_before[kSortThreads], part_total[kSortThreads];   // [part][bins / 4]
    __shared__ uint32_t warp_total[kSortWarps];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    if ((int)blockIdx.x >= a.tiles) {
        cudaTriggerProgrammaticLaunchCompletion();
        cudaGridDependencySynchronize();
        clear_share(a.clear, blockIdx.x - a.tiles);
        return;
    }
    const int bins = 1 << a.bits;
    const uint32_t mask = (uint32_t)bins - 1u;
    uint32_t* mine = next + w * bins;
    for (int k = lane; k < bins; k += 32) mine[k] = 0;
    __syncwarp();
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    const int64_t i0 = min((int64_t)a.n, (int64_t)blockIdx.x * a.tile + (int64_t)w * (a.tile / kSortWarps));
    const int64_t i1 = min((int64_t)a.n, i0 + a.tile / kSortWarps);
    uint2 item[kSortItems];
    for (int64_t b = i0; b < i1; b += 32 * kSortItems) {
#pragma unroll
        for (int j = 0; j < kSortItems; ++j)
            if (b + 32 * j + lane < i1) item[j] = sort_load<FIRST>(a, (int32_t)(b + 32 * j + lane));
#pragma unroll
        for (int j = 0; j < kSortItems; ++j)
            if (b + 32 * j + lane < i1) atomicAdd(&mine[(item[j].x >> a.shift) & mask], 1u);
    }
    const int quads = bins / 4, parts = kSortThreads / quads;
    {   // tiles before this one, and all tiles, per digit: thread t takes four digits and every parts-th tile
        const int quad = tid & (quads - 1), part = tid / quads;
        const uint4* counts = reinterpret_cast<const uint4*>(a.counts) + quad;
        uint4 before = make_uint4(0, 0, 0, 0), total = before;
#pragma unroll 8
        for (int t = part; t < a.tiles; t += parts) {
            const uint4 c = counts[(int64_t)t * quads];
            const uint32_t m = t < (int)blockIdx.x ? 0xffffffffu : 0u;
            total.x += c.x, total.y += c.y, total.z += c.z, total.w += c.w;
            before.x += c.x & m, before.y += c.y & m, before.z += c.z & m, before.w += c.w & m;
        }
        part_before[tid] = before;
        part_total[tid] = total;
    }
    __syncthreads();
    uint32_t at = 0, total = 0;
    if (tid < bins)
#pragma unroll 8
        for (int q = 0; q < parts; ++q) {
            at += reinterpret_cast<const uint32_t*>(part_before)[q * bins + tid];
            total += reinterpret_cast<const uint32_t*>(part_total)[q * bins + tid];
        }
    uint32_t incl = total;
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
    }
    if (lane == 31) warp_total[w] = incl;
    __syncthreads();
    if (tid < bins) {
        at += incl - total;
        for (int k = 0; k < w; ++k) at += warp_total[k];
        uint32_t c[kSortWarps];
#pragma unroll
        for (int k = 0; k < kSortWarps; ++k) c[k] = next[k * bins + tid];
#pragma unroll
        for (int k = 0; k < kSortWarps; ++k) {
            next[k * bins + tid] = at;
            at += c[k];
        }
    }
    __syncthreads();
    const bool whole = i1 - i0 <= 32 * kSortItems;   // the run still sits in registers
    for (int64_t b = i0; b < i1; b += 32 * kSortItems) {
        if (!whole)
#pragma unroll
            for (int j = 0; j < kSortItems; ++j)
                if (b + 32 * j + lane < i1) item[j] = sort_load<FIRST>(a, (int32_t)(b + 32 * j + lane));
#pragma unroll
        for (int j = 0; j < kSortItems; ++j) {
            if (b + 32 * j >= i1) break;
            const bool live = b + 32 * j + lane < i1;
            const uint32_t d = (item[j].x >> a.shift) & mask;
            const uint32_t peers = same_digit<kMaxDigitBits>(d, live);
            const uint32_t rank = __popc(peers & ((1u << lane) - 1u));
            uint32_t to = 0;
            if (live) to = mine[d] + rank;
            __syncwarp();
            if (live && rank == 0) mine[d] += __popc(peers);
            __syncwarp();
            if (live) a.out[to] = item[j];
        }
    }
}

// ---- sums over the sorted positions -----------------------------------------------------------
// A unit of L lanes takes R consecutive sorted positions and up to 4 L columns, gathers the rows of dout and adds them up
// in registers.  An id whose positions lie inside the unit is finished there.  The sum of an id that reaches over the
// unit's edges is left in shared memory; the CTA joins its units' sums in order, and what reaches over the CTA's edges goes
// to the workspace, where embed_finish_kernel joins it, again in order.  Work is split by positions, so an id that holds
// half of them costs no more than others.
constexpr int kSumThreads = 256;
constexpr int kSumPerSM = 4;   // CTAs per SM (41 KB of shared memory each; a fifth one fits and makes it 4 % slower)
constexpr int kAhead = 8;      // rows of dout on their way per unit

struct SumArgs {
    int32_t n;
    int64_t vocab;
    int width, accumulate;
    const uint2* pairs;
    const float* dout;
    int64_t dout_ld;
    float* dtable;
    int64_t dtable_ld;
    float scale;
    uint8_t* present;        // [vocab] set where an id occurs: once per run and unit, as setting it per position would
                             // queue the positions of a frequent id up on one byte (200 us for 2.4 M positions); NULL: not wanted
    int32_t per_unit;        // R
    int sum_ctas;
    float* head;             // [sum_ctas][width] sum of the id that comes in from the CTA before
    float* tail;             // [sum_ctas][width] sum of the id that starts here and goes on in the next one
    int4* info;              // [sum_ctas] {head present, head ends here, tail present, tail's id}
};

// Asynchronous copies to shared memory.
__device__ __forceinline__ void copy_async16(uint32_t to, const float* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async16_if(bool wanted, uint32_t to, const float* from) {
    asm volatile("{.reg .pred p; setp.ne.u32 p, %2, 0; @p cp.async.cg.shared.global [%0], [%1], 16;}" ::"r"(to), "l"(from),
                 "r"((uint32_t)wanted)
                 : "memory");
}
__device__ __forceinline__ void copy_async4(uint32_t to, const float* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
template <bool VEC>
__device__ __forceinline__ void store4(float* row, int col, int stride, int width, int accumulate, const float (&v)[4]) {
    if (VEC) {
        float4 t = make_float4(v[0], v[1], v[2], v[3]);
        if (accumulate) {
            const float4 o = *reinterpret_cast<const float4*>(row + col);
            t.x += o.x, t.y += o.y, t.z += o.z, t.w += o.w;
        }
        *reinterpret_cast<float4*>(row + col) = t;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j * stride < width) row[col + j * stride] = v[j] + (accumulate ? row[col + j * stride] : 0.f);
    }
}

constexpr int kJoin = 4;   // units that one thread joins per column: all threads of the CTA share the first half of the joining

// The rows on their way: ROWS per unit, which are also the positions of a batch.  Every thread copies and reads back its own four
// columns, so its own count of finished copies is all the waiting there is; but narrow rows that allow no accesses of 16 bytes
// (SHARED) are copied as the aligned 16 bytes that hold them, one piece more than there are lanes, and read by all lanes of the
// unit: element by element the copies alone paced the kernel (2,449,029 x 11, an id each: 281 and 226 us).  Wide ones go element
// by element: a copy is then 64 to 128 bytes long, and finding the row in its pieces costs more (600,000 x 131: 169 and 237 us).
template <int L, bool VEC>
struct RowRing {
    static constexpr bool SHARED = !VEC && L <= 8;
    static constexpr int ROWS = !SHARED ? kAhead : L == 8 ? 7 : 4;
    float4 at[ROWS][kSumThreads / L][SHARED ? L + 1 : L];   // 32 KB at most
};
// Shared memory of a CTA that sums, beside them.
template <int L>
struct SumShared {
    static constexpr int U = kSumThreads / L;
    float sums[U][2][4 * L];
    int4 unit_info[U];            // {head present, head ends here, tail's id or -1, unused}
    int4 part_info[U / kJoin];    // the same for kJoin units each
};
// The sorted positions: in memory, or (small problems) in the CTA's own shared memory as 13 bits of position under the
// id's distance from the CTA's first one.
struct PairsInMemory {
    const uint2* p;
    __device__ __forceinline__ uint2 operator()(uint32_t i) const { return p[i]; }
};
constexpr int kSmallBits = 13, kSmallN = 1 << kSmallBits;
struct PairsInShared {
    const uint32_t* p;
    uint32_t first_id, step;   // the ids of a CTA
    __device__ __forceinline__ uint2 operator()(uint32_t i) const {
        return make_uint2((p[i] >> kSmallBits) * step + first_id, p[i] & (kSmallN - 1));
    }
};

// The sums of N units (the info and the sums of every stride-th) in one column, joined in order: ids that end inside go to the table.
struct Joined {
    float head, tail;
    bool any_head, ended;
    int id;   // of the tail, or -1
};
template <int N, int W>
__device__ __forceinline__ Joined join_units(const SumArgs& a, const int4* info, const float (*sums)[2][W], int stride, int c, int table_col) {
    auto write = [&](int to, float v) {
        float* t = a.dtable + (int64_t)to * a.dtable_ld + table_col;
        *t = v + (a.accumulate ? *t : 0.f);
    };
    Joined r{0.f, 0.f, false, false, -1};
    float sum = 0.f;
    bool open = false, started = false;
    int id = -1;
    constexpr int M = N < 4 ? N : 4;   // four on their way at a time
#pragma unroll 1
    for (int k0 = 0; k0 < N; k0 += M) {
        int4 f[M];
        float hs[M], ts[M];
#pragma unroll
        for (int k = 0; k < M; ++k) f[k] = info[k0 + k], hs[k] = sums[(k0 + k) * stride][0][c], ts[k] = sums[(k0 + k) * stride][1][c];
#pragma unroll
        for (int k = 0; k < M; ++k) {
            if (f[k].x) {
                if (!open) open = true, started = false, sum = 0.f, r.any_head = true;
                sum += hs[k];
                if (f[k].y) {
                    if (started)
                        write(id, sum);
                    else
                        r.head = sum, r.ended = true;
                    open = false;
                }
            }
            if (f[k].z >= 0) open = true, started = true, sum = ts[k], id = f[k].z;
        }
    }
    if (open && started) r.tail = sum, r.id = id;
    if (open && !started) r.head = sum;
    return r;
}

// One CTA's share: positions cta * U * per_unit and on, of n.  ONE: the CTA holds all positions of its ids.
// VEC: lane l holds columns 4 l .. 4 l + 3 of the tile (16-byte accesses); else columns l, l + L, l + 2 L, l + 3 L
template <int L, bool VEC, bool ONE, typename Pairs>
__device__ __forceinline__ void sum_sorted(const SumArgs& a, const Pairs pairs, int n, int per_unit, int cta, SumShared<L>& sh, RowRing<L, VEC>& ring) {
    constexpr int U = SumShared<L>::U, A = RowRing<L, VEC>::ROWS;
    constexpr bool SHARED = RowRing<L, VEC>::SHARED;
    const int tid = threadIdx.x, l = tid & (L - 1), unit = tid / L;
    const int c0 = blockIdx.y * 4 * L;
    const int col = c0 + (VEC ? 4 * l : l);
    const bool live_col = col < a.width;
    const int64_t s64 = ((int64_t)cta * U + unit) * per_unit;
    // unsigned: what is asked for ahead of the last of 2^31 - 1 positions lies past 31 bits
    const uint32_t s = (uint32_t)min((int64_t)n, s64), e = (uint32_t)min((int64_t)n, s64 + per_unit);
    const uint32_t none = (uint32_t)a.vocab;
    const uint32_t before = s > 0 && s < e ? pairs(s - 1).x : 0xffffffffu;
    const uint32_t my_ring = (uint32_t)__cvta_generic_to_shared(&ring.at[0][unit][SHARED ? 0 : l]);
    const int count = min(4 * L, a.width - c0);   // columns of the tile
    uint32_t offs = 0;                            // where the rows on their way start in their first 16 bytes, two bits each
    uint32_t key = 0xffffffffu;
    bool first = true;             // still in the unit's first run
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    bool head = false, head_ends = false;
    int tail_id = -1;
    auto put = [&](int which) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sh.sums[unit][which][VEC ? 4 * l + j : l + j * L] = acc[j];
    };
    auto finish = [&](bool goes_on) {   // the run of `key` ends, or the unit does
        if (key >= none) return;
        if (first && key == before) {
            head = true, head_ends = !goes_on;
            put(0);
            return;
        }
        if (!ONE && a.present && l == 0 && blockIdx.y == 0) a.present[key] = 1;
        if (goes_on) {
            tail_id = (int)key;
            put(1);
        } else if (live_col) {
            store4<VEC>(a.dtable + (int64_t)key * a.dtable_ld, col, L, a.width, a.accumulate, acc);
        }
    };
    constexpr int Q = L < A ? A / L : 1;   // positions of a batch that a lane holds
    struct Batch {
        uint2 p[Q];
    };
    auto batch = [&](uint32_t b) {
        Batch t;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            t.p[q] = l < A && b + q * L + l < e ? pairs(b + q * L + l) : make_uint2(none, 0);
            if (t.p[q].x >= none) t.p[q].y = 0xffffffffu;
        }
        return t;
    };
    auto request = [&](int i, const Batch& t) {   // row i of a batch into slot i
        const uint32_t pos = __shfl_sync(0xffffffffu, t.p[i / L].y, i % L, L);
        const uint32_t slot = my_ring + i * (int)sizeof(ring.at[0]);
        const float* row = a.dout + (int64_t)pos * a.dout_ld + c0;
        if constexpr (SHARED) {
            const int off = (int)((uintptr_t)row >> 2 & 3), pieces = pos != 0xffffffffu ? (off + count + 3) / 4 : 0;
            offs = offs & ~(3u << 2 * i) | (uint32_t)off << 2 * i;
            if (pos - 3u < (uint32_t)a.n - 6u && a.n > 6 || pos == 0xffffffffu) {
                copy_async16_if(l < pieces, slot + 16 * l, row - off + 4 * l);
                copy_async16_if(l + L < pieces, slot + 16 * (l + L), row - off + 4 * (l + L));
            } else {   // beside the first and the last rows there need not be anything
                for (int q = l; q < count; q += L) copy_async4(slot + 4 * (off + q), row + q);
            }
        } else if (live_col && pos != 0xffffffffu) {
            if constexpr (VEC) {
                copy_async16(slot, row + 4 * l);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (l + j * L < count) copy_async4(slot + 4 * j, row + l + j * L);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    Batch cur = batch(s), next = batch(s + A);
    // a shared slot is filled again two steps after it was read: a barrier of the warp lies between
    constexpr int AHEAD = SHARED ? A - 2 : A - 1;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) request(i, cur);
    // All units of a warp go as many rounds, whether or not theirs is a short one: shuffles of a part of the warp take an instruction
    // each to keep its lanes in step, and its unit was three quarters busy with units of two lanes.
    const int rounds = (per_unit + A - 1) / A;
    uint32_t b = s;
    for (int r = 0; r < rounds; ++r, b += A) {
        const Batch later = batch(b + 2 * A);
        // row i of the batch is waited for; the one AHEAD of it, of this batch or the next, is asked for
        auto arrive = [&](int i) {
            if (i + AHEAD < A)
                request(i + AHEAD, cur);
            else
                request(i + AHEAD - A, next);
            asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
            if (SHARED) __syncwarp();
        };
        auto add = [&](int i) {
            if constexpr (SHARED) {
                const float* row = reinterpret_cast<const float*>(ring.at[i][unit]) + (offs >> 2 * i & 3);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (l + j * L < count) acc[j] = fmaf(a.scale, row[l + j * L], acc[j]);
            } else {
                const float4 v = ring.at[i][unit][l];
                acc[0] = fmaf(a.scale, v.x, acc[0]);
                if (VEC || l + L < count) acc[1] = fmaf(a.scale, v.y, acc[1]);
                if (VEC || l + 2 * L < count) acc[2] = fmaf(a.scale, v.z, acc[2]);
                if (VEC || l + 3 * L < count) acc[3] = fmaf(a.scale, v.w, acc[3]);
            }
        };
        bool going_on = b + A <= e && key < none;   // the whole batch belongs to the run (frequent ids): no row needs a look at its id
#pragma unroll
        for (int q = 0; q < Q; ++q) going_on = going_on && (l >= A || cur.p[q].x == key);
        if (__all_sync(0xffffffffu, going_on)) {
#pragma unroll
            for (int i = 0; i < A; ++i) {
                arrive(i);
                if (live_col) add(i);
            }
        } else {
#pragma unroll
            for (int i = 0; i < A; ++i) {
                arrive(i);
                const uint32_t k = __shfl_sync(0xffffffffu, cur.p[i / L].x, i % L, L);
                if (b + i >= e) continue;
                if (k != key) {
                    if (key != 0xffffffffu) {
                        finish(false);
                        first = false;
                    }
                    key = k;
                    acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
                }
                if (live_col && k < none) add(i);
            }
        }
        cur = next;
        next = later;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (s < e) finish(e < (uint32_t)n && pairs(e).x == key);
    if (l == 0) sh.unit_info[unit] = make_int4(head, head_ends, tail_id, 0);
    __syncthreads();
    // The units' sums are joined in order: first kJoin units per thread and column, then those results by one thread per column.
    constexpr int W = 4 * L, P = U / kJoin;   // columns of the tile, first results
    {
        const int c = tid % W, g = tid / W;   // W * P threads: all of them
        const bool inside = c0 + c < a.width;
        Joined r{0.f, 0.f, false, false, -1};
        if (inside) r = join_units<kJoin, W>(a, sh.unit_info + g * kJoin, sh.sums + g * kJoin, 1, c, c0 + c);
        __syncthreads();
        if (inside) sh.sums[g * kJoin][0][c] = r.head, sh.sums[g * kJoin][1][c] = r.tail;
        if (c == 0) sh.part_info[g] = make_int4(r.any_head, r.ended, r.id, 0);
    }
    __syncthreads();
    if (tid >= W || c0 + tid >= a.width) return;
    const Joined r = join_units<P, W>(a, sh.part_info, sh.sums, kJoin, tid, c0 + tid);
    if (ONE) return;
    if (r.id >= 0) a.tail[(int64_t)cta * a.width + c0 + tid] = r.tail;
    if (r.any_head) a.head[(int64_t)cta * a.width + c0 + tid] = r.head;
    if (tid == 0 && blockIdx.y == 0) a.info[cta] = make_int4(r.any_head, r.ended, r.id >= 0, r.id);
}

template <int L, bool VEC>
__global__ void __launch_bounds__(kSumThreads, kSumPerSM) embed_sum_kernel(const SumArgs a) {
    __shared__ SumShared<L> sh;
    __shared__ RowRing<L, VEC> ring;
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    sum_sorted<L, VEC, false>(a, PairsInMemory{a.pairs}, a.n, a.per_unit, blockIdx.x, sh, ring);
}

// Rows of up to eight columns: a lane takes a whole row, a warp 32 sorted positions at a time, and the rows of one id are added by
// shuffles.  Neighbouring ids are stored together, where a unit of two lanes stores one row of 32 bytes or less at a time (28
// instead of 54 us for 2,449,029 x 4, an id each).  Rows that allow no wide accesses are read as the aligned 16 bytes that hold
// them; the first and the last rows of dout, beside which there need not be anything, element by element.
constexpr int kNarrow = 8, kNarrowUnits = kSumThreads / 32;
template <int NW, bool VEC>
struct NarrowRow {
    static constexpr int C = VEC ? NW / 4 : NW / 4 + 1;
    float4 part[C];
    int off;   // where the row starts in the first part
    __device__ __forceinline__ void load(const SumArgs& a, uint32_t pos, bool wanted) {
        const float* row = a.dout + (int64_t)pos * a.dout_ld;
        off = VEC ? 0 : (int)((uintptr_t)row >> 2 & 3);
        const bool edge = !VEC && (pos < 3 || pos + 3 >= (uint32_t)a.n);
        if (edge) off = 0;
#pragma unroll
        for (int q = 0; q < C; ++q) {
            part[q] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (edge) {
                if (wanted && 4 * q < a.width) part[q].x = row[4 * q];
                if (wanted && 4 * q + 1 < a.width) part[q].y = row[4 * q + 1];
                if (wanted && 4 * q + 2 < a.width) part[q].z = row[4 * q + 2];
                if (wanted && 4 * q + 3 < a.width) part[q].w = row[4 * q + 3];
            } else if (wanted && 4 * q < off + a.width) {
                part[q] = __ldg(reinterpret_cast<const float4*>(row - off + 4 * q));
            }
        }
    }
    __device__ __forceinline__ void get(float scale, int width, float (&v)[NW]) const {
        float w[4 * C];
#pragma unroll
        for (int q = 0; q < C; ++q) w[4 * q] = part[q].x, w[4 * q + 1] = part[q].y, w[4 * q + 2] = part[q].z, w[4 * q + 3] = part[q].w;
        if (!VEC) {
#pragma unroll
            for (int j = 0; j + 1 < 4 * C; ++j) w[j] = off & 1 ? w[j + 1] : w[j];
#pragma unroll
            for (int j = 0; j + 2 < 4 * C; ++j) w[j] = off & 2 ? w[j + 2] : w[j];
        }
#pragma unroll
        for (int j = 0; j < NW; ++j) v[j] = j < width ? scale * w[j] : 0.f;
    }
};
template <int NW, bool VEC>
__global__ void __launch_bounds__(kSumThreads, kSumPerSM) embed_sum_narrow_kernel(const SumArgs a) {
    __shared__ float sums[kNarrowUnits][2][kNarrow];
    __shared__ int4 unit_info[kNarrowUnits];
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    const int lane = threadIdx.x & 31, unit = threadIdx.x >> 5;
    const int64_t s64 = ((int64_t)blockIdx.x * kNarrowUnits + unit) * a.per_unit;
    const uint32_t s = (uint32_t)min((int64_t)a.n, s64), e = (uint32_t)min((int64_t)a.n, s64 + a.per_unit);
    const uint32_t none = (uint32_t)a.vocab;
    auto store_row = [&](uint32_t key, const float(&v)[NW]) {
        float* row = a.dtable + (int64_t)key * a.dtable_ld;
        if (a.present) a.present[key] = 1;
        if (VEC) {
#pragma unroll
            for (int q = 0; q < NW / 4; ++q)
                if (4 * q < a.width) {
                    float4 t = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                    float4* to = reinterpret_cast<float4*>(row + 4 * q);
                    if (a.accumulate) t.x += to->x, t.y += to->y, t.z += to->z, t.w += to->w;
                    *to = t;
                }
        } else {
#pragma unroll
            for (int j = 0; j < NW; ++j)
                if (j < a.width) row[j] = v[j] + (a.accumulate ? row[j] : 0.f);
        }
    };
    auto pair = [&](uint32_t i) { return i < e ? a.pairs[i] : make_uint2(0xffffffffu, 0u); };
    // The run that comes in from the 32 positions before, or from the unit before (then it is the unit's head, and empty so far).
    uint32_t carry_key = s > 0 && s < e ? a.pairs[s - 1].x : 0xfffffffeu;
    bool carry_head = true, carry_any = false;
    float carry[NW];
#pragma unroll
    for (int j = 0; j < NW; ++j) carry[j] = 0.f;
    bool head = false, head_ends = false;
    int tail_id = -1;
    auto finish_carry = [&](bool goes_on) {
        if (!carry_any || carry_key >= none) return;
        if (carry_head || goes_on) {
            if (lane == 0)
#pragma unroll
                for (int j = 0; j < NW; ++j) sums[unit][carry_head ? 0 : 1][j] = carry[j];
            if (carry_head) {
                head = true, head_ends = !goes_on;
            } else {
                tail_id = (int)carry_key;
                if (a.present && lane == 0) a.present[carry_key] = 1;
            }
        } else if (lane == 0) {
            store_row(carry_key, carry);
        }
    };
    uint2 p = pair(s + lane), next = pair(s + 32 + lane);
    NarrowRow<NW, VEC> row, next_row;
    row.load(a, p.y, p.x < none);
    for (uint32_t b = s; b < e; b += 32) {
        const uint2 later = pair(b + 64 + lane);
        next_row.load(a, next.y, next.x < none);
        float v[NW];
        row.get(a.scale, a.width, v);
        uint32_t before = __shfl_up_sync(0xffffffffu, p.x, 1);
        if (lane == 0) before = carry_key;
        const uint32_t starts = __ballot_sync(0xffffffffu, p.x != before);
        if (starts & 1u) finish_carry(false);
        const int from = 31 - __clz(starts & (0xffffffffu >> (31 - lane)));   // the run's first lane here, -1: it came in
        if (starts != 0xffffffffu) {
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const bool same = lane - o >= max(from, 0);
#pragma unroll
                for (int j = 0; j < NW; ++j) {
                    const float t = __shfl_up_sync(0xffffffffu, v[j], o);
                    v[j] += same ? t : 0.f;
                }
            }
            if (from < 0)
#pragma unroll
                for (int j = 0; j < NW; ++j) v[j] += carry[j];
        }
        const int last = (int)min(31u, e - 1 - b);   // the last lane's run stays open
        const bool ends = lane < last && starts >> (lane + 1) & 1u && p.x < none;
        const bool is_head = ends && from < 0 && carry_head;
        if (__ballot_sync(0xffffffffu, is_head)) head = head_ends = true;
        if (is_head) {
#pragma unroll
            for (int j = 0; j < NW; ++j) sums[unit][0][j] = v[j];
        } else if (ends) {
            store_row(p.x, v);
        }
        carry_head = carry_head && __shfl_sync(0xffffffffu, from, last) < 0;
        carry_key = __shfl_sync(0xffffffffu, p.x, last);
        carry_any = true;
#pragma unroll
        for (int j = 0; j < NW; ++j) carry[j] = __shfl_sync(0xffffffffu, v[j], last);
        p = next;
        next = later;
        row = next_row;
    }
    if (s < e) finish_carry(e < (uint32_t)a.n && a.pairs[e].x == carry_key);
    if (lane == 0) unit_info[unit] = make_int4(head, head_ends, tail_id, 0);
    __syncthreads();
    const int c = threadIdx.x;
    if (c >= a.width) return;
    const Joined r = join_units<kNarrowUnits, kNarrow>(a, unit_info, sums, 1, c, c);
    if (r.id >= 0) a.tail[(int64_t)blockIdx.x * a.width + c] = r.tail;
    if (r.any_head) a.head[(int64_t)blockIdx.x * a.width + c] = r.head;
    if (c == 0) a.info[blockIdx.x] = make_int4(r.any_head, r.ended, r.id >= 0, r.id);
}

// Small problems (up to kSmallN positions): one launch that sums.  Every CTA owns every gridDim.x-th row of the table (frequent ids
// often lie next to each other: with a stretch of the table each, one CTA had half of the positions), picks the positions of its
// ids out of all of them, sorts those in shared memory and sums them as above; nothing passes between CTAs.
constexpr int kSmallRows = 1 << 16;   // rows of the table per CTA at most
template <int L>
struct SmallShared {
    SumShared<L> sum;
    alignas(16) uint32_t list[2][kSmallN];   // one of them holds the rows on their way later: two CTAs fit an SM
    static_assert(sizeof(RowRing<L, true>) <= kSmallN * sizeof(uint32_t) && sizeof(RowRing<L, false>) <= kSmallN * sizeof(uint32_t));
    uint32_t next[8][256];
    uint32_t warp_total[8];
    uint32_t before[kSmallN / kSumThreads][8];
    uint32_t present[kSmallRows / 32];
};
// Tables of more rows, or bytes, than these take a launch of their own for it; smaller ones are cleared by the CTAs that sum, row by
// row (2,000 ids x 7 of 286,000 / 1,143,000 rows: 14 / 35 us row by row, 17 / 20 us apart; x 128, 32 / 64 MB: 14 / 18 and 21 / 23 us;
// x 100, 800 MB: 297 and 133 us).
constexpr int64_t kApartRows = 1 << 19, kApartBytes = 64 << 20;
// Rows without an id of a table that is large beside so few ids.  Every CTA marks which of its rows occur while the launch that sums
// (and writes the rows that occur) is at work, and clears the others when that has ended: reads between so many stores would wait
// long, and slow them (8,000 ids of 1,900,000 x 131: 203 us side by side, 186 one after the other).  The CTAs' rows are dealt out
// in chunks, so that all write to one neighbourhood at a time, and eight CTAs per SM even out who started late (6.6 TB/s; 5.6 with a
// stretch of the table for each of two per SM).  chunk: blocks of 32 rows, 1 .. kClearWarps.
constexpr int kClearThreads = 512, kClearWarps = kClearThreads / 32, kClearCtas = 8 * kSMs;
__global__ void __launch_bounds__(kClearThreads) embed_clear_kernel(const SumArgs a, const int32_t* ids, int chunk) {
    extern __shared__ uint32_t occurs[];   // [chunks of this CTA][chunk]
    const int first = (int)(4 * threadIdx.x + (-((uintptr_t)a.dtable >> 2) & 3));   // element of a chunk where the thread's first piece starts
    const int first_row = first / a.width, first_col = first - first_row * a.width;
    const int row_step = 4 * kClearThreads / a.width, col_step = 4 * kClearThreads - row_step * a.width;
    const uint32_t blocks = (uint32_t)((a.vocab + 31) / 32), chunks = (blocks + chunk - 1) / chunk;
    const int mine = (int)((chunks - blockIdx.x + gridDim.x - 1) / gridDim.x);
    for (int k = threadIdx.x; k < mine * chunk; k += kClearThreads) occurs[k] = 0;
    __syncthreads();
#pragma unroll 4
    for (int i = threadIdx.x; i < a.n; i += kClearThreads) {
        const uint32_t id = (uint32_t)ids[i], of = id / 32 / chunk, turn = of / gridDim.x;
        if (id < (uint32_t)a.vocab && of - turn * gridDim.x == blockIdx.x) atomicOr(&occurs[turn * chunk + id / 32 % chunk], 1u << (id & 31));
    }
    __syncthreads();
    cudaGridDependencySynchronize();
    const RowClear clear(a.dtable, a.dtable_ld, a.width, 0);
    for (int k = 0; k < mine; ++k) {
        const int64_t v = (int64_t)(k * gridDim.x + blockIdx.x) * chunk * 32;
        const int rows = (int)min((int64_t)chunk * 32, a.vocab - v);
        const uint32_t* const marks = occurs + k * chunk;
        if (!clear.pieces) {
            for (int r = threadIdx.x / 32 * 32; r < rows; r += kClearThreads) {
                const int count = min(32, rows - r);
                clear.block(v + r, count, ~marks[r / 32] & 0xffffffffu >> (32 - count));
            }
            continue;
        }
        // the chunk as one span, by all threads
        auto absent = [&](int r) { return !(marks[r >> 5] >> (r & 31) & 1u); };
        float* const from = a.dtable + v * a.width;
        const int count = rows * a.width, whole = (count - clear.lead) / 4, loose = count - 4 * whole;
        if ((int)threadIdx.x < loose) {
            const int e = (int)threadIdx.x < clear.lead ? threadIdx.x : 4 * whole + threadIdx.x;
            if (absent(e < a.width ? 0 : rows - 1)) from[e] = 0.f;
        }
        int r = first_row, c = first_col;
        for (int q = threadIdx.x; q < whole; q += kClearThreads) {
            float* const to = from + clear.lead + 4 * q;
            const bool here = absent(r), next = c + 4 > a.width ? absent(r + 1) : here;
            if (here && next) {
                *reinterpret_cast<float4*>(to) = make_float4(0.f, 0.f, 0.f, 0.f);
            } else if (here || next) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + j < a.width ? here : next) to[j] = 0.f;
            }
            r += row_step, c += col_step;
            if (c >= a.width) c -= a.width, ++r;
        }
    }
}

// K: ids a thread looks at
template <int L, bool VEC, int K>
__global__ void __launch_bounds__(kSumThreads) embed_small_kernel(const SumArgs a, const int32_t* ids, uint32_t magic, int apart, int32_t* status) {
    extern __shared__ __align__(16) unsigned char raw[];
    SmallShared<L>& sh = *reinterpret_cast<SmallShared<L>*>(raw);
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    cudaTriggerProgrammaticLaunchCompletion();   // the launch that clears the other rows may prepare
    const uint32_t rows = (uint32_t)((a.vocab - blockIdx.x + gridDim.x - 1) / gridDim.x);   // blockIdx.x, + gridDim.x, ...
    auto turn = [&](int32_t v) { return gridDim.x == 1 ? (uint32_t)v : __umulhi((uint32_t)v, magic); };   // v / gridDim.x
    int32_t id[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = k * kSumThreads + tid;
        id[k] = ids[min(i, a.n - 1)];
        if (i >= a.n) id[k] = -1;
    }
    for (int k = tid; k < (int)(rows + 31) / 32; k += kSumThreads) sh.present[k] = 0;
    uint32_t mine[K];   // lanes of the warp that found one of the CTA's ids
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (blockIdx.x == 0 && blockIdx.y == 0 && status && id[k] != -1 && (uint32_t)id[k] >= (uint32_t)a.vocab) atomicOr(status, SLICEGCN_DEVSTATUS_BAD_ID);
        mine[k] = __ballot_sync(0xffffffffu, (uint32_t)id[k] < (uint32_t)a.vocab && (uint32_t)id[k] - turn(id[k]) * gridDim.x == blockIdx.x);
        if (lane == 0) sh.before[k][w] = __popc(mine[k]);
    }
    __syncthreads();
    if (w == 0) {   // K * 8 counts to exclusive sums, an equal run of them per lane
        uint32_t* c = &sh.before[0][0];
        uint32_t v[K * 8 / 32], sum = 0;
#pragma unroll
        for (int q = 0; q < K * 8 / 32; ++q) v[q] = c[lane * (K * 8 / 32) + q], sum += v[q];
        uint32_t incl = sum;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        uint32_t at = incl - sum;
#pragma unroll
        for (int q = 0; q < K * 8 / 32; ++q) c[lane * (K * 8 / 32) + q] = at, at += v[q];
        if (lane == 31) sh.warp_total[0] = incl;
    }
    __syncthreads();
    const int m = (int)sh.warp_total[0];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (mine[k] >> lane & 1u) {
            const uint32_t local = turn(id[k]);
            sh.list[0][sh.before[k][w] + __popc(mine[k] & ((1u << lane) - 1u))] = local << kSmallBits | (uint32_t)(k * kSumThreads + tid);
            atomicOr(&sh.present[local >> 5], 1u << (local & 31));
        }
    __syncthreads();
    // stable sort by the row, eight bits at a time (most CTAs own few rows: one pass, or none)
    int cur = 0;
    const int run = ((m + 255) / 256) * 32;   // positions per warp
    for (int shift = kSmallBits; m > 0 && (rows - 1) >> (shift - kSmallBits); shift += 8, cur ^= 1) {
        for (int k = lane; k < 256; k += 32) sh.next[w][k] = 0;
        __syncwarp();
        const int i0 = min(m, w * run), i1 = min(m, i0 + run);
        for (int i = i0 + lane; i < i1; i += 32) atomicAdd(&sh.next[w][sh.list[cur][i] >> shift & 255u], 1u);
        __syncthreads();
        uint32_t total = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) total += sh.next[k][tid];
        uint32_t incl = total;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        if (lane == 31) sh.warp_total[w] = incl;
        __syncthreads();
        uint32_t at = incl - total;
        for (int k = 0; k < w; ++k) at += sh.warp_total[k];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t c = sh.next[k][tid];
            sh.next[k][tid] = at;
            at += c;
        }
        __syncthreads();
        for (int b = i0; b < i1; b += 32) {
            const bool live = b + lane < i1;
            const uint32_t p = live ? sh.list[cur][b + lane] : 0, d = p >> shift & 255u;
            const uint32_t peers = same_digit<8>(d, live);
            const uint32_t rank = __popc(peers & ((1u << lane) - 1u));
            uint32_t to = 0;
            if (live) to = sh.next[w][d] + rank;
            __syncwarp();
            if (live && rank == 0) sh.next[w][d] += __popc(peers);
            __syncwarp();
            if (live) sh.list[cur ^ 1][to] = p;
        }
        __syncthreads();
    }
    constexpr int U = SumShared<L>::U;
    sum_sorted<L, VEC, true>(a, PairsInShared{sh.list[cur], blockIdx.x, gridDim.x}, m, (m + U - 1) / U, 0, sh.sum,
                           *reinterpret_cast<RowRing<L, VEC>*>(sh.list[cur ^ 1]));   // the list that is not read any more
    if (!a.accumulate && !apart) {   // rows without an id
        const int l = tid & (L - 1), col = blockIdx.y * 4 * L + (VEC ? 4 * l : l);
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
        if (col < a.width)
            for (uint32_t r = tid / L; r < rows; r += U)
                if (!(sh.present[r >> 5] >> (r & 31) & 1u))
                    store4<VEC>(a.dtable + ((int64_t)r * gridDim.x + blockIdx.x) * a.dtable_ld, col, L, a.width, 0, zero);
    }
}

// What is left after the sums.  The first join_ctas CTAs: ids that reach over the edges of the sums' CTAs, a warp for the one
// that starts in each of them; one that reaches over more than kLongJoin is added by the whole CTA, in shares of consecutive
// parts that are then added in order.  The other CTAs: rows of ids that do not occur, unless the table was cleared before.
constexpr int kLongJoin = 16;
template <int L, bool VEC>
__global__ void __launch_bounds__(256) embed_finish_kernel(const SumArgs a, int join_ctas) {
    constexpr int W = 4 * L, PER = (W + 31) / 32;   // columns of the tile, of a lane
    __shared__ float part[8][W];
    __shared__ int last_of[8], id_of[8];
    cudaGridDependencySynchronize();
    const int c0 = blockIdx.y * W;
    if ((int)blockIdx.x >= join_ctas) {
        // 32 rows per warp and step, or fewer (a multiple of four) where there are few rows for so many warps
        const int64_t ctas = gridDim.x - join_ctas, warps = gridDim.y * ctas * 8;
        const int64_t warp = (blockIdx.y * ctas + blockIdx.x - join_ctas) * 8 + threadIdx.x / 32;
        const int rows = a.vocab >= 32 * warps ? 32 : a.vocab >= 16 * warps ? 16 : 8;
        const RowClear clear(a.dtable, a.dtable_ld, a.width, 0);
        const int64_t step = warps * rows;
        for (int64_t v = warp * rows; v < a.vocab; v += 4 * step) {
            bool absent[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t r = v + q * step + clear.lane;
                absent[q] = !a.present[min(r, a.vocab - 1)] && r < a.vocab && clear.lane < rows;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t r = v + q * step;
                const uint32_t bits = __ballot_sync(0xffffffffu, absent[q]);
                if (r < a.vocab) clear.block(r, (int)min((int64_t)rows, a.vocab - r), bits);
            }
        }
        return;
    }
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, start = blockIdx.x * 8 + w;
    // the parts lo .. hi of an id's sum, in order: several on their way at a time
    auto add = [&](int lo, int hi, float(&s)[PER]) {
#pragma unroll 8
        for (int k = lo; k <= hi; ++k)
#pragma unroll
            for (int j = 0; j < PER; ++j) s[j] += a.head[(int64_t)k * a.width + min(c0 + lane + 32 * j, a.width - 1)];
    };
    auto finish = [&](int id, const float(&tail)[PER], const float(&s)[PER]) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int c = lane + 32 * j;
            if (c < W && c0 + c < a.width) {
                float* to = a.dtable + (int64_t)id * a.dtable_ld + c0 + c;
                *to = tail[j] + s[j] + (a.accumulate ? *to : 0.f);
            }
        }
    };
    const int4 none = make_int4(0, 1, 0, 0);
    int4 f = start + lane < a.sum_ctas ? a.info[start + lane] : none;   // this one and those after it
    const int has_tail = __shfl_sync(0xffffffffu, f.z, 0), id = __shfl_sync(0xffffffffu, f.w, 0);
    int last = -1;
    if (has_tail) {
        float tail[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) tail[j] = a.tail[(int64_t)start * a.width + min(c0 + lane + 32 * j, a.width - 1)];
        unsigned ends = __ballot_sync(0xffffffffu, lane > 0 && (!f.x || f.y));   // the CTA in which the id ends
        int c = start;
        while (!ends) {
            c += 32;
            f = c + lane < a.sum_ctas ? a.info[c + lane] : none;
            ends = __ballot_sync(0xffffffffu, !f.x || f.y);
        }
        last = min(c + __ffs(ends) - 1, a.sum_ctas - 1);
        if (last - start <= kLongJoin) {
            float s[PER] = {};
            add(start + 1, last, s);
            finish(id, tail, s);
            last = -1;
        }
    }
    if (lane == 0) last_of[w] = last, id_of[w] = id;
    __syncthreads();
    for (int q = 0; q < 8; ++q) {
        if (last_of[q] < 0) continue;   // the same for the whole CTA
        const int from = blockIdx.x * 8 + q, share = (last_of[q] - from + 7) / 8;
        float s[PER] = {};
        add(from + 1 + w * share, min(last_of[q], from + (w + 1) * share), s);
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (lane + 32 * j < W) part[w][lane + 32 * j] = s[j];
        __syncthreads();
        if (w == 0) {
            float tail[PER];
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                tail[j] = a.tail[(int64_t)from * a.width + min(c0 + lane + 32 * j, a.width - 1)];
                s[j] = 0.f;
                if (lane + 32 * j < W)
                    for (int o = 0; o < 8; ++o) s[j] += part[o][lane + 32 * j];
            }
            finish(id_of[q], tail, s);
        }
        __syncthreads();
    }
}

slicegcn_status_t check_desc(const slicegcn_embed_desc* d, const char* who) {
    if (!d) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: NULL description", who);
    if (d->n < 0 || d->vocab < 1 || d->width < 1) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "%s: bad sizes", who);
    if (d->n >= ((int64_t)1 << 31) || d->vocab >= ((int64_t)1 << 31) - 1)
        SGCN_FAIL(SLICEGCN_ERR_OVERFLOW, "%s: n or vocab does not fit int32", who);
    if (d->width > SLICEGCN_MAX_EMBED_WIDTH) SGCN_FAIL(SLICEGCN_ERR_UNSUPPORTED, "%s: more than %d columns", who, SLICEGCN_MAX_EMBED_WIDTH);
    return SLICEGCN_OK;
}

int64_t align256(int64_t b) { return (b + 255) / 256 * 256; }

// One launch that sums while the picking (every CTA looks at all ids) and the most frequent rows (a row is one CTA's) are cheaper
// than the sort's launches: up to 8,192 ids and 1,024 of them per row on average.  (8,192 x 128 of 4,096 rows: 8.5 us, or 19.0 sorted
// by launches; 8,192 x 131 of 20 rows: 14.4 and 16.2; of 3 rows: 50 and 23.)
bool is_small(const slicegcn_embed_desc* d) {
    return d->n > 0 && d->n <= kSmallN && (d->n + 1023) / 1024 <= d->vocab && d->vocab <= (int64_t)kSMs * kSmallRows;
}

// A table of many more rows than there are ids is cleared as a whole, beside the sort, which keeps few SMs busy: at most a quarter
// of the rows is written a second time.  Otherwise the rows that do not occur are cleared at the end.
bool clear_first(const slicegcn_embed_desc* d) { return !d->accumulate && d->vocab / 4 >= d->n; }
constexpr int kClearBytes = 128 << 10;   // of a CTA that clears

// How the gradient is cut, and where its parts lie in the workspace.
struct GradPlan {
    int passes, bits, tiles;     // digit passes and bits per digit; CTAs of a pass
    int32_t tile;                // positions per CTA of a pass
    int lanes;                   // lanes per row of dout, four columns each
    int col_tiles, sum_ctas;
    int32_t per_unit;            // sorted positions per unit of lanes
    int64_t counts, present, head, tail, info, pairs[2], total;   // byte offsets
};
GradPlan grad_plan(const slicegcn_embed_desc* d) {
    GradPlan p;
    int key_bits = 1;
    while ((d->vocab >> key_bits) > 0) ++key_bits;   // keys run up to vocab itself
    p.passes = (key_bits + kMaxDigitBits - 1) / kMaxDigitBits;
    p.bits = std::max(2, (key_bits + p.passes - 1) / p.passes);
    // one CTA per SM at most: every CTA of a pass reads all tiles' counts
    const int64_t granule = kSortWarps * 32;
    int64_t tile = (d->n + kSMs - 1) / kSMs;
    tile = std::max<int64_t>(granule, (tile + granule - 1) / granule * granule);
    p.tile = (int32_t)std::min<int64_t>(tile, (int64_t)1 << 30);
    p.tiles = (int)std::max<int64_t>(1, (d->n + p.tile - 1) / p.tile);
    const int quads = (d->width + 3) / 4;
    p.lanes = 2;
    while (p.lanes < 32 && p.lanes < quads) p.lanes *= 2;
    p.col_tiles = (quads + p.lanes - 1) / p.lanes;
    const bool narrow = d->width <= kNarrow;   // (two lanes: a warp is the unit)
    const int units = narrow ? kNarrowUnits : kSumThreads / p.lanes;
    // One wave of CTAs, or two where the units are long enough to make up for their starts and ends (one / two waves:
    // 42 / 45 us at 36 positions per unit, 319 / 311 us at 518).
    const int64_t wave = std::max<int64_t>(1, kSMs * kSumPerSM / p.col_tiles) * units;
    const int64_t per_unit = (d->n + wave - 1) / wave;
    p.per_unit = (int32_t)std::max<int64_t>(8, per_unit >= 128 ? (per_unit + 1) / 2 : per_unit);
    if (narrow) p.per_unit = (p.per_unit + 31) / 32 * 32;
    p.sum_ctas = (int)((d->n + (int64_t)p.per_unit * units - 1) / ((int64_t)p.per_unit * units));
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += align256(bytes);
        return here;
    };
    p.counts = take(((int64_t)p.tiles << p.bits) * 4);
    p.present = take(d->vocab + 16);
    p.head = take((int64_t)p.sum_ctas * d->width * 4);
    p.tail = take((int64_t)p.sum_ctas * d->width * 4);
    p.info = take((int64_t)p.sum_ctas * 16);
    p.pairs[0] = take(d->n * 8);
    p.pairs[1] = take(d->n * 8);
    p.total = at;
    return p;
}

template <int L, bool VEC>
slicegcn_status_t launch_sum(const SumArgs& a, int col_tiles, cudaStream_t st) {
    if (a.sum_ctas > 0) {
        if constexpr (L == 2)
            SGCN_TRY(launch_after(a.width <= 4 ? embed_sum_narrow_kernel<4, VEC> : embed_sum_narrow_kernel<8, VEC>, dim3(a.sum_ctas), kSumThreads, 0, st, a));
        else
            SGCN_TRY(launch_after(embed_sum_kernel<L, VEC>, dim3(a.sum_ctas, col_tiles), kSumThreads, 0, st, a));
    }
    const int join_ctas = a.sum_ctas > 1 ? (a.sum_ctas + 7) / 8 : 0;
    const unsigned zero_ctas = a.present ? (unsigned)std::min<int64_t>((a.vocab + 63) / 64, std::max(1, kSMs * 6 / col_tiles)) : 0;
    if (join_ctas + zero_ctas > 0)
        SGCN_TRY(launch_after(embed_finish_kernel<L, VEC>, dim3(join_ctas + zero_ctas, col_tiles), 256, 0, st, a, join_ctas));
    return SLICEGCN_OK;
}

template <int L, bool VEC, int K>
slicegcn_status_t launch_small(const SumArgs& a, const int32_t* ids, int32_t* status, int col_tiles, cudaStream_t st) {
    // two CTAs per SM at most over the column tiles: every CTA looks at all ids
    int64_t ctas = std::min<int64_t>(kSMs, std::max(1, 2 * kSMs / col_tiles));
    ctas = std::min<int64_t>(a.vocab, std::max<int64_t>(ctas, (a.vocab + kSmallRows - 1) / kSmallRows));
    // id / ctas by a product: exact for ids below 2^32 / ctas, which is more than kSMs * kSmallRows
    const uint32_t magic = (uint32_t)(((uint64_t)1 << 32) / ctas + 1);
    constexpr int smem = (int)sizeof(SmallShared<L>);
    SGCN_CUDA(cudaFuncSetAttribute(embed_small_kernel<L, VEC, K>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    const bool apart = !a.accumulate && (a.vocab > kApartRows || a.vocab * a.width * 4 > kApartBytes);
    embed_small_kernel<L, VEC, K><<<dim3((unsigned)ctas, col_tiles), kSumThreads, smem, st>>>(a, ids, magic, apart, status);
    SGCN_LAUNCH_CHECK();
    count_launch();
    if (!apart) return SLICEGCN_OK;
    const int64_t blocks = (a.vocab + 31) / 32;
    int chunk = kClearWarps;   // as many blocks as make 128 KB, and no more than leave every CTA a chunk
    while (chunk > 1 && ((int64_t)chunk * 128 * a.width > 128 << 10 || blocks < (int64_t)chunk * kClearCtas)) chunk /= 2;
    const int64_t chunks = (blocks + chunk - 1) / chunk, clear_ctas = std::min<int64_t>(chunks, kClearCtas);
    const size_t marks = (chunks + clear_ctas - 1) / clear_ctas * chunk * 4;   // 2 KB at most
    // as much shared memory as there is: else an SM would have to be empty before it takes these CTAs beside the others
    SGCN_CUDA(cudaFuncSetAttribute(embed_clear_kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    return launch_after(embed_clear_kernel, dim3((unsigned)clear_ctas), kClearThreads, marks, st, a, ids, chunk);
}

template <bool VEC, int K>
slicegcn_status_t launch_smalls(const SumArgs& a, const int32_t* ids, int32_t* status, int lanes, int col_tiles, cudaStream_t st) {
    switch (lanes) {
        case 2: return launch_small<2, VEC, K>(a, ids, status, col_tiles, st);
        case 4: return launch_small<4, VEC, K>(a, ids, status, col_tiles, st);
        case 8: return launch_small<8, VEC, K>(a, ids, status, col_tiles, st);
        case 16: return launch_small<16, VEC, K>(a, ids, status, col_tiles, st);
        default: return launch_small<32, VEC, K>(a, ids, status, col_tiles, st);
    }
}

// 4, 16 or 32 ids per thread (2,708 ids: 6.5 us with 16, 7.8 us with 32)
template <bool VEC>
slicegcn_status_t launch_small_for(const SumArgs& a, const int32_t* ids, int32_t* status, int lanes, int col_tiles, cudaStream_t st) {
    if (a.n <= 4 * kSumThreads) return launch_smalls<VEC, 4>(a, ids, status, lanes, col_tiles, st);
    if (a.n <= 16 * kSumThreads) return launch_smalls<VEC, 16>(a, ids, status, lanes, col_tiles, st);
    return launch_smalls<VEC, 32>(a, ids, status, lanes, col_tiles, st);
}

template <bool VEC>
slicegcn_status_t launch_sums(const SumArgs& a, int lanes, int col_tiles, cudaStream_t st) {
    switch (lanes) {
        case 2: return launch_sum<2, VEC>(a, col_tiles, st);
        case 4: return launch_sum<4, VEC>(a, col_tiles, st);
        case 8: return launch_sum<8, VEC>(a, col_tiles, st);
        case 16: return launch_sum<16, VEC>(a, col_tiles, st);
        default: return launch_sum<32, VEC>(a, col_tiles, st);
    }
}

template <typename TT, typename TO, bool VEC, int ROWS>
slicegcn_status_t forward_typed(const slicegcn_embed_desc* d, const int32_t* ids, const void* table, void* out, int32_t* status, cudaStream_t st) {
    const int quads = (d->width + 3) / 4;
    int lanes = 1;
    while (lanes < 32 && lanes < quads) lanes *= 2;
    const int64_t rows_per_cta = 8 * (32 / lanes) * ROWS;
    const dim3 grid((unsigned)((d->n + rows_per_cta - 1) / rows_per_cta), (quads + lanes - 1) / lanes);
    auto go = [&](auto kernel) {
        kernel<<<grid, 256, 0, st>>>(d->n, d->vocab, d->width, ids, static_cast<const TT*>(table), d->table_ld, static_cast<TO*>(out), d->out_ld,
                                     (float)d->scale, status);
    };
    switch (lanes) {
        case 1: go(embed_forward_kernel<TT, TO, 1, VEC, ROWS>); break;
        case 2: go(embed_forward_kernel<TT, TO, 2, VEC, ROWS>); break;
        case 4: go(embed_forward_kernel<TT, TO, 4, VEC, ROWS>); break;
        case 8: go(embed_forward_kernel<TT, TO, 8, VEC, ROWS>); break;
        case 16: go(embed_forward_kernel<TT, TO, 16, VEC, ROWS>); break;
        default: go(embed_forward_kernel<TT, TO, 32, VEC, ROWS>); break;
    }
    SGCN_LAUNCH_CHECK();
    count_launch();
    return SLICEGCN_OK;
}

template <typename TT, typename TO>
slicegcn_status_t forward_aligned(const slicegcn_embed_desc* d, const int32_t* ids, const void* table, void* out, int32_t* status, cudaStream_t st) {
    const bool vec = d->width % 4 == 0 && d->table_ld % 4 == 0 && d->out_ld % 4 == 0 && (uintptr_t)table % (4 * sizeof(TT)) == 0 &&
                     (uintptr_t)out % (4 * sizeof(TO)) == 0;
    if (d->vocab * d->width * (int64_t)sizeof(TT) <= kTableInL2)
        return vec ? forward_typed<TT, TO, true, kRowsFromL2>(d, ids, table, out, status, st)
                   : forward_typed<TT, TO, false, kRowsFromL2>(d, ids, table, out, status, st);
    return vec ? forward_typed<TT, TO, true, kRowsFromHbm>(d, ids, table, out, status, st)
               : forward_typed<TT, TO, false, kRowsFromHbm>(d, ids, table, out, status, st);
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
    if (tbf) return obf ? forward_aligned<__nv_bfloat16, __nv_bfloat16>(d, ids, table, out, status, st)
                        : forward_aligned<__nv_bfloat16, float>(d, ids, table, out, status, st);
    return obf ? forward_aligned<float, __nv_bfloat16>(d, ids, table, out, status, st) : forward_aligned<float, float>(d, ids, table, out, status, st);
}

slicegcn_status_t slicegcn_embed_workspace_bytes(const slicegcn_embed_desc* d, int64_t* bytes) {
    SGCN_TRY(check_desc(d, "embed_workspace_bytes"));
    if (!bytes) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_workspace_bytes: NULL argument");
    *bytes = grad_plan(d).total;
    return SLICEGCN_OK;
}

slicegcn_status_t slicegcn_embed_backward(const slicegcn_embed_desc* d, const int32_t* ids, const float* dout, float* dtable,
                                          int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
    SGCN_TRY(check_desc(d, "embed_backward"));
    if (d->dout_ld < d->width || d->dtable_ld < d->width) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_backward: leading dimension too small");
    if (!dtable || (d->n > 0 && (!ids || !dout))) SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_backward: NULL argument");
    if ((uintptr_t)ids % 4 || (uintptr_t)status % 4 || (uintptr_t)dout % 4 || (uintptr_t)dtable % 4 || (uintptr_t)workspace % 16)
        SGCN_FAIL(SLICEGCN_ERR_INVALID_ARG, "embed_backward: a pointer is not aligned to its element type (workspace: 16 bytes)");
    const GradPlan p = grad_plan(d);
    if (!workspace || workspace_bytes < p.total)
        SGCN_FAIL(SLICEGCN_ERR_ALLOC, "embed_backward: workspace too small (%lld < %lld bytes)", (long long)workspace_bytes, (long long)p.total);
    cudaStream_t st = (cudaStream_t)stream;
    char* ws = static_cast<char*>(workspace);
    SumArgs t;
    t.n = (int32_t)d->n;
    t.vocab = d->vocab;
    t.width = d->width;
    t.accumulate = d->accumulate;
    t.dout = dout;
    t.dout_ld = d->dout_ld;
    t.dtable = dtable;
    t.dtable_ld = d->dtable_ld;
    t.scale = (float)d->scale;
    t.present = d->accumulate || clear_first(d) ? nullptr : reinterpret_cast<uint8_t*>(ws + p.present);
    t.per_unit = p.per_unit;
    t.sum_ctas = p.sum_ctas;
    t.head = reinterpret_cast<float*>(ws + p.head);
    t.tail = reinterpret_cast<float*>(ws + p.tail);
    t.info = reinterpret_cast<int4*>(ws + p.info);
    const bool vec = d->width % 4 == 0 && d->dout_ld % 4 == 0 && d->dtable_ld % 4 == 0 && (uintptr_t)dout % 16 == 0 && (uintptr_t)dtable % 16 == 0;
    if (is_small(d)) return vec ? launch_small_for<true>(t, ids, status, p.lanes, p.col_tiles, st) : launch_small_for<false>(t, ids, status, p.lanes, p.col_tiles, st);
    SortArgs a;
    a.n = (int32_t)d->n;
    a.vocab = d->vocab;
    a.ids = ids;
    a.counts = reinterpret_cast<uint32_t*>(ws + p.counts);
    a.present = t.present;
    a.status = status;
    a.bits = p.bits;
    a.tiles = p.tiles;
    a.tile = p.tile;
    a.clear = ClearShare{dtable, d->dtable_ld, d->width, d->vocab, 0, (kClearBytes / 4 / d->width + 32) / 32 * 32};
    unsigned clear_ctas = 0;   // per launch
    const int64_t of_a_cta_each = a.clear.rows_per_cta * 2 * p.passes;   // rows that one CTA in every launch clears
    if (clear_first(d)) clear_ctas = (unsigned)((d->vocab + of_a_cta_each - 1) / of_a_cta_each);
    const int64_t clear_rows = clear_ctas * a.clear.rows_per_cta;
    constexpr int kMaxSmem = kSortWarps * 4 << kMaxDigitBits;
    SGCN_CUDA(cudaFuncSetAttribute(sort_scatter_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem));
    SGCN_CUDA(cudaFuncSetAttribute(sort_scatter_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem));
    uint2* buf[2] = {reinterpret_cast<uint2*>(ws + p.pairs[0]), reinterpret_cast<uint2*>(ws + p.pairs[1])};
    for (int k = 0; k < p.passes; ++k) {
        a.shift = k * p.bits;
        a.in = buf[(k + 1) & 1];
        a.out = buf[k & 1];
        const size_t smem = (size_t)kSortWarps * 4 << p.bits;
        const dim3 grid(p.tiles + clear_ctas);
        if (k == 0) {
            sort_count_kernel<true><<<grid, kSortThreads, 0, st>>>(a);   // after whatever the stream holds
            SGCN_LAUNCH_CHECK();
            count_launch();
        } else {
            SGCN_TRY(launch_after(sort_count_kernel<false>, grid, kSortThreads, 0, st, a));
        }
        a.clear.row0 += clear_rows;
        SGCN_TRY(launch_after(k == 0 ? sort_scatter_kernel<true> : sort_scatter_kernel<false>, grid, kSortThreads, smem, st, a));
        a.clear.row0 += clear_rows;
    }
    t.pairs = buf[(p.passes + 1) & 1];
    SGCN_TRY(vec ? launch_sums<true>(t, p.lanes, p.col_tiles, st) : launch_sums<false>(t, p.lanes, p.col_tiles, st));
    return SLICEGCN_OK;
}

}  // extern "C"
