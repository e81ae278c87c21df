// What the kernels of tree_verify_attn and of its 8-bit form share: row tiles, the order of workgroups, wavefront maxima, wait
// states behind matrix instructions, and the merge of key ranges.
#pragma once
#include "internal.h"
#include "devscope.h"

namespace w4 {

typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kHeadDim = 128;
constexpr int kKeyBlock = 32;
constexpr int kRowsPad = 64;
constexpr int kMaxRanges = 32;   // of any plan (the merge keeps one value per range in registers)
constexpr int kChipTiles = 256;  // tiles x ranges of the plans that are picked by predicted time: one workgroup per compute unit

// v_max3_f32 and v_max_f32 as they stand: fmaxf chains are compiled with a canonicalising v_max x, x per
// operand, which doubles the instruction count of a row maximum.  They pass over a NaN (the scores that the 8-bit kernels make NaN): it need
// not be in the maximum to reach the row's sum and outputs, since its exponential is NaN whatever the maximum.
// The compiler adds no wait states before inline assembly: results of matrix instructions pass through settled() first.
__device__ __forceinline__ float max_of_three(float a, float b, float c)
{
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

__device__ __forceinline__ float max_of_two(float a, float b)
{
    float d;
    asm("v_max_f32 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
    return d;
}

// Wait states until results of matrix instructions that were just issued may be read: passes + 4, that is eight after a 16x16x32 step and twelve
// after a 32x32x16 one.  settled<N>() adds N of them and keeps reads of its operands behind it; the steps and other
// instructions in between make up the rest, on every path from the products to the first read.
template <int N>
__device__ __forceinline__ void settled(float4v &a, float4v &b)
{
    static_assert(N >= 0 && N <= 8, "one s_nop");
    if constexpr (N == 0) asm volatile("" : "+v"(a), "+v"(b));
    else asm volatile("s_nop %2" : "+v"(a), "+v"(b) : "n"(N - 1));
}
__device__ __forceinline__ void settled(float16v &a) { asm volatile("s_nop 7\n\ts_nop 3" : "+v"(a)); }

// Maximum over the four lanes l, l ^ 16, l ^ 32, l ^ 48 (the lanes that share a query row), returned to
// all four.  v_permlane16_swap exchanges the odd 16-lane rows of its first operand with the even rows of
// its second, v_permlane32_swap the upper half of the first with the lower half of the second; applied
// to two copies of a value each leaves the two partners of a pair side by side in the two registers.
// They run on the vector ALU: no LDS round trip as with a cross-lane shuffle.  (Written in assembly:
// the compiler's builtin folded the maximum of the two results into one of them.)
__device__ __forceinline__ float row_group_max(float v)
{
    float a = v, b = v;
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    a = max_of_two(a, b);
    b = a;
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return max_of_two(a, b);
}

// maximum over the lanes l and l ^ 32, returned to both
__device__ __forceinline__ float half_wave_max(float v)
{
    float a = v, b = v;
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return max_of_two(a, b);
}

constexpr float kLowest = -1.0e30f;   // "no key seen yet": finite, so differences of two of them are 0, not NaN

// The rows of a row tile.  The group * M (head, query row) pairs that share a KV head, head by head, are cut into
// tiles_per_kv tiles of tile_rows rows (the last may have fewer): M for one query head per tile, d * M for d heads, or any
// other number up to the kernel's tallest tile, 32, 64 or 128 rows, where a tile ends inside a head.  Row rho of tile `unit` is pair first + rho of its KV head.
struct RowTile {
    int kvh, group, M, Hq;
    int first;    // pair of tile row 0
    int rows;     // valid rows
    int index;    // number of the tile in its KV head
    bool whole;   // one query head per tile: no division
    __device__ __forceinline__ RowTile(int kvh_, int index_, int M_, int Hq_, int group_, int tile_rows)
    {
        M = M_;
        Hq = Hq_;
        group = group_;
        kvh = kvh_;
        index = index_;
        first = index * tile_rows;
        rows = min(tile_rows, group * M - first);
        whole = tile_rows == M;
    }
    // query row and head of a tile row; rows beyond the last repeat it (and are never stored)
    __device__ __forceinline__ void locate(int rho, int &qrow, int &head) const
    {
        const int pair = first + min(rho, rows - 1);
        const int j = whole ? index : pair / M;
        qrow = pair - j * M;
        head = kvh * group + j;
    }
};

// The row tile and the key range of a workgroup.  Workgroups go to the eight XCDs in turn; numbered so that each XCD gets a run of
// consecutive numbers, and the tiles of one KV head and one range next to each other, an XCD reads few keys, and its L2 brings them
// in once for all their tiles.  Any grid, each pair once.  Before, a grid that eight does not divide kept the order of launch, and its XCDs all read all keys; and
// the ranges of a tile stood together, so that with fewer KV heads than XCDs each XCD read most keys of a head.  us: 28/4 heads, M = 28, prefix
// 11477 31.1 -> 18.7, M = 8, prefix 3404 14.4 -> 10.0; 24/3 heads, M = 36, prefix 21792 43.3 -> 25.6; 20/5 heads, M = 52, prefix 3695 17.7 -> 12.9.
struct Share {
    int kvh, tile, range;   // KV head, row tile in it, key range
    // by_tiles, by_ranges: divider() of tiles_per_kv and nsplit -- the divisions stand before the first address, where nothing hides them
    __device__ __forceinline__ Share(unsigned block, unsigned grid, int nsplit, int tiles_per_kv, uint32_t by_tiles, uint32_t by_ranges)
    {
        const unsigned xcd = block & 7u;
        const unsigned number = xcd * (grid >> 3) + min(xcd, grid & 7u) + (block >> 3);
        const unsigned rest = __umulhi(2 * number, by_tiles);
        tile = (int)(number - rest * (unsigned)tiles_per_kv);
        kvh = (int)__umulhi(2 * rest, by_ranges);
        range = (int)rest - kvh * nsplit;
    }
};
// n / d == umulhi(2 n, divider(d)) while n d < 2^31: the factor exceeds 2^31 / d by less than one, n times that stays below 2^31 / d
static uint32_t divider(int d) { return (uint32_t)(((1u << 31) + (unsigned)d - 1) / (unsigned)d); }

// Merge of the key ranges of one tile by the workgroup that finished last (fused mode): NS = compiled
// upper bound of the number of ranges, IT = items a thread handles at once (all their loads are issued
// together), PAD = rows that the partials of a range take, MARKS = a range's sum may be kPaddingMark.  Loads are device-scope: other
// workgroups, on other XCDs, wrote the partials in this kernel.
constexpr float kPaddingMark = -1.f;   // the row gets zeros, whatever the ranges hold
template <int NS, int IT, int PAD, bool MARKS>
__device__ __forceinline__ void merge_ranges(PartialBuffer unit_o, PartialBuffer unit_ml, _Float16 *__restrict__ out,
                                             int tid, int threads, const RowTile &tile, int nsplit)
{
    const int items = tile.rows * (kHeadDim / 4);   // one item = four consecutive outputs of a tile row
    const float NEG_INF = -__builtin_inff();
    for (int base = tid; base < items; base += threads * IT) {
        float ms[IT][NS], ls[IT][NS];
        float4v os[IT][NS];
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int idx = base + it * threads;
            const int trow = idx / (kHeadDim / 4), d4 = idx % (kHeadDim / 4);
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                ms[it][s] = NEG_INF;
                ls[it][s] = 0.f;
                os[it][s] = (float4v){0.f, 0.f, 0.f, 0.f};
                if (s < nsplit && idx < items) {
                    ms[it][s] = load_partial_f32(unit_ml, (s * PAD + trow) * 2);
                    ls[it][s] = load_partial_f32(unit_ml, (s * PAD + trow) * 2 + 1);
                    os[it][s] = load_partial(unit_o, (s * PAD + trow) * (kHeadDim / 4) + d4);
                }
            }
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int idx = base + it * threads;
            if (idx >= items) break;
            const int trow = idx / (kHeadDim / 4), d4 = idx % (kHeadDim / 4);
            float m_all = NEG_INF;
#pragma unroll
            for (int s = 0; s < NS; ++s) m_all = fmaxf(m_all, ms[it][s]);
            float den = 0.f;
            float4v num = {0.f, 0.f, 0.f, 0.f};
            bool padding = false;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                if constexpr (MARKS) padding |= ls[it][s] < 0.f;
                float wgt = (ms[it][s] == NEG_INF) ? 0.f : __builtin_amdgcn_exp2f(ms[it][s] - m_all);
                den += wgt * ls[it][s];
                num += wgt * os[it][s];
            }
            const float inv = padding ? 0.f : 1.f / den;   // a row that sees no key, or none but scores of -inf: 0 / 0, as from one range
            if (padding) num = (float4v){0.f, 0.f, 0.f, 0.f};
            int qrow, h;
            tile.locate(trow, qrow, h);
            typedef _Float16 half4v __attribute__((ext_vector_type(4)));
            half4v hv = {(_Float16)(num[0] * inv), (_Float16)(num[1] * inv), (_Float16)(num[2] * inv), (_Float16)(num[3] * inv)};
            *reinterpret_cast<half4v *>(out + ((size_t)qrow * tile.Hq + h) * kHeadDim + d4 * 4) = hv;
        }
    }
}

template <int PAD = kRowsPad, bool MARKS = false>
__device__ __forceinline__ void merge_tile(PartialBuffer unit_o, PartialBuffer unit_ml, _Float16 *__restrict__ out, int tid,
                                           int threads, const RowTile &tile, int nsplit)
{
    if (nsplit <= 4) merge_ranges<4, 4, PAD, MARKS>(unit_o, unit_ml, out, tid, threads, tile, nsplit);
    else if (nsplit <= 8) merge_ranges<8, 2, PAD, MARKS>(unit_o, unit_ml, out, tid, threads, tile, nsplit);
    else if (nsplit <= 16) merge_ranges<16, 1, PAD, MARKS>(unit_o, unit_ml, out, tid, threads, tile, nsplit);
    else merge_ranges<kMaxRanges, 1, PAD, MARKS>(unit_o, unit_ml, out, tid, threads, tile, nsplit);
}

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v lds_short4v;

__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return (uint32_t)(size_t)(lds_void *)p;
}
// returns once at most N LDS operations of this wavefront (the N most recent) are still under way; lo and hi are the
// oldest pair still awaited, so that no use of it, not even a copy, can be moved above the wait
template <int N>
__device__ __forceinline__ void wait_lds_reads(short4v &lo, short4v &hi)
{
    asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(lo), "+v"(hi) : "n"(N));
}
// lane l's 16 bytes at src land at lds_base + 16 l (lds_base wavefront-uniform); counted by vmcnt
__device__ __forceinline__ void row_to_lds(const uint8_t *src, uint8_t *lds_base)
{
    __builtin_amdgcn_global_load_lds((global_void *)src, (lds_void *)lds_base, 16, 0, 0);
}

// the whole group cut evenly into as few tiles as `most` rows allow; a tile may end inside a head
static void even_tiles(int pairs, int most, int &tile_rows, int &tiles_per_kv)
{
    const int n = (pairs + most - 1) / most;
    tile_rows = (pairs + n - 1) / n;
    tiles_per_kv = (pairs + tile_rows - 1) / tile_rows;
}

// the transposing read of four key rows at lds_addr + OFFSET and the four that lie eight rows further on
template <int OFFSET>
__device__ __forceinline__ void read_transposed_rows(short4v &lo, short4v &hi, uint32_t lds_addr)
{
    asm volatile("ds_read_b64_tr_b16 %0, %2 offset:%3\n\tds_read_b64_tr_b16 %1, %2 offset:%4"
                 : "=&v"(lo), "=&v"(hi)
                 : "v"(lds_addr), "n"(OFFSET), "n"(OFFSET + 8 * 256));
}

}  // namespace w4
