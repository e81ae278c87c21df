// lm_head_sample: next tokens from logits and given uniform numbers, with temperature, top-k, top-p and min-p.  Contract in
// include/w4a16.h.
//
// A token's weight is w = exp((x - max) / T), evaluated in fp64 and held as a whole number of 2^-44: sums of whole numbers do not depend
// on their order, so any split of a row gives the same token, and a border (a cumulative weight against p, or against u) is off by at most V 2^-45
// of the row's total (the largest weight is 1; 7.5e-9 for 262144 tokens) where sums in fp32 would be off by 1e-5 -- tokens near a border would change with
// the split.  Tokens more than e^31 below the row's largest weigh nothing (262144 of them 9e-9 of the total at most) and take part in nothing.
//
// Short rows take one kernel, a workgroup per row (sample_row_kernel).  Longer ones take three, each of several workgroups per
// row, that pass over the logits once:
//   sample_top_kernel    the largest logit of each chunk of kChunk tokens, its token, and the smallest number
//   sample_bins_kernel   counts and weights (fp32 is enough here) in kBins bins of even width in max - x; the row's last workgroup finds the
//                        few bins in which the limits of top-k and top-p fall, whatever the rounding.  Not launched without such limits.
//   sample_draw_kernel   exact weight of what certainly stays, by segments of 512 tokens, and a list of the tokens in those few bins; the row's last
//                        workgroup sorts the list, which gives the exact cut, draws the segment and then the token inside it
// A list of more than kList tokens is given up: the last workgroup then finds the cut by digits of the logits, in some seven passes over the row by itself.
// Thousands of nearly equal logits come to that, and so does a top-p border among many small weights: bins are (largest - smallest) / 1024 wide, and the border is
// known to 2^-16 of the row's weight (find_cut).  Normal logits of standard deviation 2.2 with some larger ones, us by top-p (none: no limits):
//   tokens, rows, T       none  0.9   0.99  0.995 0.999 0.9999
//   128256,  1, 1.0       12.7  22.0  23.8  24.3  30.4  642
//   128256,  1, 1.5       12.6  25.8  25.7  26.2  25.8  27.8
//   128256, 60, 1.0       33.6  49.5  51.7  52.2  1138  1152
//   262144,  1, 1.0       14.0  24.7  26.8  28.6  1249  1150
//   262144, 60, 1.0       54.5  76.3  77.5  81.5  2258  2292
//   262144, 60, 1.5       54.6  86.4  2081  2224  1472  2276
// Measured, the three kernels: 1 row of 32000 tokens, top-k 4 + 8 + 9 us; 7 rows of 128256, top-p 4 + 9 + 16; 60 rows of 128256, all limits
// 8 + 14 + 18, where reading the logits once takes 6.  What bounds them: for few rows the chain of dependent steps (three launches, two meetings of a
// row's workgroups, each several trips to memory); for many the vector units, which put every token in its bin and weigh the kept ones in fp64.
// One kernel for the first two, with bins of each workgroup's own width that its row's last one puts together, took 21.0, 30.0 and 39.6 us in all, against
// 21.6, 28.2 and 41.9 at the time: 3 and 5 % less at two of these sizes, 6 % more at the other, and not taken for that.
#include "internal.h"
#include "devscope.h"

namespace w4 {

constexpr int kSampleThreads = 512, kSampleWaves = kSampleThreads / 64;
constexpr int kPer = 16;                                 // tokens of a chunk per thread
constexpr int kChunk = kSampleThreads * kPer;
constexpr int kChunks = 262144 / kChunk;                 // of the largest vocabulary
constexpr int kBins = 1024;
constexpr int kList = 2048;                              // entries of a row's list
constexpr int kSegment = 512;                            // tokens whose weight is held as one number
constexpr int kSegments = kChunks * kChunk / kSegment;   // of the largest vocabulary
constexpr int kGroups = 64;                              // workgroups of a row in sample_draw_kernel
constexpr double kFarthest = 31.0;
constexpr double kOne = 17592186044416.0;                // 2^44: weight 1
constexpr int32_t kNoToken = 0x7FFFFFFF;
constexpr int kNoBin = kBins;

// 2^(-j / 32), rounded to nearest
__device__ const double kRoots[32] = {
    0x1.0000000000000p+0, 0x1.f50765b6e4540p-1, 0x1.ea4afa2a490dap-1, 0x1.dfc97337b9b5fp-1,
    0x1.d5818dcfba487p-1, 0x1.cb720dcef9069p-1, 0x1.c199bdd85529cp-1, 0x1.b7f76f2fb5e47p-1,
    0x1.ae89f995ad3adp-1, 0x1.a5503b23e255dp-1, 0x1.9c49182a3f090p-1, 0x1.93737b0cdc5e5p-1,
    0x1.8ace5422aa0dbp-1, 0x1.82589994cce13p-1, 0x1.7a11473eb0187p-1, 0x1.71f75e8ec5f74p-1,
    0x1.6a09e667f3bcdp-1, 0x1.6247eb03a5585p-1, 0x1.5ab07dd485429p-1, 0x1.5342b569d4f82p-1,
    0x1.4bfdad5362a27p-1, 0x1.44e086061892dp-1, 0x1.3dea64c123422p-1, 0x1.371a7373aa9cbp-1,
    0x1.306fe0a31b715p-1, 0x1.29e9df51fdee1p-1, 0x1.2387a6e756238p-1, 0x1.1d4873168b9aap-1,
    0x1.172b83c7d517bp-1, 0x1.11301d0125b51p-1, 0x1.0b5586cf9890fp-1, 0x1.059b0d3158574p-1};
__device__ __forceinline__ double *roots()   // the same in LDS: every kernel fills it ahead of its first barrier
{
    __shared__ double of_two[32];
    return of_two;
}
__device__ __forceinline__ void fill_roots()
{
    if (threadIdx.x < 32) roots()[threadIdx.x] = kRoots[threadIdx.x];
}

// exp(-y) for 0 <= y < 32: a power of two, a root of two and the Taylor series of exp at |f| <= ln 2 / 64 up to f^5 (remainder 3e-15)
// (2 to 4 % of a call faster than up to f^11 at |f| <= ln 2 / 2 without a table; roots gathered from memory cost more than they save)
__device__ __forceinline__ double exp_minus(double y)
{
    const double t = y * (32.0 * 1.4426950408889634074);
    const double n = rint(t);
    const int whole = (int)n;
    const double root = roots()[whole & 31];
    const double f = (n - t) * (0.69314718055994530942 / 32.0);
    // the coefficients in scalar registers, as third operands: else every multiply-add of the chain copies one first
    double c4 = 1.0 / 24.0, c3 = 1.0 / 6.0;
    asm("" : "+s"(c4));
    asm("" : "+s"(c3));
    double r = 1.0 / 120.0;
    r = fma(r, f, c4);
    r = fma(r, f, c3);
    r = fma(r, f, 0.5);
    r = fma(r, f, 1.0);
    r = fma(r, f, 1.0) * root;
    return __builtin_bit_cast(double, __builtin_bit_cast(int64_t, r) - ((int64_t)(whole >> 5) << 52));
}

// order-preserving bits of a logit: greater numbers, greater keys; -0 as 0
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

__device__ __forceinline__ float order_number(uint32_t key)
{
    return __builtin_bit_cast(float, key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
// tokens in the order of falling logits, equal ones by rising index: greater is earlier
__device__ __forceinline__ uint64_t order_of(float x, int i) { return ((uint64_t)order_key(x) << 32) | (uint32_t)~i; }

// what a row is sampled with
struct RowRule {
    float top;       // largest logit
    double inv_t;
    bool greedy;
    int k;           // 0: no limit
    double p;        // >= 1: no limit
    double min_w;    // 0: no limit
    float bins_per;  // bins of unit depth
    float deepest;   // tokens of this depth and more weigh nothing
    float u;         // the uniform number

    // Half the distance below the largest logit, in fp32: rises as x falls, the same for equal logits, and cannot overflow.  It says which tokens take part
    // (depth < deepest; not so for NaN and -inf) and which bin they are in.
    __device__ __forceinline__ float depth(float x) const { return x == top ? 0.f : __builtin_fmaf(-0.5f, x, 0.5f * top); }
    __device__ __forceinline__ int bin(float depth) const { return (int)fminf(depth * bins_per, (float)(kBins - 1)); }
    __device__ __forceinline__ float per_octave() const { return (float)(inv_t * -2.0 * 1.44269504088896340736); }   // of a weight, by depth
    __device__ __forceinline__ bool limited() const { return k != 0 || p < 1.0; }
    // distance below the largest logit in units of the temperature, of tokens that take part
    __device__ __forceinline__ double below(float x) const { return x == top ? 0.0 : ((double)top - (double)x) * inv_t; }
};
// w in whole numbers of 2^-44, 0 <= w <= 1: added to 2^52, a double's lowest bit is one
__device__ __forceinline__ uint64_t units(double w) { return __builtin_bit_cast(uint64_t, fma(w, kOne, 0x1p52)) & ((1ull << 52) - 1); }

struct SampleArgs {
    const float *logits;
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p, *uniform;
    int32_t *token;
    float *prob;
    int V, chunks, segments;
    int bin_groups, bin_chunks;      // workgroups of a row in sample_bins_kernel, chunks of each
    int groups, rounds;              // workgroups of a row in sample_draw_kernel, segments of each wavefront
    struct ChunkTop *tops;           // [M][chunks]
    unsigned long long *bins;        // [M][bin_groups][kBins]: count << 48 | weight in 2^-31; a group has 32768 tokens at most
    struct RowCut *cuts;             // [M]
    unsigned long long *kept;        // [M][segments]: weight that stays for certain and is not below min_p
    struct GroupMass *masses;        // [M][groups]
    unsigned long long *lists;       // [M][groups][kList]
    uint32_t *tickets;               // [2 M]
};
// a chunk's largest logit and its first token (order_of; that of -inf and kNoToken if it has none), and its smallest number (~order_key)
struct ChunkTop { unsigned long long order, deep; };
__device__ __forceinline__ ChunkTop chunk_top(float top, int at, float least) { return {order_of(top, at), (uint32_t)~order_key(least)}; }
// weights of all above the first border bin, and of all between the border bins and the k-th token's; the length of the group's list
struct GroupMass { unsigned long long above, between, listed, unused; };
struct RowCut { int32_t first, last, k_bin, above_k; };   // border bins of top-p (first .. last), bin of the k-th token (kNoBin: none), tokens in the bins above it

// Inclusive sum over a wavefront's lanes, on the vector ALU: within rows of 16 lanes by shifts, then over rows.
template <int CONTROL, int ROWS>
__device__ __forceinline__ uint64_t moved(uint64_t v)
{
    const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CONTROL, ROWS, 0xf, true);
    const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CONTROL, ROWS, 0xf, true);
    return ((uint64_t)high << 32) | low;
}
__device__ __forceinline__ uint64_t scan_wave(uint64_t v)
{
    v += moved<0x111, 0xf>(v);   // row_shr:1
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);   // lane 15 of a row to the next row: rows 1 and 3
    v += moved<0x143, 0xc>(v);   // lane 31 to rows 2 and 3
    return v;
}
__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane)   // lane uniform
{
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
// the greatest of a wavefront's lanes, in each of them
__device__ __forceinline__ uint64_t max_wave(uint64_t v)
{
    auto join = [&](uint64_t o) { v = o > v ? o : v; };
    join(moved<0x111, 0xf>(v));
    join(moved<0x112, 0xf>(v));
    join(moved<0x114, 0xf>(v));
    join(moved<0x118, 0xf>(v));
    join(moved<0x142, 0xa>(v));
    join(moved<0x143, 0xc>(v));
    return of_lane(v, 63);
}

// what row m asks for
struct RowParams { float t, p, min_p, u; int k; };
__device__ __forceinline__ RowParams row_params(const SampleArgs &a, int m)
{
    // all loads together: a limit that is not given reads the uniform number instead
    RowParams q = {(a.temperature ? a.temperature : a.uniform)[m], (a.top_p ? a.top_p : a.uniform)[m], (a.min_p ? a.min_p : a.uniform)[m], a.uniform[m],
                   (a.top_k ? a.top_k : reinterpret_cast<const int32_t *>(a.uniform))[m]};
    if (!a.temperature) q.t = 1.f;
    if (!a.top_k) q.k = 0;
    if (!a.top_p) q.p = 1.f;
    if (!a.min_p) q.min_p = 0.f;
    return q;
}
__device__ __forceinline__ RowRule row_rule(const RowParams &q, int V, const ChunkTop &of_row)
{
    RowRule r;
    r.u = q.u;
    r.top = order_number((uint32_t)(of_row.order >> 32));
    r.greedy = !(q.t > 0.f) || q.k == 1 || q.p <= 0.f || q.min_p > 1.f;
    r.inv_t = r.greedy ? 0.0 : 1.0 / (double)q.t;
    r.k = q.k > 0 && q.k < V ? q.k : 0;
    r.p = q.p < 1.f ? (double)q.p : 2.0;
    r.min_w = q.min_p > 0.f ? (double)q.min_p : 0.0;
    // the bins span the distances that there are, so that they stay narrow at high temperatures
    r.deepest = r.greedy ? 0.f : fmaxf((float)(0.5 * kFarthest * (double)q.t), 0x1p-149f);
    const float span = fminf(r.depth(order_number(~(uint32_t)of_row.deep)), r.deepest);
    r.bins_per = span > 0.f ? fminf((float)kBins / span, 3.0e38f) : 0.f;
    return r;
}
__device__ __forceinline__ ChunkTop join_lanes(const ChunkTop &c) { return {max_wave(c.order), max_wave(c.deep)}; }
// of row m, as sample_top_kernel left it; every lane of a wavefront calls it
__device__ __forceinline__ ChunkTop row_top(const SampleArgs &a, int m)
{
    const int lane = threadIdx.x & 63;
    return join_lanes(lane < a.chunks ? a.tops[m * a.chunks + lane] : chunk_top(-__builtin_inff(), kNoToken, __builtin_inff()));
}
__device__ __forceinline__ int32_t token_of(const ChunkTop &c) { return (int32_t)~(uint32_t)c.order; }   // kNoToken: none

// the uniform number as a rank of weight units below total
__device__ __forceinline__ uint64_t drawn_rank(float u, uint64_t total)
{
    const uint64_t r = u > 0.f ? (uint64_t)(fminf(u, 0x1.fffffep-1f) * (double)total) : 0;
    return r < total ? r : total - 1;
}

// One 64-bit value as two device-scope halves: read by another workgroup of the same kernel.
__device__ __forceinline__ void store_shared(unsigned long long *p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t load_shared(unsigned long long *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Whether this workgroup is the last of its row's to come here; what the others stored at device scope before is then there.  The ticket is left
// at zero.
__device__ __forceinline__ bool last_of_row(uint32_t *ticket, int chunks)
{
    __shared__ uint32_t drawn;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        drawn = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (drawn == (uint32_t)(chunks - 1)) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return drawn == (uint32_t)(chunks - 1);
}

// inclusive sums over the workgroup's threads, in thread order, of N numbers; total: over all
template <int N>
__device__ __forceinline__ void scan_block(uint64_t (&v)[N], uint64_t (&total)[N])
{
    __shared__ unsigned long long wave_sum[kSampleWaves][N];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();   // an earlier call's sums have been read
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = scan_wave(v[i]);
        if (lane == 63) wave_sum[wave][i] = v[i];
        total[i] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSampleWaves; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t of_wave = wave_sum[w][i];
            if (w < wave) v[i] += of_wave;
            total[i] += of_wave;
        }
}

__global__ __launch_bounds__(kSampleThreads) void sample_top_kernel(const SampleArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, m = blockIdx.y, first = blockIdx.x * kChunk;
    const float *x = a.logits + (size_t)m * a.V;
    float v[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int i = first + e * kSampleThreads + tid;
        v[e] = i < a.V ? x[i] : -__builtin_inff();
    }
    float top = -__builtin_inff(), least = __builtin_inff();
    int at = kNoToken;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {   // NaN and -inf are no tokens
        if (v[e] > top) top = v[e], at = first + e * kSampleThreads + tid;
        if (v[e] > -__builtin_inff()) least = fminf(least, v[e]);
    }
    __shared__ ChunkTop of_wave[kSampleWaves];
    ChunkTop c = chunk_top(top, at, least);
    c = join_lanes(c);
    if (lane == 0) of_wave[tid >> 6] = c;
    __syncthreads();
    if (tid < 64) {
        c = join_lanes(of_wave[lane & (kSampleWaves - 1)]);
        if (tid == 0) a.tops[m * a.chunks + blockIdx.x] = c;
    }
}

__device__ __forceinline__ void into_bins(unsigned long long *bins, const RowRule &r, float depth, float per_octave)   // a token that takes part
{
    const float w = __builtin_amdgcn_exp2f(depth * per_octave);
    atomicAdd(&bins[r.bin(depth)], (1ull << 48) + (unsigned long long)(uint32_t)(w * 2147483648.f + 0.5f));
}

// The bins in which the limits fall, from the counts and weights of bins 2 tid and 2 tid + 1 of the whole row; every thread of a workgroup calls it.
__device__ __forceinline__ RowCut find_cut(const RowRule &r, int V, const uint64_t (&count)[2], const uint64_t (&mass)[2])
{
    const int tid = threadIdx.x;
    __shared__ int k_bin, above_k, p_first, p_last;
    __shared__ unsigned long long k_low, k_high;
    uint64_t to[2] = {count[0] + count[1], mass[0] + mass[1]}, all[2];
    if (tid == 0) k_bin = kNoBin, above_k = 0, p_first = kNoBin, p_last = -1;
    scan_block(to, all);
    const uint64_t count_to[2] = {to[0] - count[1], to[0]}, mass_to[2] = {to[1] - mass[1], to[1]};
    const bool limited_k = r.k && (uint64_t)r.k < all[0];   // uniform
    if (limited_k) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (count_to[e] >= (uint64_t)r.k && count_to[e] - count[e] < (uint64_t)r.k) {   // one bin of all
                k_bin = 2 * tid + e;
                above_k = (int)(count_to[e] - count[e]);
                k_low = mass_to[e] - mass[e];
                k_high = mass_to[e];
            }
        __syncthreads();
    }
    if (r.p < 1.0) {
        // The weights here are off by less than 2^-17 of each (an fp32 exponent of up to 45 with three roundings) and by V 2^-32 in all: the true border lies between
        // `low` and `high`, and so in the bins that reach over one and begin below the other
        const double slack = (double)V * 0.5 + 1.0;   // in units of 2^-31
        const double low = r.p * (double)(limited_k ? k_low : all[1]) * (1.0 - 0x1p-16) - slack;
        const double high = r.p * (double)(limited_k ? k_high : all[1]) * (1.0 + 0x1p-16) + slack;
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (count[e] != 0 && 2 * tid + e <= k_bin) {
                const bool top = count_to[e] == count[e], bottom = count_to[e] == all[0] || 2 * tid + e == k_bin;
                const double from = (double)(mass_to[e] - mass[e]), until = (double)mass_to[e];
                auto reaches = [&](double t) { return t * (1.0 + 0x1p-16) + slack >= low; };
                auto begins = [&](double t) { return t * (1.0 - 0x1p-16) - slack < high; };
                // the first bin that reaches over `low` begins where the one before, which does not, ends; likewise the last: few come here
                if (reaches(until) && (top || !reaches(from))) atomicMin(&p_first, 2 * tid + e);
                if ((top || begins(from)) && (bottom || !begins(until))) atomicMax(&p_last, 2 * tid + e);
            }
    } else if (tid == 0) {
        p_first = p_last = k_bin;   // kNoBin: the row has fewer tokens than its limit, and nothing is cut
    }
    __syncthreads();
    return {p_first, p_last, k_bin, above_k};
}

// Rows without a limit of this kind leave at once, and so does a row's every workgroup.
__global__ __launch_bounds__(kSampleThreads) void sample_bins_kernel(const SampleArgs a)
{
    const int tid = threadIdx.x, m = blockIdx.y;
    const float *x = a.logits + (size_t)m * a.V;
    __shared__ unsigned long long bins[kBins];
    float v[kPer];
    auto fetch = [&](int chunk) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int i = chunk * kChunk + e * kSampleThreads + tid;
            v[e] = i < a.V ? x[i] : -__builtin_inff();
        }
    };
    int chunk = blockIdx.x * a.bin_chunks;
    const int chunks_end = min(chunk + a.bin_chunks, a.chunks);
    fetch(chunk);
    const RowParams params = row_params(a, m);
    const ChunkTop row = row_top(a, m);
    const RowRule r = row_rule(params, a.V, row);
    if (token_of(row) == kNoToken || r.greedy || !r.limited()) return;   // uniform over the row
    for (int b = tid; b < kBins; b += kSampleThreads) bins[b] = 0;
    __syncthreads();
    const float per_octave = r.per_octave();
    while (true) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const float d = r.depth(v[e]);
            if (d < r.deepest) into_bins(bins, r, d, per_octave);
        }
        if (++chunk >= chunks_end) break;   // uniform
        fetch(chunk);
    }
    __syncthreads();
    // two neighbouring bins per thread, here and below
    static_assert(kBins == 2 * kSampleThreads, "two bins per thread");
    typedef float float4v __attribute__((ext_vector_type(4)));
    typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
    const PartialBuffer rows = partial_buffer(reinterpret_cast<const float *>(a.bins + (size_t)m * a.bin_groups * kBins));
    store_partial(rows, blockIdx.x * (kBins / 2) + tid, __builtin_bit_cast(float4v, (u64x2){bins[2 * tid], bins[2 * tid + 1]}));
    if (!last_of_row(a.tickets + m, a.bin_groups)) return;
    // counts and weights of the whole row, and their sums up to each bin
    uint64_t count[2] = {0, 0}, mass[2] = {0, 0};
    constexpr int kTogether = 16;   // groups whose loads are under way together
    for (int c0 = 0; c0 < a.bin_groups; c0 += kTogether) {
        u64x2 n[kTogether];
#pragma unroll
        for (int c = 0; c < kTogether; ++c) n[c] = __builtin_bit_cast(u64x2, load_partial(rows, min(c0 + c, a.bin_groups - 1) * (kBins / 2) + tid));
#pragma unroll
        for (int c = 0; c < kTogether; ++c)
            if (c0 + c < a.bin_groups) {   // uniform
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    count[e] += n[c][e] >> 48;
                    mass[e] += n[c][e] & ((1ull << 48) - 1);
                }
            }
    }
    const RowCut cut = find_cut(r, a.V, count, mass);
    if (tid == 0) a.cuts[m] = cut;
}

// Cuts a row by digits of its logits, for lists that are too long; every thread of one workgroup calls it.  by_mass: the last token with less than
// `limit` of weight before it; otherwise the limit-th token (there are more).  Returns the order of the cut's last token; kept: the weight down to it.
struct DigitBins {
    unsigned long long mass[256];
    uint32_t count[256];
    unsigned long long above;
    uint32_t prefix, cut_at;
    int64_t left;
};
__device__ __attribute__((noinline)) uint64_t cut_by_digits(const float *x, int V, const RowRule &r, bool by_mass, double limit, DigitBins &sh, uint64_t &kept)
{
    const int tid = threadIdx.x;
    uint32_t prefix = 0, known = 0;
    uint64_t above = 0;      // weight of the tokens above the prefix
    int64_t left = by_mass ? 0 : (int64_t)limit;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int d = tid; d < 256; d += kSampleThreads) sh.mass[d] = 0, sh.count[d] = 0;
        __syncthreads();
        for (int i = tid; i < V; i += kSampleThreads) {
            const float v = x[i];
            const uint32_t key = order_key(v);
            if ((key & known) != prefix || !(r.depth(v) < r.deepest)) continue;
            const int d = (key >> shift) & 255;
            atomicAdd(&sh.count[d], 1u);
            atomicAdd(&sh.mass[d], (unsigned long long)units(exp_minus(r.below(v))));
        }
        __syncthreads();
        if (tid == 0) {
            int cut = -1;
            uint64_t before = above, cut_above = above;
            int64_t need = left;
            for (int d = 255; d >= 0; --d) {
                if (sh.count[d] == 0) continue;
                if (cut >= 0 && (by_mass ? !((double)before < limit) : need <= 0)) break;
                cut = d;
                cut_above = before;
                before += sh.mass[d];
                if (!by_mass) need -= sh.count[d];
            }
            if (!by_mass) need += sh.count[cut];
            if (shift == 0) {   // tokens of one logit
                const int64_t n = sh.count[cut];
                const uint64_t w = sh.mass[cut] / n;
                if (by_mass) need = (int64_t)ceil(fmin((limit - (double)cut_above) / (double)w, (double)n));
                need = need < 1 ? 1 : need > n ? n : need;
                cut_above += (uint64_t)need * w;
            }
            sh.prefix = prefix | ((uint32_t)cut << shift);
            sh.above = cut_above;
            sh.left = need;
        }
        __syncthreads();
        prefix = sh.prefix;
        above = sh.above;
        left = sh.left;
        known |= 255u << shift;
        __syncthreads();
    }
    // the index of the left-th token of that logit
    const float cut = order_number(prefix);
    uint64_t seen = 0;
    for (int b = 0; b < V; b += kSampleThreads) {
        const int i = b + tid;
        const bool tie = i < V && x[i] == cut;
        uint64_t to[1] = {tie ? 1u : 0u}, here[1];
        scan_block(to, here);
        if (tie && seen + to[0] == (uint64_t)left) sh.cut_at = (uint32_t)i;
        seen += here[0];
        if (seen >= (uint64_t)left) break;   // uniform
    }
    __syncthreads();
    kept = above;
    return order_of(cut, (int)sh.cut_at);
}

// Sorts the n > 0 entries of a list into falling order; every thread of the workgroup calls it, behind a barrier.  Counting sort by even
// stretches of the distance, then each entry by the greater ones of its stretch: 14 us fewer than by the greater ones of 600 entries, 60 barriers
// fewer than a bitonic sort.  A stretch with many entries (equal logits) makes it bitonic all the same.
constexpr int kStretches = 1024, kStretchMost = 64;
// What only the row's last workgroup holds in LDS: it lies where the segments' logits were
struct TailLds {
    unsigned long long upto[kList];
    uint32_t from[kStretches + 1], most;
    DigitBins digits;
};
__device__ __forceinline__ void sort_list(unsigned long long *list, TailLds &sh, uint32_t n, const RowRule &r, const RowCut &cut)
{
    const int tid = threadIdx.x;
    unsigned long long *const other = sh.upto;
    uint32_t *const from = sh.from;
    uint32_t &most = sh.most;
    constexpr int kEach = kList / kSampleThreads;
    const int low_bin = min(cut.first, cut.k_bin), high_bin = cut.k_bin == kNoBin ? cut.last : max(cut.last, cut.k_bin);
    const float per = (float)kStretches / (float)(high_bin - low_bin + 1);
    auto stretch = [&](uint64_t o) {   // rises with the distance, equal for equal logits
        const float b = r.depth(order_number((uint32_t)(o >> 32))) * r.bins_per - (float)low_bin;
        return (int)fminf(fmaxf(b * per, 0.f), (float)(kStretches - 1));
    };
    static_assert(kStretches == 2 * kSampleThreads, "two stretches per thread");
    from[2 * tid] = from[2 * tid + 1] = 0;
    if (tid == 0) most = 0;
    __syncthreads();
    uint64_t own[kEach];
    uint32_t at[kEach], slot[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint32_t i = tid + e * kSampleThreads;
        own[e] = i < n ? list[i] : 0;
        at[e] = slot[e] = 0;
        if (i < n) {
            at[e] = (uint32_t)stretch(own[e]);
            slot[e] = atomicAdd(&from[at[e]], 1u);
            if (slot[e] >= kStretchMost) most = 1;
        }
    }
    __syncthreads();
    if (most) {   // uniform
        // A wavefront's 64 pairs of a step of at most 64 lie in 128 entries of its own, in every such step the same ones: those steps need
        // no barrier (LDS keeps a wavefront's order).
        uint32_t padded = 128;
        while (padded < n) padded <<= 1;
        for (uint32_t i = n + tid; i < padded; i += kSampleThreads) list[i] = 0;
        __syncthreads();
        for (uint32_t size = 2; size <= padded; size <<= 1) {
            if (size > 128) __syncthreads();
            for (uint32_t step = size >> 1; step > 0; step >>= 1) {
                for (uint32_t t = tid; t < padded / 2; t += kSampleThreads) {
                    const uint32_t i = 2 * t - (t & (step - 1)), j = i + step;
                    const uint64_t p = list[i], q = list[j];
                    if ((p < q) == ((i & size) == 0)) list[i] = q, list[j] = p;
                }
                if (step > 64) __syncthreads();
                else asm volatile("" ::: "memory");
            }
        }
        __syncthreads();
        return;
    }
    const uint32_t count[2] = {from[2 * tid], from[2 * tid + 1]};
    uint64_t to[1] = {count[0] + count[1]}, all[1];
    scan_block(to, all);
    from[2 * tid] = (uint32_t)to[0] - count[1] - count[0];
    from[2 * tid + 1] = (uint32_t)to[0] - count[1];
    if (tid == 0) from[kStretches] = n;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e)
        if (tid + e * kSampleThreads < n) other[from[at[e]] + slot[e]] = own[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e)
        if (tid + e * kSampleThreads < n) {
            const uint32_t begin = from[at[e]], end = from[at[e] + 1];
            uint32_t place = begin;
            for (uint32_t i = begin; i < end; ++i) place += other[i] > own[e];
            list[place] = own[e];
        }
    __syncthreads();
}

__device__ __forceinline__ void number_to_lds(const float *src, float *lds_base)   // lane l's number at src lands at lds_base[l] (wavefront-uniform)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src, (__attribute__((address_space(3))) void *)lds_base, 4, 0, 0);
}

constexpr int kEarlyLds = kSampleWaves * 2 * kSegment * 4;   // two segments of each wavefront
constexpr int kSteps = kSegment / 64;
// One segment by one wavefront, its logits in LDS, i0 the index of the lane's first: what stays for certain and is not below min_p (the sum in lane 63), and,
// per lane, all above the first border bin and all between the border bins and the k-th token's; tokens in border bins go to the list.
__device__ __forceinline__ uint64_t weigh_segment(const float *segment, int i0, int V, const RowRule &r, const RowCut &cut, unsigned long long *list, uint32_t &listed,
                                                  uint64_t &above, uint64_t &between)
{
    const float *const here = segment + (threadIdx.x & 63);
    uint64_t kept = 0;
#pragma unroll 2
    for (int e = 0; e < kSteps; ++e) {
        const float v = here[e * 64];
        const float d = r.depth(v);
        const int b = r.bin(d);
        if (!(d < r.deepest) || i0 + e * 64 >= V || (b > cut.last && b > cut.k_bin)) continue;   // takes no part, or is beyond the limits
        if (b >= cut.first && (b <= cut.last || b == cut.k_bin)) {   // a border bin
            const uint32_t n = atomicAdd(&listed, 1u);
            if (n < kList) list[n] = order_of(v, i0 + e * 64);
        } else {
            const double w = exp_minus(r.below(v));
            const uint64_t n = units(w);
            above += b < cut.first ? n : 0;
            between += b < cut.first ? 0 : n;
            kept += b < cut.first && w >= r.min_w ? n : 0;
        }
    }
    return scan_wave(kept);
}

// The exact cut, then the draw, by one workgroup: list holds the row's n tokens in border bins (in any order; nothing if they are more than kList),
// segment_mass what stays for certain of each segment.
__device__ __forceinline__ void finish_row(const SampleArgs &a, int m, const RowRule &r, const RowCut &cut, unsigned long long *list, uint32_t n, uint64_t all_above,
                                           uint64_t all_between, unsigned long long *segment_mass, TailLds &tail)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V;
    const float *x = a.logits + (size_t)m * V;
    uint64_t cut_order = 0;   // tokens of this order and earlier ones stay
    if (n > kList) {
        DigitBins &digits = tail.digits;
        uint64_t weight;
        if (cut.k_bin != kNoBin) {
            cut_order = cut_by_digits(x, V, r, false, (double)r.k, digits, weight);
        } else {   // the list's share of the row is not known: once more from the logits
            uint64_t part[1] = {0}, total[1];
            for (int i = tid; i < V; i += kSampleThreads) {
                const float v = x[i];
                if (r.depth(v) < r.deepest) part[0] += units(exp_minus(r.below(v)));
            }
            scan_block(part, total);
            weight = total[0];
        }
        if (r.p < 1.0) cut_order = cut_by_digits(x, V, r, true, r.p * (double)weight, digits, weight);
        __syncthreads();
        segment_mass[tid] = 0;
        __syncthreads();
        for (int c = 0; c < a.segments; ++c) {
            const int i = c * kSegment + tid;
            const float v = i < V ? x[i] : -__builtin_inff();
            const double w = r.depth(v) < r.deepest && order_of(v, i) >= cut_order ? exp_minus(r.below(v)) : 0.0;
            const uint64_t part = scan_wave(w >= r.min_w ? units(w) : 0);
            if (lane == 63) atomicAdd(&segment_mass[c], (unsigned long long)part);
        }
        __syncthreads();
    } else if (n > 0) {
        __shared__ uint32_t to_k_bin, staying;
        if (tid == 0) to_k_bin = 0, staying = 0;
        __syncthreads();
        auto logit_of = [&](uint64_t o) { return order_number((uint32_t)(o >> 32)); };
        const bool apart = cut.k_bin > cut.last;   // tokens between the border bins and the k-th token's come before the latter
        auto allowed_by_k = [&](uint32_t above_k_bin) { return cut.k_bin == kNoBin ? n : above_k_bin + (uint32_t)(r.k - cut.above_k); };   // one at least
        auto stays_at = [&](uint64_t ahead, double limit) { return r.p >= 1.0 || (double)ahead < limit || ahead == 0; };   // holds for a first stretch of the list
        if (n <= 64) {
            // One entry per lane, in every wavefront alike: an entry's place and the weight ahead of it are sums over the greater ones.  No sorting and one
            // barrier: 1.5 to 2 us less than the way below, which longer lists take.
            const uint64_t o = (uint32_t)lane < n ? list[lane] : 0;
            const float x_o = logit_of(o);
            const double w_o = (uint32_t)lane < n ? exp_minus(r.below(x_o)) : 0.0;
            const uint64_t own = units(w_o);
            uint32_t place = 0;
            uint64_t ahead = all_above;
            for (uint32_t q = 0; q < n; ++q) {   // uniform
                const bool greater = of_lane(o, q) > o;
                place += greater;
                ahead += greater ? of_lane(own, q) : 0;
            }
            const uint32_t above_k_bin = (uint32_t)__popcll(__ballot((uint32_t)lane < n && r.bin(r.depth(x_o)) < cut.k_bin)), allowed = allowed_by_k(above_k_bin);
            const bool in_k = (uint32_t)lane < n && place < allowed;
            const double limit = r.p * (double)(all_above + all_between + of_lane(scan_wave(in_k ? own : 0), 63));
            if (apart && place >= above_k_bin) ahead += all_between;
            const bool stays = in_k && stays_at(ahead, limit);
            cut_order = __any(stays) ? ~max_wave(stays ? ~o : 0) : max_wave(o) + 1;
            if (wave == 0 && stays && (r.min_w == 0.0 || w_o >= r.min_w)) atomicAdd(&segment_mass[~(uint32_t)o / kSegment], (unsigned long long)own);
            __syncthreads();
        } else {
            unsigned long long *const upto = tail.upto;
            sort_list(list, tail, n, r, cut);
            // weights down the list; its places where something ends are found by the entry ahead of them
            auto logit = [&](uint32_t i) { return logit_of(list[i]); };
            auto bin_at = [&](uint32_t i) { return r.bin(r.depth(logit(i))); };
            uint64_t so_far = 0;
#pragma unroll 1
            for (uint32_t i0 = 0; i0 < n; i0 += kSampleThreads) {
                const uint32_t i = i0 + tid;
                uint64_t to[1] = {0}, all[1];
                if (i < n) {
                    to[0] = units(exp_minus(r.below(logit(i))));
                    if (bin_at(i) < cut.k_bin && (i + 1 == n || bin_at(i + 1) >= cut.k_bin)) to_k_bin = i + 1;   // one entry of all, or none
                }
                scan_block(to, all);
                if (i < n) upto[i] = so_far + to[0];
                so_far += all[0];
            }
            __syncthreads();
            const uint32_t above_k_bin = to_k_bin;
            const uint32_t allowed = allowed_by_k(above_k_bin);
            const double limit = r.p * (double)(all_above + all_between + upto[allowed - 1]);
            auto stays = [&](uint32_t i) {
                if (i >= allowed) return false;
                const uint64_t ahead = all_above + (i ? upto[i - 1] : 0) + (apart && i >= above_k_bin ? all_between : 0);
                return stays_at(ahead, limit);
            };
#pragma unroll 1
            for (uint32_t i = tid; i < n; i += kSampleThreads)
                if (stays(i) && !stays(i + 1)) staying = i + 1;   // one entry of all, or none
            __syncthreads();
            const uint32_t stay = staying;
            cut_order = stay ? list[stay - 1] : list[0] + 1;
#pragma unroll 1
            for (uint32_t i = tid; i < stay; i += kSampleThreads)
                if (r.min_w == 0.0 || exp_minus(r.below(logit(i))) >= r.min_w)
                    atomicAdd(&segment_mass[(~(uint32_t)list[i]) / kSegment], (unsigned long long)(upto[i] - (i ? upto[i - 1] : 0)));
            __syncthreads();
        }
    } else {
        __syncthreads();
    }
    // the segment, then the token
    static_assert(kSegments == kSampleThreads && kSegment == kSampleThreads, "a thread per segment, and per token of one");
    __shared__ uint64_t chosen_rank;
    __shared__ int chosen;
    uint64_t mass[1] = {segment_mass[tid]}, total[1], all[1];
    const uint64_t own = mass[0];
    scan_block(mass, total);
    const uint64_t rank = drawn_rank(r.u, total[0]);   // below the total: one thread finds it in its segment
    if (mass[0] > rank && mass[0] - own <= rank) chosen = tid, chosen_rank = rank - (mass[0] - own);
    __syncthreads();
    const int i = chosen * kSegment + tid;
    const float v = i < V ? x[i] : -__builtin_inff();
    double w = r.depth(v) < r.deepest && order_of(v, i) >= cut_order ? exp_minus(r.below(v)) : 0.0;
    if (w < r.min_w) w = 0.0;
    uint64_t to[1] = {units(w)};
    const uint64_t here = to[0];
    scan_block(to, all);
    if (to[0] > chosen_rank && to[0] - here <= chosen_rank) {
        a.token[m] = i;
        a.prob[m] = (float)(w * kOne / (double)total[0]);
    }
}

// A wavefront takes segments of 512 tokens, `rounds` of them; their logits come straight to LDS, two segments ahead, and are looked at in loops that are
// hardly unrolled: code that runs once is fetched from memory, and unrolled over 16 tokens it took 2 us longer than the work.  (LDS of a size given at
// the launch: before a read of an array that is declared with its size the compiler waits for every transfer under way.)
__global__ __launch_bounds__(kSampleThreads) void sample_draw_kernel(const SampleArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, m = blockIdx.y, V = a.V;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float *x = a.logits + (size_t)m * V;
    __shared__ unsigned long long list[kList];
    extern __shared__ float4 early[];   // kEarlyLds bytes
    static_assert(sizeof(TailLds) <= kEarlyLds, "the tail's LDS lies where the segments were");
    TailLds &tail = *reinterpret_cast<TailLds *>(early);
    __shared__ unsigned long long sums[2];
    __shared__ uint32_t listed;
    float *const mine = reinterpret_cast<float *>(early) + wave * 2 * kSegment;
    const int segment0 = blockIdx.x * kSampleWaves * a.rounds + wave;
    const int rounds = min(a.rounds, (a.segments - segment0 + kSampleWaves - 1) / kSampleWaves);   // not above 0: none
    auto request = [&](int round) {
        const int i0 = (segment0 + round * kSampleWaves) * kSegment + lane;
#pragma unroll
        for (int e = 0; e < kSteps; ++e) number_to_lds(x + min(i0 + e * 64, V - 1), mine + (round & 1) * kSegment + e * 64);
    };
    if (rounds > 0) request(0);
    if (rounds > 1) request(1);
    RowCut cut = {kNoBin, kNoBin, kNoBin, 0};
    if (a.top_k || a.top_p) cut = a.cuts[m];   // of use where sample_bins_kernel has written it
    const RowParams params = row_params(a, m);
    const ChunkTop row = row_top(a, m);
    const RowRule r = row_rule(params, V, row);
    if (token_of(row) == kNoToken || r.greedy) {   // uniform over the row
        if (blockIdx.x == 0 && tid == 0) {
            a.token[m] = token_of(row);
            a.prob[m] = token_of(row) == kNoToken ? 0.f : 1.f;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing may land in LDS that has been given to others
        return;
    }
    if (!r.limited()) cut = {kNoBin, kNoBin, kNoBin, 0};   // uniform over the row
    if (tid == 0) listed = 0, sums[0] = sums[1] = 0;
    fill_roots();
    __syncthreads();
    unsigned long long *const row_kept = a.kept + (size_t)m * a.segments;
    uint64_t above = 0, between = 0;
#pragma unroll 1
    for (int round = 0; round < rounds; ++round) {
        const int segment = segment0 + round * kSampleWaves, i0 = segment * kSegment + lane;
        if (round + 1 < rounds) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");   // the next segment may be under way
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const uint64_t kept = weigh_segment(mine + (round & 1) * kSegment, i0, V, r, cut, list, listed, above, between);
        if (round + 2 < rounds) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this segment has been read
            request(round + 2);
        }
        if (lane == 63) store_shared(row_kept + segment, kept);
    }
    above = scan_wave(above);
    between = scan_wave(between);
    if (lane == 63) {
        atomicAdd(&sums[0], (unsigned long long)above);
        atomicAdd(&sums[1], (unsigned long long)between);
    }
    __syncthreads();
    GroupMass *const masses = a.masses + m * a.groups;
    unsigned long long *const lists = a.lists + (size_t)m * a.groups * kList;
    if (tid < 2) store_shared(&masses[blockIdx.x].above + tid, sums[tid]);
    if (tid == 2) store_shared(&masses[blockIdx.x].listed, listed);
    for (uint32_t n = tid; n < min(listed, (uint32_t)kList); n += kSampleThreads) store_shared(lists + (size_t)blockIdx.x * kList + n, list[n]);
    if (!last_of_row(a.tickets + gridDim.y + m, a.groups)) return;

    // ---- the row's last workgroup: the exact cut, then the draw
    // Every wavefront fetches what the groups found (lane = group), and, not knowing their counts yet, the first 64 entries of the lists that it
    // will gather: groups wave, wave + 8, ...
    __shared__ unsigned long long segment_mass[kSegments];
    GroupMass found = {0, 0, 0, 0};
    if (lane < a.groups) {
        found.above = load_shared(&masses[lane].above);
        found.between = load_shared(&masses[lane].between);
        found.listed = load_shared(&masses[lane].listed);
    }
    const uint64_t own_kept = tid < a.segments ? load_shared(row_kept + tid) : 0;
    constexpr int kParts = kGroups / kSampleWaves;
    uint64_t entry[kParts];
#pragma unroll
    for (int q = 0; q < kParts; ++q) entry[q] = load_shared(lists + (size_t)min(wave + q * kSampleWaves, a.groups - 1) * kList + lane);
    segment_mass[tid] = own_kept;
    const uint64_t listed_to = scan_wave(found.listed);
    const uint64_t all_above = of_lane(scan_wave(found.above), 63), all_between = of_lane(scan_wave(found.between), 63);
    const uint32_t n = (uint32_t)of_lane(listed_to, 63);
    if (n <= kList) {
#pragma unroll
        for (int q = 0; q < kParts; ++q) {
            const int c = wave + q * kSampleWaves;
            if (c >= a.groups) break;   // uniform over the wavefront
            const uint32_t count = (uint32_t)of_lane(found.listed, c), base = (uint32_t)of_lane(listed_to, c) - count;
            if ((uint32_t)lane < count) list[base + lane] = entry[q];
            for (uint32_t i = 64 + lane; i < count; i += 64) list[base + i] = load_shared(lists + (size_t)c * kList + i);
        }
    }
    finish_row(a, m, r, cut, list, n, all_above, all_between, segment_mass, tail);
}

// Tokens of a row that one workgroup takes.  Measured against the three kernels above, us (1 row of 1000 tokens, top-k and top-p: 10.8 and 18.7):
//   tokens          top-k        top-p        none
//    8192, 1 row    13.5  19.9   15.4  21.2   10.5  12.0
//   12000, 1 row    16.4  20.5   19.5  21.1   13.7  12.2
//   12000, 60 rows  18.1  22.6   23.1  26.0   14.4  13.7
//   16384, 1 row    19.0  20.5   23.7  22.1   16.7  12.4
constexpr int kRowMost = 12288, kRowMostUnlimited = 8192;
__host__ __device__ constexpr int row_rounds(int segments) { return segments <= 2 * kSampleWaves ? 2 : (segments + kSampleWaves - 1) / kSampleWaves; }   // of a wavefront
constexpr int row_lds(int segments) { return kSampleWaves * row_rounds(segments) * kSegment * 4; }
static_assert(row_lds(1) >= (int)sizeof(TailLds), "the tail's LDS lies where the segments were");
// Short rows, a workgroup each: everything from one reading of the logits, which stay in LDS.
__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(const SampleArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, m = blockIdx.x, V = a.V;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float *x = a.logits + (size_t)m * V;
    __shared__ unsigned long long list[kList], bins[kBins], segment_mass[kSegments];
    extern __shared__ float4 early[];   // row_lds bytes
    TailLds &tail = *reinterpret_cast<TailLds *>(early);
    __shared__ ChunkTop of_wave[kSampleWaves];
    __shared__ unsigned long long sums[2];
    __shared__ uint32_t listed;
    const int rounds = (a.segments - wave + kSampleWaves - 1) / kSampleWaves;   // not above 0: none
    float *const mine = reinterpret_cast<float *>(early) + wave * row_rounds(a.segments) * kSegment;
    for (int round = 0; round < rounds; ++round) {
        const int i0 = (wave + round * kSampleWaves) * kSegment + lane;
#pragma unroll
        for (int e = 0; e < kSteps; ++e) number_to_lds(x + min(i0 + e * 64, V - 1), mine + round * kSegment + e * 64);
    }
    const RowParams params = row_params(a, m);
    bins[2 * tid] = bins[2 * tid + 1] = 0;
    segment_mass[tid] = 0;
    if (tid == 0) listed = 0, sums[0] = sums[1] = 0;
    fill_roots();
    float top = -__builtin_inff(), least = __builtin_inff();
    int at = kNoToken;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    auto each = [&](auto &&use) {   // logits of this wavefront, with their indices
        for (int round = 0; round < rounds; ++round) {
            const int i0 = (wave + round * kSampleWaves) * kSegment + lane;
#pragma unroll 4
            for (int e = 0; e < kSteps; ++e)
                if (i0 + e * 64 < V) use(mine[round * kSegment + e * 64 + lane], i0 + e * 64);
        }
    };
    each([&](float v, int i) {   // NaN and -inf are no tokens
        if (v > top) top = v, at = i;
        if (v > -__builtin_inff()) least = fminf(least, v);
    });
    const ChunkTop own = join_lanes(chunk_top(top, at, least));
    if (lane == 0) of_wave[wave] = own;
    __syncthreads();
    const ChunkTop row = join_lanes(of_wave[lane & (kSampleWaves - 1)]);
    const RowRule r = row_rule(params, V, row);
    if (token_of(row) == kNoToken || r.greedy) {   // uniform
        if (tid == 0) {
            a.token[m] = token_of(row);
            a.prob[m] = token_of(row) == kNoToken ? 0.f : 1.f;
        }
        return;
    }
    RowCut cut = {kNoBin, kNoBin, kNoBin, 0};
    if (r.limited()) {   // uniform
        const float per_octave = r.per_octave();
        each([&](float v, int) {
            const float d = r.depth(v);
            if (d < r.deepest) into_bins(bins, r, d, per_octave);
        });
        __syncthreads();
        const unsigned long long n[2] = {bins[2 * tid], bins[2 * tid + 1]}, weights = (1ull << 48) - 1;
        const uint64_t count[2] = {n[0] >> 48, n[1] >> 48}, mass[2] = {n[0] & weights, n[1] & weights};
        cut = find_cut(r, V, count, mass);
    }
    uint64_t above = 0, between = 0;
    for (int round = 0; round < rounds; ++round) {
        const int segment = wave + round * kSampleWaves;
        const uint64_t kept = weigh_segment(mine + round * kSegment, segment * kSegment + lane, V, r, cut, list, listed, above, between);
        if (lane == 63) segment_mass[segment] = kept;
    }
    above = scan_wave(above);
    between = scan_wave(between);
    if (lane == 63) {
        atomicAdd(&sums[0], (unsigned long long)above);
        atomicAdd(&sums[1], (unsigned long long)between);
    }
    __syncthreads();   // the segments have been read as well
    finish_row(a, m, r, cut, list, listed, sums[0], sums[1], segment_mass, tail);
}

}  // namespace w4

using namespace w4;

extern "C" {

// How a call's rows are split: about 512 workgroups at most, two per CU at work together.  More would wait for the first ones, in each of
// which a few us pass before the first logit is looked at: with 384, 512, 768 and 1024, 60 rows of 128256 tokens take 42.8, 40.7, 42.7 and 48 us with all
// limits, 56, 51.6, 52.7 and 55.8 with top-p, 30 rows 33.4, 34.6, 34.6 and 40.7.
constexpr int kMost = 512;
static_assert((kChunks * W4A16_MAX_M + kMost - 1) / kMost * kChunk < 1 << 16, "a bin counts the tokens of a group in 16 bits");
static void sample_split(int M, int V, SampleArgs &a)
{
    a.V = V;
    a.chunks = (V + kChunk - 1) / kChunk;
    a.segments = (V + kSegment - 1) / kSegment;
    a.bin_chunks = (M * a.chunks + kMost - 1) / kMost;
    a.bin_groups = (a.chunks + a.bin_chunks - 1) / a.bin_chunks;
    const int smallest = (a.segments + kSampleWaves - 1) / kSampleWaves;   // groups, at one segment per wavefront; 64 at most
    a.rounds = (M * smallest + kMost - 1) / kMost;
    a.groups = (smallest + a.rounds - 1) / a.rounds;
}

// tickets | tops | cuts | group masses | segment masses | bins | lists
constexpr int kSampleParts = 7;
static size_t sample_layout(int M, const SampleArgs &a, size_t (&at)[kSampleParts])
{
    // M groups of a call are fewer than kMost + M: taken as that, so that what serves a call serves all smaller ones
    const size_t rows = (size_t)M, most = kMost + W4A16_MAX_M, smallest = (a.segments + kSampleWaves - 1) / kSampleWaves;
    const size_t groups = rows * smallest < most ? rows * smallest : most, bin_groups = rows * a.chunks < most ? rows * a.chunks : most;
    const size_t sizes[kSampleParts] = {kTicketBytes, rows * a.chunks * sizeof(ChunkTop), rows * sizeof(RowCut), groups * sizeof(GroupMass),
                                        rows * a.segments * 8, bin_groups * kBins * 8, groups * kList * 8};
    size_t end = 0;
    for (int i = 0; i < kSampleParts; ++i) {
        at[i] = end;
        end += (sizes[i] + 255) & ~(size_t)255;   // workgroups exchange through these: no line belongs to two
    }
    return end;
}

size_t lm_head_sample_workspace_bytes(int M, int V)
{
    if (M < 1 || M > W4A16_MAX_M || V < 1 || V > kChunks * kChunk) return 0;
    SampleArgs a;
    size_t at[kSampleParts];
    sample_split(M, V, a);
    return sample_layout(M, a, at);
}

int lm_head_sample(const float *logits, int M, int V, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                   const float *uniform, int32_t *token, float *prob, void *workspace, size_t workspace_bytes, void *stream)
{
    if (M < 1 || V < 1) return W4A16_EINVAL;
    if (M > W4A16_MAX_M || V > kChunks * kChunk) return W4A16_EUNSUP;
    if (!logits || !uniform || !token || !prob) return W4A16_ENULL;
    if (misaligned(logits) || workspace_misaligned(workspace)) return W4A16_EALIGN;
    if ((reinterpret_cast<uintptr_t>(temperature) | reinterpret_cast<uintptr_t>(top_k) | reinterpret_cast<uintptr_t>(top_p) |
         reinterpret_cast<uintptr_t>(min_p) | reinterpret_cast<uintptr_t>(uniform) | reinterpret_cast<uintptr_t>(token) |
         reinterpret_cast<uintptr_t>(prob)) & 3u)
        return W4A16_EALIGN;
    SampleArgs a;
    size_t at[kSampleParts];
    sample_split(M, V, a);
    if (!workspace || workspace_bytes < sample_layout(M, a, at)) return W4A16_EWORKSPACE;
    uint8_t *ws = reinterpret_cast<uint8_t *>(workspace);
    a.logits = logits;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.uniform = uniform;
    a.token = token;
    a.prob = prob;
    a.tickets = (uint32_t *)ws;
    a.tops = (ChunkTop *)(ws + at[1]);
    a.cuts = (RowCut *)(ws + at[2]);
    a.masses = (GroupMass *)(ws + at[3]);
    a.kept = (unsigned long long *)(ws + at[4]);
    a.bins = (unsigned long long *)(ws + at[5]);
    a.lists = (unsigned long long *)(ws + at[6]);
    const auto grid = [M](int groups) { return dim3((unsigned)groups, (unsigned)M); };
    if (V <= (top_k || top_p ? kRowMost : kRowMostUnlimited)) {
        static bool lds_ok = false;   // LDS above 48 KB needs an opt-in, once
        if (!lds_ok && hipFuncSetAttribute(reinterpret_cast<const void *>(sample_row_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, row_lds(kRowMost / kSegment)) != hipSuccess)
            return W4A16_EHIP;
        lds_ok = true;
        hipLaunchKernelGGL(sample_row_kernel, dim3((unsigned)M), dim3(kSampleThreads), row_lds(a.segments), (hipStream_t)stream, a);
        return launch_status();
    }
    hipLaunchKernelGGL(sample_top_kernel, grid(a.chunks), dim3(kSampleThreads), 0, (hipStream_t)stream, a);
    if (top_k || top_p) hipLaunchKernelGGL(sample_bins_kernel, grid(a.bin_groups), dim3(kSampleThreads), 0, (hipStream_t)stream, a);
    hipLaunchKernelGGL(sample_draw_kernel, grid(a.groups), dim3(kSampleThreads), kEarlyLds, (hipStream_t)stream, a);
    return launch_status();
}

}  // extern "C"
