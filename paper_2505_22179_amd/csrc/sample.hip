// lm_head_sample: next tokens from logits and given uniform numbers, with temperature, top-k, top-p and min-p.  Contract in
// include/w4a16.h.
//
// A token's weight is w = exp((x - max) / T), evaluated in fp64 and held as a whole number of 2^-44: sums of whole numbers do not depend
// on their order, so any split of a row gives the same token, and a border (a cumulative weight against p, or against u) is off by 1e-11
// of the row's total where sums in fp32 would be off by 1e-5 -- tokens near a border would change with the split.  Tokens more than e^31 below the
// row's largest weigh nothing (262144 of them 1e-8 of the total at most) and take part in nothing.
//
// Three kernels, each over chunks of kChunk tokens of every row, pass over the logits once:
//   sample_top_kernel    the chunks' largest logit, its token, and their smallest number
//   sample_bins_kernel   counts and weights (fp32 is enough here) in kBins bins of even width in (max - x) / T; the row's last workgroup finds the
//                        few bins in which the limits of top-k and top-p fall, whatever the rounding.  Not launched without such limits.
//   sample_draw_kernel   exact weight of what certainly stays, chunk by chunk, and a list of the tokens in those few bins; the row's last
//                        workgroup sorts the list, which gives the exact cut, draws the chunk and then the token inside it
// A list of more than kList tokens (thousands of nearly equal logits) is given up: the last workgroup then finds the cut by digits of the logits.
#include "internal.h"

namespace w4 {

constexpr int kSampleThreads = 512, kSampleWaves = kSampleThreads / 64;
constexpr int kPer = 16;                                 // tokens of a chunk per thread
constexpr int kChunk = kSampleThreads * kPer;
constexpr int kChunks = 262144 / kChunk;                 // of the largest vocabulary
constexpr int kBins = 1024;
constexpr int kList = 4096;
constexpr double kFarthest = 31.0;
constexpr double kOne = 17592186044416.0;                // 2^44: weight 1
constexpr int32_t kNoToken = 0x7FFFFFFF;
constexpr int kNoBin = kBins;

// exp(-y) for 0 <= y < 32: 2^-n times the Taylor series of exp at |f| <= ln 2 / 2 up to f^12 (remainder 2e-16)
__device__ __forceinline__ double exp_minus(double y)
{
    const double t = y * 1.4426950408889634074;
    const double n = rint(t);
    const double f = (n - t) * 0.69314718055994530942;
    double r = 1.0 / 479001600.0;
    r = fma(r, f, 1.0 / 39916800.0);
    r = fma(r, f, 1.0 / 3628800.0);
    r = fma(r, f, 1.0 / 362880.0);
    r = fma(r, f, 1.0 / 40320.0);
    r = fma(r, f, 1.0 / 5040.0);
    r = fma(r, f, 1.0 / 720.0);
    r = fma(r, f, 1.0 / 120.0);
    r = fma(r, f, 1.0 / 24.0);
    r = fma(r, f, 1.0 / 6.0);
    r = fma(r, f, 0.5);
    r = fma(r, f, 1.0);
    r = fma(r, f, 1.0);
    return __builtin_bit_cast(double, __builtin_bit_cast(int64_t, r) - ((int64_t)(int)n << 52));
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
    double bins_per; // bins of unit distance

    // distance below the largest logit in units of the temperature; at least kFarthest, or NaN, for what takes no part
    __device__ __forceinline__ double below(float x) const
    {
        if (x == top) return 0.0;
        return x > -__builtin_inff() ? ((double)top - (double)x) * inv_t : kFarthest;
    }
    // y < kFarthest; rises with y, equal for equal y
    __device__ __forceinline__ int bin(double y) const { return min((int)(y * bins_per), kBins - 1); }
};
__device__ __forceinline__ uint64_t units(double w) { return (uint64_t)(w * kOne + 0.5); }

struct SampleArgs {
    const float *logits;
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p, *uniform;
    int32_t *token;
    float *prob;
    int V, chunks;
    struct ChunkTop *tops;           // [M][chunks]
    unsigned long long *bins;        // [M][chunks][kBins]: count << 50 | weight in 2^-31
    struct RowCut *cuts;             // [M]
    struct ChunkMass *masses;        // [M][chunks]
    unsigned long long *list;        // [M][kList]
    uint32_t *listed;                // [M]
    uint32_t *tickets;               // [2 M]
};
struct ChunkTop { float top; int32_t at; float least; int32_t unused; };
struct ChunkMass { unsigned long long kept, above, between, unused; };   // weights: kept for certain and not below min_p; all above the first border bin; between the border bins and the k-th token's
struct RowCut { int32_t first, last, k_bin, above_k; };   // border bins of top-p (first .. last), bin of the k-th token (kNoBin: none), tokens in the bins above it

// the rule of row m and, in at, the first token of its largest logit (kNoToken: the row has no token); every lane of a wavefront calls it
__device__ __forceinline__ RowRule row_rule(const SampleArgs &a, int m, int &at)
{
    const int lane = threadIdx.x & 63;
    ChunkTop c = {-__builtin_inff(), kNoToken, __builtin_inff(), 0};
    if (lane < a.chunks) c = a.tops[m * a.chunks + lane];
#pragma unroll
    for (int off = 1; off < kChunks; off <<= 1) {
        const float v = __shfl_xor(c.top, off, 64), least = __shfl_xor(c.least, off, 64);
        const int j = __shfl_xor(c.at, off, 64);
        if (v > c.top || (v == c.top && j < c.at)) c.top = v, c.at = j;
        c.least = fminf(c.least, least);
    }
    c.top = __shfl(c.top, 0, 64);   // lanes beyond kChunks hold nothing
    c.least = __shfl(c.least, 0, 64);
    at = __shfl(c.at, 0, 64);
    RowRule r;
    const float t = a.temperature ? a.temperature[m] : 1.f;
    const int k = a.top_k ? a.top_k[m] : 0;
    const float p = a.top_p ? a.top_p[m] : 1.f, min_p = a.min_p ? a.min_p[m] : 0.f;
    r.top = c.top;
    r.greedy = !(t > 0.f) || k == 1 || p <= 0.f || min_p > 1.f;
    r.inv_t = r.greedy ? 0.0 : 1.0 / (double)t;
    r.k = k > 0 && k < a.V ? k : 0;
    r.p = p < 1.f ? (double)p : 2.0;
    r.min_w = min_p > 0.f ? (double)min_p : 0.0;
    // the bins span the distances that there are, so that they stay narrow at high temperatures
    const double span = fmin(r.below(c.least), kFarthest);
    r.bins_per = span > 0.0 ? (double)kBins / span : 0.0;
    return r;
}

// the uniform number as a rank of weight units below total
__device__ __forceinline__ uint64_t drawn_rank(const SampleArgs &a, int m, uint64_t total)
{
    const float u = a.uniform[m];
    const uint64_t r = u > 0.f ? (uint64_t)(fminf(u, 0x1.fffffep-1f) * (double)total) : 0;
    return r < total ? r : total - 1;
}

__device__ __forceinline__ uint64_t add_over_wave(uint64_t v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor((unsigned long long)v, off, 64);
    return v;
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

// inclusive sum over the workgroup's threads, in thread order; total: over all
__device__ __forceinline__ uint64_t scan_block(uint64_t v, uint64_t &total)
{
    __shared__ unsigned long long wave_sum[kSampleWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint64_t u = __shfl_up((unsigned long long)v, off, 64);
        if (lane >= off) v += u;
    }
    __syncthreads();   // an earlier call's sums have been read
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < kSampleWaves; ++w) {
        if (w < wave) v += wave_sum[w];
        total += wave_sum[w];
    }
    return v;
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
    ChunkTop c = {-__builtin_inff(), kNoToken, __builtin_inff(), 0};
#pragma unroll
    for (int e = 0; e < kPer; ++e) {   // NaN and -inf are no tokens
        if (v[e] > c.top) c.top = v[e], c.at = first + e * kSampleThreads + tid;
        if (v[e] > -__builtin_inff()) c.least = fminf(c.least, v[e]);
    }
    __shared__ ChunkTop of_wave[kSampleWaves];
    auto join = [&](const ChunkTop &o) {
        if (o.top > c.top || (o.top == c.top && o.at < c.at)) c.top = o.top, c.at = o.at;
        c.least = fminf(c.least, o.least);
    };
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) join({__shfl_xor(c.top, off, 64), __shfl_xor(c.at, off, 64), __shfl_xor(c.least, off, 64), 0});
    if (lane == 0) of_wave[tid >> 6] = c;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int w = 1; w < kSampleWaves; ++w) join(of_wave[w]);
        a.tops[m * a.chunks + blockIdx.x] = c;
        if (blockIdx.x == 0) a.listed[m] = 0;
    }
}

// Rows without a limit of this kind leave at once, and so does a row's every workgroup.
__global__ __launch_bounds__(kSampleThreads) void sample_bins_kernel(const SampleArgs a)
{
    const int tid = threadIdx.x, m = blockIdx.y, first = blockIdx.x * kChunk;
    int at;
    const RowRule r = row_rule(a, m, at);
    if (at == kNoToken || r.greedy || (r.k == 0 && r.p >= 1.0)) return;   // uniform over the row
    const float *x = a.logits + (size_t)m * a.V;
    __shared__ unsigned long long bins[kBins];
    float v[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int i = first + e * kSampleThreads + tid;
        v[e] = i < a.V ? x[i] : -__builtin_inff();
    }
    for (int b = tid; b < kBins; b += kSampleThreads) bins[b] = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const double y = r.below(v[e]);
        if (!(y < kFarthest)) continue;
        const float w = __builtin_amdgcn_exp2f((float)y * -1.44269504f);
        atomicAdd(&bins[r.bin(y)], (1ull << 50) + (unsigned long long)(uint32_t)(w * 2147483648.f + 0.5f));
    }
    __syncthreads();
    unsigned long long *rows = a.bins + (size_t)m * a.chunks * kBins;
    for (int b = tid; b < kBins; b += kSampleThreads) store_shared(rows + (size_t)blockIdx.x * kBins + b, bins[b]);
    if (!last_of_row(a.tickets + m, a.chunks)) return;
    // counts and weights of the whole row, two neighbouring bins per thread, and their sums up to each bin
    uint64_t count[2] = {0, 0}, mass[2] = {0, 0};
    for (int c = 0; c < a.chunks; ++c)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint64_t n = load_shared(rows + (size_t)c * kBins + 2 * tid + e);
            count[e] += n >> 50;
            mass[e] += n & ((1ull << 50) - 1);
        }
    uint64_t tokens, weight;
    const uint64_t counted = scan_block(count[0] + count[1], tokens), weighed = scan_block(mass[0] + mass[1], weight);
    __shared__ int k_bin, above_k, p_first, p_last;
    __shared__ unsigned long long k_low, k_high;
    if (tid == 0) k_bin = kNoBin, above_k = 0, p_first = kNoBin, p_last = -1, k_low = weight, k_high = weight;
    __syncthreads();
    const uint64_t count_to[2] = {counted - count[1], counted}, mass_to[2] = {weighed - mass[1], weighed};
    if (r.k && (uint64_t)r.k < tokens) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (count_to[e] >= (uint64_t)r.k && count_to[e] - count[e] < (uint64_t)r.k) {   // one bin of all
                k_bin = 2 * tid + e;
                above_k = (int)(count_to[e] - count[e]);
                k_low = mass_to[e] - mass[e];
                k_high = mass_to[e];
            }
    }
    __syncthreads();
    if (r.p < 1.0) {
        // The weights here are off by less than 2^-18 of each (an fp32 exponent of up to 45) and by V 2^-32 in all: the true border lies between
        // `low` and `high`, and so in the bins that reach over one and begin below the other
        const double slack = (double)a.V * 0.5 + 1.0;   // in units of 2^-31
        const double low = (r.p * (double)k_low) * (1.0 - 0x1p-16) - slack, high = (r.p * (double)k_high) * (1.0 + 0x1p-16) + slack;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int b = 2 * tid + e;
            if (count[e] == 0 || b > k_bin) continue;
            const double to = (double)mass_to[e], from = (double)(mass_to[e] - mass[e]);
            if (to * (1.0 + 0x1p-16) + slack >= low) atomicMin(&p_first, b);
            if (b == 0 || count_to[e] == count[e] || from * (1.0 - 0x1p-16) - slack < high) atomicMax(&p_last, b);
        }
        __syncthreads();
    } else if (tid == 0) {
        p_first = p_last = k_bin;   // kNoBin: the row has fewer tokens than its limit, and nothing is cut
    }
    __syncthreads();
    if (tid == 0) a.cuts[m] = {p_first, p_last, k_bin, above_k};
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
            const double y = r.below(v);
            if ((key & known) != prefix || !(y < kFarthest)) continue;
            const int d = (key >> shift) & 255;
            atomicAdd(&sh.count[d], 1u);
            atomicAdd(&sh.mass[d], (unsigned long long)units(exp_minus(y)));
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
        uint64_t here;
        const uint64_t to = seen + scan_block(tie ? 1 : 0, here);
        if (tie && to == (uint64_t)left) sh.cut_at = (uint32_t)i;
        seen += here;
        if (seen >= (uint64_t)left) break;   // uniform
    }
    __syncthreads();
    kept = above;
    return order_of(cut, (int)sh.cut_at);
}

__global__ __launch_bounds__(kSampleThreads) void sample_draw_kernel(const SampleArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, m = blockIdx.y, first = blockIdx.x * kChunk, V = a.V;
    int at;
    const RowRule r = row_rule(a, m, at);
    if (at == kNoToken || r.greedy) {   // uniform over the row
        if (blockIdx.x == 0 && tid == 0) {
            a.token[m] = at;
            a.prob[m] = at == kNoToken ? 0.f : 1.f;
        }
        return;
    }
    const float *x = a.logits + (size_t)m * V;
    __shared__ unsigned long long list[kList];
    __shared__ uint32_t listed, list_at;
    __shared__ unsigned long long sums[3];
    float v[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int i = first + e * kSampleThreads + tid;
        v[e] = i < V ? x[i] : -__builtin_inff();
    }
    RowCut cut = {kNoBin, kNoBin, kNoBin, 0};
    const bool limited = r.k != 0 || r.p < 1.0;   // uniform over the row
    if (limited) cut = a.cuts[m];
    if (tid == 0) listed = 0, sums[0] = sums[1] = sums[2] = 0;
    __syncthreads();
    uint64_t kept = 0, above = 0, between = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const double y = r.below(v[e]);
        if (!(y < kFarthest)) continue;
        const int b = r.bin(y);
        if (b < cut.first) {
            const double w = exp_minus(y);
            above += units(w);
            if (w >= r.min_w) kept += units(w);
        } else if (b <= cut.last || b == cut.k_bin) {
            const uint32_t n = atomicAdd(&listed, 1u);
            if (n < kList) list[n] = order_of(v[e], first + e * kSampleThreads + tid);
        } else if (b < cut.k_bin) {
            between += units(exp_minus(y));
        }
    }
    kept = add_over_wave(kept);
    above = add_over_wave(above);
    between = add_over_wave(between);
    if (lane == 0) {
        atomicAdd(&sums[0], (unsigned long long)kept);
        atomicAdd(&sums[1], (unsigned long long)above);
        atomicAdd(&sums[2], (unsigned long long)between);
    }
    __syncthreads();
    const uint32_t mine = listed;
    ChunkMass *masses = a.masses + m * a.chunks;
    if (tid == 0) {
        store_shared(&masses[blockIdx.x].kept, sums[0]);
        store_shared(&masses[blockIdx.x].above, sums[1]);
        store_shared(&masses[blockIdx.x].between, sums[2]);
        list_at = mine ? __hip_atomic_fetch_add(a.listed + m, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
    }
    __syncthreads();
    unsigned long long *row_list = a.list + (size_t)m * kList;
    const uint32_t base = list_at;
    for (uint32_t n = tid; n < mine && base + n < kList; n += kSampleThreads) store_shared(row_list + base + n, list[n]);
    if (!last_of_row(a.tickets + gridDim.y + m, a.chunks)) return;

    // ---- the row's last workgroup: the exact cut, then the draw
    __shared__ unsigned long long chunk_mass[kChunks];
    uint64_t all_above = 0, all_between = 0;
    for (int c = 0; c < a.chunks; ++c) {
        all_above += load_shared(&masses[c].above);
        all_between += load_shared(&masses[c].between);
    }
    if (tid < kChunks) chunk_mass[tid] = tid < a.chunks ? load_shared(&masses[tid].kept) : 0;
    uint64_t cut_order = 0;   // tokens of this order and earlier ones stay
    // this thread's weight of the kept ones of kPer consecutive tokens from token i on
    auto kept_weight = [&](int i) {
        uint64_t sum = 0;
        for (int e = 0; e < kPer; ++e) {
            const float xv = i + e < V ? x[i + e] : -__builtin_inff();
            const double y = r.below(xv);
            if (!(y < kFarthest) || order_of(xv, i + e) < cut_order) continue;
            const double w = exp_minus(y);
            if (w >= r.min_w) sum += units(w);
        }
        return sum;
    };
    const uint32_t n = limited ? __hip_atomic_load(a.listed + m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;   // uniform
    if (n > kList) {
        __shared__ DigitBins digits;
        uint64_t weight;
        if (cut.k_bin != kNoBin) {
            cut_order = cut_by_digits(x, V, r, false, (double)r.k, digits, weight);
        } else {   // the list's share of the row is not known: once more from the logits
            uint64_t part = 0;
            for (int i = tid; i < V; i += kSampleThreads) {
                const double y = r.below(x[i]);
                if (y < kFarthest) part += units(exp_minus(y));
            }
            scan_block(part, weight);
        }
        if (r.p < 1.0) cut_order = cut_by_digits(x, V, r, true, r.p * (double)weight, digits, weight);
        for (int c = 0; c < a.chunks; ++c) {
            uint64_t total;
            scan_block(kept_weight(c * kChunk + tid * kPer), total);
            if (tid == 0) chunk_mass[c] = total;
        }
    } else if (n > 0) {
        uint32_t padded = 64;
        while (padded < n) padded <<= 1;
        for (uint32_t i = tid; i < padded; i += kSampleThreads) list[i] = i < n ? load_shared(row_list + i) : 0;
        __syncthreads();
        for (uint32_t size = 2; size <= padded; size <<= 1)   // bitonic, falling
            for (uint32_t step = size >> 1; step > 0; step >>= 1) {
                for (uint32_t t = tid; t < padded / 2; t += kSampleThreads) {
                    const uint32_t i = 2 * t - (t & (step - 1)), j = i + step;
                    const uint64_t p = list[i], q = list[j];
                    if ((p < q) == ((i & size) == 0)) list[i] = q, list[j] = p;
                }
                __syncthreads();
            }
        // weights down the list, in runs of consecutive entries per thread
        constexpr int kRun = kList / kSampleThreads;
        uint64_t w[kRun], sum = 0;
        uint32_t above_k_bin = 0;   // entries above the k-th token's bin
#pragma unroll
        for (int e = 0; e < kRun; ++e) {
            const uint32_t i = tid * kRun + e;
            w[e] = 0;
            if (i < n) {
                const double y = r.below(order_number((uint32_t)(list[i] >> 32)));
                w[e] = units(exp_minus(y));
                above_k_bin += r.bin(y) < cut.k_bin;
            }
            sum += w[e];
        }
        uint64_t list_weight, to_k_bin;
        uint64_t before = scan_block(sum, list_weight) - sum;
        scan_block(above_k_bin, to_k_bin);
        const uint64_t allowed = cut.k_bin == kNoBin ? n : to_k_bin + (uint64_t)(r.k - cut.above_k);   // entries that top-k leaves
        uint64_t part = 0, allowed_weight;
#pragma unroll
        for (int e = 0; e < kRun; ++e)
            if ((uint64_t)(tid * kRun + e) < allowed) part += w[e];
        scan_block(part, allowed_weight);
        const bool apart = cut.k_bin > cut.last;   // tokens between the border bins and the k-th token's come before the latter
        const double limit = r.p * (double)(all_above + all_between + allowed_weight);
        uint64_t stays = 0, staying;
        before += all_above;
#pragma unroll
        for (int e = 0; e < kRun; ++e) {
            const uint64_t i = (uint64_t)tid * kRun + e;
            const uint64_t ahead = before + (apart && i >= to_k_bin ? all_between : 0);
            stays += i < allowed && (r.p >= 1.0 || (double)ahead < limit || ahead == 0);
            before += w[e];
        }
        scan_block(stays, staying);
        cut_order = staying ? list[staying - 1] : list[0] + 1;
#pragma unroll
        for (int e = 0; e < kRun; ++e) {
            const uint64_t i = (uint64_t)tid * kRun + e;
            if (i >= staying) continue;
            const uint64_t o = list[i];
            if (exp_minus(r.below(order_number((uint32_t)(o >> 32)))) >= r.min_w) atomicAdd(&chunk_mass[(~(uint32_t)o) / kChunk], (unsigned long long)w[e]);
        }
    }
    __syncthreads();
    uint64_t total = 0;
    for (int c = 0; c < a.chunks; ++c) total += chunk_mass[c];
    uint64_t rank = drawn_rank(a, m, total);
    int chunk = 0;
    while (rank >= chunk_mass[chunk]) rank -= chunk_mass[chunk++];   // rank < total: ends inside
    const int i0 = chunk * kChunk + tid * kPer;
    const uint64_t here = kept_weight(i0);
    uint64_t unused;
    const uint64_t upto = scan_block(here, unused);
    if (upto > rank && upto - here <= rank) {   // one thread
        uint64_t to = upto - here;
        for (int e = 0; e < kPer; ++e) {
            const float xv = i0 + e < V ? x[i0 + e] : -__builtin_inff();
            const double y = r.below(xv);
            if (!(y < kFarthest) || order_of(xv, i0 + e) < cut_order) continue;
            const double w = exp_minus(y);
            if (!(w >= r.min_w)) continue;
            to += units(w);
            if (to > rank) {
                a.token[m] = i0 + e;
                a.prob[m] = (float)(w * kOne / (double)total);
                break;
            }
        }
    }
}

}  // namespace w4

using namespace w4;

extern "C" {

// tickets | tops | cuts | listed | masses | bins | lists
static size_t sample_layout(int M, int V, size_t (&at)[7])
{
    const size_t rows = (size_t)M, chunks = (size_t)(V + kChunk - 1) / kChunk;
    const size_t sizes[7] = {kTicketBytes, rows * chunks * sizeof(ChunkTop), rows * sizeof(RowCut), rows * sizeof(uint32_t), rows * chunks * sizeof(ChunkMass),
                             rows * chunks * kBins * 8, rows * kList * 8};
    size_t end = 0;
    for (int i = 0; i < 7; ++i) {
        at[i] = end;
        end += (sizes[i] + 255) & ~(size_t)255;   // workgroups exchange through these: no line belongs to two
    }
    return end;
}

size_t lm_head_sample_workspace_bytes(int M, int V)
{
    if (M < 1 || M > W4A16_MAX_M || V < 1 || V > kChunks * kChunk) return 0;
    size_t at[7];
    return sample_layout(M, V, at);
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
    size_t at[7];
    if (!workspace || workspace_bytes < sample_layout(M, V, at)) return W4A16_EWORKSPACE;
    uint8_t *ws = reinterpret_cast<uint8_t *>(workspace);
    const SampleArgs a = {logits, temperature, top_k, top_p, min_p, uniform, token, prob, V, (V + kChunk - 1) / kChunk, (ChunkTop *)(ws + at[1]),
                          (unsigned long long *)(ws + at[5]), (RowCut *)(ws + at[2]), (ChunkMass *)(ws + at[4]), (unsigned long long *)(ws + at[6]),
                          (uint32_t *)(ws + at[3]), (uint32_t *)ws};
    const dim3 grid((unsigned)a.chunks, (unsigned)M);
    hipLaunchKernelGGL(sample_top_kernel, grid, dim3(kSampleThreads), 0, (hipStream_t)stream, a);
    if (top_k || top_p) hipLaunchKernelGGL(sample_bins_kernel, grid, dim3(kSampleThreads), 0, (hipStream_t)stream, a);
    hipLaunchKernelGGL(sample_draw_kernel, grid, dim3(kSampleThreads), 0, (hipStream_t)stream, a);
    return launch_status();
}

}  // extern "C"
