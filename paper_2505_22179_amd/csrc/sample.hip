// lm_head_sample: next tokens from logits and given uniform numbers, with temperature, top-k, top-p and min-p.  Contract in
// include/w4a16.h.
//
// A token's weight is w = exp((x - max) / T), evaluated in fp64 and held as a whole number of 2^-44: sums of whole numbers do not depend
// on their order, so any split of a row gives the same token, and a border (a cumulative weight against p, or against u) is off by 1e-11
// of the row's total where sums in fp32 would be off by 1e-5 -- tokens near a border would change with the split.  Tokens more than e^31 below the
// row's largest weigh nothing (262144 of them 1e-8 of the total at most) and take part in nothing.
#include "internal.h"

namespace w4 {

constexpr int kSampleThreads = 1024;
constexpr int kSampleBlocks = 262144 / kSampleThreads;   // blocks of a row, of one token per thread
constexpr double kFarthest = 31.0;
constexpr double kOne = 17592186044416.0;                // 2^44: weight 1
constexpr int32_t kNoToken = 0x7FFFFFFF;

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

// what a row is sampled with
struct RowRule {
    float top;       // largest logit
    double inv_t;
    bool greedy;
    int k;           // 0: no limit
    double p;        // >= 1: no limit
    double min_w;    // <= 0: no limit

    // distance below the largest logit in units of the temperature; at least kFarthest, or NaN, for what takes no part
    __device__ __forceinline__ double below(float x) const
    {
        if (x == top) return 0.0;
        return x > -__builtin_inff() ? ((double)top - (double)x) * inv_t : kFarthest;
    }
};

struct SampleArgs {
    const float *logits;
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p, *uniform;
    int32_t *token;
    float *prob;
    int V;
};

__device__ __forceinline__ RowRule row_rule(const SampleArgs &a, int m, float top)
{
    RowRule r;
    const float t = a.temperature ? a.temperature[m] : 1.f;
    const int k = a.top_k ? a.top_k[m] : 0;
    const float p = a.top_p ? a.top_p[m] : 1.f, min_p = a.min_p ? a.min_p[m] : 0.f;
    r.top = top;
    r.greedy = !(t > 0.f) || k == 1 || p <= 0.f || min_p > 1.f;
    r.inv_t = r.greedy ? 0.0 : 1.0 / (double)t;
    r.k = k > 0 && k < a.V ? k : 0;
    r.p = p < 1.f ? (double)p : 2.0;
    r.min_w = min_p > 0.f ? (double)min_p : 0.0;
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

// One workgroup per row, whatever the logits and limits are.
struct RowShared {
    unsigned long long mass[256];
    uint32_t count[256];
    unsigned long long block_mass[kSampleBlocks];
    float wave_top[kSampleThreads / 64];
    int32_t wave_at[kSampleThreads / 64];
    uint32_t prefix, wave_ties[kSampleThreads / 64];
    unsigned long long above;
    int64_t left;
    int32_t cut_at;
};

// The cut of a row: the token (key, index) that is the last one kept in the order of falling logits, equal ones by index.  by_mass: the
// last token with less than `limit` of weight before it; otherwise the limit-th token.  Digit by digit from the top of the key; every thread of the
// workgroup calls it.  Returns the cut's key and, in left, how many of the tokens of that key are kept; kept_mass: the weight up to the cut.
__device__ void row_cut(const float *x, int V, const RowRule &r, bool by_mass, double limit, RowShared &sh, uint32_t &key, int64_t &left,
                        uint64_t &kept_mass)
{
    const int tid = threadIdx.x;
    uint32_t prefix = 0, settled_bits = 0;
    uint64_t above = 0;      // weight of the tokens above the prefix
    int64_t count_left = by_mass ? 0 : (int64_t)limit;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) sh.mass[tid] = 0, sh.count[tid] = 0;
        __syncthreads();
        for (int i = tid; i < V; i += kSampleThreads) {
            const uint32_t kx = order_key(x[i]);
            if ((kx & settled_bits) != prefix) continue;
            const double y = r.below(x[i]);
            if (!(y < kFarthest)) continue;
            const int d = (kx >> shift) & 255;
            atomicAdd(&sh.count[d], 1u);
            atomicAdd(&sh.mass[d], (unsigned long long)(exp_minus(y) * kOne + 0.5));
        }
        __syncthreads();
        if (tid == 0) {
            int cut = -1;
            uint64_t before = above, cut_above = above;
            int64_t need = count_left;
            for (int d = 255; d >= 0; --d) {
                if (sh.count[d] == 0) continue;
                if (cut >= 0 && (by_mass ? !((double)before < limit) : need <= 0)) break;
                cut = d;
                cut_above = before;
                before += sh.mass[d];
                if (!by_mass) need -= sh.count[d];
            }
            if (!by_mass) need = need > 0 ? (int64_t)V : need + sh.count[cut];   // fewer tokens than the limit: all of them
            sh.prefix = prefix | ((uint32_t)cut << shift);
            sh.above = cut_above;
            if (shift == 0) {
                const int64_t n = sh.count[cut];
                const double w = (double)sh.mass[cut] / (double)n;
                if (by_mass) need = (int64_t)ceil(fmin((limit - (double)cut_above) / w, (double)n));
                need = need < 1 ? 1 : need > n ? n : need;
                sh.above = cut_above + (uint64_t)need * (sh.mass[cut] / n);
            }
            sh.left = need;
        }
        __syncthreads();
        prefix = sh.prefix;
        above = sh.above;
        count_left = sh.left;
        settled_bits |= 255u << shift;
    }
    key = prefix;
    left = count_left;
    kept_mass = above;
    __syncthreads();
}

__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(const SampleArgs a)
{
    __shared__ RowShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = blockIdx.x, V = a.V;
    const float *x = a.logits + (size_t)m * V;
    // the largest logit and its first token
    float top = -__builtin_inff();
    int at = kNoToken;
    for (int i = tid; i < V; i += kSampleThreads) {
        const float v = x[i];
        if (v > top) top = v, at = i;   // NaN and -inf win nothing
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const float v = __shfl_xor(top, off, 64);
        const int j = __shfl_xor(at, off, 64);
        if (v > top || (v == top && j < at)) top = v, at = j;
    }
    if (lane == 0) sh.wave_top[wave] = top, sh.wave_at[wave] = at;
    for (int b = tid; b < kSampleBlocks; b += kSampleThreads) sh.block_mass[b] = 0;
    __syncthreads();
    for (int w = 0; w < kSampleThreads / 64; ++w) {
        const float v = sh.wave_top[w];
        const int j = sh.wave_at[w];
        if (v > top || (v == top && j < at)) top = v, at = j;
    }
    const RowRule r = row_rule(a, m, top);
    if (at == kNoToken || r.greedy) {   // uniform
        if (tid == 0) {
            a.token[m] = at;
            a.prob[m] = at == kNoToken ? 0.f : 1.f;
        }
        return;
    }
    uint32_t key = 0;
    int64_t ties = V;
    uint64_t kept = 0;
    if (r.k) row_cut(x, V, r, false, (double)r.k, sh, key, ties, kept);
    if (r.p < 1.0) {
        if (!r.k) {
            uint64_t mine = 0;
            for (int i = tid; i < V; i += kSampleThreads) {
                const double y = r.below(x[i]);
                if (y < kFarthest) mine += (uint64_t)(exp_minus(y) * kOne + 0.5);
            }
            if (tid == 0) sh.above = 0;
            __syncthreads();
            mine = add_over_wave(mine);
            if (lane == 0) atomicAdd(&sh.above, (unsigned long long)mine);
            __syncthreads();
            kept = sh.above;
            __syncthreads();
        }
        row_cut(x, V, r, true, r.p * (double)kept, sh, key, ties, kept);
    }
    // weight of the kept tokens by blocks of kSampleThreads tokens, the ties of the cut in token order
    const int blocks = (V + kSampleThreads - 1) / kSampleThreads;
    int64_t seen = 0;   // ties in the blocks before
    auto kept_weight = [&](int b, int64_t seen_before, int &ties_here, double &w) {   // of this thread's token of block b
        const int i = b * kSampleThreads + tid;
        const float v = i < V ? x[i] : -__builtin_inff();
        const double y = r.below(v);
        const bool part = y < kFarthest;
        w = part ? exp_minus(y) : 0.0;
        const uint32_t kx = order_key(v);
        const bool tie = part && kx == key;
        const uint64_t tied = __ballot(tie);
        __syncthreads();
        if (lane == 0) sh.wave_ties[wave] = (uint32_t)__popcll(tied);
        __syncthreads();
        int64_t before = seen_before;
        ties_here = 0;
        for (int q = 0; q < kSampleThreads / 64; ++q) {
            if (q < wave) before += sh.wave_ties[q];
            ties_here += (int)sh.wave_ties[q];
        }
        before += __popcll(tied & ((1ull << lane) - 1));
        const bool keep = part && (kx > key || (tie && before < ties)) && (w >= r.min_w);
        return keep ? (uint64_t)(w * kOne + 0.5) : (uint64_t)0;
    };
    for (int b = 0; b < blocks; ++b) {
        int here;
        double w;
        const uint64_t mass = add_over_wave(kept_weight(b, seen, here, w));
        if (lane == 0 && mass) atomicAdd(&sh.block_mass[b], (unsigned long long)mass);
        seen += here;
    }
    __syncthreads();
    uint64_t total = 0;
    for (int b = 0; b < blocks; ++b) total += sh.block_mass[b];
    uint64_t rank = drawn_rank(a, m, total);
    int block = 0;
    while (rank >= sh.block_mass[block]) rank -= sh.block_mass[block++];
    // the token inside its block
    seen = 0;
    if (key) {   // ties before the block, counted again
        uint32_t mine = 0;
        for (int i = tid; i < block * kSampleThreads; i += kSampleThreads) mine += r.below(x[i]) < kFarthest && order_key(x[i]) == key;
        if (tid == 0) sh.above = 0;
        __syncthreads();
        atomicAdd(&sh.above, (unsigned long long)mine);
        __syncthreads();
        seen = (int64_t)sh.above;
        __syncthreads();
    }
    int here;
    double w;
    const uint64_t mine = kept_weight(block, seen, here, w);
    uint64_t upto = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint64_t v = __shfl_up((unsigned long long)upto, off, 64);
        if (lane >= off) upto += v;
    }
    if (lane == 63) sh.mass[wave] = upto;
    __syncthreads();
    for (int q = 0; q < wave; ++q) upto += sh.mass[q];
    if (mine && upto > rank && upto - mine <= rank) {
        a.token[m] = block * kSampleThreads + tid;
        a.prob[m] = (float)(w * kOne / (double)total);
    }
}

}  // namespace w4

using namespace w4;

extern "C" {

size_t lm_head_sample_workspace_bytes(int M, int V)
{
    if (M < 1 || M > W4A16_MAX_M || V < 1 || V > 262144) return 0;
    return kTicketBytes;
}

int lm_head_sample(const float *logits, int M, int V, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                   const float *uniform, int32_t *token, float *prob, void *workspace, size_t workspace_bytes, void *stream)
{
    if (M < 1 || V < 1) return W4A16_EINVAL;
    if (M > W4A16_MAX_M || V > 262144) return W4A16_EUNSUP;
    if (!logits || !uniform || !token || !prob) return W4A16_ENULL;
    if (misaligned(logits) || workspace_misaligned(workspace)) return W4A16_EALIGN;
    if ((reinterpret_cast<uintptr_t>(temperature) | reinterpret_cast<uintptr_t>(top_k) | reinterpret_cast<uintptr_t>(top_p) |
         reinterpret_cast<uintptr_t>(min_p) | reinterpret_cast<uintptr_t>(uniform) | reinterpret_cast<uintptr_t>(token) |
         reinterpret_cast<uintptr_t>(prob)) & 3u)
        return W4A16_EALIGN;
    if (!workspace || workspace_bytes < lm_head_sample_workspace_bytes(M, V)) return W4A16_EWORKSPACE;
    const SampleArgs a = {logits, temperature, top_k, top_p, min_p, uniform, token, prob, V};
    hipLaunchKernelGGL(sample_row_kernel, dim3((unsigned)M), dim3(kSampleThreads), 0, (hipStream_t)stream, a);
    return launch_status();
}

}  // extern "C"
