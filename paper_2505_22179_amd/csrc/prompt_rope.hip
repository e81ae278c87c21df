// rope_table and rope_prompt: cos/sin tables scaled for long contexts, and the rotation of packed tokens with keys and values scattered to
// cache rows of a slot map.  Contracts in include/w4a16.h.
#include <math.h>
#include "internal.h"

namespace w4 {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

// ---- tables ------------------------------------------------------------------------------------------------
constexpr int kTableThreads = 256;
constexpr int kTablePositions = 128;   // of a workgroup
constexpr int kTableMostPairs = 512;

struct TableArgs {
    float *cos_t, *sin_t;
    double neg_log2_theta;   // -log2(theta) * 2 / R
    double inv_factor, turns_of_one;   // turns_of_one: original / (2 pi), the turns of a pair of frequency 1
    double low, inv_width;   // of the blend: in turns, or in pair indices
    double amplitude;
    int first, n_pos, pairs, scaling;
};

// cos and sin of a in 64 bits: a is brought within pi / 4 of a multiple of pi / 2 (its two-part constant, exact for |a| < 2^31) and the series
// around 0 are cut where their next term, (pi/4)^17 / 17! and (pi/4)^18 / 18!, is below 2^-54.
__device__ __forceinline__ void cos_sin(double a, double &c, double &s)
{
    const double n = __builtin_rint(a * 0.63661977236758134308);
    double r = __builtin_fma(-n, 1.57079632679489655800, a);
    r = __builtin_fma(-n, 6.12323399573676603587e-17, r);
    const double z = r * r;
    double ps = __builtin_fma(z, -1.0 / 1307674368000, 1.0 / 6227020800);
    ps = __builtin_fma(z, ps, -1.0 / 39916800);
    ps = __builtin_fma(z, ps, 1.0 / 362880);
    ps = __builtin_fma(z, ps, -1.0 / 5040);
    ps = __builtin_fma(z, ps, 1.0 / 120);
    ps = __builtin_fma(z, ps, -1.0 / 6);
    ps = __builtin_fma(z * r, ps, r);
    double pc = __builtin_fma(z, 1.0 / 20922789888000, -1.0 / 87178291200);
    pc = __builtin_fma(z, pc, 1.0 / 479001600);
    pc = __builtin_fma(z, pc, -1.0 / 3628800);
    pc = __builtin_fma(z, pc, 1.0 / 40320);
    pc = __builtin_fma(z, pc, -1.0 / 720);
    pc = __builtin_fma(z, pc, 1.0 / 24);
    pc = __builtin_fma(z, pc, -0.5);
    pc = __builtin_fma(z, pc, 1.0);
    const int q = (int)(long long)n;
    const double cc = (q & 1) ? ps : pc, ss = (q & 1) ? pc : ps;
    c = ((q + 1) & 2) ? -cc : cc;
    s = (q & 2) ? -ss : ss;
}

// A workgroup takes kTablePositions positions and works out the frequencies once (into LDS), with the turn from one of a thread's positions to its next.
// A thread keeps V pairs, evaluates cos and sin at its first position and turns them on from there in fp64 (four instructions an entry instead of
// some forty).  A turn is off by 2^-51 (its own roundings, cos and sin) and half a last place of its angle, at_once f; kTablePositions / at_once of
// them in a row by 2^-44 + 2^-46 f at the most, f up to 8 (a factor of 1/8), beside the rounding of the first angle.  What bounds it are the writes: 131072 positions, 64 pairs, 12.6 us, 5.3 TB/s (every
// entry evaluated by itself 16.5).
template <int V>
__global__ __launch_bounds__(kTableThreads) void rope_table_kernel(TableArgs a)
{
    typedef float Part __attribute__((ext_vector_type(V)));
    __shared__ double freq[kTableMostPairs], cos_turn[kTableMostPairs], sin_turn[kTableMostPairs];
    const int units = a.pairs / V, lanes = min(units, kTableThreads), at_once = kTableThreads / lanes;   // positions next to each other
    for (int i = threadIdx.x; i < a.pairs; i += kTableThreads) {
        double f = exp2(a.neg_log2_theta * i);
        if (a.scaling == W4A16_ROPE_LINEAR) f *= a.inv_factor;
        else if (a.scaling == W4A16_ROPE_BY_TURNS) {
            const double t = fmin(fmax((a.turns_of_one * f - a.low) * a.inv_width, 0.0), 1.0);
            f = t * f + (1.0 - t) * (f * a.inv_factor);
        } else if (a.scaling == W4A16_ROPE_BY_INDEX) {
            const double t = fmin(fmax((i - a.low) * a.inv_width, 0.0), 1.0);
            f = t * (f * a.inv_factor) + (1.0 - t) * f;
        }
        freq[i] = f;
        cos_sin(at_once * f, cos_turn[i], sin_turn[i]);
    }
    __syncthreads();
    const int p0 = blockIdx.x * kTablePositions, here = min(kTablePositions, a.n_pos - p0), row = threadIdx.x / lanes;
    if (row >= min(at_once, here)) return;
    for (int u = threadIdx.x % lanes; u < units; u += lanes) {
        double c[V], s[V], ct[V], st[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int i = u * V + e;
            cos_sin((double)(a.first + p0 + row) * freq[i], c[e], s[e]);
            c[e] *= a.amplitude;
            s[e] *= a.amplitude;
            ct[e] = cos_turn[i];
            st[e] = sin_turn[i];
        }
        for (int p = row; p < here; p += at_once) {
            Part c_out, s_out;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                c_out[e] = (float)c[e];
                s_out[e] = (float)s[e];
                const double next = __builtin_fma(c[e], ct[e], -(s[e] * st[e]));
                s[e] = __builtin_fma(s[e], ct[e], c[e] * st[e]);
                c[e] = next;
            }
            const size_t at = (size_t)(p0 + p) * a.pairs + u * V;
            *reinterpret_cast<Part *>(a.cos_t + at) = c_out;
            *reinterpret_cast<Part *>(a.sin_t + at) = s_out;
        }
    }
}

// ---- rotation and scatter ------------------------------------------------------------------------------------
constexpr int kRopeThreads = 256;

struct PromptRopeArgs {
    const _Float16 *qkv;
    const int32_t *pos, *slot;
    const float *cos_t, *sin_t;
    _Float16 *q, *k, *v;
    int n_pos, R, cache_rows, Hq, Hkv, D;
};

// 2 V elements of a head at a time: V and V of the two halves of the turned part, or 2 V next to each other (interleaved pairs, what is not
// turned, values).  A thread keeps its place in the head and goes through the heads, so that it reads its table entries once.
template <int V>
struct Unit {
    typedef _Float16 Part __attribute__((ext_vector_type(V)));
    Part a, b;
    __device__ __forceinline__ void load(const _Float16 *src, int at, int gap)
    {
        a = __builtin_nontemporal_load(reinterpret_cast<const Part *>(src + at));
        b = __builtin_nontemporal_load(reinterpret_cast<const Part *>(src + at + gap));
    }
    __device__ __forceinline__ void store(_Float16 *dst, int at, int gap) const
    {
        *reinterpret_cast<Part *>(dst + at) = a;
        *reinterpret_cast<Part *>(dst + at + gap) = b;
    }
};

// A workgroup per token, whose next head is on its way while one is turned; bound by the copy where there are many (8192 tokens of first use, 64/8 heads of 128:
// 71.5 us, 4.8 TB/s; one head after another 74.1), by the launch where there are few (16 tokens 3.6 us).
template <int V, bool INTERLEAVED>
__global__ __launch_bounds__(kRopeThreads) void rope_prompt_kernel(PromptRopeArgs a)
{
    const int m = blockIdx.x, units = a.D / (2 * V), turned = a.R / (2 * V), pairs = a.R >> 1;
    const int heads_at_once = kRopeThreads / units;
    const int u = threadIdx.x % units, h0 = threadIdx.x / units;
    if (h0 >= heads_at_once) return;
    const int heads = a.Hq + 2 * a.Hkv;
    const _Float16 *const row = a.qkv + (size_t)m * heads * a.D;
    const bool turns = u < turned;
    const int at = turns && !INTERLEAVED ? u * V : u * 2 * V, gap = turns && !INTERLEAVED ? pairs : V;   // of queries and keys
    Unit<V> ahead;   // of the next head; the first is asked for before the position is known
    auto load = [&](int head) {
        const bool value = head >= a.Hq + a.Hkv;
        ahead.load(row + (size_t)head * a.D, value ? u * 2 * V : at, value ? V : gap);
    };
    if (h0 < heads) load(h0);
    const int p = a.pos[m], to = a.slot ? a.slot[m] : m;
    const bool placed = p >= 0 && p < a.n_pos, stored = to >= 0 && to < a.cache_rows;
    float c[V], s[V];
    if (turns && placed) {
#pragma unroll
        for (int e = 0; e < V; ++e) c[e] = a.cos_t[(size_t)p * pairs + u * V + e], s[e] = a.sin_t[(size_t)p * pairs + u * V + e];
    }
    for (int head = h0; head < heads; head += heads_at_once) {
        const bool value = head >= a.Hq + a.Hkv;
        const int here = value ? u * 2 * V : at, step = value ? V : gap;
        Unit<V> x = ahead;
        if (head + heads_at_once < heads) load(head + heads_at_once);
        if (!value) {
            if (!placed) continue;   // this row's q and k are left untouched
            if (turns) {
                float lo[V], hi[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if constexpr (INTERLEAVED) {
                        lo[e] = (float)(2 * e < V ? x.a[(2 * e) % V] : x.b[(2 * e) % V]);
                        hi[e] = (float)(2 * e + 1 < V ? x.a[(2 * e + 1) % V] : x.b[(2 * e + 1) % V]);
                    } else {
                        lo[e] = (float)x.a[e];
                        hi[e] = (float)x.b[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {   // rope_append's own expressions
                    const _Float16 y = (_Float16)keep_f32(fmaf(lo[e], c[e], -hi[e] * s[e])), z = (_Float16)keep_f32(fmaf(hi[e], c[e], lo[e] * s[e]));
                    if constexpr (INTERLEAVED) {
                        if (2 * e < V) x.a[(2 * e) % V] = y; else x.b[(2 * e) % V] = y;
                        if (2 * e + 1 < V) x.a[(2 * e + 1) % V] = z; else x.b[(2 * e + 1) % V] = z;
                    } else {
                        x.a[e] = y;
                        x.b[e] = z;
                    }
                }
            }
        }
        if (head < a.Hq) x.store(a.q + ((size_t)m * a.Hq + head) * a.D, here, step);
        else if (stored) {
            _Float16 *const dst = value ? a.v : a.k;
            x.store(dst + ((size_t)to * a.Hkv + (value ? head - a.Hq - a.Hkv : head - a.Hq)) * a.D, here, step);
        }
    }
}

}  // namespace w4

using namespace w4;

extern "C" {

int rope_table(float *cos_table, float *sin_table, int first, int n_pos, int R, double theta, int scaling, double factor, double low, double high,
               double original, double amplitude, void *stream)
{
    if (first < 0 || n_pos < 1 || R < 2 || R % 2 != 0) return W4A16_EINVAL;
    if (!(theta > 1.0) || !(theta < INFINITY) || !(fabs(amplitude) < INFINITY)) return W4A16_EINVAL;
    if (scaling < W4A16_ROPE_PLAIN || scaling > W4A16_ROPE_BY_INDEX) return W4A16_EINVAL;
    if (scaling != W4A16_ROPE_PLAIN && (!(factor > 0.0) || !(factor < INFINITY))) return W4A16_EINVAL;
    if (scaling >= W4A16_ROPE_BY_TURNS && (!(low > 0.0) || !(high > low) || !(high < INFINITY) || !(original > 0.0) || !(original < INFINITY)))
        return W4A16_EINVAL;
    if (R > 2 * kTableMostPairs || (long long)first + n_pos > (1ll << 28)) return W4A16_EUNSUP;
    if (scaling != W4A16_ROPE_PLAIN && factor < 0.125) return W4A16_EUNSUP;   // angles stay below 2^31
    if (!cos_table || !sin_table) return W4A16_ENULL;
    if (misaligned(cos_table) || misaligned(sin_table)) return W4A16_EALIGN;
    TableArgs a = {cos_table, sin_table, -log2(theta) * 2.0 / R, 1.0, 0.0, low, 0.0, amplitude, first, n_pos, R / 2, scaling};
    const double turn = 6.283185307179586477;
    if (scaling != W4A16_ROPE_PLAIN) a.inv_factor = 1.0 / factor;
    if (scaling == W4A16_ROPE_BY_TURNS) {
        a.turns_of_one = original / turn;
        a.inv_width = 1.0 / (high - low);
    } else if (scaling == W4A16_ROPE_BY_INDEX) {
        // the pair index at which a pair turns n times within the original context
        const double at_high = R * log(original / (high * turn)) / (2.0 * log(theta)), at_low = R * log(original / (low * turn)) / (2.0 * log(theta));
        const double begin = fmax(floor(at_high), 0.0), end = fmin(ceil(at_low), R - 1.0);
        a.low = begin;
        a.inv_width = 1.0 / fmax(end - begin, 0.001);   // a step where the two indices meet
    }
    const dim3 grid((unsigned)((n_pos + kTablePositions - 1) / kTablePositions));
    if (a.pairs % 4 == 0) hipLaunchKernelGGL(rope_table_kernel<4>, grid, dim3(kTableThreads), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(rope_table_kernel<1>, grid, dim3(kTableThreads), 0, (hipStream_t)stream, a);
    return launch_status();
}

int rope_prompt(const void *qkv, const int32_t *pos, const float *cos_table, const float *sin_table, int n_pos, int R, int interleaved,
                const int32_t *slot, int cache_rows, void *q, void *k_cache, void *v_cache, int rows, int Hq, int Hkv, int D, void *stream)
{
    if (rows < 1 || Hq < 1 || Hkv < 1 || D < 8 || D % 8 != 0 || R < 2 || R % 2 != 0 || R > D || n_pos < 1 || cache_rows < 1) return W4A16_EINVAL;
    if (interleaved != 0 && interleaved != 1) return W4A16_EINVAL;
    if (D > 512 || rows > (1 << 23) || Hq > (1 << 16) || Hkv > (1 << 16)) return W4A16_EUNSUP;
    if (!qkv || !pos || !cos_table || !sin_table || !q || !k_cache || !v_cache) return W4A16_ENULL;
    if (misaligned(qkv) || misaligned(q) || misaligned(k_cache) || misaligned(v_cache) || misaligned(cos_table) || misaligned(sin_table) ||
        ((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(slot)) & 3u))
        return W4A16_EALIGN;
    const PromptRopeArgs a = {(const _Float16 *)qkv, pos, slot, cos_table, sin_table, (_Float16 *)q, (_Float16 *)k_cache, (_Float16 *)v_cache,
                              n_pos, R, cache_rows, Hq, Hkv, D};
#define W4_ROPE(V_)                                                                                                                         \
    hipLaunchKernelGGL((interleaved ? rope_prompt_kernel<V_, true> : rope_prompt_kernel<V_, false>), dim3((unsigned)rows), dim3(kRopeThreads), 0, \
                       (hipStream_t)stream, a)
    if (R % 16 == 0 && D % 16 == 0) W4_ROPE(8);
    else if (R % 8 == 0) W4_ROPE(4);
    else W4_ROPE(1);   // element by element, 256 pairs of the widest head fill the workgroup: 8192 tokens, 32/32 heads of 80, R 20 85 us, R 40 60
#undef W4_ROPE
    return launch_status();
}

}  // extern "C"
