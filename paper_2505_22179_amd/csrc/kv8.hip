// rope_append_qk_norm, rope_append_kv8, w4a16_kv8_read, tree_accept_kv8: norms of queries and keys for each head, the rotary embedding and the
// append to the cache in one pass, into an fp16 cache or an 8-bit one, and the 8-bit cache's way back.  Contracts in include/w4a16.h.
#include "internal.h"
#include "kv8.h"

namespace w4 {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kFp16Cache = 0;   // the other cache formats: kInt8, kE4m3
constexpr int kAppendThreads = 256;

struct AppendArgs {
    const _Float16 *qkv, *q_gamma, *k_gamma;   // gammas: both or none
    const int32_t *pos;
    const float *cos_t, *sin_t;
    _Float16 *q;
    void *k, *v;                  // cache: fp16 values or 8-bit codes
    _Float16 *k_scale, *v_scale;  // 8-bit cache only
    float eps;
    int n_pos, P, Hq, Hkv, D;
};

// A group of LANES neighbouring lanes (a power of two, at least D / 8) holds one head of one row, lane i its element pairs
// (4 i .. 4 i + 3) and (4 i + D/2 ..); lanes beyond D / 8 hold zeros.  The head's sum of squares and its largest magnitude are butterflies
// inside the group: fixed order, no LDS.  blockIdx.x: heads, blockIdx.y: row.
template <int FMT, int LANES>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(AppendArgs a)
{
    const int m = blockIdx.y, h = a.D >> 1;
    const int heads = a.Hq + 2 * a.Hkv;
    const int head = blockIdx.x * (kAppendThreads / LANES) + threadIdx.x / LANES;
    const int i = (threadIdx.x % LANES) * 4;
    if (head >= heads) return;   // uniform over the group: the butterflies stay inside it
    const bool holds = i < h;
    half4 lo = {}, hi = {};
    const _Float16 *src = a.qkv + ((size_t)m * heads + head) * a.D;
    if (holds) {
        lo = *reinterpret_cast<const half4 *>(src + i);
        hi = *reinterpret_cast<const half4 *>(src + i + h);
    }
    if (head < a.Hq + a.Hkv) {
        const int p = a.pos[m];
        if (p < 0 || p >= a.n_pos) return;   // this row's q and k are left untouched
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (float)lo[e], x[4 + e] = (float)hi[e];
        if (a.q_gamma) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
            for (int off = 1; off < LANES; off <<= 1) ss += __shfl_xor(ss, off, LANES);
            const float inv = 1.f / sqrtf(ss / (float)a.D + a.eps);
            const _Float16 *gamma = head < a.Hq ? a.q_gamma : a.k_gamma;
            if (holds) {
                const half4 glo = *reinterpret_cast<const half4 *>(gamma + i), ghi = *reinterpret_cast<const half4 *>(gamma + i + h);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = x[e] * inv * (float)glo[e], x[4 + e] = x[4 + e] * inv * (float)ghi[e];
            }
        }
        if (holds) {   // rope_append's own expressions
            const float4v c = *reinterpret_cast<const float4v *>(a.cos_t + (size_t)p * h + i);
            const float4v s = *reinterpret_cast<const float4v *>(a.sin_t + (size_t)p * h + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] = (_Float16)keep_f32(fmaf(x[e], c[e], -x[4 + e] * s[e]));
                hi[e] = (_Float16)keep_f32(fmaf(x[4 + e], c[e], x[e] * s[e]));
            }
        }
        if (head < a.Hq) {
            if (holds) {
                _Float16 *dst = a.q + ((size_t)m * a.Hq + head) * a.D;
                *reinterpret_cast<half4 *>(dst + i) = lo;
                *reinterpret_cast<half4 *>(dst + i + h) = hi;
            }
            return;
        }
    }
    const bool value = head >= a.Hq + a.Hkv;
    const size_t at = (size_t)(a.P + m) * a.Hkv + (value ? head - a.Hq - a.Hkv : head - a.Hq);   // head of a cached row
    if constexpr (FMT == kFp16Cache) {
        if (holds) {
            _Float16 *dst = (_Float16 *)(value ? a.v : a.k) + at * a.D;
            *reinterpret_cast<half4 *>(dst + i) = lo;
            *reinterpret_cast<half4 *>(dst + i + h) = hi;
        }
    } else {
        // magnitudes of fp16 numbers compare as their bits do, infinities and NaN above all others
        uint32_t most = 0;
        const u32x2 blo = __builtin_bit_cast(u32x2, lo) & 0x7FFF7FFFu, bhi = __builtin_bit_cast(u32x2, hi) & 0x7FFF7FFFu;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            most = max(most, max(blo[e] & 0xFFFFu, blo[e] >> 16));
            most = max(most, max(bhi[e] & 0xFFFFu, bhi[e] >> 16));
        }
#pragma unroll
        for (int off = 1; off < LANES; off <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off, LANES));
        const bool finite = most < kHalfInf;
        const float s = kv8_scale<FMT>((float)__builtin_bit_cast(_Float16, (uint16_t)(finite ? most : 0u)));
        const float vlo[4] = {(float)lo[0], (float)lo[1], (float)lo[2], (float)lo[3]};
        const float vhi[4] = {(float)hi[0], (float)hi[1], (float)hi[2], (float)hi[3]};
        uint8_t *dst = (uint8_t *)(value ? a.v : a.k) + at * a.D;
        if (holds) {
            *reinterpret_cast<uint32_t *>(dst + i) = finite ? kv8_codes<FMT>(vlo, s) : 0u;
            *reinterpret_cast<uint32_t *>(dst + i + h) = finite ? kv8_codes<FMT>(vhi, s) : 0u;
        }
        if (i == 0) (value ? a.v_scale : a.k_scale)[at] = finite ? (_Float16)s : __builtin_bit_cast(_Float16, (uint16_t)kHalfNan);
    }
}

template <int FMT>
int launch_append(const AppendArgs &a, int M, hipStream_t stream)
{
    const int lanes = a.D / 8, heads = a.Hq + 2 * a.Hkv;
#define W4_APPEND(L_)                                                                                                     \
    hipLaunchKernelGGL((kv_append_kernel<FMT, L_>), dim3((unsigned)((heads + kAppendThreads / L_ - 1) / (kAppendThreads / L_)), (unsigned)M), \
                       dim3(kAppendThreads), 0, stream, a)
    if (lanes <= 8) W4_APPEND(8);
    else if (lanes <= 16) W4_APPEND(16);
    else if (lanes <= 32) W4_APPEND(32);
    else W4_APPEND(64);
#undef W4_APPEND
    return launch_status();
}

// ---- an 8-bit cache back to fp16 -------------------------------------------------------------------------
// A thread turns eight codes into eight values: 8-byte loads and 16-byte stores, both contiguous over a wavefront.  A workgroup takes
// `whole` heads of consecutive rows (as many as fill its threads kReadPasses times); blockIdx.y: keys or values.
constexpr int kReadThreads = 256, kReadPasses = 4;
template <int FMT>
__global__ __launch_bounds__(kReadThreads) void kv8_read_kernel(const uint8_t *__restrict__ k, const uint8_t *__restrict__ v,
                                                                const _Float16 *__restrict__ k_scale, const _Float16 *__restrict__ v_scale,
                                                                _Float16 *__restrict__ k_out, _Float16 *__restrict__ v_out, size_t first,
                                                                size_t heads, int whole, int lanes)
{
    const uint8_t *codes = (blockIdx.y ? v : k) + first * lanes * 8;
    const _Float16 *scales = (blockIdx.y ? v_scale : k_scale) + first;
    _Float16 *out = blockIdx.y ? v_out : k_out;
    const size_t head0 = (size_t)blockIdx.x * whole;
    const int here = (int)(heads - head0 < (size_t)whole ? heads - head0 : (size_t)whole) * lanes;   // chunks of eight codes
    for (int c = threadIdx.x; c < here; c += kReadThreads) {
        const size_t at = head0 * lanes + c;
        const u32x2 w = *reinterpret_cast<const u32x2 *>(codes + at * 8);
        const _Float16 s = scales[head0 + c / lanes];
        half2v n[4];
        kv8_numbers<FMT>(w[0], n[0], n[1]);
        kv8_numbers<FMT>(w[1], n[2], n[3]);
        half8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = n[e >> 1][e & 1] * s;
        *reinterpret_cast<half8 *>(out + at * 8) = y;
    }
}

// ---- greedy acceptance and compaction of an 8-bit cache ----------------------------------------------------
// The walk of tree_accept (one wavefront, lane i = node i); then the accepted rows' codes, 8 bytes per thread and pass, and scales move to the front
// in path order: path[j] >= j and the path is increasing, so a row is read before it is overwritten, and threads share no bytes.
// It is bound by that order, one trip to memory per accepted node and pass: 8 heads of 128, back to back, 2.0 us for the root alone, 3.6 for 4 accepted nodes,
// 5.0 for 7, 7.5 for 12, 17 for 30 (tree_accept, 16 bytes per thread: 1.9, 2.6, 3.3, 4.4 and 8.9); a call of up to 7 takes 5.5, the host's part of a launch.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__global__ __launch_bounds__(256) void tree_accept_kv8_kernel(const int32_t *__restrict__ parent, const int32_t *__restrict__ token,
                                                              const int32_t *__restrict__ target, int M, int32_t *__restrict__ path,
                                                              int32_t *__restrict__ result, u32x2 *k, u32x2 *v, uint16_t *k_scale,
                                                              uint16_t *v_scale, int P, int Hkv, int chunks)
{
    __shared__ int32_t path_sh[64];
    __shared__ int32_t n_sh;
    const int tid = threadIdx.x;
    if (tid < 64) {
        const bool node = tid < M;
        const int32_t my_parent = node ? parent[tid] : -2, my_token = node ? token[tid] : 0, my_target = node ? target[tid] : 0;
        int cur = 0, n = 1;
        int32_t mine = tid == 0 ? 0 : -1;
        for (;;) {   // cur grows strictly: at most M rounds
            const int32_t want = __shfl(my_target, cur, 64);
            const uint64_t hits = __ballot(node && tid > cur && my_parent == cur && my_token == want);
            if (hits == 0) break;
            cur = __builtin_ctzll(hits);
            if (tid == n) mine = cur;
            ++n;
        }
        const int32_t next_token = __shfl(my_target, cur, 64);
        path_sh[tid] = mine;
        if (node) path[tid] = mine;
        if (tid == 0) {
            n_sh = n;
            result[0] = n;
            result[1] = next_token;
        }
    }
    __syncthreads();
    const int n = n_sh;
    for (int item = tid; item < 2 * (chunks + Hkv); item += 256) {
        const bool value = item >= chunks + Hkv;
        const int at = value ? item - chunks - Hkv : item;
        if (at < chunks) {
            u32x2 *base = (value ? v : k) + (size_t)P * chunks + at;
            for (int j = 1; j < n; ++j)
                if (path_sh[j] != j) base[(size_t)j * chunks] = base[(size_t)path_sh[j] * chunks];
        } else {
            uint16_t *base = (value ? v_scale : k_scale) + (size_t)P * Hkv + (at - chunks);
            for (int j = 1; j < n; ++j)
                if (path_sh[j] != j) base[(size_t)j * Hkv] = base[(size_t)path_sh[j] * Hkv];
        }
    }
}

// checks of the two appends; D: a lane holds four pairs, a wavefront at most one head
static int check_append(const void *qkv, const void *q_gamma, const void *k_gamma, float eps, const int32_t *pos, const float *cos_table,
                        const float *sin_table, int n_pos, const void *q, const void *k, const void *v, int M, int P, int Hq, int Hkv, int D)
{
    if (M < 1 || P < 0 || Hq < 1 || Hkv < 1 || D < 8 || D % 8 != 0 || n_pos < 1) return W4A16_EINVAL;
    if (M > 65535 || D > 512 || P > (1 << 30) || Hq > (1 << 20) || Hkv > (1 << 20)) return W4A16_EUNSUP;
    if (!qkv || !pos || !cos_table || !sin_table || !q || !k || !v) return W4A16_ENULL;
    if ((q_gamma == nullptr) != (k_gamma == nullptr)) return W4A16_ENULL;
    if (q_gamma && !(eps >= 0.f)) return W4A16_EINVAL;
    if (misaligned(qkv) || misaligned(q_gamma) || misaligned(k_gamma) || misaligned(cos_table) || misaligned(sin_table) || misaligned(q) ||
        misaligned(k) || misaligned(v) || (reinterpret_cast<uintptr_t>(pos) & 3u))
        return W4A16_EALIGN;
    return W4A16_OK;
}

}  // namespace w4

using namespace w4;

extern "C" {

int rope_append_qk_norm(const void *qkv, const void *q_gamma, const void *k_gamma, float eps, const int32_t *pos, const float *cos_table,
                        const float *sin_table, int n_pos, void *q, void *k_cache, void *v_cache, int M, int P, int Hq, int Hkv, int D,
                        void *stream)
{
    const int rc = check_append(qkv, q_gamma, k_gamma, eps, pos, cos_table, sin_table, n_pos, q, k_cache, v_cache, M, P, Hq, Hkv, D);
    if (rc != W4A16_OK) return rc;
    if (!q_gamma) return W4A16_ENULL;   // without norms this is rope_append
    const AppendArgs a = {(const _Float16 *)qkv, (const _Float16 *)q_gamma, (const _Float16 *)k_gamma, pos, cos_table, sin_table, (_Float16 *)q,
                          k_cache, v_cache, nullptr, nullptr, eps, n_pos, P, Hq, Hkv, D};
    return launch_append<kFp16Cache>(a, M, (hipStream_t)stream);
}

int rope_append_kv8(const void *qkv, const void *q_gamma, const void *k_gamma, float eps, const int32_t *pos, const float *cos_table,
               const float *sin_table, int n_pos, void *q, void *k, void *v, void *k_scale, void *v_scale, int format, int M, int P, int Hq,
               int Hkv, int D, void *stream)
{
    if (!kv8_format_known(format)) return W4A16_EINVAL;
    const int rc = check_append(qkv, q_gamma, k_gamma, eps, pos, cos_table, sin_table, n_pos, q, k, v, M, P, Hq, Hkv, D);
    if (rc != W4A16_OK) return rc;
    if (!k_scale || !v_scale) return W4A16_ENULL;
    if (misaligned(k_scale) || misaligned(v_scale)) return W4A16_EALIGN;
    const AppendArgs a = {(const _Float16 *)qkv, (const _Float16 *)q_gamma, (const _Float16 *)k_gamma, pos, cos_table, sin_table, (_Float16 *)q,
                          k, v, (_Float16 *)k_scale, (_Float16 *)v_scale, eps, n_pos, P, Hq, Hkv, D};
    return format == kInt8 ? launch_append<kInt8>(a, M, (hipStream_t)stream) : launch_append<kE4m3>(a, M, (hipStream_t)stream);
}

int w4a16_kv8_read(const void *k, const void *v, const void *k_scale, const void *v_scale, int format, int first, int rows, int Hkv, int D, void *k_out,
             void *v_out, void *stream)
{
    if (!kv8_format_known(format) || first < 0 || rows < 0 || Hkv < 1 || D < 8 || D % 8 != 0) return W4A16_EINVAL;
    if (D > 512 || first > (1 << 30) || rows > (1 << 30) || Hkv > (1 << 20)) return W4A16_EUNSUP;
    if (!k || !v || !k_scale || !v_scale || !k_out || !v_out) return W4A16_ENULL;
    if (misaligned(k) || misaligned(v) || misaligned(k_scale) || misaligned(v_scale) || misaligned(k_out) || misaligned(v_out)) return W4A16_EALIGN;
    if (rows == 0) return W4A16_OK;
    const int lanes = D / 8, whole = kReadThreads * kReadPasses / lanes;   // at least 16 heads
    const size_t heads = (size_t)rows * Hkv, groups = (heads + whole - 1) / whole;
    if (groups >= (1u << 24)) return W4A16_EUNSUP;   // 2^32 threads: more than 128 GiB of codes
    hipLaunchKernelGGL(format == kInt8 ? kv8_read_kernel<kInt8> : kv8_read_kernel<kE4m3>, dim3((unsigned)groups, 2), dim3(kReadThreads), 0,
                       (hipStream_t)stream, (const uint8_t *)k, (const uint8_t *)v, (const _Float16 *)k_scale, (const _Float16 *)v_scale,
                       (_Float16 *)k_out, (_Float16 *)v_out, (size_t)first * Hkv, heads, whole, lanes);
    return launch_status();
}

int tree_accept_kv8(const int32_t *parent, const int32_t *token, const int32_t *target, int M, int32_t *path, int32_t *result, void *k, void *v,
                    void *k_scale, void *v_scale, int P, int Hkv, int D, void *stream)
{
    if (M < 1 || P < 0 || Hkv < 1 || D < 8 || D % 8 != 0) return W4A16_EINVAL;
    if (M > W4A16_MAX_M || D > 512 || P > (1 << 30) || Hkv > (1 << 20)) return W4A16_EUNSUP;
    if (!parent || !token || !target || !path || !result || !k || !v || !k_scale || !v_scale) return W4A16_ENULL;
    if (misaligned(k) || misaligned(v) || misaligned(k_scale) || misaligned(v_scale)) return W4A16_EALIGN;
    if ((reinterpret_cast<uintptr_t>(parent) | reinterpret_cast<uintptr_t>(token) | reinterpret_cast<uintptr_t>(target) |
         reinterpret_cast<uintptr_t>(path) | reinterpret_cast<uintptr_t>(result)) & 3u)
        return W4A16_EALIGN;
    hipLaunchKernelGGL(tree_accept_kv8_kernel, dim3(1), dim3(256), 0, (hipStream_t)stream, parent, token, target, M, path, result, (u32x2 *)k,
                       (u32x2 *)v, (uint16_t *)k_scale, (uint16_t *)v_scale, P, Hkv, Hkv * D / 8);
    return launch_status();
}

}  // extern "C"
