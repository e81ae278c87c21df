// w4a16_pack / w4a16_unpack / w4a16_dequant: layout conversion kernels (offline, not on the timed
// path) and the bit-exact dequantisation test export.  See layout.h for the packed layout and
// include/w4a16.h for the contracts.
#include "internal.h"
#include "shared_entries.inc"
#include <hip/hip_fp16.h>
#include <string.h>

namespace w4 {

__device__ __forceinline__ uint32_t permute_fields_to_packed(uint32_t canon)
{
    uint32_t out = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) out |= ((canon >> (4 * p)) & 0xFu) << (4 * field_of_p(p));
    return out;
}

__device__ __forceinline__ uint32_t permute_fields_to_canonical(uint32_t packed)
{
    uint32_t out = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) out |= ((packed >> (4 * field_of_p(p))) & 0xFu) << (4 * p);
    return out;
}

// canonical column held at packed column n (n < N): n itself, or -- paired layout, pair_block > 0 -- inside
// every block of pair_block columns the tiles of the block's two halves alternate: packed tile 2j of the
// block is tile j of its first half, packed tile 2j+1 tile j of its second half.  pair_block = N pairs a
// gate projection with its up projection; pair_block = head_dim pairs the two halves of every head.
__device__ __forceinline__ int source_column(int n, int N, int pair_block)
{
    if (!pair_block) return n;
    const int block = n / pair_block, within = n - block * pair_block;
    const int tile = within >> 4;
    return block * pair_block + (tile & 1) * (pair_block >> 1) + (tile >> 1) * 16 + (within & 15);
}

// one thread per (record, tile, lane): writes the lane's 16 bytes of codes; threads with t == 0
// and r == 0 also write the record's scales and zero-points for their column index c.
__global__ void pack_kernel(const uint32_t *__restrict__ qweight, const uint16_t *__restrict__ scales,
                            const uint32_t *__restrict__ qzeros, uint8_t *__restrict__ packed,
                            int N, int K, long long total, int pair_block)
{
    long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (idx >= total) return;
    const int groups = K / kGroup;
    int lane = (int)(idx & 63);
    int t = (int)((idx >> 6) & 7);
    long long rec = idx >> 9;
    int g = (int)(rec % groups);
    int nb = (int)(rec / groups);
    int r = lane >> 4, c = lane & 15;
    int n = nb * kBlockCols + t * 16 + c;
    uint8_t *base = packed + record_offset(nb, g, groups);
    uint4 w = make_uint4(0, 0, 0, 0);
    const int src = n < N ? source_column(n, N, pair_block) : 0;
    if (n < N) {
        uint32_t v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            int kw = g * 16 + j * 4 + r;  // canonical word row: rows 8*kw .. 8*kw+7
            v[j] = permute_fields_to_packed(qweight[(size_t)kw * N + src]);
        }
        w = make_uint4(v[0], v[1], v[2], v[3]);
    }
    *reinterpret_cast<uint4 *>(base + t * 1024 + lane * 16) = w;
    if (r == 0) {
        uint16_t s = (n < N) ? scales[(size_t)g * N + src] : (uint16_t)0;
        *reinterpret_cast<uint16_t *>(base + kScalesOff + c * 16 + t * 2) = s;
        if (t == 0) {
            uint32_t zw = 0;
#pragma unroll
            for (int tt = 0; tt < 8; ++tt) {
                int nn = nb * kBlockCols + tt * 16 + c;
                uint32_t z = 0;
                if (nn < N) {
                    const int ns = source_column(nn, N, pair_block);
                    z = (qzeros[(size_t)g * (N / 8) + (ns >> 3)] >> (4 * (ns & 7))) & 0xFu;
                }
                zw |= z << (4 * tt);
            }
            *reinterpret_cast<uint32_t *>(base + kZerosOff + c * 4) = zw;
        }
    }
}

// one thread per canonical qweight word [kw, n]; the first K/128 rows of threads also restore
// scales, and threads with n % 8 == 0 restore a qzeros word.
__global__ void unpack_kernel(const uint8_t *__restrict__ packed, uint32_t *__restrict__ qweight,
                              uint16_t *__restrict__ scales, uint32_t *__restrict__ qzeros,
                              int N, int K, long long total)
{
    long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (idx >= total) return;
    const int groups = K / kGroup;
    int n = (int)(idx % N);
    int kw = (int)(idx / N);
    int g = kw >> 4, j = (kw >> 2) & 3, r = kw & 3;
    int nb = n / kBlockCols, t = (n % kBlockCols) >> 4, c = n & 15;
    const uint8_t *base = packed + record_offset(nb, g, groups);
    uint32_t pw = *reinterpret_cast<const uint32_t *>(base + t * 1024 + (r * 16 + c) * 16 + j * 4);
    qweight[(size_t)kw * N + n] = permute_fields_to_canonical(pw);
    if ((kw & 15) == 0) {
        scales[(size_t)g * N + n] = *reinterpret_cast<const uint16_t *>(base + kScalesOff + c * 16 + t * 2);
        if ((n & 7) == 0) {
            uint32_t zw = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {  // columns n .. n+7 share nb and t; c runs over c .. c+7
                uint32_t pz = *reinterpret_cast<const uint32_t *>(base + kZerosOff + (c + i) * 4);
                zw |= ((pz >> (4 * t)) & 0xFu) << (4 * i);
            }
            qzeros[(size_t)g * (N / 8) + (n >> 3)] = zw;
        }
    }
}

// one thread per element W[k, n]
__global__ void dequant_kernel(const uint8_t *__restrict__ packed, float *__restrict__ W,
                               int N, int K, long long total)
{
    long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (idx >= total) return;
    const int groups = K / kGroup;
    int n = (int)(idx % N);
    int k = (int)(idx / N);
    int g = k / kGroup, kk = k % kGroup;
    int j = kk >> 5, r = (kk >> 3) & 3, p = kk & 7;
    int nb = n / kBlockCols, t = (n % kBlockCols) >> 4, c = n & 15;
    const uint8_t *base = packed + record_offset(nb, g, groups);
    uint32_t pw = *reinterpret_cast<const uint32_t *>(base + t * 1024 + (r * 16 + c) * 16 + j * 4);
    int q = (int)((pw >> (4 * field_of_p(p))) & 0xFu);
    uint32_t pz = *reinterpret_cast<const uint32_t *>(base + kZerosOff + c * 4);
    int z = (int)((pz >> (4 * t)) & 0xFu);
    __half s = *reinterpret_cast<const __half *>(base + kScalesOff + c * 16 + t * 2);
    W[idx] = (float)(q - z) * __half2float(s);
}

// *flag = 1 unless some zero-point of a real column differs from 8 (thread = one zero-point word: the eight
// tiles of one column position of one record).  Threads that find a difference all store the same 0.
__global__ void symmetric_begin_kernel(int32_t *flag) { *flag = 1; }
__global__ __launch_bounds__(256) void symmetric_check_kernel(const uint8_t *__restrict__ packed, int32_t *flag, int N,
                                                              int groups, size_t words)
{
    const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= words) return;
    const size_t record = i >> 4;
    const int c = (int)(i & 15), nb = (int)(record / (size_t)groups);
    const uint32_t z = *reinterpret_cast<const uint32_t *>(packed + record * kRecordBytes + kZerosOff + c * 4);
    bool all8 = true;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
        if (nb * kBlockCols + t * 16 + c < N && ((z >> (4 * t)) & 0xFu) != 8u) all8 = false;
    if (!all8) *flag = 0;
}

// plain streaming read of `n16` 16-byte words: the bandwidth ceiling the GEMM is compared with.
// Workgroup b reads the contiguous 32 KB chunk b with all of its loads in flight at once, the
// fastest of the patterns tried on this GPU (strided grids and larger chunks were slower).
typedef uint32_t probe_word __attribute__((ext_vector_type(4)));
constexpr size_t kProbeChunk16 = 2048;   // 16-byte words per workgroup
__global__ __launch_bounds__(256) void read_probe_kernel(const probe_word *__restrict__ p, size_t n16, uint32_t *sink)
{
    const size_t base = (size_t)blockIdx.x * kProbeChunk16 + threadIdx.x;
    uint32_t acc = 0;
    if (base - threadIdx.x + kProbeChunk16 <= n16) {
        probe_word v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = __builtin_nontemporal_load(p + base + u * 256);
#pragma unroll
        for (int u = 0; u < 8; ++u) acc ^= v[u].x ^ v[u].y ^ v[u].z ^ v[u].w;
    } else {
        for (size_t i = base; i < n16; i += 256) {
            const probe_word v = __builtin_nontemporal_load(p + i);
            acc ^= v.x ^ v.y ^ v.z ^ v.w;
        }
    }
    if (acc == 0x9E3779B9u) *sink = acc;   // keeps the loads alive; practically never taken
}

static Params g_params;
Params &params() { return g_params; }

}  // namespace w4

using namespace w4;

extern "C" {

int w4a16_version(void) { return 100; }

static int *param_slot(const char *name)
{
    if (!name) return nullptr;
    Params &p = params();
    if (!strcmp(name, "split_k")) return &p.split_k;
    if (!strcmp(name, "fused_reduce")) return &p.fused_reduce;
    if (!strcmp(name, "attn_splits")) return &p.attn_splits;
    if (!strcmp(name, "attn_pack")) return &p.attn_pack;
    if (!strcmp(name, "attn_fused_merge")) return &p.attn_fused_merge;
    if (!strcmp(name, "lm_tiles")) return &p.lm_tiles;
    if (!strcmp(name, "attn_row_tiles")) return &p.attn_row_tiles;
    if (!strcmp(name, "tiles_per_wave")) return &p.tiles_per_wave;
    if (!strcmp(name, "waves_per_wg")) return &p.waves_per_wg;
    if (!strcmp(name, "prefetch_depth")) return &p.prefetch_depth;
    if (!strcmp(name, "k_sets")) return &p.k_sets;
    if (!strcmp(name, "even_split")) return &p.even_split;
    if (!strcmp(name, "flat_groups")) return &p.flat_groups;
    return nullptr;
}

int w4a16_set_param(const char *name, int value)
{
    int *slot = param_slot(name);
    if (!slot || value < 0 || value > 1024) return W4A16_EINVAL;
    if (slot == &params().tiles_per_wave && value != 0 && value != 2 && value != 4 && value != 8) return W4A16_EINVAL;
    *slot = value;
    return W4A16_OK;
}

int w4a16_get_param(const char *name)
{
    int *slot = param_slot(name);
    return slot ? *slot : W4A16_EINVAL;
}

size_t w4a16_packed_bytes(int N, int K, int G)
{
    if (check_weight_shape(N, K, G) != W4A16_OK) return 0;
    return (size_t)(pad_cols(N) / kBlockCols) * (size_t)(K / kGroup) * (size_t)kRecordBytes;
}

int w4a16_weight_is_symmetric(const void *packed, int N, int K, int G, int32_t *flag, void *stream)
{
    int rc = check_weight_shape(N, K, G);
    if (rc != W4A16_OK) return rc;
    if (!packed || !flag) return W4A16_ENULL;
    if (misaligned(packed) || (reinterpret_cast<uintptr_t>(flag) & 3u)) return W4A16_EALIGN;
    const int groups = K / kGroup;
    const size_t words = (size_t)(pad_cols(N) / kBlockCols) * groups * 16;
    hipLaunchKernelGGL(symmetric_begin_kernel, dim3(1), dim3(1), 0, (hipStream_t)stream, flag);
    hipLaunchKernelGGL(symmetric_check_kernel, dim3((unsigned)((words + 255) / 256)), dim3(256), 0, (hipStream_t)stream,
                       (const uint8_t *)packed, flag, N, groups, words);
    return launch_status();
}

int w4a16_read_probe(const void *buf, size_t bytes, void *sink, void *stream)
{
    if (!buf || !sink) return W4A16_ENULL;
    if (misaligned(buf) || (reinterpret_cast<uintptr_t>(sink) & 3u)) return W4A16_EALIGN;
    if (bytes < 16) return W4A16_EINVAL;
    const size_t n16 = bytes / 16, wgs = (n16 + kProbeChunk16 - 1) / kProbeChunk16;
    if (wgs > 0x7fffffffu) return W4A16_EUNSUP;
    hipLaunchKernelGGL(read_probe_kernel, dim3((unsigned)wgs), dim3(256), 0, (hipStream_t)stream,
                       (const probe_word *)buf, n16, (uint32_t *)sink);
    return launch_status();
}

static int pack_entry(const int32_t *qweight, const void *scales, const int32_t *qzeros, void *packed,
                      int N, int K, int G, void *stream, int pair_block)
{
    int rc = check_weight_shape(N, K, G);
    if (rc != W4A16_OK) return rc;
    if (pair_block && (pair_block < 32 || pair_block % 32 != 0 || N % pair_block != 0)) return W4A16_EINVAL;
    if (!qweight || !scales || !qzeros || !packed) return W4A16_ENULL;
    if (misaligned(qweight) || misaligned(scales) || misaligned(qzeros) || misaligned(packed)) return W4A16_EALIGN;
    long long total = (long long)(pad_cols(N) / kBlockCols) * (K / kGroup) * 512;
    hipLaunchKernelGGL(pack_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, (hipStream_t)stream,
                       (const uint32_t *)qweight, (const uint16_t *)scales, (const uint32_t *)qzeros,
                       (uint8_t *)packed, N, K, total, pair_block);
    return launch_status();
}

int w4a16_pack(const int32_t *qweight, const void *scales, const int32_t *qzeros, void *packed,
               int N, int K, int G, void *stream)
{
    return pack_entry(qweight, scales, qzeros, packed, N, K, G, stream, 0);
}

int w4a16_pack_gate_up(const int32_t *qweight, const void *scales, const int32_t *qzeros, void *packed,
                       int N, int K, int G, void *stream)
{
    return pack_entry(qweight, scales, qzeros, packed, N, K, G, stream, N > 0 ? N : 1);
}

int w4a16_pack_heads(const int32_t *qweight, const void *scales, const int32_t *qzeros, void *packed,
                     int N, int K, int G, int head_dim, void *stream)
{
    if (head_dim < 32) return W4A16_EINVAL;
    return pack_entry(qweight, scales, qzeros, packed, N, K, G, stream, head_dim);
}

int w4a16_unpack(const void *packed, int32_t *qweight, void *scales, int32_t *qzeros,
                 int N, int K, int G, void *stream)
{
    int rc = check_weight_shape(N, K, G);
    if (rc != W4A16_OK) return rc;
    if (!qweight || !scales || !qzeros || !packed) return W4A16_ENULL;
    if (misaligned(qweight) || misaligned(scales) || misaligned(qzeros) || misaligned(packed)) return W4A16_EALIGN;
    long long total = (long long)(K / 8) * N;
    hipLaunchKernelGGL(unpack_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, (hipStream_t)stream,
                       (const uint8_t *)packed, (uint32_t *)qweight, (uint16_t *)scales, (uint32_t *)qzeros,
                       N, K, total);
    return launch_status();
}

int w4a16_dequant(const void *packed, float *W, int N, int K, int G, void *stream)
{
    int rc = check_weight_shape(N, K, G);
    if (rc != W4A16_OK) return rc;
    if (!packed || !W) return W4A16_ENULL;
    if (misaligned(packed) || misaligned(W)) return W4A16_EALIGN;
    long long total = (long long)K * N;
    if ((total + 255) / 256 > 0x7FFFFFFFll) return W4A16_EUNSUP;
    hipLaunchKernelGGL(dequant_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, (hipStream_t)stream,
                       (const uint8_t *)packed, W, N, K, total);
    return launch_status();
}

}  // extern "C"
