// tree_verify_attn_kv8: attention of the tree-verification pass over an 8-bit cache (kv8.h) on gfx950.
//
// The mathematics is that of tree_verify_attn (attn.hip): S^T = K . Q^T, softmax online in fp32, O^T += V^T . P^T with 32x32x16 fp16
// matrix steps.  Codes become fp16 numbers exactly, so the products see the numbers that w4a16_kv8_read returns; probabilities are rounded to fp16 for
// the second product, sums and running maxima are fp32.
#include <type_traits>

#include "attn_common.h"
#include "kv8.h"

namespace w4 {

constexpr int kWaves = 8;

// lane l's two bytes at src land, zero-extended, at lds_base + 4 l (lds_base wavefront-uniform; counted by vmcnt)
__device__ __forceinline__ void half_to_lds(const _Float16 *src, uint8_t *lds_base)
{
    __builtin_amdgcn_global_load_lds((global_void *)src, (lds_void *)lds_base, 2, 0, 0);
}

// The transposing read of 8-bit elements: in each block of 16 lanes, lane s points at eight consecutive head-dim elements 8 (s % 2) .. of
// the block's key row s / 2, and lane c receives element c of the eight rows.  Assembly for the reason given in attn.hip.
template <int OFFSET>
__device__ __forceinline__ void read_transposed_codes(u32x2 &w, uint32_t lds_addr)
{
    asm volatile("ds_read_b64_tr_b8 %0, %1 offset:%2" : "=&v"(w) : "v"(lds_addr), "n"(OFFSET));
}
template <int N>
__device__ __forceinline__ void wait_lds_reads(u32x2 &w)
{
    asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(w) : "n"(N));
}

// Clears the V codes, in LDS, of some keys of a step: those that no row of the tile sees (such rows of the cache may never have been written) and those that
// keys_without_numbers finds.  A probability of zero would not keep e4m3's NaN codes, or products beyond fp16, out of the rows' sums.
__device__ __forceinline__ void clear_codes(uint8_t *tile, uint32_t keys, int lane)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((keys >> (8 * i + (lane >> 3))) & 1u) *reinterpret_cast<u32x4 *>(tile + i * 1024 + lane * 16) = (u32x4){0, 0, 0, 0};
    asm volatile("" ::: "memory");
}
// The keys of a step, in LDS, with V codes that are no numbers under their scales.  Nearly always there are none, and nothing but the first look is taken.
template <int FMT>
__device__ __forceinline__ uint32_t keys_without_numbers(const uint8_t *tile, const uint32_t *scales, int lane)
{
    bool suspect = false;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        suspect |= kv8_suspect<FMT>(FMT == kInt8 ? (u32x4){} : *reinterpret_cast<const u32x4 *>(tile + i * 1024 + lane * 16), scales[8 * i + (lane >> 3)]);
    uint32_t keys = 0;
    if (__builtin_expect(__any(suspect), 0)) {   // uniform
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            const uint64_t lanes = __ballot(kv8_no_numbers<FMT>(*reinterpret_cast<const u32x4 *>(tile + i * 1024 + lane * 16), scales[8 * i + (lane >> 3)]));
#pragma unroll 1
            for (int r = 0; r < 8; ++r) keys |= (uint32_t)(((lanes >> (8 * r)) & 0xFFu) != 0) << (8 * i + r);
        }
    }
    return keys;
}

// ---- row tiles of at most 32 rows: wavefronts with K and V tiles of their own -------------------------------
// As tree_attn_wave_kernel: eight wavefronts carry the same 32 rows, wavefront w takes key steps w, w + 8, ... of the workgroup's range and
// meets the others only at the end.  A step is 32 keys: 4 KB of K codes, 4 KB of V codes and 64 scales, brought straight to LDS one step
// ahead of their use (two buffers per wavefront; two steps ahead was no faster over long prefixes and 0.3 us slower over short ones).
// What bounds it: with few rows over a long prefix, memory (7 rows of 32/8 heads over 131072 keys: 268 MB of codes in 53 us, 5.0 TB/s, as fast as 128-byte
// pieces can be read: a kernel that does nothing else takes 53 to 56); over a short
// one, its own length (1 row of 64/8 heads over 2049 keys: 9 us, of which the walk takes 3.5, arguments, mask and Q 2, the merges 2.5); with many rows
// the turning of codes into numbers, which every 32 rows do again.
//   K fragments   lane (c, h) of a pair of matrix steps takes the 16 codes of chunk 2 j + h of key c: its first eight are slots 8 h .. of the first
//                 step, the others of the second (any order of the contraction serves, Q's fragments follow it)
//   V^T fragments through the transposing read: eight keys at one head-dim element
// 16-byte chunks of a key row are stored at chunk ^ (key / 2 % 8): rows are 128 B, so sixteen keys' equal chunks fill all banks.
constexpr int kWaveTile = kKeyBlock * kHeadDim;            // codes of a K or V tile
constexpr int kWaveBuf = 2 * kWaveTile + 64 * 4;           // K codes, V codes, 32 K and 32 V scales (4 bytes each)
constexpr int kWaveTiles = kWaves * 2 * kWaveBuf;
constexpr int kWaveRows = 32;
constexpr int kExRow = kHeadDim * 4 + 16;                  // exchange row: 128 fp32 + 16 B of padding
constexpr int kExWave = kWaveRows * kExRow;
constexpr int kWaveState = kWaves * kExWave;               // [row][wavefront] (max, sum), then [row][wavefront] (weight, weighted sum)
constexpr int kWaveWeights = kWaveState + kWaveRows * kWaves * 8;
constexpr int kWaveEnd = kWaveWeights + kWaveRows * kWaves * 8;
constexpr int kWaveLds = kWaveTiles > kWaveEnd ? kWaveTiles : kWaveEnd;
typedef float float2v __attribute__((ext_vector_type(2)));
// Running maxima are left behind the true ones by up to this many binary orders of magnitude: probabilities reach 2^8 then, which fp16 and the sums hold
// as well as 1, and sums and outputs are rescaled a few times in all, not in most steps.
constexpr float kBehind = 8.f;
// A row whose mask row is empty is padding and sees nothing, committed keys included.  Only ranges with draft keys read the mask (in the others it would cost
// up to 1.2 us of 15): they give such rows kPaddingMark for a sum, and whoever joins the ranges writes zeros.

struct Kv8Args {
    uint32_t by_tiles, by_ranges;   // divider() of tiles_per_kv and nsplit
    const _Float16 *q;
    const uint8_t *k, *v;
    const _Float16 *k_scale, *v_scale;
    const uint8_t *mask;
    _Float16 *out;
    float *part_o, *part_ml;
    uint32_t *tickets;
    int M, P, Hq, Hkv, group;
    float scale_log2e;
    int nsplit, bq, brem;           // key ranges; steps of each, the first brem one more
    int tile_rows, tiles_per_kv, fused;
};

template <int FMT>
__global__ __launch_bounds__(64 * kWaves) void tree_attn_kv8_wave_kernel(const Kv8Args a)
{
    extern __shared__ float4v smem4[];
    uint8_t *lds = reinterpret_cast<uint8_t *>(smem4);
    const int M = a.M, P = a.P, T = P + M;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, c = lane & 31;
    const Share share(blockIdx.x, (unsigned)(a.Hkv * a.tiles_per_kv * a.nsplit), a.nsplit, a.tiles_per_kv, a.by_tiles, a.by_ranges);
    const int kvh = share.kvh, unit = kvh * a.tiles_per_kv + share.tile, sp = share.range;
    const RowTile tile(kvh, share.tile, M, a.Hq, a.group, a.tile_rows);
    const int b0 = sp * a.bq + (sp < a.brem ? sp : a.brem), b1 = b0 + a.bq + (sp < a.brem ? 1 : 0);
    const size_t kv_row_bytes = (size_t)a.Hkv * kHeadDim;
    int my_row, my_head;
    tile.locate(c, my_row, my_head);

    // tree mask of the draft keys, one 64-bit word per query row: bytes requested first, words made of them behind the transfers
    __shared__ uint64_t row_bits[kRowsPad];
    const bool reaches_draft = b1 * kKeyBlock > P;   // uniform over the workgroup
    uint32_t mask_byte[8] = {};
    if (reaches_draft) {
        const int mcol = min(lane, M - 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) mask_byte[i] = a.mask[(size_t)min(wave * 8 + i, M - 1) * M + mcol];
    }
    // Q fragments (second operand of S^T): steps 2 j and 2 j + 1 take the halves of chunk 2 j + h of the row
    half8v qf[8];
    {
        const _Float16 *row = a.q + ((size_t)my_row * a.Hq + my_head) * kHeadDim + 16 * h;
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[j] = *reinterpret_cast<const half8v *>(row + 32 * (j >> 1) + 8 * (j & 1));
    }
    // transfers: lane l of transfer i fills 16 l .. of 1 KB: chunk position l % 8 of key 8 i + l / 8
    uint8_t *const mine = lds + wave * 2 * kWaveBuf;
    const uint8_t *const k_src = a.k + (size_t)kvh * kHeadDim, *const v_src = a.v + (size_t)kvh * kHeadDim;
    const _Float16 *const s_src = (h ? a.v_scale : a.k_scale) + kvh;   // lane (c, 0) brings key c's K scale, lane (c, 1) its V scale
    const int trow = lane >> 3, tchunk = lane & 7;
    uint32_t lane_src[2];   // the chunk permutation depends on the transfer's parity only
#pragma unroll
    for (int par = 0; par < 2; ++par) lane_src[par] = (uint32_t)trow * (uint32_t)kv_row_bytes + (uint32_t)((tchunk ^ ((4 * par + (trow >> 1)) & 7)) << 4);
    auto request = [&](int step, int buf) {
        const int key0 = step * kKeyBlock;
        uint8_t *dst = mine + buf * kWaveBuf;
        half_to_lds(s_src + (size_t)min(key0 + c, T - 1) * a.Hkv, dst + 2 * kWaveTile);
        if (key0 + kKeyBlock <= T) {   // uniform
            const size_t at = (size_t)key0 * kv_row_bytes;
#pragma unroll
            for (int i = 0; i < 4; ++i) row_to_lds(k_src + at + (size_t)(8 * i) * kv_row_bytes + lane_src[i & 1], dst + i * 1024);
#pragma unroll
            for (int i = 0; i < 4; ++i) row_to_lds(v_src + at + (size_t)(8 * i) * kv_row_bytes + lane_src[i & 1], dst + kWaveTile + i * 1024);
        } else {   // the last step of all: rows beyond the last key repeat it (they are hidden below)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const size_t at = (size_t)min(key0 + 8 * i + trow, T - 1) * kv_row_bytes + ((tchunk ^ ((4 * i + (trow >> 1)) & 7)) << 4);
                row_to_lds(k_src + at, dst + i * 1024);
                row_to_lds(v_src + at, dst + kWaveTile + i * 1024);
            }
        }
    };
    int step = b0 + wave;
    if (step < b1) request(step, 0);
    uint64_t mbits = 0;
    if (reaches_draft) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            asm volatile("" : "+v"(mask_byte[i]));
            const uint64_t bits = __ballot(mask_byte[i] != 0 && wave * 8 + i < M && lane < M);
            if (lane == i) row_bits[wave * 8 + i] = bits;
        }
        __syncthreads();
        mbits = row_bits[my_row];
    }
    const uint32_t kfrag = (uint32_t)(c * kHeadDim + ((h ^ ((c >> 1) & 7)) << 4));   // chunk 2 j + h: ^ (j << 5)
    // V: in 16-lane block b, lane s points at key 4 (b / 2) + r (r = s / 2 < 4) or 4 further on, chunk 2 dt + b % 2, bytes 8 (s % 2) ..
    const int vr = (lane & 15) >> 1, vkey = 4 * h + (vr < 4 ? vr : vr + 4);
    const uint32_t vfrag = (uint32_t)(vkey * kHeadDim + ((((lane >> 4) & 1) ^ ((vkey >> 1) & 7)) << 4) + 8 * (lane & 1));
    float16v o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    float m_run = kLowest, l_run = 0.f;   // l_run: this lane's share (its keys) of the row's sum

    int buf = 0;
    while (step < b1) {   // uniform over the wavefront; no barrier inside
        const int next = step + kWaves, key0 = step * kKeyBlock;
        asm volatile("" ::: "memory");
        if (next < b1) {
            request(next, buf ^ 1);
            asm volatile("s_waitcnt vmcnt(9)" ::: "memory");   // this step's tiles; the next step's nine transfers are newer
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const uint8_t *const tiles = mine + buf * kWaveBuf;
        const uint32_t *const scales = reinterpret_cast<const uint32_t *>(tiles + 2 * kWaveTile);
        // A scale that is no number marks a head that held an infinity or a NaN.  Such keys take no part in the products (a hidden one must
        // not reach the rows that do not see it): their scales are taken as zero and the scores of the rows that see them become NaN.
        const uint64_t nan_lanes = __ballot((scales[lane] & 0x7FFFu) >= kHalfInf);
        uint32_t bad = (uint32_t)nan_lanes | (uint32_t)(nan_lanes >> 32);   // bit i: key i of the step
        uint32_t ks = scales[c];
        if ((ks & 0x7FFFu) >= kHalfInf) ks = 0;
        const _Float16 k_scale = __builtin_bit_cast(_Float16, (uint16_t)ks);
        float16v sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(tiles + (kfrag ^ (j << 5)));
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                half2v n[4];
                kv8_values<FMT>(w[2 * e], k_scale, n[0], n[1]);
                kv8_values<FMT>(w[2 * e + 1], k_scale, n[2], n[3]);
                const half8v f = {n[0][0], n[0][1], n[1][0], n[1][1], n[2][0], n[2][1], n[3][0], n[3][1]};
                sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, qf[2 * j + e], sc, 0, 0, 0);
            }
        }
        // V scales in the order of the contraction: slots 8 h + p of product u are keys 16 u + 4 h + p, and 8 further on for p >= 4
        half8v vs[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            u32x4 s0 = *reinterpret_cast<const u32x4 *>(scales + 32 + 16 * u + 4 * h), s1 = *reinterpret_cast<const u32x4 *>(scales + 40 + 16 * u + 4 * h);
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                if (bad) {
                    if ((s0[p] & 0x7FFFu) >= kHalfInf) s0[p] = 0;
                    if ((s1[p] & 0x7FFFu) >= kHalfInf) s1[p] = 0;
                }
                vs[u][p] = __builtin_bit_cast(_Float16, (uint16_t)s0[p]);
                vs[u][4 + p] = __builtin_bit_cast(_Float16, (uint16_t)s1[p]);
            }
        }
        settled(sc);
        float s[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = sc[i];   // key 8 (i / 4) + 4 h + i % 4 of the step
        uint32_t seen = ~0u;
        if (key0 + kKeyBlock > P) {   // uniform: the step has draft keys; its first key is draft key `first` (negative: begins with committed keys)
            const int first = key0 - P;
            seen = (uint32_t)(first >= 0 ? mbits >> first : (mbits << -first) | ((1ull << -first) - 1));
            const uint32_t vis = seen >> (4 * h);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = ((vis >> (8 * (i >> 2) + (i & 3))) & 1u) ? s[i] : -__builtin_inff();
            uint8_t *const values = mine + buf * kWaveBuf + kWaveTile;
            uint32_t by_any = seen, strange = 0;   // keys that any row sees; keys whose values other rows are to be kept from (a single row has no others)
            if (M > 1) strange = keys_without_numbers<FMT>(values, scales + 32, lane);
#pragma unroll
            for (int off = 1; off < kWaveRows; off <<= 1) by_any |= (uint32_t)__shfl_xor((int)by_any, off, 64);
            bad |= strange;
            clear_codes(values, strange | ~by_any, lane);
        }
        if (bad) {   // uniform, rare
            const uint32_t hit = (seen & bad) >> (4 * h);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = ((hit >> (8 * (i >> 2) + (i & 3))) & 1u) ? __builtin_nanf("") : s[i];
        }
        // the scale is positive (checked by the host): the largest raw score is the largest scaled one
        const float m_a = max_of_three(max_of_three(s[0], s[1], s[2]), max_of_three(s[3], s[4], s[5]), max_of_three(s[6], s[7], s[8]));
        const float m_b = max_of_three(max_of_three(s[9], s[10], s[11]), max_of_three(s[12], s[13], s[14]), s[15]);
        const float m_step = half_wave_max(max_of_two(m_a, m_b)) * a.scale_log2e;
        if (__builtin_expect(__any(m_step > m_run + kBehind), 0)) {
            const float m_new = m_step > m_run + kBehind ? m_step : m_run;
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            l_run *= alpha;
            m_run = m_new;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
        }
        half8v pb[2];
        float sums[2] = {l_run, 0.f};
        const half2v ones = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const half2v p = {(_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale_log2e, -m_run)),
                              (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[i + 1], a.scale_log2e, -m_run))};
            pb[i >> 3][i & 7] = p[0];
            pb[i >> 3][(i & 7) + 1] = p[1];
            sums[(i >> 1) & 1] = __builtin_amdgcn_fdot2(p, ones, sums[(i >> 1) & 1], false);
        }
        l_run = sums[0] + sums[1];
        const uint32_t vtile = lds_address(tiles + kWaveTile);
        u32x2 w[8];
        auto read_v = [&](auto f) {
            constexpr int F = decltype(f)::value;
            read_transposed_codes<(F & 1) * 16 * kHeadDim>(w[F], vtile + (vfrag ^ ((F >> 1) << 5)));
        };
        auto product = [&](auto f) {
            constexpr int F = decltype(f)::value, U = F & 1;
            if constexpr (F + 2 < 8) read_v(std::integral_constant<int, F + 2>{});
            wait_lds_reads<F + 2 < 8 ? 2 : F + 1 < 8 ? 1 : 0>(w[F]);
            half2v n[4];
            kv8_numbers<FMT>(w[F][0], n[0], n[1]);
            kv8_numbers<FMT>(w[F][1], n[2], n[3]);
            const half8v x = {n[0][0], n[0][1], n[1][0], n[1][1], n[2][0], n[2][1], n[3][0], n[3][1]};
            o[F >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x * vs[U], pb[U], o[F >> 1], 0, 0, 0);
        };
        read_v(std::integral_constant<int, 0>{});
        read_v(std::integral_constant<int, 1>{});
        product(std::integral_constant<int, 0>{});
        product(std::integral_constant<int, 1>{});
        product(std::integral_constant<int, 2>{});
        product(std::integral_constant<int, 3>{});
        product(std::integral_constant<int, 4>{});
        product(std::integral_constant<int, 5>{});
        product(std::integral_constant<int, 6>{});
        product(std::integral_constant<int, 7>{});
        step = next;
        buf ^= 1;
    }

    // The states of the eight wavefronts meet in LDS; the weights are worked out once per (row, wavefront)
    l_run += __shfl_xor(l_run, 32, 64);
    if (reaches_draft && mbits == 0) l_run = kPaddingMark;
    __syncthreads();   // every wavefront has left its tiles
    uint8_t *const ex = lds + wave * kExWave;
    float2v *const state = reinterpret_cast<float2v *>(lds + kWaveState), *const weights = reinterpret_cast<float2v *>(lds + kWaveWeights);
    if (h == 0) state[c * kWaves + wave] = (float2v){m_run, l_run};
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            *reinterpret_cast<float4v *>(ex + c * kExRow + (8 * dt + 2 * b + h) * 16) =
                (float4v){o[dt][4 * b], o[dt][4 * b + 1], o[dt][4 * b + 2], o[dt][4 * b + 3]};
    __syncthreads();
    auto row_max = [&](int row) {
        float m_all = kLowest;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m_all = fmaxf(m_all, state[row * kWaves + w][0]);
        return m_all;
    };
    if (tid < kWaveRows * kWaves) {
        const float2v me = state[tid];
        const float wgt = __builtin_amdgcn_exp2f(me[0] - row_max(tid / kWaves));
        weights[tid] = me[1] < 0.f ? (float2v){0.f, kPaddingMark} : (float2v){wgt, wgt * me[1]};
    }
    __syncthreads();
    const bool last = a.nsplit == 1;
    const PartialBuffer unit_o = partial_buffer(a.part_o + (size_t)unit * a.nsplit * kWaveRows * kHeadDim);
    const PartialBuffer unit_ml = partial_buffer(a.part_ml + (size_t)unit * a.nsplit * kWaveRows * 2);
#pragma unroll
    for (int it = 0; it < 2; ++it) {   // thread t: four consecutive outputs of a row, 32 threads per row
        const int item = tid + it * (64 * kWaves);
        const int rho = item >> 5, quad = item & 31;
        float4v val = {0.f, 0.f, 0.f, 0.f};
        float l_all = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float2v wl = weights[rho * kWaves + w];
            l_all += wl[1];
            val += wl[0] * *reinterpret_cast<const float4v *>(lds + w * kExWave + rho * kExRow + quad * 16);
        }
        if (rho >= tile.rows) continue;
        if (l_all < 0.f) val = (float4v){0.f, 0.f, 0.f, 0.f}, l_all = kPaddingMark;
        if (last) {
            if (!(l_all < 0.f)) val *= 1.f / l_all;   // 0 / 0 where every score is -inf
            typedef _Float16 half4v __attribute__((ext_vector_type(4)));
            half4v hv = {(_Float16)val[0], (_Float16)val[1], (_Float16)val[2], (_Float16)val[3]};
            int qrow, head;
            tile.locate(rho, qrow, head);
            *reinterpret_cast<half4v *>(a.out + ((size_t)qrow * a.Hq + head) * kHeadDim + quad * 4) = hv;
        } else {   // written through to memory: read by the tile's last workgroup, or by the merge kernel
            store_partial(unit_o, (sp * kWaveRows + rho) * (kHeadDim / 4) + quad, val);
            if (quad == 0) {
                store_partial_f32(unit_ml, (sp * kWaveRows + rho) * 2, row_max(rho));
                store_partial_f32(unit_ml, (sp * kWaveRows + rho) * 2 + 1, l_all);
            }
        }
    }
    if (last || !a.fused) return;   // uniform over the grid
    __shared__ uint32_t ticket_sh;   // last-arriver merge of the tile's key ranges, as in tree_attn_kernel
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) ticket_sh = __hip_atomic_fetch_add(&a.tickets[unit], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (ticket_sh != (uint32_t)(a.nsplit - 1)) return;
    if (tid == 0) __hip_atomic_store(&a.tickets[unit], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    merge_tile<kWaveRows, true>(unit_o, unit_ml, a.out, tid, 64 * kWaves, tile, a.nsplit);
}

// ---- taller row tiles: K and V tiles turned into fp16 once and shared --------------------------------------
// A workgroup's eight wavefronts are WR = 4 row groups of 32 rows times WK = 2 key groups.  In a round each key group takes one 32-key step:
// its four wavefronts fetch the step's codes into registers two rounds ahead, turn their share into fp16 values and write those to LDS one round
// ahead (two buffers), in the layouts of tree_attn_wave_kernel's tiles: the products read values, and
// codes are converted once per 128 rows.  What the wavefronts of a key group have of a row meets at the end in LDS.
// Four row groups: two conversions of 16 codes per wavefront, step and lane, beside 32 probabilities' arithmetic.  Two row groups take 59 to 71 us where four
// take 50 (60 rows of 64/8 heads over 16001 keys); eight, of which fewer calls have the rows, no less than four.
// A round is two phases, products (with the next round's conversions in their shadow) and softmax, a barrier behind each.  Half of the wavefronts run a phase
// behind the others, so that a SIMD's matrix unit and its vector unit are both at work: 50 us at that size, against 54 in step with each other.  A
// round takes 2400 cycles there, of which the matrix steps need 1030 and LDS reads, at 128 B a cycle, 1250; 13 us go by before the first round, after the last
// one and in the merge.  No unit is full: by counters the matrix units work in 35 % of a CU's busy cycles, the vector units in 47, LDS in 46 (18 of them bank
// conflicts).  The two phases and the barriers behind them keep the three from overlapping.
constexpr int kTile16 = kKeyBlock * kHeadDim * 2;          // fp16 values of a K or V tile
constexpr int kStep16 = 2 * kTile16;
constexpr int kRowGroups = 4;
constexpr int kSharedRows = kRowGroups * kWaveRows;
constexpr int kSharedTiles = 2 * (kWaves / kRowGroups) * kStep16, kSharedExchange = kWaves * kExWave + kWaves * kWaveRows * 8;
constexpr int kSharedLds = kSharedTiles > kSharedExchange ? kSharedTiles : kSharedExchange;

// The transposing read of four key rows and the four that lie eight rows further on: eight keys at one head-dim element.  (No transfers go straight to
// LDS in this kernel, so the compiler's own waits are exact.)
__device__ __forceinline__ half8v transposed_rows(const uint8_t *at)
{
    typedef short short8v __attribute__((ext_vector_type(8)));
    const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(lds_void *)at);
    const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(lds_void *)(at + 8 * 256));
    const short8v both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(half8v, both);
}

template <int FMT>
__global__ __launch_bounds__(64 * kWaves) void tree_attn_kv8_shared_kernel(const Kv8Args a)
{
    constexpr int WR = kRowGroups, WK = kWaves / WR, CL = 8 / WR;   // row groups, key groups; 16-code chunks per lane and step
    extern __shared__ float4v smem4[];
    uint8_t *lds = reinterpret_cast<uint8_t *>(smem4);
    const int M = a.M, P = a.P, T = P + M;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kw = wave / WR, rh = wave % WR;
    const int h = lane >> 5, c = lane & 31;
    const Share share(blockIdx.x, (unsigned)(a.Hkv * a.tiles_per_kv * a.nsplit), a.nsplit, a.tiles_per_kv, a.by_tiles, a.by_ranges);
    const int kvh = share.kvh, unit = kvh * a.tiles_per_kv + share.tile, sp = share.range;
    const RowTile tile(kvh, share.tile, M, a.Hq, a.group, a.tile_rows);
    const int b0 = sp * a.bq + (sp < a.brem ? sp : a.brem), b1 = b0 + a.bq + (sp < a.brem ? 1 : 0);
    const int rounds = (b1 - b0 + WK - 1) / WK;
    const size_t kv_row_bytes = (size_t)a.Hkv * kHeadDim;
    int my_row, my_head;
    tile.locate(rh * kWaveRows + c, my_row, my_head);

    __shared__ uint64_t row_bits[kRowsPad];
    __shared__ uint32_t bad_keys[2][kWaves];   // [buffer][wavefront]: keys whose K or V scale, of the ones it turned, is no number
    const bool reaches_draft = b1 * kKeyBlock > P;   // uniform over the workgroup
    uint32_t mask_byte[8] = {};
    if (reaches_draft) {
        const int mcol = min(lane, M - 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) mask_byte[i] = a.mask[(size_t)min(wave * 8 + i, M - 1) * M + mcol];
    }
    half8v qf[8];   // lane (c, h): elements 16 j + 8 h .. of its row
    {
        const _Float16 *row = a.q + ((size_t)my_row * a.Hq + my_head) * kHeadDim + 8 * h;
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[j] = *reinterpret_cast<const half8v *>(row + 16 * j);
    }
    // staging: chunk i of this lane is chunk lane % 8 of key 8 (g % 4) + lane / 8, g = rh CL + i; g < 4: K, else V
    static_assert(CL <= 4, "a wavefront stages K or V, not both");
    const bool stages_k = rh * CL < 4;   // uniform over the wavefront
    const int trow = lane >> 3, tchunk = lane & 7;
    const uint8_t *const src = (stages_k ? a.k : a.v) + (size_t)kvh * kHeadDim;
    const _Float16 *const s_src = (stages_k ? a.k_scale : a.v_scale) + kvh;
    auto step_key = [&](int i) { return 8 * ((rh * CL + i) & 3) + trow; };   // key in the step
    u32x4 codes[2][CL];
    uint16_t scales[2][CL];
    // the codes of the next round that has not been asked for; beyond the last key they are zeros
    const uint32_t row_bytes = (uint32_t)kv_row_bytes;
    const uint8_t *next_rows = src + (size_t)(b0 + kw) * kKeyBlock * kv_row_bytes;
    const _Float16 *next_tops = s_src + (size_t)(b0 + kw) * kKeyBlock * a.Hkv;
    int keys_left = T - (b0 + kw) * kKeyBlock;
    auto fetch = [&](auto set_tag) {
        constexpr int S = decltype(set_tag)::value;
        const int rows_behind = max(min(keys_left, kKeyBlock) - 1, 0);
        const Stretch rows = stretch(next_rows, keys_left > 0 ? (uint32_t)rows_behind * row_bytes + kHeadDim : 0);
        const Stretch tops = stretch(next_tops, keys_left > 0 ? (uint32_t)(rows_behind * a.Hkv * 2 + 2) : 0);
#pragma unroll
        for (int i = 0; i < CL; ++i) {
            codes[S][i] = __builtin_amdgcn_raw_buffer_load_b128(rows, (uint32_t)step_key(i) * row_bytes + tchunk * 16, 0, 0);
            scales[S][i] = __builtin_amdgcn_raw_buffer_load_b16(tops, (uint32_t)(step_key(i) * a.Hkv * 2), 0, 0);
        }
        next_rows += WK * kKeyBlock * (size_t)row_bytes;
        next_tops += WK * kKeyBlock * (size_t)a.Hkv;
        keys_left -= WK * kKeyBlock;
    };
    fetch(std::integral_constant<int, 0>{});
    fetch(std::integral_constant<int, 1>{});
    uint64_t mbits = 0, any_bits = 0;   // draft keys that this row sees, and that any row sees
    if (reaches_draft) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            asm volatile("" : "+v"(mask_byte[i]));
            const uint64_t bits = __ballot(mask_byte[i] != 0 && wave * 8 + i < M && lane < M);
            if (lane == i) row_bits[wave * 8 + i] = bits;
        }
        __syncthreads();
        mbits = row_bits[my_row];
        any_bits = row_bits[lane];   // rows beyond M are clear
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) any_bits |= (uint64_t)__shfl_xor((unsigned long long)any_bits, off, 64);
    }
    uint8_t *const group_lds = lds + kw * (2 * kStep16);
    auto look_over = [&](auto set_tag, int t) {   // round t's codes, where not every row sees all of them
        constexpr int S = decltype(set_tag)::value;
        const int key0 = (b0 + t * WK + kw) * kKeyBlock;
        if (__builtin_expect(key0 + kKeyBlock > P, 0)) {   // uniform: the step has draft keys, which not every row sees
            // A scale that is no number marks a head that held an infinity or a NaN: taken as zero here, so that it does not reach the rows that
            // do not see it, and noted for the scores of those that do; likewise V codes that are no numbers.  What no row sees may never have been
            // written: zero as well.
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < CL; ++i) {
                bool no_number = false;
                if (__builtin_expect(__any(kv8_suspect<FMT>(stages_k ? (u32x4){} : codes[S][i], scales[S][i])), 0)) {   // uniform
                    no_number = (scales[S][i] & 0x7FFFu) >= kHalfInf || (!stages_k && kv8_no_numbers<FMT>(codes[S][i], scales[S][i]));
                    const uint64_t lanes = __ballot(no_number);
#pragma unroll 1
                    for (int r = 0; r < 8; ++r) bad |= (uint32_t)(((lanes >> (8 * r)) & 0xFFu) != 0) << (8 * ((rh * CL + i) & 3) + r);
                }
                const int draft = key0 + step_key(i) - P;
                if (no_number || (draft >= 0 && !(draft < 64 && ((any_bits >> (draft & 63)) & 1)))) codes[S][i] = (u32x4){0, 0, 0, 0}, scales[S][i] = 0;
            }
            if (lane == 0) bad_keys[S][wave] = bad;
        }
    };
    auto stage = [&](auto set_tag) {   // the codes of a set to its buffer, as values
        constexpr int S = decltype(set_tag)::value;
        uint8_t *const dst = group_lds + S * kStep16 + (stages_k ? 0 : kTile16);
#pragma unroll
        for (int i = 0; i < CL; ++i) {
            const u32x4 w = codes[S][i];
            const _Float16 scale = __builtin_bit_cast(_Float16, scales[S][i]);
            half2v n[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) kv8_values<FMT>(w[e], scale, n[2 * e], n[2 * e + 1]);
            const half8v lo = {n[0][0], n[0][1], n[1][0], n[1][1], n[2][0], n[2][1], n[3][0], n[3][1]};
            const half8v hi = {n[4][0], n[4][1], n[5][0], n[5][1], n[6][0], n[6][1], n[7][0], n[7][1]};
            // 16-byte chunks of a K row at chunk ^ (key % 8), of a V row at chunk ^ 4 (key % 4): each read below then meets every bank once
            const int key = step_key(i), swz = stages_k ? key & 7 : 4 * (key & 3);
            *reinterpret_cast<half8v *>(dst + key * 256 + (((2 * tchunk) ^ swz) << 4)) = lo;
            *reinterpret_cast<half8v *>(dst + key * 256 + (((2 * tchunk + 1) ^ swz) << 4)) = hi;
        }
    };
    const uint32_t kfrag = (uint32_t)(c * 256 + ((h ^ (c & 7)) << 4));   // fragment j: chunk (2 j + h) ^ (key % 8)
    // V: lane s of 16-lane block b points at key row 4 (b / 2) + s / 4 (and 8 further on), elements 32 dt + 16 (b % 2) + 4 (s % 4) ..
    const int vkey = 4 * h + ((lane & 15) >> 2);
    const uint32_t vfrag = vkey * 256 + (((2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ (4 * (vkey & 3))) << 4) + 8 * (lane & 1);
    float16v o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    float m_run = kLowest, l_run = 0.f;   // l_run: this lane's share (its keys) of the row's sum

    float16v sc;
    half8v pb[2], vf[8];
    auto read_values = [&](auto buf_tag) {   // V^T fragments of the round in buffer BUF
        const uint8_t *const vtile = group_lds + decltype(buf_tag)::value * kStep16 + kTile16;
#pragma unroll
        for (int f = 0; f < 8; ++f) vf[f] = transposed_rows(vtile + (vfrag ^ ((f >> 1) << 6)) + (f & 1) * 16 * 256);
    };
    auto meet = [&] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // First phase of round t: its scores (operands from buffer BUF), and the values of round t - 1, whose fragments were read a phase ago and whose
    // products go first, while the K fragments arrive; beside them the next round's codes are turned into values.
    auto products = [&](auto buf_tag, auto values_tag, int t) {
        constexpr int BUF = decltype(buf_tag)::value;
        constexpr bool VALUES = decltype(values_tag)::value;
        const std::integral_constant<int, BUF ^ 1> next;
        const uint8_t *const ktile = group_lds + BUF * kStep16;
        look_over(next, t + 1);
        __builtin_amdgcn_s_setprio(1);
        half8v kf[8];
#pragma unroll
        for (int f = 0; f < 8; ++f) kf[f] = *reinterpret_cast<const half8v *>(ktile + (kfrag ^ (f << 5)));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
        if constexpr (VALUES) {
#pragma unroll
            for (int f = 0; f < 8; ++f) o[f & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[2 * (f & 3) + (f >> 2)], pb[f >> 2], o[f & 3], 0, 0, 0);
        }
#pragma unroll
        for (int f = 0; f < 8; ++f) sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[f], qf[f], sc, 0, 0, 0);
        stage(next);
#pragma unroll
        for (int f = 0; f < (VALUES ? 16 : 8); ++f) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);                       // a matrix step,
            __builtin_amdgcn_sched_group_barrier(0x2, 5, 0);   // and vector instructions in its shadow
        }
        __builtin_amdgcn_s_setprio(0);
        fetch(next);
        meet();
    };
    const int plain_end = min(P, b1 * kKeyBlock);   // keys before it are visible to every row, and this workgroup's
    auto softmax = [&](auto buf_tag, int t) {
        constexpr int BUF = decltype(buf_tag)::value;
        const int key0 = (b0 + t * WK + kw) * kKeyBlock;
        settled(sc);   // element i: key 8 (i / 4) + 4 h + i % 4 of the step
        if (__builtin_expect(key0 + kKeyBlock > plain_end, 0)) {   // uniform, few: as in tree_attn_kv8_wave_kernel; a step behind the range's last shows nothing
            const int first = key0 - P;
            uint32_t bad = 0, seen = ~0u;
            if (first > -kKeyBlock) {
#pragma unroll
                for (int r = 0; r < WR; ++r) bad |= bad_keys[BUF][kw * WR + r];
                seen = (uint32_t)(first >= 0 ? mbits >> min(first, 63) : (mbits << -first) | ((1ull << -first) - 1));
            }
            if (key0 >= b1 * kKeyBlock) seen = 0;
            const uint32_t vis = seen >> (4 * h), hit = (seen & bad) >> (4 * h);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int bit = 8 * (i >> 2) + (i & 3);
                sc[i] = (vis >> bit) & 1u ? ((hit >> bit) & 1u ? __builtin_nanf("") : sc[i]) : -__builtin_inff();
            }
        }
        const float m_a = max_of_three(max_of_three(sc[0], sc[1], sc[2]), max_of_three(sc[3], sc[4], sc[5]), max_of_three(sc[6], sc[7], sc[8]));
        const float m_b = max_of_three(max_of_three(sc[9], sc[10], sc[11]), max_of_three(sc[12], sc[13], sc[14]), sc[15]);
        const float m_step = half_wave_max(max_of_two(m_a, m_b)) * a.scale_log2e;
        if (__builtin_expect(__any(m_step > m_run + kBehind), 0)) {
            const float m_new = m_step > m_run + kBehind ? m_step : m_run;
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            l_run *= alpha;
            m_run = m_new;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
        }
        float sums[2] = {l_run, 0.f};   // of the rounded probabilities, as the products see them: two per instruction
        const half2v ones = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const half2v p = {(_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.scale_log2e, -m_run)),
                              (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(sc[i + 1], a.scale_log2e, -m_run))};
            pb[i >> 3][i & 7] = p[0];
            pb[i >> 3][(i & 7) + 1] = p[1];
            sums[(i >> 1) & 1] = __builtin_amdgcn_fdot2(p, ones, sums[(i >> 1) & 1], false);
        }
        l_run = sums[0] + sums[1];
        // here, not where they are used: the compiler would move the exponentials into the phase of the products
        asm volatile("" : "+v"(pb[0]), "+v"(pb[1]), "+v"(l_run));
    };
    // Half of the wavefronts, one per SIMD, run a phase behind the others: while these keep the matrix units busy, those do their softmax
    // and conversions on the vector units.
    const bool behind = wave >= kWaves / 2;
    const std::integral_constant<bool, true> yes;
    const std::integral_constant<bool, false> no;
    auto vector_phase = [&](auto buf_tag, int t) {   // the second phase of round t
        read_values(buf_tag);
        __builtin_amdgcn_sched_barrier(0);
        softmax(buf_tag, t);
        meet();
    };
    auto round = [&](auto buf_tag, auto values_tag, int t) {   // what is staged and fetched beyond the last round is never used
        products(buf_tag, values_tag, t);
        vector_phase(buf_tag, t);
    };
    look_over(std::integral_constant<int, 0>{}, 0);
    stage(std::integral_constant<int, 0>{});
    fetch(std::integral_constant<int, 0>{});
    meet();
    if (behind) meet();
    round(std::integral_constant<int, 0>{}, no, 0);
    int t = 1;
    for (; t + 1 < rounds; t += 2) {
        round(std::integral_constant<int, 1>{}, yes, t);
        round(std::integral_constant<int, 0>{}, yes, t + 1);
    }
    if (t < rounds) round(std::integral_constant<int, 1>{}, yes, t);
#pragma unroll
    for (int f = 0; f < 8; ++f) o[f & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[2 * (f & 3) + (f >> 2)], pb[f >> 2], o[f & 3], 0, 0, 0);   // the last round's values
    if (!behind) meet();

    // the key groups' states of each row meet in LDS
    l_run += __shfl_xor(l_run, 32, 64);
    if (reaches_draft && mbits == 0) l_run = kPaddingMark;
    __syncthreads();   // every wavefront has left the tiles
    uint8_t *const ex = lds + wave * kExWave;
    float2v *const state = reinterpret_cast<float2v *>(lds + kWaves * kExWave);   // [wavefront][row]
    if (h == 0) state[wave * kWaveRows + c] = (float2v){m_run, l_run};
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            *reinterpret_cast<float4v *>(ex + c * kExRow + (8 * dt + 2 * b + h) * 16) =
                (float4v){o[dt][4 * b], o[dt][4 * b + 1], o[dt][4 * b + 2], o[dt][4 * b + 3]};
    __syncthreads();
    const bool last = a.nsplit == 1;
    const PartialBuffer unit_o = partial_buffer(a.part_o + (size_t)unit * a.nsplit * kSharedRows * kHeadDim);
    const PartialBuffer unit_ml = partial_buffer(a.part_ml + (size_t)unit * a.nsplit * kSharedRows * 2);
#pragma unroll
    for (int it = 0; it < 2 * WR; ++it) {   // thread t: four consecutive outputs of a row, 32 threads per row
        const int item = tid + it * (64 * kWaves);
        const int rho = item >> 5, quad = item & 31, group = rho >> 5, row = rho & 31;
        float2v of[WK];
        float m_all = kLowest, l_all = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) {
            of[w] = state[(w * WR + group) * kWaveRows + row];
            m_all = fmaxf(m_all, of[w][0]);
        }
        float4v val = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WK; ++w) {
            const float wgt = __builtin_amdgcn_exp2f(of[w][0] - m_all);
            l_all += wgt * of[w][1];
            val += wgt * *reinterpret_cast<const float4v *>(lds + (w * WR + group) * kExWave + row * kExRow + quad * 16);
        }
        if (rho >= tile.rows) continue;
        if (of[0][1] < 0.f) val = (float4v){0.f, 0.f, 0.f, 0.f}, l_all = kPaddingMark;
        if (last) {
            if (!(l_all < 0.f)) val *= 1.f / l_all;   // 0 / 0 where every score is -inf
            typedef _Float16 half4v __attribute__((ext_vector_type(4)));
            half4v hv = {(_Float16)val[0], (_Float16)val[1], (_Float16)val[2], (_Float16)val[3]};
            int qrow, head;
            tile.locate(rho, qrow, head);
            *reinterpret_cast<half4v *>(a.out + ((size_t)qrow * a.Hq + head) * kHeadDim + quad * 4) = hv;
        } else {
            store_partial(unit_o, (sp * kSharedRows + rho) * (kHeadDim / 4) + quad, val);
            if (quad == 0) {
                store_partial_f32(unit_ml, (sp * kSharedRows + rho) * 2, m_all);
                store_partial_f32(unit_ml, (sp * kSharedRows + rho) * 2 + 1, l_all);
            }
        }
    }
}

// The merge by a second kernel: one thread per four consecutive outputs, ranges in order; NS = compiled upper bound of their number (the
// loads of all go out together; ranges beyond the last read it again and are dropped).
template <int NS>
__global__ __launch_bounds__(256) void tree_attn_kv8_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                                  _Float16 *__restrict__ out, int M, int Hq, int group, int nsplit, int tile_rows,
                                                                  int tiles_per_kv, int pad)
{
    const int idx = blockIdx.x * 256 + threadIdx.x;   // over M * Hq * 32 quads
    if (idx >= M * Hq * (kHeadDim / 4)) return;
    const int d4 = idx % (kHeadDim / 4), h = (idx / (kHeadDim / 4)) % Hq, qrow = idx / (kHeadDim / 4) / Hq;
    const int kvh = h / group, pair = (h - kvh * group) * M + qrow, index = pair / tile_rows, row = pair - index * tile_rows;
    const size_t base = (size_t)(kvh * tiles_per_kv + index) * nsplit * pad + row;
    const float2v *ml = reinterpret_cast<const float2v *>(part_ml) + base;
    const float4v *po = reinterpret_cast<const float4v *>(part_o) + base * (kHeadDim / 4) + d4;
    float2v st[NS];
    float4v os[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const size_t at = (size_t)min(s, nsplit - 1) * pad;
        st[s] = ml[at];
        os[s] = po[at * (kHeadDim / 4)];
    }
    float m_all = st[0][0];
#pragma unroll
    for (int s = 1; s < NS; ++s) m_all = fmaxf(m_all, st[s][0]);
    float den = 0.f;
    float4v num = {0.f, 0.f, 0.f, 0.f};
    bool padding = false;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        padding |= st[s][1] < 0.f;
        const float wgt = s < nsplit ? __builtin_amdgcn_exp2f(st[s][0] - m_all) : 0.f;
        if (s < nsplit) {   // uniform
            den += wgt * st[s][1];
            num += wgt * os[s];
        }
    }
    const float inv = padding ? 0.f : 1.f / den;
    if (padding) num = (float4v){0.f, 0.f, 0.f, 0.f};
    typedef _Float16 half4v __attribute__((ext_vector_type(4)));
    half4v hv = {(_Float16)(num[0] * inv), (_Float16)(num[1] * inv), (_Float16)(num[2] * inv), (_Float16)(num[3] * inv)};
    *reinterpret_cast<half4v *>(out + ((size_t)qrow * Hq + h) * kHeadDim + d4 * 4) = hv;
}

// How a call is cut up: even row tiles of up to 32 row_groups rows, key ranges per tile, who merges the ranges.
struct Kv8Plan { int row_groups, tile_rows, tiles_per_kv, ranges, fused; int64_t time; };
static int kv8_steps(int M, int P) { return (P + M + kKeyBlock - 1) / kKeyBlock; }

// The number of ranges with the smallest estimate.  Where tiles have several, there is at most one workgroup per CU (which also bounds the partial results);
// more tiles than CUs take one range each and go in turns, since LDS holds one workgroup.  Estimates are in hundredths of a
// microsecond.  Those of the wave kernel were fitted over 38 sizes (1 to 64 query rows, 2 to 16 KV heads, 64 to 131072 keys, both formats) with
// up to 19 numbers of ranges and both ways to merge them; the number they pick is 1 % slower than the best in the mean, 9 % at most.
static Kv8Plan kv8_cut(int pairs, int Hkv, int steps, int row_groups, int format)
{
    Kv8Plan p;
    p.row_groups = row_groups;
    even_tiles(pairs, kWaveRows * row_groups, p.tile_rows, p.tiles_per_kv);
    const int units = Hkv * p.tiles_per_kv, rows = p.tile_rows;
    int most = kChipTiles / units;
    most = most > kMaxRanges ? kMaxRanges : most;
    most = most > steps ? steps : most;
    p.time = INT64_MAX;
    for (int r = 1; r <= (most < 1 ? 1 : most); ++r) {
        const int64_t range = (steps + r - 1) / r;   // steps of the longest
        const int turns = (units * r + kChipTiles - 1) / kChipTiles;
        bool fused = false;
        int64_t time;
        if (row_groups == 1) {
            const int slots = r <= 4 ? 4 : r <= 8 ? 8 : r <= 16 ? 16 : kMaxRanges;   // ranges that the merge is compiled for
            const int by_kernel = 240 + 7 * slots, by_last = 60 + (32 * rows + (3 * rows + 80) * slots) / 10;
            fused = r > 1 && units <= kMaxTickets && by_last < by_kernel;
            time = turns * (580 + 7 * rows + range * (format == kInt8 ? 24 : 19)) + (r == 1 ? 0 : fused ? by_last : by_kernel);
        } else {   // a round: a step of each key group
            time = turns * (1100 + (range + kWaves / row_groups - 1) / (kWaves / row_groups) * 110) + (r == 1 ? 0 : 350);
        }
        if (time < p.time) p.ranges = r, p.fused = fused, p.time = time;
    }
    return p;
}

// 256 keys of 32 rows take the wave kernel 1.9 us with int8 codes and 1.5 with e4m3 (it turns every code into a number once per 32 rows), the same work,
// 64 keys of 128 rows, the shared kernel 1.1 us, but that starts and ends more slowly.  Measured, wave and shared kernel, us:
//   rows, heads, keys        int8           e4m3
//   60, 64/8,  2048          18.1  19.5     15.8  19.2
//   60, 64/8,  4096          24.9  22.7     21.5  22.4
//   60, 64/8, 16001          66.2  48.7     54.9  47.6
//   37, 28/4, 16000          27.5  28.8     23.8  28.3
//   37, 28/4, 60000          72.3  63.7     59.7  62.4
//   16, 64/8, 32000          41.3  33.7     35.4  33.1
//   64, 16/16, 16000         27.4  29.7     24.7  29.8
// and where the wave kernel takes more than one turn (two, four, four, eight):
//   64, 256/32, 16001        271.7 159.7    207.2 155.9
//   64, 512/64,  2000        91.0  49.1     77.8  48.3
//   64, 512/64, 16001        502.7 300.6    419.7 302.2
//   64, 1024/128, 3000       235.3 129.8    204.2 128.3
//   33, 1024/128,  40        36.7  23.1     36.6  22.6     (five turns and two)
//    8, 4096/512, 4000       197.5 181.1    190.6 181.4    (four turns and two)
// The estimates take the slower kernel at the last of these, by 5 to 9 %, and at 37 rows of 28/4 heads over 16000 int8 keys, by up to 5 %.
static Kv8Plan kv8_plan(int M, int P, int Hq, int Hkv, int format)
{
    const int pairs = Hq / Hkv * M, steps = kv8_steps(M, P);
    const Kv8Plan wave = kv8_cut(pairs, Hkv, steps, 1, format);
    if (pairs <= kWaveRows) return wave;   // one row group would be at work
    const Kv8Plan shared = kv8_cut(pairs, Hkv, steps, kRowGroups, format);
    return shared.time < wave.time ? shared : wave;
}

static int check_attn_kv8(int M, int P, int Hq, int Hkv, int D)
{
    if (M < 1 || P < 0 || Hq < 1 || Hkv < 1 || D < 1) return W4A16_EINVAL;
    if (Hq % Hkv != 0) return W4A16_EINVAL;
    if (D != kHeadDim || M > W4A16_MAX_M || P > (1 << 30) || Hq > kMaxTickets || Hq / Hkv > 8) return W4A16_EUNSUP;
    return W4A16_OK;
}

template <typename Kernel>
static int launch_kv8(Kernel kernel, bool &lds_ok, int lds, int grid, hipStream_t stream, const Kv8Args &a)
{
    if (!lds_ok) {   // LDS above 48 KB needs an opt-in, once per kernel
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return W4A16_EHIP;
        lds_ok = true;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kWaves), lds, stream, a);
    return W4A16_OK;
}

template <int FMT>
static int launch_kv8_attn(int row_groups, int grid, hipStream_t stream, const Kv8Args &a)
{
    static bool wave_ok, shared_ok;
    return row_groups == 1 ? launch_kv8(tree_attn_kv8_wave_kernel<FMT>, wave_ok, kWaveLds, grid, stream, a)
                           : launch_kv8(tree_attn_kv8_shared_kernel<FMT>, shared_ok, kSharedLds, grid, stream, a);
}

static void launch_kv8_merge(const Kv8Args &a, int pad, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.M * a.Hq * (kHeadDim / 4) + 255) / 256));
#define W4_KV8_MERGE(NS_)                                                                                                            \
    hipLaunchKernelGGL(tree_attn_kv8_merge_kernel<NS_>, grid, dim3(256), 0, stream, (const float *)a.part_o, (const float *)a.part_ml, a.out, a.M, a.Hq, \
                       a.group, a.nsplit, a.tile_rows, a.tiles_per_kv, pad)
    if (a.nsplit <= 4) W4_KV8_MERGE(4);
    else if (a.nsplit <= 8) W4_KV8_MERGE(8);
    else if (a.nsplit <= 16) W4_KV8_MERGE(16);
    else W4_KV8_MERGE(kMaxRanges);
#undef W4_KV8_MERGE
}

}  // namespace w4

using namespace w4;

extern "C" {
size_t tree_verify_attn_kv8_workspace_bytes(int M, int P, int Hq, int Hkv, int D)
{
    if (check_attn_kv8(M, P, Hq, Hkv, D) != W4A16_OK) return 0;
    return kTicketBytes + (size_t)kChipTiles * kSharedRows * (kHeadDim + 2) * sizeof(float);
}

int tree_verify_attn_kv8_plan_describe(int M, int P, int Hq, int Hkv, int D, int format, int *out)
{
    if (!out) return W4A16_ENULL;
    if (!kv8_format_known(format)) return W4A16_EINVAL;
    const int rc = check_attn_kv8(M, P, Hq, Hkv, D);
    if (rc != W4A16_OK) return rc;
    const Kv8Plan pl = kv8_plan(M, P, Hq, Hkv, format);
    out[0] = pl.tile_rows;
    out[1] = pl.tiles_per_kv;
    out[2] = pl.ranges;
    out[3] = pl.fused;
    out[4] = pl.row_groups != 1;
    return W4A16_OK;
}

int tree_verify_attn_kv8(const void *q, const void *k, const void *v, const void *k_scale, const void *v_scale, int format, const uint8_t *mask,
                         void *out, int M, int P, int Hq, int Hkv, int D, float scale, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!kv8_format_known(format)) return W4A16_EINVAL;
    int rc = check_attn_kv8(M, P, Hq, Hkv, D);
    if (rc != W4A16_OK) return rc;
    if (!(scale > 0.f) || scale > 3.0e38f) return W4A16_EINVAL;   // the kernels take row maxima before scaling
    if (!q || !k || !v || !k_scale || !v_scale || !mask || !out) return W4A16_ENULL;
    if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(k_scale) || misaligned(v_scale) || misaligned(out) ||
        workspace_misaligned(workspace))
        return W4A16_EALIGN;
    if (!workspace || workspace_bytes < tree_verify_attn_kv8_workspace_bytes(M, P, Hq, Hkv, D)) return W4A16_EWORKSPACE;
    const Kv8Plan pl = kv8_plan(M, P, Hq, Hkv, format);
    const int units = Hkv * pl.tiles_per_kv, steps = kv8_steps(M, P);
    Kv8Args a;
    a.by_tiles = divider(pl.tiles_per_kv);
    a.by_ranges = divider(pl.ranges);
    a.q = (const _Float16 *)q;
    a.k = (const uint8_t *)k;
    a.v = (const uint8_t *)v;
    a.k_scale = (const _Float16 *)k_scale;
    a.v_scale = (const _Float16 *)v_scale;
    a.mask = mask;
    a.out = (_Float16 *)out;
    a.part_o = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(workspace) + kTicketBytes);
    const int pad = pl.row_groups * kWaveRows;
    a.part_ml = a.part_o + (size_t)units * pl.ranges * pad * kHeadDim;
    a.tickets = reinterpret_cast<uint32_t *>(workspace);
    a.M = M;
    a.P = P;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.group = Hq / Hkv;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.nsplit = pl.ranges;
    a.bq = steps / pl.ranges;
    a.brem = steps % pl.ranges;
    a.tile_rows = pl.tile_rows;
    a.tiles_per_kv = pl.tiles_per_kv;
    a.fused = pl.fused;
    rc = format == kInt8 ? launch_kv8_attn<kInt8>(pl.row_groups, units * pl.ranges, (hipStream_t)stream, a)
                         : launch_kv8_attn<kE4m3>(pl.row_groups, units * pl.ranges, (hipStream_t)stream, a);
    if (rc != W4A16_OK) return rc;
    if (pl.ranges > 1 && !pl.fused) launch_kv8_merge(a, pad, (hipStream_t)stream);
    return launch_status();
}

}  // extern "C"
