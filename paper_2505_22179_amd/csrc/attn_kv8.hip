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

// Clears the V codes, in LDS, of the keys of a step that no row of the tile sees.  Such rows of the cache may never have been written: a probability of
// zero would not keep e4m3's NaN codes, or products beyond fp16, out of the rows' sums.
__device__ __forceinline__ void clear_codes(uint8_t *tile, uint32_t keys, int lane)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((keys >> (8 * i + (lane >> 3))) & 1u) *reinterpret_cast<u32x4 *>(tile + i * 1024 + lane * 16) = (u32x4){0, 0, 0, 0};
    asm volatile("" ::: "memory");
}

// ---- row tiles of at most 32 rows: wavefronts with K and V tiles of their own -------------------------------
// As tree_attn_wave_kernel: eight wavefronts carry the same 32 rows, wavefront w takes key steps w, w + 8, ... of the workgroup's range and
// meets the others only at the end.  A step is 32 keys: 4 KB of K codes, 4 KB of V codes and 64 scales, brought straight to LDS one step
// ahead of their use (two buffers per wavefront).
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
        const uint32_t bad = (uint32_t)nan_lanes | (uint32_t)(nan_lanes >> 32);   // bit i: key i of the step
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
            uint32_t by_any = seen;
#pragma unroll
            for (int off = 1; off < kWaveRows; off <<= 1) by_any |= (uint32_t)__shfl_xor((int)by_any, off, 64);
            clear_codes(mine + buf * kWaveBuf + kWaveTile, ~by_any, lane);
        }
        if (bad) {   // uniform, rare
            const uint32_t hit = (seen & bad) >> (4 * h);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = ((hit >> (8 * (i >> 2) + (i & 3))) & 1u) ? __builtin_nanf("") : s[i];
        }
        // the scale is positive (checked by the host): the largest raw score is the largest scaled one
        const float m_a = max_of_three(max_of_three(s[0], s[1], s[2]), max_of_three(s[3], s[4], s[5]), max_of_three(s[6], s[7], s[8]));
        const float m_b = max_of_three(max_of_three(s[9], s[10], s[11]), max_of_three(s[12], s[13], s[14]), s[15]);
        const float m_new = max_of_two(m_run, half_wave_max(max_of_two(m_a, m_b)) * a.scale_log2e);
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        half8v pb[2];
        float psum[4];
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i + e], a.scale_log2e, -m_new));
                pb[i >> 3][(i & 7) + e] = (_Float16)p[e];
            }
            psum[i >> 2] = (p[0] + p[1]) + (p[2] + p[3]);
        }
        l_run = l_run * alpha + ((psum[0] + psum[1]) + (psum[2] + psum[3]));
        m_run = m_new;
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
        }
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
        weights[tid] = (float2v){wgt, wgt * me[1]};
    }
    __syncthreads();
    const bool last = a.nsplit == 1;
    const PartialBuffer unit_o = partial_buffer(a.part_o + (size_t)unit * a.nsplit * kRowsPad * kHeadDim);
    const PartialBuffer unit_ml = partial_buffer(a.part_ml + (size_t)unit * a.nsplit * kRowsPad * 2);
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
        if (last) {
            val *= l_all == 0.f ? 0.f : 1.f / l_all;   // a row that sees no key: zeros
            typedef _Float16 half4v __attribute__((ext_vector_type(4)));
            half4v hv = {(_Float16)val[0], (_Float16)val[1], (_Float16)val[2], (_Float16)val[3]};
            int qrow, head;
            tile.locate(rho, qrow, head);
            *reinterpret_cast<half4v *>(a.out + ((size_t)qrow * a.Hq + head) * kHeadDim + quad * 4) = hv;
        } else {   // written through to memory: read by the tile's last workgroup, or by the merge kernel
            store_partial(unit_o, (sp * kRowsPad + rho) * (kHeadDim / 4) + quad, val);
            if (quad == 0) {
                store_partial_f32(unit_ml, (sp * kRowsPad + rho) * 2, row_max(rho));
                store_partial_f32(unit_ml, (sp * kRowsPad + rho) * 2 + 1, l_all);
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
    merge_tile(unit_o, unit_ml, a.out, tid, 64 * kWaves, tile, a.nsplit);
}

// How a call is cut up: even row tiles, key ranges per tile, who merges the ranges.
struct Kv8Plan { int tile_rows, tiles_per_kv, ranges, fused; };
static int kv8_steps(int M, int P) { return (P + M + kKeyBlock - 1) / kKeyBlock; }
static Kv8Plan kv8_plan(int M, int P, int Hq, int Hkv)
{
    Kv8Plan p;
    even_tiles(Hq / Hkv * M, kWaveRows, p.tile_rows, p.tiles_per_kv);
    const int units = Hkv * p.tiles_per_kv, steps = kv8_steps(M, P);
    int want = kChipTiles / units;
    want = want > (steps + 3) / 4 ? (steps + 3) / 4 : want;
    want = want > kMaxRanges ? kMaxRanges : want;
    p.ranges = want < 1 ? 1 : want;
    p.fused = p.ranges > 1 && units <= kMaxTickets && p.tile_rows * p.ranges <= 256;
    return p;
}

static int check_attn_kv8(int M, int P, int Hq, int Hkv, int D)
{
    if (M < 1 || P < 0 || Hq < 1 || Hkv < 1 || D < 1) return W4A16_EINVAL;
    if (Hq % Hkv != 0) return W4A16_EINVAL;
    if (D != kHeadDim || M > W4A16_MAX_M || P > (1 << 30) || Hq > kMaxTickets || Hq / Hkv > 8) return W4A16_EUNSUP;
    return W4A16_OK;
}

template <int FMT>
static int launch_kv8_wave(int grid, hipStream_t stream, const Kv8Args &a)
{
    static bool lds_ok = false;   // LDS above 48 KB needs an opt-in, once per kernel
    if (!lds_ok) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(&tree_attn_kv8_wave_kernel<FMT>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                kWaveLds) != hipSuccess)
            return W4A16_EHIP;
        lds_ok = true;
    }
    hipLaunchKernelGGL(tree_attn_kv8_wave_kernel<FMT>, dim3((unsigned)grid), dim3(64 * kWaves), kWaveLds, stream, a);
    return W4A16_OK;
}

}  // namespace w4

using namespace w4;

extern "C" {

size_t tree_verify_attn_kv8_workspace_bytes(int M, int P, int Hq, int Hkv, int D)
{
    if (check_attn_kv8(M, P, Hq, Hkv, D) != W4A16_OK) return 0;
    return kTicketBytes + (size_t)kChipTiles * kRowsPad * (kHeadDim + 2) * sizeof(float);
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
    const Kv8Plan pl = kv8_plan(M, P, Hq, Hkv);
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
    a.part_ml = a.part_o + (size_t)units * pl.ranges * kRowsPad * kHeadDim;
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
    rc = format == kInt8 ? launch_kv8_wave<kInt8>(units * pl.ranges, (hipStream_t)stream, a) : launch_kv8_wave<kE4m3>(units * pl.ranges, (hipStream_t)stream, a);
    if (rc != W4A16_OK) return rc;
    if (pl.ranges > 1 && !pl.fused)
        launch_attn_merge(a.part_o, a.part_ml, out, M, Hq, a.group, pl.ranges, pl.tile_rows, pl.tiles_per_kv, (hipStream_t)stream);
    return launch_status();
}

}  // extern "C"
