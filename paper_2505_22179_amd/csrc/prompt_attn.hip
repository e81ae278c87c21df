// w4a16_prompt_attn: causal attention of packed sequences of different lengths over their keys in a cache.  Contract in include/w4a16.h.
//
// The (query, head) pairs that share a KV head are the rows of one problem: query-major, pair = query * group + head in its group, so that a
// tile of rows spans few queries and the keys it sees end almost together.  S^T = K . Q^T leaves a lane with scores of ONE pair (column
// lane % 32), which are the operand of O^T += V^T . P^T as they stand; the softmax runs in registers, one pass over the keys.
#include "attn_common.h"

namespace w4 {

typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) half4v lds_half4v;

constexpr int kKeyTile = 64;      // keys of a step
constexpr int kMostSplits = 32;
constexpr int kMostSequences = 4096;

struct PromptArgs {
    const _Float16 *q, *k, *v;
    const int32_t *q_start, *k_start, *k_len;   // k_start, k_len: both or none
    _Float16 *out;
    float *part_o, *part_ml;
    int B, rows, k_rows, Hq, Hkv, group, tiles, splits;   // tiles: most row tiles per KV head
    float scale_log2e;
};

// Where a workgroup works.  Row tiles are numbered from the last of the last sequence down: the tiles that see most keys of a sequence are
// the first to be dealt out.  A sequence whose rows or keys do not lie in the buffers has no tiles.
struct Place {
    int kvh, unit, split;   // unit: KV head and tile, of the partial results
    int n, T, q0, k0;       // queries and keys of the sequence, their first rows
    int first;              // pair of the tile's first row
    bool any;
};

template <int ROWS>
__device__ __forceinline__ Place find_place(const PromptArgs &a, unsigned block, int lane)
{
    Place w;
    // Workgroups go to the eight XCDs in turn.  Where the KV heads divide evenly, an XCD keeps to its own heads, or to its share of a head's
    // tiles: its L2 then holds the keys of few heads.
    const unsigned xcd = block & 7u, turn = block >> 3;
    unsigned number;   // of tile and split
    if (a.Hkv % 8 == 0) {
        const unsigned per = (unsigned)a.Hkv >> 3;
        w.kvh = (int)(xcd + 8 * (turn % per));
        number = turn / per;
    } else if (8 % a.Hkv == 0) {
        const unsigned share = 8u / (unsigned)a.Hkv;
        w.kvh = (int)(xcd % (unsigned)a.Hkv);
        number = turn * share + xcd / (unsigned)a.Hkv;
    } else {
        w.kvh = (int)(block % (unsigned)a.Hkv);
        number = block / (unsigned)a.Hkv;
    }
    const int tile = (int)(number / (unsigned)a.splits);
    w.split = (int)(number - (unsigned)tile * (unsigned)a.splits);
    w.unit = w.kvh * a.tiles + tile;
    w.any = false;
    if (tile >= a.tiles) return w;   // the grid's last round, or offsets that overlap
    int before = 0;
    for (int base = 0; base < a.B; base += 64) {   // 64 sequences at a time, the last first
        const int b = a.B - 1 - base - lane;
        int n = 0, T = 0, q0 = 0, k0 = 0, count = 0;
        if (b >= 0) {
            const int q1 = a.q_start[b + 1];
            q0 = a.q_start[b];
            if (a.k_len) {
                k0 = a.k_start[b];
                T = a.k_len[b];
            } else {
                k0 = q0;
                T = (int)max(-1ll, min((long long)q1 - q0, 0x7FFFFFFFll));
            }
            const bool valid = q0 >= 0 && q1 > q0 && q1 <= a.rows && k0 >= 0 && T >= 0 && (long long)k0 + T <= a.k_rows;
            if (valid) {
                n = q1 - q0;
                count = (int)(((long long)n * a.group + ROWS - 1) / ROWS);
            }
        }
        int upto = count;   // tiles of this sequence and of those after it
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int other = __shfl_up(upto, off, 64);
            if (lane >= off) upto += other;
        }
        const uint64_t hit = __ballot(before + upto > tile);
        if (hit) {
            const int src = __builtin_ctzll(hit);
            const int mine = tile - before - __shfl(upto - count, src, 64);   // tile of the sequence, counted from its last
            w.n = __builtin_amdgcn_readfirstlane(__shfl(n, src, 64));
            w.T = __builtin_amdgcn_readfirstlane(__shfl(T, src, 64));
            w.q0 = __builtin_amdgcn_readfirstlane(__shfl(q0, src, 64));
            w.k0 = __builtin_amdgcn_readfirstlane(__shfl(k0, src, 64));
            w.first = __builtin_amdgcn_readfirstlane((__shfl(count, src, 64) - 1 - mine) * ROWS);
            w.any = true;
            break;
        }
        before += __shfl(upto, 63, 64);
    }
    return w;
}

__device__ __forceinline__ half8v read_chunk(const uint8_t *p) { return *reinterpret_cast<const half8v *>(p); }
// four key rows of a column each, transposed (see tree_attn_wave_kernel): the compiler counts and waits for this read
__device__ __forceinline__ half4v read_transposed(const uint8_t *p)
{
    return __builtin_bit_cast(half4v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)p));
}
__device__ __forceinline__ bool not_finite(_Float16 x) { return (__builtin_bit_cast(uint16_t, x) & 0x7C00u) == 0x7C00u; }

// One workgroup of NW wavefronts: NW * 32 * RT rows, keys through LDS in tiles of 64, two buffers, one barrier per tile.
template <int D, int NW, int RT>
__global__ __launch_bounds__(64 * NW) void prompt_attn_tile_kernel(PromptArgs a)
{
    constexpr int ROWS = 32 * RT * NW;
    constexpr int ROW_BYTES = D * 2, CHUNKS = D / 8, TILE = kKeyTile * ROW_BYTES;
    constexpr int PER = 1024 / ROW_BYTES;                  // rows of a transfer
    constexpr int TRANSFERS = TILE / 1024 / NW;            // of a wavefront, K and V each
    static_assert(TRANSFERS >= 1, "");
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * TILE];   // K, V; K, V
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, c = lane & 31;
    const Place at = find_place<ROWS>(a, blockIdx.x, lane);
    if (!at.any) return;   // uniform over the workgroup
    const int pairs = at.n * a.group, last = min(at.first + ROWS, pairs) - 1;   // pairs <= 2^31 by the host's checks
    // position of a row's query among the keys: it sees keys 0 .. position
    int pair[RT], pos[RT];
    size_t elem[RT];   // of its (query, head) in q and out
    half8v qf[RT][D / 16];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        pair[r] = at.first + (wave * RT + r) * 32 + c;
        const int p = min(pair[r], pairs - 1), query = p / a.group;
        pos[r] = at.T - at.n + query;
        elem[r] = ((size_t)(at.q0 + query) * a.Hq + at.kvh * a.group + (p - query * a.group)) * D;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) qf[r][j] = *reinterpret_cast<const half8v *>(a.q + elem[r] + 16 * j + 8 * h);
    }
    const int seen = at.T - at.n + last / a.group + 1;                    // keys that the tile's last row sees
    const int steps = seen > 0 ? (seen + kKeyTile - 1) / kKeyTile : 0;
    const int s0 = (int)((long long)steps * at.split / a.splits), s1 = (int)((long long)steps * (at.split + 1) / a.splits);
    // keys up to which every row of the wavefront sees all
    const int wave_first = min(at.first + wave * RT * 32, pairs - 1);
    const int all_see = at.T - at.n + wave_first / a.group + 1;
    const int wave_seen = at.T - at.n + min(at.first + (wave + 1) * RT * 32 - 1, pairs - 1) / a.group + 1;

    const uint32_t stride = (uint32_t)a.Hkv * ROW_BYTES;
    const uint8_t *const k_src = reinterpret_cast<const uint8_t *>(a.k) + ((size_t)at.k0 * a.Hkv + at.kvh) * ROW_BYTES;
    const uint8_t *const v_src = reinterpret_cast<const uint8_t *>(a.v) + ((size_t)at.k0 * a.Hkv + at.kvh) * ROW_BYTES;
    const int trow = lane / CHUNKS, tchunk = lane % CHUNKS;
    auto request = [&](int step, uint8_t *buffer) {
        const int key0 = step * kKeyTile;
        const Stretch ks = stretch(k_src + (size_t)key0 * stride, 0x7FFFFFFF), vs = stretch(v_src + (size_t)key0 * stride, 0x7FFFFFFF);
#pragma unroll
        for (int i = 0; i < TRANSFERS; ++i) {
            const int t = wave * TRANSFERS + i, row = t * PER + trow;
            const uint32_t from = (uint32_t)min(row, at.T - 1 - key0) * stride;   // rows beyond the last key repeat it; they are masked
            quad_to_lds(ks, buffer + t * 1024, from + ((tchunk ^ (row & 7)) << 4), 0);
            quad_to_lds(vs, buffer + TILE + t * 1024, from + ((tchunk ^ (2 * row & (CHUNKS - 1))) << 4), 0);
        }
    };

    float16v o[RT][D / 32];
    float m_run[RT], l_run[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m_run[r] = kLowest;
        l_run[r] = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[r][dt][i] = 0.f;
    }
    const uint32_t kfrag = (uint32_t)(c * ROW_BYTES + ((h ^ (c & 7)) << 4));
    const int vkey = 4 * h + ((lane & 15) >> 2);
    const uint32_t vfrag = (uint32_t)(vkey * ROW_BYTES + ((((2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ (2 * vkey)) & (CHUNKS - 1)) << 4) + 8 * (lane & 1));

    auto walk = [&](int step, const uint8_t *ktile, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        const uint8_t *const vtile = ktile + TILE;
        const int key0 = step * kKeyTile;
        float16v s[RT][2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[r][kt][i] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const half8v kf = read_chunk(ktile + kt * 32 * ROW_BYTES + (kfrag ^ (j << 5)));
#pragma unroll
                for (int r = 0; r < RT; ++r) s[r][kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[r][j], s[r][kt], 0, 0, 0);
            }
        }
        half8v pb[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            settled(s[r][0]);
            settled(s[r][1]);
            if constexpr (MASKED) {
                const int room = pos[r] - key0 - 4 * h;   // key 32 kt + 8 (i / 4) + 4 h + i % 4 of the tile is seen up to the position
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[r][kt][i] = 32 * kt + 8 * (i >> 2) + (i & 3) <= room ? s[r][kt][i] : -__builtin_inff();
            }
            float m = max_of_two(s[r][0][0], s[r][0][1]);
#pragma unroll
            for (int i = 2; i < 16; i += 2) m = max_of_three(m, s[r][0][i], s[r][0][i + 1]);
#pragma unroll
            for (int i = 0; i < 16; i += 2) m = max_of_three(m, s[r][1][i], s[r][1][i + 1]);
            const float m_new = max_of_two(m_run[r], half_wave_max(m) * a.scale_log2e);
            const float alpha = __builtin_amdgcn_exp2f(m_run[r] - m_new);
            float sum[4] = {};
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][kt][i], a.scale_log2e, -m_new));
                    sum[i & 3] += p;
                    pb[r][2 * kt + (i >> 3)][i & 7] = (_Float16)p;
                }
            l_run[r] = l_run[r] * alpha + ((sum[0] + sum[1]) + (sum[2] + sum[3]));
            m_run[r] = m_new;
            if (__any(alpha != 1.0f)) {
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) o[r][dt] *= alpha;
            }
        }
        bool bad = false;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint8_t *const p = vtile + u * 16 * ROW_BYTES + (vfrag ^ (dt << 6));
                const half4v lo = read_transposed(p), hi = read_transposed(p + 8 * ROW_BYTES);
                half8v vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                if constexpr (MASKED) {   // what a row does not see may be anything: 0 times it need not be 0
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool b = not_finite(vf[e]);
                        bad |= b;
                        vf[e] = b ? (_Float16)0 : vf[e];
                    }
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) o[r][dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pb[r][u], o[r][dt], 0, 0, 0);
            }
        settled(o[RT - 1][D / 32 - 1]);   // the loop's branches go round too little for the last product
        if constexpr (MASKED) {
            if (__any(bad)) {   // rows that do see such a value: it joins their sums as it is
                for (int key = 0; key < kKeyTile; ++key)
#pragma unroll
                    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                        for (int quad = 0; quad < 4; ++quad) {   // elements 32 dt + 8 quad + 4 h ..
                            const half4v x = *reinterpret_cast<const half4v *>(vtile + key * ROW_BYTES + (((4 * dt + quad) ^ (2 * key & (CHUNKS - 1))) << 4) + 8 * h);
#pragma unroll
                            for (int r = 0; r < RT; ++r)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (not_finite(x[e]) && key0 + key <= pos[r]) o[r][dt][4 * quad + e] += (float)x[e];
                        }
            }
        }
    };

    if (s0 < s1) {
        request(s0, lds);
        for (int step = s0; step < s1; ++step) {
            uint8_t *const buffer = lds + ((step - s0) & 1) * 2 * TILE;
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // this tile has landed, the other buffer has been read
            if (step + 1 < s1) request(step + 1, lds + ((step + 1 - s0) & 1) * 2 * TILE);
            const int key1 = (step + 1) * kKeyTile;
            if (key1 <= all_see) walk(step, buffer, std::false_type{});        // uniform over the wavefront
            else if (key1 - kKeyTile < wave_seen) walk(step, buffer, std::true_type{});
        }
    }

#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float l = l_run[r] + __shfl_xor(l_run[r], 32, 64);
        if (pair[r] >= pairs) continue;
        if (a.splits == 1) {
            const float inv = pos[r] >= 0 ? 1.f / l : 0.f;   // a row that sees no key gets zeros; one whose scores are all -inf 0 / 0
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    half4v y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = (_Float16)(o[r][dt][4 * g + e] * inv);
                    *reinterpret_cast<half4v *>(a.out + elem[r] + 32 * dt + 8 * g + 4 * h) = y;
                }
        } else {
            const size_t row = ((size_t)at.unit * a.splits + at.split) * ROWS + (pair[r] - at.first);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<float4v *>(a.part_o + row * D + 32 * dt + 8 * g + 4 * h) =
                        (float4v){o[r][dt][4 * g], o[r][dt][4 * g + 1], o[r][dt][4 * g + 2], o[r][dt][4 * g + 3]};
            if (h == 0) {
                a.part_ml[2 * row] = m_run[r];
                a.part_ml[2 * row + 1] = l;
            }
        }
    }
}

// The ranges of a tile's keys joined: D / 4 threads per row, four outputs each, ranges in order.  Grid as that of the tiles with one split.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void prompt_attn_merge_kernel(PromptArgs a)
{
    const int splits = a.splits;
    a.splits = 1;   // of the grid
    const Place at = find_place<ROWS>(a, blockIdx.x, threadIdx.x & 63);
    if (!at.any) return;
    const int pairs = at.n * a.group, here = min(ROWS, pairs - at.first);
    for (int item = blockIdx.y * 256 + threadIdx.x; item < here * (D / 4); item += 256 * gridDim.y) {
        const int r = item / (D / 4), d4 = item % (D / 4), p = at.first + r, query = p / a.group;
        const size_t row = (size_t)at.unit * splits * ROWS + r;
        float m = kLowest;
        for (int s = 0; s < splits; ++s) m = fmaxf(m, a.part_ml[2 * (row + (size_t)s * ROWS)]);
        float den = 0.f;
        float4v num = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; ++s) {
            const float ms = a.part_ml[2 * (row + (size_t)s * ROWS)], ls = a.part_ml[2 * (row + (size_t)s * ROWS) + 1];
            const float w = __builtin_amdgcn_exp2f(ms - m);
            den += w * ls;
            num += w * *reinterpret_cast<const float4v *>(a.part_o + (row + (size_t)s * ROWS) * D + 4 * d4);
        }
        const float inv = at.T - at.n + query >= 0 ? 1.f / den : 0.f;
        half4v y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (_Float16)(num[e] * inv);
        *reinterpret_cast<half4v *>(a.out + ((size_t)(at.q0 + query) * a.Hq + at.kvh * a.group + (p - query * a.group)) * D + 4 * d4) = y;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------
constexpr int kTileRows = 256;

struct PromptPlan {
    int tiles, splits;
    size_t o_bytes, ml_bytes;
};

static int check_prompt_sizes(int rows, int B, int max_q, int max_k, int Hq, int Hkv, int D)
{
    if (rows < 1 || B < 1 || max_q < 1 || max_k < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || D < 1) return W4A16_EINVAL;
    if (D != 64 && D != 128) return W4A16_EUNSUP;
    if (B > kMostSequences || (long long)rows * Hq > (1 << 29) || rows > (1 << 23) || Hkv > 1024 || Hq / Hkv > 64 || max_q > (1 << 23) || max_k > (1 << 30)) return W4A16_EUNSUP;
    return W4A16_OK;
}

static PromptPlan prompt_plan(int rows, int B, int max_q, int max_k, int Hq, int Hkv, int D)
{
    PromptPlan p;
    const int group = Hq / Hkv;
    p.tiles = (int)((long long)rows * group / kTileRows) + B;
    const long long work = (long long)p.tiles * Hkv;
    // too few tiles for the compute units: their keys are cut, eight steps a range at least
    p.splits = 1;
    if (work < 256) p.splits = (int)min(min((512 + work - 1) / work, (long long)(max_k + 8 * kKeyTile - 1) / (8 * kKeyTile)), (long long)kMostSplits);
    const size_t rows_kept = p.splits > 1 ? (size_t)work * p.splits * kTileRows : 0;
    p.o_bytes = rows_kept * D * 4;
    p.ml_bytes = rows_kept * 8;
    return p;
}

// blocks of a grid that find_place() deals out
static unsigned prompt_grid(int tiles, int splits, int Hkv)
{
    const unsigned n = (unsigned)tiles * (unsigned)splits;
    if (Hkv % 8 == 0) return n * (unsigned)Hkv;
    if (8 % Hkv == 0) return (n + 8u / Hkv - 1) / (8u / Hkv) * 8u;
    return n * (unsigned)Hkv;
}

}  // namespace w4

using namespace w4;

extern "C" {

size_t w4a16_prompt_attn_workspace_bytes(int rows, int B, int max_q, int max_k, int Hq, int Hkv, int D)
{
    if (check_prompt_sizes(rows, B, max_q, max_k, Hq, Hkv, D) != W4A16_OK) return 0;
    const PromptPlan p = prompt_plan(rows, B, max_q, max_k, Hq, Hkv, D);
    return kTicketBytes + p.o_bytes + p.ml_bytes;
}

int w4a16_prompt_attn(const void *q, const void *k, const void *v, const int32_t *q_start, const int32_t *k_start, const int32_t *k_len, void *out, int B,
                      int rows, int k_rows, int max_q, int max_k, int Hq, int Hkv, int D, float scale, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_prompt_sizes(rows, B, max_q, max_k, Hq, Hkv, D);
    if (rc != W4A16_OK) return rc;
    if (k_rows < 1 || !(scale > 0.f) || !(scale < __builtin_inff())) return W4A16_EINVAL;
    if (!q || !k || !v || !q_start || !out || (k_start == nullptr) != (k_len == nullptr)) return W4A16_ENULL;
    if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) ||
        ((reinterpret_cast<uintptr_t>(q_start) | reinterpret_cast<uintptr_t>(k_start) | reinterpret_cast<uintptr_t>(k_len)) & 3u))
        return W4A16_EALIGN;
    const PromptPlan p = prompt_plan(rows, B, max_q, max_k, Hq, Hkv, D);
    if (!workspace || workspace_bytes < kTicketBytes + p.o_bytes + p.ml_bytes) return W4A16_EWORKSPACE;
    if (workspace_misaligned(workspace)) return W4A16_EALIGN;
    float *const part_o = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + kTicketBytes);
    const PromptArgs a = {(const _Float16 *)q, (const _Float16 *)k, (const _Float16 *)v, q_start, k_start, k_len, (_Float16 *)out, part_o,
                          part_o + p.o_bytes / 4, B, rows, k_rows, Hq, Hkv, Hq / Hkv, p.tiles, p.splits, scale * 1.44269504088896340736f};
    const unsigned grid = prompt_grid(p.tiles, p.splits, Hkv);
    if (D == 128) hipLaunchKernelGGL((prompt_attn_tile_kernel<128, 8, 1>), dim3(grid), dim3(512), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL((prompt_attn_tile_kernel<64, 8, 1>), dim3(grid), dim3(512), 0, (hipStream_t)stream, a);
    if (p.splits > 1) {
        const dim3 merge(prompt_grid(p.tiles, 1, Hkv), 8);
        if (D == 128) hipLaunchKernelGGL((prompt_attn_merge_kernel<128, kTileRows>), merge, dim3(256), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL((prompt_attn_merge_kernel<64, kTileRows>), merge, dim3(256), 0, (hipStream_t)stream, a);
    }
    return launch_status();
}

}  // extern "C"
