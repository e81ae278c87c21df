// w4a16_prompt_attn: causal attention of packed sequences of different lengths over their keys in a cache.  Contract in include/w4a16.h.
//
// The (query, head) pairs that share a KV head are the rows of one problem: query-major, pair = query * group + head in its group, so that a
// tile of rows spans few queries and the keys it sees end almost together.  S^T = K . Q^T leaves a lane with scores of ONE pair (column
// lane % 32), which are the operand of O^T += V^T . P^T as they stand; the softmax runs in registers, one pass over the keys.
//
// Lengths are known on the device only, so the work is dealt out there.  Where there are tiles enough, each workgroup takes one.  Where there are few,
// the tiles of all sequences and KV heads, each as long as the keys that it sees, lie end to end, and every workgroup takes an equal stretch of that
// line.  A tile that a border falls into is cut there; the pieces are joined by the last of their workgroups to finish (rows of single tokens;
// exchange as in tree_attn_kernel; a border cuts one tile, so the tickets of the workgroups do for the tiles) or by a kernel of its own.
#include "attn_common.h"

namespace w4 {

typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) half4v lds_half4v;

constexpr int kMostSequences = 4096;
constexpr int kMostTiles = 1 << 20;   // that are counted; more than workgroups anyhow
constexpr float kLag = 8.f, kRaise = 7.f;   // probabilities reach 2^(kLag + kRaise), and 2^(1/8) times that (see kFar): fp16 ends below 2^16
constexpr float kFar = 0x1p20f;   // scaled scores from here on: half a last place is 2^-4 here
constexpr float kMostScale = 0x1p60f;   // |q . k| of 128 fp16 products is below 2^39, a scaled score above kLowest
constexpr int kMostGroups = 256;   // workgroups of a call: one per compute unit, a ticket each

struct PromptArgs {
    const _Float16 *q, *k, *v;
    const int32_t *q_start, *k_start, *k_len;   // k_start, k_len: both or none
    _Float16 *out;
    float *part_o, *part_ml;   // two pieces per workgroup: the cut tile at the start of its stretch, and the one at its end
    uint32_t *tickets;
    int B, rows, k_rows, Hq, Hkv, group;
    float scale_log2e;
};

// a / b for 0 <= a < 2^62, 0 < b < 2^55 and a quotient below 2^40: exact.  The reciprocal (after one Newton step good to 2^-45 and better) makes
// the quotient off by one at the most.
__device__ __forceinline__ long long divide(long long a, long long b)
{
    const double d = (double)b, r0 = __builtin_amdgcn_rcp(d), r = __builtin_fma(__builtin_fma(-d, r0, 1.0), r0, r0);
    const long long q = (long long)((double)a * r), left = a - q * b;
    return q + (left >= b) - (left < 0);
}

// What a piece costs beside its keys (places, first transfers, exchange), in keys: 6 us and more, in which 32 or 256 rows go through some 300.  64 sequences of up to
// 4096 keys, one query each, 32/8 heads: counted as 384 keys 36 us, as 256 44, 96 70; as 512 no less.
constexpr int kPieceKeys = 384;

// A sequence, and its place on the line of work.  Tile t of a KV head reaches from cost(t) to cost(t + 1): the keys that its last query sees, about,
// and kPieceKeys, each counted `group` times: nothing is divided.
struct Sequence {
    int n, T, q0, k0, tiles;
    int ahead;   // keys ahead of the first query
};
template <int ROWS>
__device__ __forceinline__ long long cost(const Sequence &s, int group, int t)
{
    return (long long)t * (s.ahead + kPieceKeys) * group + (long long)t * (t + 1) * (ROWS / 2);
}

// sequence b, no tiles if its rows or keys do not lie in the buffers
template <int ROWS>
__device__ __forceinline__ Sequence read_sequence(const PromptArgs &a, int b)
{
    Sequence s = {0, 0, 0, 0, 0, 0};
    if (b < 0 || b >= a.B) return s;
    const int q0 = a.q_start[b], q1 = a.q_start[b + 1];
    const bool rows_fit = q0 >= 0 && q1 > q0 && q1 <= a.rows;
    const int k0 = a.k_len ? a.k_start[b] : q0, T = a.k_len ? a.k_len[b] : rows_fit ? q1 - q0 : 0;
    if (!rows_fit || k0 < 0 || T < 0 || (long long)k0 + T > a.k_rows) return s;
    s.n = q1 - q0;
    s.T = T;
    s.q0 = q0;
    s.k0 = k0;
    s.tiles = (int)(((long long)s.n * a.group + ROWS - 1) / ROWS);
    s.ahead = max(T - s.n, 0);
    return s;
}

__device__ __forceinline__ long long shuffle(long long x, int src)
{
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)x, src, 64), hi = (uint32_t)__shfl((int)(x >> 32), src, 64);
    return (long long)((uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ long long of_lane(long long x, int src)
{
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, src), hi = __builtin_amdgcn_readlane((int)(x >> 32), src);
    return (long long)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ long long uniform(long long x) { return of_lane(x, 0); }

constexpr long long kLongestLine = 1ll << 60;   // beyond any sensible call (sequences that share rows); sums stay in 64 bits

// The line of work, as one wavefront sees it (the same in all of them).  Sequences are read 64 at a time, one per lane.
template <int ROWS>
struct Line {
    long long total;              // its length
    int tiles;                    // on it (at most kMostTiles are counted)
    long long from, to;           // the sequence at hand reaches from .. to
    long long per_head;           // of each KV head
    Sequence seq;
    long long before;             // length up to the first of the 64 sequences from `base` on, among which the one at hand is
    int base;

    // sequence base + lane, and the length up to and including it (and tiles)
    __device__ __forceinline__ long long read(const PromptArgs &a, Sequence &mine, int &upto_tiles, int lane) const
    {
        mine = read_sequence<ROWS>(a, base + lane);
        long long upto = min(cost<ROWS>(mine, a.group, mine.tiles) * a.Hkv, kLongestLine);
        upto_tiles = min(mine.tiles * a.Hkv, kMostTiles);
        const int here = min(64, a.B - base);
        for (int off = 1; off < here; off <<= 1) {
            const long long other = shuffle(upto, max(lane - off, 0));
            const int other_tiles = __shfl(upto_tiles, max(lane - off, 0), 64);
            if (lane >= off) {
                upto = min(upto + other, kLongestLine);
                upto_tiles = min(upto_tiles + other_tiles, kMostTiles);
            }
        }
        return min(upto + before, kLongestLine);
    }
    __device__ __forceinline__ Line(const PromptArgs &a, int lane, Sequence &mine, long long &upto, int &upto_tiles)
    {
        total = from = to = per_head = before = 0;
        tiles = 0;
        for (base = 0; base < a.B; base += 64) {
            upto = read(a, mine, upto_tiles, lane);
            before = of_lane(upto, min(63, a.B - base - 1));
            tiles = min(tiles + __builtin_amdgcn_readlane(upto_tiles, min(63, a.B - base - 1)), kMostTiles);
        }
        total = before;
        before = 0;
        base = 0;
    }
    // brings the sequence that holds place `at` to hand; at < total, and no place before the last one asked for.  mine, upto: what the constructor
    // read, if `known`.  False if there is none: lengths that were changed under the running kernel
    __device__ __forceinline__ bool find(const PromptArgs &a, long long at, int lane, Sequence mine, long long upto, bool known)
    {
        if (at >= from && at < to) return true;
        for (; base < a.B; base += 64) {
            int upto_tiles;
            if (!known) upto = read(a, mine, upto_tiles, lane);
            known = false;
            const uint64_t hit = __ballot(upto > at && base + lane < a.B);
            if (hit) {
                const int src = __builtin_ctzll(hit);
                auto take = [&](int x) { return __builtin_amdgcn_readlane(x, src); };
                seq = {take(mine.n), take(mine.T), take(mine.q0), take(mine.k0), take(mine.tiles), take(mine.ahead)};
                per_head = cost<ROWS>(seq, a.group, seq.tiles);
                to = of_lane(upto, src);
                from = to - per_head * a.Hkv;
                return true;
            }
            before = of_lane(upto, 63);
        }
        return false;
    }
    // brings the sequence of tile `number` of the line to hand, right after the constructor (mine and the like as for find()); where the tile begins, or
    // -1 if there are fewer
    __device__ __forceinline__ long long find_tile(const PromptArgs &a, int number, int lane, Sequence mine, long long upto, int upto_tiles, bool known)
    {
        for (; base < a.B; base += 64) {
            if (!known) upto = read(a, mine, upto_tiles, lane);
            known = false;
            const uint64_t hit = __ballot(upto_tiles > number && base + lane < a.B);
            if (hit) {
                const int src = __builtin_ctzll(hit);
                auto take = [&](int x) { return __builtin_amdgcn_readlane(x, src); };
                seq = {take(mine.n), take(mine.T), take(mine.q0), take(mine.k0), take(mine.tiles), take(mine.ahead)};
                per_head = cost<ROWS>(seq, a.group, seq.tiles);
                to = of_lane(upto, src);
                from = to - per_head * a.Hkv;
                const int of_it = number - (take(upto_tiles) - seq.tiles * a.Hkv), kvh = of_it / seq.tiles;
                return from + kvh * per_head + cost<ROWS>(seq, a.group, of_it - kvh * seq.tiles);
            }
            before = of_lane(upto, 63);
            number -= __builtin_amdgcn_readlane(upto_tiles, 63);
        }
        return -1;
    }
};

// One piece of work: steps s0 .. s1 - 1 of a tile.
struct Piece {
    int kvh, first, rows;      // KV head, pair of the first row, rows
    int steps, s0, s1;         // of the whole tile; of this piece
    long long begin, end;      // of the tile on the line
};
template <int ROWS, int STEP>
__device__ __forceinline__ void tile_of(const PromptArgs &a, const Line<ROWS> &line, long long at, Piece &p)
{
    const Sequence &s = line.seq;
    long long rel = at - line.from;
    p.kvh = __builtin_amdgcn_readfirstlane((int)divide(rel, line.per_head));
    rel -= p.kvh * line.per_head;
    int lo = 0, hi = s.tiles - 1;   // the last tile that begins at or before rel
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cost<ROWS>(s, a.group, mid) <= rel) lo = mid;
        else hi = mid - 1;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    p.begin = uniform(line.from + p.kvh * line.per_head + cost<ROWS>(s, a.group, lo));
    p.end = uniform(line.from + p.kvh * line.per_head + cost<ROWS>(s, a.group, lo + 1));
    const int pairs = s.n * a.group;
    p.first = lo * ROWS;
    p.rows = min(ROWS, pairs - p.first);
    const int seen = s.T - s.n + (p.first + p.rows - 1) / a.group + 1;   // keys that the tile's last row sees
    p.steps = __builtin_amdgcn_readfirstlane(seen > 0 ? (seen + STEP - 1) / STEP : 0);
}
// step of a tile at a place on the line
__device__ __forceinline__ int step_at(const Piece &p, long long at)
{
    return at >= p.end ? p.steps : (int)divide((at - p.begin) * p.steps, p.end - p.begin);
}

// Workgroups go to the eight XCDs in turn; an XCD gets neighbouring stretches, so that its L2 holds the keys of few heads.
__device__ __forceinline__ unsigned stretch_number(unsigned block, unsigned grid)
{
    const unsigned xcd = block & 7u;
    return xcd * (grid >> 3) + min(xcd, grid & 7u) + (block >> 3);
}

__device__ __forceinline__ half8v read_chunk(const uint8_t *p) { return *reinterpret_cast<const half8v *>(p); }
// four key rows of a column each, transposed (see tree_attn_wave_kernel): the compiler counts and waits for this read
__device__ __forceinline__ half4v read_transposed(const uint8_t *p)
{
    return __builtin_bit_cast(half4v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)p));
}
__device__ __forceinline__ bool not_finite(_Float16 x) { return (__builtin_bit_cast(uint16_t, x) & 0x7C00u) == 0x7C00u; }
// one of eight: an exponent of all ones, and no other, carries into the bit of the sign
__device__ __forceinline__ bool not_finite(half8v x)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 b = (__builtin_bit_cast(u32x4, x) & 0x7FFF7FFFu) + 0x04000400u;
    return ((b[0] | b[1] | b[2] | b[3]) & 0x80008000u) != 0;
}

// Chunks of sixteen bytes lie permuted in the LDS tiles, so that fragment reads spread over the 64 banks (256 bytes, two rows of 64 values): sixteen lanes of a
// K read take one chunk of sixteen keys, 32 of a V read four chunks of four keys.  With permutations of eight chunks and of pairs a quarter of all cycles went
// to conflicts.
template <int D>
struct Tile {
    static constexpr int ROW = D * 2, CHUNKS = D / 8;
    __device__ __forceinline__ static int k_chunk(int key, int chunk) { return chunk ^ (D == 128 ? key & 15 : key >> 1 & 7); }
    __device__ __forceinline__ static int v_chunk(int key, int chunk) { return chunk ^ (D == 128 ? 4 * key & 15 : 2 * key & 7); }
    __device__ __forceinline__ static uint32_t k_place(int key, int chunk) { return (uint32_t)(key * ROW + (k_chunk(key, chunk) << 4)); }
    __device__ __forceinline__ static uint32_t v_place(int key, int chunk) { return (uint32_t)(key * ROW + (v_chunk(key, chunk) << 4)); }
};

// 32 rows (pairs) of a wavefront, lane column c = lane % 32: queries, outputs so far and the running state of the softmax
template <int D>
struct Rows {
    half8v qf[D / 16];
    float16v o[D / 32];
    float m_run, l_run;   // l_run: this lane's share (its keys) of the row's sum
    float lag;            // how far a score may exceed m_run before that moves
    int pos;              // the row sees keys 0 .. pos

    __device__ __forceinline__ void start(const PromptArgs &a, const Sequence &s, const Piece &p, int row, int h)
    {
        const int pair = p.first + min(row, p.rows - 1), query = pair / a.group;
        pos = s.T - s.n + query;
        const _Float16 *src = a.q + ((size_t)(s.q0 + query) * a.Hq + p.kvh * a.group + (pair - query * a.group)) * D + 8 * h;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) qf[j] = *reinterpret_cast<const half8v *>(src + 16 * j);
        m_run = kLowest;
        lag = kLag;
        l_run = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    }
    // Makes the compiler wait for the queries here: left to their first use, in the loop, its wait would count the transfers under way there, too.
    __device__ __forceinline__ void arrive()
    {
#pragma unroll
        for (int j = 0; j < D / 16; ++j) asm volatile("" : "+v"(qf[j]));
    }

    // scores of 32 keys, in two steps: the fragments of the K tile, and their products
    __device__ __forceinline__ static void read_keys(half8v (&kf)[D / 16], const uint8_t *ktile, uint32_t kfrag)
    {
#pragma unroll
        for (int j = 0; j < D / 16; ++j) kf[j] = read_chunk(ktile + (kfrag ^ (j << 5)));
    }
    __device__ __forceinline__ void scores(float16v &s, const half8v (&kf)[D / 16]) const
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[j], qf[j], s, 0, 0, 0);
    }

    // their probabilities, as operands of the product with the values, and the running sum; scales the outputs where their reference moves
    template <int KT>
    __device__ __forceinline__ void probabilities(float16v (&s)[KT], half8v (&pb)[2 * KT], float scale_log2e)
    {
        float m[2] = {max_of_two(s[0][0], s[0][1]), max_of_two(s[0][2], s[0][3])};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = kt ? 0 : 4; i < 16; i += 2) m[(i >> 1) & 1] = max_of_three(m[(i >> 1) & 1], s[kt][i], s[kt][i + 1]);
        // The scale is positive (checked by the host): the largest raw score is the largest scaled one.  The maximum that the exponentials are taken
        // from moves only where it has grown by kLag: the outputs are seldom scaled, and any reference that is not far below the largest score serves as well.
        // It is lowered by kRaise, so that fp16 probabilities use the range that it leaves above: up to 2^15 now, and weights down to 2^-32 of the largest count
        // (2^-25 without it: behind a key 26 binary orders above all others 9000 keys kept 15 % of their weight or none).  The products' operands are fp16
        // because the matrix instruction with fp32 has a sixteenth of the rate; rounding each probability to 11 bits leaves an output within 2^-11 of its
        // weighted magnitudes, as its own rounding does.
        // The largest score's product with the scale is rounded in the maximum and not in the multiply-add below: half a last place of the maximum, which from
        // 2^27 on is more than a probability in fp16 has room for.  Far from zero a row's scores are scaled, and so rounded alike, beforehand and their distance from the
        // maximum takes their place (over the scale, so that the multiply-add is the same for all rows): such a row comes by here in every step.
        const float m_seen = half_wave_max(max_of_two(m[0], m[1])) * scale_log2e, grown = m_seen - m_run;
        float less = kRaise - m_run;
        if (__any(grown > lag)) {
            const float m_new = grown > kLag ? m_seen : m_run, alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) o[dt] *= alpha;
            const bool far = __builtin_fabsf(m_new) >= kFar && __builtin_fabsf(m_new) < -kLowest;   // neither a row that has seen nothing nor an infinite one
            lag = far ? -__builtin_inff() : kLag;
            less = far ? kRaise : kRaise - m_new;
            if (__any(far)) {
                const float over = 1.f / scale_log2e;
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kt][i] = far ? (keep_f32(s[kt][i] * scale_log2e) - m_new) * over : s[kt][i];
            }
        }
        float sum[2] = {};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][i], scale_log2e, less));
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][i + 1], scale_log2e, less));
                const half2v both = __builtin_convertvector((float2v){p0, p1}, half2v);
                sum[(i >> 1) & 1] = __builtin_amdgcn_fdot2(both, (half2v){1, 1}, sum[(i >> 1) & 1], false);   // of what multiplies the values; one instruction for two
                pb[2 * kt + (i >> 3)][i & 7] = both[0];
                pb[2 * kt + (i >> 3)][(i & 7) + 1] = both[1];
            }
        l_run += sum[0] + sum[1];
    }

    // the same with the mask
    template <int KT, bool MASKED>
    __device__ __forceinline__ void softmax(float16v (&s)[KT], half8v (&pb)[2 * KT], int key0, float scale_log2e, int h)
    {
        if constexpr (KT == 2) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(s[0]), "+v"(s[1]));   // settled() for both
        else settled(s[0]);
        if constexpr (MASKED) {
            const int room = pos - key0 - 4 * h;   // key 32 kt + 8 (i / 4) + 4 h + i % 4 of the tile is seen up to the position
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kt][i] = 32 * kt + 8 * (i >> 2) + (i & 3) <= room ? s[kt][i] : -__builtin_inff();
        }
        probabilities<KT>(s, pb, scale_log2e);
    }

    // fragments u of the V tile: 16 keys, all D values
    __device__ __forceinline__ static void read_values(half8v (&vf)[D / 32], const uint8_t *vtile, int u, uint32_t vfrag)
    {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            const uint8_t *const p = vtile + u * 16 * Tile<D>::ROW + (vfrag ^ (dt << 6));
            const half4v lo = read_transposed(p), hi = read_transposed(p + 8 * Tile<D>::ROW);
            vf[dt] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    __device__ __forceinline__ void add_product(const half8v (&vf)[D / 32], half8v pb)
    {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[dt], pb, o[dt], 0, 0, 0);
    }
    // rows that do see a value that is not finite: it joins their sums as it is
    template <int KT>
    __device__ __forceinline__ void add_not_finite(const uint8_t *vtile, int key0, int h)
    {
        for (int key = 0; key < 32 * KT; ++key)
            for (int chunk = 0; chunk < D / 8; ++chunk) {   // elements 8 chunk + 4 h ..
                const half4v x = *reinterpret_cast<const half4v *>(vtile + Tile<D>::v_place(key, chunk) + 8 * h);
                if (!__any(not_finite(x[0]) || not_finite(x[1]) || not_finite(x[2]) || not_finite(x[3])) || key0 + key > pos) continue;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int quad = 0; quad < 4; ++quad)
                        if (4 * dt + quad == chunk)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[dt][4 * quad + e] += not_finite(x[e]) ? (float)x[e] : 0.f;
            }
    }
    template <int KT>
    __device__ __forceinline__ void values(const half8v (&pb)[2 * KT], const uint8_t *vtile, uint32_t vfrag)
    {
        half8v vf[2][D / 32];
        read_values(vf[0], vtile, 0, vfrag);
#pragma unroll
        for (int u = 0; u < 2 * KT; ++u) {
            if (u + 1 < 2 * KT) read_values(vf[(u + 1) & 1], vtile, u + 1, vfrag);
            add_product(vf[u & 1], pb[u]);
        }
        settled(o[D / 32 - 1]);   // the branches behind this go round too little for the last product
    }
};

// values that a wavefront brought to LDS, 1 KB N times: is one of them not finite (this lane's share); and zeros in the place of those
template <int N>
__device__ __forceinline__ bool any_not_finite(const uint8_t *at, int lane)
{
    bool found = false;
#pragma unroll
    for (int i = 0; i < N; ++i) found |= not_finite(read_chunk(at + i * 1024 + lane * 16));
    return found;
}
template <int N>
__device__ __forceinline__ void clear_not_finite(uint8_t *at, int lane)
{
    for (int i = 0; i < N; ++i) {
        half8v *const x = reinterpret_cast<half8v *>(at + i * 1024 + lane * 16);
        for (int e = 0; e < 8; ++e)
            if (not_finite((*x)[e])) (*x)[e] = 0;
    }
}

// V: lane s of 16-lane block b points at key row 4 (b / 2) + s / 4 (and 8 further on), elements 32 dt + 16 (b % 2) + 4 (s % 4) ..
template <int D>
__device__ __forceinline__ uint32_t v_fragment(int lane)
{
    const int key = 4 * (lane >> 5) + ((lane & 15) >> 2);
    return Tile<D>::v_place(key, 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) + 8 * (lane & 1);
}

// where a row's output belongs, and what its sum of weighted values is to be multiplied by: a row that sees no key gets zeros; one whose scores are
// all -inf 0 / 0
__device__ __forceinline__ _Float16 *row_of(const PromptArgs &a, const Sequence &s, const Piece &p, int row, int D)
{
    const int pair = p.first + row, query = pair / a.group;
    return a.out + ((size_t)(s.q0 + query) * a.Hq + p.kvh * a.group + (pair - query * a.group)) * D;
}
__device__ __forceinline__ float row_factor(const PromptArgs &a, const Sequence &s, const Piece &p, int row, float l)
{
    return s.T - s.n + (p.first + row) / a.group >= 0 ? 1.f / l : 0.f;
}
__device__ __forceinline__ void store_row_quad(const PromptArgs &a, const Sequence &s, const Piece &p, int row, int D, int d, float4v val, float l)
{
    const float inv = row_factor(a, s, p, row, l);
    half4v y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (_Float16)(val[e] * inv);
    *reinterpret_cast<half4v *>(row_of(a, s, p, row, D) + d) = y;
}

// Where the piece of a cut tile goes: workgroup i keeps the tile that its stretch begins in at 2 i, the one that it ends in at 2 i + 1.
template <int D, int ROWS>
struct Pieces {
    __device__ __forceinline__ static PartialBuffer o(const PromptArgs &a, unsigned slot) { return partial_buffer(a.part_o + (size_t)slot * ROWS * D); }
    __device__ __forceinline__ static PartialBuffer ml(const PromptArgs &a, unsigned slot) { return partial_buffer(a.part_ml + (size_t)slot * ROWS * 2); }
};

// Joins `pieces` pieces of rows row0 .. row1 - 1 of a cut tile.  Where the rows are few, several groups of threads take
// every so-manieth piece each and meet in LDS (`shared`, THREADS * 24 bytes): a piece's loads are one trip to memory, eight at a time.
// SAME: written by other workgroups of the same kernel.
template <int D, int ROWS, int THREADS, bool SAME>
__device__ __forceinline__ void join_pieces(const PromptArgs &a, const Sequence &s, const Piece &p, const uint16_t *slots, int pieces, int row0, int row1, int tid, float *shared)
{
    const int items = (row1 - row0) * (D / 4);
    const int parts = items <= THREADS / 4 ? 4 : items <= THREADS / 2 ? 2 : 1, stride = THREADS / parts;   // uniform
    const int part = tid / stride;
    for (int item = tid % stride; item < items; item += stride) {
        const int row = row0 + item / (D / 4), d4 = item % (D / 4);
        float m = kLowest, den = 0.f;
        float4v num = {0.f, 0.f, 0.f, 0.f};
        constexpr int AT_ONCE = 8;
        for (int w = part; w < pieces; w += AT_ONCE * parts) {
            float ms[AT_ONCE], ls[AT_ONCE];
            float4v os[AT_ONCE];
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) {
                const unsigned slot = __builtin_amdgcn_readfirstlane(slots[min(w + e * parts, pieces - 1)]);   // a wavefront is in one part
                if constexpr (SAME) {
                    const PartialBuffer po = Pieces<D, ROWS>::o(a, slot), pm = Pieces<D, ROWS>::ml(a, slot);
                    ms[e] = load_partial_f32(pm, 2 * row);
                    ls[e] = load_partial_f32(pm, 2 * row + 1);
                    os[e] = load_partial(po, row * (D / 4) + d4);
                } else {
                    const float *const ml = a.part_ml + (size_t)slot * ROWS * 2 + 2 * row;
                    ms[e] = ml[0];
                    ls[e] = ml[1];
                    os[e] = *reinterpret_cast<const float4v *>(a.part_o + (size_t)slot * ROWS * D + row * D + 4 * d4);
                }
            }
            float top = m;
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) top = fmaxf(top, ms[e]);
            const float keep = __builtin_amdgcn_exp2f(m - top);
            den *= keep;
            num *= keep;
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) {
                if (w + e * parts >= pieces) break;
                const float wgt = __builtin_amdgcn_exp2f(ms[e] - top);
                den += wgt * ls[e];
                num += wgt * os[e];
            }
            m = top;
        }
        if (parts > 1) {   // uniform; there is one round of items then
            *reinterpret_cast<float4v *>(shared + tid * 4) = num;
            shared[THREADS * 4 + tid] = m;
            shared[THREADS * 5 + tid] = den;
        } else store_row_quad(a, s, p, row, D, 4 * d4, num, den);
    }
    if (parts > 1) {
        __syncthreads();
        if (tid < items) {
            float m = kLowest, den = 0.f;
            float4v num = {0.f, 0.f, 0.f, 0.f};
            for (int g = 0; g < parts; ++g) m = fmaxf(m, shared[THREADS * 4 + g * stride + tid]);
            for (int g = 0; g < parts; ++g) {
                const float wgt = __builtin_amdgcn_exp2f(shared[THREADS * 4 + g * stride + tid] - m);
                den += wgt * shared[THREADS * 5 + g * stride + tid];
                num += wgt * *reinterpret_cast<const float4v *>(shared + (g * stride + tid) * 4);
            }
            store_row_quad(a, s, p, row0 + tid / (D / 4), D, tid % (D / 4) * 4, num, den);
        }
    }
}

// The cut of a line into stretches.
template <int ROWS>
struct Cut {
    unsigned groups;
    long long length, total;
    // grid: workgroups at most; least: a tile is not cut into pieces shorter than this, in keys
    __device__ __forceinline__ Cut(const Line<ROWS> &line, int group, unsigned grid, int least)
    {
        // as many workgroups as tiles, or as stretches of a length that is worth one; a multiple of the tiles, so that those of one length are cut alike
        total = line.total;
        groups = (unsigned)__builtin_amdgcn_readfirstlane((int)min((long long)grid, max((long long)max(line.tiles, 1), divide(total, (long long)least * group))));
        if (line.tiles > 0 && (unsigned)line.tiles < groups) groups -= groups % (unsigned)line.tiles;
        length = uniform(divide(total + groups - 1, groups));
    }
    __device__ __forceinline__ long long border(unsigned w) const { return min(length * w, total); }
    // Collects the pieces of a cut tile: where each is kept, in the order of their keys.  w0 .. : the workgroups among which it lies.  All threads; `slots` and
    // the count are there behind the caller's next barrier.  Returns this thread's part of the work that is left: see finish().
    struct Found {
        bool has;
        unsigned slot;
        uint64_t all;
    };
    __device__ __forceinline__ Found look(const Piece &p, unsigned w0, int tid, int lane, uint32_t *pieces_sh) const
    {
        const unsigned w1 = (unsigned)divide(p.end - 1, length), w = w0 + tid;
        Found f = {false, 0, 0};
        if (w <= w1) {
            const long long b = border(w), e = border(w + 1);
            f.has = step_at(p, max(b, p.begin)) != step_at(p, min(e, p.end));
            f.slot = 2 * w + (p.begin > b ? 1 : 0);
        }
        f.all = __ballot(f.has);
        if (lane == 0) pieces_sh[tid >> 6] = (uint32_t)__builtin_popcountll(f.all);
        return f;
    }
    template <int WAVES>
    __device__ __forceinline__ uint32_t finish(const Found &f, int tid, int lane, const uint32_t *pieces_sh, uint16_t *slots) const
    {
        uint32_t pieces = 0, ahead = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            ahead += i < (tid >> 6) ? pieces_sh[i] : 0;
            pieces += pieces_sh[i];
        }
        if (f.has) slots[ahead + __builtin_popcountll(f.all & ((1ull << lane) - 1))] = (uint16_t)f.slot;
        return pieces;
    }
};

// Goes through a workgroup's stretch, piece by piece.  work(sequence, piece, whole, slot) computes steps s0 .. s1 - 1 (s0 < s1) and stores the
// outputs (whole) or the piece's state.  JOIN: the last workgroup of a cut tile to finish joins its pieces; else prompt_attn_join_kernel does.
template <int D, int ROWS, int STEP, int LEAST, int THREADS, bool JOIN, typename Work>
__device__ __forceinline__ void go_through(const PromptArgs &a, int tid, float *shared, Work work)
{
    static_assert(kMostGroups <= THREADS, "");
    const int lane = tid & 63;
    __shared__ uint32_t ticket_sh, pieces_sh[THREADS / 64];
    __shared__ uint16_t slots[kMostGroups];
    Sequence mine;
    long long first_upto;
    int upto_tiles;
    Line<ROWS> line(a, lane, mine, first_upto, upto_tiles);
    const Cut<ROWS> cut(line, a.group, gridDim.x, LEAST);
    if (blockIdx.x >= cut.groups) return;
    const unsigned me = stretch_number(blockIdx.x, cut.groups);
    const long long start = cut.border(me), stop = cut.border(me + 1);
    long long at = start;
    if (at < stop && !line.find(a, at, lane, mine, first_upto, a.B <= 64)) return;
    while (at < stop) {   // uniform over the workgroup
        Piece p;
        tile_of<ROWS, STEP>(a, line, at, p);
        const long long upto = stop < p.end ? stop : p.end;
        p.s0 = __builtin_amdgcn_readfirstlane(step_at(p, at));
        p.s1 = __builtin_amdgcn_readfirstlane(step_at(p, upto));
        if (p.steps == 0) {   // none of its rows sees a key
            if (at == p.begin)
                for (int item = tid; item < p.rows * (D / 4); item += THREADS)
                    store_row_quad(a, line.seq, p, item / (D / 4), D, item % (D / 4) * 4, (float4v){0.f, 0.f, 0.f, 0.f}, 1.f);
        } else if (p.s0 < p.s1) {
            const bool whole = p.s1 - p.s0 == p.steps;
            work(line.seq, p, whole, 2 * me + (at > start ? 1u : 0u));
            if (JOIN && !whole) {
                const unsigned w0 = (unsigned)__builtin_amdgcn_readfirstlane((int)divide(p.begin, cut.length));   // the workgroup that the tile begins in: its ticket
                const auto found = cut.look(p, w0, tid, lane, pieces_sh);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wavefront's part of the piece has reached memory
                __syncthreads();
                const uint32_t pieces = cut.template finish<THREADS / 64>(found, tid, lane, pieces_sh, slots);
                if (tid == 0) ticket_sh = __hip_atomic_fetch_add(&a.tickets[w0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __syncthreads();
                if (ticket_sh == pieces - 1) {
                    if (tid == 0) __hip_atomic_store(&a.tickets[w0], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    join_pieces<D, ROWS, THREADS, true>(a, line.seq, p, slots, (int)pieces, 0, p.rows, tid, shared);
                }
            }
            __syncthreads();   // LDS and the ticket are free for the next piece
        }
        at = upto;
        if (at < stop && !line.find(a, at, lane, mine, 0, false)) return;
    }
}

// Joins the pieces of the tiles that the tile kernel's stretches cut, kJoinRows rows to a workgroup: a tile of 256 rows is 128 KB a piece, of which one
// workgroup alone reads 20 KB in a microsecond (4 x 64 queries behind 7936 keys, 32/8 heads: 103 us joined by the last to finish, 57 like this).
// blockIdx.x: rows (next to each other on all XCDs); blockIdx.y: the tile.  With a workgroup per stretch instead, most of which find that no tile begins
// there, 72 queries over 20000 keys and 50 over 18000, 16/2 heads, took 71 us, like this 61.
constexpr int kJoinRows = 8;
template <int D, int ROWS, int STEP, int LEAST>
__global__ __launch_bounds__(256) void prompt_attn_join_kernel(PromptArgs a, unsigned stretches)
{
    static_assert(kMostGroups <= 256, "");
    const int tid = threadIdx.x, lane = tid & 63;
    __shared__ uint32_t pieces_sh[4];
    __shared__ uint16_t slots[kMostGroups];
    __shared__ __attribute__((aligned(16))) float shared[256 * 6];
    Sequence mine;
    long long first_upto;
    int upto_tiles;
    Line<ROWS> line(a, lane, mine, first_upto, upto_tiles);
    const Cut<ROWS> cut(line, a.group, stretches, LEAST);
    const long long at = line.find_tile(a, (int)blockIdx.y, lane, mine, first_upto, upto_tiles, a.B <= 64);
    if (at < 0) return;
    Piece p;
    tile_of<ROWS, STEP>(a, line, at, p);
    const int row0 = blockIdx.x * kJoinRows;
    const unsigned me = (unsigned)__builtin_amdgcn_readfirstlane((int)divide(p.begin, cut.length));   // the stretch that it begins in
    if (p.end <= cut.border(me + 1) || p.steps == 0 || row0 >= p.rows) return;   // not cut
    const auto found = cut.look(p, me, tid, lane, pieces_sh);
    __syncthreads();
    const uint32_t pieces = cut.template finish<4>(found, tid, lane, pieces_sh, slots);
    __syncthreads();
    if (pieces < 2) return;   // one workgroup has all its steps and has stored the outputs
    join_pieces<D, ROWS, 256, false>(a, line.seq, p, slots, (int)pieces, row0, min(row0 + kJoinRows, p.rows), tid, shared);
}

// Many tiles: one per workgroup, whole.  They are numbered from the last of the last sequence down, so that the tiles that see most keys of a sequence are
// the first to be dealt out, and an XCD keeps to its own KV heads or to its share of a head's tiles: workgroups that start together read the same keys,
// which come from memory once for all of them (16384 queries, 32/8 heads: 2449 us, in equal stretches 3000).  The order of sequences stays the caller's: a prompt
// of 2000 in front of 30 of 200, 32/8 heads, begins last, 94 us, and behind them first, 84.
template <int D, int ROWS, int STEP, typename Work>
__device__ __forceinline__ void take_one(const PromptArgs &a, int lane, Work work)
{
    const unsigned xcd = blockIdx.x & 7u, turn = blockIdx.x >> 3, heads = (unsigned)a.Hkv;
    unsigned kvh, number;
    if (heads % 8 == 0) {
        kvh = xcd + 8 * (turn % (heads >> 3));
        number = turn / (heads >> 3);
    } else if (8 % heads == 0) {
        kvh = xcd % heads;
        number = turn * (8 / heads) + xcd / heads;
    } else {
        kvh = blockIdx.x % heads;
        number = blockIdx.x / heads;
    }
    long long before = 0;
    for (int base = 0; base < a.B; base += 64) {   // 64 sequences at a time, the last first
        const Sequence mine = read_sequence<ROWS>(a, a.B - 1 - base - lane);
        int upto = mine.tiles;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int other = __shfl_up(upto, off, 64);
            if (lane >= off) upto += other;
        }
        const uint64_t hit = __ballot(before + upto > (long long)number);
        if (hit) {
            const int src = __builtin_ctzll(hit);
            auto take = [&](int x) { return __builtin_amdgcn_readlane(x, src); };
            const Sequence s = {take(mine.n), take(mine.T), take(mine.q0), take(mine.k0), take(mine.tiles), take(mine.ahead)};
            Piece p;
            p.kvh = (int)kvh;
            p.first = (take(upto) - 1 - (int)(number - before)) * ROWS;   // its tiles end at `upto`: the first of them is the sequence's last
            p.rows = min(ROWS, s.n * a.group - p.first);
            const int seen = s.T - s.n + (p.first + p.rows - 1) / a.group + 1;
            p.steps = p.s1 = seen > 0 ? (seen + STEP - 1) / STEP : 0;
            p.s0 = 0;
            p.begin = p.end = 0;
            work(s, p, true, 0u);
            return;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
}

// Many rows: NW wavefronts of 32 rows each, keys through LDS in tiles of 64, one barrier per tile, STAGES buffers of which all but one are under way.
// 16384 queries, 32/8 heads: 2015 to 2180 us from card to card, 1.01 to 1.09 PFLOP/s at a clock that power holds at 1.8 GHz; matrix units busy 54 % of the cycles, vector units 46 %, LDS 28 %: a
// wavefront's products and its softmax follow one another, and two wavefronts on a SIMD hide only part of one behind the other (products alone take
// 1460 us, the vector instructions alone 1210).  Four wavefronts of 64 rows, halves of the wavefronts a phase apart, products and softmax of two tiles interleaved, priorities: 2190 to 2800.
constexpr int kTileKeys = 64, kTileLeast = 1024;
template <int D, int NW, int STAGES, bool CUT>
__global__ __launch_bounds__(64 * NW, 2) void prompt_attn_tile_kernel(PromptArgs a)
{
    constexpr int ROWS = 32 * NW, KEYS = kTileKeys, KT = KEYS / 32;
    constexpr int ROW = Tile<D>::ROW, CHUNKS = Tile<D>::CHUNKS, TILE = KEYS * ROW;
    constexpr int PER = 1024 / ROW;                  // rows of a transfer
    constexpr int TRANSFERS = TILE / 1024 / NW;      // of a wavefront, K and V each
    static_assert(TRANSFERS >= 1, "");
    extern __shared__ float4v smem4[];
    __shared__ uint32_t bad_sh[2];   // mark() of a step with such values; never cleared: one that lies there by chance costs time only
    auto mark = [](int step) { return 0x9E3779B1u * (uint32_t)(step + 1); };
    uint8_t *const lds = reinterpret_cast<uint8_t *>(smem4);   // STAGES times K, V
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, c = lane & 31;
    const uint32_t kfrag = Tile<D>::k_place(c, h), vfrag = v_fragment<D>(lane);
    const int trow = lane / CHUNKS, tchunk = lane % CHUNKS;
    const uint32_t stride = (uint32_t)a.Hkv * ROW;
    uint32_t k_lane[TRANSFERS], v_lane[TRANSFERS];
#pragma unroll
    for (int i = 0; i < TRANSFERS; ++i) {
        const int row = (wave * TRANSFERS + i) * PER + trow;
        k_lane[i] = trow * stride + (Tile<D>::k_chunk(row, tchunk) << 4);
        v_lane[i] = trow * stride + (Tile<D>::v_chunk(row, tchunk) << 4);
    }

    auto work = [&](const Sequence &s, const Piece &p, bool whole, unsigned slot) {
        const uint8_t *const k_src = reinterpret_cast<const uint8_t *>(a.k) + ((size_t)s.k0 * a.Hkv + p.kvh) * ROW;
        const uint8_t *const v_src = reinterpret_cast<const uint8_t *>(a.v) + ((size_t)s.k0 * a.Hkv + p.kvh) * ROW;
        auto stage = [&](int step) { return lds + (step & (STAGES - 1)) * 2 * TILE; };
        // Transfer i of a wavefront brings PER rows; the descriptor ends with the sequence's last key: what lies behind it, whole tiles too, is not
        // read (it is masked wherever it could count).
        auto request = [&](int step) {
            const long long key0 = (long long)step * KEYS;
            const uint32_t bytes = (uint32_t)max(0ll, min((s.T - 1 - key0) * stride + ROW, 0x7FFFFFFFll));
            uint8_t *const tile = stage(step);
            const Stretch ks = stretch(k_src + (size_t)key0 * stride, bytes), vs = stretch(v_src + (size_t)key0 * stride, bytes);
#pragma unroll
            for (int i = 0; i < TRANSFERS; ++i) {
                const int t = wave * TRANSFERS + i;
                quad_to_lds(ks, tile + t * 1024, k_lane[i], (uint32_t)(t * PER) * stride);
                quad_to_lds(vs, tile + TILE + t * 1024, v_lane[i], (uint32_t)(t * PER) * stride);
            }
        };
        // What a row does not see may be anything, and 0 times it need not be 0: a step that is masked looks its values over first, each wavefront those that it
        // brought.  If there is one that is not finite, it joins the sums of the rows that see it and is cleared (looked for where the fragments are read, by every
        // wavefront, it took 24 prompts of 200 tokens, 32/8 heads 41 us).
        Rows<D> rows;
        rows.start(a, s, p, wave * 32 + c, h);
        if (p.s0 < p.s1) {
#pragma unroll
            for (int i = 0; i < STAGES - 1; ++i) request(p.s0 + i);
        }
        rows.arrive();
        // steps that every row of the workgroup sees whole: they and the others have loops of their own, without branches in them (outputs and scores
        // that two paths write to cost hundreds of registers in copies)
        const int all_see = s.T - s.n + p.first / a.group + 1, open = min(all_see / KEYS, p.s1);
        auto body = [&](int step, auto masked) {
            constexpr bool MASKED = decltype(masked)::value;
            uint8_t *const ktile = stage(step), *const vtile = ktile + TILE;
            // this tile has landed (those asked for after it need not have), and the one before it has been read
            if constexpr (MASKED) {
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * TRANSFERS * (STAGES - 2)) : "memory");
                if (__any(any_not_finite<TRANSFERS>(vtile + wave * TRANSFERS * 1024, lane))) bad_sh[step & 1] = mark(step);
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            } else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * TRANSFERS * (STAGES - 2)) : "memory");
            request(step + STAGES - 1);
            float16v sc[KT];
            half8v pb[2 * KT];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                half8v kf[D / 16];
                rows.read_keys(kf, ktile + kt * 32 * ROW, kfrag);
                rows.scores(sc[kt], kf);
            }
            rows.template softmax<KT, MASKED>(sc, pb, step * KEYS, a.scale_log2e, h);
            if constexpr (MASKED)
                if (bad_sh[step & 1] == mark(step)) {   // uniform over the workgroup
                    rows.template add_not_finite<KT>(vtile, step * KEYS, h);
                    __syncthreads();
                    clear_not_finite<TRANSFERS>(vtile + wave * TRANSFERS * 1024, lane);
                    __syncthreads();
                }
            rows.template values<KT>(pb, vtile, vfrag);
        };
        int step = p.s0;
        for (; step < open; ++step) body(step, std::false_type{});
        for (; step < p.s1; ++step) body(step, std::true_type{});
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is under way into the buffers behind this
        const float l = rows.l_run + __shfl_xor(rows.l_run, 32, 64);
        if (whole) {
            // through LDS, so that rows leave in pieces of 16 bytes next to each other
            constexpr int OUT_ROW = ROW + 16;   // rows lie 16 bytes apart from the banks of the last
            uint8_t *const own = lds + wave * 32 * OUT_ROW;
            const float inv = row_factor(a, s, p, wave * 32 + c, l);
            __syncthreads();   // every wavefront has left the last tile
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    half4v y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = (_Float16)(rows.o[dt][4 * g + e] * inv);
                    *reinterpret_cast<half4v *>(own + c * OUT_ROW + (32 * dt + 8 * g + 4 * h) * 2) = y;
                }
#pragma unroll
            for (int i = 0; i < 32 / PER; ++i) {
                const int r = i * PER + trow;
                if (wave * 32 + r < p.rows) *reinterpret_cast<half8v *>(row_of(a, s, p, wave * 32 + r, D) + 8 * tchunk) = read_chunk(own + r * OUT_ROW + 16 * tchunk);
            }
            return;
        }
        // a piece is read by another kernel: plain stores, whose lines the L2 puts together (written through, 32 bytes at a time, 128 KB took 20 us and more)
        float *const po = a.part_o + (size_t)slot * ROWS * D, *const pm = a.part_ml + (size_t)slot * ROWS * 2;
        const int row = wave * 32 + c;
        if (row < p.rows) {
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<float4v *>(po + row * D + 32 * dt + 8 * g + 4 * h) =
                        (float4v){rows.o[dt][4 * g], rows.o[dt][4 * g + 1], rows.o[dt][4 * g + 2], rows.o[dt][4 * g + 3]};
            if (h == 0) {
                pm[2 * row] = rows.m_run;
                pm[2 * row + 1] = l;
            }
        }
    };
    if constexpr (CUT) go_through<D, ROWS, KEYS, kTileLeast, 64 * NW, false>(a, tid, reinterpret_cast<float *>(lds), work);
    else take_one<D, ROWS, KEYS>(a, lane, work);
}

// Few rows (single tokens of a batch): 32 rows, and eight wavefronts that each take every eighth step of 32 keys.  A wavefront shares no K or V tile,
// so it brings them itself and meets the others only at the end of a piece: no barrier in the walk.  Bound by the cache where it is long (16 x 8192 keys, 8 heads of
// 128: 105 us, 5.1 TB/s), else by its chain: lengths, first tiles, meeting of the wavefronts, join (one of 8192 14 us, of 100 7.4; of first use 17.7 and 8).  More than 64 sequences cost every workgroup
// one trip to memory more for the lengths of each 64 (64 of 512 keys 33 us, 65 40, 256 116, 4096 1650, 5.3 TB/s).
template <int D>
__global__ __launch_bounds__(512) void prompt_attn_few_kernel(PromptArgs a)
{
    constexpr int ROWS = 32, KEYS = 32, NW = 8;
    constexpr int ROW = Tile<D>::ROW, CHUNKS = Tile<D>::CHUNKS, TILE = KEYS * ROW, PER = 1024 / ROW, TRANSFERS = TILE / 1024;
    constexpr int EX_ROW = D * 4 + 16, EX_WAVE = ROWS * EX_ROW;        // after the walk: outputs of a wavefront, rows 16 bytes apart from the banks of the last
    constexpr int STATE = NW * EX_WAVE;                                // [row][wavefront] (max, sum)
    constexpr int LDS = STATE + ROWS * NW * 8 > NW * 2 * TILE ? STATE + ROWS * NW * 8 : NW * 2 * TILE;
    extern __shared__ float4v smem4[];
    uint8_t *const lds = reinterpret_cast<uint8_t *>(smem4);
    static_assert(LDS <= 160 * 1024 - 64, "");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, c = lane & 31;
    const uint32_t kfrag = Tile<D>::k_place(c, h), vfrag = v_fragment<D>(lane);
    const int trow = lane / CHUNKS, tchunk = lane % CHUNKS;
    const uint32_t stride = (uint32_t)a.Hkv * ROW;
    uint8_t *const ktile = lds + wave * 2 * TILE, *const vtile = ktile + TILE;

    go_through<D, ROWS, KEYS, 512, 64 * NW, true>(a, tid, reinterpret_cast<float *>(lds), [&](const Sequence &s, const Piece &p, bool whole, unsigned slot) {
        const uint8_t *const k_src = reinterpret_cast<const uint8_t *>(a.k) + ((size_t)s.k0 * a.Hkv + p.kvh) * ROW;
        const uint8_t *const v_src = reinterpret_cast<const uint8_t *>(a.v) + ((size_t)s.k0 * a.Hkv + p.kvh) * ROW;
        // what lies behind the sequence's last key or behind the piece is not read (the former is masked wherever it could count)
        uint32_t k_lane[4], v_lane[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = i * PER + trow;
            k_lane[i] = trow * stride + (Tile<D>::k_chunk(row, tchunk) << 4);
            v_lane[i] = trow * stride + (Tile<D>::v_chunk(row, tchunk) << 4);
        }
        auto request = [&](int step, const uint8_t *src, uint8_t *tile, const uint32_t (&at)[4]) {
            const long long key0 = (long long)step * KEYS;
            const uint32_t bytes = step < p.s1 ? (uint32_t)min((s.T - 1 - key0) * stride + ROW, 0x7FFFFFFFll) : 0;
            const Stretch from = stretch(src + (size_t)key0 * stride, bytes);
#pragma unroll
            for (int i = 0; i < TRANSFERS; ++i) quad_to_lds(from, tile + i * 1024, at[i & 3], (uint32_t)(i * PER) * stride);
        };
        Rows<D> rows;
        rows.start(a, s, p, c, h);
        __builtin_amdgcn_sched_barrier(0);   // Q before K before V: the waits count on it
        int step = p.s0 + wave;
        request(step, k_src, ktile, k_lane);
        __builtin_amdgcn_sched_barrier(0);
        request(step, v_src, vtile, v_lane);
        __builtin_amdgcn_sched_barrier(0);
        rows.arrive();
        const int all_see = s.T - s.n + p.first / a.group + 1, open = min(all_see / KEYS, p.s1);
        auto body = [&](auto masked) {
            constexpr bool MASKED = decltype(masked)::value;
            const int next = step + NW, key0 = step * KEYS;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(TRANSFERS) : "memory");   // K of this step; its V is newer
            float16v sc[1];
            half8v pb[2];
            half8v kf[D / 16];
            rows.read_keys(kf, ktile, kfrag);
            rows.scores(sc[0], kf);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the K tile has been read
            request(next, k_src, ktile, k_lane);
            rows.template softmax<1, MASKED>(sc, pb, key0, a.scale_log2e, h);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(TRANSFERS) : "memory");   // V of this step; the next K is newer
            if constexpr (MASKED)
                if (__any(any_not_finite<TRANSFERS>(vtile, lane))) {
                    rows.template add_not_finite<1>(vtile, key0, h);
                    clear_not_finite<TRANSFERS>(vtile, lane);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
            rows.template values<1>(pb, vtile, vfrag);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the V tile has been read
            request(next, v_src, vtile, v_lane);
            step = next;
        };
        while (step < open) body(std::false_type{});
        while (step < p.s1) body(std::true_type{});
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is under way into the tiles behind this
        // the states of the wavefronts meet in LDS
        const float l_run = rows.l_run + __shfl_xor(rows.l_run, 32, 64);
        __syncthreads();   // every wavefront has left its tiles
        float *const state = reinterpret_cast<float *>(lds + STATE);
        if (c < p.rows && h == 0) {
            state[(c * NW + wave) * 2] = rows.m_run;
            state[(c * NW + wave) * 2 + 1] = l_run;
        }
        if (c < p.rows)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4v *>(lds + wave * EX_WAVE + c * EX_ROW + (32 * dt + 8 * g + 4 * h) * 4) =
                    (float4v){rows.o[dt][4 * g], rows.o[dt][4 * g + 1], rows.o[dt][4 * g + 2], rows.o[dt][4 * g + 3]};
        __syncthreads();
        const PartialBuffer po = Pieces<D, ROWS>::o(a, slot), pm = Pieces<D, ROWS>::ml(a, slot);
        for (int item = tid; item < p.rows * (D / 4); item += 64 * NW) {
            const int row = item / (D / 4), d4 = item % (D / 4);
            float m = kLowest, l = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) m = fmaxf(m, state[(row * NW + w) * 2]);
            float4v val = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float wgt = __builtin_amdgcn_exp2f(state[(row * NW + w) * 2] - m);
                l += wgt * state[(row * NW + w) * 2 + 1];
                val += wgt * *reinterpret_cast<const float4v *>(lds + w * EX_WAVE + row * EX_ROW + d4 * 16);
            }
            if (whole) store_row_quad(a, s, p, row, D, 4 * d4, val, l);
            else {
                store_partial(po, row * (D / 4) + d4, val);
                if (d4 == 0) {
                    store_partial_f32(pm, 2 * row, m);
                    store_partial_f32(pm, 2 * row + 1, l);
                }
            }
        }
    });
}
template <int D>
constexpr int few_lds() { return 8 * 32 * (D * 4 + 16) + 32 * 8 * 8 > 8 * 2 * 32 * D * 2 ? 8 * 32 * (D * 4 + 16) + 32 * 8 * 8 : 8 * 2 * 32 * D * 2; }

// ---- host ------------------------------------------------------------------------------------------------------
constexpr int kFewRows = 32;

struct PromptPlan {
    bool few, cut;
    int rows, grid, tiles;   // of a tile; workgroups; tiles at most
    size_t o_bytes, ml_bytes;
};

static int check_prompt_sizes(int rows, int B, int max_q, int max_k, int Hq, int Hkv, int D)
{
    if (rows < 1 || B < 1 || max_q < 1 || max_k < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || D < 1) return W4A16_EINVAL;
    if (D != 64 && D != 128) return W4A16_EUNSUP;
    if (B > kMostSequences || (long long)rows * Hq > (1 << 29) || rows > (1 << 23) || Hkv > 1024 || Hq / Hkv > 64 || max_q > (1 << 23) || max_k > (1 << 30))
        return W4A16_EUNSUP;
    return W4A16_OK;
}

static PromptPlan prompt_plan(int rows, int B, int max_q, int max_k, int Hq, int Hkv, int D)
{
    PromptPlan p;
    const int group = Hq / Hkv;
    auto tiles_of = [&](int height) { return ((long long)rows * group + (long long)(height - 1) * B) / height; };   // most of a KV head
    p.few = (long long)max_q * group <= 2 * kFewRows;
    p.rows = kFewRows;
    p.cut = true;
    if (!p.few) {
        // Whole tiles of 128 rows, two and more to a compute unit (D 128: a step of 64 keys takes 1.35 us alone, 1.65 with a neighbour, a round of many 2.15), or
        // of 256 where prompts are long and workgroups many and D is 128: 4096 queries, 32/8 heads 152 us (128 rows: 158), 16384 2095 (2121), but 16 x 1000, 16/16 heads
        // 135 (123), 8 prompts of up to 1500, 64/8 heads 155 (149); D 64, 4096 queries 103 (94), 24 prompts of 700, 28/4 heads 114 (92), of up to 700 26 (20).
        // Few tiles behind many keys are cut into equal stretches (40 us more for pieces written, read and joined) where that is shorter, were all sequences as
        // long as the longest; of several behind prefixes, which seldom are, 0.6 of that: the longest holds whole tiles up, equal stretches the sum.  32/8 heads:
        // 4 x 64 queries behind 2936 keys 48 us (whole 78), 2048 queries 89 (61), 8 single tokens over up to 8000 keys with a prompt of 1000 72 (205), 16 of them over up to
        // 4000 with a prompt of 512 67 to 80 (101 to 105).  The host does not see how uneven lengths are, so the choice is wrong where they are not what the factor takes
        // them for: 16 tokens over 4000 each with that prompt 118 cut, as they are, 108 whole; 8 x 100 behind up to 4000 104 whole, as they are, 76 cut (behind 2000 each 60
        // and 68), 32 tokens over up to 4000 with 256 queries behind 2744 121 whole, as they are, 103 cut.
        const long long steps = (max_k + 63) / 64, part = max_q >= max_k ? 1 : 2;   // a whole prompt's rows see half of its keys on average
        const long long high = tiles_of(256) * Hkv, low = tiles_of(128) * Hkv, of_size = D == 128 ? 100 : 62;
        const long long halves = steps * of_size * (low <= 256 ? 1350 : 1650) / 100, evenly = high * steps * part * of_size * 1075 / 256 / 100;
        const long long cut = (B > 1 && part == 2 ? evenly * 6 / 10 : evenly) + 40000;
        p.cut = low <= 512 && cut < halves;
        p.rows = p.cut || (D == 128 && high >= 512 && (long long)rows * group >= 16384ll * B) ? 256 : 128;
    }
    const long long tiles = tiles_of(p.rows);
    if (p.cut) {   // no more workgroups than there can be work for, were every sequence as long as the longest
        p.tiles = (int)min(tiles * Hkv, 65535ll);
        p.grid = (int)min(tiles * Hkv * (((long long)max_k + 255) / 256), (long long)kMostGroups);
        p.o_bytes = (size_t)p.grid * 2 * p.rows * D * 4;
        p.ml_bytes = (size_t)p.grid * 2 * p.rows * 8;
    } else {       // whole tiles, as take_one() deals them out
        p.grid = (int)(8 % Hkv == 0 ? (tiles + 8 / Hkv - 1) / (8 / Hkv) * 8 : tiles * Hkv);
        p.o_bytes = p.ml_bytes = 0;
        p.tiles = 0;
    }
    return p;
}

template <int WHICH, typename Kernel>
static int launch_with_lds(Kernel kernel, int lds, int threads, const PromptArgs &a, const PromptPlan &p, hipStream_t stream)
{
    static bool ready = false;   // the LDS size is granted once for each of them
    if (!ready) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return W4A16_EHIP;
        ready = true;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.grid), dim3(threads), lds, stream, a);
    return launch_status();
}
template <int D>
static int launch_prompt(const PromptArgs &a, const PromptPlan &p, hipStream_t stream)
{
    constexpr int stage = 2 * kTileKeys * D * 2;
    if (p.few) return launch_with_lds<D>(&prompt_attn_few_kernel<D>, few_lds<D>(), 512, a, p, stream);
    if (p.cut) {
        const int rc = launch_with_lds<D + 1>(&prompt_attn_tile_kernel<D, 8, 4, true>, 4 * stage, 512, a, p, stream);
        if (rc != W4A16_OK) return rc;
        hipLaunchKernelGGL((prompt_attn_join_kernel<D, 256, kTileKeys, kTileLeast>), dim3(256 / kJoinRows, (unsigned)p.tiles), dim3(256), 0, stream, a, (unsigned)p.grid);
        return launch_status();
    }
    if constexpr (D == 128)
        if (p.rows == 256) return launch_with_lds<D + 3>(&prompt_attn_tile_kernel<D, 8, 4, false>, 4 * stage, 512, a, p, stream);
    return launch_with_lds<D + 2>(&prompt_attn_tile_kernel<D, 4, 2, false>, 2 * stage, 256, a, p, stream);
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

int w4a16_prompt_attn_plan_describe(int rows, int B, int max_q, int max_k, int Hq, int Hkv, int D, int *out)
{
    if (!out) return W4A16_ENULL;
    const int rc = check_prompt_sizes(rows, B, max_q, max_k, Hq, Hkv, D);
    if (rc != W4A16_OK) return rc;
    const PromptPlan p = prompt_plan(rows, B, max_q, max_k, Hq, Hkv, D);
    out[0] = p.few ? 0 : p.cut ? 2 : 1;
    out[1] = p.rows;
    out[2] = p.grid;
    return W4A16_OK;
}

int w4a16_prompt_attn(const void *q, const void *k, const void *v, const int32_t *q_start, const int32_t *k_start, const int32_t *k_len, void *out, int B,
                      int rows, int k_rows, int max_q, int max_k, int Hq, int Hkv, int D, float scale, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_prompt_sizes(rows, B, max_q, max_k, Hq, Hkv, D);
    if (rc != W4A16_OK) return rc;
    if (k_rows < 1 || !(scale > 0.f) || !(scale < __builtin_inff())) return W4A16_EINVAL;
    if (scale > kMostScale) return W4A16_EUNSUP;
    if (!q || !k || !v || !q_start || !out || (k_start == nullptr) != (k_len == nullptr)) return W4A16_ENULL;
    if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) ||
        ((reinterpret_cast<uintptr_t>(q_start) | reinterpret_cast<uintptr_t>(k_start) | reinterpret_cast<uintptr_t>(k_len)) & 3u))
        return W4A16_EALIGN;
    const PromptPlan p = prompt_plan(rows, B, max_q, max_k, Hq, Hkv, D);
    if (!workspace || workspace_bytes < kTicketBytes + p.o_bytes + p.ml_bytes) return W4A16_EWORKSPACE;
    if (workspace_misaligned(workspace)) return W4A16_EALIGN;
    float *const part_o = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + kTicketBytes);
    const PromptArgs a = {(const _Float16 *)q, (const _Float16 *)k, (const _Float16 *)v, q_start, k_start, k_len, (_Float16 *)out, part_o,
                          part_o + p.o_bytes / 4, (uint32_t *)workspace, B, rows, k_rows, Hq, Hkv, Hq / Hkv, scale * 1.44269504088896340736f};
    return D == 128 ? launch_prompt<128>(a, p, (hipStream_t)stream) : launch_prompt<64>(a, p, (hipStream_t)stream);
}

}  // extern "C"
