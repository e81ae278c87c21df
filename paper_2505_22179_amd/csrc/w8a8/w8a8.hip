// W8A8 linear: quantisation of tokens, the product of int8 codes, packing.  Contracts in include/w8a8.h.
#include "../internal.h"
#include "../devscope.h"
#include "../shared_entries.inc"
#include "../../../include/w8a8.h"

namespace w4 {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t ushort2v __attribute__((ext_vector_type(2)));

constexpr int kMostK = 65536;       // 65536 * 128 * 127 < 2^31: no sum of products leaves 32 bits
constexpr int kMostTokens = 1 << 20;
__host__ __device__ inline int k_blocks(int K) { return (K + 127) / 128 * 2; }   // tiles of a row of tiles
// byte of codes (r, 16 chunk .. 16 chunk + 15)
__host__ __device__ inline size_t chunk_offset(int r, int chunk, int blocks)
{
    return ((size_t)(r >> 4) * blocks + (chunk >> 2)) * 1024 + (chunk & 3) * 256 + (r & 15) * 16;
}

// ---- packing -----------------------------------------------------------------------------------------------
// A thread moves 16 codes of a row; the sixteen rows of a tile lie in neighbouring threads, so the packed side is contiguous.
__global__ __launch_bounds__(256) void w8a8_pack_kernel(const int8_t *__restrict__ w, uint8_t *__restrict__ packed, int rows, int K, int blocks)
{
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;   // 16-byte place in the packed buffer
    const size_t tile = at >> 6;
    const int r = (int)(tile / blocks) * 16 + (int)(at & 15), chunk = (int)(tile % blocks) * 4 + (int)((at >> 4) & 3);
    if (r >= (rows + 15) / 16 * 16) return;
    u32x4 x = {};
    if (r < rows && chunk * 16 < K) x = *reinterpret_cast<const u32x4 *>(w + (size_t)r * K + chunk * 16);
    *reinterpret_cast<u32x4 *>(packed + at * 16) = x;
}
__global__ __launch_bounds__(256) void w8a8_unpack_kernel(const uint8_t *__restrict__ packed, int8_t *__restrict__ w, int rows, int K, int blocks)
{
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
    const int chunks = K / 16, r = (int)(at / chunks), chunk = (int)(at % chunks);
    if (r >= rows) return;
    *reinterpret_cast<u32x4 *>(w + (size_t)r * K + chunk * 16) = *reinterpret_cast<const u32x4 *>(packed + chunk_offset(r, chunk, blocks));
}

// ---- quantisation --------------------------------------------------------------------------------------------
// Nearest whole number to x / s, ties to even.  The product with the reciprocal is off by a rounding or two, so the number found may be a neighbour
// where the quotient lies next to a half: what is left, x - n s, is exact in fp32 (a multiple of the last place of s or of x, no larger than s),
// and tells.
__device__ __forceinline__ int nearest_code(float x, float s, float inv)
{
    float n = __builtin_rintf(x * inv);
    const float left = __builtin_fmaf(-n, s, x), half = 0.5f * s;
    const float over = __builtin_fabsf(left);
    if (over > half || (over == half && ((int)n & 1))) n += left > 0.f ? 1.f : -1.f;
    return (int)n;
}

// The codes of sixteen values.  x * inv is within 2^-16 of the quotient, so unless its fraction is as near to a half as that, rounding it gives the nearest
// whole number, by an addition that leaves it in the low byte (8192 tokens of 4096 behind a norm: 38 us with nearest_code() throughout, vector units full).
__device__ __forceinline__ u32x4 codes_of(const half8 (&v)[2], float s, float inv)
{
    constexpr float magic = 12582912.f;   // 1.5 * 2^23
    u32x4 packed;
    float nearest_half = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t m[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = (float)v[w >> 1][4 * (w & 1) + e], sum = __builtin_fmaf(x, inv, magic);
            nearest_half = fmaxf(nearest_half, __builtin_fabsf(__builtin_fmaf(x, inv, -(sum - magic))));
            m[e] = __builtin_bit_cast(uint32_t, sum);
        }
        packed[w] = __builtin_amdgcn_perm(m[1], m[0], 0x0C0C0400u) | __builtin_amdgcn_perm(m[3], m[2], 0x04000C0Cu);
    }
    if (nearest_half >= 0.5f - 0x1p-15f) {
        packed = (u32x4){0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) packed[2 * p + (e >> 2)] |= (uint32_t)(nearest_code((float)v[p][e], s, inv) & 0xFF) << (8 * (e & 3));
    }
    return packed;
}

// One token by the first T threads of a workgroup; a thread keeps PER chunks of sixteen values in registers: one pass over the input.
// 8192 tokens of 4096 as they are 23 us, behind a norm 30, of which the copy rate allows 20: vector units 75 % busy and two barriers a token.  777 gated ones of
// 14336 17, of which 11: `up` is asked for eight values at a time, behind the gate that it multiplies, a trip to memory each.
// store(chunk, codes) receives the chunks, those of the padding too (zeros).  Returns the scale (in the first T threads).  Two barriers, for all threads.
template <int PRE, int T, int PER, typename Store>
__device__ __forceinline__ float quantize_row(const _Float16 *__restrict__ row, const _Float16 *__restrict__ gamma, float eps, int K, int padded,
                                              int tid, float *sums, uint32_t *tops, Store store)
{
    const int chunks = K / 16;
    const bool works = tid < T;
    half8 v[PER][2];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int ch = tid + i * T;
        v[i][0] = v[i][1] = (half8)(_Float16)0;
        if (works && ch < chunks) {
            v[i][0] = *reinterpret_cast<const half8 *>(row + ch * 16);
            v[i][1] = *reinterpret_cast<const half8 *>(row + ch * 16 + 8);
        }
    }
    if constexpr (PRE == W8A8_SILU_MUL) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int ch = tid + i * T;
            if (works && ch < chunks) {
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const half8 up = *reinterpret_cast<const half8 *>(row + K + ch * 16 + 8 * p);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float g = (float)v[i][p][e];
                        v[i][p][e] = (_Float16)keep_f32(g * __builtin_amdgcn_rcpf(1.f + __expf(-g)) * (float)up[e]);   // the reciprocal is off by 2^-23 at most, and is rounded to 11 bits
                    }
                }
            }
        }
    } else if constexpr (PRE == W8A8_RMS_NORM) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = __builtin_fmaf((float)v[i][p][e], (float)v[i][p][e], ss);
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) ss += __shfl_xor(ss, off, 64);
        if (works && (tid & 63) == 0) sums[tid >> 6] = ss;
        __syncthreads();
        ss = 0.f;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) ss += sums[w];
        const float inv = 1.f / sqrtf(ss / (float)K + eps);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int ch = tid + i * T;
            if (works && ch < chunks) {
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const half8 g = *reinterpret_cast<const half8 *>(gamma + ch * 16 + 8 * p);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[i][p][e] = (_Float16)keep_f32((float)v[i][p][e] * inv * (float)g[e]);
                }
            }
        }
    }
    // magnitudes of fp16 numbers compare as their bits do, infinities and NaN above all others
    ushort2v tops_of = {0, 0};
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const u32x4 b = __builtin_bit_cast(u32x4, v[i][p]) & 0x7FFF7FFFu;
#pragma unroll
            for (int e = 0; e < 4; ++e) tops_of = __builtin_elementwise_max(tops_of, __builtin_bit_cast(ushort2v, (uint32_t)b[e]));
        }
    uint32_t top = max(tops_of[0], tops_of[1]);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, 64));
    if (works && (tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
    top = 0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) top = max(top, tops[w]);
    const bool finite = top < 0x7C00u, some = finite && top > 0;
    const float s = (float)__builtin_bit_cast(_Float16, (uint16_t)top) / 127.f;   // 0 for a row of zeros
    const float inv = some ? 1.f / s : 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int ch = tid + i * T;
        if (works && ch < padded) {
            u32x4 packed = {};
            if (some) packed = codes_of(v[i], s, inv);
            store(ch, packed);
        }
    }
    return finite ? s : __builtin_nanf("");
}

template <int PRE, int T, int PER>
__global__ __launch_bounds__(T) void w8a8_quantize_kernel(const _Float16 *__restrict__ x, const _Float16 *__restrict__ gamma, float eps,
                                                          uint8_t *__restrict__ codes, float *__restrict__ scale, int M, int K, int blocks)
{
    __shared__ float sums[T / 64];
    __shared__ uint32_t tops[T / 64];
    // The sixteen tokens of a tile share the cache lines of its codes: workgroups go to the eight XCDs in turn, and a tile's go to one, whose L2
    // puts the lines together (8192 tokens of 8192: 67 us in the order of launch, 34 like this)
    const int m = (int)(((blockIdx.x >> 7) * 8 + (blockIdx.x & 7)) * 16 + ((blockIdx.x >> 3) & 15));
    if (m >= M) return;
    const float s = quantize_row<PRE, T, PER>(x + (size_t)m * K * (PRE == W8A8_SILU_MUL ? 2 : 1), gamma, eps, K, blocks * 4, threadIdx.x, sums, tops,
                                              [&](int chunk, u32x4 packed) { *reinterpret_cast<u32x4 *>(codes + chunk_offset(m, chunk, blocks)) = packed; });
    if (threadIdx.x == 0) scale[m] = s;
}

// ---- products ------------------------------------------------------------------------------------------------
struct GemmArgs {
    const uint8_t *codes, *packed;
    const float *scale, *w_scale;
    const _Float16 *residual;
    _Float16 *y;
    float *partials;
    uint32_t *tickets;
    int M, N, blocks, splits;
    // of a kernel that quantises by itself
    const _Float16 *x, *gamma;
    float eps;
    int K;
};

// sums of channels n .. n + 3 of token m become outputs
__device__ __forceinline__ void finish(const GemmArgs &a, const float *scale, int4v acc, int m, int n)
{
    if (m >= a.M || n >= a.N) return;   // N is a multiple of eight: four channels are all there or none
    const float s = scale[m];
    const float4v t = *reinterpret_cast<const float4v *>(a.w_scale + n);
    const size_t at = (size_t)m * a.N + n;
    half4 r = {}, y;
    if (a.residual) r = *reinterpret_cast<const half4 *>(a.residual + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (_Float16)((float)acc[e] * s * t[e] + (float)r[e]);
    *reinterpret_cast<half4 *>(a.y + at) = y;
}

// More than 16 tokens: a workgroup of WM x WN wavefronts takes 16 MT WM tokens by 16 NT WN channels, a wavefront MT x NT tiles of them, in steps of 128
// values of k.  The activations, which WN wavefronts read, go through LDS (three buffers: two steps under way); the weights go straight to
// registers, AHEAD steps ahead: with both operands in LDS its bandwidth was as scarce as the matrix pipe (256 x 256: 2048 clocks a step each).  Tiles lie in
// operand order already, so a load or transfer is 1 KB in one piece and fragments are read without bank conflicts.
// Where the tiles are few, `splits` workgroups share the walk along k; the last of them to finish adds the others' sums (whole numbers: in any order)
// to its own.
template <int WM, int WN, int MT, int NT, int AHEAD>
__global__ __launch_bounds__(64 * WM * WN) void w8a8_tile_kernel(GemmArgs a)
{
    constexpr int XT = WM * MT, WT = WN * NT, WAVES = WM * WN, STAGE = XT * 2048, TRANSFERS = (XT * 2 + WAVES - 1) / WAVES, STAGES = 3;
    constexpr int RING = AHEAD + 1, UNROLL = RING % 2 ? 2 * RING : RING;   // in halves of a step
    extern __shared__ u32x4 smem[];
    uint8_t *const lds = reinterpret_cast<uint8_t *>(smem);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int x_tiles = (a.M + 15) / 16, w_tiles = (a.N + 15) / 16;
    // An XCD gets neighbouring places; bands of eight blocks of tokens, so that workgroups that run together share both operands.
    const unsigned xcd = blockIdx.x & 7u, grid = gridDim.x;
    const unsigned number = xcd * (grid >> 3) + min(xcd, grid & 7u) + (blockIdx.x >> 3);
    const unsigned split = number % (unsigned)a.splits, place = number / (unsigned)a.splits;
    const unsigned rows = (unsigned)(x_tiles + XT - 1) / XT, cols = (unsigned)(w_tiles + WT - 1) / WT;
    const unsigned band = place / (8 * cols), in_band = place - band * 8 * cols, high = min(8u, rows - 8 * band);
    const int bm = (int)(8 * band + in_band % high), bn = (int)(in_band / high);
    const int all = a.blocks / 2, first = (int)((long long)all * split / a.splits), steps = (int)((long long)all * (split + 1) / a.splits) - first;

    const uint8_t *xs[TRANSFERS];
#pragma unroll
    for (int i = 0; i < TRANSFERS; ++i)
        xs[i] = a.codes + ((size_t)min(bm * XT + (wave * TRANSFERS + i) / 2, x_tiles - 1) * a.blocks + 2 * first + (wave * TRANSFERS + i) % 2) * 1024;
    auto transfer = [&](int step, int i) {
        if (XT * 2 % WAVES == 0 || wave * TRANSFERS + i < XT * 2)   // uniform; what is asked for behind the last step is not there, so no load needs a branch
            quad_to_lds(stretch(xs[i], 2048 * steps - 1024), lds + step % STAGES * STAGE + (wave * TRANSFERS + i) * 1024, lane * 16, step * 2048);
    };
    Stretch ws[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
        ws[j] = stretch(a.packed + ((size_t)min(bn * WT + wn * NT + j, w_tiles - 1) * a.blocks + 2 * first) * 1024, 2048 * steps);
    int4v wf[RING][NT];
    auto fetch = [&](int half, int j) {
        return __builtin_bit_cast(int4v, __builtin_amdgcn_raw_buffer_load_b128(ws[j], lane * 16, half * 1024, WM == 1 ? kStreamed : 0));
    };
    int4v acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = (int4v){0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < TRANSFERS; ++i) transfer(s, i);
    __builtin_amdgcn_sched_barrier(0);   // the waits below count on this order
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int j = 0; j < NT; ++j) wf[u][j] = fetch(u, j);
    auto body = [&](int u, int step, auto last) __attribute__((always_inline)) {
        // This step's activations have landed and the step before this one has been read.  Newer than they are the next step's activations and the
        // weights asked for in three halves; those that the last steps would ask for the compiler leaves out.
        constexpr int NEWER = TRANSFERS + (decltype(last)::value ? 0 : NT * (AHEAD > 2 ? 3 : AHEAD));
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(NEWER) : "memory");
        const uint8_t *const stage = lds + step % STAGES * STAGE;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            int4v xf[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) xf[i] = *reinterpret_cast<const int4v *>(stage + ((wm * MT + i) * 2 + half) * 1024 + lane * 16);
            // Loads go out between the products: a compute unit takes 64 bytes a clock, and a wavefront that asks for all at once stands still meanwhile.
            // Activations first (the wait above counts on it).
            constexpr int HERE = (TRANSFERS + 1) / 2, LOADS = HERE + NT, GAP = MT * NT / LOADS > 0 ? MT * NT / LOADS : 1;
            auto load = [&](int n) {
                if (n < HERE) {
                    if (half * HERE + n < TRANSFERS) transfer(step + 2, half * HERE + n);
                } else if (n < LOADS) wf[(u + half + AHEAD) % RING][n - HERE] = fetch(2 * step + half + AHEAD, n - HERE);
                __builtin_amdgcn_sched_barrier(0);
            };
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const int at = i * NT + j;
                    if (at % GAP == 0 && at / GAP < LOADS) load(at / GAP);
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[(u + half) % RING][j], xf[i], acc[i][j], 0, 0, 0);
                }
#pragma unroll
            for (int n = (MT * NT + GAP - 1) / GAP; n < LOADS; ++n) load(n);
        }
    };
    int step0 = 0;
    for (; step0 + UNROLL / 2 <= steps; step0 += UNROLL / 2)
#pragma unroll
        for (int u = 0; u < UNROLL; u += 2) body(u, step0 + u / 2, std::false_type{});
#pragma unroll
    for (int u = 0; u < UNROLL - 2; u += 2) {
        if (step0 + u / 2 >= steps) break;   // uniform
        body(u, step0 + u / 2, std::true_type{});
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is under way into LDS behind this
    if (a.splits > 1) {
        constexpr int QUADS = WAVES * MT * NT * 64;   // of a workgroup's sums
        const PartialBuffer mine = partial_buffer(a.partials + ((size_t)place * a.splits + split) * QUADS * 4);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) store_partial(mine, ((wave * MT + i) * NT + j) * 64 + lane, __builtin_bit_cast(float4v, acc[i][j]));
        uint32_t *const ticket_sh = reinterpret_cast<uint32_t *>(lds);   // exchange as in the linears of 4 bits
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) *ticket_sh = __hip_atomic_fetch_add(&a.tickets[place], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (*ticket_sh != (uint32_t)(a.splits - 1)) return;
        if (threadIdx.x == 0) __hip_atomic_store(&a.tickets[place], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        for (unsigned s = 0; s < (unsigned)a.splits; ++s) {
            if (s == split) continue;
            const PartialBuffer other = partial_buffer(a.partials + ((size_t)place * a.splits + s) * QUADS * 4);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] += __builtin_bit_cast(int4v, load_partial(other, ((wave * MT + i) * NT + j) * 64 + lane));
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            finish(a, a.scale, acc[i][j], (bm * XT + wm * MT + i) * 16 + (lane & 15), (bn * WT + wn * NT + j) * 16 + 4 * (lane >> 4));
}

// Few tokens, bound by the weights: eight wavefronts share TW tiles of channels and take every eighth tile of k; weights go straight to registers.
// One tile of channels: AHEAD tiles of k are always under way, each asked for as soon as its registers are free (one token 14336 -> 4096 11.3 us, asked for
// four at a time 12.6: 5.2 TB/s; 28672 -> 8192 39.4, 43).  Two, of which fewer workgroups come to a compute unit: four at a time (60 tokens 8192 -> 8192
// 17.2, always under way 19.7).
// FUSED: one token of up to kFusedK values, quantised by every workgroup for itself into LDS while its first weights are on the way: a launch less, in the
// other kernel's arrangement and so with its bits.  A normed token 4096 -> 28672 25.1 -> 21.8 us, 4096 -> 6144 10.9 -> 8.0.  Longer rows or more
// tokens cost every workgroup more than the launch: 8192 -> 57344 82 -> 84, two tokens 4096 -> 28672 25 -> 29.
constexpr int kFusedK = 4096;
template <int MT, int TW, int PRE = W8A8_PLAIN, bool FUSED = false>
__global__ __launch_bounds__(512) void w8a8_stream_kernel(GemmArgs a)
{
    constexpr int AHEAD = 4;
    __shared__ int4v sums[8][MT * TW][64];
    __shared__ u32x4 row_codes[FUSED ? kFusedK / 16 : 1];
    __shared__ float row_scale, norm_sums[4];
    __shared__ uint32_t tops[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int x_tiles = (a.M + 15) / 16, w_tiles = (a.N + 15) / 16, tile0 = blockIdx.x * TW;
    int4v acc[MT][TW];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < TW; ++j) acc[i][j] = (int4v){0, 0, 0, 0};
    Stretch xs[MT], ws[TW];   // a row of tiles each: what is asked for behind its end is zero, and adds nothing
#pragma unroll
    for (int i = 0; i < MT; ++i) xs[i] = stretch(a.codes + (size_t)min(i, x_tiles - 1) * a.blocks * 1024, a.blocks * 1024);
#pragma unroll
    for (int j = 0; j < TW; ++j) ws[j] = stretch(a.packed + (size_t)min(tile0 + j, w_tiles - 1) * a.blocks * 1024, a.blocks * 1024);
    int4v wf[AHEAD][TW], xf[AHEAD][MT];
    auto load = [&](int u, int at) {
#pragma unroll
        for (int j = 0; j < TW; ++j) wf[u][j] = __builtin_bit_cast(int4v, __builtin_amdgcn_raw_buffer_load_b128(ws[j], at * 1024 + lane * 16, 0, kStreamed));
        if constexpr (!FUSED)
#pragma unroll
            for (int i = 0; i < MT; ++i) xf[u][i] = __builtin_bit_cast(int4v, __builtin_amdgcn_raw_buffer_load_b128(xs[i], at * 1024 + lane * 16, 0, 0));
    };
    if constexpr (TW == 1)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load(u, wave + 8 * u);
    if constexpr (FUSED) {
        __builtin_amdgcn_sched_barrier(0);
        const float s = quantize_row<PRE, 256, 1>(a.x, a.gamma, a.eps, a.K, a.blocks * 4, threadIdx.x, norm_sums, tops,
                                                  [&](int chunk, u32x4 packed) { row_codes[chunk] = packed; });
        if (threadIdx.x == 0) row_scale = s;
        __syncthreads();
    }
    auto add = [&](int u, int at) {
        if constexpr (FUSED) xf[u][0] = __builtin_bit_cast(int4v, row_codes[min(at, a.blocks - 1) * 4 + (lane >> 4)]);   // the token's, for all sixteen rows
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < TW; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[u][j], xf[u][i], acc[i][j], 0, 0, 0);
    };
    int b = wave;
    if constexpr (TW == 1) {
        for (; b + 8 * AHEAD < a.blocks; b += 8 * AHEAD) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                add(u, b + 8 * u);
                load(u, b + 8 * (u + AHEAD));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) add(u, b + 8 * u);
    } else {
        for (; b < a.blocks; b += 8 * AHEAD) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) load(u, b + 8 * u);
            if constexpr (MT == 2) __builtin_amdgcn_sched_barrier(0);   // left to itself the compiler puts the loads next to their products: 32 tokens 4096 -> 6144 7.5 us, 8.4
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) add(u, b + 8 * u);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < TW; ++j) sums[wave][i * TW + j][lane] = acc[i][j];
    __syncthreads();
    for (int t = wave; t < MT * TW; t += 8) {
        int4v all = sums[0][t][lane];
#pragma unroll
        for (int w = 1; w < 8; ++w) all += sums[w][t][lane];
        finish(a, FUSED ? &row_scale : a.scale, all, t / TW * 16 + (lane & 15), (tile0 + t % TW) * 16 + 4 * (lane >> 4));
    }
}

// ---- host ------------------------------------------------------------------------------------------------------
static int check_codes_shape(int rows, int K)
{
    if (rows < 1 || K < 1 || K % 16 != 0) return W4A16_EINVAL;
    if (K > kMostK || rows > (1 << 24)) return W4A16_EUNSUP;
    return W4A16_OK;
}
static size_t codes_bytes(int rows, int K) { return (size_t)((rows + 15) / 16) * k_blocks(K) * 1024; }
static int check_gemm_shape(int M, int N, int K)
{
    if (M < 1 || N < 1 || K < 1 || K % 16 != 0 || N % 8 != 0) return W4A16_EINVAL;
    if (K > kMostK || N > (1 << 20) || M > kMostTokens) return W4A16_EUNSUP;
    return W4A16_OK;
}
static size_t aligned256(size_t n) { return (n + 255) / 256 * 256; }

static int check_quantize(const void *x, int pre, const void *gamma, float eps, int K)
{
    if (pre < W8A8_PLAIN || pre > W8A8_SILU_MUL) return W4A16_EINVAL;
    if (!x) return W4A16_ENULL;
    if (pre == W8A8_RMS_NORM) {
        if (!gamma) return W4A16_ENULL;
        if (!(eps >= 0.f)) return W4A16_EINVAL;
    } else if (gamma) return W4A16_EINVAL;
    if (misaligned(x) || misaligned(gamma)) return W4A16_EALIGN;
    return W4A16_OK;
}

static int launch_quantize(const void *x, int pre, const void *gamma, float eps, void *codes, float *scale, int M, int K, hipStream_t stream)
{
    const int blocks = k_blocks(K), chunks = blocks * 4;
    const unsigned grid = M <= 16 ? 1u + 8u * (unsigned)(M - 1) : ((unsigned)M + 127u) / 128u * 128u;   // one tile: its tokens are those at 8 m
#define W8_QUANTIZE(P_, T_, N_)                                                                                                                 \
    hipLaunchKernelGGL((w8a8_quantize_kernel<P_, T_, N_>), dim3(grid), dim3(T_), 0, stream, (const _Float16 *)x, (const _Float16 *)gamma, eps, \
                       (uint8_t *)codes, scale, M, K, blocks)
    // A thread per sixteen values, so that a row is one trip to memory, up to 16384 values; of more rows than there is room for workgroups of 1024 threads, two each,
    // whose barriers hold up fewer (4096 rows of 14336 behind a norm 46 us, of 1024 threads 69; 256 rows 7.5, 7.0)
#define W8_QUANTIZE_PRE(P_)                                        \
    do {                                                           \
        if (chunks <= 256) W8_QUANTIZE(P_, 256, 1);                \
        else if (chunks <= 512) W8_QUANTIZE(P_, 512, 1);           \
        else if (chunks <= 1024 && M > 512) W8_QUANTIZE(P_, 512, 2); \
        else if (chunks <= 1024) W8_QUANTIZE(P_, 1024, 1);         \
        else if (chunks <= 2048) W8_QUANTIZE(P_, 1024, 2);         \
        else W8_QUANTIZE(P_, 1024, 4);                             \
    } while (0)
    if (pre == W8A8_PLAIN) W8_QUANTIZE_PRE(W8A8_PLAIN);
    else if (pre == W8A8_RMS_NORM) W8_QUANTIZE_PRE(W8A8_RMS_NORM);
    else W8_QUANTIZE_PRE(W8A8_SILU_MUL);
#undef W8_QUANTIZE_PRE
#undef W8_QUANTIZE
    return launch_status();
}

// How a product is cut: the kernel, its tile and the number of workgroups that share a tile's walk along k.
struct GemmPlan {
    int kind, rows, cols, splits;
};

template <int WM, int WN, int MT, int NT, int AHEAD>
static int launch_tile(GemmArgs a, const GemmPlan &p, hipStream_t stream)
{
    constexpr int lds = WM * MT * 2048 * 3;
    static bool ready = false;   // the LDS size is granted once
    if (!ready) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(&w8a8_tile_kernel<WM, WN, MT, NT, AHEAD>), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
            return W4A16_EHIP;
        ready = true;
    }
    a.splits = p.splits;
    const unsigned grid = (unsigned)((a.M + p.rows - 1) / p.rows) * (unsigned)((a.N + p.cols - 1) / p.cols) * (unsigned)p.splits;
    hipLaunchKernelGGL((w8a8_tile_kernel<WM, WN, MT, NT, AHEAD>), dim3(grid), dim3(64 * WM * WN), lds, stream, a);
    return launch_status();
}

// The kernels, by measurement over 28 shapes (M 1 .. 4096, N 1024 .. 28672, K 4096 .. 14336), us:
//   up to 16 tokens, and up to 64 where k is short, the stream kernel: 60 tokens 4096 -> 4096 7.1 (tiles of 64 x 128, walk shared by four, 10.6), 8192 -> 8192 16.8
//   (20.6); with many channels or a long k its wavefronts' own copies of the activations cost more than an exchange: 60 tokens 4096 -> 28672 30.1 (21.7),
//   14336 -> 4096 20.0 (18.4).  Two tiles of channels to a wavefront where that still fills the chip: 60 tokens 8192 -> 8192 23.8 with one
//   up to 128 tokens tiles of 64 x 128 with a shared walk unless 128 x 128 fill the chip: 100 tokens 4096 -> 4096 11.3 (16.5), 128 tokens 4096 -> 28672 35.9 (33.8)
//   more: of 256 x 256, 128 x 256 and 128 x 128 the one that takes the shortest time by its rounds over 256 compute units, a step of 128 values of k in
//   1.64, 0.91 and 0.5 us and 4 us to begin and end a round: 4096 tokens 4096 -> 4096 61, 77 and 84; 777 tokens 8192 -> 8192 85, 59 and 69; 1024 tokens
//   4096 -> 4096 -, 33 and 22
enum { kStream = 0, kTile64x128, kTile128x128, kTile128x256, kTile256x256 };

static GemmPlan gemm_plan(int M, int N, int K)
{
    const long long steps = k_blocks(K) / 2;
    auto tiles = [&](int rows, int cols) { return (long long)((M + rows - 1) / rows) * ((N + cols - 1) / cols); };
    auto shared = [&](int kind, int rows, int cols) {   // the walks shared by as many workgroups as fill the chip, four steps each at least
        const long long n = tiles(rows, cols);
        return GemmPlan{kind, rows, cols, n < 256 ? (int)max(1ll, min(min(256 / n, steps / 4), 16ll)) : 1};
    };
    if (M <= 16 || (M <= 64 && K <= 8192 && tiles(64, 128) < 192)) return {kStream, 16 * (M <= 16 ? 1 : M <= 32 ? 2 : 4), M > 16 && N >= 6144 ? 32 : 16, 1};
    if (M <= 64 || (M <= 128 && tiles(128, 128) < 160)) return shared(kTile64x128, 64, 128);
    const GemmPlan whole[3] = {{kTile256x256, 256, 256, 1}, {kTile128x256, 128, 256, 1}, {kTile128x128, 128, 128, 1}};
    const int step_ns[3] = {1640, 910, 500}, round_ns = 4000;
    GemmPlan best = shared(kTile128x128, 128, 128);
    long long least = best.splits > 1 ? (steps + best.splits - 1) / best.splits * step_ns[2] + round_ns + 6000 : 1ll << 62;   // the exchange takes 6 us
    for (int i = 0; i < 3; ++i) {
        const long long ns = (tiles(whole[i].rows, whole[i].cols) + 255) / 256 * (steps * step_ns[i] + round_ns);
        if (ns < least) least = ns, best = whole[i];
    }
    return best;
}

// of any number of tokens up to M: tiles times splits are 256 at most where a walk is split
static size_t most_partials(int M) { return M <= 16 ? 0 : (size_t)256 * 4 * (M <= 64 ? 64 * 128 : 128 * 128); }

static int launch_gemm(const GemmArgs &a, const GemmPlan &p, hipStream_t stream)
{
#define W8_STREAM(MT_, TW_) \
    hipLaunchKernelGGL((w8a8_stream_kernel<MT_, TW_>), dim3((unsigned)((a.N + 16 * TW_ - 1) / (16 * TW_))), dim3(512), 0, stream, a)
    switch (p.kind) {
    case kStream:
        if (p.rows == 16) W8_STREAM(1, 1);
        else if (p.rows == 32) {
            if (p.cols == 16) W8_STREAM(2, 1);
            else W8_STREAM(2, 2);
        } else if (p.cols == 16) W8_STREAM(4, 1);
        else W8_STREAM(4, 2);
        return launch_status();
    case kTile64x128: return launch_tile<1, 8, 4, 1, 13>(a, p, stream);
    case kTile128x128: return launch_tile<2, 4, 4, 2, 7>(a, p, stream);
    case kTile128x256: return launch_tile<1, 8, 8, 2, 7>(a, p, stream);
    default: return launch_tile<2, 4, 8, 4, 2>(a, p, stream);
    }
#undef W8_STREAM
}

static int check_gemm(const void *packed, const float *w_scale, const void *residual, const void *y)
{
    if (!packed || !w_scale || !y) return W4A16_ENULL;
    if (misaligned(packed) || misaligned(w_scale) || misaligned(residual) || misaligned(y)) return W4A16_EALIGN;
    return W4A16_OK;
}

}  // namespace w4

using namespace w4;

extern "C" {

size_t w8a8_packed_bytes(int rows, int K) { return check_codes_shape(rows, K) == W4A16_OK ? codes_bytes(rows, K) : 0; }

int w8a8_pack(const int8_t *w, void *packed, int rows, int K, void *stream)
{
    const int rc = check_codes_shape(rows, K);
    if (rc != W4A16_OK) return rc;
    if (!w || !packed) return W4A16_ENULL;
    if (misaligned(w) || misaligned(packed)) return W4A16_EALIGN;
    const size_t groups = (codes_bytes(rows, K) / 16 + 255) / 256;
    if (groups >= (1u << 24)) return W4A16_EUNSUP;
    hipLaunchKernelGGL(w8a8_pack_kernel, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, w, (uint8_t *)packed, rows, K, k_blocks(K));
    return launch_status();
}

int w8a8_unpack(const void *packed, int8_t *w, int rows, int K, void *stream)
{
    const int rc = check_codes_shape(rows, K);
    if (rc != W4A16_OK) return rc;
    if (!w || !packed) return W4A16_ENULL;
    if (misaligned(w) || misaligned(packed)) return W4A16_EALIGN;
    const size_t groups = ((size_t)rows * (K / 16) + 255) / 256;
    if (groups >= (1u << 24)) return W4A16_EUNSUP;
    hipLaunchKernelGGL(w8a8_unpack_kernel, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, (const uint8_t *)packed, w, rows, K, k_blocks(K));
    return launch_status();
}

int w8a8_quantize(const void *x, int pre, const void *gamma, float eps, void *codes, float *scale, int M, int K, void *stream)
{
    int rc = check_codes_shape(M, K);
    if (rc != W4A16_OK) return rc;
    if (M > kMostTokens) return W4A16_EUNSUP;
    if (!codes || !scale) return W4A16_ENULL;
    rc = check_quantize(x, pre, gamma, eps, K);
    if (rc != W4A16_OK) return rc;
    if (misaligned(codes) || misaligned(scale)) return W4A16_EALIGN;
    return launch_quantize(x, pre, gamma, eps, codes, scale, M, K, (hipStream_t)stream);
}

size_t w8a8_workspace_bytes(int M, int N, int K)
{
    if (check_gemm_shape(M, N, K) != W4A16_OK) return 0;
    return kTicketBytes + codes_bytes(M, K) + aligned256((size_t)M * 4) + most_partials(M);
}

int w8a8_gemm_plan_describe(int M, int N, int K, int *out)
{
    if (!out) return W4A16_ENULL;
    const int rc = check_gemm_shape(M, N, K);
    if (rc != W4A16_OK) return rc;
    const GemmPlan p = gemm_plan(M, N, K);
    out[0] = p.kind != kStream;
    out[1] = p.rows;
    out[2] = p.cols;
    out[3] = p.splits;
    return W4A16_OK;
}

int w8a8_gemm(const void *codes, const float *scale, const void *packed, const float *w_scale, const void *residual, void *y, int M, int N, int K,
              void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_gemm_shape(M, N, K);
    if (rc != W4A16_OK) return rc;
    if (!codes || !scale) return W4A16_ENULL;
    rc = check_gemm(packed, w_scale, residual, y);
    if (rc != W4A16_OK) return rc;
    if (misaligned(codes) || misaligned(scale)) return W4A16_EALIGN;
    if (!workspace || workspace_bytes < w8a8_workspace_bytes(M, N, K)) return W4A16_EWORKSPACE;
    if (workspace_misaligned(workspace)) return W4A16_EALIGN;
    uint8_t *const partials = static_cast<uint8_t *>(workspace) + kTicketBytes + codes_bytes(M, K) + aligned256((size_t)M * 4);
    const GemmArgs a = {(const uint8_t *)codes, (const uint8_t *)packed, scale, w_scale, (const _Float16 *)residual, (_Float16 *)y,
                        (float *)partials, (uint32_t *)workspace, M, N, k_blocks(K), 1, nullptr, nullptr, 0.f, K};
    return launch_gemm(a, gemm_plan(M, N, K), (hipStream_t)stream);
}

int w8a8_linear(const void *x, int pre, const void *gamma, float eps, const void *packed, const float *w_scale, const void *residual, void *y, int M,
                int N, int K, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_gemm_shape(M, N, K);
    if (rc != W4A16_OK) return rc;
    rc = check_quantize(x, pre, gamma, eps, K);
    if (rc != W4A16_OK) return rc;
    rc = check_gemm(packed, w_scale, residual, y);
    if (rc != W4A16_OK) return rc;
    if (!workspace || workspace_bytes < w8a8_workspace_bytes(M, N, K)) return W4A16_EWORKSPACE;
    if (workspace_misaligned(workspace)) return W4A16_EALIGN;
    uint8_t *const codes = static_cast<uint8_t *>(workspace) + kTicketBytes;
    float *const scale = reinterpret_cast<float *>(codes + codes_bytes(M, K));
    const GemmArgs a = {codes, (const uint8_t *)packed, scale, w_scale, (const _Float16 *)residual, (_Float16 *)y,
                        reinterpret_cast<float *>(codes + codes_bytes(M, K) + aligned256((size_t)M * 4)), (uint32_t *)workspace, M, N, k_blocks(K), 1,
                        (const _Float16 *)x, (const _Float16 *)gamma, eps, K};
    // in place the token has to be read before the first output is written
    const uintptr_t x0 = (uintptr_t)x, y0 = (uintptr_t)y;
    const bool apart = x0 + (size_t)K * (pre == W8A8_SILU_MUL ? 4 : 2) <= y0 || y0 + (size_t)N * 2 <= x0;
    if (M == 1 && K <= kFusedK && apart) {
        auto *const kernel = pre == W8A8_PLAIN      ? &w8a8_stream_kernel<1, 1, W8A8_PLAIN, true>
                             : pre == W8A8_RMS_NORM ? &w8a8_stream_kernel<1, 1, W8A8_RMS_NORM, true>
                                                    : &w8a8_stream_kernel<1, 1, W8A8_SILU_MUL, true>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((N + 15) / 16)), dim3(512), 0, (hipStream_t)stream, a);
        return launch_status();
    }
    rc = launch_quantize(x, pre, gamma, eps, codes, scale, M, K, (hipStream_t)stream);
    return rc != W4A16_OK ? rc : launch_gemm(a, gemm_plan(M, N, K), (hipStream_t)stream);
}

}  // extern "C"
