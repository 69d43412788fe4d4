// A mixture-of-experts layer for a few tokens (T <= 64): router, selection, gated experts, weighted sum.
//
//   z = x Wg^T,  (idx, p) = top k,   h_j = p_j act(W1 x) * (W3 x),   y = residual + sum_j W2 h_j
//
// Every weight of every expert that some token picked is needed once and the arithmetic per weight is tiny: reading them is
// what bounds the layer, so the kernels stream weight rows from memory into the registers of the matrix instructions with as
// many loads in flight as fit, and tokens are the narrow operand.  Four launches:
//   router_kernel      scores of 16 experts over a slice of d, partial sums to the workspace
//   finalize (finalize.hip)  adds the slices, softmax and top-k: the selection is the predictor's, to the bit
//   up_kernel          one expert's 16 gate rows and the 16 rows beside them over all of d, for the tokens that picked it:
//                      the four waves split d.  h goes to the workspace, already weighed by p; in bf16 storage as two bf16
//                      parts, high and low (16 bits of it: a second rounding to 8 bits would cost the result as much as its own)
//   down_kernel        16 rows of d over all active experts: the eight waves split (expert, part of f); sums per token in LDS
// A fragment of 16 rows x 64 bytes is fetched with four neighbouring lanes on 64 contiguous bytes of a row, and a fixed lane
// permutation puts it into the operand layout (as in predict_decode.hip).
#include <type_traits>

#include "../../include/paep.h"

#include "paep_device.h"
#include "paep_internal.h"

namespace paep {

template <int V> using IC = std::integral_constant<int, V>;
template <int N, class F> __device__ __forceinline__ void static_for(F&& f)
{
    if constexpr (N > 0) {
        static_for<N - 1>(f);
        f(IC<N - 1>{});
    }
}

static constexpr int STEP = 64;                      // bytes of a row that one fragment covers
static constexpr int MOE_MAX_POS = PAEP_MOE_MAX_T * PAEP_MAX_K;

// A += W fragment x token fragment, both 16 rows x 64 bytes
template <bool BF16> __device__ __forceinline__ f32x4 product(const u32x4& w, const u32x4& x, f32x4 acc)
{
    if constexpr (BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i]), __uint_as_float(x[i]), acc, 0, 0, 0);
        return acc;
    }
}

// lane 4r + c's 16 bytes (row r, piece c) to lane r + 16c
__device__ __forceinline__ u32x4 to_operand(const u32x4& f, int lane)
{
    const int from = (4 * (lane & 15) + (lane >> 4)) * 4;
    return u32x4{(uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)f[0]), (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)f[1]),
                 (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)f[2]), (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)f[3])};
}

// 16 bytes at row + off, zeros where there are none (off past the row, or no such row)
__device__ __forceinline__ u32x4 piece(const unsigned char* row, int off, bool there)
{
    const u32x4 f = *(const u32x4*)(row + (there ? off : 0));
    u32x4 z;
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = there ? f[i] : 0u;
    return z;
}

// ---------------------------------------------------------------------------
// Router: partial[slice][t][e].  A workgroup per 16 experts and slice of d, its four waves a quarter of the slice each.
// ---------------------------------------------------------------------------
static constexpr int ROUTER_THREADS = 256, ROUTER_WAVE_STEPS = 4, ROUTER_STEPS = 4 * ROUTER_WAVE_STEPS;

template <bool BF16, int NT>
__global__ __launch_bounds__(ROUTER_THREADS) void router_kernel(int T, int E, int row_bytes, int tiles, const unsigned char* __restrict__ x,
                                                                const unsigned char* __restrict__ Wg, float* __restrict__ partial)
{
    __shared__ __attribute__((aligned(16))) f32x4 part[3][NT][64];
    const int tile = blockIdx.x % tiles, slice = blockIdx.x / tiles;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane >> 2, at = (slice * ROUTER_STEPS + wave * ROUTER_WAVE_STEPS) * STEP + (lane & 3) * 16;
    const int e = tile * 16 + row;
    u32x4 w[ROUTER_WAVE_STEPS], xf[NT][ROUTER_WAVE_STEPS];
#pragma unroll
    for (int u = 0; u < ROUTER_WAVE_STEPS; ++u) {
        const bool in = at + u * STEP < row_bytes;
        w[u] = piece(Wg + (long long)(e < E ? e : 0) * row_bytes, at + u * STEP, in && e < E);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int t = nt * 16 + row;
            xf[nt][u] = piece(x + (long long)(t < T ? t : 0) * row_bytes, at + u * STEP, in && t < T);
        }
    }
    f32x4 acc[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < ROUTER_WAVE_STEPS; ++u) {
        const u32x4 wo = to_operand(w[u], lane);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[nt] = product<BF16>(wo, to_operand(xf[nt][u], lane), acc[nt]);
    }
    if (wave > 0)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) part[wave - 1][nt][lane] = acc[nt];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int t = nt * 16 + (lane & 15), e0 = tile * 16 + (lane >> 4) * 4;
        f32x4 s = acc[nt];
#pragma unroll
        for (int v = 0; v < 3; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += part[v][nt][lane][i];
        if (t >= T) continue;
        float* dst = partial + ((long long)slice * T + t) * E + e0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e0 + i < E) dst[i] = s[i];
    }
}

// ---------------------------------------------------------------------------
// Who picked what, in LDS, by every workgroup for itself: the active experts in ascending order and, one after the other,
// their positions p = t * k + j (an id that stands in a row several times at its first place only; ids outside [0, E) nowhere).
// The order of one expert's positions differs from run to run; no result depends on it.
// ---------------------------------------------------------------------------
struct Lists {
    uint16_t expert[PAEP_MAX_E];                     // active experts
    uint16_t first[PAEP_MAX_E + 1];                  // where their positions begin
    uint16_t position[MOE_MAX_POS];
    int32_t count[PAEP_MAX_E];
    int n;
};

template <int THREADS> __device__ __forceinline__ void build_lists(Lists& ls, const int32_t* __restrict__ idx, int T, int k, int E)
{
    const int tid = threadIdx.x, n = T * k;
    for (int e = tid; e < E; e += THREADS) ls.count[e] = 0;
    __syncthreads();
    constexpr int MINE = (MOE_MAX_POS + THREADS - 1) / THREADS;
    int id[MINE], rank[MINE];
#pragma unroll
    for (int u = 0; u < MINE; ++u) {
        const int p = tid + u * THREADS;
        id[u] = -1;
        if (p >= n) continue;
        const int e = idx[p];
        bool first = (uint32_t)e < (uint32_t)E;
        for (int q = p / k * k; first && q < p; ++q) first = idx[q] != e;
        if (!first) continue;
        id[u] = e;
        rank[u] = atomicAdd(&ls.count[e], 1);
    }
    __syncthreads();
    if (tid < 64) {                                  // one wave: offsets of the experts, and those that are active
        int active = 0, before = 0;
        for (int e0 = 0; e0 < E; e0 += 64) {
            const int e = e0 + tid, c = e < E ? ls.count[e] : 0;
            int upto = c;
            for (int s = 1; s < 64; s <<= 1) {
                const int o = __shfl_up(upto, s, 64);
                if (tid >= s) upto += o;
            }
            const unsigned long long who = __ballot(c > 0);
            if (c > 0) {
                const int slot = active + __popcll(who & ((1ull << tid) - 1));
                ls.expert[slot] = (uint16_t)e;
                ls.first[slot] = (uint16_t)(before + upto - c);
                ls.count[e] = before + upto - c;     // from here on: where its positions begin
            }
            active += __popcll(who);
            before += __shfl(upto, 63, 64);
        }
        if (tid == 0) {
            ls.n = active;
            ls.first[active] = (uint16_t)before;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MINE; ++u)
        if (id[u] >= 0) ls.position[ls.count[id[u]] + rank[u]] = (uint16_t)(tid + u * THREADS);
    __syncthreads();
}

// what weighs position p: the sum over the places of its id in the row
__device__ __forceinline__ float position_weight(const int32_t* idx, const float* probs, int k, int p)
{
    const int t0 = p / k * k, e = idx[p];
    float w = 0.0f;
    for (int q = t0; q < t0 + k; ++q)
        if (idx[q] == e) w += probs[q];
    return w;
}

// ---------------------------------------------------------------------------
// h: [T * k][f], fp32, or the bf16 planes high and low one after the other
// ---------------------------------------------------------------------------
static constexpr int UP_THREADS = 256;

// NT: blocks of 16 tokens at a time
template <bool BF16, int NT>
__device__ __forceinline__ void up_tokens(const MoeArgs& a, const Lists& ls, int e, int list0, int tokens, int unit0,
                                          f32x4 (&part)[4][2][4][64], void* h)
{
    constexpr int U = NT == 1 ? 8 : NT == 2 ? 4 : 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row_bytes = a.d * (BF16 ? 2 : 4), nsteps = (row_bytes + STEP - 1) / STEP, quarter = (nsteps + 3) / 4;
    const int s_begin = wave * quarter, s_end = s_begin + quarter < nsteps ? s_begin + quarter : nsteps;
    const int row = lane >> 2, lane_off = (lane & 3) * 16;
    const unsigned char* w[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {                    // rows past f: the last one again, not stored
        const int unit = unit0 + row < a.f ? unit0 + row : a.f - 1;
        w[r] = (const unsigned char*)a.W13 + ((long long)e * 2 * a.f + r * a.f + unit) * row_bytes;
    }
    const unsigned char* x[NT];
    bool there[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        there[nt] = nt * 16 + row < tokens;
        x[nt] = (const unsigned char*)a.x + (there[nt] ? (long long)(ls.position[list0 + nt * 16 + row] / a.k) * row_bytes : 0);
    }
    f32x4 acc[2][NT];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[r][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 fw[2][U][2], fx[2][U][NT];
    auto load = [&](auto buf_c, int s0) {
        constexpr int buf = decltype(buf_c)::value;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int off = (s0 + u) * STEP + lane_off;
            const bool in = s0 + u < s_end && off < row_bytes;
#pragma unroll
            for (int r = 0; r < 2; ++r) fw[buf][u][r] = piece(w[r], off, in);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) fx[buf][u][nt] = piece(x[nt], off, in && there[nt]);
        }
    };
    load(IC<0>{}, s_begin);
    for (int s0 = s_begin; s0 < s_end; s0 += 2 * U)
        static_for<2>([&](auto b_c) {
            constexpr int b = decltype(b_c)::value;
            if (s0 + (b + 1) * U < s_end) load(IC<1 - b>{}, s0 + (b + 1) * U);       // wave-uniform
            if (s0 + b * U < s_end)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    u32x4 xo[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) xo[nt] = to_operand(fx[b][u][nt], lane);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const u32x4 wo = to_operand(fw[b][u][r], lane);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) acc[r][nt] = product<BF16>(wo, xo[nt], acc[r][nt]);
                    }
                }
        });
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) part[wave][r][nt][lane] = acc[r][nt];
    __syncthreads();
    // the quarters added in order; lane (n, g) of block nt: token n, units 4g .. 4g + 3
    for (int i = threadIdx.x; i < NT * 64; i += UP_THREADS) {
        const int nt = i >> 6, ln = i & 63, n = nt * 16 + (ln & 15), unit = unit0 + 4 * (ln >> 4);
        if (n >= tokens || unit >= a.f) continue;
        const int p = ls.position[list0 + n];
        const float weight = position_weight(a.idx, a.probs, a.k, p);
        float v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float gate = ((part[0][0][nt][ln][c] + part[1][0][nt][ln][c]) + part[2][0][nt][ln][c]) + part[3][0][nt][ln][c];
            const float up = ((part[0][1][nt][ln][c] + part[1][1][nt][ln][c]) + part[2][1][nt][ln][c]) + part[3][1][nt][ln][c];
            v[c] = weight * apply_act(gate, a.act) * up;
        }
        const long long at = (long long)p * a.f + unit;
        if constexpr (BF16) {
            const u32x2 hi = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
            float lo[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) lo[c] = v[c] - __uint_as_float(c & 1 ? hi[c >> 1] & 0xFFFF0000u : hi[c >> 1] << 16);
            *(u32x2*)((uint16_t*)h + at) = hi;
            *(u32x2*)((uint16_t*)h + (long long)a.T * a.k * a.f + at) = u32x2{pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3])};
        } else {
            *(f32x4*)((float*)h + at) = f32x4{v[0], v[1], v[2], v[3]};
        }
    }
    __syncthreads();
}

template <bool BF16>
__global__ __launch_bounds__(UP_THREADS, 2) void up_kernel(MoeArgs a, int tiles, void* __restrict__ h)
{
    __shared__ Lists ls;
    __shared__ __attribute__((aligned(16))) f32x4 part[4][2][4][64];
    build_lists<UP_THREADS>(ls, a.idx, a.T, a.k, a.E);
    const int slot = blockIdx.x / tiles, unit0 = (blockIdx.x % tiles) * 16;
    if (slot >= ls.n) return;
    const int e = ls.expert[slot], list0 = ls.first[slot], tokens = ls.first[slot + 1] - list0;
    if (tokens <= 16)      up_tokens<BF16, 1>(a, ls, e, list0, tokens, unit0, part, h);
    else if (tokens <= 32) up_tokens<BF16, 2>(a, ls, e, list0, tokens, unit0, part, h);
    else                   up_tokens<BF16, 4>(a, ls, e, list0, tokens, unit0, part, h);
}

// ---------------------------------------------------------------------------
// y
// ---------------------------------------------------------------------------
static constexpr int DOWN_THREADS = 512, DOWN_WAVES = DOWN_THREADS / 64;

// One unit: steps s0 .. s0 + U - 1 of expert slot `slot`, into the wave's sums ysum[t][16].  NT: blocks of columns; a column
// is a token, in bf16 storage a token's high (columns 0..7 of a block) or low part (8..15).
template <bool BF16, int NT, int U> struct DownUnit {
    static constexpr int TOK = BF16 ? 8 : 16;        // tokens of a block
    u32x4 fw[U], fh[U][NT];

    __device__ __forceinline__ void load(const MoeArgs& a, const Lists& ls, const void* h, int slot, int block0, int s0, int row0, int lane)
    {
        const int row_bytes = a.f * (BF16 ? 2 : 4), row = lane >> 2, lane_off = (lane & 3) * 16;
        const int r = row0 + row < a.d ? row0 + row : a.d - 1;                       // rows past d: not stored
        const unsigned char* w = (const unsigned char*)a.W2 + ((long long)ls.expert[slot] * a.d + r) * row_bytes;
        const int list0 = ls.first[slot], tokens = ls.first[slot + 1] - list0;
        const unsigned char* hp[NT];
        bool there[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int n = (block0 + nt) * TOK + (row & (TOK - 1));
            there[nt] = n < tokens;
            const int p = there[nt] ? ls.position[list0 + n] : 0;
            hp[nt] = (const unsigned char*)h + ((long long)p + (BF16 && row >= TOK ? (long long)a.T * a.k : 0)) * row_bytes;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int off = (s0 + u) * STEP + lane_off;
            const bool in = off < row_bytes;
            fw[u] = piece(w, off, in);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) fh[u][nt] = piece(hp[nt], off, in && there[nt]);
        }
    }

    __device__ __forceinline__ void add(const MoeArgs& a, const Lists& ls, int slot, int block0, int lane, float* ysum) const
    {
        f32x4 acc[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const u32x4 wo = to_operand(fw[u], lane);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[nt] = product<BF16>(wo, to_operand(fh[u][nt], lane), acc[nt]);
        }
        const int list0 = ls.first[slot], tokens = ls.first[slot + 1] - list0, col = lane & 15;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if constexpr (BF16) {                    // low part onto high part
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nt][i] += __shfl_xor(acc[nt][i], 8, 64);
            }
            const int n = (block0 + nt) * TOK + col;
            if (col < TOK && n < tokens) {
                f32x4* y = (f32x4*)(ysum + (ls.position[list0 + n] / a.k) * 16 + 4 * (lane >> 4));
                f32x4 v = *y;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += acc[nt][i];
                *y = v;
            }
        }
    }
};

template <bool BF16>
__global__ __launch_bounds__(DOWN_THREADS) void down_kernel(MoeArgs a, const void* __restrict__ h)
{
    __shared__ Lists ls;
    extern __shared__ __attribute__((aligned(16))) float ysums[];                    // [wave][T][16]
    build_lists<DOWN_THREADS>(ls, a.idx, a.T, a.k, a.E);
    const int row0 = blockIdx.x * 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int i = threadIdx.x; i < DOWN_WAVES * a.T * 16; i += DOWN_THREADS) ysums[i] = 0.0f;
    __syncthreads();
    float* ysum = ysums + wave * a.T * 16;
    constexpr int U = 8, TOK = BF16 ? 8 : 16;
    const int nsteps = (a.f * (BF16 ? 2 : 4) + STEP - 1) / STEP, parts = (nsteps + U - 1) / U, units = ls.n * parts;

    DownUnit<BF16, 1, U> ring[2];
    int i = wave;
    if (i < units) ring[0].load(a, ls, h, i / parts, 0, i % parts * U, row0, lane);
    for (; i < units; i += 2 * DOWN_WAVES)
        static_for<2>([&](auto b_c) {
            constexpr int b = decltype(b_c)::value;
            const int now = i + b * DOWN_WAVES, next = now + DOWN_WAVES;
            if (next < units) ring[1 - b].load(a, ls, h, next / parts, 0, next % parts * U, row0, lane);
            if (now < units) {
                const int slot = now / parts, tokens = ls.first[slot + 1] - ls.first[slot];
                ring[b].add(a, ls, slot, 0, lane, ysum);
                for (int block = 1; block * TOK < tokens; ++block) {                 // more tokens: the weights are in a cache by now
                    DownUnit<BF16, 1, U> more;
                    more.load(a, ls, h, slot, block, now % parts * U, row0, lane);
                    more.add(a, ls, slot, block, lane, ysum);
                }
            }
        });
    __syncthreads();
    for (int q = threadIdx.x; q < a.T * 16; q += DOWN_THREADS) {
        const int t = q >> 4, r = row0 + (q & 15);
        if (r >= a.d) continue;
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < DOWN_WAVES; ++w) y += ysums[w * a.T * 16 + q];
        const long long at = (long long)t * a.d + r;
        if constexpr (BF16) {
            if (a.residual) y += bf16_bits_to_f32(((const uint16_t*)a.residual)[at]);
            ((uint16_t*)a.y)[at] = f32_to_bf16_bits(y);
        } else {
            if (a.residual) y += ((const float*)a.residual)[at];
            ((float*)a.y)[at] = y;
        }
    }
}

// ---------------------------------------------------------------------------

static int row_steps(const MoeArgs& a, int n) { return (n * (a.dtype == PAEP_BF16 ? 2 : 4) + STEP - 1) / STEP; }
static int router_slices(const MoeArgs& a) { return (row_steps(a, a.d) + ROUTER_STEPS - 1) / ROUTER_STEPS; }
static size_t h_bytes(const MoeArgs& a) { return ((size_t)a.T * a.k * a.f * 4 + 15) & ~(size_t)15; }      // two bf16 planes or one of fp32

size_t moe_workspace_bytes(const MoeArgs& a) { return h_bytes(a) + (size_t)router_slices(a) * a.T * a.E * 4; }

template <bool BF16> static hipError_t launch(const MoeArgs& a)
{
    float* partial = (float*)((unsigned char*)a.workspace + h_bytes(a));
    if (a.Wg) {
        const int tiles = (a.E + 15) / 16, slices = router_slices(a), row_bytes = a.d * (BF16 ? 2 : 4);
        auto kern = a.T <= 16 ? router_kernel<BF16, 1> : a.T <= 32 ? router_kernel<BF16, 2> : router_kernel<BF16, 4>;
        hipLaunchKernelGGL(kern, dim3(tiles * slices), dim3(ROUTER_THREADS), 0, a.stream, a.T, a.E, row_bytes, tiles,
                           (const unsigned char*)a.x, (const unsigned char*)a.Wg, partial);
        PredictArgs r{};
        r.T = a.T; r.E = a.E; r.k = a.k; r.L = 1; r.dtype = a.dtype; r.b2 = a.bg;
        r.idx = a.idx; r.probs = a.probs; r.counts = a.counts; r.prob_mode = a.prob_mode; r.stream = a.stream;
        const hipError_t err = launch_finalize(r, partial, slices, 1, a.T, 0, 1);
        if (err != hipSuccess) return err;
    }
    const int tiles = (a.f + 15) / 16, most = a.T * a.k < a.E ? a.T * a.k : a.E;     // active experts at most
    hipLaunchKernelGGL(up_kernel<BF16>, dim3(most * tiles), dim3(UP_THREADS), 0, a.stream, a, tiles, a.workspace);
    hipLaunchKernelGGL(down_kernel<BF16>, dim3((a.d + 15) / 16), dim3(DOWN_THREADS), sizeof(float) * DOWN_WAVES * a.T * 16, a.stream, a,
                       a.workspace);
    return hipGetLastError();
}

hipError_t launch_moe(const MoeArgs& a) { return a.dtype == PAEP_BF16 ? launch<true>(a) : launch<false>(a); }

}  // namespace paep
