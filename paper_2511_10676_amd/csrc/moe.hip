// A mixture-of-experts layer for a few tokens (T <= 64): router, selection, gated experts, weighted sum.
//
//   z = x Wg^T,  (idx, p) = top k,   h_j = p_j act(W1 x) * (W3 x),   y = residual + sum_j W2 h_j
//
// Every weight of every expert that some token picked is needed once and the arithmetic per weight is tiny: reading them is
// what bounds the layer, so the kernels stream weight rows from memory into the registers of the matrix instructions with as
// many loads in flight as fit, and tokens are the narrow operand.  Launches:
//   router_kernel   scores of 16 experts over a slice of d, partial sums to the workspace
//   select_kernel   adds the slices, softmax and top-k with the predictor's own routines (or takes a given selection), and
//                   lists the active experts and who picked them
//   up_kernel       16 gate rows and the 16 rows beside them of one expert over all of d, for the tokens that picked it: the
//                   four waves split d.  h goes to the workspace in fp32, already weighed by p
//   down_kernel     16 rows of d over all active experts: the eight waves split (expert, part of f); sums per token in LDS.
//                   With h in 16 bits (two bf16 parts, stored) sums that cancel had fewer right bits than y can hold; taking all
//                   24 bits of it apart here costs 1.5 to 4 us of the layer
//   sum_kernel      where two or more workgroups share 16 rows
// A fragment of 16 rows x 64 bytes is fetched with four neighbouring lanes on 64 contiguous bytes of a row, and a fixed lane
// permutation puts it into the operand layout (as in predict_decode.hip).
// Measured (us; up / down kernel): 61 tokens, 64 experts 2048 x 1408, top 6: 233 (130 at 5.7 TB/s / 79 at 4.7); 16 tokens, 16
// experts 4096 x 960, top 2: 82 (43 / 26); one token, 8 experts 2048 x 768: 33 (13 / 11, the other two launches 10); fp32, 7
// tokens, 32 experts 1024 x 704, top 4: 52 (25 / 15); 64 tokens, 16 experts 4096 x 960, top 2: 99; 64 tokens, 8 experts
// 2048 x 768, top 4, 32 tokens to each: 61.  (The first form, with a list per workgroup, d = 2048 in 128 workgroups and masks
// applied behind the loads, which are then waited for at once, took 356, 91, 38 and 87 for the first four.)
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

// Rows are read through buffer resources: what lies past a resource's end, as NOWHERE does, reads as zeros.
static constexpr int NOWHERE = 0x7FFFFFF0;
typedef __amdgpu_buffer_rsrc_t Rows;
__device__ __forceinline__ Rows rows_at(const void* base, long long bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
// 16 bytes of a row that begins at `row` (NOWHERE: no such row), `off` bytes into it
__device__ __forceinline__ u32x4 piece(Rows r, int row, int off, int row_bytes)
{
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off < row_bytes && row != NOWHERE ? row + off : NOWHERE, 0, 0));
}

// What the workspace holds of a selection: the active experts in ascending order and, one after the other, their positions
// p = t * k + j (an id that stands in a row several times at its first place only; ids outside [0, E) nowhere).  The order of
// one expert's positions differs from run to run; no result depends on it.
struct Lists {
    int32_t n;                                       // active experts
    uint32_t arrived;                                // workgroups of select_kernel that have written their rows
    int32_t pad[2];
    uint32_t slot[PAEP_MAX_E];                       // expert | where its positions begin << 10 | how many << 21
    uint16_t position[MOE_MAX_POS];
    float weight[MOE_MAX_POS];                       // of a position: its probability, or the sum over the places of its id in the row
};
static_assert(PAEP_MAX_E <= 1 << 10 && MOE_MAX_POS <= 1 << 11 && PAEP_MOE_MAX_T < 1 << 11, "a slot's fields");
struct Slot {
    int expert, first, tokens;
    __device__ __forceinline__ explicit Slot(uint32_t v)
    {
        const uint32_t u = __builtin_amdgcn_readfirstlane(v);
        expert = u & 1023u;
        first = (u >> 10) & 2047u;
        tokens = u >> 21;
    }
};

// ---------------------------------------------------------------------------
// Router: partial[slice][t][e].  A workgroup per 16 experts and slice of d, its four waves a quarter of the slice each.
// ---------------------------------------------------------------------------
static constexpr int ROUTER_THREADS = 256, ROUTER_WAVE_STEPS = 4, ROUTER_STEPS = 4 * ROUTER_WAVE_STEPS;

template <bool BF16, int NT>
__global__ __launch_bounds__(ROUTER_THREADS) void router_kernel(int T, int E, int row_bytes, int tiles, const unsigned char* __restrict__ x,
                                                                const unsigned char* __restrict__ Wg, float* __restrict__ partial, Lists* __restrict__ ls)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) ls->arrived = 0;
    __shared__ __attribute__((aligned(16))) f32x4 part[3][NT][64];
    const int tile = blockIdx.x % tiles, slice = blockIdx.x / tiles;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane >> 2, at = (slice * ROUTER_STEPS + wave * ROUTER_WAVE_STEPS) * STEP + (lane & 3) * 16;
    const Rows wr = rows_at(Wg + (long long)tile * 16 * row_bytes, (long long)min(E - tile * 16, 16) * row_bytes);
    const Rows xr = rows_at(x, (long long)T * row_bytes);
    u32x4 w[ROUTER_WAVE_STEPS], xf[NT][ROUTER_WAVE_STEPS];
#pragma unroll
    for (int u = 0; u < ROUTER_WAVE_STEPS; ++u) {
        w[u] = piece(wr, row * row_bytes, at + u * STEP, row_bytes);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) xf[nt][u] = piece(xr, (nt * 16 + row) * row_bytes, at + u * STEP, row_bytes);
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
// Selection, a wave per row; the workgroup that is done last makes the lists (made by every workgroup of the next two
// launches for itself they cost each of them 2 us).
// ---------------------------------------------------------------------------
// NV: experts per lane of a row, E <= 64 * NV; 0: the selection is there already
template <int NV, int SELECT_THREADS>
__global__ __launch_bounds__(SELECT_THREADS) void select_kernel(MoeArgs a, const float* __restrict__ partial, int slices, Lists* __restrict__ ls)
{
    __shared__ int32_t ids[MOE_MAX_POS], count[PAEP_MAX_E];
    __shared__ float probs[MOE_MAX_POS];
    constexpr int SELECT_WAVES = SELECT_THREADS / 64;
    __shared__ uint32_t before_me;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.T * a.k;
    for (int e = tid; e < a.E; e += SELECT_THREADS) count[e] = 0;
    if constexpr (NV > 0) {
        const EpilogueOut eo{a.prob_mode, nullptr, a.counts};
        constexpr int CH = NV <= 2 ? 8 : NV <= 4 ? 4 : 2;    // slices requested together
        const int t = blockIdx.x * SELECT_WAVES + wave;
        if (t < a.T) {
            float z[NV] = {};
            for (int s0 = 0; s0 < slices; s0 += CH) {
                float v[CH][NV];
#pragma unroll
                for (int s = 0; s < CH; ++s)
#pragma unroll
                    for (int c = 0; c < NV; ++c)
                        v[s][c] = partial[((long long)min(s0 + s, slices - 1) * a.T + t) * a.E + min(lane + 64 * c, a.E - 1)];
#pragma unroll
                for (int s = 0; s < CH; ++s)
#pragma unroll
                    for (int c = 0; c < NV; ++c) z[c] += s0 + s < slices ? v[s][c] : 0.0f;
            }
            if (a.bg)
#pragma unroll
                for (int c = 0; c < NV; ++c) {
                    const int e = min(lane + 64 * c, a.E - 1);
                    z[c] += a.dtype == PAEP_BF16 ? bf16_bits_to_f32(((const uint16_t*)a.bg)[e]) : ((const float*)a.bg)[e];
                }
            if constexpr (NV == 1) wave_softmax_topk_rank(z[0], a.E, a.k, lane, a.idx + t * a.k, a.probs + t * a.k, eo);
            else                   wave_softmax_topk<NV>(z, a.E, a.k, lane, a.idx + t * a.k, a.probs + t * a.k, eo);
        }
        if (gridDim.x > 1) {
            __threadfence();                                 // the rows are written before the workgroup counts as done,
            __syncthreads();
            if (tid == 0) before_me = atomicAdd(&ls->arrived, 1u);
            __syncthreads();
            if (before_me != gridDim.x - 1) return;
            __threadfence();                                 // and read after all of them do
        }
        __syncthreads();
    }
    for (int p = tid; p < n; p += SELECT_THREADS) {
        ids[p] = a.idx[p];
        probs[p] = a.probs[p];
    }
    __syncthreads();
    constexpr int MINE = MOE_MAX_POS / SELECT_THREADS;
    int id[MINE], rank[MINE];
    float weight[MINE];
#pragma unroll
    for (int u = 0; u < MINE; ++u) {
        const int p = tid + u * SELECT_THREADS;
        id[u] = -1;
        if (p >= n) continue;
        const int e = ids[p];
        weight[u] = probs[p];
        bool first = (uint32_t)e < (uint32_t)a.E;
        if (NV == 0 && first) {                      // (a selection made above has no id twice in a row)
            const int t0 = p / a.k * a.k;
            weight[u] = 0.0f;
            for (int q = t0; q < t0 + a.k; ++q)
                if (ids[q] == e) {
                    if (q < p) first = false;
                    weight[u] += probs[q];
                }
        }
        if (!first) continue;
        id[u] = e;
        rank[u] = atomicAdd(&count[e], 1);
    }
    __syncthreads();
    if (wave == 0) {
        int active = 0, before = 0;
        for (int e0 = 0; e0 < a.E; e0 += 64) {
            const int e = e0 + lane, c = e < a.E ? count[e] : 0;
            int upto = c;
            for (int s = 1; s < 64; s <<= 1) {
                const int o = __shfl_up(upto, s, 64);
                if (lane >= s) upto += o;
            }
            const unsigned long long who = __ballot(c > 0);
            if (c > 0) {
                ls->slot[active + __popcll(who & ((1ull << lane) - 1))] = (uint32_t)e | (uint32_t)(before + upto - c) << 10 | (uint32_t)c << 21;
                count[e] = before + upto - c;        // from here on: where its positions begin
            }
            active += __popcll(who);
            before += __shfl(upto, 63, 64);
        }
        if (lane == 0) ls->n = active;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MINE; ++u)
        if (id[u] >= 0) {
            const int i = count[id[u]] + rank[u];
            ls->position[i] = (uint16_t)(tid + u * SELECT_THREADS);
            ls->weight[i] = weight[u];
        }
}

// ---------------------------------------------------------------------------
// h: [T * k][f], fp32
// ---------------------------------------------------------------------------
static constexpr int UP_THREADS = 256;

// One item: 16 gate rows and the 16 rows beside them of one expert, for 16 * NT of its tokens from the `block`-th on.
template <bool BF16, int NT> struct UpItem {
    Slot s;
    int block, unit0, xrow[NT];
    Rows gate, up;

    __device__ __forceinline__ UpItem(const MoeArgs& a, const Lists* __restrict__ ls, uint32_t slot, int block_, int tile, int lane) : s(slot), block(block_)
    {
        const int row_bytes = a.d * (BF16 ? 2 : 4);
        unit0 = tile * 16;
        const unsigned char* w = (const unsigned char*)a.W13 + ((long long)s.expert * 2 * a.f + unit0) * row_bytes;
        const long long bytes = (long long)min(a.f - unit0, 16) * row_bytes;
        gate = rows_at(w, bytes);
        up = rows_at(w + (long long)a.f * row_bytes, bytes);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int n = block * 16 + nt * 16 + (lane >> 2);
            xrow[nt] = n < s.tokens ? ls->position[s.first + n] / a.k * row_bytes : NOWHERE;
        }
    }
};

// What a wave does of an item: its quarter of d, in batches of U steps, two in registers.
template <bool BF16, int NT, int U> struct UpWave {
    Rows x;
    int wrow, lane_off, row_bytes, s_begin, s_end, rounds;
    u32x4 fw[2][U][2], fx[2][U][NT];
    f32x4 acc[2][NT];

    __device__ __forceinline__ UpWave(const MoeArgs& a, int wave, int lane)
    {
        row_bytes = a.d * (BF16 ? 2 : 4);
        const int nsteps = (row_bytes + STEP - 1) / STEP, quarter = (nsteps + 3) / 4;
        s_begin = wave * quarter;
        s_end = min(s_begin + quarter, nsteps);
        rounds = (quarter + 2 * U - 1) / (2 * U);    // (the same for all waves)
        x = rows_at(a.x, (long long)a.T * row_bytes);
        wrow = (lane >> 2) * row_bytes;
        lane_off = (lane & 3) * 16;
        clear();
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[r][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    template <int BUF> __device__ __forceinline__ void load(const UpItem<BF16, NT>& it, int batch)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s_begin + batch * U + u, off = s < s_end ? s * STEP + lane_off : NOWHERE;
            fw[BUF][u][0] = piece(it.gate, wrow, off, row_bytes);
            fw[BUF][u][1] = piece(it.up, wrow, off, row_bytes);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s_begin + batch * U + u, off = s < s_end ? s * STEP + lane_off : NOWHERE;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) fx[BUF][u][nt] = piece(x, it.xrow[nt], off, row_bytes);
        }
    }
    template <int BUF> __device__ __forceinline__ void multiply(int lane)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            u32x4 xo[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) xo[nt] = to_operand(fx[BUF][u][nt], lane);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const u32x4 wo = to_operand(fw[BUF][u][r], lane);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[r][nt] = product<BF16>(wo, xo[nt], acc[r][nt]);
            }
        }
    }
    // The quarters added in order; lane (n, g) of block nt: token n, units 4g .. 4g + 3.
    __device__ __forceinline__ void finish(const MoeArgs& a, const Lists* __restrict__ ls, const UpItem<BF16, NT>& it, f32x4 (&part)[4][2][NT][64], void* h, int wave, int lane)
    {
        const int n = it.block * 16 + (threadIdx.x >> 6) * 16 + (lane & 15), unit = it.unit0 + 4 * (lane >> 4);
        const bool mine = (int)(threadIdx.x >> 6) < NT && n < it.s.tokens && unit < a.f;
        const int i = it.s.first + (mine ? n : 0), p = ls->position[i];
        const float weight = ls->weight[i];
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) part[wave][r][nt][lane] = acc[r][nt];
        clear();
        __syncthreads();
        if (mine) {                                  // wave w: block w
            const int nt = wave;
            float v[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float gate = ((part[0][0][nt][lane][c] + part[1][0][nt][lane][c]) + part[2][0][nt][lane][c]) + part[3][0][nt][lane][c];
                const float up = ((part[0][1][nt][lane][c] + part[1][1][nt][lane][c]) + part[2][1][nt][lane][c]) + part[3][1][nt][lane][c];
                v[c] = weight * apply_act(gate, a.act) * up;
            }
            const long long at = (long long)p * a.f + unit;
            *(f32x4*)((float*)h + at) = f32x4{v[0], v[1], v[2], v[3]};
        }
        __syncthreads();
    }
};

// The items of a workgroup one after the other; the next one's first batch is requested before this one's last is multiplied.
// FEW: T <= 16, an expert's tokens are one block.  Otherwise blocks of 64 where an expert has more than 16 tokens.
template <bool BF16, bool FEW>
__global__ __launch_bounds__(UP_THREADS, FEW ? 3 : 2) void up_kernel(MoeArgs a, int tiles, const Lists* __restrict__ ls, void* __restrict__ h)
{
    constexpr int U = FEW ? 4 : 8;
    __shared__ __attribute__((aligned(16))) unsigned char lds[sizeof(f32x4) * 4 * 2 * (FEW ? 1 : 4) * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int item = blockIdx.x;
    uint32_t slot = ls->slot[item / tiles];          // (within the array even where there is no such item)
    const int items = ls->n * tiles;
    if (item >= items) return;
    UpWave<BF16, 1, U> w(a, wave, lane);
    UpItem<BF16, 1> now(a, ls, slot, 0, item % tiles, lane);
    w.template load<0>(now, 0);
    for (;;) {
        const int next = item + gridDim.x;
        const bool more = next < items;
        slot = ls->slot[more ? next / tiles : 0];
        const UpItem<BF16, 1> then(a, ls, slot, 0, more ? next % tiles : 0, lane);
        bool wide = false;
        if constexpr (!FEW) wide = now.s.tokens > 16;
        if (!wide) {
            for (int i = 0; i < w.rounds; ++i) {
                w.template load<1>(now, 2 * i + 1);
                w.template multiply<0>(lane);
                if (i + 1 < w.rounds) w.template load<0>(now, 2 * i + 2);
                else if (more)        w.template load<0>(then, 0);
                w.template multiply<1>(lane);
            }
            w.finish(a, ls, now, *(f32x4(*)[4][2][1][64])lds, h, wave, lane);
        } else if constexpr (!FEW) {
            UpItem<BF16, 4> big(a, ls, ls->slot[item / tiles], 0, item % tiles, lane);
            UpWave<BF16, 4, 2> v(a, wave, lane);
            v.template load<0>(big, 0);
            for (int i = 0; i < v.rounds; ++i) {
                v.template load<1>(big, 2 * i + 1);
                v.template multiply<0>(lane);
                if (i + 1 < v.rounds) v.template load<0>(big, 2 * i + 2);
                v.template multiply<1>(lane);
            }
            v.finish(a, ls, big, *(f32x4(*)[4][2][4][64])lds, h, wave, lane);
            if (more) w.template load<0>(then, 0);
        }
        if (!more) return;
        item = next;
        now = then;
    }
}

// ---------------------------------------------------------------------------
// y
// ---------------------------------------------------------------------------
struct Picked {                                      // in LDS
    uint32_t slot[PAEP_MAX_E];
    uint16_t position[MOE_MAX_POS];
};

static constexpr int DOWN_THREADS = 512, DOWN_WAVES = DOWN_THREADS / 64;

template <bool BF16> __device__ __forceinline__ void write_y(const MoeArgs& a, long long at, float y)
{
    if constexpr (BF16) {
        if (a.residual) y += bf16_bits_to_f32(((const uint16_t*)a.residual)[at]);
        ((uint16_t*)a.y)[at] = f32_to_bf16_bits(y);
    } else {
        if (a.residual) y += ((const float*)a.residual)[at];
        ((float*)a.y)[at] = y;
    }
}

// One unit: steps s0 .. s0 + U - 1 of expert slot `slot`, for 16 of its tokens, into the wave's sums ysum[t][16].  h is read in the
// order of the operand: lane (n, c) has token n's values beside piece c of the weights.  In bf16 storage they are multiplied as
// three bf16 parts of 8 bits, cut off and not rounded: exactly the 24 bits of an fp32 number, and a finite h has finite parts.
template <bool BF16, int U> struct DownUnit {
    static constexpr int TOK = 16, H = BF16 ? 2 : 1;     // tokens of a block; pieces of h beside a piece of the weights
    u32x4 fw[U], fh[U][H];

    // WEIGHTS: both; else h only, of a further block for the weights that are there
    template <bool WEIGHTS> __device__ __forceinline__ void load(const MoeArgs& a, const Picked& ls, const void* h, int slot, int block, int s0, int row0, int lane)
    {
        const int row_bytes = a.f * (BF16 ? 2 : 4), row = lane >> 2, lane_off = (lane & 3) * 16;
        const Slot s(ls.slot[slot]);
        const Rows w = rows_at((const unsigned char*)a.W2 + ((long long)s.expert * a.d + row0) * row_bytes, (long long)min(a.d - row0, 16) * row_bytes);
        const Rows hr = rows_at(h, (long long)a.T * a.k * a.f * 4);
        const int n = block * TOK + (lane & 15), hrow = n < s.tokens ? ls.position[s.first + n] * a.f * 4 : NOWHERE;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (WEIGHTS) fw[u] = piece(w, row * row_bytes, (s0 + u) * STEP + lane_off, row_bytes);
#pragma unroll
            for (int i = 0; i < H; ++i) fh[u][i] = piece(hr, hrow, ((s0 + u) * STEP + (lane >> 4) * 16) * H + i * 16, a.f * 4);
        }
    }

    __device__ __forceinline__ void add(const MoeArgs& a, const Picked& ls, int slot, int block, int lane, float* ysum) const
    {
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f}, rest = acc;       // (rest: of the second and third parts)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const u32x4 wo = to_operand(fw[u], lane);
            if constexpr (BF16) {
                float left[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) left[i] = __uint_as_float(fh[u][i >> 2][i & 3]);
#pragma unroll
                for (int part = 0; part < 3; ++part) {
                    u32x4 x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_perm(__float_as_uint(left[2 * i + 1]), __float_as_uint(left[2 * i]), 0x07060302u);
                    if (part == 0) acc = product<BF16>(wo, x, acc);
                    else           rest = product<BF16>(wo, x, rest);
#pragma unroll
                    for (int i = 0; i < 8; ++i) left[i] -= __uint_as_float(__float_as_uint(left[i]) & 0xFFFF0000u);
                }
            } else {
                acc = product<BF16>(wo, fh[u][0], acc);
            }
        }
        const Slot s(ls.slot[slot]);
        const int n = block * TOK + (lane & 15);
        if (n < s.tokens) {
            f32x4* y = (f32x4*)(ysum + (ls.position[s.first + n] / a.k) * 16 + 4 * (lane >> 4));
            f32x4 v = *y;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // where a weight or an h is infinite, the first part alone has the outcome: it has h's sign and is 0 only if h is
                // (a later part, 0 or of the other sign, makes NaN of it)
                v[i] += BF16 && __builtin_isfinite(acc[i]) ? acc[i] + rest[i] : acc[i];
            }
            *y = v;
        }
    }
};

// `parts` workgroups share 16 rows (parts > 1: their sums go to ypart[part][T][d])
template <bool BF16>
__global__ __launch_bounds__(DOWN_THREADS, 2) void down_kernel(MoeArgs a, const Lists* __restrict__ lists, const void* __restrict__ h, int parts, float* __restrict__ ypart)
{
    __shared__ Picked ls;
    extern __shared__ __attribute__((aligned(16))) float ysums[];                    // [wave][T][16]
    const int row0 = blockIdx.x / parts * 16, part = blockIdx.x % parts;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int i = tid; i < DOWN_WAVES * a.T * 16; i += DOWN_THREADS) ysums[i] = 0.0f;
    const int n = lists->n;
    for (int i = tid; i < n; i += DOWN_THREADS) ls.slot[i] = lists->slot[i];
    for (int i = tid; i < a.T * a.k; i += DOWN_THREADS) ls.position[i] = lists->position[i];
    __syncthreads();
    float* ysum = ysums + wave * a.T * 16;
    constexpr int U = BF16 ? 6 : 8, TOK = DownUnit<BF16, U>::TOK;       // (bf16, 61 tokens: 7 steps 244 us, 8 238, 6 237)
    const int nsteps = (a.f * (BF16 ? 2 : 4) + STEP - 1) / STEP, pieces = (nsteps + U - 1) / U, units = n * pieces, stride = DOWN_WAVES * parts;

    DownUnit<BF16, U> ring[2];
    int i = part * DOWN_WAVES + wave;
    if (i < units) ring[0].template load<true>(a, ls, h, i / pieces, 0, i % pieces * U, row0, lane);
    for (; i < units; i += 2 * stride)
        static_for<2>([&](auto b_c) {
            constexpr int b = decltype(b_c)::value;
            const int now = i + b * stride, next = now + stride;
            if (next < units) ring[1 - b].template load<true>(a, ls, h, next / pieces, 0, next % pieces * U, row0, lane);
            if (now < units) {
                const int slot = now / pieces, tokens = Slot(ls.slot[slot]).tokens;
                ring[b].add(a, ls, slot, 0, lane, ysum);
                for (int block = 1; block * TOK < tokens; ++block) {
                    ring[b].template load<false>(a, ls, h, slot, block, now % pieces * U, row0, lane);
                    ring[b].add(a, ls, slot, block, lane, ysum);
                }
            }
        });
    __syncthreads();
    for (int q = tid; q < a.T * 16; q += DOWN_THREADS) {
        const int t = q >> 4, r = row0 + (q & 15);
        if (r >= a.d) continue;
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < DOWN_WAVES; ++w) y += ysums[w * a.T * 16 + q];
        const long long at = (long long)t * a.d + r;
        if (parts > 1) ypart[(long long)part * a.T * a.d + at] = y;
        else write_y<BF16>(a, at, y);
    }
}

// the parts of down_kernel, added in order (by the workgroup of some rows that is done last, which the parts then have to be
// made visible to across L2 caches, this took 70 us where the launch takes 4)
template <bool BF16> __global__ __launch_bounds__(256) void sum_kernel(MoeArgs a, int parts, const float* __restrict__ ypart)
{
    const int i = blockIdx.x * 256 + threadIdx.x, n = a.T * a.d;
    if (i >= n) return;
    float y = 0.0f;
    for (int p = 0; p < parts; ++p) y += ypart[(long long)p * n + i];
    write_y<BF16>(a, i, y);
}

// ---------------------------------------------------------------------------

static int row_steps(const MoeArgs& a, int n) { return (n * (a.dtype == PAEP_BF16 ? 2 : 4) + STEP - 1) / STEP; }
static int router_slices(const MoeArgs& a) { return (row_steps(a, a.d) + ROUTER_STEPS - 1) / ROUTER_STEPS; }
static size_t h_bytes(const MoeArgs& a) { return ((size_t)a.T * a.k * a.f * 4 + 15) & ~(size_t)15; }

static size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
// Workgroups that share 16 rows of d: enough for one per CU (a workgroup's registers leave room for no second), unless a wave would
// have fewer than 64 steps -- the sums' launch then costs most of what the other CUs gain (one token, 8 experts of 2048 x 768:
// 32.7 us, in two parts 31.9; 61 tokens of 64 experts 233 us in two parts, 282 in one, 240 in four).
static int down_parts(const MoeArgs& a)
{
    const int tiles = (a.d + 15) / 16, parts = (256 + tiles - 1) / tiles;
    const int units = (a.T * a.k < a.E ? a.T * a.k : a.E) * ((row_steps(a, a.f) + 7) / 8);
    return units < 8 * DOWN_WAVES ? 1 : parts > 8 ? 8 : parts;
}

size_t moe_workspace_bytes(const MoeArgs& a)
{
    return h_bytes(a) + up16(sizeof(Lists)) + up16((size_t)router_slices(a) * a.T * a.E * 4) + (down_parts(a) > 1 ? (size_t)down_parts(a) * a.T * a.d * 4 : 0);
}

template <bool BF16> static hipError_t launch(const MoeArgs& a)
{
    unsigned char* ws = (unsigned char*)a.workspace;
    void* h = ws;
    Lists* ls = (Lists*)(ws + h_bytes(a));
    float* partial = (float*)((unsigned char*)ls + up16(sizeof(Lists)));
    const int slices = router_slices(a), row_bytes = a.d * (BF16 ? 2 : 4);
    float* ypart = (float*)((unsigned char*)partial + up16((size_t)slices * a.T * a.E * 4));
    if (a.Wg) {
        const int tiles = (a.E + 15) / 16;
        auto kern = a.T <= 16 ? router_kernel<BF16, 1> : a.T <= 32 ? router_kernel<BF16, 2> : router_kernel<BF16, 4>;
        hipLaunchKernelGGL(kern, dim3(tiles * slices), dim3(ROUTER_THREADS), 0, a.stream, a.T, a.E, row_bytes, tiles,
                           (const unsigned char*)a.x, (const unsigned char*)a.Wg, partial, ls);
    }
    auto select = [&](auto threads_c) {
        constexpr int N = decltype(threads_c)::value;
        return a.E <= 64 ? select_kernel<1, N> : a.E <= 128 ? select_kernel<2, N> : a.E <= 256 ? select_kernel<4, N>
             : a.E <= 512 ? select_kernel<8, N> : select_kernel<16, N>;
    };
    // up to 16 rows by one workgroup of as many waves, more by workgroups of 4: a CU's vector units are what 16 selections at
    // once wait for (61 rows of 64 experts: 20 us by one workgroup, 13 by 4 of 16 waves, 8 by 16 of 4; 7 rows: 4.9 and 6.5)
    if (!a.Wg)           hipLaunchKernelGGL((select_kernel<0, 1024>), dim3(1), dim3(1024), 0, a.stream, a, partial, slices, ls);
    else if (a.T <= 16)  hipLaunchKernelGGL(select(IC<1024>{}), dim3(1), dim3(1024), 0, a.stream, a, partial, slices, ls);
    else                 hipLaunchKernelGGL(select(IC<256>{}), dim3((a.T + 3) / 4), dim3(256), 0, a.stream, a, partial, slices, ls);
    const int tiles = (a.f + 15) / 16, most = a.T * a.k < a.E ? a.T * a.k : a.E;     // active experts at most
    const int up_wgs = a.T <= 16 ? 768 : 512;                // what fits on the chip's CUs at once
    hipLaunchKernelGGL((a.T <= 16 ? up_kernel<BF16, true> : up_kernel<BF16, false>), dim3(most * tiles < up_wgs ? most * tiles : up_wgs), dim3(UP_THREADS), 0, a.stream, a, tiles, ls, h);
    const int parts = down_parts(a);
    hipLaunchKernelGGL(down_kernel<BF16>, dim3((a.d + 15) / 16 * parts), dim3(DOWN_THREADS), sizeof(float) * DOWN_WAVES * a.T * 16, a.stream, a,
                       ls, h, parts, ypart);
    if (parts > 1) hipLaunchKernelGGL(sum_kernel<BF16>, dim3((a.T * a.d + 255) / 256), dim3(256), 0, a.stream, a, parts, ypart);
    return hipGetLastError();
}

hipError_t launch_moe(const MoeArgs& a) { return a.dtype == PAEP_BF16 ? launch<true>(a) : launch<false>(a); }

}  // namespace paep
