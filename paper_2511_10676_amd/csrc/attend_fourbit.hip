// Attention of one new token per sequence over a paged cache held in 4 bits: the formula of attend.hip on
//
//   k = code * 2^(byte - 127),   v likewise        32 neighbours of a row share a byte
//
// A code times a power of two is a bf16 number, so nothing is rounded on the way from the cache to the matrix instructions.
// The products are those of attend.hip, with 32 positions of a wave at a time: S^T = K Q^T, lane (m, g) holding 16 bytes, a whole
// group, of key m; O^T = V^T P^T, lane (c, g) holding the same dimensions of 8 positions, whose codes become pairs of one position
// and then, by a byte permutation, pairs of neighbouring positions.  P is three bf16 parts, 24 bits, and what a part leaves is one dot
// product.  Queries of fp32 are three parts as well.  Scores are in units of log2, an addition away from their exponentials, and the
// reference point of those moves only where a score is more than 8 above it, so that lanes seldom talk to each other.
// The sequences' positions, in units of 128, are laid end to end and cut into equal spans for each block of up to 16 query heads; a
// workgroup walks its span, sequence by sequence.  Where a sequence is cut, the pieces are joined by attend_fourbit_join_kernel.
// (One workgroup for 512 positions of each sequence took 137 us for 31 sequences of 2000 to 32768 positions, 8 heads: half of it
// before the first product and behind the last.)
// What bounds it: a position of 128 + 128 dimensions is 136 bytes, 17 / 64 of bf16 storage.  Those 31 sequences, 380 MB, take 96 us
// (4.0 TB/s), and as long with the products left out: what bounds them is reading 64-byte rows of 3000 streams, and with pages that stay
// on the chip they take some 65 us.  131071 positions of 4 heads, 71 MB, 19 us, 5 of them before the first product and behind the last, and
// 9.7 us of join.  Rows fetched through LDS, so that neighbouring lanes read neighbouring bytes, or two tiles ahead, take as long.
#include <type_traits>

#include "attend_device.h"
#include "fourbit_device.h"

namespace paep {

static constexpr int FOUR_THREADS = 256, FOUR_WAVES = FOUR_THREADS / 64;
static constexpr int FOUR_TILE = 32;             // positions of a wave at a time, two halves of 16
static constexpr int UNIT = FOUR_WAVES * FOUR_TILE;          // of a workgroup: what spans are counted in
// A span has at least 2 units, and more where that leaves 512 spans, two for every CU; from 16 units on there are as many spans as
// that gives, up to 2304 (times of both launches: 61 sequences of 1400 positions, 64 query heads of 8: 31 us, with 8 in place of the 16,
// which cuts every sequence, 50; 31 of 2000 to 32768 positions: 116.5 us, with 8 119, for 768 spans 118, 1536 115.5, 4096 116.4; one of
// 131071 positions, 4 heads: 28.5 us, with 8 28.6, for 768 to 4096 spans 28.2 to 28.4).
static constexpr int LEAST_UNITS = 2, ENOUGH_UNITS = 16, ENOUGH_SPANS = 512, MOST_SPANS = 2304;
static constexpr int SEQUENCES = 1024;           // of a launch
static constexpr float LOG2E_REST = 1.92596303e-8f;          // log2 e - LOG2E
// Scores in units of log2 up to this are right.  A reference point is such a score rounded, and the exponentials, of what fmaf has unrounded,
// and `rest` below carry a power of 2 that grows with that rounding: less than 4 up to here, past fp32's range from 2^31 on.
static constexpr float FARTHEST = 0x1p24f;

struct FourPlan {
    int G, head_blocks;          // query heads of a key-value head, blocks of 16 of them
    int columns, spans, enough;  // blocks of query heads of all key-value heads; spans of each, at most and where they are short
    int b0, n;                   // the launch's sequences b0 .. b0 + n - 1
    f32x4* o;                    // [columns][spans][2][VD][64] what pieces of sequences that are cut came to, each over its own sum:
                                 // of a span's first piece where that began before it, of its last where that goes on behind it
    float2* ml;                  // [columns][spans][2][16] their scores' reference points, and their sums
    uint32_t* before;            // [n + 1] units before each sequence
};

__device__ __forceinline__ f32x4 mfma32(const u32x4& x, const u32x4& y, f32x4 acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
}
// v less one of two bf16 numbers: which = -1 in its place, 0 in the other (and no constant, which the compiler puts in wrongly)
__device__ __forceinline__ float less_one(float v, uint32_t both, uint32_t which)
{
    typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2v, both), __builtin_bit_cast(bf16x2v, which), v, false);
}
__device__ __forceinline__ float across_groups_max(float v)      // over the four lanes of one head
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
// units of a sequence: one at least, so that someone writes the zeros of an empty one
__device__ __forceinline__ uint32_t units_of(int start, int len)
{
    return start < len ? ((uint32_t)(len - (start & ~15)) + UNIT - 1) / UNIT : 1u;
}
// Units of a span, of `total`.
__device__ __forceinline__ uint32_t span_units(uint32_t total, const FourPlan& pl)
{
    const uint32_t even = (total + pl.enough - 1) / (uint32_t)pl.enough;
    return max(min(max(even, (uint32_t)LEAST_UNITS), (uint32_t)ENOUGH_UNITS), (total + pl.spans - 1) / (uint32_t)pl.spans);
}
// entry i of a row of the page table, the same for the whole wave
__device__ __forceinline__ int uniform_entry(const int32_t* row, int i)
{
    return ((const __attribute__((address_space(4))) int32_t*)row)[i];
}

// 4 W bytes (W = 0: 2, W = -1: 1) at an address that is the wave's, and a lane's offset from it
template <int W> __device__ __forceinline__ void load_at(const unsigned char* base, uint32_t lane_at, uint32_t at, uint32_t* to)
{
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0x7FFFFFFF, 0x00020000);
    if constexpr (W == -1) to[0] = __builtin_amdgcn_raw_buffer_load_b8(r, lane_at, at, 0);
    else if constexpr (W == 0) to[0] = __builtin_amdgcn_raw_buffer_load_b16(r, lane_at, at, 0);
    else if constexpr (W == 1) to[0] = __builtin_amdgcn_raw_buffer_load_b32(r, lane_at, at, 0);
    else if constexpr (W == 2) { const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, lane_at, at, 0)); to[0] = x[0]; to[1] = x[1]; }
    else { const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_at, at, 0)); for (int i = 0; i < 4; ++i) to[i] = x[i]; }
}
// ... or one of the lane's own
template <int W> __device__ __forceinline__ void load_own(const unsigned char* at, uint32_t* to)
{
    if constexpr (W == -1) to[0] = *at;
    else if constexpr (W == 0) to[0] = *(const uint16_t*)at;
    else if constexpr (W == 1) to[0] = *(const uint32_t*)at;
    else if constexpr (W == 2) { const u32x2 x = *(const u32x2*)at; to[0] = x[0]; to[1] = x[1]; }
    else { const u32x4 x = *(const u32x4*)at; for (int i = 0; i < 4; ++i) to[i] = x[i]; }
}

// QP: bf16 parts of a query element (1: bf16 storage, 3: fp32); KW: 4-byte words of a key in a lane (16 lanes' worth of 4 words
// cover 128 dimensions); VD: dimensions of a value in a lane; PAGED16: 16 neighbours are on one page, whose address is the
// wave's (else every lane looks up its rows' pages, one load behind the other; pages of 16 or 64 and of 8 positions: the 31 sequences
// above 116.5 and 209 us, the one of 131071 28.5 and 42, 61 of 1400 31 and 54)
template <int QP, int KW, int VD, bool PAGED16>
__global__ __launch_bounds__(FOUR_THREADS, KW <= 4 && VD <= 8 && QP == 1 && PAGED16 ? 3 : KW == 8 && QP == 3 ? 1 : 2)
void attend_fourbit_kernel(AttendFourbitArgs a, FourPlan pl)
{
    constexpr bool BF16 = QP == 1;
    constexpr int VW = VD >= 8 ? VD / 8 : 1;     // 4-byte words of a value in a lane (of 4 dimensions: half of one)
    constexpr int OD = VD < 8 ? VD : 8;          // dimensions of a lane that are joined at a time
    __shared__ __attribute__((aligned(16))) f32x4 lds_o[FOUR_WAVES][OD][64];
    __shared__ float wave_m[FOUR_WAVES][16], wave_l[FOUR_WAVES][16];
    __shared__ uint32_t after[SEQUENCES];        // units up to the end of each sequence
    __shared__ uint32_t wave_units[FOUR_WAVES], first_sequence;

    // Eight neighbours run on eight XCDs: where there are enough spans, the columns of one, whose rows share cache lines or are the
    // same, are put on one (8 heads side by side in a page's slots: 126 -> 100 us).
    const CacheView& cv = a.a.c;
    const uint32_t item = blockIdx.x, group = pl.spans < 8 ? item : item / 8;
    uint32_t span = group / (uint32_t)pl.columns;
    const int column = (int)(group - span * pl.columns), kvh = pl.head_blocks == 1 ? column : column / pl.head_blocks, hb = column - kvh * pl.head_blocks;
    if (pl.spans >= 8) span = span * 8 + item % 8;
    if (span >= (uint32_t)pl.spans) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, g = lane >> 4;
    const int* lengths = a.a.lengths + pl.b0;
    const int* starts = a.a.starts ? a.a.starts + pl.b0 : nullptr;

    // where the span begins
    uint32_t total;
    if (pl.n == 1) {
        const int len = clamped_length(lengths, 0, a.a.max_len), start = starts && starts[0] > 0 ? starts[0] : 0;
        total = units_of(start, len);
        if (threadIdx.x == 0) { after[0] = total; first_sequence = 0; }
    } else {
        const int per = (pl.n + FOUR_THREADS - 1) / FOUR_THREADS;            // sequences of a thread, up to 4
        uint32_t mine[SEQUENCES / FOUR_THREADS], sum = 0;
#pragma unroll
        for (int i = 0; i < SEQUENCES / FOUR_THREADS; ++i) {
            const int b = threadIdx.x * per + i;
            mine[i] = i < per && b < pl.n ? units_of(starts && starts[b] > 0 ? starts[b] : 0, clamped_length(lengths, b, a.a.max_len)) : 0u;
            sum += mine[i];
        }
        uint32_t upto = sum;
        for (int s = 1; s < 64; s <<= 1) {
            const uint32_t o = __shfl_up(upto, s, 64);
            if (lane >= s) upto += o;
        }
        if (lane == 63) wave_units[wave] = upto;
        __syncthreads();
        total = 0;
        uint32_t at = upto - sum;
#pragma unroll
        for (int w = 0; w < FOUR_WAVES; ++w) {
            at += w < wave ? wave_units[w] : 0u;
            total += wave_units[w];
        }
        const uint32_t begin = span * span_units(total, pl);
#pragma unroll
        for (int i = 0; i < SEQUENCES / FOUR_THREADS; ++i) {
            const int b = threadIdx.x * per + i;
            if (i >= per || b >= pl.n) break;
            if (at <= begin && begin < at + mine[i]) first_sequence = b;
            at += mine[i];
            after[b] = at;
        }
    }
    __syncthreads();
    if (item == 0 && pl.before)
        for (int i = threadIdx.x; i <= pl.n; i += FOUR_THREADS) pl.before[i] = i == 0 ? 0u : after[i - 1];
    const uint32_t span_size = span_units(total, pl), span_end = min((span + 1) * span_size, total);
    if (span * span_size >= total) return;

    const int h = hb * 16 + m;                   // the lane's head, of the group
    const int slots = (1 << cv.page_shift) - 1;
    const int kblocks = cv.Dk / 32, vblocks = cv.Dv / 32;
    // of this head: codes of page 0, scale bytes of page 0, and how far apart two pages' scale bytes are
    const unsigned char* kbase = cv.k + kvh * cv.k_head;
    const unsigned char* vbase = cv.v + kvh * cv.v_head;
    const uint8_t* kscales = a.k_scales + ((long long)(kvh * kblocks) << cv.page_shift);
    const uint8_t* vscales = a.v_scales + ((long long)(kvh * vblocks) << cv.page_shift);
    const long long kscales_page = (long long)(cv.Hkv * kblocks) << cv.page_shift, vscales_page = (long long)(cv.Hkv * vblocks) << cv.page_shift;
    // Lane (m, g) holds key m's words of dimensions g KD .. g KD + 8 KW - 1 (KW = 8: 32 of them, and 32 that lie 128 further), all of
    // one scale byte (KW = 8: of two).  Pieces past a row's end are read from its beginning; queries are 0 there, and what it makes of
    // values is not stored.
    constexpr int KD = KW <= 4 ? 8 * KW : 32, KU = KW <= 4 ? 1 : 2;
    uint32_t k_at[KU], ks_at[KU];
#pragma unroll
    for (int u = 0; u < KU; ++u) {
        const int d = g * KD + u * 128 < cv.Dk ? g * KD + u * 128 : 0;
        k_at[u] = d / 2 + (PAGED16 ? m * (uint32_t)cv.k_slot : 0u);
        ks_at[u] = ((uint32_t)(d / 32) << cv.page_shift) + (PAGED16 ? m : 0);
    }
    const int v_d = m * VD < cv.Dv ? m * VD : 0;
    const uint32_t v_at = v_d / 2 + (PAGED16 ? 4 * g * (uint32_t)cv.v_slot : 0u), vs_at = ((uint32_t)(v_d / 32) << cv.page_shift) + (PAGED16 ? 4 * g : 0);
    const float scale = fabsf(a.a.scale);
    uint32_t minus_first = 0x0000BF80u, minus_second = 0xBF800000u;
    asm("" : "+s"(minus_first), "+s"(minus_second));

    uint32_t at_unit = span * span_size;
    for (int sequence = __builtin_amdgcn_readfirstlane(first_sequence); at_unit < span_end; ++sequence) {
        const uint32_t from_unit = sequence == 0 ? 0u : __builtin_amdgcn_readfirstlane(after[sequence - 1]);
        const uint32_t to_unit = __builtin_amdgcn_readfirstlane(after[sequence]);
        const uint32_t stop_unit = min(to_unit, span_end);
        const int len = clamped_length(lengths, sequence, a.a.max_len), start = starts && starts[sequence] > 0 ? starts[sequence] : 0;
        const int begin = (start & ~15) + (int)(at_unit - from_unit) * UNIT;
        const int end = (int)min((long long)(start & ~15) + (long long)(stop_unit - from_unit) * UNIT, (long long)len);      // (below begin: nothing)
        const bool cut = from_unit < span * span_size || to_unit > span_end;
        const long long part = (((long long)column * pl.spans + span) * 2 + (from_unit < span * span_size ? 0 : 1));
        const int b = pl.b0 + sequence;
        const long long hq = (long long)b * a.a.Hq + kvh * pl.G + h;
        const int32_t* table = cv.table + (long long)b * cv.max_pages;
        at_unit = stop_unit;

        // queries: operand B, zeros past Dk and past the group
        u32x4 qf[KW][QP];
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            const int d = g * KD + (w & 3) * 8 + (w >> 2) * 128;
            u32x4 x[BF16 ? 1 : 2] = {};
            if (h < pl.G && d < cv.Dk) {
                const unsigned char* q = (const unsigned char*)a.a.q + b * a.a.q_seq + (long long)(kvh * pl.G + h) * a.a.q_head + (BF16 ? 2 : 4) * d;
#pragma unroll
                for (int i = 0; i < (BF16 ? 1 : 2); ++i) x[i] = *(const u32x4*)(q + 16 * i);
            }
            // the sign of the scale goes into the queries: the largest score is that of the largest product
            if (a.a.scale < 0.0f)
#pragma unroll
                for (int i = 0; i < (BF16 ? 1 : 2); ++i) x[i] ^= BF16 ? 0x80008000u : 0x80000000u;
            if constexpr (BF16) {
                qf[w][0] = x[0];
            } else {
                // three times the upper 16 bits of what is left: 24 bits, all of an fp32 number (an infinite one and NaN are their first part)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t left[2] = {x[i >> 1][2 * (i & 1)], x[i >> 1][2 * (i & 1) + 1]};
#pragma unroll
                    for (int j = 0; j < 2; ++j) left[j] = (left[j] & 0x7FFFFFFFu) > 0x7F800000u ? 0x7FC00000u : left[j];
#pragma unroll
                    for (int u = 0; u < QP; ++u) {
                        qf[w][u][i] = __builtin_amdgcn_perm(left[1], left[0], 0x07060302u);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const float hi = __uint_as_float(left[j] & 0xFFFF0000u);
                            left[j] = __builtin_isfinite(hi) ? __float_as_uint(__uint_as_float(left[j]) - hi) : 0u;
                        }
                    }
                }
            }
        }

        // All of the piece, its results written.  True where it has to be done again, SPECIAL.
        // Otherwise scores are in units of log2, one multiplication and addition away from the products.
        auto run = [&](auto special_c) {
            constexpr bool SPECIAL = decltype(special_c)::value;
            constexpr float unit = SPECIAL ? 0x1p-32f : 1.0f;    // what an exponential of 0 counts as
            constexpr float NEAR = SPECIAL ? 8.0f : 8.0f * LOG2E;
            const float by_scale = SPECIAL ? scale : scale * LOG2E;
            auto power = [&](float v) { return SPECIAL ? exp_(v) : __builtin_amdgcn_exp2f(v); };       // of differences of scores
            f32x4 o[VD];
            float top = -__builtin_inff(), sum = 0.0f;           // the exponentials' reference point
#pragma unroll
            for (int j = 0; j < VD; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (begin < end) {
                // A tile's keys are requested when the one before is multiplied, its values likewise.
                struct Tile {
                    uint32_t kf[2][KW], ks[2][KU];   // keys of both halves, their scale bytes
                    uint32_t vf[8][VW], vs[2];       // values of the lane's 8 positions, 4g .. 4g + 3 of each half, and their scale bytes
                    int page[2];                     // PAGED16: the halves' pages, -1 for none
                    uint32_t live;                   // else: which of the 8 positions take part
                } t;

                // Rows that do not take part (before the start, past the end, on no page) are read from a slot that exists.
                const int last_entry = (end - 1) >> cv.page_shift;
                auto valid = [&](int e) { return (uint32_t)e < (uint32_t)cv.n_pages ? e : -1; };
                auto own_entry = [&](int pos) { return valid(table[min(pos >> cv.page_shift, last_entry)]); };
                auto takes_part = [&](int pos, int page) { return (int)(pos >= start) & (int)(pos < end) & (int)(page >= 0); };
                struct Entries { int e[2]; };        // PAGED16: of the page table, for the two halves of a tile
                auto find = [&](int p) {
                    Entries f = {};
                    if constexpr (PAGED16)
#pragma unroll
                        for (int i = 0; i < 2; ++i) f.e[i] = uniform_entry(table, min((p + 16 * i) >> cv.page_shift, last_entry));
                    return f;
                };
                auto load_k = [&](int p, const Entries& f) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if constexpr (PAGED16) {
                            t.page[i] = valid(f.e[i]);
                            const int page = max(t.page[i], 0), slot = (p + 16 * i) & slots;
#pragma unroll
                            for (int u = 0; u < KU; ++u) {
                                load_at<KW == 2 ? 2 : 4>(kbase + page * cv.k_page + slot * cv.k_slot, k_at[u], 0, t.kf[i] + 4 * u);
                                load_at<-1>(kscales + page * kscales_page + slot, ks_at[u], 0, t.ks[i] + u);
                            }
                        } else {
                            const int pos = p + 16 * i + m, e = own_entry(pos), page = max(e, 0), slot = e < 0 ? 0 : pos & slots;
#pragma unroll
                            for (int u = 0; u < KU; ++u) {
                                load_own<KW == 2 ? 2 : 4>(kbase + page * cv.k_page + slot * cv.k_slot + k_at[u], t.kf[i] + 4 * u);
                                load_own<-1>(kscales + page * kscales_page + slot + ks_at[u], t.ks[i] + u);
                            }
                        }
                    }
                };
                auto load_v = [&](int p) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if constexpr (PAGED16) {
                            const int page = max(t.page[i], 0), slot = (p + 16 * i) & slots;
#pragma unroll
                            for (int j = 0; j < 4; ++j) load_at<VD / 8>(vbase + page * cv.v_page + slot * cv.v_slot, v_at, j * (uint32_t)cv.v_slot, t.vf[4 * i + j]);
                            load_at<1>(vscales + page * vscales_page + slot, vs_at, 0, t.vs + i);
                        } else {
                            t.vs[i] = 0;
                            if (i == 0) t.live = 0;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int pos = p + 16 * i + 4 * g + j, e = own_entry(pos), page = max(e, 0), slot = e < 0 ? 0 : pos & slots;
                                load_own<VD / 8>(vbase + page * cv.v_page + slot * cv.v_slot + v_at, t.vf[4 * i + j]);
                                t.live |= takes_part(pos, e) << (4 * i + j);
                                t.vs[i] |= (uint32_t)(vscales + page * vscales_page + slot)[vs_at] << (8 * j);
                            }
                        }
                    }
                };

                Entries ahead;
                auto step = [&](int p) {
                    f32x4 s[2];
                    s[0] = s[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < KW; ++w) {
                        u32x4 x[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float by = __uint_as_float(t.ks[i][w >> 2] << 23);
                            x[i] = u32x4{pair_bf16<0>(t.kf[i][w], by), pair_bf16<1>(t.kf[i][w], by), pair_bf16<2>(t.kf[i][w], by), pair_bf16<3>(t.kf[i][w], by)};
                        }
#pragma unroll
                        for (int u = QP - 1; u >= 0; --u)
#pragma unroll
                            for (int i = 0; i < 2; ++i) s[i] = mfma32(x[i], qf[w][u], s[i]);      // (neighbours that do not wait for each other)
                    }
                    const bool whole = PAGED16 ? (t.page[0] | t.page[1]) >= 0 && p >= start && p + FOUR_TILE <= end : __all(t.live == 255u);
                    uint32_t now = t.live;
                    if (PAGED16 && !whole) {
                        now = 0;
#pragma unroll
                        for (int j = 0; j < 8; ++j) now |= takes_part(p + 16 * (j >> 2) + 4 * g + (j & 3), t.page[j >> 2]) << j;
                    }
                    load_k(p + UNIT, ahead);
                    ahead = find(p + 2 * UNIT);
                    __builtin_amdgcn_sched_barrier(0);           // requested here, not where they are used

                    float z[8], most;
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] = SPECIAL ? s[j >> 2][j & 3] * by_scale : s[j >> 2][j & 3];
                    if (!whole) {
                        // what stands in a row that does not take part may be anything: no NaN of it may reach the sums
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            z[j] = (now >> j) & 1u ? z[j] : -__builtin_inff();
                            t.vs[j >> 2] = (now >> j) & 1u ? t.vs[j >> 2] : (t.vs[j >> 2] & ~(255u << (8 * (j & 3)))) | 127u << (8 * (j & 3));
                        }
                    }
                    most = fmaxf(fmaxf(z[0], z[1]), z[2]);
#pragma unroll
                    for (int j = 3; j < 8; ++j) most = fmaxf(most, z[j]);
                    if constexpr (!SPECIAL) most *= by_scale;
                    // The reference point need not be the maximum: it is moved where a score is more than 8 above it.
                    if (__any(most > top + NEAR)) {
                        most = across_groups_max(most);
                        const float higher = fmaxf(top, most), keep = power(top - origin(higher));
                        top = higher;
                        sum *= keep;
#pragma unroll
                        for (int j = 0; j < VD; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[j][i] *= keep;
                    }
                    const float at = origin(top);
                    float e[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        e[j] = SPECIAL ? exp_(z[j] - at) * unit : __builtin_amdgcn_exp2f(fmaf(z[j], by_scale, -at));
                        sum += e[j];
                    }
                    u32x4 prob[3];                   // P: the nearest bf16 numbers, the nearest to what is left, and what then is left
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float left[2] = {e[2 * i], e[2 * i + 1]};
#pragma unroll
                        for (int u = 0; u < 3; ++u) {
                            const uint32_t both = pack_bf16x2(left[0], left[1]);
                            prob[u][i] = both;
                            left[0] = less_one(left[0], both, minus_first);
                            left[1] = less_one(left[1], both, minus_second);
                        }
                    }
                    float by[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) by[j] = __uint_as_float((j & 3) < 3 ? t.vs[j >> 2] << (23 - 8 * (j & 3)) : t.vs[j >> 2] >> 1);    // (the exponent's bits count)
                    // two dimensions of all 8 positions at a time: the pairs of one position become pairs of neighbouring positions
                    auto add = [&](auto byte_c) {
                        constexpr int B = decltype(byte_c)::value;
#pragma unroll
                        for (int w = 0; w < VW; ++w) {
                            uint32_t y[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) y[j] = pair_bf16<B>(t.vf[j][w], by[j]);
                            u32x4 x[2];
#pragma unroll
                            for (int half = 0; half < 2; ++half)
#pragma unroll
                                for (int i = 0; i < 4; ++i) x[half][i] = __builtin_amdgcn_perm(y[2 * i + 1], y[2 * i], half ? 0x07060302u : 0x05040100u);
#pragma unroll
                            for (int u = 0; u < 3; ++u)
#pragma unroll
                                for (int half = 0; half < 2; ++half) o[8 * w + 2 * B + half] = mfma32(x[half], prob[u], o[8 * w + 2 * B + half]);
                        }
                    };
                    add(std::integral_constant<int, 0>{});
                    add(std::integral_constant<int, 1>{});
                    if constexpr (VD > 4) {
                        add(std::integral_constant<int, 2>{});
                        add(std::integral_constant<int, 3>{});
                    }
                    load_v(p + UNIT);
                    __builtin_amdgcn_sched_barrier(0);           // here, not at the top of the next step
                };

                const int p0 = begin + wave * FOUR_TILE;
                ahead = find(p0);
                load_k(p0, ahead);
                ahead = find(p0 + UNIT);
                __builtin_amdgcn_sched_barrier(0);               // in this order here too: what is waited for first is requested first
                load_v(p0);
                __builtin_amdgcn_sched_barrier(0);
                for (int p = p0; p < end; p += UNIT) step(p);
            }

            // the four waves' results: o[j][i] of lane (m, g) is head m, dimension (4g + i) * VD + j
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (g == 0) {
                wave_m[wave][m] = top;
                wave_l[wave][m] = sum;
            }
            __syncthreads();
            float all = wave_m[0][m], whole_sum = 0.0f;
#pragma unroll
            for (int w = 1; w < FOUR_WAVES; ++w) all = fmaxf(all, wave_m[w][m]);
#pragma unroll
            for (int w = 0; w < FOUR_WAVES; ++w) whole_sum += wave_l[w][m] * power(wave_m[w][m] - origin(all));
            const float mine = power(top - origin(all));
            const float by = whole_sum == 0.0f ? 0.0f : 1.0f / whole_sum;    // no position, or none above -infinity: zeros
            // no weight at all, or scores past the range of this form
            bool odd = begin < end && (!(whole_sum > 0.0f) || fabsf(all) > FARTHEST);
            if (wave == 0 && g == 0 && h < pl.G) {
                // the reference point as a natural exponent; what its rounding leaves goes into the sum
                const float ref = SPECIAL || all == -__builtin_inff() ? all : all * LN2;
                const float rest = SPECIAL || all == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(fmaf(-ref, LOG2E_REST, fmaf(-ref, LOG2E, all)));
                if (cut) pl.ml[part * 16 + m] = make_float2(ref, whole_sum * rest / unit);
                else if (a.a.lse) a.a.lse[hq] = origin(ref) + __log2f(whole_sum * rest / unit) * LN2;
            }
#pragma unroll
            for (int j0 = 0; j0 < VD; j0 += OD) {
                if (j0 > 0) __syncthreads();
#pragma unroll
                for (int j = 0; j < OD; ++j) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[j0 + j][i] *= mine;
                    lds_o[wave][j][lane] = o[j0 + j];
                }
                __syncthreads();
                // wave w adds up OD / 4 neighbouring dimensions
                constexpr int MINE = OD / 4;
                f32x4 v[MINE];
#pragma unroll
                for (int u = 0; u < MINE; ++u) {
                    const int j = wave * MINE + u;
                    v[u] = ((lds_o[0][j][lane] + lds_o[1][j][lane]) + (lds_o[2][j][lane] + lds_o[3][j][lane]));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[u][i] = by == 0.0f ? 0.0f : v[u][i] * by;
                        odd = odd || !__builtin_isfinite(v[u][i]);
                    }
                }
                if (h >= pl.G) continue;
                if (cut) {
#pragma unroll
                    for (int u = 0; u < MINE; ++u) pl.o[(part * VD + j0 + wave * MINE + u) * 64 + lane] = v[u];
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int d = (4 * g + i) * VD + j0 + wave * MINE;
                        if (d >= cv.Dv) continue;
                        if constexpr (BF16) {
                            uint16_t* to = (uint16_t*)a.a.out + hq * cv.Dv + d;
                            if constexpr (MINE == 2) *(uint32_t*)to = pack_bf16x2(v[0][i], v[1][i]);
                            else *to = f32_to_bf16_bits(v[0][i]);
                        } else {
                            float* to = (float*)a.a.out + hq * cv.Dv + d;
#pragma unroll
                            for (int u = 0; u < MINE; ++u) to[u] = v[u][i];
                        }
                    }
                }
            }
            return odd;
        };
        // Scores in units of log2 may be past the largest number where they are not, and the sum over up to 2^31 values may where their
        // average is not: a piece whose results are not finite, that has no weight, or whose scores are past FARTHEST, is done again, with
        // scores as they are and 2^-32 of each term.  That is the only way where the scale is below the normal numbers: by 0 the scores of
        // rows that take part are equal, and those of the others have to be -infinity all the same.
        const bool odd = scale < 0x1p-126f || run(std::false_type{});
        if (__builtin_expect(__syncthreads_or(odd), 0)) run(std::true_type{});
    }
}

// ---------------------------------------------------------------------------

static constexpr int FOUR_JOIN_THREADS = 256, FOUR_JOIN_WAVES = FOUR_JOIN_THREADS / 64;
static constexpr int PIECES = 256;               // at a time
static constexpr int EACH = PIECES / (FOUR_JOIN_THREADS / 16);

// A workgroup joins the pieces of one sequence at one block of query heads, for 2 of the dimensions of each lane.
template <bool BF16, int VD>
__global__ __launch_bounds__(FOUR_JOIN_THREADS) void attend_fourbit_join_kernel(AttendFourbitArgs a, FourPlan pl)
{
    constexpr int GROUPS = VD / 2;
    __shared__ float2 wave_ml[FOUR_JOIN_WAVES][16];
    __shared__ float weight[PIECES][16];
    __shared__ __attribute__((aligned(16))) f32x4 sums[FOUR_JOIN_WAVES][2][64];
    const uint32_t rest = blockIdx.x / GROUPS, group = blockIdx.x % GROUPS;
    const int sequence = (int)(rest / (uint32_t)pl.columns), column = (int)(rest - sequence * pl.columns);
    const uint32_t from = pl.before[sequence], to = pl.before[sequence + 1], size = span_units(pl.before[pl.n], pl);
    const int first = (int)(from / size), last = (int)((to - 1) / size);
    if (first == last) return;                   // written already
    const int n = last - first + 1;
    const long long base = (long long)column * pl.spans + first;
    auto piece = [&](int c) { return (base + c) * 2 + (c == 0 ? 1 : 0); };

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = tid & 15;
    const int kvh = column / pl.head_blocks, h = column % pl.head_blocks * 16 + m;
    // each wave adds up every fourth piece, BATCH of them requested together
    constexpr int BATCH = 8;
    f32x4 x[BATCH], y[BATCH];
    auto request = [&](int i0, int stop) {
#pragma unroll
        for (int r = 0; r < BATCH; ++r) {
            const int i = i0 + r * FOUR_JOIN_WAVES;
            if (i >= stop) break;
            const f32x4* o = pl.o + (piece(i) * VD + group * 2) * 64 + (h < pl.G ? lane : lane & 48);
            x[r] = o[0];
            y[r] = o[64];
        }
    };
    // reference point and sum of every head: thread (head, c) takes pieces c, c + 16, ...
    float top = -__builtin_inff(), total = 0.0f;
    float2 v[EACH];
    auto load = [&](int c0) {
#pragma unroll
        for (int r = 0; r < EACH; ++r) {
            const int c = c0 + (tid >> 4) + r * (FOUR_JOIN_THREADS / 16);
            v[r] = c < n ? pl.ml[piece(c) * 16 + m] : make_float2(-__builtin_inff(), 0.0f);
        }
    };
    auto fold = [&](float ref, float l) {
        const float higher = fmaxf(top, ref);
        total = total * exp_(top - origin(higher)) + l * exp_(ref - origin(higher));
        top = higher;
    };
    for (int c0 = 0; c0 < n; c0 += PIECES) {
        load(c0);
        float higher = top;
#pragma unroll
        for (int r = 0; r < EACH; ++r) higher = fmaxf(higher, v[r].x);
        total *= exp_(top - origin(higher));
        top = higher;
#pragma unroll
        for (int r = 0; r < EACH; ++r) total += v[r].y * exp_(v[r].x - origin(top));
    }
    for (int mask = 16; mask < 64; mask <<= 1) {
        const float o = __shfl_xor(top, mask, 64), l = __shfl_xor(total, mask, 64);
        fold(o, l);
    }
    if (lane < 16) wave_ml[wave][lane] = make_float2(top, total);
    __syncthreads();
    top = -__builtin_inff();
    total = 0.0f;
#pragma unroll
    for (int w = 0; w < FOUR_JOIN_WAVES; ++w) fold(wave_ml[w][m].x, wave_ml[w][m].y);
    const float at = origin(top), by = total == 0.0f ? 0.0f : 1.0f / total;

    const long long hq = (long long)(pl.b0 + sequence) * a.a.Hq + kvh * pl.G + h;
    if (group == 0 && tid < 16 && a.a.lse && h < pl.G) a.a.lse[hq] = at + __log2f(total) * LN2;
    f32x4 acc[2] = {};
    for (int c0 = 0; c0 < n; c0 += PIECES) {
        if (c0 > 0) __syncthreads();
        if (n > PIECES) load(c0);
#pragma unroll
        for (int r = 0; r < EACH; ++r) weight[(tid >> 4) + r * (FOUR_JOIN_THREADS / 16)][m] = exp_(v[r].x - at) * v[r].y * by;
        __syncthreads();
        const int stop = min(n, c0 + PIECES);
        for (int i0 = c0 + wave; i0 < stop; i0 += BATCH * FOUR_JOIN_WAVES) {
            request(i0, stop);
#pragma unroll
            for (int r = 0; r < BATCH; ++r) {
                const int i = i0 + r * FOUR_JOIN_WAVES;
                if (i >= stop) break;
                const float w = weight[i - c0][m];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    acc[0][u] = fmaf(x[r][u], w, acc[0][u]);
                    acc[1][u] = fmaf(y[r][u], w, acc[1][u]);
                }
            }
        }
    }
    sums[wave][0][lane] = acc[0];
    sums[wave][1][lane] = acc[1];
    __syncthreads();
    // thread (lane, i): two neighbouring dimensions, (4g + i) * VD + 2 group ..
    const int d = (4 * (lane >> 4) + wave) * VD + group * 2;
    if (h >= pl.G || d >= a.a.c.Dv) return;
    float out[2] = {};
#pragma unroll
    for (int w = 0; w < FOUR_JOIN_WAVES; ++w)
#pragma unroll
        for (int u = 0; u < 2; ++u) out[u] += sums[w][u][lane][wave];
    if constexpr (BF16) *(uint32_t*)((uint16_t*)a.a.out + hq * a.a.c.Dv + d) = pack_bf16x2(out[0], out[1]);
    else *(float2*)((float*)a.a.out + hq * a.a.c.Dv + d) = make_float2(out[0], out[1]);
}

// ---------------------------------------------------------------------------

static int value_dims(int Dk, int Dv) { return Dk <= 64 && Dv <= 64 ? 4 : Dv <= 128 ? 8 : 16; }        // of a lane

static long long most_units(const AttendFourbitArgs& a) { return a.a.max_len > 0 ? (a.a.max_len + 15ll + UNIT - 1) / UNIT : 1; }      // of a sequence
static FourPlan plan_of(const AttendFourbitArgs& a)
{
    FourPlan pl{};
    pl.G = a.a.Hq / a.a.c.Hkv;
    pl.head_blocks = (pl.G + 15) / 16;
    pl.columns = a.a.c.Hkv * pl.head_blocks;
    pl.enough = ENOUGH_SPANS / pl.columns > 1 ? ENOUGH_SPANS / pl.columns : 1;
    const long long spans = MOST_SPANS / pl.columns > 1 ? MOST_SPANS / pl.columns : 1, filled = (a.a.c.B * most_units(a) + LEAST_UNITS - 1) / LEAST_UNITS;
    pl.spans = (int)(filled < 1 ? 1 : filled < spans ? filled : spans);
    return pl;
}
// sequences of a launch: the spans' units have 31 bits
static int most_sequences(const AttendFourbitArgs& a)
{
    const long long n = (1ll << 30) / most_units(a);
    return n < SEQUENCES ? (int)n : SEQUENCES;
}
// whether a sequence can be cut at all
static bool may_cut(const AttendFourbitArgs& a)
{
    return a.a.max_len + 15 > UNIT * (a.a.c.B > 1 ? 1 : LEAST_UNITS);
}

bool attend_fourbit_fits(const AttendFourbitArgs& a)
{
    return (long long)a.a.c.B * a.a.c.Hkv < (1ll << 23) && (long long)a.a.c.B * a.a.Hq < (1ll << 23);
}

static size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

// Never less for a longer cache or a larger batch: one workspace serves every step's own.
size_t attend_fourbit_workspace_bytes(const AttendFourbitArgs& a)
{
    const FourPlan pl = plan_of(a);
    const size_t parts = (size_t)pl.columns * pl.spans * 2;
    return a.a.c.B > 0 && may_cut(a) ? up16((SEQUENCES + 1) * 4) + parts * (value_dims(a.a.c.Dk, a.a.c.Dv) * 1024 + 128) : 0;
}

template <int QP, bool PAGED16> static auto kernel_of(int Dk, int Dv)
{
    if (Dk <= 64) return Dv <= 64 ? attend_fourbit_kernel<QP, 2, 4, PAGED16> : Dv <= 128 ? attend_fourbit_kernel<QP, 2, 8, PAGED16> : attend_fourbit_kernel<QP, 2, 16, PAGED16>;
    if (Dk <= 128) return Dv <= 128 ? attend_fourbit_kernel<QP, 4, 8, PAGED16> : attend_fourbit_kernel<QP, 4, 16, PAGED16>;
    return Dv <= 128 ? attend_fourbit_kernel<QP, 8, 8, PAGED16> : attend_fourbit_kernel<QP, 8, 16, PAGED16>;
}
template <bool BF16> static auto join_of(int vd)
{
    return vd == 4 ? attend_fourbit_join_kernel<BF16, 4> : vd == 8 ? attend_fourbit_join_kernel<BF16, 8> : attend_fourbit_join_kernel<BF16, 16>;
}

hipError_t launch_attend_fourbit(const AttendFourbitArgs& a)
{
    const CacheView& c = a.a.c;
    FourPlan pl = plan_of(a);
    const int vd = value_dims(c.Dk, c.Dv);
    const size_t parts = (size_t)pl.columns * pl.spans * 2;
    if (may_cut(a)) {
        unsigned char* ws = (unsigned char*)a.a.workspace;
        pl.before = (uint32_t*)ws;
        pl.o = (f32x4*)(ws + up16((SEQUENCES + 1) * 4));
        pl.ml = (float2*)(pl.o + parts * vd * 64);
    }
    // (a lane's offset from the first of 16 rows has 31 bits)
    const bool paged16 = c.page_shift >= 4 && c.k_slot < (1 << 26) && c.v_slot < (1 << 26);
    const auto kern = c.dtype == 1 ? (paged16 ? kernel_of<1, true>(c.Dk, c.Dv) : kernel_of<1, false>(c.Dk, c.Dv))
                                   : (paged16 ? kernel_of<3, true>(c.Dk, c.Dv) : kernel_of<3, false>(c.Dk, c.Dv));
    const auto join = c.dtype == 1 ? join_of<true>(vd) : join_of<false>(vd);
    for (int b0 = 0; b0 < c.B; b0 += most_sequences(a)) {
        pl.b0 = b0;
        pl.n = c.B - b0 < most_sequences(a) ? c.B - b0 : most_sequences(a);
        hipLaunchKernelGGL(kern, dim3((unsigned)((pl.spans < 8 ? pl.spans : (pl.spans + 7) / 8 * 8) * pl.columns)), dim3(FOUR_THREADS), 0, a.a.stream, a, pl);
        hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
        if (!may_cut(a)) continue;
        hipLaunchKernelGGL(join, dim3((unsigned)(pl.n * pl.columns * (vd / 2))), dim3(FOUR_JOIN_THREADS), 0, a.a.stream, a, pl);
        err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace paep
