// Attention of one new token per sequence over a paged key-value cache.
//
//   s = scale q k^T,  P = exp(s - max) / sum,  out = P V       one row of s per query head
//
// Every key and value is needed once by the G query heads that share it, so what bounds the operator is reading the cache.
// attend_kernel: a workgroup of four waves takes one chunk of one sequence's positions at one key-value head, for up to 16 of
// its query heads; a wave takes every fourth tile of 16 positions.  Keys and values go from memory straight into the
// registers of the matrix instructions, no LDS in between:
//   S^T = K Q^T   a wave's operand A is 16 keys, lane (m, g) holding 16 bytes of key m: four lanes fetch 64 contiguous bytes.
//                 Lane (m, g) of the result holds head m's scores of keys 4g .. 4g + 3, which is operand B of the second
//                 product as it stands:
//   O^T = V^T P^T operand A wants 4 keys of one dimension in a lane.  Lane (c, g) fetches dimensions 8c .. 8c + 7 of the
//                 4 keys that its lane group g holds (16 lanes read a whole row), and one byte permutation per register
//                 transposes the block inside the lane.  Row c of the j-th of 8 products is dimension 8c + j.
// (fp32 storage: the same with 16-byte pieces of 4 and the 16x16x4 instruction, key by key.)  The running maximum and sum are
// per lane, one head each, and the accumulated O is rescaled in place, where a maximum grew, without any exchange between
// lanes.  P is multiplied as three bf16 parts, 24 bits, all that an fp32 number has: with two of them, 16 bits, the outcome of
// sums that cancel had fewer right bits than its storage, and the third instruction costs nothing next to the loads (the
// cases below: 0.2 % at most).
// The next tile's keys are requested once this tile's are multiplied, the next values likewise, so that a wave always has a
// tile in flight.  Tiles of 16 positions, not of 32, leave registers for three workgroups on a CU instead of two (when taken,
// 131071 positions 58 -> 56 us, 32 heads on one key-value head of width 256 56 -> 48 us), and one block of 16 query heads to a
// workgroup, not two, for two (likewise, 32 heads of width 256 94 -> 55 us, of width 128 32 -> 25 us).  Waves are joined in LDS, chunks by
// attend_join_kernel, in a fixed order.
// A chunk whose results are not all finite is done a second time, in a form for infinite values and sums past the largest
// number; looking whether they are costs 0.4 us of a call.
// Measured: 131071 positions of 4 key-value heads of 128 57 us (4.7 TB/s, 5.2 without the join's launch); 61 sequences of
// 17 to 8192 positions, 8 heads, with mass 104 us; fp32, 5 sequences of up to 4096 positions, 3 heads of 80, 18 us.
#include <type_traits>

#include "attend_device.h"

namespace paep {

static constexpr int ATT_THREADS = 256, ATT_WAVES = ATT_THREADS / 64;
static constexpr int TILE = 16;                  // positions of a wave at a time
static constexpr int TABLE = 2048;               // page-table entries in LDS at a time

struct AttendPlan {
    int G, head_blocks;          // query heads of a key-value head, blocks of 16 of them
    int chunk, S;                // positions of a workgroup, chunks of the longest sequence
    int rows;                    // B * Hkv
    float* o;                    // [rows][S][G][Dv] outputs of the chunks, each over its own sum (S > 1)
    float2* ml;                  // [rows][S][G] the maxima of their scores, and their sums (S > 1 or mass)
    float* scores;               // [rows][S][G][chunk] (mass)
};

// the part of a sequence that is looked at: positions start .. len, counted in chunks from start rounded down to a multiple of 16
struct Range { int start, first, len, chunks; };
__device__ __forceinline__ Range range_of(const int32_t* lengths, const int32_t* starts, int b, int max_len, int chunk)
{
    Range r;
    r.len = clamped_length(lengths, b, max_len);
    r.start = starts && starts[b] > 0 ? starts[b] : 0;
    r.first = r.start & ~15;
    r.chunks = r.start < r.len ? (int)(((uint32_t)(r.len - r.first) + (uint32_t)chunk - 1) / (uint32_t)chunk) : 0;
    return r;
}

// 16 x 16 products of two operands of 16 rows x 64 bytes
template <bool BF16> __device__ __forceinline__ f32x4 product(const u32x4& x, const u32x4& y, f32x4 acc)
{
    if constexpr (BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[i]), __uint_as_float(y[i]), acc, 0, 0, 0);
        return acc;
    }
}

// two bf16 numbers, 0 in place of an infinite one or NaN
__device__ __forceinline__ uint32_t finite_halves(uint32_t v)
{
    return ((v & 0x7F80u) == 0x7F80u ? 0u : v & 0xFFFFu) | ((v & 0x7F800000u) == 0x7F800000u ? 0u : v & 0xFFFF0000u);
}

// KS: 16-byte steps of four lanes that cover a key; VB: blocks of 16 lanes x 16 bytes that cover a value;
// MASS: the scores are kept for attend_join_kernel
template <bool BF16, int KS, int VB, bool MASS>
__global__ __launch_bounds__(ATT_THREADS, BF16 ? (VB == 1 && KS <= 4 ? 3 : 2) : (VB == 2 && KS <= 8 ? 2 : 1)) void attend_kernel(AttendArgs a, AttendPlan pl)
{
    constexpr int PER = BF16 ? 8 : 4;            // elements of a 16-byte piece
    __shared__ __attribute__((aligned(16))) union {
        int pages[TABLE + 1];                    // while the positions are walked
        f32x4 o[ATT_WAVES][PER][64];             // the waves' results, a block of dimensions at a time
    } lds;
    __shared__ float wave_m[ATT_WAVES][16], wave_l[ATT_WAVES][16];

    const int item = blockIdx.x;
    // eight neighbours run on eight XCDs: the head blocks of one chunk, which read the same rows, are put on one
    const int hb = item / 8 % pl.head_blocks;
    const int rest = item / (8 * pl.head_blocks) * 8 + item % 8;
    if (rest >= pl.rows * pl.S) return;
    const int split = rest / pl.rows, row = rest % pl.rows;
    const int b = row / a.c.Hkv, kvh = row % a.c.Hkv;
    const Range r = range_of(a.lengths, a.starts, b, a.max_len, pl.chunk);
    if (split >= r.chunks && split > 0) return;  // the first workgroup of an empty range writes its zeros

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, g = lane >> 4;
    const long long lo = r.first + (long long)split * pl.chunk;
    const int begin = (int)lo, end = r.chunks == 0 ? begin : (int)(lo + pl.chunk < r.len ? lo + pl.chunk : r.len);

    const int h = hb * 16 + m;                   // the lane's head, of the group
    const long long hq = (long long)b * a.Hq + kvh * pl.G + h;

    // queries: operand B, lane (m, g): head m, piece ks * 4 + g; zeros past Dk and past the group
    u32x4 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = u32x4{0u, 0u, 0u, 0u};
        if (h < pl.G && (ks * 4 + g) * PER < a.c.Dk)
            qf[ks] = *(const u32x4*)((const unsigned char*)a.q + b * a.q_seq + (long long)(kvh * pl.G + h) * a.q_head + (ks * 4 + g) * 16);
    }

    const long long part = ((long long)row * pl.S + split) * pl.G + h;
    const int heads_here = min(pl.G - hb * 16, 16);
    const __amdgpu_buffer_rsrc_t kept = __builtin_amdgcn_make_buffer_rsrc(
        MASS ? (void*)(pl.scores + (((long long)row * pl.S + split) * pl.G + hb * 16) * pl.chunk) : nullptr, 0,
        MASS ? heads_here * pl.chunk * 4 : 0, 0x00020000);

    const unsigned char* kbase = a.c.k + kvh * a.c.k_head;
    const unsigned char* vbase = a.c.v + kvh * a.c.v_head;
    const int slots = (1 << a.c.page_shift) - 1;
    // All of the chunk, its results written.  True where one of this thread's is not finite.  SPECIAL: the values may be infinite or
    // NaN, or near the largest number.
    auto run = [&](auto special_c) {
        constexpr bool SPECIAL = decltype(special_c)::value;
        constexpr float unit = SPECIAL ? 0x1p-32f : 1.0f;    // what an exponential of 0 counts as
        f32x4 o[VB][PER];
        float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
        for (int vb = 0; vb < VB; ++vb)
#pragma unroll
            for (int j = 0; j < PER; ++j) o[vb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 kf[KS], vf[4][VB];
        uint32_t live = 0;                           // which of the lane's 4 keys take part

        const long long stretch = (long long)TABLE << a.c.page_shift;        // positions whose page-table entries fit in LDS
        for (long long p0 = begin; p0 < end; p0 += stretch) {
            const int stop = p0 + stretch < end ? (int)(p0 + stretch) : end;
            const int page0 = (int)p0 >> a.c.page_shift;
            __syncthreads();
            for (int i = threadIdx.x; i <= ((stop - 1) >> a.c.page_shift) - page0; i += ATT_THREADS)
                lds.pages[i] = page_entry(a.c.table, a.c.max_pages, a.c.n_pages, b, page0 + i);
            __syncthreads();

            // Rows that do not take part (before the start, past the end, on no page) are read from the head's first row.  No
            // branches: the entry is read at an index that is always in the table, and thrown away where the position is none.
            const int last_entry = ((stop - 1) >> a.c.page_shift) - page0;
            auto page_of = [&](int pos) {
                const int i = (pos >> a.c.page_shift) - page0, page = lds.pages[min(max(i, 0), last_entry)];
                return (int)(pos >= r.start) & (int)(pos < stop) & (int)(page >= 0) ? page : -1;
            };
            auto row_at = [&](const unsigned char* base, long long page_bytes, long long slot_bytes, int page, int pos) {
                return base + max(page, 0) * page_bytes + (page < 0 ? 0 : pos & slots) * slot_bytes;
            };
            auto load_k = [&](int p) {
                const unsigned char* at = row_at(kbase, a.c.k_page, a.c.k_slot, page_of(p + m), p + m);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int piece = ks * 4 + g;
                    kf[ks] = *(const u32x4*)(at + (piece * PER < a.c.Dk ? piece : 0) * 16);
                }
            };
            auto load_v = [&](int p) {
                const int pos = p + g * 4;
                int page[4];
                if (a.c.page_shift >= 2) {           // four neighbours are on one page
                    const int i = (pos >> a.c.page_shift) - page0, one = lds.pages[min(max(i, 0), last_entry)];
#pragma unroll
                    for (int j = 0; j < 4; ++j) page[j] = (int)(pos + j >= r.start) & (int)(pos + j < stop) & (int)(one >= 0) ? one : -1;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) page[j] = page_of(pos + j);
                }
                live = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned char* at = row_at(vbase, a.c.v_page, a.c.v_slot, page[j], pos + j);
                    live |= page[j] < 0 ? 0u : 1u << j;
#pragma unroll
                    for (int vb = 0; vb < VB; ++vb) {
                        const int piece = vb * 16 + m;
                        vf[j][vb] = *(const u32x4*)(at + (piece * PER < a.c.Dv ? piece : 0) * 16);
                    }
                }
            };

            int p = (int)p0 + wave * TILE;
            load_k(p);
            load_v(p);
            for (; p < stop; p += ATT_WAVES * TILE) {
                if (a.c.Dk != KS * 4 * PER) {        // pieces past the key's end
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                        for (int i = 0; i < 4; ++i) kf[ks][i] = (ks * 4 + g) * PER < a.c.Dk ? kf[ks][i] : 0u;
                }
                f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) s = product<BF16>(kf[ks], qf[ks], s);
                const uint32_t now = live;
                const int next = p + ATT_WAVES * TILE;
                load_k(next);
                __builtin_amdgcn_sched_barrier(0);   // requested here, not where they are used

                if (!__all(now == 15u)) {
                    // what stands in a row that does not take part may be anything: no NaN of it may reach the sums
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                            for (int i = 0; i < 4; ++i) vf[j][vb][i] = (now >> j) & 1u ? vf[j][vb][i] : 0u;
                }
                float z[4], most = -__builtin_inff();
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    z[j] = (now >> j) & 1u ? s[j] * a.scale : -__builtin_inff();
                    most = fmaxf(most, z[j]);
                }
                if constexpr (MASS) {
                    // (a store without a branch, which the counting of outstanding loads would have to assume taken: what lies
                    // behind the head's row of the chunk, or past the group, is dropped by its offset)
                    const int at = p + g * 4 - begin;
                    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3])},
                                                           kept, at < pl.chunk ? (m * pl.chunk + at) * 4 : 0x7FFFFFF0, 0, 0);
                }
                most = fmaxf(most, __shfl_xor(most, 16, 64));
                most = fmaxf(most, __shfl_xor(most, 32, 64));
                if (__any(most > top)) {
                    const float higher = fmaxf(top, most), keep = exp_(top - origin(higher));
                    top = higher;
                    sum *= keep;
#pragma unroll
                    for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                        for (int j = 0; j < PER; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[vb][j][i] *= keep;
                }
                const float at = origin(top);
                float e[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    e[j] = exp_(z[j] - at) * unit;
                    sum += e[j];
                }
                if constexpr (BF16) {
                    u32x2 part[3];                   // P: the nearest bf16 numbers, the nearest to what is left, and what then is left
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float left[2] = {e[2 * i], e[2 * i + 1]};
#pragma unroll
                        for (int u = 0; u < 3; ++u) {
                            const uint32_t both = pack_bf16x2(left[0], left[1]);
                            part[u][i] = both;
                            left[0] -= __uint_as_float(both << 16);
                            left[1] -= __uint_as_float(both & 0xFFFF0000u);
                        }
                    }
#pragma unroll
                    for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                        for (int j = 0; j < PER; ++j) {
                            u32x2 t;                 // dimension 8c + j of the lane's 4 keys
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                t[i] = __builtin_amdgcn_perm(vf[2 * i + 1][vb][j >> 1], vf[2 * i][vb][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                            for (int u = 0; u < 3; ++u) {
                                o[vb][j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(short4v, t), __builtin_bit_cast(short4v, part[u]), o[vb][j], 0, 0, 0);
                                if (SPECIAL && u == 0)
#pragma unroll
                                    for (int i = 0; i < 2; ++i) t[i] = finite_halves(t[i]);
                            }
                        }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                            for (int j = 0; j < PER; ++j)
                                o[vb][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[i][vb][j]), e[i], o[vb][j], 0, 0, 0);
                }
                load_v(next);
                asm volatile("" ::: "memory");       // here, not at the top of the next round
            }
        }

        // the four waves' results: o[vb][j][i] of lane (m, g) is head m, dimension (vb * 16 + 4g + i) * PER + j.  They are added in
        // LDS, wave w then writing the dimensions of i = w.
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (g == 0) {
            wave_m[wave][m] = top;
            wave_l[wave][m] = sum;
        }
        __syncthreads();
        float all = wave_m[0][m], total = 0.0f;
#pragma unroll
        for (int w = 1; w < ATT_WAVES; ++w) all = fmaxf(all, wave_m[w][m]);
#pragma unroll
        for (int w = 0; w < ATT_WAVES; ++w) total += wave_l[w][m] * exp_(wave_m[w][m] - origin(all));
        const float mine = exp_(top - origin(all));
        const bool direct = r.chunks <= 1;
        const float by = 1.0f / total;
        bool odd = false;
        if (wave == 0 && g == 0 && h < pl.G) {
            if (!direct || MASS) pl.ml[part] = make_float2(all, total / unit);
            if (direct && a.lse) a.lse[hq] = origin(all) + __log2f(total / unit) * LN2;
        }
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) {
            if (vb > 0) __syncthreads();
#pragma unroll
            for (int j = 0; j < PER; ++j) {
#pragma unroll
                for (int i = 0; i < 4; ++i) o[vb][j][i] *= mine;
                lds.o[wave][j][lane] = o[vb][j];
            }
            __syncthreads();
            const int dim = (vb * 16 + 4 * g + wave) * PER;
            if (h >= pl.G || dim >= a.c.Dv) continue;
            float v[PER];
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                v[j] = ((lds.o[0][j][lane][wave] + lds.o[1][j][lane][wave]) + (lds.o[2][j][lane][wave] + lds.o[3][j][lane][wave])) * by;
                v[j] = total == 0.0f ? 0.0f : v[j];          // no position, or none above -infinity
                odd = odd || !__builtin_isfinite(v[j]);
            }
            if (BF16 && direct) {
                *(u32x4*)((uint16_t*)a.out + hq * a.c.Dv + dim) =
                    u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[PER - 4], v[PER - 3]), pack_bf16x2(v[PER - 2], v[PER - 1])};
            } else {
                float* dst = direct ? (float*)a.out + hq * a.c.Dv + dim : pl.o + part * a.c.Dv + dim;
#pragma unroll
                for (int j = 0; j < PER; j += 4) *(f32x4*)(dst + j) = f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]};
            }
        }
        return odd;
    };
    // An infinite value is right with the first part of P alone: a later one, 0 or below it, makes NaN of it.  So where a result
    // is not finite the chunk is done again, with zeros for such values in the later products.  And the sum over up to 2^31 values
    // may pass the largest number where their average does not: there its terms are 2^-32 of what they are.
    const bool odd = run(std::false_type{});
    if (__builtin_expect(__syncthreads_or(odd), 0)) run(std::true_type{});
}

static constexpr int JOIN_THREADS = 256, JOIN_WAVES = JOIN_THREADS / 64;
static constexpr int MASS_POSITIONS = 4 * JOIN_THREADS;      // of a workgroup

// maximum and sum over a head's chunks, by a wave (ml: of the first chunk, G entries to the next)
__device__ __forceinline__ float2 join_chunks(const float2* ml, int chunks, int G, int lane)
{
    float top = -__builtin_inff(), total = 0.0f;
    for (int s = lane; s < chunks; s += 64) {
        const float2 c = ml[(long long)s * G];
        const float higher = fmaxf(top, c.x);
        total = total * exp_(top - origin(higher)) + c.y * exp_(c.x - origin(higher));
        top = higher;
    }
#pragma unroll
    for (int mask = 1; mask < 64; mask <<= 1) {
        const float ot = __shfl_xor(top, mask, 64), ol = __shfl_xor(total, mask, 64), higher = fmaxf(top, ot);
        total = total * exp_(top - origin(higher)) + ol * exp_(ot - origin(higher));
        top = higher;
    }
    // (two lanes may have rounded their sum of two products differently: everyone takes the first lane's)
    return make_float2(__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(top))),
                       __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(total))));
}

// Workgroups 0 .. B * Hq - 1: one query head's chunks are joined.  The others add the attention weight of MASS_POSITIONS
// positions at one key-value head to mass.
template <bool BF16>
__global__ __launch_bounds__(JOIN_THREADS) void attend_join_kernel(AttendArgs a, AttendPlan pl, int joins, int mass_blocks)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if ((int)blockIdx.x < joins) {
        __shared__ float weight[JOIN_THREADS];
        __shared__ __attribute__((aligned(16))) f32x4 part_o[JOIN_THREADS];
        const int b = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, kvh = hq / pl.G, h = hq % pl.G;
        const Range r = range_of(a.lengths, a.starts, b, a.max_len, pl.chunk);
        if (r.chunks <= 1) return;                           // written already
        const long long part0 = ((long long)(b * a.c.Hkv + kvh) * pl.S) * pl.G + h;
        const float2 joined = join_chunks(pl.ml + part0, r.chunks, pl.G, lane);      // the same in every wave
        const float at = origin(joined.x), by = joined.y == 0.0f ? 0.0f : 1.0f / joined.y;
        // columns of 4 values; the threads of one column share the chunks
        const int cols = a.c.Dv / 4, groups = JOIN_THREADS / cols, col = tid % cols, grp = tid / cols;
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int s0 = 0; s0 < r.chunks; s0 += JOIN_THREADS) {
            if (s0 > 0) __syncthreads();
            if (s0 + tid < r.chunks) {
                const float2 c = pl.ml[part0 + (long long)(s0 + tid) * pl.G];
                weight[tid] = exp_(c.x - at) * c.y * by;
            }
            __syncthreads();
            const int n = r.chunks - s0 < JOIN_THREADS ? r.chunks - s0 : JOIN_THREADS;
            if (grp < groups)
#pragma unroll 8
                for (int s = grp; s < n; s += groups) {
                    const f32x4 v = *(const f32x4*)(pl.o + (part0 + (long long)(s0 + s) * pl.G) * a.c.Dv + col * 4);
                    const float w = weight[s];
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i] = fmaf(v[i], w, acc[i]);
                }
        }
        part_o[tid] = acc;
        __syncthreads();
        const long long out = (long long)b * a.Hq + hq;
        if (tid == 0 && a.lse) a.lse[out] = at + __log2f(joined.y) * LN2;
        if (grp > 0) return;
        for (int q = 1; q < groups; ++q) {
            const f32x4 v = part_o[q * cols + col];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += v[i];
        }
        if constexpr (BF16) *(u32x2*)((uint16_t*)a.out + out * a.c.Dv + col * 4) = u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
        else *(f32x4*)((float*)a.out + out * a.c.Dv + col * 4) = acc;
    } else {
        constexpr int HEADS = 64;                            // at a time
        __shared__ float head_m[HEADS], head_by[HEADS];
        const int i = blockIdx.x - joins, row = i / mass_blocks, b = row / a.c.Hkv;
        const Range r = range_of(a.lengths, a.starts, b, a.max_len, pl.chunk);
        const int p = r.first + (i % mass_blocks) * MASS_POSITIONS + tid;
        if (p - tid >= r.len || r.chunks == 0) return;       // the whole workgroup
        // (positions that do not take part read the first one's, and are not stored)
        float* mass = a.mass + (long long)row * a.mass_stride;
        float w[4] = {}, was[4];
        bool in[4];
        long long from[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int pos = p + j * JOIN_THREADS;
            in[j] = pos >= r.start && pos < r.len;
            const uint32_t off = in[j] ? pos - r.first : r.start - r.first, split = off / (uint32_t)pl.chunk;
            from[j] = (long long)split * pl.G * pl.chunk + (off - split * (uint32_t)pl.chunk);
            was[j] = mass[in[j] ? pos : r.start];
        }
        for (int h0 = 0; h0 < pl.G; h0 += HEADS) {
            if (h0 > 0) __syncthreads();
            const int n = pl.G - h0 < HEADS ? pl.G - h0 : HEADS;
            for (int h = wave; h < n; h += JOIN_WAVES) {
                const float2 joined = join_chunks(pl.ml + (long long)row * pl.S * pl.G + h0 + h, r.chunks, pl.G, lane);
                if (lane == 0) {
                    head_m[h] = origin(joined.x);
                    head_by[h] = joined.y == 0.0f ? 0.0f : 1.0f / joined.y;
                }
            }
            __syncthreads();
            const float* s = pl.scores + ((long long)row * pl.S * pl.G + h0) * pl.chunk;
#pragma unroll 4
            for (int h = 0; h < n; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] += exp_(s[from[j] + (long long)h * pl.chunk] - head_m[h]) * head_by[h];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (in[j]) mass[p + j * JOIN_THREADS] = was[j] + w[j];
    }
}

// ---------------------------------------------------------------------------

// How the positions are cut.  The longest sequences are cut into enough chunks that there are two workgroups for every CU, if
// a chunk then still has 256 positions (four tiles per wave): a smaller one costs a join that takes longer than it saves (one
// sequence of 151 positions 8.5 us whole, 11.3 in two chunks; 131071 positions 58 us, for three workgroups per CU 63).  With several
// sequences a chunk has at most 512 positions, because their lengths differ and the host does not know them (61 sequences of
// 17 to 8192 positions with mass: 105 us, 129 in chunks of 2048; where the lengths are equal it costs: 61 of 1400 each 80 us, and
// 66 in one chunk each); one sequence is cut into chunks of up to 2048.
static constexpr int TARGET = 512, LEAST = 256;      // workgroups; positions of a chunk
static constexpr int STEP = ATT_WAVES * TILE;        // positions that a workgroup's waves take at once
// the most positions of a chunk: 2048, 512 where there are several sequences, and 1 / 256 of the longest where that is more
static long long longest_chunk(const AttendArgs& a)
{
    const long long most = a.c.B > 1 ? 512 : 2048, share = (a.max_len + 255ll) / 256;
    return most > share ? most : share;
}
static AttendPlan plan_of(const AttendArgs& a)
{
    AttendPlan pl{};
    pl.G = a.Hq / a.c.Hkv;
    pl.head_blocks = (pl.G + 15) / 16;
    pl.rows = a.c.B * a.c.Hkv;
    const long long items = pl.rows > 0 ? (long long)pl.rows * pl.head_blocks : 1;
    long long chunk = ((long long)a.max_len * items + TARGET - 1) / TARGET;
    if (chunk > longest_chunk(a)) chunk = longest_chunk(a);
    if (chunk < LEAST) chunk = LEAST;
    if (chunk > a.max_len + 16ll) chunk = a.max_len + 16ll;      // a first position is rounded down
    pl.chunk = (int)((chunk + STEP - 1) / STEP * STEP);
    pl.S = (int)((a.max_len + 15ll + pl.chunk - 1) / pl.chunk);
    if (pl.S < 1) pl.S = 1;
    return pl;
}

static size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

bool attend_fits(const AttendArgs& a)
{
    if ((long long)a.c.B * a.c.Hkv >= (1ll << 23) || (long long)a.c.B * a.Hq >= (1ll << 23)) return false;
    const AttendPlan pl = plan_of(a);
    const long long wgs = ((long long)pl.rows * pl.S + 7) * pl.head_blocks;
    const long long join = (long long)a.c.B * a.Hq + (a.mass ? (long long)pl.rows * ((a.max_len + 15ll) / MASS_POSITIONS + 1) : 0);
    return wgs < (1ll << 23) && join < (1ll << 23);              // a launch's threads stay below 2^32
}

// Enough for this call and for every one with a smaller max_len, B or Hkv (of the same G): the number of chunks falls where their
// size grows by a step, so what is counted here are bounds that only grow.  For unrounded chunks of c positions,
//   c >= LEAST                              chunks of all heads <= heads * ceil((max_len + 15) / LEAST)
//   c = max_len * items / TARGET            <= TARGET * (query heads of an item) + 2 heads
//   c = longest_chunk                       <= heads * ceil((max_len + 15) / c), and never more than 258 of a head
// and a head's chunks have less than max_len + 15 + c positions together, c <= longest_chunk, max_len + 16, rounded to STEP.
size_t attend_workspace_bytes(const AttendArgs& a)
{
    const AttendPlan pl = plan_of(a);
    const size_t heads = (size_t)a.c.B * a.Hq, positions = (size_t)a.max_len + 15;
    auto least = [](size_t x, size_t y) { return x < y ? x : y; };
    auto most = [](size_t x, size_t y) { return x > y ? x : y; };
    auto chunks_of = [&](size_t c) { return (positions + c - 1) / c; };
    const size_t parts = least(heads * chunks_of(LEAST), most(((size_t)TARGET * pl.G + pl.head_blocks - 1) / pl.head_blocks + 2 * heads,
                                                              heads * least(chunks_of(a.c.B > 1 ? 512 : 2048), 258)));
    size_t n = 0;
    if (chunks_of(LEAST) > 1) n += up16(parts * a.c.Dv * 4);
    if (chunks_of(LEAST) > 1 || a.mass) n += up16(parts * 8);
    if (a.mass) n += heads * (positions + least(most(longest_chunk(a), LEAST), positions + 1) + STEP) * 4;
    return heads ? n : 0;
}

template <bool BF16> static hipError_t launch(const AttendArgs& a, const AttendPlan& pl)
{
    constexpr int W = BF16 ? 1 : 2;                              // an fp32 row has twice the pieces
    const bool wide = a.c.Dv > 128;
    auto kern = [&](auto mass_c) {
        constexpr bool MASS = decltype(mass_c)::value;
        return a.c.Dk <= 64 ? (wide ? attend_kernel<BF16, 2 * W, 2 * W, MASS> : attend_kernel<BF16, 2 * W, W, MASS>)
             : a.c.Dk <= 128 ? (wide ? attend_kernel<BF16, 4 * W, 2 * W, MASS> : attend_kernel<BF16, 4 * W, W, MASS>)
                             : (wide ? attend_kernel<BF16, 8 * W, 2 * W, MASS> : attend_kernel<BF16, 8 * W, W, MASS>);
    };
    hipLaunchKernelGGL((a.mass ? kern(std::true_type{}) : kern(std::false_type{})), dim3((unsigned)((pl.rows * pl.S + 7) / 8 * 8 * pl.head_blocks)), dim3(ATT_THREADS), 0, a.stream, a, pl);
    hipError_t err = hipGetLastError();
    const int joins = pl.S > 1 ? a.c.B * a.Hq : 0;
    const int mass_blocks = a.mass ? (int)((a.max_len + 15ll) / MASS_POSITIONS + 1) : 0;
    const long long wgs = joins + (long long)pl.rows * mass_blocks;
    if (err != hipSuccess || wgs == 0) return err;
    hipLaunchKernelGGL(attend_join_kernel<BF16>, dim3((unsigned)wgs), dim3(JOIN_THREADS), 0, a.stream, a, pl, joins, mass_blocks);
    return hipGetLastError();
}

hipError_t launch_attend(const AttendArgs& a)
{
    AttendPlan pl = plan_of(a);
    const size_t parts = (size_t)a.c.B * a.Hq * pl.S;
    unsigned char* ws = (unsigned char*)a.workspace;
    if (pl.S > 1) { pl.o = (float*)ws; ws += up16(parts * a.c.Dv * 4); }
    if (pl.S > 1 || a.mass) { pl.ml = (float2*)ws; ws += up16(parts * 8); }
    if (a.mass) pl.scores = (float*)ws;
    return a.c.dtype == 1 ? launch<true>(a, pl) : launch<false>(a, pl);
}

}  // namespace paep
