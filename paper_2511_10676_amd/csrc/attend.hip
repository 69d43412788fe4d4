// Attention of one new token per sequence over a paged key-value cache.
//
//   s = scale q k^T,  P = exp(s - max) / sum,  out = P V       one row of s per query head
//
// Every key and value is needed once by the G query heads that share it, so what bounds the operator is reading the cache.
// attend_kernel: a workgroup of four waves takes one chunk of one sequence's positions at one key-value head, for up to
// 16 * HT of its query heads; a wave takes every fourth tile of 32 positions (16 in fp32 storage).  Keys and values go from
// memory straight into the registers of the matrix instructions, no LDS in between:
//   S^T = K Q^T   a wave's operand A is 16 keys, lane (m, g) holding 16 bytes of key m: four lanes fetch 64 contiguous bytes.
//                 Lane (m, g) of the result holds head m's scores of keys 4g .. 4g + 3, which is operand B of the second
//                 product as it stands, if its summation index runs over keys in that order:
//   O^T = V^T P^T operand A wants 8 keys of one dimension in a lane.  Lane (c, g) fetches dimensions 8c .. 8c + 7 of the
//                 8 keys that its lane group g holds (16 lanes read a whole row), and one byte permutation per register
//                 transposes the 8 x 8 block inside the lane.  Row c of the j-th of 8 products is dimension 8c + j.
// (fp32 storage: the same with 16-byte pieces of 4 and the 16x16x4 instruction, key by key.)  The running maximum and sum are
// per lane, one head each, and the accumulated O is rescaled in place, where a maximum grew, without any exchange between lanes.
// P is multiplied as two bf16 parts (16 bits of it): the second instruction costs nothing next to the loads, and the result
// keeps the accuracy of fp32 probabilities.
// The next tile's keys are requested once this tile's are multiplied, the next values likewise, so that a wave always has
// a tile in flight.  Waves are joined in LDS, chunks by attend_join_kernel, in a fixed order.
#include <type_traits>

#include "cache_device.h"

namespace paep {

static constexpr int ATT_THREADS = 256, ATT_WAVES = ATT_THREADS / 64;
static constexpr int TABLE = 2048;               // page-table entries in LDS at a time
static constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;

struct AttendPlan {
    int G, head_blocks, HT;      // query heads of a key-value head, blocks of 16 * HT of them
    int chunk, S;                // positions of a workgroup, chunks of the longest sequence
    int rows;                    // B * Hkv
    float* o;                    // [rows][S][G][Dv] unnormalised outputs of the chunks (S > 1)
    float2* ml;                  // [rows][S][G] their maxima (of scores in units of log2) and sums (S > 1 or mass)
    float* scores;               // [B][Hq][score_stride], in units of log2 (mass)
    long long score_stride;
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

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }
// the reference point of exponentials whose maximum is m: 0 where nothing was above -infinity
__device__ __forceinline__ float origin(float m) { return m == -__builtin_inff() ? 0.0f : m; }

// KS: 16-byte steps of four lanes that cover a key; VB: blocks of 16 lanes x 16 bytes that cover a value; HT: blocks of 16 heads
template <bool BF16, int KS, int VB, int HT>
__global__ __launch_bounds__(ATT_THREADS) void attend_kernel(AttendArgs a, AttendPlan pl)
{
    constexpr int PER = BF16 ? 8 : 4;            // elements of a 16-byte piece
    constexpr int KT = BF16 ? 2 : 1;             // 16-key blocks of a tile
    constexpr int TILE = 16 * KT, NK = 4 * KT;   // keys of a tile; of them in a lane
    __shared__ int pages[TABLE + 1];
    __shared__ float wave_m[ATT_WAVES][HT * 16], wave_l[ATT_WAVES][HT * 16];
    __shared__ __attribute__((aligned(16))) f32x4 wave_o[2][VB * PER][64];

    const int item = blockIdx.x;
    const int hb = item % pl.head_blocks;
    const int rest = item / pl.head_blocks;
    const int split = rest / pl.rows, row = rest % pl.rows;
    const int b = row / a.c.Hkv, kvh = row % a.c.Hkv;
    const Range r = range_of(a.lengths, a.starts, b, a.max_len, pl.chunk);
    if (split >= r.chunks && split > 0) return;  // the first workgroup of an empty range writes its zeros

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, g = lane >> 4;
    const int head0 = hb * 16 * HT;              // of the group
    const float factor = a.scale * LOG2E;
    const long long lo = r.first + (long long)split * pl.chunk;
    const int begin = (int)lo, end = r.chunks == 0 ? begin : (int)(lo + pl.chunk < r.len ? lo + pl.chunk : r.len);

    // queries: operand B, lane (m, g): head m, piece ks * 4 + g; zeros past Dk and past the group
    u32x4 qf[HT][KS];
#pragma unroll
    for (int ht = 0; ht < HT; ++ht)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ht][ks] = u32x4{0u, 0u, 0u, 0u};
            const int h = head0 + ht * 16 + m, piece = ks * 4 + g;
            if (h < pl.G && piece * PER < a.c.Dk)
                qf[ht][ks] = *(const u32x4*)((const unsigned char*)a.q + b * a.q_seq + (long long)(kvh * pl.G + h) * a.q_head + piece * 16);
        }

    f32x4 o[HT][VB][PER];
    float top[HT], sum[HT];
#pragma unroll
    for (int ht = 0; ht < HT; ++ht) {
        top[ht] = -__builtin_inff();
        sum[ht] = 0.0f;
#pragma unroll
        for (int vb = 0; vb < VB; ++vb)
#pragma unroll
            for (int j = 0; j < PER; ++j) o[ht][vb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const unsigned char* kbase = a.c.k + kvh * a.c.k_head;
    const unsigned char* vbase = a.c.v + kvh * a.c.v_head;
    const int slots = (1 << a.c.page_shift) - 1;
    u32x4 kf[KT][KS], vf[NK][VB];
    uint32_t live = 0;                           // which of the lane's NK keys take part

    const long long stretch = (long long)TABLE << a.c.page_shift;        // positions whose page-table entries fit in LDS
    for (long long p0 = begin; p0 < end; p0 += stretch) {
        const int stop = p0 + stretch < end ? (int)(p0 + stretch) : end;
        const int page0 = (int)p0 >> a.c.page_shift;
        __syncthreads();
        for (int i = threadIdx.x; i <= ((stop - 1) >> a.c.page_shift) - page0; i += ATT_THREADS)
            pages[i] = page_entry(a.c.table, a.c.max_pages, a.c.n_pages, b, page0 + i);
        __syncthreads();

        // Rows that do not take part (before the start, past the end, on no page) are read from the pool's first row.
        auto page_of = [&](int p) { return p >= r.start && p < stop ? pages[(p >> a.c.page_shift) - page0] : -1; };
        auto load_k = [&](int p) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const int pos = p + kt * 16 + m, page = page_of(pos);
                const unsigned char* at = page < 0 ? a.c.k : kbase + page * a.c.k_page + (pos & slots) * a.c.k_slot;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int piece = ks * 4 + g;
                    const bool in = piece * PER < a.c.Dk;
                    const u32x4 f = *(const u32x4*)(at + (in ? piece : 0) * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) kf[kt][ks][i] = in ? f[i] : 0u;
                }
            }
        };
        auto load_v = [&](int p) {
            live = 0;
#pragma unroll
            for (int j = 0; j < NK; ++j) {
                const int pos = p + (j >> 2) * 16 + g * 4 + (j & 3), page = page_of(pos);
                const unsigned char* at = page < 0 ? a.c.v : vbase + page * a.c.v_page + (pos & slots) * a.c.v_slot;
                live |= page < 0 ? 0u : 1u << j;
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
            f32x4 s[HT][KT];
#pragma unroll
            for (int ht = 0; ht < HT; ++ht)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    s[ht][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        if constexpr (BF16) {
                            s[ht][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[kt][ks]),
                                                                                __builtin_bit_cast(bf16x8, qf[ht][ks]), s[ht][kt], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                s[ht][kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[kt][ks][i]),
                                                                                 __uint_as_float(qf[ht][ks][i]), s[ht][kt], 0, 0, 0);
                        }
                    }
                }
            const uint32_t now = live;
            const int next = p + ATT_WAVES * TILE;
            load_k(next);

            if (!__all(now == (1u << NK) - 1)) {
                // what stands in a row that does not take part may be anything: no NaN of it may reach the sums
#pragma unroll
                for (int j = 0; j < NK; ++j)
#pragma unroll
                    for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) vf[j][vb][i] = (now >> j) & 1u ? vf[j][vb][i] : 0u;
            }
            u32x4 phi[HT], plo[HT];              // bf16: P in two parts, packed; fp32: phi holds P itself
#pragma unroll
            for (int ht = 0; ht < HT; ++ht) {
                float z[NK], most = -__builtin_inff();
#pragma unroll
                for (int j = 0; j < NK; ++j) {
                    z[j] = (now >> j) & 1u ? s[ht][j >> 2][j & 3] * factor : -__builtin_inff();
                    most = fmaxf(most, z[j]);
                }
                if (a.mass) {
                    const int h = head0 + ht * 16 + m;
                    if (h < pl.G) {
                        float* dst = pl.scores + ((long long)b * a.Hq + kvh * pl.G + h) * pl.score_stride + p + g * 4;
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt)
                            if (p + kt * 16 + g * 4 < stop) *(f32x4*)(dst + kt * 16) = f32x4{z[4 * kt], z[4 * kt + 1], z[4 * kt + 2], z[4 * kt + 3]};
                    }
                }
                most = fmaxf(most, __shfl_xor(most, 16, 64));
                most = fmaxf(most, __shfl_xor(most, 32, 64));
                if (__any(most > top[ht])) {
                    const float now_top = fmaxf(top[ht], most), keep = exp2_(top[ht] - origin(now_top));
                    top[ht] = now_top;
                    sum[ht] *= keep;
#pragma unroll
                    for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                        for (int j = 0; j < PER; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[ht][vb][j][i] *= keep;
                }
                const float at = origin(top[ht]);
                float e[NK];
#pragma unroll
                for (int j = 0; j < NK; ++j) {
                    e[j] = exp2_(z[j] - at);
                    sum[ht] += e[j];
                }
                if constexpr (BF16) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        phi[ht][i] = pack_bf16x2(e[2 * i], e[2 * i + 1]);
                        plo[ht][i] = pack_bf16x2(e[2 * i] - __uint_as_float(phi[ht][i] << 16),
                                                 e[2 * i + 1] - __uint_as_float(phi[ht][i] & 0xFFFF0000u));
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) phi[ht][i] = __float_as_uint(e[i]);
                }
            }
#pragma unroll
            for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    if constexpr (BF16) {
                        u32x4 t;                 // dimension 8c + j of the lane's 8 keys
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            t[i] = __builtin_amdgcn_perm(vf[2 * i + 1][vb][j >> 1], vf[2 * i][vb][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                        for (int ht = 0; ht < HT; ++ht) {
                            o[ht][vb][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t), __builtin_bit_cast(bf16x8, phi[ht]), o[ht][vb][j], 0, 0, 0);
                            o[ht][vb][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t), __builtin_bit_cast(bf16x8, plo[ht]), o[ht][vb][j], 0, 0, 0);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int ht = 0; ht < HT; ++ht)
                                o[ht][vb][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[i][vb][j]), __uint_as_float(phi[ht][i]), o[ht][vb][j], 0, 0, 0);
                    }
                }
            load_v(next);
        }
    }

    // the four waves' results: o[ht][vb][j][i] of lane (m, g) is head m, dimension (vb * 16 + 4g + i) * PER + j
#pragma unroll
    for (int ht = 0; ht < HT; ++ht) {
        sum[ht] += __shfl_xor(sum[ht], 16, 64);
        sum[ht] += __shfl_xor(sum[ht], 32, 64);
        if (g == 0) {
            wave_m[wave][ht * 16 + m] = top[ht];
            wave_l[wave][ht * 16 + m] = sum[ht];
        }
    }
    __syncthreads();
    const bool direct = r.chunks <= 1;
#pragma unroll
    for (int ht = 0; ht < HT; ++ht) {
        float all = wave_m[0][ht * 16 + m], total = 0.0f;
#pragma unroll
        for (int w = 1; w < ATT_WAVES; ++w) all = fmaxf(all, wave_m[w][ht * 16 + m]);
        const float at = origin(all);
#pragma unroll
        for (int w = 0; w < ATT_WAVES; ++w) total += wave_l[w][ht * 16 + m] * exp2_(wave_m[w][ht * 16 + m] - at);
        const float mine = exp2_(top[ht] - at);
#pragma unroll
        for (int step = 2; step >= 1; step >>= 1) {          // waves 2 and 3 to 0 and 1, then 1 to 0
            __syncthreads();
#pragma unroll
            for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    if (step == 2)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[ht][vb][j][i] *= mine;
                    if (wave >= step && wave < 2 * step) wave_o[wave - step][vb * PER + j][lane] = o[ht][vb][j];
                }
            __syncthreads();
            if (wave < step)
#pragma unroll
                for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
                        const f32x4 other = wave_o[wave][vb * PER + j][lane];
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[ht][vb][j][i] += other[i];
                    }
        }
        const int h = head0 + ht * 16 + m;
        if (wave == 0 && h < pl.G) {
            const long long hq = (long long)b * a.Hq + kvh * pl.G + h, part = ((long long)row * pl.S + split) * pl.G + h;
            const float inv = total == 0.0f ? 0.0f : 1.0f / total;
            if (g == 0) {
                if (!direct || a.mass) pl.ml[part] = make_float2(all, total);
                if (direct && a.lse) a.lse[hq] = (origin(all) + __log2f(total)) * LN2;
            }
#pragma unroll
            for (int vb = 0; vb < VB; ++vb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int dim = (vb * 16 + 4 * g + i) * PER;
                    if (dim >= a.c.Dv) continue;
                    float v[PER];
#pragma unroll
                    for (int j = 0; j < PER; ++j) v[j] = direct ? o[ht][vb][j][i] * inv : o[ht][vb][j][i];
                    if (!direct || !BF16) {
                        float* dst = direct ? (float*)a.out + hq * a.c.Dv + dim : pl.o + part * a.c.Dv + dim;
#pragma unroll
                        for (int j = 0; j < PER; j += 4) *(f32x4*)(dst + j) = f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]};
                    } else if constexpr (BF16) {
                        *(u32x4*)((uint16_t*)a.out + hq * a.c.Dv + dim) =
                            u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
                    }
                }
        }
    }
}

static constexpr int JOIN_THREADS = 256;

// Workgroups 0 .. B * Hq - 1: one query head's chunks are joined.  The others add the attention weight of JOIN_THREADS
// positions at one key-value head to mass.
template <bool BF16>
__global__ __launch_bounds__(JOIN_THREADS) void attend_join_kernel(AttendArgs a, AttendPlan pl, int joins, int mass_blocks)
{
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < joins) {
        __shared__ float weight[JOIN_THREADS];
        __shared__ float all_m[JOIN_THREADS / 64], all_l[JOIN_THREADS / 64];
        __shared__ __attribute__((aligned(16))) f32x4 part_o[JOIN_THREADS];
        const int b = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, kvh = hq / pl.G, h = hq % pl.G;
        const Range r = range_of(a.lengths, a.starts, b, a.max_len, pl.chunk);
        if (r.chunks <= 1) return;                           // written already
        const long long part0 = ((long long)(b * a.c.Hkv + kvh) * pl.S) * pl.G + h;
        const int lane = tid & 63, wave = tid >> 6;
        float top = -__builtin_inff();
        for (int s = tid; s < r.chunks; s += JOIN_THREADS) top = fmaxf(top, pl.ml[part0 + (long long)s * pl.G].x);
        for (int mask = 1; mask < 64; mask <<= 1) top = fmaxf(top, __shfl_xor(top, mask, 64));
        if (lane == 0) all_m[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(all_m[0], all_m[1]), fmaxf(all_m[2], all_m[3]));
        const float at = origin(top);
        // columns of 4 values; the other threads share the chunks
        const int cols = a.c.Dv / 4, groups = JOIN_THREADS / cols, col = tid % cols, grp = tid / cols;
        float total = 0.0f;
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int s0 = 0; s0 < r.chunks; s0 += JOIN_THREADS) {
            __syncthreads();
            if (s0 + tid < r.chunks) {
                const float2 ml = pl.ml[part0 + (long long)(s0 + tid) * pl.G];
                weight[tid] = exp2_(ml.x - at);
                total += ml.y * weight[tid];
            }
            __syncthreads();
            const int n = r.chunks - s0 < JOIN_THREADS ? r.chunks - s0 : JOIN_THREADS;
            if (grp < groups)
#pragma unroll 4
                for (int s = grp; s < n; s += groups) {
                    const f32x4 v = *(const f32x4*)(pl.o + (part0 + (long long)(s0 + s) * pl.G) * a.c.Dv + col * 4);
                    const float w = weight[s];
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i] = fmaf(v[i], w, acc[i]);
                }
        }
        for (int mask = 1; mask < 64; mask <<= 1) total += __shfl_xor(total, mask, 64);
        if (lane == 0) all_l[wave] = total;
        part_o[tid] = acc;
        __syncthreads();
        total = (all_l[0] + all_l[1]) + (all_l[2] + all_l[3]);
        const long long out = (long long)b * a.Hq + hq;
        if (tid == 0 && a.lse) a.lse[out] = (at + __log2f(total)) * LN2;
        if (grp > 0) return;
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        for (int q = 1; q < groups; ++q) {
            const f32x4 v = part_o[q * cols + col];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += v[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] *= inv;
        if constexpr (BF16) *(u32x2*)((uint16_t*)a.out + out * a.c.Dv + col * 4) = u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
        else *(f32x4*)((float*)a.out + out * a.c.Dv + col * 4) = acc;
    } else {
        __shared__ float head_m[JOIN_THREADS], head_inv[JOIN_THREADS];
        const long long i = blockIdx.x - joins;
        const int row = (int)(i / mass_blocks), b = row / a.c.Hkv, kvh = row % a.c.Hkv;
        const Range r = range_of(a.lengths, a.starts, b, a.max_len, pl.chunk);
        const int p = r.first + (int)(i % mass_blocks) * JOIN_THREADS + tid;
        if (p - tid >= r.len || r.chunks == 0) return;       // the whole workgroup
        const bool in = p >= r.start && p < r.len;
        float w = 0.0f;
        for (int h0 = 0; h0 < pl.G; h0 += JOIN_THREADS) {
            __syncthreads();
            if (h0 + tid < pl.G) {
                const float2* ml = pl.ml + ((long long)row * pl.S) * pl.G + h0 + tid;
                float top = -__builtin_inff(), total = 0.0f;
                for (int s = 0; s < r.chunks; ++s) top = fmaxf(top, ml[(long long)s * pl.G].x);
                for (int s = 0; s < r.chunks; ++s) total += ml[(long long)s * pl.G].y * exp2_(ml[(long long)s * pl.G].x - origin(top));
                head_m[tid] = origin(top);
                head_inv[tid] = total == 0.0f ? 0.0f : 1.0f / total;
            }
            __syncthreads();
            const int n = pl.G - h0 < JOIN_THREADS ? pl.G - h0 : JOIN_THREADS;
            const float* s = pl.scores + ((long long)b * a.Hq + kvh * pl.G + h0) * pl.score_stride + p;
            if (in)
                for (int h = 0; h < n; ++h) w += exp2_(s[h * pl.score_stride] - head_m[h]) * head_inv[h];
        }
        if (in) a.mass[(long long)row * a.mass_stride + p] += w;
    }
}

// ---------------------------------------------------------------------------

static AttendPlan plan_of(const AttendArgs& a)
{
    AttendPlan pl{};
    pl.G = a.Hq / a.c.Hkv;
    pl.HT = pl.G > 16 ? 2 : 1;
    pl.head_blocks = (pl.G + 16 * pl.HT - 1) / (16 * pl.HT);
    pl.rows = a.c.B * a.c.Hkv;
    const int step = ATT_WAVES * (a.c.dtype == 1 ? 32 : 16);     // positions that a workgroup's waves take at once
    const long long items = pl.rows > 0 ? (long long)pl.rows * pl.head_blocks : 1;
    constexpr int TARGET = 512, MINC = 256, MAXC = 2048;
    long long chunk = ((long long)a.max_len * items + TARGET - 1) / TARGET;
    if (chunk < MINC) chunk = MINC;
    if (chunk > MAXC && (long long)a.max_len <= 256ll * MAXC) chunk = MAXC;
    if (chunk > a.max_len + 16ll) chunk = a.max_len + 16ll;      // a first position is rounded down
    chunk = (chunk + step - 1) / step * step;
    pl.chunk = (int)chunk;
    pl.S = (int)((a.max_len + 15ll + chunk - 1) / chunk);
    if (pl.S < 1) pl.S = 1;
    pl.score_stride = ((long long)a.max_len + 3) / 4 * 4;
    return pl;
}

static size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

bool attend_fits(const AttendArgs& a)
{
    if ((long long)a.c.B * a.c.Hkv >= (1ll << 23) || (long long)a.c.B * a.Hq >= (1ll << 23)) return false;
    const AttendPlan pl = plan_of(a);
    const long long wgs = (long long)pl.rows * pl.head_blocks * pl.S;
    const long long join = (long long)a.c.B * a.Hq + (long long)pl.rows * ((a.max_len + 15ll) / JOIN_THREADS + 1);
    return wgs < (1ll << 23) && join < (1ll << 23);              // a launch's threads stay below 2^32
}

size_t attend_workspace_bytes(const AttendArgs& a)
{
    const AttendPlan pl = plan_of(a);
    const size_t parts = (size_t)a.c.B * a.Hq * pl.S;
    size_t n = 0;
    if (pl.S > 1) n += up16(parts * a.c.Dv * 4);
    if (pl.S > 1 || a.mass) n += up16(parts * 8);
    if (a.mass) n += (size_t)a.c.B * a.Hq * pl.score_stride * 4;
    return n;
}

template <bool BF16, int KS, int VB> static void launch_ht(const AttendArgs& a, const AttendPlan& pl)
{
    const dim3 grid((unsigned)(pl.rows * pl.head_blocks * pl.S));
    if (pl.HT == 1) hipLaunchKernelGGL((attend_kernel<BF16, KS, VB, 1>), grid, dim3(ATT_THREADS), 0, a.stream, a, pl);
    else            hipLaunchKernelGGL((attend_kernel<BF16, KS, VB, 2>), grid, dim3(ATT_THREADS), 0, a.stream, a, pl);
}

template <bool BF16> static hipError_t launch(const AttendArgs& a, const AttendPlan& pl)
{
    constexpr int W = BF16 ? 1 : 2;                              // an fp32 row has twice the pieces
    const bool wide = a.c.Dv > 128;
    if (a.c.Dk <= 64)       wide ? launch_ht<BF16, 2 * W, 2 * W>(a, pl) : launch_ht<BF16, 2 * W, W>(a, pl);
    else if (a.c.Dk <= 128) wide ? launch_ht<BF16, 4 * W, 2 * W>(a, pl) : launch_ht<BF16, 4 * W, W>(a, pl);
    else                    wide ? launch_ht<BF16, 8 * W, 2 * W>(a, pl) : launch_ht<BF16, 8 * W, W>(a, pl);
    hipError_t err = hipGetLastError();
    const int joins = pl.S > 1 ? a.c.B * a.Hq : 0;
    const int mass_blocks = a.mass ? (int)((a.max_len + 15ll) / JOIN_THREADS + 1) : 0;
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
