// Attention of one new token per sequence over a paged cache held in 4 bits: the formula of attend.hip on
//
//   k = code * 2^(byte - 127),   v likewise        32 neighbours of a row share a byte
//
// A code times a power of two is a bf16 number, so nothing is rounded on the way from the cache to the matrix instructions.
// What bounds it: a position of 128 + 128 dimensions is 136 bytes, 17 / 64 of bf16 storage, and the vector instructions that
// take codes apart and turn values round are as long as its loads.
#include <type_traits>

#include "attend_device.h"
#include "fourbit_device.h"

namespace paep {

static constexpr int FOUR_THREADS = 256, FOUR_WAVES = FOUR_THREADS / 64;
static constexpr int FOUR_TILE = 32;              // positions of a wave at a time, two halves of 16
static constexpr int FOUR_TABLE = 2048;           // page-table entries in LDS at a time

__device__ __forceinline__ f32x4 mfma32(const u32x4& x, const u32x4& y, f32x4 acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
}
__device__ __forceinline__ float across_groups_max(float v)      // over the four lanes of one head
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}

// QP: bf16 parts of a query element (1: bf16 storage, 3: fp32); KW: 4-byte words of a key in a lane (16 lanes' worth of 4 words
// cover 128 dimensions); VD: dimensions of a value in a lane; PAGED16: 16 neighbours are on one page, whose address is the wave's
template <int QP, int KW, int VD, bool PAGED16>
__global__ __launch_bounds__(FOUR_THREADS, KW <= 4 && VD <= 8 ? 3 : 2) void attend_fourbit_kernel(AttendFourbitArgs a, AttendPlan pl)
{
    constexpr bool BF16 = QP == 1;
    constexpr int VW = VD >= 8 ? VD / 8 : 1;     // 4-byte words of a value in a lane (of 4 dimensions: half of one)
    constexpr int OD = VD < 8 ? VD : 8;          // dimensions of a lane that are joined at a time
    __shared__ __attribute__((aligned(16))) union {
        int pages[FOUR_TABLE + 1];
        f32x4 o[FOUR_WAVES][OD][64];
    } lds;
    __shared__ float wave_m[FOUR_WAVES][16], wave_l[FOUR_WAVES][16];

    const int item = blockIdx.x;
    // eight neighbours run on eight XCDs: the head blocks of one chunk, which read the same rows, are put on one
    const int hb = item / 8 % pl.head_blocks;
    const int rest = item / (8 * pl.head_blocks) * 8 + item % 8;
    if (rest >= pl.rows * pl.S) return;
    const int split = rest / pl.rows, row = rest % pl.rows;
    const CacheView& cv = a.a.c;
    const int b = row / cv.Hkv, kvh = row % cv.Hkv;
    const Range r = range_of(a.a.lengths, a.a.starts, b, a.a.max_len, pl.chunk);
    if (split >= r.chunks && split > 0) return;  // the first workgroup of an empty range writes its zeros

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, g = lane >> 4;
    const long long lo = r.first + (long long)split * pl.chunk;
    const int begin = (int)lo, end = r.chunks == 0 ? begin : (int)(lo + pl.chunk < r.len ? lo + pl.chunk : r.len);
    const int h = hb * 16 + m;                   // the lane's head, of the group
    const long long hq = (long long)b * a.a.Hq + kvh * pl.G + h;
    const long long part = ((long long)row * pl.S + split) * pl.G + h;

    // Lane (m, g) holds key m's words of dimensions kd .. kd + 8 KW - 1 (KW = 8: 32 of them, and 32 that lie 128 further), all of
    // one scale byte (KW = 8: of two); queries likewise, as operand B, zeros past Dk and past the group.
    constexpr int KD = KW <= 4 ? 8 * KW : 32, KU = KW <= 4 ? 1 : 2;
    u32x4 qf[KW][QP];
#pragma unroll
    for (int w = 0; w < KW; ++w) {
        const int d = g * KD + (w & 3) * 8 + (w >> 2) * 128;
        u32x4 x[BF16 ? 1 : 2] = {};
        if (h < pl.G && d < cv.Dk) {
            const unsigned char* at = (const unsigned char*)a.a.q + b * a.a.q_seq + (long long)(kvh * pl.G + h) * a.a.q_head + (BF16 ? 2 : 4) * d;
#pragma unroll
            for (int i = 0; i < (BF16 ? 1 : 2); ++i) x[i] = *(const u32x4*)(at + 16 * i);
        }
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

    const unsigned char* kbase = cv.k + kvh * cv.k_head;
    const unsigned char* vbase = cv.v + kvh * cv.v_head;
    const int ps = 1 << cv.page_shift, slots = ps - 1;
    const int kblocks = cv.Dk / 32, vblocks = cv.Dv / 32;
    // pieces past a row's end are read from its beginning; queries are 0 there, and what it makes of values is not stored
    int k_at[KU], k_blk[KU];
#pragma unroll
    for (int u = 0; u < KU; ++u) {
        const int d = g * KD + u * 128 < cv.Dk ? g * KD + u * 128 : 0;
        k_at[u] = d / 2;
        k_blk[u] = d / 32;
    }
    const int v_d = m * VD < cv.Dv ? m * VD : 0, v_at = v_d / 2, v_blk = v_d / 32;

    // All of the chunk, its results written.  True where one of this thread's is not finite.  SPECIAL: the values may be near the
    // largest number.
    auto run = [&](auto special_c) {
        constexpr bool SPECIAL = decltype(special_c)::value;
        constexpr float unit = SPECIAL ? 0x1p-32f : 1.0f;    // what an exponential of 0 counts as
        f32x4 o[VD];
        float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
        for (int j = 0; j < VD; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        uint32_t kf[2][KW], ks[2][KU];               // keys of both halves, their scale bytes
        uint32_t vf[8][VW], vs[2];                   // values of the lane's 8 positions, 4g .. 4g + 3 of each half, and their scale bytes
        uint32_t live = 0;                           // which of the 8 take part

        const long long stretch = (long long)FOUR_TABLE << cv.page_shift;
        for (long long p0 = begin; p0 < end; p0 += stretch) {
            const int stop = p0 + stretch < end ? (int)(p0 + stretch) : end;
            const int page0 = (int)p0 >> cv.page_shift, last_entry = ((stop - 1) >> cv.page_shift) - page0;
            __syncthreads();
            for (int i = threadIdx.x; i <= last_entry; i += FOUR_THREADS)
                lds.pages[i] = page_entry(cv.table, cv.max_pages, cv.n_pages, b, page0 + i);
            __syncthreads();

            // Rows that do not take part (before the start, past the end, on no page) are read from a slot that exists.
            auto entry_of = [&](int pos) { return lds.pages[min(max((pos >> cv.page_shift) - page0, 0), last_entry)]; };
            auto takes_part = [&](int pos, int page) { return (int)(pos >= r.start) & (int)(pos < stop) & (int)(page >= 0); };
            auto load_k = [&](int p) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const unsigned char *at, *sc;
                    if constexpr (PAGED16) {
                        const int pos = p + 16 * i;
                        const long long page = max(__builtin_amdgcn_readfirstlane(entry_of(pos)), 0);
                        at = kbase + page * cv.k_page + (pos & slots) * cv.k_slot + (uint32_t)(m * (int)cv.k_slot);
                        sc = a.k_scales + (((page * cv.Hkv + kvh) * kblocks) << cv.page_shift) + (pos & slots) + (uint32_t)m;
                    } else {
                        const int pos = p + 16 * i + m, e = entry_of(pos);
                        const long long page = max(e, 0), slot = e < 0 ? 0 : pos & slots;
                        at = kbase + page * cv.k_page + slot * cv.k_slot;
                        sc = a.k_scales + (((page * cv.Hkv + kvh) * kblocks) << cv.page_shift) + slot;
                    }
#pragma unroll
                    for (int u = 0; u < KU; ++u) {
                        if constexpr (KW == 2) {
                            const u32x2 x = *(const u32x2*)(at + k_at[u]);
                            kf[i][0] = x[0];
                            kf[i][1] = x[1];
                        } else {
                            const u32x4 x = *(const u32x4*)(at + k_at[u]);
#pragma unroll
                            for (int w = 0; w < 4; ++w) kf[i][4 * u + w] = x[w];
                        }
                        ks[i][u] = sc[k_blk[u] << cv.page_shift];
                    }
                }
            };
            auto load_word = [&](const unsigned char* at, uint32_t* to) {
                if constexpr (VD == 4) to[0] = *(const uint16_t*)at;
                else if constexpr (VD == 8) to[0] = *(const uint32_t*)at;
                else { const u32x2 x = *(const u32x2*)at; to[0] = x[0]; to[1] = x[1]; }
            };
            auto load_v = [&](int p) {
                live = 0;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (PAGED16) {
                        const int pos = p + 16 * i, e = __builtin_amdgcn_readfirstlane(entry_of(pos));
                        const long long page = max(e, 0);
                        const unsigned char* at = vbase + page * cv.v_page + (pos & slots) * cv.v_slot;
                        const unsigned char* sc = a.v_scales + (((page * cv.Hkv + kvh) * vblocks) << cv.page_shift) + (pos & slots);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            load_word(at + j * cv.v_slot + (uint32_t)(4 * g * (int)cv.v_slot + v_at), vf[4 * i + j]);
                            live |= takes_part(pos + 4 * g + j, e) << (4 * i + j);
                        }
                        vs[i] = *(const uint32_t*)(sc + (uint32_t)((v_blk << cv.page_shift) + 4 * g));
                    } else {
                        vs[i] = 0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int pos = p + 16 * i + 4 * g + j, e = entry_of(pos);
                            const long long page = max(e, 0), slot = e < 0 ? 0 : pos & slots;
                            load_word(vbase + page * cv.v_page + slot * cv.v_slot + v_at, vf[4 * i + j]);
                            live |= takes_part(pos, e) << (4 * i + j);
                            vs[i] |= (uint32_t)a.v_scales[(((page * cv.Hkv + kvh) * vblocks + v_blk) << cv.page_shift) + slot] << (8 * j);
                        }
                    }
                }
            };

            int p = (int)p0 + wave * FOUR_TILE;
            load_k(p);
            load_v(p);
            for (; p < stop; p += FOUR_WAVES * FOUR_TILE) {
                f32x4 s[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < KW; ++w) {
                        const float by = __uint_as_float(ks[i][w >> 2] << 23);
                        const u32x4 x = {pair_bf16<0>(kf[i][w], by), pair_bf16<1>(kf[i][w], by), pair_bf16<2>(kf[i][w], by), pair_bf16<3>(kf[i][w], by)};
#pragma unroll
                        for (int u = QP - 1; u >= 0; --u) s[i] = mfma32(x, qf[w][u], s[i]);
                    }
                }
                const uint32_t now = live;
                const int next = p + FOUR_WAVES * FOUR_TILE;
                load_k(next);
                __builtin_amdgcn_sched_barrier(0);   // requested here, not where they are used

                float z[8], most = -__builtin_inff();
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = s[j >> 2][j & 3] * a.a.scale;
                if (!__all(now == 255u)) {
                    // what stands in a row that does not take part may be anything: no NaN of it may reach the sums
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        z[j] = (now >> j) & 1u ? z[j] : -__builtin_inff();
                        vs[j >> 2] = (now >> j) & 1u ? vs[j >> 2] : (vs[j >> 2] & ~(255u << (8 * (j & 3)))) | 127u << (8 * (j & 3));
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, z[j]);
                // The exponentials' reference point need not be the maximum: it is moved where a score is more than 8 above it.
                if (__any(most > top + 8.0f)) {
                    most = across_groups_max(most);
                    const float higher = fmaxf(top, most), keep = exp_(top - origin(higher));
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
                    e[j] = exp_(z[j] - at) * unit;
                    sum += e[j];
                }
                u32x4 prob[3];                       // P: the nearest bf16 numbers, the nearest to what is left, and what then is left
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float left[2] = {e[2 * i], e[2 * i + 1]};
#pragma unroll
                    for (int u = 0; u < 3; ++u) {
                        const uint32_t both = pack_bf16x2(left[0], left[1]);
                        prob[u][i] = both;
                        left[0] -= __uint_as_float(both << 16);
                        left[1] -= __uint_as_float(both & 0xFFFF0000u);
                    }
                }
                float by[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) by[j] = __uint_as_float((vs[j >> 2] >> (8 * (j & 3)) & 255u) << 23);
                // two dimensions of all 8 positions at a time: the pairs of one position become pairs of neighbouring positions
                auto add = [&](auto byte_c) {
                    constexpr int B = decltype(byte_c)::value;
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        uint32_t t[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) t[j] = pair_bf16<B>(vf[j][w], by[j]);
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            u32x4 x;
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_perm(t[2 * i + 1], t[2 * i], half ? 0x07060302u : 0x05040100u);
                            f32x4& to = o[8 * w + 2 * B + half];
#pragma unroll
                            for (int u = 0; u < 3; ++u) to = mfma32(x, prob[u], to);
                        }
                    }
                };
                add(std::integral_constant<int, 0>{});
                add(std::integral_constant<int, 1>{});
                if constexpr (VD > 4) {
                    add(std::integral_constant<int, 2>{});
                    add(std::integral_constant<int, 3>{});
                }
                load_v(next);
                asm volatile("" ::: "memory");       // here, not at the top of the next round
            }
        }

        // the four waves' results: o[j][i] of lane (m, g) is head m, dimension (4g + i) * VD + j.  They are added in LDS, wave w
        // then writing the dimensions of i = w.
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (g == 0) {
            wave_m[wave][m] = top;
            wave_l[wave][m] = sum;
        }
        __syncthreads();
        float all = wave_m[0][m], total = 0.0f;
#pragma unroll
        for (int w = 1; w < FOUR_WAVES; ++w) all = fmaxf(all, wave_m[w][m]);
#pragma unroll
        for (int w = 0; w < FOUR_WAVES; ++w) total += wave_l[w][m] * exp_(wave_m[w][m] - origin(all));
        const float mine = exp_(top - origin(all));
        const bool direct = r.chunks <= 1;
        const float by = 1.0f / total;
        bool odd = false;
        if (wave == 0 && g == 0 && h < pl.G) {
            if (!direct) pl.ml[part] = make_float2(all, total / unit);
            else if (a.a.lse) a.a.lse[hq] = origin(all) + __log2f(total / unit) * LN2;
        }
#pragma unroll
        for (int j0 = 0; j0 < VD; j0 += OD) {
            if (j0 > 0) __syncthreads();
#pragma unroll
            for (int j = 0; j < OD; ++j) {
#pragma unroll
                for (int i = 0; i < 4; ++i) o[j0 + j][i] *= mine;
                lds.o[wave][j][lane] = o[j0 + j];
            }
            __syncthreads();
            const int dim = (4 * g + wave) * VD + j0;
            if (h >= pl.G || dim >= cv.Dv) continue;
            float v[OD];
#pragma unroll
            for (int j = 0; j < OD; ++j) {
                v[j] = ((lds.o[0][j][lane][wave] + lds.o[1][j][lane][wave]) + (lds.o[2][j][lane][wave] + lds.o[3][j][lane][wave])) * by;
                v[j] = total == 0.0f ? 0.0f : v[j];          // no position, or none above -infinity
                odd = odd || !__builtin_isfinite(v[j]);
            }
            if (BF16 && direct) {
#pragma unroll
                for (int j = 0; j < OD; j += 4)
                    *(u32x2*)((uint16_t*)a.a.out + hq * cv.Dv + dim + j) = u32x2{pack_bf16x2(v[j], v[j + 1]), pack_bf16x2(v[j + 2], v[j + 3])};
            } else {
                float* dst = direct ? (float*)a.a.out + hq * cv.Dv + dim : pl.o + part * cv.Dv + dim;
#pragma unroll
                for (int j = 0; j < OD; j += 4) *(f32x4*)(dst + j) = f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]};
            }
        }
        return odd;
    };
    // The sum over up to 2^31 values may pass the largest number where their average does not: a chunk whose results are not finite
    // is done again, with 2^-32 of its terms.
    const bool odd = run(std::false_type{});
    if (__builtin_expect(__syncthreads_or(odd), 0)) run(std::true_type{});
}

// ---------------------------------------------------------------------------

static constexpr AttendCut FOUR_CUT = {512, 256, FOUR_WAVES * FOUR_TILE, 2048, 512};

bool attend_fourbit_fits(const AttendFourbitArgs& a) { return attend_plan_fits(a.a, FOUR_CUT); }
size_t attend_fourbit_workspace_bytes(const AttendFourbitArgs& a) { return attend_plan_workspace(a.a, FOUR_CUT); }

template <int QP, bool PAGED16> static auto kernel_of(int Dk, int Dv)
{
    if (Dk <= 64) return Dv <= 64 ? attend_fourbit_kernel<QP, 2, 4, PAGED16> : Dv <= 128 ? attend_fourbit_kernel<QP, 2, 8, PAGED16> : attend_fourbit_kernel<QP, 2, 16, PAGED16>;
    if (Dk <= 128) return Dv <= 128 ? attend_fourbit_kernel<QP, 4, 8, PAGED16> : attend_fourbit_kernel<QP, 4, 16, PAGED16>;
    return Dv <= 128 ? attend_fourbit_kernel<QP, 8, 8, PAGED16> : attend_fourbit_kernel<QP, 8, 16, PAGED16>;
}

hipError_t launch_attend_fourbit(const AttendFourbitArgs& a)
{
    const AttendPlan pl = attend_plan_placed(a.a, FOUR_CUT);
    const CacheView& c = a.a.c;
    // (a lane's offset from the first of 16 rows has 31 bits)
    const bool paged16 = c.page_shift >= 4 && c.k_slot < (1 << 26) && c.v_slot < (1 << 26);
    const auto kern = c.dtype == 1 ? (paged16 ? kernel_of<1, true>(c.Dk, c.Dv) : kernel_of<1, false>(c.Dk, c.Dv))
                                   : (paged16 ? kernel_of<3, true>(c.Dk, c.Dv) : kernel_of<3, false>(c.Dk, c.Dv));
    hipLaunchKernelGGL(kern, dim3((unsigned)((pl.rows * pl.S + 7) / 8 * 8 * pl.head_blocks)), dim3(FOUR_THREADS), 0, a.a.stream, a, pl);
    const hipError_t err = hipGetLastError();
    return err != hipSuccess ? err : launch_attend_join(a.a, pl);
}

}  // namespace paep
