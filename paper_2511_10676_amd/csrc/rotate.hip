// Norms of queries and keys for each head and the rotation by position, in one pass; with APPEND the keys and values go into a
// paged cache.
//
//   x' = w x / sqrt(mean(x^2) + eps)                    where there are weights w
//   y_a = x'_a cos - x'_b sin,  y_b = x'_a sin + x'_b cos    for each of the rot / 2 pairs (a, b) of the rotated dimensions
//
// Every element is read and written once, and that is what bounds it.  A head's row of up to 256 elements is spread over `lanes`
// neighbouring lanes, each with two 16-byte pieces that hold both numbers of its pairs, so that nothing but the sum of squares
// goes from lane to lane.  Where pairs do not fill pieces, a row goes through LDS.
// Measured: 8191 bf16 tokens of 36 heads of 128, with norms, 151 MB, 27 us (5.6 TB/s); 4096 fp32 tokens of 27 heads of 80 into a cache,
// 71 MB, 16 us (4.6 TB/s); 61 tokens of 48 heads 4.1 us, one token 2.1 us, a launch.
// Through LDS, where each element reads a cosine, a sine and its other half: 8191 bf16 tokens of 36 heads of 80, 40 of their dimensions
// rotated, 59 us, 27 for all 80 (not through LDS); 4096 fp32 tokens, 20 dimensions, 33 us, 24 for all.
#include <type_traits>

#include "cache_device.h"

namespace paep {

static constexpr int ROT_THREADS = 256;

// sum over 2^n neighbouring lanes
__device__ __forceinline__ float sum_lanes(float v, int lanes)
{
    auto add = [&](auto ctrl) { v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xF, 0xF, true)); };
    if (lanes > 1) add(std::integral_constant<int, 0xB1>{});         // lane ^ 1
    if (lanes > 2) add(std::integral_constant<int, 0x4E>{});         // lane ^ 2
    if (lanes > 4) add(std::integral_constant<int, 0x141>{});        // 7 - lane of 8: both halves hold one number each
    if (lanes > 8) add(std::integral_constant<int, 0x140>{});        // 15 - lane of 16
    if (lanes > 16) v += __shfl_xor(v, 16, 64);
    return v;
}

// STREAM: the results are written past the caches
template <bool BF16, bool APPEND, bool THROUGH_LDS, bool STREAM>
__global__ __launch_bounds__(ROT_THREADS) void rotate_kernel(RotateArgs a, int first, uint32_t rows, int log_lanes)
{
    constexpr int PER = BF16 ? 8 : 4, N = 2 * PER;           // elements of a piece, of a lane
    __shared__ float whole[THROUGH_LDS ? ROT_THREADS * N : 1];
    const int lanes = 1 << log_lanes, t = threadIdx.x & (lanes - 1);
    const uint32_t row = (blockIdx.x * (uint32_t)ROT_THREADS + threadIdx.x) >> log_lanes;
    const int heads = a.Hq + (APPEND ? 2 : 1) * a.Hk;
    const uint32_t token = row / (uint32_t)heads;
    const int head = (int)(row - token * heads);
    const long long i = (long long)first + token;
    const int at = row < rows ? a.angles[i] : -1;
    const bool is_q = head < a.Hq, is_v = APPEND && head >= a.Hq + a.Hk;
    const int h = is_q ? head : is_v ? head - a.Hq - a.Hk : head - a.Hq;

    bool on = (uint32_t)at < (uint32_t)a.table_rows;         // a token at no row of the table is left out
    const unsigned char* from = (is_q ? (const unsigned char*)a.q + i * a.q_row + h * a.q_head
                                 : is_v ? (const unsigned char*)a.v + i * a.v_row + h * a.v_head
                                        : (const unsigned char*)a.k + i * a.k_row + h * a.k_head);
    unsigned char* to;
    if (is_q) {
        to = (unsigned char*)a.q_out + i * a.q_out_row + h * a.q_out_head;
    } else if (!APPEND) {
        to = (unsigned char*)a.k_out + i * a.k_out_row + h * a.k_out_head;
    } else {
        to = nullptr;
        if (on) {
            const int b = a.sequences ? a.sequences[i] : (int)i, p = a.positions[i];
            const int page = (uint32_t)b < (uint32_t)a.c.B && p >= 0 ? page_entry(a.c.table, a.c.max_pages, a.c.n_pages, b, p >> a.c.page_shift) : -1;
            const int slot = p & ((1 << a.c.page_shift) - 1);
            on = page >= 0;
            if (on) {
                to = is_v ? a.c.v + page * a.c.v_page + h * a.c.v_head + slot * a.c.v_slot : a.c.k + page * a.c.k_page + h * a.c.k_head + slot * a.c.k_slot;
                if (!is_v && t == 0 && a.mass && p < a.mass_stride) a.mass[((long long)b * a.c.Hkv + h) * a.mass_stride + p] = 0.0f;
            }
        }
    }
    const int half = a.rot / 2, pairs = THROUGH_LDS ? 0 : half / PER;        // lanes that hold rotated pairs
    const bool halves = !THROUGH_LDS && a.style == 0;
    // the lane's pieces
    const int one = halves && t < pairs ? t : 2 * t, two = halves && t < pairs ? t + pairs : 2 * t + 1;
    const int pieces = (is_v ? a.c.Dv : a.D) / PER;
    const bool has_one = on && one < pieces, has_two = on && two < pieces;
    u32x4 raw[2] = {};
    if (has_one) raw[0] = *(const u32x4*)(from + one * 16);
    if (has_two) raw[1] = *(const u32x4*)(from + two * 16);
    if (is_v) {
        if (has_one) *(u32x4*)(to + one * 16) = raw[0];
        if (has_two) *(u32x4*)(to + two * 16) = raw[1];
        if (!THROUGH_LDS) return;
    }
    auto widen = [&](const u32x4& p, float* x) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (BF16) {
                x[2 * j] = __uint_as_float(p[j] << 16);
                x[2 * j + 1] = __uint_as_float(p[j] & 0xFFFF0000u);
            } else {
                x[j] = __uint_as_float(p[j]);
            }
        }
    };
    float x[N];
    widen(raw[0], x);
    widen(raw[1], x + PER);

    const void* weight = is_v ? nullptr : is_q ? a.q_weight : a.k_weight;
    if (weight) {
        u32x4 wraw[2] = {};
        if (has_one) wraw[0] = *(const u32x4*)((const unsigned char*)weight + one * 16);
        if (has_two) wraw[1] = *(const u32x4*)((const unsigned char*)weight + two * 16);
        float w[N], squares[2] = {0.0f, 0.0f};
        widen(wraw[0], w);
        widen(wraw[1], w + PER);
#pragma unroll
        for (int j = 0; j < N; ++j) squares[j & 1] = fmaf(x[j], x[j], squares[j & 1]);
        const float mean = sum_lanes(squares[0] + squares[1], lanes) / (float)a.D + a.eps;
        if (__builtin_expect(mean > 1e-25f && mean < 1e37f, 1)) {
            const float by = __builtin_amdgcn_rsqf(mean);
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = x[j] * by * w[j];
        } else {
            // squares that may have left the range of fp32
            double wide = 0.0;
#pragma unroll
            for (int j = 0; j < N; ++j) wide += (double)x[j] * x[j];
            for (int mask = 1; mask < lanes; mask <<= 1) wide += __shfl_xor(wide, mask, 64);
            const double by = 1.0 / sqrt(wide / a.D + (double)a.eps);
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = (float)(x[j] * by) * w[j];
        }
    }

    if constexpr (THROUGH_LDS) {
        float* mine = whole + (threadIdx.x >> log_lanes) * (lanes * N);
#pragma unroll
        for (int j = 0; j < N; ++j) mine[t * N + j] = x[j];
        __syncthreads();
        if (is_v) return;
        if (on) {
            const float* turn = a.table + (long long)at * a.rot;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int d = t * N + j;
                if (d >= a.rot) break;
                const bool second = a.style == 0 ? d >= half : d & 1;
                const int pair = a.style == 0 ? (second ? d - half : d) : d >> 1;
                const int other = a.style == 0 ? (second ? d - half : d + half) : d ^ 1;
                const float c = turn[pair], s = turn[half + pair], y = mine[other];
                x[j] = second ? fmaf(x[j], c, y * s) : fmaf(x[j], c, -(y * s));
            }
        }
    } else if (t < pairs && on) {
        const float* turn = a.table + (long long)at * a.rot + t * PER;
        float c[PER], s[PER];
#pragma unroll
        for (int j = 0; j < PER; j += 4) {
            const f32x4 cv = *(const f32x4*)(turn + j), sv = *(const f32x4*)(turn + half + j);
#pragma unroll
            for (int u = 0; u < 4; ++u) { c[j + u] = cv[u]; s[j + u] = sv[u]; }
        }
        if (halves) {
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const float p = x[j], q = x[PER + j];
                x[j] = fmaf(p, c[j], -(q * s[j]));
                x[PER + j] = fmaf(q, c[j], p * s[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const float p = x[2 * j], q = x[2 * j + 1];
                x[2 * j] = fmaf(p, c[j], -(q * s[j]));
                x[2 * j + 1] = fmaf(q, c[j], p * s[j]);
            }
        }
    }
    auto store = [&](int piece, const float* y) {
        u32x4 p;
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = BF16 ? pack_bf16x2(y[BF16 ? 2 * j : 0], y[BF16 ? 2 * j + 1 : 0]) : __float_as_uint(y[j]);
        if (STREAM) __builtin_nontemporal_store(p, (u32x4*)(to + piece * 16));
        else *(u32x4*)(to + piece * 16) = p;
    };
    if (has_one) store(one, x);
    if (has_two) store(two, x + PER);
}

hipError_t launch_rotate(const RotateArgs& a)
{
    const bool bf16 = a.dtype == 1, append = a.append;
    const int per = bf16 ? 8 : 4, widest = append && a.c.Dv > a.D ? a.c.Dv : a.D;
    int log_lanes = 0;
    while ((2 * per << log_lanes) < widest) ++log_lanes;
    const bool lds = a.rot % (2 * per) != 0;                 // pairs that do not fill pieces
    // Outputs of many tokens leave the caches alone where a row's lanes write whole cache lines together (where they write every
    // second 16 bytes it takes longer, 4096 fp32 tokens into a cache 16.4 -> 22.2 us).  Heads of 128, through the caches and past them, alone,
    // and with a copy of all queries behind it, which then has to fetch them from memory (the rule goes by the call alone):
    //   19 MB out: 10.7, 9.8 us; 16.5, 17.3        38 MB: 16.6, 16.1; 30.8, 32.3        57 MB: 27.6, 22.4; 46.0, 47.7
    //   67 MB: 32.2, 25.6; 51.0, 55.5              75 MB: 35.4, 28.0; 55.9, 61.0
    //   151 MB: 62.7, 57.9; 122, 111               302 MB: 118, 111; 216, 214
    const bool stream = !append && !lds && a.style == 0 && a.rot == a.D && a.D * 16 / per >= 256 &&
                        (long long)a.n * (a.Hq + a.Hk) * a.D * 16 / per >= (64ll << 20);
    auto kern = bf16 ? (append ? (lds ? rotate_kernel<true, true, true, false> : rotate_kernel<true, true, false, false>)
                               : lds ? rotate_kernel<true, false, true, false>
                                     : stream ? rotate_kernel<true, false, false, true> : rotate_kernel<true, false, false, false>)
                     : (append ? (lds ? rotate_kernel<false, true, true, false> : rotate_kernel<false, true, false, false>)
                               : lds ? rotate_kernel<false, false, true, false>
                                     : stream ? rotate_kernel<false, false, false, true> : rotate_kernel<false, false, false, false>);
    const long long heads = a.Hq + (append ? 2ll : 1ll) * a.Hk;
    const int most = (int)(((1ll << 30) / heads) >> log_lanes);              // tokens of a launch: its threads stay below 2^31
    for (int first = 0; first < a.n; first += most) {
        const uint32_t rows = (uint32_t)((a.n - first < most ? a.n - first : most) * heads);
        const uint32_t threads = rows << log_lanes;
        hipLaunchKernelGGL(kern, dim3((threads + ROT_THREADS - 1) / ROT_THREADS), dim3(ROT_THREADS), 0, a.stream, a, first, rows, log_lanes);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace paep
