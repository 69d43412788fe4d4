// Writing and reading a paged key-value cache in 4 bits.
//
// 32 neighbours of a row, a group, share a byte, the power 2^(byte - 127); each is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, two to
// a byte.  A group's power is the smallest with which its largest magnitude is at most 7 powers (which goes to 6): then no element
// is further from the number it becomes than half the distance of two neighbours there, the largest included.  It is one
// addition on the bits of that magnitude: m 2^E, 1 <= m < 2, wants 2^(E - 2) where m <= 1.75 and 2^(E - 1) above.
// Every byte is read and written once; what bounds it is memory, and for few tokens a chain of three dependent loads (61 tokens of
// 8 heads 4.6 us).  5 sequences of 1000 to 9001 positions back in fp32, 123 MB: 25 us into one buffer, 32 into two in turn.
#include "cache_device.h"
#include "fourbit_device.h"

namespace paep {

static constexpr int CELL_THREADS = 256;
static constexpr int CELL = 8;                   // elements of a thread: four threads to a group

// Element q * CELL of head h of a key (or value): where its codes stand, and its group's byte.
struct Cell { unsigned char* codes; uint8_t* scale; };
__device__ __forceinline__ Cell cell_of(const CacheView& c, bool is_k, uint8_t* k_scales, uint8_t* v_scales, long long page, int slot, int h, int q)
{
    const int blocks = (is_k ? c.Dk : c.Dv) / 32;
    unsigned char* base = is_k ? c.k + page * c.k_page + h * c.k_head + slot * c.k_slot : c.v + page * c.v_page + h * c.v_head + slot * c.v_slot;
    return {base + q * (CELL / 2), (is_k ? k_scales : v_scales) + (((page * c.Hkv + h) * blocks + q / 4) << c.page_shift) + slot};
}

// What a thread works on: tokens U i .. U i + U - 1, head h, piece q of their keys or values.
struct Place { int i, h, q; bool is_k; };
__device__ __forceinline__ Place place_of(uint32_t at, int k_pieces, int v_pieces, int Hkv)
{
    const uint32_t k_all = k_pieces * Hkv, per_row = k_all + v_pieces * Hkv;
    Place w;
    w.i = (int)(at / per_row);
    const uint32_t piece = at - w.i * per_row;
    w.is_k = piece < k_all;
    const uint32_t rest = w.is_k ? piece : piece - k_all, per = w.is_k ? k_pieces : v_pieces;
    w.h = (int)(rest / per);
    w.q = (int)(rest - w.h * per);
    return w;
}

// Pages and positions of U tokens from `first` on; -1 where one names no place or lies behind the last.
template <int U> struct Spots { int page[U], slot[U]; };
template <int U>
__device__ __forceinline__ Spots<U> spots_of(const CacheView& c, long long first, int n, const int32_t* sequences, const int32_t* positions)
{
    Spots<U> s;
    int b[U], p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long i = min(first + u, (long long)n - 1);
        b[u] = sequences ? sequences[i] : (int)i;
        p[u] = positions[i];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool in = first + u < n && (uint32_t)b[u] < (uint32_t)c.B && p[u] >= 0;
        s.page[u] = in ? page_entry(c.table, c.max_pages, c.n_pages, b[u], p[u] >> c.page_shift) : -1;
        s.slot[u] = p[u] & ((1 << c.page_shift) - 1);
    }
    return s;
}

__device__ __forceinline__ uint32_t quad_max(uint32_t v)
{
    uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true);         // lane ^ 1
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true);                  // lane ^ 2
    return v > o ? v : o;
}

template <bool BF16, int U>
__global__ __launch_bounds__(CELL_THREADS) void append_fourbit_kernel(
    CacheView c, int first, int n, uint32_t cells, const unsigned char* __restrict__ k, long long k_row, long long k_head,
    const unsigned char* __restrict__ v, long long v_row, long long v_head, uint8_t* __restrict__ k_scales, uint8_t* __restrict__ v_scales,
    const int32_t* __restrict__ sequences, const int32_t* __restrict__ positions)
{
    const uint32_t at = blockIdx.x * CELL_THREADS + threadIdx.x;
    if (at >= cells) return;                                 // (whole groups)
    const Place w = place_of(at, c.Dk / CELL, c.Dv / CELL, c.Hkv);
    const long long i = (long long)first + (long long)w.i * U, row = w.is_k ? k_row : v_row;
    const unsigned char* from = (w.is_k ? k + w.h * k_head : v + w.h * v_head) + w.q * (CELL * (BF16 ? 2 : 4));
    const Spots<U> s = spots_of<U>(c, i, n, sequences, positions);
    u32x4 raw[U][BF16 ? 1 : 2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < (BF16 ? 1 : 2); ++j) raw[u][j] = *(const u32x4*)(from + min(i + u, (long long)n - 1) * row + 16 * j);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (BF16) { x[2 * j] = raw[u][0][j] << 16; x[2 * j + 1] = raw[u][0][j] & 0xFFFF0000u; }
            else { x[j] = raw[u][0][j]; x[4 + j] = raw[u][BF16 ? 0 : 1][j]; }
        }
        uint32_t most = 0;                                   // bits of magnitudes: infinity above every number, NaN above infinity
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, x[j] & 0x7FFFFFFFu);
        most = quad_max(most);
        const bool nan = most > 0x7F800000u;
        const int byte = nan ? 255 : min(max((int)((most + 0x1FFFFFu) >> 23) - 2, FOUR_LEAST_BYTE), FOUR_MOST_BYTE);
        const float scale = __uint_as_float((uint32_t)(nan ? 127 : byte) << 23);
        uint32_t codes = 0;                                  // (to nearest, of two the even code, what is past 6 powers to 6)
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x[0]), __uint_as_float(x[1]), scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x[2]), __uint_as_float(x[3]), scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x[4]), __uint_as_float(x[5]), scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x[6]), __uint_as_float(x[7]), scale, 3);
        if (s.page[u] < 0) continue;
        const Cell to = cell_of(c, w.is_k, k_scales, v_scales, s.page[u], s.slot[u], w.h, w.q);
        *(uint32_t*)to.codes = codes;
        if (w.q % 4 == 0) *to.scale = (uint8_t)byte;
    }
}

template <bool BF16, int U>
__global__ __launch_bounds__(CELL_THREADS) void read_fourbit_kernel(
    CacheView c, int first, int n, uint32_t cells, uint8_t* __restrict__ k_scales, uint8_t* __restrict__ v_scales,
    const int32_t* __restrict__ sequences, const int32_t* __restrict__ positions, unsigned char* __restrict__ k, unsigned char* __restrict__ v)
{
    const uint32_t at = blockIdx.x * CELL_THREADS + threadIdx.x;
    if (at >= cells) return;
    const Place w = place_of(at, c.Dk / CELL, c.Dv / CELL, c.Hkv);
    const long long i = (long long)first + (long long)w.i * U;
    const Spots<U> s = spots_of<U>(c, i, n, sequences, positions);
    uint32_t codes[U], byte[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Cell from = cell_of(c, w.is_k, k_scales, v_scales, max(s.page[u], 0), s.page[u] < 0 ? 0 : s.slot[u], w.h, w.q);
        codes[u] = *(const uint32_t*)from.codes;
        byte[u] = *from.scale;
    }
    const int width = w.is_k ? c.Dk : c.Dv;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (i + u >= n) break;
        const uint32_t x = s.page[u] < 0 ? 0u : codes[u];
        const float scale = __uint_as_float((s.page[u] < 0 ? 127u : byte[u]) << 23);
        unsigned char* to = (w.is_k ? k : v) + (((i + u) * c.Hkv + w.h) * width + w.q * CELL) * (BF16 ? 2 : 4);
        const uint32_t t[4] = {pair_bf16<0>(x, scale), pair_bf16<1>(x, scale), pair_bf16<2>(x, scale), pair_bf16<3>(x, scale)};
        if constexpr (BF16) {
            *(u32x4*)to = u32x4{t[0], t[1], t[2], t[3]};
        } else {
            *(u32x4*)to = u32x4{t[0] << 16, t[0] & 0xFFFF0000u, t[1] << 16, t[1] & 0xFFFF0000u};
            *(u32x4*)(to + 16) = u32x4{t[2] << 16, t[2] & 0xFFFF0000u, t[3] << 16, t[3] & 0xFFFF0000u};
        }
    }
}

// Calls `launch(tokens of a thread, first token, end, cells)` for parts whose threads stay below 2^31.  A thread works on several tokens
// where there are enough of them to fill the device: finding its place among heads and pieces is most of what it computes.  8 heads of
// 128 + 128, us for one token of a thread and for four, append; read.  bf16: 8192 tokens 15.3, 11.7 (3.6 TB/s); 14.5, 11.7.  4096, the
// switch: 9.6, 8.5; 9.4, 8.4.  2048: 6.1, 5.6; 5.8, 5.6.  1024: 4.5, 4.7; 4.4, 4.7.  fp32: 16384 tokens 37.5, 35.7; 46.4, 48.8.
// 8192: 16.3, 15.8; 19.1, 20.0.  4096: 10.3, 10.1; 11.9, 11.9.  2048: 7.0, 7.4; 8.0, 8.2.
static constexpr int SEVERAL = 4;
template <typename F> static hipError_t in_parts(const CacheView& c, int n, F launch)
{
    const long long per_row = (long long)c.Hkv * (c.Dk + c.Dv) / CELL;
    const int of = n * per_row >= (1ll << 20) ? SEVERAL : 1;
    const int most = (int)((1ll << 31) / per_row) - 1;
    for (int first = 0; first < n; first += most) {
        const int rows = n - first < most ? n - first : most;
        launch(of, first, first + rows, (uint32_t)((rows + of - 1) / of * per_row));
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

hipError_t launch_cache_append_fourbit(const CacheView& c, uint8_t* k_scales, uint8_t* v_scales, int n, const void* k, long long k_row,
                                       long long k_head, const void* v, long long v_row, long long v_head, const int32_t* sequences,
                                       const int32_t* positions, hipStream_t stream)
{
    return in_parts(c, n, [&](int of, int first, int end, uint32_t cells) {
        const auto kern = c.dtype == 1 ? (of == 1 ? append_fourbit_kernel<true, 1> : append_fourbit_kernel<true, SEVERAL>)
                                       : (of == 1 ? append_fourbit_kernel<false, 1> : append_fourbit_kernel<false, SEVERAL>);
        hipLaunchKernelGGL(kern, dim3((cells + CELL_THREADS - 1) / CELL_THREADS), dim3(CELL_THREADS), 0, stream, c, first, end, cells,
                           (const unsigned char*)k, k_row, k_head, (const unsigned char*)v, v_row, v_head, k_scales, v_scales, sequences, positions);
    });
}

hipError_t launch_cache_read_fourbit(const CacheView& c, const uint8_t* k_scales, const uint8_t* v_scales, int n, const int32_t* sequences,
                                     const int32_t* positions, void* k, void* v, hipStream_t stream)
{
    return in_parts(c, n, [&](int of, int first, int end, uint32_t cells) {
        const auto kern = c.dtype == 1 ? (of == 1 ? read_fourbit_kernel<true, 1> : read_fourbit_kernel<true, SEVERAL>)
                                       : (of == 1 ? read_fourbit_kernel<false, 1> : read_fourbit_kernel<false, SEVERAL>);
        hipLaunchKernelGGL(kern, dim3((cells + CELL_THREADS - 1) / CELL_THREADS), dim3(CELL_THREADS), 0, stream, c, first, end, cells,
                           const_cast<uint8_t*>(k_scales), const_cast<uint8_t*>(v_scales), sequences, positions, (unsigned char*)k, (unsigned char*)v);
    });
}

}  // namespace paep
