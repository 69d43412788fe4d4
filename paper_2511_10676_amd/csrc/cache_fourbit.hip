// Writing and reading a paged key-value cache in 4 bits.
//
// 32 neighbours of a row, a group, share a byte, the power 2^(byte - 127); each is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, two to
// a byte.  A group's power is the smallest with which its largest magnitude is at most 7 powers (which goes to 6): then no element
// is further from the number it becomes than half the distance of two neighbours there, the largest included.  It is one
// addition on the bits of that magnitude: m 2^E, 1 <= m < 2, wants 2^(E - 2) where m <= 1.75 and 2^(E - 1) above.
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

// What a thread works on: token i, head h, piece q of its key or value.
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

__device__ __forceinline__ uint32_t quad_max(uint32_t v)
{
    uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true);         // lane ^ 1
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true);                  // lane ^ 2
    return v > o ? v : o;
}

template <bool BF16>
__global__ __launch_bounds__(CELL_THREADS) void append_fourbit_kernel(
    CacheView c, int first, uint32_t cells, const unsigned char* __restrict__ k, long long k_row, long long k_head,
    const unsigned char* __restrict__ v, long long v_row, long long v_head, uint8_t* __restrict__ k_scales, uint8_t* __restrict__ v_scales,
    const int32_t* __restrict__ sequences, const int32_t* __restrict__ positions)
{
    const uint32_t at = blockIdx.x * CELL_THREADS + threadIdx.x;
    if (at >= cells) return;                                 // (whole groups)
    const Place w = place_of(at, c.Dk / CELL, c.Dv / CELL, c.Hkv);
    const long long i = (long long)first + w.i;
    const int b = sequences ? sequences[i] : (int)i, p = positions[i];
    const unsigned char* from = (w.is_k ? k + i * k_row + w.h * k_head : v + i * v_row + w.h * v_head) + w.q * (CELL * (BF16 ? 2 : 4));
    uint32_t x[8];
    const u32x4 lo = *(const u32x4*)from;
    if constexpr (BF16) {
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[2 * j] = lo[j] << 16; x[2 * j + 1] = lo[j] & 0xFFFF0000u; }
    } else {
        const u32x4 hi = *(const u32x4*)(from + 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[j] = lo[j]; x[4 + j] = hi[j]; }
    }
    if ((uint32_t)b >= (uint32_t)c.B || p < 0) return;
    const int page = page_entry(c.table, c.max_pages, c.n_pages, b, p >> c.page_shift);
    if (page < 0) return;
    uint32_t most = 0;                                       // bits of magnitudes: infinity above every number, NaN above infinity
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, x[j] & 0x7FFFFFFFu);
    most = quad_max(most);
    const bool nan = most > 0x7F800000u;
    const int byte = nan ? 255 : min(max((int)((most + 0x1FFFFFu) >> 23) - 2, FOUR_LEAST_BYTE), FOUR_MOST_BYTE);
    const float scale = __uint_as_float((uint32_t)(nan ? 127 : byte) << 23);
    uint32_t codes = 0;                                      // (to nearest, of two the even code, what is past 6 powers to 6)
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x[0]), __uint_as_float(x[1]), scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x[2]), __uint_as_float(x[3]), scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x[4]), __uint_as_float(x[5]), scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x[6]), __uint_as_float(x[7]), scale, 3);
    const Cell to = cell_of(c, w.is_k, k_scales, v_scales, page, p & ((1 << c.page_shift) - 1), w.h, w.q);
    *(uint32_t*)to.codes = codes;
    if (w.q % 4 == 0) *to.scale = (uint8_t)byte;
}

template <bool BF16>
__global__ __launch_bounds__(CELL_THREADS) void read_fourbit_kernel(
    CacheView c, int first, uint32_t cells, uint8_t* __restrict__ k_scales, uint8_t* __restrict__ v_scales,
    const int32_t* __restrict__ sequences, const int32_t* __restrict__ positions, unsigned char* __restrict__ k, unsigned char* __restrict__ v)
{
    const uint32_t at = blockIdx.x * CELL_THREADS + threadIdx.x;
    if (at >= cells) return;
    const Place w = place_of(at, c.Dk / CELL, c.Dv / CELL, c.Hkv);
    const long long i = (long long)first + w.i;
    const int b = sequences ? sequences[i] : (int)i, p = positions[i];
    const int page = (uint32_t)b < (uint32_t)c.B && p >= 0 ? page_entry(c.table, c.max_pages, c.n_pages, b, p >> c.page_shift) : -1;
    uint32_t codes = 0;
    float scale = 1.0f;
    if (page >= 0) {
        const Cell from = cell_of(c, w.is_k, k_scales, v_scales, page, p & ((1 << c.page_shift) - 1), w.h, w.q);
        codes = *(const uint32_t*)from.codes;
        scale = __uint_as_float((uint32_t)*from.scale << 23);
    }
    const long long width = w.is_k ? c.Dk : c.Dv, element = (i * c.Hkv + w.h) * width + w.q * CELL;
    unsigned char* to = (w.is_k ? k : v) + element * (BF16 ? 2 : 4);
    if constexpr (BF16) {
        *(u32x4*)to = u32x4{pair_bf16<0>(codes, scale), pair_bf16<1>(codes, scale), pair_bf16<2>(codes, scale), pair_bf16<3>(codes, scale)};
    } else {
        const uint32_t t[4] = {pair_bf16<0>(codes, scale), pair_bf16<1>(codes, scale), pair_bf16<2>(codes, scale), pair_bf16<3>(codes, scale)};
        *(u32x4*)to = u32x4{t[0] << 16, t[0] & 0xFFFF0000u, t[1] << 16, t[1] & 0xFFFF0000u};
        *(u32x4*)(to + 16) = u32x4{t[2] << 16, t[2] & 0xFFFF0000u, t[3] << 16, t[3] & 0xFFFF0000u};
    }
}

// Calls `launch(first row, cells)` for parts whose threads stay below 2^31.
template <typename F> static hipError_t in_parts(const CacheView& c, int n, F launch)
{
    const long long per_row = (long long)c.Hkv * (c.Dk + c.Dv) / CELL;
    const int most = (int)((1ll << 31) / per_row) - 1;
    for (int first = 0; first < n; first += most) {
        const int rows = n - first < most ? n - first : most;
        launch(first, (uint32_t)(rows * per_row));
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

hipError_t launch_cache_append_fourbit(const CacheView& c, uint8_t* k_scales, uint8_t* v_scales, int n, const void* k, long long k_row,
                                   long long k_head, const void* v, long long v_row, long long v_head, const int32_t* sequences,
                                   const int32_t* positions, hipStream_t stream)
{
    return in_parts(c, n, [&](int first, uint32_t cells) {
        hipLaunchKernelGGL((c.dtype == 1 ? append_fourbit_kernel<true> : append_fourbit_kernel<false>), dim3((cells + CELL_THREADS - 1) / CELL_THREADS),
                           dim3(CELL_THREADS), 0, stream, c, first, cells, (const unsigned char*)k, k_row, k_head,
                           (const unsigned char*)v, v_row, v_head, k_scales, v_scales, sequences, positions);
    });
}

hipError_t launch_cache_read_fourbit(const CacheView& c, const uint8_t* k_scales, const uint8_t* v_scales, int n, const int32_t* sequences,
                                 const int32_t* positions, void* k, void* v, hipStream_t stream)
{
    return in_parts(c, n, [&](int first, uint32_t cells) {
        hipLaunchKernelGGL((c.dtype == 1 ? read_fourbit_kernel<true> : read_fourbit_kernel<false>), dim3((cells + CELL_THREADS - 1) / CELL_THREADS),
                           dim3(CELL_THREADS), 0, stream, c, first, cells, const_cast<uint8_t*>(k_scales), const_cast<uint8_t*>(v_scales),
                           sequences, positions, (unsigned char*)k, (unsigned char*)v);
    });
}

}  // namespace paep
