// Upkeep of a paged key-value cache: new tokens appended, old positions evicted.
#include "cache_device.h"

namespace paep {

static constexpr int APPEND_THREADS = 256;

// Rows of 16-byte pieces, one thread each: the keys' pieces of a token, then the values', `per_row` together.  Every byte is
// read and written once.
__global__ __launch_bounds__(APPEND_THREADS) void append_kernel(
    CacheView c, int first, int n, int k_pieces, int v_pieces, const unsigned char* __restrict__ k, long long k_row,
    const unsigned char* __restrict__ v, long long v_row, const int32_t* __restrict__ sequences,
    const int32_t* __restrict__ positions, float* __restrict__ mass, long long mass_stride)
{
    const int per_head = k_pieces + v_pieces, per_row = per_head * c.Hkv;
    const long long at = (long long)blockIdx.x * APPEND_THREADS + threadIdx.x;
    const long long i = first + at / per_row;
    if (i >= n) return;
    const int piece = (int)(at % per_row);
    const int b = sequences ? sequences[i] : (int)i, p = positions[i];
    if ((uint32_t)b >= (uint32_t)c.B || p < 0) return;
    const int page = page_entry(c.table, c.max_pages, c.n_pages, b, p >> c.page_shift);
    if (page < 0) return;
    const int slot = p & ((1 << c.page_shift) - 1);
    const int k_all = k_pieces * c.Hkv;
    if (piece < k_all) {
        const int h = piece / k_pieces, q = piece - h * k_pieces;
        *(u32x4*)(c.k + page * c.k_page + h * c.k_head + slot * c.k_slot + q * 16) = *(const u32x4*)(k + i * k_row + piece * 16ll);
        if (q == 0 && mass && p < mass_stride) mass[((long long)b * c.Hkv + h) * mass_stride + p] = 0.0f;
    } else {
        const int r = piece - k_all, h = r / v_pieces, q = r - h * v_pieces;
        *(u32x4*)(c.v + page * c.v_page + h * c.v_head + slot * c.v_slot + q * 16) = *(const u32x4*)(v + i * v_row + r * 16ll);
    }
}

hipError_t launch_cache_append(const CacheView& c, int n, const void* k, long long k_row, const void* v, long long v_row,
                               const int32_t* sequences, const int32_t* positions, float* mass, long long mass_stride,
                               hipStream_t stream)
{
    const int s = c.dtype == 1 ? 2 : 4, kp = c.Dk * s / 16, vp = c.Dv * s / 16;
    const long long per_row = (long long)c.Hkv * (kp + vp);
    const int most = (int)((1ll << 31) / per_row);           // rows of a launch: its threads stay below 2^32
    for (int first = 0; first < n; first += most) {
        const int part = n - first < most ? n - first : most;
        hipLaunchKernelGGL(append_kernel, dim3((unsigned)((part * per_row + APPEND_THREADS - 1) / APPEND_THREADS)),
                           dim3(APPEND_THREADS), 0, stream, c, first, first + part, kp, vp, (const unsigned char*)k, k_row,
                           (const unsigned char*)v, v_row, sequences, positions, mass, mass_stride);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

// ---------------------------------------------------------------------------
// Eviction.  Kernel 1: which positions each head keeps; kernel 2: their rows are copied.
// ---------------------------------------------------------------------------
static constexpr int SEL_THREADS = 1024, SEL_WAVES = SEL_THREADS / 64;

// A workgroup per sequence and head.  The (budget - recent)-th largest mass is found digit by digit on the ordered 32-bit
// patterns (four histograms of 8 bits in LDS); everything above it is kept, and of its equals the lowest positions.
__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(
    int Hkv, int max_len, int budget, int recent, const int32_t* __restrict__ lengths, const float* __restrict__ mass,
    long long mass_stride, int32_t* __restrict__ kept, float* __restrict__ mass_out, long long mass_out_stride,
    int32_t* __restrict__ lengths_out)
{
    __shared__ uint32_t hist[256], chosen[2];
    __shared__ uint32_t totals[SEL_WAVES];
    const int b = blockIdx.x / Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = clamped_length(lengths, b, max_len);
    const float* in = mass + (long long)blockIdx.x * mass_stride;
    int32_t* ids = kept + (long long)blockIdx.x * budget;
    float* out = mass_out + (long long)blockIdx.x * mass_out_stride;
    const int keep = n < budget ? n : budget;
    if (blockIdx.x % Hkv == 0 && tid == 0) lengths_out[b] = keep;
    for (int j = keep + tid; j < budget; j += SEL_THREADS) ids[j] = -1;
    for (int j = keep + tid; j < mass_out_stride; j += SEL_THREADS) out[j] = 0.0f;
    if (n <= budget) {
        for (int j = tid; j < n; j += SEL_THREADS) { ids[j] = j; out[j] = in[j]; }
        return;
    }
    const int old = n - recent, best = budget - recent;
    for (int j = tid; j < recent; j += SEL_THREADS) { ids[best + j] = old + j; out[best + j] = in[old + j]; }
    if (best == 0) return;

    uint32_t threshold = 0, need = best;                     // the threshold's digits so far, and its rank among the keys that share them
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int p = tid; p < old; p += SEL_THREADS) {
            const uint32_t key = orderable(in[p]);
            if (shift == 24 || (key >> (shift + 8)) == (threshold >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (wave == 0) {                                     // lane l: digits 255 - 4l .. 252 - 4l
            uint32_t c[4], sum = 0;
            for (int u = 0; u < 4; ++u) { c[u] = hist[255 - 4 * lane - u]; sum += c[u]; }
            uint32_t upto = sum;                             // inclusive over lanes
            for (int s = 1; s < 64; s <<= 1) {
                const uint32_t o = __shfl_up(upto, s, 64);
                if (lane >= s) upto += o;
            }
            uint32_t before = upto - sum;
            for (int u = 0; u < 4; ++u) {
                if (before < need && need <= before + c[u]) { chosen[0] = 255 - 4 * lane - u; chosen[1] = need - before; }
                before += c[u];
            }
        }
        __syncthreads();
        threshold |= chosen[0] << shift;
        need = chosen[1];
        __syncthreads();
    }
    // in ascending position: everything above the threshold and the first `need` at it
    uint32_t above = 0, equal = 0;                           // of the positions before this tile
    for (int p0 = 0; p0 < old; p0 += SEL_THREADS) {
        const int p = p0 + tid;
        const float m = p < old ? in[p] : 0.0f;
        const uint32_t key = orderable(m);
        const bool gt = p < old && key > threshold, eq = p < old && key == threshold;
        const unsigned long long bg = __ballot(gt), be = __ballot(eq), lower = (1ull << lane) - 1;
        if (lane == 0) totals[wave] = (uint32_t)__popcll(bg) | (uint32_t)__popcll(be) << 16;
        __syncthreads();
        uint32_t g = above + (uint32_t)__popcll(bg & lower), e = equal + (uint32_t)__popcll(be & lower);
        for (int w = 0; w < SEL_WAVES; ++w) {
            const uint32_t t = totals[w];
            if (w < wave) { g += t & 0xFFFFu; e += t >> 16; }
            above += t & 0xFFFFu;
            equal += t >> 16;
        }
        if (gt || (eq && e < need)) {
            const uint32_t j = g + (e < need ? e : need);
            ids[j] = p;
            out[j] = m;
        }
        __syncthreads();
    }
}

static constexpr int MOVE_THREADS = 256, MOVE_ROWS = 64;

// A workgroup per sequence, head and MOVE_ROWS kept positions: 16-byte pieces of their keys and values.
__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(CacheView c, int k_pieces, int v_pieces, int budget, int parts,
                                                                  const int32_t* __restrict__ kept,
                                                                  const int32_t* __restrict__ out_table, int out_max_pages)
{
    const int row = blockIdx.x / parts, part = blockIdx.x % parts;
    const int b = row / c.Hkv, h = row % c.Hkv, slots = (1 << c.page_shift) - 1;
    const int32_t* ids = kept + (long long)row * budget;
    const int per = k_pieces + v_pieces;
    for (int i = threadIdx.x; i < MOVE_ROWS * per; i += MOVE_THREADS) {
        const int j = part * MOVE_ROWS + i / per, piece = i % per;
        if (j >= budget) break;
        const int p = ids[j];
        if (p < 0) continue;
        const int from = page_entry(c.table, c.max_pages, c.n_pages, b, p >> c.page_shift);
        const int to = page_entry(out_table, out_max_pages, c.n_pages, b, j >> c.page_shift);
        if (from < 0 || to < 0) continue;
        if (piece < k_pieces)
            *(u32x4*)(c.k + to * c.k_page + h * c.k_head + (j & slots) * c.k_slot + piece * 16) =
                *(const u32x4*)(c.k + from * c.k_page + h * c.k_head + (p & slots) * c.k_slot + piece * 16);
        else
            *(u32x4*)(c.v + to * c.v_page + h * c.v_head + (j & slots) * c.v_slot + (piece - k_pieces) * 16) =
                *(const u32x4*)(c.v + from * c.v_page + h * c.v_head + (p & slots) * c.v_slot + (piece - k_pieces) * 16);
    }
}

hipError_t launch_cache_evict(const CacheView& c, int max_len, int budget, int recent, const int32_t* lengths,
                              const float* mass, long long mass_stride, const int32_t* out_table, int out_max_pages,
                              int32_t* kept, float* mass_out, long long mass_out_stride, int32_t* lengths_out,
                              hipStream_t stream)
{
    hipLaunchKernelGGL(evict_select_kernel, dim3(c.B * c.Hkv), dim3(SEL_THREADS), 0, stream, c.Hkv, max_len, budget, recent,
                       lengths, mass, mass_stride, kept, mass_out, mass_out_stride, lengths_out);
    hipError_t err = hipGetLastError();
    const int most = budget < max_len ? budget : max_len, parts = (most + MOVE_ROWS - 1) / MOVE_ROWS;
    if (err != hipSuccess || parts == 0) return err;
    const int s = c.dtype == 1 ? 2 : 4;
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)((long long)c.B * c.Hkv * parts)), dim3(MOVE_THREADS), 0, stream, c,
                       c.Dk * s / 16, c.Dv * s / 16, budget, parts, kept, out_table, out_max_pages);
    return hipGetLastError();
}

}  // namespace paep
