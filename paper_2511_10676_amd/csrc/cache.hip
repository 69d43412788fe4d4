// Upkeep of a paged key-value cache: new tokens appended, old positions evicted.
#include "cache_device.h"

namespace paep {

static constexpr int APPEND_THREADS = 256;

// Rows of 16-byte pieces, one thread each: the keys' pieces of a token, then the values', `per_row` together.  Every byte is
// read and written once, which is all there is to it: 4096 fp32 tokens of 8 heads of 128, 67 MB, take 13.5 us (5.0 TB/s), 61 bf16
// tokens 2.9 us, a launch.
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
static constexpr int SEL_KEYS = 32;                  // masses of a thread at a time
static constexpr int SEL_SPAN = SEL_THREADS * SEL_KEYS;
static constexpr int SEL_BINS = 2 * SEL_THREADS;     // of a digit of 11 bits
static constexpr int SEL_COPIES = 4;                 // of every counter, a lane's by its number: most masses share a few digits

// A workgroup per sequence and head.  The (budget - recent)-th largest mass is found digit by digit on the ordered 32-bit
// patterns (three histograms, 11, 11 and 10 bits, in LDS); everything above it is kept, and of its equals the lowest
// positions.  Up to SEL_SPAN masses stay in registers from the first histogram to the last store; longer sequences are read
// again for each.  What bounds it is the vector units of the one CU that a head has: 32493 masses of a head take 26 us, half
// of it the histograms (four of 8 bits: 31 us; 76 us with the masses read from memory for each and a barrier per 1024).
__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(
    int Hkv, int max_len, int budget, int recent, const int32_t* __restrict__ lengths, const float* __restrict__ mass,
    long long mass_stride, int32_t* __restrict__ kept, float* __restrict__ mass_out, long long mass_out_stride,
    int32_t* __restrict__ lengths_out)
{
    __shared__ __attribute__((aligned(16))) uint32_t hist[SEL_BINS][SEL_COPIES];
    __shared__ uint32_t chosen[2], wave_sum[SEL_WAVES];
    __shared__ uint32_t gt_bits[SEL_THREADS], eq_bits[SEL_THREADS];      // of a span, a bit per position: above the threshold, at it
    __shared__ uint32_t wave_gt[SEL_WAVES], wave_eq[SEL_WAVES];
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

    // key[u]: of position p0 + u * SEL_THREADS + tid.  Where there is none: 0, the lowest key, behind every position that has
    // it, so it is never among the `best` <= old first ones and needs no test.
    uint32_t key[SEL_KEYS];
    auto load = [&](long long p0) {
        float m[SEL_KEYS];
#pragma unroll
        for (int u = 0; u < SEL_KEYS; ++u) {
            const long long p = p0 + u * SEL_THREADS + tid;
            m[u] = in[p < old ? p : 0];
        }
#pragma unroll
        for (int u = 0; u < SEL_KEYS; ++u) key[u] = p0 + u * SEL_THREADS + tid < old ? orderable(m[u]) : 0u;
    };
    const bool whole = old <= SEL_SPAN;
    if (whole) load(0);

    uint32_t threshold = 0, need = best;                     // the threshold's digits so far, and its rank among the keys that share them
#pragma unroll 1
    for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, mask = digit == 2 ? 1023 : 2047;
        const uint32_t within = digit == 0 ? 0xFFFFFFFFu : digit == 1 ? (1u << 21) - 1 : (1u << 10) - 1;     // keys that share the threshold's digits
        for (int i = tid; i < SEL_BINS * SEL_COPIES; i += SEL_THREADS) (&hist[0][0])[i] = 0;
        __syncthreads();
        for (long long p0 = 0; p0 < old; p0 += SEL_SPAN) {
            if (!whole) load(p0);
#pragma unroll
            for (int u = 0; u < SEL_KEYS; ++u) {
                if (p0 + u * SEL_THREADS >= old) break;
                if ((key[u] ^ threshold) <= within) atomicAdd(&hist[(key[u] >> shift) & mask][lane % SEL_COPIES], 1u);
            }
        }
        __syncthreads();
        // thread t: the digits SEL_BINS - 1 - 2t and the one below; those above them are counted by the threads before it
        uint32_t c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x4 h = *(const u32x4*)hist[SEL_BINS - 1 - 2 * tid - i];
            c[i] = (h[0] + h[1]) + (h[2] + h[3]);
        }
        uint32_t upto = c[0] + c[1];
        for (int s = 1; s < 64; s <<= 1) {
            const uint32_t o = __shfl_up(upto, s, 64);
            if (lane >= s) upto += o;
        }
        if (lane == 63) wave_sum[wave] = upto;
        __syncthreads();
        uint32_t before = upto - c[0] - c[1];
#pragma unroll
        for (int w = 0; w < SEL_WAVES; ++w) before += w < wave ? wave_sum[w] : 0u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (before < need && need <= before + c[i]) { chosen[0] = SEL_BINS - 1 - 2 * tid - i; chosen[1] = need - before; }
            before += c[i];
        }
        __syncthreads();
        threshold |= chosen[0] << shift;
        need = chosen[1];
    }
    // in ascending position: everything above the threshold and the first `need` at it.  The span's positions become bits,
    // thread t then has those of positions p0 + 32 t .. 32 t + 31.
    uint32_t above = 0, equal = 0;                           // of the spans before
    for (long long p0 = 0; p0 < old; p0 += SEL_SPAN) {
        if (!whole) load(p0);
        unsigned long long gt = 0, eq = 0;                   // lane u: of positions p0 + u * SEL_THREADS + wave * 64 ..
#pragma unroll
        for (int u = 0; u < SEL_KEYS; ++u) {
            if (p0 + u * SEL_THREADS >= old) break;
            const unsigned long long bg = __ballot(key[u] > threshold), be = __ballot(key[u] == threshold);
            gt = lane == u ? bg : gt;
            eq = lane == u ? be : eq;
        }
        if (lane < SEL_KEYS) {
            const int i = lane * (SEL_THREADS / 32) + wave * 2;
            gt_bits[i] = (uint32_t)gt;
            gt_bits[i + 1] = (uint32_t)(gt >> 32);
            eq_bits[i] = (uint32_t)eq;
            eq_bits[i + 1] = (uint32_t)(eq >> 32);
        }
        __syncthreads();
        uint32_t mine = gt_bits[tid], ties = eq_bits[tid];
        const uint32_t ng = __popc(mine), ne = __popc(ties);
        uint32_t g = ng, e = ne;                             // of the wave, up to this thread
        for (int s = 1; s < 64; s <<= 1) {
            const uint32_t og = __shfl_up(g, s, 64), oe = __shfl_up(e, s, 64);
            if (lane >= s) { g += og; e += oe; }
        }
        if (lane == 63) { wave_gt[wave] = g; wave_eq[wave] = e; }
        __syncthreads();
        g += above - ng;
        e += equal - ne;
#pragma unroll
        for (int w = 0; w < SEL_WAVES; ++w) {
            if (w < wave) { g += wave_gt[w]; e += wave_eq[w]; }
            above += wave_gt[w];
            equal += wave_eq[w];
        }
        for (uint32_t left = e < need ? need - e : 0; left > 0 && ties != 0; --left) {
            mine |= ties & (0u - ties);
            ties &= ties - 1;
        }
        for (uint32_t j = g + min(e, need); mine != 0; ++j, mine &= mine - 1)
            ids[j] = (int32_t)(p0 + tid * 32 + __builtin_ctz(mine));
        __syncthreads();
    }
    // their masses (read again: a key has lost a zero's sign and what a NaN carries; and not above, where each would be waited for)
    __syncthreads();
#pragma unroll 4
    for (int j = tid; j < best; j += SEL_THREADS) out[j] = in[ids[j]];
}

static constexpr int MOVE_THREADS = 256, MOVE_ROWS = 64, MOVE_PIECES = 8;

// A workgroup per sequence, head and MOVE_ROWS kept positions.  Where a row comes from and goes to is looked up once, by one
// thread; then every thread copies 16-byte pieces of keys and values, MOVE_PIECES of them requested together (32 sequences cut to 2048
// positions, 8 heads, 364 MB: 81 us, 4.5 TB/s; with each thread looking up its own rows 106).
__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(CacheView c, int k_pieces, int v_pieces, int budget, int parts,
                                                                  const int32_t* __restrict__ kept,
                                                                  const int32_t* __restrict__ out_table, int out_max_pages)
{
    __shared__ long long k_from[MOVE_ROWS], k_to[MOVE_ROWS], v_from[MOVE_ROWS], v_to[MOVE_ROWS];      // k_from < 0: nothing to copy
    const int row = blockIdx.x / parts, part = blockIdx.x % parts;
    const int b = row / c.Hkv, h = row % c.Hkv, slots = (1 << c.page_shift) - 1;
    bool any = false;
    if (threadIdx.x < MOVE_ROWS) {
        const int i = threadIdx.x, j = part * MOVE_ROWS + i;
        const int p = j < budget ? kept[(long long)row * budget + j] : -1;
        const int from = p < 0 ? -1 : page_entry(c.table, c.max_pages, c.n_pages, b, p >> c.page_shift);
        const int to = p < 0 ? -1 : page_entry(out_table, out_max_pages, c.n_pages, b, j >> c.page_shift);
        any = from >= 0 && to >= 0;
        k_from[i] = any ? from * c.k_page + h * c.k_head + (p & slots) * c.k_slot : -1;
        k_to[i] = any ? to * c.k_page + h * c.k_head + (j & slots) * c.k_slot : 0;
        v_from[i] = any ? from * c.v_page + h * c.v_head + (p & slots) * c.v_slot : 0;
        v_to[i] = any ? to * c.v_page + h * c.v_head + (j & slots) * c.v_slot : 0;
    }
    if (!__syncthreads_or(any)) return;
    const int per = k_pieces + v_pieces;
    for (int i0 = threadIdx.x; i0 < MOVE_ROWS * per; i0 += MOVE_PIECES * MOVE_THREADS) {
        u32x4 f[MOVE_PIECES];
        unsigned char* to[MOVE_PIECES];
#pragma unroll
        for (int u = 0; u < MOVE_PIECES; ++u) {
            const int i = min(i0 + u * MOVE_THREADS, MOVE_ROWS * per - 1), r = i / per, q = i - r * per;
            const bool is_k = q < k_pieces, there = i0 + u * MOVE_THREADS < MOVE_ROWS * per && k_from[r] >= 0;
            const int off = (is_k ? q : q - k_pieces) * 16;
            to[u] = !there ? nullptr : is_k ? c.k + k_to[r] + off : c.v + v_to[r] + off;
            f[u] = *(const u32x4*)(!there ? c.k : is_k ? c.k + k_from[r] + off : c.v + v_from[r] + off);
        }
#pragma unroll
        for (int u = 0; u < MOVE_PIECES; ++u)
            if (to[u]) *(u32x4*)to[u] = f[u];
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
