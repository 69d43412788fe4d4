// Attention of one new token per sequence over a paged key-value cache.
#include "cache_device.h"

namespace paep {

static constexpr int ATT_THREADS = 256;

template <bool BF16> __device__ __forceinline__ float element(const unsigned char* p, int i)
{
    if constexpr (BF16) return bf16_bits_to_f32(((const uint16_t*)p)[i]);
    else return ((const float*)p)[i];
}

// A workgroup per sequence and key-value head, one query head after the other; a wave per key, four keys at a time.
template <bool BF16>
__global__ __launch_bounds__(ATT_THREADS) void attend_simple_kernel(AttendArgs a)
{
    const int G = a.Hq / a.c.Hkv, b = blockIdx.x / a.c.Hkv, g = blockIdx.x % a.c.Hkv;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int len = clamped_length(a.lengths, b, a.max_len);
    const int start = a.starts && a.starts[b] > 0 ? a.starts[b] : 0;
    __shared__ float part_m[4], part_l[4], part_o[4][256], tops[1024], sums[1024];
    const int slots = (1 << a.c.page_shift) - 1;
    float qv[4];
    auto load_q = [&](int h) {
        const unsigned char* q = (const unsigned char*)a.q + b * a.q_seq + h * a.q_head;
        for (int i = 0; i < 4; ++i) qv[i] = lane + 64 * i < a.c.Dk ? element<BF16>(q, lane + 64 * i) : 0.0f;
    };
    auto score = [&](int p, long long page) {
        const unsigned char* k = a.c.k + page * a.c.k_page + g * a.c.k_head + (p & slots) * a.c.k_slot;
        float s = 0.0f;
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < a.c.Dk) s = fmaf(qv[i], element<BF16>(k, lane + 64 * i), s);
        for (int mask = 1; mask < 64; mask <<= 1) s += __shfl_xor(s, mask, 64);
        return s * a.scale;
    };
    for (int h = g * G; h < (g + 1) * G; ++h) {
        load_q(h);
        float m = -__builtin_inff(), l = 0.0f, o[4] = {};
        for (int p = start + wave; p < len; p += 4) {
            const int page = page_entry(a.c.table, a.c.max_pages, a.c.n_pages, b, p >> a.c.page_shift);
            if (page < 0) continue;
            const float s = score(p, page), mn = fmaxf(m, s), ms = mn == -__builtin_inff() ? 0.0f : mn;
            const float r = __expf(m - ms), e = __expf(s - ms);
            const unsigned char* v = a.c.v + page * a.c.v_page + g * a.c.v_head + (p & slots) * a.c.v_slot;
            l = l * r + e;
            for (int i = 0; i < 4; ++i)
                if (lane + 64 * i < a.c.Dv) o[i] = fmaf(e, element<BF16>(v, lane + 64 * i), o[i] * r);
            m = mn;
        }
        __syncthreads();
        if (lane == 0) { part_m[wave] = m; part_l[wave] = l; }
        for (int i = 0; i < 4; ++i) part_o[wave][lane + 64 * i] = o[i];
        __syncthreads();
        float top = fmaxf(fmaxf(part_m[0], part_m[1]), fmaxf(part_m[2], part_m[3]));
        if (top == -__builtin_inff()) top = 0.0f;
        float sum = 0.0f, w[4];
        for (int u = 0; u < 4; ++u) { w[u] = __expf(part_m[u] - top); sum += w[u] * part_l[u]; }
        const long long row = (long long)b * a.Hq + h;
        if ((int)threadIdx.x < a.c.Dv) {
            float acc = 0.0f;
            for (int u = 0; u < 4; ++u) acc += w[u] * part_o[u][threadIdx.x];
            acc = sum == 0.0f ? 0.0f : acc / sum;
            if constexpr (BF16) ((uint16_t*)a.out)[row * a.c.Dv + threadIdx.x] = f32_to_bf16_bits(acc);
            else ((float*)a.out)[row * a.c.Dv + threadIdx.x] = acc;
        }
        if (threadIdx.x == 0) {
            if (a.lse) a.lse[row] = top + logf(sum);
            tops[h - g * G] = top;
            sums[h - g * G] = sum;
        }
    }
    if (!a.mass) return;
    __syncthreads();
    float* mass = a.mass + ((long long)b * a.c.Hkv + g) * a.mass_stride;
    for (int p = start + wave; p < len; p += 4) {
        const int page = page_entry(a.c.table, a.c.max_pages, a.c.n_pages, b, p >> a.c.page_shift);
        if (page < 0) continue;
        float w = 0.0f;
        for (int h = 0; h < G; ++h) {
            load_q(g * G + h);
            if (sums[h] != 0.0f) w += __expf(score(p, page) - tops[h]) / sums[h];
        }
        if (lane == 0) mass[p] += w;
    }
}

bool attend_fits(const AttendArgs& a) { return (long long)a.c.B * a.c.Hkv < (1ll << 23); }

size_t attend_workspace_bytes(const AttendArgs&) { return 0; }

hipError_t launch_attend(const AttendArgs& a)
{
    hipLaunchKernelGGL((a.c.dtype == 1 ? attend_simple_kernel<true> : attend_simple_kernel<false>), dim3(a.c.B * a.c.Hkv),
                       dim3(ATT_THREADS), 0, a.stream, a);
    return hipGetLastError();
}

}  // namespace paep
