// A mixture-of-experts layer for a few tokens.
#include "../../include/paep.h"

#include "paep_device.h"
#include "paep_internal.h"

namespace paep {

static constexpr int MOE_THREADS = 256;

template <bool BF16> __device__ __forceinline__ float element(const void* p, long long i)
{
    if constexpr (BF16) return bf16_bits_to_f32(((const uint16_t*)p)[i]);
    else return ((const float*)p)[i];
}

__device__ __forceinline__ float wave_sum(float s)
{
    for (int mask = 1; mask < 64; mask <<= 1) s += __shfl_xor(s, mask, 64);
    return s;
}

// a wave per token and expert
template <bool BF16>
__global__ __launch_bounds__(MOE_THREADS) void router_simple_kernel(MoeArgs a, float* __restrict__ z)
{
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (i >= a.T * a.E) return;
    const int t = i / a.E, e = i % a.E;
    float s = 0.0f;
    for (int c = lane; c < a.d; c += 64) s = fmaf(element<BF16>(a.x, (long long)t * a.d + c), element<BF16>(a.Wg, (long long)e * a.d + c), s);
    s = wave_sum(s);
    if (lane == 0) z[i] = s;
}

// the weight of position p = t * k + j: 0 where its id is none or stood earlier in the row, else the sum over the id's places
__device__ __forceinline__ float position_weight(const int32_t* idx, const float* probs, int k, int E, int p)
{
    const int t0 = p / k * k, e = idx[p];
    if ((uint32_t)e >= (uint32_t)E) return 0.0f;
    float w = 0.0f;
    for (int q = t0; q < t0 + k; ++q)
        if (idx[q] == e) {
            if (q < p) return 0.0f;
            w += probs[q];
        }
    return w;
}

// a wave per position and inner unit
template <bool BF16>
__global__ __launch_bounds__(MOE_THREADS) void up_simple_kernel(MoeArgs a, float* __restrict__ h)
{
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (i >= (long long)a.T * a.k * a.f) return;
    const int p = (int)(i / a.f), u = (int)(i % a.f), t = p / a.k, e = a.idx[p];
    if ((uint32_t)e >= (uint32_t)a.E) return;
    const long long row = ((long long)e * 2 * a.f + u) * a.d;
    float g = 0.0f, w = 0.0f;
    for (int c = lane; c < a.d; c += 64) {
        const float x = element<BF16>(a.x, (long long)t * a.d + c);
        g = fmaf(x, element<BF16>(a.W13, row + c), g);
        w = fmaf(x, element<BF16>(a.W13, row + (long long)a.f * a.d + c), w);
    }
    g = wave_sum(g);
    w = wave_sum(w);
    if (lane == 0) h[i] = position_weight(a.idx, a.probs, a.k, a.E, p) * apply_act(g, a.act) * w;
}

// a wave per token and output unit
template <bool BF16>
__global__ __launch_bounds__(MOE_THREADS) void down_simple_kernel(MoeArgs a, const float* __restrict__ h)
{
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (i >= (long long)a.T * a.d) return;
    const int t = (int)(i / a.d), c = (int)(i % a.d);
    float y = 0.0f;
    for (int j = 0; j < a.k; ++j) {
        const int e = a.idx[t * a.k + j];
        if ((uint32_t)e >= (uint32_t)a.E) continue;
        for (int u = lane; u < a.f; u += 64)
            y = fmaf(h[((long long)t * a.k + j) * a.f + u], element<BF16>(a.W2, ((long long)e * a.d + c) * a.f + u), y);
    }
    y = wave_sum(y);
    if (lane) return;
    if (a.residual) y += element<BF16>(a.residual, i);
    if constexpr (BF16) ((uint16_t*)a.y)[i] = f32_to_bf16_bits(y);
    else ((float*)a.y)[i] = y;
}

size_t moe_workspace_bytes(const MoeArgs& a) { return 4 * ((size_t)a.T * a.k * a.f + (size_t)a.T * a.E); }

template <bool BF16> static hipError_t launch(const MoeArgs& a)
{
    float* h = (float*)a.workspace;
    float* z = h + (size_t)a.T * a.k * a.f;
    auto grid = [](long long waves) { return dim3((unsigned)((waves + 3) / 4)); };
    if (a.Wg) {
        hipLaunchKernelGGL(router_simple_kernel<BF16>, grid(a.T * a.E), dim3(MOE_THREADS), 0, a.stream, a, z);
        PredictArgs r{};
        r.T = a.T; r.E = a.E; r.k = a.k; r.L = 1; r.dtype = a.dtype; r.b2 = a.bg;
        r.idx = a.idx; r.probs = a.probs; r.counts = a.counts; r.prob_mode = a.prob_mode; r.stream = a.stream;
        const hipError_t err = launch_finalize(r, z, 1, 1, a.T, 0, 1);
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL(up_simple_kernel<BF16>, grid((long long)a.T * a.k * a.f), dim3(MOE_THREADS), 0, a.stream, a, h);
    hipLaunchKernelGGL(down_simple_kernel<BF16>, grid((long long)a.T * a.d), dim3(MOE_THREADS), 0, a.stream, a, h);
    return hipGetLastError();
}

hipError_t launch_moe(const MoeArgs& a) { return a.dtype == PAEP_BF16 ? launch<true>(a) : launch<false>(a); }

}  // namespace paep
