// Host-side launcher prototypes shared between the C-ABI layer and the kernel
// translation units.  Every launcher assumes its arguments were validated by
// the C-ABI layer and returns the hipError_t of its launches.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

namespace paep {

struct PredictArgs {
    int T, d, r, E, k, L, dtype, act;
    long long x_stride, w1_stride, w2_stride;   // elements
    const void* x;
    const void* W1;
    const void* W2;
    const void* b1;
    const void* b2;
    int32_t* idx;
    float* probs;
    float* logits;      // nullable
    int32_t* counts;    // nullable: [L][E] activation counts, added to
    int prob_mode;      // 0 softmax over all E, 1 softmax over the k selected, 2 sigmoid
    float* margin;      // nullable: [L][T] last selected score minus the best score left out
    void* workspace;    // null: the call does without
    size_t workspace_bytes;
    hipStream_t stream;
};

// A kernel's dynamic-LDS limit is raised once per (kernel instantiation, device),
// not on every launch: `bytes` remembers what has been granted on each device.
struct LdsLimit {
    std::atomic<int> bytes[16];
};
inline hipError_t ensure_lds_limit(LdsLimit& st, const void* kern, size_t lds)
{
    int dev = 0;
    hipError_t err = hipGetDevice(&dev);
    if (err != hipSuccess) return err;
    const bool tracked = dev >= 0 && dev < 16;
    if (tracked && (int)lds <= st.bytes[dev].load(std::memory_order_relaxed)) return hipSuccess;
    err = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (err == hipSuccess && tracked) st.bytes[dev].store((int)lds, std::memory_order_relaxed);
    return err;
}

// adds `S` slices of partial scores, laid out [tile][slice][BM][E] from tile `tile0` on, and finishes their rows
// (softmax, top-k); decode, fp32 and prefill calls that cut r over workgroups end with it
hipError_t launch_finalize(const PredictArgs& a, const float* partial, int S, int tiles, int BM, int tile0,
                           int tiles_per_layer);

// fp32 storage, any shape: fp32 matrix instructions
bool f32_supported(const PredictArgs& a);
size_t f32_workspace_bytes(const PredictArgs& a);
hipError_t launch_predict_f32(const PredictArgs& a);

// bf16 storage, shapes that the matrix-core kernels do not take: plain vector arithmetic
bool simple_supported(const PredictArgs& a);
hipError_t launch_predict_simple(const PredictArgs& a);

// bf16 weight-streaming kernel for T <= 64
bool decode_supported(const PredictArgs& a);
size_t decode_workspace_bytes(const PredictArgs& a);
size_t decode_workspace_min(const PredictArgs& a);       // with less than this the call is refused
hipError_t launch_predict_decode(const PredictArgs& a);

// bf16 fused matrix-core kernel for large T
bool prefill_supported(const PredictArgs& a);
size_t prefill_workspace_bytes(const PredictArgs& a);
size_t prefill_workspace_min(const PredictArgs& a);      // with less than this the call is refused
hipError_t launch_predict_prefill(const PredictArgs& a);
// tile configuration id, workgroups per token tile, chunks of r per workgroup (what the launcher will use, given the
// workspace of prefill_workspace_bytes)
void prefill_plan(const PredictArgs& a, int* cfg, int* groups, int* chunks_per_group);
// what the launcher runs in a workspace of a.workspace_bytes: kernel, token x hidden-unit tile, order of the grid
const char* prefill_kernel_name(const PredictArgs& a);

size_t group_workspace_bytes(int L, int T, int k, int E);
hipError_t launch_group(const int32_t* idx, int L, int T, int k, int E,
                        int32_t* counts, int32_t* offsets, int32_t* token_pos,
                        int32_t* active, int32_t* n_active, int32_t* n_invalid,
                        void* workspace, hipStream_t stream);

hipError_t launch_fold_batchnorm(const void* W1, const void* b1, const float* gamma, const float* beta,
                                 const float* mean, const float* var, float eps, int L, int r, int d, int dtype,
                                 void* W1_out, void* b1_out, hipStream_t stream);

hipError_t launch_activation_profile(const int32_t* counts, int L, int E, int32_t* order, int32_t* n_active,
                                     double* entropy, hipStream_t stream);

// device-ceiling probes
static constexpr int PROBE_READ_GROUPS = 4096;
hipError_t launch_probe_read(const void* src, size_t bytes, void* sink, hipStream_t stream);
hipError_t launch_probe_mfma(int groups, int iters, void* sink, hipStream_t stream);

hipError_t launch_score(const int32_t* idx, int k_pred, const int32_t* ref, int k_ref,
                        int L, int T, int E, const int32_t* k_row, long long* counters, hipStream_t stream);
hipError_t launch_confidence_select(const int32_t* idx, const float* probs, int L, int T, int k_pred, int k_base,
                                    float ratio, int32_t* idx_out, int32_t* k_row, int32_t* n_wide,
                                    hipStream_t stream);


// ---- paged key-value cache, attention of one new token, expert layer ----

// A cache as the kernels see it: strides in bytes, page_size = 1 << page_shift.
struct CacheView {
    int B, Hkv, Dk, Dv, page_shift, n_pages, max_pages, dtype;
    long long k_page, k_head, k_slot, v_page, v_head, v_slot;
    const int32_t* table;
    unsigned char* k;
    unsigned char* v;
};

struct AttendArgs {
    CacheView c;
    int Hq, max_len;
    float scale;
    long long q_seq, q_head;       // bytes
    const void* q;
    const int32_t* lengths;
    const int32_t* starts;         // nullable
    void* out;
    float* lse;                    // nullable
    float* mass;                   // nullable
    long long mass_stride;         // floats
    void* workspace;
    hipStream_t stream;
};
bool attend_fits(const AttendArgs& a);                       // the grid holds this shape
size_t attend_workspace_bytes(const AttendArgs& a);          // (a.mass: whether there is one)
hipError_t launch_attend(const AttendArgs& a);

// over a cache in 4 bits: strides of the view count bytes of codes; its dtype is that of q and out
struct AttendFourbitArgs {
    AttendArgs a;
    const uint8_t* k_scales;       // [n_pages][Hkv][Dk / 32][page size]
    const uint8_t* v_scales;
};
bool attend_fourbit_fits(const AttendFourbitArgs& a);
size_t attend_fourbit_workspace_bytes(const AttendFourbitArgs& a);
hipError_t launch_attend_fourbit(const AttendFourbitArgs& a);

hipError_t launch_cache_append(const CacheView& c, int n, const void* k, long long k_row, const void* v, long long v_row,
                               const int32_t* sequences, const int32_t* positions, float* mass, long long mass_stride,
                               hipStream_t stream);
hipError_t launch_cache_evict(const CacheView& c, int max_len, int budget, int recent, const int32_t* lengths,
                              const float* mass, long long mass_stride, const int32_t* out_table, int out_max_pages,
                              int32_t* kept, float* mass_out, long long mass_out_stride, int32_t* lengths_out,
                              hipStream_t stream);

// the same for a cache in 4 bits (scales as in AttendFourbitArgs; strides of k and v in bytes)
hipError_t launch_cache_append_fourbit(const CacheView& c, uint8_t* k_scales, uint8_t* v_scales, int n, const void* k, long long k_row,
                                   long long k_head, const void* v, long long v_row, long long v_head, const int32_t* sequences,
                                   const int32_t* positions, hipStream_t stream);
hipError_t launch_cache_read_fourbit(const CacheView& c, const uint8_t* k_scales, const uint8_t* v_scales, int n, const int32_t* sequences,
                                 const int32_t* positions, void* k, void* v, hipStream_t stream);

// norms and rotation of queries and keys; append: the keys, and the values, go into the cache
struct RotateArgs {
    int n, Hq, Hk, D, rot, table_rows, dtype, style;
    float eps;
    bool append;
    const void* q;
    const void* k;
    void* q_out;
    void* k_out;                   // (without append)
    long long q_row, q_head, k_row, k_head, q_out_row, q_out_head, k_out_row, k_out_head;      // bytes
    const void* q_weight;          // nullable: no norm
    const void* k_weight;
    const int32_t* angles;         // rows of the table
    const float* table;            // [table_rows][rot]
    // with append
    CacheView c;
    const void* v;
    long long v_row, v_head;       // bytes
    const int32_t* sequences;      // nullable
    const int32_t* positions;
    float* mass;                   // nullable
    long long mass_stride;
    hipStream_t stream;
};
hipError_t launch_rotate(const RotateArgs& a);

struct MoeArgs {
    int T, d, f, E, k, dtype, act, prob_mode;
    const void* x;
    const void* Wg;                // null: idx and probs are inputs
    const void* bg;                // nullable
    const void* W13;
    const void* W2;
    const void* residual;          // nullable
    void* y;
    int32_t* idx;
    float* probs;
    int32_t* counts;               // nullable
    void* workspace;
    hipStream_t stream;
};
size_t moe_workspace_bytes(const MoeArgs& a);
hipError_t launch_moe(const MoeArgs& a);

}  // namespace paep
