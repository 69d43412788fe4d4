// C-ABI layer of a decode step's operators beside the predictor (rotation,
// attention over a paged key-value cache, the cache's upkeep, the expert layer): argument
// validation on the host, before any HIP call, and dispatch.  See
// include/paep.h for the contract of every entry point.
#include "../../include/paep.h"

#include "paep_internal.h"

#include <math.h>

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// byte size of an element, 0 for an unknown dtype
inline int element_bytes(int dtype) { return dtype == PAEP_F32 ? 4 : dtype == PAEP_BF16 ? 2 : 0; }

constexpr long long MAX_STRIDE = 1ll << 40;                  // elements: byte offsets of 2^31 pages stay below 2^63 with the checks below

// strides of one pool: none overlaps the row it steps over, and the last page's offset fits in 62 bits; per16: elements in 16 bytes
paep_status check_strides(long long page, long long head, long long slot, int width, const paep_cache_desc* c, int per16)
{
    for (long long s : {page, head, slot})
        if (s < 0 || s > MAX_STRIDE) return PAEP_ERR_SHAPE;
    if ((c->n_pages > 1 && page < width) || (c->Hkv > 1 && head < width) || (c->page_size > 1 && slot < width))
        return PAEP_ERR_SHAPE;
    if (page > (1ll << 60) / c->n_pages || head > (1ll << 58) / c->Hkv || slot > (1ll << 58) / c->page_size)
        return PAEP_ERR_SHAPE;
    return page % per16 || head % per16 || slot % per16 ? PAEP_ERR_ALIGN : PAEP_OK;
}

// fourbit: the pools hold elements of 4 bits in groups of 32
paep_status check_cache(const paep_cache_desc* c, bool fourbit = false)
{
    if (!c) return PAEP_ERR_NULL;
    if (!element_bytes(c->dtype)) return PAEP_ERR_DTYPE;
    if (c->B < 0 || c->Hkv < 1 || c->Hkv > PAEP_MAX_HEADS || c->n_pages < 1 || c->max_pages < 1) return PAEP_ERR_SHAPE;
    for (int w : {c->Dk, c->Dv})
        if (w < 8 || w > PAEP_MAX_HEAD_DIM || w % (fourbit ? 32 : 8)) return PAEP_ERR_SHAPE;
    if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return PAEP_ERR_SHAPE;
    const int per16 = fourbit ? 32 : 16 / element_bytes(c->dtype);
    const paep_status st = check_strides(c->k_page_stride, c->k_head_stride, c->k_slot_stride, c->Dk, c, per16);
    return st != PAEP_OK ? st : check_strides(c->v_page_stride, c->v_head_stride, c->v_slot_stride, c->Dv, c, per16);
}

// positions are 32-bit in the kernels, with room for a tile past the last
bool length_ok(const paep_cache_desc* c, long long max_len)
{
    return max_len >= 0 && max_len <= (long long)c->max_pages * c->page_size && max_len <= 0x7FFF0000ll;
}

paep::CacheView to_view(const paep_cache_desc* c, const void* k, const void* v, const int32_t* table)
{
    const long long s = element_bytes(c->dtype);
    paep::CacheView w{};
    w.B = c->B; w.Hkv = c->Hkv; w.Dk = c->Dk; w.Dv = c->Dv; w.n_pages = c->n_pages; w.max_pages = c->max_pages;
    w.dtype = c->dtype;
    while ((1 << w.page_shift) < c->page_size) ++w.page_shift;
    w.k_page = c->k_page_stride * s; w.k_head = c->k_head_stride * s; w.k_slot = c->k_slot_stride * s;
    w.v_page = c->v_page_stride * s; w.v_head = c->v_head_stride * s; w.v_slot = c->v_slot_stride * s;
    w.table = table;
    w.k = static_cast<unsigned char*>(const_cast<void*>(k));
    w.v = static_cast<unsigned char*>(const_cast<void*>(v));
    return w;
}

// the same view with strides in bytes of codes
paep::CacheView to_fourbit_view(const paep_cache_desc* c, const void* k, const void* v, const int32_t* table)
{
    paep::CacheView w = to_view(c, k, v, table);
    w.k_page = c->k_page_stride / 2; w.k_head = c->k_head_stride / 2; w.k_slot = c->k_slot_stride / 2;
    w.v_page = c->v_page_stride / 2; w.v_head = c->v_head_stride / 2; w.v_slot = c->v_slot_stride / 2;
    return w;
}

// strides between the rows of n tokens and between H heads of `width` in a tensor beside the cache; `out`: they may not overlap
paep_status check_rows(long long row, long long head, int n, int H, int width, int dtype, bool out)
{
    for (long long s : {row, head})
        if (s < 0 || s > MAX_STRIDE) return PAEP_ERR_SHAPE;
    if (H > 1 && head < width) return PAEP_ERR_SHAPE;
    if (n > 1 && out && row < width) return PAEP_ERR_SHAPE;
    const int per16 = 16 / element_bytes(dtype);
    if (row % per16 || head % per16) return PAEP_ERR_ALIGN;
    // heads within rows, or rows within heads
    return out && n > 1 && H > 1 && row < (H - 1) * head + width && (__int128)head < (__int128)(n - 1) * row + width ? PAEP_ERR_SHAPE : PAEP_OK;
}

paep_status check_rotate(const paep_rotate_desc* d, bool append)
{
    if (!d) return PAEP_ERR_NULL;
    if (!element_bytes(d->dtype) || (d->style != PAEP_ROTATE_HALVES && d->style != PAEP_ROTATE_PAIRS)) return PAEP_ERR_DTYPE;
    if (d->n < 0 || d->n > (1 << 24) || d->Hq < 0 || d->Hq > PAEP_MAX_HEADS || d->Hk < 0 || d->Hk > PAEP_MAX_HEADS || d->Hq + d->Hk < 1)
        return PAEP_ERR_SHAPE;
    if (d->D < 8 || d->D > PAEP_MAX_HEAD_DIM || d->D % 8 || d->rot < 2 || d->rot > d->D || d->rot % 2 || d->table_rows < 1 || d->reserved != 0)
        return PAEP_ERR_SHAPE;
    if (!isfinite(d->eps) || !(d->eps > 0.0f)) return PAEP_ERR_SHAPE;
    paep_status st = PAEP_OK;
    if (d->Hq > 0) {
        st = check_rows(d->q_row_stride, d->q_head_stride, d->n, d->Hq, d->D, d->dtype, false);
        if (st == PAEP_OK) st = check_rows(d->q_out_row_stride, d->q_out_head_stride, d->n, d->Hq, d->D, d->dtype, true);
    }
    if (d->Hk > 0) {
        if (st == PAEP_OK) st = check_rows(d->k_row_stride, d->k_head_stride, d->n, d->Hk, d->D, d->dtype, false);
        if (st == PAEP_OK && !append) st = check_rows(d->k_out_row_stride, d->k_out_head_stride, d->n, d->Hk, d->D, d->dtype, true);
    }
    return st;
}

paep::RotateArgs to_rotate(const paep_rotate_desc* d, bool append)
{
    const long long s = element_bytes(d->dtype);
    paep::RotateArgs a{};
    a.n = d->n; a.Hq = d->Hq; a.Hk = d->Hk; a.D = d->D; a.rot = d->rot; a.table_rows = d->table_rows; a.dtype = d->dtype; a.style = d->style;
    a.eps = d->eps; a.append = append;
    a.q_row = d->q_row_stride * s; a.q_head = d->q_head_stride * s; a.k_row = d->k_row_stride * s; a.k_head = d->k_head_stride * s;
    a.q_out_row = d->q_out_row_stride * s; a.q_out_head = d->q_out_head_stride * s;
    a.k_out_row = d->k_out_row_stride * s; a.k_out_head = d->k_out_head_stride * s;
    return a;
}

paep_status check_attend(const paep_cache_desc* c, const paep_attend_desc* d, bool mass, bool fourbit = false)
{
    const paep_status st = check_cache(c, fourbit);
    if (st != PAEP_OK) return st;
    if (!d) return PAEP_ERR_NULL;
    if (d->Hq < 1 || d->Hq > PAEP_MAX_HEADS || d->Hq % c->Hkv || d->reserved != 0) return PAEP_ERR_SHAPE;
    if (!length_ok(c, d->max_len) || !isfinite(d->scale)) return PAEP_ERR_SHAPE;
    if (d->q_seq_stride < 0 || d->q_seq_stride > MAX_STRIDE || d->q_head_stride < 0 || d->q_head_stride > MAX_STRIDE)
        return PAEP_ERR_SHAPE;
    if (mass && (d->mass_stride < d->max_len || d->mass_stride > MAX_STRIDE)) return PAEP_ERR_SHAPE;
    const int per16 = 16 / element_bytes(c->dtype);
    return d->q_seq_stride % per16 || d->q_head_stride % per16 ? PAEP_ERR_ALIGN : PAEP_OK;
}

paep::AttendArgs to_attend(const paep_cache_desc* c, const paep_attend_desc* d, const void* k, const void* v, const int32_t* table)
{
    const long long s = element_bytes(c->dtype);
    paep::AttendArgs a{};
    a.c = to_view(c, k, v, table);
    a.Hq = d->Hq; a.max_len = d->max_len; a.scale = d->scale;
    a.q_seq = d->q_seq_stride * s; a.q_head = d->q_head_stride * s; a.mass_stride = d->mass_stride;
    return a;
}

paep_status check_moe(const paep_moe_desc* d)
{
    if (!d) return PAEP_ERR_NULL;
    if (!element_bytes(d->dtype)) return PAEP_ERR_DTYPE;
    if (d->act != PAEP_ACT_NONE && d->act != PAEP_ACT_SILU && d->act != PAEP_ACT_GELU) return PAEP_ERR_DTYPE;
    if (d->prob != PAEP_PROB_SOFTMAX_ALL && d->prob != PAEP_PROB_SOFTMAX_TOPK && d->prob != PAEP_PROB_SIGMOID)
        return PAEP_ERR_DTYPE;
    if (d->T < 0 || d->T > PAEP_MOE_MAX_T || d->E < 1 || d->E > PAEP_MAX_E) return PAEP_ERR_SHAPE;
    if (d->d < 8 || d->d % 8 || d->d > 65536 || d->f < 8 || d->f % 8 || d->f > 65536) return PAEP_ERR_SHAPE;
    if (d->k < 1 || d->k > d->E || d->k > PAEP_MAX_K) return PAEP_ERR_K;
    return PAEP_OK;
}

paep::MoeArgs to_moe(const paep_moe_desc* d)
{
    paep::MoeArgs a{};
    a.T = d->T; a.d = d->d; a.f = d->f; a.E = d->E; a.k = d->k; a.dtype = d->dtype; a.act = d->act; a.prob_mode = d->prob;
    return a;
}

paep_status moe_common(const paep_moe_desc* desc, const void* x, const void* Wg, const void* bg, const void* W13,
                       const void* W2, const void* residual, void* y, int32_t* idx, float* probs, int32_t* counts,
                       void* workspace, size_t workspace_bytes, void* stream)
{
    if (!W13 || !W2 || (desc->T > 0 && (!x || !y || !idx || !probs))) return PAEP_ERR_NULL;
    for (const void* p : {x, Wg, W13, W2, residual, (const void*)y})
        if (!aligned16(p)) return PAEP_ERR_ALIGN;
    paep::MoeArgs a = to_moe(desc);
    const size_t need = paep::moe_workspace_bytes(a);
    if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return PAEP_ERR_WORKSPACE;
    if (desc->T == 0) return PAEP_OK;
    a.x = x; a.Wg = Wg; a.bg = bg; a.W13 = W13; a.W2 = W2; a.residual = residual; a.y = y;
    a.idx = idx; a.probs = probs; a.counts = counts; a.workspace = workspace;
    a.stream = static_cast<hipStream_t>(stream);
    return paep::launch_moe(a) == hipSuccess ? PAEP_OK : PAEP_ERR_HIP;
}

}  // namespace

extern "C" {

size_t paep_attend_workspace_bytes(const paep_cache_desc* cache, const paep_attend_desc* desc, int32_t want_mass)
{
    if (check_attend(cache, desc, want_mass != 0) != PAEP_OK) return 0;
    paep::AttendArgs a = to_attend(cache, desc, nullptr, nullptr, nullptr);
    static float present;                                    // only its address matters: "there is a mass output"
    a.mass = want_mass ? &present : nullptr;
    return paep::attend_fits(a) ? paep::attend_workspace_bytes(a) : 0;
}

paep_status paep_attend(const paep_cache_desc* cache, const paep_attend_desc* desc, const void* q_dev,
                        const void* k_pages_dev, const void* v_pages_dev, const int32_t* page_table_dev,
                        const int32_t* lengths_dev, const int32_t* starts_dev,
                        void* out_dev, float* lse_dev, float* mass_dev,
                        void* workspace_dev, size_t workspace_bytes, void* stream)
{
    const paep_status st = check_attend(cache, desc, mass_dev != nullptr);
    if (st != PAEP_OK) return st;
    if (!k_pages_dev || !v_pages_dev) return PAEP_ERR_NULL;
    if (cache->B > 0 && (!q_dev || !page_table_dev || !lengths_dev || !out_dev)) return PAEP_ERR_NULL;
    if (!aligned16(q_dev) || !aligned16(k_pages_dev) || !aligned16(v_pages_dev) || !aligned16(out_dev)) return PAEP_ERR_ALIGN;
    paep::AttendArgs a = to_attend(cache, desc, k_pages_dev, v_pages_dev, page_table_dev);
    a.mass = mass_dev;
    if (!paep::attend_fits(a)) return PAEP_ERR_SHAPE;
    const size_t need = paep::attend_workspace_bytes(a);
    if (need > 0 && (!workspace_dev || !aligned16(workspace_dev) || workspace_bytes < need)) return PAEP_ERR_WORKSPACE;
    if (cache->B == 0) return PAEP_OK;
    a.q = q_dev; a.lengths = lengths_dev; a.starts = starts_dev; a.out = out_dev; a.lse = lse_dev;
    a.workspace = workspace_dev;
    a.stream = static_cast<hipStream_t>(stream);
    return paep::launch_attend(a) == hipSuccess ? PAEP_OK : PAEP_ERR_HIP;
}

paep_status paep_cache_append(const paep_cache_desc* cache, int32_t n, const void* k_dev, int64_t k_row_stride,
                              const void* v_dev, int64_t v_row_stride, void* k_pages_dev, void* v_pages_dev,
                              const int32_t* page_table_dev, const int32_t* sequences_dev, const int32_t* positions_dev,
                              float* mass_dev, int64_t mass_stride, void* stream)
{
    const paep_status st = check_cache(cache);
    if (st != PAEP_OK) return st;
    if (n < 0 || n > (1 << 24) || (!sequences_dev && n > cache->B)) return PAEP_ERR_SHAPE;
    const long long kw = (long long)cache->Hkv * cache->Dk, vw = (long long)cache->Hkv * cache->Dv;
    if (k_row_stride < 0 || k_row_stride > MAX_STRIDE || v_row_stride < 0 || v_row_stride > MAX_STRIDE) return PAEP_ERR_SHAPE;
    if (n > 1 && (k_row_stride < kw || v_row_stride < vw)) return PAEP_ERR_SHAPE;
    if (mass_dev && (mass_stride < 0 || mass_stride > MAX_STRIDE)) return PAEP_ERR_SHAPE;
    if (!k_pages_dev || !v_pages_dev) return PAEP_ERR_NULL;
    if (n > 0 && (!k_dev || !v_dev || !page_table_dev || !positions_dev)) return PAEP_ERR_NULL;
    const int per16 = 16 / element_bytes(cache->dtype);
    if (k_row_stride % per16 || v_row_stride % per16) return PAEP_ERR_ALIGN;
    if (!aligned16(k_dev) || !aligned16(v_dev) || !aligned16(k_pages_dev) || !aligned16(v_pages_dev)) return PAEP_ERR_ALIGN;
    if (n == 0 || cache->B == 0) return PAEP_OK;
    const long long s = element_bytes(cache->dtype);
    const hipError_t err = paep::launch_cache_append(to_view(cache, k_pages_dev, v_pages_dev, page_table_dev), n, k_dev,
                                                     k_row_stride * s, v_dev, v_row_stride * s, sequences_dev, positions_dev,
                                                     mass_dev, mass_stride, static_cast<hipStream_t>(stream));
    return err == hipSuccess ? PAEP_OK : PAEP_ERR_HIP;
}

paep_status paep_cache_evict(const paep_cache_desc* cache, int32_t max_len, int32_t budget, int32_t recent,
                             void* k_pages_dev, void* v_pages_dev, const int32_t* page_table_dev,
                             const int32_t* lengths_dev, const float* mass_dev, int64_t mass_stride,
                             const int32_t* out_table_dev, int32_t out_max_pages,
                             int32_t* kept_dev, float* mass_out_dev, int64_t mass_out_stride, int32_t* lengths_out_dev,
                             void* stream)
{
    const paep_status st = check_cache(cache);
    if (st != PAEP_OK) return st;
    if (!length_ok(cache, max_len) || out_max_pages < 1 || budget < 1 || recent < 0 || recent > budget) return PAEP_ERR_SHAPE;
    if (budget > (long long)out_max_pages * cache->page_size || budget > 0x7FFF0000) return PAEP_ERR_SHAPE;
    const long long most = budget < max_len ? budget : max_len;
    if (mass_stride < max_len || mass_stride > MAX_STRIDE || mass_out_stride < most || mass_out_stride > 0x7FFF0000ll)
        return PAEP_ERR_SHAPE;
    // a workgroup per head and sequence, and per part of its rows
    const long long heads = (long long)cache->B * cache->Hkv;
    if (heads >= (1ll << 21) || heads * (1 + most / 64) >= (1ll << 23)) return PAEP_ERR_SHAPE;
    if (!k_pages_dev || !v_pages_dev) return PAEP_ERR_NULL;
    if (cache->B > 0 && (!page_table_dev || !lengths_dev || !mass_dev || !out_table_dev || !kept_dev || !mass_out_dev || !lengths_out_dev))
        return PAEP_ERR_NULL;
    if (!aligned16(k_pages_dev) || !aligned16(v_pages_dev)) return PAEP_ERR_ALIGN;
    if (cache->B == 0) return PAEP_OK;
    const hipError_t err = paep::launch_cache_evict(to_view(cache, k_pages_dev, v_pages_dev, page_table_dev), max_len, budget,
                                                    recent, lengths_dev, mass_dev, mass_stride, out_table_dev, out_max_pages,
                                                    kept_dev, mass_out_dev, mass_out_stride, lengths_out_dev,
                                                    static_cast<hipStream_t>(stream));
    return err == hipSuccess ? PAEP_OK : PAEP_ERR_HIP;
}

size_t paep_attend_fourbit_workspace_bytes(const paep_cache_desc* cache, const paep_attend_desc* desc)
{
    if (check_attend(cache, desc, false, true) != PAEP_OK) return 0;
    const paep::AttendFourbitArgs a{to_attend(cache, desc, nullptr, nullptr, nullptr), nullptr, nullptr};
    return paep::attend_fourbit_fits(a) ? paep::attend_fourbit_workspace_bytes(a) : 0;
}

paep_status paep_attend_fourbit(const paep_cache_desc* cache, const paep_attend_desc* desc, const void* q_dev,
                            const void* k_pages_dev, const void* v_pages_dev, const uint8_t* k_scales_dev,
                            const uint8_t* v_scales_dev, const int32_t* page_table_dev, const int32_t* lengths_dev,
                            const int32_t* starts_dev, void* out_dev, float* lse_dev,
                            void* workspace_dev, size_t workspace_bytes, void* stream)
{
    const paep_status st = check_attend(cache, desc, false, true);
    if (st != PAEP_OK) return st;
    if (!k_pages_dev || !v_pages_dev || !k_scales_dev || !v_scales_dev) return PAEP_ERR_NULL;
    if (cache->B > 0 && (!q_dev || !page_table_dev || !lengths_dev || !out_dev)) return PAEP_ERR_NULL;
    for (const void* p : {q_dev, k_pages_dev, v_pages_dev, (const void*)k_scales_dev, (const void*)v_scales_dev, (const void*)out_dev})
        if (!aligned16(p)) return PAEP_ERR_ALIGN;
    paep::AttendFourbitArgs f{to_attend(cache, desc, k_pages_dev, v_pages_dev, page_table_dev), k_scales_dev, v_scales_dev};
    f.a.c = to_fourbit_view(cache, k_pages_dev, v_pages_dev, page_table_dev);
    if (!paep::attend_fourbit_fits(f)) return PAEP_ERR_SHAPE;
    const size_t need = paep::attend_fourbit_workspace_bytes(f);
    if (need > 0 && (!workspace_dev || !aligned16(workspace_dev) || workspace_bytes < need)) return PAEP_ERR_WORKSPACE;
    if (cache->B == 0) return PAEP_OK;
    f.a.q = q_dev; f.a.lengths = lengths_dev; f.a.starts = starts_dev; f.a.out = out_dev; f.a.lse = lse_dev;
    f.a.workspace = workspace_dev;
    f.a.stream = static_cast<hipStream_t>(stream);
    return paep::launch_attend_fourbit(f) == hipSuccess ? PAEP_OK : PAEP_ERR_HIP;
}

paep_status paep_cache_append_fourbit(const paep_cache_desc* cache, int32_t n, const void* k_dev, int64_t k_row_stride,
                                  int64_t k_head_stride, const void* v_dev, int64_t v_row_stride, int64_t v_head_stride,
                                  void* k_pages_dev, void* v_pages_dev, uint8_t* k_scales_dev, uint8_t* v_scales_dev,
                                  const int32_t* page_table_dev, const int32_t* sequences_dev, const int32_t* positions_dev,
                                  void* stream)
{
    paep_status st = check_cache(cache, true);
    if (st != PAEP_OK) return st;
    if (n < 0 || n > (1 << 24) || (!sequences_dev && n > cache->B)) return PAEP_ERR_SHAPE;
    st = check_rows(k_row_stride, k_head_stride, n, cache->Hkv, cache->Dk, cache->dtype, false);
    if (st == PAEP_OK) st = check_rows(v_row_stride, v_head_stride, n, cache->Hkv, cache->Dv, cache->dtype, false);
    if (st != PAEP_OK) return st;
    if (!k_pages_dev || !v_pages_dev || !k_scales_dev || !v_scales_dev) return PAEP_ERR_NULL;
    if (n > 0 && (!k_dev || !v_dev || !positions_dev || (cache->B > 0 && !page_table_dev))) return PAEP_ERR_NULL;
    for (const void* p : {k_dev, v_dev, (const void*)k_pages_dev, (const void*)v_pages_dev, (const void*)k_scales_dev, (const void*)v_scales_dev})
        if (!aligned16(p)) return PAEP_ERR_ALIGN;
    if (n == 0 || cache->B == 0) return PAEP_OK;
    const long long s = element_bytes(cache->dtype);
    const hipError_t err = paep::launch_cache_append_fourbit(to_fourbit_view(cache, k_pages_dev, v_pages_dev, page_table_dev), k_scales_dev,
                                                         v_scales_dev, n, k_dev, k_row_stride * s, k_head_stride * s, v_dev,
                                                         v_row_stride * s, v_head_stride * s, sequences_dev, positions_dev,
                                                         static_cast<hipStream_t>(stream));
    return err == hipSuccess ? PAEP_OK : PAEP_ERR_HIP;
}

paep_status paep_cache_read_fourbit(const paep_cache_desc* cache, int32_t n, const void* k_pages_dev, const void* v_pages_dev,
                                const uint8_t* k_scales_dev, const uint8_t* v_scales_dev, const int32_t* page_table_dev,
                                const int32_t* sequences_dev, const int32_t* positions_dev, void* k_out_dev, void* v_out_dev,
                                void* stream)
{
    const paep_status st = check_cache(cache, true);
    if (st != PAEP_OK) return st;
    if (n < 0 || n > (1 << 24) || (!sequences_dev && n > cache->B)) return PAEP_ERR_SHAPE;
    if (!k_pages_dev || !v_pages_dev || !k_scales_dev || !v_scales_dev) return PAEP_ERR_NULL;
    if (n > 0 && (!positions_dev || !k_out_dev || !v_out_dev || (cache->B > 0 && !page_table_dev))) return PAEP_ERR_NULL;
    for (const void* p : {k_pages_dev, v_pages_dev, (const void*)k_scales_dev, (const void*)v_scales_dev, (const void*)k_out_dev, (const void*)v_out_dev})
        if (!aligned16(p)) return PAEP_ERR_ALIGN;
    if (n == 0) return PAEP_OK;
    const hipError_t err = paep::launch_cache_read_fourbit(to_fourbit_view(cache, k_pages_dev, v_pages_dev, page_table_dev), k_scales_dev,
                                                       v_scales_dev, n, sequences_dev, positions_dev, k_out_dev, v_out_dev,
                                                       static_cast<hipStream_t>(stream));
    return err == hipSuccess ? PAEP_OK : PAEP_ERR_HIP;
}

paep_status paep_rotate(const paep_rotate_desc* desc, const void* q_dev, const void* k_dev,
                        const void* q_weight_dev, const void* k_weight_dev, const int32_t* positions_dev,
                        const float* table_dev, void* q_out_dev, void* k_out_dev, void* stream)
{
    const paep_status st = check_rotate(desc, false);
    if (st != PAEP_OK) return st;
    if (!table_dev) return PAEP_ERR_NULL;
    if (desc->n > 0 && (!positions_dev || (desc->Hq > 0 && (!q_dev || !q_out_dev)) || (desc->Hk > 0 && (!k_dev || !k_out_dev)))) return PAEP_ERR_NULL;
    for (const void* p : {q_dev, k_dev, q_weight_dev, k_weight_dev, (const void*)table_dev, (const void*)q_out_dev, (const void*)k_out_dev})
        if (!aligned16(p)) return PAEP_ERR_ALIGN;
    if (desc->n == 0) return PAEP_OK;
    paep::RotateArgs a = to_rotate(desc, false);
    a.q = q_dev; a.k = k_dev; a.q_out = q_out_dev; a.k_out = k_out_dev; a.q_weight = q_weight_dev; a.k_weight = k_weight_dev;
    a.angles = positions_dev; a.table = table_dev;
    a.stream = static_cast<hipStream_t>(stream);
    return paep::launch_rotate(a) == hipSuccess ? PAEP_OK : PAEP_ERR_HIP;
}

paep_status paep_rotate_append(const paep_rotate_desc* desc, const paep_cache_desc* cache, const void* q_dev,
                               const void* k_dev, const void* v_dev, int64_t v_row_stride, int64_t v_head_stride,
                               const void* q_weight_dev, const void* k_weight_dev, const float* table_dev,
                               const int32_t* angles_dev, void* q_out_dev, void* k_pages_dev, void* v_pages_dev,
                               const int32_t* page_table_dev, const int32_t* sequences_dev, const int32_t* positions_dev,
                               float* mass_dev, int64_t mass_stride, void* stream)
{
    paep_status st = check_rotate(desc, true);
    if (st == PAEP_OK) st = check_cache(cache);
    if (st != PAEP_OK) return st;
    if (cache->Hkv != desc->Hk || cache->Dk != desc->D) return PAEP_ERR_SHAPE;
    if (cache->dtype != desc->dtype) return PAEP_ERR_DTYPE;
    if (!sequences_dev && desc->n > cache->B) return PAEP_ERR_SHAPE;
    st = check_rows(v_row_stride, v_head_stride, desc->n, cache->Hkv, cache->Dv, cache->dtype, false);
    if (st != PAEP_OK) return st;
    if (mass_dev && (mass_stride < 0 || mass_stride > MAX_STRIDE)) return PAEP_ERR_SHAPE;
    if (!table_dev || !k_pages_dev || !v_pages_dev) return PAEP_ERR_NULL;
    if (desc->n > 0 && (!k_dev || !v_dev || !positions_dev || (desc->Hq > 0 && (!q_dev || !q_out_dev)) || (cache->B > 0 && !page_table_dev)))
        return PAEP_ERR_NULL;
    for (const void* p : {q_dev, k_dev, v_dev, q_weight_dev, k_weight_dev, (const void*)table_dev, (const void*)q_out_dev,
                          (const void*)k_pages_dev, (const void*)v_pages_dev})
        if (!aligned16(p)) return PAEP_ERR_ALIGN;
    if (desc->n == 0) return PAEP_OK;
    paep::RotateArgs a = to_rotate(desc, true);
    a.c = to_view(cache, k_pages_dev, v_pages_dev, page_table_dev);
    a.q = q_dev; a.k = k_dev; a.v = v_dev; a.q_out = q_out_dev; a.q_weight = q_weight_dev; a.k_weight = k_weight_dev;
    const long long s = element_bytes(desc->dtype);
    a.v_row = v_row_stride * s; a.v_head = v_head_stride * s;
    a.angles = angles_dev ? angles_dev : positions_dev; a.table = table_dev;
    a.sequences = sequences_dev; a.positions = positions_dev; a.mass = mass_dev; a.mass_stride = mass_stride;
    a.stream = static_cast<hipStream_t>(stream);
    return paep::launch_rotate(a) == hipSuccess ? PAEP_OK : PAEP_ERR_HIP;
}

size_t paep_moe_workspace_bytes(const paep_moe_desc* desc)
{
    return check_moe(desc) == PAEP_OK ? paep::moe_workspace_bytes(to_moe(desc)) : 0;
}

paep_status paep_moe_layer(const paep_moe_desc* desc, const void* x_dev, const void* Wg_dev, const void* bg_dev,
                           const void* W13_dev, const void* W2_dev, const void* residual_dev,
                           void* y_dev, int32_t* idx_dev, float* probs_dev, int32_t* counts_dev,
                           void* workspace_dev, size_t workspace_bytes, void* stream)
{
    const paep_status st = check_moe(desc);
    if (st != PAEP_OK) return st;
    if (!Wg_dev) return PAEP_ERR_NULL;
    return moe_common(desc, x_dev, Wg_dev, bg_dev, W13_dev, W2_dev, residual_dev, y_dev, idx_dev, probs_dev, counts_dev,
                      workspace_dev, workspace_bytes, stream);
}

paep_status paep_moe_experts(const paep_moe_desc* desc, const void* x_dev, const void* W13_dev, const void* W2_dev,
                             const int32_t* idx_dev, const float* probs_dev, const void* residual_dev, void* y_dev,
                             void* workspace_dev, size_t workspace_bytes, void* stream)
{
    const paep_status st = check_moe(desc);
    if (st != PAEP_OK) return st;
    return moe_common(desc, x_dev, nullptr, nullptr, W13_dev, W2_dev, residual_dev, y_dev, const_cast<int32_t*>(idx_dev),
                      const_cast<float*>(probs_dev), nullptr, workspace_dev, workspace_bytes, stream);
}

}  // extern "C"
