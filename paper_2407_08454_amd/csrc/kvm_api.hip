// Host side of the C ABI declared in include/kvm.h: argument validation, workspace
// carving, error strings and kernel dispatch.  No allocation, no synchronisation.
#include <math.h>
#include <algorithm>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "kvm_common.h"

namespace kvm {

static thread_local char g_err[512] = "";

void set_error(const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
}

kvm_status check_launch(const char *what)
{
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
        set_error("%s: launch failed: %s", what, hipGetErrorString(e));
        return KVM_ERR_LAUNCH;
    }
    return KVM_OK;
}

static size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// ---- optional per-kernel timing ---------------------------------------------------------
struct ProfState {
    bool on = false;
    int cap = 0, used = 0;
    hipEvent_t *ev = nullptr;        // 2 per timed launch
    const char **names = nullptr;    // kernel name per timed launch (string literals)
};
static ProfState g_prof;

ProfScope::ProfScope(const char *name, hipStream_t s) : slot(-1), st(s)
{
    if (!g_prof.on || g_prof.used >= g_prof.cap) return;
    // a stream that is being captured into a graph is not timed: the event records would become
    // nodes of the caller's graph
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &cap) != hipSuccess || cap != hipStreamCaptureStatusNone) return;
    slot = g_prof.used++;
    g_prof.names[slot] = name;
    (void)hipEventRecord(g_prof.ev[2 * slot], st);
}

ProfScope::~ProfScope()
{
    if (slot >= 0) (void)hipEventRecord(g_prof.ev[2 * slot + 1], st);
}

static kvm_status check_shape(const kvm_shape *sh, const char *fn)
{
    if (!sh) { set_error("%s: shape is NULL", fn); return KVM_ERR_INVALID_ARG; }
    if (sh->B < 0 || sh->H_kv < 1 || sh->G < 1 || sh->N < 0) {
        set_error("%s: invalid sizes B=%d H_kv=%d G=%d N=%d", fn, sh->B, sh->H_kv, sh->G, sh->N);
        return KVM_ERR_INVALID_ARG;
    }
    if (sh->d != HEAD_DIM) { set_error("%s: head dimension %d is not supported (only %d)", fn, sh->d, HEAD_DIM); return KVM_ERR_UNSUPPORTED; }
    if (sh->dtype != KVM_F32 && sh->dtype != KVM_F16 && sh->dtype != KVM_BF16) {
        set_error("%s: unknown dtype %d", fn, sh->dtype);
        return KVM_ERR_UNSUPPORTED;
    }
    // grids and int32 offsets inside a slice
    const long long slices = (long long)sh->B * sh->H_kv * sh->G;
    if (slices > (1ll << 24) || (long long)sh->N > (1ll << 22)) {
        set_error("%s: shape too large (B*H_kv*G=%lld, N=%d)", fn, slices, sh->N);
        return KVM_ERR_UNSUPPORTED;
    }
    return KVM_OK;
}

static kvm_status check_params(const kvm_params *pr, const char *fn)
{
    if (!pr) { set_error("%s: params is NULL", fn); return KVM_ERR_INVALID_ARG; }
    const bool ok = pr->budget >= 0.0 && pr->budget <= 1.0 && pr->recent_ratio >= 0.0 && pr->recent_ratio <= 1.0 &&
                    pr->heavy_ratio >= 0.0 && pr->heavy_ratio <= 1.0;
    if (!ok) {
        set_error("%s: budget/recent_ratio/heavy_ratio must lie in [0,1] (%g, %g, %g)", fn, pr->budget,
                  pr->recent_ratio, pr->heavy_ratio);
        return KVM_ERR_INVALID_ARG;
    }
    if (pr->enforce_budget && pr->recent_ratio + pr->heavy_ratio > pr->budget) {
        set_error("%s: recent_ratio + heavy_ratio = %g exceeds the budget %g", fn, pr->recent_ratio + pr->heavy_ratio,
                  pr->budget);
        return KVM_ERR_INVALID_ARG;
    }
    if (!(pr->threshold == pr->threshold)) { set_error("%s: threshold is NaN", fn); return KVM_ERR_INVALID_ARG; }
    if (pr->sigma_mode != KVM_SIGMA_MEAN_DIST && pr->sigma_mode != KVM_SIGMA_FIXED) {
        set_error("%s: unknown sigma_mode %d", fn, pr->sigma_mode);
        return KVM_ERR_UNSUPPORTED;
    }
    if (pr->weights != KVM_WEIGHTS_GAUSSIAN && pr->weights != KVM_WEIGHTS_AVERAGE) {
        set_error("%s: unknown weights %d", fn, pr->weights);
        return KVM_ERR_UNSUPPORTED;
    }
    if (pr->set_rule != KVM_SETS_ADJACENT && pr->set_rule != KVM_SETS_ANCHOR) {
        set_error("%s: unknown set_rule %d", fn, pr->set_rule);
        return KVM_ERR_UNSUPPORTED;
    }
    if (pr->pivot_rule < KVM_PIVOT_MAX_SCORE || pr->pivot_rule > KVM_PIVOT_RANDOM) {
        set_error("%s: unknown pivot_rule %d", fn, pr->pivot_rule);
        return KVM_ERR_UNSUPPORTED;
    }
    if (pr->sigma_mode == KVM_SIGMA_FIXED && !(pr->sigma > 0.f)) {
        set_error("%s: fixed sigma must be > 0 (%g)", fn, (double)pr->sigma);
        return KVM_ERR_INVALID_ARG;
    }
    return KVM_OK;
}

static int capacity(const kvm_shape *sh, const kvm_params *pr)
{
    return pr->enforce_budget ? (int)floor(pr->budget * (double)sh->N) : sh->N;
}

static size_t ws_attn(const kvm_shape *sh)
{
    // row statistics, then one flag per (query slice, row tile); the decode-time update keeps its
    // scores in the first part and two floats per (query slice, 64 keys) in the second, which is
    // the larger need
    const size_t q_slices = (size_t)sh->B * sh->H_kv * sh->G;
    const size_t second = std::max((size_t)attn_row_tiles(sh->N), (size_t)attn_lse_stride(sh->N) / 64 * 2);
    return align_up(q_slices * attn_lse_stride(sh->N) * sizeof(float) + q_slices * second * sizeof(float), 256);
}
static size_t ws_identify(const kvm_shape *sh)
{
    const size_t tok = (size_t)sh->B * sh->H_kv * sh->N;
    // adjacent similarities, inverse key norms, run lengths of the anchor rule, flag bytes
    return 3 * align_up(tok * sizeof(float), 256) + align_up(tok, 256);
}

// what every call accepts; the single score pass asks for room beyond it
static size_t ws_plain(const kvm_shape *sh, int cap)
{
    return std::max(std::max(ws_attn(sh), ws_identify(sh)), merge_refresh_workspace_bytes(*sh, cap)) + 256;
}

// ---- the paged cache and the compacted prefixes ------------------------------------------
static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
static int elem_bytes(const kvm_shape *sh) { return sh->dtype == KVM_F32 ? 4 : 2; }

// rows of B * T tokens with `heads` heads each, `stride` elements apart
static kvm_status check_rows(const kvm_shape *sh, const char *fn, const char *name, const void *p, int64_t stride, int64_t heads)
{
    if (!p) { set_error("%s: %s must not be NULL", fn, name); return KVM_ERR_INVALID_ARG; }
    if (!aligned16(p) || stride * elem_bytes(sh) % 16 != 0) {
        set_error("%s: %s and its stride of %lld elements must be multiples of 16 bytes", fn, name, (long long)stride);
        return KVM_ERR_INVALID_ARG;
    }
    if (stride < heads * HEAD_DIM || stride > (1ll << 31)) {
        set_error("%s: tokens of %s are %lld elements apart, its heads take %lld", fn, name, (long long)stride, (long long)(heads * HEAD_DIM));
        return KVM_ERR_INVALID_ARG;
    }
    return KVM_OK;
}

static kvm_status check_pages(const kvm_shape *sh, const kvm_pages *pg, const char *fn)
{
    if (pg->n_pages < 0 || pg->max_pages < 0 || pg->page_size < 1 || pg->page_size > 65536 || (pg->page_size & (pg->page_size - 1)) != 0) {
        set_error("%s: invalid pages (n_pages=%d, max_pages=%d, page_size=%d, a power of two up to 65536)", fn, pg->n_pages, pg->max_pages,
                  pg->page_size);
        return KVM_ERR_INVALID_ARG;
    }
    if ((int64_t)pg->max_pages * pg->page_size > (1ll << 22)) {
        set_error("%s: a row of %d pages of %d tokens is too long", fn, pg->max_pages, pg->page_size);
        return KVM_ERR_UNSUPPORTED;
    }
    if ((pg->n_pages > 0 && (!pg->K || !pg->V)) || (sh->B > 0 && pg->max_pages > 0 && !pg->table) || !aligned16(pg->K) || !aligned16(pg->V)) {
        set_error("%s: the pages' K, V and table must not be NULL, K and V multiples of 16 bytes", fn);
        return KVM_ERR_INVALID_ARG;
    }
    return KVM_OK;
}

static kvm_status check_prefix(const kvm_shape *sh, const kvm_prefix *px, const char *fn)
{
    if (px->P < 0 || px->capacity < 0 || px->capacity > (1 << 22) || (int64_t)px->P * sh->H_kv > (1 << 24)) {
        set_error("%s: invalid prefix sizes P=%d capacity=%d", fn, px->P, px->capacity);
        return KVM_ERR_INVALID_ARG;
    }
    if (!px->row_start && px->P > 0 && sh->B % px->P != 0) {
        set_error("%s: %d rows do not divide among %d prompts: row_start is needed", fn, sh->B, px->P);
        return KVM_ERR_INVALID_ARG;
    }
    if (((int64_t)px->P * px->capacity > 0 && (!px->K || !px->V)) || !aligned16(px->K) || !aligned16(px->V)) {
        set_error("%s: the prefixes' K and V must not be NULL and multiples of 16 bytes", fn);
        return KVM_ERR_INVALID_ARG;
    }
    return KVM_OK;
}

// tokens and head rows of a call, for the grids
static kvm_status check_tokens(const kvm_shape *sh, const char *fn)
{
    const int64_t tokens = (int64_t)sh->B * sh->N;
    if (tokens > (1ll << 22) || tokens * sh->H_kv * (sh->G + 2) > (1ll << 26)) {
        set_error("%s: %lld tokens with %d query and %d key heads are too many for one call", fn, (long long)tokens, sh->H_kv * sh->G, sh->H_kv);
        return KVM_ERR_UNSUPPORTED;
    }
    return KVM_OK;
}

}  // namespace kvm

using namespace kvm;

extern "C" {

kvm_status kvm_params_for_budget(double budget, kvm_params *out)
{
    if (!out || !(budget > 0.0 && budget <= 1.0)) {
        set_error("kvm_params_for_budget: need out != NULL and 0 < budget <= 1");
        return KVM_ERR_INVALID_ARG;
    }
    memset(out, 0, sizeof(*out));
    out->budget = budget;
    if (budget == 0.5) { out->recent_ratio = 0.17; out->heavy_ratio = 0.12; }
    else if (budget == 0.35) { out->recent_ratio = 0.08; out->heavy_ratio = 0.02; }
    else { out->recent_ratio = 0.34 * budget; out->heavy_ratio = 0.24 * budget; }
    out->threshold = 0.75f;
    out->sigma_mode = KVM_SIGMA_MEAN_DIST;
    out->sigma = 0.f;
    out->value_scale_by_set_size = 1;
    out->enforce_budget = 1;
    out->weights = KVM_WEIGHTS_GAUSSIAN;
    out->pivot_rule = KVM_PIVOT_MAX_SCORE;
    out->pivot_seed = 0;
    out->set_rule = KVM_SETS_ADJACENT;
    out->sim_given = 0;
    return KVM_OK;
}

int32_t kvm_out_capacity(const kvm_shape *shape, const kvm_params *params)
{
    if (check_shape(shape, "kvm_out_capacity") != KVM_OK || check_params(params, "kvm_out_capacity") != KVM_OK) return -1;
    return capacity(shape, params);
}

size_t kvm_workspace_bytes(const kvm_shape *shape, const kvm_params *params)
{
    if (check_shape(shape, "kvm_workspace_bytes") != KVM_OK) return 0;
    // (the refresh of a compacted cache needs two ints per output row on top of what kvm_merge asks for; without
    // params the capacity is taken as N)
    if (!params || check_params(params, "kvm_workspace_bytes") != KVM_OK) return ws_plain(shape, shape->N);
    const size_t single = attn_single_bytes(*shape);
    return single ? ws_plain(shape, shape->N) + single : ws_plain(shape, capacity(shape, params));
}

static kvm_status attn_mass_entry(const char *who, const kvm_shape *shape, const void *Q, const void *K, const float *row_lse,
                                  bool with_lse, float *mass, float *sim, bool with_sim, void *ws, size_t ws_bytes,
                                  void *stream)
{
    kvm_status rc = check_shape(shape, who);
    if (rc != KVM_OK) return rc;
    const bool empty = (long long)shape->B * shape->N == 0;
    if (!empty && (!Q || !K || !mass || (with_lse && !row_lse))) {
        set_error("%s: Q, K%s and mass must not be NULL", who, with_lse ? ", row_lse" : "");
        return KVM_ERR_INVALID_ARG;
    }
    if (!empty && with_sim && !sim) {
        set_error("%s: sim must not be NULL", who);
        return KVM_ERR_INVALID_ARG;
    }
    if (empty) return KVM_OK;
    if (!ws || ws_bytes < ws_attn(shape)) {
        set_error("%s: workspace of %zu bytes needed, %zu given", who, ws_attn(shape), ws ? ws_bytes : (size_t)0);
        return KVM_ERR_WORKSPACE;
    }
    if (!with_lse) {
        const size_t single = attn_single_bytes(*shape);
        if (single && ws_bytes >= ws_plain(shape, shape->N) + single)
            return launch_attn_single(*shape, Q, K, mass, (float *)ws, with_sim ? sim : nullptr, (hipStream_t)stream);
    }
    return launch_attn_mass(*shape, Q, K, with_lse ? row_lse : nullptr, mass, (float *)ws, with_sim ? sim : nullptr,
                            (hipStream_t)stream);
}

kvm_status kvm_attn_mass(const kvm_shape *shape, const void *Q, const void *K, float *mass, void *ws, size_t ws_bytes,
                         void *stream)
{
    return attn_mass_entry("kvm_attn_mass", shape, Q, K, nullptr, false, mass, nullptr, false, ws, ws_bytes, stream);
}

kvm_status kvm_attn_mass_sim(const kvm_shape *shape, const void *Q, const void *K, float *mass, float *sim, void *ws,
                             size_t ws_bytes, void *stream)
{
    return attn_mass_entry("kvm_attn_mass_sim", shape, Q, K, nullptr, false, mass, sim, true, ws, ws_bytes, stream);
}

kvm_status kvm_attn_mass_from_lse(const kvm_shape *shape, const void *Q, const void *K, const float *row_lse, float *mass,
                                  void *ws, size_t ws_bytes, void *stream)
{
    return attn_mass_entry("kvm_attn_mass_from_lse", shape, Q, K, row_lse, true, mass, nullptr, false, ws, ws_bytes, stream);
}

kvm_status kvm_attn_mass_append(const kvm_shape *shape, const void *q_new, const void *K, float *mass, void *ws,
                                size_t ws_bytes, void *stream)
{
    kvm_status rc = check_shape(shape, "kvm_attn_mass_append");
    if (rc != KVM_OK) return rc;
    if ((long long)shape->B * shape->N == 0) return KVM_OK;
    if (!q_new || !K || !mass) { set_error("kvm_attn_mass_append: q_new, K and mass must not be NULL"); return KVM_ERR_INVALID_ARG; }
    if (!ws || ws_bytes < ws_attn(shape)) {
        set_error("kvm_attn_mass_append: workspace of %zu bytes needed, %zu given", ws_attn(shape), ws ? ws_bytes : (size_t)0);
        return KVM_ERR_WORKSPACE;
    }
    return launch_attn_append(*shape, q_new, K, mass, (float *)ws, (hipStream_t)stream);
}

kvm_status kvm_sim_append(const kvm_shape *shape, const void *K, float *sim, void *stream)
{
    kvm_status rc = check_shape(shape, "kvm_sim_append");
    if (rc != KVM_OK) return rc;
    if ((long long)shape->B * shape->N == 0) return KVM_OK;
    if (!K || !sim) { set_error("kvm_sim_append: K and sim must not be NULL"); return KVM_ERR_INVALID_ARG; }
    return launch_sim_append(*shape, K, sim, (hipStream_t)stream);
}

kvm_status kvm_identify_sets(const kvm_shape *shape, const kvm_params *params, const void *K, const float *mass,
                             int32_t *set_id, int32_t *set_start, int32_t *pivot, int32_t *n_sets, float *sim_opt,
                             int32_t *slice_status, void *ws, size_t ws_bytes, void *stream)
{
    kvm_status rc = check_shape(shape, "kvm_identify_sets");
    if (rc != KVM_OK) return rc;
    rc = check_params(params, "kvm_identify_sets");
    if (rc != KVM_OK) return rc;
    if (shape->B == 0) return KVM_OK;
    if (!set_start || !n_sets || !slice_status || (capacity(shape, params) > 0 && !pivot) ||
        (shape->N > 0 && ((!K && !params->sim_given) || !mass || !set_id))) {
        set_error("kvm_identify_sets: a required pointer is NULL");
        return KVM_ERR_INVALID_ARG;
    }
    if (params->sim_given && (!sim_opt || params->set_rule != KVM_SETS_ADJACENT)) {
        set_error("kvm_identify_sets: sim_given needs sim_opt and the adjacent set rule");
        return KVM_ERR_INVALID_ARG;
    }
    if (ws_identify(shape) > 0 && (!ws || ws_bytes < ws_identify(shape))) {
        set_error("kvm_identify_sets: workspace of %zu bytes needed, %zu given", ws_identify(shape), ws ? ws_bytes : (size_t)0);
        return KVM_ERR_WORKSPACE;
    }
    const size_t tok = (size_t)shape->B * shape->H_kv * shape->N;
    float *sim = sim_opt ? sim_opt : (float *)ws;
    const size_t stride = align_up(tok * sizeof(float), 256);
    float *inv_norm = (float *)((uint8_t *)ws + stride);
    int32_t *run = (int32_t *)((uint8_t *)ws + 2 * stride);
    uint8_t *flags = (uint8_t *)ws + 3 * stride;
    return launch_identify(*shape, *params, capacity(shape, params), K, mass, set_id, set_start, pivot, n_sets, sim,
                           inv_norm, run, flags, slice_status, (hipStream_t)stream);
}

static kvm_status evict_common(const char *fn, bool merge_values, const kvm_shape *shape, const kvm_params *params, const void *K,
                               const void *V, const float *mass, int32_t *kept, int32_t *n_kept, void *K_out, void *V_out,
                               void *ws, size_t ws_bytes, void *stream)
{
    kvm_status rc = check_shape(shape, fn);
    if (rc != KVM_OK) return rc;
    rc = check_params(params, fn);
    if (rc != KVM_OK) return rc;
    if (shape->B == 0) return KVM_OK;
    const int cap = capacity(shape, params);
    if (!n_kept || (cap > 0 && (!kept || !K_out || !V_out)) || (shape->N > 0 && (!K || !V || !mass))) {
        set_error("%s: a required pointer is NULL", fn);
        return KVM_ERR_INVALID_ARG;
    }
    if (ws_identify(shape) > 0 && (!ws || ws_bytes < ws_identify(shape))) {
        set_error("%s: workspace of %zu bytes needed, %zu given", fn, ws_identify(shape), ws ? ws_bytes : (size_t)0);
        return KVM_ERR_WORKSPACE;
    }
    const size_t tok = (size_t)shape->B * shape->H_kv * shape->N;
    uint8_t *flags = (uint8_t *)ws + 3 * align_up(tok * sizeof(float), 256);
    return launch_evict(*shape, *params, cap, K, V, mass, kept, n_kept, K_out, V_out, flags, merge_values, (hipStream_t)stream);
}

kvm_status kvm_evict(const kvm_shape *shape, const kvm_params *params, const void *K, const void *V, const float *mass,
                     int32_t *kept, int32_t *n_kept, void *K_out, void *V_out, void *ws, size_t ws_bytes, void *stream)
{
    return evict_common("kvm_evict", false, shape, params, K, V, mass, kept, n_kept, K_out, V_out, ws, ws_bytes, stream);
}

kvm_status kvm_evict_merge_values(const kvm_shape *shape, const kvm_params *params, const void *K, const void *V,
                                  const float *mass, int32_t *kept, int32_t *n_kept, void *K_out, void *V_out, void *ws,
                                  size_t ws_bytes, void *stream)
{
    return evict_common("kvm_evict_merge_values", true, shape, params, K, V, mass, kept, n_kept, K_out, V_out, ws, ws_bytes,
                        stream);
}

kvm_status kvm_merge(const kvm_shape *shape, const kvm_params *params, const void *K, const void *V,
                     const int32_t *set_start, const int32_t *pivot, const int32_t *n_sets, void *K_out, void *V_out,
                     float *w_opt, void *ws, size_t ws_bytes, void *stream)
{
    kvm_status rc = check_shape(shape, "kvm_merge");
    if (rc != KVM_OK) return rc;
    rc = check_params(params, "kvm_merge");
    if (rc != KVM_OK) return rc;
    const int cap = capacity(shape, params);
    if ((long long)shape->B * shape->N == 0 || cap == 0) return KVM_OK;
    if (!K || !V || !set_start || !pivot || !n_sets || !K_out || !V_out) {
        set_error("kvm_merge: a required pointer is NULL");
        return KVM_ERR_INVALID_ARG;
    }
    if (!ws || ws_bytes < merge_workspace_bytes(*shape)) {
        set_error("kvm_merge: workspace of %zu bytes needed, %zu given", merge_workspace_bytes(*shape), ws ? ws_bytes : (size_t)0);
        return KVM_ERR_WORKSPACE;
    }
    return launch_merge(*shape, *params, cap, K, V, set_start, pivot, n_sets, K_out, V_out, w_opt, (hipStream_t)stream);
}

kvm_status kvm_merge_refresh(const kvm_shape *shape, const kvm_params *params, const void *K, const void *V,
                             const int32_t *prev_set_id, const int32_t *prev_set_start, const int32_t *prev_pivot,
                             const int32_t *prev_n_sets, const int32_t *set_start, const int32_t *pivot, const int32_t *n_sets,
                             void *K_out, void *V_out, int32_t *n_changed_opt, void *ws, size_t ws_bytes, void *stream)
{
    kvm_status rc = check_shape(shape, "kvm_merge_refresh");
    if (rc != KVM_OK) return rc;
    rc = check_params(params, "kvm_merge_refresh");
    if (rc != KVM_OK) return rc;
    const int cap = capacity(shape, params);
    if ((long long)shape->B * shape->N == 0 || cap == 0) return KVM_OK;
    if (!K || !V || !prev_set_id || !prev_set_start || !prev_pivot || !prev_n_sets || !set_start || !pivot || !n_sets || !K_out ||
        !V_out) {
        set_error("kvm_merge_refresh: a required pointer is NULL");
        return KVM_ERR_INVALID_ARG;
    }
    if (prev_set_start == set_start || prev_pivot == pivot || prev_n_sets == n_sets) {
        set_error("kvm_merge_refresh: the previous and the new maps must be different buffers");
        return KVM_ERR_INVALID_ARG;
    }
    const size_t need = merge_refresh_workspace_bytes(*shape, cap);
    if (!ws || ws_bytes < need) {
        set_error("kvm_merge_refresh: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
        return KVM_ERR_WORKSPACE;
    }
    return launch_merge_refresh(*shape, *params, cap, K, V, prev_set_id, prev_set_start, prev_pivot, prev_n_sets, set_start, pivot,
                                n_sets, K_out, V_out, n_changed_opt, (int32_t *)ws, ws_bytes, (hipStream_t)stream);
}

kvm_status kvm_merge_static(const kvm_shape *shape, const kvm_params *params, const void *K, const void *V,
                            const int32_t *set_start, const int32_t *pivot, const int32_t *n_sets, void *K_out, void *V_out,
                            float *w_opt, void *stream)
{
    kvm_status rc = check_shape(shape, "kvm_merge_static");
    if (rc != KVM_OK) return rc;
    rc = check_params(params, "kvm_merge_static");
    if (rc != KVM_OK) return rc;
    const int cap = capacity(shape, params);
    if ((long long)shape->B * shape->N == 0 || cap == 0) return KVM_OK;
    if (!K || !V || !set_start || !pivot || !n_sets || !K_out || !V_out) {
        set_error("kvm_merge_static: a required pointer is NULL");
        return KVM_ERR_INVALID_ARG;
    }
    return launch_merge_static(*shape, *params, cap, K, V, set_start, pivot, n_sets, K_out, V_out, w_opt, (hipStream_t)stream);
}

kvm_status kvm_paged_append(const kvm_shape *shape, const kvm_pages *pages, const kvm_rotation *rotation, const void *q_new,
                            int64_t q_stride, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                            const int32_t *past_lens, const int32_t *pos_base, void *q_out, int32_t *kv_lens, void *stream)
{
    const char *fn = "kvm_paged_append";
    kvm_status rc = check_shape(shape, fn);
    if (rc != KVM_OK) return rc;
    if (!pages || !rotation) { set_error("%s: pages and rotation must not be NULL", fn); return KVM_ERR_INVALID_ARG; }
    rc = check_pages(shape, pages, fn);
    if (rc == KVM_OK) rc = check_tokens(shape, fn);
    if (rc != KVM_OK) return rc;
    if (rotation->rot_dim < 0 || rotation->rot_dim > HEAD_DIM || rotation->rot_dim % 16 != 0) {
        set_error("%s: rot_dim %d is not a multiple of 16 up to %d", fn, rotation->rot_dim, HEAD_DIM);
        return KVM_ERR_UNSUPPORTED;
    }
    if (shape->B == 0) return KVM_OK;
    if (!past_lens || !kv_lens || past_lens == kv_lens) {
        set_error("%s: past_lens and kv_lens must be two buffers", fn);
        return KVM_ERR_INVALID_ARG;
    }
    if (kv_lens == shape->seq_lens || kv_lens == pos_base) {    // read by some workgroups while another writes kv_lens
        set_error("%s: kv_lens must be a buffer of its own, not seq_lens or pos_base", fn);
        return KVM_ERR_INVALID_ARG;
    }
    if (shape->N > 0) {
        if (rotation->rot_dim > 0 && !rotation->inv_freq) { set_error("%s: inv_freq must not be NULL", fn); return KVM_ERR_INVALID_ARG; }
        if (!q_new != !q_out) { set_error("%s: q_new and q_out go together", fn); return KVM_ERR_INVALID_ARG; }
        const int64_t HG = (int64_t)shape->H_kv * shape->G;
        if (q_new) {
            rc = check_rows(shape, fn, "q_new", q_new, q_stride, HG);
            if (rc == KVM_OK) rc = check_rows(shape, fn, "q_out", q_out, HG * HEAD_DIM, HG);
            if (rc != KVM_OK) return rc;
            if (q_new == q_out && q_stride != HG * HEAD_DIM) {
                set_error("%s: q_out may be q_new only if that is contiguous", fn);
                return KVM_ERR_INVALID_ARG;
            }
        }
        rc = check_rows(shape, fn, "k_new", k_new, k_stride, shape->H_kv);
        if (rc == KVM_OK) rc = check_rows(shape, fn, "v_new", v_new, v_stride, shape->H_kv);
        if (rc != KVM_OK) return rc;
    }
    return launch_paged_append(*shape, *pages, *rotation, q_new, q_stride, k_new, k_stride, v_new, v_stride, past_lens, pos_base, q_out,
                               kv_lens, (hipStream_t)stream);
}

static kvm_status check_attn_sources(const kvm_shape *shape, const kvm_prefix *prefix, const kvm_pages *pages, const char *fn)
{
    kvm_status rc = check_shape(shape, fn);
    if (rc != KVM_OK) return rc;
    if (!prefix && !pages) { set_error("%s: prefix and pages must not both be NULL", fn); return KVM_ERR_INVALID_ARG; }
    rc = check_tokens(shape, fn);
    if (rc == KVM_OK && prefix) rc = check_prefix(shape, prefix, fn);
    if (rc == KVM_OK && pages) rc = check_pages(shape, pages, fn);
    return rc;
}

size_t kvm_prefix_attn_workspace_bytes(const kvm_shape *shape, const kvm_prefix *prefix, const kvm_pages *pages)
{
    if (check_attn_sources(shape, prefix, pages, "kvm_prefix_attn_workspace_bytes") != KVM_OK) return 0;
    return prefix_attn_workspace_bytes(*shape, prefix, pages);
}

kvm_status kvm_prefix_attn(const kvm_shape *shape, const kvm_prefix *prefix, const kvm_pages *pages, const void *Q, int64_t q_stride,
                           const int32_t *kv_lens, void *out, float *lse_opt, void *ws, size_t ws_bytes, void *stream)
{
    const char *fn = "kvm_prefix_attn";
    kvm_status rc = check_attn_sources(shape, prefix, pages, fn);
    if (rc != KVM_OK) return rc;
    if ((long long)shape->B * shape->N == 0) return KVM_OK;
    const int64_t HG = (int64_t)shape->H_kv * shape->G;
    rc = check_rows(shape, fn, "Q", Q, q_stride, HG);
    if (rc == KVM_OK) rc = check_rows(shape, fn, "out", out, HG * HEAD_DIM, HG);
    if (rc != KVM_OK) return rc;
    if (pages && !kv_lens) { set_error("%s: kv_lens must not be NULL", fn); return KVM_ERR_INVALID_ARG; }
    const size_t need = prefix_attn_workspace_bytes(*shape, prefix, pages);
    if (!ws || ws_bytes < need) {
        set_error("%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
        return KVM_ERR_WORKSPACE;
    }
    if (!aligned16(ws)) { set_error("%s: the workspace must be 256-byte aligned", fn); return KVM_ERR_INVALID_ARG; }
    return launch_prefix_attn(*shape, prefix, pages, Q, q_stride, kv_lens, out, lse_opt, ws, (hipStream_t)stream);
}

kvm_status kvm_profile_disable(void)
{
    if (g_prof.ev) {
        for (int i = 0; i < 2 * g_prof.cap; ++i) (void)hipEventDestroy(g_prof.ev[i]);
        delete[] g_prof.ev;
        delete[] g_prof.names;
    }
    g_prof = ProfState();
    return KVM_OK;
}

kvm_status kvm_profile_enable(int32_t max_launches)
{
    kvm_profile_disable();
    if (max_launches < 1 || max_launches > (1 << 20)) {
        set_error("kvm_profile_enable: max_launches must lie in [1, 2^20]");
        return KVM_ERR_INVALID_ARG;
    }
    g_prof.ev = new hipEvent_t[2 * (size_t)max_launches];
    g_prof.names = new const char *[max_launches];
    for (int i = 0; i < 2 * max_launches; ++i) {
        if (hipEventCreate(&g_prof.ev[i]) != hipSuccess) {
            for (int j = 0; j < i; ++j) (void)hipEventDestroy(g_prof.ev[j]);   // cap is still 0: disable frees the arrays only
            kvm_profile_disable();
            set_error("kvm_profile_enable: hipEventCreate failed");
            return KVM_ERR_LAUNCH;
        }
    }
    g_prof.cap = max_launches;
    g_prof.used = 0;
    g_prof.on = true;
    return KVM_OK;
}

int32_t kvm_profile_collect(kvm_kernel_time *out, int32_t max_records)
{
    if (!g_prof.on || !out || max_records < 1) return 0;
    int n = 0;
    for (int i = 0; i < g_prof.used; ++i) {
        float ms = 0.f;
        if (hipEventSynchronize(g_prof.ev[2 * i + 1]) != hipSuccess) continue;
        if (hipEventElapsedTime(&ms, g_prof.ev[2 * i], g_prof.ev[2 * i + 1]) != hipSuccess) continue;
        int r = 0;
        while (r < n && strcmp(out[r].name, g_prof.names[i]) != 0) ++r;
        if (r == n) {
            if (n == max_records) continue;
            memset(&out[n], 0, sizeof(out[n]));
            strncpy(out[n].name, g_prof.names[i], sizeof(out[n].name) - 1);
            ++n;
        }
        out[r].launches += 1;
        out[r].total_ms += ms;
    }
    g_prof.used = 0;
    return n;
}

const char *kvm_last_error(void) { return g_err; }

const char *kvm_version(void) { return "0.1.0"; }

}  // extern "C"
