// Host side of the entry points without routing (windows, paged caches): argument checks, workspace layout, launches.
// See include/dhsa.h for the contract of every one.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <initializer_list>

#include "paged.h"

using namespace dhsa;

namespace {

#define DHSA_API __attribute__((visibility("default")))

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool odd_words(std::initializer_list<const void *> all) {
    for (const void *p : all)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return true;
    return false;
}
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

// What the two problem structs have in common.
dhsa_status heads(int64_t H_q, int64_t H_kv, int32_t D, int32_t dtype, float scale, SpanArgs *a) {
    if (dtype != DHSA_F32 && dtype != DHSA_BF16) return DHSA_ERR_DTYPE;
    if (H_q < 1 || H_kv < 1 || H_q % H_kv != 0 || H_q > 65535 - H_kv) return DHSA_ERR_SHAPE;
    if (D != 64 && D != 128) return DHSA_ERR_SHAPE;
    if (!(scale >= 0.f) || !isfinite(scale)) return DHSA_ERR_SHAPE;
    *a = SpanArgs{};
    a->H_kv = (int)H_kv;
    a->G = (int)(H_q / H_kv);
    set_divisor((uint32_t)a->G, &a->g_mul, &a->g_shift);
    a->scale_log2e = (scale > 0.f ? scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
    return DHSA_OK;
}

// A stride in elements between n of something: the default where it is 0 or nothing is that far apart, at least `least`, a
// multiple of 16 bytes.
dhsa_status stride(int64_t in, int64_t n, int64_t packed, int64_t least, int esz, int64_t *out) {
    *out = in && n > 1 ? in : packed;
    if (*out < least || *out > INT64_MAX / 64) return DHSA_ERR_SHAPE;
    return (*out * esz) % 16 != 0 ? DHSA_ERR_ALIGN : DHSA_OK;
}

// Do n rows of `step` elements' distance, behind m of `far`, end within 64 GiB?
bool fits(int64_t n, int64_t step, int64_t m, int64_t far, int D, int esz) {
    const __int128 last = (__int128)(n - 1) * step + (__int128)(m - 1) * far + D;
    return last * esz < (__int128)1 << 36;
}

dhsa_status resolve_paged(const dhsa_paged *in, SpanArgs *a, AppendArgs *ap) {
    if (!in) return DHSA_ERR_NULL;
    dhsa_status st = heads(in->H_q, in->H_kv, in->D, in->dtype, in->scale, a);
    if (st != DHSA_OK) return st;
    if (in->n_seq < 0 || in->n_seq > 65535 || in->T < 0 || in->T > INT_MAX / a->G) return DHSA_ERR_SHAPE;
    if (in->page_size < 1 || in->n_pages < 1 || in->max_pages < 1) return DHSA_ERR_SHAPE;
    if ((int64_t)in->page_size * in->max_pages > (int64_t)1 << 30) return DHSA_ERR_SHAPE;
    if (in->window < 0 || in->sinks < 0) return DHSA_ERR_SHAPE;
    const int esz = in->dtype == DHSA_F32 ? 4 : 2;
    const int64_t D = in->D, T = in->T, ps = in->page_size, H_kv = in->H_kv;
    int64_t ks_p, ks_h, ks_s, vs_p, vs_h, vs_s, kn_h, kn_t, vn_h, vn_t;
    const int64_t H_q = in->H_q, np = in->n_pages;
    const struct { int64_t in, n, packed, least; int64_t *out; } all[] = {
        {in->q_stride_h, H_q, std::max<int64_t>(T, 1) * D, 0, &a->qs_h}, {in->q_stride_t, T, D, D, &a->qs_t},
        {in->o_stride_h, H_q, std::max<int64_t>(T, 1) * D, 0, &a->os_h}, {in->o_stride_t, T, D, D, &a->os_t},
        {in->k_stride_p, np, H_kv * ps * D, D, &ks_p}, {in->k_stride_h, H_kv, ps * D, 0, &ks_h}, {in->k_stride_s, ps, D, D, &ks_s},
        {in->v_stride_p, np, H_kv * ps * D, D, &vs_p}, {in->v_stride_h, H_kv, ps * D, 0, &vs_h}, {in->v_stride_s, ps, D, D, &vs_s},
        {in->kn_stride_h, H_kv, std::max<int64_t>(T, 1) * D, 0, &kn_h}, {in->kn_stride_t, T, D, D, &kn_t},
        {in->vn_stride_h, H_kv, std::max<int64_t>(T, 1) * D, 0, &vn_h}, {in->vn_stride_t, T, D, D, &vn_t}};
    for (const auto &x : all)
        if ((st = stride(x.in, x.n, x.packed, x.least, esz, x.out)) != DHSA_OK) return st;
    if (!fits(in->n_pages, ks_p, ps, ks_s, in->D, esz) || !fits(in->n_pages, vs_p, ps, vs_s, in->D, esz)) return DHSA_ERR_SHAPE;
    a->T = T;
    a->n_seq = in->n_seq;
    a->n_pages = in->n_pages; a->max_pages = in->max_pages; a->page_size = in->page_size;
    a->slots_max = in->page_size * in->max_pages;
    set_divisor((uint32_t)in->page_size, &a->div_mul, &a->div_shift);
    a->window = in->window == 0 || in->window > INT_MAX ? INT_MAX : (int)in->window;
    a->sinks = (int)std::min<int64_t>(in->sinks, INT_MAX);
    // (a stride of a single page or slot is not used and may not fit)
    a->ks_p = in->n_pages > 1 ? (uint32_t)(ks_p * esz / 16) : 0; a->ks_s = ps > 1 ? (uint32_t)(ks_s * esz / 16) : 0;
    a->vs_p = in->n_pages > 1 ? (uint32_t)(vs_p * esz / 16) : 0; a->vs_s = ps > 1 ? (uint32_t)(vs_s * esz / 16) : 0;
    a->ks_h = ks_h * esz; a->vs_h = vs_h * esz;
    if (ap) { ap->kns_h = kn_h * esz; ap->kns_t = kn_t * esz; ap->vns_h = vn_h * esz; ap->vns_t = vn_t * esz; }
    return DHSA_OK;
}

// Workspace of dhsa_paged_attend in bytes: what a call wants, and the least that it runs with.
struct PagedWs { int64_t off_state, off_part, off_cut, off_norm, off_scores, bytes, least; };
PagedWs paged_ws(SpanArgs *a, int D, int dtype, bool weights) {
    choose_tiles(a, dtype, true);
    const int64_t M = a->M;
    PagedWs w;
    const int64_t rows = a->T * a->H_kv * a->G;
    w.off_state = 0;
    w.off_part = w.off_state + up256((int64_t)a->part_cap * M * 8);
    w.off_cut = w.off_part + up256((int64_t)a->part_cap * M * D * 4);
    w.off_norm = w.off_cut + up256(rows * 8);
    w.off_scores = w.off_norm + (weights ? up256(rows * 8) : 0);
    // Scores that are kept for the weights: every slot of the pool once, for as many rows as a sequence has in the mean (a
    // step of a batch has the same number of each).  What does not fit is computed again.  Where the mean is no longer few
    // rows one sequence has more and keeps none (63 single tokens of 1000..32000 and a chunk of 2048 in fp32: 4.9 ms, 6.0 with none kept).
    a->score_units = 0;
    if (weights && a->M <= kFewRows && a->T > 0 && a->n_seq > 0) {
        const int64_t mean = (a->T * a->G + a->n_seq - 1) / a->n_seq, pool = (int64_t)a->n_pages * a->page_size;
        const int64_t rows_kept = mean <= kFewRows ? a->T * a->G : (int64_t)kFewRows * (a->n_seq - 1);
        const int64_t every = rows_kept * ((a->slots_max + 63) / 64);      // of a kv-head, were all sequences as long as they can be
        const int64_t once = std::min(mean, (int64_t)kFewRows) * (pool / 64) + rows_kept;
        a->score_units = (int)std::min<int64_t>(std::min(every, once) * a->H_kv, kScoreUnitsMax);
    }
    w.bytes = w.off_scores + (int64_t)a->score_units * 256;
    // Room for scores makes the size fall where more tokens mean that fewer are kept.  A workspace of any larger T has to do: from T1
    // on only what comes before the scores is needed, which never falls; below, that of T1 is enough.
    w.least = w.bytes;
    if (a->score_units > 0) {
        const int64_t T1 = dtype == DHSA_BF16 ? ((int64_t)(kFewMean + 1) * a->n_seq + a->G - 1) / a->G : (int64_t)kFewRows * a->n_seq / a->G + 1;
        if (a->T >= T1) {
            w.least = w.off_scores;
        } else {
            SpanArgs b = *a;
            b.T = T1;
            w.least = std::min(w.bytes, paged_ws(&b, D, dtype, true).off_scores);
        }
    }
    return w;
}

dhsa_status hip_status(hipError_t e) { return e == hipSuccess ? DHSA_OK : DHSA_ERR_HIP; }

}  // namespace

extern "C" {

DHSA_API dhsa_status dhsa_window_prefill(const dhsa_problem *prob, int64_t window, int64_t sinks, const void *Q_dev,
                                         const void *K_dev, const void *V_dev, void *O_dev, void *stream) {
    if (!prob) return DHSA_ERR_NULL;
    SpanArgs a;
    dhsa_status st = heads(prob->H_q, prob->H_kv, prob->D, prob->dtype, prob->scale, &a);
    if (st != DHSA_OK) return st;
    if (prob->L < 1 || prob->L > INT_MAX / a.G || window < 1 || sinks < 0) return DHSA_ERR_SHAPE;
    const int esz = prob->dtype == DHSA_F32 ? 4 : 2;
    const int64_t D = prob->D, L = prob->L;
    int64_t ks_h, ks_l, vs_h, vs_l;
    const int64_t H_q = prob->H_q, H_kv = prob->H_kv;
    const struct { int64_t in, n, packed, least; int64_t *out; } all[] = {
        {prob->q_stride_h, H_q, L * D, 0, &a.qs_h}, {prob->q_stride_l, L, D, D, &a.qs_t}, {prob->k_stride_h, H_kv, L * D, 0, &ks_h},
        {prob->k_stride_l, L, D, D, &ks_l}, {prob->v_stride_h, H_kv, L * D, 0, &vs_h}, {prob->v_stride_l, L, D, D, &vs_l},
        {prob->o_stride_h, H_q, L * D, 0, &a.os_h}, {prob->o_stride_l, L, D, D, &a.os_t}};
    for (const auto &x : all)
        if ((st = stride(x.in, x.n, x.packed, x.least, esz, x.out)) != DHSA_OK) return st;
    if (!fits(L, ks_l, 1, 0, prob->D, esz) || !fits(L, vs_l, 1, 0, prob->D, esz)) return DHSA_ERR_SHAPE;
    // (as dhsa_prefill: the bf16 rows of a head are addressed with 32-bit offsets)
    if (prob->dtype == DHSA_BF16 && (L * ks_l * 2 > (int64_t)1 << 32 || L * vs_l * 2 > (int64_t)1 << 32)) return DHSA_ERR_SHAPE;
    if (!Q_dev || !K_dev || !V_dev || !O_dev) return DHSA_ERR_NULL;
    if (misaligned(Q_dev) || misaligned(K_dev) || misaligned(V_dev) || misaligned(O_dev)) return DHSA_ERR_ALIGN;
    a.Q = Q_dev; a.K = K_dev; a.V = V_dev; a.O = O_dev;
    a.T = L; a.n_seq = 1;
    a.window = window > INT_MAX ? INT_MAX : (int)window;
    a.sinks = (int)std::min<int64_t>(sinks, INT_MAX);
    a.ks_s = L > 1 ? (uint32_t)(ks_l * esz / 16) : 0; a.vs_s = L > 1 ? (uint32_t)(vs_l * esz / 16) : 0;
    a.ks_h = ks_h * esz; a.vs_h = vs_h * esz;
    choose_tiles(&a, prob->dtype, false);
    return hip_status(launch_span(a, prob->D, prob->dtype, static_cast<hipStream_t>(stream)));
}

DHSA_API dhsa_status dhsa_paged_append(const dhsa_paged *prob, const void *K_new_dev, const void *V_new_dev, void *K_dev,
                                       void *V_dev, const int32_t *table_dev, const int32_t *q_start_dev,
                                       const int32_t *kv_len_dev, float *weights_dev, void *stream) {
    SpanArgs a;
    AppendArgs ap;
    const dhsa_status st = resolve_paged(prob, &a, &ap);
    if (st != DHSA_OK) return st;
    if (a.n_seq == 0 || a.T == 0) return DHSA_OK;
    if (!K_new_dev || !V_new_dev || !K_dev || !V_dev || !table_dev || !q_start_dev || !kv_len_dev) return DHSA_ERR_NULL;
    if (misaligned(K_new_dev) || misaligned(V_new_dev) || misaligned(K_dev) || misaligned(V_dev) ||
        odd_words({table_dev, q_start_dev, kv_len_dev, weights_dev}))
        return DHSA_ERR_ALIGN;
    a.table = table_dev; a.q_start = q_start_dev; a.kv_len = kv_len_dev;
    ap.Kn = (const char *)K_new_dev; ap.Vn = (const char *)V_new_dev; ap.K = (char *)K_dev; ap.V = (char *)V_dev;
    ap.weights = weights_dev;
    return hip_status(launch_append(a, ap, prob->D * (prob->dtype == DHSA_F32 ? 4 : 2), static_cast<hipStream_t>(stream)));
}

DHSA_API size_t dhsa_paged_workspace_bytes(const dhsa_paged *prob, int weights) {
    SpanArgs a;
    if (resolve_paged(prob, &a, nullptr) != DHSA_OK) return 0;
    return (size_t)std::max<int64_t>(paged_ws(&a, prob->D, prob->dtype, weights != 0).bytes, 256);
}

DHSA_API dhsa_status dhsa_paged_attend(const dhsa_paged *prob, const void *Q_dev, const void *K_dev, const void *V_dev,
                                       const int32_t *table_dev, const int32_t *q_start_dev, const int32_t *kv_len_dev,
                                       void *O_dev, float *lse_dev, float *weights_dev, float decay, void *ws_dev,
                                       size_t ws_bytes, void *stream) {
    SpanArgs a;
    const dhsa_status st = resolve_paged(prob, &a, nullptr);
    if (st != DHSA_OK) return st;
    if (!(decay >= 0.f && decay <= 1.f)) return DHSA_ERR_SHAPE;
    if (a.n_seq == 0 || (a.T == 0 && !weights_dev)) return DHSA_OK;
    if ((a.T > 0 && (!Q_dev || !O_dev)) || !K_dev || !V_dev || !table_dev || !q_start_dev || !kv_len_dev || !ws_dev)
        return DHSA_ERR_NULL;
    if (misaligned(Q_dev) || misaligned(K_dev) || misaligned(V_dev) || misaligned(O_dev) || misaligned(ws_dev) ||
        odd_words({table_dev, q_start_dev, kv_len_dev, lse_dev, weights_dev}))
        return DHSA_ERR_ALIGN;
    const PagedWs w = paged_ws(&a, prob->D, prob->dtype, weights_dev != nullptr);
    if (ws_bytes < (size_t)w.least) return DHSA_ERR_WORKSPACE;
    a.score_units = (int)std::min<uint64_t>(a.score_units, (ws_bytes - (size_t)w.off_scores) / 256);      // (least has what comes before)
    char *ws = static_cast<char *>(ws_dev);
    a.Q = Q_dev; a.K = K_dev; a.V = V_dev; a.O = O_dev; a.lse = lse_dev;
    a.table = table_dev; a.q_start = q_start_dev; a.kv_len = kv_len_dev;
    a.cut = reinterpret_cast<int2 *>(ws + w.off_cut);
    a.state = reinterpret_cast<float2 *>(ws + w.off_state);
    a.part = reinterpret_cast<float *>(ws + w.off_part);
    if (weights_dev) a.norm = reinterpret_cast<float2 *>(ws + w.off_norm);
    if (a.score_units > 0) a.scores = reinterpret_cast<float *>(ws + w.off_scores);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = a.T > 0 ? launch_span(a, prob->D, prob->dtype, s) : hipSuccess;
    if (e == hipSuccess && weights_dev) e = launch_weights(a, prob->D, prob->dtype, weights_dev, decay, s);
    return hip_status(e);
}

DHSA_API size_t dhsa_paged_evict_workspace_bytes(const dhsa_paged *prob, int32_t keep) {
    SpanArgs a;
    if (resolve_paged(prob, &a, nullptr) != DHSA_OK || keep < 1 || keep > 1 << 30) return 0;
    const int64_t lists = (int64_t)std::max(a.n_seq, 1) * a.H_kv;
    return (size_t)(up256(lists * 4) + up256(lists * std::min<int64_t>(keep, a.slots_max) * 4));
}

DHSA_API dhsa_status dhsa_paged_evict(const dhsa_paged *prob, void *K_dev, void *V_dev, float *weights_dev,
                                      const int32_t *table_dev, const int32_t *kv_len_dev, int32_t keep, int32_t first,
                                      int32_t recent, const int32_t *table_out_dev, int32_t *kv_len_out_dev,
                                      int32_t *idx_dev, void *ws_dev, size_t ws_bytes, void *stream) {
    SpanArgs a;
    const dhsa_status st = resolve_paged(prob, &a, nullptr);
    if (st != DHSA_OK) return st;
    if (keep < 1 || keep > 1 << 30 || first < 0 || recent < 0 || (int64_t)first + recent > keep) return DHSA_ERR_BUDGET;
    if (a.n_seq == 0) return DHSA_OK;
    if (!K_dev || !V_dev || !weights_dev || !table_dev || !kv_len_dev || !table_out_dev || !kv_len_out_dev || !ws_dev)
        return DHSA_ERR_NULL;
    if (misaligned(K_dev) || misaligned(V_dev) || misaligned(ws_dev) ||
        odd_words({table_dev, kv_len_dev, table_out_dev, kv_len_out_dev, idx_dev, weights_dev}))
        return DHSA_ERR_ALIGN;
    if (ws_bytes < dhsa_paged_evict_workspace_bytes(prob, keep)) return DHSA_ERR_WORKSPACE;
    a.table = table_dev; a.kv_len = kv_len_dev;
    EvictArgs e;
    e.K = (char *)K_dev; e.V = (char *)V_dev; e.weights = weights_dev;
    e.table_out = table_out_dev; e.kv_out = kv_len_out_dev; e.idx = idx_dev;
    e.keep = keep; e.first = first; e.recent = recent;
    e.stride = (int)std::min<int64_t>(keep, a.slots_max);
    e.count = static_cast<int32_t *>(ws_dev);
    e.list = reinterpret_cast<int32_t *>(static_cast<char *>(ws_dev) + up256((int64_t)a.n_seq * a.H_kv * 4));
    return hip_status(launch_evict(a, e, prob->D * (prob->dtype == DHSA_F32 ? 4 : 2), static_cast<hipStream_t>(stream)));
}

}  // extern "C"
