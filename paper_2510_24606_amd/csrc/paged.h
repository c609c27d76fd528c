// Shared by the translation units of attention without routing: windows and paged caches (see include/dhsa.h).
#pragma once
#include "dhsa_internal.h"
#include "divide.h"

namespace dhsa {

// Kernel arguments.  A contiguous K / V (dhsa_window_prefill) is one sequence of one page, q_start = nullptr.
// Strides of K and V are in units of 16 bytes, so that the place of a row fits 32 bits (64 GiB).
struct SpanArgs {
    const void *Q, *K, *V;
    void *O;
    float *lse;                  // [H_q][T] or nullptr
    float2 *norm;                // [H_q][T] or nullptr: exponent reference (log2) and 1 / sum of each row, for the weights
    const int32_t *table, *q_start, *kv_len;
    int64_t T;
    int n_seq, H_kv, G;
    int n_pages, max_pages, page_size;
    uint32_t div_mul;            // of page_size (see divide.h)
    int div_shift;
    int window, sinks;           // window = INT_MAX: none
    int slots_max;               // max_pages page_size
    float scale_log2e;
    int64_t qs_h, qs_t, os_h, os_t;                 // elements
    uint32_t ks_p, ks_s, vs_p, vs_s;                // 16 bytes
    int64_t ks_h, vs_h;                             // bytes
    // pieces of key ranges: about `target` of them over all (0: every row tile has its range in one piece); what is cut
    // leaves the states of its rows in `part` (piece, row: D floats) and `state` (reference, sum), and in `cut` ([H_q][T]) where
    // a row's first state is and how many pieces it has (one: the row is done)
    int M, target, part_cap;     // M: rows of a tile
    float *part;
    float2 *state;
    int2 *cut;
    int g_shift;                 // of G
    uint32_t g_mul;
    // scores of sequences of at most kFewRows rows a kv-head, for the weights (nullptr: none are kept): score_units times 64.  A
    // kv-head of a sequence has 64 ceil(kv / 64) for each row, its packed keys in blocks of 32, the rows of a block side by side
    float *scores;
    int score_units;
};

// What a row's state (reference m, log2; sum l) gives.  Without a key m = -inf and l = 0; a row whose scores are NaN has l = NaN and
// says so in O and lse, while a key that it does not see has its factor of 0 in the weights (those that it sees have its NaN score).
__device__ __forceinline__ float inv_of(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f; }
__device__ __forceinline__ float2 norm_of(float m, float l) { return l > 0.f ? make_float2(m, 1.f / l) : make_float2(1e30f, 0.f); }

constexpr int kIntMaxP = 0x7fffffff;
constexpr int kFewRows = 32;
constexpr int kFewMean = 16;                 // rows a kv-head and sequence in the mean up to which tiles are the smallest
constexpr int kScoreUnitsMax = 1 << 24;      // 4 GiB; 64 times that fits 32 bits

// One sequence as the kernels see it: whatever is in the arrays, rows stay below T and slots below slots_max.  What does not fit is
// left out; the rows and slots that are there keep their places.
struct Seq {
    int64_t q0;   // first row
    int n, kv;    // rows, slots that there are
    int base;     // slot (position) of the first row: negative for rows that see nothing, kv and more for those behind the slots
};
__device__ __forceinline__ Seq read_seq(const SpanArgs &a, int s) {
    Seq q;
    if (!a.q_start) { q.q0 = 0; q.n = q.kv = (int)a.T; q.base = 0; return q; }
    int b = a.q_start[s], e = a.q_start[s + 1], kv = a.kv_len[s];
    const int T = (int)a.T;
    b = b < 0 ? 0 : b > T ? T : b;
    kv = kv < 0 ? 0 : kv;
    q.base = e > b ? kv - (e - b) : 0;                   // the row before e has slot kv - 1
    e = e < b ? b : e > T ? T : e;
    kv = kv > a.slots_max ? a.slots_max : kv;
    q.q0 = b; q.n = e - b; q.kv = kv;
    return q;
}

// The keys of the slots [0, kv) that the rows at positions p0 .. p1 (p0 <= p1) see: [0, head) and [lo, hi), packed one behind the
// other.
struct Span {
    int lo, head, total;     // packed position x is slot x for x < head, x - head + lo behind
    __device__ __forceinline__ int slot(int x) const { return x < head ? x : x - head + lo; }
};
__device__ __forceinline__ Span make_span(const SpanArgs &a, int p0, int p1, int kv) {
    Span s;
    const int hi = p1 < 0 ? 0 : p1 < kv ? p1 + 1 : kv;
    s.lo = p0 >= a.window ? p0 - a.window + 1 : 0;
    s.lo = s.lo < hi ? s.lo : hi;
    s.head = a.sinks < s.lo ? a.sinks : s.lo;
    s.total = s.head + hi - s.lo;
    return s;
}

// Row key limits: a row at position p takes the key of slot j iff key_lo(j) < p < key_hi(j)
__device__ __forceinline__ int key_hi(const SpanArgs &a, int j) {
    return j < a.sinks || j > kIntMaxP - a.window ? kIntMaxP : j + a.window;
}

__device__ __forceinline__ int page_of(const SpanArgs &a, int slot) {
    return divided(slot, a.div_mul, a.div_shift);
}

__device__ __forceinline__ int token_of(const SpanArgs &a, int R) {
    return divided(R, a.g_mul, a.g_shift);
}

// Blocks of kept scores that a sequence needs: 0 if none are kept of it.  Sequences get theirs one after another; one that
// would end behind score_units has none (its weights are made from Q and K again).
__device__ __forceinline__ int score_need(const SpanArgs &a, const Seq &q) {
    const int64_t rows = (int64_t)q.n * a.G;
    if (!a.scores || rows > kFewRows) return 0;
    const int64_t need = rows * a.H_kv * ((q.kv + 63) >> 6);
    return need > kScoreUnitsMax ? kScoreUnitsMax + 1 : (int)need;
}
__device__ __forceinline__ int capped(int units) { return units > kScoreUnitsMax ? kScoreUnitsMax + 1 : units; }   // (fits no workspace)

// fp32 sum over the wave, in every lane; the order is fixed
__device__ __forceinline__ float wave_sum(float x) {
#define DHSA_STEP(CTRL, ROWS) x += __int_as_float(dpp_or<CTRL, ROWS>(0, __float_as_int(x)));
    DHSA_DPP_STEPS(DHSA_STEP)
#undef DHSA_STEP
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// A workgroup's share: rows [R0, R0 + rows) of kv-head g in sequence s (row R is token R / G, query head g G + R % G) and the
// packed keys [x0, x1) of what these rows see.
struct Item {
    Seq q;
    int s, g, R0, rows, piece, pieces, slot;
    float *scores;   // of the kv-head, or nullptr
};
__device__ __forceinline__ int64_t score_at(int rows, int R, int x) { return ((int64_t)(x >> 5) * rows + R) * 32 + (x & 31); }

// Which share workgroup b has, M rows a tile and U keys a unit.  Every wave finds out for itself, without a barrier: lane i
// looks at sequence 64 r + i.  A sequence's tiles all have as many pieces as its longest one needs, so that a piece has at most
// P units, where P makes about `target` pieces of all.  Later rows (longer ranges) come first.
__device__ __forceinline__ bool find_item(const SpanArgs &a, unsigned b, int M, int U, Item *it) {
    const int lane = threadIdx.x & 63;
    const int g = (int)(b % (unsigned)a.H_kv), want = (int)(b / (unsigned)a.H_kv);
    int P = kIntMaxP;
    const int t_in = (M + a.G - 1) / a.G + 1;                           // most tokens a tile touches
    const auto measure = [&](int s, Seq *q, int *tiles, int *units) {
        *tiles = *units = 0;
        q->n = 0;
        if (s >= a.n_seq) return;
        *q = read_seq(a, s);
        *tiles = (int)(((unsigned)(q->n * a.G) + (M - 1)) / M);         // (n G < 2^31)
        const int p1 = q->base + q->n - 1, p0 = p1 - t_in + 1 > 0 ? p1 - t_in + 1 : 0;
        *units = (make_span(a, p0, p1, q->kv).total + U - 1) / U;
    };
    Seq q;
    int tiles, units;
    if (a.target > 0) {
        float cost = 0.f;
        for (int s = lane; s < a.n_seq + lane; s += 64) {
            measure(s, &q, &tiles, &units);
            cost += (float)tiles * (float)units;
        }
        cost = wave_sum(cost);
        const float p = cost * (float)a.H_kv / (float)a.target;
        P = p < 1e9f ? (int)(p * 1.00001f) + 1 : 1000000000;
    }
    int base = 0, part = 0, units_before = 0;
    bool found = false;
    for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
        if (s0 > 0 || a.n_seq > 64 || a.target <= 0) measure(s0 + lane, &q, &tiles, &units);
        const int pieces = units > P ? (units + P - 1) / P : 1;
        const int np = tiles * pieces, cut = pieces > 1 ? np : 0;
        const int end = wave_incl_scan(np), cut_end = wave_incl_scan(cut);
        const int total = __builtin_amdgcn_readlane(end, 63), cut_total = __builtin_amdgcn_readlane(cut_end, 63);
        int need = 0, need_end = 0;
        if (a.scores) {
            need = s0 + lane < a.n_seq ? score_need(a, q) : 0;
            need_end = wave_incl_scan(need);
        }
        if (want < base + total) {
            const int from = base + end - np;
            const unsigned long long hit = __ballot(want >= from && want < base + end);
            if (hit == 0) return false;      // (arrays that are no sequences, whose tiles overflow)
            const int l = __builtin_ctzll(hit);
            const auto of = [l](int x) { return __builtin_amdgcn_readlane(x, l); };
            it->s = s0 + l;
            it->g = g;
            it->q.q0 = of((int)q.q0); it->q.n = of(q.n); it->q.kv = of(q.kv); it->q.base = of(q.base);
            const int at = want - of(from), t = of(tiles);
            it->pieces = of(pieces);
            it->piece = at % it->pieces;
            it->R0 = (t - 1 - at / it->pieces) * M;
            const int64_t left = (int64_t)it->q.n * a.G - it->R0;
            it->rows = left < M ? (int)left : M;
            it->slot = it->pieces > 1 ? (part + of(cut_end - cut) + at) * a.H_kv + g : -1;
            it->scores = nullptr;
            const int units = of(need), end_units = capped(units_before + of(need_end));
            if (units > 0 && end_units <= a.score_units)
                it->scores = a.scores + (int64_t)(end_units - units) * 64 + (int64_t)g * it->q.n * a.G * ((it->q.kv + 63) >> 6 << 6);
            found = true;
        }
        units_before = capped(units_before + __builtin_amdgcn_readlane(need_end, 63));
        base += total;
        part += cut_total;
        if (found) break;
    }
    return found;
}

// ---- launchers ----
constexpr int kTallRows = 128;                                      // rows of a tile of span_tall.hip
void choose_tiles(SpanArgs *a, int dtype, bool paged);              // sets M, target and part_cap: workspace and launches go by them
hipError_t launch_span_tall(const SpanArgs &a, int D, unsigned blocks, unsigned block0, hipStream_t s);
hipError_t launch_span(const SpanArgs &a, int D, int dtype, hipStream_t s);
hipError_t launch_weights(const SpanArgs &a, int D, int dtype, float *weights, float decay, hipStream_t s);

struct AppendArgs {
    const char *Kn, *Vn;
    char *K, *V;
    float *weights;
    int64_t kns_h, kns_t, vns_h, vns_t;     // bytes
};
hipError_t launch_append(const SpanArgs &a, const AppendArgs &ap, int row_bytes, hipStream_t s);

struct EvictArgs {
    char *K, *V;
    float *weights;
    const int32_t *table_out;
    int32_t *kv_out, *idx, *list, *count;   // list [n_seq][H_kv][stride], count [n_seq][H_kv]
    int keep, first, recent, stride;
};
hipError_t launch_evict(const SpanArgs &a, const EvictArgs &e, int row_bytes, hipStream_t s);

}  // namespace dhsa
