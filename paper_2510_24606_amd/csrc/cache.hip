// A paged cache written and cut down: dhsa_paged_append, dhsa_paged_evict.
#include <algorithm>

#include "paged.h"

namespace dhsa {

// ---------------------------------------------------------------------------
// Append: a workgroup per new token moves its rows of all kv-heads, 16 bytes a thread.  Bound by a chain of three loads (the
// sequence of the token, its length, the page) where tokens are few (64 tokens of 8 kv-heads of 128, bf16: 3.0 us of kernel), by the
// copy where they are many (24K tokens, 195 MB: 38.2 us, 5.1 TB/s).
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_append(SpanArgs a, AppendArgs ap, int row16, int t0) {
    const int t = t0 + blockIdx.x, lane = threadIdx.x & 63;
    int s = 0;                                        // sequences that end at or before the token
    for (int s0 = 0; s0 < a.n_seq; s0 += 64) s += __popcll(__ballot(s0 + lane < a.n_seq && a.q_start[s0 + lane + 1] <= t));
    if (s >= a.n_seq) return;
    const Seq q = read_seq(a, s);
    const int slot = q.base + (t - (int)q.q0);
    if (t < q.q0 || t >= q.q0 + q.n || slot < 0 || slot >= q.kv) return;
    const int pi = page_of(a, slot), in = slot - pi * a.page_size, page = a.table[(int64_t)s * a.max_pages + pi];
    if ((unsigned)page >= (unsigned)a.n_pages) return;
    const int64_t kd = (int64_t)((uint64_t)((uint32_t)page * a.ks_p + (uint32_t)in * a.ks_s) << 4);
    const int64_t vd = (int64_t)((uint64_t)((uint32_t)page * a.vs_p + (uint32_t)in * a.vs_s) << 4);
    for (int x = threadIdx.x; x < a.H_kv * row16; x += 256) {
        const int g = x / row16, c = 16 * (x % row16);
        const uint4 k = *reinterpret_cast<const uint4 *>(ap.Kn + g * ap.kns_h + t * ap.kns_t + c);
        const uint4 v = *reinterpret_cast<const uint4 *>(ap.Vn + g * ap.vns_h + t * ap.vns_t + c);
        *reinterpret_cast<uint4 *>(ap.K + g * a.ks_h + kd + c) = k;
        *reinterpret_cast<uint4 *>(ap.V + g * a.vs_h + vd + c) = v;
    }
    if (ap.weights)
        for (int g = threadIdx.x; g < a.H_kv; g += 256) ap.weights[((int64_t)page * a.H_kv + g) * a.page_size + in] = 0.f;
}

hipError_t launch_append(const SpanArgs &a, const AppendArgs &ap, int row_bytes, hipStream_t s) {
    hipError_t e = hipSuccess;
    for (int64_t t0 = 0; t0 < a.T && e == hipSuccess; t0 += kGridMax) {
        hipLaunchKernelGGL(k_append, dim3((unsigned)std::min<int64_t>(a.T - t0, kGridMax)), dim3(256), 0, s, a, ap, row_bytes / 16, (int)t0);
        e = hipGetLastError();
    }
    return e;
}

// ---------------------------------------------------------------------------
// Eviction, first launch: which slots stay.  A workgroup per sequence and kv-head.  The middle slots [first, kv - recent) are
// ordered by a 32-bit key of their weight; the key of the last one that stays is found digit by digit (counts in LDS), then
// the slots above it, and of those equal to it the first ones, are listed in order.  What bounds it is the instructions of one CU
// per list: 1 us for each 1024 slots, behind 7 us of passes and barriers (8 x 8 lists of 8192..32768 slots 40 us).
// ---------------------------------------------------------------------------
// larger weight, larger key; -0 = 0; NaN and slots without a page: 0, less than any number
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;

// A wave has consecutive slots, 64 at a time; IT times 1024 slots keep their keys in registers (of IT = 32 the rounds' conditions spill
// 226 scalar registers into lanes of vector registers).  What is longer reads them again in each of five passes, page and weight one
// after the other: a list of 131072 takes 300 us.
// 8 x 8 lists of up to 32768 slots: 83 us with the keys read five times, by page and slot each time.
template <int IT>
__global__ __launch_bounds__(kEvictThreads) void k_evict_select(SpanArgs a, EvictArgs e) {
    __shared__ int hist[2048];
    __shared__ int s_gt[kEvictWaves], s_eq[kEvictWaves], s_scan[kEvictWaves];
    __shared__ int s_digit, s_left;
    const int g = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int kv = a.kv_len[s];
    kv = kv < 0 ? 0 : kv > a.slots_max ? a.slots_max : kv;
    const int64_t at = (int64_t)s * a.H_kv + g;
    int32_t *list = e.list + at * e.stride, *idx = e.idx ? e.idx + at * e.keep : nullptr;
    const int n = kv < e.keep ? kv : e.keep;
    if (tid == 0) e.count[at] = n;
    for (int x = n + tid; idx && x < e.keep; x += kEvictThreads) idx[x] = -1;
    const auto put = [&](int x, int slot) { list[x] = slot; if (idx) idx[x] = slot; };
    if (kv <= e.keep) {
        for (int x = tid; x < n; x += kEvictThreads) put(x, x);
        return;
    }
    const int m0 = e.first, m1 = kv - e.recent, need = e.keep - e.first - e.recent;
    for (int x = tid; x < e.first; x += kEvictThreads) put(x, x);
    for (int x = tid; x < e.recent; x += kEvictThreads) put(e.keep - e.recent + x, m1 + x);
    if (need == 0) return;
    const int32_t *table = a.table + (int64_t)s * a.max_pages;
    const int rounds = (m1 - m0 + kEvictThreads - 1) / kEvictThreads, w0 = m0 + wave * rounds * 64;
    // (page numbers and weights are asked for eight at a time, without a branch between them: one by one each round of the wave took
    // two trips to memory, 51 us for the lists above)
    const auto page_at = [&](int slot) { return table[page_of(a, slot)]; };
    const auto weight_at = [&](int slot, int page) {
        const bool ok = (unsigned)page < (unsigned)a.n_pages;
        const float w = e.weights[((int64_t)(ok ? page : 0) * a.H_kv + g) * a.page_size + (slot - page_of(a, slot) * a.page_size)];
        return ok ? weight_key(w) : 0u;
    };
    const auto read = [&](int slot) { return weight_at(slot, page_at(slot)); };
    uint32_t held[IT];
    if (rounds <= IT) {
        const auto slot = [&](int i) { const int x = w0 + 64 * i + lane; return x < m1 ? x : m1 - 1; };
        constexpr int B = IT < 8 ? IT : 8;
#pragma unroll
        for (int i0 = 0; i0 < IT; i0 += B) {
            if (i0 >= rounds) break;
            int page[B];
#pragma unroll
            for (int i = 0; i < B; ++i) page[i] = page_at(slot(i0 + i));
#pragma unroll
            for (int i = 0; i < B; ++i) held[i0 + i] = weight_at(slot(i0 + i), page[i]);
        }
    }
    // f(slot or -1, key) for every round of this wave
    const auto each = [&](auto f) {
        if (rounds <= IT) {
#pragma unroll
            for (int i = 0; i < IT; ++i)
                if (i < rounds) { const int x = w0 + 64 * i + lane; f(x < m1 ? x : -1, held[i]); }
        } else {
            for (int i = 0; i < rounds; ++i) { const int x = w0 + 64 * i + lane; f(x < m1 ? x : -1, read(x < m1 ? x : m1 - 1)); }
        }
    };
    // digits of 11, 11 and 10 bits
    uint32_t prefix = 0;
    int left = need;             // of the slots whose higher digits equal the prefix, how many stay
    for (int d = 0; d < 3; ++d) {
        const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, bins = d == 2 ? 1024 : 2048, above_shift = d == 2 ? 10 : 21;
        for (int x = tid; x < 2048; x += kEvictThreads) hist[x] = 0;
        __syncthreads();
        each([&](int x, uint32_t k) {
            if (x >= 0 && (d == 0 || k >> above_shift == prefix)) atomicAdd(&hist[k >> shift & (bins - 1)], 1);
        });
        __syncthreads();
        // thread i has the bins 2047 - 2 i and 2046 - 2 i: counts from the top down
        const int h1 = hist[2047 - 2 * tid], h0 = hist[2046 - 2 * tid];
        const int inc = wave_incl_scan(h0 + h1);
        if (lane == 63) s_scan[wave] = inc;
        __syncthreads();
        int above = inc - h0 - h1;
#pragma unroll
        for (int w = 0; w < kEvictWaves; ++w) above += w < wave ? s_scan[w] : 0;
        if (above < left && left <= above + h1) { s_digit = 2047 - 2 * tid; s_left = left - above; }
        else if (above + h1 < left && left <= above + h1 + h0) { s_digit = 2046 - 2 * tid; s_left = left - above - h1; }
        __syncthreads();
        prefix = prefix << (d == 2 ? 10 : 11) | (uint32_t)s_digit;
        left = s_left;
    }
    int gt = 0, eq = 0;
    each([&](int x, uint32_t k) {
        gt += x >= 0 && k > prefix;
        eq += x >= 0 && k == prefix;
    });
    gt = __builtin_amdgcn_readlane(wave_incl_scan(gt), 63);
    eq = __builtin_amdgcn_readlane(wave_incl_scan(eq), 63);
    if (lane == 0) { s_gt[wave] = gt; s_eq[wave] = eq; }
    __syncthreads();
    int gt0 = 0, eq0 = 0;        // above and equal in the slots before
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) {
        gt0 += w < wave ? s_gt[w] : 0;
        eq0 += w < wave ? s_eq[w] : 0;
    }
    each([&](int x, uint32_t k) {
        const unsigned long long mg = __ballot(x >= 0 && k > prefix), me = __ballot(x >= 0 && k == prefix);
        const unsigned long long below = (1ull << lane) - 1ull;
        const int ge = gt0 + __popcll(mg & below), ee = eq0 + __popcll(me & below);
        if (x >= 0 && (k > prefix || (k == prefix && ee < left))) put(e.first + ge + (ee < left ? ee : left), x);
        gt0 += __popcll(mg);
        eq0 += __popcll(me);
    });
}

// ---------------------------------------------------------------------------
// Eviction, second launch: the rows move.  In place one workgroup does its columns of a head: kept slots ascend, so row t moves
// from a slot >= t; batches are read whole before they are written, and a batch is written below everything that a later one
// reads.  Into other pages every batch has a workgroup of its own: 8 x 8 heads, 4096 rows each of K and V, 268 MB read and written,
// 50 us (5.3 TB/s); in place, where a head's columns are one workgroup's, 67 us.
// blockIdx.x: part (K columns, V columns, weights) and batch, y: kv-head, z: sequence.
// ---------------------------------------------------------------------------
constexpr int kMoveU = 4;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

template <typename V, int THREADS>
__device__ __forceinline__ void move_rows(const SpanArgs &a, const EvictArgs &e, int s, int n, const int32_t *list, char *base, uint64_t p16,
                                          uint64_t s16, int unit, int lanes, int width, int batch, int batches) {
    // lanes threads per row, width bytes each; strides in `unit` bytes
    const int tid = threadIdx.x, r = tid / lanes, c = tid % lanes * width, rows = THREADS / lanes;
    const int32_t *table = a.table + (int64_t)s * a.max_pages, *table_out = e.table_out + (int64_t)s * a.max_pages;
    const auto place = [&](int page, int slot) {
        return base + ((uint64_t)page * p16 + (uint64_t)(slot - page_of(a, slot) * a.page_size) * s16) * unit + c;
    };
    for (int t0 = batch * rows * kMoveU; t0 < n; t0 += batches * rows * kMoveU) {
        // slots, pages, rows: each of the kMoveU is asked for beside the others
        V x[kMoveU];
        int to[kMoveU], from[kMoveU], from_page[kMoveU], to_page[kMoveU];
        bool ok[kMoveU];
#pragma unroll
        for (int u = 0; u < kMoveU; ++u) {
            to[u] = t0 + u * rows + r < n ? t0 + u * rows + r : n - 1;
            from[u] = list[to[u]];
        }
#pragma unroll
        for (int u = 0; u < kMoveU; ++u) { from_page[u] = table[page_of(a, from[u])]; to_page[u] = table_out[page_of(a, to[u])]; }
#pragma unroll
        for (int u = 0; u < kMoveU; ++u) {
            const bool stays = table == table_out && from[u] == to[u];
            ok[u] = t0 + u * rows + r < n && !stays && (unsigned)from_page[u] < (unsigned)a.n_pages && (unsigned)to_page[u] < (unsigned)a.n_pages;
            x[u] = V{};
            if (ok[u]) x[u] = *reinterpret_cast<const V *>(place(from_page[u], from[u]));
        }
        if constexpr (THREADS == kEvictThreads) __syncthreads();
#pragma unroll
        for (int u = 0; u < kMoveU; ++u)
            if (ok[u]) *reinterpret_cast<V *>(place(to_page[u], to[u])) = x[u];
        if constexpr (THREADS == kEvictThreads) __syncthreads();
    }
}

// kEvictThreads: in place, one batch after another
constexpr int kMoveThreads = 256;
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_evict_move(SpanArgs a, EvictArgs e, int row16, int parts) {
    const int g = blockIdx.y, s = blockIdx.z, part = blockIdx.x % (2 * parts + 1), batch = blockIdx.x / (2 * parts + 1);
    const int batches = gridDim.x / (2 * parts + 1);
    const int64_t at = (int64_t)s * a.H_kv + g;
    const int n = e.count[at];
    const int32_t *list = e.list + at * e.stride;
    if (part == 2 * parts) {
        move_rows<float, THREADS>(a, e, s, n, list, (char *)(e.weights + (int64_t)g * a.page_size), (uint64_t)a.H_kv * a.page_size, 1, 4, 1, 4,
                         batch, batches);
        if (g == 0 && batch == 0 && threadIdx.x == 0) e.kv_out[s] = n;      // (nothing of this launch reads kv_len)
        return;
    }
    const bool is_k = part < parts;
    const int lanes = row16 / parts, c0 = (is_k ? part : part - parts) * lanes * 16;
    move_rows<u32x4_t, THREADS>(a, e, s, n, list, (is_k ? e.K + g * a.ks_h : e.V + g * a.vs_h) + c0, is_k ? a.ks_p : a.vs_p, is_k ? a.ks_s : a.vs_s, 16,
                     lanes, 16, batch, batches);
}

hipError_t launch_evict(const SpanArgs &a, const EvictArgs &e, int row_bytes, hipStream_t s) {
    const int row16 = row_bytes / 16;
    if (a.slots_max <= 4 * kEvictThreads) hipLaunchKernelGGL(k_evict_select<4>, dim3(a.H_kv, a.n_seq), dim3(kEvictThreads), 0, s, a, e);
    else hipLaunchKernelGGL(k_evict_select<32>, dim3(a.H_kv, a.n_seq), dim3(kEvictThreads), 0, s, a, e);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    if (e.table_out == a.table) {
        const int parts = row16 / 8;      // 128 bytes a part: what is in order is the work of one workgroup each
        hipLaunchKernelGGL(k_evict_move<kEvictThreads>, dim3(2 * parts + 1, a.H_kv, a.n_seq), dim3(kEvictThreads), 0, s, a, e, row16, parts);
    } else {
        const int64_t pieces = (int64_t)e.stride * row16, batches = std::min<int64_t>((pieces + kMoveThreads * kMoveU - 1) / (kMoveThreads * kMoveU), 256);
        hipLaunchKernelGGL(k_evict_move<kMoveThreads>, dim3((unsigned)(3 * batches), a.H_kv, a.n_seq), dim3(kMoveThreads), 0, s, a, e, row16, 1);
    }
    return hipGetLastError();
}

}  // namespace dhsa
