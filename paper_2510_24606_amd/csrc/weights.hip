// What each cached key has got of attention (dhsa_paged_attend with weights).  With the exponent reference and the sum of each row,
// which attention has left, a score gives its probability at once: exp2(s c - reference) / sum.  Every key's sum over rows and heads
// is made by one workgroup in a fixed order; nothing is added with atomics.
//
// A workgroup takes shares of two kinds, one after another:
//   * 4096 keys of a kv-head of a sequence whose scores were kept (few rows): they are read, four times four keys a thread.
//   * otherwise the scores are made again from Q and K.  bf16: 128 keys, 32 in the registers of each wave, and the rows that see
//     them staged through LDS in blocks of 64 (K from memory once, Q once per 128 keys).  S^T (keys x rows) = K Q^T, so a lane
//     has 16 keys of one row: it adds up its own keys over its rows, and the 32 rows of a block follow once at the end.  Bound
//     by the vector unit: an exponential, a product and two sums a pair beside 16 cycles of matrix unit for 64 pairs.
//     fp32: 64 keys in the registers of every wave, each of which takes every fourth block of 16 rows.
// Kept scores of 64 conversations (74 MB, 578K tokens of 8 kv-heads) 31 us; computing them again from K would read 1.2 GB, 215 us.
// 5718 new tokens of 12 sequences, groups of seven heads, a window of 4096: 249 us (vector unit busy 63 % of the cycles).  fp32, 1024
// tokens behind 7168, 32 heads of 8 kv-heads of 128: 567 us (114 TFLOP/s).
#include <algorithm>

#include "attn_mfma.h"
#include "paged.h"

namespace dhsa {

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kKeptKeys = 4096;
constexpr int kStages = 3;       // of 64 rows in LDS: two are on their way while one is worked on

template <typename T> struct Heavy;
template <> struct Heavy<bf16_t> { static constexpr int kKeys = 128; };
template <> struct Heavy<float> { static constexpr int kKeys = 64; };

template <typename T, int D> struct WeightsSmem;
template <int D> struct WeightsSmem<bf16_t, D> {
    alignas(1024) uint16_t q[kStages][64 * D];
    float norm[kStages][4][64];      // references, 1 / sums, and what the other two waves load beside their rows
    float sum[128];
};
template <int D> struct WeightsSmem<float, D> {
    float sum[4][64];
};

// The rows (of a kv-head) that may see one of the keys j0 .. j1: [r0, r1)
__device__ __forceinline__ void rows_of(const SpanArgs &a, const Seq &sq, int j0, int j1, int *r0, int *r1) {
    const int64_t first = (int64_t)j0 - sq.base;       // row of the token at j0
    const int64_t far = (int64_t)key_hi(a, j1) - sq.base;      // no row from here on sees the last key
    const int t0 = first < 0 ? 0 : first < sq.n ? (int)first : sq.n;
    const int t1 = j0 < a.sinks || far >= sq.n ? sq.n : far < t0 ? t0 : (int)far;
    *r0 = t0 * a.G;
    *r1 = t1 * a.G;
}

__device__ __forceinline__ void put_weight(const SpanArgs &a, const int32_t *table, int g, int j, float *W, float decay, float x) {
    const int pi = page_of(a, j), page = table[pi];
    if ((unsigned)page >= (unsigned)a.n_pages) return;
    float *w = W + ((int64_t)page * a.H_kv + g) * a.page_size + (j - pi * a.page_size);
    *w = decay > 0.f ? decay * *w + x : x;
}

__device__ __forceinline__ void load16_to_lds(uint64_t addr, unsigned lds_window) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(addr), "s"(lds_window) : "memory");
#else
    (void)addr; (void)lds_window;
#endif
}
__device__ __forceinline__ void load4_to_lds(uint64_t addr, unsigned lds_window) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(addr), "s"(lds_window) : "memory");
#else
    (void)addr; (void)lds_window;
#endif
}
template <int N> __device__ __forceinline__ void wait_loads() {      // all but the last N of this wave have landed
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
#endif
}

// byte address of row j of K of kv-head g (a page that is none: page 0, whose sums are not written)
__device__ __forceinline__ const char *key_row(const SpanArgs &a, const int32_t *table, int g, int j) {
    const int pi = page_of(a, j);
    int page = table[pi];
    if ((unsigned)page >= (unsigned)a.n_pages) page = 0;
    return (const char *)a.K + g * a.ks_h + ((uint64_t)((uint32_t)page * a.ks_p + (uint32_t)(j - pi * a.page_size) * a.ks_s) << 4);
}

// ---- bf16: the sums of keys j0 .. j0 + keys - 1 (at most 128), left in sm.sum ----
template <int D>
__device__ __forceinline__ void heavy_sums(WeightsSmem<bf16_t, D> &sm, const SpanArgs &a, const Seq &sq, const int32_t *table, int g, int j0,
                                           int keys) {
    constexpr int OPR = D / 8, NS = D / 16, LPS = 64 * OPR / 256, RPW = 64 / OPR;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 31, g2 = lane >> 5, base = sq.base;
    const float c = a.scale_log2e;
    int R0, R1;
    rows_of(a, sq, j0, j0 + keys - 1, &R0, &R1);
    const int kw = j0 + 32 * wave;                     // this wave's first key
    f32x16 sum;
#pragma unroll
    for (int x = 0; x < 16; ++x) sum[x] = 0.f;
    __syncthreads();                                   // the stages and sums of the share before have been read
    if (R0 < R1) {
        bf16x8 kf[NS];
        {
            const char *row = key_row(a, table, g, kw + lr < j0 + keys ? kw + lr : j0 + keys - 1) + 16 * g2;
#pragma unroll
            for (int s = 0; s < NS; ++s) kf[s] = *reinterpret_cast<const bf16x8 *>(row + 32 * s);
        }
        // Staging: load i of a wave fills the KiB 4 i + wave of the stage; pieces of a row are swizzled as in span_tall.hip.  Wave 0
        // also loads the rows' references, wave 1 their 1 / sums, the others something, so that all wait for the same number.
        const int ld_row0 = wave * RPW + lane / OPR;
        const unsigned ld_piece = 16u * ((lane % OPR) ^ piece_swizzle(ld_row0, OPR));
        const unsigned lds_q = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint16_t *)sm.q;
        const unsigned lds_n = (unsigned)(uintptr_t)(__attribute__((address_space(3))) float *)sm.norm;
        const uint64_t Qg = (uint64_t)(uintptr_t)((const uint16_t *)a.Q + (int64_t)g * a.G * a.qs_h + sq.q0 * a.qs_t) + ld_piece;
        const uint64_t Ng = (uint64_t)(uintptr_t)(a.norm + (int64_t)g * a.G * a.T + sq.q0) + (wave == 1 ? 4 : 0);
        const auto ask = [&](int R, int buf) {         // rows from R on (behind the last one: that one again)
#pragma unroll
            for (int i = 0; i < LPS; ++i) {
                const int r = R + ld_row0 + 4 * RPW * i, rr = r < R1 ? r : R1 - 1, t = token_of(a, rr), h = rr - t * a.G;
                load16_to_lds(Qg + 2 * (h * a.qs_h + t * a.qs_t), lds_q + buf * 128 * D + wave * 1024 + 4096 * i);
            }
            const int rr = R + lane < R1 ? R + lane : R1 - 1, t = token_of(a, rr), h = rr - t * a.G;
            load4_to_lds(Ng + 8 * (h * a.T + t), lds_n + (buf * 4 + wave) * 256);
        };
        ask(R0, 0);
        ask(R0 + 64, 1);
        __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0), in words that the compiler counts too: the keys are there
        __syncthreads();
        const int q_sw = piece_swizzle(lr, OPR);
        const int k_last = kw + 31 < sq.kv ? kw + 31 : sq.kv - 1;
        const int k_far = kw < a.sinks && k_last < a.sinks ? kIntMaxP : key_hi(a, kw < a.sinks ? a.sinks : kw);
        for (int R = R0, buf = 0; R < R1; R += 64, buf = buf == kStages - 1 ? 0 : buf + 1) {
            ask(R + 128, buf == 0 ? kStages - 1 : buf - 1);
            // do all rows of the stage see all keys of the wave?
            const int p0 = base + token_of(a, R), p1 = base + token_of(a, R + 63 < R1 ? R + 63 : R1 - 1);
            const bool masked = k_last > p0 || k_far <= p1;
#pragma unroll
            for (int rb = 0; rb < 2; ++rb) {
                f32x16 s_;
#pragma unroll
                for (int x = 0; x < 16; ++x) s_[x] = 0.f;
                const char *qp = (const char *)sm.q[buf] + 2 * (rb * 32 + lr) * D;
#pragma unroll
                for (int s = 0; s < NS; ++s)
                    s_ = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], *reinterpret_cast<const bf16x8 *>(qp + 16 * ((2 * s + g2) ^ q_sw)), s_, 0, 0, 0);
                const float ref = sm.norm[buf][0][rb * 32 + lr], inv = R + rb * 32 + lr < R1 ? sm.norm[buf][1][rb * 32 + lr] : 0.f;
                if (masked) {
                    // distance to the wave's first key of this lane; one comparison says both "not behind the row" and "in the window"
                    const int p = base + token_of(a, R + rb * 32 + lr < R1 ? R + rb * 32 + lr : R1 - 1), d = p - kw - 4 * g2;
                    if (kw < a.sinks) {
#pragma unroll
                        for (int x = 0; x < 16; ++x) {
                            const int k = (x & 3) + 8 * (x >> 2);
                            s_[x] = (unsigned)(d - k) < (unsigned)a.window || (kw + 4 * g2 + k < a.sinks && d >= k) ? s_[x] : -INFINITY;
                        }
                    } else {
#pragma unroll
                        for (int x = 0; x < 16; ++x) s_[x] = (unsigned)(d - (x & 3) - 8 * (x >> 2)) < (unsigned)a.window ? s_[x] : -INFINITY;
                    }
                }
#pragma unroll
                for (int x = 0; x < 16; ++x) sum[x] += __builtin_amdgcn_exp2f(s_[x] * c - ref) * inv;
            }
            wait_loads<LPS + 1>();                     // of the next stage; those of the one behind it may be on their way
            __syncthreads();
        }
        wait_loads<0>();
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) {
        float v = sum[x];
        v += __shfl_xor(v, 1); v += __shfl_xor(v, 2); v += __shfl_xor(v, 4); v += __shfl_xor(v, 8); v += __shfl_xor(v, 16);
        if (lr == 0) sm.sum[32 * wave + (x & 3) + 8 * (x >> 2) + 4 * g2] = v;
    }
    __syncthreads();
}

// ---- fp32: the sums of at most 64 keys of this wave's rows, left in sm.sum ----
template <int D>
__device__ __forceinline__ void heavy_sums(WeightsSmem<float, D> &sm, const SpanArgs &a, const Seq &sq, const int32_t *table, int g, int j0,
                                           int keys) {
    constexpr int NT = D / 16;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, q = lane >> 4, base = sq.base;
    const float c = a.scale_log2e;
    f32x4_t kf[4][NT], sum[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const char *row = key_row(a, table, g, j0 + (16 * h + n < keys ? 16 * h + n : keys - 1));
#pragma unroll
        for (int t = 0; t < NT; ++t) kf[h][t] = *reinterpret_cast<const f32x4_t *>(row + 64 * t + 16 * q);
        sum[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    int R0, R1;
    rows_of(a, sq, j0, j0 + keys - 1, &R0, &R1);
    for (int R = R0 + 16 * wave; R < R1; R += 64) {
        const int rr = R + n < R1 ? R + n : R1 - 1, t = token_of(a, rr), h0 = g * a.G + rr - t * a.G;
        const char *row = (const char *)((const float *)a.Q + h0 * a.qs_h + (sq.q0 + t) * a.qs_t);
        f32x4_t qf[NT];
#pragma unroll
        for (int u = 0; u < NT; ++u) qf[u] = *reinterpret_cast<const f32x4_t *>(row + 64 * u + 16 * q);
        const float2 nm = a.norm[h0 * a.T + sq.q0 + t];
        const int p = R + n < R1 ? base + t : -1;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[h][u][e], qf[u][e], x, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = j0 + 16 * h + 4 * q + i;
                const float e = __builtin_amdgcn_exp2f(x[i] * c - nm.x) * nm.y;
                sum[h][i] += j <= p && p < key_hi(a, j) ? e : 0.f;
            }
        }
    }
    __syncthreads();     // the sums of the share before have been read
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = sum[h][i];
            x += __shfl_xor(x, 1); x += __shfl_xor(x, 2); x += __shfl_xor(x, 4); x += __shfl_xor(x, 8);
            if (n == 0) sm.sum[wave][16 * h + 4 * q + i] = x;
        }
    __syncthreads();
}

template <int D> __device__ __forceinline__ float sum_of(const WeightsSmem<bf16_t, D> &sm, int k) { return sm.sum[k]; }
template <int D> __device__ __forceinline__ float sum_of(const WeightsSmem<float, D> &sm, int k) {
    return (sm.sum[0][k] + sm.sum[1][k]) + (sm.sum[2][k] + sm.sum[3][k]);
}

}  // namespace

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void k_weights(SpanArgs a, float *__restrict__ W, float decay) {
    constexpr int KEYS = Heavy<T>::kKeys;
    __shared__ WeightsSmem<T, D> sm;
    const int tid = threadIdx.x, lane = tid & 63;
    for (uint64_t b = blockIdx.x;; b += gridDim.x) {      // (sequences may share pages: their tiles together may pass 32 bits)
        // the share: as find_item, of key tiles
        const int g = (int)(b % (unsigned)a.H_kv);
        const int64_t want = (int64_t)(b / (unsigned)a.H_kv);
        int s = -1, tile = 0, units = 0, end_units = 0, before = 0;
        int64_t seen = 0;
        for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
            int tiles = 0, need = 0;
            if (s0 + lane < a.n_seq) {
                const Seq q = read_seq(a, s0 + lane);
                need = score_need(a, q);
                tiles = q.kv;
            }
            const int need_end = capped(before + wave_incl_scan(need));
            const bool kept = need > 0 && need_end <= a.score_units;
            tiles = kept ? (tiles + kKeptKeys - 1) / kKeptKeys : (tiles + KEYS - 1) / KEYS;
            const int end = wave_incl_scan(tiles), total = __builtin_amdgcn_readlane(end, 63);
            if (want < seen + total) {
                const int l = __builtin_ctzll(__ballot(want < seen + end));
                s = s0 + l;
                tile = (int)(want - seen) - __builtin_amdgcn_readlane(end - tiles, l);
                units = __builtin_amdgcn_readlane(kept ? need : 0, l);
                end_units = __builtin_amdgcn_readlane(need_end, l);
                break;
            }
            seen += total;
            before = __builtin_amdgcn_readlane(need_end, 63);
        }
        if (s < 0) return;
        const Seq sq = read_seq(a, s);
        const int32_t *table = a.table + (int64_t)s * a.max_pages;
        if (units == 0) {
            const int j0 = tile * KEYS, keys = sq.kv - j0 < KEYS ? sq.kv - j0 : KEYS;
            heavy_sums<D>(sm, a, sq, table, g, j0, keys);
            if (tid < keys) put_weight(a, table, g, j0 + tid, W, decay, sum_of<D>(sm, tid));
            continue;
        }
        // kept scores: row R of tile R / M has them in the order of the tile's span
        const int rows = sq.n * a.G, base = sq.base;
        const float *from = a.scores + (int64_t)(end_units - units) * 64 + (int64_t)g * rows * ((sq.kv + 63) >> 6 << 6);
        constexpr int U = kKeptKeys / 1024;
        const int j0 = tile * kKeptKeys + 4 * tid;
        f32x4_t sum[U];
#pragma unroll
        for (int u = 0; u < U; ++u) sum[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int R = 0; R < rows; ++R) {
            const int t = token_of(a, R), R0 = R / a.M * a.M;
            const int R_end = (R0 + a.M < rows ? R0 + a.M : rows) - 1;
            const Span span = make_span(a, base + token_of(a, R0), base + token_of(a, R_end), sq.kv);
            const float2 nm = a.norm[(int64_t)(g * a.G + R - t * a.G) * a.T + sq.q0 + t];
            f32x4_t x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + 1024 * u;
                if (span.lo == 0 && j + 3 < span.total) {
                    x[u] = *reinterpret_cast<const f32x4_t *>(from + score_at(rows, R, j));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = j + i < span.head ? j + i : j + i >= span.lo ? j + i - span.lo + span.head : kIntMaxP;
                        x[u][i] = at < span.total ? from[score_at(rows, R, at)] : -INFINITY;
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[u][i] += __builtin_amdgcn_exp2f(x[u][i] - nm.x) * nm.y;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (j0 + 1024 * u + i < sq.kv) put_weight(a, table, g, j0 + 1024 * u + i, W, decay, sum[u][i]);
    }
}

hipError_t launch_weights(const SpanArgs &a, int D, int dtype, float *W, float decay, hipStream_t s) {
    // One workgroup a share where the pool's slots are in one sequence each (they take further ones where they are not): shares differ
    // by how many rows see their keys, and the chip hands out workgroups as others end.  Chunks of 1..1024 tokens of 12 sequences, 1024
    // workgroups with every 1024th share 358 us.  Where scores may be kept shares are up to 64 times as large and there is no telling
    // how many: at most 1024 workgroups, so that a step of a batch does not begin with tens of thousands that find nothing.
    const int64_t keys = dtype == DHSA_F32 ? Heavy<float>::kKeys : Heavy<bf16_t>::kKeys;
    const int64_t shares = ((int64_t)a.n_pages * a.page_size / keys + a.n_seq) * a.H_kv;
    const dim3 grid((unsigned)std::min<int64_t>(shares, a.scores ? 1024 : 1 << 16));
    if (dtype == DHSA_F32) {
        if (D == 64) hipLaunchKernelGGL((k_weights<float, 64>), grid, dim3(256), 0, s, a, W, decay);
        else hipLaunchKernelGGL((k_weights<float, 128>), grid, dim3(256), 0, s, a, W, decay);
    } else {
        if (D == 64) hipLaunchKernelGGL((k_weights<bf16_t, 64>), grid, dim3(256), 0, s, a, W, decay);
        else hipLaunchKernelGGL((k_weights<bf16_t, 128>), grid, dim3(256), 0, s, a, W, decay);
    }
    return hipGetLastError();
}

}  // namespace dhsa
