// Attention without routing over a range of keys: windows and paged caches (dhsa_window_prefill, dhsa_paged_attend).
//
// Work unit (find_item): 16 RB rows of one kv-head and sequence -- the query heads of a group lie side by side, row R is
// token R / G -- and a piece of the keys that they see.  Four waves; each takes every fourth block of BK keys and all
// rows, with K and V from memory straight into the registers that the matrix unit reads, so there is no barrier in the
// loop; the waves' softmax states are joined at the end through LDS.
//
// Lane l = 16 q + n.  S^T (keys x rows) = K Q^T: the lane has the scores of row n against 4 keys 4 q + {0..3} of each 16.
// These are, after the exponential, the B operand of O^T (columns x rows) += V^T P^T when the contraction runs over the keys
// in that order.
//   bf16, BK = 32 (v_mfma_f32_16x16x32_bf16): the lane loads 16 bytes (8 for D = 64) at column D/16 n of the keys
//   {4 q + i, 16 + 4 q + i}, whole rows of V a quarter wave; operand j of V^T takes element j of each of the eight, put
//   together by byte permutes.  Row m of output block j is column D/16 m + j.
//   fp32, BK = 16 (v_mfma_f32_16x16x4_f32): K as 16 bytes at 16 s + 4 q, V as 16 bytes at 64 t + 4 n of key 4 q + i.  Row m
//   of output block (t, j) is column 64 t + 4 m + j.
//
// Tiles of 16 rows over a long cache are bound by the memory: 64 conversations of 578K tokens, 2.37 GB of K and V, 375 us (6.3 TB/s);
// one of 128K tokens 89 us (6.0 TB/s).  Tiles of a short prompt by chains of loads and, in fp32, by the matrix unit: 1021 tokens of 4 heads
// of 64, a window of 256 8.8 us a call.
#include <algorithm>

#include "paged.h"

namespace dhsa {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// Byte permutes: the low (high) halves of a and b, a below
__device__ __forceinline__ uint32_t halves_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100); }
__device__ __forceinline__ uint32_t halves_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302); }

// What the two types differ in.
template <typename T, int D, int RB> struct Tile;

template <int D, int RB> struct Tile<bf16_t, D, RB> {
    static constexpr int BK = 32, NT = D / 32, NJ = D / 16;
    typedef uint32_t vload __attribute__((ext_vector_type(D == 128 ? 4 : 2)));
    bf16x8_t qf[RB][NT];
    f32x4_t o[RB][NJ];
    struct Keys {
        bf16x8_t k[2][NT];
        vload v[8];
    };
    __device__ void load_q(int r, const char *row, int q) {
#pragma unroll
        for (int t = 0; t < NT; ++t) qf[r][t] = *reinterpret_cast<const bf16x8_t *>(row + 64 * t + 16 * q);
    }
    // Offsets (16 bytes) of the block's rows are in LDS.  ONCE: a sequence of one tile has these rows for itself, so they go past the
    // caches (64 conversations of 578K tokens, K and V 2.4 GB: 427 -> 389 us).  A longer chunk among single tokens, whose many tiles
    // all read the same rows, pays for it: 512 tokens behind 30K of them 279 us alone, 1810 more among 255 single tokens.
    template <typename V_, bool ONCE> __device__ static V_ get(const char *p) {
        if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const V_ *>(p));
        else return *reinterpret_cast<const V_ *>(p);
    }
    template <bool ONCE> __device__ static void load(Keys &x, const char *K, const char *V, const uint32_t *koff, const uint32_t *voff, int n, int q) {
        uint32_t ko[2] = {koff[n], koff[16 + n]};
        const uint4 v0 = *reinterpret_cast<const uint4 *>(voff + 4 * q), v1 = *reinterpret_cast<const uint4 *>(voff + 16 + 4 * q);
        const uint32_t vo[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < NT; ++t)
                x.k[h][t] = get<bf16x8_t, ONCE>(K + ((uint64_t)ko[h] << 4) + 64 * t + 16 * q);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x.v[i] = get<vload, ONCE>(V + ((uint64_t)vo[i] << 4) + sizeof(vload) * n);
    }
    // keys that are not there: what was loaded in their place must not meet the matrix unit (0 times NaN)
    __device__ static void clear(Keys &x, uint64_t bad, int q) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (bad >> (16 * (i >> 2) + 4 * q + (i & 3)) & 1) x.v[i] = vload(0u);
    }
    // scores of row block r: s[8 keys], key 16 (x >> 2) + 4 q + (x & 3)
    __device__ void scores(const Keys &x, int r, float *s) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < NT; ++t) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.k[h][t], qf[r][t], acc, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[4 * h + i] = acc[i];
        }
    }
    // probabilities are rounded to bf16, the type of the V that they meet in the matrix unit (as in dhsa_prefill)
    __device__ void add(const Keys &x, const float (*p)[8]) {
        bf16x8_t pf[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) pf[r][i] = (__bf16)p[r][i];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            union { uint32_t w[4]; bf16x8_t v; } vt;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                vt.w[e] = (j & 1) ? halves_hi(x.v[2 * e][j >> 1], x.v[2 * e + 1][j >> 1])
                                  : halves_lo(x.v[2 * e][j >> 1], x.v[2 * e + 1][j >> 1]);
#pragma unroll
            for (int r = 0; r < RB; ++r) o[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt.v, pf[r], o[r][j], 0, 0, 0);
        }
    }
    // column of element (j, i) of this lane's output row
    __device__ static int column(int q, int j, int i) { return (4 * q + i) * NJ + j; }
};

template <int D, int RB> struct Tile<float, D, RB> {
    static constexpr int BK = 16, NS = D / 16, NJ = D / 16;     // NJ = 4 (D / 64): output blocks (t, j)
    f32x4_t qf[RB][NS];
    f32x4_t o[RB][NJ];
    struct Keys {
        f32x4_t k[NS], v[4][D / 64];
    };
    __device__ void load_q(int r, const char *row, int q) {
#pragma unroll
        for (int s = 0; s < NS; ++s) qf[r][s] = *reinterpret_cast<const f32x4_t *>(row + 64 * s + 16 * q);
    }
    // (longer chunks have several tiles of rows here, which find one another's K and V in the caches)
    template <bool ONCE> __device__ static void load(Keys &x, const char *K, const char *V, const uint32_t *koff, const uint32_t *voff, int n, int q) {
        const uint32_t ko = koff[n];
        const uint4 v0 = *reinterpret_cast<const uint4 *>(voff + 4 * q);
        const uint32_t vo[4] = {v0.x, v0.y, v0.z, v0.w};
#pragma unroll
        for (int s = 0; s < NS; ++s) x.k[s] = *reinterpret_cast<const f32x4_t *>(K + ((uint64_t)ko << 4) + 64 * s + 16 * q);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < D / 64; ++t)
                x.v[i][t] = *reinterpret_cast<const f32x4_t *>(V + ((uint64_t)vo[i] << 4) + 256 * t + 16 * n);
    }
    __device__ static void clear(Keys &x, uint64_t bad, int q) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (bad >> (4 * q + i) & 1)
#pragma unroll
                for (int t = 0; t < D / 64; ++t) x.v[i][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    __device__ void scores(const Keys &x, int r, float *s) const {
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < NS; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.k[t][e], qf[r][t][e], acc, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = acc[i];
    }
    __device__ void add(const Keys &x, const float (*p)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < RB; ++r)
                    o[r][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[i][j >> 2][j & 3], p[r][i], o[r][j], 0, 0, 0);
    }
    __device__ static int column(int q, int j, int i) { return 64 * (j >> 2) + 4 * (4 * q + i) + (j & 3); }
};

__device__ __forceinline__ void store_out(float *p, float x) { *p = x; }
__device__ __forceinline__ void store_out(bf16_t *p, float x) {
    union { __bf16 b; uint16_t u; } c;
    c.b = (__bf16)x;
    p->bits = c.u;
}

}  // namespace

// ---------------------------------------------------------------------------
// grid: find_item's shares, from block0 on
// ---------------------------------------------------------------------------
template <typename T, int D, int RB, bool PAGED>
__global__ __launch_bounds__(256, 2) void k_span(SpanArgs a, unsigned block0) {
    using Tl = Tile<T, D, RB>;
    constexpr int M = 16 * RB, BK = Tl::BK, NP = BK / 4, NJ = Tl::NJ;
    constexpr int kPad = D + 4;
    struct Lists { alignas(16) uint32_t k[4][BK], v[4][BK]; alignas(16) float s[4][kFewRows][BK]; };
    struct Merge { float o[4][M][kPad]; float m[4][M], l[4][M]; };
    __shared__ union { Lists li; Merge me; } sm;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, q = lane >> 4;
    Item it;
    if (!find_item(a, block0 + blockIdx.x, M, 4 * BK, &it)) return;
    if (it.pieces > 1 && (unsigned)it.slot >= (unsigned)a.part_cap) return;      // (there are never so many)
    const int base = it.q.base;                              // position of the first new token
    const int p_lo = base + it.R0 / a.G, p_hi = base + (it.R0 + it.rows - 1) / a.G;
    const Span span = make_span(a, p_lo, p_hi, it.q.kv);
    const int units = (span.total + 4 * BK - 1) / (4 * BK), per = (units + it.pieces - 1) / it.pieces;
    const int x_lo = it.piece * per * 4 * BK;
    const int x_hi = x_lo + per * 4 * BK < span.total ? x_lo + per * 4 * BK : span.total;
    const char *Kg = (const char *)a.K + it.g * a.ks_h, *Vg = (const char *)a.V + it.g * a.vs_h;
    const int32_t *table = PAGED ? a.table + (int64_t)it.s * a.max_pages : nullptr;

    Tl tl;
    int pos[RB];
    float m_ref[RB], l_run[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int row = 16 * r + n < it.rows ? 16 * r + n : it.rows - 1;    // rows past the end repeat the last one (never stored)
        const int R = it.R0 + row, t = token_of(a, R), h = it.g * a.G + R - t * a.G;
        tl.load_q(r, (const char *)((const T *)a.Q + h * a.qs_h + (it.q.q0 + t) * a.qs_t), q);
        pos[r] = base + t;
        m_ref[r] = -INFINITY;
        l_run[r] = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) tl.o[r][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    uint32_t *const koff = sm.li.k[wave], *const voff = sm.li.v[wave];
    const float c = a.scale_log2e;
    // this lane's key of the block at x; keys past the end repeat the last one
    const auto slot_at = [&](int x) {
        const int xk = x + (lane & (BK - 1));
        return span.slot(xk < x_hi ? xk : x_hi - 1);
    };
    const auto ask = [&](int x) { return PAGED && x < x_hi ? table[page_of(a, slot_at(x))] : 0; };
    struct Block {
        typename Tl::Keys kv;
        unsigned long long bad;      // keys that are not there
        bool masked;                 // some row of the tile does not see some key of the block
    };
    int page = ask(x_lo + wave * BK);     // asked for a block ahead: the answer does not wait behind the block in between
    const auto fetch = [&](Block &b, int x) {
        const int slot = slot_at(x);
        bool bad = x + (lane & (BK - 1)) >= x_hi;
        uint32_t ko, vo;
        if constexpr (PAGED) {
            const int in = slot - page_of(a, slot) * a.page_size;
            if ((unsigned)page >= (unsigned)a.n_pages) { bad = true; page = 0; }
            ko = (uint32_t)page * a.ks_p + (uint32_t)in * a.ks_s;
            vo = (uint32_t)page * a.vs_p + (uint32_t)in * a.vs_s;
            page = ask(x + 4 * BK);
        } else {
            ko = (uint32_t)slot * a.ks_s;
            vo = (uint32_t)slot * a.vs_s;
        }
        if (lane < BK) { koff[lane] = ko; voff[lane] = vo; }
        // (a wave's LDS operations are executed in order: only the compiler has to keep them so)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        b.bad = __ballot(bad);
        b.masked = __any(bad || slot > p_lo || key_hi(a, slot) <= p_hi);
        Tl::template load<PAGED>(b.kv, Kg, Vg, koff, voff, n, q);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    // Scores that are kept gather in LDS, as many blocks as kFewRows allows, before they are stored: the rows of later keys come behind
    // a store that was issued before them (64 conversations, one block at a time: 515 us so, 535 when every block stored its own).
    // (There is room for whole blocks in memory, and pieces begin at multiples of 4 BK.)
    int kept = 0;
    const int keep_most = PAGED && it.scores ? kFewRows / it.rows : 0, keep_step = keep_most > 0 ? it.q.n * a.G * 32 : 0;   // floats from block of 32 keys to block
    const auto flush = [&](int x_last) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        for (int k = 0; k < kept; ++k) {
            const int x = x_last - 4 * BK * (kept - 1 - k);
            float *to = it.scores + (int64_t)(x >> 5) * keep_step + it.R0 * 32 + (x & 31);
            for (int i = lane; i < it.rows * (BK / 4); i += 64)
                *reinterpret_cast<f32x4_t *>(to + i / (BK / 4) * 32 + i % (BK / 4) * 4) =
                    *reinterpret_cast<const f32x4_t *>(&sm.li.s[wave][k * it.rows + i / (BK / 4)][i % (BK / 4) * 4]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        kept = 0;
    };
    const auto step = [&](Block &b, int x) {
        if (PAGED && b.bad) Tl::clear(b.kv, b.bad, q);
        float p[RB][NP];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            float s[NP];
            tl.scores(b.kv, r, s);
            if (b.masked) {
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const int key = 16 * (i >> 2) + 4 * q + (i & 3), j = span.slot(x + key);
                    const bool sees = j <= pos[r] && pos[r] < key_hi(a, j) && !(b.bad >> key & 1);
                    s[i] = sees ? s[i] : -INFINITY;
                }
            }
            if (keep_most > 0 && 16 * r + n < it.rows) {
#pragma unroll
                for (int h = 0; h < NP / 4; ++h)
                    *reinterpret_cast<f32x4_t *>(&sm.li.s[wave][kept * it.rows + 16 * r + n][16 * h + 4 * q]) =
                        f32x4_t{s[4 * h] * c, s[4 * h + 1] * c, s[4 * h + 2] * c, s[4 * h + 3] * c};
            }
            float mx = s[0];
#pragma unroll
            for (int i = 1; i < NP; ++i) mx = fmaxf(mx, s[i]);
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            // the reference is kept scaled and rounded: one that stays makes a factor of exactly 1
            const float m_new = fmaxf(m_ref[r], mx * c);
            const float ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m_ref[r] - ref);
            m_ref[r] = m_new;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                p[r][i] = __builtin_amdgcn_exp2f(s[i] * c - ref);
                sum += p[r][i];
            }
            l_run[r] = l_run[r] * alpha + sum;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) tl.o[r][j][i] *= alpha;
        }
        tl.add(b.kv, p);
        if (keep_most > 0 && ++kept == keep_most) flush(x);
    };
    int x = x_lo + wave * BK;
    if constexpr (RB == 1 || D == 64) {
        // the next block is on its way while this one is worked on
        Block b0, b1;
        if (x < x_hi) fetch(b0, x);
        for (; x < x_hi; x += 8 * BK) {
            if (x + 4 * BK < x_hi) fetch(b1, x + 4 * BK);
            step(b0, x);
            if (x + 4 * BK >= x_hi) break;
            if (x + 8 * BK < x_hi) fetch(b0, x + 8 * BK);
            step(b1, x + 4 * BK);
        }
    } else {
        Block b;         // (two would not fit the registers of two waves a SIMD)
        for (; x < x_hi; x += 4 * BK) {
            fetch(b, x);
            step(b, x);
        }
    }

    if (kept > 0) flush(x_lo + (wave + (x_hi - 1 - x_lo - wave * BK) / (4 * BK) * 4) * BK);      // up to this wave's last block

    // ---- join the four waves ----
    __syncthreads();                          // the lists are dead
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        float l = l_run[r] + __shfl_xor(l_run[r], 16);
        l += __shfl_xor(l, 32);
        if (q == 0) {
            sm.me.m[wave][16 * r + n] = m_ref[r];
            sm.me.l[wave][16 * r + n] = l;
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sm.me.o[wave][16 * r + n][Tl::column(q, j, i)] = tl.o[r][j][i];
    }
    __syncthreads();
    constexpr int LPR = 16;                   // lanes per row, D / 16 adjacent columns each
    constexpr int CPL = D / LPR;
    for (int row = tid / LPR; row < it.rows; row += 256 / LPR) {
        const int c0 = (tid % LPR) * CPL;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm.me.m[w][row]);
        float l = 0.f, o[CPL];
#pragma unroll
        for (int e = 0; e < CPL; ++e) o[e] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = sm.me.m[w][row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm.me.m[w][row] - mx);
            l += sm.me.l[w][row] * f;
#pragma unroll
            for (int e = 0; e < CPL; ++e) o[e] += sm.me.o[w][row][c0 + e] * f;
        }
        const int R = it.R0 + row, h = it.g * a.G + R % a.G;
        const int64_t t = it.q.q0 + R / a.G;
        if (c0 == 0 && it.piece == 0 && a.target > 0) a.cut[h * a.T + t] = make_int2(it.slot * M + row, it.pieces);
        if (it.pieces > 1) {
            float *po = a.part + ((int64_t)it.slot * M + row) * D + c0;
#pragma unroll
            for (int e = 0; e < CPL; ++e) po[e] = o[e];
            if (c0 == 0) a.state[(int64_t)it.slot * M + row] = make_float2(mx, l);
            continue;
        }
        const float inv = inv_of(l);                       // no visible key: zeros
        T *op = (T *)a.O + h * a.os_h + t * a.os_t + c0;
#pragma unroll
        for (int e = 0; e < CPL; ++e) store_out(op + e, o[e] * inv);
        if (c0 == 0) {
            if (a.lse) a.lse[h * a.T + t] = lse_of(mx, l);
            if (a.norm) a.norm[h * a.T + t] = norm_of(mx, l);
        }
    }
}

// ---------------------------------------------------------------------------
// The pieces of cut rows put together.  A workgroup looks at `per` rows at once and does the cut ones one after another: sixteen
// lanes a piece, sixteen pieces side by side and four of each in flight.  Bound by a chain of three loads: 32 rows of 128 pieces 5.6 us,
// 2048 rows of a few 7 us, rows of which none is cut 4 us (a wave a row, one piece at a time: 61 us for the first).
// ---------------------------------------------------------------------------
constexpr int kJoinRows = 4096;     // workgroups, as long as each has at most 64 rows

template <typename T, int D>
__global__ __launch_bounds__(256) void k_span_join(SpanArgs a, int per, int64_t row0) {
    constexpr int CPL = D / 16, U = 4;
    __shared__ float s_m[16], s_l[16], s_o[16][D];
    const int tid = threadIdx.x, lane = tid & 63, grp = tid >> 4, c0 = (tid & 15) * CPL;
    const int64_t rows = a.T * a.H_kv * a.G, r0 = row0 + (int64_t)blockIdx.x * per;
    const int begin = a.q_start[0], end = a.q_start[a.n_seq];      // other rows are nobody's: what lies in `cut` means nothing
    int2 cut = make_int2(0, 0);
    const int t_me = (int)((r0 + lane) % a.T);
    if (lane < per && r0 + lane < rows && t_me >= begin && t_me < end) cut = a.cut[r0 + lane];
    // (nor where the arrays are no sequences: nothing is read outside the states)
    const bool is_cut = cut.y > 1 && cut.x >= 0 && cut.x / a.M + (int64_t)(cut.y - 1) * a.H_kv < a.part_cap;
    for (unsigned long long left = __ballot(is_cut); left; left &= left - 1) {
        const int i = __builtin_ctzll(left);
        const int64_t at = __builtin_amdgcn_readlane(cut.x, i), step = (int64_t)a.H_kv * a.M;
        const int pieces = __builtin_amdgcn_readlane(cut.y, i);
        float mx = -INFINITY, l = 0.f, o[CPL];
#pragma unroll
        for (int e = 0; e < CPL; ++e) o[e] = 0.f;
        for (int x0 = grp; x0 < pieces; x0 += 16 * U) {
            float2 st[U];
            float po[U][CPL];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t x = at + step * (x0 + 16 * u < pieces ? x0 + 16 * u : x0);
                st[u] = a.state[x];
#pragma unroll
                for (int e = 0; e < CPL; ++e) po[u][e] = a.part[x * D + c0 + e];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (x0 + 16 * u >= pieces || st[u].y == 0.f) continue;      // no key there
                const float m_new = fmaxf(mx, st[u].x);
                const float f0 = __builtin_amdgcn_exp2f(mx - m_new), f1 = __builtin_amdgcn_exp2f(st[u].x - m_new);
                l = l * f0 + st[u].y * f1;
#pragma unroll
                for (int e = 0; e < CPL; ++e) o[e] = o[e] * f0 + po[u][e] * f1;
                mx = m_new;
            }
        }
        __syncthreads();                         // the row before has been read
        if (c0 == 0) { s_m[grp] = mx; s_l[grp] = l; }
#pragma unroll
        for (int e = 0; e < CPL; ++e) s_o[grp][c0 + e] = o[e];
        __syncthreads();
        if (tid < D) {
            float m = -INFINITY;
#pragma unroll
            for (int x = 0; x < 16; ++x) m = fmaxf(m, s_m[x]);
            float sum = 0.f, acc = 0.f;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const float f = s_m[x] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[x] - m);
                sum += s_l[x] * f;
                acc += s_o[x][tid] * f;
            }
            const int64_t r = r0 + i;
            const int h = (int)(r / a.T);
            const int64_t t = r - h * a.T;
            store_out((T *)a.O + h * a.os_h + t * a.os_t + tid, acc * inv_of(sum));
            if (tid == 0) {
                if (a.lse) a.lse[r] = lse_of(m, sum);
                if (a.norm) a.norm[r] = norm_of(m, sum);
            }
        }
    }
}

// Rows of a tile, us of the two sides.
// bf16, paged (K and V pass once a tile): 128 rows from 17 rows a kv-head and sequence on; of 32 rows, 16 sequences of 4096 tokens,
// 32-row tiles 64 and 128-row tiles 44; one of 32768 37 and 24; of 36 rows 88 and 45.  Up to 16 rows the few wide loads of 16-row
// tiles keep the memory busy.  The mean decides for the whole call, so a batch of single tokens and a chunk has one side's tiles for
// both: 255 tokens (2.19M cached) and a chunk of 512 behind 30K 3347, alone 1535 and 279; 63 tokens (445K) and one of 2048 behind 6144
// 670, alone 304 and 252.
// bf16, one prompt: 128 rows from 144 tiles on: 2000 tokens, 8 heads of 2 kv-heads (125 tiles), a window of 2000 36 with smaller
// tiles, 44 with 128 rows; 3500 tokens, a window of 300 26 and 17.
// Else 32 rows from 17 rows a kv-head and sequence on; one prompt, if they make 320 tiles: fp32, 4 heads of 64, a window of 256, 1021
// tokens 16 rows 9.9 and 32 rows 13.6; 4000 tokens 24.8 and 22.  fp32, paged, without that limit, groups of four: 16 sequences of 4096
// tokens, 8 kv-heads of 128, 5 new tokens 16 rows 135 and 32 rows 116, 64 tokens 812 and 622; 2 kv-heads of 64, 5 tokens 32 and 30, 16
// tokens 41 and 47 (the one of 24 such pairs that is worse than 3 %); one sequence of 32768, 5 tokens 89 and 71, 512 tokens 3129 and 2379.
void choose_tiles(SpanArgs *a, int dtype, bool paged) {
    const int64_t rows = a->T * a->G, mean = rows / std::max(a->n_seq, 1);
    a->M = mean > kFewMean && (paged || rows * a->H_kv >= 320 * 32) ? 32 : 16;
    if (dtype == DHSA_BF16 && mean > kFewMean && (paged || rows * a->H_kv >= 144 * kTallRows)) a->M = kTallRows;
    a->target = !paged ? 0 : a->M == kTallRows ? 512 : 1024;
    a->part_cap = paged ? 2 * a->target + a->H_kv : 0;
}

hipError_t launch_span(const SpanArgs &a, int D, int dtype, hipStream_t s) {
    const int M = a.M;
    const int64_t tiles = a.T * a.G / M + std::min<int64_t>(a.n_seq, a.T);
    const int64_t blocks = (tiles + (a.target + a.H_kv - 1) / a.H_kv) * a.H_kv;
    for (int64_t b0 = 0; b0 < blocks; b0 += kGridMax) {
        const dim3 grid((unsigned)std::min<int64_t>(blocks - b0, kGridMax));
#define DHSA_SPAN3(T_, D_, RB, PAGED) hipLaunchKernelGGL((k_span<T_, D_, RB, PAGED>), grid, dim3(256), 0, s, a, (unsigned)b0)
// (bf16 has no paged tiles of 32 rows)
#define DHSA_SPAN2(T_, D_, RB) \
    do { if (a.table) DHSA_SPAN3(T_, D_, (sizeof(T_) == 2 ? 1 : RB), true); else DHSA_SPAN3(T_, D_, RB, false); } while (0)
#define DHSA_SPAN1(T_, D_) do { if (M == 16) DHSA_SPAN2(T_, D_, 1); else DHSA_SPAN2(T_, D_, 2); } while (0)
        if (M == kTallRows) {
            const hipError_t e = launch_span_tall(a, D, grid.x, (unsigned)b0, s);
            if (e != hipSuccess) return e;
            continue;
        }
        if (dtype == DHSA_F32) { if (D == 64) DHSA_SPAN1(float, 64); else DHSA_SPAN1(float, 128); }
        else { if (D == 64) DHSA_SPAN1(bf16_t, 64); else DHSA_SPAN1(bf16_t, 128); }
#undef DHSA_SPAN1
#undef DHSA_SPAN2
#undef DHSA_SPAN3
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.target > 0) {
        const int64_t rows = a.T * a.H_kv * a.G;
        const int per = (int)std::min<int64_t>(64, (rows + kJoinRows - 1) / kJoinRows);
        for (int64_t r0 = 0; r0 < rows; r0 += (int64_t)kGridMax * per) {
            const dim3 grid((unsigned)std::min<int64_t>((rows - r0 + per - 1) / per, kGridMax));
#define DHSA_JOIN(T_, D_) hipLaunchKernelGGL((k_span_join<T_, D_>), grid, dim3(256), 0, s, a, per, r0)
            if (dtype == DHSA_F32) { if (D == 64) DHSA_JOIN(float, 64); else DHSA_JOIN(float, 128); }
            else { if (D == 64) DHSA_JOIN(bf16_t, 64); else DHSA_JOIN(bf16_t, 128); }
#undef DHSA_JOIN
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace dhsa
