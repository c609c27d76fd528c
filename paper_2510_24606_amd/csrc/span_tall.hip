// bf16 attention without routing for many rows: tiles of 128 rows of a kv-head and sequence (row R = token R / G, query head
// g G + R % G) over a piece of the keys that they see (see paged.h, span.hip).
//
// Four waves, each with one block of 32 rows; K and V in tiles of 64 keys that all four read from LDS, so a row of K or V that
// was fetched once serves 128 rows.  S^T = K Q^T (v_mfma_f32_32x32x16_bf16, keys are the M dimension), so a lane has 16 keys of
// ONE row per 32-key block: sums stay in the lane, and the exponentials lie as the B operand of O^T += V^T P^T wants them.
// V^T is read with the transposing LDS read (ds_read_b64_tr_b16).
//
// K and V rows go from memory straight into LDS (global_load_lds_dwordx4, 16 bytes a lane), unpadded; bank conflicts are
// avoided by an XOR swizzle of the 16-byte pieces of a row, made by which piece a lane fetches.  Where a row lies (page, slot)
// is worked out once per key, by one wave for a whole tile, four tiles ahead, from page numbers that were requested four
// tiles before that; the addresses pass through LDS.
//
// Tile n: scores of the next block of 32 keys on the matrix unit while the vector unit takes exponentials of the present one,
// then O += P V; the loads of the upper half of K(n + 1), of V(n + 1) and of the lower half of K(n + 2) are spread in
// between; one barrier a tile.  O / l is exact whatever the exponents' reference is, so a row's reference is its maximum over
// its first block with a key and moves only when a block's sum passes 2^20.
//
// Bound by the matrix and vector units and how well they overlap, at two waves a SIMD (LDS and registers allow no third): a window of 8192
// over 128K tokens 15.6 ms, 1.10 PFLOP/s; of 2048 over 32K tokens 1.09 ms (a fifth of a workgroup's time is its beginning and end): matrix
// unit busy 48 % of the cycles, vector unit 44 %, waves waiting 28 %, at 2.0 GHz.  2048 new tokens behind 30K of a paged cache 1.02 ms.
#include <type_traits>

#include "attn_mfma.h"
#include "paged.h"

namespace dhsa {

namespace {

constexpr int kTallKeys = 64;

template <int D, typename Addr>
struct TallSmem {
    static constexpr int kTile = kTallKeys * D;
    alignas(1024) uint16_t K[2 * kTile];
    alignas(1024) uint16_t V[2 * kTile];
    // of the keys of eight tiles: addresses of the rows (contiguous K and V: offsets, a head spans at most 4 GiB; 16.36 -> 15.99 ms for
    // a window of 8192 over 128K tokens), in the order the loading lanes want them; a row at position p takes
    // the key iff lo < p < hi
    alignas(16) Addr kaddr[8][kTallKeys], vaddr[8][kTallKeys];
    alignas(16) int lo[8][kTallKeys], hi[8][kTallKeys];
    int flags[8];        // does some row of the tile not take some key of it?
};

__device__ const uint4 zero_row[16] = {};     // what a key without a page has for K and V

__device__ __forceinline__ void load16_to_lds(uint64_t addr, const char *, unsigned lds_window) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(addr), "s"(lds_window) : "memory");
#else
    (void)addr; (void)lds_window;
#endif
}

__device__ __forceinline__ void load16_to_lds(uint32_t offset, const char *base, unsigned lds_window) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" ::"v"(offset), "s"(lds_window), "s"(base) : "memory");
#else
    (void)offset; (void)base; (void)lds_window;
#endif
}

}  // namespace

template <int D, bool PAGED>
__global__ __launch_bounds__(256, 2) void k_span_tall(SpanArgs a, unsigned block0) {
    using Addr = std::conditional_t<PAGED, uint64_t, uint32_t>;
    using Smem = TallSmem<D, Addr>;
    constexpr int OPR = D / 8;          // 16-byte pieces per row
    constexpr int KPT = OPR / 4;        // load instructions per wave and tile (K and V each)
    constexpr int NS = D / 16;          // matrix steps of K Q^T
    constexpr int NDB = D / 32;         // blocks of 32 output columns
    constexpr int kTile = Smem::kTile;
    __shared__ Smem sm;
    Item it;
    if (!find_item(a, block0 + blockIdx.x, kTallRows, kTallKeys, &it)) return;
    if (it.pieces > 1 && (unsigned)it.slot >= (unsigned)a.part_cap) return;      // (there are never so many)
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 31, g2 = lane >> 5;
    const int base = it.q.base;                              // position of the first new token
    const int p_lo = base + it.R0 / a.G, p_hi = base + (it.R0 + it.rows - 1) / a.G;
    const Span span = make_span(a, p_lo, p_hi, it.q.kv);
    const int units = (span.total + kTallKeys - 1) / kTallKeys, per = (units + it.pieces - 1) / it.pieces;
    const int x_lo = it.piece * per * kTallKeys;
    const int x_hi = x_lo + per * kTallKeys < span.total ? x_lo + per * kTallKeys : span.total;
    const int ntiles = x_hi > x_lo ? (x_hi - x_lo + kTallKeys - 1) / kTallKeys : 0;
    const char *Kg = (const char *)a.K + it.g * a.ks_h, *Vg = (const char *)a.V + it.g * a.vs_h;
    const int32_t *table = PAGED ? a.table + (int64_t)it.s * a.max_pages : nullptr;
    const float c = a.scale_log2e;

    // this wave's rows (which wave has which block goes round with the workgroup, so that waves without rows do not always sit
    // on the same SIMD); a row that is not there has q = 0 and a reference that makes every p 0
    const int rb = (wave + (blockIdx.x >> 3)) & 3;
    const bool live = rb * 32 < it.rows, pad_row = rb * 32 + lr >= it.rows;
    const int R = it.R0 + (pad_row ? it.rows - 1 : rb * 32 + lr), tok = token_of(a, R), h = it.g * a.G + R - tok * a.G;
    const int pos = base + tok;
    bf16x8 qf[NS];
    {
        const uint16_t *qp = (const uint16_t *)a.Q + h * a.qs_h + (it.q.q0 + tok) * a.qs_t + 8 * g2;
#pragma unroll
        for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const bf16x8 *>(qp + 16 * s);
    }
    f32x16 oacc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) oacc[db][x] = 0.f;
    float m_ref = pad_row ? 1e30f : __builtin_nanf(""), l_run = 0.f;     // NaN: no key yet

    // staging: load i of a wave fills the KiB 4 i + wave of a tile; this lane's piece there belongs to row ld_row0 + 4 i RPW
    constexpr int RPW = 64 / OPR, RSTR = 4 * RPW;
    const int ld_row0 = wave * RPW + lane / OPR;
    const unsigned ld_piece = 16u * ((lane % OPR) ^ piece_swizzle(ld_row0, OPR));
    const int slot_wr = (lane % RSTR) * KPT + lane / RSTR, slot_rd = ld_row0 * KPT;
    const unsigned lds_K = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint16_t *)sm.K;
    const unsigned lds_V = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint16_t *)sm.V;
    // operands (byte offsets): K row lr of a block, piece 2 s + g2; V^T by transposing reads of row 8 half + 4 g2 + cc of 16
    const int k_sw = piece_swizzle(lr, OPR);
    int k_off[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) k_off[s] = 2 * (lr * D + 8 * ((2 * s + g2) ^ k_sw));
    const int tr_c = (lane & 15) >> 2, tr_r = lane & 3, tr_dh = (lane >> 4) & 1;
    const int tr_low2 = ((tr_r >> 1) ^ g2) | ((tr_dh ^ (tr_c & 1)) << 1);
    const int tr_l0 = (4 * g2 + tr_c) * D + 8 * tr_low2 + 4 * (tr_r & 1);
    int v_base_e = 2 * (tr_l0 + 32 * (tr_c >> 1)), v_base_o = 2 * (tr_l0 - 32 * (tr_c >> 1));
    const char *const smK8 = reinterpret_cast<const char *>(sm.K);
    const char *const smV8 = reinterpret_cast<const char *>(sm.V);

    const auto slot_of = [&](int n) {
        const int x = x_lo + n * kTallKeys + lane;
        return span.slot(x < x_hi ? x : x_hi - 1);
    };
    const auto page_ask = [&](int n) { return PAGED && n < ntiles ? table[page_of(a, slot_of(n))] : 0; };
    // one wave: addresses and limits of the keys of tile n, whose page numbers are there
    const auto make_list = [&](int n, int page) {
        const int j = slot_of(n), in = PAGED ? j - page_of(a, j) * a.page_size : j;
        const bool none = PAGED && (unsigned)page >= (unsigned)a.n_pages;
        const uint32_t ko = (PAGED ? (uint32_t)page * a.ks_p : 0u) + (uint32_t)in * a.ks_s;
        const uint32_t vo = (PAGED ? (uint32_t)page * a.vs_p : 0u) + (uint32_t)in * a.vs_s;
        if constexpr (PAGED) {
            const uint64_t zero = (uint64_t)(uintptr_t)zero_row;
            sm.kaddr[n & 7][slot_wr] = none ? zero : (uint64_t)(uintptr_t)Kg + ((uint64_t)ko << 4);
            sm.vaddr[n & 7][slot_wr] = none ? zero : (uint64_t)(uintptr_t)Vg + ((uint64_t)vo << 4);
        } else {
            sm.kaddr[n & 7][slot_wr] = ko << 4;
            sm.vaddr[n & 7][slot_wr] = vo << 4;
        }
        const bool out = none || x_lo + n * kTallKeys + lane >= x_hi;
        const int lo = out ? kIntMaxP : j - 1, hi = key_hi(a, j);
        sm.lo[n & 7][lane] = lo;
        sm.hi[n & 7][lane] = hi;
        const bool any = __any(lo >= p_lo || hi <= p_hi);
        if (lane == 0) sm.flags[n & 7] = any;
    };
#define TALL_ADDRS(dst, tab, n, c0, c1) \
    _Pragma("unroll") for (int i = c0; i < c1; ++i) dst[i] = sm.tab[(n) & 7][slot_rd + i];
#define TALL_LOAD(X, addrs, n, c0, c1) \
    _Pragma("unroll") for (int i = c0; i < c1; ++i) \
        load16_to_lds((Addr)(addrs[i] + ld_piece), X##g, lds_##X + (((n) & 1) * kTile + wave * 512) * 2 + i * 4096);
// S^T of the 32-key block whose K rows start at element kb of the buffer that k_off points into
#define TALL_QK(kb, s_) \
    { \
        _Pragma("unroll") for (int x = 0; x < 16; ++x) s_[x] = 0.f; \
        _Pragma("unroll") for (int s = 0; s < NS; ++s) \
            s_ = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(smK8 + k_off[s] + 2 * (kb)), qf[s], s_, 0, 0, 0); \
    }
#define TALL_MASK(n, kb, s_, flag) \
    if (flag) { \
        _Pragma("unroll") for (int q4 = 0; q4 < 4; ++q4) { \
            const int key_ = (kb) * 32 + q4 * 8 + g2 * 4; \
            const int4 lo_ = *reinterpret_cast<const int4 *>(&sm.lo[(n) & 7][key_]); \
            const int4 hi_ = *reinterpret_cast<const int4 *>(&sm.hi[(n) & 7][key_]); \
            s_[q4 * 4 + 0] = ((pos > lo_.x) & (pos < hi_.x)) ? s_[q4 * 4 + 0] : -INFINITY; \
            s_[q4 * 4 + 1] = ((pos > lo_.y) & (pos < hi_.y)) ? s_[q4 * 4 + 1] : -INFINITY; \
            s_[q4 * 4 + 2] = ((pos > lo_.z) & (pos < hi_.z)) ? s_[q4 * 4 + 2] : -INFINITY; \
            s_[q4 * 4 + 3] = ((pos > lo_.w) & (pos < hi_.w)) ? s_[q4 * 4 + 3] : -INFINITY; \
        } \
    }
// maximum of a row over a block (two lanes have a row)
#define TALL_MAX(s_, mx) \
    { \
        float m_ = s_[0]; \
        _Pragma("unroll") for (int x = 1; x < 16; ++x) m_ = fmaxf(m_, s_[x]); \
        mx = fmaxf(m_, __shfl_xor(m_, 32)); \
    }
// P = exp2(S c - m_ref c), rounded to the two bf16 operands of the block (V is bf16, and so is what it meets); the sums are of
// what was not rounded yet
#define TALL_EXP(s_, pf) \
    { \
        const float mc_ = m_ref * c; \
        float sum_ = 0.f; \
        _Pragma("unroll") for (int x = 0; x < 16; ++x) { \
            const float e_ = __builtin_amdgcn_exp2f(s_[x] * c - mc_); \
            sum_ += e_; \
            pf[x >> 3][x & 7] = (__bf16)e_; \
        } \
        if (__any(!(sum_ < 1048576.f))) {      /* too large, or no reference yet (then nothing has been added up) */ \
            float mx_; \
            TALL_MAX(s_, mx_); \
            const float m_new_ = fmaxf(m_ref, mx_);        /* the other one if one is NaN */ \
            const bool none_ = m_new_ == -INFINITY; \
            const float alpha_ = m_ref != m_ref ? 0.f : __builtin_amdgcn_exp2f((m_ref - m_new_) * c); \
            l_run *= alpha_; \
            _Pragma("unroll") for (int db = 0; db < NDB; ++db) \
                _Pragma("unroll") for (int x = 0; x < 16; ++x) oacc[db][x] *= alpha_; \
            const float ref_ = none_ ? 0.f : m_new_ * c; \
            m_ref = none_ ? __builtin_nanf("") : m_new_; \
            sum_ = 0.f; \
            _Pragma("unroll") for (int x = 0; x < 16; ++x) { \
                const float e_ = __builtin_amdgcn_exp2f(s_[x] * c - ref_); \
                sum_ += e_; \
                pf[x >> 3][x & 7] = (__bf16)e_; \
            } \
        } \
        l_run += sum_; \
    }
// O^T += V^T P^T of the 32-key block kb of the buffer that v_base_* point into.  The physical piece of a row's column block
// differs from the logical one by the row's swizzle: two bases a lane, the rest is an immediate.
#define TALL_PV(kb, pf) \
    { \
        _Pragma("unroll") for (int kk = 0; kk < 2; ++kk) \
            _Pragma("unroll") for (int db = 0; db < NDB; ++db) { \
                union { s16x4 h[2]; bf16x8 v; } vf_; \
                _Pragma("unroll") for (int half = 0; half < 2; ++half) { \
                    const int x2_ = (OPR == 16) ? (db ^ (2 * half)) : db; \
                    const char *vp_ = smV8 + ((x2_ & 1) ? v_base_o : v_base_e) + 2 * (((kb) * 32 + 16 * kk + 8 * half) * D + 32 * x2_); \
                    vf_.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)vp_); \
                } \
                oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf_.v, pf[kk], oacc[db], 0, 0, 0); \
            } \
    }

    if (ntiles > 0) {
        f32x16 s_a, s_b;                      // scores of two consecutive blocks
        int toggle = 2 * kTile;
        Addr ka[KPT], va[KPT];                // addresses of the loads this lane issues next (lower half of K: of the tile after)
        int page = page_ask(4 + wave);
        if (wave < ntiles) make_list(wave, page_ask(wave));
        __syncthreads();
        TALL_ADDRS(ka, kaddr, 0, 0, KPT);
        TALL_ADDRS(va, vaddr, 0, 0, KPT);
        TALL_LOAD(K, ka, 0, 0, KPT);
        TALL_LOAD(V, va, 0, 0, KPT);
        if (ntiles > 1) {
            TALL_ADDRS(ka, kaddr, 1, 0, KPT / 2);
            TALL_LOAD(K, ka, 1, 0, KPT / 2);
        }
        int fl_cur = __builtin_amdgcn_readfirstlane(sm.flags[0]);
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): this wave's pieces are in LDS
        __syncthreads();
        if (live) {
            if (pad_row) {
#pragma unroll
                for (int s = 0; s < NS; ++s) qf[s] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
            }
            TALL_QK(0, s_a);
            TALL_MASK(0, 0, s_a, fl_cur);
            float mx0;
            TALL_MAX(s_a, mx0);
            if (mx0 != -INFINITY) m_ref = fmaxf(m_ref, mx0);
        }
        __syncthreads();                      // the lower half of K(0) may be overwritten from here on
        int n = 0;
        for (; n + 1 < ntiles; ++n) {
            if ((n & 3) == 0) {
                if (n + 4 + wave < ntiles) make_list(n + 4 + wave, page);
                page = page_ask(n + 8 + wave);
            }
            TALL_ADDRS(ka, kaddr, n + 1, KPT / 2, KPT);
            TALL_ADDRS(va, vaddr, n + 1, 0, KPT);
            TALL_ADDRS(ka, kaddr, n + 2, 0, KPT / 2);
            const int fl_next = __builtin_amdgcn_readfirstlane(sm.flags[(n + 1) & 7]);
            if (live) {
                bf16x8 pf[2];
                TALL_LOAD(K, ka, n + 1, KPT / 2, KPT);
                TALL_QK(32 * D, s_b);                      // block 1 of tile n
                TALL_EXP(s_a, pf);
                TALL_LOAD(V, va, n + 1, 0, KPT / 2);
                TALL_PV(0, pf);
                TALL_MASK(n, 1, s_b, fl_cur);
#pragma unroll
                for (int s = 0; s < NS; ++s) k_off[s] += toggle;   // now the K buffer of tile n + 1
                TALL_LOAD(V, va, n + 1, KPT / 2, KPT);
                TALL_QK(0, s_a);                           // block 0 of tile n + 1
                TALL_EXP(s_b, pf);
                if (n + 2 < ntiles) TALL_LOAD(K, ka, n + 2, 0, KPT / 2);
                TALL_PV(1, pf);
                TALL_MASK(n + 1, 0, s_a, fl_next);
                v_base_e += toggle;                        // now the V buffer of tile n + 1
                v_base_o += toggle;
                toggle = -toggle;
            } else {
                TALL_LOAD(K, ka, n + 1, KPT / 2, KPT);
                TALL_LOAD(V, va, n + 1, 0, KPT);
                if (n + 2 < ntiles) TALL_LOAD(K, ka, n + 2, 0, KPT / 2);
            }
            fl_cur = fl_next;
            __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): the pieces this wave requested have landed
            __syncthreads();
        }
        if (live) {
            bf16x8 pf[2];
            TALL_QK(32 * D, s_b);
            TALL_EXP(s_a, pf);
            TALL_PV(0, pf);
            TALL_MASK(n, 1, s_b, fl_cur);
            TALL_EXP(s_b, pf);
            TALL_PV(1, pf);
        }
    }
#undef TALL_ADDRS
#undef TALL_LOAD
#undef TALL_QK
#undef TALL_MASK
#undef TALL_MAX
#undef TALL_EXP
#undef TALL_PV

    // lane: row lr of the block, columns 32 db + 8 q4 + 4 g2 + {0..3}
    if (!live) return;
    const float l = l_run + __shfl_xor(l_run, 32), mx = m_ref != m_ref ? -INFINITY : m_ref * c;
    if (pad_row) return;
    const int64_t t = it.q.q0 + tok;
    if (g2 == 0 && it.piece == 0 && a.target > 0) a.cut[h * a.T + t] = make_int2(it.slot * kTallRows + rb * 32 + lr, it.pieces);
    if (it.pieces > 1) {
        const int64_t at = (int64_t)it.slot * kTallRows + rb * 32 + lr;
        float *po = a.part + at * D;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<float4 *>(po + db * 32 + q4 * 8 + g2 * 4) =
                    make_float4(oacc[db][4 * q4], oacc[db][4 * q4 + 1], oacc[db][4 * q4 + 2], oacc[db][4 * q4 + 3]);
        if (g2 == 0) a.state[at] = make_float2(mx, l);
        return;
    }
    const float inv = inv_of(l);                 // no visible key: zeros
    uint16_t *op = (uint16_t *)a.O + h * a.os_h + t * a.os_t;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            union { __bf16 b[4]; uint2 u; } pk;
#pragma unroll
            for (int x = 0; x < 4; ++x) pk.b[x] = (__bf16)(oacc[db][q4 * 4 + x] * inv);
            *reinterpret_cast<uint2 *>(op + db * 32 + q4 * 8 + g2 * 4) = pk.u;
        }
    if (g2 == 0) {
        if (a.lse) a.lse[h * a.T + t] = lse_of(mx, l);
        if (a.norm) a.norm[h * a.T + t] = norm_of(mx, l);
    }
}

hipError_t launch_span_tall(const SpanArgs &a, int D, unsigned blocks, unsigned block0, hipStream_t s) {
    if (D == 64) {
        if (a.table) hipLaunchKernelGGL((k_span_tall<64, true>), dim3(blocks), dim3(256), 0, s, a, block0);
        else hipLaunchKernelGGL((k_span_tall<64, false>), dim3(blocks), dim3(256), 0, s, a, block0);
    } else {
        if (a.table) hipLaunchKernelGGL((k_span_tall<128, true>), dim3(blocks), dim3(256), 0, s, a, block0);
        else hipLaunchKernelGGL((k_span_tall<128, false>), dim3(blocks), dim3(256), 0, s, a, block0);
    }
    return hipGetLastError();
}

}  // namespace dhsa
