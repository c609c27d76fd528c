// What each cached key has got of attention (dhsa_paged_attend with weights): the scores are made again from Q and K, and with
// the exponent reference and the sum of each row, which attention has left, every probability is known at once.
//
// Work unit: 64 keys of a kv-head and sequence.  They stay in the registers that the matrix unit reads; the rows that see
// them pass by, every fourth block of 16 to each of the four waves.  S^T (keys x rows) = K Q^T: a lane adds up the
// probabilities of its 16 keys over its rows, the 16 lanes of other rows and the four waves follow once at the end, so the
// order of a sum is fixed and nothing is added with atomics.
#include <algorithm>

#include "paged.h"

namespace dhsa {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// 16 bytes of a row as the matrix unit takes them: element e of step t is column 32 t + 8 q + e (bf16) or 16 t + 4 q + e (fp32)
template <typename T> struct Frag;
template <> struct Frag<bf16_t> {
    typedef bf16x8_t type;
    __device__ static f32x4_t mfma(const type &k, const type &x, f32x4_t acc) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, x, acc, 0, 0, 0);
    }
};
template <> struct Frag<float> {
    typedef f32x4_t type;
    __device__ static f32x4_t mfma(const type &k, const type &x, f32x4_t acc) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], x[e], acc, 0, 0, 0);
        return acc;
    }
};

}  // namespace

constexpr int kWKeys = 64;

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void k_weights(SpanArgs a, float *__restrict__ W, float decay) {
    typedef typename Frag<T>::type F;
    constexpr int NT = D * (int)sizeof(T) / 64;
    __shared__ float s_sum[4][kWKeys];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, q = lane >> 4;
    const float c = a.scale_log2e;
    for (unsigned b = blockIdx.x;; b += gridDim.x) {
        // the item: as find_item, of key tiles
        const int g = (int)(b % (unsigned)a.H_kv);
        int want = (int)(b / (unsigned)a.H_kv), s = -1, tile = 0;
        for (int s0 = 0, base = 0; s0 < a.n_seq; s0 += 64) {
            int tiles = 0;
            if (s0 + lane < a.n_seq) tiles = (read_seq(a, s0 + lane).kv + kWKeys - 1) / kWKeys;
            const int end = wave_incl_scan(tiles), total = __builtin_amdgcn_readlane(end, 63);
            if (want < base + total) {
                const int l = __builtin_ctzll(__ballot(want < base + end));
                s = s0 + l;
                tile = want - base - __builtin_amdgcn_readlane(end - tiles, l);
                break;
            }
            base += total;
        }
        if (s < 0) return;
        const Seq sq = read_seq(a, s);
        const int j0 = tile * kWKeys, base = sq.kv - sq.n;
        const int keys = sq.kv - j0 < kWKeys ? sq.kv - j0 : kWKeys;
        const int32_t *table = a.table + (int64_t)s * a.max_pages;
        const char *Kg = (const char *)a.K + g * a.ks_h;
        F kf[4][NT];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int key = 16 * h + n < keys ? 16 * h + n : keys - 1, slot = j0 + key;
            const int pi = page_of(a, slot);
            int page = table[pi];
            if ((unsigned)page >= (unsigned)a.n_pages) page = 0;
            const char *row = Kg + ((uint64_t)((uint32_t)page * a.ks_p + (uint32_t)(slot - pi * a.page_size) * a.ks_s) << 4);
#pragma unroll
            for (int t = 0; t < NT; ++t) kf[h][t] = *reinterpret_cast<const F *>(row + 64 * t + 16 * q);
        }
        f32x4_t sum[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) sum[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        // the new tokens that may see one of the keys
        const int t_lo = j0 > base ? j0 - base : 0;
        const int far = key_hi(a, j0 + keys - 1);       // no position from here on sees the last key, unless it is ...
        const int t_hi = j0 < a.sinks || far >= sq.kv ? sq.n : far - base;      // ... behind one that stays visible
        const int64_t R1 = t_hi > t_lo ? (int64_t)t_hi * a.G : 0;
        for (int64_t R0 = (int64_t)t_lo * a.G + 16 * wave; R0 < R1; R0 += 64) {
            const int R = (int)(R0 + n < R1 ? R0 + n : R1 - 1), t = R / a.G, h0 = g * a.G + R % a.G;
            const bool live = R0 + n < R1;
            const char *row = (const char *)((const T *)a.Q + h0 * a.qs_h + (sq.q0 + t) * a.qs_t);
            F qf[NT];
#pragma unroll
            for (int u = 0; u < NT; ++u) qf[u] = *reinterpret_cast<const F *>(row + 64 * u + 16 * q);
            const float2 nm = a.norm[h0 * a.T + sq.q0 + t];
            const int p = live ? base + t : -1;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int u = 0; u < NT; ++u) x = Frag<T>::mfma(kf[h][u], qf[u], x);
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
                if (n == 0) s_sum[wave][16 * h + 4 * q + i] = x;
            }
        __syncthreads();
        if (tid < keys) {
            const int slot = j0 + tid, pi = page_of(a, slot), page = table[pi];
            if ((unsigned)page < (unsigned)a.n_pages) {
                float *w = W + ((int64_t)page * a.H_kv + g) * a.page_size + (slot - pi * a.page_size);
                const float x = (s_sum[0][tid] + s_sum[1][tid]) + (s_sum[2][tid] + s_sum[3][tid]);
                *w = decay > 0.f ? decay * *w + x : x;
            }
        }
    }
}

hipError_t launch_weights(const SpanArgs &a, int D, int dtype, float *W, float decay, hipStream_t s) {
    const dim3 grid(1024);
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
