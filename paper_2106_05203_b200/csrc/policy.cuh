// Clipped policy loss with a KL term, with the gradient of every token's log-probability.
//
//   d = lp - old, r = exp(d); pg = -min(r A, clip(r, 1 - lo, 1 + hi) A); delta = ref - lp, kl = exp(delta) - delta - 1
//   loss = sum w (pg + weight kl),  w = 1 / tokens, or 1 / (rows with tokens * tokens of the row), 0 where the mask leaves a token out
//   d loss / d lp = w (-A r [not clipped] - weight (exp(delta) - 1));  clipped: A > 0 and r > 1 + hi, or A < 0 and r < 1 - lo
//
// Two kernels over the data: the tokens are counted (the mask alone, 1 of 14 to 21 bytes), then everything else is one pass.  Which side of a border a
// ratio lies on is decided on d, in 64 bits: the gradient jumps there.
#pragma once
#include "element.cuh"
#include "preference.cuh"

namespace ef21 {

constexpr int PO_THREADS = 256;
constexpr int PO_MAX_BLOCKS = 148 * 8;

struct PolicyShape {
    i64 rows, length;
    i64 logp_stride, old_stride, ref_stride, mask_stride, adv_stride;
    int adv_per_token;
    int by_sequence;
    double log_low, log_high;                // log(1 - lo), log(1 + hi)
    float low, high;                         // 1 - lo, 1 + hi
    float kl_weight;
    double norm;                             // 0: counted
    int count_blocks;
};

// exp(x) - 1 - x >= 0, to a few units in the last place: the series about 0, where the difference would lose everything.
__device__ __forceinline__ float exp_minus_line(float x) {
    if (fabsf(x) > 1.f) return expf(x) - 1.f - x;
    float p = 1.f / 39916800.f;                                          // 1 / 11!
    p = fmaf(p, x, 1.f / 3628800.f); p = fmaf(p, x, 1.f / 362880.f); p = fmaf(p, x, 1.f / 40320.f); p = fmaf(p, x, 1.f / 5040.f);
    p = fmaf(p, x, 1.f / 720.f); p = fmaf(p, x, 1.f / 120.f); p = fmaf(p, x, 1.f / 24.f); p = fmaf(p, x, 1.f / 6.f); p = fmaf(p, x, 0.5f);
    return p * x * x;
}

// Tokens of every row, and per block how many tokens (by_sequence: rows that have any) its rows hold.
__global__ void __launch_bounds__(PO_THREADS) policy_count_kernel(const unsigned char* mask, int* tokens, i64* partial, i64 rows, i64 length, i64 stride, int by_sequence) {
    pdl_wait(mask, tokens, partial);
    pdl_trigger();
    __shared__ i64 scratch[PO_THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    i64 mine = 0;
    for (i64 r = (i64)blockIdx.x * (PO_THREADS / 32) + warp; r < rows; r += (i64)gridDim.x * (PO_THREADS / 32)) {
        const unsigned char* m = mask + r * stride;
        const int head = (int)min((i64)row_head(m), length);
        const i64 vectors = (length - head) / 16, tail = head + vectors * 16;
        int n = 0;
        if (lane < head) n += m[lane] != 0;
        for (i64 v = lane; v < vectors; v += 32) {
            const uint4 u = *reinterpret_cast<const uint4*>(m + head + v * 16);
            n += __popc(__vcmpne4(u.x, 0u) & 0x01010101u) + __popc(__vcmpne4(u.y, 0u) & 0x01010101u) + __popc(__vcmpne4(u.z, 0u) & 0x01010101u) +
                 __popc(__vcmpne4(u.w, 0u) & 0x01010101u);
        }
        if (tail + lane < length) n += m[tail + lane] != 0;
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) tokens[r] = n;
        mine += by_sequence ? (n > 0) : n;
    }
    if (lane == 0) scratch[warp] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        i64 sum = 0;
        for (int w = 0; w < PO_THREADS / 32; ++w) sum += scratch[w];
        partial[blockIdx.x] = sum;
    }
}

struct PolicySums { double pg = 0.0, kl = 0.0, clipped = 0.0; };

// One token of weight w; adds its terms and returns its gradient.
__device__ __forceinline__ float policy_token(float lp, float old, float ref, bool has_ref, float A, float w, const PolicyShape& s, float& pg, float& kl, float& clip) {
    const double d = (double)lp - (double)old;
    const bool clipped = (A > 0.f && d > s.log_high) || (A < 0.f && d < s.log_low);
    const float r = clipped ? (A > 0.f ? s.high : s.low) : (A == 0.f ? 0.f : expf(lp - old));
    float g = clipped ? 0.f : -A * r;
    pg -= w * (r * A);
    clip += clipped ? w : 0.f;
    if (has_ref) {
        const float delta = ref - lp, k = exp_minus_line(delta);
        kl += w * k;
        g -= s.kl_weight * (k + delta);
    }
    return w * g;
}

// FLAT: all arrays are contiguous, a vector of VEC tokens may run over the end of a row.  Otherwise token by token, any strides.
template <typename T, bool FLAT>
__global__ void __launch_bounds__(PO_THREADS) policy_kernel(const T* logps, const T* old, const T* ref, const T* adv, const unsigned char* mask, const int* tokens, const i64* counted,
                                                            T* grad, PolicySums* partial, PolicyShape s) {
    pdl_wait(logps, old, ref, adv, mask, tokens, counted, grad, partial);
    pdl_trigger();
    constexpr int VEC = FLAT ? Elem<T>::VEC : 1;
    typedef typename MaskWord<Elem<T>::VEC>::type Word;
    __shared__ double scratch[PO_THREADS / 32];
    const int tid = threadIdx.x;
    double norm = s.norm;
    if (norm == 0.0) {
        if (counted) {
            double n = 0.0;
            for (int b = tid; b < s.count_blocks; b += PO_THREADS) n += (double)counted[b];
            norm = block_sum<PO_THREADS>(n, scratch);
        } else {
            norm = s.by_sequence ? (s.length > 0 ? (double)s.rows : 0.0) : (double)s.rows * (double)s.length;
        }
    }
    const float inverse = norm > 0.0 ? (float)(1.0 / norm) : 0.f;
    auto weight = [&](i64 row) {
        if (!s.by_sequence) return inverse;
        const i64 n = tokens ? (i64)tokens[row] : s.length;
        return n > 0 ? inverse / (float)n : 0.f;
    };
    PolicySums sums;
    const i64 all = s.rows * s.length, vectors = all / VEC, step = (i64)gridDim.x * PO_THREADS;
    auto token = [&](i64 i) {                                       // one token, any strides
        const i64 row = i / s.length, t = i - row * s.length;
        T* g = grad + i;
        if (mask && !mask[row * s.mask_stride + t]) { *g = Elem<T>::put(0.f); return; }
        float pg = 0.f, kl = 0.f, clip = 0.f;
        const float A = Elem<T>::get(adv[row * s.adv_stride + (s.adv_per_token ? t : 0)]);
        const float v = policy_token(Elem<T>::get(logps[row * s.logp_stride + t]), Elem<T>::get(old[row * s.old_stride + t]),
                                     ref ? Elem<T>::get(ref[row * s.ref_stride + t]) : 0.f, ref != nullptr, A, weight(row), s, pg, kl, clip);
        *g = Elem<T>::put(v);
        sums.pg += (double)pg; sums.kl += (double)kl; sums.clipped += (double)clip;
    };
    for (i64 v = (i64)blockIdx.x * PO_THREADS + tid; v < vectors; v += step) {
        const i64 i = v * VEC;
        if (!FLAT) { token(i); continue; }
        const Word w = mask ? *reinterpret_cast<const Word*>(mask + i) : ~(Word)0;
        if (w == 0) { store_vec(grad + i, make_uint4(0u, 0u, 0u, 0u)); continue; }
        float x[Elem<T>::VEC], o[Elem<T>::VEC], f[Elem<T>::VEC], A[Elem<T>::VEC], g[Elem<T>::VEC];
        const uint4 ux = load_once(logps + i), uo = load_once(old + i), uf = ref ? load_once(ref + i) : make_uint4(0u, 0u, 0u, 0u);
        const uint4 ua = s.adv_per_token ? load_once(adv + i) : make_uint4(0u, 0u, 0u, 0u);
        i64 row = i / s.length, left = s.length - (i - row * s.length);          // tokens of the row from here on
        Elem<T>::unpack(ux, x); Elem<T>::unpack(uo, o); Elem<T>::unpack(uf, f); Elem<T>::unpack(ua, A);
        float rowA = s.adv_per_token ? 0.f : Elem<T>::get(adv[row * s.adv_stride]), rowW = weight(row);
        float pg = 0.f, kl = 0.f, clip = 0.f;
#pragma unroll
        for (int e = 0; e < Elem<T>::VEC; ++e) {
            if (left == 0) {
                ++row; left = s.length;
                if (!s.adv_per_token) rowA = Elem<T>::get(adv[row * s.adv_stride]);
                rowW = weight(row);
            }
            --left;
            g[e] = (w >> (8 * e) & 255u) != 0 ? policy_token(x[e], o[e], f[e], ref != nullptr, s.adv_per_token ? A[e] : rowA, rowW, s, pg, kl, clip) : 0.f;
        }
        store_vec(grad + i, Elem<T>::pack(g));
        sums.pg += (double)pg; sums.kl += (double)kl; sums.clipped += (double)clip;
    }
    if (FLAT && blockIdx.x == 0 && vectors * VEC + tid < all) token(vectors * VEC + tid);
    sums.pg = block_sum<PO_THREADS>(sums.pg, scratch);
    sums.kl = block_sum<PO_THREADS>(sums.kl, scratch);
    sums.clipped = block_sum<PO_THREADS>(sums.clipped, scratch);
    if (tid == 0) partial[blockIdx.x] = sums;
}

__global__ void __launch_bounds__(PO_THREADS) policy_finish_kernel(const PolicySums* partial, float* terms, int blocks, double kl_weight) {
    pdl_wait(partial, terms);
    pdl_trigger();
    __shared__ double scratch[PO_THREADS / 32];
    PolicySums v;
    for (int b = threadIdx.x; b < blocks; b += PO_THREADS) { v.pg += partial[b].pg; v.kl += partial[b].kl; v.clipped += partial[b].clipped; }
    v.pg = block_sum<PO_THREADS>(v.pg, scratch);
    v.kl = block_sum<PO_THREADS>(v.kl, scratch);
    v.clipped = block_sum<PO_THREADS>(v.clipped, scratch);
    if (threadIdx.x == 0) {
        terms[0] = (float)(kl_weight == 0.0 ? v.pg : v.pg + kl_weight * v.kl);
        terms[1] = (float)v.pg; terms[2] = (float)v.kl; terms[3] = (float)v.clipped;
    }
}

}  // namespace ef21
