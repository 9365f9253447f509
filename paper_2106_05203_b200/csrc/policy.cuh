// Clipped policy loss with a KL term, with the gradient of every token's log-probability.
//
//   d = lp - old, r = exp(d); pg = -min(r A, clip(r, 1 - lo, 1 + hi) A); delta = ref - lp, kl = exp(delta) - delta - 1
//   loss = sum w (pg + weight kl),  w = 1 / tokens, or 1 / (rows with tokens * tokens of the row), 0 where the mask leaves a token out
//   d loss / d lp = w (-A r [not clipped] - weight (exp(delta) - 1));  clipped: A > 0 and r > 1 + hi, or A < 0 and r < 1 - lo
//
// The tokens are counted first (the mask alone, 1 of 14 to 21 bytes), then everything else is one pass, and a third kernel adds up the blocks' terms.
// Few tokens: one cluster does it all, every block counting for itself.  Which side of a border a ratio lies on is decided on d, in 64 bits where 32
// could err: the gradient jumps there.
//
// 1,024 x 8,192 fp32, 45 % of it masked, by sequence: 45 us, the pass at 0.58 of the issue slots (some 60 instructions a token), count and sum some 7 of it; 8 x 300: 7.0 us, a launch.
#pragma once
#include "cluster.cuh"
#include "element.cuh"
#include "preference.cuh"

namespace ef21 {

constexpr int PO_THREADS = 128;              // small blocks: where a mask leaves runs of tokens out, blocks differ in their work
constexpr int PO_VECTORS = 8;                // per thread, more where there would be more than PO_MAX_BLOCKS blocks
constexpr int PO_MAX_BLOCKS = 8192;
constexpr int PO_COUNT_THREADS = 256, PO_COUNT_BLOCKS = 128;
constexpr int PO_FINISH_THREADS = 1024;
constexpr i64 PO_ONE_TOKENS = 16384;         // up to here (and PO_ONE_ROWS rows): one cluster of up to eight blocks
constexpr int PO_ONE_ROWS = 1024;
constexpr unsigned PO_CLUSTER = 8;

struct PolicyShape {
    i64 rows, length;
    i64 logp_stride, old_stride, ref_stride, mask_stride, adv_stride;
    int adv_per_token;
    int by_sequence;
    double log_low, log_high;                // log(1 - lo), log(1 + hi)
    float near;                              // how close to these a difference in 32 bits says nothing
    float low, high;                         // 1 - lo, 1 + hi
    float kl_weight;
    double norm;                             // 0: counted
    int count_blocks;
    i64 per_block;                           // vectors (flat) or tokens of a block
    int one;                                 // all blocks are one cluster: they count, and write the terms
};

// exp(x) - 1 - x >= 0, to a few units in the last place, for |x| <= 1: the series about 0, where the difference would lose everything.
__device__ __forceinline__ float exp_minus_line(float x) {
    float p = 1.f / 39916800.f;                                          // 1 / 11!
    p = fmaf(p, x, 1.f / 3628800.f); p = fmaf(p, x, 1.f / 362880.f); p = fmaf(p, x, 1.f / 40320.f); p = fmaf(p, x, 1.f / 5040.f);
    p = fmaf(p, x, 1.f / 720.f); p = fmaf(p, x, 1.f / 120.f); p = fmaf(p, x, 1.f / 24.f); p = fmaf(p, x, 1.f / 6.f); p = fmaf(p, x, 0.5f);
    return p * x * x;
}

// Bytes of a mask word that are not 0.
__device__ __forceinline__ int count_bytes(unsigned w) { return __popc(__vcmpne4(w, 0u) & 0x01010101u); }
__device__ __forceinline__ int count_bytes(unsigned long long w) { return count_bytes((unsigned)w) + count_bytes((unsigned)(w >> 32)); }

// Tokens of every row, and per block how many tokens (by_sequence: rows that have any) its rows hold.
__global__ void __launch_bounds__(PO_COUNT_THREADS) policy_count_kernel(const unsigned char* mask, int* tokens, i64* partial, i64 rows, i64 length, i64 stride, int by_sequence) {
    pdl_wait(mask, tokens, partial);
    pdl_trigger();
    __shared__ i64 scratch[PO_COUNT_THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    i64 mine = 0;
    for (i64 r = (i64)blockIdx.x * (PO_COUNT_THREADS / 32) + warp; r < rows; r += (i64)gridDim.x * (PO_COUNT_THREADS / 32)) {
        const unsigned char* m = mask + r * stride;
        const int head = (int)min((i64)row_head(m), length);
        const i64 vectors = (length - head) / 16, tail = head + vectors * 16;
        int n = 0;
        if (lane < head) n += m[lane] != 0;
        for (i64 v = lane; v < vectors; v += 8 * 32) {
            uint4 u[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = v + k * 32 < vectors ? *reinterpret_cast<const uint4*>(m + head + (v + k * 32) * 16) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int k = 0; k < 8; ++k) n += count_bytes(u[k].x) + count_bytes(u[k].y) + count_bytes(u[k].z) + count_bytes(u[k].w);
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
        for (int w = 0; w < PO_COUNT_THREADS / 32; ++w) sum += scratch[w];
        partial[blockIdx.x] = sum;
    }
}

struct PolicySums { double pg = 0.0, kl = 0.0, clipped = 0.0; };

__device__ __forceinline__ void write_terms(float* terms, double pg, double kl, double clipped, double kl_weight) {
    terms[0] = (float)(kl_weight == 0.0 ? pg : pg + kl_weight * kl);
    terms[1] = (float)pg; terms[2] = (float)kl; terms[3] = (float)clipped;
}

// N tokens, ALL or those whose byte of the mask word is not 0: their terms without their weight are added to pg, kl and clip, g is their gradient
// (without the weight; 0 for the others).  No branch but two rare ones: lanes differ.
template <int N, bool ALL, typename Word>
__device__ __forceinline__ void policy_tokens(const float (&lp)[N], const float (&old)[N], const float (&ref)[N], bool has_ref, const float (&A)[N], Word w, const PolicyShape& s,
                                              float (&g)[N], float& pg, float& kl, float& clip) {
    // past the border that counts for the sign of A?  The fp32 difference is good to half a step of its own; next to a border the exact one is taken
    bool cut[N];
    float closest = INFINITY;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float past = (lp[e] - old[e]) - (A[e] > 0.f ? (float)s.log_high : (float)s.log_low);
        closest = fminf(closest, fabsf(past));
        cut[e] = past * 1e30f * A[e] > 0.f;                               // (of the same sign; the factor keeps a small A from taking the product to 0)
    }
    if (closest <= s.near) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const double exact = (double)lp[e] - (double)old[e];
            cut[e] = A[e] > 0.f ? exact > s.log_high : A[e] < 0.f && exact < s.log_low;
        }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const bool in = ALL || (w >> (8 * e) & 255u) != 0;
        const float r = cut[e] ? (A[e] > 0.f ? s.high : s.low) : A[e] == 0.f ? 0.f : exp_fast(lp[e] - old[e]), gain = r * A[e];
        pg -= in ? gain : 0.f;
        clip += in && cut[e] ? 1.f : 0.f;
        g[e] = cut[e] ? 0.f : -gain;
    }
    if (has_ref) {
        const bool in_loss = s.kl_weight != 0.f;                          // (a term that is only told has no slope, be it infinite)
        float farthest = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float delta = ref[e] - lp[e];
            farthest = delta != delta ? INFINITY : fmaxf(farthest, fabsf(delta));
        }
        if (farthest <= 1.f) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const bool in = ALL || (w >> (8 * e) & 255u) != 0;
                const float delta = ref[e] - lp[e], k = exp_minus_line(delta);
                kl += in ? k : 0.f;
                if (in_loss) g[e] -= s.kl_weight * (k + delta);
            }
        } else {
            // far from 0 the slope exp(delta) - 1 comes first: taken from the difference, -1 would be lost where a reference all but rules a token out
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const bool in = ALL || (w >> (8 * e) & 255u) != 0;
                const float delta = ref[e] - lp[e];
                const bool close = fabsf(delta) <= 1.f;
                float k, slope;
                if (close) { k = exp_minus_line(delta); slope = k + delta; }
                else { slope = expf(delta) - 1.f; k = slope - delta; }
                kl += in ? k : 0.f;
                if (in_loss) g[e] -= s.kl_weight * slope;
            }
        }
    }
    if (!ALL) {
#pragma unroll
        for (int e = 0; e < N; ++e) if ((w >> (8 * e) & 255u) == 0) g[e] = 0.f;
    }
}

constexpr float PO_MOST = 3.402823466e38f;   // the largest finite fp32

// One token whose terms are beyond fp32 before their weight: what is infinite (or NaN) in 32 bits is formed in 64, weighted there, rounded once.  pg, kl and clip are those of
// policy_tokens; the result is the weighted gradient, the weighted terms are added to the sums.
__device__ __forceinline__ float far_token(float lp, float old, float ref, bool has_ref, float A, float pg, float kl, float clip, float weighs, const PolicyShape& s, PolicySums& sums) {
    double P = (double)pg, slope = 0.0;
    if (fabsf(pg) <= PO_MOST || clip != 0.f) {
        sums.pg += (double)(weighs * pg);                                 // (as any token's)
    } else {
        P = -exp((double)lp - (double)old) * (double)A;
        sums.pg += (double)weighs * P;
    }
    if (has_ref) {
        const double delta = (double)ref - (double)lp;
        if (fabsf(kl) <= PO_MOST) {
            slope = (double)kl + delta;
            sums.kl += (double)(weighs * kl);
        } else {
            slope = exp(delta) - 1.0;
            sums.kl += (double)weighs * (slope - delta);
        }
    }
    sums.clipped += (double)(weighs * clip);
    double g = clip != 0.f ? 0.0 : P;
    if (s.kl_weight != 0.f) g -= (double)s.kl_weight * slope;
    return (float)((double)weighs * g);
}

// FLAT: all arrays are contiguous, a vector of VEC tokens may run over the end of a row.  Otherwise token by token, any strides.
template <typename T, bool FLAT>
__global__ void __launch_bounds__(PO_THREADS) policy_kernel(const T* logps, const T* old, const T* ref, const T* adv, const unsigned char* mask, const int* tokens, const i64* counted,
                                                            T* grad, PolicySums* partial, float* terms, PolicyShape s) {
    pdl_wait(logps, old, ref, adv, mask, tokens, counted, grad, partial, terms);
    pdl_trigger();
    constexpr int VEC = FLAT ? Elem<T>::VEC : 1;
    typedef typename MaskWord<Elem<T>::VEC>::type Word;
    __shared__ int row_tokens[PO_ONE_ROWS], seen;
    const int tid = threadIdx.x;
    const bool in_block = s.one && mask && (s.norm == 0.0 || s.by_sequence);
    if (in_block) {
        if (tid == 0) seen = 0;
        for (int r = tid; r < (int)s.rows; r += PO_THREADS) row_tokens[r] = 0;
        __syncthreads();
        const unsigned all = (unsigned)(s.rows * s.length), length = (unsigned)s.length, words = FLAT ? all / Elem<T>::VEC : 0u;
        int n = 0;                                                     // tokens, whole numbers: any order
        auto add = [&](unsigned row, int k) { if (s.by_sequence) atomicAdd(&row_tokens[row], k); else n += k; };
        if constexpr (FLAT) {
            for (unsigned base = tid; base < words; base += 4 * PO_THREADS) {
                Word w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = base + k * PO_THREADS < words ? reinterpret_cast<const Word*>(mask)[base + k * PO_THREADS] : (Word)0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (w[k] == 0) continue;
                    const unsigned i = (base + k * PO_THREADS) * Elem<T>::VEC, row = s.by_sequence ? i / length : 0u;
                    if (!s.by_sequence || i + Elem<T>::VEC <= (row + 1) * length) {
                        add(row, count_bytes(w[k]));
                    } else {
                        for (int e = 0; e < Elem<T>::VEC; ++e) if (w[k] >> (8 * e) & 255u) add((i + e) / length, 1);
                    }
                }
            }
        }
        for (unsigned i = words * Elem<T>::VEC + tid; i < all; i += PO_THREADS) {
            const unsigned row = i / length;
            if (mask[(i64)row * s.mask_stride + (i - row * length)]) add(row, 1);
        }
        __syncthreads();
        if (s.by_sequence) for (int r = tid; r < (int)s.rows; r += PO_THREADS) n += row_tokens[r] > 0;
        n = __reduce_add_sync(0xffffffffu, n);
        if ((tid & 31) == 0 && n) atomicAdd(&seen, n);
        __syncthreads();
    }
    double norm = s.norm;
    if (norm == 0.0) {
        if (in_block) {
            norm = (double)seen;
        } else if (counted) {                                          // every warp for itself: whole numbers
            i64 n = 0;
#pragma unroll
            for (int b = 0; b < PO_COUNT_BLOCKS; b += 32) n += b + (tid & 31) < s.count_blocks ? counted[b + (tid & 31)] : 0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
            norm = (double)n;
        } else {
            norm = s.by_sequence ? (s.length > 0 ? (double)s.rows : 0.0) : (double)s.rows * (double)s.length;
        }
    }
    const float inverse = norm > 0.0 ? (float)(1.0 / norm) : 0.f;
    auto weight = [&](i64 row) {
        if (!s.by_sequence) return inverse;
        const i64 n = in_block ? (i64)row_tokens[row] : tokens ? (i64)tokens[row] : s.length;
        return n > 0 ? __fdividef(inverse, (float)n) : 0.f;
    };
    PolicySums sums;
    const i64 all = s.rows * s.length, vectors = all / VEC, step = PO_THREADS;
    const bool small = all < (1ll << 31);                              // (a division of 32 bits)
    auto token = [&](i64 i) {                                       // one token, any strides
        const i64 row = small ? (i64)((unsigned)i / (unsigned)s.length) : i / s.length, t = i - row * s.length;
        T* g = grad + i;
        if (mask && !mask[row * s.mask_stride + t]) { *g = Elem<T>::put(0.f); return; }
        float pg = 0.f, kl = 0.f, clip = 0.f;
        const float A = Elem<T>::get(adv[row * s.adv_stride + (s.adv_per_token ? t : 0)]), weighs = weight(row);
        const float x[1] = {Elem<T>::get(logps[row * s.logp_stride + t])}, o[1] = {Elem<T>::get(old[row * s.old_stride + t])}, a[1] = {A};
        const float f[1] = {ref ? Elem<T>::get(ref[row * s.ref_stride + t]) : 0.f};
        float v[1];
        policy_tokens<1, true, unsigned>(x, o, f, ref != nullptr, a, 1u, s, v, pg, kl, clip);
        if (!(fabsf(pg) + fabsf(kl) <= PO_MOST)) {
            *g = Elem<T>::put(far_token(x[0], o[0], f[0], ref != nullptr, A, pg, kl, clip, weighs, s, sums));
            return;
        }
        *g = Elem<T>::put(weighs * v[0]);
        sums.pg += (double)(weighs * pg); sums.kl += (double)(weighs * kl); sums.clipped += (double)(weighs * clip);
    };
    const i64 start = (i64)blockIdx.x * s.per_block + tid, stop = min(start - tid + s.per_block, vectors);
    auto word = [&](i64 v) { return !FLAT || v >= stop ? (Word)0 : mask ? *reinterpret_cast<const Word*>(mask + v * VEC) : ~(Word)0; };
    if constexpr (!FLAT) {
        for (i64 v = start; v < stop; v += step) token(v);
    } else if (start < stop) {
        Word next = word(start);
        // row and position of the vector, carried along
        const i64 skip_rows = step * VEC / s.length, skip = step * VEC - skip_rows * s.length;
        i64 row = start * VEC / s.length, t = start * VEC - row * s.length;
        for (i64 v = start; v < stop; v += step) {
            const i64 i = v * VEC;
            const Word w = next;
            next = word(v + step);                                     // (on its way while this one's tokens are)
            if (w == 0) {
                store_vec(grad + i, make_uint4(0u, 0u, 0u, 0u));
            } else {
                float x[VEC], o[VEC], f[VEC], A[VEC], g[VEC];
                const uint4 ux = load_once(logps + i), uo = load_once(old + i), uf = ref ? load_once(ref + i) : make_uint4(0u, 0u, 0u, 0u);
                const uint4 ua = s.adv_per_token ? load_once(adv + i) : make_uint4(0u, 0u, 0u, 0u);
                const float weighs = weight(row);
                Elem<T>::unpack(ux, x); Elem<T>::unpack(uo, o); Elem<T>::unpack(uf, f); Elem<T>::unpack(ua, A);
                if (!s.adv_per_token) {
                    const float a = Elem<T>::get(adv[row * s.adv_stride]);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) A[e] = a;
                }
                float pg = 0.f, kl = 0.f, clip = 0.f;
                const bool in_row = t + VEC <= s.length;               // else it runs over the end of one
                if (in_row) {
                    // (a word of ones: all; other bytes may stand for true, they are looked at one by one)
                    if (!mask || w == (Word)0x0101010101010101ull) policy_tokens<VEC, true, Word>(x, o, f, ref != nullptr, A, w, s, g, pg, kl, clip);
                    else policy_tokens<VEC, false, Word>(x, o, f, ref != nullptr, A, w, s, g, pg, kl, clip);
                }
                if (!in_row || !(fabsf(pg) + fabsf(kl) <= PO_MOST)) {  // (or a term, or the sum of some, is beyond 32 bits)
                    const PolicySums before = sums;
#pragma unroll 1
                    for (int e = 0; e < VEC; ++e) token(i + e);
                    if (in_row) {                                      // a term that is not beyond them is added up as any other vector's: the other one leaves no trace in it
                        if (fabsf(pg) <= PO_MOST) sums.pg = before.pg + (double)(weighs * pg);
                        if (fabsf(kl) <= PO_MOST) sums.kl = before.kl + (double)(weighs * kl);
                        sums.clipped = before.clipped + (double)(weighs * clip);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) g[e] *= weighs;
                    store_vec(grad + i, Elem<T>::pack(g));
                    sums.pg += (double)(weighs * pg); sums.kl += (double)(weighs * kl); sums.clipped += (double)(weighs * clip);
                }
            }
            row += skip_rows; t += skip;
            if (t >= s.length) { t -= s.length; ++row; }
        }
    }
    if (FLAT && blockIdx.x == 0 && vectors * VEC + tid < all) token(vectors * VEC + tid);
    __shared__ PolicySums of_warp[PO_THREADS / 32];
    sums.pg = warp_sum(sums.pg); sums.kl = warp_sum(sums.kl); sums.clipped = warp_sum(sums.clipped);
    if ((tid & 31) == 0) of_warp[tid >> 5] = sums;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int w = 1; w < PO_THREADS / 32; ++w) { sums.pg += of_warp[w].pg; sums.kl += of_warp[w].kl; sums.clipped += of_warp[w].clipped; }
    }
    if (s.one) {
        __shared__ double mine[3];
        double all_sums[3] = {sums.pg, sums.kl, sums.clipped};
        cluster_sums(all_sums, mine);
        if (tid == 0 && cluster_rank() == 0) write_terms(terms, all_sums[0], all_sums[1], all_sums[2], (double)s.kl_weight);
        return;
    }
    if (tid == 0) partial[blockIdx.x] = sums;
}

__global__ void __launch_bounds__(PO_FINISH_THREADS) policy_finish_kernel(const PolicySums* partial, float* terms, int blocks, float kl_weight) {
    pdl_wait(partial, terms);
    pdl_trigger();
    __shared__ double scratch[PO_FINISH_THREADS / 32];
    PolicySums v;
    for (int b = threadIdx.x; b < blocks; b += PO_FINISH_THREADS) { v.pg += partial[b].pg; v.kl += partial[b].kl; v.clipped += partial[b].clipped; }
    v.pg = block_sum<PO_FINISH_THREADS>(v.pg, scratch);
    v.kl = block_sum<PO_FINISH_THREADS>(v.kl, scratch);
    v.clipped = block_sum<PO_FINISH_THREADS>(v.clipped, scratch);
    if (threadIdx.x == 0) write_terms(terms, v.pg, v.kl, v.clipped, (double)kl_weight);
}

}  // namespace ef21
