// Balance loss of a router, tokens per expert, and the gradient of the router's logits.
//
//   p_t = softmax(x_t);  counts_e = tokens that chose e;  N = tokens that count;  f_e = counts_e / (K N);  P_e = 1/N sum_t p_te
//   loss = weight E sum_e f_e P_e;   dx_tj = weight E / N p_tj (f_j - sum_e f_e p_te)
//
// The gradient needs the counts of the whole batch, but not P: so the choices are counted first (4 or 8 bytes each), then one pass over the logits
// forms the softmax, its column sums and the gradient, and a last kernel adds the blocks' column sums up.  Few rows: one cluster does it all, every block
// counting for itself.  f is taken about its mean: f_e - 1/E = (counts_e E - K N) / (K N E), exact in whole numbers, since the sum over p takes a constant away -- a
// balanced router has small differences of shares that are alike.
//
// 131,072 x 256 bf16, 8 chosen: 40 us, of which the pass 32 by itself (140 instructions per row and warp at 0.59 of the issue slots, 16 lanes a row; 32 lanes a row: 218 and 45 us); 512 x 8: 8.6 us, a
// launch.  Rows that are no whole aligned vectors move element by element, each with its own bound check: 100,000 x 255 bf16 85 us, five times its bytes.
#pragma once
#include "cluster.cuh"
#include "element.cuh"
#include "preference.cuh"

namespace ef21 {

constexpr int BL_THREADS = 256, BL_COUNT_THREADS = 1024;
constexpr int BL_MAX_EXPERTS = 1024;
constexpr int BL_MAX_BLOCKS = 148 * 3;         // (registers for three blocks an SM)
constexpr int BL_FINISH_COLUMNS = 8, BL_FINISH_GROUPS = 128;
constexpr unsigned BL_CLUSTER = 8;
constexpr float BL_FUSED = 1e6f;               // logits up to here: the exponent by one operation
constexpr i64 BL_ONE_CHOICES = 16384, BL_ONE_LOGITS = 32768;      // up to here: one cluster

struct BalanceShape {
    i64 rows;
    int experts, chosen, wide;
    i64 logit_stride, choice_stride;
    double weight;
    int lanes;                              // that share a row (a power of two)
    int one;                                // all blocks are one cluster: they count, and write everything
    int whole_in, whole_out;                // rows of the logits, of the gradient begin on 16 bytes
};

struct BalanceWork { unsigned tokens, ticket; };

__global__ void __launch_bounds__(BL_THREADS) balance_clear_kernel(int* counts, BalanceWork* work, int experts) {
    pdl_wait(counts, work);
    pdl_trigger();
    for (int e = threadIdx.x; e < experts; e += BL_THREADS) counts[e] = 0;
    if (threadIdx.x == 0) { work->tokens = 0; work->ticket = 0; }
}

// Adds choices [first, all) of every `step` to here[experts], the tokens among them to n.  Whole numbers: the order of the additions does not show.
__device__ __forceinline__ void count_choices(const void* choices, const unsigned char* mask, const BalanceShape& s, unsigned first, unsigned step, int* here, unsigned& n) {
    const unsigned all = (unsigned)(s.rows * s.chosen), chosen = (unsigned)s.chosen;
    for (unsigned long long base = first; base < all; base += 4ull * step) {
        i64 e[4];
        bool in[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned long long i = base + (unsigned long long)k * step;
            in[k] = i < all;
            if (!in[k]) continue;
            const unsigned row = (unsigned)i / chosen, j = (unsigned)i - row * chosen;
            in[k] = !mask || mask[row];
            e[k] = index_at(choices, s.wide, (i64)row * s.choice_stride + j);
            n += in[k] && j == 0;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) if (in[k] && e[k] >= 0 && e[k] < s.experts) atomicAdd(&here[e[k]], 1);
    }
}

__global__ void __launch_bounds__(BL_COUNT_THREADS) balance_count_kernel(const void* choices, const unsigned char* mask, int* counts, BalanceWork* work, BalanceShape s) {
    pdl_wait(choices, mask, counts, work);
    pdl_trigger();
    __shared__ int here[BL_MAX_EXPERTS];
    __shared__ unsigned tokens;
    for (int e = threadIdx.x; e < s.experts; e += BL_COUNT_THREADS) here[e] = 0;
    if (threadIdx.x == 0) tokens = 0;
    __syncthreads();
    unsigned mine = 0;
    count_choices(choices, mask, s, blockIdx.x * BL_COUNT_THREADS + threadIdx.x, gridDim.x * BL_COUNT_THREADS, here, mine);
    mine = __reduce_add_sync(0xffffffffu, mine);
    if ((threadIdx.x & 31) == 0 && mine) atomicAdd(&tokens, mine);
    __syncthreads();
    for (int e = threadIdx.x; e < s.experts; e += BL_COUNT_THREADS) if (here[e]) atomicAdd(counts + e, here[e]);
    if (threadIdx.x == 0 && tokens) atomicAdd(&work->tokens, tokens);
}

// A team of s.lanes lanes takes ROWS rows at a time; lane l has PER vectors of VEC columns, lanes side by side, the last vector of a row perhaps not full.  Rows that are
// no whole aligned vectors are read and written element by element, in the same order of lanes and additions.
// LANES: 32 or 16, or 0 where s.lanes may be fewer.
template <typename T, int PER, int ROWS, int LANES>
__global__ void __launch_bounds__(BL_THREADS, PER * Elem<T>::VEC <= 16 ? 3 : 1) balance_kernel(const T* logits, const void* choices, const unsigned char* mask, int* counts, const BalanceWork* work, T* grad, float* partial,
                                                             float* probs, float* loss, BalanceShape s) {
    pdl_wait(logits, choices, mask, counts, work, grad, partial, probs, loss);
    pdl_trigger();
    constexpr int VEC = Elem<T>::VEC;
    __shared__ float column[BL_MAX_EXPERTS];
    __shared__ int here[BL_MAX_EXPERTS];
    extern __shared__ float of_warp[];                                // [warps][E]
    __shared__ unsigned seen;
    __shared__ double terms, scratch[BL_THREADS / 32];
    const int tid = threadIdx.x, lanes = LANES ? LANES : s.lanes, lane = tid & (lanes - 1), group = tid / lanes, groups = BL_THREADS / lanes, E = s.experts;
    if (s.one) {
        for (int e = tid; e < E; e += BL_THREADS) here[e] = 0;
        if (tid == 0) seen = 0;
        __syncthreads();
        unsigned mine = 0;
        count_choices(choices, mask, s, tid, BL_THREADS, here, mine);
        mine = __reduce_add_sync(0xffffffffu, mine);
        if ((tid & 31) == 0 && mine) atomicAdd(&seen, mine);
        __syncthreads();
        if (blockIdx.x == 0) for (int e = tid; e < E; e += BL_THREADS) counts[e] = here[e];
    }
    const double N = (double)(s.one ? seen : work->tokens), KN = N * s.chosen;
    auto column_of = [&](int i) { return (lane + i / VEC * lanes) * VEC + i % VEC; };
    constexpr int PAIRS = PER * VEC / 2;
    __shared__ float about_mean[BL_MAX_EXPERTS];
    for (int e = tid; e < E; e += BL_THREADS) about_mean[e] = N > 0.0 ? (float)(((double)(s.one ? here[e] : counts[e]) * E - KN) / (KN * E)) : 0.f;
    __syncthreads();
    auto share = [&](int e) { return e < E ? about_mean[e] : 0.f; };
    Two apart[PAIRS], sum[PAIRS];
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
        apart[i] = two(share(column_of(2 * i)), share(column_of(2 * i + 1)));
        sum[i] = two(0.f);
    }
    const float factor = N > 0.0 ? (float)(s.weight * E / N) : 0.f;
    const i64 step = (i64)gridDim.x * groups;
    uint4 raw[ROWS][PER];
    bool counts_in[ROWS];
    auto fetch = [&](i64 row0) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const i64 row = row0 + r * step;
            counts_in[r] = row < s.rows && (!mask || mask[row]);
            const T* x = logits + row * s.logit_stride;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = (lane + i * lanes) * VEC;
                if (row >= s.rows || at >= E) continue;
                if (s.whole_in) { raw[r][i] = load_once(x + at); continue; }
                float v[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[e] = at + e < E ? Elem<T>::get(x[at + e]) : -INFINITY;
                raw[r][i] = Elem<T>::pack(v);
            }
        }
    };
    fetch((i64)blockIdx.x * groups + group);
    for (i64 row0 = (i64)blockIdx.x * groups + group; row0 - group < s.rows; row0 += step * ROWS) {     // (whole warps: the shuffles need every lane)
        // (fp32 pairs: one instruction for two columns)
        Two f[ROWS][PAIRS];
        float top[ROWS], total[ROWS], mean[ROWS];
        bool keep[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) keep[r] = counts_in[r];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            top[r] = -INFINITY;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                constexpr unsigned nothing = Elem<T>::NEG_INF;
                if (!keep[r] || (lane + i * lanes) * VEC >= E) raw[r][i] = make_uint4(nothing, nothing, nothing, nothing);
                top[r] = fmaxf(top[r], Elem<T>::top(raw[r][i]));
                float v[VEC];
                Elem<T>::unpack(raw[r][i], v);
#pragma unroll
                for (int e = 0; e < VEC; e += 2) f[r][(i * VEC + e) / 2] = two(v[e], v[e + 1]);
            }
        }
        fetch(row0 + step * ROWS);                                           // (on their way while these rows are worked on)
#pragma unroll
        for (int o = lanes >> 1; o > 0; o >>= 1) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], o));
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float base = top[r] == -INFINITY ? 0.f : top[r];                 // (a row of -inf only, or left out: all 0)
            const Two exponent = two(LOG2E);
            // The exponent is one fused operation about base log2 e, whose rounding all of the row have in common: it cancels in p as long as it is small (0.06 in base 2
            // at the border).  Beyond -- a mask of a large value that leaves nothing, a choice forced by one -- it would leave the range of 2^x, and the maximum is
            // subtracted first.
            if (fabsf(base) > BL_FUSED) {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) f[r][i] = add2(f[r][i], two(-base));
                base = 0.f;
            }
            const Two shift = two(-base * LOG2E);
            Two sum2 = two(0.f), mean2 = two(0.f);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                float a, b;
                split(fma2(f[r][i], exponent, shift), a, b);
                f[r][i] = two(exp2_fast(a), exp2_fast(b));
                sum2 = add2(sum2, f[r][i]);
                mean2 = fma2(f[r][i], apart[i], mean2);
            }
            float a, b;
            split(sum2, a, b); total[r] = a + b;
            split(mean2, a, b); mean[r] = a + b;
        }
#pragma unroll
        for (int o = lanes >> 1; o > 0; o >>= 1) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                total[r] += __shfl_xor_sync(0xffffffffu, total[r], o);
                mean[r] += __shfl_xor_sync(0xffffffffu, mean[r], o);
            }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const i64 row = row0 + r * step;
            if (row >= s.rows) continue;
            const float scale = total[r] == 0.f ? 0.f : __fdividef(1.f, total[r]), slope = factor * scale;
            const Two p = two(scale), m = two(slope), about = two(-mean[r] * scale * slope);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                sum[i] = fma2(f[r][i], p, sum[i]);
                f[r][i] = mul2(f[r][i], fma2(apart[i], m, about));
            }
            T* g = grad + row * E;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = (lane + i * lanes) * VEC;
                if (at >= E) continue;
                float v[VEC];
#pragma unroll
                for (int e = 0; e < VEC; e += 2) split(f[r][(i * VEC + e) / 2], v[e], v[e + 1]);
                if (s.whole_out) { store_vec(g + at, Elem<T>::pack(v)); continue; }
#pragma unroll
                for (int e = 0; e < VEC; ++e) if (at + e < E) g[at + e] = Elem<T>::put(v[e]);
            }
        }
    }
    // column sums: a warp's teams by shuffles, then the block's warps one after the other
    for (int o = lanes; o < 32; o <<= 1) {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) sum[i] = add2(sum[i], __shfl_xor_sync(0xffffffffu, sum[i], o));
    }
    if ((tid & 31) < lanes) {
        float* mine = of_warp + (tid >> 5) * E;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            float a, b;
            split(sum[i], a, b);
            const int e = column_of(2 * i);
            if (e < E) mine[e] = a;
            if (e + 1 < E) mine[e + 1] = b;
        }
    }
    __syncthreads();
    for (int e = tid; e < E; e += BL_THREADS) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < BL_THREADS / 32; ++w) v += of_warp[w * E + e];
        column[e] = v;
    }
    __syncthreads();
    if (!s.one) {
        for (int e = tid; e < E; e += BL_THREADS) partial[(i64)blockIdx.x * E + e] = column[e];
        return;
    }
    const unsigned C = cluster_blocks(), rank = cluster_rank();
    if (C > 1) cluster_barrier();
    double term = 0.0;
    for (int e = (int)rank * BL_THREADS + tid; e < E; e += (int)C * BL_THREADS) {
        double v = 0.0;
        for (unsigned r = 0; r < C; ++r) v += (double)(C > 1 ? remote_float(&column[e], r) : column[e]);
        v = N > 0.0 ? v / N : 0.0;
        probs[e] = (float)v;
        if (N > 0.0) term += (double)here[e] / KN * v;
    }
    double all[1] = {block_sum<BL_THREADS>(term, scratch)};
    cluster_sums(all, &terms);                                    // (its barriers are behind the reads of column)
    if (tid == 0 && rank == 0) *loss = (float)(s.weight * E * all[0]);
}

// Mean probabilities, BL_FINISH_COLUMNS columns to a block, and the loss by the block that comes last (from the others' sums, in their order).
__global__ void __launch_bounds__(BL_FINISH_COLUMNS * BL_FINISH_GROUPS) balance_finish_kernel(const float* partial, const int* counts, BalanceWork* work, double* part, float* probs, float* loss,
                                                                                             int blocks, int experts, int chosen, double weight) {
    pdl_wait(partial, counts, work, part, probs, loss);
    pdl_trigger();
    __shared__ double sums[BL_FINISH_GROUPS][BL_FINISH_COLUMNS];
    __shared__ bool last;
    const int x = threadIdx.x % BL_FINISH_COLUMNS, y = threadIdx.x / BL_FINISH_COLUMNS, e = blockIdx.x * BL_FINISH_COLUMNS + x;
    constexpr int MOST = (BL_MAX_BLOCKS + BL_FINISH_GROUPS - 1) / BL_FINISH_GROUPS;
    float v[MOST];
#pragma unroll
    for (int k = 0; k < MOST; ++k) v[k] = e < experts && y + k * BL_FINISH_GROUPS < blocks ? partial[(i64)(y + k * BL_FINISH_GROUPS) * experts + e] : 0.f;
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < MOST; ++k) sum += (double)v[k];
    sums[y][x] = sum;
    __syncthreads();
    if (threadIdx.x < 32) {                                       // four lanes to a column
        const int col = threadIdx.x % BL_FINISH_COLUMNS, at = blockIdx.x * BL_FINISH_COLUMNS + col, share = threadIdx.x / BL_FINISH_COLUMNS;
        constexpr int SHARE = BL_FINISH_GROUPS * BL_FINISH_COLUMNS / 32;
        const double N = (double)work->tokens;
        sum = 0.0;
        for (int g = share * SHARE; g < (share + 1) * SHARE; ++g) sum += sums[g][col];
        for (int o = BL_FINISH_COLUMNS; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const double mean = N > 0.0 ? sum / N : 0.0;
        double term = 0.0;
        if (at < experts && share == 0) {
            probs[at] = (float)mean;
            if (N > 0.0) term = (double)counts[at] / (N * chosen) * mean;
        }
        term = warp_sum(term);
        if (threadIdx.x == 0) {
            *(volatile double*)(part + blockIdx.x) = term;
            __threadfence();
            last = atomicAdd(&work->ticket, 1u) == gridDim.x - 1;
        }
    }
    __syncthreads();
    if (last && threadIdx.x < 32) {
        __threadfence();
        double all = 0.0;
        for (int b = threadIdx.x; b < (int)gridDim.x; b += 32) all += *(volatile double*)(part + b);
        all = warp_sum(all);
        if (threadIdx.x == 0) *loss = (float)(weight * experts * all);
    }
}

}  // namespace ef21
