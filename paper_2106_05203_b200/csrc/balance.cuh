// Balance loss of a router, tokens per expert, and the gradient of the router's logits.
//
//   p_t = softmax(x_t);  counts_e = tokens that chose e;  N = tokens that count;  f_e = counts_e / (K N);  P_e = 1/N sum_t p_te
//   loss = weight E sum_e f_e P_e;   dx_tj = weight E / N p_tj (f_j - sum_e f_e p_te)
//
// The gradient needs the counts of the whole batch, but not P: so the choices are counted first (2 to 64 bytes a token), then one pass over the logits
// forms the softmax, its column sums and the gradient.  f is taken about its mean: f_e - 1/E = (counts_e E - K N) / (K N E), exact in
// whole numbers, since the sum over p takes a constant away -- a balanced router has small differences of shares that are alike.
#pragma once
#include "element.cuh"
#include "preference.cuh"

namespace ef21 {

constexpr int BL_THREADS = 256;
constexpr int BL_MAX_EXPERTS = 1024;
constexpr int BL_MAX_BLOCKS = 148 * 4;
constexpr int BL_FINISH_COLUMNS = 32, BL_FINISH_GROUPS = 32;

struct BalanceShape {
    i64 rows;
    int experts, chosen, wide;
    i64 logit_stride, choice_stride;
    double weight;
};

struct BalanceWork { unsigned tokens, ticket; };

__global__ void __launch_bounds__(BL_THREADS) balance_clear_kernel(int* counts, BalanceWork* work, int experts) {
    pdl_wait(counts, work);
    pdl_trigger();
    for (int e = threadIdx.x; e < experts; e += BL_THREADS) counts[e] = 0;
    if (threadIdx.x == 0) { work->tokens = 0; work->ticket = 0; }
}

// Whole numbers: the order of the additions does not show.
__global__ void __launch_bounds__(BL_THREADS) balance_count_kernel(const void* choices, const unsigned char* mask, int* counts, BalanceWork* work, BalanceShape s) {
    pdl_wait(choices, mask, counts, work);
    pdl_trigger();
    __shared__ int here[BL_MAX_EXPERTS];
    __shared__ unsigned tokens;
    for (int e = threadIdx.x; e < s.experts; e += BL_THREADS) here[e] = 0;
    if (threadIdx.x == 0) tokens = 0;
    __syncthreads();
    unsigned mine = 0;
    const i64 all = s.rows * s.chosen;
    for (i64 i = (i64)blockIdx.x * BL_THREADS + threadIdx.x; i < all; i += (i64)gridDim.x * BL_THREADS) {
        const i64 row = i / s.chosen;
        const int k = (int)(i - row * s.chosen);
        if (mask && !mask[row]) continue;
        mine += k == 0;
        const i64 e = index_at(choices, s.wide, row * s.choice_stride + k);
        if (e >= 0 && e < s.experts) atomicAdd(&here[e], 1);
    }
    mine = __reduce_add_sync(0xffffffffu, mine);
    if ((threadIdx.x & 31) == 0 && mine) atomicAdd(&tokens, mine);
    __syncthreads();
    for (int e = threadIdx.x; e < s.experts; e += BL_THREADS) if (here[e]) atomicAdd(counts + e, here[e]);
    if (threadIdx.x == 0 && tokens) atomicAdd(&work->tokens, tokens);
}

// `lanes` lanes (a power of two) share a row, lane l its columns l, l + lanes, ...: PER of them at most.
template <typename T, int PER>
__global__ void __launch_bounds__(BL_THREADS) balance_kernel(const T* logits, const unsigned char* mask, const int* counts, const BalanceWork* work, T* grad, float* partial, BalanceShape s, int lanes) {
    pdl_wait(logits, mask, counts, work, grad, partial);
    pdl_trigger();
    __shared__ float column[BL_MAX_EXPERTS];
    const int tid = threadIdx.x, lane = tid & (lanes - 1), group = tid / lanes, groups = BL_THREADS / lanes, E = s.experts;
    const double N = (double)work->tokens, KN = N * s.chosen;
    float apart[PER], sum[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane + i * lanes;
        apart[i] = e < E && N > 0.0 ? (float)(((double)counts[e] * E - KN) / (KN * E)) : 0.f;
        sum[i] = 0.f;
    }
    const float factor = N > 0.0 ? (float)(s.weight * E / N) : 0.f;
    const i64 rounds = (s.rows + (i64)gridDim.x * groups - 1) / ((i64)gridDim.x * groups);
    for (i64 k = 0; k < rounds; ++k) {                                   // (whole warps: the shuffles need every lane)
        const i64 row = ((k * gridDim.x) + blockIdx.x) * groups + group;
        const bool in = row < s.rows, keep = in && (!mask || mask[row]);
        const T* x = logits + row * s.logit_stride;
        float f[PER], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = lane + i * lanes;
            f[i] = keep && e < E ? Elem<T>::get(x[e]) : -INFINITY;
            top = fmaxf(top, f[i]);
        }
        for (int o = lanes >> 1; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float base = top == -INFINITY ? 0.f : top;         // (a row of -inf only, or left out: all 0)
        float total = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) { f[i] = exp2_fast((f[i] - base) * LOG2E); total += f[i]; }
        for (int o = lanes >> 1; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        const float scale = !keep || total == 0.f ? 0.f : 1.f / total;
        float mean = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) { f[i] *= scale; mean = fmaf(f[i], apart[i], mean); sum[i] += f[i]; }
        for (int o = lanes >> 1; o > 0; o >>= 1) mean += __shfl_xor_sync(0xffffffffu, mean, o);
        if (in) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = lane + i * lanes;
                if (e < E) grad[row * E + e] = Elem<T>::put(keep ? factor * f[i] * (apart[i] - mean) : 0.f);
            }
        }
    }
    // column sums of the block, group after group
    for (int g = 0; g < groups; ++g) {
        if (group == g) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = lane + i * lanes;
                if (e < E) column[e] = g == 0 ? sum[i] : column[e] + sum[i];
            }
        }
        __syncthreads();
    }
    for (int e = tid; e < E; e += BL_THREADS) partial[(i64)blockIdx.x * E + e] = column[e];
}

// Mean probabilities, 32 columns to a block, and the loss by the block that comes last (from the others' sums, in their order).
__global__ void __launch_bounds__(BL_FINISH_COLUMNS * BL_FINISH_GROUPS) balance_finish_kernel(const float* partial, const int* counts, BalanceWork* work, double* part, float* probs, float* loss,
                                                                                             int blocks, int experts, int chosen, double weight) {
    pdl_wait(partial, counts, work, part, probs, loss);
    pdl_trigger();
    __shared__ double sums[BL_FINISH_GROUPS][BL_FINISH_COLUMNS + 1];
    __shared__ bool last;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, e = blockIdx.x * BL_FINISH_COLUMNS + x;
    double v = 0.0;
    if (e < experts) for (int b = y; b < blocks; b += BL_FINISH_GROUPS) v += (double)partial[(i64)b * experts + e];
    sums[y][x] = v;
    __syncthreads();
    if (y == 0) {
        const double N = (double)work->tokens;
        double sum = 0.0;
        for (int g = 0; g < BL_FINISH_GROUPS; ++g) sum += sums[g][x];
        const double mean = N > 0.0 ? sum / N : 0.0;
        double term = 0.0;
        if (e < experts) {
            probs[e] = (float)mean;
            if (N > 0.0) term = (double)counts[e] / (N * chosen) * mean;
        }
        term = warp_sum(term);
        if (x == 0) {
            *(volatile double*)(part + blockIdx.x) = term;
            __threadfence();
            last = atomicAdd(&work->ticket, 1u) == gridDim.x - 1;
        }
    }
    __syncthreads();
    if (last && threadIdx.x == 0) {
        __threadfence();
        double sum = 0.0;
        for (int b = 0; b < (int)gridDim.x; ++b) sum += *(volatile double*)(part + b);
        *loss = (float)(weight * experts * sum);
    }
}

}  // namespace ef21
