// Rows of a table by token, scaled, and the table's gradient: for every token the sum of the gradients at its positions, in ascending order of the
// positions, in 32 bits, rounded once.
//
//   out_t = s W[tok_t]          dW_v = s sum_{t: tok_t = v} g_t
//
// The gradient is no scatter (float atomics add in any order): positions are sorted by token (stable), then every row of the table is formed
// by one block from its run of positions and written once, zeros where no token names it.  A run of more than ED_CHUNK positions is
// added up ED_CHUNK sorted positions at a time by blocks of their own, whose sums its row adds in order.
//
// Sorting: up to ED_RANK_TOKENS tokens by counting, for every token, those in front of it -- one launch; more by a radix sort, digits of up to nine bits.
#pragma once
#include "element.cuh"

namespace ef21 {

constexpr int ED_THREADS = 256;
constexpr int ED_CHUNK = 32;
constexpr int ED_RANK_TOKENS = 8192;
constexpr int ED_RANK_THREADS = 256;
constexpr int RX_THREADS = 1024, RX_ITEMS = 4, RX_TILE = RX_THREADS * RX_ITEMS, RX_MAX_BITS = 9, RX_WARPS = RX_THREADS / 32;

// ---- lookup -------------------------------------------------------------------------------------------------------------------------------

// VECTORS: rows are whole numbers of 16 bytes and aligned.  One thread per 16 bytes (or element) of the output.
template <typename T, bool VECTORS>
__global__ void __launch_bounds__(ED_THREADS) embedding_kernel(const T* weight, const void* tokens, T* out, i64 count, i64 vocab, i64 dim, i64 stride, int wide, float scale) {
    pdl_wait(weight, tokens, out);
    pdl_trigger();
    constexpr int VEC = VECTORS ? Elem<T>::VEC : 1;
    const i64 per = dim / VEC, all = count * per;
    for (i64 i = (i64)blockIdx.x * ED_THREADS + threadIdx.x; i < all; i += (i64)gridDim.x * ED_THREADS) {
        const i64 t = i / per, j = (i - t * per) * VEC;
        const i64 v = index_at(tokens, wide, t);
        const bool in = v >= 0 && v < vocab;
        if (VECTORS) {
            float f[Elem<T>::VEC];
            Elem<T>::unpack(in ? *reinterpret_cast<const uint4*>(weight + v * stride + j) : make_uint4(0u, 0u, 0u, 0u), f);
#pragma unroll
            for (int e = 0; e < Elem<T>::VEC; ++e) f[e] *= scale;
            if (!in) {
#pragma unroll
                for (int e = 0; e < Elem<T>::VEC; ++e) f[e] = 0.f;
            }
            store_vec(out + t * dim + j, Elem<T>::pack(f));
        } else {
            out[t * dim + j] = Elem<T>::put(in ? Elem<T>::get(weight[v * stride + j]) * scale : 0.f);
        }
    }
}

// ---- sorting positions by token -------------------------------------------------------------------------------------------------------------

// A token that has a row and a gradient, else `vocab` (sorted behind all others and left there).
__device__ __forceinline__ int token_key(const void* tokens, int wide, i64 i, i64 vocab, i64 padding) {
    const i64 v = index_at(tokens, wide, i);
    return v >= 0 && v < vocab && v != padding ? (int)v : (int)vocab;
}

// Runs of all tokens: none yet.
__global__ void __launch_bounds__(ED_THREADS) embedding_clear_kernel(int2* runs, i64 vocab) {
    pdl_wait(runs);
    pdl_trigger();
    for (i64 v = (i64)blockIdx.x * ED_THREADS + threadIdx.x; v < vocab; v += (i64)gridDim.x * ED_THREADS) runs[v] = make_int2(0, 0);
}

// Few tokens: the place of each is the number of smaller ones plus that of equal ones before it.  A warp takes one token at a time.
__global__ void __launch_bounds__(ED_RANK_THREADS) embedding_rank_kernel(const void* tokens, int wide, int count, i64 vocab, i64 padding, int2* sorted, int2* runs) {
    pdl_wait(tokens, sorted, runs);
    pdl_trigger();
    extern __shared__ int keys[];
    for (int i = threadIdx.x; i < count; i += ED_RANK_THREADS) keys[i] = token_key(tokens, wide, i, vocab, padding);
    __syncthreads();
    const int lane = threadIdx.x & 31;
    for (int i = blockIdx.x * (ED_RANK_THREADS / 32) + (threadIdx.x >> 5); i < count; i += gridDim.x * (ED_RANK_THREADS / 32)) {
        const int key = keys[i];
        int less = 0, before = 0, equal = 0;
        for (int j = lane; j < count; j += 32) {
            const int other = keys[j];
            less += other < key;
            equal += other == key;
            before += other == key && j < i;
        }
        less = __reduce_add_sync(0xffffffffu, less);
        equal = __reduce_add_sync(0xffffffffu, equal);
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) {
            sorted[less + before] = make_int2(key, i);
            if (before == 0 && key < vocab) runs[key] = make_int2(less, less + equal);
        }
    }
}

// One pass of a radix sort over digits of `bits` bits: counts per tile, their places, the move.
// source: pairs (key, position) of the last pass, or null for the tokens themselves.
__device__ __forceinline__ int2 radix_item(const int2* source, const void* tokens, int wide, i64 i, i64 vocab, i64 padding) {
    return source ? source[i] : make_int2(token_key(tokens, wide, i, vocab, padding), (int)i);
}

__global__ void __launch_bounds__(RX_THREADS) radix_count_kernel(const int2* source, const void* tokens, int wide, i64 count, i64 vocab, i64 padding, int shift, int bits, int* counts) {
    pdl_wait(source, tokens, counts);
    pdl_trigger();
    __shared__ int here[1 << RX_MAX_BITS];
    const int bins = 1 << bits;
    for (int b = threadIdx.x; b < bins; b += RX_THREADS) here[b] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < RX_ITEMS; ++k) {
        const i64 i = (i64)blockIdx.x * RX_TILE + k * RX_THREADS + threadIdx.x;
        if (i < count) atomicAdd(&here[(radix_item(source, tokens, wide, i, vocab, padding).x >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += RX_THREADS) counts[(i64)blockIdx.x * bins + b] = here[b];
}

// counts[tile][bin] becomes the number of the bin's items in earlier tiles; totals[bin] that of all.  32 bins to a block, 32 groups of tiles.
__global__ void __launch_bounds__(RX_THREADS) radix_places_kernel(int* counts, int* totals, i64 tiles, int bins) {
    pdl_wait(counts, totals);
    pdl_trigger();
    __shared__ int sums[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, bin = blockIdx.x * 32 + x;
    const i64 per = (tiles + 31) / 32, begin = min(y * per, tiles), end = min(begin + per, tiles);
    int sum = 0;
    if (bin < bins) for (i64 t = begin; t < end; ++t) sum += counts[t * bins + bin];
    sums[y][x] = sum;
    __syncthreads();
    if (y == 0) {
        int before = 0;
        for (int g = 0; g < 32; ++g) { const int v = sums[g][x]; sums[g][x] = before; before += v; }
        if (bin < bins) totals[bin] = before;
    }
    __syncthreads();
    if (bin < bins) {
        int before = sums[y][x];
        for (i64 t = begin; t < end; ++t) { const int v = counts[t * bins + bin]; counts[t * bins + bin] = before; before += v; }
    }
}

__global__ void __launch_bounds__(RX_THREADS) radix_move_kernel(const int2* source, const void* tokens, int wide, i64 count, i64 vocab, i64 padding, int shift, int bits,
                                                               const int* counts, const int* totals, int2* target) {
    pdl_wait(source, tokens, counts, totals, target);
    pdl_trigger();
    __shared__ unsigned short warp_count[RX_WARPS][1 << RX_MAX_BITS];
    __shared__ int place[1 << RX_MAX_BITS];
    __shared__ unsigned scan[33];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, bins = 1 << bits;
    for (int b = lane; b < bins; b += 32) warp_count[warp][b] = 0;
    unsigned all;
    const unsigned mine = tid < bins ? (unsigned)totals[tid] : 0u;
    const unsigned before = block_excl_scan(mine, scan, all);
    if (tid < bins) place[tid] = (int)before + counts[(i64)blockIdx.x * bins + tid];
    // a warp's items are consecutive: (warp, k, lane) is their order
    int2 item[RX_ITEMS];
    int digit[RX_ITEMS], rank[RX_ITEMS];
    __syncwarp();
#pragma unroll
    for (int k = 0; k < RX_ITEMS; ++k) {
        const i64 i = (i64)blockIdx.x * RX_TILE + warp * (RX_ITEMS * 32) + k * 32 + lane;
        const bool in = i < count;
        item[k] = in ? radix_item(source, tokens, wide, i, vocab, padding) : make_int2(0, 0);
        digit[k] = in ? (item[k].x >> shift) & (bins - 1) : -1;
        const unsigned peers = __match_any_sync(0xffffffffu, digit[k]);
        const int first = __ffs(peers) - 1, ahead = __popc(peers & ((1u << lane) - 1u));
        int base = 0;
        if (in && lane == first) { base = warp_count[warp][digit[k]]; warp_count[warp][digit[k]] = (unsigned short)(base + __popc(peers)); }
        rank[k] = __shfl_sync(0xffffffffu, base, first) + ahead;
        __syncwarp();
    }
    __syncthreads();
    for (int b = tid; b < bins; b += RX_THREADS) {
        int sum = 0;
        for (int w = 0; w < RX_WARPS; ++w) { const int v = warp_count[w][b]; warp_count[w][b] = (unsigned short)sum; sum += v; }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < RX_ITEMS; ++k)
        if (digit[k] >= 0) target[place[digit[k]] + warp_count[warp][digit[k]] + rank[k]] = item[k];
}

// The run of every token that is there.
__global__ void __launch_bounds__(ED_THREADS) embedding_runs_kernel(const int2* sorted, int2* runs, i64 count, i64 vocab) {
    pdl_wait(sorted, runs);
    pdl_trigger();
    const i64 i = (i64)blockIdx.x * ED_THREADS + threadIdx.x;
    if (i >= count) return;
    const int key = sorted[i].x;
    if (key >= vocab) return;
    if (i == 0 || sorted[i - 1].x != key) runs[key].x = (int)i;
    if (i == count - 1 || sorted[i + 1].x != key) runs[key].y = (int)(i + 1);
}

// ---- the table's gradient -------------------------------------------------------------------------------------------------------------------

// Sum over sorted positions [begin, end) of VEC columns from j on, in order.
template <typename T, int VEC>
__device__ __forceinline__ void add_run(const T* grad, i64 stride, const int2* sorted, int begin, int end, i64 j, float (&sum)[VEC]) {
    int i = begin;
    if (VEC > 1) {
        constexpr int N = 4;
        for (; i + N <= end; i += N) {
            uint4 u[N];
#pragma unroll
            for (int k = 0; k < N; ++k) u[k] = load_once(grad + (i64)sorted[i + k].y * stride + j);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float f[Elem<T>::VEC];
                Elem<T>::unpack(u[k], f);
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] += f[e];
            }
        }
    }
    for (; i < end; ++i) {
        const T* g = grad + (i64)sorted[i].y * stride + j;
        if (VEC > 1) {
            float f[Elem<T>::VEC];
            Elem<T>::unpack(load_once(g), f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += f[e];
        } else {
            sum[0] += Elem<T>::get(*g);
        }
    }
}

// Chunks of ED_CHUNK sorted positions: the sums of the long runs that they cut.  A run longer than a chunk holds the chunk's first or
// its last position wherever it meets one: partial[chunk][0] belongs to the first position's run, [1] to the last one's where that is another.
template <typename T, bool VECTORS>
__global__ void __launch_bounds__(ED_THREADS) embedding_long_kernel(const T* grad, const int2* sorted, const int2* runs, float* partial, i64 count, i64 vocab, i64 dim, i64 stride) {
    pdl_wait(grad, sorted, runs, partial);
    pdl_trigger();
    constexpr int VEC = VECTORS ? Elem<T>::VEC : 1;
    const i64 chunk = blockIdx.x;
    const int c0 = (int)(chunk * ED_CHUNK), c1 = (int)min(chunk * ED_CHUNK + ED_CHUNK, count);
    const int ends[2] = {sorted[c0].x, sorted[c1 - 1].x};
#pragma unroll
    for (int slot = 0; slot < 2; ++slot) {
        const int key = ends[slot];
        if (key >= vocab || (slot == 1 && key == ends[0])) continue;
        const int2 run = runs[key];
        if (run.y - run.x <= ED_CHUNK) continue;
        const int begin = max(run.x, c0), end = min(run.y, c1);
        for (i64 j = (i64)threadIdx.x * VEC; j < dim; j += (i64)ED_THREADS * VEC) {
            float sum[VEC] = {};
            add_run<T, VEC>(grad, stride, sorted, begin, end, j, sum);
            float* p = partial + (chunk * 2 + slot) * dim + j;
#pragma unroll
            for (int e = 0; e < VEC; ++e) p[e] = sum[e];
        }
    }
}

// Every row of the table.
template <typename T, typename O, bool VECTORS>
__global__ void __launch_bounds__(ED_THREADS) embedding_rows_kernel(const T* grad, const int2* sorted, const int2* runs, const float* partial, O* out, i64 dim, i64 stride, i64 out_stride,
                                                                    float scale, int accumulate) {
    pdl_wait(grad, sorted, runs, partial, out);
    pdl_trigger();
    constexpr int VEC = VECTORS ? Elem<T>::VEC : 1;
    const i64 v = blockIdx.x;
    const int2 run = runs[v];
    if (run.x == run.y && accumulate) return;
    for (i64 j = (i64)threadIdx.x * VEC; j < dim; j += (i64)ED_THREADS * VEC) {
        float sum[VEC] = {};
        if (run.y - run.x <= ED_CHUNK) {
            add_run<T, VEC>(grad, stride, sorted, run.x, run.y, j, sum);
        } else {
            for (int chunk = run.x / ED_CHUNK; chunk <= (run.y - 1) / ED_CHUNK; ++chunk) {
                const int slot = chunk * ED_CHUNK < run.x;                // the run's first position is not the chunk's: it is its last run
                const float* p = partial + ((i64)chunk * 2 + slot) * dim + j;
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] += p[e];
            }
        }
        O* o = out + v * out_stride + j;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float r = accumulate ? fmaf(scale, sum[e], Elem<O>::get(o[e])) : scale * sum[e];
            o[e] = Elem<O>::put(r);
        }
    }
}

}  // namespace ef21
