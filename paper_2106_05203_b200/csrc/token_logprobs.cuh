// Log-probabilities of given tokens from rows of logits, and the logits' gradient.
//
//   lse_r  = log sum_j exp(s x_rj)          logp_r = s x_r,t(r) - lse_r
//   dx_rj  = s g_r (1[j = t(r)] - exp(s x_rj - lse_r))
//
// Both directions read every logit once; the forward pass carries the running maximum m and the sum of 2^((x - m) c), c = s log2 e.  The maximum
// is subtracted before anything is multiplied: a row that a mask of the type's lowest value leaves nothing of must not overflow.
//
// Gradient of 4,096 x 131,072 bf16: 304 us, 6.7 TB/s read and written, HBM.  Forward pass of 4,088 x 50,257 half, a third of it ignored: 55 to 58 us, 4.9 TB/s.  The exponential
// unit, 16 results per SM and cycle, is busy 75 % of the cycles in which an SM works: 5.15 M warp instructions, 37 of the unit kernel's 55 us at 1,876 MHz; 4.3 M are the
// logits' exponentials, 0.45 M rescalings and warp_merge (ten a lane and unit), the rest what a warp does once.  20 x 32,768: 5 us, a launch.
#pragma once
#include "cluster.cuh"
#include "element.cuh"

namespace ef21 {

struct LogprobShape {
    i64 length, vocab;                      // rows per batch entry, columns
    i64 batch_stride, row_stride;           // logits, in elements
    i64 target_stride;                      // targets per batch entry
    i64 ignore;
    int wide;                               // 64-bit targets
    float scale;
};

constexpr int LP_THREADS = 256;
constexpr int LP_UNROLL = 4;                // vectors of 16 bytes per thread in flight
constexpr int LP_UNIT = 16;                 // vectors per lane of a unit
constexpr int LG_UNROLL = 4;                // the gradient's vectors per thread in flight
constexpr i64 LP_WARP_VOCAB = 2048;         // rows up to this length belong to one warp

// Maximum and sum of 2^((x - m) c) over what a thread has seen; m = -inf: nothing but -inf so far.
struct Running { float m = -INFINITY, s = 0.f; };

__device__ __forceinline__ Running merge(Running a, Running b, float c) {
    Running r;
    r.m = fmaxf(a.m, b.m);
    const float base = r.m == -INFINITY ? 0.f : r.m;
    r.s = a.s * exp2_fast((a.m - base) * c) + b.s * exp2_fast((b.m - base) * c);      // (a NaN stays one; +inf makes one: inf - inf)
    return r;
}

__device__ __forceinline__ Running warp_merge(Running r, float c) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Running other;
        other.m = __shfl_xor_sync(0xffffffffu, r.m, o);
        other.s = __shfl_xor_sync(0xffffffffu, r.s, o);
        r = merge(r, other, c);
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void run_one(const T* x, float c, Running& r) {
    const float v = Elem<T>::get(*x);
    Running one;
    if (v == v) { one.m = v; one.s = v == -INFINITY ? 0.f : 1.f; } else one.s = NAN;
    r = merge(r, one, c);
}

// N vectors.
template <typename T, int N>
__device__ __forceinline__ void run_vectors(const uint4 (&u)[N], float c, Running& r) {
    constexpr int VEC = Elem<T>::VEC;
    float top = Elem<T>::top(u[0]);
#pragma unroll
    for (int k = 1; k < N; ++k) top = fmaxf(top, Elem<T>::top(u[k]));
    const float m = fmaxf(r.m, top), base = m == -INFINITY ? 0.f : m;
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float f[VEC];
        Elem<T>::unpack(u[k], f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e % 2] += exp2_fast((f[e] - base) * c);
    }
    r.s = r.s * exp2_fast((r.m - base) * c) + (sum[0] + sum[1]);
    r.m = m;
}

// Vectors [tid, count) in steps of `threads`, LP_UNROLL at a time.
template <typename T>
__device__ __forceinline__ void run_body(const T* body, int count, float c, int tid, int threads, Running& r) {
    constexpr int VEC = Elem<T>::VEC;
    const int step = threads * LP_UNROLL, whole = count / step * step;
    const T* mine = body + tid * VEC;
    for (int v = 0; v < whole; v += step) {
        uint4 u[LP_UNROLL];
#pragma unroll
        for (int k = 0; k < LP_UNROLL; ++k) u[k] = load_once(mine + ((i64)v + k * threads) * VEC);
        run_vectors<T>(u, c, r);
    }
    if (whole + tid < count) {
        uint4 u[LP_UNROLL];
#pragma unroll
        for (int k = 0; k < LP_UNROLL; ++k) {
            u[k] = make_uint4(Elem<T>::NEG_INF, Elem<T>::NEG_INF, Elem<T>::NEG_INF, Elem<T>::NEG_INF);
            if (whole + tid + k * threads < count) u[k] = load_once(mine + ((i64)whole + k * threads) * VEC);
        }
        run_vectors<T>(u, c, r);
    }
}

// `count` elements from x on, shared by `threads` threads.
template <typename T>
__device__ __forceinline__ Running run_span(const T* x, int count, float c, int tid, int threads) {
    constexpr int VEC = Elem<T>::VEC;
    Running r;
    const int head = min(row_head(x), count), vectors = (count - head) / VEC, tail = count - head - vectors * VEC;
    if (tid < head) run_one(x + tid, c, r);
    if (tid < tail) run_one(x + count - tail + tid, c, r);
    run_body(x + head, vectors, c, tid, threads, r);
    return r;
}

__device__ __forceinline__ void write_logprob(Running r, float xt, bool inside, float scale, float* logp, float* lse) {
    const float l = log2f(r.s);
    if (!inside) { *logp = NAN; *lse = NAN; }
    else if (r.s == 0.f) { *logp = -INFINITY; *lse = -INFINITY; }          // no logit but -inf: no distribution
    else { *logp = fmaf(xt - r.m, scale, -l * LN2); *lse = fmaf(r.m, scale, l * LN2); }
}

template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_warp_kernel(const T* logits, const void* targets, float* logps, float* lse, LogprobShape s, i64 rows) {
    pdl_wait(logits, targets, logps, lse);
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const i64 row = (i64)blockIdx.x * (LP_THREADS / 32) + (threadIdx.x >> 5);
    if (row >= rows) return;
    const i64 b = row / s.length, t = row - b * s.length;
    const i64 target = index_at(targets, s.wide, b * s.target_stride + t);
    if (target == s.ignore) {
        if (lane == 0) { logps[row] = 0.f; lse[row] = 0.f; }
        return;
    }
    const T* x = logits + b * s.batch_stride + t * s.row_stride;
    const bool inside = target >= 0 && target < s.vocab;
    const float xt = inside ? Elem<T>::get(x[target]) : 0.f, c = s.scale * LOG2E;
    const Running r = warp_merge(run_span(x, (int)s.vocab, c, lane, 32), c);
    if (lane == 0) write_logprob(r, xt, inside, s.scale, logps + row, lse + row);
}

// Many long rows: a warp takes LP_UNIT aligned vectors per lane of a row and leaves maximum and sum in part[row][unit]; logprobs_join_kernel has a warp per row, and
// the elements in front of the first and behind the last vector.  Warps wait for nobody, and the last rows do not run alone.
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_unit_kernel(const T* logits, const void* targets, float2* part, LogprobShape s, i64 units, int per_row) {
    pdl_wait(logits, targets, part);
    pdl_trigger();
    constexpr int VEC = Elem<T>::VEC, SPAN = LP_UNIT * 32;
    const int lane = threadIdx.x & 31;
    const i64 unit = (i64)blockIdx.x * (LP_THREADS / 32) + (threadIdx.x >> 5);
    if (unit >= units) return;
    const i64 row = unit / per_row, b = row / s.length, t = row - b * s.length;
    if (index_at(targets, s.wide, b * s.target_stride + t) == s.ignore) return;
    const T* x = logits + b * s.batch_stride + t * s.row_stride;
    const int head = row_head(x), vectors = ((int)s.vocab - head) / VEC, begin = (int)(unit - row * per_row) * SPAN;
    Running r;
    if (begin < vectors) run_body(x + head + (i64)begin * VEC, min(SPAN, vectors - begin), s.scale * LOG2E, lane, 32, r);
    r = warp_merge(r, s.scale * LOG2E);
    if (lane == 0) part[unit] = make_float2(r.m, r.s);
}

template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_join_kernel(const T* logits, const void* targets, const float2* part, float* logps, float* lse, LogprobShape s, i64 rows, int per_row) {
    pdl_wait(logits, targets, part, logps, lse);
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const i64 row = (i64)blockIdx.x * (LP_THREADS / 32) + (threadIdx.x >> 5);
    if (row >= rows) return;
    const i64 b = row / s.length, t = row - b * s.length;
    const i64 target = index_at(targets, s.wide, b * s.target_stride + t);
    if (target == s.ignore) {
        if (lane == 0) { logps[row] = 0.f; lse[row] = 0.f; }
        return;
    }
    const bool inside = target >= 0 && target < s.vocab;
    const T* x = logits + b * s.batch_stride + t * s.row_stride;
    const float xt = inside ? Elem<T>::get(x[target]) : 0.f, c = s.scale * LOG2E;
    const int head = row_head(x), behind = head + ((int)s.vocab - head) / Elem<T>::VEC * Elem<T>::VEC;
    Running r;
    if (lane < head) run_one(x + lane, c, r);
    if (behind + lane < (int)s.vocab) run_one(x + behind + lane, c, r);
    for (int u = lane; u < per_row; u += 32) {
        const float2 p = part[row * per_row + u];
        Running one;
        one.m = p.x; one.s = p.y;
        r = merge(r, one, c);
    }
    r = warp_merge(r, c);
    if (lane == 0) write_logprob(r, xt, inside, s.scale, logps + row, lse + row);
}

// One cluster per row, its blocks an equal share of the columns each.
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_block_kernel(const T* logits, const void* targets, float* logps, float* lse, LogprobShape s, unsigned C) {
    pdl_wait(logits, targets, logps, lse);
    pdl_trigger();
    __shared__ Running part[LP_THREADS / 32], whole;
    const int tid = threadIdx.x;
    const i64 row = blockIdx.x / C;
    const unsigned rank = blockIdx.x - (unsigned)row * C;
    const i64 b = row / s.length, t = row - b * s.length;
    const i64 target = index_at(targets, s.wide, b * s.target_stride + t);
    if (target == s.ignore) {                                  // (all blocks of the cluster alike)
        if (tid == 0 && rank == 0) { logps[row] = 0.f; lse[row] = 0.f; }
        return;
    }
    const T* x = logits + b * s.batch_stride + t * s.row_stride;
    const bool inside = target >= 0 && target < s.vocab;
    const float c = s.scale * LOG2E;
    const float xt = inside && tid == 0 && rank == 0 ? Elem<T>::get(x[target]) : 0.f;
    const i64 share = (s.vocab + C - 1) / C, begin = min(rank * share, s.vocab), end = min(begin + share, s.vocab);
    Running r = warp_merge(run_span(x + begin, (int)(end - begin), c, tid, LP_THREADS), c);
    if ((tid & 31) == 0) part[tid >> 5] = r;
    __syncthreads();
    if (tid < 32) {
        Running w;
        if (tid < LP_THREADS / 32) w = part[tid];
        r = warp_merge(w, c);
    }
    if (C > 1) {
        if (tid == 0) whole = r;
        cluster_barrier();
        if (rank == 0 && tid < 32) {
            Running w;
            if (tid < (int)C) { w.m = remote_float(&whole.m, tid); w.s = remote_float(&whole.s, tid); }
            r = warp_merge(w, c);
        }
        cluster_barrier();                                     // nobody leaves while it is read
    }
    if (tid == 0 && rank == 0) write_logprob(r, xt, inside, s.scale, logps + row, lse + row);
}

// What the gradient of one row needs: dx_j = a 1[j = target] - a exp(scale x_j - lse).
struct RowGrad {
    float a, scale, lse;
    i64 target;
    bool zero;
};

__device__ __forceinline__ RowGrad row_grad(const void* targets, const float* lse, const float* grad, const LogprobShape& s, i64 row, i64 b, i64 t) {
    RowGrad r;
    r.target = index_at(targets, s.wide, b * s.target_stride + t);
    const float l = lse[row];
    r.a = grad[row] * s.scale;
    r.scale = s.scale;
    r.zero = r.target == s.ignore || grad[row] == 0.f || l == -INFINITY;
    r.lse = r.target >= 0 && r.target < s.vocab ? l : NAN;
    return r;
}

// Columns [begin, end) of one row.
template <typename T>
__device__ __forceinline__ void grad_span(const T* x, T* out, i64 begin, i64 end, const RowGrad& r, int tid, int threads) {
    constexpr int VEC = Elem<T>::VEC;
    auto value = [&](float f, i64 j) {
        const float p = r.a * exp2_fast(fmaf(f, r.scale, -r.lse) * LOG2E);
        return j == r.target ? r.a - p : -p;
    };
    auto gradient = [&](uint4 u, i64 j) {                              // of the vector at j
        float f[VEC];
        Elem<T>::unpack(u, f);
        const bool named = r.target >= j && r.target < j + VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = -r.a * exp2_fast(fmaf(f[e], r.scale, -r.lse) * LOG2E);
        if (named) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) if (j + e == r.target) f[e] += r.a;
        }
        return Elem<T>::pack(f);
    };
    auto one = [&](i64 j) { out[j] = Elem<T>::put(r.zero ? 0.f : value(Elem<T>::get(x[j]), j)); };
    const i64 head = min((i64)row_head(out + begin), end - begin), vectors = (end - begin - head) / VEC, tail = end - begin - head - vectors * VEC;
    if (tid < head) one(begin + tid);
    if (tid < tail) one(end - tail + tid);
    const i64 body = begin + head;
    if (row_head(x + begin) != row_head(out + begin) && !r.zero) {       // logits of another alignment
        constexpr int N = 2;
        for (i64 v = tid; v - (tid & 31) < vectors; v += (i64)threads * N) {
            const void* p[N];
            bool in[N], last[N];
            uint4 u[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const i64 at = v + (i64)k * threads;
                p[k] = x + body + at * VEC; in[k] = at < vectors; last[k] = at + 1 == vectors;
            }
            load_unaligned<N>(p, in, last, u);
#pragma unroll
            for (int k = 0; k < N; ++k) if (in[k]) store_vec(out + body + (v + (i64)k * threads) * VEC, gradient(u[k], body + (v + (i64)k * threads) * VEC));
        }
        return;
    }
    for (i64 v = tid; v < vectors; v += (i64)threads * LG_UNROLL) {
        uint4 u[LG_UNROLL];
#pragma unroll
        for (int k = 0; k < LG_UNROLL; ++k) {
            const i64 at = v + (i64)k * threads;
            if (at < vectors && !r.zero) u[k] = load_once(x + body + at * VEC);
        }
#pragma unroll
        for (int k = 0; k < LG_UNROLL; ++k) {
            const i64 at = v + (i64)k * threads, j = body + at * VEC;
            if (at >= vectors) break;
            if (r.zero) { store_vec(out + j, make_uint4(0u, 0u, 0u, 0u)); continue; }
            store_vec(out + j, gradient(u[k], j));
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_grad_warp_kernel(const T* logits, const void* targets, const float* lse, const float* grad, T* out,
                                                                        LogprobShape s, i64 out_batch_stride, i64 out_row_stride, i64 rows) {
    pdl_wait(logits, targets, lse, grad, out);
    pdl_trigger();
    const i64 row = (i64)blockIdx.x * (LP_THREADS / 32) + (threadIdx.x >> 5);
    if (row >= rows) return;
    const i64 b = row / s.length, t = row - b * s.length;
    const RowGrad r = row_grad(targets, lse, grad, s, row, b, t);
    grad_span(logits + b * s.batch_stride + t * s.row_stride, out + b * out_batch_stride + t * out_row_stride, 0, s.vocab, r, threadIdx.x & 31, 32);
}

// One block per slab of a row's columns.
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_grad_block_kernel(const T* logits, const void* targets, const float* lse, const float* grad, T* out,
                                                                         LogprobShape s, i64 out_batch_stride, i64 out_row_stride, unsigned slabs, i64 slab) {
    pdl_wait(logits, targets, lse, grad, out);
    pdl_trigger();
    const i64 row = blockIdx.x / slabs, at = (i64)(blockIdx.x - (unsigned)row * slabs) * slab;
    const i64 b = row / s.length, t = row - b * s.length;
    const RowGrad r = row_grad(targets, lse, grad, s, row, b, t);
    grad_span(logits + b * s.batch_stride + t * s.row_stride, out + b * out_batch_stride + t * out_row_stride, at, min(at + slab, s.vocab), r, threadIdx.x, LP_THREADS);
}

}  // namespace ef21
