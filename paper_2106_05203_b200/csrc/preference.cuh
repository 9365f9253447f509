// Preference loss: the logistic loss of paired log ratios, with the gradient of every token's log-probability.
//
//   s_r = sum_t m_rt (lp_rt - ref_rt)       z_p = beta (s_p - s_{P+p})
//   loss = 1/N sum_p [ -(1 - eps) log sigma(z_p) - eps log sigma(-z_p) ]
//   d loss / d lp_rt = -+ beta/N (sigma(-z_p) - eps) m_rt       (minus: chosen row p; plus: rejected row P + p)
//
// A pair belongs to one block, which reads its two rows, and writes the gradient -- one value per row -- where the mask holds.  What the mask
// leaves out is not read.
#pragma once
#include "element.cuh"

namespace ef21 {

constexpr int PF_THREADS = 256;

struct PreferenceShape {
    i64 pairs, length;
    i64 logp_stride, ref_stride, mask_stride;
    double beta, smoothing, norm;
    int vectors;                              // rows of all arrays have the same phase against 16 bytes (mask: VEC bytes)
};

// A mask word: VEC bytes, true where not 0.
template <int VEC> struct MaskWord;
template <> struct MaskWord<4> { typedef unsigned type; };
template <> struct MaskWord<8> { typedef unsigned long long type; };

// Calls vec(j) for the vectors and one(j) for the elements around them of a row whose first `head` elements are in front of the first vector.
template <int VEC, typename Vec, typename One>
__device__ __forceinline__ void for_row(i64 head, i64 length, int tid, int threads, Vec vec, One one) {
    if (VEC == 1) {
        for (i64 j = tid; j < length; j += threads) one(j);
        return;
    }
    head = min(head, length);
    const i64 vectors = (length - head) / VEC, tail = head + vectors * VEC;
    if (tid < head) one(tid);
    for (i64 v = tid; v < vectors; v += threads) vec(head + v * VEC);
    if (tail + tid < length) one(tail + tid);
}

// Sum over the block in a fixed order, in every thread; scratch: one double per warp.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* scratch) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) s += scratch[w];
    return s;
}

template <typename T, bool VECTORS>
__global__ void __launch_bounds__(PF_THREADS) preference_kernel(const T* logps, const T* ref, const unsigned char* mask, float* rewards, T* grad, double* partial,
                                                                PreferenceShape s) {
    pdl_wait(logps, ref, mask, rewards, grad, partial);
    pdl_trigger();
    constexpr int VEC = VECTORS ? Elem<T>::VEC : 1;
    typedef typename MaskWord<Elem<T>::VEC>::type Word;
    __shared__ double scratch[PF_THREADS / 32], slope;
    const int tid = threadIdx.x;
    double loss = 0.0;
    for (i64 p = blockIdx.x; p < s.pairs; p += gridDim.x) {
        double total[2];
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const i64 r = p + side * s.pairs;
            const T *a = logps + r * s.logp_stride, *b = ref ? ref + r * s.ref_stride : nullptr;
            const unsigned char* m = mask ? mask + r * s.mask_stride : nullptr;
            double sum = 0.0;
            for_row<VEC>(row_head(a), s.length, tid, PF_THREADS, [&](i64 j) {
                const Word w = m ? *reinterpret_cast<const Word*>(m + j) : ~(Word)0;
                if (w == 0) return;
                float x[Elem<T>::VEC], y[Elem<T>::VEC];
                const uint4 u = load_once(a + j), v = b ? load_once(b + j) : make_uint4(0u, 0u, 0u, 0u);
                Elem<T>::unpack(u, x);
                Elem<T>::unpack(v, y);
                float some = 0.f;
#pragma unroll
                for (int e = 0; e < Elem<T>::VEC; ++e) some += (w >> (8 * e) & 255u) != 0 ? x[e] - y[e] : 0.f;
                sum += (double)some;
            }, [&](i64 j) {
                if (!m || m[j]) sum += (double)(Elem<T>::get(a[j]) - (b ? Elem<T>::get(b[j]) : 0.f));
            });
            total[side] = block_sum<PF_THREADS>(sum, scratch);
        }
        if (tid == 0) {
            const double z = s.beta * (total[0] - total[1]), e = exp(-fabs(z));
            const double low = log1p(e) + fmax(-z, 0.0);                       // -log sigma(z); -log sigma(-z) is larger by z
            const double sigma = (z >= 0.0 ? e : 1.0) / (1.0 + e);             // of -z
            loss += s.smoothing == 0.0 ? low : low + s.smoothing * z;
            slope = s.beta / s.norm * (sigma - s.smoothing);
            rewards[p] = (float)(s.beta * total[0]);
            rewards[p + s.pairs] = (float)(s.beta * total[1]);
        }
        __syncthreads();
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const i64 r = p + side * s.pairs;
            const unsigned char* m = mask ? mask + r * s.mask_stride : nullptr;
            const float value = (float)(side == 0 ? -slope : slope);
            T* g = grad + r * s.length;
            for_row<VEC>(row_head(g), s.length, tid, PF_THREADS, [&](i64 j) {
                const Word w = m ? *reinterpret_cast<const Word*>(m + j) : ~(Word)0;
                float x[Elem<T>::VEC];
#pragma unroll
                for (int e = 0; e < Elem<T>::VEC; ++e) x[e] = (w >> (8 * e) & 255u) != 0 ? value : 0.f;
                store_vec(g + j, Elem<T>::pack(x));
            }, [&](i64 j) { g[j] = Elem<T>::put(!m || m[j] ? value : 0.f); });
        }
        __syncthreads();
    }
    if (tid == 0) partial[blockIdx.x] = loss;
}

// The blocks' losses in their order.
__global__ void __launch_bounds__(PF_THREADS) preference_finish_kernel(const double* partial, float* loss, int blocks, double norm) {
    pdl_wait(partial, loss);
    pdl_trigger();
    __shared__ double scratch[PF_THREADS / 32];
    double v = 0.0;
    for (int b = threadIdx.x; b < blocks; b += PF_THREADS) v += partial[b];
    v = block_sum<PF_THREADS>(v, scratch);
    if (threadIdx.x == 0) *loss = (float)(v / norm);
}

}  // namespace ef21
