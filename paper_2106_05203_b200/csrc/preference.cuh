// Preference loss: the logistic loss of paired log ratios, with the gradient of every token's log-probability.
//
//   s_r = sum_t m_rt (lp_rt - ref_rt)       z_p = beta (s_p - s_{P+p})
//   loss = 1/N sum_p [ -(1 - eps) log sigma(z_p) - eps log sigma(-z_p) ]
//   d loss / d lp_rt = -+ beta/N (sigma(-z_p) - eps) m_rt       (minus: chosen row p; plus: rejected row P + p)
//
// 512 pairs x 8,191 fp32: 20.6 us, 5.3 TB/s of what is there (4.1 of what is read and written), two reductions between reading and writing; 4 pairs x 512: 6.9 us, a launch.
//
// What the mask leaves out is not read; the gradient -- one value per row -- is written where it holds.  Short rows: a warp has a pair, a block eight.  Longer
// ones: a pair has one block, or up to eight that form a cluster and add up their sums; PF_PART elements are one vector of 16 bytes (fp32) per thread, so that both rows'
// loads are on their way at once.  Where all blocks fit one cluster it writes the loss as well, otherwise a second kernel adds up the pairs'.
#pragma once
#include <type_traits>

#include "cluster.cuh"
#include "element.cuh"

namespace ef21 {

constexpr int PF_THREADS = 256;
constexpr int PF_FINISH_THREADS = 1024;
constexpr i64 PF_PART = 1024;
constexpr i64 PF_WARP_LENGTH = 256;           // rows up to this length: a warp per pair
constexpr unsigned PF_CLUSTER = 8;

struct PreferenceShape {
    i64 pairs, length;
    i64 logp_stride, ref_stride, mask_stride;
    double beta, smoothing, norm;
    unsigned split;                           // blocks per pair
    int one;                                  // all blocks are one cluster
};

// A mask word: VEC bytes, true where not 0.
template <int VEC> struct MaskWord;
template <> struct MaskWord<4> { typedef unsigned type; };
template <> struct MaskWord<8> { typedef unsigned long long type; };

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

// Elements [begin, end) of a row, of which [body, body + vectors * VEC) are whole aligned vectors.
struct RowPart { i64 begin, body, end, vectors; };

// Part `part` of `parts` of a row whose first `head` elements are in front of its first aligned vector.
template <int VEC>
__device__ __forceinline__ RowPart row_part(i64 length, i64 head, unsigned part, unsigned parts) {
    const i64 chunk = (length + (i64)parts * 8 - 1) / ((i64)parts * 8) * 8;          // (whole vectors of any type)
    RowPart r;
    r.begin = part == 0 ? 0 : min(head + part * chunk, length);
    r.end = part + 1 == parts ? length : min(head + (part + 1) * chunk, length);
    r.body = part == 0 ? min(head, r.end) : r.begin;
    r.vectors = (r.end - r.body) / VEC;
    return r;
}

// A token's log ratio: rounded once in 32 bits, and in 64 where it is beyond them (the lowest value on one side, the largest on the other).
__device__ __forceinline__ double log_ratio(float logp, float ref) {
    const float d = logp - ref;
    return fabsf(d) <= 3.4028234e38f ? (double)d : (double)logp - (double)ref;
}

template <typename T, bool VECTORS, int TEAM>
__global__ void __launch_bounds__(PF_THREADS) preference_kernel(const T* logps, const T* ref, const unsigned char* mask, float* rewards, T* grad, double* partial, float* loss_out,
                                                                PreferenceShape s) {
    pdl_wait(logps, ref, mask, rewards, grad, partial, loss_out);
    pdl_trigger();
    constexpr int VEC = VECTORS ? Elem<T>::VEC : 1;
    typedef typename std::conditional<VECTORS, typename MaskWord<Elem<T>::VEC>::type, unsigned char>::type Word;
    __shared__ double scratch[PF_THREADS / 32], sums[2], slope_of_block, losses;
    const int tid = threadIdx.x, lane = tid & (TEAM - 1);
    const i64 p = TEAM == 32 ? (i64)blockIdx.x * (PF_THREADS / 32) + (tid >> 5) : (i64)(blockIdx.x / s.split);
    const unsigned part = TEAM == 32 ? 0u : blockIdx.x % s.split, parts = TEAM == 32 ? 1u : s.split;
    const bool there = p < s.pairs;                               // (a cluster's blocks stay for its barriers)
    const T *a[2], *b[2];
    const unsigned char* m[2];
    T* g[2];
    RowPart r[2];
    double sum[2] = {0.0, 0.0};
    Word first[2] = {};
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const i64 row = there ? p + side * s.pairs : 0;
        a[side] = logps + row * s.logp_stride;
        b[side] = ref ? ref + row * s.ref_stride : nullptr;
        m[side] = mask ? mask + row * s.mask_stride : nullptr;
        g[side] = grad + row * s.length;
        r[side] = row_part<VEC>(there ? s.length : 0, VECTORS ? (i64)row_head(a[side]) : 0, part, parts);
    }
    const i64 rounds = max(r[0].vectors, r[1].vectors);
    auto word = [&](int side, i64 v) {
        return v >= r[side].vectors ? (Word)0 : m[side] ? *reinterpret_cast<const Word*>(m[side] + r[side].body + v * VEC) : (Word)~(Word)0;
    };
    Word next[2] = {word(0, lane), word(1, lane)};
    first[0] = next[0]; first[1] = next[1];
    for (i64 v = lane; v < rounds; v += TEAM) {
        const Word w[2] = {next[0], next[1]};
        next[0] = word(0, v + TEAM); next[1] = word(1, v + TEAM);      // (on its way while this round's log-probabilities are)
        if constexpr (VECTORS) {
            uint4 x[2], y[2];
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                if (w[side] == 0) continue;
                x[side] = load_once(a[side] + r[side].body + v * VEC);
                y[side] = b[side] ? load_once(b[side] + r[side].body + v * VEC) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                if (w[side] == 0) continue;
                float fx[VEC], fy[VEC], some = 0.f;
                Elem<T>::unpack(x[side], fx);
                Elem<T>::unpack(y[side], fy);
#pragma unroll
                for (int e = 0; e < VEC; ++e) some += (w[side] >> (8 * e) & 255u) != 0 ? fx[e] - fy[e] : 0.f;
                if (!(fabsf(some) <= 3.4028234e38f)) {                // (lowest values of a mask: their sum is beyond 32 bits, each is not)
                    double exact = 0.0;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) exact += (w[side] >> (8 * e) & 255u) != 0 ? (double)fx[e] - (double)fy[e] : 0.0;
                    sum[side] += exact;
                } else {
                    sum[side] += (double)some;
                }
            }
        } else {
#pragma unroll
            for (int side = 0; side < 2; ++side)
                if (w[side]) sum[side] += log_ratio(Elem<T>::get(a[side][r[side].body + v]), b[side] ? Elem<T>::get(b[side][r[side].body + v]) : 0.f);
        }
    }
    auto ends = [&](int side, auto one) {                          // the elements around the vectors: fewer than a team
        const RowPart& q = r[side];
        if (q.begin + lane < q.body) one(q.begin + lane);
        if (q.body + q.vectors * VEC + lane < q.end) one(q.body + q.vectors * VEC + lane);
    };
    if (VECTORS) {
#pragma unroll
        for (int side = 0; side < 2; ++side)
            ends(side, [&](i64 j) { if (!m[side] || m[side][j]) sum[side] += log_ratio(Elem<T>::get(a[side][j]), b[side] ? Elem<T>::get(b[side][j]) : 0.f); });
    }
    if (TEAM == 32) {
        sum[0] = warp_sum(sum[0]); sum[1] = warp_sum(sum[1]);
    } else {
        sum[0] = block_sum<PF_THREADS>(sum[0], scratch);
        sum[1] = block_sum<PF_THREADS>(sum[1], scratch);
        if (parts > 1) {                                           // the pair's blocks follow one another in the cluster
            if (tid == 0) { sums[0] = sum[0]; sums[1] = sum[1]; }
            cluster_barrier();
            if (tid == 0) {
                const unsigned base = cluster_rank() - part;
                sum[0] = sum[1] = 0.0;
                for (unsigned q = 0; q < parts; ++q) { sum[0] += remote_double(&sums[0], base + q); sum[1] += remote_double(&sums[1], base + q); }
            }
        }
    }
    double loss = 0.0;
    float slope = 0.f;
    if (lane == 0 && there) {
        const double z = s.beta * (sum[0] - sum[1]), e = exp(-fabs(z));
        const double low = log1p(e);                                           // -log sigma(|z|); -log sigma(-|z|) is larger by |z|
        const double sigma = (z >= 0.0 ? e : 1.0) / (1.0 + e);                 // of -z
        slope = (float)(s.beta / s.norm * (sigma - s.smoothing));
        if (part == 0) {
            const double share = z < 0.0 ? 1.0 - s.smoothing : s.smoothing;
            loss = share == 0.0 ? low : low + share * fabs(z);
            rewards[p] = (float)(s.beta * sum[0]);
            rewards[p + s.pairs] = (float)(s.beta * sum[1]);
        }
    }
    if (TEAM == 32) {
        slope = __shfl_sync(0xffffffffu, slope, 0);
    } else {
        if (tid == 0) slope_of_block = (double)slope;
        __syncthreads();
        slope = (float)slope_of_block;
    }
    for (i64 v = lane; v < rounds; v += TEAM) {
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            if (v >= r[side].vectors) continue;
            const float value = side == 0 ? -slope : slope;
            const i64 j = r[side].body + v * VEC;
            const Word w = v == lane ? first[side] : m[side] ? *reinterpret_cast<const Word*>(m[side] + j) : (Word)~(Word)0;
            if constexpr (VECTORS) {
                float x[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[e] = (w >> (8 * e) & 255u) != 0 ? value : 0.f;
                store_vec(g[side] + j, Elem<T>::pack(x));
            } else {
                g[side][j] = Elem<T>::put(w ? value : 0.f);
            }
        }
    }
    if (VECTORS) {
#pragma unroll
        for (int side = 0; side < 2; ++side)
            ends(side, [&](i64 j) { g[side][j] = Elem<T>::put(!m[side] || m[side][j] ? (side == 0 ? -slope : slope) : 0.f); });
    }
    if (TEAM == 32) loss = block_sum<PF_THREADS>(lane == 0 ? loss : 0.0, scratch);
    if (s.one) {
        double all[1] = {loss};
        cluster_sums(all, &losses);
        if (tid == 0 && cluster_rank() == 0) *loss_out = (float)(all[0] / s.norm);
    } else {
        if (tid == 0 && part == 0) partial[blockIdx.x / parts] = loss;
        if (parts > 1) cluster_barrier();                          // the sums have been read
    }
}

// The pairs' (or blocks') losses in their order.
__global__ void __launch_bounds__(PF_FINISH_THREADS) preference_finish_kernel(const double* partial, float* loss, i64 count, double norm) {
    pdl_wait(partial, loss);
    pdl_trigger();
    __shared__ double scratch[PF_FINISH_THREADS / 32];
    double v = 0.0;
    for (i64 b = threadIdx.x; b < count; b += PF_FINISH_THREADS) v += partial[b];
    v = block_sum<PF_FINISH_THREADS>(v, scratch);
    if (threadIdx.x == 0) *loss = (float)(v / norm);
}

}  // namespace ef21
