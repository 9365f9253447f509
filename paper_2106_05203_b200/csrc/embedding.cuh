// Rows of a table by token, scaled, and the table's gradient: for every token the sum of the gradients at its positions, in ascending order of the
// positions, in 32 bits, rounded once.
//
//   out_t = s W[tok_t]          dW_v = s sum_{t: tok_t = v} g_t
//
// The gradient is no scatter (float atomics add in any order): positions are sorted by token (stable); then every row of the table that
// has at most ED_CHUNK positions is formed by the lanes of one team and written once, zeros where no token names it, while other blocks of the same
// launch add up the longer runs ED_CHUNK sorted positions at a time; a last launch joins these sums, in order.
//
// Lookup of 16,384 x 4,096 bf16: 32.5 us, 5.9 TB/s.  Gradient of 65,536 tokens (the most frequent 6,000 times) into 50,257 x 2,048 fp32: 167 us as
// dependent launches; each by itself, caches warm: the seven of the sort 39, the sums 138 (269 MB read, 373 written while it runs: 4.7 TB/s; 80 registers, 44 / 84 bytes of spills), the
// join 15.  1,000 tokens into 1,024 x 257 fp32: 10.5 us; 3,000 into 10,000 x 64 half 19, 8,000 into 500 x 40 bf16 23 (24 and 28 with two positions in flight, as large tables
// have).  Rows that are no whole vectors move by single elements: 60,000 bf16 tokens into 98,621 x 917 fp32 425, six times its bytes.
//
// Sorting: up to ED_RANK_TOKENS tokens by counting, for every token, those in front of it -- one launch; more by a radix sort, digits of up to nine bits, three launches
// each.  (All passes in the shared memory of one cluster were measured, too: 4 us faster at 9,000 tokens, as fast at 30,000, 10 us slower at 65,000.)
#pragma once
#include <type_traits>

#include "element.cuh"

namespace ef21 {

constexpr int ED_THREADS = 256;
constexpr int ED_SUM_THREADS = 64;          // (a block keeps its place until its slowest team is done)
constexpr int ED_CHUNK = 32;                // sorted positions that one team adds up
constexpr int ED_VECS = 2;                  // vectors per lane and row
constexpr int ED_SINGLES = 2, ED_MANY_SINGLES = 4;   // elements per lane and row where rows are no whole vectors: with eight positions in flight, with four
constexpr int ED_ROW_VECS = 4, ED_SHORT = 512;
constexpr int ED_JOIN_THREADS = 512, ED_SHARES = ED_JOIN_THREADS / 32;
constexpr int ED_ROWS = 4;                  // rows of the table per team where that leaves enough teams
constexpr int ED_RANK_TOKENS = 4096;
constexpr int ED_RANK_THREADS = 256;
constexpr int RX_THREADS = 1024, RX_TILE = RX_THREADS, RX_MAX_BITS = 9, RX_WARPS = RX_THREADS / 32;       // an item a thread

// ---- lookup -------------------------------------------------------------------------------------------------------------------------------

// A warp takes ED_ROW_VECS times 32 vectors of one row.  ALIGNED: rows of the table and of the output are whole aligned vectors; otherwise vectors are those of the output, and
// the first and the last warp of a row write the elements around them.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(ED_THREADS) embedding_kernel(const T* weight, const void* tokens, T* out, i64 items, int slabs, i64 vocab, i64 dim, i64 stride, int wide, float scale) {
    pdl_wait(weight, tokens, out);
    pdl_trigger();
    constexpr int VEC = Elem<T>::VEC;
    const i64 item = (i64)blockIdx.x * (ED_THREADS / 32) + (threadIdx.x >> 5);
    if (item >= items) return;
    const int lane = threadIdx.x & 31;
    const i64 t = slabs == 1 ? item : item / slabs;
    const int slab = (int)(item - t * slabs);
    const i64 v = index_at(tokens, wide, t);
    const bool in = v >= 0 && v < vocab;
    const T* row = weight + (in ? v : 0) * stride;
    T* o = out + t * dim;
    const i64 head = ALIGNED ? 0 : min((i64)row_head(o), dim), vectors = (dim - head) / VEC, first = (i64)slab * (32 * ED_ROW_VECS) + lane;
    uint4 u[ED_ROW_VECS];
    if (ALIGNED) {
#pragma unroll
        for (int k = 0; k < ED_ROW_VECS; ++k)
            u[k] = in && first + k * 32 < vectors ? *reinterpret_cast<const uint4*>(row + (first + k * 32) * VEC) : make_uint4(0u, 0u, 0u, 0u);
    } else {
        const void* p[ED_ROW_VECS];
        bool there[ED_ROW_VECS], last[ED_ROW_VECS];
#pragma unroll
        for (int k = 0; k < ED_ROW_VECS; ++k) {
            p[k] = row + head + (first + k * 32) * VEC;
            there[k] = in && first + k * 32 < vectors; last[k] = first + k * 32 + 1 == vectors;
        }
        load_unaligned<ED_ROW_VECS>(p, there, last, u);
        auto one = [&](i64 j) { o[j] = Elem<T>::put(in ? Elem<T>::get(row[j]) * scale : 0.f); };
        if (slab == 0 && lane < head) one(lane);
        if (slab == slabs - 1 && head + vectors * VEC + lane < dim) one(head + vectors * VEC + lane);
    }
#pragma unroll
    for (int k = 0; k < ED_ROW_VECS; ++k) {
        float f[VEC];
        Elem<T>::unpack(u[k], f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = in ? f[e] * scale : 0.f;
        if (first + k * 32 < vectors) store_vec(o + head + (first + k * 32) * VEC, Elem<T>::pack(f));
    }
}

// Short rows that are no whole aligned vectors (up to ED_SHORT elements): a warp has a row.
template <typename T>
__global__ void __launch_bounds__(ED_THREADS) embedding_short_kernel(const T* weight, const void* tokens, T* out, i64 count, i64 vocab, i64 dim, i64 stride, int wide, float scale) {
    pdl_wait(weight, tokens, out);
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const i64 t = (i64)blockIdx.x * (ED_THREADS / 32) + (threadIdx.x >> 5);
    if (t >= count) return;
    const i64 v = index_at(tokens, wide, t);
    const bool in = v >= 0 && v < vocab;
    const T* row = weight + (in ? v : 0) * stride;
    float f[ED_SHORT / 32];
#pragma unroll
    for (int k = 0; k < ED_SHORT / 32; ++k) f[k] = in && lane + k * 32 < dim ? Elem<T>::get(row[lane + k * 32]) : 0.f;
#pragma unroll
    for (int k = 0; k < ED_SHORT / 32; ++k) if (lane + k * 32 < dim) out[t * dim + lane + k * 32] = Elem<T>::put(in ? f[k] * scale : 0.f);
}

// ---- sorting positions by token -------------------------------------------------------------------------------------------------------------

// A token that has a row and a gradient, else `vocab` (sorted behind all others and left there).
__device__ __forceinline__ int token_key(const void* tokens, int wide, i64 i, i64 vocab, i64 padding) {
    const i64 v = index_at(tokens, wide, i);
    return v >= 0 && v < vocab && v != padding ? (int)v : (int)vocab;
}

// Few tokens: the place of each is the number of smaller ones plus that of equal ones before it -- of those not larger in front of it and of smaller ones behind it.  A
// warp takes one token at a time.
__global__ void __launch_bounds__(ED_RANK_THREADS) embedding_rank_kernel(const void* tokens, int wide, int count, i64 vocab, i64 padding, int2* sorted, int2* runs) {
    pdl_wait(tokens, sorted, runs);
    pdl_trigger();
    extern __shared__ __align__(16) int keys[];
    const int lane = threadIdx.x & 31, padded = (count + 127) / 128 * 128;
    for (int base = threadIdx.x; base < padded; base += 8 * ED_RANK_THREADS) {
        int key[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = base + k * ED_RANK_THREADS;
            key[k] = i < count ? token_key(tokens, wide, i, vocab, padding) : 0x7fffffff;                  // (above every token)
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) if (base + k * ED_RANK_THREADS < padded) keys[base + k * ED_RANK_THREADS] = key[k];
    }
    __syncthreads();
    for (int i = blockIdx.x * (ED_RANK_THREADS / 32) + (threadIdx.x >> 5); i < count; i += gridDim.x * (ED_RANK_THREADS / 32)) {
        const int key = keys[i], own = i / 4;
        int less = 0, up_to = 0, place = 0;                               // smaller ones, and those not larger
#pragma unroll 4
        for (int j = lane; j < padded / 4; j += 32) {
            const int4 v = *reinterpret_cast<const int4*>(keys + j * 4);
            const int low = (v.x < key) + (v.y < key) + (v.z < key) + (v.w < key), up = (v.x <= key) + (v.y <= key) + (v.z <= key) + (v.w <= key);
            less += low; up_to += up; place += j < own ? up : low;
        }
        if (lane < i - own * 4) place += keys[own * 4 + lane] == key;     // (in front of it among its own four)
        place = __reduce_add_sync(0xffffffffu, place);
        less = __reduce_add_sync(0xffffffffu, less);
        up_to = __reduce_add_sync(0xffffffffu, up_to);
        if (lane == 0) {
            sorted[place] = make_int2(key, i);
            if (place == less && key < vocab) runs[key] = make_int2(less, up_to);
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
    const i64 i = (i64)blockIdx.x * RX_TILE + threadIdx.x;
    if (i < count) atomicAdd(&here[(radix_item(source, tokens, wide, i, vocab, padding).x >> shift) & (bins - 1)], 1);
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

// How many items of the same digit a warp has in front of a lane's (digit -1: no item).  of_warp[digit] becomes the number of all of them.
__device__ __forceinline__ int radix_rank(int digit, unsigned short* of_warp, int bits) {
    const int lane = threadIdx.x & 31;
    // lanes with the same digit, bit by bit (a ballot each: the match instruction takes several times as long)
    unsigned peers = __ballot_sync(0xffffffffu, digit >= 0);
    for (int b = 0; b < bits; ++b) {
        const bool one = digit >> b & 1;
        const unsigned ones = __ballot_sync(0xffffffffu, one);
        peers &= one ? ones : ~ones;
    }
    const int ahead = __popc(peers & ((1u << lane) - 1u));
    if (digit >= 0 && ahead == 0) of_warp[digit] = (unsigned short)__popc(peers);
    return ahead;
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
    const i64 i = (i64)blockIdx.x * RX_TILE + tid;
    const bool in = i < count;
    const int2 item = in ? radix_item(source, tokens, wide, i, vocab, padding) : make_int2(0, 0);
    const int digit = in ? (item.x >> shift) & (bins - 1) : -1;
    __syncwarp();
    const int rank = radix_rank(digit, warp_count[warp], bits);
    __syncthreads();
    for (int b = tid; b < bins; b += RX_THREADS) {
        int sum = 0;
        for (int w = 0; w < RX_WARPS; ++w) { const int v = warp_count[w][b]; warp_count[w][b] = (unsigned short)sum; sum += v; }
    }
    __syncthreads();
    if (in) target[place[digit] + warp_count[warp][digit] + rank] = item;
}

// The run of every token that is there.  (The other entries of runs are never written: who reads one looks whether the position it names holds the token.)
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

struct TableShape {
    i64 count, vocab, dim, stride, out_stride;
    float scale;
    int accumulate;
    int lanes, slabs;                       // lanes of a team (a power of two); teams side by side that cover a row
    unsigned long_blocks;                   // blocks that add up chunks of long runs; the others form rows
    int by_run;                             // rows by their runs: only those that tokens name (zeros have been written, or are not wanted: always where the sums are added to what is there)
};

template <int VEC> __device__ __forceinline__ void put_floats(float* p, const float (&f)[VEC]) {
    if constexpr (VEC == 8)
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7])
                     : "memory");
    else if constexpr (VEC == 4)
        *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    else
        *p = f[0];
}
template <int VEC> __device__ __forceinline__ void get_floats(const float* p, float (&f)[VEC]) {
    if constexpr (VEC == 1) {
        f[0] = *p;
    } else {
#pragma unroll
        for (int e = 0; e < VEC; e += 4) {
            const float4 v = *reinterpret_cast<const float4*>(p + e);
            f[e] = v.x; f[e + 1] = v.y; f[e + 2] = v.z; f[e + 3] = v.w;
        }
    }
}

// VEC elements of a row of the table: 16 bytes, or 32 (fp32 from 16-bit gradients), or one element.
template <typename O, int VEC> __device__ __forceinline__ void put_elements(O* o, const float (&f)[VEC]) {
    if constexpr (sizeof(O) == 4) put_floats<VEC>(o, f);
    else if constexpr (VEC == Elem<O>::VEC) store_vec(o, Elem<O>::pack(f));
    else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = Elem<O>::put(f[e]);
    }
}

// The columns of one lane: VECS vectors, a team's lanes side by side.
template <int VEC, int VECS>
struct Columns {
    i64 first, step, dim;
    __device__ __forceinline__ Columns(const TableShape& s, int slab, int lane) : first(((i64)slab * VECS * s.lanes + lane) * VEC), step((i64)s.lanes * VEC), dim(s.dim) {}
    __device__ __forceinline__ i64 at(int k) const { return first + k * step; }
    __device__ __forceinline__ bool in(int k) const { return at(k) < dim; }
};

// Sums over sorted positions [begin, end), in order.  MANY teams and 16-bit vectors: two at a time, what is left over alone (registers; whatever else was tried costs the
// large table 3 %).  Others: four or eight at a time, the next ones' places looked up meanwhile -- small tables wait for the longest run.
template <bool MANY, typename T, int VEC, int VECS>
__device__ __forceinline__ void add_run(const T* grad, i64 stride, const int2* sorted, int begin, int end, const Columns<VEC, VECS>& c, float (&sum)[VECS][VEC]) {
    if constexpr (VEC == 8 && MANY) {
        auto two_or_one = [&](int i, auto n) {
            constexpr int N = decltype(n)::value;
            const T* g[N];
#pragma unroll
            for (int p = 0; p < N; ++p) g[p] = grad + (i64)sorted[i + p].y * stride;
            uint4 u[N][VECS];
#pragma unroll
            for (int p = 0; p < N; ++p)
#pragma unroll
                for (int k = 0; k < VECS; ++k) if (c.in(k)) u[p][k] = load_once(g[p] + c.at(k));
#pragma unroll
            for (int p = 0; p < N; ++p)
#pragma unroll
                for (int k = 0; k < VECS; ++k) {
                    float f[Elem<T>::VEC];
                    Elem<T>::unpack(u[p][k], f);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[k][e] += f[e];
                }
        };
        int i = begin;
        for (; i + 2 <= end; i += 2) two_or_one(i, std::integral_constant<int, 2>{});
        if (i < end) two_or_one(i, std::integral_constant<int, 1>{});
        return;
    }
    constexpr int N = MANY ? 4 : 8;
    int at[N];
#pragma unroll
    for (int p = 0; p < N; ++p) at[p] = begin + p < end ? sorted[begin + p].y : 0;
    for (int i = begin; i < end; i += N) {
        if constexpr (VEC > 1) {
            uint4 u[N][VECS];
#pragma unroll
            for (int p = 0; p < N; ++p)
#pragma unroll
                for (int k = 0; k < VECS; ++k) {
                    u[p][k] = make_uint4(0u, 0u, 0u, 0u);
                    if (i + p < end && c.in(k)) u[p][k] = load_once(grad + (i64)at[p] * stride + c.at(k));
                }
#pragma unroll
            for (int p = 0; p < N; ++p) at[p] = i + N + p < end ? sorted[i + N + p].y : 0;
#pragma unroll
            for (int p = 0; p < N; ++p)
#pragma unroll
                for (int k = 0; k < VECS; ++k) {
                    float f[Elem<T>::VEC];
                    Elem<T>::unpack(u[p][k], f);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[k][e] += f[e];
                }
        } else {
            float f[N][VECS];
#pragma unroll
            for (int p = 0; p < N; ++p)
#pragma unroll
                for (int k = 0; k < VECS; ++k) f[p][k] = i + p < end && c.in(k) ? Elem<T>::get(grad[(i64)at[p] * stride + c.at(k)]) : 0.f;
#pragma unroll
            for (int p = 0; p < N; ++p) at[p] = i + N + p < end ? sorted[i + N + p].y : 0;
#pragma unroll
            for (int p = 0; p < N; ++p)
#pragma unroll
                for (int k = 0; k < VECS; ++k) sum[k][0] += f[p][k];
        }
    }
}

// A row's first gradient on its way; zeros where there is none.
template <typename T, int VEC, int VECS>
struct First {
    typedef typename std::conditional<(VEC > 1), uint4, float>::type Raw;
    Raw raw[VECS];
    __device__ __forceinline__ void fetch(const T* g, const Columns<VEC, VECS>& c, bool there) {
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            if constexpr (VEC > 1) raw[k] = there && c.in(k) ? load_once(g + c.at(k)) : make_uint4(0u, 0u, 0u, 0u);
            else raw[k] = there && c.in(k) ? Elem<T>::get(g[c.at(k)]) : 0.f;
        }
    }
    __device__ __forceinline__ void take(float (&sum)[VECS][VEC]) const {
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            if constexpr (VEC > 1) Elem<T>::unpack(raw[k], sum[k]);
            else sum[k][0] = raw[k];
        }
    }
};

// One row's columns of a lane: scaled, added to what is there where that is asked for, rounded.
template <typename O, int VEC, int VECS>
__device__ __forceinline__ void put_row(O* row, const Columns<VEC, VECS>& c, const float (&sum)[VECS][VEC], const TableShape& s) {
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        if (!c.in(k)) continue;
        O* o = row + c.at(k);
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = s.scale * sum[k][e];
        if (s.accumulate) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = fmaf(s.scale, sum[k][e], Elem<O>::get(o[e]));
        }
        put_elements(o, f);
    }
}

// Zeros, 16 KB of a row to a block (a table without gaps is one row).
template <typename O>
__global__ void __launch_bounds__(ED_THREADS) embedding_fill_kernel(O* out, i64 slabs, i64 dim, i64 stride) {
    pdl_wait(out);
    pdl_trigger();
    constexpr int VEC = Elem<O>::VEC, SLAB = ED_THREADS * 4;             // vectors
    const i64 row = blockIdx.x / slabs, slab = blockIdx.x - row * slabs;
    O* o = out + row * stride;
    const i64 head = min((i64)row_head(o), dim), vectors = (dim - head) / VEC, tail = head + vectors * VEC;
    if (slab == 0) {
        if (threadIdx.x < head) o[threadIdx.x] = Elem<O>::put(0.f);
        if (tail + threadIdx.x < dim) o[tail + threadIdx.x] = Elem<O>::put(0.f);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const i64 v = slab * SLAB + k * ED_THREADS + threadIdx.x;
        if (v < vectors) store_vec(o + head + v * VEC, make_uint4(0u, 0u, 0u, 0u));
    }
}

// long_blocks of the blocks: chunks of ED_CHUNK sorted positions, the sums of the long runs that they cut.  A run longer than a chunk holds the chunk's first
// or its last position wherever it meets one: partial[chunk][0] belongs to the first position's run, [1] to the last one's where that is another.
// The others: rows of the table with no or few positions.
// MANY: there are more teams than the device holds; fewer of them, with more columns and, one after the other, ED_ROWS rows each, take less of everything.
// Otherwise the launch takes as long as its longest run.
template <typename T, typename O, bool VECTORS, bool MANY>
__global__ void __launch_bounds__(ED_SUM_THREADS, MANY || !VECTORS ? 12 : 8) embedding_sums_kernel(const T* grad, const int2* sorted, const int2* runs, float* partial, O* out, TableShape s) {
    pdl_wait(grad, sorted, runs, partial, out);
    pdl_trigger();
    constexpr int VEC = VECTORS ? Elem<T>::VEC : 1, VECS = VECTORS ? ED_VECS : MANY ? ED_MANY_SINGLES : ED_SINGLES, ROWS = MANY ? ED_ROWS : 1;
    const int lane = threadIdx.x & (s.lanes - 1), team = threadIdx.x / s.lanes, teams = ED_SUM_THREADS / s.lanes;
    // blocks of the two kinds take turns: chunks wait for one gradient after the other, rows write
    const unsigned before = (unsigned)((unsigned long long)blockIdx.x * s.long_blocks / gridDim.x);
    const bool chunks = before != (unsigned)((unsigned long long)(blockIdx.x + 1) * s.long_blocks / gridDim.x);
    const i64 item = (i64)(chunks ? before : blockIdx.x - before) * teams + team;
    const i64 at = s.slabs == 1 ? item : item / s.slabs;
    const Columns<VEC, VECS> c(s, (int)(item - at * s.slabs), lane);
    if (chunks) {
        const i64 c0 = at * ED_CHUNK, c1 = min(c0 + ED_CHUNK, s.count);
        if (c0 >= s.count) return;
        const int ends[2] = {sorted[c0].x, sorted[c1 - 1].x};
#pragma unroll
        for (int slot = 0; slot < 2; ++slot) {
            const int key = ends[slot];
            if (key >= s.vocab || (slot == 1 && key == ends[0])) continue;
            const int2 run = runs[key];
            if (run.y - run.x <= ED_CHUNK) continue;
            float sum[VECS][VEC] = {};
            add_run<MANY, T, VEC, VECS>(grad, s.stride, sorted, max(run.x, (int)c0), min(run.y, (int)c1), c, sum);
            float* p = partial + (at * 2 + slot) * s.dim;
#pragma unroll
            for (int k = 0; k < VECS; ++k) if (c.in(k)) put_floats<VEC>(p + c.at(k), sum[k]);
        }
        return;
    }
    // ROWS rows, one after the other: their runs are looked up together, and a row's first gradient is on its way while the row before it is formed
    const i64 first = s.by_run ? at : at * ROWS;
    int2 run[ROWS], head[ROWS];
    if (s.by_run) {
        if (first >= s.count) return;
        head[0] = sorted[first];
        if (head[0].x >= s.vocab || (first > 0 && sorted[first - 1].x == head[0].x)) return;             // (no run begins here)
        run[0] = runs[head[0].x];
        if (run[0].y - run[0].x > ED_CHUNK) return;
        First<T, VEC, VECS> one;
        float sum[VECS][VEC];
        one.fetch(grad + (i64)head[0].y * s.stride, c, true);
        one.take(sum);
        if (run[0].y - run[0].x > 1) add_run<MANY, T, VEC, VECS>(grad, s.stride, sorted, run[0].x + 1, run[0].y, c, sum);
        put_row<O, VEC, VECS>(out + (i64)head[0].x * s.out_stride, c, sum, s);
        return;
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        run[r] = first + r < s.vocab ? runs[first + r] : make_int2(-1, -1);
        head[r] = run[r].x >= 0 && run[r].x < s.count ? sorted[run[r].x] : make_int2(-1, 0);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) if (head[r].x != first + r) run[r] = make_int2(0, 0);          // no such token
    First<T, VEC, VECS> next;
    next.fetch(grad + (i64)head[0].y * s.stride, c, run[0].y > run[0].x && run[0].y - run[0].x <= ED_CHUNK);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int n = run[r].y - run[r].x;
        float sum[VECS][VEC];
        next.take(sum);
        if (r + 1 < ROWS) {
            const int m = run[(r + 1) % ROWS].y - run[(r + 1) % ROWS].x;
            next.fetch(grad + (i64)head[(r + 1) % ROWS].y * s.stride, c, m > 0 && m <= ED_CHUNK);
        }
        if (first + r >= s.vocab || n > ED_CHUNK) continue;
        if (n > 1) add_run<MANY, T, VEC, VECS>(grad, s.stride, sorted, run[r].x + 1, run[r].y, c, sum);
        put_row<O, VEC, VECS>(out + (first + r) * s.out_stride, c, sum, s);
    }
}

// Adds up the partial sums of chunks [begin, end), four on their way at a time.  A run's first chunk holds it last (`first` is that chunk, where the run does not begin
// with it; else -1), every other one first.
template <int VEC>
__device__ __forceinline__ void add_partials(const float* partial, int begin, int end, int first, const Columns<VEC, 1>& c, float (&sum)[1][VEC]) {
    if (!c.in(0)) return;
    for (int i = begin; i < end; i += 4) {
        float f[4][VEC] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) if (i + k < end) get_floats<VEC>(partial + ((i64)(i + k) * 2 + (i + k == first)) * c.dim + c.at(0), f[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[0][e] += f[k][e];
    }
}

// The long runs, by their first chunk (a long run that begins in a chunk is its last one): a block looks through ED_SHARES chunks at once and joins, slab by slab
// of blockIdx.y, what begins there.  ED_SHARES teams (a block has that many or more) add up a share of the run's chunks each, in order, then the
// shares are added in order: the same order however wide a team is.  One vector a lane: the partial sums of a run come from memory, the more of them at once the better.
template <typename O, int VEC>
__global__ void __launch_bounds__(ED_JOIN_THREADS) embedding_join_kernel(const int2* sorted, const int2* runs, const float* partial, O* out, TableShape s) {
    pdl_wait(sorted, runs, partial, out);
    pdl_trigger();
    __shared__ float shares[ED_JOIN_THREADS * VEC];                // (ED_SHARES teams of up to 32 lanes)
    __shared__ int2 found[ED_SHARES];
    __shared__ int keys[ED_SHARES];
    int2 run = make_int2(0, 0);
    if (threadIdx.x < ED_SHARES) {
        const i64 c0 = ((i64)blockIdx.x * ED_SHARES + threadIdx.x) * ED_CHUNK;
        int key = 0;
        if (c0 < s.count) {
            key = sorted[min(c0 + ED_CHUNK, s.count) - 1].x;
            if (key < s.vocab) run = runs[key];
            if (run.y - run.x <= ED_CHUNK || run.x < c0) run = make_int2(0, 0);
        }
        found[threadIdx.x] = run;
        keys[threadIdx.x] = key;
    }
    const int chunks_of = run.y == 0 ? 0 : (run.y - 1) / ED_CHUNK - run.x / ED_CHUNK + 1;
    if (!__syncthreads_or(chunks_of)) return;
    const bool longest = __syncthreads_or(chunks_of > ED_SHARES);
    const int lane = threadIdx.x & (s.lanes - 1), team = threadIdx.x / s.lanes;
    const Columns<VEC, 1> c(s, blockIdx.y, lane);
    // runs of up to ED_SHARES chunks: a team each, a share being a chunk
    if (team < ED_SHARES && found[team].y != 0) {
        const int2 run = found[team];
        const int chunk = run.x / ED_CHUNK, n = (run.y - 1) / ED_CHUNK - chunk + 1;
        if (n <= ED_SHARES) {
            float sum[1][VEC] = {};
            add_partials(partial, chunk, chunk + n, run.x > chunk * ED_CHUNK ? chunk : -1, c, sum);
            put_row<O, VEC, 1>(out + (i64)keys[team] * s.out_stride, c, sum, s);
        }
    }
    if (!longest) return;
    for (int w = 0; w < ED_SHARES; ++w) {
        const int2 run = found[w];
        const int chunk = run.x / ED_CHUNK, n = (run.y - 1) / ED_CHUNK - chunk + 1, per = (n + ED_SHARES - 1) / ED_SHARES;
        if (run.y == 0 || n <= ED_SHARES) continue;                // (the same in all threads)
        const int begin = chunk + min(team * per, n), end = chunk + min((team + 1) * per, n);
        float* mine = shares + (size_t)team * s.lanes * VEC + lane;                                // [team][element][lane]
        float sum[1][VEC] = {};
        if (team < ED_SHARES) {
            add_partials(partial, begin, end, run.x > chunk * ED_CHUNK ? chunk : -1, c, sum);
#pragma unroll
            for (int e = 0; e < VEC; ++e) mine[e * s.lanes] = sum[0][e];
        }
        __syncthreads();
        if (team == 0) {
            for (int t = 1; t < min(ED_SHARES, n); ++t)
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[0][e] += mine[(size_t)t * s.lanes * VEC + e * s.lanes];
            put_row<O, VEC, 1>(out + (i64)keys[w] * s.out_stride, c, sum, s);
        }
        __syncthreads();
    }
}

}  // namespace ef21
