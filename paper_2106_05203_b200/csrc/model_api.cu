// libef21: C-ABI entry points of a language model's worker -- objectives with their gradients, and the embedding table (see include/ef21.h).
#include <cmath>

#include "balance.cuh"
#include "embedding.cuh"
#include "launch.cuh"
#include "policy.cuh"
#include "preference.cuh"
#include "token_logprobs.cuh"

using namespace ef21;

namespace {

constexpr i64 MOST = 0x7fffffffll;            // rows, columns and positions are counted in 31 bits, elements in 63
constexpr int SMS = 148;

cudaStream_t stream_of(void* s) { return reinterpret_cast<cudaStream_t>(s); }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int bytes_of(int32_t dtype) { return dtype == EF21_DTYPE_F32 ? 4 : 2; }
bool index_aligned(const void* p, int32_t type) { return aligned(p, type == EF21_INDEX_I64 ? 8 : 4); }
bool floats_aligned(const void* a, const void* b = nullptr, const void* c = nullptr) { return aligned(a, 4) && aligned(b, 4) && aligned(c, 4); }
bool valid_dtype(int32_t dtype) { return dtype >= EF21_DTYPE_F32 && dtype <= EF21_DTYPE_F16; }
bool valid_index(int32_t t) { return t == EF21_INDEX_I32 || t == EF21_INDEX_I64; }
unsigned grid_of(i64 items, i64 per, i64 most) {
    const i64 n = ceil_div(items, per);
    return (unsigned)(n < 1 ? 1 : n > most ? most : n);
}

// f with a null pointer of the element type.
template <typename F>
ef21_status by_dtype(int32_t dtype, F f) {
    switch (dtype) {
        case EF21_DTYPE_F32: return f(static_cast<float*>(nullptr));
        case EF21_DTYPE_BF16: return f(static_cast<__nv_bfloat16*>(nullptr));
        default: return f(static_cast<__half*>(nullptr));
    }
}
template <typename P> struct Pointee;
template <typename T> struct Pointee<T*> { typedef T type; };

// Sections of a workspace, 256-byte aligned.
struct Sections {
    char* base;
    size_t used = 0;
    explicit Sections(void* p) : base(static_cast<char*>(p)) {}
    template <typename T> T* take(size_t n) {
        T* p = reinterpret_cast<T*>(base + used);
        used += align_up(n * sizeof(T));
        return p;
    }
};
// What a size query answers for `used` bytes: a call that keeps something asks for more than EF21_NO_WORKSPACE, however little it is.
size_t workspace_size(size_t used) { return used == 0 ? (size_t)EF21_NO_WORKSPACE : used > EF21_NO_WORKSPACE ? used : EF21_NO_WORKSPACE + ALIGN; }
bool workspace_fits(const void* p, size_t have, size_t need) { return p != nullptr && have >= need && aligned(p, ALIGN); }

// ---- token log-probabilities --------------------------------------------------------------------------------------------------------------

bool valid_logits(int32_t dtype, i64 batch, i64 length, i64 vocab, int32_t index, float scale) {
    return valid_dtype(dtype) && valid_index(index) && batch >= 0 && length >= 0 && vocab >= 1 && vocab <= MOST && batch <= MOST && length <= MOST &&
           batch * length <= MOST && std::isfinite(scale * LOG2E) && scale > 0.f;
}

// Blocks that share a row: one where the rows fill the device, up to eight of at least 2,048 columns each where they do not.
unsigned logprob_cluster(i64 rows, i64 vocab) {
    unsigned C = 1;
    while (C < 8 && rows * C * 2 <= SMS * 4 && vocab / (C * 2) >= 2048) C *= 2;
    return C;
}

// Units of one warp per row, 0 where a row has a warp, a block or a cluster: rows that one warp takes, and batches that end with few rows running alone either way.
i64 logprob_units(int32_t dtype, i64 rows, i64 vocab) {
    const i64 bytes = bytes_of(dtype), span = (i64)LP_UNIT * 32 * 16 / bytes;
    return vocab <= LP_WARP_VOCAB || rows < SMS * 2 ? 0 : ceil_div(vocab, span);
}

// ---- preference loss: which kernel --------------------------------------------------------------------------------------------------------

// Blocks per pair: one where the pairs fill the device, up to eight of at least PF_PART elements each where they do not.  (A cluster's barriers cost: 512 pairs x
// 8,191 fp32 by one block each 22 us, by eight 52; replayed from a graph.)
struct PreferencePlan { bool by_warp, one; unsigned split, blocks; i64 losses; };
PreferencePlan preference_plan(i64 pairs, i64 length) {
    PreferencePlan p;
    p.by_warp = length <= PF_WARP_LENGTH;
    p.split = 1;
    if (!p.by_warp) while (p.split < PF_CLUSTER && p.split * PF_PART < length && pairs * p.split * 2 <= SMS * 2) p.split *= 2;
    p.blocks = (unsigned)(p.by_warp ? ceil_div(pairs, PF_THREADS / 32) : pairs * p.split);
    p.one = p.blocks <= PF_CLUSTER;
    p.losses = p.blocks / p.split;
    return p;
}

// ---- policy loss: which kernel ------------------------------------------------------------------------------------------------------------

struct PolicyWork { int* tokens; i64* counted; PolicySums* partial; };
size_t policy_layout(void* p, i64 rows, PolicyWork& w) {
    Sections s(p);
    w.tokens = s.take<int>((size_t)rows);
    w.counted = s.take<i64>(PO_COUNT_BLOCKS);
    w.partial = s.take<PolicySums>(PO_MAX_BLOCKS);
    return s.used;
}
bool valid_rows(i64 rows, i64 length) { return rows >= 0 && length >= 0 && rows <= MOST && length <= MOST; }

struct BalanceBuffers { BalanceWork* work; double* part; float* partial; };
size_t balance_layout(void* p, i64 experts, BalanceBuffers& w) {
    Sections s(p);
    w.work = s.take<BalanceWork>(1);
    w.part = s.take<double>((size_t)ceil_div(experts, BL_FINISH_COLUMNS));
    w.partial = s.take<float>((size_t)BL_MAX_BLOCKS * (size_t)experts);
    return s.used;
}

// ---- embedding ----------------------------------------------------------------------------------------------------------------------------

struct RadixPlan { int passes, bits; i64 tiles; };
RadixPlan radix_plan(i64 count, i64 vocab) {
    int need = 1;
    while (need < 31 && (vocab >> need) != 0) ++need;                 // the key `vocab` itself is there too
    RadixPlan p;
    p.passes = (need + RX_MAX_BITS - 1) / RX_MAX_BITS;
    p.bits = (need + p.passes - 1) / p.passes;
    p.tiles = ceil_div(count, RX_TILE);
    return p;
}
struct EmbeddingWork { int2 *runs, *sorted, *other; int *counts, *totals; float* partial; };
size_t embedding_layout(void* p, i64 count, i64 vocab, i64 dim, EmbeddingWork& w) {
    Sections s(p);
    w.runs = s.take<int2>((size_t)vocab);
    w.sorted = s.take<int2>((size_t)count);
    w.other = nullptr; w.counts = w.totals = nullptr;
    if (count > ED_RANK_TOKENS) {
        w.other = s.take<int2>((size_t)count);
        w.counts = s.take<int>((size_t)radix_plan(count, vocab).tiles << RX_MAX_BITS);
        w.totals = s.take<int>(1 << RX_MAX_BITS);
    }
    w.partial = s.take<float>((size_t)ceil_div(count, ED_CHUNK) * 2 * (size_t)dim);
    return s.used;
}
// Whether the table is cleared and only rows that tokens name are formed, instead of every row by its run: one launch more, zeros at the speed of a plain
// store.  (131,072 x 64 fp32: 4 tokens 8.9 us row by row and 9.9 cleared, 20,000 tokens 54 and 42; 98,621 x 917: 4 tokens 187 and 54, 60,000 356 and 379.)
bool embedding_by_run(i64 count, i64 vocab, i64 row_bytes) {
    return count * 4 <= vocab && vocab * row_bytes >= (16 << 20);
}
bool valid_table(i64 count, i64 vocab, i64 dim) {
    return count >= 0 && count <= MOST - RX_TILE && vocab >= 1 && vocab < MOST && dim >= 1 && dim <= MOST && dim <= (1ll << 40) / vocab && dim <= (1ll << 40) / (count + 1);
}

// Sorted positions and the runs of all tokens.
ef21_status enqueue_sort(cudaStream_t st, const void* tokens, int wide, i64 count, i64 vocab, i64 padding, const EmbeddingWork& w) {
    if (count <= ED_RANK_TOKENS) {
        CU(launch(embedding_rank_kernel, grid_of(count, ED_RANK_THREADS / 32, SMS * 4), ED_RANK_THREADS, (size_t)ceil_div(count, 128) * 128 * sizeof(int), st, 1, tokens, wide, (int)count, vocab, padding,
                  w.sorted, w.runs));
        return EF21_OK;
    }
    const RadixPlan p = radix_plan(count, vocab);
    const int2* source = nullptr;
    for (int k = 0; k < p.passes; ++k) {
        int2* target = (p.passes - k) % 2 ? w.sorted : w.other;       // the last pass ends in `sorted`
        CU(launch(radix_count_kernel, (unsigned)p.tiles, RX_THREADS, 0, st, 1, source, tokens, wide, count, vocab, padding, k * p.bits, p.bits, w.counts));
        CU(launch(radix_places_kernel, (unsigned)ceil_div(1 << p.bits, 32), RX_THREADS, 0, st, 1, w.counts, w.totals, p.tiles, 1 << p.bits));
        CU(launch(radix_move_kernel, (unsigned)p.tiles, RX_THREADS, 0, st, 1, source, tokens, wide, count, vocab, padding, k * p.bits, p.bits, w.counts, w.totals, target));
        source = target;
    }
    CU(launch(embedding_runs_kernel, (unsigned)ceil_div(count, ED_THREADS), ED_THREADS, 0, st, 1, w.sorted, w.runs, count, vocab));
    return EF21_OK;
}

}  // namespace

extern "C" {

size_t ef21_token_logprobs_workspace_bytes(int32_t dtype, int64_t batch, int64_t length, int64_t vocab) {
    if (!valid_logits(dtype, batch, length, vocab, EF21_INDEX_I64, 1.f)) return 0;
    const i64 units = logprob_units(dtype, batch * length, vocab);
    return workspace_size(align_up(sizeof(float2) * (size_t)(batch * length) * (size_t)units));
}

ef21_status ef21_token_logprobs(const void* logits_dev, int32_t dtype, int64_t batch, int64_t length, int64_t vocab, int64_t batch_stride, int64_t row_stride,
                                const void* targets_dev, int32_t index_type, int64_t targets_batch_stride, float scale, int64_t ignore,
                                float* logps_out_dev, float* lse_out_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
    if (!valid_logits(dtype, batch, length, vocab, index_type, scale)) return EF21_ERR_INVALID_ARG;
    const i64 rows = batch * length;
    if (rows == 0) return EF21_OK;
    if (!logits_dev || !targets_dev || !logps_out_dev || !lse_out_dev || !aligned(logits_dev, bytes_of(dtype)) || !index_aligned(targets_dev, index_type) ||
        !floats_aligned(logps_out_dev, lse_out_dev))
        return EF21_ERR_INVALID_ARG;
    if (!workspace_fits(workspace_dev, workspace_bytes, ef21_token_logprobs_workspace_bytes(dtype, batch, length, vocab))) return EF21_ERR_WORKSPACE;
    const LogprobShape s{length, vocab, batch_stride, row_stride, targets_batch_stride, ignore, index_type, scale};
    return by_dtype(dtype, [&](auto* type) -> ef21_status {
        typedef typename Pointee<decltype(type)>::type T;
        const T* logits = static_cast<const T*>(logits_dev);
        cudaStream_t st = stream_of(cuda_stream);
        if (vocab <= LP_WARP_VOCAB) {
            CU(launch(logprobs_warp_kernel<T>, (unsigned)ceil_div(rows, LP_THREADS / 32), LP_THREADS, 0, st, 1, logits, targets_dev, logps_out_dev, lse_out_dev, s, rows));
        } else if (const i64 per_row = logprob_units(dtype, rows, vocab)) {
            if (ceil_div(rows * per_row, LP_THREADS / 32) > MOST) return EF21_ERR_UNSUPPORTED;        // (beyond any device's memory)
            float2* part = static_cast<float2*>(workspace_dev);
            CU(launch(logprobs_unit_kernel<T>, (unsigned)ceil_div(rows * per_row, LP_THREADS / 32), LP_THREADS, 0, st, 1, logits, targets_dev, part, s, rows * per_row, (int)per_row));
            CU(launch(logprobs_join_kernel<T>, (unsigned)ceil_div(rows, LP_THREADS / 32), LP_THREADS, 0, st, 1, logits, targets_dev, part, logps_out_dev, lse_out_dev, s, rows, (int)per_row));
        } else {
            const unsigned C = logprob_cluster(rows, vocab);
            CU(launch(logprobs_block_kernel<T>, (unsigned)(rows * C), LP_THREADS, 0, st, C, logits, targets_dev, logps_out_dev, lse_out_dev, s, C));
        }
        return EF21_OK;
    });
}

ef21_status ef21_token_logprobs_grad(const void* logits_dev, int32_t dtype, int64_t batch, int64_t length, int64_t vocab, int64_t batch_stride, int64_t row_stride,
                                     const void* targets_dev, int32_t index_type, int64_t targets_batch_stride, const float* lse_dev, const float* grad_dev,
                                     float scale, int64_t ignore, void* out_dev, int64_t out_batch_stride, int64_t out_row_stride, void* cuda_stream) {
    if (!valid_logits(dtype, batch, length, vocab, index_type, scale)) return EF21_ERR_INVALID_ARG;
    const i64 rows = batch * length;
    if (rows == 0) return EF21_OK;
    if (!logits_dev || !targets_dev || !lse_dev || !grad_dev || !out_dev || !aligned(logits_dev, bytes_of(dtype)) || !aligned(out_dev, bytes_of(dtype)) ||
        !index_aligned(targets_dev, index_type) || !floats_aligned(lse_dev, grad_dev))
        return EF21_ERR_INVALID_ARG;
    const LogprobShape s{length, vocab, batch_stride, row_stride, targets_batch_stride, ignore, index_type, scale};
    return by_dtype(dtype, [&](auto* type) -> ef21_status {
        typedef typename Pointee<decltype(type)>::type T;
        const T* logits = static_cast<const T*>(logits_dev);
        T* out = static_cast<T*>(out_dev);
        cudaStream_t st = stream_of(cuda_stream);
        if (vocab <= LP_WARP_VOCAB) {
            CU(launch(logprobs_grad_warp_kernel<T>, (unsigned)ceil_div(rows, LP_THREADS / 32), LP_THREADS, 0, st, 1, logits, targets_dev, lse_dev, grad_dev, out, s, out_batch_stride,
                      out_row_stride, rows));
            return EF21_OK;
        }
        const i64 slab = (i64)LP_THREADS * Elem<T>::VEC * LG_UNROLL * 2, slabs = ceil_div(vocab, slab);
        if (rows * slabs > MOST) return EF21_ERR_UNSUPPORTED;         // (more than 2^31 slabs of 16 KB or more: no device holds them)
        CU(launch(logprobs_grad_block_kernel<T>, (unsigned)(rows * slabs), LP_THREADS, 0, st, 1, logits, targets_dev, lse_dev, grad_dev, out, s, out_batch_stride, out_row_stride,
                  (unsigned)slabs, slab));
        return EF21_OK;
    });
}

size_t ef21_preference_loss_workspace_bytes(int64_t pairs, int64_t length) {
    if (pairs < 1 || pairs > MOST / 16 || length < 0 || length > MOST) return 0;
    const PreferencePlan p = preference_plan(pairs, length);
    return workspace_size(p.one ? 0 : align_up(sizeof(double) * (size_t)p.losses));
}

ef21_status ef21_preference_loss(const void* logps_dev, const void* ref_dev, const uint8_t* mask_dev, int32_t dtype, int64_t pairs, int64_t length,
                                 int64_t logps_stride, int64_t ref_stride, int64_t mask_stride, double beta, double smoothing, double norm,
                                 float* loss_out_dev, float* rewards_out_dev, void* grad_out_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
    const size_t need = ef21_preference_loss_workspace_bytes(pairs, length);
    if (need == 0 || !valid_dtype(dtype) || !std::isfinite(beta) || !(smoothing >= 0.0 && smoothing <= 1.0) || !(norm > 0.0) || !std::isfinite(norm)) return EF21_ERR_INVALID_ARG;
    if (!loss_out_dev || !rewards_out_dev || (length > 0 && (!logps_dev || !grad_out_dev))) return EF21_ERR_INVALID_ARG;
    const size_t e = bytes_of(dtype);
    if (!aligned(logps_dev, e) || !aligned(ref_dev, e) || !aligned(grad_out_dev, e) || !floats_aligned(loss_out_dev, rewards_out_dev)) return EF21_ERR_INVALID_ARG;
    if (!workspace_fits(workspace_dev, workspace_bytes, need)) return EF21_ERR_WORKSPACE;
    double* partial = static_cast<double*>(workspace_dev);
    const PreferencePlan P = preference_plan(pairs, length);
    cudaStream_t st = stream_of(cuda_stream);
    return by_dtype(dtype, [&](auto* type) -> ef21_status {
        typedef typename Pointee<decltype(type)>::type T;
        constexpr int VEC = Elem<T>::VEC;
        const T *logps = static_cast<const T*>(logps_dev), *ref = static_cast<const T*>(ref_dev);
        T* grad = static_cast<T*>(grad_out_dev);
        const PreferenceShape s{pairs, length, logps_stride, ref_stride, mask_stride, beta, smoothing, norm, P.split, (int)P.one};
        const bool vectors = aligned(logps, 16) && aligned(ref, 16) && aligned(grad, 16) && aligned(mask_dev, VEC) && (logps_stride - length) % VEC == 0 &&
                             (!ref || (ref_stride - length) % VEC == 0) && (!mask_dev || (mask_stride - length) % VEC == 0);
        auto run = [&](auto kernel) -> ef21_status {
            CU(launch(kernel, P.blocks, PF_THREADS, 0, st, P.one ? P.blocks : P.split, logps, ref, mask_dev, rewards_out_dev, grad, partial, loss_out_dev, s));
            return EF21_OK;
        };
        if (P.by_warp) EF(vectors ? run(preference_kernel<T, true, 32>) : run(preference_kernel<T, false, 32>));
        else EF(vectors ? run(preference_kernel<T, true, PF_THREADS>) : run(preference_kernel<T, false, PF_THREADS>));
        if (!P.one) CU(launch(preference_finish_kernel, 1, PF_FINISH_THREADS, 0, st, 1, partial, loss_out_dev, P.losses, norm));
        return EF21_OK;
    });
}

size_t ef21_policy_loss_workspace_bytes(int64_t rows, int64_t length) {
    PolicyWork w;
    return valid_rows(rows, length) ? workspace_size(policy_layout(nullptr, rows, w)) : 0;
}

ef21_status ef21_policy_loss(const void* logps_dev, const void* old_dev, const void* ref_dev, const void* advantages_dev, const uint8_t* mask_dev, int32_t dtype,
                             int64_t rows, int64_t length, int64_t logps_stride, int64_t old_stride, int64_t ref_stride, int64_t advantages_stride, int64_t mask_stride,
                             int32_t advantages_per_token, double clip_low, double clip_high, double kl_weight, int32_t reduction, double norm,
                             float* terms_out_dev, void* grad_out_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
    const size_t need = ef21_policy_loss_workspace_bytes(rows, length);
    if (need == 0 || !valid_dtype(dtype) || !(clip_low >= 0.0 && clip_low < 1.0) || !(clip_high >= 0.0) || !std::isfinite(clip_high) || !std::isfinite((float)kl_weight) ||
        (reduction != EF21_REDUCE_TOKENS && reduction != EF21_REDUCE_SEQUENCES) || !(norm >= 0.0) || !std::isfinite(norm) || (norm > 0.0 && !std::isfinite((float)(1.0 / norm))) || (!ref_dev && kl_weight != 0.0))
        return EF21_ERR_INVALID_ARG;
    if (!terms_out_dev || (rows * length > 0 && (!logps_dev || !old_dev || !advantages_dev || !grad_out_dev))) return EF21_ERR_INVALID_ARG;
    const size_t e = bytes_of(dtype);
    if (!aligned(logps_dev, e) || !aligned(old_dev, e) || !aligned(ref_dev, e) || !aligned(advantages_dev, e) || !aligned(grad_out_dev, e) || !floats_aligned(terms_out_dev))
        return EF21_ERR_INVALID_ARG;
    if (!workspace_fits(workspace_dev, workspace_bytes, need)) return EF21_ERR_WORKSPACE;
    PolicyWork w;
    policy_layout(workspace_dev, rows, w);
    cudaStream_t st = stream_of(cuda_stream);
    const bool by_sequence = reduction == EF21_REDUCE_SEQUENCES, count = mask_dev && (norm == 0.0 || by_sequence);
    const unsigned count_blocks = grid_of(rows, PO_COUNT_THREADS / 32, PO_COUNT_BLOCKS);
    const i64 all = rows * length;
    auto whole = [&](const void* p, i64 stride) { return aligned(p, 16) && (!p || rows <= 1 || stride == length); };
    const int vec = 16 / bytes_of(dtype);
    const bool flat = whole(logps_dev, logps_stride) && whole(old_dev, old_stride) && whole(ref_dev, ref_stride) && (!advantages_per_token || whole(advantages_dev, advantages_stride)) &&
                      aligned(grad_out_dev, 16) && aligned(mask_dev, vec) && (!mask_dev || rows <= 1 || mask_stride == length);
    // one cluster: its blocks count all tokens themselves, words of 4 or 8 where the arrays are flat, else one by one
    const bool one = rows <= PO_ONE_ROWS && all <= (flat ? PO_ONE_TOKENS : PO_ONE_TOKENS / 8);
    if (count && !one) CU(launch(policy_count_kernel, count_blocks, PO_COUNT_THREADS, 0, st, 1, mask_dev, w.tokens, w.counted, rows, length, mask_stride, (int)by_sequence));
    return by_dtype(dtype, [&](auto* type) -> ef21_status {
        typedef typename Pointee<decltype(type)>::type T;
        constexpr int VEC = Elem<T>::VEC;
        const T *logps = static_cast<const T*>(logps_dev), *old = static_cast<const T*>(old_dev), *ref = static_cast<const T*>(ref_dev), *adv = static_cast<const T*>(advantages_dev);
        T* grad = static_cast<T*>(grad_out_dev);
        const i64 items = flat ? all / VEC : all, most = one ? PO_CLUSTER : PO_MAX_BLOCKS;
        const i64 per_block = PO_THREADS * (one ? ceil_div(items, PO_THREADS * most) : ceil_div(items, PO_THREADS * PO_VECTORS * most) * PO_VECTORS);
        const unsigned blocks = grid_of(items, per_block > 0 ? per_block : 1, most);
        const PolicyShape s{rows, length, logps_stride, old_stride, ref_stride, mask_stride, advantages_stride, advantages_per_token, by_sequence,
                            std::log1p(-clip_low), std::log1p(clip_high), (float)(1e-6 * (1.0 + std::fmax(-std::log1p(-clip_low), std::log1p(clip_high)))), (float)(1.0 - clip_low), (float)(1.0 + clip_high), (float)kl_weight, norm, (int)count_blocks, per_block, (int)one};
        const int* tokens = count && !one ? w.tokens : nullptr;
        const i64* counted = count && !one ? w.counted : nullptr;
        if (flat) CU(launch(policy_kernel<T, true>, blocks, PO_THREADS, 0, st, one ? blocks : 1, logps, old, ref, adv, mask_dev, tokens, counted, grad, w.partial, terms_out_dev, s));
        else CU(launch(policy_kernel<T, false>, blocks, PO_THREADS, 0, st, one ? blocks : 1, logps, old, ref, adv, mask_dev, tokens, counted, grad, w.partial, terms_out_dev, s));
        if (!one) CU(launch(policy_finish_kernel, 1, PO_FINISH_THREADS, 0, st, 1, w.partial, terms_out_dev, (int)blocks, (float)kl_weight));
        return EF21_OK;
    });
}

size_t ef21_balance_loss_workspace_bytes(int64_t rows, int64_t experts) {
    BalanceBuffers w;
    return rows < 0 || rows > MOST || experts < 1 || experts > BL_MAX_EXPERTS ? 0 : workspace_size(balance_layout(nullptr, experts, w));
}

ef21_status ef21_balance_loss(const void* logits_dev, int32_t dtype, int64_t rows, int64_t experts, int64_t logits_stride, const void* choices_dev, int32_t index_type, int64_t chosen,
                              int64_t choices_stride, const uint8_t* mask_dev, double weight, float* loss_out_dev, int32_t* counts_out_dev, float* probs_out_dev, void* grad_out_dev,
                              void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
    const size_t need = ef21_balance_loss_workspace_bytes(rows, experts);
    if (need == 0 || !valid_dtype(dtype) || !valid_index(index_type) || chosen < 1 || chosen > experts || rows * chosen > MOST || !std::isfinite((float)(weight * (double)experts))) return EF21_ERR_INVALID_ARG;
    if (!loss_out_dev || !counts_out_dev || !probs_out_dev || (rows > 0 && (!logits_dev || !choices_dev || !grad_out_dev))) return EF21_ERR_INVALID_ARG;
    if (!aligned(logits_dev, bytes_of(dtype)) || !aligned(grad_out_dev, bytes_of(dtype)) || !index_aligned(choices_dev, index_type) ||
        !floats_aligned(loss_out_dev, counts_out_dev, probs_out_dev))
        return EF21_ERR_INVALID_ARG;
    if (!workspace_fits(workspace_dev, workspace_bytes, need)) return EF21_ERR_WORKSPACE;
    BalanceBuffers w;
    balance_layout(workspace_dev, experts, w);
    cudaStream_t st = stream_of(cuda_stream);
    return by_dtype(dtype, [&](auto* type) -> ef21_status {
        typedef typename Pointee<decltype(type)>::type T;
        constexpr int V = Elem<T>::VEC;
        const T* logits = static_cast<const T*>(logits_dev);
        T* grad = static_cast<T*>(grad_out_dev);
        const i64 columns = ceil_div(experts, V);
        BalanceShape s{rows, (int)experts, (int)chosen, index_type, logits_stride, choices_stride, weight, 1, 0, experts % V == 0 && aligned(logits, 16) && logits_stride % V == 0, experts % V == 0 && aligned(grad, 16)};
        // two vectors a lane where there are enough: a row's shuffles, division and addresses are shared by fewer lanes
        while (s.lanes < 32 && s.lanes * 2 < columns) s.lanes *= 2;
        s.one = rows * chosen <= BL_ONE_CHOICES && rows * experts <= BL_ONE_LOGITS;
        const unsigned blocks = grid_of(rows, BL_THREADS / s.lanes, s.one ? BL_CLUSTER : BL_MAX_BLOCKS);
        if (!s.one) {
            CU(launch(balance_clear_kernel, 1, BL_THREADS, 0, st, 1, counts_out_dev, w.work, (int)experts));
            CU(launch(balance_count_kernel, grid_of(rows * chosen, BL_COUNT_THREADS * 4, SMS * 2), BL_COUNT_THREADS, 0, st, 1, choices_dev, mask_dev, counts_out_dev, w.work, s));
        }
        auto run = [&](auto kernel) -> ef21_status {
            CU(launch(kernel, blocks, BL_THREADS, sizeof(float) * (size_t)(BL_THREADS / 32 * experts), st, s.one ? blocks : 1, logits, choices_dev, mask_dev, counts_out_dev, w.work, grad, w.partial, probs_out_dev, loss_out_dev, s));
            return EF21_OK;
        };
        // rows in flight per team: 16 values per lane or more
        if (columns <= 64) EF(s.lanes == 32 ? run(balance_kernel<T, 2, 8 / V, 32>) : s.lanes == 16 ? run(balance_kernel<T, 2, 8 / V, 16>) : run(balance_kernel<T, 2, 8 / V, 0>));
        else if (columns <= 128) EF(run(balance_kernel<T, 4, 1, 32>));
        else if constexpr (V == 4) EF(run(balance_kernel<T, 8, 1, 32>));
        if (!s.one) CU(launch(balance_finish_kernel, (unsigned)ceil_div(experts, BL_FINISH_COLUMNS), BL_FINISH_COLUMNS * BL_FINISH_GROUPS, 0, st, 1, w.partial, counts_out_dev, w.work, w.part,
                              probs_out_dev, loss_out_dev, (int)blocks, (int)experts, (int)chosen, weight));
        return EF21_OK;
    });
}

ef21_status ef21_embedding(const void* weight_dev, int32_t dtype, int64_t vocab, int64_t dim, int64_t weight_stride, const void* tokens_dev, int32_t index_type, int64_t count, float scale,
                           void* out_dev, void* cuda_stream) {
    if (!valid_dtype(dtype) || !valid_index(index_type) || !valid_table(count, vocab, dim) || !std::isfinite(scale)) return EF21_ERR_INVALID_ARG;
    if (count == 0) return EF21_OK;
    if (!weight_dev || !tokens_dev || !out_dev || !aligned(weight_dev, bytes_of(dtype)) || !aligned(out_dev, bytes_of(dtype)) || !index_aligned(tokens_dev, index_type)) return EF21_ERR_INVALID_ARG;
    return by_dtype(dtype, [&](auto* type) -> ef21_status {
        typedef typename Pointee<decltype(type)>::type T;
        constexpr int VEC = Elem<T>::VEC;
        const T* weight = static_cast<const T*>(weight_dev);
        T* out = static_cast<T*>(out_dev);
        cudaStream_t st = stream_of(cuda_stream);
        const bool vectors = aligned(weight, 16) && aligned(out, 16) && dim % VEC == 0 && weight_stride % VEC == 0;
        if (!vectors && dim <= ED_SHORT) {                            // (30,000 rows of 63 bf16: 6 us, 16 by vectors of the output)
            CU(launch(embedding_short_kernel<T>, (unsigned)ceil_div(count, ED_THREADS / 32), ED_THREADS, 0, st, 1, weight, tokens_dev, out, count, vocab, dim, weight_stride, index_type, scale));
            return EF21_OK;
        }
        const i64 slabs = ceil_div(dim, (i64)32 * ED_ROW_VECS * VEC), items = count * slabs;
        if (ceil_div(items, ED_THREADS / 32) > MOST) return EF21_ERR_UNSUPPORTED;        // (1 TB of output and more)
        const unsigned blocks = (unsigned)ceil_div(items, ED_THREADS / 32);
        if (vectors) CU(launch(embedding_kernel<T, true>, blocks, ED_THREADS, 0, st, 1, weight, tokens_dev, out, items, (int)slabs, vocab, dim, weight_stride, index_type, scale));
        else CU(launch(embedding_kernel<T, false>, blocks, ED_THREADS, 0, st, 1, weight, tokens_dev, out, items, (int)slabs, vocab, dim, weight_stride, index_type, scale));
        return EF21_OK;
    });
}

size_t ef21_embedding_grad_workspace_bytes(int64_t count, int64_t vocab, int64_t dim) {
    EmbeddingWork w;
    return valid_table(count, vocab, dim) ? workspace_size(embedding_layout(nullptr, count, vocab, dim, w)) : 0;
}

ef21_status ef21_embedding_grad(const void* grad_dev, int32_t dtype, int64_t count, int64_t dim, int64_t grad_stride, const void* tokens_dev, int32_t index_type, int64_t vocab,
                                int64_t padding, float scale, void* out_dev, int32_t out_dtype, int64_t out_stride, int32_t accumulate, void* workspace_dev, size_t workspace_bytes,
                                void* cuda_stream) {
    const size_t need = ef21_embedding_grad_workspace_bytes(count, vocab, dim);
    if (need == 0 || !valid_dtype(dtype) || (out_dtype != dtype && out_dtype != EF21_DTYPE_F32) || !valid_index(index_type) || !std::isfinite(scale) || !out_dev ||
        (count > 0 && (!grad_dev || !tokens_dev)) || !aligned(grad_dev, bytes_of(dtype)) || !aligned(out_dev, bytes_of(out_dtype)) || !index_aligned(tokens_dev, index_type))
        return EF21_ERR_INVALID_ARG;
    if (!workspace_fits(workspace_dev, workspace_bytes, need)) return EF21_ERR_WORKSPACE;
    EmbeddingWork w;
    embedding_layout(workspace_dev, count, vocab, dim, w);
    cudaStream_t st = stream_of(cuda_stream);
    EF(enqueue_sort(st, tokens_dev, index_type, count, vocab, padding, w));
    return by_dtype(dtype, [&](auto* type) -> ef21_status {
        typedef typename Pointee<decltype(type)>::type T;
        const T* grad = static_cast<const T*>(grad_dev);
        auto run = [&](auto* out) -> ef21_status {
            typedef typename Pointee<decltype(out)>::type O;
            constexpr int VEC = Elem<T>::VEC;
            const bool vectors = aligned(grad, 16) && dim % VEC == 0 && grad_stride % VEC == 0 && aligned(out, VEC * sizeof(O)) && out_stride % VEC == 0;
            TableShape s{count, vocab, dim, grad_stride, out_stride, scale, accumulate, 1, 1, 0, 0};
            const i64 columns = dim / (vectors ? VEC : 1);
            s.by_run = accumulate || embedding_by_run(count, vocab, dim * (i64)sizeof(O));
            const i64 items = s.by_run ? count : vocab;
            // (50,000 rows of 8 columns fill a quarter of the device: 24 us for 4,000 positions four rows at a time, as long as the longest runs of four rows take, and 12 one by one)
            const bool many = items * ceil_div(columns, vectors ? ED_VECS : ED_SINGLES) >= (i64)SMS * 24 * 32 * ED_ROWS;
            const int vecs = vectors ? ED_VECS : many ? ED_MANY_SINGLES : ED_SINGLES, per_team = many && !s.by_run ? ED_ROWS : 1;
            while (s.lanes < 32 && (i64)s.lanes * vecs < columns) s.lanes *= 2;
            s.slabs = (int)ceil_div(columns, (i64)s.lanes * vecs);
            const i64 teams = ED_SUM_THREADS / s.lanes, chunks = count > ED_CHUNK ? ceil_div(count, ED_CHUNK) : 0;
            const i64 long_blocks = ceil_div(chunks * s.slabs, teams), row_blocks = ceil_div(ceil_div(items, per_team) * s.slabs, teams);
            if (long_blocks + row_blocks > MOST || columns > 65535ll * 32) return EF21_ERR_UNSUPPORTED;      // (beyond any device's memory; rows of two million columns)
            if (s.by_run && !accumulate) {
                const bool gaps = out_stride != dim;
                const i64 row = gaps ? dim : dim * vocab, slabs = ceil_div(row, (i64)ED_THREADS * 4 * Elem<O>::VEC), blocks = slabs * (gaps ? vocab : 1);
                if (blocks > MOST) return EF21_ERR_UNSUPPORTED;
                CU(launch(embedding_fill_kernel<O>, (unsigned)blocks, ED_THREADS, 0, st, 1, out, slabs, row, out_stride));
            }
            s.long_blocks = (unsigned)long_blocks;
            const unsigned blocks = (unsigned)(long_blocks + row_blocks);
            if (blocks == 0) return EF21_OK;                          // (no token, and no row to be written)
            auto sums = [&](auto kernel) -> ef21_status {
                CU(launch(kernel, blocks, ED_SUM_THREADS, 0, st, 1, grad, w.sorted, w.runs, w.partial, out, s));
                return EF21_OK;
            };
            if (vectors) EF(many ? sums(embedding_sums_kernel<T, O, true, true>) : sums(embedding_sums_kernel<T, O, true, false>));
            else EF(many ? sums(embedding_sums_kernel<T, O, false, true>) : sums(embedding_sums_kernel<T, O, false, false>));
            if (chunks == 0) return EF21_OK;
            s.lanes = 1;                                              // the join's teams: one vector a lane
            while (s.lanes < 32 && s.lanes < columns) s.lanes *= 2;
            s.slabs = (int)ceil_div(columns, s.lanes);
            const dim3 grid((unsigned)ceil_div(chunks, ED_SHARES), (unsigned)s.slabs);
            if (vectors) CU(launch(embedding_join_kernel<O, VEC>, grid, ED_JOIN_THREADS, 0, st, 1, w.sorted, w.runs, w.partial, out, s));
            else CU(launch(embedding_join_kernel<O, 1>, grid, ED_JOIN_THREADS, 0, st, 1, w.sorted, w.runs, w.partial, out, s));
            return EF21_OK;
        };
        return out_dtype == EF21_DTYPE_F32 ? run(static_cast<float*>(out_dev)) : run(static_cast<T*>(out_dev));
    });
}

}  // extern "C"
