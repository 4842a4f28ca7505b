// C-ABI entries of the operators that a worker's gradient begins with: top logits, the distillation loss, the balance loss.
// Argument checks and launches on the caller's stream, as in api.cu.
#include "../../include/fastsgd.h"

#include <cmath>

#include "host.cuh"
#include "top.cuh"
#include "distill.cuh"
#include "balance.cuh"

namespace {

using namespace fsg;

constexpr double kLog2E = 1.4426950408889634;
constexpr float  kLeastTemperature = 1.f / 1048576.f, kMostTemperature = 1048576.f;

bool is_temperature(float t) { return t >= kLeastTemperature && t <= kMostTemperature; }

// A gradient: of the logits' shape, in their type or fp32; the logits' own place, element for element, or apart from them.
int check_grad(const fastsgd_matrix* grad, const fastsgd_matrix* logits) {
    const int rc = check_matrix(grad);
    if (rc) return rc;
    if (grad->rows != logits->rows || grad->cols != logits->cols) return FASTSGD_E_BAD_PARAM;
    if (grad->type != logits->type && grad->type != FASTSGD_F32) return FASTSGD_E_BAD_PARAM;
    const uintptr_t a = reinterpret_cast<uintptr_t>(grad->data), b = reinterpret_cast<uintptr_t>(logits->data);
    const bool same = a == b && grad->type == logits->type && grad->row_stride == logits->row_stride;
    if (!same && a < b + span_bytes(logits) && b < a + span_bytes(grad)) return FASTSGD_E_BAD_PARAM;
    return FASTSGD_OK;
}

template <class T, int MODE> const void* distill_kernel_of(uint32_t g) {
    if constexpr (MODE != kLossOnly && sizeof(T) == 2) if (g == FASTSGD_F32) return (const void*)k_distill<T, float, MODE>;
    return (const void*)k_distill<T, T, MODE>;
}
template <int MODE> const void* distill_kernel(uint32_t z, uint32_t g) {
    return z == FASTSGD_F32 ? distill_kernel_of<float, MODE>(g) : z == FASTSGD_BF16 ? distill_kernel_of<__nv_bfloat16, MODE>(g) : distill_kernel_of<__half, MODE>(g);
}
// Lanes that share a token: with 16 of its experts each, where that is quicker than 8 (us for 65536 tokens with 8, with 16: bf16 x 16: 6.5, 6.0, x 64:
// 10.1, 7.9, x 256: 21.0, 16.1; fp32 x 16: 6.6, 7.0, x 32: 7.7, 8.0, x 64: 10.4, 9.7, x 256: 26.7, 23.0).
uint32_t balance_lanes(uint32_t type, uint32_t experts) {
    const uint32_t each = experts > 8u && (type != FASTSGD_F32 || experts > 32u) ? 16u : 8u;
    uint32_t lanes = 1u;
    while (lanes < 32u && lanes * each < experts) lanes *= 2u;
    return lanes;
}
template <class T, class TG> const void* balance_kernel_of(uint32_t experts) {
    if (experts <= 8u) return (const void*)k_balance<T, TG, 1, 1>;
    constexpr int FEW = sizeof(T) == 4 ? 1 : 2;            // (up to 32 experts)
    if (experts <= 32u) return experts <= 16u ? (const void*)k_balance<T, TG, 2 / FEW, FEW> : (const void*)k_balance<T, TG, 4 / FEW, FEW>;
    return experts <= 64u ? (const void*)k_balance<T, TG, 4, 2> : experts <= 128u ? (const void*)k_balance<T, TG, 8, 2> : experts <= 256u ? (const void*)k_balance<T, TG, 16, 2>
         : experts <= 512u ? (const void*)k_balance<T, TG, 32, 2> : (const void*)k_balance<T, TG, 32, 4>;
}
const void* balance_kernel(uint32_t x, uint32_t g, uint32_t experts) {
    if (x == FASTSGD_F32) return balance_kernel_of<float, float>(experts);
    if (x == FASTSGD_BF16) return g == FASTSGD_F32 ? balance_kernel_of<__nv_bfloat16, float>(experts) : balance_kernel_of<__nv_bfloat16, __nv_bfloat16>(experts);
    return g == FASTSGD_F32 ? balance_kernel_of<__half, float>(experts) : balance_kernel_of<__half, __half>(experts);
}
template <uint32_t MOST> const void* top_kernel(uint32_t type) {
    return type == FASTSGD_F32 ? (const void*)k_top<float, MOST> : type == FASTSGD_BF16 ? (const void*)k_top<__nv_bfloat16, MOST> : (const void*)k_top<__half, MOST>;
}
template <class T> const void* top_rows_kernel_of(uint32_t cols) {
    return cols <= 32u ? (const void*)k_top_rows<T, 1> : cols <= 64u ? (const void*)k_top_rows<T, 2> : cols <= 128u ? (const void*)k_top_rows<T, 4>
         : cols <= 256u ? (const void*)k_top_rows<T, 8> : cols <= 512u ? (const void*)k_top_rows<T, 16> : (const void*)k_top_rows<T, 32>;
}
template <class T> const void* top_lanes_kernel_of(uint32_t width) {
    return width == 8u ? (const void*)k_top_lanes<T, 8> : width == 16u ? (const void*)k_top_lanes<T, 16> : (const void*)k_top_lanes<T, 32>;
}
const void* top_lanes_kernel(uint32_t type, uint32_t width) {
    return type == FASTSGD_F32 ? top_lanes_kernel_of<float>(width) : type == FASTSGD_BF16 ? top_lanes_kernel_of<__nv_bfloat16>(width) : top_lanes_kernel_of<__half>(width);
}
const void* top_rows_kernel(uint32_t type, uint32_t cols) {
    return type == FASTSGD_F32 ? top_rows_kernel_of<float>(cols) : type == FASTSGD_BF16 ? top_rows_kernel_of<__nv_bfloat16>(cols) : top_rows_kernel_of<__half>(cols);
}

int distill(int mode, const fastsgd_matrix* student, const fastsgd_pairs* teacher, float temperature, const float* weight,
            float* loss, float* stats_out, const float* stats_in, const float* grad_loss, const fastsgd_matrix* grad, void* stream) {
    int rc = check_matrix(student);
    if (rc) return rc;
    if (!teacher) return FASTSGD_E_NULL;
    if (!is_type(teacher->type) || teacher->k < 1u || teacher->k > kDistillMaxPairs || !is_temperature(temperature)) return FASTSGD_E_BAD_PARAM;
    if (student->rows && (!teacher->keys || !teacher->values)) return FASTSGD_E_NULL;
    if (!aligned_to(teacher->keys, 4) || !aligned_to(teacher->values, size_of(teacher->type)) || !aligned_to(teacher->tail, 4) || !aligned_to(weight, 4)
        || !aligned_to(loss, 4) || !aligned_to(stats_out, 4) || !aligned_to(stats_in, 4) || !aligned_to(grad_loss, 4)) return FASTSGD_E_ALIGN;
    if (grad) { rc = check_grad(grad, student); if (rc) return rc; }
    if (student->cols > kDistillMaxCols) return FASTSGD_E_NOT_IMPLEMENTED;
    if (!student->rows) return FASTSGD_OK;
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    DistillArgs a{};
    a.z = student->data; a.rows = student->rows; a.cols = (uint32_t)student->cols; a.z_stride = student->row_stride;
    if (grad) { a.grad = grad->data; a.grad_stride = grad->row_stride; }
    a.keys = teacher->keys; a.values = teacher->values; a.tail = teacher->tail; a.k = teacher->k; a.values_type = teacher->type;
    a.weight = weight; a.grad_loss = grad_loss; a.stats_in = stats_in; a.loss = loss; a.stats_out = stats_out;
    a.temperature = temperature; a.inv_t = 1.f / temperature; a.c = (float)(kLog2E / (double)temperature); a.slack = exp_slack(a.c);
    a.tries = dev.tries;
    const uint32_t gt = grad ? grad->type : student->type;
    const void* fn = mode == kLossOnly ? distill_kernel<kLossOnly>(student->type, gt)
                   : mode == kLossAndGrad ? distill_kernel<kLossAndGrad>(student->type, gt) : distill_kernel<kGradOnly>(student->type, gt);
    // Both passes: a row in the shared memory of as many blocks as hold it at 64 KB each (three blocks on an SM), of eight at most (above
    // half a megabyte: two blocks on an SM, and what does not fit is read twice).  One pass: a block, with 32 KB of copies ahead, as long as
    // three find room with their maps of keys.  Few rows: more blocks each, as long as a block has a vector for every thread.
    const uint32_t vecs = a.cols * size_of(student->type) / 16u;
    const bool one_pass = mode != kLossAndGrad;
    auto share = [&](unsigned blocks) { return (vecs + blocks - 1u) / blocks; };
    unsigned blocks = 1u;
    while (blocks < kDistillMaxBlocks && ((one_pass ? distill_smem(8u, a.k, share(blocks)) > 74u * 1024u : share(blocks) > 4096u) || (a.rows * blocks * 2u <= 2u * (uint64_t)dev.sm_count && share(blocks) > kDistillThreads))) blocks *= 2u;
    a.per = share(blocks);
    a.slots = (a.per + kDistillThreads - 1u) / kDistillThreads;
    if (!a.slots) a.slots = 1u;
    a.kept = one_pass && a.slots > 8u ? 8u : a.slots;
    while (!one_pass && a.kept > 4u && distill_smem(a.kept, a.k, a.per) > (a.slots <= 16u ? 100u : 108u) * 1024u) --a.kept;
    const size_t smem = (distill_smem(a.kept, a.k, a.per) + 1023u) & ~(size_t)1023u;      // (few different sizes)
    uint64_t resident = 0;                                 // (asked for so that the kernel may use as much shared memory)
    rc = resident_blocks(fn, kDistillBlock, smem, dev, &resident);
    if (rc) return rc;
    a.claims = a.rows * blocks > resident / 2u;
    // a cluster per row: one that has finished its row takes over the next that has not begun
    if (a.rows * blocks >= 1ull << 31) return FASTSGD_E_BAD_N;
    void* kargs[] = {&a};
    return launched(launch_overlapped(fn, (unsigned)(a.rows * blocks), kDistillBlock, smem, kargs, static_cast<cudaStream_t>(stream), blocks));
}

// tokens a block of the router's kernels takes, and the blocks
uint32_t rows_per_block(uint64_t tokens, uint64_t least, uint64_t blocks) {
    uint64_t rows = (tokens + blocks - 1) / blocks;
    return (uint32_t)(rows < least ? least : rows);
}

int check_tokens(uint64_t tokens, uint32_t segments, const uint64_t* offsets) {
    if (tokens >= (1ull << 31)) return FASTSGD_E_BAD_N;
    if (segments < 1u || segments > (1u << 24)) return FASTSGD_E_BAD_PARAM;
    if (!offsets && segments != 1u) return FASTSGD_E_NULL;
    return aligned_to(offsets, 8) ? FASTSGD_OK : FASTSGD_E_ALIGN;
}

}  // namespace

extern "C" {

int fastsgd_top_logits(const fastsgd_matrix* logits, uint32_t k, float temperature, int32_t* keys, void* values,
                       float* lse, float* tail, void* stream) {
    int rc = check_matrix(logits);
    if (rc) return rc;
    if (k < 1u || k > kTopMaxPairs || k > logits->cols || !is_temperature(temperature)) return FASTSGD_E_BAD_PARAM;
    if (logits->rows && (!keys || !values)) return FASTSGD_E_NULL;
    if (!aligned_to(keys, 4) || !aligned_to(values, size_of(logits->type)) || !aligned_to(lse, 4) || !aligned_to(tail, 4)) return FASTSGD_E_ALIGN;
    if (logits->cols > kTopMaxCols) return FASTSGD_E_NOT_IMPLEMENTED;
    if (!logits->rows) return FASTSGD_OK;
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    TopArgs a{};
    a.z = logits->data; a.rows = logits->rows; a.cols = (uint32_t)logits->cols; a.z_stride = logits->row_stride;
    a.keys = keys; a.values = values; a.lse = lse; a.tail = tail; a.k = k;
    a.temperature = temperature; a.c = (float)(kLog2E / (double)temperature); a.slack = exp_slack(a.c);
    a.tries = dev.tries;
    void* kargs[] = {&a};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.cols <= kTopRowsMaxCols && k <= kTopRowsMaxPairs) {
        // A lane per row takes as long for 32 rows of a warp as for one: worth it from 1024 rows a column that it has registers for
        // (us, a warp against a lane per row: 2048 x 8, k = 2: 1.8, 2.0; 8192 x 8: 2.9, 2.0; 8192 x 16: 2.9, 3.4; 32768 x 16: 7.9, 3.6;
        // 8192 x 32: 2.9, 5.4; 32768 x 32, k = 1, 8, 16: 7.4, 10.6, 14.5 and 5.0, 10.4, 16.5; 65536 x 32, k = 8: 19.8, 12.2; 65536 x 64, k = 8:
        // 24.9, 30.6 with 64 registers of ranks).
        const uint32_t width = a.cols <= 8u ? 8u : a.cols <= 16u ? 16u : 32u;
        if (a.cols <= width && a.rows >= 1024u * width) {
            const unsigned grid = (unsigned)((a.rows + kTopLanesThreads - 1) / kTopLanesThreads);
            return launched(launch_overlapped(top_lanes_kernel(logits->type, width), grid, kTopLanesThreads, 0, kargs, st));
        }
        // One by one each pair costs five instructions a value of a lane (four or eight and more of them); by the bar it is one, after some
        // 150, and above 16 pairs more than 32 candidates become likely (us, one by one against the bar, 65536 x 128, k = 4, 6, 16: 26.1, 31.0, 55.9
        // and 26.6, 29.7, 44.1; 65536 x 256, k = 2, 4, 8, 16, 32: 32.4, 41.7, 61.2, 101.7, 183 and 34.3, 36.8, 42.6, 55.3, 214).
        a.by_bar = k <= 16u && (a.cols > 128u ? k >= 4u : a.cols > 64u && k >= 6u);
        const unsigned grid = (unsigned)((a.rows + kTopRowsThreads / 32 - 1) / (kTopRowsThreads / 32));
        return launched(launch_overlapped(top_rows_kernel(logits->type, a.cols), grid, kTopRowsThreads, 0, kargs, st));
    }
    const void* fn = k <= kTopFewPairs ? top_kernel<kTopFewPairs>(logits->type) : top_kernel<kTopMaxPairs>(logits->type);
    const size_t smem = k <= kTopFewPairs ? sizeof(TopShared<kTopFewPairs>) : sizeof(TopShared<kTopMaxPairs>);
    uint64_t resident = 0;
    rc = resident_blocks(fn, kTopThreads, smem, dev, &resident);
    if (rc) return rc;
    // few rows: a cluster of up to 8 blocks shares each, as long as a block has two tiles' worth of 16-bit values for every four threads
    unsigned blocks = 1u;
    while (blocks < 8u && a.rows * blocks * 2u <= resident && a.cols / (2u * blocks) >= 8192u) blocks *= 2u;
    a.slice = ((a.cols + blocks - 1u) / blocks + 63u) & ~63u;
    // (with clusters every row has its own; otherwise a block that has finished its row takes over the next that has not begun)
    a.claims = blocks == 1u && a.rows > resident / 2u;
    return launched(launch_overlapped(fn, (unsigned)(a.rows * blocks), kTopThreads, smem, kargs, st, blocks));
}

int fastsgd_distill_loss(const fastsgd_matrix* student, const fastsgd_pairs* teacher, float temperature, const float* weight,
                         float* loss, float* stats, const fastsgd_matrix* grad, void* stream) {
    if (!loss && !stats && !grad) return FASTSGD_E_NULL;
    return distill(grad ? kLossAndGrad : kLossOnly, student, teacher, temperature, weight, loss, stats, nullptr, nullptr, grad, stream);
}

int fastsgd_distill_loss_backward(const fastsgd_matrix* student, const fastsgd_pairs* teacher, float temperature, const float* weight,
                                  const float* stats, const float* grad_loss, const fastsgd_matrix* grad, void* stream) {
    if (!grad) return FASTSGD_E_NULL;
    if (student && student->rows && !stats) return FASTSGD_E_NULL;
    return distill(kGradOnly, student, teacher, temperature, weight, nullptr, nullptr, stats, grad_loss, grad, stream);
}

int fastsgd_expert_counts(const int32_t* selected, uint64_t tokens, uint32_t k, uint32_t experts, const uint8_t* mask,
                          const uint64_t* offsets, uint32_t segments, uint32_t* counts, uint32_t* counted, void* stream) {
    int rc = check_tokens(tokens, segments, offsets);
    if (rc) return rc;
    if (experts < 1u || experts > kBalanceMaxExperts || k < 1u || k > experts) return FASTSGD_E_BAD_PARAM;
    if (!counts || !counted || (tokens && !selected)) return FASTSGD_E_NULL;
    if (!aligned_to(selected, 4) || !aligned_to(counts, 4) || !aligned_to(counted, 4)) return FASTSGD_E_ALIGN;
    if (tokens * k >= (1ull << 31)) return FASTSGD_E_BAD_N;
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    CountArgs a{};
    a.selected = selected; a.mask = mask; a.offsets = offsets; a.counts = counts; a.counted = counted;
    a.tokens = tokens; a.k = k; a.experts = experts; a.segments = segments;
    void* kargs[] = {&a};
    // A cluster per segment; for many selections in few segments (one block of a cluster of eight would count more than 2^14 of them, if
    // they are alike) two launches that spread over the GPU.  (The offsets are not known here: where one of many segments has nearly all tokens its
    // cluster counts them alone.  39 M selections in 300 equal segments: 86 us, all in one of the 300: 1760, in one segment: 112.)
    if (tokens * k <= (1ull << 17) * segments) {
        unsigned blocks = 1u;
        while (blocks < 8u && tokens * k > 2048ull * segments * blocks) blocks *= 2u;
        uint64_t grid = (uint64_t)segments * blocks;
        const uint64_t most = (uint64_t)dev.sm_count / 8u * 8u * 4u;
        if (grid > most) grid = most;
        return launched(launch_overlapped((const void*)k_expert_counts, (unsigned)grid, kCountThreads, 0, kargs, st, blocks));
    }
    a.rows_per_block = rows_per_block(tokens, 64u, (uint64_t)dev.sm_count);
    const unsigned grid = (unsigned)((tokens + a.rows_per_block - 1) / a.rows_per_block);
    const uint64_t cells = ((uint64_t)segments * experts + kCountThreads - 1) / kCountThreads;
    rc = launched(launch_overlapped((const void*)k_clear_counts, (unsigned)(cells < 512u ? cells : 512u), kCountThreads, 0, kargs, st));
    return rc ? rc : launched(launch_overlapped((const void*)k_add_expert_counts, grid, kCountThreads, 0, kargs, st));
}

int fastsgd_balance_loss(const fastsgd_matrix* logits, const uint8_t* mask, const uint64_t* offsets, uint32_t segments,
                         const uint32_t* counts, const uint32_t* counted, float coef, const float* grad_loss,
                         float* loss, const fastsgd_matrix* grad, void* stream) {
    int rc = check_matrix(logits);
    if (rc) return rc;
    rc = check_tokens(logits->rows, segments, offsets);
    if (rc) return rc;
    if ((!loss && !grad) || !counts || !counted) return FASTSGD_E_NULL;
    if (logits->cols > kBalanceMaxExperts || !std::isfinite(coef)) return FASTSGD_E_BAD_PARAM;
    if (!aligned_to(counts, 4) || !aligned_to(counted, 4) || !aligned_to(grad_loss, 4) || !aligned_to(loss, 4)) return FASTSGD_E_ALIGN;
    if (grad) { rc = check_grad(grad, logits); if (rc) return rc; }
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (loss && (!dev.ws || dev.ws_bytes < kPartialsOffset + 8ull * (kBalanceMaxBlocks + (uint64_t)segments))) return FASTSGD_E_NO_WORKSPACE;
    if (!logits->rows) {
        if (loss && cudaMemsetAsync(loss, 0, 4ull * segments, st) != cudaSuccess) { cudaGetLastError(); return FASTSGD_E_CUDA; }
        return FASTSGD_OK;
    }
    BalanceArgs a{};
    a.x = logits->data; a.x_stride = logits->row_stride; a.tokens = logits->rows; a.experts = (uint32_t)logits->cols;
    if (grad) { a.grad = grad->data; a.grad_stride = grad->row_stride; }
    a.mask = mask; a.offsets = offsets; a.segments = segments; a.counts = counts; a.counted = counted; a.grad_loss = grad_loss;
    a.loss = loss; a.coef = coef;
    a.partials = reinterpret_cast<double*>(static_cast<unsigned char*>(dev.ws) + kPartialsOffset);
    a.done = loss ? &static_cast<Control*>(dev.ws)->loss_done : nullptr;
    const void* fn = balance_kernel(logits->type, grad ? grad->type : logits->type, a.experts);
    uint64_t blocks = 0;
    rc = resident_blocks(fn, kBalanceThreads, 0, dev, &blocks);
    if (rc) return rc;
    if (blocks > kBalanceMaxBlocks) blocks = kBalanceMaxBlocks;
    // whole steps of a block: every group of lanes as many tokens
    const uint32_t lanes = balance_lanes(logits->type, a.experts);
    const uint64_t step = (uint64_t)kBalanceWarps * (32u / lanes);
    a.rows_per_block = (uint32_t)((rows_per_block(a.tokens, 1u, blocks) + step - 1) / step * step);
    void* kargs[] = {&a};
    const unsigned grid = (unsigned)((a.tokens + a.rows_per_block - 1) / a.rows_per_block);
    return launched(launch_overlapped(fn, grid, kBalanceThreads, 0, kargs, st));
}

}  // extern "C"
