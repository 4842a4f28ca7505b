// C-ABI entries of the operators on rows that are chosen by an id: ids in order, an embedding's lookup and gradient, a router's
// experts' products.  Argument checks and launches on the caller's stream, as in losses.cu.
#include <atomic>
#include <initializer_list>

#include "host.cuh"
#include "order.cuh"
#include "embed.cuh"
#include "experts.cuh"

namespace {

using namespace fsg;

bool apart(const void* p, uint64_t p_bytes, const void* q, uint64_t q_bytes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return !p || !q || a + p_bytes <= b || b + q_bytes <= a;
}
// What a call writes lies apart from the whole numbers that it reads: blocks read them while others write.
struct Words { const void* data; uint64_t count; };
bool apart(const void* p, uint64_t p_bytes, std::initializer_list<Words> words) {
    for (const Words& w : words) if (!apart(p, p_bytes, w.data, 4u * w.count)) return false;
    return true;
}
bool apart(const fastsgd_matrix* p, const fastsgd_matrix* q) { return apart(p->data, span_bytes(p), q->data, span_bytes(q)); }

// one of the two is of 32 bits, or they are alike
bool types_go(uint32_t from, uint32_t to) { return from == to || from == FASTSGD_F32 || to == FASTSGD_F32; }
bool rows_on_16(const fastsgd_matrix* m) { return aligned_to(m->data, 16) && (m->rows < 2 || m->row_stride * size_of(m->type) % 16u == 0); }

uint64_t up_to(uint64_t x, uint64_t unit) { return (x + unit - 1) / unit * unit; }

// ---- ids in order ---------------------------------------------------------------------------------

// tiles of 1024 ids where the GPU holds them all at once, of eight times as many at most
uint64_t order_tile(uint64_t count) {
    uint64_t rounds = 1;
    while (rounds < kOrderTileRounds && count > 128u * kOrderThreads * rounds) ++rounds;
    return kOrderThreads * rounds;
}
uint64_t order_blocks(uint64_t count) { return (count + order_tile(count) - 1) / order_tile(count); }
uint64_t order_bytes(uint64_t count, uint64_t blocks) {    // behind the workspace's fixed part
    return count <= kOrderMaxFew ? 0 : 4u * up_to(4u * count, 256) + up_to(4ull * kOrderMaxBins * blocks, 256) + 4u * kOrderMaxBins;
}
uint64_t order_bytes(uint64_t count) { return order_bytes(count, order_blocks(count)); }
// ... of so many ids or fewer.  (Blocks become fewer where tiles become longer: 128 before each step.)
uint64_t most_order_bytes(uint64_t count) {
    const uint64_t blocks = order_blocks(count);
    return order_bytes(count, count > 128u * kOrderThreads && blocks < 128u ? 128u : blocks);
}

// ---- an embedding's gradient -------------------------------------------------------------------------

// Lanes that share a chunk of a row, chunks of a row, and positions of a tile: from 16 on as many as leave so many warps or fewer; of those with
// 24 warps an SM the GPU holds 3552 at once.  (us with 2^12, 2^13, 2^14 warps: 65536 x 768 bf16 of 2 rows 33, 45, 65; 65536 x 512 of 1000 rows 23, 26, 34; 30001 x 1001
// fp16 37.5, 38.5, 44.7; 49152 x 2048 bf16 52, 52, 58; pairs of 16384 x 2048 bf16 57, 49, 53: but their sums are those of the dense gradient, bit for bit.)
constexpr uint32_t kSumWarpsLog = 12u;
struct GradientShape { uint32_t lanes_log, chunks, tile_log, tiles; uint64_t part_stride; };
GradientShape gradient_shape(uint64_t count, uint64_t cols) {
    GradientShape g{};
    while (g.lanes_log < 5u && (8ull << g.lanes_log) < cols) ++g.lanes_log;
    const uint64_t chunks = (cols + (8ull << g.lanes_log) - 1) / (8ull << g.lanes_log);
    g.chunks = (uint32_t)chunks;
    g.tile_log = 4;
    while ((((count + (1ull << g.tile_log) - 1) >> g.tile_log) * chunks << g.lanes_log) > (32ull << kSumWarpsLog) && (1ull << g.tile_log) < count) ++g.tile_log;
    g.tiles = (uint32_t)((count + (1ull << g.tile_log) - 1) >> g.tile_log);
    g.part_stride = up_to(cols, 4);
    return g;
}
uint64_t part_bytes(const GradientShape& g) { return up_to(8ull * g.tiles * g.part_stride, 256) + 16ull * g.tiles; }
// ... of so many rows and columns or fewer: tiles become longer, and fewer, where rows or columns become more.  Tiles x chunks x lanes are no more than
// the warps allow, a lane has eight columns, and there is always one tile.
uint64_t most_part_bytes(uint64_t count, uint64_t cols) {
    const uint64_t lanes = 32ull << kSumWarpsLog, stride = up_to(cols, 4);
    uint64_t tiles = (count + 15u) / 16u;
    if (tiles > lanes) tiles = lanes;
    uint64_t values = tiles * stride;
    if (values > 8u * lanes) values = 8u * lanes;
    if (count && values < stride) values = stride;
    return up_to(8u * values, 256) + 16u * tiles;
}

struct SumKernel { const void* fn; size_t smem; };
template <class T, class TO, bool WIDE, bool PAIRS> SumKernel sum_kernel_as(bool full) {
    if (!full) return {(const void*)k_embedding_sum<T, TO, WIDE, PAIRS, false>, 0};
    if constexpr (WIDE) return {(const void*)k_embedding_sum<T, TO, true, PAIRS, true>, 0};
    else return {(const void*)k_embedding_sum_shifted<T, TO, PAIRS>, sizeof(SumShared<T>)};
}
template <class T, bool WIDE, bool PAIRS> SumKernel sum_kernel_of(uint32_t to, bool full) {
    if constexpr (PAIRS) return sum_kernel_as<T, float, WIDE, true>(full);
    else {
        if (to == FASTSGD_F32) return sum_kernel_as<T, float, WIDE, false>(full);
        if constexpr (sizeof(T) == 4) return to == FASTSGD_BF16 ? sum_kernel_as<T, __nv_bfloat16, WIDE, false>(full) : sum_kernel_as<T, __half, WIDE, false>(full);
        else return sum_kernel_as<T, T, WIDE, false>(full);
    }
}
template <bool WIDE, bool PAIRS> SumKernel sum_kernel_for(uint32_t from, uint32_t to, bool full) {
    return from == FASTSGD_F32 ? sum_kernel_of<float, WIDE, PAIRS>(to, full) : from == FASTSGD_BF16 ? sum_kernel_of<__nv_bfloat16, WIDE, PAIRS>(to, full) : sum_kernel_of<__half, WIDE, PAIRS>(to, full);
}
template <bool WIDE, bool PAIRS> const void* join_kernel(uint32_t to) {
    if constexpr (PAIRS) return (const void*)k_embedding_join<float, WIDE, true>;
    else return to == FASTSGD_F32 ? (const void*)k_embedding_join<float, WIDE, false> : to == FASTSGD_BF16 ? (const void*)k_embedding_join<__nv_bfloat16, WIDE, false>
                                                                                       : (const void*)k_embedding_join<__half, WIDE, false>;
}
template <class T, bool WIDE, bool SHORT> const void* lookup_kernel_of(uint32_t to) {
    if (to == FASTSGD_F32) return (const void*)k_embedding<T, float, WIDE, SHORT>;
    if constexpr (sizeof(T) == 4) return to == FASTSGD_BF16 ? (const void*)k_embedding<T, __nv_bfloat16, WIDE, SHORT> : (const void*)k_embedding<T, __half, WIDE, SHORT>;
    else return (const void*)k_embedding<T, T, WIDE, SHORT>;
}
template <bool WIDE, bool SHORT> const void* lookup_kernel(uint32_t from, uint32_t to) {
    return from == FASTSGD_F32 ? lookup_kernel_of<float, WIDE, SHORT>(to) : from == FASTSGD_BF16 ? lookup_kernel_of<__nv_bfloat16, WIDE, SHORT>(to) : lookup_kernel_of<__half, WIDE, SHORT>(to);
}
int launch_lookup(const fastsgd_matrix* table, const int32_t* ids, uint32_t per_row, float scale, const fastsgd_matrix* out, const DeviceView& dev, cudaStream_t st) {
    const GradientShape g = gradient_shape(1, table->cols);
    LookupArgs a{};
    a.table = table->data; a.table_stride = table->row_stride; a.ids = ids; a.per_row = per_row;
    a.count = (uint32_t)out->rows; a.vocab = (uint32_t)table->rows; a.cols = (uint32_t)table->cols;
    a.lanes_log = g.lanes_log; a.scale = scale; a.out = out->data; a.out_stride = out->row_stride;
    const bool wide = rows_on_16(table) && rows_on_16(out), brief = g.chunks == 1u;
    a.spans = (g.chunks + kLookupAhead - 1u) / kLookupAhead;
    a.units = brief ? (out->rows + kLookupAhead - 1u) / kLookupAhead : out->rows * a.spans;
    const uint64_t groups = (uint64_t)kEmbedThreads >> g.lanes_log, blocks = (a.units + groups - 1) / groups;
    if (blocks >= 1ull << 31) return FASTSGD_E_BAD_N;
    void* kargs[] = {&a};
    const void* fn = wide ? (brief ? lookup_kernel<true, true>(table->type, out->type) : lookup_kernel<true, false>(table->type, out->type))
                          : (brief ? lookup_kernel<false, true>(table->type, out->type) : lookup_kernel<false, false>(table->type, out->type));
    return launched(launch_overlapped(fn, (unsigned)blocks, kEmbedThreads, 0, kargs, st));
}

template <bool PAIRS> int launch_gradient(GradientArgs& a, const GradientShape& g, bool wide, uint32_t from, uint32_t to, const DeviceView& dev, cudaStream_t st) {
    if (part_bytes(g) && (!dev.ws || dev.ws_bytes < kPartialsOffset + part_bytes(g))) return FASTSGD_E_NO_WORKSPACE;
    a.lanes_log = g.lanes_log; a.chunks = g.chunks; a.tile_log = g.tile_log; a.tiles = g.tiles; a.part_stride = g.part_stride;
    a.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(dev.ws) + kPartialsOffset);
    a.follow = reinterpret_cast<uint4*>(static_cast<unsigned char*>(dev.ws) + kPartialsOffset + up_to(8ull * g.tiles * g.part_stride, 256));
    const uint64_t groups = (uint64_t)kEmbedThreads >> g.lanes_log;
    a.sum_blocks = (uint32_t)(((uint64_t)g.tiles * g.chunks + groups - 1) / groups);
    uint64_t blocks = a.sum_blocks;
    if (!PAIRS) {                                          // (eight blocks an SM that clear, of 64 rows at most)
        a.clear_rows = 1u;
        while (a.clear_rows < 64u && a.vocab > a.clear_rows * 8ull * (uint64_t)dev.sm_count) a.clear_rows *= 2u;
        a.clear_blocks = (a.vocab + a.clear_rows - 1u) / a.clear_rows;
        blocks += a.clear_blocks;
    }
    if (blocks >= 1ull << 31 || (uint64_t)g.tiles * g.chunks >= 1ull << 31) return FASTSGD_E_BAD_N;
    void* kargs[] = {&a};
    if (blocks) {
        const SumKernel k = wide ? sum_kernel_for<true, PAIRS>(from, to, g.lanes_log == 5u) : sum_kernel_for<false, PAIRS>(from, to, g.lanes_log == 5u);
        uint64_t resident = 0;
        int rc = resident_blocks(k.fn, kEmbedThreads, k.smem, dev, &resident);
        if (!rc) rc = launched(launch_overlapped(k.fn, (unsigned)blocks, kEmbedThreads, k.smem, kargs, st));
        if (rc) return rc;
    }
    if (g.tiles < 2u) return FASTSGD_OK;
    return launched(launch_overlapped(wide ? join_kernel<true, PAIRS>(to) : join_kernel<false, PAIRS>(to), (g.tiles + kJoinTiles - 1u) / kJoinTiles * g.chunks, kEmbedThreads, 0, kargs, st));
}

// ---- experts' products ----------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static std::atomic<EncodeTiled> known{nullptr};
    EncodeTiled fn = known.load(std::memory_order_relaxed);
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) { cudaGetLastError(); return nullptr; }
        fn = reinterpret_cast<EncodeTiled>(p);
        known.store(fn, std::memory_order_relaxed);
    }
    return fn;
}
// A map of a matrix of 16-bit values (experts > 0: of so many of them) for boxes of 64 columns and box_rows rows.
int map_rows(CUtensorMap* map, const void* data, uint32_t type, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t box_rows, uint64_t experts = 0, uint64_t expert_stride = 0) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return FASTSGD_E_CUDA;
    const cuuint64_t dims[3] = {cols, rows, experts}, strides[2] = {stride * 2u, expert_stride * 2u};
    const cuuint32_t box[3] = {64u, box_rows, 1u}, steps[3] = {1u, 1u, 1u};
    const CUresult rc = encode(map, type == FASTSGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, experts ? 3u : 2u, const_cast<void*>(data), dims, strides, box, steps,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? FASTSGD_OK : FASTSGD_E_CUDA;
}

// The map of a gradient of weights for boxes of 32 rows of 64 bytes.
int map_gradient(CUtensorMap* map, const fastsgd_experts* w) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return FASTSGD_E_CUDA;
    const uint32_t size = size_of(w->type);
    const cuuint64_t dims[3] = {w->ins, w->outs, w->experts}, strides[2] = {w->row_stride * size, w->expert_stride * size};
    const cuuint32_t box[3] = {64u / size, 32u, 1u}, steps[3] = {1u, 1u, 1u};
    const CUtensorMapDataType type = w->type == FASTSGD_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : w->type == FASTSGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const CUresult rc = encode(map, type, 3u, w->data, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? FASTSGD_OK : FASTSGD_E_CUDA;
}

// Rows of a product: of 16 bits (an output: or of 32), on 16 bytes, in vectors of 8 values.
int check_product_rows(const fastsgd_matrix* m, bool output) {
    const int rc = check_matrix(m);
    if (rc) return rc;
    if (!output && m->type == FASTSGD_F32) return FASTSGD_E_NOT_IMPLEMENTED;
    if (!aligned_to(m->data, 16) || m->cols % 8u || m->row_stride % 8u) return FASTSGD_E_ALIGN;
    return FASTSGD_OK;
}
int check_experts(const fastsgd_experts* w, bool output) {
    if (!w || !w->data) return FASTSGD_E_NULL;
    if (!is_type(w->type) || w->reserved || w->experts < 1 || w->experts > kProductMaxExperts) return FASTSGD_E_BAD_PARAM;
    if (!w->outs || !w->ins || w->outs >= 1ull << 31 || w->ins >= 1ull << 31) return FASTSGD_E_BAD_N;
    if (w->row_stride < w->ins || w->row_stride >= 1ull << 31 || w->expert_stride / w->row_stride < w->outs || w->expert_stride >= 1ull << 38) return FASTSGD_E_BAD_PARAM;
    if (!output && w->type == FASTSGD_F32) return FASTSGD_E_NOT_IMPLEMENTED;
    if (!aligned_to(w->data, 16) || w->ins % 8u || w->outs % 8u || w->row_stride % 8u || w->expert_stride % 8u) return FASTSGD_E_ALIGN;
    return FASTSGD_OK;
}
// Rows in the order of their experts.  Rows by an order are laid out in the workspace first: fetched within the product, once for each 256 of
// the weights' rows, they take longer (16384 x 4096 x 14336, 8 experts: 1245 us of sorted rows, 1900 to 2140 fetched, by their own copies of
// four rows or 16 bytes a thread alike; laid out 60 more).
uint64_t sorted_bytes(uint64_t rows, uint64_t cols) { return up_to(rows * cols * 2u, 256); }
int sort_rows(const fastsgd_matrix* x, const uint32_t* order, uint32_t per_row, uint64_t rows, const DeviceView& dev, cudaStream_t st, fastsgd_matrix* sorted) {
    *sorted = *x;
    if (!order) return FASTSGD_OK;
    if (!dev.ws || dev.ws_bytes < kPartialsOffset + sorted_bytes(rows, x->cols)) return FASTSGD_E_NO_WORKSPACE;
    sorted->data = static_cast<unsigned char*>(dev.ws) + kPartialsOffset;
    sorted->rows = rows; sorted->row_stride = x->cols;
    return launch_lookup(x, reinterpret_cast<const int32_t*>(order), per_row, 1.f, sorted, dev, st);
}
uint64_t span_bytes(const fastsgd_experts* w) { return ((w->experts - 1) * w->expert_stride + (w->outs - 1) * w->row_stride + w->ins) * size_of(w->type); }

template <class TO, int MODE> const void* product_kernel_of(bool sums, bool split) {
    if (split) return (const void*)k_product<TO, MODE, true, true>;
    if constexpr (sizeof(TO) == 4) return (const void*)k_product<TO, MODE, true, false>;
    else return sums ? (const void*)k_product<TO, MODE, true, false> : (const void*)k_product<TO, MODE, false, false>;
}
template <int MODE> const void* product_kernel(uint32_t to, bool sums, bool split) {
    return to == FASTSGD_F32 ? product_kernel_of<float, MODE>(sums, split) : to == FASTSGD_BF16 ? product_kernel_of<__nv_bfloat16, MODE>(sums, split) : product_kernel_of<__half, MODE>(sums, split);
}

// `tiles`: at most; `steps`: of a contraction, about
template <int MODE> int launch_product(ProductArgs& a, uint64_t tiles, uint64_t steps, uint32_t to, const DeviceView& dev, cudaStream_t st) {
    if (tiles >= 1ull << 31) return FASTSGD_E_BAD_N;
    a.tries = dev.tries;
    const uint32_t turned = MODE == kWeights ? 8u * kProductTurned : 0u;
    a.stages = (uint32_t)((215u * 1024u - turned) / product_stage_bytes<MODE>(a.most_n));
    if (a.stages > kProductMaxStages) a.stages = kProductMaxStages;
    // Few tiles of a contraction of at least `least` stages: up to eight pairs of blocks share it, as long as each has eight stages, and as clusters
    // of them all find room at once (of sixteen blocks one in each of the GPU's groups of 16 to 20 SMs, of eight and four two and four).  Adding up
    // wide tiles takes as long as some 30 stages, and those of the weights' gradients are 256 wide.  Unshared and shared, us:
    //   8 rows, 1024 / 2048 / 4096 -> 512: 7.3, 10.5, 16.9 and 7.3, 7.4, 7.7;  200 rows, 2048 -> 1024: 13.5 and 11.0, 1024 -> 2048: 9.7 and 12.1
    //   gradient of 512 x 512 weights, 2000 / 3000 / 4096 / 60000 rows: 14.4, 18.1, 22.9, 267 and 16.1, 13.1, 14.0, 48
    const uint64_t least = a.most_n <= 64u ? 16u : MODE == kWeights ? 48u : 32u;
    a.splits = 1u;
    while (a.splits < 8u && tiles * a.splits * 2u <= 8ull * ((uint64_t)dev.sm_count / 20u) && steps >= (a.splits > 1u ? a.splits * 16ull : least)) a.splits *= 2u;
    const uint64_t longest = MODE == kWeights ? a.rows : a.k;
    const void* fn = product_kernel<MODE>(to, longest > (to == FASTSGD_F16 ? kProductLongF16 : kProductLongBF16), a.splits > 1u);
    a.sum_stages = to == FASTSGD_F32 || a.splits > 1u ? kProductSum : kProductLongSum;
    const size_t smem = (size_t)a.stages * product_stage_bytes<MODE>(a.most_n) + turned + 1024u;
    uint64_t resident = 0;
    const int rc = resident_blocks(fn, kProductThreads, smem, dev, &resident);
    if (rc) return rc;
    const uint64_t clusters = a.splits > 1u || tiles < resident / 2u ? tiles : resident / 2u;
    void* kargs[] = {&a};
    return launched(launch_overlapped(fn, (unsigned)(2u * a.splits * clusters), kProductThreads, smem, kargs, st, 2u * a.splits));
}

// tiles of the rows, at most: every expert that has any may have one that is not full
uint64_t row_tiles(uint64_t rows, uint64_t experts, uint32_t most_n) { return rows / most_n + (experts < rows ? experts : rows); }
// Columns of a tile where the rows' side is ragged: enough for most experts' rows in one.
uint32_t columns_for(uint64_t rows, uint64_t experts) {
    uint32_t n = 32u;
    while (n < 256u && n * experts < 2u * rows) n *= 2u;
    return n;
}

}  // namespace

extern "C" {

uint64_t fastsgd_rows_workspace_bytes(uint64_t count, uint64_t cols) {
    if (count >= (1ull << 31) || cols < 1 || cols >= (1ull << 31)) return 0;
    const uint64_t order = most_order_bytes(count), parts = most_part_bytes(count, cols);
    return up_to(kPartialsOffset + (order > parts ? order : parts), 256);
}

uint64_t fastsgd_products_workspace_bytes(uint64_t rows, uint64_t ins) {
    if (rows >= (1ull << 31) || ins < 1 || ins >= (1ull << 31)) return 0;
    const uint64_t order = most_order_bytes(rows), sorted = sorted_bytes(rows, ins);
    return up_to(kPartialsOffset + (order > sorted ? order : sorted), 256);
}

int fastsgd_order_ids(const int32_t* ids, uint64_t count, uint64_t range, uint32_t* order, uint32_t* starts, uint32_t* distinct, uint32_t* number, void* stream) {
    if (count >= (1ull << 31)) return FASTSGD_E_BAD_N;
    if (range < 1) return FASTSGD_E_BAD_PARAM;
    if ((count && (!ids || !order)) || !starts) return FASTSGD_E_NULL;
    if (!aligned_to(ids, 4) || !aligned_to(order, 4) || !aligned_to(starts, 4) || !aligned_to(distinct, 4) || !aligned_to(number, 4)) return FASTSGD_E_ALIGN;
    if (range > kOrderMaxRange) return FASTSGD_E_NOT_IMPLEMENTED;
    const uint64_t some = count < range ? count : range;
    if (!apart(order, 4u * count, {{ids, count}, {starts, range + 1u}, {distinct, some}, {number, 1u}}) || !apart(starts, 4u * (range + 1u), {{ids, count}, {distinct, some}, {number, 1u}})
        || !apart(distinct, 4u * some, {{ids, count}, {number, 1u}}) || !apart(number, 4u, {{ids, count}})) return FASTSGD_E_BAD_PARAM;
    DeviceView dev;
    int rc = device_view(&dev);
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    OrderArgs a{};
    a.ids = ids; a.count = (uint32_t)count; a.range = (uint32_t)range; a.order = order; a.starts = starts; a.distinct = distinct; a.number = number;
    uint32_t width = 1;                                    // of the keys, the range itself among them
    while ((range >> width) != 0) ++width;
    a.passes = (width + 9u) / 10u;
    a.bits = (width + a.passes - 1u) / a.passes;
    void* kargs[] = {&a};
    uint64_t resident = 0;
    if (count <= kOrderMaxFew) {
        rc = resident_blocks((const void*)k_order, kOrderThreads, sizeof(OrderShared), dev, &resident);
        return rc ? rc : launched(launch_overlapped((const void*)k_order, kOrderBlocks, kOrderThreads, sizeof(OrderShared), kargs, st, kOrderBlocks));
    }
    if (!dev.ws || dev.ws_bytes < kPartialsOffset + order_bytes(count)) return FASTSGD_E_NO_WORKSPACE;
    a.blocks = (uint32_t)order_blocks(count);
    a.tile = (uint32_t)order_tile(count);
    unsigned char* at = static_cast<unsigned char*>(dev.ws) + kPartialsOffset;
    for (uint32_t** p : {&a.keys[0], &a.keys[1], &a.places[0], &a.places[1]}) { *p = reinterpret_cast<uint32_t*>(at); at += up_to(4u * count, 256); }
    a.table = reinterpret_cast<uint32_t*>(at);
    a.totals = reinterpret_cast<uint32_t*>(at + up_to(4ull * kOrderMaxBins * a.blocks, 256));
    for (const void* fn : {(const void*)k_order_tile<0>, (const void*)k_order_tile<1>}) {
        rc = resident_blocks(fn, kOrderThreads, sizeof(OrderTileShared), dev, &resident);
        if (rc) return rc;
    }
    for (a.pass = 0; a.pass < a.passes; ++a.pass) {
        cudaError_t err = launch_overlapped((const void*)k_order_tile<0>, a.blocks, kOrderThreads, sizeof(OrderTileShared), kargs, st);
        if (err == cudaSuccess) err = launch_overlapped((const void*)k_order_offsets, (1u << a.bits) / 8u + 1u, 256, 0, kargs, st);
        if (err == cudaSuccess) err = launch_overlapped((const void*)k_order_tile<1>, a.blocks, kOrderThreads, sizeof(OrderTileShared), kargs, st);
        rc = launched(err, 3);
        if (rc) return rc;
    }
    rc = launched(launch_overlapped((const void*)k_order_starts, a.range / 256u + 1u, 256, 0, kargs, st));
    if (rc || (!distinct && !number)) return rc;
    rc = resident_blocks((const void*)k_order_distinct, kOrderThreads, 0, dev, &resident);
    if (rc) return rc;
    return launched(launch_overlapped((const void*)k_order_distinct, kOrderBlocks, kOrderThreads, 0, kargs, st, kOrderBlocks));
}

int fastsgd_embedding(const fastsgd_matrix* table, const int32_t* ids, float scale, const fastsgd_matrix* out, void* stream) {
    int rc = check_matrix(table);
    if (rc) return rc;
    rc = check_matrix(out);
    if (rc) return rc;
    if (table->cols != out->cols || !types_go(table->type, out->type) || !apart(table, out)) return FASTSGD_E_BAD_PARAM;
    if (out->rows && !ids) return FASTSGD_E_NULL;
    if (!aligned_to(ids, 4)) return FASTSGD_E_ALIGN;
    if (!apart(out->data, span_bytes(out), {{ids, out->rows}})) return FASTSGD_E_BAD_PARAM;
    if (!out->rows) return FASTSGD_OK;
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    return launch_lookup(table, ids, 1u, scale, out, dev, static_cast<cudaStream_t>(stream));
}

int fastsgd_embedding_backward(const fastsgd_matrix* grad, const int32_t* ids, const uint32_t* order, const uint32_t* starts, float scale, const fastsgd_matrix* table_grad, void* stream) {
    int rc = check_matrix(grad);
    if (rc) return rc;
    rc = check_matrix(table_grad);
    if (rc) return rc;
    if (grad->cols != table_grad->cols || !types_go(grad->type, table_grad->type) || !apart(grad, table_grad)) return FASTSGD_E_BAD_PARAM;
    if ((grad->rows && (!ids || !order)) || !starts) return FASTSGD_E_NULL;
    if (!aligned_to(ids, 4) || !aligned_to(order, 4) || !aligned_to(starts, 4)) return FASTSGD_E_ALIGN;
    if (!table_grad->rows) return FASTSGD_E_BAD_N;
    if (!apart(table_grad->data, span_bytes(table_grad), {{ids, grad->rows}, {order, grad->rows}, {starts, table_grad->rows + 1u}})) return FASTSGD_E_BAD_PARAM;
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    GradientArgs a{};
    a.grad = grad->data; a.grad_stride = grad->row_stride; a.ids = ids; a.order = order; a.starts = starts;
    a.count = (uint32_t)grad->rows; a.vocab = (uint32_t)table_grad->rows; a.cols = (uint32_t)grad->cols; a.scale = scale; a.out = table_grad->data; a.out_stride = table_grad->row_stride;
    return launch_gradient<false>(a, gradient_shape(grad->rows, grad->cols), rows_on_16(grad) && rows_on_16(table_grad), grad->type, table_grad->type, dev, static_cast<cudaStream_t>(stream));
}

int fastsgd_embedding_backward_pairs(const fastsgd_matrix* grad, const int32_t* ids, const uint32_t* order, const uint32_t* starts, const uint32_t* distinct, const uint32_t* number,
                                     uint64_t range, float scale, uint32_t* keys, float* values, uint64_t most, void* stream) {
    int rc = check_matrix(grad);
    if (rc) return rc;
    if (range < 1 || range * grad->cols >= (1ull << 31) || range >= (1ull << 31) || most >= (1ull << 31)) return FASTSGD_E_BAD_N;
    if (!starts || !number || (grad->rows && (!ids || !order || !distinct)) || (most && (!keys || !values))) return FASTSGD_E_NULL;
    if (!aligned_to(ids, 4) || !aligned_to(order, 4) || !aligned_to(starts, 4) || !aligned_to(distinct, 4) || !aligned_to(number, 4) || !aligned_to(keys, 4) || !aligned_to(values, 4))
        return FASTSGD_E_ALIGN;
    const uint64_t bytes = 4u * most * grad->cols;
    if (!apart(grad->data, span_bytes(grad), keys, bytes) || !apart(grad->data, span_bytes(grad), values, bytes) || !apart(keys, bytes, values, bytes)) return FASTSGD_E_BAD_PARAM;
    const uint64_t some = grad->rows < range ? grad->rows : range;
    for (const void* written : {static_cast<const void*>(keys), static_cast<const void*>(values)})
        if (!apart(written, bytes, {{ids, grad->rows}, {order, grad->rows}, {starts, range + 1u}, {distinct, some}, {number, 1u}})) return FASTSGD_E_BAD_PARAM;
    if (!grad->rows) return FASTSGD_OK;
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    GradientArgs a{};
    a.grad = grad->data; a.grad_stride = grad->row_stride; a.ids = ids; a.order = order; a.starts = starts; a.distinct = distinct; a.number = number;
    a.count = (uint32_t)grad->rows; a.vocab = (uint32_t)range; a.cols = (uint32_t)grad->cols; a.scale = scale; a.keys = keys; a.values = values;
    a.most = (uint32_t)(most < grad->rows ? most : grad->rows);      // (no more ids occur than there are rows, or ids)
    if (a.most > a.vocab) a.most = a.vocab;
    const bool wide = rows_on_16(grad) && aligned_to(keys, 16) && aligned_to(values, 16) && grad->cols % 4u == 0;
    return launch_gradient<true>(a, gradient_shape(grad->rows, grad->cols), wide, grad->type, FASTSGD_F32, dev, static_cast<cudaStream_t>(stream));
}

int fastsgd_expert_product(const fastsgd_matrix* x, const uint32_t* order, uint32_t per_row, const uint32_t* starts, const fastsgd_experts* weights, const fastsgd_matrix* y, void* stream) {
    int rc = check_product_rows(x, false);
    if (!rc) rc = check_experts(weights, false);
    if (!rc) rc = check_product_rows(y, true);
    if (rc) return rc;
    if (x->cols != weights->ins || y->cols != weights->outs || x->type != weights->type || (y->type != x->type && y->type != FASTSGD_F32)) return FASTSGD_E_BAD_PARAM;
    if (per_row < 1u || (!order && per_row != 1u) || x->rows * per_row != y->rows) return FASTSGD_E_BAD_PARAM;
    if (!apart(x, y) || !apart(weights->data, span_bytes(weights), y->data, span_bytes(y))) return FASTSGD_E_BAD_PARAM;
    if (!starts) return FASTSGD_E_NULL;
    if (!aligned_to(order, 4) || !aligned_to(starts, 4)) return FASTSGD_E_ALIGN;
    if (!apart(y->data, span_bytes(y), {{order, y->rows}, {starts, weights->experts + 1u}})) return FASTSGD_E_BAD_PARAM;
    if (!y->rows || !x->rows) return FASTSGD_OK;
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    fastsgd_matrix sorted;
    rc = sort_rows(x, order, per_row, y->rows, dev, static_cast<cudaStream_t>(stream), &sorted);
    if (rc) return rc;
    ProductArgs a{};
    a.most_n = columns_for(y->rows, weights->experts);
    a.box = a.most_n < 128u ? a.most_n / 2u : 64u;
    rc = map_rows(&a.a_map, weights->data, weights->type, weights->outs, weights->ins, weights->row_stride, kProductM / 2u, weights->experts, weights->expert_stride);
    if (!rc) rc = map_rows(&a.b_map, sorted.data, x->type, sorted.rows, x->cols, sorted.row_stride, a.box);
    if (rc) return rc;
    a.starts = starts; a.experts = (uint32_t)weights->experts; a.rows = (uint32_t)y->rows;
    a.m = (uint32_t)weights->outs; a.k = (uint32_t)weights->ins; a.out = y->data; a.out_stride = y->row_stride;
    a.kind = product_kind(x->type == FASTSGD_BF16, false, false);
    return launch_product<kForward>(a, row_tiles(y->rows, weights->experts, a.most_n) * ((weights->outs + kProductM - 1) / kProductM), weights->ins / kProductK, y->type, dev, static_cast<cudaStream_t>(stream));
}

int fastsgd_expert_product_backward_input(const fastsgd_matrix* grad_y, const uint32_t* starts, const fastsgd_experts* weights, const fastsgd_matrix* grad_x, void* stream) {
    int rc = check_product_rows(grad_y, false);
    if (!rc) rc = check_experts(weights, false);
    if (!rc) rc = check_product_rows(grad_x, true);
    if (rc) return rc;
    if (grad_y->cols != weights->outs || grad_x->cols != weights->ins || grad_y->rows != grad_x->rows || grad_y->type != weights->type
        || (grad_x->type != grad_y->type && grad_x->type != FASTSGD_F32)) return FASTSGD_E_BAD_PARAM;
    if (!apart(grad_y, grad_x) || !apart(weights->data, span_bytes(weights), grad_x->data, span_bytes(grad_x))) return FASTSGD_E_BAD_PARAM;
    if (!starts) return FASTSGD_E_NULL;
    if (!aligned_to(starts, 4)) return FASTSGD_E_ALIGN;
    if (!apart(grad_x->data, span_bytes(grad_x), {{starts, weights->experts + 1u}})) return FASTSGD_E_BAD_PARAM;
    if (!grad_y->rows) return FASTSGD_OK;
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    ProductArgs a{};
    a.most_n = columns_for(grad_y->rows, weights->experts);
    a.box = a.most_n < 128u ? a.most_n / 2u : 64u;
    rc = map_rows(&a.a_map, weights->data, weights->type, weights->outs, weights->ins, weights->row_stride, kProductK, weights->experts, weights->expert_stride);
    if (!rc) rc = map_rows(&a.b_map, grad_y->data, grad_y->type, grad_y->rows, grad_y->cols, grad_y->row_stride, a.box);
    if (rc) return rc;
    a.starts = starts; a.experts = (uint32_t)weights->experts; a.rows = (uint32_t)grad_y->rows;
    a.m = (uint32_t)weights->ins; a.k = (uint32_t)weights->outs; a.out = grad_x->data; a.out_stride = grad_x->row_stride;
    a.kind = product_kind(grad_y->type == FASTSGD_BF16, true, false);
    return launch_product<kInput>(a, row_tiles(grad_y->rows, weights->experts, a.most_n) * ((weights->ins + kProductM - 1) / kProductM), weights->outs / kProductK, grad_x->type, dev, static_cast<cudaStream_t>(stream));
}

int fastsgd_expert_product_backward_weights(const fastsgd_matrix* grad_y, const fastsgd_matrix* x, const uint32_t* order, uint32_t per_row, const uint32_t* starts, const fastsgd_experts* grad_weights,
                                            void* stream) {
    int rc = check_product_rows(grad_y, false);
    if (!rc) rc = check_product_rows(x, false);
    if (!rc) rc = check_experts(grad_weights, true);
    if (rc) return rc;
    if (grad_y->cols != grad_weights->outs || x->cols != grad_weights->ins || grad_y->type != x->type || (grad_weights->type != x->type && grad_weights->type != FASTSGD_F32)) return FASTSGD_E_BAD_PARAM;
    if (per_row < 1u || (!order && per_row != 1u) || x->rows * per_row != grad_y->rows) return FASTSGD_E_BAD_PARAM;
    if (!apart(grad_weights->data, span_bytes(grad_weights), grad_y->data, span_bytes(grad_y)) || !apart(grad_weights->data, span_bytes(grad_weights), x->data, span_bytes(x))) return FASTSGD_E_BAD_PARAM;
    if (!starts) return FASTSGD_E_NULL;
    if (!aligned_to(order, 4) || !aligned_to(starts, 4)) return FASTSGD_E_ALIGN;
    if (!apart(grad_weights->data, span_bytes(grad_weights), {{order, grad_y->rows}, {starts, grad_weights->experts + 1u}})) return FASTSGD_E_BAD_PARAM;
    DeviceView dev;
    rc = device_view(&dev);
    if (rc) return rc;
    ProductArgs a{};
    a.rows = x->rows ? (uint32_t)grad_y->rows : 0u;        // (none: the kernel writes zeros and uses no map)
    a.most_n = grad_weights->ins <= 64 ? 64u : grad_weights->ins <= 128 ? 128u : 256u;
    a.box = kProductK;
    if (a.rows) {
        fastsgd_matrix sorted;
        rc = sort_rows(x, order, per_row, grad_y->rows, dev, static_cast<cudaStream_t>(stream), &sorted);
        if (!rc) rc = map_rows(&a.a_map, grad_y->data, grad_y->type, grad_y->rows, grad_y->cols, grad_y->row_stride, kProductK);
        if (!rc) rc = map_rows(&a.b_map, sorted.data, x->type, sorted.rows, x->cols, sorted.row_stride, kProductK);
        if (rc) return rc;
    }
    rc = map_gradient(&a.out_map, grad_weights);
    if (rc) return rc;
    a.starts = starts; a.experts = (uint32_t)grad_weights->experts;
    a.m = (uint32_t)grad_weights->outs; a.n = (uint32_t)grad_weights->ins; a.out = grad_weights->data; a.out_stride = grad_weights->row_stride; a.out_expert = grad_weights->expert_stride;
    a.kind = product_kind(x->type == FASTSGD_BF16, true, true);
    return launch_product<kWeights>(a, grad_weights->experts * ((grad_weights->outs + kProductM - 1) / kProductM) * ((grad_weights->ins + a.most_n - 1) / a.most_n), a.rows / grad_weights->experts / kProductK,
                                    grad_weights->type, dev,
                                    static_cast<cudaStream_t>(stream));
}

}  // extern "C"
