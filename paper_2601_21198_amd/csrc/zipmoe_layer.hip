// zm_layer: the compressed experts of one MoE layer, resident in device memory (ZipMoE, arXiv 2601.21198,
// Sec. 3.1: the serialised objects made offline are what the run-time system holds).  The handle keeps what
// the hot call otherwise takes as arrays -- device addresses, chunk tables, tensor descriptions -- so that a
// caller hands over expert ids and output buffers only.  It owns no device memory: the blobs live in an arena the
// caller provides.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "zipmoe.h"
#include "zipmoe_moe.h"
#include "zipmoe_product.h"

struct zm_layer {
    int n_experts = 0, tensors_per_expert = 0;
    std::vector<zm_tensor_info> infos;
    std::vector<const void *> blobs;                // device address of every blob
    std::vector<const uint64_t *> tables;           // device address of every chunk table (inside the blob)
    size_t bytes = 0;                               // of the arena in use
};

namespace {

constexpr size_t kAlign = 256;

inline size_t aligned(size_t n) { return (n + kAlign - 1) & ~(kAlign - 1); }

// ---- experts of few tokens from their compressed form: products (zipmoe_product.h) of gate and up, middle, products of down, join ----

using namespace zipmoe;

struct LayerCall {
    const float *first, *second;    // sums of the products: [gate and up][pairs][pieces], [pairs][pieces]
    const int32_t *ids;
    const float *weights;
    const uint16_t *residual;
    uint16_t *out, *h, *h_rest;
    int64_t residual_stride, out_stride;
    uint32_t n_pairs, top_k, hidden, intermediate, stream_values, first_pieces, second_pieces;
    uint32_t n;
    int32_t id[ZM_MOE_MAX_EXPERTS];
};

// Row r of a matrix, its pieces added up in order.
__device__ __forceinline__ float row_sum(const float *pieces, uint32_t r, uint32_t width, uint32_t stream_values)
{
    const uint64_t from = static_cast<uint64_t>(r) * width;
    const uint32_t first = static_cast<uint32_t>(from / stream_values), last = static_cast<uint32_t>((from + width - 1) / stream_values);
    // the first two, all there are of most rows, without waiting for one another
    const float one = pieces[first + r], two = pieces[min(first + 1, last) + r];
    float s = last > first ? one + two : one;
    for (uint32_t g = first + 2; g <= last; ++g) s += pieces[g + r];
    return s;
}

// h = weight * silu(g) * u of every pair, in two bf16 parts; of a token that names an expert twice the first pair stands for both
__global__ void __launch_bounds__(256) zm_layer_middle_kernel(const LayerCall c)
{
    const uint32_t r = blockIdx.x * 256 + threadIdx.x, pair = blockIdx.y;
    if (r >= c.intermediate) return;
    const uint64_t gate = static_cast<uint64_t>(pair) * c.first_pieces, up = (static_cast<uint64_t>(c.n_pairs) + pair) * c.first_pieces;
    const float g = row_sum(c.first + gate, r, c.hidden, c.stream_values), u = row_sum(c.first + up, r, c.hidden, c.stream_values);
    const int32_t id = c.ids[pair];
    float weight = 0.0f;
    const uint32_t end = (pair / c.top_k + 1) * c.top_k;
    for (uint32_t p0 = pair; p0 < end; p0 += 4) {
        int32_t ids[4];
        float weights[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) ids[i] = c.ids[min(p0 + i, end - 1)], weights[i] = c.weights[min(p0 + i, end - 1)];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) weight += p0 + i < end && ids[i] == id ? weights[i] : 0.0f;
    }
    const float h = g / (1.0f + expf(-g)) * u * weight;
    const __bf16 most = static_cast<__bf16>(h);
    const float rest = h - static_cast<float>(most);
    const uint64_t at = static_cast<uint64_t>(pair) * c.intermediate + r;
    c.h[at] = __builtin_bit_cast(uint16_t, most);
    c.h_rest[at] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(fabsf(rest) < INFINITY ? rest : 0.0f));      // most tells of what is not finite
}

__global__ void __launch_bounds__(256) zm_layer_join_kernel(const LayerCall c)
{
    const uint32_t col = blockIdx.x * 256 + threadIdx.x, token = blockIdx.y, lane = threadIdx.x % 64;
    const int32_t low = lane < c.n ? c.id[lane] : 0, high = lane + 64 < c.n ? c.id[lane + 64] : 0;
    float s = 0.0f;
    if (c.residual && col < c.hidden) s = __builtin_bit_cast(float, static_cast<uint32_t>(c.residual[token * c.residual_stride + col]) << 16);
    const uint32_t start = token * c.top_k, end = start + c.top_k, own = min(col, c.hidden - 1);
    // four pairs' sums are asked for before it is known which of them count
    for (uint32_t p0 = start; p0 < end; p0 += 4) {
        int32_t ids[4];
        float y[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t p = min(p0 + i, end - 1);
            ids[i] = c.ids[p], y[i] = row_sum(c.second + static_cast<uint64_t>(p) * c.second_pieces, own, c.intermediate, c.stream_values);
        }
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            bool there = p0 + i < end && __builtin_amdgcn_ballot_w64((lane < c.n && low == ids[i]) || (lane + 64 < c.n && high == ids[i])) != 0;
#pragma unroll
            for (uint32_t q = 0; q < i; ++q) there = there && ids[q] != ids[i];
            for (uint32_t q = start; q < p0; ++q) there = there && c.ids[q] != ids[i];
            s += there ? y[i] : 0.0f;
        }
    }
    if (col < c.hidden) c.out[token * c.out_stride + col] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(s));
}

int launch(const void *fn, dim3 grid, void *call, hipStream_t stream)
{
    void *args[] = {call};
    return hipLaunchKernel(fn, grid, dim3(256), args, 0, stream) == hipSuccess ? ZM_OK : ZM_E_HIP;
}

// Whether the named experts take that way, and the bytes of its sums.
bool takes_products(const zm_layer &layer, const int32_t *ids, int n, const zm_moe_args &a, size_t &sums)
{
    const uint64_t pairs = static_cast<uint64_t>(a.n_tokens) * static_cast<uint64_t>(a.top_k);
    if (n == 0) return false;
    const uint32_t W = layer.infos[3 * ids[0]].stream_values, hidden = static_cast<uint32_t>(a.hidden), intermediate = static_cast<uint32_t>(a.intermediate);
    if (!product_fits(hidden, intermediate, W, a.n_tokens, pairs)) return false;
    bool long_codes = false;
    for (int i = 0; i < n; ++i)
        for (int m = 0; m < 3; ++m) {
            const zm_tensor_info &info = layer.infos[3 * ids[i] + m];
            if (info.stream_values != W) return false;
            long_codes = long_codes || info.max_len > 8;
        }
    if (!product_pays(hidden, intermediate, W, long_codes, a.n_tokens, pairs, static_cast<uint64_t>(n))) return false;
    const uint64_t streams = (layer.infos[3 * ids[0]].n_values + W - 1) / W;
    sums = sizeof(float) * pairs * (2 * (streams + a.intermediate) + streams + a.hidden);
    return true;
}

int layer_products(const zm_layer &layer, const int32_t *ids, int n, const zm_moe_args &a, void *workspace, float *sums, hipStream_t stream)
{
    const void *blobs[2 * ZM_MOE_MAX_EXPERTS];
    const uint64_t *tables[2 * ZM_MOE_MAX_EXPERTS];
    const zm_tensor_info *infos[2 * ZM_MOE_MAX_EXPERTS];
    auto take = [&](int i, int tensor) {
        blobs[i] = layer.blobs[tensor], tables[i] = layer.tables[tensor], infos[i] = &layer.infos[tensor];
    };
    const MoePlaces to = moe_places(workspace, a);
    const uint32_t W = layer.infos[3 * ids[0]].stream_values, pairs = static_cast<uint32_t>(a.n_tokens * a.top_k);
    const uint32_t streams = static_cast<uint32_t>((layer.infos[3 * ids[0]].n_values + W - 1) / W);
    LayerCall c;
    c.first_pieces = streams + static_cast<uint32_t>(a.intermediate), c.second_pieces = streams + static_cast<uint32_t>(a.hidden);
    float *const second = sums + 2ull * pairs * c.first_pieces;
    c.first = sums, c.second = second, c.ids = a.ids, c.weights = a.weights, c.residual = static_cast<const uint16_t *>(a.residual);
    c.out = static_cast<uint16_t *>(a.out), c.h = to.h, c.h_rest = to.h_rest, c.residual_stride = a.residual_stride, c.out_stride = a.out_stride;
    c.n_pairs = pairs, c.top_k = static_cast<uint32_t>(a.top_k), c.hidden = static_cast<uint32_t>(a.hidden), c.intermediate = static_cast<uint32_t>(a.intermediate);
    c.stream_values = W, c.n = static_cast<uint32_t>(n);
    for (int i = 0; i < n; ++i) c.id[i] = ids[i];

    ProductCall product{a.ids, static_cast<const uint16_t *>(a.x), nullptr, sums, a.x_stride, pairs, c.top_k, 0, c.hidden, c.first_pieces};
    int status = ZM_OK;
    if (a.x_type == ZM_MXFP8) {
        status = moe_widen(a, to, stream);
        product.x = to.wide_x, product.x_stride = to.wide_stride;
    }
    for (int i = 0; i < 2 * n; ++i) take(i, 3 * ids[i / 2] + i % 2);
    if (status == ZM_OK) status = product_launch(blobs, tables, infos, ids, 2 * n, 2, product, stream);
    if (status == ZM_OK) status = launch(reinterpret_cast<const void *>(&zm_layer_middle_kernel), dim3((c.intermediate + 255) / 256, pairs), &c, stream);
    product = {a.ids, to.h, to.h_rest, second, a.intermediate, pairs, c.top_k, 1, c.intermediate, c.second_pieces};
    for (int i = 0; i < n; ++i) take(i, 3 * ids[i] + 2);
    if (status == ZM_OK) status = product_launch(blobs, tables, infos, ids, n, 1, product, stream);
    if (status == ZM_OK) status = launch(reinterpret_cast<const void *>(&zm_layer_join_kernel), dim3((c.hidden + 255) / 256, static_cast<uint32_t>(a.n_tokens)), &c, stream);
    return status;
}

}  // namespace

extern "C" {

int zm_layer_arena_bytes(const size_t *blob_sizes, int n_tensors, size_t *bytes)
{
    if (!blob_sizes || !bytes || n_tensors <= 0) return ZM_E_ARG;
    size_t total = 0;
    for (int i = 0; i < n_tensors; ++i) {
        const size_t a = aligned(blob_sizes[i]);
        if (a < blob_sizes[i] || total + a < total) return ZM_E_ARG;
        total += a;
    }
    *bytes = total;
    return ZM_OK;
}

int zm_layer_create(const void *const *host_blobs, const size_t *blob_sizes, int n_experts, int tensors_per_expert,
                    void *arena, size_t arena_bytes, zm_layer **out)
{
    if (out) *out = nullptr;
    if (!host_blobs || !blob_sizes || !arena || !out || n_experts <= 0 || tensors_per_expert <= 0 ||
        static_cast<int64_t>(n_experts) * tensors_per_expert > (1 << 24) ||
        (reinterpret_cast<uintptr_t>(arena) & (kAlign - 1))) return ZM_E_ARG;
    const int n = n_experts * tensors_per_expert;
    size_t need = 0;
    int rc = zm_layer_arena_bytes(blob_sizes, n, &need);
    if (rc != ZM_OK) return rc;
    if (need > arena_bytes) return ZM_E_SIZE;
    zm_layer *L = new (std::nothrow) zm_layer;
    if (!L) return ZM_E_NOMEM;
    try {
        L->infos.resize(n);
        L->blobs.resize(n);
        L->tables.resize(n);
    } catch (const std::bad_alloc &) {
        delete L;
        return ZM_E_NOMEM;
    }
    L->n_experts = n_experts;
    L->tensors_per_expert = tensors_per_expert;
    // every blob is checked in full before the first byte is uploaded: the kernels trust what is resident
    for (int i = 0; i < n; ++i) {
        if (!host_blobs[i]) rc = ZM_E_ARG;
        if (rc == ZM_OK) rc = zm_validate_blob(host_blobs[i], blob_sizes[i]);
        if (rc == ZM_OK) rc = zm_blob_info(host_blobs[i], blob_sizes[i], &L->infos[i]);
        if (rc == ZM_OK && L->infos[i].blob_size != blob_sizes[i]) rc = ZM_E_FORMAT;
        if (rc != ZM_OK) {
            delete L;
            return rc;
        }
    }
    uint8_t *at = static_cast<uint8_t *>(arena);
    for (int i = 0; i < n; ++i) {
        if (hipMemcpy(at, host_blobs[i], blob_sizes[i], hipMemcpyHostToDevice) != hipSuccess) {
            delete L;
            return ZM_E_HIP;
        }
        L->blobs[i] = at;
        L->tables[i] = reinterpret_cast<const uint64_t *>(at + L->infos[i].table_offset);
        at += aligned(blob_sizes[i]);
    }
    L->bytes = need;
    *out = L;
    return ZM_OK;
}

int zm_layer_tensor_info(const zm_layer *layer, int expert, int tensor, zm_tensor_info *info_out, const void **device_blob_out)
{
    if (!layer || !info_out || expert < 0 || expert >= layer->n_experts || tensor < 0 || tensor >= layer->tensors_per_expert)
        return ZM_E_ARG;
    const size_t i = static_cast<size_t>(expert) * layer->tensors_per_expert + tensor;
    *info_out = layer->infos[i];
    if (device_blob_out) *device_blob_out = layer->blobs[i];
    return ZM_OK;
}

int zm_layer_decode(const zm_layer *layer, const int32_t *expert_ids, int n_selected, void *const *out_bf16, int stores,
                    void *stream)
{
    if (!layer) return ZM_E_ARG;
    return zm_decode_experts_stores(layer->blobs.data(), layer->tables.data(), layer->infos.data(), layer->n_experts,
                                    layer->tensors_per_expert, expert_ids, n_selected, out_bf16, stores, stream);
}

int zm_layer_moe_workspace_bytes(const zm_layer *layer, int n_selected, int64_t n_tokens, int top_k, int hidden, size_t *bytes)
{
    if (!layer || !bytes || n_selected < 0 || n_selected > ZM_MOE_MAX_EXPERTS || hidden < 1 || layer->tensors_per_expert != 3) return ZM_E_ARG;
    const uint64_t values = layer->infos[0].n_values, h = static_cast<uint64_t>(hidden);
    if (values % h || values >= (1ull << 31)) return ZM_E_ARG;
    const int rc = zm_moe_workspace_bytes(n_tokens, top_k, hidden, static_cast<int>(values / h), n_selected, bytes);
    if (rc == ZM_OK) *bytes += 3 * static_cast<size_t>(n_selected) * aligned(2 * values);
    return rc;
}

int zm_layer_moe(const zm_layer *layer, const int32_t *expert_ids, int n_selected, const zm_moe_args *args, void *workspace, size_t workspace_bytes,
                 void *stream)
{
    if (!layer || !args || n_selected < 0 || (n_selected && !expert_ids)) return ZM_E_ARG;
    size_t need = 0;
    const int rc = zm_layer_moe_workspace_bytes(layer, n_selected, args->n_tokens, args->top_k, args->hidden, &need);
    if (rc != ZM_OK) return rc;
    const uint64_t values = layer->infos[0].n_values;
    if (static_cast<uint64_t>(args->hidden) * static_cast<uint64_t>(args->intermediate > 0 ? args->intermediate : 0) != values ||
        (reinterpret_cast<uintptr_t>(workspace) & (kAlign - 1))) return ZM_E_ARG;
    for (int i = 0; i < n_selected; ++i) {
        if (expert_ids[i] < 0 || expert_ids[i] >= layer->n_experts) return ZM_E_ARG;
        for (int m = 0; m < 3; ++m)
            if (layer->infos[3 * expert_ids[i] + m].n_values != values) return ZM_E_ARG;
        for (int j = 0; j < i; ++j)
            if (expert_ids[j] == expert_ids[i]) return ZM_E_ARG;
    }
    if (args->n_tokens == 0) return zm_moe(nullptr, nullptr, 0, args, workspace, workspace_bytes, stream);
    if (!workspace) return ZM_E_ARG;
    if (workspace_bytes < need) return ZM_E_SIZE;
    // the matrices, or the sums of products with them, go to the end of the workspace
    const size_t each = aligned(2 * values), room = 3 * static_cast<size_t>(n_selected) * each;
    uint8_t *at = static_cast<uint8_t *>(workspace) + (need - room);
    if (!moe_check(*args, workspace)) return ZM_E_ARG;
    size_t sums = 0;
    if (takes_products(*layer, expert_ids, n_selected, *args, sums) && sums <= room)
        return layer_products(*layer, expert_ids, n_selected, *args, workspace, reinterpret_cast<float *>(at), static_cast<hipStream_t>(stream));
    // one call decodes at most 256 of them
    void *tensors[3 * ZM_MOE_MAX_EXPERTS];
    for (int i = 0; i < 3 * n_selected; ++i) tensors[i] = at + static_cast<size_t>(i) * each;
    constexpr int kPerCall = 256 / 3;
    for (int i = 0; i < n_selected; i += kPerCall) {
        const int n = n_selected - i < kPerCall ? n_selected - i : kPerCall;
        const int status = zm_layer_decode(layer, expert_ids + i, n, tensors + 3 * i, ZM_STORES_CACHED, stream);
        if (status != ZM_OK) return status;
    }
    return zm_moe(tensors, expert_ids, n_selected, args, workspace, workspace_bytes, stream);
}

void zm_layer_destroy(zm_layer *layer) { delete layer; }

}  // extern "C"
