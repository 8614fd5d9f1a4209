// zm_route: the gate of a sparse layer -- router product, softmax, and the top_k experts of every token.
//
// Two experts' logits can lie closer to each other than sums in 32 bits are exact, and which of them is ahead decides which expert's
// tensors are read.  Products of two 16-bit floating-point values are exact in 32 bits, of two 32-bit ones in 64; they are summed in
// 64 bits, where another order moves a sum by 1e-16 of its terms.  So the product is bound by 64-bit arithmetic (78 TFLOP/s, vector
// and matrix instructions alike), where the bytes alone would take a tenth of the time.
//
//   few tokens    logits: a wave takes two experts and up to four tokens and leaves their logits in the workspace; choose: a wave per token
//   many tokens   a workgroup takes a tile of 16 tokens and all experts: 64-bit matrix instructions, then a wave per token chooses
//
// 4096 tokens of 2048 values and 64 experts take 28 us, 14 of them at the rate of the matrix instructions; one token of 60 experts 7.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "zipmoe.h"
#include "zipmoe_rows.h"

namespace {

using namespace zipmoe;

static_assert(sizeof(zm_route_args) == 104);

struct Route {
    const void *x, *weight;
    const float *bias;
    const uint8_t *token_mask;
    int32_t *ids;
    float *weights, *logits;
    double *sums;              // workspace [n_tokens, n_experts]
    int64_t x_stride, weight_stride;
    uint32_t n_tokens, hidden, n_experts, top_k, renormalise;
    float scale;
};

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// The largest of the lanes' values, for all lanes: shifts inside rows of 16 lanes, then across them.
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x111, 0xf, 0xf, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x112, 0xf, 0xf, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x114, 0xf, 0xf, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x118, 0xf, 0xf, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x142, 0xa, 0xf, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x143, 0xc, 0xf, false)));
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63));
}

// One wave finishes a token: l[0 .. n_experts) are its logits, NaN replaced by -infinity.  A logit's bits, turned so that they order as
// unsigned numbers, are its key, 0 where there is nothing to choose; place after place the wave finds the largest key that is left, by its
// upper half, and where several lanes share that, by its lower half, and then by the expert's number.  kPer: experts per lane.
// (Counting for every expert those ahead of it took 45 us for 256 experts, and 4 of 34 us for 4096 tokens of 64.)
template <int kPer>
__device__ __forceinline__ void choose(const Route &p, uint32_t token, const double *l, uint32_t lane)
{
    int32_t *ids = p.ids + static_cast<uint64_t>(token) * p.top_k;
    float *weights = p.weights + static_cast<uint64_t>(token) * p.top_k;
    if (p.token_mask && p.token_mask[token] == 0) {
        for (uint32_t k = lane; k < p.top_k; k += 64) ids[k] = -1, weights[k] = 0.0f;
        return;
    }
    double value[kPer], most = -INFINITY;
    uint64_t key[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const uint32_t e = lane + 64 * i;
        value[i] = e < p.n_experts ? l[e] + 0.0 : -INFINITY;                  // -0 is 0
        most = fmax(most, value[i]);
        const uint64_t b = __builtin_bit_cast(uint64_t, value[i]);
        key[i] = value[i] > -INFINITY ? b ^ ((b >> 63) ? ~0ull : 1ull << 63) : 0;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) most = fmax(most, __shfl_xor(most, d));
    // exp of a difference in 32 bits; where the largest logit is infinite its holders share everything
    auto share_of = [&](double v) { return v == -INFINITY ? 0.0f : v == most ? 1.0f : expf(static_cast<float>(v - most)); };
    float total = 0.0f;
    if (!p.renormalise) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) total += share_of(value[i]);
#pragma unroll
        for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
    }
    for (uint32_t base = 0; base < p.top_k; base += 64) {                     // lane j keeps place base + j
        const uint32_t places = min(p.top_k - base, 64u);
        int32_t id = -1;
        uint64_t chosen = 0;
        for (uint32_t k = 0; k < places; ++k) {
            uint64_t best = key[0];
            uint32_t at = 0;
#pragma unroll
            for (int i = 1; i < kPer; ++i) {
                at = key[i] > best ? i : at;
                best = key[i] > best ? key[i] : best;
            }
            const uint32_t high = static_cast<uint32_t>(best >> 32), low = static_cast<uint32_t>(best);
            const uint32_t top = wave_max(high);
            if (top == 0) break;                                              // nothing left
            uint64_t who = __builtin_amdgcn_ballot_w64(high == top);
            if (who & (who - 1)) {
                const uint32_t next = wave_max(high == top ? low : 0);
                who = __builtin_amdgcn_ballot_w64(high == top && low == next);
                if (kPer > 1 && (who & (who - 1))) {
                    const uint32_t earliest = ~wave_max(who >> lane & 1 ? ~at : 0);
                    who = __builtin_amdgcn_ballot_w64((who >> lane & 1) && at == earliest);
                }
            }
            const uint32_t winner = static_cast<uint32_t>(__builtin_ctzll(who));
            const uint32_t slot = kPer > 1 ? static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(at), static_cast<int>(winner))) : 0;
            const uint32_t low_w = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(low), static_cast<int>(winner)));
            if (lane == k) id = static_cast<int32_t>(winner + 64 * slot), chosen = static_cast<uint64_t>(top) << 32 | low_w;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (lane == winner && static_cast<uint32_t>(i) == slot) key[i] = 0;
        }
        const double v = __builtin_bit_cast(double, chosen ^ ((chosen >> 63) ? 1ull << 63 : ~0ull));
        float share = id < 0 ? 0.0f : share_of(v);
        if (p.renormalise) {
            float part = share;
#pragma unroll
            for (int d = 32; d; d >>= 1) part += __shfl_xor(part, d);
            total += part;
        }
        const bool known = !p.renormalise || p.top_k <= 64;
        if (lane < places) {
            ids[base + lane] = id;
            weights[base + lane] = id < 0 ? 0.0f : known ? share / total * p.scale : share;
        }
    }
    if (p.renormalise && p.top_k > 64)
        for (uint32_t k = lane; k < p.top_k; k += 64)
            if (weights[k] != 0.0f) weights[k] = weights[k] / total * p.scale;
}

__device__ __forceinline__ void choose(const Route &p, uint32_t token, const double *l, uint32_t lane)
{
    if (p.n_experts <= 64) choose<1>(p, token, l, lane);
    else if (p.n_experts <= 256) choose<4>(p, token, l, lane);
    else choose<16>(p, token, l, lane);
}

// What is left to do with a sum: the bias, the caller's copy, and no NaN.
__device__ __forceinline__ double finished(const Route &p, uint32_t token, uint32_t e, double sum)
{
    if (p.bias) sum += static_cast<double>(p.bias[e]);
    if (p.logits) p.logits[static_cast<uint64_t>(token) * p.n_experts + e] = static_cast<float>(sum);
    return sum == sum ? sum : -INFINITY;
}

// ---- few tokens ----

constexpr uint32_t kWaveExperts = 2;

// A wave: two experts and kTokens tokens (blockIdx.y-th group), lane j values 8 j .. + 7 of every 512.
template <class T, bool kTight, int kTokens>
__global__ void __launch_bounds__(256) zm_route_logits_kernel(const Route p)
{
    const uint32_t lane = threadIdx.x % 64, e0 = (blockIdx.x * 4 + threadIdx.x / 64) * kWaveExperts, t0 = blockIdx.y * kTokens;
    if (e0 >= p.n_experts) return;
    const T *x[kTokens], *w[kWaveExperts];
#pragma unroll
    for (uint32_t t = 0; t < kTokens; ++t) x[t] = static_cast<const T *>(p.x) + min(t0 + t, p.n_tokens - 1) * p.x_stride;
#pragma unroll
    for (uint32_t e = 0; e < kWaveExperts; ++e) w[e] = static_cast<const T *>(p.weight) + min(e0 + e, p.n_experts - 1) * p.weight_stride;
    double sum[kTokens][kWaveExperts] = {};
#pragma unroll 2
    for (uint32_t at = 8u * lane; at < p.hidden; at += 512) {
        float a[kTokens][8], b[kWaveExperts][8];
#pragma unroll
        for (int t = 0; t < kTokens; ++t) load8<T, kTight>(x[t] + at, p.hidden - at, a[t]);
#pragma unroll
        for (uint32_t e = 0; e < kWaveExperts; ++e) load8<T, kTight>(w[e] + at, p.hidden - at, b[e]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int t = 0; t < kTokens; ++t)
#pragma unroll
                for (uint32_t e = 0; e < kWaveExperts; ++e) sum[t][e] = fma(static_cast<double>(a[t][i]), static_cast<double>(b[e][i]), sum[t][e]);
    }
#pragma unroll
    for (uint32_t t = 0; t < kTokens; ++t)
#pragma unroll
        for (uint32_t e = 0; e < kWaveExperts; ++e) {
            const double l = wave_sum(sum[t][e]);
            if (lane == 0 && t0 + t < p.n_tokens && e0 + e < p.n_experts)
                p.sums[static_cast<uint64_t>(t0 + t) * p.n_experts + e0 + e] = finished(p, t0 + t, e0 + e, l);
        }
}

__global__ void __launch_bounds__(64) zm_route_choose_kernel(const Route p)
{
    __shared__ double l[ZM_ROUTE_MAX_EXPERTS];
    const double *sums = p.sums + static_cast<uint64_t>(blockIdx.x) * p.n_experts;
    for (uint32_t e = threadIdx.x; e < p.n_experts; e += 64) l[e] = sums[e];
    __syncthreads();
    choose(p, blockIdx.x, l, threadIdx.x);
}

// ---- many tokens ----

typedef double f64x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kTileExperts = 256;      // the most that a workgroup's 16 waves hold, 16 each

// v_mfma_f64_16x16x4: lane l holds row l % 16 (a token) and column l % 16 (an expert) of four values' number l / 16, and receives rows
// l / 16 + 4 r of column l % 16.  Which four values meet in one instruction is free: lane group g takes values 32 n + 8 g .. + 7 with one load, and
// the n-th eight instructions one of each.  A wave takes kEach times 16 experts, so that a token's values are converted to 64 bits
// once for them; what is left of 16 waves splits the rows' length.
template <class T, bool kTight, int kEach>
__global__ void __launch_bounds__(1024) zm_route_tile_kernel(const Route p)
{
    __shared__ double part[16][kEach][16][17];                             // of every wave: [expert][token]
    __shared__ double l[16 * kTileExperts];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), t0 = blockIdx.x * 16;
    const uint32_t tiles = (p.n_experts + 16 * kEach - 1) / (16 * kEach), splits = 16 / tiles, tile = wave % tiles, split = wave / tiles;
    if (split < splits) {
        const T *x = static_cast<const T *>(p.x) + min(t0 + lane % 16, p.n_tokens - 1) * p.x_stride;
        const T *w[kEach];
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) w[j] = static_cast<const T *>(p.weight) + min((tile * kEach + j) * 16 + lane % 16, p.n_experts - 1) * p.weight_stride;
        f64x4 sum[kEach][2] = {};
        struct Values { float x[8], w[kEach][8]; };
        auto load = [&](uint32_t k) {
            Values v;
            const uint32_t at = k + 8 * (lane / 16);
            if (kTight ? at < p.hidden : at + 8 <= p.hidden) {
                load8<T, kTight>(x + at, 8, v.x);
#pragma unroll
                for (int j = 0; j < kEach; ++j) load8<T, kTight>(w[j] + at, 8, v.w[j]);
            } else {
                const uint32_t n = at < p.hidden ? p.hidden - at : 0;
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) {
                    v.x[i] = i < n ? static_cast<float>(x[at + i]) : 0.0f;
#pragma unroll
                    for (int j = 0; j < kEach; ++j) v.w[j][i] = i < n ? static_cast<float>(w[j][at + i]) : 0.0f;
                }
            }
            return v;
        };
        auto multiply = [&](const Values &v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double x = static_cast<double>(v.x[i]);
#pragma unroll
                for (int j = 0; j < kEach; ++j) sum[j][i & 1] = __builtin_amdgcn_mfma_f64_16x16x4f64(x, static_cast<double>(v.w[j][i]), sum[j][i & 1], 0, 0, 0);
            }
        };
        const uint32_t step = 32 * splits;
        uint32_t k = 32 * split;
        if (k < p.hidden) {
            Values v = load(k);
            for (; k + step < p.hidden; k += step) {
                const Values next = load(k + step);
                multiply(v);
                v = next;
            }
            multiply(v);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) part[wave][j][lane % 16][lane / 16 + 4 * r] = sum[j][0][r] + sum[j][1][r];
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 16 * p.n_experts; i += 1024) {
        const uint32_t token = i / p.n_experts, e = i % p.n_experts;
        double sum = 0.0;
        for (uint32_t s = 0; s < splits; ++s) sum += part[e / (16 * kEach) + s * tiles][e / 16 % kEach][e % 16][token];
        l[token * kTileExperts + e] = t0 + token < p.n_tokens ? finished(p, t0 + token, e, sum) : 0.0;
    }
    __syncthreads();
    if (t0 + wave < p.n_tokens) choose(p, t0 + wave, l + wave * kTileExperts, lane);
}

template <class T, bool kTight>
int launch_route(const Route &p, bool few, hipStream_t stream)
{
    Route q = p;
    void *args[] = {&q};
    const uint32_t across = (p.n_experts + 4 * kWaveExperts - 1) / (4 * kWaveExperts);
    // a grid has less than 2^32 threads along an axis, 1024 for a tile's 16 tokens; its y axis has 16 bits
    const uint32_t most = few ? 65535u : 1u << 25;
    for (uint32_t done = 0; done < p.n_tokens;) {
        q = p;
        const uint32_t n = p.n_tokens - done < most ? p.n_tokens - done : most;
        const uint32_t size = static_cast<uint32_t>(sizeof(T));
        q.x = static_cast<const uint8_t *>(p.x) + done * p.x_stride * size;
        q.n_tokens = n;
        q.ids += static_cast<uint64_t>(done) * p.top_k, q.weights += static_cast<uint64_t>(done) * p.top_k;
        if (q.logits) q.logits += static_cast<uint64_t>(done) * p.n_experts;
        if (q.token_mask) q.token_mask += done;
        q.sums += static_cast<uint64_t>(done) * p.n_experts;
        done += n;
        if (!few) {
            const void *fn = p.n_experts > 16 ? reinterpret_cast<const void *>(&zm_route_tile_kernel<T, kTight, 2>) : reinterpret_cast<const void *>(&zm_route_tile_kernel<T, kTight, 1>);
            if (hipLaunchKernel(fn, dim3((n + 15) / 16), dim3(1024), args, 0, stream) != hipSuccess) return ZM_E_HIP;
            continue;
        }
        const bool one = n < 4;
        const void *fn = one ? reinterpret_cast<const void *>(&zm_route_logits_kernel<T, kTight, 1>) : reinterpret_cast<const void *>(&zm_route_logits_kernel<T, kTight, 4>);
        if (hipLaunchKernel(fn, dim3(across, one ? n : (n + 3) / 4), dim3(256), args, 0, stream) != hipSuccess) return ZM_E_HIP;
        if (hipLaunchKernel(reinterpret_cast<const void *>(&zm_route_choose_kernel), dim3(n), dim3(64), args, 0, stream) != hipSuccess) return ZM_E_HIP;
    }
    return ZM_OK;
}

// Whether a call goes without tiles.  A tile's product takes hidden * 16 ceil(n_experts / 16) * 0.17 ns, on as many compute units at once as there are 16
// tokens; without tiles all of them take part in hidden * n_experts * n_tokens * 0.102 ps, and a second launch takes 3 us.  us without / with tiles:
// 64 experts of 2048, 512 tokens 14.1 / 26.0, 2048 35.2 / 26.3; 256 experts, 1024 tokens 60 / 89, 2048 112 / 90; 8 experts of 4096, 1024 tokens
// 11.2 / 16.3, 4096 21.9 / 18.4; 16 experts of 512, 9 tokens 7.2 / 5.2.
bool takes_few(int64_t n_tokens, int64_t hidden, int64_t n_experts)
{
    const int64_t full = (n_experts + 15) / 16 * 16, rounds = (n_tokens + 4095) / 4096;
    return n_experts > static_cast<int64_t>(kTileExperts) || static_cast<double>(n_tokens) * n_experts * hidden + 29.4e6 < 1667.0 * hidden * full * rounds;
}

}  // namespace

extern "C" {

int zm_route_workspace_bytes(int64_t n_tokens, int hidden, int n_experts, size_t *bytes)
{
    if (!bytes || n_tokens < 0 || n_tokens >= (1ll << 31) || hidden < 1 || n_experts < 1 || n_experts > ZM_ROUTE_MAX_EXPERTS) return ZM_E_ARG;
    *bytes = 256 + sizeof(double) * static_cast<size_t>(n_tokens) * static_cast<size_t>(n_experts);      // logits of a call without tiles
    return ZM_OK;
}

int zm_route(const zm_route_args *a, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!a) return ZM_E_ARG;
    if (a->type != ZM_BF16 && a->type != ZM_FP16 && a->type != ZM_FP32) return ZM_E_ARG;
    if (a->hidden > (1 << 24) || a->top_k < 1 || a->top_k > a->n_experts || a->x_stride < 0 || a->weight_stride < 0) return ZM_E_ARG;
    size_t need = 0;
    const int rc = zm_route_workspace_bytes(a->n_tokens, a->hidden, a->n_experts, &need);
    if (rc != ZM_OK) return rc;
    if (a->n_tokens == 0) return ZM_OK;
    if (!a->x || !a->weight || !a->ids || !a->weights || !workspace) return ZM_E_ARG;
    const size_t size = type_bytes(a->type);
    if (!aligned_to(workspace, 16) || !aligned_to(a->x, size) || !aligned_to(a->weight, size) || !aligned_to(a->bias, 4) ||
        !aligned_to(a->ids, 4) || !aligned_to(a->weights, 4) || !aligned_to(a->logits, 4)) return ZM_E_ARG;
    if (workspace_bytes < need) return ZM_E_SIZE;
    const bool tight = a->hidden % 8 == 0 && aligned_to(a->x, 16) && aligned_to(a->weight, 16) &&
                       (a->n_tokens == 1 || a->x_stride * size % 16 == 0) && (a->n_experts == 1 || a->weight_stride * size % 16 == 0);
    Route p{a->x, a->weight, a->bias, a->token_mask, a->ids, a->weights, a->logits, static_cast<double *>(workspace), a->x_stride, a->weight_stride,
            static_cast<uint32_t>(a->n_tokens), static_cast<uint32_t>(a->hidden), static_cast<uint32_t>(a->n_experts),
            static_cast<uint32_t>(a->top_k), a->renormalise != 0, a->scale};
    const bool few = takes_few(a->n_tokens, a->hidden, a->n_experts);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a->type == ZM_BF16) return tight ? launch_route<__bf16, true>(p, few, st) : launch_route<__bf16, false>(p, few, st);
    if (a->type == ZM_FP16) return tight ? launch_route<_Float16, true>(p, few, st) : launch_route<_Float16, false>(p, few, st);
    return tight ? launch_route<float, true>(p, few, st) : launch_route<float, false>(p, few, st);
}

}  // extern "C"
