// zm_rms_norm: root-mean-square norm behind a residual addition, in the activations' type and in 8 bits.
//
//   s = x + residual,   y = s / sqrt(mean(s^2) + eps) * weight,   e4m3(y / 2^b) with one b per 32 values
//
// One pass over the data: a row's s stays in registers between the sum of its squares and the scaling.  It is bound by
// bytes (8192 rows of 4096 bf16 values with a residual and all three results: 303 MB in 64.6 us, 55.8 of them in the
// kernel, 5.4 TB/s, where a plain mover of so many bytes reaches 6.15 with ordinary stores); the
// lanes of a row take runs of eight neighbouring values, so the 32 values that share a scale lie in four neighbouring lanes.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "zipmoe.h"
#include "zipmoe_rows.h"

namespace {

using namespace zipmoe;

static_assert(sizeof(zm_norm_args) == 128);

struct Norm {
    const void *x, *residual, *weight;
    void *sum_out, *out;
    uint8_t *out8, *scales;
    int64_t x_stride, residual_stride, sum_stride, out_stride, out8_stride, scales_stride;
    uint32_t n_rows, hidden;
    float eps, share;          // 1 / hidden
};

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Eight values of y and the four lanes' common scale: the least power of two p = 2^(byte - 127) with max |y| <= 448 p.  With
// max = m 2^e, m in [1/2, 1): 448 = 7/8 2^9, so p is 2^(e-9) where m is at most 7/8 and twice that else.
__device__ __forceinline__ uint2 eight_bits(const float (&y)[8], uint32_t &byte)
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(y[i]));              // passes over NaN
    most = fmaxf(most, __shfl_xor(most, 1));
    most = fmaxf(most, __shfl_xor(most, 2));
    int e;
    const float m = frexpf(most, &e);
    int b = e + (m <= 0.875f ? 127 - 9 : 127 - 8);
    b = b < 0 || most == 0.0f ? 0 : b;
    b = b > 254 || most == INFINITY ? 254 : b;
    byte = static_cast<uint32_t>(b);
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        q[i] = ldexpf(y[i], 127 - b);
        q[i] = fabsf(q[i]) <= 448.0f ? q[i] : NAN;                            // infinities and NaN
    }
    uint2 w;
    w.x = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    w.x = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w.x, true);
    w.y = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
    w.y = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], w.y, true);
    return w;
}

// kLanes lanes take a row, 256 of a workgroup at least; lane j holds values 8 (j + kLanes c) .. + 7 for c < kChunks.  kChunks = 0: rows of any
// length, read twice.
template <class T, int kLanes, int kChunks, bool kTight>
__global__ void __launch_bounds__(kLanes < 256 ? 256 : kLanes) zm_norm_kernel(const Norm p)
{
    constexpr int kRows = kLanes < 256 ? 256 / kLanes : 1, kWaves = kLanes / 64;
    const uint32_t lane = kLanes < 256 ? threadIdx.x % kLanes : threadIdx.x;
    const uint64_t row = static_cast<uint64_t>(blockIdx.x) * kRows + (kLanes < 256 ? threadIdx.x / kLanes : 0);
    if (kRows > 1 && row >= p.n_rows) return;                                 // whole waves, no barrier below
    const T *x = static_cast<const T *>(p.x) + row * p.x_stride;
    const T *residual = p.residual ? static_cast<const T *>(p.residual) + row * p.residual_stride : nullptr;
    const T *weight = static_cast<const T *>(p.weight);

    auto take = [&](uint32_t at, float (&s)[8]) {
        const uint32_t n = p.hidden - at;
        load8<T, kTight>(x + at, n, s);
        if (residual) {
            float r[8];
            load8<T, kTight>(residual + at, n, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += r[i];
        }
    };
    constexpr int kHeld = kChunks ? kChunks : 1;
    float s[kHeld][8], w[kHeld][8];
    float squares = 0.0f;
    if constexpr (kChunks != 0) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const uint32_t at = 8u * (lane + kLanes * c);
            if (at < p.hidden) {
                take(at, s[c]);
                load8<T, kTight>(weight + at, p.hidden - at, w[c]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) s[c][i] = w[c][i] = 0.0f;
            }
        }
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) squares += s[c][i] * s[c][i];
    } else {
        for (uint32_t at = 8u * lane; at < p.hidden; at += 8u * kLanes) {
            take(at, s[0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) squares += s[0][i] * s[0][i];
        }
    }
    squares = wave_sum(squares);
    if constexpr (kWaves > 1) {
        __shared__ float part[kWaves];
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = squares;
        __syncthreads();
        squares = 0.0f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) squares += part[i];
    }
    const float scale = 1.0f / sqrtf(squares * p.share + p.eps);

    auto give = [&](uint32_t at, const float (&s)[8], const float (&w)[8]) {
        // lanes behind the end of the row come along: four lanes share a scale
        const uint32_t n = at < p.hidden ? p.hidden - at : 0;
        if (n && p.sum_out) store8<T, kTight>(static_cast<T *>(p.sum_out) + row * p.sum_stride + at, n, s);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = s[i] * scale * w[i];
        if (n && p.out) store8<T, kTight>(static_cast<T *>(p.out) + row * p.out_stride + at, n, y);
        if (p.out8) {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                if (!kTight && i >= n) y[i] = 0.0f;                           // 0 * infinity behind the end is none of the group's
            uint32_t byte;
            const uint2 q = eight_bits(y, byte);
            uint8_t *to = p.out8 + row * p.out8_stride + at;
            if (n >= 8) {
                __builtin_memcpy(to, &q, 8);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    if (i < n) to[i] = static_cast<uint8_t>((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
            }
            if (n && (lane & 3) == 0) p.scales[row * p.scales_stride + at / 32] = static_cast<uint8_t>(byte);
        }
    };
    if constexpr (kChunks != 0) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) give(8u * (lane + kLanes * c), s[c], w[c]);
    } else {
        for (uint32_t first = 0; first < p.hidden; first += 8u * kLanes) {
            const uint32_t at = first + 8u * lane;
            if (at < p.hidden) {
                take(at, s[0]);
                load8<T, kTight>(weight + at, p.hidden - at, w[0]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) s[0][i] = w[0][i] = 0.0f;
            }
            give(at, s[0], w[0]);
        }
    }
}

template <class T, bool kTight>
const void *kernel_for(uint32_t hidden, uint32_t &lanes)
{
    const uint32_t runs = (hidden + 7) / 8;
#define ZM_NORM(LANES, CHUNKS) (lanes = LANES, reinterpret_cast<const void *>(&zm_norm_kernel<T, LANES, CHUNKS, kTight>))
    if (runs <= 64) return ZM_NORM(64, 1);
    if (runs <= 128) return ZM_NORM(64, 2);
    if (runs <= 256) return ZM_NORM(256, 1);
    if (runs <= 512) return ZM_NORM(256, 2);
    if (runs <= 1024) return ZM_NORM(256, 4);
    if (runs <= 2048) return ZM_NORM(1024, 2);
    return ZM_NORM(1024, 0);
#undef ZM_NORM
}

}  // namespace

extern "C" int zm_rms_norm(const zm_norm_args *a, void *stream)
{
    if (!a || (a->type != ZM_BF16 && a->type != ZM_FP16 && a->type != ZM_FP32)) return ZM_E_ARG;
    if (a->n_rows < 0 || a->n_rows >= (1ll << 31) || a->hidden < 1 || a->hidden > (1 << 24) || a->reserved) return ZM_E_ARG;
    if (a->n_rows == 0) return ZM_OK;                                         // whose rows may have no address
    if (!a->x || !a->weight || !(a->sum_out || a->out || a->out8) || !a->out8 != !a->scales) return ZM_E_ARG;
    const int64_t h = a->hidden;
    if (a->x_stride < 0 || (a->residual && a->residual_stride < 0) || (a->n_rows > 1 && ((a->sum_out && a->sum_stride < h) ||
        (a->out && a->out_stride < h) || (a->out8 && (a->out8_stride < h || a->scales_stride < (h + 31) / 32))))) return ZM_E_ARG;
    const size_t size = type_bytes(a->type);
    bool tight = h % 8 == 0;
    const void *const rows[] = {a->x, a->residual, a->weight, a->sum_out, a->out};
    const int64_t strides[] = {a->x_stride, a->residual_stride, 0, a->sum_stride, a->out_stride};
    for (int i = 0; i < 5; ++i) {
        if (!rows[i]) continue;
        if (!aligned_to(rows[i], size)) return ZM_E_ARG;
        if (!aligned_to(rows[i], 16) || (a->n_rows > 1 && strides[i] * static_cast<int64_t>(size) % 16 != 0)) tight = false;
    }
    Norm p{a->x, a->residual, a->weight, a->sum_out, a->out, static_cast<uint8_t *>(a->out8), static_cast<uint8_t *>(a->scales),
           a->x_stride, a->residual_stride, a->sum_stride, a->out_stride, a->out8_stride, a->scales_stride,
           static_cast<uint32_t>(a->n_rows), static_cast<uint32_t>(h), a->eps, 1.0f / static_cast<float>(h)};
    uint32_t lanes = 0;
    const void *fn = nullptr;
    if (a->type == ZM_BF16) fn = tight ? kernel_for<__bf16, true>(p.hidden, lanes) : kernel_for<__bf16, false>(p.hidden, lanes);
    else if (a->type == ZM_FP16) fn = tight ? kernel_for<_Float16, true>(p.hidden, lanes) : kernel_for<_Float16, false>(p.hidden, lanes);
    else fn = tight ? kernel_for<float, true>(p.hidden, lanes) : kernel_for<float, false>(p.hidden, lanes);
    const uint32_t block = lanes < 256 ? 256 : lanes, per_block = block / lanes;
    void *args[] = {&p};
    // a grid has less than 2^32 threads along an axis
    const int64_t most = (1ll << 31) / block * per_block;
    auto rows_from = [](const void *rows, int64_t elements, size_t each) {
        return rows ? const_cast<uint8_t *>(static_cast<const uint8_t *>(rows)) + elements * static_cast<int64_t>(each) : nullptr;
    };
    for (int64_t done = 0; done < a->n_rows; done += most) {
        p.x = rows_from(a->x, done * a->x_stride, size), p.residual = rows_from(a->residual, done * a->residual_stride, size);
        p.sum_out = rows_from(a->sum_out, done * a->sum_stride, size), p.out = rows_from(a->out, done * a->out_stride, size);
        p.out8 = rows_from(a->out8, done * a->out8_stride, 1), p.scales = rows_from(a->scales, done * a->scales_stride, 1);
        p.n_rows = static_cast<uint32_t>(a->n_rows - done < most ? a->n_rows - done : most);
        if (hipLaunchKernel(fn, dim3((p.n_rows + per_block - 1) / per_block), dim3(block), args, 0, static_cast<hipStream_t>(stream)) != hipSuccess) return ZM_E_HIP;
    }
    return ZM_OK;
}
