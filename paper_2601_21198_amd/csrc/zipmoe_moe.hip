// zm_moe: the experts that a router chose.
//
//   out_t = residual_t + sum_j weights_tj * down_e (silu(gate_e x_t) * (up_e x_t)),   e = ids_tj
//
// A pair is a token and one of its experts, numbered t * top_k + j.
//
// Few tokens (up to 32, with up to 512 pairs) are bound by the matrices' bytes (experts of 1408 x 2048, one token through 4: 69 MB in 21.2 us where they stay cached, 24.3 where not; of 1024 x
// 2048, 16 tokens through 8 of 64: 470 MB in 122 us): two launches, each of which finds out for itself which experts
// somebody chose and streams their matrices from memory into matrix instructions, once.
//   few_first    16 rows of gate and up of one expert times the tokens that chose it; the weighted h in two bf16 parts
//   few_second   16 rows of down of every chosen expert times h; an expert's column for a token is its weighted h, so one
//                accumulator sums over experts
// Many tokens are bound by the matrix cores: the pairs are put in the order of their experts, and tiles of pairs multiply 256 rows.  4096 tokens
// through 2 of 8 experts of 4096 x 14336 take 2.4 ms, 1190 TFLOP/s (a plain library product of these sizes 1545 on the same card).
//   list         one workgroup per expert: its pairs, in order, from the number of pairs with smaller ids on
//   product      gate and up, then down, in tiles of 128 pairs; wide: in tiles of 256 or 288.  h is rounded to bf16 once, which the result shows (off by
//                2.3e-3 of its norm, its own rounding alone by 1.7e-3): a second part would be half as many matrix instructions again
//   join         residual + the weighted sum over a token's pairs
//
// The matrix instruction v_mfma_f32_16x16x32_bf16 multiplies 16 rows of 32 values (lane l: row l % 16, values 8 (l / 16) .. + 7) with 16
// columns of 32 (lane l: column l % 16, the same values); lane l receives rows 4 (l / 16) .. + 3 of column l % 16.  Matrices
// are the rows and tokens the columns.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "zipmoe.h"
#include "zipmoe_moe.h"
#include "zipmoe_rows.h"

namespace {

using namespace zipmoe;

static_assert(sizeof(zm_moe_args) == 104);

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct Experts {
    uint32_t n;
    int32_t id[ZM_MOE_MAX_EXPERTS];
    const uint16_t *tensor[ZM_MOE_MAX_EXPERTS][3];
};
struct Call {
    const void *x;
    const uint8_t *scales;
    const int32_t *ids;
    const float *weights;
    const uint16_t *residual;
    uint16_t *out;
    int64_t x_stride, scales_stride, residual_stride, out_stride;
    uint32_t n_tokens, top_k, hidden, intermediate, n_pairs;
    // workspace
    uint32_t *first, *count;      // [n] of every expert: its first place in the list, its pairs
    uint32_t *list;               // [n_pairs] pairs in the order of their experts
    uint16_t *h;                  // [n_pairs, intermediate]: of many tokens in the order of the list, of few in the order of the pairs
    uint16_t *h_rest;             // few tokens: what rounding h to bf16 leaves
    float *y;                     // [n_pairs, hidden] in the order of the pairs
    uint16_t *wide_x;             // [n_tokens, wide_stride] e4m3 rows as bf16
    uint32_t wide_stride;
};
// The runtime copies a kernel's arguments for every launch, so only those kernels that read matrices take the table of them.
struct Ids {
    uint32_t n;
    int32_t id[ZM_MOE_MAX_EXPERTS];
};
static_assert(sizeof(Experts) + sizeof(Call) <= 4096);

// ---- list ----

__global__ void __launch_bounds__(1024) zm_moe_list_kernel(const Call c, const Ids e)
{
    __shared__ uint32_t before[17], below[17];
    const int32_t id = e.id[blockIdx.x];
    const uint32_t each = (c.n_pairs + 1023u) / 1024u, from = min(threadIdx.x * each, c.n_pairs), to = min(from + each, c.n_pairs);
    // the first of a thread's pairs are asked for at once and kept for the second pass: where each waited for the one before, a list of 3108 took 7.7 us
    constexpr uint32_t kHeld = 8;
    int32_t held[kHeld];
#pragma unroll
    for (uint32_t i = 0; i < kHeld; ++i) held[i] = from + i < to ? c.ids[from + i] : 0;
    uint32_t less = 0, mine = 0;
    auto count = [&](int32_t v) { less += v < id, mine += v == id; };
#pragma unroll
    for (uint32_t i = 0; i < kHeld; ++i)
        if (from + i < to) count(held[i]);
#pragma unroll 8
    for (uint32_t p = from + kHeld; p < to; ++p) count(c.ids[p]);
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t up_to = mine, all_less = less;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(up_to, d);
        up_to += lane >= static_cast<uint32_t>(d) ? o : 0u;
        all_less += __shfl_xor(all_less, d);
    }
    if (lane == 63) before[wave + 1] = up_to, below[wave + 1] = all_less;
    __syncthreads();
    uint32_t at = up_to - mine, total = 0, first = 0;
    for (uint32_t w = 0; w < 16; ++w) {
        at += w < wave ? before[w + 1] : 0u;
        total += before[w + 1];
        first += below[w + 1];
    }
    at += first;
#pragma unroll
    for (uint32_t i = 0; i < kHeld; ++i)
        if (from + i < to && held[i] == id) c.list[at++] = from + i;
#pragma unroll 8
    for (uint32_t p = from + kHeld; p < to; ++p)
        if (c.ids[p] == id) c.list[at++] = p;
    if (threadIdx.x == 0) c.first[blockIdx.x] = first, c.count[blockIdx.x] = total;
}

// ---- loads ----

// Values k .. k + 7 of a row of `width` bf16 values, zeros behind its end.
template <bool kTight>
__device__ __forceinline__ bf16x8 eight(const uint16_t *row, uint32_t k, uint32_t width)
{
    union { uint16_t w[8]; bf16x8 v; } u;
    if (k + 8 <= width) {
        if constexpr (kTight) __builtin_memcpy(u.w, __builtin_assume_aligned(row + k, 16), 16);
        else __builtin_memcpy(u.w, row + k, 16);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) u.w[i] = k + i < width ? row[k + i] : 0;
    }
    return u.v;
}

// The same of an e4m3 row with its scales: four significant bits times a power of two is a bf16 value as it is, from 2^-130 (below, bf16's
// steps are 2^-133) up to 2^128 (infinity).  Scale byte 255 is e8m0's NaN.
__device__ __forceinline__ bf16x8 eight_scaled(const uint8_t *row, const uint8_t *scales, uint32_t k, uint32_t width)
{
    union { uint8_t b[8]; uint32_t w[2]; } q;
    q.w[0] = q.w[1] = 0;
    if (k >= width) return bf16x8{};
    if (k + 8 <= width) {
        __builtin_memcpy(q.b, row + k, 8);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (k + i < width) q.b[i] = row[k + i];
    }
    const uint8_t scale = scales[k / 32];
    const int b = static_cast<int>(scale) - 127;
    bf16x8 v;
    if (scale == 255) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<__bf16>(NAN);
        return v;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(q.w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(q.w[i], true);
        v[4 * i] = static_cast<__bf16>(ldexpf(lo[0], b));
        v[4 * i + 1] = static_cast<__bf16>(ldexpf(lo[1], b));
        v[4 * i + 2] = static_cast<__bf16>(ldexpf(hi[0], b));
        v[4 * i + 3] = static_cast<__bf16>(ldexpf(hi[1], b));
    }
    return v;
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float silu(float g) { return g / (1.0f + expf(-g)); }
// Where the result is rounded to bf16: 2^-22 (2 + |g|) from it, in a third of the instructions.
__device__ __forceinline__ float silu_short(float g) { return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g)); }
__device__ __forceinline__ bool finite(float v) { return fabsf(v) < INFINITY; }
__device__ __forceinline__ uint16_t bits(__bf16 v) { return __builtin_bit_cast(uint16_t, v); }
__device__ __forceinline__ float of_bf16(uint16_t w) { return __builtin_bit_cast(float, static_cast<uint32_t>(w) << 16); }

// ---- few tokens ----

// us as few / as many: 32 tokens through 8 of 64 experts of 1024 x 2048 191 / 175, through 2 of 8 of 14336 x 4096 622 / 622, through 4 of 60 of 1408 x 2048
// 199 / 217; 48 tokens 211 / 158, 714 / 625, 236 / 213.
constexpr uint32_t kFewTokens = 32, kFewPairs = 512;
constexpr uint32_t kFirstWaves = 8, kSecondWaves = 16;

__device__ __forceinline__ uint32_t bits_of(uint64_t m) { return static_cast<uint32_t>(__builtin_popcountll(m)); }
__device__ __forceinline__ uint32_t first_of(uint64_t m) { return static_cast<uint32_t>(__builtin_ctzll(m)); }
__device__ __forceinline__ uint32_t read_lane(uint32_t v, uint32_t lane) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), static_cast<int>(lane))); }

// The addresses of one matrix of every expert, two per lane.  All of them are asked for at once, with the ids: an address that is looked up
// when its expert is known is one more read that the matrices wait for.
struct Addresses {
    uint64_t low, high;
    __device__ __forceinline__ Addresses(const Experts &e, uint32_t m, uint32_t lane)
        : low(lane < e.n ? reinterpret_cast<uint64_t>(e.tensor[lane][m]) : 0), high(lane + 64 < e.n ? reinterpret_cast<uint64_t>(e.tensor[lane + 64][m]) : 0) {}
    __device__ __forceinline__ const uint16_t *of(uint32_t slot) const
    {
        const uint64_t v = slot < 64 ? low : high;
        return reinterpret_cast<const uint16_t *>(static_cast<uint64_t>(read_lane(static_cast<uint32_t>(v >> 32), slot % 64)) << 32 | read_lane(static_cast<uint32_t>(v), slot % 64));
    }
};

// What a workgroup knows of the routing: which experts somebody chose, and which pair joins an expert and a token.  (Of a token that names an
// expert twice it is the first pair, which stands for both.)
//
// Up to 64 pairs: every wave for itself, a pair per lane, without LDS or barriers.
struct FewPairs {
    struct Shared {};
    uint64_t chosen[2];        // experts, one bit each
    uint32_t slot;             // of this lane's pair, or none
    uint32_t top_k, token;

    __device__ __forceinline__ FewPairs(Shared &, const Call &c, const Experts &e)
    {
        const uint32_t lane = threadIdx.x % 64;
        const int32_t id = lane < c.n_pairs ? c.ids[lane] : 0, low = lane < e.n ? e.id[lane] : 0, high = lane + 64 < e.n ? e.id[lane + 64] : 0;
        chosen[0] = chosen[1] = 0, slot = ~0u, top_k = c.top_k, token = lane / c.top_k;
        for (uint32_t p = 0; p < c.n_pairs; ++p) {
            const int32_t v = __builtin_amdgcn_readlane(id, static_cast<int>(p));
            const uint64_t m = __builtin_amdgcn_ballot_w64(lane < e.n && low == v), n = __builtin_amdgcn_ballot_w64(lane + 64 < e.n && high == v);
            chosen[0] |= m, chosen[1] |= n;
            if (lane == p && (m | n)) slot = m ? first_of(m) : 64 + first_of(n);
        }
    }
    __device__ __forceinline__ uint32_t count() const { return bits_of(chosen[0]) + bits_of(chosen[1]); }
    // the i-th chosen expert
    __device__ __forceinline__ uint32_t expert(const Shared &, uint32_t i) const
    {
        uint64_t m = chosen[0];
        uint32_t n = bits_of(m), base = 0;
        if (i >= n) m = chosen[1], i -= n, base = 64;
        for (; i; --i) m &= m - 1;
        return base + first_of(m);
    }
    __device__ __forceinline__ uint64_t pairs_of(uint32_t expert) const { return __builtin_amdgcn_ballot_w64(slot == expert); }
    // the expert's pairs: lane j gets the j-th plus one, those behind the last 0
    __device__ __forceinline__ uint32_t list(const Shared &, uint32_t expert, uint32_t &n) const
    {
        const uint32_t lane = threadIdx.x % 64;
        const uint64_t all = pairs_of(expert), below = (1ull << lane) - 1, start = (1ull << token * top_k) - 1;
        const bool mine = slot == expert && (all & below & ~start) == 0;
        const uint64_t firsts = __builtin_amdgcn_ballot_w64(mine);
        n = bits_of(firsts);
        // lanes without a pair send nothing to a place that is read: place 63 has a pair only if every lane has
        const uint32_t got = static_cast<uint32_t>(__builtin_amdgcn_ds_permute(static_cast<int>(4 * (mine ? bits_of(firsts & below) : 63u)), static_cast<int>(mine ? lane + 1 : 0)));
        return lane < n ? got : 0;
    }
    // the pair that joins the expert and a token, plus one, or 0
    __device__ __forceinline__ uint32_t pair(const Shared &, const Call &c, uint32_t expert, uint32_t t) const
    {
        const uint64_t all = pairs_of(expert), own = top_k < 64 ? (1ull << top_k) - 1 : ~0ull;
        const uint64_t m = t < c.n_tokens ? all >> t * top_k & own : 0;
        return m ? t * top_k + first_of(m) + 1 : 0;
    }
};

// More pairs: a thread per pair, tables in LDS.
struct MorePairs {
    struct Shared {
        int32_t id[kFewPairs];
        uint16_t pair[ZM_MOE_MAX_EXPERTS * kFewTokens];
        uint8_t any[ZM_MOE_MAX_EXPERTS];
        uint8_t slot[ZM_MOE_MAX_EXPERTS];
    };
    uint32_t n, n_tokens;

    __device__ __forceinline__ MorePairs(Shared &s, const Call &c, const Experts &e) : n_tokens(c.n_tokens)
    {
        const uint32_t thread = threadIdx.x, lane = thread % 64;
        const int32_t id = thread < c.n_pairs ? c.ids[thread] : -1;
        for (uint32_t i = thread; i < (e.n * n_tokens + 1) / 2; i += blockDim.x) reinterpret_cast<uint32_t *>(s.pair)[i] = 0;
        if (thread < ZM_MOE_MAX_EXPERTS) s.any[thread] = 0;
        if (thread < c.n_pairs) s.id[thread] = id;
        __syncthreads();
        if (thread < c.n_pairs) {
            // experts named in the order of their ids are found at once
            uint32_t slot = static_cast<uint32_t>(id);
            bool named = slot < e.n && e.id[slot] == id;
            if (__builtin_amdgcn_ballot_w64(!named) != 0)
                for (uint32_t k = 0; k < e.n; ++k)
                    if (e.id[k] == id) named = true, slot = k;
            const uint32_t token = thread / c.top_k;
            for (uint32_t p = token * c.top_k; p < thread; ++p)
                if (s.id[p] == id) named = false;
            if (named) s.pair[slot * n_tokens + token] = static_cast<uint16_t>(thread + 1), s.any[slot] = 1;
        }
        __syncthreads();
        const uint64_t low = __builtin_amdgcn_ballot_w64(s.any[lane] != 0), high = __builtin_amdgcn_ballot_w64(s.any[lane + 64] != 0);
        const uint64_t below = (1ull << lane) - 1;
        n = bits_of(low) + bits_of(high);
        if (thread < 64) {
            if (low >> lane & 1) s.slot[bits_of(low & below)] = static_cast<uint8_t>(lane);
            if (high >> lane & 1) s.slot[bits_of(low) + bits_of(high & below)] = static_cast<uint8_t>(lane + 64);
        }
        __syncthreads();
    }
    __device__ __forceinline__ uint32_t count() const { return n; }
    __device__ __forceinline__ uint32_t expert(const Shared &s, uint32_t i) const { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(s.slot[i])); }
    __device__ __forceinline__ uint32_t list(const Shared &s, uint32_t expert, uint32_t &n) const
    {
        const uint32_t lane = threadIdx.x % 64, own = lane < n_tokens ? s.pair[expert * n_tokens + lane] : 0;
        const uint64_t there = __builtin_amdgcn_ballot_w64(own != 0);
        n = bits_of(there);
        const uint32_t got = static_cast<uint32_t>(__builtin_amdgcn_ds_permute(static_cast<int>(4 * (own ? bits_of(there & ((1ull << lane) - 1)) : 63u)), static_cast<int>(own)));
        return lane < n ? got : 0;
    }
    __device__ __forceinline__ uint32_t pair(const Shared &s, const Call &c, uint32_t expert, uint32_t t) const
    {
        return t < c.n_tokens ? s.pair[expert * c.n_tokens + t] : 0;
    }
};

// How a wave reads rows, for up to 16 / kParts tokens.  The 16 rows of a matrix instruction are kParts parts of kSide rows: part p holds
// values 32 p .. + 31 of every 32 kParts, and so do the columns 16 / kParts p .. of the tokens.  What a part of the rows gives with another part of the
// columns is not added up.  So one read of a wave takes kSide rows of 64 kParts bytes, up to 1 KB of one row, for a token; a wave's 16
// rows of 64 bytes are slower where there is little to read: 46 MB take 9.6 us in pieces of 1 KB, 11.5 of 128 bytes, 12.2 of 64.  (537 MB: 90 us, all three.)
template <int kParts>
struct Shape {
    static constexpr uint32_t kSide = 16 / kParts, kSpan = 32 * kParts, kUnit = 4 * kSpan;
    // this lane's row or column in its part, and where its values lie in a span
    static __device__ __forceinline__ uint32_t line(uint32_t lane) { return lane % kSide; }
    static __device__ __forceinline__ uint32_t within(uint32_t lane) { return lane % 16 / kSide * 32 + lane / 16 * 8; }
};

// Four matrix instructions' worth of a row: values k + kSpan i + within .. + 7, i = 0 .. 3; k is the same for all lanes.
struct Run {
    bf16x8 v[4];
};
template <bool kTight, int kParts>
__device__ __forceinline__ Run run_of(const uint16_t *row, uint32_t k, uint32_t within, uint32_t width)
{
    constexpr uint32_t kSpan = Shape<kParts>::kSpan;
    Run r;
    if (k + 4 * kSpan <= width) {
        row += k + within;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (kTight) __builtin_memcpy(&r.v[i], __builtin_assume_aligned(row + kSpan * i, 16), 16);
            else __builtin_memcpy(&r.v[i], row + kSpan * i, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t at = k + kSpan * i + within;
            if constexpr (kTight) {
                // eight values lie before the end or behind it.  No branch, which would wait for the request before: lanes behind
                // the end read the row's last values and drop them (a row of 1408 values, where this is all there is: 12.3 -> 9.8 us)
                __builtin_memcpy(&r.v[i], __builtin_assume_aligned(row + min(at, width - 8), 16), 16);
                if (at >= width) r.v[i] = bf16x8{};
            } else {
                r.v[i] = eight<false>(row, at, width);
            }
        }
    }
    return r;
}

// The rows of a tile, cut into blocks of kSide; a wave keeps to one block and takes its share of the rows' length.
template <int kParts>
struct FirstTile {
    static constexpr uint32_t kTileRows = kParts == 16 ? 8 : 16, kBlocks = kTileRows / Shape<kParts>::kSide, kSplits = kFirstWaves / kBlocks;
};

// Tiles of 16 rows (8 for one token) of gate and up of one chosen expert, taken in turn by the workgroups.
// kTiles: 16 tokens each that the call has at most.  Four waves per SIMD leave 128 registers, of which those for 2 to 16 tokens keep 4 to 8 in scratch memory.
template <class Pairs, bool kTight, int kTiles, int kParts>
__global__ void __launch_bounds__(64 * kFirstWaves, kTiles == 1 ? 4 : 2) zm_moe_few_first_kernel(const Call c, const Experts e)
{
    using Lines = Shape<kParts>;
    using Tile = FirstTile<kParts>;
    __shared__ typename Pairs::Shared s;
    __shared__ float part[kFirstWaves][2][16][17];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), within = Lines::within(lane);
    const uint32_t block = wave % Tile::kBlocks, split = wave / Tile::kBlocks;
    const Addresses gates(e, 0, lane), ups(e, 1, lane);
    const Pairs pairs(s, c, e);
    const uint32_t across = (c.intermediate + Tile::kTileRows - 1) / Tile::kTileRows, all = pairs.count() * across;
    struct Weights { Run g, u; };
    for (uint32_t tile = blockIdx.x; tile < all; tile += gridDim.x) {
        const uint32_t slot = pairs.expert(s, tile / across), row0 = tile % across * Tile::kTileRows;
        const uint64_t row = static_cast<uint64_t>(min(row0 + block * Lines::kSide + Lines::line(lane), c.intermediate - 1u)) * c.hidden;
        const uint16_t *gate = gates.of(slot) + row, *up = ups.of(slot) + row;
        auto weights_at = [&](uint32_t k) {
            return Weights{run_of<kTight, kParts>(gate, k, within, c.hidden), run_of<kTight, kParts>(up, k, within, c.hidden)};
        };
        constexpr uint32_t kStep = Lines::kUnit * Tile::kSplits;
        uint32_t k = Lines::kUnit * split;
        Weights w;
        if (k < c.hidden) w = weights_at(k);
        uint32_t count;
        const uint32_t listed = pairs.list(s, slot, count);
        const uint16_t *x[kTiles];
        bool has[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const uint32_t pair = static_cast<uint32_t>(__shfl(static_cast<int>(listed), 16 * t + static_cast<int>(Lines::line(lane))));
            has[t] = pair != 0;
            const uint32_t token = pair ? (pair - 1) / c.top_k : 0;
            x[t] = static_cast<const uint16_t *>(c.x) + token * c.x_stride;
        }
        f32x4 g[kTiles] = {}, u[kTiles] = {};
        auto multiply = [&](const Weights &w, uint32_t k) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                if (kTiles > 1 && 16u * t >= count) break;
                Run b{};
                if (has[t]) b = run_of<kTight, kParts>(x[t], k, within, c.hidden);
#pragma unroll
                for (int i = 0; i < 4; ++i) g[t] = mfma(w.g.v[i], b.v[i], g[t]), u[t] = mfma(w.u.v[i], b.v[i], u[t]);
            }
        };
        if (k < c.hidden) {
            for (; k + kStep < c.hidden; k += kStep) {                  // the next run's bytes are on their way while this one is multiplied
                const Weights next = weights_at(k + kStep);
                multiply(w, k);
                w = next;
            }
            multiply(w, k);
        }
        for (int t = 0; t < kTiles; ++t) {
            if (kTiles > 1 && 16u * t >= count) break;
            if (t || tile != blockIdx.x) __syncthreads();
            f32x4 gt = g[0], ut = u[0];
#pragma unroll
            for (int i = 1; i < kTiles; ++i)
                if (i == t) gt = g[i], ut = u[i];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                part[wave][0][lane % 16][4 * (lane / 16) + r] = gt[r];
                part[wave][1][lane % 16][4 * (lane / 16) + r] = ut[r];
            }
            __syncthreads();
            const uint32_t col = threadIdx.x / Tile::kTileRows, r = threadIdx.x % Tile::kTileRows;
            const uint32_t pair = static_cast<uint32_t>(__shfl(static_cast<int>(listed), static_cast<int>((16 * t + col) % 64)));
            if (col < Lines::kSide && pair && row0 + r < c.intermediate) {
                float gs = 0.0f, us = 0.0f, weight = 0.0f;
#pragma unroll
                for (uint32_t i = 0; i < Tile::kSplits; ++i)
#pragma unroll
                    for (uint32_t q = 0; q < kParts; ++q) {
                        const uint32_t of = r / Lines::kSide + i * Tile::kBlocks;
                        gs += part[of][0][col + Lines::kSide * q][r % Lines::kSide + Lines::kSide * q];
                        us += part[of][1][col + Lines::kSide * q][r % Lines::kSide + Lines::kSide * q];
                    }
                const uint32_t end = ((pair - 1) / c.top_k + 1) * c.top_k;
                const int32_t id = c.ids[pair - 1];
                for (uint32_t p0 = pair - 1; p0 < end; p0 += 4) {                     // four at once, without waiting for one another
                    int32_t ids[4];
                    float weights[4];
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) ids[i] = c.ids[min(p0 + i, end - 1)], weights[i] = c.weights[min(p0 + i, end - 1)];
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) weight += p0 + i < end && ids[i] == id ? weights[i] : 0.0f;
                }
                const float h = silu(gs) * us * weight;
                const __bf16 most = static_cast<__bf16>(h);
                const uint64_t at = static_cast<uint64_t>(pair - 1) * c.intermediate + row0 + r;
                c.h[at] = bits(most);
                const float rest = h - static_cast<float>(most);
                c.h_rest[at] = bits(static_cast<__bf16>(finite(rest) ? rest : 0.0f));      // most tells of what is not finite
            }
        }
    }
}

// 16 rows (8 for up to eight tokens, which gives twice as many workgroups) of every chosen expert's matrix down; the waves of a block take turns at the
// experts' runs.  gridDim.y > 1: each takes a part of the runs and leaves its sums in y for zm_moe_few_join_kernel.
template <class Pairs, bool kTight, int kTiles, int kParts>
__global__ void __launch_bounds__(64 * kSecondWaves, 4) zm_moe_few_second_kernel(const Call c, const Experts e)
{
    using Lines = Shape<kParts>;
    constexpr uint32_t kTileRows = kParts == 1 ? 16 : 8, kBlocks = kTileRows / Lines::kSide, kSplits = kSecondWaves / kBlocks;
    __shared__ typename Pairs::Shared s;
    __shared__ float part[kSecondWaves][16][17];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), within = Lines::within(lane);
    const uint32_t block = wave % kBlocks, split = wave / kBlocks, row0 = blockIdx.x * kTileRows;
    const Addresses downs(e, 2, lane);
    const Pairs pairs(s, c, e);
    const uint32_t runs = (c.intermediate + Lines::kUnit - 1) / Lines::kUnit, units = pairs.count() * runs;
    const uint64_t row = static_cast<uint64_t>(min(row0 + block * Lines::kSide + Lines::line(lane), c.hidden - 1u)) * c.intermediate;
    f32x4 y[kTiles] = {};
    // with one tile of columns h is asked for with the rows, a unit ahead; two tiles would not fit into the registers
    constexpr bool kAhead = kTiles == 1;
    struct Columns { Run most, rest; };
    struct Unit {
        Run w;
        Columns h;
        uint32_t slot, k, pair;
    };
    auto columns_at = [&](uint32_t pair, uint32_t k) {
        Columns n{};
        if (pair) {
            const uint64_t at = static_cast<uint64_t>(pair - 1) * c.intermediate;
            n.most = run_of<kTight, kParts>(c.h + at, k, within, c.intermediate);
            n.rest = run_of<kTight, kParts>(c.h_rest + at, k, within, c.intermediate);
        }
        return n;
    };
    auto load = [&](uint32_t unit) {
        Unit n;
        n.slot = pairs.expert(s, unit / runs), n.k = unit % runs * Lines::kUnit;
        n.w = run_of<kTight, kParts>(downs.of(n.slot) + row, n.k, within, c.intermediate);
        if constexpr (kAhead) {
            n.pair = pairs.pair(s, c, n.slot, Lines::line(lane));
            n.h = columns_at(n.pair, n.k);
        }
        return n;
    };
    auto multiply = [&](const Unit &n) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const uint32_t pair = kAhead ? n.pair : pairs.pair(s, c, n.slot, 16 * t + Lines::line(lane));
            if (!kAhead && __builtin_amdgcn_ballot_w64(pair != 0) == 0) continue;
            const Columns h = kAhead ? n.h : columns_at(pair, n.k);
            f32x4 sum = {}, rest = {};
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = mfma(n.w.v[i], h.most.v[i], sum), rest = mfma(n.w.v[i], h.rest.v[i], rest);
            // an infinite weight times the zeros of a token that did not choose the expert is none of the token's, nor is one times a remainder
            // of zero, or of the other sign: where the first parts give no finite sum they give the result
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[r] += finite(sum[r]) ? rest[r] : 0.0f;
            if (pair) y[t] += sum;
        }
    };
    const uint32_t step = kSplits * gridDim.y;
    uint32_t unit = blockIdx.y * kSplits + split;
    if (unit < units) {
        Unit n = load(unit);
        for (; unit + step < units; unit += step) {
            const Unit next = load(unit + step);
            multiply(n);
            n = next;
        }
        multiply(n);
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        if (t) __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r) part[wave][lane % 16][4 * (lane / 16) + r] = y[t][r];
        __syncthreads();
        const uint32_t col = threadIdx.x / kTileRows, token = 16 * t + col, r = threadIdx.x % kTileRows;
        if (col < Lines::kSide && token < c.n_tokens && row0 + r < c.hidden) {
            const bool whole = gridDim.y == 1;
            float sum = whole && c.residual ? of_bf16(c.residual[token * c.residual_stride + row0 + r]) : 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < kSplits; ++i)
#pragma unroll
                for (uint32_t q = 0; q < kParts; ++q)
                    sum += part[r / Lines::kSide + i * kBlocks][col + Lines::kSide * q][r % Lines::kSide + Lines::kSide * q];
            if (whole) c.out[token * c.out_stride + row0 + r] = bits(static_cast<__bf16>(sum));
            else c.y[(static_cast<uint64_t>(blockIdx.y) * c.n_tokens + token) * c.hidden + row0 + r] = sum;
        }
    }
}

__global__ void __launch_bounds__(256) zm_moe_few_join_kernel(const Call c, uint32_t parts)
{
    const uint32_t col = blockIdx.x * 256 + threadIdx.x, token = blockIdx.y;
    if (col >= c.hidden) return;
    float sum = c.residual ? of_bf16(c.residual[token * c.residual_stride + col]) : 0.0f;
    for (uint32_t p = 0; p < parts; ++p) sum += c.y[(static_cast<uint64_t>(p) * c.n_tokens + token) * c.hidden + col];
    c.out[token * c.out_stride + col] = bits(static_cast<__bf16>(sum));
}

// ---- many tokens: product ----

// A workgroup of four waves multiplies 128 pairs with 256 rows, a wave 64 with 128; 32 values of each at a time lie in LDS, three times
// 24 KB, so that two workgroups share a compute unit and the bytes of the step after next are on their way.  They go from memory to
// LDS without passing through registers.  A row's 64 bytes are four pieces of 16; piece q of row r lies in place q ^ (r / 2) % 4, so that the 16 rows
// that a wave reads at once spread over all banks.
constexpr uint32_t kPairs = 128, kRows = 256, kDeep = 32, kStages = 3, kStageBytes = (kPairs + kRows) * 2 * kDeep;

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// 16 bytes per lane from memory to LDS, lane after lane from `to` on.
__device__ __forceinline__ void to_lds(uint32_t to, uint32_t offset, i32x4 from, uint32_t step)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(offset), "s"(from), "s"(step) : "memory", "m0");
}
// All but the last n requests have arrived, for every wave of the workgroup, and nobody reads the stage before any more.
template <int n>
__device__ __forceinline__ void arrived()
{
    static_assert(n == 0 || n == 6 || n == 8);
    if constexpr (n == 8) asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else if constexpr (n == 6) asm volatile("s_waitcnt vmcnt(6) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ __forceinline__ i32x4 descriptor(const void *p, uint32_t bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return i32x4{__builtin_amdgcn_readfirstlane(static_cast<int32_t>(a)), __builtin_amdgcn_readfirstlane(static_cast<int32_t>(a >> 32 & 0xffff)),
                 __builtin_amdgcn_readfirstlane(static_cast<int32_t>(bytes)), 0x00027000};
}

// Which tile of kPairs pairs (or kMore, where an expert has fewer tiles of that height) and kColumns columns a workgroup takes: experts one after
// the other, and inside an expert all tiles of pairs before the next columns.  An XCD's eighth of the workgroups (every eighth) takes tiles that
// lie together, which read the same rows and pairs.
struct TileOf {
    uint32_t slot, count, first, pair0, column0, height;

    template <uint32_t kPairs, uint32_t kMore, uint32_t kColumns>
    __device__ __forceinline__ bool find(const Call &c, const Experts &e, uint32_t columns)
    {
        auto tiles_of = [](uint32_t n) { return min((n + kPairs - 1) / kPairs, (n + kMore - 1) / kMore); };
        const uint32_t lane = threadIdx.x % 64, across = (columns + kColumns - 1) / kColumns;
        const uint32_t count0 = lane < e.n ? c.count[lane] : 0, count1 = lane + 64 < e.n ? c.count[lane + 64] : 0;
        uint32_t end0 = tiles_of(count0), end1 = tiles_of(count1);
        const uint32_t tiles0 = end0, tiles1 = end1;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t a = __shfl_up(end0, d), b = __shfl_up(end1, d);
            if (lane >= static_cast<uint32_t>(d)) end0 += a, end1 += b;
        }
        end1 += __builtin_amdgcn_readlane(end0, 63);
        const uint32_t tiles = static_cast<uint32_t>(__builtin_amdgcn_readlane(end1, 63)) * across, each = (tiles + 7) / 8;
        const uint32_t tile = blockIdx.x % 8 * each + blockIdx.x / 8;
        if (blockIdx.x / 8 >= each || tile >= tiles) return false;
        slot = __builtin_popcountll(__builtin_amdgcn_ballot_w64(end0 * across <= tile)) + __builtin_popcountll(__builtin_amdgcn_ballot_w64(end1 * across <= tile));
        const uint32_t from = slot % 64;
        const uint32_t down = slot < 64 ? read_lane(tiles0, from) : read_lane(tiles1, from), end = slot < 64 ? read_lane(end0, from) : read_lane(end1, from);
        count = slot < 64 ? read_lane(count0, from) : read_lane(count1, from);
        const uint32_t within = tile - (end - down) * across;
        height = down < (count + kPairs - 1) / kPairs ? kMore : kPairs;
        pair0 = within % down * height, column0 = within / down * kColumns;
        first = c.first[slot];
        return true;
    }
};

// kFirst: gate and up, 16 rows of one after 16 of the other, to h; else down, to y.  kDirect: 16-byte-aligned rows.  Others pass through registers, and a workgroup
// takes half as many of them, which leaves room for two steps' bytes.
template <bool kFirst, bool kDirect>
__global__ void __launch_bounds__(256, 2) zm_moe_product_kernel(const Call c, const Experts e)
{
    __shared__ alignas(16) uint8_t lds[kStages * kStageBytes];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t depth = kFirst ? c.hidden : c.intermediate, columns = kFirst ? c.intermediate : c.hidden;
    constexpr uint32_t kTall = kDirect ? kRows : kRows / 2, kColumns = kFirst ? kTall / 2 : kTall, kAsks = kTall / 64, kBlocks = kTall / 32;
    TileOf of;
    if (!of.find<kPairs, kPairs, kColumns>(c, e, columns)) return;
    const uint32_t slot = of.slot, count = of.count, pair0 = of.pair0, column0 = of.column0, first = of.first;

    // Rows of the pairs (two requests of a wave) and of the matrices (kAsks): this lane's row and its piece of it.
    const uint32_t piece = 8 * ((lane % 4) ^ (lane / 8 % 4));
    const uint16_t *base = kFirst ? static_cast<const uint16_t *>(c.x) : c.h + static_cast<uint64_t>(first + pair0) * depth;
    uint64_t pair_at[2];
    uint32_t row_at[kAsks];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t p = min(pair0 + (2 * wave + j) * 16 + lane / 4, count - 1);
        pair_at[j] = kFirst ? static_cast<uint64_t>(c.list[first + p] / c.top_k) * c.x_stride : static_cast<uint64_t>(p - pair0) * depth;
    }
    const uint16_t *const matrix[2] = {e.tensor[slot][kFirst ? 0 : 2], e.tensor[slot][kFirst ? 1 : 2]};
#pragma unroll
    for (uint32_t j = 0; j < kAsks; ++j) {
        const uint32_t r = (kAsks * wave + j) * 16 + lane / 4;
        row_at[j] = min(column0 + (kFirst ? r / 32 * 16 + r % 16 : r), columns - 1) * depth;
    }
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t *)lds));
    // where the lane reads: row lane % 16 of 16, piece lane / 16
    const uint32_t read = lane % 16 * 64 + 16 * ((lane / 16) ^ (lane % 16 / 2 % 4));
    const uint32_t read_pairs = wave % 2 * 64 * 64 + read, read_rows = kPairs * 64 + wave / 2 * (kTall / 2) * 64 + read;

    f32x4 acc[kBlocks][4] = {};
    auto multiply = [&](uint32_t stage) {
        const uint8_t *at = lds + stage * kStageBytes;
        bf16x8 a[kBlocks], b[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) b[t] = *reinterpret_cast<const bf16x8 *>(at + read_pairs + t * 1024);
#pragma unroll
        for (uint32_t u = 0; u < kBlocks; ++u) a[u] = *reinterpret_cast<const bf16x8 *>(at + read_rows + u * 1024);
#pragma unroll
        for (uint32_t u = 0; u < kBlocks; ++u)
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[u][t] = mfma(a[u], b[t], acc[u][t]);
    };

    uint32_t k = 0;
    if constexpr (kDirect) {
        const uint64_t extent = kFirst ? (static_cast<uint64_t>(c.n_tokens - 1) * c.x_stride + depth) * 2 : static_cast<uint64_t>(min(count - pair0, kPairs)) * depth * 2;
        const i32x4 pairs = descriptor(base, static_cast<uint32_t>(extent));
        const i32x4 rows0 = descriptor(matrix[0], columns * depth * 2), rows1 = descriptor(matrix[1], columns * depth * 2);
        uint32_t pair_byte[2], row_byte[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) pair_byte[j] = static_cast<uint32_t>(2 * (pair_at[j] + piece));
#pragma unroll
        for (int j = 0; j < 4; ++j) row_byte[j] = 2 * (row_at[j] + piece);
        const uint32_t steps = depth / kDeep;
        auto request = [&](uint32_t step) {
            const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + step % kStages * kStageBytes), at = step * kDeep * 2;
#pragma unroll
            for (int j = 0; j < 2; ++j) to_lds(to + (2 * wave + j) * 1024, pair_byte[j], pairs, at);
#pragma unroll
            for (int j = 0; j < 4; ++j) to_lds(to + kPairs * 64 + (4 * wave + j) * 1024, row_byte[j], j % 2 ? rows1 : rows0, at);
        };
        if (steps > 0) request(0);
        if (steps > 1) request(1);
        for (uint32_t step = 0; step < steps; ++step) {
            if (step + 1 < steps) arrived<6>();
            else arrived<0>();
            if (step + 2 < steps) request(step + 2);
            multiply(step % kStages);
        }
        k = steps * kDeep;
        if (k < depth) arrived<0>();
    }
    if (k < depth) {
        // what is left of the rows, or all of them: through registers, two steps ahead, zeros behind their end.  A stage is written anew three steps
        // later, behind two barriers.
        bf16x8 held[2][2 + kAsks];
        auto load = [&](bf16x8 (&to)[2 + kAsks], uint32_t at) {
#pragma unroll
            for (int j = 0; j < 2; ++j) to[j] = eight<false>(base + pair_at[j], at + piece, depth);
#pragma unroll
            for (uint32_t j = 0; j < kAsks; ++j) to[2 + j] = eight<false>(matrix[j % 2] + row_at[j], at + piece, depth);
        };
        auto store = [&](uint32_t stage, const bf16x8 (&from)[2 + kAsks]) {
            uint8_t *to = lds + stage * kStageBytes + 16 * lane;
#pragma unroll
            for (int j = 0; j < 2; ++j) *reinterpret_cast<bf16x8 *>(to + (2 * wave + j) * 1024) = from[j];
#pragma unroll
            for (uint32_t j = 0; j < kAsks; ++j) *reinterpret_cast<bf16x8 *>(to + kPairs * 64 + (kAsks * wave + j) * 1024) = from[2 + j];
        };
        load(held[0], k);
        if (k + kDeep < depth) load(held[1], k + kDeep);
        uint32_t stage = 0;
        auto step = [&](bf16x8 (&own)[2 + kAsks]) {
            store(stage, own);
            __syncthreads();
            if (k + 2 * kDeep < depth) load(own, k + 2 * kDeep);
            multiply(stage);
            stage = stage == kStages - 1 ? 0 : stage + 1, k += kDeep;
        };
        while (true) {
            step(held[0]);
            if (k >= depth) break;
            step(held[1]);
            if (k >= depth) break;
        }
    }

    // lane: pair lane % 16 of 16, columns 4 (lane / 16) .. + 3 of 16
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t p = pair0 + wave % 2 * 64 + 16 * t + lane % 16;
        if (p >= count) continue;
        if constexpr (kFirst) {
            uint16_t *to = c.h + static_cast<uint64_t>(first + p) * columns;
#pragma unroll
            for (uint32_t u = 0; u < kBlocks; u += 2) {
                const uint32_t col = column0 + (wave / 2 * (kBlocks / 2) + u / 2) * 16 + 4 * (lane / 16);
                uint16_t w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = bits(static_cast<__bf16>(silu_short(acc[u][t][r]) * acc[u + 1][t][r]));
                if (col + 4 <= columns) __builtin_memcpy(to + col, w, 8);
                else
                    for (uint32_t r = 0; r < 4; ++r)
                        if (col + r < columns) to[col + r] = w[r];
            }
        } else {
            float *to = c.y + static_cast<uint64_t>(c.list[first + p]) * columns;
#pragma unroll
            for (uint32_t u = 0; u < kBlocks; ++u) {
                const uint32_t col = column0 + (wave / 2 * kBlocks + u) * 16 + 4 * (lane / 16);
                if (col + 4 <= columns) __builtin_memcpy(to + col, &acc[u][t], 16);
                else
                    for (uint32_t r = 0; r < 4; ++r)
                        if (col + r < columns) to[col + r] = acc[u][t][r];
            }
        }
    }
}

// The same for experts of many pairs, whose rows are a multiple of 64 values and 16-byte aligned.  A workgroup of eight waves multiplies 256
// pairs with 256 rows, a wave 128 with 64: two thirds of the bytes that the tile above asks of memory for a product, seven eighths of
// those that pass through LDS.  Where 288 pairs make fewer tiles of an expert, a wave takes 144: a router that spreads its tokens evenly gives experts a
// few pairs more or less than a multiple of 256, and a tile of a few pairs takes as long to read the matrices as a full one.
//
// A step of 64 values, whole cache lines, takes 68 KB of LDS, two of them.  Of a row's 128 bytes in eight pieces of 16, piece q of row r lies in
// place q ^ (r / 2) % 8: no read meets two of one bank.  A step is multiplied in two halves; the operands of the half after are read
// from LDS meanwhile, and a step's place is asked for anew once its second half is in registers, so that the bytes have the time of a step to arrive.
constexpr uint32_t kWidePairs = 256, kWideMore = 288, kWideDeep = 64, kWideStageBytes = (kWideMore + kRows) * 2 * kWideDeep;

template <bool kFirst>
__global__ void __launch_bounds__(512, 2) zm_moe_wide_kernel(const Call c, const Experts e)
{
    __shared__ alignas(16) uint8_t lds[2 * kWideStageBytes];
    __shared__ uint32_t kept[7][512];            // what a lane adds to the addresses of its requests: registers are for operands and sums
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t depth = kFirst ? c.hidden : c.intermediate, columns = kFirst ? c.intermediate : c.hidden;
    constexpr uint32_t kColumns = kFirst ? kRows / 2 : kRows;
    TileOf of;
    if (!of.find<kWidePairs, kWideMore, kColumns>(c, e, columns)) return;
    const uint32_t pair0 = of.pair0, column0 = of.column0, first = of.first, count = min(of.count, pair0 + of.height);

    // four requests of a wave for rows of the pairs, four for rows of the matrices, eight rows each: this lane's row of the eight and its piece of
    // it; of 288 pairs the first waves ask for the last 32.  Eight rows of a matrix lie inside it or behind its end (64 are).
    uint32_t group_byte[4];
    struct Offsets { uint32_t pair[5], row[2]; };
    const bool fifth = __builtin_amdgcn_readfirstlane(count - pair0) > kWidePairs && wave < 4;
#pragma unroll
    for (uint32_t j = 0; j < 5; ++j) {
        const uint32_t r = (j < 4 ? (4 * wave + j) * 8 : kWidePairs + wave % 4 * 8) + lane / 8, piece = 8 * ((lane % 8) ^ (r / 2 % 8)), p = min(pair0 + r, count - 1);
        kept[j][threadIdx.x] = static_cast<uint32_t>(2 * ((kFirst ? static_cast<uint64_t>(c.list[first + p] / c.top_k) * c.x_stride : static_cast<uint64_t>(p - pair0) * depth) + piece));
        if (j < 2) kept[5 + j][threadIdx.x] = 2 * (lane / 8 * depth + piece);
        if (j < 4) group_byte[j] = __builtin_amdgcn_readfirstlane(2 * min(column0 + (kFirst ? 16 * wave + j % 2 * 8 : 32 * wave + 8 * j), columns - 8) * depth);
    }
    const uint16_t *base = kFirst ? static_cast<const uint16_t *>(c.x) : c.h + static_cast<uint64_t>(first + pair0) * depth;
    const uint64_t extent = kFirst ? (static_cast<uint64_t>(c.n_tokens - 1) * c.x_stride + depth) * 2 : static_cast<uint64_t>(count - pair0) * depth * 2;
    const i32x4 pairs = descriptor(base, static_cast<uint32_t>(extent));
    const i32x4 rows[2] = {descriptor(e.tensor[of.slot][kFirst ? 0 : 2], columns * depth * 2), descriptor(e.tensor[of.slot][kFirst ? 1 : 2], columns * depth * 2)};
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t *)lds));
    const uint32_t steps = depth / kWideDeep;
    auto offsets = [&]() __attribute__((always_inline)) {
        Offsets o;
#pragma unroll
        for (int j = 0; j < 5; ++j) o.pair[j] = kept[j][threadIdx.x];
#pragma unroll
        for (int j = 0; j < 2; ++j) o.row[j] = kept[5 + j][threadIdx.x];
        return o;
    };
    auto request = [&](uint32_t step, uint32_t place, const Offsets &o) __attribute__((always_inline)) {
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + place * kWideStageBytes), at = step * kWideDeep * 2;
#pragma unroll
        for (int j = 0; j < 4; ++j) to_lds(to + (4 * wave + j) * 1024, o.pair[j], pairs, at);
#pragma unroll
        for (int j = 0; j < 4; ++j) to_lds(to + kWideMore * 128 + (4 * wave + j) * 1024, o.row[j % 2], rows[j / 2], group_byte[j] + at);
        if (fifth) to_lds(to + kWidePairs * 128 + wave * 1024, o.pair[4], pairs, at);
    };

    // waves 0 .. 3 take the first half of the pairs, 64 rows each, the others the rest
    const uint32_t pairs_of_wave = wave / 4 * (of.height / 2);
    const uint32_t blocks = __builtin_amdgcn_readfirstlane(min((max(count - pair0, pairs_of_wave) - pairs_of_wave + 15) / 16, of.height / 32));
    // piece lane / 16 (first half) or that + 4 (second) of row lane % 16, behind the wave's first row of either kind
    const uint32_t within = lane % 16 * 128 + 16 * ((lane / 16) ^ (lane % 16 / 2)), pairs_at = pairs_of_wave * 128, rows_at = (kWideMore + wave % 4 * 64) * 128;
    constexpr int kMost = kWideMore / 32, kSpare = 3;
    f32x4 acc[kMost][4] = {};
    // kBlocks times 16 pairs.  The operands of a half wait in b[0 ..], and the next half's take the place of those that are multiplied, kSpare
    // blocks of them ahead: so many registers more, and no read that has just been asked for is waited for at the barrier.
    auto run = [&](auto number) __attribute__((always_inline)) {
        constexpr int kBlocks = number.value;
        bf16x8 a[2][4], b[kMost + kSpare];
        auto read_a = [&](uint32_t step, int half) __attribute__((always_inline)) {
            const uint8_t *at = lds + step % 2 * kWideStageBytes + rows_at + (within ^ (half * 64u));
#pragma unroll
            for (int u = 0; u < 4; ++u) a[half][u] = *reinterpret_cast<const bf16x8 *>(at + u * 2048);
        };
        auto read_b = [&](uint32_t step, int half, int t) __attribute__((always_inline)) { return *reinterpret_cast<const bf16x8 *>(lds + step % 2 * kWideStageBytes + pairs_at + (within ^ (half * 64u)) + t * 2048); };
        auto multiply = [&](int half, int t, const bf16x8 &of) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < 4; ++u) acc[t][u] = mfma(a[half][u], of, acc[t][u]);
        };
        constexpr int kTurns = kBlocks > kSpare ? kBlocks - kSpare : 0, kFree = kBlocks - kTurns;      // kFree: blocks in the spare places
        if (steps > 1) arrived<8>();
        else arrived<0>();
        if constexpr (kBlocks > 0) {
            read_a(0, 0);
#pragma unroll
            for (int t = 0; t < kBlocks; ++t) b[t] = read_b(0, 0, t);
        }
        // the halves of a step: the first, in b[0 ..], while the second is read; the second while the next step's first is read
        auto early = [&](uint32_t step) __attribute__((always_inline)) {
            read_a(step, 1);
#pragma unroll
            for (int t = 0; t < kFree; ++t) b[kMost + t] = read_b(step, 1, t);
#pragma unroll
            for (int t = 0; t < kTurns; ++t) {
                multiply(0, t, b[t]);
                b[t] = read_b(step, 1, kFree + t);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int t = kTurns; t < kBlocks; ++t) multiply(0, t, b[t]);
        };
        for (uint32_t step = 0; step + 1 < steps; ++step) {
            if constexpr (kBlocks > 0) early(step);
            const Offsets o = offsets();
            arrived<0>();                              // the next step, and nobody has a read of this one under way
            request(min(step + 2, steps - 1), step % 2, o);    // behind the last step: bytes that nobody reads
            if constexpr (kBlocks > 0) {
                read_a(step + 1, 0);
#pragma unroll
                for (int t = kTurns; t < kBlocks; ++t) b[t] = read_b(step + 1, 0, t);
#pragma unroll
                for (int t = 0; t < kTurns; ++t) {
                    multiply(1, kFree + t, b[t]);
                    b[t] = read_b(step + 1, 0, t);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int t = 0; t < kFree; ++t) multiply(1, t, b[kMost + t]);
            }
        }
        if constexpr (kBlocks > 0) {
            early(steps - 1);
#pragma unroll
            for (int t = 0; t < kTurns; ++t) multiply(1, kFree + t, b[t]);
#pragma unroll
            for (int t = 0; t < kFree; ++t) multiply(1, t, b[kMost + t]);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // LDS that is written belongs to this workgroup still
    };
    request(0, 0, offsets());
    if (steps > 1) request(1, 1, offsets());
    // few code paths: the others multiply some blocks more, of columns that nobody stores
    if (blocks > 8) run(std::integral_constant<int, 9>{});
    else if (blocks > 4) run(std::integral_constant<int, 8>{});
    else if (blocks > 2) run(std::integral_constant<int, 4>{});
    else if (blocks > 0) run(std::integral_constant<int, 2>{});
    else run(std::integral_constant<int, 0>{});

    // lane: pair lane % 16 of 16, columns 4 (lane / 16) .. + 3 of 16
#pragma unroll
    for (int t = 0; t < kMost; ++t) {
        const uint32_t p = pair0 + pairs_of_wave + 16 * t + lane % 16;
        if (16u * t >= of.height / 2 || p >= count) continue;
        if constexpr (kFirst) {
            uint16_t *to = c.h + static_cast<uint64_t>(first + p) * columns;
#pragma unroll
            for (int u = 0; u < 4; u += 2) {
                const uint32_t col = column0 + (wave % 4 * 2 + u / 2) * 16 + 4 * (lane / 16);
                uint16_t w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = bits(static_cast<__bf16>(silu_short(acc[t][u][r]) * acc[t][u + 1][r]));
                if (col < columns) __builtin_memcpy(to + col, w, 8);
            }
        } else {
            float *to = c.y + static_cast<uint64_t>(c.list[first + p]) * columns;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t col = column0 + (wave % 4 * 4 + u) * 16 + 4 * (lane / 16);
                if (col < columns) __builtin_memcpy(to + col, &acc[t][u], 16);
            }
        }
    }
}

// e4m3 rows as bf16 ones, zeros up to a multiple of eight values
__global__ void __launch_bounds__(256) zm_moe_widen_kernel(const Call c)
{
    const uint64_t runs = c.wide_stride / 8, at = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (at >= runs * c.n_tokens) return;
    const uint64_t token = at / runs;
    const uint32_t k = static_cast<uint32_t>(at % runs) * 8;
    const bf16x8 v = eight_scaled(static_cast<const uint8_t *>(c.x) + token * c.x_stride, c.scales + token * c.scales_stride, k, c.hidden);
    __builtin_memcpy(__builtin_assume_aligned(c.wide_x + token * c.wide_stride + k, 16), &v, 16);
}

// ---- join ----

// Four columns of a token per lane; four pairs' sums are asked for before it is known which of them count.
__global__ void __launch_bounds__(256) zm_moe_join_kernel(const Call c, const Ids e)
{
    const uint32_t token = blockIdx.y, lane = threadIdx.x % 64, col = 4 * (blockIdx.x * 256u + threadIdx.x), there = col < c.hidden ? min(c.hidden - col, 4u) : 0;
    const int32_t low = lane < e.n ? e.id[lane] : -1, high = lane + 64 < e.n ? e.id[lane + 64] : -1;
    const uint64_t pair0 = static_cast<uint64_t>(token) * c.top_k;
    auto four = [&](const auto *from, auto (&to)[4]) {
        if (there == 4) {
            __builtin_memcpy(to, from, sizeof to);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) to[i] = i < there ? from[i] : 0;
        }
    };
    float sum[4] = {};
    if (c.residual) {
        uint16_t r[4];
        four(c.residual + token * c.residual_stride + col, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = of_bf16(r[i]);
    }
    for (uint32_t j0 = 0; j0 < c.top_k; j0 += 4) {
        float y[4][4];
        int32_t id[4];
        float weight[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint64_t pair = pair0 + min(j0 + j, c.top_k - 1);
            id[j] = c.ids[pair], weight[j] = c.weights[pair];
            four(c.y + pair * c.hidden + col, y[j]);
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const bool named = __builtin_amdgcn_ballot_w64((lane < e.n && low == id[j]) || (lane + 64 < e.n && high == id[j])) != 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += named && j0 + j < c.top_k ? weight[j] * y[j][i] : 0.0f;
        }
    }
    uint16_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = bits(static_cast<__bf16>(sum[i]));
    uint16_t *to = c.out + token * c.out_stride + col;
    if (there == 4) {
        __builtin_memcpy(to, r, sizeof r);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (i < there) to[i] = r[i];
    }
}

// ---- host ----

constexpr uint32_t kUnits = 256;         // compute units
constexpr uint32_t kFewGrid = 1024;      // workgroups of few_first
// Pairs per expert that the call names from which the large tiles are taken; how they spread over the experts is known on the device only.  us small / large tiles, experts of 4096 x 14336, 128 pairs each 796 / 818, 192 905 / 839,
// 1024 3216 / 2392; of 2048 x 1024, 128 259 / 287, 192 296 / 291, 512 655 / 595; of 2048 x 1408, 137 318 / 353, 273 574 / 533.
constexpr uint64_t kWideFrom = 160;
constexpr uint32_t kFewParts = 4;        // most workgroups that share the rows of few_second

constexpr size_t kAlign = 256;
size_t aligned(size_t n) { return (n + kAlign - 1) & ~(kAlign - 1); }

bool sizes_ok(int64_t n_tokens, int64_t top_k, int64_t hidden, int64_t intermediate, int64_t n_experts)
{
    return n_tokens >= 0 && n_tokens < (1ll << 24) && top_k >= 1 && top_k <= 1024 && n_tokens * top_k < (1ll << 24) && hidden >= 1 && intermediate >= 1 &&
           hidden <= (1ll << 20) && intermediate <= (1ll << 20) && hidden * intermediate < (1ll << 31) && n_experts >= 0 && n_experts <= ZM_MOE_MAX_EXPERTS;
}

// Places of the workspace's parts; the bytes of all of them.
size_t place(Call &c, uint8_t *base, int64_t n_tokens, int64_t top_k, int64_t hidden, int64_t intermediate)
{
    const size_t pairs = static_cast<size_t>(n_tokens * top_k);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t was = at; at += aligned(bytes); return base + was; };
    c.first = reinterpret_cast<uint32_t *>(take(4 * ZM_MOE_MAX_EXPERTS));
    c.count = reinterpret_cast<uint32_t *>(take(4 * ZM_MOE_MAX_EXPERTS));
    c.list = reinterpret_cast<uint32_t *>(take(4 * pairs));
    c.h = reinterpret_cast<uint16_t *>(take(2 * pairs * static_cast<size_t>(intermediate)));
    c.wide_stride = static_cast<uint32_t>((hidden + 7) / 8 * 8);
    c.wide_x = reinterpret_cast<uint16_t *>(take(2 * static_cast<size_t>(n_tokens) * c.wide_stride));
    // few tokens need the rest of h, many of them y: what a smaller call needs of either is there too
    c.h_rest = reinterpret_cast<uint16_t *>(base + at);
    at += aligned(2 * (pairs < kFewPairs ? pairs : kFewPairs) * static_cast<size_t>(intermediate));
    const size_t few = static_cast<size_t>(n_tokens < kFewTokens ? n_tokens : kFewTokens) * kFewParts;
    c.y = reinterpret_cast<float *>(take(4 * (pairs > few ? pairs : few) * static_cast<size_t>(hidden)));
    return at;
}

int launch(const void *fn, dim3 grid, dim3 block, void **args, hipStream_t stream)
{
    return hipLaunchKernel(fn, grid, block, args, 0, stream) == hipSuccess ? ZM_OK : ZM_E_HIP;
}

int widen(Call &c, hipStream_t stream)
{
    const uint64_t runs = static_cast<uint64_t>(c.wide_stride / 8) * c.n_tokens;
    void *args[] = {&c};
    return launch(reinterpret_cast<const void *>(&zm_moe_widen_kernel), dim3(static_cast<uint32_t>((runs + 255) / 256)), dim3(256), args, stream);
}

// The kernels of few tokens: up to 64 pairs without tables, parts by the number of tokens (Shape), and the rows of their tiles.
struct Few {
    const void *first, *second;
    uint32_t first_rows, second_rows;
};
template <class Pairs, bool kTight, bool kTightDown, int kTiles, int kParts>
Few few_kernels()
{
    return {reinterpret_cast<const void *>(&zm_moe_few_first_kernel<Pairs, kTight, kTiles, kParts>),
            reinterpret_cast<const void *>(&zm_moe_few_second_kernel<Pairs, kTightDown, kTiles, kParts>), FirstTile<kParts>::kTileRows, kParts == 1 ? 16u : 8u};
}
template <bool kTight, bool kTightDown>
Few few_of(const Call &c)
{
    if (c.n_tokens > 16) return few_kernels<MorePairs, kTight, kTightDown, 2, 1>();
    if (c.n_pairs > 64) return few_kernels<MorePairs, kTight, kTightDown, 1, 1>();
    if (c.n_tokens > 8) return few_kernels<FewPairs, kTight, kTightDown, 1, 1>();
    if (c.n_tokens > 4) return few_kernels<FewPairs, kTight, kTightDown, 1, 2>();
    if (c.n_tokens > 1) return few_kernels<FewPairs, kTight, kTightDown, 1, 4>();
    return few_kernels<FewPairs, kTight, kTightDown, 1, 16>();
}

}  // namespace

bool zipmoe::moe_check(const zm_moe_args &a, const void *workspace)
{
    const bool scaled = a.x_type == ZM_MXFP8;
    return a.x && a.ids && a.weights && a.out && workspace && (scaled || a.x_type == ZM_BF16) && scaled == (a.scales != nullptr) && a.x_stride >= 0 &&
           (!scaled || a.scales_stride >= 0) && (!a.residual || a.residual_stride >= 0) && (a.n_tokens <= 1 || a.out_stride >= a.hidden) &&
           aligned_to(workspace, kAlign) && aligned_to(a.x, type_bytes(a.x_type)) && aligned_to(a.ids, 4) && aligned_to(a.weights, 4) &&
           aligned_to(a.residual, 2) && aligned_to(a.out, 2);
}

zipmoe::MoePlaces zipmoe::moe_places(void *workspace, const zm_moe_args &a)
{
    Call c;
    place(c, static_cast<uint8_t *>(workspace), a.n_tokens, a.top_k, a.hidden, a.intermediate);
    return {c.h, c.h_rest, c.wide_x, c.wide_stride};
}

int zipmoe::moe_widen(const zm_moe_args &a, const MoePlaces &to, hipStream_t stream)
{
    Call c{};
    c.x = a.x, c.scales = static_cast<const uint8_t *>(a.scales), c.x_stride = a.x_stride, c.scales_stride = a.scales_stride;
    c.n_tokens = static_cast<uint32_t>(a.n_tokens), c.hidden = static_cast<uint32_t>(a.hidden), c.wide_x = to.wide_x, c.wide_stride = to.wide_stride;
    return widen(c, stream);
}

extern "C" {

int zm_moe_workspace_bytes(int64_t n_tokens, int top_k, int hidden, int intermediate, int n_experts, size_t *bytes)
{
    if (!bytes || !sizes_ok(n_tokens, top_k, hidden, intermediate, n_experts)) return ZM_E_ARG;
    Call c;
    *bytes = place(c, nullptr, n_tokens, top_k, hidden, intermediate);
    return ZM_OK;
}

int zm_moe(const void *const *tensors, const int32_t *expert_ids, int n_experts, const zm_moe_args *a, void *workspace, size_t workspace_bytes,
           void *stream)
{
    if (!a || n_experts < 0 || (n_experts && (!tensors || !expert_ids))) return ZM_E_ARG;
    if (a->x_type != ZM_BF16 && a->x_type != ZM_MXFP8) return ZM_E_ARG;
    size_t need = 0;
    const int rc = zm_moe_workspace_bytes(a->n_tokens, a->top_k, a->hidden, a->intermediate, n_experts, &need);
    if (rc != ZM_OK) return rc;
    if (a->n_tokens == 0) return ZM_OK;
    const bool scaled = a->x_type == ZM_MXFP8;
    if (!moe_check(*a, workspace)) return ZM_E_ARG;
    Experts e;
    Ids ids;
    e.n = ids.n = static_cast<uint32_t>(n_experts);
    bool even[2] = {a->hidden % 8 == 0, a->intermediate % 8 == 0};           // rows of gate and up, of down: all 16-byte aligned
    for (int i = 0; i < n_experts; ++i) {
        for (int j = 0; j < i; ++j)
            if (expert_ids[j] == expert_ids[i]) return ZM_E_ARG;
        e.id[i] = ids.id[i] = expert_ids[i];
        for (int m = 0; m < 3; ++m) {
            if (!tensors[3 * i + m] || !aligned_to(tensors[3 * i + m], 2)) return ZM_E_ARG;
            if (!aligned_to(tensors[3 * i + m], 16)) even[m == 2] = false;
            e.tensor[i][m] = static_cast<const uint16_t *>(tensors[3 * i + m]);
        }
    }
    if (workspace_bytes < need) return ZM_E_SIZE;
    Call c{};
    c.x = a->x, c.scales = static_cast<const uint8_t *>(a->scales), c.ids = a->ids, c.weights = a->weights;
    c.residual = static_cast<const uint16_t *>(a->residual), c.out = static_cast<uint16_t *>(a->out);
    c.x_stride = a->x_stride, c.scales_stride = a->scales_stride, c.residual_stride = a->residual_stride, c.out_stride = a->out_stride;
    c.n_tokens = static_cast<uint32_t>(a->n_tokens), c.top_k = static_cast<uint32_t>(a->top_k), c.hidden = static_cast<uint32_t>(a->hidden);
    c.intermediate = static_cast<uint32_t>(a->intermediate), c.n_pairs = c.n_tokens * c.top_k;
    place(c, static_cast<uint8_t *>(workspace), a->n_tokens, a->top_k, a->hidden, a->intermediate);
    hipStream_t st = static_cast<hipStream_t>(stream);
    void *with_ids[] = {&c, &ids}, *with_experts[] = {&c, &e};
    int status = ZM_OK;
    if (scaled && n_experts) {
        // once for all tiles that multiply them.  Tokens of 2048 values through 8 of 64 experts of 1024, us where each tile widens them itself / in
        // front: one token 35.2 / 32.0, 16 142 / 116, 64 250 / 220
        status = widen(c, st);
        if (status != ZM_OK) return status;
        c.x = c.wide_x, c.x_stride = c.wide_stride;
    }
    if (c.n_tokens <= kFewTokens && c.n_pairs <= kFewPairs) {
        const bool tight = even[0] && aligned_to(c.x, 16) && c.x_stride % 8 == 0;
        const Few few = tight ? (even[1] ? few_of<true, true>(c) : few_of<true, false>(c)) : (even[1] ? few_of<false, true>(c) : few_of<false, false>(c));
        const uint32_t chosen = c.n_pairs < e.n ? c.n_pairs : e.n, tiles = (c.intermediate + few.first_rows - 1) / few.first_rows * chosen;
        if (chosen) status = launch(few.first, dim3(tiles < kFewGrid ? tiles : kFewGrid), dim3(64 * kFirstWaves), with_experts, st);
        const uint32_t across = (c.hidden + few.second_rows - 1) / few.second_rows;
        const uint32_t parts = c.n_tokens > 8 && across < kUnits ? (kUnits / across < kFewParts ? kUnits / across : kFewParts) : 1;
        if (status == ZM_OK) status = launch(few.second, dim3(across, parts), dim3(64 * kSecondWaves), with_experts, st);
        if (status == ZM_OK && parts > 1) {
            uint32_t n = parts;
            void *joined[] = {&c, &n};
            status = launch(reinterpret_cast<const void *>(&zm_moe_few_join_kernel), dim3((c.hidden + 255) / 256, c.n_tokens), dim3(256), joined, st);
        }
        return status;
    }
    if (n_experts) {
        status = launch(reinterpret_cast<const void *>(&zm_moe_list_kernel), dim3(e.n), dim3(1024), with_ids, st);
        // a row's requests name it by 32 bits
        const bool direct = even[0] && aligned_to(c.x, 16) && c.x_stride % 8 == 0 &&
                            (static_cast<uint64_t>(c.n_tokens) * static_cast<uint64_t>(c.x_stride) + c.hidden) < (1ull << 31);
        const uint64_t groups = c.n_pairs < e.n ? c.n_pairs : e.n;
        const bool wide = direct && even[1] && c.hidden % kWideDeep == 0 && c.intermediate % kWideDeep == 0 && c.n_pairs >= kWideFrom * e.n;
        const uint64_t tiles = c.n_pairs / (wide ? kWidePairs : kPairs) + groups;
        // rows of a tile: of gate and up together, of down
        const uint32_t tall = direct ? kRows : kRows / 2, tall_down = even[1] ? kRows : kRows / 2;
        const uint64_t first = (c.intermediate + tall / 2 - 1) / (tall / 2) * tiles, second = (c.hidden + tall_down - 1) / tall_down * tiles;
        const void *const fn[2] = {
            wide ? reinterpret_cast<const void *>(&zm_moe_wide_kernel<true>)
                 : direct ? reinterpret_cast<const void *>(&zm_moe_product_kernel<true, true>) : reinterpret_cast<const void *>(&zm_moe_product_kernel<true, false>),
            wide ? reinterpret_cast<const void *>(&zm_moe_wide_kernel<false>)
                 : even[1] ? reinterpret_cast<const void *>(&zm_moe_product_kernel<false, true>) : reinterpret_cast<const void *>(&zm_moe_product_kernel<false, false>)};
        const dim3 block(wide ? 512 : 256);
        if (status == ZM_OK) status = launch(fn[0], dim3(static_cast<uint32_t>((first + 7) / 8 * 8)), block, with_experts, st);
        if (status == ZM_OK) status = launch(fn[1], dim3(static_cast<uint32_t>((second + 7) / 8 * 8)), block, with_experts, st);
    }
    // rows of the grid's y axis are 16 bits wide
    for (uint32_t done = 0; status == ZM_OK && done < c.n_tokens; done += 65535u) {
        Call part = c;
        part.ids += static_cast<uint64_t>(done) * c.top_k, part.weights += static_cast<uint64_t>(done) * c.top_k;
        part.y += static_cast<uint64_t>(done) * c.top_k * c.hidden, part.out += done * c.out_stride;
        if (c.residual) part.residual += done * c.residual_stride;
        with_ids[0] = &part;
        status = launch(reinterpret_cast<const void *>(&zm_moe_join_kernel), dim3((c.hidden + 1023) / 1024, c.n_tokens - done < 65535u ? c.n_tokens - done : 65535u), dim3(256), with_ids, st);
    }
    return status;
}

}  // extern "C"
