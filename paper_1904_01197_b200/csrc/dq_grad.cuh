// Gradients of many tensors: the global norm over a list of tensors, and one pass that multiplies every element by the
// clipping factor on its way into another list (or into place).
//
//   N = sqrt(sum_t sum_i x_ti^2)  or  max |x_ti|;   c = 1 if N <= limit, else limit / N;   y_ti = round(c x_ti)
//
// Both are bound by memory (one or two operations per element), and short lists by launches.  The tensors of a launch
// travel in its parameters: no table has to be uploaded, a call can be captured, and nothing outlives it.
//
// A tensor is cut into tiles of 1024 * 2^k elements, one warp works on one tile at a time, and a CTA owns a contiguous
// run of the launch's tiles, so that it meets few tensors.  Within a tile a lane owns groups of 8 consecutive
// elements, four of them in flight (16-byte loads and stores).  Tiles are counted from an aligned address at or before
// the tensor's first element (`phase` elements before it), of the destination where there is one; a source that is not
// aligned there is read in aligned 16-byte pieces that are shifted into place, which keeps both sides at full width
// whatever the offset between them.
//
// L2 sums run in fp64: an fp32 sum of 10^8 squares loses digits, and squares of fp32 values leave the fp32 range at
// both ends.  Maxima are maxima of the bit patterns without the sign, where a NaN is above every number.  No atomics
// are involved: the order of a sum depends on the sizes and the device only, not on timing.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dq_device.cuh"

namespace dq {

constexpr int kGradThreads = 256;
constexpr uint32_t kGradWarps = kGradThreads / 32;
constexpr uint32_t kGradBatch = 4;                           // groups of a lane in flight
constexpr uint32_t kGradTileLog2 = 10;                       // 32 lanes * 8 elements * kGradBatch
constexpr int kGradClusterThreads = 512;
constexpr int kGradCluster = 16;                             // 8 where a cluster of 16 cannot be resident

constexpr uint32_t kWarnNonfiniteNorm = 0x8u;      // DQ_WARN_NONFINITE_NORM

enum GradType : uint32_t { kGradF32 = 0, kGradBF16 = 1, kGradF16 = 2 };

// How a tensor is walked.  Flat: contiguous on both sides.  Rows: rows of contiguous elements at a fixed distance, every
// row a multiple of 8 elements that starts at a 16-byte boundary.  Loose: rows of any other kind, element by element.
enum GradWalk : uint32_t { kGradFlat = 0, kGradRows = 1, kGradLoose = 2 };

struct GradEntry {
    const void* src;
    uint64_t n;
    uint32_t row, src_stride;        // rows: elements per row, and from one row to the next
    uint32_t form;                   // src type | dst type << 2 | walk << 4 | phase << 8 | byte shift of the source << 12
    uint32_t dst_stride;
    void* dst;
};

__host__ __device__ __forceinline__ uint32_t grad_form(uint32_t src_type, uint32_t dst_type, uint32_t walk, uint32_t phase,
                                                       uint32_t shift)
{
    return src_type | dst_type << 2 | walk << 4 | phase << 8 | shift << 12;
}

// first_tile[count] is the launch's number of tiles.
template <int N>
struct GradTable {
    static constexpr int kCapacity = N;
    uint32_t count, tile_log2;
    uint32_t first_tile[N + 1];
    GradEntry e[N];
};

// ------------------------------------------------------------------------------------------ values of a group
__device__ __forceinline__ void widen_bf16(const uint32_t (&w)[4], float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

__device__ __forceinline__ void widen_f16(const uint32_t (&w)[4], float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

__device__ __forceinline__ float load_element(const void* p, uint64_t i, uint32_t type)
{
    if (type == kGradF32) return static_cast<const float*>(p)[i];
    const uint16_t h = static_cast<const uint16_t*>(p)[i];
    return type == kGradBF16 ? __uint_as_float((uint32_t)h << 16) : __half2float(__ushort_as_half(h));
}

// One rounding, of the product in fp32 to the destination's type (to nearest, ties to even).
__device__ __forceinline__ void store_element(void* p, uint64_t i, uint32_t type, float x)
{
    if (type == kGradF32)
        static_cast<float*>(p)[i] = x;
    else if (type == kGradBF16)
        static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
    else
        static_cast<__half*>(p)[i] = __float2half_rn(x);
}

// W words that start `shift` bytes into the P pieces at q: word moves by the shift's two upper bits, half a word by the
// next (16-bit elements only).
template <int P, int W, bool HALF>
__device__ __forceinline__ void shifted_words(const uint4 (&q)[P], uint32_t shift, uint32_t (&out)[W])
{
    uint32_t w[4 * P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        w[4 * i] = q[i].x;
        w[4 * i + 1] = q[i].y;
        w[4 * i + 2] = q[i].z;
        w[4 * i + 3] = q[i].w;
    }
    if (shift & 8u) {
#pragma unroll
        for (int i = 0; i + 2 < 4 * P; ++i) w[i] = w[i + 2];
    }
    if (shift & 4u) {
#pragma unroll
        for (int i = 0; i + 1 < 4 * P; ++i) w[i] = w[i + 1];
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        out[i] = w[i];
        if constexpr (HALF) {
            if (shift & 2u) out[i] = __funnelshift_r(w[i], w[i + 1], 16);
        }
    }
}

// ------------------------------------------------------------------------------------------ a warp's place in the table
// The tensor that owns tile `tile`: the last one whose first tile is at or before it.  The lanes look at 32 places at
// once, since every line of the parameters is a cache miss that a short kernel waits for.
template <class Table>
__device__ __forceinline__ uint32_t find_tensor(const Table& t, uint32_t tile)
{
    const uint32_t lane = threadIdx.x & 31u;
    uint32_t block = 0u;
    if constexpr (Table::kCapacity > 32) {
        static_assert(Table::kCapacity <= 1024, "two steps of 32");
        const uint32_t i = lane * 32u;
        block = 32u * (__popc(__ballot_sync(0xFFFFFFFFu, i < t.count && t.first_tile[i < t.count ? i : 0u] <= tile)) - 1u);
    }
    const uint32_t i = block + lane;
    return block + __popc(__ballot_sync(0xFFFFFFFFu, i < t.count && t.first_tile[i < t.count ? i : 0u] <= tile)) - 1u;
}

// A tile's place in its tensor.
struct TileSpan {
    uint64_t start;              // of the tile, in elements from the aligned origin
    uint32_t lo, hi;             // the tensor's elements in the tile: [lo, hi) from the tile's start
};

__device__ __forceinline__ TileSpan tile_span(const GradEntry& e, uint32_t index, uint32_t tile_log2)
{
    const uint32_t phase = (e.form >> 8) & 15u;
    TileSpan s;
    s.start = (uint64_t)index << tile_log2;
    s.lo = s.start < phase ? phase - (uint32_t)s.start : 0u;
    const uint64_t left = e.n + phase - s.start;
    s.hi = left < (1ull << tile_log2) ? (uint32_t)left : 1u << tile_log2;
    return s;
}

// Element offsets of a row-wise tensor: the tile's first element is (row r0, column c0).
struct RowPlace {
    uint64_t r0;
    uint32_t c0;
};

__device__ __forceinline__ RowPlace row_place(const GradEntry& e, const TileSpan& s)
{
    RowPlace p;
    p.r0 = s.start / e.row;
    p.c0 = (uint32_t)(s.start - p.r0 * e.row);
    return p;
}

__device__ __forceinline__ void row_offset(const RowPlace& p, uint32_t rel, uint32_t row, uint64_t& r, uint32_t& c)
{
    const uint32_t v = p.c0 + rel, q = v / row;          // (c0 < row < 2^31, rel < 2^31)
    r = p.r0 + q;
    c = v - q * row;
}

// The values of a lane's kGradBatch groups at `rel` (from the tile's start) + 256 j + 8 lane; loose tensors: at rel + 256 j
// + 32 i + lane.  Elements outside the tensor are 0, and so are the groups that only lie partly inside, or so near an
// end that an aligned piece of a shifted source would reach past it: those are left to the caller, element by element.
struct Batch {
    float x[kGradBatch][8];
    uint32_t whole;              // bit j: group j was loaded
};

__device__ __forceinline__ void load_batch(const GradEntry& e, const TileSpan& s, const RowPlace& place, uint32_t rel, Batch& b)
{
    const uint32_t lane = threadIdx.x & 31u;
    const uint32_t type = e.form & 3u, walk = (e.form >> 4) & 3u, shift = (e.form >> 12) & 15u;
    b.whole = 0u;
    if (walk == kGradLoose) {
#pragma unroll
        for (uint32_t j = 0; j < kGradBatch; ++j) {
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                const uint32_t v = rel + 256u * j + 32u * i + lane;
                b.x[j][i] = 0.0f;
                if (v >= s.lo && v < s.hi) {
                    uint64_t r;
                    uint32_t c;
                    row_offset(place, v, e.row, r, c);
                    b.x[j][i] = load_element(e.src, r * e.src_stride + c, type);
                }
            }
        }
        return;
    }
    // byte address of the group's first element, and of the aligned piece that holds it
    const uint32_t size = type == kGradF32 ? 4u : 2u;
    const char* p[kGradBatch];
    const uint32_t margin = shift ? 8u : 0u;
#pragma unroll
    for (uint32_t j = 0; j < kGradBatch; ++j) {
        const uint32_t v = rel + 256u * j + 8u * lane;
        if (v >= s.lo && v + 8u <= s.hi) {
            // (the margin is counted from the ends of the tensor, not of the tile)
            const uint64_t at = s.start + v, phase = (e.form >> 8) & 15u;
            if (!margin || (at >= phase + margin && at + 8u + margin <= phase + e.n)) b.whole |= 1u << j;
        }
        if (walk == kGradRows) {
            uint64_t r;
            uint32_t c;
            row_offset(place, v, e.row, r, c);
            p[j] = static_cast<const char*>(e.src) + (r * e.src_stride + c) * size;
        } else {
            p[j] = static_cast<const char*>(e.src) - (uint64_t)((e.form >> 8) & 15u) * size - shift + (s.start + v) * size;
        }
    }
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    if (type == kGradF32) {
        if (shift == 0u) {
            uint4 q[kGradBatch][2];
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) {
                const uint4* a = reinterpret_cast<const uint4*>(p[j]);
                const bool in = b.whole >> j & 1u;
                q[j][0] = in ? a[0] : zero;
                q[j][1] = in ? a[1] : zero;
            }
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    b.x[j][4 * h] = __uint_as_float(q[j][h].x);
                    b.x[j][4 * h + 1] = __uint_as_float(q[j][h].y);
                    b.x[j][4 * h + 2] = __uint_as_float(q[j][h].z);
                    b.x[j][4 * h + 3] = __uint_as_float(q[j][h].w);
                }
            }
        } else {
            uint4 q[kGradBatch][3];
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) {
                const uint4* a = reinterpret_cast<const uint4*>(p[j]);
                const bool in = b.whole >> j & 1u;
                q[j][0] = in ? a[0] : zero;
                q[j][1] = in ? a[1] : zero;
                q[j][2] = in ? a[2] : zero;
            }
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) {
                uint32_t w[8];
                shifted_words<3, 8, false>(q[j], shift, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) b.x[j][i] = __uint_as_float(w[i]);
            }
        }
    } else {
        uint32_t w[kGradBatch][4];
        if (shift == 0u) {
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) {
                const uint4 q = (b.whole >> j & 1u) ? *reinterpret_cast<const uint4*>(p[j]) : zero;
                w[j][0] = q.x;
                w[j][1] = q.y;
                w[j][2] = q.z;
                w[j][3] = q.w;
            }
        } else {
            uint4 q[kGradBatch][2];
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) {
                const uint4* a = reinterpret_cast<const uint4*>(p[j]);
                const bool in = b.whole >> j & 1u;
                q[j][0] = in ? a[0] : zero;
                q[j][1] = in ? a[1] : zero;
            }
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) shifted_words<2, 4, true>(q[j], shift, w[j]);
        }
        if (type == kGradBF16) {
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) widen_bf16(w[j], b.x[j]);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) widen_f16(w[j], b.x[j]);
        }
    }
}

// ------------------------------------------------------------------------------------------ norm
// A lane's part of a norm: the sum of squares in fp64, or the largest bit pattern without the sign.
template <bool MAX> struct NormPart;

template <> struct NormPart<false> {
    double s;
    __device__ __forceinline__ void add(float x)
    {
        const double d = (double)x;
        s = __fma_rn(d, d, s);
    }
    __device__ __forceinline__ void join(const NormPart& o) { s = __dadd_rn(s, o.s); }
    __device__ __forceinline__ NormPart other(int lane_mask) const
    {
        NormPart o;
        o.s = __shfl_xor_sync(0xFFFFFFFFu, s, lane_mask);
        return o;
    }
    __device__ __forceinline__ float norm() const { return __double2float_rn(__dsqrt_rn(s)); }
};

template <> struct NormPart<true> {
    uint64_t s;
    __device__ __forceinline__ void add(float x)
    {
        const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
        s = max((uint32_t)s, u);
    }
    __device__ __forceinline__ void join(const NormPart& o) { s = max((uint32_t)s, (uint32_t)o.s); }
    __device__ __forceinline__ NormPart other(int lane_mask) const
    {
        NormPart o;
        o.s = __shfl_xor_sync(0xFFFFFFFFu, (uint32_t)s, lane_mask);
        return o;
    }
    __device__ __forceinline__ float norm() const { return __uint_as_float((uint32_t)s); }
};

template <bool MAX>
__device__ __forceinline__ void reduce_warp(NormPart<MAX>& a)
{
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) a.join(a.other(m));
}

// Every thread has a part; thread 0 gets the whole.  `parts`: one per warp.
template <bool MAX>
__device__ __forceinline__ void reduce_block(NormPart<MAX>& a, NormPart<MAX>* parts, uint32_t warps)
{
    reduce_warp(a);
    if ((threadIdx.x & 31u) == 0u) parts[threadIdx.x >> 5] = a;
    __syncthreads();
    if (threadIdx.x < 32u) {
        NormPart<MAX> b = {};
        if (threadIdx.x < warps) b = parts[threadIdx.x];
        reduce_warp(b);
        a = b;
    }
}

// Adds one tile of a tensor to a lane's part.
template <bool MAX>
__device__ __forceinline__ void norm_tile(const GradEntry& e, uint32_t index, uint32_t tile_log2, NormPart<MAX>& acc)
{
    const TileSpan s = tile_span(e, index, tile_log2);
    const uint32_t walk = (e.form >> 4) & 3u;
    RowPlace place = {0u, 0u};
    if (walk != kGradFlat) place = row_place(e, s);
    for (uint32_t rel = 0u; rel < s.hi; rel += 1u << kGradTileLog2) {
        Batch b;
        load_batch(e, s, place, rel, b);
#pragma unroll
        for (uint32_t j = 0; j < kGradBatch; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) acc.add(b.x[j][i]);
        }
        if (walk == kGradLoose) continue;
        const uint32_t type = e.form & 3u, phase = (e.form >> 8) & 15u;
#pragma unroll 1
        for (uint32_t j = 0; j < kGradBatch; ++j) {
            const uint32_t v = rel + 256u * j + 8u * (threadIdx.x & 31u);
            if ((b.whole >> j & 1u) || v + 8u <= s.lo || v >= s.hi) continue;
#pragma unroll 1
            for (uint32_t i = max(v, s.lo); i < min(v + 8u, s.hi); ++i) acc.add(load_element(e.src, s.start + i - phase, type));
        }
    }
}

// Writes the norm and reports one that is no finite number.
__device__ __forceinline__ void publish_norm(float norm, float* out_norm, uint32_t* status)
{
    if (out_norm) *out_norm = norm;
    if (status && !(fabsf(norm) <= 3.402823466e38f)) atomicOr(status, kWarnNonfiniteNorm);
}

// A part of the norm per CTA (slots[blockIdx]), or with EACH per tile (slots[tile]).
template <class Table, bool MAX, bool EACH>
__global__ void __launch_bounds__(kGradThreads)
grad_norm_kernel(const __grid_constant__ Table t, NormPart<MAX>* slots)
{
    __shared__ NormPart<MAX> parts[kGradWarps];
    grid_dependency_wait();
    grid_dependency_launch_next();
    const uint32_t tiles = t.first_tile[t.count];
    const uint32_t begin = (uint32_t)((uint64_t)tiles * blockIdx.x / gridDim.x);
    const uint32_t end = (uint32_t)((uint64_t)tiles * (blockIdx.x + 1u) / gridDim.x);
    NormPart<MAX> acc = {};
    for (uint32_t tile = begin + (threadIdx.x >> 5); tile < end; tile += kGradWarps) {
        const uint32_t k = find_tensor(t, tile);
        norm_tile<MAX>(t.e[k], tile - t.first_tile[k], t.tile_log2, acc);
        if constexpr (EACH) {
            reduce_warp(acc);
            if ((threadIdx.x & 31u) == 0u) slots[tile] = acc;
            acc = {};
        }
    }
    if constexpr (!EACH) {
        reduce_block(acc, parts, kGradWarps);
        if (threadIdx.x == 0u) slots[blockIdx.x] = acc;
    }
}

// The whole from the slots of all launches before it.
constexpr int kGradJoinThreads = 1024;

template <bool MAX>
__global__ void __launch_bounds__(kGradJoinThreads)
grad_norm_join_kernel(const NormPart<MAX>* slots, uint32_t num_slots, float* out_norm, uint32_t* status)
{
    __shared__ NormPart<MAX> parts[kGradJoinThreads / 32];
    grid_dependency_wait();
    grid_dependency_launch_next();
    NormPart<MAX> acc = {};
    for (uint32_t i = threadIdx.x; i < num_slots; i += kGradJoinThreads) acc.join(slots[i]);
    reduce_block(acc, parts, kGradJoinThreads / 32);
    if (threadIdx.x == 0u) publish_norm(acc.norm(), out_norm, status);
}

// The norms of single tensors from the slots of their tiles; tensor i of the launch owns the slots [first[i], first[i + 1]).
constexpr int kGradEachCapacity = 8000;

struct GradEachTable {
    uint32_t count;
    uint32_t first[kGradEachCapacity + 1];
};

template <bool MAX>
__global__ void __launch_bounds__(kGradThreads)
grad_norms_each_kernel(const __grid_constant__ GradEachTable t, const NormPart<MAX>* slots, float* out_norms)
{
    grid_dependency_wait();
    grid_dependency_launch_next();
    const uint32_t i = blockIdx.x * kGradWarps + (threadIdx.x >> 5);
    if (i >= t.count) return;
    NormPart<MAX> acc = {};
    for (uint32_t k = t.first[i] + (threadIdx.x & 31u); k < t.first[i + 1u]; k += 32u) acc.join(slots[k]);
    reduce_warp(acc);
    if ((threadIdx.x & 31u) == 0u) out_norms[i] = acc.norm();
}

// ------------------------------------------------------------------------------------------ clipping
// What the elements are multiplied by.
struct ClipArgs {
    float max_norm;
    uint32_t num_slots;          // parts of the norm; 0: it is at `norm`, or nothing is clipped (`norm` null)
    const void* slots;
    const float* norm;
    float* out_norm;             // optional
    uint32_t* status;            // optional
    uint32_t in_place;
};

__device__ __forceinline__ float clip_factor(float norm, float max_norm)
{
    return norm <= max_norm ? 1.0f : __fdiv_rn(max_norm, norm);
}

// Multiplies one tile by c into the destination.
__device__ __forceinline__ void scale_tile(const GradEntry& e, uint32_t index, uint32_t tile_log2, float c)
{
    const TileSpan s = tile_span(e, index, tile_log2);
    const uint32_t walk = (e.form >> 4) & 3u, type = (e.form >> 2) & 3u;
    const uint32_t lane = threadIdx.x & 31u;
    RowPlace place = {0u, 0u};
    if (walk != kGradFlat) place = row_place(e, s);
    for (uint32_t rel = 0u; rel < s.hi; rel += 1u << kGradTileLog2) {
        Batch b;
        load_batch(e, s, place, rel, b);
#pragma unroll
        for (uint32_t j = 0; j < kGradBatch; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) b.x[j][i] = __fmul_rn(b.x[j][i], c);
        }
        if (walk == kGradLoose) {
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) {
#pragma unroll
                for (uint32_t i = 0; i < 8u; ++i) {
                    const uint32_t v = rel + 256u * j + 32u * i + lane;
                    if (v >= s.lo && v < s.hi) {
                        uint64_t r;
                        uint32_t col;
                        row_offset(place, v, e.row, r, col);
                        store_element(e.dst, r * e.dst_stride + col, type, b.x[j][i]);
                    }
                }
            }
            continue;
        }
        const uint32_t size = type == kGradF32 ? 4u : 2u, phase = (e.form >> 8) & 15u;
        char* p[kGradBatch];
#pragma unroll
        for (uint32_t j = 0; j < kGradBatch; ++j) {
            const uint32_t v = rel + 256u * j + 8u * lane;
            uint64_t at = s.start + v - phase;
            if (walk == kGradRows) {
                uint64_t r;
                uint32_t col;
                row_offset(place, v, e.row, r, col);
                at = r * e.dst_stride + col;
            }
            p[j] = static_cast<char*>(e.dst) + at * size;
        }
        if (type == kGradF32) {
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) {
                if (b.whole >> j & 1u) {
                    float4* a = reinterpret_cast<float4*>(p[j]);
                    a[0] = make_float4(b.x[j][0], b.x[j][1], b.x[j][2], b.x[j][3]);
                    a[1] = make_float4(b.x[j][4], b.x[j][5], b.x[j][6], b.x[j][7]);
                }
            }
        } else {
#pragma unroll
            for (uint32_t j = 0; j < kGradBatch; ++j) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (type == kGradBF16) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(b.x[j][2 * i], b.x[j][2 * i + 1]);
                        w[i] = *reinterpret_cast<const uint32_t*>(&h);
                    } else {
                        const __half2 h = __floats2half2_rn(b.x[j][2 * i], b.x[j][2 * i + 1]);
                        w[i] = *reinterpret_cast<const uint32_t*>(&h);
                    }
                }
                if (b.whole >> j & 1u) *reinterpret_cast<uint4*>(p[j]) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
#pragma unroll 1
        for (uint32_t j = 0; j < kGradBatch; ++j) {
            const uint32_t v = rel + 256u * j + 8u * lane;
            if ((b.whole >> j & 1u) || v + 8u <= s.lo || v >= s.hi) continue;
#pragma unroll 1
            for (uint32_t i = max(v, s.lo); i < min(v + 8u, s.hi); ++i) {
                const uint64_t at = s.start + i - phase;
                store_element(e.dst, at, type, __fmul_rn(load_element(e.src, at, e.form & 3u), c));
            }
        }
    }
}

// The last tiles first: they are what the norm's pass has left in L2.
template <class Table, bool MAX>
__global__ void __launch_bounds__(kGradThreads)
grad_scale_kernel(const __grid_constant__ Table t, const __grid_constant__ ClipArgs a)
{
    __shared__ NormPart<MAX> parts[kGradWarps];
    __shared__ float factor;
    grid_dependency_wait();
    float c = 1.0f;
    if (a.num_slots) {
        NormPart<MAX> acc = {};
        for (uint32_t i = threadIdx.x; i < a.num_slots; i += kGradThreads)
            acc.join(static_cast<const NormPart<MAX>*>(a.slots)[i]);
        reduce_block(acc, parts, kGradWarps);
        if (threadIdx.x == 0u) {
            const float norm = acc.norm();
            factor = clip_factor(norm, a.max_norm);
            if (blockIdx.x == 0u) publish_norm(norm, a.out_norm, a.status);
        }
        __syncthreads();
        c = factor;
    } else if (a.norm) {
        const float norm = *a.norm;
        c = clip_factor(norm, a.max_norm);
        if (blockIdx.x == 0u && threadIdx.x == 0u) publish_norm(norm, a.out_norm, a.status);
    }
    grid_dependency_launch_next();
    if (a.in_place && c == 1.0f) return;
    const uint32_t tiles = t.first_tile[t.count], cta = gridDim.x - 1u - blockIdx.x;
    const uint32_t begin = (uint32_t)((uint64_t)tiles * cta / gridDim.x);
    const uint32_t end = (uint32_t)((uint64_t)tiles * (cta + 1u) / gridDim.x);
    for (uint32_t tile = begin + (threadIdx.x >> 5); tile < end; tile += kGradWarps) {
        const uint32_t k = find_tensor(t, tile);
        scale_tile(t.e[k], tile - t.first_tile[k], t.tile_log2, c);
    }
}

// ------------------------------------------------------------------------------------------ short lists
// Norm and clipping of a short list in one launch: a cluster of CTAs whose parts of the norm meet over distributed
// shared memory.  SCALE: multiplies as well.  Two launches that wait for one another cost more than the work.
template <class Table, bool MAX, bool SCALE>
__global__ void __launch_bounds__(kGradClusterThreads)
grad_cluster_kernel(const __grid_constant__ Table t, const __grid_constant__ ClipArgs a)
{
    constexpr uint32_t kWarps = kGradClusterThreads / 32;
    __shared__ NormPart<MAX> parts[kWarps];
    __shared__ NormPart<MAX> mine;
    __shared__ float factor;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const uint32_t tiles = t.first_tile[t.count], step = gridDim.x * kWarps;
    const uint32_t first = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;
    NormPart<MAX> acc = {};
    for (uint32_t tile = first; tile < tiles; tile += step) {
        const uint32_t k = find_tensor(t, tile);
        norm_tile<MAX>(t.e[k], tile - t.first_tile[k], t.tile_log2, acc);
    }
    reduce_block(acc, parts, kWarps);
    if (threadIdx.x == 0u) mine = acc;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (threadIdx.x < 32u) {
        NormPart<MAX> all = {};
        if (threadIdx.x < gridDim.x) {
            uint32_t remote;
            uint64_t v;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(&mine)), "r"(threadIdx.x));
            asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(remote) : "memory");
            static_assert(sizeof(NormPart<MAX>) == sizeof(v), "a part is 64 bits");
            memcpy(&all, &v, sizeof(v));
        }
        reduce_warp(all);
        if (threadIdx.x == 0u) {
            const float norm = all.norm();
            factor = SCALE ? clip_factor(norm, a.max_norm) : 1.0f;
            if (blockIdx.x == 0u) publish_norm(norm, a.out_norm, a.status);
        }
    }
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");     // (no CTA leaves while its part is read)
    if constexpr (SCALE) {
        const float c = factor;
        if (!(a.in_place && c == 1.0f)) {
            for (uint32_t tile = first; tile < tiles; tile += step) {
                const uint32_t k = find_tensor(t, tile);
                scale_tile(t.e[k], tile - t.first_tile[k], t.tile_log2, c);
            }
        }
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

}  // namespace dq
