// Gradients of many tensors: the global norm over a list of tensors, and one pass that multiplies every element by the
// clipping factor on its way into another list (or into place).
//
//   N = sqrt(sum_t sum_i x_ti^2)  or  max |x_ti|;   c = 1 if N <= limit, else limit / N;   y_ti = round(c x_ti)
//
// Both are bound by memory (one or two operations per element), and short lists by launches.  The tensors of a launch
// travel in its parameters: no table has to be uploaded, a call can be captured, and nothing outlives it.
//
// A tensor is cut into tiles, and one warp works on a tile at a time.  The warps of a launch take consecutive tiles, so that
// what is in flight at one time lies close together.  Within a tile a lane keeps eight 16-byte loads in flight (the elements of
// a 16-bit side, where the other is fp32, in 8 bytes), and a warp's loads and stores are contiguous.  Tiles are counted from an
// aligned address at or before the tensor's first element (`phase` elements before it), of the destination where there is
// one; a source that is not aligned there is read in its own aligned pieces, which are shifted into place between neighbouring
// lanes, so that both sides keep their width whatever the offset between them.
//
// L2 sums run in fp64: an fp32 sum of 10^8 squares loses digits, and squares of fp32 values leave the fp32 range at
// both ends.  Maxima are maxima of the bit patterns without the sign, where a NaN is above every number.  No atomics
// are involved: the order of a sum does not depend on timing.  It does depend on how a call cuts its tensors up, that is on the
// sizes, types, strides and addresses modulo 16 bytes (of the destination too, where one launch does all), on which call it is
// and on the device: the same values elsewhere may have a norm that is one fp32 step away.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dq_device.cuh"

namespace dq {

constexpr int kGradThreads = 256;
constexpr int kGradNormCtas = 4, kGradScaleCtas = 3;         // resident CTAs per SM: 64 and 80 registers
constexpr uint32_t kGradWarps = kGradThreads / 32;
constexpr uint32_t kGradTileStep = 1024;                     // a warp's batch of 8 loads of 16 bytes per lane, in fp32
constexpr int kGradClusterThreads = 512;
constexpr int kGradCluster = 16;                             // 8 where a cluster of 16 cannot be resident

constexpr uint32_t kWarnNonfiniteNorm = 0x8u;      // DQ_WARN_NONFINITE_NORM

enum GradType : uint32_t { kGradF32 = 0, kGradBF16 = 1, kGradF16 = 2 };

// How a tensor is walked.  Flat: contiguous on both sides.  Of tensors in rows, Wide: in 16-byte pieces across the rows, which
// are multiples of 8 elements and start at 16-byte boundaries.  Long: rows of another kind, each like a contiguous tensor of
// its own.  Loose: element by element, where those are short.
enum GradWalk : uint32_t { kGradFlat = 0, kGradLong = 1, kGradWide = 2, kGradLoose = 3 };

// Tiles of a Long tensor: parts of a row, of nearly equal length, where a row does not fit a tile whatever its alignment,
// else several whole rows.
struct GradRowTiles {
    uint32_t per_row, rows;      // tiles per row, rows per tile: one of them is 1
    uint32_t len;                // of a part

    __host__ __device__ __forceinline__ GradRowTiles(uint32_t row, uint32_t tile_len)
        : per_row((row + 7u + tile_len - 1u) / tile_len), rows(per_row > 1u ? 1u : tile_len / row),
          len((row + 7u + 8u * per_row - 1u) / (8u * per_row) * 8u)
    {
    }
    __host__ __device__ __forceinline__ uint64_t tiles(uint64_t all_rows) const
    {
        return per_row > 1u ? all_rows * per_row : (all_rows + rows - 1u) / rows;
    }
};

// A tensor in a launch's table, in as few words as hold it: addresses have at most 57 bits, lengths 34.
//   w[0], low 25 bits of w[1]   address of the source        w[1] 25..26 type, 27..28 walk, 29..30 upper bits of n
//   w[2]                        lower bits of n
//   w[3], low 25 bits of w[4]   address of the destination   w[4] 25..26 type                      (where there is one)
// A tensor in rows takes the next entry too, which owns no tiles: w[0] elements per row, w[1] from one row of the source to
// the next, w[2] of the destination.
template <int W>
struct GradEntry {
    uint32_t w[W];
};

// first_tile[count] is the launch's number of tiles.  The tiles below stream_below are not wanted in L2 for long; rows: a
// tensor of the table lies in rows.
template <int N, int W>
struct GradTable {
    static constexpr int kCapacity = N, kWords = W;
    uint32_t count, tile_len, stream_below, rows;
    uint32_t first_tile[N + 1];
    GradEntry<W> e[N];
};

// ... unpacked.
struct GradTensor {
    const char* src;
    char* dst;
    uint64_t n;
    uint32_t src_type, dst_type, walk;
    uint32_t row, src_stride, dst_stride;
};

template <bool ROWS, class Table>
__device__ __forceinline__ GradTensor tensor_at(const Table& t, uint32_t k)
{
    GradTensor g;
    const uint32_t w1 = t.e[k].w[1];
    g.src = reinterpret_cast<const char*>((uint64_t)(w1 & 0x1FFFFFFu) << 32 | t.e[k].w[0]);
    g.src_type = w1 >> 25 & 3u;
    g.walk = w1 >> 27 & 3u;
    g.n = (uint64_t)(w1 >> 29 & 3u) << 32 | t.e[k].w[2];
    g.dst = nullptr;
    g.dst_type = 0u;
    if constexpr (Table::kWords > 3) {
        const uint32_t w4 = t.e[k].w[4];
        g.dst = reinterpret_cast<char*>((uint64_t)(w4 & 0x1FFFFFFu) << 32 | t.e[k].w[3]);
        g.dst_type = w4 >> 25 & 3u;
    }
    g.row = g.src_stride = g.dst_stride = 0u;
    if (ROWS && g.walk != kGradFlat) {
        g.row = t.e[k + 1u].w[0];
        g.src_stride = t.e[k + 1u].w[1];
        g.dst_stride = t.e[k + 1u].w[2];
    }
    return g;
}

// ------------------------------------------------------------------------------------------ a warp's place in the table
// The tensor that owns tile `tile`: the last one whose first tile is at or before it.  The lanes look at 32 places at
// once, since every line of the parameters is a cache miss that a short kernel waits for.
template <class Table>
__device__ __forceinline__ uint32_t find_tensor(const Table& t, uint32_t tile)
{
    const uint32_t lane = threadIdx.x & 31u;
    auto at_or_before = [&](uint32_t i) {
        const bool in = i < t.count;
        return (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, in && t.first_tile[in ? i : 0u] <= tile));
    };
    if constexpr (Table::kCapacity <= 32) {
        return at_or_before(lane) - 1u;
    } else {
        constexpr uint32_t kStep = (Table::kCapacity + 1023) / 1024 * 32;
        const uint32_t block = kStep * (at_or_before(lane * kStep) - 1u);
        uint32_t k = block - 1u;
#pragma unroll
        for (uint32_t i = 0u; i < kStep; i += 32u) k += at_or_before(block + i + lane);
        return k;
    }
}

// A warp's current tensor.
struct TensorRun {
    GradTensor g;
    uint32_t first, end;         // its tiles

    // Before the wait for the previous kernel: the parameters' cache misses pass in its shadow.
    template <bool ROWS, class Table>
    __device__ __forceinline__ void start(const Table& t, uint32_t tile, uint32_t tiles)
    {
        first = end = 0u;
        if (tile < tiles) seek<ROWS>(t, tile);
    }

    template <bool ROWS, class Table>
    __device__ __forceinline__ void seek(const Table& t, uint32_t tile)
    {
        const uint32_t k = find_tensor(t, tile);
        g = tensor_at<ROWS>(t, k);
        first = t.first_tile[k];
        end = t.first_tile[k + 1u];
    }
};

// How many elements before the first one a contiguous tensor's tiles begin: where the destination is aligned, or the
// source where there is none.  (The host counts tiles by the same rule.)
__device__ __forceinline__ uint32_t tile_phase(const GradTensor& g)
{
    const uint32_t size = (g.dst ? g.dst_type : g.src_type) == kGradF32 ? 4u : 2u;
    return (uint32_t)(reinterpret_cast<uintptr_t>(g.dst ? g.dst : g.src) / size) % (16u / size);
}

// Calls work(piece, tile, tile_len) for what a tile covers.  Pieces are contiguous tensors, a row each, or the tensor itself
// (which is contiguous unless ROWS).
template <bool ROWS, class Work>
__device__ __forceinline__ void for_pieces(const GradTensor& g, uint32_t tile, uint32_t tile_len, Work&& work)
{
    if constexpr (!ROWS) {
        work(g, tile, tile_len);
    } else {
        GradTensor p = g;
        uint32_t rows = 1u;
        if (g.walk == kGradLong) {
            const GradRowTiles t(g.row, tile_len);
            const uint32_t q = tile / t.per_row;
            const uint64_t r = (uint64_t)q * t.rows;
            tile -= q * t.per_row;
            tile_len = t.per_row > 1u ? t.len : tile_len;
            rows = (uint32_t)min((uint64_t)t.rows, g.n / g.row - r);
            p.src += r * g.src_stride * (g.src_type == kGradF32 ? 4u : 2u);
            if (g.dst) p.dst += r * g.dst_stride * (g.dst_type == kGradF32 ? 4u : 2u);
            p.n = g.row;
        }
#pragma unroll 1
        for (;;) {
            work(p, tile, tile_len);
            if (--rows == 0u) break;
            p.src += (uint64_t)g.src_stride * (g.src_type == kGradF32 ? 4u : 2u);
            if (g.dst) p.dst += (uint64_t)g.dst_stride * (g.dst_type == kGradF32 ? 4u : 2u);
        }
    }
}

// A tile's place in its tensor, whose elements are counted from `phase` elements before the first one.
struct TileSpan {
    uint64_t start;              // of the tile
    uint32_t lo, hi;             // the tensor's elements in the tile: [lo, hi) from the tile's start
};

__device__ __forceinline__ TileSpan tile_span(uint64_t n, uint32_t phase, uint32_t index, uint32_t tile_len)
{
    TileSpan s;
    s.start = (uint64_t)index * tile_len;
    s.lo = s.start < phase ? phase - (uint32_t)s.start : 0u;
    const uint64_t end = n + phase;                 // (a row's last tile may lie behind it)
    const uint64_t left = end > s.start ? end - s.start : 0u;
    s.hi = left < tile_len ? (uint32_t)left : tile_len;
    return s;
}

// A walk over a tensor of rows in equal steps.
struct RowCursor {
    uint64_t at;                 // the element's offset in memory
    uint64_t step_at;            // what a step adds
    uint32_t c, step_c, row;     // its column
    uint32_t gap;                // from the end of one row to the next

    // From element `v` on (of all, in row order), `step` elements at a time.
    __device__ __forceinline__ RowCursor(uint64_t v, uint32_t step, uint32_t row_, uint32_t stride) : row(row_)
    {
        const uint64_t r = v / row;
        c = (uint32_t)(v - r * row);
        at = r * stride + c;
        const uint32_t rows = step / row;
        step_c = step - rows * row;
        step_at = (uint64_t)rows * stride + step_c;
        gap = stride - row;
    }
    __device__ __forceinline__ void next()
    {
        at += step_at;
        c += step_c;
        if (c >= row) {
            c -= row;
            at += gap;
        }
    }
};

// ------------------------------------------------------------------------------------------ values
// How long L2 keeps what an access touches.
__device__ __forceinline__ uint64_t l2_policy(bool evict_first)
{
    uint64_t first, normal;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(first));
    asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(normal));
    return evict_first ? first : normal;
}

__device__ __forceinline__ uint4 load16(const void* p, uint64_t policy)
{
    uint4 v;
    asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p), "l"(policy) : "memory");
    return v;
}

// 0 where `in` is false.  (One predicated instruction: with a branch around each, loads would not be in flight together.)
__device__ __forceinline__ uint4 load16_if(bool in, const void* p, uint64_t policy)
{
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    asm volatile("{\n\t.reg .pred in;\n\tsetp.ne.u32 in, %6, 0;\n\t"
                 "@in ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;\n\t}"
                 : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w) : "l"(p), "l"(policy), "r"((uint32_t)in) : "memory");
    return v;
}

__device__ __forceinline__ uint2 load8(const void* p, uint64_t policy)
{
    uint2 v;
    asm volatile("ld.global.L2::cache_hint.v2.u32 {%0, %1}, [%2], %3;" : "=r"(v.x), "=r"(v.y) : "l"(p), "l"(policy) : "memory");
    return v;
}

__device__ __forceinline__ void store16(void* p, uint4 v, uint64_t policy)
{
    asm volatile("st.global.L2::cache_hint.v4.u32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w),
                 "l"(policy) : "memory");
}

__device__ __forceinline__ void store8(void* p, uint2 v, uint64_t policy)
{
    asm volatile("st.global.L2::cache_hint.v2.u32 [%0], {%1, %2}, %3;" ::"l"(p), "r"(v.x), "r"(v.y), "l"(policy) : "memory");
}

__device__ __forceinline__ float load_element(const char* p, uint64_t i, uint32_t type)
{
    if (type == kGradF32) return reinterpret_cast<const float*>(p)[i];
    const uint16_t h = reinterpret_cast<const uint16_t*>(p)[i];
    return type == kGradBF16 ? __uint_as_float((uint32_t)h << 16) : __half2float(__ushort_as_half(h));
}

// One rounding, of the product in fp32 to the destination's type (to nearest, ties to even).
__device__ __forceinline__ void store_element(char* p, uint64_t i, uint32_t type, float x)
{
    if (type == kGradF32)
        reinterpret_cast<float*>(p)[i] = x;
    else if (type == kGradBF16)
        reinterpret_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
    else
        reinterpret_cast<__half*>(p)[i] = __float2half_rn(x);
}

// The two values of a word.
__device__ __forceinline__ float2 widen(uint32_t w, uint32_t type)
{
    if (type == kGradBF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

__device__ __forceinline__ uint32_t narrow(float a, float b, uint32_t type)
{
    if (type == kGradBF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// The elements of a lane that lie 32 apart in a tensor of loose rows, several in flight; 0 from `end` on.
constexpr uint32_t kGradLooseFlight = 16;

template <bool F32>
__device__ __forceinline__ void load_loose(float (&x)[kGradLooseFlight], const char* src, uint32_t type, uint32_t v, uint32_t end,
                                           RowCursor& cur)
{
    uint32_t w[kGradLooseFlight];
#pragma unroll
    for (uint32_t j = 0; j < kGradLooseFlight; ++j) {
        w[j] = 0u;
        if (v + 32u * j < end) {
            if constexpr (F32)
                w[j] = reinterpret_cast<const uint32_t*>(src)[cur.at];
            else
                w[j] = reinterpret_cast<const uint16_t*>(src)[cur.at];
        }
        cur.next();
    }
#pragma unroll
    for (uint32_t j = 0; j < kGradLooseFlight; ++j) x[j] = F32 ? __uint_as_float(w[j]) : widen(w[j], type).x;
}

// ------------------------------------------------------------------------------------------ norm
// A lane's part of a norm: the sum of squares in fp64, or the largest bit pattern without the sign.
template <bool MAX> struct NormPart;

template <> struct NormPart<false> {
    double s;
    __device__ __forceinline__ void add(float x)
    {
        // (volatile: in this order, or dozens of values in 64 bits would be alive at once)
        asm volatile("{\n\t.reg .f64 d;\n\tcvt.f64.f32 d, %1;\n\tfma.rn.f64 %0, d, d, %0;\n\t}" : "+d"(s) : "f"(x));
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
    __device__ __forceinline__ void add(float x) { s = max((uint32_t)s, __float_as_uint(x) & 0x7FFFFFFFu); }
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

// Adds the 16-byte pieces of a lane.  Halves of the maximum of 16-bit types are kept in `pair`, one pattern in each.
template <bool MAX, bool F32, int P>
__device__ __forceinline__ void norm_pieces(const uint4 (&q)[P], uint32_t type, NormPart<MAX> (&acc)[2], uint32_t& pair)
{
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const uint32_t w[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (F32) {
                acc[i & 1].add(__uint_as_float(w[i]));
            } else if constexpr (MAX) {
                pair = __vmaxu2(pair, w[i] & 0x7FFF7FFFu);
            } else {
                const float2 x = widen(w[i], type);
                acc[0].add(x.x);
                acc[1].add(x.y);
            }
        }
    }
}

// The pieces of a lane among `count` of a tile; address() gives one after the other.
template <bool MAX, bool F32, class Address>
__device__ __forceinline__ void norm_piece_range(uint32_t count, uint32_t type, uint64_t policy, NormPart<MAX> (&acc)[2],
                                                 uint32_t& pair, Address&& address)
{
    constexpr uint32_t kFlight = 8;
    for (uint32_t p = threadIdx.x & 31u; p < count; p += 32u * kFlight) {
        uint4 q[kFlight];
#pragma unroll
        for (uint32_t j = 0; j < kFlight; ++j) {
            const uint4* a = address();
            q[j] = load16_if(p + 32u * j < count, a, policy);
        }
        norm_pieces<MAX, F32>(q, type, acc, pair);
    }
}

template <bool ROWS, bool MAX, bool F32>
__device__ __forceinline__ void norm_tile(const GradTensor& g, uint32_t index, uint32_t tile_len, uint64_t policy,
                                          NormPart<MAX> (&acc)[2])
{
    constexpr uint32_t kSize = F32 ? 4u : 2u, kPerPiece = 16u / kSize;
    const uint32_t lane = threadIdx.x & 31u;
    uint32_t pair = 0u;
    if (!ROWS || g.walk <= kGradLong) {
        // the tile's elements, which begin at an aligned address only where the source sets the phase
        const uint32_t phase = tile_phase(g);
        const TileSpan s = tile_span(g.n, phase, index, tile_len);
        const char* first = g.src + (s.start + s.lo - phase) * kSize;
        const uint32_t count = s.hi - s.lo;
        const uint32_t head = min(count, (uint32_t)(0u - reinterpret_cast<uintptr_t>(first) / kSize) % kPerPiece);
        const uint32_t whole = (count - head) / kPerPiece;
        const uint4* pieces = reinterpret_cast<const uint4*>(first + head * kSize) + lane;
        norm_piece_range<MAX, F32>(whole, g.src_type, policy, acc, pair, [&] {
            const uint4* a = pieces;
            pieces += 32;
            return a;
        });
        const uint32_t behind = head + whole * kPerPiece + lane;
        if (lane < head) acc[0].add(load_element(first, lane, g.src_type));
        if (behind < count) acc[1].add(load_element(first, behind, g.src_type));
    } else if constexpr (ROWS) {
        const TileSpan s = tile_span(g.n, 0u, index, tile_len);
        if (g.walk == kGradWide) {
            RowCursor cur(s.start + lane * kPerPiece, 32u * kPerPiece, g.row, g.src_stride);
            norm_piece_range<MAX, F32>(s.hi / kPerPiece, g.src_type, policy, acc, pair, [&] {
                const uint4* a = reinterpret_cast<const uint4*>(g.src + cur.at * kSize);
                cur.next();
                return a;
            });
        } else {
            RowCursor cur(s.start + lane, 32u, g.row, g.src_stride);
            for (uint32_t v = lane; v < s.hi; v += 32u * kGradLooseFlight) {
                float x[kGradLooseFlight];
                load_loose<F32>(x, g.src, g.src_type, v, s.hi, cur);
#pragma unroll
                for (uint32_t j = 0; j < kGradLooseFlight; ++j) acc[j & 1u].add(x[j]);
            }
        }
    }
    if constexpr (MAX && !F32) {
        const float2 x = widen(pair, g.src_type);
        acc[0].add(x.x);
        acc[1].add(x.y);
    }
}

// Adds one tile of a tensor to a lane's part.
template <bool ROWS, bool MAX>
__device__ __forceinline__ void norm_tile(const GradTensor& g, uint32_t tile, uint32_t tile_len, uint64_t policy,
                                          NormPart<MAX> (&acc)[2])
{
    for_pieces<ROWS>(g, tile, tile_len, [&](const GradTensor& p, uint32_t index, uint32_t len) {
        if (p.src_type == kGradF32)
            norm_tile<ROWS, MAX, true>(p, index, len, policy, acc);
        else
            norm_tile<ROWS, MAX, false>(p, index, len, policy, acc);
    });
}

// Writes the norm and reports one that is no finite number.
__device__ __forceinline__ void publish_norm(float norm, float* out_norm, uint32_t* status)
{
    if (out_norm) *out_norm = norm;
    if (status && !(fabsf(norm) <= 3.402823466e38f)) atomicOr(status, kWarnNonfiniteNorm);
}

// A part of the norm per CTA (slots[blockIdx]), or with EACH per tile (slots[tile]).  One wave of four CTAs per SM (64
// registers: 128 KB in flight per SM).  Bound by HBM: with the join behind it 124 M bf16 elements take 43.7 us (5.7 TB/s; their
// maximum 40.6), 124 M fp32 78 us (6.4 TB/s), 25.6 M fp32 20.7 us (4.9 TB/s: 5 us are launch, ramp and join).  Five CTAs spill,
// CTAs of 1024 threads are 1 us slower on short lists, more waves no faster.  (The next kernel is one of the same call, which
// waits: it may be let in at once.)
template <class Table, bool ROWS, bool MAX, bool EACH>
__global__ void __launch_bounds__(kGradThreads, kGradNormCtas)
grad_norm_kernel(const __grid_constant__ Table t, NormPart<MAX>* slots)
{
    __shared__ NormPart<MAX> parts[kGradWarps];
    const uint32_t tiles = t.first_tile[t.count], first = blockIdx.x * kGradWarps + (threadIdx.x >> 5);
    NormPart<MAX> acc[2] = {};
    TensorRun run;
    run.start<ROWS>(t, first, tiles);
    grid_dependency_wait();
    grid_dependency_launch_next();
    for (uint32_t tile = first; tile < tiles; tile += gridDim.x * kGradWarps) {
        if (tile >= run.end) run.seek<ROWS>(t, tile);
        norm_tile<ROWS, MAX>(run.g, tile - run.first, t.tile_len, l2_policy(tile < t.stream_below), acc);
        if constexpr (EACH) {
            acc[0].join(acc[1]);
            reduce_warp(acc[0]);
            if ((threadIdx.x & 31u) == 0u) slots[tile] = acc[0];
            acc[0] = acc[1] = {};
        }
    }
    if constexpr (!EACH) {
        acc[0].join(acc[1]);
        reduce_block(acc[0], parts, kGradWarps);
        if (threadIdx.x == 0u) slots[blockIdx.x] = acc[0];
    }
}

// Joins the slots begin, begin + step, ... below end: F of them are in flight together.
template <uint32_t F, bool MAX>
__device__ __forceinline__ void join_slots(NormPart<MAX>& acc, const NormPart<MAX>* slots, uint32_t begin, uint32_t end,
                                           uint32_t step)
{
    for (uint32_t i = begin; i < end; i += F * step) {
        NormPart<MAX> part[F];
#pragma unroll
        for (uint32_t j = 0; j < F; ++j) {
            part[j] = slots[min(i + j * step, end - 1u)];
            if (i + j * step >= end) part[j] = {};
        }
#pragma unroll
        for (uint32_t j = 0; j < F; ++j) acc.join(part[j]);
    }
}

// The whole from the slots of all launches before it (CTA 0, where `out_norm` is given), and the norms of single tensors
// from the slots of their tiles, a warp each: tensor i of the launch owns the slots [first[i], first[i + 1]).  The slots lie in
// the call's workspace, which the caller may have given back by now, and the next kernel may be an encode that has been handed
// that memory and stores without waiting (EncodeArgs::early_store): this kernel lets it in by its end only.  (Norms of 25.6 M fp32
// elements and of their 161 tensors, back to back: 21.8 us; let in behind the last read of a slot 22.8, and at once, which is
// not sound, 20.7.)
constexpr int kGradJoinThreads = 1024;

template <int N>
struct GradEachTable {
    static constexpr int kCapacity = N;
    uint32_t count;
    uint32_t first[N + 1];
};

template <class Table, bool MAX>
__global__ void __launch_bounds__(kGradJoinThreads)
grad_norm_join_kernel(const __grid_constant__ Table t, const NormPart<MAX>* slots, uint32_t num_slots, float* out_norm,
                      float* out_norms, uint32_t* status)
{
    __shared__ NormPart<MAX> parts[kGradJoinThreads / 32];
    grid_dependency_wait();
    NormPart<MAX> acc = {};
    if (blockIdx.x == 0u) {
        if (!out_norm) return;
        join_slots<8>(acc, slots, threadIdx.x, num_slots, kGradJoinThreads);
        reduce_block(acc, parts, kGradJoinThreads / 32);
        if (threadIdx.x == 0u) publish_norm(acc.norm(), out_norm, status);
        return;
    }
    const uint32_t i = (blockIdx.x - 1u) * (kGradJoinThreads / 32u) + (threadIdx.x >> 5);
    if (i >= t.count) return;
    join_slots<16>(acc, slots, t.first[i] + (threadIdx.x & 31u), t.first[i + 1u], 32u);
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
    uint16_t in_place;           // the destination is the source
    uint16_t max_kind;           // the slots are maxima
    uint16_t norm_in_workspace;  // `norm` is not the caller's
};

__device__ __forceinline__ float clip_factor(float norm, float max_norm)
{
    return norm <= max_norm ? 1.0f : __fdiv_rn(max_norm, norm);
}

// A lane's unit of work: the elements that are 16 bytes on the wider side, so that a warp's loads and stores are contiguous.
template <bool SF32, bool DF32> constexpr uint32_t kGradGroup = SF32 || DF32 ? 4u : 8u;

// 16 or 8 bytes as words.
template <int W> struct GradPiece {
    uint32_t w[W];
    __device__ __forceinline__ void load(const char* p, uint64_t policy)
    {
        if constexpr (W == 4) {
            const uint4 v = load16(p, policy);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else {
            const uint2 v = load8(p, policy);
            w[0] = v.x, w[1] = v.y;
        }
    }
};

// The words that start `shift` bytes (whole elements) into a, with what lies behind it: the next lane's piece, and behind
// the last lane's the first lane's next one.  The piece's own size is the most that it can be shifted by.
template <int W, bool HALF>
__device__ __forceinline__ GradPiece<W> shifted(const GradPiece<W>& a, const GradPiece<W>& next, uint32_t shift)
{
    constexpr int kBehind = HALF ? W : W - 1;              // words that are needed from behind
    const uint32_t lane = threadIdx.x & 31u;
    uint32_t v[2 * W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        v[i] = a.w[i];
        if (i < kBehind) v[W + i] = __shfl_sync(0xFFFFFFFFu, lane == 0u ? next.w[i] : a.w[i], lane + 1u);
        else v[W + i] = 0u;
    }
    if constexpr (W == 4) {
        if (shift & 8u) {
#pragma unroll
            for (int i = 0; i + 2 < 2 * W; ++i) v[i] = v[i + 2];
        }
    }
    if (shift & 4u) {
#pragma unroll
        for (int i = 0; i + 1 < 2 * W; ++i) v[i] = v[i + 1];
    }
    GradPiece<W> out;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        out.w[i] = v[i];
        if constexpr (HALF) {
            if (shift & 2u) out.w[i] = __funnelshift_r(v[i], v[i + 1], 16);
        }
    }
    return out;
}

// The factor, and the L2 policies of both sides.
struct Scaling {
    float c;
    uint64_t src, dst;
};

// A group, from the words it was read as to its destination.
template <bool SF32, bool DF32, int W>
__device__ __forceinline__ void store_group(const GradPiece<W>& w, const GradTensor& g, const Scaling& f, char* d)
{
    constexpr uint32_t kGroup = kGradGroup<SF32, DF32>;
    float x[kGroup];
#pragma unroll
    for (uint32_t i = 0; i < kGroup; i += 2u) {
        float2 v;
        if constexpr (SF32)
            v = make_float2(__uint_as_float(w.w[i]), __uint_as_float(w.w[i + 1u]));
        else
            v = widen(w.w[i / 2u], g.src_type);
        x[i] = __fmul_rn(v.x, f.c);
        x[i + 1u] = __fmul_rn(v.y, f.c);
    }
    if constexpr (DF32) {
        store16(d, make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])), f.dst);
    } else if constexpr (kGroup == 4u) {
        store8(d, make_uint2(narrow(x[0], x[1], g.dst_type), narrow(x[2], x[3], g.dst_type)), f.dst);
    } else {
        store16(d, make_uint4(narrow(x[0], x[1], g.dst_type), narrow(x[2], x[3], g.dst_type), narrow(x[4], x[5], g.dst_type),
                              narrow(x[6], x[7], g.dst_type)), f.dst);
    }
}

// The next kFlight groups of every lane of a contiguous tile; with EDGE those from `left` on are no longer the tile's: the
// last one that may be read is read again, and nothing is stored.
template <bool SF32, bool DF32, bool SHIFT, bool EDGE, uint32_t kFlight>
__device__ __forceinline__ void scale_batch(const char* src, char* dst, uint32_t left, const GradTensor& g, uint32_t shift,
                                            const Scaling& f)
{
    constexpr uint32_t kGroup = kGradGroup<SF32, DF32>;
    constexpr uint32_t kSrc = kGroup * (SF32 ? 4u : 2u), kDst = kGroup * (DF32 ? 4u : 2u);
    const uint32_t lane = threadIdx.x & 31u, last = SHIFT ? left : left - 1u;
    auto from = [&](uint32_t p) { return src + (EDGE ? min(p, last) : p) * kSrc; };
    GradPiece<kSrc / 4u> q[kFlight + (SHIFT ? 1 : 0)];
#pragma unroll
    for (uint32_t j = 0; j < kFlight; ++j) q[j].load(from(32u * j + lane), f.src);
    if constexpr (SHIFT) q[kFlight].load(from(32u * kFlight), f.src);
#pragma unroll
    for (uint32_t j = 0; j < kFlight; ++j) {
        GradPiece<kSrc / 4u> w = q[j];
        if constexpr (SHIFT) w = shifted<kSrc / 4u, !SF32>(q[j], q[j + 1u], shift);
        const uint32_t p = 32u * j + lane;
        if (!EDGE || p < left) store_group<SF32, DF32>(w, g, f, dst + p * kDst);
    }
}

// The whole groups [begin, end) of a contiguous tile, eight of a lane in flight (four of 16-bit elements on both sides).
// Group p lies at src + p and dst + p groups, both aligned to the group's size there; the source there is `shift` bytes
// before the group's first element, and group `end` may be read too where shift is not 0.
template <bool SF32, bool DF32, bool SHIFT>
__device__ __forceinline__ void scale_groups(uint32_t begin, uint32_t end, const GradTensor& g, uint32_t shift, const Scaling& f,
                                             const char* src, char* dst)
{
    constexpr uint32_t kGroup = kGradGroup<SF32, DF32>, kFlight = kGroup == 8u ? 4u : 8u;
    constexpr uint32_t kSrc = kGroup * (SF32 ? 4u : 2u), kDst = kGroup * (DF32 ? 4u : 2u);
    uint32_t left = end - begin;
    src += begin * kSrc;
    dst += begin * kDst;
    for (; left >= 32u * kFlight; left -= 32u * kFlight) {
        scale_batch<SF32, DF32, SHIFT, false, kFlight>(src, dst, left, g, shift, f);
        src += 32u * kFlight * kSrc;
        dst += 32u * kFlight * kDst;
    }
#pragma unroll 1
    while (left != 0u) {
        scale_batch<SF32, DF32, SHIFT, true, 4u>(src, dst, left, g, shift, f);
        left -= min(left, 128u);
        src += 128u * kSrc;
        dst += 128u * kDst;
    }
}

// The groups of a tile of a tensor in rows.
template <bool SF32, bool DF32>
__device__ __forceinline__ void scale_row_groups(const TileSpan& s, const GradTensor& g, const Scaling& f)
{
    constexpr uint32_t kGroup = kGradGroup<SF32, DF32>, kFlight = 4u;
    constexpr uint32_t kSrc = kGroup * (SF32 ? 4u : 2u), kDst = kGroup * (DF32 ? 4u : 2u);
    const uint32_t end = s.hi / kGroup;
    const uint64_t v = s.start + (threadIdx.x & 31u) * kGroup;
    RowCursor from(v, 32u * kGroup, g.row, g.src_stride), to(v, 32u * kGroup, g.row, g.dst_stride);
    for (uint32_t p = threadIdx.x & 31u; p < end; p += 32u * kFlight) {
        GradPiece<kSrc / 4u> q[kFlight] = {};
#pragma unroll
        for (uint32_t j = 0; j < kFlight; ++j) {
            if (p + 32u * j < end) q[j].load(g.src + from.at * (kSrc / kGroup), f.src);
            from.next();
        }
#pragma unroll
        for (uint32_t j = 0; j < kFlight; ++j) {
            if (p + 32u * j < end) store_group<SF32, DF32>(q[j], g, f, g.dst + to.at * (kDst / kGroup));
            to.next();
        }
    }
}

template <bool ROWS, bool SF32, bool DF32>
__device__ __forceinline__ void scale_tile(const GradTensor& g, uint32_t index, uint32_t tile_len, const Scaling& f)
{
    constexpr uint32_t kSrc = SF32 ? 4u : 2u, kDst = DF32 ? 4u : 2u, kGroup = kGradGroup<SF32, DF32>;
    const uint32_t lane = threadIdx.x & 31u;
    if (!ROWS || g.walk <= kGradLong) {
        const uint32_t phase = tile_phase(g);
        const TileSpan s = tile_span(g.n, phase, index, tile_len);
        const char* src = g.src - phase * kSrc;
        char* dst = g.dst - phase * kDst;
        const uint32_t shift = (uint32_t)reinterpret_cast<uintptr_t>(src) & (kGroup * kSrc - 1u);
        uint32_t lo = s.lo, hi = s.hi;
        if (shift) {
            // the pieces of a shifted group reach up to a group before and behind it: not past the tensor
            if (s.start < phase + kGroup) lo = phase + kGroup - (uint32_t)s.start;
            const uint64_t left = g.n + phase - s.start;
            if (left < (uint64_t)hi + kGroup) hi = left < kGroup ? 0u : (uint32_t)left - kGroup;
        }
        const uint32_t begin = (lo + kGroup - 1u) / kGroup, end = max(begin, hi / kGroup);
        const char* a = src + s.start * kSrc - shift;
        char* b = dst + s.start * kDst;
        if (shift)
            scale_groups<SF32, DF32, true>(begin, end, g, shift, f, a, b);
        else
            scale_groups<SF32, DF32, false>(begin, end, g, 0u, f, a, b);
        // what lies before the first of these groups and behind the last one: at most 15 elements each
        const uint32_t before = s.lo + lane, behind = end * kGroup + lane;
        if (before < min(begin * kGroup, s.hi))
            store_element(dst, s.start + before, g.dst_type, __fmul_rn(load_element(src, s.start + before, g.src_type), f.c));
        if (behind < s.hi)
            store_element(dst, s.start + behind, g.dst_type, __fmul_rn(load_element(src, s.start + behind, g.src_type), f.c));
    } else if constexpr (ROWS) {
        const TileSpan s = tile_span(g.n, 0u, index, tile_len);
        if (g.walk == kGradWide) {
            scale_row_groups<SF32, DF32>(s, g, f);
        } else {
            RowCursor from(s.start + lane, 32u, g.row, g.src_stride), to(s.start + lane, 32u, g.row, g.dst_stride);
            for (uint32_t v = lane; v < s.hi; v += 32u * kGradLooseFlight) {
                float x[kGradLooseFlight];
                load_loose<SF32>(x, g.src, g.src_type, v, s.hi, from);
#pragma unroll
                for (uint32_t j = 0; j < kGradLooseFlight; ++j) {
                    if (v + 32u * j < s.hi) store_element(g.dst, to.at, g.dst_type, __fmul_rn(x[j], f.c));
                    to.next();
                }
            }
        }
    }
}

// Multiplies one tile by c into the destination.
template <bool ROWS>
__device__ __forceinline__ void scale_tile(const GradTensor& g, uint32_t tile, uint32_t tile_len, const Scaling& f)
{
    for_pieces<ROWS>(g, tile, tile_len, [&](const GradTensor& p, uint32_t index, uint32_t len) {
        if (p.src_type == kGradF32) {
            if (p.dst_type == kGradF32)
                scale_tile<ROWS, true, true>(p, index, len, f);
            else
                scale_tile<ROWS, true, false>(p, index, len, f);
        } else {
            if (p.dst_type == kGradF32)
                scale_tile<ROWS, false, true>(p, index, len, f);
            else
                scale_tile<ROWS, false, false>(p, index, len, f);
        }
    });
}

// The norm from its parts, by one warp: every CTA begins with it, so all loads of up to 640 parts are in flight together.
template <bool MAX>
__device__ __forceinline__ float joined_norm(const ClipArgs& a)
{
    NormPart<MAX> acc = {};
    join_slots<20>(acc, static_cast<const NormPart<MAX>*>(a.slots), threadIdx.x & 31u, a.num_slots, 32u);
    reduce_warp(acc);
    return acc.norm();
}

// The last tiles first: they are what the norm's pass has left in L2.  What is read here is read for the last time, and what
// is written need not push the rest of the gradient out: both go with the policy to leave L2 first.  Bound by HBM: 124 M fp32
// elements, given the norm, 149 us (6.7 TB/s); after the norm's pass of the same call, which reads them too, 230 us for both.
// Where both passes' data fit in L2 (11.7 M fp16 to fp32: 20 us) two launches, their ramps and the joined norm are a third.
template <class Table, bool ROWS>
__global__ void __launch_bounds__(kGradThreads, kGradScaleCtas)
grad_scale_kernel(const __grid_constant__ Table t, const __grid_constant__ ClipArgs a)
{
    __shared__ float factor;
    const uint32_t tiles = t.first_tile[t.count], first = blockIdx.x * kGradWarps + (threadIdx.x >> 5);
    TensorRun run;
    run.start<ROWS>(t, tiles - 1u - first, tiles);
    grid_dependency_wait();
    float c = 1.0f;
    if (a.num_slots) {
        if (threadIdx.x < 32u) {
            const float norm = a.max_kind ? joined_norm<true>(a) : joined_norm<false>(a);
            if (threadIdx.x == 0u) {
                factor = clip_factor(norm, a.max_norm);
                if (blockIdx.x == 0u) publish_norm(norm, a.out_norm, a.status);
            }
        }
        __syncthreads();
        c = factor;
    } else if (a.norm) {
        const float norm = *a.norm;
        c = clip_factor(norm, a.max_norm);
        if (blockIdx.x == 0u && threadIdx.x == 0u) publish_norm(norm, a.out_norm, a.status);
        if (a.norm_in_workspace) {
            // one thread lets the next kernel in for its CTA: not before all have their factor (see grad_norm_join_kernel)
            asm volatile("" ::"f"(c));
            __syncthreads();
        }
    }
    grid_dependency_launch_next();
    if (a.in_place && c == 1.0f) return;
    const Scaling f = {c, l2_policy(true), l2_policy(true)};
    for (uint32_t i = first; i < tiles; i += gridDim.x * kGradWarps) {
        const uint32_t tile = tiles - 1u - i;
        if (tile < run.first || tile >= run.end) run.seek<ROWS>(t, tile);
        scale_tile<ROWS>(run.g, tile - run.first, t.tile_len, f);
    }
}

// ------------------------------------------------------------------------------------------ short lists
// Norm and clipping of a short list in one launch: a cluster of CTAs whose parts of the norm meet over distributed
// shared memory.  SCALE: multiplies as well.  Bound by one launch and two passes of latency: norm of 266,610 fp32 elements 4.5
// us, norm and clipping of 65,536 4.0 us.  (On the GPU two launches would take 3.7 and 4.5 us, but their host work takes 7.)
template <class Table, bool ROWS, bool MAX, bool SCALE>
__global__ void __launch_bounds__(kGradClusterThreads)
grad_cluster_kernel(const __grid_constant__ Table t, const __grid_constant__ ClipArgs a)
{
    constexpr uint32_t kWarps = kGradClusterThreads / 32;
    __shared__ NormPart<MAX> parts[kWarps];
    __shared__ NormPart<MAX> mine;
    __shared__ float factor;
    const uint32_t tiles = t.first_tile[t.count], step = gridDim.x * kWarps;
    const uint32_t first = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;
    NormPart<MAX> acc[2] = {};
    TensorRun run;
    run.start<ROWS>(t, first, tiles);
    grid_dependency_wait();
    grid_dependency_launch_next();
    for (uint32_t tile = first; tile < tiles; tile += step) {
        if (tile >= run.end) run.seek<ROWS>(t, tile);
        norm_tile<ROWS, MAX>(run.g, tile - run.first, t.tile_len, l2_policy(tile < t.stream_below), acc);
    }
    acc[0].join(acc[1]);
    reduce_block(acc[0], parts, kWarps);
    if (threadIdx.x == 0u) mine = acc[0];
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
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
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");     // (no CTA leaves while its part is read)
    if constexpr (SCALE) {
        const float c = factor;
        if (!(a.in_place && c == 1.0f)) {
            const Scaling f = {c, l2_policy(false), l2_policy(false)};
            if (step < tiles) run.end = 0u;          // (a warp of one tile is still at its tensor)
            for (uint32_t tile = first; tile < tiles; tile += step) {
                if (tile >= run.end) run.seek<ROWS>(t, tile);
                scale_tile<ROWS>(run.g, tile - run.first, t.tile_len, f);
            }
        }
    }
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

}  // namespace dq
