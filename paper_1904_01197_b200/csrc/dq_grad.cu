// Host side of the calls on gradients of many tensors (include/dq.h): argument checks, the tables of tensors that travel
// in the kernels' parameters, launches.  The kernels are in dq_grad.cuh.
#include "dq_grad.cuh"

#include <algorithm>
#include <initializer_list>
#include <memory>
#include <mutex>
#include <new>

#include "dq.h"
#include "dq_launch.h"

static_assert(dq::kWarnNonfiniteNorm == DQ_WARN_NONFINITE_NORM, "status bit of the norm kernels");
static_assert((int)dq::kGradF32 == DQ_F32 && (int)dq::kGradBF16 == DQ_BF16 && (int)dq::kGradF16 == DQ_F16, "types");

namespace {

// Tables of three sizes: a launch passes them by value, and every KB of parameters costs it 0.08 us.  A tensor takes 16
// bytes of the norm's table and 24 of the other one.
template <int W> constexpr int kSmall = 16;
template <int W> constexpr int kMiddle = 256;
template <int W> constexpr int kLarge = W == 3 ? 2040 : 1360;
constexpr int kNorm = 3, kScale = 5;             // words of an entry
static_assert(sizeof(dq::GradTable<kLarge<kNorm>, kNorm>) + 8 <= 32764, "kernel parameters");
static_assert(sizeof(dq::GradTable<kLarge<kScale>, kScale>) + sizeof(dq::ClipArgs) <= 32764, "kernel parameters");
constexpr int kEachMiddle = 512, kEachLarge = 8000;          // tables of the single tensors' slots, 4 bytes each
static_assert(sizeof(dq::GradEachTable<kEachLarge>) + 64 <= 32764, "kernel parameters");

// Lists up to this many elements (and half of kMiddle tensors) are done by one cluster in one launch.  Where the GPU is through
// sooner with two launches (norm, from 200,000 elements on: 524,288 3.8 us and 5.9 with the cluster; norm and scaling 4.8 and 8.2,
// 262,144 4.8 and 5.9), it still waits for the host, whose work is 4 us for one launch and 7.3 for two.
constexpr uint64_t kShortNorm = 1ull << 19, kShortScale = 3ull << 17;

// Parts of the norm: at most kMaxGrid of a launch, or one per tile where each tensor's norm is wanted as well.
constexpr uint32_t kMaxGrid = 1024u;
constexpr uint64_t kEachTiles = 16384u;          // of full length

// Host memory for a list that is too long for the stack, kept by the thread: fresh pages for every call would take longer than
// what is done with them.  Null where there is none.
template <class T>
T* host_scratch(size_t count)
{
    struct Kept {
        std::unique_ptr<T[]> p;
        size_t count = 0u;
    };
    static thread_local Kept kept;
    if (kept.count < count) {
        kept.count = 0u;
        kept.p.reset(new (std::nothrow) T[count + count / 2u]);
        if (kept.p) kept.count = count + count / 2u;
    }
    return kept.p.get();
}

uint32_t size_log2(uint32_t dtype) { return dtype == DQ_F32 ? 2u : 1u; }
uint32_t element_size(uint32_t dtype) { return 1u << size_log2(dtype); }

bool has_rows(const dq_tensor& t) { return t.row != 0u && t.row_stride != t.row && t.row != t.n; }

dq_status check_tensor(const dq_tensor& t)
{
    if ((uint32_t)t.dtype > (uint32_t)DQ_F16 || t.reserved != 0u) return DQ_ERR_INVALID_ARG;
    if (t.n == 0u) return DQ_OK;
    if (!t.data) return DQ_ERR_INVALID_ARG;
    if (t.n >= (1ull << 34)) return DQ_ERR_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(t.data) & (element_size(t.dtype) - 1u)) != 0u) return DQ_ERR_ALIGNMENT;
    if (reinterpret_cast<uintptr_t>(t.data) >> 57) return DQ_ERR_UNSUPPORTED;           // (no device address is as large)
    if (t.row != 0u) {
        if (t.n % t.row != 0u || t.row_stride < t.row) return DQ_ERR_INVALID_ARG;
        if (has_rows(t) && (t.row >= (1ull << 31) || t.row_stride >= (1ull << 32) ||
                            t.n / t.row > (1ull << 57) / (t.row_stride << size_log2(t.dtype))))
            return DQ_ERR_UNSUPPORTED;
    }
    return DQ_OK;
}

// What the checks find out about a list on the way.
struct ListInfo {
    uint64_t total = 0u, bytes = 0u;
};

dq_status check_list(const dq_tensor* list, uint32_t count, ListInfo* info)
{
    *info = ListInfo();
    if (count > DQ_MAX_TENSORS) return DQ_ERR_UNSUPPORTED;
    if (count != 0u && !list) return DQ_ERR_INVALID_ARG;
    for (uint32_t i = 0; i < count; ++i) {
        const dq_status s = check_tensor(list[i]);
        if (s != DQ_OK) return s;
        info->total += list[i].n;
        info->bytes += list[i].n << size_log2(list[i].dtype);
        if (info->total >= (1ull << 34)) return DQ_ERR_UNSUPPORTED;
    }
    return DQ_OK;
}

// ------------------------------------------------------------------------------------------ overlap
struct Extent {
    uintptr_t lo, hi;            // bytes
    uint64_t width, pitch;       // of a row; pitch 0: one piece
    bool out;
};

Extent extent_of(const dq_tensor& t, bool out)
{
    const uint64_t size = element_size(t.dtype);
    Extent e;
    e.lo = reinterpret_cast<uintptr_t>(t.data);
    e.out = out;
    if (has_rows(t)) {
        e.width = t.row * size;
        e.pitch = t.row_stride * size;
        e.hi = e.lo + (t.n / t.row - 1u) * e.pitch + e.width;
    } else {
        e.width = t.n * size;
        e.pitch = 0u;
        e.hi = e.lo + e.width;
    }
    return e;
}

// a.lo <= b.lo < a.hi.  Blocks of rows of one pitch may lie side by side; anything else that interleaves counts.
bool rows_overlap(const Extent& a, const Extent& b)
{
    if (a.pitch == 0u || (b.pitch != 0u && b.pitch != a.pitch)) return true;
    const uint64_t column = (b.lo - a.lo) % a.pitch;
    return column < a.width || column + b.width > a.pitch;
}

// The extents in the order of their addresses.  Tensors that were allocated one after the other form ascending runs, which
// are merged (std::sort does not notice them: 2000 tensors into 2000 others, 49 us with it and 21 so; in no order 150 and 110).
struct Place {
    uintptr_t lo;
    uint32_t i;
};

// `order` and `other` have a place for every extent, `runs` one more; the result is in `order`, which may be the other one then.
void by_address(const Extent* e, uint32_t count, Place*& order, Place*& other, uint32_t* runs)
{
    uint32_t num_runs = 0u;
    for (uint32_t i = 0; i < count; ++i) {
        order[i] = {e[i].lo, i};
        if (i == 0u || e[i].lo < e[i - 1u].lo) runs[num_runs++] = i;
    }
    runs[num_runs] = count;
    auto before = [](const Place& a, const Place& b) { return a.lo < b.lo; };
    while (num_runs > 1u) {
        uint32_t merged = 0u;
        for (uint32_t r = 0; r < num_runs; r += 2u) {
            const uint32_t lo = runs[r], mid = runs[r + 1u], hi = r + 1u < num_runs ? runs[r + 2u] : mid;
            std::merge(order + lo, order + mid, order + mid, order + hi, other + lo, before);
            runs[merged++] = lo;
        }
        runs[merged] = count;
        num_runs = merged;
        std::swap(order, other);
    }
}

// A group: extents in the order of their addresses that reach, one over another, from the first to the last.  Small ones (the
// blocks of a fused layer, say) are compared pair by pair; beyond this many that takes longer (ns of the host per tensor clipped in
// place: groups of 32 blocks 75 pair by pair and 84 otherwise, of 48 104 and 92, of 4000 7100 and 330, of 65,536 119,000 and 416).
constexpr uint32_t kPairs = 40u;

bool pairs_overlap(const Extent* e, const Place* order, uint32_t count)
{
    for (uint32_t i = 1; i < count; ++i) {
        const Extent& x = e[order[i].i];
        for (uint32_t k = 0; k < i; ++k) {
            const Extent& y = e[order[k].i];
            if ((x.out || y.out) && y.hi > x.lo && rows_overlap(y, x)) return true;
        }
    }
    return false;
}

// The furthest end of rows of one pitch, and of rows of any other.
struct RowReach {
    uintptr_t best = 0u, other = 0u;
    uint64_t pitch = 0u;

    uintptr_t beside(uint64_t p) const { return p == pitch ? other : best; }
    void add(uint64_t p, uintptr_t hi)
    {
        if (p == pitch) {
            best = std::max(best, hi);
        } else if (hi > best) {
            other = best;
            best = hi;
            pitch = p;
        } else {
            other = std::max(other, hi);
        }
    }
};

// How far the blocks of one pitch reach that have been added, by column: a tree over the columns between the sorted `points`,
// where the blocks begin and end.  A block is a range of columns (two, if it begins in one row and ends in the next).
struct ColumnReach {
    uint64_t pitch;
    uintptr_t *points, *best, *tag;      // best: of a node's columns; tag: of blocks that have all of them
    uint32_t columns;

    // Words of memory for this many blocks.
    static size_t words(size_t blocks) { return 2u * blocks + 2u + 3u * (2u * blocks + 1u); }

    template <class F>
    void for_ranges(const Extent& x, F&& f) const
    {
        const uint64_t c = x.lo % pitch, end = c + std::min(x.width, pitch);
        f(c, std::min(end, pitch));
        if (end > pitch) f((uint64_t)0u, end - pitch);
    }
    // ... of at least one block each
    template <class F>
    void lay_out(uint64_t p, uintptr_t* memory, uint32_t blocks, F&& block)
    {
        pitch = p;
        points = memory;
        uint32_t m = 0u;
        points[m++] = 0u;
        points[m++] = pitch;
        for (uint32_t k = 0; k < blocks; ++k) {
            const Extent& x = block(k);
            points[m++] = x.lo % pitch;
            points[m++] = (x.lo + x.width) % pitch;
        }
        std::sort(points, points + m);
        columns = (uint32_t)(std::unique(points, points + m) - points) - 1u;
        best = points + columns + 1u;
        tag = best + 2u * columns;
    }
    void clear() { std::fill(best, tag + columns, (uintptr_t)0u); }
    void add(const Extent& x)
    {
        for_ranges(x, [&](uint64_t from, uint64_t to) {
            const uint32_t lo = column(from) + columns, hi = column(to) + columns;
            auto raise = [&](uint32_t node) {
                best[node] = std::max(best[node], x.hi);
                if (node < columns) tag[node] = std::max(tag[node], x.hi);
            };
            for (uint32_t l = lo, r = hi; l < r; l /= 2u, r /= 2u) {
                if (l & 1u) raise(l++);
                if (r & 1u) raise(--r);
            }
            for (uint32_t node : {lo, hi - 1u})
                while ((node /= 2u) != 0u) best[node] = std::max({best[2u * node], best[2u * node + 1u], tag[node]});
        });
    }
    // ... over the columns of x, of whatever kind.
    uintptr_t over(const Extent& x) const
    {
        uintptr_t reach = 0u;
        for_ranges(x, [&](uint64_t from, uint64_t to) {
            const uint32_t lo = column(from) + columns;
            const uint32_t hi = (uint32_t)(std::lower_bound(points, points + columns, to) - points) + columns;
            for (uint32_t l = lo, r = hi; l < r; l /= 2u, r /= 2u) {
                if (l & 1u) reach = std::max(reach, best[l++]);
                if (r & 1u) reach = std::max(reach, best[--r]);
            }
            for (uint32_t node : {lo, hi - 1u})
                while ((node /= 2u) != 0u) reach = std::max(reach, tag[node]);
        });
        return reach;
    }

private:
    // The one that begins at or before `at`.
    uint32_t column(uint64_t at) const { return (uint32_t)(std::upper_bound(points, points + columns + 1u, at) - points) - 1u; }
};

// The same of a large group, in n log n: whatever meets a contiguous extent, or rows of another pitch, overlaps it; of the rest,
// rows of one pitch, and contiguous extents between them, it depends on the columns.  (A contiguous output is looked up once
// for every pitch that its group has.)  `by_pitch` has a place for every extent.
dq_status group_overlaps(const Extent* e, const Place* order, Place* by_pitch, uint32_t count, bool* overlaps)
{
    *overlaps = true;
    uintptr_t flat_reach = 0u, flat_out_reach = 0u;
    RowReach rows, out_rows;
    uint32_t flats = 0u, outs = 0u;
    for (uint32_t i = 0; i < count; ++i) {
        const Extent& x = e[order[i].i];
        by_pitch[i] = {(uintptr_t)x.pitch, i};
        outs += x.out ? 1u : 0u;
        if (x.lo < (x.out ? flat_reach : flat_out_reach)) return DQ_OK;
        if (x.pitch == 0u) {
            ++flats;
            flat_reach = std::max(flat_reach, x.hi);
            if (x.out) flat_out_reach = std::max(flat_out_reach, x.hi);
        } else {
            if (x.lo < (x.out ? rows : out_rows).beside(x.pitch)) return DQ_OK;
            rows.add(x.pitch, x.hi);
            if (x.out) out_rows.add(x.pitch, x.hi);
        }
    }
    *overlaps = false;
    if (outs == 0u) return DQ_OK;
    std::sort(by_pitch, by_pitch + count, [](const Place& a, const Place& b) { return a.lo != b.lo ? a.lo < b.lo : a.i < b.i; });
    auto at = [&](uint32_t k) -> const Extent& { return e[order[by_pitch[k].i].i]; };
    for (uint32_t begin = flats, end; begin < count; begin = end) {
        for (end = begin; end < count && by_pitch[end].lo == by_pitch[begin].lo;) ++end;
        if (end - begin == 1u && flats == 0u) continue;
        uintptr_t* memory = host_scratch<uintptr_t>(ColumnReach::words(end - begin));
        if (!memory) return DQ_ERR_CUDA;
        ColumnReach reach;
        reach.lay_out(by_pitch[begin].lo, memory, end - begin, [&](uint32_t k) -> const Extent& { return at(begin + k); });
        // outputs against everything, then inputs against outputs
        for (const bool out : {true, false}) {
            if (!out && outs == count) break;
            reach.clear();
            for (uint32_t f = 0u, r = begin; f < flats || r < end;) {
                const bool flat = r == end || (f < flats && by_pitch[f].i < by_pitch[r].i);
                const Extent& x = at(flat ? f++ : r++);
                if ((out || x.out) && reach.over(x) > x.lo) {
                    *overlaps = true;
                    return DQ_OK;
                }
                if (!flat && x.out == out) reach.add(x);
            }
        }
    }
    return DQ_OK;
}

// DQ_ERR_INVALID_ARG where an output overlaps another tensor.  `spare` has a place for every extent.
dq_status check_overlap(const Extent* e, const Place* order, Place* spare, uint32_t count)
{
    for (uint32_t begin = 0u, end; begin < count; begin = end) {
        uintptr_t reach = e[order[begin].i].hi;
        for (end = begin + 1u; end < count && order[end].lo < reach; ++end) reach = std::max(reach, e[order[end].i].hi);
        bool overlaps;
        if (end - begin <= kPairs) {
            overlaps = pairs_overlap(e, order + begin, end - begin);
        } else {
            const dq_status s = group_overlaps(e, order + begin, spare, end - begin, &overlaps);
            if (s != DQ_OK) return s;
        }
        if (overlaps) return DQ_ERR_INVALID_ARG;
    }
    return DQ_OK;
}

// ... of the call that clips: the tensors of both sides (in place: outputs only) and the words of the norm.
dq_status check_outputs(const dq_tensor* in, uint32_t in_count, const dq_tensor* out, uint32_t out_count, const dq_clip* clip)
{
    struct Memory {
        Extent* e;
        Place *order, *other;
        uint32_t* runs;
    };
    constexpr uint32_t kFew = 512u;
    Extent few[kFew];
    Place few_places[2u * kFew];
    uint32_t few_runs[kFew + 1u];
    const uint32_t most = in_count + out_count + 3u;
    Memory mem = {few, few_places, few_places + kFew, few_runs};
    if (most > kFew) {
        Place* places = host_scratch<Place>(2u * (size_t)most);
        mem = {host_scratch<Extent>(most), places, places ? places + most : nullptr, host_scratch<uint32_t>(most + 1u)};
        if (!mem.e || !places || !mem.runs) return DQ_ERR_CUDA;
    }
    Extent* e = mem.e;
    uint32_t m = 0u;
    for (uint32_t i = 0; i < in_count; ++i)
        if (in[i].n) e[m++] = extent_of(in[i], false);
    for (uint32_t i = 0; i < out_count; ++i)
        if (out[i].n) e[m++] = extent_of(out[i], true);
    auto word = [&](const void* p, bool written) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p) e[m++] = {at, at + 4u, 4u, 0u, written};
    };
    if (clip) {
        word(clip->norm, false);
        word(clip->out_norm, true);
        word(clip->status_word, true);
    }
    by_address(e, m, mem.order, mem.other, mem.runs);
    return check_overlap(e, mem.order, mem.other, m);
}

// ------------------------------------------------------------------------------------------ tables
// Rows that are not Wide and at least this long are walked one by one, shorter ones element by element (12 M elements clipped,
// fp32 and bf16: rows of 400 45 and 58 us one by one, 43 and 46 by elements; rows of 700 33 and 33).
constexpr uint64_t kLongRow = 512u;

// How a tensor is walked, and how many elements before the first one its tiles begin: where the destination (the source,
// where there is none) is aligned.
struct Walk {
    uint32_t walk, phase;
    uint64_t row, src_stride, dst_stride;
};

Walk flat_walk(const dq_tensor& src, const dq_tensor* dst)
{
    const dq_tensor& to = dst ? *dst : src;
    return {dq::kGradFlat, (uint32_t)(reinterpret_cast<uintptr_t>(to.data) & 15u) >> size_log2(to.dtype), 0u, 0u, 0u};
}

Walk walk_of(const dq_tensor& src, const dq_tensor* dst)
{
    const dq_tensor& to = dst ? *dst : src;
    const uint32_t ss = element_size(src.dtype), ds = element_size(to.dtype);
    const uintptr_t s = reinterpret_cast<uintptr_t>(src.data), d = reinterpret_cast<uintptr_t>(to.data);
    if (!has_rows(src) && !has_rows(to)) return flat_walk(src, dst);
    Walk w = {dq::kGradLoose, 0u, has_rows(src) ? src.row : to.row, 0u, 0u};
    w.src_stride = has_rows(src) ? src.row_stride : w.row;
    w.dst_stride = has_rows(to) ? to.row_stride : w.row;
    if (w.row % 8u == 0u && ((s | d) & 15u) == 0u && w.src_stride * ss % 16u == 0u && w.dst_stride * ds % 16u == 0u)
        w.walk = dq::kGradWide;
    else if (w.row >= kLongRow)
        w.walk = dq::kGradLong;
    return w;
}

uint32_t flat_tiles(uint64_t n, uint32_t phase, uint32_t tile_len)
{
    const uint64_t m = n + phase + tile_len - 1u;
    return m >> 32 ? (uint32_t)(m / tile_len) : (uint32_t)m / tile_len;          // (a division of 64 bits takes twice as long)
}

uint32_t tiles_of(uint64_t n, const Walk& w, uint32_t tile_len)
{
    if (w.walk == dq::kGradLong) return (uint32_t)dq::GradRowTiles((uint32_t)w.row, tile_len).tiles(n / w.row);
    const uint64_t m = n + w.phase + tile_len - 1u;
    return m >> 32 ? (uint32_t)(m / tile_len) : (uint32_t)m / tile_len;
}

uint32_t step_up(uint64_t len)
{
    return (uint32_t)std::max<uint64_t>(1u, (len + dq::kGradTileStep - 1u) / dq::kGradTileStep) * dq::kGradTileStep;
}

// The tiles of the norm's kernel, which runs in one wave: 8 KB, two batches of 16-byte loads of a lane, but 1024 elements where
// that leaves warps without a tile, and more where a warp has more than four of them, which costs it look-ups (n = 124 M
// bf16: 2048 to 16384 elements 40 us; 25.6 M fp32: 2048 19.8 us, 4096 20.8, 1024 21.5; 25.6 M bf16: 4096 13.7, 2048 14.9; 1.7 M
// fp32: 1024 4.1, 2048 4.4).
uint32_t norm_tile_length(const ListInfo& info, int sms)
{
    const uint64_t warps = (uint64_t)sms * dq::kGradNormCtas * dq::kGradWarps;
    if (info.total < warps * 1024u) return 1024u;
    const uint64_t tile = info.bytes < 3u * info.total ? 4096u : 2048u;
    return (uint32_t)(tile * (info.total / (warps * tile * 4u) + 1u));
}

// The tiles of the kernel that scales.  Up to two tiles of 4096 per resident warp it runs in one wave or little more, since every
// CTA begins with the parts of the norm; longer lists run in many short CTAs, which the hardware hands out as others end: 124 M
// fp32 elements 149 us, in one wave of long CTAs 166 (11.7 M: 4096 elements 21.5 us, 2048 23.0; 1.7 M: 1024 7.0 us, 4096 9.0).
uint32_t scale_tile_length(uint64_t total, int sms)
{
    const uint64_t warps = (uint64_t)sms * dq::kGradScaleCtas * dq::kGradWarps;
    return total < warps * 8192u ? std::min(4096u, step_up(total / warps + 1u)) : 2048u;
}
constexpr uint32_t kScaleGrid = 24u;             // CTAs per SM of a launch, resident or not

// The tiles of a cluster: one per warp.
uint32_t cluster_tile_length(uint64_t total, uint32_t count)
{
    const uint32_t warps = dq::kGradCluster * dq::kGradClusterThreads / 32u;
    return step_up(total / (warps - std::min(count, warps / 2u)) + 1u);
}

// What the norm's pass leaves in L2 for the pass that scales, which begins at the end: more than this is read with the policy
// to go first (n = 124 M fp32, 64 MB: 229 us; all kept: 232, none: 237, and with ordinary stores 242).
constexpr uint64_t kKeepBytes = 64ull << 20;

uint32_t entries_of(const dq_tensor& src, const dq_tensor* dst)
{
    return src.n == 0u ? 0u : has_rows(src) || (dst && has_rows(*dst)) ? 2u : 1u;
}

// Fills a table from list position *next on.  first_slot, where given, has a place for every tensor of the list and one more,
// and counts tiles on from what stands at *next.
template <int N, int W>
void fill(dq::GradTable<N, W>& t, const dq_tensor* src, const dq_tensor* dst, uint32_t count, uint32_t tile_len, uint32_t* next,
          uint32_t* first_slot)
{
    const uint32_t slot = first_slot ? first_slot[*next] : 0u;
    uint32_t entries = 0u, tiles = 0u;
    t.rows = 0u;
    for (; *next < count; ++*next) {
        const uint32_t i = *next;
        const dq_tensor& x = src[i];
        const dq_tensor* to = dst ? dst + i : nullptr;
        const bool rows = has_rows(x) || (to && has_rows(*to));
        const uint64_t n = x.n;
        if (n != 0u) {
            if (entries + (rows ? 2u : 1u) > (uint32_t)N) break;
            const uint64_t s = reinterpret_cast<uintptr_t>(x.data);
            const Walk w = rows ? walk_of(x, to) : flat_walk(x, to);
            dq::GradEntry<W>& e = t.e[entries];
            t.first_tile[entries++] = tiles;
            tiles += rows ? tiles_of(n, w, tile_len) : flat_tiles(n, w.phase, tile_len);
            e.w[0] = (uint32_t)s;
            e.w[1] = (uint32_t)(s >> 32) | (uint32_t)x.dtype << 25 | w.walk << 27 | (uint32_t)(n >> 32) << 29;
            e.w[2] = (uint32_t)n;
            if constexpr (W > 3) {
                const uint64_t d = reinterpret_cast<uintptr_t>(to->data);
                e.w[3] = (uint32_t)d;
                e.w[4] = (uint32_t)(d >> 32) | (uint32_t)to->dtype << 25;
            }
            if (rows) {
                t.rows = 1u;
                dq::GradEntry<W>& r = t.e[entries];
                t.first_tile[entries++] = tiles;
                r.w[0] = (uint32_t)w.row;
                r.w[1] = (uint32_t)w.src_stride;
                r.w[2] = (uint32_t)w.dst_stride;
            }
        }
        if (first_slot) first_slot[i + 1u] = slot + tiles;
    }
    t.first_tile[entries] = tiles;
    t.count = entries;
    t.tile_len = tile_len;
    t.stream_below = 0u;
}

uint32_t grid_for(uint32_t tiles, uint32_t warps, uint32_t most)
{
    return std::max(1u, std::min((tiles + warps - 1u) / warps, most));
}

bool entries_fit(const dq_tensor* src, const dq_tensor* dst, uint32_t count, uint32_t most)
{
    uint32_t entries = 0u;
    for (uint32_t i = 0; i < count && entries <= most; ++i) entries += entries_of(src[i], dst ? dst + i : nullptr);
    return entries <= most;
}

// Calls f(table) with the smallest table that holds the rest of the list; there is none larger than MOST entries.
template <int W, int MOST = kLarge<W>, class F>
cudaError_t with_table(const dq_tensor* src, const dq_tensor* dst, uint32_t count, uint32_t tile_len, uint32_t* next,
                       uint32_t* first_slot, F&& f)
{
    const dq_tensor* to = dst ? dst + *next : nullptr;
    if (entries_fit(src + *next, to, count - *next, kSmall<W>)) {
        dq::GradTable<kSmall<W>, W> t;
        fill(t, src, dst, count, tile_len, next, first_slot);
        return f(t);
    }
    if constexpr (MOST > kMiddle<W>) {
        if (!entries_fit(src + *next, to, count - *next, kMiddle<W>)) {
            dq::GradTable<MOST, W> t;
            fill(t, src, dst, count, tile_len, next, first_slot);
            return f(t);
        }
    }
    dq::GradTable<kMiddle<W>, W> t;
    fill(t, src, dst, count, tile_len, next, first_slot);
    return f(t);
}

// A list that one cluster does in one launch.  (A tensor in rows on either side takes two entries of the table.)
bool is_short(uint32_t count, uint64_t total, uint64_t most)
{
    return total == 0u || (total <= most && 2u * (uint64_t)count <= (uint64_t)kMiddle<kScale>);
}

constexpr int kMaxDevices = 64;

// CTAs of the cluster kernels: 16 (which needs an attribute per kernel and device) where one can be resident, else the
// portable 8; 0 on a CUDA error.
template <class Table, bool ROWS, bool MAX, bool SCALE>
uint32_t cluster_size()
{
    static std::mutex mu;
    static uint32_t size[kMaxDevices] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0u;
    std::lock_guard<std::mutex> lock(mu);
    if (size[dev] == 0u) {
        auto kernel = dq::grad_cluster_kernel<Table, ROWS, MAX, SCALE>;
        uint32_t s = 8u;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(dq::kGradCluster);
            cfg.blockDim = dim3(dq::kGradClusterThreads);
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = dq::kGradCluster;
            attr[0].val.clusterDim.y = 1;
            attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            int clusters = 0;
            if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters > 0)
                s = (uint32_t)dq::kGradCluster;
        }
        cudaGetLastError();
        size[dev] = s;
    }
    return size[dev];
}

template <bool ROWS, bool MAX, bool SCALE, class Table>
cudaError_t launch_cluster_of(const Table& t, const dq::ClipArgs& a, cudaStream_t st)
{
    static_assert(Table::kCapacity <= kMiddle<Table::kWords>, "short lists have no larger tables");
    const uint32_t most = cluster_size<Table, ROWS, MAX, SCALE>();
    if (most == 0u) return cudaErrorUnknown;
    // no CTA without a tile for every other warp
    const uint32_t tiles = t.first_tile[t.count];
    uint32_t ctas = 1u;
    while (ctas < most && tiles > ctas * (dq::kGradClusterThreads / 64u)) ctas *= 2u;
    const cudaError_t e = dq::launch_overlapped(dq::grad_cluster_kernel<Table, ROWS, MAX, SCALE>, ctas,
                                                (uint32_t)dq::kGradClusterThreads, 0, st, ctas, t, a);
    if (e == cudaSuccess) dq::count_launch();
    return e;
}

template <bool MAX, bool SCALE, class Table>
cudaError_t launch_cluster(const Table& t, const dq::ClipArgs& a, cudaStream_t st)
{
    return t.rows ? launch_cluster_of<true, MAX, SCALE>(t, a, st) : launch_cluster_of<false, MAX, SCALE>(t, a, st);
}

// The parts of the norm of a list into slots; *num_slots counts them.
template <bool MAX, bool EACH>
cudaError_t launch_parts(const dq_tensor* list, uint32_t count, uint32_t tile_len, int sms, uint64_t keep,
                         dq::NormPart<MAX>* slots, uint32_t* num_slots, uint32_t* first_slot, cudaStream_t st)
{
    *num_slots = 0u;
    for (uint32_t next = 0u; next < count;) {
        const cudaError_t e = with_table<kNorm>(list, nullptr, count, tile_len, &next, first_slot, [&](auto& t) {
            using Table = std::remove_reference_t<decltype(t)>;
            const uint32_t tiles = t.first_tile[t.count];
            if (tiles == 0u) return cudaSuccess;
            const uint64_t kept = keep / tile_len;
            t.stream_below = tiles > kept ? (uint32_t)(tiles - kept) : 0u;
            const uint32_t grid = grid_for(tiles, dq::kGradWarps, std::min((uint32_t)sms * dq::kGradNormCtas, kMaxGrid));
            const cudaError_t r = dq::launch_overlapped(t.rows ? dq::grad_norm_kernel<Table, true, MAX, EACH>
                                                               : dq::grad_norm_kernel<Table, false, MAX, EACH>,
                                                        grid, (uint32_t)dq::kGradThreads, 0, st, 1u, t, slots + *num_slots);
            if (r == cudaSuccess) dq::count_launch();
            *num_slots += EACH ? tiles : grid;
            return r;
        });
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// The whole from its parts, and with a table the norms of its tensors.
template <bool MAX, class Table>
cudaError_t launch_join(const Table& t, const dq::NormPart<MAX>* slots, uint32_t num_slots, float* out_norm, float* out_norms,
                        uint32_t* status, cudaStream_t st)
{
    constexpr uint32_t kPerCta = dq::kGradJoinThreads / 32;
    const cudaError_t e = dq::launch_overlapped(dq::grad_norm_join_kernel<Table, MAX>, 1u + (t.count + kPerCta - 1u) / kPerCta,
                                                (uint32_t)dq::kGradJoinThreads, 0, st, 1u, t, slots, num_slots, out_norm,
                                                out_norms, status);
    if (e == cudaSuccess) dq::count_launch();
    return e;
}

template <bool MAX>
cudaError_t launch_join(const dq::NormPart<MAX>* slots, uint32_t num_slots, float* out_norm, uint32_t* status, cudaStream_t st)
{
    dq::GradEachTable<1> none;
    none.count = 0u;
    return launch_join<MAX>(none, slots, num_slots, out_norm, nullptr, status, st);
}

// The same with the norms of single tensors: tensor i has the slots from first_slot[i] to first_slot[i + 1].
template <bool MAX>
cudaError_t launch_join_each(uint32_t count, const uint32_t* first_slot, const dq::NormPart<MAX>* slots, uint32_t num_slots,
                             float* out_norm, float* out_norms, uint32_t* status, cudaStream_t st)
{
    uint32_t done = 0u;
    auto launch = [&](auto& t) {
        t.count = std::min(count - done, (uint32_t)t.kCapacity);
        std::copy_n(first_slot + done, t.count + 1u, t.first);
        const cudaError_t e = launch_join<MAX>(t, slots, num_slots, done == 0u ? out_norm : nullptr, out_norms + done, status, st);
        done += t.count;
        return e;
    };
    cudaError_t e = cudaSuccess;
    while (done < count && e == cudaSuccess) {
        if (count - done <= (uint32_t)kEachMiddle) {
            dq::GradEachTable<kEachMiddle> t;
            e = launch(t);
        } else {
            dq::GradEachTable<kEachLarge> t;
            e = launch(t);
        }
    }
    return e;
}

template <bool MAX>
dq_status norm_of(const dq_tensor* list, uint32_t count, const ListInfo& info, float* out_norm, float* out_norms,
                  uint32_t* status, void* workspace, cudaStream_t st)
{
    const int sms = dq::device_sm_count();
    if (sms <= 0) return DQ_ERR_CUDA;
    auto* slots = static_cast<dq::NormPart<MAX>*>(workspace);
    uint32_t num_slots = 0u;
    cudaError_t e;
    if (out_norms && count) {
        uint32_t* first_slot = host_scratch<uint32_t>(count + 1u);
        if (!first_slot) return DQ_ERR_CUDA;
        first_slot[0] = 0u;
        // (no more slots than the workspace has)
        const uint32_t tile_len = std::max(norm_tile_length(info, sms), step_up(info.total / kEachTiles + 1u));
        e = launch_parts<MAX, true>(list, count, tile_len, sms, ~0ull, slots, &num_slots, first_slot, st);
        if (e == cudaSuccess)
            e = launch_join_each<MAX>(count, first_slot, slots, num_slots, out_norm, out_norms, status, st);
    } else if (is_short(count, info.total, kShortNorm)) {
        dq::ClipArgs a = {};
        a.out_norm = out_norm;
        a.status = status;
        uint32_t next = 0u;
        e = with_table<kNorm, kMiddle<kNorm>>(list, nullptr, count, cluster_tile_length(info.total, count), &next, nullptr,
                                              [&](const auto& t) { return launch_cluster<MAX, false>(t, a, st); });
    } else {
        e = launch_parts<MAX, false>(list, count, norm_tile_length(info, sms), sms, ~0ull, slots, &num_slots, nullptr, st);
        if (e == cudaSuccess) e = launch_join<MAX>(slots, num_slots, out_norm, status, st);
    }
    return e == cudaSuccess ? DQ_OK : DQ_ERR_CUDA;
}

// A list that is clipped: src[i] * c into dst[i].  The norm is that of norm_list, which is the same elements; `info` is about it.
struct Job {
    const dq_tensor *src, *dst;
    uint32_t count;
    const dq_tensor* norm_list;
    uint32_t norm_count;
    ListInfo info;
    const dq_clip* clip;         // null: nothing is clipped
    bool in_place;
};

template <bool MAX>
dq_status scale(const Job& job, void* workspace, cudaStream_t st)
{
    const int sms = dq::device_sm_count();
    if (sms <= 0) return DQ_ERR_CUDA;
    const dq_tensor *src = job.src, *dst = job.dst;
    const uint32_t count = job.count;
    const ListInfo& info = job.info;
    const dq_clip* clip = job.clip;
    dq::ClipArgs a = {};
    a.in_place = job.in_place ? 1u : 0u;
    a.max_kind = MAX ? 1u : 0u;
    a.max_norm = clip ? clip->max_norm : 0.0f;
    uint32_t next = 0u;
    if (clip) {
        a.norm = clip->norm;
        a.out_norm = clip->out_norm;
        a.status = clip->status_word;
    }
    if (clip && !clip->norm) {
        if (is_short(count, info.total, kShortScale)) {
            const cudaError_t e = with_table<kScale, kMiddle<kScale>>(
                src, dst, count, cluster_tile_length(info.total, count), &next, nullptr,
                [&](const auto& t) { return launch_cluster<MAX, true>(t, a, st); });
            return e == cudaSuccess ? DQ_OK : DQ_ERR_CUDA;
        }
        auto* slots = reinterpret_cast<dq::NormPart<MAX>*>(static_cast<char*>(workspace) + 16);
        const uint64_t keep = info.bytes ? kKeepBytes * info.total / info.bytes : 0u;
        cudaError_t e = launch_parts<MAX, false>(job.norm_list, job.norm_count, norm_tile_length(info, sms), sms, keep, slots,
                                                 &a.num_slots, nullptr, st);
        if (e != cudaSuccess) return DQ_ERR_CUDA;
        a.slots = slots;
        if (!entries_fit(src, dst, count, kLarge<kScale>)) {
            // several launches follow: they take the norm itself
            float* norm = a.out_norm ? a.out_norm : static_cast<float*>(workspace);
            if (launch_join<MAX>(slots, a.num_slots, norm, a.status, st) != cudaSuccess) return DQ_ERR_CUDA;
            a.norm = norm;
            a.norm_in_workspace = a.out_norm ? 0u : 1u;
            a.num_slots = 0u;
            a.out_norm = nullptr;
            a.status = nullptr;
        }
    }
    const uint32_t tile_len = scale_tile_length(info.total, sms);
    bool first = true;
    while (next < count || first) {
        const cudaError_t e = with_table<kScale>(src, dst, count, tile_len, &next, nullptr, [&](const auto& t) {
            using Table = std::remove_cv_t<std::remove_reference_t<decltype(t)>>;
            const uint32_t tiles = t.first_tile[t.count];
            if (tiles == 0u && !(first && (a.out_norm || a.status))) return cudaSuccess;
            const cudaError_t r = dq::launch_overlapped(t.rows ? dq::grad_scale_kernel<Table, true>
                                                               : dq::grad_scale_kernel<Table, false>, grid_for(tiles, dq::kGradWarps, (uint32_t)sms * kScaleGrid),
                                                        (uint32_t)dq::kGradThreads, 0, st, 1u, t, a);
            if (r == cudaSuccess) dq::count_launch();
            return r;
        });
        if (e != cudaSuccess) return DQ_ERR_CUDA;
        first = false;
        a.out_norm = nullptr;        // (reported once)
        a.status = nullptr;
    }
    return DQ_OK;
}

dq_status check_clip(const dq_clip* clip)
{
    if (!(clip->max_norm >= 0.0f)) return DQ_ERR_INVALID_ARG;
    if (clip->kind != DQ_NORM_L2 && clip->kind != DQ_NORM_MAX) return DQ_ERR_INVALID_ARG;
    for (const void* p : {(const void*)clip->norm, (const void*)clip->out_norm, (const void*)clip->status_word})
        if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0u) return DQ_ERR_ALIGNMENT;
    return DQ_OK;
}

uint64_t workspace_bytes_for(uint32_t count, const ListInfo& info, bool each)
{
    if (info.total == 0u || (!each && is_short(count, info.total, std::min(kShortNorm, kShortScale)))) return 0u;
    // (tiles of a tensor in rows may be half as long, and every tensor may have two that are short)
    const uint64_t slots = each ? 2u * kEachTiles + kEachTiles / 8u + 2u * (uint64_t)count
                                : (uint64_t)kMaxGrid * (2u * (uint64_t)count / (uint64_t)(kLarge<kNorm> - 1) + 1u);
    return (16u + 8u * slots + 255u) / 256u * 256u;
}

dq_status check_workspace(uint64_t need, const void* workspace, uint64_t bytes)
{
    if (need == 0u) return DQ_OK;
    if (!workspace || bytes < need) return DQ_ERR_INVALID_ARG;
    return (reinterpret_cast<uintptr_t>(workspace) & 15u) == 0u ? DQ_OK : DQ_ERR_ALIGNMENT;
}

// The last check and the launch that clip, gather and scatter share.
dq_status scale_checked(const Job& job, void* workspace, uint64_t workspace_bytes, cudaStream_t st)
{
    if (job.clip && !job.clip->norm) {
        const dq_status s = check_workspace(workspace_bytes_for(job.count, job.info, false), workspace, workspace_bytes);
        if (s != DQ_OK) return s;
    }
    return job.clip && job.clip->kind == DQ_NORM_MAX ? scale<true>(job, workspace, st) : scale<false>(job, workspace, st);
}

// The slices of a flat vector that belong to the tensors of a list.
struct Slices {
    static constexpr uint32_t kFew = 256u;
    dq_tensor few[kFew];
    dq_tensor* t = few;

    bool cut(const float* flat, const dq_tensor* list, uint32_t count)
    {
        if (count > kFew) {
            t = host_scratch<dq_tensor>(count);
            if (!t) return false;
        }
        for (uint32_t i = 0; i < count; ++i) {
            t[i] = {const_cast<float*>(flat), list[i].n, 0u, 0u, DQ_F32, 0u};
            flat += list[i].n;
        }
        return true;
    }
};

}  // namespace

extern "C" {

uint64_t dq_grad_workspace_bytes(const dq_tensor* list, uint32_t count, int each)
{
    ListInfo info;
    return check_list(list, count, &info) == DQ_OK ? workspace_bytes_for(count, info, each != 0) : 0u;
}

dq_status dq_grad_norm(const dq_tensor* grads, uint32_t count, dq_norm kind, float* out_norm, float* out_norms,
                       uint32_t* status_word, void* workspace, uint64_t workspace_bytes, void* cuda_stream)
{
    ListInfo info;
    dq_status s = check_list(grads, count, &info);
    if (s != DQ_OK) return s;
    if (!out_norm || (kind != DQ_NORM_L2 && kind != DQ_NORM_MAX)) return DQ_ERR_INVALID_ARG;
    for (const void* p : {(const void*)out_norm, (const void*)out_norms, (const void*)status_word})
        if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0u) return DQ_ERR_ALIGNMENT;
    s = check_workspace(workspace_bytes_for(count, info, out_norms != nullptr), workspace, workspace_bytes);
    if (s != DQ_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return kind == DQ_NORM_MAX ? norm_of<true>(grads, count, info, out_norm, out_norms, status_word, workspace, st)
                               : norm_of<false>(grads, count, info, out_norm, out_norms, status_word, workspace, st);
}

dq_status dq_grad_clip(const dq_tensor* grads, uint32_t count, const dq_clip* clip, const dq_tensor* out, void* workspace,
                       uint64_t workspace_bytes, void* cuda_stream)
{
    ListInfo info, out_info;
    dq_status s = check_list(grads, count, &info);
    if (s != DQ_OK) return s;
    if (!clip) return DQ_ERR_INVALID_ARG;
    s = check_clip(clip);
    if (s != DQ_OK) return s;
    if (out) {
        s = check_list(out, count, &out_info);
        if (s != DQ_OK) return s;
        for (uint32_t i = 0; i < count; ++i) {
            if (out[i].n != grads[i].n) return DQ_ERR_INVALID_ARG;
            if (has_rows(out[i]) && has_rows(grads[i]) && out[i].row != grads[i].row) return DQ_ERR_UNSUPPORTED;
        }
    }
    s = out ? check_outputs(grads, count, out, count, clip) : check_outputs(nullptr, 0u, grads, count, clip);
    if (s != DQ_OK) return s;
    return scale_checked({grads, out ? out : grads, count, grads, count, info, clip, out == nullptr}, workspace, workspace_bytes,
                         static_cast<cudaStream_t>(cuda_stream));
}

dq_status dq_grad_gather(const dq_tensor* grads, uint32_t count, const dq_clip* clip, float* out_flat, void* workspace,
                         uint64_t workspace_bytes, void* cuda_stream)
{
    ListInfo info;
    dq_status s = check_list(grads, count, &info);
    if (s != DQ_OK) return s;
    if (clip && (s = check_clip(clip)) != DQ_OK) return s;
    if (info.total != 0u && !out_flat) return DQ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(out_flat) & 15u) != 0u) return DQ_ERR_ALIGNMENT;
    const dq_tensor flat = {out_flat, info.total, 0u, 0u, DQ_F32, 0u};
    s = check_outputs(grads, count, &flat, 1u, clip);
    if (s != DQ_OK) return s;
    Slices to;
    if (!to.cut(out_flat, grads, count)) return DQ_ERR_CUDA;
    return scale_checked({grads, to.t, count, grads, count, info, clip, false}, workspace, workspace_bytes,
                         static_cast<cudaStream_t>(cuda_stream));
}

dq_status dq_grad_scatter(const float* flat, const dq_clip* clip, const dq_tensor* out, uint32_t count, void* workspace,
                          uint64_t workspace_bytes, void* cuda_stream)
{
    ListInfo info;
    dq_status s = check_list(out, count, &info);
    if (s != DQ_OK) return s;
    if (clip && (s = check_clip(clip)) != DQ_OK) return s;
    if (info.total != 0u && !flat) return DQ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(flat) & 15u) != 0u) return DQ_ERR_ALIGNMENT;
    const dq_tensor whole = {const_cast<float*>(flat), info.total, 0u, 0u, DQ_F32, 0u};
    s = check_outputs(&whole, 1u, out, count, clip);
    if (s != DQ_OK) return s;
    Slices from;
    if (!from.cut(flat, out, count)) return DQ_ERR_CUDA;
    info.bytes = 4u * info.total;
    return scale_checked({from.t, out, count, &whole, 1u, info, clip, false}, workspace, workspace_bytes,
                         static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
