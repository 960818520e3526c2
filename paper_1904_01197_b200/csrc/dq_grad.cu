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

using dq::GradEntry;
using dq::GradTable;

// Tables of three sizes: a launch passes them by value, and 32 KB more of parameters cost it about a microsecond.
constexpr int kSmall = 16, kMiddle = 160, kLarge = 620;
static_assert(sizeof(GradTable<kLarge>) + sizeof(dq::ClipArgs) <= 32764, "kernel parameters");
static_assert(sizeof(dq::GradEachTable) + 16 <= 32764, "kernel parameters");

// Lists up to this many elements (and kMiddle tensors) are done by one cluster in one launch.
constexpr uint64_t kShortElements = 1ull << 19;

// Parts of the norm: at most kMaxGrid of a launch, or one per tile where each tensor's norm is wanted as well.
constexpr uint32_t kMaxGrid = 2048u;
constexpr uint64_t kEachTiles = 16384u;

uint32_t element_size(uint32_t dtype) { return dtype == DQ_F32 ? 4u : 2u; }

bool has_rows(const dq_tensor& t) { return t.row != 0u && t.row_stride != t.row && t.row != t.n; }

dq_status check_tensor(const dq_tensor& t)
{
    if ((uint32_t)t.dtype > (uint32_t)DQ_F16 || t.reserved != 0u) return DQ_ERR_INVALID_ARG;
    if (t.n == 0u) return DQ_OK;
    if (!t.data) return DQ_ERR_INVALID_ARG;
    if (t.n >= (1ull << 34)) return DQ_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(t.data) % element_size(t.dtype) != 0u) return DQ_ERR_ALIGNMENT;
    if (t.row != 0u) {
        if (t.n % t.row != 0u || t.row_stride < t.row) return DQ_ERR_INVALID_ARG;
        if (has_rows(t) && (t.row >= (1ull << 31) || t.row_stride >= (1ull << 32))) return DQ_ERR_UNSUPPORTED;
    }
    return DQ_OK;
}

dq_status check_list(const dq_tensor* list, uint32_t count, uint64_t* total)
{
    *total = 0u;
    if (count > DQ_MAX_TENSORS) return DQ_ERR_UNSUPPORTED;
    if (count != 0u && !list) return DQ_ERR_INVALID_ARG;
    for (uint32_t i = 0; i < count; ++i) {
        const dq_status s = check_tensor(list[i]);
        if (s != DQ_OK) return s;
        *total += list[i].n;
        if (*total >= (1ull << 34)) return DQ_ERR_UNSUPPORTED;
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

// DQ_ERR_INVALID_ARG where an output overlaps another tensor.
dq_status check_overlap(Extent* e, uint32_t count)
{
    auto before = [](const Extent& a, const Extent& b) { return a.lo < b.lo; };
    if (!std::is_sorted(e, e + count, before)) std::sort(e, e + count, before);
    uint32_t group = 0u;         // the first extent of those that reach, one over another, to the current one
    uintptr_t reach = 0u;
    for (uint32_t i = 0; i < count; ++i) {
        if (e[i].lo >= reach) group = i;
        for (uint32_t k = group; k < i; ++k)
            if ((e[i].out || e[k].out) && e[k].hi > e[i].lo && rows_overlap(e[k], e[i])) return DQ_ERR_INVALID_ARG;
        reach = std::max(reach, e[i].hi);
    }
    return DQ_OK;
}

// ... of the call that clips: the tensors of both sides (in place: outputs only) and the words of the norm.
dq_status check_outputs(const dq_tensor* in, uint32_t in_count, const dq_tensor* out, uint32_t out_count, const dq_clip* clip)
{
    constexpr uint32_t kFew = 512u;
    Extent few[kFew];
    std::unique_ptr<Extent[]> many;
    Extent* e = few;
    if (in_count + out_count + 3u > kFew) {
        many.reset(new (std::nothrow) Extent[in_count + out_count + 3u]);
        if (!many) return DQ_ERR_CUDA;
        e = many.get();
    }
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
    return check_overlap(e, m);
}

// ------------------------------------------------------------------------------------------ tables
// The walk of one tensor.  src alone: `dst` null.
GradEntry entry_of(const dq_tensor& src, const dq_tensor* dst)
{
    GradEntry e = {};
    const dq_tensor& to = dst ? *dst : src;
    const uint32_t ss = element_size(src.dtype), ds = element_size(to.dtype);
    const uintptr_t s = reinterpret_cast<uintptr_t>(src.data), d = reinterpret_cast<uintptr_t>(to.data);
    e.src = src.data;
    e.dst = to.data;
    e.n = src.n;
    if (!has_rows(src) && !has_rows(to)) {
        // groups begin where the destination (the source, where there is none) is aligned
        const uint32_t phase = (uint32_t)(d / ds % (16u / ds));
        const uint32_t shift = (uint32_t)((s - phase * ss) & 15u);
        e.form = dq::grad_form(src.dtype, to.dtype, dq::kGradFlat, phase, shift);
        return e;
    }
    e.row = (uint32_t)(has_rows(src) ? src.row : to.row);
    e.src_stride = has_rows(src) ? (uint32_t)src.row_stride : e.row;
    e.dst_stride = has_rows(to) ? (uint32_t)to.row_stride : e.row;
    const bool wide = e.row % 8u == 0u && ((s | d) & 15u) == 0u && (uint64_t)e.src_stride * ss % 16u == 0u &&
                      (uint64_t)e.dst_stride * ds % 16u == 0u;
    e.form = dq::grad_form(src.dtype, to.dtype, wide ? dq::kGradRows : dq::kGradLoose, 0u, 0u);
    return e;
}

uint32_t tiles_of(const GradEntry& e, uint32_t tile_log2)
{
    return (uint32_t)((e.n + ((e.form >> 8) & 15u) + (1ull << tile_log2) - 1u) >> tile_log2);
}

// Fills a table from list position *next on; first[i], where given, is the first slot of tensor i.
template <int N>
void fill(GradTable<N>& t, const dq_tensor* src, const dq_tensor* dst, uint32_t count, uint32_t tile_log2, uint32_t* next)
{
    t.count = 0u;
    t.tile_log2 = tile_log2;
    uint32_t tiles = 0u;
    while (*next < count && t.count < (uint32_t)N) {
        const uint32_t i = (*next)++;
        if (src[i].n == 0u) continue;
        const GradEntry e = entry_of(src[i], dst ? dst + i : nullptr);
        t.first_tile[t.count] = tiles;
        t.e[t.count++] = e;
        tiles += tiles_of(e, tile_log2);
    }
    t.first_tile[t.count] = tiles;
}

uint32_t grid_for(uint32_t tiles, int sms, uint32_t ctas_per_sm)
{
    const uint32_t most = std::min((uint32_t)sms * ctas_per_sm, kMaxGrid);
    return std::max(1u, std::min((tiles + dq::kGradWarps - 1u) / dq::kGradWarps, most));
}

// Calls f(table) with the smallest table that holds the rest of the list.
template <class F>
cudaError_t with_table(const dq_tensor* src, const dq_tensor* dst, uint32_t count, uint32_t tile_log2, uint32_t* next, F&& f)
{
    uint32_t left = 0u;
    for (uint32_t i = *next; i < count && left <= (uint32_t)kMiddle; ++i) left += src[i].n != 0u;
    if (left <= (uint32_t)kSmall) {
        GradTable<kSmall> t;
        fill(t, src, dst, count, tile_log2, next);
        return f(t);
    }
    if (left <= (uint32_t)kMiddle) {
        GradTable<kMiddle> t;
        fill(t, src, dst, count, tile_log2, next);
        return f(t);
    }
    GradTable<kLarge> t;
    fill(t, src, dst, count, tile_log2, next);
    return f(t);
}

bool is_short(const dq_tensor* list, uint32_t count, uint64_t total)
{
    if (total > kShortElements) return false;
    uint32_t tensors = 0u;
    for (uint32_t i = 0; i < count; ++i) tensors += list[i].n != 0u;
    return tensors <= (uint32_t)kMiddle;
}

constexpr int kMaxDevices = 64;

// CTAs of the cluster kernels: 16 (which needs an attribute per kernel and device) where one can be resident, else the
// portable 8; 0 on a CUDA error.
template <class Table, bool MAX, bool SCALE>
uint32_t cluster_size()
{
    static std::mutex mu;
    static uint32_t size[kMaxDevices] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0u;
    std::lock_guard<std::mutex> lock(mu);
    if (size[dev] == 0u) {
        auto kernel = dq::grad_cluster_kernel<Table, MAX, SCALE>;
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

template <bool MAX, bool SCALE, class Table>
cudaError_t launch_cluster(const Table& t, const dq::ClipArgs& a, cudaStream_t st)
{
    const uint32_t most = cluster_size<Table, MAX, SCALE>();
    if (most == 0u) return cudaErrorUnknown;
    // no CTA without a tile for every other warp
    const uint32_t tiles = t.first_tile[t.count];
    uint32_t ctas = 1u;
    while (ctas < most && tiles > ctas * (dq::kGradClusterThreads / 64u)) ctas *= 2u;
    const cudaError_t e = dq::launch_overlapped(dq::grad_cluster_kernel<Table, MAX, SCALE>, ctas,
                                                (uint32_t)dq::kGradClusterThreads, 0, st, ctas, t, a);
    if (e == cudaSuccess) dq::count_launch();
    return e;
}

// The parts of the norm of a list into slots; *num_slots counts them.
template <bool MAX, bool EACH>
cudaError_t launch_parts(const dq_tensor* list, uint32_t count, uint32_t tile_log2, int sms, dq::NormPart<MAX>* slots,
                         uint32_t* num_slots, cudaStream_t st)
{
    *num_slots = 0u;
    for (uint32_t next = 0u; next < count;) {
        const cudaError_t e = with_table(list, nullptr, count, tile_log2, &next, [&](const auto& t) {
            using Table = std::remove_cv_t<std::remove_reference_t<decltype(t)>>;
            const uint32_t tiles = t.first_tile[t.count];
            if (tiles == 0u) return cudaSuccess;
            const uint32_t grid = grid_for(tiles, sms, 8u);
            const cudaError_t r = dq::launch_overlapped(dq::grad_norm_kernel<Table, MAX, EACH>, grid,
                                                        (uint32_t)dq::kGradThreads, 0, st, 1u, t, slots + *num_slots);
            if (r == cudaSuccess) dq::count_launch();
            *num_slots += EACH ? tiles : grid;
            return r;
        });
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <bool MAX>
cudaError_t launch_join(const dq::NormPart<MAX>* slots, uint32_t num_slots, float* out_norm, uint32_t* status, cudaStream_t st)
{
    const cudaError_t e = dq::launch_overlapped(dq::grad_norm_join_kernel<MAX>, 1u, (uint32_t)dq::kGradJoinThreads, 0, st, 1u,
                                                slots, num_slots, out_norm, status);
    if (e == cudaSuccess) dq::count_launch();
    return e;
}

// The norms of single tensors, after launch_parts<MAX, true>.
template <bool MAX>
cudaError_t launch_each(const dq_tensor* list, uint32_t count, uint32_t tile_log2, const dq::NormPart<MAX>* slots,
                        float* out_norms, cudaStream_t st)
{
    uint32_t slot = 0u;
    for (uint32_t i = 0u; i < count;) {
        dq::GradEachTable t;
        const uint32_t begin = i;
        t.count = 0u;
        t.first[0] = slot;
        for (; i < count && t.count < (uint32_t)dq::kGradEachCapacity; ++i) {
            if (list[i].n) slot += tiles_of(entry_of(list[i], nullptr), tile_log2);
            t.first[++t.count] = slot;
        }
        const cudaError_t e = dq::launch_overlapped(dq::grad_norms_each_kernel<MAX>,
                                                    (t.count + dq::kGradWarps - 1u) / dq::kGradWarps,
                                                    (uint32_t)dq::kGradThreads, 0, st, 1u, t, slots, out_norms + begin);
        if (e != cudaSuccess) return e;
        dq::count_launch();
    }
    return cudaSuccess;
}

template <bool MAX>
dq_status norm_of(const dq_tensor* list, uint32_t count, uint64_t total, float* out_norm, float* out_norms, uint32_t* status,
                  void* workspace, cudaStream_t st)
{
    const int sms = dq::device_sm_count();
    if (sms <= 0) return DQ_ERR_CUDA;
    auto* slots = static_cast<dq::NormPart<MAX>*>(workspace);
    uint32_t num_slots = 0u, tile_log2 = dq::kGradTileLog2;
    cudaError_t e;
    if (out_norms && count) {
        while ((total >> tile_log2) > kEachTiles) ++tile_log2;
        e = launch_parts<MAX, true>(list, count, tile_log2, sms, slots, &num_slots, st);
        if (e == cudaSuccess) e = launch_each<MAX>(list, count, tile_log2, slots, out_norms, st);
        if (e == cudaSuccess) e = launch_join<MAX>(slots, num_slots, out_norm, status, st);
    } else if (is_short(list, count, total)) {
        dq::ClipArgs a = {};
        a.out_norm = out_norm;
        a.status = status;
        uint32_t next = 0u;
        e = with_table(list, nullptr, count, tile_log2, &next,
                       [&](const auto& t) { return launch_cluster<MAX, false>(t, a, st); });
    } else {
        e = launch_parts<MAX, false>(list, count, tile_log2, sms, slots, &num_slots, st);
        if (e == cudaSuccess) e = launch_join<MAX>(slots, num_slots, out_norm, status, st);
    }
    return e == cudaSuccess ? DQ_OK : DQ_ERR_CUDA;
}

// src[i] * c into dst[i]; the norm is that of norm_list, which is the same elements.
template <bool MAX>
dq_status scale(const dq_tensor* src, const dq_tensor* dst, uint32_t count, uint64_t total, const dq_tensor* norm_list,
                uint32_t norm_count, const dq_clip* clip, bool in_place, void* workspace, cudaStream_t st)
{
    const int sms = dq::device_sm_count();
    if (sms <= 0) return DQ_ERR_CUDA;
    dq::ClipArgs a = {};
    a.in_place = in_place ? 1u : 0u;
    a.max_norm = clip ? clip->max_norm : 0.0f;
    uint32_t next = 0u, tile_log2 = dq::kGradTileLog2;
    if (clip) {
        a.norm = clip->norm;
        a.out_norm = clip->out_norm;
        a.status = clip->status_word;
    }
    if (clip && !clip->norm) {
        if (is_short(src, count, total)) {
            const cudaError_t e = with_table(src, dst, count, tile_log2, &next,
                                             [&](const auto& t) { return launch_cluster<MAX, true>(t, a, st); });
            return e == cudaSuccess ? DQ_OK : DQ_ERR_CUDA;
        }
        auto* slots = reinterpret_cast<dq::NormPart<MAX>*>(static_cast<char*>(workspace) + 16);
        cudaError_t e = launch_parts<MAX, false>(norm_list, norm_count, tile_log2, sms, slots, &a.num_slots, st);
        if (e != cudaSuccess) return DQ_ERR_CUDA;
        a.slots = slots;
        uint32_t tensors = 0u;
        for (uint32_t i = 0; i < count; ++i) tensors += src[i].n != 0u;
        if (tensors > (uint32_t)kLarge) {
            // several launches follow: they take the norm itself
            float* norm = a.out_norm ? a.out_norm : static_cast<float*>(workspace);
            if (launch_join<MAX>(slots, a.num_slots, norm, a.status, st) != cudaSuccess) return DQ_ERR_CUDA;
            a.norm = norm;
            a.num_slots = 0u;
            a.out_norm = nullptr;
            a.status = nullptr;
        }
    }
    bool first = true;
    while (next < count || first) {
        const cudaError_t e = with_table(src, dst, count, tile_log2, &next, [&](const auto& t) {
            using Table = std::remove_cv_t<std::remove_reference_t<decltype(t)>>;
            const uint32_t tiles = t.first_tile[t.count];
            if (tiles == 0u && !(first && (a.out_norm || a.status))) return cudaSuccess;
            const cudaError_t r = dq::launch_overlapped(dq::grad_scale_kernel<Table, MAX>, grid_for(tiles, sms, 8u),
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

dq_status check_workspace(const dq_tensor* list, uint32_t count, int each, const void* workspace, uint64_t bytes)
{
    const uint64_t need = dq_grad_workspace_bytes(list, count, each);
    if (need == 0u) return DQ_OK;
    if (!workspace || bytes < need) return DQ_ERR_INVALID_ARG;
    return (reinterpret_cast<uintptr_t>(workspace) & 15u) == 0u ? DQ_OK : DQ_ERR_ALIGNMENT;
}

// The checks and the launch that clip, gather and scatter share.  `list` is the list of tensors (the other side of gather
// and scatter is `flat`, cut into tensors of the list's sizes).
dq_status scale_checked(const dq_tensor* src, const dq_tensor* dst, uint32_t count, uint64_t total, const dq_tensor* list,
                        const dq_tensor* norm_list, uint32_t norm_count, const dq_clip* clip, bool in_place, void* workspace,
                        uint64_t workspace_bytes, cudaStream_t st)
{
    if (clip && !clip->norm) {
        const dq_status s = check_workspace(list, count, 0, workspace, workspace_bytes);
        if (s != DQ_OK) return s;
    }
    if (clip && clip->kind == DQ_NORM_MAX)
        return scale<true>(src, dst, count, total, norm_list, norm_count, clip, in_place, workspace, st);
    return scale<false>(src, dst, count, total, norm_list, norm_count, clip, in_place, workspace, st);
}

// The slices of a flat vector that belong to the tensors of a list.
struct Slices {
    static constexpr uint32_t kFew = 256u;
    dq_tensor few[kFew];
    std::unique_ptr<dq_tensor[]> many;
    dq_tensor* t = few;

    bool cut(const float* flat, const dq_tensor* list, uint32_t count)
    {
        if (count > kFew) {
            many.reset(new (std::nothrow) dq_tensor[count]);
            if (!many) return false;
            t = many.get();
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
    uint64_t total;
    if (check_list(list, count, &total) != DQ_OK || (!each && is_short(list, count, total))) return 0u;
    const uint64_t slots = each ? kEachTiles + 2u * (uint64_t)count
                                : (uint64_t)kMaxGrid * ((count + (uint32_t)kLarge - 1u) / (uint32_t)kLarge);
    return (16u + 8u * slots + 255u) / 256u * 256u;
}

dq_status dq_grad_norm(const dq_tensor* grads, uint32_t count, dq_norm kind, float* out_norm, float* out_norms,
                       uint32_t* status_word, void* workspace, uint64_t workspace_bytes, void* cuda_stream)
{
    uint64_t total;
    dq_status s = check_list(grads, count, &total);
    if (s != DQ_OK) return s;
    if (!out_norm || (kind != DQ_NORM_L2 && kind != DQ_NORM_MAX)) return DQ_ERR_INVALID_ARG;
    for (const void* p : {(const void*)out_norm, (const void*)out_norms, (const void*)status_word})
        if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0u) return DQ_ERR_ALIGNMENT;
    s = check_workspace(grads, count, out_norms != nullptr, workspace, workspace_bytes);
    if (s != DQ_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return kind == DQ_NORM_MAX ? norm_of<true>(grads, count, total, out_norm, out_norms, status_word, workspace, st)
                               : norm_of<false>(grads, count, total, out_norm, out_norms, status_word, workspace, st);
}

dq_status dq_grad_clip(const dq_tensor* grads, uint32_t count, const dq_clip* clip, const dq_tensor* out, void* workspace,
                       uint64_t workspace_bytes, void* cuda_stream)
{
    uint64_t total, out_total;
    dq_status s = check_list(grads, count, &total);
    if (s != DQ_OK) return s;
    if (!clip) return DQ_ERR_INVALID_ARG;
    s = check_clip(clip);
    if (s != DQ_OK) return s;
    if (out) {
        s = check_list(out, count, &out_total);
        if (s != DQ_OK) return s;
        for (uint32_t i = 0; i < count; ++i) {
            if (out[i].n != grads[i].n) return DQ_ERR_INVALID_ARG;
            if (has_rows(out[i]) && has_rows(grads[i]) && out[i].row != grads[i].row) return DQ_ERR_UNSUPPORTED;
        }
    }
    s = out ? check_outputs(grads, count, out, count, clip) : check_outputs(nullptr, 0u, grads, count, clip);
    if (s != DQ_OK) return s;
    return scale_checked(grads, out ? out : grads, count, total, grads, grads, count, clip, out == nullptr, workspace,
                         workspace_bytes, static_cast<cudaStream_t>(cuda_stream));
}

dq_status dq_grad_gather(const dq_tensor* grads, uint32_t count, const dq_clip* clip, float* out_flat, void* workspace,
                         uint64_t workspace_bytes, void* cuda_stream)
{
    uint64_t total;
    dq_status s = check_list(grads, count, &total);
    if (s != DQ_OK) return s;
    if (clip && (s = check_clip(clip)) != DQ_OK) return s;
    if (total != 0u && !out_flat) return DQ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(out_flat) & 15u) != 0u) return DQ_ERR_ALIGNMENT;
    const dq_tensor flat = {out_flat, total, 0u, 0u, DQ_F32, 0u};
    s = check_outputs(grads, count, &flat, 1u, clip);
    if (s != DQ_OK) return s;
    Slices to;
    if (!to.cut(out_flat, grads, count)) return DQ_ERR_CUDA;
    return scale_checked(grads, to.t, count, total, grads, grads, count, clip, false, workspace, workspace_bytes,
                         static_cast<cudaStream_t>(cuda_stream));
}

dq_status dq_grad_scatter(const float* flat, const dq_clip* clip, const dq_tensor* out, uint32_t count, void* workspace,
                          uint64_t workspace_bytes, void* cuda_stream)
{
    uint64_t total;
    dq_status s = check_list(out, count, &total);
    if (s != DQ_OK) return s;
    if (clip && (s = check_clip(clip)) != DQ_OK) return s;
    if (total != 0u && !flat) return DQ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(flat) & 15u) != 0u) return DQ_ERR_ALIGNMENT;
    const dq_tensor whole = {const_cast<float*>(flat), total, 0u, 0u, DQ_F32, 0u};
    s = check_outputs(&whole, 1u, out, count, clip);
    if (s != DQ_OK) return s;
    Slices from;
    if (!from.cut(flat, out, count)) return DQ_ERR_CUDA;
    return scale_checked(from.t, out, count, total, out, &whole, 1u, clip, false, workspace, workspace_bytes,
                         static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
