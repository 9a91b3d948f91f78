// sg_evict: cuts paged sets to a budget by accumulated weight.
//
// Select: one workgroup of 1024 threads per unit ranks the unit's rows like
// sg_topk (select_common.h; guarded rows carry the highest key of all) into an
// ascending list of the k kept rows.  The list splits at row k: its first c
// entries stay where they are, the other k - c move, and they fill the k - c
// rows below k that are missing from the first part.  Hole i is i + j for the
// smallest j with list[j] - j > i (list[j] - j rows are missing before list[j],
// a non-decreasing count), one binary search per hole.  Sources lie at or past
// k and destinations below it, so the moves need no order among themselves.
//
// Move: K and V rows (and scales) of the listed moves, 16 bytes per lane.
#include "select_common.h"

namespace sg {

constexpr int MOVE_THREADS = 256;
constexpr int MOVE_UNROLL = 4;

// Key of a guarded row: above that of every weight (+inf has 0xff800000), and
// not the largest word (the select looks at keys above its threshold).
constexpr uint32_t GUARD_KEY = 0xff800001u;

constexpr int evict_waves(int items) { return items <= 32 ? 8 : 4; }

// Workspace: int2 moves [units][cap / 2] (pool rows: to, from), int32 list
// [units][cap], int32 counts [units].
template <int ITEMS>
__global__ __launch_bounds__(TOPK_THREADS) __attribute__((amdgpu_waves_per_eu(evict_waves(ITEMS)))) void evict_select_kernel(
    int64_t pool_rows, const int32_t *__restrict__ page_table, const int32_t *n_rows, int page_size, int max_pages,
    const int32_t *__restrict__ budget, const float *weight, const int32_t *pos, int64_t stride, int sinks,
    const int32_t *__restrict__ recent_from, int32_t *n_kept, float *weight_out, int32_t *pos_out,
    int2 *__restrict__ moves, int32_t *list_all, int32_t *__restrict__ counts) {
    __shared__ SelectSmem sm;
    const int64_t unit = blockIdx.x;
    const int tid = threadIdx.x, cap = max_pages * page_size;
    const int n = min(max((int)n_rows[unit], 0), cap);
    const int k = min(max((int)budget[unit], 0), n);
    const float *w = weight + unit * stride;
    const int32_t *ps = pos ? pos + unit * stride : nullptr;
    float *wo = weight_out + unit * stride;
    int32_t *po = pos_out ? pos_out + unit * stride : nullptr;
    int32_t *list = list_all + unit * cap;
    const int32_t *pt = page_table + unit * max_pages;
    int c = k, m = 0;           // kept rows that stay, that move
    if (k > 0 && k < n) {
        const int32_t recent = recent_from ? recent_from[unit] : 0x7fffffff;
        const int it = select_items(n), entry0 = select_entry(it);
        uint32_t key[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            key[i] = 0u;
            if (i < it) {
                const int row = entry0 + i * 64, at = min(row, n - 1);
                const float x = w[at];
                const int32_t p = ps ? ps[at] : at;
                const bool guard = p < sinks || (recent_from && p >= recent);
                if (row < n) key[i] = guard ? GUARD_KEY : order_key(x);
            }
        }
        select_top<ITEMS>(key, it, k, list, sm);
        __syncthreads();        // the list is read by other threads than wrote it
        int lo = 0, hi = k;     // entries below k
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (list[mid] < k) lo = mid + 1;
            else hi = mid;
        }
        c = lo;
        m = k - c;
    }
    for (int i = tid; i < c; i += TOPK_THREADS) {
        const int row = k < n ? list[i] : i;
        if (wo != w) wo[row] = w[row];
        if (po && po != ps) po[row] = ps[row];
    }
    auto pool_row = [&](int row) -> int {
        const int64_t x = (int64_t)pt[row / page_size] + row % page_size;
        return x >= 0 && x < pool_rows ? (int)x : -1;
    };
    for (int i = tid; i < m; i += TOPK_THREADS) {
        int lo = 0, hi = c;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (list[mid] - mid > i) hi = mid;
            else lo = mid + 1;
        }
        const int to = i + lo, from = list[c + i];
        const int pr_to = pool_row(to), pr_from = pool_row(from);
        moves[unit * (cap / 2) + i] = pr_to >= 0 && pr_from >= 0 ? make_int2(pr_to, pr_from) : make_int2(-1, -1);
        wo[to] = w[from];
        if (po) po[to] = ps[from];
    }
    __syncthreads();            // every weight that moves has been read
    for (int i = k + tid; i < n; i += TOPK_THREADS) {
        wo[i] = 0.f;
        if (po) po[i] = -1;
    }
    if (tid == 0) {
        counts[unit] = m;
        n_kept[unit] = k;
    }
}

// CPR: 16-byte vectors per K (or V) row; SB: bytes of a row's scales.
template <int CPR, int SB>
__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(int cap, const int2 *__restrict__ moves,
                                                                  const int32_t *__restrict__ counts, v4u *k_pool,
                                                                  v4u *v_pool, uint8_t *s_pool) {
    constexpr int EPI = MOVE_THREADS / CPR, EPB = EPI * MOVE_UNROLL;
    const int64_t unit = blockIdx.x;
    const int m = counts[unit];
    const int2 *mv = moves + unit * (cap / 2);
    const int c = threadIdx.x % CPR, sub = threadIdx.x / CPR;
    for (int base = blockIdx.y * EPB; base < m; base += (int)gridDim.y * EPB) {
        int2 e[MOVE_UNROLL];
#pragma unroll
        for (int j = 0; j < MOVE_UNROLL; ++j) {
            const int i = base + sub + j * EPI;
            e[j] = mv[min(i, m - 1)];
            if (i >= m) e[j].x = -1;
        }
        v4u kr[MOVE_UNROLL], vr[MOVE_UNROLL];
        uint2 sr[MOVE_UNROLL];
#pragma unroll
        for (int j = 0; j < MOVE_UNROLL; ++j)
            if (e[j].x >= 0) {
                kr[j] = __builtin_nontemporal_load(k_pool + (int64_t)e[j].y * CPR + c);
                vr[j] = __builtin_nontemporal_load(v_pool + (int64_t)e[j].y * CPR + c);
                if constexpr (SB > 0)
                    if (c == 0) {
                        const uint8_t *p = s_pool + (int64_t)e[j].y * SB;
                        if constexpr (SB == 8) sr[j] = *reinterpret_cast<const uint2 *>(p);
                        else sr[j].x = *reinterpret_cast<const uint32_t *>(p);
                    }
            }
#pragma unroll
        for (int j = 0; j < MOVE_UNROLL; ++j)
            if (e[j].x >= 0) {
                __builtin_nontemporal_store(kr[j], k_pool + (int64_t)e[j].x * CPR + c);
                __builtin_nontemporal_store(vr[j], v_pool + (int64_t)e[j].x * CPR + c);
                if constexpr (SB > 0)
                    if (c == 0) {
                        uint8_t *p = s_pool + (int64_t)e[j].x * SB;
                        if constexpr (SB == 8) *reinterpret_cast<uint2 *>(p) = sr[j];
                        else *reinterpret_cast<uint32_t *>(p) = sr[j].x;
                    }
            }
    }
}

}  // namespace sg

using namespace sg;

extern "C" size_t sg_evict_workspace_size(int units, int max_pages, int page_size) {
    if (units <= 0 || max_pages <= 0 || page_size <= 0) return 0;
    const size_t cap = (size_t)max_pages * page_size;
    return (size_t)units * (cap / 2 * sizeof(int2) + cap * 4 + 4);
}

extern "C" int sg_evict(void *stream, sg_dtype dt, int units, int d, void *k_pool, void *v_pool, uint8_t *s_pool,
                        int64_t pool_rows, const int32_t *page_table, const int32_t *n_rows, int page_size,
                        int max_pages, const int32_t *budget, const float *weight, const int32_t *pos, int64_t stride,
                        int sinks, const int32_t *recent_from, int32_t *n_kept, float *weight_out, int32_t *pos_out,
                        void *ws, size_t ws_bytes) {
    const char *fn = "sg_evict";
    SG_REQUIRE(dt == SG_F32 || dt == SG_BF16 || dt == SG_FP4, SG_EINVAL, "%s: unknown dtype %d", fn, (int)dt);
    SG_REQUIRE(units >= 0 && pool_rows >= 0 && sinks >= 0, SG_EINVAL, "%s: negative size", fn);
    SG_REQUIRE(d == 64 || d == 128, SG_EUNSUPPORTED, "%s: head dimension %d not supported (64 or 128)", fn, d);
    SG_REQUIRE(page_size >= 1 && max_pages >= 1, SG_EINVAL, "%s: page_size and max_pages must be >= 1", fn);
    SG_REQUIRE((int64_t)max_pages * page_size <= 80 * TOPK_THREADS, SG_EUNSUPPORTED, "%s: %lld rows per unit, above %d",
               fn, (long long)max_pages * page_size, 80 * TOPK_THREADS);
    SG_REQUIRE(pool_rows <= 0x7fffffffll, SG_EUNSUPPORTED, "%s: pool above 2^31 rows", fn);
    const int cap = max_pages * page_size;
    SG_REQUIRE(stride >= cap, SG_EINVAL, "%s: weight rows of %lld entries hold no %d rows", fn, (long long)stride, cap);
    SG_REQUIRE(max_workgroups(TOPK_THREADS) >= units, SG_EUNSUPPORTED, "%s: too many units", fn);
    if (units == 0) return SG_OK;
    SG_REQUIRE(k_pool && v_pool && page_table && n_rows && budget && weight && n_kept && weight_out, SG_EINVAL,
               "%s: null pointer", fn);
    SG_REQUIRE((dt == SG_FP4) == (s_pool != nullptr), SG_EINVAL, "%s: scales go with SG_FP4 pools, and only with them",
               fn);
    SG_REQUIRE((pos == nullptr) == (pos_out == nullptr), SG_EINVAL, "%s: pos and pos_out go together", fn);
    SG_REQUIRE(aligned16(k_pool) && aligned16(v_pool) && aligned16(s_pool) && aligned16(ws), SG_EINVAL,
               "%s: pools and workspace must be 16-byte aligned", fn);
    const size_t need = sg_evict_workspace_size(units, max_pages, page_size);
    SG_REQUIRE(ws && ws_bytes >= need, SG_EWORKSPACE, "%s: needs %zu bytes of workspace, %zu given", fn, need, ws_bytes);
    int2 *moves = reinterpret_cast<int2 *>(ws);
    int32_t *list = reinterpret_cast<int32_t *>(moves + (size_t)units * (cap / 2));
    int32_t *counts = list + (size_t)units * cap;
    hipStream_t s = as_stream(stream);
    const int items = (int)ceil_div(cap, TOPK_THREADS);
#define SG_SELECT(I)                                                                                                 \
    evict_select_kernel<I><<<(unsigned)units, TOPK_THREADS, 0, s>>>(pool_rows, page_table, n_rows, page_size,        \
                                                                    max_pages, budget, weight, pos, stride, sinks,   \
                                                                    recent_from, n_kept, weight_out, pos_out, moves, \
                                                                    list, counts)
    if (items <= 2) SG_SELECT(2);
    else if (items <= 4) SG_SELECT(4);
    else if (items <= 8) SG_SELECT(8);
    else if (items <= 16) SG_SELECT(16);
    else if (items <= 32) SG_SELECT(32);
    else if (items <= 64) SG_SELECT(64);
    else SG_SELECT(80);
#undef SG_SELECT
    const int cpr = dt == SG_FP4 ? d / 32 : d * esize_of(dt) / 16;
    const int64_t epb = MOVE_THREADS / cpr * MOVE_UNROLL;
    // about eight workgroups per CU over the units, each unit's moves a grid
    // stride apart
    const int64_t ny = std::min(std::max<int64_t>(1, ceil_div(cap / 2, epb)), ceil_div(8 * device_cus(), units));
    const dim3 grid((unsigned)units, (unsigned)ny);
    v4u *kp = reinterpret_cast<v4u *>(k_pool), *vp = reinterpret_cast<v4u *>(v_pool);
#define SG_MOVE(C, SB) evict_move_kernel<C, SB><<<grid, MOVE_THREADS, 0, s>>>(cap, moves, counts, kp, vp, s_pool)
    switch (cpr) {
        case 2: SG_MOVE(2, 4); break;
        case 4: SG_MOVE(4, 8); break;
        case 8: SG_MOVE(8, 0); break;
        case 16: SG_MOVE(16, 0); break;
        case 32: SG_MOVE(32, 0); break;
        default: set_error("%s: internal row size", fn); return SG_EINTERNAL;
    }
#undef SG_MOVE
    return launch_status(fn);
}
