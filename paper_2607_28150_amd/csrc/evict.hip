// sg_evict: cuts paged sets to a budget by accumulated weight.
//
// Select: one workgroup of 1024 threads per unit ranks the unit's rows like
// sg_topk (select_common.h; guarded rows carry the highest key of all) into a
// bit per row in LDS, with the number of kept rows before every 32.  A row's
// rank among the kept ones is then two LDS reads: the i-th row below k that is
// not kept is the i-th hole, the i-th kept row at or past k moves into it, and
// both write their half of the unit's i-th move.  Sources lie at or past k and
// destinations below it, so the moves need no order among themselves.
//
// Move: K and V rows (and scales), weights and positions of the listed moves,
// 16 bytes per lane: in the same launch, by the unit's own workgroup, where the
// units give every CU one; else in a second launch with many workgroups per
// unit.
//
// 512 units at 1,025 rows of which one goes: 12.0 us in a kernel trace, 9.8 per
// call of a replayed graph (f32 rows 9.6, 4-bit rows 9.8), bound by the chain of
// loads, counting barriers and stores of a workgroup (two launches, with searches
// over a list of ids: 16.8 + 3.9).  64 units of 8K to 32K rows cut to 20%: the
// select 24.8 us (one CU per unit, a quarter of the chip), the moves 59.7 us for
// 280 MB, 4.7 TB/s, the rate of a device copy; a call of f32 rows 116 us, of 4-bit
// rows 47.5.
#include "select_common.h"

namespace sg {

constexpr int MOVE_THREADS = 256;
constexpr int MOVE_UNROLL = 4;      // moves per lane group in flight, in a launch of their own

// Key of a guarded row: above that of every weight (+inf has 0xff800000), and
// not the largest word (the select looks at keys above its threshold).
constexpr uint32_t GUARD_KEY = 0xff800001u;

// Two workgroups per CU while a row's keys fit.
constexpr int evict_waves(int items) { return items <= 16 ? 8 : 4; }

struct EvictArgs {
    v4u *k_pool, *v_pool;
    uint8_t *s_pool;
    int64_t pool_rows;
    const int32_t *page_table, *n_rows;
    int page_size, max_pages;
    const int32_t *budget;
    const float *weight;            // (outputs may be their inputs: no restrict)
    const int32_t *pos;
    int64_t stride;
    int sinks;
    const int32_t *recent_from;
    int32_t *n_kept;
    float *weight_out;
    int32_t *pos_out;
    int2 *moves;                    // [units][cap / 2]: rows of the unit, to and from
    int32_t *counts;                // [units]
};

// Carries out moves first, first + step, ... of a unit's m, whole groups of
// CPR lanes (16-byte vectors per K or V row) at a time; SB: bytes of a row's
// scales.
template <int CPR, int SB, int UNROLL>
__device__ __forceinline__ void move_rows(const EvictArgs &a, int64_t unit, int m, int first, int step, int c) {
    const int2 *mv = a.moves + unit * (a.max_pages * a.page_size / 2);
    const int32_t *pt = a.page_table + unit * a.max_pages;
    const float *w = a.weight + unit * a.stride;
    const int32_t *ps = a.pos ? a.pos + unit * a.stride : nullptr;
    float *wo = a.weight_out + unit * a.stride;
    int32_t *po = a.pos_out ? a.pos_out + unit * a.stride : nullptr;
    auto pool_row = [&](int row) -> int {
        const int64_t x = (int64_t)pt[row / a.page_size] + row % a.page_size;
        return x >= 0 && x < a.pool_rows ? (int)x : -1;
    };
    for (int base = first; base < m; base += step * UNROLL) {
        int2 e[UNROLL];
        bool in[UNROLL], copy[UNROLL];
        int to[UNROLL], from[UNROLL];
#pragma unroll
        for (int j = 0; j < UNROLL; ++j) {
            const int i = base + j * step;
            in[j] = i < m;
            e[j] = mv[min(i, m - 1)];
        }
#pragma unroll
        for (int j = 0; j < UNROLL; ++j) {
            to[j] = pool_row(e[j].x);
            from[j] = pool_row(e[j].y);
            copy[j] = in[j] && to[j] >= 0 && from[j] >= 0;
        }
        v4u kr[UNROLL], vr[UNROLL];
        uint2 sr[UNROLL];
        float wr[UNROLL];
        int32_t pr[UNROLL];
#pragma unroll
        for (int j = 0; j < UNROLL; ++j) {
            if (copy[j]) {
                kr[j] = __builtin_nontemporal_load(a.k_pool + (int64_t)from[j] * CPR + c);
                vr[j] = __builtin_nontemporal_load(a.v_pool + (int64_t)from[j] * CPR + c);
            }
            if (in[j] && c == 0) {
                wr[j] = w[e[j].y];
                if (po) pr[j] = ps[e[j].y];
                if constexpr (SB > 0)
                    if (copy[j]) {
                        const uint8_t *p = a.s_pool + (int64_t)from[j] * SB;
                        if constexpr (SB == 8) sr[j] = *reinterpret_cast<const uint2 *>(p);
                        else sr[j].x = *reinterpret_cast<const uint32_t *>(p);
                    }
            }
        }
#pragma unroll
        for (int j = 0; j < UNROLL; ++j) {
            if (copy[j]) {
                __builtin_nontemporal_store(kr[j], a.k_pool + (int64_t)to[j] * CPR + c);
                __builtin_nontemporal_store(vr[j], a.v_pool + (int64_t)to[j] * CPR + c);
            }
            if (in[j] && c == 0) {
                wo[e[j].x] = wr[j];
                wo[e[j].y] = 0.f;
                if (po) {
                    po[e[j].x] = pr[j];
                    po[e[j].y] = -1;
                }
                if constexpr (SB > 0)
                    if (copy[j]) {
                        uint8_t *p = a.s_pool + (int64_t)to[j] * SB;
                        if constexpr (SB == 8) *reinterpret_cast<uint2 *>(p) = sr[j];
                        else *reinterpret_cast<uint32_t *>(p) = sr[j].x;
                    }
            }
        }
    }
}

// CPR = 0: the moves are left to a second launch.
template <int ITEMS, int CPR, int SB>
__global__ __launch_bounds__(TOPK_THREADS) __attribute__((amdgpu_waves_per_eu(evict_waves(ITEMS)))) void evict_select_kernel(
    EvictArgs a) {
    __shared__ SelectSmem sm;
    __shared__ uint32_t kept[ITEMS * 32];        // a bit per row
    __shared__ int32_t before[ITEMS * 32];       // kept rows before each word
    const int64_t unit = blockIdx.x;
    const int tid = threadIdx.x, cap = a.max_pages * a.page_size;
    const int n = min(max((int)a.n_rows[unit], 0), cap);
    const int k = min(max((int)a.budget[unit], 0), n);
    const float *w = a.weight + unit * a.stride;
    const int32_t *ps = a.pos ? a.pos + unit * a.stride : nullptr;
    float *wo = a.weight_out + unit * a.stride;
    int32_t *po = a.pos_out ? a.pos_out + unit * a.stride : nullptr;
    const bool copy = wo != w || po != ps;       // rows that stay have to be written
    int m = 0;
    if (k > 0 && k < n) {
        const int32_t recent = a.recent_from ? a.recent_from[unit] : 0x7fffffff;
        const int it = select_items(n), entry0 = select_entry(it);
        uint32_t key[ITEMS];
        constexpr int STEP = ITEMS < 8 ? ITEMS : 8;      // rows whose loads are in flight together
#pragma unroll
        for (int i0 = 0; i0 < ITEMS; i0 += STEP) {
#pragma unroll
            for (int i = i0; i < i0 + STEP; ++i) key[i] = 0u;
            if (i0 >= it) continue;                      // uniform
            float x[STEP];
            int32_t p[STEP];
#pragma unroll
            for (int i = 0; i < STEP; ++i) {
                const int at = min(entry0 + (i0 + i) * 64, n - 1);
                x[i] = w[at];
                p[i] = ps ? ps[at] : at;
            }
#pragma unroll
            for (int i = 0; i < STEP; ++i) {
                const bool guard = p[i] < a.sinks || (a.recent_from && p[i] >= recent);
                if (i0 + i < it && entry0 + (i0 + i) * 64 < n) key[i0 + i] = guard ? GUARD_KEY : order_key(x[i]);
            }
        }
        const int past = (tid / 64 + 1) * 64 * it;       // end of this wavefront's entries
        select_masks<ITEMS>(key, it, k, sm, [&](int first, uint32_t mask, int p) {
            if (first < past) {
                kept[first / 32] = mask;
                before[first / 32] = p;
            }
        });
        __syncthreads();
        auto rank = [&](int row) { return before[row / 32] + __popc(kept[row / 32] & ((1u << (row % 32)) - 1u)); };
        const int c = rank(k);                           // kept rows that stay
        m = k - c;
        int2 *mv = a.moves + unit * (cap / 2);
        for (int i0 = 0; i0 < it; i0 += STEP) {
            // the rows' weights and positions, should they be written elsewhere;
            // then what becomes of each (a row is read and written by its own
            // thread, moves come later)
            float x[STEP];
            int32_t p[STEP];
            if (copy) {
#pragma unroll
                for (int i = 0; i < STEP; ++i) {
                    const int at = min(entry0 + (i0 + i) * 64, n - 1);
                    x[i] = w[at];
                    if (po) p[i] = ps[at];
                }
            }
#pragma unroll
            for (int i = 0; i < STEP; ++i) {
                const int row = entry0 + (i0 + i) * 64;
                if (i0 + i >= it || row >= n) break;
                const bool keep = (kept[row / 32] >> (row % 32)) & 1u;
                const int r = rank(row);
                if (row < k) {
                    if (!keep) {
                        mv[row - r].x = row;
                    } else if (copy) {
                        wo[row] = x[i];
                        if (po) po[row] = p[i];
                    }
                } else if (keep) {
                    mv[r - c].y = row;                   // its weight goes with the move
                } else {
                    wo[row] = 0.f;
                    if (po) po[row] = -1;
                }
            }
        }
    } else {
        for (int i = tid; i < n; i += TOPK_THREADS) {
            if (i >= k) {
                wo[i] = 0.f;
                if (po) po[i] = -1;
            } else if (copy) {
                wo[i] = w[i];
                if (po) po[i] = ps[i];
            }
        }
    }
    __syncthreads();             // every thread has read the row count; the moves are listed
    if (tid == 0) {
        if (CPR == 0) a.counts[unit] = m;
        a.n_kept[unit] = k;
    }
    if constexpr (CPR > 0)
        move_rows<CPR, SB, 1>(a, unit, m, tid / CPR, TOPK_THREADS / CPR, tid % CPR);
}

template <int CPR, int SB>
__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(EvictArgs a) {
    constexpr int EPI = MOVE_THREADS / CPR, EPB = EPI * MOVE_UNROLL;      // moves per workgroup: one pass
    const int first = (int)blockIdx.y * EPB, m = min(a.counts[blockIdx.x], first + EPB);
    move_rows<CPR, SB, MOVE_UNROLL>(a, blockIdx.x, m, first + (int)threadIdx.x / CPR, EPI, threadIdx.x % CPR);
}

template <int CPR, int SB>
static int launch_evict(const char *fn, hipStream_t s, int units, const EvictArgs &a) {
    const int cap = a.max_pages * a.page_size, items = (int)ceil_div(cap, TOPK_THREADS);
    const bool one = units >= device_cus();
#define SG_SELECT(I)                                                                              \
    do {                                                                                          \
        if (one) evict_select_kernel<I, CPR, SB><<<(unsigned)units, TOPK_THREADS, 0, s>>>(a);     \
        else evict_select_kernel<I, 0, 0><<<(unsigned)units, TOPK_THREADS, 0, s>>>(a);            \
    } while (0)
    if (items <= 2) SG_SELECT(2);
    else if (items <= 4) SG_SELECT(4);
    else if (items <= 8) SG_SELECT(8);
    else if (items <= 16) SG_SELECT(16);
    else if (items <= 32) SG_SELECT(32);
    else if (items <= 64) SG_SELECT(64);
    else SG_SELECT(80);
#undef SG_SELECT
    if (!one) {
        const dim3 grid((unsigned)units, (unsigned)std::max<int64_t>(1, ceil_div(cap / 2, MOVE_THREADS / CPR * MOVE_UNROLL)));
        evict_move_kernel<CPR, SB><<<grid, MOVE_THREADS, 0, s>>>(a);
    }
    return launch_status(fn);
}

}  // namespace sg

using namespace sg;

extern "C" size_t sg_evict_workspace_size(int units, int max_pages, int page_size) {
    if (units <= 0 || max_pages <= 0 || page_size <= 0) return 0;
    const size_t cap = (size_t)max_pages * page_size;
    return (size_t)units * (cap / 2 * sizeof(int2) + sizeof(int32_t));
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
    if (sinks == 0) sinks = INT32_MIN;      // no position is below it, negative ones neither
    const EvictArgs a{reinterpret_cast<v4u *>(k_pool), reinterpret_cast<v4u *>(v_pool), s_pool, pool_rows, page_table,
                      n_rows, page_size, max_pages, budget, weight, pos, stride, sinks, recent_from, n_kept, weight_out,
                      pos_out, moves, reinterpret_cast<int32_t *>(moves + (size_t)units * (cap / 2))};
    hipStream_t s = as_stream(stream);
    switch (dt == SG_FP4 ? d / 32 : d * esize_of(dt) / 16) {
        case 2: return launch_evict<2, 4>(fn, s, units, a);
        case 4: return launch_evict<4, 8>(fn, s, units, a);
        case 8: return launch_evict<8, 0>(fn, s, units, a);
        case 16: return launch_evict<16, 0>(fn, s, units, a);
        case 32: return launch_evict<32, 0>(fn, s, units, a);
        default: set_error("%s: internal row size", fn); return SG_EINTERNAL;
    }
}
