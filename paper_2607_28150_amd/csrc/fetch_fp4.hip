// sg_fetch_fp4: sg_fetch into or out of a 4-bit pool (fp4.h).
//
// Eight channels per lane, so LPR = d / 8 lanes cover a row and the four lanes
// of a quad hold one 32-channel block: the block's largest magnitude is two
// quad DPP steps, the conversion instructions do the rest, and the row's scale
// bytes meet in its first lane by row DPP moves.  Bound by memory: a bf16 row
// pair of d = 128 is 512 bytes in, 136 out, and both directions run at the rate
// of a device copy (4.7 TB/s).
#include "fp4.h"

namespace sg {

// One wavefront per workgroup, two entries per lane group: of 256 and 64
// threads with one, two and four entries, the fastest for many rows (209,664
// bf16 rows of d = 128 written in 28.8 us and read back in 31.0; 256 threads
// with four entries 31.5 and 33.0) and next to it for few (512 rows 4.0 and
// 4.2 us; 5.6 and 6.0).  From a host source: larger workgroups with more in
// flight, see the launch.
constexpr int FETCH4_THREADS = 64, FETCH4_UNROLL = 2;
constexpr int FETCH4_HOST_THREADS = 256, FETCH4_HOST_UNROLL = 4;

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}
constexpr int D4_XOR1 = 0xB1, D4_XOR2 = 0x4E, D4_HALF_MIRROR = 0x141, D4_ROR4 = 0x124, D4_ROR8 = 0x128;

struct F4 {};      // tag of 4-bit rows

// One lane's 8 channels of a row as they lie in memory.
template <typename T>
struct Slice8;
template <>
struct Slice8<float> {
    v4u a, b;
    __device__ void load(const void *base, int64_t row, int lpr, int c) {
        const v4u *p = reinterpret_cast<const v4u *>(base) + (row * lpr + c) * 2;
        a = __builtin_nontemporal_load(p);
        b = __builtin_nontemporal_load(p + 1);
    }
    __device__ void unpack(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = __uint_as_float(a[i]);
            x[4 + i] = __uint_as_float(b[i]);
        }
    }
};
template <>
struct Slice8<uint16_t> {
    v4u a;
    __device__ void load(const void *base, int64_t row, int lpr, int c) {
        a = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(base) + row * lpr + c);
    }
    __device__ void unpack(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(a[i]);
            x[2 * i + 1] = bf16_hi(a[i]);
        }
    }
};
template <>
struct Slice8<F4> {
    uint32_t a;
    __device__ void load(const void *base, int64_t row, int lpr, int c) {
        a = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(base) + row * lpr + c);
    }
};

// Codes of the lane's 8 channels and its block's scale byte.
template <typename T>
__device__ __forceinline__ uint32_t encode_slice(const Slice8<T> &s, uint32_t &byte) {
    float x[8];
    s.unpack(x);
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);     // NaN above every number
    top = max(top, dpp_u32<D4_XOR1>(top));
    top = max(top, dpp_u32<D4_XOR2>(top));
    byte = fp4_scale_byte(top);
    return byte == FP4_NAN_SCALE ? 0u : fp4_encode8(x, fp4_scale(byte));
}

// The row's scale bytes {K blocks, V blocks} from its lanes' own (equal within
// a quad): 8 bytes for d = 128 (16 lanes), 4 for d = 64 (8 lanes).
template <int LPR>
__device__ __forceinline__ uint2 gather_scales(uint32_t kb, uint32_t vb, int c) {
    if constexpr (LPR == 16) {
        kb <<= 8 * (c / 4);
        vb <<= 8 * (c / 4);
        kb |= dpp_u32<D4_ROR4>(kb);
        vb |= dpp_u32<D4_ROR4>(vb);
        return make_uint2(kb | dpp_u32<D4_ROR8>(kb), vb | dpp_u32<D4_ROR8>(vb));
    } else {
        uint32_t w = (kb | (vb << 16)) << (8 * (c / 4));
        return make_uint2(w | dpp_u32<D4_HALF_MIRROR>(w), 0u);
    }
}

// SRC, DST: float, uint16_t (bf16) or F4; one of them is F4.
template <typename SRC, typename DST, int D, int THREADS, int UNROLL>
__global__ __launch_bounds__(THREADS) void fetch4_kernel(
    int rows, const int32_t *__restrict__ row_off, int64_t total, const int32_t *__restrict__ index,
    const int32_t *__restrict__ n_valid, const int64_t *__restrict__ src_row_base, int64_t src_rows,
    const void *__restrict__ k_src, const void *__restrict__ v_src, const uint8_t *__restrict__ s_src,
    const int32_t *__restrict__ page_table, int page_size, int max_pages, const int32_t *__restrict__ dst_start,
    void *__restrict__ k_pool, void *__restrict__ v_pool, uint8_t *__restrict__ s_pool, int64_t pool_rows) {
    constexpr bool FROM4 = std::is_same_v<SRC, F4>, TO4 = std::is_same_v<DST, F4>;
    constexpr int LPR = D / 8, SB = 2 * D / FP4_BLOCK;     // lanes and scale bytes of a row
    constexpr int EPI = THREADS / LPR, EPB = EPI * UNROLL;
    const int c = threadIdx.x % LPR, sub = threadIdx.x / LPR;
    if (src_rows <= 0) return;
    for (int r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t o = row_off[r], e = row_off[r + 1];
        if (o < 0 || e < o || e > total) continue;
        int64_t n = e - o;
        if (n_valid) n = min<int64_t>(n, max<int32_t>(n_valid[r], 0));
        const int64_t sbase = src_row_base[r], lbase = dst_start[r];
        const int32_t *pt = page_table + (int64_t)r * max_pages;
        for (int64_t base = (int64_t)blockIdx.y * EPB; base < n; base += (int64_t)gridDim.y * EPB) {
            // the index loads of the pass, then the row loads (an entry that is
            // not copied reads source row 0), then the stores
            int64_t tok[UNROLL];
#pragma unroll
            for (int j = 0; j < UNROLL; ++j) {
                const int64_t i = min(base + sub + j * EPI, n - 1);
                tok[j] = index ? (int64_t)index[o + i] : i;
            }
            Slice8<SRC> ks[UNROLL], vs[UNROLL];
            uint2 sc[UNROLL];
            int64_t dst[UNROLL];
#pragma unroll
            for (int j = 0; j < UNROLL; ++j) {
                const int64_t i = base + sub + j * EPI, src = sbase + tok[j], lr = lbase + i;
                const bool live = i < n && src >= 0 && src < src_rows;
                const int64_t s_row = live ? src : 0;
                ks[j].load(k_src, s_row, LPR, c);
                vs[j].load(v_src, s_row, LPR, c);
                if constexpr (FROM4) {
                    if constexpr (SB == 8) sc[j] = *reinterpret_cast<const uint2 *>(s_src + s_row * SB);
                    else sc[j] = make_uint2(*reinterpret_cast<const uint32_t *>(s_src + s_row * SB), 0u);
                }
                dst[j] = -1;
                if (live && lr >= 0 && lr / page_size < max_pages) {
                    const int64_t pr = (int64_t)pt[lr / page_size] + lr % page_size;
                    if (pr >= 0 && pr < pool_rows) dst[j] = pr;
                }
            }
#pragma unroll
            for (int j = 0; j < UNROLL; ++j) {
                if constexpr (TO4) {
                    uint32_t kc, vc;
                    uint2 s;
                    if constexpr (FROM4) {
                        kc = ks[j].a;
                        vc = vs[j].a;
                        s = sc[j];
                    } else {
                        uint32_t kb, vb;
                        kc = encode_slice(ks[j], kb);
                        vc = encode_slice(vs[j], vb);
                        s = gather_scales<LPR>(kb, vb, c);
                    }
                    if (dst[j] < 0) continue;
                    __builtin_nontemporal_store(kc, reinterpret_cast<uint32_t *>(k_pool) + dst[j] * LPR + c);
                    __builtin_nontemporal_store(vc, reinterpret_cast<uint32_t *>(v_pool) + dst[j] * LPR + c);
                    if (c == 0) {
                        uint8_t *p = s_pool + dst[j] * SB;
                        if constexpr (SB == 8) *reinterpret_cast<uint2 *>(p) = s;
                        else *reinterpret_cast<uint32_t *>(p) = s.x;
                    }
                } else {
                    if (dst[j] < 0) continue;
                    // bytes of the lane's block: K's first, then V's
                    const int blk = c / 4;
                    const uint32_t kb = (sc[j].x >> (8 * blk)) & 255u;
                    const uint32_t vb = SB == 8 ? (sc[j].y >> (8 * blk)) & 255u : (sc[j].x >> (16 + 8 * blk)) & 255u;
                    auto put = [&](uint32_t codes, uint32_t byte, void *pool) {
                        const float scale = fp4_scale(byte);
                        const v4u h = {fp4_bf16_pair<0>(codes, scale), fp4_bf16_pair<1>(codes, scale),
                                       fp4_bf16_pair<2>(codes, scale), fp4_bf16_pair<3>(codes, scale)};
                        if constexpr (std::is_same_v<DST, uint16_t>) {
                            __builtin_nontemporal_store(h, reinterpret_cast<v4u *>(pool) + dst[j] * LPR + c);
                        } else {
                            v4u lo, hi;
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                lo[2 * i] = h[i] << 16;
                                lo[2 * i + 1] = h[i] & 0xffff0000u;
                                hi[2 * i] = h[2 + i] << 16;
                                hi[2 * i + 1] = h[2 + i] & 0xffff0000u;
                            }
                            v4u *p = reinterpret_cast<v4u *>(pool) + (dst[j] * LPR + c) * 2;
                            __builtin_nontemporal_store(lo, p);
                            __builtin_nontemporal_store(hi, p + 1);
                        }
                    };
                    put(ks[j].a, kb, k_pool);
                    put(vs[j].a, vb, v_pool);
                }
            }
        }
    }
}

}  // namespace sg

using namespace sg;

extern "C" int sg_fetch_fp4(void *stream, sg_dtype src_dt, sg_dtype dst_dt, int d, int rows, const int32_t *row_off,
                            int64_t total, const int32_t *index, const int32_t *n_valid, const int64_t *src_row_base,
                            int64_t src_rows, const void *k_src, const void *v_src, const uint8_t *s_src,
                            const int32_t *page_table, int page_size, int max_pages, const int32_t *dst_start,
                            void *k_pool, void *v_pool, uint8_t *s_pool, int64_t pool_rows) {
    const char *fn = "sg_fetch_fp4";
    auto known = [](sg_dtype t) { return t == SG_F32 || t == SG_BF16 || t == SG_FP4; };
    SG_REQUIRE(known(src_dt) && known(dst_dt), SG_EINVAL, "%s: unknown dtype %d or %d", fn, (int)src_dt, (int)dst_dt);
    SG_REQUIRE(src_dt == SG_FP4 || dst_dt == SG_FP4, SG_EINVAL, "%s: source or pool must be SG_FP4 (else sg_fetch)", fn);
    SG_REQUIRE(d == 64 || d == 128, SG_EUNSUPPORTED, "%s: head dimension %d not supported (64 or 128)", fn, d);
    SG_REQUIRE(rows >= 0 && total >= 0 && src_rows >= 0 && pool_rows >= 0, SG_EINVAL, "%s: negative size", fn);
    SG_REQUIRE(page_size >= 1 && max_pages >= 1, SG_EINVAL, "%s: page_size and max_pages must be >= 1", fn);
    if (rows == 0 || total == 0) return SG_OK;
    SG_REQUIRE(row_off && src_row_base && k_src && v_src && page_table && dst_start && k_pool && v_pool, SG_EINVAL,
               "%s: null pointer", fn);
    SG_REQUIRE((src_dt == SG_FP4) == (s_src != nullptr) && (dst_dt == SG_FP4) == (s_pool != nullptr), SG_EINVAL,
               "%s: scales go with SG_FP4 rows, and only with them", fn);
    SG_REQUIRE(aligned16(k_src) && aligned16(v_src) && aligned16(s_src) && aligned16(k_pool) && aligned16(v_pool) &&
                   aligned16(s_pool),
               SG_EINVAL, "%s: row arrays must be 16-byte aligned", fn);
    const bool host = host_memory(k_src) || host_memory(v_src);
    dim3 grid;
    if (!host) {
        // workgroups per index row: one pass over a row of average length, more
        // where the rows alone would leave the chip idle; longer rows are
        // covered by the stride loop
        const int64_t epb = FETCH4_THREADS / (d / 8) * FETCH4_UNROLL;
        const int64_t ny = std::max(ceil_div(ceil_div(total, rows), epb), std::min(ceil_div(total, epb), ceil_div(2048, rows)));
        grid = dim3((unsigned)std::min<int64_t>(rows, max_workgroups(FETCH4_THREADS)), (unsigned)std::min<int64_t>(ny, 65535));
    } else {
        // as many bytes in flight as sg_fetch has from a host source: HOST_LINK_WORKGROUPS
        // times 256 threads with eight entries of two 16-byte vectors
        const int slice = src_dt == SG_F32 ? 32 : src_dt == SG_BF16 ? 16 : 4;
        const int wgs = HOST_LINK_WORKGROUPS * 8 * 16 / (FETCH4_HOST_UNROLL * slice);
        grid = dim3((unsigned)std::min(rows, wgs), (unsigned)std::max(1, wgs / std::min(rows, wgs)));
    }
    hipStream_t s = as_stream(stream);
#define SG_FETCH4_L(S, T, D, THREADS, UNROLL)                                                                          \
    fetch4_kernel<S, T, D, THREADS, UNROLL><<<grid, THREADS, 0, s>>>(                                                  \
        rows, row_off, total, index, n_valid, src_row_base, src_rows, k_src, v_src, s_src, page_table, page_size,      \
        max_pages, dst_start, k_pool, v_pool, s_pool, pool_rows)
#define SG_FETCH4(S, T, D)                                                                                             \
    do {                                                                                                               \
        if (host) SG_FETCH4_L(S, T, D, FETCH4_HOST_THREADS, FETCH4_HOST_UNROLL);                                       \
        else SG_FETCH4_L(S, T, D, FETCH4_THREADS, FETCH4_UNROLL);                                                      \
    } while (0)
#define SG_FETCH4_D(S, T)                  \
    do {                                   \
        if (d == 64) SG_FETCH4(S, T, 64);  \
        else SG_FETCH4(S, T, 128);         \
    } while (0)
    if (src_dt == SG_FP4 && dst_dt == SG_FP4) SG_FETCH4_D(F4, F4);
    else if (src_dt == SG_F32) SG_FETCH4_D(float, F4);
    else if (src_dt == SG_BF16) SG_FETCH4_D(uint16_t, F4);
    else if (dst_dt == SG_F32) SG_FETCH4_D(F4, float);
    else SG_FETCH4_D(F4, uint16_t);
#undef SG_FETCH4_D
#undef SG_FETCH4
#undef SG_FETCH4_L
    return launch_status(fn);
}
