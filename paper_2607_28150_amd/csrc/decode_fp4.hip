// sg_decode_attn_fp4: GQA decode attention over a paged set of 4-bit rows
// (fp4.h), with or without the weights the rows receive (decode_weights.h).
//
// Grid: x = (sequence, KV head) unit, y = split of the unit's rows.  A
// workgroup's four wavefronts take consecutive ranges of the split's rows, 32
// rows a step, and serve all G <= 16 query heads of the unit with matrix
// instructions (16 x 16 x 32, bf16 in, fp32 out):
//   logits : A = 16 K rows x 32 channels, B = the same channels of 16 heads.
//            The channels of a product may come in any order, so lane (row m,
//            quarter kg) takes kg's d / 4 consecutive channels of its row, 8 of
//            them per instruction.
//   values : A = 16 heads x 32 rows (the probabilities), B = 32 rows x 16
//            channels.  The logits leave head n, rows 4 kg .. 4 kg + 3 of both
//            16-row tiles in lane (n, kg): taken as that lane's 8 of the 32
//            rows, the probabilities are where the next product wants them.
//            Lane (n, kg) reads the matching 8 V rows, d / 16 consecutive
//            channels each, one channel per instruction.
// 4-bit values times their scale are exact in bf16.  Queries in bf16 are too;
// fp32 queries and the probabilities are cut into three bf16 parts of 8 bits
// that add up to them exactly, so nothing is rounded below fp32.
//
// Softmax as in sg_decode_attn: online in log2 units against a reference max
// per head that is raised only when a logit passes it by 2^16.
#include "decode_weights.h"
#include "fp4.h"

namespace sg {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int D4_WAVES = 4;
constexpr int D4_STEP = 32;                  // rows per wavefront and step
constexpr int D4_PT_CAP = 2048;              // page entries of one split staged in LDS
constexpr int D4_MIN_SPLIT_ROWS = D4_WAVES * D4_STEP;
constexpr float D4_LAZY = 16.f;              // log2 headroom before the reference max is raised

__device__ __forceinline__ bf16x8 as_bf16x8(const v4u &w) {
    bf16x8 r;
    __builtin_memcpy(&r, &w, sizeof(r));
    return r;
}

// x cut into three parts of 8 significant bits each, as bf16 bits in the high
// half: x = p[0] + p[1] + p[2] exactly (a part below the smallest normal is
// lost).
__device__ __forceinline__ void split3(float x, uint32_t (&p)[3]) {
    p[0] = __float_as_uint(x) & 0xffff0000u;
    const float r = x - __uint_as_float(p[0]);
    p[1] = __float_as_uint(r) & 0xffff0000u;
    p[2] = __float_as_uint(r - __uint_as_float(p[1])) & 0xffff0000u;
}
__device__ __forceinline__ uint32_t high_halves(uint32_t lo, uint32_t hi) { return (lo >> 16) | hi; }

// T: type of the queries; W: the logits are kept for the weights.
template <typename T, int D, bool W>
__global__ __launch_bounds__(64 * D4_WAVES) void decode4_kernel(
    int Hq, int Hkv, float scale_log2, const T *__restrict__ q, const uint8_t *__restrict__ k_pool,
    const uint8_t *__restrict__ v_pool, const uint8_t *__restrict__ s_pool, int64_t pool_rows,
    const int32_t *__restrict__ page_table, const int32_t *__restrict__ n_rows, int page_size, int max_pages,
    int64_t split_rows, float *__restrict__ out, float *__restrict__ states, float *__restrict__ z_out,
    int64_t z_stride) {
    constexpr int STEPS = D / 32;            // K products per 16 rows: 8 channels of every lane each
    constexpr int NC = D / 16;               // V channels per lane, and products per 32 rows
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int SB = 2 * D / FP4_BLOCK;    // scale bytes per row: K's, then V's
    __shared__ int32_t pte[D4_PT_CAP];
    __shared__ float o_s[D4_WAVES][16 * D], m_s[D4_WAVES][16], l_s[D4_WAVES][16];

    const int tid = threadIdx.x, lane = tid % 64, n16 = lane % 16, kg = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int64_t unit = blockIdx.x;
    const int split = blockIdx.y, nsplit = gridDim.y;
    const int b = (int)(unit / Hkv), h = (int)(unit % Hkv), G = Hq / Hkv;
    const int64_t max_rows = (int64_t)max_pages * page_size;
    const int64_t n = max<int64_t>(0, min<int64_t>((int64_t)n_rows[unit], max_rows));
    const int64_t r0 = (int64_t)split * split_rows;
    if (nsplit > 1 && r0 >= n) return;       // writes no state: whoever joins them reads the row count
    const int64_t r1 = pool_rows > 0 ? min<int64_t>(n, r0 + split_rows) : r0;
    const int64_t pg0 = r0 / page_size;      // splits start on a page
    const int npg = (int)min<int64_t>(D4_PT_CAP, max<int64_t>(0, ceil_div(r1, page_size) - pg0));
    for (int i = tid; i < npg; i += 64 * D4_WAVES) pte[i] = page_table[unit * max_pages + pg0 + i];

    // the queries: head n16, channels of quarter kg, 8 per product
    bf16x8 qf[PARTS][STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const T *qp = q + ((int64_t)b * Hq + (int64_t)h * G + min(n16, G - 1)) * D + kg * (D / 4) + s * 8;
        v4u w[PARTS];
        if constexpr (PARTS == 1) {
            w[0] = *reinterpret_cast<const v4u *>(qp);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t a[3], c[3];
                split3(qp[2 * i], a);
                split3(qp[2 * i + 1], c);
#pragma unroll
                for (int p = 0; p < 3; ++p) w[p][i] = high_halves(a[p], c[p]);
            }
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) qf[p][s] = as_bf16x8(n16 < G ? w[p] : v4u{0u, 0u, 0u, 0u});
    }
    __syncthreads();    // page entries staged

    float m = -INFINITY, l = 0.f;            // of head n16 (l: this lane's rows)
    f32x4 o[NC];                             // o[j][i]: head 4 kg + i, channel NC n16 + j
#pragma unroll
    for (int j = 0; j < NC; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int64_t len = max<int64_t>(0, r1 - r0);
    const int64_t per = ceil_div(ceil_div(len, D4_WAVES), D4_STEP) * D4_STEP;
    const int64_t w0 = r0 + wave * per, w1 = min<int64_t>(r1, w0 + per);
    // pool row of logical row lr, or -1
    auto pool_row = [&](int64_t lr) -> int {
        const uint32_t rel = (uint32_t)(min<int64_t>(lr, r1 - 1) - pg0 * page_size);
        const uint32_t pi = rel / (uint32_t)page_size;
        const int64_t x = (int64_t)pte[pi] + (int)(rel - pi * (uint32_t)page_size);
        return lr < w1 && x >= 0 && x < pool_rows ? (int)x : -1;
    };
    for (int64_t t = w0; t < w1; t += D4_STEP) {
        const uint32_t live = (uint32_t)__ballot(pool_row(t + lane % 32) >= 0);    // bit i: row t + i counts
        // logits: lane (n16, kg) of tile u gets rows 16 u + 4 kg + i of head n16
        float z[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t row = max(pool_row(t + 16 * u + n16), 0);
            const uint32_t byte = s_pool[row * SB + kg * (D / 4) / FP4_BLOCK];
            const float sc = fp4_scale(byte);
            const uint32_t *kp = reinterpret_cast<const uint32_t *>(k_pool + row * (D / 2) + kg * (D / 8));
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const uint32_t w = kp[s];
                const bf16x8 kf = as_bf16x8(v4u{fp4_bf16_pair<0>(w, sc), fp4_bf16_pair<1>(w, sc),
                                                fp4_bf16_pair<2>(w, sc), fp4_bf16_pair<3>(w, sc)});
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[p][s], acc, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                z[4 * u + i] = (live >> (16 * u + 4 * kg + i)) & 1u ? acc[i] * scale_log2 : -INFINITY;
        }
        if constexpr (W) {
            if (n16 < G) {
                float *zp = z_out + (unit * G + n16) * z_stride + t + 4 * kg;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (t + 16 * u + 4 * kg + i < w1) zp[16 * u + i] = z[4 * u + i];
            }
        }
        float top = z[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, z[i]);
        if (__any(top > m + D4_LAZY)) {      // raise every head's reference (rare)
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float mn = fmaxf(m, top);
            const float a = mn == m ? 1.f : __builtin_amdgcn_exp2f(m - mn);
            l *= a;
            m = mn;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float ai = __shfl(a, 4 * kg + i, 64);
#pragma unroll
                for (int j = 0; j < NC; ++j) o[j][i] *= ai;
            }
        }
        const float ref = m == -INFINITY ? 0.f : m;
        uint32_t pw[3][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = __builtin_amdgcn_exp2f(z[i] - ref);
            l += p;
            uint32_t x[3];
            split3(p, x);
#pragma unroll
            for (int k = 0; k < 3; ++k) pw[k][i] = x[k];
        }
        bf16x8 pf[3];
#pragma unroll
        for (int k = 0; k < 3; ++k)
            pf[k] = as_bf16x8(v4u{high_halves(pw[k][0], pw[k][1]), high_halves(pw[k][2], pw[k][3]),
                                  high_halves(pw[k][4], pw[k][5]), high_halves(pw[k][6], pw[k][7])});
        // values: 8 rows x NC channels per lane, as bf16 pairs of channels, then of rows
        uint32_t vb[8][NC / 2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int rr = i < 4 ? 4 * kg + i : 16 + 4 * kg + i - 4;
            const int pr = pool_row(t + rr);
            const int64_t row = max(pr, 0);
            // a row that is left out may stand in pool row 0: its zero
            // probability must not meet a NaN
            const uint32_t byte = pr >= 0 ? s_pool[row * SB + SB / 2 + n16 * NC / FP4_BLOCK] : 0u;
            const float sc = fp4_scale(byte);
            uint32_t w;
            if constexpr (NC == 8) w = *reinterpret_cast<const uint32_t *>(v_pool + row * (D / 2) + n16 * 4);
            else w = *reinterpret_cast<const uint16_t *>(v_pool + row * (D / 2) + n16 * 2);
            vb[i][0] = fp4_bf16_pair<0>(w, sc);
            vb[i][1] = fp4_bf16_pair<1>(w, sc);
            if constexpr (NC == 8) {
                vb[i][2] = fp4_bf16_pair<2>(w, sc);
                vb[i][3] = fp4_bf16_pair<3>(w, sc);
            }
        }
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            v4u w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = vb[2 * i][j / 2], c = vb[2 * i + 1][j / 2];
                w[i] = j % 2 == 0 ? (a & 0xffffu) | (c << 16) : (a >> 16) | (c & 0xffff0000u);
            }
            const bf16x8 vf = as_bf16x8(w);
#pragma unroll
            for (int k = 0; k < 3; ++k) o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[k], vf, o[j], 0, 0, 0);
        }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (kg == 0) {
        m_s[wave][n16] = m;
        l_s[wave][n16] = l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < NC; ++j) o_s[wave][(4 * kg + i) * D + NC * n16 + j] = o[j][i];
    __syncthreads();
    for (int it = tid; it < G * D; it += 64 * D4_WAVES) {
        const int g = it / D, c = it % D;
        float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
        for (int w = 0; w < D4_WAVES; ++w) M = fmaxf(M, m_s[w][g]);
#pragma unroll
        for (int w = 0; w < D4_WAVES; ++w) {
            const float a = m_s[w][g] == M ? 1.f : __builtin_amdgcn_exp2f(m_s[w][g] - M);
            L += a * l_s[w][g];
            O += a * o_s[w][it];
        }
        if (!W && nsplit == 1) {
            out[((int64_t)b * Hq + (int64_t)h * G + g) * D + c] = O * (L == 0.f ? 0.f : 1.f / L);
        } else {
            float *p = states + ((unit * nsplit + split) * G + g) * (int64_t)(D + 2);
            if (c == 0) {
                p[0] = M;
                p[1] = L;
            }
            p[2 + c] = O;
        }
    }
}

// Rows per split: enough workgroups for every CU where the units alone are
// fewer, whole pages, no more page entries than the LDS stage holds.
static int64_t plan_split4(int64_t units, int64_t max_rows, int page_size) {
    const int64_t want = units < device_cus() ? ceil_div(device_cus(), units) : 1;
    int64_t rows = std::max<int64_t>(ceil_div(max_rows, want), D4_MIN_SPLIT_ROWS);
    rows = std::min<int64_t>(rows, (int64_t)D4_PT_CAP * page_size);
    return ceil_div(rows, page_size) * page_size;
}

// Most splits a call can use: its splits are at least D4_MIN_SPLIT_ROWS rows,
// or as long as D4_PT_CAP pages reach.
static int64_t max_splits4(int64_t max_rows) { return std::max<int64_t>(1, ceil_div(max_rows, D4_MIN_SPLIT_ROWS)); }

template <typename T, int D>
static int launch_decode4(const char *fn, hipStream_t s, int B, int Hq, int Hkv, float sl2, const void *q,
                          const uint8_t *k_pool, const uint8_t *v_pool, const uint8_t *s_pool, int64_t pool_rows,
                          const int32_t *page_table, const int32_t *n_rows, int page_size, int max_pages, float *out,
                          Weights w, float *ws, size_t ws_bytes) {
    const int G = Hq / Hkv;
    const int64_t units = (int64_t)B * Hkv, max_rows = (int64_t)max_pages * page_size;
    const int64_t split_rows = plan_split4(units, max_rows, page_size), nsplit = ceil_div(max_rows, split_rows);
    SG_REQUIRE(nsplit <= 65535, SG_EUNSUPPORTED, "%s: %lld splits are not supported", fn, (long long)nsplit);
    w.z_stride = z_stride_of(max_rows);
    const bool weights = w.out != nullptr;
    const size_t zb = weights ? (size_t)units * G * w.z_stride * sizeof(float) : 0;
    const size_t sb = weights || nsplit > 1 ? (size_t)units * nsplit * G * (D + 2) * sizeof(float) : 0;
    SG_REQUIRE(zb + sb <= ws_bytes && (zb + sb == 0 || ws), SG_EWORKSPACE, "%s: needs %zu bytes of workspace, %zu given",
               fn, zb + sb, ws_bytes);
    w.z = ws;
    float *states = weights ? ws + zb / sizeof(float) : ws;
    const dim3 grid((unsigned)units, (unsigned)nsplit);
    const T *qq = reinterpret_cast<const T *>(q);
    if (weights)
        decode4_kernel<T, D, true><<<grid, 64 * D4_WAVES, 0, s>>>(Hq, Hkv, sl2, qq, k_pool, v_pool, s_pool, pool_rows,
                                                                  page_table, n_rows, page_size, max_pages, split_rows,
                                                                  out, states, w.z, w.z_stride);
    else
        decode4_kernel<T, D, false><<<grid, 64 * D4_WAVES, 0, s>>>(Hq, Hkv, sl2, qq, k_pool, v_pool, s_pool, pool_rows,
                                                                   page_table, n_rows, page_size, max_pages, split_rows,
                                                                   out, states, nullptr, 0);
    if (weights || nsplit > 1) {
        const dim3 fgrid((unsigned)units, weights ? (unsigned)ceil_div(max_rows, FINISH_ROWS) : 1u);
        decode_finish_kernel<D><<<fgrid, FINISH_THREADS, 0, s>>>(Hq, Hkv, (int)nsplit, n_rows, max_rows, split_rows,
                                                                 states, out, w);
    }
    return launch_status(fn);
}

}  // namespace sg

using namespace sg;

extern "C" size_t sg_decode_attn_fp4_workspace_size(int B, int Hq, int Hkv, int d, int max_pages, int page_size,
                                                    int weights) {
    if (B <= 0 || Hkv <= 0 || Hq <= 0 || Hq % Hkv != 0 || d <= 0 || max_pages <= 0 || page_size <= 0) return 0;
    const int64_t max_rows = (int64_t)max_pages * page_size, cap = max_splits4(max_rows);
    const size_t heads = (size_t)B * Hq;
    const size_t states = weights || cap > 1 ? heads * cap * (size_t)(d + 2) * sizeof(float) : 0;
    return states + (weights ? heads * (size_t)z_stride_of(max_rows) * sizeof(float) : 0);
}

extern "C" int sg_decode_attn_fp4(void *stream, sg_dtype dt, int B, int Hq, int Hkv, int d, float scale, const void *q,
                                  const uint8_t *k_pool, const uint8_t *v_pool, const uint8_t *s_pool,
                                  int64_t pool_rows, const int32_t *page_table, const int32_t *n_rows, int page_size,
                                  int max_pages, float *out, const float *weight_in, float decay, float *weight_out,
                                  int64_t weight_stride, void *ws, size_t ws_bytes) {
    const char *fn = "sg_decode_attn_fp4";
    SG_REQUIRE(dt == SG_F32 || dt == SG_BF16, SG_EINVAL, "%s: unknown dtype %d of the queries", fn, (int)dt);
    SG_REQUIRE(B >= 0 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0, SG_EINVAL, "%s: need Hq %% Hkv == 0 (Hq=%d, Hkv=%d)", fn,
               Hq, Hkv);
    SG_REQUIRE(Hq / Hkv <= FINISH_MAX_G, SG_EUNSUPPORTED, "%s: group size %d above %d", fn, Hq / Hkv, FINISH_MAX_G);
    SG_REQUIRE(d == 64 || d == 128, SG_EUNSUPPORTED, "%s: head dimension %d not supported", fn, d);
    SG_REQUIRE(page_size >= 1 && max_pages >= 1 && pool_rows >= 0, SG_EINVAL, "%s: bad page geometry", fn);
    SG_REQUIRE((int64_t)max_pages * page_size <= (1ll << 30), SG_EINVAL, "%s: page table too large", fn);
    SG_REQUIRE(pool_rows <= 0x7fffffffll, SG_EUNSUPPORTED, "%s: pool above 2^31 rows", fn);
    SG_REQUIRE(scale > 0.f && scale <= 3.4e38f, SG_EINVAL, "%s: scale must be positive and finite", fn);
    SG_REQUIRE((int64_t)B * Hkv <= 0x7fffffffll / (64 * D4_WAVES), SG_EUNSUPPORTED, "%s: too many units", fn);
    if (weight_out) {
        SG_REQUIRE(weight_stride >= (int64_t)max_pages * page_size, SG_EINVAL, "%s: weight rows of %lld floats hold no %lld rows",
                   fn, (long long)weight_stride, (long long)max_pages * page_size);
        SG_REQUIRE(decay >= 0.f && decay <= 1.f, SG_EINVAL, "%s: decay must lie in [0, 1]", fn);
    }
    SG_REQUIRE(weight_out || !weight_in, SG_EINVAL, "%s: weight_in without weight_out", fn);
    if (B == 0) return SG_OK;
    SG_REQUIRE(q && page_table && n_rows && out && (pool_rows == 0 || (k_pool && v_pool && s_pool)), SG_EINVAL,
               "%s: null pointer", fn);
    SG_REQUIRE(aligned16(q) && aligned16(k_pool) && aligned16(v_pool) && aligned16(s_pool) && aligned16(ws), SG_EINVAL,
               "%s: q, pools and workspace must be 16-byte aligned", fn);
    const float sl2 = scale * 1.4426950408889634f;     // log2(e)
    hipStream_t s = as_stream(stream);
    const Weights w{weight_in, weight_out, weight_stride, decay, nullptr, 0};
    float *wsf = reinterpret_cast<float *>(ws);
#define SG_D4(T, D)                                                                                                  \
    launch_decode4<T, D>(fn, s, B, Hq, Hkv, sl2, q, k_pool, v_pool, s_pool, pool_rows, page_table, n_rows, page_size, \
                         max_pages, out, w, wsf, ws_bytes)
    if (dt == SG_F32) return d == 64 ? SG_D4(float, 64) : SG_D4(float, 128);
    return d == 64 ? SG_D4(uint16_t, 64) : SG_D4(uint16_t, 128);
#undef SG_D4
}
