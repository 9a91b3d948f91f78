// The second launch of a decode attention that accumulates weights: joins the
// split states of a unit (per head: max m in log2 units, sum l, output o) and
// turns the logits z (log2 units) that the first launch left in the workspace
// into the weights the unit's rows received,
//
//   weight_out[i] = decay * weight_in[i] + sum over g of 2^(z[g][i] - M_g) / L_g
//
// z is [units][G][z_stride], states as the split states of sg_decode_attn.
// (Weights need the final max and sum of every head, so either the logits are
// kept, 4 G bytes per row written and read, or the keys are read again.)
//
// Of 64 requests of 245 to 3,932 rows, 4 heads per unit: 6.0 us for the outputs,
// 10.6 with the weights (26 MB of logits and weights); of one request 3.6 to 3.9.
//
// A state's factor is 1 where its max is the joint one, so a set whose logits
// are all NaN keeps its NaN sums; one without rows, or with -inf alone, gives
// zeros.
#pragma once

#include "sg_internal.h"

namespace sg {

constexpr int FINISH_MAX_G = 16;

struct Weights {
    const float *in;      // NULL: zeros
    float *out;           // NULL: no weights
    int64_t stride;       // floats per unit
    float decay;
    float *z;             // logits in the workspace
    int64_t z_stride;
};

// Floats of a head's logits of a unit in the workspace (whole tiles of 32, so
// that a tile is stored without a look at its rows).
inline int64_t z_stride_of(int64_t max_rows) { return ceil_div(max_rows, 32) * 32; }

// Splits of a unit of n rows that wrote a state (split_rows == 0: equal parts).
__device__ __forceinline__ int used_splits(int64_t n, int nsplit, int64_t split_rows) {
    return split_rows > 0 ? (int)min<int64_t>(nsplit, ceil_div(n, split_rows)) : (n > 0 ? nsplit : 0);
}

// Grid: x = unit; y below G: a head's outputs, THREADS / D threads per channel
// sharing its states; then chunks of 4 * THREADS rows' weights, a grid stride apart.  States of a unit: nsplit places, of
// which the used ones come first; or, with `spans`, places unit +
// spans[unit].x .. unit + spans[unit].y, where a unit with one state and no
// weights has its output already.
//
// Latency alone for small calls: the loads of a step are issued together (row
// count and span, then eight states per thread; for the weights the rows' logits
// of four heads), so either kind of block takes three round trips.
template <int D, int THREADS>
static __global__ __launch_bounds__(THREADS) void decode_finish_kernel(
    int G, int nsplit, const int32_t *__restrict__ n_rows, int64_t max_rows, int64_t split_rows,
    const int2 *__restrict__ spans, const float *__restrict__ states, float *__restrict__ out, Weights w) {
    constexpr int GROUP = 8;       // states whose loads are in flight together
    constexpr int ROWS = THREADS * 4;
    const int64_t unit = blockIdx.x;
    const int2 sp = spans ? spans[unit] : make_int2(0, 0);
    const int64_t n = max<int64_t>(0, min<int64_t>(n_rows[unit], max_rows));
    const int chunk = (int)blockIdx.y - G;
    if (chunk >= 0 && (int64_t)chunk * ROWS >= n) return;       // uniform
    int used = used_splits(n, nsplit, split_rows);
    int64_t first = unit * nsplit;
    if (spans && n > 0) {
        if (sp.x == sp.y && !w.out) return;      // uniform
        used = sp.y - sp.x + 1;
        first = unit + sp.x;
    }
    const float *st = states + first * G * (int64_t)(D + 2);
    const int64_t step = (int64_t)G * (D + 2);

    if (chunk < 0) {
        constexpr int SHARE = THREADS / D;
        __shared__ float part[SHARE][3][D];      // max, sum and output of each thread's states
        const int g = blockIdx.y, c = threadIdx.x % D, k = threadIdx.x / D;
        const float *p = st + (int64_t)g * (D + 2);
        float M = -INFINITY, L = 0.f, O = 0.f;
        auto join = [&](float m, float l, float o) {       // in a fixed order
            const float top = fmaxf(M, m);
            const float f = M == top ? 1.f : __builtin_amdgcn_exp2f(M - top), a = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
            L = f * L + a * l;
            O = f * O + a * o;
            M = top;
        };
        for (int s0 = k * GROUP; s0 < used; s0 += SHARE * GROUP) {
            float m[GROUP], l[GROUP], o[GROUP];
#pragma unroll
            for (int j = 0; j < GROUP; ++j) {
                const float *x = p + min(s0 + j, used - 1) * step;
                m[j] = x[0];
                l[j] = x[1];
                o[j] = x[2 + c];
            }
#pragma unroll
            for (int j = 0; j < GROUP; ++j)
                if (s0 + j < used) join(m[j], l[j], o[j]);
        }
        if (used > GROUP) {                      // uniform; else the first thread has them all
            part[k][0][c] = M;
            part[k][1][c] = L;
            part[k][2][c] = O;
            __syncthreads();
            if (k == 0)
                for (int j = 1; j < SHARE; ++j) join(part[j][0][c], part[j][1][c], part[j][2][c]);
        }
        if (k == 0) out[(unit * G + g) * D + c] = L == 0.f ? 0.f : O / L;
        return;
    }

    __shared__ float M_s[FINISH_MAX_G], inv_s[FINISH_MAX_G];
    const int lane = threadIdx.x % 64;
    for (int g = threadIdx.x / 64; g < G; g += THREADS / 64) {
        const float *p = st + (int64_t)g * (D + 2);
        float M = -INFINITY, L = 0.f;
        for (int s0 = 0; s0 < used; s0 += 64) {
            const bool in = s0 + lane < used;
            const float *x = p + min(s0 + lane, used - 1) * step;
            const float m = x[0], l = x[1];
            const float top = fmaxf(M, wave_max(m));
            const float a = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
            const float sum = wave_sum(in ? a * l : 0.f);
            L = L * (M == top ? 1.f : __builtin_amdgcn_exp2f(M - top)) + sum;
            M = top;
        }
        if (lane == 0) {
            M_s[g] = M == -INFINITY ? 0.f : M;
            inv_s[g] = L == 0.f ? 0.f : 1.f / L;
        }
    }
    __syncthreads();
    // four rows per thread, four heads at a time (rows past n lie within the
    // unit's logits, or are not read)
    for (int64_t base = (int64_t)chunk * ROWS; base < n; base += (int64_t)(gridDim.y - G) * ROWS) {
        const int64_t i = base + threadIdx.x * 4;
        if (i >= n) break;
        float add[4] = {0.f, 0.f, 0.f, 0.f}, old[4];
        const int64_t at = unit * w.stride + i;
#pragma unroll
        for (int j = 0; j < 4; ++j) old[j] = w.in && i + j < n ? w.in[at + j] : 0.f;
        for (int g0 = 0; g0 < G; g0 += 4) {
            float4 z[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                z[k] = *reinterpret_cast<const float4 *>(w.z + (unit * G + min(g0 + k, G - 1)) * w.z_stride + i);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (g0 + k < G && inv_s[g0 + k] != 0.f) {      // (an empty pool leaves z unwritten)
                    const float M = M_s[g0 + k], f = inv_s[g0 + k];
                    add[0] += __builtin_amdgcn_exp2f(z[k].x - M) * f;
                    add[1] += __builtin_amdgcn_exp2f(z[k].y - M) * f;
                    add[2] += __builtin_amdgcn_exp2f(z[k].z - M) * f;
                    add[3] += __builtin_amdgcn_exp2f(z[k].w - M) * f;
                }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < n) w.out[at + j] = w.decay * old[j] + add[j];
    }
}

// Threads of a block that joins about `expect` states per unit: eight states
// each in one go, a block of 1,024 threads for a head's few hundred, of 128
// where every unit has a handful and the heads fill the chip.  `expect` is the
// mean: where one unit is far longer than the others, its states take rounds one
// after another (4-bit rows, one request of 32,768 rows beside 63 of 300: 42.7
// us; the same rows spread evenly 4.3).
inline int finish_threads(int d, int64_t expect) {
    const int64_t threads = ceil_div(expect, 8) * d;
    return threads <= 128 ? 128 : threads <= 256 ? 256 : threads <= 512 ? 512 : 1024;
}

template <int D>
static void launch_finish(hipStream_t s, int64_t units, int G, int64_t expect, int nsplit, const int32_t *n_rows,
                          int64_t max_rows, int64_t split_rows, const int2 *spans, const float *states, float *out,
                          const Weights &w) {
    auto launch = [&](auto kernel, int threads) {
        // (chunks past the launch's limit are taken in strides)
        const int64_t chunks = w.out ? std::min<int64_t>(ceil_div(max_rows, threads * 4), 32768) : 0;
        const dim3 grid((unsigned)units, (unsigned)(G + chunks));
        kernel<<<grid, threads, 0, s>>>(G, nsplit, n_rows, max_rows, split_rows, spans, states, out, w);
    };
    switch (finish_threads(D, expect)) {
        case 128: return launch(decode_finish_kernel<D, 128>, 128);
        case 256: return launch(decode_finish_kernel<D, 256>, 256);
        case 512: return launch(decode_finish_kernel<D, 512>, 512);
        default: return launch(decode_finish_kernel<D, 1024>, 1024);
    }
}

}  // namespace sg
