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
// A state's factor is 1 where its max is the joint one, so a set whose logits
// are all NaN keeps its NaN sums; one without rows, or with -inf alone, gives
// zeros.
#pragma once

#include "sg_internal.h"

namespace sg {

constexpr int FINISH_THREADS = 256;
constexpr int FINISH_ROWS = FINISH_THREADS * 4;      // rows per workgroup
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

// Grid: x = unit, y = chunk of FINISH_ROWS rows (chunk 0 also writes the
// unit's outputs).  States of a unit: nsplit places, of which the used ones come
// first; or, with `spans`, places unit + spans[unit].x .. unit + spans[unit].y,
// where a unit with one state and no weights has its output already.
template <int D>
static __global__ __launch_bounds__(FINISH_THREADS) void decode_finish_kernel(
    int Hq, int Hkv, int nsplit, const int32_t *__restrict__ n_rows, int64_t max_rows, int64_t split_rows,
    const int2 *__restrict__ spans, const float *__restrict__ states, float *__restrict__ out, Weights w) {
    __shared__ float M[FINISH_MAX_G], inv[FINISH_MAX_G];
    const int G = Hq / Hkv;
    const int64_t unit = blockIdx.x;
    const int64_t n = max<int64_t>(0, min<int64_t>(n_rows[unit], max_rows));
    if (blockIdx.y > 0 && (int64_t)blockIdx.y * FINISH_ROWS >= n) return;      // uniform
    int used = used_splits(n, nsplit, split_rows);
    int64_t first = unit * nsplit;
    if (spans && n > 0) {
        const int2 sp = spans[unit];
        if (sp.x == sp.y && !w.out) return;      // uniform
        used = sp.y - sp.x + 1;
        first = unit + sp.x;
    }
    const float *st = states + first * G * (int64_t)(D + 2);
    const int lane = threadIdx.x % 64;
    for (int g = threadIdx.x / 64; g < G; g += FINISH_THREADS / 64) {
        float m = -INFINITY, l = 0.f;
        for (int s = lane; s < used; s += 64) m = fmaxf(m, st[((int64_t)s * G + g) * (D + 2)]);
        m = wave_max(m);
        for (int s = lane; s < used; s += 64) {
            const float *p = st + ((int64_t)s * G + g) * (D + 2);
            l += p[1] * (p[0] == m ? 1.f : __builtin_amdgcn_exp2f(p[0] - m));
        }
        l = wave_sum(l);
        if (lane == 0) {
            M[g] = m;
            inv[g] = l == 0.f ? 0.f : 1.f / l;
        }
    }
    __syncthreads();
    if (blockIdx.y == 0) {
        const int b = (int)(unit / Hkv), h = (int)(unit % Hkv);
        for (int i = threadIdx.x; i < G * D; i += FINISH_THREADS) {
            const int g = i / D, c = i % D;
            float o = 0.f;
            for (int s = 0; s < used; ++s) {
                const float *p = st + ((int64_t)s * G + g) * (D + 2);
                o += p[2 + c] * (p[0] == M[g] ? 1.f : __builtin_amdgcn_exp2f(p[0] - M[g]));
            }
            out[((int64_t)b * Hq + (int64_t)h * G + g) * D + c] = o * inv[g];
        }
    }
    if (!w.out) return;
    const int64_t i0 = (int64_t)blockIdx.y * FINISH_ROWS + threadIdx.x;
    for (int j = 0; j < 4; ++j) {
        const int64_t i = i0 + j * FINISH_THREADS;
        if (i >= n) break;
        float p = 0.f;
        for (int g = 0; g < G; ++g) {
            const float z = w.z[(unit * G + g) * w.z_stride + i];
            const float e = __builtin_amdgcn_exp2f(z - (M[g] == -INFINITY ? 0.f : M[g]));
            p += inv[g] == 0.f ? 0.f : e * inv[g];     // (an empty pool leaves z unwritten)
        }
        const float old = w.in ? w.decay * w.in[unit * w.stride + i] : 0.f;
        w.out[unit * w.stride + i] = old + p;
    }
}

}  // namespace sg
