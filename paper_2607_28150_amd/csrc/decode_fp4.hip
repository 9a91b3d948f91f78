// sg_decode_attn_fp4: GQA decode attention over a paged set of 4-bit rows
// (fp4.h), with or without the weights the rows receive (decode_weights.h).
//
// Work.  Every (sequence, KV head) unit is cut into tiles of 32 rows, and the
// tiles of all units stand in one line, of which as many wavefronts as the chip
// holds (Plan4) take equal shares: the end of one unit, whole
// units, the start of another.  A wavefront serves all G <= 16 query heads of a
// unit and leaves a state for every unit it touches; a second launch joins
// them.  Wavefronts are workgroups of their own: nothing waits for another, and
// the loads run on across the units of a share.  (Workgroups of four wavefronts
// that shared a unit's rows and met at its end: 64 requests 66 us, 16 long
// prompts 82.)  More units than one lookup covers: a wavefront takes a whole one.
//
// Memory.  A wavefront streams its tiles through an LDS ring with direct
// global->LDS loads, NS - 1 tiles ahead of its arithmetic, the tiles' page
// entries another NS - 1 tiles ahead of those: codes of 16 K and 16 V rows per
// instruction (d = 128), the tile's scales in one more.  Every step issues the
// same loads, so one constant counter wait covers a tile's rows and the page
// entries that are due with it.  A lane may fetch any row into its place of
// the ring, so the places are chosen for the reads: K's 16-byte pieces rotated
// against the bank conflicts of whole rows, V's rows in the order 0, 4, 8, 12,
// 1, ... in which four quarters of a wavefront read them.
//
// Arithmetic.  Matrix instructions (16 x 16 x 32, bf16 in, fp32 out):
//   logits : A = 16 K rows x 32 channels, B = the same channels of 16 heads.
//            The channels of a product may come in any order, so lane (row m,
//            quarter kg) takes kg's d / 4 consecutive channels of its row, 8 of
//            them per instruction.
//   values : A = 16 heads x 32 rows (the probabilities), B = 32 rows x 16
//            channels.  The logits leave head n, rows 4 kg .. 4 kg + 3 of both
//            16-row halves in lane (n, kg): taken as that lane's 8 of the 32
//            rows, the probabilities are where the next product wants them.
//            Lane (n, kg) reads the matching 8 V rows, d / 16 consecutive
//            channels each, one channel per instruction.
// 4-bit values times their scale are exact in bf16.  Queries in bf16 are too;
// fp32 queries and the probabilities are cut into three bf16 parts of 8 bits
// that add up to them exactly, so nothing is rounded below fp32.
//
// Bound by memory where the work is large (16 prompts of 8K to 32K rows: 68 us
// for 321 MB, 4.7 TB/s, the rate of a device copy; whole calls differ by 7 us
// from card to card; the counters see every byte read once), by start and end
// where it is not: a launch, the lookup, the first rows' round trips and the
// states are what 64 requests of 146 MB take beyond a copy's time, 6 of 36.5 us,
// and nearly all of 7.2 us for one.  Vector instructions fill 47% of a SIMD's
// cycles in the batch, matrix instructions 17%.
//
// Softmax as in sg_decode_attn: online in log2 units against a reference max
// per head that is raised only when a logit passes it by 2^16.
#include "decode_weights.h"
#include "fp4.h"

namespace sg {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2u __attribute__((ext_vector_type(2), aligned(4)));     // outputs may start at any float

constexpr int D4_TILE = 32;                  // rows per step
constexpr float D4_LAZY = 16.f;              // log2 headroom before the reference max is raised
constexpr int D4_MIN_SHARE = 2;              // tiles of a share at least
constexpr int D4_SHARED_UNITS = 64 * 64;     // most units shared that way

// Wavefronts of a launch and their rings.  Three wavefronts per SIMD with a ring
// of two tiles stream as much as two with three, and hide more of the arithmetic's
// latency (4.84 against 4.69 TB/s over 570 MB, 64 requests of 2,048 rows 39.6
// against 40.7 us; deeper rings 0.8 to 0.9 of that); fp32 queries take registers
// for two.
template <typename T>
struct Plan4 {
    static constexpr int WAVES = sizeof(T) == 4 ? 2 : 3;      // per SIMD
    static constexpr int NS = sizeof(T) == 4 ? 3 : 2;         // ring slots
    static constexpr int SHARES = WAVES * 4 * 256;            // wavefronts that share the tiles of all units
};

// One ring slot: a tile's K codes, V codes and scales.
template <int D>
struct Tile4 {
    static constexpr int CODES = D4_TILE * D / 2;
    static constexpr int SB = 2 * D / FP4_BLOCK;     // scale bytes per row: K's, then V's
    static constexpr int SLOT = 2 * CODES + 256;
    static constexpr int LOADS = 2 * CODES / 1024 + 1;     // of a tile
};

__device__ __forceinline__ bf16x8 as_bf16x8(const v4u &w) {
    bf16x8 r;
    __builtin_memcpy(&r, &w, sizeof(r));
    return r;
}

// x cut into three parts of 8 significant bits each, in the high halves of
// p[0], p[1], p[2] (what the low halves hold does not count): their sum is x,
// less what lies below 2^-133, the least bf16.
__device__ __forceinline__ void split3(float x, uint32_t (&p)[3]) {
    p[0] = __float_as_uint(x);
    const float r = x - __uint_as_float(p[0] & 0xffff0000u);
    p[1] = __float_as_uint(r);
    p[2] = __float_as_uint(r - __uint_as_float(p[1] & 0xffff0000u));
}
// The high halves of two words, or their low halves, as a pair.
__device__ __forceinline__ uint32_t high_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }
__device__ __forceinline__ uint32_t low_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x05040100u); }

// Direct global->LDS load of 4 bytes per lane: lane i's land at LDS offset
// lds + 4 i (see dma16 in sg_internal.h).
__device__ __forceinline__ void dma4(const void *src, unsigned lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void dma4_nt(const void *src, unsigned lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off nt" ::"v"(src), "{m0}"(lds) : "memory");
}

// The same loads from a uniform base and a 32-bit offset per lane.  (Five wait
// states: a scalar register that a vector instruction wrote may not be read by
// a load before, and the compiler does not look into the assembly.  Unoptimised
// builds, which check the host side, keep no pointer in scalar registers.)
__device__ __forceinline__ void dma16_nt(const void *base, unsigned off, unsigned lds) {
#ifdef __OPTIMIZE__
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
#else
    dma16_nt(reinterpret_cast<const char *>(base) + off, lds);
#endif
}

// A uniform load through the scalar cache of data that nothing writes during
// the kernel (the constant address space says so).
__device__ __forceinline__ int32_t scalar_load(const int32_t *p) {
    return *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(p));
}

struct Decode4Args {
    int Hq, Hkv;
    float scale_log2;
    const void *q;
    const uint8_t *k_pool, *v_pool, *s_pool;
    int64_t pool_rows;
    const int32_t *page_table, *n_rows;
    int page_size, max_pages, units;
    uint32_t page_mul;
    int page_shift;
    float *out, *states;
    int2 *spans;           // per unit: first and last wavefront that left a state (shared tiles)
    float *z;              // logits [units][G][z_stride], or unused
    int64_t z_stride;
};

// A place in a share: tile `tile` of unit `unit` (n rows); `left` tiles of the
// share from here on.
struct Cursor4 {
    int unit, tile, n, left;
};

// T: type of the queries; KEEP: the logits are kept for the weights and every
// unit leaves a state; SHARED: wavefronts share the tiles of all units; HALVES:
// pages are multiples of 16 rows, so each half of a tile lies in one page.
template <typename T, int D, bool KEEP, bool SHARED, bool HALVES>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(Plan4<T>::WAVES))) void decode4_kernel(Decode4Args a) {
    using L = Tile4<D>;
    constexpr int STEPS = D / 32;            // K products per 16 rows: 8 channels of every lane each
    constexpr int NC = D / 16;               // V channels per lane, and products per 32 rows
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int NS = Plan4<T>::NS, SB = L::SB;
    static_assert((NS - 1) * (L::LOADS + 1) <= 63, "loads in flight");
    __shared__ __attribute__((aligned(16))) char ring[NS * L::SLOT];
    __shared__ int32_t entries[HALVES ? 1 : NS][64];      // page entries of a tile's rows (each twice)

    const int lane = threadIdx.x, n16 = lane % 16, kg = lane / 16;
    const int Hq = a.Hq, Hkv = a.Hkv, G = Hq / Hkv, page_size = a.page_size;
    const int64_t max_rows = (int64_t)a.max_pages * page_size;
    auto rows_of = [&](int u) { return (int)max<int64_t>(0, min<int64_t>((int64_t)a.n_rows[u], max_rows)); };
    auto rows_of_unit = [&](int u) { return (int)max<int64_t>(0, min<int64_t>((int64_t)scalar_load(a.n_rows + u), max_rows)); };
    auto tiles_of = [](int n) { return (n + D4_TILE - 1) / D4_TILE; };
    Cursor4 cur{(int)blockIdx.x, 0, 0, 0};
    int near = 0, n_near = 0;                // lane i: rows of unit near + i
    if constexpr (SHARED) {
        // The tile this share starts with: lane i sums the tiles of units [64 i,
        // 64 i + 64), read whole lines at a time (strided, a lane's units side by
        // side, 2,048 units took 6 to 8 us longer); the lane whose 64 hold it,
        // then the unit.
        const int per = (a.units + 63) / 64;         // at most 64
        int mine = 0, first8[8];
        auto rows8 = [&](int i0, int (&n)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) n[i] = a.n_rows[min((i0 + i) * 64 + lane, a.units - 1)];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = (i0 + i) * 64 + lane < a.units;
                n[i] = in ? (int)max<int64_t>(0, min<int64_t>(n[i], max_rows)) : 0;
                if (i0 + i < per) {          // uniform
                    const int sum = __builtin_amdgcn_readlane(wave_scan_incl(tiles_of(n[i])), 63);
                    mine = lane == i0 + i ? sum : mine;
                }
            }
        };
        rows8(0, first8);
        for (int i0 = 8; i0 < per; i0 += 8) {
            int n[8];
            rows8(i0, n);
        }
        const int upto = wave_scan_incl(mine), total = __builtin_amdgcn_readlane(upto, 63);      // below 2^31
        // Tiles of a share, at least: its time goes with them, that of joining a
        // unit's shares with their number, so a part of the root of a unit's tiles
        // (of 0, 0.3, 0.5 and 1 times the root, one request of 32,768 rows 36, 28.5,
        // 31.3 and 46.5 us, of 819 rows within 1 us for the first three).  Never a
        // share without a tile: a unit's states lie side by side.
        const int tiles = max(D4_MIN_SHARE, (int)(0.3f * sqrtf((float)total / (float)a.units)));
        const int shares = max(1, min((int)gridDim.x, total / tiles)), share = (int)blockIdx.x;
        if (share >= shares || total == 0) return;
        // total / shares tiles each, the first total % shares one more
        const int each = total / shares, more = total - each * shares;
        const int p0 = share * each + min(share, more), p1 = p0 + each + (share < more ? 1 : 0);
        const int at = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(p0 < upto)) - 1);
        const int before = __builtin_amdgcn_readlane(upto - mine, at);
        near = at * 64;
        if (at < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) n_near = at == i ? first8[i] : n_near;
        } else {
            n_near = near + lane < a.units ? rows_of(near + lane) : 0;
        }
        const int t = tiles_of(n_near);
        const int end = before + wave_scan_incl(t);
        const int i = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(p0 < end)) - 1);
        cur.unit = near + i;
        cur.n = __builtin_amdgcn_readlane(n_near, i);
        cur.tile = p0 - __builtin_amdgcn_readlane(end - t, i);
        cur.left = p1 - p0;
    } else {
        cur.n = rows_of_unit(cur.unit);
        cur.left = tiles_of(cur.n);
    }
    auto advance = [&](Cursor4 &c) {
        if (--c.left <= 0) return;           // past the share it stays where it is
        if (++c.tile * D4_TILE < c.n) return;
        c.tile = 0;
        do {
            ++c.unit;                        // tiles are left, so units with rows are
            c.n = c.unit - near < 64 ? __builtin_amdgcn_readlane(n_near, c.unit - near) : rows_of_unit(c.unit);
        } while (c.n == 0);
    };

    unsigned valid = 0u;     // bit s: the row of slot s's tile that this lane stands for counts
    unsigned full = 0u;      // bit s: every row of slot s's tile counts
    // Loads of a tile whose row i lies at pool row `row` of lanes i and i + 32.
    auto load_rows = [&](int row, int slot) {
        const unsigned base = lds_addr(ring + slot * L::SLOT);
        if constexpr (D == 128) {
            const int m4 = lane / 4, piece = lane % 4;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t kr = __shfl(row, 16 * u + m4, 64);
                dma16_nt(a.k_pool + kr * 64 + (piece ^ (m4 / 4)) * 16, base + u * 1024);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t vr = __shfl(row, 16 * u + (m4 % 4) * 4 + m4 / 4, 64);
                dma16_nt(a.v_pool + vr * 64 + piece * 16, base + L::CODES + u * 1024);
            }
            const int64_t sr = __shfl(row, lane / 2, 64);
            dma4_nt(a.s_pool + sr * 8 + (lane % 2) * 4, base + 2 * L::CODES);
        } else {
            const int p = lane / 2, piece = lane % 2;
            const int64_t kr = __shfl(row, p, 64);
            dma16_nt(a.k_pool + kr * 32 + piece * 16, base);
            const int64_t vr = __shfl(row, (p / 16) * 16 + (p % 4) * 4 + (p % 16) / 4, 64);
            dma16_nt(a.v_pool + vr * 32 + piece * 16, base + L::CODES);
            dma4_nt(a.s_pool + (int64_t)row * 4, base + 2 * L::CODES);     // lanes 32 .. 63: the same again
        }
    };
    // The same where the halves of the tile are 16 consecutive pool rows each,
    // from x0 and x1 on: nothing but the scales' addresses takes vector work.
    const unsigned k_off = D == 128 ? lane / 4 * 64 + (lane % 4 ^ lane / 16) * 16 : lane % 32 * 16;
    const unsigned v_off = D == 128 ? (lane / 4 % 4 * 4 + lane / 16) * 64 + lane % 4 * 16
                                    : (lane / 2 % 4 * 4 + lane / 2 % 16 / 4) * 32 + lane % 2 * 16;
    auto load_halves = [&](int x0, int x1, int slot) {
        const unsigned base = lds_addr(ring + slot * L::SLOT);
        if constexpr (D == 128) {
            dma16_nt(a.k_pool + (int64_t)x0 * 64, k_off, base);
            dma16_nt(a.k_pool + (int64_t)x1 * 64, k_off, base + 1024);
            dma16_nt(a.v_pool + (int64_t)x0 * 64, v_off, base + L::CODES);
            dma16_nt(a.v_pool + (int64_t)x1 * 64, v_off, base + L::CODES + 1024);
            const int64_t x = lane < 32 ? x0 : x1;
            dma4_nt(a.s_pool + x * 8 + lane % 32 * 4, base + 2 * L::CODES);
        } else {
            // lanes 0 .. 31 the first half, 32 .. 63 the second
            const int64_t x = lane < 32 ? x0 : x1;
            dma16_nt(a.k_pool + x * 32 + k_off, base);
            dma16_nt(a.v_pool + x * 32 + v_off, base + L::CODES);
            const int64_t y = lane % 32 < 16 ? x0 : x1;
            dma4_nt(a.s_pool + (y + lane % 16) * 4, base + 2 * L::CODES);
        }
    };
    // Row of a tile that a lane stands for, its page and its place there
    auto locate = [&](const Cursor4 &c, int &lr, uint32_t &page, int &off) {
        lr = c.tile * D4_TILE + lane % 32;
        const uint32_t in = (uint32_t)min(lr, c.n - 1);
        page = (uint32_t)(((uint64_t)in * a.page_mul) >> a.page_shift);
        off = (int)(in - page * (uint32_t)page_size);
    };
    auto issue_entries = [&](const Cursor4 &c, int slot) {
        int lr, off;
        uint32_t page;
        locate(c, lr, page, off);
        dma4(a.page_table + (int64_t)c.unit * a.max_pages + page, lds_addr(&entries[slot][0]));
    };
    // Loads of a tile's rows into a ring slot.  A row that is left out (past the
    // unit's rows or the share, or outside the pool) reads pool row 0.
    auto issue_rows = [&](const Cursor4 &c, int slot) {
        int lr, off;
        uint32_t page;
        locate(c, lr, page, off);
        const int64_t x = (int64_t)entries[slot][lane] + off;
        const bool ok = c.left > 0 && lr < c.n && x >= 0 && x < a.pool_rows;
        valid = (valid & ~(1u << slot)) | ((ok ? 1u : 0u) << slot);
        full &= ~(1u << slot);
        load_rows(ok ? (int)x : 0, slot);
    };
    // Pool rows of the halves of a tile (below 2^32, as the entries give them)
    auto half_rows = [&](const Cursor4 &c, int64_t &x0, int64_t &x1) {
        const int32_t *pt = a.page_table + (int64_t)c.unit * a.max_pages;
        const uint32_t r0 = (uint32_t)c.tile * D4_TILE, r1 = r0 + 16 < (uint32_t)c.n ? r0 + 16 : r0;
        const uint32_t p0 = (uint32_t)(((uint64_t)r0 * a.page_mul) >> a.page_shift);
        const uint32_t p1 = (uint32_t)(((uint64_t)r1 * a.page_mul) >> a.page_shift);
        x0 = (int64_t)scalar_load(pt + p0) + (int)(r0 - p0 * (uint32_t)page_size);
        x1 = (int64_t)scalar_load(pt + p1) + (int)(r1 - p1 * (uint32_t)page_size);
    };
    auto issue_halves = [&](const Cursor4 &c, int64_t x0, int64_t x1, int slot) {
        if (c.left > 0 && (c.tile + 1) * D4_TILE <= c.n && min(x0, x1) >= 0 && max(x0, x1) + 16 <= a.pool_rows) {
            full |= 1u << slot;
            load_halves((int)x0, (int)x1, slot);
        } else {
            const int64_t x = (lane % 32 < 16 ? x0 : x1) + lane % 16;
            const bool ok = c.left > 0 && c.tile * D4_TILE + lane % 32 < c.n && x >= 0 && x < a.pool_rows;
            valid = (valid & ~(1u << slot)) | ((ok ? 1u : 0u) << slot);
            full &= ~(1u << slot);
            load_rows(ok ? (int)x : 0, slot);
        }
    };

    bf16x8 qf[PARTS][STEPS];                 // head n16, channels of quarter kg, 8 per product
    float m, l;                              // of head n16 (l: this lane's rows)
    f32x4 o[NC];                             // o[j][i]: head 4 kg + i, channel NC n16 + j
    int begun = cur.tile;                    // first tile taken of the current unit
    float scale = a.scale_log2;              // of head n16's logits
    auto begin_unit = [&](int unit) {
        const int b = unit / Hkv, h = unit % Hkv;
        const T *qp = reinterpret_cast<const T *>(a.q) +
                      ((int64_t)b * Hq + (int64_t)h * G + min(n16, G - 1)) * D + kg * (D / 4);
        if constexpr (PARTS == 1) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const v4u w = *reinterpret_cast<const v4u *>(qp + s * 8);
                qf[0][s] = as_bf16x8(n16 < G ? w : v4u{0u, 0u, 0u, 0u});
            }
        } else {
            float x[STEPS][8], top = 0.f;
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const v4u w = *reinterpret_cast<const v4u *>(qp + s * 8 + i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[s][i + j] = __uint_as_float(w[j]);
                }
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[s][i]));
            auto cut = [&](auto split) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    v4u w[PARTS];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t c[3], e[3];
                        split(x[s][2 * i], c);
                        split(x[s][2 * i + 1], e);
#pragma unroll
                        for (int p = 0; p < 3; ++p) w[p][i] = high_halves(c[p], e[p]);
                    }
#pragma unroll
                    for (int p = 0; p < 3; ++p) qf[p][s] = as_bf16x8(n16 < G ? w[p] : v4u{0u, 0u, 0u, 0u});
                }
            };
            scale = a.scale_log2;
            if (__all(top >= 0x1p-60f && top < INFINITY)) {          // uniform
                cut(split3);
            } else {
                // Parts below 2^-133 do not exist in bf16: a head of small values
                // is taken 2^48 times, where the least bit of any float lies above
                // that and 128 products with the largest key (6 * 2^125) stay
                // finite.  An infinity is its first part alone.
                const uint64_t large = __ballot(top >= 0x1p-60f);    // bit 16 kg + n16
                const bool small = !(((large | large >> 16 | large >> 32 | large >> 48) >> n16) & 1u);
                const float up = small ? 0x1p48f : 1.f;
                if (small) scale *= 0x1p-48f;
                cut([&](float v, uint32_t (&p)[3]) {
                    split3(v * up, p);
                    if (fabsf(v) == INFINITY) p[1] = p[2] = 0u;
                });
            }
        }
        // waited for here, once per unit: the compiler does not see the ring's
        // loads and would otherwise drain them at every step
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) asm volatile("" ::"v"(qf[p][s]));
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    // The unit's state, or its outputs where this share held all of it.
    auto end_unit = [&](int unit, bool last) {
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        const bool whole = !KEEP && begun == 0 && last;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int64_t slot = SHARED ? (int64_t)unit + blockIdx.x : unit;   // both only go up: their sum numbers the states
        float *st = a.states + slot * G * (D + 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int g = 4 * kg + i;
            const float f = __shfl(inv, g, 64);
            if (g >= G) continue;
            float *p = whole ? a.out + ((int64_t)unit * G + g) * D + NC * n16 : st + g * (D + 2) + 2 + NC * n16;
#pragma unroll
            for (int j = 0; j < NC; j += 2)
                *reinterpret_cast<f32x2u *>(p + j) = whole ? f32x2u{o[j][i] * f, o[j + 1][i] * f}
                                                           : f32x2u{o[j][i], o[j + 1][i]};
        }
        if (!whole && kg == 0 && n16 < G) *reinterpret_cast<float2 *>(st + n16 * (D + 2)) = make_float2(m, l);
        if constexpr (SHARED) {
            if (lane == 0) {
                if (begun == 0) a.spans[unit].x = blockIdx.x;
                if (last) a.spans[unit].y = blockIdx.x;
            }
        }
    };

    if (cur.left == 0) {                     // a whole unit without rows
        begin_unit(cur.unit);
        end_unit(cur.unit, true);
        return;
    }
    Cursor4 rows = cur, ents = cur;
    const int steps = cur.left;
    int64_t x0 = 0, x1 = 0;                  // halves of the tile `rows` stands at
    if constexpr (HALVES) {
        half_rows(rows, x0, x1);
        begin_unit(cur.unit);
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) {
            issue_halves(rows, x0, x1, s);
            advance(rows);
            half_rows(rows, x0, x1);
        }
    } else {
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) {
            issue_entries(ents, s);
            advance(ents);
        }
        begin_unit(cur.unit);                // its queries on the same round trip
        wait_vmem<0>();
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) {
            issue_rows(rows, s);
            advance(rows);
            issue_entries(ents, (s + NS - 1) % NS);
            advance(ents);
        }
    }
    for (int st = 0; st < steps; ++st) {
        // This step's rows (and the entries of the rows issued next) have
        // landed: what else was issued since, logits and states, only makes the
        // wait stricter.
        if constexpr (HALVES) {
            issue_halves(rows, x0, x1, (st + NS - 1) % NS);
            advance(rows);
            half_rows(rows, x0, x1);
            wait_vmem<(NS - 1) * L::LOADS>();
        } else {
            wait_vmem<(NS - 2) * (L::LOADS + 1)>();
            issue_rows(rows, (st + NS - 1) % NS);
            advance(rows);
            issue_entries(ents, (st + NS - 2) % NS);
            advance(ents);
        }
        const int slot = st % NS;
        const char *sb = ring + slot * L::SLOT;
        const uint8_t *sc = reinterpret_cast<const uint8_t *>(sb + 2 * L::CODES);
        // bit i: row i of the tile counts
        const uint32_t live = (full >> slot) & 1u ? 0xffffffffu : (uint32_t)__ballot((valid >> slot) & 1u);
        // logits: lane (n16, kg) of half u gets rows 16 u + 4 kg + i of head n16
        float z[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int row = 16 * u + n16;
            uint32_t kw[STEPS];
            uint32_t byte;
            if constexpr (D == 128) {
                const v4u x = *reinterpret_cast<const v4u *>(sb + row * 64 + ((kg ^ (n16 / 4)) * 16));
#pragma unroll
                for (int s = 0; s < STEPS; ++s) kw[s] = x[s];
                byte = sc[row * SB + kg];
            } else {
                const uint2 x = *reinterpret_cast<const uint2 *>(sb + row * 32 + kg * 8);
                kw[0] = x.x;
                kw[1] = x.y;
                byte = sc[row * SB + kg / 2];
            }
            const float ks = fp4_scale(byte);
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const bf16x8 kf = as_bf16x8(v4u{fp4_bf16_pair<0>(kw[s], ks), fp4_bf16_pair<1>(kw[s], ks),
                                                fp4_bf16_pair<2>(kw[s], ks), fp4_bf16_pair<3>(kw[s], ks)});
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[p][s], acc, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * u + i] = acc[i];         // unscaled
        }
        if (live != 0xffffffffu) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                z[i] = (live >> (16 * (i / 4) + 4 * kg + i % 4)) & 1u ? z[i] : -INFINITY;
        }
        if constexpr (KEEP) {
            if (n16 < G) {
                float *zp = a.z + ((int64_t)cur.unit * G + n16) * a.z_stride + (int64_t)cur.tile * D4_TILE + 4 * kg;
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    *reinterpret_cast<float4 *>(zp + 16 * u) =
                        make_float4(z[4 * u] * scale, z[4 * u + 1] * scale, z[4 * u + 2] * scale,
                                    z[4 * u + 3] * scale);
            }
        }
        float top = z[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, z[i]);
        top *= scale;
        if (__any(top > m + D4_LAZY)) {      // raise every head's reference (rare)
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float mn = fmaxf(m, top);
            const float f = mn == m ? 1.f : __builtin_amdgcn_exp2f(m - mn);
            l *= f;
            m = mn;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float fi = __shfl(f, 4 * kg + i, 64);
#pragma unroll
                for (int j = 0; j < NC; ++j) o[j][i] *= fi;
            }
        }
        const float ref = m == -INFINITY ? 0.f : m;
        uint32_t pw[3][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = __builtin_amdgcn_exp2f(fmaf(z[i], scale, -ref));
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
            const int place = 16 * (i / 4) + 4 * (i % 4) + kg, row = 16 * (i / 4) + 4 * kg + i % 4;
            const char *vp = sb + L::CODES + place * (D / 2);
            uint32_t byte = sc[row * SB + SB / 2 + n16 * NC / FP4_BLOCK];
            // a row that is left out stands on pool row 0: its zero
            // probability must not meet a NaN
            if (live != 0xffffffffu) byte = (live >> row) & 1u ? byte : 0u;
            const float vs = fp4_scale(byte);
            uint32_t w;
            if constexpr (NC == 8) w = *reinterpret_cast<const uint32_t *>(vp + n16 * 4);
            else w = *reinterpret_cast<const uint16_t *>(vp + n16 * 2);
            vb[i][0] = fp4_bf16_pair<0>(w, vs);
            vb[i][1] = fp4_bf16_pair<1>(w, vs);
            if constexpr (NC == 8) {
                vb[i][2] = fp4_bf16_pair<2>(w, vs);
                vb[i][3] = fp4_bf16_pair<3>(w, vs);
            }
        }
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            v4u w;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = j % 2 == 0 ? low_halves(vb[2 * i][j / 2], vb[2 * i + 1][j / 2])
                                    : high_halves(vb[2 * i][j / 2], vb[2 * i + 1][j / 2]);
            const bf16x8 vf = as_bf16x8(w);
#pragma unroll
            for (int k = 0; k < 3; ++k)
                o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[k], vf, o[j], 0, 0, 0);
        }
        const int unit = cur.unit;
        const bool last = (cur.tile + 1) * D4_TILE >= cur.n;
        advance(cur);
        if (last || cur.left <= 0) {
            end_unit(unit, last);
            if (cur.left > 0) {
                begun = 0;
                begin_unit(cur.unit);
            }
        }
    }
    wait_vmem<0>();                          // nothing is under way to the LDS of whoever runs here next
}

// Whether wavefronts share the tiles of all units: where the units are long, not
// too many for the lookup (64 per lane, more than the chip holds wavefronts), and
// the tiles can be counted in 31 bits.  Above the lookup's limit a long unit holds
// up the rest: 4,096 units of which eight have 32,768 rows and the others 300 take
// 75 us, 4,104 such 1,192 (300 rows each: 45).  One wavefront per short unit costs neither
// the lookup nor, without weights, the launch that joins states; a long one keeps
// its wavefront busy behind the others.  In us, shared / a wavefront per unit
// (d = 128, G = 4, bf16 queries, all units with table room for max_rows rows):
//   8 units     128 rows 12.4 / 9.6    256 rows 12.8 / 12.3    512 rows 12.2 / 21.6
//   512 units   128 rows 13.5 / 9.5    256 rows 15.9 / 13.0    512 rows 20.9 / 22.9
//   1,024       128 rows 18.1 / 9.5    256 rows 23.7 / 13.3    512 rows 29.0 / 23.3
//   2,048       128 rows 28.6 / 11.9   256 rows 35.4 / 19.3    512 rows 46.8 / 33.2
//   2,048       256 to 2,048 rows 77 / 106
//   with weights (1 to max_rows rows): 8 units of 128 rows 13.5 / 13.6, of 256
//   rows 13.3 / 17.0; 1,024 units of 128 rows 19.6 / 17.6, of 256 rows 22.8 / 24.2
static bool shares_tiles(int64_t units, int64_t max_rows, bool weights) {
    const int64_t whole = weights ? 128 : units >= 1024 ? 512 : 256;
    return max_rows > whole && units <= D4_SHARED_UNITS && units * ceil_div(max_rows, D4_TILE) <= 0x7fffffffll;
}
// Wavefronts that share them (the kernel uses fewer where the units are short).
template <typename T>
static int64_t shared_waves(int64_t units, int64_t max_rows) {
    return std::max<int64_t>(1, std::min<int64_t>(Plan4<T>::SHARES, units * ceil_div(max_rows, D4_TILE) / D4_MIN_SHARE));
}

struct Decode4Sizes {      // bytes of the workspace's parts (for either type of queries)
    size_t z, states, spans;
};
static Decode4Sizes decode4_sizes(int64_t units, int G, int d, int64_t max_rows, bool weights) {
    const bool shared = shares_tiles(units, max_rows, weights);
    const size_t slots = shared ? (size_t)(units + shared_waves<uint16_t>(units, max_rows)) : weights ? (size_t)units : 0;
    return {weights ? (size_t)units * G * z_stride_of(max_rows) * sizeof(float) : 0,
            slots * G * (size_t)(d + 2) * sizeof(float), shared ? (size_t)units * sizeof(int2) : 0};
}

template <typename T, int D>
static int launch_decode4(const char *fn, hipStream_t s, int B, Decode4Args a, Weights w, char *ws, size_t ws_bytes) {
    const int G = a.Hq / a.Hkv;
    const int64_t units = (int64_t)B * a.Hkv, max_rows = (int64_t)a.max_pages * a.page_size;
    const bool weights = w.out != nullptr, shared = shares_tiles(units, max_rows, weights);
    const unsigned grid = shared ? (unsigned)shared_waves<T>(units, max_rows) : (unsigned)units;
    const int64_t expect = shared ? grid / units + 1 : 1;      // states per unit
    SG_REQUIRE(!(weights || shared) || units <= max_workgroups(finish_threads(D, expect)), SG_EUNSUPPORTED,
               "%s: too many units", fn);
    const Decode4Sizes sz = decode4_sizes(units, G, D, max_rows, weights);
    const size_t need = sz.z + sz.states + sz.spans;
    SG_REQUIRE(need <= ws_bytes && (need == 0 || ws), SG_EWORKSPACE, "%s: needs %zu bytes of workspace, %zu given", fn,
               need, ws_bytes);
    a.units = (int)units;
    a.z = w.z = reinterpret_cast<float *>(ws);
    a.z_stride = w.z_stride = z_stride_of(max_rows);
    a.spans = shared ? reinterpret_cast<int2 *>(ws + sz.z) : nullptr;
    a.states = reinterpret_cast<float *>(ws + sz.z + sz.spans);
    const bool halves = a.page_size % 16 == 0;
#define SG_D4(KEEP, SHARED)                                                           \
    do {                                                                              \
        if (halves) decode4_kernel<T, D, KEEP, SHARED, true><<<grid, 64, 0, s>>>(a);  \
        else decode4_kernel<T, D, KEEP, SHARED, false><<<grid, 64, 0, s>>>(a);        \
    } while (0)
    if (weights && shared) SG_D4(true, true);
    else if (weights) SG_D4(true, false);
    else if (shared) SG_D4(false, true);
    else SG_D4(false, false);
#undef SG_D4
    if (weights || shared)
        launch_finish<D>(s, units, G, expect, 1, a.n_rows, max_rows, 0, a.spans, a.states, a.out, w);
    return launch_status(fn);
}

}  // namespace sg

using namespace sg;

extern "C" size_t sg_decode_attn_fp4_workspace_size(int B, int Hq, int Hkv, int d, int max_pages, int page_size,
                                                    int weights) {
    if (B <= 0 || Hkv <= 0 || Hq <= 0 || Hq % Hkv != 0 || d <= 0 || max_pages <= 0 || page_size <= 0) return 0;
    const Decode4Sizes sz = decode4_sizes((int64_t)B * Hkv, Hq / Hkv, d, (int64_t)max_pages * page_size, weights != 0);
    return sz.z + sz.states + sz.spans;
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
    SG_REQUIRE(scale > 0.f && scale <= 2e38f, SG_EINVAL, "%s: scale must be positive and finite", fn);
    SG_REQUIRE((int64_t)B * Hkv <= max_workgroups(64), SG_EUNSUPPORTED, "%s: too many units", fn);
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
    // division by the page size as a multiply-shift (as in sg_decode_attn)
    int lg = 0;
    while ((1ll << lg) < page_size) ++lg;
    const int shift = 30 + lg;
    const uint32_t mul = (uint32_t)(((1ull << shift) + (uint64_t)page_size - 1) / (uint64_t)page_size);
    // rows that are left out read pool row 0 and nothing comes of it: where the
    // pool has no rows, the queries (a row of them is longer) stand for it
    if (pool_rows == 0) k_pool = v_pool = s_pool = reinterpret_cast<const uint8_t *>(q);
    const Decode4Args a{Hq, Hkv, scale * 1.4426950408889634f /* log2(e) */, q, k_pool, v_pool, s_pool, pool_rows,
                        page_table, n_rows, page_size, max_pages, 0, mul, shift, out, nullptr, nullptr, nullptr, 0};
    hipStream_t s = as_stream(stream);
    const Weights w{weight_in, weight_out, weight_stride, decay, nullptr, 0};
    char *wsb = reinterpret_cast<char *>(ws);
#define SG_D4(T, D) launch_decode4<T, D>(fn, s, B, a, w, wsb, ws_bytes)
    if (dt == SG_F32) return d == 64 ? SG_D4(float, 64) : SG_D4(float, 128);
    return d == 64 ? SG_D4(uint16_t, 64) : SG_D4(uint16_t, 128);
#undef SG_D4
}
