// Matmuls in 8-bit integers: what the kernels of i8_gemm.hip and i8_blocks.hip share -- which tile a workgroup takes, where its operands
// lie, and what becomes of its sums.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "i8_ops.h"
#include "lane_types.h"

namespace ftk {

typedef int32_t i8_i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t i8_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t i8_u32x2 __attribute__((ext_vector_type(2)));
typedef float i8_f32x2 __attribute__((ext_vector_type(2)));
typedef float i8_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 i8_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 i8_f16x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kOutside = 0x80000000u;          // an offset beyond every buffer: reads as zeros

__device__ __forceinline__ __amdgpu_buffer_rsrc_t i8_rsrc(const int8_t *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p), 0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ i8_u32x4 i8_load(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return __builtin_bit_cast(i8_u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0));
}
__device__ __forceinline__ i8_i32x4 i8_mfma(i8_u32x4 b, i8_u32x4 a, i8_i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i8_i32x4, b), __builtin_bit_cast(i8_i32x4, a), c, 0, 0, 0);
}
// the bytes of a fragment at k .. k + 15 that lie before K
__device__ __forceinline__ i8_u32x4 i8_cut(i8_u32x4 v, uint32_t k, uint32_t K) {
    const int left = (int)K - (int)k;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = left - 4 * i;                          // bytes of this word
        v[i] = n >= 4 ? v[i] : n <= 0 ? 0u : v[i] & ((1u << (8 * n)) - 1u);
    }
    return v;
}

// Where a workgroup's tile lies: rows row0 .. row0 + rows - 1 of C, columns n0 .., weight `expert`.
struct I8Tile {
    uint32_t row0, rows, n0, expert;
    bool some;                                               // false: nothing left for this workgroup
};

// Every XCD (workgroup b of the grid runs on XCD b % 8) takes one contiguous run of the `total` tiles, so that those which share a panel of B
// meet in one L2; its workgroups take the run's tiles in turn.  u: the place of workgroup b's `turn`-th tile.
__device__ __forceinline__ bool i8_position(uint32_t b, uint32_t grid, uint32_t turn, uint32_t total, uint32_t *u) {
    const uint32_t x = b & 7u, q = total >> 3, r = total & 7u, mine = (grid - x + 7u) >> 3, j = (b >> 3) + turn * mine;
    *u = x * q + (x < r ? x : r) + j;
    return j < q + (x < r ? 1u : 0u);
}

// The tiles of a launch.  By expert the counts of each are on the device: the lanes of a wave count 64 experts' row tiles at a time, and their
// prefix sums, the first 64 of which stay for as long as the workgroup lives, say whose a tile is.  The first tile takes its rows from those lanes and
// sums by lane moves, as nothing runs beside them then (4 tokens, 2 of 16 experts 10.8 -> 10.5 us).
template <int TM, int TN, bool GROUPED> struct I8Tiles {
    struct Rows { uint32_t beg, count; };
    uint32_t total, upto;                                    // all tiles; row tiles up to and with those of expert `lane`
    Rows first;                                              // rows of expert `lane`, for the first tile
    __device__ __forceinline__ I8Tiles(const I8Args &a) {
        if constexpr (!GROUPED) total = a.row_tiles * a.col_tiles;
        else {
            const uint32_t lane = threadIdx.x & 63u;
            first = lane < a.experts ? rows_of(a, lane) : Rows{0u, 0u};
            upto = upto_of(first);
            uint32_t sum = __builtin_amdgcn_readlane(upto, 63);
            for (uint32_t at = 64; at < a.experts; at += 64u) sum += __builtin_amdgcn_readlane(upto_of(a, at), 63);
            total = sum * a.col_tiles;
        }
    }
    // rows of expert e, from offsets that are held to 0 .. m (nothing writes them while the kernel runs: a uniform e reads them as constants)
    static __device__ __forceinline__ Rows rows_of(const I8Args &a, uint32_t e) {
        const auto *const o = (const __attribute__((address_space(4))) int32_t *)a.offsets;
        int32_t s = o[e], n = o[e + 1];
        s = s < 0 ? 0 : s > (int32_t)a.m ? (int32_t)a.m : s;
        n = n < s ? s : n > (int32_t)a.m ? (int32_t)a.m : n;
        return Rows{(uint32_t)s, (uint32_t)(n - s)};
    }
    static __device__ __forceinline__ uint32_t upto_of(const I8Args &a, uint32_t at) {
        const uint32_t lane = threadIdx.x & 63u;
        return upto_of(at + lane < a.experts ? rows_of(a, at + lane) : Rows{0u, 0u});
    }
    // prefix sums over the lanes: within rows of 16, then those before a row's
    static __device__ __forceinline__ uint32_t upto_of(Rows r) {
        int v = (int)((r.count + TM - 1u) / TM);
        v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // from 1, 2, 4, 8 lanes lower
        v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
        v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
        v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
        v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // a row's last lane to the row above, for rows 1 and 3
        v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // row 1's last lane to rows 2 and 3
        return (uint32_t)v;
    }
    __device__ __forceinline__ I8Tile take(const I8Args &a, uint32_t turn) const {
        I8Tile t;
        uint32_t u;
        t.some = i8_position(blockIdx.x, gridDim.x, turn, total, &u);
        t.row0 = t.rows = t.n0 = t.expert = 0;
        if (!t.some) return t;
        if constexpr (!GROUPED) {
            // bands of `group` rows of tiles, column by column
            const uint32_t band = u / (a.group * a.col_tiles), w = u - band * a.group * a.col_tiles;
            const uint32_t high = a.row_tiles - band * a.group < a.group ? a.row_tiles - band * a.group : a.group;
            const uint32_t col = w / high;
            t.row0 = (band * a.group + w - col * high) * TM;
            t.rows = a.m - t.row0 < (uint32_t)TM ? a.m - t.row0 : (uint32_t)TM;
            t.n0 = col * TN;
            return t;
        }
        uint32_t before = 0;
        for (uint32_t at = 0; at < a.experts; at += 64u) {
            const uint32_t here = at ? upto_of(a, at) : upto;
            const uint64_t behind = __ballot((before + here) * a.col_tiles > u);
            if (behind) {
                const uint32_t l = (uint32_t)__builtin_ctzll(behind), under = before + (l ? __builtin_amdgcn_readlane(here, l - 1u) : 0u);
                Rows r;
                if (turn == 0u && at == 0u) r = Rows{(uint32_t)__builtin_amdgcn_readlane(first.beg, l), (uint32_t)__builtin_amdgcn_readlane(first.count, l)};
                else r = rows_of(a, at + l);
                const uint32_t n_tiles = (r.count + TM - 1u) / TM, w = u - under * a.col_tiles, col = w / n_tiles, row = w - col * n_tiles, rows = r.count - row * TM;
                t.expert = at + l;
                t.row0 = r.beg + row * TM;
                t.rows = rows < (uint32_t)TM ? rows : (uint32_t)TM;
                t.n0 = col * TN;
                t.some = n_tiles != 0u && col < a.col_tiles; // (offsets that are not ascending can say otherwise, and sums of many such wrap)
                return t;
            }
            before += __builtin_amdgcn_readlane(here, 63);
        }
        t.some = false;                                      // (not reached: u < total)
        return t;
    }
};

// Row of A that row r of C takes; one that is not there: ~0
template <bool GROUPED> __device__ __forceinline__ uint32_t i8_source(const I8Args &a, uint32_t r) {
    if constexpr (!GROUPED) return r;
    const uint32_t s = a.a_row ? (uint32_t)a.a_row[r] : r;
    return s < a.a_rows ? s : ~0u;
}

// A tile's columns: where their rows of B begin, for blocks of 16, and their places in C
template <int TN, bool GATED> struct I8Columns {
    __amdgpu_buffer_rsrc_t b, values;
    uint32_t first, of_c;                                    // first column of the tile in C, columns of C
    __device__ __forceinline__ I8Columns(const I8Args &a, const I8Tile &t) {
        const int8_t *const w = a.B + (uint64_t)t.expert * a.n * a.ldb;
        constexpr uint32_t WIDTH = GATED ? TN / 2 : TN;
        first = GATED ? t.n0 / 2u : t.n0;
        of_c = GATED ? a.n / 2u : a.n;
        const uint32_t rows = of_c - first < WIDTH ? of_c - first : WIDTH;
        b = i8_rsrc(w + (uint64_t)first * a.ldb, rows * a.ldb);
        values = GATED ? i8_rsrc(w + (uint64_t)(of_c + first) * a.ldb, rows * a.ldb) : b;
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t operand(int j) const { return GATED && j % 2 ? values : b; }
};
// four neighbouring values of a vector of `n`, at any alignment; beyond its end the first of them again
struct __attribute__((packed, aligned(4))) I8Four {
    i8_f32x4 v;
};
__device__ __forceinline__ i8_f32x4 i8_four(const float *p, uint32_t at, uint32_t n) {
    if (at + 4u <= n) return reinterpret_cast<const I8Four *>(p + at)->v;
    i8_f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = p[at + e < n ? at + e : at];
    return v;
}
// What four neighbouring columns of a tile are scaled with: read before anything is stored, which may lie anywhere for all the compiler knows
template <bool GATED> struct I8Scales {
    i8_f32x4 b, other;                                       // scales; the bias, or the scales of the values
    template <typename COLS> __device__ __forceinline__ void load(const COLS &cols, const I8Args &a, const I8Tile &t, uint32_t col) {
        const float *const sb = a.scale_b + (uint64_t)t.expert * a.n;
        b = i8_four(sb, col, cols.of_c);
        if constexpr (GATED) other = i8_four(sb + cols.of_c, col, cols.of_c);
        else if (a.bias) other = i8_four(a.bias + (uint64_t)t.expert * a.n, col, cols.of_c);
        else other = i8_f32x4{0.f, 0.f, 0.f, 0.f};
    }
};
__device__ __forceinline__ i8_f32x4 i8_scaled(const I8Scales<false> &s, float sa, i8_i32x4 v) {
    i8_f32x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (float)v[e] * sa * s.b[e] + s.other[e];
    return out;
}
__device__ __forceinline__ i8_f32x4 i8_gated(const I8Scales<true> &s, float sa, i8_i32x4 g, i8_i32x4 u) {
    i8_f32x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = silu_mul((float)g[e] * sa * s.b[e], (float)u[e] * sa * s.other[e]);
    return out;
}
// two values rounded to 16 bits, to nearest even
__device__ __forceinline__ uint32_t i8_pack(uint32_t out_kind, float x, float y) {
    if (out_kind == 1) return __builtin_bit_cast(uint32_t, i8_f16x2{(_Float16)x, (_Float16)y});
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(i8_f32x2{x, y}, i8_bf16x2));
}

// Four neighbouring columns of a row of C, at any address that is aligned to its elements (value by value only where the row ends among them: all rows
// of 715 fp32 so: 2000 x 1430 x 1000 gated took 13.1 us, now 10.8)
typedef float I8AnyF32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t I8AnyU32x2 __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void i8_store4(const I8Args &a, uint32_t row, uint32_t col, uint32_t columns, i8_f32x4 v) {
    const uint64_t at = (uint64_t)row * a.ldc + col;
    if (a.out_kind == 0) {
        float *const c = static_cast<float *>(a.C) + at;
        if (col + 4u <= columns) *reinterpret_cast<I8AnyF32x4 *>(c) = v;
        else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (col + e < columns) c[e] = v[e];
        }
    } else {
        uint16_t *const c = static_cast<uint16_t *>(a.C) + at;
        const i8_u32x2 h = {i8_pack(a.out_kind, v[0], v[1]), i8_pack(a.out_kind, v[2], v[3])};
        if (col + 4u <= columns) *reinterpret_cast<I8AnyU32x2 *>(c) = h;
        else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (col + e < columns) c[e] = (uint16_t)(h[e / 2] >> (e % 2 * 16));
        }
    }
}

}  // namespace ftk
