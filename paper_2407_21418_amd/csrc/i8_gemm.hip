// Matmuls in 8-bit integers, one scale for each row of either operand; plain and for rows sorted by expert.
//
//   C[i, j] = scale_a[i] scale_b[j] sum_k A[i, k] B[j, k] (+ bias[j]),  B stored [N][K]
//
// v_mfma_i32_16x16x64_i8 adds exact 32-bit integers (|sum| <= 131071 * 2^14 < 2^31); what follows is fp32, rounded once
// where C has 16 bits.  Both operands lie with k contiguous, and a lane's fragment is 16 of its row's bytes.  B's fragment is handed
// over first, so that a lane ends up with four neighbouring columns of a row of C.  Only A is cut at the end of the reduce axis: a
// zero times whatever lies beyond it in B is zero.
//
// With gates (silu(p[i, j]) * p[i, n / 2 + j]) a tile's blocks of 16 columns are gates and their values in turn, so that both meet in one
// workgroup and the activation is part of the epilogue, in fp32.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ft_internal.h"
#include "i8_ops.h"
#include "lane_types.h"
#include "lds_limit.h"
#include "op_launch.h"

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

// Every XCD (workgroup b runs on XCD b % 8) takes one contiguous run of the `total` tiles: those that share a panel of B meet in one L2.
__device__ __forceinline__ bool i8_position(uint32_t b, uint32_t total, uint32_t *u) {
    const uint32_t x = b & 7u, j = b >> 3, q = total >> 3, r = total & 7u;
    *u = x * q + (x < r ? x : r) + j;
    return j < q + (x < r ? 1u : 0u);
}

template <int TM, int TN, bool GROUPED> __device__ __forceinline__ I8Tile i8_tile(const I8Args &a, uint32_t b) {
    I8Tile t;
    uint32_t u;
    if constexpr (!GROUPED) {
        t.some = i8_position(b, a.row_tiles * a.col_tiles, &u);
        // bands of `group` rows of tiles, column by column
        const uint32_t band = u / (a.group * a.col_tiles), w = u - band * a.group * a.col_tiles;
        const uint32_t high = a.row_tiles - band * a.group < a.group ? a.row_tiles - band * a.group : a.group;
        const uint32_t col = w / high;
        t.row0 = (band * a.group + w - col * high) * TM;
        t.rows = a.m - t.row0 < (uint32_t)TM ? a.m - t.row0 : (uint32_t)TM;
        t.n0 = col * TN;
        t.expert = 0;
        return t;
    } else {
        // Each lane counts the row tiles of an expert; prefix sums over the lanes say whose tile this is.
        const uint32_t lane = threadIdx.x & 63u;
        auto group = [&](uint32_t e, uint32_t *beg) -> uint32_t {       // rows of expert e
            if (e >= a.experts) { *beg = 0; return 0u; }
            int32_t s = a.offsets[e], n = a.offsets[e + 1];
            s = s < 0 ? 0 : s > (int32_t)a.m ? (int32_t)a.m : s;
            n = n < s ? s : n > (int32_t)a.m ? (int32_t)a.m : n;
            *beg = (uint32_t)s;
            return (uint32_t)(n - s);
        };
        auto scan = [&](uint32_t v) -> uint32_t {
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const uint32_t up = __shfl_up(v, d);
                if (lane >= (uint32_t)d) v += up;
            }
            return v;
        };
        uint32_t beg, count = group(lane, &beg), tiles = (count + TM - 1u) / TM, upto = scan(tiles);
        uint32_t total = __builtin_amdgcn_readlane(upto, 63);
        for (uint32_t at = 64; at < a.experts; at += 64u) {
            uint32_t skip;
            total += __builtin_amdgcn_readlane(scan((group(at + lane, &skip) + TM - 1u) / TM), 63);
        }
        t.some = i8_position(b, total * a.col_tiles, &u);
        t.row0 = t.rows = t.n0 = t.expert = 0;
        if (!t.some) return t;
        uint32_t before = 0;
        for (uint32_t at = 0;; at += 64u) {
            if (at) {
                count = group(at + lane, &beg);
                tiles = (count + TM - 1u) / TM;
                upto = scan(tiles);
            }
            const uint64_t behind = __ballot((before + upto) * a.col_tiles > u);
            if (behind) {
                const int l = __builtin_ctzll(behind);
                const uint32_t n_tiles = __builtin_amdgcn_readlane(tiles, l), w = u - (before + __builtin_amdgcn_readlane(upto, l) - n_tiles) * a.col_tiles;
                const uint32_t col = w / n_tiles, row = w - col * n_tiles, rows = __builtin_amdgcn_readlane(count, l) - row * TM;
                t.expert = at + (uint32_t)l;
                t.row0 = __builtin_amdgcn_readlane(beg, l) + row * TM;
                t.rows = rows < (uint32_t)TM ? rows : (uint32_t)TM;
                t.n0 = col * TN;
                t.some = col < a.col_tiles;                  // (offsets that are not ascending can say otherwise)
                return t;
            }
            before += __builtin_amdgcn_readlane(upto, 63);
            if (at + 64u >= a.experts) { t.some = false; return t; }    // (not reached: u < total * col_tiles)
        }
    }
}

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
    __device__ __forceinline__ uint32_t row_of_block(int j) const { return (GATED ? j / 2 : j) * 16u; }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t operand(int j) const { return GATED && j % 2 ? values : b; }
};
template <typename COLS> __device__ __forceinline__ i8_f32x4 i8_scaled(const COLS &cols, const I8Args &a, const I8Tile &t, uint32_t col, float sa, i8_i32x4 v) {
    const uint64_t at = (uint64_t)t.expert * a.n;
    i8_f32x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint64_t c = at + (col + e < cols.of_c ? col + e : col);
        out[e] = (float)v[e] * sa * a.scale_b[c];
        if (a.bias) out[e] += a.bias[c];
    }
    return out;
}
template <typename COLS> __device__ __forceinline__ i8_f32x4 i8_gated(const COLS &cols, const I8Args &a, const I8Tile &t, uint32_t col, float sa, i8_i32x4 g, i8_i32x4 u) {
    const uint64_t at = (uint64_t)t.expert * a.n;
    i8_f32x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint64_t c = at + (col + e < cols.of_c ? col + e : col);
        out[e] = silu_mul((float)g[e] * sa * a.scale_b[c], (float)u[e] * sa * a.scale_b[c + cols.of_c]);
    }
    return out;
}

// Four neighbouring columns of a row of C
__device__ __forceinline__ void i8_store4(const I8Args &a, uint32_t row, uint32_t col, uint32_t columns, i8_f32x4 v) {
    const uint64_t at = (uint64_t)row * a.ldc + col;
    if (a.out_kind == 0) {
        float *const c = static_cast<float *>(a.C) + at;
        if (a.vec) *reinterpret_cast<i8_f32x4 *>(c) = v;
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < columns) c[e] = v[e];
        }
    } else {
        uint16_t *const c = static_cast<uint16_t *>(a.C) + at;
        i8_u32x2 h;
        if (a.out_kind == 1) h = i8_u32x2{__builtin_bit_cast(uint32_t, i8_f16x2{(_Float16)v[0], (_Float16)v[1]}), __builtin_bit_cast(uint32_t, i8_f16x2{(_Float16)v[2], (_Float16)v[3]})};
        else h = i8_u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(i8_f32x2{v[0], v[1]}, i8_bf16x2)),
                          __builtin_bit_cast(uint32_t, __builtin_convertvector(i8_f32x2{v[2], v[3]}, i8_bf16x2))};
        if (a.vec) *reinterpret_cast<i8_u32x2 *>(c) = h;
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < columns) c[e] = (uint16_t)(h[e / 2] >> (e % 2 * 16));
        }
    }
}

// Few rows: tiles of 16 MB x 16 NB whose W waves take turns along the reduce axis, 128 bytes of it at a time, straight from memory into the
// matrix cores' operands; their sums meet in LDS.  Every byte of either operand is loaded by one wave of a workgroup once.
template <int MB, int NB, int W, int AHEAD, bool GROUPED, bool GATED> __global__ __launch_bounds__(W * 64) void ft_i8_stream(I8Args a) {
    static_assert(!GATED || NB % 2 == 0, "gates and values in pairs");
    extern __shared__ i8_i32x4 sums[];                       // [W][MB * NB][64]
    constexpr int TM = MB * 16, TN = NB * 16;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u);
    const I8Tile t = i8_tile<TM, TN, GROUPED>(a, blockIdx.x);
    if (!t.some) return;
    const __amdgpu_buffer_rsrc_t ar = GROUPED ? i8_rsrc(a.A, a.a_rows * a.lda) : i8_rsrc(a.A + (uint64_t)t.row0 * a.lda, t.rows * a.lda);
    const I8Columns<TN, GATED> cols(a, t);
    const uint32_t kc = (lane >> 4) * 16u;
    uint32_t off_a[MB], off_b[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const uint32_t r = i * 16u + (lane & 15u);
        if constexpr (GROUPED) {
            const uint32_t s = r < t.rows ? i8_source<true>(a, t.row0 + r) : ~0u;
            off_a[i] = s == ~0u ? kOutside : s * a.lda + kc;
        } else off_a[i] = r * a.lda + kc;
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) off_b[j] = (cols.row_of_block(j) + (lane & 15u)) * a.ldb + kc;
    i8_i32x4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = i8_i32x4{0, 0, 0, 0};

    struct Step { i8_u32x4 a[2][MB], b[2][NB]; };
    auto load = [&](uint32_t s, Step &f) {                   // (beyond the reduce axis: zeros)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t k = s * 128u + h * 64u;
            const bool in = k + kc < a.k;
#pragma unroll
            for (int j = 0; j < NB; ++j) f.b[h][j] = i8_load(cols.operand(j), in ? off_b[j] + k : kOutside);
#pragma unroll
            for (int i = 0; i < MB; ++i) f.a[h][i] = i8_load(ar, in ? off_a[i] + k : kOutside);
        }
    };
    auto use = [&](uint32_t s, Step &f) {
        if (s * 128u + 128u > a.k) {                         // the last step's rows end inside
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MB; ++i) f.a[h][i] = i8_cut(f.a[h][i], s * 128u + h * 64u + kc, a.k);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = i8_mfma(f.b[h][j], f.a[h][i], acc[i][j]);
    };
    const uint32_t steps = (a.k + 127u) / 128u;
    Step f[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load(wave + i * W, f[i]);
    for (uint32_t s = wave; s < steps; s += AHEAD * W) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            use(s + i * W, f[i]);                            // (beyond the last step: zeros)
            load(s + (i + AHEAD) * W, f[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) sums[(wave * (MB * NB) + i * NB + j) * 64u + lane] = acc[i][j];
    __syncthreads();
    constexpr int NP = GATED ? NB / 2 : NB;                  // blocks of columns of C
    for (uint32_t item = threadIdx.x; item < MB * NP * 64u; item += W * 64u) {
        const uint32_t l = item & 63u, j = item / 64u % NP, i = item / 64u / NP, r = i * 16u + (l & 15u), col = cols.first + j * 16u + (l >> 4) * 4u;
        if (r >= t.rows || col >= cols.of_c) continue;
        auto sum = [&](uint32_t block) {
            i8_i32x4 v = sums[(i * NB + block) * 64u + l];
#pragma unroll
            for (int w = 1; w < W; ++w) v += sums[(w * (MB * NB) + i * NB + block) * 64u + l];
            return v;
        };
        const uint32_t s = i8_source<GROUPED>(a, t.row0 + r);
        const float sa = s == ~0u ? 0.f : a.scale_a[s];
        i8_f32x4 out;
        if constexpr (GATED) out = i8_gated(cols, a, t, col, sa, sum(2u * j), sum(2u * j + 1u));
        else out = i8_scaled(cols, a, t, col, sa, sum(j));
        i8_store4(a, t.row0 + r, col, cols.of_c, out);
    }
}

}  // namespace ftk

using namespace ftk;

namespace {

template <int MB, int NB, int W, int AHEAD, bool GROUPED, bool GATED> ft_status launch_stream(I8Args &a, hipStream_t s) {
    constexpr uint32_t TM = MB * 16, TN = NB * 16;
    // (grouped: every group but the last row tile of each is full)
    const uint64_t rows = GROUPED ? (uint64_t)a.m / TM + (a.experts < a.m ? a.experts : a.m) : ((uint64_t)a.m + TM - 1) / TM;
    a.col_tiles = (a.n + TN - 1) / TN;
    if (rows * a.col_tiles > 0x7fffffffull) return FT_ERR_UNSUPPORTED;
    a.row_tiles = (uint32_t)rows;
    a.group = a.row_tiles < 16u ? a.row_tiles : 16u;
    hipLaunchKernelGGL((ft_i8_stream<MB, NB, W, AHEAD, GROUPED, GATED>), dim3(a.row_tiles * a.col_tiles), dim3(W * 64), W * MB * NB * 1024u, s, a);
    return op_launched();
}
template <bool GROUPED, bool GATED> ft_status run(I8Args &a, hipStream_t s) {
    const uint32_t rows = GROUPED ? (a.m + a.experts - 1u) / a.experts : a.m;         // of a group, if they are alike
    if (rows <= 16u) return launch_stream<1, GATED ? 2 : 1, 8, 2, GROUPED, GATED>(a, s);
    if (rows <= 32u) return launch_stream<2, 2, 8, 2, GROUPED, GATED>(a, s);
    return launch_stream<4, 2, 8, 1, GROUPED, GATED>(a, s);
}
template <bool GROUPED> ft_status run(I8Args &a, void *stream) {
    const ft_status st = op_stream_check(stream);
    if (st != FT_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.gated ? run<GROUPED, true>(a, s) : run<GROUPED, false>(a, s);
}

}  // namespace

extern "C" {

ft_status ft_i8_matmul(const ft_i8_desc *desc, uint32_t m, const int8_t *A, const float *scale_a, const int8_t *B, const float *scale_b, const float *bias, void *C,
                       void *hip_stream) {
    I8Args a = {};
    bool go;
    const ft_status st = i8_check(desc, false, m, nullptr, A, scale_a, 0, nullptr, B, scale_b, bias, C, &a, &go);
    return st != FT_OK || !go ? st : run<false>(a, hip_stream);
}

ft_status ft_i8_matmul_experts(const ft_i8_desc *desc, uint32_t rows, const int32_t *offsets, const int8_t *A, const float *scale_a, const int32_t *a_row, uint32_t a_rows,
                               const int8_t *B, const float *scale_b, const float *bias, void *C, void *hip_stream) {
    I8Args a = {};
    bool go;
    const ft_status st = i8_check(desc, true, rows, offsets, A, scale_a, a_rows, a_row, B, scale_b, bias, C, &a, &go);
    return st != FT_OK || !go ? st : run<true>(a, hip_stream);
}

}  // extern "C"
