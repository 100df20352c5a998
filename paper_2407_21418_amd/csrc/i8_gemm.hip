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

#include <atomic>

#include "ft_internal.h"
#include "i8_blocks.h"
#include "i8_tile.h"
#include "op_launch.h"

namespace ftk {

// Few rows: tiles of 16 rows by 16 columns (by 16 gates and their values) whose eight waves take turns along the reduce axis, 128 bytes of it
// at a time, straight from memory into the matrix cores' operands, AHEAD turns under way; their sums meet in LDS.  Every byte of either
// operand is loaded by one wave of a workgroup once.  What the sums are scaled with is asked for before the products.  Bound by one read of the
// weight from the caches or memory, or by latency where that is small: 1 x 4096 x 4096 5.6 us (3.0 TB/s), 1 x 768 x 768 2.8, with gates 3.2, 16 x 8192
// x 2048 gated 6.1; 1 x 22016 x 4096 gated 22.4 (4.0 TB/s).  A wave that has no turn left asks for nothing: loads whose results are zeros cost their
// issue all the same (77 x 768 x 768, six turns for eight waves, 3.5 us with them, 3.1 without; 4 tokens, 2 of 8 experts, 2816 x 1024 gated 9.2 and 7.3).
template <int AHEAD, bool GROUPED, bool GATED> __global__ __launch_bounds__(512) void ft_i8_stream(I8Args a) {
    constexpr int W = 8, NB = GATED ? 2 : 1;
    __shared__ i8_i32x4 sums[W][NB][64];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u);
    const I8Tile t = I8Tiles<16, 16 * NB, GROUPED>(a).take(a, 0);
    if (!t.some) return;
    const I8Columns<16 * NB, GATED> cols(a, t);
    const uint32_t kc = (lane >> 4) * 16u, r = lane & 15u, steps = (a.k + 127u) / 128u, off_b = r * a.ldb + kc;
    const uint32_t source = r < t.rows ? i8_source<GROUPED>(a, t.row0 + r) : ~0u;
    struct Step { i8_u32x4 a[2], b[2][NB]; };
    Step f[AHEAD];
    auto load_b = [&](uint32_t s, Step &f) {                 // (beyond the reduce axis: zeros)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NB; ++j) f.b[h][j] = i8_load(cols.operand(j), s * 128u + h * 64u + kc < a.k ? off_b + s * 128u + h * 64u : kOutside);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (wave + i * W < steps) load_b(wave + i * W, f[i]);
    const __amdgpu_buffer_rsrc_t ar = GROUPED ? i8_rsrc(a.A, a.a_rows * a.lda) : i8_rsrc(a.A + (uint64_t)t.row0 * a.lda, t.rows * a.lda);
    const uint32_t off_a = GROUPED ? (source == ~0u ? kOutside : source * a.lda + kc) : r * a.lda + kc;
    auto load_a = [&](uint32_t s, Step &f) {
#pragma unroll
        for (int h = 0; h < 2; ++h) f.a[h] = i8_load(ar, s * 128u + h * 64u + kc < a.k ? off_a + s * 128u + h * 64u : kOutside);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (wave + i * W < steps) load_a(wave + i * W, f[i]);
    // wave 0 has the tile's results: row r, four columns from `col`
    const uint32_t col = cols.first + (lane >> 4) * 4u;
    const bool mine = wave == 0 && r < t.rows && col < cols.of_c;
    I8Scales<GATED> scales;
    float sa = 0.f;
    if (mine) {
        scales.load(cols, a, t, col);
        if (source != ~0u) sa = a.scale_a[source];
    }
    i8_i32x4 acc[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[j] = i8_i32x4{0, 0, 0, 0};
    for (uint32_t s = wave; s < steps; s += AHEAD * W) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const uint32_t now = s + i * W;
            if (now >= steps) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (now * 128u + 128u > a.k) f[i].a[h] = i8_cut(f[i].a[h], now * 128u + h * 64u + kc, a.k);      // rows end inside the last step
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[j] = i8_mfma(f[i].b[h][j], f[i].a[h], acc[j]);
            }
            if (now + AHEAD * W < steps) {
                load_b(now + AHEAD * W, f[i]);
                load_a(now + AHEAD * W, f[i]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    if (!mine) return;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int w = 1; w < W; ++w) acc[j] += sums[w][j][lane];
    if constexpr (GATED) i8_store4(a, t.row0 + r, col, cols.of_c, i8_gated(scales, sa, acc[0], acc[1]));
    else i8_store4(a, t.row0 + r, col, cols.of_c, i8_scaled(scales, sa, acc[0]));
}

}  // namespace ftk

using namespace ftk;

namespace {

template <bool GROUPED, bool GATED> ft_status launch_stream(I8Args &a, hipStream_t s) {
    if (!i8_grid(a, 16, GATED ? 32 : 16, GROUPED)) return FT_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((ft_i8_stream<2, GROUPED, GATED>), dim3(a.row_tiles * a.col_tiles), dim3(512), 0, s, a);
    return op_launched();
}
// compute units of the current device
int compute_units() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}
template <bool GROUPED> ft_status run(I8Args &a, void *stream) {
    const ft_status st = op_stream_check(stream);
    if (st != FT_OK) return st;
    a.cus = (uint32_t)compute_units();
    const I8Kind kind = i8_choose(a, GROUPED);
    if (kind != I8_STREAM) return i8_launch_blocks(kind, GROUPED, a, stream);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.gated ? launch_stream<GROUPED, true>(a, s) : launch_stream<GROUPED, false>(a, s);
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
