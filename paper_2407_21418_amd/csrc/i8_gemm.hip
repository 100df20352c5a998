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

// Few rows: tiles of 16 MB x 16 NB whose W waves take turns along the reduce axis, 128 bytes of it at a time, straight from memory into the
// matrix cores' operands; their sums meet in LDS.  Every byte of either operand is loaded by one wave of a workgroup once.
template <int MB, int NB, int W, int AHEAD, bool GROUPED, bool GATED> __global__ __launch_bounds__(W * 64) void ft_i8_stream(I8Args a) {
    static_assert(!GATED || NB % 2 == 0, "gates and values in pairs");
    __shared__ i8_i32x4 sums[W * MB * NB * 64];
    constexpr int TM = MB * 16, TN = NB * 16;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u);
    const I8Tile t = I8Tiles<TM, TN, GROUPED>(a).take(a, 0);
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
        I8Scales<GATED> scales;
        scales.load(cols, a, t, col);
        if constexpr (GATED) i8_store4(a, t.row0 + r, col, cols.of_c, i8_gated(scales, sa, sum(2u * j), sum(2u * j + 1u)));
        else i8_store4(a, t.row0 + r, col, cols.of_c, i8_scaled(scales, sa, sum(j)));
    }
}

}  // namespace ftk

using namespace ftk;

namespace {

template <int MB, int NB, int W, int AHEAD, bool GROUPED, bool GATED> ft_status launch_stream(I8Args &a, hipStream_t s) {
    if (!i8_grid(a, MB * 16, NB * 16, GROUPED)) return FT_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((ft_i8_stream<MB, NB, W, AHEAD, GROUPED, GATED>), dim3(a.row_tiles * a.col_tiles), dim3(W * 64), 0, s, a);
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
    return a.gated ? launch_stream<1, 2, 8, 2, GROUPED, true>(a, s) : launch_stream<1, 1, 8, 2, GROUPED, false>(a, s);
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
