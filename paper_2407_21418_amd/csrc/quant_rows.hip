// Rows of values as 8-bit integers with one scale each, where asked after silu(gate) * up.
//
// Bound by memory: a row is read once, stays in its threads' registers while its largest magnitude is found, and
// leaves as integers.  Rows of more than 32768 columns are read a second time.  From memory 65536 x 1408 fp32 take 82 us (5.6 TB/s; 75 behind the
// product that leaves a part of them in the last-level cache), 8192 x 4096 bf16 20.7 (4.9), 2048 x 2 x 11008 bf16 gated 24.6 (4.6), the same in
// fp32 42.0 (4.8), 65536 x 2 x 1408 fp32 gated 154 (5.4), where a copy reaches 4.8; one row of 4096 2.8 us, most of which is any launch's.
//
// scale = amax / 127 and q = 127 f / amax to nearest even.  For 16-bit f this is exact without a division for each value: with 127 / amax
// as the sum of two fp32, t = f * hi + f * lo is the quotient rounded once, 2^-24 of itself.  127 f / amax lies exactly in the middle
// between two integers, and then t is that middle, or at least 2^-19 of itself away from there (f = a 2^p, amax = d 2^q with a,
// d < 2^11 make 254 a 2^p - odd d 2^q a multiple of 2^p, and 2^p / (2 d 2^q) over 127 a 2^p / (d 2^q) is more than 2^-19): t rounds to
// the integer that the quotient rounds to.  Adding 1.5 * 2^23 does that and leaves the integer in the low byte.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ft_internal.h"
#include "i8_ops.h"
#include "lane_types.h"
#include "op_launch.h"

namespace ftk {

// The values of a piece of 8 columns, zeros beyond the row's end
template <int DT, bool GATED> struct QuantPiece {
    using T = RowType<DT>;
    static constexpr int N = 8 / T::V;                       // loads of 16 bytes
    struct Raw { row_u32x4 x[N], up[GATED ? N : 1]; };
    static __device__ __forceinline__ void eight(const row_u32x4 (&x)[N], float (&f)[8]) {
#pragma unroll
        for (int h = 0; h < N; ++h) {
            float part[T::V];
            T::floats(x[h], part);
#pragma unroll
            for (int i = 0; i < T::V; ++i) f[h * T::V + i] = part[i];
        }
    }
    static __device__ __forceinline__ void values(const Raw &r, float (&f)[8]) {
        eight(r.x, f);
        if constexpr (GATED) {
            float u[8];
            eight(r.up, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = silu_mul(f[i], u[i]);
        }
    }
    static __device__ __forceinline__ void clear(Raw &r) {
#pragma unroll
        for (int h = 0; h < N; ++h) {
            r.x[h] = row_u32x4{0u, 0u, 0u, 0u};
            if constexpr (GATED) r.up[h] = row_u32x4{0u, 0u, 0u, 0u};
        }
    }
    static __device__ __forceinline__ void load(const QuantArgs &a, const unsigned char *row, uint32_t p, Raw &r) {
        clear(r);
        const uint32_t n = a.cols - p * 8u;
#pragma unroll
        for (int h = 0; h < N; ++h) {
            if (h && n <= (uint32_t)(h * T::V)) continue;
            r.x[h] = T::load(row + p * (8u * T::BYTES) + h * 16u, n - h * T::V);
            if constexpr (GATED) r.up[h] = T::load(row + (a.cols + p * 8u) * T::BYTES + h * 16u, n - h * T::V);
        }
    }
};

// Largest magnitude as bits: magnitudes compare as their bits do, infinities and NaNs above all others
__device__ __forceinline__ uint32_t largest(const float (&f)[8], uint32_t m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __builtin_bit_cast(uint32_t, f[i]) & 0x7fffffffu;
        m = b > m ? b : m;
    }
    return m;
}

// Rows of very small or large values are multiplied with a power of two first, so that 127 / amax and what it leaves are normal.
struct RowScale {
    float lift, hi, lo, scale;
    bool fine;
    __device__ __forceinline__ explicit RowScale(uint32_t bits) : lift(1.f), hi(0.f), lo(0.f), scale(0.f), fine(bits < 0x7f800000u) {
        const float amax = __builtin_bit_cast(float, bits);
        if (!fine) scale = __builtin_nanf("");
        else if (bits != 0) {
            if (amax < 0x1p-60f) lift = 0x1p100f;
            else if (amax > 0x1p60f) lift = 0x1p-60f;
            const float peak = amax * lift;
            hi = 127.f / peak;
            lo = __builtin_fmaf(-hi, peak, 127.f) / peak;
            scale = amax / 127.f;
        }
    }
    __device__ __forceinline__ uint2 integers(float (&f)[8]) const {
        if (!fine) return make_uint2(0u, 0u);
        if (lift != 1.f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= lift;
        }
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = __builtin_bit_cast(uint32_t, __builtin_fmaf(f[i], hi, f[i] * lo) + 0x1.8p23f);
        return make_uint2(low_bytes(q[0], q[1], q[2], q[3]), low_bytes(q[4], q[5], q[6], q[7]));
    }
    static __device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
        return __builtin_amdgcn_perm(b, a, 0x0c0c0400u) | __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    }
};

// `threads` threads for a row: 64, four rows to a workgroup, or a whole workgroup.  HELD: pieces that a thread keeps; 0: as many as
// there are, read twice
template <int DT, bool GATED, int HELD> __global__ __launch_bounds__(1024) void ft_quant(QuantArgs a, uint32_t threads) {
    using P = QuantPiece<DT, GATED>;
    __shared__ uint32_t most[16];
    const uint32_t per = threads == 64u ? blockDim.x / 64u : 1u;
    const uint32_t r = blockIdx.x * per + (per > 1u ? threadIdx.x / 64u : 0u), tid = per > 1u ? threadIdx.x & 63u : threadIdx.x;
    if (per > 1u && r >= a.rows) return;                     // (whole waves, and no barrier below for them)
    const unsigned char *const row = static_cast<const unsigned char *>(a.X) + (uint64_t)r * a.ldx * P::T::BYTES;
    unsigned char *const out = reinterpret_cast<unsigned char *>(a.Q) + (uint64_t)r * a.ldq;
    const uint32_t pieces = (a.cols + 7u) / 8u;
    constexpr int H = HELD ? HELD : 1;
    float f[H][8];
    uint32_t m = 0;
    if constexpr (HELD > 0) {
        typename P::Raw x[H];
#pragma unroll
        for (int i = 0; i < H; ++i) {
            if (tid + i * threads < pieces) P::load(a, row, tid + i * threads, x[i]);
            else P::clear(x[i]);
        }
#pragma unroll
        for (int i = 0; i < H; ++i) {
            P::values(x[i], f[i]);
            m = largest(f[i], m);
        }
    } else {
        for (uint32_t p = tid; p < pieces; p += threads) {
            typename P::Raw x;
            P::load(a, row, p, x);
            P::values(x, f[0]);
            m = largest(f[0], m);
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_xor(m, d);
        m = o > m ? o : m;
    }
    if (threads > 64u) {
        if ((threadIdx.x & 63u) == 0) most[threadIdx.x / 64u] = m;
        __syncthreads();
        for (uint32_t w = 0; w < threads / 64u; ++w) m = most[w] > m ? most[w] : m;
    }
    const RowScale s(m);
    if (tid == 0) a.scale[r] = s.scale;
    if constexpr (HELD > 0) {
#pragma unroll
        for (int i = 0; i < H; ++i)
            if (tid + i * threads < pieces) *reinterpret_cast<uint2 *>(out + (tid + i * threads) * 8u) = s.integers(f[i]);
    } else {
        for (uint32_t p = tid; p < pieces; p += threads) {
            typename P::Raw x;
            P::load(a, row, p, x);
            P::values(x, f[0]);
            *reinterpret_cast<uint2 *>(out + p * 8u) = s.integers(f[0]);
        }
    }
    for (uint32_t p = pieces + tid; p < a.ldq / 8u; p += threads) *reinterpret_cast<uint2 *>(out + p * 8u) = make_uint2(0u, 0u);
}

}  // namespace ftk

using namespace ftk;

namespace {

template <int DT, bool GATED> ft_status launch(QuantArgs a, hipStream_t s) {
    // Pieces of a thread: one where a few rows leave the device idle (16 x 4096 bf16 3.0 us, with two 3.25; from 1024 rows on alike), four where
    // more in flight is what wide rows lack (8192 x 4096 bf16 20.8 us, with two 22.1; 8192 x 11008 48.9 and 50.9), else two (65536 x 1408 fp32
    // 81.0 us, with four 83.2; 2048 x 2 x 11008 gated 24.0 and 25.8; 8192 x 2048 bf16 12.7 and 13.6; each pair on one card in turn).
    const uint32_t pieces = (a.cols + 7u) / 8u;
    const uint32_t hold = a.rows <= 256u ? 1u : !GATED && DT != ROW_F32 && a.cols >= 4096u ? 4u : 2u;
    uint32_t threads = ((pieces + hold - 1u) / hold + 63u) / 64u * 64u;
    if (threads > 1024u) threads = 1024u;
    const uint32_t per = threads == 64u ? 4u : 1u;
    const uint32_t most = launch_rows(per, threads * per);
    for (;; a.rows -= most) {
        QuantArgs part = a;
        if (part.rows > most) part.rows = most;
        const dim3 grid((part.rows + per - 1u) / per), block(threads * per);
        if (pieces <= threads) hipLaunchKernelGGL((ft_quant<DT, GATED, 1>), grid, block, 0, s, part, threads);
        else if (pieces <= 2u * threads) hipLaunchKernelGGL((ft_quant<DT, GATED, 2>), grid, block, 0, s, part, threads);
        else if (pieces <= 4u * threads) hipLaunchKernelGGL((ft_quant<DT, GATED, 4>), grid, block, 0, s, part, threads);
        else hipLaunchKernelGGL((ft_quant<DT, GATED, 0>), grid, block, 0, s, part, threads);
        const ft_status st = op_launched();
        if (st != FT_OK || a.rows <= most) return st;
        a.X = static_cast<const unsigned char *>(a.X) + (uint64_t)most * a.ldx * RowType<DT>::BYTES;
        a.Q += (uint64_t)most * a.ldq;
        a.scale += most;
    }
}

}  // namespace

extern "C" ft_status ft_i8_quantize(const ft_quant_desc *desc, uint32_t rows, const void *X, int8_t *Q, float *scale, void *hip_stream) {
    QuantArgs a = {};
    bool go;
    ft_status st = quant_check(desc, rows, X, Q, scale, &a, &go);
    if (st == FT_OK && go) st = op_stream_check(hip_stream);
    if (st != FT_OK || !go) return st;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const bool gated = desc->act == FT_ACT_SILU_MUL;
    if (desc->dtype == FT_F16) return gated ? launch<ROW_F16, true>(a, s) : launch<ROW_F16, false>(a, s);
    if (desc->dtype == FT_BF16) return gated ? launch<ROW_BF16, true>(a, s) : launch<ROW_BF16, false>(a, s);
    return gated ? launch<ROW_F32, true>(a, s) : launch<ROW_F32, false>(a, s);
}
