// Rows of 16- or 32-bit values in pieces of 16 bytes, as floats: loads and stores of the row kernels (quant_rows.hip, experts.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ftk {

// gfx950 loads and stores 16 bytes at any address that is aligned to the elements: rows of any pitch take one path
typedef uint32_t row_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t RowPiece __attribute__((ext_vector_type(4), aligned(2)));

typedef float row_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 row_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 row_f16x2 __attribute__((ext_vector_type(2)));

enum { ROW_F16 = 0, ROW_BF16 = 1, ROW_F32 = 2 };
template <int DT> struct RowType {
    static constexpr int BYTES = DT == ROW_F32 ? 4 : 2, V = 16 / BYTES;      // elements of a piece
    static __device__ __forceinline__ void floats(row_u32x4 v, float (&f)[V]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t word = v[i];          // (the compiler's bit cast of a vector's element takes the first one, whichever is named)
            if constexpr (DT == ROW_F32) f[i] = __builtin_bit_cast(float, word);
            else if constexpr (DT == ROW_BF16) {
                f[2 * i] = __builtin_bit_cast(float, word << 16);
                f[2 * i + 1] = __builtin_bit_cast(float, word & 0xffff0000u);
            } else {
                const row_f16x2 h = __builtin_bit_cast(row_f16x2, word);
                f[2 * i] = (float)h[0];
                f[2 * i + 1] = (float)h[1];
            }
        }
    }
    // rounded to nearest even where the type has 16 bits
    static __device__ __forceinline__ row_u32x4 pack(const float (&f)[V]) {
        row_u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == ROW_F32) v[i] = __builtin_bit_cast(uint32_t, f[i]);
            else if constexpr (DT == ROW_BF16) v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(row_f32x2{f[2 * i], f[2 * i + 1]}, row_bf16x2));
            else v[i] = __builtin_bit_cast(uint32_t, row_f16x2{(_Float16)f[2 * i], (_Float16)f[2 * i + 1]});
        }
        return v;
    }
    // piece of a row at p, of which n >= 1 elements are the row's; the others read as zeros
    // STREAM: what is not asked for again is not kept in the caches
    template <bool STREAM = false> static __device__ __forceinline__ row_u32x4 load(const unsigned char *p, uint32_t n) {
        if (n >= (uint32_t)V) {
            if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const RowPiece *>(p));
            else return *reinterpret_cast<const RowPiece *>(p);
        }
        row_u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < V - 1; ++i) {
            if ((uint32_t)i >= n) continue;
            if constexpr (BYTES == 4) v[i] = reinterpret_cast<const uint32_t *>(p)[i];
            else v[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << (i % 2 * 16);
        }
        return v;
    }
    template <bool STREAM = false> static __device__ __forceinline__ void store(unsigned char *p, row_u32x4 v, uint32_t n) {
        if (n >= (uint32_t)V) {
            if constexpr (STREAM) __builtin_nontemporal_store((RowPiece)v, reinterpret_cast<RowPiece *>(p));
            else *reinterpret_cast<RowPiece *>(p) = v;
            return;
        }
#pragma unroll
        for (int i = 0; i < V - 1; ++i) {
            if ((uint32_t)i >= n) continue;
            if constexpr (BYTES == 4) reinterpret_cast<uint32_t *>(p)[i] = v[i];
            else reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(v[i / 2] >> (i % 2 * 16));
        }
    }
};

// g / (1 + exp(-g)) * u.  exp(-g) is 2^(-g log2 e) with the exponent rounded: within (1.22 |g| + 2) 2^-24 of itself, which a gate far below zero
// feels most; a third of the instructions of a call of expf, and infinities and NaNs come out as by the formula.  The reciprocal is of a quarter of the sum: of
// one beyond 2^126, for gates below -87.3, the instruction leaves zero, where the result need not be small (-88 times 3e38: -160).  Below -88.72 exp(-g) is
// infinite, and the result is zero.
__device__ __forceinline__ float silu_mul(float g, float u) {
    const float quarter = __builtin_fmaf(0.25f, __builtin_amdgcn_exp2f(-0x1.715476p+0f * g), 0.25f);
    return g * (0.25f * __builtin_amdgcn_rcpf(quarter)) * u;
}

}  // namespace ftk
