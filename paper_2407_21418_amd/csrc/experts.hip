// Tokens sorted by expert and back.
//
// The sort is a counting sort that keeps the order of the entries: row = rows of lower experts + earlier entries of the same
// expert.  A wave ranks 64 entries at a time (those of one id find each other with a ballot for each bit of the id), every wave
// of a workgroup has counts of its own for its stretch of the entries, and their prefix sums give each wave the row
// where its next entry of an expert goes.  No atomic decides an order.
//
// Bound by latency: 8192 x 8 entries 9.9 us in a graph (counts and places 4.7 and 7.1 each by itself), up to 16384 entries one launch, whose blocks count all
// of them: 4 x 2 3.3 us, 1234 x 6 5.9.
//
// The moves are bound by memory: a workgroup's threads hold a token's row in pieces of 16 bytes and read or write it once
// for all of its entries; rows of entries are read or written once.  8192 x 8 of 4096 bf16: gather 119 us (5.1 TB/s), combine 110 (5.5), the
// gradients 226 (5.1), where a copy reaches 4.8; 64 x 4 of 2048 2.6, 2.9 and 5.3 us, of which 2.1 are any launch's and its first read's.  (The same
// launch again and again in a graph; in a pass of several, whose rows another kernel has just left, small ones take up to a microsecond more.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ft_internal.h"
#include "i8_ops.h"
#include "lane_types.h"
#include "lds_limit.h"
#include "op_launch.h"

namespace ftk {

struct SortArgs {
    const int32_t *ids;
    int32_t *offsets, *row_token, *row_of;
    uint32_t *counts;                    // [blocks][experts]; NULL: a block counts all entries itself
    uint32_t n, experts, top_k;
    uint32_t blocks, per_block;          // entries of a block
    uint32_t id_bits;                    // bits of experts - 1
};

// The ids of a wave's stretch [s0, s1) of the entries, 64 at a time: the first kHeld steps are asked for together and stay in registers, so that a
// stretch of up to 512 entries waits for memory once.  No id: ~0.
constexpr int kHeld = 8;
struct Stretch {
    uint32_t s0, s1, lane, held[kHeld];
    __device__ __forceinline__ uint32_t read(const SortArgs &a, uint32_t at) const {
        const uint32_t id = at + lane < s1 ? (uint32_t)a.ids[at + lane] : ~0u;
        return id < a.experts ? id : ~0u;
    }
    __device__ __forceinline__ Stretch(const SortArgs &a, uint32_t wave, uint32_t waves, uint32_t lane_) : lane(lane_) {
        // whole steps of the block's entries, as many for each wave
        const uint32_t b0 = blockIdx.x * a.per_block, b1 = a.n - b0 < a.per_block ? a.n : b0 + a.per_block;
        const uint32_t steps = (b1 - b0 + 63u) / 64u, per = (steps + waves - 1u) / waves * 64u;
        s0 = b1 - b0 < wave * per ? b1 : b0 + wave * per;
        s1 = b1 - s0 < per ? b1 : s0 + per;
#pragma unroll
        for (int u = 0; u < kHeld; ++u) held[u] = read(a, s0 + u * 64u);
    }
    // f(first entry, this lane's id) for every step
    template <typename F> __device__ __forceinline__ void each(const SortArgs &a, F f) const {
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
            if (s0 + u * 64u < s1) f(s0 + u * 64u, held[u]);
        for (uint32_t at = s0 + kHeld * 64u; at < s1; at += 64u) f(at, read(a, at));
    }
    // counts of every id
    __device__ __forceinline__ void count(const SortArgs &a, uint32_t *counts) const {
        each(a, [&](uint32_t, uint32_t id) {
            if (id != ~0u) atomicAdd(&counts[id], 1u);
        });
    }
};
// exclusive prefix sums of v[0 .. n) by one wave, in place; v[n] receives the total
__device__ __forceinline__ void scan_by_wave(uint32_t *v, uint32_t n, uint32_t lane) {
    uint32_t carry = 0;
    for (uint32_t at = 0; at < n; at += 64u) {
        const uint32_t x = at + lane < n ? v[at + lane] : 0u;
        uint32_t sum = x;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t up = __shfl_up(sum, d);
            if (lane >= (uint32_t)d) sum += up;
        }
        if (at + lane < n) v[at + lane] = carry + sum - x;
        carry += __shfl(sum, 63);
    }
    if (lane == 0) v[n] = carry;
}

// counts[block][expert]
__global__ __launch_bounds__(1024) void ft_expert_count(SortArgs a) {
    __shared__ uint32_t lds[kMaxExperts];
    const uint32_t tid = threadIdx.x, threads = blockDim.x;
    const Stretch stretch(a, tid / 64u, threads / 64u, tid & 63u);
    for (uint32_t e = tid; e < a.experts; e += threads) lds[e] = 0u;
    __syncthreads();
    stretch.count(a, lds);
    __syncthreads();
    for (uint32_t e = tid; e < a.experts; e += threads) a.counts[(uint64_t)blockIdx.x * a.experts + e] = lds[e];
}

__global__ __launch_bounds__(1024) void ft_expert_place(SortArgs a) {
    // cnt [waves][experts], first [experts + 1], below [experts]
    extern __shared__ uint32_t lds[];
    const uint32_t tid = threadIdx.x, threads = blockDim.x, lane = tid & 63u, wave = tid / 64u, waves = threads / 64u, E = a.experts;
    uint32_t *const cnt = lds, *const first = lds + waves * E, *const below = first + E + 1u, *const mine = cnt + wave * E;
    const uint32_t b0 = blockIdx.x * a.per_block, b1 = a.n - b0 < a.per_block ? a.n : b0 + a.per_block;
    const Stretch stretch(a, wave, waves, lane);
    for (uint32_t i = tid; i < waves * E; i += threads) cnt[i] = 0u;
    for (uint32_t e = tid; e < E; e += threads) first[e] = below[e] = 0u;
    __syncthreads();
    stretch.count(a, mine);
    // first: the entries of all other blocks; below: of those before this one
    if (a.counts) {
        // parts of the threads take turns with the blocks
        const uint32_t parts = threads / E ? threads / E : 1u;
        for (uint32_t i = tid; i < parts * E; i += threads) {
            const uint32_t e = i % E;
            uint32_t others = 0, before = 0;
            for (uint32_t b = i / E; b < a.blocks; b += parts) {
                const uint32_t c = b == blockIdx.x ? 0u : a.counts[(uint64_t)b * E + e];
                others += c;
                before += b < blockIdx.x ? c : 0u;
            }
            atomicAdd(&first[e], others);
            atomicAdd(&below[e], before);
        }
    } else if (a.blocks > 1u) {
        for (uint32_t at = 0; at < a.n; at += threads * kHeld) {
            uint32_t id[kHeld];
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                const uint32_t i = at + u * threads + tid;
                id[u] = i < a.n && (i < b0 || i >= b1) ? (uint32_t)a.ids[i] : ~0u;
            }
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                if (id[u] >= E) continue;
                atomicAdd(&first[id[u]], 1u);
                if (at + u * threads + tid < b0) atomicAdd(&below[id[u]], 1u);
            }
        }
    }
    __syncthreads();
    // the waves' counts to prefix sums over the waves
    for (uint32_t e = tid; e < E; e += threads) {
        uint32_t sum = 0;
        for (uint32_t w = 0; w < waves; ++w) {
            const uint32_t c = cnt[w * E + e];
            cnt[w * E + e] = sum;
            sum += c;
        }
        first[e] += sum;
    }
    __syncthreads();
    if (wave == 0) scan_by_wave(first, E, lane);
    __syncthreads();
    if (blockIdx.x == 0)
        for (uint32_t e = tid; e <= E; e += threads) a.offsets[e] = (int32_t)first[e];
    for (uint32_t e = lane; e < E; e += 64u) mine[e] += first[e] + below[e];
    // (a wave's LDS accesses are in order: what follows touches its own counts only)
    __builtin_amdgcn_wave_barrier();
    stretch.each(a, [&](uint32_t at, uint32_t id) {
        const uint32_t i = at + lane;
        const bool has = id != ~0u;
        uint64_t peers = __ballot(has);
        for (uint32_t bit = 0; bit < a.id_bits; ++bit) {
            const uint64_t set = __ballot((id >> bit) & 1u);
            peers &= (id >> bit) & 1u ? set : ~set;
        }
        const uint32_t rank = __builtin_popcountll(peers & ((1ull << lane) - 1ull));
        uint32_t row = 0;
        if (has) row = mine[id] + rank;
        __builtin_amdgcn_wave_barrier();
        if (has && rank == 0) mine[id] += (uint32_t)__builtin_popcountll(peers);
        __builtin_amdgcn_wave_barrier();
        if (i < stretch.s1) a.row_of[i] = has ? (int32_t)row : -1;
        if (has) a.row_token[row] = (int32_t)(i / a.top_k);
    });
    // rows behind the last one
    const uint32_t used = first[E];
    for (uint32_t r = b0 + tid; r < b1; r += threads)
        if (r >= used) a.row_token[r] = -1;
}

// ---- moves: `lanes` threads (a power of two) for each token ----
// Entries are taken kEntries at a time, so that their loads are under way together.
constexpr int kEntries = 8;

struct MoveShape {
    uint32_t lanes, pieces;              // threads of a token, pieces of a row
};

// Piece p of a row: n elements from `at`.  A last one that the row ends inside begins earlier, so that it is whole as well; its first `again` elements are
// also the piece's before it (read value by value, a last piece cost each entry a wait of its own: 1234 x 6 of 1001 fp16 combine 5.6 us, now
// 4.6).
template <int V> struct MovePiece {
    uint32_t at, n, again;
    __device__ __forceinline__ MovePiece(uint32_t cols, uint32_t p) : at(p * V), n(cols - p * V), again(0) {
        if (n < (uint32_t)V && cols >= (uint32_t)V) again = V - n, at = cols - V, n = V;
    }
};

// The rows of entries j0 .. of token t, ~0 where there is none
template <int DT> __device__ __forceinline__ void entries_of(const MoveArgs &a, uint32_t t, uint32_t j0, uint32_t (&row)[kEntries]) {
    const uint32_t n = a.top_k - j0 < (uint32_t)kEntries ? a.top_k - j0 : (uint32_t)kEntries;
#pragma unroll
    for (int j = 0; j < kEntries; ++j) {
        row[j] = (uint32_t)j < n ? (uint32_t)a.row_of[(uint64_t)t * a.top_k + j0 + j] : ~0u;
        if (row[j] >= a.entries) row[j] = ~0u;
    }
}

template <int DT, bool STREAM> __global__ __launch_bounds__(256) void ft_expert_gather_kernel(MoveArgs a, MoveShape s) {
    using T = RowType<DT>;
    const uint32_t t = blockIdx.x * (256u / s.lanes) + threadIdx.x / s.lanes;
    if (t >= a.tokens) return;
    const unsigned char *const src = static_cast<const unsigned char *>(a.src) + (uint64_t)t * a.ld_token * T::BYTES;
    unsigned char *const dst = static_cast<unsigned char *>(a.dst);
    const uint64_t pitch = (uint64_t)a.ld_row * T::BYTES;
    for (uint32_t j0 = 0; j0 < a.top_k; j0 += kEntries) {
        uint32_t row[kEntries];
        entries_of<DT>(a, t, j0, row);
        for (uint32_t p = threadIdx.x & (s.lanes - 1u); p < s.pieces; p += s.lanes) {
            const MovePiece<T::V> piece(a.cols, p);
            const uint32_t n = piece.n, at = piece.at * T::BYTES;
            const row_u32x4 v = T::template load<STREAM>(src + at, n);
#pragma unroll
            for (int j = 0; j < kEntries; ++j)
                if (row[j] != ~0u) T::template store<STREAM>(dst + row[j] * pitch + at, v, n);
        }
    }
}

template <int DT, bool STREAM> __global__ __launch_bounds__(256) void ft_expert_combine_kernel(MoveArgs a, MoveShape s) {
    using T = RowType<DT>;
    const uint32_t t = blockIdx.x * (256u / s.lanes) + threadIdx.x / s.lanes;
    if (t >= a.tokens) return;
    const unsigned char *const src = static_cast<const unsigned char *>(a.src);
    unsigned char *const dst = static_cast<unsigned char *>(a.dst) + (uint64_t)t * a.ld_token * T::BYTES;
    const uint64_t pitch = (uint64_t)a.ld_row * T::BYTES;
    for (uint32_t p = threadIdx.x & (s.lanes - 1u); p < s.pieces; p += s.lanes) {
        const MovePiece<T::V> piece(a.cols, p);
        const uint32_t n = piece.n, at = piece.at * T::BYTES;
        float sum[T::V] = {};
        for (uint32_t j0 = 0; j0 < a.top_k; j0 += kEntries) {
            uint32_t row[kEntries];
            float w[kEntries];
            entries_of<DT>(a, t, j0, row);
            row_u32x4 v[kEntries];
#pragma unroll
            for (int j = 0; j < kEntries; ++j) {
                v[j] = row_u32x4{0u, 0u, 0u, 0u};
                w[j] = 1.f;
                if (row[j] == ~0u) continue;
                v[j] = T::template load<STREAM>(src + row[j] * pitch + at, n);
                if (a.weights) w[j] = a.weights[(uint64_t)t * a.top_k + j0 + j];
            }
#pragma unroll
            for (int j = 0; j < kEntries; ++j) {
                if (row[j] == ~0u) continue;
                float f[T::V];
                T::floats(v[j], f);
#pragma unroll
                for (int i = 0; i < T::V; ++i) sum[i] = __builtin_fmaf(w[j], f[i], sum[i]);
            }
        }
        T::template store<STREAM>(dst + at, T::pack(sum), n);
    }
}

// dY and, where DW, dweights: each thread's share of the products dOut * Y in fp32, then over the token's threads -- all entries' sums side by side, as a
// step of one of them waits for the step before (4 tokens x 2 of 1024 bf16 6.5 us one entry after the other, 4.1 so; 1234 x 6 of 1001 fp16 12.2 and 10.8)
template <int DT, bool DW, bool STREAM> __global__ __launch_bounds__(256) void ft_expert_grad_kernel(MoveArgs a, MoveShape s) {
    using T = RowType<DT>;
    __shared__ float parts[4][kEntries];
    const uint32_t t = blockIdx.x * (256u / s.lanes) + threadIdx.x / s.lanes, lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
    const bool there = t < a.tokens;     // (a token's threads stay for the barriers where they are several waves)
    const unsigned char *const dout = static_cast<const unsigned char *>(a.src) + (there ? (uint64_t)t * a.ld_token * T::BYTES : 0u);
    const unsigned char *const y = static_cast<const unsigned char *>(a.other);
    unsigned char *const dst = static_cast<unsigned char *>(a.dst);
    const uint64_t pitch = (uint64_t)a.ld_row * T::BYTES;
    for (uint32_t j0 = 0; j0 < a.top_k; j0 += kEntries) {
        uint32_t row[kEntries];
        float w[kEntries], dot[kEntries];
#pragma unroll
        for (int j = 0; j < kEntries; ++j) { row[j] = ~0u; w[j] = 1.f; dot[j] = 0.f; }
        if (there) {
            entries_of<DT>(a, t, j0, row);
            if (a.weights) {
                for (int j = 0; j < kEntries; ++j)
                    if (row[j] != ~0u) w[j] = a.weights[(uint64_t)t * a.top_k + j0 + j];
            }
            for (uint32_t p = threadIdx.x & (s.lanes - 1u); p < s.pieces; p += s.lanes) {
                const MovePiece<T::V> piece(a.cols, p);
                const uint32_t n = piece.n, at = piece.at * T::BYTES;
                float d[T::V];
                T::floats(T::template load<STREAM>(dout + at, n), d);
                row_u32x4 v[kEntries];
                if constexpr (DW) {
#pragma unroll
                    for (int j = 0; j < kEntries; ++j) {
                        v[j] = row_u32x4{0u, 0u, 0u, 0u};
                        if (row[j] != ~0u) v[j] = T::template load<STREAM>(y + row[j] * pitch + at, n);
                    }
                }
#pragma unroll
                for (int j = 0; j < kEntries; ++j) {
                    if (row[j] == ~0u) continue;
                    float g[T::V];
#pragma unroll
                    for (int i = 0; i < T::V; ++i) g[i] = w[j] * d[i];
                    T::template store<STREAM>(dst + row[j] * pitch + at, T::pack(g), n);
                    if constexpr (DW) {
                        float f[T::V];
                        T::floats(v[j], f);
                        if (piece.again == 0) {
#pragma unroll
                            for (int i = 0; i < T::V; ++i) dot[j] = __builtin_fmaf(d[i], f[i], dot[j]);
                        } else {
#pragma unroll
                            for (int i = 1; i < T::V; ++i)
                                if ((uint32_t)i >= piece.again) dot[j] = __builtin_fmaf(d[i], f[i], dot[j]);
                        }
                    }
                }
            }
        }
        if constexpr (DW) {
            const uint32_t in_wave = s.lanes < 64u ? s.lanes : 64u, n = a.top_k - j0 < (uint32_t)kEntries ? a.top_k - j0 : (uint32_t)kEntries;
            for (uint32_t m = 1; m < in_wave; m *= 2) {
#pragma unroll
                for (int j = 0; j < kEntries; ++j)
                    if ((uint32_t)j < n) dot[j] += __shfl_xor(dot[j], (int)m);
            }
            const uint32_t mine = threadIdx.x & (s.lanes - 1u);  // (an entry without a row: its sum is 0)
            float *const to = a.dweights + ((uint64_t)t * a.top_k + j0);
            if (s.lanes > 64u) {                             // (the same in every thread of the launch)
                __syncthreads();
                if (lane == 0) {
#pragma unroll
                    for (int j = 0; j < kEntries; ++j) parts[wave][j] = dot[j];
                }
                __syncthreads();
                if (there && mine < n) {
                    const uint32_t w0 = wave & ~(s.lanes / 64u - 1u);
                    float sum = parts[w0][mine];
                    for (uint32_t k = 1; k < s.lanes / 64u; ++k) sum += parts[w0 + k][mine];
                    to[mine] = sum;
                }
            } else if (there && mine == 0) {
#pragma unroll
                for (int j = 0; j < kEntries; ++j)
                    if ((uint32_t)j < n) to[j] = dot[j];
            }
        }
    }
}

}  // namespace ftk

using namespace ftk;

namespace {

template <int DT> MoveShape move_shape(const MoveArgs &a) {
    MoveShape s;
    s.pieces = (a.cols + RowType<DT>::V - 1) / RowType<DT>::V;
    s.lanes = 8;
    while (s.lanes < 256u && s.lanes < s.pieces) s.lanes *= 2u;
    return s;
}
enum { MOVE_GATHER, MOVE_COMBINE, MOVE_GRAD };
template <int DT, bool STREAM> ft_status move_launch(int what, MoveArgs a, hipStream_t stream) {
    const MoveShape s = move_shape<DT>(a);
    const uint32_t per = 256u / s.lanes, most = launch_rows(per, 256u);
    for (;; a.tokens -= most) {
        MoveArgs part = a;
        if (part.tokens > most) part.tokens = most;
        const dim3 grid((part.tokens + per - 1u) / per), block(256);
        if (what == MOVE_GATHER) hipLaunchKernelGGL((ft_expert_gather_kernel<DT, STREAM>), grid, block, 0, stream, part, s);
        else if (what == MOVE_COMBINE) hipLaunchKernelGGL((ft_expert_combine_kernel<DT, STREAM>), grid, block, 0, stream, part, s);
        else if (a.dweights) hipLaunchKernelGGL((ft_expert_grad_kernel<DT, true, STREAM>), grid, block, 0, stream, part, s);
        else hipLaunchKernelGGL((ft_expert_grad_kernel<DT, false, STREAM>), grid, block, 0, stream, part, s);
        const ft_status st = op_launched();
        if (st != FT_OK || a.tokens <= most) return st;
        const uint64_t bytes = (uint64_t)most * a.ld_token * RowType<DT>::BYTES, entries = (uint64_t)most * a.top_k;
        if (what == MOVE_COMBINE) a.dst = static_cast<unsigned char *>(a.dst) + bytes;
        else a.src = static_cast<const unsigned char *>(a.src) + bytes;
        a.row_of += entries;
        if (a.weights) a.weights += entries;
        if (a.dweights) a.dweights += entries;
    }
}
template <int DT> ft_status move_launch(int what, const MoveArgs &a, hipStream_t stream) {
    return move_streams(a, RowType<DT>::BYTES) ? move_launch<DT, true>(what, a, stream) : move_launch<DT, false>(what, a, stream);
}
ft_status move(int what, const ft_expert_desc *desc, const MoveArgs &a, void *stream) {
    const ft_status st = op_stream_check(stream);
    if (st != FT_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (desc->dtype == FT_F16) return move_launch<ROW_F16>(what, a, s);
    if (desc->dtype == FT_BF16) return move_launch<ROW_BF16>(what, a, s);
    return move_launch<ROW_F32>(what, a, s);
}

}  // namespace

extern "C" {

ft_status ft_expert_workspace(const ft_expert_desc *desc, uint32_t tokens, uint64_t *bytes) { return expert_workspace(desc, tokens, bytes); }

ft_status ft_expert_sort(const ft_expert_desc *desc, uint32_t tokens, const int32_t *expert_of, int32_t *offsets, int32_t *row_token, int32_t *row_of, void *workspace,
                         uint64_t workspace_bytes, void *hip_stream) {
    ft_status st = sort_check(desc, tokens, expert_of, offsets, row_token, row_of, workspace, workspace_bytes);
    if (st == FT_OK) st = op_stream_check(hip_stream);
    if (st != FT_OK) return st;
    SortArgs a = {};
    a.ids = expert_of; a.offsets = offsets; a.row_token = row_token; a.row_of = row_of;
    a.n = tokens * desc->top_k; a.experts = desc->experts; a.top_k = desc->top_k;
    a.counts = a.n > kSortRecount ? static_cast<uint32_t *>(workspace) : nullptr;
    a.blocks = sort_blocks(a.n);
    a.per_block = (uint32_t)(((uint64_t)a.n + a.blocks - 1u) / a.blocks + 63u) / 64u * 64u;
    if (a.per_block == 0u) a.per_block = 64u;
    a.blocks = a.n ? (a.n + a.per_block - 1u) / a.per_block : 1u;
    while (a.id_bits < 10u && (1u << a.id_bits) < a.experts) ++a.id_bits;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    uint32_t waves = (uint32_t)(((uint64_t)a.per_block + 63u) / 64u);
    if (waves > 16u) waves = 16u;
    const hipError_t e = raise_lds_limit<&ft_expert_place>();
    if (e != hipSuccess) { ftd_set_hip_error((int)e); return FT_ERR_HIP; }
    if (a.counts) {
        hipLaunchKernelGGL(ft_expert_count, dim3(a.blocks), dim3(1024), 0, s, a);
        st = op_launched();
        if (st != FT_OK) return st;
    }
    hipLaunchKernelGGL(ft_expert_place, dim3(a.blocks), dim3(waves * 64u), (waves * a.experts + 2u * a.experts + 1u) * 4u, s, a);
    return op_launched();
}

ft_status ft_expert_gather(const ft_expert_desc *desc, uint32_t tokens, const void *X, const int32_t *row_of, void *Y, void *hip_stream) {
    MoveArgs a = {};
    a.src = X; a.dst = Y; a.row_of = row_of;
    bool launch;
    const ft_status st = move_check(desc, tokens, false, &a, &launch);
    return st != FT_OK || !launch ? st : move(MOVE_GATHER, desc, a, hip_stream);
}

ft_status ft_expert_combine(const ft_expert_desc *desc, uint32_t tokens, const void *Y, const int32_t *row_of, const float *weights, void *Out, void *hip_stream) {
    MoveArgs a = {};
    a.src = Y; a.dst = Out; a.row_of = row_of; a.weights = weights;
    bool launch;
    const ft_status st = move_check(desc, tokens, false, &a, &launch);
    return st != FT_OK || !launch ? st : move(MOVE_COMBINE, desc, a, hip_stream);
}

ft_status ft_expert_combine_grad(const ft_expert_desc *desc, uint32_t tokens, const void *dOut, const void *Y, const int32_t *row_of, const float *weights, void *dY,
                                 float *dweights, void *hip_stream) {
    MoveArgs a = {};
    a.src = dOut; a.other = Y; a.dst = dY; a.row_of = row_of; a.weights = weights; a.dweights = dweights;
    bool launch;
    const ft_status st = move_check(desc, tokens, dweights != nullptr, &a, &launch);
    return st != FT_OK || !launch ? st : move(MOVE_GRAD, desc, a, hip_stream);
}

}  // extern "C"
