// Matmuls in 8-bit integers in blocks that pass through LDS: products of many rows.
//
// The loop is that of the large 16-bit products (big_gemm.hip), for the same bytes and twice the products: k-tiles of 128 bytes,
// the fragments of one k-step of 64 in registers while the MFMAs of the other run, one barrier for each k-tile half-way
// through its MFMAs, copies straight into LDS spread between them.  Both operands lie with k contiguous, so both are read with
// ds_read_b128; chunks of 16 bytes are swizzled by their row.
//
// What bounds them: the largest blocks the matrix cores and the power they draw (8192 x 8192 x 8192 fp32 398 .. 404 us, 2.76 POP/s, 8192 x 11008 x 4096
// bf16 290 .. 337 by the clock; of 352k cycles of MFMAs for each SIMD the launch takes 620k: 5.4 rounds of blocks are 6, then what lies
// between two blocks).  That is, of a 256 x 256 block's 56k cycles at K = 2048 with gates, 33k of MFMAs in 39k of products, 10k of scaling and
// exponentials, 5k to the next tile's place and 2 .. 4k of its first copies (65536 x 2816 x 2048 gated 322 us, 38 of them for results).
// Smaller blocks are for fewer tiles than the device has places: 64 x 128 hides a latency behind two workgroups of a CU, 64 x 64 takes the reduce
// axis in two groups of waves (256 x 768 x 768 4.9 us, 2.9 of them launch, first copies and results).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ft_internal.h"
#include "i8_blocks.h"
#include "i8_tile.h"
#include "lds_limit.h"
#include "op_launch.h"

namespace ftk {

template <int OFF> __device__ __forceinline__ i8_u32x4 i8_read(uint32_t addr) {
    i8_u32x4 v;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int N> __device__ __forceinline__ void i8_wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void i8_copy(__amdgpu_buffer_rsrc_t r, unsigned char *lds_wave_base, uint32_t lane_off, uint32_t tile_off) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)lds_wave_base, 16, (int)lane_off, (int)tile_off, 0, 0);
}
// sixteen rows read at four neighbouring chunks: no bank conflicts (counted)
__device__ __forceinline__ uint32_t i8_swizzle(uint32_t row) { return row & 7u; }
template <int Q, int E, typename F> __device__ __forceinline__ void i8_each(F f) {
    if constexpr (Q < E) { f(std::integral_constant<int, Q>{}); i8_each<Q + 1, E>(f); }
}

// A block of GM * WM rows by GN * WN columns.  STAGES = 0: A and B tiles are equally large and take turns in five slots (tile t: A in slot
// 2t mod 5, B in slot (2t + 1) mod 5).  Otherwise a ring of STAGES stages of A and B.  GK = 2: two groups of GM * GN waves take every other
// k-tile, each through a ring of its own, and share out the rows when their sums meet in LDS.
template <int WM, int WN, int GM, int GN, int GK, int STAGES, bool GROUPED, bool GATED> struct I8Block {
    static constexpr bool SLOTS = STAGES == 0;
    static constexpr int TM = GM * WM, TN = GN * WN, NW = GM * GN, WAVES = NW * GK, BM = WM / 16, BN = WN / 16;
    static constexpr int A_BYTES = TM * 128, B_BYTES = TN * 128, STAGE = A_BYTES + B_BYTES;
    static constexpr int LA = A_BYTES / NW / 1024, LB = B_BYTES / NW / 1024;
    static constexpr int NR = BM + BN, NM = BM * BN;
    static constexpr int RING = SLOTS ? 5 * A_BYTES : STAGES * STAGE, LDS = GK * RING;
    static constexpr int FAR = SLOTS ? 3 : STAGES;           // the furthest copy is of tile t + FAR
    static constexpr int AHEAD = SLOTS ? LA : (STAGES - 2) * (LA + LB);       // copies in flight beyond the next tile, steady state
    static_assert(!SLOTS || A_BYTES == B_BYTES, "five equal slots");
    static_assert(LDS <= 163840 && A_BYTES % (NW * 1024) == 0 && B_BYTES % (NW * 1024) == 0, "a CU's LDS; whole copies");
    static_assert(!GATED || BN % 2 == 0, "gates and values in pairs");
    static constexpr int KEEP = BM / GK;                     // blocks of rows that a wave stores
    static_assert(GK == 1 || (GK == 2 && BM % 2 == 0 && NW * BM * BN * 1024 <= LDS), "two groups share out the rows");

    struct Frag { i8_u32x4 a[BM], b[BN]; };
    // r-th LDS read of k-step KS's fragments: B first (its blocks are all used by the first row of blocks)
    template <int KS, int R> __device__ static __forceinline__ void read_one(uint32_t aa, uint32_t ba, Frag &f) {
        if constexpr (R < BN) f.b[R] = i8_read<R * 2048>(KS ? ba ^ 64u : ba);
        else f.a[R - BN] = i8_read<(R - BN) * 2048>(KS ? aa ^ 64u : aa);
    }
    template <int KS, int R, int E> __device__ static __forceinline__ void read_range(uint32_t aa, uint32_t ba, Frag &f) {
        if constexpr (R < E && R < NR) {
            read_one<KS, R>(aa, ba, f);
            read_range<KS, R + 1, E>(aa, ba, f);
        }
    }
    // every read of the set has arrived; its registers are produced here
    __device__ static __forceinline__ void arrived(Frag &f) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int i = 0; i < BM; ++i) asm volatile("" : "+v"(f.a[i]));
#pragma unroll
        for (int i = 0; i < BN; ++i) asm volatile("" : "+v"(f.b[i]));
    }
    // m-th MFMA of a k-step: rows of blocks in turn, columns back and forth, so that one operand stays
    __device__ static __forceinline__ void mfma_one(const Frag &f, i8_i32x4 (&acc)[BM][BN], int m) {
        const int bi = m / BN, bj = (bi & 1) ? BN - 1 - m % BN : m % BN;
        acc[bi][bj] = i8_mfma(f.b[bj], f.a[bi], acc[bi][bj]);
    }
    // The MFMAs of `use`, with the reads of `fill` (k-step KS of some tile) in the first three quarters and, where COPY,
    // LA + LB copies spread over all of them.  Pinned: left alone, the compiler gathers the reads in front.
    template <int KS, bool COPY, int M = 0, typename F>
    __device__ static __forceinline__ void phase(uint32_t aa, uint32_t ba, Frag &fill, const Frag &use, i8_i32x4 (&acc)[BM][BN], F copy) {
        read_range<KS, M * NR * 4 / (NM * 3), (M + 1) * NR * 4 / (NM * 3)>(aa, ba, fill);
        if constexpr (COPY) i8_each<M *(LA + LB) / NM, (M + 1) * (LA + LB) / NM>(copy);
        mfma_one(use, acc, M);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (M + 1 < NM) phase<KS, COPY, M + 1>(aa, ba, fill, use, acc, copy);
    }

    // By expert: the rows of A that this lane's copies of a tile take, asked for a tile ahead
    struct CopyRows {
        uint32_t of_a[GROUPED ? LA : 1];
        __device__ __forceinline__ void ask(const I8Args &g, const I8Tile &tile, uint32_t wave, uint32_t lane) {
            if constexpr (GROUPED) {
#pragma unroll
                for (int i = 0; i < LA; ++i) {
                    const uint32_t row = wave * (LA * 8) + i * 8 + lane / 8u;
                    of_a[i] = row < tile.rows ? i8_source<true>(g, tile.row0 + row) : ~0u;
                }
            }
        }
    };
    // Where a tile's operands lie.  Copies: wave instruction i fills 1 KB, eight rows, of the tile.  A row that is not there, and what lies beyond the
    // last one, reads as zeros by the buffer's bound; bytes beyond K are whatever follows, and are cut from A's fragments.
    struct Source {
        __amdgpu_buffer_rsrc_t a;
        I8Columns<TN, GATED> cols;
        uint32_t off_a[LA], off_b[LB];
        uint32_t first_k, whole_k;
        // (wave: in its group; a group's t-th k-tile is the block's GK * t + group)
        __device__ __forceinline__ Source(const I8Args &g, const I8Tile &tile, const CopyRows &rows, uint32_t wave, uint32_t group, uint32_t lane) : cols(g, tile) {
            whole_k = g.k / (128u * GK);
            first_k = g.k >= 8192u ? (blockIdx.x & 7u) * whole_k / 8u : 0u;
            a = GROUPED ? i8_rsrc(g.A, g.a_rows * g.lda) : i8_rsrc(g.A + (uint64_t)tile.row0 * g.lda, tile.rows * g.lda);
#pragma unroll
            for (int i = 0; i < LA; ++i) {
                const uint32_t row = wave * (LA * 8) + i * 8 + lane / 8u, kc = (lane & 7u) ^ i8_swizzle(row), at = group * 128u + kc * 16u;
                if constexpr (GROUPED) off_a[i] = rows.of_a[i] == ~0u ? kOutside : rows.of_a[i] * g.lda + at;
                else off_a[i] = row * g.lda + at;
            }
#pragma unroll
            for (int i = 0; i < LB; ++i) {
                const uint32_t row = wave * (LB * 8) + i * 8 + lane / 8u, kc = (lane & 7u) ^ i8_swizzle(row);
                off_b[i] = ((GATED ? row / 32u * 16u + (row & 15u) : row) * g.ldb) + group * 128u + kc * 16u;
            }
        }
        // Where the t-th turn's k-tiles begin: from another place on for every XCD where the reduce axis is long, so that they do not all ask for the same
        // part of the same rows.  128 x 256: 2048 x 4096 x 11008 89 us all from the beginning, 85.5 so, 2048 x 5120 x 13824 180 and 173, 2048 x 4096 x 4096 32
        // both; 256 x 256 has no scalar instructions to spare in its loop: 8192 x 8192 x 8192 396 and 404.
        __device__ __forceinline__ uint32_t at_k(uint32_t t) const {
            if constexpr (SLOTS) return t * 128u;
            return i8_turn_begin(t, GK, first_k, whole_k);
        }
        template <int I> __device__ __forceinline__ void copy_a(unsigned char *smem, uint32_t wave, uint32_t t, uint32_t slot) const {
            i8_copy(a, smem + slot + wave * (LA * 1024) + I * 1024, off_a[I], at_k(t));
        }
        template <int I> __device__ __forceinline__ void copy_b(unsigned char *smem, uint32_t wave, uint32_t t, uint32_t slot) const {
            const bool values = GATED && (((wave * (LB * 8) + I * 8) / 16u) & 1u);
            i8_copy(values ? cols.values : cols.b, smem + slot + wave * (LB * 1024) + I * 1024, off_b[I], at_k(t));
        }
    };
    static __device__ __forceinline__ uint32_t next_slot(uint32_t s) {
        constexpr uint32_t STEP = SLOTS ? 2 * A_BYTES : STAGE;
        return s + STEP >= (uint32_t)RING ? s + STEP - RING : s + STEP;
    }
    // the ring full
    static __device__ __forceinline__ void fill(const Source &src, unsigned char *ring, uint32_t wave, uint32_t nk) {
        uint32_t pa = 0, pb = A_BYTES;
#pragma unroll
        for (int t = 0; t < FAR; ++t) {
            if ((uint32_t)t < nk) {
                i8_each<0, LA>([&](auto i) { src.template copy_a<decltype(i)::value>(ring, wave, t, pa); });
                if (!SLOTS || t < 2) i8_each<0, LB>([&](auto i) { src.template copy_b<decltype(i)::value>(ring, wave, t, pb); });
            }
            pa = next_slot(pa); pb = next_slot(pb);
        }
    }

    static constexpr int PER = GATED ? 2 : 1, NP = BN / PER;         // blocks of columns of C that a wave has
    // Where a wave's results lie -- lane l holds row l % 16, columns 4 * (l / 16) .. + 3 of every 16 x 16 block -- and what they are scaled with
    struct Finals {
        // (the four lanes of a row share out its blocks' rows of A, and pass the scales on)
        static constexpr int MINE = (KEEP + 3) / 4;
        uint32_t r0, c0, source[MINE];
        float sr[MINE];
        I8Scales<GATED> scales[NP];
        // the rows of A (by expert a read that scales wait for: asked for before the products), then all else
        __device__ __forceinline__ void sources(const I8Args &g, const I8Tile &tile, uint32_t wave, uint32_t group, uint32_t lane) {
#pragma unroll
            for (int p = 0; p < MINE; ++p) {
                const uint32_t i = (lane >> 4) * MINE + p, r = (wave / GN) * WM + (group * KEEP + i) * 16 + (lane & 15u);
                source[p] = i < (uint32_t)KEEP && r < tile.rows ? i8_source<GROUPED>(g, tile.row0 + r) : ~0u;
            }
        }
        __device__ __forceinline__ void ask(const I8Args &g, const I8Tile &tile, const I8Columns<TN, GATED> &cols, uint32_t wave, uint32_t group, uint32_t lane) {
            r0 = (wave / GN) * WM + group * (KEEP * 16) + (lane & 15u);
            c0 = cols.first + (wave % GN) * (WN / PER) + (lane >> 4) * 4u;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const uint32_t col = c0 + j * 16u;
                scales[j].load(cols, g, tile, col < cols.of_c ? col : cols.of_c - 1u);
            }
#pragma unroll
            for (int p = 0; p < MINE; ++p) sr[p] = source[p] == ~0u ? 0.f : g.scale_a[source[p]];
        }
        __device__ __forceinline__ void rows(uint32_t lane, float (&all)[KEEP]) const {
#pragma unroll
            for (int i = 0; i < KEEP; ++i) all[i] = __shfl(sr[i % MINE], (int)(i / MINE * 16 + (lane & 15u)));
        }
    };
    // Small waves ask for their scales before the products (128 x 4096 x 4096 9.9 -> 9.55 us, 1024 x 2304 x 768 8.35 -> 8.1); large ones have no
    // registers for that, and by expert the copies would wait behind two reads in a row (16 experts of 125 rows 15.8 -> 16.6).
    static constexpr bool EARLY = BM * BN <= 8 && !GROUPED;

    // All tiles of a workgroup.  The ring is filled for the next one while the last one's sums are scaled and stored.
    __device__ static __forceinline__ void run(const I8Args &g, unsigned char *smem) {
        const uint32_t tid = threadIdx.x, lane = tid & 63u, all = __builtin_amdgcn_readfirstlane(tid >> 6), wave = GK > 1 ? all % NW : all, group = GK > 1 ? all / NW : 0u;
        unsigned char *const ring = smem + group * RING;
        const I8Tiles<TM, TN, GROUPED> tiles(g);
        const uint32_t nk = ((g.k + 127u) / 128u + GK - 1u) / GK;    // k-tiles of a group (the last of the second may be nothing: it is cut)
        I8Tile tile = tiles.take(g, 0);
        if (!tile.some) return;
        CopyRows rows;
        rows.ask(g, tile, wave, lane);
        Source src(g, tile, rows, wave, group, lane);
        Finals fin;
        if constexpr (EARLY) {
            fin.sources(g, tile, wave, group, lane);
            fin.ask(g, tile, src.cols, wave, group, lane);
        }
        fill(src, ring, wave, nk);
        for (uint32_t turn = 1;; ++turn) {
            i8_i32x4 acc[BM][BN];
#pragma unroll
            for (int i = 0; i < BM; ++i)
#pragma unroll
                for (int j = 0; j < BN; ++j) acc[i][j] = i8_i32x4{0, 0, 0, 0};
            const I8Tile next = tiles.take(g, turn);
            if constexpr (GROUPED) {
                fin.sources(g, tile, wave, group, lane);
                if (next.some) rows.ask(g, next, wave, lane);
            }
            // a wave whose part of the tile lies beyond the last row or column copies for the others, and leaves them the matrix cores
            const bool idle = (wave / GN) * WM >= tile.rows || src.cols.first + (wave % GN) * (WN / PER) >= src.cols.of_c;
            if (idle) copies_alone(src, ring, wave, nk, turn > 1 && counted(g));
            else products(g, src, ring, wave, group, lane, nk, turn > 1 && counted(g), acc);
            const I8Tile done = tile;
            const I8Columns<TN, GATED> cols = src.cols;
            i8_i32x4 kept[KEEP][BN];
            if constexpr (GK > 1) meet(smem, wave, group, lane, acc, kept);
            uint32_t l = lane;
            asm volatile("" : "+v"(l));                              // (nothing of what follows is worked out before the products and kept over them)
            if constexpr (!EARLY) {
                if constexpr (!GROUPED) fin.sources(g, done, wave, group, l);
                fin.ask(g, done, cols, wave, group, l);
            }
            if (next.some) {
                // (every wave has read the last k-tile: they met after its second k-step had arrived)
                if constexpr (GK > 1) __syncthreads();               // the sums have been read
                src = Source(g, next, rows, wave, group, l);
                fill(src, ring, wave, nk);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (GK > 1) results(g, done, cols, fin, l, kept);
            else results(g, done, cols, fin, l, acc);
            if (!next.some) return;
            tile = next;
            if constexpr (EARLY) {
                fin.sources(g, tile, wave, group, lane);
                fin.ask(g, tile, src.cols, wave, group, lane);
            }
        }
    }

    // The two groups' sums: each wave gives the rows away that the other one's wave of the same place keeps.
    __device__ static __forceinline__ void meet(unsigned char *smem, uint32_t wave, uint32_t group, uint32_t lane, const i8_i32x4 (&acc)[BM][BN], i8_i32x4 (&kept)[KEEP][BN]) {
        i8_i32x4 *const sums = reinterpret_cast<i8_i32x4 *>(smem);
        const uint32_t give = ((1u - group) * NW + wave) * (KEEP * BN * 64u) + lane, take = (group * NW + wave) * (KEEP * BN * 64u) + lane;
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j) {
                const i8_i32x4 low = acc[i][j], high = acc[BM - KEEP + i][j];
                sums[give + (i * BN + j) * 64u] = group ? low : high;
                kept[i][j] = group ? high : low;
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j) kept[i][j] += sums[take + (i * BN + j) * 64u];
    }

    // k-tile 0 has landed / tile t has been read by this wave and tile t + 1 has landed.  In flight beyond it: A of t + 2 (slots), or the stages up
    // to t + STAGES - 1.  The last tile's results were stored after the first copies: where it is known how many stores those were (STORES at
    // least), they may still be under way when the copies have landed.
    static constexpr int STORES = KEEP * NP / (NP % 2 == 0 ? 2 : 1);
    static __device__ __forceinline__ void first_landed(uint32_t nk, bool stores) {
        constexpr int BEHIND = SLOTS ? 2 * LA + LB : (STAGES - 1) * (LA + LB), MOST = BEHIND + STORES < 63 ? BEHIND + STORES : 63;
        if (nk >= (uint32_t)FAR) {
            if (stores) i8_wait_copies<MOST>();
            else i8_wait_copies<BEHIND>();
        } else i8_wait_copies<0>();
        __builtin_amdgcn_s_barrier();
    }
    template <bool STEADY> static __device__ __forceinline__ void next_landed(uint32_t t, uint32_t nk) {
        const uint32_t behind = nk - 1u - t;                          // tiles after t
        if (STEADY || (SLOTS ? behind >= 2u : behind >= (uint32_t)STAGES - 1u)) i8_wait_copies<AHEAD>();
        else i8_wait_copies<0>();
        __builtin_amdgcn_s_barrier();
    }
    // the Q-th of the copies that are due once tile t has been read
    template <int Q, bool STEADY> static __device__ __forceinline__ void copy_behind(const Source &src, unsigned char *ring, uint32_t wave, uint32_t t, uint32_t nk, uint32_t sa, uint32_t sb) {
        if constexpr (SLOTS) {
            if constexpr (Q < LB) { if (STEADY || t + 2u < nk) src.template copy_b<Q>(ring, wave, t + 2u, sa); }
            else if constexpr (STEADY) src.template copy_a<Q - LB>(ring, wave, t + 3u, sb);
        } else if constexpr (STEADY) {
            if constexpr (Q < LA) src.template copy_a<Q>(ring, wave, t + STAGES, sa);
            else src.template copy_b<Q - LA>(ring, wave, t + STAGES, sb);
        }
    }

    __device__ static __forceinline__ void copies_alone(const Source &src, unsigned char *ring, uint32_t wave, uint32_t nk, bool stores) {
        uint32_t sa = 0, sb = A_BYTES, t = 0;
        first_landed(nk, stores);
        for (; t + FAR < nk; ++t) {
            next_landed<true>(t, nk);
            i8_each<0, LA + LB>([&](auto q) { copy_behind<decltype(q)::value, true>(src, ring, wave, t, nk, sa, sb); });
            sa = next_slot(sa); sb = next_slot(sb);
        }
        for (; t < nk; ++t) {
            next_landed<false>(t, nk);
            i8_each<0, LA + LB>([&](auto q) { copy_behind<decltype(q)::value, false>(src, ring, wave, t, nk, sa, sb); });
            sa = next_slot(sa); sb = next_slot(sb);
        }
    }

    __device__ static __forceinline__ void products(const I8Args &g, const Source &src, unsigned char *ring, uint32_t wave, uint32_t group, uint32_t lane, uint32_t nk, bool stores, i8_i32x4 (&acc)[BM][BN]) {
        const uint32_t wm = wave / GN, wn = wave % GN;
        const uint32_t sbase = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)ring;
        const uint32_t ra = wm * WM + (lane & 15u), rb = wn * WN + (lane & 15u);
        const uint32_t fa = sbase + ra * 128u + (((lane >> 4) ^ i8_swizzle(ra)) << 4);
        const uint32_t fb = sbase + rb * 128u + (((lane >> 4) ^ i8_swizzle(rb)) << 4);
        uint32_t sa = 0, sb = A_BYTES;                               // slots of the tile being consumed
        first_landed(nk, stores);
        Frag f0, f1;
        read_range<0, 0, NR>(fa + sa, fb + sb, f0);
        auto step = [&](uint32_t t, auto steady_c) {
            constexpr bool STEADY = decltype(steady_c)::value;        // every copy of the steady state is due
            arrived(f0);
            if constexpr (!STEADY) {
                const uint32_t k0 = (t * GK + group) * 128u;
                if (k0 + 128u > g.k) {
                    uint32_t l = lane;
                    asm volatile("" : "+v"(l));                      // (what the cut takes is worked out here, not kept over the loop)
#pragma unroll
                    for (int i = 0; i < BM; ++i) f0.a[i] = i8_cut(f0.a[i], k0 + (l >> 4) * 16u, g.k);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            phase<1, false>(fa + sa, fb + sb, f1, f0, acc, [](auto) {});
            arrived(f1);
            if constexpr (!STEADY) {
                const uint32_t k0 = (t * GK + group) * 128u;
                if (k0 + 128u > g.k) {
                    uint32_t l = lane;
                    asm volatile("" : "+v"(l));
#pragma unroll
                    for (int i = 0; i < BM; ++i) f1.a[i] = i8_cut(f1.a[i], k0 + 64u + (l >> 4) * 16u, g.k);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            next_landed<STEADY>(t, nk);
            __builtin_amdgcn_sched_barrier(0);
            const uint32_t na = next_slot(sa), nb = next_slot(sb);
            // (past the last tile the reads fetch what happens to be there, for nobody)
            phase<0, SLOTS || STEADY>(fa + na, fb + nb, f0, f1, acc, [&](auto q) { copy_behind<decltype(q)::value, STEADY>(src, ring, wave, t, nk, sa, sb); });
            sa = na; sb = nb;
        };
        uint32_t t = 0;
        for (; t + FAR < nk; ++t) step(t, std::true_type{});
        for (; t < nk; ++t) step(t, std::false_type{});
        arrived(f0);                                                  // nothing of the last reads outlives the loop
    }

    // Whether results are written with buffer stores, the same number by every wave
    static __device__ __forceinline__ bool counted(const I8Args &g) { return g.out_kind ? g.vec : g.vec && g.through; }
    // Sums to C
    __device__ static __forceinline__ void results(const I8Args &g, const I8Tile &tile, const I8Columns<TN, GATED> &cols, const Finals &fin, uint32_t lane, const i8_i32x4 (&acc)[KEEP][BN]) {
        const uint32_t r0 = fin.r0, c0 = fin.c0, q4 = lane >> 4;
        float sr[KEEP];
        fin.rows(lane, sr);
        auto value = [&](int i, int j) -> i8_f32x4 {
            if constexpr (GATED) return i8_gated(fin.scales[j], sr[i], acc[i][2 * j], acc[i][2 * j + 1]);
            else return i8_scaled(fin.scales[j], sr[i], acc[i][j]);
        };
        if (!counted(g)) {
            asm volatile("; results, single values");
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    const uint32_t r = r0 + i * 16u, col = c0 + j * 16u;
                    if (r < tile.rows && col < cols.of_c) i8_store4(g, tile.row0 + r, col, cols.of_c, value(i, j));
                }
            return;
        }
        // Buffer stores: what lies beyond the last row or column is dropped, so that every wave issues the same number of them (see first_landed)
        const uint32_t es = g.out_kind ? 2u : 4u, pitch = g.ldc * es;
        const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(static_cast<unsigned char *>(g.C) + (uint64_t)tile.row0 * pitch, 0, (int)((tile.rows - 1u) * pitch + cols.of_c * es), 0x00020000);
        // (the row goes into the lane's offset, not into a scalar one: a 16-byte store with that may read its last register too late)
        auto place = [&](uint32_t col) { return col < cols.of_c ? r0 * pitch + col * es : kOutside; };
        if (g.out_kind == 0) {
            asm volatile("; results, 32 bits");
            uint32_t at[NP];
#pragma unroll
            for (int j = 0; j < NP; ++j) at[j] = place(c0 + j * 16u);
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i8_u32x4, value(i, j)), rc, (int)(at[j] + i * 16u * pitch), 0, 18);
                    __builtin_amdgcn_sched_barrier(0);            // (left alone, the compiler scales everything first and spills)
                }
            }
        } else if constexpr (NP % 2 == 0) {
            // two neighbouring blocks: after the swap of odd and even 16-lane rows a lane holds 8 columns of one of them
            const uint32_t cc = c0 - q4 * 4u + (q4 & 1u) * 16u + (q4 >> 1) * 8u;
            auto store = [&](auto kind, auto policy) {
                constexpr uint32_t KIND = decltype(kind)::value;
                asm volatile("; results, kind %0, policy %1" ::"n"(KIND), "n"(decltype(policy)::value));
                uint32_t at[NP / 2];
#pragma unroll
                for (int j = 0; j < NP; j += 2) at[j / 2] = place(cc + j * 16u);
#pragma unroll
                for (int i = 0; i < KEEP; ++i) {
#pragma unroll
                    for (int j = 0; j < NP; j += 2) {
                        const i8_f32x4 x = value(i, j), y = value(i, j + 1);
                        const auto lo = __builtin_amdgcn_permlane16_swap(i8_pack(KIND, x[0], x[1]), i8_pack(KIND, y[0], y[1]), false, false);
                        const auto hi = __builtin_amdgcn_permlane16_swap(i8_pack(KIND, x[2], x[3]), i8_pack(KIND, y[2], y[3]), false, false);
                        __builtin_amdgcn_raw_buffer_store_b128(i8_u32x4{lo[0], hi[0], lo[1], hi[1]}, rc, (int)(at[j / 2] + i * 16u * pitch), 0, decltype(policy)::value);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };
            if (g.out_kind == 1u) {
                if (g.through) store(std::integral_constant<uint32_t, 1>{}, std::integral_constant<int, 18>{});
                else store(std::integral_constant<uint32_t, 1>{}, std::integral_constant<int, 0>{});
            } else {
                if (g.through) store(std::integral_constant<uint32_t, 2>{}, std::integral_constant<int, 18>{});
                else store(std::integral_constant<uint32_t, 2>{}, std::integral_constant<int, 0>{});
            }
        } else {
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    const i8_f32x4 x = value(i, j);
                    __builtin_amdgcn_raw_buffer_store_b64(i8_u32x2{i8_pack(g.out_kind, x[0], x[1]), i8_pack(g.out_kind, x[2], x[3])}, rc, (int)(place(c0 + j * 16u) + i * 16u * pitch), 0, 0);
                }
        }
    }
};

template <typename BODY, int WAVES_PER_SIMD> __global__ __launch_bounds__(BODY::WAVES * 64, WAVES_PER_SIMD) void ft_i8_block(I8Args a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    BODY::run(a, smem);
}

}  // namespace ftk

using namespace ftk;

namespace {

// PER_CU workgroups fit a CU: as many are launched as the device holds, and take the tiles in turn
template <typename BODY, int PER_CU, bool GROUPED> ft_status launch(I8Args &a, hipStream_t s) {
    constexpr auto KERNEL = &ft_i8_block<BODY, BODY::WAVES / 4 * PER_CU>;
    const hipError_t e = raise_lds_limit<KERNEL>();
    if (e != hipSuccess) { ftd_set_hip_error((int)e); return FT_ERR_HIP; }
    if (!i8_grid(a, BODY::TM, BODY::TN, GROUPED)) return FT_ERR_UNSUPPORTED;
    const uint32_t tiles = a.row_tiles * a.col_tiles, most = a.cus * PER_CU;
    hipLaunchKernelGGL(KERNEL, dim3(tiles < most ? tiles : most), dim3(BODY::WAVES * 64), BODY::LDS, s, a);
    return op_launched();
}
template <bool GROUPED, bool GATED> ft_status run(I8Kind kind, I8Args &a, hipStream_t s) {
    switch (kind) {
        case I8_256x256: return launch<I8Block<128, 64, 2, 4, 1, 0, GROUPED, GATED>, 1, GROUPED>(a, s);
        case I8_128x256: return launch<I8Block<64, 64, 2, 4, 1, 3, GROUPED, GATED>, 1, GROUPED>(a, s);
        case I8_128x128: return launch<I8Block<64, 64, 2, 2, 1, 2, GROUPED, GATED>, 2, GROUPED>(a, s);
        case I8_64x128: return launch<I8Block<32, 64, 2, 2, 1, 3, GROUPED, GATED>, 2, GROUPED>(a, s);
        default: return launch<I8Block<32, 32, 2, 2, 2, 4, GROUPED, GATED>, 1, GROUPED>(a, s);
    }
}

}  // namespace

namespace ftk {

ft_status i8_launch_blocks(I8Kind kind, bool grouped, I8Args &a, void *stream) {
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (grouped) return a.gated ? run<true, true>(kind, a, s) : run<true, false>(kind, a, s);
    return a.gated ? run<false, true>(kind, a, s) : run<false, false>(kind, a, s);
}

}  // namespace ftk
