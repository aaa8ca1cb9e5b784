// The experts' products on the 5th-generation tensor cores: grouped matrix products over the rows that the dispatch
// tables put side by side, one kernel template for the six products of a gated expert and its gradients.
//
//   GATE_UP       [g; u] = W_gate_up x        h = silu(g) u,  stores w h (and g, u for the backward)
//   DOWN          o = W_down (w h)            per slot; the sum over a token's slots is combine_kernel's
//   DH            dh = W_down^T dy            grad_w = <dh, h>,  dg = w dh u s (1 + g (1 - s)),  du = w dh silu(g)
//   DX            dx = W_gate_up^T [dg; du]   per slot
//   DW_DOWN       dW_down = dy^T (w h)        sum over the expert's slots
//   DW_GATE_UP    dW_gate_up = [dg; du]^T x
//
// A block per SM walks over output tiles.  Warp 0 brings operand tiles of 64 along the contraction into a ring of
// shared-memory stages by TMA, one thread of warp 1 issues tcgen05.mma into one of two accumulators in TMEM, warps 4 to 11 (4 to 7
// in DH) read the other one and finish the previous tile.  Operands that the contraction runs along the rows of (W_down in DH, W_gate_up in DX, both
// sides of the weight gradients) are read as they lie in memory: the tensor core takes them "MN-major".
//
// Measured on pairs of blocks (8192 tokens, 4 of 32 experts, 2048 x 1024, bf16; each kernel alone under the profiler): GATE_UP 225 us, DOWN
// 116 us, DX 219 us with the tensor pipe 68 to 75 % busy (1.18 to 1.26 PFLOP/s on the real rows), the weight gradients 126 and 232 us
// (57 and 64 % busy), DH 142 us (55 %: one set of warps does the heaviest epilogue).  Whole passes reach 0.85 to 0.99 PFLOP/s at 990 W and 1.34
// to 1.43 GHz; a library matrix product alone reaches 1.39 at 1.32 GHz under the same power limit, so the rest is pipe time: the shares above,
// 6 to 8 % padded rows and 15 % in tables, copies and sums.  With few tokens they are bound by the weights: 6.0 TB/s at 48 tokens on 128 experts.
//
// Roundings: the inputs of a product are 16-bit, so w h, g, u, dg, du are rounded to the storage type once, sums are
// fp32 in TMEM; o and dx are rounded once per slot before the fp32 sum over the slots: an fp32 copy would double the traffic of
// the combine (1.1 GB more, 0.16 ms by its bytes, on 1.65 ms for 131072 slots) to take away an error of the size of the final
// rounding.  Against 64 bits the outputs are 2.9e-3 (y, bf16; one rounding alone gives 1.7e-3) to 3.4e-3 (grad_x) off in the 2-norm.
#pragma once

#include <type_traits>

#include "common.cuh"
#include "tensor_core.cuh"

namespace lapsum {

enum ExpertsMode { GATE_UP = 0, DOWN = 1, DH = 2, DX = 3, DW_DOWN = 4, DW_GATE_UP = 5 };

struct ExpertsArgs {
    // The tables are the caller's memory: whatever they hold (a dispatch that was never run, a race of the caller's), no index
    // read from them is used unchecked; an entry, slot or expert out of range counts as a hole.
    const int32_t *entry_of, *tile_expert, *offsets, *counts;
    int entries, capacity;          // tokens k, slots
    const float *w;                 // per entry (token, choice)
    float *partial;                 // DH: per slot and column tile, <dh, h>
    uint32_t *status;
    unsigned long long wait_ns;     // bound of every wait
    int E, D, F, k, tokens;
    int keep;                       // GATE_UP: store g and u
    int row_tiles;                  // row tiles that the batch may need at most; those it does not need have tile_expert -1
    int early;                      // the tables were complete before the previous kernel of the stream began
    int hold;                       // test hook: the producer brings nothing, so the waits run out
};

template <typename T>
__device__ __forceinline__ void store8(T *p, const float *v)
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i];
    *reinterpret_cast<uint4 *>(p) = Io<T>::pack(x);
}
template <typename T>
__device__ __forceinline__ void load8(const T *p, float *v)
{
    float x[8];
    Io<T>::unpack(*reinterpret_cast<const uint4 *>(p), x);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i];
}
__device__ __forceinline__ float sigmoid_fast(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }

// The backward's silu(g) and slope s + silu(g) (1 - s), s = sigmoid(g), from a g that was kept in 16 bits.  fp16 keeps a g beyond 65504 as an
// infinity: there silu(-inf) is 0, not -inf x 0, and the slopes are 0 and 1, not an infinity times 0.  A NaN stays one through s.
template <typename T>
__device__ __forceinline__ float silu_of(float g, float s)
{
    return std::is_same<T, __half>::value ? fmaxf(g, -65504.f) * s : g * s;
}
template <typename T>
__device__ __forceinline__ float below_infinity(float a)
{
    return std::is_same<T, __half>::value ? fminf(a, 65504.f) : a;
}

// ---------------------------------------------------------------- the kernel ----
// Row tiles up to GATHER_ROWS take their tokens' rows from x by TMA gather, four rows per instruction.  A gather takes about 40
// cycles whatever the reuse (measured: 32 of them per step of 64 made the first product of 131072 slots 2.43 ms instead of
// 0.84 and 0.10 for the copy), so wider tiles read a copy of x in slot order that experts_gather_kernel writes at memory speed (8 of 64 experts,
// 2048 x 1024: 64-row tiles at 384 tokens 175 us with the copy, 198 us gathered; 128-row tiles at 512 tokens 177 and 223).
constexpr int GATHER_ROWS = 32;

// AR: rows of the row tile (slots), or of the output tile of a weight gradient (128 or 256).
//   256   a cluster of two blocks works on one 256 x 256 tile (cta_group::2): each block brings 128 rows of A and half of B, and
//         the tensor cores of both read both halves.  A single block's 128 x 256 tile needs 96 bytes per clock of shared memory
//         for the operands and another 96 for the copies, more than the 128 there are; the pair needs 64 + 64.
//   128   one block, M = 128.
//   < 128 the tensor core still works on M = 128: rows AR..127 are whatever the following stages hold, and nobody reads their
//         results.  Such tiles are bound by the weights they stream.
// KS: steps of 64 along the contraction in one stage.  With few rows a stage of several steps lets a row of weights arrive in
// runs of 128 KS bytes.
template <int MODE, int AR, int BN, int KS_>
struct ExpertsShape {
    static constexpr bool PAIR = AR == 256;
    static constexpr bool WGRAD = MODE == DW_DOWN || MODE == DW_GATE_UP;
    static constexpr bool A_GATHER = MODE == GATE_UP && AR <= GATHER_ROWS;
    static constexpr bool A_MN = WGRAD, B_MN = MODE >= DH;
    static constexpr int KS = KS_;
    static constexpr int ROWS = PAIR ? 128 : AR, COLS = PAIR ? BN / 2 : BN;  // what one block brings of A and B
    static constexpr int A_SUB = ROWS * 128, B_SUB = COLS * 128;             // bytes of one step
    static constexpr int A_BYTES = KS * A_SUB, B_BYTES = KS * B_SUB, STAGE = A_BYTES + B_BYTES;
    static constexpr int SLAB = 4096;                                        // 32 rows x 64 columns of results of one epilogue warp
    // Epilogue warps come in sets of four (a set reads the 128 lanes of TMEM); two sets share a tile's columns.  DH has one set and
    // four slabs per warp, two of which are loaded while the others are used.  Elsewhere a warp has two slabs where the ring keeps
    // four stages beside them (a prompt of 1021 tokens on 128 x 256 tiles: 262 us with one and four stages, 275 us with two and three).
    static constexpr int SETS = MODE == DH ? 1 : 2, SLABS = MODE == DH ? 4 : AR >= 128 && BN == 256 ? 1 : 2;
    static constexpr int THREADS = 128 + 128 * SETS;
    static constexpr int WARPS = SETS * (ROWS < 32 ? 1 : ROWS / 32);         // epilogue warps with rows
    static constexpr int FIT = (229376 - WARPS * SLABS * SLAB) / STAGE;
    static constexpr int STAGES = FIT < 12 ? FIT : 12;
    static constexpr int ACC = 2;  // accumulators: one is finished while the next is computed
    static constexpr int TMEM = ACC * BN;
    static constexpr int NSTEP = MODE == GATE_UP ? BN / 2 : BN;  // output columns of a tile
    static constexpr int SMEM = STAGES * STAGE + WARPS * SLABS * SLAB + 1024 + 512;
    // the A ring comes first: M = 128 rows read from its last stage stay inside the B ring behind it
    static_assert(STAGES >= 2 && STAGES * B_BYTES >= 16384 - A_SUB && TMEM <= 512 && NSTEP % 64 == 0, "tile does not fit");
};

struct ExpertsMaps {
    CUtensorMap a, b;    // operands
    CUtensorMap out;     // results: 64 columns x min(32, AR) rows
    CUtensorMap gu;      // g and u of a slot as [capacity][2][F]: stored by GATE_UP (training), loaded by DH
};

template <int MODE, int AR, int BN, int KS, typename T>
__global__ void __launch_bounds__((ExpertsShape<MODE, AR, BN, KS>::THREADS), 1) experts_kernel(const __grid_constant__ ExpertsMaps maps, const ExpertsArgs P)
{
    using S = ExpertsShape<MODE, AR, BN, KS>;
    constexpr bool PAIR = S::PAIR;
    extern __shared__ uint8_t raw[];
    const uint32_t ring_a = (smem_u32(raw) + 1023) & ~1023u, ring_b = ring_a + S::STAGES * S::A_BYTES;
    const uint32_t slabs = ring_b + S::STAGES * S::B_BYTES, bars = slabs + S::WARPS * S::SLABS * S::SLAB;
    const uint32_t full = bars, empty = full + 8 * S::STAGES, acc_full = empty + 8 * S::STAGES, acc_empty = acc_full + 8 * S::ACC,
                   drain = acc_empty + 8 * S::ACC, loaded = drain + 8;  // loaded: DH, two per epilogue warp
    __shared__ uint32_t tmem_at;
    __shared__ int abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = PAIR ? cluster_rank() : 0;

    if (tid == 0) {
        abort_flag = 0;
        for (int s = 0; s < S::STAGES; ++s) mbar_init(full + 8 * s, 1), mbar_init(empty + 8 * s, 1);
        for (int a = 0; a < S::ACC; ++a) mbar_init(acc_full + 8 * a, 1), mbar_init(acc_empty + 8 * a, (PAIR ? 8 : 4) * S::SETS);
        mbar_init(drain, 1);
        if constexpr (MODE == DH)
            for (int i = 0; i < 8; ++i) mbar_init(loaded + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (tid == 96) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.out) : "memory");
    }
    if (warp == 2) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_at)), "n"(S::TMEM) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_at)), "n"(S::TMEM) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        tc_fence_before();
    }
    __syncthreads();
    if constexpr (PAIR) cluster_barrier();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    // Weights may be brought while the previous kernel still writes the other operand: the producer waits for that kernel
    // behind its first copies of weights.  The next kernel may be scheduled from here on; it waits for this one in turn.
    const bool early = !S::WGRAD && P.early && warp == 0;
    if (!early) pdl_wait();
    if (tid == 64) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    constexpr int MT = PAIR ? 256 : 128;                                           // output rows of a weight gradient's tile
    const int M = MODE == DW_DOWN ? P.D : 2 * P.F;                                 // weight gradients only
    const int N = (MODE == DOWN || MODE == DX || MODE == DW_GATE_UP) ? P.D : P.F;  // output columns
    const int K = (MODE == GATE_UP || MODE == DH) ? P.D : MODE == DOWN ? P.F : 2 * P.F;
    const int nts = (N + S::NSTEP - 1) / S::NSTEP, mts = S::WGRAD ? (M + MT - 1) / MT : P.row_tiles;
    const int64_t tiles = S::WGRAD ? (int64_t)P.E * mts * nts : (int64_t)mts * nts;
    const int64_t tile0 = PAIR ? blockIdx.x / 2 : blockIdx.x, tile_step = PAIR ? gridDim.x / 2 : gridDim.x;

    struct Tile {
        int e, m0, n0, kb, nkb;  // expert (-1: no tile from here on), first slot (or output row), first output column, first slot of the contraction, stages
    };
    auto tile_at = [&](int64_t i) {
        Tile t;
        int nt;
        int64_t rest;
        if (tiles >> 31) {
            nt = (int)(i % nts), rest = i / nts;
        } else {  // divisions of 64 bits cost hundreds of cycles
            const uint32_t q = (uint32_t)i / (uint32_t)nts;
            nt = (int)((uint32_t)i - q * (uint32_t)nts), rest = q;
        }
        t.n0 = nt * S::NSTEP;
        if constexpr (S::WGRAD) {
            t.e = (int)((uint32_t)rest / (uint32_t)mts);  // experts x row tiles stay below 2^31
            t.m0 = (int)((uint32_t)rest - (uint32_t)t.e * (uint32_t)mts) * MT + (int)rank * 128;
            t.kb = min(max(ld(P.offsets + t.e), 0), P.capacity);
            t.nkb = (min(max(ld(P.counts + t.e), 0), P.capacity) + 63) / 64;  // the last stage's holes are zeros
        } else {
            t.e = __ldcg(P.tile_expert + rest);  // past L1: it may be read before griddepcontrol.wait
            if ((unsigned)t.e >= (unsigned)P.E) t.e = -1;
            t.m0 = (int)rest * AR + (int)rank * 128;
            t.kb = 0;
            t.nkb = (K + 64 * KS - 1) / (64 * KS);  // columns beyond K read as zeros
        }
        return t;
    };
    Waits waits{&abort_flag, P.status, P.wait_ns, LAPSUM_ST_EXPERTS_TIMEOUT};

    if (warp == 0) {
        // ------------------------------------------------ producer
        uint32_t fill = 0;
        bool ok = true;
        auto load_2d = [&](uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
            if constexpr (PAIR) tma_pair_2d(dst, map, x, y, bar);
            else tma_load_2d(dst, map, x, y, bar);
        };
        auto load_3d = [&](uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
            if constexpr (PAIR) tma_pair_3d(dst, map, x, y, z, bar);
            else tma_load_3d(dst, map, x, y, z, bar);
        };
        // The next tile's expert and tokens are on their way while this tile's copies are issued.
        Tile next;
        next.e = -1;
        int4 entries = make_int4(0, 0, 0, 0);
        auto look_ahead = [&](int64_t i) {
            if (i < tiles) next = tile_at(i);
            else next.e = -1;
            if constexpr (S::A_GATHER)  // four neighbouring slots per lane
                if (i < tiles && lane < AR / 4) entries = ld(reinterpret_cast<const int4 *>(P.entry_of + next.m0 + 4 * lane));
        };
        int4 rows = make_int4(0, 0, 0, 0);  // the tile's tokens; holes give a row beyond the matrix, which reads as zeros
        int fours = 0;                      // fours of slots with a token, from the tile's start; the others' rows keep what they hold
        auto bring_a = [&](const Tile &t, int kb, uint32_t s, uint32_t bar) {
            const uint32_t a = ring_a + s * S::A_BYTES;
            if constexpr (S::WGRAD) {
                if (lane < 2) load_2d(a + lane * 8192, &maps.a, t.m0 + lane * 64, t.kb + kb * 64, bar);
            } else {
#pragma unroll
                for (int q = 0; q < KS; ++q) {
                    const int k0 = (kb * KS + q) * 64;
                    if constexpr (S::A_GATHER) {
                        if (lane < fours) tma_gather4(a + q * S::A_SUB + lane * 512, &maps.a, k0, rows, bar);
                    } else {
                        if (lane == 0) load_2d(a + q * S::A_SUB, &maps.a, k0, t.m0, bar);
                    }
                }
            }
        };
        auto bring_b = [&](const Tile &t, int kb, uint32_t s, uint32_t bar) {
            const uint32_t b = ring_b + s * S::B_BYTES;
            const int n0 = t.n0 + (int)rank * S::COLS;  // of this block; GATE_UP: see below
            if constexpr (S::WGRAD) {
                if (lane >= 2 && lane < 2 + S::COLS / 64)
                    load_2d(b + (lane - 2) * 8192, &maps.b, n0 + (lane - 2) * 64, t.kb + kb * 64, bar);
            } else {
#pragma unroll
                for (int q = 0; q < KS; ++q) {
                    const int k0 = (kb * KS + q) * 64;
                    const uint32_t bq = b + q * S::B_SUB;
                    if constexpr (MODE == GATE_UP) {  // gate rows, then up rows; a pair's blocks bring one kind each
                        if constexpr (PAIR) {
                            if (lane == 0) load_3d(bq, &maps.b, k0, t.n0, 2 * t.e + (int)rank, bar);
                        } else {
                            if (lane < 2) load_3d(bq + lane * (S::B_SUB / 2), &maps.b, k0, t.n0, 2 * t.e + lane, bar);
                        }
                    } else if constexpr (MODE == DOWN) {
                        if (lane == 0) load_3d(bq, &maps.b, k0, n0, t.e, bar);
                    } else {
                        if (lane < S::COLS / 64) load_3d(bq + lane * 8192, &maps.b, n0 + lane * 64, k0, t.e, bar);
                    }
                }
            }
        };
        auto barrier_of = [&](uint32_t s) { return PAIR ? in_block(full + 8 * s, 0) : full + 8 * s; };  // a pair's first block counts for both
        auto announce = [&](uint32_t s) {
            const uint32_t bytes = S::A_GATHER ? KS * 512 * fours + S::B_BYTES : S::STAGE;
            if (lane == 0 && rank == 0) mbar_expect_tx(full + 8 * s, PAIR ? 2 * bytes : bytes);
            __syncwarp();
        };
        look_ahead(tile0);
        int ahead = 0;  // stages of the first tile that have their weights already
        if (early) {
            if (next.e >= 0 && !P.hold)
                for (; ahead < next.nkb && ahead < S::STAGES; ++ahead) {
                    announce(ahead);
                    bring_b(next, ahead, ahead, barrier_of(ahead));
                }
            pdl_wait();
        }
        for (int64_t i = tile0; i < tiles && ok; i += tile_step) {
            const Tile t = next;
            if (t.e < 0) break;
            if constexpr (S::A_GATHER) {
                rows = make_int4(entries.x < 0 ? P.tokens : entries.x / P.k, entries.y < 0 ? P.tokens : entries.y / P.k,
                                 entries.z < 0 ? P.tokens : entries.z / P.k, entries.w < 0 ? P.tokens : entries.w / P.k);
                fours = __popc(__ballot_sync(FULL, lane < AR / 4 && entries.x >= 0));  // a tile's entries come before its holes
            }
            look_ahead(i + tile_step);
            for (int kb = 0; kb < t.nkb; ++kb, ++fill) {
                const uint32_t s = fill % S::STAGES, phase = (fill / S::STAGES) & 1;
                ok = waits.wait(empty + 8 * s, phase ^ 1);
                ok = __all_sync(FULL, ok);
                if (!ok || P.hold) break;
                const bool there = (int)fill < ahead;
                if (!there) announce(s);
                bring_a(t, kb, s, barrier_of(s));
                if (!there) bring_b(t, kb, s, barrier_of(s));
            }
            if (P.hold) break;
        }
        // every copy has landed and every product has read its stage before the block may end
        const uint32_t first = fill > S::STAGES ? fill - S::STAGES : 0;
        for (uint32_t f = first; f < fill; ++f) {
            const uint32_t s = f % S::STAGES, phase = (f / S::STAGES) & 1;
            if (rank == 0) waits.plain(full + 8 * s, phase, false);
            if (ok) waits.wait(empty + 8 * s, phase);
        }
    } else if (warp == 1) {
        // ------------------------------------------------ one thread issues the products (a pair's: one of its first block)
        if (lane == 0 && rank == 0) {
            constexpr uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
            constexpr uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | ((S::A_MN ? 1u : 0u) << 15) |
                                       ((S::B_MN ? 1u : 0u) << 16) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((PAIR ? 256 : 128) >> 4) << 24);
            constexpr uint32_t step_a = S::A_MN ? 2048 : 32, step_b = S::B_MN ? 2048 : 32;  // 16 along the contraction
            uint32_t fill = 0, it = 0;
            bool ok = true, any = false;
            for (int64_t i = tile0; i < tiles && ok; i += tile_step) {
                const Tile t = tile_at(i);
                if (t.e < 0) break;
                if (t.nkb == 0) continue;
                const uint32_t buf = it % S::ACC, phase = (it / S::ACC) & 1;
                ++it;
                ok = waits.wait(acc_empty + 8 * buf, phase ^ 1);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + buf * BN;
                for (int kb = 0; kb < t.nkb; ++kb, ++fill) {
                    const uint32_t s = fill % S::STAGES;
                    ok = waits.wait(full + 8 * s, (fill / S::STAGES) & 1);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int h = 0; h < KS; ++h) {
                        const uint64_t a = smem_desc(ring_a + s * S::A_BYTES + h * S::A_SUB, S::A_MN),
                                       b = smem_desc(ring_b + s * S::B_BYTES + h * S::B_SUB, S::B_MN);
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            tc_mma<PAIR>(d, a + q * (step_a >> 4), b + q * (step_b >> 4), idesc, (kb | h | q) != 0);
                    }
                    any = true;
                    tc_commit<PAIR>(empty + 8 * s);
                }
                if (ok) tc_commit<PAIR>(acc_full + 8 * buf);
            }
            if (!ok && any) {  // a wait ran out: the products already issued end before the block does
                tc_commit<PAIR>(drain);
                waits.plain(drain, 0, false);
            }
        }
    } else if (warp >= 4) {
        // ------------------------------------------------ epilogue: one accumulator row per thread, 64 columns at a time.
        // A warp puts its 32 rows x 64 columns as 16-bit values into a slab of its own (rows of 128 bytes, 16-byte pieces
        // exchanged by the row's low three bits, as TMA's 128-byte swizzle has it) and stores it with one TMA instruction:
        // a row per thread written directly costs the load / store unit 32 lines per instruction.
        const int ew = warp & 3, set = (warp - 4) >> 2, row = 32 * ew + lane;
        const uint32_t lanes = (uint32_t)ew << 21;  // 32 TMEM lanes per warp, lane index in the upper half
        const uint32_t slab = slabs + (set * (S::WARPS / S::SETS) + ew) * S::SLABS * S::SLAB;  // of live warps only
        const bool live = ew * 32 < S::ROWS, mine = row < S::ROWS;  // live: uniform in the warp
        auto piece = [&](uint32_t base, int j) { return base + lane * 128 + ((j ^ (lane & 7)) << 4); };  // 8 columns of my row
        auto put = [&](uint32_t base, int j, const float *v) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = v[i];
            const uint4 q = Io<T>::pack(x);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece(base, j)), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
        };
        auto get = [&](uint32_t base, int j, float *v) {
            uint4 q;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(piece(base, j)) : "memory");
            float x[8];
            Io<T>::unpack(q, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x[i];
        };
        uint32_t it = 0, chunk = 0, used = 0;  // chunk: DH: pairs of slabs used so far; used: slabs
        bool ok = true;
        auto bring = [&](const Tile &t, int c, uint32_t q) {  // DH: g and u of 64 columns into pair q & 1
            const uint32_t at = slab + (q & 1) * 2 * S::SLAB, bar = loaded + 8 * (2 * ew + (q & 1));
            if (lane == 0) {
                mbar_expect_tx(bar, 2 * S::SLAB);
                tma_load_3d(at, &maps.gu, t.n0 + c, 0, t.m0 + 32 * ew, bar);
                tma_load_3d(at + S::SLAB, &maps.gu, t.n0 + c, 1, t.m0 + 32 * ew, bar);
            }
        };
        for (int64_t i = tile0; i < tiles; i += tile_step) {
            const Tile t = tile_at(i);
            if (t.e < 0) break;
            const uint32_t buf = it % S::ACC, phase = (it / S::ACC) & 1;
            int entry = -1;
            float w = 0.f, dot = 0.f;
            if constexpr (MODE == GATE_UP || MODE == DH) {
                if (mine) entry = ld(P.entry_of + t.m0 + row);
                if ((unsigned)entry >= (unsigned)P.entries) entry = -1;
                if (entry >= 0) w = ld(P.w + entry);
            }
            if constexpr (MODE == DH) {
                if (live) {
                    if (lane == 0) tma_store_wait_read<0>();
                    __syncwarp();
                    bring(t, 0, chunk);
                }
            }
            if (t.nkb > 0) {
                ++it;
                ok = waits.wait(acc_full + 8 * buf, phase);
                if (!__all_sync(FULL, ok)) {
                    if (MODE == DH && live) waits.plain(loaded + 8 * (2 * ew + (chunk & 1)), (chunk >> 1) & 1, false);  // the copy in flight
                    break;
                }
                tc_fence_after();
            }
            const uint32_t d = tmem + buf * BN + lanes;
            if (live && (!S::WGRAD || t.m0 + 32 * ew < M)) {
#pragma unroll 1
                for (int c = 64 * set; c < S::NSTEP && t.n0 + c < N; c += 64 * S::SETS, ++chunk) {
                    if constexpr (MODE == GATE_UP) {
                        // w h, and for the backward g and u, one after the other
                        for (int what = 0; what < (P.keep ? 3 : 1); ++what) {
                            const uint32_t at = slab + (used++ % S::SLABS) * S::SLAB;
                            if (lane == 0) tma_store_wait_read<S::SLABS - 1>();
                            __syncwarp();
#pragma unroll
                            for (int j = 0; j < 64; j += 32) {
                                float g[2][16], u[2][16];
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    if (what != 2) tmem_ld16(d + c + j + 16 * h, g[h]);
                                    if (what != 1) tmem_ld16(d + BN / 2 + c + j + 16 * h, u[h]);
                                }
                                tmem_wait_ld(g[0]);
                                tmem_pin(g[1]), tmem_pin(u[0]), tmem_pin(u[1]);
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    if (what == 0) {
#pragma unroll
                                        for (int v = 0; v < 16; ++v)
                                            g[h][v] = entry >= 0 ? w * (g[h][v] * sigmoid_fast(g[h][v]) * u[h][v]) : 0.f;
                                    } else if (what == 2) {
#pragma unroll
                                        for (int v = 0; v < 16; ++v) g[h][v] = u[h][v];
                                    }
                                    if (mine) put(at, j / 8 + 2 * h, g[h]), put(at, j / 8 + 2 * h + 1, g[h] + 8);
                                }
                            }
                            fence_async_smem();
                            __syncwarp();
                            if (lane == 0) {
                                if (what == 0) tma_store_2d(&maps.out, at, t.n0 + c, t.m0 + 32 * ew);
                                else tma_store_3d(&maps.gu, at, t.n0 + c, what - 1, t.m0 + 32 * ew);
                                tma_store_commit();
                            }
                        }
                    } else if constexpr (MODE == DH) {
                        // the pair of slabs holds g and u and takes dg and du in their place; the other pair is filled meanwhile
                        const uint32_t at = slab + (chunk & 1) * 2 * S::SLAB;
                        if (c + 64 < S::NSTEP && t.n0 + c + 64 < N) {
                            if (lane == 0) tma_store_wait_read<0>();
                            __syncwarp();
                            bring(t, c + 64, chunk + 1);
                        }
                        waits.plain(loaded + 8 * (2 * ew + (chunk & 1)), (chunk >> 1) & 1, false);  // whatever the others do: the copy must land
#pragma unroll
                        for (int j = 0; j < 64; j += 16) {
                            float dh[16];
                            tmem_ld16(d + c + j, dh);
                            tmem_wait_ld(dh);
#pragma unroll
                            for (int p = 0; p < 2; ++p) {
                                float g[8], u[8];
                                get(at, j / 8 + p, g);
                                get(at + S::SLAB, j / 8 + p, u);
                                // a hole's gradients are zeros whatever the weights and the buffers hold; so are columns beyond F
                                const bool real = entry >= 0 && t.n0 + c + j + 8 * p < N;
#pragma unroll
                                for (int v = 0; v < 8; ++v) {
                                    const float s = sigmoid_fast(g[v]), a = silu_of<T>(g[v], s), x = dh[8 * p + v], xw = x * w, uv = u[v];
                                    dot += real ? x * a * uv : 0.f;
                                    g[v] = real ? xw * uv * (s + below_infinity<T>(a) * (1.f - s)) : 0.f;
                                    u[v] = real ? xw * a : 0.f;
                                }
                                put(at, j / 8 + p, g);
                                put(at + S::SLAB, j / 8 + p, u);
                            }
                        }
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_3d(&maps.out, at, t.n0 + c, 0, t.m0 + 32 * ew);
                            tma_store_3d(&maps.out, at + S::SLAB, t.n0 + c, 1, t.m0 + 32 * ew);
                            tma_store_commit();
                        }
                    } else {
                        const uint32_t at = slab + (used++ % S::SLABS) * S::SLAB;
                        float v[4][16];  // all 64 columns are asked for before the first is used
                        if (t.nkb > 0) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) tmem_ld16(d + c + 16 * j, v[j]);
                            tmem_wait_ld(v[0]);
                            tmem_pin(v[1]), tmem_pin(v[2]), tmem_pin(v[3]);
                        } else {  // an expert without tokens
#pragma unroll
                            for (int j = 0; j < 64; ++j) v[j / 16][j % 16] = 0.f;
                        }
                        if (lane == 0) tma_store_wait_read<S::SLABS - 1>();
                        __syncwarp();
                        if (mine) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) put(at, j, v[j / 2] + 8 * (j % 2));
                        }
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            if constexpr (S::WGRAD) tma_store_3d(&maps.out, at, t.n0 + c, t.m0 + 32 * ew, t.e);
                            else tma_store_2d(&maps.out, at, t.n0 + c, t.m0 + 32 * ew);
                            tma_store_commit();
                        }
                    }
                }
            }
            if (MODE == DH && mine) P.partial[(int64_t)(t.m0 + row) * nts + t.n0 / S::NSTEP] = dot;
            if (t.nkb > 0) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(PAIR ? in_block(acc_empty + 8 * buf, 0) : acc_empty + 8 * buf);
            }
        }
        if (lane == 0) tma_store_wait_all();
    }
    __syncwarp();
    __syncthreads();
    if constexpr (PAIR) cluster_barrier();
    if (warp == 2) {
        tc_fence_after();
        if constexpr (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM) : "memory");
    }
}

// ------------------------------------------------------------- a few tokens ----
// One or a few tokens: every weight is used once, so the products are streams of weights at memory speed and the tensor core
// has nothing to add, as long as tokens hardly share experts (few_tokens, experts_api.cu).  Each lane keeps eight or more 16-byte loads in flight; a token's choices are finished in one warp, so
// there is neither a table of slots to combine nor a rounding per slot.
// hw[entry][f] = w silu(g) u.  A block has FEW_FEATURES features of one entry (so its expert is looked up once), a warp one
// feature at a time: sixteen loads of its two rows at once, 16 warps per SM, 128 KB on their way.  (Three blocks per SM spill and
// are no faster; 8, 32 or 64 features a block are within 5 %.)
constexpr int FEW_FEATURES = 16;
template <typename T>
__global__ void __launch_bounds__(256, 2) experts_few_gate_up_kernel(const T *x, int64_t stride, const T *w_gate_up, const float *w,
                                                                     const int32_t *slot_of, const int32_t *tile_expert, int shift, int capacity,
                                                                     int E, T *hw, int k, int D, int F)
{
    pdl_wait();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, entry = blockIdx.y;
    const int slot = ld(slot_of + entry);
    if ((unsigned)slot >= (unsigned)capacity) return;  // dropped: the second product skips it too
    const int64_t e = ld(tile_expert + (slot >> shift));
    if (e < 0 || e >= E) return;
    const T *const xt = x + entry / k * stride;
    const float scale = ld(w + entry);
    const int f1 = min(F, (int)(blockIdx.x + 1) * FEW_FEATURES);
    for (int f = blockIdx.x * FEW_FEATURES + (threadIdx.x >> 5); f < f1; f += 8) {
        const T *const gate = w_gate_up + (e * 2 * F + f) * D, *const up = gate + (int64_t)F * D;
        float g = 0.f, u = 0.f;
        for (int c = 8 * lane; c < D; c += 2048) {
            uint4 a[8], b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = c + 256 * i < D;
                a[i] = in ? __ldcs(reinterpret_cast<const uint4 *>(gate + c + 256 * i)) : Io<T>::zero();
                b[i] = in ? __ldcs(reinterpret_cast<const uint4 *>(up + c + 256 * i)) : Io<T>::zero();
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + 256 * i < D) {
                    const uint4 v = ld(reinterpret_cast<const uint4 *>(xt + c + 256 * i));
                    g = dot8<T>(a[i], v, g);
                    u = dot8<T>(b[i], v, u);
                }
        }
        g = warp_total(g), u = warp_total(u);
        if (lane == 0) Io<T>::store1(hw + (int64_t)entry * F + f, scale * (g * sigmoid_fast(g) * u));
    }
}

// y[t][d] = sum over the token's choices of <W_down[e][d], hw>.  A block has four values of d, a warp every eighth choice: four
// rows in steps of 1024, sixteen loads at once (three blocks per SM, though that spills some 60 bytes), the first of them before the activations are there.  The warps' sums are added
// in order.
template <typename T>
__global__ void __launch_bounds__(256, 3) experts_few_down_kernel(const T *w_down, const T *hw, const int32_t *slot_of, const int32_t *tile_expert,
                                                                  int shift, int capacity, int E, T *y, int k, int D, int F)
{
    __shared__ float part[8][4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = blockIdx.y, d = 4 * blockIdx.x;  // D is a multiple of 8
    float sum[4] = {};
    bool waited = false;
    for (int j = warp; j < k; j += 8) {
        const int slot = __ldcg(slot_of + (int64_t)t * k + j);
        if ((unsigned)slot >= (unsigned)capacity) continue;
        const int64_t e = __ldcg(tile_expert + (slot >> shift));
        if (e < 0 || e >= E) continue;
        const T *const rows = w_down + (e * D + d) * F, *const v = hw + ((int64_t)t * k + j) * F;
        for (int c = 8 * lane; c < F; c += 1024) {
            uint4 a[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    a[r][i] = c + 256 * i < F ? __ldcs(reinterpret_cast<const uint4 *>(rows + (int64_t)r * F + c + 256 * i)) : Io<T>::zero();
            if (!waited) pdl_wait(), waited = true;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + 256 * i < F) {
                    const uint4 h = ld(reinterpret_cast<const uint4 *>(v + c + 256 * i));
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[r] = dot8<T>(a[r][i], h, sum[r]);
                }
        }
    }
    if (!waited) pdl_wait();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        sum[r] = warp_total(sum[r]);
        if (lane == 0) part[warp][r] = sum[r];
    }
    __syncthreads();
    if (threadIdx.x < 4) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += part[i][threadIdx.x];
        Io<T>::store1(y + (int64_t)t * D + d + threadIdx.x, s);
    }
}

// Rows of a matrix in slot order.  The first blocks have a warp per token and 1024 columns, which reads them once and writes them
// to the token's slots; the others (backward only: the sums over slots must not meet what a hole's row held) fill the holes below
// the last used slot with zeros, a warp per four slots.  Bound by the bytes written: 131072 slots of 4 KB in 98 us (6.1 TB/s).
template <typename T>
__global__ void __launch_bounds__(256) experts_gather_kernel(const T *x, int64_t stride, const int32_t *slot_of, const int32_t *entry_of,
                                                             const int32_t *used, T *out, int64_t tokens, int token_blocks, int capacity, int k, int D)
{
    pdl_wait();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, n = D / 8, parts = (D + 1023) / 1024;
    const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if ((int)blockIdx.x < token_blocks) {
        const int64_t t = unit / parts;
        if (t >= tokens) return;
        const int i = (int)(unit - t * parts) * 128 + lane;
        const int mine = lane < k ? ld(slot_of + t * k + lane) : -1;
        const uint4 *const from = reinterpret_cast<const uint4 *>(x + t * stride);
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + 32 * j < n) v[j] = ld(from + i + 32 * j);
        for (int c = 0; c < k; ++c) {
            const int slot = __shfl_sync(FULL, mine, c);
            if ((unsigned)slot >= (unsigned)capacity) continue;
            uint4 *const to = reinterpret_cast<uint4 *>(out + (int64_t)slot * D);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + 32 * j < n) to[i + 32 * j] = v[j];
        }
    } else {
        const int64_t slot0 = (unit - 8 * (int64_t)token_blocks) * 4;
        if (slot0 >= min(ld(used), capacity)) return;  // both multiples of 64
        const int4 e = ld(reinterpret_cast<const int4 *>(entry_of + slot0));
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if ((s == 0 ? e.x : s == 1 ? e.y : s == 2 ? e.z : e.w) >= 0) continue;
            uint4 *const to = reinterpret_cast<uint4 *>(out + (slot0 + s) * D);
            for (int i = lane; i < n; i += 32) to[i] = make_uint4(0, 0, 0, 0);
        }
    }
}

// y_t = sum over the token's slots, in the order of its choices, eight columns per thread; dropped entries (-1) add nothing.
// With `partial` also grad_w of the token's entries: the column tiles' sums in order.  Bound by memory: 131072 slots of 4 KB in 89 us
// (6.7 TB/s).  The last kernel of a call lets no other start early: its results may go to kernels that read through the non-coherent path.
template <typename T>
__global__ void __launch_bounds__(256) experts_combine_kernel(const T *slots, const int32_t *slot_of, T *out, int64_t out_stride,
                                                              const float *partial, void *grad_w, int grad_w_f32, int64_t tokens, int capacity, int k, int D,
                                                              int nts)
{
    pdl_wait();
    const int per = D / 8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t t = id / per;
    if (t >= tokens) return;
    const int c = (int)(id - t * per);
    float sum[8] = {};
    const int32_t *const at = slot_of + t * k;
    for (int j0 = 0; j0 < k; j0 += 8) {  // eight slots' loads in flight
        int s[8];
        uint4 q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = j0 + j < k ? ld(at + j0 + j) : -1;
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = (unsigned)s[j] < (unsigned)capacity ? ld(reinterpret_cast<const uint4 *>(slots + (int64_t)s[j] * D + 8 * c)) : Io<T>::zero();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v[8];
            Io<T>::unpack(q[j], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        }
    }
    store8(out + t * out_stride + 8 * c, sum);
    if (partial != nullptr)
        for (int j = c; j < k; j += per) {
            const int s = ld(at + j);
            float g = 0.f;
            if ((unsigned)s < (unsigned)capacity)
                for (int n = 0; n < nts; ++n) g += partial[(int64_t)s * nts + n];
            if (grad_w_f32) static_cast<float *>(grad_w)[t * k + j] = g;
            else Io<T>::store1(static_cast<T *>(grad_w) + t * k + j, g);
        }
}

}  // namespace lapsum
