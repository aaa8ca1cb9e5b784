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
// shared-memory stages by TMA, one thread of warp 1 issues tcgen05.mma into one of two accumulators in TMEM, warps 4-7 read the other one
// and finish the previous tile.  Operands that the contraction runs along the rows of (W_down in DH, W_gate_up in DX, both
// sides of the weight gradients) are read as they lie in memory: the tensor core takes them "MN-major".
//
// Roundings: the inputs of a product are 16-bit, so w h, g, u, dg, du are rounded to the storage type once, sums are
// fp32 in TMEM; o and dx are rounded once per slot before the fp32 sum over the slots (an fp32 copy would double the
// traffic of the combine for an error of the size of the final rounding).
#pragma once
#include <cuda.h>

#include <type_traits>

#include "common.cuh"

namespace lapsum {

enum ExpertsMode { GATE_UP = 0, DOWN = 1, DH = 2, DX = 3, DW_DOWN = 4, DW_GATE_UP = 5 };

struct ExpertsArgs {
    const int32_t *entry_of, *tile_expert, *offsets;
    const float *w;                 // per entry (token, choice)
    void *out0, *out1;              // per mode, see the epilogues
    const void *in0;                // DH: the saved [g, u]
    float *partial;                 // DH: per slot and column tile, <dh, h>
    uint32_t *status;
    int64_t slots;                  // capacity of the slot buffers
    unsigned long long wait_ns;     // bound of every wait
    int E, D, F, k, tokens, rows;   // rows: slots per row tile
    int hold;                       // test hook: the producer brings nothing, so the waits run out
};

// ------------------------------------------------------------------- PTX ----
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long global_ns()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
// four rows of a matrix, 64 columns each; a row index beyond the matrix reads as zeros
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap *map, int x, int4 r, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(map), "r"(x), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&v)[16])
{
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
// The wait names the loaded registers as its operands, so that no use of theirs can be scheduled before it.
__device__ __forceinline__ void tmem_pin(float (&v)[16])
{
    asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]),
                 "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]));
}
__device__ __forceinline__ void tmem_wait_ld(float (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    tmem_pin(v);
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a),
                 "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle.  K-major: rows of 64 elements along the contraction, groups of 8 rows
// 1024 bytes apart.  MN-major: rows of 64 elements along M or N, one per index of the contraction; groups of 8 such rows
// 1024 bytes apart, the next 64 of M or N 8192 bytes (64 rows) further on.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, bool mn_major)
{
    const uint64_t lbo = mn_major ? 8192 >> 4 : 1, sbo = 1024 >> 4;
    return (uint64_t)((addr & 0x3ffff) >> 4) | (lbo << 16) | (sbo << 32) | (1ull << 46) | (2ull << 61);
}

// Waits of one block: bounded; the first that runs out raises the block's flag, on which all others give up.
struct Waits {
    volatile int *abort;
    uint32_t *status;
    unsigned long long limit;
    __device__ __forceinline__ bool plain(uint32_t bar, uint32_t parity, bool heed)
    {
        if (mbar_try(bar, parity)) return true;
        const unsigned long long t0 = global_ns();
        for (;;) {
            for (int i = 0; i < 32; ++i)
                if (mbar_try(bar, parity)) return true;
            if (heed && *abort) return false;
            if (global_ns() - t0 > limit) {
                *abort = 1;
                atomicOr(status, LAPSUM_ST_EXPERTS_TIMEOUT);
                return false;
            }
        }
    }
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) { return plain(bar, parity, true); }
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

// ---------------------------------------------------------------- the kernel ----
// AR: rows of the A tile that are brought (the slots of a row tile; 128 = M for the weight gradients).  The tensor core
// always works on M = 128 rows: with AR < 128 it reads the next stages' bytes as rows AR..127, whose results nobody reads.
// Row tiles up to GATHER_ROWS take their tokens' rows from x by TMA gather, four rows per instruction.  A gather takes about 40
// cycles whatever the reuse (measured: 32 of them per step of 64 made the first product of 131072 slots 2.43 ms instead of
// 0.9), so wider tiles read a copy of x in slot order that gather_rows_kernel writes at memory speed.
constexpr int GATHER_ROWS = 32;

template <int MODE, int AR, int BN>
struct ExpertsShape {
    static constexpr bool WGRAD = MODE == DW_DOWN || MODE == DW_GATE_UP;
    static constexpr bool A_GATHER = MODE == GATE_UP && AR <= GATHER_ROWS;
    static constexpr bool A_MN = WGRAD, B_MN = MODE >= DH;
    static constexpr int A_BYTES = AR * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = (196608 / STAGE) < 16 ? (196608 / STAGE) : 16;
    static constexpr int ACC = 2;                       // accumulators
    static constexpr int TMEM = ACC * BN < 32 ? 32 : ACC * BN;
    static constexpr int NSTEP = MODE == GATE_UP ? BN / 2 : BN;  // output columns of a tile
    // the A ring comes first: M = 128 rows read from its last stage stay inside the B ring behind it
    static constexpr int SMEM = STAGES * STAGE + 1024 + 512;
    static_assert(STAGES * B_BYTES >= 16384 - A_BYTES, "the A operand's 128 rows must stay inside the allocation");
};

template <int MODE, int AR, int BN, typename T>
__global__ void __launch_bounds__(256, 1)
experts_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const ExpertsArgs P)
{
    using S = ExpertsShape<MODE, AR, BN>;
    extern __shared__ uint8_t raw[];
    const uint32_t raw_at = smem_u32(raw), ring_a = (raw_at + 1023) & ~1023u, ring_b = ring_a + S::STAGES * S::A_BYTES;
    const uint32_t bars = ring_b + S::STAGES * S::B_BYTES;
    const uint32_t full = bars, empty = bars + 8 * S::STAGES, acc_full = empty + 8 * S::STAGES, acc_empty = acc_full + 8 * S::ACC,
                   drain = acc_empty + 8 * S::ACC;
    __shared__ uint32_t tmem_at;
    __shared__ int abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        abort_flag = 0;
        for (int s = 0; s < S::STAGES; ++s) mbar_init(full + 8 * s, 1), mbar_init(empty + 8 * s, 1);
        for (int a = 0; a < S::ACC; ++a) mbar_init(acc_full + 8 * a, 1), mbar_init(acc_empty + 8 * a, 128);
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_at)), "n"(S::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    pdl_wait();

    const int M = MODE == DW_DOWN ? P.D : 2 * P.F;                                 // weight gradients only
    const int N = (MODE == DOWN || MODE == DX || MODE == DW_GATE_UP) ? P.D : P.F;  // output columns
    const int K = (MODE == GATE_UP || MODE == DH) ? P.D : MODE == DOWN ? P.F : 2 * P.F;
    const int nts = (N + S::NSTEP - 1) / S::NSTEP, mts = S::WGRAD ? (M + 127) / 128 : __ldg(P.offsets + P.E) / P.rows;
    const int64_t tiles = S::WGRAD ? (int64_t)P.E * mts * nts : (int64_t)mts * nts;

    struct Tile {
        int e, m0, n0, kb, nkb;  // expert, first slot (or output row), first output column, first slot of the contraction, steps
    };
    auto tile_at = [&](int64_t i) {
        Tile t;
        const int nt = (int)(i % nts);
        const int64_t rest = i / nts;
        t.n0 = nt * S::NSTEP;
        if constexpr (S::WGRAD) {
            t.e = (int)(rest / mts);
            t.m0 = (int)(rest % mts) * 128;
            t.kb = __ldg(P.offsets + t.e);
            t.nkb = (__ldg(P.offsets + t.e + 1) - t.kb) / 64;
        } else {
            t.e = __ldg(P.tile_expert + rest);
            t.m0 = (int)rest * P.rows;
            t.kb = 0;
            t.nkb = (K + 63) / 64;
        }
        return t;
    };
    Waits waits{&abort_flag, P.status, P.wait_ns};

    if (warp == 0) {
        // ------------------------------------------------ producer: all lanes, one gather (four rows) each
        uint32_t fill = 0;
        bool ok = true;
        auto tokens4 = [&](int slot) {  // the tokens of four neighbouring slots; holes give a row beyond the matrix
            const int4 e = __ldg(reinterpret_cast<const int4 *>(P.entry_of + slot));
            return make_int4(e.x < 0 ? P.tokens : e.x / P.k, e.y < 0 ? P.tokens : e.y / P.k, e.z < 0 ? P.tokens : e.z / P.k,
                             e.w < 0 ? P.tokens : e.w / P.k);
        };
        for (int64_t i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
            const Tile t = tile_at(i);
            int4 rows = make_int4(0, 0, 0, 0);
            if constexpr (S::A_GATHER)
                if (lane < AR / 4) rows = tokens4(t.m0 + 4 * lane);
            for (int kb = 0; kb < t.nkb; ++kb, ++fill) {
                const uint32_t s = fill % S::STAGES, phase = (fill / S::STAGES) & 1;
                ok = waits.wait(empty + 8 * s, phase ^ 1);
                ok = __all_sync(FULL, ok);
                if (!ok || P.hold) break;
                const uint32_t a = ring_a + s * S::A_BYTES, b = ring_b + s * S::B_BYTES, bar = full + 8 * s;
                if (lane == 0) mbar_expect_tx(bar, S::STAGE);
                __syncwarp();
                const int k0 = kb * 64;
                if constexpr (S::WGRAD) {
                    const int slot = t.kb + k0;
                    if (lane < 2) tma_load_2d(a + lane * 8192, &map_a, t.m0 + lane * 64, slot, bar);
                    if (lane >= 2 && lane < 2 + BN / 64) tma_load_2d(b + (lane - 2) * 8192, &map_b, t.n0 + (lane - 2) * 64, slot, bar);
                } else {
                    if constexpr (S::A_GATHER) {
                        if (lane < AR / 4) tma_gather4(a + lane * 512, &map_a, k0, rows, bar);
                    } else {
                        if (lane == 0) tma_load_2d(a, &map_a, k0, t.m0, bar);
                    }
                    if constexpr (MODE == GATE_UP) {
                        if (lane < 2) tma_load_3d(b + lane * (S::B_BYTES / 2), &map_b, k0, t.n0, 2 * t.e + lane, bar);
                    } else if constexpr (MODE == DOWN) {
                        if (lane == 0) tma_load_3d(b, &map_b, k0, t.n0, t.e, bar);
                    } else {
                        if (lane < BN / 64) tma_load_3d(b + lane * 8192, &map_b, t.n0 + lane * 64, k0, t.e, bar);
                    }
                }
            }
            if (P.hold) break;
        }
        // every copy has landed and every product has read its stage before the block may end
        const uint32_t first = fill > S::STAGES ? fill - S::STAGES : 0;
        for (uint32_t f = first; f < fill; ++f) {
            const uint32_t s = f % S::STAGES, phase = (f / S::STAGES) & 1;
            waits.plain(full + 8 * s, phase, false);
            if (ok) waits.wait(empty + 8 * s, phase);
        }
    } else if (warp == 1) {
        // ------------------------------------------------ one thread issues the products
        if (lane == 0) {
            constexpr uint32_t type = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
            constexpr uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | ((S::A_MN ? 1u : 0u) << 15) |
                                       ((S::B_MN ? 1u : 0u) << 16) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
            constexpr uint32_t step_a = S::A_MN ? 2048 : 32, step_b = S::B_MN ? 2048 : 32;  // 16 along the contraction
            uint32_t fill = 0, it = 0;
            bool ok = true, any = false;
            for (int64_t i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
                const Tile t = tile_at(i);
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
                    const uint64_t a = smem_desc(ring_a + s * S::A_BYTES, S::A_MN), b = smem_desc(ring_b + s * S::B_BYTES, S::B_MN);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        tc_mma(d, a + q * (step_a >> 4), b + q * (step_b >> 4), idesc, (kb | q) != 0);
                    any = true;
                    tc_commit(empty + 8 * s);
                }
                if (ok) tc_commit(acc_full + 8 * buf);
            }
            if (!ok && any) {  // a wait ran out: the products already issued end before the block does
                tc_commit(drain);
                waits.plain(drain, 0, false);
            }
        }
    } else if (warp >= 4) {
        // ------------------------------------------------ epilogue: one accumulator row per thread
        const int row = tid - 128;
        const uint32_t lanes = (uint32_t)(warp - 4) << 21;  // 32 TMEM lanes per warp, lane index in the upper half
        uint32_t it = 0;
        bool ok = true;
        for (int64_t i = blockIdx.x; i < tiles; i += gridDim.x) {
            const Tile t = tile_at(i);
            const uint32_t buf = it % S::ACC, phase = (it / S::ACC) & 1;
            if (t.nkb > 0) {
                ++it;
                ok = waits.wait(acc_full + 8 * buf, phase);
                if (!__all_sync(FULL, ok)) break;
                tc_fence_after();
            }
            const uint32_t d = tmem + buf * BN + lanes;
            const bool live = (warp - 4) * 32 < (S::WGRAD ? min(128, M - t.m0) : AR);  // uniform in the warp
            if (live) {
                const bool mine = S::WGRAD ? t.m0 + row < M : row < AR;
                const int64_t slot = t.m0 + row;  // row modes
                if constexpr (MODE == GATE_UP) {
                    const int entry = mine ? __ldg(P.entry_of + slot) : -1;
                    const float w = entry >= 0 ? __ldg(P.w + entry) : 0.f;
                    T *const hw = reinterpret_cast<T *>(P.out0) + slot * P.F;
                    T *const gu = P.out1 ? reinterpret_cast<T *>(P.out1) + slot * 2 * P.F : nullptr;
#pragma unroll 1
                    for (int c = 0; c < BN / 2 && t.n0 + c < P.F; c += 16) {
                        float g[16], u[16], h[16];
                        tmem_ld16(d + c, g);
                        tmem_ld16(d + BN / 2 + c, u);
                        tmem_wait_ld(g);
                        tmem_pin(u);
#pragma unroll
                        for (int j = 0; j < 16; ++j) h[j] = entry >= 0 ? w * (g[j] * sigmoid_fast(g[j]) * u[j]) : 0.f;
                        if (mine) {
#pragma unroll
                            for (int j = 0; j < 16; j += 8) {
                                const int f = t.n0 + c + j;
                                if (f < P.F) {
                                    store8(hw + f, h + j);
                                    if (gu && entry >= 0) store8(gu + f, g + j), store8(gu + P.F + f, u + j);
                                }
                            }
                        }
                    }
                } else if constexpr (MODE == DH) {
                    const int entry = mine ? __ldg(P.entry_of + slot) : -1;
                    const float w = entry >= 0 ? __ldg(P.w + entry) : 0.f;
                    const T *const gu = reinterpret_cast<const T *>(P.in0) + slot * 2 * P.F;
                    T *const dgu = reinterpret_cast<T *>(P.out0) + slot * 2 * P.F;
                    float dot = 0.f;
#pragma unroll 1
                    for (int c = 0; c < BN && t.n0 + c < P.F; c += 16) {
                        float dh[16];
                        tmem_ld16(d + c, dh);
                        tmem_wait_ld(dh);
                        if (mine) {
#pragma unroll
                            for (int j = 0; j < 16; j += 8) {
                                const int f = t.n0 + c + j;
                                if (f < P.F) {
                                    float g[8] = {}, u[8] = {};
                                    if (entry >= 0) {  // a hole's gradients are zeros whatever the weights hold
                                        load8(gu + f, g);
                                        load8(gu + P.F + f, u);
#pragma unroll
                                        for (int v = 0; v < 8; ++v) {
                                            const float s = sigmoid_fast(g[v]), a = g[v] * s, x = dh[j + v], xw = x * w;
                                            dot += x * a * u[v];
                                            g[v] = xw * u[v] * (s + a * (1.f - s));
                                            u[v] = xw * a;
                                        }
                                    }
                                    store8(dgu + f, g);
                                    store8(dgu + P.F + f, u);
                                }
                            }
                        }
                    }
                    if (mine) P.partial[slot * nts + t.n0 / S::NSTEP] = dot;
                } else {
                    T *const out = S::WGRAD ? reinterpret_cast<T *>(P.out0) + ((int64_t)t.e * M + slot) * N
                                            : reinterpret_cast<T *>(P.out0) + slot * N;
#pragma unroll 1
                    for (int c = 0; c < BN && t.n0 + c < N; c += 16) {
                        float v[16];
                        if (t.nkb > 0) {
                            tmem_ld16(d + c, v);
                            tmem_wait_ld(v);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = 0.f;
                        }
                        if (mine) {
#pragma unroll
                            for (int j = 0; j < 16; j += 8)
                                if (t.n0 + c + j < N) store8(out + t.n0 + c + j, v + j);
                        }
                    }
                }
            }
            if (t.nkb > 0) {
                tc_fence_before();
                mbar_arrive(acc_empty + 8 * buf);
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM) : "memory");
    }
}

// Rows of a matrix in slot order, a warp per slot; holes become zeros.  Bound by memory: it writes 2 D bytes a slot and reads
// every token's row once from HBM, k - 1 times from L2.
template <typename T>
__global__ void __launch_bounds__(256) experts_gather_kernel(const T *x, int64_t stride, const int32_t *entry_of, const int32_t *used, T *out,
                                                             int k, int D)
{
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t slot = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (slot >= __ldg(used)) return;
    const int entry = __ldg(entry_of + slot);
    const uint4 *const from = reinterpret_cast<const uint4 *>(x + (int64_t)(entry < 0 ? 0 : entry / k) * stride);
    uint4 *const to = reinterpret_cast<uint4 *>(out + slot * D);
    const int n = D / 8;
    for (int i = lane; i < n; i += 256) {
        uint4 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (entry >= 0 && i + 32 * j < n) ? __ldg(from + i + 32 * j) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + 32 * j < n) to[i + 32 * j] = v[j];
    }
}

// y_t = sum over the token's slots, in the order of its choices, eight columns per thread; dropped entries (-1) add nothing.
// With `partial` also grad_w of the token's entries: the column tiles' sums in order.
template <typename T>
__global__ void __launch_bounds__(256) experts_combine_kernel(const T *slots, const int32_t *slot_of, T *out, int64_t out_stride,
                                                              const float *partial, T *grad_w, int64_t tokens, int k, int D, int nts)
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
        for (int j = 0; j < 8; ++j) s[j] = j0 + j < k ? __ldg(at + j0 + j) : -1;
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = s[j] >= 0 ? __ldg(reinterpret_cast<const uint4 *>(slots + (int64_t)s[j] * D + 8 * c)) : Io<T>::zero();
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
            const int s = __ldg(at + j);
            float g = 0.f;
            if (s >= 0)
                for (int n = 0; n < nts; ++n) g += partial[(int64_t)s * nts + n];
            Io<T>::store1(grad_w + t * k + j, g);
        }
}

}  // namespace lapsum
