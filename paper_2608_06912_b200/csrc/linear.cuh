// A dense product with its epilogue, and its gradients:
//
//   forward   P = x W^T + bias,  y = act(P) + residual      x: rows x k, W: n x k, y: rows x n
//   backward  dP = dy act'(P),   dx = dP W,   dW = dP^T x,   dbias = sum over the rows of dP
//
// Every product is computed as D[lane][column]: the dimension that is contiguous in the result runs over the 128 lanes of the
// accumulator in TMEM, the result's rows over its columns:
//
//   forward   lanes n,  columns rows,  contraction k        A = W (K-major),    B = x (K-major)
//   dx        lanes k,  columns rows,  contraction n        A = W (MN-major),   B = dP (K-major)
//   dW        lanes k,  columns n,     contraction rows     A = x (MN-major),   B = dP (MN-major)
//
// so a few tokens are a narrow column tile beside full 128-row tiles of weights, and in the epilogue the 32 lanes of a warp hold
// 32 neighbouring values of one row of the result: loads and stores of it are contiguous whatever n, the strides and the alignment,
// and a bias is one value per thread.
//
// Measured in bf16 on two boards, operands not in L2 (a library's product of the same shape beside it): 16384 x 8192 x 2048 forward without an epilogue 373 - 393 us,
// 1.47 PFLOP/s (344 - 358), with silu and P kept in fp32 (805 MB of results) 416 - 453; dx 352 - 373 (348), dW 399 - 455 (341), all at the power limit; dW with fp32 digits
// 990 - 1110 for twice the products.  Logits of 48 rows, 128000 x 2048, 106 us, 5.1 TB/s of weights (107); the router 65536 x 128 x 2048 65 - 68 us,
// 4.5 TB/s (70), 256 tiles on 148 SMs, so that 40 of them have one and the others two; a prompt of 1021 rows, 2048 x 5632, 33 us (26): 32 large tiles, their contraction
// shared by two pairs each, so a join; one row of 2048 x 1024 7 - 9 us, the host's call (2.6 in a graph).
#pragma once
#include <climits>
#include <type_traits>

#include "common.cuh"
#include "tensor_core.cuh"

namespace lapsum {

struct LinearMaps {
    CUtensorMap a, b, b_low;  // b_low: what the rounding of b to 16 bits left, where the contraction runs over both
};

struct LinearArgs {
    void *out;             // fp32 (out_f32) or T, rows out_stride elements apart
    const void *residual;  // like out, or null
    const void *bias;      // fp32 (bias_f32) or T, or null
    void *pre;             // fp32 (pre_f32) or T, rows pre_stride elements apart, or null
    int64_t out_stride, residual_stride, pre_stride;
    int L, C, K;           // lanes, columns, contraction
    int lane_tiles, col_tiles;
    int act, out_f32, bias_f32, pre_f32;
    int twice;             // the contraction runs over (a, b), then over (a, b_low)
    int round;             // WIDE: steps of 64 that one accumulator takes
    int split;             // blocks of a cluster that share the contraction of one tile
    int parts;             // of the contraction, each a block's of its own, whose results lie one behind the other (fp32, C rows each)
    const uint32_t *largest;  // fp16 gradients: the largest |dP| of every column of the result, by which its operand was scaled (grad_scale), or null
    int hold;              // test hook: the producer brings nothing, so the waits run out
    uint32_t *status;
    unsigned long long wait_ns;
};

// ---------------------------------------------------------------- activations ----
// 1 / (1 + e^-x) to about 3 ulp: the product with log2(e) split in two, the hardware's 2^x and reciprocal.  (Subnormal e^-x are 0 beside the 1.)
__device__ __forceinline__ float exp_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(fmaf(x, 1.44269502f, x * 1.92596299e-8f)));
    return y;
}
__device__ __forceinline__ float sigmoid_of(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(1.f + exp_of(-x)));
    return y;
}
// The normal distribution's Phi(x), and e^(-x^2 / 2): Phi(-|x|) = t P(t) e^(-x^2 / 2), t = 1 / (1 + 0.35 |x|), with a polynomial fitted for the least relative error
// over 0 <= |x| <= 14.5 (C. L. Lawson's reweighted least squares, 1961): 3.2e-8, in fp32 some 3 ulp, and x^2 ulp to the left from the exponential's argument.  0.5 (1 + erf)
// leaves nothing of the value from x = -6 on.  The forward of 16384 x 8192 x 2048 takes 449 us with this as with erff, with erfcf 518.
__device__ __forceinline__ float normal_below(float x, float &e)
{
    float t;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(0.35f, fabsf(x), 1.f)));
    e = exp_of(-0.5f * x * x);
    float p = fmaf(-0.0291580297f, t, 0.144031614f);
    p = fmaf(p, t, -0.255840421f);
    p = fmaf(p, t, 0.159321293f);
    p = fmaf(p, t, -0.0232134108f);
    p = fmaf(p, t, 0.105552934f);
    p = fmaf(p, t, 0.119821183f);
    p = fmaf(p, t, 0.139863521f);
    p = fmaf(p, t, 0.139621302f);
    p = p * t * e;
    return x < 0.f ? p : 1.f - p;
}
constexpr float GELU_A = 0.797884561f, GELU_B = 0.044715f;  // sqrt(2 / pi), the tanh form's cubic term

template <int ACT>
__device__ __forceinline__ float activate(float x)
{
    if constexpr (ACT == LAPSUM_ACT_RELU) return x > 0.f ? x : x == x ? 0.f : x;
    else if constexpr (ACT == LAPSUM_ACT_SILU) return x * sigmoid_of(x);
    else if constexpr (ACT == LAPSUM_ACT_GELU) {
        float e;
        return x * normal_below(x, e);
    } else if constexpr (ACT == LAPSUM_ACT_GELU_TANH)
        return x * sigmoid_of(2.f * GELU_A * x * fmaf(GELU_B * x, x, 1.f));  // (1 + tanh u) / 2 = sigmoid(2 u)
    else return x;
}
template <int ACT>
struct Act {
    static constexpr int value = ACT;
};
template <typename F>
__device__ __forceinline__ void by_activation(int act, F f)
{
    switch (act) {
    case LAPSUM_ACT_RELU: f(Act<LAPSUM_ACT_RELU>()); break;
    case LAPSUM_ACT_SILU: f(Act<LAPSUM_ACT_SILU>()); break;
    case LAPSUM_ACT_GELU: f(Act<LAPSUM_ACT_GELU>()); break;
    case LAPSUM_ACT_GELU_TANH: f(Act<LAPSUM_ACT_GELU_TANH>()); break;
    default: f(Act<LAPSUM_ACT_NONE>()); break;
    }
}
// The slope at a pre-activation that was kept in 16 bits; beyond +-1000 every activation's slope is its limit (an infinity kept by
// fp16 included, where the formulas would give infinity times 0).
template <int ACT>
__device__ __forceinline__ float slope_of(float x)
{
    x = x > 1000.f ? 1000.f : x < -1000.f ? -1000.f : x;  // NaN stays
    if constexpr (ACT == LAPSUM_ACT_RELU) {
        return x > 0.f ? 1.f : x == x ? 0.f : x;
    } else if constexpr (ACT == LAPSUM_ACT_SILU) {
        const float s = sigmoid_of(x);
        return s * fmaf(x, 1.f - s, 1.f);
    } else if constexpr (ACT == LAPSUM_ACT_GELU) {
        float e;
        const float below = normal_below(x, e);
        return fmaf(0.398942280f * x, e, below);
    } else if constexpr (ACT == LAPSUM_ACT_GELU_TANH) {
        const float s = sigmoid_of(2.f * GELU_A * x * fmaf(GELU_B * x, x, 1.f));
        return fmaf(2.f * GELU_A * x * s, (1.f - s) * fmaf(3.f * GELU_B * x, x, 1.f), s);
    } else {
        return 1.f;
    }
}

template <typename T>
__device__ __forceinline__ float load_either(const void *p, int64_t i, bool f32)
{
    return f32 ? ld(static_cast<const float *>(p) + i) : Io<T>::from_storage(ld(static_cast<const T *>(p) + i));
}
template <typename T>
__device__ __forceinline__ void store_either(void *p, int64_t i, bool f32, float v)
{
    if (f32) static_cast<float *>(p)[i] = v;
    else Io<T>::store1(static_cast<T *>(p) + i, v);
}

// fp16 ends at 6e-8 and at 65504, so there dP takes a power of two per row (for dx) or column (for dW) that brings the largest finite one of it, whose
// bits these are, to between 2^14 and 2^15; the products' epilogues take it back.  Both are exact, and +-126 at most, so that neither is subnormal.
__device__ __forceinline__ uint32_t grad_scale_exponent(uint32_t largest) { return min(268 - (largest >> 23), 253u); }
__device__ __forceinline__ float grad_scale(uint32_t largest) { return __uint_as_float(grad_scale_exponent(largest) << 23); }
__device__ __forceinline__ float grad_unscale(uint32_t largest) { return __uint_as_float((254 - grad_scale_exponent(largest)) << 23); }

// n of N values, `stride` apart
template <typename S, int N>
__device__ __forceinline__ void load_rows(const void *base, int64_t at, int64_t stride, int n, float (&v)[N])
{
    const S *p = static_cast<const S *>(base) + at;
    S q[N];
    if (n >= N) {
#pragma unroll
        for (int j = 0; j < N; ++j, p += stride) q[j] = ld(p);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = Io<S>::from_storage(q[j]);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j, p += stride) v[j] = j < n ? Io<S>::from_storage(ld(p)) : 0.f;
    }
}
template <typename S, int N>
__device__ __forceinline__ void store_rows(void *base, int64_t at, int64_t stride, int n, const float (&v)[N])
{
    S *p = static_cast<S *>(base) + at;
    if (n >= N) {
#pragma unroll
        for (int j = 0; j < N; ++j, p += stride) Io<S>::store1(p, v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j, p += stride)
            if (j < n) Io<S>::store1(p, v[j]);
    }
}
// The same for 16-bit values of 32 neighbouring lanes: two lanes exchange every other value, so that each stores two neighbouring ones of every other row, with
// half the instructions: products of 16384 x 8192 x 2048 394 -> 373, 376 -> 352, 423 -> 399 us.
template <typename T, int N>
__device__ __forceinline__ void store_row_pairs(void *base, int64_t at, int64_t stride, int n, const float (&v)[N])
{
    const bool odd = threadIdx.x & 1;
    T *p = static_cast<T *>(base) + at + (odd ? stride - 1 : 0);
#pragma unroll
    for (int j = 0; j + 1 < N; j += 2, p += 2 * stride) {
        const float other = __shfl_xor_sync(FULL, odd ? v[j] : v[j + 1], 1);
        T two[2];
        Io<T>::store1(two, odd ? other : v[j]);
        Io<T>::store1(two + 1, odd ? v[j + 1] : other);
        uint32_t q;
        memcpy(&q, two, 4);
        if (j + odd < n) *reinterpret_cast<uint32_t *>(p) = q;
    }
}
// N values of lane l, rows r0 .. : bias, pre-activation, activation, residual, result
template <typename T, int N>
__device__ __forceinline__ void linear_finish(const LinearArgs &P, float (&v)[N], int l, int r0, float bias, int64_t shift = 0,
                                              bool pairs = false)  // pairs: 32 neighbouring lanes, results at multiples of 4 bytes
{
    const int n = P.C - r0;
    float res[N];
    if (P.residual != nullptr) {
        const int64_t at = (int64_t)r0 * P.residual_stride + l;
        if (P.out_f32) load_rows<float>(P.residual, at, P.residual_stride, n, res);
        else load_rows<T>(P.residual, at, P.residual_stride, n, res);
    }
    if constexpr (std::is_same<T, __half>::value) {
        if (P.largest != nullptr) {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] *= j < n ? grad_unscale(ld(P.largest + r0 + j)) : 0.f;
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] += bias;
    if (P.pre != nullptr) {
        const int64_t at = (int64_t)r0 * P.pre_stride + l;
        if (P.pre_f32) store_rows<float>(P.pre, at, P.pre_stride, n, v);
        else store_rows<T>(P.pre, at, P.pre_stride, n, v);
    }
    if (P.act != LAPSUM_ACT_NONE)
        by_activation(P.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = activate<decltype(act)::value>(v[j]);
        });
    if (P.residual != nullptr) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] += res[j];
    }
    const int64_t at = shift + (int64_t)r0 * P.out_stride + l;
    if (P.out_f32) store_rows<float>(P.out, at, P.out_stride, n, v);
    else if (pairs) store_row_pairs<T>(P.out, at, P.out_stride, n, v);
    else store_rows<T>(P.out, at, P.out_stride, n, v);
}

// ---------------------------------------------------------------- the kernel ----
// Warp 0 brings operand tiles of 64 along the contraction into a ring of stages by TMA, one thread of warp 1 issues tcgen05.mma
// into one of two accumulators in TMEM, warps 4 to 11 (two sets of four; a set reads the 128 lanes) finish the previous tile.
//   PAIR   a cluster of two blocks works on one 256 x 256 tile (cta_group::2): each block brings 128 rows of A and half of B, 64 bytes per
//          clock of tensor work instead of the 96 that a 128 x 256 tile of one block needs.
//   parts  the same without a cluster: blocks of their own leave fp32 results one behind the other, for linear_parts_kernel to add.
//   WIDE   the tensor core's own additions truncate, all towards zero: 2e-6 of the sum at K = 2048 and 2e-5 at 16384 where signs are mixed, five times that where all terms
//          have one sign.  A 16-bit result of a short contraction does not show it.  For an fp32 result, or a long contraction, an accumulator takes some steps (512 of the
//          contraction, 2048), and the epilogue adds the rounds' sums in fp32 registers, rounded to nearest, while the next round is computed in the other accumulator:
//          5e-7 for fp32, with one sign 3e-6.
//   split  a cluster of `split` blocks, or pairs, shares the contraction of one tile, for shapes with few tiles: each leaves its sums in its shared
//          memory, and after a cluster barrier adds its share of the columns over the blocks, in their order.
template <int BN, bool PAIR_>
struct LinearShape {
    static constexpr bool PAIR = PAIR_;
    static constexpr int COLS = PAIR ? BN / 2 : BN;  // columns of B that one block brings
    static constexpr int A_BYTES = 128 * 128, B_BYTES = COLS * 128, STAGE = A_BYTES + B_BYTES;
    static constexpr int FIT = 229376 / STAGE, STAGES = FIT < 12 ? FIT : 12;
    static constexpr int ACC = 2, TMEM = ACC * BN;
    static constexpr int CHUNKS = (BN + 31) / 32;  // runs of 16 columns of one set of epilogue warps
    static constexpr int THREADS = 384;
    static constexpr int SMEM = STAGES * STAGE + 1024 + 512;
    static_assert(STAGES >= 2 && TMEM >= 32 && TMEM <= 512 && BN * 512 <= STAGES * STAGE, "tile does not fit");
};

template <bool A_MN, bool B_MN, int BN, bool PAIR, bool WIDE, typename T>
__global__ void __launch_bounds__(384, 1) linear_kernel(const __grid_constant__ LinearMaps maps, const LinearArgs P)
{
    using S = LinearShape<BN, PAIR>;
    static_assert(!B_MN || S::COLS % 64 == 0, "MN-major columns come in runs of 64");
    extern __shared__ uint8_t raw[];
    const uint32_t ring_a = (smem_u32(raw) + 1023) & ~1023u, ring_b = ring_a + S::STAGES * S::A_BYTES;
    const uint32_t full = ring_b + S::STAGES * S::B_BYTES, empty = full + 8 * S::STAGES, acc_full = empty + 8 * S::STAGES,
                   acc_empty = acc_full + 8 * S::ACC, drain = acc_empty + 8 * S::ACC;
    __shared__ uint32_t tmem_at;
    __shared__ int abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool split = P.split > 1, spread = !PAIR && P.parts > 1;
    // of a pair: its first block's rank, which of the two this is; of a shared contraction: which part of it
    const uint32_t rank = PAIR || split ? cluster_rank() : 0, first = rank & ~1u, half = PAIR ? rank & 1 : 0, part = PAIR ? rank >> 1 : rank;

    if (tid == 0) {
        abort_flag = 0;
        for (int s = 0; s < S::STAGES; ++s) mbar_init(full + 8 * s, 1), mbar_init(empty + 8 * s, 1);
        for (int a = 0; a < S::ACC; ++a) mbar_init(acc_full + 8 * a, 1), mbar_init(acc_empty + 8 * a, PAIR ? 16 : 8);
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (tid == 96) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b) : "memory");
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
    pdl_wait();

    constexpr bool LOW = WIDE && A_MN && B_MN;  // dW alone has a b_low
    const int once = (P.K + 63) / 64, steps = LOW && P.twice ? 2 * once : once;
    const int ways = spread ? P.parts : P.split, share = (steps + ways - 1) / ways;
    const int64_t tiles = (int64_t)P.lane_tiles * P.col_tiles;
    const int64_t group = (PAIR ? 2 : 1) * P.split, tile0 = spread ? blockIdx.x % tiles : blockIdx.x / group, tile_step = spread ? tiles : gridDim.x / group;
    const int mine = spread ? (int)(blockIdx.x / tiles) : (int)part;  // which part of the contraction
    const int64_t shift = spread ? (int64_t)mine * P.C * P.out_stride : 0;
    const int k_first = split || spread ? min(mine * share, steps) : 0, nkb = min(share, steps - k_first);
    // An accumulator takes `round` steps, and never steps of both b and b_low: those of b_low begin at `turn`.
    const int round = WIDE ? P.round : nkb, turn = LOW && P.twice ? once - k_first : INT_MAX;
    auto round_end = [&](int k0) { return min(k0 < turn ? min(k0 + round, turn) : k0 + round, nkb); };
    // Tiles in groups of eight column tiles, lane tiles outside: what the SMs work on at one time shares its operands in L2.
    struct Tile {
        int l0, c0;
    };
    auto tile_at = [&](int64_t i) {
        const int64_t per = (int64_t)8 * P.lane_tiles, g = i / per;
        const int rest = (int)(i - g * per), wide = (int)min((int64_t)8, P.col_tiles - 8 * g);
        const int lt = rest / wide, ct = (int)(8 * g) + rest - lt * wide;
        return Tile{(PAIR ? 256 : 128) * lt + 128 * (int)half, BN * ct};
    };
    Waits waits{&abort_flag, P.status, P.wait_ns, LAPSUM_ST_LINEAR_TIMEOUT};

    if (warp == 0) {
        // ------------------------------------------------ producer
        uint32_t fill = 0;
        bool ok = true;
        auto load = [&](uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
            if constexpr (PAIR) tma_pair_2d(dst, map, x, y, bar);
            else tma_load_2d(dst, map, x, y, bar);
        };
        for (int64_t i = tile0; i < tiles && ok; i += tile_step) {
            const Tile t = tile_at(i);
            const int c0 = t.c0 + (int)half * S::COLS;
            for (int kb = 0; kb < nkb; ++kb, ++fill) {
                const uint32_t s = fill % S::STAGES, phase = (fill / S::STAGES) & 1;
                ok = waits.wait(empty + 8 * s, phase ^ 1);
                ok = __all_sync(FULL, ok);
                if (!ok || P.hold) break;
                const uint32_t bar = PAIR ? in_block(full + 8 * s, first) : full + 8 * s;  // a pair's first block counts for both
                if (lane == 0 && half == 0) mbar_expect_tx(full + 8 * s, PAIR ? 2 * S::STAGE : S::STAGE);
                __syncwarp();
                const bool low = k_first + kb >= once;
                const int k0 = (k_first + kb - (low ? once : 0)) * 64;
                const CUtensorMap *const map_b = low ? &maps.b_low : &maps.b;
                const uint32_t a = ring_a + s * S::A_BYTES, b = ring_b + s * S::B_BYTES;
                if constexpr (A_MN) {
                    if (lane < 2) load(a + lane * 8192, &maps.a, t.l0 + lane * 64, k0, bar);
                } else {
                    if (lane == 0) load(a, &maps.a, k0, t.l0, bar);
                }
                if constexpr (B_MN) {
                    if (lane >= 2 && lane < 2 + S::COLS / 64) load(b + (lane - 2) * 8192, map_b, c0 + (lane - 2) * 64, k0, bar);
                } else {
                    if (lane == 2) load(b, map_b, k0, c0, bar);
                }
            }
            if (P.hold) break;
        }
        // every copy has landed and every product has read its stage before the block may end
        const uint32_t first = fill > S::STAGES ? fill - S::STAGES : 0;
        for (uint32_t f = first; f < fill; ++f) {
            const uint32_t s = f % S::STAGES, phase = (f / S::STAGES) & 1;
            if (half == 0) waits.plain(full + 8 * s, phase, false);
            if (ok) waits.wait(empty + 8 * s, phase);
        }
    } else if (warp == 1) {
        // ------------------------------------------------ one thread issues the products (a pair's: one of its first block)
        if (lane == 0 && half == 0) {
            constexpr uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
            constexpr uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
                                   ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((PAIR ? 256 : 128) >> 4) << 24);
            constexpr uint32_t step_a = A_MN ? 2048 : 32, step_b = B_MN ? 2048 : 32;  // 16 along the contraction
            uint32_t fill = 0, it = 0;
            bool ok = true, any = false;
            for (int64_t i = tile0; i < tiles && ok; i += tile_step)
                for (int k0 = 0, k1; k0 < nkb && ok; k0 = k1, ++it) {
                    k1 = round_end(k0);
                    const uint32_t buf = it % S::ACC, phase = (it / S::ACC) & 1;
                    ok = waits.wait(acc_empty + 8 * buf, phase ^ 1);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t d = tmem + buf * BN;
                    for (int kb = k0; kb < k1; ++kb, ++fill) {
                        const uint32_t s = fill % S::STAGES;
                        ok = waits.wait(full + 8 * s, (fill / S::STAGES) & 1);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t a = smem_desc(ring_a + s * S::A_BYTES, A_MN), b = smem_desc(ring_b + s * S::B_BYTES, B_MN);
#pragma unroll
                        for (int q = 0; q < 4; ++q) tc_mma<PAIR>(d, a + q * (step_a >> 4), b + q * (step_b >> 4), idesc, (kb - k0) | q ? 1 : 0);
                        any = true;
                        tc_commit<PAIR>(empty + 8 * s, first);
                    }
                    if (ok) tc_commit<PAIR>(acc_full + 8 * buf, first);
                }
            if (!ok && any) {  // a wait ran out: the products already issued end before the block does
                tc_commit<PAIR>(drain, first);
                waits.plain(drain, 0, false);
            }
        }
    } else if (warp >= 4) {
        // ------------------------------------------------ epilogue: a lane of the accumulator per thread, 16 columns at a time
        const int ew = warp & 3, set = (warp - 4) >> 2;
        const uint32_t lanes = (uint32_t)ew << 21;  // 32 TMEM lanes per warp, lane index in the upper half
        uint32_t it = 0;
        bool ok = true;
        for (int64_t i = tile0; i < tiles && ok; i += tile_step) {
            const Tile t = tile_at(i);
            const int l = t.l0 + 32 * ew + lane;
            float bias = 0.f;
            if (P.bias != nullptr && l < P.L && !split) bias = load_either<T>(P.bias, l, P.bias_f32);
            // the residual's tile comes into L2 while the products run: waiting for it afterwards, 16 columns at a time, took as long as they did
            if (P.residual != nullptr && l < P.L)
                for (int c = lane; c < BN / 2; c += 32) {
                    const int row = t.c0 + c / 16 * 32 + 16 * set + c % 16;
                    const int64_t at = (int64_t)row * P.residual_stride + t.l0 + 32 * ew;
                    if (row < P.C) asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint8_t *>(P.residual) + at * (P.out_f32 ? 4 : 2)) : "memory");
                }
            const bool pairs = !WIDE && !P.out_f32 && t.l0 + 32 * ew + 32 <= P.L && P.out_stride % 2 == 0 && (reinterpret_cast<uintptr_t>(P.out) & 3) == 0;
            const auto finish = [&](float (&v)[16], int c0) {  // columns c0 .. of the tile
                if (split) {
                    // the ring is free: all products of this block's only tile have ended.  [column][lane]
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(ring_a + 4 * ((c0 + j) * 128 + 32 * ew + lane)), "f"(v[j]) : "memory");
                } else if (pairs || l < P.L) {
                    linear_finish<T>(P, v, l, t.c0 + c0, bias, shift, pairs);
                }
            };
            float sum[WIDE ? S::CHUNKS : 1][16];
            if constexpr (WIDE) {
#pragma unroll
                for (int c = 0; c < S::CHUNKS; ++c)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[c][j] = 0.f;
            }
            for (int k0 = 0; k0 < nkb; k0 = round_end(k0), ++it) {
                const uint32_t buf = it % S::ACC, phase = (it / S::ACC) & 1;
                ok = waits.wait(acc_full + 8 * buf, phase);
                ok = __all_sync(FULL, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + buf * BN + lanes + 16 * set;
                if constexpr (WIDE) {
#pragma unroll
                    for (int c = 0; c < S::CHUNKS; ++c) {
                        if (16 * set + 32 * c >= BN) continue;
                        float v[16];
                        tmem_ld16(d + 32 * c, v);
                        tmem_wait_ld(v);
                        if (LOW && k0 >= turn) {
                            // an infinity or NaN of a's has reached the sums of b: beside the remainders, zeros or of the other sign, it would only make a NaN
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = fabsf(v[j]) <= 3.402823466e38f ? v[j] : 0.f;
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[c][j] += v[j];
                    }
                } else {
#pragma unroll 1
                    for (int c = 0; 16 * set + c < BN && t.c0 + 16 * set + c < P.C; c += 32) {
                        tmem_ld16(d + c, sum[0]);
                        tmem_wait_ld(sum[0]);
                        finish(sum[0], 16 * set + c);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(PAIR ? in_block(acc_empty + 8 * buf, first) : acc_empty + 8 * buf);
            }
            if (!ok) break;
            if constexpr (WIDE) {
                // a loop that is not unrolled, over sums that move up: unrolled, it is 80 KB of code, and instruction fetches bound the kernel
#pragma unroll 1
                for (int c = 16 * set; c < BN && t.c0 + c < P.C; c += 32) {
                    finish(sum[0], c);
#pragma unroll
                    for (int i = 0; i + 1 < S::CHUNKS; ++i)
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[i][j] = sum[i + 1][j];
                }
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (PAIR || split) cluster_barrier();
    if (split) {
        const Tile t = tile_at(tile0);
        const int l = tid & 127, per = BN / P.split;  // columns of one block: four or more, for BN >= 16 and up to four blocks
        const int c1 = ((int)part + 1) * per;
        if (t.l0 + l < P.L) {
            const float bias = P.bias != nullptr ? load_either<T>(P.bias, t.l0 + l, P.bias_f32) : 0.f;
#pragma unroll 1
            for (int c = (int)part * per + 8 * (tid >> 7); c < c1 && t.c0 + c < P.C; c += 24) {
                float v[8] = {};
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    if (s < P.split) {
                        const uint32_t from = in_block(ring_a + 4 * (c * 128 + l), PAIR ? 2 * s + half : s);
                        float sums[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(sums[j]) : "r"(from + 512 * j) : "memory");
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] += sums[j];
                    }
                if (per >= 8) {
                    linear_finish<T>(P, v, t.l0 + l, t.c0 + c, bias);
                } else {
                    LinearArgs Q = P;  // the next columns are another block's
                    Q.C = min(P.C, t.c0 + c1);
                    linear_finish<T>(Q, v, t.l0 + l, t.c0 + c, bias);
                }
            }
        }
        __syncwarp();
        cluster_barrier();  // nobody leaves while others read
    }
    if (warp == 2) {
        tc_fence_after();
        if constexpr (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM) : "memory");
    }
}

// The parts' results added in order: a long contraction for few tiles (the gradients of a router's weights) that clusters do not spread over the SMs.
template <typename T>
__global__ void __launch_bounds__(256) linear_parts_kernel(const float *partial, int parts, int C, int L, void *out, int64_t out_stride, int out_f32,
                                                           const uint32_t *largest)
{
    pdl_wait();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)C * L;
    if (i >= n) return;
    float s = 0.f;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) s += ld(partial + p * n + i);
    const int64_t c = i / L;
    if (largest != nullptr) s *= grad_unscale(ld(largest + c));
    store_either<T>(out, c * out_stride + i - c * L, out_f32, s);
}

// ------------------------------------------------------------- a few rows ----
// One to four rows: a stream of weights, without the tensor core.  A warp has two features, four loads of each at once.
template <typename T, int R>
__global__ void __launch_bounds__(256) linear_few_kernel(const T *x, int64_t x_stride, const T *w, const LinearArgs P)
{
    pdl_wait();
    const int lane = threadIdx.x & 31, f0 = 2 * (blockIdx.x * 8 + (threadIdx.x >> 5));
    if (f0 >= P.L) return;
    const T *const w0 = w + (int64_t)f0 * P.K, *const w1 = f0 + 1 < P.L ? w0 + P.K : w0;
    float sum[2][R] = {};
    for (int c = 8 * lane; c < P.K; c += 1024) {
        uint4 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = c + 256 * i < P.K;
            a[i] = in ? __ldcs(reinterpret_cast<const uint4 *>(w0 + c + 256 * i)) : Io<T>::zero();
            b[i] = in ? __ldcs(reinterpret_cast<const uint4 *>(w1 + c + 256 * i)) : Io<T>::zero();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + 256 * i < P.K) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint4 v = ld(reinterpret_cast<const uint4 *>(x + r * x_stride + c + 256 * i));
                    sum[0][r] = dot8<T>(a[i], v, sum[0][r]);
                    sum[1][r] = dot8<T>(b[i], v, sum[1][r]);
                }
            }
    }
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int r = 0; r < R; ++r) sum[f][r] = warp_total(sum[f][r]);
    // lane 2 r + f finishes row r of feature f0 + f
    float mine[1] = {0.f};
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (lane == 2 * r + f) mine[0] = sum[f][r];
    const int l = f0 + (lane & 1), r = lane >> 1;
    if (r < R && l < P.L) {
        const float bias = P.bias != nullptr ? load_either<T>(P.bias, l, P.bias_f32) : 0.f;
        linear_finish<T>(P, mine, l, r, bias);
    }
}

// ---------------------------------------------------------- dP and its column sums ----
// dP = dy act'(P) in 16 bits, the operand of both products, and the sums over a block's rows of the values before that rounding, which linear_bias_kernel adds in order.  A warp has 256 columns, eight per lane, and every eighth row of the block.
// One rounding of dP is of the size of a 16-bit result's own.  Where grad_w is fp32 it would be the largest error by far (2^-9 against
// 2^-20), so there what the rounding left is kept in 16 bits as well, and the contraction of dW runs over both: twice the products for
// gradients with the digits of an fp32 sum (3e-6).
// fp16's range would cut small dP off and make large ones infinite, so there dP is written scaled, by rows for dx and by columns for dW (a factor has to stay the
// same along the contraction), and linear_largest_kernel finds the largest of each first.  Within a row or column the two 16-bit parts reach 2^-40 of the largest.
// What that costs, us of the backward without / with it: 777 x 1003 x 520 with gelu 27 / 32; 16384 x 8192 x 2048 with silu 1121 / 1346 (another pass over dy and P),
// with an fp32 grad_w 1563 / 1973 (two: dx's operand takes the room of dW's after its product).
// Rows of a block: 64, or as few as 16 while there are no 128 blocks of rows.
inline int64_t grad_blocks_most(int64_t rows)  // never less for more rows, for workspaces
{
    const int64_t few = (rows + 15) / 16, many = (rows + 63) / 64;
    return few < 128 ? few : many < 128 ? 128 : many;
}
inline int grad_block_rows(int64_t rows) { return rows <= 128 * 16 ? 16 : rows <= 128 * 32 ? 32 : 64; }
struct LinearGradArgs {
    const void *grad_y;  // fp32 (y_f32) or T
    const void *pre;     // fp32 (pre_f32) or T, null without an activation
    void *dp;            // T, null where grad_y itself serves; scaled by columns where col_largest is given
    void *dp_low;        // T, dP less its rounding, null where grad_w is 16-bit or dP a copy of grad_y
    void *dp_rows;       // T, dP scaled by rows, or null
    uint32_t *row_largest, *col_largest;  // bits of the largest finite |dP| of every row, of every column; either may be null
    float *partial;      // [blocks of rows][n], null without a bias
    int64_t y_stride, pre_stride, dp_stride, rows;
    int n, y_f32, pre_f32, block_rows;
};
__device__ __forceinline__ void load8f(const float *p, float (&x)[8])
{
    const float4 a = ld(reinterpret_cast<const float4 *>(p)), b = ld(reinterpret_cast<const float4 *>(p) + 1);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
// A lane's eight columns of a row, from c on: side by side (VEC), or 32 apart, so that single values are read side by side as well
template <typename T, int ACT, bool VEC>
__device__ __forceinline__ void load_dp(const LinearGradArgs &P, int64_t r, int c, float (&g)[8])
{
    float p[8];
    if (VEC) {
        if (P.y_f32) load8f(static_cast<const float *>(P.grad_y) + r * P.y_stride + c, g);
        else Io<T>::unpack(ld(reinterpret_cast<const uint4 *>(static_cast<const T *>(P.grad_y) + r * P.y_stride + c)), g);
        if constexpr (ACT != LAPSUM_ACT_NONE) {
            if (P.pre_f32) load8f(static_cast<const float *>(P.pre) + r * P.pre_stride + c, p);
            else Io<T>::unpack(ld(reinterpret_cast<const uint4 *>(static_cast<const T *>(P.pre) + r * P.pre_stride + c)), p);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            g[i] = c + 32 * i < P.n ? load_either<T>(P.grad_y, r * P.y_stride + c + 32 * i, P.y_f32) : 0.f;
            if constexpr (ACT != LAPSUM_ACT_NONE) p[i] = c + 32 * i < P.n ? load_either<T>(P.pre, r * P.pre_stride + c + 32 * i, P.pre_f32) : 0.f;
        }
    }
    if constexpr (ACT != LAPSUM_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] *= slope_of<ACT>(p[i]);
    }
}
// The same columns of a row of `to`
template <typename T, bool VEC>
__device__ __forceinline__ void store_dp(const LinearGradArgs &P, void *to, int64_t r, int c, const float (&v)[8])
{
    T *const at = static_cast<T *>(to) + r * P.dp_stride + c;
    if (VEC) {
        *reinterpret_cast<uint4 *>(at) = Io<T>::pack(v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + 32 * i < P.n) Io<T>::store1(at + 32 * i, v[i]);
    }
}
template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(256, 2) linear_grad_kernel(const LinearGradArgs P)
{
    pdl_wait();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ float part[8][256];
    constexpr int STEP = VEC ? 1 : 32;
    constexpr bool SCALED = std::is_same<T, __half>::value;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = (int)blockIdx.y * 256 + (VEC ? 8 * lane : lane);
    const int64_t row0 = (int64_t)blockIdx.x * P.block_rows, row1 = min(P.rows, row0 + P.block_rows);
    float sum[8] = {};
    if (c < P.n) {
        float by_col[SCALED ? 8 : 1];
        if constexpr (SCALED) {
#pragma unroll
            for (int i = 0; i < 8; ++i) by_col[i] = P.col_largest != nullptr && c + STEP * i < P.n ? grad_scale(ld(P.col_largest + c + STEP * i)) : 1.f;
        }
        // two rows at a time: stores of one would hold up the next one's loads
        for (int64_t r0 = row0 + warp; r0 < row1; r0 += 16) {
            float both[2][8], by_row[2] = {1.f, 1.f};
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int64_t r = min(r0 + 8 * q, row1 - 1);
                load_dp<T, ACT, VEC>(P, r, c, both[q]);
                if constexpr (SCALED) by_row[q] = P.dp_rows != nullptr ? grad_scale(ld(P.row_largest + r)) : 1.f;
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int64_t r = r0 + 8 * q;
                if (r >= row1) break;
                float(&g)[8] = both[q];
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += g[i];
                if constexpr (SCALED) {
                    if (P.dp_rows != nullptr) {
                        float h[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) h[i] = g[i] * by_row[q];
                        store_dp<T, VEC>(P, P.dp_rows, r, c, h);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] *= by_col[i];
                }
                if (P.dp != nullptr) {
                    store_dp<T, VEC>(P, P.dp, r, c, g);
                    if (P.dp_low != nullptr) {
                        float h[8];
                        Io<T>::unpack(Io<T>::pack(g), h);
#pragma unroll
                        for (int i = 0; i < 8; ++i) h[i] = isfinite(h[i]) ? g[i] - h[i] : 0.f;  // an infinity has no remainder
                        store_dp<T, VEC>(P, P.dp_low, r, c, h);
                    }
                }
            }
        }
    }
    if (P.partial == nullptr) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[warp][VEC ? 8 * lane + i : lane + 32 * i] = sum[i];
    __syncthreads();
    const int mine = (int)blockIdx.y * 256 + threadIdx.x;
    if (mine < P.n) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += part[i][threadIdx.x];
        P.partial[(int64_t)blockIdx.x * P.n + mine] = s;
    }
}
// The words that linear_largest_kernel is about to raise.  (A kernel rather than a memset, beside which no kernel starts early: 1 us of a small step.)
__global__ void __launch_bounds__(256) linear_zero_kernel(uint32_t *to, int64_t n)
{
    pdl_wait();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) to[i] = 0;
}
// The largest finite |dP| of every row and of every column, into words that were zero: the order of fp32's bits is the order of values that are not negative, and
// a largest one does not depend on the atomics' order.
template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(256, 2) linear_largest_kernel(const LinearGradArgs P)
{
    pdl_wait();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ uint32_t part[8][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = (int)blockIdx.y * 256 + (VEC ? 8 * lane : lane);
    const int64_t row0 = (int64_t)blockIdx.x * P.block_rows, row1 = min(P.rows, row0 + P.block_rows);
    uint32_t most[8] = {};
    for (int64_t r0 = row0 + warp; r0 < row1; r0 += 16) {
        uint32_t of_row[2] = {};
        if (c < P.n) {
            float g[2][8];
#pragma unroll
            for (int q = 0; q < 2; ++q) load_dp<T, ACT, VEC>(P, min(r0 + 8 * q, row1 - 1), c, g[q]);  // a row twice changes nothing
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t b = __float_as_uint(fabsf(g[q][i])), finite = b < 0x7f800000u ? b : 0;
                    most[i] = max(most[i], finite), of_row[q] = max(of_row[q], finite);
                }
        }
        __syncwarp();
        if (P.row_largest != nullptr) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                of_row[q] = __reduce_max_sync(FULL, of_row[q]);
                if (lane == 0) atomicMax(P.row_largest + min(r0 + 8 * q, row1 - 1), of_row[q]);
            }
        }
    }
    if (P.col_largest == nullptr) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[warp][VEC ? 8 * lane + i : lane + 32 * i] = most[i];
    __syncthreads();
    const int mine = (int)blockIdx.y * 256 + threadIdx.x;
    if (mine < P.n) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, part[i][threadIdx.x]);
        atomicMax(P.col_largest + mine, m);
    }
}
// 32 columns per block, the blocks of rows dealt out to its warps; the warps' sums are added in order
template <typename T>
__global__ void __launch_bounds__(1024) linear_bias_kernel(const float *partial, int64_t parts, int n, void *out, int out_f32)
{
    pdl_wait();
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = (int)blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < n) {
#pragma unroll 4
        for (int64_t r = warp; r < parts; r += 32) s += ld(partial + r * n + c);
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < n) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += part[i][lane];
        store_either<T>(out, c, out_f32, s);
    }
}

}  // namespace lapsum
