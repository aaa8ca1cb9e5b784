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
#pragma once
#include <type_traits>

#include "common.cuh"
#include "tensor_core.cuh"

namespace lapsum {

struct LinearMaps {
    CUtensorMap a, b;
};

struct LinearArgs {
    void *out;             // fp32 (out_f32) or T, rows out_stride elements apart
    const void *residual;  // like out, or null
    const void *bias;      // fp32 (bias_f32) or T, or null
    void *pre;             // T, rows pre_stride elements apart, or null
    int64_t out_stride, residual_stride, pre_stride;
    int L, C, K;           // lanes, columns, contraction
    int lane_tiles, col_tiles;
    int act, out_f32, bias_f32;
    int split;             // blocks of a cluster that share the contraction of one tile
    int hold;              // test hook: the producer brings nothing, so the waits run out
    uint32_t *status;
    unsigned long long wait_ns;
};

// ---------------------------------------------------------------- activations ----
// e^x to about 2 ulp: the product with log2(e) split in two
__device__ __forceinline__ float exp_of(float x) { return exp2f(fmaf(x, 1.44269502f, x * 1.92596299e-8f)); }
__device__ __forceinline__ float sigmoid_of(float x) { return __fdividef(1.f, 1.f + exp_of(-x)); }
constexpr float GELU_A = 0.797884561f, GELU_B = 0.044715f;  // sqrt(2 / pi), the tanh form's cubic term

__device__ __forceinline__ float activate(float x, int act)
{
    switch (act) {
    case LAPSUM_ACT_RELU: return x > 0.f ? x : x == x ? 0.f : x;
    case LAPSUM_ACT_SILU: return x * sigmoid_of(x);
    case LAPSUM_ACT_GELU: return 0.5f * x * (1.f + erff(0.707106781f * x));
    case LAPSUM_ACT_GELU_TANH: return x * sigmoid_of(2.f * GELU_A * x * fmaf(GELU_B * x, x, 1.f));  // (1 + tanh u) / 2 = sigmoid(2 u)
    default: return x;
    }
}
// The slope at a pre-activation that was kept in 16 bits; beyond +-1000 every activation's slope is its limit (an infinity kept by
// fp16 included, where the formulas would give infinity times 0).
__device__ __forceinline__ float slope_of(float x, int act)
{
    x = x > 1000.f ? 1000.f : x < -1000.f ? -1000.f : x;  // NaN stays
    switch (act) {
    case LAPSUM_ACT_RELU: return x > 0.f ? 1.f : x == x ? 0.f : x;
    case LAPSUM_ACT_SILU: {
        const float s = sigmoid_of(x);
        return s * fmaf(x, 1.f - s, 1.f);
    }
    case LAPSUM_ACT_GELU: return fmaf(0.398942280f * x, exp_of(-0.5f * x * x), 0.5f + 0.5f * erff(0.707106781f * x));
    case LAPSUM_ACT_GELU_TANH: {
        const float s = sigmoid_of(2.f * GELU_A * x * fmaf(GELU_B * x, x, 1.f));
        return fmaf(2.f * GELU_A * x * s, (1.f - s) * fmaf(3.f * GELU_B * x, x, 1.f), s);
    }
    default: return 1.f;
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

// N values of lane l, rows r0 .. : bias, pre-activation, activation, residual, result
template <typename T, int N>
__device__ __forceinline__ void linear_finish(const LinearArgs &P, float (&v)[N], int l, int r0, float bias)
{
    const int n = min(N, P.C - r0);
    float res[N];
    if (P.residual != nullptr) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < n) res[j] = load_either<T>(P.residual, (int64_t)(r0 + j) * P.residual_stride + l, P.out_f32);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] += bias;
    if (P.pre != nullptr) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < n) Io<T>::store1(static_cast<T *>(P.pre) + (int64_t)(r0 + j) * P.pre_stride + l, v[j]);
    }
    if (P.act != LAPSUM_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = activate(v[j], P.act);
    }
    if (P.residual != nullptr) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] += res[j];
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < n) store_either<T>(P.out, (int64_t)(r0 + j) * P.out_stride + l, P.out_f32, v[j]);
}

// ---------------------------------------------------------------- the kernel ----
// Warp 0 brings operand tiles of 64 along the contraction into a ring of stages by TMA, one thread of warp 1 issues tcgen05.mma
// into one of two accumulators in TMEM, warps 4 to 11 (two sets of four; a set reads the 128 lanes) finish the previous tile.
//   PAIR   a cluster of two blocks works on one 256 x 256 tile (cta_group::2): each block brings 128 rows of A and half of B, 64 bytes per
//          clock of tensor work instead of the 96 that a 128 x 256 tile of one block needs.
//   split  a cluster of `split` blocks shares the contraction of one tile, for shapes with few tiles: each leaves its sums in its shared
//          memory, and after a cluster barrier adds its share of the columns over the blocks, in their order.
template <int BN, bool PAIR_>
struct LinearShape {
    static constexpr bool PAIR = PAIR_;
    static constexpr int COLS = PAIR ? BN / 2 : BN;  // columns of B that one block brings
    static constexpr int A_BYTES = 128 * 128, B_BYTES = COLS * 128, STAGE = A_BYTES + B_BYTES;
    static constexpr int FIT = 229376 / STAGE, STAGES = FIT < 12 ? FIT : 12;
    static constexpr int ACC = 2, TMEM = ACC * BN;
    static constexpr int THREADS = 384;
    static constexpr int SMEM = STAGES * STAGE + 1024 + 512;
    static_assert(STAGES >= 2 && TMEM >= 32 && TMEM <= 512 && BN * 512 <= STAGES * STAGE, "tile does not fit");
};

template <bool A_MN, bool B_MN, int BN, bool PAIR, typename T>
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
    const bool split = !PAIR && P.split > 1;
    const uint32_t rank = PAIR || split ? cluster_rank() : 0;

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

    const int steps = (P.K + 63) / 64;
    const int share = split ? (steps + P.split - 1) / P.split : steps;
    const int k_first = split ? min((int)rank * share, steps) : 0, nkb = min(share, steps - k_first);  // 0: a block without a part
    const int64_t tiles = (int64_t)P.lane_tiles * P.col_tiles;
    const int64_t group = PAIR ? 2 : split ? P.split : 1, tile0 = blockIdx.x / group, tile_step = gridDim.x / group;

    // Tiles in groups of eight column tiles, lane tiles outside: what the SMs work on at one time shares its operands in L2.
    struct Tile {
        int l0, c0;
    };
    auto tile_at = [&](int64_t i) {
        const int64_t per = (int64_t)8 * P.lane_tiles, g = i / per;
        const int rest = (int)(i - g * per), wide = (int)min((int64_t)8, P.col_tiles - 8 * g);
        const int lt = rest / wide, ct = (int)(8 * g) + rest - lt * wide;
        return Tile{(PAIR ? 256 : 128) * lt + (PAIR ? 128 * (int)rank : 0), BN * ct};
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
            const int c0 = t.c0 + (PAIR ? (int)rank * S::COLS : 0);
            for (int kb = 0; kb < nkb; ++kb, ++fill) {
                const uint32_t s = fill % S::STAGES, phase = (fill / S::STAGES) & 1;
                ok = waits.wait(empty + 8 * s, phase ^ 1);
                ok = __all_sync(FULL, ok);
                if (!ok || P.hold) break;
                const uint32_t bar = PAIR ? in_block(full + 8 * s, 0) : full + 8 * s;  // a pair's first block counts for both
                if (lane == 0 && (!PAIR || rank == 0)) mbar_expect_tx(full + 8 * s, PAIR ? 2 * S::STAGE : S::STAGE);
                __syncwarp();
                const int k0 = (k_first + kb) * 64;
                const uint32_t a = ring_a + s * S::A_BYTES, b = ring_b + s * S::B_BYTES;
                if constexpr (A_MN) {
                    if (lane < 2) load(a + lane * 8192, &maps.a, t.l0 + lane * 64, k0, bar);
                } else {
                    if (lane == 0) load(a, &maps.a, k0, t.l0, bar);
                }
                if constexpr (B_MN) {
                    if (lane >= 2 && lane < 2 + S::COLS / 64) load(b + (lane - 2) * 8192, &maps.b, c0 + (lane - 2) * 64, k0, bar);
                } else {
                    if (lane == 2) load(b, &maps.b, k0, c0, bar);
                }
            }
            if (P.hold) break;
        }
        // every copy has landed and every product has read its stage before the block may end
        const uint32_t first = fill > S::STAGES ? fill - S::STAGES : 0;
        for (uint32_t f = first; f < fill; ++f) {
            const uint32_t s = f % S::STAGES, phase = (f / S::STAGES) & 1;
            if (!PAIR || rank == 0) waits.plain(full + 8 * s, phase, false);
            if (ok) waits.wait(empty + 8 * s, phase);
        }
    } else if (warp == 1) {
        // ------------------------------------------------ one thread issues the products (a pair's: one of its first block)
        if (lane == 0 && (!PAIR || rank == 0)) {
            constexpr uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
            constexpr uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
                                       ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((PAIR ? 256 : 128) >> 4) << 24);
            constexpr uint32_t step_a = A_MN ? 2048 : 32, step_b = B_MN ? 2048 : 32;  // 16 along the contraction
            uint32_t fill = 0, it = 0;
            bool ok = true, any = false;
            for (int64_t i = tile0; i < tiles && ok && nkb > 0; i += tile_step, ++it) {
                const uint32_t buf = it % S::ACC, phase = (it / S::ACC) & 1;
                ok = waits.wait(acc_empty + 8 * buf, phase ^ 1);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + buf * BN;
                for (int kb = 0; kb < nkb; ++kb, ++fill) {
                    const uint32_t s = fill % S::STAGES;
                    ok = waits.wait(full + 8 * s, (fill / S::STAGES) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t a = smem_desc(ring_a + s * S::A_BYTES, A_MN), b = smem_desc(ring_b + s * S::B_BYTES, B_MN);
#pragma unroll
                    for (int q = 0; q < 4; ++q) tc_mma<PAIR>(d, a + q * (step_a >> 4), b + q * (step_b >> 4), idesc, (kb | q) != 0);
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
        // ------------------------------------------------ epilogue: a lane of the accumulator per thread, 16 columns at a time
        const int ew = warp & 3, set = (warp - 4) >> 2;
        const uint32_t lanes = (uint32_t)ew << 21;  // 32 TMEM lanes per warp, lane index in the upper half
        uint32_t it = 0;
        for (int64_t i = tile0; i < tiles; i += tile_step, ++it) {
            const Tile t = tile_at(i);
            const uint32_t buf = it % S::ACC, phase = (it / S::ACC) & 1;
            const int l = t.l0 + 32 * ew + lane;
            float bias = 0.f;
            if (P.bias != nullptr && l < P.L && !split) bias = load_either<T>(P.bias, l, P.bias_f32);
            if (nkb > 0) {
                const bool ok = waits.wait(acc_full + 8 * buf, phase);
                if (!__all_sync(FULL, ok)) break;
                tc_fence_after();
            }
            const uint32_t d = tmem + buf * BN + lanes;
#pragma unroll 1
            for (int c = 16 * set; c < BN && t.c0 + c < P.C; c += 32) {
                float v[16];
                if (nkb > 0) {
                    tmem_ld16(d + c, v);
                    tmem_wait_ld(v);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = 0.f;
                }
                if (split) {
                    // the ring is free: all products of this block's only tile have ended.  [column][lane]
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(ring_a + 4 * ((c + j) * 128 + 32 * ew + lane)), "f"(v[j]) : "memory");
                } else if (l < P.L) {
                    linear_finish<T>(P, v, l, t.c0 + c, bias);
                }
            }
            if (nkb > 0) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(PAIR ? in_block(acc_empty + 8 * buf, 0) : acc_empty + 8 * buf);
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if constexpr (PAIR) cluster_barrier();
    if constexpr (!PAIR) {
        if (split) {
            cluster_barrier();
            const Tile t = tile_at(tile0);
            const int l = tid & 127, per = (BN + P.split - 1) / P.split;
            const int c1 = min(min(((int)rank + 1) * per, BN), P.C - t.c0);
            if (t.l0 + l < P.L) {
                const float bias = P.bias != nullptr ? load_either<T>(P.bias, t.l0 + l, P.bias_f32) : 0.f;
                for (int c = (int)rank * per + (tid >> 7); c < c1; c += 3) {
                    float part[8], v[1] = {0.f};
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        if (s < P.split)
                            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part[s]) : "r"(in_block(ring_a + 4 * (c * 128 + l), s)) : "memory");
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        if (s < P.split) v[0] += part[s];
                    linear_finish<T>(P, v, t.l0 + l, t.c0 + c, bias);
                }
            }
            __syncwarp();
            cluster_barrier();  // nobody leaves while others read
        }
    }
    if (warp == 2) {
        tc_fence_after();
        if constexpr (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM) : "memory");
    }
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
    if (r < R && l < P.L) linear_finish<T>(P, mine, l, r, P.bias != nullptr ? load_either<T>(P.bias, l, P.bias_f32) : 0.f);
}

// ---------------------------------------------------------- dP and its column sums ----
// dP = dy act'(P) in 16 bits, the operand of both products (one rounding; the bias' gradient sums the values before it), and the sums over
// GRAD_ROWS rows, which linear_bias_kernel adds in order.  A warp has 256 columns, eight per lane, and every eighth row of the block.
constexpr int GRAD_ROWS = 64;
struct LinearGradArgs {
    const void *grad_y;  // fp32 (y_f32) or T
    const void *pre;     // T, null without an activation
    void *dp;            // T, null where grad_y itself serves
    float *partial;      // [blocks of rows][n], null without a bias
    int64_t y_stride, pre_stride, dp_stride, rows;
    int n, act, y_f32;
};
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) linear_grad_kernel(const LinearGradArgs P)
{
    pdl_wait();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ float part[8][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = (int)blockIdx.y * 256 + 8 * lane;
    const int64_t row0 = (int64_t)blockIdx.x * GRAD_ROWS, row1 = min(P.rows, row0 + GRAD_ROWS);
    float sum[8] = {};
    if (c < P.n) {
#pragma unroll 2
        for (int64_t r = row0 + warp; r < row1; r += 8) {
            float g[8];
            if (VEC) {
                if (P.y_f32) {
                    const float4 *const q = reinterpret_cast<const float4 *>(static_cast<const float *>(P.grad_y) + r * P.y_stride + c);
                    const float4 a = ld(q), b = ld(q + 1);
                    g[0] = a.x, g[1] = a.y, g[2] = a.z, g[3] = a.w, g[4] = b.x, g[5] = b.y, g[6] = b.z, g[7] = b.w;
                } else {
                    Io<T>::unpack(ld(reinterpret_cast<const uint4 *>(static_cast<const T *>(P.grad_y) + r * P.y_stride + c)), g);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = c + i < P.n ? load_either<T>(P.grad_y, r * P.y_stride + c + i, P.y_f32) : 0.f;
            }
            if (P.pre != nullptr) {
                float p[8];  // rows of pre are whole vectors
                Io<T>::unpack(ld(reinterpret_cast<const uint4 *>(static_cast<const T *>(P.pre) + r * P.pre_stride + c)), p);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = c + i < P.n ? g[i] * slope_of(p[i], P.act) : 0.f;  // the padding is nobody's
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += g[i];
            if (P.dp != nullptr) *reinterpret_cast<uint4 *>(static_cast<T *>(P.dp) + r * P.dp_stride + c) = Io<T>::pack(g);
        }
    }
    if (P.partial == nullptr) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[warp][8 * lane + i] = sum[i];
    __syncthreads();
    const int mine = (int)blockIdx.y * 256 + threadIdx.x;
    if (mine < P.n) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += part[i][threadIdx.x];
        P.partial[(int64_t)blockIdx.x * P.n + mine] = s;
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
