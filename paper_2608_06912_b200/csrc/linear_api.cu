// C entries of the dense product: lapsum_linear_*.  Argument checks, buffer layout, choice of tiles, tensor maps and launches; nothing is
// allocated and the host never waits.
#include <cstring>

#include "../../include/lapsum.h"
#include "api.h"
#include "host.h"
#include "linear.cuh"

using namespace lapsum;

namespace {

struct LinearLayout {
    size_t off_dp, off_low, off_partial, off_parts, off_largest;
    int64_t ld, parts;  // row stride of pre and dP, blocks of rows of the bias' partial sums
};

// A gradient whose tiles are fewer than an eighth of the SMs, with a long contraction: as many parts of it as fill the SMs, of 16 steps of 64 at least, each with
// a tile's fp32 results in the workspace.  Measured, dW without / with parts, us: 65536 x 128 x 2048 86 / 71, in fp32 186 / 130; 65536 x 64 x 512 83 / 30, 177 / 56;
// 65536 x 11 x 72 100 / 36; 4096 x 128 x 256 17 / 16; dx of 100 x 60000 x 128 78 / 22.
constexpr int PARTS_UNITS = 148;  // the SMs of a B200: a workspace is described without a device
constexpr size_t PARTS_BYTES = (size_t)PARTS_UNITS * 128 * 128 * 4;
int linear_layout(const lapsum_linear_dims *p, LinearLayout &X, lapsum_linear_layout *out)
{
    if (!p) return LAPSUM_ERR_NULL;
    if (p->rows < 0 || p->rows > (int64_t)1 << 30 || p->n < 1 || p->n > (int64_t)1 << 23 || p->k < 8 || p->k > (int64_t)1 << 20 || p->k % 8)
        return LAPSUM_ERR_SHAPE;
    if (p->io_dtype != LAPSUM_IO_F16 && p->io_dtype != LAPSUM_IO_BF16) return LAPSUM_ERR_UNSUPPORTED;
    for (const int32_t t : {p->out_dtype, p->bias_dtype, p->grad_w_dtype, p->pre_dtype})
        if (t != p->io_dtype && t != LAPSUM_IO_F32) return LAPSUM_ERR_UNSUPPORTED;
    if (p->activation < LAPSUM_ACT_NONE || p->activation > LAPSUM_ACT_GELU_TANH || (p->training != 0 && p->training != 1)) return LAPSUM_ERR_PARAM;
    X.ld = (p->n + 7) / 8 * 8;
    X.parts = ceil_div(p->rows, grad_block_rows(p->rows));
    size_t at = 256;  // control block: the status word
    X.off_dp = at, at += p->training ? align_up((size_t)p->rows * (size_t)X.ld * 2) : 0;
    // a 16-bit grad_y without an activation is dP itself, copied at most: no remainder, nothing to scale
    const bool computed = p->activation != LAPSUM_ACT_NONE || p->out_dtype == LAPSUM_IO_F32;
    X.off_low = at, at += p->training && computed ? align_up((size_t)p->rows * (size_t)X.ld * 2) : 0;
    X.off_partial = at, at += p->training ? align_up((size_t)grad_blocks_most(p->rows) * (size_t)p->n * 4) : 0;
    X.off_parts = at, at += p->training ? PARTS_BYTES : 0;
    X.off_largest = at, at += p->training && computed && p->io_dtype == LAPSUM_IO_F16 ? align_up((size_t)(p->rows + p->n) * 4) : 0;
    out->workspace_bytes = at;
    out->pre_bytes = p->training && p->activation != LAPSUM_ACT_NONE ? (size_t)p->rows * (size_t)X.ld * (p->pre_dtype == LAPSUM_IO_F32 ? 4 : 2) : 0;
    out->pre_stride = X.ld;
    return LAPSUM_OK;
}

// Tiles of a product of L lanes, C columns and K along the contraction.  For every form of tile the time is taken as rounds of the SMs times
// (steps of 64 x clocks per step + the tile's own time), and the least wins.  Clocks per step: the tensor core's 2 x BN, or the operands' bytes
// at BYTES_PER_CLOCK for each SM, whichever is more; a pair of blocks shares its operands.  A shared contraction costs its join.
// Measured, tile columns / blocks per tile, us: 1021 x 2048 x 5632 128 41, 128 / 2 49, 256 / 2 35, pairs 45, pairs / 2 33; 512 x 2048 x 2048 64 19, 128 18, 128 / 2 18,
// 128 / 4 27; 16384 x 8192 x 2048 128 617, 256 461, pairs 428 (of 224 columns, which leave no round half empty, 4 % slower: the power limit); 65536 x 128 x 2048 64 84, 128 70, 256 68, pairs 86; 48 x 2048 x 1024 64 15, 64 / 4 14, 64 / 8 21.
constexpr double BYTES_PER_CLOCK = 45.0;
struct Choice {
    int bn, split;
    bool pair;
};
Choice choose(int64_t L, int64_t C, int64_t K, bool b_mn, int sms)
{
    const int64_t steps = ceil_div(K, 64);
    Choice best{b_mn ? 64 : 16, 1, false};
    double least = 1e300;
    for (int bn = b_mn ? 64 : 16; bn <= 256; bn *= 2) {
        if (bn >= 2 * C && bn > (b_mn ? 64 : 16)) break;  // half of the tile and more would be empty
        const int64_t tiles = ceil_div(L, 128) * ceil_div(C, bn);
        const double bytes = 128 * (128 + bn) / BYTES_PER_CLOCK, step = bytes > 2.0 * bn ? bytes : 2.0 * bn;
        for (int split = 1; split <= 4; split *= 2) {
            if (split > 1 && (steps < 4 * split || tiles * split > sms)) break;
            if ((split - 1) * ceil_div(steps, split) >= steps) continue;  // a block without a part
            const int64_t rounds = ceil_div(tiles * split, sms);
            const double t = (double)rounds * ((double)ceil_div(steps, split) * step + 10.0 * bn) + (split > 1 ? 2000.0 + 20.0 * bn : 0.0);
            if (t < least) least = t, best = Choice{bn, split, false};
        }
    }
    const int64_t tiles = ceil_div(L, 256) * ceil_div(C, 256);
    for (int split = 1; split <= 2 && C > 128; split *= 2) {
        if (split > 1 && (steps < 4 * split || 2 * split * tiles > sms)) break;
        const double t = (double)ceil_div(2 * split * tiles, sms) * ((double)ceil_div(steps, split) * 256 * 128 / BYTES_PER_CLOCK + 2560.0) + (split > 1 ? 7120.0 : 0.0);
        if (t < least) least = t, best = Choice{256, split, true};
    }
    return best;
}

template <bool A_MN, bool B_MN, int BN, bool PAIR, bool WIDE, typename T>
int run_tiles(const LinearMaps &maps, const LinearArgs &A, int sms, cudaStream_t st)
{
    using S = LinearShape<BN, PAIR>;
    static thread_local int dev_ready = -1;  // the attribute belongs to the device's context
    int dev = 0;
    CU_OK(cudaGetDevice(&dev));
    const auto kernel = linear_kernel<A_MN, B_MN, BN, PAIR, WIDE, T>;
    if (dev != dev_ready) {
        CU_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
        dev_ready = dev;
    }
    const int64_t tiles = (int64_t)A.lane_tiles * A.col_tiles, units = A.split > 1 || A.parts > 1 ? tiles * A.parts : PAIR ? sms / 2 : sms;
    const int cluster = (PAIR ? 2 : 1) * A.split;
    return launch_clusters((unsigned)cluster, kernel, (unsigned)((tiles * A.parts < units ? tiles * A.parts : units) * cluster), S::THREADS, S::SMEM, st, maps, A);
}
template <bool A_MN, bool B_MN, bool WIDE, typename T>
int run_choice(const LinearMaps &m, const LinearArgs &A, const Choice &ch, int sms, cudaStream_t st)
{
    if (ch.pair) return run_tiles<A_MN, B_MN, 256, true, WIDE, T>(m, A, sms, st);
    switch (ch.bn) {
    case 256: return run_tiles<A_MN, B_MN, 256, false, WIDE, T>(m, A, sms, st);
    case 128: return run_tiles<A_MN, B_MN, 128, false, WIDE, T>(m, A, sms, st);
    case 64: return run_tiles<A_MN, B_MN, 64, false, WIDE, T>(m, A, sms, st);
    default: break;
    }
    if constexpr (!B_MN) {
        if (ch.bn == 32) return run_tiles<A_MN, B_MN, 32, false, WIDE, T>(m, A, sms, st);
        return run_tiles<A_MN, B_MN, 16, false, WIDE, T>(m, A, sms, st);
    }
    return LAPSUM_ERR_PARAM;
}

struct Operand {
    const void *base;
    int64_t cols, rows, stride;  // as it lies in memory; the contraction runs along the columns, or (MN-major) along the rows
};

// Steps of 64 that one accumulator takes for a 16-bit result.  The tensor core's additions truncate; where all terms have one sign that adds up to 6.3e-9 of the
// sum per term (measured: fp16 sums of 16384 terms off by -1.0e-4 in the mean, of 400003 by -6.4e-4 in four parts).  Up to here it stays below a ninth of the largest
// rounding of the type, 2^-11 or 2^-8; beyond, rounds are summed in registers: of 2048 (off by 1.3e-5), which cost 7 % (dW of 16384 x 8192 x 2048 fp16 410 -> 438 us);
// rounds of 512, as fp32 results have them, 16 %.
constexpr int64_t LONG_F16 = 8192 / 64, LONG_BF16 = 65536 / 64;
constexpr int ROUND_F32 = 512 / 64, ROUND_16 = 2048 / 64;

// One product.  A: [L][K] or, A_MN, [K][L]; B: [C][K] or, B_MN, [K][C].
// `partial`: room for parts of the contraction (PARTS_BYTES), gradients only.
template <bool A_MN, bool B_MN, typename T>
int product(const Operand &a, const Operand &b, LinearArgs A, int dtype, cudaStream_t st, float *partial = nullptr, const void *low = nullptr)
{
    int sms = 0;
    RUN(sm_count(&sms));
    A.twice = low != nullptr;
    A.round = A.out_f32 ? ROUND_F32 : ROUND_16;
    Choice ch = choose(A.L, A.C, A.K * (low ? 2ll : 1ll), B_MN, sms);
    const LinearArgs whole = A;
    if (partial) {
        const int64_t steps = ceil_div(A.K, 64) * (low ? 2 : 1), bn = A.C > 64 ? 128 : 64, tiles = ceil_div(A.L, 128) * ceil_div(A.C, bn);
        int64_t parts = PARTS_UNITS / tiles;
        if (parts > steps / 16) parts = steps / 16;
        if (parts >= 8) {
            parts = ceil_div(steps, ceil_div(steps, parts));  // none without a part
            ch = Choice{(int)bn, 1, false};
            A.parts = (int)parts;
            A.out = partial, A.out_stride = A.L, A.out_f32 = 1, A.largest = nullptr;
        }
    }
    A.split = ch.split;
    A.lane_tiles = (int)ceil_div(A.L, ch.pair ? 256 : 128), A.col_tiles = (int)ceil_div(A.C, ch.bn);
    LinearMaps m;
    RUN(map_2d(&m.a, dtype, a.base, a.cols, a.rows, a.stride, A_MN ? 64 : 128));
    RUN(map_2d(&m.b, dtype, b.base, b.cols, b.rows, b.stride, B_MN ? 64 : ch.pair ? 128 : ch.bn));
    m.b_low = m.b;
    if (low) RUN(map_2d(&m.b_low, dtype, low, b.cols, b.rows, b.stride, B_MN ? 64 : ch.pair ? 128 : ch.bn));
    if constexpr (A_MN) {
        if (A.parts > 1) {
            RUN((ch.bn == 128 ? run_tiles<A_MN, B_MN, 128, false, true, T>(m, A, sms, st) : run_tiles<A_MN, B_MN, 64, false, true, T>(m, A, sms, st)));
            return launch_pdl(linear_parts_kernel<T>, (unsigned)ceil_div((int64_t)A.C * A.L, 256), 256, 0, st, partial, A.parts, A.C, A.L, whole.out,
                              whole.out_stride, whole.out_f32, whole.largest);
        }
    }
    const bool rounds = A.out_f32 || ceil_div(ceil_div(A.K, 64), ch.split) > (dtype == LAPSUM_IO_F16 ? LONG_F16 : LONG_BF16);
    return rounds ? run_choice<A_MN, B_MN, true, T>(m, A, ch, sms, st) : run_choice<A_MN, B_MN, false, T>(m, A, ch, sms, st);
}

constexpr int64_t FEW_ROWS = 4;

template <typename T>
int few(const void *x, int64_t x_stride, const void *w, const LinearArgs &A, cudaStream_t st)
{
    const unsigned blocks = (unsigned)ceil_div(A.L, 16);
    const T *const xt = static_cast<const T *>(x), *const wt = static_cast<const T *>(w);
    switch (A.C) {
    case 1: return launch_pdl(linear_few_kernel<T, 1>, blocks, 256, 0, st, xt, x_stride, wt, A);
    case 2: return launch_pdl(linear_few_kernel<T, 2>, blocks, 256, 0, st, xt, x_stride, wt, A);
    case 3: return launch_pdl(linear_few_kernel<T, 3>, blocks, 256, 0, st, xt, x_stride, wt, A);
    default: return launch_pdl(linear_few_kernel<T, 4>, blocks, 256, 0, st, xt, x_stride, wt, A);
    }
}

template <typename T>
int forward_t(const lapsum_linear_dims &p, const void *x, int64_t x_stride, const void *w, const LinearArgs &A, cudaStream_t st)
{
    if (p.rows <= FEW_ROWS && !A.hold) return few<T>(x, x_stride, w, A, st);
    return product<false, false, T>(Operand{w, p.k, p.n, p.k}, Operand{x, p.k, p.rows, x_stride}, A, p.io_dtype, st);
}

LinearArgs base_args(void *ws)
{
    LinearArgs A;
    std::memset(&A, 0, sizeof(A));
    A.split = A.parts = 1;
    A.status = static_cast<uint32_t *>(ws);
    A.wait_ns = 2000000000ull;
    return A;
}

template <typename T, int ACT>
int grad(bool vec, bool largest, dim3 grid, const LinearGradArgs &G, cudaStream_t st)
{
    if constexpr (std::is_same<T, __half>::value) {
        if (largest) return launch_pdl(vec ? linear_largest_kernel<T, ACT, true> : linear_largest_kernel<T, ACT, false>, grid, 256, 0, st, G);
    }
    return launch_pdl(vec ? linear_grad_kernel<T, ACT, true> : linear_grad_kernel<T, ACT, false>, grid, 256, 0, st, G);
}
template <typename T>
int grad_by_act(int act, bool vec, bool largest, dim3 grid, const LinearGradArgs &G, cudaStream_t st)
{
    switch (act) {
    case LAPSUM_ACT_RELU: return grad<T, LAPSUM_ACT_RELU>(vec, largest, grid, G, st);
    case LAPSUM_ACT_SILU: return grad<T, LAPSUM_ACT_SILU>(vec, largest, grid, G, st);
    case LAPSUM_ACT_GELU: return grad<T, LAPSUM_ACT_GELU>(vec, largest, grid, G, st);
    case LAPSUM_ACT_GELU_TANH: return grad<T, LAPSUM_ACT_GELU_TANH>(vec, largest, grid, G, st);
    default: return grad<T, LAPSUM_ACT_NONE>(vec, largest, grid, G, st);
    }
}

template <typename T>
int backward_t(const lapsum_linear_dims &p, const LinearLayout &X, const void *grad_y, int64_t gy_stride, const void *x, int64_t x_stride,
               const void *w, const void *pre, void *grad_x, int64_t gx_stride, void *grad_w, void *grad_bias, uint8_t *ws, cudaStream_t st)
{
    const bool y_f32 = p.out_dtype == LAPSUM_IO_F32, wide = p.grad_w_dtype == LAPSUM_IO_F32;
    // grad_y is dP itself where there is no activation and the tensor maps can take it as it lies
    const bool same = p.activation == LAPSUM_ACT_NONE && !y_f32, direct = same && gy_stride % 8 == 0 && aligned(grad_y, 16);
    const bool products = grad_x || grad_w, keep_low = grad_w && !same && wide;
    // fp16 that is computed: dW's operand is scaled by columns, dx's by rows.  Both are written at once, the second in the room of the remainder, or, where dW
    // needs that, one after the other.
    const bool scaled = products && !same && p.io_dtype == LAPSUM_IO_F16, again = scaled && grad_x && keep_low;
    LinearGradArgs G;
    std::memset(&G, 0, sizeof(G));
    G.grad_y = grad_y, G.pre = pre, G.pre_f32 = p.pre_dtype == LAPSUM_IO_F32;
    G.y_stride = gy_stride, G.pre_stride = G.dp_stride = X.ld, G.rows = p.rows, G.n = (int)p.n, G.y_f32 = y_f32, G.block_rows = grad_block_rows(p.rows);
    const bool vec = gy_stride % 8 == 0 && p.n % 8 == 0 && aligned(grad_y, 16);
    const dim3 grid((unsigned)X.parts, (unsigned)ceil_div(p.n, 256));
    if (scaled) {
        uint32_t *const largest = reinterpret_cast<uint32_t *>(ws + X.off_largest);
        G.row_largest = grad_x ? largest : nullptr, G.col_largest = grad_w ? largest + p.rows : nullptr;
        RUN(launch_pdl(linear_zero_kernel, (unsigned)ceil_div(p.rows + p.n, 256), 256, 0, st, largest, p.rows + p.n));
        RUN((grad_by_act<T>(p.activation, vec, true, grid, G, st)));
    }
    uint8_t *const dp_w = ws + X.off_dp, *const dp_x = scaled && grad_w && !again ? ws + X.off_low : ws + X.off_dp;
    if (grad_bias || (products && !direct)) {
        G.partial = grad_bias ? reinterpret_cast<float *>(ws + X.off_partial) : nullptr;
        if (scaled ? grad_w != nullptr : products && !direct) G.dp = dp_w;
        if (scaled && grad_x && !again) G.dp_rows = dp_x;
        if (keep_low) G.dp_low = ws + X.off_low;
        RUN((grad_by_act<T>(p.activation, vec, false, grid, G, st)));
        if (grad_bias)
            RUN(launch_pdl(linear_bias_kernel<T>, (unsigned)ceil_div(p.n, 32), 1024, 0, st, G.partial, X.parts, (int)p.n, grad_bias,
                           p.bias_dtype == LAPSUM_IO_F32 ? 1 : 0));
    }
    const auto operand = [&](const uint8_t *dp) { return direct ? Operand{grad_y, p.n, p.rows, gy_stride} : Operand{dp, p.n, p.rows, X.ld}; };
    float *const partial = reinterpret_cast<float *>(ws + X.off_parts);
    const auto to_x = [&] {
        LinearArgs A = base_args(ws);
        A.out = grad_x, A.out_stride = gx_stride, A.out_f32 = 0, A.largest = G.row_largest;
        A.L = (int)p.k, A.C = (int)p.rows, A.K = (int)p.n;
        return product<true, false, T>(Operand{w, p.k, p.n, p.k}, operand(dp_x), A, p.io_dtype, st, partial);
    };
    if (grad_x && !again) RUN(to_x());
    if (grad_w) {
        LinearArgs A = base_args(ws);
        A.out = grad_w, A.out_stride = p.k, A.out_f32 = wide, A.largest = G.col_largest;
        A.L = (int)p.k, A.C = (int)p.n, A.K = (int)p.rows;
        RUN((product<true, true, T>(Operand{x, p.k, p.rows, x_stride}, operand(dp_w), A, p.io_dtype, st, partial, keep_low ? ws + X.off_low : nullptr)));
    }
    if (again) {
        G.partial = nullptr, G.dp = G.dp_low = nullptr, G.dp_rows = dp_x;
        RUN((grad_by_act<T>(p.activation, vec, false, grid, G, st)));
        RUN(to_x());
    }
    return LAPSUM_OK;
}

}  // namespace

extern "C" {

int lapsum_linear_describe(const lapsum_linear_dims *dims, lapsum_linear_layout *out)
{
    if (!out) return LAPSUM_ERR_NULL;
    LinearLayout X;
    return linear_layout(dims, X, out);
}

int lapsum_linear_workspace_init(void *ws, size_t bytes, const lapsum_linear_dims *dims, void *stream)
{
    LinearLayout X;
    lapsum_linear_layout out;
    RUN(linear_layout(dims, X, &out));
    if (!ws) return LAPSUM_ERR_NULL;
    if (!aligned(ws, 256) || bytes < out.workspace_bytes) return LAPSUM_ERR_WORKSPACE;
    CU_OK(cudaMemsetAsync(ws, 0, 256, static_cast<cudaStream_t>(stream)));
    return LAPSUM_OK;
}

int lapsum_linear_status(void *ws, void *stream, uint32_t *status_bits) { return lapsum_experts_status(ws, stream, status_bits); }

int lapsum_linear_forward(const void *x, int64_t x_stride, const void *w, const void *bias, const void *residual, int64_t residual_stride,
                          void *y, int64_t y_stride, void *pre, size_t pre_bytes, const lapsum_linear_dims *dims, void *ws, size_t ws_bytes,
                          void *stream)
{
    LinearLayout X;
    lapsum_linear_layout out;
    RUN(linear_layout(dims, X, &out));
    if (!ws) return LAPSUM_ERR_NULL;
    if (!aligned(ws, 256) || ws_bytes < out.workspace_bytes) return LAPSUM_ERR_WORKSPACE;
    if (dims->rows == 0) return LAPSUM_OK;
    if (x_stride < dims->k || x_stride % 8 || y_stride < dims->n || (residual && residual_stride < dims->n)) return LAPSUM_ERR_SHAPE;
    if (!x || !w || !y || (out.pre_bytes && !pre)) return LAPSUM_ERR_NULL;
    if (!out.pre_bytes && pre) return LAPSUM_ERR_PARAM;
    if (pre && (!aligned(pre, 256) || pre_bytes < out.pre_bytes)) return LAPSUM_ERR_WORKSPACE;
    if (!aligned(x, 16) || !aligned(w, 16)) return LAPSUM_ERR_ALIGN;
    LinearArgs A = base_args(ws);
    A.out = y, A.residual = residual, A.bias = bias, A.pre = pre;
    A.out_stride = y_stride, A.residual_stride = residual_stride, A.pre_stride = X.ld;
    A.L = (int)dims->n, A.C = (int)dims->rows, A.K = (int)dims->k, A.act = dims->activation;
    A.out_f32 = dims->out_dtype == LAPSUM_IO_F32, A.bias_f32 = dims->bias_dtype == LAPSUM_IO_F32, A.pre_f32 = dims->pre_dtype == LAPSUM_IO_F32;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dims->io_dtype == LAPSUM_IO_BF16 ? forward_t<__nv_bfloat16>(*dims, x, x_stride, w, A, st) : forward_t<__half>(*dims, x, x_stride, w, A, st);
}

int lapsum_linear_backward(const void *grad_y, int64_t grad_y_stride, const void *x, int64_t x_stride, const void *w, const void *pre,
                           size_t pre_bytes, void *grad_x, int64_t grad_x_stride, void *grad_w, void *grad_bias,
                           const lapsum_linear_dims *dims, void *ws, size_t ws_bytes, void *stream)
{
    LinearLayout X;
    lapsum_linear_layout out;
    RUN(linear_layout(dims, X, &out));
    if (!dims->training) return LAPSUM_ERR_UNSUPPORTED;
    if (!ws) return LAPSUM_ERR_NULL;
    if (!aligned(ws, 256) || ws_bytes < out.workspace_bytes) return LAPSUM_ERR_WORKSPACE;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dims->rows == 0) {  // no row: the weights' gradients are zeros
        if (grad_w) CU_OK(cudaMemsetAsync(grad_w, 0, (size_t)dims->n * (size_t)dims->k * (dims->grad_w_dtype == LAPSUM_IO_F32 ? 4 : 2), st));
        if (grad_bias) CU_OK(cudaMemsetAsync(grad_bias, 0, (size_t)dims->n * (dims->bias_dtype == LAPSUM_IO_F32 ? 4 : 2), st));
        return LAPSUM_OK;
    }
    if (grad_y_stride < dims->n || x_stride < dims->k || x_stride % 8 || (grad_x && grad_x_stride < dims->k)) return LAPSUM_ERR_SHAPE;
    if (!grad_y || !x || !w || (out.pre_bytes && !pre)) return LAPSUM_ERR_NULL;
    if (!out.pre_bytes && pre) return LAPSUM_ERR_PARAM;
    if (pre && (!aligned(pre, 256) || pre_bytes < out.pre_bytes)) return LAPSUM_ERR_WORKSPACE;
    if (!aligned(x, 16) || !aligned(w, 16)) return LAPSUM_ERR_ALIGN;
    uint8_t *const at = static_cast<uint8_t *>(ws);
    return dims->io_dtype == LAPSUM_IO_BF16 ? backward_t<__nv_bfloat16>(*dims, X, grad_y, grad_y_stride, x, x_stride, w, pre, grad_x,
                                                                        grad_x_stride, grad_w, grad_bias, at, st)
                                            : backward_t<__half>(*dims, X, grad_y, grad_y_stride, x, x_stride, w, pre, grad_x, grad_x_stride,
                                                                 grad_w, grad_bias, at, st);
}

int lapsum_debug_linear_timeout(int64_t wait_us, const void *x, const void *w, void *y, const lapsum_linear_dims *dims, void *ws,
                                size_t ws_bytes, void *stream)
{
    LinearLayout X;
    lapsum_linear_layout out;
    RUN(linear_layout(dims, X, &out));
    if (!ws || !x || !w || !y) return LAPSUM_ERR_NULL;
    if (!aligned(ws, 256) || ws_bytes < out.workspace_bytes) return LAPSUM_ERR_WORKSPACE;
    if (dims->rows <= FEW_ROWS || dims->io_dtype != LAPSUM_IO_BF16) return LAPSUM_ERR_UNSUPPORTED;
    if (wait_us < 1 || wait_us > 100000) return LAPSUM_ERR_PARAM;
    if (!aligned(x, 16) || !aligned(w, 16)) return LAPSUM_ERR_ALIGN;
    LinearArgs A = base_args(ws);
    A.out = y, A.out_stride = dims->n, A.L = (int)dims->n, A.C = (int)dims->rows, A.K = (int)dims->k, A.out_f32 = dims->out_dtype == LAPSUM_IO_F32;
    A.hold = 1, A.wait_ns = (unsigned long long)wait_us * 1000;
    return forward_t<__nv_bfloat16>(*dims, x, dims->k, w, A, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
