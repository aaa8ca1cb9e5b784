// C entries of the mixture-of-experts operators: lapsum_route_*, lapsum_dispatch*, lapsum_experts_*.  Argument checks,
// buffer layout, tensor maps and launches; nothing is allocated and the host never waits.
#include <cmath>
#include <cstring>

#include "../../include/lapsum.h"
#include "experts.cuh"
#include "host.h"
#include "routing.cuh"

using namespace lapsum;

namespace {

inline size_t align_up(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

#define CU_OK(x)                                      \
    do {                                              \
        const cudaError_t e__ = (x);                  \
        if (e__ != cudaSuccess) return cuda_fail(e__); \
    } while (0)
#define RUN(x)                    \
    do {                          \
        const int rc__ = (x);     \
        if (rc__ != 0) return rc__; \
    } while (0)

// ------------------------------------------------------------------- route ----
int route_check(int64_t tokens, int64_t experts, int64_t stride, const lapsum_route_params *p)
{
    if (!p) return LAPSUM_ERR_NULL;
    if (tokens < 0 || tokens > (int64_t)1 << 30 || experts < 1 || experts > ROUTE_MAX_E || stride < experts) return LAPSUM_ERR_SHAPE;
    if (p->score < LAPSUM_ROUTE_SOFTMAX || p->score > LAPSUM_ROUTE_GIVEN || p->io_dtype < LAPSUM_IO_F32 || p->io_dtype > LAPSUM_IO_BF16 ||
        p->grad_w_dtype < LAPSUM_IO_F32 || p->grad_w_dtype > LAPSUM_IO_BF16 || p->k < 1 || p->k > ROUTE_MAX_K || p->k > experts ||
        p->groups < 1 || p->groups > ROUTE_MAX_GROUPS || experts % p->groups || p->groups_kept < 1 || p->groups_kept > p->groups ||
        p->group_top < 1 || p->group_top > 2 || !std::isfinite(p->scale) || p->scale == 0.0 || (float)p->scale == 0.f ||
        !std::isfinite((float)p->scale))
        return LAPSUM_ERR_PARAM;
    return LAPSUM_OK;
}

inline unsigned route_grid(int64_t tokens, int lanes) { return (unsigned)((tokens * lanes + 32 * ROUTE_WARPS - 1) / (32 * ROUTE_WARPS)); }

template <typename T, int L, int NV>
struct RouteShape {
    // whole vectors at aligned addresses in every row
    static bool vec(const void *p, int64_t stride, int E)
    {
        constexpr int V = 16 / (int)sizeof(T) < NV ? 16 / (int)sizeof(T) : NV;  // elements of a vector access
        return E % V == 0 && stride % V == 0 && aligned(p, V * sizeof(T));
    }

    static int forward(const RouteArgs &A, cudaStream_t st)
    {
        const bool v = vec(A.logits, A.stride, A.E);
        const auto kernel = A.groups > 1
                                ? (v ? route_forward_kernel<T, L, NV, true, true, false> : route_forward_kernel<T, L, NV, false, true, false>)
                                : (v ? route_forward_kernel<T, L, NV, true, false, false> : route_forward_kernel<T, L, NV, false, false, false>);
        return launch_pdl(kernel, route_grid(A.tokens, L), 32 * ROUTE_WARPS, 0, st, A);
    }
    static int plain(const RouteArgs &A, cudaStream_t st)
    {
        return launch_pdl(route_forward_kernel<T, L, NV, true, false, true>, route_grid(A.tokens, L), 32 * ROUTE_WARPS, 0, st, A);
    }
    static int dense(const RouteBackArgs &A, cudaStream_t st)
    {
        const bool v = vec(A.logits, A.stride, A.E) && vec(A.grad, A.E, A.E);
        return launch_pdl(v ? route_backward_dense_kernel<T, L, NV, true> : route_backward_dense_kernel<T, L, NV, false>,
                          route_grid(A.tokens, L), 32 * ROUTE_WARPS, 0, st, A);
    }
};
// Lanes per token where scores, biases and groups are held in registers: eight with up to 16 logits each, more only where a row is
// longer.
#define BY_WIDTH(T, what, E, ...)                                 \
    ((E) <= 32    ? RouteShape<T, 8, 4>::what(__VA_ARGS__)        \
     : (E) <= 64  ? RouteShape<T, 8, 8>::what(__VA_ARGS__)        \
     : (E) <= 128 ? RouteShape<T, 8, 16>::what(__VA_ARGS__)       \
     : (E) <= 256 ? RouteShape<T, 16, 16>::what(__VA_ARGS__)      \
     : (E) <= 512 ? RouteShape<T, 32, 16>::what(__VA_ARGS__)      \
                  : RouteShape<T, 32, 32>::what(__VA_ARGS__))
#define BY_TYPE(fn, dtype, ...)                                  \
    ((dtype) == LAPSUM_IO_F32   ? fn<float>(__VA_ARGS__)          \
     : (dtype) == LAPSUM_IO_F16 ? fn<__half>(__VA_ARGS__)         \
                                : fn<__nv_bfloat16>(__VA_ARGS__))

template <typename T>
int route_forward_t(const RouteArgs &A, cudaStream_t st)
{
    // Four lanes per token and more where a lane would have over 32 logits; whole vectors of four.
    if (A.bias == nullptr && A.groups == 1 && A.E % 4 == 0 && A.stride % 4 == 0 && aligned(A.logits, 4 * sizeof(T)))
        return A.E <= 32    ? RouteShape<T, 4, 8>::plain(A, st)
               : A.E <= 64  ? RouteShape<T, 4, 16>::plain(A, st)
               : A.E <= 128 ? RouteShape<T, 4, 32>::plain(A, st)
               : A.E <= 256 ? RouteShape<T, 8, 32>::plain(A, st)
               : A.E <= 512 ? RouteShape<T, 16, 32>::plain(A, st)
                            : RouteShape<T, 32, 32>::plain(A, st);
    return BY_WIDTH(T, forward, A.E, A, st);
}
template <typename T, int L>
int route_sparse(const RouteBackArgs &A, cudaStream_t st)
{
    constexpr int V = 16 / (int)sizeof(T);
    const bool v = (32 / L) * A.E % V == 0 && A.tokens * A.E % V == 0 && aligned(A.grad, 16);  // whole vectors per warp
    return launch_pdl(v ? route_backward_kernel<T, L, true> : route_backward_kernel<T, L, false>, route_grid(A.tokens, L), 32 * ROUTE_WARPS, 0,
                      st, A);
}
template <typename T>
int route_backward_t(const RouteBackArgs &A, cudaStream_t st)
{
    if (A.score == LAPSUM_ROUTE_SOFTMAX && !A.renorm) return BY_WIDTH(T, dense, A.E, A, st);
    return A.k <= 8 ? route_sparse<T, 8>(A, st) : A.k <= 16 ? route_sparse<T, 16>(A, st) : route_sparse<T, 32>(A, st);
}

// ---------------------------------------------------------------- dispatch ----
// chunks of neighbouring entries that one block works off, and the blocks that need
inline int64_t dispatch_chunks(int64_t entries)
{
    const int64_t chunks = (entries + DISPATCH_CHUNK - 1) / DISPATCH_CHUNK;
    return chunks <= DISPATCH_BLOCKS ? 1 : (chunks + DISPATCH_BLOCKS - 1) / DISPATCH_BLOCKS;
}
inline int64_t dispatch_blocks(int64_t entries)
{
    const int64_t per = dispatch_chunks(entries) * DISPATCH_CHUNK;
    return entries <= per ? 1 : (entries + per - 1) / per;
}
// More than 48 KB of a block's shared memory, its static part included, has to be asked for.  The kernel for over 256 experts asks for
// what 1024 of them need: the same value from every call, so that threads with different widths do not take it from one another.
int dispatch_allow_widest()
{
    static_assert(dispatch_place_smem(256) + 1024 <= 48 * 1024, "the narrower kernels' memory is given without asking");
    static thread_local int dev_ready = -1;  // the attribute belongs to the device's context
    int dev = 0;
    CU_OK(cudaGetDevice(&dev));
    if (dev != dev_ready) {
        CU_OK(cudaFuncSetAttribute(dispatch_place_kernel<10>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dispatch_place_smem(ROUTE_MAX_E)));
        dev_ready = dev;
    }
    return LAPSUM_OK;
}
int dispatch_layout(int64_t tokens, int32_t k, int64_t experts, int32_t rows, lapsum_dispatch_layout *L)
{
    if (tokens < 0 || k < 1 || k > ROUTE_MAX_K || experts < 1 || experts > ROUTE_MAX_E) return LAPSUM_ERR_SHAPE;
    if (rows != 16 && rows != 32 && rows != 64 && rows != 128 && rows != 256) return LAPSUM_ERR_PARAM;
    if (tokens > ((int64_t)1 << 30) / k) return LAPSUM_ERR_SHAPE;
    const int64_t entries = tokens * k;
    const int64_t used = entries < experts ? entries : experts;
    L->capacity = (entries + used * (rows - 1)) / rows * rows;
    L->tiles = L->capacity / rows;
    size_t at = 0;
    auto take = [&](size_t words) {
        const size_t o = at;
        at += align_up(4 * words);
        return o;
    };
    L->off_counts = take((size_t)experts);
    L->off_offsets = take((size_t)experts + 1);
    L->off_slot_of = take((size_t)entries);
    L->off_entry_of = take((size_t)L->capacity);
    L->off_tile_expert = take((size_t)L->tiles);
    L->off_partial = take((size_t)(dispatch_blocks(entries) * dispatch_stride((int)experts)));
    L->bytes = at;
    return LAPSUM_OK;
}

// ----------------------------------------------------------------- experts ----
struct ExpertsLayout {
    lapsum_dispatch_layout d;
    size_t off_slots, off_hw, off_dgu, off_partial, off_gu_saved, off_hw_saved;
    int nts_dh;    // column tiles of DH
    bool wide_dh;  // of 256 columns
};

// Columns of an output tile: 256, the most that two accumulators in TMEM allow; 128 where 256 would leave SMs without work (fewer
// than two tiles for each; pairs of blocks always take 256).  Measured: 48 tokens on 128 experts 210 us with 256 columns and 215 us with
// 128, eight experts' first product for one row tile each 43 us and 35 us, DH of 777 tokens on 24 experts 26 us and 19 us.
constexpr int MIN_TILES = 2 * 148;
inline bool wide_tiles(const lapsum_experts_dims *p, const lapsum_dispatch_layout &d, int64_t cols, bool gate_up)
{
    const int step = gate_up ? 128 : 256;
    return p->tile_rows == 256 || d.tiles * ((cols + step - 1) / step) >= MIN_TILES;
}

int experts_layout(const lapsum_experts_dims *p, ExpertsLayout &X, lapsum_experts_layout *out)
{
    if (!p) return LAPSUM_ERR_NULL;
    if (p->d < 8 || p->f < 8 || p->d % 8 || p->f % 8 || p->d > 1 << 16 || p->f > 1 << 16) return LAPSUM_ERR_SHAPE;
    if (p->io_dtype != LAPSUM_IO_F16 && p->io_dtype != LAPSUM_IO_BF16) return LAPSUM_ERR_UNSUPPORTED;
    if ((p->training != 0 && p->training != 1) || (p->grad_w_f32 != 0 && p->grad_w_f32 != 1)) return LAPSUM_ERR_PARAM;
    RUN(dispatch_layout(p->tokens, p->k, p->experts, p->tile_rows, &X.d));
    if (p->training && p->tile_rows < 64) return LAPSUM_ERR_PARAM;
    const size_t cap = (size_t)X.d.capacity, D = (size_t)p->d, F = (size_t)p->f;
    X.wide_dh = wide_tiles(p, X.d, p->f, false);
    X.nts_dh = (int)((p->f + (X.wide_dh ? 255 : 127)) / (X.wide_dh ? 256 : 128));
    size_t at = 256;  // control block: the status word
    X.off_slots = at, at += align_up(cap * D * 2);
    X.off_hw = at, at += p->training ? 0 : align_up(cap * F * 2);
    X.off_dgu = at, at += p->training ? align_up(cap * F * 4) : 0;
    X.off_partial = at, at += p->training ? align_up(cap * (size_t)X.nts_dh * 4) : 0;
    out->workspace_bytes = at;
    X.off_gu_saved = 0;
    X.off_hw_saved = align_up(cap * F * 4);
    out->saved_bytes = p->training ? X.off_hw_saved + align_up(cap * F * 2) : 0;
    return LAPSUM_OK;
}

using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
EncodeFn encode_fn()
{
    static const EncodeFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}

// dims from the innermost; strides in elements for dimensions 1..; 128-byte swizzle; reads beyond the tensor give zeros
int tensor_map(CUtensorMap *map, int dtype, const void *base, int rank, const int64_t *dims, const int64_t *strides, const int *box)
{
    const EncodeFn fn = encode_fn();
    if (!fn) return cuda_fail(cudaErrorNotSupported);
    cuuint64_t d[3], s[2];
    cuuint32_t b[3], one[3] = {1, 1, 1};
    for (int i = 0; i < rank; ++i) d[i] = (cuuint64_t)dims[i], b[i] = (cuuint32_t)box[i];
    for (int i = 0; i + 1 < rank; ++i) s[i] = (cuuint64_t)strides[i] * 2;
    const CUresult r = fn(map, dtype == LAPSUM_IO_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank,
                          const_cast<void *>(base), d, s, b, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? LAPSUM_OK : cuda_fail(cudaErrorInvalidValue);
}
int map_2d(CUtensorMap *m, int dtype, const void *base, int64_t cols, int64_t rows, int64_t stride, int box_rows)
{
    const int64_t d[2] = {cols, rows}, s[1] = {stride};
    const int b[2] = {64, box_rows};
    return tensor_map(m, dtype, base, 2, d, s, b);
}
int map_3d(CUtensorMap *m, int dtype, const void *base, int64_t cols, int64_t rows, int64_t depth, int box_rows)
{
    const int64_t d[3] = {cols, rows, depth}, s[2] = {cols, cols * rows};
    const int b[3] = {64, box_rows, 1};
    return tensor_map(m, dtype, base, 3, d, s, b);
}

// [slots][2][F]: g and u, or their gradients, 64 columns of one of the two
int map_gu(CUtensorMap *m, int dtype, const void *base, int64_t f, int64_t slots, int box_rows)
{
    const int64_t d[3] = {f, 2, slots}, s[2] = {f, 2 * f};
    const int b[3] = {64, 1, box_rows};
    return tensor_map(m, dtype, base, 3, d, s, b);
}

int sm_count(int *n)
{
    static thread_local int dev_known = -1, sms = 0;
    int dev = 0;
    CU_OK(cudaGetDevice(&dev));
    if (dev != dev_known) {
        CU_OK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        dev_known = dev;
    }
    *n = sms;
    return LAPSUM_OK;
}

template <int MODE, int AR, int BN, int KS, typename T>
int run_experts(const ExpertsMaps &maps, const ExpertsArgs &P, int64_t tiles_max, cudaStream_t st)
{
    using S = ExpertsShape<MODE, AR, BN, KS>;
    static thread_local int dev_ready = -1;  // the attribute belongs to the device's context
    int dev = 0, sms = 0;
    CU_OK(cudaGetDevice(&dev));
    RUN(sm_count(&sms));
    const auto kernel = experts_kernel<MODE, AR, BN, KS, T>;
    if (dev != dev_ready) {
        CU_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
        dev_ready = dev;
    }
    const int64_t units = S::PAIR ? sms / 2 : sms, n = tiles_max < 1 ? 1 : tiles_max < units ? tiles_max : units;
    return launch_clusters(S::PAIR ? 2 : 1, kernel, (unsigned)(S::PAIR ? 2 * n : n), S::THREADS, S::SMEM, st, maps, P);
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Call {
    const lapsum_experts_dims *p;
    ExpertsLayout X;
    lapsum_experts_layout out;
    ExpertsArgs A;
    uint8_t *ws;
};

int begin_call(const lapsum_experts_dims *p, const void *dispatch, size_t dispatch_bytes, void *ws, size_t ws_bytes, Call &c)
{
    RUN(experts_layout(p, c.X, &c.out));
    if (!dispatch || !ws) return LAPSUM_ERR_NULL;
    if (!aligned(ws, 256) || ws_bytes < c.out.workspace_bytes || !aligned(dispatch, 256) || dispatch_bytes < c.X.d.bytes)
        return LAPSUM_ERR_WORKSPACE;
    c.p = p;
    c.ws = static_cast<uint8_t *>(ws);
    const uint8_t *d = static_cast<const uint8_t *>(dispatch);
    std::memset(&c.A, 0, sizeof(c.A));
    c.A.entry_of = reinterpret_cast<const int32_t *>(d + c.X.d.off_entry_of);
    c.A.tile_expert = reinterpret_cast<const int32_t *>(d + c.X.d.off_tile_expert);
    c.A.offsets = reinterpret_cast<const int32_t *>(d + c.X.d.off_offsets);
    c.A.counts = reinterpret_cast<const int32_t *>(d + c.X.d.off_counts);
    c.A.status = reinterpret_cast<uint32_t *>(ws);
    c.A.wait_ns = 2000000000ull;
    c.A.row_tiles = (int)c.X.d.tiles;
    c.A.entries = (int)(p->tokens * p->k), c.A.capacity = (int)c.X.d.capacity;
    c.A.E = (int)p->experts, c.A.D = (int)p->d, c.A.F = (int)p->f, c.A.k = p->k, c.A.tokens = (int)p->tokens;
    return LAPSUM_OK;
}

// Up to four tokens the products run without the tensor core, which saves a launch and the tiles' prologue (some 9 us) but reads an
// expert's weights once for every token that chose it.  So only where that reads at most 48 MiB again, by the experts that so many
// tokens choose on average.  Measured, without / on tiles, us: one token on 8 of 64 experts of 2048 x 1024 27 / 37, 2: 44 / 52, 4: 74 / 75,
// 6: 105 / 88; on 8 of 8 one token 27 / 36, 2: 39 / 36, 4: 62 / 37; on 8 of 16 2: 42 / 48, 3: 55 / 49; 4 tokens on 2 of 4 experts of 1000 x 520
// 15 / 24.
constexpr int64_t FEW_TOKENS = 4, FEW_AGAIN = 48 << 20;
inline bool few_tokens(const lapsum_experts_dims &p)
{
    if (p.tokens > FEW_TOKENS) return false;
    const double entries = (double)p.tokens * p.k, E = (double)p.experts;
    const double chosen = E * (1.0 - std::pow(std::fmax(0.0, 1.0 - p.k / E), (double)p.tokens));
    return (entries - chosen) * 6.0 * (double)p.d * (double)p.f <= (double)FEW_AGAIN;
}

// One of the four products whose rows are slots
template <int MODE, typename T>
int run_rows(const Call &c, const ExpertsMaps &maps, const ExpertsArgs &P, int64_t cols, bool wide, cudaStream_t st)
{
    constexpr bool BACK = MODE == DH || MODE == DX;
    const int step = (wide ? 256 : 128) / (MODE == GATE_UP ? 2 : 1);
    const int64_t tiles = c.X.d.tiles * ceil_div(cols, step);
    switch (c.p->tile_rows) {
    case 256: return run_experts<MODE, 256, 256, 1, T>(maps, P, tiles, st);
    case 128: return wide ? run_experts<MODE, 128, 256, 1, T>(maps, P, tiles, st) : run_experts<MODE, 128, 128, 1, T>(maps, P, tiles, st);
    case 64: return wide ? run_experts<MODE, 64, 256, 1, T>(maps, P, tiles, st) : run_experts<MODE, 64, 128, 2, T>(maps, P, tiles, st);
    default: break;
    }
    if constexpr (!BACK) {
        if (c.p->tile_rows == 32)
            return wide ? run_experts<MODE, 32, 256, 1, T>(maps, P, tiles, st) : run_experts<MODE, 32, 128, 2, T>(maps, P, tiles, st);
        if (c.p->tile_rows == 16)
            return wide ? run_experts<MODE, 16, 256, 1, T>(maps, P, tiles, st) : run_experts<MODE, 16, 128, 2, T>(maps, P, tiles, st);
    }
    return LAPSUM_ERR_PARAM;
}
template <int MODE, typename T>
int run_weights(const Call &c, const ExpertsMaps &maps, int64_t m, int64_t n, cudaStream_t st)
{
    if (c.p->tile_rows == 256)
        return run_experts<MODE, 256, 256, 1, T>(maps, c.A, c.p->experts * ceil_div(m, 256) * ceil_div(n, 256), st);
    return run_experts<MODE, 128, 256, 1, T>(maps, c.A, c.p->experts * ceil_div(m, 128) * ceil_div(n, 256), st);
}

template <typename T>
int gather(const Call &c, const uint8_t *dispatch, const void *x, int64_t stride, bool holes, cudaStream_t st)
{
    const int64_t token_blocks = ceil_div(c.p->tokens * ceil_div(c.p->d, 1024), 8), hole_blocks = holes ? ceil_div(c.X.d.capacity, 32) : 0;
    return launch_pdl(experts_gather_kernel<T>, (unsigned)(token_blocks + hole_blocks), 256, 0, st, static_cast<const T *>(x), stride,
                      reinterpret_cast<const int32_t *>(dispatch + c.X.d.off_slot_of), c.A.entry_of, c.A.offsets + c.A.E,
                      reinterpret_cast<T *>(c.ws + c.X.off_slots), c.p->tokens, (int)token_blocks, c.A.capacity, (int)c.p->k, (int)c.p->d);
}

template <typename T>
int combine(const Call &c, const uint8_t *dispatch, void *out, int64_t stride, const float *partial, void *grad_w, cudaStream_t st)
{
    const int64_t work = c.p->tokens * (c.p->d / 8);
    return launch_pdl(experts_combine_kernel<T>, (unsigned)ceil_div(work, 256), 256, 0, st, reinterpret_cast<const T *>(c.ws + c.X.off_slots),
                      reinterpret_cast<const int32_t *>(dispatch + c.X.d.off_slot_of), static_cast<T *>(out), stride, partial,
                      grad_w, (int)c.p->grad_w_f32, c.p->tokens, c.A.capacity, (int)c.p->k, (int)c.p->d, c.X.nts_dh);
}

template <typename T>
int forward_t(Call &c, const void *x, int64_t x_stride, const void *w_gate_up, const void *w_down, const float *w, const uint8_t *dispatch,
              uint8_t *saved, void *y, int hold, cudaStream_t st)
{
    const lapsum_experts_dims &p = *c.p;
    const int dt = p.io_dtype, rows = p.tile_rows < 128 ? p.tile_rows : 128, out_rows = rows < 32 ? rows : 32;
    const int64_t cap = c.X.d.capacity;
    const bool pair = p.tile_rows == 256;
    if (!saved && !hold && few_tokens(p)) {
        const int32_t *slot_of = reinterpret_cast<const int32_t *>(dispatch + c.X.d.off_slot_of);
        T *hw = reinterpret_cast<T *>(c.ws + c.X.off_hw);
        int shift = 4;
        while ((1 << shift) < p.tile_rows) ++shift;
        RUN(launch_pdl(experts_few_gate_up_kernel<T>, dim3((unsigned)ceil_div(p.f, FEW_FEATURES), (unsigned)(p.tokens * p.k)), 256, 0, st,
                       static_cast<const T *>(x), x_stride, static_cast<const T *>(w_gate_up), w, slot_of, c.A.tile_expert, shift, c.A.capacity, c.A.E, hw, (int)p.k,
                       (int)p.d, (int)p.f));
        return launch_pdl(experts_few_down_kernel<T>, dim3((unsigned)(p.d / 4), (unsigned)p.tokens), 256, 0, st, static_cast<const T *>(w_down),
                          hw, slot_of, c.A.tile_expert, shift, c.A.capacity, c.A.E, static_cast<T *>(y), (int)p.k, (int)p.d, (int)p.f);
    }
    uint8_t *rowbuf = c.ws + c.X.off_slots;  // in turn: x in slot order, the second product's results
    void *hw = saved ? saved + c.X.off_hw_saved : c.ws + c.X.off_hw;
    ExpertsMaps m;
    if (rows > GATHER_ROWS) {
        if (!hold) RUN(gather<T>(c, dispatch, x, x_stride, false, st));
        RUN(map_2d(&m.a, dt, rowbuf, p.d, cap, p.d, rows));
    } else {
        RUN(map_2d(&m.a, dt, x, p.d, p.tokens, x_stride, 1));
    }
    bool wide = wide_tiles(&p, c.X.d, p.f, true);
    RUN(map_3d(&m.b, dt, w_gate_up, p.d, p.f, 2 * p.experts, wide ? 128 : 64));
    RUN(map_2d(&m.out, dt, hw, p.f, cap, p.f, out_rows));
    if (saved) RUN(map_gu(&m.gu, dt, saved + c.X.off_gu_saved, p.f, cap, out_rows));
    else m.gu = m.out;  // not used
    ExpertsArgs A = c.A;
    A.w = w;
    A.keep = saved != nullptr;
    A.hold = hold;
    A.early = rows > GATHER_ROWS && !hold;  // the gather came between
    RUN((run_rows<GATE_UP, T>(c, m, A, p.f, wide, st)));
    if (hold) return LAPSUM_OK;

    wide = wide_tiles(&p, c.X.d, p.d, false);
    RUN(map_2d(&m.a, dt, hw, p.f, cap, p.f, rows));
    RUN(map_3d(&m.b, dt, w_down, p.f, p.d, p.experts, wide && !pair ? 256 : 128));
    RUN(map_2d(&m.out, dt, rowbuf, p.d, cap, p.d, out_rows));
    A = c.A;
    A.early = 1;
    RUN((run_rows<DOWN, T>(c, m, A, p.d, wide, st)));
    return combine<T>(c, dispatch, y, p.d, nullptr, nullptr, st);
}

template <typename T>
int backward_t(Call &c, const void *grad_y, int64_t gy_stride, const void *x, int64_t x_stride, const void *w_gate_up, const void *w_down,
               const float *w, const uint8_t *dispatch, const uint8_t *saved, void *grad_x, void *grad_w_gate_up, void *grad_w_down,
               void *grad_w, cudaStream_t st)
{
    const lapsum_experts_dims &p = *c.p;
    const int dt = p.io_dtype, rows = p.tile_rows < 128 ? p.tile_rows : 128;
    const int64_t cap = c.X.d.capacity;
    const uint8_t *hw = saved + c.X.off_hw_saved;
    uint8_t *dgu = c.ws + c.X.off_dgu;
    float *partial = reinterpret_cast<float *>(c.ws + c.X.off_partial);
    void *rowbuf = c.ws + c.X.off_slots;  // in turn: grad_y in slot order, x in slot order, grad_x per slot
    ExpertsMaps m;
    RUN(gather<T>(c, dispatch, grad_y, gy_stride, true, st));
    RUN(map_2d(&m.a, dt, rowbuf, p.d, cap, p.d, rows));
    RUN(map_3d(&m.b, dt, w_down, p.f, p.d, p.experts, 64));
    RUN(map_gu(&m.out, dt, dgu, p.f, cap, 32));
    RUN(map_gu(&m.gu, dt, saved + c.X.off_gu_saved, p.f, cap, 32));
    ExpertsArgs A = c.A;
    A.w = w, A.partial = partial, A.early = 1;
    RUN((run_rows<DH, T>(c, m, A, p.f, c.X.wide_dh, st)));

    RUN(map_2d(&m.a, dt, rowbuf, p.d, cap, p.d, 64));
    RUN(map_2d(&m.b, dt, hw, p.f, cap, p.f, 64));
    RUN(map_3d(&m.out, dt, grad_w_down, p.f, p.d, p.experts, 32));
    RUN((run_weights<DW_DOWN, T>(c, m, p.d, p.f, st)));

    RUN(gather<T>(c, dispatch, x, x_stride, true, st));
    RUN(map_2d(&m.a, dt, dgu, 2 * p.f, cap, 2 * p.f, 64));
    RUN(map_2d(&m.b, dt, rowbuf, p.d, cap, p.d, 64));
    RUN(map_3d(&m.out, dt, grad_w_gate_up, p.d, 2 * p.f, p.experts, 32));
    RUN((run_weights<DW_GATE_UP, T>(c, m, 2 * p.f, p.d, st)));

    RUN(map_2d(&m.a, dt, dgu, 2 * p.f, cap, 2 * p.f, rows));
    RUN(map_3d(&m.b, dt, w_gate_up, p.d, 2 * p.f, p.experts, 64));
    RUN(map_2d(&m.out, dt, rowbuf, p.d, cap, p.d, 32));
    A = c.A;
    A.early = 1;
    RUN((run_rows<DX, T>(c, m, A, p.d, wide_tiles(&p, c.X.d, p.d, false), st)));
    return combine<T>(c, dispatch, grad_x, p.d, partial, grad_w, st);
}

}  // namespace

extern "C" {

void lapsum_route_default_params(lapsum_route_params *p)
{
    if (!p) return;
    std::memset(p, 0, sizeof(*p));
    p->scale = 1.0;
    p->score = LAPSUM_ROUTE_SOFTMAX;
    p->k = p->groups = p->groups_kept = 1;
    p->group_top = 2;
    p->renormalise = 1;
    p->io_dtype = p->grad_w_dtype = LAPSUM_IO_F32;
}

int lapsum_route_forward(const void *logits, int64_t tokens, int64_t experts, int64_t stride, const float *bias,
                         const lapsum_route_params *prm, int32_t *idx, float *w, void *stream)
{
    RUN(route_check(tokens, experts, stride, prm));
    if (tokens == 0) return LAPSUM_OK;
    if (!logits || !idx || !w) return LAPSUM_ERR_NULL;
    const RouteArgs A{logits, bias, idx, w, tokens, stride, (int)experts, prm->k, prm->groups, prm->groups_kept, prm->group_top,
                      prm->score, prm->renormalise != 0, experts % 4 == 0 && aligned(bias, 16), (float)prm->scale};
    return BY_TYPE(route_forward_t, prm->io_dtype, A, static_cast<cudaStream_t>(stream));
}

int lapsum_route_backward(const void *grad_w, const void *logits, int64_t tokens, int64_t experts, int64_t stride, const int32_t *idx,
                          const float *w, const lapsum_route_params *prm, void *grad_logits, void *stream)
{
    RUN(route_check(tokens, experts, stride, prm));
    if (tokens == 0) return LAPSUM_OK;
    if (!grad_w || !logits || !idx || !w || !grad_logits) return LAPSUM_ERR_NULL;
    const RouteBackArgs A{grad_w, logits, idx, w, grad_logits, tokens, stride, (int)experts, prm->k, prm->score, prm->renormalise != 0,
                          prm->grad_w_dtype, (float)prm->scale};
    return BY_TYPE(route_backward_t, prm->io_dtype, A, static_cast<cudaStream_t>(stream));
}

int lapsum_dispatch_tile_rows(int64_t tokens, int32_t k, int64_t experts, int32_t training, int32_t *rows)
{
    if (!rows) return LAPSUM_ERR_NULL;
    if (tokens < 0 || k < 1 || k > ROUTE_MAX_K || experts < 1 || experts > ROUTE_MAX_E) return LAPSUM_ERR_SHAPE;
    const double mean = (double)tokens * k / (double)experts;  // entries per expert
    *rows = mean > 384 ? 256 : mean > 48 ? 128 : mean > 24 || training ? 64 : mean > 8 ? 32 : 16;
    return LAPSUM_OK;
}

int lapsum_dispatch_describe(int64_t tokens, int32_t k, int64_t experts, int32_t tile_rows, lapsum_dispatch_layout *out)
{
    if (!out) return LAPSUM_ERR_NULL;
    return dispatch_layout(tokens, k, experts, tile_rows, out);
}

int lapsum_dispatch(const int32_t *idx, int64_t tokens, int32_t k, int64_t experts, int32_t tile_rows, void *dispatch, size_t bytes,
                    void *stream)
{
    lapsum_dispatch_layout L;
    RUN(dispatch_layout(tokens, k, experts, tile_rows, &L));
    if ((!idx && tokens > 0) || !dispatch) return LAPSUM_ERR_NULL;
    if (!aligned(dispatch, 256) || bytes < L.bytes) return LAPSUM_ERR_WORKSPACE;
    uint8_t *d = static_cast<uint8_t *>(dispatch);
    DispatchArgs A;
    A.idx = idx;
    A.entries = tokens * k, A.capacity = L.capacity;
    A.E = (int)experts, A.rows = tile_rows;
    A.chunks = (int)dispatch_chunks(A.entries), A.blocks = (int)dispatch_blocks(A.entries);
    const auto place = experts <= 128 ? dispatch_place_kernel<7> : experts <= 256 ? dispatch_place_kernel<8> : dispatch_place_kernel<10>;
    const size_t smem = dispatch_place_smem((int)experts);
    if (experts > 256) RUN(dispatch_allow_widest());
    A.counts = reinterpret_cast<int32_t *>(d + L.off_counts), A.offsets = reinterpret_cast<int32_t *>(d + L.off_offsets);
    A.slot_of = reinterpret_cast<int32_t *>(d + L.off_slot_of), A.entry_of = reinterpret_cast<int32_t *>(d + L.off_entry_of);
    A.tile_expert = reinterpret_cast<int32_t *>(d + L.off_tile_expert), A.partial = reinterpret_cast<int32_t *>(d + L.off_partial);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (A.blocks > 1) RUN(launch_pdl(dispatch_count_kernel, (unsigned)A.blocks, DISPATCH_THREADS, 4 * (size_t)dispatch_stride((int)experts), st, A));
    A.shift = 4;
    while ((1 << A.shift) < tile_rows) ++A.shift;
    return launch_pdl(place, (unsigned)A.blocks, DISPATCH_THREADS, smem, st, A);
}

int lapsum_experts_describe(const lapsum_experts_dims *dims, lapsum_experts_layout *out)
{
    if (!out) return LAPSUM_ERR_NULL;
    ExpertsLayout X;
    return experts_layout(dims, X, out);
}

int lapsum_experts_workspace_init(void *ws, size_t bytes, const lapsum_experts_dims *dims, void *stream)
{
    ExpertsLayout X;
    lapsum_experts_layout out;
    RUN(experts_layout(dims, X, &out));
    if (!ws) return LAPSUM_ERR_NULL;
    if (!aligned(ws, 256) || bytes < out.workspace_bytes) return LAPSUM_ERR_WORKSPACE;
    CU_OK(cudaMemsetAsync(ws, 0, 256, static_cast<cudaStream_t>(stream)));
    return LAPSUM_OK;
}

int lapsum_experts_status(void *ws, void *stream, uint32_t *status_bits)
{
    if (!ws || !status_bits) return LAPSUM_ERR_NULL;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    CU_OK(cudaMemcpyAsync(status_bits, ws, sizeof(uint32_t), cudaMemcpyDeviceToHost, st));
    CU_OK(cudaStreamSynchronize(st));
    return LAPSUM_OK;
}

int lapsum_experts_forward(const void *x, int64_t x_stride, const void *w_gate_up, const void *w_down, const float *w,
                           const void *dispatch, size_t dispatch_bytes, void *saved, size_t saved_bytes, void *y,
                           const lapsum_experts_dims *dims, void *ws, size_t ws_bytes, void *stream)
{
    Call c;
    RUN(begin_call(dims, dispatch, dispatch_bytes, ws, ws_bytes, c));
    if (dims->tokens == 0) return LAPSUM_OK;
    if (dims->training && !saved) return LAPSUM_ERR_NULL;
    if (!dims->training && saved) return LAPSUM_ERR_PARAM;
    if (saved && (!aligned(saved, 256) || saved_bytes < c.out.saved_bytes)) return LAPSUM_ERR_WORKSPACE;
    if (x_stride < dims->d || x_stride % 8) return LAPSUM_ERR_SHAPE;
    if (!x || !w_gate_up || !w_down || !w || !y) return LAPSUM_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w_gate_up, 16) || !aligned(w_down, 16) || !aligned(y, 16)) return LAPSUM_ERR_ALIGN;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const uint8_t *d = static_cast<const uint8_t *>(dispatch);
    uint8_t *s = static_cast<uint8_t *>(saved);
    return dims->io_dtype == LAPSUM_IO_BF16 ? forward_t<__nv_bfloat16>(c, x, x_stride, w_gate_up, w_down, w, d, s, y, 0, st)
                                            : forward_t<__half>(c, x, x_stride, w_gate_up, w_down, w, d, s, y, 0, st);
}

int lapsum_experts_backward(const void *grad_y, int64_t grad_y_stride, const void *x, int64_t x_stride, const void *w_gate_up,
                            const void *w_down, const float *w, const void *dispatch, size_t dispatch_bytes, const void *saved,
                            size_t saved_bytes, void *grad_x, void *grad_w_gate_up, void *grad_w_down, void *grad_w,
                            const lapsum_experts_dims *dims, void *ws, size_t ws_bytes, void *stream)
{
    Call c;
    RUN(begin_call(dims, dispatch, dispatch_bytes, ws, ws_bytes, c));
    if (!dims->training) return LAPSUM_ERR_UNSUPPORTED;
    if (!grad_w_gate_up || !grad_w_down) return LAPSUM_ERR_NULL;
    if (!aligned(grad_w_gate_up, 16) || !aligned(grad_w_down, 16)) return LAPSUM_ERR_ALIGN;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dims->tokens == 0) {  // no token: every weight's gradient is zero
        const size_t bytes = (size_t)dims->experts * (size_t)dims->d * (size_t)dims->f * 2;
        CU_OK(cudaMemsetAsync(grad_w_gate_up, 0, 2 * bytes, st));
        CU_OK(cudaMemsetAsync(grad_w_down, 0, bytes, st));
        return LAPSUM_OK;
    }
    if (!saved) return LAPSUM_ERR_NULL;
    if (!aligned(saved, 256) || saved_bytes < c.out.saved_bytes) return LAPSUM_ERR_WORKSPACE;
    if (x_stride < dims->d || x_stride % 8 || grad_y_stride < dims->d || grad_y_stride % 8) return LAPSUM_ERR_SHAPE;
    if (!grad_y || !x || !w_gate_up || !w_down || !w || !grad_x || !grad_w) return LAPSUM_ERR_NULL;
    if (!aligned(grad_y, 16) || !aligned(x, 16) || !aligned(w_gate_up, 16) || !aligned(w_down, 16) || !aligned(grad_x, 16))
        return LAPSUM_ERR_ALIGN;
    const uint8_t *d = static_cast<const uint8_t *>(dispatch), *s = static_cast<const uint8_t *>(saved);
    return dims->io_dtype == LAPSUM_IO_BF16
               ? backward_t<__nv_bfloat16>(c, grad_y, grad_y_stride, x, x_stride, w_gate_up, w_down, w, d, s, grad_x, grad_w_gate_up,
                                           grad_w_down, grad_w, st)
               : backward_t<__half>(c, grad_y, grad_y_stride, x, x_stride, w_gate_up, w_down, w, d, s, grad_x, grad_w_gate_up, grad_w_down,
                                    grad_w, st);
}

int lapsum_debug_experts_timeout(int64_t wait_us, void *ws, size_t ws_bytes, const void *dispatch, size_t dispatch_bytes, const void *x,
                                 const void *w_gate_up, const float *w, const lapsum_experts_dims *dims, void *stream)
{
    Call c;
    RUN(begin_call(dims, dispatch, dispatch_bytes, ws, ws_bytes, c));
    if (!x || !w_gate_up || !w) return LAPSUM_ERR_NULL;
    if (dims->tokens < 1 || dims->training || dims->io_dtype != LAPSUM_IO_BF16) return LAPSUM_ERR_UNSUPPORTED;
    if (wait_us < 1 || wait_us > 100000) return LAPSUM_ERR_PARAM;
    if (!aligned(x, 16) || !aligned(w_gate_up, 16)) return LAPSUM_ERR_ALIGN;
    c.A.wait_ns = (unsigned long long)wait_us * 1000;
    return forward_t<__nv_bfloat16>(c, x, dims->d, w_gate_up, nullptr, w, static_cast<const uint8_t *>(dispatch), nullptr, nullptr, 1,
                                    static_cast<cudaStream_t>(stream));
}

}  // extern "C"
