// Embedding: rows of a table by token id, and the table's gradient by sorted ids.
//
//   forward    out_i = scale E[id_i]
//   backward   dE[v] = scale sum of dout_i over id_i = v, every row written
//
// The gradient in three kernels: a stable sort of the positions by id (embed_sort_kernel), the sums of all rows with few positions and
// partial sums of pieces of the others (embed_grad_kernel), the sums of the pieces (embed_join_kernel).  Every sum has a fixed order.
//
// Measured: 65536 ids into 128000 x 2048 bf16: forward 65 us (380 MB, 5.8 TB/s); gradient in fp32 324 us: sort 35, sums 261 (1.32 GB, most of it the zeros of rows
// that do not occur, 5.0 TB/s), pieces 12; in bf16 245.  4093 ids into 50021 x 1000 fp16: 10 and 42 us (100 MB of zeros take 16), three dependent kernels.
#pragma once
#include <type_traits>

#include "common.cuh"

namespace lapsum {

struct EmbedArgs {
    const void *ids;
    int wide_ids;             // ids are int64
    int64_t tokens, vocab, d;
    int64_t skip;             // an id that adds nothing, or -1
    const void *table, *grad_out;
    int64_t table_stride, out_stride, grad_stride;
    void *out, *grad;
    float scale;
    int grad_f32;
    int64_t chunk_blocks;
    // workspace
    int32_t *row_start;       // [vocab + 1]: first sorted position of every id
    int32_t *order;           // [tokens]: positions, by id, then by position
    uint32_t *long_count;     // rows with more than EMBED_LONG positions
    int32_t *long_rows;
    float *partial;           // [chunks][2][partial_stride]
    int64_t partial_stride;   // d, rounded up to whole vectors
};

// Rows of more than EMBED_LONG positions are summed in pieces: runs of EMBED_LONG sorted positions (chunks) cut them.  A warp takes four positions at
// a time, so this bounds its longest chain.  16 / 32, us: 4093 ids into 50021 x 1000 42 / 53, 65536 into 128000 x 2048 324 / 314.
constexpr int EMBED_LONG = 16;
// Ids that one block of the sort takes care of, and its warps
constexpr int EMBED_RANGE = 512, EMBED_WARPS = 32;

__device__ __forceinline__ int64_t embed_id(const EmbedArgs &P, int64_t i)
{
    return P.wide_ids ? ld(static_cast<const int64_t *>(P.ids) + i) : (int64_t)ld(static_cast<const int32_t *>(P.ids) + i);
}

// A warp per row and 32 x N accesses of W values.  W: values per access, 16 bytes' or one.
template <typename T, bool VEC>
struct EmbedShape {
    static constexpr int W = VEC ? Io<T>::V : 1, N = VEC ? 2 : 8, SPAN = 32 * N * W;  // columns of a warp
    using Raw = typename std::conditional<VEC, typename Io<T>::Vec, T>::type;
    static __device__ __forceinline__ Raw fetch(const T *p) { return ld(reinterpret_cast<const Raw *>(p)); }
    static __device__ __forceinline__ void unpack(const Raw &q, float (&x)[W])
    {
        if constexpr (VEC) Io<T>::unpack(q, x);
        else x[0] = Io<T>::from_storage(q);
    }
    static __device__ __forceinline__ void load(const T *p, float (&x)[W]) { unpack(fetch(p), x); }
    static __device__ __forceinline__ void store(T *p, const float (&x)[W])
    {
        if constexpr (VEC) __stcs(reinterpret_cast<typename Io<T>::Vec *>(p), Io<T>::pack(x));  // read by a later kernel at the earliest
        else Io<T>::store1(p, x[0]);
    }
    static __device__ __forceinline__ void store_f32(float *p, const float (&x)[W])
    {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < W; i += 4) __stcs(reinterpret_cast<float4 *>(p + i), make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]));
        } else {
            p[0] = x[0];
        }
    }
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) embed_forward_kernel(const EmbedArgs P)
{
    using E = EmbedShape<T, VEC>;
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t parts = (P.d + E::SPAN - 1) / E::SPAN, unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), i = unit / parts;
    if (i >= P.tokens) return;
    const int c0 = (int)(unit - i * parts) * E::SPAN + lane * E::W, d = (int)P.d;
    const int64_t id = embed_id(P, i);
    const bool real = (uint64_t)id < (uint64_t)P.vocab;
    const T *const from = static_cast<const T *>(P.table) + (real ? id : 0) * P.table_stride;
    T *const to = static_cast<T *>(P.out) + i * P.out_stride;
    float x[E::N][E::W] = {};
#pragma unroll
    for (int j = 0; j < E::N; ++j)
        if (real && c0 + 32 * j * E::W < d) E::load(from + c0 + 32 * j * E::W, x[j]);
#pragma unroll
    for (int j = 0; j < E::N; ++j)
        if (c0 + 32 * j * E::W < d) {
#pragma unroll
            for (int v = 0; v < E::W; ++v) x[j][v] = real ? x[j][v] * P.scale : 0.f;
            E::store(to + c0 + 32 * j * E::W, x[j]);
        }
}

// A block has EMBED_RANGE neighbouring ids and reads all of them: it counts, per warp (a run of positions) and id, and how many ids lie below its
// range, which is where its part of the order begins; then it reads them again and puts its positions where the counts say.  No
// block waits for another.  Bound by instructions, some eight per id in every block: 35 us for 65536 ids and 250 blocks, with 64-bit comparisons 59.
template <typename Id>
__global__ void __launch_bounds__(32 * EMBED_WARPS) embed_sort_kernel(const EmbedArgs P)
{
    extern __shared__ int32_t counts[];  // [EMBED_WARPS][EMBED_RANGE]
    __shared__ int32_t start[EMBED_RANGE], warp_total_of[EMBED_WARPS], below_of[EMBED_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < EMBED_WARPS * EMBED_RANGE; i += 32 * EMBED_WARPS) counts[i] = 0;
    pdl_wait();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (blockIdx.x == 0 && tid == 0) *P.long_count = 0;
    __syncthreads();
    // vocab and tokens are below 2^31, so one unsigned comparison tells whether an id is in the range
    const uint32_t lo = blockIdx.x * (uint32_t)EMBED_RANGE, range = min((uint32_t)EMBED_RANGE, (uint32_t)P.vocab - lo);
    const uint32_t skip = (uint64_t)P.skip < (uint64_t)P.vocab ? (uint32_t)P.skip : 0xffffffffu;
    const int per = (int)((P.tokens + 32 * EMBED_WARPS - 1) / (32 * EMBED_WARPS) * 32), w0 = (int)min((int64_t)warp * per, P.tokens),
              w1 = (int)min((int64_t)w0 + per, P.tokens);
    int32_t *const mine = counts + warp * EMBED_RANGE;
    // eight ids of a lane, 32 apart: all loads at once.  0xffffffff: beyond the end, or an int64 that is no id
    const auto ids_at = [&](int i, uint32_t (&id)[8]) {
        const Id *const from = static_cast<const Id *>(P.ids) + i;
        Id raw[8];
        if (i - lane + 256 <= w1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) raw[j] = ld(from + 32 * j);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) raw[j] = i + 32 * j < w1 ? ld(from + 32 * j) : (Id)-1;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) id[j] = sizeof(Id) == 4 || (uint64_t)raw[j] < 0x80000000ull ? (uint32_t)raw[j] : 0xffffffffu;
    };
    int below = 0;
    for (int i = w0 + lane; i - lane < w1; i += 32 * 8) {
        uint32_t id[8];
        ids_at(i, id);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            below += id[j] < lo && id[j] != skip;
            if (id[j] - lo < range && id[j] != skip) atomicAdd(mine + (id[j] - lo), 1);
        }
    }
    below = (int)warp_sum((long long)below);
    if (lane == 0) below_of[warp] = below;
    __syncthreads();
    // per id: the warps' counts become offsets; then the ids' totals become starts
    int total = 0;
    if (tid < EMBED_RANGE)
        for (int w = 0; w < EMBED_WARPS; ++w) {
            const int c = counts[w * EMBED_RANGE + tid];
            counts[w * EMBED_RANGE + tid] = total;
            total += c;
        }
    int upto = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int b = __shfl_up_sync(FULL, upto, o);
        if (lane >= o) upto += b;
    }
    if (lane == 31) warp_total_of[warp] = upto;
    __syncthreads();
    int base = 0;
    for (int w = 0; w < EMBED_WARPS; ++w) base += below_of[w] + (w < warp ? warp_total_of[w] : 0);
    if (tid < EMBED_RANGE) {
        start[tid] = base + upto - total;
        if ((uint32_t)tid < range) P.row_start[lo + tid] = base + upto - total;
        if ((uint32_t)tid == range - 1 && (int64_t)lo + range == P.vocab) P.row_start[P.vocab] = base + upto;
    }
    __syncthreads();
    for (int i0 = w0; i0 < w1; i0 += 32 * 8) {
        uint32_t id[8];
        ids_at(i0 + lane, id);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = id[j] - lo < range && id[j] != skip;
            const unsigned any = __ballot_sync(FULL, in);
            if (any == 0) continue;
            if (in) {
                const int at = (int)(id[j] - lo);
                const unsigned peers = __match_any_sync(any, at);
                const int before = mine[at];
                __syncwarp(any);
                const int to = start[at] + before + __popc(peers & ((1u << lane) - 1));
                if (to < P.tokens) P.order[to] = (int32_t)(i0 + 32 * j + lane);  // beyond only if the ids changed meanwhile
                if (lane == __ffs(peers) - 1) mine[at] = before + __popc(peers);
            }
            __syncwarp();
        }
    }
}

// Adds rows of grad_out, those at order[first .. last), to `sum`, four rows' loads at once; a warp, its columns from c0 on.  before(i) comes before the row of
// position i is added.
template <typename T, bool VEC, typename F>
__device__ __forceinline__ void embed_sum(const EmbedArgs &P, int first, int last, int c0, float (&sum)[EmbedShape<T, VEC>::N][EmbedShape<T, VEC>::W],
                                          F before)
{
    using E = EmbedShape<T, VEC>;
    const int lane = threadIdx.x & 31, d = (int)P.d;
    const T *const g = static_cast<const T *>(P.grad_out) + c0;
    for (int b = first; b < last; b += 32) {
        const int pos = b + lane < last ? ld(P.order + b + lane) : 0, n = min(32, last - b);
        for (int e = 0; e < n; e += 4) {
            typename E::Raw q[4][E::N];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const T *const row = g + (int64_t)__shfl_sync(FULL, pos, min(e + k, n - 1)) * P.grad_stride;
#pragma unroll
                for (int j = 0; j < E::N; ++j)
                    if (e + k < n && c0 + 32 * j * E::W < d) q[k][j] = E::fetch(row + 32 * j * E::W);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (e + k >= n) break;
                before(b + e + k);
#pragma unroll
                for (int j = 0; j < E::N; ++j)
                    if (c0 + 32 * j * E::W < d) {
                        float x[E::W];
                        E::unpack(q[k][j], x);
#pragma unroll
                        for (int v = 0; v < E::W; ++v) sum[j][v] += x[v];
                    }
            }
        }
    }
}

// The first blocks have a chunk of sorted positions and a run of columns per warp: the piece of the long row that reaches into the chunk from
// before (or starts with it), and the piece of the one that goes on behind it.  The others have EMBED_ROWS neighbouring rows of the table and a run of
// columns per warp: zeros, or the sum over a row's few positions; neighbouring rows' positions lie side by side, so where they are is two loads for all.
constexpr int EMBED_ROWS = 8;
template <typename T, bool VEC>
__global__ void __launch_bounds__(256, 3) embed_grad_kernel(const EmbedArgs P)
{
    using E = EmbedShape<T, VEC>;
    pdl_wait();
    if (P.tokens > EMBED_LONG) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // otherwise the last of its call
    const int lane = threadIdx.x & 31, d = (int)P.d;
    const int64_t parts = (P.d + E::SPAN - 1) / E::SPAN;
    int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    float sum[E::N][E::W] = {};
    if ((int64_t)blockIdx.x < P.chunk_blocks) {
        const int64_t chunk = unit / parts;
        const int part = (int)(unit - chunk * parts), c0 = part * E::SPAN + lane * E::W;
        const int all = ld(P.row_start + P.vocab);
        const int first = (int)(chunk * EMBED_LONG), end = min(first + EMBED_LONG, all);
        if (chunk * EMBED_LONG >= all) return;
        const int64_t v[2] = {embed_id(P, ld(P.order + first)), embed_id(P, ld(P.order + end - 1))};
#pragma unroll 1
        for (int s = 0; s < 2; ++s) {
            if ((uint64_t)v[s] >= (uint64_t)P.vocab) continue;  // only if the ids changed meanwhile
            const int r0 = ld(P.row_start + v[s]), r1 = ld(P.row_start + v[s] + 1);
            if (r1 - r0 <= EMBED_LONG || (s == 1 && v[1] == v[0])) continue;
#pragma unroll
            for (int j = 0; j < E::N; ++j)
#pragma unroll
                for (int i = 0; i < E::W; ++i) sum[j][i] = 0.f;
            embed_sum<T, VEC>(P, max(r0, first), min(r1, end), c0, sum, [](int) {});
            float *const out = P.partial + (2 * chunk + s) * P.partial_stride + c0;
#pragma unroll
            for (int j = 0; j < E::N; ++j)
                if (c0 + 32 * j * E::W < d) E::store_f32(out + 32 * j * E::W, sum[j]);
            if (part == 0 && lane == 0 && r0 >= first) P.long_rows[atomicAdd(P.long_count, 1u)] = (int32_t)v[s];  // the row starts here
        }
        return;
    }
    unit -= 8 * P.chunk_blocks;
    const int64_t v0 = unit / parts * EMBED_ROWS;
    if (v0 >= P.vocab) return;
    const int c0 = (int)(unit % parts) * E::SPAN + lane * E::W, rows = (int)min((int64_t)EMBED_ROWS, P.vocab - v0);
    const int start = ld(P.row_start + v0 + min(lane, rows)), next = __shfl_down_sync(FULL, start, 1);
    const unsigned is_long = __ballot_sync(FULL, lane < rows && next - start > EMBED_LONG);
    const auto flush = [&](int row) {
#pragma unroll
        for (int j = 0; j < E::N; ++j)
            if (c0 + 32 * j * E::W < d) {
#pragma unroll
                for (int i = 0; i < E::W; ++i) sum[j][i] *= P.scale;
                const int64_t at = (v0 + row) * P.d + c0 + 32 * j * E::W;
                if (P.grad_f32) E::store_f32(static_cast<float *>(P.grad) + at, sum[j]);
                else E::store(static_cast<T *>(P.grad) + at, sum[j]);
#pragma unroll
                for (int i = 0; i < E::W; ++i) sum[j][i] = 0.f;
            }
    };
    for (int row = 0; row < rows;) {
        if (is_long >> row & 1) {
            ++row;
            continue;
        }
        const unsigned behind = is_long >> row;
        const int stop = behind ? row + __ffs(behind) - 1 : rows;  // the next long row
        int end = __shfl_sync(FULL, start, row + 1);
        embed_sum<T, VEC>(P, __shfl_sync(FULL, start, row), __shfl_sync(FULL, start, stop), c0, sum, [&](int i) {
            while (i >= end && row + 1 < stop) {
                flush(row++);
                end = __shfl_sync(FULL, start, row + 1);
            }
        });
        for (; row < stop; ++row) flush(row);
    }
}

// A block has a long row and 128 columns: its warps have runs of the pieces, and their sums are added in order.  Which row a block finds in the
// list depends on scheduling, what it computes does not.
template <typename T>
__global__ void __launch_bounds__(256) embed_join_kernel(const EmbedArgs P)
{
    pdl_wait();
    __shared__ float4 part[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t parts = (P.d + 127) / 128, units = (int64_t)ld(P.long_count) * parts;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int64_t v = ld(P.long_rows + unit / parts), c = unit % parts * 128 + 4 * lane;
        const int r0 = ld(P.row_start + v), r1 = ld(P.row_start + v + 1);
        const int first = r0 / EMBED_LONG, last = (r1 - 1) / EMBED_LONG, n = last - first + 1, each = (n + 7) / 8;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < P.d) {
#pragma unroll 4
            for (int i = warp * each; i < min(n, (warp + 1) * each); ++i) {
                const int64_t slot = 2 * (int64_t)(first + i) + (i == 0 && r0 % EMBED_LONG != 0 ? 1 : 0);
                const float4 q = ld(reinterpret_cast<const float4 *>(P.partial + slot * P.partial_stride + c));  // beyond d: nobody's, not stored
                sum.x += q.x, sum.y += q.y, sum.z += q.z, sum.w += q.w;
            }
        }
        part[warp][lane] = sum;
        __syncthreads();
        if (warp < 4) {  // a warp per 32 columns, a column per lane
            const int64_t at = unit % parts * 128 + 32 * warp + lane;
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += reinterpret_cast<const float *>(part[i])[32 * warp + lane];
            s *= P.scale;
            if (at < P.d) {
                if (P.grad_f32) static_cast<float *>(P.grad)[v * P.d + at] = s;
                else Io<T>::store1(static_cast<T *>(P.grad) + v * P.d + at, s);
            }
        }
        __syncthreads();
    }
}

}  // namespace lapsum
