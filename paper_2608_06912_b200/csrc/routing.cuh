// Routing of tokens to experts and the dispatch tables that bring every expert's tokens side by side.
//
// route    one warp per token, the token's E logits in registers (E <= 1024: 32 per lane).
//          keys   c_i = l_i (softmax or sigmoid without a bias: both rise with the logit), else s_i + bias_i
//          groups the `kept` groups with the largest sum of their best `group_top` keys keep their experts
//          choice k largest keys, ties to the lower index; weights from the scores s, never from the bias
// dispatch a stable counting sort of the T k entries by expert, integers only.
#pragma once
#include "common.cuh"

namespace lapsum {

constexpr int ROUTE_MAX_E = 1024, ROUTE_MAX_K = 32, ROUTE_MAX_GROUPS = 32;
constexpr int ROUTE_WARPS = 8;  // tokens per block

struct RouteArgs {
    const void *logits;
    const float *bias;
    int32_t *idx;
    float *w;
    int64_t tokens, stride;
    int E, k, groups, kept, top, score, renorm;
    float scale;
};

__device__ __forceinline__ float warp_sum_f(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}
__device__ __forceinline__ float warp_max_f(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(FULL, v, o));
    return v;
}

// 0 for an expert that cannot be chosen (-inf or NaN), else the order-preserving key; -0 counts as +0
__device__ __forceinline__ uint32_t route_key(float x)
{
    return (x > -CUDART_INF_F) ? float_to_key(x + 0.f) : 0u;
}
__device__ __forceinline__ float sigmoid_f(float x) { return 1.f / (1.f + expf(-x)); }

// The lane's NV logits, four neighbours at a time: register 4 q + v holds expert 128 q + 4 lane + v.  With VEC the four
// arrive in one 16-byte (fp32) or 8-byte (16-bit) load.
template <typename T, int NV, bool VEC>
__device__ __forceinline__ void load_row(const T *row, int E, int lane, float (&x)[NV])
{
#pragma unroll
    for (int q = 0; q < NV / 4; ++q) {
        const int i = 128 * q + 4 * lane;
        if constexpr (VEC) {
            if (i < E) {
                if constexpr (sizeof(T) == 4) {
                    const float4 f = __ldg(reinterpret_cast<const float4 *>(row + i));
                    x[4 * q] = f.x, x[4 * q + 1] = f.y, x[4 * q + 2] = f.z, x[4 * q + 3] = f.w;
                } else {
                    const uint2 u = __ldg(reinterpret_cast<const uint2 *>(row + i));
                    T h[4];
                    *reinterpret_cast<uint2 *>(h) = u;
#pragma unroll
                    for (int v = 0; v < 4; ++v) x[4 * q + v] = Io<T>::from_storage(h[v]);
                }
            } else {
#pragma unroll
                for (int v = 0; v < 4; ++v) x[4 * q + v] = -CUDART_INF_F;
            }
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v) x[4 * q + v] = (i + v < E) ? Io<T>::load1(row + i + v) : -CUDART_INF_F;
        }
    }
}

// The best `top` keys' sum of every group, by the lanes of the warp: lane l works for group l / per_lanes.  `sh` holds
// the row's keys as floats (-inf where unavailable).  Returns the mask of the groups that stay.
__device__ __forceinline__ uint32_t kept_groups(const float *sh, const RouteArgs &A, int lane)
{
    const int size = A.E / A.groups;
    int lanes = 1;  // lanes per group: a power of two
    while (2 * lanes * A.groups <= 32) lanes *= 2;
    const int g = lane / lanes;
    float a = -CUDART_INF_F, b = -CUDART_INF_F;  // best and second best
    if (g < A.groups)
        for (int i = lane % lanes; i < size; i += lanes) {
            const float v = sh[g * size + i];
            b = fmaxf(b, fminf(a, v));
            a = fmaxf(a, v);
        }
    for (int o = 1; o < lanes; o <<= 1) {
        const float a2 = __shfl_xor_sync(FULL, a, o), b2 = __shfl_xor_sync(FULL, b, o);
        b = fmaxf(fmaxf(b, b2), fminf(a, a2));
        a = fmaxf(a, a2);
    }
    const float s = (A.top > 1 && b > -CUDART_INF_F) ? a + b : a;  // a group with one expert left counts that one
    uint32_t key = (g < A.groups && lane % lanes == 0) ? route_key(s) : 0u;
    uint32_t keep = 0;
    for (int j = 0; j < A.kept; ++j) {
        const uint32_t m = __reduce_max_sync(FULL, key);
        if (m == 0) break;
        const int src = __ffs(__ballot_sync(FULL, key == m)) - 1;  // lowest lane = lowest group
        keep |= 1u << (src / lanes);
        if (lane == src) key = 0;
    }
    return keep;
}

template <typename T, int NV, bool VEC, bool GROUPS>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) route_forward_kernel(const RouteArgs A)
{
    extern __shared__ float route_sh[];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = (int64_t)blockIdx.x * ROUTE_WARPS + warp;
    if (t >= A.tokens) return;
    const T *row = reinterpret_cast<const T *>(A.logits) + t * A.stride;
    float x[NV];
    load_row<T, NV, VEC>(row, A.E, lane, x);

    // softmax over the whole row, where the scores themselves are needed
    const bool by_score = A.bias != nullptr || GROUPS;
    float top = 0.f, total = 1.f;
    if (A.score == LAPSUM_ROUTE_SOFTMAX && (by_score || !A.renorm)) {
        float m = -CUDART_INF_F;
#pragma unroll
        for (int i = 0; i < NV; ++i) m = fmaxf(m, x[i]);  // fmaxf skips NaN
        top = warp_max_f(m);
        if (top == -CUDART_INF_F) top = 0.f;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) s += (x[i] > -CUDART_INF_F) ? expf(x[i] - top) : 0.f;
        total = warp_sum_f(s);
    }

    uint32_t key[NV];
    float *sh = route_sh + warp * A.E;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = 128 * (i / 4) + 4 * lane + (i & 3);
        float c = x[i];
        if (by_score) {
            float s = c;
            if (A.score == LAPSUM_ROUTE_SOFTMAX) s = expf(c - top) / total;
            else if (A.score == LAPSUM_ROUTE_SIGMOID) s = sigmoid_f(c);
            const bool there = c > -CUDART_INF_F;
            if (A.bias != nullptr && e < A.E) s += __ldg(A.bias + e);
            s = there ? s : -CUDART_INF_F;
            if (GROUPS && e < A.E) sh[e] = (s > -CUDART_INF_F) ? s : -CUDART_INF_F;  // a NaN (bias) counts as unavailable
            // without a bias the experts of the kept groups are compared by their logits, which the score rises with
            if (A.bias != nullptr) c = s;
        }
        key[i] = route_key(c);
    }
    if constexpr (GROUPS) {
        __syncwarp();
        const uint32_t keep = kept_groups(sh, A, lane);
        const int size = A.E / A.groups;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = 128 * (i / 4) + 4 * lane + (i & 3);
            if (e < A.E && !((keep >> (e / size)) & 1u)) key[i] = 0u;
        }
    }

    // k times the warp's largest key; among equal keys the lowest expert
    int mine = -1;  // lane j keeps the j-th choice
    uint32_t best = 0;
    int at = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (key[i] > best) best = key[i], at = i;
    for (int j = 0; j < A.k; ++j) {
        const uint32_t m = __reduce_max_sync(FULL, best);
        if (m == 0) break;
        const uint32_t e = 128 * (at / 4) + 4 * lane + (at & 3);
        const uint32_t win = __reduce_min_sync(FULL, best == m ? e : 0xffffffffu);
        if (lane == j) mine = (int)win;
        if (best == m && e == win) {
            best = 0;
            int next = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i == at) key[i] = 0u;
                if (key[i] > best) best = key[i], next = i;
            }
            at = next;
        }
    }

    // weights: lane j holds its choice's logit again
    const float l = (mine >= 0) ? Io<T>::load1(row + mine) : -CUDART_INF_F;
    float w = 0.f;
    if (A.score == LAPSUM_ROUTE_SOFTMAX) {
        if (A.renorm) {  // the softmax of the chosen logits alone: never 0 / 0
            const float m = warp_max_f(l);
            w = (mine >= 0) ? expf(l - m) : 0.f;
            const float s = warp_sum_f(w);
            w = (mine >= 0) ? w / s : 0.f;
        } else {
            w = (mine >= 0) ? expf(l - top) / total : 0.f;
        }
    } else if (A.score == LAPSUM_ROUTE_SIGMOID) {
        if (A.renorm) {  // s_j e^{-m} = 1 / (e^m + e^{m - l}), m = min(0, largest l): the sum cannot underflow
            const float m = fminf(0.f, warp_max_f(l));
            w = (mine >= 0) ? 1.f / (expf(m) + expf(m - l)) : 0.f;
            const float s = warp_sum_f(w);
            w = (mine >= 0) ? w / s : 0.f;
        } else {
            w = (mine >= 0) ? sigmoid_f(l) : 0.f;
        }
    } else {
        w = (mine >= 0) ? l : 0.f;
        if (A.renorm) {
            const float s = warp_sum_f(w);
            w = (s != 0.f) ? w / s : 0.f;
        }
    }
    if (lane < A.k) {
        A.idx[t * A.k + lane] = mine;
        A.w[t * A.k + lane] = A.scale * w;
    }
}

struct RouteBackArgs {
    const void *grad_w;
    const void *logits;
    const int32_t *idx;
    const float *w;
    void *grad;
    int64_t tokens, stride;
    int E, k, score, renorm, gw_dtype;
    float scale;
};

// Gradient of one token's logits by one warp: lane j holds choice j.  With W = sum_j gw_j w_j / scale and
// g_j = w_j (gw_j - W):  softmax renormalised: g_j;  sigmoid renormalised: g_j (1 - s_j);  sigmoid: gw_j scale s (1 - s);
// softmax: p_i (scale [i chosen] gw - scale sum_j gw_j p_j), the one case that is dense in i;
// given: scale gw_j, renormalised (scale gw_j - sum gw w) / sum s.
// The row is zeroed (or filled with the dense part) first and the chosen entries are written over it by the same warp.
template <typename T, int NV, bool VEC>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) route_backward_kernel(const RouteBackArgs A)
{
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = (int64_t)blockIdx.x * ROUTE_WARPS + warp;
    if (t >= A.tokens) return;
    const T *row = reinterpret_cast<const T *>(A.logits) + t * A.stride;
    T *out = reinterpret_cast<T *>(A.grad) + t * A.E;
    int mine = -1;
    float w = 0.f, gw = 0.f;
    if (lane < A.k) {
        const int64_t at = t * A.k + lane;
        mine = __ldg(A.idx + at);
        if (mine >= A.E) mine = -1;
        w = __ldg(A.w + at);
        gw = A.gw_dtype == LAPSUM_IO_F32   ? __ldg(reinterpret_cast<const float *>(A.grad_w) + at)
             : A.gw_dtype == LAPSUM_IO_F16 ? Io<__half>::load1(reinterpret_cast<const __half *>(A.grad_w) + at)
                                           : Io<__nv_bfloat16>::load1(reinterpret_cast<const __nv_bfloat16 *>(A.grad_w) + at);
    }
    const bool chosen = mine >= 0;
    if (!chosen) w = 0.f, gw = 0.f;
    const float gww = warp_sum_f(gw * w);  // = scale * W
    float g = 0.f, dense = 0.f, top = 0.f, inv = 0.f;
    float x[NV];
    const bool full = A.score == LAPSUM_ROUTE_SOFTMAX && !A.renorm;
    if (full) {
        load_row<T, NV, VEC>(row, A.E, lane, x);
        float m = -CUDART_INF_F;
#pragma unroll
        for (int i = 0; i < NV; ++i) m = fmaxf(m, x[i]);
        top = warp_max_f(m);
        if (top == -CUDART_INF_F) top = 0.f;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            x[i] = (x[i] > -CUDART_INF_F) ? expf(x[i] - top) : 0.f;
            s += x[i];
        }
        s = warp_sum_f(s);
        inv = s > 0.f ? 1.f / s : 0.f;
        dense = -gww;
        g = w * (gw - gww / A.scale);  // w = scale p
    } else if (A.score == LAPSUM_ROUTE_SOFTMAX) {
        g = w * (gw - gww / A.scale);
    } else {
        const float l = chosen ? Io<T>::load1(row + mine) : 0.f;
        if (A.score == LAPSUM_ROUTE_SIGMOID) {
            const float e = expf(-fabsf(l));  // 1 - s = 1 / (1 + e^l) without cancellation
            const float rest = (l >= 0.f ? e : 1.f) / (1.f + e);
            g = (A.renorm ? w * (gw - gww / A.scale) : w * gw) * rest;
        } else if (A.renorm) {
            const float s = warp_sum_f(l);
            g = s != 0.f ? (A.scale * gw - gww) / s : 0.f;
        } else {
            g = A.scale * gw;
        }
    }
#pragma unroll
    for (int q = 0; q < NV / 4; ++q) {
        const int i = 128 * q + 4 * lane;
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        if (full) {
#pragma unroll
            for (int v = 0; v < 4; ++v) y[v] = x[4 * q + v] * inv * dense;
        }
        if constexpr (VEC) {
            if (i < A.E) {
                if constexpr (sizeof(T) == 4) {
                    *reinterpret_cast<float4 *>(out + i) = make_float4(y[0], y[1], y[2], y[3]);
                } else {
                    T h[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) Io<T>::store1(h + v, y[v]);
                    *reinterpret_cast<uint2 *>(out + i) = *reinterpret_cast<const uint2 *>(h);
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (i + v < A.E) Io<T>::store1(out + i + v, y[v]);
        }
    }
    __syncwarp();  // orders the row's stores before the chosen entries'
    if (chosen) Io<T>::store1(out + mine, g);
}

// ------------------------------------------------------------------ dispatch ----
constexpr int DISPATCH_THREADS = 256, DISPATCH_CHUNK = 4096;  // entries per block; a warp takes 512 neighbours
__host__ __device__ constexpr int dispatch_stride(int E) { return (E + 3) & ~3; }  // words of one row of counts: 16-byte rows

struct DispatchArgs {
    const int32_t *idx;
    int64_t entries, capacity;
    int E, rows, shift, chunks, bits;  // rows = 1 << shift
    int32_t *counts, *offsets, *slot_of, *entry_of, *tile_expert, *partial;
};

// Entries per expert of one chunk (integer atomics in shared memory: the counts do not depend on their order)
__global__ void __launch_bounds__(DISPATCH_THREADS) dispatch_count_kernel(const DispatchArgs A)
{
    extern __shared__ int32_t dispatch_sh[];
    const int stride = dispatch_stride(A.E);
    for (int e = threadIdx.x; e < stride; e += DISPATCH_THREADS) dispatch_sh[e] = 0;
    pdl_wait();
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * DISPATCH_CHUNK;
    const int n = (int)min((int64_t)DISPATCH_CHUNK, A.entries - begin);
#pragma unroll 8
    for (int i = threadIdx.x; i < n; i += DISPATCH_THREADS) {
        const int e = __ldg(A.idx + begin + i);
        if ((unsigned)e < (unsigned)A.E) atomicAdd(dispatch_sh + e, 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < stride; e += DISPATCH_THREADS) A.partial[(int64_t)blockIdx.x * stride + e] = dispatch_sh[e];
}

// Positions.  Every block sums the chunks' counts itself (chunks x E words from L2: less than another launch), scans the
// experts' padded lengths, then gives its entries their slots in order: a warp's 32 entries find their equals by ballot.
__global__ void __launch_bounds__(DISPATCH_THREADS) dispatch_place_kernel(const DispatchArgs A)
{
    extern __shared__ __align__(16) int32_t dispatch_sh[];
    constexpr int W = DISPATCH_THREADS / 32;
    const int E = A.E, stride = dispatch_stride(E);
    int32_t *const hist = dispatch_sh;          // [W][stride]: a warp's entries per expert, then its next slot
    int32_t *const before = hist + W * stride;  // [stride]: entries of the chunks before this one
    int32_t *const count = before + stride;     // [stride]: entries of all chunks
    int32_t *const offset = count + stride;     // [E + 1]
    __shared__ int32_t scan[W];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < (W + 2) * stride; i += DISPATCH_THREADS) hist[i] = 0;
    pdl_wait();
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * DISPATCH_CHUNK;
    const int n = max(0, (int)min((int64_t)DISPATCH_CHUNK, A.entries - begin));
    const int per = (n + 32 * W - 1) / (32 * W) * 32;  // entries of a warp: neighbours, so that the order is kept
    const int w0 = min(n, warp * per), w1 = min(n, w0 + per);
#pragma unroll 8
    for (int i = w0 + lane; i < w1; i += 32) {
        const int e = __ldg(A.idx + begin + i);
        if ((unsigned)e < (unsigned)E) {
            atomicAdd(hist + warp * stride + e, 1);
            if (A.chunks == 1) atomicAdd(count + e, 1);
        }
    }
    if (A.chunks > 1) {  // four experts of one chunk per load
        const int quads = stride / 4;
        const int4 *const p = reinterpret_cast<const int4 *>(A.partial);
#pragma unroll 8
        for (int i = tid; i < A.chunks * quads; i += DISPATCH_THREADS) {
            const int4 v = __ldg(p + i);
            const int c = i / quads, q = 4 * (i - c * quads);
            int32_t *const all = count + q, *const b = before + q;
            if (v.x) atomicAdd(all, v.x);
            if (v.y) atomicAdd(all + 1, v.y);
            if (v.z) atomicAdd(all + 2, v.z);
            if (v.w) atomicAdd(all + 3, v.w);
            if (c < (int)blockIdx.x) {
                if (v.x) atomicAdd(b, v.x);
                if (v.y) atomicAdd(b + 1, v.y);
                if (v.z) atomicAdd(b + 2, v.z);
                if (v.w) atomicAdd(b + 3, v.w);
            }
        }
    }
    __syncthreads();
    // exclusive scan of the padded lengths: a thread takes `own` neighbouring experts
    const int own = (E + DISPATCH_THREADS - 1) / DISPATCH_THREADS;
    auto padded = [&](int e) { return (count[e] + A.rows - 1) >> A.shift << A.shift; };
    int sum = 0;
    for (int j = 0; j < own; ++j)
        if (tid * own + j < E) sum += padded(tid * own + j);
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(FULL, run, o);
        if (lane >= o) run += v;
    }
    if (lane == 31) scan[warp] = run;
    __syncthreads();
    int base = run - sum;
    for (int w = 0; w < warp; ++w) base += scan[w];
    for (int j = 0; j < own; ++j) {
        const int e = tid * own + j;
        if (e >= E) break;
        offset[e] = base;
        int next = base + before[e];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int v = hist[w * stride + e];
            hist[w * stride + e] = next;
            next += v;
        }
        base += padded(e);
        if (e == E - 1) offset[E] = base;
    }
    __syncthreads();
    for (int i = w0; i < w1; i += 32) {
        const int at = i + lane;
        const int e = at < w1 ? __ldg(A.idx + begin + at) : -1;
        const bool there = (unsigned)e < (unsigned)E;
        const uint32_t id = there ? (uint32_t)e : (uint32_t)E;
        unsigned peers = FULL;
        for (int b = 0; b < A.bits; ++b) {
            const bool bit = (id >> b) & 1u;
            const unsigned bal = __ballot_sync(FULL, bit);
            peers &= bit ? bal : ~bal;
        }
        const int rank = __popc(peers & ((1u << lane) - 1u));
        int slot = -1;
        if (there) slot = hist[warp * stride + e] + rank;
        __syncwarp();
        if (there && rank == 0) hist[warp * stride + e] += __popc(peers);
        __syncwarp();
        if (at < w1) {
            A.slot_of[begin + at] = slot;
            if (there) A.entry_of[slot] = (int32_t)(begin + at);
        }
    }
    // the tables' rest: holes of the slots, experts of the row tiles, counts and offsets; a warp per expert
    for (int e = blockIdx.x * W + warp; e < E; e += gridDim.x * W) {
        const int lo = offset[e], hi = offset[e + 1], c = count[e];
        for (int s = lo + c + lane; s < hi; s += 32) A.entry_of[s] = -1;
        for (int r = (lo >> A.shift) + lane; r < (hi >> A.shift); r += 32) A.tile_expert[r] = e;
        if (lane == 0) A.counts[e] = c, A.offsets[e] = lo;
    }
    const int all = offset[E];
    if (blockIdx.x == 0 && tid == 0) A.offsets[E] = all;
    for (int64_t s = all + (int64_t)blockIdx.x * DISPATCH_THREADS + tid; s < A.capacity; s += (int64_t)gridDim.x * DISPATCH_THREADS) A.entry_of[s] = -1;
    for (int64_t r = (all >> A.shift) + (int64_t)blockIdx.x * DISPATCH_THREADS + tid; r < (A.capacity >> A.shift); r += (int64_t)gridDim.x * DISPATCH_THREADS)
        A.tile_expert[r] = -1;
}

}  // namespace lapsum
