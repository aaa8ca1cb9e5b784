// Routing of tokens to experts and the dispatch tables that bring every expert's tokens side by side.
//
// route    L lanes per token (4 to 32), each with a run of NV neighbouring logits.
//          keys   c_i = l_i (softmax or sigmoid without a bias: both rise with the logit), else s_i + bias_i
//          groups the `kept` groups with the largest sum of their best `group_top` keys keep their experts
//          choice k largest keys, ties to the lower index; weights from the scores s, never from the bias
//          Bound by integer instructions, not by memory, so the work per choice is kept small: a lane knows the maxima of
//          its runs of four keys, log2 L exchanges find the row's largest, a ballot the lane (lanes hold ascending
//          runs, so the lowest lane is the lowest index), and that lane alone looks into one run in shared memory.
//          A choice costs a warp the same instructions however many tokens it holds, so few lanes per token are better:
//          65536 x 128 fp32, k = 8, forward: 47 us with 32 lanes, 24 us with 8, 20 us with 4 (160 instructions a token, the
//          integer pipe 60 % busy; its 38 MB would take 6 us); the backward takes 11 us for 40 MB, both together
//          25.9 us.  16381 x 256 bf16 sigmoid with a bias and 8 groups (16 lanes): 24.0 us together.
// dispatch a stable counting sort of the T k entries by expert, integers only.  65536 x 8 entries, 128 experts: 11 us in two
//          launches (6.4 MB would take 1 us; two dependent passes of latency and 27 k instructions a block); 32 x 8: 5.5 us.
#pragma once
#include "common.cuh"

namespace lapsum {

constexpr int ROUTE_MAX_E = 1024, ROUTE_MAX_K = 32, ROUTE_MAX_GROUPS = 32;
constexpr int ROUTE_WARPS = 8;  // warps per block

struct RouteArgs {
    const void *logits;
    const float *bias;
    int32_t *idx;
    float *w;
    int64_t tokens, stride;
    int E, k, groups, kept, top, score, renorm;
    int bias_vec;  // four experts' bias per load
    float scale;
};

// What experts are compared by: -inf for one that cannot be chosen (NaN, by fmaxf's rule), +0 for -0
__device__ __forceinline__ float route_key(float x) { return fmaxf(x + 0.f, -CUDART_INF_F); }
// For weights and keys alike.  (Keys of the fast exponential and quotient, several units of 2^-23 off, took a sixth of neighbouring logits
// between -60 and -8 in the wrong order.)
__device__ __forceinline__ float sigmoid_f(float x) { return 1.f / (1.f + expf(-x)); }

template <int L>
__device__ __forceinline__ float row_sum_f(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}
template <int L>
__device__ __forceinline__ float row_max_f(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(FULL, v, o));
    return v;
}

// NV neighbouring logits from `first` on, -inf beyond the row's end.  VEC: rows of whole vectors at aligned addresses.
template <typename T, int NV, bool VEC>
__device__ __forceinline__ void load_run(const T *row, int first, int E, float (&x)[NV])
{
    if constexpr (VEC) {
        constexpr int V = 16 / sizeof(T) < NV ? 16 / sizeof(T) : NV;  // logits per load
#pragma unroll
        for (int q = 0; q < NV / V; ++q) {
            T h[V];
            if (first + q * V < E) {
                if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4 *>(h) = ld(reinterpret_cast<const uint4 *>(row + first + q * V));
                else *reinterpret_cast<uint2 *>(h) = ld(reinterpret_cast<const uint2 *>(row + first + q * V));
            }
#pragma unroll
            for (int v = 0; v < V; ++v) x[q * V + v] = (first + q * V < E) ? Io<T>::from_storage(h[v]) : -CUDART_INF_F;
        }
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v) x[v] = (first + v < E) ? Io<T>::from_storage(ld(row + first + v)) : -CUDART_INF_F;
    }
}

// The groups that keep their experts, as a bit mask, by the row's L lanes; `c` holds the row's keys as floats (-inf =
// unavailable), element e at c[place(e)], `strength` 32 floats of the row.
template <int L, typename Place>
__device__ __forceinline__ uint32_t kept_groups(const float *c, float *strength, const RouteArgs &A, int r, int row_lane, Place place)
{
    const int size = A.E / A.groups;
    int lanes = 1;  // lanes that share a group's experts: a power of two
    while (2 * lanes * A.groups <= L && 4 * lanes < size) lanes *= 2;
    const int share = r % lanes;
    for (int g0 = 0; g0 < A.groups; g0 += L / lanes) {
        const int g = g0 + r / lanes;
        float a = -CUDART_INF_F, b = -CUDART_INF_F;  // best and second best
        auto take = [&](float v) {
            b = fmaxf(b, fminf(a, v));
            a = fmaxf(a, v);
        };
        if (g < A.groups) {
            if (size % 4 == 0) {  // whole runs of four
                for (int i = g * size + 4 * share; i < (g + 1) * size; i += 4 * lanes) {
                    const float4 v = *reinterpret_cast<const float4 *>(c + place(i));
                    take(v.x), take(v.y), take(v.z), take(v.w);
                }
            } else {
                for (int i = g * size + share; i < (g + 1) * size; i += lanes) take(c[place(i)]);
            }
        }
        for (int o = 1; o < lanes; o <<= 1) {
            const float a2 = __shfl_xor_sync(FULL, a, o), b2 = __shfl_xor_sync(FULL, b, o);
            b = fmaxf(fmaxf(b, b2), fminf(a, a2));
            a = fmaxf(a, a2);
        }
        if (g < A.groups && share == 0) strength[g] = (A.top > 1 && b > -CUDART_INF_F) ? a + b : a;  // one expert left: that one
    }
    __syncwarp();
    uint32_t keep = 0;
    for (int g0 = 0; g0 < A.groups; g0 += L) {
        const int g = g0 + r;
        bool in = false;
        if (g < A.groups && strength[g] > -CUDART_INF_F) {
            int ahead = 0;  // groups that come before this one
            for (int o = 0; o < A.groups; ++o) ahead += strength[o] > strength[g] || (strength[o] == strength[g] && o < g);
            in = ahead < A.kept;
        }
        const uint32_t bal = __ballot_sync(FULL, in) >> row_lane;
        keep |= (L == 32 ? bal : bal & ((1u << (L & 31)) - 1u)) << g0;
    }
    return keep;
}

// PLAIN: no bias and no groups, so the logits are the keys and nothing else of the row is kept: the warp brings its rows in whole
// lines and hands each lane its run through shared memory, and four lanes hold a token of up to 128 logits.
template <typename T, int L, int NV, bool VEC, bool GROUPS, bool PLAIN>
__global__ void __launch_bounds__(32 * ROUTE_WARPS, NV > 16 && !PLAIN ? 2 : 4) route_forward_kernel(const RouteArgs A)
{
    constexpr int ROWS = 32 / L * ROUTE_WARPS, PITCH = NV + 4;  // a lane's keys: 16-byte pieces of eight lanes meet no bank twice
    __shared__ __align__(16) float keys[32 * ROUTE_WARPS * PITCH];
    __shared__ short choice[ROWS * ROUTE_MAX_K];
    __shared__ float strength[GROUPS ? ROWS * ROUTE_MAX_GROUPS : 1];
    pdl_wait();
    const int lane = threadIdx.x & 31, r = lane % L, row_lane = lane - r, row_in_block = threadIdx.x / L;
    const int64_t t = (int64_t)blockIdx.x * ROWS + row_in_block;
    const bool live = t < A.tokens;
    const T *row = reinterpret_cast<const T *>(A.logits) + (live ? t : A.tokens - 1) * A.stride;
    float *const mine = keys + threadIdx.x * PITCH;
    const int first = r * NV;
    float top = 0.f, total = 1.f;                       // softmax: the row's largest logit and sum
    float run[NV / 4], best = -CUDART_INF_F;            // maxima of the lane's runs of four keys
    if constexpr (PLAIN) {
        constexpr int EP = L * NV;  // a row, padded
        const int64_t t0 = (int64_t)blockIdx.x * ROWS + (threadIdx.x >> 5) * (32 / L);
        float *const all = keys + (threadIdx.x - lane) * PITCH;
#pragma unroll
        for (int q = 0; q < NV / 4; ++q) {
            const int f = (32 * q + lane) * 4, rr = f / EP, e = f % EP;
            float4 k4 = make_float4(-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F);
            if (t0 + rr < A.tokens && e < A.E) {
                T h[4];
                const T *const from = reinterpret_cast<const T *>(A.logits) + (t0 + rr) * A.stride + e;
                if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4 *>(h) = ld(reinterpret_cast<const uint4 *>(from));
                else *reinterpret_cast<uint2 *>(h) = ld(reinterpret_cast<const uint2 *>(from));
                k4 = make_float4(route_key(Io<T>::from_storage(h[0])), route_key(Io<T>::from_storage(h[1])), route_key(Io<T>::from_storage(h[2])),
                                 route_key(Io<T>::from_storage(h[3])));
            }
            *reinterpret_cast<float4 *>(all + (rr * L + e / NV) * PITCH + e % NV) = k4;
        }
        __syncwarp();
#pragma unroll
        for (int q = 0; q < NV / 4; ++q) {
            const float4 k4 = *reinterpret_cast<const float4 *>(mine + 4 * q);
            run[q] = fmaxf(fmaxf(k4.x, k4.y), fmaxf(k4.z, k4.w));
            best = fmaxf(best, run[q]);
        }
        if (A.score == LAPSUM_ROUTE_SOFTMAX && !A.renorm) {
            top = row_max_f<L>(best);
            if (top == -CUDART_INF_F) top = 0.f;
            float s = 0.f;
#pragma unroll
            for (int q = 0; q < NV / 4; ++q) {
                const float4 k4 = *reinterpret_cast<const float4 *>(mine + 4 * q);
                s += (expf(k4.x - top) + expf(k4.y - top)) + (expf(k4.z - top) + expf(k4.w - top));  // 0 for -inf
            }
            total = row_sum_f<L>(s);
        }
    } else {
        float x[NV];
        load_run<T, NV, VEC>(row, first, A.E, x);
        // softmax over the whole row, where the scores themselves are needed
        const bool by_score = A.bias != nullptr || GROUPS;
        if (A.score == LAPSUM_ROUTE_SOFTMAX && (by_score || !A.renorm)) {
            float m = -CUDART_INF_F;
#pragma unroll
            for (int i = 0; i < NV; ++i) m = fmaxf(m, x[i]);  // fmaxf skips NaN
            top = row_max_f<L>(m);
            if (top == -CUDART_INF_F) top = 0.f;
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) s += (x[i] > -CUDART_INF_F) ? expf(x[i] - top) : 0.f;
            total = row_sum_f<L>(s);
        }
        if (by_score) {
            float c[NV], offset[NV];  // the bias of my experts
#pragma unroll
            for (int q = 0; q < NV / 4; ++q) {
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                const int i = first + 4 * q;
                if (A.bias != nullptr) {
                    if (A.bias_vec) {
                        if (i < A.E) v = ld(reinterpret_cast<const float4 *>(A.bias + i));
                    } else {
                        if (i < A.E) v.x = ld(A.bias + i);
                        if (i + 1 < A.E) v.y = ld(A.bias + i + 1);
                        if (i + 2 < A.E) v.z = ld(A.bias + i + 2);
                        if (i + 3 < A.E) v.w = ld(A.bias + i + 3);
                    }
                }
                offset[4 * q] = v.x, offset[4 * q + 1] = v.y, offset[4 * q + 2] = v.z, offset[4 * q + 3] = v.w;
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float s = x[i];
                if (A.score == LAPSUM_ROUTE_SOFTMAX) s = expf(s - top) / total;
                else if (A.score == LAPSUM_ROUTE_SIGMOID) s = sigmoid_f(s);
                s += offset[i];
                c[i] = (x[i] > -CUDART_INF_F && s > -CUDART_INF_F) ? s : -CUDART_INF_F;  // a NaN counts as unavailable
            }
            if constexpr (GROUPS) {
#pragma unroll
                for (int q = 0; q < NV / 4; ++q) *reinterpret_cast<float4 *>(mine + 4 * q) = make_float4(c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]);
                __syncwarp();
                const uint32_t keep = kept_groups<L>(keys + (threadIdx.x - r) * PITCH, strength + row_in_block * ROUTE_MAX_GROUPS, A, r, row_lane,
                                                     [](int e) { return e / NV * PITCH + e % NV; });
                __syncwarp();
                const int size = A.E / A.groups;
                int g = first / size;
                if (size % NV == 0) {  // all of the lane's experts are of one group
                    const bool in = (keep >> (g & 31)) & 1u;
#pragma unroll
                    for (int i = 0; i < NV; ++i) c[i] = in ? c[i] : -CUDART_INF_F, x[i] = in ? x[i] : -CUDART_INF_F;
                } else {
                    int left = (g + 1) * size - first;  // experts until the next group
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        if (!((keep >> (g & 31)) & 1u)) c[i] = x[i] = -CUDART_INF_F;
                        if (--left == 0) ++g, left = size;
                    }
                }
            }
            // without a bias the experts of the kept groups are compared by their logits, which the score rises with
            if (A.bias != nullptr) {
#pragma unroll
                for (int i = 0; i < NV; ++i) x[i] = c[i];
            }
        }
#pragma unroll
        for (int q = 0; q < NV / 4; ++q) {
            const float4 k4 = make_float4(route_key(x[4 * q]), route_key(x[4 * q + 1]), route_key(x[4 * q + 2]), route_key(x[4 * q + 3]));
            *reinterpret_cast<float4 *>(mine + 4 * q) = k4;
            run[q] = fmaxf(fmaxf(k4.x, k4.y), fmaxf(k4.z, k4.w));
            best = fmaxf(best, run[q]);
        }
    }
    short *const out = choice + row_in_block * ROUTE_MAX_K;
    for (int j = 0; j < A.k; ++j) {
        const float m = row_max_f<L>(best);
        const uint32_t bal = __ballot_sync(FULL, best == m);
        const uint32_t owners = (L == 32) ? bal : (bal >> row_lane) & ((1u << (L & 31)) - 1u);
        if (r == __ffs(owners) - 1) {
            int e = -1;
            if (m > -CUDART_INF_F) {
                int q = NV / 4 - 1;
#pragma unroll
                for (int i = NV / 4 - 2; i >= 0; --i) q = run[i] == m ? i : q;
                const float4 k4 = *reinterpret_cast<const float4 *>(mine + 4 * q);
                // the run's first largest goes: the largest of the others stays
                const float lo = fmaxf(k4.z, k4.w), next = k4.x == m ? fmaxf(k4.y, lo) : k4.y == m ? fmaxf(k4.x, lo) : fmaxf(fmaxf(k4.x, k4.y), k4.z == m ? k4.w : k4.z);
                const int v = k4.x == m ? 0 : k4.y == m ? 1 : k4.z == m ? 2 : 3;
                mine[4 * q + v] = -CUDART_INF_F;
                best = -CUDART_INF_F;
#pragma unroll
                for (int i = 0; i < NV / 4; ++i) {
                    run[i] = i == q ? next : run[i];
                    best = fmaxf(best, run[i]);
                }
                e = first + 4 * q + v;
            }
            out[j] = (short)e;
        }
    }
    __syncwarp();

    // weights: lane r of the row has the choices r, r + L, ...
    constexpr int C = ROUTE_MAX_K / L;
    int e[C];
    float l[C], w[C];
#pragma unroll
    for (int p = 0; p < C; ++p) {
        e[p] = (p * L + r < A.k) ? out[p * L + r] : -1;
        l[p] = (e[p] >= 0) ? Io<T>::from_storage(ld(row + e[p])) : -CUDART_INF_F;
    }
    float peak = l[0], sum = 0.f;
    if (A.renorm && A.score != LAPSUM_ROUTE_GIVEN) {
#pragma unroll
        for (int p = 1; p < C; ++p) peak = fmaxf(peak, l[p]);
        peak = row_max_f<L>(peak);
    }
    const float floor_ = fminf(0.f, peak), e_floor = A.renorm && A.score == LAPSUM_ROUTE_SIGMOID ? expf(floor_) : 0.f;
#pragma unroll
    for (int p = 0; p < C; ++p) {
        if (p * L >= A.k) break;
        float v = 0.f;
        if (e[p] >= 0) {
            if (A.score == LAPSUM_ROUTE_SOFTMAX)  // renormalised: the softmax of the chosen logits alone, never 0 / 0
                v = A.renorm ? expf(l[p] - peak) : expf(l[p] - top) / total;
            else if (A.score == LAPSUM_ROUTE_SIGMOID)  // s e^{-m} = 1 / (e^m + e^{m - l}), m = min(0, largest l): no underflow of the sum
                v = A.renorm ? 1.f / (e_floor + expf(floor_ - l[p])) : sigmoid_f(l[p]);
            else
                v = l[p];
        }
        w[p] = v;
        sum += v;
    }
    if (A.renorm) sum = row_sum_f<L>(sum);
#pragma unroll
    for (int p = 0; p < C; ++p) {
        const int j = p * L + r;
        if (j >= A.k) break;
        if (A.renorm) w[p] = (e[p] >= 0 && sum != 0.f) ? w[p] / sum : 0.f;
        if (live) {
            A.idx[t * A.k + j] = e[p];
            A.w[t * A.k + j] = A.scale * w[p];
        }
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

__device__ __forceinline__ float route_grad_w(const RouteBackArgs &A, int64_t at)
{
    return A.gw_dtype == LAPSUM_IO_F32   ? ld(reinterpret_cast<const float *>(A.grad_w) + at)
           : A.gw_dtype == LAPSUM_IO_F16 ? Io<__half>::from_storage(ld(reinterpret_cast<const __half *>(A.grad_w) + at))
                                         : Io<__nv_bfloat16>::from_storage(ld(reinterpret_cast<const __nv_bfloat16 *>(A.grad_w) + at));
}

// Gradient of the logits where only the chosen ones have one: with W = sum_j gw_j w_j / scale and g_j = w_j (gw_j - W),
// softmax renormalised: g_j;  sigmoid renormalised: g_j (1 - s_j);  sigmoid: gw_j scale s_j (1 - s_j);
// given: scale gw_j, renormalised (scale gw_j - sum gw w) / sum s.
// A warp has 32 / L tokens, a lane per choice.  It writes zeros over its rows, which lie side by side, and then the chosen entries.
template <typename T, int L, bool VEC>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) route_backward_kernel(const RouteBackArgs A)
{
    constexpr int R = 32 / L;
    pdl_wait();
    const int lane = threadIdx.x & 31, r = lane % L;
    const int64_t t0 = ((int64_t)blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5)) * R, t = t0 + lane / L;
    if (t0 >= A.tokens) return;
    int mine = -1;
    float w = 0.f, gw = 0.f, l = 0.f;
    if (r < A.k && t < A.tokens) {
        const int64_t at = t * A.k + r;
        mine = ld(A.idx + at);
        w = ld(A.w + at);
        gw = route_grad_w(A, at);
    }
    T *const out = reinterpret_cast<T *>(A.grad) + t0 * A.E;
    const int n = (int)min((int64_t)R, A.tokens - t0) * A.E;
    if constexpr (VEC) {
        constexpr int V = 16 / sizeof(T);
        for (int i = lane * V; i < n; i += 32 * V) *reinterpret_cast<uint4 *>(out + i) = make_uint4(0, 0, 0, 0);
    } else {
        for (int i = lane; i < n; i += 32) Io<T>::store1(out + i, 0.f);
    }
    const bool chosen = mine >= 0 && mine < A.E;
    if (!chosen) w = 0.f, gw = 0.f;
    if (chosen && A.score != LAPSUM_ROUTE_SOFTMAX) l = Io<T>::from_storage(ld(reinterpret_cast<const T *>(A.logits) + t * A.stride + mine));
    const float gww = row_sum_f<L>(gw * w);  // = scale W
    float g;
    if (A.score == LAPSUM_ROUTE_SOFTMAX) {
        g = w * (gw - gww / A.scale);
    } else if (A.score == LAPSUM_ROUTE_SIGMOID) {
        const float e = expf(-fabsf(l));  // 1 - s = 1 / (1 + e^l) without cancellation
        g = (A.renorm ? w * (gw - gww / A.scale) : w * gw) * ((l >= 0.f ? e : 1.f) / (1.f + e));
    } else if (A.renorm) {
        const float s = row_sum_f<L>(chosen ? l : 0.f);
        g = s != 0.f ? (A.scale * gw - gww) / s : 0.f;
    } else {
        g = A.scale * gw;
    }
    __syncwarp();  // orders the zeros before the chosen entries
    if (chosen) Io<T>::store1(out + (int64_t)(lane / L) * A.E + mine, g);
}

// Softmax without renormalisation: p_i (scale [i chosen] gw_i - scale sum_j gw_j p_j), dense in i.  L lanes per token.
// 65536 x 128 fp32, k = 8: 19 us (73 MB would take 11).
template <typename T, int L, int NV, bool VEC>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) route_backward_dense_kernel(const RouteBackArgs A)
{
    constexpr int ROWS = 32 / L * ROUTE_WARPS, C = ROUTE_MAX_K / L;
    pdl_wait();
    const int lane = threadIdx.x & 31, r = lane % L;
    const int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / L;
    const bool live = t < A.tokens;
    const T *row = reinterpret_cast<const T *>(A.logits) + (live ? t : A.tokens - 1) * A.stride;
    T *const out = reinterpret_cast<T *>(A.grad) + t * A.E;
    const int first = r * NV;
    float x[NV];
    load_run<T, NV, VEC>(row, first, A.E, x);
    int mine[C];
    float w[C], gw[C], gww = 0.f;
#pragma unroll
    for (int p = 0; p < C; ++p) {
        const int j = p * L + r;
        mine[p] = -1, w[p] = gw[p] = 0.f;
        if (live && j < A.k) {
            mine[p] = ld(A.idx + t * A.k + j);
            if (mine[p] >= A.E) mine[p] = -1;
            if (mine[p] >= 0) w[p] = ld(A.w + t * A.k + j), gw[p] = route_grad_w(A, t * A.k + j);
        }
        gww += gw[p] * w[p];
    }
    gww = row_sum_f<L>(gww);  // w = scale p
    float m = -CUDART_INF_F, s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) m = fmaxf(m, x[i]);
    m = row_max_f<L>(m);
    if (m == -CUDART_INF_F) m = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        x[i] = (x[i] > -CUDART_INF_F) ? expf(x[i] - m) : 0.f;
        s += x[i];
    }
    s = row_sum_f<L>(s);
    const float inv = s > 0.f ? 1.f / s : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = -x[i] * inv * gww;
    if (live) {
        if constexpr (VEC) {
            constexpr int V = 16 / sizeof(T) < NV ? 16 / sizeof(T) : NV;
#pragma unroll
            for (int q = 0; q < NV / V; ++q)
                if (first + q * V < A.E) {
                    T h[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) Io<T>::store1(h + v, x[q * V + v]);
                    if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4 *>(out + first + q * V) = *reinterpret_cast<const uint4 *>(h);
                    else *reinterpret_cast<uint2 *>(out + first + q * V) = *reinterpret_cast<const uint2 *>(h);
                }
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (first + v < A.E) Io<T>::store1(out + first + v, x[v]);
        }
    }
    __syncwarp();  // orders the row's stores before the chosen entries'
#pragma unroll
    for (int p = 0; p < C; ++p)
        if (mine[p] >= 0) Io<T>::store1(out + mine[p], w[p] * (gw[p] - gww / A.scale));
}

// ------------------------------------------------------------------ dispatch ----
// A block takes 4096 neighbouring entries, a warp 128 of them; a batch of up to 4096 entries needs one launch of one block.  The
// kernel is bound by its instructions (one block per SM, IPC 2 to 2.5), so 65536 x 8 entries are spread over 128 blocks.
// More than DISPATCH_BLOCKS of them are worked off one after the other, so that the blocks' counts stay a small table.
constexpr int DISPATCH_BLOCKS = 512;
constexpr int DISPATCH_THREADS = 1024, DISPATCH_WARPS = DISPATCH_THREADS / 32, DISPATCH_PER = 4, DISPATCH_CHUNK = DISPATCH_THREADS * DISPATCH_PER;
__host__ __device__ constexpr int dispatch_stride(int E) { return (E + 3) & ~3; }  // words of one row of counts: 16-byte rows
__host__ __device__ constexpr int dispatch_pitch(int E) { return (E / 2 * 2 + 2) | ((E / 2 + 1) % 2 ? 0 : 2); }  // 16-bit counts of a warp: an odd number of words
constexpr size_t dispatch_place_smem(int E) { return 12 * (size_t)dispatch_stride(E) + 16 + 2 * (size_t)DISPATCH_WARPS * (size_t)dispatch_pitch(E); }

struct DispatchArgs {
    const int32_t *idx;
    int64_t entries, capacity;
    int E, rows, shift, blocks, chunks;  // rows = 1 << shift; blocks: of `chunks` neighbouring chunks each
    int32_t *counts, *offsets, *slot_of, *entry_of, *tile_expert, *partial;
};

// Entries per expert of one block's chunks (integer atomics in shared memory: the counts do not depend on their order)
__global__ void __launch_bounds__(DISPATCH_THREADS) dispatch_count_kernel(const DispatchArgs A)
{
    extern __shared__ __align__(16) int32_t dispatch_sh[];
    const int stride = dispatch_stride(A.E);
    for (int e = threadIdx.x; e < stride; e += DISPATCH_THREADS) dispatch_sh[e] = 0;
    pdl_wait();
    __syncthreads();
    for (int c = 0; c < A.chunks; ++c) {
        const int64_t begin = ((int64_t)blockIdx.x * A.chunks + c) * DISPATCH_CHUNK;
        int e[DISPATCH_PER];
#pragma unroll
        for (int j = 0; j < DISPATCH_PER; ++j) {
            const int64_t i = begin + j * DISPATCH_THREADS + threadIdx.x;
            e[j] = i < A.entries ? ld(A.idx + i) : -1;
        }
#pragma unroll
        for (int j = 0; j < DISPATCH_PER; ++j)
            if ((unsigned)e[j] < (unsigned)A.E) atomicAdd(dispatch_sh + e[j], 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < stride; i += DISPATCH_THREADS) A.partial[(int64_t)blockIdx.x * stride + i] = dispatch_sh[i];
}

// Positions.  A warp numbers its entries per expert 32 at a time (equals are found by ballot), the block scans the warps'
// counts of every expert and, once, the experts' padded lengths; with several blocks every one of them sums the blocks' counts
// itself (blocks x E words from L2: less than another launch).
template <int BITS>  // of an expert's number
__global__ void __launch_bounds__(DISPATCH_THREADS) dispatch_place_kernel(const DispatchArgs A)
{
    extern __shared__ __align__(16) int32_t dispatch_sh[];
    const int E = A.E, stride = dispatch_stride(E), pitch = dispatch_pitch(E);
    int32_t *const count = dispatch_sh;      // [stride]: entries of all blocks
    int32_t *const next = count + stride;    // [stride]: entries of the blocks before this one, then the next slot
    int32_t *const offset = next + stride;   // [E + 1]
    uint16_t *const hist = reinterpret_cast<uint16_t *>(offset + stride + 4);  // [warps][pitch]: a warp's entries, then those of the warps before
    __shared__ int32_t scan[DISPATCH_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint16_t *const mine = hist + warp * pitch;
    for (int i = tid; i < 2 * stride; i += DISPATCH_THREADS) count[i] = 0;
    for (int i = tid; i < DISPATCH_WARPS * pitch / 2; i += DISPATCH_THREADS) reinterpret_cast<uint32_t *>(hist)[i] = 0;
    pdl_wait();
    __syncthreads();
    if (A.blocks > 1) {  // a thread has four experts of every `groups`-th block
        const int quads = stride / 4, groups = DISPATCH_THREADS / quads, c0 = tid / quads, q = 4 * (tid - c0 * quads);
        if (c0 < groups) {
            int4 all = make_int4(0, 0, 0, 0), b = make_int4(0, 0, 0, 0);
#pragma unroll 4
            for (int c = c0; c < A.blocks; c += groups) {
                const int4 v = ld(reinterpret_cast<const int4 *>(A.partial + (int64_t)c * stride + q));
                all.x += v.x, all.y += v.y, all.z += v.z, all.w += v.w;
                if (c < (int)blockIdx.x) b.x += v.x, b.y += v.y, b.z += v.z, b.w += v.w;
            }
            atomicAdd(count + q, all.x), atomicAdd(count + q + 1, all.y), atomicAdd(count + q + 2, all.z), atomicAdd(count + q + 3, all.w);
            atomicAdd(next + q, b.x), atomicAdd(next + q + 1, b.y), atomicAdd(next + q + 2, b.z), atomicAdd(next + q + 3, b.w);
        }
    }
    for (int chunk = 0; chunk < A.chunks; ++chunk) {
        const int64_t from = ((int64_t)blockIdx.x * A.chunks + chunk) * DISPATCH_CHUNK;
        if (from >= A.entries && chunk > 0) break;  // uniform in the block
        const int n = (int)min((int64_t)DISPATCH_CHUNK, A.entries - from);
        const int rounds = (n + DISPATCH_THREADS - 1) / DISPATCH_THREADS;  // of 32 entries per warp: few entries are spread over the warps
        const int64_t begin = from + warp * 32 * rounds + lane;
        int e[DISPATCH_PER], rank[DISPATCH_PER];
#pragma unroll
        for (int j = 0; j < DISPATCH_PER; ++j) {
            const int v = j < rounds && begin + 32 * j < A.entries ? ld(A.idx + begin + 32 * j) : -1;
            e[j] = (unsigned)v < (unsigned)E ? v : E;  // E: dropped
        }
#pragma unroll
        for (int j = 0; j < DISPATCH_PER; ++j) {
            const unsigned valid = __ballot_sync(FULL, e[j] < E);
            if (valid == 0) continue;
            const unsigned peers = valid & match_bits<BITS>((uint32_t)e[j]);
            const int before = __popc(peers & ((1u << lane) - 1u));
            rank[j] = e[j] < E ? mine[e[j]] + before : 0;
            __syncwarp();
            if (e[j] < E && before == 0) mine[e[j]] = (uint16_t)(mine[e[j]] + __popc(peers));
            __syncwarp();
        }
        __syncthreads();
        int total = 0;  // of expert `tid` in this chunk (E <= threads)
        if (tid < E) {
            int v[DISPATCH_WARPS];
#pragma unroll
            for (int w = 0; w < DISPATCH_WARPS; ++w) v[w] = hist[w * pitch + tid];
#pragma unroll
            for (int w = 0; w < DISPATCH_WARPS; ++w) {
                hist[w * pitch + tid] = (uint16_t)total;
                total += v[w];
            }
        }
        if (chunk == 0) {  // exclusive scan of the padded lengths, a thread per expert
            if (tid < E && A.blocks == 1) count[tid] = total;  // then there is one chunk too
            const int padded = tid < E ? (count[tid] + A.rows - 1) >> A.shift << A.shift : 0;
            int run = padded;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(FULL, run, o);
                if (lane >= o) run += v;
            }
            if (lane == 31) scan[warp] = run;
            __syncthreads();
            if (tid < E) {
                int base = run - padded;
                for (int w = 0; w < warp; ++w) base += scan[w];
                offset[tid] = base;
                next[tid] += base;
                if (tid == E - 1) offset[E] = base + padded;
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < DISPATCH_PER; ++j) {
            if (j < rounds && begin + 32 * j < A.entries) {
                int slot = -1;
                if (e[j] < E) {
                    slot = next[e[j]] + mine[e[j]] + rank[j];
                    if ((unsigned)slot < (unsigned)A.capacity) A.entry_of[slot] = (int32_t)(begin + 32 * j);
                    else slot = -1;  // only if the caller changes idx between the two kernels
                }
                A.slot_of[begin + 32 * j] = slot;
            }
        }
        if (chunk + 1 < A.chunks) {
            __syncthreads();
            if (tid < E) next[tid] += total;
            for (int i = tid; i < DISPATCH_WARPS * pitch / 2; i += DISPATCH_THREADS) reinterpret_cast<uint32_t *>(hist)[i] = 0;
            __syncthreads();
        }
    }
    // the tables' rest: holes of the slots, experts of the row tiles, counts and offsets; a warp per expert
    for (int i = blockIdx.x * DISPATCH_WARPS + warp; i < E; i += gridDim.x * DISPATCH_WARPS) {
        const int lo = offset[i], hi = offset[i + 1], c = count[i];
        for (int s = lo + c + lane; s < hi; s += 32) A.entry_of[s] = -1;
        for (int r = (lo >> A.shift) + lane; r < (hi >> A.shift); r += 32) A.tile_expert[r] = i;
        if (lane == 0) A.counts[i] = c, A.offsets[i] = lo;
    }
    const int all = offset[E];
    if (blockIdx.x == 0 && tid == 0) A.offsets[E] = all;
    for (int64_t s = all + (int64_t)blockIdx.x * DISPATCH_THREADS + tid; s < A.capacity; s += (int64_t)gridDim.x * DISPATCH_THREADS) A.entry_of[s] = -1;
    for (int64_t r = (all >> A.shift) + (int64_t)blockIdx.x * DISPATCH_THREADS + tid; r < (A.capacity >> A.shift); r += (int64_t)gridDim.x * DISPATCH_THREADS)
        A.tile_expert[r] = -1;
}

}  // namespace lapsum
