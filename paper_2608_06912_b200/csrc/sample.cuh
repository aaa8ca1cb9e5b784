// The next token of every row of logits: temperature, top-k, min-p, top-p, and one given random number per row.
//
//   e_i = exp((x_i - max) / T);   rank: by x, largest first, equal ones by the lower index
//   kept: the first min(top_k, #{e_i >= min_p}) of the rank, and of those the least number whose sum reaches top_p of theirs
//   token: the first i, by index, at which the kept e sum to more than u times the sum of all kept
//
// A cluster of up to 8 blocks of 512 threads has one row; each block brings its run of the row into shared memory once, every later pass reads it there.
// Or, for many long rows without top-p, one block of 1024 threads has one and reads it again, from L2: no cluster barriers and no loads from other
// blocks' memory, which take 2000 clocks and more.
//
// What bounds it.  One row (50021 tokens, 9 to 32 us with the call, by the way that its settings take): a chain of three to nine cluster barriers and the fetch of
// code that runs once.  48 x 128000 in 16 bits without filters 25.6 us (12 MB): 192 blocks on 148 SMs, so 44 SMs have two and twice the tokens; there the schedulers issue in 83 %
// of the active cycles, 47 % in the mean, some 50 instructions a token in all, 9 of them in 64 bits (their pipe is at 29 % there), with 5 warps a scheduler in the mean, and what they wait for is
// their own fixed latencies (2.4 of 11 cycles), shared memory and barriers.  256 x 128000 fp32 (131 MB, 20 us by its bytes): without filters 90 us, 256 blocks of 1024 threads
// on 148 SMs, so two rounds, 57 % of the issue slots, and waits for the second reading; with top-k, where only listed tokens are weighed, 63; rows of all kinds 187.
//
// Weights are integers, e_i 2^S rounded (S = 45 up to 2^18 tokens), from an exponential in 64 bits: their sums are exact in any order, so the
// result depends neither on the cluster nor on atomics, and it is the definition's unless u or top_p falls within vocab 2^-(S + 1) of a border, mostly some 2^-37.
// With fp32 sums one draw in a few hundred over a vocabulary of 2^17 would pick a neighbour.
//
// The short way: the row's threads form 128 groups, and the largest logits of k groups are k tokens, so nothing below the k-th of them is among
// the first k; in the same way the groups' largest weights bound the cut of top-p.  What lies above goes into a list of at most 256 tokens, and
// one block finishes it: rank, filters, draw.  Two or three cluster barriers, which are what a single row's time consists of.
//
// The long way, where k is large, the weight spread out or a value repeated: the cut of top-k and top-p is the rank's G-th token, or the one at
// which the weights reach G.  A histogram over the distance from
// the largest logit finds the bucket that holds it; its members, if they are few, are listed and sorted, otherwise buckets are
// cut again, by their keys, until one holds few tokens or one value.  What cannot hold the cut stays out of the histograms, whose atomics
// would cost more than all else: for top-k everything below the k-th largest of the threads' own maxima, for top-p the tokens that
// together weigh less than what may be missing.
// Code that runs once is bound by its fetch: 128 comparisons, unrolled, took 12700 clocks of a single row's 90000.  So the filters and the draw are
// turns of one loop around one copy of each pass, and loops are rolled where they are not the whole row's.
#pragma once
#include <climits>

#include "common.cuh"
#include "tensor_core.cuh"

namespace lapsum {

struct SampleArgs {
    const void *logits;
    int64_t stride;
    const float *u, *temperature_row, *top_p_row, *min_p_row;  // the last three may be null: one value for all rows
    const int32_t *top_k_row;
    double temperature, top_p, min_p;
    int64_t top_k;
    int32_t *token, *kept;  // kept and logprob may be null
    float *logprob;
    int vocab, chunk;  // chunk: tokens of a block, a multiple of 128
    int cluster;
    int bits;  // S
};

constexpr int SAMPLE_BUCKETS = 1024, SAMPLE_LIST = 256, SAMPLE_GROUPS = 128;
// tokens that the groups' bound lets through: 128 ln(1 / (1 - k / 128)) if the order is random, 177 for this k
constexpr int SAMPLE_SHORT_K = 96;

// Read by the cluster's other blocks, each behind the barrier that follows its writing, and written again only behind another one (or a row's first time):
//   key_max, groups      behind the row's first barrier; groups are never written again, key_min and key_max in descend(), behind crossing()'s
//   block_mass, _count   sum_and_find(): the next one comes behind the barriers of what lies between, crossing() or finish_short(), or was the row's last
//   mass, count          as histograms, between crossing()'s two barriers; before and afterwards they are this block's own
//   slice_...            behind crossing()'s second; written between the next one's two
//   list, list_count     written by all blocks, read behind finish_list()'s or finish_short()'s; the count is cleared behind crossing()'s first
//   index                descend(), between its last two; elsewhere this block's own
// All the rest, warp_mass among it, is this block's alone.  How many barriers a block passes depends on values that all blocks read alike.
template <int THREADS, bool TOP_P>
struct alignas(16) SampleShared {
    static constexpr int NEAR = TOP_P ? 128 : 1;  // tokens of a warp's near list, which top-p alone needs: with 64 KB of the row two blocks of 512 threads fit an SM
    double power[64 * 16];  // 2^(j / 64 + S), sixteen of each: a lane reads its own, so that no two meet in a bank
    unsigned long long mass[SAMPLE_BUCKETS];
    uint32_t count[SAMPLE_BUCKETS];
    unsigned long long slice_mass[SAMPLE_BUCKETS];  // this block's share of the buckets, summed over the cluster
    uint32_t slice_count[SAMPLE_BUCKETS];
    unsigned long long list[SAMPLE_LIST], sorted[SAMPLE_LIST];
    uint32_t near[THREADS / 32][NEAR], near_of[THREADS / 32];  // where in this block's run the tokens from a bound on are, for top-p
    uint32_t groups[SAMPLE_GROUPS], ranked[SAMPLE_GROUPS];  // this block's groups' largest keys; those of all blocks, largest first
    unsigned long long warp_mass[THREADS / 32];
    uint32_t warp_count[THREADS / 32];
    unsigned long long block_mass, slice_total;
    uint32_t block_count, list_count;
    uint32_t key_min, key_max;
    int index;
    // results of one block's search, for its own threads
    unsigned long long above;
    uint32_t bucket, members;
    unsigned long long cut;
};

__device__ __forceinline__ unsigned long long far_u64(const void *p, uint32_t rank)
{
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(in_block(smem_u32(p), rank)) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t far_u32(const void *p, uint32_t rank)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(in_block(smem_u32(p), rank)) : "memory");
    return v;
}
__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}
__device__ __forceinline__ unsigned long long warp_scan(unsigned long long v, int lane)  // inclusive
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long b = __shfl_up_sync(FULL, v, o);
        if (lane >= o) v += b;
    }
    return v;
}

// The same variable of all blocks of the cluster, 0 beyond them: eight loads at once (a loop would wait for each, a microsecond a piece)
__device__ __forceinline__ void far_all(const unsigned long long *p, int cluster, unsigned long long (&v)[8])
{
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] = r < cluster ? far_u64(p, r) : 0;
}
__device__ __forceinline__ void far_all(const uint32_t *p, int cluster, uint32_t (&v)[8])
{
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] = r < cluster ? far_u32(p, r) : 0;
}

// One row as one block sees it
template <typename T, int THREADS, bool RESIDENT, bool TOP_P>
struct SampleRow {
    static constexpr int V = Io<T>::V, WARPS = THREADS / 32;
    const SampleArgs &P;
    SampleShared<THREADS, TOP_P> &S;
    const T *row, *mine;     // the row in memory; this block's run of it in shared memory
    int begin, len, padded;  // the run; `padded` is a multiple of V
    bool whole;              // vectors of the run in memory are aligned
    uint32_t rank, home;     // home: the block that holds the row's list and finishes it
    int tid, lane, warp;
    float top;               // the largest logit
    double factor;           // 64 log2(e) / T
    float none_x;            // logits up to here weigh less than half of the last digit: nothing
    float cut_x;             // kept: x > cut_x, or x == cut_x and index <= cut_i
    int cut_i;

    // A NaN passes no comparison, so it is never kept.
    __device__ __forceinline__ float at(int i) const { return RESIDENT ? Io<T>::from_storage(mine[i]) : Io<T>::from_storage(ld(row + begin + i)); }
    __device__ __forceinline__ void get(int i, float (&x)[V]) const  // V tokens from position i of the run on; -inf beyond the row
    {
        if constexpr (RESIDENT) {
            Io<T>::unpack(*reinterpret_cast<const typename Io<T>::Vec *>(mine + i), x);
        } else if (whole && i + V <= len) {
            Io<T>::unpack(ld(reinterpret_cast<const typename Io<T>::Vec *>(row + begin + i)), x);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = i + j < len ? Io<T>::from_storage(ld(row + begin + i + j)) : -CUDART_INF_F;
        }
    }
    // f(x, i) for vectors from position b on, one per lane, up to b1: Q loads at once where a warp's are all whole.  All lanes call f, with -inf beyond b1.
    template <int Q, typename F>
    __device__ __forceinline__ void stream(int b, int b1, int step, F f) const
    {
        for (; b < b1; b += Q * step) {
            const int end = b + (Q - 1) * step + 32 * V, i = b + lane * V;
            if (RESIDENT ? end <= b1 : whole && end <= min(b1, len)) {
                typename Io<T>::Vec q[Q];
                const typename Io<T>::Vec *const from = reinterpret_cast<const typename Io<T>::Vec *>((RESIDENT ? mine : row + begin) + i);
#pragma unroll
                for (int j = 0; j < Q; ++j) q[j] = ld(from + j * (step / V));
#pragma unroll
                for (int j = 0; j < Q; ++j) {
                    float x[V];
                    Io<T>::unpack(q[j], x);
                    f(x, i + j * step);
                }
            } else {
#pragma unroll 1
                for (int j = 0; j < Q; ++j) {
                    float x[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) x[v] = -CUDART_INF_F;
                    if (i + j * step < b1) get(i + j * step, x);
                    __syncwarp();
                    f(x, i + j * step);
                }
            }
        }
    }
    template <int Q, typename F>
    __device__ __forceinline__ void stream_all(F f) const { stream<Q>(warp * 32 * V, padded, THREADS * V, f); }
    __device__ __forceinline__ static float largest(const float (&x)[V])
    {
        float m = x[0];
#pragma unroll
        for (int j = 1; j < V; ++j) m = fmaxf(m, x[j]);
        return m;
    }
    __device__ __forceinline__ static uint32_t key_of(float x) { return float_to_key(x + 0.f); }  // -0 and 0 are equal
    // fp32 to fp64 by its bits: the conversion instruction runs at a sixteenth of the rate.  0 becomes 2^-127, what is below the normal range is off by
    // up to 2^-127: nothing at a temperature from 1e-27 on.  (Exact conversions there alone, behind a branch, made rows of all temperatures 3 to 8 % slower.)
    __device__ __forceinline__ static double widened(float x)
    {
        const int b = __float_as_int(x);
        return __hiloint2double(((b >> 3) & 0x8fffffff) + 0x38000000, b << 29);
    }
    // 2^52 + e^((x - top) / T) 2^S, rounded, for an x from none_x on: exponent and one of 64 fractions by table, the rest by a polynomial (P. T. P. Tang,
    // Table-driven implementation of the exponential function, 1989).  The remainder is below ln 2 / 128, so five terms leave 2^-44 of the
    // weight at its ends.  Nine operations in 64 bits and a dozen others; a library exponential and its conversions took 45 in all.  (512 fractions, read from
    // one copy, save one of the nine, but their bank conflicts took as long as all the rest: 50000 clocks for 128000 tokens on one SM.)
    __device__ __forceinline__ unsigned long long raised(float x) const
    {
        const double d = widened(x) - widened(top);
        const double shifted = fma(d, factor, 6755399441055744.0);  // 1.5 2^52: rounds to whole numbers
        const int n = __double2loint(shifted);
        const double f = fma(d, factor, 6755399441055744.0 - shifted);
        constexpr double C = 0.69314718055994530942 / 64;
        double p = fma(f, C * C * C * C / 24, C * C * C / 6);
        p = fma(f, p, C * C / 2);
        p = fma(f, p, C);
        p = fma(f, p, 1.0);
        const double t = S.power[(n & 63) * 16 + (lane & 15)];
        const double scale = __hiloint2double(__double2hiint(t) + (int)((uint32_t)(n & ~63) << 14), __double2loint(t));
        return (unsigned long long)__double_as_longlong(fma(scale, p, 4503599627370496.0));
    }
    static constexpr unsigned long long RAISED = 0x433ull << 52;  // 2^52
    __device__ __forceinline__ unsigned long long weight(float x) const { return raised(fmaxf(x, none_x)) - RAISED; }

    __device__ __forceinline__ void barrier() const
    {
        __syncwarp();
        if (P.cluster > 1) cluster_barrier();
        else __syncthreads();
    }
    // the same in two: between them a block goes on with what is its own
    __device__ __forceinline__ void arrive() const
    {
        __syncwarp();
        if (P.cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    }
    __device__ __forceinline__ void wait() const
    {
        __syncwarp();
        if (P.cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        else __syncthreads();
    }

    // ---- sums by index: of the kept tokens' weights, or (ONES) of the tokens equal to `value` ----
    // V tokens from position i of the run on: their sum (v: each), and in n how many are kept.  A token that weighs nothing is taken at none_x, where the
    // rounding leaves 0; what the raised weights have too much goes off at the end.
    template <bool ONES>
    __device__ __forceinline__ unsigned long long values(float value, const float (&x)[V], int i, uint32_t &n, unsigned long long (&v)[V]) const
    {
        unsigned long long sum = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = 0;
        if constexpr (ONES) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = x[j] == value, sum += v[j];
        } else {
            if (largest(x) >= cut_x) {
                uint32_t m = 0;
                if (cut_i == INT_MAX) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const unsigned long long w = raised(fmaxf(x[j], none_x));
                        if (x[j] >= cut_x) v[j] = w, sum += w, ++m;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const unsigned long long w = raised(fmaxf(x[j], none_x));
                        if (x[j] > cut_x || (x[j] == cut_x && begin + i + j <= cut_i)) v[j] = w, sum += w, ++m;
                    }
                }
                sum -= m * RAISED;
                n += m;
            }
        }
        return sum;
    }
    struct Span {
        int i0, i1;
    };
    __device__ __forceinline__ Span run_of(int w) const  // a warp's tokens: a run of its own
    {
        const int per = (padded + WARPS * 32 * V - 1) / (WARPS * 32 * V) * (32 * V), i0 = min(w * per, padded);
        return Span{i0, min(i0 + per, padded)};
    }
    // Total and count over the cluster, behind a barrier; the index of the token at which the values sum to more than goal(total) comes to `found` in one
    // thread of the cluster where one is wanted; then a wait() is to follow.
    template <bool ONES, typename G, typename F>
    __device__ __forceinline__ unsigned long long sum_and_find(float value, bool wanted, G goal_of, F found) const
    {
        unsigned long long v[V], sum = 0;
        uint32_t n = 0;
        {
            const Span span = run_of(warp);
            stream<2>(span.i0, span.i1, 32 * V, [&](const float (&x)[V], int i) { sum += values<ONES>(value, x, i, n, v); });
        }
        __syncwarp();
        sum = warp_sum(sum);
        n = __reduce_add_sync(FULL, n);
        if (lane == 0) S.warp_mass[warp] = sum, S.warp_count[warp] = n;
        __syncthreads();
        const unsigned long long own = lane < WARPS ? S.warp_mass[lane] : 0;
        if (warp == 0) {
            sum = warp_sum(own);
            n = __reduce_add_sync(FULL, lane < WARPS ? S.warp_count[lane] : 0);
            if (lane == 0) S.block_mass = sum, S.block_count = n;
        }
        barrier();
        // a lane per block: loads from other blocks' memory are slow, four for each of 32 lanes in every warp took 8000 clocks
        const unsigned long long mass = lane < P.cluster ? far_u64(&S.block_mass, lane) : 0, blocks_upto = warp_scan(mass, lane),
                                 total = __shfl_sync(FULL, blocks_upto, 31);
        const uint32_t count = __reduce_add_sync(FULL, lane < P.cluster ? far_u32(&S.block_count, lane) : 0);
        if (!wanted) return total;
        arrive();  // the other blocks' sums have been read
        const unsigned long long goal = goal_of(total);
        const int holder = __ffs(__ballot_sync(FULL, goal < blocks_upto)) - 1;
        if (holder == (int)rank) {  // the whole block goes over the run of the warp that has it, a vector per thread
            const unsigned long long upto = __shfl_sync(FULL, blocks_upto - mass, holder) + warp_scan(own, lane);
            const int which = __ffs(__ballot_sync(FULL, lane < WARPS && goal < upto)) - 1;
            unsigned long long before = __shfl_sync(FULL, upto - own, which);
            const Span span = run_of(which);
            for (int base = span.i0; base < span.i1; base += THREADS * V) {
                const int i = base + tid * V;
                unsigned long long s = 0;
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = 0;
                if (i < span.i1) {
                    float x[V];
                    get(i, x);
                    s = values<ONES>(value, x, i, n, v);
                }
                __syncwarp();
                unsigned long long run = warp_scan(s, lane);
                __syncthreads();
                if (lane == 31) S.warp_mass[warp] = run;
                __syncthreads();
                unsigned long long lower = before;
#pragma unroll 4
                for (int w = 0; w < WARPS; ++w) {
                    if (w < warp) lower += S.warp_mass[w];
                    before += S.warp_mass[w];
                }
                run += lower - s;
                if (run <= goal && goal < run + s) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const unsigned long long w = ONES || v[j] == 0 ? v[j] : v[j] - RAISED;
                        if (run <= goal && goal < run + w) found(begin + i + j, total, count);
                        run += w;
                    }
                }
                if (goal < before) break;
            }
        }
        return total;
    }

    // ---- the list ----
    // which tokens: from `low` on; with members: those of one bucket by distance (shift < 0) or of a range of keys
    struct Which {
        float low, scale;
        uint32_t bucket, k0, k1;
        int shift;
        bool members, mass;  // mass: only tokens that weigh something
    };
    __device__ __forceinline__ static uint32_t linear(float top, float scale, float x)  // falls as x rises
    {
        return (uint32_t)min(SAMPLE_BUCKETS - 1, (int)((top - x) * scale));
    }
    __device__ __forceinline__ bool accepts(const Which &w, float x) const
    {
        if (!(x >= w.low)) return false;
        if (w.members) {
            if (w.shift < 0) {
                if (linear(top, w.scale, x) != w.bucket) return false;
            } else if (key_of(x) < w.k0 || key_of(x) > w.k1) {
                return false;
            }
        }
        return !w.mass || weight(x) != 0;
    }
    // tokens of all blocks into the home block's list; its counter tells whether they were too many
    __device__ __forceinline__ void append(const Which &which, bool near) const
    {
        const uint32_t counter = in_block(smem_u32(&S.list_count), home), list = in_block(smem_u32(&S.list[0]), home);
        const auto take = [&](int i) {
            const float x = at(i);
            if (!accepts(which, x)) return true;
            uint32_t to;
            asm volatile("atom.shared::cluster.add.u32 %0, [%1], 1;" : "=r"(to) : "r"(counter) : "memory");
            const unsigned long long item = ((unsigned long long)key_of(x) << 32) | (0xffffffffu - (uint32_t)(begin + i));
            if (to < SAMPLE_LIST) asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(list + 8 * to), "l"(item) : "memory");
            return to < SAMPLE_LIST;
        };
        bool room = true;
        if (near) {
            for (int i = lane; i < (int)S.near_of[warp] && room; i += 32) room = take((int)S.near[warp][i]);
        } else {
            stream_all<4>([&](const float (&x)[V], int i0) {
                if (room && largest(x) >= which.low)
#pragma unroll 1
                    for (int i = i0; i < min(i0 + V, len) && room; ++i) room = take(i);
            });
        }
        __syncwarp();
    }
    // `sorted` <- the home block's list of n items, largest first (by logit, then by the lower index)
    __device__ __forceinline__ void sort_list(int n) const
    {
        unsigned long long item = 0;
        if (tid < n) {
            item = far_u64(&S.list[tid], home);
            S.mass[tid] = item;  // a copy: the histogram is done with
        }
        __syncthreads();
        if (tid < n) {
            int to = 0;
#pragma unroll 2
            for (int j = 0; j < n; ++j) to += S.mass[j] > item;
            S.sorted[to] = item;
        }
        __syncthreads();
    }
    // `ranked` <- the groups' largest keys, of all blocks, in order.  The last bits make way for the group's number: a bound a little lower.
    __device__ __forceinline__ void rank_groups() const
    {
        const int each = SAMPLE_GROUPS / P.cluster;
        uint32_t *const all = S.count;  // not yet in use
        uint32_t key = 0;
        if (tid < SAMPLE_GROUPS) all[tid] = key = (far_u32(&S.groups[tid % each], tid / each) & ~(SAMPLE_GROUPS - 1u)) | (uint32_t)tid;
        __syncthreads();
        if (tid < SAMPLE_GROUPS) {
            int to = 0;
#pragma unroll 2
            for (int j = 0; j < SAMPLE_GROUPS; j += 4) {
                const uint4 q = *reinterpret_cast<const uint4 *>(all + j);
                to += (q.x > key) + (q.y > key) + (q.z > key) + (q.w > key);
            }
            S.ranked[to] = key & ~(SAMPLE_GROUPS - 1u);
        }
        __syncthreads();
    }

    // ---- the histogram ----
    // Over the tokens of `which` (by distance, or by key within k0 .. k1), in buckets of falling x; from the near list where there is one.
    __device__ __forceinline__ void histogram(const Which &which, bool near) const
    {
        for (int i = tid; i < SAMPLE_BUCKETS; i += THREADS) S.count[i] = 0, S.mass[i] = 0;
        __syncthreads();
        const int n = near ? (int)S.near_of[warp] : len;
#pragma unroll 2
        for (int i = near ? lane : tid; i < n; i += near ? 32 : THREADS) {
            const float x = at(near ? (int)S.near[warp][i] : i);
            if (!(x >= which.low)) continue;
            uint32_t b;
            if (which.shift < 0) {
                b = linear(top, which.scale, x);
            } else {
                const uint32_t k = key_of(x);
                if (k < which.k0 || k > which.k1) continue;
                b = (which.k1 - k) >> which.shift;
            }
            if (which.mass) {
                const unsigned long long w = weight(x);
                if (w == 0) continue;  // never at the border
                atomicAdd(&S.mass[b], w);
            }
            atomicAdd(&S.count[b], 1u);
        }
        __syncwarp();
    }
    // The first bucket at which the cluster's counts (or weights) from the largest on reach the goal, into S.bucket, .members and .above; false: they
    // never do.
    __device__ __forceinline__ bool crossing(bool mass, unsigned long long goal) const
    {
        barrier();
        if (tid == 0) S.list_count = 0;  // the last list has been read, the next one comes behind another barrier
        const int share = SAMPLE_BUCKETS / P.cluster;
        for (int i = tid; i < share; i += THREADS) {
            uint32_t c = 0, cs[8];
            unsigned long long m = 0, ms[8];
            far_all(&S.count[rank * share + i], P.cluster, cs);
            far_all(&S.mass[rank * share + i], P.cluster, ms);
#pragma unroll
            for (int r = 0; r < 8; ++r) c += cs[r], m += ms[r];
            S.slice_count[i] = c;
            S.slice_mass[i] = mass ? m : c;
        }
        __syncthreads();
        if (warp == 0) {
            unsigned long long m = 0;
            for (int i = lane; i < share; i += 32) m += S.slice_mass[i];
            m = warp_sum(m);
            if (lane == 0) S.slice_total = m;
        }
        barrier();
        // the slice that holds the goal; a copy of it (the histogram has been read); one warp walks the copy
        unsigned long long above = 0, upto = 0, part[8];
        int q = P.cluster;
        far_all(&S.slice_total, P.cluster, part);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            if (r < P.cluster && q == P.cluster && upto + part[r] >= goal) q = r, above = upto;
            upto += part[r];
        }
        if (q == P.cluster) return false;
        for (int i = tid; i < share; i += THREADS) {
            S.mass[i] = far_u64(&S.slice_mass[i], q);
            S.count[i] = far_u32(&S.slice_count[i], q);
        }
        __syncthreads();
        if (warp == 0) {
            const int each = share / 32;
            unsigned long long s = 0;
            for (int i = 0; i < each; ++i) s += S.mass[lane * each + i];
            const unsigned long long run = above + warp_scan(s, lane);
            if (lane == __ffs(__ballot_sync(FULL, run >= goal)) - 1) {
                unsigned long long a = run - s;
                for (int i = lane * each; i < (lane + 1) * each; ++i) {
                    a += S.mass[i];
                    if (a >= goal) {
                        S.bucket = q * share + i;
                        S.members = S.count[i];
                        S.above = a - S.mass[i];
                        break;
                    }
                }
            }
        }
        __syncthreads();
        return true;
    }
    // `near` <- where this block's tokens from `low` on are, so that weights, which cost much for a token here and there, are computed densely
    __device__ __forceinline__ bool bring_near(float low) const
    {
        uint32_t to = 0;  // a list for every warp, of its own tokens
        const unsigned lower = (1u << lane) - 1;
        stream_all<4>([&](const float (&x)[V], int i) {
            if (!__any_sync(FULL, largest(x) >= low)) return;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const unsigned who = __ballot_sync(FULL, x[j] >= low);
                const uint32_t at_ = to + __popc(who & lower);
                if (x[j] >= low && at_ < SampleShared<THREADS, TOP_P>::NEAR) S.near[warp][at_] = (uint32_t)(i + j);
                to += __popc(who);
            }
        });
        if (lane == 0) S.near_of[warp] = to;
        return !__syncthreads_or(to > SampleShared<THREADS, TOP_P>::NEAR);
    }

    // (cut_x, cut_i) <- the token of the rank at which the counts (or weights) of the tokens from `low` on reach the goal
    __device__ __forceinline__ void descend(bool mass, float low, float range, unsigned long long goal)
    {
        Which which{low, range > 0.f ? SAMPLE_BUCKETS / range : 0.f, 0, 0, 0, -1, false, mass};
        const bool near = mass && bring_near(low);
        histogram(which, near);
        if (!crossing(mass, goal)) return;
        which.members = true;
        unsigned long long above = S.above;
        for (int level = 0; level < 8; ++level) {  // distance, then 32 bits of key in steps of ten: five at most
            which.bucket = S.bucket;
            if (S.members <= SAMPLE_LIST) {
                finish_list(which, near && which.shift < 0, goal, above);
                return;
            }
            if (which.shift < 0) {  // the keys that the bucket holds
                if (tid == 0) S.key_min = 0xffffffffu, S.key_max = 0;
                __syncthreads();
                uint32_t lo = 0xffffffffu, hi = 0;
                for (int i = tid; i < len; i += THREADS) {
                    const float x = at(i);
                    if (accepts(which, x)) lo = min(lo, key_of(x)), hi = max(hi, key_of(x));
                }
                __syncwarp();
                lo = __reduce_min_sync(FULL, lo), hi = __reduce_max_sync(FULL, hi);
                if (lane == 0) atomicMin(&S.key_min, lo), atomicMax(&S.key_max, hi);
                barrier();
                uint32_t los[8], his[8];
                far_all(&S.key_min, P.cluster, los);
                far_all(&S.key_max, P.cluster, his);
                which.k0 = 0xffffffffu, which.k1 = 0;
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < P.cluster) which.k0 = min(which.k0, los[r]), which.k1 = max(which.k1, his[r]);
            } else {
                which.k1 -= which.bucket << which.shift;
                const uint32_t span = (1u << which.shift) - 1;
                which.k0 = which.k1 - which.k0 < span ? which.k0 : which.k1 - span;
            }
            if (which.k0 == which.k1) {  // one value: its first tokens by index, as many as are still missing
                const float x0 = key_to_float(which.k0);
                const unsigned long long missing = goal - above, each = mass ? weight(x0) : 1, n = (missing + each - 1) / each;
                if (tid == 0) S.index = -1;
                sum_and_find<true>(x0, true, [&](unsigned long long) { return n - 1; }, [&](int index, unsigned long long, uint32_t) { S.index = index; });
                wait();
                barrier();
                uint32_t indices[8];
                far_all(reinterpret_cast<const uint32_t *>(&S.index), P.cluster, indices);
                cut_x = x0, cut_i = INT_MAX;
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < P.cluster && (int)indices[r] >= 0) cut_i = (int)indices[r];
                barrier();
                return;
            }
            which.shift = 0;
            while (((which.k1 - which.k0) >> which.shift) >= SAMPLE_BUCKETS) ++which.shift;
            histogram(which, false);
            crossing(mass, goal - above);
            above += S.above;
        }
    }
    // The bucket's tokens through the list; every block sorts a copy and walks it.
    __device__ __forceinline__ void finish_list(Which which, bool near, unsigned long long goal, unsigned long long above)
    {
        if (which.shift >= 0) {  // the bucket's range of keys
            which.k1 -= which.bucket << which.shift;
            const uint32_t span = (1u << which.shift) - 1;
            which.k0 = which.k1 - which.k0 < span ? which.k0 : which.k1 - span;
        }
        append(which, near);
        barrier();
        const int n = min((int)far_u32(&S.list_count, home), SAMPLE_LIST);
        sort_list(n);
        if (warp == 0) {
            constexpr int EACH = SAMPLE_LIST / 32;
            unsigned long long s = 0;
#pragma unroll 1
            for (int i = lane * EACH; i < (lane + 1) * EACH; ++i) {
                const unsigned long long w = i >= n ? 0 : which.mass ? weight(key_to_float((uint32_t)(S.sorted[i] >> 32))) : 1;
                S.mass[i] = w;
                s += w;
            }
            const unsigned long long run = above + warp_scan(s, lane);
            const unsigned who = __ballot_sync(FULL, run >= goal);
            if (who && lane == __ffs(who) - 1) {
                unsigned long long a = run - s;
#pragma unroll 1
                for (int i = lane * EACH; i < (lane + 1) * EACH; ++i) {
                    a += S.mass[i];
                    if (a >= goal) {
                        S.cut = S.sorted[i];
                        break;
                    }
                }
            }
        }
        __syncthreads();
        cut_x = key_to_float((uint32_t)(S.cut >> 32)), cut_i = (int)(0xffffffffu - (uint32_t)S.cut);
    }

    // ---- results ----
    __device__ __forceinline__ void give(int64_t r, int token, float logprob, int kept) const
    {
        P.token[r] = token;
        if (P.logprob) P.logprob[r] = logprob;
        if (P.kept) P.kept[r] = kept;
    }
    // from the logit: the weight itself has lost digits where it is small
    __device__ __forceinline__ void give_drawn(int64_t r, int index, float x, double T_, unsigned long long total, uint32_t count) const
    {
        const double z = ((double)x - (double)top) / T_;
        give(r, index, (float)(z - log((double)total / (double)(1ull << P.bits))), (int)count);
    }
    __device__ __forceinline__ static unsigned long long reach(double p, unsigned long long total)  // what p of the total takes
    {
        const unsigned long long g = (unsigned long long)ceil(p * (double)total);
        return g < 1 ? 1 : g < total ? g : total;
    }
    __device__ __forceinline__ static unsigned long long drawn(float u, unsigned long long total)
    {
        const unsigned long long g = (unsigned long long)((double)u * (double)total);
        return g < total ? g : total - 1;
    }

    // The short way: the tokens from `low` on, which hold everything that k and p leave of those from cut_x on, through the list.  `all`: the weight
    // of all tokens from cut_x on, for p without k.  False: they are too many, and nothing has happened.
    __device__ __forceinline__ bool finish_short(int64_t r, float low, int64_t k, double p, float u, double T_, unsigned long long all) const
    {
        append(Which{low, 0.f, 0, 0, 0, -1, false, false}, false);
        barrier();
        const uint32_t n = far_u32(&S.list_count, home);
        if (n > SAMPLE_LIST) {
            barrier();
            return false;
        }
        arrive();
        if (rank == home) {
            sort_list((int)n);
            const bool real = tid < (int)n;
            const unsigned long long item = real ? S.sorted[tid] : 0;
            const float x = key_to_float((uint32_t)(item >> 32));
            const uint32_t back = (uint32_t)item;  // falls with the index
            const bool first = real && (k <= 0 || tid < k);
            const unsigned long long w = first ? weight(x) : 0;
            // running sums in the rank's order
            unsigned long long run = warp_scan(w, lane);
            if (lane == 31) S.warp_mass[warp] = run;
            S.mass[tid] = w;
            if (tid < SAMPLE_LIST) S.list[tid] = back;
            if (tid == 0) S.members = 0;
            __syncthreads();
            unsigned long long total = 0;
#pragma unroll 1
            for (int i = 0; i < SAMPLE_LIST / 32; ++i) {
                if (i < warp) run += S.warp_mass[i];
                total += S.warp_mass[i];
            }
            const unsigned long long goal = p < 1 ? reach(p, k > 0 ? total : all) : ~0ull;
            if (first && run - w < goal) atomicAdd(&S.members, 1u);  // all before the goal is reached, and the one that reaches it
            __syncthreads();
            const int kept = (int)S.members;
            if (tid == kept - 1) S.above = run;
            __syncthreads();
            total = S.above;
            const unsigned long long draw = drawn(u, total);
            if (tid < kept) {  // by index
                unsigned long long upto = 0;
#pragma unroll 2
                for (int j = 0; j < kept; ++j)
                    if ((uint32_t)S.list[j] >= back) upto += S.mass[j];
                if (upto - w <= draw && draw < upto) give_drawn(r, (int)(0xffffffffu - back), x, T_, total, (uint32_t)kept);
            }
        }
        wait();  // the list's block stays until its count has been read
        return true;
    }

    __device__ __forceinline__ void run(int64_t r)
    {
        // the run, and its largest logit
        float most = -CUDART_INF_F;
        if constexpr (RESIDENT) {
            T *const to = const_cast<T *>(mine);
            const T *const from = row + begin;
            int done = 0;
            if ((reinterpret_cast<uintptr_t>(from) & 15) == 0) {
                done = len / V * V;
                const int each = THREADS * V;
                for (int i = tid * V; i < done; i += 4 * each) {
                    typename Io<T>::Vec q[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (i + j * each < done) q[j] = __ldcs(reinterpret_cast<const typename Io<T>::Vec *>(from + i + j * each));
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (i + j * each < done) {
                            *reinterpret_cast<typename Io<T>::Vec *>(to + i + j * each) = q[j];
                            float x[V];
                            Io<T>::unpack(q[j], x);
#pragma unroll
                            for (int v = 0; v < V; ++v) most = fmaxf(most, x[v]);  // not a NaN
                        }
                }
            }
            for (int i = done + tid; i < padded; i += THREADS) {
                const float x = i < len ? Io<T>::from_storage(ld(from + i)) : -CUDART_INF_F;
                Io<T>::store1(to + i, x);
                most = fmaxf(most, x);
            }
        } else {
            stream_all<4>([&](const float (&x)[V], int) { most = fmaxf(most, largest(x)); });
        }
        __syncwarp();
        uint32_t key = key_of(most), group = key;
        const int of_a_group = THREADS / SAMPLE_GROUPS * P.cluster;  // threads
        for (int o = 1; o < of_a_group; o <<= 1) group = max(group, __shfl_xor_sync(FULL, group, o));
        if (tid % of_a_group == 0) S.groups[tid / of_a_group] = group;
        key = __reduce_max_sync(FULL, key);
        if (lane == 0) atomicMax(&S.key_max, key);
        barrier();
        uint32_t keys[8];
        far_all(&S.key_max, P.cluster, keys);
#pragma unroll
        for (int q = 0; q < 8; ++q) key = max(key, keys[q]);
        top = key_to_float(key);

        const double T_ = P.temperature_row ? (double)ld(P.temperature_row + r) : P.temperature;
        const double p = !TOP_P ? 1.0 : P.top_p_row ? (double)ld(P.top_p_row + r) : P.top_p, m = P.min_p_row ? (double)ld(P.min_p_row + r) : P.min_p;
        const int64_t k = P.top_k_row ? (int64_t)ld(P.top_k_row + r) : P.top_k;
        const float u = ld(P.u + r);
        const bool valid = T_ >= 0 && T_ < CUDART_INF && p > 0 && m >= 0 && m <= 1 && u >= 0.f && u < 1.f;  // false for NaN
        if (!valid || top == -CUDART_INF_F) {
            if (rank == home && tid == 0) give(r, -1, valid ? -CUDART_INF_F : CUDART_NAN_F, 0);
            barrier();
            return;
        }
        const bool greedy = T_ == 0 || k == 1;
        if (greedy || top == CUDART_INF_F) {
            // the first of the largest; or infinities, beside which nothing else weighs anything: they share the draw, as far as the filters leave them
            unsigned long long left = 1;
            sum_and_find<true>(
                top, true,
                [&](unsigned long long total) {
                    if (!greedy) left = k > 0 && (unsigned long long)k < total ? (unsigned long long)k : total;
                    if (!greedy && p < 1) left = reach(p, left);
                    return drawn(u, left);
                },
                [&](int index, unsigned long long, uint32_t) { give(r, index, (float)-log((double)left), (int)left); });
            wait();
            return;
        }
        factor = 64 * 1.4426950408889634074 / T_;
        constexpr float LOWEST = -3.402823466e38f;
        none_x = fmaxf(fminf(__double2float_rd((double)top - T_ * 0.69314718055994530942 * (P.bits + 2)), nextafterf(top, -CUDART_INF_F)), LOWEST);
        // where the next logit below already weighs nothing, it is put where the exponent still has room
        if (none_x == nextafterf(top, -CUDART_INF_F)) factor = fmin(factor, 64.0 * (P.bits + 4) / ((double)top - (double)none_x));
        cut_x = LOWEST, cut_i = INT_MAX;
        if (m > 0) {  // the least x with (top - x) / T <= -log(min_p)
            const double far = -log(m), inv = 1.0 / T_;
            float x = fminf(fmaxf((float)((double)top - far * T_), cut_x), top);
            const auto inside = [&](float v) { return ((double)top - (double)v) * inv <= far; };
#pragma unroll 1
            for (int i = 0; i < 4 && !inside(x); ++i) x = nextafterf(x, CUDART_INF_F);
#pragma unroll 1
            for (int i = 0; i < 4 && inside(nextafterf(x, -CUDART_INF_F)); ++i) x = nextafterf(x, -CUDART_INF_F);
            cut_x = fmaxf(cut_x, fminf(x, top));  // at a temperature whose reciprocal is infinite nothing is inside
        }
        // turns: the cut of top-k; the sum, the cut of top-p; the sum, the draw
        bool need_k = k > 0 && k < P.vocab, need_p = p < 1;
        const bool by_k = need_k;
        for (int turn = 0; turn < 3; ++turn) {
            unsigned long long goal = (unsigned long long)k, total = 0;
            if (!need_k) {
                total = sum_and_find<false>(
                    0.f, !need_p, [&](unsigned long long all) { return drawn(u, all); },
                    [&](int index, unsigned long long all, uint32_t count) { give_drawn(r, index, at(index - begin), T_, all, count); });
                if (!need_p) break;
                goal = reach(p, total);
            }
            // a bound of the cut by the groups, for k or for p without k: the k-th of them, or the first at which their weights reach the goal
            float low = cut_x;
            if (need_k || !by_k) {
                rank_groups();
                int to = k <= SAMPLE_GROUPS ? (int)k - 1 : SAMPLE_GROUPS;
                if (!need_k) {
                    if (warp == 0) {
                        constexpr int EACH = SAMPLE_GROUPS / 32;
                        unsigned long long s = 0;
#pragma unroll 1
                        for (int i = lane * EACH; i < (lane + 1) * EACH; ++i) {
                            const float x = key_to_float(S.ranked[i]);
                            const unsigned long long w = x >= cut_x ? weight(x) : 0;
                            S.mass[i] = w;
                            s += w;
                        }
                        unsigned long long upto = warp_scan(s, lane);
                        int first = SAMPLE_GROUPS;
#pragma unroll 1
                        for (int i = (lane + 1) * EACH - 1; i >= lane * EACH; --i) {
                            if (upto >= goal) first = i;
                            upto -= S.mass[i];
                        }
                        first = __reduce_min_sync(FULL, first);
                        if (lane == 0) S.index = first;
                    }
                    __syncthreads();
                    to = S.index;
                }
                if (to < SAMPLE_GROUPS) low = fmaxf(low, key_to_float(S.ranked[to]));
                if (to < SAMPLE_SHORT_K && finish_short(r, low, by_k ? k : 0, p, u, T_, total)) return;
            }
            float range = fminf(top - low, 32.f);
            if (!need_k) {
                // tokens of at most this weight are together no more than total - goal, so the goal is reached before them
                const double light = (double)((total - goal) / (unsigned)P.vocab) / (double)(1ull << P.bits);
                low = fmaxf(low, light > 0 ? __double2float_rd((double)top + T_ * log(light)) : none_x);
                range = top - low;
            }
            descend(TOP_P && !need_k, low, range, goal);
            if (need_k) need_k = false;
            else need_p = false;
        }
        wait();  // nobody leaves while others read
    }
};

template <typename T, int THREADS, bool RESIDENT, bool TOP_P>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) sample_kernel(const SampleArgs P)
{
    extern __shared__ __align__(16) uint8_t raw[];
    SampleShared<THREADS, TOP_P> &S = *reinterpret_cast<SampleShared<THREADS, TOP_P> *>(raw);
    static_assert(THREADS >= SAMPLE_LIST && THREADS >= SAMPLE_GROUPS && THREADS % 64 == 0, "a thread per item");
    {
        const double power = exp2((double)(threadIdx.x & 63) / 64 + P.bits);
#pragma unroll
        for (int i = (int)threadIdx.x >> 6; i < 16; i += THREADS / 64) S.power[(threadIdx.x & 63) * 16 + i] = power;
    }
    if (threadIdx.x == 0) S.list_count = 0, S.key_max = 0;
    pdl_wait();
    __syncthreads();
    const uint32_t rank = P.cluster > 1 ? cluster_rank() : 0;
    const int begin = min((int)rank * P.chunk, P.vocab), len = min(P.chunk, P.vocab - begin);
    const int64_t r = blockIdx.x / P.cluster;
    const T *const row = static_cast<const T *>(P.logits) + r * P.stride;
    SampleRow<T, THREADS, RESIDENT, TOP_P> s{P, S, row, reinterpret_cast<const T *>(raw + sizeof(S)), begin, len, (len + Io<T>::V - 1) / Io<T>::V * Io<T>::V,
                                      (reinterpret_cast<uintptr_t>(row + begin) & 15) == 0, rank, (uint32_t)(r % P.cluster), (int)threadIdx.x,
                                      (int)threadIdx.x & 31, (int)threadIdx.x >> 5};
    s.run(r);
}

}  // namespace lapsum
