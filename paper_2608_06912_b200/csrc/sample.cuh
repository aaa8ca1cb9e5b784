// The next token of every row of logits: temperature, top-k, min-p, top-p, and one given random number per row.
//
//   e_i = exp((x_i - max) / T);   rank: by x, largest first, equal ones by the lower index
//   kept: the first min(top_k, #{e_i >= min_p}) of the rank, and of those the least number whose sum reaches top_p of theirs
//   token: the first i, by index, at which the kept e sum to more than u times the sum of all kept
//
// A cluster of 1 to 8 blocks has one row: each block brings its run of the row into shared memory once, every later pass reads it there.
//
// Weights are integers, e_i 2^S rounded (S = 45 up to 2^17 tokens), from an exponential in 64 bits: their sums are exact in any order, so the
// result depends neither on the cluster nor on atomics, and it is the definition's unless u or top_p falls within about 2^-37 of a border.
// With fp32 sums one draw in a few hundred over a vocabulary of 2^17 would pick a neighbour.
//
// The cut of top-k and top-p is the rank's G-th token, or the one at which the weights reach G.  A histogram over the distance from
// the largest logit finds the bucket that holds it; its members, if they are few, are listed and sorted, otherwise buckets are
// cut again, by their keys, until one holds few tokens or one value.
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
    int cluster, resident;
    int bits;  // S
};

constexpr int SAMPLE_THREADS = 512, SAMPLE_BUCKETS = 1024, SAMPLE_LIST = 256;

struct alignas(16) SampleShared {
    double power[64];  // 2^(j / 64)
    unsigned long long mass[SAMPLE_BUCKETS];
    unsigned long long slice_mass[SAMPLE_BUCKETS];  // this block's share of the buckets, summed over the cluster
    uint32_t count[SAMPLE_BUCKETS], slice_count[SAMPLE_BUCKETS];
    unsigned long long list[SAMPLE_LIST], sorted[SAMPLE_LIST];
    unsigned long long warp_mass[SAMPLE_THREADS / 32];
    uint32_t warp_count[SAMPLE_THREADS / 32];
    unsigned long long block_mass, slice_total_mass;  // read by the cluster's other blocks
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

template <typename T>
struct Sampler {
    static constexpr int V = Io<T>::V;
    const SampleArgs &P;
    SampleShared &S;
    const T *row, *mine;    // the row in memory; this block's run of it in shared memory
    int begin, len, padded; // the run; `padded` is a multiple of V
    uint32_t rank;
    int tid, lane, warp;
    float top;              // the largest logit
    double factor;          // 64 log2(e) / T
    float floor_x;          // the least logit that min_p leaves
    float cut_x;            // kept: x > cut_x, or x == cut_x and index <= cut_i
    int cut_i;

    __device__ __forceinline__ static float usable(float x) { return x > -CUDART_INF_F ? x + 0.f : -CUDART_INF_F; }  // no NaN, no -0
    // V tokens from position i of the run on; -inf beyond the row
    __device__ __forceinline__ void get(int i, float (&x)[V]) const
    {
        if (P.resident) {
            Io<T>::unpack(*reinterpret_cast<const typename Io<T>::Vec *>(mine + i), x);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = i + j < len ? Io<T>::from_storage(ld(row + begin + i + j)) : -CUDART_INF_F;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = usable(x[j]);
    }
    // e^((x - top) / T) 2^S: exponent and one of 64 fractions by table, the rest by a polynomial (P. T. P. Tang, Table-driven
    // implementation of the exponential function, 1989); the remainder is below 2^-7.5, so five terms leave 2^-54.
    __device__ __forceinline__ unsigned long long weight(float x) const
    {
        if (x == top) return 1ull << P.bits;
        const double z = ((double)x - (double)top) * factor;
        if (!(z > -64.0 * 48)) return 0;
        const double shifted = z + 6755399441055744.0;  // 1.5 2^52: rounds to whole numbers
        const int n = __double2loint(shifted);
        const double f = (z - (shifted - 6755399441055744.0)) * (0.69314718055994530942 / 64);
        double p = fma(f, 1.0 / 120, 1.0 / 24);
        p = fma(f, p, 1.0 / 6);
        p = fma(f, p, 0.5);
        p = fma(f, p, 1.0);
        p = fma(f, p, 1.0);
        const double t = S.power[n & 63];
        const double scale = __hiloint2double(__double2hiint(t) + (((n >> 6) + P.bits) << 20), __double2loint(t));
        return (unsigned long long)__double_as_longlong(fma(scale, p, 4503599627370496.0)) & 0xfffffffffffffull;  // + 2^52: rounds
    }
    __device__ __forceinline__ bool keeps(float x, int index) const { return x > cut_x || (x == cut_x && index <= cut_i); }
    __device__ __forceinline__ void barrier() const
    {
        __syncwarp();
        if (P.cluster > 1) cluster_barrier();
        else __syncthreads();
    }

    // The first token, by index, at which the cluster's values sum to more than what `target` makes of their total; value(x, index)
    // gives a token's.  Every block gets the total and the number of tokens with a value; `found` runs in one thread of the cluster.
    template <typename F, typename G, typename H>
    __device__ __forceinline__ void locate(F value, G target, H found)
    {
        const int warps = SAMPLE_THREADS / 32, step = 32 * V;
        const int per = (padded + warps * step - 1) / (warps * step) * step;  // tokens of a warp: a run of its own
        const int w0 = min(warp * per, padded), w1 = min(w0 + per, padded);
        unsigned long long sum = 0;
        uint32_t n = 0;
        for (int i = w0 + lane * V; i < w1; i += step) {
            float x[V];
            get(i, x);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const unsigned long long v = value(x[j], begin + i + j, n);
                sum += v;
            }
        }
        sum = warp_sum(sum);
        n = (uint32_t)warp_sum((long long)n);
        if (lane == 0) S.warp_mass[warp] = sum, S.warp_count[warp] = n;
        __syncthreads();
        if (warp == 0) {
            unsigned long long m = lane < warps ? S.warp_mass[lane] : 0;
            long long c = lane < warps ? S.warp_count[lane] : 0;
            m = warp_sum(m), c = warp_sum(c);
            if (lane == 0) S.block_mass = m, S.block_count = (uint32_t)c;
        }
        barrier();
        if (warp != 0) return;
        unsigned long long before = 0, total = 0;
        uint32_t count = 0;
        {
            const unsigned long long m = lane < P.cluster ? far_u64(&S.block_mass, lane) : 0;
            const uint32_t c = lane < P.cluster ? far_u32(&S.block_count, lane) : 0;
            total = warp_sum(m);
            count = (uint32_t)warp_sum((long long)c);
            before = warp_sum(lane < (int)rank ? m : 0ull);
        }
        const unsigned long long goal = target(total), own = S.block_mass;
        if (!(before <= goal && goal < before + own)) return;
        // this block has it: the warp's run, then the step of the run, then the lane, then the token
        unsigned long long m = lane < warps ? S.warp_mass[lane] : 0;
        unsigned long long run = before + warp_scan(m, lane);
        const int w = __ffs(__ballot_sync(FULL, goal < run)) - 1;
        run = __shfl_sync(FULL, run - m, w);
        const int r0 = min(w * per, padded), r1 = min(r0 + per, padded);
        for (int base = r0; base < r1; base += step) {
            const int i = base + lane * V;
            unsigned long long v[V], s = 0;
            uint32_t none = 0;
            if (i < r1) {
                float x[V];
                get(i, x);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = value(x[j], begin + i + j, none), s += v[j];
            }
            const unsigned long long upto = run + warp_scan(s, lane);
            const unsigned who = __ballot_sync(FULL, goal < upto);
            if (who) {
                if (lane == __ffs(who) - 1) {
                    unsigned long long at = upto - s;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        at += v[j];
                        if (goal < at) {
                            found(begin + i + j, total, count);
                            break;
                        }
                    }
                }
                return;
            }
            run = __shfl_sync(FULL, upto, 31);
        }
    }

    // Histogram of the tokens that `in` accepts over bucket(x) (descending x: bucket 0 holds the largest), summed over the cluster; then
    // the first bucket at which the counts (or the weights) from the largest on reach goal(total).  False: they never do.
    template <bool MASS, typename F, typename G, typename H>
    __device__ __forceinline__ bool search(F in, G bucket, H goal_of, unsigned long long &goal)
    {
        for (int i = tid; i < SAMPLE_BUCKETS; i += SAMPLE_THREADS) {
            S.count[i] = 0;
            if (MASS) S.mass[i] = 0;
        }
        __syncthreads();
        for (int i = tid * V; i < padded; i += SAMPLE_THREADS * V) {
            float x[V];
            get(i, x);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (in(x[j])) {
                    if (MASS) {
                        const unsigned long long w = weight(x[j]);
                        if (w == 0) continue;  // never at the border
                        atomicAdd(&S.mass[bucket(x[j])], w);
                    }
                    atomicAdd(&S.count[bucket(x[j])], 1u);
                }
        }
        barrier();
        const int share = SAMPLE_BUCKETS / P.cluster;
        for (int i = tid; i < share; i += SAMPLE_THREADS) {
            uint32_t c = 0;
            unsigned long long m = 0;
            for (int r = 0; r < P.cluster; ++r) {
                c += far_u32(&S.count[rank * share + i], r);
                if (MASS) m += far_u64(&S.mass[rank * share + i], r);
            }
            S.slice_count[i] = c;
            S.slice_mass[i] = MASS ? m : c;
        }
        __syncthreads();
        if (warp == 0) {
            unsigned long long m = 0;
            for (int i = lane; i < share; i += 32) m += S.slice_mass[i];
            m = warp_sum(m);
            if (lane == 0) S.slice_total_mass = m;
        }
        barrier();
        if (warp == 0) {
            const unsigned long long t = lane < P.cluster ? far_u64(&S.slice_total_mass, lane) : 0;
            const unsigned long long upto = warp_scan(t, lane), total = __shfl_sync(FULL, upto, 31);
            const unsigned long long g = goal_of(total);
            const unsigned who = __ballot_sync(FULL, upto >= g);
            if (g > total || who == 0) {
                if (lane == 0) S.members = 0;
            } else {
                const int q = __ffs(who) - 1, each = share / 32;
                unsigned long long above = __shfl_sync(FULL, upto - t, q), s = 0;
                for (int i = 0; i < each; ++i) s += far_u64(&S.slice_mass[lane * each + i], q);
                const unsigned long long run = above + warp_scan(s, lane);
                const int owner = __ffs(__ballot_sync(FULL, run >= g)) - 1;
                if (lane == owner) {
                    unsigned long long at = run - s;
                    for (int i = 0; i < each; ++i) {
                        const unsigned long long v = far_u64(&S.slice_mass[lane * each + i], q);
                        if (at + v >= g) {
                            S.bucket = q * share + lane * each + i;
                            S.members = far_u32(&S.slice_count[lane * each + i], q);
                            S.above = at;
                            break;
                        }
                        at += v;
                    }
                }
            }
            if (lane == 0) S.block_mass = g;  // for this block's threads
        }
        __syncthreads();
        goal = S.block_mass;
        return S.members != 0;
    }

    // (cut_x, cut_i) <- the token of the rank at which the counts (or weights) of the kept reach goal(total)
    template <bool MASS, typename H>
    __device__ __forceinline__ void descend(float scale, H goal_of)
    {
        const float low = cut_x;
        const auto linear = [&](float x) { return min(SAMPLE_BUCKETS - 1, (int)((top - x) * scale)); };  // falls as x rises
        unsigned long long goal, above = 0;
        if (!search<MASS>([&](float x) { return x >= low; }, linear, goal_of, goal)) return;
        uint32_t b = S.bucket, members = S.members;
        above = S.above;
        uint32_t k0 = 0, k1 = 0;
        int shift = -1;  // the level above cut by distance, not yet by keys
        for (;;) {
            const auto member = [&](float x) {
                if (!(x >= low)) return false;
                if (shift < 0) return (uint32_t)linear(x) == b;
                const uint32_t k = float_to_key(x);
                return k >= k0 && k <= k1;
            };
            if (members <= SAMPLE_LIST) {
                finish_list<MASS>(member, goal, above);
                return;
            }
            if (shift < 0) {  // the keys that the bucket holds
                if (tid == 0) S.key_min = 0xffffffffu, S.key_max = 0;
                __syncthreads();
                uint32_t lo = 0xffffffffu, hi = 0;
                for (int i = tid * V; i < padded; i += SAMPLE_THREADS * V) {
                    float x[V];
                    get(i, x);
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (member(x[j]) && (!MASS || weight(x[j]) != 0)) {
                            const uint32_t k = float_to_key(x[j]);
                            lo = min(lo, k), hi = max(hi, k);
                        }
                }
                lo = __reduce_min_sync(FULL, lo), hi = __reduce_max_sync(FULL, hi);
                if (lane == 0) atomicMin(&S.key_min, lo), atomicMax(&S.key_max, hi);
                barrier();
                k0 = 0xffffffffu, k1 = 0;
                for (int r = 0; r < P.cluster; ++r) k0 = min(k0, far_u32(&S.key_min, r)), k1 = max(k1, far_u32(&S.key_max, r));
            }
            if (k0 == k1) {  // one value: its first tokens by index, as many as are still missing
                const float x0 = key_to_float(k0);
                const unsigned long long missing = goal - above, each = MASS ? weight(x0) : 1, n = (missing + each - 1) / each;
                barrier();  // key_min and key_max have been read
                cut_x = x0, cut_i = INT_MAX;
                if (tid == 0) S.index = -1;
                __syncthreads();
                locate([&](float x, int, uint32_t &) { return (unsigned long long)(x == x0); }, [&](unsigned long long) { return n - 1; },
                       [&](int index, unsigned long long, uint32_t) { S.index = index; });
                barrier();
                for (int r = 0; r < P.cluster; ++r) {
                    const int index = (int)far_u32(&S.index, r);
                    if (index >= 0) cut_i = index;
                }
                barrier();
                return;
            }
            shift = 0;
            while (((k1 - k0) >> shift) >= SAMPLE_BUCKETS) ++shift;
            const unsigned long long g = goal - above;
            unsigned long long unused;
            const uint32_t top_key = k1;
            search<MASS>([&](float x) { return member(x); }, [&](float x) { return (top_key - float_to_key(x)) >> shift; },
                         [&](unsigned long long) { return g; }, unused);
            b = S.bucket, members = S.members;
            above += S.above;
            k1 = top_key - (b << shift);
            const uint32_t span = (1u << shift) - 1;
            k0 = k1 - k0 < span ? k0 : k1 - span;
        }
    }

    // The bucket's tokens, from all blocks, in a list of the first block's; every block sorts a copy and walks it.
    template <bool MASS, typename F>
    __device__ __forceinline__ void finish_list(F member, unsigned long long goal, unsigned long long above)
    {
        const uint32_t counter = in_block(smem_u32(&S.list_count), 0), list = in_block(smem_u32(&S.list[0]), 0);
        for (int i = tid * V; i < padded; i += SAMPLE_THREADS * V) {
            float x[V];
            get(i, x);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (member(x[j]) && (!MASS || weight(x[j]) != 0)) {
                    uint32_t at;
                    asm volatile("atom.shared::cluster.add.u32 %0, [%1], 1;" : "=r"(at) : "r"(counter) : "memory");
                    const unsigned long long item = ((unsigned long long)float_to_key(x[j]) << 32) | (0xffffffffu - (uint32_t)(begin + i + j));
                    if (at < SAMPLE_LIST) asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(list + 8 * at), "l"(item) : "memory");
                }
        }
        barrier();
        const int n = min((int)far_u32(&S.list_count, 0), SAMPLE_LIST);
        unsigned long long item = 0;
        if (tid < n) {
            item = far_u64(&S.list[tid], 0);
            S.mass[tid] = item;  // a copy: the histogram is done with
        }
        __syncthreads();
        if (tid < n) {
            int at = 0;
            for (int j = 0; j < n; ++j) at += S.mass[j] > item;
            S.sorted[at] = item;
        }
        __syncthreads();
        if (warp == 0) {
            constexpr int EACH = SAMPLE_LIST / 32;
            unsigned long long w[EACH], s = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int at = lane * EACH + i;
                w[i] = at >= n ? 0 : MASS ? weight(key_to_float((uint32_t)(S.sorted[at] >> 32))) : 1;
                s += w[i];
            }
            const unsigned long long run = above + warp_scan(s, lane);
            const unsigned who = __ballot_sync(FULL, run >= goal);
            if (who && lane == __ffs(who) - 1) {
                unsigned long long at = run - s;
                for (int i = 0; i < EACH; ++i) {
                    at += w[i];
                    if (at >= goal) {
                        S.cut = S.sorted[lane * EACH + i];
                        break;
                    }
                }
            }
        }
        barrier();  // the list has been read
        if (tid == 0) S.list_count = 0;
        cut_x = key_to_float((uint32_t)(S.cut >> 32)), cut_i = (int)(0xffffffffu - (uint32_t)S.cut);
    }

    __device__ __forceinline__ void give(int64_t r, int token, float logprob, int kept) const
    {
        P.token[r] = token;
        if (P.logprob) P.logprob[r] = logprob;
        if (P.kept) P.kept[r] = kept;
    }

    __device__ __forceinline__ void run(int64_t r)
    {
        // the run, its largest and its smallest usable logit
        float hi = -CUDART_INF_F, lo = CUDART_INF_F;
        const auto see = [&](float x) {
            x = usable(x);
            hi = fmaxf(hi, x);
            if (x > -CUDART_INF_F) lo = fminf(lo, x);
        };
        if (P.resident) {
            T *const to = const_cast<T *>(mine);
            const T *const from = row + begin;
            int done = 0;
            if ((reinterpret_cast<uintptr_t>(from) & 15) == 0) {
                done = len / V * V;
                const int each = SAMPLE_THREADS * V;
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
                            for (int v = 0; v < V; ++v) see(x[v]);
                        }
                }
            }
            for (int i = done + tid; i < padded; i += SAMPLE_THREADS) {
                const float x = i < len ? Io<T>::from_storage(ld(from + i)) : -CUDART_INF_F;
                Io<T>::store1(to + i, x);
                see(x);
            }
        } else {
            for (int i = tid * V; i < padded; i += SAMPLE_THREADS * V) {
                float x[V];
                get(i, x);
#pragma unroll
                for (int j = 0; j < V; ++j) see(x[j]);
            }
        }
        uint32_t kh = __reduce_max_sync(FULL, float_to_key(hi)), kl = __reduce_min_sync(FULL, float_to_key(lo));
        if (lane == 0) atomicMax(&S.key_max, kh), atomicMin(&S.key_min, kl);
        barrier();
        for (int q = 0; q < P.cluster; ++q) kh = max(kh, far_u32(&S.key_max, q)), kl = min(kl, far_u32(&S.key_min, q));
        top = key_to_float(kh);
        const float least = key_to_float(kl);

        const double T_ = P.temperature_row ? (double)ld(P.temperature_row + r) : P.temperature;
        const double p = P.top_p_row ? (double)ld(P.top_p_row + r) : P.top_p, m = P.min_p_row ? (double)ld(P.min_p_row + r) : P.min_p;
        const int64_t k = P.top_k_row ? (int64_t)ld(P.top_k_row + r) : P.top_k;
        const float u = ld(P.u + r);
        const bool valid = T_ >= 0 && T_ < CUDART_INF && p > 0 && m >= 0 && m <= 1 && u >= 0.f && u < 1.f;  // false for NaN
        if (!valid || top == -CUDART_INF_F) {
            if (rank == 0 && tid == 0) give(r, -1, valid ? -CUDART_INF_F : CUDART_NAN_F, 0);
            barrier();
            return;
        }
        factor = T_ > 0 ? 64 * 1.4426950408889634074 / T_ : 0;
        cut_x = least, cut_i = INT_MAX;
        if (top == CUDART_INF_F) cut_x = top;  // beside an infinity nothing else has a weight
        if (T_ == 0 || k == 1) {               // the first of the largest
            cut_x = top;
            locate([&](float x, int, uint32_t &) { return (unsigned long long)(x == top); }, [](unsigned long long) { return 0ull; },
                   [&](int index, unsigned long long, uint32_t) { give(r, index, 0.f, 1); });
            barrier();
            return;
        }
        if (m > 0) {  // the least x with (top - x) / T <= -log(min_p)
            const double reach = -log(m), inv = 1.0 / T_;
            float x = (float)((double)top - reach * T_);
            x = fminf(fmaxf(x, -3.402823466e38f), top);
            const auto inside = [&](float v) { return ((double)top - (double)v) * inv <= reach; };
            for (int i = 0; i < 4 && !inside(x); ++i) x = nextafterf(x, CUDART_INF_F);
            for (int i = 0; i < 4 && inside(nextafterf(x, -CUDART_INF_F)); ++i) x = nextafterf(x, -CUDART_INF_F);
            cut_x = fmaxf(cut_x, usable(x));
        }
        if (k > 0 && k < P.vocab) {
            const float range = fminf(top - cut_x, 32.f);
            descend<false>(range > 0.f ? SAMPLE_BUCKETS / range : 0.f, [&](unsigned long long) { return (unsigned long long)k; });
        }
        if (p < 1) {
            // ties beyond cut_i change no sum of larger logits, but they must not count for the total
            const float range = fminf(top - cut_x, (float)(34 * T_));
            const bool limited = cut_i != INT_MAX;
            unsigned long long total = 0;
            if (limited) total = kept_total();
            descend<true>(range > 0.f ? SAMPLE_BUCKETS / range : 0.f, [&](unsigned long long all) {
                const unsigned long long t = limited ? total : all;
                const unsigned long long g = (unsigned long long)ceil(p * (double)t);
                return g < 1 ? 1ull : g > t ? t : g;
            });
        }
        locate(
            [&](float x, int index, uint32_t &n) {
                if (!keeps(x, index)) return 0ull;
                ++n;
                return weight(x);
            },
            [&](unsigned long long total) {
                const unsigned long long g = (unsigned long long)((double)u * (double)total);
                return g < total ? g : total - 1;
            },
            [&](int index, unsigned long long total, uint32_t count) {
                const float x = usable(Io<T>::from_storage(ld(row + index)));  // the weight itself has lost digits where it is small
                const double z = x == top ? 0.0 : ((double)x - (double)top) / T_;
                give(r, index, (float)(z - log((double)total / (double)(1ull << P.bits))), (int)count);
            });
        barrier();  // nobody leaves while others read
    }

    // the kept tokens' weights, over the cluster
    __device__ __forceinline__ unsigned long long kept_total()
    {
        unsigned long long sum = 0;
        for (int i = tid * V; i < padded; i += SAMPLE_THREADS * V) {
            float x[V];
            get(i, x);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (keeps(x[j], begin + i + j)) sum += weight(x[j]);
        }
        sum = warp_sum(sum);
        if (lane == 0) S.warp_mass[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            unsigned long long m = lane < SAMPLE_THREADS / 32 ? S.warp_mass[lane] : 0;
            m = warp_sum(m);
            if (lane == 0) S.block_mass = m;
        }
        barrier();
        unsigned long long total = 0;
        for (int q = 0; q < P.cluster; ++q) total += far_u64(&S.block_mass, q);
        barrier();
        return total;
    }
};

template <typename T>
__global__ void __launch_bounds__(SAMPLE_THREADS) sample_kernel(const SampleArgs P)
{
    extern __shared__ __align__(16) uint8_t raw[];
    SampleShared &S = *reinterpret_cast<SampleShared *>(raw);
    if (threadIdx.x < 64) S.power[threadIdx.x] = exp2((double)threadIdx.x / 64);
    if (threadIdx.x == 64) S.list_count = 0, S.key_max = 0, S.key_min = 0xffffffffu;
    pdl_wait();
    __syncthreads();
    const int64_t r = blockIdx.x / P.cluster;
    const uint32_t rank = P.cluster > 1 ? cluster_rank() : 0;
    const int begin = min((int)rank * P.chunk, P.vocab), len = min(P.chunk, P.vocab - begin);
    Sampler<T> s{P, S, static_cast<const T *>(P.logits) + r * P.stride, reinterpret_cast<const T *>(raw + sizeof(SampleShared)), begin, len,
                 (len + Io<T>::V - 1) / Io<T>::V * Io<T>::V, rank, (int)threadIdx.x, (int)threadIdx.x & 31, (int)threadIdx.x >> 5};
    s.run(r);
}

}  // namespace lapsum
