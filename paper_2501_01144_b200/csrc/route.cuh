// Routing to experts: scores, selection, weights, and where each assignment's row lies among the experts' rows.
//
// Per token, over E experts:  score s = softmax(x) or 1 / (1 + exp(-x));  key = s + bias (without a bias the order of the
// logits);  with groups only the experts of the groups with the largest sums of their one or two largest keys stay;  the
// top_k largest keys, equal ones by number;  weights s (or s / sum of the chosen s) times a factor.
// A choice hangs on the last bits of keys that lie close together, so keys that are computed (a bias, or groups) decide in 64 bits
// where they are close.  One warp per token, expert 32 i + lane in the lane's i-th register, each key as an integer of the same order:
// the largest is found by a warp-wide integer maximum, and only the winner's lane looks for its next best again.
//
// The plan is a counting sort that is stable and has no order of atomics in its result: 64 tokens make a block, each expert
// has a 64-bit mask of the block's tokens that chose it, a row's rank inside the block is the number of set bits below its
// token's, and the ranks of earlier blocks come from a table of counts.  A token that names an expert twice has one row.
// At most 64 tokens: all in one launch; else two launches behind the routing, counts and places.
//
// Bound: T E logits read and 12 T k bytes written, 9 MB for 8192 x 256 x 8, are a microsecond or two: what counts is the latency of a
// token's chain of steps, and for many tokens the instructions it takes.  Measured (B200, from a graph, plan and all): 64 of 128 experts 5.5 us
// (one launch), 64 of 256 with a bias and groups 9.5; 8192 of 256 with a bias and groups 30.5 us, of 512 49; 8192 of 256 by softmax alone 20.3 us,
// not renormalised 23.1 (its sum in 64 bits); 1001 of 8 7.0 us (three launches).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "bd_common.cuh"
#include "quantize.cuh"

namespace bd {
namespace rt {

constexpr int kBlockTokens = 64;             // tokens of a block: the bits of an expert's mask
constexpr int kPlanThreads = 512;            // of the kernels that only plan
constexpr int kWarps = 8, kRouteThreads = 32 * kWarps;   // of a routing CTA: a warp per token
constexpr int kMaxCluster = kBlockTokens / kWarps;       // routing CTAs that share a block
constexpr int kMaxExperts = 512, kMaxTopK = 32, kMaxGroups = 32;
constexpr int kRowAlign = 128;               // an expert's rows start at multiples of a scale atom's rows

// bytes of one block's counts (a byte per expert: at most 64)
__host__ __device__ inline int64_t count_pitch(int64_t experts) { return (experts + 15) / 16 * 16; }
inline int64_t blocks_of(int64_t tokens) { return (tokens + kBlockTokens - 1) / kBlockTokens; }

struct Plan {
    int32_t *count, *start, *place;          // [E], [E + 1], [T][k]
    uint8_t *counts;                         // [blocks][count_pitch]
};
struct Rule {
    const void *logits;
    int64_t ld;
    const float *bias;
    const int32_t *valid;                    // rows that count, on the device; NULL: all
    int32_t *ids;                            // [T][k]
    float *weights;                          // [T][k]; NULL in the kernel that takes given ids
    int dt, tokens, experts, top_k, groups, top_groups, group_top;
    float scale;
    int renormalise;
    FastDiv group_of;                        // expert -> group, and the lanes that a group has in `kept_groups`, as a power of two
    int group_size, lane_shift;
};

// Order-preserving integers of floating-point numbers; 0 is below every number's.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t ordered(double x) {
    const uint64_t b = (uint64_t)__double_as_longlong(x);
    return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double number(uint64_t k) { return __longlong_as_double((long long)(k >> 63 ? k & ~(1ull << 63) : ~k)); }

__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ uint64_t warp_max(uint64_t v) {
    const uint32_t hi = warp_max((uint32_t)(v >> 32));
    const uint32_t lo = warp_max((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

__device__ __forceinline__ float logit(const char *p, int e, int dt) {
    return __uint_as_float(dt == BD_F32 ? Loader<BD_F32>::one(p + 4 * e) : dt == BD_BF16 ? Loader<BD_BF16>::one(p + 2 * e) : Loader<BD_F16>::one(p + 2 * e));
}

// Places of `tokens` tokens from t0 on, from the masks of their block (shared), the experts' first free rows in it (shared) and the number of
// the first of them in the block.
__device__ __forceinline__ void write_places(const Rule &r, const Plan &p, const unsigned long long *mask, const int32_t *first, int t0, int in_block, int tokens) {
    for (int i = threadIdx.x; i < tokens * r.top_k; i += blockDim.x) {
        const int e = r.ids[(int64_t)t0 * r.top_k + i];           // (written by this CTA before a barrier, or given)
        const bool ok = e >= 0 && e < r.experts;
        p.place[(int64_t)t0 * r.top_k + i] = ok ? first[e] + __popcll(mask[e] & ((1ull << (in_block + i / r.top_k)) - 1ull)) : -1;
    }
}
// Starts of all experts from their numbers of rows: thread t has experts PER * t, ...; writes them (and the counts) where asked to.
template <int THREADS>
struct Starts {
    static constexpr int kPer = kMaxExperts / THREADS;
    int rows[kPer], start[kPer];
    __device__ __forceinline__ int expert(int q) const { return (int)threadIdx.x * kPer + q; }
    __device__ __forceinline__ void scan(const Rule &r, const Plan &p, bool writes, int32_t *warp_sums) {
        const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
        int mine = 0;
#pragma unroll
        for (int q = 0; q < kPer; q++) {
            start[q] = mine;
            mine += (rows[q] + kRowAlign - 1) / kRowAlign * kRowAlign;
        }
        int incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
        if (lane == 31) warp_sums[warp] = incl;
        __syncthreads();
        int before = incl - mine;
#pragma unroll
        for (int w = 0; w < THREADS / 32; w++) before += w < warp ? warp_sums[w] : 0;
#pragma unroll
        for (int q = 0; q < kPer; q++) {
            start[q] += before;
            const int e = expert(q);
            if (writes && e < r.experts) {
                p.count[e] = rows[q];
                p.start[e] = start[q];
                if (e == r.experts - 1) p.start[r.experts] = start[q] + (rows[q] + kRowAlign - 1) / kRowAlign * kRowAlign;
            }
        }
    }
};

__device__ __forceinline__ float number(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ float largest(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double largest(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ float smallest(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ double smallest(double a, double b) { return fmin(a, b); }

// The groups that stay, as a bit mask, from the keys in `scratch` (-Inf: not there).  A group has the lanes that 32 / groups allows (a power of
// two).  `gap`: how far the last group that stays lies above the best that does not.
template <typename F>
__device__ __forceinline__ uint32_t kept_groups(const Rule &r, const F *scratch, F &gap) {
    using Key = typename std::conditional<sizeof(F) == 8, uint64_t, uint32_t>::type;
    const int lane = threadIdx.x % 32, size = r.group_size, lanes = 1 << r.lane_shift;
    const int g = lane >> r.lane_shift, sub = lane & (lanes - 1);
    const int turn = g * lanes - size * (int)fast_div((uint32_t)(g * lanes), r.group_of);   // (each group begins elsewhere: other banks)
    F a = -INFINITY, b = -INFINITY;                               // its two largest keys
    if (g < r.groups)
#pragma unroll 4
        for (int j = sub; j < size; j += lanes) {
            const int k = j + turn < size ? j + turn : j + turn - size;
            const F v = scratch[g * size + k];
            b = largest(b, smallest(a, v));
            a = largest(a, v);
        }
    for (int d = 1; d < lanes; d <<= 1) {
        const F a2 = __shfl_xor_sync(0xffffffffu, a, d), b2 = __shfl_xor_sync(0xffffffffu, b, d);
        b = largest(smallest(a, a2), largest(b, b2));
        a = largest(a, a2);
    }
    if (r.group_top == 2 && b != -INFINITY) a += b;
    Key mine = g < r.groups && sub == 0 && a != -INFINITY ? ordered(a) : 0;   // the group's first lane: its value
    uint32_t kept = 0;
    Key last = 0;
    for (int n = 0; n < r.top_groups; n++) {
        const Key best = warp_max(mine);
        if (best == 0) break;
        const int owner = __ffs(__ballot_sync(0xffffffffu, mine == best)) - 1;   // equal values: the lower group
        kept |= 1u << (owner >> r.lane_shift);
        last = best;
        if (lane == owner) mine = 0;
    }
    const Key rest = warp_max(mine);
    gap = rest == 0 ? (F)INFINITY : number(last) - number(rest);
    return kept;
}

// The `count` largest keys in descending order, equal ones by number: lane j keeps the j-th (id -1: none left).
template <int NV, typename Key>
__device__ __forceinline__ void select_largest(Key (&key)[NV], int count, int &my_id, Key &my_key) {
    const int lane = threadIdx.x % 32;
    my_id = -1;
    my_key = 0;
    Key best;
    int at;
    auto look = [&]() {                                           // the lane's best: the first of equal ones has the lowest number
        best = key[0];
        at = 0;
#pragma unroll
        for (int i = 1; i < NV; i++)
            if (key[i] > best) { best = key[i]; at = i; }
    };
    look();
    for (int j = 0; j < count; j++) {
        const Key m = warp_max(best);
        if (m == 0) break;
        const uint32_t e = ~warp_max(best == m ? ~(uint32_t)(32 * at + lane) : 0u);
        if (lane == (int)(e % 32u)) {
#pragma unroll
            for (int i = 0; i < NV; i++)
                if (i == at) key[i] = 0;
            look();
        }
        if (lane == j) { my_id = (int)e; my_key = m; }
    }
}

// One token by one warp.  NV: experts per lane.  WIDE: keys that are computed (a bias or groups).  Those are compared in 64 bits, but a
// 64-bit exponential per expert, 64-bit comparisons and maxima are ten times the work: keys in 32 bits come first, and only where
// two that decide lie closer together than 32 bits can be off does the token go through 64 bits (some in a thousand of random
// ones).  How far a 32-bit key can be off.  Softmax: an exponential by 2^-22 of itself and by its argument's rounding, a sum of up to
// 16 + 5 additions by 2^-19, the rest by 2^-23: together below 2^-19 of the largest score.  Sigmoid: the exponential's 2^-22 counts with
// s (1 - s) <= 1/4, the sum and the quotient are rounded by 2^-24 each: together below 2^-22.  2^-24 of the key by the bias' addition.
template <int NV, bool SIGMOID, bool WIDE>
__device__ __forceinline__ void route_token(const Rule &r, int t, double *scratch, uint32_t *mask) {
    const int lane = threadIdx.x % 32;
    const char *row = (const char *)r.logits + (int64_t)t * r.ld * (r.dt == BD_F32 ? 4 : 2);
    float x[NV], b[WIDE ? NV : 1];
    bool odd = false;
    if (WIDE) {                                                   // (on their way together with the logits)
#pragma unroll
        for (int i = 0; i < NV; i++) b[i] = r.bias && 32 * i + lane < r.experts ? r.bias[32 * i + lane] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int e = 32 * i + lane;
        x[i] = e < r.experts ? logit(row, e, r.dt) + 0.0f : -INFINITY;   // (-0 and 0 are one number)
        // NaN counts as an expert that is not there, +Inf as the largest number; both are told
        if (x[i] != x[i] || x[i] == INFINITY) {
            odd = true;
            x[i] = x[i] != x[i] ? -INFINITY : 3.402823466e38f;
        }
    }
    float top = -INFINITY;
    if (!SIGMOID) {
#pragma unroll
        for (int i = 0; i < NV; i++) top = fmaxf(top, x[i]);
        top = number(warp_max(ordered(top)));
    }
    auto value_of = [&](int id) {                                 // the logit of the lane's expert (-1: -Inf), from the lane that holds it
        float v = -INFINITY;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const float u = __shfl_sync(0xffffffffu, x[i], id & 31);
            if (id >> 5 == i) v = u;
        }
        return v;
    };
    int my_id = -1;                                               // lane j: the j-th expert
    if (!WIDE) {
        uint32_t key[NV], unused;                                 // 0 = not there, or taken
#pragma unroll
        for (int i = 0; i < NV; i++) key[i] = x[i] != -INFINITY ? ordered(x[i]) : 0;
        select_largest<NV>(key, r.top_k, my_id, unused);
    } else {
        float s[NV], inv = 1.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) s[i] = SIGMOID ? 1.0f / (1.0f + expf(-x[i])) : (x[i] == -INFINITY ? 0.0f : expf(x[i] - top));
        if (!SIGMOID) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; i++) sum += s[i];
            sum = warp_sum(sum);
            inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        }
        uint32_t key[NV];
        float *const mine = (float *)scratch;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int e = 32 * i + lane;
            float k = s[i] * inv;
            if (r.bias && e < r.experts) {
                k += b[i];
                odd = odd || k != k;
            }
            const bool there = x[i] != -INFINITY && k == k && k != -INFINITY;
            key[i] = there ? ordered(r.bias ? k + 0.0f : x[i]) : 0;   // (without a bias experts compare by the logits, groups by the scores)
            if (r.groups > 1 && e < r.experts) mine[e] = there ? k : -INFINITY;
        }
        const float off = SIGMOID ? 4.7684e-7f : 3.8147e-6f * inv;   // 2^-21, 2^-18: of two keys, without the bias' part
        bool close = false;
        if (r.groups > 1) {
            __syncwarp();
            float gap;
            const uint32_t kept = kept_groups(r, mine, gap);
            float biggest = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                const int e = 32 * i + lane;
                if (e < r.experts && mine[e] != -INFINITY) biggest = fmaxf(biggest, fabsf(mine[e]));
                if (e < r.experts && !(kept >> fast_div(e, r.group_of) & 1u)) key[i] = 0;
            }
            biggest = number(warp_max(ordered(biggest)));
            close = !(gap > 2.0f * off + 4.7684e-7f * biggest);   // (sums of two keys and their own rounding: 2^-21)
        }
        uint32_t my_key;
        select_largest<NV>(key, min(r.bias ? r.top_k + 1 : r.top_k, 32), my_id, my_key);
        if (r.bias) {
            // each key against the next one, the first that is not chosen among them; equal logits with equal biases are equal
            const float mx = value_of(my_id), mb = my_id >= 0 ? r.bias[my_id] : 0.0f;
            const float k = my_key ? number(my_key) : 0.0f, nk = __shfl_down_sync(0xffffffffu, k, 1), nx = __shfl_down_sync(0xffffffffu, mx, 1), nb = __shfl_down_sync(0xffffffffu, mb, 1);
            const bool next = __shfl_down_sync(0xffffffffu, my_id, 1) >= 0 && lane < 31;
            close = close || (my_id >= 0 && next && !(k - nk > off + 1.1921e-7f * (fabsf(k) + fabsf(nk))) && !(mx == nx && mb == nb));
            close = close || r.top_k == 32;                       // (no lane is left for the one behind them)
            if (lane >= r.top_k) my_id = -1;
        }
        if (__any_sync(0xffffffffu, close)) {
            __syncwarp();
            double wide[NV], sum = 0.0;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                wide[i] = SIGMOID ? 1.0 / (1.0 + exp(-(double)x[i])) : (x[i] == -INFINITY ? 0.0 : exp((double)x[i] - (double)top));
                sum += wide[i];
            }
            if (!SIGMOID) {
                sum = warp_sum(sum);
#pragma unroll
                for (int i = 0; i < NV; i++) wide[i] = sum > 0.0 ? wide[i] / sum : 0.0;
            }
            uint64_t exact[NV], unused;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                const int e = 32 * i + lane;
                double k = wide[i];
                if (r.bias && e < r.experts) k = k + (double)r.bias[e] + 0.0;
                const bool there = x[i] != -INFINITY && k == k && k != -INFINITY;
                exact[i] = there ? ordered(r.bias ? k : (double)x[i]) : 0;
                if (r.groups > 1 && e < r.experts) scratch[e] = there ? k : -INFINITY;
            }
            if (r.groups > 1) {
                __syncwarp();
                double gap;
                const uint32_t kept = kept_groups(r, scratch, gap);
#pragma unroll
                for (int i = 0; i < NV; i++)
                    if (32 * i + lane < r.experts && !(kept >> fast_div(32 * i + lane, r.group_of) & 1u)) exact[i] = 0;
            }
            select_largest<NV>(exact, r.top_k, my_id, unused);
        }
    }
    if (__any_sync(0xffffffffu, odd) && lane == 0) atomicOr(&g_status_word, kStatusNonfinite);
    // weights in 64 bits, rounded once
    const float my_x = value_of(my_id);
    double w = 0.0;
    if (SIGMOID) {
        w = my_id >= 0 ? 1.0 / (1.0 + exp(-(double)my_x)) : 0.0;
    } else if (r.renormalise) {
        const float ref = number(warp_max(my_id >= 0 ? ordered(my_x) : 0u));   // relative to the largest chosen one: no underflow of all
        w = my_id >= 0 ? exp((double)my_x - (double)ref) : 0.0;
    } else {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < NV; i++) sum += x[i] == -INFINITY ? 0.0 : exp((double)x[i] - (double)top);
        sum = warp_sum(sum);
        w = my_id >= 0 && sum > 0.0 ? exp((double)my_x - (double)top) / sum : 0.0;
    }
    if (r.renormalise) {
        const double sum = warp_sum(w);
        w = sum > 0.0 ? w / sum : 0.0;
    }
    if (lane < r.top_k) {
        r.ids[(int64_t)t * r.top_k + lane] = my_id;
        r.weights[(int64_t)t * r.top_k + lane] = (float)(w * (double)r.scale);
        if (mask && my_id >= 0) atomicOr(mask + my_id, 1u << (t % kWarps));
    }
}

__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t v;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(v));
    return v;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t v;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(v));
    return v;
}
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_word(const uint32_t *word, uint32_t rank) {
    uint32_t a, v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(word)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
// A CTA per eight tokens.  With a plan (at most 64 tokens, which are one block) the CTAs are one cluster: each puts the experts' masks together from
// the parts in the others' shared memory and places its own tokens' rows.  (One CTA for the 64 tokens, four a warp one after the
// other: 14 us instead of 5; clusters for the blocks of more tokens: 12 us more for 8192 than the two launches that plan by themselves.)
template <int NV, bool SIGMOID, bool WIDE>
__global__ void __launch_bounds__(kRouteThreads, NV == 16 ? 4 : 6) route_kernel(const Rule r, const Plan plan) {
    __shared__ uint32_t part[kMaxExperts];                        // bit i: this CTA's token i chose the expert
    __shared__ unsigned long long mask[kMaxExperts];
    __shared__ int32_t first[kMaxExperts];
    __shared__ int32_t warp_sums[kWarps];
    extern __shared__ double scratch[];                           // [warps][E + 1], where groups are asked for
    const int t0 = blockIdx.x * kWarps, tokens = min(kWarps, r.tokens - t0), warp = threadIdx.x / 32;
    const bool plans = plan.place != nullptr;
    if (plans) {
        for (int e = threadIdx.x; e < r.experts; e += kRouteThreads) part[e] = 0;
        __syncthreads();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int valid = r.valid ? *r.valid : r.tokens;
    if (warp < tokens) {
        const int t = t0 + warp;
        if (t < valid) {
            route_token<NV, SIGMOID, WIDE>(r, t, scratch + warp * (r.experts + 1), plans ? part : nullptr);
        } else if (threadIdx.x % 32 < r.top_k) {
            r.ids[(int64_t)t * r.top_k + threadIdx.x % 32] = -1;
            r.weights[(int64_t)t * r.top_k + threadIdx.x % 32] = 0.0f;
        }
    }
    if (!plans) return;
    const uint32_t parts = cluster_size();
    __syncwarp();
    cluster_sync();
    Starts<kRouteThreads> s;
#pragma unroll
    for (int q = 0; q < s.kPer; q++) {
        const int e = s.expert(q);
        unsigned long long m = 0;
        if (e < r.experts) {
#pragma unroll
            for (uint32_t c = 0; c < (uint32_t)kMaxCluster; c++)
                if (c < parts) m |= (unsigned long long)peer_word(part + e, c) << (kWarps * c);
            mask[e] = m;
        }
        s.rows[q] = __popcll(m);
    }
    s.scan(r, plan, cluster_rank() == 0, warp_sums);
#pragma unroll
    for (int q = 0; q < s.kPer; q++)
        if (s.expert(q) < r.experts) first[s.expert(q)] = s.start[q];
    __syncthreads();
    if (tokens > 0) write_places(r, plan, mask, first, t0, t0, tokens);
    cluster_sync();                                               // the peers may still read this CTA's part
}

// The masks of one block from its ids.
__device__ __forceinline__ void masks_of(const Rule &r, unsigned long long *mask, int t0, int tokens, bool tells) {
    for (int e = threadIdx.x; e < r.experts; e += kPlanThreads) mask[e] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * r.top_k; i += kPlanThreads) {
        const int e = r.ids[(int64_t)t0 * r.top_k + i];
        const int tok = i / r.top_k;                              // (32-bit halves: 64-bit atomics on shared memory are loops)
        if (e >= 0 && e < r.experts) atomicOr((uint32_t *)(mask + e) + tok / 32, 1u << (tok % 32));
        else if (e >= r.experts && tells) atomicOr(&g_status_word, kStatusIndex);
    }
    __syncthreads();
}
// Given ids: the counts of each block (one block: the whole plan).
__global__ void __launch_bounds__(kPlanThreads) plan_count_kernel(const Rule r, const Plan plan) {
    __shared__ unsigned long long mask[kMaxExperts];
    __shared__ int32_t first[kMaxExperts];
    __shared__ int32_t warp_sums[kPlanThreads / 32];
    const int t0 = blockIdx.x * kBlockTokens, tokens = min(kBlockTokens, r.tokens - t0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    masks_of(r, mask, t0, tokens, true);
    if (gridDim.x == 1) {
        const int e = threadIdx.x;
        Starts<kPlanThreads> s;
        s.rows[0] = e < r.experts ? __popcll(mask[e]) : 0;
        s.scan(r, plan, true, warp_sums);
        if (e < r.experts) first[e] = s.start[0];
        __syncthreads();
        write_places(r, plan, mask, first, t0, 0, tokens);
    } else {
        for (int e = threadIdx.x; e < r.experts; e += kPlanThreads)
            plan.counts[(int64_t)blockIdx.x * count_pitch(r.experts) + e] = (uint8_t)__popcll(mask[e]);
    }
}
// The plan of several blocks: CTA c takes `per` consecutive blocks.  It adds up the counts of all blocks (an expert's total, for the
// starts) and of those before its own (the ranks its rows begin with): threads take four experts of a row of the table at a time.
__global__ void __launch_bounds__(kPlanThreads) plan_place_kernel(const Rule r, const Plan plan, int blocks, int per) {
    __shared__ unsigned long long mask[kMaxExperts];
    __shared__ int32_t first[kMaxExperts], total[kMaxExperts];
    __shared__ int32_t warp_sums[kPlanThreads / 32];
    const int begin = blockIdx.x * per, end = min(blocks, begin + per);
    for (int e = threadIdx.x; e < kMaxExperts; e += kPlanThreads) first[e] = total[e] = 0;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t pitch = count_pitch(r.experts);
    const int words = (r.experts + 3) / 4;
    const int rows = kPlanThreads / words, w = threadIdx.x % words;   // (words is at most 128)
    if (threadIdx.x / words < rows) {
        int before[4] = {0, 0, 0, 0}, all[4] = {0, 0, 0, 0};
#pragma unroll 8
        for (int b = threadIdx.x / words; b < blocks; b += rows) {
            const uint32_t v = *(const uint32_t *)(plan.counts + b * pitch + 4 * w);
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const int n = (int)(v >> (8 * q) & 255u);
                all[q] += n;
                before[q] += b < begin ? n : 0;
            }
        }
#pragma unroll
        for (int q = 0; q < 4; q++)
            if (4 * w + q < r.experts) {                          // (sums of integers: the order does not matter)
                atomicAdd(first + 4 * w + q, before[q]);
                atomicAdd(total + 4 * w + q, all[q]);
            }
    }
    __syncthreads();
    const int e = threadIdx.x;
    Starts<kPlanThreads> s;
    s.rows[0] = e < r.experts ? total[e] : 0;
    s.scan(r, plan, blockIdx.x == 0, warp_sums);
    if (e < r.experts) first[e] += s.start[0];
    for (int b = begin; b < end; b++) {
        const int t0 = b * kBlockTokens, tokens = min(kBlockTokens, r.tokens - t0);
        masks_of(r, mask, t0, tokens, false);                     // (begins and ends with barriers around the masks)
        write_places(r, plan, mask, first, t0, 0, tokens);
        __syncthreads();
        if (e < r.experts) first[e] += __popcll(mask[e]);
        __syncthreads();
    }
}

}  // namespace rt
}  // namespace bd
