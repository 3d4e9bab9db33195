// Routing to experts: scores, selection, weights, and where each assignment's row lies among the experts' rows.
//
// Per token, over E experts:  score s = softmax(x) or 1 / (1 + exp(-x));  key = s + bias (without a bias the order of the
// logits);  with groups only the experts of the groups with the largest sums of their one or two largest keys stay;  the
// top_k largest keys, equal ones by number;  weights s (or s / sum of the chosen s) times a factor.
// A choice hangs on the last bits of keys that lie close together, so keys that are computed (a bias, or groups) are held in
// 64 bits; one warp per token, expert 32 i + lane in the lane's i-th register, each key as an integer of the same order.
// The largest key is found by two (64-bit keys: up to three) warp-wide integer maxima and only the winner's lane looks for its next
// best again, so a choice costs a few dozen instructions whatever E is.
//
// The plan is a counting sort that is stable and has no order of atomics in its result: 64 tokens make a block, each expert
// has a 64-bit mask of the block's tokens that chose it, a row's rank inside the block is the number of set bits below its
// token's, and the ranks of earlier blocks come from a table of counts.  A token that names an expert twice has one row.
// At most 64 tokens: all in one launch; else the counts leave with the routing and a second launch adds them up.
//
// Bound: T E logits read and 12 T k bytes written, 9 MB for 8192 x 256 x 8, are a microsecond or two: what counts is the latency of a
// token's chain of steps and, with a bias, 64-bit exponentials.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "bd_common.cuh"
#include "quantize.cuh"

namespace bd {
namespace rt {

constexpr int kBlockTokens = 64;             // tokens of a block: the bits of an expert's mask
constexpr int kThreads = 512, kWarps = kThreads / 32;
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

// A block's part of the plan: from the masks (shared) and the experts' first free rows (shared) to the places of its assignments.
__device__ __forceinline__ void write_places(const Rule &r, const Plan &p, const unsigned long long *mask, const int32_t *first, int t0, int tokens) {
    for (int i = threadIdx.x; i < tokens * r.top_k; i += kThreads) {
        const int e = r.ids[(int64_t)t0 * r.top_k + i];           // (written by this CTA before a barrier, or given)
        const bool ok = e >= 0 && e < r.experts;
        p.place[(int64_t)t0 * r.top_k + i] = ok ? first[e] + __popcll(mask[e] & ((1ull << (i / r.top_k)) - 1ull)) : -1;
    }
}
// Exclusive scan over kThreads values (one per thread).
__device__ __forceinline__ int scan_exclusive(int v, int32_t *warp_sums, int &total) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int incl = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += up;
    }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; w++) {
        const int s = warp_sums[w];
        before += w < warp ? s : 0;
        total += s;
    }
    return before + incl - v;
}
// Counts and starts of all experts from their totals; thread e has expert e (kMaxExperts == kThreads).
__device__ __forceinline__ int write_starts(const Rule &r, const Plan &p, int total_rows, bool writes, int32_t *warp_sums) {
    static_assert(kMaxExperts <= kThreads, "a thread per expert");
    const int e = threadIdx.x;
    const int padded = (total_rows + kRowAlign - 1) / kRowAlign * kRowAlign;
    int all;
    const int start = scan_exclusive(padded, warp_sums, all);
    if (writes && e < r.experts) {
        p.count[e] = total_rows;
        p.start[e] = start;
        if (e == r.experts - 1) p.start[r.experts] = all;
    }
    return start;
}

// One token by one warp.  NV: experts per lane.  WIDE: keys in 64 bits (a bias or groups).
template <int NV, bool SIGMOID, bool WIDE>
__device__ __forceinline__ void route_token(const Rule &r, int t, double *scratch, unsigned long long *mask) {
    using Key = typename std::conditional<WIDE, uint64_t, uint32_t>::type;
    const int lane = threadIdx.x % 32;
    const char *row = (const char *)r.logits + (int64_t)t * r.ld * (r.dt == BD_F32 ? 4 : 2);
    float x[NV];
    bool odd = false;
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
        const uint32_t m = warp_max(ordered(top));
        top = __uint_as_float(m & 0x80000000u ? m & 0x7fffffffu : ~m);
    }
    // keys; 0 = not there, or taken
    Key key[NV];
    double sum_wide = 0.0;
    if (WIDE) {
        double s[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            s[i] = SIGMOID ? 1.0 / (1.0 + exp(-(double)x[i])) : (x[i] == -INFINITY ? 0.0 : exp((double)x[i] - (double)top));
            sum_wide += s[i];
        }
        if (!SIGMOID) {
            sum_wide = warp_sum(sum_wide);
#pragma unroll
            for (int i = 0; i < NV; i++) s[i] = sum_wide > 0.0 ? s[i] / sum_wide : 0.0;
        }
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int e = 32 * i + lane;
            double k = s[i];
            if (r.bias && e < r.experts) k = k + (double)r.bias[e] + 0.0;
            if (k != k) odd = true;
            const bool there = x[i] != -INFINITY && k == k && k != -INFINITY;
            key[i] = there ? (Key)ordered(k) : 0;
            if (!r.bias && r.groups > 1) {                        // groups compare scores, experts the logits
                if (e < r.experts) scratch[e] = there ? k : -INFINITY;
                key[i] = there ? (Key)ordered((double)x[i]) : 0;
            } else if (r.groups > 1 && e < r.experts) {
                scratch[e] = there ? k : -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; i++) key[i] = x[i] != -INFINITY ? (Key)ordered(x[i]) : 0;
    }
    if (__any_sync(0xffffffffu, odd) && lane == 0) atomicOr(&g_status_word, kStatusNonfinite);
    if (WIDE && r.groups > 1) {
        const int size = r.experts / r.groups;
        __syncwarp();
        uint64_t mine = 0;                                        // lane g: the group's value
        if (lane < r.groups) {
            double a = -INFINITY, b = -INFINITY;                  // its two largest keys
            for (int j = 0, k = lane % size; j < size; j++, k = k + 1 == size ? 0 : k + 1) {   // (each lane begins elsewhere: other banks)
                const double v = scratch[lane * size + k];
                b = fmax(b, fmin(a, v));
                a = fmax(a, v);
            }
            if (r.group_top == 2 && b != -INFINITY) a += b;
            mine = a != -INFINITY ? ordered(a) : 0;
        }
        uint32_t kept = 0;
        for (int n = 0; n < r.top_groups; n++) {
            const uint64_t best = warp_max(mine);
            if (best == 0) break;
            const int g = __ffs(__ballot_sync(0xffffffffu, mine == best)) - 1;
            kept |= 1u << g;
            if (lane == g) mine = 0;
        }
#pragma unroll
        for (int i = 0; i < NV; i++)
            if (32 * i + lane < r.experts && !(kept >> ((32 * i + lane) / size) & 1u)) key[i] = 0;
        __syncwarp();
    }
    // the top_k largest keys: lane j keeps the j-th expert and its logit
    int my_id = -1;
    float my_x = -INFINITY;
    Key best = 0;
    int at = 0;
    auto look = [&]() {                                           // the lane's best: the first of equal ones has the lowest number
        best = 0;
#pragma unroll
        for (int i = 0; i < NV; i++)
            if (key[i] > best) { best = key[i]; at = i; }
    };
    look();
    for (int j = 0; j < r.top_k; j++) {
        const Key m = warp_max(best);
        if (m == 0) break;
        // equal keys: the lowest number
        const uint32_t e = ~warp_max(best == m ? ~(uint32_t)(32 * at + lane) : 0u);
        const int owner = e % 32;
        float xe = 0.0f;
        if (lane == owner) {
#pragma unroll
            for (int i = 0; i < NV; i++)
                if (i == at) { xe = x[i]; key[i] = 0; }
            look();
        }
        xe = __shfl_sync(0xffffffffu, xe, owner);
        if (lane == j) { my_id = (int)e; my_x = xe; }
    }
    // weights in 64 bits, rounded once
    double w = 0.0;
    if (SIGMOID) {
        w = my_id >= 0 ? 1.0 / (1.0 + exp(-(double)my_x)) : 0.0;
    } else if (r.renormalise) {
        const uint32_t m = warp_max(my_id >= 0 ? ordered(my_x) : 0u);   // relative to the largest chosen one: no underflow of all
        const float ref = __uint_as_float(m & 0x80000000u ? m & 0x7fffffffu : ~m);
        w = my_id >= 0 ? exp((double)my_x - (double)ref) : 0.0;
    } else {
        double sum = sum_wide;
        if (!WIDE) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; i++) s += x[i] == -INFINITY ? 0.0f : expf(x[i] - top);
            sum = (double)warp_sum(s);
        }
        w = my_id >= 0 && sum > 0.0 ? exp((double)my_x - (double)top) / sum : 0.0;
    }
    if (r.renormalise) {
        const double sum = warp_sum(w);
        w = sum > 0.0 ? w / sum : 0.0;
    }
    if (lane < r.top_k) {
        r.ids[(int64_t)t * r.top_k + lane] = my_id;
        r.weights[(int64_t)t * r.top_k + lane] = (float)(w * (double)r.scale);
        if (mask && my_id >= 0) atomicOr(mask + my_id, 1ull << (t % kBlockTokens));
    }
}

// A CTA per block of 64 tokens.  plan.place NULL: no plan.  With one block the plan is finished here.
template <int NV, bool SIGMOID, bool WIDE>
__global__ void __launch_bounds__(kThreads) route_kernel(const Rule r, const Plan plan) {
    __shared__ unsigned long long mask[kMaxExperts];
    __shared__ int32_t first[kMaxExperts];
    __shared__ int32_t warp_sums[kWarps];
    extern __shared__ double scratch[];                           // [warps][E + 1], where groups are asked for
    const int t0 = blockIdx.x * kBlockTokens, tokens = min(kBlockTokens, r.tokens - t0);
    for (int e = threadIdx.x; e < r.experts; e += kThreads) mask[e] = 0;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int valid = r.valid ? *r.valid : r.tokens;
    for (int i = threadIdx.x / 32; i < tokens; i += kWarps) {
        const int t = t0 + i;
        if (t < valid) {
            route_token<NV, SIGMOID, WIDE>(r, t, scratch + (threadIdx.x / 32) * (r.experts + 1), mask);
        } else if (threadIdx.x % 32 < r.top_k) {
            r.ids[(int64_t)t * r.top_k + threadIdx.x % 32] = -1;
            r.weights[(int64_t)t * r.top_k + threadIdx.x % 32] = 0.0f;
        }
    }
    if (!plan.place) return;
    __syncthreads();
    if (gridDim.x == 1) {
        const int e = threadIdx.x;
        const int rows = e < r.experts ? __popcll(mask[e]) : 0;
        const int start = write_starts(r, plan, rows, true, warp_sums);
        if (e < r.experts) first[e] = start;
        __syncthreads();
        write_places(r, plan, mask, first, t0, tokens);
    } else {
        for (int e = threadIdx.x; e < r.experts; e += kThreads)
            plan.counts[(int64_t)blockIdx.x * count_pitch(r.experts) + e] = (uint8_t)__popcll(mask[e]);
    }
}

// The masks of one block from its ids.
__device__ __forceinline__ void masks_of(const Rule &r, unsigned long long *mask, int t0, int tokens, bool tells) {
    for (int e = threadIdx.x; e < r.experts; e += kThreads) mask[e] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * r.top_k; i += kThreads) {
        const int e = r.ids[(int64_t)t0 * r.top_k + i];
        if (e >= 0 && e < r.experts) atomicOr(mask + e, 1ull << (i / r.top_k));
        else if (e >= r.experts && tells) atomicOr(&g_status_word, kStatusIndex);
    }
    __syncthreads();
}
// Given ids: the counts of each block (one block: the whole plan).
__global__ void __launch_bounds__(kThreads) plan_count_kernel(const Rule r, const Plan plan) {
    __shared__ unsigned long long mask[kMaxExperts];
    __shared__ int32_t first[kMaxExperts];
    __shared__ int32_t warp_sums[kWarps];
    const int t0 = blockIdx.x * kBlockTokens, tokens = min(kBlockTokens, r.tokens - t0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    masks_of(r, mask, t0, tokens, true);
    if (gridDim.x == 1) {
        const int e = threadIdx.x;
        const int start = write_starts(r, plan, e < r.experts ? __popcll(mask[e]) : 0, true, warp_sums);
        if (e < r.experts) first[e] = start;
        __syncthreads();
        write_places(r, plan, mask, first, t0, tokens);
    } else {
        for (int e = threadIdx.x; e < r.experts; e += kThreads)
            plan.counts[(int64_t)blockIdx.x * count_pitch(r.experts) + e] = (uint8_t)__popcll(mask[e]);
    }
}
// The plan of several blocks: CTA c takes `per` consecutive blocks.  It adds up the counts of all blocks (an expert's total, for the
// starts) and of those before its own (the ranks its rows begin with): threads take four experts of a row of the table at a time.
__global__ void __launch_bounds__(kThreads) plan_place_kernel(const Rule r, const Plan plan, int blocks, int per) {
    __shared__ unsigned long long mask[kMaxExperts];
    __shared__ int32_t first[kMaxExperts], total[kMaxExperts];
    __shared__ int32_t warp_sums[kWarps];
    const int begin = blockIdx.x * per, end = min(blocks, begin + per);
    for (int e = threadIdx.x; e < kMaxExperts; e += kThreads) first[e] = total[e] = 0;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t pitch = count_pitch(r.experts);
    const int words = (r.experts + 3) / 4;
    const int rows = kThreads / words, w = threadIdx.x % words;   // (words is at most 128)
    if (threadIdx.x / words < rows) {
        int before[4] = {0, 0, 0, 0}, all[4] = {0, 0, 0, 0};
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
    const int start = write_starts(r, plan, e < r.experts ? total[e] : 0, blockIdx.x == 0, warp_sums);
    if (e < r.experts) first[e] += start;
    for (int b = begin; b < end; b++) {
        const int t0 = b * kBlockTokens, tokens = min(kBlockTokens, r.tokens - t0);
        masks_of(r, mask, t0, tokens, false);                     // (begins and ends with barriers around the masks)
        write_places(r, plan, mask, first, t0, tokens);
        __syncthreads();
        if (e < r.experts) first[e] += __popcll(mask[e]);
        __syncthreads();
    }
}

}  // namespace rt
}  // namespace bd
