// Attention of a step's queries over the paged cache, few rows per KV head (storage: paged_common.cuh).
//
//   o_i = sum_j p_ij v_j,  p_i = softmax over the visible j of  cap * tanh(scale * q_i . k_j / cap)  (or scale * q_i . k_j)
//
// with q in bf16 or fp16 as given, k and v the values the cache stands for (the rows of an unfinished value chunk in
// their source type).  Position kv - t + i sees the tokens up to itself, with a window w the last w of them.
//
// Work is counted in units of one chunk (32 tokens) of one KV head.  The units of the whole batch, sequence by sequence
// and head by head, are cut into equal runs, up to four per resident warp, so ragged batches load every SM alike; the warps of
// an SM take its runs in turn (the schedulers favour some warps: with one fixed share each, the last ones ended alone).
// A run that covers a head's visible chunks alone writes the result, the others leave (output, maximum, sum) in the workspace,
// which a second kernel joins in unit order: which warp did a run does not show in the result.  (One CTA per sequence,
// head and share instead left the SMs 40 % idle on 32 sequences of 1500 to 4113 tokens.)
// Both products run on the warp-level fp16 MMA with the cache as the 16-row operand and the queries (or the transposed
// probabilities) as the 8-column operand, so the few rows of a decode step fill half a tile and nothing of the cache is
// expanded twice.  A code becomes the fp16 number index-value * 2^-24 (a subnormal: the half-unit integer itself in the
// low byte, the sign on top) without any conversion; the block's power-of-two scale multiplies the fp32 block sum.  bf16
// queries are first scaled per row by a power of two into the range of fp16 (exact down to 2^-29 of the row's largest
// element).  Probabilities are rounded to fp16 (2^-11, and an absolute 2^-32 of the row's largest) for the second product, and their
// fp32 values are what the row sum adds; the unfinished chunk's values meet probabilities split in two bf16 parts (bf16 caches) or the same fp16 ones.
// What bounds it: the integer (ALU) pipe, which takes two cycles per warp instruction.  A code word costs ten of them, a
// block two; the left shift of a block's scale goes to the multiply-add pipe.  64 sequences of 6000 to 12000 tokens, 8 KV heads
// x 128: 211 us = 3.2 TB/s, that pipe 69 % busy, 924 warp instructions per chunk; the copies alone run at 5.5 TB/s (120 us).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "paged.cuh"

namespace bd {
namespace pg {

struct Attention {
    Pool pool;
    Batch batch;
    const uint8_t *q;
    int64_t ldq, hsq;                 // elements between rows / heads
    uint8_t *o;
    int64_t ldo, hso;
    float *lse;                       // [rows][q_heads] or null
    float *part;                      // partial results: of the warps' runs (rows kernel; see Runs), or of the splits
                                      // [splits][rows][q_heads][d + 2] (chunk kernel): output, maximum (log2 units), sum
    float scale;
    float score;                      // rows kernel: scale * log2 e * 2^23, from block sums to scores in units of log2 e
    float cap, cap_inv;               // the cap in units of log2 e, and its reciprocal
    int q_heads, group, window, splits, row_tiles, odtype;
    bool whole;                       // rows kernel: a CTA per head (workers: its warps)
    int workers, rounds;              // rows kernel: warps that share the units, runs per warp at most
    FastDiv by_runs[4], by_page, by_group;      // division by workers * (1 .. 4), by the chunks of a page, by `group`
    __device__ __forceinline__ int token(int row) const { return (int)fast_div((uint32_t)row, by_group); }     // of the sequence's rows
    uint8_t *images;                  // chunk kernel: expanded tiles (null: expanded by every CTA), [n][kv_heads][image_tiles]
    uint32_t *image_ok;
    int image_tiles;
    uint32_t *head_of_part;           // rows kernel: [n + 1] units in front of each sequence, then all units
    uint32_t k23;                     // 2^23: a left shift as a multiplication by an operand the compiler does not see
};

constexpr int kRowStages = 2;
constexpr float kPeak = 7.0f;         // log2 of a row's largest probability as it goes into fp16
constexpr int kRunUnits = 8;          // units that make a further round of runs worth its joins
__host__ __device__ constexpr int row_warps(int nt) { return nt == 1 ? 16 : 12; }    // warps of a CTA = of an SM, by registers

__device__ __forceinline__ void expand_f16(uint32_t w, uint2 tb, uint32_t (&r)[4]) {
    const uint32_t sel = w & 0x77777777u;
    const uint32_t xa = prmt_b32(tb.x, tb.y, sel), xb = prmt_b32(tb.x, tb.y, sel >> 16);
    const uint32_t odd = w & 0x80808080u, even = (w << 4) & 0x80808080u;   // signs of the odd / even nibbles, one per byte
    r[0] = prmt_b32(xa, even, 0x5240u);   // nibbles 0, 2 = elements 0, 1
    r[1] = prmt_b32(xa, odd, 0x5341u);    // nibbles 1, 3 = elements 2, 3
    r[2] = prmt_b32(xb, even, 0x7260u);   // nibbles 4, 6 = elements 4, 5
    r[3] = prmt_b32(xb, odd, 0x7361u);    // nibbles 5, 7 = elements 6, 7
}
// The same product without an accumulator in front.
__device__ __forceinline__ void mma_f16_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *(const uint32_t *)&h;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *(const uint32_t *)&h;
}
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// cap * tanh(y / cap) = cap * x P(x^2) / Q(x^2), x = y / cap within +-8 (where tanh is 1 - 2^-22).  The quotient was fitted here to
// tanh(x) / x with the constants 1 kept (iteratively reweighted least squares, relative error 2^-22.6); all coefficients are positive, so
// nothing cancels and scores keep their bits however large the cap is: within 2^-20 of the result in fp32.  (cap - 2 cap / (e^2x + 1), with an
// exponential more, is off by 2^-22 caps.)
constexpr float kCapP1 = 1.29303646e-01f, kCapP2 = 2.95581807e-03f, kCapP3 = 1.14752201e-05f;
constexpr float kCapQ1 = 4.62636188e-01f, kCapQ2 = 2.38358284e-02f, kCapQ3 = 2.39316360e-04f, kCapQ4 = 2.47326551e-07f;
__device__ __forceinline__ float cap_range(float x) {
    asm("min.NaN.f32 %0, %0, 0f41000000;\n\tmax.NaN.f32 %0, %0, 0fC1000000;" : "+f"(x));
    return x;
}
__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Two fp32 numbers of a 64-bit register: one issue slot for both.
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint64_t pair_of(float a) { return pair_of(a, a); }
__device__ __forceinline__ void unpair(uint64_t r, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t cap_pair(uint64_t y, float inverse, float cap) {
    float a, b;
    unpair(mul_pair(y, pair_of(inverse)), a, b);
    const uint64_t x = pair_of(cap_range(a), cap_range(b)), u = mul_pair(x, x);
    const uint64_t n = fma_pair(fma_pair(fma_pair(u, pair_of(kCapP3), pair_of(kCapP2)), u, pair_of(kCapP1)), u, pair_of(1.0f));
    const uint64_t d = fma_pair(fma_pair(fma_pair(fma_pair(u, pair_of(kCapQ4), pair_of(kCapQ3)), u, pair_of(kCapQ2)), u, pair_of(kCapQ1)), u, pair_of(1.0f));
    unpair(d, a, b);
    return mul_pair(mul_pair(x, n), mul_pair(pair_of(cap), pair_of(reciprocal(a), reciprocal(b))));
}

// One row's result: 2^23 is what the half-unit subnormals left out (2^-24 per code, 0.5 per half unit).
__device__ __forceinline__ void store_out(const Attention &p, int64_t row, int head, int ch, float v) {
    uint8_t *o = p.o + (row * p.ldo + (int64_t)head * p.hso + ch) * (p.odtype == BD_F32 ? 4 : 2);
    if (p.odtype == BD_F32) *(float *)o = v;
    else if (p.odtype == BD_BF16) *(__nv_bfloat16 *)o = __float2bfloat16_rn(v);
    else *(__half *)o = __float2half_rn(v);
}

// The chunks a sequence's rows see, and how the batch's units are numbered: sequence by sequence, KV head by KV head,
// chunk by chunk; a sequence with rows that see nothing counts one (empty) unit per head, so that its zeros are written.
struct Visible {
    int begin, end;                   // chunks; end > begin, or equal for the empty unit
    int units;                        // per head
};
__device__ __forceinline__ Visible visible_of(const Sequence &s, int window) {
    Visible v{0, 0, 0};
    if (!s.ok || s.t == 0) return v;
    v.begin = window ? max(0, s.kv - s.t - window + 1) / kChunk : 0;
    v.end = max((s.kv + kChunk - 1) / kChunk, v.begin);
    v.units = max(1, v.end - v.begin);
    return v;
}
// Runs: the first `extra` of them have size + 1 units, the others size.  (Unit numbers fit 32 bits: the entry point bounds
// n * kv_heads * chunks.)
struct Runs {
    uint32_t total, count, extra, size;
    __device__ uint32_t begin(uint32_t w) const { return w * size + min(w, extra); }
    __device__ uint32_t owner(uint32_t u) const {
        const uint32_t big = extra * (size + 1u);
        return u < big ? u / (size + 1u) : extra + (u - big) / size;
    }
};
__device__ __forceinline__ Runs runs_of(uint32_t total, const Attention &p) {
    const uint32_t round = (uint32_t)p.workers * kRunUnits;
    int k = 1;                                                    // rounds of runs
    while (k < p.rounds && total >= (uint32_t)(k + 1) * round) k++;
    if (total <= (uint32_t)p.workers) return Runs{total, total, 0, 1};
    Runs r{total, (uint32_t)(p.workers * k), 0, 0};
    r.size = fast_div(total, p.by_runs[k - 1]);
    r.extra = total - r.size * r.count;
    return r;
}
// One sequence per lane, 32 at a time.  The first 32 stay in registers, which is the whole batch for most decode steps.
struct Scan {
    uint32_t in_front, mine, first;                               // of this lane's sequence among the first 32; the 32's sum
};
__device__ __forceinline__ Scan scan_group(const Attention &p, int lane, int b0) {
    Scan s;
    s.mine = b0 + lane < p.batch.n ? (uint32_t)visible_of(sequence_of(p.batch, b0 + lane), p.window).units * (uint32_t)p.pool.kv_heads : 0u;
    uint32_t inc = s.mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, inc, d);
        if (lane >= d) inc += o;
    }
    s.in_front = inc - s.mine;
    s.first = __shfl_sync(0xffffffffu, inc, 31);
    return s;
}
__device__ __forceinline__ uint32_t all_units(const Attention &p, int lane, Scan &s) {
    s = scan_group(p, lane, 0);
    uint32_t sum = s.first;
    for (int b0 = 32; b0 < p.batch.n; b0 += 32) sum += scan_group(p, lane, b0).first;
    return sum;
}
// The sequence that holds unit u, and the units in front of it.
__device__ __forceinline__ int sequence_at(const Attention &p, int lane, const Scan &first, uint32_t u, uint32_t &before) {
    Scan s = first;
    uint32_t sum = 0;
    int b0 = 0;
    while (u >= sum + s.first && b0 + 32 < p.batch.n) {
        sum += s.first;
        b0 += 32;
        s = scan_group(p, lane, b0);
    }
    const int l = __ffs(__ballot_sync(0xffffffffu, u < sum + s.in_front + s.mine)) - 1;
    before = sum + __shfl_sync(0xffffffffu, s.in_front, l);
    return b0 + l;
}
// The partial results of run w: slot 2 w for the head that its first unit belongs to, 2 w + 1 for the head of its last unit.
// Per slot the fragments, 4 floats per lane and step, then maximum and sum per row.
template <int NB, int NT>
__device__ __host__ constexpr int part_floats() { return NT * NB * 2 * 128 + 2 * 8 * NT; }

template <int NB, int NT>
struct RowSmem {
    static constexpr int D = 32 * NB, ROWS = 8 * NT;
    static constexpr int warps = row_warps(NT), stage = 35 * D;
    static constexpr int table = 0, bars = 128, words = bars + warps * kRowStages * 8, ring = 512;      // the warps' records come last
    // per warp: its records, then its queries' fragments
    static constexpr int queries = kRowStages * stage, per_warp = (queries + NT * NB * 512 + 127) / 128 * 128;
    static constexpr int bytes(int warps) { return ring + warps * per_warp; }
    static_assert(words + 16 <= ring, "room for the table and the barriers");
};

// What a warp keeps of the head it works on.
template <int DT, int NB, int NT, bool CAP>
struct RowWork {
    static constexpr int D = 32 * NB;
    uint4 *qf;                                                    // queries: fragments of the 8-column operand in fp16, [NT][NB][32 lanes] (shared memory)
    float mul[NT][2];                                             // bf16: the power of two that the column's query was divided by
    int pos[NT][2];
    float O[NT][NB][2][4], m_run[NT][2], l_run[NT][2];
    Sequence s;
    int h, n_rows, first_pos, last_pos, full;

    // A head begins: its queries, and nothing seen yet.
    __device__ __forceinline__ void begin(const Attention &p, const Sequence &seq, int head, uint4 *fragments, int lane) {
        const int g = lane / 4, t4 = lane % 4;
        s = seq;
        h = head;
        qf = fragments + lane;
        n_rows = s.t * p.group;
        first_pos = s.kv - s.t;
        last_pos = s.kv - 1;
        full = s.kv / kChunk;
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            const int r = 8 * nt + g;
            const bool valid = r < n_rows;
            const uint8_t *src = p.q + ((int64_t)(s.q0 + p.token(r)) * p.ldq + (int64_t)(h * p.group + (r - p.token(r) * p.group)) * p.hsq) * 2;
            uint4 raw[NB];
#pragma unroll
            for (int b = 0; b < NB; b++) raw[b] = valid ? *(const uint4 *)(src + (32 * b + 8 * t4) * 2) : make_uint4(0, 0, 0, 0);
            float qs = 1.0f;
            if (DT == BD_BF16) {
                uint32_t m = 0;
#pragma unroll
                for (int b = 0; b < NB; b++) m = absmax_bf16x2(m, absmax_bf16x2(absmax_bf16x2(raw[b].x, raw[b].y), absmax_bf16x2(raw[b].z, raw[b].w)));
                m = max(m & 0x7fffu, m >> 16 & 0x7fffu);
                m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
                m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
                const int ex = min(max((int)(m >> 7), 27), 254);      // biased exponent of the row's largest element
                const float up = __uint_as_float((uint32_t)(127 + 14 + 127 - ex) << 23);
                qs = __uint_as_float((uint32_t)(ex - 14) << 23);
#pragma unroll
                for (int b = 0; b < NB; b++) {
                    const uint32_t w[4] = {raw[b].x, raw[b].y, raw[b].z, raw[b].w};
                    uint32_t f[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) f[i] = pack_f16(__uint_as_float(w[i] << 16) * up, __uint_as_float(w[i] & 0xffff0000u) * up);
                    qf[(nt * NB + b) * 32] = make_uint4(f[0], f[1], f[2], f[3]);
                }
            } else {
#pragma unroll
                for (int b = 0; b < NB; b++) qf[(nt * NB + b) * 32] = raw[b];
            }
#pragma unroll
            for (int i = 0; i < 2; i++) {                     // this lane's columns 2 t4 + i of the score fragments
                mul[nt][i] = __shfl_sync(0xffffffffu, qs, 4 * (2 * t4 + i));
                const int rc = 8 * nt + 2 * t4 + i;
                pos[nt][i] = rc < n_rows ? first_pos + p.token(rc) : -1;
                m_run[nt][i] = -INFINITY;
                l_run[nt][i] = 0.0f;
            }
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
                for (int i = 0; i < 8; i++) O[nt][b][i / 4][i % 4] = 0.0f;
        }
    }

    // The 32 tokens of chunk c, whose record is at `rec` (shared memory); table: the dialects' magnitudes.
    __device__ __forceinline__ void chunk(const Attention &p, const uint8_t *rec, const uint8_t *table, int at, int c, int lane) {
        const int g = lane / 4, t4 = lane % 4;
        // scale bytes of the lane's four rows (a word per row, a byte per tile) and 8 * id as bytes, likewise
        uint32_t scl[4], ide[4];
        auto load_entries = [&](int64_t scales, int64_t ids) {
            if (NB == 4) {
                const uint4 u = *(const uint4 *)(rec + scales + 16 * g);
                scl[0] = u.x; scl[1] = u.y; scl[2] = u.z; scl[3] = u.w;
                const uint2 v = *(const uint2 *)(rec + ids + 8 * g);
                ide[0] = v.x * 8u & 0x78787878u;              // even tiles of rows j = 0, 1: bytes 2 j + b / 2
                ide[1] = v.x >> 1 & 0x78787878u;              // odd tiles
                ide[2] = v.y * 8u & 0x78787878u;
                ide[3] = v.y >> 1 & 0x78787878u;
            } else {
                const uint2 u = *(const uint2 *)(rec + scales + 8 * g);
                scl[0] = u.x; scl[1] = u.x >> 16; scl[2] = u.y; scl[3] = u.y >> 16;
                const uint32_t v = *(const uint32_t *)(rec + ids + 4 * g);
                ide[0] = v * 8u & 0x78787878u;                // even tiles of row j: byte j
                ide[1] = v >> 1 & 0x78787878u;
            }
        };
        auto table_of = [&](int j, int b) {
            const uint32_t x = NB == 4 ? ide[2 * (j / 2) + b % 2] : ide[b % 2];
            const int byte = NB == 4 ? 2 * (j % 2) + b / 2 : j;
            return *(const uint2 *)(table + prmt_b32(x, 0u, 0x4440u + byte));
        };
        auto factor_of = [&](int j, int b) { return __uint_as_float(prmt_b32(scl[j], 0u, 0x4440u + b) * p.k23); };   // 2^e (scale byte 0: below 2^-126)
        float sc[NT][2][4];
        load_entries(key_scales(D), key_ids(D));
#pragma unroll
        for (int b = 0; b < NB; b++) {
            const uint4 w4 = *(const uint4 *)(rec + b * 512 + lane * 16);
            const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
            uint32_t a[4][4];
#pragma unroll
            for (int j = 0; j < 4; j++) expand_f16(w[j], table_of(j, b), a[j]);
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                const uint4 q = qf[(nt * NB + b) * 32];          // (this lane wrote it)
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    float acc[4];
                    mma_f16_zero(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], q.x, q.y);
                    mma_f16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], q.z, q.w);
                    const float f0 = factor_of(2 * x, b), f1 = factor_of(2 * x + 1, b);
                    sc[nt][x][0] = b ? fmaf(acc[0], f0, sc[nt][x][0]) : acc[0] * f0;
                    sc[nt][x][1] = b ? fmaf(acc[1], f0, sc[nt][x][1]) : acc[1] * f0;
                    sc[nt][x][2] = b ? fmaf(acc[2], f1, sc[nt][x][2]) : acc[2] * f1;
                    sc[nt][x][3] = b ? fmaf(acc[3], f1, sc[nt][x][3]) : acc[3] * f1;
                }
            }
        }
        // ---- softmax: rows of the fragment are tokens (row 8 j + g = token 8 (g / 2) + 2 j + g % 2), columns queries ----
        const int tok0 = c * kChunk + 8 * (g / 2) + g % 2;
        const bool masked = (c + 1) * kChunk > first_pos + 1 || (p.window && c * kChunk <= last_pos - p.window);
        // m_run, the same in the eight lanes of a column, is kPeak below the running maximum and moves only when a score exceeds it
        // by kPeak + 8: probabilities are up to 2^15 (fp16 ends at 2^16, sums are fp32), so that fp16's subnormals begin at 2^-21 of the
        // row's largest and lose 2^-32 of it; without a move no lane needs another's scores.
        uint32_t pf[NT][4];
        bool grew = false;
        float x[NT][4][2], top[NT][2], pv[NT][4][2];
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                // (the power first: with the scale's factors it could pass the range of fp32, where the score does not)
                uint64_t y = pair_of(sc[nt][j / 2][2 * (j % 2)], sc[nt][j / 2][2 * (j % 2) + 1]);
                if (DT == BD_BF16) y = mul_pair(y, pair_of(mul[nt][0], mul[nt][1]));
                y = mul_pair(y, pair_of(p.score));
                if (CAP) y = cap_pair(y, p.cap_inv, p.cap);
                unpair(y, x[nt][j][0], x[nt][j][1]);
            }
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    float &y = x[nt][j][i];
                    if (masked) {
                        const int tok = tok0 + 2 * j;
                        if (tok > pos[nt][i] || (p.window && tok <= pos[nt][i] - p.window)) y = -INFINITY;
                    }
                }
                top[nt][i] = fmaxf(fmaxf(x[nt][0][i], x[nt][1][i]), fmaxf(x[nt][2][i], x[nt][3][i]));
                grew |= top[nt][i] > m_run[nt][i] + (kPeak + 8.0f);
            }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    float m = fmaxf(top[nt][i] - kPeak, m_run[nt][i]);
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                    const float alpha = m == -INFINITY ? 1.0f : fast_exp2(m_run[nt][i] - m);
                    m_run[nt][i] = m;
                    l_run[nt][i] *= alpha;
#pragma unroll
                    for (int b = 0; b < NB; b++)
#pragma unroll
                        for (int y = 0; y < 4; y++) O[nt][b][y / 2][2 * (y % 2) + i] *= alpha;
                }
        }
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float base = m_run[nt][i] == -INFINITY ? 0.0f : m_run[nt][i];
#pragma unroll
                for (int j = 0; j < 4; j++) pv[nt][j][i] = fast_exp2(x[nt][j][i] - base);
                l_run[nt][i] += (pv[nt][0][i] + pv[nt][1][i]) + (pv[nt][2][i] + pv[nt][3][i]);
            }
        if (c < full) {
            // ---- values stored in 4 bits ----
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int j = 0; j < 4; j++) pf[nt][j] = transpose8x8(pack_f16(pv[nt][j][0], pv[nt][j][1]));
            load_entries(value_scales(D), value_ids(D));
#pragma unroll
            for (int b = 0; b < NB; b++) {
                const uint4 w4 = *(const uint4 *)(rec + value_codes(D) + b * 512 + lane * 16);
                const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
                uint32_t a[4][4];
#pragma unroll
                for (int j = 0; j < 4; j++) expand_f16(w[j], table_of(j, b), a[j]);
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        float acc[4];
                        mma_f16_zero(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], pf[nt][0], pf[nt][1]);
                        mma_f16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], pf[nt][2], pf[nt][3]);
                        const float f0 = factor_of(2 * x, b), f1 = factor_of(2 * x + 1, b);
                        O[nt][b][x][0] = fmaf(acc[0], f0, O[nt][b][x][0]);
                        O[nt][b][x][1] = fmaf(acc[1], f0, O[nt][b][x][1]);
                        O[nt][b][x][2] = fmaf(acc[2], f1, O[nt][b][x][2]);
                        O[nt][b][x][3] = fmaf(acc[3], f1, O[nt][b][x][3]);
                    }
            }
        } else {
            // ---- the unfinished chunk: rows of the tail; tokens behind the last one count as zeros ----
            uint32_t lo[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    float a = pv[nt][j][0], b = pv[nt][j][1];
                    if (DT == BD_BF16) {                          // (in the units of O: bf16's values may be as large as fp32's)
                        a *= 1.0f / 8388608.0f;
                        b *= 1.0f / 8388608.0f;
                        const uint32_t hi = pack_bf16(a, b);
                        pf[nt][j] = transpose8x8(hi);
                        lo[nt][j] = transpose8x8(pack_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u)));
                    } else {
                        pf[nt][j] = transpose8x8(pack_f16(a, b));
                    }
                }
            const int slot = p.batch.slot[at];
            const bool slot_ok = slot >= 0 && slot < p.pool.slots;
            if (!slot_ok && lane == 0) atomicOr(&g_status_word, kStatusIndex);
            const uint16_t *tail = (const uint16_t *)p.pool.tail + tail_offset(p.pool, slot_ok ? slot : 0, h, c * kChunk);
            const int left = slot_ok ? s.kv - c * kChunk : 0;
#pragma unroll
            for (int b = 0; b < NB; b++) {
                uint32_t a[4][4];
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {             // rows 2 a + i of the 8 x 8 tile: tokens 8 a + 2 e + i
                        const int tok = 8 * (g / 2) + 2 * e + g % 2;
                        a[j][e] = transpose8x8(tok < left ? *(const uint32_t *)(tail + tok * D + 32 * b + 8 * j + 2 * t4) : 0u);
                    }
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        if (DT == BD_BF16) {
                            float (&acc)[4] = O[nt][b][x];
                            mma_bf16(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], pf[nt][0], pf[nt][1]);
                            mma_bf16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], pf[nt][2], pf[nt][3]);
                            mma_bf16(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], lo[nt][0], lo[nt][1]);
                            mma_bf16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], lo[nt][2], lo[nt][3]);
                        } else {
                            float acc[4];
                            mma_f16_zero(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], pf[nt][0], pf[nt][1]);
                            mma_f16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], pf[nt][2], pf[nt][3]);
#pragma unroll
                            for (int y = 0; y < 4; y++) O[nt][b][x][y] = fmaf(acc[y], 1.0f / 8388608.0f, O[nt][b][x][y]);
                        }
                    }
            }
        }
    }

    // The warp's sums over the tokens are in place in every lane.
    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                float &l = l_run[nt][i];
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
            }
    }
    // The fragments, then maximum and sum per row, in the order the joins read.
    __device__ __forceinline__ void store_part(float *to, int lane) const {
        const int g = lane / 4, t4 = lane % 4;
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            if (8 * nt + 2 * t4 < n_rows)
#pragma unroll
                for (int b = 0; b < NB; b++)
#pragma unroll
                    for (int x = 0; x < 2; x++) *(float4 *)(to + (((nt * NB + b) * 2 + x) * 32 + lane) * 4) = make_float4(O[nt][b][x][0], O[nt][b][x][1], O[nt][b][x][2], O[nt][b][x][3]);
            if (g == 0)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    float *ml = to + NT * NB * 2 * 128 + 2 * (8 * nt + 2 * t4 + i);
                    ml[0] = m_run[nt][i];
                    ml[1] = l_run[nt][i];
                }
        }
    }
};

// Writes one head's rows from the fragments: this lane holds channels 32 b + 8 j + g of rows 8 nt + 2 t4 + i.
template <int DT, int NB, int NT, bool CAP>
__device__ __forceinline__ void store_rows(const Attention &p, const RowWork<DT, NB, NT, CAP> &k, int lane) {
    const int g = lane / 4, t4 = lane % 4;
#pragma unroll
    for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int r = 8 * nt + 2 * t4 + i;
            if (r >= k.n_rows) continue;
            const int64_t row = k.s.q0 + p.token(r);
            const int head = k.h * p.group + (r - p.token(r) * p.group);
            const float lr = k.l_run[nt][i], f = lr > 0.0f ? 8388608.0f / lr : (lr == 0.0f ? 0.0f : lr);
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
                for (int j = 0; j < 4; j++) store_out(p, row, head, 32 * b + 8 * j + g, k.O[nt][b][j / 2][2 * (j % 2) + i] * f);
            if (g == 0 && p.lse) p.lse[row * p.q_heads + head] = lr > 0.0f ? (k.m_run[nt][i] + log2f(lr)) * 0.6931471805599453f : (lr == 0.0f ? -INFINITY : lr);
        }
}

// Waits for a record.  (The loop that polls is not inlined: it would cost the callers registers.)
__device__ __noinline__ bool wait_longer(uint32_t bar, uint32_t parity, volatile uint32_t *flags) { return tc::mbar_wait_warp(bar, parity, flags); }
__device__ __forceinline__ bool wait_record(uint32_t bar, uint32_t parity, volatile uint32_t *flags) {
    return __all_sync(0xffffffffu, tc::mbar_try_wait(bar, parity)) || wait_longer(bar, parity, flags);
}
// A warp's wait ran out (status word).  Copies that may be in flight arrive first (a stage without one costs the limit); then its run's parts,
// and those of all the runs it would still take, get a negative sum, by which the join kernel knows that they were not written.
// (Not inlined: it would cost the main loop registers.)
__device__ __noinline__ void drain_stages(uint32_t bar0, uint32_t phase) {
    for (int st = 0; st < kRowStages; st++) tc::mbar_drain(bar0 + 8 * st, phase >> st & 1u);
}
template <int NB, int NT>
__device__ __noinline__ void give_up(float *part, uint32_t count, uint32_t run, uint32_t turn, volatile uint32_t *flags, uint32_t bar0, uint32_t phase, int lane) {
    drain_stages(bar0, phase);
    while (run < count) {
        for (int i = lane; i < 16 * NT; i += 32) part[(int64_t)(2 * run + i % 2) * part_floats<NB, NT>() + NT * NB * 2 * 128 + 2 * (i / 2) + 1] = -1.0f;
        run = turn * gridDim.x + blockIdx.x;
        if (lane == 0) turn = atomicAdd((uint32_t *)&flags[3], 1u);
        turn = __shfl_sync(0xffffffffu, turn, 0);
    }
}

template <int DT, int NB, int NT, bool CAP>
__global__ void __launch_bounds__(32 * row_warps(NT), 1) attention_rows_kernel(const __grid_constant__ Attention p) {
    using S = RowSmem<NB, NT>;
    extern __shared__ __align__(128) uint8_t smem[];
    volatile uint32_t *flags = (volatile uint32_t *)(smem + S::words);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (threadIdx.x < 16) ((uint2 *)(smem + S::table))[threadIdx.x] = make_uint2(c_tables.int_lo[threadIdx.x], c_tables.int_hi[threadIdx.x]);
    if (threadIdx.x == 0) {
        flags[0] = 0; flags[1] = 1;
        flags[2] = g_debug_spin_limit ? g_debug_spin_limit : tc::kSpinLimit;
        flags[3] = S::warps;                                      // the SM's next run: each warp begins with that of its own number
    }
    const uint32_t bar0 = tc::smem_u32(smem + S::bars) + warp * kRowStages * 8;
    if (lane == 0)
        for (int i = 0; i < kRowStages; i++) tc::mbar_init(bar0 + 8 * i, i + warp + blockIdx.x == 0 && g_debug_skip_first_code_stage ? 2 : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    pdl_wait();
    pdl_release();

    if (warp * gridDim.x + blockIdx.x >= (uint32_t)(p.workers * p.rounds)) return;
    Scan first;
    const uint32_t total = all_units(p, lane, first);
    const Runs runs = runs_of(total, p);
    if (blockIdx.x == 0 && warp == 0)                             // sequences with bad numbers have no units: told here
        for (int b = lane; b < p.batch.n; b += 32)
            if (!sequence_of(p.batch, b).ok) atomicOr(&g_status_word, kStatusIndex);
    // the join kernel finds its parts with these
    if (blockIdx.x == gridDim.x - 1 && warp == 0) {
        uint32_t sum = 0;
        for (int b0 = 0; b0 < p.batch.n; b0 += 32) {
            const Scan sc = b0 ? scan_group(p, lane, b0) : first;
            if (b0 + lane < p.batch.n) p.head_of_part[b0 + lane] = sum + sc.in_front;
            sum += sc.first;
        }
        if (lane == 0) p.head_of_part[p.batch.n] = sum;
    }
    if (total == 0) return;
    uint8_t *const ring = smem + S::ring + warp * S::per_warp;
    uint32_t loaded = 0, phase = 0;                               // bits per stage: a record is in flight or there; the barrier's parity
    const int per_page = p.pool.chunks_per_page;

  // run r is the SM r % gridDim's: heads of one sequence spread over the SMs
  for (uint32_t turn = warp;;) {
    const uint32_t run = turn * gridDim.x + blockIdx.x;
    if (run >= runs.count) return;
    if (lane == 0) turn = atomicAdd((uint32_t *)&flags[3], 1u);
    turn = __shfl_sync(0xffffffffu, turn, 0);
    const uint32_t u_begin = runs.begin(run);
    const int n_units = (int)(runs.begin(run + 1) - u_begin);
    uint32_t before;
    // the place in the run that is worked on: sequence, head, chunk
    int at = sequence_at(p, lane, first, u_begin, before);
    Visible v = visible_of(sequence_of(p.batch, at), p.window);
    int h = (int)((u_begin - before) / (uint32_t)v.units);
    int c = v.begin + (int)(u_begin - before - (uint32_t)(h * v.units));
    // the place whose record is fetched next, two units ahead; the page numbers come a page early
    int a_at = at, a_h = h, a_c = c, a_in = 0, a_next = -1, fetched = 0;
    Visible a_v = v;
    const uint8_t *a_src = nullptr;                               // nullptr: a page number outside the pool
    auto page_at = [&](int page) -> const uint8_t * {
        if (page < 0 || page >= p.pool.pages) {
            if (lane == 0) atomicOr(&g_status_word, kStatusIndex);
            return nullptr;
        }
        return p.pool.base + (((int64_t)page * p.pool.kv_heads + a_h) * per_page + a_in) * S::stage;
    };
    auto enter = [&]() {                                          // a head, from chunk a_c on
        if (a_c >= a_v.end) { a_src = nullptr; return; }          // (the empty unit)
        const int32_t *row = p.batch.table + (int64_t)a_at * p.batch.ld_table + fast_div(a_c, p.by_page);
        a_in = a_c - (int)fast_div(a_c, p.by_page) * per_page;
        a_src = page_at(row[0]);
        a_next = a_c + per_page - a_in < a_v.end ? row[1] : -1;
    };
    auto fetch = [&]() {
        const int st = fetched % kRowStages;
        loaded = a_src ? loaded | 1u << st : loaded & ~(1u << st);
        if (a_src && lane == 0) {
            tc::mbar_expect_tx(bar0 + 8 * st, S::stage);
            tc::bulk_load(tc::smem_u32(ring + st * S::stage), a_src, S::stage, bar0 + 8 * st);
        }
        if (++fetched == n_units) return;
        if (++a_c < a_v.begin + a_v.units) {
            if (++a_in < per_page) {
                if (a_src) a_src += S::stage;
            } else {
                a_in = 0;
                a_src = page_at(a_next);
                if (a_c + per_page < a_v.end) a_next = p.batch.table[(int64_t)a_at * p.batch.ld_table + fast_div(a_c, p.by_page) + 1];
            }
            return;
        }
        if (++a_h == p.pool.kv_heads) {
            a_h = 0;
            do {
                a_at++;
                a_v = visible_of(sequence_of(p.batch, a_at), p.window);
            } while (a_v.units == 0);
        }
        a_c = a_v.begin;
        enter();
    };
    enter();
    for (int i = 0; i < kRowStages && i < n_units; i++) fetch();

    RowWork<DT, NB, NT, CAP> work;
    bool starts_head = true;                                      // this piece begins at the head's first unit
    for (int unit = 0; unit < n_units; unit++) {
        if (unit == 0 || c == v.begin) {                          // a head begins (or the run does, inside one)
            work.begin(p, sequence_of(p.batch, at), h, (uint4 *)(ring + S::queries), lane);
            starts_head = c == v.begin;
        }
        const int st = unit % kRowStages;
        if (loaded >> st & 1u) {
            if (!wait_record(bar0 + 8 * st, phase >> st & 1u, flags)) {
                give_up<NB, NT>(p.part, runs.count, run, turn, flags, bar0, phase, lane);
                return;
            }
            phase ^= 1u << st;
            work.chunk(p, ring + st * S::stage, smem + S::table, at, c, lane);
        }
        __syncwarp();                                             // every lane is done with the stage
        if (fetched < n_units) fetch();
        const bool ends_head = c + 1 == v.begin + v.units;
        if (ends_head || unit + 1 == n_units) {
            // the piece is done: the head's result, or a part of it
            work.finish();
            if (starts_head && ends_head) {
                store_rows(p, work, lane);
            } else {
                // the piece at the run's start has slot 0; one that begins a head later in the run is the run's last: slot 1
                const bool at_start = unit <= c - v.begin;
                work.store_part(p.part + (int64_t)(2 * run + (at_start ? 0 : 1)) * part_floats<NB, NT>(), lane);
            }
        }
        if (ends_head && unit + 1 < n_units) {
            if (++h == p.pool.kv_heads) {
                h = 0;
                do {
                    at++;
                    v = visible_of(sequence_of(p.batch, at), p.window);
                } while (v.units == 0);
            }
            c = v.begin;
        } else {
            c++;
        }
    }
  }
}

// Short contexts: a CTA takes a whole head, its warps the head's chunks in turn, and the warps' parts meet in shared memory,
// so that the call is one launch (one sequence of 513 tokens: 9.4 us a call against 11.3 through runs and the join kernel).
template <int DT, int NB, int NT, bool CAP>
__global__ void __launch_bounds__(32 * row_warps(NT), 1) attention_head_kernel(const __grid_constant__ Attention p) {
    using S = RowSmem<NB, NT>;
    static_assert(part_floats<NB, NT>() * 4 <= S::per_warp, "a warp's part takes the place of its records");
    extern __shared__ __align__(128) uint8_t smem[];
    volatile uint32_t *flags = (volatile uint32_t *)(smem + S::words);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32, h = blockIdx.x, seq = blockIdx.y;
    if (threadIdx.x < 16) ((uint2 *)(smem + S::table))[threadIdx.x] = make_uint2(c_tables.int_lo[threadIdx.x], c_tables.int_hi[threadIdx.x]);
    if (threadIdx.x == 0) {
        flags[0] = 0; flags[1] = 1;
        flags[2] = g_debug_spin_limit ? g_debug_spin_limit : tc::kSpinLimit;
    }
    const uint32_t bar0 = tc::smem_u32(smem + S::bars) + warp * kRowStages * 8;
    if (lane == 0)
        for (int i = 0; i < kRowStages; i++) tc::mbar_init(bar0 + 8 * i, i + warp + blockIdx.x + blockIdx.y == 0 && g_debug_skip_first_code_stage ? 2 : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    pdl_wait();
    pdl_release();
    const Sequence s = sequence_of(p.batch, seq);
    if (!s.ok) {
        if (threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
        return;
    }
    if (s.t == 0) return;
    const Visible v = visible_of(s, p.window);
    uint8_t *const ring = smem + S::ring + warp * S::per_warp;
    const int n = v.end > v.begin + warp ? (v.end - v.begin - warp + warps - 1) / warps : 0;     // this warp's chunks
    const int32_t *pages = p.batch.table + (int64_t)seq * p.batch.ld_table;
    uint32_t loaded = 0, phase = 0;
    int page = -1;
    auto look_up = [&](int i) { if (i < n) page = pages[fast_div(v.begin + warp + i * warps, p.by_page)]; };
    auto fetch = [&](int i) {
        const int st = i % kRowStages, c = v.begin + warp + i * warps;
        const bool ok = page >= 0 && page < p.pool.pages;
        if (!ok && lane == 0) atomicOr(&g_status_word, kStatusIndex);
        loaded = ok ? loaded | 1u << st : loaded & ~(1u << st);
        if (ok && lane == 0) {
            const int in = c - (int)fast_div(c, p.by_page) * p.pool.chunks_per_page;
            tc::mbar_expect_tx(bar0 + 8 * st, S::stage);
            tc::bulk_load(tc::smem_u32(ring + st * S::stage), p.pool.base + (((int64_t)page * p.pool.kv_heads + h) * p.pool.chunks_per_page + in) * S::stage, S::stage, bar0 + 8 * st);
        }
        look_up(i + 1);
    };
    look_up(0);
    for (int i = 0; i < kRowStages && i < n; i++) fetch(i);
    RowWork<DT, NB, NT, CAP> work;
    work.begin(p, s, h, (uint4 *)(ring + S::queries), lane);
    for (int i = 0; i < n; i++) {
        const int st = i % kRowStages;
        if (loaded >> st & 1u) {
            if (!wait_record(bar0 + 8 * st, phase >> st & 1u, flags)) {
                drain_stages(bar0, phase);
                break;
            }
            phase ^= 1u << st;
            work.chunk(p, ring + st * S::stage, smem + S::table, seq, v.begin + warp + i * warps, lane);
        }
        __syncwarp();
        if (i + kRowStages < n) fetch(i + kRowStages);
    }
    work.finish();
    __syncwarp();                                                 // (the warp's records are read)
    work.store_part((float *)ring, lane);
    __syncthreads();
    if (flags[0]) return;                                         // a wait ran out (status word): nothing is written
    // thread = fragment piece and lane, as in the join kernel
    for (int i = threadIdx.x; i < NT * NB * 2 * 32; i += blockDim.x) {
        const int piece = i / 32, nt = piece / (2 * NB), b = piece / 2 % NB, x = piece % 2, t4 = lane % 4, g = lane / 4;
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int r = 8 * nt + 2 * t4 + k;
            if (r >= work.n_rows) continue;
            float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
            for (int w = 0; w < warps; w++) m = fmaxf(m, ((const float *)(smem + S::ring + w * S::per_warp))[NT * NB * 2 * 128 + 2 * r]);
            const float zero = m == -INFINITY ? 0.0f : m;
            for (int w = 0; w < warps; w++) {
                const float *part = (const float *)(smem + S::ring + w * S::per_warp);
                const float f = fast_exp2(part[NT * NB * 2 * 128 + 2 * r] - zero);
                l = fmaf(part[NT * NB * 2 * 128 + 2 * r + 1], f, l);
                o0 = fmaf(part[(piece * 32 + lane) * 4 + k], f, o0);
                o1 = fmaf(part[(piece * 32 + lane) * 4 + 2 + k], f, o1);
            }
            const int64_t row = s.q0 + p.token(r);
            const int head = h * p.group + (r - p.token(r) * p.group);
            const float f = l > 0.0f ? 8388608.0f / l : (l == 0.0f ? 0.0f : l);
            store_out(p, row, head, 32 * b + 16 * x + g, o0 * f);
            store_out(p, row, head, 32 * b + 16 * x + 8 + g, o1 * f);
            if (b == 0 && x == 0 && g == 0 && p.lse) p.lse[row * p.q_heads + head] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : (l == 0.0f ? -INFINITY : l);
        }
    }
}

// Joins the parts of heads that several runs share, in unit order.  A CTA per sequence and KV head; thread = the fragment
// piece (row group nt, channels b, half x, lane) that it adds up, the rows' weights come from shared memory.
template <int NB, int NT>
__global__ void __launch_bounds__(64 * NB * NT) attention_rows_join_kernel(const __grid_constant__ Attention p) {
    constexpr int ROWS = 8 * NT, kParts = 64, kAhead = 8, THREADS = 64 * NB * NT;
    __shared__ float2 ml[kParts][ROWS];                           // maximum and sum, then weight and weighted sum
    __shared__ float keep[ROWS], top[ROWS], sums[ROWS];
    const int h = blockIdx.x, seq = blockIdx.y, lane = threadIdx.x % 32, t4 = lane % 4, g = lane / 4;
    const int piece = threadIdx.x / 32, nt = piece / (2 * NB), b = piece / 2 % NB, x = piece % 2;
    pdl_wait();
    pdl_release();
    const uint32_t total = p.head_of_part[p.batch.n], before = p.head_of_part[seq];
    const Sequence s = sequence_of(p.batch, seq);
    const Visible v = visible_of(s, p.window);
    if (v.units <= 1) return;                                     // nothing to do, or never shared
    const Runs runs = runs_of(total, p);
    const uint32_t u0 = before + (uint32_t)(h * v.units), u1 = u0 + (uint32_t)v.units;
    const int w0 = (int)runs.owner(u0), w1 = (int)runs.owner(u1 - 1);
    if (w0 == w1) return;
    const int n_rows = s.t * p.group, first_slot = runs.begin(w0) >= u0 ? 0 : 1;   // (only the first run can begin in front of the head)
    auto part_of = [&](int w) { return p.part + (int64_t)(2 * w + (w == w0 ? first_slot : 0)) * part_floats<NB, NT>(); };
    const bool active = 8 * nt + 2 * t4 < n_rows;
    float O[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int base = w0; base <= w1; base += kParts) {
        const int n = min(kParts, w1 - base + 1);
        float4 ahead[kAhead];                                     // the first parts' values, in flight while the weights are made
        auto load = [&](int k) { return active && k < n ? *(const float4 *)(part_of(base + k) + (piece * 32 + lane) * 4) : make_float4(0.0f, 0.0f, 0.0f, 0.0f); };
#pragma unroll
        for (int k = 0; k < kAhead; k++) ahead[k] = load(k);
        bool missing = false;
        for (int i = threadIdx.x; i < n * ROWS; i += THREADS) {
            const int r = i % ROWS;
            if (r < n_rows) {
                const float2 x = *(const float2 *)(part_of(base + i / ROWS) + NT * NB * 2 * 128 + 2 * r);
                ml[i / ROWS][r] = x;
                missing |= x.y < 0.0f;
            }
        }
        if (__syncthreads_or(missing)) return;                    // a warp gave up: the head's rows stay unwritten
        for (int r = piece; r < n_rows; r += THREADS / 32) {      // a warp per row
            const float2 a = lane < n ? ml[lane][r] : make_float2(-INFINITY, 0.0f), c = lane + 32 < n ? ml[lane + 32][r] : make_float2(-INFINITY, 0.0f);
            const float old = base == w0 ? -INFINITY : top[r];
            float m = fmaxf(fmaxf(a.x, c.x), old);
#pragma unroll
            for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            const float zero = m == -INFINITY ? 0.0f : m, fa = fast_exp2(a.x - zero), fc = fast_exp2(c.x - zero);
            float l = fmaf(a.y, fa, c.y * fc);
#pragma unroll
            for (int d = 16; d; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
            if (lane < n) ml[lane][r].x = fa;
            if (lane + 32 < n) ml[lane + 32][r].x = fc;
            if (lane == 0) {
                const float k = fast_exp2(old - zero);
                keep[r] = k;
                sums[r] = base == w0 ? l : fmaf(sums[r], k, l);
                top[r] = m;
            }
        }
        __syncthreads();
        if (active) {
            const int r = 8 * nt + 2 * t4;
            const bool two = r + 1 < n_rows;
            if (base != w0) {
                O[0] *= keep[r]; O[2] *= keep[r];
                if (two) { O[1] *= keep[r + 1]; O[3] *= keep[r + 1]; }
            }
            auto add = [&](int k, const float4 &a) {
                const float f0 = ml[k][r].x, f1 = two ? ml[k][r + 1].x : 0.0f;
                O[0] = fmaf(a.x, f0, O[0]);
                O[1] = fmaf(a.y, f1, O[1]);
                O[2] = fmaf(a.z, f0, O[2]);
                O[3] = fmaf(a.w, f1, O[3]);
            };
#pragma unroll
            for (int k = 0; k < kAhead; k++)
                if (k < n) add(k, ahead[k]);
            for (int k0 = kAhead; k0 < n; k0 += kAhead) {
#pragma unroll
                for (int k = 0; k < kAhead; k++) ahead[k] = load(k0 + k);
#pragma unroll
                for (int k = 0; k < kAhead; k++)
                    if (k0 + k < n) add(k0 + k, ahead[k]);
            }
        }
        __syncthreads();                                          // (the weights are read; the next round overwrites them)
    }
    if (!active) return;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int r = 8 * nt + 2 * t4 + i;
        if (r >= n_rows) continue;
        const int64_t row = s.q0 + p.token(r);
        const int head = h * p.group + (r - p.token(r) * p.group);
        const float l = sums[r], f = l > 0.0f ? 8388608.0f / l : (l == 0.0f ? 0.0f : l);
#pragma unroll
        for (int j = 0; j < 2; j++) store_out(p, row, head, 32 * b + 16 * x + 8 * j + g, O[2 * j + i] * f);
        if (b == 0 && x == 0 && g == 0 && p.lse) p.lse[row * p.q_heads + head] = l > 0.0f ? (top[r] + log2f(l)) * 0.6931471805599453f : (l == 0.0f ? -INFINITY : l);
    }
}

// Joins the splits of a row (chunk kernel), in split order.  A warp per row and head.
template <int D>
__global__ void __launch_bounds__(128) attention_join_kernel(const __grid_constant__ Attention p) {
    pdl_wait();
    pdl_release();
    const int seq = blockIdx.z, head = blockIdx.y, lane = threadIdx.x % 32;
    const Sequence s = sequence_of(p.batch, seq);
    const int i = blockIdx.x * 4 + threadIdx.x / 32;
    if (!s.ok || i >= s.t) return;
    const int64_t row = s.q0 + i, step = (int64_t)p.batch.rows * p.q_heads * (D + 2);
    const float *src = p.part + (row * p.q_heads + head) * (D + 2);
    float m = -INFINITY;
    bool missing = false;
    for (int k = 0; k < p.splits; k++) {
        m = fmaxf(m, src[k * step + D]);
        missing |= src[k * step + D + 1] < 0.0f;
    }
    if (missing) return;                                          // a CTA gave up (status word): the row stays unwritten
    const float base = m == -INFINITY ? 0.0f : m;
    float l = 0.0f, o[D / 32] = {};
    for (int k = 0; k < p.splits; k++) {
        const float f = fast_exp2(src[k * step + D] - base);
        l = fmaf(src[k * step + D + 1], f, l);
#pragma unroll
        for (int x = 0; x < D / 32; x++) o[x] = fmaf(src[k * step + lane + 32 * x], f, o[x]);
    }
#pragma unroll
    for (int x = 0; x < D / 32; x++) store_out(p, row, head, lane + 32 * x, l > 0.0f ? o[x] / l : (l == 0.0f ? 0.0f : l));
    if (lane == 0 && p.lse) p.lse[row * p.q_heads + head] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : (l == 0.0f ? -INFINITY : l);
}

}  // namespace pg
}  // namespace bd
