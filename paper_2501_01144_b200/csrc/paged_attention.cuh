// Attention of a step's queries over the paged cache, few rows per KV head (storage: paged_common.cuh).
//
//   o_i = sum_j p_ij v_j,  p_i = softmax over the visible j of  cap * tanh(scale * q_i . k_j / cap)  (or scale * q_i . k_j)
//
// with q in bf16 or fp16 as given, k and v the values the cache stands for (the rows of an unfinished value chunk in
// their source type).  Position kv - t + i sees the tokens up to itself, with a window w the last w of them.
//
// A warp takes chunks of 32 tokens one by one.  Both products run on the warp-level fp16 MMA with the cache as the
// 16-row operand and the queries (or the transposed probabilities) as the 8-column operand, so the few rows of a decode
// step fill half a tile and nothing of the cache is expanded twice.  A code becomes the fp16 number index-value * 2^-24
// (a subnormal: the half-unit integer itself in the low byte, the sign on top) without any conversion; the block's
// power-of-two scale multiplies the fp32 block sum.  bf16 queries are first scaled per row by a power of two into the
// range of fp16 (exact down to 2^-29 of the row's largest element).  Probabilities are rounded to fp16 (2^-11) for the
// second product, and their fp32 values are what the row sum adds; the unfinished chunk's values meet probabilities
// split in two bf16 parts (bf16 caches) or the same fp16 ones (fp16 caches).
// Every warp keeps its own running maximum, sum and output; the warps of a CTA are joined in shared memory, the CTAs of
// a split sequence through the workspace by a second kernel, in a fixed order.
// What bounds it: 140 bytes of cache per token and head (d = 128) against 11 integer instructions per code word and
// lane, half-rate on this machine: about 5.5 cycles of an SM's integer pipes per token and head, and 5.9 cycles of its
// share of the memory bandwidth.
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
    float *part;                      // [splits][rows][q_heads][d + 2] (split > 1): output, maximum (log2 units), sum
    float scale, softcap, unit;       // unit: factor of the partial outputs
    int q_heads, group, window, splits, row_tiles, odtype;
};

constexpr int kRowWarps = 4;
constexpr int kRowStages = 2;

__device__ __forceinline__ void expand_f16(uint32_t w, uint2 tb, uint32_t (&r)[4]) {
    const uint32_t sel = w & 0x77777777u;
    const uint32_t xa = prmt_b32(tb.x, tb.y, sel), xb = prmt_b32(tb.x, tb.y, sel >> 16);
    const uint32_t odd = w & 0x80808080u, even = (w << 4) & 0x80808080u;   // signs of the odd / even nibbles, one per byte
    r[0] = prmt_b32(xa, even, 0x5240u);   // nibbles 0, 2 = elements 0, 1
    r[1] = prmt_b32(xa, odd, 0x5341u);    // nibbles 1, 3 = elements 2, 3
    r[2] = prmt_b32(xb, even, 0x7260u);   // nibbles 4, 6 = elements 4, 5
    r[3] = prmt_b32(xb, odd, 0x7361u);    // nibbles 5, 7 = elements 6, 7
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
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
// cap * tanh(x), through exp2; xl = 2 x log2 e.  Absolute error of the tanh about 1e-7.
__device__ __forceinline__ float capped(float xl, float cap) { return cap - __fdividef(2.0f * cap, fast_exp2(xl) + 1.0f); }

// One row's result: 2^23 is what the half-unit subnormals left out (2^-24 per code, 0.5 per half unit).
__device__ __forceinline__ void store_out(const Attention &p, int64_t row, int head, int ch, float v) {
    uint8_t *o = p.o + (row * p.ldo + (int64_t)head * p.hso + ch) * (p.odtype == BD_F32 ? 4 : 2);
    if (p.odtype == BD_F32) *(float *)o = v;
    else if (p.odtype == BD_BF16) *(__nv_bfloat16 *)o = __float2bfloat16_rn(v);
    else *(__half *)o = __float2half_rn(v);
}

template <int NB, int NT>
struct RowSmem {
    static constexpr int D = 32 * NB, ROWS = 8 * NT;
    static constexpr int stage = 35 * D;
    static constexpr int ring = kRowWarps * kRowStages * stage;
    static constexpr int joined = kRowWarps * ROWS * (D + 2) * 4;      // takes the ring's place at the end
    static constexpr int body = ((ring > joined ? ring : joined) + 127) / 128 * 128;
    static constexpr int table = body, bars = table + 128, words = bars + kRowWarps * kRowStages * 8, total = words + 16;
};

template <int DT, int NB, int NT, bool CAP>
__global__ void __launch_bounds__(32 * kRowWarps) attention_rows_kernel(const __grid_constant__ Attention p) {
    using S = RowSmem<NB, NT>;
    constexpr int D = S::D, ROWS = S::ROWS;
    extern __shared__ __align__(128) uint8_t smem[];
    uint2 *table = (uint2 *)(smem + S::table);
    volatile uint32_t *flags = (volatile uint32_t *)(smem + S::words);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t4 = lane % 4;
    if (threadIdx.x < 16) table[threadIdx.x] = make_uint2(c_tables.int_lo[threadIdx.x], c_tables.int_hi[threadIdx.x]);
    if (threadIdx.x == 0) {
        flags[0] = 0; flags[1] = 1; flags[2] = tc::kSpinLimit;
        const uint32_t limit = g_debug_spin_limit;
        if (limit) flags[2] = limit;
    }
    const uint32_t bar0 = tc::smem_u32(smem + S::bars) + warp * kRowStages * 8;
    if (lane == 0)
        for (int i = 0; i < kRowStages; i++) tc::mbar_init(bar0 + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    pdl_wait();
    pdl_release();

    const int seq = blockIdx.z, h = blockIdx.y, rt = blockIdx.x % p.row_tiles, split = blockIdx.x / p.row_tiles;
    const Sequence s = sequence_of(p.batch, seq);
    if (!s.ok) {
        if (threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
        return;
    }
    const int r0 = rt * ROWS, n_rows = s.t * p.group;             // row = token * group + head of the group
    if (r0 >= n_rows) return;
    const int row_end = min(r0 + ROWS, n_rows);
    // chunks that any row of the tile sees, and this split's share of them
    const int first_pos = s.kv - s.t + r0 / p.group, last_pos = s.kv - s.t + (row_end - 1) / p.group;
    const int seen_end = max(0, last_pos + 1);
    const int seen_begin = p.window ? max(0, first_pos - p.window + 1) : 0;
    const int c_lo = seen_begin / kChunk, c_hi = (seen_end + kChunk - 1) / kChunk;
    const int per = (max(0, c_hi - c_lo) + p.splits - 1) / p.splits;
    const int c_begin = c_lo + split * per, c_end = min(c_hi, c_begin + per);
    const int full = s.kv / kChunk;                               // chunks whose values are stored in 4 bits

    // queries: fragments of the 8-column operand, in fp16
    uint32_t qf[NT][NB][4];
    float mul[NT][2];                                             // column's factor from block sums to scores
    int pos[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
        const int r = r0 + 8 * nt + g;
        const bool valid = r < n_rows;
        const uint8_t *src = p.q + ((int64_t)(s.q0 + r / p.group) * p.ldq + (int64_t)(h * p.group + r % p.group) * p.hsq) * 2;
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
            const int ex = min(max((int)(m >> 7), 27), 240);      // biased exponent of the row's largest element
            const float up = __uint_as_float((uint32_t)(127 + 14 + 127 - ex) << 23);
            qs = __uint_as_float((uint32_t)(ex - 14) << 23);
#pragma unroll
            for (int b = 0; b < NB; b++) {
                const uint32_t w[4] = {raw[b].x, raw[b].y, raw[b].z, raw[b].w};
#pragma unroll
                for (int i = 0; i < 4; i++)
                    qf[nt][b][i] = pack_f16(__uint_as_float(w[i] << 16) * up, __uint_as_float(w[i] & 0xffff0000u) * up);
            }
        } else {
#pragma unroll
            for (int b = 0; b < NB; b++) { qf[nt][b][0] = raw[b].x; qf[nt][b][1] = raw[b].y; qf[nt][b][2] = raw[b].z; qf[nt][b][3] = raw[b].w; }
        }
#pragma unroll
        for (int i = 0; i < 2; i++) {                             // this lane's columns 2 t4 + i of the score fragments
            const float f = __shfl_sync(0xffffffffu, qs, 4 * (2 * t4 + i));
            const float k = f * 8388608.0f * p.scale;
            mul[nt][i] = CAP ? k / p.softcap * (2.0f * 1.4426950408889634f) : k * 1.4426950408889634f;
            const int rc = r0 + 8 * nt + 2 * t4 + i;
            pos[nt][i] = rc < n_rows ? s.kv - s.t + rc / p.group : -1;
        }
    }
    float O[NT][NB][2][4], m_run[NT][2], l_run[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
#pragma unroll
        for (int b = 0; b < NB; b++)
#pragma unroll
            for (int i = 0; i < 8; i++) O[nt][b][i / 4][i % 4] = 0.0f;
        m_run[nt][0] = m_run[nt][1] = -INFINITY;
        l_run[nt][0] = l_run[nt][1] = 0.0f;
    }

    // the warp's chunks: c_begin + warp, + kRowWarps, ...; a record per stage
    const int mine = c_begin + warp < c_end ? (c_end - c_begin - warp + kRowWarps - 1) / kRowWarps : 0;
    uint8_t *ring = smem + warp * kRowStages * S::stage;
    uint32_t loaded = 0;                                          // bit per stage: the record is in flight or there
    auto fetch = [&](int i) {
        const int st = i % kRowStages, c = c_begin + warp + i * kRowWarps;
        const int64_t off = record_offset(p.pool, p.batch, seq, h, c);
        if (off < 0) {
            if (lane == 0) atomicOr(&g_status_word, kStatusIndex);
            loaded &= ~(1u << st);
            return;
        }
        loaded |= 1u << st;
        if (lane == 0) {
            tc::mbar_expect_tx(bar0 + 8 * st, S::stage);
            tc::bulk_load(tc::smem_u32(ring + st * S::stage), p.pool.base + off, S::stage, bar0 + 8 * st);
        }
    };
    uint32_t phase = 0;                                           // bit per stage
    for (int i = 0; i < kRowStages && i < mine; i++) fetch(i);
    for (int i = 0; i < mine; i++) {
        const int st = i % kRowStages, c = c_begin + warp + i * kRowWarps;
        const uint8_t *rec = ring + st * S::stage;
        const bool there = loaded >> st & 1u;
        if (there) {
            if (!tc::mbar_wait(bar0 + 8 * st, phase >> st & 1u, flags)) break;
            phase ^= 1u << st;
            __syncwarp();
            // ---- scores of 32 tokens ----
            float sc[NT][2][4];
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int x = 0; x < 8; x++) sc[nt][x / 4][x % 4] = 0.0f;
            uint32_t scl[4], idw[4];
            auto load_entries = [&](int64_t scales, int64_t ids) {   // per row j: NB scale bytes, NB id nibbles
                if (NB == 4) {
                    const uint4 u = *(const uint4 *)(rec + scales + 16 * g);
                    scl[0] = u.x; scl[1] = u.y; scl[2] = u.z; scl[3] = u.w;
                    const uint2 v = *(const uint2 *)(rec + ids + 8 * g);
                    idw[0] = v.x; idw[1] = v.x >> 16; idw[2] = v.y; idw[3] = v.y >> 16;
                } else {
                    const uint2 u = *(const uint2 *)(rec + scales + 8 * g);
                    scl[0] = u.x; scl[1] = u.x >> 16; scl[2] = u.y; scl[3] = u.y >> 16;
                    const uint32_t v = *(const uint32_t *)(rec + ids + 4 * g);
                    idw[0] = v; idw[1] = v >> 8; idw[2] = v >> 16; idw[3] = v >> 24;
                }
            };
            load_entries(key_scales(D), key_ids(D));
#pragma unroll
            for (int b = 0; b < NB; b++) {
                const uint4 w4 = *(const uint4 *)(rec + b * 512 + lane * 16);
                const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
                uint32_t a[4][4];
                float f[4];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    expand_f16(w[j], table[idw[j] >> (4 * b) & 15u], a[j]);
                    f[j] = __uint_as_float((scl[j] >> (8 * b) & 255u) << 23);     // 2^e (scale byte 0: nothing but zeros or 2^-127)
                }
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        mma_f16(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], qf[nt][b][0], qf[nt][b][1]);
                        mma_f16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], qf[nt][b][2], qf[nt][b][3]);
                        sc[nt][x][0] = fmaf(acc[0], f[2 * x], sc[nt][x][0]);
                        sc[nt][x][1] = fmaf(acc[1], f[2 * x], sc[nt][x][1]);
                        sc[nt][x][2] = fmaf(acc[2], f[2 * x + 1], sc[nt][x][2]);
                        sc[nt][x][3] = fmaf(acc[3], f[2 * x + 1], sc[nt][x][3]);
                    }
            }
            // ---- softmax: rows of the fragment are tokens (row 8 j + g = token 8 (g / 2) + 2 j + g % 2), columns queries ----
            const int tok0 = c * kChunk + 8 * (g / 2) + g % 2;
            const bool masked = (c + 1) * kChunk > first_pos + 1 || (p.window && c * kChunk <= last_pos - p.window);
            uint32_t pf[NT][4];
            float alpha[NT][2];
            bool grew = false;
            float pv[NT][4][2];
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    float x[4], top = -INFINITY;
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        x[j] = sc[nt][j / 2][2 * (j % 2) + i] * mul[nt][i];
                        if (CAP) x[j] = capped(x[j], p.softcap * 1.4426950408889634f);
                        if (masked) {
                            const int tok = tok0 + 2 * j;
                            if (tok > pos[nt][i] || (p.window && tok <= pos[nt][i] - p.window)) x[j] = -INFINITY;
                        }
                        top = fmaxf(top, x[j]);
                    }
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                    const float m_new = fmaxf(m_run[nt][i], top);
                    const float base = m_new == -INFINITY ? 0.0f : m_new;
                    alpha[nt][i] = fast_exp2(m_run[nt][i] - base);
                    grew |= m_new > m_run[nt][i];
                    m_run[nt][i] = m_new;
                    float sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        pv[nt][j][i] = fast_exp2(x[j] - base);
                        sum += pv[nt][j][i];
                    }
                    l_run[nt][i] = fmaf(l_run[nt][i], alpha[nt][i], sum);
                }
            if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int b = 0; b < NB; b++)
#pragma unroll
                        for (int x = 0; x < 8; x++) O[nt][b][x / 4][x % 4] *= alpha[nt][x % 2];
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
                    float f[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        expand_f16(w[j], table[idw[j] >> (4 * b) & 15u], a[j]);
                        f[j] = __uint_as_float((scl[j] >> (8 * b) & 255u) << 23);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int x = 0; x < 2; x++) {
                            float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                            mma_f16(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], pf[nt][0], pf[nt][1]);
                            mma_f16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], pf[nt][2], pf[nt][3]);
                            O[nt][b][x][0] = fmaf(acc[0], f[2 * x], O[nt][b][x][0]);
                            O[nt][b][x][1] = fmaf(acc[1], f[2 * x], O[nt][b][x][1]);
                            O[nt][b][x][2] = fmaf(acc[2], f[2 * x + 1], O[nt][b][x][2]);
                            O[nt][b][x][3] = fmaf(acc[3], f[2 * x + 1], O[nt][b][x][3]);
                        }
                }
            } else {
                // ---- the unfinished chunk: rows of the tail; tokens behind the last one count as zeros ----
                uint32_t lo[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float a = pv[nt][j][0], b = pv[nt][j][1];
                        if (DT == BD_BF16) {
                            const uint32_t hi = pack_bf16(a, b);
                            pf[nt][j] = transpose8x8(hi);
                            lo[nt][j] = transpose8x8(pack_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u)));
                        } else {
                            pf[nt][j] = transpose8x8(pack_f16(a, b));
                        }
                    }
                const int slot = p.batch.slot[seq];
                const bool slot_ok = slot >= 0 && slot < p.pool.slots;
                if (!slot_ok && lane == 0) atomicOr(&g_status_word, kStatusIndex);
                const uint16_t *tail = (const uint16_t *)p.pool.tail + tail_offset(p.pool, slot_ok ? slot : 0, h, c * kChunk);
                const int left = slot_ok ? s.kv - c * kChunk : 0;
#pragma unroll 1
                for (int b = 0; b < NB; b++) {
                    uint32_t a[4][4];
#pragma unroll
                    for (int j = 0; j < 4; j++)
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            const int tok = 8 * t4 + 2 * e, ch = 32 * b + 8 * j + g;
                            const uint32_t x = tok < left ? tail[tok * D + ch] : 0u, y = tok + 1 < left ? tail[(tok + 1) * D + ch] : 0u;
                            a[j][e] = x | y << 16;
                        }
                    float add[NT][2][4];
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int x = 0; x < 2; x++) {
                            float (&acc)[4] = add[nt][x];
                            acc[0] = acc[1] = acc[2] = acc[3] = 0.0f;
                            if (DT == BD_BF16) {
                                mma_bf16(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], pf[nt][0], pf[nt][1]);
                                mma_bf16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], pf[nt][2], pf[nt][3]);
                                mma_bf16(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], lo[nt][0], lo[nt][1]);
                                mma_bf16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], lo[nt][2], lo[nt][3]);
                            } else {
                                mma_f16(acc, a[2 * x][0], a[2 * x + 1][0], a[2 * x][1], a[2 * x + 1][1], pf[nt][0], pf[nt][1]);
                                mma_f16(acc, a[2 * x][2], a[2 * x + 1][2], a[2 * x][3], a[2 * x + 1][3], pf[nt][2], pf[nt][3]);
                            }
                        }
#pragma unroll
                    for (int bb = 0; bb < NB; bb++)              // (b is a run-time index here: registers are picked by comparison)
                        if (bb == b)
#pragma unroll
                            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                                for (int x = 0; x < 8; x++) O[nt][bb][x / 4][x % 4] = fmaf(add[nt][x / 4][x % 4], 1.0f / 8388608.0f, O[nt][bb][x / 4][x % 4]);
                }
            }
        }
        __syncwarp();                                             // every lane is done with the stage
        if (i + kRowStages < mine) fetch(i + kRowStages);
    }
    // ---- join the warps ----
    __syncthreads();
    if (flags[0]) return;                                         // a wait ran out (status word): nothing is written
    float *jo = (float *)smem, *jm = jo + kRowWarps * ROWS * D, *jl = jm + kRowWarps * ROWS;
#pragma unroll
    for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int i = 0; i < 2; i++) {
            float l = l_run[nt][i];
            l += __shfl_xor_sync(0xffffffffu, l, 4);
            l += __shfl_xor_sync(0xffffffffu, l, 8);
            l += __shfl_xor_sync(0xffffffffu, l, 16);
            const int r = warp * ROWS + 8 * nt + 2 * t4 + i;
            if (g == 0) { jm[r] = m_run[nt][i]; jl[r] = l; }
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
                for (int j = 0; j < 4; j++) jo[r * D + 32 * b + 8 * j + g] = O[nt][b][j / 2][2 * (j % 2) + i];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < (row_end - r0) * D; i += blockDim.x) {
        const int r = i / D, ch = i % D;
        float m = -INFINITY, l = 0.0f, o = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowWarps; w++) m = fmaxf(m, jm[w * ROWS + r]);
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int w = 0; w < kRowWarps; w++) {
            const float f = fast_exp2(jm[w * ROWS + r] - base);
            l = fmaf(jl[w * ROWS + r], f, l);
            o = fmaf(jo[(w * ROWS + r) * D + ch], f, o);
        }
        const int64_t row = s.q0 + (r0 + r) / p.group;
        const int head = h * p.group + (r0 + r) % p.group;
        if (p.splits == 1) {
            store_out(p, row, head, ch, l > 0.0f ? o * (8388608.0f / l) : (l == 0.0f ? 0.0f : l));
            if (ch == 0 && p.lse) p.lse[row * p.q_heads + head] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : (l == 0.0f ? -INFINITY : l);
        } else {
            float *to = p.part + (((int64_t)split * p.batch.rows + row) * p.q_heads + head) * (D + 2);
            to[ch] = o;
            if (ch == 0) { to[D] = m; to[D + 1] = l; }
        }
    }
}

// Joins the splits of a row, in split order.  A warp per row and head.
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
    for (int k = 0; k < p.splits; k++) m = fmaxf(m, src[k * step + D]);
    const float base = m == -INFINITY ? 0.0f : m;
    float l = 0.0f, o[D / 32] = {};
    for (int k = 0; k < p.splits; k++) {
        const float f = fast_exp2(src[k * step + D] - base);
        l = fmaf(src[k * step + D + 1], f, l);
#pragma unroll
        for (int x = 0; x < D / 32; x++) o[x] = fmaf(src[k * step + lane + 32 * x], f, o[x]);
    }
#pragma unroll
    for (int x = 0; x < D / 32; x++) store_out(p, row, head, lane + 32 * x, l > 0.0f ? o[x] * (p.unit / l) : (l == 0.0f ? 0.0f : l));
    if (lane == 0 && p.lse) p.lse[row * p.q_heads + head] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : (l == 0.0f ? -INFINITY : l);
}

}  // namespace pg
}  // namespace bd
