// Attention of a chunk of new tokens over the paged cache on the tcgen05 tensor cores (formula: paged_attention.cuh).
//
// A CTA takes 256 rows (row = token * group + head of the group) of one KV head as two tiles of 128 and walks over the
// visible tokens in tiles of 128:
//   S_t = Q_t K^T      both operands in shared memory, S in tensor memory (128 lanes x 128 fp32 columns);
//   P_t = exp2(S_t - m) written back over S_t as 16-bit pairs;
//   O_t += P_t V       P_t as the A operand in tensor memory, V^T (channels x tokens) in shared memory.
// Warps: two groups of four run the softmax of a tile each (thread = row, so no exchange between threads), four expand
// the cache, one issues the MMAs: while one tile's softmax runs, the tensor pipe works on the other tile.  The output
// stays in tensor memory and is rescaled only when a row's maximum has grown by more than 2^8 since the last time
// (probabilities up to 2^8, 2^15 in fp16, do no harm in 16 bits with fp32 sums).
// Expansion: a thread owns a block (row of a key or value tile).  Its dialect's eight magnitudes as 16-bit floats of
// the block's scale are two eight-byte tables, low and high bytes, read from shared memory with the scale added to the
// exponent bits; a code word becomes eight values with byte permutes alone.  Keys keep the record's row order in the
// tile, which only permutes the columns of S; P is written in token order.
// P is rounded to the cache's type (8 or 11 bits): the MMA takes both operands of one type.
// When many CTAs read the same tokens (IMAGES), a kernel in front expands every tile once into the workspace, in the layout it
// has in shared memory, and one thread copies the tiles with bulk copies: the softmax then has the SM's issue slots for itself.
// 4096 new of 16384 tokens, 32 / 8 heads x 128: 880 us a call = 1090 TFLOP/s (817 back to back before the power cap lowers the clock, 866
// after).  The tensor pipe and the exponential unit would each need 2048 cycles per pair of tiles; a pair takes about 3500, the softmax of
// one tile about 1700 of them and then a wait for its products.
// All waits are bounded; a wait that runs out raises the abort word, every role waits for what it has in flight, and the CTA's rows
// that are not finished stay unwritten (of a shared tile all rows: the join kernel is told).
#pragma once
#include <type_traits>

#include "gemm_tc.cuh"
#include "paged_attention.cuh"

namespace bd {
namespace pg {

constexpr int kChunkThreads = 512;            // launched with 128 registers a thread = 4 warpgroups x 128; split 184 + 184 + 96 + 48, or 208 + 208 + 48 + 48
constexpr int kTileTokens = 128;

template <int NB>
struct ChunkSmem {
    static constexpr int D = 32 * NB;
    static constexpr int q_tile = 128 * D * 2, kv_tile = 128 * D * 2;
    static constexpr int q = 0, k = q + 2 * q_tile, v = k + 2 * kv_tile, table = v + 2 * kv_tile, bars = table + 512, words = bars + 128, flags = words + 64,
                         total = flags + 64 + 1024;              // + slack for 1024-byte alignment
};

__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tcgen05_st_x16(uint32_t taddr, const uint32_t *r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// Two fp32 lanes of a 64-bit register: a * b + c.
__device__ __forceinline__ void fma2(float &x, float &y, float b, float c) {
    asm("{\n\t.reg .b64 u, v, w;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %2};\n\tmov.b64 w, {%3, %3};\n\tfma.rn.f32x2 u, u, v, w;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(x), "+f"(y) : "f"(b), "f"(c));
}
__device__ __forceinline__ void add2(float &x, float &y, float a, float b) {
    asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tadd.rn.f32x2 u, u, v;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}

// 16-byte piece `piece` (of 16-bit elements 8 piece ..) of row `row` in a K-major tile of `rows` rows: halves of 64
// elements, 128-byte rows, 128-byte swizzle.
__device__ __forceinline__ uint32_t swizzled(int rows, int row, int piece) {
    return (uint32_t)(piece >> 3) * (uint32_t)(rows * 128) + (uint32_t)(row * 128) + (uint32_t)(((piece & 7) ^ (row & 7)) * 16);
}

// One operand (keys or values) of one record in a lane's registers: the block of each tile b in row `lane`.
template <int NB>
struct Lane {
    uint32_t w[NB][4];
    uint32_t scales, ids;
};

// A tile's values of the chunk that is not in 4 bits: rows of the tail as columns (`left` of them, zeros behind).
template <int NB>
__device__ __forceinline__ void tail_columns(const uint16_t *src, int left, uint8_t *vt, int e, int lane) {
    constexpr int D = 32 * NB;
#pragma unroll 1
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int k = 8 * q + 2 * i;
                const uint32_t x = k < left ? src[k * D + 32 * b + lane] : 0u, y = k + 1 < left ? src[(k + 1) * D + 32 * b + lane] : 0u;
                w[i] = x | y << 16;
            }
            *(uint4 *)(vt + swizzled(D, 32 * b + lane, 4 * e + q)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
}
template <int NB>
__device__ __forceinline__ void load_lane(const Pool &pool, int64_t off, bool values, int lane, Lane<NB> &x) {
    constexpr int D = 32 * NB;
    const int entry = entry_of(NB, 0, lane);
    const uint8_t *rec = pool.base + off;
    const uint8_t *codes = rec + (values ? value_codes(D) : 0), *sc = rec + (values ? value_scales(D) : key_scales(D)) + entry,
                  *id = rec + (values ? value_ids(D) : key_ids(D)) + entry / 2;
    x.scales = NB == 4 ? *(const uint32_t *)sc : *(const uint16_t *)sc;
    x.ids = NB == 4 ? *(const uint16_t *)id : *id;
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int t = 0; t < 4; t++) x.w[b][t] = *(const uint32_t *)(codes + word_byte(b, lane, t));
}
// Chunk e of a tile from a lane's registers: keys in rows 32 e + lane, values (columns 32 e ..) in rows 32 b + lane.  The tables of
// all the lane's blocks come first, and whether one of them has to be built value by value (fp16 subnormals) is asked once:
// a branch at each block kept the blocks' latencies apart.  128 new of 4096 tokens, 4 x 32 heads x 128 fp16: 93 us with the branches,
// 86 without them, 76 with the page numbers looked up a tile early as well (bf16, which had no branches: 87 -> 74 us).
template <int DT, int NB>
__device__ __forceinline__ void expand_lane(const uint4 *table, const Lane<NB> &x, bool values, uint8_t *tile, int e, int lane) {
    constexpr int D = 32 * NB;
    auto blocks = [&](auto low) {
        uint4 t[NB];
#pragma unroll
        for (int b = 0; b < NB; b++) t[b] = block_table<DT, false, decltype(low)::value>(table, x.ids >> (4 * b) & 15u, x.scales >> (8 * b) & 255u);
#pragma unroll
        for (int b = 0; b < NB; b++)
#pragma unroll
            for (int q = 0; q < 4; q++)
                *(uint4 *)(tile + (values ? swizzled(D, 32 * b + lane, 4 * e + q) : swizzled(128, 32 * e + lane, 4 * b + q))) = expand_word(x.w[b][q], t[b]);
    };
    bool low = false;
#pragma unroll
    for (int b = 0; b < NB; b++) low |= (x.scales >> (8 * b) & 255u) < kF16Normal;
    if (DT == BD_F16 && low) blocks(std::true_type{});
    else blocks(std::false_type{});
}

// Expanded tiles: per sequence, KV head and tile of 128 tokens the key image and the value image, and a word that says which
// of its four chunks have a page.
__device__ __forceinline__ int64_t image_index(const Attention &p, int seq, int h, int tile) { return ((int64_t)seq * p.pool.kv_heads + h) * p.image_tiles + tile; }

template <int DT, int NB>
__global__ void __launch_bounds__(256) expand_kernel(const __grid_constant__ Attention p) {
    constexpr int D = 32 * NB, kImage = 128 * D * 2;
    __shared__ uint4 table[32];
    make_base_tables<DT>(table);
    pdl_wait();
    pdl_release();
    __syncthreads();
    const int tile = blockIdx.x, h = blockIdx.y, seq = blockIdx.z, warp = threadIdx.x / 32, e = warp % 4, lane = threadIdx.x % 32;
    const bool values = warp >= 4;
    const Sequence s = sequence_of(p.batch, seq);
    if (!s.ok || s.t == 0) return;
    if (tile * kTileTokens >= s.kv || (p.window && (tile + 1) * kTileTokens <= s.kv - s.t - p.window + 1)) return;   // nobody sees it
    const int c = 4 * tile + e, full = s.kv / kChunk, n_chunks = (s.kv + kChunk - 1) / kChunk;
    const bool seen = c < n_chunks && c >= (p.window ? max(0, s.kv - s.t - p.window + 1) / kChunk : 0);   // pages in front of the window are not looked up
    const int64_t off = seen ? record_offset(p.pool, p.batch, seq, h, c) : -1, at = image_index(p, seq, h, tile);
    uint8_t *image = p.images + at * (2 * kImage) + (values ? kImage : 0);
    if (off < 0 && seen && lane == 0) atomicOr(&g_status_word, kStatusIndex);
    __shared__ uint32_t ok;
    if (threadIdx.x == 0) ok = 0;
    __syncthreads();
    if (!values && off >= 0 && lane == 0) atomicOr(&ok, 1u << e);
    if (off >= 0 && (!values || c < full)) {
        Lane<NB> x;
        load_lane<NB>(p.pool, off, values, lane, x);
        expand_lane<DT, NB>(table, x, values, image, e, lane);
    } else if (values) {
        const int slot = p.batch.slot[seq];
        const bool tail = c == full && c < n_chunks && off >= 0, slot_ok = slot >= 0 && slot < p.pool.slots;
        if (tail && !slot_ok && lane == 0) atomicOr(&g_status_word, kStatusIndex);
        const int left = tail && slot_ok ? s.kv - c * kChunk : 0;
        tail_columns<NB>((const uint16_t *)p.pool.tail + tail_offset(p.pool, left ? slot : 0, h, c * kChunk), left, image, e, lane);
    }
    __syncthreads();
    if (threadIdx.x == 0) p.image_ok[at] = ok;
}

template <int DT, int NB, bool CAP, bool IMAGES>
__global__ void __launch_bounds__(kChunkThreads, 1) attention_chunk_kernel(const __grid_constant__ Attention p) {
    using S = ChunkSmem<NB>;
    constexpr int D = S::D;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *const sm = smem_raw + (base - tc::smem_u32(smem_raw));
    const uint32_t bars = base + S::bars;
    const uint32_t q_full = bars, s_full = bars + 8, p_full = bars + 24, k_full = bars + 40, k_empty = bars + 56, v_full = bars + 72, v_empty = bars + 88, p_half = bars + 104, drained = bars + 120;
    volatile uint32_t *const words = (volatile uint32_t *)(sm + S::words), *const abort_flag = words + 1;
    volatile uint32_t *const chunk_ok = (volatile uint32_t *)(sm + S::flags);       // [8 tiles]: bit e = chunk e of the tile has a page
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, wg = warp / 4;

    make_base_tables<DT>((uint4 *)(sm + S::table));
    if (threadIdx.x < 8) chunk_ok[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        abort_flag[0] = 0;
        abort_flag[1] = 1;
        abort_flag[2] = g_debug_spin_limit ? g_debug_spin_limit : tc::kSpinLimit;
        abort_flag[4] = 0;                                        // the final wait's own words
        abort_flag[5] = 1;
        abort_flag[6] = tc::kSpinLimit;
        tc::mbar_init(q_full, 8);
        tc::mbar_init(drained, 1);
        for (int i = 0; i < 2; i++) {
            tc::mbar_init(s_full + 8 * i, 1);
            tc::mbar_init(p_full + 8 * i, 4);
            tc::mbar_init(p_half + 8 * i, 4);
            tc::mbar_init(k_full + 8 * i, (IMAGES ? 1 : 4) + (i + blockIdx.x == 0 && g_debug_skip_first_code_stage ? 1 : 0));
            tc::mbar_init(k_empty + 8 * i, 1);
            tc::mbar_init(v_full + 8 * i, IMAGES ? 1 : 4);
            tc::mbar_init(v_empty + 8 * i, 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();                                                   // (before the first decision that depends on the batch's numbers)
    pdl_release();

    // Which rows: the items (sequence, tile of 256 rows) in the order of their work, heaviest first, all heads of one behind
    // each other: CTAs start in this order, so the light ones fill up what the heavy ones leave (six ragged chunks, 32 heads x 64:
    // 92 -> 84 us).  More items than the CTA has threads: as they are numbered, tiles from the last.
    const int heads = p.pool.kv_heads * p.splits, items = p.row_tiles * p.batch.n;
    int item = (int)(blockIdx.x / (uint32_t)heads);
    if (items <= kChunkThreads && items > 1) {
        int *weight = (int *)(sm + S::q);                         // (the queries come later)
        int mine = 0;
        if ((int)threadIdx.x < items) {
            const Sequence q = sequence_of(p.batch, threadIdx.x / p.row_tiles);
            const int first = (int)(threadIdx.x % p.row_tiles) * 256, rows = q.t * p.group;
            if (q.ok && first < rows) {
                const int last = q.kv - q.t + p.token(min(first + 256, rows) - 1), from = p.window ? max(0, q.kv - q.t + p.token(first) - p.window + 1) : 0;
                mine = max(0, last + 1 - from) + 1;
            }
            weight[threadIdx.x] = mine;
        }
        __syncthreads();
        if ((int)threadIdx.x < items) {
            int rank = 0;
            for (int i = 0; i < items; i++) rank += weight[i] > mine || (weight[i] == mine && i < (int)threadIdx.x);
            if (rank == item) words[8] = threadIdx.x;
        }
        __syncthreads();
        item = (int)words[8];
    } else {
        item = item / p.row_tiles * p.row_tiles + p.row_tiles - 1 - item % p.row_tiles;
    }
    const int seq = item / p.row_tiles, pair = item % p.row_tiles, h = (int)(blockIdx.x % (uint32_t)heads) / p.splits, split = (int)blockIdx.x % p.splits;
    const Sequence s = sequence_of(p.batch, seq);
    if (!s.ok) {
        if (threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
        return;
    }
    const int r0 = pair * 256, n_rows = s.t * p.group;
    if (r0 >= n_rows) return;
    const int row_end = min(r0 + 256, n_rows), n_q = row_end - r0 > 128 ? 2 : 1;
    const int first_pos = s.kv - s.t + p.token(r0), last_pos = s.kv - s.t + p.token(row_end - 1);
    const int seen_end = max(0, last_pos + 1), seen_begin = p.window ? max(0, first_pos - p.window + 1) : 0;
    const int t_lo = seen_begin / kTileTokens, t_hi = (seen_end + kTileTokens - 1) / kTileTokens;
    const int per = (max(0, t_hi - t_lo) + p.splits - 1) / p.splits;
    const int t_begin = t_lo + split * per, n_tiles = max(0, min(t_hi, t_begin + per) - t_begin);

    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32((const void *)words)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc::tcgen05_fence_before();
    __syncthreads();
    tc::tcgen05_fence_after();
    const uint32_t tmem = *words;
    // tensor memory: S_0, S_1 at columns 0, 128 (P over their first halves), O_0, O_1 at 256, 384
    constexpr uint32_t kFmt = DT == BD_BF16 ? 1u : 0u;
    // what the reference of a row's exponentials lies below its maximum when it moves: fp16 subnormals then lose 2^-32 of the row's largest
    // probability (see RowWork::chunk); bf16 has fp32's exponents
    constexpr float kAbove = DT == BD_BF16 ? 0.0f : kPeak;

    if (wg < 2) {
        if (IMAGES) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
        // ---- softmax of tile wg; thread = row = tensor-memory lane ----
        const int quad = warp % 4, row = 128 * wg + 32 * quad + lane, r = r0 + row;
        {                                                         // queries of this tile into shared memory
            const uint32_t flip = p.scale < 0.0f ? 0x80008000u : 0u;
            constexpr int kPieces = D / 8;
            const int tid = threadIdx.x % 128;
#pragma unroll 4
            for (int i = tid; i < 128 * kPieces; i += 128) {
                const int qr = i / kPieces, piece = i % kPieces, rr = r0 + 128 * wg + qr;
                uint4 x = make_uint4(0, 0, 0, 0);
                if (rr < n_rows) {
                    x = *(const uint4 *)(p.q + ((int64_t)(s.q0 + p.token(rr)) * p.ldq + (int64_t)(h * p.group + (rr - p.token(rr) * p.group)) * p.hsq + 8 * piece) * 2);
                    x.x ^= flip; x.y ^= flip; x.z ^= flip; x.w ^= flip;
                }
                *(uint4 *)(sm + S::q + wg * S::q_tile + swizzled(128, qr, piece)) = x;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) tc::mbar_arrive_local(q_full);
        }
        if (wg < n_q) {
            const int pos = r < n_rows ? s.kv - s.t + p.token(r) : -1;
            const float mul = fmaxf(fabsf(p.scale), 1.4e-45f) * 1.4426950408889634f;     // (the smallest number for zero: masked scores stay -inf)
            const uint32_t t_s = tmem + 128u * wg + ((uint32_t)(32 * quad) << 16), t_o = tmem + 256u + 128u * wg + ((uint32_t)(32 * quad) << 16);
            // positions of the warp's 32 rows: the tiles that need a mask
            const int w_first = s.kv - s.t + p.token(r0 + 128 * wg + 32 * quad);
            const int w_last = s.kv - s.t + p.token(min(r0 + 128 * wg + 32 * quad + 31, n_rows - 1));
            float m = -INFINITY, l = 0.0f;
            bool alive = true;
            for (int j = 0; j < n_tiles && alive; j++) {
                alive = tc::mbar_wait_warp(s_full + 8 * wg, j & 1, abort_flag, 0);
                if (!alive) break;
                tc::tcgen05_fence_after();
                if (CAP) {
                    // 32 columns a turn, back into tensor memory: with all 128 in registers at once 176 us (spills) instead of 156 for 4 x 256
                    // new of 4096 tokens, 32 / 8 heads x 128; without a cap 86
#pragma unroll 1
                    for (int c = 0; c < 4; c++) {
                        uint32_t z[32];
                        tc::tcgen05_ld_32x32b_x32(t_s + 32 * c, z);
                        tc::tcgen05_wait_ld();
#pragma unroll
                        for (int n = 0; n < 32; n += 2) {
                            float a, b;
                            unpair(cap_pair(mul_pair(pair_of(__uint_as_float(z[n]), __uint_as_float(z[n + 1])), pair_of(mul)), p.cap_inv, p.cap), a, b);
                            z[n] = __float_as_uint(a);
                            z[n + 1] = __float_as_uint(b);
                        }
                        tcgen05_st_x16(t_s + 32 * c, z);
                        tcgen05_st_x16(t_s + 32 * c + 16, z + 16);
                    }
                    tc::tcgen05_wait_st();
                }
                uint32_t x[4][32];
#pragma unroll
                for (int c = 0; c < 4; c++) tc::tcgen05_ld_32x32b_x32(t_s + 32 * c, x[c]);
                tc::tcgen05_wait_ld();
                const int tok0 = (t_begin + j) * kTileTokens;
                const uint32_t there = chunk_ok[j & 7];
                if (tok0 + kTileTokens - 1 > w_first || w_first < 0 || (p.window && tok0 <= w_last - p.window) || there != 15u) {
                    const int hi = pos - tok0, lo = p.window ? pos - p.window - tok0 : -1;
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        const bool ok = there >> c & 1u;
#pragma unroll
                        for (int n = 0; n < 32; n++) {
                            const int tok = 32 * c + key_token(n);
                            if (tok > hi || tok <= lo || !ok) x[c][n] = 0xff800000u;
                        }
                    }
                }
                // The exponentials of the first half start from the maximum of the tiles before; under them the tile's own
                // maximum is found, and only if a row's has grown by more than 2^8 are they done again (and O rescaled).
                const float k = CAP ? 1.0f : mul;
                float l0 = 0.0f, l1 = 0.0f;
                uint32_t out[2][16];
                auto exponentials = [&](int c, float sub, uint32_t (&to)[16]) {
#pragma unroll
                    for (int n = 0; n < 32; n += 2) {
                        float a = __uint_as_float(x[c][n]), b = __uint_as_float(x[c][n + 1]);
                        fma2(a, b, k, sub);
                        a = fast_exp2(a);
                        b = fast_exp2(b);
                        add2(l0, l1, a, b);
                        // columns n, n + 1 are tokens 8 x + 2 y + {0, 1} with n = 8 y + 2 x: pair 4 x + y in token order
                        to[4 * (n % 8 / 2) + n / 8] = DT == BD_BF16 ? pack_bf16(a, b) : pack_f16(a, b);
                    }
                };
                float sub = m == -INFINITY ? 0.0f : -m;
                exponentials(0, sub, out[0]);
                exponentials(1, sub, out[1]);
                float top[4];
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    top[c] = __uint_as_float(x[c][0]);
#pragma unroll
                    for (int n = 1; n < 32; n++) top[c] = fmaxf(top[c], __uint_as_float(x[c][n]));
                }
                const float m_new = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * k;       // (k > 0)
                const bool grew = m_new > m + (kAbove + 8.0f);    // m = -inf: the first visible token; m_new = -inf: none
                if (__any_sync(0xffffffffu, grew)) {
                    const float alpha = grew ? fast_exp2(m - (m_new - kAbove)) : 1.0f;
                    if (grew) m = m_new - kAbove;
                    l *= alpha;
                    if (j > 0) {                                  // S(j) complete implies that the products up to j - 1 are
#pragma unroll 1
                        for (int c = 0; c < D / 16; c++) {
                            uint32_t o[16];
                            tc::tcgen05_ld_32x32b_x16(t_o + 16 * c, o);
                            tc::tcgen05_wait_ld();
#pragma unroll
                            for (int n = 0; n < 16; n++) o[n] = __float_as_uint(__uint_as_float(o[n]) * alpha);
                            tcgen05_st_x16(t_o + 16 * c, o);
                        }
                    }
                    sub = m == -INFINITY ? 0.0f : -m;
                    l0 = l1 = 0.0f;
                    exponentials(0, sub, out[0]);
                    exponentials(1, sub, out[1]);
                }
#pragma unroll
                for (int half = 0; half < 2; half++) {
                    if (half) {
                        exponentials(2, sub, out[0]);
                        exponentials(3, sub, out[1]);
                    }
                    tcgen05_st_x16(t_s + 32 * half, out[0]);
                    tcgen05_st_x16(t_s + 32 * half + 16, out[1]);
                    tc::tcgen05_wait_st();
                    tc::tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive_local((half ? p_full : p_half) + 8 * wg);
                }
                l += l0 + l1;
            }
            // ---- the tile's result ----
            if (n_tiles > 0 && alive) alive = tc::mbar_wait_warp(s_full + 8 * wg, n_tiles & 1, abort_flag);
            tc::tcgen05_fence_after();
            if (alive) {
                const int64_t out_row = s.q0 + p.token(r);
                const int head = h * p.group + (r - p.token(r) * p.group);
                const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
                float *part = p.splits > 1 ? p.part + (((int64_t)split * p.batch.rows + out_row) * p.q_heads + head) * (D + 2) : nullptr;
#pragma unroll
                for (int c = 0; c < D / 32; c++) {
                    uint32_t o[32];
                    if (n_tiles > 0) {
                        tc::tcgen05_ld_32x32b_x32(t_o + 32 * c, o);
                        tc::tcgen05_wait_ld();
                    } else {
#pragma unroll
                        for (int n = 0; n < 32; n++) o[n] = 0u;
                    }
                    if (r < row_end) {
                        if (p.splits > 1) {
#pragma unroll
                            for (int n = 0; n < 32; n += 2) *(float2 *)(part + 32 * c + n) = make_float2(__uint_as_float(o[n]), __uint_as_float(o[n + 1]));
                        } else if (p.odtype == BD_F32) {
                            float *to = (float *)p.o + out_row * p.ldo + (int64_t)head * p.hso + 32 * c;
#pragma unroll
                            for (int n = 0; n < 32; n += 4)
                                *(float4 *)(to + n) = make_float4(__uint_as_float(o[n]) * inv, __uint_as_float(o[n + 1]) * inv, __uint_as_float(o[n + 2]) * inv, __uint_as_float(o[n + 3]) * inv);
                        } else {
                            uint16_t *to = (uint16_t *)p.o + out_row * p.ldo + (int64_t)head * p.hso + 32 * c;
#pragma unroll
                            for (int n = 0; n < 32; n += 8) {
                                uint32_t w[4];
#pragma unroll
                                for (int i = 0; i < 4; i++) {
                                    const float a = __uint_as_float(o[n + 2 * i]) * inv, b = __uint_as_float(o[n + 2 * i + 1]) * inv;
                                    w[i] = DT == BD_BF16 ? pack_bf16(a, b) : pack_f16(a, b);
                                }
                                *(uint4 *)(to + n) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        }
                    }
                }
                if (r < row_end) {
                    if (p.splits > 1) { part[D] = m; part[D + 1] = l; }
                    else if (p.lse) p.lse[out_row * p.q_heads + head] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : (l == 0.0f ? -INFINITY : l);
                }
            } else if (p.splits > 1 && r < row_end) {
                p.part[(((int64_t)split * p.batch.rows + s.q0 + p.token(r)) * p.q_heads + h * p.group + (r - p.token(r) * p.group)) * (D + 2) + D + 1] = -1.0f;
            }
        }
    } else if (wg == 2) {
        if (IMAGES) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
        const int e = warp % 4, full = s.kv / kChunk, n_chunks = (s.kv + kChunk - 1) / kChunk;
        bool alive = true;
        if (IMAGES) {
            // ---- bulk copies of the expanded tiles, by one thread ----
            if (e == 0 && lane == 0) {
                const uint8_t *src = p.images + image_index(p, seq, h, t_begin) * (2 * S::kv_tile);
                const uint32_t *ok = p.image_ok + image_index(p, seq, h, t_begin);
                int keys = 0, values = 0;                         // copies begun
                for (int j = 0; j < n_tiles && alive; j++, src += 2 * S::kv_tile) {
                    const int st = j & 1;
                    const uint32_t parity = (uint32_t)(j >> 1 & 1) ^ 1u;
                    const uint32_t there = ok[j];
                    alive = tc::mbar_wait(k_empty + 8 * st, parity, abort_flag);
                    if (!alive) break;
                    chunk_ok[j & 7] = there;
                    tc::mbar_expect_tx(k_full + 8 * st, S::kv_tile);
                    tc::bulk_load(base + S::k + st * S::kv_tile, src, S::kv_tile, k_full + 8 * st);
                    keys++;
                    alive = tc::mbar_wait(v_empty + 8 * st, parity, abort_flag);
                    if (!alive) break;
                    tc::mbar_expect_tx(v_full + 8 * st, S::kv_tile);
                    tc::bulk_load(base + S::v + st * S::kv_tile, src + S::kv_tile, S::kv_tile, v_full + 8 * st);
                    values++;
                }
                // the last copies into each stage have arrived before the CTA ends, also when nobody takes them any more
                for (int j = max(0, keys - 2); j < keys; j++) tc::mbar_drain(k_full + 8 * (j & 1), j >> 1 & 1);
                for (int j = max(0, values - 2); j < values; j++) tc::mbar_drain(v_full + 8 * (j & 1), j >> 1 & 1);
            }
            __syncwarp();
        } else {
        // ---- expansion: warp e takes chunk e of every tile; lane = row of the record's tiles ----
        const uint4 *table = (const uint4 *)(sm + S::table);
        const int first_seen = seen_begin / kChunk;
        // page numbers are looked up two tiles ahead, records fetched one ahead
        auto look_up = [&](int j) -> int {
            const int c = 4 * (t_begin + j) + e;
            return j < n_tiles && c < n_chunks && c >= first_seen ? p.batch.table[(int64_t)seq * p.batch.ld_table + (int)fast_div(c, p.by_page)] : -1;
        };
        auto place = [&](int j, int page) -> int64_t {            // the chunk's record, -1: none (pages in front of the window may be gone: not looked up)
            const int c = 4 * (t_begin + j) + e;
            if (j >= n_tiles || c >= n_chunks || c < first_seen) return -1;
            if (page < 0 || page >= p.pool.pages) {
                if (lane == 0) atomicOr(&g_status_word, kStatusIndex);
                return -1;
            }
            return (((int64_t)page * p.pool.kv_heads + h) * p.pool.chunks_per_page + c - (int)fast_div(c, p.by_page) * p.pool.chunks_per_page) * (35 * D);
        };
        Lane<NB> kx, vx;
        int64_t off = place(0, look_up(0));
        int page_ahead = look_up(1);
        if (off >= 0) load_lane<NB>(p.pool, off, false, lane, kx);
        for (int j = 0; j < n_tiles && alive; j++) {
            const int st = j & 1;
            const uint32_t parity = (uint32_t)(j >> 1 & 1) ^ 1u;
            const int c = 4 * (t_begin + j) + e;
            const bool stored = c < full && off >= 0;
            if (stored) load_lane<NB>(p.pool, off, true, lane, vx);
            alive = tc::mbar_wait_warp(k_empty + 8 * st, parity, abort_flag);
            if (!alive) break;
            if (off >= 0) expand_lane<DT, NB>(table, kx, false, sm + S::k + st * S::kv_tile, e, lane);
            // tile j + 8 reuses this flag: eight tiles on, every reader of tile j is done (two tiles in shared memory, one in S)
            if (lane == 0) {
                if (off >= 0) atomicOr((uint32_t *)&chunk_ok[j & 7], 1u << e);
                else atomicAnd((uint32_t *)&chunk_ok[j & 7], ~(1u << e));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) tc::mbar_arrive_local(k_full + 8 * st);
            const int64_t next = place(j + 1, page_ahead);
            page_ahead = look_up(j + 2);
            if (next >= 0) load_lane<NB>(p.pool, next, false, lane, kx);
            alive = tc::mbar_wait_warp(v_empty + 8 * st, parity, abort_flag);
            if (!alive) break;
            uint8_t *vt = sm + S::v + st * S::kv_tile;
            if (stored) {
                expand_lane<DT, NB>(table, vx, true, vt, e, lane);
            } else {
                // the unfinished chunk from the tail; nothing (zeros) behind it and where there is no page
                const int slot = p.batch.slot[seq];
                const bool tail = c == full && c < n_chunks && off >= 0, slot_ok = slot >= 0 && slot < p.pool.slots;
                if (tail && !slot_ok && lane == 0) atomicOr(&g_status_word, kStatusIndex);
                const int left = tail && slot_ok ? s.kv - c * kChunk : 0;
                tail_columns<NB>((const uint16_t *)p.pool.tail + tail_offset(p.pool, left ? slot : 0, h, c * kChunk), left, vt, e, lane);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) tc::mbar_arrive_local(v_full + 8 * st);
            off = next;
        }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        if (warp == 12) {
            // ---- MMA issuer ----
            const uint32_t hi = tc::desc_hi(1024, tc::kLayoutSwizzle128);
            const uint32_t idesc_s = 1u << 4 | kFmt << 7 | kFmt << 10 | (uint32_t)(128 >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
            const uint32_t idesc_o = 1u << 4 | kFmt << 7 | kFmt << 10 | (uint32_t)(D >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
            const uint32_t lo_q = (base + S::q) >> 4 | 1u << 16, lo_k = (base + S::k) >> 4 | 1u << 16, lo_v = (base + S::v) >> 4 | 1u << 16;
            auto scores = [&](int t, int st) {
                if (tc::elect_one()) {
#pragma unroll
                    for (int k = 0; k < D / 16; k++) {            // 64 elements per half, 16 per instruction
                        const uint32_t at = (uint32_t)(k / 4) * (128 * 128 >> 4) + 2u * (uint32_t)(k % 4);
                        mma_f16_ss(tmem + 128u * t, tc::desc_join(lo_q + (uint32_t)t * (S::q_tile >> 4) + at, hi), tc::desc_join(lo_k + (uint32_t)st * (S::kv_tile >> 4) + at, hi), idesc_s, k > 0);
                    }
                }
                __syncwarp();
            };
            auto values = [&](int t, int st, bool first, int half) {
                if (tc::elect_one()) {
#pragma unroll
                    for (int i = 0; i < kTileTokens / 32; i++) {
                        const int k = half * (kTileTokens / 32) + i;
                        const uint32_t at = (uint32_t)(k / 4) * (uint32_t)(D * 128 >> 4) + 2u * (uint32_t)(k % 4);
                        mma_f16_ts(tmem + 256u + 128u * t, tmem + 128u * t + 8u * k, tc::desc_join(lo_v + (uint32_t)st * (S::kv_tile >> 4) + at, hi), idesc_o, !(first && k == 0));
                    }
                }
                __syncwarp();
            };
            auto signal = [&](uint32_t bar) {
                if (tc::elect_one()) commit(bar);
                __syncwarp();
            };
            bool alive = n_tiles > 0 && tc::mbar_wait(q_full, 0, abort_flag, 0) && tc::mbar_wait(k_full, 0, abort_flag, 0);
            if (alive) {
                tc::tcgen05_fence_after();
                for (int t = 0; t < n_q; t++) {
                    scores(t, 0);
                    signal(s_full + 8 * t);
                }
                signal(k_empty);
            }
            for (int j = 0; j < n_tiles && alive; j++) {
                const int st = j & 1, nx = st ^ 1;
                const bool more = j + 1 < n_tiles;
                alive = tc::mbar_wait(v_full + 8 * st, j >> 1 & 1, abort_flag, 0);
                for (int t = 0; t < n_q && alive; t++) {
                    alive = tc::mbar_wait(p_half + 8 * t, j & 1, abort_flag, 0);
                    if (!alive) break;
                    tc::tcgen05_fence_after();
                    values(t, st, j == 0, 0);
                    alive = tc::mbar_wait(p_full + 8 * t, j & 1, abort_flag, 0);
                    if (!alive) break;
                    tc::tcgen05_fence_after();
                    values(t, st, false, 1);
                    if (more) {
                        if (t == 0) alive = tc::mbar_wait(k_full + 8 * nx, (j + 1) >> 1 & 1, abort_flag, 0);
                        if (!alive) break;
                        tc::tcgen05_fence_after();
                        scores(t, nx);
                    }
                    signal(s_full + 8 * t);
                }
                if (!alive) break;
                signal(v_empty + 8 * st);
                if (more) signal(k_empty + 8 * nx);
            }
            signal(drained);                                      // whatever was issued is complete before tensor memory goes back
            tc::mbar_wait(drained, 0, abort_flag + 4);            // (words of its own: an abort elsewhere must not cut this wait short)
        }
    }
    tc::tcgen05_fence_before();
    __syncthreads();
    tc::tcgen05_fence_after();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

}  // namespace pg
}  // namespace bd
