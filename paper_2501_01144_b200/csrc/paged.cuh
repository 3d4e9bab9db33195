// Writing the paged cache and reading it back (storage: paged_common.cuh).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bd_common.cuh"
#include "paged_common.cuh"
#include "quantize.cuh"

namespace bd {
namespace pg {

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <int DT>
__device__ __forceinline__ float load_one(const void *p) {
    if (DT == BD_F32) return *(const float *)p;
    if (DT == BD_BF16) return __uint_as_float((uint32_t) * (const uint16_t *)p << 16);
    return __half2float(*(const __half *)p);
}
// Whether a 32-bit word of elements holds an infinity or a NaN.
template <int DT>
__device__ __forceinline__ bool nonfinite(uint32_t w) {
    if (DT == BD_F32) return (w & 0x7f800000u) == 0x7f800000u;
    const uint32_t ones = DT == BD_BF16 ? 0x7f80u : 0x7c00u;
    return (w & ones) == ones || (w >> 16 & ones) == ones;
}
// A block in a thread's registers as the quantizers take it, and its quantisation into the record's words.
template <int DT>
struct Block {
    uint32_t bits[32];
    __device__ __forceinline__ void load(const void *p) { Loader<DT>::contiguous(p, bits); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < 32; k++) bits[k] = 0;
    }
    // column `ch` of 32 rows of `pitch` bytes in shared memory
    __device__ __forceinline__ void column(const uint8_t *rows, int pitch, int ch) {
#pragma unroll
        for (int k = 0; k < 32; k++) bits[k] = __float_as_uint(load_one<DT>(rows + k * pitch + ch * Loader<DT>::kElemBytes));
    }
    __device__ __forceinline__ void quantize(const SmemTables &tab, BlockResult &res) const {
        uint32_t unused[8];
        bool nonfinite;
        quantize_two_stage_f32<false, true>(bits, tab, res, unused, nonfinite);
        if (nonfinite) atomicOr(&g_status_word, kStatusNonfinite);
    }
};
template <>
struct Block<BD_BF16> {                                           // two elements per register
    uint32_t pairs[16];
    __device__ __forceinline__ void load(const void *p) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint4 u = __ldg((const uint4 *)p + i);
            pairs[4 * i] = u.x; pairs[4 * i + 1] = u.y; pairs[4 * i + 2] = u.z; pairs[4 * i + 3] = u.w;
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < 16; k++) pairs[k] = 0;
    }
    __device__ __forceinline__ void column(const uint8_t *rows, int pitch, int ch) {
#pragma unroll
        for (int k = 0; k < 16; k++)
            pairs[k] = (uint32_t) * (const uint16_t *)(rows + 2 * k * pitch + 2 * ch) | (uint32_t) * (const uint16_t *)(rows + (2 * k + 1) * pitch + 2 * ch) << 16;
    }
    __device__ __forceinline__ void quantize(const SmemTables &tab, BlockResult &res) const {
        uint32_t unused[8];
        quantize_bf16_block<false, true>(pairs, tab, res, unused);
    }
};

// ---------------------------------------------------------------------------
// Append.  A CTA takes one chunk of one sequence and head.  The chunk's value rows are copied to shared memory if this
// step completes it (those of earlier steps from the tail); under that copy its threads quantise the chunk's new keys
// (thread = token and block of 32 dimensions), then the values (thread = channel).  The CTA of the sequence's first chunk
// also stores the step's newest value rows in the tail, after it has read the waiting ones: those of the newest chunk
// and of the one before it.
// A record's part that is new as a whole is assembled in shared memory and leaves as 16-byte pieces; the keys of a partly new
// chunk go out as the few words that are theirs, since their neighbours belong to other steps.
// Bound: 2 * 2 d bytes read and 35 / 32 d written per token and head for 16-bit sources.  7346 bf16 tokens x 8 heads x 128: 14.0 us =
// 2.7 TB/s; 58 % of the issue slots while SMs are active, the warps waiting for each other at the chunk's barriers and for shared-memory
// instructions (a value block is 32 two-byte reads).  One token of 64 sequences: 3.4 us.
// ---------------------------------------------------------------------------
template <int DT, int NB>
__global__ void __launch_bounds__(NB * 32) append_kernel(Pool pool, Batch batch, const uint8_t *__restrict__ K,
                                                         const uint8_t *__restrict__ V, int64_t ldk, int64_t ldv,
                                                         int64_t hsk, int64_t hsv) {
    constexpr int D = 32 * NB, EB = Loader<DT>::kElemBytes, kPieces = D * EB / 16, kPitch = D * EB;
    __shared__ SmemTables tab;
    __shared__ __align__(16) uint8_t rec[35 * D];
    __shared__ __align__(16) uint8_t rows[32 * kPitch];
    __shared__ uint8_t vid[D];
    load_tables(tab);
    pdl_wait();
    pdl_release();
    const int seq = blockIdx.z, h = blockIdx.y;
    const Sequence s = sequence_of(batch, seq);
    const int slot = batch.slot[seq];
    if (!s.ok || s.t > s.kv || (s.t > 0 && (slot < 0 || slot >= pool.slots))) {   // (a sequence without rows needs no slot)
        if (threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
        return;
    }
    if (s.t == 0) return;
    const int p0 = s.kv - s.t, p1 = s.kv;
    const int c = p0 / kChunk + blockIdx.x;
    if (c * kChunk >= p1) return;
    const int lo = max(p0, c * kChunk) - c * kChunk, hi = min(p1 - c * kChunk, kChunk);   // the new tokens of this chunk
    const bool whole_keys = lo == 0 && hi == kChunk, whole_values = hi == kChunk;
    const uint8_t *Ks = K + ((int64_t)(s.q0 - p0 + c * kChunk) * ldk + (int64_t)h * hsk) * EB;   // row of the chunk's token 0
    const uint8_t *Vs = V + ((int64_t)(s.q0 - p0 + c * kChunk) * ldv + (int64_t)h * hsv) * EB;
    uint8_t *tail = (uint8_t *)pool.tail;
    if (whole_values)                                             // the chunk's 32 value rows
        for (int i = threadIdx.x; i < 32 * kPieces; i += NB * 32) {
            const int tok = i / kPieces, piece = i % kPieces;
            const uint8_t *src = tok >= lo ? Vs + (int64_t)tok * ldv * EB : tail + tail_offset(pool, slot, h, c * kChunk + tok) * EB;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(rows + 16 * i)), "l"((const uint4 *)src + piece) : "memory");
        }
    const int tok = threadIdx.x / NB, b = threadIdx.x % NB;
    const bool mine = tok >= lo && tok < hi;
    Block<DT> block;
    if (mine) block.load(Ks + ((int64_t)tok * ldk + 32 * b) * EB);
    else block.clear();
    const int64_t off = record_offset(pool, batch, seq, h, c);
    if (off < 0 && threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
    uint8_t *out = pool.base + (off < 0 ? 0 : off);
    BlockResult res;
    if (whole_keys || __any_sync(0xffffffffu, mine)) {
        block.quantize(tab, res);
        // the NB lanes of a token put its scales and ids together
        uint32_t sc = res.scale << (8 * b), ids = res.id << (4 * b);
#pragma unroll
        for (int x = 1; x < NB; x *= 2) {
            sc |= __shfl_xor_sync(0xffffffffu, sc, x);
            ids |= __shfl_xor_sync(0xffffffffu, ids, x);
        }
        const int r = key_row(tok), e = entry_of(NB, 0, r);
        uint8_t *to = whole_keys ? rec : out;
        if (mine && off >= 0) {
#pragma unroll
            for (int t = 0; t < 4; t++) *(uint32_t *)(to + word_byte(b, r, t)) = res.words[t];
            if (b == 0) {
                if (NB == 4) {
                    *(uint32_t *)(to + key_scales(D) + e) = sc;
                    *(uint16_t *)(to + key_ids(D) + e / 2) = (uint16_t)ids;
                } else {
                    *(uint16_t *)(to + key_scales(D) + e) = (uint16_t)sc;
                    *(to + key_ids(D) + e / 2) = (uint8_t)ids;
                }
            }
        }
    }
    if (whole_values) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        const int ch = threadIdx.x, vb = ch / 32, r = ch % 32, e = entry_of(NB, vb, r);
        block.column(rows, kPitch, ch);
        block.quantize(tab, res);
#pragma unroll
        for (int t = 0; t < 4; t++) *(uint32_t *)(rec + value_codes(D) + word_byte(vb, r, t)) = res.words[t];
        rec[value_scales(D) + e] = (uint8_t)res.scale;
        vid[e] = (uint8_t)res.id;
    }
    if (whole_values || whole_keys) {
        __syncthreads();
        if (whole_values && threadIdx.x < D / 2) rec[value_ids(D) + threadIdx.x] = vid[2 * threadIdx.x] | vid[2 * threadIdx.x + 1] << 4;
        __syncthreads();
        // whole parts of the record in 16-byte pieces (every part is a multiple of 16 bytes: D is 64 or 128)
        if (off >= 0)
            for (int i = threadIdx.x; i < 35 * D / 16; i += NB * 32) {
                const int at = 16 * i;
                const bool of_keys = at < 16 * D || (at >= 32 * D && at < 33 * D) || (at >= 34 * D && at < 34 * D + D / 2);
                if (of_keys ? whole_keys : whole_values) ((uint4 *)out)[i] = ((const uint4 *)rec)[i];
            }
    }
    if (blockIdx.x == 0) {
        // (the waiting rows are in shared memory of every thread's copy: it waited, and met the others, above)
        const int from = max(p0, p1 / kChunk * kChunk - kChunk);
        bool bad = false;
        for (int i = threadIdx.x; i < (p1 - from) * kPieces; i += NB * 32) {
            const int row = from + i / kPieces, piece = i % kPieces;
            const uint8_t *src = V + ((int64_t)(s.q0 + row - p0) * ldv + (int64_t)h * hsv) * EB;
            const uint4 x = *((const uint4 *)src + piece);
            *((uint4 *)(tail + tail_offset(pool, slot, h, row) * EB) + piece) = x;
            bad |= nonfinite<DT>(x.x) || nonfinite<DT>(x.y) || nonfinite<DT>(x.z) || nonfinite<DT>(x.w);
        }
        if (bad) atomicOr(&g_status_word, kStatusNonfinite);      // (told with the step, not when the chunk is full)
    }
}

// 2^(scale - 128), the factor of the half-unit integers; subnormal for scales 0 and 1.
__device__ __forceinline__ float half_unit(uint32_t scale) {
    return scale > 1u ? __uint_as_float((scale - 1u) << 23) : __uint_as_float(scale ? 0x00400000u : 0x00200000u);
}
// Byte tables of a block's magnitudes h * 2^(scale - 128) in bf16 or fp16, lo[8] and hi[8]: the dialect's table (see
// float_table; copied to shared memory by the first threads of a CTA) with the block's scale added to the exponent bits.
// Blocks outside the range of those sums (bf16: scale < 2, fp16: scale < 114, where subnormals begin) are built value by value.
template <int DT>
__device__ __forceinline__ void make_base_tables(uint4 *to) {
    const uint32_t *from = DT == BD_BF16 ? &c_tables.bf16[0].w[0] : &c_tables.f16[0].w[0];
    for (int i = threadIdx.x; i < (DT == BD_BF16 ? 128 : 64); i += blockDim.x) ((uint32_t *)to)[i] = from[i];
}
// TINY: bf16 blocks of scale < 2 (magnitudes below 2^-123) keep their subnormal values; otherwise they count as zeros.
// LOW: fp16 blocks may have scales below kF16Normal.
constexpr uint32_t kF16Normal = 114;
template <int DT, bool TINY, bool LOW = true>
__device__ __forceinline__ uint4 block_table(const uint4 *base, uint32_t id, uint32_t scale) {
    uint4 t = base[DT == BD_BF16 ? 2 * id + (scale & 1u) : id];
    const uint32_t k = DT == BD_BF16 ? (scale >> 1) - 1u : (scale - 113u) * 4u;
    t.z += k * 0x01010100u;
    t.w += k * 0x01010101u;
    if (DT == BD_BF16 && !TINY) {
        if (scale < 2u) t = make_uint4(0, 0, 0, 0);
    } else if (LOW && scale < (DT == BD_BF16 ? 2u : kF16Normal)) {
        uint32_t b[4] = {0, 0, 0, 0};
        const uint32_t tlo = c_tables.int_lo[id], thi = c_tables.int_hi[id];
#pragma unroll
        for (int i = 1; i < 8; i++) {
            const float v = (float)((i < 4 ? tlo >> (8 * i) : thi >> (8 * (i - 4))) & 255u) * half_unit(scale);
            const uint32_t h = DT == BD_BF16 ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v)) : (uint32_t)__half_as_ushort(__float2half_rn(v));
            b[i / 4] |= (h & 255u) << (8 * (i % 4));
            b[2 + i / 4] |= (h >> 8) << (8 * (i % 4));
        }
        t = make_uint4(b[0], b[1], b[2], b[3]);
    }
    return t;
}
__device__ __forceinline__ uint4 expand_word(uint32_t w, const uint4 &t) {
    const uint32_t sel = w & 0x77777777u, sel_b = sel >> 16, even = w << 4;
    const uint32_t lo_a = prmt_b32(t.x, t.y, sel), lo_b = prmt_b32(t.x, t.y, sel_b);
    const uint32_t hi_a = prmt_b32(t.z, t.w, sel) | (prmt_b32(even, w, 0x5140u) & 0x80808080u);
    const uint32_t hi_b = prmt_b32(t.z, t.w, sel_b) | (prmt_b32(even, w, 0x7362u) & 0x80808080u);
    return make_uint4(prmt_b32(lo_a, hi_a, 0x6240u), prmt_b32(lo_a, hi_a, 0x7351u), prmt_b32(lo_b, hi_b, 0x6240u), prmt_b32(lo_b, hi_b, 0x7351u));
}

// The eight values of a word as fp32, in element order; f = 2^(e - 1).
__device__ __forceinline__ void word_values(uint32_t w, uint32_t tlo, uint32_t thi, float f, float (&v)[8]) {
    const uint32_t sel = w & 0x77777777u;
    const uint32_t xa = prmt_b32(tlo, thi, sel), xb = prmt_b32(tlo, thi, sel >> 16);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const int n = place_of<true>(e);
        const uint32_t h = ((n < 4 ? xa : xb) >> (8 * (n & 3))) & 0xffu;
        v[e] = __uint_as_float(__float_as_uint((float)h * f) | ((w >> (4 * n + 3)) & 1u) << 31);
    }
}

// ---------------------------------------------------------------------------
// Read back: the last t tokens of each sequence as values of the cache's type (exact for fp32 and bf16; fp16 rounds what
// lies below its normal range).  A CTA takes one chunk of one head, warp b its tile b of keys and of values; lane 4 g + t reads
// the words t of the rows g, 8 + g, 16 + g, 24 + g as one 16-byte piece of each.
// 16-bit types: a word becomes eight values with byte permutes (see block_table).  A key word is then 16 consecutive bytes of
// a token's result; the value words of a warp are eight tokens of a channel each, which stmatrix turns around on the way to
// shared memory (pieces exchanged within a row so that its eight rows meet different banks), from where whole tokens leave.
// fp32 (read_f32_kernel): the record comes to shared memory, values are multiplied out element by element.
// The tokens of an unfinished chunk come from the tail.  7346 bf16 tokens x 8 heads x 128: 10.2 us, of which writing 30 MB is
// the larger part (a fill reaches 3.9 TB/s here).
// ---------------------------------------------------------------------------
__device__ __forceinline__ int turned_piece(int token, int piece) { return piece ^ ((token >> 3) << 1 | (token & 1)); }

template <int DT, int NB>
__global__ void __launch_bounds__(NB * 32) read_kernel(Pool pool, Batch batch, uint8_t *__restrict__ K, uint8_t *__restrict__ V,
                                                       int64_t ldk, int64_t ldv, int64_t hsk, int64_t hsv) {
    constexpr int D = 32 * NB, kPieces = D / 8;
    __shared__ uint4 base[32];
    __shared__ __align__(16) uint8_t rows[32 * D * 2];
    make_base_tables<DT>(base);
    pdl_wait();
    pdl_release();
    const int seq = blockIdx.z, h = blockIdx.y, b = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const Sequence s = sequence_of(batch, seq);
    if (!s.ok || s.t > s.kv) {
        if (threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
        return;
    }
    if (s.t == 0) return;
    const int p0 = s.kv - s.t, p1 = s.kv;
    const int c = p0 / kChunk + blockIdx.x;
    if (c * kChunk >= p1) return;
    const int lo = max(p0, c * kChunk) - c * kChunk, hi = min(p1 - c * kChunk, kChunk);
    const bool waiting = (c + 1) * kChunk > p1;                   // the unfinished chunk: its values are in the tail
    const int64_t off = record_offset(pool, batch, seq, h, c);
    const int slot = waiting ? batch.slot[seq] : 0;
    const bool slot_ok = slot >= 0 && slot < pool.slots;
    if ((off < 0 || !slot_ok) && threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
    const int64_t row0 = (int64_t)s.q0 - p0 + c * kChunk;         // output row of the chunk's token 0
    struct Tile {
        uint4 w;
        uint32_t scale, id;                                       // a byte and a nibble per row
    };
    auto fetch = [&](bool key) {                                  // (no page: scales, ids and codes 0, which is the value 0)
        Tile x{make_uint4(0, 0, 0, 0), 0, 0};
        if (off >= 0) {
            const uint8_t *rec = pool.base + off;
            x.w = *(const uint4 *)(rec + (key ? 0 : value_codes(D)) + 512 * b + 16 * lane);
            const uint8_t *sc = rec + (key ? key_scales(D) : value_scales(D)) + 4 * NB * g + b, *id = rec + (key ? key_ids(D) : value_ids(D)) + (4 * NB * g + b) / 2;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                x.scale |= (uint32_t)sc[NB * j] << (8 * j);
                x.id |= (uint32_t)(id[NB / 2 * j] >> (4 * (b & 1)) & 15) << (4 * j);
            }
        }
        return x;
    };
    const Tile key = fetch(true);
    Tile value = {};
    if (!waiting) value = fetch(false);
    __syncthreads();
    auto expand = [&](const Tile &x, int j) {
        const uint32_t w = j == 0 ? x.w.x : j == 1 ? x.w.y : j == 2 ? x.w.z : x.w.w;
        return expand_word(w, block_table<DT, true>(base, x.id >> (4 * j) & 15u, x.scale >> (8 * j) & 255u));
    };
    {
        uint8_t *to = K + (row0 * ldk + (int64_t)h * hsk + 32 * b + 8 * t) * 2;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint4 x = expand(key, j);
            const int tok = key_token(8 * j + g);
            if (tok >= lo && tok < hi) *(uint4 *)(to + tok * ldk * 2) = x;
        }
    }
    if (!waiting) {
        // matrix p of four: eight channels x the tokens 8 a + 2 p + i; this lane addresses the row i' of matrix lane / 8
        const int tok = 8 * (lane % 8 / 2) + 2 * (lane / 8) + lane % 2;
        const uint32_t row = (uint32_t)__cvta_generic_to_shared(rows) + tok * D * 2;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint4 x = expand(value, j);
            asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                         ::"r"(row + 16 * turned_piece(tok, 4 * b + j)), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
        }
        __syncthreads();
    }
    const int piece = threadIdx.x % kPieces;
    constexpr int kRowsATurn = NB * 32 / kPieces;
    const uint8_t *from = (const uint8_t *)pool.tail + (tail_offset(pool, slot_ok ? slot : 0, h, c * kChunk) + 8 * piece) * 2;
    uint8_t *to = V + (row0 * ldv + (int64_t)h * hsv + 8 * piece) * 2;
    for (int tok = lo + threadIdx.x / kPieces; tok < hi; tok += kRowsATurn) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (!waiting) x = ((const uint4 *)rows)[tok * kPieces + turned_piece(tok, piece)];
        else if (slot_ok) x = *(const uint4 *)(from + tok * D * 2);
        *(uint4 *)(to + tok * ldv * 2) = x;
    }
}

template <int NB>
__global__ void __launch_bounds__(NB * 32) read_f32_kernel(Pool pool, Batch batch, uint8_t *__restrict__ K, uint8_t *__restrict__ V,
                                                       int64_t ldk, int64_t ldv, int64_t hsk, int64_t hsv) {
    constexpr int D = 32 * NB, EB = 4, kPieces = D * EB / 16, kPitch = D * EB + 16;
    __shared__ uint2 table[16];
    __shared__ __align__(16) uint8_t rec[35 * D];
    __shared__ __align__(16) uint8_t rows[32 * kPitch];
    if (threadIdx.x < 16) table[threadIdx.x] = make_uint2(c_tables.int_lo[threadIdx.x], c_tables.int_hi[threadIdx.x]);
    pdl_wait();
    pdl_release();
    const int seq = blockIdx.z, h = blockIdx.y;
    const Sequence s = sequence_of(batch, seq);
    if (!s.ok || s.t > s.kv) {
        if (threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
        return;
    }
    if (s.t == 0) return;
    const int p0 = s.kv - s.t, p1 = s.kv;
    const int c = p0 / kChunk + blockIdx.x;
    if (c * kChunk >= p1) return;
    const int lo = max(p0, c * kChunk) - c * kChunk, hi = min(p1 - c * kChunk, kChunk);
    const bool waiting = (c + 1) * kChunk > p1;                   // the unfinished chunk: its values are in the tail
    const int64_t off = record_offset(pool, batch, seq, h, c);
    const int slot = waiting ? batch.slot[seq] : 0;
    const bool slot_ok = slot >= 0 && slot < pool.slots;
    if ((off < 0 || !slot_ok) && threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
    const int64_t row0 = (int64_t)s.q0 - p0 + c * kChunk;         // output row of the chunk's token 0
    for (int i = threadIdx.x; i < 35 * D / 16; i += NB * 32)      // (no page: scales, ids and codes 0, which is the value 0)
        ((uint4 *)rec)[i] = off >= 0 ? ((const uint4 *)(pool.base + off))[i] : make_uint4(0, 0, 0, 0);
    __syncthreads();
    // word t of row r of tile b
    auto word = [&](bool key, int b, int r, int t, const uint2 &tb, float f, float (&v)[8]) {
        word_values(*(const uint32_t *)(rec + (key ? 0 : value_codes(D)) + word_byte(b, r, t)), tb.x, tb.y, f, v);
    };
    auto entry = [&](bool key, int b, int r, uint2 &tb, float &f) {
        const int e = entry_of(NB, b, r);
        tb = table[rec[(key ? key_ids(D) : value_ids(D)) + e / 2] >> (4 * (e & 1)) & 15];
        f = half_unit(rec[(key ? key_scales(D) : value_scales(D)) + e]);
    };
    uint2 tb;
    float f = 0.0f, v[8];
    // keys: neighbouring threads take neighbouring words of a token, so that their stores join
    {
        const int b = threadIdx.x / 4 % NB, t = threadIdx.x % 4;
        uint8_t *to = K + ((row0 + lo + threadIdx.x / (4 * NB)) * ldk + (int64_t)h * hsk + 32 * b + 8 * t) * EB;
        for (int tok = lo + threadIdx.x / (4 * NB); tok < hi; tok += 8, to += 8 * ldk * EB) {
            const int r = key_row(tok);
            entry(true, b, r, tb, f);
            word(true, b, r, t, tb, f, v);
            ((float4 *)to)[0] = make_float4(v[0], v[1], v[2], v[3]);
            ((float4 *)to)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
    if (!waiting) {
        const int ch = threadIdx.x, b = ch / 32, r = ch % 32;
        uint8_t *to = rows + ch * EB;
        entry(false, b, r, tb, f);
#pragma unroll
        for (int t = 0; t < 4; t++) {
            word(false, b, r, t, tb, f, v);
#pragma unroll
            for (int k = 0; k < 8; k++) *(float *)(to + (8 * t + k) * kPitch) = v[k];
        }
        __syncthreads();
    }
    const int piece = threadIdx.x % kPieces;
    constexpr int kRowsATurn = NB * 32 / kPieces;
    int tok = lo + threadIdx.x / kPieces;
    uint8_t *to = V + ((row0 + tok) * ldv + (int64_t)h * hsv) * EB + 16 * piece;
    const uint8_t *from = waiting ? (const uint8_t *)pool.tail + tail_offset(pool, slot_ok ? slot : 0, h, c * kChunk + tok) * EB + 16 * piece : rows + tok * kPitch + 16 * piece;
    for (; tok < hi; tok += kRowsATurn, to += kRowsATurn * ldv * EB, from += kRowsATurn * (waiting ? D * EB : kPitch))
        *(uint4 *)to = !waiting || slot_ok ? *(const uint4 *)from : make_uint4(0, 0, 0, 0);
}

// ---------------------------------------------------------------------------
// Queries and keys of a step: y = x / sqrt(mean(x^2) + eps) * w per head (w may be absent: no normalisation), then the
// rotation of the first `rot` elements, (a, b) -> (a cos - b sin, b cos + a sin), with cos and sin from the caller's
// table [positions][rot] (rot / 2 cosines, then rot / 2 sines).  Pairs are (i, i + rot / 2), or (2 i, 2 i + 1).
// All arithmetic in fp32, one rounding at the end.
// D / 8 lanes hold a head, eight elements each as two groups of four: of the rotated part elements 4 l .. and rot / 2 + 4 l ..
// (pairs that are half the part apart meet in one lane, no exchange), else eight neighbours.  A group of lanes does up to
// five heads of its row, all loads in front, with the row's cosines and sines in registers.
// Bound: bytes (every element read and written once).  8192 rows x 40 heads x 128 bf16: 33 us = 5.3 TB/s; 64 rows: 1.9 us.
// ---------------------------------------------------------------------------
template <int DT>
struct Quad { typedef uint2 Type; };                              // four elements
template <>
struct Quad<BD_F32> { typedef uint4 Type; };
__device__ __forceinline__ void unpack_f32(const uint4 &u, float *x) {
    x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
}
template <int DT>
__device__ __forceinline__ void unpack4(const uint2 &u, float *x) {
    const uint32_t w[2] = {u.x, u.y};
#pragma unroll
    for (int i = 0; i < 2; i++) {
        if (DT == BD_BF16) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const float2 f = __half22float2(*(const __half2 *)&w[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
}
template <int DT>
__device__ __forceinline__ void unpack4(const uint4 &u, float *x) { unpack_f32(u, x); }
template <int DT>
__device__ __forceinline__ void store4(uint8_t *p, const float *x) {
    if (DT == BD_F32) {
        *(float4 *)p = make_float4(x[0], x[1], x[2], x[3]);
    } else if (DT == BD_BF16) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
        *(uint2 *)p = make_uint2(*(const uint32_t *)&a, *(const uint32_t *)&b);
    } else {
        const __half2 a = __floats2half2_rn(x[0], x[1]), b = __floats2half2_rn(x[2], x[3]);
        *(uint2 *)p = make_uint2(*(const uint32_t *)&a, *(const uint32_t *)&b);
    }
}

struct Rotation {
    const uint8_t *q, *k;
    uint8_t *q_out, *k_out;
    int64_t ldq, hsq, ldk, hsk, ldqo, hsqo, ldko, hsko;           // elements
    const void *wq, *wk;
    const int32_t *pos;
    const float *table;
    int64_t positions;
    int rows, q_heads, k_heads, rot;
    float eps;
};
constexpr int kRotateThreads = 128, kRotateHeads = 5;             // 16 or 8 groups of lanes, heads a group has in flight

template <int DT, int D, bool NEIGHBOURS, int HEADS>
__global__ void __launch_bounds__(kRotateThreads) rotate_kernel(Rotation p) {
    constexpr int EB = DT == BD_F32 ? 4 : 2, LANES = D / 8, GROUPS = kRotateThreads / LANES;
    typedef typename Quad<DT>::Type Q4;
    pdl_wait();
    pdl_release();
    const int row = blockIdx.x, l = threadIdx.x % LANES, h0 = blockIdx.y * GROUPS * HEADS + threadIdx.x / LANES, heads = p.q_heads + p.k_heads;
    const int half = p.rot / 2;
    const bool turned = 8 * l < p.rot;
    const int e0 = !NEIGHBOURS && turned ? 4 * l : 8 * l, e1 = !NEIGHBOURS && turned ? half + 4 * l : 8 * l + 4;
    const int pos = p.pos[row];
    const uint8_t *q = p.q + ((int64_t)row * p.ldq + e0) * EB, *kk = p.k + ((int64_t)row * p.ldk + e0) * EB;
    const int de = (e1 - e0) * EB;
    const int64_t hsq = p.hsq * EB, hsk = p.hsk * EB, hsqo = p.hsqo * EB, hsko = p.hsko * EB;
    Q4 raw[HEADS][2];
#pragma unroll
    for (int i = 0; i < HEADS; i++) {                             // all loads in front, none waits for the position
        const int h = h0 + i * GROUPS;
        if (h < heads) {
            const uint8_t *src = h < p.q_heads ? q + (int64_t)h * hsq : kk + (int64_t)(h - p.q_heads) * hsk;
            raw[i][0] = *(const Q4 *)src;
            raw[i][1] = *(const Q4 *)(src + de);
        }
    }
    if (pos < 0 || pos >= p.positions) {                          // (the whole CTA)
        if (threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
        return;
    }
    float4 co = make_float4(1.0f, 1.0f, 1.0f, 1.0f), si = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (turned) {
        const float *tb = p.table + (int64_t)pos * p.rot + 4 * l;
        co = *(const float4 *)tb;
        si = *(const float4 *)(tb + half);
    }
    uint8_t *qo = p.q_out + ((int64_t)row * p.ldqo + e0) * EB, *ko = p.k_out + ((int64_t)row * p.ldko + e0) * EB;
#pragma unroll
    for (int i = 0; i < HEADS; i++) {
        const int h = h0 + i * GROUPS;
        if (h - (int)(threadIdx.x / LANES) >= heads) return;      // whole warps take every turn (shuffles)
        const bool is_q = h < p.q_heads;
        float x[8] = {}, y[8];
        if (h < heads) {
            unpack4<DT>(raw[i][0], x);
            unpack4<DT>(raw[i][1], x + 4);
        }
        if (p.wq || p.wk) {                                       // (the same in all lanes)
            float ss = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; j++) ss = fmaf(x[j], x[j], ss);
#pragma unroll
            for (int m = 1; m < LANES; m *= 2) ss += __shfl_xor_sync(0xffffffffu, ss, m);
            const uint8_t *w = (const uint8_t *)(is_q ? p.wq : p.wk);
            if (w) {
                const float inv = rsqrtf(ss * (1.0f / D) + p.eps);
                float g[8];
                unpack4<DT>(*(const Q4 *)(w + e0 * EB), g);
                unpack4<DT>(*(const Q4 *)(w + e0 * EB + de), g + 4);
#pragma unroll
                for (int j = 0; j < 8; j++) x[j] = x[j] * inv * g[j];
            }
        }
        const float c[4] = {co.x, co.y, co.z, co.w}, s[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int a = NEIGHBOURS ? 2 * j : j, b = NEIGHBOURS ? 2 * j + 1 : j + 4;
            y[a] = turned ? x[a] * c[j] - x[b] * s[j] : x[a];
            y[b] = turned ? x[b] * c[j] + x[a] * s[j] : x[b];
        }
        if (h < heads) {
            uint8_t *to = is_q ? qo + (int64_t)h * hsqo : ko + (int64_t)(h - p.q_heads) * hsko;
            store4<DT>(to, y);
            store4<DT>(to + de, y + 4);
        }
    }
}

}  // namespace pg
}  // namespace bd
