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

// Element e of a word sits in nibble kNibble[e] (its own inverse): the quantizer gets its elements in that order.
__device__ __forceinline__ constexpr int nibble_of(int e) {
    return e == 1 ? 2 : e == 2 ? 1 : e == 5 ? 6 : e == 6 ? 5 : e;
}
// The quantizer's word (signs of slots 0..3 in bits 8 s + 7, of 4..7 in bits 8 (s - 4) + 3) with each sign in bit 3 of
// its own nibble.
__device__ __forceinline__ uint32_t signs_to_nibbles(uint32_t w) {
    uint32_t lo = (w >> 7) & 0x01010101u, hi = (w >> 3) & 0x01010101u;
    lo = (lo | lo >> 4) & 0x00110011u;
    hi = (hi | hi >> 4) & 0x00110011u;
    lo = (lo | lo >> 8) & 0x1111u;
    hi = (hi | hi >> 8) & 0x1111u;
    return (w & 0x77777777u) | lo << 3 | hi << 19;
}
template <int DT>
__device__ __forceinline__ float load_one(const void *p) {
    if (DT == BD_F32) return *(const float *)p;
    if (DT == BD_BF16) return __uint_as_float((uint32_t) * (const uint16_t *)p << 16);
    return __half2float(*(const __half *)p);
}
template <int DT>
__device__ __forceinline__ void store_one(void *p, float v) {
    if (DT == BD_F32) *(float *)p = v;
    else if (DT == BD_BF16) *(__nv_bfloat16 *)p = __float2bfloat16_rn(v);
    else *(__half *)p = __float2half_rn(v);
}
// Quantises 32 fp32 bit patterns (in element order) into four words in the record's nibble order.
__device__ __forceinline__ void quantize_words(const uint32_t (&bits)[32], const SmemTables &tab, uint32_t (&words)[4],
                                               uint32_t &id, uint32_t &scale) {
    uint32_t ordered[32], unused[8];
#pragma unroll
    for (int k = 0; k < 32; k++) ordered[(k & ~7) + nibble_of(k & 7)] = bits[k];
    BlockResult res;
    bool nonfinite;
    quantize_two_stage_f32<false>(ordered, tab, res, unused, nonfinite);
    if (nonfinite) atomicOr(&g_status_word, kStatusNonfinite);
#pragma unroll
    for (int w = 0; w < 4; w++) words[w] = signs_to_nibbles(res.words[w]);
    id = res.id;
    scale = res.scale;
}

// ---------------------------------------------------------------------------
// Append.  A CTA takes one chunk of one sequence and head: its first half quantises the chunk's new keys (thread =
// token and block of 32 dimensions), its second half the chunk's values if this step completes it (thread = channel;
// the rows of earlier steps come from the tail).  The CTA of the sequence's first chunk also stores the step's newest
// value rows in the tail, after it has read the waiting ones: those of the newest chunk and of the one before it.
// Everything is assembled in shared memory.  A chunk whose 32 keys are all new leaves as whole 16-byte pieces; the
// keys of a partly new chunk go out as the few words that are theirs, since their neighbours belong to other steps.
// Bytes set the bound: 2 * 2 d read and 35 / 32 d written per token and head for 16-bit sources.
// ---------------------------------------------------------------------------
template <int DT, int NB>
__global__ void __launch_bounds__(NB * 64) append_kernel(Pool pool, Batch batch, const uint8_t *__restrict__ K,
                                                         const uint8_t *__restrict__ V, int64_t ldk, int64_t ldv,
                                                         int64_t hsk, int64_t hsv) {
    constexpr int D = 32 * NB, EB = Loader<DT>::kElemBytes, HALF = NB * 32;
    __shared__ SmemTables tab;
    __shared__ __align__(16) uint8_t rec[35 * D];
    __shared__ __align__(16) uint8_t rows[32 * D * EB];
    __shared__ uint8_t vid[D];
    load_tables(tab);
    pdl_wait();
    pdl_release();
    const int seq = blockIdx.z, h = blockIdx.y;
    const Sequence s = sequence_of(batch, seq);
    const int slot = batch.slot[seq];
    if (!s.ok || s.t > s.kv || slot < 0 || slot >= pool.slots) {
        if (threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
        return;
    }
    if (s.t == 0) return;
    const int p0 = s.kv - s.t, p1 = s.kv;
    const int c = p0 / kChunk + blockIdx.x;
    if (c * kChunk >= p1) return;
    const int64_t off = record_offset(pool, batch, seq, h, c);
    if (off < 0 && threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
    uint8_t *out = pool.base + (off < 0 ? 0 : off);
    const int lo = max(p0, c * kChunk) - c * kChunk, hi = min(p1 - c * kChunk, kChunk);   // the new tokens of this chunk
    const bool whole_keys = lo == 0 && hi == kChunk, whole_values = hi == kChunk;
    const uint8_t *Ks = K + ((int64_t)(s.q0 - p0 + c * kChunk) * ldk + (int64_t)h * hsk) * EB;   // row of the chunk's token 0
    const uint8_t *Vs = V + ((int64_t)(s.q0 - p0 + c * kChunk) * ldv + (int64_t)h * hsv) * EB;
    uint8_t *tail = (uint8_t *)pool.tail;

    if (whole_values && off >= 0) {                               // the chunk's 32 value rows
        constexpr int kPieces = D * EB / 16;
        for (int i = threadIdx.x; i < 32 * kPieces; i += blockDim.x) {
            const int tok = i / kPieces, piece = i % kPieces;
            const uint8_t *src = tok >= lo ? Vs + (int64_t)tok * ldv * EB : tail + tail_offset(pool, slot, h, c * kChunk + tok) * EB;
            ((uint4 *)rows)[i] = *((const uint4 *)src + piece);
        }
    }
    __syncthreads();
    const bool keys = threadIdx.x < HALF;
    uint32_t bits[32], words[4], id, scale;
    if (keys && off >= 0) {
        const int tok = threadIdx.x / NB, b = threadIdx.x % NB;
        const bool mine = tok >= lo && tok < hi;
        if (mine) Loader<DT>::contiguous(Ks + ((int64_t)tok * ldk + 32 * b) * EB, bits);
        else
#pragma unroll
            for (int k = 0; k < 32; k++) bits[k] = 0;
        quantize_words(bits, tab, words, id, scale);
        // the NB lanes of a token put its scales and ids together
        uint32_t sc = scale << (8 * b), ids = id << (4 * b);
#pragma unroll
        for (int x = 1; x < NB; x *= 2) {
            sc |= __shfl_xor_sync(0xffffffffu, sc, x);
            ids |= __shfl_xor_sync(0xffffffffu, ids, x);
        }
        const int r = key_row(tok), e = entry_of(NB, 0, r);
        uint8_t *to = whole_keys ? rec : out;
        if (mine) {
#pragma unroll
            for (int t = 0; t < 4; t++) *(uint32_t *)(to + word_byte(b, r, t)) = words[t];
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
    } else if (!keys && whole_values && off >= 0) {
        const int ch = threadIdx.x - HALF;
#pragma unroll
        for (int k = 0; k < 32; k++) bits[k] = __float_as_uint(load_one<DT>(rows + (k * D + ch) * EB));
        quantize_words(bits, tab, words, id, scale);
        const int b = ch / 32, r = ch % 32, e = entry_of(NB, b, r);
#pragma unroll
        for (int t = 0; t < 4; t++) *(uint32_t *)(rec + value_codes(D) + word_byte(b, r, t)) = words[t];
        rec[value_scales(D) + e] = (uint8_t)scale;
        vid[e] = (uint8_t)id;
    }
    __syncthreads();
    if (off >= 0) {
        if (whole_values && threadIdx.x < D / 2) rec[value_ids(D) + threadIdx.x] = vid[2 * threadIdx.x] | vid[2 * threadIdx.x + 1] << 4;
        __syncthreads();
        // whole parts of the record in 16-byte pieces (every part is a multiple of 16 bytes: D is 64 or 128)
        for (int i = threadIdx.x; i < 35 * D / 16; i += blockDim.x) {
            const int at = 16 * i;
            const bool of_keys = at < 16 * D || (at >= 32 * D && at < 33 * D) || (at >= 34 * D && at < 34 * D + D / 2);
            if (of_keys ? whole_keys : whole_values) ((uint4 *)out)[i] = ((const uint4 *)rec)[i];
        }
    }
    if (blockIdx.x == 0) {                                        // (the waiting rows were read above)
        const int from = max(p0, p1 / kChunk * kChunk - kChunk);
        constexpr int kPieces = D * EB / 16;
        for (int i = threadIdx.x; i < (p1 - from) * kPieces; i += blockDim.x) {
            const int tok = from + i / kPieces, piece = i % kPieces;
            const uint8_t *src = V + ((int64_t)(s.q0 + tok - p0) * ldv + (int64_t)h * hsv) * EB;
            *((uint4 *)(tail + tail_offset(pool, slot, h, tok) * EB) + piece) = *((const uint4 *)src + piece);
        }
    }
}

// The eight values of a word as fp32, in element order; f = 2^(e - 1).
__device__ __forceinline__ void word_values(uint32_t w, uint32_t tlo, uint32_t thi, float f, float (&v)[8]) {
    const uint32_t sel = w & 0x77777777u;
    const uint32_t xa = prmt_b32(tlo, thi, sel), xb = prmt_b32(tlo, thi, sel >> 16);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const int n = nibble_of(e);
        const uint32_t h = ((n < 4 ? xa : xb) >> (8 * (n & 3))) & 0xffu;
        const float m = (float)h * f;
        v[e] = __uint_as_float(__float_as_uint(m) | ((w >> (4 * n + 3)) & 1u) << 31);
    }
}
// 2^(scale - 128), the factor of the half-unit integers; subnormal for scales 0 and 1.
__device__ __forceinline__ float half_unit(uint32_t scale) {
    return scale > 1u ? __uint_as_float((scale - 1u) << 23) : __uint_as_float(scale ? 0x00400000u : 0x00200000u);
}

// ---------------------------------------------------------------------------
// Read back: the last t tokens of each sequence as values of the cache's type (exact for fp32 and bf16; fp16 rounds
// what lies below its subnormals).  A CTA takes one chunk of one head; the first half of its threads expands key
// blocks (thread = token and block, 32 consecutive outputs), the second half value blocks (thread = channel), which
// meet in shared memory and leave token by token; the tokens of an unfinished chunk come from the tail.
// ---------------------------------------------------------------------------
template <int DT, int NB>
__global__ void __launch_bounds__(NB * 64) read_kernel(Pool pool, Batch batch, uint8_t *__restrict__ K, uint8_t *__restrict__ V,
                                                       int64_t ldk, int64_t ldv, int64_t hsk, int64_t hsv) {
    constexpr int D = 32 * NB, EB = Loader<DT>::kElemBytes, HALF = NB * 32, kPieces = D * EB / 16;
    __shared__ uint2 table[16];
    __shared__ __align__(16) uint8_t rows[32 * (D * EB + 16)];    // value rows, padded by 16 bytes
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
    const uint8_t *rec = pool.base + (off < 0 ? 0 : off);
    const int64_t row0 = (int64_t)s.q0 - p0 + c * kChunk;         // output row of the chunk's token 0
    __syncthreads();
    if (threadIdx.x < HALF) {
        const int tok = threadIdx.x / NB, b = threadIdx.x % NB;
        if (tok >= lo && tok < hi) {
            const int r = key_row(tok), e = entry_of(NB, b, r);
            uint8_t *to = K + ((row0 + tok) * ldk + (int64_t)h * hsk + 32 * b) * EB;
            uint2 tb = make_uint2(0, 0);
            float f = 0.0f;
            if (off >= 0) {
                tb = table[rec[key_ids(D) + e / 2] >> (4 * (e & 1)) & 15];
                f = half_unit(rec[key_scales(D) + e]);
            }
#pragma unroll
            for (int t = 0; t < 4; t++) {
                float v[8];
                const uint32_t w = off >= 0 ? *(const uint32_t *)(rec + word_byte(b, r, t)) : 0u;
                word_values(w, tb.x, tb.y, f, v);
                __align__(16) uint8_t piece[8 * EB];
#pragma unroll
                for (int k = 0; k < 8; k++) store_one<DT>(piece + k * EB, v[k]);
#pragma unroll
                for (int k = 0; k < EB / 2; k++) ((uint4 *)(to + t * 8 * EB))[k] = ((const uint4 *)piece)[k];
            }
        }
    } else if (!waiting) {
        const int ch = threadIdx.x - HALF, b = ch / 32, r = ch % 32, e = entry_of(NB, b, r);
        uint2 tb = make_uint2(0, 0);
        float f = 0.0f;
        if (off >= 0) {
            tb = table[rec[value_ids(D) + e / 2] >> (4 * (e & 1)) & 15];
            f = half_unit(rec[value_scales(D) + e]);
        }
#pragma unroll
        for (int t = 0; t < 4; t++) {
            float v[8];
            const uint32_t w = off >= 0 ? *(const uint32_t *)(rec + value_codes(D) + word_byte(b, r, t)) : 0u;
            word_values(w, tb.x, tb.y, f, v);
#pragma unroll
            for (int k = 0; k < 8; k++) store_one<DT>(rows + (8 * t + k) * (D * EB + 16) + ch * EB, v[k]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (hi - lo) * kPieces; i += blockDim.x) {
        const int tok = lo + i / kPieces, piece = i % kPieces;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (!waiting) x = ((const uint4 *)(rows + tok * (D * EB + 16)))[piece];
        else if (slot_ok) x = *((const uint4 *)((const uint8_t *)pool.tail + tail_offset(pool, slot, h, c * kChunk + tok) * EB) + piece);
        *((uint4 *)(V + ((row0 + tok) * ldv + (int64_t)h * hsv) * EB) + piece) = x;
    }
}

// ---------------------------------------------------------------------------
// Queries and keys of a step: y = x / sqrt(mean(x^2) + eps) * w per head (w may be absent: no normalisation), then the
// rotation of the first `rot` elements, (a, b) -> (a cos - b sin, b cos + a sin), with cos and sin from the caller's
// table [positions][rot] (rot / 2 cosines, then rot / 2 sines).  Pairs are (i, i + rot / 2), or (2 i, 2 i + 1).
// All arithmetic in fp32, one rounding at the end.  D / 8 lanes hold a head, eight elements each; a warp's lanes walk
// over the heads of one row, so the row's cosines and sines are read once per lane and stay in registers.
// Bound: bytes (every element read and written once).
// ---------------------------------------------------------------------------
template <int DT>
__device__ __forceinline__ void load8(const uint8_t *p, float (&x)[8]) {
    if (DT == BD_F32) {
        const float4 a = ((const float4 *)p)[0], b = ((const float4 *)p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 u = *(const uint4 *)p;
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
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
}
template <int DT>
__device__ __forceinline__ void store8(uint8_t *p, const float (&x)[8]) {
    if (DT == BD_F32) {
        ((float4 *)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        ((float4 *)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (DT == BD_BF16) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *(const uint32_t *)&v;
            } else {
                const __half2 v = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *(const uint32_t *)&v;
            }
        }
        *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
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

template <int DT, int D, bool NEIGHBOURS>
__global__ void __launch_bounds__(256) rotate_kernel(Rotation p) {
    constexpr int EB = DT == BD_F32 ? 4 : 2, LANES = D / 8, GROUPS = 256 / LANES;
    pdl_wait();
    pdl_release();
    const int row = blockIdx.x, l = threadIdx.x % LANES, grp = threadIdx.x / LANES;
    const int pos = p.pos[row];
    const bool ok = pos >= 0 && pos < p.positions;
    if (!ok && threadIdx.x == 0) atomicOr(&g_status_word, kStatusIndex);
    // this lane's cosines and sines: one per element (halves) or per pair (neighbours); 1 and 0 outside the rotated part
    const bool turned = ok && 8 * l < p.rot;
    const int half = p.rot / 2;
    float co[8], si[8];
    const float *tb = p.table + (int64_t)(ok ? pos : 0) * p.rot;
    if (turned) {
        if (NEIGHBOURS) {
            const float4 a = *(const float4 *)(tb + 4 * l), b = *(const float4 *)(tb + half + 4 * l);
            co[0] = a.x; co[1] = a.y; co[2] = a.z; co[3] = a.w;
            si[0] = b.x; si[1] = b.y; si[2] = b.z; si[3] = b.w;
        } else {
            const int e = 8 * l < half ? 8 * l : 8 * l - half;
            const float sign = 8 * l < half ? -1.0f : 1.0f;
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float4 a = *(const float4 *)(tb + e + 4 * i), b = *(const float4 *)(tb + half + e + 4 * i);
                co[4 * i] = a.x; co[4 * i + 1] = a.y; co[4 * i + 2] = a.z; co[4 * i + 3] = a.w;
                si[4 * i] = sign * b.x; si[4 * i + 1] = sign * b.y; si[4 * i + 2] = sign * b.z; si[4 * i + 3] = sign * b.w;
            }
        }
    }
    const int partner = turned ? (8 * l < half ? l + half / 8 : l - half / 8) : l;
    const int lane0 = threadIdx.x % 32 - l;                       // the head's first lane in the warp
    const int heads = p.q_heads + p.k_heads;
    for (int h0 = 0; h0 < heads; h0 += GROUPS) {                  // whole warps take every turn (shuffles)
        const int h = h0 + grp;
        const bool active = h < heads, is_q = h < p.q_heads;
        const int hh = is_q ? h : h - p.q_heads;
        float x[8];
        if (active) load8<DT>((is_q ? p.q + (row * p.ldq + hh * p.hsq) * EB : p.k + (row * p.ldk + hh * p.hsk) * EB) + 8 * l * EB, x);
        else
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = 0.0f;
        const void *w = is_q ? p.wq : p.wk;
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i++) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int m = 1; m < LANES; m *= 2) ss += __shfl_xor_sync(0xffffffffu, ss, m);
        if (w) {
            const float inv = rsqrtf(ss * (1.0f / D) + p.eps);
            float g[8];
            load8<DT>((const uint8_t *)w + 8 * l * EB, g);
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = x[i] * inv * g[i];
        }
        float y[8];
        if (NEIGHBOURS) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                y[2 * i] = turned ? x[2 * i] * co[i] - x[2 * i + 1] * si[i] : x[2 * i];
                y[2 * i + 1] = turned ? x[2 * i + 1] * co[i] + x[2 * i] * si[i] : x[2 * i + 1];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float other = __shfl_sync(0xffffffffu, x[i], lane0 + partner);
                y[i] = turned ? x[i] * co[i] + other * si[i] : x[i];
            }
        }
        if (active && ok)
            store8<DT>((is_q ? p.q_out + (row * p.ldqo + hh * p.hsqo) * EB : p.k_out + (row * p.ldko + hh * p.hsko) * EB) + 8 * l * EB, y);
    }
}

}  // namespace pg
}  // namespace bd
