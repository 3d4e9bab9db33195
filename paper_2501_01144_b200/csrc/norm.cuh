// The norms around a block, fused with the residual sum between them:
//     u = norm(y) * (post_weight + offset) + post_bias     (or y itself)
//     h = residual + scale * gate * u
//     n = norm(h) * (weight + offset) + bias               (of the unrounded h; rounded to the rows' type once)
// with norm(x) = x / sqrt(mean(x^2) + eps), or (x - mean x) / sqrt(var x + eps); n may leave as a DialectFP4 operand, quantised from
// the rounded value by the two-stage rule, so that it has the bits that storing n and quantising it would give.
//
// A row lives in the registers of its threads (VPT pieces of eight elements each) from the first load to the last store: every
// input is read once, every output written once, and what stays are the reductions.  Sums, means and variances are fp32; the
// variance comes from the centred values in registers, not from a difference of squares.  For the quantised result a thread
// owns a whole block of 32 (rows that such blocks cover with aligned 16-byte accesses), or the row passes through shared memory, where a
// thread picks up a block.
// Bound: memory; a row's latency (two to four reductions) where there are few rows.  Measured (B200, from a graph): 8192 x 4096 bf16 with a
// residual and two norms, both results 48 us (268 MB, 5.6 TB/s), quantised 56 us (the quantiser's instructions); 1001 x 2559 fp32 (two layer norms) 13.0 us
// (rows of odd length: 4-byte accesses); 3000 x 768 fp16 4.7 us; 64 x 4096 quantised 3.2 us (one row's latency).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bd_common.cuh"
#include "quantize.cuh"

namespace bd {
namespace nm {

constexpr int kMaxDim = 16384, kMaxThreads = 512;

struct Args {
    const uint8_t *y, *residual, *gate, *post_weight, *post_bias, *weight, *bias;
    uint8_t *h, *n;
    int64_t ldy, ldr, ldh, ldn, gate_row;
    QView q;                                 // the quantised result (QUANT)
    int rows, dim, gate_col, layer, row_threads, row_groups;   // threads of a row, rows a CTA has at a time
    float scale, eps, offset;
};

// A piece of eight elements as it comes from memory.  VEC: neighbours, in one or two 16-byte accesses; else elements `step` apart.  Those
// behind `dim` are zeros.
template <int DT, bool VEC>
struct Piece {
    static constexpr int EB = Loader<DT>::kElemBytes, W = VEC ? EB / 2 : 1;
    uint4 raw[W];
    float one[VEC ? 1 : 8];
    __device__ __forceinline__ void load(const uint8_t *p, int e, int step, int dim) {
        if (VEC) {
#pragma unroll
            for (int i = 0; i < W; i++) raw[i] = e < dim ? *((const uint4 *)(p + (int64_t)e * EB) + i) : make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
            for (int q = 0; q < 8; q++) {
                const int at = e + q * step;
                float v = 0.0f;
                if (at < dim) {
                    const uint8_t *src = p + (int64_t)at * EB;
                    if (DT == BD_F32) v = *(const float *)src;
                    else if (DT == BD_BF16) v = __uint_as_float((uint32_t) * (const uint16_t *)src << 16);
                    else v = __half2float(*(const __half *)src);
                }
                one[VEC ? 0 : q] = v;
            }
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if (!VEC) {
#pragma unroll
            for (int q = 0; q < 8; q++) v[q] = one[VEC ? 0 : q];
        } else if (DT == BD_F32) {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const uint4 u = raw[W == 2 ? i : 0];
                v[4 * i] = __uint_as_float(u.x); v[4 * i + 1] = __uint_as_float(u.y); v[4 * i + 2] = __uint_as_float(u.z); v[4 * i + 3] = __uint_as_float(u.w);
            }
        } else {
            const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
            for (int q = 0; q < 4; q++) {
                if (DT == BD_BF16) {
                    v[2 * q] = __uint_as_float(w[q] << 16);
                    v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
                } else {
                    const float2 f = __half22float2(*(const __half2 *)&w[q]);
                    v[2 * q] = f.x;
                    v[2 * q + 1] = f.y;
                }
            }
        }
    }
};
template <int DT, bool VEC>
__device__ __forceinline__ void load8(const uint8_t *p, int e, int step, int dim, float (&v)[8]) {
    Piece<DT, VEC> t;
    t.load(p, e, step, dim);
    t.values(v);
}
template <int DT>
__device__ __forceinline__ uint32_t pair_of(float a, float b) {
    if (DT == BD_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *(const uint32_t *)&h;
    }
    const __half2 h = __floats2half2_rn(a, b);
    return *(const uint32_t *)&h;
}
template <int DT, bool VEC>
__device__ __forceinline__ void store8(uint8_t *p, int e, int step, int dim, const float (&v)[8]) {
    constexpr int EB = Loader<DT>::kElemBytes;
    if (VEC) {
        if (e >= dim) return;
        uint4 *dst = (uint4 *)(p + (int64_t)e * EB);
        if (DT == BD_F32) {
            dst[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            dst[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
        } else {
            dst[0] = make_uint4(pair_of<DT>(v[0], v[1]), pair_of<DT>(v[2], v[3]), pair_of<DT>(v[4], v[5]), pair_of<DT>(v[6], v[7]));
        }
    } else {
#pragma unroll
        for (int q = 0; q < 8; q++) {
            const int at = e + q * step;
            if (at >= dim) continue;
            uint8_t *dst = p + (int64_t)at * EB;
            if (DT == BD_F32) *(float *)dst = v[q];
            else *(uint16_t *)dst = (uint16_t)pair_of<DT>(v[q], 0.0f);
        }
    }
}

// Where element e of the row lies in the shared row buffer: 16-byte pieces, those of a block permuted so that eight threads that
// read the same piece of neighbouring blocks meet eight different groups of banks.
template <int DT>
__device__ __forceinline__ int place(int e) {
    constexpr int EB = Loader<DT>::kElemBytes, kPieces = 2 * EB, kPer = 16 / EB;   // pieces of a block, elements of a piece
    const int b = e / kBlock, p = e % kBlock / kPer;
    const int s = EB == 4 ? p ^ (b & 7) : p ^ ((b >> 1) & 3);
    return (b * kPieces + s) * 16 + e % kPer * EB;
}

template <int DT, int VPT, bool QUANT, bool VEC>
__global__ void __launch_bounds__(kMaxThreads, QUANT && DT == BD_BF16 ? 2 : VPT == 4 || QUANT ? 1 : VPT == 2 ? 2 : 3) residual_norm_kernel(const __grid_constant__ Args a) {
    __shared__ __align__(8) float part[2][64];                    // sums of 32 pieces
    __shared__ SmemTables tab;
    extern __shared__ __align__(16) uint8_t row_buffer[];         // QUANT: [row groups] rows of dim elements
    if (QUANT) load_tables(tab);
    const int rt = a.row_threads, group = threadIdx.x / rt, t = threadIdx.x % rt, lane = threadIdx.x % 32;
    const int warps = rt / 32;
    const float inv = 1.0f / (float)a.dim;
    int turn = 0;
    // OWN: a thread has the 32 neighbours of one block and quantises them from its registers; otherwise the row goes through shared memory first
    constexpr bool OWN = QUANT && VEC && VPT == 4;
    // Sum over the row of the pieces' sums: a binary tree over the pieces' numbers, lowest bit first, whichever threads have them, so that a row of
    // aligned operands has the same sums in every layout, stored or quantised, and among any number of rows.  The warps' sums of 32 pieces
    // meet in `part`, whose two halves take turns, so one barrier a sum is enough.  (Rows that share a CTA have one warp each.)
    auto row_sum = [&](float (&s)[VPT]) {
        if (OWN) {                                                // pieces 4 t .. 4 t + 3: eight lanes have 32 of them
            float v = __fadd_rn(__fadd_rn(s[0], s[VPT > 1 ? 1 : 0]), __fadd_rn(s[VPT > 2 ? 2 : 0], s[VPT > 3 ? 3 : 0]));
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
            if (warps == 1) {
                v += __shfl_xor_sync(0xffffffffu, v, 8);
                return v + __shfl_xor_sync(0xffffffffu, v, 16);
            }
            turn ^= 1;
            if (lane % 8 == 0) part[turn][t / 8] = v;
        } else {                                                  // piece v rt + t: a warp has 32 neighbouring ones of each v
            // (lanes of one bit go on with one v, those of the other bit with the other: in the end lane v has that v's sum)
            float v = s[0];
            if (VPT > 1) v = (lane & 1 ? s[VPT > 1 ? 1 : 0] : s[0]) + __shfl_xor_sync(0xffffffffu, lane & 1 ? s[0] : s[VPT > 1 ? 1 : 0], 1);
            if (VPT > 2) {
                const float hi = (lane & 1 ? s[VPT > 2 ? 3 : 0] : s[VPT > 2 ? 2 : 0]) + __shfl_xor_sync(0xffffffffu, lane & 1 ? s[VPT > 2 ? 2 : 0] : s[VPT > 2 ? 3 : 0], 1);
                v = (lane & 2 ? hi : v) + __shfl_xor_sync(0xffffffffu, lane & 2 ? v : hi, 2);
            }
#pragma unroll
            for (int d = VPT; d < 32; d <<= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
            if (warps == 1) {
#pragma unroll
                for (int d = 1; d < VPT; d <<= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
                return v;
            }
            turn ^= 1;
            if (lane < VPT) part[turn][lane * warps + t / 32] = v;
        }
        __syncthreads();
        const int sums = OWN ? 4 * warps : VPT * warps;
        const float2 two = *(const float2 *)&part[turn][2 * lane];
        float v = (2 * lane < sums ? two.x : 0.0f) + (2 * lane + 1 < sums ? two.y : 0.0f);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        return v;
    };
    // first element of piece v; the others follow, or are rt apart
    auto elem = [&](int v) { return OWN ? (t * 4 + v) * 8 : VEC ? (v * rt + t) * 8 : v * 8 * rt + t; };
    auto normalise = [&](float (&x)[VPT][8], const uint8_t *w, const uint8_t *b) {
        // (products that a sum follows are rounded by themselves: no layout's code has them in one operation where another's has two)
        float s[VPT];
        if (a.layer) {
#pragma unroll
            for (int v = 0; v < VPT; v++) {
                s[v] = x[v][0];
#pragma unroll
                for (int q = 1; q < 8; q++) s[v] += x[v][q];      // (elements behind the row are zeros)
            }
            const float mean = __fmul_rn(row_sum(s), inv);
#pragma unroll
            for (int v = 0; v < VPT; v++)
#pragma unroll
                for (int q = 0; q < 8; q++) x[v][q] = (VEC ? elem(v) : elem(v) + q * rt) < a.dim ? x[v][q] - mean : 0.0f;
        }
#pragma unroll
        for (int v = 0; v < VPT; v++) {
            s[v] = 0.0f;
#pragma unroll
            for (int q = 0; q < 8; q++) s[v] = fmaf(x[v][q], x[v][q], s[v]);
        }
        const float f = rsqrtf(fmaf(row_sum(s), inv, a.eps));
#pragma unroll
        for (int v = 0; v < VPT; v++) {
            float g[8];
            load8<DT, VEC>(w, elem(v), rt, a.dim, g);
#pragma unroll
            for (int q = 0; q < 8; q++) x[v][q] = __fmul_rn(x[v][q] * f, g[q] + a.offset);
            if (b) {
                load8<DT, VEC>(b, elem(v), rt, a.dim, g);
#pragma unroll
                for (int q = 0; q < 8; q++) x[v][q] += g[q];
            }
        }
    };
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int EB = Loader<DT>::kElemBytes;
    // Row numbers are unsigned: the last round's first row may lie a step (up to 9472 rows) behind the last of 2^31 - 1.
    const uint32_t rows = (uint32_t)a.rows, total = QUANT ? (uint32_t)row_tiles(a.q.rows) * kRowTile : rows;
    const int kgs = QUANT ? (int)k_groups(a.q.K) : 0;
    // The next round's rows are on their way while this one's are worked on (AHEAD: whole pieces; single elements would cost too many
    // registers): with the loads of a row in front of its own reductions, memory idles while a CTA reduces.
    constexpr bool AHEAD = VEC && !QUANT;
    Piece<DT, VEC> ny[AHEAD ? VPT : 1], nr[AHEAD ? VPT : 1];
    auto fetch = [&](uint32_t r) {
        if (AHEAD && r < rows) {
#pragma unroll
            for (int v = 0; v < (AHEAD ? VPT : 1); v++) {
                ny[v].load(a.y + (int64_t)r * a.ldy * EB, elem(v), rt, a.dim);
                if (a.residual) nr[v].load(a.residual + (int64_t)r * a.ldr * EB, elem(v), rt, a.dim);
            }
        }
    };
    const uint32_t step = gridDim.x * (uint32_t)a.row_groups;
    fetch(blockIdx.x * a.row_groups + group);
    // every thread of the CTA goes through the same number of rounds (barriers inside); a group behind the last row only keeps step
    for (uint32_t base = blockIdx.x * (uint32_t)a.row_groups; base < total; base += step) {
        const uint32_t r = base + (uint32_t)group;
        const bool there = r < rows;
        float x[VPT][8], g[8];
        Piece<DT, VEC> res[AHEAD ? VPT : 1];
#pragma unroll
        for (int v = 0; v < VPT; v++) {
            if (there) {
                if (AHEAD) ny[AHEAD ? v : 0].values(x[v]);
                else load8<DT, VEC>(a.y + (int64_t)r * a.ldy * EB, elem(v), rt, a.dim, x[v]);
                if (AHEAD) res[AHEAD ? v : 0] = nr[AHEAD ? v : 0];
            } else {
#pragma unroll
                for (int q = 0; q < 8; q++) x[v][q] = 0.0f;
            }
        }
        if (base + step < total) fetch(r + step);
        if (a.post_weight) normalise(x, a.post_weight, a.post_bias);
        if (there) {
            if (a.gate || a.residual) {
                const float one = a.gate && a.gate_col == 0 ? 1.0f : 0.0f;
                float row_gate = a.scale;
                if (one != 0.0f) {
                    const uint8_t *p = a.gate + (int64_t)r * a.gate_row * EB;
                    row_gate *= __uint_as_float(Loader<DT>::one(p));
                }
#pragma unroll
                for (int v = 0; v < VPT; v++) {
                    if (a.gate && a.gate_col) {
                        load8<DT, VEC>(a.gate + (int64_t)r * a.gate_row * EB, elem(v), rt, a.dim, g);
#pragma unroll
                        for (int q = 0; q < 8; q++) x[v][q] *= g[q];
                    }
#pragma unroll
                    for (int q = 0; q < 8; q++) g[q] = 0.0f;
                    if (a.residual) {
                        if (AHEAD) res[AHEAD ? v : 0].values(g);
                        else load8<DT, VEC>(a.residual + (int64_t)r * a.ldr * EB, elem(v), rt, a.dim, g);
                    }
#pragma unroll
                    for (int q = 0; q < 8; q++) x[v][q] = fmaf(row_gate, x[v][q], g[q]);
                }
            } else if (a.scale != 1.0f) {
#pragma unroll
                for (int v = 0; v < VPT; v++)
#pragma unroll
                    for (int q = 0; q < 8; q++) x[v][q] *= a.scale;
            }
            if (a.h) {
#pragma unroll
                for (int v = 0; v < VPT; v++) store8<DT, VEC>(a.h + (int64_t)r * a.ldh * EB, elem(v), rt, a.dim, x[v]);
            }
        }
        if (!QUANT && !a.n) continue;
        normalise(x, a.weight, a.bias);
        if (!QUANT) {
            if (there) {
#pragma unroll
                for (int v = 0; v < VPT; v++) store8<DT, VEC>(a.n + (int64_t)r * a.ldn * EB, elem(v), rt, a.dim, x[v]);
            }
            continue;
        }
        uint8_t *row = row_buffer + group * a.dim * EB;
        if (!OWN) {
#pragma unroll
            for (int v = 0; v < VPT; v++) {
                if (VEC) {                                            // eight neighbours: one piece of 16 bytes, fp32 two
                    if (elem(v) < a.dim) {
                        if (DT == BD_F32) {
                            *(uint4 *)(row + place<DT>(elem(v))) = make_uint4(__float_as_uint(x[v][0]), __float_as_uint(x[v][1]), __float_as_uint(x[v][2]), __float_as_uint(x[v][3]));
                            *(uint4 *)(row + place<DT>(elem(v) + 4)) = make_uint4(__float_as_uint(x[v][4]), __float_as_uint(x[v][5]), __float_as_uint(x[v][6]), __float_as_uint(x[v][7]));
                        } else {
                            *(uint4 *)(row + place<DT>(elem(v))) = make_uint4(pair_of<DT>(x[v][0], x[v][1]), pair_of<DT>(x[v][2], x[v][3]), pair_of<DT>(x[v][4], x[v][5]), pair_of<DT>(x[v][6], x[v][7]));
                        }
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 8; q++)
                        if (elem(v) + q * rt < a.dim) {
                            if (DT == BD_F32) *(float *)(row + place<DT>(elem(v) + q * rt)) = x[v][q];
                            else *(uint16_t *)(row + place<DT>(elem(v) + q * rt)) = (uint16_t)pair_of<DT>(x[v][q], 0.0f);
                        }
                }
            }
            if (warps == 1) __syncwarp();
            else __syncthreads();
        }
        const int nb = a.dim / kBlock;
        for (int b0 = 0; b0 < kgs * kBlocksPerAtom; b0 += rt) {   // (whole quads of lanes: rt is a multiple of 32)
            const int b = b0 + t;
            BlockResult res;
            res.id = 0; res.scale = 0;
            if (there && b < nb) {
                uint32_t unused[8];
                if (DT == BD_BF16) {
                    uint32_t pairs[16];
#pragma unroll
                    for (int p = 0; p < 4; p++) {
                        if (OWN) {
#pragma unroll
                            for (int q = 0; q < 4; q++) pairs[4 * p + q] = pair_of<DT>(x[OWN ? p : 0][2 * q], x[OWN ? p : 0][2 * q + 1]);
                        } else {
                            const uint4 u = *(const uint4 *)(row + place<DT>(b * kBlock + 8 * p));
                            pairs[4 * p] = u.x; pairs[4 * p + 1] = u.y; pairs[4 * p + 2] = u.z; pairs[4 * p + 3] = u.w;
                        }
                    }
                    quantize_bf16_block<false>(pairs, tab, res, unused);
                } else {
                    uint32_t bits[32];
                    if (OWN) {
#pragma unroll
                        for (int k = 0; k < 32; k++) {
                            const float v = x[OWN ? k / 8 : 0][k % 8];
                            bits[k] = __float_as_uint(DT == BD_F16 ? __half2float(__float2half_rn(v)) : v);
                        }
                    }
#pragma unroll
                    for (int p = 0; p < (OWN ? 0 : 2 * EB); p++) {
                        const uint4 u = *(const uint4 *)(row + place<DT>(b * kBlock + 16 / EB * p));
                        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int q = 0; q < 4; q++) {
                            if (DT == BD_F32) {
                                bits[4 * p + q] = w[q];
                            } else {
                                const float2 f = __half22float2(*(const __half2 *)&w[q]);
                                bits[(8 * p + 2 * q) % 32] = __float_as_uint(f.x);
                                bits[(8 * p + 2 * q + 1) % 32] = __float_as_uint(f.y);
                            }
                        }
                    }
                    bool nonfinite;
                    quantize_two_stage_f32<false>(bits, tab, res, unused, nonfinite);
                    if (nonfinite) atomicOr(&g_status_word, kStatusNonfinite);
                }
                *(uint4 *)(a.q.codes + (int64_t)r * a.q.ldc + (int64_t)b * 16) = make_uint4(res.words[0], res.words[1], res.words[2], res.words[3]);
            }
            // four neighbouring lanes' scale bytes and id nibbles go out together; padding of the atoms as zeros
            uint32_t sc = res.scale << (8 * (t & 3)), idn = res.id << (4 * (t & 3));
            sc |= __shfl_xor_sync(0xffffffffu, sc, 1);
            idn |= __shfl_xor_sync(0xffffffffu, idn, 1);
            sc |= __shfl_xor_sync(0xffffffffu, sc, 2);
            idn |= __shfl_xor_sync(0xffffffffu, idn, 2);
            if ((t & 3) == 0 && b < kgs * kBlocksPerAtom && r < total) {
                *(uint32_t *)(a.q.scales + scale_offset(a.q.rows, r, b)) = sc;
                *(uint16_t *)(a.q.ids + id_byte_offset(a.q.rows, r, b)) = (uint16_t)idn;
            }
        }
        if (OWN || warps == 1) __syncwarp();
        else __syncthreads();                                     // the buffer is the next round's
    }
}

}  // namespace nm
}  // namespace bd
