// The experts' gated products of a mixture-of-experts block, in DialectFP4:
//     y_t = sum_j w_tj * D_e q(act(G_e q(x_t)) * (U_e q(x_t))),   e = the j-th expert of token t,
// q the online two-stage quantisation, G, U, D stored in DialectFP4.  Four launches:
//   spread    quantises each token once and writes its operand bytes to the rows of its experts (each expert's rows begin at a multiple of
//             128, the rows of a scale atom);
//   product   gate and up rows of all experts against those rows; the epilogue forms act(g) * u and requantises it (GATED);
//   product   the down rows against the result: the experts' parts, in fp32 whatever type their sum is rounded to (rounded to bf16 they
//             take the result's error from 0.0017 to 0.0024; they cost 60 -> 60, 104 -> 104, 148 -> 160 and 2240 -> 2250 us a call for 16
//             tokens of 64 experts and the last three cases below);
//   combine   the weighted sum of a token's rows, in the order of its experts (fp32, the same in every run).
//
// The products are the tile of gemm_tc.cuh (256 weight rows x up to 256 tokens per pair of CTAs, weights expanded into tensor memory, one
// block-scaled MMA per block of 32) under a schedule that each CTA works out from the experts' counts, which live on the
// device: item = (expert, 256 weight rows, up to 256 of its tokens), clusters take items in turn.  The MMA is as wide as the item has
// tokens (rounded up to 16), so a decode step, where an expert has a few tokens, pays for the weights' way through the SM and
// little else.  The gate and up rows of 32 channels are neighbours (rows 64 j + i and 64 j + 32 + i): they meet in the warps of
// one CTA, and 32 channels are one block of the next product's operand.
//
// Bound: few tokens per expert, some 20 us of launches and first k-steps, the weights' bytes (5.9 TB/s with 1/8 of the MMAs and of the
// expansion) and the part of the expansion that does not hide under them (a tenth); many tokens, the block-scaled MMA at the clock that the
// power cap leaves.  Whole calls from a graph, us: 29, 105, 162 and 2280 for the cases below.  Measured (B200; first + second product, us, cold):
//     1 token, 64 experts, 8 a token, 2048 -> 1024          17.9 + 13.3    27.5 MB: latency of 8 and 4 k-steps behind a launch
//     64 tokens, 128 experts, 8, 2048 -> 1024               67 + 40        434 MB: 4.3 and 3.6 TB/s
//     1500 tokens, 64 experts, 6, 2048 -> 1408 (f16)        93 + 51        156 GFLOP
//     8192 tokens, 8 experts, 2, 4096 -> 14336              1535 + 667     5.77 TFLOP: 2.5 and 2.9 PFLOP/s
#pragma once
#include "bd_common.cuh"
#include "gemm_tc.cuh"
#include "ptx_sm100.cuh"
#include "quantize.cuh"

namespace bd {
namespace ex {

using namespace tc;

constexpr int kMaxExperts = 512;
constexpr int kBoxes = 5;                    // tensor maps of the token operand: 8, 16, 32, 64, 128 rows per CTA
constexpr int kRowAlign = 128;

// Most rows that the experts' segments can take: every expert's rows are rounded up to 128.
inline int64_t padded_rows(int64_t assignments, int64_t experts) {
    const int64_t used = experts < assignments ? experts : assignments;
    return (assignments + (kRowAlign - 1) * used) / kRowAlign * kRowAlign;
}
// Bytes between the rows of an operand that a product reads: whole k-groups (the part behind K holds zeros).
__host__ __device__ inline int64_t row_pitch(int64_t K) { return (K + 127) / 128 * 128; }

struct Experts {                             // what the kernels know of the plan
    const int32_t *count, *start;
    int experts, rows, tokens;               // rows: of the padded operand; tokens: of the call, more than which no expert has
};
struct Maps {
    CUtensorMap x[kBoxes], codes, ids, sfw, sfx, y, y_rest;           // y: boxes of 32 rows, y_rest: of 8
};
struct Product {
    int w_pairs, row_tiles, k_groups, clusters;
    int w_first, col0, cols;                 // down product: the first of the pass's 256-row tiles, its first column and number of columns
    int live_k;                              // GATED: blocks of the result (inter / 32)
    uint8_t *h;                              // GATED: operand bytes [rows][row_pitch(inter)] and scale atoms of the result
    uint8_t *h_scales;
    int64_t h_pitch;
    int gelu;
};

// A k-step is 256 elements of K, two k-groups.  The hand-overs of a k-step (a barrier wait, an election, a copy instruction: some 70 ns
// each for the one thread that does it) set the pace of the narrow items and much of the wide ones', whatever a step holds; with
// steps of 128 they took 0.33 to 0.4 us each.
constexpr int kStep = 2;                     // k-groups of a k-step
constexpr int kGroupBytes = 128;             // operand bytes of a row and k-group
constexpr int kCodeBytes = 128 * kStep * 64; // packed codes of 128 weight rows

// TOK: most tokens of an item.  256: an accumulator of 256 columns, room for three decoded k-steps behind it.  128, where experts have few
// tokens: an accumulator of 128 columns, which items of up to 64 tokens use half by half in turn, so that the next item's products run
// while one is read out; five decoded k-steps, so that a decode group does not wait for the products of its last one (with three:
// 1190 cycles a k-step for a few tokens, 970 of 3490 of a group's waiting; now 1120); smaller token stages and a fourth decode group.
template <bool GATED, int TOK>
struct Layout {
    static constexpr int kSlots = TOK == 256 ? 1 : 2;            // accumulators in turn
    // k-steps on the way to the MMA: the token tile and scales of one in shared memory, its decoded weights in tensor memory (64 columns)
    static constexpr int kBufs = TOK == 256 ? 3 : 5;
    // Warps: four for control (token producer, MMA issuer, code producer, one idle), the decode groups, two epilogue halves.  Each is a
    // warpgroup, since registers are handed from one to the other: at launch every thread has kLaunchRegs.
    static constexpr int kGroups = TOK == 256 ? 3 : 4;
    static constexpr int kDecode0 = 4, kEpilogue0 = kDecode0 + 4 * kGroups, kThreads = 32 * (kEpilogue0 + kEpilogueWarps);
    static constexpr int kLaunchRegs = TOK == 256 ? 80 : 72, kControlRegs = 40, kDecodeRegs = 56, kEpilogueRegs = TOK == 256 ? 136 : 120;
    static_assert(128 * kControlRegs + 128 * kGroups * kDecodeRegs + 32 * kEpilogueWarps * kEpilogueRegs <= kLaunchRegs * kThreads, "more registers than the launch brings");
    // Stages of packed codes, each always used by the same decode group: copies land out of order, and a group that came to a stage before
    // the contents in front of its own had landed would take the barrier's last-but-one phase for its own (a barrier tells a phase from the
    // next, not from the one after that).  The ring of k-steps above needs no such rule, since its MMAs complete in order.
    static constexpr int kCS = kGroups;
    static_assert(kCS % kGroups == 0, "a stage belongs to one group");
    static constexpr int kXBytes = kStep * (TOK / 2) * kGroupBytes;
    static constexpr int kSfxBytes = kStep * (TOK / 128) * kScaleAtomBytes;
    static constexpr int kStage = 8192;                          // epilogue staging of a warp: two 32 x 32 tiles of fp32
    static constexpr int x = 0;
    static constexpr int codes = x + kBufs * kXBytes;
    static constexpr int sfw = codes + kCS * kCodeBytes;
    static constexpr int sfx = sfw + kBufs * kStep * kScaleAtomBytes;
    static constexpr int ids = sfx + kBufs * kSfxBytes;
    static constexpr int bars = ids + kCS * kStep * kIdAtomBytes;
    static constexpr int words = bars + 256;
    static constexpr int seen = words + 16;                      // a word per decode warp
    static constexpr int luts = words + 80;
    static_assert(16 + 4 * 4 * kGroups <= 80, "words");
    static constexpr int qtab = luts + 128;
    static constexpr int first = (qtab + (int)sizeof(SmemTables) + 15) / 16 * 16;   // first item of each expert
    static constexpr int where = first + 4 * (kMaxExperts + 4);
    static constexpr int out = (where + 4 * kMaxExperts + 1023) / 1024 * 1024;
    static constexpr int total = out + kEpilogueWarps * kStage + 1024 /* alignment slack */;
    static_assert((2 * kBufs + 2 * kCS + 2 * kSlots) * 8 <= 256, "barrier area too small");
    static_assert(total <= 227 * 1024, "shared memory budget");
    // tensor memory columns: accumulators, decoded weights, scales of the weights and of the tokens (per k-group 4, and 4 per 128 tokens)
    static constexpr int kColA = TOK, kColSfW = kColA + 64 * kBufs, kColSfX = kColSfW + 4 * kStep;
    static_assert(kColSfX + kStep * 4 * (TOK / 128) <= 512, "tensor memory budget");
};

struct Item {
    int expert, w_pair;
    int row0;                                // first row of the token operand, a multiple of 128
    int live;                                // rows of this item that are tokens
    int n;                                   // the N of the MMA: live rounded up to 16
    int box;                                 // tensor map of the token operand: 8 << box rows per CTA
};
// Items of cluster c: c, c + clusters, ...; numbered expert by expert, then weight rows, the token tile running fastest.
template <int TOK>
struct Walk {
    const int *first;                        // items before each expert's, [experts + 1]
    const uint32_t *where;                   // an expert's first row / 128, and (low byte) the tokens of its last tile - 1
    int w_first, w_pairs, experts, clusters, c, e;
    __device__ bool operator()(int i, Item &t) {
        const int item = i * clusters + c;
        if (item >= first[experts]) return false;
        while (item >= first[e + 1]) e++;
        const int tiles = (first[e + 1] - first[e]) / w_pairs, in = item - first[e], tt = in % tiles;
        const uint32_t w = where[e];
        t.expert = e;
        t.w_pair = w_first + in / tiles;
        t.row0 = (int)(w >> 8) * kRowAlign + tt * TOK;
        t.live = tt + 1 < tiles ? TOK : (int)(w & 255u) + 1;
        t.n = (t.live + 15) / 16 * 16;
        t.box = t.n <= 16 ? 0 : 28 - __clz(t.n - 1);               // 8 << box >= n / 2
        return true;
    }
};

__device__ __forceinline__ float gated(float g, float u, int gelu) {
    // act(g) = g / (1 + exp(-a)), a = g (silu) or 2 sqrt(2 / pi) (g + 0.044715 g^3) (gelu in its tanh form), with e = exp(-|a|) <= 1: the
    // divisor lies between 1 and 2, where the fast division is within two steps (it gives 0 for divisors above 2^126).  The fast exponential is
    // off by up to 2 + 1.2 |a| steps, which counts where a < 0; expf costs 2 to 5 % of a call (1500 tokens of 64 experts: 160 -> 168 us).
    const float a = gelu ? 1.5957691216057308f * fmaf(0.044715f * g * g, g, g) : g;
    const float e = __expf(-fabsf(a));
    return g * __fdividef(a < 0.0f ? e : 1.0f, 1.0f + e) * u;
}

template <int N>
__device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// TMA load whose completion is counted on a barrier of the pair's leader CTA.
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

__device__ __forceinline__ void store_box(const CUtensorMap *map, int x, int y, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}

__device__ __forceinline__ int load_relaxed(const int32_t *p) {
    int v;
    asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

template <bool GATED, int TOK>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__((Layout<GATED, TOK>::kThreads), 1)
expert_product_kernel(const __grid_constant__ Maps maps, const Experts ex, const Product p) {
    using L = Layout<GATED, TOK>;
    constexpr int kCS = L::kCS, kSlots = L::kSlots, kBufs = L::kBufs, kDecode0 = L::kDecode0, kEpilogue0 = L::kEpilogue0, kGroups = L::kGroups;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    auto x_tile = [&](int s) { return base + L::x + (uint32_t)s * L::kXBytes; };
    auto code_tile = [&](int s) { return base + L::codes + (uint32_t)s * kCodeBytes; };
    auto sfw_tile = [&](int s) { return base + L::sfw + (uint32_t)s * (kStep * kScaleAtomBytes); };
    auto sfx_tile = [&](int s) { return base + L::sfx + (uint32_t)s * L::kSfxBytes; };
    auto id_tile = [&](int s) { return base + L::ids + (uint32_t)s * (kStep * kIdAtomBytes); };
    const uint32_t bars = base + L::bars;
    // One pair of barriers per k-step, for the token tile and the decoded weights together: the issuing warp's waits, probes and commits are
    // what a narrow k-step takes longest for.
    auto full = [&](int s) { return bars + 8u * s; };                             // leader: tile + scales landed, weights written, both CTAs
    auto empty = [&](int s) { return bars + 8u * (kBufs + s); };                  // both: the MMAs of the k-step have completed
    auto c_full = [&](int s) { return bars + 8u * (2 * kBufs + s); };             // local: codes + ids landed
    auto c_empty = [&](int s) { return bars + 8u * (2 * kBufs + kCS + s); };      // local: codes read by the decode group
    auto d_full = [&](int d) { return bars + 8u * (2 * kBufs + 2 * kCS + d); };             // both: accumulator complete
    auto d_empty = [&](int d) { return bars + 8u * (2 * kBufs + 2 * kCS + kSlots + d); };   // leader: accumulator read out
    volatile uint32_t *const shared_words = (volatile uint32_t *)(base_ptr + L::words);
    volatile uint32_t *const tmem_slot = shared_words;
    volatile uint32_t *const abort_flag = shared_words + 1;
    uint32_t *const luts = (uint32_t *)(base_ptr + L::luts);
    int *const first = (int *)(base_ptr + L::first);
    uint32_t *const where = (uint32_t *)(base_ptr + L::where);

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_ctarank();
    const int cluster = blockIdx.x / 2;

    if (threadIdx.x == 0) {
        abort_flag[0] = 0;
        abort_flag[1] = 0;                                        // set once the previous kernel has completed
        abort_flag[2] = g_debug_spin_limit ? g_debug_spin_limit : kSpinLimit;
        for (int s = 0; s < kBufs; s++) {
            mbar_init(full(s), 3);                                // the leader's token producer, and a decode group of each CTA
            mbar_init(empty(s), 1);
        }
        for (int s = 0; s < kCS; s++) {
            mbar_init(c_full(s), 1);
            mbar_init(c_empty(s), 4);                             // one arrival per warp of the decode group
        }
        for (int d = 0; d < kSlots; d++) {
            mbar_init(d_full(d), 1);
            mbar_init(d_empty(d), 2 * kEpilogueWarps);            // the epilogue warps of both CTAs
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < 32)
        luts[threadIdx.x] = threadIdx.x < 16 ? c_tables.e4m3_lo[threadIdx.x] : c_tables.e4m3_hi[threadIdx.x - 16];
    SmemTables &qtab = *(SmemTables *)(base_ptr + L::qtab);
    if (GATED) load_tables(qtab);                                 // (ends with __syncthreads())
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32((const void *)tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();                                           // both CTAs: running, barriers initialised, TMEM allocated
    tcgen05_fence_after();
    // The schedule: items of the experts before each one, by a scan in the leader's first warp, which writes it to both CTAs: they hand
    // over to one another item by item, so they must go by the same numbers whatever happens to the plan meanwhile.  The plan and the weights
    // are older than the kernel in front, which starts this one only behind its own wait for all that came before: they are read without
    // waiting for it (the plan past the first-level cache, whose lines may be older), and codes are loaded and expanded while it ends.
    // Numbers that cannot be (a plan overwritten by the caller) leave the expert out and are told: nothing is addressed by them.
    if (warp == 0 && rank == 0) {
        const uint32_t to_first = map_to_cta(smem_u32(first), 1), to_where = map_to_cta(smem_u32(where), 1);
        auto share = [](uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); };
        int before = 0;
        for (int e0 = 0; e0 < ex.experts; e0 += 32) {
            const int e = e0 + lane;
            int cnt = 0, start = 0;
            if (e < ex.experts) {
                cnt = load_relaxed(ex.count + e);
                start = load_relaxed(ex.start + e);
                if (cnt < 0 || start < 0 || start % kRowAlign || cnt > ex.tokens || cnt > ex.rows || start > ex.rows - cnt) {
                    cnt = start = 0;
                    atomicOr(&g_status_word, kStatusIndex);
                }
            }
            const int items = (cnt + TOK - 1) / TOK * p.w_pairs;
            int incl = items;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += up;
            }
            if (e < ex.experts) {
                const uint32_t w = (uint32_t)(start / kRowAlign) << 8 | (uint32_t)((cnt + TOK - 1) % TOK);
                first[e] = before + incl - items;
                where[e] = w;
                share(to_first + 4u * e, (uint32_t)(before + incl - items));
                share(to_where + 4u * e, w);
            }
            before += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) {
            first[ex.experts] = before;
            share(to_first + 4u * (uint32_t)ex.experts, (uint32_t)before);
        }
        __syncwarp();
    }
    __syncthreads();
    cluster_sync_all();
    const uint32_t tmem = *tmem_slot;
    const int steps = (p.k_groups + kStep - 1) / kStep;
    auto accumulator = [](const Item &t, int slot) { return kSlots == 2 && t.n <= 64 ? 64u * (uint32_t)slot : 0u; };
    Walk<TOK> next{first, where, GATED ? 0 : p.w_first, p.w_pairs, ex.experts, p.clusters, cluster, 0};
    Item t;

    if (warp < kDecode0) {
        registers_down<L::kControlRegs>();
        if (warp == 0) {
            // ---- TMA producer of the token tile and the scale atoms; the one warp that reads what the kernel in front wrote ----
            asm volatile("griddepcontrol.wait;" ::: "memory");
            asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (behind the wait: the next kernel takes it that all before this one is done)
            if (lane == 0) abort_flag[1] = 1;                     // from here on every bounded wait counts its polls
            int s = 0;
            uint32_t ph = 1;
            const uint32_t full_leader = map_to_cta(full(0), 0);
            for (int i = 0; next(i, t); i++) {
                // each CTA holds half of the MMA's tokens (and, where the box is higher, rows that are not looked at)
                const int t0 = t.row0 + (int)rank * (t.n / 2), sf_z = t.expert * p.k_groups;
                const uint32_t tx_pair = 2u * (kStep * (8u << t.box) * kGroupBytes + kStep * kScaleAtomBytes + L::kSfxBytes);
                for (int k = 0; k < steps; k++) {
                    if (!mbar_wait_warp(empty(s), ph, abort_flag)) break;
                    const uint32_t fb = full_leader + 8u * (uint32_t)s;
                    if (elect_one()) {
                        if (rank == 0) mbar_expect_tx(full(s), tx_pair);
                        tma_load_3d_pair(x_tile(s), &maps.x[t.box], 0, t0, kStep * k, fb);
                        tma_load_3d_pair(sfw_tile(s), &maps.sfw, 0, t.w_pair * 2 + (int)rank, sf_z + kStep * k, fb);
                        tma_load_3d_pair(sfx_tile(s), &maps.sfx, 0, t.row0 / kRowAlign, kStep * k, fb);
                    }
                    __syncwarp();
                    if (++s == kBufs) { s = 0; ph ^= 1u; }
                }
                if (*abort_flag) break;
            }
        } else if (warp == 2) {
            // ---- TMA producer of this CTA's packed codes and ids ----
            int s = 0;
            uint32_t ph = 1;
            const bool skip_first = g_debug_skip_first_code_stage != 0;   // test hook: see bd_debug_fault
            for (int i = 0; next(i, t); i++) {
                const int my_tile = t.w_pair * 2 + (int)rank, id_z = t.expert * p.k_groups;
                for (int k = 0; k < steps; k++) {
                    if (!mbar_wait_warp(c_empty(s), ph, abort_flag)) break;
                    if (elect_one() && !(skip_first && i == 0 && k == 0)) {
                        mbar_expect_tx(c_full(s), kCodeBytes + kStep * kIdAtomBytes);
                        tma_load_3d(code_tile(s), &maps.codes, k * (kStep * 64), my_tile * 128, t.expert, c_full(s));
                        tma_load_3d(id_tile(s), &maps.ids, 0, my_tile, id_z + kStep * k, c_full(s));
                    }
                    __syncwarp();
                    if (++s == kCS) { s = 0; ph ^= 1u; }
                }
                if (*abort_flag) break;
            }
        } else if (warp == 1 && rank == 0) {
            // ---- MMA issuer (leader CTA; whole warp converged, one elected lane issues) ----
            const uint32_t hi_op = desc_hi(1024, kLayoutSwizzle128), hi_sf = desc_hi(128, kLayoutNone);
            const uint32_t lo_x0 = (x_tile(0) >> 4) | 1u << 16;
            const uint32_t lo_sfw0 = sfw_tile(0) >> 4, lo_sfx0 = sfx_tile(0) >> 4;
            // (instruction descriptor: see gemm_tc.cuh; N >> 3 at bit 17 follows the item)
            const uint32_t idesc_m = 1u << 23 | (uint32_t)(256 >> 4) << 24;
            const uint32_t t_sfw = tmem + L::kColSfW, t_sfx = tmem + L::kColSfX;
            int s = 0;
            uint32_t ph = 0;
            bool ready = false, wide = false;                     // wide: the item before had both halves of the accumulator
            for (int i = 0; next(i, t); i++) {
                const uint32_t idesc0 = idesc_m | (uint32_t)(t.n >> 3) << 17, x_half = (8u << t.box) * kGroupBytes >> 4;
                const int slot = i % kSlots;
                const uint32_t t_d = tmem + accumulator(t, slot);
                if (i >= kSlots) mbar_wait_warp(d_empty(slot), (uint32_t)(i / kSlots - 1) & 1u, abort_flag);
                if (kSlots == 2 && i > 0 && (wide || t.n > 64)) mbar_wait_warp(d_empty(slot ^ 1), (uint32_t)((i - 1) / kSlots) & 1u, abort_flag);
                wide = t.n > 64;
                tcgen05_fence_after();
                for (int k = 0; k < steps; k++) {
                    // (slow path: the probe at the end of the previous k-step found the barrier open)
                    if (!ready && !mbar_wait_warp(full(s), ph, abort_flag)) break;
                    tcgen05_fence_after();
                    const uint32_t lo_sfw = lo_sfw0 + (uint32_t)s * (kStep * kScaleAtomBytes >> 4);
                    const uint32_t lo_sfx = lo_sfx0 + (uint32_t)s * (L::kSfxBytes >> 4);
                    const uint32_t lo_x = lo_x0 + (uint32_t)s * (L::kXBytes >> 4);
                    const uint32_t t_a = tmem + L::kColA + 64u * (uint32_t)s;
                    const bool both = kStep * k + 1 < p.k_groups;     // (K may end with the step's first k-group)
                    if (elect_one()) {
#pragma unroll
                        for (int h = 0; h < kStep; h++) {
                            if (h > 0 && !both) break;
                            tcgen05_cp_pair(t_sfw + 4 * h, desc_join(lo_sfw + h * (kScaleAtomBytes >> 4), hi_sf));
#pragma unroll
                            for (int q = 0; q < TOK / 128; q++)
                                tcgen05_cp_pair(t_sfx + 4 * (h * (TOK / 128) + q), desc_join(lo_sfx + (h * (TOK / 128) + q) * (kScaleAtomBytes >> 4), hi_sf));
#pragma unroll
                            for (int j = 0; j < 4; j++)
                                tcgen05_mma_mxf8_pair_atmem(t_d, t_a + 32u * h + 8u * j, desc_join(lo_x + h * x_half + 2 * j, hi_op),
                                                            idesc0 | (uint32_t)j << 4 | (uint32_t)j << 29, t_sfw + 4 * h, t_sfx + 4 * h * (TOK / 128),
                                                            h == 0 && j == 0 ? (k > 0 ? 1u : 0u) : 1u);
                        }
                        tcgen05_commit_pair(empty(s));
                    }
                    __syncwarp();
                    if (++s == kBufs) { s = 0; ph ^= 1u; }
                    // probe the next k-step's barrier now (the ring runs across items): the round trip overlaps the issue above
                    ready = __all_sync(0xffffffffu, mbar_test_wait(full(s), ph));
                }
                if (*abort_flag && elect_one()) {
                    // this CTA is aborting: tell the peer before its epilogue warps are woken by the commit below
                    asm volatile("st.shared::cluster.u32 [%0], %1;\n\tfence.acq_rel.cluster;"
                                 ::"r"(map_to_cta(smem_u32((const void *)abort_flag), 1)), "r"(1u) : "memory");
                }
                __syncwarp();
                if (elect_one()) tcgen05_commit_pair(d_full(slot));
                __syncwarp();
                if (*abort_flag) break;
            }
        }
    } else if (warp < kEpilogue0) {
        // ---- decode warps: group g takes this CTA's k-steps g, g + groups, ... (counted across items); a warp may only touch the TMEM
        // lanes 32 * (warp % 4) .. + 31, so thread `lane` of warp w owns weight row (and TMEM lane) j = 32 * (w % 4) + lane ----
        registers_down<L::kDecodeRegs>();
        const int group = (warp - kDecode0) / 4, quad = warp % 4;
        const int j = quad * 32 + lane;
        const bool group_leader = quad == 0 && lane == 0;
        const uint32_t swz = (uint32_t)j & 7u;
        const uint32_t full_leader = map_to_cta(full(0), 0);
        const uint32_t t_row = tmem + ((uint32_t)(quad * 32) << 16) + L::kColA;
        const int items = first[ex.experts];
        const int total = cluster < items ? ((items - cluster + p.clusters - 1) / p.clusters) * steps : 0;
        int s = group % kCS, b = group % kBufs;
        uint32_t s_par = 0, b_par = 1;
        static_assert(kGroups <= kCS && kGroups <= kBufs, "one wrap per step at most");
        bool dead = false;                                        // (a warp whose wait ran out keeps meeting its group at the barrier)
        for (int g = group; g < total; g += kGroups) {
            uint4 w[8];
            uint32_t ids[kStep] = {0, 0};
            if (!dead) dead = !mbar_wait_warp(c_full(s), s_par, abort_flag);
            if (!dead) {
                const uint8_t *codes = base_ptr + L::codes + s * kCodeBytes + j * 128;
#pragma unroll
                for (int h = 0; h < kStep; h++)
                    ids[h] = *(const uint16_t *)(base_ptr + L::ids + (s * kStep + h) * kIdAtomBytes + (j % 32) * 8 + (j / 32) * 2);
#pragma unroll
                for (int c = 0; c < 8; c++) w[c] = *(const uint4 *)(codes + 16 * ((uint32_t)c ^ swz));
                // The stage goes back to its producer once the loads have arrived, not only been issued: the epilogue's stores can hold them
                // up for longer than a refill takes, and then rows were seen to be decoded from the stage's next contents.  A store of
                // something made of all of them cannot leave before them, nor the hand-over before the store.
                uint32_t seen = ids[0] ^ ids[1];
#pragma unroll
                for (int c = 0; c < 8; c++) seen ^= w[c].x;
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + (uint32_t)L::seen + 4u * (uint32_t)(warp - kDecode0)), "r"(seen) : "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_local(c_empty(s));
                dead = !mbar_wait_warp(empty(b), b_par, abort_flag);
            }
            if (!dead) {
                tcgen05_fence_after();                            // the MMAs that read this buffer have completed
#pragma unroll
                for (int c = 0; c < 8; c++) {
                    const uint32_t id = (ids[c / 4] >> (4 * (c % 4))) & 15u;
                    const uint32_t lo = luts[id], hi = luts[16 + id];
                    uint32_t o[8];
                    decode_word(w[c].x, lo, hi, o[0], o[1]);
                    decode_word(w[c].y, lo, hi, o[2], o[3]);
                    decode_word(w[c].z, lo, hi, o[4], o[5]);
                    decode_word(w[c].w, lo, hi, o[6], o[7]);
                    tcgen05_st_32x32b_x8(t_row + 64u * (uint32_t)b + 8u * (uint32_t)c, o);
                }
                tcgen05_wait_st();
                tcgen05_fence_before();
            }
            asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");   // the four warps of this group are done
            if (group_leader && !dead) mbar_arrive_cluster(full_leader + 8u * b);
            __syncwarp();
            s += kGroups;
            if (s >= kCS) { s -= kCS; s_par ^= 1u; }
            b += kGroups;
            if (b >= kBufs) { b -= kBufs; b_par ^= 1u; }
        }
    } else {
        // ---- epilogue: warp w reads the TMEM lanes 32 * (w % 4) .. + 31 (weight rows) of this CTA's accumulator ----
        registers_up<L::kEpilogueRegs>();
        const int quad = warp % 4, half = (warp - kEpilogue0) / 4, slot_of_warp = warp - kEpilogue0;
        const uint32_t d_empty_leader = map_to_cta(d_empty(0), 0);
        const uint32_t stage_out = base + L::out + (uint32_t)slot_of_warp * L::kStage;
        uint8_t *const stage_ptr = base_ptr + L::out + slot_of_warp * L::kStage;
        uint32_t stage_turn = 0;
        auto staging_free = [&]() -> uint32_t {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            __syncwarp();
            stage_turn ^= 1u;
            return stage_turn * (L::kStage / 2);
        };
        for (int i = 0; next(i, t); i++) {
            const int slot = i % kSlots;
            auto release_accumulator = [&]() {
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(d_empty_leader + 8u * (uint32_t)slot);
                __syncwarp();
            };
            mbar_wait_warp(d_full(slot), (uint32_t)(i / kSlots) & 1u, abort_flag, 256);
            tcgen05_fence_after();
            const uint32_t t_base = tmem + ((uint32_t)(quad * 32) << 16) + accumulator(t, slot);
            if (GATED) {
                // Tokens 64 at a time; the two epilogue halves take turns.  The warps of quadrants 2 m and 2 m + 1 hold the gate and
                // the up rows of the same 32 channels (block 2 m of this CTA's): both store two 32 x 32 tiles of sums (element
                // (token q, row r) at q * 32 + (r ^ q): rows are written and tokens read without bank conflicts), meet, and then the
                // first finishes the first 32 tokens and the second the others, a token's block per lane.  A half's second 64 tokens
                // are fetched before the first ones are quantised: the accumulator is free while that goes on.  (Fetched at once, into
                // registers, they spilled: local memory does not fit beside this much shared memory, and the epilogue took twice as long.)
                const int groups = (t.n + 63) / 64, pair = quad / 2, which = quad & 1;
                const int b = t.w_pair * 4 + (int)rank * 2 + pair;                     // block of the result
                const bool block_ok = b < p.live_k;
                const uint32_t *const tile_g = (const uint32_t *)(base_ptr + L::out + (slot_of_warp - which) * L::kStage) + which * 1024;
                const uint32_t *const tile_u = (const uint32_t *)(base_ptr + L::out + (slot_of_warp - which + 1) * L::kStage) + which * 1024;
                uint32_t *const tile = (uint32_t *)stage_ptr;
                auto meet = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + kGroups + half * 2 + pair) : "memory"); };
                uint32_t bits[32];
                auto activate = [&]() {
                    meet();
#pragma unroll
                    for (int k = 0; k < 32; k++) {
                        bits[k] = __float_as_uint(gated(__uint_as_float(tile_g[lane * 32 + (k ^ lane)]), __uint_as_float(tile_u[lane * 32 + (k ^ lane)]), p.gelu));
                        if (k % 8 == 7) asm volatile("" ::: "memory");   // (no more than eight pairs on the way at a time: registers)
                    }
                    meet();                                       // the tiles may be written again
                };
                auto store = [&](int g) {
                    const int tok = g * 64 + which * 32 + lane, row = t.row0 + tok;
                    if (tok < t.live && b < (p.live_k + 3) / 4 * 4 && !*abort_flag) {
                        BlockResult res;
                        uint32_t o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                        res.scale = 0;
                        if (block_ok) {
                            bool nonfinite;
                            quantize_two_stage_f32<true>(bits, qtab, res, o, nonfinite);
                            if (nonfinite) atomicOr(&g_status_word, kStatusNonfinite);
                        }
                        // (blocks behind the last one, up to the k-group's four: zeros)
                        uint4 *dst = (uint4 *)(p.h + (int64_t)row * p.h_pitch + (int64_t)b * 32);
                        dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
                        dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
                        p.h_scales[((int64_t)(b / kBlocksPerAtom) * (ex.rows / kRowAlign) + row / kRowTile) * kScaleAtomBytes + (row % 32) * 16 + (row % kRowTile / 32) * 4 + b % kBlocksPerAtom] = (uint8_t)res.scale;
                    }
                    __syncwarp();                                 // (the whole warp works on tensor memory again)
                };
                if (half >= groups) {
                    release_accumulator();
                } else {
                    const bool more = TOK == 256 && half + 2 < groups;
                    auto fetch = [&](int g) {
                        uint32_t r[32];
#pragma unroll
                        for (int v = 0; v < 2; v++) {
                            tcgen05_ld_32x32b_x32(t_base + g * 64 + v * 32, r);
                            tcgen05_wait_ld();
#pragma unroll
                            for (int q = 0; q < 32; q++) tile[v * 1024 + q * 32 + (lane ^ q)] = r[q];
                        }
                    };
                    fetch(half);
                    if (!more) release_accumulator();
                    activate();
                    if (more) {
                        fetch(half + 2);
                        release_accumulator();
                    }
                    store(half);
                    if (more) {
                        activate();
                        store(half + 2);
                    }
                }
            } else {
                // Chunks of 32 tokens, fetched two at a time: the first half's warps take the larger part.  The experts' parts stay fp32 whatever
                // type the sum is rounded to; warps whose 32 weight rows are not among the pass's columns only release the accumulator.
                const int chunks = (t.n + 31) / 32, mine0 = half ? (chunks + 1) / 2 : 0;
                const int n0 = t.w_pair * 256 + (int)rank * 128 + quad * 32 - p.col0;
                const int mine = n0 < 0 || n0 >= p.cols ? 0 : half ? chunks / 2 : (chunks + 1) / 2;
                const uint32_t t_mine = t_base + mine0 * 32;
                if (mine == 0) release_accumulator();
                for (int c = 0; c < mine; c += 2) {
                    uint32_t r[2][32];
                    const bool two = c + 1 < mine;
                    tcgen05_ld_32x32b_x32(t_mine + c * 32, r[0]);
                    if (two) tcgen05_ld_32x32b_x32(t_mine + c * 32 + 32, r[1]);
                    tcgen05_wait_ld();
                    if (c + 2 >= mine) release_accumulator();
#pragma unroll
                    for (int v = 0; v < 2; v++) {
                        if (v == 1 && !two) break;
                        const uint32_t sb = staging_free();
#pragma unroll
                        for (int q = 0; q < 32; q++) *(uint32_t *)(stage_ptr + sb + q * 128 + lane * 4) = r[v][q];
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0 && !*abort_flag) {
                            const int row = (mine0 + c + v) * 32, rest = t.live - row;
                            if (rest > 24) store_box(&maps.y, n0, t.row0 + row, stage_out + sb);
                            else for (int q = 0; q < rest; q += 8) store_box(&maps.y_rest, n0, t.row0 + row + q, stage_out + sb + q * 128);
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                    }
                }
                __syncwarp();
            }
        }
        // the staging buffers must outlive the stores' reads of them; the writes themselves complete with the grid
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    }

    // After a wait ran out copies and products may be in flight still, to barriers that will not complete: they arrive within some
    // microseconds, and nothing of the pair's memory goes back before (about a millisecond).
    if (*abort_flag)
        for (int i = 0; i < 64; i++) __nanosleep(16384);
    __syncwarp();
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();                                           // the peer may still signal our barriers until here
    if (warp == 1) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Quantises the tokens and writes each to the rows of its experts: thread = (token, block of 32), four lanes a scale word.
// Bound: a launch where tokens are few (6 us for 1 token, cold), else reading x and the operand's k copies (8192 x 4096, 2 each: 29.5 us).
template <int DT>
__global__ void __launch_bounds__(256) spread_kernel(const uint8_t *__restrict__ X, int64_t ldx, int tokens, int top_k, const int32_t *__restrict__ place,
                                                     int nb, int kgroups, int rows, uint8_t *__restrict__ x8, uint8_t *__restrict__ scales, FastDiv div_row) {
    __shared__ SmemTables tab;
    load_tables(tab);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t per_row = (uint32_t)kgroups * kBlocksPerAtom, items = (uint32_t)tokens * per_row;
    for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < (items + 31u) / 32u * 32u; i += gridDim.x * 256u) {   // (whole warps)
        const uint32_t t = fast_div(i, div_row), b = i - t * per_row;
        uint32_t o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        BlockResult res;
        res.scale = 0;
        const bool valid = i < items && b < (uint32_t)nb;
        if (valid) {
            const uint8_t *src = X + ((int64_t)t * ldx + b * 32u) * Loader<DT>::kElemBytes;
            if (DT == BD_BF16) {
                uint32_t pairs[16];
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const uint4 u = __ldg((const uint4 *)src + q);
                    pairs[4 * q] = u.x; pairs[4 * q + 1] = u.y; pairs[4 * q + 2] = u.z; pairs[4 * q + 3] = u.w;
                }
                quantize_bf16_block<true>(pairs, tab, res, o);
            } else {
                uint32_t bits[32];
                bool nonfinite;
                Loader<DT>::contiguous(src, bits);
                quantize_two_stage_f32<true>(bits, tab, res, o, nonfinite);
                if (nonfinite) atomicOr(&g_status_word, kStatusNonfinite);
            }
        }
        uint32_t sc = res.scale << (8 * (b & 3u));
        sc |= __shfl_xor_sync(0xffffffffu, sc, 1);
        sc |= __shfl_xor_sync(0xffffffffu, sc, 2);
        if (i >= items) continue;
        for (int j = 0; j < top_k; j++) {
            const int row = __ldg(place + (int64_t)t * top_k + j);
            if (row < 0) continue;
            if (row >= rows) {
                atomicOr(&g_status_word, kStatusIndex);
                continue;
            }
            uint4 *dst = (uint4 *)(x8 + (int64_t)row * ((int64_t)kgroups * 128) + b * 32u);   // (zeros up to the k-group's end)
            dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
            dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
            if ((b & 3u) == 0)
                *(uint32_t *)(scales + ((int64_t)(b / 4) * (rows / kRowTile) + row / kRowTile) * kScaleAtomBytes + (row % 32) * 16 + (row % kRowTile / 32) * 4) = sc;
        }
    }
}

// y_t = sum_j w_tj * part[place_tj] in fp32, rounded once; thread = V neighbouring outputs of a token.  A token without experts gets zeros.
// Bound: memory, a launch where tokens are few.  Four outputs a thread up to two CTAs per SM (64 tokens of 128 experts: the whole call 104 us,
// with eight 106), eight beyond (512 of 64: 97 us, with four 103).
template <bool BF16, int V>
__global__ void __launch_bounds__(256) combine_kernel(const float *__restrict__ part, const int32_t *__restrict__ place, const float *__restrict__ weights,
                                                      int tokens, int top_k, int rows, int n, void *__restrict__ Y, int64_t ldy) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int per_row = n / V;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)tokens * per_row; i += (int64_t)gridDim.x * 256) {
        const int t = (int)(i / per_row), c = (int)(i - (int64_t)t * per_row) * V;
        float acc[V];
#pragma unroll
        for (int q = 0; q < V; q++) acc[q] = 0.0f;
#pragma unroll 4
        for (int j = 0; j < top_k; j++) {
            const int row = __ldg(place + (int64_t)t * top_k + j);
            if (row < 0 || row >= rows) continue;
            const float w = __ldg(weights + (int64_t)t * top_k + j);
#pragma unroll
            for (int q = 0; q < V; q += 4) {
                const float4 u = __ldcs((const float4 *)(part + (int64_t)row * n + c + q));
                acc[q] = fmaf(w, u.x, acc[q]);
                acc[q + 1] = fmaf(w, u.y, acc[q + 1]);
                acc[q + 2] = fmaf(w, u.z, acc[q + 2]);
                acc[q + 3] = fmaf(w, u.w, acc[q + 3]);
            }
        }
        if (BF16) {
            uint32_t o[V / 2];
#pragma unroll
            for (int q = 0; q < V / 2; q++) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(acc[2 * q], acc[2 * q + 1]);
                o[q] = *(const uint32_t *)&h;
            }
            uint16_t *dst = (uint16_t *)Y + (int64_t)t * ldy + c;
            if (V == 8) *(uint4 *)dst = make_uint4(o[0], o[1], o[V / 2 - 2], o[V / 2 - 1]);
            else *(uint2 *)dst = make_uint2(o[0], o[1]);
        } else {
#pragma unroll
            for (int q = 0; q < V; q += 4) *(float4 *)((float *)Y + (int64_t)t * ldy + c + q) = make_float4(acc[q], acc[q + 1], acc[q + 2], acc[q + 3]);
        }
    }
}

// The values that the second product reads, for checking: out[token][slot][inter] in fp32 (zeros where no expert serves).
__global__ void __launch_bounds__(256) inner_kernel(const uint8_t *__restrict__ h, const uint8_t *__restrict__ scales, const int32_t *__restrict__ place,
                                                    int64_t assignments, int rows, int inter, int64_t pitch, float *__restrict__ out) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int nb = inter / 32;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < assignments * nb; i += (int64_t)gridDim.x * 256) {
        const int64_t a = i / nb;
        const int b = (int)(i - a * nb), row = __ldg(place + a);
        float *dst = out + a * inter + b * 32;
        const bool there = row >= 0 && row < rows;
        const int e = there ? (int)scales[((int64_t)(b / 4) * (rows / kRowTile) + row / kRowTile) * kScaleAtomBytes + (row % 32) * 16 + (row % kRowTile / 32) * 4 + b % 4] - 127 : 0;
        for (int k = 0; k < 32; k++) {
            float v = 0.0f;
            if (there) {
                const uint32_t x = h[(int64_t)row * pitch + b * 32 + k];              // E4M3: no magnitude here is subnormal
                const uint32_t f = x >> 3 & 15u;
                if (f) v = scalbnf(1.0f + (float)(x & 7u) * 0.125f, (int)f - 7 + e);
                if (x & 0x80u) v = -v;
            }
            dst[k] = v;
        }
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------
inline bool make_map_3d(CUtensorMap *map, CUtensorMapDataType type, const void *ptr, uint64_t inner, uint64_t rows, uint64_t outer, uint64_t row_bytes,
                        uint64_t outer_bytes, uint32_t box_inner, uint32_t box_rows, uint32_t box_outer, CUtensorMapSwizzle swizzle) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {inner, rows, outer}, strides[2] = {row_bytes, outer_bytes};
    cuuint32_t box[3] = {box_inner, box_rows, box_outer}, elem[3] = {1, 1, 1};
    return fn(map, type, 3, (void *)ptr, dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool GATED, int TOK>
inline cudaError_t launch_product(const uint8_t *x8, const uint8_t *sfx, const Experts &ex, int64_t tokens, int64_t pair_items, const bd_experts *W, Product p, float *parts, cudaStream_t st) {
    using L = Layout<GATED, TOK>;
    Maps m;
    const int64_t N = W->rows, K = W->K, rtw = row_tiles(N), kg = k_groups(K), pitch = row_pitch(K), tiles_x = ex.rows / kRowAlign;
    constexpr CUtensorMapDataType kBytes = CU_TENSOR_MAP_DATA_TYPE_UINT8, kWords = CU_TENSOR_MAP_DATA_TYPE_UINT32;
    // (an item has no more tokens than the call: a small call's maps are the few that it can need)
    for (int b = 0; b < kBoxes; b++)
        if (b > 0 && (8 << b) > TOK / 2) m.x[b] = m.x[b - 1];
        else if (b > 0 && (8 << b) >= 2 * tokens) m.x[b] = m.x[b - 1];
        else if (!make_map_3d(&m.x[b], kBytes, x8, kGroupBytes, ex.rows, kg, pitch, kGroupBytes, kGroupBytes, 8u << b, kStep, CU_TENSOR_MAP_SWIZZLE_128B)) return cudaErrorInvalidValue;
    if (!make_map_3d(&m.codes, kBytes, W->codes, K / 2, N, W->experts, K / 2, (uint64_t)N * (K / 2), kStep * 64, 128, 1, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map_3d(&m.ids, kWords, W->ids, kIdAtomBytes / 4, rtw, (uint64_t)kg * W->experts, kIdAtomBytes, (uint64_t)rtw * kIdAtomBytes, kIdAtomBytes / 4, 1, kStep, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !make_map_3d(&m.sfw, kWords, W->scales, kScaleAtomBytes / 4, rtw, (uint64_t)kg * W->experts, kScaleAtomBytes, (uint64_t)rtw * kScaleAtomBytes, kScaleAtomBytes / 4, 1, kStep, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !make_map_3d(&m.sfx, kWords, sfx, kScaleAtomBytes / 4, tiles_x, kg, kScaleAtomBytes, (uint64_t)tiles_x * kScaleAtomBytes, kScaleAtomBytes / 4, TOK / 128, kStep, CU_TENSOR_MAP_SWIZZLE_NONE))
        return cudaErrorInvalidValue;
    if (!GATED) {
        if (!make_map_2d(&m.y, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, parts, p.cols, ex.rows, (uint64_t)p.cols * 4, 32, 32, CU_TENSOR_MAP_SWIZZLE_NONE) ||
            !make_map_2d(&m.y_rest, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, parts, p.cols, ex.rows, (uint64_t)p.cols * 4, 32, 8, CU_TENSOR_MAP_SWIZZLE_NONE))
            return cudaErrorInvalidValue;
    } else {
        m.y = m.y_rest = m.sfx;                                       // unused, but must be valid objects
    }
    static bool configured[tc::kMaxDevices] = {};
    const int dev = current_device();
    if (!configured[dev]) {
        cudaError_t e = cudaFuncSetAttribute(expert_product_kernel<GATED, TOK>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::total);
        if (e != cudaSuccess) return e;
        // the warpgroups trade the registers that the launch brings: with fewer, the ones that ask for more would wait for good
        cudaFuncAttributes a;
        if ((e = cudaFuncGetAttributes(&a, expert_product_kernel<GATED, TOK>)) != cudaSuccess) return e;
        if (a.numRegs < L::kLaunchRegs) return cudaErrorLaunchOutOfResources;
        configured[dev] = true;
    }
    p.w_first = GATED ? 0 : p.col0 / 256;
    p.w_pairs = (int)(((GATED ? N : (int64_t)p.col0 + p.cols) + 255) / 256) - p.w_first;
    p.row_tiles = (int)rtw;
    p.k_groups = (int)kg;
    const int resident = max_resident_clusters();
    const int64_t most = pair_items * p.w_pairs;
    p.clusters = most < resident ? (int)most : resident;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * p.clusters);
    cfg.blockDim = dim3(L::kThreads);
    cfg.dynamicSmemBytes = L::total;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, expert_product_kernel<GATED, TOK>, m, ex, p);
}

}  // namespace ex
}  // namespace bd
