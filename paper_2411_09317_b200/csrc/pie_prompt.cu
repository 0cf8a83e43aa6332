// Causal attention over whole prompts, packed one after the other (Section 2.1: the prefill stage computes all prompt tokens at
// once), on the fifth-generation tensor cores: keys and values as the projection left them, nothing cached before them.
//
// A row is a (token, query head of the KV head's group) pair, token-major.  Work item = (sequence, KV head, two tiles of 128
// consecutive rows): the two tiles take turns on the tensor core and share every K and V stage, so that one tile's softmax runs
// while the other's products do, and a stage's 64 KiB (head_dim 128) cross from L2 to the SM once per 256 rows - with one tile
// per CTA and two CTAs per SM that traffic alone, 64 bytes per clock and SM, is more than L2 delivers.
//   - The loading warp brings the Q tiles and the K and V stages (128 tokens; TMA tiles of 64 elements, 128-byte swizzle) through
//     a ring of stage buffers: K0, V0, K1, V1, ...
//   - One thread of the issuing warp issues the MMAs.  Per tile and stage: S = Q K^T (128 x 128 x D, fp32, 128 TMEM columns) and
//     O += P V (D TMEM columns) with P read from TMEM, in two halves of the stage's tokens, so that the first half's products run
//     beside the second half's exponentials (642 -> 636 us for 10007 tokens, 127 -> 124 us for the ragged prompts; in quarters, or
//     three quarters and one: 643 and 647, 125 and 126).  The order is O0 += P0 V(j), S0(j + 1), O1 += P1 V(j), S1(j + 1): tcgen05
//     MMAs of one thread complete in order, so S may follow O += P V over the same columns without a wait, and a softmax warp
//     that sees S(j + 1) knows O += P V of stage j to be complete.
//   - Eight softmax warps, four per tile, a thread per row: the 128 scores in registers, maximum (three-input), one packed
//     multiply-add per pair of elements, exponentials, packed sums, P back into TMEM over the scores.
//   - Two warps clear NaN and infinities from values that some row of the item may not see: a probability of 0 hides all else.
// A CTA per SM takes items until none is left and goes from one to the next without a break: the next item's query rows, keys and
// first scores arrive behind the last stage of the item before it.
// Bound: a stage of both tiles takes some 3300 cycles (2048 of products, as many of exponentials; a tile's chain from scores to
// scores is longer than the other tile covers) and, under load, the power limit.  Two score buffers of 64 columns per tile, which
// cut the chain, lose more: a product of 64 columns takes as long as one of 128 (782 us against 638).  One prompt of 10007 tokens,
// 32 / 8 heads of 128, bf16: 636 us, 1290 TFLOP/s (half a second of it: 750 us at 1.63 GHz); 16 ragged prompts of 12112 tokens:
// 124 us called back to back, which leaves their arrays in L2, and 149 with arrays that come from HBM; 32 of 512: 108 us (back to
// back); heads of 64, fp16, one prompt of 10007 tokens: 545 us, 566 from HBM (half a stage's products, all of its exponentials: the
// special-function unit alone takes 2048 cycles a stage, 356 us in all); 45 tokens: 7 us, most of it the host's.  Short prompts pay 1.4 us per item for the epilogue, whose
// stores take a line per lane: exchanging sectors between two lanes or four first costs as much as it saves (128 and 130 us for the
// ragged prompts, then at 129).
// Scores and sums in fp32.  P is rounded once to the 16-bit type on its way to the tensor core (a second operand with the
// rounding remainder, as the chunked kernel has for bf16, costs half as many MMAs again and buys less than the output's own
// rounding); the row's sum is of the unrounded probabilities.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstring>

#include "../../include/pie.h"
#include "pie_kernels.h"
#include "pie_tc.h"

namespace pie {

namespace {

constexpr int PR_KV = 128;                    // tokens of a stage
constexpr int PR_SOFTMAX_THREADS = 256;       // warps 0 .. 3: tile 0, warps 4 .. 7: tile 1
constexpr int PR_THREADS = PR_SOFTMAX_THREADS + 128;  // + the issuing warp (8), the loading warp (9) and two that look V over (10, 11)
// Registers: 384 threads get 168 each at launch; the softmax warpgroups, whose threads hold a row of 128 scores, take over what
// the third gives up: 2 x 128 x 208 + 128 x 88 = 384 x 168.
constexpr int PR_REGS_SOFTMAX = 208, PR_REGS_REST = 88;
static_assert(2 * PR_REGS_SOFTMAX + PR_REGS_REST == 3 * 168, "what one side takes the other gives");
constexpr int PR_TMEM_COLS = 512;             // S0, S1 (128 each; P over them), O0, O1 (128 each)
// A row's running maximum is raised - and its O and sum rescaled - only when a stage exceeds it by more than this (log2
// units): probabilities are then at most 2^8, harmless in fp32 sums and in both 16-bit types, and after the first stages
// hardly any stage rescales.
constexpr float PR_LAZY = 8.f;
// fp16 has only subnormal numbers below 2^-14 and none below 2^-24: beside one dominating key thousands of small probabilities
// would lose bits, or all of them, while the row's sum counts them.  For fp16 the running maximum is therefore kept less 7, and all
// probabilities are 2^7 as large (2^15 at most; O and the sum carry the factor, which cancels): what one loses below fp16's smallest
// step is then at most 2^-32 of the row's largest probability.  (As long as before where no P was lost; where many were zero the
// products of zeros had taken less power: 10007 tokens, 32 / 8 heads of 128, scores of N(0, 4^2): 795 -> 831 us.)
constexpr float PR_SHIFT_F16 = 15.f - PR_LAZY;

constexpr int PR_INLINE = 480;   // items that travel with the launch's parameters (7.5 KiB): no copy in front of the call.  It saves 7 us
                                 // (16 ragged prompts: 135 -> 128 us); with 960 a call of 45 tokens takes 0.5 us longer, with 1900 1.8 us

struct PromptParams {
    const int4 *items;       // {first token of the sequence, first token of the item (within it), sequence length, -}; NULL: inline
    uint16_t *out;
    const uint16_t *v;       // (the values again, for the rare repair below)
    int32_t *status;
    int64_t v_stride;
    int32_t n_q_heads, n_kv_heads, group, tile_tokens;
    int32_t n_work;          // items * KV heads
    float scale_log2e;
    int4 inline_items[PR_INLINE];
};

template <int D>
struct PrSmem {
    static constexpr int Q_BYTES = 2 * TC_M * D * 2;   // two tiles of [D / 64][128 rows][128 B]
    static constexpr int STAGE = PR_KV * D * 2;        // [D / 64][128 tokens][128 B]
    static constexpr int RING = D == 128 ? 5 : 8;
    static constexpr int OFF_Q = 0;
    static constexpr int OFF_RING = OFF_Q + Q_BYTES;
    static constexpr int OFF_BAR = OFF_RING + RING * STAGE;   // full[4], clean[4], free[4], s[2], pa[2], pb[2], done[2], q[2], k0, end
    static constexpr int OFF_MISC = OFF_BAR + 24 * 8;         // [0] TMEM base, [1] abort, [4], [5] the first and the last item (+ 1) with a value not finite
    static constexpr int BYTES = OFF_MISC + 32;
};

__device__ __forceinline__ void pr_tma_3d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}

// true in one lane of the (whole) warp: the branch of an elected lane keeps the operands in uniform registers
__device__ __forceinline__ bool pr_elect() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// the larger of three; NaN if any of them is one
__device__ __forceinline__ float pr_max3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float2 pr_fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(*reinterpret_cast<uint64_t *>(&r))
        : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)), "l"(*reinterpret_cast<uint64_t *>(&c)));
    return r;
}
__device__ __forceinline__ float2 pr_add2(float2 a, float2 b) {
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(*reinterpret_cast<uint64_t *>(&r))
        : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return r;
}

__device__ __forceinline__ void pr_tmem_ld8(uint32_t taddr, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void pr_tmem_st8(uint32_t taddr, const uint32_t (&v)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

// largest magnitude bits of the two halves of each word; >= EXP in a half: that value is not finite
template <bool BF16>
__device__ __forceinline__ bool pr_not_finite(const uint4 &w) {
    const uint32_t m = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
    constexpr uint32_t EXP = BF16 ? 0x7f80u : 0x7c00u;
    return (m & 0xffffu) >= EXP || (m >> 16) >= EXP;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pr_clear_not_finite(uint32_t w) {
    constexpr uint32_t EXP = BF16 ? 0x7f80u : 0x7c00u;
    if ((w & 0x7fffu) >= EXP) w &= 0xffff0000u;
    if (((w >> 16) & 0x7fffu) >= EXP) w &= 0xffffu;
    return w;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(PR_THREADS, 1)
prompt_attn_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const PromptParams p) {
    using SM = PrSmem<D>;
    constexpr int HALVES = D / 64;
    constexpr int RING = SM::RING;
    // (All exponentials in the special-function unit, 16 a clock and SM: as long for a stage's as the tensor core for its products.
    // An eighth, a quarter, three eighths of them by a polynomial in the arithmetic pipes cost heads of 128 as many instructions as
    // that relief gives back.  One prompt of 10007 tokens, 32 / 8 heads of 128, bf16: 0, 1, 2, 3 eighths 649, 653, 654, 685 us; 16
    // ragged prompts: 127, 127, 128, 149 us.  Heads of 64, fp16, 10007 tokens, the kernel as it was then: 585, 594, 564, 619 us - a
    // quarter gained 4 % there; one form was kept for both.)
    extern __shared__ __align__(1024) uint8_t pr_smem[];
    uint8_t *smem = pr_smem;
    const uint32_t base = pf_smem_u32(pr_smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (base & 1023u) {   // the swizzled tiles need a 1024-byte boundary: never seen otherwise, but do not compute garbage
        if (tid == 0) pf_raise(p.status, STATUS_WAIT_TIMEOUT);
        return;
    }
    // A CTA works through its items without a break: the stages of all of them form one sequence g = 0, 1, ...  Ring entry 2 g
    // is K, 2 g + 1 is V of stage g.  full[g & 3]: V(g) and K(g + 1) have landed; clean[g & 3]: and V(g) may be multiplied.
    // free[f & 3]: f = 0: the first scores, f = g + 1: all MMAs of stage g (O += P V of both tiles and the next scores) are
    // complete.  Per tile: s: scores complete, pa, pb: the halves of P in place, done: O of the item complete, q: its query rows
    // have landed.  k0: the first keys.  end: where the CTA gives up, the MMAs issued by then are complete.
    const uint32_t bar_full = base + SM::OFF_BAR, bar_clean = bar_full + 32, bar_free = bar_clean + 32, bar_s = bar_free + 32, bar_pa = bar_s + 16, bar_pb = bar_pa + 16;
    const uint32_t bar_done = bar_pb + 16, bar_q = bar_done + 16, bar_k0 = bar_q + 16, bar_end = bar_k0 + 8;
    volatile uint32_t *misc = reinterpret_cast<volatile uint32_t *>(smem + SM::OFF_MISC);

    // ---- the CTA's items: the list goes from long to short, and every other pass over the CTAs runs backwards, so that all get
    // about the same number of stages (every warp works the sequence out for itself)
    const int32_t G = p.group, TT = p.tile_tokens;
    struct Item {
        int32_t kvh, seq0, tok0, len, n0, n1, n;   // n0, n1: stages of each tile - what its last token sees (0: no such tile); n: the larger
    };
    auto get_item = [&](int32_t k, Item &it) {     // the CTA's k-th; false: there are no more
        const int32_t x = (k & 1) ? (k + 1) * (int32_t)gridDim.x - 1 - (int32_t)blockIdx.x : k * (int32_t)gridDim.x + (int32_t)blockIdx.x;
        if (x >= p.n_work) return false;
        const int32_t i = x / p.n_kv_heads;
        const int4 v = p.items != nullptr ? __ldg(p.items + i) : p.inline_items[i];
        it.kvh = x - i * p.n_kv_heads;
        it.seq0 = v.x;
        it.tok0 = v.y;
        it.len = v.z;
        const int32_t end0 = min(it.tok0 + TT, it.len), end1 = min(it.tok0 + 2 * TT, it.len);
        it.n0 = (end0 + PR_KV - 1) / PR_KV;
        it.n1 = end1 > end0 ? (end1 + PR_KV - 1) / PR_KV : 0;
        it.n = max(it.n0, it.n1);
        return true;
    };

    if (tid == 0) {
        for (int i = 0; i < 4; ++i) {
            pf_mbar_init(bar_full + 8 * i, 1);
            pf_mbar_init(bar_clean + 8 * i, 2);   // warps 10 and 11
            pf_mbar_init(bar_free + 8 * i, 1);
        }
        misc[4] = 0xffffffffu;
        misc[5] = 0;
        pf_mbar_init(bar_k0, 1);
        pf_mbar_init(bar_end, 1);
        for (int t = 0; t < 2; ++t) {
            pf_mbar_init(bar_q + 8 * t, 1);
            pf_mbar_init(bar_s + 8 * t, 1);
            pf_mbar_init(bar_pa + 8 * t, 4);   // a warp each
            pf_mbar_init(bar_pb + 8 * t, 4);
            pf_mbar_init(bar_done + 8 * t, 1);
        }
        misc[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 8) tmem_alloc(base + SM::OFF_MISC, PR_TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = misc[0];
    if (tmem != 0 && tid == 0) {   // (every column is this CTA's: cannot be) - the issuing warp goes by it
        pf_raise(p.status, STATUS_WAIT_TIMEOUT);
        misc[1] = 1;
    }

    auto dead = [&]() { return __any_sync(0xffffffffu, misc[1] != 0); };
    // by every lane of a warp; false: give up (the wait ran out, here or in another warp).  Bounded: about a second.  Lanes may get
    // different answers from a barrier whose phase completes at that moment, so whether the warp polls on is one vote of all its
    // lanes: every way out leads through the same votes.
    auto wait_all = [&](uint32_t bar, uint32_t parity) {
        if (__all_sync(0xffffffffu, pf_mbar_try_wait(bar, parity)) != 0) return true;
        bool there = false;
        for (uint32_t i = 0; i < (1u << 22) && !there; ++i) {
            there = pf_mbar_try_wait(bar, parity);
            if (!there && i > 64) {
                if (misc[1] != 0) break;
                __nanosleep(200);
            }
        }
        if (!there) {
            pf_raise(p.status, STATUS_WAIT_TIMEOUT);
            misc[1] = 1;
        }
        return __all_sync(0xffffffffu, there) != 0;
    };

    // (each role's own branch holds its register instruction: the compiler allocates by region)
    if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_REGS_REST));
    if (warp == 9) {
        // =============================================================================== the loading warp
        int32_t freed = -1;   // free[] waited for so far
        auto need = [&](int32_t f) {
            for (; freed < f; ++freed)
                if (!wait_all(bar_free + 8 * ((freed + 1) & 3), (uint32_t)(((freed + 1) >> 2) & 1))) return false;
            return true;
        };
        auto load_q = [&](const Item &it) {
            if (lane == 0)
                for (int t = 0; t < (it.n1 > 0 ? 2 : 1); ++t) {
                    pf_mbar_expect_tx(bar_q + 8 * t, (uint32_t)(G * TT) * D * 2);
                    for (int h = 0; h < HALVES; ++h)
                        pr_tma_3d(base + SM::OFF_Q + t * (TC_M * D * 2) + h * (TC_M * 128), &map_q, 64 * h, it.kvh * G, it.seq0 + it.tok0 + t * TT, bar_q + 8 * t);
                }
            __syncwarp();
        };
        auto load_kv = [&](const CUtensorMap *map, const Item &it, int32_t j, uint32_t slot, uint32_t bar) {
            if (lane == 0)
                for (int h = 0; h < HALVES; ++h)
                    pr_tma_3d(base + SM::OFF_RING + slot * SM::STAGE + h * (PR_KV * 128), map, 64 * h, it.kvh, it.seq0 + j * PR_KV, bar);
            __syncwarp();
        };
        Item it, next;
        bool more = get_item(0, it), ok = true;
        int32_t g = 0, q_count[2] = {0, 0};
        uint32_t slot = 1;
        if (more) {
            if (lane == 0) pf_mbar_expect_tx(bar_k0, SM::STAGE);
            __syncwarp();
            load_q(it);
            load_kv(&map_k, it, 0, 0, bar_k0);
            q_count[0] = 1;
            q_count[1] = it.n1 > 0;
        }
        for (int32_t k = 0; more && ok; ++k) {
            more = get_item(k + 1, next);
            for (int32_t j = 0; j < it.n && ok; ++j, ++g) {
                const bool last = j + 1 == it.n;
                const uint32_t bar = bar_full + 8 * (g & 3);
                // the slot of V(g) held K(g - 2), used in stage g - 3 (ring of 5; of 8: V(g - 4)); that of K(g + 1) held V(g - 2) (of 8: K(g - 3))
                ok = need(RING == 5 ? g - 2 : g - 3);
                if (!ok) break;
                if (lane == 0) pf_mbar_expect_tx(bar, last && !more ? SM::STAGE : 2 * SM::STAGE);
                __syncwarp();
                load_kv(&map_v, it, j, slot, bar);
                slot = slot + 1 == RING ? 0 : slot + 1;
                if (!last || more) {
                    if (need(RING == 5 ? g - 1 : g - 3)) load_kv(&map_k, last ? next : it, last ? 0 : j + 1, slot, bar);
                    else ok = false;
                }
                slot = slot + 1 == RING ? 0 : slot + 1;
                if (last && more && ok) {   // the item's last scores are complete: its query rows make room
                    ok = need(g);
                    if (ok) {
                        load_q(next);
                        q_count[0] += 1;
                        q_count[1] += next.n1 > 0;
                    }
                }
            }
            it = next;
        }
        if (!ok || dead()) {   // giving up: wait (bounded) for the copies that still write into this CTA's shared memory
            for (int t = 0; t < 2; ++t)
                if (q_count[t] > 0) pf_mbar_wait(bar_q + 8 * t, (uint32_t)((q_count[t] - 1) & 1));
            if (q_count[0] > 0) pf_mbar_wait(bar_k0, 0);
            for (int32_t i = max(0, g - 3); i <= g; ++i) pf_mbar_wait(bar_full + 8 * (i & 3), (uint32_t)((i >> 2) & 1));
        }
        __syncwarp();
    } else if (warp == 8) {
        // =============================================================================== the issuing warp
        // The operands are warp-uniform values and the branch is an elected lane's, so that the MMAs take them from uniform
        // registers as they come: formed in the branch of lane 0, each MMA waited for the moves (863 us for 10007 tokens), issued
        // without a branch, by a predicate, it cost some ten instructions (715 us; so 679 us, the rest of the kernel as it was then).  TMEM: all 512 columns are this
        // CTA's, so its base is column 0.
        constexpr uint32_t IDESC_S = instr_desc(BF16, PR_KV, false), IDESC_O = instr_desc(BF16, D, true);
        const uint64_t q_desc = smem_desc(base + SM::OFF_Q, 16, 1024), k_desc = smem_desc(base + SM::OFF_RING, 16, 1024);
        const uint64_t v_desc = smem_desc(base + SM::OFF_RING, PR_KV * 128, 1024);
        // S of a tile, K in ring slot `slot`
        auto issue_s = [&](int t, uint32_t slot) {
            tc_fence_after();
            const uint64_t qd = q_desc + (uint64_t)(t * (TC_M * D * 2) >> 4), kd = k_desc + (uint64_t)(slot * (SM::STAGE >> 4));
            if (pr_elect()) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    mma_f16(t * 128, qd + (uint64_t)(((ks >> 2) * (TC_M * 128) + (ks & 3) * 32) >> 4),
                            kd + (uint64_t)(((ks >> 2) * (PR_KV * 128) + (ks & 3) * 32) >> 4), IDESC_S, ks > 0 ? 1u : 0u);
                tc_commit(bar_s + 8 * t);
            }
            __syncwarp();
        };
        // O += P V of half the stage's tokens
        auto issue_o = [&](int t, int half, uint64_t vd, bool add, bool last = false) {
            tc_fence_after();
            if (pr_elect()) {
#pragma unroll
                for (int i = 0; i < PR_KV / 32; ++i) {   // V: 16 tokens further per step, 64-element chunks of D are 16 KiB apart
                    const int ks = half * (PR_KV / 32) + i;
                    mma_f16_ts(256 + t * 128, t * 128 + ks * 8, vd + (uint64_t)(ks * 2048 >> 4), IDESC_O, (add || i > 0) ? 1u : 0u);
                }
                if (last) tc_commit(bar_done + 8 * t);
            }
            __syncwarp();
        };
        Item it, next;
        bool more = get_item(0, it), ok = true;
        uint32_t p_count[2] = {0, 0}, q_count[2] = {0, 0};
        if (more) {
            ok = wait_all(bar_k0, 0);
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (ok && (t == 0 || it.n1 > 0)) {
                    ok = wait_all(bar_q + 8 * t, 0);
                    q_count[t] = 1;
                    if (ok) issue_s(t, 0);
                }
            if (pr_elect()) tc_commit(bar_free);
            __syncwarp();
        }
        uint32_t v_slot = 1;
        int32_t g = 0;
        for (int32_t k = 0; more && ok; ++k) {
            more = get_item(k + 1, next);
            const int32_t nx0 = more ? next.n0 : 0, nx1 = more ? next.n1 : 0;
            for (int32_t j = 0; ok && j < it.n; ++j, ++g) {
                const uint32_t k_slot = v_slot + 1 == RING ? 0 : v_slot + 1;
                const uint64_t vd = v_desc + (uint64_t)(v_slot * (SM::STAGE >> 4));
                const bool last = j + 1 == it.n;
                ok = wait_all(bar_clean + 8 * (g & 3), (uint32_t)((g >> 2) & 1));   // V(g) and K(g + 1) are there
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int32_t n = t == 0 ? it.n0 : it.n1, nx = t == 0 ? nx0 : nx1;
                    if (ok && j < n) {
                        // (the first half's products run while the softmax warps work on the second)
                        ok = wait_all(bar_pa + 8 * t, p_count[t] & 1u);
                        if (ok) {
                            issue_o(t, 0, vd, j > 0);
                            ok = wait_all(bar_pb + 8 * t, p_count[t] & 1u);
                        }
                        ++p_count[t];
                        if (!ok) continue;
                        issue_o(t, 1, vd, true, j + 1 == n);
                    }
                    if (ok && (j + 1 < n || (last && nx > 0))) {   // the item's next scores, or the next item's first
                        if (j + 1 >= n) {
                            ok = wait_all(bar_q + 8 * t, q_count[t] & 1u);
                            ++q_count[t];
                        }
                        if (ok) issue_s(t, k_slot);
                    }
                }
                if (pr_elect()) tc_commit(bar_free + 8 * ((g + 1) & 3));
                __syncwarp();
                v_slot = k_slot + 1 == RING ? 0 : k_slot + 1;
            }
            it = next;
        }
        if (!ok || dead()) {   // giving up: the MMAs in flight still read this CTA's shared memory and write its tensor memory - wait (bounded) for them
            if (pr_elect()) tc_commit(bar_end);
            __syncwarp();
            pf_mbar_wait(bar_end, 0);
        }
        __syncwarp();
    } else {
        // =============================================================================== the warps that look V over
        // Values that some row of the item may not see meet P = 0 there, which hides everything but NaN and infinities.  Those
        // are cleared in the stage and, if there were any, added at the end to the rows that do see them.  (Done by the softmax
        // warps in front of their arrival it took 1000 to 1700 cycles of every masked stage.)
        Item it, next;
        bool more = get_item(0, it), ok = true;
        const int me = (warp - 10) * 32 + lane;
        int32_t g = 0;
        for (int32_t k = 0; more && ok; ++k) {
            more = get_item(k + 1, next);
            for (int32_t j = 0; j < it.n; ++j, ++g) {
                ok = wait_all(bar_full + 8 * (g & 3), (uint32_t)((g >> 2) & 1));
                if (!ok) break;
                const int32_t first = it.tok0 + 1 - j * PR_KV;   // rows of the stage from here on are masked for some row of the item
                if (first < PR_KV) {
                    uint8_t *vs = smem + SM::OFF_RING + (2 * g + 1) % RING * SM::STAGE;
                    bool found = false;
                    for (int e = max(0, first) * 8 + me; e < PR_KV * 8; e += 256) {
                        uint4 w[4][HALVES];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int h = 0; h < HALVES; ++h)
                                w[u][h] = e + 64 * u < PR_KV * 8 ? *reinterpret_cast<const uint4 *>(vs + h * (PR_KV * 128) + (e + 64 * u) * 16) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int h = 0; h < HALVES; ++h)
                                if (pr_not_finite<BF16>(w[u][h])) {
                                    found = true;
                                    *reinterpret_cast<uint4 *>(vs + h * (PR_KV * 128) + (e + 64 * u) * 16) =
                                        make_uint4(pr_clear_not_finite<BF16>(w[u][h].x), pr_clear_not_finite<BF16>(w[u][h].y),
                                                   pr_clear_not_finite<BF16>(w[u][h].z), pr_clear_not_finite<BF16>(w[u][h].w));
                                }
                    }
                    if (found) {
                        atomicMin(const_cast<uint32_t *>(misc + 4), (uint32_t)k + 1u);
                        atomicMax(const_cast<uint32_t *>(misc + 5), (uint32_t)k + 1u);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                }
                __syncwarp();
                if (lane == 0) pf_mbar_arrive(bar_clean + 8 * (g & 3));
            }
            it = next;
        }
        __syncwarp();
    }
    } else {
        // =============================================================================== the softmax warps
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PR_REGS_SOFTMAX));
        const int t = warp >> 2;
        const int r = tid & 127;                                      // row of the tile
        const int32_t my_tok = r / G, my_g = r - my_tok * G;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tmem_s = t * 128 + lane_addr, tmem_o = 256 + t * 128 + lane_addr;
        Item it, next;
        bool more = get_item(0, it), ok = true;
        uint32_t s_count = 0, done_count = 0;
        for (int32_t k = 0; more && ok; ++k, it = next) {
        const int32_t n = t == 0 ? it.n0 : it.n1, tok0 = it.tok0;
        if (n == 0) {
            more = get_item(k + 1, next);
            continue;
        }
        const int32_t first = tok0 + t * TT;                          // the tile's first position
        const int32_t my_pos = first + my_tok;
        const bool row_valid = my_tok < TT && my_pos < it.len;
        float m_run = -INFINITY, l_run = 0.f;
        bool spoiled = false;                                         // a score the row sees is NaN or +inf: so is the softmax
        for (int32_t j = 0; j < n; ++j) {
            if (!wait_all(bar_s + 8 * t, s_count & 1u)) { ok = false; break; }
            ++s_count;
            tc_fence_after();
            uint32_t sv[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(tmem_s + 32 * c, sv[c]);
            tmem_wait_ld();
            const int32_t t_base = j * PR_KV;
            const bool masked = t_base + PR_KV - 1 > first;           // some row of the tile does not see the whole stage
            float scale = p.scale_log2e;
            if (masked || scale <= 0.f) {
                if (scale <= 0.f) {                                   // (the maximum is taken of the scaled scores)
#pragma unroll
                    for (int c = 0; c < 128; ++c) sv[c >> 5][c & 31] = __float_as_uint(__uint_as_float(sv[c >> 5][c & 31]) * scale);
                    scale = 1.f;
                }
                // what a row may not see becomes -inf (by selection: NaN scores too), in the quarters that some row does not see whole
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (t_base + 32 * u + 31 > first) {
#pragma unroll
                        for (int c = 0; c < 32; ++c) sv[u][c] = t_base + 32 * u + c <= my_pos ? sv[u][c] : 0xff800000u;
                    }
            }
            float a0 = -INFINITY, a1 = -INFINITY, a2 = -INFINITY, a3 = -INFINITY;
#pragma unroll
            for (int c = 0; c < 32; c += 2) {
                a0 = pr_max3(a0, __uint_as_float(sv[0][c]), __uint_as_float(sv[0][c + 1]));
                a1 = pr_max3(a1, __uint_as_float(sv[1][c]), __uint_as_float(sv[1][c + 1]));
                a2 = pr_max3(a2, __uint_as_float(sv[2][c]), __uint_as_float(sv[2][c + 1]));
                a3 = pr_max3(a3, __uint_as_float(sv[3][c]), __uint_as_float(sv[3][c + 1]));
            }
            const float mx = pr_max3(a0, a1, pr_max3(a2, a3, a3)) * scale - (BF16 ? 0.f : PR_SHIFT_F16);
            spoiled |= !(mx < INFINITY);
            const float m_cand = fmaxf(m_run, mx);
            const bool grow = m_cand > m_run + PR_LAZY;               // (m_run = -inf: true unless the row has seen nothing finite yet)
            const float m_new = grow ? m_cand : m_run;
            const float alpha = grow ? pf_exp2(m_run - m_cand) : 1.f; // (m_run = -inf gives 0: nothing accumulated yet)
            m_run = m_new;
            const float neg_m = m_new == -INFINITY ? 0.f : -m_new;    // (a row that has seen nothing: exponents stay -inf)
            // ---- O *= alpha where a row's maximum moved (skipped by warps in which none did; few columns at a time: the scores
            // are in registers)
            if (j >= 1 && __any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 8) {
                    uint32_t ov[8];
                    pr_tmem_ld8(tmem_o + c0, ov);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 8; ++c) ov[c] = __float_as_uint(__uint_as_float(ov[c]) * alpha);
                    pr_tmem_st8(tmem_o + c0, ov);
                }
            }
            const float2 sc2 = make_float2(scale, scale), nm2 = make_float2(neg_m, neg_m);
            float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t pw[32];
#pragma unroll
                for (int w = 0; w < 32; ++w) {
                    const int c = 64 * h + 2 * w;
                    const float2 x = pr_fma2(make_float2(__uint_as_float(sv[c >> 5][c & 31]), __uint_as_float(sv[c >> 5][(c & 31) + 1])), sc2, nm2);
                    const float2 e = make_float2(pf_exp2(x.x), pf_exp2(x.y));
                    if (w & 1) s1 = pr_add2(s1, e);
                    else s0 = pr_add2(s0, e);
                    pw[w] = pf_pack2<BF16>(e.x, e.y);
                    if (h == 1 && w == 7) {                           // the first half is in place (stored long enough ago not to wait)
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) pf_mbar_arrive(bar_pa + 8 * t);
                    }
                }
                tmem_st32(tmem_s + 32 * h, pw);   // a thread overwrites only its own row's scores, which it has read
            }
            s0 = pr_add2(s0, s1);
            l_run = l_run * alpha + (s0.x + s0.y);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) pf_mbar_arrive(bar_pb + 8 * t);
        }
        more = get_item(k + 1, next);                                 // (looked up while the last products run)
        if (ok) ok = wait_all(bar_done + 8 * t, done_count & 1u);
        ++done_count;
        // ---- out = O / l, rounded to the 16-bit type (nearest even).  The TMEM loads are warp-wide: rows beyond the tile take
        // part in them and store nothing.
        if (ok) {
            tc_fence_after();
            const float inv = spoiled ? __int_as_float(0x7fc00000) : 1.f / l_run;
            const bool wide_out = (reinterpret_cast<uintptr_t>(p.out) & 31) == 0;
            // (items between the first and the last such item look for nothing in vain; a flag per item could be overwritten while a
            // tile that has no part in the items in between is still behind)
            const bool repair = misc[4] <= (uint32_t)k + 1u && (uint32_t)k + 1u <= misc[5];
            uint4 *dst = reinterpret_cast<uint4 *>(p.out + ((int64_t)(it.seq0 + my_pos) * p.n_q_heads + it.kvh * G + my_g) * D);
            const uint16_t *vrow = p.v + (int64_t)(it.seq0 + tok0 + 1) * p.v_stride + (int64_t)it.kvh * D;
#pragma unroll 1
            for (int c0 = 0; c0 < D; c0 += 32) {
                uint32_t ov[32];
                tmem_ld32(tmem_o + c0, ov);
                tmem_wait_ld();
                if (row_valid) {
                    if (repair) {
                        for (int32_t k = 0; tok0 + 1 + k <= my_pos; ++k)
#pragma unroll
                            for (int c = 0; c < 32; ++c) {
                                const uint32_t b = vrow[k * p.v_stride + c0 + c];
                                const float x = BF16 ? __uint_as_float(b << 16) : __half2float(__ushort_as_half((uint16_t)b));
                                if ((b & 0x7fffu) >= (BF16 ? 0x7f80u : 0x7c00u)) ov[c] = __float_as_uint(__uint_as_float(ov[c]) + x);
                            }
                    }
                    uint32_t w[16];
#pragma unroll
                    for (int c = 0; c < 16; ++c) w[c] = pf_pack2<BF16>(__uint_as_float(ov[2 * c]) * inv, __uint_as_float(ov[2 * c + 1]) * inv);
                    // whole sectors (32 bytes) a store: the rows lie apart, and a sector written in two halves takes the way to L2 twice
                    if (wide_out) {
#pragma unroll
                        for (int c = 0; c < 16; c += 8)
                            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + c0 / 8 + c / 4), "r"(w[c]), "r"(w[c + 1]),
                                         "r"(w[c + 2]), "r"(w[c + 3]), "r"(w[c + 4]), "r"(w[c + 5]), "r"(w[c + 6]), "r"(w[c + 7])
                                         : "memory");
                    } else {
#pragma unroll
                        for (int c = 0; c < 16; c += 4) dst[c0 / 8 + c / 4] = make_uint4(w[c], w[c + 1], w[c + 2], w[c + 3]);
                    }
                }
            }
        }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, PR_TMEM_COLS);
}

// [tokens][heads][head_dim] as tiles of 64 elements x `heads` heads x `tokens` tokens
cudaError_t make_token_map(const void *x, int64_t n_tokens, int64_t stride, int n_heads, int head_dim, int box_heads, int box_tokens,
                           CUtensorMap *map) {
    typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                      const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                      CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static EncodeTiledFn encode = nullptr;
    if (!encode) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
        if (e != cudaSuccess) return e;
        if (fn == nullptr || qres != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
        encode = reinterpret_cast<EncodeTiledFn>(fn);
    }
    cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)n_heads, (cuuint64_t)n_tokens};
    cuuint64_t strides[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)stride * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
    cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void *>(x), dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <typename F>
cudaError_t dispatch_prompt(int head_dim, int dtype, F &&f) {
    if (head_dim == 128) return dtype == PIE_BF16 ? f(prompt_attn_kernel<128, true>, PrSmem<128>::BYTES) : f(prompt_attn_kernel<128, false>, PrSmem<128>::BYTES);
    return dtype == PIE_BF16 ? f(prompt_attn_kernel<64, true>, PrSmem<64>::BYTES) : f(prompt_attn_kernel<64, false>, PrSmem<64>::BYTES);
}

}  // namespace

cudaError_t prompt_configure(int head_dim, int dtype) {
    return dispatch_prompt(head_dim, dtype, [](auto kernel, int smem) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        return cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    });
}

int64_t prompt_inline_items() { return PR_INLINE; }

cudaError_t launch_prompt_attention(const AttnShape &sh, const PromptLaunch &a, int n_sms, cudaStream_t stream) {
    if (a.n_items <= 0) return cudaSuccess;
    const int group = sh.n_q_heads / sh.n_kv_heads;
    CUtensorMap map_q, map_k, map_v;
    cudaError_t e = make_token_map(a.q, a.n_tokens, a.q_stride, sh.n_q_heads, sh.head_dim, group, a.tile_tokens, &map_q);
    if (e == cudaSuccess) e = make_token_map(a.k, a.n_tokens, a.k_stride, sh.n_kv_heads, sh.head_dim, 1, PR_KV, &map_k);
    if (e == cudaSuccess) e = make_token_map(a.v, a.n_tokens, a.v_stride, sh.n_kv_heads, sh.head_dim, 1, PR_KV, &map_v);
    if (e != cudaSuccess) return e;
    PromptParams p;
    p.items = reinterpret_cast<const int4 *>(a.items);
    if (a.items == nullptr) std::memcpy(p.inline_items, a.items_host, (size_t)a.n_items * 16);
    p.n_work = (int32_t)(a.n_items * sh.n_kv_heads);
    p.out = (uint16_t *)a.out;
    p.v = (const uint16_t *)a.v;
    p.status = a.status;
    p.v_stride = a.v_stride;
    p.n_q_heads = sh.n_q_heads;
    p.n_kv_heads = sh.n_kv_heads;
    p.group = group;
    p.tile_tokens = a.tile_tokens;
    p.scale_log2e = a.scale * 1.4426950408889634f;
    return dispatch_prompt(sh.head_dim, sh.dtype, [&](auto kernel, int smem) {
        kernel<<<(unsigned)std::min<int64_t>(p.n_work, n_sms), PR_THREADS, smem, stream>>>(map_q, map_k, map_v, p);
        return cudaGetLastError();
    });
}

}  // namespace pie
