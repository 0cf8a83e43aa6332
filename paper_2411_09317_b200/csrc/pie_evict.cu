// Eviction from the paged cache by accumulated attention weight: per (sequence, KV head) the newest `recent` tokens stay, and of
// the older ones the budget - recent with the largest weights; the kept tokens' keys, values and weights move to the front.
//
// Two kernels.  evict_select_kernel, one CTA per (sequence, KV head): the weight of the last token that still gets a place is
// found digit by digit (radix select over the weights' order-preserving bit patterns, 12 + 10 + 10 bits: exact, whatever their
// distribution, where a sort would move every weight several times).  The weights are read once into registers; the few that
// share the first digit are ranked among themselves by comparison where they fit a list.  Then one pass in token order writes the
// kept positions, their weights and the cache rows they lie in.  evict_copy_kernel (out of place) or evict_move_kernel (in place)
// moves the rows; it is a programmatic dependent of the first.  (Both in one CTA: 264 us against 246 for 32 x 32 pairs, 41 against
// 34 for 24 x 8: the selecting CTAs' shared memory and barriers leave too few copies in flight.)
// Bound: bytes (kept rows in and out; the weights once): 1.1 GB in 225 us, 76 % of a plain copy's rate; rows of 256 bytes lie
// scattered, and 30 us of it are the selection, which the first rows wait for.
#include <algorithm>
#include <type_traits>

#include "../../include/pie.h"
#include "pie_kernels.h"

namespace pie {

namespace {

constexpr int SEL_THREADS = 512;
constexpr int SEL_WARPS = SEL_THREADS / 32;
constexpr int SEL_BINS = 4096;        // of the first digit: sign, exponent, three bits of the fraction - eight bins an octave keep
                                      // the counters of a warp's weights mostly apart
constexpr int SEL_LIST = 512;         // candidates that share the first digit and are ranked by comparison
constexpr int SEL_SLOTS = 7000;       // blocks of a sequence whose slots are kept in shared memory; beyond that they are looked up again
                                      // (24 sequences of up to 3500 tokens: 32.5 us, looked up 32.8; 32 of 4096: 225 and 226)
constexpr int MOVE_THREADS = 256;
constexpr int MOVE_ROWS = 128;        // rows of a CTA of the move out of place
constexpr int MOVE_DEPTH = 4;         // in place: 16-byte vectors a thread holds per batch

struct EvictParams {
    EvictLaunch a;
    int64_t n_gpu_slots;
    int32_t n_kv_heads, n_logical, row_vecs;   // row_vecs: 16-byte vectors of one K (or V) row
};

// bit patterns in the order of the values (-0 and 0 alike); NaN below everything.  Weights are handled as bit patterns
// throughout: float instructions, a selection among them, flush subnormal weights (a long decayed tail has them) to zero.
__device__ __forceinline__ uint32_t weight_key(uint32_t b) {
    const uint32_t magnitude = b & 0x7fffffffu;
    if (magnitude > 0x7f800000u) return 0u;
    return magnitude == 0u ? 0x80000000u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ int32_t unit_slot(const EvictParams &p, const int32_t *table_row, int32_t i) {
    const int32_t b = __ldg(table_row + i);
    const int32_t slot = (b >= 0 && b < p.n_logical) ? __ldcg(p.a.slot_table + b) : -1;
    return slot < p.n_gpu_slots ? slot : -1;
}

__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Of 16 words in shared memory, one per warp: the sum of those in front of this warp's, and of all.
__device__ __forceinline__ uint32_t warps_before(const int32_t *sums, uint32_t *all) {
    static_assert(SEL_WARPS == 16, "");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t mine = lane < SEL_WARPS ? (uint32_t)sums[lane] : 0u;
    uint32_t inc = mine;
#pragma unroll
    for (int o = 1; o < SEL_WARPS; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    *all = __shfl_sync(0xffffffffu, inc, SEL_WARPS - 1);
    return __shfl_sync(0xffffffffu, inc - mine, warp);
}

// The bin (counted from the top) in which the count from above reaches *rank; *rank becomes the rank inside it.  BINS
// counters in shared memory, read by every thread of the CTA.  Three barriers.
template <int BINS>
__device__ __forceinline__ uint32_t find_bin(const int32_t *hist, int32_t *rank, int32_t *warp_sums, volatile int32_t *answer) {
    constexpr int PER = BINS / SEL_THREADS;   // consecutive bins of a thread, from the top: read as vectors (no bank conflicts)
    static_assert(PER == 8 || PER == 2, "");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t c[PER], mine = 0;
    if constexpr (PER == 8) {
        const int4 hi = reinterpret_cast<const int4 *>(hist)[BINS / 4 - 1 - 2 * tid], lo = reinterpret_cast<const int4 *>(hist)[BINS / 4 - 2 - 2 * tid];
        c[0] = hi.w, c[1] = hi.z, c[2] = hi.y, c[3] = hi.x, c[4] = lo.w, c[5] = lo.z, c[6] = lo.y, c[7] = lo.x;
    } else {
        const int2 v = reinterpret_cast<const int2 *>(hist)[BINS / 2 - 1 - tid];
        c[0] = v.y, c[1] = v.x;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) mine += c[i];
    int32_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    uint32_t all;
    int32_t above = inc - mine + (int32_t)warps_before(warp_sums, &all);
    const int32_t want = *rank;
    if (above < want && want <= above + mine) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (above < want && want <= above + c[i]) {
                answer[0] = BINS - 1 - (PER * tid + i);
                answer[1] = want - above;
            }
            above += c[i];
        }
    }
    __syncthreads();
    const uint32_t bin = (uint32_t)answer[0];
    *rank = answer[1];
    __syncthreads();
    return bin;
}

// ITEMS: consecutive weights that a thread holds; sequences of more than SEL_THREADS * ITEMS tokens go in pieces, read again
// in every pass.
template <int ITEMS>
__global__ void __launch_bounds__(SEL_THREADS, ITEMS <= 8 ? 4 : 2)   // (latency: the more CTAs on an SM the better)
evict_select_kernel(const EvictParams p, int32_t smem_slots) {
    constexpr int PIECE = SEL_THREADS * ITEMS;
    __shared__ __align__(16) int32_t hist[SEL_BINS];
    __shared__ uint32_t list[SEL_LIST];
    __shared__ int32_t n_list;
    __shared__ int32_t warp_sums[2 * SEL_WARPS];
    __shared__ volatile int32_t answer[2];
    extern __shared__ int32_t slots[];   // of the sequence's blocks, where they fit
    const EvictLaunch &a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t pair = blockIdx.x, s = pair / p.n_kv_heads;
    const int32_t ctx = __ldg(a.ctx_lens + s), n_new = min(ctx, a.budget);
    const int32_t *src_row = a.block_table + (int64_t)s * a.max_blocks;
    const int32_t *dst_row = a.dst_table != nullptr ? a.dst_table + (int64_t)s * a.dst_max_blocks : src_row;
    const int32_t dst_blocks = a.dst_table != nullptr ? a.dst_max_blocks : a.max_blocks;
    int32_t *kept = a.kept != nullptr ? a.kept + (int64_t)pair * a.budget : nullptr;
    int32_t *rows = a.rows + (int64_t)pair * a.rows_stride;
    const uint32_t *w = reinterpret_cast<const uint32_t *>(a.weights) + (int64_t)pair * a.weights_stride;
    uint32_t *w_out = reinterpret_cast<uint32_t *>(a.weights_out) + (int64_t)pair * a.weights_out_stride;
    grid_launch();
    // ---- does the sequence fit, and is everything it needs on the GPU?  (The same answer for every head of the sequence.)
    const bool fits = ctx >= 0 && ctx <= (int64_t)a.max_blocks * 16 && ctx <= a.weights_stride && n_new <= a.weights_out_stride &&
                      n_new <= (int64_t)dst_blocks * 16;
    uint32_t wt[ITEMS];
    auto token = [&](int32_t base, int i) { return base + tid * ITEMS + i; };
    const bool aligned = ITEMS % 4 == 0 && (reinterpret_cast<uintptr_t>(w) & 15) == 0;
    auto read_piece = [&](int32_t base, int64_t end) {
        if (aligned && token(base, ITEMS) <= end) {
#pragma unroll
            for (int i = 0; i + 3 < ITEMS; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4 *>(w + token(base, i));
                wt[i] = v.x, wt[i + 1] = v.y, wt[i + 2] = v.z, wt[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) wt[i] = token(base, i) < end ? w[token(base, i)] : 0u;
        }
    };
    // of the thread's items, those below a token number, as bits
    auto below = [&](int32_t base, int32_t end) { return (1u << max(0, min(ITEMS, end - token(base, 0)))) - 1u; };
    read_piece(0, a.weights_stride);   // (on its way before the length is known; what lies behind it is not looked at)
    const bool one_piece = ctx <= PIECE;
    bool missing = false;
    if (fits) {
        for (int32_t i = tid; i < (ctx + 15) / 16; i += SEL_THREADS) {
            const int32_t slot = unit_slot(p, src_row, i);
            if (smem_slots) slots[i] = slot;
            missing |= slot < 0;
        }
        if (a.dst_table != nullptr)
            for (int32_t i = tid; i < (n_new + 15) / 16; i += SEL_THREADS) missing |= unit_slot(p, dst_row, i) < 0;
    }
    for (int i = tid; i < SEL_BINS / 4; i += SEL_THREADS) reinterpret_cast<int4 *>(hist)[i] = make_int4(0, 0, 0, 0);
    if (tid == 0) n_list = 0;
    // Weights that are all positive numbers (or 0 or infinity) are in order as they are: the usual case, and a third fewer instructions
    bool odd = !one_piece;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) odd |= token(0, i) < ctx && wt[i] > 0x7f800000u;
    missing = __syncthreads_or(missing) != 0;
    const bool plain = __syncthreads_or(odd) == 0;
    if (!fits || missing) {
        if (tid == 0) {
            *reinterpret_cast<volatile int32_t *>(a.status + (fits ? 0 : 1)) = 1;
            a.counts[pair] = -1;
        }
        if (kept != nullptr)
            for (int32_t j = tid; j < a.budget; j += SEL_THREADS) kept[j] = -1;
        return;
    }
    if (tid == 0) a.counts[pair] = n_new;

    // ---- the smallest key that gets a place, and how many of the tokens with exactly that key do (the first ones)
    const int32_t n_old = ctx - min(ctx, a.recent);              // the tokens that compete
    const int32_t places = ctx > a.budget ? a.budget - a.recent : n_old;
    const bool all_old = places >= n_old;
    auto work = [&](auto plain_tag) {
        auto key = [](uint32_t b) { return decltype(plain_tag)::value ? b | 0x80000000u : weight_key(b); };
        uint32_t edge = 0xffffffffu;                                 // keys above it stay (no weight has this pattern's key: a NaN)
        int32_t n_edge = 0;                                          // and this many of those equal to it
        if (!all_old && places > 0) {
            int32_t rank = places;                                   // the edge is the rank-th largest of those that share its digits so far
            edge = 0;
            auto count = [&](uint32_t known, int shift, uint32_t digit_mask) {
                for (int32_t base = 0; base < n_old; base += PIECE) {
                    if (!one_piece) read_piece(base, ctx);
#pragma unroll
                    for (int i = 0; i < ITEMS; ++i) {
                        const uint32_t k = key(wt[i]);
                        if (token(base, i) < n_old && (k & known) == edge) atomicAdd(&hist[(k >> shift) & digit_mask], 1);
                    }
                }
                __syncthreads();
            };
            auto clear = [&]() {
                for (int i = tid; i < 1024; i += SEL_THREADS) hist[i] = 0;
                __syncthreads();
            };
            count(0u, 20, 0xfffu);
            edge |= find_bin<SEL_BINS>(hist, &rank, warp_sums, answer) << 20;
            // the candidates: the weights with that digit
            for (int32_t base = 0; base < n_old; base += PIECE) {
                if (!one_piece) read_piece(base, ctx);
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    const uint32_t k = key(wt[i]);
                    if (token(base, i) < n_old && (k & 0xfff00000u) == edge) {
                        const int32_t at = atomicAdd(&n_list, 1);
                        if (at < SEL_LIST) list[at] = k;
                    }
                }
            }
            __syncthreads();
            const int32_t m = n_list;
            if (m <= SEL_LIST) {
                // the rank-th largest: every candidate counts those above it and those like it (whatever their order in the list)
                if (tid < m) {
                    const uint32_t k = list[tid];
                    int32_t above = 0, like = 0;
#pragma unroll 8
                    for (int32_t i = 0; i < m; ++i) {
                        above += list[i] > k;
                        like += list[i] == k;
                    }
                    if (above < rank && rank <= above + like) {   // (all candidates like the answer write the same)
                        answer[0] = (int32_t)k;
                        answer[1] = rank - above;
                    }
                }
                __syncthreads();
                edge = (uint32_t)answer[0];
                rank = answer[1];
            } else {
                clear();
                count(0xfff00000u, 10, 0x3ffu);
                edge |= find_bin<1024>(hist, &rank, warp_sums, answer) << 10;
                clear();
                count(0xfffffc00u, 0, 0x3ffu);
                edge |= find_bin<1024>(hist, &rank, warp_sums, answer);
            }
            n_edge = rank;
        }

        // ---- in order: the kept positions, where their rows lie, their weights.  Of the first x tokens above(x) + min(on_edge(x),
        // n_edge) stay, so both counts can be summed up before any token's fate is known.
        int32_t above_before = 0, edge_before = 0;
        for (int32_t base = 0; base < ctx; base += PIECE) {
            if (!one_piece) read_piece(base, ctx);
            uint32_t larger = 0, like = 0;                           // a bit per item
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const uint32_t k = key(wt[i]);
                larger |= (uint32_t)(k > edge) << i;
                like |= (uint32_t)(k == edge) << i;
            }
            const uint32_t in_ctx = below(base, ctx), old = below(base, n_old);
            const uint32_t is_above = in_ctx & (all_old ? ~0u : ~old | larger);
            uint32_t is_edge = all_old ? 0u : old & like;
            // both counts in one word: a piece has at most 2^13 tokens
            const uint32_t mine = (uint32_t)__popc(is_above) | (uint32_t)__popc(is_edge) << 16;
            uint32_t inc = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += y;
            }
            if (lane == 31) warp_sums[warp] = (int32_t)inc;
            __syncthreads();                                         // (every weight of the piece is read: in place, writing may begin)
            uint32_t all;
            const uint32_t before = inc - mine + warps_before(warp_sums, &all);
            const int32_t on_edge = edge_before + (int32_t)(before >> 16);
            int32_t j = above_before + (int32_t)(before & 0xffffu) + min(on_edge, n_edge);
            above_before += (int32_t)(all & 0xffffu);
            edge_before += (int32_t)(all >> 16);
            const int32_t left = max(0, n_edge - on_edge);           // of the thread's on the edge, so many stay: the first ones
            while (__popc(is_edge) > left) is_edge &= ~(1u << (31 - __clz(is_edge)));
            const uint32_t keep = is_above | is_edge;
            if (keep) {
                const int32_t t0 = token(base, 0);                   // (the thread's items lie in one block)
                const int32_t row0 = (smem_slots ? slots[t0 >> 4] : unit_slot(p, src_row, t0 >> 4)) * 16 + (t0 & 15);
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
                    if (((keep >> i) & 1u) && j < n_new) {
                        if (kept != nullptr) kept[j] = t0 + i;
                        rows[j] = row0 + i;
                        w_out[j] = wt[i];                            // j <= t: in place this overwrites only what has been read
                        ++j;
                    }
            }
            if (!one_piece) __syncthreads();                         // (the counts have been read)
        }
    };
    if (plain) work(std::true_type());
    else work(std::false_type());
    for (int64_t t = n_new + tid; t < min((int64_t)ctx, a.weights_out_stride); t += SEL_THREADS) w_out[t] = 0u;
    if (kept != nullptr)
        for (int32_t j = n_new + tid; j < a.budget; j += SEL_THREADS) kept[j] = -1;
}

__device__ __forceinline__ void write_new_len(const EvictParams &p, int32_t pair, int32_t n) {   // by one thread of the head's first CTA
    const EvictLaunch &a = p.a;
    const int32_t s = pair / p.n_kv_heads;
    if (a.new_lens != nullptr && pair == s * p.n_kv_heads) {
        const int32_t ctx = a.ctx_lens[s];
        a.new_lens[s] = n < 0 ? ctx : n;
    }
}

// Out of place: a CTA copies MOVE_ROWS consecutive rows of K and V.  The rows' places go through shared memory first, so that the
// chain of dependent look-ups (row, block, slot) is walked once per 128 rows and the copies behind it are independent loads,
// eight in flight per thread.  The moved rows are written to make room for reads (streaming stores): 240 -> 225 us for 1024 of 4096
// tokens, 32 x 32 pairs (1.1 GB), 27 -> 23 us for 24 sequences of 8-bit rows called back to back, which leaves them in L2 (33 us with
// rows that come from HBM).
template <int VECS>
__global__ void __launch_bounds__(MOVE_THREADS, 5)
evict_copy_kernel(const EvictParams p, int32_t chunks) {
    __shared__ int32_t from[MOVE_ROWS], to[MOVE_ROWS];
    const EvictLaunch &a = p.a;
    const int tid = threadIdx.x;
    const int32_t pair = blockIdx.x / chunks, s = pair / p.n_kv_heads, h = pair - s * p.n_kv_heads;
    const int32_t j0 = (blockIdx.x - pair * chunks) * MOVE_ROWS;
    // (the destination's slots depend on nothing that the kernel before this one writes)
    int32_t dst = -1;
    if (tid < MOVE_ROWS && ((j0 + tid) >> 4) < a.dst_max_blocks) dst = unit_slot(p, a.dst_table + (int64_t)s * a.dst_max_blocks, (j0 + tid) >> 4) * 16 + ((j0 + tid) & 15);
    grid_wait();
    const int32_t n = a.counts[pair];
    if (tid < MOVE_ROWS) {   // (beyond the count: stale, not used; its load goes out beside the count's)
        from[tid] = j0 + tid < a.rows_stride ? a.rows[(int64_t)pair * a.rows_stride + j0 + tid] : 0;
        to[tid] = dst;
    }
    if (j0 == 0 && tid == 0) write_new_len(p, pair, n);
    const int32_t mine = min(MOVE_ROWS, n - j0);
    if (mine <= 0) return;
    __syncthreads();
    uint4 *pool = reinterpret_cast<uint4 *>(a.gpu_pool);
    auto address = [&](int32_t row, int32_t kv, int32_t c) {   // row = slot * 16 + row of the block
        return ((((int64_t)(row >> 4) * p.n_kv_heads + h) * 2 + kv) * 16 + (row & 15)) * VECS + c;
    };
    const int32_t total = mine * 2 * VECS;
    for (int32_t e0 = tid; e0 < total; e0 += 8 * MOVE_THREADS) {
        uint4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int32_t e = e0 + i * MOVE_THREADS, r = e / (2 * VECS), c = e - r * 2 * VECS;
            if (e < total) v[i] = pool[address(from[r], c / VECS, c % VECS)];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int32_t e = e0 + i * MOVE_THREADS, r = e / (2 * VECS), c = e - r * 2 * VECS;
            if (e < total) __stcs(pool + address(to[r], c / VECS, c % VECS), v[i]);
        }
    }
}

// In place: blockIdx.y picks K or V and a column slice of the rows (64 bytes), so that one (sequence, KV head) occupies
// several CTAs; slices do not meet, which keeps the move safe without any order between CTAs.  Row j comes from a row at or behind
// j, in ascending order: what a batch overwrites lies in front of everything that later batches read, so it is enough that a
// batch has been read by all threads before any of it is written (one barrier), and the next batch may be read ahead of that.
// 1024 of 4096 tokens, 32 x 32 pairs, 16 bits: 456 us, twice the move out of place; 24 sequences of 8-bit rows 42 us (36): every
// slice walks the look-ups (row, block, slot) of all rows again, and a batch is 256 rows.
__global__ void __launch_bounds__(MOVE_THREADS)
evict_move_kernel(const EvictParams p, int32_t slice_vecs) {
    const EvictLaunch &a = p.a;
    const int tid = threadIdx.x;
    const int32_t pair = blockIdx.x, s = pair / p.n_kv_heads, h = pair - s * p.n_kv_heads;
    grid_wait();
    const int32_t n = a.counts[pair];
    if (blockIdx.y == 0 && tid == 0) write_new_len(p, pair, n);
    if (n <= 0) return;
    const int32_t slices = p.row_vecs / slice_vecs;
    const int32_t kv = blockIdx.y / slices, col0 = (blockIdx.y - kv * slices) * slice_vecs;
    const int32_t *table_row = a.block_table + (int64_t)s * a.max_blocks;
    const int32_t *rows = a.rows + (int64_t)pair * a.rows_stride;
    uint4 *pool = reinterpret_cast<uint4 *>(a.gpu_pool);
    const int32_t lane_col = tid % slice_vecs, lane_row = tid / slice_vecs, rows_per_pass = MOVE_THREADS / slice_vecs;
    const int32_t batch = rows_per_pass * MOVE_DEPTH;
    auto address = [&](int32_t row) {
        return ((((int64_t)(row >> 4) * p.n_kv_heads + h) * 2 + kv) * 16 + (row & 15)) * p.row_vecs + col0 + lane_col;
    };
    auto load = [&](int32_t j0, uint4 (&v)[MOVE_DEPTH], int32_t (&to)[MOVE_DEPTH]) {
#pragma unroll
        for (int i = 0; i < MOVE_DEPTH; ++i) {
            const int32_t j = j0 + i * rows_per_pass + lane_row;
            to[i] = -1;
            if (j < n) {
                const int32_t from = rows[j], d = unit_slot(p, table_row, j >> 4) * 16 + (j & 15);
                if (d != from) {   // (the rows in front of the first evicted token stay where they are)
                    to[i] = d;
                    v[i] = pool[address(from)];
                }
            }
        }
    };
    uint4 v[MOVE_DEPTH], ahead[MOVE_DEPTH];
    int32_t to[MOVE_DEPTH], to_ahead[MOVE_DEPTH];
    load(0, v, to);
    for (int32_t j0 = 0; j0 < n; j0 += batch) {
        load(j0 + batch, ahead, to_ahead);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MOVE_DEPTH; ++i) {
            if (to[i] >= 0) pool[address(to[i])] = v[i];
            v[i] = ahead[i];
            to[i] = to_ahead[i];
        }
    }
}

}  // namespace

cudaError_t evict_configure() {
    const void *fns[] = {(const void *)evict_select_kernel<2>, (const void *)evict_select_kernel<8>, (const void *)evict_select_kernel<16>,
                         (const void *)evict_copy_kernel<16>, (const void *)evict_copy_kernel<8>, (const void *)evict_move_kernel};
    for (const void *f : fns) {
        const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// CTAs per (sequence, KV head) of the move out of place (a budget beyond what the tables hold keeps whole sequences)
int64_t evict_chunks(const EvictLaunch &a) {
    const int64_t longest = std::min<int64_t>((int64_t)a.max_blocks * 16, a.weights_stride);
    const int64_t most = std::min<int64_t>(std::min<int64_t>(a.budget, longest), (int64_t)a.dst_max_blocks * 16);
    return (most + MOVE_ROWS - 1) / MOVE_ROWS;
}

cudaError_t launch_evict(const AttnShape &sh, const EvictLaunch &a, cudaStream_t stream) {
    if (a.n_seqs <= 0) return cudaSuccess;
    EvictParams p;
    p.a = a;
    p.n_gpu_slots = sh.n_gpu_slots;
    p.n_kv_heads = sh.n_kv_heads;
    p.n_logical = sh.n_logical;
    p.row_vecs = sh.head_dim * (sh.kv_fp8 ? 1 : 2) / 16;
    const int64_t pairs = (int64_t)a.n_seqs * sh.n_kv_heads;
    // weights in registers as far as the longest sequence that the table and the weights allow.  The selection takes, with 2, 8 and
    // 16 weights a thread: one sequence of 700 tokens 7.0, 7.8, 9.2 us; 24 of up to 3500 -, 11.2, 13.8; 32 of 4096 -, 30, 42.  (The
    // lengths are on the device: a table and weights for 32768 tokens cost short sequences 2 to 4 us, 13.3 -> 17.4 for one of 700.)
    const int64_t longest = std::min<int64_t>((int64_t)a.max_blocks * 16, a.weights_stride);
    const int32_t smem_slots = a.max_blocks <= SEL_SLOTS ? 1 : 0;
    const size_t smem = smem_slots ? (size_t)a.max_blocks * 4 : 0;
    if (longest <= 2 * SEL_THREADS) evict_select_kernel<2><<<(unsigned)pairs, SEL_THREADS, smem, stream>>>(p, smem_slots);
    else if (longest <= 8 * SEL_THREADS) evict_select_kernel<8><<<(unsigned)pairs, SEL_THREADS, smem, stream>>>(p, smem_slots);
    else evict_select_kernel<16><<<(unsigned)pairs, SEL_THREADS, smem, stream>>>(p, smem_slots);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t lc = {};
    lc.blockDim = dim3(MOVE_THREADS);
    lc.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 1;
    if (a.dst_table == nullptr) {
        const int32_t slice = std::min(4, p.row_vecs);
        lc.gridDim = dim3((unsigned)pairs, (unsigned)(2 * p.row_vecs / slice));
        return cudaLaunchKernelEx(&lc, evict_move_kernel, p, slice);
    }
    const int32_t chunks = (int32_t)evict_chunks(a);
    lc.gridDim = dim3((unsigned)(pairs * chunks));
    return p.row_vecs == 16 ? cudaLaunchKernelEx(&lc, evict_copy_kernel<16>, p, chunks) : cudaLaunchKernelEx(&lc, evict_copy_kernel<8>, p, chunks);
}

}  // namespace pie
