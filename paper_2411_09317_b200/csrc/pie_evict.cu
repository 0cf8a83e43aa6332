// Eviction from the paged cache by accumulated attention weight: per (sequence, KV head) the newest `recent` tokens stay, and of
// the older ones the budget - recent with the largest weights; the kept tokens' keys, values and weights move to the front.
//
// Two kernels.  evict_select_kernel, one CTA per (sequence, KV head): the weight of the last token that still gets a place is
// found digit by digit (radix select: four passes of 256 counters over the weights' order-preserving bit patterns - exact,
// whatever their distribution, where a sort would move every weight several times), then one pass over the tokens in order
// writes the kept positions, their weights and the cache rows they lie in.  evict_move_kernel copies the rows.
#include <algorithm>

#include "../../include/pie.h"
#include "pie_kernels.h"

namespace pie {

namespace {

constexpr int SEL_THREADS = 512;
constexpr int SEL_WARPS = SEL_THREADS / 32;
constexpr int MOVE_THREADS = 256;
constexpr int MOVE_DEPTH = 4;   // 16-byte vectors a thread holds

struct EvictParams {
    EvictLaunch a;
    int64_t n_gpu_slots;
    int32_t n_kv_heads, n_logical, row_vecs;   // row_vecs: 16-byte vectors of one K (or V) row
};

// bit patterns in the order of the values (-0 and 0 alike); NaN below everything.  By integers throughout: float arithmetic
// would flush subnormal weights, which a long decayed tail has, to one and the same zero.
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t b = __float_as_uint(w), magnitude = b & 0x7fffffffu;
    if (magnitude > 0x7f800000u) return 0u;
    return magnitude == 0u ? 0x80000000u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ int32_t unit_slot(const EvictParams &p, const int32_t *table_row, int32_t i) {
    const int32_t b = __ldg(table_row + i);
    const int32_t slot = (b >= 0 && b < p.n_logical) ? __ldcg(p.a.slot_table + b) : -1;
    return slot < p.n_gpu_slots ? slot : -1;
}

// Exclusive prefix sum over the CTA of one count per thread; *total: the CTA's sum.  Two barriers.
__device__ __forceinline__ int32_t block_scan(int32_t x, int32_t *total, int32_t *warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    int32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < SEL_WARPS; ++w) {
        const int32_t v = warp_sums[w];
        before += w < warp ? v : 0;
        all += v;
    }
    __syncthreads();
    *total = all;
    return before + inc - x;
}

__global__ void __launch_bounds__(SEL_THREADS)
evict_select_kernel(const EvictParams p) {
    __shared__ int32_t hist[256];
    __shared__ int32_t warp_sums[SEL_WARPS];
    __shared__ uint32_t sh_digit;
    __shared__ int32_t sh_rank;
    const EvictLaunch &a = p.a;
    const int tid = threadIdx.x;
    const int32_t pair = blockIdx.x, s = pair / p.n_kv_heads;
    const int32_t ctx = __ldg(a.ctx_lens + s), n_new = min(ctx, a.budget);
    const int32_t *src_row = a.block_table + (int64_t)s * a.max_blocks;
    const int32_t *dst_row = a.dst_table != nullptr ? a.dst_table + (int64_t)s * a.dst_max_blocks : src_row;
    const int32_t dst_blocks = a.dst_table != nullptr ? a.dst_max_blocks : a.max_blocks;
    int32_t *kept = a.kept != nullptr ? a.kept + (int64_t)pair * a.budget : nullptr;
    int32_t *rows = a.rows + (int64_t)pair * a.budget;
    // ---- does the sequence fit, and is everything it needs on the GPU?  (The same answer for every head of the sequence.)
    const bool fits = ctx >= 0 && (ctx + 15) / 16 <= a.max_blocks && ctx <= a.weights_stride && n_new <= a.weights_out_stride &&
                      (n_new + 15) / 16 <= dst_blocks;
    bool missing = false;
    if (fits) {
        for (int32_t i = tid; i < (ctx + 15) / 16; i += SEL_THREADS) missing |= unit_slot(p, src_row, i) < 0;
        if (a.dst_table != nullptr)
            for (int32_t i = tid; i < (n_new + 15) / 16; i += SEL_THREADS) missing |= unit_slot(p, dst_row, i) < 0;
    }
    missing = __syncthreads_or(missing) != 0;
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
    const float *w = a.weights + (int64_t)pair * a.weights_stride;
    float *w_out = a.weights_out + (int64_t)pair * a.weights_out_stride;

    // ---- the smallest key that gets a place, and how many of the tokens with exactly that key do (the first ones)
    const int32_t n_old = ctx - min(ctx, a.recent);              // the tokens that compete
    int32_t places = ctx > a.budget ? a.budget - a.recent : n_old;
    uint32_t edge = 0;                                          // keys above it stay
    int32_t n_edge = 0;                                         // and this many of those equal to it
    if (places < n_old && places > 0) {
        int32_t rank = places;                                  // the edge is the rank-th largest of those that share its prefix
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += SEL_THREADS) hist[i] = 0;
            __syncthreads();
            const uint32_t prefix_mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            for (int32_t t = tid; t < n_old; t += SEL_THREADS) {
                const uint32_t k = weight_key(w[t]);
                if ((k & prefix_mask) == edge) atomicAdd(&hist[(k >> shift) & 255u], 1);
            }
            __syncthreads();
            if (tid < 32) {   // the digit at which the count from above reaches the rank
                int32_t mine = 0;
                for (int i = 0; i < 8; ++i) mine += hist[255 - (8 * tid + i)];
                int32_t inc = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int32_t y = __shfl_up_sync(0xffffffffu, inc, o);
                    if (tid >= o) inc += y;
                }
                int32_t above = inc - mine;
                if (above < rank && rank <= inc) {
                    for (int i = 0; i < 8; ++i) {
                        const int32_t c = hist[255 - (8 * tid + i)];
                        if (rank <= above + c) {
                            sh_digit = 255u - (8 * tid + i);
                            sh_rank = rank - above;
                            break;
                        }
                        above += c;
                    }
                }
            }
            __syncthreads();
            edge |= sh_digit << shift;
            rank = sh_rank;
            __syncthreads();
        }
        n_edge = rank;
    }
    const bool all_old = places >= n_old, no_old = places <= 0;

    // ---- in order: the kept positions, where their rows lie, their weights
    int32_t kept_before = 0, edge_before = 0;
    for (int32_t base = 0; base < ctx; base += SEL_THREADS) {
        const int32_t t = base + tid;
        const float wt = t < ctx ? w[t] : 0.f;
        const uint32_t k = weight_key(wt);
        const bool recent = t >= n_old && t < ctx, old = t < n_old;
        const bool on_edge = old && !all_old && !no_old && k == edge;
        int32_t n_on_edge, n_kept;
        const int32_t edge_rank = edge_before + block_scan(on_edge, &n_on_edge, warp_sums);
        const bool keep = recent || (old && !no_old && (all_old || k > edge || (on_edge && edge_rank < n_edge)));
        const int32_t j = kept_before + block_scan(keep, &n_kept, warp_sums);   // (its barriers: every weight of this pass is read)
        if (keep && j < n_new) {
            if (kept != nullptr) kept[j] = t;
            rows[j] = unit_slot(p, src_row, t >> 4) * 16 + (t & 15);
            w_out[j] = wt;                                       // j <= t: in place this overwrites only what has been read
        }
        edge_before += n_on_edge;
        kept_before += n_kept;
    }
    for (int64_t t = n_new + tid; t < min((int64_t)ctx, a.weights_out_stride); t += SEL_THREADS) w_out[t] = 0.f;
    if (kept != nullptr)
        for (int32_t j = n_new + tid; j < a.budget; j += SEL_THREADS) kept[j] = -1;
}

// Row slices: blockIdx.y picks K or V and a column slice of the rows (64 bytes), so that one (sequence, KV head) occupies
// several CTAs; slices do not meet, which keeps the move in place safe without any order between CTAs.  In place, row j comes
// from a row at or behind j, in ascending order: what a batch overwrites lies in front of everything that later batches
// read, so it is enough that a batch has been read by all threads before any of it is written (one barrier), and later batches
// may be read ahead of that.
template <bool IN_PLACE>
__global__ void __launch_bounds__(MOVE_THREADS)
evict_move_kernel(const EvictParams p, int32_t slice_vecs) {
    const EvictLaunch &a = p.a;
    const int tid = threadIdx.x;
    const int32_t pair = blockIdx.x, s = pair / p.n_kv_heads, h = pair - s * p.n_kv_heads;
    const int32_t n = a.counts[pair];
    if (blockIdx.y == 0 && blockIdx.z == 0 && h == 0 && tid == 0 && a.new_lens != nullptr) {
        const int32_t ctx = a.ctx_lens[s];
        a.new_lens[s] = n < 0 ? ctx : n;
    }
    if (n <= 0) return;
    const int32_t slices = p.row_vecs / slice_vecs;
    const int32_t kv = blockIdx.y / slices, col0 = (blockIdx.y - kv * slices) * slice_vecs;
    const int32_t *dst_row = a.dst_table != nullptr ? a.dst_table + (int64_t)s * a.dst_max_blocks : a.block_table + (int64_t)s * a.max_blocks;
    const int32_t *rows = a.rows + (int64_t)pair * a.budget;
    uint4 *pool = reinterpret_cast<uint4 *>(a.gpu_pool);
    const int32_t lane_col = tid % slice_vecs, lane_row = tid / slice_vecs, rows_per_pass = MOVE_THREADS / slice_vecs;
    const int32_t batch = rows_per_pass * MOVE_DEPTH;
    auto address = [&](int32_t row) {   // row = slot * 16 + row of the block
        return ((((int64_t)(row >> 4) * p.n_kv_heads + h) * 2 + kv) * 16 + (row & 15)) * p.row_vecs + col0 + lane_col;
    };
    for (int32_t j0 = IN_PLACE ? 0 : (int32_t)blockIdx.z * batch; j0 < n; j0 += IN_PLACE ? batch : (int32_t)gridDim.z * batch) {
        uint4 v[MOVE_DEPTH];
        int32_t to[MOVE_DEPTH];
#pragma unroll
        for (int i = 0; i < MOVE_DEPTH; ++i) {
            const int32_t j = j0 + i * rows_per_pass + lane_row;
            to[i] = -1;
            if (j < n) {
                const int32_t from = rows[j];
                const int32_t d = unit_slot(p, dst_row, j >> 4) * 16 + (j & 15);
                if (d != from) {
                    to[i] = d;
                    v[i] = pool[address(from)];
                }
            }
        }
        if (IN_PLACE) __syncthreads();
#pragma unroll
        for (int i = 0; i < MOVE_DEPTH; ++i)
            if (to[i] >= 0) pool[address(to[i])] = v[i];
        if (IN_PLACE) __syncthreads();
    }
}

}  // namespace

cudaError_t evict_configure() {
    const void *fns[] = {(const void *)evict_select_kernel, (const void *)evict_move_kernel<true>, (const void *)evict_move_kernel<false>};
    for (const void *f : fns) {
        const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_evict(const AttnShape &sh, const EvictLaunch &a, int n_sms, cudaStream_t stream) {
    if (a.n_seqs <= 0) return cudaSuccess;
    EvictParams p;
    p.a = a;
    p.n_gpu_slots = sh.n_gpu_slots;
    p.n_kv_heads = sh.n_kv_heads;
    p.n_logical = sh.n_logical;
    p.row_vecs = sh.head_dim * (sh.kv_fp8 ? 1 : 2) / 16;
    const int64_t pairs = (int64_t)a.n_seqs * sh.n_kv_heads;
    evict_select_kernel<<<(unsigned)pairs, SEL_THREADS, 0, stream>>>(p);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    if (a.dst_table == nullptr) {
        const int32_t slice = std::min(4, p.row_vecs);
        evict_move_kernel<true><<<dim3((unsigned)pairs, (unsigned)(2 * p.row_vecs / slice)), MOVE_THREADS, 0, stream>>>(p, slice);
    } else {
        const int32_t slice = p.row_vecs, batch = MOVE_THREADS / slice * MOVE_DEPTH;
        const int64_t z = std::max<int64_t>(1, std::min<int64_t>((a.budget + batch - 1) / batch, (8 * n_sms + 2 * pairs - 1) / (2 * pairs)));
        evict_move_kernel<false><<<dim3((unsigned)pairs, 2, (unsigned)z), MOVE_THREADS, 0, stream>>>(p, slice);
    }
    return cudaGetLastError();
}

}  // namespace pie
