// Rotary positions of several axes (time, height, width ...) fused with the write into the paged cache.
//
// A token's pair i turns by positions[axis(i)][token] * f_i.  The frequencies come as 2^64-ths of a turn per position, so the
// angle is one 64-bit integer product whose low word IS the fraction of a turn: nothing is lost at far positions (an fp32
// product has no fraction left at 2^24 radians and is off by 0.06 at a million), and no range reduction is needed before
// sincospif.
//
// The work is moving bytes: q, k and v are read once, q_out, k_out and the cache rows written once.  A CTA takes a few
// consecutive tokens (and, where there are few tokens, a share of their heads).  It first puts the cosines and sines of
// its tokens' pairs into shared memory - they are shared by all heads, and evaluating them per head would cost more
// instructions than everything else - and then walks over (token, head, 16 elements): two 16-byte loads, which hold both
// elements of eight pairs in either pair layout, and two 16-byte stores per destination.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "../../include/pie.h"
#include "pie_kernels.h"

namespace pie {

namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_MAX_TOKENS = 8;   // tokens of a CTA at most (shared memory: 8 x 64 pairs x 8 bytes)

struct RopeParams {
    RopeTable table;
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_out;
    const int32_t *positions, *token_seq, *token_pos, *block_table, *slot_table;
    uint8_t *pool;
    int32_t *status;
    int64_t n_tokens, q_stride, k_stride, v_stride, n_gpu_slots;
    int32_t n_q_heads, n_kv_heads, head_dim, max_blocks, n_seqs, n_logical;
    int32_t tokens_per_cta;
    float k_scale, v_scale;
};

template <bool BF16>
__device__ __forceinline__ void rope_unpack(const uint4 &w, float (&x)[8]) {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) {
            x[2 * i] = __uint_as_float(a[i] << 16);
            x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&a[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
}
template <bool BF16>
__device__ __forceinline__ uint4 rope_pack(const float (&x)[8]) {
    uint32_t a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            a[i] = *reinterpret_cast<const uint32_t *>(&v);
        } else {
            const __half2 v = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            a[i] = *reinterpret_cast<const uint32_t *>(&v);
        }
    }
    return make_uint4(a[0], a[1], a[2], a[3]);
}
// eight values -> eight E4M3 bytes of value / scale: the append's rule (fp32 quotient, nearest even, saturating)
__device__ __forceinline__ uint2 rope_pack8(const float (&x)[8], float scale) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint16_t r;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(__fdiv_rn(x[2 * i + 1], scale)), "f"(__fdiv_rn(x[2 * i], scale)));
        b[i] = r;
    }
    return make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
}

template <bool BF16, bool KV8>
__global__ void __launch_bounds__(ROPE_THREADS)
rope_kv_kernel(const __grid_constant__ RopeParams p) {
    __shared__ float2 cs[ROPE_MAX_TOKENS][64];
    __shared__ int32_t place[ROPE_MAX_TOKENS];   // slot * 16 + row of the token, -1: not written
    const int tid = threadIdx.x;
    const int64_t t0 = (int64_t)blockIdx.x * p.tokens_per_cta;
    const int nt = (int)min((int64_t)p.tokens_per_cta, p.n_tokens - t0);
    const int pairs = p.table.rotary_dim >> 1;

    for (int i = tid; i < nt * pairs; i += ROPE_THREADS) {
        const int tt = i / pairs, pr = i - tt * pairs;
        const int32_t pos = __ldg(p.positions + p.table.axis[pr] * p.n_tokens + t0 + tt);
        const unsigned long long turn = (unsigned long long)(long long)pos * p.table.turns[pr];
        float s, c;
        sincospif((float)(int32_t)(turn >> 32) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns
        cs[tt][pr] = make_float2(c * p.table.amplitude, s * p.table.amplitude);
    }
    if (p.block_table != nullptr && tid >= ROPE_THREADS - 32 && (tid & 31) < nt) {
        const int tt = tid & 31;
        const int32_t s = __ldg(p.token_seq + t0 + tt), pos = __ldg(p.token_pos + t0 + tt);
        int32_t at = -1;
        if (s < 0 || s >= p.n_seqs || pos < 0 || (pos >> 4) >= p.max_blocks) {
            *reinterpret_cast<volatile int32_t *>(p.status + 1) = 1;
        } else {
            const int32_t b = __ldg(p.block_table + (int64_t)s * p.max_blocks + (pos >> 4));
            const int32_t slot = (b >= 0 && b < p.n_logical) ? __ldcg(p.slot_table + b) : -1;
            if (slot < 0 || slot >= p.n_gpu_slots) *reinterpret_cast<volatile int32_t *>(p.status) = 1;
            else at = slot * 16 + (pos & 15);
        }
        place[tt] = at;
    }
    __syncthreads();

    const int D = p.head_dim, per_head = D >> 4, rot = p.table.rotary_dim >> 4;   // items of 16 elements: all, rotated ones
    const int hq = p.q != nullptr ? p.n_q_heads : 0, hk = p.k != nullptr ? p.n_kv_heads : 0;
    const int hv = p.block_table != nullptr ? p.n_kv_heads : 0;
    const int per_token = (hq + hk + hv) * per_head;
    const int first = blockIdx.y * ROPE_THREADS + tid, step = gridDim.y * ROPE_THREADS;
    for (int i = first; i < nt * per_token; i += step) {
        const int tt = i / per_token, r = i - tt * per_token;
        const int head = r / per_head, j = r - head * per_head;
        const int64_t t = t0 + tt;
        const bool is_q = head < hq, is_v = head >= hq + hk;
        const int h = is_q ? head : is_v ? head - hq - hk : head - hq;
        const uint16_t *src = is_q ? p.q + t * p.q_stride : is_v ? p.v + t * p.v_stride : p.k + t * p.k_stride;
        // the item's two vectors of eight: both elements of eight pairs, or 16 elements behind the rotated ones
        const bool turned = !is_v && j < rot;
        const bool halves = turned && !p.table.adjacent;
        const int va = halves ? j : 2 * j, vb = halves ? j + rot : 2 * j + 1;
        const uint4 *row = reinterpret_cast<const uint4 *>(src + (int64_t)h * D);
        uint4 wa = row[va], wb = row[vb];
        float a[8], b[8];
        if (turned || KV8) {
            rope_unpack<BF16>(wa, a);
            rope_unpack<BF16>(wb, b);
        }
        if (turned) {
            const float4 *c4 = reinterpret_cast<const float4 *>(&cs[tt][8 * j]);
            float2 c[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 f = c4[e];
                c[2 * e] = make_float2(f.x, f.y);
                c[2 * e + 1] = make_float2(f.z, f.w);
            }
            if (p.table.adjacent) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x0 = a[2 * e], y0 = a[2 * e + 1], x1 = b[2 * e], y1 = b[2 * e + 1];
                    a[2 * e] = x0 * c[e].x - y0 * c[e].y;
                    a[2 * e + 1] = y0 * c[e].x + x0 * c[e].y;
                    b[2 * e] = x1 * c[4 + e].x - y1 * c[4 + e].y;
                    b[2 * e + 1] = y1 * c[4 + e].x + x1 * c[4 + e].y;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = a[e], y = b[e];
                    a[e] = x * c[e].x - y * c[e].y;
                    b[e] = y * c[e].x + x * c[e].y;
                }
            }
            wa = rope_pack<BF16>(a);
            wb = rope_pack<BF16>(b);
        }
        if (is_q) {
            uint4 *dst = reinterpret_cast<uint4 *>(p.q_out + (t * p.n_q_heads + h) * D);
            dst[va] = wa;
            dst[vb] = wb;
            continue;
        }
        if (!is_v && p.k_out != nullptr) {
            uint4 *dst = reinterpret_cast<uint4 *>(p.k_out + (t * p.n_kv_heads + h) * D);
            dst[va] = wa;
            dst[vb] = wb;
        }
        if (hv == 0 || place[tt] < 0) continue;
        const int32_t slot = place[tt] >> 4, tr = place[tt] & 15;
        const int64_t cache_row = (((int64_t)slot * p.n_kv_heads + h) * 2 + (is_v ? 1 : 0)) * 16 + tr;
        if (KV8) {
            const float sc = is_v ? p.v_scale : p.k_scale;
            uint2 *dst = reinterpret_cast<uint2 *>(p.pool + cache_row * D);
            dst[va] = rope_pack8(a, sc);
            dst[vb] = rope_pack8(b, sc);
        } else {
            uint4 *dst = reinterpret_cast<uint4 *>(p.pool + cache_row * D * 2);
            dst[va] = wa;
            dst[vb] = wb;
        }
    }
}

}  // namespace

cudaError_t rope_configure() {
    const void *fns[] = {(const void *)rope_kv_kernel<true, false>, (const void *)rope_kv_kernel<false, false>,
                         (const void *)rope_kv_kernel<true, true>, (const void *)rope_kv_kernel<false, true>};
    for (const void *f : fns) {
        const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_rope_kv(const AttnShape &sh, const RopeLaunch &a, const RopeTable &table, int n_sms, cudaStream_t stream) {
    if (a.n_tokens <= 0) return cudaSuccess;
    RopeParams p;
    p.table = table;
    p.q = (const uint16_t *)a.q;
    p.k = (const uint16_t *)a.k;
    p.v = (const uint16_t *)a.v;
    p.q_out = (uint16_t *)a.q_out;
    p.k_out = (uint16_t *)a.k_out;
    p.positions = a.positions;
    p.token_seq = a.token_seq;
    p.token_pos = a.token_pos;
    p.block_table = a.block_table;
    p.slot_table = a.slot_table;
    p.pool = (uint8_t *)a.gpu_pool;
    p.status = a.status;
    p.n_tokens = a.n_tokens;
    p.q_stride = a.q_stride;
    p.k_stride = a.k_stride;
    p.v_stride = a.v_stride;
    p.n_gpu_slots = sh.n_gpu_slots;
    p.n_q_heads = sh.n_q_heads;
    p.n_kv_heads = sh.n_kv_heads;
    p.head_dim = sh.head_dim;
    p.max_blocks = a.max_blocks;
    p.n_seqs = a.n_seqs;
    p.n_logical = sh.n_logical;
    p.k_scale = a.k_scale;
    p.v_scale = a.v_scale;
    const int64_t items = (int64_t)(sh.n_q_heads + 2 * sh.n_kv_heads) * (sh.head_dim / 16);
    p.tokens_per_cta = (int32_t)std::max<int64_t>(1, std::min<int64_t>(ROPE_MAX_TOKENS, a.n_tokens / (8 * n_sms)));
    const int64_t gx = (a.n_tokens + p.tokens_per_cta - 1) / p.tokens_per_cta;
    // few tokens: their heads are shared out among CTAs until there are about four per SM
    const int64_t rounds = (items * p.tokens_per_cta + ROPE_THREADS - 1) / ROPE_THREADS;
    const int64_t gy = std::max<int64_t>(1, std::min<int64_t>(rounds, 4 * n_sms / gx));
    if (gx > 0x7fffffffll) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)gx, (unsigned)gy);
    if (sh.kv_fp8) {
        if (sh.dtype == PIE_BF16) rope_kv_kernel<true, true><<<grid, ROPE_THREADS, 0, stream>>>(p);
        else rope_kv_kernel<false, true><<<grid, ROPE_THREADS, 0, stream>>>(p);
    } else {
        if (sh.dtype == PIE_BF16) rope_kv_kernel<true, false><<<grid, ROPE_THREADS, 0, stream>>>(p);
        else rope_kv_kernel<false, false><<<grid, ROPE_THREADS, 0, stream>>>(p);
    }
    return cudaGetLastError();
}

}  // namespace pie
