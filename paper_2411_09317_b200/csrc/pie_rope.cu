// Rotary positions of several axes (time, height, width ...) fused with the write into the paged cache.
//
// A token's pair i turns by positions[axis(i)][token] * f_i.  The frequencies come as 2^64-ths of a turn per position, so the
// angle is one 64-bit integer product whose low word IS the fraction of a turn: far positions lose nothing (an fp32
// product has no fraction left at 2^24 radians and is off by 0.06 at a million), and no range reduction is needed before
// sincospif, whose fp32 argument is off by 2^-26 of a turn at most.
//
// The work is moving bytes: q, k and v are read once, q_out, k_out and the cache rows written once.  A CTA takes T consecutive
// tokens.  It first puts the cosines and sines of its tokens' pairs into shared memory - all heads share them, and evaluating
// them per head would cost more instructions than everything else.  Then a thread keeps one place of the head (16 elements, both
// halves of eight pairs in either pair layout) of one token, with the pairs' factors in registers, and walks over heads: two
// 16-byte loads and two 16-byte stores per destination each, the next heads' loads in flight.  The query heads come first: the
// chain of look-ups that ends in the token's cache row (sequence, block, slot: three dependent loads) hides behind them.
// Bound: bytes.  16411 tokens of 64 + 8 + 8 heads of 128 (706 MB) in 135 us, 5.2 TB/s, 81 % of a plain copy's rate; 2045 tokens of
// 32 + 8 + 8 into an 8-bit cache (50 MB) in 15.5 us, half the floor's speed: launch, the wait for the positions and one wave's tail.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <type_traits>

#include "../../include/pie.h"
#include "pie_kernels.h"

namespace pie {

namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_AHEAD = 2;        // query heads whose loads are in flight (and one of the keys' and values')

struct RopeParams {
    RopeTable table;
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_out;
    const int32_t *positions, *token_seq, *token_pos, *block_table, *slot_table;
    uint8_t *pool;
    int32_t *status;
    int64_t n_tokens, q_stride, k_stride, v_stride, n_gpu_slots;
    int32_t n_q_heads, n_kv_heads, head_dim, max_blocks, n_seqs, n_logical;
    float k_scale, v_scale;
    float k_inv, v_inv;      // 1 / scale where that is exact (a power of two), else 0
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
// eight values -> eight E4M3 bytes of value / scale: the append's rule (fp32 quotient, nearest even, saturating).  The product
// with the reciprocal of a power of two is that quotient; for other scales it would not always be.
__device__ __forceinline__ uint2 rope_pack8(const float (&x)[8], float scale, float inv) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = inv != 0.f ? x[2 * i] * inv : __fdiv_rn(x[2 * i], scale), hi = inv != 0.f ? x[2 * i + 1] * inv : __fdiv_rn(x[2 * i + 1], scale);
        uint16_t r;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
        b[i] = r;
    }
    return make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
}

template <int D, int T, bool BF16, bool KV8>
__global__ void __launch_bounds__(ROPE_THREADS, 4)
rope_kv_kernel(const __grid_constant__ RopeParams p) {
    constexpr int PLACES = D / 16, LANES = ROPE_THREADS / (PLACES * T);   // threads per head and token; heads side by side
    __shared__ __align__(16) float2 cs[T][D / 2];
    __shared__ int32_t place[T];   // slot * 16 + row of the token, -1: not written
    const int tid = threadIdx.x;
    const int64_t t0 = (int64_t)blockIdx.x * T;
    const int nt = (int)min((int64_t)T, p.n_tokens - t0);
    const int pairs = p.table.rotary_dim >> 1;
    const int j = tid % PLACES, tt = tid / PLACES % T, lane = tid / (PLACES * T);
    const int64_t t = t0 + tt;
    const bool live = tt < nt;
    const int hq = live && p.q != nullptr ? p.n_q_heads : 0, hk = p.k != nullptr ? p.n_kv_heads : 0;
    const int hkv = live ? hk + (p.block_table != nullptr ? p.n_kv_heads : 0) : 0;   // the key heads, then the value heads
    const int rot = p.table.rotary_dim >> 4;
    const bool turned = j < rot, adjacent = p.table.adjacent != 0;
    // the two vectors of eight that a turned place consists of (one that is passed through: 2 j, 2 j + 1)
    const int ta = turned && !adjacent ? j : 2 * j, tb = turned && !adjacent ? j + rot : 2 * j + 1;
    const uint16_t *src_q = p.q + t * p.q_stride, *src_k = p.k + t * p.k_stride, *src_v = p.v + t * p.v_stride;
    auto load_q = [&](int head, uint4 &wa, uint4 &wb) {
        const uint4 *row = reinterpret_cast<const uint4 *>(src_q + head * D);
        wa = row[ta];
        wb = row[tb];
    };
    auto load_kv = [&](int head, uint4 &wa, uint4 &wb) {
        const bool is_v = head >= hk;
        const uint4 *row = reinterpret_cast<const uint4 *>(is_v ? src_v + (head - hk) * D : src_k + head * D);
        wa = row[is_v ? 2 * j : ta];
        wb = row[is_v ? 2 * j + 1 : tb];
    };
    uint4 qa[ROPE_AHEAD], qb[ROPE_AHEAD], ka, kb;
#pragma unroll
    for (int u = 0; u < ROPE_AHEAD; ++u)
        if (lane + u * LANES < hq) load_q(lane + u * LANES, qa[u], qb[u]);   // (in flight while the factors are worked out)
    if (lane < hkv) load_kv(lane, ka, kb);

    // the last warp's first lanes look the tokens' places up; the other warps work the factors out
    const int look = p.block_table != nullptr && tid >= ROPE_THREADS - 32 ? tid & 31 : T;
    int32_t s = 0, pos = 0;
    if (look < nt) {
        s = __ldg(p.token_seq + t0 + look);
        pos = __ldg(p.token_pos + t0 + look);
    }
    if (tid < ROPE_THREADS - 32) {
        for (int i = tid; i < T * (D / 2); i += ROPE_THREADS - 32) {
            const int it = i / (D / 2), pr = i % (D / 2);
            if (it < nt && pr < pairs) {
                const int32_t at = __ldg(p.positions + p.table.axis[pr] * p.n_tokens + t0 + it);
                const unsigned long long turn = (unsigned long long)(long long)at * p.table.turns[pr];
                float sn, cn;
                sincospif((float)(int32_t)(turn >> 32) * 4.656612873077393e-10f, &sn, &cn);   // 2^-31: half turns
                cs[it][pr] = make_float2(cn * p.table.amplitude, sn * p.table.amplitude);
            }
        }
    }
    __syncthreads();   // the factors
    if (look < nt) {   // (the places are wanted behind the query heads only)
        int32_t at = -1;
        if (s < 0 || s >= p.n_seqs || pos < 0 || (pos >> 4) >= p.max_blocks) {
            *reinterpret_cast<volatile int32_t *>(p.status + 1) = 1;
        } else {
            const int32_t b = __ldg(p.block_table + (int64_t)s * p.max_blocks + (pos >> 4));
            const int32_t slot = (b >= 0 && b < p.n_logical) ? __ldcg(p.slot_table + b) : -1;
            if (slot < 0 || slot >= p.n_gpu_slots) *reinterpret_cast<volatile int32_t *>(p.status) = 1;
            else at = slot * 16 + (pos & 15);
        }
        place[look] = at;
    }
    float2 c[8];
    if (turned && live) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float4 f = reinterpret_cast<const float4 *>(&cs[tt][8 * j])[e];
            c[2 * e] = make_float2(f.x, f.y);
            c[2 * e + 1] = make_float2(f.z, f.w);
        }
    }
    auto turn = [&](uint4 &wa, uint4 &wb, float (&a)[8], float (&b)[8]) {
        rope_unpack<BF16>(wa, a);
        rope_unpack<BF16>(wb, b);
        if (adjacent) {
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
    };
    for (int h0 = lane; h0 < hq; h0 += ROPE_AHEAD * LANES) {
#pragma unroll
        for (int u = 0; u < ROPE_AHEAD; ++u) {
            const int h = h0 + u * LANES;
            if (h < hq) {
                if (turned) {
                    float a[8], b[8];
                    turn(qa[u], qb[u], a, b);
                }
                uint4 *dst = reinterpret_cast<uint4 *>(p.q_out + (t * p.n_q_heads + h) * D);
                dst[ta] = qa[u];
                dst[tb] = qb[u];
                if (h + ROPE_AHEAD * LANES < hq) load_q(h + ROPE_AHEAD * LANES, qa[u], qb[u]);
            }
        }
    }
    __syncthreads();   // the tokens' places
    const int32_t at = p.block_table != nullptr && live ? place[tt] : -1;
    for (int head = lane; head < hkv; head += LANES) {
        const bool is_v = head >= hk;
        const int h = is_v ? head - hk : head, va = is_v ? 2 * j : ta, vb = is_v ? 2 * j + 1 : tb;
        uint4 wa = ka, wb = kb;
        if (head + LANES < hkv) load_kv(head + LANES, ka, kb);
        float a[8], b[8];
        if (turned && !is_v) {
            turn(wa, wb, a, b);
        } else if (KV8) {
            rope_unpack<BF16>(wa, a);
            rope_unpack<BF16>(wb, b);
        }
        if (!is_v && p.k_out != nullptr) {
            uint4 *dst = reinterpret_cast<uint4 *>(p.k_out + (t * p.n_kv_heads + h) * D);
            dst[va] = wa;
            dst[vb] = wb;
        }
        if (at >= 0) {
            const int64_t cache_row = (((int64_t)(at >> 4) * p.n_kv_heads + h) * 2 + (is_v ? 1 : 0)) * 16 + (at & 15);
            if (KV8) {
                const float sc = is_v ? p.v_scale : p.k_scale, inv = is_v ? p.v_inv : p.k_inv;
                uint2 *dst = reinterpret_cast<uint2 *>(p.pool + cache_row * D);
                dst[va] = rope_pack8(a, sc, inv);
                dst[vb] = rope_pack8(b, sc, inv);
            } else {
                uint4 *dst = reinterpret_cast<uint4 *>(p.pool + cache_row * D * 2);
                dst[va] = wa;
                dst[vb] = wb;
            }
        }
    }
}

template <typename F>
cudaError_t dispatch_rope(const AttnShape &sh, bool one, F &&f) {   // one token per CTA, or four
    auto by_type = [&](auto d, auto t) -> cudaError_t {
        constexpr int D = decltype(d)::value, T = decltype(t)::value;
        if (sh.kv_fp8) return sh.dtype == PIE_BF16 ? f(rope_kv_kernel<128, T, true, true>, T) : f(rope_kv_kernel<128, T, false, true>, T);
        return sh.dtype == PIE_BF16 ? f(rope_kv_kernel<D, T, true, false>, T) : f(rope_kv_kernel<D, T, false, false>, T);
    };
    using C64 = std::integral_constant<int, 64>;
    using C128 = std::integral_constant<int, 128>;
    using One = std::integral_constant<int, 1>;
    using Four = std::integral_constant<int, 4>;
    if (sh.head_dim == 128) return one ? by_type(C128(), One()) : by_type(C128(), Four());
    return one ? by_type(C64(), One()) : by_type(C64(), Four());
}

}  // namespace

cudaError_t rope_configure(const AttnShape &sh) {
    for (const bool one : {true, false}) {
        const cudaError_t e = dispatch_rope(sh, one, [](auto kernel, int) {
            return cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
        });
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
    auto exact_inverse = [](float x) {
        int e = 0;
        return std::frexp(x, &e) == 0.5f && e > -120 && e < 120 ? 1.f / x : 0.f;
    };
    p.k_inv = exact_inverse(a.k_scale);
    p.v_inv = exact_inverse(a.v_scale);
    // Tokens per CTA: four where a token has few rows per thread (one token per CTA, four: 32 + 8 + 8 heads of 128, 16411 tokens 98
    // and 86 us; 8 + 2 + 2: 77 and 35; 32 + 8 + 8 of 64: 68 and 47), one where a thread has two and a half of them anyway (64 + 8 + 8:
    // 134 and 137 us; 32 + 32 + 32: 170 and 182) and where four would leave SMs without a CTA (500 tokens, 32 + 32 + 32: 8.3 and 12.4
    // us; 64 + 8 + 8: 6.5 and 9.8).
    const bool one = a.n_tokens < 4 * n_sms || (sh.n_q_heads + 2 * sh.n_kv_heads) * sh.head_dim >= 40 * ROPE_THREADS;
    return dispatch_rope(sh, one, [&](auto kernel, int tokens) {
        const int64_t grid = (a.n_tokens + tokens - 1) / tokens;
        if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
        kernel<<<(unsigned)grid, ROPE_THREADS, 0, stream>>>(p);
        return cudaGetLastError();
    });
}

}  // namespace pie
