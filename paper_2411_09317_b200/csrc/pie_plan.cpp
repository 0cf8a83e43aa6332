// Host-only halves of calls that launch kernels: argument checks and plans that need no GPU.
#include <cmath>
#include <cstdint>

#include "../../include/pie.h"

extern "C" {

int pie_rope_plan(int32_t head_dim, int32_t rotary_dim, const int32_t *pair_axis, const double *inv_freq, uint64_t *turns,
                  int32_t *n_axes) {
    if (!pair_axis || !inv_freq || !turns || !n_axes || rotary_dim <= 0 || rotary_dim > head_dim) return PIE_ERR_INVALID;
    if (rotary_dim % 16 != 0 || head_dim > 128) return PIE_ERR_UNSUPPORTED;   // the kernel turns eight pairs at a time
    int32_t top = 0;
    for (int32_t i = 0; i < rotary_dim / 2; ++i) {
        if (pair_axis[i] < 0 || pair_axis[i] >= PIE_ROPE_MAX_AXES || !std::isfinite(inv_freq[i])) return PIE_ERR_INVALID;
        top = pair_axis[i] > top ? pair_axis[i] : top;
    }
    for (int32_t i = 0; i < rotary_dim / 2; ++i) {
        // whole turns per position do not count: positions are whole numbers
        const long double turn = (long double)inv_freq[i] * 0.15915494309189533576888376337251436L;   // 1 / (2 pi)
        const long double scaled = std::floor(std::ldexp(turn - std::floor(turn), 64) + 0.5L);
        turns[i] = scaled >= 18446744073709551616.0L ? 0u : (uint64_t)scaled;
    }
    *n_axes = top + 1;
    return PIE_OK;
}
}
