// Host-only halves of calls that launch kernels: argument checks and plans that need no GPU.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

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

int pie_prompt_plan(const int32_t *offsets, int32_t n_seqs, int32_t item_tokens, int32_t *items, int64_t capacity,
                    int64_t *n_items) {
    if (n_seqs < 0 || item_tokens <= 0 || !n_items || (n_seqs > 0 && (!offsets || offsets[0] != 0))) return PIE_ERR_INVALID;
    int64_t n = 0, most = 0;   // items in all, items of the longest sequence
    for (int32_t s = 0; s < n_seqs; ++s) {
        const int64_t len = (int64_t)offsets[s + 1] - offsets[s];
        if (len < 0) return PIE_ERR_INVALID;
        const int64_t mine = (len + item_tokens - 1) / item_tokens;
        n += mine;
        most = mine > most ? mine : most;
    }
    *n_items = n;
    if (!items) return PIE_OK;
    if (n > capacity) return PIE_ERR_NOMEM;
    // The i-th item of a sequence sees about i * item_tokens keys: rank by rank from the last, so that the launch ends with
    // the short ones.  (Sequences in order within a rank: their items lie beside each other in memory.)
    try {
        std::vector<int32_t> live;   // the sequences that have an item of the rank
        std::vector<int32_t> by_rank(n_seqs);
        for (int32_t s = 0; s < n_seqs; ++s) by_rank[(size_t)s] = s;
        std::stable_sort(by_rank.begin(), by_rank.end(), [&](int32_t a, int32_t b) {
            return offsets[a + 1] - offsets[a] > offsets[b + 1] - offsets[b];
        });
        size_t next = 0;
        int64_t at = 0;
        for (int64_t rank = most - 1; rank >= 0; --rank) {
            while (next < by_rank.size() && (int64_t)offsets[by_rank[next] + 1] - offsets[by_rank[next]] > rank * item_tokens) live.push_back(by_rank[next++]);
            for (int32_t s : live) {
                items[4 * at] = offsets[s];
                items[4 * at + 1] = (int32_t)(rank * item_tokens);
                items[4 * at + 2] = offsets[s + 1] - offsets[s];
                items[4 * at + 3] = s;
                ++at;
            }
        }
    } catch (const std::bad_alloc &) {
        return PIE_ERR_NOMEM;
    }
    return PIE_OK;
}
}
