// Gradient norm and clipping: how many tensors' elements are shared out, and the checks of a call's list.  Plain C++: the host
// and the tests share it.
#pragma once

#include <algorithm>
#include <vector>

#include "log_probs_plan.h"
#include "shifter.h"

namespace shifter {

// A launch takes its tensors as arguments (4 KB of them), 24 bytes each: nothing is copied to the device and a recorded
// call keeps them.  Elements are counted in chunks, none of which has two tensors' elements; each block takes a run of
// chunks, as many as any other block or one less.
constexpr uint32_t GRAD_CHUNK = 2048;              // elements: eight for each thread of a block
constexpr uint32_t GRAD_SMALL = 4096;              // eights of elements, of all tensors, that one block holds
constexpr uint32_t GRAD_LIST = 164;                // tensors of a launch
constexpr uint32_t GRAD_BLOCKS = 512;              // of a launch at most; each leaves one sum
constexpr uint64_t GRAD_HEAD = 256;                // bytes between the counters and the sums: the norm in 64 bits

struct GradList {
    uint32_t low[3][GRAD_LIST];                    // addresses of the elements, of the results and of the mask, 48 bits
    uint16_t high[3][GRAD_LIST];
    uint32_t first[GRAD_LIST];                     // a tensor's first chunk
    uint16_t last[GRAD_LIST];                      // elements of its last chunk less one, and above them its type
    uint32_t n, chunks;                            // tensors; chunks of all
};
static_assert(GRAD_CHUNK <= 8192 && sizeof(GradList) <= 4000, "13 bits; 4 KB of arguments with the others");

inline uint64_t grad_launches(uint64_t count) { return count == 0 ? 1 : (count + GRAD_LIST - 1) / GRAD_LIST; }
inline uint64_t grad_norm_bytes(uint64_t count) { return LEARN_TICKETS + GRAD_HEAD + 8ull * GRAD_BLOCKS * grad_launches(count); }

// The tensors [from, from + GRAD_LIST) of a list without empty ones, in chunks of so many elements.
inline void grad_list(const std::vector<shifter_grad>& all, uint64_t from, uint32_t chunk, GradList* l) {
    l->n = (uint32_t)std::min<uint64_t>(GRAD_LIST, all.size() - from);
    l->chunks = 0;
    for (uint32_t i = 0; i < l->n; ++i) {
        const shifter_grad& g = all[from + i];
        const uint64_t at[3] = {reinterpret_cast<uint64_t>(g.d_g), reinterpret_cast<uint64_t>(g.d_out), reinterpret_cast<uint64_t>(g.d_mask)};
        for (int j = 0; j < 3; ++j) {
            l->low[j][i] = (uint32_t)at[j];
            l->high[j][i] = (uint16_t)(at[j] >> 32);
        }
        l->first[i] = l->chunks;
        l->last[i] = (uint16_t)((g.n - 1) % chunk | (uint32_t)g.dtype << 13);
        l->chunks += (uint32_t)((g.n + chunk - 1) / chunk);
    }
}

// Whether one block does it all, the elements in its registers.
inline bool grad_small(const std::vector<shifter_grad>& all) {
    uint64_t eights = 0;
    for (const shifter_grad& g : all) eights += g.n > 8ull * GRAD_SMALL ? GRAD_SMALL + 1u : (g.n + 7u) / 8u;
    return all.size() <= GRAD_LIST && eights <= GRAD_SMALL;
}

// What is wrong with a list, or nullptr.
inline const char* grad_bad(const shifter_grad* h, uint64_t count, bool write) {
    uint64_t chunks = 0;
    for (uint64_t i = 0; i < count; ++i) {
        const shifter_grad& g = h[i];
        if (g.dtype != SHIFTER_F32 && g.dtype != SHIFTER_BF16 && g.dtype != SHIFTER_F16) return "unknown element type";
        if (g.n == 0) continue;
        const uint64_t size = g.dtype == SHIFTER_F32 ? 4 : 2;
        if (!g.d_g || (write && !g.d_out)) return "NULL pointer argument";
        if (q8_off(g.d_g, size) || (write && q8_off(g.d_out, size))) return "a pointer is not aligned to its elements";
        const uint64_t ends[3] = {reinterpret_cast<uint64_t>(g.d_g), reinterpret_cast<uint64_t>(g.d_out), reinterpret_cast<uint64_t>(g.d_mask)};
        if ((ends[0] | ends[1] | ends[2]) >> 48) return "an address of more than 48 bits";
        if (g.n >> 40) return "2^40 elements or more";
        chunks += (g.n + GRAD_CHUNK - 1) / GRAD_CHUNK;
    }
    return chunks >> 31 ? "2^42 elements or more" : nullptr;
}

// Whether a tensor that is written lies over another one, over its own elements in another place or over a mask: blocks would read what others have
// written already.
inline bool grad_overlap(const std::vector<shifter_grad>& all) {
    struct Span {
        uint64_t from, to;
        bool written;
    };
    std::vector<Span> spans;
    spans.reserve(3 * all.size());
    for (uint32_t i = 0; i < all.size(); ++i) {
        const uint64_t bytes = all[i].n * (all[i].dtype == SHIFTER_F32 ? 4 : 2), g = reinterpret_cast<uint64_t>(all[i].d_g),
                       out = reinterpret_cast<uint64_t>(all[i].d_out), mask = reinterpret_cast<uint64_t>(all[i].d_mask);
        spans.push_back({out, out + bytes, true});
        if (out != g) spans.push_back({g, g + bytes, false});
        if (mask) spans.push_back({mask, mask + all[i].n, false});
    }
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
    uint64_t any = 0, written = 0;                 // ends of what came before
    for (const Span& s : spans) {
        if (s.from < written || (s.written && s.from < any)) return true;
        any = std::max(any, s.to);
        if (s.written) written = std::max(written, s.to);
    }
    return false;
}

}  // namespace shifter
