// Arithmetic of the paged cache that host and kernels share: division by a page's length, and how the attention's work is
// cut.  No CUDA types, so that a host compiler can check it.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define PAFU_HD __host__ __device__ __forceinline__
#else
#define PAFU_HD inline
#endif

namespace pafu {

// n / d for 0 <= n < 2^31 as a product: m = floor(2^(31+s) / d) + 1 with s = ceil(log2 d) has an excess below
// 2^(31+s) / 2^31, so the quotient is exact (round-up method of division by an invariant integer).
struct FastDiv {
    uint32_t d, m, s;
};
PAFU_HD FastDiv fast_div(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return FastDiv{d, (uint32_t)(((1ull << (31 + s)) / d) + 1), s};
}
PAFU_HD uint32_t div_by(uint32_t n, const FastDiv& f) { return (uint32_t)(((uint64_t)n * f.m) >> (31 + f.s)); }

PAFU_HD uint64_t div_u64(uint64_t a, uint64_t b) {             // the 32-bit division takes a quarter of the time
    return (a | b) >> 32 ? a / b : (uint64_t)((uint32_t)a / (uint32_t)b);
}

constexpr int kPaItemCost = 1;        // what an item costs beside its steps, in steps
constexpr int kPaMinShare = 2;        // steps and item costs that a CTA takes at least (where there are as many)

// The items of a call laid end to end, each of cost = steps + kPaItemCost, in `n` shares: cut k (0 to n) lies at all * k / n, and
// moves to the end of its item where it would leave fewer than `snap` steps of the item on that side.
struct PagedCuts {
    uint64_t all;
    uint32_t n;
    int32_t snap;
};
PAFU_HD PagedCuts paged_cuts(uint64_t all, uint32_t grid) {
    PagedCuts c;
    c.all = all;
    const uint64_t n = div_u64(all, kPaMinShare);
    c.n = n < 1 ? 1u : n < grid ? (uint32_t)n : grid;
    const uint64_t share = div_u64(all, c.n);
    c.snap = share < 32 ? 2 : 1;
    return c;
}
PAFU_HD uint64_t paged_cut(const PagedCuts& c, uint32_t k) { return div_u64(c.all * k, c.n); }

// Where a cut at offset o of an item goes: -1 to its beginning, 1 to its end, 0 it stays
PAFU_HD int paged_cut_moves(const PagedCuts& c, int32_t o, int32_t cost) { return o < c.snap ? -1 : cost - o <= c.snap ? 1 : 0; }

// The pieces of the item that begins at `at`: n of them, the first is that of CTA `first` (n below 2: the item is whole, and `first` means nothing)
struct PagedPieces {
    int32_t first, n;
};
PAFU_HD PagedPieces paged_pieces(const PagedCuts& c, uint64_t at, int32_t cost) {
    // cuts that stay: all * k / n >= at + snap and <= at + cost - snap - 1
    const uint64_t k0 = div_u64((at + c.snap) * c.n + c.all - 1, c.all), k1 = div_u64((at + cost - c.snap) * c.n + c.all - 1, c.all);
    return PagedPieces{(int32_t)k0 - 1, (int32_t)(k1 - k0) + 1};
}

}  // namespace pafu
