// Host harness for the paged cache's arithmetic.  Built by test_paged_plan.py with a plain host compiler.
#include "../paper_2601_21896_b200/csrc/paged_plan.cuh"

using namespace pafu;

// 1 if n / d is right for every n of the list
extern "C" int divides(uint32_t d, const uint32_t* n, int count) {
    const FastDiv f = fast_div(d);
    for (int i = 0; i < count; ++i)
        if (div_by(n[i], f) != n[i] / d) return 0;
    return 1;
}

// The items' steps as every CTA of a grid takes them, by the kernel's rule; out[k] = {first position, end} of CTA k after the cuts moved;
// pieces[i] = {first, n} for item i.  Returns the number of CTAs used.
extern "C" int plan(int n_items, const int32_t* steps, int grid, int64_t* out, int32_t* pieces, int32_t* snap) {
    uint64_t all = 0;
    for (int i = 0; i < n_items; ++i) all += steps[i] + kPaItemCost;
    const PagedCuts c = paged_cuts(all, grid);
    *snap = c.snap;
    uint64_t at = 0;
    for (int i = 0; i < n_items; ++i) {
        const PagedPieces p = paged_pieces(c, at, steps[i] + kPaItemCost);
        pieces[2 * i] = p.first;
        pieces[2 * i + 1] = p.n;
        at += steps[i] + kPaItemCost;
    }
    int i = 0;
    at = 0;
    for (uint32_t k = 0; k <= c.n; ++k) {
        const uint64_t b = paged_cut(c, k);
        uint64_t to = b;
        if (b < all) {
            while (b >= at + steps[i] + kPaItemCost) at += steps[i++] + kPaItemCost;
            const int cost = steps[i] + kPaItemCost, moves = paged_cut_moves(c, (int)(b - at), cost);
            to = moves < 0 ? at : moves > 0 ? at + cost : b;
        }
        if (k < c.n) out[2 * k] = (int64_t)to;
        if (k > 0) out[2 * k - 1] = (int64_t)to;
    }
    return (int)c.n;
}
