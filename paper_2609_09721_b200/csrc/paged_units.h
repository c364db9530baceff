// How the kernels of the paged attention share a step's work: the arithmetic, for the host as well.
//
// A unit is one tile of keys of one query tile of one KV head of one sequence.  All units of the step stand in a row (sequence, KV
// head, query tile, key tile) and every CTA takes an equal run of them, so that a single long context, many short ones and
// the triangle of a causal chunk all fill the chip, and lengths that only the device knows decide nothing on the host.  A query tile whose
// units lie in one CTA is finished there; otherwise each of its CTAs leaves the maximum, the sum and the unnormalised output of its
// part, and a second kernel joins the parts in their order (no atomics: the same step gives the same bits).  A CTA leaves two
// parts at most, one of the query tile that its run begins in and one of that it ends in, whatever the step looks like.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define EFQ_HD __host__ __device__ __forceinline__
#else
#define EFQ_HD inline
#endif

namespace efq {

// sum over i < n of floor((a i + b) / m); a, b >= 0.  The lattice points below a line, by Euclid's algorithm on (m, a).
EFQ_HD int64_t floor_sum(uint64_t n, uint64_t m, uint64_t a, uint64_t b)
{
    uint64_t sum = 0;
    while (n > 0) {
        sum += n * (n - 1) / 2 * (a / m) + n * (b / m);
        a %= m;
        b %= m;
        const uint64_t top = a * n + b;
        if (top < m) break;
        n = top / m;
        b = top % m;
        const uint64_t t = m;
        m = a;
        a = t;
    }
    return static_cast<int64_t>(sum);
}

// One sequence of the step: lq new tokens in query tiles of `step` tokens, len keys in tiles of `keys`.
struct SeqWork {
    int32_t lq, len, step, keys, causal;
    int32_t none = 0;           // its length names keys that its row of the page table has no room for: rows of NaN

    EFQ_HD int tiles() const { return (lq + step - 1) / step; }
    // keys that the last token of tile i sees
    EFQ_HD int limit(int i) const
    {
        if (!causal) return len;
        const int64_t upto = static_cast<int64_t>(i + 1) * step;
        const int64_t n = static_cast<int64_t>(len) - lq + (upto < lq ? upto : lq);
        return n < 0 ? 0 : static_cast<int>(n);
    }
    // a tile that sees nothing is a unit too: its rows have to be written
    EFQ_HD int units(int i) const
    {
        const int64_t n = (static_cast<int64_t>(limit(i)) + keys - 1) / keys;
        return n > 0 ? static_cast<int>(n) : 1;
    }
    // units of the first n tiles
    EFQ_HD int64_t units_before(int n) const
    {
        const int nt = tiles();
        if (n <= 0) return 0;
        if (!causal || nt == 1) return static_cast<int64_t>(n) * units(0);
        const int64_t base = static_cast<int64_t>(len) - lq;
        const int64_t blind = base >= 0 ? 0 : -base / step;                     // tiles that see nothing
        const int full = n < nt ? n : nt - 1;                                   // the last one ends at len and not at a multiple of step
        int64_t sum = blind < full ? blind : full;
        if (full > blind)
            sum += floor_sum(static_cast<uint64_t>(full - blind), static_cast<uint64_t>(keys), static_cast<uint64_t>(step),
                             static_cast<uint64_t>(base + (blind + 1) * step + keys - 1));
        return n == nt ? sum + units(nt - 1) : sum;
    }
    EFQ_HD int64_t units_per_head() const { return lq > 0 ? units_before(tiles()) : 0; }
    // the tile that holds unit `off` of a head
    EFQ_HD int tile_of(int64_t off) const
    {
        int lo = 0, hi = tiles();
        while (hi - lo > 1) {
            const int mid = lo + (hi - lo) / 2;
            if (units_before(mid) <= off) lo = mid;
            else hi = mid;
        }
        return lo;
    }
};

// The run of units of one CTA, and a walk along it.  Every role of a kernel walks by itself.
struct PagedRun {
    int64_t left;                       // units
    int32_t seq, head, tile, unit;      // where it begins
    int32_t begins;                     // CTA that holds unit 0 of that query tile
};

struct PagedSegment {
    SeqWork w;
    int32_t seq, head, token0, tokens;              // tokens of the step: token0 .. token0 + tokens - 1
    int32_t base;                                   // token i of the tile sees base + i + 1 keys (causal), all len otherwise
    int32_t j0, j1, n;                              // key tiles of the run, of the query tile
};

// Of `total` units, the first that CTA c of `ctas` takes (total >= ctas: every CTA has one), and the CTA that takes unit u.
EFQ_HD int64_t paged_first_unit(int64_t total, int64_t ctas, int64_t c) { return total * c / ctas; }
EFQ_HD int paged_cta_of(int64_t total, int64_t ctas, int64_t u)
{
    int64_t c = u * ctas / total;
    while (paged_first_unit(total, ctas, c + 1) <= u) ++c;
    while (paged_first_unit(total, ctas, c) > u) --c;
    return static_cast<int>(c);
}
// The run of CTA c, which begins at unit `off` of sequence s.
EFQ_HD void paged_begin_run(const SeqWork& w, int s, int64_t off, int64_t total, int64_t ctas, int64_t c, PagedRun* run)
{
    const int64_t per_head = w.units_per_head(), u0 = paged_first_unit(total, ctas, c);
    run->left = paged_first_unit(total, ctas, c + 1) - u0;
    run->seq = s;
    run->head = static_cast<int32_t>(off / per_head);
    off -= run->head * per_head;
    run->tile = w.tile_of(off);
    run->unit = static_cast<int32_t>(off - w.units_before(run->tile));
    run->begins = paged_cta_of(total, ctas, u0 - run->unit);
}

// `Read`: the sequence s and, by reference, its first token in the step.
template <typename Read>
struct PagedWalk {
    Read read;
    int n_seqs, heads;
    int64_t left;
    int seq, head, tile, unit, begin;
    SeqWork w;

    EFQ_HD PagedWalk(Read r, int n, int h, const PagedRun& run)
        : read(r), n_seqs(n), heads(h), left(run.left), seq(run.seq), head(run.head), tile(run.tile), unit(run.unit), begin(0), w()
    {
        if (left > 0) w = read(seq, begin);
    }
    // the next segment of the run; false at its end
    EFQ_HD bool next(PagedSegment& g)
    {
        if (left <= 0) return false;
        if (tile == w.tiles()) {
            tile = 0;
            if (++head == heads) {
                head = 0;
                do {
                    if (++seq >= n_seqs) {          // tables that changed under way
                        left = 0;
                        return false;
                    }
                    w = read(seq, begin);
                } while (w.lq == 0);
            }
        }
        const int first = tile * w.step, n = w.units(tile);
        g.w = w;
        g.seq = seq;
        g.head = head;
        g.token0 = begin + first;
        g.tokens = w.lq - first < w.step ? w.lq - first : w.step;
        g.base = w.len - w.lq + first;
        g.n = n;
        g.j0 = unit;
        g.j1 = n - unit < left ? n : static_cast<int>(unit + left);
        left -= g.j1 - g.j0;
        unit = 0;
        ++tile;
        return true;
    }
};

}  // namespace efq
