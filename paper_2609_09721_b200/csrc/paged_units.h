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
#define EFQ_HD_CALLED __host__ __device__ __noinline__      // once a CTA: kept out of the way of the loops' code
#else
#define EFQ_HD inline
#define EFQ_HD_CALLED inline
#endif

namespace efq {

// sum over i < n of floor((a i + b) / m); a, b >= 0.  The lattice points below a line, by Euclid's algorithm on (m, a).
EFQ_HD_CALLED int64_t floor_sum(uint64_t n, uint64_t m, uint64_t a, uint64_t b)
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

// One sequence of the step: lq new tokens in query tiles of `step` tokens, len keys in tiles of 2^kShift.
template <int kShift>
struct SeqWork {
    static constexpr int kKeys = 1 << kShift;
    int32_t lq, len, step, tiles;
    int32_t causal;
    int32_t none;               // its length names keys that its row of the page table has no room for: rows of NaN

    EFQ_HD void set(int lq_, int len_, int step_, int causal_, int none_ = 0)
    {
        lq = lq_;
        len = len_;
        step = step_;
        tiles = static_cast<int>((static_cast<uint32_t>(lq_) + static_cast<uint32_t>(step_) - 1u) / static_cast<uint32_t>(step_));
        causal = causal_;
        none = none_;
    }
    // keys that the last token of tile i sees
    EFQ_HD int limit(int i) const
    {
        if (!causal || i + 1 >= tiles) return len;
        const int n = len - lq + (i + 1) * step;
        return n < 0 ? 0 : n;
    }
    // a tile that sees nothing is a unit too: its rows have to be written
    EFQ_HD int units(int i) const
    {
        const int n = static_cast<int>((static_cast<uint32_t>(limit(i)) + (kKeys - 1u)) >> kShift);
        return n > 0 ? n : 1;
    }
    // units of the first n tiles
    EFQ_HD int64_t units_before(int n) const
    {
        if (n <= 0) return 0;
        if (!causal || tiles == 1) return static_cast<int64_t>(n) * units(0);
        const int64_t base = static_cast<int64_t>(len) - lq;
        const int64_t blind = base >= 0 ? 0 : -base / step;                     // tiles that see nothing
        const int full = n < tiles ? n : tiles - 1;                             // the last one ends at len and not at a multiple of step
        int64_t sum = blind < full ? blind : full;
        if (full > blind)
            sum += floor_sum(static_cast<uint64_t>(full - blind), static_cast<uint64_t>(kKeys), static_cast<uint64_t>(step),
                             static_cast<uint64_t>(base + (blind + 1) * step + kKeys - 1));
        return n == tiles ? sum + units(tiles - 1) : sum;
    }
    EFQ_HD int64_t units_per_head() const { return units_before(tiles); }
    // the tile that holds unit `off` of a head
    EFQ_HD int tile_of(int64_t off) const
    {
        int lo = 0, hi = tiles;
        while (hi - lo > 1) {
            const int mid = lo + (hi - lo) / 2;
            if (units_before(mid) <= off) lo = mid;
            else hi = mid;
        }
        return lo;
    }
};

// The run of units of one CTA, and a walk along it.  Every role of a kernel walks by itself.
template <int kShift>
struct PagedRun {
    int64_t left;                       // units
    int32_t seq, begin, head, tile, unit;       // where it begins; the sequence's first token in the step
    int32_t begins;                     // CTA that holds unit 0 of that query tile
    SeqWork<kShift> w;                  // of that sequence
};

template <int kShift>
struct PagedSegment {
    SeqWork<kShift> w;
    int32_t seq, head, token0, tokens;              // tokens of the step: token0 .. token0 + tokens - 1
    int32_t base;                                   // token i of the tile sees base + i + 1 keys (causal), all len otherwise
    int32_t j0, j1, n;                              // key tiles of the run, of the query tile
};

// Quotients whose operands mostly fit 32 bits
EFQ_HD uint64_t paged_divide(uint64_t a, uint64_t b)
{
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}
// CTA c of `ctas` takes each = total / ctas units, the first `more` CTAs one more (total >= ctas: every CTA has one).
struct PagedShares {
    int64_t each, more;
    EFQ_HD PagedShares(int64_t total, int64_t ctas) : each(static_cast<int64_t>(paged_divide(total, ctas))), more(total - each * ctas) {}
    EFQ_HD int64_t first(int64_t c) const { return each * c + (c < more ? c : more); }
    EFQ_HD int64_t units(int64_t c) const { return each + (c < more ? 1 : 0); }
    EFQ_HD int64_t cta_of(int64_t unit) const
    {
        const int64_t wide = (each + 1) * more;
        return static_cast<int64_t>(unit < wide ? paged_divide(unit, each + 1) : more + paged_divide(unit - wide, each));
    }
};
// The run of CTA c, which begins at unit `off` of sequence s.
template <int kShift>
EFQ_HD void paged_begin_run(const SeqWork<kShift>& w, int s, int begin, int64_t per_head, int64_t off, const PagedShares& shares, int64_t c, PagedRun<kShift>* run)
{
    run->left = shares.units(c);
    run->seq = s;
    run->begin = begin;
    run->w = w;
    run->head = static_cast<int32_t>(paged_divide(off, per_head));
    off -= run->head * per_head;
    run->tile = w.tile_of(off);
    run->unit = static_cast<int32_t>(off - w.units_before(run->tile));
    run->begins = static_cast<int32_t>(shares.cta_of(shares.first(c) - run->unit));
}

// `Read`: sequence s of the step and its first token there.
template <int kShift, typename Read>
struct PagedWalk {
    Read read;
    int n_seqs, heads;
    int64_t left;
    int seq, head, tile, unit, begin;
    SeqWork<kShift> w;

    EFQ_HD PagedWalk(Read r, int n, int h, const PagedRun<kShift>& run)
        : read(r), n_seqs(n), heads(h), left(run.left), seq(run.seq), head(run.head), tile(run.tile), unit(run.unit), begin(run.begin), w(run.w)
    {
    }
    // the next segment of the run; false at its end
    EFQ_HD bool next(PagedSegment<kShift>& g)
    {
        if (left <= 0) return false;
        if (tile == w.tiles) {
            tile = 0;
            if (++head == heads) {
                head = 0;
                do {
                    if (++seq >= n_seqs) {          // tables that changed under way
                        left = 0;
                        return false;
                    }
                    read(seq, w, begin);
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
