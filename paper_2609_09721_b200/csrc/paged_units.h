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

// sum over i < n of floor((b + a i) / 2^shift), a > 0, b >= 0.  The terms grow by a fixed amount from one period of
// 2^shift / gcd(a, 2^shift) terms to the next, so two partial periods are summed term by term and the rest is arithmetic.
EFQ_HD int64_t paged_floor_sum(int64_t n, int shift, uint32_t a, uint32_t b)
{
    int low = 0;
    while (low < shift && ((a >> low) & 1u) == 0u) ++low;
    const int period_log = shift - low;
    const uint32_t period = 1u << period_log;
    const int64_t full = n >> period_log, grows = static_cast<int64_t>(a) >> low;         // period * a / 2^shift
    const uint32_t rest = static_cast<uint32_t>(n - (full << period_log)), upto = full > 0 ? period : rest;
    int64_t of_period = 0, of_rest = 0;
    uint64_t x = b;
    for (uint32_t i = 0; i < upto; ++i, x += a) {
        if (i == rest) of_rest = of_period;
        of_period += static_cast<int64_t>(x >> shift);
    }
    if (rest == upto) of_rest = of_period;
    return full * of_period + grows * static_cast<int64_t>(period) * (full * (full - 1) / 2) + static_cast<int64_t>(rest) * full * grows + of_rest;
}

// One sequence of the step: lq new tokens in query tiles of `step` tokens, len keys in tiles of 2^kShift.  A query tile costs its key tiles and
// kItem more (its queries' load, its output): so many units of it stand for no key tile.
template <int kShift, int kItem>
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
    // one that sees nothing has a key tile all the same: its rows have to be written
    EFQ_HD int key_tiles(int i) const
    {
        const int n = static_cast<int>((static_cast<uint32_t>(limit(i)) + (kKeys - 1u)) >> kShift);
        return n > 0 ? n : 1;
    }
    EFQ_HD int units(int i) const { return key_tiles(i) + kItem; }
    // units of the first n tiles
    EFQ_HD int64_t units_before(int n) const
    {
        if (n <= 0) return 0;
        if (!causal || tiles == 1) return static_cast<int64_t>(n) * units(0);
        const int base = len - lq;
        const int blind = base >= 0 ? 0 : -base / step;                         // tiles that see nothing
        const int full = n < tiles ? n : tiles - 1;                             // the last one ends at len and not at a multiple of step
        int64_t sum = (blind < full ? blind : full) + static_cast<int64_t>(n) * kItem;
        if (full > blind)
            sum += paged_floor_sum(full - blind, kShift, static_cast<uint32_t>(step),
                                   static_cast<uint32_t>(static_cast<int64_t>(base) + static_cast<int64_t>(blind + 1) * step + kKeys - 1));
        return n == tiles ? sum + key_tiles(tiles - 1) : sum;
    }
    EFQ_HD int64_t units_per_head() const { return units_before(tiles); }
};

// The run of units of one CTA, and a walk along it.  Every role of a kernel walks by itself.
template <int kShift, int kItem>
struct PagedRun {
    int64_t left, off;                  // units; the first one's place in its head
    int32_t seq, begin, head, tile, unit;       // where it begins; the sequence's first token in the step
    int32_t begins;                     // CTA that holds unit 0 of that query tile
    SeqWork<kShift, kItem> w;           // of that sequence
};

template <int kShift, int kItem>
struct PagedSegment {
    SeqWork<kShift, kItem> w;
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
// The run of CTA c, which begins at unit `off` of sequence s; paged_begin_tile() has to follow with the query tile that holds unit run->unit of
// the head.
template <int kShift, int kItem>
EFQ_HD void paged_begin_run(const SeqWork<kShift, kItem>& w, int s, int begin, int64_t per_head, int64_t off, const PagedShares& shares, int64_t c,
                            PagedRun<kShift, kItem>* run)
{
    run->left = shares.units(c);
    run->seq = s;
    run->begin = begin;
    run->w = w;
    run->head = static_cast<int32_t>(paged_divide(off, per_head));
    run->off = off - run->head * per_head;
    run->tile = 0;
    run->unit = 0;
    run->begins = static_cast<int32_t>(c);
}
// Whether query tile `tile` holds the run's first unit; if so, the run begins there.
template <int kShift, int kItem>
EFQ_HD bool paged_begin_tile(int tile, const PagedShares& shares, int64_t c, PagedRun<kShift, kItem>* run)
{
    const int64_t unit = run->off - run->w.units_before(tile);
    if (unit < 0 || unit >= run->w.units(tile)) return false;
    run->tile = tile;
    run->unit = static_cast<int32_t>(unit);
    run->begins = static_cast<int32_t>(shares.cta_of(shares.first(c) - unit));
    return true;
}

// `Read`: sequence s of the step and its first token there.
template <int kShift, int kItem, typename Read>
struct PagedWalk {
    Read read;
    int n_seqs, heads;
    int64_t left;
    int seq, head, tile, unit, begin;
    SeqWork<kShift, kItem> w;

    EFQ_HD PagedWalk(Read r, int n, int h, const PagedRun<kShift, kItem>& run)
        : read(r), n_seqs(n), heads(h), left(run.left), seq(run.seq), head(run.head), tile(run.tile), unit(run.unit), begin(run.begin), w(run.w)
    {
    }
    // the next segment of the run; false at its end
    EFQ_HD bool next(PagedSegment<kShift, kItem>& g)
    {
        while (left > 0) {
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
            const int first = tile * w.step, n = w.key_tiles(tile), from = unit, all = n + kItem - from;
            const int taken = all < left ? all : static_cast<int>(left);
            left -= taken;
            unit = 0;
            ++tile;
            if (from >= n) continue;                    // only what stands for no key tile
            g.w = w;
            g.seq = seq;
            g.head = head;
            g.token0 = begin + first;
            g.tokens = w.lq - first < w.step ? w.lq - first : w.step;
            g.base = w.len - w.lq + first;
            g.n = n;
            g.j0 = from;
            g.j1 = from + taken < n ? from + taken : n;
            return true;
        }
        return false;
    }
};

}  // namespace efq
