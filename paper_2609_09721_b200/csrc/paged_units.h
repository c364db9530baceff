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

// Keys of a tile (log2), and what a query tile costs beside its key tiles, in key tiles.  Few rows, 1 and 3 instead of 2: up to 2 % more.  Many rows, with 0,
// 1, 2 and 3: a mixed batch of 16 sequences 290, 281, 276 and 279 us, 300 tokens on 9000 59.6, 58.1, 57.0 and 57.2, 64 on 2000 21.5, 21.4, 21.5 and 22.2.
constexpr int kFewShift = 6, kFewItem = 2;
constexpr int kChunkShift = 7, kChunkItem = 2;

// All numbers of units fit 31 bits: a step that might have more is refused (paged_too_many_units()).  The search for a CTA's run stands before its
// first load, and it is the instructions that cost there, fetched for the first time; 64 bits made three of one.

// sum over i < n of floor((b + a i) / 2^shift), a > 0, which fits 32 bits.  The terms grow by a fixed amount from one period of
// 2^shift / gcd(a, 2^shift) terms to the next, so two partial periods are summed term by term and the rest is arithmetic.
EFQ_HD uint32_t paged_floor_sum(uint32_t n, int shift, uint32_t a, uint32_t b)
{
    int low = 0;
    while (low < shift && ((a >> low) & 1u) == 0u) ++low;
    const int period_log = shift - low;
    const uint32_t period = 1u << period_log, full = n >> period_log, rest = n & (period - 1u), grows = a >> low;      // grows = period * a / 2^shift
    const uint32_t upto = full > 0 ? period : rest;
    uint32_t of_period = 0, of_rest = 0;
    for (uint32_t i = 0, x = b; i < upto; ++i, x += a) {
        if (i == rest) of_rest = of_period;
        of_period += x >> shift;
    }
    if (rest == upto) of_rest = of_period;
    const uint32_t pairs = full > 0 ? ((full & 1u) != 0u ? (full - 1u) / 2u * full : full / 2u * (full - 1u)) : 0u;
    return full * of_period + grows * period * pairs + rest * full * grows + of_rest;
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
    EFQ_HD int units_before(int n) const
    {
        if (n <= 0) return 0;
        if (!causal || tiles == 1) return n * units(0);
        const int base = len - lq;
        const int blind = base >= 0 ? 0 : -base / step;                         // tiles that see nothing
        const int full = n < tiles ? n : tiles - 1;                             // the last one ends at len and not at a multiple of step
        int sum = (blind < full ? blind : full) + n * kItem;
        if (full > blind)       // blind * step <= lq and base + step <= len + 256: below 2^32 with what is added
            sum += static_cast<int>(paged_floor_sum(static_cast<uint32_t>(full - blind), kShift, static_cast<uint32_t>(step),
                                                    static_cast<uint32_t>(base) + static_cast<uint32_t>(blind + 1) * static_cast<uint32_t>(step) + (kKeys - 1u)));
        return n == tiles ? sum + key_tiles(tiles - 1) : sum;
    }
    EFQ_HD int units_per_head() const { return units_before(tiles); }
};

// The run of units of one CTA, and a walk along it.  Every role of a kernel walks by itself.
template <int kShift, int kItem>
struct PagedRun {
    int32_t left, off;                  // units; the first one's place in its head
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

// CTA c of `ctas` takes each = total / ctas units, the first `more` CTAs one more (total >= ctas: every CTA has one).
struct PagedShares {
    uint32_t each, more;
    EFQ_HD PagedShares(uint32_t total, uint32_t ctas) : each(total / ctas), more(total - each * ctas) {}
    EFQ_HD uint32_t first(uint32_t c) const { return each * c + (c < more ? c : more); }
    EFQ_HD uint32_t units(uint32_t c) const { return each + (c < more ? 1u : 0u); }
    EFQ_HD uint32_t cta_of(uint32_t unit) const
    {
        const uint32_t wide = (each + 1u) * more;
        return unit < wide ? unit / (each + 1u) : more + (unit - wide) / each;
    }
};
// Whether a step may have more units than 31 bits hold: `tokens` new ones (below 2^31) in n_seqs sequences of at most `keys` keys (below 2^31).
EFQ_HD bool paged_too_many_units(int64_t tokens, int n_seqs, int64_t keys, int heads, int step, int shift, int item)
{
    const int64_t tiles = tokens / step + n_seqs, of_tile = (keys >> shift) + 1 + item;         // below 2^32 and 2^31: no product of three
    return tiles > ((int64_t{1} << 31) - 1) / of_tile / heads;
}
// The run of CTA c, which begins at unit `off` of sequence s; paged_begin_tile() has to follow with the query tile that holds unit run->unit of
// the head.
template <int kShift, int kItem>
EFQ_HD void paged_begin_run(const SeqWork<kShift, kItem>& w, int s, int begin, uint32_t per_head, uint32_t off, const PagedShares& shares, uint32_t c,
                            PagedRun<kShift, kItem>* run)
{
    run->left = static_cast<int32_t>(shares.units(c));
    run->seq = s;
    run->begin = begin;
    run->w = w;
    const uint32_t head = off / per_head;
    run->head = static_cast<int32_t>(head);
    run->off = static_cast<int32_t>(off - head * per_head);
    run->tile = 0;
    run->unit = 0;
    run->begins = static_cast<int32_t>(c);
}
// Whether query tile `tile` holds the run's first unit; if so, the run begins there.
template <int kShift, int kItem>
EFQ_HD bool paged_begin_tile(int tile, const PagedShares& shares, uint32_t c, PagedRun<kShift, kItem>* run)
{
    const int unit = run->off - run->w.units_before(tile);
    if (unit < 0 || unit >= run->w.units(tile)) return false;
    run->tile = tile;
    run->unit = unit;
    run->begins = static_cast<int32_t>(shares.cta_of(shares.first(c) - static_cast<uint32_t>(unit)));
    return true;
}

// `Read`: sequence s of the step and its first token there.
template <int kShift, int kItem, typename Read>
struct PagedWalk {
    Read read;
    int n_seqs, heads, left;
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
            const int taken = all < left ? all : left;
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
