"""How the kernels of the paged attention share a step's work (csrc/paged_units.h), on the host: the sums in closed form, and that
the runs of all CTAs hold every unit once, in order, with the CTA that begins a query tile named rightly."""
import ctypes
import random
import subprocess

import pytest

from paper_2609_09721_b200 import build

HARNESS = r"""
#include "paged_units.h"
template <int kShift, int kItem>
struct Reader {
    const int32_t *cu, *lens;
    int step, causal;
    void operator()(int s, efq::SeqWork<kShift, kItem>& w, int& begin) const { begin = cu[s]; w.set(cu[s + 1] - cu[s], lens[s], step, causal); }
};
template <int kShift, int kItem>
int64_t before_of(int lq, int len, int step, int causal, int n)
{
    efq::SeqWork<kShift, kItem> w;
    w.set(lq, len, step, causal);
    return w.units_before(n);
}
extern "C" int64_t before(int lq, int len, int step, int keys, int item, int causal, int n)
{
    return keys == 64 ? item ? before_of<6, 1>(lq, len, step, causal, n) : before_of<6, 0>(lq, len, step, causal, n)
                      : item ? before_of<7, 2>(lq, len, step, causal, n) : before_of<7, 0>(lq, len, step, causal, n);
}
template <int kShift, int kItem>
int64_t all_segments(const int32_t* cu, const int32_t* lens, int n_seqs, int heads, int step, int causal, int grid, int32_t* out, int64_t most)
{
    const Reader<kShift, kItem> read{cu, lens, step, causal};
    efq::SeqWork<kShift, kItem> w;
    uint32_t total = 0;
    int64_t n = 0;
    int b;
    for (int s = 0; s < n_seqs; ++s) {
        read(s, w, b);
        total += w.units_per_head() * heads;
    }
    const uint32_t ctas = (uint32_t)grid < total ? grid : total;
    if (total == 0) return 0;
    const efq::PagedShares shares(total, ctas);
    for (uint32_t c = 0; c < ctas; ++c) {
        efq::PagedRun<kShift, kItem> run{};
        uint32_t off = shares.first(c);
        if (shares.cta_of(off) != c) return -2;
        for (int s = 0; s < n_seqs; ++s) {
            read(s, w, b);
            const uint32_t per_head = w.units_per_head();
            if (off < per_head * heads) { efq::paged_begin_run(w, s, b, per_head, off, shares, c, &run); break; }
            off -= per_head * heads;
        }
        int found = 0;
        for (int i = 0; i < run.w.tiles; ++i) found += efq::paged_begin_tile(i, shares, c, &run) ? 1 : 0;
        if (found != 1) return -3;
        efq::PagedWalk<kShift, kItem, Reader<kShift, kItem>> walk(read, n_seqs, heads, run);
        efq::PagedSegment<kShift, kItem> g;
        bool first = true;
        while (walk.next(g)) {
            if (n == most) return -1;
            const int32_t v[10] = {(int32_t)c, first && g.j0 > 0 ? run.begins : (int32_t)c, g.seq, g.head, g.token0, g.tokens, g.base, g.j0, g.j1, g.n};
            for (int i = 0; i < 10; ++i) out[10 * n + i] = v[i];
            ++n;
            first = false;
        }
    }
    return n;
}
// segments of all CTAs: (cta, begins, seq, head, token0, tokens, base, j0, j1, n) each; the number of them, below zero if there is a mistake
extern "C" int64_t segments(const int32_t* cu, const int32_t* lens, int n_seqs, int heads, int step, int keys, int causal, int grid, int32_t* out, int64_t most)
{
    return keys == 64 ? all_segments<6, 1>(cu, lens, n_seqs, heads, step, causal, grid, out, most)
                      : all_segments<7, 2>(cu, lens, n_seqs, heads, step, causal, grid, out, most);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("units")
    (d / "units.cpp").write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, str(d / "units.cpp"), "-o", str(d / "units.so")], check=True)
    so = ctypes.CDLL(str(d / "units.so"))
    so.before.restype = so.segments.restype = ctypes.c_int64
    so.segments.argtypes = [ctypes.POINTER(ctypes.c_int32)] * 2 + [ctypes.c_int] * 6 + [ctypes.POINTER(ctypes.c_int32), ctypes.c_int64]
    return so


def _units(lq, len_, step, keys, causal):
    """Units of each query tile, one by one."""
    out = []
    for first in range(0, lq, step):
        seen = max(0, len_ - lq + min(first + step, lq)) if causal else len_
        out.append(max(1, -(-seen // keys)))
    return out


def test_units_in_closed_form(lib):
    rng = random.Random(1)
    for _ in range(4000):
        lq, len_ = rng.choice([1, rng.randint(1, 40), rng.randint(1, 700)]), rng.choice([0, 1, rng.randint(0, 900), rng.randint(0, 9000)])
        step, keys, causal = rng.choice([1, 2, 3, 4, 5, 8, 18, 36, 42, 50, 64, 256]), rng.choice([64, 128]), rng.randint(0, 1)
        item = rng.choice([0, 1 if keys == 64 else 2])
        want = [n + item for n in _units(lq, len_, step, keys, causal)]
        n = rng.randint(0, len(want))
        assert lib.before(lq, len_, step, keys, item, causal, n) == sum(want[:n]), (lq, len_, step, keys, causal, n)


def test_units_of_the_longest_sequences(lib):
    """Whole prompts of millions of tokens up to the 2^31 units that a step may have, and the last tile before 2^31 keys."""
    for lq, step in ((2_000_003, 64), (2_000_003, 50), (500_000, 1), (5_000_000, 256)):
        want = _units(lq, lq, step, 128, 1)
        assert sum(want) < 2**31 and lib.before(lq, lq, step, 128, 0, 1, len(want)) == sum(want)
    assert lib.before(1, 2**31 - 1, 16, 64, 0, 1, 1) == 2**25
    assert lib.before(200, 2**31 - 1, 64, 128, 0, 1, 4) == sum(_units(200, 2**31 - 1, 64, 128, 1))


@pytest.mark.parametrize("seed", range(60))
def test_runs_hold_every_unit_once(lib, seed):
    rng = random.Random(seed)
    n, heads, grid = rng.choice([1, 2, 5, 40, 300]), rng.choice([1, 2, 8]), rng.choice([1, 3, 148])
    step, keys, causal = rng.choice([1, 4, 5, 16, 64, 84]), rng.choice([64, 128]), rng.randint(0, 1)
    lens_q = [rng.choice([0, 1, 1, rng.randint(1, 9), rng.randint(1, 300)]) for _ in range(n)]
    lens_k = [rng.choice([0, 1, rng.randint(1, 200), rng.randint(1, 4000)]) for _ in range(n)]
    cu = [sum(lens_q[:i]) for i in range(n + 1)]
    item = 1 if keys == 64 else 2
    want = [(s, h, cu[s] + t * step, j, u) for s in range(n) for h in range(heads)
            for t, u in enumerate(_units(lens_q[s], lens_k[s], step, keys, causal)) for j in range(u)]
    most = len(want) + 1
    out = (ctypes.c_int32 * (10 * most))()
    got = lib.segments((ctypes.c_int32 * (n + 1))(*cu), (ctypes.c_int32 * n)(*lens_k), n, heads, step, keys, causal, grid, out, most)
    assert got >= 0, got
    rows = [tuple(out[10 * i:10 * i + 10]) for i in range(got)]
    assert [(s, h, t0, j, u) for _, _, s, h, t0, _, _, j0, j1, u in rows for j in range(j0, j1)] == want
    sizes, begun = {}, {}
    for c, begins, s, h, t0, tokens, base, j0, j1, u in rows:
        sizes[c] = sizes.get(c, 0) + j1 - j0 + (item if j1 == u else 0)
        if j0 == 0:
            begun[s, h, t0] = c
        assert begun[s, h, t0] == begins, (c, s, h, t0, j0)    # also the second and later CTAs of a query tile
        first = t0 - cu[s]
        assert tokens == min(step, lens_q[s] - first) and base == lens_k[s] - lens_q[s] + first
    total = len(want) + item * len({x[:3] for x in want})
    if want:            # shares are equal, of key tiles and what a query tile costs beside them (which may lie with the CTA after its last key tile)
        assert max(sizes.values()) <= -(-total // min(grid, total)) + item


# ------------------------------------------------------------ the same with the constants that the kernels have
SHIPPED = HARNESS + r"""
extern "C" int64_t shipped_before(int many, int lq, int len, int step, int causal, int n)
{
    return many ? before_of<efq::kChunkShift, efq::kChunkItem>(lq, len, step, causal, n) : before_of<efq::kFewShift, efq::kFewItem>(lq, len, step, causal, n);
}
extern "C" int64_t shipped_segments(int many, const int32_t* cu, const int32_t* lens, int n_seqs, int heads, int step, int causal, int grid, int32_t* out, int64_t most)
{
    return many ? all_segments<efq::kChunkShift, efq::kChunkItem>(cu, lens, n_seqs, heads, step, causal, grid, out, most)
                : all_segments<efq::kFewShift, efq::kFewItem>(cu, lens, n_seqs, heads, step, causal, grid, out, most);
}
extern "C" void shipped_constants(int many, int* keys, int* item)
{
    *keys = 1 << (many ? efq::kChunkShift : efq::kFewShift);
    *item = many ? efq::kChunkItem : efq::kFewItem;
}
"""


@pytest.fixture(scope="module")
def shipped(tmp_path_factory):
    d = tmp_path_factory.mktemp("shipped")
    (d / "units.cpp").write_text(SHIPPED)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, str(d / "units.cpp"), "-o", str(d / "shipped.so")], check=True)
    so = ctypes.CDLL(str(d / "shipped.so"))
    so.shipped_before.restype = so.shipped_segments.restype = ctypes.c_int64
    so.shipped_segments.argtypes = [ctypes.c_int] + [ctypes.POINTER(ctypes.c_int32)] * 2 + [ctypes.c_int] * 5 + [ctypes.POINTER(ctypes.c_int32), ctypes.c_int64]
    return so


def _constants(so, many):
    keys, item = ctypes.c_int(), ctypes.c_int()
    so.shipped_constants(many, ctypes.byref(keys), ctypes.byref(item))
    return keys.value, item.value


def _steps(many):
    """New tokens of a query tile for every number of query heads on a KV head."""
    return sorted({128 // g * 2 for g in range(1, 129)} if many else {rows // g for rows in (16, 32) for g in range(1, 33) if rows >= g})


@pytest.mark.parametrize("many", [0, 1])
def test_units_of_the_kernels_in_closed_form(shipped, many):
    keys, item = _constants(shipped, many)
    rng = random.Random(2)
    for step in _steps(many):
        for _ in range(60):
            lq, len_ = rng.choice([1, rng.randint(1, 40), rng.randint(1, 900)]), rng.choice([0, 1, rng.randint(0, 900), rng.randint(0, 9000)])
            causal = rng.randint(0, 1)
            want = [n + item for n in _units(lq, len_, step, keys, causal)]
            for n in {0, 1, len(want) // 2, len(want)} - ({1} if not want else set()):
                assert shipped.shipped_before(many, lq, len_, step, causal, n) == sum(want[:n]), (lq, len_, step, causal, n)


@pytest.mark.parametrize("many", [0, 1])
@pytest.mark.parametrize("seed", range(40))
def test_runs_of_the_kernels_hold_every_unit_once(shipped, many, seed):
    keys, item = _constants(shipped, many)
    rng = random.Random(1000 + seed)
    n, heads, grid, step, causal = rng.choice([1, 2, 5, 40, 300]), rng.choice([1, 2, 8]), rng.choice([1, 3, 148]), rng.choice(_steps(many)), rng.randint(0, 1)
    lens_q = [rng.choice([0, 1, 1, rng.randint(1, 9), rng.randint(1, 300)]) for _ in range(n)]
    lens_k = [rng.choice([0, 1, rng.randint(1, 200), rng.randint(1, 4000)]) for _ in range(n)]
    cu = [sum(lens_q[:i]) for i in range(n + 1)]
    want = [(s, h, cu[s] + t * step, j, u) for s in range(n) for h in range(heads)
            for t, u in enumerate(_units(lens_q[s], lens_k[s], step, keys, causal)) for j in range(u)]
    out = (ctypes.c_int32 * (10 * (len(want) + 1)))()
    got = shipped.shipped_segments(many, (ctypes.c_int32 * (n + 1))(*cu), (ctypes.c_int32 * n)(*lens_k), n, heads, step, causal, grid, out, len(want) + 1)
    assert got >= 0, got
    rows = [tuple(out[10 * i:10 * i + 10]) for i in range(got)]
    assert [(s, h, t0, j, u) for _, _, s, h, t0, _, _, j0, j1, u in rows for j in range(j0, j1)] == want
    sizes, begun, parts = {}, {}, {}
    for c, begins, s, h, t0, tokens, base, j0, j1, u in rows:
        sizes[c] = sizes.get(c, 0) + j1 - j0 + (item if j1 == u else 0)
        if j0 == 0:
            begun[s, h, t0] = c
        if (j0, j1) != (0, u):                                   # a part: two places a CTA, one for a tile that it begins
            parts.setdefault((c, j0 == 0), []).append((s, h, t0))
        assert begun[s, h, t0] == begins, (c, s, h, t0, j0)
        first = t0 - cu[s]
        assert tokens == min(step, lens_q[s] - first) and base == lens_k[s] - lens_q[s] + first
    assert all(len(x) == 1 for x in parts.values())
    total = len(want) + item * len({x[:3] for x in want})
    if want:
        assert max(sizes.values()) <= -(-total // min(grid, total)) + item
