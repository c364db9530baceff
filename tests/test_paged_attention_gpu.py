"""efq_paged_attention_fwd against softmax attention in 64 bits: query rows of a KV group from one to many, lengths around the tiles and
pages, every type and layout, steps of many sequences, and what must not matter (stale pages, unused entries, other rows)."""
import math
import random

import pytest
import torch

from paged_reference import D, Paged
from paper_2609_09721_b200 import binding

pytestmark = pytest.mark.gpu


def _run(p, causal=True, lse=True, scale=0.0, **more):
    o = torch.full((p.total, p.Hq, D), 7.0, dtype=p.dtype, device="cuda")
    l = torch.full((p.total, p.Hq), 7.0, device="cuda") if lse else None
    got = binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, *p.tables, more.pop("max_q", p.max_q), causal, scale, o, l, **more)
    assert got is o
    return o, l


def _check(p, o, lse, causal=True, scale=None):
    want, want_lse, tol, lse_tol = p.attention(causal, scale)
    n = int(p.cu[-1])
    assert torch.isfinite(o[:n]).all()
    off = (o[:n].double() - want[:n]).abs() - tol[:n]
    assert float(off.max() if off.numel() else 0.0) <= 0.0, float(off.max())
    assert (o[n:] == 7.0).all()                                   # rows behind the last sequence
    if lse is not None:
        seen = torch.isfinite(want_lse[:n])
        assert (lse[:n][~seen] == -math.inf).all()
        off = ((lse[:n].double() - want_lse[:n]).abs() - lse_tol[:n])[seen]
        assert float(off.max() if off.numel() else 0.0) <= 0.0, float(off.max())
        assert (lse[n:] == 7.0).all()


# (lens, Hq, Hkv, page): rows of a KV group are Hq / Hkv times the new tokens
FEW = [
    ([(1, 1)], 1, 1, 16), ([(1, 2)], 8, 8, 16), ([(1, 63)], 4, 1, 16), ([(1, 64)], 8, 2, 32), ([(1, 65)], 8, 2, 64), ([(1, 128)], 4, 4, 128),
    ([(1, 8191)], 32, 8, 16), ([(1, 20001)], 1, 1, 64), ([(1, 300)], 16, 1, 16), ([(1, 1000)], 5, 1, 256), ([(1, 999)], 3, 1, 16),
    ([(1, 777)], 17, 1, 32), ([(1, 500)], 32, 1, 16), ([(1, 5)], 24, 2, 1024),
    ([(4, 4)], 4, 1, 16), ([(2, 130)], 8, 1, 16), ([(5, 2000)], 32, 8, 32), ([(8, 1025)], 8, 2, 16), ([(16, 40)], 1, 1, 16),
    ([(3, 64)], 20, 4, 64), ([(32, 4000)], 2, 2, 128), ([(7, 7)], 4, 1, 16), ([(9, 700)], 3, 1, 16),
    ([(1, n) for n in (1, 70, 300, 4096, 16, 129, 2000)], 32, 8, 16), ([(1, 1 + 37 * i) for i in range(130)], 8, 2, 16),
    ([(1 + i % 4, 4 + 53 * i) for i in range(40)], 8, 4, 32), ([(1, 17)] * 700, 2, 2, 16), ([(0, 50), (1, 60), (0, 0), (2, 2), (0, 9)], 4, 2, 16),
]
CHUNK = [
    ([(33, 33)], 1, 1, 16), ([(128, 128)], 1, 1, 16), ([(129, 129)], 2, 2, 16), ([(256, 257)], 1, 1, 128), ([(300, 300)], 4, 1, 64),
    ([(300, 9000)], 32, 8, 64), ([(64, 5000)], 4, 4, 32), ([(17, 1200)], 2, 1, 16), ([(100, 3001)], 28, 4, 16), ([(77, 800)], 10, 2, 256),
    ([(50, 51)], 3, 1, 16),
    ([(2000, 2100)], 2, 2, 128), ([(1, 700), (300, 400), (5, 2000), (0, 10), (128, 128), (1, 1), (40, 999)], 8, 2, 16),
    ([(37, 37 + 100 * i) for i in range(20)], 4, 2, 64), ([(1024, 1024)], 4, 4, 512),
    ([(1, 640)], 64, 1, 16), ([(2, 333)], 128, 1, 16), ([(1, 1)], 128, 1, 16), ([(3, 100)], 50, 1, 32), ([(5, 64)], 33, 1, 16),
]


@pytest.mark.parametrize("lens,Hq,Hkv,page", FEW + CHUNK)
@pytest.mark.parametrize("causal", [True, False])
def test_against_64_bits(lens, Hq, Hkv, page, causal):
    p = Paged(lens, Hq, Hkv, page, seed=len(lens) + Hq)
    _check(p, *_run(p, causal), causal)


@pytest.mark.parametrize("lens,Hq,Hkv,page", [FEW[6], FEW[16], FEW[24], CHUNK[5], CHUNK[12]])
def test_fp16(lens, Hq, Hkv, page):
    p = Paged(lens, Hq, Hkv, page, torch.float16, seed=3)
    _check(p, *_run(p))
    o, _ = _run(p, lse=False)
    _check(p, o, None)


@pytest.mark.parametrize("max_q", [1, 6, 40, 4000])
def test_the_announced_length_only_chooses_the_kernel(max_q):
    """Sequences with more new tokens than announced are computed all the same."""
    p = Paged([(70, 200), (1, 900), (33, 33)], 8, 2, 16, seed=5)
    o, lse = _run(p, max_q=max_q)
    _check(p, o, lse)


@pytest.mark.parametrize("lens,Hq,Hkv", [([(1, 900), (2, 77)], 8, 2), ([(200, 900), (3, 500)], 8, 2)])
def test_strides(lens, Hq, Hkv):
    """q as a part of a wider projection, o into a wider buffer, a token-major cache, a table that is a part of a wider one, rows behind the
    last sequence: they are left as they were."""
    p = Paged(lens, Hq, Hkv, 32, seed=6, token_major=True, tail=5)
    want = _run(p)
    _check(p, *want)
    wide = torch.zeros(p.total, Hq + 3, D + 64, dtype=p.dtype, device="cuda")
    wide[:, 1:Hq + 1, 64:] = p.d_q
    out = torch.full((p.total, 2 * Hq, D), 7.0, dtype=p.dtype, device="cuda")
    table = torch.full((len(lens), p.d_table.shape[1] + 9), 1 << 30, dtype=torch.int32, device="cuda")
    table[:, :-9] = p.d_table
    binding.efq_paged_attention_fwd(wide[:, 1:Hq + 1, 64:], p.d_k_cache, p.d_v_cache, table, p.d_cu, p.d_seq_lens, p.max_q, o=out[:, ::2])
    assert torch.equal(out[:, ::2], want[0]) and (out[:, 1::2] == 7.0).all()
    odd = torch.full((p.total, Hq, D + 8), 7.0, dtype=p.dtype, device="cuda")      # rows on 16 bytes and no more
    binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, *p.tables, p.max_q, o=odd[..., 8:])
    assert torch.equal(odd[..., 8:], want[0]) and (odd[..., :8] == 7.0).all()


# rows of a KV group from 17 to 32 in the longest sequence, fewer in others: warps without rows, sequences without tokens or keys
MIDDLE = [
    ([(5, 300), (1, 200), (2, 64), (0, 5), (5, 5), (3, 1), (4, 1000), (1, 1)], 8, 2, 16), ([(8, 70), (1, 5000), (8, 4097), (5, 63)], 8, 2, 64),
    ([(1, 100 + 61 * i) for i in range(90)], 32, 1, 32), ([(1 + i % 5, 6 + 40 * i) for i in range(70)], 20, 4, 16), ([(2, 3000), (1, 2999)], 32, 2, 128),
    ([(1, 1), (1, 64), (1, 65)], 17, 1, 16), ([(32, 32), (31, 700), (1, 700), (16, 40), (17, 40)], 3, 3, 16),
]


@pytest.mark.parametrize("lens,Hq,Hkv,page", MIDDLE)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_17_to_32_rows(lens, Hq, Hkv, page, dtype):
    p = Paged(lens, Hq, Hkv, page, seed=19, dtype=dtype, tail=3)
    _check(p, *_run(p))
    o, _ = _run(p, causal=False)
    _check(p, o, None, causal=False)


@pytest.mark.parametrize("lens,Hq,Hkv", [([(150, 20000)], 2, 1), ([(40, 9000), (300, 12345), (1, 7000)], 4, 2), ([(64, 30000)], 8, 4)])
@pytest.mark.parametrize("causal", [True, False])
def test_runs_that_begin_inside_long_contexts(lens, Hq, Hkv, causal):
    """The tiles of such a run are read in another order than that of the keys."""
    p = Paged(lens, Hq, Hkv, 128, seed=20)
    _check(p, *_run(p, causal), causal=causal)


@pytest.mark.parametrize("lens,Hq,Hkv", [([(1, 9000), (2, 77), (0, 3), (1, 1)], 8, 2), ([(200, 900), (3, 500), (130, 7000)], 8, 2), ([(33, 4000)], 3, 1)])
def test_output_in_the_place_of_the_queries(lens, Hq, Hkv):
    p = Paged(lens, Hq, Hkv, 32, seed=17)
    want, _ = _run(p)
    for _ in range(3):
        q = p.d_q.clone()
        binding.efq_paged_attention_fwd(q, p.d_k_cache, p.d_v_cache, *p.tables, p.max_q, o=q)
        assert torch.equal(q, want)


@pytest.mark.parametrize("n", [1, 100])
def test_queries_and_pages_of_no_stride(n):
    """One token's queries for all of them, one head's for all heads, and caches with a broadcast axis: dimensions with a stride of zero."""
    p = Paged([(n, 700), (n, 90)], 8, 2, 16, seed=18)
    for q in (p.d_q[:1].expand(p.total, -1, -1), p.d_q[:, :1].expand(-1, 8, -1), p.d_q[:1, :1].expand(p.total, 8, -1)):
        want = binding.efq_paged_attention_fwd(q.contiguous(), p.d_k_cache, p.d_v_cache, *p.tables, p.max_q)
        got = binding.efq_paged_attention_fwd(q, p.d_k_cache, p.d_v_cache, *p.tables, p.max_q, o=torch.empty_like(want))
        assert torch.equal(got, want)
    k = p.d_k_cache[:, :1].expand(-1, 2, -1, -1)
    want = binding.efq_paged_attention_fwd(p.d_q, k.contiguous(), p.d_v_cache, *p.tables, p.max_q)
    assert torch.equal(binding.efq_paged_attention_fwd(p.d_q, k, p.d_v_cache, *p.tables, p.max_q), want)


@pytest.mark.parametrize("lens,Hq", [([(8, 3), (1, 0), (2, 500)], 2), ([(300, 100), (64, 0), (5, 5)], 2), ([(40, 1)], 32)])
def test_tokens_that_see_nothing(lens, Hq):
    """More new tokens than tokens: the first ones see no key and get zeros, with lse = -inf."""
    p = Paged([(a, b) for a, b in lens], Hq, 2, 16, seed=7)
    o, lse = _run(p)
    _check(p, o, lse)
    a, b = lens[0]
    assert (o[:a - b] == 0).all() and (lse[:a - b] == -math.inf).all()


@pytest.mark.parametrize("lens,Hq,Hkv", [([(1, 700), (2, 90)], 4, 2), ([(90, 700), (2, 90)], 8, 2)])
def test_pages_that_are_none(lens, Hq, Hkv):
    """An entry that names no page, or a sequence longer than its row of the table: rows of NaN, for that sequence alone."""
    p = Paged(lens, Hq, Hkv, 16, seed=8)
    want, _ = _run(p)
    n = lens[0][0]
    for bad in (-1, -2**31, p.d_k_cache.shape[0], 2**31 - 1):
        table = p.d_table.clone()
        table[0, 0] = bad
        o = binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, table, p.d_cu, p.d_seq_lens, p.max_q)
        assert torch.isnan(o[:n]).all() and torch.equal(o[n:], want[n:]), bad
    for length in (p.d_table.shape[1] * 16 + 1, 2**31 - 1):
        lens_now = p.d_seq_lens.clone()
        lens_now[0] = length
        o = binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, p.d_table, p.d_cu, lens_now, p.max_q)
        assert torch.isnan(o[:n]).all() and torch.equal(o[n:], want[n:])
    lens_now = p.d_seq_lens.clone()
    lens_now[0] = -5                                             # no keys
    o = binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, p.d_table, p.d_cu, lens_now, p.max_q)
    assert (o[:n] == 0).all() and torch.equal(o[n:], want[n:])


@pytest.mark.parametrize("lens,Hq,Hkv", [([(1, 3000)], 8, 2), ([(200, 3000)], 8, 2), ([(1, 10 + i) for i in range(50)], 8, 2)])
def test_the_same_call_gives_the_same_bits(lens, Hq, Hkv):
    p = Paged(lens, Hq, Hkv, 16, seed=9)
    first = _run(p)
    workspace = torch.full((binding.efq_paged_attention_workspace_bytes(Hq, Hkv, p.max_q),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        again = _run(p, workspace=workspace)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("n", [1, 100])
def test_large_scores_and_scales(n):
    """Scores far from zero: the running maximum keeps the exponentials in range, in whatever order the keys come."""
    p = Paged([(n, 1500)], 4, 2, 64, seed=10, hot=0)
    k = p.k[0].double()
    k[:, :, 0] = torch.linspace(-200, 200, 1500)[:, None]        # grows along the keys: every tile has a new maximum
    p.k[0] = k.to(p.dtype)
    at, slot = torch.arange(1500) // 64, torch.arange(1500) % 64
    p.d_k_cache[p.table[0].long()[at].cuda(), :, slot.cuda()] = p.k[0].cuda()
    p.d_q[..., 0] = 3.0
    for scale in (0.0, 0.5, 1e-3):
        _check(p, *_run(p, scale=scale), scale=scale or None)


def test_recorded_into_a_graph_it_follows_the_tables():
    """Lengths, tables and the cache live on the device: a replay computes what they say then."""
    p = Paged([(1, 400), (1, 900), (1, 31)], 8, 2, 16, seed=11)
    o = torch.zeros(p.total, 8, D, dtype=p.dtype, device="cuda")
    workspace = torch.empty(binding.efq_paged_attention_workspace_bytes(8, 2, 1), dtype=torch.uint8, device="cuda")
    lens, table = p.d_seq_lens.clone(), p.d_table.clone()
    call = lambda: binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, table, p.d_cu, lens, 1, o=o, workspace=workspace)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for cut in (0, 17, 30):
        lens.copy_(p.d_seq_lens - cut)
        o.zero_()
        graph.replay()
        q = Paged([(1, m - cut) for _, m in p.lens], 8, 2, 16, seed=11)
        for i, (_, m) in enumerate(q.lens):
            q.k[i], q.v[i] = p.k[i][:m], p.v[i][:m]
        q.d_q = p.d_q
        _check(q, o, None)


def test_on_a_side_stream():
    p = Paged([(1, 3000), (60, 500)], 8, 2, 16, seed=12)
    want, _ = _run(p)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o = torch.zeros_like(want)
    o.record_stream(s)
    workspace = torch.empty(binding.efq_paged_attention_workspace_bytes(8, 2, 60), dtype=torch.uint8, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, *p.tables, 60, o=o, workspace=workspace, stream=s)
    s.synchronize()
    assert torch.equal(o, want)


@pytest.mark.parametrize("seed", range(48))
def test_drawn_steps(seed):
    """Steps of every kind drawn at random: decode, drafts, chunks and mixtures, heads, pages, types, layouts, masks."""
    rng = random.Random(seed)
    Hkv = rng.choice([1, 2, 3, 8])
    G = rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16, 24, 48])
    kind = rng.choice(["decode", "draft", "chunk", "mixed"])
    n = rng.choice([1, 2, 5, 17, 60])
    top = {"decode": 1, "draft": 7, "chunk": 700, "mixed": 90}[kind]
    lens = []
    for _ in range(n if kind != "chunk" else min(n, 2)):
        a = rng.choice([0, 1, top, rng.randint(1, top)])
        lens.append((a, rng.choice([a, max(a - 3, 0), a + rng.randint(0, 40), a + rng.randint(0, 3000)])))
    p = Paged(lens, Hkv * G, Hkv, rng.choice([16, 32, 64, 128, 256]), rng.choice([torch.bfloat16, torch.bfloat16, torch.float16]), seed, hot=rng.choice([0, 8]),
              token_major=rng.random() < 0.4, tail=rng.choice([0, 3]), slack=rng.choice([1, 5]))
    causal = rng.random() < 0.7
    if p.total:
        _check(p, *_run(p, causal), causal)


@pytest.mark.parametrize("n", [1, 40])
def test_a_cache_of_more_than_32_bits(n):
    """Pages whose elements lie past 2^31 from the cache's start, written by the append and read by the attention."""
    Hq, Hkv, page, pages = 8, 4, 64, 70000
    cache = [torch.empty(pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert cache[0].numel() > 2**31
    ids = torch.tensor([[pages - 1, 65600, 3, pages - 2, 66000, -1]], dtype=torch.int32, device="cuda")
    p = Paged([(n, 300)], Hq, Hkv, page, seed=13)
    for c in cache:
        c[ids[0, :5].long()] = math.nan
    cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 300], [300]))
    binding.efq_paged_append(p.k[0].cuda(), p.v[0].cuda(), *cache, ids, cu, lens)
    o = binding.efq_paged_attention_fwd(p.d_q, *cache, ids, p.d_cu, p.d_seq_lens, n)
    _check(p, o, None)
    assert torch.equal(cache[1][65600, :, 5], p.v[0][69].cuda())


def test_two_streams_at_once():
    """Calls that overlap, each with outputs and a workspace of its own (made by the binding on the call's stream): the same bits as alone."""
    ps = [Paged([(1, 5000), (1, 300)], 8, 2, 16, seed=14), Paged([(130, 2000), (7, 900)], 8, 2, 32, seed=15)]
    want = [_run(p, lse=False)[0] for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for p, s, g in zip(ps, streams, got):
            g.append(binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, *p.tables, p.max_q, stream=s))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(w, x) for x in g)


def test_nothing_to_do():
    p = Paged([(3, 30)], 4, 2, 16, seed=16)
    o = binding.efq_paged_attention_fwd(p.d_q[:0], p.d_k_cache, p.d_v_cache, p.d_table, torch.zeros(2, dtype=torch.int32, device="cuda"), p.d_seq_lens, 0)
    assert o.shape == (0, 4, D)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    o = torch.full_like(p.d_q, 7.0)
    binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, p.d_table[:0], torch.zeros(1, dtype=torch.int32, device="cuda"), none, 3, o=o)
    assert (o == 7.0).all()
    for cu in ([0, 0], [5, 2], [-3, 1], [2, 9]):                 # no new tokens, and prefix sums that are none of the step's: nothing is written
        binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, p.d_table, torch.tensor(cu, dtype=torch.int32, device="cuda"), p.d_seq_lens, 3, o=o)
        assert (o == 7.0).all(), cu


def _page_zero_is_nan(p):
    """Moves what page 0 holds to a free page: what a kernel might read in the place of a page that is none is NaN."""
    free = next(i for i in range(1, p.d_k_cache.shape[0]) if not (p.d_table == i).any())
    for c in (p.d_k_cache, p.d_v_cache):
        c[free] = c[0]
        c[0] = math.nan
    p.d_table[p.d_table == 0] = free


@pytest.mark.parametrize("n,Hq,Hkv", [(2, 4, 2), (4, 4, 1), (5, 8, 2), (8, 8, 2), (7, 3, 1), (16, 2, 2), (32, 1, 1)])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_a_last_page_that_is_none_is_for_the_tokens_that_see_it(n, Hq, Hkv, page):
    """Tokens of a draft that lie before the page keep their results, to the bit, whichever kernel the announced length chooses."""
    for m in (page * 3 + 1, page * 3 + (n + 1) // 2, page * 5 + n - 1):
        p = Paged([(n, m), (1, 50)], Hq, Hkv, page, seed=21)
        _page_zero_is_nan(p)
        table = p.d_table.clone()
        at = (m - 1) // page
        table[0, at] = -1
        sees = torch.zeros(p.total, dtype=torch.bool, device="cuda")
        sees[max(0, at * page - (m - n)):n] = True              # token i sees m - n + i + 1 keys
        for max_q in (n, 4000):
            for causal in (True, False):
                want, want_lse = _run(p, causal, max_q=max_q)
                assert torch.isfinite(want).all()
                lse = torch.zeros(p.total, Hq, device="cuda")
                o = binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, table, p.d_cu, p.d_seq_lens, max_q, causal, lse=lse)
                hit = sees if causal else torch.arange(p.total, device="cuda") < n
                assert torch.isnan(o[hit]).all() and torch.isnan(lse[hit]).all()
                assert torch.equal(o[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])


@pytest.mark.parametrize("n,Hq,Hkv", [(1, 8, 2), (5, 8, 2), (32, 1, 1), (40, 8, 2)])
def test_a_page_that_is_none_inside_a_long_context(n, Hq, Hkv):
    """One of many parts of a context lies on it: all tokens behind it are NaN, other sequences are as they were."""
    p = Paged([(3, 700), (n, 20000), (1, 900)], Hq, Hkv, 16, seed=25)
    want, want_lse = _run(p)
    for at in (0, 3, 617, 1240):
        table = p.d_table.clone()
        table[1, at] = p.d_k_cache.shape[0] + 5
        o = torch.zeros_like(want)
        binding.efq_paged_attention_fwd(p.d_q, p.d_k_cache, p.d_v_cache, table, p.d_cu, p.d_seq_lens, p.max_q, o=o)
        assert torch.isnan(o[3:3 + n]).all() and torch.equal(o[:3], want[:3]) and torch.equal(o[3 + n:], want[3 + n:]), at


@pytest.mark.parametrize("dtype,size", [(torch.float16, 4.0), (torch.float16, 4096.0), (torch.float16, 30000.0), (torch.bfloat16, 2.0 ** 16), (torch.bfloat16, 2.0 ** 40)])
@pytest.mark.parametrize("max_q", [1, 8, 1000])
def test_scores_whose_steps_are_large(dtype, size, max_q):
    """Scores up to 2^87, between which FP32 has steps of 2^64: each row has one key far above the others, whose value it gets, and lse is its score."""
    n, m = 40, 700
    p = Paged([(n, m)], 4, 2, 16, dtype, seed=26, hot=0)
    g = torch.Generator().manual_seed(2)
    sign = torch.randint(0, 2, (n, 4, D), generator=g).mul(2).sub(1).float()
    best = torch.randint(0, m - n, (n, 2), generator=g)
    k = torch.zeros(m, 2, D)
    # token t of heads 2 h and 2 h + 1 agrees in all channels with its own key and in some with those of others
    sign[:, 1::2] = sign[:, ::2]
    for t in range(n):
        for h in range(2):
            k[best[t, h], h] = size * 1.1 * sign[t, 2 * h]
    k = k.to(dtype)
    q = (size * 1.3 * sign).to(dtype)
    at, slot = torch.arange(m) // 16, torch.arange(m) % 16
    p.d_k_cache[p.table[0].long()[at].cuda(), :, slot.cuda()] = k.cuda()
    p.d_q.copy_(q)
    o, lse = _run(p, max_q=max_q)
    scores = torch.einsum("thd,mhd->thm", q.double(), k.double().repeat_interleave(2, 1)) / math.sqrt(D)
    top, key = scores.max(-1)
    rest = scores.scatter(-1, key[..., None], -math.inf).amax(-1)
    clear = top - rest > 40 + math.log(m)                        # what the others weigh together is less than 2^-57
    assert clear.float().mean() > 0.7
    want = torch.stack([p.v[0][key[:, h], h // 2] for h in range(4)], 1)
    # the weight of the key is 1 up to FP32 sums: its value comes out as it is
    assert torch.equal(o.cpu()[clear], want[clear])
    # a sum of 128 products: 8 steps of up to 2^-22 of it, and two roundings of 2^-24
    assert float(((lse.cpu().double() - top).abs() / top)[clear].max()) <= 2.0 ** -18


@pytest.mark.parametrize("n,Hq,Hkv,m", [(1, 1, 1, 65537), (1, 32, 8, 4097), (5, 8, 2, 131072), (32, 1, 1, 20000), (40, 2, 1, 65576), (300, 2, 1, 131372), (130, 8, 2, 2000),
                                         (1, 160, 160, 4097), (3, 160, 40, 4099), (24, 150, 150, 4119), (300, 40, 40, 4396), (40, 192, 48, 4136)])
@pytest.mark.parametrize("below", [12.25, 18.25, 25.25])
def test_a_key_above_a_long_flat_tail(n, Hq, Hkv, m, below):
    """The first key's score is 2^below times the weight of each of the others, which in fp16 would be a number without all its bits, or 0: the
    values of the many others have to be in the output all the same, also where the first key's is 0."""
    for dtype in (torch.float16, torch.bfloat16):
        p = Paged([(n, m)], Hq, Hkv, 64, dtype, seed=22, hot=0)
        g = torch.Generator().manual_seed(1)
        p.k[0] = torch.zeros(m, Hkv, D, dtype=dtype)
        p.k[0][0, :, 0] = below
        v = torch.rand(m, Hkv, D, generator=g) + 0.5
        v[0, :, ::2] = 0.0
        p.v[0] = v.to(dtype)
        at, slot = p.table[0].long()[torch.arange(m) // 64].cuda(), (torch.arange(m) % 64).cuda()
        p.d_k_cache[at, :, slot], p.d_v_cache[at, :, slot] = p.k[0].cuda(), p.v[0].cuda()
        p.d_q.zero_()
        p.d_q[..., 0] = 1.0
        o, lse = _run(p, scale=math.log(2.0))
        want, want_lse, tol, lse_tol = p.attention(True, math.log(2.0))
        # beside what other values of the tests may be off by: a probability below 2^-20 of the row's maximum is rounded to a step of 2^-30 of it
        tail = 2.0 ** -31 * p.v[0].double().sum(0).max() if dtype == torch.float16 else 0.0
        assert float(((o.double() - want).abs() - tol - tail).max()) <= 0.0
        assert float(((lse.double() - want_lse).abs() - lse_tol).max()) <= 0.0


@pytest.mark.parametrize("grows", [2, 4, 6, 8, 14, 16])
@pytest.mark.parametrize("max_q", [1, 1000])
def test_a_maximum_that_grows_by_little_far_from_zero(grows, max_q):
    """Scores near 2^25 / log2(e), where FP32 has steps of 2 in units of log2, and one in a later tile that is 2^grows as heavy: what is kept of the maximum
    must not be rounded to where the probability is more than fp16 holds."""
    n, m = 40, 700
    p = Paged([(n, m)], 2, 2, 16, torch.float16, seed=27, hot=0)
    k = torch.zeros(m, 2, D)
    k[:, :, 0], k[:, :, 1] = 16384.0, -64.0 - 32.0               # the others weigh 2^-32 and less of the first
    k[0, :, 1], k[300, :, 1] = -64.0, -64.0 + grows
    p.k[0] = k.half()
    at, slot = p.table[0].long()[torch.arange(m) // 16].cuda(), (torch.arange(m) % 16).cuda()
    p.d_k_cache[at, :, slot] = p.k[0].cuda()
    p.d_q.zero_()
    p.d_q[..., 0], p.d_q[..., 1] = 2048.0, 1.0
    o, _ = _run(p, scale=math.log(2.0), max_q=max_q)
    v, w = p.v[0].double(), 2.0 ** grows
    near = ((v[0] + w * v[300]) / (1 + w))[None].cuda()          # the steps of 2 are exact here: probabilities and the output are rounded once
    bound = 2.0 ** -11 * ((v[0].abs() + w * v[300].abs()) / (1 + w)).cuda() * 2.1 + 700 * 2.0 ** -32 * 4
    assert float(((o.double() - near).abs() - bound).max()) <= 0.0


def _ms(call):
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    call()
    b.record()
    b.synchronize()
    return a.elapsed_time(b)


@pytest.mark.parametrize("n,Hq,Hkv", [(33, 32, 32), (5, 256, 32), (100, 32, 32)])
def test_rows_that_no_query_has_do_not_matter_to_the_time(n, Hq, Hkv):
    """Rows behind the last sequence lie in its query tile too.  Nothing that they hold may be a reason to rescale the output, as a maximum that is
    NaN is at every tile of keys: both kinds of rows take the same time, but for the clock (5 %)."""
    p = Paged([(n, 20000)], Hq, Hkv, 128, seed=23, tail=256)
    rows = {"zero": p.d_q.clone(), "nan": p.d_q.clone()}
    rows["zero"][n:] = 0.0
    rows["nan"][n:] = math.nan
    workspace = torch.empty(binding.efq_paged_attention_workspace_bytes(Hq, Hkv, 1000), dtype=torch.uint8, device="cuda")
    o = torch.empty_like(p.d_q)
    times = {x: 1e9 for x in rows}
    for _ in range(40):
        for x, q in rows.items():
            times[x] = min(times[x], _ms(lambda: binding.efq_paged_attention_fwd(q, p.d_k_cache, p.d_v_cache, *p.tables, 1000, o=o, workspace=workspace)))
    assert times["nan"] <= 1.05 * times["zero"], times
