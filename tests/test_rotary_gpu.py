"""efq_rotary and efq_paged_append against their formulas in 64 bits: axes, pair layouts, partly turned channels, far positions, types,
strides, and what has to stay as it was."""
import math

import pytest
import torch

from paged_reference import D, Paged, rotate, rotate_slack
from paper_2609_09721_b200 import binding

pytestmark = pytest.mark.gpu

CASES = [                                    # sections, interleaved, one ladder an axis, first position
    ((64,), False, False, 0), ((64,), True, False, 7), ((22, 21, 21), True, True, 0), ((16, 24, 24), False, False, 900000),
    ((20, 12), False, True, -40), ((8, 8, 8), True, False, 1 << 30), ((8,), False, False, 3), ((0, 64), False, False, 5),
    ((10, 20, 30, 4), False, True, 2**31 - 400), ((5, 3), True, False, 11),
]


def _rotary(sections, interleaved, per_axis, theta=1e6):
    return binding.Rotary.of(sections, theta, interleaved, per_axis)


def _positions(axes, tokens, first):
    t = torch.arange(tokens, dtype=torch.int32, device="cuda")
    return torch.stack([(t // (a + 1) + first).int() for a in range(axes)])


def _near(got, want, slack, what=""):
    u = torch.finfo(got.dtype).eps / 2
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 0.0
    off = (got.double() - want).abs() - (u * want.abs() * (1 + 2.0 ** -10) + slack + tiny)
    assert float(off.max()) <= 0.0, (what, float(off.max()))


@pytest.mark.parametrize("sections,interleaved,per_axis,first", CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("inverse", [False, True])
def test_against_64_bits(sections, interleaved, per_axis, first, dtype, inverse):
    g = torch.Generator(device="cuda").manual_seed(1)
    for B, S, Hq, Hkv in ((1, 1, 1, 1), (2, 37, 5, 3), (1, 301, 8, 2)):
        q, k = (torch.randn(B, H, S, D, generator=g, device="cuda").to(dtype) for H in (Hq, Hkv))
        r, pos = _rotary(sections, interleaved, per_axis), _positions(len(sections), S, first)
        got = binding.efq_rotary(q, k, pos, r, inverse)
        for x, y in zip((q, k), got):
            assert y.is_contiguous()
            _near(y, rotate(x, pos, r.inv_freq, sections, interleaved, inverse), rotate_slack(x, dtype, sections, interleaved))
            R = sum(sections)
            assert torch.equal(y[..., 2 * R:], x[..., 2 * R:])       # what lies behind the turned channels


@pytest.mark.parametrize("B,S,Hq,Hkv", [(1, 1, 40, 8), (3, 130, 28, 4), (1, 5000, 3, 1), (65, 1, 2, 2), (1, 4097, 24, 24)])
def test_layouts_in_place_and_one_tensor(B, S, Hq, Hkv):
    """Token-major views of a projection in, head-major out; in place; q or k alone: the same bits."""
    g = torch.Generator(device="cuda").manual_seed(2)
    sections = (22, 21, 21)
    r = _rotary(sections, True, True)
    pos = _positions(3, S, 4)
    qkv = torch.randn(B, S, Hq + 2 * Hkv, D, generator=g, device="cuda").bfloat16()
    kept = qkv.clone()
    q, k = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hkv].transpose(1, 2)
    yq, yk = binding.efq_rotary(q, k, pos, r)
    assert torch.equal(qkv, kept)
    dense = binding.efq_rotary(q.contiguous(), k.contiguous(), pos, r)
    assert torch.equal(yq, dense[0]) and torch.equal(yk, dense[1])
    alone, none = binding.efq_rotary(q, None, pos, r)
    assert none is None and torch.equal(alone, yq)
    none, alone = binding.efq_rotary(None, k, pos, r)
    assert none is None and torch.equal(alone, yk)
    batched = torch.stack([pos + b for b in range(B)], dim=1)
    per_entry, _ = binding.efq_rotary(q, None, batched, r)
    for b in range(B):
        assert torch.equal(per_entry[b:b + 1], binding.efq_rotary(q[b:b + 1], None, pos + b, r)[0])
    binding.efq_rotary(q, k, pos, r, q_out=q, k_out=k)
    assert torch.equal(qkv[:, :, :Hq].transpose(1, 2), yq) and torch.equal(qkv[:, :, Hq:Hq + Hkv].transpose(1, 2), yk)
    assert torch.equal(qkv[:, :, Hq + Hkv:], kept[:, :, Hq + Hkv:])


def test_the_inverse_is_the_gradient():
    """d <w, rotate(x)> / dx is w turned back: against differences of the formula, and against the formula's own derivative."""
    g = torch.Generator(device="cuda").manual_seed(3)
    sections = (20, 12)
    r, pos = _rotary(sections, False, False), _positions(2, 9, 100)
    x = torch.randn(1, 2, 9, D, generator=g, device="cuda", dtype=torch.float64).requires_grad_()
    w = torch.randn(1, 2, 9, D, generator=g, device="cuda").bfloat16()
    y = rotate(x.detach(), pos, r.inv_freq, sections, False)
    step = 2.0 ** -10
    got, _ = binding.efq_rotary(w, None, pos, r, inverse=True)
    for at in [(0, 0, 0, 0), (0, 1, 8, 31), (0, 1, 5, 32), (0, 0, 3, 63), (0, 0, 3, 64), (0, 1, 2, 127)]:
        e = torch.zeros_like(x.detach())
        e[at] = step
        by_difference = ((rotate(x.detach() + e, pos, r.inv_freq, sections, False) - y) * w.double()).sum() / step
        # the formula is linear: the difference is exact but for the rounding of y (2^-53 of a sum of 2304 values, over the step)
        assert abs(float(got[at]) - float(by_difference)) <= abs(float(by_difference)) * 2.0 ** -8 + 2.0 ** -20, at
    rotated = []
    R = 32
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    angle = torch.stack([pos[axis[p]].double() * r.inv_freq[p] for p in range(R)], dim=-1)
    a, b = x[..., :R], x[..., R:2 * R]
    rotated = torch.cat((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos(), x[..., 2 * R:]), dim=-1)
    grad, = torch.autograd.grad((rotated * w.double()).sum(), x)
    _near(got, grad, rotate_slack(w, torch.bfloat16, sections, False))


@pytest.mark.parametrize("lens,Hq,Hkv,page", [
    ([(1, 1)], 1, 1, 16), ([(1, 64)], 8, 2, 64), ([(1, 1 + 31 * i) for i in range(70)], 32, 8, 16), ([(300, 300)], 4, 4, 16),
    ([(129, 1000)], 5, 1, 128), ([(0, 9), (3, 40), (0, 0), (17, 17), (0, 5), (1, 4096)], 8, 2, 32), ([(1, 20)] * 2000, 2, 1, 16),
    ([(2500, 5000)], 28, 4, 256),
])
@pytest.mark.parametrize("own_positions", [False, True])
def test_append(lens, Hq, Hkv, page, own_positions):
    """New tokens of every sequence land in their places, keys rotated; nothing else in the cache changes, nor do rows behind the last one."""
    tail = 3
    sections = (16, 24, 24) if own_positions else (64,)
    p = Paged(lens, Hq, Hkv, page, seed=4, tail=tail, token_major=len(lens) > 2)
    r = _rotary(sections, own_positions, False)
    n = int(p.cu[-1])
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn(p.total, Hkv, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    index = torch.cat([torch.arange(m - a, m) for a, m in lens] + [torch.zeros(tail, dtype=torch.long)]).cuda()
    pos = torch.stack([index // 100, index // 10 % 10, index % 10]).int() if own_positions else index[None].int()
    want_k, want_v = p.d_k_cache.clone(), p.d_v_cache.clone()
    place = [(int(p.table[s, i // page]), i % page) for s, (a, m) in enumerate(lens) for i in range(m - a, m)]
    pages, slots = (torch.tensor([x[j] for x in place], device="cuda") for j in (0, 1))
    turned = lambda x: rotate(x.transpose(0, 1), pos, r.inv_freq, sections, own_positions).transpose(0, 1)  # noqa: E731
    q_out = torch.full((p.total, Hq, D), 7.0, dtype=p.dtype, device="cuda")
    got = binding.efq_paged_append(k, v, p.d_k_cache, p.d_v_cache, *p.tables, r, pos if own_positions else None, p.d_q, q_out)
    assert got is q_out and (q_out[n:] == 7.0).all()
    _near(q_out[:n], turned(p.d_q)[:n], rotate_slack(p.d_q, p.dtype, sections, own_positions)[:n])
    _near(p.d_k_cache[pages, :, slots], turned(k)[:n], rotate_slack(k, p.dtype, sections, own_positions)[:n])
    want_k[pages, :, slots] = p.d_k_cache[pages, :, slots]
    want_v[pages, :, slots] = v[:n]
    same = lambda a, b: torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))  # noqa: E731
    assert same(p.d_k_cache, want_k) and same(p.d_v_cache, want_v)


def test_append_without_rotation_and_without_queries():
    p = Paged([(5, 50), (1, 300)], 4, 2, 16, seed=6)
    k, v = (torch.randn(6, 2, D, device="cuda").bfloat16() for _ in range(2))
    assert binding.efq_paged_append(k, v, p.d_k_cache, p.d_v_cache, *p.tables) is None
    for t, (s, i) in enumerate([(0, 45), (0, 46), (0, 47), (0, 48), (0, 49), (1, 299)]):
        at = (int(p.table[s, i // 16]), slice(None), i % 16)
        assert torch.equal(p.d_k_cache[at], k[t]) and torch.equal(p.d_v_cache[at], v[t])


def test_tokens_without_a_place_are_not_stored():
    """A padding token's entry -1, an entry past the cache, an index below zero or past the table: nothing is written for them."""
    p = Paged([(2, 40), (3, 30), (4, 2), (1, 100)], 4, 2, 16, seed=7)
    table = p.d_table.clone()
    table[0, 2] = -1                              # tokens 38 and 39 of sequence 0
    table[1, 1] = p.d_k_cache.shape[0]            # tokens 27 to 29 of sequence 1
    lens = p.d_seq_lens.clone()
    lens[3] = p.d_table.shape[1] * 16 + 1         # the new token lies one past the table
    k, v = (torch.randn(10, 2, D, device="cuda").bfloat16() for _ in range(2))
    before_k, before_v = p.d_k_cache.clone(), p.d_v_cache.clone()
    r = _rotary((64,), False, False)
    q = binding.efq_paged_append(k, v, p.d_k_cache, p.d_v_cache, table, p.d_cu, lens, r, None, p.d_q)
    assert torch.isfinite(q).all()
    for t, i in ((7, 0), (8, 1)):                 # of sequence 2 the last two tokens have an index
        at = (int(p.table[2, 0]), slice(None), i)
        before_v[at] = v[t]
        before_k[at] = p.d_k_cache[at]
    assert torch.equal(before_v.view(torch.int16), p.d_v_cache.view(torch.int16)) and torch.equal(before_k.view(torch.int16), p.d_k_cache.view(torch.int16))


def test_a_step_of_a_model():
    """Appended keys and values are what the attention reads: a prompt in two chunks, then single tokens, against the whole in 64 bits."""
    Hq, Hkv, page, sections = 8, 2, 16, (64,)
    r = _rotary(sections, False, False)
    g = torch.Generator(device="cuda").manual_seed(8)
    total = 150
    q, k, v = (torch.randn(total, H, D, generator=g, device="cuda").bfloat16() for H in (Hq, Hkv, Hkv))
    k_cache, v_cache = (torch.full((12, Hkv, page, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[7, 3, 11, 0, 5, 2, 9, 1, 10, 4, -1]], dtype=torch.int32, device="cuda")
    o = torch.empty_like(q)
    at = 0
    for n in (100, 47, 1, 1, 1):
        new = slice(at, at + n)
        at += n
        cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [at]))
        turned = binding.efq_paged_append(k[new], v[new], k_cache, v_cache, table, cu, lens, r, None, q[new])
        o[new] = binding.efq_paged_attention_fwd(turned, k_cache, v_cache, table, cu, lens, n)
    pos = torch.arange(total, device="cuda", dtype=torch.int32)[None]
    u = 2.0 ** -8
    Q, K = (rotate(x.transpose(0, 1), pos, r.inv_freq, sections, False) for x in (q, k))      # [H, tokens, D]
    seen = torch.ones(total, total, dtype=torch.bool, device="cuda").tril()
    for h in range(Hq):
        s = (Q[h] @ K[h // (Hq // Hkv)].T / math.sqrt(D))
        # rotated q and k are rounded: u of each factor of every product, 2 u and u^2 of the sum of sizes
        ds = (Q[h].abs() @ K[h // (Hq // Hkv)].abs().T / math.sqrt(D)).amax(1, keepdim=True) * (2.1 * u)
        p = torch.softmax(s.masked_fill(~seen, -math.inf), dim=1)
        V = v[:, h // (Hq // Hkv)].double()
        tol = (torch.expm1(2 * ds) + 1.1 * u) * (p @ V.abs()) + u * (p @ V).abs()
        assert float(((o[:, h].double() - p @ V).abs() - tol).max()) <= 0.0


def test_recorded_into_a_graph():
    p = Paged([(1, 30), (1, 200)], 4, 2, 16, seed=9)
    r = _rotary((64,), False, False)
    k, v = (torch.randn(2, 2, D, device="cuda").bfloat16() for _ in range(2))
    q_out = torch.zeros_like(p.d_q)
    call = lambda: binding.efq_paged_append(k, v, p.d_k_cache, p.d_v_cache, *p.tables, r, None, p.d_q, q_out)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for back in (1, 14):                          # other lengths: other places and positions
        p.d_seq_lens.copy_(p.seq_lens - back)
        graph.replay()
        want = torch.empty_like(q_out)
        kc, vc = p.d_k_cache.clone(), p.d_v_cache.clone()
        binding.efq_paged_append(k, v, kc, vc, *p.tables, r, None, p.d_q, want)
        assert torch.equal(want, q_out) and torch.equal(vc.view(torch.int16), p.d_v_cache.view(torch.int16))
        at = (int(p.table[1, (199 - back) // 16]), slice(None), (199 - back) % 16)
        assert torch.equal(p.d_v_cache[at], v[1])


@pytest.mark.parametrize("workload", ["single", "video"])
def test_calibration_on_rotated_workloads(workload, capsys):
    """The tool's --rotary turns the workload's q and k as the formula does: its surface is that of the inputs turned in 64 bits, up to
    what a rounding of q and k that falls the other way may change (a few elements in ten thousand, each by a step of 2^-8)."""
    import numpy as np

    from paper_2609_09721_b200 import calibrate, inputs
    case = inputs.case_single_head(512, 1) if workload == "single" else inputs.case_wan22(1600, seed=5, H=2)
    taus, hs = [-3.06, -2.1], [2.3]
    got, best = calibrate.surface(case, taus, hs, rotary=True)
    r = inputs.rotary_recipe(case)
    assert r.positions.shape == (len(r.sections), case.Sk)
    if workload == "video":
        assert r.positions[:, 0].tolist() == [0, 0, 0] and r.positions[:, 1599].tolist() == [1, 0, 39]
    turn = binding.Rotary.of(r.sections, r.theta, r.interleaved, r.ladder_per_axis)
    q, k, v = (torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16) for x in inputs.make_qkv(case))
    pos = torch.from_numpy(r.positions).cuda()
    q, k = (rotate(x, pos, turn.inv_freq, r.sections, r.interleaved).to(torch.bfloat16) for x in (q, k))
    want, want_best = binding.efq_calibrate(q, k, v, binding.efq_exact_attention_fwd(q, k, v, case.causal), taus, hs, case.causal)
    assert np.allclose(got, np.array(want), rtol=1e-3) and best == want_best
    plain, _ = calibrate.surface(case, taus, hs)
    assert not np.allclose(got, plain, rtol=1e-3)               # the positions matter
    assert calibrate.main(["--workload", "single_head_1024", "--tau=-3.0:-2.7:0.3", "--h", "2.0:2.0:0.2", "--rotary"]) == 0
    assert "with rotary positions" in capsys.readouterr().out


def test_nothing_to_do():
    r = _rotary((64,), False, False)
    pos = torch.zeros(1, 0, dtype=torch.int32, device="cuda")
    x = torch.zeros(2, 4, 0, D, dtype=torch.bfloat16, device="cuda")
    assert binding.efq_rotary(x, x, pos, r)[1].shape == x.shape
    x = torch.zeros(0, 4, 3, D, dtype=torch.bfloat16, device="cuda")
    assert binding.efq_rotary(x, None, torch.zeros(1, 3, dtype=torch.int32, device="cuda"), r)[0].shape == x.shape
    p = Paged([(3, 30)], 4, 2, 16, seed=16)
    k = torch.ones(3, 2, D, device="cuda").bfloat16()
    before = p.d_v_cache.clone()
    q = torch.full_like(p.d_q, 7.0)
    none, zero = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.efq_paged_append(k[:0], k[:0], p.d_k_cache, p.d_v_cache, p.d_table, torch.zeros(2, dtype=torch.int32, device="cuda"), p.d_seq_lens, r, None, p.d_q[:0])
    binding.efq_paged_append(k, k, p.d_k_cache, p.d_v_cache, p.d_table[:0], zero, none, r, None, p.d_q, q)
    binding.efq_paged_append(k, k, p.d_k_cache, p.d_v_cache, p.d_table, torch.zeros(2, dtype=torch.int32, device="cuda"), p.d_seq_lens, r, None, p.d_q, q)
    assert (q == 7.0).all() and torch.equal(before.view(torch.int16), p.d_v_cache.view(torch.int16))


def _step():
    p = Paged([(5, 50), (1, 300)], 4, 2, 16, seed=31)
    k, v = (torch.randn(6, 2, D, device="cuda").bfloat16() for _ in range(2))
    return p, k, v, _rotary((64,), False, False)


def test_what_is_written_counts_as_changed():
    """A tensor's version grows with every call that writes it, and with none that reads it, so that autograd notices that a value it kept is gone."""
    p, k, v, r = _step()
    q_out, lse, o = torch.empty_like(p.d_q), torch.zeros(p.total, 4, device="cuda"), torch.empty_like(p.d_q)
    x, y = p.d_q.transpose(0, 1)[None], k.transpose(0, 1)[None]
    pos = _positions(1, 6, 0)
    read = [k, v, p.d_q, *p.tables, pos, r.inv_freq]
    before = [t._version for t in read]

    def grows(call, *written):
        old = [t._version for t in written]
        call()
        assert all(t._version > a for t, a in zip(written, old)) and [t._version for t in read] == before

    grows(lambda: binding.efq_paged_append(k, v, p.d_k_cache, p.d_v_cache, *p.tables, r, None, p.d_q, q_out), p.d_k_cache, p.d_v_cache, q_out)
    grows(lambda: binding.efq_paged_append(k, v, p.d_k_cache, p.d_v_cache, *p.tables), p.d_k_cache, p.d_v_cache)
    grows(lambda: binding.efq_paged_attention_fwd(q_out, p.d_k_cache, p.d_v_cache, *p.tables, 5, o=o, lse=lse), o, lse)
    grows(lambda: binding.efq_paged_attention_fwd(q_out, p.d_k_cache, p.d_v_cache, *p.tables, 5, o=o), o)
    a, b = torch.empty_like(x), torch.empty_like(y)
    grows(lambda: binding.efq_rotary(x, y, pos, r, q_out=a, k_out=b), a, b)
    grows(lambda: binding.efq_rotary(a, None, pos, r, q_out=a), a)
    w = torch.randn(D, 3, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    kept = p.d_v_cache.clone()[0, 0]
    table = torch.zeros_like(p.d_table)
    cache = kept[None, None].clone()
    loss = (cache[0, 0] @ w).sum()                                # keeps the cache for w's gradient
    lens, cu = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([1], [0, 1]))
    binding.efq_paged_append(k[:1, :1], v[:1, :1], cache.clone(), cache, table[:1], cu, lens)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_tensors_of_the_inference_mode():
    """They have no version; what they get is the same, in the mode and outside."""
    p, k, v, r = _step()
    q_out = binding.efq_paged_append(k, v, p.d_k_cache, p.d_v_cache, *p.tables, r, None, p.d_q)
    want = binding.efq_paged_attention_fwd(q_out, p.d_k_cache, p.d_v_cache, *p.tables, 5)
    with torch.inference_mode():
        kc, vc, q2 = torch.empty_like(p.d_k_cache), torch.empty_like(p.d_v_cache), torch.empty_like(q_out)
        kc.copy_(p.d_k_cache)
        vc.copy_(p.d_v_cache)
        binding.efq_paged_append(k, v, kc, vc, *p.tables, r, None, p.d_q, q2)
        assert torch.equal(binding.efq_paged_attention_fwd(q2, kc, vc, *p.tables, 5), want)
    o = torch.empty_like(want)
    binding.efq_paged_append(k, v, kc, vc, *p.tables, r, None, p.d_q, q2)
    assert torch.equal(binding.efq_paged_attention_fwd(q2, kc, vc, *p.tables, 5, o=o), want)
    assert torch.equal(binding.efq_rotary(q2.transpose(0, 1)[None], None, _positions(1, 6, 0), r, q_out=q2.transpose(0, 1)[None])[0][0].transpose(0, 1), q2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sections,interleaved,inverse", [((64,), False, False), ((22, 21, 21), True, False), ((20, 12), False, True), ((5, 3), True, True)])
def test_gradients(dtype, sections, interleaved, inverse):
    """Through autograd: of both tensors, of one of them, of a projection that both are views of, and of a sum; against the formula in 64 bits."""
    B, S, Hq, Hkv = 2, 37, 5, 3
    g = torch.Generator(device="cuda").manual_seed(32)
    r, pos = _rotary(sections, interleaved, False), _positions(len(sections), S, 700)
    q, k, wq, wk = (torch.randn(B, H, S, D, generator=g, device="cuda").to(dtype) for H in (Hq, Hkv, Hq, Hkv))

    def want(w):
        return rotate(w, pos, r.inv_freq, sections, interleaved, not inverse), rotate_slack(w, dtype, sections, interleaved)

    plain = binding.efq_rotary(q, k, pos, r, inverse)
    q.requires_grad_()
    k.requires_grad_()
    y = binding.efq_rotary(q, k, pos, r, inverse)
    assert all(a.requires_grad and torch.equal(a, b) for a, b in zip(y, plain))
    dq, dk = torch.autograd.grad(y, (q, k), (wq, wk))
    _near(dq, *want(wq))
    _near(dk, *want(wk))
    assert all(torch.equal(a, b) for a, b in zip((dq, dk), binding.efq_rotary(wq, wk, pos, r, not inverse)))
    for a, b, w in ((q, None, wq), (None, k, wk)):               # one tensor alone
        y = [x for x in binding.efq_rotary(a, b, pos, r, inverse) if x is not None]
        _near(torch.autograd.grad(y[0], a if b is None else b, w)[0], *want(w))
    yq, yk = binding.efq_rotary(q, k.detach(), pos, r, inverse)   # one of the two
    assert yq.requires_grad and not yk.requires_grad
    assert torch.equal(torch.autograd.grad(yq, q, wq)[0], dq)
    yq, yk = binding.efq_rotary(q, k, pos, r, inverse)            # one output is not used
    got = torch.autograd.grad(yk, (q, k), wk, allow_unused=True)
    assert got[0] is None and torch.equal(got[1], dk)
    ones = torch.ones(B, Hq, S, D, dtype=dtype, device="cuda")
    _near(torch.autograd.grad(binding.efq_rotary(q, None, pos, r, inverse)[0].sum(), q)[0], *want(ones))
    _near(torch.autograd.grad(binding.efq_rotary(q, None, pos, r, inverse)[0].transpose(2, 3).contiguous(), q, wq.transpose(2, 3).contiguous())[0], *want(wq))
    x = torch.randn(B, S, Hq + 2 * Hkv, D, generator=g, device="cuda").to(dtype).requires_grad_()
    yq, yk = binding.efq_rotary(x[:, :, :Hq].transpose(1, 2), x[:, :, Hq:Hq + Hkv].transpose(1, 2), pos, r, inverse)
    torch.autograd.backward((yq, yk), (wq, wk))
    assert torch.equal(x.grad[:, :, :Hq].transpose(1, 2), dq) and torch.equal(x.grad[:, :, Hq:Hq + Hkv].transpose(1, 2), dk) and (x.grad[:, :, Hq + Hkv:] == 0).all()


def test_gradients_of_gradients_and_of_changed_positions():
    g = torch.Generator(device="cuda").manual_seed(33)
    r, pos = _rotary((64,), False, False), _positions(1, 9, 50)
    q, w, u = (torch.randn(1, 2, 9, D, generator=g, device="cuda").bfloat16() for _ in range(3))
    q.requires_grad_()
    w.requires_grad_()
    dq, = torch.autograd.grad(binding.efq_rotary(q, None, pos, r)[0], q, w, create_graph=True)
    ddw, = torch.autograd.grad(dq, w, u)                          # dq is w turned back, so u is turned on
    assert torch.equal(ddw, binding.efq_rotary(u, None, pos, r)[0])
    y, _ = binding.efq_rotary(q, None, pos, r)
    pos.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(w.detach())


def test_where_there_is_no_gradient():
    """Outputs that are given: refused where a gradient would be lost.  Without gradients all is as before."""
    r, pos = _rotary((64,), False, False), _positions(1, 9, 50)
    q = torch.randn(1, 2, 9, D, device="cuda").bfloat16().requires_grad_()
    k = q.detach().clone()
    want = binding.efq_rotary(k, None, pos, r)[0]
    for args in (dict(q_out=torch.empty_like(k)), dict(q_out=q), dict(q_out=k)):
        with pytest.raises(AssertionError, match="no_grad"):
            binding.efq_rotary(q, None, pos, r, **args)
    with pytest.raises(AssertionError, match="no_grad"):
        binding.efq_rotary(k, None, pos, r, q_out=q)
    with pytest.raises(AssertionError, match="no_grad"):
        binding.efq_rotary(k, q, pos, r, k_out=torch.empty_like(k))
    with torch.no_grad():
        y, _ = binding.efq_rotary(q, None, pos, r)
        assert not y.requires_grad and torch.equal(y, want)
        assert torch.equal(binding.efq_rotary(q, None, pos, r, q_out=torch.empty_like(k))[0], want)
    assert not binding.efq_rotary(k, k, pos, r)[1].requires_grad
    for bad in ((q.float(), None, pos), (q, None, pos[:, :4]), (q, k[:, :, :4], pos)):
        with pytest.raises(AssertionError):
            binding.efq_rotary(*bad, r)


def test_gradients_on_a_side_stream_and_in_a_graph():
    g = torch.Generator(device="cuda").manual_seed(34)
    r, pos = _rotary((64,), False, False), _positions(1, 4000, 50)
    q, w = (torch.randn(1, 8, 4000, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    want = binding.efq_rotary(w, None, pos, r, inverse=True)[0]
    q.requires_grad_()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        s.wait_stream(torch.cuda.current_stream())
        y, _ = binding.efq_rotary(q, None, pos, r, stream=stream)
        torch.cuda.current_stream().wait_stream(s)
        dq, = torch.autograd.grad(y, q, w)
        assert torch.equal(dq, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = binding.efq_rotary(q, None, pos, r)
        dq, = torch.autograd.grad(y, q, w)
    w.copy_(w.flip(2))
    graph.replay()
    assert torch.equal(dq, binding.efq_rotary(w, None, pos, r, inverse=True)[0])


@pytest.mark.parametrize("lens,Hq,Hkv,page", [([(1, 1)], 1, 1, 16), ([(1, 1 + 31 * i) for i in range(70)], 32, 8, 16), ([(300, 300)], 4, 4, 64), ([(129, 1000), (0, 7), (5, 5)], 5, 1, 128),
                                              ([(700, 5000)], 28, 4, 256)])
@pytest.mark.parametrize("sections,interleaved", [((64,), False), ((22, 21, 21), True), ((20, 12), False), (None, False)])
def test_append_of_fp16(lens, Hq, Hkv, page, sections, interleaved):
    """Values up to where the turned ones almost end the type's range, small ones where it has few bits, and a step without a rotation."""
    p = Paged(lens, Hq, Hkv, page, torch.float16, seed=35, tail=2, token_major=len(lens) > 1)
    n = int(p.cu[-1])
    g = torch.Generator(device="cuda").manual_seed(36)
    sizes = 2.0 ** torch.randint(-20, 13, (p.total, 1, 1), generator=g, device="cuda")           # a size a token: both channels of a pair have it
    k, v = ((torch.randn(p.total, Hkv, D, generator=g, device="cuda") * sizes).half() for _ in range(2))
    r = None if sections is None else _rotary(sections, interleaved, False)
    index = torch.cat([torch.arange(m - a, m) for a, m in lens] + [torch.zeros(2, dtype=torch.long)]).cuda()
    pos = None if sections is None else torch.stack([index // (3 ** a) for a in range(len(sections))]).int()
    turned = (lambda x: x.double()) if r is None else lambda x: rotate(x.transpose(0, 1), pos, r.inv_freq, sections, interleaved).transpose(0, 1)  # noqa: E731
    slack = (lambda x: torch.zeros_like(x, dtype=torch.float64)) if r is None else lambda x: rotate_slack(x, torch.float16, sections, interleaved)  # noqa: E731
    assert float(k.abs().max()) * 2 ** 0.5 < 65504
    want_k, want_v = p.d_k_cache.clone(), p.d_v_cache.clone()
    place = [(int(p.table[s, i // page]), i % page) for s, (a, m) in enumerate(lens) for i in range(m - a, m)]
    pages, slots = (torch.tensor([x[j] for x in place], device="cuda") for j in (0, 1))
    q_out = torch.full((p.total, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    binding.efq_paged_append(k, v, p.d_k_cache, p.d_v_cache, *p.tables, r, pos, p.d_q, q_out)
    assert (q_out[n:] == 7.0).all()
    _near(q_out[:n], turned(p.d_q)[:n], slack(p.d_q)[:n])
    _near(p.d_k_cache[pages, :, slots], turned(k)[:n], slack(k)[:n])
    want_k[pages, :, slots], want_v[pages, :, slots] = p.d_k_cache[pages, :, slots], v[:n]
    same = lambda a, b: torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))  # noqa: E731
    assert same(p.d_k_cache, want_k) and same(p.d_v_cache, want_v)


def test_a_step_of_a_model_in_fp16():
    """Append and attention of one step, against the whole in 64 bits."""
    Hq, Hkv, page, n, total = 8, 2, 32, 40, 300
    p = Paged([(n, total)], Hq, Hkv, page, torch.float16, seed=37, hot=0)
    r = _rotary((64,), False, False)
    k, v = p.k[0].cuda(), p.v[0].cuda()
    cu = torch.tensor([0, total], dtype=torch.int32, device="cuda")
    binding.efq_paged_append(k, v, p.d_k_cache, p.d_v_cache, p.d_table, cu, p.d_seq_lens, r)      # the prompt, its last tokens among it
    q = binding.efq_paged_append(k[-n:], v[-n:], p.d_k_cache, p.d_v_cache, *p.tables, r, None, p.d_q)
    o = binding.efq_paged_attention_fwd(q, p.d_k_cache, p.d_v_cache, *p.tables, n)
    pos = torch.arange(total, device="cuda", dtype=torch.int32)[None]
    Q = rotate(p.d_q.transpose(0, 1), pos[:, -n:], r.inv_freq, (64,), False)
    K = rotate(k.transpose(0, 1), pos, r.inv_freq, (64,), False)
    seen = torch.ones(n, total, dtype=torch.bool, device="cuda").tril(total - n)
    u = 2.0 ** -11
    for h in range(Hq):
        s = Q[h] @ K[h // 4].T / math.sqrt(D)
        # rotated q and k are rounded: u of each factor of every product, 2 u and u^2 of the sum of sizes
        ds = (Q[h].abs() @ K[h // 4].abs().T / math.sqrt(D)).amax(1, keepdim=True) * (2.1 * u)
        w = torch.softmax(s.masked_fill(~seen, -math.inf), dim=1)
        V = v[:, h // 4].double()
        tol = (torch.expm1(2 * ds) + 1.1 * u) * (w @ V.abs()) + u * (w @ V).abs() + 2.0 ** -25
        assert float(((o[:, h].double() - w @ V).abs() - tol).max()) <= 0.0
