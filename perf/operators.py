"""Operators around a paged cache and rotary positions: their cases and their plain forms.

Three operators of paper_2609_09721_b200.binding:

  rotary      efq_rotary: positions with one or several axes turned into q and k before a dense forward, or, inverse, into their
              gradients behind it
  append      efq_paged_append: new keys and values into a paged cache, keys (and the queries beside them) rotated on the way
  attention   efq_paged_attention_fwd: softmax attention of the new tokens of each sequence over its pages

Shapes are those of the package's own workloads: Qwen3-8B-shaped GQA serving (32 query heads on 8 KV heads of 128 channels, K with
outlier channels) and WAN2.2-shaped video self-attention (24 heads, 32760 tokens = 21 x 30 x 52 positions in time, height, width).
"""
import math
import random

import torch

own = False

D = 128
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, kind, **more):
    return dict({"name": name} if name else {}, kind=kind, **more)


def _rotary(name, B, S, Hq, Hkv, sections, interleaved, theta, ladder, first, dtype, inverse):
    return _case(name, "rotary", B=B, S=S, Hq=Hq, Hkv=Hkv, sections=sections, interleaved=interleaved, theta=theta, ladder=ladder,
                 first=first, dtype=dtype, inverse=inverse)


def _append(name, Hq, Hkv, n_seqs, q_min, q_max, k_min, k_max, page, sections, interleaved, dtype, lengths):
    return _case(name, "append", Hq=Hq, Hkv=Hkv, n_seqs=n_seqs, q_min=q_min, q_max=q_max, k_min=k_min, k_max=k_max, page=page,
                 sections=sections, interleaved=interleaved, theta=1e6, ladder="shared", dtype=dtype, lengths=lengths)


def _attention(name, Hq, Hkv, n_seqs, q_min, q_max, k_min, k_max, page, causal, dtype, lse, lengths):
    return _case(name, "attention", Hq=Hq, Hkv=Hkv, n_seqs=n_seqs, q_min=q_min, q_max=q_max, k_min=k_min, k_max=k_max, page=page,
                 causal=causal, dtype=dtype, lse=lse, lengths=lengths)


def listed():
    return [
        # video diffusion: q and k of a self-attention over 21 x 30 x 52 latent positions, from the projections' token-major layout
        _rotary("rotary_video_32760", 1, 32760, 24, 24, "22,21,21", True, 1e4, "own", 0, "bf16", False),
        # the gradients of the same for a short clip
        _rotary("rotary_video_grad_4097", 1, 4097, 24, 24, "22,21,21", True, 1e4, "own", 0, "bf16", True),
        # two prompts late in a long document: far positions
        _rotary("rotary_prompt_1087", 2, 1087, 32, 8, "64", False, 1e6, "shared", 900000, "fp16", False),
        # a decode step of 64 conversations: one token each, latency
        _append("append_decode_64", 32, 8, 64, 1, 1, 512, 2048, 16, "64", False, "bf16", 1),
        # a chunk of a long prompt, with image tokens that have a time, a height and a width
        _append("append_chunk_8192", 32, 8, 1, 8192, 8192, 12001, 12001, 64, "16,24,24", False, "bf16", 2),
        # one decode step of one conversation: a single token over a ragged context, latency
        _attention("decode_one_8191", 32, 8, 1, 1, 1, 8191, 8191, 16, True, "bf16", False, 3),
        # a decode step over 64 conversations
        _attention("decode_64", 32, 8, 64, 1, 1, 4096, 8192, 64, True, "bf16", False, 4),
        # a speculative step: five draft tokens in each of 16 conversations
        _attention("draft_16x5", 32, 8, 16, 5, 5, 2000, 9000, 32, True, "fp16", True, 5),
        # chunks and single tokens of mixed lengths in one batch, as a server forms it
        _attention("mixed_16", 28, 4, 16, 1, 700, 700, 6000, 16, True, "bf16", True, 6),
        # a short chunk behind a cached prompt
        _attention("chunk_300", 32, 8, 1, 300, 300, 9000, 9000, 64, True, "bf16", False, 7),
        # prompt processing in chunks: one of the last of a long document
        _attention("chunk_2048", 32, 8, 1, 2048, 2048, 32768, 32768, 128, True, "bf16", False, 8),
        # queries of another text over a cached document, no mask
        _attention("cross_999", 24, 24, 2, 999, 999, 3000, 5001, 128, False, "bf16", True, 9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(1, 1), (4, 4), (8, 2), (16, 2), (24, 24), (28, 4), (32, 8), (40, 8), (32, 32), (12, 4), (8, 1)]
SECTIONS = ["64", "64", "32", "16,24,24", "22,21,21", "20,12", "8,8,8"]
SCORES_MAX = 2048 * 32768 * 32               # scores of the largest listed case, padded to the longest sequence as the plain form does
ELEMENTS_MAX = 2 * 32760 * 24 * D


def draw(rng):
    """One more case of the same ranges."""
    while True:
        c = _draw(rng)
        if c["kind"] == "rotary":
            if c["B"] * c["S"] * (c["Hq"] + c["Hkv"]) * D <= ELEMENTS_MAX:
                return c
            continue
        q, k = _lengths(c)
        if sum(k) * c["Hkv"] * D > 4e8 or sum(q) * (c["Hq"] + 2 * c["Hkv"]) * D > ELEMENTS_MAX:
            continue
        if c["kind"] == "append" or len(q) * max(q) * max(k) * c["Hq"] <= SCORES_MAX and len(k) * max(k) * c["Hkv"] * D <= 8e8:
            return c


def _draw(rng):
    Hq, Hkv = rng.choice(HEADS)
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp16"])
    sections, interleaved = rng.choice(SECTIONS), rng.random() < 0.4
    page, lengths = rng.choice([16, 16, 32, 64, 128, 256]), rng.randrange(1 << 20)
    kind = rng.choice(["rotary", "append", "append", "decode", "draft", "mixed", "chunk", "cross"])
    if kind == "rotary":
        return _rotary("", rng.choice([1, 1, 2, 3]), _log(rng, 1, 32760), Hq, Hkv, sections, interleaved, rng.choice([1e4, 1e6]),
                       rng.choice(["own", "shared"]), rng.choice([0, 0, _log(rng, 1, 1000000)]), dtype, rng.random() < 0.4)
    if kind == "append":
        if rng.random() < 0.5:
            top = _log(rng, 16, 4096)
            return _append("", Hq, Hkv, _log(rng, 1, 200), 1, rng.choice([1, 1, 4]), max(1, top // 4), top, page, sections, interleaved,
                           dtype, lengths)
        top = _log(rng, 5, 9000)
        return _append("", Hq, Hkv, rng.randint(1, 6), max(1, top // 3), top, top, top + _log(rng, 1, 9000), page, sections, interleaved,
                       dtype, lengths)
    lse = rng.random() < 0.5
    if kind == "decode":
        top = _log(rng, 60, 30000)
        return _attention("", Hq, Hkv, _log(rng, 1, 128), 1, 1, max(1, top // 4), top, page, True, dtype, lse, lengths)
    if kind == "draft":
        top = _log(rng, 60, 16000)
        return _attention("", Hq, Hkv, _log(rng, 1, 64), 1, rng.randint(2, 9), max(10, top // 3), max(10, top), page, True, dtype, lse, lengths)
    if kind == "mixed":
        top = _log(rng, 20, 1500)
        return _attention("", Hq, Hkv, rng.randint(2, 24), 1, top, top, top + _log(rng, 10, 8000), page, True, dtype, lse, lengths)
    if kind == "chunk":
        n = _log(rng, 20, 4000)
        return _attention("", Hq, Hkv, rng.choice([1, 1, 2]), n, n, n, n + _log(rng, 1, 40000), page, True, dtype, lse, lengths)
    return _attention("", Hq, Hkv, rng.randint(1, 4), 1, _log(rng, 16, 2000), 1, _log(rng, 30, 8000), page, False, dtype, lse, lengths)


def _lengths(case):
    """New tokens and all tokens of each sequence."""
    rng = random.Random(case["lengths"])
    q = [rng.randint(case["q_min"], case["q_max"]) for _ in range(case["n_seqs"])]
    k = [rng.randint(case["k_min"], case["k_max"]) for _ in range(case["n_seqs"])]
    return q, [max(a, b) for a, b in zip(q, k)] if case.get("causal", True) else k


def _sections(case):
    return tuple(int(x) for x in case["sections"].split(","))


def _frequencies(case):
    """Radians a position of each pair: one falling ladder over all pairs, or one for each axis."""
    s = _sections(case)
    if case["ladder"] == "own":
        e = [j / n for n in s for j in range(n)]
    else:
        e = [j / sum(s) for j in range(sum(s))]
    return torch.tensor([case["theta"] ** -x for x in e], dtype=torch.float64, device="cuda")


def _axis(case):
    """Of each pair: the axis whose position turns it."""
    return torch.tensor([i for i, n in enumerate(_sections(case)) for _ in range(n)], device="cuda")


def _positions(case, tokens, first):
    """int32 [axes, tokens]: a text's running index, or places in a grid of frames."""
    n = len(_sections(case))
    t = torch.arange(tokens, device="cuda", dtype=torch.int32) + first
    if n == 1:
        return t[None].contiguous()
    w, h = 52, 30
    grid = [t // (w * h), t // w % h, t % w] if n == 3 else [t // w, t % w]
    return torch.stack(grid).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    if case["kind"] == "rotary":
        B, S = case["B"], case["S"]
        s = {"kind": "rotary", "inverse": case["inverse"], "sections": _sections(case), "interleaved": case["interleaved"],
             "inv_freq": _frequencies(case), "axis": _axis(case), "positions": _positions(case, S, case["first"])}
        for name, H in (("q", case["Hq"]), ("k", case["Hkv"])):
            # a forward takes the projections, token-major, and leaves what the dense forwards read, head-major; a gradient comes
            # from the head-major side and goes back to the projections
            x = normal(B, S, H, D).to(dtype).permute(0, 2, 1, 3)
            out = torch.empty((B, H, S, D), dtype=dtype, device="cuda")
            s[name], s[name + "_out"] = (out.copy_(x), torch.empty_like(x)) if case["inverse"] else (x, out)
        return s
    q_len, k_len = _lengths(case)
    n, Hq, Hkv, page = len(q_len), case["Hq"], case["Hkv"], case["page"]
    used = [-(-k // page) for k in k_len]
    pages = sum(used) + 3                                                    # some stay free
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)    # pages are handed out in no order
    rows = torch.full((n, max(used) + 1), -1, dtype=torch.int64)             # unused entries name no page
    at = 0
    for i, u in enumerate(used):
        rows[i, :u] = torch.arange(at, at + u)
        at += u
    rows = rows.cuda()
    table = torch.where(rows < 0, -1, order[rows.clamp(min=0)]).to(torch.int32).contiguous()
    T = sum(q_len)
    cu = torch.tensor([sum(q_len[:i]) for i in range(n + 1)], dtype=torch.int32, device="cuda")
    s = {"kind": case["kind"], "page_table": table, "cu_seqlens": cu, "seq_lens": torch.tensor(k_len, dtype=torch.int32, device="cuda"),
         "max_q": max(q_len), "max_k": max(k_len)}
    # queries, keys and values of the new tokens lie side by side in a row, as one projection leaves them
    qkv = normal(T, Hq + 2 * Hkv, D)
    hot = torch.randperm(D, generator=g, device="cuda")[:8]
    qkv[:, Hq:Hq + Hkv, hot] *= 10.0                                         # outlier channels of K
    qkv = qkv.to(dtype)
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    s["k_cache"] = torch.empty((pages, Hkv, page, D), dtype=dtype, device="cuda")
    s["v_cache"] = torch.empty_like(s["k_cache"])
    step = max(1, (1 << 27) // (Hkv * page * D))
    for p in range(0, pages, step):
        x = normal(min(step, pages - p), Hkv, page, D)
        x[..., hot] *= 10.0
        s["k_cache"][p:p + step] = x.to(dtype)
        s["v_cache"][p:p + step] = normal(min(step, pages - p), Hkv, page, D).to(dtype)
    if case["kind"] == "append":
        seq = torch.repeat_interleave(torch.arange(n), torch.tensor(q_len)).cuda()
        index = (s["seq_lens"] - cu.diff())[seq] + torch.arange(T, device="cuda", dtype=torch.int32) - cu[seq]
        axes = len(_sections(case))
        grid = [index // 1560, index // 52 % 30, index % 52] if axes == 3 else [index // 52, index % 52] if axes == 2 else [index]
        s["positions"] = torch.stack(grid).to(torch.int32).contiguous()
        s |= {"sections": _sections(case), "interleaved": case["interleaved"], "inv_freq": _frequencies(case), "axis": _axis(case),
              "q_out": torch.empty((T, Hq, D), dtype=dtype, device="cuda")}
    else:
        s |= {"causal": case["causal"], "o": torch.empty((T, Hq, D), dtype=dtype, device="cuda"),
              "lse": torch.empty((T, Hq), dtype=torch.float32, device="cuda") if case["lse"] else None}
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_turn(x, s, inverse=False):
    """x [..., H, T, D]: the rotated values, rounded once."""
    inv_freq, interleaved = s["inv_freq"], s["interleaved"]
    angle = s["positions"].double()[s["axis"]].T * inv_freq                  # [T, pairs], 64 bits: positions reach far
    cos, sin = angle.cos().float(), angle.sin().float()
    if inverse:
        sin = -sin
    R = inv_freq.numel()
    f = x.float()
    a, b = (f[..., 0:2 * R:2], f[..., 1:2 * R:2]) if interleaved else (f[..., :R], f[..., R:2 * R])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((u, v), dim=-1).flatten(-2) if interleaved else torch.cat((u, v), dim=-1)
    return torch.cat((turned, f[..., 2 * R:]), dim=-1).to(x.dtype)


def _sequence_of(s):
    """Of each new token: its sequence, and its index there."""
    cu = s["cu_seqlens"].long()
    t = torch.arange(s["q"].shape[0], device=cu.device)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return seq, (s["seq_lens"].long() - cu.diff())[seq] + t - cu[seq]


def _plain_append(s):
    turn = lambda x: _plain_turn(x.transpose(0, 1), s).transpose(0, 1)  # noqa: E731
    s["q_out"].copy_(turn(s["q"]))
    seq, index = _sequence_of(s)
    P = s["k_cache"].shape[2]
    page, slot = s["page_table"].long()[seq, index // P], index % P
    s["k_cache"][page, :, slot] = turn(s["k"])
    s["v_cache"][page, :, slot] = s["v"]
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    q, cu = s["q"], s["cu_seqlens"].long()
    _, Hkv, P, _ = s["k_cache"].shape
    n, T, Hq = cu.numel() - 1, q.shape[0], q.shape[1]
    G, top = Hq // Hkv, s["max_q"]
    pages = s["page_table"].long()[:, :-(-s["max_k"] // P)].clamp(min=0)
    K, V = (c[pages].float().transpose(1, 2).reshape(n, Hkv, -1, D) for c in (s["k_cache"], s["v_cache"]))
    L = K.shape[2]
    key = torch.arange(L, device=q.device)
    lens, q_lens = s["seq_lens"].long(), cu.diff()
    V = V.masked_fill((key >= lens[:, None])[:, None, :, None], 0.0)
    at = (cu[:-1, None] + torch.arange(top, device=q.device)).clamp(max=T - 1)
    Q = q.float()[at].reshape(n, top, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * top, D)
    last = lens[:, None].expand(n, top)
    if s["causal"]:
        last = torch.minimum(last, (lens - q_lens)[:, None] + torch.arange(top, device=q.device) + 1)
    hidden = (key >= last[:, :, None])[:, None, None]                        # [n, 1, 1, top, L]
    S = torch.matmul(Q, K.transpose(2, 3)).mul_(D ** -0.5)
    S.view(n, Hkv, G, top, L).masked_fill_(hidden, -math.inf)
    m = S.amax(dim=-1, keepdim=True)
    base = m.masked_fill(m == -math.inf, 0.0)
    p = S.sub_(base).exp_()
    l = p.sum(dim=-1, keepdim=True)
    O = torch.matmul(p, V) / l.masked_fill(l == 0.0, 1.0)
    lse = (base + l.log()).squeeze(-1)
    seq, index = _sequence_of(s)
    i = index - (lens - q_lens)[seq]
    s["o"].copy_(O.view(n, Hkv, G, top, D).permute(0, 3, 1, 2, 4).reshape(n, top, Hq, D)[seq, i])
    out = {"o": s["o"]}
    if s["lse"] is not None:
        out["lse"] = s["lse"].copy_(lse.view(n, Hkv, G, top).permute(0, 3, 1, 2).reshape(n, top, Hq)[seq, i])
    return out


def _plain(s):
    if s["kind"] == "rotary":
        return {x: s[x + "_out"].copy_(_plain_turn(s[x], s, s["inverse"])) for x in ("q", "k")}
    return _plain_append(s) if s["kind"] == "append" else _plain_attention(s)


# ------------------------------------------------------------------------------------------------ the framework's operators

def _rotary_of(s, binding):
    """The description of the rotation that a program makes once and keeps."""
    if "rotary" not in s:
        s["rotary"] = binding.Rotary(s["inv_freq"], s["sections"], s["interleaved"])
    return s["rotary"]


def _own(s):
    from paper_2609_09721_b200 import binding
    if s["kind"] == "rotary":
        q, k = binding.efq_rotary(s["q"], s["k"], s["positions"], _rotary_of(s, binding), s["inverse"], s["q_out"], s["k_out"])
        return {"q": q, "k": k}
    if s["kind"] == "append":
        q = binding.efq_paged_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["page_table"], s["cu_seqlens"], s["seq_lens"],
                                     _rotary_of(s, binding), s["positions"], s["q"], s["q_out"])
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if "workspace" not in s:
        s["workspace"] = torch.empty(binding.efq_paged_attention_workspace_bytes(s["q"].shape[1], s["k_cache"].shape[1], s["max_q"], D),
                                     dtype=torch.uint8, device="cuda")
    o = binding.efq_paged_attention_fwd(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["cu_seqlens"], s["seq_lens"], s["max_q"],
                                        s["causal"], 0.0, s["o"], s["lse"], s["workspace"])
    return {"o": o} if s["lse"] is None else {"o": o, "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# ------------------------------------------------------------------------------------------------ work, and the definitions in 64 bits

def work(case):
    if case["kind"] == "rotary":
        n = case["B"] * case["S"] * (case["Hq"] + case["Hkv"])
        return {"bytes": 4 * n * D + 4 * len(_sections(case)) * case["S"], "flops": 6 * n * sum(_sections(case))}
    q, k = _lengths(case)
    Hq, Hkv = case["Hq"], case["Hkv"]
    tables = 4 * (2 * len(q) + 1 + sum(-(-x // case["page"]) for x in k))
    if case["kind"] == "append":
        n = sum(q) * (Hq + 2 * Hkv)
        return {"bytes": 4 * n * D + 4 * len(_sections(case)) * sum(q) + tables, "flops": 6 * sum(q) * (Hq + Hkv) * sum(_sections(case))}
    pairs = sum(a * b - (a * (a - 1) // 2 if case["causal"] else 0) for a, b in zip(q, k))
    return {"bytes": 4 * D * (sum(k) * Hkv + sum(q) * Hq) + tables + (4 * sum(q) * Hq if case["lse"] else 0), "flops": 4.0 * D * Hq * pairs}


def _exact_turn(x, positions, case):
    """x [..., tokens, D] in 64 bits; each pair is a complex number that is turned by its angle."""
    s, R = _sections(case), sum(_sections(case))
    places = torch.cat([positions[i].double()[:, None].expand(-1, n) for i, n in enumerate(s)], dim=1)
    angle = places * _frequencies(case)
    turn = torch.polar(torch.ones_like(angle), -angle if case.get("inverse") else angle)
    y = x.double().clone()
    first, second = (slice(0, 2 * R, 2), slice(1, 2 * R, 2)) if case["interleaved"] else (slice(0, R), slice(R, 2 * R))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return {x: _exact_turn(s[x], s["positions"], case) for x in ("q", "k")}
    q_len, k_len = _lengths(case)
    P, table = case["page"], s["page_table"].tolist()
    if case["kind"] == "append":
        out = {"q": _exact_turn(s["q"].transpose(0, 1), s["positions"], case).transpose(0, 1).contiguous(), "k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double()}
        k = _exact_turn(s["k"].transpose(0, 1), s["positions"], case).transpose(0, 1)
        t = 0
        for i, n in enumerate(q_len):
            index = torch.arange(k_len[i] - n, k_len[i])
            page, slot = torch.tensor(table[i])[index // P].cuda(), (index % P).cuda()
            out["k_cache"][page, :, slot] = k[t:t + n]
            out["v_cache"][page, :, slot] = s["v"][t:t + n].double()
            t += n
        return out
    Hq, Hkv = case["Hq"], case["Hkv"]
    T, G = sum(q_len), Hq // Hkv
    o = torch.zeros((T, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    t = 0
    for i, (n, m) in enumerate(zip(q_len, k_len)):
        pages = torch.tensor(table[i][:-(-m // P)], dtype=torch.long, device="cuda")
        seen = torch.ones((n, m), dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen = seen.tril(m - n)
        for h in range(Hkv):
            k, v = (c[pages, h].reshape(-1, D)[:m].double() for c in (s["k_cache"], s["v_cache"]))
            for j in range(h * G, (h + 1) * G):
                scores = (s["q"][t:t + n, j].double() @ k.T / math.sqrt(D)).masked_fill(~seen, -math.inf)
                lse[t:t + n, j] = torch.logsumexp(scores, dim=1)
                o[t:t + n, j] = torch.softmax(scores, dim=1).nan_to_num(0.0) @ v
        t += n
    return {"o": o} if s["lse"] is None else {"o": o, "lse": lse}
