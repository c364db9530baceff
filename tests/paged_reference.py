"""Plain forms in 64 bits of the operators around a paged cache, and paged problems to run them on."""
import math

import torch

D = 128


def rotate(x, positions, inv_freq, sections, interleaved, inverse=False):
    """x [..., tokens, D], positions [axes, tokens]: float64, pair by pair."""
    y = x.double().clone()
    R = sum(sections)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    for p in range(R):
        angle = positions[axis[p]].double() * inv_freq[p].double()
        c, s = angle.cos(), angle.sin() * (-1.0 if inverse else 1.0)
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + R)
        a, b = x[..., i].double(), x[..., j].double()
        y[..., i], y[..., j] = a * c - b * s, a * s + b * c
    return y


def rotate_slack(x, dtype, sections, interleaved):
    """How far a rotated value may be off beside half a step of its type: sine and cosine are FP32 functions (2 ulp) of an FP32 argument
    (half an ulp of at most pi), two products and a sum are rounded: 8 half-ulps of what the pair holds."""
    y = torch.zeros_like(x, dtype=torch.float64)
    R = sum(sections)
    for p in range(R):
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + R)
        size = x[..., i].double().abs() + x[..., j].double().abs()
        y[..., i] = y[..., j] = size * 8 * 2.0 ** -24
    return y


class Paged:
    """A step on a paged cache: `lens` holds (new tokens, tokens) of each sequence.  Pages are handed out in no order, what no sequence owns
    and what lies behind a sequence's last token is NaN, and unused entries of the table are -1."""

    def __init__(self, lens, Hq, Hkv, page, dtype=torch.bfloat16, seed=0, device="cuda", hot=8, spare=2, token_major=False, tail=0, slack=1):
        self.lens, self.Hq, self.Hkv, self.page, self.dtype = lens, Hq, Hkv, page, dtype
        g = torch.Generator().manual_seed(seed)
        n = len(lens)
        used = [-(-k // page) for _, k in lens]
        pages = sum(used) + spare
        order = torch.randperm(pages, generator=g)
        self.table = torch.full((n, max(used, default=0) + slack), -1, dtype=torch.int32)
        at = 0
        for i, u in enumerate(used):
            self.table[i, :u] = order[at:at + u].int()
            at += u
        q_len = [a for a, _ in lens]
        self.cu = torch.tensor([sum(q_len[:i]) for i in range(n + 1)], dtype=torch.int32)
        self.seq_lens = torch.tensor([k for _, k in lens], dtype=torch.int32)
        self.total = sum(q_len) + tail
        self.q = torch.randn(self.total, Hq, D, generator=g).to(dtype)
        shape = (pages, page, Hkv, D) if token_major else (pages, Hkv, page, D)
        self.k_cache, self.v_cache = (torch.full(shape, math.nan, dtype=dtype) for _ in range(2))
        if token_major:
            self.k_cache, self.v_cache = self.k_cache.transpose(1, 2), self.v_cache.transpose(1, 2)
        channels = torch.randperm(D, generator=g)[:hot]
        self.k, self.v = [], []
        for i, (_, m) in enumerate(lens):
            k, v = torch.randn(m, Hkv, D, generator=g), torch.randn(m, Hkv, D, generator=g).to(dtype)
            k[..., channels] *= 10.0
            k = k.to(dtype)
            self.k.append(k)
            self.v.append(v)
            at, slot = torch.arange(m) // page, torch.arange(m) % page
            p = self.table[i].long()[at]
            self.k_cache[p, :, slot], self.v_cache[p, :, slot] = k, v
        self.device = device
        for name in ("table", "cu", "seq_lens", "q", "k_cache", "v_cache"):
            setattr(self, "d_" + name, getattr(self, name).to(device))
        if token_major:         # .to() keeps the strides of a dense permuted tensor; the test relies on it
            assert self.d_k_cache.stride(2) == Hkv * D

    @property
    def tables(self):
        return self.d_table, self.d_cu, self.d_seq_lens

    @property
    def max_q(self):
        return max((a for a, _ in self.lens), default=0)

    def attention(self, causal, scale=None):
        """o [total, Hq, D] and lse [total, Hq] in 64 bits (rows behind the last sequence 0), and how far each may be off."""
        scale = 1.0 / math.sqrt(D) if scale is None else scale
        dev = self.device
        o = torch.zeros(self.total, self.Hq, D, dtype=torch.float64, device=dev)
        lse = torch.full((self.total, self.Hq), -math.inf, dtype=torch.float64, device=dev)
        o_tol, lse_tol = torch.zeros_like(o), torch.zeros_like(lse)
        u = torch.finfo(self.dtype).eps / 2
        G, t = self.Hq // self.Hkv, 0
        for (n, m), k, v in zip(self.lens, self.k, self.v):
            if n == 0:
                continue
            k, v = k.to(dev).double(), v.to(dev).double()
            seen = torch.ones(n, m, dtype=torch.bool, device=dev)
            if causal:
                seen = seen.tril(m - n)
            for h in range(self.Hq if m else 0):
                q, kh, vh = self.d_q[t:t + n, h].double(), k[:, h // G], v[:, h // G]
                s = (q @ kh.T * scale).masked_fill(~seen, -math.inf)
                top = s.amax(1, keepdim=True)
                top = top.masked_fill(top == -math.inf, 0.0)
                p = (s - top).exp()
                l = p.sum(1, keepdim=True)
                safe = l.masked_fill(l == 0, 1.0)
                o[t:t + n, h] = p @ vh / safe
                lse[t:t + n, h] = (top + l.log())[:, 0]
                # a score of 128 products comes out of 8 steps of the tensor core, each a truncated addition of up to 2^-22 of what is summed;
                # in units of log2 and less the maximum it is rounded three times more
                size = (q.abs() @ kh.abs().T * scale).masked_fill(~seen, 0.0).amax(1, keepdim=True)
                ds = 2.0 ** -19 * size + 2.0 ** -21
                # probabilities are rounded once (u of each), FP32 sums of up to m terms in tiles: 2^-24 a step over at most 512 sequential
                # steps, the output is rounded once
                mean = p @ vh.abs() / safe
                o_tol[t:t + n, h] = (u * 1.01 + 2 * ds + 2.0 ** -15) * mean + u * o[t:t + n, h].abs()
                lse_tol[t:t + n, h] = (ds + 2.0 ** -15)[:, 0] + 2.0 ** -22 * lse[t:t + n, h].nan_to_num(0, 0, 0).abs()
            t += n
        if self.dtype == torch.float16:
            o_tol += 2.0 ** -25         # its smallest steps
        return o, lse, o_tol, lse_tol
