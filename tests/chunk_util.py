"""Inputs and 64-bit references for the cache calls and the attention of token chunks."""
from __future__ import annotations

import math

import torch

PAGE = 16
STALE_CODE, STALE_SCALE = 0x7F, 255          # what slots without a token hold


def gen(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def i32(values, device="cuda"):
    return torch.tensor(values, dtype=torch.int32, device=device)


def two_to(e):
    """2^e in 64 bits, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantise64(x):
    """(values of the codes, exponents) of rows [..., D] by the definition, in 64 bits."""
    x = x.double()
    finite = torch.isfinite(x)
    a = torch.where(finite, x, 0.0).abs().amax(-1, keepdim=True)
    e = torch.where(a > 0, torch.frexp(a).exponent.long() - 10, -100).clamp(min=-100)
    e = torch.where(a > 448.0 * two_to(e), e + 1, e)
    e = torch.where(a > 448.0 * two_to(e), e + 1, e)
    y = x * two_to(-e)
    step = two_to(torch.frexp(torch.where(finite, y, 0.0).abs().clamp(min=2.0 ** -6)).exponent.long() - 4)
    code = torch.round(y / step) * step
    code = torch.where((e == 120) & finite, code.clamp(-240.0, 240.0), code)
    return torch.where(finite, code, math.nan), e[..., 0]


def as_bytes(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


class Cache:
    """A cache of random rows for requests of need[b] slots; slots past them hold no numbers, block table entries past them no blocks."""

    def __init__(self, g, need, heads, dim, dtype, paged, device="cuda", layers=None, slack=5):
        self.need, self.heads, self.dim, self.paged = need, heads, dim, paged
        e4m3 = dtype == torch.float8_e4m3fn
        if paged:
            blocks = [-(-n // PAGE) for n in need]
            pool = sum(blocks) + 2
            order = torch.randperm(pool, generator=g, device=device).to(torch.int32)
            self.table = torch.full((len(need), max(max(blocks), 1)), 1 << 30, dtype=torch.int32, device=device)
            at = 0
            for b, n in enumerate(blocks):
                self.table[b, :n] = order[at:at + n]
                at += n
            rows, per = pool, PAGE
        else:
            self.table, rows, per = None, len(need), max(max(need), 1) + slack
        self.capacity = self.table.shape[1] * PAGE if paged else per
        used = torch.zeros((rows, per), dtype=torch.bool, device=device)
        for b, n in enumerate(need):
            if paged:
                for t in range(-(-n // PAGE)):
                    used[int(self.table[b, t]), :min(PAGE, n - t * PAGE)] = True
            else:
                used[b, :n] = True
        self.made = []
        for _ in range(2 * (layers or 1)):
            x = torch.empty((rows, heads, per, dim), dtype=torch.float32, device=device).normal_(generator=g)
            if e4m3:
                x = x * torch.exp(torch.empty((rows, heads, per, 1), device=device).normal_(0, 0.7, generator=g))
                code, e = quantise64(x)
                code = code.float().to(torch.float8_e4m3fn).view(torch.uint8).masked_fill(~used[:, None, :, None], STALE_CODE)
                scale = (e + 127).to(torch.uint8).masked_fill(~used[:, None], STALE_SCALE)
                self.made.append((code.contiguous().view(torch.float8_e4m3fn), scale.contiguous()))
            else:
                self.made.append((x.to(dtype).masked_fill(~used[:, None, :, None], math.nan).contiguous(), None))
        if layers:
            stack = lambda ts: torch.stack([as_bytes(t) for t in ts]).view(dtype if ts[0].dtype != torch.uint8 else torch.uint8)
            (self.k, self.ks), (self.v, self.vs) = ((stack([m[0] for m in self.made[i::2]]),
                                                     stack([m[1] for m in self.made[i::2]]) if e4m3 else None) for i in (0, 1))
        else:
            (self.k, self.ks), (self.v, self.vs) = self.made

    @property
    def scales(self):
        return None if self.ks is None else (self.ks, self.vs)

    def places(self, b, slots):
        if not self.paged:
            return [(b, t) for t in slots]
        return [(int(self.table[b, t // PAGE]), t % PAGE) for t in slots]

    def rows64(self, b, slots, which):
        """[slots, heads, D] values in 64 bits of K (which 0) or V."""
        at = self.places(b, slots)
        r, t = (torch.tensor([p[i] for p in at], dtype=torch.long, device=self.k.device) for i in (0, 1))
        c, s = ((self.k, self.ks), (self.v, self.vs))[which]
        x = as_bytes(c)[r, :, t].view(c.dtype).double()
        return x if s is None else x * two_to(s[r, :, t].long() - 127)[..., None]


def sees(n, P, parent):
    """[n, P + n] whether new token i sees slot j."""
    m = torch.zeros((n, P + n), dtype=torch.bool)
    m[:, :P] = True
    for i in range(n):
        if parent is None:
            m[i, P:P + i + 1] = True
        else:
            j = i
            while j >= 0:
                m[i, P + j] = True
                j = int(parent[j])
    return m


def attention64(q, cache, b, P, n, parent=None, scale=None):
    """(o, lse, bound of o's error, bound of lse's) of request b, [n, H, D] and [H, n], in 64 bits.

    What the kernel may be off by: weights and results are rounded to bf16, half a step (2^-8 of the value) each; a score is an fp32 sum of
    D products (D 2^-24 of the sum of their magnitudes) and exp2, a division and sums over the keys add a few 2^-24 of the value each."""
    H, D = q.shape[-2:]
    k, v = (cache.rows64(b, range(P + n), w) for w in (0, 1))
    group = H // cache.heads
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    hidden = ~sees(n, P, None if parent is None else parent[b].tolist()).to(q.device)
    o, lse, o_tol, lse_tol = [], [], [], []
    for h in range(H):
        kh, vh, qh = k[:, h // group], v[:, h // group], q[b, :n, h].double()
        x = (qh @ kh.T * scale).masked_fill(hidden, -math.inf)
        w = torch.softmax(x, dim=1)
        mass = w @ torch.nan_to_num(vh.abs(), nan=0.0)
        size = (qh.abs() @ torch.nan_to_num(kh.abs(), nan=0.0).T * scale).masked_fill(hidden, 0.0).amax(1)
        off = (D + 8) * 2.0 ** -24 * size + 2.0 ** -22 * x.masked_fill(hidden, 0.0).abs().amax(1) + (32 + (P + n) / 64) * 2.0 ** -24
        o.append(w @ vh)
        lse.append(torch.logsumexp(x, dim=1))
        o_tol.append(2.0 ** -8 * (mass + o[-1].abs()) + 2 * off[:, None] * mass)
        lse_tol.append(off + 2.0 ** -22 * lse[-1].abs())
    return torch.stack(o, 1), torch.stack(lse), torch.stack(o_tol, 1), torch.stack(lse_tol)


def check_attention(sv, q, cache, prefix, new, *, parent=None, softmax_scale=0.0, workspace=None, num_splits=0, stream=None, call=None):
    """Runs the call on `cache` and holds its rows to the reference and every other row to what it held before."""
    B, N, H, D = q.shape
    out = torch.full_like(q, 7.0)
    lse = torch.full((B, H, N), 7.0, dtype=torch.float32, device=q.device)
    err = torch.zeros(1, dtype=torch.int32, device=q.device)
    kw = dict(num_new=i32(new), parent=parent, block_table=cache.table, scales=cache.scales, out=out, lse=lse, workspace=workspace,
              err_flag=err, softmax_scale=softmax_scale, num_splits=num_splits, stream=stream)
    (call or sv.specvlm_chunk_attn)(q, cache.k, cache.v, i32(prefix), **kw)
    torch.cuda.synchronize()
    assert int(err) == 0
    for b, (P, n) in enumerate(zip(prefix, new)):
        assert bool((out[b, n:] == 7.0).all()) and bool((lse[b, :, n:] == 7.0).all()), f"request {b}: rows past its tokens were written"
        if not n:
            continue
        o, l, o_tol, l_tol = attention64(q, cache, b, P, n, parent, softmax_scale or None)
        worst = ((out[b, :n].double() - o).abs() / o_tol).max()
        assert bool(torch.isfinite(out[b, :n]).all()) and worst <= 1, f"request {b}: off by {float(worst):.3g} of its bound"
        worst = ((lse[b, :, :n].double() - l).abs() / l_tol).max()
        assert worst <= 1, f"request {b}: lse off by {float(worst):.3g} of its bound"
    return out, lse


def random_tree(g, nodes, device="cuda"):
    at = torch.arange(nodes, device=device)
    back = 1 + (torch.rand(nodes, generator=g, device=device) ** 2 * 10).long()
    return torch.where(at == 0, -1, (at - back).clamp(min=0)).to(torch.int32)
