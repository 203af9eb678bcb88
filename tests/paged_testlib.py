"""Shared helpers of the paged cache's GPU tests: caches with everything around the tokens poisoned, and the operators'
definitions in 64 bits with bounds for what the kernels may round.

Bounds.  h = half a step of the 16-bit type (bf16 2^-8, fp16 2^-11).  A score is a sum of d products in fp32 (in any
order, the tensor cores' included): off by at most (d + 4) 2^-24 sum_c |q_c k_c| * scale, and 2^-20 for the exponential and
the scaling of arguments up to 16 (2^-24 of the argument each); call that delta, relative on a weight.  A weight is rounded to
16 bits before its product with v: h.  So an output is off by at most (h + 2 delta) * sum_j p_j |v_j| (2: numerator and
denominator) and by its own rounding, h |out|; in fp16 a weight may also fall below the smallest normal number, 2^-25 per
key against a maximum that is at least 1."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}


class World:
    """Sequences with `news` new tokens and `lens` tokens, on pages whose every other slot holds NaN."""

    def __init__(self, paged, news, lens, heads=4, kv_heads=2, d=64, dtype="bf16", page=16, order="head", layout="head", pad=0,
                 seed=0, spare_pages=3, extra_width=1, weights=True):
        self.paged, self.news, self.lens_list = paged, news, lens
        self.H, self.K, self.d, self.P, self.dt = heads, kv_heads, d, page, DTYPE[dtype]
        self.layout, self.n, self.rows = layout, sum(news), sum(news) + pad
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        B = len(news)
        want = [-(-l // page) for l in lens]
        n_pages = sum(want) + spare_pages
        perm = torch.randperm(n_pages, device="cuda", generator=self.gen).to(torch.int32)
        self.table = torch.full((B, max(want + [0]) + extra_width), 2 ** 30, dtype=torch.int32, device="cuda")   # (no page: never looked at)
        at = 0
        for b, m in enumerate(want):
            self.table[b, :m] = perm[at:at + m]
            at += m
        self.spare = perm[at:]
        shape = (n_pages, kv_heads, page, d) if order == "head" else (n_pages, page, kv_heads, d)
        self.k_pages, self.v_pages = (torch.full(shape, math.nan, device="cuda", dtype=self.dt) for _ in range(2))
        if order == "slot":
            self.k_pages, self.v_pages = self.k_pages.transpose(1, 2), self.v_pages.transpose(1, 2)
        self.weights = torch.full((n_pages, kv_heads, page), math.nan, device="cuda") if weights else None
        self.k, self.v = [], []                     # [kv_heads][len][d] per sequence
        for b, l in enumerate(lens):
            self.k.append(self.rand(kv_heads, l, d, gain=2.0))
            self.v.append(self.rand(kv_heads, l, d))
            self.put(b, 0, l)
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        starts = [sum(news[:b]) for b in range(B + 1)]
        self.starts = starts
        self.q_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.q = self.tokens(heads)
        self.p = paged.PagedParams(heads, kv_heads, d, page, n_pages, B, dtype)
        self.cache = paged.PagedCache(self.p, self.k_pages, self.v_pages, self.weights)
        self.batch = paged.PagedBatch(self.q_start, self.lens, self.table, self.rows, max(news + [0]))
        self.scale = d ** -0.5

    def rand(self, *shape, gain=1.0):
        return (torch.randn(shape, device="cuda", generator=self.gen) * gain).to(self.dt)

    def tokens(self, heads):
        """Token rows; those of nobody hold NaN."""
        x = self.rand(heads, self.rows, self.d) if self.layout == "head" else self.rand(self.rows, heads, self.d).transpose(0, 1)
        x[:, self.n:] = math.nan
        return x

    def pages_of(self, slots, b, table=None):
        return (self.table if table is None else table)[b, slots // self.P].long(), slots % self.P

    def put(self, b, lo, hi):
        if hi > lo:
            slots = torch.arange(lo, hi, device="cuda")
            page, place = self.pages_of(slots, b)
            self.k_pages[page, :, place] = self.k[b][:, lo:hi].transpose(0, 1)
            self.v_pages[page, :, place] = self.v[b][:, lo:hi].transpose(0, 1)
            if self.weights is not None:
                self.weights[page, :, place] = torch.rand(hi - lo, self.K, device="cuda", generator=self.gen)

    def get(self, pages, b, l, table=None):
        """[kv_heads][l](...) of a pool."""
        page, place = self.pages_of(torch.arange(l, device="cuda"), b, table)
        return pages[page, :, place].transpose(0, 1)

    def scores(self, b, full):
        """Scaled scores in 64 bits [H][new][len] (hidden: -inf), and the bound delta."""
        m, l = self.news[b], self.lens_list[b]
        q = self.q[:, self.starts[b]:self.starts[b] + m].double()
        k = self.k[b].double().repeat_interleave(self.H // self.K, 0)
        s = q @ k.transpose(1, 2) * self.scale
        size = q.abs() @ k.abs().transpose(1, 2) * self.scale
        delta = (self.d + 4) * 2.0 ** -24 * size.amax().item() + 2.0 ** -20 if s.numel() else 0.0
        if not full:
            i = torch.arange(m, device="cuda")[:, None]
            s = s.masked_fill(torch.arange(l, device="cuda") > i + (l - m), -math.inf)
        return s, delta

    def check_attention(self, out, lse, full, before_out, before_lse, tag=""):
        h = HALF[self.dt]
        for b, (m, l) in enumerate(zip(self.news, self.lens_list)):
            if m == 0:
                continue
            rows = slice(self.starts[b], self.starts[b] + m)
            s, delta = self.scores(b, full)
            v = self.v[b].double().repeat_interleave(self.H // self.K, 0)
            empty = torch.isneginf(s).all(-1) if l else torch.ones(self.H, m, dtype=torch.bool, device="cuda")
            p = torch.softmax(s, -1).nan_to_num(0.0) if l else s
            ref = p @ v
            room = h * ref.abs() + (h + 2 * delta) * (p @ v.abs()) + 2.0 ** -30
            if self.dt == torch.float16 and l:
                room += l * 2.0 ** -25 * v.abs().amax() + 2.0 ** -25        # (and outputs below the smallest normal number)
            got = out[:, rows].double()
            assert torch.isfinite(got).all(), f"{tag} sequence {b}: not finite"
            over = (got - ref).abs() - room
            assert over.amax() <= 0, f"{tag} sequence {b}: {(got - ref).abs().amax():.3e} off, {over.amax():.3e} over"
            if lse is not None:
                want = torch.logsumexp(s, -1) if l else torch.full((self.H, m), -math.inf, device="cuda", dtype=torch.float64)
                got = lse[:, rows].double()
                assert torch.equal(torch.isneginf(got), empty), f"{tag} sequence {b}: rows without a token"
                off = (got - want).masked_fill(empty, 0.0).abs() - (delta + 2.0 ** -20 + want.masked_fill(empty, 0.0).abs() * 2.0 ** -22)
                assert off.amax() <= 0, f"{tag} sequence {b}: lse {off.amax():.3e} over"
        # nobody's rows stay as they were
        assert torch.equal(out[:, self.n:].view(torch.int16), before_out[:, self.n:].view(torch.int16)), f"{tag}: rows behind the last sequence"
        if lse is not None:
            assert torch.equal(lse[:, self.n:], before_lse[:, self.n:]), f"{tag}: lse behind the last sequence"

    def attend(self, full=False, impl=0, batch=None, with_lse=True):
        out = torch.full_like(self.q, 7.0)
        lse = torch.full((self.H, self.rows), 7.0, device="cuda") if with_lse else None
        before = out.clone(), None if lse is None else lse.clone()
        self.cache.attn_paged_causal(batch or self.batch, self.q, out=out, lse=lse, mask=int(full), impl=impl)
        return out, lse, before

    def weight_sums(self, b, full, lse):
        """What every token got [kv_heads][len] in 64 bits, and the bound on it.  An argument of the exponential, up to 64
        here, is rounded where the score is scaled and where lse is, and lse itself was: 3 * 2^-24 * 64 * log2(e), below 2^-16."""
        m = self.news[b]
        s, delta = self.scores(b, full)
        p = torch.exp(s - lse[:, self.starts[b]:self.starts[b] + m].double()[..., None])
        p = torch.where(torch.isneginf(s), 0.0, p)
        got = p.unflatten(0, (self.K, self.H // self.K)).sum((1, 2))
        return got, (delta + 2.0 ** -16) * got + 2.0 ** -100


def lse_of(world, full):
    """The 64-bit lse, rounded to 32, as the input of the weights' tests; NaN in nobody's rows."""
    lse = torch.full((world.H, world.rows), math.nan, device="cuda")
    for b, m in enumerate(world.news):
        if m:
            s, _ = world.scores(b, full)
            lse[:, world.starts[b]:world.starts[b] + m] = torch.logsumexp(s, -1).float() if world.lens_list[b] else -math.inf
    return lse


def turned(x, positions, rot, axes=1, interleaved=False, base=10000.0, factor=1.0, original=0, fast=32.0, slow=1.0, magnitude=1.0,
           inverse=False):
    """[heads][n][d] turned, in 64 bits; and the bound of the products' rounding (sine and cosine off by 2^-22)."""
    x = x.double()
    out, room = x.clone(), torch.zeros_like(x)
    i = torch.arange(rot // 2, device=x.device, dtype=torch.float64)
    w = base ** (-2.0 * i / rot)
    if original:
        keep = ((original * w / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        w = keep * w + (1 - keep) * w / factor
    else:
        w = w / factor
    for a in range(axes):
        angle = positions[a].double()[:, None] * w * (-1.0 if inverse else 1.0)
        lo = a * rot
        first = slice(lo, lo + rot, 2) if interleaved else slice(lo, lo + rot // 2)
        second = slice(lo + 1, lo + rot, 2) if interleaved else slice(lo + rot // 2, lo + rot)
        c, s = magnitude * torch.cos(angle), magnitude * torch.sin(angle)
        out[..., first] = x[..., first] * c - x[..., second] * s
        out[..., second] = x[..., second] * c + x[..., first] * s
        room[..., first] = room[..., second] = magnitude * 2.0 ** -21 * (x[..., first].abs() + x[..., second].abs())
    return out, room
