"""The operators of the paged cache and the rotary positions, as cases that can be timed and compared.

  rotary   xkv_rotary: queries and keys of n tokens turned by their positions
  append   kv_paged_append: new tokens of several sequences, queries and keys turned, keys and values
           written to their pages
  attend   attn_paged_causal: the new tokens' queries over the cached tokens of their sequence
  weights  kv_paged_weights: what every cached token got of those queries' softmax weights
  evict    kv_paged_evict: the heaviest tokens of every sequence and key head, moved to other pages

seqs = sequences, new = new tokens of each, cached = tokens that it holds besides; with ragged != 0 the
lengths differ (ragged seeds them, new and cached are then the largest).  heads / kv_heads, d = channels of
a head, page = tokens of a page, pool = order of a page ("head": [heads][tokens][d], "slot":
[tokens][heads][d]), layout = order of the token tensors ("head": [heads][n][d], "token": [n][heads][d]),
pad = rows behind the last sequence that belong to nobody, causal = new tokens see their predecessors only
(else all tokens of the sequence, as within one frame).
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
OUTLIER_CHANNELS, OUTLIER_GAIN = 4, 4.0     # key channels with large magnitudes, per head


def _case(op, **more):
    c = dict(op=op, dtype="bf16", heads=32, kv_heads=8, d=128, seqs=1, new=1, cached=0, ragged=0, page=64, pool="head",
             layout="token", pad=0)
    if op in ("rotary", "append"):
        c.update(rot=c["d"], axes=1, interleaved=False, factor=1.0, trained=0, far=0)
    if op in ("attend", "weights"):
        c.update(causal=True)
    if op == "weights":
        c.update(decay=1.0)
    if op == "evict":
        c.update(keep=0, first=0, recent=0)
    c.update(more)
    return c


def listed():
    return [
        # queries and keys of one 518 x 518 frame, patches turned by their row and column
        _case("rotary", heads=16, kv_heads=16, d=64, new=1374, rot=32, axes=2, layout="head", name="rotary_frame"),
        # a long prompt far beyond the trained length, half of every head turned, frequencies scaled by bands
        _case("rotary", new=8192, rot=64, interleaved=True, factor=16.0, trained=8192, far=120000, dtype="fp16",
              name="rotary_long"),
        # one decoding step of a batch
        _case("append", seqs=64, cached=8191, ragged=3, page=16, pool="slot", name="append_tokens"),
        # prompts of several requests
        _case("append", seqs=4, new=2048, cached=2048, ragged=5, factor=4.0, pad=100, name="append_chunks"),
        # one token over a short cache of one 224 x 224 clip: latency counts
        _case("attend", heads=16, kv_heads=16, d=64, cached=1023, layout="head", name="attend_token"),
        # one decoding step of a batch of long and short requests
        _case("attend", seqs=64, cached=8191, ragged=3, page=16, pool="slot", name="attend_tokens"),
        # a 518 x 518 frame over a cache of 16384 tokens: a frame sees itself whole
        _case("attend", heads=16, kv_heads=16, d=64, new=1374, cached=15010, causal=False, layout="head", name="attend_frame"),
        # prompts that arrive in chunks
        _case("attend", seqs=4, new=2048, cached=14336, ragged=7, dtype="fp16", pad=60, name="attend_chunks"),
        # accumulated weights while decoding
        _case("weights", seqs=16, cached=8191, ragged=9, page=32, name="weights_tokens"),
        # accumulated weights of a frame, faded from frame to frame
        _case("weights", heads=16, kv_heads=16, d=64, new=1374, cached=15010, causal=False, decay=0.9, layout="head",
              name="weights_frame"),
        # a small cache back to its budget after a 224 x 224 frame
        _case("evict", heads=16, kv_heads=16, d=64, new=261, cached=1024, keep=1024, first=261, recent=261, name="evict_frame"),
        # requests cut to half of what they hold
        _case("evict", seqs=8, cached=16384, ragged=11, keep=8192, first=64, recent=1024, page=16, pool="slot",
              dtype="fp16", name="evict_batch"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, evenly over its logarithm."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["rotary", "append", "attend", "attend", "attend", "weights", "weights", "evict"])
    d = rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    group = rng.choice([1, 1, 2, 3, 4, 4, 6, 8]) if kv_heads < 16 else 1
    c = _case(op, heads=kv_heads * group, kv_heads=kv_heads, d=d, dtype=rng.choice(["bf16", "bf16", "fp16"]),
              page=rng.choice([16, 32, 64, 128, 256]), pool=rng.choice(["head", "slot"]),
              layout=rng.choice(["head", "token"]), seqs=_spread(rng, 1, 64), ragged=rng.randint(0, 1000),
              pad=rng.choice([0, 0, rng.randint(1, 64)]))
    if op in ("rotary", "append"):
        c["axes"] = rng.choice([1, 1, 1, 2])
        c["rot"] = rng.choice([d // c["axes"], d // c["axes"] // 2, d // c["axes"] // 4])
        c["interleaved"] = rng.random() < 0.5
        c["factor"] = rng.choice([1.0, 1.0, 4.0, 16.0])
        c["trained"] = rng.choice([0, 4096, 8192])
        c["far"] = rng.choice([0, 0, 100000])
    if op == "rotary":
        c.update(seqs=1, new=_spread(rng, 1, 8192), ragged=0, pad=0)
    elif op == "evict":
        c.update(new=rng.choice([1, 64, 261]), cached=_spread(rng, 64, 16384), seqs=_spread(rng, 1, 8))
        c["keep"] = max(8, int((c["cached"] + c["new"]) * rng.uniform(0.3, 1.0)))
        c["first"] = rng.randint(0, c["keep"] // 3)
        c["recent"] = rng.randint(0, c["keep"] // 3)
    elif rng.random() < 0.5:
        c.update(new=1, cached=_spread(rng, 1, 16384))
    else:
        c.update(new=_spread(rng, 2, 2048), cached=_spread(rng, 1, 16384), seqs=_spread(rng, 1, 8))
    if op in ("attend", "weights"):
        c["causal"] = rng.random() < 0.7
    if op == "weights":
        c["decay"] = rng.choice([0.0, 0.5, 0.9, 1.0])
    # no more work than the largest listed case of the operator
    most = max(_cost(x) for x in listed() if x["op"] == op)
    while _cost(c) > most:
        if c["seqs"] > 1:
            c["seqs"] = c["seqs"] * 3 // 4
        elif c["new"] > 64 and op != "evict":
            c["new"] = c["new"] * 3 // 4
        else:
            c["cached"] = c["cached"] * 3 // 4
    return c


def _lengths(case):
    """(new tokens, cached tokens with them) of every sequence."""
    if not case["ragged"]:
        return [case["new"]] * case["seqs"], [case["cached"] + case["new"]] * case["seqs"]
    r = random.Random(case["ragged"])
    news, lens = [], []
    for b in range(case["seqs"]):
        new = case["new"] if b == 0 else _spread(r, max(1, case["new"] // 64), case["new"])
        cached = 0 if case["cached"] == 0 else case["cached"] if b == 0 else _spread(r, max(1, case["cached"] // 32), case["cached"])
        news.append(new)
        lens.append(cached + new)
    return news, lens


def _seen(case):
    """Cached tokens that the new tokens see, added up over all new tokens."""
    news, lens = _lengths(case)
    return sum(n * l - (n * (n - 1) // 2 if case["causal"] else 0) for n, l in zip(news, lens))


def work(case):
    """Each tensor read and each written once, of the cache what the operator cannot do without."""
    news, lens = _lengths(case)
    n, H, K, d = sum(news), case["heads"], case["kv_heads"], case["d"]
    row = 2 * d
    turned = case.get("rot", 0) * case.get("axes", 0)
    if case["op"] == "rotary":
        return {"bytes": 2 * n * (H + K) * row + 4 * n * case["axes"], "flops": 3 * n * (H + K) * turned}
    if case["op"] == "append":
        return {"bytes": n * (2 * (H + 2 * K) * row + 4 * K + 4 * case["axes"]), "flops": 3 * n * (H + K) * turned}
    if case["op"] == "attend":
        return {"bytes": n * H * (2 * row + 4) + 2 * sum(lens) * K * row, "flops": 4 * _seen(case) * H * d}
    if case["op"] == "weights":
        return {"bytes": n * H * (row + 4) + sum(lens) * K * (row + 8), "flops": 2 * _seen(case) * H * d}
    kept = sum(min(l, case["keep"]) for l in lens)
    return {"bytes": K * (4 * sum(lens) + kept * (4 * row + 8)), "flops": 0}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 200)


def _rotary_values(case):
    """(base, factor, tokens of the trained length or 0 = factor for all alike, beta_fast, beta_slow, magnitude)."""
    magnitude = 0.1 * math.log(case["factor"]) + 1.0 if case["trained"] and case["factor"] > 1.0 else 1.0
    return 10000.0, case["factor"], case["trained"], 32.0, 1.0, magnitude


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, H, K, d, P = DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["d"], case["page"]
    news, lens = _lengths(case)
    n = sum(news)
    rows = n + case["pad"]

    def tokens(heads):
        x = torch.randn((heads, rows, d) if case["layout"] == "head" else (rows, heads, d), device="cuda", generator=gen)
        return x.to(dt) if case["layout"] == "head" else x.to(dt).transpose(0, 1)

    gain = torch.where(torch.rand(K, d, device="cuda", generator=gen).argsort(dim=-1) < OUTLIER_CHANNELS, OUTLIER_GAIN, 1.0)
    s = {"case": case, "q": tokens(H)}
    starts = [sum(news[:b]) for b in range(case["seqs"] + 1)]
    if case["op"] in ("rotary", "append"):
        s["k"] = (tokens(K).float() * gain[:, None]).to(dt)
        if case["layout"] == "token":
            s["k"] = s["k"].transpose(0, 1).contiguous().transpose(0, 1)
        s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
        if case["axes"] > 1:     # rows and columns of patches
            pos = torch.randint(0, 37, (case["axes"], rows), device="cuda", generator=gen)
        else:
            first = [l - m + case["far"] for m, l in zip(news, lens)]
            pos = torch.cat([torch.arange(f, f + m) for f, m in zip(first, news)] + [torch.zeros(case["pad"], dtype=torch.int64)])
            pos = pos[None].cuda()
        s["positions"] = pos.to(torch.int32)
    if case["op"] == "rotary":
        if own:
            import paper_2601_01204_b200.paged as paged
            s["rotary"], s["turn"] = _own_rotary(case), paged.xkv_rotary
        return s

    # the pages: every sequence has its own, in no order; those of the eviction's targets behind them
    want = [-(-l // P) for l in lens]
    kept = [-(-min(l, case["keep"]) // P) if case["op"] == "evict" else 0 for l in lens]
    n_pages = sum(want) + sum(kept) + 1
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    s["table"], s["dst"] = (torch.full((case["seqs"], max(max(w), 1)), -1, dtype=torch.int32, device="cuda") for w in (want, kept))
    at = 0
    for table, counts in ((s["table"], want), (s["dst"], kept)):
        for b, m in enumerate(counts):
            table[b, :m] = order[at:at + m]
            at += m
    shape = (n_pages, K, P, d) if case["pool"] == "head" else (n_pages, P, K, d)

    def pool(scaled):
        x = torch.randn(shape, device="cuda", dtype=dt, generator=gen)
        if scaled:
            x *= (gain[:, None] if case["pool"] == "head" else gain).to(dt)
        return x if case["pool"] == "head" else x.transpose(1, 2)

    s["k_pages"], s["v_pages"] = pool(True), pool(False)
    # what attention has left so far: most tokens got little, a few much
    s["weights"] = torch.rand(n_pages, K, P, device="cuda", generator=gen).pow_(8) * 10.0
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    # row r of the token tensors is token `index` of sequence `seq`
    s["seq"] = torch.repeat_interleave(torch.arange(case["seqs"]), torch.tensor(news)).cuda()
    s["index"] = torch.arange(n, device="cuda") - s["q_start"].long()[s["seq"]]
    s["n"], s["max_new"], s["max_len"] = n, max(news), max(lens)
    if case["op"] == "append":
        s["v"] = tokens(K)
    if case["op"] in ("attend", "weights"):
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(H, rows, device="cuda")
    if case["op"] == "weights":
        _plain_attend(s)         # fills s["lse"]
        s.pop("out")
    if case["op"] == "evict":
        s["kept"] = torch.zeros(case["seqs"], K, case["keep"], dtype=torch.int32, device="cuda")
        s["lens_out"] = torch.zeros(case["seqs"], dtype=torch.int32, device="cuda")
    if own:
        import paper_2601_01204_b200.paged as paged
        p = paged.PagedParams(n_heads=H, n_kv_heads=K, head_dim=d, page_tokens=P, n_pages=n_pages, max_seqs=case["seqs"],
                            dtype=case["dtype"])
        s["cache"] = paged.PagedCache(p, s["k_pages"], s["v_pages"], s["weights"])
        s["batch"] = paged.PagedBatch(s["q_start"], s["lens"], s["table"], n_tokens=rows, max_new=s["max_new"])
        s["mask"] = paged.MASK_CAUSAL if case.get("causal", True) else paged.MASK_FULL
        s["rotary"] = _own_rotary(case) if case["op"] == "append" else None
    return s


def run(s):
    return (_own_run if own else _plain_run)(s)


# ---- the framework's calls ----------------------------------------------------------------------

def _own_rotary(case):
    import paper_2601_01204_b200.paged as paged
    base, factor, trained, fast, slow, magnitude = _rotary_values(case)
    return paged.RotaryParams(rotary_dim=case["rot"], n_axes=case["axes"], interleaved=case["interleaved"], base=base, factor=factor,
                            original_tokens=trained, beta_fast=fast, beta_slow=slow, magnitude=magnitude)


def _own_run(s):
    case = s["case"]
    op = case["op"]
    if op == "rotary":
        s["turn"](s["rotary"], s["positions"], s["q"], s["k"], q_out=s["q_out"], k_out=s["k_out"])
        return s["q_out"], s["k_out"]
    if op == "append":
        s["cache"].kv_paged_append(s["batch"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rotary=s["rotary"], positions=s["positions"])
        return s["q_out"], s["k_pages"], s["v_pages"], s["weights"]
    if op == "attend":
        s["cache"].attn_paged_causal(s["batch"], s["q"], out=s["out"], lse=s["lse"], mask=s["mask"])
        return s["out"], s["lse"]
    if op == "weights":
        s["cache"].kv_paged_weights(s["batch"], s["q"], s["lse"], decay=case["decay"], mask=s["mask"])
        return s["weights"]
    s["cache"].kv_paged_evict(s["batch"], s["dst"], keep=case["keep"], n_first=case["first"], n_recent=case["recent"],
                              kept=s["kept"], lens_out=s["lens_out"])
    return s["kept"], s["lens_out"], s["k_pages"], s["v_pages"], s["weights"]


# ---- the plain form -----------------------------------------------------------------------------

def _plain_rotary(case, positions, x):
    """x: [heads][n][d].  Angles in 64 bits, products in 32."""
    base, factor, trained, fast, slow, magnitude = _rotary_values(case)
    r = case["rot"]
    w = base ** (torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / -r)
    if trained:
        keep = ((trained * w / (2 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
        w = w * keep + w / factor * (1.0 - keep)
    else:
        w = w / factor
    angle = positions.double()[:, :, None] * w                      # [axes][n][r / 2]
    cos, sin = ((f(angle) * magnitude).float().transpose(0, 1) for f in (torch.cos, torch.sin))
    t = x[..., :case["axes"] * r].float().unflatten(-1, (case["axes"], 2, r // 2) if not case["interleaved"] else (case["axes"], r // 2, 2))
    a, b = t.unbind(-1 if case["interleaved"] else -2)
    turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1 if case["interleaved"] else -2).flatten(-3)
    return torch.cat([turned.to(x.dtype), x[..., case["axes"] * r:]], dim=-1)


def _plain_cached(s, pages):
    """[sequences][kv_heads][longest][d] of a pool, in 32 bits."""
    return pages[s["table"].clamp(min=0).long()].transpose(1, 2).flatten(2, 3)[:, :, :s["max_len"]].float()


def _plain_scores(s):
    """Scaled scores [sequences][kv_heads][group][new][longest], and which of them are seen [sequences][1][1][new][longest]."""
    case = s["case"]
    H, K, d = case["heads"], case["kv_heads"], case["d"]
    q = torch.zeros(case["seqs"], s["max_new"], H, d, device="cuda")
    q[s["seq"], s["index"]] = s["q"][:, :s["n"]].transpose(0, 1).float()
    q = q.transpose(1, 2).reshape(case["seqs"], K, H // K * s["max_new"], d)
    scores = (q @ _plain_cached(s, s["k_pages"]).transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).unflatten(2, (H // K, s["max_new"]))
    new = s["q_start"][1:] - s["q_start"][:-1]
    token = torch.arange(s["max_new"], device="cuda")
    limit = s["lens"][:, None].expand(-1, s["max_new"])
    if case["causal"]:
        limit = limit - new[:, None] + token + 1
    seen = (torch.arange(s["max_len"], device="cuda") < limit[..., None]) & (token < new[:, None])[..., None]
    return scores, seen[:, None, None]


def _plain_attend(s):
    scores, seen = _plain_scores(s)
    scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = _plain_cached(s, s["v_pages"])
    out = (p.flatten(2, 3) @ v).unflatten(2, p.shape[2:4]) / torch.where(total == 0, 1.0, total)
    lse = (torch.log(total) + top).squeeze(-1)
    s["out"][:, :s["n"]] = out.flatten(1, 2)[s["seq"], :, s["index"]].transpose(0, 1).to(s["out"].dtype)
    s["lse"][:, :s["n"]] = lse.flatten(1, 2)[s["seq"], :, s["index"]].transpose(0, 1)
    return s["out"], s["lse"]


def _plain_slots(s):
    """(sequence, slot, page, place on the page) of every cached token."""
    b, slot = torch.nonzero(torch.arange(s["max_len"], device="cuda") < s["lens"][:, None], as_tuple=True)
    P = s["case"]["page"]
    return b, slot, s["table"][b, slot // P].long(), slot % P


def _plain_run(s):
    case = s["case"]
    op, P = case["op"], case["page"]
    if op == "rotary":
        s["q_out"].copy_(_plain_rotary(case, s["positions"], s["q"]))
        s["k_out"].copy_(_plain_rotary(case, s["positions"], s["k"]))
        return s["q_out"], s["k_out"]
    if op == "append":
        n = s["n"]
        s["q_out"][:, :n] = _plain_rotary(case, s["positions"][:, :n], s["q"][:, :n])
        k = _plain_rotary(case, s["positions"][:, :n], s["k"][:, :n])
        new = s["q_start"][1:] - s["q_start"][:-1]
        slot = (s["lens"] - new).long()[s["seq"]] + s["index"]
        page = s["table"][s["seq"], slot // P].long()
        s["k_pages"][page, :, slot % P] = k.transpose(0, 1)
        s["v_pages"][page, :, slot % P] = s["v"][:, :n].transpose(0, 1)
        s["weights"][page, :, slot % P] = 0.0
        return s["q_out"], s["k_pages"], s["v_pages"], s["weights"]
    if op == "attend":
        return _plain_attend(s)
    if op == "weights":
        scores, seen = _plain_scores(s)
        group = case["heads"] // case["kv_heads"]
        lse = torch.zeros(case["seqs"], s["max_new"], case["heads"], device="cuda")
        lse[s["seq"], s["index"]] = s["lse"][:, :s["n"]].T
        lse = lse.transpose(1, 2).reshape(case["seqs"], -1, group, s["max_new"], 1)
        got = scores.sub_(lse).exp_().masked_fill_(~seen, 0.0).sum((2, 3))
        b, slot, page, place = _plain_slots(s)
        s["weights"][page, :, place] = case["decay"] * s["weights"][page, :, place] + got[b, :, slot]
        return s["weights"]
    w = s["weights"][s["table"].clamp(min=0).long()].transpose(1, 2).flatten(2, 3)[:, :, :s["max_len"]]
    slot = torch.arange(s["max_len"], device="cuda")
    lens = s["lens"][:, None, None]
    fixed = (slot < case["first"]) | (slot >= lens - case["recent"]) | (lens <= case["keep"])
    w = torch.where(fixed, math.inf, w).masked_fill_(slot >= lens, -math.inf)
    take = min(case["keep"], s["max_len"])
    top = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :take].sort(-1).values
    s["lens_out"].copy_(s["lens"].clamp(max=case["keep"]))
    held = torch.arange(take, device="cuda") < s["lens_out"][:, None, None]
    s["kept"].fill_(-1)
    s["kept"][..., :take] = torch.where(held, top, -1)
    b, h, to = torch.nonzero(held.expand_as(top), as_tuple=True)
    src = top[b, h, to]
    here, there = (s["table"][b, src // P].long(), h, src % P), (s["dst"][b, to // P].long(), h, to % P)
    for pages in (s["k_pages"], s["v_pages"], s["weights"]):
        pages[there] = pages[here]
    return s["kept"], s["lens_out"], s["k_pages"], s["v_pages"], s["weights"]


# ---- the definition in 64 bits ------------------------------------------------------------------

def _exact_turned(case, positions, x):
    """Pairs as complex numbers, one axis after the other."""
    base, factor, trained, fast, slow, magnitude = _rotary_values(case)
    r, x = case["rot"], x.double().clone()
    for axis in range(case["axes"]):
        freq = []
        for i in range(r // 2):
            f = base ** (-2.0 * i / r)
            part = min(1.0, max(0.0, (trained * f / (2.0 * math.pi) - slow) / (fast - slow))) if trained else 0.0
            freq.append(part * f + (1.0 - part) * f / factor)
        turn = positions[axis].double()[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.full_like(turn, magnitude), turn)
        lo = axis * r
        even, odd = (slice(lo, lo + r, 2), slice(lo + 1, lo + r, 2)) if case["interleaved"] else \
            (slice(lo, lo + r // 2), slice(lo + r // 2, lo + r))
        z = torch.complex(x[..., even], x[..., odd]) * turn
        x[..., even], x[..., odd] = z.real, z.imag
    return x


def exact(case, seed):
    s = prepare(case, seed)
    news, lens = _lengths(case)
    op, P, d, K = case["op"], case["page"], case["d"], case["kv_heads"]
    if op == "rotary":
        return _exact_turned(case, s["positions"], s["q"]), _exact_turned(case, s["positions"], s["k"])
    starts = s["q_start"].tolist()
    pages = [[s["table"][b, j // P].item() for j in range(0, l, P)] for b, l in enumerate(lens)]
    if op == "append":
        q_out = s["q_out"].double()
        q_out[:, :s["n"]] = _exact_turned(case, s["positions"], s["q"])[:, :s["n"]]
        k = _exact_turned(case, s["positions"], s["k"])
        kp, vp, w = s["k_pages"].double(), s["v_pages"].double(), s["weights"].double()
        for b, (m, l) in enumerate(zip(news, lens)):
            for j in range(l - m, l):
                row = starts[b] + j - (l - m)
                kp[pages[b][j // P], :, j % P], vp[pages[b][j // P], :, j % P] = k[:, row], s["v"][:, row].double()
                w[pages[b][j // P], :, j % P] = 0.0
        return q_out, kp, vp, w
    if op == "evict":            # copies and whole numbers: nothing is computed
        return None
    group = case["heads"] // K
    out, lse, w = s["q"].double() * 0.0, s["lse"].double() * 0.0, s["weights"].double()
    for b, (m, l) in enumerate(zip(news, lens)):
        rows = slice(starts[b], starts[b] + m)
        last = torch.arange(m, device="cuda")[:, None] + (l - m) if case["causal"] else l - 1
        hidden = torch.arange(l, device="cuda") > last if case["causal"] else torch.zeros(m, l, dtype=torch.bool, device="cuda")
        for h in range(K):
            key, value = (torch.cat([x[p, h] for p in pages[b]])[:l].double() for x in (s["k_pages"], s["v_pages"]))
            total = torch.zeros(l, dtype=torch.float64, device="cuda")
            for g in range(h * group, (h + 1) * group):
                score = (s["q"][g, rows].double() @ key.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                if op == "attend":
                    out[g, rows], lse[g, rows] = torch.softmax(score, -1) @ value, torch.logsumexp(score, -1)
                else:
                    total += torch.exp(score - s["lse"][g, rows].double()[:, None]).sum(0)
            if op == "weights":
                slots = torch.arange(l, device="cuda")
                page = torch.tensor(pages[b], device="cuda")[slots // P]
                w[page, h, slots % P] = case["decay"] * w[page, h, slots % P] + total
    return (out, lse) if op == "attend" else w
