"""The paged cache where its numbers are not finite, its tables name pages that do not exist, its caches are very long, and
with enough work for every ring and every cut of the kernels to go round more than once."""
import math

import pytest
import torch

from paged_testlib import DTYPE, HALF, World, lse_of, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def paged():
    assert torch.cuda.is_available()
    import paper_2601_01204_b200.paged as m
    return m


def bits(x):
    return x.contiguous().view(torch.int32 if x.dtype == torch.float32 else torch.int16)


# ---- weights: rows that are not finite, arguments outside the exponential's range --------------

ROWS = [dict(heads=4, kv_heads=2), dict(heads=2, kv_heads=2, d=128, dtype="fp16"), dict(heads=8, kv_heads=1, page=64)]


def weigh(w, lse, full, decay=0.0):
    w.weights.fill_(7.0)
    w.cache.kv_paged_weights(w.batch, w.q, lse, decay=decay, mask=int(full))
    assert w.cache.xkv_paged_poll_status() == 0
    return w.get(w.weights, 0, w.lens_list[0])


@pytest.mark.parametrize("m", ROWS, ids=str)
@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("what", ["query", "lse"])
def test_weights_carry_a_nan(paged, m, full, what):
    """A NaN row makes every slot that it sees NaN, whatever its place among the rows, and no other."""
    w = World(paged, news=[64], lens=[700], **m)
    lse, q, group = lse_of(w, full), w.q.clone(), w.H // w.K
    want, room = w.weight_sums(0, full, lse)
    for place in range(16):
        token, head = place // group, place % group
        w.q.copy_(q)
        bad = lse.clone()
        if what == "query":
            w.q[head, token, 5] = math.nan
        else:
            bad[head, token] = math.nan
        got = weigh(w, bad, full)
        seen = 700 if full else 700 - 64 + token + 1
        assert got[0, :seen].isnan().all(), place
        got = got.double()
        assert ((got[0, seen:] - want[0, seen:]).abs() <= room[0, seen:] + 2.0 ** -22 * want[0, seen:]).all(), place
        assert ((got[1:] - want[1:]).abs() <= room[1:] + 2.0 ** -22 * want[1:]).all(), place


@pytest.mark.parametrize("m", ROWS, ids=str)
@pytest.mark.parametrize("full", [False, True])
def test_weights_outside_the_range(paged, m, full):
    """Weights below 2^-149 are 0 and above 2^128 infinite in 32 bits; a row that saw nothing (lse -infinity) gives nothing."""
    w = World(paged, news=[64], lens=[700], **m)
    lse = lse_of(w, full)
    assert (weigh(w, lse + 150.0, full) == 0).all()             # exp(-150) < 2^-149 for the largest of them
    assert (weigh(w, torch.full_like(lse, -math.inf), full) == 0).all()
    assert (weigh(w, torch.full_like(lse, math.inf), full) == 0).all()
    s, _ = w.scores(0, full)
    low = s.masked_fill(torch.isneginf(s), math.inf).amin()     # every score that is seen has a weight above exp(100) > 2^128
    assert torch.isinf(weigh(w, torch.full_like(lse, low.item() - 100.0), full)).all()


# ---- weights: a cache whose length times the rows of a token passes 2^31 ------------------------

def test_weights_of_a_very_long_cache(paged):
    """34 304 000 tokens (all but the first page's are one page, again and again), 63 heads on one key head."""
    G, d, P, again = 63, 64, 256, 133999
    length = P * (again + 1)
    assert (length - 1) * G > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(4)
    kp, vp = (torch.randn(2, 1, P, d, device="cuda", generator=gen).bfloat16() for _ in range(2))
    weights = torch.zeros(2, 1, P, device="cuda")
    cache = paged.PagedCache(paged.PagedParams(G, 1, d, P, 2, 1), kp, vp, weights)
    table = torch.ones(1, again + 1, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    batch = paged.PagedBatch(torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                             torch.tensor([length], dtype=torch.int32, device="cuda"), table, 1, 1)
    q = torch.randn(G, 1, d, device="cuda", generator=gen).bfloat16()
    s = torch.einsum("gd,ptd->gpt", q[:, 0].double(), kp[:, 0].double()) * d ** -0.5
    lse = torch.log(torch.exp(s[:, 0]).sum(-1) + again * torch.exp(s[:, 1]).sum(-1))[:, None]
    cache.kv_paged_weights(batch, q, lse.float(), decay=0.0)
    assert cache.xkv_paged_poll_status() == 0
    want = torch.exp(s - lse[..., None]).sum(0)                 # (the second page's slots are written many times, with the same)
    size = torch.einsum("gd,ptd->gpt", q[:, 0].double().abs(), kp[:, 0].double().abs()).amax().item() * d ** -0.5
    delta = (d + 4) * 2.0 ** -24 * size + 2.0 ** -20
    assert ((weights[:, 0].double() - want).abs() <= (delta + 2.0 ** -16 + 2.0 ** -22) * want).all()


# ---- pages that do not exist read as zero --------------------------------------------------------

def without_page(w, b, at):
    """Entry `at` of sequence b's table names no page; the world's own copy of those tokens becomes zero."""
    w.table[b, at] = w.p.n_pages + 5
    lo, hi = at * w.P, min((at + 1) * w.P, w.lens_list[b])
    w.k[b][:, lo:hi] = 0
    w.v[b][:, lo:hi] = 0
    return lo, hi


@pytest.mark.parametrize("page", [16, 64])
def test_evict_from_a_page_that_is_not_there(paged, page):
    """Its tokens have weight 0, and those that are kept are zeros in the new pages."""
    l, keep, recent = 6 * page, 5 * page, 5
    first = 2 * page + page // 2                                # half of the missing page is protected
    w = World(paged, news=[0], lens=[l], page=page, spare_pages=8)
    x = torch.rand(l, w.K, device="cuda", generator=w.gen) + 0.5
    x[::2] *= -1
    at, place = w.pages_of(torch.arange(l, device="cuda"), 0)
    w.weights[at, :, place] = x
    k, v = w.k[0].clone(), w.v[0].clone()
    lo, hi = 2 * page, 3 * page
    w.table[0, 2] = w.p.n_pages
    k[:, lo:hi], v[:, lo:hi], x[lo:hi] = 0, 0, 0
    dst = w.spare[:5].reshape(1, 5).contiguous()
    kept, lens_out = w.cache.kv_paged_evict(w.batch, dst, keep, first, recent)
    assert w.cache.xkv_paged_poll_status() == -1 and lens_out.tolist() == [keep]
    for h in range(w.K):
        middle = sorted(range(first, l - recent), key=lambda j: (-x[j, h].item(), j))[:keep - first - recent]
        want = sorted(list(range(first)) + middle + list(range(l - recent, l)))
        assert any(lo <= j < hi for j in middle) and not all(j in middle for j in range(first, l - recent) if x[j, h] < 0)
        assert kept[0, h].tolist() == want
        idx = torch.tensor(want, device="cuda")
        for pool, old in ((w.k_pages, k), (w.v_pages, v)):
            assert torch.equal(bits(w.get(pool, 0, keep, dst)[h]), bits(old[h][idx]))
        assert torch.equal(w.get(w.weights, 0, keep, dst)[h], x[:, h][idx])


# ---- attention: rows that see nothing, values that a row does not see ----------------------------

@pytest.mark.parametrize("m", [
    dict(news=[6], lens=[2], heads=2, kv_heads=2), dict(news=[3, 2], lens=[1, 40], heads=4, kv_heads=1, d=128, dtype="fp16"),
    dict(news=[150], lens=[100], heads=5, kv_heads=1), dict(news=[200, 40], lens=[199, 20], heads=2, kv_heads=2, d=128),
    dict(news=[700, 300], lens=[500, 200], heads=16, kv_heads=16, dtype="fp16")], ids=str)
@pytest.mark.parametrize("impl", [1, 0])
def test_rows_without_a_token_beside_values_that_are_not_finite(paged, m, impl):
    w = World(paged, **m)
    for b, l in enumerate(w.lens_list):
        w.v[b][:, :, ::2] = math.nan
        w.v[b][:, :, 1::2] = math.inf
        w.put(b, 0, l)
    out, lse, _ = w.attend(impl=impl)
    for b, (n, l) in enumerate(zip(w.news, w.lens_list)):
        rows = slice(w.starts[b], w.starts[b] + max(0, n - l))
        assert (out[:, rows] == 0).all() and torch.isneginf(lse[:, rows]).all()
    assert w.cache.xkv_paged_poll_status() == 0


UNSEEN = [
    # few rows
    dict(news=[4, 3], lens=[200, 37], heads=4, kv_heads=2), dict(news=[16], lens=[16], heads=2, kv_heads=2, d=128, dtype="fp16"),
    dict(news=[2, 1, 5], lens=[1030, 300, 5], heads=6, kv_heads=2, d=128, page=64), dict(news=[8, 7], lens=[2000, 1999], heads=2, kv_heads=1, dtype="fp16"),
    # chunks: all of them cut between blocks, some, and sequences that see less than their new tokens
    dict(news=[300], lens=[700], heads=4, kv_heads=2), dict(news=[130, 40], lens=[2000, 40], heads=4, kv_heads=1, d=128, page=64, dtype="fp16"),
    dict(news=[700, 1, 300], lens=[700, 500, 1500], heads=16, kv_heads=16, pad=3), dict(news=[257, 140], lens=[900, 140], heads=16, kv_heads=8, d=128),
    dict(news=[150], lens=[100], heads=5, kv_heads=1, dtype="fp16"), dict(news=[20], lens=[9000], heads=64, kv_heads=1, page=256),
]


@pytest.mark.parametrize("m", UNSEEN, ids=str)
@pytest.mark.parametrize("impl", [1, 0])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_values_behind_a_token_never_reach_it(paged, m, impl, bad):
    """Some channels of a new token's value are not finite: those channels of it and of the tokens behind it are not finite,
    and nothing else differs from the definition."""
    w = World(paged, **m)
    clean, lse0, before = w.attend(impl=impl)
    w.check_attention(clean, lse0, False, *before)
    b = 0
    n, l = w.news[b], w.lens_list[b]
    v = w.v[b].clone()
    for token in sorted({max(0, n - l), n // 2, n - 1}):
        channels = torch.arange(w.d, device="cuda") % 7 == 3
        slot = l - n + token
        w.v[b][0, slot, channels] = bad
        w.v[b][w.K - 1, slot, 0] = bad
        w.put(b, slot, slot + 1)
        out, lse, _ = w.attend(impl=impl)
        reached = torch.zeros_like(out, dtype=torch.bool)
        group = w.H // w.K
        reached[:group, w.starts[b] + token:w.starts[b] + n] = channels
        reached[w.H - group:, w.starts[b] + token:w.starts[b] + n, 0] = True
        assert not torch.isfinite(out[reached]).any(), token
        w.v[b] = v.clone()
        w.put(b, slot, slot + 1)
        w.check_attention(torch.where(reached, clean, out), lse, False, *before, tag=f"token {token}")
        rest = slice(w.starts[b] + n, None)                     # (the other sequences to the bit)
        assert torch.equal(bits(out[:, rest]), bits(clean[:, rest])) and torch.equal(bits(lse), bits(lse0))
    again, _, _ = w.attend(impl=impl)
    assert torch.equal(bits(again), bits(clean))
    assert w.cache.xkv_paged_poll_status() == 0


@pytest.mark.parametrize("m", [dict(news=[5], lens=[50], heads=2, kv_heads=1), dict(news=[400], lens=[900], heads=8, kv_heads=4),
                               dict(news=[200], lens=[3000], heads=4, kv_heads=4, d=128, dtype="fp16", page=64)], ids=str)
def test_values_that_are_nan_throughout(paged, m):
    """From a token on every value is NaN: the tokens before it keep their results, the others are NaN in every channel."""
    w = World(paged, **m)
    clean, lse0, before = w.attend()
    n, l = w.news[0], w.lens_list[0]
    for token in (0, n // 3, n - 1):
        slots = slice(l - n + token, l)
        v = w.v[0].clone()
        w.v[0][:, slots] = math.nan
        w.put(0, l - n, l)
        out, lse, _ = w.attend()
        assert out[:, token:].isnan().all() and torch.equal(bits(lse), bits(lse0))
        w.v[0] = v
        w.put(0, l - n, l)
        out[:, token:] = clean[:, token:]
        w.check_attention(out, lse, False, *before, tag=f"token {token}")
    assert w.cache.xkv_paged_poll_status() == 0


# ---- rotary and append in blocks of two, four and eight tokens -------------------------------------

MANY = [dict(rot=64), dict(rot=64, interleaved=True), dict(rot=32, axes=2), dict(rot=6, axes=3), dict(rot=10, interleaved=True)]


@pytest.mark.parametrize("n", [600, 1300, 5000])
@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("m", MANY, ids=str)
def test_rotary_of_many_tokens(paged, m, n, layout):
    gen = torch.Generator(device="cuda").manual_seed(6)
    for d, heads, k_heads, dtype in ((64, 7, 2, "bf16"), (128, 5, 0, "fp16")):
        def make(h):
            x = torch.randn((h, n, d) if layout == "head" else (n, h, d), device="cuda", generator=gen).to(DTYPE[dtype])
            return x if layout == "head" else x.transpose(0, 1)
        q, k = make(heads), make(k_heads) if k_heads else None
        pos = torch.randint(0, 100000, (m.get("axes", 1), n), device="cuda", generator=gen).to(torch.int32)
        outs = paged.xkv_rotary(paged.RotaryParams(m["rot"], m.get("axes", 1), m.get("interleaved", False)), pos, q, k)
        for x, got in zip((q, k), outs):
            if x is None:
                continue
            want, room = turned(x, pos, **m)
            assert ((got.double() - want).abs() <= HALF[DTYPE[dtype]] * want.abs() + room * 1.01 + (2.0 ** -25 if dtype == "fp16" else 0.0)).all()
            keep = m["rot"] * m.get("axes", 1)
            assert torch.equal(got[..., keep:], x[..., keep:])


@pytest.mark.parametrize("n", [600, 1300, 5000])
@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("m", MANY[:4], ids=str)
def test_append_of_many_tokens(paged, m, n, layout):
    news = [n // 3, 0, n - n // 3 - 40, 1, 39]
    w = World(paged, news=news, lens=[x + 37 * i for i, x in enumerate(news)], heads=6, kv_heads=3, page=32, order="slot" if layout == "token" else "head",
              layout=layout, pad=11)
    k, v = w.tokens(w.K), w.tokens(w.K)
    pos = torch.randint(0, 100000, (m.get("axes", 1), w.rows), device="cuda", generator=w.gen).to(torch.int32)
    pools = [x.clone() for x in (w.k_pages, w.v_pages, w.weights)]
    q_out = torch.full_like(w.q, 7.0)
    w.cache.kv_paged_append(w.batch, k, v, q=w.q, q_out=q_out, positions=pos,
                            rotary=paged.RotaryParams(m["rot"], m.get("axes", 1), m.get("interleaved", False)))
    h = HALF[w.dt]
    want_k, room_k = turned(k, pos, **m)
    want_q, room_q = turned(w.q, pos, **m)
    ours = slice(0, w.n)
    assert ((q_out[:, ours].double() - want_q[:, ours]).abs() <= h * want_q[:, ours].abs() + room_q[:, ours] * 1.01).all()
    assert (q_out[:, w.n:] == 7.0).all()
    written = torch.zeros_like(w.weights, dtype=torch.bool)
    for b, (c, l) in enumerate(zip(w.news, w.lens_list)):
        if not c:
            continue
        rows = slice(w.starts[b], w.starts[b] + c)
        page, place = w.pages_of(torch.arange(l - c, l, device="cuda"), b)
        written[page, :, place] = True
        got = w.k_pages[page, :, place].transpose(0, 1).double()
        assert ((got - want_k[:, rows]).abs() <= h * want_k[:, rows].abs() + room_k[:, rows] * 1.01).all()
        assert torch.equal(w.v_pages[page, :, place].transpose(0, 1), v[:, rows])
        assert (w.weights[page, :, place] == 0).all()
    for now, before in zip((w.k_pages, w.v_pages, w.weights), pools):
        assert ((now == before) | (now.isnan() & before.isnan()))[~written].all()
    assert w.cache.xkv_paged_poll_status() == 0


@pytest.mark.parametrize("start", [1, 2])
def test_append_beside_a_sequence_out_of_bounds(paged, start):
    """A row number beyond the tensors in the middle of q_start: both sequences that it bounds are left out, no other."""
    w = World(paged, news=[2, 30, 9, 1, 5], lens=[50, 90, 20, 7, 64], pad=4)
    w.q_start[start] = 10 ** 6
    good = [b for b in range(5) if b not in (start - 1, start)]
    k, v = w.tokens(w.K), w.tokens(w.K)
    q_out = torch.full_like(w.q, 7.0)
    pools = w.k_pages.clone()
    w.cache.kv_paged_append(w.batch, k, v, q=w.q, q_out=q_out)
    assert w.cache.xkv_paged_poll_status() == -1
    written = torch.zeros(pools.shape[:3], dtype=torch.bool, device="cuda")
    for b in range(5):
        rows, n = slice(w.starts[b], w.starts[b] + w.news[b]), w.news[b]
        if b in good:
            assert torch.equal(w.get(w.k_pages, b, w.lens_list[b])[:, -n:], k[:, rows]), b
            assert torch.equal(w.get(w.v_pages, b, w.lens_list[b])[:, -n:], v[:, rows]), b
            assert torch.equal(q_out[:, rows], w.q[:, rows]), b
            page, place = w.pages_of(torch.arange(w.lens_list[b] - n, w.lens_list[b], device="cuda"), b)
            written[page, :, place] = True
        else:
            assert (q_out[:, rows] == 7.0).all(), b
    assert ((w.k_pages == pools) | (w.k_pages.isnan() & pools.isnan()))[~written].all()
    news = list(w.news)
    for b in range(5):
        w.k[b], w.v[b] = w.get(w.k_pages, b, w.lens_list[b]), w.get(w.v_pages, b, w.lens_list[b])
    for impl in (1, 0):
        w.news = news
        out, lse, before = w.attend(impl=impl)
        assert w.cache.xkv_paged_poll_status() == -1
        w.news = [n if b in good else 0 for b, n in enumerate(news)]
        w.check_attention(out, lse, False, *before, tag=f"impl {impl}")


# ---- pages that several sequences read --------------------------------------------------------------

def test_shared_pages(paged):
    """Two sequences with a common prefix on the same pages: attention in one call; weights through a handle each, with weights
    of their own, or through calls one after the other, which add up."""
    P, prefix, d = 16, 160, 64
    w = World(paged, news=[3, 2], lens=[prefix + 40, prefix + 25], page=P)
    w.table[1, :prefix // P] = w.table[0, :prefix // P]
    w.k[1][:, :prefix], w.v[1][:, :prefix] = w.k[0][:, :prefix], w.v[0][:, :prefix]
    out, lse, before = w.attend()
    w.check_attention(out, lse, False, *before)
    sums = [w.weight_sums(b, False, lse) for b in range(2)]
    one = [paged.PagedBatch(torch.tensor([w.starts[b], w.starts[b + 1]], dtype=torch.int32, device="cuda"), w.lens[b:b + 1].clone(),
                            w.table[b:b + 1].clone(), w.rows, 3) for b in range(2)]
    own = [torch.zeros_like(w.weights) for _ in range(2)]
    for b in range(2):
        paged.PagedCache(w.p, w.k_pages, w.v_pages, own[b]).kv_paged_weights(one[b], w.q, lse)
        got, room = w.get(own[b], b, w.lens_list[b]).double(), sums[b][1]
        assert ((got - sums[b][0]).abs() <= room + 2.0 ** -22 * sums[b][0]).all()
    w.weights.zero_()
    for b in range(2):
        w.cache.kv_paged_weights(one[b], w.q, lse)
    got = w.get(w.weights, 0, prefix).double()
    want, room = sums[0][0][:, :prefix] + sums[1][0][:, :prefix], sums[0][1][:, :prefix] + sums[1][1][:, :prefix]
    assert ((got - want).abs() <= room + 2.0 ** -22 * want).all()


@pytest.mark.parametrize("m", [dict(heads=4, kv_heads=2, news=[1] * 12), dict(heads=2, kv_heads=2, d=128, dtype="fp16", news=[140, 200, 1, 30, 7])], ids=str)
def test_weights_of_a_shared_prefix_add_up(paged, m):
    """Sequences that share their first pages, in one call without fading: a slot gets what all of them gave it."""
    prefix, B = 320, len(m["news"])
    w = World(paged, lens=[prefix + n + 9 * b for b, n in enumerate(m["news"])], **m)
    for b in range(1, B):
        w.table[b, :prefix // w.P] = w.table[0, :prefix // w.P]
        w.k[b][:, :prefix] = w.k[0][:, :prefix]
    lse = lse_of(w, False)
    sums = [w.weight_sums(b, False, lse) for b in range(B)]
    before = w.weights.clone()
    w.cache.kv_paged_weights(w.batch, w.q, lse)
    shared = sum(s[:, :prefix] for s, _ in sums), sum(r[:, :prefix] for _, r in sums)
    for b in range(B):
        got, old = w.get(w.weights, b, w.lens_list[b]).double(), w.get(before, b, w.lens_list[b]).double()
        want, room = (torch.cat([x, y[:, prefix:]], 1) for x, y in zip(shared, sums[b]))
        assert ((got - old - want).abs() <= room + (B + 3) * 2.0 ** -24 * (want + old)).all(), b       # (B + 3 roundings of the running sum)
    assert w.cache.xkv_paged_poll_status() == 0


# ---- enough work for the rings to go round ------------------------------------------------------------

def multiprocessors():
    return torch.cuda.get_device_properties(0).multi_processor_count


def units_per_block(w, full, rows):
    """Units of 128 tokens that a block has of the attention's line: an item is `rows` rows of a sequence and a key head."""
    toks, units, items = rows // (w.H // w.K), 0, 0
    for n, l in zip(w.news, w.lens_list):
        for lo in range(0, n, toks):
            seen = l if full else max(0, l - n + min(n, lo + toks))
            units += w.K * max(1, -(-seen // 128))
            items += w.K
    return units / multiprocessors(), items / multiprocessors()


CHUNKS = [dict(heads=16, kv_heads=16, page=64), dict(heads=16, kv_heads=16, d=128, dtype="fp16", page=128), dict(heads=32, kv_heads=8, d=128, page=32, order="slot"),
          dict(heads=24, kv_heads=8, dtype="fp16", page=256)]


def move(w, kind):
    """Keys and queries whose scaled scores rise along the cache, fall, or jump, up to 50."""
    scale = 50.0 / (w.d * w.scale)
    for b, l in enumerate(w.lens_list):
        x = torch.arange(l, device="cuda") / max(l, 1)
        if kind == "falling":
            x = 1 - x
        elif kind == "steps":
            x = ((x * 11).floor() % 4) / 4 + 0.25 * (torch.arange(l, device="cuda") % 97 == 50)
        w.k[b] = (w.k[b].float() * 0.05 + (x * scale)[None, :, None]).to(w.dt)
        w.put(b, 0, l)
    sign = torch.where(torch.arange(w.n, device="cuda") % 3 == 1, -1.0, 1.0)[None, :, None]
    head = torch.linspace(0.3, 1.0, w.H, device="cuda")[:, None, None]
    w.q[:, :w.n] = (sign * head + 0.02 * w.q[:, :w.n].float()).to(w.dt)


@pytest.mark.parametrize("m", CHUNKS, ids=str)
@pytest.mark.parametrize("kind", ["random", "rising", "falling", "steps"])
@pytest.mark.parametrize("full", [False, True])
def test_chunks_of_many_units(paged, m, kind, full):
    """Ten units of 128 tokens and more per block: the rings of K and V go round, and references move within a part."""
    w = World(paged, news=[300, 150, 1, 40], lens=[6000, 4500, 2000, 1000], pad=5, **m)
    units, items = units_per_block(w, full, 256)
    assert units >= 10 and items >= 0.4
    if kind != "random":
        move(w, kind)
    out, lse, before = w.attend(full)
    w.check_attention(out, lse, full, *before)
    again, _, _ = w.attend(full)
    assert torch.equal(bits(again), bits(out))
    assert w.cache.xkv_paged_poll_status() == 0


@pytest.mark.parametrize("m", [dict(heads=16, kv_heads=16, page=64), dict(heads=16, kv_heads=8, d=128, dtype="fp16", page=16, order="slot")], ids=str)
@pytest.mark.parametrize("full", [False, True])
def test_chunks_of_many_items(paged, m, full):
    """Parts of three items in most blocks: queries and accumulators are replaced."""
    news = [257, 300, 513, 129, 260, 400, 130, 700]
    w = World(paged, news=news, lens=[n + 300 * i for i, n in enumerate(news)], **m)
    units, items = units_per_block(w, full, 256)
    assert items >= 1.5 and units >= 10
    out, lse, before = w.attend(full)
    w.check_attention(out, lse, full, *before)
    assert w.cache.xkv_paged_poll_status() == 0


@pytest.mark.parametrize("m", [dict(heads=16, kv_heads=16, page=64), dict(heads=32, kv_heads=8, d=128, dtype="fp16", page=16, order="slot"),
                               dict(heads=16, kv_heads=8, d=128, page=256)], ids=str)
@pytest.mark.parametrize("kind", ["random", "rising", "falling", "steps"])
@pytest.mark.parametrize("n", [1, 2])
def test_few_rows_of_many_units(paged, m, kind, n):
    """At least eight units per block, so that items have their cost in the cut, and rings of stages that go round."""
    lens = [(1733 * i) % 6000 + n for i in range(30)] + [1, 9000]
    w = World(paged, news=[n] * len(lens), lens=[max(l, n) for l in lens], pad=2, **m)
    units, _ = units_per_block(w, False, 16)
    assert units >= 10
    if kind != "random":
        move(w, kind)
    out, lse, before = w.attend()
    w.check_attention(out, lse, False, *before)
    again, _, _ = w.attend()
    assert torch.equal(bits(again), bits(out))
    assert w.cache.xkv_paged_poll_status() == 0


@pytest.mark.parametrize("m", [dict(heads=16, kv_heads=16, page=64, news=[200, 130, 300]), dict(heads=16, kv_heads=16, d=128, dtype="fp16", page=16, news=[129, 260, 140]),
                               dict(heads=64, kv_heads=16, page=256, news=[70, 33, 100])], ids=str)
@pytest.mark.parametrize("full", [False, True])
def test_weights_of_many_items(paged, m, full):
    """More than sixteen items per block, of two and more query tiles each, so that the places where their halves meet are used
    again; and the same bits when the call is repeated."""
    w = World(paged, lens=[17000, 15000, 12000], **m)
    items = sum(-(-l // 256) for l in w.lens_list) * w.K / multiprocessors()
    assert items >= 17 and all(n * w.H // w.K > 128 for n in w.news)
    lse = lse_of(w, full)
    before = w.weights.clone()
    w.cache.kv_paged_weights(w.batch, w.q, lse, decay=0.5, mask=int(full))
    first = w.weights.clone()
    for b, l in enumerate(w.lens_list):
        got, old = w.get(w.weights, b, l).double(), 0.5 * w.get(before, b, l).double()
        want, room = w.weight_sums(b, full, lse)
        assert ((got - want - old).abs() <= room + 2.0 ** -22 * (want + old)).all(), b
    for _ in range(3):
        w.weights.copy_(before)
        w.cache.kv_paged_weights(w.batch, w.q, lse, decay=0.5, mask=int(full))
        assert torch.equal(bits(w.weights), bits(first))
    assert w.cache.xkv_paged_poll_status() == 0


# ---- a missing page, in attention and weights ---------------------------------------------------------

@pytest.mark.parametrize("m", [dict(news=[1, 1], lens=[200, 90]), dict(news=[3, 2], lens=[200, 90], d=128, dtype="fp16"),
                               dict(news=[100, 20], lens=[400, 90], page=32), dict(news=[140, 20], lens=[700, 90], d=128, page=128)], ids=str)
@pytest.mark.parametrize("full", [False, True])
def test_a_page_that_is_not_there_reads_as_zero(paged, m, full):
    w = World(paged, **m)
    lo, hi = without_page(w, 0, 1)
    for impl in (1, 0):
        out, lse, before = w.attend(full, impl=impl)
        assert w.cache.xkv_paged_poll_status() == -1
        w.check_attention(out, lse, full, *before, tag=f"impl {impl}")
    ref = lse_of(w, full)
    w.weights.fill_(7.0)
    w.cache.kv_paged_weights(w.batch, w.q, ref, decay=0.0, mask=int(full))
    assert w.cache.xkv_paged_poll_status() == -1
    slots = torch.cat([torch.arange(lo), torch.arange(hi, w.lens_list[0])]).cuda()
    page, place = w.pages_of(slots, 0)
    got = w.weights[page, :, place].T.double()
    want, room = (x[:, slots] for x in w.weight_sums(0, full, ref))
    assert ((got - want).abs() <= room + 2.0 ** -22 * want).all()


# ---- batches and caches whose attributes somebody tries to change ------------------------------------

def test_attributes_are_fixed(paged):
    w = World(paged, news=[3], lens=[20])
    out, lse, before = w.attend()
    for x, name in ((w.batch, "lens"), (w.batch, "q_start"), (w.batch, "table"), (w.cache, "k_pages"), (w.cache, "workspace"), (w.cache, "weights")):
        with pytest.raises(AttributeError, match=name):
            setattr(x, name, torch.zeros_like(getattr(x, name)))
    w.p.n_heads, w.cache.p.n_heads = 8, 2                      # (the handle's own numbers stay)
    with pytest.raises(Exception):
        w.cache.attn_paged_causal(w.batch, w.q[:2].contiguous())
    again, _, _ = w.attend()
    assert torch.equal(bits(again), bits(out))
    w.check_attention(again, lse, False, *before)


# ---- arguments that the other tests leave at their defaults ------------------------------------------

FORMS = [dict(news=[1, 1], lens=[700, 33], heads=8, kv_heads=2), dict(news=[3, 2], lens=[300, 40], heads=4, kv_heads=1, d=128, dtype="fp16"),
         dict(news=[150, 300], lens=[400, 900], heads=4, kv_heads=2), dict(news=[700, 40], lens=[1500, 40], heads=16, kv_heads=16, d=128, dtype="fp16", page=64),
         dict(news=[1, 20], lens=[50, 90], heads=64, kv_heads=64), dict(news=[9], lens=[300], heads=63, kv_heads=1, d=128)]


@pytest.mark.parametrize("m", FORMS, ids=str)
@pytest.mark.parametrize("full", [False, True])
def test_another_scale(paged, m, full):
    w = World(paged, **m)
    w.scale *= 2.5
    for impl in (1, 0):
        out = torch.full_like(w.q, 7.0)
        lse = torch.full((w.H, w.rows), 7.0, device="cuda")
        before = out.clone(), lse.clone()
        w.cache.attn_paged_causal(w.batch, w.q, out=out, lse=lse, scale=w.scale, mask=int(full), impl=impl)
        w.check_attention(out, lse, full, *before, tag=f"impl {impl}")
    ref = lse_of(w, full)
    w.cache.kv_paged_weights(w.batch, w.q, ref, scale=w.scale, decay=0.0, mask=int(full))
    for b, l in enumerate(w.lens_list):
        want, room = w.weight_sums(b, full, ref)
        assert ((w.get(w.weights, b, l).double() - want).abs() <= room + 2.0 ** -22 * want).all(), b
    assert w.cache.xkv_paged_poll_status() == 0


@pytest.mark.parametrize("m", FORMS, ids=str)
def test_output_in_place_of_the_queries(paged, m):
    w = World(paged, **m)
    for impl in (1, 0):
        for full in (False, True):
            out, lse, before = w.attend(full, impl)
            w.check_attention(out, lse, full, *before)
            x = w.q.clone()
            w.cache.attn_paged_causal(w.batch, x, out=x, mask=int(full), impl=impl)
            assert torch.equal(bits(x[:, :w.n]), bits(out[:, :w.n])) and torch.equal(bits(x[:, w.n:]), bits(w.q[:, w.n:]))


def test_batch_smaller_than_the_handle(paged):
    """A handle for 1024 sequences, calls of three of them, one after the other with other numbers."""
    w = World(paged, news=[200, 1, 40], lens=[300, 90, 40], heads=4, kv_heads=2)
    w.p.max_seqs = 1024
    cache = paged.PagedCache(w.p, w.k_pages, w.v_pages, w.weights)
    w.cache = cache
    for _ in range(2):
        out, lse, before = w.attend()
        w.check_attention(out, lse, False, *before)
        slot = w.lens_list[0] - 50
        v = w.v[0][:, slot].clone()
        w.v[0][:, slot] = math.nan
        w.put(0, slot, slot + 1)
        odd, _, _ = w.attend()
        assert odd[:, 150:200].isnan().all()
        w.v[0][:, slot] = v
        w.put(0, slot, slot + 1)
        odd[:, 150:200] = out[:, 150:200]
        w.check_attention(odd, lse, False, *before)
    assert cache.xkv_paged_poll_status() == 0
