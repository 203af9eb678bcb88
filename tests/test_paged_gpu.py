"""The paged cache and the rotary positions against their definitions in 64 bits, at the sizes and masks where they can go wrong."""
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


# ---- rotary positions ------------------------------------------------------------------------

ROTARY = [
    dict(rot=64), dict(rot=64, interleaved=True), dict(rot=32), dict(rot=32, axes=2), dict(rot=16, axes=2, interleaved=True),
    dict(rot=6), dict(rot=6, axes=3), dict(rot=10, interleaved=True), dict(rot=2, axes=4), dict(rot=8), dict(rot=24),
    dict(rot=64, factor=8.0), dict(rot=64, factor=16.0, original=4096, magnitude=1.25), dict(rot=32, interleaved=True, factor=4.0, original=64, fast=4.0, slow=0.5),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("m", ROTARY, ids=str)
def test_rotary(paged, m, dtype):
    gen = torch.Generator(device="cuda").manual_seed(1)
    for d, heads, k_heads, n, layout in ((64, 3, 2, 5, "head"), (128, 4, 1, 37, "token"), (64, 16, 0, 1, "head")):
        def make(h):
            x = torch.randn((h, n, d) if layout == "head" else (n, h, d), device="cuda", generator=gen).to(DTYPE[dtype])
            return x if layout == "head" else x.transpose(0, 1)
        q, k = make(heads), make(k_heads) if k_heads else None
        pos = torch.randint(-1000, 2 ** 31 - 1, (m.get("axes", 1), n), device="cuda", generator=gen).to(torch.int32)
        r = paged.RotaryParams(m["rot"], m.get("axes", 1), m.get("interleaved", False), factor=m.get("factor", 1.0),
                               original_tokens=m.get("original", 0), beta_fast=m.get("fast", 32.0), beta_slow=m.get("slow", 1.0),
                               magnitude=m.get("magnitude", 1.0))
        for inverse in (False, True):
            outs = paged.xkv_rotary(r, pos, q, k, inverse=inverse)
            for x, got in zip((q, k), outs):
                if x is None:
                    assert got is None
                    continue
                want, room = turned(x, pos, **m, inverse=inverse)
                assert ((got.double() - want).abs() <= HALF[DTYPE[dtype]] * want.abs() + room * 1.01 + (2.0 ** -25 if dtype == "fp16" else 0.0)).all()
                keep = m["rot"] * m.get("axes", 1)
                assert torch.equal(got[..., keep:], x[..., keep:])
            a, b = q.clone(), None if k is None else k.clone()          # in place
            paged.xkv_rotary(r, pos, a, b, q_out=a, k_out=b, inverse=inverse)
            assert torch.equal(a, outs[0]) and (k is None or torch.equal(b, outs[1]))


def test_rotary_gradient(paged):
    """The gradient of sum(g * rotary(x)) is the inverse rotation of g: against differences of the definition."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    n, d, rot = 7, 64, 32
    x, g = (torch.randn(2, n, d, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
    pos = torch.randint(0, 5000, (2, n), device="cuda", generator=gen).to(torch.int32)
    got, _ = paged.xkv_rotary(paged.RotaryParams(rot, 2), pos, g, inverse=True)
    f = lambda y: (turned(y, pos, rot, 2)[0] * g.double()).sum()
    xd = x.double()
    for at in [(0, 0, 0), (1, 3, 17), (0, 6, 63), (1, 5, 40)]:
        e = torch.zeros_like(xd)
        e[at] = 0.5
        slope = (f(xd + e) - f(xd - e)).item()              # (f is linear: differences of any size are exact)
        assert abs(got[at].item() - slope) <= HALF[torch.bfloat16] * abs(slope) + 2.0 ** -20 * g.abs().max().item()


# ---- append ----------------------------------------------------------------------------------

APPENDS = [
    dict(news=[1], lens=[1]), dict(news=[1, 1, 1], lens=[5, 16, 17]), dict(news=[5, 0, 33, 1], lens=[5, 9, 40, 0], pad=3),
    dict(news=[70], lens=[100], page=64, order="slot", layout="token"), dict(news=[300, 20], lens=[300, 275], page=256, d=128, dtype="fp16"),
    dict(news=[0, 0], lens=[3, 0], pad=2), dict(news=[20], lens=[7]),
]


@pytest.mark.parametrize("m", APPENDS, ids=str)
@pytest.mark.parametrize("mode", ["plain", "turned", "q"])
def test_append(paged, m, mode):
    w = World(paged, **m)
    k, v = w.tokens(w.K), w.tokens(w.K)
    rot = paged.RotaryParams(32) if mode != "plain" else None
    pos = torch.arange(w.rows, device="cuda", dtype=torch.int32) * 1000
    pools = [x.clone() for x in (w.k_pages, w.v_pages, w.weights)]
    q_out = torch.full_like(w.q, 7.0) if mode == "q" else None
    w.cache.kv_paged_append(w.batch, k, v, q=w.q if mode == "q" else None, q_out=q_out, rotary=rot, positions=pos)
    h = HALF[w.dt]
    want_k, room = turned(k, pos[None], 32) if rot else (k.double(), torch.zeros_like(k, dtype=torch.float64))
    written = torch.zeros_like(w.weights, dtype=torch.bool)
    for b, (n, l) in enumerate(zip(w.news, w.lens_list)):
        for i in range(n):
            slot, row = l - n + i, w.starts[b] + i
            if slot < 0:
                continue
            page, place = int(w.table[b, slot // w.P]), slot % w.P
            written[page, :, place] = True
            got = w.k_pages[page, :, place].double()
            if rot:
                assert ((got - want_k[:, row]).abs() <= h * want_k[:, row].abs() + room[:, row] * 1.01 + 2.0 ** -25).all()
            else:
                assert torch.equal(got, want_k[:, row])
            assert torch.equal(w.v_pages[page, :, place], v[:, row])
            assert (w.weights[page, :, place] == 0).all()
    for now, before in zip((w.k_pages, w.v_pages, w.weights), pools):      # everything else as it was
        same = (now == before) | (now.isnan() & before.isnan())
        assert same[~written].all()
    if mode == "q":
        want, room = turned(w.q[:, :w.n], pos[None, :w.n], 32)
        assert ((q_out[:, :w.n].double() - want).abs() <= h * want.abs() + room * 1.01 + 2.0 ** -25).all()
        assert (q_out[:, w.n:] == 7.0).all()
    assert w.cache.xkv_paged_poll_status() == 0


# ---- attention -------------------------------------------------------------------------------

ATTENTION = [
    # single tokens: one key, edges of 16, 32, 64, 128 and 256 keys, many sequences, none at all
    dict(news=[1], lens=[1]), dict(news=[1] * 6, lens=[1, 15, 16, 17, 33, 64]), dict(news=[1, 1, 0, 1], lens=[129, 0, 50, 127], pad=2),
    dict(news=[1, 1], lens=[1000, 257], heads=8, kv_heads=1, d=128), dict(news=[1] * 3, lens=[300, 5, 2049], heads=16, kv_heads=16, page=64),
    dict(news=[1, 1], lens=[4000, 130], heads=6, kv_heads=2, d=128, dtype="fp16", page=32, order="slot", layout="token"),
    dict(news=[1] * 40, lens=[37 * i % 500 + 1 for i in range(40)], heads=4, kv_heads=1, page=128),
    dict(news=[1], lens=[20000], heads=2, kv_heads=1, d=128, page=256),
    # a few tokens: rows of a group at the edges of 16
    dict(news=[2, 3, 4], lens=[2, 100, 37], heads=8, kv_heads=2), dict(news=[4, 5], lens=[200, 260], heads=8, kv_heads=2),
    dict(news=[16, 17], lens=[16, 300], heads=2, kv_heads=2, dtype="fp16"), dict(news=[3], lens=[2]),
    # chunks: edges of 128 rows, groups that do not divide 128, more new tokens than tokens, one sequence of each kind
    dict(news=[128], lens=[128], heads=2, kv_heads=2), dict(news=[127, 129], lens=[500, 129], heads=2, kv_heads=1),
    dict(news=[257], lens=[300], heads=1, kv_heads=1, d=128), dict(news=[300, 1, 0, 77], lens=[700, 333, 12, 77], heads=12, kv_heads=4, d=128, page=32),
    dict(news=[90, 41], lens=[90, 1000], heads=14, kv_heads=2, dtype="fp16", order="slot", layout="token", pad=9),
    dict(news=[150], lens=[100], heads=5, kv_heads=1), dict(news=[200, 100], lens=[130, 0], heads=2, kv_heads=2, d=128),
    dict(news=[700], lens=[3000], heads=3, kv_heads=1, page=64, dtype="fp16"), dict(news=[1374], lens=[2748], heads=2, kv_heads=2, page=64),
    dict(news=[33], lens=[9000], heads=64, kv_heads=1, d=128, page=256),
]


@pytest.mark.parametrize("impl", [1, 0])
@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("m", ATTENTION, ids=str)
def test_attention(paged, m, full, impl):
    w = World(paged, **m)
    out, lse, (out0, lse0) = w.attend(full, impl)
    w.check_attention(out, lse, full, out0, lse0)
    assert w.cache.xkv_paged_poll_status() == 0
    again, _, _ = w.attend(full, impl, with_lse=False)             # the same bits, with and without lse
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("m", [
    dict(news=[1, 3], lens=[900, 300], heads=4, kv_heads=1), dict(news=[2, 1], lens=[2000, 517], heads=2, kv_heads=2, d=128, dtype="fp16", page=64),
    dict(news=[100, 37], lens=[1500, 300], heads=4, kv_heads=2, page=32), dict(news=[200], lens=[2100], heads=3, kv_heads=1, dtype="fp16"),
    dict(news=[130, 257], lens=[900, 2000], heads=2, kv_heads=1, d=128), dict(news=[90], lens=[700], heads=8, kv_heads=2, d=128, dtype="fp16")], ids=str)
@pytest.mark.parametrize("kind", ["rising", "falling", "steps"])
@pytest.mark.parametrize("full", [False, True])
def test_attention_with_moving_maxima(paged, m, kind, full):
    """Scores that rise along the cache by more than 2^14 in their weights, again and again, for some heads; that fall; that
    jump inside a unit, differently for neighbouring rows.  (Scaled scores up to 50.)"""
    w = World(paged, **m)
    scale = 50.0 / (w.d * w.scale)
    for b, l in enumerate(w.lens_list):
        x = torch.arange(l, device="cuda") / l
        if kind == "falling":
            x = 1 - x
        elif kind == "steps":
            x = ((x * 11).floor() % 4) / 4 + 0.25 * (torch.arange(l, device="cuda") % 97 == 50)
        w.k[b] = (w.k[b].float() * 0.05 + (x * scale)[None, :, None]).to(w.dt)
        w.put(b, 0, l)
    sign = torch.where(torch.arange(w.n, device="cuda") % 3 == 1, -1.0, 1.0)[None, :, None]
    head = torch.linspace(0.3, 1.0, w.H, device="cuda")[:, None, None]
    w.q[:, :w.n] = (sign * head + 0.02 * w.q[:, :w.n].float()).to(w.dt)
    out, lse, (out0, lse0) = w.attend(full)
    w.check_attention(out, lse, full, out0, lse0)
    assert w.cache.xkv_paged_poll_status() == 0


@pytest.mark.parametrize("m", [
    dict(news=[1] * 1000, lens=[(13 * i) % 61 + 1 for i in range(1000)], heads=2, kv_heads=1),
    dict(news=[i % 3 for i in range(1024)], lens=[(7 * i) % 40 for i in range(1024)], heads=3, kv_heads=1),
    dict(news=[(5 * i) % 23 for i in range(700)], lens=[(11 * i) % 90 for i in range(700)], heads=2, kv_heads=2, d=128),
    dict(news=[0] * 650 + [40, 1], lens=[3] * 650 + [300, 20], heads=2, kv_heads=1, dtype="fp16")], ids=lambda m: f"{len(m['news'])}")
def test_many_sequences(paged, m):
    w = World(paged, **m)
    out, lse, before = w.attend(False)
    w.check_attention(out, lse, False, *before)
    ref = lse_of(w, False)
    old = w.weights.clone()
    w.cache.kv_paged_weights(w.batch, w.q, ref)
    for b in range(0, len(w.news), 7):
        if w.news[b] and w.lens_list[b]:
            want, room = w.weight_sums(b, False, ref)
            was = w.get(old, b, w.lens_list[b]).double()
            assert ((w.get(w.weights, b, w.lens_list[b]).double() - want - was).abs() <= room + 2.0 ** -22 * (want + was)).all(), b
    k, v = w.tokens(w.K), w.tokens(w.K)
    w.cache.kv_paged_append(w.batch, k, v)
    for b in range(0, len(w.news), 5):
        n = min(w.news[b], w.lens_list[b])
        if n:
            rows = slice(w.starts[b] + w.news[b] - n, w.starts[b] + w.news[b])
            assert torch.equal(w.get(w.k_pages, b, w.lens_list[b])[:, -n:], k[:, rows]) and torch.equal(w.get(w.v_pages, b, w.lens_list[b])[:, -n:], v[:, rows])
    assert w.cache.xkv_paged_poll_status() == 0


# ---- weights ---------------------------------------------------------------------------------

@pytest.mark.parametrize("decay", [1.0, 0.0, 0.75])
@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("m", ATTENTION, ids=str)
def test_weights(paged, m, full, decay):
    w = World(paged, **m)
    lse = lse_of(w, full)
    before = w.weights.clone()
    w.cache.kv_paged_weights(w.batch, w.q, lse, decay=decay, mask=int(full))
    touched = torch.zeros_like(before, dtype=torch.bool)
    for b, l in enumerate(w.lens_list):
        if not l or not w.news[b]:
            continue
        got = w.get(w.weights, b, l).double()
        old = w.get(before, b, l).double() * decay
        want, room = w.weight_sums(b, full, lse)
        assert ((got - want - old).abs() <= room + 2.0 ** -22 * (want + old)).all(), b
        page, place = w.pages_of(torch.arange(l, device="cuda"), b)
        touched[page, :, place] = True
    same = (w.weights == before) | (w.weights.isnan() & before.isnan())
    assert same[~touched].all()
    assert w.cache.xkv_paged_poll_status() == 0


# ---- eviction --------------------------------------------------------------------------------

def chosen(weights, keep, first, recent):
    """Kept slots of one head by the definition."""
    l = len(weights)
    if l <= keep:
        return list(range(l))
    middle = sorted(range(first, l - recent), key=lambda j: (math.isnan(weights[j]), 0.0 if math.isnan(weights[j]) else -weights[j], j))
    return sorted(list(range(first)) + middle[:keep - first - recent] + list(range(l - recent, l)))


EVICTIONS = [
    dict(lens=[40], keep=17, first=3, recent=5), dict(lens=[100, 16, 0, 65], keep=64, first=0, recent=0), dict(lens=[33, 200], keep=1, first=0, recent=1),
    dict(lens=[64], keep=64, first=10, recent=10), dict(lens=[300], keep=40, first=20, recent=20), dict(lens=[3000], keep=1500, first=261, recent=100, page=64, order="slot"),
    dict(lens=[70000], keep=30000, first=5, recent=7, page=256, heads=1, kv_heads=1), dict(lens=[500, 900], keep=333, first=1, recent=64, d=128, dtype="fp16", page=32),
]


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("m", EVICTIONS, ids=str)
def test_evict(paged, m, kind):
    m = dict(m)
    keep, first, recent = m.pop("keep"), m.pop("first"), m.pop("recent")
    lens = m["lens"]
    want_pages = sum(-(-min(l, keep) // m.get("page", 16)) for l in lens)
    w = World(paged, news=[0] * len(lens), spare_pages=want_pages + 2, **m)
    for b, l in enumerate(lens):
        if not l:
            continue
        x = torch.rand(l, w.K, device="cuda", generator=w.gen)
        if kind == "ties":
            x = (x * 5).floor() / 7
        elif kind == "equal":
            x = torch.full_like(x, 0.25)
        elif kind == "odd":
            x = torch.randn(l, w.K, device="cuda", generator=w.gen)
            x[::7] = math.nan
            x[::11] = math.inf
            x[::5] = -0.0
            x[1::5] = 0.0
            x[::13] = -math.inf
            x[2::17] = 1e-42
        page, place = w.pages_of(torch.arange(l, device="cuda"), b)
        w.weights[page, :, place] = x
    dst = torch.full((len(lens), -(-keep // w.P) + 1), 2 ** 30, dtype=torch.int32, device="cuda")
    at = 0
    for b, l in enumerate(lens):
        c = -(-min(l, keep) // w.P)
        dst[b, :c] = w.spare[at:at + c]
        at += c
    pools = [x.clone() for x in (w.k_pages, w.v_pages, w.weights)]
    kept, lens_out = w.cache.kv_paged_evict(w.batch, dst, keep, first, recent)
    assert w.cache.xkv_paged_poll_status() == 0
    assert lens_out.tolist() == [min(l, keep) for l in lens]
    written = torch.zeros_like(w.weights, dtype=torch.bool)
    bits = lambda x: x.contiguous().view(torch.int32 if x.dtype == torch.float32 else torch.int16)
    for b, l in enumerate(lens):
        new = min(l, keep)
        values = w.get(pools[2], b, l).tolist() if l else []
        page, place = w.pages_of(torch.arange(new, device="cuda"), b, dst)
        written[page, :, place] = True
        for h in range(w.K):
            want = chosen(values[h], keep, first, recent) if l else []
            assert kept[b, h].tolist() == want + [-1] * (keep - new), (b, h)
            idx = torch.tensor(want, dtype=torch.int64, device="cuda")
            for pool, old in zip((w.k_pages, w.v_pages, w.weights), pools):
                if new:
                    assert torch.equal(bits(w.get(pool, b, new, dst)[h]), bits(w.get(old, b, l)[h][idx])), (b, h)
    for now, before in zip((w.k_pages, w.v_pages, w.weights), pools):
        assert ((now == before) | (now.isnan() & before.isnan()))[~written].all()


# ---- what the device refuses -----------------------------------------------------------------

@pytest.mark.parametrize("kind", ["page", "negative page", "length", "negative length", "rows", "max_new"])
def test_bad_sequences_are_left_out(paged, kind):
    w = World(paged, news=[2, 40, 1], lens=[50, 90, 20], heads=4, kv_heads=2)
    good = [0, 2]
    if kind == "page":
        w.table[1, 2] = w.p.n_pages
    elif kind == "negative page":
        w.table[1, 0] = -5
    elif kind == "length":
        w.lens[1] = w.table.shape[1] * w.P + 1
    elif kind == "negative length":
        w.lens[1] = -1
    elif kind == "rows":
        w.q_start[3] = w.rows + 1
        good = [0, 1]
    batch = w.batch
    if kind == "max_new":
        batch = paged.PagedBatch(w.q_start, w.lens, w.table, w.rows, 39)
    k, v = w.tokens(w.K), w.tokens(w.K)
    bad_rows = slice(w.starts[3 - sum(good)], w.starts[3 - sum(good) + 1])
    page_kind = "page" in kind
    for impl in (1, 0):
        out, lse, before = w.attend(impl=impl, batch=batch)
        assert w.cache.xkv_paged_poll_status() == -1
        assert w.cache.xkv_paged_poll_status() == 0            # (the word is cleared)
        if not page_kind:
            assert (out[:, bad_rows] == 7.0).all() and (lse[:, bad_rows] == 7.0).all()
        news = list(w.news)
        w.news = [n if b in good else 0 for b, n in enumerate(news)]
        w.check_attention(out, lse, False, *before, tag=f"impl {impl}")
        w.news = news
    lse = lse_of(w, False)
    weights = w.weights.clone()
    w.cache.kv_paged_weights(batch, w.q, lse)
    assert w.cache.xkv_paged_poll_status() == -1
    for b in good:
        want, room = w.weight_sums(b, False, lse)
        old = w.get(weights, b, w.lens_list[b]).double()
        assert ((w.get(w.weights, b, w.lens_list[b]).double() - want - old).abs() <= room + 2.0 ** -22 * (want + old)).all()
    before = [x.clone() for x in (w.k_pages, w.v_pages)]
    w.cache.kv_paged_append(batch, k, v)
    assert w.cache.xkv_paged_poll_status() == (0 if page_kind else -1)       # (the page that is not there holds no new token's slot)
    for b in good:
        rows = slice(w.starts[b], w.starts[b] + w.news[b])
        assert torch.equal(w.get(w.k_pages, b, w.lens_list[b])[:, -w.news[b]:], k[:, rows])
    w.k_pages.copy_(before[0])
    w.v_pages.copy_(before[1])
    if kind not in ("rows", "max_new"):
        dst = w.spare[:3].reshape(3, 1).contiguous()
        kept, lens_out = w.cache.kv_paged_evict(w.batch, dst, 16, 2, 3)
        assert w.cache.xkv_paged_poll_status() == -1
        assert [lens_out[b].item() for b in good] == [16, 16] and (page_kind or lens_out[1].item() == 0)
        for b in good:
            for h in range(w.K):
                idx = kept[b, h].long()
                assert torch.equal(w.get(w.k_pages, b, 16, dst)[h], w.k[b][h][idx])


# ---- streams, graphs, the operators together ---------------------------------------------------

def test_replayed_graph_reads_new_lengths(paged):
    """One captured decoding step, replayed while the sequences grow."""
    w = World(paged, news=[1, 1], lens=[1, 1], spare_pages=12, extra_width=5)
    w.table[:, :5] = torch.arange(10, device="cuda", dtype=torch.int32).reshape(2, 5)
    for b in range(2):
        w.k[b], w.v[b] = w.k[b][:, :0], w.v[b][:, :0]
    k, v = w.tokens(w.K), w.tokens(w.K)
    pos = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(w.q), torch.zeros(w.H, 2, device="cuda")
    rot = paged.RotaryParams(64)
    q_in, q_rot = w.q, torch.zeros_like(w.q)
    w.lens.zero_()

    def step():
        w.lens.add_(1)
        w.cache.kv_paged_append(w.batch, k, v, q=q_in, q_out=q_rot, rotary=rot, positions=pos)
        w.cache.attn_paged_causal(w.batch, q_rot, out=out, lse=lse)
        w.cache.kv_paged_weights(w.batch, q_rot, lse)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()                                       # warm-up
        side.synchronize()
        w.lens.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    w.lens.zero_()
    for t in range(70):
        k.copy_(w.rand(*k.shape)), v.copy_(w.rand(*v.shape)), q_in.copy_(w.rand(*q_in.shape))
        pos.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        w.lens_list = [t + 1] * 2
        w.q = q_rot
        for b in range(2):
            w.k[b] = torch.cat([w.k[b], w.get(w.k_pages, b, t + 1)[:, -1:]], 1)     # (the rotation has tests of its own)
            w.v[b] = torch.cat([w.v[b], v[:, b:b + 1]], 1)
            assert torch.equal(w.get(w.v_pages, b, t + 1), w.v[b]) and torch.equal(w.get(w.k_pages, b, t + 1), w.k[b])
        w.check_attention(out, lse, False, out, lse, f"step {t}")
    assert w.cache.xkv_paged_poll_status() == 0


def test_replayed_graph_of_a_chunk(paged):
    """A captured chunk: attention, weights and eviction, replayed with other lengths, tables and tokens in the same places."""
    w = World(paged, news=[60, 100], lens=[200, 300], heads=4, kv_heads=2, d=128, page=32, spare_pages=8)
    out, lse = torch.zeros_like(w.q), torch.zeros(w.H, w.rows, device="cuda")
    dst = w.spare[:8].reshape(2, 4).contiguous()
    kept, lens_out = torch.zeros(2, w.K, 100, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")

    def step():
        w.cache.attn_paged_causal(w.batch, w.q, out=out, lse=lse)
        w.cache.kv_paged_weights(w.batch, w.q, lse, decay=0.0)
        w.cache.kv_paged_evict(w.batch, dst, 100, 5, 20, kept=kept, lens_out=lens_out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for news, lens, flip in (([60, 100], [200, 300], False), ([10, 3], [180, 299], False), ([100, 60], [300, 200], True), ([0, 100], [17, 100], False)):
        if flip:
            w.table.copy_(w.table.flip(0))
            w.k.reverse(), w.v.reverse()
        w.q.copy_(w.rand(*w.q.shape))
        w.news, w.lens_list, w.starts, w.n = news, lens, [0, news[0], sum(news)], sum(news)
        k, v = list(w.k), list(w.v)
        w.k, w.v = [x[:, :l] for x, l in zip(k, lens)], [x[:, :l] for x, l in zip(v, lens)]
        w.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        w.q_start.copy_(torch.tensor(w.starts, dtype=torch.int32))
        out.fill_(7.0), lse.fill_(7.0)
        before = out.clone(), lse.clone()
        graph.replay()
        torch.cuda.synchronize()
        w.check_attention(out, lse, False, *before)
        for b in range(2):
            if news[b]:
                want, room = w.weight_sums(b, False, lse)
                got = w.get(w.weights, b, lens[b])
                assert ((got.double() - want).abs() <= room + 2.0 ** -22 * want).all()
                for h in range(w.K):
                    assert kept[b, h, :min(lens[b], 100)].tolist() == chosen(got[h].tolist(), 100, 5, 20)
        assert lens_out.tolist() == [min(l, 100) for l in lens]
        w.k, w.v = k, v
        if flip:
            w.table.copy_(w.table.flip(0))
            w.k.reverse(), w.v.reverse()
    assert w.cache.xkv_paged_poll_status() == 0


@pytest.mark.parametrize("dtype, d, heads, kv_heads, page", [("bf16", 64, 4, 4, 16), ("fp16", 128, 8, 2, 64)])
def test_run_together(paged, dtype, d, heads, kv_heads, page):
    """Requests that arrive in chunks, decode, and are cut back: append, attention, weights, eviction, and on."""
    B, budget, first, recent = 3, 150, 8, 40
    chunks = [[100, 7, 0], [33, 130, 90], [1, 1, 1], [1, 1, 1], [60, 0, 1]]
    width, half = 16, B * 16
    dt = DTYPE[dtype]
    gen = torch.Generator(device="cuda").manual_seed(3)
    kp, vp = (torch.full((2 * half, kv_heads, page, d), math.nan, device="cuda", dtype=dt) for _ in range(2))
    wp = torch.full((2 * half, kv_heads, page), math.nan, device="cuda")
    cache = paged.PagedCache(paged.PagedParams(heads, kv_heads, d, page, 2 * half, B, dtype), kp, vp, wp)
    perm = torch.randperm(2 * half, device="cuda", generator=gen).to(torch.int32)
    tables = [perm[:half].reshape(B, width).contiguous(), perm[half:].reshape(B, width).contiguous()]
    rot = paged.RotaryParams(d // 2, interleaved=True)
    ref_k = [torch.zeros(kv_heads, 0, d, device="cuda", dtype=dt) for _ in range(B)]
    ref_v = [torch.zeros(kv_heads, 0, d, device="cuda", dtype=dt) for _ in range(B)]
    ref_w = [torch.zeros(kv_heads, 0, device="cuda", dtype=torch.float64) for _ in range(B)]
    lens, at = [0] * B, [0] * B                       # cached tokens, positions so far
    for step, news in enumerate(chunks):
        n = sum(news)
        starts = [sum(news[:b]) for b in range(B + 1)]
        lens = [l + m for l, m in zip(lens, news)]
        make = lambda h: torch.randn(n, h, d, device="cuda", generator=gen).to(dt).transpose(0, 1)
        q, k, v = make(heads), make(kv_heads), make(kv_heads)
        pos = torch.cat([torch.arange(a, a + m) for a, m in zip(at, news)]).to(torch.int32).cuda()
        at = [a + m for a, m in zip(at, news)]
        dev_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        batch = paged.PagedBatch(torch.tensor(starts, dtype=torch.int32, device="cuda"), dev_lens, tables[0], n, max(news))
        turned_q = cache.kv_paged_append(batch, k, v, q=q, rotary=rot, positions=pos)
        lse = torch.zeros(heads, n, device="cuda")
        out = cache.attn_paged_causal(batch, turned_q, lse=lse)
        cache.kv_paged_weights(batch, turned_q, lse)
        # the definition, on the keys and queries as they were turned (checked here to half a step)
        view = World.__new__(World)
        view.H, view.K, view.d, view.dt, view.P, view.scale = heads, kv_heads, d, dt, page, d ** -0.5
        view.news, view.lens_list, view.starts, view.n, view.rows, view.q, view.table = news, lens, starts, n, n, turned_q, tables[0]
        want_q, room_q = turned(q, pos[None], d // 2, interleaved=True)
        want_k, room_k = turned(k, pos[None], d // 2, interleaved=True)
        assert ((turned_q.double() - want_q).abs() <= HALF[dt] * want_q.abs() + room_q * 1.01 + 2.0 ** -25).all()
        for b in range(B):
            rows = slice(starts[b], starts[b + 1])
            new_k = view.get(kp, b, lens[b])[:, lens[b] - news[b]:]
            assert ((new_k.double() - want_k[:, rows]).abs() <= HALF[dt] * want_k[:, rows].abs() + room_k[:, rows] * 1.01 + 2.0 ** -25).all()
            ref_k[b], ref_v[b] = torch.cat([ref_k[b], new_k], 1), torch.cat([ref_v[b], v[:, rows]], 1)
            ref_w[b] = torch.cat([ref_w[b], torch.zeros(kv_heads, news[b], device="cuda", dtype=torch.float64)], 1)
            assert torch.equal(view.get(kp, b, lens[b]), ref_k[b]) and torch.equal(view.get(vp, b, lens[b]), ref_v[b])
        view.k, view.v = ref_k, ref_v
        view.check_attention(out, lse, False, out, lse, f"step {step}")
        for b in range(B):
            if news[b]:
                got, room = view.weight_sums(b, False, lse)
                ref_w[b] = ref_w[b] + got
                assert ((view.get(wp, b, lens[b]).double() - ref_w[b]).abs() <= room + 2.0 ** -16 * ref_w[b]).all()
                ref_w[b] = view.get(wp, b, lens[b]).double()              # (so that choices below are on the same numbers)
        kept, lens_out = cache.kv_paged_evict(batch, tables[1], budget, first, recent)
        for b in range(B):
            for h in range(kv_heads):
                want = chosen(ref_w[b][h].tolist(), budget, first, recent)
                assert kept[b, h, :len(want)].tolist() == want
            idx = kept[b, :, :min(lens[b], budget)].long()
            gather = lambda x: torch.gather(x, 1, idx[..., None].expand(-1, -1, d))
            ref_k[b], ref_v[b], ref_w[b] = gather(ref_k[b]), gather(ref_v[b]), torch.gather(ref_w[b], 1, idx)
        lens = [min(l, budget) for l in lens]
        assert lens_out.tolist() == lens
        tables.reverse()
    assert cache.xkv_paged_poll_status() == 0 and max(lens) == budget


def test_other_stream_and_strides(paged):
    """Token tensors inside larger ones, on a stream of their own."""
    w = World(paged, news=[20, 3], lens=[60, 33], heads=4, kv_heads=2, layout="token")
    big = torch.full((w.rows, 3, w.H + w.K, w.d), math.nan, device="cuda", dtype=w.dt)
    view = big[:, 1, :w.H].transpose(0, 1)
    view.copy_(w.q)
    w.q = view
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        big_out = torch.full((w.H, w.rows, 2 * w.d), 7.0, device="cuda", dtype=w.dt)
        out, lse = big_out[..., w.d:], torch.zeros(w.H, w.rows, device="cuda")
        w.cache.attn_paged_causal(w.batch, w.q, out=out, lse=lse)
    side.synchronize()
    w.check_attention(out, lse, False, out, lse)
    assert (big_out[..., :w.d] == 7.0).all()


def test_large_pool(paged):
    """Pages beyond 2^32 bytes of a pool."""
    n_pages, K, P, d = 140000, 1, 256, 64                      # 4.6 GB a pool
    kp, vp = (torch.empty(n_pages, K, P, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    wp = torch.zeros(n_pages, K, P, device="cuda")
    cache = paged.PagedCache(paged.PagedParams(2, K, d, P, n_pages, 1), kp, vp, wp)
    w = World(paged, news=[200], lens=[500], heads=2, kv_heads=1, page=256)
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    kp[table[0].long()] = w.k_pages[w.table[0, :2].long()]
    vp[table[0].long()] = w.v_pages[w.table[0, :2].long()]
    for news, rows in ((200, 200), (1, 1)):
        batch = paged.PagedBatch(torch.tensor([0, rows], dtype=torch.int32, device="cuda"), w.lens, table, rows, rows)
        w.news, w.starts, w.n, w.rows, w.q = [rows], [0, rows], rows, rows, w.q[:, :rows]
        out, lse = torch.zeros_like(w.q), torch.zeros(w.H, rows, device="cuda")
        cache.attn_paged_causal(batch, w.q, out=out, lse=lse)
        w.check_attention(out, lse, False, out, lse)
        wp.zero_()
        cache.kv_paged_weights(batch, w.q, lse)
        got, room = w.weight_sums(0, False, lse)
        assert ((w.get(wp, 0, 500, table).double() - got).abs() <= room + 2.0 ** -22 * got).all()
    dst = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    kept, _ = cache.kv_paged_evict(batch, dst, 300, 0, 10)
    assert torch.equal(w.get(kp, 0, 300, dst)[0], w.k[0][0][kept[0, 0].long()])
    k, v = torch.ones(1, 1, d, device="cuda", dtype=torch.bfloat16), torch.ones(1, 1, d, device="cuda", dtype=torch.bfloat16)
    cache.kv_paged_append(batch, k, v)
    assert (w.get(kp, 0, 500, table)[0, -1] == 1).all() and (w.get(vp, 0, 500, table)[0, -1] == 1).all()
    assert cache.xkv_paged_poll_status() == 0
