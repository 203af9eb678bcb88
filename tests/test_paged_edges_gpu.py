"""The paged cache where its numbers are not finite, its tables name pages that do not exist, its caches are very long, and
with enough work for every ring and every cut of the kernels to go round more than once."""
import math

import pytest
import torch

from paged_testlib import World, lse_of

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
