"""CPU-side checks of the paged cache's C ABI: exports, and every refusal, on a device that launches nothing."""
import ctypes as C
import os
import re
import struct
import subprocess

import pytest

from paper_2601_01204_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))
OK, INVALID, STATE, NOMEM, UNSUPPORTED, LIMIT = 0, -1, -2, -3, -4, -7
A = 1 << 40                                   # an address that nobody reads


@pytest.fixture(scope="module")
def paged():
    build.build()
    import paper_2601_01204_b200.paged as m
    return m


@pytest.fixture(scope="module")
def lib(paged, tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host_paged") / "libfake.so")
    subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-shared", "-cudart", "none",
                    "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                    os.path.join(build.CSRC, "xkv_paged_host.cu"), os.path.join(HERE, "host_paged", "fake_device.cpp"), "-o", so],
                   check=True)
    fake = C.CDLL(so)
    for name in paged.EXPORTED:
        getattr(fake, name).restype = getattr(paged.lib, name).restype
        getattr(fake, name).argtypes = getattr(paged.lib, name).argtypes
    return fake


def test_exports_match_header(paged, repo_root):
    text = open(os.path.join(repo_root, "include", "xkv_paged.h")).read()
    declared = re.findall(r"XKV_API\s+[\w\s\*]+?\b(\w+)\s*\(", text)
    assert sorted(declared) == sorted(paged.EXPORTED)
    for name in declared:
        assert hasattr(paged.lib, name), name


def params(paged, **more):
    v = dict(n_heads=8, n_kv_heads=2, head_dim=64, dtype=0, page_tokens=16, n_pages=10, max_seqs=4, reserved=0,
             page_stride=2048, head_stride=1024, slot_stride=64)
    v.update(more)
    return paged.xkv_paged_params(*[v[n] for n, _ in paged.xkv_paged_params._fields_])


@pytest.mark.parametrize("more, code", [
    (dict(), OK), (dict(n_heads=0), INVALID), (dict(n_heads=7), INVALID), (dict(n_kv_heads=0), INVALID), (dict(n_heads=128), INVALID),
    (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=-1), INVALID), (dict(dtype=2), INVALID), (dict(page_tokens=8), UNSUPPORTED),
    (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=512), UNSUPPORTED), (dict(page_tokens=0), INVALID), (dict(n_pages=0), INVALID),
    (dict(max_seqs=0), INVALID), (dict(max_seqs=1025), INVALID), (dict(reserved=1), INVALID), (dict(page_stride=0), INVALID),
    (dict(head_stride=4), INVALID), (dict(slot_stride=56), INVALID), (dict(slot_stride=-64), INVALID), (dict(page_stride=1 << 40), INVALID),
])
def test_create_refuses(paged, lib, more, code):
    p, h = params(paged, **more), C.c_void_p(1)
    need = lib.xkv_paged_workspace_bytes(C.byref(p), 148)
    assert (need > 0) == (code == OK)
    assert lib.xkv_paged_create(C.byref(p), A, A, A, A, 1 << 40, None, C.byref(h)) == code
    assert bool(h.value) == (code == OK)
    if h.value:
        assert lib.xkv_paged_destroy(h) == OK


def test_create_refuses_pointers(paged, lib):
    p, h = params(paged), C.c_void_p()
    need = lib.xkv_paged_workspace_bytes(C.byref(p), 148)
    call = lambda *x: lib.xkv_paged_create(C.byref(p), *x, None, C.byref(h))
    assert call(None, A, A, A, need) == INVALID
    assert call(A + 8, A, A, A, need) == INVALID
    assert call(A, A + 2, A, A, need) == INVALID
    assert call(A, A, A + 2, A, need) == INVALID
    assert call(A, A, A, A + 128, need) == INVALID
    assert call(A, A, A, A, need - 1) == NOMEM
    assert call(A, A, None, A, need) == OK
    assert lib.xkv_paged_destroy(h) == OK and lib.xkv_paged_destroy(None) == INVALID
    assert lib.xkv_paged_create(None, A, A, A, A, need, None, C.byref(h)) == INVALID
    assert lib.xkv_paged_create(C.byref(p), A, A, A, A, need, None, None) == INVALID
    assert lib.xkv_paged_workspace_bytes(C.byref(p), 0) == 0


def rows(*tensors):
    """An array of xkv_rows."""
    return struct.pack(f"{len(tensors)}q", *tensors)


class Calls:
    """The calls with arguments that are in order, each of which a test can put out of order."""

    def __init__(self, paged, lib, weights=A):
        self.paged, self.lib = paged, lib
        p = params(paged)
        self.h = C.c_void_p()
        assert lib.xkv_paged_create(C.byref(p), A, A, weights, A, 1 << 40, None, C.byref(self.h)) == OK

    def batch(self, **m):
        v = dict(n_seqs=2, n_tokens=5, max_new=3, table_width=4, q_start=A, lens=A, table=A)
        v.update(m)
        return C.byref(self.paged.xkv_paged_batch(*[v[n] for n, _ in self.paged.xkv_paged_batch._fields_]))

    def rotary(self, **m):
        v = dict(rotary_dim=64, n_axes=1, interleaved=0, original_tokens=0, base=1e4, factor=1.0, beta_fast=32.0, beta_slow=1.0, magnitude=1.0)
        v.update(m)
        return C.byref(self.paged.xkv_rotary_params(*[v[n] for n, _ in self.paged.xkv_rotary_params._fields_]))

    def append(self, batch=None, k=A, kt=64, kh=512, v=A, vt=64, vh=512, q=A, qt=64, qh=512, o=A + 4096, ot=64, oh=512, rot="", pos=A, ps=5, h=""):
        return self.lib.kv_paged_append(self.h if h == "" else h, batch or self.batch(), rows(k, kt, kh, v, vt, vh, q, qt, qh, o, ot, oh),
                                        self.rotary() if rot == "" else rot, pos, ps, None)

    def attend(self, batch=None, q=A, qt=64, qh=512, o=A, ot=64, oh=512, lse=A, scale=0.125, mask=0, impl=0, h=""):
        return self.lib.attn_paged_causal(self.h if h == "" else h, batch or self.batch(), rows(q, qt, qh, o, ot, oh), lse, scale, mask, impl, None)

    def weigh(self, batch=None, q=A, qt=64, qh=512, lse=A, scale=0.125, decay=1.0, mask=0, h=""):
        return self.lib.kv_paged_weights(self.h if h == "" else h, batch or self.batch(), rows(q, qt, qh), lse, scale, decay, mask, None)

    def evict(self, batch=None, dst=A + 4096, width=4, keep=40, first=4, recent=8, kept=A, lens=A + 64, h=""):
        return self.lib.kv_paged_evict(self.h if h == "" else h, batch or self.batch(), dst, width, keep, first, recent, kept, lens, None)


@pytest.fixture()
def calls(paged, lib):
    c = Calls(paged, lib)
    yield c
    lib.xkv_paged_destroy(c.h)


BAD_BATCHES = [dict(n_seqs=0), dict(n_seqs=5), dict(n_tokens=-1), dict(max_new=-1), dict(table_width=-1), dict(table_width=1 << 27),
               dict(q_start=0), dict(lens=0), dict(table=0), dict(lens=A + 2)]


def test_batches_are_refused(calls):
    n = calls.lib.fake_launches()
    for m in BAD_BATCHES:
        for call in (calls.append, calls.attend, calls.weigh):
            assert call(batch=calls.batch(**m)) == INVALID, m
        if not {"q_start", "n_tokens", "max_new"} & set(m):
            assert calls.evict(batch=calls.batch(**m)) == INVALID, m
    assert calls.lib.fake_launches() == n
    # what a call does not read may be missing
    assert calls.evict(batch=calls.batch(q_start=0, n_tokens=-1, max_new=-1)) == OK


def test_calls_without_work_launch_nothing(calls):
    n = calls.lib.fake_launches()
    empty = calls.batch(n_tokens=0)
    assert calls.append(batch=empty, k=0, v=0, q=0) == OK
    assert calls.attend(batch=empty, q=0, o=0, lse=0) == OK
    assert calls.attend(batch=calls.batch(max_new=0)) == OK
    assert calls.weigh(batch=empty, q=0) == OK
    assert calls.lib.fake_launches() == n
    assert calls.lib.kv_paged_append(calls.h, calls.batch(), None, None, None, 0, None) == INVALID
    assert calls.lib.attn_paged_causal(calls.h, calls.batch(), None, A, 1.0, 0, 0, None) == INVALID
    assert calls.lib.kv_paged_weights(calls.h, calls.batch(), None, A, 1.0, 1.0, 0, None) == INVALID
    assert calls.lib.fake_launches() == n
    assert calls.append() == OK and calls.append(q=0) == OK and calls.append(rot=None, pos=0) == OK
    assert calls.attend() == OK and calls.attend(lse=0) == OK and calls.attend(impl=1, mask=1) == OK
    assert calls.weigh() == OK and calls.evict() == OK
    assert calls.lib.fake_launches() == n + 8


@pytest.mark.parametrize("m", [dict(h=None), dict(k=0), dict(k=A + 8), dict(kt=60), dict(kh=0), dict(v=0), dict(vt=-64), dict(vh=4),
                               dict(q=A + 2), dict(o=0), dict(ot=63), dict(qh=1 << 40), dict(o=A, ot=128), dict(pos=0), dict(pos=A + 2)])
def test_append_refuses(calls, m):
    assert calls.append(**m) == INVALID


@pytest.mark.parametrize("m", [dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=66), dict(n_axes=0), dict(n_axes=5), dict(n_axes=2),
                               dict(base=1.0), dict(base=float("nan")), dict(factor=0.5), dict(factor=float("inf")), dict(magnitude=0.0),
                               dict(original_tokens=-1), dict(original_tokens=10, beta_fast=1.0), dict(original_tokens=10, beta_slow=-1.0)])
def test_rotary_parameters_are_refused(calls, m):
    r = calls.rotary(**m)
    assert calls.append(rot=r) == INVALID
    assert calls.lib.xkv_rotary(r, 0, 64, A, 5, 5, rows(A, 64, 512, A, 64, 512, 0, 0, 0, 0, 0, 0), 2, 0, 0, None) == INVALID


def test_rotary_refuses(calls):
    def call(dtype=0, d=64, pos=A, ps=5, n=5, q=A, o=A, heads=2, qt=64, qh=512, ot=64, oh=512, k=A, ko=A, kheads=2, kt=64, kh=512, kot=64, koh=512, **m):
        return calls.lib.xkv_rotary(calls.rotary(rotary_dim=32, **m), dtype, d, pos, ps, n, rows(q, qt, qh, o, ot, oh, k, kt, kh, ko, kot, koh),
                                    heads, kheads, 0, None)
    assert call() == OK and call(k=0, ko=0, kheads=0) == OK and call(n=0, q=0, pos=0) == OK and call(n_axes=2) == OK
    for m in (dict(dtype=2), dict(d=60), dict(d=256), dict(d=16), dict(n=-1), dict(pos=0), dict(q=0), dict(o=0), dict(heads=0), dict(qt=4),
              dict(k=0), dict(ko=A + 8), dict(kt=0), dict(ot=128), dict(koh=1024), dict(kheads=-1), dict(n_axes=2, ps=4)):
        assert call(**m) == INVALID, m


@pytest.mark.parametrize("m", [dict(h=None), dict(q=0), dict(q=A + 8), dict(o=0), dict(qt=0), dict(oh=12), dict(lse=A + 1), dict(scale=0.0),
                               dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(mask=2), dict(mask=-1), dict(impl=2)])
def test_attention_refuses(calls, m):
    assert calls.attend(**m) == INVALID


@pytest.mark.parametrize("m", [dict(h=None), dict(q=0), dict(qh=0), dict(lse=0), dict(lse=A + 2), dict(scale=0.0), dict(decay=-0.5),
                               dict(decay=float("nan")), dict(decay=float("inf")), dict(mask=3)])
def test_weights_refuse(calls, m):
    assert calls.weigh(**m) == INVALID


@pytest.mark.parametrize("m", [dict(h=None), dict(dst=0), dict(width=2), dict(width=0), dict(width=1 << 27), dict(keep=0), dict(first=-1), dict(recent=-1),
                               dict(first=30, recent=11), dict(kept=0), dict(lens=0), dict(kept=A + 2), dict(lens=A),
                               dict(lens=A + 4), dict(dst=A)])
def test_eviction_refuses(calls, m):
    assert calls.evict(**m) == INVALID


def test_work_beyond_the_counters_is_refused(calls):
    big = calls.batch(n_seqs=4, table_width=(1 << 27) - (1 << 13), max_new=1 << 20, n_tokens=1 << 22)
    n = calls.lib.fake_launches()
    assert calls.attend(batch=big) == LIMIT and calls.weigh(batch=big) == LIMIT
    assert calls.lib.fake_launches() == n
    assert calls.attend(batch=calls.batch(n_seqs=4, table_width=(1 << 27) - (1 << 13), max_new=1)) == OK


def test_without_weights(paged, lib):
    c = Calls(paged, lib, weights=None)
    assert c.append() == OK and c.attend() == OK
    assert c.weigh() == STATE and c.evict() == STATE
    lib.xkv_paged_destroy(c.h)


def test_other_device(calls):
    calls.lib.fake_set_device(1)
    try:
        assert calls.append() == INVALID and calls.attend() == INVALID and calls.weigh() == INVALID and calls.evict() == INVALID
        assert calls.lib.xkv_paged_poll_status(calls.h, None) == INVALID
    finally:
        calls.lib.fake_set_device(0)
    assert calls.lib.xkv_paged_poll_status(calls.h, None) == OK and calls.lib.xkv_paged_poll_status(None, None) == INVALID


def test_binding_refuses_before_the_library(paged):
    import torch
    from paper_2601_01204_b200.xkv import XkvError
    with pytest.raises(XkvError):
        paged.xkv_rotary(paged.RotaryParams(64), torch.zeros(4, dtype=torch.int32), torch.zeros(2, 4, 64, dtype=torch.bfloat16))
    with pytest.raises(XkvError):
        paged.PagedBatch(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32), 4, 4)
    with pytest.raises(XkvError):
        paged.PagedCache(paged.PagedParams(8, 2, 64, 16, 1, 1), torch.zeros(1, 2, 16, 64), torch.zeros(1, 2, 16, 64))
