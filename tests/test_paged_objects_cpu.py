"""What a batch and a cache hold for the library is set once."""
import pytest

from paper_2601_01204_b200 import build


@pytest.fixture(scope="module")
def paged():
    build.build()
    import paper_2601_01204_b200.paged as m
    return m


@pytest.mark.parametrize("kind, names", [
    ("PagedBatch", ("q_start", "lens", "table", "n_tokens", "max_new", "n_seqs", "device", "struct", "ref")),
    ("PagedCache", ("k_pages", "v_pages", "weights", "workspace", "p", "device", "dtype"))])
def test_attributes_that_the_library_points_to_are_fixed(paged, kind, names):
    x = getattr(paged, kind).__new__(getattr(paged, kind))
    if kind == "PagedCache":
        x.handle = None
    for name in names:
        setattr(x, name, 1)
        with pytest.raises(AttributeError, match=name):
            setattr(x, name, 2)
        with pytest.raises(AttributeError, match=name):
            delattr(x, name)
        assert getattr(x, name) == 1
    x.scale = 0.5
    x.scale = 0.25                  # (read by the binding itself, at every call)
