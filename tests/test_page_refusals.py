"""The calls over pages without a context: refused before anything is looked at, through both marshallings; the structures of the
binding against the header's."""
import ctypes

import pytest
import torch

import paper_2406_19707_amd as ig
from paper_2406_19707_amd import binding

COUNTS = {"ig_rotate_rows": 13, "ig_append_pages": 15, "ig_page_attention": 10, "ig_gather_pages": 9}


def pages():
    K = torch.zeros((2, 1, 16, 64), dtype=torch.int8)
    return ig.IgPages(torch.zeros((1, 1), dtype=torch.int32), K, K.clone(), torch.ones((2, 1)), torch.ones((2, 1)), ig.IG_CODE_I8)


def arguments(name, structures):
    d, p = ig.IgDesc(B=1, H=1, d=64, r=1, N=8), pages() if structures else None
    r = ig.IgRotary(torch.zeros(32, dtype=torch.float64)) if structures else None
    t = torch.zeros(64)
    return {"ig_rotate_rows": [None, 1, 1, 1, 64, r, 0, t, t, 0, t, 0, None],
            "ig_append_pages": [None, d, p, r, 1, 1, t, t, t, 0, None, None, None, t, None],
            "ig_page_attention": [None, d, p, 1, 1, t, None, None, t, None],
            "ig_gather_pages": [None, d, p, t, 1, t, t, t, None]}[name]


@pytest.mark.parametrize("structures", [True, False])
@pytest.mark.parametrize("name", COUNTS)
def test_no_context(name, structures):
    args = arguments(name, structures)
    assert len(getattr(binding.lib(), name).argtypes) == COUNTS[name] == len(args)
    assert binding._through_ctypes(name, *args) == ig.IG_EINVAL
    assert getattr(binding._Entries(), name)(*args) == ig.IG_EINVAL


@pytest.mark.parametrize("wrong", ["a tensor", b"x" * 48, 7, "descriptor", "the other structure"])
def test_other_things_in_a_structures_place(wrong):
    """The same outcome from both marshallings: an exception, never a call."""
    what = {"a tensor": torch.zeros(6, dtype=torch.int64), "descriptor": ig.IgDesc(B=1, H=1, d=64, r=1, N=8),
            "the other structure": ig.IgRotary(torch.zeros(32, dtype=torch.float64))}.get(wrong, wrong) if isinstance(wrong, str) else wrong
    args = arguments("ig_page_attention", True)
    args[2] = what
    for call in (lambda: binding._through_ctypes("ig_page_attention", *args), lambda: binding._Entries().ig_page_attention(*args)):
        with pytest.raises((ctypes.ArgumentError, TypeError)):
            call()


def test_reserve_without_context():
    assert ig.lib().ig_reserve_pages(None, None, 1, 1) == ig.IG_EINVAL


def test_structures_hold_their_tensors():
    p = pages()
    K = p.tensors[1]
    assert p.K == K.data_ptr() and (p.n_pages, p.page_size, p.table_stride, p.code) == (2, 16, 1, ig.IG_CODE_I8)
    assert ctypes.sizeof(ig.IgPages) == 4 * 4 + 5 * 8 and ctypes.sizeof(ig.IgRotary) == 24
    r = ig.IgRotary(torch.zeros(32, dtype=torch.float64), interleaved=True, magnitude=1.5)
    assert (r.dims, r.interleaved, r.magnitude, r.freq) == (64, 1, 1.5, r.tensors[0].data_ptr())


@pytest.mark.parametrize("change", ["V shape", "scale shape", "code type", "scale type", "table type", "not dense"])
def test_structures_look_at_shapes(change):
    K, V, s, t = torch.zeros((2, 1, 16, 64), dtype=torch.int8), torch.zeros((2, 1, 16, 64), dtype=torch.int8), torch.ones((2, 1)), \
        torch.zeros((1, 1), dtype=torch.int32)
    args = {"V shape": (t, K, V[:1], s, s), "scale shape": (t, K, V, s[:, 0], s), "code type": (t, K.half(), V.half(), s, s),
            "scale type": (t, K, V, s.double(), s.double()), "table type": (t.long(), K, V, s, s),
            "not dense": (t, K.transpose(2, 3).contiguous().transpose(2, 3), V, s, s)}[change]
    with pytest.raises(AssertionError):
        ig.IgPages(*args)
