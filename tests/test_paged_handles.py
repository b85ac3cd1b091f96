"""A handle's tensors stay those that it was made with: the calls go by their addresses.  Without a GPU."""
import pytest
import torch

import paper_2505_21136_amd as sage
from paper_2505_21136_amd import paged


@pytest.fixture
def handles(monkeypatch):
    monkeypatch.setattr(paged, "_current", lambda: -1)      # host tensors, that no call gets
    monkeypatch.setattr(paged, "_here", lambda t, what: None)
    pages = sage.PageTable.empty(6, page_tokens=64, slots=3, width=2, device="cpu")
    return pages, sage.PagedCache.empty(pages, 2, 64, torch.float16, k_shift=torch.zeros(2, 64))


@pytest.mark.parametrize("name", ["table", "lens", "refs", "page_tokens", "n_pages", "slots", "width", "ref", "device_index"])
def test_a_table_keeps_what_it_was_made_with(handles, name):
    pages, _ = handles
    old = getattr(pages, name)
    with pytest.raises(sage.SageError, match=f"PageTable.{name}"):
        setattr(pages, name, old.clone() if isinstance(old, torch.Tensor) else object())
    with pytest.raises(sage.SageError, match=f"PageTable.{name}"):
        delattr(pages, name)
    assert getattr(pages, name) is old


@pytest.mark.parametrize("name", ["pages", "k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "k_shift", "Hkv", "d", "fmt", "dtype", "ref"])
def test_a_cache_keeps_what_it_was_made_with(handles, name):
    _, cache = handles
    old = getattr(cache, name)
    with pytest.raises(sage.SageError, match=f"PagedCache.{name}"):
        setattr(cache, name, old.clone() if isinstance(old, torch.Tensor) else object())
    with pytest.raises(sage.SageError, match=f"PagedCache.{name}"):
        delattr(cache, name)
    assert getattr(cache, name) is old


def test_a_shift_cannot_be_brought_later(handles):
    pages, _ = handles
    cache = sage.PagedCache.empty(pages, 2, 64, torch.float16)
    with pytest.raises(sage.SageError, match="PagedCache.k_shift"):
        cache.k_shift = torch.zeros(2, 64)


def test_values_are_changed_in_place(handles):
    pages, cache = handles
    at = pages.lens.data_ptr()
    pages.lens[:] = torch.tensor([7, 8, 9], dtype=torch.int32)
    pages.lens.sub_(1)
    pages.lens -= 1                                          # (Python sets the attribute to the same tensor again)
    pages.lens[0] += 3
    cache.v_scale.mul_(2.0)
    cache.v_scale *= 2.0
    assert pages.lens.tolist() == [8, 6, 7] and pages.lens.data_ptr() == at == pages._c.lens


def test_a_workspace_of_fewer_bytes_than_elements_is_refused(handles):
    """A broadcast tensor has as many elements as one likes and the memory of one: the calls would write behind it."""
    pages, cache = handles
    q = torch.zeros(3, 2, 64, dtype=torch.float16)
    wide = torch.zeros(64, dtype=torch.uint8).expand(1 << 16, 64)
    for ws in (wide, wide.flatten()[:1].expand(1 << 20), torch.zeros(1 << 16)[::2]):
        for call in (lambda: sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=128, split_keys=64, workspace=ws),
                     lambda: sage.sage_pages_compact(pages, workspace=ws)):
            with pytest.raises(sage.SageError, match="workspace must be contiguous"):
                call()
