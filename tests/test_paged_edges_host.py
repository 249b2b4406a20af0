"""Paged caches and their pipeline on the host: refusals at the ends of the arguments' ranges, and which sequence holds which pages (no GPU
needed)."""
import pytest
import torch

import paper_2410_18311_b200 as ci
from test_paged_host import P, cache, lib  # noqa: F401


def test_attention_refuses_scales_beyond_what_base_2_takes(lib):  # noqa: F811
    """scale log2(e) is what the kernels work with: 0 times an infinite one would be NaN."""
    call = lambda scale: lib.coreinfer_paged_attention(cache(), P, 2, P, 256, 4, scale, 0, 0, P, 256, None, 0, None)  # noqa: E731
    for scale in (2.4e38, -2.4e38, 3.4e38):
        assert call(scale) == ci.ERR_INVALID_ARG
    for scale in (2.3e38, -2.3e38, 1e-45, 0.0):
        assert call(scale) == ci.ERR_WORKSPACE


def test_a_workspace_that_grows_leaves_the_one_before_alone():
    """Calls captured before hold its address: it stays allocated, and check() looks at it too."""
    import weakref

    from paper_2410_18311_b200.pipeline import PagedKVCache, Pages
    pages = Pages(1, 8, 16, 64, device="cpu")
    one = PagedKVCache(pages, 4, 2, 64)
    before, size = weakref.ref(one.ws), one.ws.numel()
    q = torch.zeros(500, 4, 64, dtype=torch.bfloat16)
    for _ in range(2):
        with pytest.raises(ci.CoreInferError):                   # host tensors: no call is made
            one.attend(q, torch.zeros_like(q))
        assert before() is not None and before().numel() == size
        assert one.ws.numel() >= ci.coreinfer_paged_attention_workspace_bytes(one.cache, 4, 500) > size
    grown = one.ws.data_ptr()
    with pytest.raises(ci.CoreInferError):
        one.attend(q[:1], torch.zeros_like(q[:1]))
    assert one.ws.data_ptr() == grown
    looked = []
    status, ci.binding.coreinfer_workspace_status = ci.binding.coreinfer_workspace_status, lambda ws, stream=None: looked.append(ws.data_ptr())
    try:
        one.check()
    finally:
        ci.binding.coreinfer_workspace_status = status
    assert set(looked) == {before().data_ptr(), grown}
    assert (before()[:4] == 0).all() and (one.ws[:4] == 0).all()     # neither has been written by a call


def pages_of(batch=3, n_pages=12, size=16, most=64):
    from paper_2410_18311_b200.pipeline import Pages
    return Pages(batch, n_pages, size, most, device="cpu")


def test_a_sequence_that_has_ended_sits_out_the_steps():
    """Lengths on the device and counts on the host stay 0 from release() to the next add(), whose prompt then begins at position 0."""
    pages = pages_of()
    pages.add([20, 5, 9])
    pages.reserve(40)
    pages.decoding()
    for _ in range(3):
        pages.one_more()
    pages.counted(3)
    pages.release(1)
    for _ in range(4):
        pages.one_more()
    pages.counted(4)
    assert pages.length.tolist() == pages.tokens == [27, 0, 16]
    assert pages.add([1, 7, 1]) == 9
    assert pages.length.tolist() == pages.tokens == [28, 7, 17]
    assert [len(h) for h in pages.held] == [3, 1, 3] and (pages.table[1, 1:] == -1).all()
    pages.one_more()
    pages.counted(1)
    assert pages.length.tolist() == pages.tokens == [29, 8, 18]


def test_a_sequence_not_begun_sits_out_and_a_batch_may_begin_with_steps():
    pages = pages_of()
    pages.add([20, 0, 9])
    pages.reserve(40)
    pages.one_more()
    pages.counted(1)
    assert pages.length.tolist() == pages.tokens == [21, 0, 10]
    pages = pages_of()
    pages.reserve(16)
    pages.decoding()
    for _ in range(16):
        pages.one_more()
    pages.counted(16)
    assert pages.length.tolist() == pages.tokens == [16, 16, 16]


@pytest.mark.parametrize("new", [[1], [1, 2], [1, 2, 3, 4], [3, -1, 1], [-20, 0, 0], 5, [1.5, 0, 0], []])
def test_pages_refuse_numbers_that_are_not_one_per_sequence(new):
    pages = pages_of()
    pages.add([20, 0, 9])
    state = lambda: ([list(h) for h in pages.held], list(pages.free), pages.tokens, pages.length.tolist(), pages.start.tolist(),  # noqa: E731
                     pages.table.tolist(), pages.runs)
    before = state()
    with pytest.raises(ci.CoreInferError):
        pages.add(new)
    assert state() == before
    if new != 5:                                                 # a number is one for all there
        with pytest.raises(ci.CoreInferError):
            pages.reserve(new)
    assert state() == before


@pytest.mark.parametrize("b", [-1, 3, 1.0])
def test_pages_refuse_to_release_what_is_no_sequence(b):
    pages = pages_of()
    pages.add([20, 3, 9])
    with pytest.raises(ci.CoreInferError):
        pages.release(b)
    assert pages.tokens == [20, 3, 9] and len(pages.free) == 12 - 4


def test_steps_behind_the_reserved_pages_are_told():
    """counted() raises where steps had no pages for their tokens; what is held stays usable."""
    pages = pages_of()
    pages.add([20, 16, 9])
    pages.decoding()
    pages.reserve([32, 20, 0])
    for _ in range(16):
        pages.one_more()
    with pytest.raises(ci.CoreInferError):
        pages.counted(16)
    assert pages.tokens == pages.length.tolist() == [32, 32, 16]
    pages.release(0)
    pages.one_more()
    with pytest.raises(ci.CoreInferError):
        pages.counted(1)
    assert pages.tokens == pages.length.tolist() == [0, 32, 16]
    with pytest.raises(ci.CoreInferError):
        pages.counted(-1)
    assert pages.add([1, 2, 3]) == 6 and pages.tokens == pages.length.tolist() == [1, 34, 19]
