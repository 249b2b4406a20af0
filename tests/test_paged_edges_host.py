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
