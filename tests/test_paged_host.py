"""Rotary positions and the paged cache: what the library and its binding refuse, and the frequency tables (no GPU needed)."""
import ctypes
import math

import pytest
import torch

import paper_2410_18311_b200 as ci
from paper_2410_18311_b200 import _build
from paper_2410_18311_b200.binding import PagedCache, Rope


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return ci.binding.load()


NULL = ctypes.c_void_p(None)
BUF = (ctypes.c_char * 4096)()
P = (ctypes.addressof(BUF) + 255) // 256 * 256


def cache(**kw):
    c = dict(k=P, v=P, table=P, length=P, page_stride=2 * 16 * 64, head_stride=16 * 64, token_stride=64, dtype=ci.BF16, n_pages=4, page_size=16,
             kv_heads=2, head_dim=64, batch=3, max_pages=2, reserved=0)
    c.update(kw)
    return PagedCache(**c)


def rope(**kw):
    r = dict(turns=P, q_norm=None, k_norm=None, eps=1e-6, magnitude=1.0, rot_dim=64, interleaved=0)
    r.update(kw)
    return Rope(**r)


def test_frequencies(lib):
    from paged_ref import frequencies
    for kind, code in (("plain", ci.ROPE_PLAIN), ("linear", ci.ROPE_LINEAR), ("ntk", ci.ROPE_NTK), ("yarn", ci.ROPE_YARN), ("bands", ci.ROPE_BANDS)):
        for rot in (16, 48, 128, 256):
            for base, factor, context in ((10000.0, 4.0, 2048), (500000.0, 1.0, 8192), (1e6, 40.0, 32768)):
                f, m = frequencies(rot, base, kind, factor, context)
                turns, got = ci.coreinfer_rope_frequencies(rot, base, code, factor, context)
                assert got == pytest.approx(m, rel=1e-6)
                for t, x in zip(turns.tolist(), f.tolist()):
                    assert abs(t / 2.0 ** 64 - x / (2 * math.pi)) <= 4e-16 * rot + 2.0 ** -63


@pytest.mark.parametrize("bad,status", [
    (dict(rot_dim=24), "UNSUPPORTED"), (dict(rot_dim=0), "UNSUPPORTED"), (dict(rot_dim=272), "UNSUPPORTED"), (dict(base=1.0), "INVALID_ARG"),
    (dict(base=math.nan), "INVALID_ARG"), (dict(scaling=5), "UNSUPPORTED"), (dict(scaling=1, factor=0.5), "INVALID_ARG"),
    (dict(scaling=3, factor=2.0), "INVALID_ARG"), (dict(scaling=4, factor=2.0, original_context=10, low=4.0, high=4.0), "INVALID_ARG"),
    (dict(scaling=4, factor=math.inf, original_context=10), "INVALID_ARG"),
])
def test_frequencies_refused(lib, bad, status):
    args = dict(rot_dim=64, base=10000.0)
    args.update(bad)
    with pytest.raises(ci.CoreInferError) as e:
        ci.coreinfer_rope_frequencies(**args)
    assert e.value.status == getattr(ci, "ERR_" + status)


def test_rope_apply_refused(lib):
    call = lambda r=None, pos=P, dtype=ci.BF16, tokens=2, hq=2, h=1, D=64, q=P, lq=128, k=P, lk=64, qo=P, lqo=128, ko=P, lko=64: lib.coreinfer_rope_apply(
        r if r is not None else rope(), pos, dtype, tokens, hq, h, D, q, lq, k, lk, qo, lqo, ko, lko, None)
    bad, no = ci.ERR_INVALID_ARG, ci.ERR_UNSUPPORTED
    assert lib.coreinfer_rope_apply(None, P, ci.BF16, 1, 1, 1, 64, P, 64, P, 64, P, 64, P, 64, None) == bad
    for want, kw in ((bad, dict(pos=None)), (no, dict(dtype=5)), (no, dict(D=96)), (bad, dict(tokens=0)), (bad, dict(hq=0, h=0)), (bad, dict(q=None)),
                     (bad, dict(q=P + 8)), (bad, dict(lq=120)), (bad, dict(lk=68)), (bad, dict(ko=None)), (bad, dict(lqo=64)), (no, dict(hq=5000, lq=5000 * 64, lqo=5000 * 64)),
                     (no, dict(tokens=1 << 29)), (no, dict(r=rope(rot_dim=80))), (no, dict(r=rope(rot_dim=24))), (bad, dict(r=rope(turns=None))),
                     (bad, dict(r=rope(q_norm=P + 2))), (bad, dict(r=rope(eps=-1.0))), (bad, dict(r=rope(eps=math.nan))), (bad, dict(hq=-1))):
        assert call(**kw) == want, kw


BAD_CACHES = [
    ("UNSUPPORTED", dict(dtype=3)), ("UNSUPPORTED", dict(head_dim=96)), ("UNSUPPORTED", dict(page_size=8)), ("UNSUPPORTED", dict(page_size=48)),
    ("UNSUPPORTED", dict(page_size=512)), ("INVALID_ARG", dict(batch=0)), ("UNSUPPORTED", dict(batch=1025)), ("INVALID_ARG", dict(n_pages=0)),
    ("INVALID_ARG", dict(max_pages=0)), ("UNSUPPORTED", dict(max_pages=1 << 26)), ("UNSUPPORTED", dict(kv_heads=1025)), ("INVALID_ARG", dict(k=None)),
    ("INVALID_ARG", dict(v=P + 2)), ("INVALID_ARG", dict(table=None)), ("INVALID_ARG", dict(length=P + 1)), ("INVALID_ARG", dict(token_stride=56)),
    ("INVALID_ARG", dict(token_stride=68)), ("INVALID_ARG", dict(page_stride=1024)), ("INVALID_ARG", dict(head_stride=64)), ("INVALID_ARG", dict(head_stride=-1024)),
    ("UNSUPPORTED", dict(page_stride=1 << 39)), ("UNSUPPORTED", dict(n_pages=1 << 27)),
]


@pytest.mark.parametrize("status,bad", BAD_CACHES)
def test_caches_refused(lib, status, bad):
    want = getattr(ci, "ERR_" + status)
    c = cache(**bad)
    assert lib.coreinfer_paged_append(c, P, 2, P, 128, P, 128, None, None, None, 0, 0, None, 0, None) == want
    assert lib.coreinfer_paged_attention(c, P, 2, P, 256, 4, 0.1, 0, 0, P, 256, P, 1 << 40, None) == want
    assert lib.coreinfer_paged_attention_workspace_bytes(c, 4, 2) == 0


def test_append_refused(lib):
    bad, no = ci.ERR_INVALID_ARG, ci.ERR_UNSUPPORTED
    call = lambda c=None, start=P, tokens=2, k=P, lk=128, v=P, lv=128, r=None, pos=None, q=None, lq=0, hq=0, qo=None, lqo=0: lib.coreinfer_paged_append(
        c or cache(), start, tokens, k, lk, v, lv, r, pos, q, lq, hq, qo, lqo, None)
    assert lib.coreinfer_paged_append(None, P, 2, P, 128, P, 128, None, None, None, 0, 0, None, 0, None) == bad
    for want, kw in ((bad, dict(start=None)), (bad, dict(tokens=0)), (bad, dict(k=None)), (bad, dict(v=P + 8)), (bad, dict(lk=64)), (bad, dict(lv=132)),
                     (bad, dict(q=P, lq=128, hq=2, qo=P, lqo=128)), (bad, dict(r=rope(), q=P, lq=128, hq=2)), (bad, dict(r=rope(), hq=2)),
                     (bad, dict(r=rope(), q=P, lq=128, hq=0, qo=P, lqo=128)), (bad, dict(r=rope(), q=P, lq=64, hq=2, qo=P, lqo=128)),
                     (no, dict(r=rope(rot_dim=128))), (bad, dict(pos=P + 2)), (no, dict(tokens=1 << 28))):
        assert call(**kw) == want, kw


def test_attention_refused(lib):
    bad, no = ci.ERR_INVALID_ARG, ci.ERR_UNSUPPORTED
    call = lambda c=None, start=P, tokens=2, q=P, lq=256, hq=4, scale=0.1, window=0, sinks=0, out=P, lo=256, ws=P, n=1 << 40: lib.coreinfer_paged_attention(
        c or cache(), start, tokens, q, lq, hq, scale, window, sinks, out, lo, ws, n, None)
    for want, kw in ((bad, dict(start=None)), (bad, dict(tokens=0)), (bad, dict(q=None)), (bad, dict(out=P + 8)), (bad, dict(lq=128)), (bad, dict(lo=260)),
                     (bad, dict(hq=3)), (bad, dict(hq=0)), (no, dict(hq=4098, lq=4098 * 64, lo=4098 * 64)), (bad, dict(window=-1)), (bad, dict(sinks=-1)),
                     (no, dict(window=(1 << 30) + 1)), (bad, dict(scale=math.inf)), (bad, dict(scale=math.nan)), (no, dict(tokens=1 << 28)),
                     (ci.ERR_WORKSPACE, dict(ws=None)), (ci.ERR_WORKSPACE, dict(ws=P + 8)), (ci.ERR_WORKSPACE, dict(n=64))):
        assert call(**kw) == want, kw
    assert lib.coreinfer_paged_attention_workspace_bytes(cache(), 3, 2) == 0
    assert lib.coreinfer_paged_attention_workspace_bytes(cache(), 4, 0) == 0
    sizes = [lib.coreinfer_paged_attention_workspace_bytes(cache(), 4, n) for n in (1, 2, 5, 17, 100, 1000, 100000)]
    assert all(0 < a <= b for a, b in zip(sizes, sizes[1:]))


def test_binding_refuses():
    """Shapes, types and host tensors, before anything reaches the library."""
    pool, table, length = torch.zeros(4, 2, 16, 64), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for args in ((pool, pool[:, :1], table, length), (pool, pool.half(), table, length), (pool, pool, table.long(), length), (pool, pool, table, length[:2]),
                 (pool, pool.transpose(2, 3), table, length), (pool[0], pool[0], table, length)):
        with pytest.raises(ci.CoreInferError):
            ci.make_paged_cache(*args)
    c = ci.make_paged_cache(pool, pool, table, length)
    start, q = torch.zeros(4, dtype=torch.int32), torch.zeros(5, 4, 64)
    kv = torch.zeros(5, 2, 64)
    ws = torch.zeros(64, dtype=torch.uint8)
    for call in (lambda: ci.coreinfer_paged_append(c, start, kv, kv),            # a host tensor
                 lambda: ci.coreinfer_paged_append(c, start[:3], kv, kv), lambda: ci.coreinfer_paged_append(c, start.long(), kv, kv),
                 lambda: ci.coreinfer_paged_append(c, start, kv.half(), kv.half()), lambda: ci.coreinfer_paged_append(c, start, kv[:, :1], kv),
                 lambda: ci.coreinfer_paged_append(c, start, kv, kv[:4]), lambda: ci.coreinfer_paged_append(c, start, kv, kv, None, None, q),
                 lambda: ci.coreinfer_paged_append(c, start, kv.transpose(1, 2).contiguous().transpose(1, 2), kv),
                 lambda: ci.coreinfer_paged_attention(c, start, q, 0.1, q, ws), lambda: ci.coreinfer_paged_attention(c, start, q[0], 0.1, q, ws),
                 lambda: ci.coreinfer_paged_attention(c, start, q, 0.1, q[:4], ws), lambda: ci.coreinfer_paged_attention(c, start, q.half(), 0.1, q, ws)):
        with pytest.raises(ci.CoreInferError):
            call()
    turns, m = ci.coreinfer_rope_frequencies(64)
    for args in ((turns.float(),), (turns, False, m, torch.ones(64), torch.ones(32)), (turns, False, m, torch.ones(64), torch.ones(64).half())):
        with pytest.raises(ci.CoreInferError):
            ci.make_rope(*args)
    r = ci.make_rope(turns, False, m, torch.ones(32))
    at = torch.zeros(5, dtype=torch.int32)
    for call in (lambda: ci.coreinfer_rope_apply(r, at, q, None, q, None), lambda: ci.coreinfer_rope_apply(ci.make_rope(turns), at, q, None, q, None),
                 lambda: ci.coreinfer_rope_apply(r, at, None, None, None, None), lambda: ci.coreinfer_rope_apply(r, at, q, None, None, None),
                 lambda: ci.coreinfer_rope_apply(r, at, q.double(), None, q.double(), None), lambda: ci.coreinfer_rope_apply(r, at, q, kv[:4], q, kv[:4])):
        with pytest.raises(ci.CoreInferError):
            call()
