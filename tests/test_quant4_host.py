"""Refusals of the 4-bit operators: arguments are checked on the host before any CUDA call."""
import ctypes

import pytest
import torch

import paper_2410_18311_b200 as ci
from paper_2410_18311_b200 import _build

NULL = None
BUF = (ctypes.c_char * 4096)()
P = (ctypes.addressof(BUF) + 63) & ~63


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return ci.binding.load()


def matrix(**kw):
    f = dict(codes=P, pairs=P, N=32, K=64, group=32)
    f.update(kw)
    return ci.binding.W4Matrix(f["codes"], f["pairs"], f["N"], f["K"], f["group"], 0)


def cache(**kw):
    f = dict(k_codes=P, k_pairs=P, v_codes=P, v_pairs=P, state=P, weight=P, position=P, batch=2, kv_heads=2, capacity=32, head_dim=64, group=32)
    f.update(kw)
    return ci.binding.KV4Cache(*(f[n] for n, _ in ci.binding.KV4Cache._fields_[:-1]), 0)


def test_sizes(lib):
    assert ci.coreinfer_w4_codes_bytes(17, 129) == 2 * 2 * 1024 and ci.coreinfer_w4_pairs_bytes(17, 129, 32) == 2 * 2 * 4 * 64
    assert ci.coreinfer_w4_codes_bytes(0, 5) == 0 and ci.coreinfer_w4_pairs_bytes(16, 128, 48) == 0
    assert ci.coreinfer_w4_codes_bytes(1 << 20, 1 << 20) == 1 << 39
    assert ci.coreinfer_kv4_evict_workspace_bytes(cache()) >= 2 * 2 * 32 * 4 and ci.coreinfer_kv4_evict_workspace_bytes(cache(head_dim=96)) == 0
    assert ci.coreinfer_kv4_attention_workspace_bytes(cache(), 4, 1) > 0
    for heads, T in ((3, 1), (0, 1), (4, 0), (4, 17)):
        assert ci.coreinfer_kv4_attention_workspace_bytes(cache(), heads, T) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(group=48), "UNSUPPORTED"), (dict(dtype=5), "UNSUPPORTED"), (dict(N=0), "INVALID_ARG"), (dict(K=0), "INVALID_ARG"),
    (dict(w=NULL), "INVALID_ARG"), (dict(w=P + 2), "INVALID_ARG"), (dict(codes=P + 8), "INVALID_ARG"), (dict(pairs=NULL), "INVALID_ARG"),
    (dict(N=16 * 65536), "UNSUPPORTED")])
def test_quantize_refuses(lib, kw, status):
    f = dict(w=P, dtype=ci.F32, N=8, K=8, sn=8, sk=1, group=32, codes=P, pairs=P)
    f.update(kw)
    assert lib.coreinfer_w4_quantize(*f.values(), NULL) == getattr(ci, "ERR_" + status)


@pytest.mark.parametrize("kw,status", [
    (dict(w=NULL), "INVALID_ARG"), (dict(w=matrix(group=16)), "UNSUPPORTED"), (dict(w=matrix(N=0)), "INVALID_ARG"),
    (dict(w=matrix(codes=None)), "INVALID_ARG"), (dict(w=matrix(pairs=P + 4)), "INVALID_ARG"), (dict(x=NULL), "INVALID_ARG"),
    (dict(x=P + 1), "INVALID_ARG"), (dict(batch=0), "UNSUPPORTED"), (dict(batch=9), "UNSUPPORTED"), (dict(ld_x=63), "INVALID_ARG"),
    (dict(dtype=7), "UNSUPPORTED"), (dict(y_dtype=ci.F16), "UNSUPPORTED"), (dict(act=3), "UNSUPPORTED"), (dict(y=NULL), "INVALID_ARG"),
    (dict(ld_y=31), "INVALID_ARG"), (dict(mul=P, ld_mul=8), "INVALID_ARG"), (dict(bias=P + 1), "INVALID_ARG"), (dict(y=P + 2), "INVALID_ARG")])
def test_matvec_refuses(lib, kw, status):
    f = dict(w=matrix(), x=P, batch=2, ld_x=64, dtype=ci.BF16, act=0, bias=NULL, mul=NULL, ld_mul=0, y=P, y_dtype=ci.F32, ld_y=32)
    f.update(kw)
    assert lib.coreinfer_w4_matvec(*f.values(), NULL) == getattr(ci, "ERR_" + status)
    assert lib.coreinfer_last_error()


BAD_CACHES = [(dict(head_dim=96), "UNSUPPORTED"), (dict(group=128), "UNSUPPORTED"), (dict(capacity=40), "INVALID_ARG"), (dict(capacity=0), "INVALID_ARG"),
              (dict(batch=0), "INVALID_ARG"), (dict(batch=1025), "UNSUPPORTED"), (dict(k_codes=None), "INVALID_ARG"), (dict(v_pairs=P + 4), "INVALID_ARG"),
              (dict(state=None), "INVALID_ARG"), (dict(weight=None), "INVALID_ARG"), (dict(kv_heads=1025), "UNSUPPORTED")]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_bad_caches_are_refused_everywhere(lib, kw, status):
    want, c = getattr(ci, "ERR_" + status), cache(**kw)
    assert lib.coreinfer_kv4_append(c, P, P, ci.BF16, 1, 128, NULL, NULL, NULL) == want
    assert lib.coreinfer_kv4_attention(c, P, ci.BF16, 2, 1, 128, 1.0, P, 128, 0, P, 1 << 30, NULL) == want
    assert lib.coreinfer_kv4_evict(c, c, 8, 0, 0, P, 1 << 30, NULL) == want
    assert lib.coreinfer_kv4_append(NULL, P, P, ci.BF16, 1, 128, NULL, NULL, NULL) == ci.ERR_INVALID_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=9), "UNSUPPORTED"), (dict(T=0), "INVALID_ARG"), (dict(k=NULL), "INVALID_ARG"), (dict(v=P + 8), "INVALID_ARG"),
    (dict(ld=120), "INVALID_ARG"), (dict(ld=132), "INVALID_ARG"), (dict(ks=P), "INVALID_ARG"), (dict(T=1 << 30), "UNSUPPORTED")])
def test_append_refuses(lib, kw, status):
    f = dict(c=cache(), k=P, v=P, dtype=ci.BF16, T=1, ld=128, ks=NULL, vs=NULL)
    f.update(kw)
    assert lib.coreinfer_kv4_append(*f.values(), NULL) == getattr(ci, "ERR_" + status)


@pytest.mark.parametrize("kw,status", [
    (dict(q=NULL), "INVALID_ARG"), (dict(out=P + 2), "INVALID_ARG"), (dict(dtype=3), "UNSUPPORTED"), (dict(heads=3), "INVALID_ARG"),
    (dict(heads=0), "INVALID_ARG"), (dict(T=0), "UNSUPPORTED"), (dict(T=17), "UNSUPPORTED"), (dict(ld_q=248), "INVALID_ARG"),
    (dict(ld_out=260), "INVALID_ARG"), (dict(scale=float("nan")), "INVALID_ARG"), (dict(scale=float("inf")), "INVALID_ARG"),
    (dict(c=cache(weight=None, position=None), acc=1), "INVALID_ARG"), (dict(ws=NULL), "WORKSPACE"), (dict(n=16), "WORKSPACE")])
def test_attention_refuses(lib, kw, status):
    f = dict(c=cache(), q=P, dtype=ci.BF16, heads=4, T=1, ld_q=256, scale=0.125, out=P, ld_out=256, acc=0, ws=P, n=1 << 30)
    f.update(kw)
    assert lib.coreinfer_kv4_attention(*f.values(), NULL) == getattr(ci, "ERR_" + status)


@pytest.mark.parametrize("kw,status", [
    (dict(budget=0), "INVALID_ARG"), (dict(recent=-1), "INVALID_ARG"), (dict(recent=6, first=3), "INVALID_ARG"), (dict(first=-2), "INVALID_ARG"),
    (dict(recent=2 ** 31 - 1, first=2 ** 31 - 1), "INVALID_ARG"), (dict(dst=cache(k_codes=P + 64)), "INVALID_ARG"),
    (dict(dst=cache(head_dim=128)), "INVALID_ARG"), (dict(src=cache(weight=None, position=None)), "INVALID_ARG"),
    (dict(ws=NULL), "WORKSPACE"), (dict(n=8), "WORKSPACE")])
def test_evict_refuses(lib, kw, status):
    f = dict(src=cache(), dst=cache(), budget=8, recent=0, first=0, ws=P, n=1 << 30)
    f.update(kw)
    assert lib.coreinfer_kv4_evict(*f.values(), NULL) == getattr(ci, "ERR_" + status)
    small = cache(capacity=16, **{n: P + 64 * (i + 1) for i, n in enumerate(("k_codes", "k_pairs", "v_codes", "v_pairs", "state", "weight", "position"))})
    assert lib.coreinfer_kv4_evict(cache(), small, 17, 0, 0, P, 1 << 30, NULL) == ci.ERR_INVALID_ARG


def test_binding_checks_shapes():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    w = matrix()
    for x, y in ((z(2, 63), z(2, 32)), (z(2, 64), z(2, 31)), (z(2, 128)[:, ::2], z(2, 32))):
        with pytest.raises(ci.CoreInferError):
            ci.coreinfer_w4_matvec(w, x, ci.ACT_NONE, None, None, y)
    with pytest.raises(ci.CoreInferError):
        ci.make_w4_matrix(z(10, dtype=torch.uint8), z(4096, dtype=torch.float16), 32, 64, 32)
    u8, f16, i32 = torch.uint8, torch.float16, torch.int32
    good = [z(2, 2, 32, 32, dtype=u8), z(2, 2, 32, 2, 2, dtype=f16), z(2, 2, 32, 32, dtype=u8), z(2, 2, 32, 2, 2, dtype=f16), z(2, 4, dtype=i32)]
    c = ci.make_kv4_cache(*good)
    assert (c.batch, c.kv_heads, c.capacity, c.head_dim, c.group) == (2, 2, 32, 64, 32)
    with pytest.raises(ci.CoreInferError):
        ci.make_kv4_cache(*good[:4], z(2, 3, dtype=i32))
    with pytest.raises(ci.CoreInferError):
        ci.coreinfer_kv4_append(c, z(2, 1, 2, 64), z(2, 1, 2, 64).transpose(1, 2).reshape(2, 1, 2, 64)[:, :, :, :32])
    with pytest.raises(ci.CoreInferError):
        ci.coreinfer_kv4_append(c, z(2, 3, 3, 64)[:, :, :2].transpose(0, 1), z(2, 3, 3, 64)[:, :, :2].transpose(0, 1))


def test_attention_workspace_does_not_shrink_with_more_tokens(lib):
    """One workspace of the size asked for at the most tokens serves every shorter call."""
    for B in (1, 2, 8, 64):
        for H in (1, 4, 12, 32):
            for share in (1, 2, 3, 5, 7, 8, 16, 40):
                for D, group, capacity in ((64, 32, 16), (128, 64, 32), (128, 32, 1024), (256, 32, 9008)):
                    c = cache(batch=B, kv_heads=H, capacity=capacity, head_dim=D, group=group)
                    sizes = [ci.coreinfer_kv4_attention_workspace_bytes(c, H * share, T) for T in range(1, 17)]
                    assert sizes[0] > 0 and sizes == sorted(sizes), (B, H, share, D, group, capacity)


@pytest.mark.parametrize("q_heads,kv_heads", [(4, 4), (128, 1), (129, 1), (200, 1), (512, 2), (2048, 1)])
def test_cache_object_has_room_for_every_call(lib, q_heads, kv_heads):
    """Above 128 query heads per key head the limit on rows, and not the 16 tokens, bounds a call."""
    from paper_2410_18311_b200.pipeline import KV4Cache
    c = KV4Cache(1, q_heads, kv_heads, 32, 64, 32, device="cpu")
    assert c.max_tokens == max(T for T in range(1, 17) if T * q_heads // kv_heads <= ci.KV4_MAX_ROWS)
    for T in range(1, c.max_tokens + 1):
        assert 0 < ci.coreinfer_kv4_attention_workspace_bytes(c.cache, q_heads, T) <= c.ws.numel()


def test_quantize_binding_checks_its_buffers(lib):
    """The kernel writes as many bytes as the sizes say: smaller or strided buffers are refused before it starts."""
    w = torch.zeros(33, 200)
    codes, pairs = (torch.zeros(n, dtype=torch.uint8) for n in (ci.coreinfer_w4_codes_bytes(33, 200), ci.coreinfer_w4_pairs_bytes(33, 200, 64)))
    for c, p in ((codes[:-1], pairs), (codes, pairs[:-2]), (torch.zeros(0, dtype=torch.uint8), pairs)):
        with pytest.raises(ci.CoreInferError, match="smaller"):
            ci.coreinfer_w4_quantize(w, 64, c, p)
    with pytest.raises(ci.CoreInferError, match="contiguous"):
        ci.coreinfer_w4_quantize(w, 64, torch.zeros(2 * codes.numel(), dtype=torch.uint8)[::2], pairs)
    with pytest.raises(ci.CoreInferError, match="matrix"):
        ci.coreinfer_w4_quantize(w[0], 64, codes, pairs)
    with pytest.raises(ci.CoreInferError, match="host"):
        ci.coreinfer_w4_quantize(w, 64, codes, pairs)
    with pytest.raises(ci.CoreInferError, match="q_heads"):
        ci.coreinfer_kv4_attention(cache(), torch.zeros(2, 4, 64), 1.0, torch.zeros(2, 4, 64), False, codes)
