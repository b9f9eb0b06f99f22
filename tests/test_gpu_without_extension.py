"""Contexts, caches and the calls through ctypes work where the argument extension has not been built."""
import pytest
import torch

from paper_2609_33184_b200 import binding as ssb
from paper_2609_33184_b200 import build as ssbuild


@pytest.fixture
def without(monkeypatch):
    ssbuild.build()

    def missing():
        raise RuntimeError("_marshal.so not found")
    monkeypatch.setattr(ssb, "marshal", missing)


def test_caches(without):
    for kind in (ssb.Cache8, ssb.Cache16):
        cache = kind.empty(4, 2, 16, 64, torch.zeros(2, 2, dtype=torch.int32), device="cpu")
        assert cache.requests == 2 and cache.ref is not None
        with pytest.raises(RuntimeError):
            cache.known


@pytest.mark.gpu
def test_older_calls(without):
    dev = "cuda:0"
    g = torch.Generator().manual_seed(0)
    rnd = lambda *s: torch.randn(s, generator=g).bfloat16().to(dev)
    K, V, Q = rnd(1, 2, 5, 64), rnd(1, 2, 5, 64), rnd(1, 4, 1, 64)
    cache = ssb.Cache8.empty(1, 2, 16, 64)
    ctx = ssb.Context(1, 4, 2, 64, 1, 1, 16)
    n = torch.tensor([5], dtype=torch.int32, device=dev)
    O, LSE, Kr, Vr = torch.empty_like(Q), torch.empty(1, 4, 1, device=dev), torch.empty_like(K), torch.empty_like(V)
    ctx.ss_kv8_write(cache, K, V)
    ctx.ss_kv8_read(cache, Kr, Vr)
    ctx.ss_decode8(Q, 0.125, cache, n, O, LSE)
    ctx.ss_verify_begin(Q, 0.125)
    ctx.ss_verify_chunk8(cache, n)
    ctx.ss_verify_finalize(O, LSE)
    assert ctx.ss_poll_status() == (0, 0) and torch.isfinite(LSE).all() and (Kr != 0).any()
    with pytest.raises(RuntimeError):
        ctx.ss_rope_rotate(ssb.Rope([1.0] * 32), Q, None, Q, None)
    ctx.close()
