"""The windowed calls and the binding's argument checks without a GPU."""
import pytest
import torch

from paper_2609_33184_b200 import binding as ssb
from paper_2609_33184_b200 import build as ssbuild


@pytest.fixture(scope="module", autouse=True)
def lib():
    ssbuild.build()
    return ssb.load()


def test_calls_without_a_context_or_cache_are_refused(lib):
    no = ssb.ss_tensor(None, 0, 0, 0)
    for name in ("ss_decode_window", "ss_decode8_window"):
        assert getattr(lib, name)(None, no, 1, 1, 1.0, None, 1, 0, None, None, None, None) == ssb.SS_ERR_ARG
    for name in ("ss_verify_chunk_window", "ss_verify_chunk8_window"):
        assert getattr(lib, name)(None, None, 1, 0, None, None, None) == ssb.SS_ERR_ARG


@pytest.fixture
def call():
    """A context that is none (no handle: every call that passes the checks comes back as SS_ERR_ARG), on the CPU."""
    m = ssb.marshal()
    me = m.context(None, -1, 4, 2, 64)
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    pool, table = z(6, 2, 16, 64), torch.zeros(3, 2, dtype=torch.int32)
    return m, me, z, ssb.Cache16(pool, pool.clone(), table), ssb.Cache8.empty(6, 2, 16, 64, table, device="cpu")


def test_what_fits_gets_through(call):
    m, me, z, c16, c8 = call
    Q, K = z(3, 4, 5, 64), z(3, 2, 5, 64)
    n = torch.zeros(3, dtype=torch.int32)
    pos, idx = torch.zeros(2, 3, 5, dtype=torch.int32), torch.zeros(3, 5, dtype=torch.int32)
    rope = ssb.Rope([1.0] * 32, [0, 1] * 16, 2)
    O, LSE = z(3, 4, 5, 64), torch.zeros(3, 4, 5)
    strided = z(3, 5, 4, 72)[..., :64].transpose(1, 2)         # [B, H, T, d] in another order, padded
    for c, append, decode, chunk in ((c16, m.kv_append, m.decode_window, m.verify_chunk_window),
                                     (c8, m.kv8_append, m.decode8_window, m.verify_chunk8_window)):
        assert append(me, c.known, K, K, rope.at, pos, strided, Q, n, n, None, 0) == ssb.SS_ERR_ARG
        assert append(me, c.known, K, K, None, None, None, None, n, n, idx, 0) == ssb.SS_ERR_ARG
        assert decode(me, strided, 0.5, c.known, 2 ** 31 - 1, 0, n, O, LSE, None) == ssb.SS_ERR_ARG
        assert decode(me, Q, 1, c.known, 1, 0, None, O, None, 0) == ssb.SS_ERR_ARG
        assert chunk(me, c.known, 1, 0, n, idx, 3, 5, 0) == ssb.SS_ERR_ARG
    assert m.rope_rotate(me, rope.at, Q, None, Q, None, pos, n, n, 0) == ssb.SS_ERR_ARG
    assert m.rope_rotate(me, rope.at, None, K, None, K, None, n, n, 0) == ssb.SS_ERR_ARG


def test_what_does_not_fit_is_refused(call):
    m, me, z, c16, c8 = call
    Q, K = z(3, 4, 5, 64), z(3, 2, 5, 64)
    n, pos, idx = torch.zeros(3, dtype=torch.int32), torch.zeros(1, 3, 5, dtype=torch.int32), torch.zeros(3, 5, dtype=torch.int32)
    rope = ssb.Rope([1.0] * 32).at
    O, LSE = z(3, 4, 5, 64), torch.zeros(3, 4, 5)
    bad = [
        lambda: m.kv_append(me, c8.known, K, K, rope, pos, Q, Q, n, n, None, 0),            # a cache of the other kind
        lambda: m.kv8_append(me, c16.known, K, K, rope, pos, Q, Q, n, n, None, 0),
        lambda: m.kv_append(me, None, K, K, rope, pos, Q, Q, n, n, None, 0),
        lambda: m.kv_append(me, c16.known, Q, K, rope, pos, None, None, n, n, None, 0),     # heads
        lambda: m.kv_append(me, c16.known, K, z(3, 2, 4, 64), rope, pos, None, None, n, n, None, 0),
        lambda: m.kv_append(me, c16.known, z(4, 2, 5, 64), z(4, 2, 5, 64), rope, None, None, None, None, None, None, 0),  # more requests than the table
        lambda: m.kv_append(me, c16.known, K.float(), K, rope, pos, None, None, n, n, None, 0),
        lambda: m.kv_append(me, c16.known, z(3, 2, 5, 128)[..., ::2], K, rope, pos, None, None, n, n, None, 0),
        lambda: m.kv_append(me, c16.known, K[0], K, rope, pos, None, None, n, n, None, 0),
        lambda: m.kv_append(me, c16.known, K, K, rope, idx[:, :4], None, None, n, n, None, 0),
        lambda: m.kv_append(me, c16.known, K, K, rope, pos.long(), None, None, n, n, None, 0),
        lambda: m.kv_append(me, c16.known, K, K, rope, pos, None, None, n[:2], n, None, 0),
        lambda: m.kv_append(me, c16.known, K, K, rope, pos, None, None, n, n, idx.t(), 0),
        lambda: m.kv_append(me, c16.known, K, K, rope, pos, None, Q, n, n, None, 0),        # rows out without rows in
        lambda: m.kv_append(me, c16.known, K, K, rope, pos, Q, None, n, n, None, 0),
        lambda: m.kv_append(None, c16.known, K, K, rope, pos, None, None, n, n, None, 0),   # a closed context
        lambda: m.decode_window(me, Q, 1.0, c16.known, 1, 0, n, O[:, :, :4], LSE, 0),
        lambda: m.decode_window(me, Q, 1.0, c16.known, 1, 0, n, O.transpose(1, 2), LSE, 0),
        lambda: m.decode_window(me, Q, 1.0, c16.known, 1, 0, n, O, LSE.half(), 0),
        lambda: m.decode_window(me, Q, 1.0, c16.known, 1, 0, n, None, LSE, 0),
        lambda: m.verify_chunk_window(me, c16.known, 1, 0, n, idx, 3, 4, 0),
        lambda: m.rope_rotate(me, rope, None, None, None, None, None, None, None, 0),
        lambda: m.rope_rotate(me, rope, Q, z(3, 2, 4, 64), Q, z(3, 2, 4, 64), None, None, None, 0),
    ]
    for f in bad:
        with pytest.raises(AssertionError):
            f()
    for f in (lambda: m.decode_window(me), lambda: m.decode_window(me, Q, "x", c16.known, 1, 0, n, O, LSE, 0),
              lambda: m.decode_window(me, Q, 1.0, c16.known, 1.5, 0, n, O, LSE, 0), lambda: m.context(1)):
        with pytest.raises(TypeError):
            f()
    with pytest.raises(OverflowError):
        m.decode_window(me, Q, 1.0, c16.known, 2 ** 31, 0, n, O, LSE, 0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32, torch.int16])
def test_a_cache_of_another_type_is_refused(dtype):
    good = torch.zeros(2, 1, 8, 64, dtype=torch.bfloat16)
    bad = torch.zeros(2, 1, 8, 64, dtype=dtype)
    for K, V in ((bad, good), (good, bad), (good, good[:1]), (good.transpose(2, 3), good.transpose(2, 3))):
        with pytest.raises(AssertionError):
            ssb.Cache16(K, V)
    with pytest.raises(AssertionError):
        ssb.Cache16(good, good, torch.zeros(2, 1))


def test_an_empty_cache():
    table = torch.zeros(2, 3, dtype=torch.int32)
    cache = ssb.Cache16.empty(6, 2, 16, 64, table, device="cpu")
    assert [t.shape for t in cache.tensors] == [(6, 2, 16, 64), (6, 2, 16, 64), (2, 3)] and cache.requests == 2
    assert all(t.dtype is torch.bfloat16 and not t.any() for t in cache.tensors[:2])
    assert cache.tensors[0].data_ptr() != cache.tensors[1].data_ptr()
    assert ssb.Cache16.empty(3, 2, 16, 64, device="cpu").requests == 3


def test_a_tensor_without_strides_is_refused(call):
    m, me, z, c16, _ = call
    Q, K, n = z(3, 4, 5, 64), z(3, 2, 5, 64), torch.zeros(3, dtype=torch.int32)
    nested = torch.nested.nested_tensor([K[0], K[1], K[2]])
    wide = z(64).as_strided((3, 2, 2 ** 32 + 1, 64), (0, 0, 0, 1))  # more rows than a call takes
    for bad in (K.to_sparse(), nested, wide):
        for f in (lambda: m.kv_append(me, c16.known, bad, K, None, None, None, None, None, None, None, 0),
                  lambda: m.kv_append(me, c16.known, K, bad, None, None, None, None, None, None, None, 0),
                  lambda: m.decode_window(me, bad, 1.0, c16.known, 1, 0, n, Q, None, 0),
                  lambda: m.decode_window(me, Q, 1.0, c16.known, 1, 0, n.to_sparse(), Q, None, 0),
                  lambda: m.decode_window(me, Q, 1.0, c16.known, 1, 0, n, Q.to_sparse(), None, 0)):
            with pytest.raises(AssertionError):
                f()
