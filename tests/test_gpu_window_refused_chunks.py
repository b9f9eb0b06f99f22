"""A chunk that is refused enqueues nothing, also where the round's sets are full and the next chunk would fold them."""
import pytest
import torch

from tests.test_gpu_window import _gen, _i32, queries

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_refused_window_leaves_the_round_as_it_was():
    from paper_2609_33184_b200 import binding as ssb
    T, room = 40, 2 ** 31 - 16384 - 64                         # room and queries together pass 31 bits: refused
    g = _gen(1)
    far = ssb.Cache16.empty(1, 1, 64, 64, torch.zeros(1, room // 64, dtype=torch.int32, device=DEV))
    near = ssb.Cache16.empty(1, 1, 256, 64)
    for x in near.tensors[:2]:
        x.copy_(torch.randn(x.shape, generator=g))
    near8 = ssb.Cache8.empty(1, 1, 256, 64)
    K, V, Q = queries(g, 1, 1, 30, 64), queries(g, 1, 1, 30, 64), queries(g, 1, 1, T, 64)
    ctx = ssb.Context(1, 1, 1, 64, T, T, room, max_chunks=2)
    out = []
    for refused in (False, True):
        O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
        ctx.ss_verify_begin(Q, 0.125)
        ctx.ss_verify_chunk(K, V)
        ctx.ss_verify_chunk8(near8, _i32([9]))                 # (its pieces would be joined too)
        if refused:
            before = ctx.launch_count()
            with pytest.raises(ssb.SpecStreamError) as e:
                ctx.ss_verify_chunk_window(far, 100, 0, _i32([7]))
            assert e.value.status == ssb.SS_ERR_SHAPE and ctx.launch_count() == before
        ctx.ss_verify_chunk_window(near, 70, 3, _i32([200]))
        ctx.ss_verify_finalize(O, LSE)
        assert ctx.ss_poll_status() == (0, 0)
        out.append((O, LSE))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    ctx.close()
