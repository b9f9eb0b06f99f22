"""Whole rounds over the 8-bit cache on the GPU: captured ones, more rows than one row tile holds, the CUDA-core kernel,
tree masks; each against one fp64 softmax over everything that a row sees."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv8 import DEV, _gen, _ssb, check_attention, history, make_cache, poison

pytestmark = pytest.mark.gpu


def f64(t, b, n=None):
    return t[b, :, :n].double().cpu().numpy()


def check_round(Q, O, LSE, pieces, near, rows):
    """pieces(b): the history's K, V pieces in fp64; near(b, i): those of the local segment that query i sees."""
    for i in rows:
        def kv(b):
            parts = list(pieces(b)) + [near(b, i)]
            return [np.concatenate([p[k] for p in parts], 1) for k in (0, 1)]
        check_attention(Q[:, :, i:i + 1], O[:, :, i:i + 1], LSE[:, :, i:i + 1], kv, Q.shape[3] ** -0.5)


def test_captured_round_follows_lengths_and_pages():
    """One captured round replayed while the requests grow, shrink and empty, bit for bit as the calls give it."""
    ssb = _ssb()
    for flags in (0, ssb.SS_FLAG_OVERLAP_CHUNKS):
        B, H_q, H_kv, d, T, page = 3, 8, 2, 128, 4, 16
        cache = make_cache(ssb, B, H_kv, d, page, 2000, 8)
        ctx = ssb.Context(B, H_q, H_kv, d, T, T, 2048, flags=flags)
        g = _gen(2)
        Q = torch.zeros(B, H_q, T, d, dtype=torch.bfloat16, device=DEV)
        Kl, Vl = (torch.zeros(B, H_kv, T, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        O, LSE = torch.empty_like(Q), torch.empty(B, H_q, T, device=DEV)
        n = torch.zeros(B, dtype=torch.int32, device=DEV)

        def step():
            ctx.ss_verify_begin(Q, d ** -0.5)
            ctx.ss_verify_chunk8(cache, n)
            ctx.ss_verify_local(Kl, Vl)
            ctx.ss_verify_finalize(O, LSE)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for lens in ([1, 1, 1], [1500, 2, 1999], [64, 700, 128], [0, 0, 0], [0, 1, 129], [2000, 1025, 1023]):
            for t in (Q, Kl, Vl):
                t.copy_(torch.randn(t.shape, generator=g).bfloat16())
            cache.tensors[4].copy_(cache.tensors[4][[1, 2, 0]].clone())
            n.copy_(torch.tensor(lens, dtype=torch.int32))
            graph.replay()
            torch.cuda.synchronize()
            assert ctx.ss_poll_status() == (0, 0)
            check_round(Q, O, LSE, lambda b: [history(cache, b, lens[b])], lambda b, i: (f64(Kl, b, i + 1), f64(Vl, b, i + 1)),
                        (0, T - 1))
            got = O.clone(), LSE.clone()
            step()
            torch.cuda.synchronize()
            assert torch.equal(got[0].view(torch.int16), O.view(torch.int16)) and torch.equal(got[1], LSE)
        del graph
        ctx.close()


@pytest.mark.parametrize("joined", [False, True], ids=["straight", "joined"])
@pytest.mark.parametrize("G,T", [(1, 2), (5, 8), (8, 8), (3, 33), (5, 64)])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (128, 24), (64, 0)])
def test_rounds_with_any_number_of_rows(d, page, G, T, joined):
    """One row tile and several, straight from the pieces to the output and joined into a partial state before a merge
    with a bf16 chunk; 24-token pages take the CUDA cores."""
    ssb = _ssb()
    B, H_kv, lens = 3, 2, [2500, 0, 131]
    H_q = G * H_kv
    cache = make_cache(ssb, B, H_kv, d, page, 2520, 5 * G + T)
    poison(cache, lens)
    g = _gen(G)
    rnd = lambda *s: torch.randn(s, generator=g).bfloat16().to(DEV)
    Q, Kl, Vl, K, V = rnd(B, H_q, T, d), rnd(B, H_kv, T, d), rnd(B, H_kv, T, d), rnd(B, H_kv, 192, d), rnd(B, H_kv, 192, d)
    vl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ctx = ssb.Context(B, H_q, H_kv, d, T, T, 4096)
    outs = []
    for _ in range(2):
        O, LSE = torch.empty_like(Q), torch.empty(B, H_q, T, device=DEV)
        ctx.ss_verify_begin(Q, d ** -0.5)
        ctx.ss_verify_chunk8(cache, vl)
        assert ctx.last_chunk_kernel() == ("kv8-simt" if page == 24 else "kv8-tcgen05")
        if joined:
            ctx.ss_verify_chunk(K, V)
        ctx.ss_verify_local(Kl, Vl)
        ctx.ss_verify_finalize(O, LSE)
        assert ctx.ss_poll_status() == (0, 0)
        outs.append((O, LSE))
    assert torch.equal(outs[0][0].view(torch.int16), outs[1][0].view(torch.int16)) and torch.equal(outs[0][1], outs[1][1])
    pieces = lambda b: [history(cache, b, lens[b])] + ([(f64(K, b), f64(V, b))] if joined else [])
    check_round(Q, O, LSE, pieces, lambda b, i: (f64(Kl, b, i + 1), f64(Vl, b, i + 1)), sorted({0, T // 2, T - 1}))
    ctx.close()


@pytest.mark.parametrize("joined", [False, True], ids=["straight", "joined"])
@pytest.mark.parametrize("lens", [[900, 0, 140], [0, 0, 0]], ids=["history", "no_history"])
def test_tree_masks_beside_an_8_bit_history(lens, joined):
    """Every node sees its path; one row sees no local token at all, with no history nothing: O = 0 and LSE = -inf."""
    ssb = _ssb()
    B, H_q, H_kv, d, T = 3, 8, 2, 128, 7
    cache = make_cache(ssb, B, H_kv, d, 16, 912, 3)
    poison(cache, lens)
    parent = [-1, 0, 0, 1, 1, 2, 4]
    path = [{i} if p < 0 else set() for i, p in enumerate(parent)]
    for i in range(1, T):
        path[i] = path[parent[i]] | {i}
    path[5] = set()
    words = torch.tensor([sum(1 << j for j in s) for s in path], dtype=torch.int64)
    bits = words.view(1, T, 1).repeat(B, 1, 1).contiguous().to(DEV)
    g = _gen(4)
    rnd = lambda *s: torch.randn(s, generator=g).bfloat16().to(DEV)
    Q, Kl, Vl = rnd(B, H_q, T, d), rnd(B, H_kv, T, d), rnd(B, H_kv, T, d)
    vl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    none = torch.zeros(B, dtype=torch.int32, device=DEV)
    O, LSE = torch.empty_like(Q), torch.empty(B, H_q, T, device=DEV)
    ctx = ssb.Context(B, H_q, H_kv, d, T, T, 1024)
    ctx.ss_verify_begin(Q, d ** -0.5)
    if joined:
        ctx.ss_verify_chunk8(cache, none)     # a chunk without a visible token
    ctx.ss_verify_chunk8(cache, vl)
    ctx.ss_verify_local(Kl, Vl, ssb.SS_MASK_TREE_BITS, bits)
    ctx.ss_verify_finalize(O, LSE)
    assert ctx.ss_poll_status() == (0, 0)
    see = [sorted(s) for s in path]
    check_round(Q, O, LSE, lambda b: [history(cache, b, lens[b])], lambda b, i: (f64(Kl, b)[:, see[i]], f64(Vl, b)[:, see[i]]), range(T))
    ctx.close()
