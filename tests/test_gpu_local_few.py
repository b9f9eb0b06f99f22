"""The local segment's kernel for up to 8 keys against the one for more: the same bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _state(ssb, ctx, Q, K, V, words, d):
    B, H_q, T, _ = Q.shape
    ml, a = torch.full((B * H_q * T, 2), 7.0, device=DEV), torch.full((B * H_q * T, d), 7.0, device=DEV)
    ctx.ss_verify_begin(Q, d ** -0.5)
    if words is None:
        ctx.ss_verify_local(K, V)
    else:
        ctx.ss_verify_local(K, V, ssb.SS_MASK_TREE_BITS, words)
    ctx.ss_verify_export_state(ml, a)
    ctx.ss_verify_abort()
    torch.cuda.synchronize()
    return ml, a


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,T_loc", [(1, 1), (2, 2), (5, 5), (8, 8), (3, 7), (13, 6), (40, 8)])
@pytest.mark.parametrize("G", [1, 4, 5])
@pytest.mark.parametrize("strided", [False, True])
def test_few_local_keys(d, T, T_loc, G, strided):
    """A tree over T_loc keys; the other kernel gets a ninth and tenth key that nobody sees, NaN."""
    from paper_2609_33184_b200 import binding as ssb
    B, H_kv = 3, 2
    g = torch.Generator().manual_seed(T * 100 + T_loc + G)
    rnd = lambda H, n: (torch.randn(B, n, H, d, generator=g).bfloat16().to(DEV).transpose(1, 2) if strided
                        else torch.randn(B, H, n, d, generator=g).bfloat16().to(DEV))
    Q, K, V = rnd(H_kv * G, T), rnd(H_kv, T_loc), rnd(H_kv, T_loc)
    K[0, 0, 0] *= 40.0
    words = torch.randint(0, 1 << T_loc, (B, T, 1), generator=g, dtype=torch.int64)
    words[1, 0] = 0                                            # a row that sees nothing
    hidden = T_loc - 1
    words &= ~(1 << hidden) if T_loc > 1 else -1               # nobody sees the last key, which is NaN
    if T_loc > 1:
        K[:, :, hidden], V[:, :, hidden] = float("nan"), float("nan")
    words = words.to(DEV)
    nan = torch.full((B, H_kv, 10, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    K10, V10 = nan.clone(), nan.clone()
    K10[:, :, :T_loc], V10[:, :, :T_loc] = K, V
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, 10, 8)
    few, many = _state(ssb, ctx, Q, K, V, words, d), _state(ssb, ctx, Q, K10, V10, words, d)
    live = few[0][:, 1] != 0
    assert torch.equal(few[0], many[0]) and torch.equal(few[1][live], many[1][live])
    assert not torch.isnan(few[1][live]).any()
    if T_loc >= T and T_loc > 1:                               # the chain rule as tree words
        K, V = torch.nan_to_num(K), torch.nan_to_num(V)
        K10[:, :, :T_loc], V10[:, :, :T_loc] = K, V
        chain = torch.tensor([(1 << (i + T_loc - T + 1)) - 1 for i in range(T)], dtype=torch.int64).view(1, T, 1).repeat(B, 1, 1)
        few, many = _state(ssb, ctx, Q, K, V, None, d), _state(ssb, ctx, Q, K10, V10, chain.to(DEV), d)
        assert torch.equal(few[0], many[0]) and torch.equal(few[1], many[1])
    ctx.close()
