"""Calls that need more threads than a launch holds, 2^32 (what is beyond is left out without an error): rows and lists are taken in turns.  What comes out is compared with calls on a few
rows or sequences at both ends and around the places where a turn may end."""
import pytest
import torch


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def ranges(n, places):
    yield 0, 8
    for p in places:
        yield p - 8, p + 8
    yield n - 8, n


@pytest.mark.gpu
def test_norm_of_more_than_2_26_rows(lemo):
    """Four rows a workgroup: 2^24 workgroups of 256 threads and some."""
    M, C = 2 ** 26 + 701, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    Y, R = (torch.randn(M, C, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    w = torch.randn(C, generator=g, device="cuda", dtype=torch.bfloat16)
    before = {a: R[a:z].clone() for a, z in ranges(M, (2 ** 25, 2 ** 26))}
    N, stats = lemo.lemo_norm_residual(Y, R, post=2, next=1, w_next=w, residual_scale=0.5, block_scale=0.25)
    for a, z in ranges(M, (2 ** 25, 2 ** 26)):
        r = before[a]
        n, s = lemo.lemo_norm_residual(Y[a:z], r, post=2, next=1, w_next=w, residual_scale=0.5, block_scale=0.25)
        assert torch.equal(R[a:z], r) and torch.equal(N[a:z], n) and torch.equal(stats[a:z], s), a


@pytest.mark.gpu
def test_single_tokens_of_more_than_2_24_lists(lemo):
    """A workgroup of 256 threads a list.  All sequences share one cache (a sequence stride of 0)."""
    B, H, d, b, S, T = 2 ** 19 + 9, 32, 64, 32, 96, 2
    g = torch.Generator(device="cuda").manual_seed(2)
    Q = torch.randn(B, H, d, generator=g, device="cuda", dtype=torch.bfloat16)
    means = torch.randn(B, 3, H, d, generator=g, device="cuda")
    K, V = (torch.randn(1, S, H, d, generator=g, device="cuda", dtype=torch.bfloat16).expand(B, S, H, d) for _ in range(2))
    lengths = torch.randint(0, S + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    blocks = lemo.lemo_select_blocks_step(Q, means, lengths, b, T, S_max=S)
    O = lemo.lemo_block_attention_step(Q, K, V, lengths, blocks, b)
    for a, z in ranges(B, (2 ** 18, 2 ** 19)):
        few = lemo.lemo_select_blocks_step(Q[a:z], means[a:z], lengths[a:z], b, T, S_max=S)
        assert torch.equal(blocks[a:z], few), a
        # (few sequences share a list out to several workgroups: the order of their sums differs; each result is off by two roundings of 2^-8)
        o = lemo.lemo_block_attention_step(Q[a:z], K[a:z], V[a:z], lengths[a:z], few, b)
        assert (O[a:z].float() - o.float()).abs().max() <= 2.0 ** -6 * V.abs().max(), a
        assert not O[a:z][lengths[a:z] == 0].any()
    means_now = means[:, :, :1].contiguous()
    del means
    one = torch.randn(1, S, 1, d, generator=g, device="cuda", dtype=torch.bfloat16)
    lemo.lemo_block_means_step(one.expand(B, S, 1, d), torch.full_like(lengths, 64), b, means_now)
    assert (means_now[:, 1] == lemo.lemo_block_means(one[0, 32:64], b)).all()


@pytest.mark.gpu
def test_means_of_more_than_2_24_blocks(lemo):
    """Keys that overlap in memory, 8 elements apart."""
    S, b, d = 2 ** 29 + 65, 32, 64
    flat = torch.randn(S * 8 + 64, device="cuda", dtype=torch.bfloat16)
    K = flat.as_strided((S, 1, d), (8, d, 1))
    means = lemo.lemo_block_means(K, b)
    assert means.shape[0] == 2 ** 24 + 3
    for a, z in ranges(2 ** 24 + 3, (2 ** 22, 2 ** 23, 2 ** 24)):
        assert torch.equal(means[a:z], lemo.lemo_block_means(K[a * b:min(z * b, S)], b)), a

@pytest.mark.gpu
@pytest.mark.parametrize("mode", [0, 1])
def test_scatter_of_more_than_2_24_rows(lemo, mode):
    M, C = 2 ** 24 + 41, 8
    S = M + 1000
    g = torch.Generator(device="cuda").manual_seed(4)
    G, dX = (torch.randn(n, C, generator=g, device="cuda", dtype=torch.bfloat16) for n in (M, S))
    idx = torch.randperm(S, generator=g, device="cuda")[:M].sort().values.int()
    want = dX.float() if mode == 0 else torch.zeros(S, C, device="cuda")
    want[idx.long()] += G.float()
    lemo.lemo_scatter_grad(G, idx, dX, mode)
    assert torch.equal(dX, want.bfloat16())


@pytest.mark.gpu
def test_choice_from_more_segments_than_a_launch_holds_workgroups(lemo):
    """Segments of two tokens, one of them kept: 256 threads a segment, 1024 where the mean over the heads is taken as well."""
    for n in (2 ** 24 + 5, 2 ** 22 + 5):
        S = 2 * n
        scores = torch.randn(S, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda")
        pairs = scores.view(n, 2)
        want = (pairs[:, 1] > pairs[:, 0]).int() + torch.arange(n, device="cuda", dtype=torch.int32) * 2
        assert torch.equal(lemo.lemo_select_topk(scores, 2, 1), want)
    got, kept = lemo.lemo_head_mean_select_topk(scores.view(1, S), torch.zeros(1, S, device="cuda"), 2, 1)
    assert torch.equal(got, scores) and torch.equal(kept, want)


@pytest.mark.gpu
def test_choice_from_nearly_2_31_scores(lemo):
    """The last segment ends where 32-bit sums of a length and a segment do not."""
    S, L, k = 2 ** 31 - 1, 32768, 16
    scores = torch.zeros(S, device="cuda")
    n = 2 ** 16
    mark = torch.arange(n, device="cuda") * L + torch.arange(n, device="cuda") % 16384
    scores[mark] = 1.0
    kept = lemo.lemo_select_topk(scores, L, k)
    want = torch.arange(n, device="cuda")[:, None] * L + torch.arange(k, device="cuda")  # the first of equal scores, but for the marked one
    want[:, -1] = torch.where(mark % L >= k, mark, want[:, -1])
    assert kept.numel() == n * k and torch.equal(kept.view(n, k).long(), want)


@pytest.mark.gpu
def test_weight_gradient_of_no_rows_and_2_24_outputs(lemo):
    N, C = 2 ** 24 + 4, 4
    dW = torch.ones(N, C, device="cuda")
    empty = torch.empty(0, N, device="cuda"), torch.empty(5, C, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    lemo.lemo_gather_gemm_dw(*empty, dW=dW)
    assert not dW.any()


def test_more_key_heads_than_a_launch_has_rows_of_workgroups():
    """On the host alone."""
    from paper_2501_09767_amd import lemo
    P = 0x100000
    assert lemo._lib.lemo_block_means(P, 100, 65536, 64, 1, 0, 64, 32, P, None) == -6
    assert lemo._lib.lemo_select_blocks(P, 100, 65536, 65536, 64, 1, 64, 64, P, 100, 0, 32, 16, 4, 1, P, None) == -6
    assert lemo._lib.lemo_block_attention_grad(P, P, P, P, P, P, 32, 32, 65536, 65536, 64, 1, 64, 0, 64, 0, 64, 0, 64, 0, 64, 0, P, 1, 32, 32, 0, 0.0, 1, P, P, P, P,
                                               1 << 62, None) == -6
