"""Weights of the norms of queries and keys: whether they are each head's own or shared is what their shapes say, and a flag that says otherwise is refused before
anything is launched (shared weights taken for the heads' own would be read, and their gradients written, behind their end)."""
import pytest
import torch

from paper_2501_09767_amd import lemo


def test_the_flag_is_refused_with_shared_weights():
    Q, K = torch.ones(3, 4, 64), torch.ones(3, 2, 64)
    w, w_q, w_k = torch.ones(64), torch.ones(4, 64), torch.ones(2, 64)
    for weights in ((w, None), (None, w), (w, w)):
        for flags in (lemo.WEIGHTS_PER_HEAD, lemo.WEIGHTS_PER_HEAD | lemo.ROTATE_PAIRS):
            with pytest.raises(ValueError, match="WEIGHTS_PER_HEAD"):
                lemo._rotate_sizes(Q, K, None, lemo.NORM_RMS, *weights, flags)
    # what the shapes say needs no flag, and may have it; without weights it says nothing
    for weights, flags, want in (((w, w), 0, 0), ((w_q, w_k), 0, 2), ((w_q, w_k), 2, 2), ((w_q, None), 3, 3), ((None, None), 2, 2), ((w, None), 1, 1)):
        assert lemo._rotate_sizes(Q, K, None, lemo.NORM_RMS, *weights, flags)[-1] == want


class Refusing:
    """In the place of the native module: always the long way."""
    def __getattr__(self, name):
        return lambda *a: None


@pytest.mark.gpu
@pytest.mark.parametrize("way", ["native", "python"])
def test_all_calls_refuse_it_either_way(monkeypatch, way):
    if way == "python":
        monkeypatch.setattr(lemo, "_native", Refusing())
    M, H, Hkv, d = 5, 4, 2, 64
    Q, K, cache = torch.randn(M, H, d, device="cuda"), torch.randn(M, Hkv, d, device="cuda"), torch.randn(M, 7, Hkv, d, device="cuda")
    f, w, lengths = torch.rand(16, device="cuda"), torch.rand(d, device="cuda"), torch.arange(M, device="cuda", dtype=torch.int32)
    kept = cache.clone()
    for weights in (dict(w_q=w, w_k=w), dict(w_q=w), dict(w_k=w)):
        for call in (lambda **kw: lemo.lemo_qk_rotate(Q, K, f, **kw), lambda **kw: lemo.lemo_qk_rotate_grad(Q, K, Q, K, f, **kw),
                     lambda **kw: lemo.lemo_qk_rotate_step(Q, K, None, cache, None, lengths, f, **kw)):
            with pytest.raises(ValueError, match="WEIGHTS_PER_HEAD"):
                call(flags=lemo.WEIGHTS_PER_HEAD, **weights)
    assert torch.equal(cache, kept)
    # the heads' own, with the flag: as without it
    own = dict(w_q=w.expand(H, d).contiguous(), w_k=w.expand(Hkv, d).contiguous())
    for a, b, c in zip(lemo.lemo_qk_rotate(Q, K, f, flags=lemo.WEIGHTS_PER_HEAD, **own), lemo.lemo_qk_rotate(Q, K, f, **own), lemo.lemo_qk_rotate(Q, K, f, w_q=w, w_k=w)):
        assert torch.equal(a, b) and torch.equal(a, c)
