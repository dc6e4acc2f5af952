"""Results of lemo_norm_residual_grad that the caller gives, in the place of operands too, and sums that are not asked for: by the native
marshalling and by the steps in Python."""
import pytest
import torch

from test_native_binding_layer import Refusing
from test_norm_residual import inputs


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def given(lemo, dtype, gate, post, nxt, C=264):
    t = {k: v.cuda() if v is not None else None for k, v in inputs(dtype, 33, 70, C, post, nxt, gate, "dropped", seed=post + 3 * nxt).items()}
    how = dict(gate=t["gate"], post=post, next=nxt, w_post=t["w_post"], b_post=t["b_post"], w_next=t["w_next"], residual_scale=0.6, block_scale=0.4,
               flags=lemo.GATE_SIGMOID if gate == "sigmoid" else 0)
    R = t["R"].clone()
    _, stats = lemo.lemo_norm_residual(t["Y"], R, t["idx"], b_next=t["b_next"], **how)
    return t, R, stats, how


CASES = [(torch.bfloat16, "rows", 1, 2), (torch.bfloat16, "sigmoid", 0, 1), (torch.float32, "row", 2, 1), (torch.float32, "none", 1, 0), (torch.bfloat16, "rows", 0, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("n", range(len(CASES)))
def test_given_results_and_sums_that_are_not_asked_for(lemo, monkeypatch, n, native):
    dtype, gate, post, nxt = CASES[n]
    t, R, stats, how = given(lemo, dtype, gate, post, nxt)
    M, C = t["Y"].shape
    calls, real = [], lemo._native

    class Watching:
        def __getattr__(self, name):
            def f(*a):
                calls.append(getattr(real, name)(*a))
                return calls[-1]
            return f

    monkeypatch.setattr(lemo, "_native", Watching() if native else Refusing())
    dR = t["dR"].clone()
    want = lemo.lemo_norm_residual_grad(t["dN"], dR, R, t["Y"], t["idx"], stats, **how)
    # with frozen weights: the same without the sums
    dR1 = t["dR"].clone()
    got = lemo.lemo_norm_residual_grad(t["dN"], dR1, R, t["Y"], t["idx"], stats, weights=False, **how)
    assert torch.equal(dR, dR1) and got.dw_post is got.db_post is got.dw_next is got.db_next is None
    assert torch.equal(got.dY, want.dY) and (got.dgate is None) == (gate == "none") and (gate == "none" or torch.equal(got.dgate, want.dgate))
    # dY in the place of dN, inside a larger tensor; dgate in the place of the gate, or the sums' own place
    wide = torch.full((M, C + 24), 9.0, dtype=dtype, device="cuda")
    dN = wide[:, :C]
    dN.copy_(t["dN"])
    dR2, dg = t["dR"].clone(), None
    if gate in ("rows", "sigmoid"):
        how["gate"] = dg = how["gate"].clone()
    elif gate == "row":
        dg = torch.full((C,), 9.0, device="cuda")
    got = lemo.lemo_norm_residual_grad(dN, dR2, R, t["Y"], t["idx"], stats, dY=dN, dgate=dg, **how)
    assert got.dY.data_ptr() == wide.data_ptr() and (wide[:, C:] == 9).all() and (dg is None or got.dgate.data_ptr() == dg.data_ptr())
    assert torch.equal(dR, dR2) and all((x is None) == (y is None) and (x is None or torch.equal(x, y)) for x, y in zip(got, want))
    assert not native or (len(calls) == 3 and all(c[0] == 0 for c in calls))


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_results_that_do_not_fit(lemo, monkeypatch, native):
    t, R, stats, how = given(lemo, torch.bfloat16, "rows", 1, 2)
    if not native:
        monkeypatch.setattr(lemo, "_native", Refusing())
    dR = t["dR"].clone()

    def refused(error=ValueError, Y=t["Y"], **kw):
        with pytest.raises(error):
            lemo.lemo_norm_residual_grad(t["dN"], dR, R, Y, t["idx"], stats, **{**how, **kw})

    refused(dY=t["dN"][:5])
    refused(dY=t["dN"].float())
    refused(dY=t["dN"].cpu())
    refused(dgate=t["gate"][:, :64])
    refused(dgate=torch.zeros(t["gate"].shape[1], device="cuda"))
    refused(dgate=t["gate"], gate=None)
    refused(dgate=t["gate"], gate=t["gate"][0])
    refused(dgate=torch.zeros(t["gate"].shape[1], dtype=torch.bfloat16, device="cuda"), gate=t["gate"][0])
    refused(Y=None, dY=t["dN"], gate=None, post=0, w_post=None)
    refused(lemo.LemoError, dY=torch.empty(33, 268, dtype=torch.bfloat16, device="cuda")[:, :264])  # rows that are not at multiples of 16 bytes
    assert torch.equal(dR, t["dR"])
