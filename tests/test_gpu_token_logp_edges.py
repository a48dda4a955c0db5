"""Token log probabilities where a wait runs out on workspaces that hold anything, and beside NaN."""
import pytest
import torch

import paper_2609_14306_b200 as vp
from test_gpu_token_logp import F8, IGN, bf16_grid, fp8_grid, outputs, run, run8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,d,V,top", [(4, 1024, 3000, 4), (40, 1024, 3000, 0), (100, 1024, 3000, 20), (300, 1024, 3000, 0), (5000, 512, 20000, 20)])
def test_a_lost_copy_on_a_workspace_of_arbitrary_bytes(T, d, V, top, fp8):
    """Nothing that the workspace held is taken for a state or a count of candidates: no results, and the next call starts clean.
    (5000 tokens: two chunks of two strips or more.)"""
    ops, _, tokens = fp8_grid(T, d, V, seed=1)
    H, W, _ = bf16_grid(T, d, V, seed=1)
    args = ops if fp8 else (H, W)
    call = vp.vp_token_logp_fp8_forward if fp8 else vp.vp_token_logp_forward
    n = (vp.vp_token_logp_fp8_workspace_bytes if fp8 else vp.vp_token_logp_workspace_bytes)(T, d, V, top)

    def workspace():                                        # as counts: 1061109567
        ws = torch.full((n + 4096,), 0x3f, dtype=torch.uint8, device="cuda")
        return ws, ws[:n]

    want = outputs(T, top)
    call(*args, tokens, 1.0, IGN, *want, workspace()[1])
    before = vp.vp_ce_set_wait_limit_ns(20_000_000)
    try:
        whole, ws = workspace()
        got = outputs(T, top)
        vp.vp_token_logp_debug_drop(2)
        call(*args, tokens, 1.0, IGN, *got, ws)
        assert vp.vp_ce_device_status(ws) & 2
    finally:
        vp.vp_ce_set_wait_limit_ns(before)
        vp.vp_token_logp_debug_drop(-1)
    logp, lse, entropy, top_logp, top_ids = got
    assert torch.isnan(lse).all() and torch.isnan(entropy).all()
    assert torch.isnan(logp[tokens != IGN]).all() and (logp[tokens == IGN] == 0).all()
    if top:
        assert (top_ids == -1).all() and (top_logp == -float("inf")).all()
    assert (whole[n:] == 0x3f).all()
    again = outputs(T, top)
    call(*args, tokens, 1.0, IGN, *again, ws)
    assert vp.vp_ce_device_status(ws) == 0
    assert all(a is None or torch.equal(a, b) for a, b in zip(want, again))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,V,top", [(7, 128, 5), (65, 128, 5), (300, 128, 20), (200, 256, 5), (1000, 1000, 8)])
def test_alternatives_beside_columns_of_nan(T, V, top, fp8):
    """A NaN is not an alternative and takes no other column's place: four neighbours of NaN (all that one bound looks at) at every
    place, and single ones.  Ids are the definition's, the sums being exact."""
    (hq, hs, wq, ws), (full_h, full_w), tokens = fp8_grid(T, 128, V, seed=T + V)
    H, W, _ = bf16_grid(T, 128, V, seed=T + V)
    x = full_h @ full_w.mT if fp8 else H.double() @ W.double().mT
    for first in (0, 28, 64, 124):
        gone = torch.zeros(V, dtype=torch.bool, device="cuda")
        gone[first:first + 4] = True
        gone[::17] = True
        if fp8:
            bad = wq.view(torch.uint8).clone()
            bad[gone, 3] = 0x7f
            _, lse, _, top_logp, top_ids = run8((hq, hs, bad.view(F8), ws), tokens, top)
        else:
            bad = W.clone()
            bad[gone, 3] = float("nan")
            _, lse, _, top_logp, top_ids = run(H, bad, tokens, top)
        want = torch.sort(x.masked_fill(gone, -float("inf")), dim=1, descending=True, stable=True)[1][:, :top]
        assert torch.equal(top_ids.long(), want)
        assert torch.isnan(lse).all() and torch.isnan(top_logp).all()
