"""Policy and preference loss at the edges of what the C entries accept, where the paths of small and large calls meet, and
where the terms are small differences of large numbers.  Oracle and helpers are those of test_gpu_sequence_loss."""
import numpy as np
import pytest
import torch

import paper_2609_14306_b200 as vp

pytestmark = pytest.mark.gpu


def library():
    vp.vp_policy_loss_workspace_bytes(0, 0)                              # binds the signatures
    return vp.load_library()


def stream():
    return torch.cuda.current_stream().cuda_stream


# ------------------------------------------------------------------------------------------------ calls without sequences
@pytest.mark.parametrize("T", [0, 1, 300, 8192, 8193])
def test_no_sequences_and_null_offsets(T):
    """n_seqs == 0 needs no offsets: statistics and gradients are 0 in the one-launch and the three-launch path."""
    lib = library()
    x = torch.randn(max(T, 1), device="cuda")
    d = torch.full((T + 8,), 9.0, device="cuda")
    s4, s3 = torch.full((4,), 9.0, device="cuda"), torch.full((3,), 9.0, device="cuda")
    ws = torch.full((vp.vp_policy_loss_workspace_bytes(T, 0),), 255, dtype=torch.uint8, device="cuda")
    for per_token in (0, 1):
        for aggregate in (0, 1):
            d.fill_(9.0), s4.fill_(9.0)
            args = (x.data_ptr(), x.data_ptr(), x.data_ptr(), x.data_ptr() if per_token else None, per_token, None, None, T, 0, 0.2,
                    0.2, 0.1, aggregate)
            assert lib.vp_policy_loss(*args, s4.data_ptr(), d.data_ptr(), None, ws.data_ptr(), ws.numel(), stream()) == 0
            torch.cuda.synchronize()
            assert not s4.any() and not d[:T].any() and (d[T:] == 9).all()
            d.fill_(9.0)
            assert lib.vp_policy_loss_backward(*args, d.data_ptr(), None, ws.data_ptr(), ws.numel(), stream()) == 0
            torch.cuda.synchronize()
            assert not d[:T].any() and (d[T:] == 9).all()
    for kind in (0, 1):
        d.fill_(9.0), s3.fill_(9.0)
        assert lib.vp_preference_loss(x.data_ptr(), None, None, None, T, 0, 0.1, 0.0, 0.0, kind, 0, s3.data_ptr(), None, d.data_ptr(), None,
                                      ws.data_ptr(), ws.numel(), stream()) == 0
        torch.cuda.synchronize()
        assert not s3.any() and not d[:T].any() and (d[T:] == 9).all()


# ------------------------------------------------------------------------------------------------ sequences without tokens
@pytest.mark.parametrize("n", [2, 1024, 1026, 5000])
def test_sequences_but_no_tokens(n):
    """T == 0 with few and with many sequences: every sequence is empty.  The policy loss is 0; the preference loss is the loss
    of D = 0, exactly (one fp32 rounding of log 2 and its like)."""
    f = torch.empty(0, device="cuda")
    off = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    adv = torch.randn(n, device="cuda")
    for aggregate in ("token_mean", "seq_mean"):
        stats = torch.full((4,), 9.0, device="cuda")
        ws = torch.full((vp.vp_policy_loss_workspace_bytes(0, n),), 255, dtype=torch.uint8, device="cuda")
        vp.vp_policy_loss(f, f, f, adv, None, off, 0.2, 0.2, 0.1, aggregate, stats, f.clone(), ws, adv_per_token=False)
        vp.vp_policy_loss_backward(f, f, f, adv, None, off, 0.2, 0.2, 0.1, aggregate, f.clone(), ws, adv_per_token=False)
        assert not stats.any()
    for kind, loss in (("sigmoid", np.log(2.0)), ("ipo", 25.0)):
        stats, rewards = torch.full((3,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
        ws = torch.full((vp.vp_preference_loss_workspace_bytes(0, n // 2),), 255, dtype=torch.uint8, device="cuda")
        vp.vp_preference_loss(f, None, None, off, 0.1, 0.0, 0.0, kind, True, stats, rewards, f.clone(), ws)
        vp.vp_preference_loss_backward(None, off, f.clone(), ws)
        got = stats.cpu().numpy()
        assert abs(got[0] - loss) <= 2.0 ** -22 * loss and got[1] == 0 and got[2] == 0
        assert not rewards.any()
