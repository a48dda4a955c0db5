"""The give-up path of Muon's bounded waits, exercised without any invalid access.

The library's test hook makes one signal of one launch "get lost" (copies that are not issued, a product whose end is not
signalled): a wait runs out, the kernel ends what it has in flight, frees its tensor memory and returns, and the status word
says so.  The tests check that the call returns promptly, what its outputs hold, and that the next call on the same workspace
is right."""
import time

import pytest
import torch

import paper_2609_14306_b200 as vp

pytestmark = pytest.mark.gpu

WAIT_EXPIRED = 2
LIMIT_NS = 2_000_000          # 2 ms; the default is 2 s


def state(batch, rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    p, m, g = (torch.randn(batch, rows, cols, generator=gen, device="cuda") for _ in range(3))
    return 0.02 * p, 2e-3 * m, 1e-3 * g, (0.02 * p).bfloat16()


def step(p, m, g, w, ws):
    vp.muon_step(p, m, g, w, 0.02, 0.95, 0.1, vp.muon_rms_scale(*p.shape[1:]), ws)
    return vp.muon_device_status(ws)


# kind 1 (one launch): one CTA and a CTA pair a matrix, wide and tall, one matrix and several; the first, a middle and the last product
SMALL = [(1, batch, rows, cols, k, 1) for batch, rows, cols in ((1, 100, 400), (3, 200, 250), (1, 250, 130)) for k in (0, 7, 14)]
# kind 0: copies of the first tile lost in the leader, in the other CTA, in both
LARGE = [(0, 1, 300, 301, 1, 1), (0, 2, 700, 520, 0, 2), (0, 1, 300, 301, 4, 3)]


@pytest.mark.parametrize("kind,batch,rows,cols,index,ranks", SMALL + LARGE)
def test_lost_signal_expires_the_waits_and_the_next_call_is_clean(kind, batch, rows, cols, index, ranks):
    ws = torch.full((vp.muon_workspace_bytes(batch, rows, cols),), 255, dtype=torch.uint8, device="cuda")
    p0, m0, g, w0 = state(batch, rows, cols)
    p1, m1, w1 = p0.clone(), m0.clone(), w0.clone()
    assert step(p1, m1, g, w1, ws) == 0
    p, m, w = p0.clone(), m0.clone(), w0.clone()
    torch.cuda.synchronize()
    prev = vp.vp_ce_set_wait_limit_ns(LIMIT_NS)
    try:
        vp.muon_debug_drop(kind, index, ranks)
        t0 = time.perf_counter()
        status = step(p, m, g, w, ws)
        dt = time.perf_counter() - t0
    finally:
        vp.muon_debug_drop(-1)
        vp.vp_ce_set_wait_limit_ns(prev)
    assert status == WAIT_EXPIRED
    assert dt < 1.0, dt                                                  # a few limits, not the default and not a hang
    assert torch.equal(m, m1)
    assert ((p == p0) | (p == p1)).all() and ((w == w0) | (w == w1)).all()
    assert torch.equal(p[0], p0[0]) and torch.equal(w[0], w0[0])         # the matrix whose product is lost
    # the context is intact and the same workspace serves a normal call right away
    p, m, w = p0.clone(), m0.clone(), w0.clone()
    assert step(p, m, g, w, ws) == 0
    assert torch.equal(p, p1) and torch.equal(m, m1) and torch.equal(w, w1)


def test_an_armed_hook_for_another_kernel_leaves_a_call_alone():
    g = state(1, 64, 64)[2]
    ws = torch.empty(vp.muon_workspace_bytes(1, 64, 64), dtype=torch.uint8, device="cuda")
    a, b = torch.empty_like(g), torch.empty_like(g)
    vp.muon_orthogonalize(g, a, ws)
    try:
        vp.muon_debug_drop(0, 0, 1)                                      # the kernel of large matrices: not launched here
        vp.muon_orthogonalize(g, b, ws)
        assert vp.muon_device_status(ws) == 0
    finally:
        vp.muon_debug_drop(-1)
    assert torch.equal(a, b)
    for bad in ((2, 0, 1), (0, -1, 1), (0, 0, 0), (1, 0, 4), (0, 1 << 16, 1)):
        with pytest.raises(vp.VpceError) as ei:
            vp.muon_debug_drop(*bad)
        assert ei.value.code == 1
