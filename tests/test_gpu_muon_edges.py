"""Muon: repeats of the whole update, and a bound on single elements.  Oracle and helpers are those of test_gpu_muon."""
import numpy as np
import pytest
import torch

import paper_2609_14306_b200 as vp
import test_gpu_muon as muon

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,rows,cols", [(1, 256, 256), (5, 100, 500), (3, 1999, 501), (2, 300, 1000), (1, 1100, 1100)])
def test_updates_repeat_bit_for_bit(batch, rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(1)
    p, m, g = (torch.randn(batch, rows, cols, generator=gen, device="cuda") for _ in range(3))
    first = None
    for _ in range(4):
        now = [p.clone(), m.clone(), torch.empty(p.shape, dtype=torch.bfloat16, device="cuda")]
        vp.muon_step(now[0], now[1], 1e-3 * g, now[2], 0.02, 0.95, 0.1, vp.muon_rms_scale(rows, cols), muon.workspace(batch, rows, cols))
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


@pytest.mark.parametrize("batch,rows,cols", [(2, 100, 500), (1, 256, 250), (1, 700, 900), (2, 1300, 400)])
def test_single_elements(batch, rows, cols):
    """The roundings behind TOL_O (a relative Frobenius error) are spread over the matrix by products with rows of many entries, so a
    single error is close to normal with at most that deviation: the largest of 10^6 stays below 5 deviations, 6 with a margin
    for its unevenness over rows."""
    g = muon.gradient(batch, rows, cols, seed=rows)
    o = muon.orth(g).double().cpu().numpy()
    ref = muon.oracle(g)
    for i in range(batch):
        assert np.abs(o[i] - ref[i]).max() <= 6 * muon.TOL_O * np.sqrt((ref[i] ** 2).mean())
