"""CPU-side checks of the operators around the head: every declared symbol is exported and bound, and the pure-host entry
points (workspace sizes, refusals before any launch) behave."""
import ctypes
import os
import re

import paper_2609_14306_b200 as vp
from paper_2609_14306_b200.build import build_library

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_symbol_is_exported_and_bound():
    build_library()
    raw = ctypes.CDLL(vp.library_path())
    seen = set()
    for fn in ("layer_norm.h", "sequence_loss.h", "muon.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", fn)).read(), flags=re.S)
        names = re.findall(r"\b((?:vp_ln|vp_policy|vp_preference|muon)_\w+)\s*\(", text)
        assert names
        for n in names:
            assert hasattr(raw, n), n
            assert hasattr(vp, n), f"python binding lacks {n}"
        seen.update(names)
    assert {"vp_ln_forward", "vp_ln_backward", "vp_policy_loss", "vp_preference_loss", "muon_step", "muon_orthogonalize"} <= seen
    for n in ("layer_norm", "policy_loss", "preference_loss", "muon_rms_scale"):
        assert callable(getattr(vp, n))


def test_workspace_sizes():
    assert vp.vp_ln_workspace_bytes(16, 2880) >= 2 * 2880 * 4 and vp.vp_ln_workspace_bytes(0, 1) > 0
    assert vp.vp_ln_workspace_bytes(-1, 8) == 0 and vp.vp_ln_workspace_bytes(4, 0) == 0
    # the partial sums stay small next to the rows they stand for
    assert vp.vp_ln_workspace_bytes(65536, 7168) <= 65536 * 7168 * 2 // 16
    assert vp.vp_policy_loss_workspace_bytes(-1, 1) == 0 and vp.vp_policy_loss_workspace_bytes(0, 0) > 0
    assert vp.vp_policy_loss_workspace_bytes(1 << 20, 256) < 1 << 18
    assert vp.vp_preference_loss_workspace_bytes(1000, 7) == vp.vp_policy_loss_workspace_bytes(1000, 14)
    assert vp.vp_preference_loss_workspace_bytes(1000, -1) == 0
    n = vp.muon_workspace_bytes(4, 2880, 2880)
    assert 4 * 4 * 2 * 2880 * 2880 <= n <= 4 * 4 * 2 * 2880 * 2880 * 1.02 + (1 << 20)      # X twice, A, B in fp16
    assert vp.muon_workspace_bytes(1, 100, 300) == vp.muon_workspace_bytes(1, 300, 100)
    assert vp.muon_workspace_bytes(-1, 4, 4) == 0 and vp.muon_workspace_bytes(1, 1 << 30, 1 << 30) == 0
    assert abs(vp.muon_rms_scale(2048, 7168) - 0.2 * 7168 ** 0.5) < 1e-12


def test_c_entries_refuse_before_any_launch():
    vp.vp_ln_workspace_bytes(1, 1)                            # binds the signatures
    lib = vp.load_library()
    # null operands, unknown types, impossible sizes: status 1 without touching a device
    assert lib.vp_ln_forward(None, 0, 4, 8, 8, None, None, 0, 1e-5, None, 8, None, None, None) == 1
    assert lib.vp_ln_forward(16, 7, 4, 8, 8, None, None, 0, 1e-5, 16, 8, None, None, None) == 1
    assert lib.vp_ln_forward(16, 0, 4, 8, 7, None, None, 0, 1e-5, 16, 8, None, None, None) == 1
    assert lib.vp_ln_forward(17, 0, 4, 8, 8, None, None, 0, 1e-5, 16, 8, None, None, None) == 2
    assert lib.vp_ln_forward(16, 0, 0, 8, 8, None, None, 0, 1e-5, 16, 8, None, None, None) == 0
    assert lib.vp_policy_loss(None, None, None, None, 1, None, None, 5, 1, 0.2, 0.2, 0.0, 0, None, None, None, None, 0, None) == 1
    assert lib.vp_policy_loss(16, 16, None, 16, 1, None, 16, 5, 1, 0.2, 0.2, 0.0, 9, 16, None, None, 16, 1 << 20, None) == 1
    assert lib.vp_policy_loss(16, 16, None, 16, 1, None, 16, 5, 1, 0.2, 0.2, 0.0, 0, 16, None, None, 16, 8, None) == 3
    assert lib.vp_preference_loss(16, None, None, 16, 5, 1, -1.0, 0.0, 0.0, 0, 0, 16, None, None, None, 16, 1 << 20, None) == 1
    assert lib.muon_orthogonalize(None, 0, None, 0, 1, 4, 4, None, 5, 1e-7, None, 0, None) == 1
    assert lib.muon_orthogonalize(256, 0, 256, 0, 1, 4, 4, None, 0, 1e-7, 256, 1 << 20, None) == 1
    assert lib.muon_orthogonalize(256, 0, 256, 0, 1, 4, 4, None, 5, 1e-7, 256, 64, None) == 3
    assert lib.muon_orthogonalize(256, 0, 256, 0, 0, 4, 4, None, 5, 1e-7, None, 0, None) == 0
    # a bound on X beyond the fp16 range
    coeffs = (ctypes.c_double * 3)(9.0, 1.0, 1.0)
    assert lib.muon_orthogonalize(256, 0, 256, 0, 1, 4, 4, coeffs, 1, 1e-7, 256, 1 << 20, None) == 2
