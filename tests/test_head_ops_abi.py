"""CPU-side checks of the operators from the residual stream to log probabilities: every declared symbol is exported and bound, the
pure-host entry points behave, refusals come before any launch, and the float64 definitions agree with differences."""
import ctypes
import os
import re

import torch

import paper_2609_14306_b200 as vp
from oracle import head_ops_oracle as orc
from paper_2609_14306_b200.build import build_library

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_symbol_is_exported_and_bound():
    build_library()
    raw = ctypes.CDLL(vp.library_path())
    for fn, least in (("rms_norm.h", 4), ("token_logp.h", 6), ("fp8_blocks.h", 1)):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", fn)).read(), flags=re.S)
        names = re.findall(r"\b(vp_(?:rms|token_logp|fp8)_\w+)\s*\(", text)
        assert len(names) >= least
        for n in names:
            assert hasattr(raw, n), n
            assert hasattr(vp, n), f"python binding lacks {n}"
    for n in ("rms_norm", "rms_norm_fp8", "token_log_probs", "token_log_probs_fp8", "quantize_blocks_fp8"):
        assert callable(getattr(vp, n))


def test_workspace_sizes():
    assert vp.vp_rms_workspace_bytes(65536, 7168) <= 65536 * 7168 * 2 // 16
    assert vp.vp_rms_workspace_bytes(0, 1) > 0 and vp.vp_rms_workspace_bytes(-1, 8) == 0 and vp.vp_rms_workspace_bytes(4, 0) == 0
    size = vp.vp_token_logp_workspace_bytes
    # bounded, whatever the tokens and the vocabulary, and small for a few tokens
    assert max(size(T, 2880, V, top) for T in (65, 4096, 8192, 1 << 20) for V in (1000, 201088, 1 << 22) for top in (0, 20)) < 100 << 20
    assert size(1, 2880, 201088, 8) < 1 << 14
    assert size(1, 2884, 1000, 0) == 0 and size(1, 8, 5, 6) == 0 and size(1, 8, 100, 21) == 0 and size(-1, 8, 100, 0) == 0
    assert vp.vp_token_logp_fp8_workspace_bytes(1, 2888, 1000, 0) == 0 and vp.vp_token_logp_fp8_workspace_bytes(1, 16400, 1000, 0) == 0
    assert vp.vp_token_logp_fp8_workspace_bytes(1, 16384, 1000, 0) > 0
    assert vp.fp8_blocks(1) == 1 and vp.fp8_blocks(128) == 1 and vp.fp8_blocks(129) == 2


def test_c_entries_refuse_before_any_launch():
    vp.vp_rms_workspace_bytes(1, 1)                           # binds the signatures
    lib = vp.load_library()
    rms = lambda x, dt=0, rows=4, d=8, xs=8, r=None, eps=1e-6, y=16, z=None: lib.vp_rms_forward(  # noqa: E731
        x, dt, rows, d, xs, r, 8, None, 0, eps, y, 8, z, 8, None, None)
    assert rms(None) == 1 and rms(16, dt=7) == 1 and rms(16, xs=7) == 1 and rms(16, eps=-1.0) == 1 and rms(16, y=None) == 1
    assert rms(16, z=32) == 1                                 # a sum without a residual
    assert rms(17) == 2 and rms(16, r=17) == 2 and rms(16, rows=0) == 0
    assert lib.vp_rms_forward_fp8(16, 0, 4, 8, 8, None, 8, None, 0, 1e-6, 16, 8, None, None, 8, None, None) == 1        # no scales
    assert lib.vp_rms_backward(16, 8, None, 8, 16, 8, 0, 4, 8, None, 0, None, 16, 8, None, None, 0, None) == 1          # no rstd
    assert lib.vp_rms_backward(16, 8, None, 8, 16, 8, 0, 4, 8, None, 0, 16, 16, 8, 16, 16, 8, None) == 3
    fwd = lambda H=16, W=16, tok=16, T=4, d=64, V=300, temp=1.0, logp=16, tl=16, ti=16, top=2, ws=256, n=1 << 20: lib.vp_token_logp_forward(  # noqa: E731
        H, W, tok, T, d, V, temp, -100, logp, None, None, tl, ti, top, ws, n, None)
    assert fwd(H=None) == 1 and fwd(W=None) == 1 and fwd(ws=None) == 1 and fwd(tok=None) == 1 and fwd(logp=None) == 1 and fwd(tl=None) == 1
    assert fwd(temp=0.0) == 1 and fwd(temp=float("inf")) == 1 and fwd(top=21) == 1 and fwd(V=1) == 1 and fwd(T=-1) == 1
    assert fwd(H=24) == 2 and fwd(d=60) == 2 and fwd(ti=18) == 2 and fwd(n=64) == 3 and fwd(T=0) == 0
    fp8 = lambda Hs=16, d=64: lib.vp_token_logp_fp8_forward(  # noqa: E731
        16, Hs, 16, 16, 16, 4, d, 300, 1.0, -100, 16, None, None, None, None, 0, 256, 1 << 20, None)
    assert fp8(Hs=None) == 1 and fp8(d=72) == 2 and fp8(d=16400) == 2 and fp8(Hs=18) == 2
    bwd = lambda u=16, v=16, ent=16, temp=1.0: lib.vp_token_logp_backward(  # noqa: E731
        16, 16, 16, 16, ent, u, v, 16, None, 4, 64, 300, temp, 256, -100, 128, 0, 0, 256, 64, None)
    assert bwd(u=None, v=None) == 1 and bwd(ent=None) == 1 and bwd(temp=-1.0) == 1 and bwd() == 3
    q = lambda w=16, dt=0, rows=4, ws=64, s=16: lib.vp_fp8_quantize_blocks(w, dt, rows, 64, ws, 16, 64, s, None)  # noqa: E731
    assert q(w=None) == 1 and q(dt=5) == 1 and q(ws=63) == 1 and q(s=None) == 1 and q(w=17) == 2 and q(rows=0) == 0
    assert lib.vp_token_logp_debug_drop(-1) == 0


def test_the_definitions_gradients_against_differences():
    gen = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    h, w, u, v = r(5, 6), r(9, 6), r(5), r(5)
    tokens = torch.tensor([0, 8, -100, 3, 3])
    dH, dW, _ = orc.token_logp_grad(h, w, tokens, u, v, 0.7)

    def value(a, b):
        o = orc.token_logp(a, b, tokens, 0.7)
        return float((o["logp"] * u).sum() + (o["entropy"] * v).sum())

    eps = 1e-6
    for t, g in ((h, dH), (w, dW)):
        e = r(*t.shape)
        plus, minus = ((h + eps * e, w), (h - eps * e, w)) if t is h else ((h, w + eps * e), (h, w - eps * e))
        assert abs((value(*plus) - value(*minus)) / (2 * eps) - float((g * e).sum())) < 1e-7
    z, g, dy, dz = r(4, 7), r(7), r(4, 7), r(4, 7)
    dx, dg = orc.rms_norm_grad(dy, dz, z, g, 1e-3)
    norm = lambda a, b: float((orc.rms_norm(a, b, 1e-3)[0] * dy).sum() + (a * dz).sum())  # noqa: E731
    e = r(4, 7)
    assert abs((norm(z + eps * e, g) - norm(z - eps * e, g)) / (2 * eps) - float((dx * e).sum())) < 1e-7
    e = r(7)
    assert abs((norm(z, g + eps * e) - norm(z, g - eps * e)) / (2 * eps) - float((dg * e).sum())) < 1e-7


def test_default_strip_width_is_whole_tiles_in_bounded_memory():
    from paper_2609_14306_b200.head_ops import _strip_width
    for chunk in (128, 256, 1024, 4096, 8192, 16384, 65536):
        for V in (1, 255, 256, 257, 8193, 201088, 2 ** 31 - 300):
            width = _strip_width(chunk, V)
            assert width > 0 and width % 256 == 0 and (width >= V or width >= 8192)
            assert width <= 8192 or chunk * width <= 2 ** 27
            assert width < V + 256 and vp.vp_ce_workspace_bytes(chunk, 64, width) > 0
