"""The entry points of a network on sequences of tokens reject bad arguments before any HIP call (no GPU needed). The same
tests run a second time, in a child process, against a build with AddressSanitizer and UndefinedBehaviorSanitizer on its
host code."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2105_08810_amd import snn

SAN_LIB = os.environ.get("SNN_TOKENS_SANITIZED_LIB")
NAN, INF = float("nan"), float("inf")
FAKE = 0x1000  # never dereferenced: every call below must fail validation first
INVALID, UNSUPPORTED = snn.SNN_ERR_INVALID_ARG, snn.SNN_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    if SAN_LIB:
        l = ctypes.CDLL(SAN_LIB)
        for name, (res, args) in snn._SIGNATURES.items():
            getattr(l, name).restype = res
            getattr(l, name).argtypes = args
        return l
    if not os.path.exists(snn.LIB_PATH):
        from paper_2105_08810_amd import build
        build.build(verbose=False)
    return snn.lib()


def _call(fn, base, kw):
    assert set(kw) <= set(base)
    return fn(*[kw.get(k, v) for k, v in base.items()])


def _embed(lib, **kw):
    return _call(lib.snn_embed, dict(E=FAKE, dtype=0, V=10, N=8, ld_e=8, ids=FAKE, R=5, scale=1.0, out=FAKE, ld_out=8,
                                     stream=None), kw)


def _embed_grad(lib, **kw):
    return _call(lib.snn_embed_grad, dict(ids=FAKE, R=5, dout=FAKE, dtype=0, ld_out=8, V=10, N=8, scale=1.0, dE=FAKE,
                                          ld_e=8, accumulate=0, ws=FAKE, ws_bytes=1 << 50, stream=None), kw)


def _norm(lib, **kw):
    return _call(lib.snn_layer_norm, dict(x=FAKE, x_dtype=0, R=5, N=8, ld_x=8, gamma=FAKE, beta=FAKE, eps=1e-5, y=FAKE,
                                          y_dtype=0, ld_y=8, mean=FAKE, rstd=FAKE, stream=None), kw)


def _norm_grad(lib, **kw):
    return _call(lib.snn_layer_norm_grad,
                 dict(dy=FAKE, y_dtype=0, ld_dy=8, x=FAKE, x_dtype=0, ld_x=8, R=5, N=8, gamma=FAKE, mean=FAKE, rstd=FAKE,
                      dx=FAKE, ld_dx=8, dgamma=FAKE, dbeta=FAKE, ws=FAKE, ws_bytes=1 << 50, stream=None), kw)


def _ce(lib, **kw):
    return _call(lib.snn_linear_ce,
                 dict(x=FAKE, W=FAKE, dtype=0, R=5, H=8, C=12, ld_x=8, ld_w=12, targets=FAKE, weight=None, loss=FAKE,
                      row_loss=FAKE, dx=FAKE, ld_dx=8, dW=FAKE, ld_dw=12, ws=FAKE, ws_bytes=1 << 50, stream=None), kw)


def _leak(lib, **kw):
    return _call(lib.snn_leak_grad,
                 dict(x=FAKE, in_row_ptr=None, in_col_idx=None, in_g=None, in_cap=0, T=4, B=3, N=8, alpha=0.9, y=FAKE,
                      out_row_ptr=None, out_col_idx=None, out_cap=0, stream=None), kw)


def _currents(lib, **kw):
    return _call(lib.snn_lif_forward_currents,
                 dict(V=FAKE, T=4, B=3, N=8, alpha=0.9, theta=1.0, b_th=0.2, s_out=FAKE, trace_out=None, alpha_next=0.9,
                      active_bits=None, stream=None), kw)


REJECTED = [
    (_embed, [dict(E=None), dict(ids=None), dict(out=None), dict(dtype=3), dict(dtype=-1), dict(V=0), dict(V=-1), dict(N=0),
              dict(R=0), dict(R=-1), dict(ld_e=7), dict(ld_out=7), dict(scale=NAN), dict(E=FAKE + 2), dict(out=FAKE + 1),
              dict(dtype=1, E=FAKE + 1)]),
    (_embed_grad, [dict(ids=None), dict(dout=None), dict(dE=None), dict(ws=None), dict(dtype=3), dict(V=0), dict(N=-1),
                   dict(R=0), dict(ld_e=7), dict(ld_out=7), dict(scale=NAN), dict(dout=FAKE + 2), dict(dE=FAKE + 3),
                   dict(dtype=2, dE=FAKE + 1), dict(ws_bytes=100)]),
    (_norm, [dict(x=None), dict(y=None), dict(x_dtype=3), dict(y_dtype=-1), dict(R=0), dict(N=0), dict(ld_x=7), dict(ld_y=7),
             dict(eps=-1e-9), dict(eps=NAN), dict(eps=INF), dict(x=FAKE + 2), dict(y_dtype=1, y=FAKE + 1)]),
    (_norm_grad, [dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None, dgamma=None, dbeta=None),
                  dict(x_dtype=3), dict(y_dtype=3), dict(R=-1), dict(N=0), dict(ld_dy=7), dict(ld_x=7), dict(ld_dx=7),
                  dict(ws=None), dict(ws_bytes=10), dict(dx=FAKE + 2), dict(dy=FAKE + 1), dict(x=FAKE + 3)]),
    (_ce, [dict(x=None), dict(W=None), dict(targets=None), dict(loss=None), dict(ws=None), dict(ws_bytes=1000), dict(dtype=3),
           dict(R=0), dict(H=0), dict(C=-1), dict(ld_x=7), dict(ld_w=11), dict(ld_dx=7), dict(ld_dw=11), dict(x=FAKE + 2),
           dict(W=FAKE + 2), dict(dx=FAKE + 1), dict(dW=FAKE + 1), dict(dtype=1, W=FAKE + 1)]),
    (_leak, [dict(x=None), dict(y=None), dict(T=0), dict(B=0), dict(N=-1), dict(T=1 << 16, B=1 << 15), dict(alpha=0.0),
             dict(alpha=1.1), dict(alpha=NAN), dict(in_col_idx=FAKE), dict(in_g=FAKE), dict(out_col_idx=FAKE),
             dict(in_row_ptr=FAKE, in_cap=3), dict(out_row_ptr=FAKE, out_cap=3), dict(in_row_ptr=FAKE, in_cap=-1),
             dict(in_row_ptr=FAKE, in_col_idx=FAKE, in_cap=3, x=None), dict(out_row_ptr=FAKE, out_col_idx=FAKE, out_cap=3, y=None)]),
    (_currents, [dict(V=None), dict(s_out=None), dict(T=0), dict(B=-1), dict(N=0), dict(T=1 << 16, B=1 << 15), dict(alpha=0.0),
                 dict(theta=NAN), dict(trace_out=FAKE, alpha_next=0.0), dict(active_bits=FAKE, b_th=-1.0),
                 dict(active_bits=FAKE, b_th=NAN)]),
]


@pytest.mark.parametrize("call,kw", [(c, k) for c, ks in REJECTED for k in ks])
def test_rejected(lib, call, kw):
    assert call(lib, **kw) == INVALID


@pytest.mark.parametrize("call,kw", [
    (_embed, dict(V=1 << 31)), (_embed, dict(R=1 << 31)), (_embed, dict(N=(1 << 20) + 1, ld_e=1 << 21, ld_out=1 << 21)),
    (_embed_grad, dict(V=1 << 31)), (_embed_grad, dict(R=1 << 31)), (_embed_grad, dict(R=1 << 30)),
    (_norm, dict(R=1 << 31)), (_norm, dict(N=(1 << 20) + 1, ld_x=1 << 21, ld_y=1 << 21)), (_norm_grad, dict(R=1 << 31)),
    (_ce, dict(R=(1 << 24) + 1)), (_ce, dict(H=(1 << 16) + 1, ld_x=1 << 17, ld_dx=1 << 17)),
    (_ce, dict(C=(1 << 20) + 1, ld_w=1 << 21, ld_dw=1 << 21)), (_ce, dict(ld_w=1 << 31)),
    (_leak, dict(T=1, B=1 << 25, N=1))])
def test_unsupported(lib, call, kw):
    assert call(lib, **kw) == UNSUPPORTED


def test_workspaces(lib):
    grad = lib.snn_embed_grad_workspace
    assert grad(0, 10, 8, 5) > 0 and grad(1, 1 << 20, 64, 1 << 20) > grad(1, 1 << 20, 64, 1 << 10) > 0
    for bad in ((3, 10, 8, 5), (0, 0, 8, 5), (0, 10, 0, 5), (0, 10, 8, 0), (0, 1 << 31, 8, 5), (0, 10, 8, 1 << 30),
                (0, 10, (1 << 20) + 1, 5)):
        assert grad(*bad) == 0
    norm = lib.snn_layer_norm_grad_workspace
    assert norm(0, 0, 5, 8) > 0 and norm(1, 1, 1 << 30, 1 << 20) > 0
    for bad in ((3, 0, 5, 8), (0, 3, 5, 8), (0, 0, 0, 8), (0, 0, 5, 0), (0, 0, 1 << 31, 8), (0, 0, 5, (1 << 20) + 1)):
        assert norm(*bad) == 0
    ce = lib.snn_linear_ce_workspace
    for dtype in range(3):
        assert ce(dtype, 5, 8, 12, 1) >= ce(dtype, 5, 8, 12, 0) > 0
        assert ce(dtype, 1 << 24, 1 << 16, 1 << 20, 1) > 0
        # far below all logits
        assert ce(dtype, 1 << 15, 1024, 1 << 20, 1) < (1 << 15) * (1 << 20)
    for bad in ((3, 5, 8, 12, 1), (0, 0, 8, 12, 1), (0, 5, 0, 12, 1), (0, 5, 8, 0, 1), (0, (1 << 24) + 1, 8, 12, 1)):
        assert ce(*bad) == 0


@pytest.mark.skipif(SAN_LIB is not None, reason="the binding loads the ordinary library")
def test_binding_checks_before_the_call():
    x, ids = torch.zeros((3, 5)), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        snn.embed(x, ids)
    with pytest.raises(ValueError, match="device"):
        snn.embed_grad(ids, x, 10)
    with pytest.raises(ValueError, match="device"):
        snn.layer_norm(x)
    with pytest.raises(ValueError, match="device"):
        snn.linear_ce(x, torch.zeros((5, 4)), ids)
    with pytest.raises(ValueError, match="device"):
        snn.leak_grad(torch.zeros((2, 3, 4)), 0.5, (2, 3, 4))
    with pytest.raises(ValueError, match="accumulate"):
        snn.embed_grad(ids, x, 10, accumulate=True)


@pytest.mark.skipif(SAN_LIB is not None, reason="this is the child process")
def test_validation_under_sanitizers():
    from paper_2105_08810_amd import build
    sources = [os.path.join(build.CSRC, f) for f in os.listdir(build.CSRC) if f.endswith((".hip", ".h"))]
    path = build.SAN_LIB  # built by this file or another that tests with it, if no source is newer
    if not os.path.exists(path) or os.path.getmtime(path) < max(map(os.path.getmtime, sources + [snn.HEADER])):
        path = build.build_sanitized()
    env = dict(os.environ)
    env.update(SNN_TOKENS_SANITIZED_LIB=path, LD_PRELOAD=build.asan_runtime(),
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", os.path.abspath(__file__)],
                       capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
