"""The entry points on rows of logits reject bad arguments before any HIP call (no GPU needed). The same tests run a
second time, in a child process, against a build with AddressSanitizer and UndefinedBehaviorSanitizer on its host code."""
import ctypes
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2105_08810_amd import snn

SAN_LIB = os.environ.get("SNN_ROWS_SANITIZED_LIB")
NAN, INF = float("nan"), math.inf
FAKE = 0x1000  # never dereferenced: every call below must fail validation first


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


ROWS_INVALID = [dict(logits=None), dict(dtype=-1), dict(dtype=3), dict(R=0), dict(R=-5), dict(C=0), dict(C=-1),
                dict(ld=99), dict(ld=-1), dict(logits=FAKE + 2), dict(dtype=1, logits=FAKE + 1)]
ROWS_UNSUPPORTED = [dict(R=1 << 31), dict(C=(1 << 20) + 1, ld=1 << 21), dict(R=1 << 30, ld=1 << 40),
                    dict(R=(1 << 31) - 1, ld=(1 << 63) - 1)]


def _call(fn, order, base, kw):
    a = dict(base)
    a.update(kw)
    return fn(*[a[k] for k in order])


def _top(lib, **kw):
    return _call(lib.snn_readout_top, "logits dtype R C ld K tau ids vals lse ws ws_bytes stream".split(),
                 dict(logits=FAKE, dtype=0, R=10, C=100, ld=100, K=5, tau=1.0, ids=FAKE, vals=FAKE, lse=FAKE, ws=None,
                      ws_bytes=0, stream=None), kw)


def _distill(lib, **kw):
    order = ("logits dtype R C ld ids vals lse K tau weight loss row_loss grad ld_grad accumulate ws ws_bytes "
             "stream").split()
    return _call(lib.snn_readout_distill, order,
                 dict(logits=FAKE, dtype=0, R=10, C=100, ld=100, ids=FAKE, vals=FAKE, lse=FAKE, K=5, tau=1.0,
                      weight=FAKE, loss=FAKE, row_loss=FAKE, grad=FAKE, ld_grad=100, accumulate=0, ws=FAKE,
                      ws_bytes=1 << 40, stream=None), kw)


def _sample(lib, **kw):
    return _call(lib.snn_readout_sample, ("logits dtype R C ld u temperature top_k top_p min_p cls logp kept ws "
                                          "ws_bytes stream").split(),
                 dict(logits=FAKE, dtype=0, R=10, C=100, ld=100, u=FAKE, temperature=FAKE, top_k=FAKE, top_p=FAKE,
                      min_p=FAKE, cls=FAKE, logp=FAKE, kept=FAKE, ws=None, ws_bytes=0, stream=None), kw)


@pytest.mark.parametrize("call", [_top, _distill, _sample])
@pytest.mark.parametrize("kw", ROWS_INVALID)
def test_rows_rejected(lib, call, kw):
    assert call(lib, **kw) == snn.SNN_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [_top, _distill, _sample])
@pytest.mark.parametrize("kw", ROWS_UNSUPPORTED)
def test_rows_unsupported(lib, call, kw):
    assert call(lib, **kw) == snn.SNN_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(ids=None), dict(vals=None), dict(K=0), dict(K=-1), dict(K=101), dict(tau=0.0),
                                dict(tau=-1.0), dict(tau=NAN), dict(tau=INF)])
@pytest.mark.parametrize("call", [_top, _distill])
def test_record_rejected(lib, call, kw):
    assert call(lib, **kw) == snn.SNN_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [_top, _distill])
def test_record_too_long(lib, call):
    assert call(lib, K=1025, C=5000, ld=5000, **({"ld_grad": 5000} if call is _distill else {})) == snn.SNN_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(loss=None), dict(ws=None), dict(ws_bytes=1), dict(ld_grad=99), dict(grad=FAKE + 2)])
def test_distill_rejects(lib, kw):
    assert _distill(lib, **kw) == snn.SNN_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(u=None), dict(cls=None), dict(R=1, C=131072, ld=131072),
                                dict(R=1, C=131072, ld=131072, ws=FAKE, ws_bytes=100)])
def test_sample_rejects(lib, kw):
    assert _sample(lib, **kw) == snn.SNN_ERR_INVALID_ARG


def test_distill_workspace(lib):
    size = lib.snn_readout_distill_workspace
    assert size(10, 100, 0) > 0 and size(1, 1, 2) > 0
    assert size((1 << 31) - 1, 1 << 20, 1) >= ((1 << 31) - 1) * 4
    for bad in ((0, 100, 0), (-1, 100, 0), (10, 0, 0), (10, 100, 3), (1 << 31, 100, 0), (10, (1 << 20) + 1, 0)):
        assert size(*bad) == 0
    assert size(777, 333, 1) == size(777, 333, 1)


@pytest.mark.parametrize("kw", [dict(), dict(ws=FAKE, ws_bytes=100)])
def test_top_needs_its_workspace(lib, kw):
    assert _top(lib, R=1, C=131072, ld=131072, **kw) == snn.SNN_ERR_INVALID_ARG


def test_top_workspace(lib):
    size = lib.snn_readout_top_workspace
    assert size(1, 131072, 0, 5) > 0 and size(2, 131072, 1, 5) > size(1, 131072, 1, 5) > 0  # few long rows
    assert size(1, 1000, 0, 5) == 0 and size(100000, 131072, 0, 5) == 0 and size(1, 131072, 0, 1000) == 0
    for bad in ((0, 131072, 0, 5), (-1, 131072, 0, 5), (1, 0, 0, 5), (1, 131072, 3, 5), (1 << 31, 131072, 0, 5),
                (1, (1 << 20) + 1, 0, 5), (1, 131072, 0, 0), (1, 100, 0, 101)):
        assert size(*bad) == 0


def test_sample_workspace(lib):
    size = lib.snn_readout_sample_workspace
    assert size(1, 131072, 0) > 0 and size(2, 131072, 1) > size(1, 131072, 1) > 0  # few long rows
    assert size(1, 1000, 0) == 0 and size(100000, 131072, 0) == 0 and size(1, 1 << 20, 0) == 0
    for bad in ((0, 131072, 0), (-1, 131072, 0), (1, 0, 0), (1, 131072, 3), (1 << 31, 131072, 0), (1, (1 << 20) + 1, 0)):
        assert size(*bad) == 0


@pytest.mark.skipif(SAN_LIB is not None, reason="the binding loads the ordinary library")
def test_binding_checks_before_the_call():
    z = torch.zeros((3, 5))
    with pytest.raises(ValueError, match="device"):
        snn.readout_top(z, 2)
    with pytest.raises(ValueError, match="device"):
        snn.readout_sample(z, torch.zeros(3))
    with pytest.raises(ValueError, match="accumulate"):
        snn.readout_distill(z, torch.zeros((3, 2), dtype=torch.int32), torch.zeros((3, 2)), accumulate=True)


@pytest.mark.skipif(SAN_LIB is not None, reason="runs in the parent process only")
def test_validation_under_sanitizers():
    from paper_2105_08810_amd import build
    path = build.build_sanitized()
    env = dict(os.environ)
    env.update(SNN_ROWS_SANITIZED_LIB=path, LD_PRELOAD=build.asan_runtime(),
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", __file__],
                       capture_output=True, text=True, env=env, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "runtime error" not in out and "AddressSanitizer" not in out, out[-4000:]
    assert " passed" in out
