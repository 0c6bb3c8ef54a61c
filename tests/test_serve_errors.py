"""Errors of the HIP runtime around the serving operators: an error that an earlier call left pending is not theirs, and
an error of their own launch is raised and not tried again (a second append would rotate queries in place twice)."""
from __future__ import annotations

import ctypes
import importlib.util
import os
import shutil
import subprocess

import pytest
import torch

from paper_2608_01662_amd import lsa

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not os.path.exists(lsa.LIB_PATH), reason="liblsa.so not built")]
DEV = "cuda"
BF = torch.bfloat16
HIP_ERROR = 4    # LSA_ERR_HIP


def _append():
    """(params, arguments) of an append of three sequences' last tokens whose queries are rotated in place."""
    torch.manual_seed(7)
    x = lambda *s: torch.randn(s, device=DEV).to(BF)
    q = x(3, 4, 64)
    return lsa.AppendParams(4, 2, 64, 64, 0, 64), dict(
        k=x(3, 2, 64), v=x(3, 2, 64), q=q, q_out=q, k_cache=torch.zeros((3, 2, 16, 64), dtype=BF, device=DEV),
        v_cache=torch.zeros((3, 2, 16, 64), dtype=BF, device=DEV), rope=torch.randn((16, 64), device=DEV),
        page_table=torch.arange(3, dtype=torch.int32, device=DEV)[:, None].contiguous(),
        ctx_len=torch.tensor([2, 9, 16], dtype=torch.int32, device=DEV))


def _attn(width):
    torch.manual_seed(8)
    x = lambda *s: torch.randn(s, device=DEV).to(BF)
    prm = lsa.DecodeAttnParams(8, 2, 64, 64, False, 0.125)
    a = dict(q=x(2, 8, 64), k_cache=x(6, 2, 64, 64), v_cache=x(6, 2, 64, 64), ctx_len=torch.tensor([100, 190], dtype=torch.int32, device=DEV),
             page_table=torch.zeros((2, width), dtype=torch.int32, device=DEV), out=torch.zeros((2, 8, 64), dtype=BF, device=DEV),
             lse=torch.zeros((2, 8), device=DEV),
             workspace=torch.empty(max(1, lsa.decode_attn_workspace_size(prm, 2, 1, width, 64)), dtype=torch.uint8, device=DEV))
    a["page_table"][:, :3] = torch.arange(6, dtype=torch.int32, device=DEV).view(2, 3)
    return prm, a


def _runtime():
    """The HIP runtime that this process has loaded."""
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64.so" in line)
    return ctypes.CDLL(path)


def _with_pending_error(call):
    """call() while the runtime holds an error of an earlier call of this thread (a device that does not exist)."""
    hip = _runtime()
    torch.cuda.synchronize()
    assert hip.hipSetDevice(4096) != 0
    try:
        return call()
    finally:
        hip.hipGetLastError()


def test_append_beside_a_pending_error_rotates_once():
    prm, a = _append()
    want = {n: t.clone() for n, t in a.items()}
    lsa.cache_append(prm, **{**want, "q_out": want["q"]})
    _with_pending_error(lambda: lsa.cache_append(prm, **a))
    torch.cuda.synchronize()
    for n in ("q", "k_cache", "v_cache"):
        assert torch.equal(a[n], want[n]), n


@pytest.mark.parametrize("width", [4, 256], ids=["whole", "cut"])
def test_attention_beside_a_pending_error(width):
    prm, a = _attn(width)
    out, lse = (t.clone() for t in lsa.decode_attn(prm, **a))
    a["out"].zero_()
    _with_pending_error(lambda: lsa.decode_attn(prm, **a))
    torch.cuda.synchronize()
    assert torch.equal(a["out"], out) and torch.equal(a["lse"], lse)


STUB = """
#include <stddef.h>
static int calls, status;
int stub_calls(void) { return calls; }
void stub_status(int s) { status = s; calls = 0; }
int lsa_cache_append(const void* p, const void* t, long n, int a, int b, int c, int d, long e, void* s) { ++calls; return status; }
int lsa_decode_attn() { ++calls; return status; }
size_t lsa_decode_attn_workspace_size(const void* p, int a, int b, int c, int d) { return 0; }
"""


@pytest.fixture(scope="module")
def failing(tmp_path_factory):
    """The binding against a library whose calls return a given status (its symbols come first in the process, so a
    second copy of the binding takes them)."""
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler for the stub library")
    lsa._serving()
    d = tmp_path_factory.mktemp("stub")
    (d / "stub.c").write_text(STUB)
    subprocess.run([cc, "-shared", "-fPIC", "-o", str(d / "stub.so"), str(d / "stub.c")], check=True, timeout=60)
    stub = ctypes.CDLL(str(d / "stub.so"), mode=ctypes.RTLD_GLOBAL)
    shutil.copy(lsa.SERVE_PATH, d / "_serve.so")
    os.symlink(lsa.LIB_PATH, d / "liblsa.so")
    spec = importlib.util.spec_from_file_location("stubbed._serve", str(d / "_serve.so"))
    serve = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(serve)
    serve.check = getattr(lsa._serving(), "check", None)
    return stub, serve


def test_a_launch_error_of_the_append_is_raised_once(failing, monkeypatch):
    stub, serve = failing
    prm, a = _append()
    before = a["q"].clone()
    monkeypatch.setattr(lsa, "_serve", serve)
    stub.stub_status(HIP_ERROR)
    with pytest.raises(lsa.LSAError) as e:
        lsa.cache_append(prm, **a)
    assert e.value.status == HIP_ERROR and "lsa_cache_append" in str(e.value)
    assert stub.stub_calls() == 1 and torch.equal(a["q"], before) and a["k_cache"].count_nonzero() == 0


def test_a_launch_error_of_the_attention_is_raised_once(failing, monkeypatch):
    stub, serve = failing
    prm, a = _attn(4)
    monkeypatch.setattr(lsa, "_serve", serve)
    stub.stub_status(HIP_ERROR)
    with pytest.raises(lsa.LSAError) as e:
        lsa.decode_attn(prm, **a)
    assert e.value.status == HIP_ERROR and "lsa_decode_attn" in str(e.value)
    assert stub.stub_calls() == 1 and a["out"].count_nonzero() == 0


def test_a_refusal_is_left_to_the_checks_in_python(failing, monkeypatch):
    """(here they find nothing wrong, and the library behind them runs the call)"""
    stub, serve = failing
    prm, a = _attn(4)
    monkeypatch.setattr(lsa, "_serve", serve)
    for status in (1, 2, 3):
        stub.stub_status(status)
        a["out"].zero_()
        lsa.decode_attn(prm, **a)
        assert stub.stub_calls() == 1 and a["out"].count_nonzero() > 0
