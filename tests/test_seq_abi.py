"""The sequence operators at the C ABI, without a GPU: struct layouts against the C compiler, workspace
sizes, and arguments that are refused before any device call."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2607_05272_gb300 import build as B
from paper_2607_05272_gb300 import simx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = [("simx_logits", simx.Logits), ("simx_token_loss", simx.TokenLoss),
           ("simx_preference_loss", simx.PreferenceLoss), ("simx_seq", simx.Seq),
           ("simx_scan", simx.Scan), ("simx_norm", simx.Norm)]
FAKE = 1 << 20  # a device address that no refused call looks at


@pytest.fixture(scope="module")
def lib():
    B.build()
    return simx.lib()


def test_struct_offsets_match_the_c_compiler(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "simx.h"', "int main(void) {"]
    for name, cls in STRUCTS:
        lines.append('  printf("%s . %%zu\\n", sizeof(%s));' % (name, name))
        for f in cls._fields_:
            lines.append('  printf("%s %s %%zu\\n", offsetof(%s, %s));' % (name, f[0], name, f[0]))
    src, exe = tmp_path / "l.c", tmp_path / "l"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    got = {}
    for ln in subprocess.check_output([str(exe)]).decode().splitlines():
        name, field, v = ln.split()
        got[name, field] = int(v)
    for name, cls in STRUCTS:
        assert got[name, "."] == C.sizeof(cls), name
        for f in cls._fields_:
            assert got[name, f[0]] == getattr(cls, f[0]).offset, (name, f[0])


def test_workspace_sizes(lib):
    assert simx.token_loss_grad_workspace_size(0) > 0 and simx.token_loss_grad_workspace_size(-1) == 0
    assert simx.preference_loss_grad_workspace_size(100, 3) >= 100 * 12
    assert simx.preference_loss_grad_workspace_size(1, -1) == 0
    assert simx.gated_scan_workspace_size(3, 100, 8) >= 3 * 8 * 4
    assert simx.gated_scan_workspace_size(-1, 1, 1) == 0
    assert simx.dropout_add_norm_grad_workspace_size(10, 64) >= 64 * 4
    assert simx.dropout_add_norm_grad_workspace_size(10, 16385) == 0


def _refused(lib, status):
    assert status == simx.EINVAL, status
    assert lib.simx_last_error()


def _logits(**kw):
    d = dict(logits=FAKE, grad=FAKE, ld=8, grad_ld=8, n=4, vocab=8, dtype=0, temperature=1.0)
    d.update(kw)
    return simx.Logits(**d)


def _token(**kw):
    d = dict(action=FAKE, adv=FAKE, clip_low=0.2, clip_high=0.2, stats=FAKE)
    d.update(kw)
    return simx.TokenLoss(**d)


@pytest.mark.parametrize("x,l", [
    (dict(dtype=2), {}), (dict(n=-1), {}), (dict(vocab=0), {}), (dict(vocab=1 << 31), {}),
    (dict(ld=7), {}), (dict(grad_ld=7), {}), (dict(logits=None), {}), (dict(logits=FAKE + 2), {}),
    (dict(grad_ld=16, grad=FAKE), {}), (dict(temperature=0.0), {}), (dict(temperature=float("inf")), {}),
    (dict(temperature=1e-45), {}), ({}, dict(stats=None)), ({}, dict(action=None)),
    ({}, dict(clip_low=-1.0)), ({}, dict(clip_high=float("nan"))), ({}, dict(c_entropy=float("inf")))])
def test_token_loss_refusals(lib, x, l):
    a, b = _logits(**x), _token(**l)
    _refused(lib, lib.simx_token_loss_grad(C.byref(a), C.byref(b), FAKE, 1 << 30, None))


def test_null_arguments_and_workspaces(lib):
    a, b = _logits(), _token()
    _refused(lib, lib.simx_token_loss_grad(None, C.byref(b), FAKE, 1 << 30, None))
    _refused(lib, lib.simx_token_loss_grad(C.byref(a), None, FAKE, 1 << 30, None))
    _refused(lib, lib.simx_token_loss_grad(C.byref(a), C.byref(b), None, 1 << 30, None))
    _refused(lib, lib.simx_token_loss_grad(C.byref(a), C.byref(b), FAKE, 16, None))
    _refused(lib, lib.simx_token_loss_grad(C.byref(a), C.byref(b), FAKE + 4, 1 << 30, None))
    _refused(lib, lib.simx_preference_loss_grad(C.byref(a), None, FAKE, 1 << 30, None))
    _refused(lib, lib.simx_gated_scan(None, None, 0, None))
    _refused(lib, lib.simx_gated_scan_grad(None, None, 0, None))
    _refused(lib, lib.simx_dropout_add_norm(None, None))
    _refused(lib, lib.simx_dropout_add_norm_grad(None, None, 0, None))


@pytest.mark.parametrize("kw", [dict(pairs=-1), dict(pairs=1 << 30), dict(seq_start=None), dict(token=None),
                                dict(beta=float("inf")), dict(label_smoothing=-0.1), dict(stats=None)])
def test_preference_loss_refusals(lib, kw):
    d = dict(token=FAKE, seq_start=FAKE, pairs=2, beta=0.1, stats=FAKE)
    d.update(kw)
    a, b = _logits(), simx.PreferenceLoss(**d)
    _refused(lib, lib.simx_preference_loss_grad(C.byref(a), C.byref(b), FAKE, 1 << 30, None))


def _scan(**kw):
    q = simx.Seq(FAKE, 32, 8)
    d = dict(batch=2, len=4, channels=8, dtype=0, x=q, gate=q, h=q, dh=q, dx=q, dgate=q)
    d.update(kw)
    return simx.Scan(**d)


@pytest.mark.parametrize("kw", [
    dict(dtype=5), dict(batch=-1), dict(len=-1), dict(channels=(1 << 31) + 1), dict(batch=1 << 30, channels=1 << 30),
    dict(x=simx.Seq(None, 32, 8)), dict(gate=simx.Seq(FAKE + 1, 32, 8)), dict(x=simx.Seq(FAKE, 32, -8)),
    dict(h=simx.Seq(FAKE, 32, 7)), dict(h=simx.Seq(FAKE, 8, 8)), dict(h=simx.Seq(FAKE, 0, 8))])
def test_scan_refusals(lib, kw):
    s = _scan(**kw)
    _refused(lib, lib.simx_gated_scan(C.byref(s), None, 0, None))


@pytest.mark.parametrize("kw", [dict(dh=simx.Seq(None, 32, 8)), dict(dx=simx.Seq(FAKE, 32, 4)), dict(dgate=simx.Seq(None, 0, 0))])
def test_scan_gradient_refusals(lib, kw):
    s = _scan(**kw)
    _refused(lib, lib.simx_gated_scan_grad(C.byref(s), FAKE, 1 << 30, None))
    s = _scan()
    _refused(lib, lib.simx_gated_scan_grad(C.byref(s), None, 0, None))


def _norm(**kw):
    d = dict(n=4, width=16, dtype=0, p=0.1, eps=1e-6, gain=FAKE, rstd=FAKE)
    for k in ("x", "residual", "z", "y", "dy", "dz", "dx", "dresidual"):
        d[k], d[k + "_ld"] = FAKE, 16
    d.update(kw)
    return simx.Norm(**d)


BAD = [dict(dtype=9), dict(n=-1), dict(n=1 << 33), dict(width=0), dict(width=16385), dict(p=-0.1), dict(p=1.0),
       dict(p=float("nan")), dict(gain=None), dict(z_ld=15), dict(n=5, row_base=(1 << 32) - 4)]


@pytest.mark.parametrize("kw", BAD + [dict(eps=0.0), dict(eps=float("nan")), dict(x=None), dict(y=None), dict(x=FAKE + 2)])
def test_norm_refusals(lib, kw):
    a = _norm(**kw)
    _refused(lib, lib.simx_dropout_add_norm(C.byref(a), None))


@pytest.mark.parametrize("kw", BAD + [dict(rstd=None), dict(z=None), dict(dy=None), dict(dx_ld=3)])
def test_norm_gradient_refusals(lib, kw):
    a = _norm(dgain=FAKE, **kw)
    _refused(lib, lib.simx_dropout_add_norm_grad(C.byref(a), FAKE, 1 << 30, None))
    a = _norm(dgain=FAKE)
    _refused(lib, lib.simx_dropout_add_norm_grad(C.byref(a), FAKE, 16, None))


def test_empty_problems_are_no_error(lib):
    s = _scan(batch=0)
    assert lib.simx_gated_scan(C.byref(s), None, 0, None) == simx.OK
    assert lib.simx_gated_scan_grad(C.byref(s), None, 0, None) == simx.OK
    a = _norm(n=0, gain=None)
    assert lib.simx_dropout_add_norm(C.byref(a), None) == simx.OK


def test_binding_refuses_host_tensors(lib):
    import torch
    x = torch.zeros(4, 8)
    for call in (lambda: simx.token_loss_grad(x, None, None, None, None),
                 lambda: simx.gated_scan(x[None], x[None], x[None]),
                 lambda: simx.dropout_add_norm(x, None, x)):
        with pytest.raises(simx.SimxError) as e:
            call()
        assert e.value.status == simx.EINVAL


@pytest.mark.parametrize("name,ptr", [
    ("action", 4), ("adv", 2), ("logp_old", 1), ("logp_ref", 2), ("weight", 2), ("logp", 3), ("entropy", 2), ("stats", 2)])
def test_misaligned_rows_of_the_token_loss(lib, name, ptr):
    a, b = _logits(), _token(**{name: FAKE + ptr})
    _refused(lib, lib.simx_token_loss_grad(C.byref(a), C.byref(b), FAKE, 1 << 30, None))


@pytest.mark.parametrize("name,ptr", [
    ("token", 4), ("seq_start", 4), ("logp_ref", 2), ("weight", 2), ("ratio", 1), ("margin", 2), ("stats", 3)])
def test_misaligned_rows_of_the_preference_loss(lib, name, ptr):
    d = dict(token=FAKE, seq_start=FAKE, pairs=2, beta=0.1, stats=FAKE)
    d[name] = FAKE + ptr
    a, b = _logits(), simx.PreferenceLoss(**d)
    _refused(lib, lib.simx_preference_loss_grad(C.byref(a), C.byref(b), FAKE, 1 << 30, None))


@pytest.mark.parametrize("name", ["bias", "h0", "h_last", "dh_last", "dbias", "dh0"])
def test_misaligned_states_of_the_scan(lib, name):
    s = _scan(**{name: FAKE + 2})
    _refused(lib, lib.simx_gated_scan(C.byref(s), None, 0, None))
    _refused(lib, lib.simx_gated_scan_grad(C.byref(s), FAKE, 1 << 30, None))


@pytest.mark.parametrize("name", ["gain", "rstd", "dgain"])
def test_misaligned_rows_of_the_norm(lib, name):
    a = _norm(**{name: FAKE + 2})
    _refused(lib, lib.simx_dropout_add_norm(C.byref(a), None))
    _refused(lib, lib.simx_dropout_add_norm_grad(C.byref(a), FAKE, 1 << 30, None))


@pytest.mark.parametrize("sb,st", [(-4, 1), (4, -1), (1 << 41, 1), (4, 1 << 41)])
def test_strides_of_episode_ends(lib, sb, st):
    s = _scan(done=FAKE, done_sb=sb, done_st=st)
    _refused(lib, lib.simx_gated_scan(C.byref(s), None, 0, None))
    _refused(lib, lib.simx_gated_scan_grad(C.byref(s), FAKE, 1 << 30, None))


def _leaves(value):
    for name, kind in type(value)._fields_:
        v = getattr(value, name)
        yield from _leaves(v) if issubclass(kind, C.Structure) else [v]


@pytest.mark.parametrize("image,cls", [
    (simx._logits_image, simx.Logits), (simx._token_loss_image, simx.TokenLoss),
    (simx._preference_loss_image, simx.PreferenceLoss), (simx._scan_image, simx.Scan), (simx._norm_image, simx.Norm)])
def test_packed_images_are_the_structures(image, cls):
    n = len(list(_leaves(cls())))
    assert list(_leaves(cls.from_buffer_copy(image(*range(1, n + 1))))) == list(range(1, n + 1))
    for bad in (1e40, 1 << 70, "x"):  # beyond every field, or no number
        with pytest.raises(simx.SimxError) as e:
            image(*[bad] * n)
        assert e.value.status == simx.EINVAL


@pytest.mark.parametrize("t", [3e-39, 3.5e-39, 4.2e-39])
def test_temperatures_whose_scale_is_beyond_fp32(lib, t):
    """1 / t is finite in fp32, log2(e) / t is not: equal logits would give 0 times infinity."""
    a, b = _logits(temperature=t), _token()
    assert a.temperature > 0 and 1 / a.temperature < 3.4028235e38 < 1.442695 / a.temperature
    _refused(lib, lib.simx_token_loss_grad(C.byref(a), C.byref(b), FAKE, 1 << 30, None))
    p = simx.PreferenceLoss(token=FAKE, seq_start=FAKE, pairs=2, beta=0.1, stats=FAKE)
    _refused(lib, lib.simx_preference_loss_grad(C.byref(a), C.byref(p), FAKE, 1 << 30, None))
