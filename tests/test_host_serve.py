"""The rotation's table, the paged cache's addresses and the refusals that need
no GPU.  CPU only."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2407_16847_amd as splat

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def frequencies(R, base=10000.0, factor=1.0, ramp=None, original=0):
    f = base ** (-np.arange(0, R, 2, dtype=np.float64) / R)
    if ramp is None:
        return f / factor
    k = np.clip((original * f / (2 * np.pi) - ramp[0]) / (ramp[1] - ramp[0]), 0, 1)
    return f * k + f / factor * (1 - k)


@pytest.mark.parametrize("kw", [
    dict(max_len=1, rot_dim=16), dict(max_len=70000, rot_dim=32), dict(max_len=300, rot_dim=128, base=5e5),
    dict(max_len=100, rot_dim=64, factor=4.0, magnitude=1.3),
    dict(max_len=5000, rot_dim=96, factor=8.0, ramp=(1.0, 4.0), original_len=1024, interleaved=True)])
def test_table(kw):
    r = splat.Rotary(**kw)
    f = frequencies(kw["rot_dim"], kw.get("base", 10000.0), kw.get("factor", 1.0), kw.get("ramp"),
                    kw.get("original_len", 0))
    a = np.arange(kw["max_len"])[:, None] * f[None, :]
    want = np.stack((np.cos(a), np.sin(a)), -1) * kw.get("magnitude", 1.0)
    # rounded once, half a step of values up to the magnitude; angles of 64 bits
    # carry 2^-53 of up to 70000 and the frequencies' own roundings
    assert np.abs(r.export() - want).max() <= 2.0 ** -24 * kw.get("magnitude", 1.0) + 1e-10


@pytest.mark.parametrize("kw", [
    dict(max_len=0, rot_dim=16), dict(max_len=(1 << 20) + 1, rot_dim=16), dict(max_len=8, rot_dim=0),
    dict(max_len=8, rot_dim=24), dict(max_len=8, rot_dim=144), dict(max_len=8, rot_dim=16, base=1.0),
    dict(max_len=8, rot_dim=16, base=float("nan")), dict(max_len=8, rot_dim=16, base=float("inf")),
    dict(max_len=8, rot_dim=16, factor=0.5), dict(max_len=8, rot_dim=16, factor=float("inf")),
    dict(max_len=8, rot_dim=16, magnitude=0.0), dict(max_len=8, rot_dim=16, magnitude=float("nan")),
    dict(max_len=8, rot_dim=16, ramp=(-1.0, 4.0), original_len=8),
    dict(max_len=8, rot_dim=16, ramp=(1.0, float("inf")), original_len=8),
    dict(max_len=8, rot_dim=16, ramp=(1.0, 4.0))])
def test_table_refusals(kw):
    with pytest.raises(splat.SplatError) as e:
        splat.Rotary(**kw)
    assert e.value.name == "INVALID_ARG"


def test_more_refusals():
    with pytest.raises(ValueError):
        splat.Rotary(8, 16, ramp=(4.0, 4.0), original_len=8)
    lib = splat.load()
    assert lib.splat_rotary_build(None, ctypes.byref(ctypes.c_void_p())) == 1
    assert lib.splat_rotary_export(None, None) == 1
    lib.splat_rotary_destroy(None)
    a = splat.Acsr(splat.Pattern.window(64, 4))
    for bad in ((0, 4, 4, 64), (1, 4, 3, 64), (1, 4, 0, 64), (1, 4, 8, 64), (1, 4, 4, 32), (1, 70000, 1, 64)):
        with pytest.raises(splat.SplatError):
            splat.decode_workspace(a, *bad)
    assert splat.decode_workspace(a, 8, 64, 64, 64) == 0
    r = splat.Rotary(8, 16)
    x = torch.zeros(1, 1, 1, 64)
    with pytest.raises(TypeError):
        splat.rotary(r, x)
    with pytest.raises(TypeError):
        splat.cache_append(x, x, x, x, x, x)
    with pytest.raises(TypeError):
        splat.sparse_mhsa_decode(a, x, x, x, x, x, 1.0)
    r.close()
    with pytest.raises(ValueError):
        r.export()


def test_cache_addresses(tmp_path):
    cxx = shutil.which(os.environ.get("CXX", "g++"))
    if cxx is None:
        pytest.fail("a host C++ compiler is needed for the sanitizer build")
    exe = str(tmp_path / "serve_check")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=all", os.path.join(ROOT, "tests", "native", "serve_check.cpp"),
                        "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.returncode, r.stderr[-2000:])


def test_backward_passes_are_not_captured(monkeypatch):
    """A backward pass under capture is refused before anything is launched, and
    positions that change between the passes are noticed."""
    from paper_2407_16847_amd import autograd as sag
    x = torch.zeros(1, 1, 1, 64, requires_grad=True)
    monkeypatch.setattr(sag, "_rotary", lambda rot, X, positions=None, inverse=False: X * 1.0)
    y = sag.rotary(None, x, torch.zeros(1, 1, dtype=torch.int32))
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="not captured"):
        y.sum().backward()
    monkeypatch.undo()
    monkeypatch.setattr(sag, "_rotary", lambda rot, X, positions=None, inverse=False: X * 1.0)
    at = torch.zeros(1, 1, dtype=torch.int32)
    y = sag.rotary(None, x, at)
    at += 1
    with pytest.raises(RuntimeError, match="modified"):
        y.sum().backward()
