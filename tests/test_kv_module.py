"""The C++ module of the key-value cache's usual calls is a short cut: without it
the package imports, the library is built, and the calls give the same bits."""
import importlib.util
import os
import subprocess
import sys
import warnings

import pytest
import torch

import paper_1402_3788_amd as km

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

IMPORT = """
import sys, types
module = {module}
sys.modules["paper_1402_3788_amd._kv_call"] = module
import paper_1402_3788_amd as km
assert km.kv._fast is None
assert km.kmeans_workspace_bytes(1000, 25, 16) > 0 and km.strerror(0)
print(km.kv._without)
"""


def build_script():
    spec = importlib.util.spec_from_file_location(
        "_kv_build", os.path.join(ROOT, "paper_1402_3788_amd", "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_the_module_is_there():
    assert km.kv._fast is not None, km.kv._without
    assert os.path.basename(km.kv._fast.__file__) == os.path.basename(build_script().CALLS)


@pytest.mark.parametrize("module,why", [
    ("None", "_kv_call"),                                       # as if it were not there
    ("types.ModuleType('m')", "not built for torch " + torch.__version__),
])
def test_import_without_it(module, why):
    got = subprocess.run([sys.executable, "-c", IMPORT.format(module=module)], cwd=ROOT,
                         capture_output=True, text=True)
    assert got.returncode == 0, got.stderr
    assert why in got.stdout


def no_torch(out):
    raise ImportError("no torch here")


@pytest.mark.parametrize("command,why", [
    (no_torch, "no torch here"),
    (lambda out: ["/nowhere/g++", out], "nowhere"),
    (lambda out: [sys.executable, "-c", "import sys; sys.exit('Python.h: not found')"],
     "Python.h: not found"),
])
def test_build_without_it(tmp_path, monkeypatch, capsys, command, why):
    """What the module needs is missing: told, not raised, and no old module stays."""
    build = build_script()
    old = tmp_path / "_kv_call.so"
    old.write_bytes(b"of earlier sources")
    monkeypatch.setattr(build, "CALLS", str(old))
    monkeypatch.setattr(build, "calls_command", command)
    assert build._finish_calls(build._start_calls()) is False
    assert not old.exists()
    assert why in capsys.readouterr().err


@pytest.mark.gpu
def test_the_same_bits_without_it(monkeypatch):
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(0)
    centres = [torch.randn(2, 16, 256, 4, generator=g).to(torch.bfloat16).to(dev)
               for _ in range(2)]
    k, v = (torch.randn(70, 2, 64, generator=g).to(torch.bfloat16).to(dev) for _ in range(2))
    q = torch.randn(2, 8, 64, generator=g).to(torch.bfloat16).to(dev)
    slots = torch.arange(70, device=dev)
    table = torch.tensor([[0, 1, 2, 3, 4], [4, 3, 2, 1, 0]], dtype=torch.int32, device=dev)
    lengths = torch.tensor([70, 11], dtype=torch.int32, device=dev)

    def all_calls():
        cache = km.KVCodes.empty(*centres, 5, 16)
        km.kmeans_kv_write(cache, k, v, slots)
        return (cache.k_codes, cache.v_codes, *km.kmeans_kv_read(cache, slots),
                *km.kmeans_kv_attend(cache, q, table, lengths))

    with warnings.catch_warnings():
        warnings.simplefilter("error")
        want = all_calls()
    monkeypatch.setattr(km.kv, "_fast", None)
    with pytest.warns(RuntimeWarning, match="_kv_call"):
        got = all_calls()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
