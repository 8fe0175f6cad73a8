"""The CPython module of the small calls is optional: where it cannot be built or loaded the binding does without it."""
import os
import shutil
import subprocess
import sys
from pathlib import Path

import pytest

from paper_2509_22951_b200 import binding as tq
from paper_2509_22951_b200 import build

ROOT = Path(build.__file__).resolve().parent.parent


@pytest.fixture
def copy(tmp_path):
    """The package without built files; the library is the one that is built here."""
    for d in ("paper_2509_22951_b200", "include"):
        shutil.copytree(ROOT / d, tmp_path / d, ignore=shutil.ignore_patterns("*.so", "__pycache__"))
    return tmp_path


def _import(at, path=None, code="", **env):
    code = "import paper_2509_22951_b200.binding as b; assert b.__file__.startswith(%r); " % str(at) + (code or "print('fast', b._fast is not None)")
    env = dict(os.environ, TQ_LIBTQ=str(build.LIB), PYTHONPATH=str(at), **env)
    if path:
        env["PATH"] = f"{path}:{env['PATH']}"
    return subprocess.run([sys.executable, "-W", "always", "-c", code], cwd=at, env=env, capture_output=True, text=True)


def _compiler(at, script):
    d = at / "bin"
    d.mkdir()
    (d / "g++").write_text("#!/bin/sh\n" + script)
    (d / "g++").chmod(0o755)
    return d


def test_a_compiler_that_fails(copy):
    r = _import(copy, _compiler(copy, "echo no such interface >&2; exit 1\n"))
    assert r.returncode == 0 and "fast False" in r.stdout and "go through Python" in r.stderr, r.stderr
    assert not list((copy / "paper_2509_22951_b200").glob("*.so"))


def test_a_module_that_does_not_load(copy):
    """A compiler that ends well and leaves what is no module."""
    r = _import(copy, _compiler(copy, 'for a; do last=$a; done; echo nothing > "$last"\n'))
    assert r.returncode == 0 and "fast False" in r.stdout and "not loaded" in r.stderr, r.stderr


def test_a_compiler_that_cannot_write(copy):
    """As where the package lies in a folder that cannot be written: nothing is there to be moved to its place."""
    r = _import(copy, _compiler(copy, "exit 0\n"))
    assert r.returncode == 0 and "fast False" in r.stdout, r.stderr


def test_the_file_is_that_of_this_interpreter_and_torch(copy, monkeypatch):
    import sysconfig

    import torch
    name = build.fast_path().name
    assert sysconfig.get_config_var("SOABI") in name and torch.__version__ in name
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build.fast_path().name != name
    shutil.which("g++") or pytest.skip("no g++")
    r = _import(copy)
    assert r.returncode == 0 and "fast True" in r.stdout, r.stderr
    assert [p.name for p in (copy / "paper_2509_22951_b200").glob("*.so")] == [name]


def test_force_says_what_is_wrong(monkeypatch, tmp_path):
    monkeypatch.setattr(build, "PKG", tmp_path)
    monkeypatch.setenv("PATH", str(_compiler(tmp_path, "exit 1\n")) + ":" + os.environ["PATH"])
    with pytest.raises(subprocess.CalledProcessError):
        build.build_fast(force=True)
    with pytest.warns(RuntimeWarning):
        assert build.build_fast() is None
    with pytest.warns(RuntimeWarning):
        assert tq._load_fast() is None


def test_a_torch_without_cuda_still_imports_the_binding():
    code = "import torch\nfor n in ('_cuda_getCurrentRawStream', '_cuda_getDevice'): delattr(torch._C, n)\n" \
           "import paper_2509_22951_b200.binding as b, numpy as np\nassert b._fast is None\n" \
           "q, s = b.tq_quantize_rows(np.ones((2, 8), np.float32)); print(int(q[0, 0]))"
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.split() == ["127"], r.stderr
