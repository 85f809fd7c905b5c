"""The part of the binding that is in C: built for the interpreter that asks, with its compiler, and needed by its own calls alone."""
import os
import subprocess
import sys
import sysconfig

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def python(code, **env):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, env={**os.environ, **env}, capture_output=True, text=True)


def test_the_file_is_this_interpreters():
    from paper_2403_18647_gb300 import build as b
    assert os.path.basename(b.NATIVE) == "_native" + sysconfig.get_config_var("EXT_SUFFIX")
    import paper_2403_18647_gb300 as sd
    sd._types()
    assert os.path.samefile(sd._calls.__file__, b.NATIVE)


def test_other_calls_do_not_need_it():
    """Without the extension the library loads, tensors are checked, and only the calls that are in C raise."""
    r = python("""
import sys
sys.modules["paper_2403_18647_gb300._native"] = None            # (an import of it raises)
import torch
import paper_2403_18647_gb300 as sd
assert sd.lib().sdsat_status_string(0) == b"ok"
for call in (lambda: sd._rows(torch.zeros(2, 3)), lambda: sd._array(torch.zeros(3), sd._f32, 3)):
    try:
        call()
    except ValueError:
        pass
    else:
        raise SystemExit("a host tensor was taken")
try:
    sd.Context.op_chunk_attention(None, *[None] * 10)
except ImportError:
    print("as it should be")
""")
    assert r.returncode == 0 and r.stdout.strip() == "as it should be", r.stderr


def test_the_compiler_may_be_chosen(tmp_path, monkeypatch):
    from paper_2403_18647_gb300 import build as b
    monkeypatch.setattr(b, "NATIVE", str(tmp_path / "_native.so"))
    monkeypatch.setenv("CC", "/nowhere/compiler -pipe")
    assert b.cc() == ["/nowhere/compiler", "-pipe"]
    with pytest.raises(RuntimeError):
        b.build_native()
    monkeypatch.delenv("CC")
    assert b.build_native() == b.NATIVE and os.path.exists(b.NATIVE)
    monkeypatch.setattr(b.sysconfig, "get_config_var", lambda name: "/nowhere/compiler")
    assert b.cc() == ["cc"]
