"""What the build needs for which of its two libraries, and when the paged calls' marshalling counts as out of date.  The
compilers are stand-ins that write the file they are asked for."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def tree(tmp_path):
    """A copy of what the build reads, and a PATH whose nvcc and g++ only write their output."""
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    shutil.copytree(os.path.join(ROOT, "paper_2502_17599_b200", "csrc"), tmp_path / "pkg" / "csrc")
    shutil.copy(os.path.join(ROOT, "paper_2502_17599_b200", "build.py"), tmp_path / "pkg")
    tools = tmp_path / "tools"
    tools.mkdir()
    for name in ("nvcc", "g++"):
        tool = tools / name
        tool.write_text(f"""#!{sys.executable}
import sys
open({str(tmp_path)!r} + "/calls", "a").write("{name}\\n")
if "{name}" in open({str(tmp_path)!r} + "/broken").read().split():
    sys.exit(1)
text = [a.split("=", 1)[1].strip('"') for a in sys.argv if a.startswith("-DMEDA_BUILT_FOR=")]
open(sys.argv[sys.argv.index("-o") + 1], "wb").write("".join(text).encode() + b"\\0")
""")
        tool.chmod(0o755)
    (tmp_path / "broken").write_text("")
    return tmp_path


def run(tree, *, torch=True, broken="", version=None, args=()):
    (tree / "broken").write_text(broken)
    (tree / "calls").write_text("")
    code = f"import runpy, sys; sys.argv = ['build.py'] + {list(args)!r}\n"
    if not torch:
        code += ("import importlib.util as u; find = u.find_spec\n"
                 "u.find_spec = lambda name, *a: None if name == 'torch' else find(name, *a); sys.modules['torch'] = None\n")
    elif version:
        code += f"import torch; torch.__version__ = {version!r}\n"
    code += f"runpy.run_path({str(tree / 'pkg' / 'build.py')!r}, run_name='__main__')"
    env = dict(os.environ, PATH=f"{tree / 'tools'}:{os.environ['PATH']}")
    r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True)
    return r, (tree / "calls").read_text().split()


def test_the_library_is_built_without_torch(tree):
    r, calls = run(tree, torch=False)
    assert r.returncode == 0, r.stderr
    assert calls == ["nvcc"] and (tree / "pkg" / "libmeda.so").exists() and not (tree / "pkg" / "_pages.so").exists()
    assert "_pages.so" in r.stderr


def test_a_failing_marshalling_build_leaves_the_library(tree):
    r, calls = run(tree, broken="g++")
    assert r.returncode != 0 and "g++ failed" in r.stderr
    assert calls == ["nvcc", "g++"] and (tree / "pkg" / "libmeda.so").exists()


def test_nothing_is_built_twice_and_another_torch_rebuilds_the_marshalling(tree):
    assert run(tree)[1] == ["nvcc", "g++"]
    assert run(tree)[1] == []
    assert run(tree, version="9.8.7")[1] == ["g++"]
    assert run(tree, version="9.8.7")[1] == []
    assert run(tree, version="9.8")[1] == ["g++"]                  # (not a beginning of the other)
    assert run(tree)[1] == ["g++"]
    assert run(tree, args=["--force"])[1] == ["nvcc", "g++"]


def test_a_marshalling_library_of_another_torch_is_not_loaded(monkeypatch):
    from paper_2502_17599_b200 import binding, build
    build.build()
    monkeypatch.setattr(binding, "_NATIVE", None)
    monkeypatch.setattr(build, "binding_tag", lambda: b"built for torch 0.0.0, none")
    with pytest.raises(RuntimeError, match="another torch"):
        binding.load_native()
