"""What the build takes for up to date, with the compilers' runs noted instead of made."""
import os

import pytest


@pytest.fixture
def build(tmp_path, monkeypatch):
    """The build module in an empty place, with a torch of its own and compilers that only make their output files."""
    from paper_1905_00689_gb300 import build as b
    torch = tmp_path / "torch"
    torch.mkdir()
    (torch / "version.py").write_text("__version__ = '1'\n")
    for name in ("LIB", "MODULE", "MODULE_FOR"):
        if hasattr(b, name):
            monkeypatch.setattr(b, name, str(tmp_path / "_build" / os.path.basename(getattr(b, name))))
    monkeypatch.setattr(b, "BUILD", str(tmp_path / "_build"))
    b.found_torch_dir = b._torch_dir
    monkeypatch.setattr(b, "_torch_dir", lambda: str(torch))
    runs = []

    def run(cmd, what, verbose=False):
        runs.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
    monkeypatch.setattr(b, "_run", run)
    monkeypatch.setattr(b, "_nvcc", lambda: "/usr/local/cuda/bin/nvcc")
    b.runs, b.torch = runs, torch
    yield b
    del b.runs, b.torch, b.found_torch_dir


def test_built_once(build):
    assert not build.up_to_date()
    build.build()
    assert build.up_to_date() and any("g++" in c[0] for c in build.runs)
    build.runs.clear()
    build.build()
    assert build.runs == []


def test_another_torch_needs_another_module(build):
    """The module links against torch's libraries: after a change of torch it is built again, though no source has
    changed."""
    build.build()
    build.runs.clear()
    (build.torch / "version.py").write_text("__version__ = '2'\n")
    assert not build.up_to_date()
    build.build()
    assert any("torch_ops.cpp" in " ".join(c) for c in build.runs) and build.up_to_date()


def test_the_library_needs_no_torch(build, monkeypatch):
    """Without a torch the library is built as ever; the module, which only torch's users load, is left out until there
    is one."""
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    monkeypatch.setattr(build, "_torch_dir", build.found_torch_dir)
    build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.MODULE) and build.up_to_date()
    assert not any("g++" in c[0] for c in build.runs)
    monkeypatch.setattr(build, "_torch_dir", lambda: str(build.torch))
    assert not build.up_to_date()
    build.build()
    assert os.path.exists(build.MODULE) and build.up_to_date()


def test_the_library_is_there_where_the_module_fails(build, monkeypatch):
    plain = build._run

    def run(cmd, what, verbose=False):
        if "torch_ops.cpp" in " ".join(cmd):
            raise RuntimeError(what)
        plain(cmd, what, verbose)
    monkeypatch.setattr(build, "_run", run)
    with pytest.raises(RuntimeError, match="torch_ops.cpp"):
        build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.MODULE) and not build.up_to_date()
