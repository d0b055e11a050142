"""What the library needs to be built and loaded (no GPU): the solver needs nvcc alone; the Python extension of the operators on
4-bit codes is built where they are first used."""
import os
import sys

import pytest


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """The extension's built file in a folder where there is none yet."""
    from paper_2608_18147_gb300 import build
    build.build()
    monkeypatch.setattr(build, "BINDING", str(tmp_path / os.path.basename(build.BINDING)))
    return build


def test_the_library_does_not_need_a_c_compiler(elsewhere, monkeypatch):
    monkeypatch.setenv("CC", "/nonexistent/cc")
    assert elsewhere.build() == elsewhere.LIB
    assert not os.path.exists(elsewhere.BINDING)
    with pytest.raises(RuntimeError, match="/nonexistent/cc"):
        elsewhere.build_binding()


def test_the_library_does_not_need_the_extensions_source(elsewhere, monkeypatch, tmp_path):
    monkeypatch.setattr(elsewhere, "BINDING_SRC", str(tmp_path / "binding.c"))
    assert elsewhere.build() == elsewhere.LIB
    with pytest.raises(RuntimeError, match="binding.c"):
        elsewhere.build_binding()
    with open(elsewhere.BINDING, "wb"):  # built elsewhere and shipped without its source: taken as it is
        pass
    assert elsewhere.build_binding() == elsewhere.BINDING


def test_a_compiler_of_several_words(elsewhere, monkeypatch):
    monkeypatch.setenv("CC", (os.environ.get("CC") or "gcc") + " -pthread")
    path = elsewhere.build_binding()
    assert os.path.exists(path)
    built = os.path.getmtime(path)
    assert elsewhere.build_binding() == path and os.path.getmtime(path) == built


def test_a_process_without_a_compiler_uses_the_solver(elsewhere, tmp_path):
    """The library loads in a fresh process that has neither a C compiler nor the extension."""
    import subprocess
    src = ("from paper_2608_18147_gb300 import build, native\n"
           "build.BINDING = %r\n"
           "assert native.lib().ecasq_version() > 0\n" % elsewhere.BINDING)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", src], cwd=root, env=dict(os.environ, CC="/nonexistent/cc"), capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
