"""The binding's reader of lists of tensors is host code that knows torch's classes: one that was built with another torch is refused, not called, and where it cannot be
built at all the kernels' library is there all the same."""
import os

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def B():
    from paper_2305_09887_amd import binding, build
    if not os.path.exists(build.LISTS):
        build.build_lists()
    binding._lists.cache_clear()
    yield binding
    binding._lists.cache_clear()


def test_the_torch_that_it_was_built_with(B, monkeypatch):
    B._lists()
    B._lists.cache_clear()
    monkeypatch.setattr(torch, "__version__", "1.2.3+other")
    with pytest.raises(B.TmaError, match=r"built with torch .*1\.2\.3\+other"):
        B._lists()


def test_a_file_that_cannot_be_loaded(B, monkeypatch, tmp_path):
    monkeypatch.setattr(B, "_PKG", str(tmp_path))
    with pytest.raises(B.TmaError, match="not found"):
        B._lists()
    (tmp_path / "libtma_lists.so").write_bytes(b"no library")
    with pytest.raises(B.TmaError, match="libtma_lists.so"):
        B._lists()


def test_the_kernels_library_without_it(monkeypatch, tmp_path):
    from paper_2305_09887_amd import build
    linked = []

    def no_compiler():
        raise FileNotFoundError("g++")

    monkeypatch.setattr(build, "OBJ", str(tmp_path))
    monkeypatch.setattr(build, "_compile", lambda src: src + ".o")
    monkeypatch.setattr(build, "build_lists", no_compiler)
    monkeypatch.setattr(build.subprocess, "check_call", lambda command, **_: linked.append(command))
    with pytest.raises(FileNotFoundError):
        build.build(verbose=False)
    assert len(linked) == 1 and build.LIB in linked[0] and "-shared" in linked[0]
