"""What the build makes, and in which order: with fakes of the compiler and the linker (no GPU)."""
import os
import sysconfig

import pytest


@pytest.fixture
def fake(aatc, monkeypatch, tmp_path):
    """The build module with its products in an empty folder; `log` is what was compiled and linked."""
    from paper_2608_14191_gb300 import build as b
    log = []
    for name in ("LIB", "CALLS", "BUILD"):
        monkeypatch.setattr(b, name, str(tmp_path / os.path.basename(getattr(b, name))))
    monkeypatch.setattr(b, "_compile", lambda src, verbose: log.append(src) or src)

    def link(out, args):
        log.append(os.path.basename(out))
        open(out, "w").close()

    monkeypatch.setattr(b, "_link", link)
    b.log = log
    yield b
    del b.log


def test_library_and_extension(fake):
    assert fake.build() == fake.LIB
    assert sorted(fake.log) == sorted(fake.SOURCES + [fake.CALLS_SOURCE, "libaatc.so", os.path.basename(fake.CALLS)])
    fake.log.clear()
    assert fake.build() == fake.LIB and fake.log == []             # up to date
    os.remove(fake.CALLS)
    fake.build()
    assert os.path.basename(fake.CALLS) in fake.log


def test_library_without_python_headers(fake, monkeypatch, tmp_path, capsys):
    """The library needs no Python: it is linked, and up to date afterwards."""
    monkeypatch.setattr(sysconfig, "get_paths", lambda real=sysconfig.get_paths: {**real(), "include": str(tmp_path / "none")})
    assert fake.build() == fake.LIB
    assert sorted(fake.log) == sorted(fake.SOURCES + ["libaatc.so"])
    assert "headers" in capsys.readouterr().err
    fake.log.clear()
    assert fake.build() == fake.LIB and fake.log == []


def test_extension_that_fails_leaves_the_library(fake, monkeypatch):
    def compile_(src, verbose):
        if src == fake.CALLS_SOURCE:
            raise RuntimeError("nvcc failed")
        return src

    monkeypatch.setattr(fake, "_compile", compile_)
    with pytest.raises(RuntimeError, match="nvcc failed"):
        fake.build()
    assert os.path.exists(fake.LIB) and not os.path.exists(fake.CALLS)


def test_extension_has_the_interpreters_name(aatc):
    from paper_2608_14191_gb300 import _calls, build
    assert os.path.basename(build.CALLS) == "_calls" + sysconfig.get_config_var("EXT_SUFFIX")
    assert os.path.samefile(_calls.__file__, build.CALLS)
