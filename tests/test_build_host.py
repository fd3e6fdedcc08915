"""What build() compiles: the library needs hipcc alone, as for callers of its C
interface without PyTorch."""
import sys

import pytest

from paper_2304_13724_amd import build


@pytest.fixture
def compiled(monkeypatch):
    done = []
    monkeypatch.setattr(build, "_compile", lambda cmd, out, verbose: done.append(out))
    return done


def test_with_pytorch(compiled):
    assert build.build() == build.LIB
    assert compiled == [build.LIB, build.TENSORS]


def test_without_pytorch(compiled, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)  # importing it raises ImportError
    assert build.build() == build.LIB
    assert compiled == [build.LIB]
    assert "_ranking.so" in capsys.readouterr().err
    with pytest.raises(ImportError):
        build.build_tensors()


def test_a_compiler_s_failure_is_not_passed_over(monkeypatch):
    def fail(cmd, out, verbose):
        if out == build.TENSORS:
            raise RuntimeError("g++ failed")
    monkeypatch.setattr(build, "_compile", fail)
    with pytest.raises(RuntimeError):
        build.build()
