"""Building and loading the argument marshalling (_marshal.so), apart from the library itself."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2601_11676_b200 import binding as B
from paper_2601_11676_b200 import build


@pytest.fixture(scope="module")
def built():
    return build.build()


def call():
    """A call through the marshalling that is refused for its tensors, once they are looked at."""
    with pytest.raises(ValueError):
        B.halo_quantize_rows_mx4(128, 1, B.F32, torch.zeros((1, 128)), torch.zeros((1, 64), dtype=torch.uint8),
                                 torch.zeros(512, dtype=torch.uint8))


def test_marshalling_made_for_another_torch_is_not_loaded(built, monkeypatch):
    monkeypatch.setattr(B, "_native", None)
    call()
    monkeypatch.setattr(B, "_native", None)
    monkeypatch.setattr(torch, "__version__", "2.99.0")
    with pytest.raises(ImportError, match="2.99.0.*paper_2601_11676_b200.build"):
        call()


def test_missing_marshalling_says_how_to_build_it(built, monkeypatch):
    monkeypatch.setattr(B, "_native", None)
    monkeypatch.setitem(sys.modules, "paper_2601_11676_b200._marshal", None)
    with pytest.raises(ImportError, match="paper_2601_11676_b200.build"):
        call()


def test_library_builds_where_the_marshalling_cannot(built, monkeypatch, tmp_path):
    """No host compiler of its own, or no headers: the library stands, no outdated module stays, the reason is told."""
    old = tmp_path / "_marshal.so"
    old.write_bytes(b"")
    monkeypatch.setattr(build, "MARSHAL", str(old))
    monkeypatch.setattr(build, "OBJ", str(tmp_path))
    real = subprocess.run

    def run(cmd, *args, **kw):
        if cmd[0] == "g++":
            raise FileNotFoundError("g++")
        return real(cmd, *args, **kw)

    monkeypatch.setattr(subprocess, "run", run)
    monkeypatch.setattr(build, "sources", lambda: [])
    with pytest.warns(UserWarning, match="g\\+\\+"):
        assert build.build() == build.LIB
    assert os.path.exists(build.LIB) and not old.exists()
