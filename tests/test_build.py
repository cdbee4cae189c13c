"""How the library and the native half of the operators' binding are built (no GPU, no compiler run)."""
import os
import subprocess

import pytest

from paper_2608_02611_b200 import build


@pytest.fixture
def no_native(tmp_path, monkeypatch):
    """A tree whose _kb_torch.so is missing and cannot be built; the library itself is up to date."""
    build.build()
    monkeypatch.setattr(build, "NATIVE", str(tmp_path / "_kb_torch.so"))

    def run(cmd, **kw):
        assert cmd[0] == "g++"
        raise failure[0]

    failure = [FileNotFoundError("g++")]
    monkeypatch.setattr(build.subprocess, "run", run)
    return failure


@pytest.mark.parametrize("error", [FileNotFoundError("g++"), subprocess.CalledProcessError(1, "g++")])
def test_the_gate_builds_where_the_operators_binding_does_not(no_native, error):
    no_native[0] = error
    with pytest.warns(UserWarning, match="the gate works without it"):
        assert build.build() == build.LIB
    with pytest.raises(type(error)):
        build.build_native()


def test_the_binding_is_built_again_for_another_torch(tmp_path, monkeypatch):
    native = tmp_path / "_kb_torch.so"
    monkeypatch.setattr(build, "NATIVE", str(native))
    assert build.native_stale()
    native.write_bytes(b"..." + build.native_marker().encode() + b"\0...")
    assert not build.native_stale()
    os.utime(native, (0, 0))
    assert build.native_stale()                     # older than its source
    native.write_bytes(b"..." + build.native_marker().encode() + b"1\0...")
    assert build.native_stale()                     # 2.1 is not 2.11
    import torch
    native.write_bytes(b"..." + build.native_marker().encode() + b"\0...")
    monkeypatch.setattr(torch, "__version__", "1.0.0")
    assert build.native_stale()


def test_the_built_binding_names_what_it_was_built_for():
    build.build_native()
    from paper_2608_02611_b200 import _kb_torch
    assert _kb_torch.built_for == build.native_marker() and not build.native_stale()
