"""CPU tests of the native calls as modules: the codec's stand without torch's libraries, and without those of the layer calls."""
import os
import shutil
import sys
import sysconfig

import pytest

from paper_2502_18554_amd import binding as b
from paper_2502_18554_amd import build

SUFFIX = sysconfig.get_config_var("EXT_SUFFIX")


def test_the_codecs_calls_are_not_linked_to_torch(monkeypatch, tmp_path):
    ran = []
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_zc_calls.so"))
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, check: ran.append(cmd))
    build.build_calls()
    if not ran:
        pytest.skip("no headers of this Python or no g++")
    (cmd,) = ran
    assert not [a for a in cmd if "torch" in a or a.startswith("-lc10") or "zc_layer_calls" in a]


def test_the_layers_calls_are_built_beside_them(monkeypatch, tmp_path):
    ran = []
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_zc_calls.so"))
    monkeypatch.setattr(build, "LAYER_CALLS", str(tmp_path / "_zc_layer_calls.so"))
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, check: ran.append(cmd))
    (tmp_path / "_zc_layer_calls.so").write_bytes(b"of other sources")
    assert build.build_all() == build.LIB
    if len(ran) < 3:
        pytest.skip("no headers of this Python or of torch, or no g++")
    assert [cmd[cmd.index("-o") + 1] for cmd in ran] == [build.LIB, build.CALLS, build.LAYER_CALLS]
    assert not (tmp_path / "_zc_layer_calls.so").exists()
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)           # (no torch)
    ran.clear()
    build.build_all()
    assert len(ran) == 2


@pytest.mark.parametrize("layers", [None, b"built elsewhere"])
def test_layer_calls_that_do_not_load_leave_the_codecs(monkeypatch, tmp_path, layers):
    L = b.lib()
    if b._native is None or b._native_layers is None:
        pytest.skip("the native calls are not built")
    shutil.copy(os.path.join(b._HERE, "_zc_calls" + SUFFIX), tmp_path / ("_zc_calls" + SUFFIX))
    if layers:
        (tmp_path / ("_zc_layer_calls" + SUFFIX)).write_bytes(layers)
    monkeypatch.setattr(b, "_HERE", str(tmp_path))
    monkeypatch.setattr(b, "_native", None)
    monkeypatch.setattr(b, "_native_layers", None)
    monkeypatch.setattr(sys, "modules", dict(sys.modules))
    b._load_native(L)
    assert b._native is not None and b._native_layers is None
