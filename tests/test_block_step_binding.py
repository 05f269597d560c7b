"""The compiled short way into the calls for single tokens: how it is built and when it is not used (no GPU needed)."""
import os
import struct
import sys

import pytest

from paper_2603_09221_b200 import block, build


@pytest.mark.parametrize("fails", [True, False])
def test_a_build_takes_the_place_of_the_old_file_once_it_is_whole(tmp_path, monkeypatch, fails):
    """Another process may import the module while it is compiled: it finds the old file, or the new one, never a part of it."""
    target, seen = tmp_path / "_step.so", tmp_path / "seen"
    target.write_text("old")
    cxx = tmp_path / "cxx"
    cxx.write_text("""#!%s
import sys
out = sys.argv[sys.argv.index("-o") + 1]
open(out, "w").write("half")
open(%r, "w").write(open(%r).read())
open(out, "w").write("whole")
sys.exit(%d)
""" % (sys.executable, str(seen), str(target), fails))
    cxx.chmod(0o755)
    monkeypatch.setenv("CXX", str(cxx))
    monkeypatch.setattr(build, "STEP", str(target))
    if fails:
        with pytest.raises(Exception):
            build.build_step_binding(force=True)
    else:
        build.build_step_binding(force=True)
        assert os.access(target, os.R_OK | os.X_OK)
    assert seen.read_text() == "old" and target.read_text() == ("old" if fails else "whole")
    assert sorted(p.name for p in tmp_path.iterdir()) == ["_step.so", "cxx", "seen"]


@pytest.mark.parametrize("record", ["_CONV_ARGS", "_SCAN_ARGS", "_LINEAR_ARGS"])
def test_a_module_built_for_other_records_is_not_used(monkeypatch, record):
    lib = block._load()
    assert block._short_way(lib) is not block._LongWay
    monkeypatch.setattr(block, record, struct.Struct(getattr(block, record).format + "q"))
    with pytest.warns(UserWarning, match="records"):
        assert block._short_way(lib) is block._LongWay
