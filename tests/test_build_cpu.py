"""Building the library: what a failed link says, which step gets the caller's flags, and where the objects are, with a stand-in
for the compiler."""
import os
import subprocess
import sys

import pytest

from paper_2007_14152_amd import build as hip_build

COMPILER = """#!%s
import os, sys
args = sys.argv[1:]
out = args[args.index("-o") + 1]
with open(os.environ["CALLS"], "a") as f:
    f.write(repr(args) + "\\n")
if "-c" not in args and os.environ.get("FAIL") == "link":
    sys.stderr.write("undefined symbol: the_symbol\\n")
    sys.exit(1)
if "-c" in args and os.environ.get("FAIL") == "compile" and args[args.index("-c") + 1].endswith("rows.hip"):
    sys.stderr.write("error: the_error\\n")
    sys.exit(1)
for kernel in %r:
    sys.stderr.write("x: remark: Function Name: %%s\\n" %% kernel)
    for figure in ("ScratchSize [bytes/lane]", "LDS Size [bytes/block]"):
        sys.stderr.write("x: remark:     %%s: 0\\n" %% figure)
open(out, "w").write(str(len(args)))
"""


@pytest.fixture
def stand_in(tmp_path, monkeypatch):
    exe = tmp_path / "compiler"
    exe.write_text(COMPILER % (sys.executable, hip_build.NO_SCRATCH_KERNELS + hip_build.LDS_FROM_ZERO_KERNELS))
    exe.chmod(0o755)
    csrc = tmp_path / "csrc"
    csrc.mkdir()
    sources = [str(csrc / os.path.basename(s)) for s in hip_build.SOURCES]
    for s in sources:
        open(s, "w").close()
    monkeypatch.setenv("HIPCC", str(exe))
    monkeypatch.setenv("CALLS", str(tmp_path / "calls"))
    monkeypatch.setattr(hip_build, "CSRC", str(csrc))
    monkeypatch.setattr(hip_build, "SOURCES", sources)
    monkeypatch.setattr(hip_build, "LIB", str(csrc / "lib.so"))
    monkeypatch.setattr(hip_build, "ORDER_HOST_LIB", str(csrc / "host.so"))

    def calls():
        return [eval(line) for line in (tmp_path / "calls").read_text().splitlines()]

    return calls, csrc


def left(csrc):
    return sorted(n for n in os.listdir(csrc) if not n.endswith(".hip"))


def test_a_failed_link_says_why_and_leaves_nothing(stand_in, monkeypatch, capfd):
    calls, csrc = stand_in
    (csrc / "lib.so").write_text("the library that was there")
    monkeypatch.setenv("FAIL", "link")
    with pytest.raises(subprocess.CalledProcessError):
        hip_build.build()
    assert "undefined symbol: the_symbol" in capfd.readouterr().err
    assert left(csrc) == ["lib.so"] and (csrc / "lib.so").read_text() == "the library that was there"


def test_a_failed_compilation_says_why_and_leaves_nothing(stand_in, monkeypatch, capfd):
    calls, csrc = stand_in
    monkeypatch.setenv("FAIL", "compile")
    with pytest.raises(subprocess.CalledProcessError):
        hip_build.build()
    assert "error: the_error" in capfd.readouterr().err
    assert left(csrc) == []


def test_flags_of_the_caller_reach_every_step(stand_in):
    calls, csrc = stand_in
    hip_build.build(extra=["-lsome", "-DTHIS"])
    assert len(calls()) == len(hip_build.SOURCES) + 1
    assert all("-lsome" in c and "-DTHIS" in c for c in calls())
    assert left(csrc) == ["host.so", "lib.so"]


def test_two_builds_do_not_share_a_file_that_is_being_written(stand_in):
    calls, csrc = stand_in
    hip_build.build()
    hip_build.build()
    written = [c[c.index("-o") + 1] for c in calls()]
    assert len(set(written)) == len(written) == 2 * (len(hip_build.SOURCES) + 1)
    assert str(csrc / "lib.so") not in written
