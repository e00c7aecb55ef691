"""What a variant of the library is built with."""
import os
import subprocess

from paper_2502_11034_amd import build as lib_build


def test_extra_flags_reach_every_compiler_and_the_linker(monkeypatch, tmp_path):
    commands = []

    def run(cmd, **_):
        commands.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(subprocess, "run", run)
    out = str(tmp_path / "variant.so")
    assert lib_build.build(extra_flags=iter(["-DSOMETHING=1", "-Wl,-Map=map"]), out=out) == out and os.path.exists(out)
    assert len(commands) == len(lib_build.SOURCES) + 1
    for cmd in commands:
        assert "-DSOMETHING=1" in cmd and "-Wl,-Map=map" in cmd
    link = commands[-1]
    assert "-shared" in link and "-c" not in link
    compiled = sorted(cmd[cmd.index("-c") + 1] for cmd in commands[:-1])
    assert compiled == sorted(os.path.join(lib_build.CSRC, s) for s in lib_build.SOURCES)
    assert sorted(cmd[cmd.index("-o") + 1] for cmd in commands[:-1]) == sorted(a for a in link if a.endswith(".o"))
