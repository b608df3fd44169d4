"""Flags that a caller adds to the build (SALS_EXTRA_FLAGS) reach every compilation and the link: sanitizers and libraries are wanted at both."""
import subprocess

from paper_2510_24273_amd import build


def test_added_flags_reach_compilations_and_link(monkeypatch, tmp_path):
    ran = []

    class Done:
        def __init__(self, cmd):
            ran.append(cmd)

        def wait(self):
            return 0

    monkeypatch.setattr(subprocess, "Popen", Done)
    monkeypatch.setattr(subprocess, "run", lambda cmd, check: ran.append(cmd))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setenv("SALS_EXTRA_FLAGS", "-DONE=1 -Wl,-z,now -lm")
    build.build()
    compiled, linked = [c for c in ran if "-c" in c], [c for c in ran if "-c" not in c]
    assert len(compiled) == len(build.sources()) and len(linked) == 1
    for cmd in compiled + linked:
        assert all(f in cmd for f in ("-DONE=1", "-Wl,-z,now", "-lm", "--offload-arch=gfx950")), cmd
    objects = [c[c.index("-o") + 1] for c in compiled]
    assert all(o in linked[0] for o in objects) and "-shared" in linked[0] and linked[0][linked[0].index("-o") + 1] == build.LIB
    # (a library is looked up for the objects in front of it)
    assert linked[0].index("-lm") > max(linked[0].index(o) for o in objects)
